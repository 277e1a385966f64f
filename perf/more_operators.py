"""What stands around the chunk attention over paged caches: which proposed tokens stay, and which pages hold their keys.

A case is a dict of plain values.  `stage` names what a pass does:

  verify    the proposed tokens of a batch against the target's distributions, from given random numbers: how many of each
            question's stand, and the token behind them (dbsa_draft_verify)
  fork      rows of a page table become copies of others that share their pages: answers that branch, a beam that is
            reordered (dbsa_pages_fork)
  reserve   room for new tokens: pages from the free ones, a shared last page replaced by a copy of its rows in all layers
            (dbsa_pages_reserve, dbsa_pages_copy)
  trim      pages behind the tokens that stayed go back (dbsa_pages_trim)
  compact   the pages in use move to the front of the arena, in all layers (dbsa_pages_compact, dbsa_pages_copy)

Workspaces, result tensors, caches and tables are made in prepare(): a program keeps them from step to step.  The calls on
pages change table, counts and lengths in place; these three lie in one buffer, which a pass takes from the copy that
the state keeps, so that each pass does the same.  Where `own` is false the same is computed from elementary operations,
the distributions in 64 bits (the choice of a token lies next to a border when the vocabulary is large).
"""
import json
import math
import random

import torch

own = False


def listed():
    cache = {"heads": 8, "dim": 128, "dtype": "bf16"}
    return [
        # four proposed tokens of one conversation: what the launches cost
        {"name": "verify_one", "stage": "verify", "form": "logits", "dtype": "bf16", "queries": 1, "chunk": 5, "vocab": 32000,
         "draft": True, "temperature": "one", "ragged": False, "padded": False},
        # a batch of 128, three proposals of a small model each, logits in fp32: the largest
        {"name": "verify_b128", "stage": "verify", "form": "logits", "dtype": "f32", "queries": 128, "chunk": 4, "vocab": 128256,
         "draft": True, "temperature": "mixed", "ragged": False, "padded": False},
        # proposals looked up in the prompt: no distribution behind them, as many as were found
        {"name": "verify_lookup_b16", "stage": "verify", "form": "logits", "dtype": "bf16", "queries": 16, "chunk": 8, "vocab": 50257,
         "draft": False, "temperature": "mixed", "ragged": True, "padded": False},
        # probabilities that the program has filtered itself
        {"name": "verify_probs_b64", "stage": "verify", "form": "probs", "dtype": "f32", "queries": 64, "chunk": 6, "vocab": 102400,
         "draft": True, "temperature": "one", "ragged": False, "padded": True},
        # one prompt's caches become eight answers
        {"name": "fork_answers", "stage": "fork", "queries": 8, "columns": 64, "past": 900, "page": 16, "forked": 0.9, "pages": 2048,
         "ragged": False},
        # a beam over long caches is reordered
        {"name": "fork_beams", "stage": "fork", "queries": 512, "columns": 1024, "past": 8000, "page": 16, "forked": 0.5,
         "pages": 262144, "ragged": True},
        # 64 branches of 16 questions each get a token: 48 last pages are copied in 16 layers
        dict(cache, name="reserve_branches", stage="reserve", layers=16, queries=64, columns=32, past=500, page=64, branch=4, add=8,
             pages=512, ragged=True),
        # the prompts of a batch come in, nothing is shared
        dict(cache, name="reserve_prompts", stage="reserve", layers=0, queries=128, columns=512, past=1, page=16, branch=1, add=900,
             pages=32768, ragged=True),
        # what a check of proposals left over
        {"name": "trim_step", "stage": "trim", "queries": 16, "columns": 256, "past": 1500, "page": 16, "extra": 1, "ended": 0.0,
         "pages": 4096, "ragged": True},
        # a large batch with long caches, a fifth of it finished
        {"name": "trim_batch", "stage": "trim", "queries": 512, "columns": 2048, "past": 16000, "page": 16, "extra": 4, "ended": 0.2,
         "pages": 524288, "ragged": True},
        # a small arena in 8 bits
        dict(cache, name="compact_small", stage="compact", dtype="e4m3", layers=4, queries=12, columns=16, page=32, pages=160, used=0.6),
        # an arena of 8 layers, half of it free: a quarter of its pages move
        dict(cache, name="compact_arena", stage="compact", layers=8, queries=128, columns=64, page=64, pages=1024, used=0.5),
    ]


def draw(rng):
    while True:
        c = _draw(rng)
        # none larger than the largest listed ones
        if c["stage"] == "verify" and c["queries"] * c["chunk"] * c["vocab"] * _SIZE[c["dtype"]] <= 2.6e8:
            return c
        if c["stage"] in ("fork", "trim"):
            return c
        if c["stage"] in ("reserve", "compact") and c["layers"] * c["pages"] * _page_bytes(c) <= 1.08e9:
            return c


def _draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    stage = rng.choice(["verify"] * 4 + ["fork", "reserve", "reserve", "trim", "compact", "compact"])
    if stage == "verify":
        form = rng.choice(["logits", "logits", "probs"])
        return {"stage": stage, "form": form, "dtype": rng.choice(["bf16", "f32"]), "queries": log_int(1, 128), "chunk": log_int(1, 12),
                "vocab": log_int(1000, 152064), "draft": rng.random() < 0.7,
                "temperature": "one" if form == "probs" else rng.choice(["one", "mixed", "greedy"]), "ragged": rng.random() < 0.5,
                "padded": rng.random() < 0.3}
    page = rng.choice([16, 16, 32, 64, 128])
    if stage == "compact":
        heads, dim = rng.choice([(8, 128), (8, 128), (1, 128), (4, 64), (5, 64)])
        pages = log_int(8, 4096)
        return {"stage": stage, "heads": heads, "dim": dim, "dtype": rng.choice(["bf16", "f32", "e4m3"]), "layers": rng.randint(1, 16),
                "queries": log_int(1, 256), "columns": log_int(1, 300), "page": page, "pages": pages,
                "used": round(rng.uniform(0.05, 0.95), 3)}
    queries, columns = log_int(1, 512), log_int(2, 1024)
    past = log_int(1, max(1, page * columns // 2))
    held = queries * (columns + 1)  # most pages that are in use or asked for
    c = {"stage": stage, "queries": queries, "columns": columns, "past": past, "page": page, "pages": held + log_int(1, 5000),
         "ragged": rng.random() < 0.5}
    if stage == "fork":
        return dict(c, forked=round(rng.random(), 3))
    if stage == "trim":
        return dict(c, extra=log_int(1, max(1, columns // 2)), ended=rng.choice([0.0, 0.2, 0.6]))
    heads, dim = rng.choice([(8, 128), (8, 128), (1, 128), (4, 64), (5, 64)])
    add = log_int(1, max(1, page * columns - past))
    branch, held = rng.choice([1, 2, 4, 8]), -(-past // page)
    asked = queries * (-(-(past + add) // page) - held + 1)
    return dict(c, heads=heads, dim=dim, dtype=rng.choice(["bf16", "f32", "e4m3"]), layers=rng.choice([0, 1, 2, 8]), branch=branch, add=add,
                # now and then there are fewer free ones than asked for
                pages=-(-queries // branch) * held + max(1, int(asked * rng.uniform(0.4, 1.5))))


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

_SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}


def _page_bytes(case):
    return case["page"] * case["heads"] * case["dim"] * _SIZE[case["dtype"]]


def _rnd(case):
    """Lengths belong to the case."""
    return random.Random(json.dumps({x: case[x] for x in sorted(case) if x != "name"}))


def _length(rnd, top, ragged):
    return rnd.randint((top + 1) // 2, top) if ragged else top


def _rows_of(case):
    """New tokens of each question."""
    rnd = _rnd(case)
    return [_length(rnd, case["chunk"], case["ragged"]) for _ in range(case["queries"])]


def _verify_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed + 7)
    rows, v, b = _rows_of(case), case["vocab"], case["queries"]
    cu = torch.tensor([0] + rows, device="cuda").cumsum(0)
    n, k = int(cu[-1]), max(rows) - 1
    dtype = _TYPE[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def rand(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    # a few likely tokens in front of a long tail; the small model is near to the large one
    logits = 2.0 * randn(n, v) + 9.0 * (rand(n, v) < 4.0 / v)
    t = {"cu": cu.to(torch.int32), "uniform": rand(n), "tokens": torch.randint(0, v, (n,), generator=gen, device="cuda", dtype=torch.int32)}
    temperature = torch.ones(b, device="cuda")
    if case["temperature"] == "mixed":
        temperature = torch.tensor([0.0, 0.6, 1.0, 1.3], device="cuda")[torch.randint(0, 4, (b,), generator=gen, device="cuda")]
    if case["temperature"] == "greedy":
        temperature = torch.zeros(b, device="cuda")
    t["temperature"] = temperature if case["form"] == "logits" and case["temperature"] != "one" else None
    if k > 0:
        of = torch.repeat_interleave(torch.arange(b, device="cuda"), torch.tensor(rows, device="cuda"))
        step = torch.arange(n, device="cuda") - cu[of]
        last = step == torch.tensor(rows, device="cuda")[of] - 1
        near = logits + 0.7 * randn(n, v)
        # what the small model proposes comes from its own distribution; what was looked up is often the likeliest
        cut = (temperature[of] > 0).float()[:, None]
        noise = cut * -torch.log(-torch.log(rand(n, v).clamp(1e-9, 1 - 1e-7))) * temperature[of].clamp_min(0.1)[:, None]
        pick = (near + (noise if case["draft"] else 0)).argmax(1).to(torch.int32)
        if case["padded"]:  # fewer proposals than the chunk has room for
            pick = torch.where(rand(n) < 0.15, torch.full_like(pick, -1), pick)
        at = torch.nonzero(~last).flatten()
        t["tokens"][at + 1] = pick[at]
        if case["draft"]:
            t["draft"] = torch.zeros((b, k, v), device="cuda", dtype=dtype)
            kept = near[at] if case["form"] == "logits" else _filtered(near[at])
            t["draft"][of[at], step[at]] = kept.to(dtype)
    t["target"] = (logits if case["form"] == "logits" else _filtered(logits)).to(dtype)
    t["self_len"] = torch.randint(0, 5000, (b,), generator=gen, device="cuda", dtype=torch.int32) + torch.tensor(rows, device="cuda", dtype=torch.int32)
    return t


def _filtered(x):
    """Probabilities of what lies within 6 of the likeliest token."""
    top = x.amax(1, keepdim=True)
    return torch.softmax(x.masked_fill(x < top - 6.0, -math.inf), 1)


def _pages_of(case, tokens):
    return -(-tokens // case["page"])


def _plan(case):
    """What belongs to the case: own tokens of each row, pages each row names, for reserve the row whose pages it shares."""
    rnd, b, most = _rnd(case), case["queries"], case["columns"] * case["page"]
    if case["stage"] == "compact":
        return None, [rnd.randint(0, case["columns"]) for _ in range(b)], list(range(b))
    past = [min(_length(rnd, case["past"], case["ragged"]), most) for _ in range(b)]
    parent = list(range(b))
    if case["stage"] == "reserve":
        parent = [u - u % case["branch"] for u in range(b)]
        past = [past[p] for p in parent]
    named = [_pages_of(case, x) for x in past]
    if case["stage"] == "trim":  # pages behind the tokens that stay, all of them where a question has ended
        named = [min(case["columns"], x + case["extra"]) for x in named]
        past = [0 if rnd.random() < case["ended"] else x for x in past]
    return past, named, parent


def _book(case, seed):
    """(one buffer, {refs, table, self_len} as views of it): pages lie anywhere in the arena."""
    b, c, p = case["queries"], case["columns"], case["pages"]
    gen = torch.Generator(device="cuda").manual_seed(seed + 11)
    past, named, parent = _plan(case)
    width = -(-p // 64) * 64
    book = torch.zeros(width + b * c + b, dtype=torch.int32, device="cuda")
    v = _views(book, case)
    place = torch.randperm(p, generator=gen, device="cuda").to(torch.int32)
    if case["stage"] == "compact":  # the rows name pages out of those in use, some of them shared
        live = place[:max(1, int(case["used"] * p))]
        table = live[torch.randint(0, live.numel(), (b, c), generator=gen, device="cuda")]
        v["refs"][live.long()] = 1  # (tables of other batches name each, too)
    else:
        mine = torch.tensor([0 if parent[u] != u else named[u] for u in range(b)], device="cuda")
        first = (torch.cumsum(mine, 0) - mine)[torch.tensor(parent, device="cuda")]
        table = place[(first[:, None] + torch.arange(c, device="cuda")).clamp_max(p - 1)]
        v["self_len"].copy_(torch.tensor(past, device="cuda"))
    there = torch.arange(c, device="cuda") < torch.tensor(named, device="cuda")[:, None]
    v["table"].copy_(torch.where(there, table, torch.full_like(table, -1)))
    v["refs"].index_add_(0, table[there].long(), torch.ones_like(table[there]))
    return book, v


def _views(book, case):
    b, c, p = case["queries"], case["columns"], case["pages"]
    width = -(-p // 64) * 64
    return {"refs": book[:p], "table": book[width:width + b * c].view(b, c), "self_len": book[width + b * c:]}


def _cache(case, seed):
    """[layers, pages, page tokens, heads, D]: any finite values of the type."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shape = (case["layers"], case["pages"], case["page"], case["heads"], case["dim"])
    if case["dtype"] != "e4m3":
        return torch.randn(shape, generator=gen, device="cuda", dtype=_TYPE[case["dtype"]])
    return torch.randint(0, 127, shape, generator=gen, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)


def prepare(case, seed):
    state = {"case": case}
    if case["stage"] == "verify":
        t = _verify_inputs(case, seed)
        n, b = t["tokens"].numel(), case["queries"]
        state.update(t)
        for x, m, dtype in (("out", n, torch.int32), ("accepted", b, torch.int32), ("logp", n, torch.float32), ("new_len", b, torch.int32)):
            state[x] = torch.empty(m, dtype=dtype, device="cuda")
        if own:
            from paper_2503_08640_amd import binding as B
            need = B.dbsa_draft_verify_workspace_bytes(n, b, case["vocab"])
            state["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
        return state
    b, p = case["queries"], case["pages"]
    state["book0"], state["old"] = _book(case, seed)
    state["book"] = state["book0"].clone()
    state["now"] = _views(state["book"], case)
    if case["stage"] == "fork":
        gen = torch.Generator(device="cuda").manual_seed(seed + 13)
        other = torch.randint(0, b, (b,), generator=gen, device="cuda", dtype=torch.int32)
        stays = torch.rand(b, generator=gen, device="cuda") >= case["forked"]
        state["source"] = torch.where(stays, torch.arange(b, device="cuda", dtype=torch.int32), other)
    if case["stage"] == "reserve":
        rnd = _rnd(case)
        state["add"] = torch.tensor([_length(rnd, case["add"], case["ragged"]) for _ in range(b)], dtype=torch.int32, device="cuda")
        state["got"] = torch.zeros(b, dtype=torch.int32, device="cuda")
    if case["stage"] in ("reserve", "compact"):
        state["copies"] = torch.zeros((b if case["stage"] == "reserve" else max(1, p // 2), 3), dtype=torch.int32, device="cuda")
        state["n_copies"] = torch.zeros(1 if case["stage"] == "reserve" else 2, dtype=torch.int32, device="cuda")
        state["spare"] = torch.zeros(p, dtype=torch.int32, device="cuda")  # free pages, or where each page went
        if case["layers"]:
            state["k"], state["v"] = _cache(case, seed + 1), _cache(case, seed + 2)
    return state


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_2503_08640_amd import binding as B
    stage = s["case"]["stage"]
    if stage == "verify":
        B.dbsa_draft_verify(s["target"], s["tokens"], s["cu"], s["uniform"], draft=s.get("draft"), temperature=s["temperature"],
                            probs=s["case"]["form"] == "probs", out=s["out"], accepted=s["accepted"], logp=s["logp"],
                            self_len=s["self_len"], new_len=s["new_len"], workspace=s["workspace"])
        return {x: s[x] for x in ("out", "accepted", "logp", "new_len")}
    s["book"].copy_(s["book0"])
    now, page = s["now"], s["case"]["page"]
    if stage == "fork":
        B.dbsa_pages_fork(now["table"], now["refs"], now["self_len"], s["source"], page)
        return dict(now)
    if stage == "trim":
        B.dbsa_pages_trim(now["table"], now["refs"], now["self_len"], page)
        return dict(now)
    if stage == "reserve":
        B.dbsa_pages_reserve(now["table"], now["refs"], now["self_len"], s["add"], page, got=s["got"], copies=s["copies"],
                             n_copies=s["n_copies"], workspace=s["spare"])
    else:
        B.dbsa_pages_compact(now["refs"], now["table"], page, copies=s["copies"], counts=s["n_copies"], new_place=s["spare"])
    if s["case"]["layers"]:
        B.dbsa_pages_copy(s["k"], s["v"], s["copies"], s["n_copies"])
    return _moved(s, now)


def _bits(x):
    """Copied elements, as what they are: whole numbers, or the values of 8 bits."""
    return x.view(torch.int16) if x.dtype == torch.bfloat16 else x.view(torch.int32) if x.dtype == torch.float32 else x


def _moved(s, now):
    out = dict(now, copies=s["copies"], n_copies=s["n_copies"])
    if s["case"]["stage"] == "reserve":
        out["got"] = s["got"]
    else:
        out["new_place"] = s["spare"]
    if s["case"]["layers"]:
        out.update(k=_bits(s["k"]), v=_bits(s["v"]))
    return out


def _plain(s):
    stage = s["case"]["stage"]
    if stage == "verify":
        return _plain_verify(s)
    if stage == "fork":
        return _plain_fork(s)
    if stage == "trim":
        return _plain_trim(s)
    return _plain_reserve(s) if stage == "reserve" else _plain_compact(s)


# ---- verification


def _plain_distribution(x, inv, greedy, logits):
    """Rows of scores as probabilities in 64 bits."""
    x = x.double()
    if not logits:
        return x
    top = x.amax(1, keepdim=True)
    e = torch.exp((x - top) * inv[:, None])
    p = e / e.sum(1, keepdim=True)
    place = torch.arange(x.shape[1], device=x.device)
    first = torch.where(x == top, place, x.shape[1]).amin(1)
    return torch.where(greedy[:, None], (place == first[:, None]).double(), p)


def _plain_verify(s):
    case, target, tokens, cu = s["case"], s["target"], s["tokens"].long(), s["cu"].long()
    n, v, b = target.shape[0], target.shape[1], cu.numel() - 1
    logits = case["form"] == "logits"
    row = torch.arange(n, device=target.device)
    of = torch.searchsorted(cu, row, right=True) - 1
    step, last = row - cu[of], row == cu[of + 1] - 1
    heat = s["temperature"].double() if s["temperature"] is not None else torch.ones(b, device=target.device, dtype=torch.float64)
    greedy = heat <= 0
    inv = 1.0 / torch.where(greedy, torch.ones_like(heat), heat)
    p = _plain_distribution(target, inv[of], greedy[of], logits)
    x = torch.cat([tokens[1:], tokens[:1]])  # what row t checks
    there = ~last & (x >= 0) & (x < v)
    x = x.clamp(0, v - 1)
    px = p.gather(1, x[:, None])[:, 0]
    if "draft" in s:
        at = torch.nonzero(~last).flatten()
        q = torch.zeros_like(p)
        q[at] = _plain_distribution(s["draft"][of[at], step[at]], inv[of[at]], greedy[of[at]], logits)
    else:
        q = torch.zeros_like(p).scatter_(1, x[:, None], 1.0)
    qx = q.gather(1, x[:, None])[:, 0]
    stands = there & (s["uniform"].double() * qx < px)
    # the first row of each question whose proposal does not stand
    stop = torch.full((b,), n, device=row.device).scatter_reduce_(0, of, torch.where(stands, n, row), "amin")
    refused = there[stop]  # (a real proposal: what both have in common is taken out)
    w = torch.where(refused[:, None], (p[stop] - q[stop]).clamp_min(0), p[stop])
    w = torch.where(w.sum(1, keepdim=True) > 0, w, p[stop])
    c = w.cumsum(1)
    want = s["uniform"][cu[1:] - 1].double() * c[:, -1]
    place = torch.arange(v, device=row.device)
    token = (c <= want[:, None]).sum(1)
    token = torch.minimum(token, torch.where(w > 0, place, -1).amax(1))
    s["accepted"].copy_(stop - cu[:-1])
    given = torch.where(row < stop[of], x, torch.where(row == stop[of], token[of], -1))
    s["out"].copy_(given)
    plain = _plain_distribution(target, inv[of], torch.zeros_like(greedy)[of], logits)
    logp = torch.log(plain.gather(1, given.clamp_min(0)[:, None])[:, 0])
    s["logp"].copy_(torch.where(given >= 0, logp, 0.0))
    s["new_len"].copy_(s["self_len"] - (cu[1:] - 1 - stop))
    return {x: s[x] for x in ("out", "accepted", "logp", "new_len")}


# ---- pages


def _plain_counts(refs, entries, sign):
    return refs.index_add(0, entries.long(), torch.full_like(entries, sign))


def _plain_fork(s):
    old, case = s["old"], s["case"]
    table, refs, length = old["table"], old["refs"], old["self_len"]
    b, c = table.shape
    row, column = torch.arange(b, device=table.device), torch.arange(c, device=table.device)
    source = s["source"].long()
    forks = (source >= 0) & (source < b) & (source != row)
    source = torch.where(forks, source, row)
    used = (length.clamp(0, c * case["page"]) + case["page"] - 1) // case["page"]
    copied = torch.where(column < used[source][:, None], table[source], -1)
    new = torch.where(forks[:, None], copied, table)
    refs = _plain_counts(refs, table[forks[:, None] & (table >= 0)], -1)
    refs = _plain_counts(refs, new[forks[:, None] & (new >= 0)], 1)
    return {"table": new, "refs": refs, "self_len": length[source]}


def _plain_trim(s):
    old, case = s["old"], s["case"]
    table, length = old["table"], old["self_len"]
    column = torch.arange(table.shape[1], device=table.device)
    keep = (length.clamp_min(0) + case["page"] - 1) // case["page"]
    gone = (column >= keep[:, None]) & (table >= 0)
    return {"table": torch.where(gone, -1, table), "refs": _plain_counts(old["refs"], table[gone], -1), "self_len": length}


def _plain_reserve(s):
    old, case, add = s["old"], s["case"], s["add"].long()
    table, refs, length, page = old["table"], old["refs"], old["self_len"].long(), s["case"]["page"]
    b, c = table.shape
    row, column = torch.arange(b, device=table.device), torch.arange(c, device=table.device)
    fits = (add > 0) & (length + add <= c * page)
    rows = length % page  # of the last page that are in use
    tail = table.gather(1, (length // page).clamp_max(c - 1)[:, None])[:, 0].long()
    fits &= (rows == 0) | (tail >= 0)
    writes = fits & (rows > 0)
    # a page is replaced while more than one names it, counting the replacements of earlier questions
    before = ((tail[:, None] == tail[None, :]) & writes[None, :] & (row[None, :] < row[:, None])).sum(1)
    shared = writes & (refs[tail.clamp_min(0)] - before > 1)
    first, behind = (length + page - 1) // page, (length + add + page - 1) // page
    missing = fits[:, None] & (column >= first[:, None]) & (column < behind[:, None]) & (table < 0)
    ask = missing.sum(1) + shared
    free = torch.nonzero(refs <= 0).flatten()
    total = ask.cumsum(0)
    served = total <= free.numel()
    start = total - ask
    gets, copied = served[:, None] & missing, served & shared
    spare = torch.cat([free, torch.zeros(1, dtype=free.dtype, device=free.device)])  # (none may be free)
    number = (start + shared)[:, None] + missing.cumsum(1) - 1
    new = torch.where(gets, spare[number.clamp(0, free.numel())].int(), table)
    fresh = spare[start.clamp(0, free.numel())].int()
    new = torch.where(copied[:, None] & (column == (length // page)[:, None]), fresh[:, None], new)
    refs = _plain_counts(refs, tail[copied].int(), -1)
    refs = _plain_counts(refs, torch.cat([new[gets], fresh[copied]]), 1)
    list_ = torch.stack([tail, fresh.long(), rows], 1)[copied].int()
    s["copies"].zero_()
    s["copies"][:list_.shape[0]] = list_
    s["n_copies"].copy_(copied.sum())
    s["got"].copy_(torch.where(fits & served, add, 0))
    length = old["self_len"] + s["got"]
    _plain_copy(s, list_)
    return _moved(s, {"table": new, "refs": refs, "self_len": length})


def _plain_compact(s):
    old = s["old"]
    table, refs = old["table"], old["refs"]
    live = refs > 0
    count = int(live.sum())
    place = torch.arange(refs.numel(), device=refs.device, dtype=torch.int32)
    to, come = place[:count][~live[:count]], place[count:][live[count:]]
    where = torch.where(live, place, -1)
    where[come.long()] = to
    new = refs.clone()
    new[to.long()] = refs[come.long()]
    new[come.long()] = 0
    list_ = torch.stack([come, to, torch.full_like(to, s["case"]["page"])], 1)
    s["copies"].zero_()
    s["copies"][:list_.shape[0]] = list_
    s["n_copies"].copy_(torch.tensor([list_.shape[0], count]))
    s["spare"].copy_(where)
    _plain_copy(s, list_)
    return _moved(s, {"table": torch.where(table >= 0, where[table.clamp_min(0).long()], table), "refs": new, "self_len": old["self_len"]})


def _plain_copy(s, list_):
    if not s["case"]["layers"]:
        return
    src, dst, rows = list_.long().unbind(1)
    page = s["case"]["page"]
    kept = (torch.arange(page, device=rows.device) < rows[:, None])[None, :, :, None, None]
    _plain_copy_one(_raw(s["k"]), src, dst, kept)
    _plain_copy_one(_raw(s["v"]), src, dst, kept)


def _raw(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


def _plain_copy_one(x, src, dst, kept):
    x[:, dst] = torch.where(kept, x[:, src], x[:, dst])


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------


def work(case):
    if case["stage"] == "verify":
        rows, size = _rows_of(case), _SIZE[case["dtype"]]
        n, b = sum(rows), case["queries"]
        if case["form"] == "probs":  # one row of each kind decides
            read = b * (1 + (1 if case["draft"] and case["chunk"] > 1 else 0))
            return {"bytes": float(read * case["vocab"] * size + 20 * n), "flops": float(2 * read * case["vocab"])}
        read = n + (n - b if case["draft"] else 0)
        return {"bytes": float(read * case["vocab"] * size + 20 * n), "flops": float(16 * read * case["vocab"])}
    past, named, parent = _plan(case)
    b, page = case["queries"], case["page"]
    if case["stage"] == "fork":  # a row read and a row written, the counts of the pages of both
        moved = case["forked"] * sum(named) * 4 * 6
        return {"bytes": float(moved + 16 * b), "flops": float(moved / 4 + b)}
    if case["stage"] == "trim":
        gone = sum(n - _pages_of(case, x) for n, x in zip(named, past))
        return {"bytes": float(4 * b * (case["columns"] + 1) + 12 * gone), "flops": float(b * case["columns"])}
    if case["stage"] == "compact":
        live = max(1, int(case["used"] * case["pages"]))
        moves = live * (1 - live / case["pages"])
        table = 8 * sum(named) + 12 * case["pages"]
        return {"bytes": float(table + 4 * moves * case["layers"] * _page_bytes(case)), "flops": float(2 * case["pages"])}
    rnd = _rnd(case)
    add = [_length(rnd, case["add"], case["ragged"]) for _ in range(b)]
    asked, copied = 0, 0
    for u in range(b):
        if past[u] + add[u] > case["columns"] * page:
            continue
        asked += _pages_of(case, past[u] + add[u]) - _pages_of(case, past[u])
        if past[u] % page and u + 1 < b and parent[u + 1] == parent[u]:  # all but the last of those that share it
            copied += past[u] % page
    moved = 4 * copied * case["layers"] * _page_bytes(case) / page
    return {"bytes": float(4 * case["pages"] + 16 * b + 8 * asked + moved), "flops": float(case["pages"] + b)}


# ---------------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definition
# ---------------------------------------------------------------------------------------------------------------


def exact(case, seed):
    if case["stage"] != "verify":
        return None  # whole numbers and copied bits
    t = _verify_inputs(case, seed)
    v, cu = case["vocab"], t["cu"].tolist()
    logp = torch.zeros(cu[-1], dtype=torch.float64, device="cuda")
    for u in range(case["queries"]):
        heat = 1.0 if t["temperature"] is None else float(t["temperature"][u])
        ids = t["tokens"][cu[u]:cu[u + 1]].tolist()[1:]

        def scores(x):
            """Natural logarithms of the distribution, and of the one that is drawn from."""
            if case["form"] == "probs":
                return torch.log(x.double()), torch.log(x.double())
            free = torch.log_softmax(x.double() / (heat if heat > 0 else 1.0), 0)
            if heat > 0:
                return free, free
            sure = torch.full_like(free, -math.inf)
            sure[int(torch.nonzero(x == x.max())[0])] = 0.0
            return free, sure

        a = 0
        while True:
            row = cu[u] + a
            free, p = scores(t["target"][row])
            token = ids[a] if a < len(ids) else -1
            if not 0 <= token < v:
                w = p.exp()
                break
            q = torch.full_like(p, -math.inf)
            q[token] = 0.0
            if case["draft"]:
                q = scores(t["draft"][u, a])[1]
            if float(t["uniform"][row]) * math.exp(q[token]) < math.exp(p[token]):
                logp[row] = free[token]
                a += 1
                continue
            w = torch.relu(p.exp() - q.exp())
            if float(w.sum()) == 0:
                w = p.exp()
            break
        c = torch.cumsum(w, 0)
        more = torch.nonzero(c > float(t["uniform"][cu[u + 1] - 1]) * float(c[-1]))
        token = int(more[0]) if len(more) else int(torch.nonzero(w > 0)[-1])
        logp[row] = free[token]
    return {"out": None, "accepted": None, "logp": logp, "new_len": None}
