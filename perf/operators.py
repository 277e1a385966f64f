"""The chunk attention over paged caches and the 8-bit cache it reads, as cases to time and to compare.

A case is a dict of plain values.  `stage` names what a pass does:

  chunk     stage 2 for several new tokens per question: every new token attends the sink, the question's selected
            groups and its own keys up to itself, the own keys (older ones and the new tokens') lying in pages
            (dbsa_chunk_attn, or dbsa_chunk_attn_kv8 where pool and pages are 8-bit floats)
  quantise  a pool, or a group that joins one, becomes 8-bit floats: one scale per KV head from the rotated keys and
            from the values, then every row rotated, divided and written (dbsa_kv8_scales, dbsa_kv8_write)
  append    the new tokens of a batch join their caches in pages, rotated at their ids, with the scales the caches
            have (dbsa_kv8_write at scattered rows)
  read      rows of an 8-bit cache come back as bf16 or fp32 (dbsa_kv8_read)

Layouts, workspaces, outputs, page tables and rotary tables are made in prepare(): a program keeps them for the layers of
a model.  Where `own` is false the same is computed from elementary operations in 32 bits, with the rows each question
sees as an index list.  Values: N(0, 1), keys scaled per channel by exp(0.5 z), demonstrations of random length, groups
closed at the demonstration boundary next to equal shares: the distributions of the benchmark's synthetic inputs.
"""
import json
import math
import random

import numpy as np
import torch

own = False

ROPE_BASE = 500000.0
E4M3_MAX = 448.0


def listed():
    gqa = {"heads": 32, "kv_heads": 8, "dim": 128, "sink": 64}
    pool90 = {"pool": 90112, "groups": 22, "demo_lo": 32, "demo_hi": 256}
    pool30 = {"pool": 32768, "groups": 8, "demo_lo": 32, "demo_hi": 128}
    return [
        # one token of one question over a small pool: what a launch costs
        dict(gqa, name="chunk_one_token", stage="chunk", dtype="bf16", pool=2048, groups=4, demo_lo=32, demo_hi=128, ratio=0.5,
             queries=1, chunk=1, past=40, page=16, ragged=False),
        # a few proposed tokens of each of 16 questions are checked in one pass
        dict(gqa, name="chunk_check_b16", stage="chunk", dtype="bf16", **pool90, ratio=0.3, queries=16, chunk=8, past=500, page=64,
             ragged=True),
        # the same of a large batch, everything cached in 8 bits
        dict(gqa, name="chunk_check_kv8_b128", stage="chunk", dtype="kv8", **pool90, ratio=0.3, queries=128, chunk=4, past=200,
             page=32, ragged=False),
        # follow-up turns of 12 conversations, lengths all different
        dict(gqa, name="chunk_turn_b12", stage="chunk", dtype="bf16", **pool90, ratio=0.3, queries=12, chunk=229, past=900, page=128,
             ragged=True),
        # a long document behind the demonstrations, one piece of its prefill: the largest call
        dict(gqa, name="chunk_document", stage="chunk", dtype="bf16", **pool90, ratio=0.3, queries=1, chunk=2048, past=30000, page=256,
             ragged=False),
        # prompts of a multi-head model with 64 channels over an 8-bit pool
        dict(name="chunk_mha_d64_kv8", stage="chunk", dtype="kv8", heads=16, kv_heads=16, dim=64, sink=333, **pool30, ratio=0.5,
             queries=6, chunk=150, past=77, page=64, ragged=True),
        # fp32 throughout, three query heads to a KV head
        dict(name="chunk_f32", stage="chunk", dtype="f32", heads=12, kv_heads=4, dim=128, sink=4, pool=4096, groups=5, demo_lo=16,
             demo_hi=48, ratio=0.5, queries=3, chunk=33, past=100, page=16, ragged=True),
        # set-up of a 90k-token pool in 8 bits
        dict(name="quantise_pool", stage="quantise", dtype="bf16", kv_heads=8, dim=128, tokens=90176, first=0),
        # one group of 50 demonstrations, computed in fp32
        dict(name="quantise_group_f32", stage="quantise", dtype="f32", kv_heads=8, dim=128, tokens=1923, first=40000),
        # the new token of each of 16 questions joins its cache
        dict(name="append_b16", stage="append", dtype="bf16", kv_heads=8, dim=128, tokens=16, rows=8192),
        # the groups a question selected, back in bf16
        dict(name="read_selected", stage="read", dtype="bf16", kv_heads=8, dim=128, tokens=27100, rows=90176),
        # a small model's group, back in fp32
        dict(name="read_group_d64", stage="read", dtype="f32", kv_heads=16, dim=64, tokens=1100, rows=16384),
    ]


def draw(rng):
    while True:
        c = _draw(rng)
        if c["stage"] != "chunk":
            return c
        # none larger than the largest listed one, for the kernels (fp32 at a sixteenth of the rate) and for the
        # plain form with its padding
        w = work(c)
        keys = c["sink"] + _selected(c) * (c["pool"] / c["groups"] + c["demo_hi"]) + c["past"] + c["chunk"] + c["page"]
        if (w["flops"] < (1.2e11 if c["dtype"] == "f32" else 1.9e12) and c["queries"] * c["chunk"] * c["heads"] * keys < 3.6e9 and
                c["queries"] * keys * c["kv_heads"] * c["dim"] < 3.6e9):
            return c


def _draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    stage = rng.choice(["chunk"] * 7 + ["quantise", "append", "read", "read"])
    if stage != "chunk":
        kv_heads, dim = rng.choice([(8, 128)] * 3 + [(4, 128), (32, 128), (8, 64), (16, 64), (1, 128), (5, 64)])
        c = {"stage": stage, "dtype": rng.choice(["bf16", "bf16", "f32"]), "kv_heads": kv_heads, "dim": dim}
        top = 90176 if kv_heads <= 8 else 32768
        if stage == "quantise":
            return dict(c, tokens=log_int(1, top), first=rng.choice([0, rng.randint(1, 60000)]))
        tokens = log_int(1, 2048 if stage == "append" else top // 2)
        return dict(c, tokens=tokens, rows=tokens + log_int(16, 20000))
    heads, kv_heads, dim = rng.choice([(32, 8, 128)] * 5 + [(32, 32, 128)] * 2 +
                                      [(32, 4, 128), (12, 4, 128), (40, 8, 128), (32, 8, 64), (16, 16, 64), (10, 2, 64)])
    dtype = rng.choice(["bf16"] * 4 + ["kv8"] * 3 + ["f32"])
    top = 8192 if dtype == "f32" else 90112 if (heads, kv_heads, dim) == (32, 8, 128) else 32768
    pool = log_int(1024, top)
    queries = log_int(1, 128)
    return {"stage": "chunk", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "dim": dim, "sink": rng.choice([0, 4, 64, 64, 333]),
            "pool": pool, "groups": max(2, pool // log_int(500, 4800)), "demo_lo": rng.choice([28, 32]),
            "demo_hi": rng.choice([47, 128, 256]), "ratio": rng.choice([0.1, 0.3, 0.3, 0.5, 1.0]), "queries": queries,
            "chunk": log_int(1, 200 if dtype == "f32" else 2048 if queries <= 4 else 300), "past": log_int(1, 30000) - 1,
            "page": rng.choice([16, 16, 32, 64, 128, 256, 1024]), "ragged": rng.random() < 0.5}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------


def _selected(case):
    return max(1, int(math.floor(case["ratio"] * case["groups"] + 0.5)))


def _structure(case, seed):
    """Offsets of the demonstrations and of the groups, new and older own tokens of each question, selected groups.
    Lengths belong to the case, selections to the seed."""
    rnd = random.Random(json.dumps({x: case[x] for x in sorted(case) if x != "name"}))
    lens, total, lo, hi = [], 0, case["demo_lo"], case["demo_hi"]
    while total < case["pool"]:
        lens.append(rnd.randint(lo, hi))
        total += lens[-1]
    lens[-1] -= total - case["pool"]
    demos = case["sink"] + np.concatenate([[0], np.cumsum(lens)])
    starts = [0]
    for g in range(1, case["groups"]):
        want = case["sink"] + g * case["pool"] / case["groups"]
        starts.append(max(starts[-1] + 1, int(np.argmin(np.abs(demos - want)))))
    starts.append(len(lens))
    s = {"demos": demos.astype(np.int32), "starts": np.asarray(starts, np.int32), "n": int(demos[-1])}
    s["bounds"] = [int(x) for x in s["demos"][s["starts"]]]

    def length(top):
        return rnd.randint((top + 1) // 2, top) if case["ragged"] else top

    s["new"] = [length(case["chunk"]) for _ in range(case["queries"])]
    s["own"] = [length(case["past"]) + t for t in s["new"]]
    s["cu"] = np.concatenate([[0], np.cumsum(s["new"])]).astype(np.int32)
    rnd = random.Random(1000003 * seed + 17)
    s["sel"] = [sorted(rnd.sample(range(case["groups"]), _selected(case))) for _ in s["new"]]
    return s


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _as_8bit(x):
    """One scale per KV head, the largest value at the top of the format."""
    scale = (x.float().abs().amax(dim=tuple(i for i in range(x.dim()) if i != x.dim() - 2)) / E4M3_MAX).clamp_min(1e-12)
    return (x.float() / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn), scale.contiguous()


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed + 7)
    h, d, dtype = case["kv_heads"], case["dim"], _dtype(case)
    spread = torch.exp(0.5 * torch.randn((1, h, d), generator=gen, device="cuda"))

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    def keys(n):
        return (torch.randn((n, h, d), generator=gen, device="cuda") * spread).to(dtype)

    if case["stage"] != "chunk":
        n = case["tokens"]
        t = {}
        if case["stage"] != "read":
            t.update(k=keys(n), v=normal(n, h, d))
        if case["stage"] != "quantise":
            t["k8"], t["k_scale"] = _as_8bit(keys(case["rows"]))
            t["v8"], t["v_scale"] = _as_8bit(normal(case["rows"], h, d))
            t["rows"] = torch.randperm(case["rows"], generator=gen, device="cuda")[:n].to(torch.int32)
        if case["stage"] == "append":  # ids the new tokens' keys are rotated at
            t["ids"] = torch.randint(0, case["rows"], (n,), generator=gen, device="cuda", dtype=torch.int32)
        return None, t
    s = _structure(case, seed)
    page, b = case["page"], case["queries"]
    used = [-(-n // page) for n in s["own"]]
    total = sum(used) + 3  # pages of questions that are not in this batch
    place = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.zeros((b, max(used)), dtype=torch.int32, device="cuda")
    at = 0
    for u, m in enumerate(used):
        table[u, :m] = place[at:at + m]
        at += m
    t = {"q": normal(int(s["cu"][-1]), case["heads"], d), "k": keys(s["n"]), "v": normal(s["n"], h, d),
         "k_pages": keys(total * page).view(total, page, h, d), "v_pages": normal(total, page, h, d), "table": table,
         "self_len": torch.tensor(s["own"], dtype=torch.int32, device="cuda")}
    if case["dtype"] == "kv8":  # pool and pages are one cache: the same scales
        for x in ("k", "v"):
            both, t[x + "_scale"] = _as_8bit(torch.cat([t[x], t[x + "_pages"].view(-1, h, d)]))
            t[x], t[x + "_pages"] = both[:s["n"]].clone(), both[s["n"]:].clone().view(total, page, h, d)
    return s, t


def _rope_table(n, d):
    """[n, D/2, 2] of (cos, sin)(id * frequency), fp32 from fp64 angles."""
    freq = torch.as_tensor(ROPE_BASE ** (-np.arange(0, d, 2, dtype=np.float64) / d), device="cuda")
    angle = torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([torch.cos(angle), torch.sin(angle)], dim=2).float().contiguous()


def _seen_rows(s):
    """Pool rows each question sees, padded with -1 to one length; new tokens of each question, likewise."""
    b = s["bounds"]
    seen = [np.concatenate([np.arange(b[0])] + [np.arange(b[g], b[g + 1]) for g in sel]) for sel in s["sel"]]
    new = [np.arange(s["cu"][u], s["cu"][u + 1]) for u in range(len(s["sel"]))]

    def padded(lists):
        out = np.full((len(lists), max(len(x) for x in lists)), -1, np.int64)
        for u, x in enumerate(lists):
            out[u, :len(x)] = x
        return torch.from_numpy(out).cuda()

    return padded(seen), padded(new)


def prepare(case, seed):
    s, t = _inputs(case, seed)
    state = dict(t, case=case)
    h, d = case["kv_heads"], case["dim"]
    if case["stage"] == "quantise":
        state["table"] = _rope_table(case["first"] + case["tokens"], d)
        for x in ("k8", "v8"):
            state[x] = torch.zeros((case["tokens"], h, d), device="cuda", dtype=torch.float8_e4m3fn)
        for x in ("k_scale", "v_scale"):
            state[x] = torch.zeros(h, device="cuda", dtype=torch.float32)
    if case["stage"] == "append":
        state["table"] = _rope_table(case["rows"], d)
    if case["stage"] == "read":
        for x in ("k_out", "v_out"):
            state[x] = torch.empty((case["tokens"], h, d), device="cuda", dtype=_dtype(case))
    if case["stage"] == "chunk":
        state["scale"] = 1.0 / math.sqrt(d)
        state["o"] = torch.empty_like(t["q"])
        if own:
            from paper_2503_08640_amd import binding as B
            state["layout"] = B.dbsa_layout_build_chunk(
                case["sink"], s["demos"], s["starts"], cu_qlens=s["cu"], sel_ptr=np.cumsum([0] + [len(x) for x in s["sel"]]),
                sel_idx=[g for x in s["sel"] for g in x], n_q_heads=case["heads"], n_kv_heads=h, own_tokens=s["own"])
            need = state["layout"].workspace_bytes(case["heads"], d)
            state["workspace"] = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
        else:
            state["seen"], state["new"] = _seen_rows(s)
    return state


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_2503_08640_amd import binding as B
    stage = s["case"]["stage"]
    if stage == "chunk":
        args = (s["layout"], s["q"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["self_len"])
        if s["case"]["dtype"] == "kv8":
            return {"o": B.dbsa_chunk_attn_kv8(*args, s["k_scale"], s["v_scale"], s["scale"], out=s["o"], workspace=s["workspace"])}
        return {"o": B.dbsa_chunk_attn(*args, s["scale"], out=s["o"], workspace=s["workspace"])}
    if stage == "quantise":
        first = s["case"]["first"]
        B.dbsa_kv8_scales(s["k"], s["v"], table=s["table"], first_id=first, k_scale=s["k_scale"], v_scale=s["v_scale"])
        B.dbsa_kv8_write(s["k"], s["v"], s["k8"], s["v8"], s["k_scale"], s["v_scale"], first_row=0, table=s["table"], first_id=first)
        return {x: s[x] for x in ("k8", "v8", "k_scale", "v_scale")}
    if stage == "append":
        B.dbsa_kv8_write(s["k"], s["v"], s["k8"], s["v8"], s["k_scale"], s["v_scale"], rows=s["rows"], table=s["table"],
                         positions=s["ids"])
        return {"k8": s["k8"], "v8": s["v8"]}
    k, v = B.dbsa_kv8_read(s["k8"], s["v8"], s["k_scale"], s["v_scale"], rows=s["rows"], k_out=s["k_out"], v_out=s["v_out"])
    return {"k": k, "v": v}


def _plain_rotate(x, pairs):
    """x [T, H, D] in fp32 by the table rows [T, D/2, 2]; channel i pairs with channel i + D/2."""
    c, s = pairs[:, None, :, 0], pairs[:, None, :, 1]
    lo, hi = x.chunk(2, dim=2)
    return torch.cat([lo * c - hi * s, hi * c + lo * s], dim=2)


def _plain_8bit(x, scale):
    return (x / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)


def _plain(s):
    case = s["case"]
    if case["stage"] == "chunk":
        s["o"].copy_(_plain_chunk(s))
        return {"o": s["o"]}
    if case["stage"] == "quantise":
        k, v = _plain_rotate(s["k"].float(), s["table"][case["first"]:]), s["v"].float()
        s["k_scale"].copy_(k.abs().amax(dim=(0, 2)) / E4M3_MAX)
        s["v_scale"].copy_(v.abs().amax(dim=(0, 2)) / E4M3_MAX)
        s["k8"].copy_(_plain_8bit(k, s["k_scale"]))
        s["v8"].copy_(_plain_8bit(v, s["v_scale"]))
        return {x: s[x] for x in ("k8", "v8", "k_scale", "v_scale")}
    rows = s["rows"].long()
    if case["stage"] == "append":
        k8 = _plain_8bit(_plain_rotate(s["k"].float(), s["table"][s["ids"].long()]), s["k_scale"])
        s["k8"].view(torch.uint8)[rows] = k8.view(torch.uint8)
        s["v8"].view(torch.uint8)[rows] = _plain_8bit(s["v"].float(), s["v_scale"]).view(torch.uint8)
        return {"k8": s["k8"], "v8": s["v8"]}
    s["k_out"].copy_(s["k8"].view(torch.uint8)[rows].view(torch.float8_e4m3fn).float() * s["k_scale"][:, None])
    s["v_out"].copy_(s["v8"].view(torch.uint8)[rows].view(torch.float8_e4m3fn).float() * s["v_scale"][:, None])
    return {"k": s["k_out"], "v": s["v_out"]}


def _plain_cache(s, x):
    """[B, keys, Hkv, D] in fp32: the pool rows each question sees, then its pages."""
    case = s["case"]
    bits = torch.uint8 if case["dtype"] == "kv8" else s[x].dtype
    pool = s[x].view(bits)[s["seen"].clamp_min(0)]
    pages = s[x + "_pages"].view(bits)[s["table"].long()].flatten(1, 2)
    both = torch.cat([pool, pages], dim=1)
    if case["dtype"] == "kv8":
        return both.view(torch.float8_e4m3fn).float() * s[x + "_scale"][:, None]
    return both.float()


def _plain_chunk(s):
    case, seen, new = s["case"], s["seen"], s["new"]
    b, t, hq, h, d = new.shape[0], new.shape[1], case["heads"], case["kv_heads"], case["dim"]
    r = hq // h
    q = s["q"][new.clamp_min(0)].float().view(b, t, h, r, d).permute(0, 2, 3, 1, 4).reshape(b, h, r * t, d)
    scores = q @ _plain_cache(s, "k").permute(0, 2, 3, 1).contiguous()
    scores *= s["scale"]
    # token a of question u, T_u of its n_u own keys being new, sees own keys 0 .. n_u - T_u + a
    last = (s["self_len"].long() - (new >= 0).sum(1))[:, None] + torch.arange(t, device=new.device)
    keys = torch.arange(scores.shape[3] - seen.shape[1], device=new.device)
    visible = torch.cat([(seen >= 0)[:, None, :].expand(b, t, -1), keys <= last[:, :, None]], dim=2)
    scores = scores.view(b, h, r, t, -1).masked_fill_(~visible[:, None, None], -math.inf)
    scores -= scores.amax(dim=4, keepdim=True)
    scores.exp_()
    total = scores.sum(dim=4)
    o = scores.view(b, h, r * t, -1) @ _plain_cache(s, "v").permute(0, 2, 1, 3).contiguous()
    o = (o.view(b, h, r, t, d) / total[..., None]).permute(0, 3, 1, 2, 4).reshape(b, t, hq, d)
    return o[new >= 0]


# ---------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------------------------------------------


def work(case):
    h, d, es = case["kv_heads"], case["dim"], 4 if case["dtype"] == "f32" else 2
    if case["stage"] != "chunk":
        n = case["tokens"]
        moved = 2 * n * h * d * (1 + es)
        if case["stage"] != "read":
            moved += 4 * n * d  # rows of the rotary table
        return {"bytes": float(moved), "flops": float(2 * n * h * d * (1 if case["stage"] == "read" else 4))}
    s = _structure(case, 1)
    b = s["bounds"]
    union = b[0] + sum(b[g + 1] - b[g] for g in set(g for x in s["sel"] for g in x))
    row = h * d * (1 if case["dtype"] == "kv8" else es)
    pairs = 0
    for t, n, sel in zip(s["new"], s["own"], s["sel"]):
        pairs += t * (b[0] + sum(b[g + 1] - b[g] for g in sel) + n - t) + t * (t + 1) // 2
    moved = 2 * (union + sum(s["own"])) * row + 2 * sum(s["new"]) * case["heads"] * d * es
    return {"bytes": float(moved), "flops": 4.0 * d * case["heads"] * pairs}


# ---------------------------------------------------------------------------------------------------------------
# the same in 64 bits, from the definition
# ---------------------------------------------------------------------------------------------------------------


def _nearest_e4m3(x):
    """Nearest value of the format in 64 bits, ties to the even mantissa: 3 bits behind the leading one, steps of 2^-9
    below 2^-6, at most 448."""
    size = x.abs().clamp_max(E4M3_MAX)
    exponent = torch.floor(torch.log2(size.clamp_min(2.0 ** -6)))
    step = torch.exp2(exponent - 3)
    return torch.sign(x) * torch.round(size / step) * step  # (torch.round takes ties to even)


def _exact_rotate(x, ids, table):
    """By the fp32 table that the call is given."""
    pairs = table[ids].double()
    z = torch.complex(x[..., :x.shape[-1] // 2], x[..., x.shape[-1] // 2:])
    z = z * torch.complex(pairs[..., 0], pairs[..., 1])[:, None]
    return torch.cat([z.real, z.imag], dim=-1)


def exact(case, seed):
    s, t = _inputs(case, seed)
    d = case["dim"]
    if case["stage"] == "quantise":
        ids = torch.arange(case["first"], case["first"] + case["tokens"], device="cuda")
        k, v = _exact_rotate(t["k"].double(), ids, _rope_table(int(ids[-1]) + 1, d)), t["v"].double()
        k_scale, v_scale = (x.abs().amax(dim=(0, 2)) / E4M3_MAX for x in (k, v))
        # (rows are divided by the scale as it is held)
        k8, v8 = (_nearest_e4m3(x / y.float().double()[:, None]) for x, y in ((k, k_scale), (v, v_scale)))
        return {"k8": k8, "v8": v8, "k_scale": k_scale, "v_scale": v_scale}
    if case["stage"] == "append":
        k8, v8, rows = t["k8"].float().double(), t["v8"].float().double(), t["rows"].long()
        k = _exact_rotate(t["k"].double(), t["ids"].long(), _rope_table(case["rows"], d))
        k8[rows] = _nearest_e4m3(k / t["k_scale"].double()[:, None])
        v8[rows] = _nearest_e4m3(t["v"].double() / t["v_scale"].double()[:, None])
        return {"k8": k8, "v8": v8}
    if case["stage"] == "read":
        rows = t["rows"].long()
        return {x: t[x + "8"].float().double()[rows] * t[x + "_scale"].double()[:, None] for x in ("k", "v")}
    hq, h, scale, page = case["heads"], case["kv_heads"], 1.0 / math.sqrt(d), case["page"]
    r, b, out = hq // h, s["bounds"], []
    for u, sel in enumerate(s["sel"]):
        n, lo, hi = s["own"][u], int(s["cu"][u]), int(s["cu"][u + 1])
        key = torch.arange(n, device="cuda")
        row = t["table"][u].long()[key // page] * page + key % page
        cache = {}
        for x in ("k", "v"):
            parts = [t[x][:b[0]]] + [t[x][b[g]:b[g + 1]] for g in sel] + [t[x + "_pages"].view(-1, h, d).view(
                torch.uint8 if case["dtype"] == "kv8" else t[x].dtype)[row].view(t[x].dtype)]
            cache[x] = torch.cat([y.float().double() for y in parts])
            if case["dtype"] == "kv8":
                cache[x] = cache[x] * t[x + "_scale"].double()[:, None]
        before = cache["k"].shape[0] - (hi - lo)
        place = torch.arange(cache["k"].shape[0], device="cuda")
        hidden = place[None, :] > before + torch.arange(hi - lo, device="cuda")[:, None]
        q, o = t["q"][lo:hi].double(), torch.empty((hi - lo, hq, d), dtype=torch.float64, device="cuda")
        for head in range(hq):
            w = scale * (q[:, head].contiguous() @ cache["k"][:, head // r].t().contiguous())
            o[:, head] = torch.softmax(w.masked_fill_(hidden, -math.inf), 1) @ cache["v"][:, head // r].contiguous()
        out.append(o)
    return {"o": torch.cat(out)}
