"""The chunk attention over paged caches against the fp64 oracle, at the shapes, lengths and masks where it can go wrong.

Tolerances.  bf16 and 8-bit caches: the products are exact in fp32, the probabilities are rounded to bf16 once (half a step,
2^-8 of each) before they weigh the values, the output once more; exponentials and sums in fp32 are far below:
|error| <= 2^-8 (sum p |v| + |o|) (1 + 2^-4), and what the scores are off by.  Both types: a score is a sum of D products in
fp32, off by at most e = (D + 2) 2^-24 scale sum |q k|, which counts twice (numerator and denominator).  fp32: an exponential
is off by 2^-22, a sum of n terms by n 2^-24."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle as orc
from paper_2503_08640_amd import binding as B

pytestmark = pytest.mark.gpu

SINK, DEMOS = 70, [60, 33, 91, 128, 7, 200, 64, 130, 19, 55]
KINDS = [("bf16", 8, 2, 128), ("bf16", 4, 4, 128), ("bf16", 10, 2, 128), ("bf16", 32, 1, 128), ("bf16", 6, 2, 64), ("bf16", 16, 16, 64),
         ("f32", 4, 2, 128), ("f32", 3, 3, 64), ("kv8", 8, 2, 128), ("kv8", 3, 1, 128), ("kv8", 12, 4, 64)]
IDS = ["%s-%d-%d-%d" % k for k in KINDS]


def structure(sink=SINK):
    demos = sink + np.concatenate([[0], np.cumsum(DEMOS)])
    return sink, demos, np.arange(0, len(DEMOS) + 1, 2)


class Case:
    """Inputs of one batch: lens new tokens, own keys in all, selected groups, pages in random places."""

    def __init__(self, kind, lens, own, sels, page=16, seed=0, sink=SINK, spread=0.3, extra_rows=0, table_width=None):
        self.dtype, self.hq, self.hkv, self.d = kind
        rng = np.random.default_rng(seed)
        self.pool, self.lens, self.own, self.sels, self.page = structure(sink), list(lens), list(own), sels, page
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        n, t = int(self.pool[1][-1]), int(self.cu[-1])
        width = table_width or max(1, max(-(-x // page) for x in own))
        used = sum(-(-max(x, 0) // page) for x in own)
        total = used + 2
        place = rng.permutation(total)
        self.table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for u, x in enumerate(own):
            m = -(-max(x, 0) // page)
            self.table[u, :m] = place[at:at + m][:width]
            at += m

        def normal(*shape):
            return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).cuda()

        storage = torch.float32 if self.dtype == "f32" else torch.bfloat16
        scale = torch.exp(spread * normal(1, self.hkv, self.d))
        self.q = normal(t + extra_rows, self.hq, self.d).to(storage)[:t]
        self.k, self.v = (normal(n, self.hkv, self.d) * scale).to(storage), normal(n, self.hkv, self.d).to(storage)
        self.kp = (normal(total, page, self.hkv, self.d) * scale).to(storage)
        self.vp = normal(total, page, self.hkv, self.d).to(storage)
        self.ks = self.vs = None
        if self.dtype == "kv8":
            self.ks, self.vs = (0.004 + 0.01 * torch.rand(self.hkv, generator=torch.Generator().manual_seed(seed))).cuda(), None
            self.vs = (self.ks * 0.7 + 0.002).contiguous()
            self.k, self.kp = (self.to8(x, self.ks) for x in (self.k, self.kp))
            self.v, self.vp = (self.to8(x, self.vs) for x in (self.v, self.vp))
        self.scale = 1.0 / np.sqrt(self.d)

    @staticmethod
    def to8(x, scale):
        return (x.float() / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn)

    def layout(self, own="true", **kw):
        return B.dbsa_layout_build_chunk(*self.pool, cu_qlens=self.cu, sel_ptr=np.cumsum([0] + [len(s) for s in self.sels]),
                                         sel_idx=[g for s in self.sels for g in s], n_q_heads=self.hq, n_kv_heads=self.hkv,
                                         own_tokens=[max(x, 0) for x in self.own] if own == "true" else own, **kw)

    def device_tables(self):
        return torch.from_numpy(self.table).cuda(), torch.tensor(self.own, dtype=torch.int32, device="cuda")

    def call(self, layout, tables=None, **kw):
        table, own = tables or self.device_tables()
        if self.dtype == "kv8":
            return B.dbsa_chunk_attn_kv8(layout, self.q, self.k, self.v, self.kp, self.vp, table, own, self.ks, self.vs, self.scale, **kw)
        return B.dbsa_chunk_attn(layout, self.q, self.k, self.v, self.kp, self.vp, table, own, self.scale, **kw)

    def f64(self, x, scale=None):
        x = x.float().double().cpu().numpy()
        return x if scale is None else x * scale.double().cpu().numpy()[:, None]

    def oracle(self):
        return orc.chunk_attn(self.f64(self.q), self.f64(self.k, self.ks), self.f64(self.v, self.vs), self.f64(self.kp, self.ks),
                              self.f64(self.vp, self.vs), self.table, self.own, *self.pool, self.cu,
                              np.cumsum([0] + [len(s) for s in self.sels]), np.array([g for s in self.sels for g in s], np.int64), self.scale)

    def check(self, o, lse=None, want=None, rows=slice(None)):
        want = want or self.oracle()
        keys = np.maximum(want["keys"], 1)[:, None]
        score = (self.d + 2) * 2.0 ** -24 * want["reach"]  # [T, Hq]
        if self.dtype == "f32":
            tol = (2 * score + 2.0 ** -21 + 2 * keys * 2.0 ** -24)[:, :, None] * want["weight"] + 2.0 ** -23 * np.abs(want["o"])
        else:
            tol = 2.0 ** -8 * (want["weight"] + np.abs(want["o"])) * (1 + 2.0 ** -4) + 2 * score[:, :, None] * want["weight"]
        got = self.f64(o)
        assert np.isfinite(got[rows]).all()
        over = (np.abs(got - want["o"]) - tol)[rows]
        assert over.max() <= 0, (over.max(), np.unravel_index(over.argmax(), over.shape))
        if lse is not None:
            got, ref = lse.double().cpu().numpy(), want["lse"]
            empty = np.isinf(ref)
            assert (got[empty] == -np.inf).all()
            tol = 2 * score.T + 2.0 ** -20 + keys.T * 2.0 ** -24 + 2.0 ** -22 * np.abs(np.where(empty, 0, ref))
            assert (np.abs(got[~empty] - ref[~empty]) <= tol[~empty]).all()
        return want


def batches():
    return {
        "mixed": dict(lens=[1, 7, 64, 130, 3], own=[1, 24, 564, 193, 1003], sels=[[3, 0], [], [1], [0, 1, 2, 3, 4], [2]], page=16),
        "one_token_each": dict(lens=[1] * 40, own=list(range(1, 41)), sels=[[u % 5, (u + 2) % 5] for u in range(40)], page=32),
        "few_tokens_shared": dict(lens=[3 + u % 4 for u in range(20)], own=[90 + 13 * u for u in range(20)],
                                  sels=[[u % 5, (u + 1) % 5, (u + 3) % 5][:1 + u % 3] for u in range(20)], page=64),
        "one_long": dict(lens=[300], own=[300], sels=[[4, 2]], page=128),
        "one_token": dict(lens=[1], own=[1], sels=[[]], page=16),
        "long_past": dict(lens=[2, 33], own=[2500, 3001], sels=[[0], [0, 1, 2, 3, 4]], page=256),
        "no_sink": dict(lens=[5, 70], own=[64, 127], sels=[[], [3]], page=64, sink=0),
    }


@pytest.mark.parametrize("batch", sorted(batches()))
@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_against_the_oracle(kind, batch):
    c = Case(kind, seed=len(batch), **batches()[batch])
    lse = torch.full((c.hq, int(c.cu[-1])), 7.0, device="cuda")
    o = c.call(c.layout(), lse=lse)
    c.check(o, lse)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_rows_without_keys_and_left_padding(kind):
    """self_len below the chunk's length: the first tokens have no own keys; with no pool either they give zeros."""
    c = Case(kind, lens=[9, 9, 9, 80], own=[4, 0, 9, 30], sels=[[], [], [], []], sink=0, page=16, seed=3, table_width=8)
    c.own[1] = -5  # (taken as 0)
    lse = torch.zeros((c.hq, int(c.cu[-1])), device="cuda")
    o = c.call(c.layout(own=None), lse=lse)
    want = c.check(o, lse)
    assert (want["keys"][:5] == 0).all() and (want["keys"][9:18] == 0).all() and (want["keys"][5:9] == np.arange(1, 5)).all()
    assert not o[:5].any() and not o[9:18].any() and not o[27:77].any() and (lse[:, :5] == -torch.inf).all()
    # the same rows with a pool see the pool alone
    c = Case(kind, lens=[9, 9, 9, 80], own=[4, 0, 9, 30], sels=[[1], [2], [], [0]], page=16, seed=4, table_width=8)
    c.check(c.call(c.layout(own=None)))


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[6], KINDS[8]], ids=["bf16", "f32", "kv8"])
def test_the_expected_own_tokens_only_balance(kind):
    c = Case(kind, lens=[5, 40, 1], own=[1300, 40, 700], sels=[[0], [1, 2], [0, 4]], page=32, seed=5)
    want = c.oracle()
    for hint in (None, [0, 0, 0], [5, 4000, 1], [20000, 1, 1]):
        c.check(c.call(c.layout(own=hint)), want=want)


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[4], KINDS[6], KINDS[8]], ids=["bf16", "d64", "f32", "kv8"])
def test_pages_that_are_not_there_hide_their_keys(kind):
    """Entries outside the pages are masked; a table row shorter than self_len counts only what it holds."""
    c = Case(kind, lens=[4, 50], own=[200, 300], sels=[[1], []], page=16, seed=6)
    c.table[0, 3], c.table[0, 7], c.table[1, 2], c.table[1, 18] = -1, c.kp.shape[0], 2 ** 31 - 1, -2 ** 31
    lse = torch.zeros((c.hq, int(c.cu[-1])), device="cuda")
    c.check(c.call(c.layout(), lse=lse), lse)
    c.own = [200, 2 ** 30]
    c.check(c.call(c.layout(own=None)))


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_what_no_row_sees_may_hold_anything(kind):
    """NaN and infinities in groups nobody selected, on pages of nobody, behind a question's last key."""
    c = Case(kind, lens=[6, 90], own=[37, 155], sels=[[2, 0], [4]], page=32, seed=7)
    want = c.oracle()
    bounds = c.pool[1][c.pool[2]]
    for x in (c.k, c.v):
        x[bounds[1]:bounds[2]] = torch.nan
        x[bounds[3]:bounds[4]] = torch.nan if c.dtype == "kv8" else torch.inf
    used = set(c.table[c.table >= 0].tolist())
    for x in (c.kp, c.vp):
        for page in range(x.shape[0]):
            if page not in used:
                x[page] = torch.nan
        for u, n in enumerate(c.own):
            x[c.table[u, n // 32], n % 32:] = torch.nan
    c.check(c.call(c.layout()), want=want)


@pytest.mark.parametrize("kind", KINDS, ids=IDS)
def test_non_finite_values_of_later_tokens_do_not_reach_earlier_rows(kind):
    c = Case(kind, lens=[70, 9, 200], own=[170, 9, 203], sels=[[0], [], [1, 3]], page=64, seed=8)
    want = c.oracle()
    first_bad = []
    for u, (j, what) in enumerate([(150, torch.nan), (4, torch.nan if c.dtype == "kv8" else torch.inf), (100, torch.nan)]):
        c.vp[c.table[u, j // 64], j % 64] = what
        if u != 1:  # a key too
            c.kp[c.table[u, j // 64], j % 64, :, 3] = torch.nan
        first_bad.append(int(c.cu[u]) + max(0, j - (c.own[u] - c.lens[u])))
    o = c.call(c.layout())
    rows = np.zeros(int(c.cu[-1]), bool)
    for u in range(3):
        rows[c.cu[u]:first_bad[u]] = True
    assert rows.sum() > 100
    c.check(o, want=want, rows=rows)
    assert not torch.isfinite(o.float()).all(dim=2).all(dim=1).cpu().numpy()[~rows].any()


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[6], KINDS[8]], ids=["bf16", "f32", "kv8"])
def test_large_scores_and_growing_maxima(kind):
    """Scores that rise by hundreds along every segment and along the own keys: the running maximum moves again and again."""
    c = Case(kind, lens=[3, 64], own=[700, 130], sels=[[0, 1, 2], [4, 3]], page=16, seed=9)
    ramp = torch.linspace(0, 1, c.k.shape[0], device="cuda")[:, None, None]
    sign = torch.sign(torch.randn(c.d, generator=torch.Generator().manual_seed(1))).cuda()
    top = 40.0 if c.dtype != "kv8" else 40.0 * 0.004
    unscale = 1.0 if c.dtype != "kv8" else 1.0 / c.ks[:, None]
    c.k = (ramp * sign * top * unscale).clamp(-448, 448).expand(-1, c.hkv, -1).to(c.k.dtype).contiguous()
    j = torch.rand(c.kp.shape[:2], generator=torch.Generator().manual_seed(2)).cuda()[:, :, None, None]
    c.kp = (j * sign * top * unscale).clamp(-448, 448).expand(-1, -1, c.hkv, -1).to(c.kp.dtype).contiguous()
    c.q = (sign + 0.1 * c.q.float()).to(c.q.dtype)
    lse = torch.zeros((c.hq, int(c.cu[-1])), device="cuda")
    c.check(c.call(c.layout(), lse=lse), lse)


def test_scales_of_zero_and_below():
    c = Case(KINDS[10], lens=[5, 70], own=[90, 200], sels=[[0], [1, 2]], page=16, seed=10)
    for ks, vs in [([0.0, -0.01, 1e-30, 0.01], [0.0, -0.01, 0.02, 1.0])]:
        c.ks, c.vs = torch.tensor(ks, device="cuda"), torch.tensor(vs, device="cuda")
        c.check(c.call(c.layout()))


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[4], KINDS[6], KINDS[8]], ids=["bf16", "d64", "f32", "kv8"])
def test_strides_and_rows_behind_the_last(kind):
    c = Case(kind, lens=[4, 66, 1], own=[100, 66, 64], sels=[[0], [1, 4], []], page=32, seed=11)
    want = c.oracle()
    t = c.q.shape[0]
    bits = torch.uint8 if c.dtype == "kv8" else c.k.dtype

    def spaced(x, before, after):  # the same values with other elements between the heads and between the tokens
        y = x.view(bits) if x.element_size() == 1 else x
        wide = torch.full((*y.shape[:-2], y.shape[-2] + 3, before + c.d + after), 0x7F if c.dtype == "kv8" else torch.nan,
                          dtype=y.dtype, device="cuda")
        view = wide[..., 1:1 + y.shape[-2], before:before + c.d]
        view.copy_(y)
        return view.view(x.dtype) if x.element_size() == 1 else view

    wide_q = torch.full((t + 5, c.hq + 2, 2 * c.d), torch.nan, dtype=c.q.dtype, device="cuda")
    wide_q[:t, 1:1 + c.hq, c.d:] = c.q
    c.q = wide_q[:t, 1:1 + c.hq, c.d:]
    c.k, c.v, c.kp, c.vp = spaced(c.k, 16, 32), spaced(c.v, 32, 16), spaced(c.kp, 16, 16), spaced(c.vp, 16, 16)
    whole = torch.full((t + 5, c.hq + 2, c.d + 16), 3.0, dtype=c.q.dtype, device="cuda")
    out = whole[:t, 1:1 + c.hq, 8:8 + c.d]
    c.call(c.layout(), out=out)
    c.check(out, want=want)
    out.fill_(3.0)
    assert (whole == 3.0).all()


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[1], KINDS[4], KINDS[6]], ids=["bf16", "mha", "d64", "f32"])
def test_agrees_with_the_prefill_and_the_decode_step(kind):
    """No older own keys and contiguous pages: the query prefill.  One token each: the decode step."""
    c = Case(kind, lens=[20, 64, 7], own=[20, 64, 7], sels=[[0, 3], [1], []], page=64, seed=12)
    c.table = np.arange(3, dtype=np.int32)[:, None]
    args = dict(cu_qlens=c.cu, sel_ptr=[0, 2, 3, 3], sel_idx=[0, 3, 1])
    ask = B.dbsa_layout_build(*c.pool, **args, block_m=32)
    own = [torch.cat([x[u, :n] for u, n in enumerate(c.lens)]) for x in (c.kp, c.vp)]
    a, b = c.call(c.layout()), B.dbsa_query_attn(ask, c.q, *own, c.k, c.v, c.scale)
    c.check(a)
    assert (a.float() - b.float()).abs().max() <= (2e-2 if c.dtype != "f32" else 2e-5)
    c = Case(kind, lens=[1, 1, 1], own=[20, 64, 7], sels=[[0, 3], [1], []], page=64, seed=13)
    c.table = np.arange(3, dtype=np.int32)[:, None]
    ask = B.dbsa_layout_build(*c.pool, **dict(args, cu_qlens=c.cu), block_m=32)
    table, n = c.device_tables()
    a, b = c.call(c.layout()), B.dbsa_decode_attn(ask, c.q, c.kp[:3], c.vp[:3], n, c.k, c.v, c.scale)
    c.check(a)
    assert (a.float() - b.float()).abs().max() <= (2e-2 if c.dtype != "f32" else 2e-5)


def test_groups_in_arena_pages():
    c = Case(KINDS[0], lens=[9, 40], own=[30, 400], sels=[[4, 0], [2]], page=16, seed=14)
    want = c.oracle()
    bounds = np.concatenate([[0], c.pool[1][c.pool[2]]])
    start = np.array([900, 40, -1, 2000, -1, 1500])
    arena_k, arena_v = (torch.full((2600, *x.shape[1:]), torch.nan, dtype=x.dtype, device="cuda") for x in (c.k, c.v))
    for i, s in enumerate(start):
        if s >= 0:
            for a, x in ((arena_k, c.k), (arena_v, c.v)):
                a[s:s + bounds[i + 1] - bounds[i]] = x[bounds[i]:bounds[i + 1]]
    c.k, c.v = arena_k, arena_v
    c.check(c.call(c.layout(page_start=start)), want=want)


def test_captured_into_a_graph_and_replayed_on_changed_inputs():
    c = Case(KINDS[0], lens=[5, 5, 5], own=[60, 200, 7], sels=[[0, 1], [1], [2, 3]], page=16, seed=15, table_width=40)
    lay, tables = c.layout(), c.device_tables()
    spare = torch.arange(c.kp.shape[0], device="cuda", dtype=torch.int32)
    ws = torch.empty(max(16, lay.workspace_bytes(c.hq, c.d)), dtype=torch.uint8, device="cuda")
    out, eager = torch.empty_like(c.q), torch.empty_like(c.q)
    c.call(lay, tables, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(lay, tables, out=out, workspace=ws)
    for step in range(4):
        c.own = [60 + 5 * step, 200 - 40 * step, 7 + step]
        tables[1].copy_(torch.tensor(c.own))
        c.table[0, :5] = spare.roll(step)[:5].cpu().numpy()
        tables[0].copy_(torch.from_numpy(c.table))
        c.q.copy_(c.q.flip(0))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        c.check(out)
        c.call(lay, tables, out=eager)
        assert torch.equal(out, eager)
    lay.destroy()


def test_on_another_stream_with_the_layout_destroyed_behind_the_call():
    c = Case(KINDS[8], lens=[5, 130], own=[60, 500], sels=[[0, 1], [4]], page=16, seed=16)
    want, tables, side = c.oracle(), c.device_tables(), torch.cuda.Stream()
    first = c.call(c.layout(), tables)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        outs = []
        for _ in range(6):
            lay = c.layout()  # (its lists are copied on the default stream)
            outs.append(c.call(lay, tables))
            lay.destroy()
    side.synchronize()
    for o in outs:
        assert torch.equal(o, first)
    c.check(first, want=want)


def test_two_calls_at_once_with_a_workspace_each():
    c = Case(KINDS[0], lens=[5, 30], own=[900, 700], sels=[[0, 1], [4]], page=16, seed=17)
    d = Case(KINDS[0], lens=[1] * 7, own=[100] * 7, sels=[[u % 5] for u in range(7)], page=16, seed=18)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    lays, tables = [c.layout(), d.layout()], [c.device_tables(), d.device_tables()]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(5):
        for i, x in enumerate((c, d)):
            with torch.cuda.stream(streams[i]):
                outs[i].append(x.call(lays[i], tables[i]))
    torch.cuda.synchronize()
    for i, x in enumerate((c, d)):
        x.check(outs[i][0])
        assert all(torch.equal(o, outs[i][0]) for o in outs[i])


def test_page_offsets_beyond_32_bits():
    """9 GB of 8-bit pages, the question's own keys at both ends; rows of the pool behind 2^31 bytes too."""
    c = Case(("kv8", 8, 2, 128), lens=[6], own=[40], sels=[[1]], page=16, seed=19)
    want = c.oracle()
    n_pages = 2 ** 20 + 7
    big_k = torch.empty((n_pages, 16, 2, 128), dtype=torch.float8_e4m3fn, device="cuda")
    big_v = torch.empty_like(big_k)
    places = [0, n_pages - 1, 2 ** 19 + 3]
    for i, place in enumerate(places):
        big_k[place], big_v[place] = c.kp[c.table[0, i]], c.vp[c.table[0, i]]
        c.table[0, i] = place
    start = 16 * (n_pages // 2)
    rows_k, rows_v = big_k.view(-1, 2, 128), big_v.view(-1, 2, 128)
    bounds = np.concatenate([[0], c.pool[1][c.pool[2]]])
    page_start = np.full(6, -1)
    for i, at in ((0, start + 100), (2, 16 * n_pages - 1000)):
        for big, x in ((rows_k, c.k), (rows_v, c.v)):
            big[at:at + bounds[i + 1] - bounds[i]] = x[bounds[i]:bounds[i + 1]]
        page_start[i] = at
    c.k, c.v, c.kp, c.vp = rows_k, rows_v, big_k, big_v
    o = c.call(c.layout(page_start=page_start))
    c.check(o, want=want)


@pytest.mark.parametrize("dtype", ["bf16", "kv8", "f32"])
@pytest.mark.parametrize("lens,own,sink", [([130], [4500], 70), ([3], [300], 4400)])
def test_walks_of_many_tiles(dtype, lens, own, sink):
    """256 KV heads leave a head one or two workers: more steps to a walk than lanes to a wave, own ones and the sink's.  Checked
    on two of the heads."""
    c = Case((dtype, 256, 256, 64), lens=lens, own=own, sels=[[0, 1]], page=16 if sink == 70 else 64, seed=21, sink=sink)
    assert len(c.layout().export_chunk(lens[0])["worker_ptr"]) <= 3
    o = c.call(c.layout())
    some = [3, 255]
    c.q, c.k, c.v = (x[:, some] for x in (c.q, c.k, c.v))
    c.kp, c.vp = c.kp[:, :, some], c.vp[:, :, some]
    if dtype == "kv8":
        c.ks, c.vs = c.ks[some], c.vs[some]
    c.check(o[:, some])


@pytest.mark.parametrize("kind", [KINDS[0], KINDS[8]], ids=["bf16", "kv8"])
def test_tokens_far_apart(kind):
    """Token strides of 2^22 elements, in pool and pages: 64 rows do not lie within 32 bits of bytes."""
    c = Case(kind, lens=[4, 50], own=[60, 90], sels=[[1], [0]], page=32, seed=22)
    want = c.oracle()
    bits = torch.uint8 if c.dtype == "kv8" else c.k.dtype

    def apart(x):
        flat = x.view(bits).reshape(-1, c.hkv, c.d)
        room = torch.empty((flat.shape[0], 2 ** 22), dtype=bits, device="cuda")
        view = room[:, :c.hkv * c.d].unflatten(1, (c.hkv, c.d))
        view.copy_(flat)
        return (view if x.dim() == 3 else view.unflatten(0, x.shape[:2])).view(x.dtype)

    c.k, c.v, c.kp, c.vp = (apart(x) for x in (c.k, c.v, c.kp, c.vp))
    c.check(c.call(c.layout()), want=want)


def test_tensors_with_fewer_rows_than_the_layout_names_are_refused():
    c = Case(KINDS[0], lens=[5, 3], own=[60, 30], sels=[[0, 4], [1]], page=16, seed=23)
    lay, (table, own) = c.layout(), c.device_tables()
    args = [lay, c.q, c.k, c.v, c.kp, c.vp, table, own, c.scale]
    B.dbsa_chunk_attn(*args)
    for change in ({1: c.q[:7]}, {2: c.k[:-1], 3: c.v[:-1]}, {3: c.v[:-1]}, {6: table[:1], 7: own[:1]}, {7: own[:1]}):
        with pytest.raises(AssertionError):
            B.dbsa_chunk_attn(*[change.get(i, x) for i, x in enumerate(args)])
    with pytest.raises(AssertionError):
        B.dbsa_chunk_attn(*args, lse=torch.empty((c.hq, 7), device="cuda"))
    with pytest.raises(AssertionError):
        B.dbsa_chunk_attn(*[x.cpu() if i == 6 else x for i, x in enumerate(args)])


def test_a_layout_of_other_heads_is_refused():
    c = Case(KINDS[0], lens=[5], own=[60], sels=[[0, 1]], page=16, seed=20)
    lay = B.dbsa_layout_build_chunk(*c.pool, cu_qlens=c.cu, sel_ptr=[0, 2], sel_idx=[0, 1], n_q_heads=16, n_kv_heads=2)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    ask = B.dbsa_layout_build(*c.pool, cu_qlens=c.cu, sel_ptr=[0, 2], sel_idx=[0, 1])
    for layout in (lay, ask):
        with pytest.raises(B.DbsaError) as e:
            c.call(layout, workspace=ws)
        assert e.value.code == B.DBSA_ERR_INVALID_ARG
    chunk = c.layout()
    with pytest.raises(B.DbsaError) as e:
        c.call(chunk, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert e.value.code == B.DBSA_ERR_WORKSPACE
    for call in (lambda: B.dbsa_query_attn(chunk, c.q, c.q[:, :2], c.q[:, :2], c.k, c.v, c.scale, workspace=ws),
                 lambda: B.dbsa_preencode_attn(chunk, c.q, c.k, c.v, c.scale)):
        with pytest.raises(B.DbsaError) as e:
            call()
        assert e.value.code == B.DBSA_ERR_INVALID_ARG
    with pytest.raises(AssertionError):
        B.dbsa_chunk_attn(chunk, c.q, c.k, c.v, c.kp.float(), c.vp.float(), *c.device_tables(), c.scale)
