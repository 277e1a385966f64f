"""Chunk attention where a workgroup takes many records one after the other, in both shapes (128 and 256 rows), for every storage
type and head size: what one record leaves in shared memory, in registers and in flight must not reach the next, least of
all behind a record that was walked a second time.  Many KV heads leave each a handful of workgroups; two of the heads are checked
against the fp64 oracle, with the tolerances of test_gpu_chunk.py."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu

LENS, OWN, SELS = [260, 300, 40, 120, 7], [260, 420, 300, 120, 500], [[0, 1], [4], [2, 3, 1], [], [0]]
TYPES = [("bf16", 128), ("bf16", 64), ("kv8", 128), ("kv8", 64), ("f32", 128), ("f32", 64)]
# heads, KV heads, rows of a workgroup that the plan takes for them
SHAPES = [(128, 128, 128), (256, 128, 256)]
GRID = [(t, d, *s) for t, d in TYPES for s in SHAPES]
IDS = ["%s-%d-rows%d" % (g[0], g[1], g[4]) for g in GRID]


def batch(dtype, d, hq, hkv, rows, seed, page=32, **kw):
    c = Case((dtype, hq, hkv, d), lens=LENS, own=OWN, sels=SELS, page=page, seed=seed, **kw)
    plan = c.layout().export_chunk(sum(LENS))
    taken = np.diff(plan["worker_ptr"])
    assert plan["rows"] == rows and taken.min() >= 3, "not the plan this test is for"
    # records that finish their rows and records that leave partial states, own keys in the middle of a worker's records
    middle = np.concatenate([plan["records"][a + 1:b - 1] for a, b in zip(plan["worker_ptr"], plan["worker_ptr"][1:])])
    assert (middle[:, 4] >= 0).any() and (plan["records"][:, 8] >= 0).any() and (plan["records"][:, 8] < 0).any()
    return c


def of_two_heads(c, o, lse):
    """The case as its KV heads 3 and 126 alone see it, and these heads' results."""
    some, r = [3, 126], c.hq // c.hkv
    heads = [s * r + i for s in some for i in range(r)]
    c.q, c.k, c.v, c.kp, c.vp = c.q[:, heads], c.k[:, some], c.v[:, some], c.kp[:, :, some], c.vp[:, :, some]
    if c.dtype == "kv8":
        c.ks, c.vs = c.ks[some], c.vs[some]
    return o[:, heads], lse[heads]


def run(c):
    lse = torch.zeros((c.hq, int(c.cu[-1])), device="cuda")
    return c.call(c.layout(), lse=lse), lse


def grow(c, x):
    """Keys whose scores rise by hundreds, for x [keys, ...] in 0 .. 1 (see aim)."""
    sign = torch.sign(torch.randn(c.d, generator=torch.Generator().manual_seed(1))).cuda()
    top = 40.0 * x[..., None, None] * sign
    return top.expand(*x.shape, c.hkv, c.d) if c.dtype != "kv8" else (top * 0.004 / c.ks[:, None]).clamp(-448, 448)


def aim(c):
    """Turns the queries to the keys of grow()."""
    sign = torch.sign(torch.randn(c.d, generator=torch.Generator().manual_seed(1))).cuda()
    c.q = (sign + 0.1 * c.q.float()).to(c.q.dtype)


@pytest.mark.parametrize("dtype,d,hq,hkv,rows", GRID, ids=IDS)
def test_records_one_after_the_other(dtype, d, hq, hkv, rows):
    c = batch(dtype, d, hq, hkv, rows, seed=40)
    o, lse = of_two_heads(c, *run(c))
    c.check(o, lse)


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("dtype,d,hq,hkv,rows", GRID, ids=IDS)
def test_second_walks_between_quick_ones(dtype, d, hq, hkv, rows, page):
    """Scores that outgrow their first keys in a pool group, in the middle of question 1's own keys and in question 3's, and a
    key and a value of question 1 that are not finite and that its earlier tokens do not see."""
    c = batch(dtype, d, hq, hkv, rows, seed=41, page=page)
    aim(c)
    lo, hi = (int(c.pool[1][c.pool[2]][g]) for g in (3, 4))  # group 3: question 2's
    c.k[lo:hi] = grow(c, torch.linspace(0, 1, hi - lo, device="cuda")).to(c.k.dtype)
    for u, first in ((1, 64), (3, 0)):
        j = np.arange(first, OWN[u])
        at = torch.from_numpy(c.table[u][j // page].astype(np.int64) * page + j % page).cuda()
        c.kp.view(-1, c.hkv, d)[at] = grow(c, torch.linspace(0, 1, len(j), device="cuda")).to(c.kp.dtype)
    first = OWN[1] - LENS[1]
    j = first + 170  # seen by tokens 170 .. 299 of question 1
    want_rows = np.ones(sum(LENS), bool)
    want_rows[c.cu[1] + 170:c.cu[2]] = False
    clean = [x.clone() for x in (c.kp, c.vp)]
    for x in (c.kp, c.vp):
        x[c.table[1, j // page], j % page, :, 5] = torch.nan
    o, lse = run(c)
    c.kp, c.vp = clean
    o, _ = of_two_heads(c, o, lse)
    c.check(o, rows=want_rows)
    assert torch.isnan(o[int(c.cu[1]) + 170:int(c.cu[2]), :, 5]).all()


@pytest.mark.parametrize("dtype,d,hq,hkv,rows", GRID, ids=IDS)
def test_pages_missing_in_the_middle(dtype, d, hq, hkv, rows):
    c = batch(dtype, d, hq, hkv, rows, seed=42, page=16)
    c.table[1, 5], c.table[1, 20], c.table[2, 7], c.table[3, 2], c.table[4, 30] = -1, c.kp.shape[0], 2 ** 31 - 1, -2 ** 31, -7
    o, lse = of_two_heads(c, *run(c))
    c.check(o, lse)


@pytest.mark.parametrize("dtype,d,hq,hkv,rows", [g for g in GRID if g[1] == 128], ids=[i for g, i in zip(GRID, IDS) if g[1] == 128])
def test_tokens_far_apart_in_every_shape(dtype, d, hq, hkv, rows):
    """Token strides of 2^22 elements in pool and pages, where 64 rows do not lie within 32 bits of bytes."""
    c = batch(dtype, d, hq, hkv, rows, seed=43, page=64)
    bits = torch.uint8 if c.dtype == "kv8" else c.k.dtype

    def apart(x):
        flat = x.view(bits).reshape(-1, c.hkv, c.d)
        view = torch.empty((flat.shape[0], 2 ** 22), dtype=bits, device="cuda")[:, :c.hkv * c.d].unflatten(1, (c.hkv, c.d))
        view.copy_(flat)
        return (view if x.dim() == 3 else view.unflatten(0, x.shape[:2])).view(x.dtype)

    near = c.k, c.v, c.kp, c.vp
    c.k, c.v, c.kp, c.vp = (apart(x) for x in near)
    o, lse = run(c)
    c.k, c.v, c.kp, c.vp = near
    o, lse = of_two_heads(c, o, lse)
    c.check(o, lse)


@pytest.mark.parametrize("dtype,d,hq,hkv,rows", GRID, ids=IDS)
def test_captured_records(dtype, d, hq, hkv, rows):
    """Replays with other lengths give what eager calls give, bit for bit: nothing is carried from one replay to the next."""
    c = batch(dtype, d, hq, hkv, rows, seed=44, page=64)
    lay, tables = c.layout(), c.device_tables()
    ws = torch.empty(lay.workspace_bytes(c.hq, c.d), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(c.q)
    c.call(lay, tables, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(lay, tables, out=out, workspace=ws)
    for step in range(3):
        tables[1].copy_(torch.tensor([260 - step, 420, 300 - 70 * step, 120, 500 - 100 * step]))
        c.q.copy_(c.q.flip(0))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, c.call(lay, tables)) and torch.isfinite(out.float()).all()
    lay.destroy()
