"""Chunk attention and 8-bit caches at the edge of what they accept: scales that are not finite, nothing, tiny or huge, values near
the top of their type, infinities that a row does see.  Against the fp64 oracle, with the tolerances of test_gpu_chunk.py."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu

# heads, KV heads; lens, own: one question whose tokens walk by themselves, some that share their groups' tiles, and (128 KV heads)
# workgroups with many records
BATCHES = {
    "alone": dict(lens=[300], own=[420], sels=[[4, 2]]),
    "shared": dict(lens=[3, 1, 9], own=[90, 200, 9], sels=[[0, 1], [1], [3, 0]]),
    "one": dict(lens=[1], own=[70], sels=[[1]]),
}


def case(dtype, d, batch, seed, heads=(8, 2), **kw):
    return Case((dtype, *heads, d), page=32, seed=seed, **dict(BATCHES[batch], **kw))


def run(c):
    lse = torch.zeros((c.hq, int(c.cu[-1])), device="cuda")
    return c.call(c.layout(), lse=lse), lse


def second_half_higher(c, by):
    """Scores of about 0 for the first 32 keys of every 64, `by` (log2 units) for the others: in the sink, in every group, in the
    own keys."""
    sign = torch.sign(torch.randn(c.d, generator=torch.Generator().manual_seed(1))).cuda()
    size = by * np.log(2) / np.sqrt(c.d)  # (q = sign: the product is size * D, the scale 1 / sqrt D)
    bounds = np.concatenate([[0], c.pool[1][c.pool[2]]])
    at = np.concatenate([np.arange(b - a) for a, b in zip(bounds, bounds[1:])])
    own = np.arange(c.kp.shape[0] * c.page).reshape(c.kp.shape[:2]) % c.page
    for u in range(len(c.lens)):
        for i, page in enumerate(c.table[u]):
            if page >= 0:
                own[page] = i * c.page + np.arange(c.page)

    def keys(x):
        high = torch.from_numpy((x % 64 >= 32).astype(np.float32)).cuda()[..., None, None] * size * sign
        high = high.expand(*x.shape, c.hkv, c.d)
        return high if c.ks is None else high / c.ks[:, None]

    c.k, c.kp = keys(at).to(c.k.dtype).contiguous(), keys(own).to(c.k.dtype).contiguous()
    c.q = sign.expand(c.q.shape).to(c.q.dtype).contiguous()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("batch", sorted(BATCHES))
def test_a_scale_that_is_no_number_gives_no_numbers(batch, d):
    for which in ("ks", "vs"):
        c = case("kv8", d, batch, seed=50, heads=(8, 4))
        want = c.oracle()
        getattr(c, which)[1] = torch.nan
        o = run(c)[0]
        assert torch.isnan(o[:, 2:4]).all()
        rest = [0, 1, 4, 5, 6, 7]
        c.hq, c.hkv = 6, 3
        c.check(o[:, rest], want={k: v if k == "keys" else v[rest] if k == "lse" else v[:, rest] for k, v in want.items()})


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("batch", sorted(BATCHES))
def test_a_tiny_softmax_scale(dtype, d, batch):
    c = case(dtype, d, batch, seed=51)
    c.q, c.k, c.kp = (x * 1e16 for x in (c.q, c.k, c.kp))
    c.scale = 1e-32 / np.sqrt(d)
    o, lse = run(c)
    c.check(o, lse)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("batch", sorted(BATCHES))
def test_tiny_key_scales_and_none(batch, d):
    """Factors far below 1 against queries far above it, of either sign; under a scale of zero all keys weigh the same, and a
    product of queries and bytes beyond fp32 does not matter."""
    c = case("kv8", d, batch, seed=52, heads=(8, 4))
    c.ks = torch.tensor([1e-34, -3e-35, 0.0, -0.0], device="cuda")
    c.q[:, :4] *= 1e32
    c.q[:, 4:] *= 1e37
    o, lse = run(c)
    c.check(o, lse)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("heads", [(8, 2), (128, 128), (256, 128)])
def test_an_infinite_value_that_is_seen_stays_infinite(dtype, d, heads):
    """In the last row of segments that end inside a tile, and inside a tile."""
    c = case(dtype, d, "shared" if heads == (8, 2) else "alone", seed=53, heads=heads, **({} if heads == (8, 2) else {"lens": [300], "own": [300]}))
    bounds = c.pool[1][c.pool[2]]
    want, some = c.oracle() if heads == (8, 2) else None, [0, 1]
    r = c.hq // c.hkv
    sign, channels = [1, -1, 1], [5, d - 1, 0]
    rows = [c.pool[0] - 1, int(bounds[c.sels[0][0] + 1]) - 1, int(bounds[c.sels[0][1]]) + 10]
    sees = [np.ones(int(c.cu[-1]), bool)] + [np.concatenate([np.full(n, c.sels[0][i] in s) for n, s in zip(c.lens, c.sels)]) for i in (0, 1)]
    near = c.v.clone()
    for row, s, ch in zip(rows, sign, channels):
        c.v[row, :, ch] = s * torch.inf
    o = run(c)[0]
    c.v = near
    if want is None:
        heads = [h * r + i for h in some for i in range(r)]
        o = o[:, heads]
        c.q, c.k, c.v, c.kp, c.vp = c.q[:, heads], c.k[:, some], c.v[:, some], c.kp[:, :, some], c.vp[:, :, some]
        want = c.oracle()
    got = o.clone()
    for s, ch, see in zip(sign, channels, sees):
        see = torch.from_numpy(see).cuda()
        assert see.any() and (got[see][:, :, ch] == s * torch.inf).all()
        place = torch.zeros_like(got, dtype=torch.bool)
        place[:, :, ch] = see[:, None]
        got = torch.where(place, torch.from_numpy(want["o"]).cuda().to(got.dtype), got)
    c.check(got, want=want)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("batch", sorted(BATCHES))
def test_values_near_the_top_of_their_type(dtype, d, batch):
    """The weighted mean of finite values is finite, however many there are, and however far the weights rise along the keys."""
    for power, by in ((110, 20), (126, 20), (126, 0), (126, 60)):
        c = case(dtype, d, batch, seed=54)
        second_half_higher(c, by)
        for x in (c.v, c.vp):
            x.copy_((1 + torch.rand(x.shape, generator=torch.Generator("cuda").manual_seed(3), device="cuda")) * 2.0 ** (power - 1))
        o, lse = run(c)
        c.check(o, lse)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("batch", sorted(BATCHES))
def test_tiny_and_huge_value_scales(batch, d):
    for size in (1.2e-38, 1e35):
        c = case("kv8", d, batch, seed=55)
        second_half_higher(c, 18)
        c.vs = torch.full((c.hkv,), size, device="cuda")
        o, lse = run(c)
        c.check(o, lse)
