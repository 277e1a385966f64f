"""Quantising a cache as it is written, and reading it back.  Without a rotation every result is defined by single fp32
operations and compared exactly; a rotated key may be off by half a step of the format, and by the fp32 rounding of the
rotation in front of it."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle, rope_oracle
from oracle import dbsa_oracle as orc
from paper_2503_08640_amd import binding as B
from paper_2503_08640_amd import synth
from gpu_util import assert_close, to_f64

pytestmark = pytest.mark.gpu

F8 = torch.float8_e4m3fn


def normal(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def as_8bit(x, scale):
    """The definition: x / scale in fp32, clamped, to the nearest value; zeros where the scale has no finite inverse."""
    none = ~torch.isfinite(1.0 / scale) | ~torch.isfinite(scale)
    return torch.where(none[:, None], torch.zeros_like(x.float()), (x.float() / scale[:, None]).clamp(-448, 448)).to(F8)


def top(x):
    """Largest magnitude per head over 448, one correctly rounded division."""
    a = x.float().abs().amax(dim=(0, 2))
    return a / torch.full_like(a, 448)


def same_bytes(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


SHAPES = [(1, 1, 64), (1, 8, 128), (5, 5, 64), (700, 8, 128), (333, 3, 128), (64, 70, 128), (40, 130, 64), (3001, 2, 64)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,h,d", SHAPES)
def test_scales_are_the_largest_magnitudes(n, h, d, dtype):
    k, v = normal(1, n, h, d, dtype=dtype), 3 * normal(2, n, h, d, dtype=dtype)
    ks, vs = B.dbsa_kv8_scales(k, v)
    assert torch.equal(ks, top(k)) and torch.equal(vs, top(v))
    # running: only what is larger moves a scale
    more = ks.clone() * torch.linspace(0.5, 1.5, h, device="cuda")
    want = torch.maximum(more, ks)
    B.dbsa_kv8_scales(k, v, k_scale=more, v_scale=vs, running=True)
    assert torch.equal(more, want) and torch.equal(vs, top(v))


def test_scales_pass_over_what_is_not_finite_and_zeros_give_zero():
    k, v = normal(3, 50, 4, 64), normal(4, 50, 4, 64)
    k[7, 1, 5], k[9, 2, 60], v[0, 0, 0], v[49, 3, 63] = torch.inf, torch.nan, -torch.inf, torch.nan
    k[:, 3] = 0
    ks, vs = B.dbsa_kv8_scales(k, v)
    finite = [torch.where(torch.isfinite(x.float()), x.float().abs(), torch.zeros(1, device="cuda")) for x in (k, v)]
    assert torch.equal(ks, top(finite[0])) and torch.equal(vs, top(finite[1])) and ks[3] == 0
    empty = torch.empty((0, 4, 64), dtype=torch.bfloat16, device="cuda")
    ks, vs = B.dbsa_kv8_scales(empty, empty)
    assert not ks.any() and not vs.any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,h,d", SHAPES)
def test_rows_are_written_where_they_belong(n, h, d, dtype):
    k, v = normal(5, n, h, d, dtype=dtype), normal(6, n, h, d, dtype=dtype)
    ks, vs = B.dbsa_kv8_scales(k, v)
    ks, vs = ks * 0.9, vs * 0.5  # (some elements beyond the format)
    room = n + 9
    k8, v8 = ((torch.arange(room * h * d, device="cuda") % 251).to(torch.uint8).view(room, h, d).view(F8).clone() for _ in range(2))
    want_k, want_v = k8.clone(), v8.clone()
    B.dbsa_kv8_write(k, v, k8, v8, ks, vs, first_row=4)
    want_k.view(torch.uint8)[4:4 + n], want_v.view(torch.uint8)[4:4 + n] = (as_8bit(x, s).view(torch.uint8) for x, s in ((k, ks), (v, vs)))
    assert same_bytes(k8, want_k) and same_bytes(v8, want_v)
    # scattered rows, some tokens without a place
    rows = torch.randperm(room, generator=torch.Generator().manual_seed(n))[:n].to(torch.int32)
    lost = torch.arange(n) % 5 == 3
    rows[lost] = torch.tensor([-1, room, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32)[torch.arange(int(lost.sum())) % 4]
    B.dbsa_kv8_write(k, v, k8, v8, ks, vs, rows=rows.cuda())
    at = rows[~lost].long().cuda()
    want_k.view(torch.uint8)[at], want_v.view(torch.uint8)[at] = (as_8bit(x, s).view(torch.uint8)[~lost.cuda()] for x, s in ((k, ks), (v, vs)))
    assert same_bytes(k8, want_k) and same_bytes(v8, want_v)


def test_every_bf16_value_is_rounded_to_the_nearest():
    """All 65536 patterns under scales 1 and 3; ties to even, saturation, NaN, subnormal results."""
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).cuda().view(512, 1, 128)
    x = torch.cat([bits, bits], dim=1).contiguous()
    scale = torch.tensor([1.0, 3.0], device="cuda")
    k8, v8 = (torch.zeros((512, 2, 128), dtype=F8, device="cuda") for _ in range(2))
    B.dbsa_kv8_write(x, x, k8, v8, scale, scale)
    want = as_8bit(x, scale)
    nan = torch.isnan(x.float())
    assert torch.isnan(k8.float())[nan].all() and torch.equal(torch.isnan(k8.float()), nan)
    assert torch.equal(k8.view(torch.uint8)[~nan], want.view(torch.uint8)[~nan]) and same_bytes(k8, v8)
    assert (k8.float()[torch.isinf(x.float())].abs() == 448).all()


def test_scales_without_an_inverse_give_zeros():
    x = normal(7, 20, 4, 64)
    scale = torch.tensor([0.0, 1e-39, 2.0, torch.inf], device="cuda")
    k8, v8 = (torch.full((20, 4, 64), 1.0, device="cuda").to(F8) for _ in range(2))
    B.dbsa_kv8_write(x, x, k8, v8, scale, scale)
    assert not k8.float()[:, [0, 1, 3]].any() and same_bytes(k8[:, 2], as_8bit(x, scale)[:, 2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,h,d", SHAPES)
def test_keys_are_rotated_on_their_way(n, h, d, dtype):
    """Off by half a step (2^-4 of the value, 2^-10 below the normal range, in units of the scale) and by the rotation's fp32
    rounding: three operations on numbers below |u| + |w|.  The scales see the rotated keys the same way."""
    f = rope_oracle.inv_freq(500000.0, d)
    table = B.dbsa_rope_table(f, 5000)
    k, v = normal(8, n, h, d, dtype=dtype), normal(9, n, h, d, dtype=dtype)
    ids = torch.randint(0, 5000, (n,), generator=torch.Generator().manual_seed(n), dtype=torch.int32)
    for kw, at in ((dict(positions=ids.cuda()), ids.numpy()), (dict(first_id=1234), 1234 + np.arange(n))):
        ks, vs = B.dbsa_kv8_scales(k, v, table=table, **kw)
        k8, v8 = (torch.zeros((n, h, d), dtype=F8, device="cuda") for _ in range(2))
        B.dbsa_kv8_write(k, v, k8, v8, ks, vs, table=table, **kw)
        want = rope_oracle.rope(k.double().cpu().numpy(), at, f)
        pair = np.abs(k.double().cpu().numpy())
        pair = pair + np.roll(pair, d // 2, axis=2)
        most = np.abs(want).max(axis=(0, 2))
        scale = ks.double().cpu().numpy()
        assert (np.abs(scale * 448 - most) <= 2.0 ** -21 * pair.max(axis=(0, 2))).all()
        got = k8.float().double().cpu().numpy() * scale[:, None]
        bound = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * scale[:, None]) * (1 + 2.0 ** -20) + 2.0 ** -21 * pair
        assert (np.abs(got - want) <= bound).all()
        assert torch.equal(vs, top(v)) and same_bytes(v8, as_8bit(v, vs))


def test_ids_outside_the_table_take_its_nearest_row():
    table = B.dbsa_rope_table(rope_oracle.inv_freq(500000.0, 64), 100)
    k = normal(10, 4, 2, 64)
    one = torch.full((2,), 0.01, device="cuda")
    a, b, c = (torch.zeros((4, 2, 64), dtype=F8, device="cuda") for _ in range(3))
    B.dbsa_kv8_write(k, k, a, c, one, one, table=table, positions=torch.tensor([-7, 100, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda"))
    B.dbsa_kv8_write(k, k, b, c, one, one, table=table, positions=torch.tensor([0, 99, 99, 0], dtype=torch.int32, device="cuda"))
    assert same_bytes(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n,h,d", SHAPES)
def test_rows_come_back(n, h, d, dtype):
    room = n + 300
    k8, v8 = ((torch.arange(room * h * d, device="cuda") * m % 256).to(torch.uint8).view(room, h, d).view(F8) for m in (1, 3))
    ks, vs = torch.linspace(0.01, 2, h, device="cuda"), torch.linspace(-1, 3, h, device="cuda")

    def want(x, s):
        return (x.float() * s[:, None]).to(dtype)

    def same(a, b):
        a, b = a.float(), b.float()
        return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[~torch.isnan(a)], b[~torch.isnan(b)])

    k, v = B.dbsa_kv8_read(k8, v8, ks, vs, first_row=17, n_tokens=n, dtype=dtype)
    assert k.dtype == dtype and same(k, want(k8, ks)[17:17 + n]) and same(v, want(v8, vs)[17:17 + n])
    rows = torch.randint(0, room, (n,), generator=torch.Generator().manual_seed(n), dtype=torch.int32)  # (repeats too)
    away = torch.arange(n) % 7 == 2
    rows[away] = torch.tensor([-1, room, 2 ** 31 - 1], dtype=torch.int32)[torch.arange(int(away.sum())) % 3]
    k, v = B.dbsa_kv8_read(k8, v8, ks, vs, rows=rows.cuda(), dtype=dtype)
    at = rows.clamp(0, room - 1).long().cuda()
    assert same(k[~away.cuda()], want(k8, ks)[at][~away.cuda()]) and same(v[~away.cuda()], want(v8, vs)[at][~away.cuda()])
    assert not k[away.cuda()].any() and not v[away.cuda()].any()


def test_strides_and_what_lies_between():
    n, h, d = 37, 3, 128
    wide = normal(11, n, 2 * h + 1, d + 8, dtype=torch.float32)
    k, v = wide[:, :h, 4:4 + d], wide[:, h:2 * h, 4:4 + d]
    ks, vs = B.dbsa_kv8_scales(k, v)
    assert torch.equal(ks, top(k)) and torch.equal(vs, top(v))
    cache = torch.full((50, 2 * h + 2, d + 32), 9, dtype=torch.uint8, device="cuda")
    k8, v8 = cache[:, :h, 16:16 + d].view(F8), cache[:, h + 1:2 * h + 1, 16:16 + d].view(F8)
    B.dbsa_kv8_write(k, v, k8, v8, ks, vs, first_row=13)
    assert same_bytes(k8[13:], as_8bit(k, ks)) and same_bytes(v8[13:], as_8bit(v, vs))
    out = torch.full((n, 2 * h + 1, d + 8), 5.0, device="cuda")
    B.dbsa_kv8_read(k8, v8, ks, vs, first_row=13, n_tokens=n, k_out=out[:, :h, 4:4 + d], v_out=out[:, h + 1:, 4:4 + d])
    assert torch.equal(out[:, :h, 4:4 + d], as_8bit(k, ks).float() * ks[:, None])
    cache[13:, :h, 16:16 + d], cache[13:, h + 1:2 * h + 1, 16:16 + d] = 9, 9
    out[:, :h, 4:4 + d], out[:, h + 1:, 4:4 + d] = 5, 5
    assert (cache == 9).all() and (out == 5).all()


def test_rows_beyond_32_bits_of_bytes():
    rows = 2 ** 24 + 100
    k8, v8 = (torch.zeros((rows, 2, 128), dtype=F8, device="cuda") for _ in range(2))  # 4.3 GB each
    k, v = normal(12, 6, 2, 128), normal(13, 6, 2, 128)
    ks, vs = B.dbsa_kv8_scales(k, v)
    at = torch.tensor([0, rows - 1, 2 ** 23, 2 ** 24 + 1, 5, rows - 50], dtype=torch.int32, device="cuda")
    B.dbsa_kv8_write(k, v, k8, v8, ks, vs, rows=at)
    assert same_bytes(k8[at.long()], as_8bit(k, ks)) and same_bytes(v8[at.long()], as_8bit(v, vs))
    a, b = B.dbsa_kv8_read(k8, v8, ks, vs, rows=at, dtype=torch.float32)
    assert torch.equal(a, as_8bit(k, ks).float() * ks[:, None]) and torch.equal(b, as_8bit(v, vs).float() * vs[:, None])
    assert int((k8.view(torch.uint8) != 0).any(dim=2).any(dim=1).sum()) == 6


def test_captured_calls_and_another_stream():
    k, v = normal(14, 40, 4, 128), normal(15, 40, 4, 128)
    table = B.dbsa_rope_table(rope_oracle.inv_freq(500000.0, 128), 200)
    ks, vs = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda")
    k8, v8 = (torch.zeros((64, 4, 128), dtype=F8, device="cuda") for _ in range(2))
    ko, vo = torch.empty_like(k), torch.empty_like(v)
    rows = torch.arange(40, dtype=torch.int32, device="cuda")

    def passes(ks, vs, k8, v8, ko, vo):
        B.dbsa_kv8_scales(k, v, k_scale=ks, v_scale=vs, table=table, first_id=7)
        B.dbsa_kv8_write(k, v, k8, v8, ks, vs, rows=rows, table=table, first_id=7)
        B.dbsa_kv8_read(k8, v8, ks, vs, rows=rows, k_out=ko, v_out=vo)

    buffers = (ks, vs, k8, v8, ko, vo)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        passes(*buffers)
    side = torch.cuda.Stream()
    for step in range(3):
        k.copy_(normal(20 + step, 40, 4, 128) * (3 - step))
        v.copy_(normal(30 + step, 40, 4, 128))
        rows.copy_(torch.randperm(64)[:40].to(torch.int32))
        for b in buffers:
            b.zero_()
        graph.replay()
        torch.cuda.synchronize()
        other = [torch.zeros_like(b) for b in buffers]
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            passes(*other)
        side.synchronize()
        for a, b in zip(buffers, other):
            assert same_bytes(a, b)


@pytest.mark.parametrize("hq,hkv", [(8, 2), (4, 4)])
def test_a_question_answered_from_an_8bit_cache(hq, hkv):
    """The calls together: the pool is quantised once, a prompt and two follow-up chunks are written into pages and attended
    (dbsa_kv8_write, dbsa_chunk_attn_kv8), and the decode step over the same pool agrees (dbsa_decode_attn_kv8 over the
    pages read back by dbsa_kv8_read)."""
    pc = synth.make_pool_case("kv8c", 6100 + hq, dtype="bf16", n_q_heads=hq, n_kv_heads=hkv, head_dim=128, sink_len=70,
                              pool_tokens=3000, demo_len_range=(30, 200), n_groups=5, k_channel_sigma=0.5)
    p = pc.pool

    def dev(x):
        return torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)

    k, v = dev(pc.k), dev(pc.v)
    ks, vs = B.dbsa_kv8_scales(k, v)
    k8, v8 = (torch.zeros(x.shape, dtype=F8, device="cuda") for x in (k, v))
    B.dbsa_kv8_write(k, v, k8, v8, ks, vs)
    page, sels, turns = 32, [[3, 0], [1], [4, 2, 0]], [[50, 1, 33], [5, 5, 5], [1, 1, 1]]
    table = torch.randperm(9, generator=torch.Generator().manual_seed(3)).to(torch.int32).view(3, 3)
    kp, vp = (torch.zeros((9, page, hkv, 128), dtype=F8, device="cuda") for _ in range(2))
    sel = dict(sel_ptr=np.cumsum([0] + [len(s) for s in sels]), sel_idx=[g for s in sels for g in s])
    own = np.zeros(3, np.int64)
    kq, vq = (x.float().double().cpu().numpy() * s.double().cpu().numpy()[:, None] for x, s in ((k8, ks), (v8, vs)))
    for step, lens in enumerate(turns):
        t, cu = sum(lens), np.concatenate([[0], np.cumsum(lens)])
        new_k, new_v, q = normal(50 + step, t, hkv, 128), normal(60 + step, t, hkv, 128), normal(70 + step, t, hq, 128)
        rows = [int(table[u, j // page]) * page + j % page for u in range(3) for j in range(own[u], own[u] + lens[u])]
        B.dbsa_kv8_scales(new_k, new_v, k_scale=ks.clone(), v_scale=vs.clone(), running=True)  # (the cache keeps its scales)
        B.dbsa_kv8_write(new_k, new_v, kp.view(-1, hkv, 128), vp.view(-1, hkv, 128), ks, vs,
                         rows=torch.tensor(rows, dtype=torch.int32, device="cuda"))
        own += lens
        lay = B.dbsa_layout_build_chunk(p.sink_len, p.demo_offsets, p.group_demo_offsets, cu_qlens=cu, **sel, n_q_heads=hq,
                                        n_kv_heads=hkv, own_tokens=own)
        self_len = torch.tensor(own, dtype=torch.int32, device="cuda")
        o = B.dbsa_chunk_attn_kv8(lay, q, k8, v8, kp, vp, table.cuda(), self_len, ks, vs, pc.scale)
        kpq, vpq = (x.float().double().cpu().numpy() * s.double().cpu().numpy()[:, None] for x, s in ((kp, ks), (vp, vs)))
        want = chunk_oracle.chunk_attn(to_f64(q), kq, vq, kpq, vpq, table.numpy(), own, p.sink_len, p.demo_offsets, p.group_demo_offsets,
                                       cu, sel["sel_ptr"], np.asarray(sel["sel_idx"]), pc.scale)
        tol = 2.0 ** -8 * (want["weight"] + np.abs(want["o"])) * (1 + 2.0 ** -4)
        assert (np.abs(to_f64(o) - want["o"]) <= tol).all()
    # the last turn was one token each: the decode step over the same caches, own keys back in bf16
    rows = torch.tensor([[int(table[u, j // page]) * page + j % page for j in range(3 * page)] for u in range(3)], dtype=torch.int32, device="cuda")
    kc, vc = B.dbsa_kv8_read(kp.view(-1, hkv, 128), vp.view(-1, hkv, 128), ks, vs, rows=rows.view(-1))
    ask = B.dbsa_layout_build(p.sink_len, p.demo_offsets, p.group_demo_offsets, cu_qlens=[0, 1, 2, 3], **sel, block_m=32)
    kc, vc = kc.view(3, 3 * page, hkv, 128), vc.view(3, 3 * page, hkv, 128)
    step = B.dbsa_decode_attn_kv8(ask, q, kc, vc, self_len, k8, v8, ks, vs, pc.scale)
    ref = orc.decode_attn(to_f64(q), to_f64(kc), to_f64(vc), own, kq, vq, p.sink_len, p.demo_offsets, p.group_demo_offsets,
                          sel["sel_ptr"], np.asarray(sel["sel_idx"]), pc.scale)
    assert_close(to_f64(step), ref, "decode over the same caches")
    assert_close(to_f64(o), ref, "one-token chunk over the same caches")


def test_absent_rows_are_read_as_zeros_under_any_scale():
    k8 = torch.full((5, 4, 64), 3.0, device="cuda").to(F8)
    scale = torch.tensor([torch.inf, torch.nan, -torch.inf, -2.0], device="cuda")
    rows = torch.tensor([-1, 5, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    for dtype in (torch.bfloat16, torch.float32):
        for x in B.dbsa_kv8_read(k8, k8, scale, scale, rows=rows, dtype=dtype):
            assert (x == 0).all()
