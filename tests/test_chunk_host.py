"""Host side of the chunk attention: what the plan of a chunk layout covers, and what is refused.  No GPU."""
import ctypes as C

import numpy as np
import pytest

from paper_2503_08640_amd import binding as B


def pool(sink, lens, per_group):
    demos = sink + np.concatenate([[0], np.cumsum(lens)])
    return sink, demos, np.arange(0, len(lens) + 1, per_group)


def build(p, lens, sels, hq, hkv, own=None, **kw):
    return B.dbsa_layout_build_chunk(*p, cu_qlens=np.concatenate([[0], np.cumsum(lens)]), sel_ptr=np.cumsum([0] + [len(s) for s in sels]),
                                     sel_idx=[g for s in sels for g in s], n_q_heads=hq, n_kv_heads=hkv, own_tokens=own,
                                     host_only=True, **kw)


def random_case(seed):
    rng = np.random.default_rng(seed)
    groups = int(rng.integers(1, 9))
    sink = int(rng.choice([0, 4, 64, 333]))
    p = pool(sink, rng.integers(1, 300, size=4 * groups), 4)
    b = int(rng.choice([1, 2, 5, 40, 130]))
    lens = rng.integers(1, int(rng.choice([2, 9, 70, 400])), size=b)
    sels = [list(rng.permutation(groups)[:int(rng.integers(0, groups + 1))]) for _ in range(b)]
    hq, hkv = [(8, 2), (32, 8), (32, 32), (5, 1), (6, 2), (32, 1), (1, 1), (700, 700)][int(rng.integers(8))]
    own = None if rng.random() < 0.3 else lens + rng.integers(0, int(rng.choice([1, 100, 9000])), size=b)
    return p, lens, sels, hq, hkv, own


@pytest.mark.parametrize("seed", range(60))
def test_every_token_meets_each_of_its_tiles_once(seed):
    p, lens, sels, hq, hkv, own = random_case(seed)
    T, cu = int(sum(lens)), np.concatenate([[0], np.cumsum(lens)])
    lay = build(p, lens, sels, hq, hkv, own)
    plan = lay.export_chunk(T)
    r = hq // hkv
    bounds = np.asarray(p[1])[p[2]]
    assert plan["rows"] in (32, 64, 128, 256) and plan["rows"] >= r
    assert plan["worker_ptr"][0] == 0 and (np.diff(plan["worker_ptr"]) >= 0).all()

    def tiles_of(lo, hi):
        return [(a, min(64, hi - a)) for a in range(int(lo), int(hi), 64)]

    pool_seen = [[] for _ in range(T)]
    own_seen = [[] for _ in range(T)]
    parts = [[] for _ in range(T)]
    rows_used = 0
    for rec in plan["records"]:
        tok, n, ent, n_ent, u, lo, hi, out_of, part, first, new, zero = (int(x) for x in rec)
        assert 1 <= n and n * r <= plan["rows"] and zero == 0 and n_ent >= 0 and (n_ent > 0 or hi > lo)
        toks = plan["tokens"][tok:tok + n]
        assert (np.diff(toks) > 0).all()
        for t in toks:
            pool_seen[t] += [(int(a), int(b)) for a, b in plan["tiles"][ent:ent + n_ent]]
        if u >= 0:
            assert 0 <= lo < hi <= out_of and (first, new) == (cu[u], lens[u]) and (toks >= cu[u]).all() and (toks < cu[u + 1]).all()
            last = max((own[u] if own is not None else lens[u]) - (cu[u + 1] - 1 - toks[-1]), 1)
            assert out_of == -(-last // 64)
            for t in toks:
                own_seen[t].append((lo, hi, out_of))
        else:
            assert (lo, hi, first, new) == (0, 0, 0, 0)
        if part >= 0:
            rows_used = max(rows_used, part + n)
            for i, t in enumerate(toks):
                parts[t].append(part + i)
        else:
            for t in toks:
                parts[t].append(None)
    for u in range(len(lens)):
        want = tiles_of(0, p[0]) + [x for g in sels[u] for x in tiles_of(bounds[g], bounds[g + 1])]
        for t in range(cu[u], cu[u + 1]):
            assert sorted(pool_seen[t]) == sorted(want)
            ranges = sorted(own_seen[t])
            assert ranges[0][0] == 0 and ranges[-1][1] == ranges[-1][2] and all(a[1] == b[0] for a, b in zip(ranges, ranges[1:]))
    # a token is finished by its only record, or all its records have partial rows of their own
    listed = []
    for t in range(T):
        got = plan["parts"][plan["part_ptr"][t]:plan["part_ptr"][t + 1]].tolist()
        if parts[t] == [None]:
            assert got == []
        else:
            assert None not in parts[t] and sorted(got) == sorted(parts[t])
            listed += got
    assert len(set(listed)) == len(listed) and rows_used == len(listed)
    assert lay.workspace_bytes(hq, 128) == rows_used * hq * 132 * 4 and lay.workspace_bytes(hq + 1, 128) == 0


@pytest.mark.parametrize("lens,own,hq,hkv", [([2048], [32000], 32, 8), ([8] * 16, [500] * 16, 32, 8), ([1] * 128, None, 32, 8),
                                             ([229, 130, 200], [900, 700, 1100], 32, 32)])
def test_workers_get_equal_shares(lens, own, hq, hkv):
    p = pool(64, [128] * 220, 10)
    sels = [list(range(u % 5, 22, 3)) for u in range(len(lens))]
    plan = build(p, lens, sels, hq, hkv, own).export_chunk(sum(lens))
    cost = [sum(int(r[3]) + max(int(r[6]) - int(r[5]), 0) + 3 for r in plan["records"][a:b])
            for a, b in zip(plan["worker_ptr"], plan["worker_ptr"][1:])]
    assert max(cost) <= 1.1 * sum(cost) / len(cost) + 9


def test_arena_pages_are_named_by_the_tiles():
    p = pool(10, [100, 150], 1)
    plan = build(p, [3], [[1]], 2, 2, page_start=[500, -1, 700]).export_chunk(3)
    assert plan["tiles"].tolist()[-4:] == [[500, 10], [700, 64], [764, 64], [828, 22]]


def refused(code, f):
    with pytest.raises(B.DbsaError) as e:
        f()
    assert e.value.code == code


def test_refusals_of_the_build():
    p = pool(4, [10, 20], 1)
    refused(B.DBSA_ERR_UNSUPPORTED, lambda: build(p, [2], [[0]], 5, 2))
    refused(B.DBSA_ERR_UNSUPPORTED, lambda: build(p, [2], [[0]], 33, 1))
    refused(B.DBSA_ERR_INVALID_ARG, lambda: build(p, [2], [[0]], 0, 1))
    refused(B.DBSA_ERR_INVALID_ARG, lambda: build(p, [2], [[0]], 2, -1))
    refused(B.DBSA_ERR_INVALID_ARG, lambda: build(p, [2], [[0]], 2, 2, own=[-1]))
    refused(B.DBSA_ERR_BAD_BOUNDS, lambda: build(p, [2, 0], [[0], [1]], 2, 2))
    refused(B.DBSA_ERR_BAD_SELECTION, lambda: build(p, [2], [[2]], 2, 2))
    refused(B.DBSA_ERR_BAD_SELECTION, lambda: build(p, [2], [[0, 0]], 2, 2))
    refused(B.DBSA_ERR_BAD_SELECTION, lambda: build(p, [2], [[0]], 2, 2, page_start=[0, -1, 100]))
    out = C.c_void_p()
    do, gdo = B._i32(p[1]), B._i32(p[2])
    desc = B.PoolDesc(4, 2, B._p32(do), 2, B._p32(gdo), 0)
    assert B.lib().dbsa_layout_build_chunk(C.byref(desc), None, 2, 2, None, 1, None, C.byref(out)) == B.DBSA_ERR_INVALID_ARG
    assert B.lib().dbsa_layout_build_chunk(None, None, 2, 2, None, 1, None, C.byref(out)) == B.DBSA_ERR_INVALID_ARG
    assert B.lib().dbsa_layout_build_chunk(C.byref(desc), None, 2, 2, None, 1, None, None) == B.DBSA_ERR_INVALID_ARG
    assert not out.value


def test_layouts_of_the_wrong_stage():
    p = pool(4, [10, 20], 1)
    chunk = build(p, [2], [[0]], 2, 2)
    ask = B.dbsa_layout_build(*p, cu_qlens=[0, 2], sel_ptr=[0, 1], sel_idx=[0], host_only=True)
    refused(B.DBSA_ERR_INVALID_ARG, lambda: ask.export_chunk(2))
    refused(B.DBSA_ERR_INVALID_ARG, lambda: chunk.export_decode(1))
    refused(B.DBSA_ERR_INVALID_ARG, lambda: chunk.export_schedule(4))
    refused(B.DBSA_ERR_INVALID_ARG, lambda: chunk.export_cut_schedule(4, 8))
    refused(B.DBSA_ERR_INVALID_ARG, lambda: chunk.export_matrix_records())
    assert chunk.export()[0].shape == (0, 4)


# ---- calls: every check comes before anything is launched, so that made-up addresses are never read ----

def tensor(dtype_bytes=2, d=128, heads=2, at=4096):
    return B.Tensor(at, heads * d, d)


def chunk_call(layout, kv8=False, **change):
    a = dict(q=tensor(), k=tensor(), v=tensor(), o=tensor(), kp=tensor(), vp=tensor(), page=16 * 256, table=64, stride=4, tokens=16,
             pages=8, own=True, self_len=64, dtype=B.DBSA_BF16, hq=2, hkv=2, d=128, scale=0.1, ws=None, ws_bytes=0, ks=64, vs=64)
    a.update(change)
    own = B.Pages(a["kp"], a["vp"], a["page"], a["table"], a["stride"], a["tokens"], a["pages"])
    ref = C.byref(own) if a["own"] else None
    tail = (a["hq"], a["hkv"], a["d"], a["scale"], a["ws"], a["ws_bytes"], None)
    if kv8:
        return B.lib().dbsa_chunk_attn_kv8(layout, a["q"], a["k"], a["v"], ref, a["self_len"], a["ks"], a["vs"], a["o"], None, *tail)
    return B.lib().dbsa_chunk_attn(layout, a["q"], a["k"], a["v"], ref, a["self_len"], a["o"], None, a["dtype"], *tail)


@pytest.mark.parametrize("kv8", [False, True])
def test_a_host_layout_is_refused_by_the_calls(kv8):
    lay = build(pool(4, [10, 20], 1), [2], [[0]], 2, 2)
    assert chunk_call(lay.handle, kv8) == B.DBSA_ERR_INVALID_ARG
    assert chunk_call(None, kv8) == B.DBSA_ERR_INVALID_ARG
    ask = B.dbsa_layout_build(4, [4, 14], [0, 1], cu_qlens=[0, 2], sel_ptr=[0, 1], sel_idx=[0], host_only=True)
    assert chunk_call(ask.handle, kv8) == B.DBSA_ERR_INVALID_ARG
    assert chunk_call(lay.handle, dtype=7) == B.DBSA_ERR_UNSUPPORTED


@pytest.mark.parametrize("kv8", [False, True])
def test_refusals_of_the_chunk_calls(kv8):
    p = pool(64, [128] * 40, 10)
    lay = build(p, [40, 3], [[0, 1, 2], [1]], 2, 2)
    need = lay.workspace_bytes(2, 128)
    assert need > 0
    for change, code in [(dict(d=96), B.DBSA_ERR_UNSUPPORTED), (dict(hq=3), B.DBSA_ERR_UNSUPPORTED), (dict(tokens=24), B.DBSA_ERR_UNSUPPORTED),
                         (dict(tokens=8), B.DBSA_ERR_UNSUPPORTED), (dict(tokens=2 ** 20, pages=2 ** 20), B.DBSA_ERR_UNSUPPORTED),
                         (dict(ws=4096, ws_bytes=need - 1), B.DBSA_ERR_WORKSPACE), (dict(ws=None), B.DBSA_ERR_WORKSPACE),
                         (dict(ws=4104, ws_bytes=need), B.DBSA_ERR_WORKSPACE)]:
        assert chunk_call(lay.handle, kv8, **change) == code, change
    # (with a workspace the call comes to the check that the layout is on a device)
    for change in [dict(), dict(hq=4), dict(hq=4, hkv=4), dict(scale=0.0), dict(scale=float("nan")), dict(own=False), dict(table=None),
                   dict(self_len=None), dict(stride=0), dict(pages=0), dict(page=0), dict(page=4100), dict(q=tensor(at=8)),
                   dict(o=tensor(at=None)), dict(k=B.Tensor(4096, 256, 4)), dict(vp=tensor(at=4104))]:
        assert chunk_call(lay.handle, kv8, **{"ws": 4096, "ws_bytes": need, **change}) == B.DBSA_ERR_INVALID_ARG, change


def kv8_call(which, **change):
    a = dict(k=tensor(), v=tensor(), n=3, rows=None, first=0, k8=tensor(), v8=tensor(), n_rows=8, ks=64, vs=64, hkv=2, d=128,
             dtype=B.DBSA_BF16, pos=None, first_id=0, table=None, n_pos=0)
    a.update(change)
    rope = (a["pos"], a["first_id"], a["table"], a["n_pos"])
    if which == "scales":
        return B.lib().dbsa_kv8_scales(a["k"], a["v"], a["n"], a["hkv"], a["d"], a["dtype"], *rope, 0, a["ks"], a["vs"], None)
    if which == "write":
        return B.lib().dbsa_kv8_write(a["k"], a["v"], a["n"], a["rows"], a["first"], a["k8"], a["v8"], a["n_rows"], a["ks"], a["vs"],
                                      a["hkv"], a["d"], a["dtype"], *rope, None)
    return B.lib().dbsa_kv8_read(a["k8"], a["v8"], a["n_rows"], a["rows"], a["first"], a["n"], a["ks"], a["vs"], a["k"], a["v"],
                                 a["hkv"], a["d"], a["dtype"], None)


@pytest.mark.parametrize("which", ["scales", "write", "read"])
def test_refusals_of_the_8bit_calls(which):
    bad = [(dict(dtype=2), B.DBSA_ERR_UNSUPPORTED), (dict(d=96), B.DBSA_ERR_UNSUPPORTED), (dict(n=-1), B.DBSA_ERR_INVALID_ARG),
           (dict(hkv=0), B.DBSA_ERR_INVALID_ARG), (dict(ks=None), B.DBSA_ERR_INVALID_ARG), (dict(vs=None), B.DBSA_ERR_INVALID_ARG),
           (dict(k=tensor(at=4104)), B.DBSA_ERR_INVALID_ARG), (dict(v=tensor(at=0)), B.DBSA_ERR_INVALID_ARG),
           (dict(k=B.Tensor(4096, 252, 128)), B.DBSA_ERR_INVALID_ARG), (dict(n=2 ** 31 - 1, hkv=2 ** 20), B.DBSA_ERR_UNSUPPORTED)]
    if which != "scales":
        bad += [(dict(k8=tensor(at=4104)), B.DBSA_ERR_INVALID_ARG), (dict(v8=B.Tensor(4096, 256, 120)), B.DBSA_ERR_INVALID_ARG),
                (dict(first=-1), B.DBSA_ERR_INVALID_ARG), (dict(first=6), B.DBSA_ERR_INVALID_ARG),
                (dict(n_rows=0), B.DBSA_ERR_INVALID_ARG), (dict(first=2 ** 62), B.DBSA_ERR_INVALID_ARG)]
    if which != "read":
        bad += [(dict(table=64, n_pos=0), B.DBSA_ERR_INVALID_ARG), (dict(table=64, n_pos=2), B.DBSA_ERR_INVALID_ARG),
                (dict(table=64, n_pos=9, first_id=-1), B.DBSA_ERR_INVALID_ARG), (dict(table=72, n_pos=9), B.DBSA_ERR_INVALID_ARG)]
    for change, code in bad:
        assert kv8_call(which, **change) == code, change


@pytest.mark.parametrize("seed", range(60))
def test_workgroups_have_four_or_eight_waves(seed):
    p, lens, sels, hq, hkv, own = random_case(seed)
    assert build(p, lens, sels, hq, hkv, own).export_chunk(int(sum(lens)))["rows"] in (128, 256)


def test_a_chunk_layout_has_no_lists_of_the_other_stages():
    chunk = build(pool(4, [10, 20], 1), [2], [[0]], 2, 2)
    tab, ptr, ent = chunk.export()
    assert tab.shape == (0, 4) and ptr.tolist() == [0] and ent.shape == (0, 2) and chunk.export_order().shape == (0,)
    for export in (lambda: chunk.export_decode(1), lambda: chunk.export_decode_groups(2, 1), lambda: chunk.export_positions(1),
                   chunk.export_matrix_records, lambda: chunk.export_matrix_plan(1), lambda: chunk.export_schedule(4),
                   lambda: chunk.export_cut_schedule(4, 8)):
        refused(B.DBSA_ERR_INVALID_ARG, export)
