"""Verification of proposed tokens and the pages of the caches: pins of their oracles, and what the calls refuse before they touch a
GPU (pointers are never followed on the host, so that any non-null number stands for one)."""
import ctypes as C
import itertools

import numpy as np
import pytest
import torch

from oracle import steps_oracle as orc
from paper_2503_08640_amd import binding as B

A = 4096  # an aligned address that nothing reads


# ---- pins ------------------------------------------------------------------------------------------------------

def _law(target, draft, steps, points=64):
    """Law of the tokens that come out when proposals are drawn from draft [steps, V]: every combination of proposals with its
    probability, uniform numbers on a grid of `points` midpoints."""
    vocab = target.shape[1]
    law = {}
    grid = (np.arange(points) + 0.5) / points
    for xs in itertools.product(range(vocab), repeat=steps):
        weight = np.prod([draft[a][x] for a, x in enumerate(xs)])
        for us in itertools.product(grid, repeat=steps + 1):
            r = orc.draft_verify(target, [0, *xs], [0, steps + 1], us, draft=draft[None], probabilities=True)
            key = int(r["out"][0])
            law[key] = law.get(key, 0.0) + weight / points ** (steps + 1)
    return np.array([law.get(i, 0.0) for i in range(vocab)])


def test_what_comes_out_follows_the_target():
    """The first token's law is the target's, whatever proposed (up to the grid's 2 * V / points)."""
    target = np.array([[0.5, 0.2, 0.3], [0.1, 0.6, 0.3]])
    for draft in ([[0.1, 0.8, 0.1]], [[1.0, 0.0, 0.0]], [[0.5, 0.2, 0.3]]):
        law = _law(target, np.array(draft), 1)
        assert np.abs(law - target[0]).max() <= 2 * 3 / 64


def test_worked_example_of_a_refusal():
    """p = (.5, .2, .3), q = (.1, .8, .1), proposal 1: stands below .25; else max(p - q, 0) = (.4, 0, .2) is drawn from."""
    p, q = np.array([[0.5, 0.2, 0.3], [0.1, 0.1, 0.8]]), np.array([[[0.1, 0.8, 0.1]]])
    run = lambda u, v: orc.draft_verify(p, [9, 1], [0, 2], [u, v], draft=q, probabilities=True)  # noqa: E731
    assert list(run(0.24, 0.15)["out"]) == [1, 1] and run(0.24, 0.15)["accepted"][0] == 1
    assert list(run(0.26, 0.66)["out"]) == [0, -1] and list(run(0.26, 0.67)["out"]) == [2, -1]
    assert run(0.26, 0.67)["accepted"][0] == 0


def test_greedy_is_the_limit_of_low_temperatures():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 30))
    tokens = [0, int(x[0].argmax()), int(x[1].argmin()), 4]
    a = orc.draft_verify(x, tokens, [0, 4], rng.random(4), temperature=[0.0])
    b = orc.draft_verify(x, tokens, [0, 4], rng.random(4), temperature=[1e-4])
    assert list(a["out"]) == list(b["out"]) == [tokens[1], int(x[1].argmax()), -1, -1]


def test_books_stay_consistent():
    """Random runs: counts are the entries that name a page, no free page is named, what a question writes to is its own."""
    rng = np.random.default_rng(5)
    b, c, pages, page = 9, 6, 60, 16
    k = orc.Books(np.full((b, c), -1), np.zeros(pages), np.zeros(b), page)
    for _ in range(200):
        what = rng.integers(4)
        if what == 0:
            k.fork([int(x) for x in np.where(rng.random(b) < 0.3, rng.integers(0, b, b), np.arange(b))])
        if what == 1:
            got, copies = k.reserve(rng.integers(-2, 30, b))
            for u in np.nonzero(got)[0]:
                for i in range((k.self_len[u] - got[u]) // page, -(-k.self_len[u] // page)):
                    assert k.refs[k.table[u, i]] == 1
            assert not set(x[0] for x in copies) & set(x[1] for x in copies)
        if what == 2:
            k.self_len = np.maximum(k.self_len - rng.integers(0, 20, b), 0)
            k.trim()
        if what == 3:
            copies, live, place = k.compact()
            assert (k.refs[:live] > 0).all() and (k.refs[live:] == 0).all()
        named = k.table[k.table >= 0]
        assert (np.bincount(named, minlength=pages) == k.refs).all()
        for u in range(b):
            assert (k.table[u, :k._used(k.self_len[u])] >= 0).all()


def test_what_is_written_to_is_not_shared():
    """A question that was cut without a trim still names pages behind its tokens.  Those of them that others name too are not handed to
    it for its new tokens: they are given back, and pages of its own stand in their place."""
    table, refs = np.full((2, 4), -1), np.zeros(8)
    table[0, :3], refs[:3] = [0, 1, 2], 1
    k = orc.Books(table, refs, [40, 0], 16)
    k.fork([0, 0])
    k.self_len[1] = 20
    got, copies = k.reserve([0, 20])
    assert list(got) == [0, 20] and copies == [(1, 3, 4)]
    # (page 2 is not question 0's alone until question 1 has given it back: then page 4 takes its place)
    assert k.table.tolist() == [[0, 1, 2, -1], [0, 3, 4, -1]] and k.refs.tolist() == [2, 1, 1, 1, 1, 0, 0, 0]
    # both are cut to nothing: page 0 goes back twice and is the lowest free one
    k.self_len[:] = 0
    got, copies = k.reserve([16, 16])
    assert copies == [] and k.table.tolist() == [[0, 1, 2, -1], [5, 3, 4, -1]] and k.refs.tolist() == [1, 1, 1, 1, 1, 1, 0, 0]
    # there are too few free ones: what was shared is given back all the same, the rest stays
    k = orc.Books(np.array([[0, 1], [0, 1]]), [2, 2], [16, 0], 16)
    got, copies = k.reserve([0, 32])
    assert list(got) == [0, 0] and copies == [] and k.table.tolist() == [[0, 1], [-1, -1]] and k.refs.tolist() == [1, 1]
    assert k.self_len.tolist() == [16, 0]


def test_books_without_trims():
    """Random runs in which rows keep naming what lies behind their tokens: nobody is handed a page that another entry names, and what a
    copy reads is still named."""
    rng = np.random.default_rng(6)
    b, c, pages, page = 9, 6, 70, 16
    for _ in range(40):
        k = orc.Books(np.full((b, c), -1), np.zeros(pages), np.zeros(b), page)
        for _ in range(12):
            k.fork([int(x) for x in np.where(rng.random(b) < 0.3, rng.integers(0, b, b), np.arange(b))])
            k.self_len = np.maximum(k.self_len - rng.integers(0, 50, b), 0)
            got, copies = k.reserve(rng.integers(-2, 40, b))
            for u in np.nonzero(got)[0]:
                for i in range((k.self_len[u] - got[u]) // page, -(-k.self_len[u] // page)):
                    assert k.refs[k.table[u, i]] == 1
            assert not set(x[0] for x in copies) & set(x[1] for x in copies) and all(k.refs[x[0]] > 0 for x in copies)
            named = k.table[k.table >= 0]
            assert (np.bincount(named, minlength=pages) == k.refs).all()


# ---- refusals of the library -----------------------------------------------------------------------------------

def verify(**change):
    a = dict(target=A, stride=1000, draft=None, tokens=A, cu=A, n=5, b=1, vocab=1000, dtype=B.DBSA_BF16, form=B.DBSA_LOGITS, heat=None,
             uniform=A, out=1 << 40, accepted=A, logp=None, self_len=None, new_len=None, ws=A, ws_bytes=None)
    a.update(change)
    d = None if a["draft"] is None else C.byref(B.Draft(*a["draft"]))
    need = B.dbsa_draft_verify_workspace_bytes(a["n"], a["b"], a["vocab"]) if a["ws_bytes"] is None else a["ws_bytes"]
    return B.lib().dbsa_draft_verify(a["target"], a["stride"], d, a["tokens"], a["cu"], a["n"], a["b"], a["vocab"], a["dtype"], a["form"],
                                     a["heat"], a["uniform"], a["out"], a["accepted"], a["logp"], a["self_len"], a["new_len"], a["ws"],
                                     need, None)


@pytest.mark.parametrize("change,code", [
    (dict(target=None), B.DBSA_ERR_INVALID_ARG), (dict(tokens=None), B.DBSA_ERR_INVALID_ARG), (dict(cu=None), B.DBSA_ERR_INVALID_ARG),
    (dict(uniform=None), B.DBSA_ERR_INVALID_ARG), (dict(out=None), B.DBSA_ERR_INVALID_ARG), (dict(accepted=None), B.DBSA_ERR_INVALID_ARG),
    (dict(n=-1), B.DBSA_ERR_INVALID_ARG), (dict(b=0), B.DBSA_ERR_INVALID_ARG), (dict(vocab=0), B.DBSA_ERR_INVALID_ARG),
    (dict(out=A), B.DBSA_ERR_INVALID_ARG), (dict(out=A + 4), B.DBSA_ERR_INVALID_ARG), (dict(out=A - 16), B.DBSA_ERR_INVALID_ARG),
    (dict(logp=A + 8), B.DBSA_ERR_INVALID_ARG), (dict(self_len=A), B.DBSA_ERR_INVALID_ARG), (dict(new_len=A), B.DBSA_ERR_INVALID_ARG),
    (dict(target=A + 1), B.DBSA_ERR_INVALID_ARG), (dict(target=A + 2, dtype=B.DBSA_F32), B.DBSA_ERR_INVALID_ARG),
    (dict(stride=-1), B.DBSA_ERR_INVALID_ARG), (dict(draft=(A + 1, 1, 1, 1)), B.DBSA_ERR_INVALID_ARG),
    (dict(draft=(A, -1, 1, 1)), B.DBSA_ERR_INVALID_ARG), (dict(draft=(A, 1, -1, 1)), B.DBSA_ERR_INVALID_ARG),
    (dict(draft=(A, 1, 1, -1)), B.DBSA_ERR_INVALID_ARG), (dict(form=B.DBSA_PROBABILITIES, heat=A), B.DBSA_ERR_INVALID_ARG),
    (dict(dtype=B.DBSA_E4M3), B.DBSA_ERR_UNSUPPORTED), (dict(form=2), B.DBSA_ERR_UNSUPPORTED),
    (dict(vocab=(1 << 30) + 1, ws_bytes=1 << 60), B.DBSA_ERR_UNSUPPORTED), (dict(n=1 << 20, vocab=200000), B.DBSA_ERR_UNSUPPORTED),
    (dict(ws=None), B.DBSA_ERR_WORKSPACE), (dict(ws=A + 8), B.DBSA_ERR_WORKSPACE), (dict(ws_bytes=64), B.DBSA_ERR_WORKSPACE),
])
def test_verify_refuses(change, code):
    assert verify(**change) == code


@pytest.mark.parametrize("written", ["out", "logp", "accepted", "new_len"])
@pytest.mark.parametrize("read", ["tokens", "uniform", "cu", "heat", "self_len"])
def test_outputs_over_what_is_read_are_refused(written, read):
    """Every workgroup of a question reads what one of them writes beside: only the lengths may be one array."""
    at = dict(tokens=1 << 20, uniform=2 << 20, cu=3 << 20, heat=4 << 20, self_len=5 << 20, out=6 << 20, logp=7 << 20, accepted=8 << 20,
              new_len=9 << 20, target=10 << 20, ws=11 << 20, n=40, b=30)
    last = 4 * (dict(tokens=40, uniform=40, cu=31, heat=30, self_len=30)[read] - 1)
    first = 4 * (dict(out=40, logp=40, accepted=30, new_len=30)[written] - 1)
    for off in (last, -first) + ((0,) if (written, read) != ("new_len", "self_len") else (4, -4)):
        assert verify(**dict(at, **{written: at[read] + off})) == B.DBSA_ERR_INVALID_ARG, off


@pytest.mark.parametrize("one,other", itertools.combinations(["out", "logp", "accepted", "new_len"], 2))
def test_outputs_over_each_other_are_refused(one, other):
    at = dict(tokens=1 << 20, uniform=2 << 20, cu=3 << 20, self_len=5 << 20, out=6 << 20, logp=7 << 20, accepted=8 << 20, new_len=9 << 20,
              target=10 << 20, ws=11 << 20, n=40, b=30)
    for off in (0, 4 * 29, -4 * 29):
        assert verify(**dict(at, **{one: at[other] + off})) == B.DBSA_ERR_INVALID_ARG, off


def test_the_most_that_is_checked():
    """Rows, or questions, times pieces of 4096 words: 2^23, and not one more (seen by which argument is refused)."""
    for n, b, vocab, code in ((1 << 23, 1, 4096, B.DBSA_ERR_WORKSPACE), (1 << 23, 1, 4097, B.DBSA_ERR_UNSUPPORTED),
                              (1, 1 << 23, 4096, B.DBSA_ERR_WORKSPACE), ((1 << 23) + 1, 1, 1, B.DBSA_ERR_UNSUPPORTED),
                              (1 << 22, 1, 8192, B.DBSA_ERR_WORKSPACE), (1 << 22, 1, 8193, B.DBSA_ERR_UNSUPPORTED),
                              (32, 1, 1 << 30, B.DBSA_ERR_WORKSPACE), (33, 1, 1 << 30, B.DBSA_ERR_UNSUPPORTED)):
        assert verify(n=n, b=b, vocab=vocab, ws=None) == code, (n, b, vocab)


def test_workspace_grows_with_what_is_checked():
    size = B.dbsa_draft_verify_workspace_bytes
    assert size(-1, 1, 9) == size(1, 0, 9) == size(1, 1, 0) == size(1, 1, (1 << 30) + 1) == 0
    assert 0 < size(1, 1, 1) < size(2, 1, 1) < size(2, 2, 1) < size(2, 2, 200000)
    assert size(0, 1, 1) > 0 and all(size(n, b, v) % 16 == 0 for n, b, v in ((1, 1, 1), (3, 5, 50257), (7, 2, 8190)))


def book(**change):
    a = dict(table=A, refs=A, self_len=A, b=3, columns=8, page=16, pages=50)
    a.update(change)
    return C.byref(B.PageBook(*(a[x] for x in ("table", "refs", "self_len", "b", "columns", "page", "pages"))))


BAD_BOOKS = [(dict(refs=None), B.DBSA_ERR_INVALID_ARG), (dict(pages=0), B.DBSA_ERR_INVALID_ARG), (dict(table=None), B.DBSA_ERR_INVALID_ARG),
             (dict(columns=0), B.DBSA_ERR_INVALID_ARG), (dict(b=-1), B.DBSA_ERR_INVALID_ARG), (dict(page=8), B.DBSA_ERR_UNSUPPORTED),
             (dict(page=48), B.DBSA_ERR_UNSUPPORTED), (dict(page=0), B.DBSA_ERR_UNSUPPORTED), (dict(b=4097), B.DBSA_ERR_UNSUPPORTED),
             (dict(columns=(1 << 20) + 1), B.DBSA_ERR_UNSUPPORTED)]


@pytest.mark.parametrize("change,code", BAD_BOOKS + [(dict(self_len=None), B.DBSA_ERR_INVALID_ARG), (dict(b=0), B.DBSA_ERR_INVALID_ARG)])
def test_books_refuse(change, code):
    L = B.lib()
    assert L.dbsa_pages_fork(book(**change), A, None) == code
    assert L.dbsa_pages_trim(book(**change), None) == code
    assert L.dbsa_pages_reserve(book(**change), A, A, A, A, A, 200, None) == code


@pytest.mark.parametrize("change,code", BAD_BOOKS)
def test_compact_refuses(change, code):
    assert B.lib().dbsa_pages_compact(book(**change), A, A, A, None) == code


def test_missing_arrays_are_refused():
    L = B.lib()
    bad = B.DBSA_ERR_INVALID_ARG
    assert L.dbsa_pages_fork(None, A, None) == L.dbsa_pages_fork(book(), None, None) == bad
    for i in range(4):
        args = [A] * 4
        args[i] = None
        assert L.dbsa_pages_reserve(book(), *args, A, 200, None) == bad
    for ws, size in ((None, 200), (A, 199), (A + 2, 200)):
        assert L.dbsa_pages_reserve(book(), A, A, A, A, ws, size, None) == B.DBSA_ERR_WORKSPACE
    for i in range(3):
        args = [A] * 3
        args[i] = None
        assert L.dbsa_pages_compact(book(), *args, None) == bad


def copy(**change):
    a = dict(k=(A, 1024, 128), v=(A, 1024, 128), stride_page=16384, page=16, pages=50, layers=2, stride_layer=1 << 20, copies=A, n=A, most=3,
             heads=8, dim=128, dtype=B.DBSA_BF16)
    a.update(change)
    pages = B.Pages(B.Tensor(*a["k"]), B.Tensor(*a["v"]), a["stride_page"], None, 0, a["page"], a["pages"])
    return B.lib().dbsa_pages_copy(C.byref(pages), a["layers"], a["stride_layer"], a["copies"], a["n"], a["most"], a["heads"], a["dim"],
                                   a["dtype"], None)


@pytest.mark.parametrize("change,code", [
    (dict(k=(None, 1024, 128)), B.DBSA_ERR_INVALID_ARG), (dict(v=(A + 8, 1024, 128)), B.DBSA_ERR_INVALID_ARG),
    (dict(k=(A, 1023, 128)), B.DBSA_ERR_INVALID_ARG), (dict(v=(A, 1024, 0)), B.DBSA_ERR_INVALID_ARG),
    (dict(k=(A, 1032, 136), dtype=B.DBSA_E4M3), B.DBSA_ERR_INVALID_ARG), (dict(stride_page=0), B.DBSA_ERR_INVALID_ARG),
    (dict(stride_page=16385), B.DBSA_ERR_INVALID_ARG), (dict(layers=0), B.DBSA_ERR_INVALID_ARG),
    (dict(stride_layer=-8), B.DBSA_ERR_INVALID_ARG), (dict(stride_layer=4), B.DBSA_ERR_INVALID_ARG),
    (dict(stride_layer=0), B.DBSA_ERR_INVALID_ARG), (dict(copies=None), B.DBSA_ERR_INVALID_ARG), (dict(n=None), B.DBSA_ERR_INVALID_ARG),
    (dict(most=-1), B.DBSA_ERR_INVALID_ARG), (dict(heads=0), B.DBSA_ERR_INVALID_ARG), (dict(pages=0), B.DBSA_ERR_INVALID_ARG),
    (dict(dim=96), B.DBSA_ERR_UNSUPPORTED), (dict(dtype=3), B.DBSA_ERR_UNSUPPORTED), (dict(page=24), B.DBSA_ERR_UNSUPPORTED),
    (dict(page=1 << 29), B.DBSA_ERR_UNSUPPORTED), (dict(page=1 << 20, layers=1 << 22), B.DBSA_ERR_UNSUPPORTED),
])
def test_copy_refuses(change, code):
    assert copy(**change) == code


def test_nothing_to_copy_is_no_error():
    assert copy(most=0) == B.DBSA_OK


# ---- refusals of the binding, on host tensors ------------------------------------------------------------------

def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.mark.parametrize("change", [
    dict(tokens=ints(4)), dict(tokens=torch.zeros(5)), dict(cu_qlens=ints(1)), dict(uniform=torch.zeros(4)),
    dict(uniform=torch.zeros(5, dtype=torch.float64)), dict(temperature=torch.zeros(2)), dict(logp=torch.zeros(6)), dict(out=ints(4)),
    dict(accepted=ints(2)), dict(self_len=ints(1)), dict(self_len=ints(1), new_len=ints(2)), dict(draft=torch.zeros(2, 4, 9)),
    dict(draft=torch.zeros(1, 4, 8)), dict(draft=torch.zeros(1, 4, 9, dtype=torch.bfloat16)), dict(target=torch.zeros(9, 5).t()),
])
def test_verify_arguments(change):
    a = dict(target=torch.zeros(5, 9), tokens=ints(5), cu_qlens=ints(2), uniform=torch.zeros(5))
    a.update(change)
    with pytest.raises(AssertionError):
        B.dbsa_draft_verify(**a)


def test_books_arguments():
    table, refs, n = ints(3, 8), ints(50), ints(3)
    for bad in (dict(page_table=table.float()), dict(page_table=ints(8, 3).t()), dict(refs=ints(5, 10)), dict(self_len=ints(2)), dict(source=ints(4))):
        a = dict(page_table=table, refs=refs, self_len=n, source=n, page_tokens=16)
        a.update(bad)
        with pytest.raises(AssertionError):
            B.dbsa_pages_fork(**a)
    for bad in (dict(add=ints(2)), dict(got=ints(4)), dict(copies=ints(2, 3)), dict(copies=ints(3, 2)), dict(n_copies=ints(2))):
        a = dict(page_table=table, refs=refs, self_len=n, add=n, page_tokens=16)
        a.update(bad)
        with pytest.raises(AssertionError):
            B.dbsa_pages_reserve(**a)
    for bad in (dict(copies=ints(24, 3)), dict(counts=ints(1)), dict(new_place=ints(49)), dict(refs=ints(5, 10), page_table=None)):
        a = dict(refs=refs, page_table=table, page_tokens=16)
        a.update(bad)
        with pytest.raises(AssertionError):
            B.dbsa_pages_compact(**a)
    k = torch.zeros(5, 16, 2, 64)
    for bad in (dict(v_pages=torch.zeros(5, 16, 2, 128)), dict(v_pages=torch.zeros(5, 16, 2, 64, dtype=torch.bfloat16)), dict(copies=ints(3)),
                dict(copies=ints(3, 2)), dict(n_copies=ints(0))):
        a = dict(k_pages=k, v_pages=k.clone(), copies=ints(3, 3), n_copies=ints(1))
        a.update(bad)
        with pytest.raises(AssertionError):
            B.dbsa_pages_copy(**a)
