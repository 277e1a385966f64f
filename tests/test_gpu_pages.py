"""The books of paged caches against an oracle that changes them question by question, and the copies that go with them: whole
numbers and bits, so that everything has to be equal."""
import numpy as np
import pytest
import torch

from oracle import chunk_oracle, steps_oracle as orc
from paper_2503_08640_amd import binding as B

pytestmark = pytest.mark.gpu


class Pair:
    """The oracle's books and the device's, side by side."""

    def __init__(self, table, refs, self_len, page):
        self.want, self.page = orc.Books(table, refs, self_len, page), page
        self.table, self.refs, self.self_len = (torch.from_numpy(np.array(x, np.int32)).cuda() for x in (table, refs, self_len))

    def check(self, what):
        torch.cuda.synchronize()
        for x in ("table", "refs", "self_len"):
            got, want = getattr(self, x).cpu().numpy(), getattr(self.want, x)
            assert (got == want).all(), (what, x, np.argwhere(got != want)[:5].tolist())

    def fork(self, source):
        self.want.fork(source)
        B.dbsa_pages_fork(self.table, self.refs, self.self_len, dev(source), self.page)
        self.check("fork")

    def reserve(self, add):
        got, copies = self.want.reserve(add)
        g, c, n = B.dbsa_pages_reserve(self.table, self.refs, self.self_len, dev(add), self.page,
                                       copies=torch.full((len(add), 3), -9, dtype=torch.int32, device="cuda"))
        self.check("reserve")
        assert (g.cpu().numpy() == got).all(), "reserve: got"
        assert int(n) == len(copies) and c[:len(copies)].tolist() == [list(x) for x in copies], "reserve: copies"
        assert (c[len(copies):] == -9).all()
        return c, n

    def set_len(self, n):
        self.want.self_len = np.array(n, np.int64)
        self.self_len.copy_(dev(n))

    def trim(self):
        self.want.trim()
        B.dbsa_pages_trim(self.table, self.refs, self.self_len, self.page)
        self.check("trim")

    def compact(self):
        copies, live, place = self.want.compact()
        n = len(self.want.refs)
        c, counts, where = B.dbsa_pages_compact(self.refs, self.table, self.page,
                                                copies=torch.full((max(1, n // 2), 3), -9, dtype=torch.int32, device="cuda"))
        self.check("compact")
        assert counts.tolist() == [len(copies), live] and c[:len(copies)].tolist() == [list(x) for x in copies]
        assert (c[len(copies):] == -9).all() and (where.cpu().numpy() == place).all()
        return c, counts


def dev(x):
    return torch.from_numpy(np.array(x, np.int32)).cuda()


def books(seed, b, columns, pages, page, full=0.5, stray=True):
    """Rows with pages out of a shuffled arena; some share, some hold pages behind their tokens, some entries name nothing."""
    rng = np.random.default_rng(seed)
    free = list(rng.permutation(pages))
    table, length, refs = np.full((b, columns), -1, np.int64), np.zeros(b, np.int64), np.zeros(pages, np.int64)
    for u in range(b):
        if u and rng.random() < 0.3:
            s = int(rng.integers(0, u))
            n = -(-length[s] // page)
            table[u, :n], length[u] = table[s, :n], length[s]
            continue
        n = min(int(rng.integers(0, max(1, int(full * columns)) + 1)), len(free))
        table[u, :n] = [free.pop() for _ in range(n)]
        length[u] = max(0, n * page - int(rng.integers(0, 2 * page)))
    if stray:
        table[table < 0] = rng.choice([-1, -7, pages, 2 ** 31 - 1], (table < 0).sum())
    for e in table[(table >= 0) & (table < pages)]:
        refs[e] += 1
    other = rng.permutation(pages)[:pages // 10]  # another batch's tables
    refs[other] += rng.integers(1, 3, len(other))
    return Pair(table, refs, length, page)


SHAPES = [(1, 1, 1, 16), (1, 5, 9, 16), (3, 8, 40, 32), (16, 70, 900, 16), (65, 33, 2500, 64), (130, 9, 700, 128), (7, 1500, 9000, 16)]


@pytest.mark.parametrize("b,columns,pages,page", SHAPES)
def test_random_runs(b, columns, pages, page):
    rng = np.random.default_rng(b + columns)
    for seed in range(3):
        k = books(seed, b, columns, pages, page)
        for step in range(8):
            print(f"[pages] {b} {columns} {pages} {page}: seed {seed} step {step}", flush=True)
            k.fork(np.where(rng.random(b) < 0.4, rng.integers(-2, b + 2, b), np.arange(b)))
            k.reserve(rng.integers(-1, [2, 9, 3 * page, columns * page // 2 + 2][step % 4], b))
            k.set_len(np.maximum(k.want.self_len - rng.integers(0, 12, b), 0))
            k.trim()
            if step % 3 == 2:
                k.compact()


@pytest.mark.parametrize("b,columns,pages,page", SHAPES + [(1100, 6, 9000, 16)])
def test_random_runs_without_trims(b, columns, pages, page):
    """Rows go on naming what lies behind their tokens: what others name too is not written to."""
    rng = np.random.default_rng(7 * b + columns)
    for seed in range(3):
        k = books(50 + seed, b, columns, pages, page)
        for step in range(8):
            print(f"[pages] {b} {columns} {pages} {page}: without trims, seed {seed} step {step}", flush=True)
            k.fork(np.where(rng.random(b) < 0.4, rng.integers(-2, b + 2, b), np.arange(b)))
            k.set_len(np.maximum(k.want.self_len - rng.integers(0, [12, 5 * page, columns * page][step % 3], b), 0))
            k.reserve(rng.integers(-1, [2, 9, 3 * page, columns * page // 2 + 2][step % 4], b))
            if step % 3 == 2:
                k.compact()


def test_pages_that_are_shared_behind_the_tokens():
    """A fork that was cut: entries that are reached and shared go back and others stand in their place, be they few or many, is the page
    another's last one or named by another table, or is there no free one."""
    page = 16
    for columns, add in ((4, 20), (30, 300)):
        table, refs = np.full((3, columns), -1), np.zeros(90)
        n = 3 if columns == 4 else 25
        table[0, :n], refs[:n] = np.arange(n), 1
        refs[1] += 1  # another table names it
        k = Pair(table, refs, [n * page - 8, 0, 0], page)
        k.fork([0, 0, 0])
        k.set_len([n * page - 8, 20, 0])
        k.reserve([4, add, 0])
        end = -(-(20 + add) // page)
        assert k.refs[k.table[1, 1:end].long()].tolist() == [1] * (end - 1)
        k.fork([0, 1, 0])
        k.set_len([3, 0, 16])
        k.reserve([1, 17, add])
        k.set_len([0, 0, 0])
        k.reserve([add, add, add])
    k = Pair([[0, 1], [0, 1]], [2, 2], [16, 0], page)  # none is free
    k.reserve([0, 32])
    assert k.table.tolist() == [[0, 1], [-1, -1]]
    k = Pair([[0, 0, 0], [1, 2, 1]], [3, 2, 1], [5, 5], page)  # a row that names a page several times
    k.reserve([30, 30])


def test_rows_go_round_in_a_circle():
    for b in (2, 3, 300, 1500):
        k = books(b, b, 6, 8 * b, 16, full=0.8)
        k.fork(np.roll(np.arange(b), 1))
        k.fork(np.arange(b)[::-1])
        k.fork(np.zeros(b))


def test_most_questions():
    """4096 rows: the most a call takes."""
    k = books(3, 4096, 3, 9000, 16, full=1.0)
    k.fork(np.random.default_rng(0).integers(0, 4096, 4096))
    k.reserve(np.ones(4096))
    k.trim()
    k.compact()


@pytest.mark.parametrize("free", [0, 1, 2, 5, 6, 7, 30])
def test_pages_run_out(free):
    """Served in order; from the first that does not fit on, nothing changes, though a later one could do with what it has."""
    page = 16
    table = np.full((6, 8), -1)
    refs = np.zeros(6 + free)
    for u, n in enumerate((1, 1, 1, 1)):
        table[u, 0] = u
    table[4, 0] = 0  # shares its last page with the first
    refs[[0, 1, 2, 3, 4, 5]] = [2, 1, 1, 1, 1, 1]
    k = Pair(table, refs, [5, 5, 16, 3, 5, 0], page)
    k.reserve([30, 2, 40, 1, 1, 16])


def test_last_page_shared_by_all_that_write():
    """The last of those that share a page keeps it, as long as no other table names it."""
    for others in (0, 1):
        table = np.full((4, 4), -1)
        table[:, 0] = 7
        refs = np.zeros(20)
        refs[7] = 4 + others
        k = Pair(table, refs, [3, 9, 16, 9], 16)  # (the third's is whole: it does not write to it)
        c, n = k.reserve([1, 1, 1, 1])
        assert int(n) == 3
        k.reserve([100, 1, 1, 1])  # (the first does not fit into its row)


def test_questions_that_cannot_be_served():
    """A last page that is not there, a row that is too short, lengths that mean nothing: left as they are."""
    table = np.full((7, 2), -1)
    table[1], table[3, 0] = [0, 1], 2
    refs = np.zeros(30)
    refs[[0, 1, 2]] = 1
    big = 2 ** 31 - 1
    k = Pair(table, refs, [5, 30, -3, 16, big, 0, 0], 16)
    k.reserve([1, 3, 4, 17, 1, 33, big])
    k.fork([4, 1, 2, 2, 4, 5, 6])
    k.set_len([-3, 31, 2, 16, big, 0, 5])
    k.trim()


def test_more_pages_than_one_step_looks_at():
    """Free pages far behind, between full stretches; entries that are there already in the middle of the range."""
    pages = 70001
    refs = np.ones(pages)
    refs[[4095, 4096, 8191, 65535, 65536, 70000]] = 0
    table = np.full((3, 90), -1)
    refs[[1, 2, 3]] = [1, 1, 1]
    table[0, 2], table[1, 70], table[2, 1] = 1, 2, 3
    k = Pair(table, refs, [0, 0, 0], 16)
    k.reserve([48, 0, 64])
    k.set_len([0, 0, 0])
    k.trim()
    refs = np.zeros(pages)
    refs[np.random.default_rng(1).permutation(pages)[:33000]] = 2
    k = Pair(np.random.default_rng(2).permutation(np.nonzero(refs)[0])[:600].reshape(6, 100), refs, [0] * 6, 16)
    k.reserve([0] * 6)
    k.compact()
    k.reserve([0] * 5 + [1600])
    k = Pair(np.full((40, 1500), -1), np.zeros(pages), [0] * 40, 16)
    k.reserve(np.random.default_rng(3).integers(0, 24001, 40))


@pytest.mark.parametrize("pages,live", [(1, 0), (1, 1), (2, 1), (5000, 0), (5000, 5000), (4097, 4096), (8192, 1)])
def test_compact_ends(pages, live):
    refs = np.zeros(pages)
    refs[pages - live:] = 3
    k = Pair(np.full((1, 1), pages - 1 if live else -1), refs, [0], 16)
    k.compact()
    before = k.refs.clone()
    k.compact()  # nothing is left to move
    assert torch.equal(k.refs, before)


def test_compact_without_a_table():
    refs = dev([0, 2, 0, 1, 1])
    copies, counts, place = B.dbsa_pages_compact(refs, None, 16)
    assert counts.tolist() == [2, 3] and copies[:2].tolist() == [[3, 0, 16], [4, 2, 16]]
    assert place.tolist() == [-1, 1, -1, 0, 2] and refs.tolist() == [1, 2, 1, 0, 0]


# ---- copies ----------------------------------------------------------------------------------------------------

def cache(seed, shape, dtype):
    """Any bits at all, those of no numbers among them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    size = torch.empty(0, dtype=dtype).element_size()
    return torch.randint(0, 256, (*shape[:-1], shape[-1] * size), generator=g, device="cuda", dtype=torch.uint8).view(dtype)


def bits(x):
    return x.contiguous().view(torch.uint8)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.uint8, torch.float8_e4m3fn])
@pytest.mark.parametrize("heads,dim,page", [(8, 128, 64), (1, 64, 16), (5, 64, 32), (3, 128, 256)])
@pytest.mark.parametrize("layers", [0, 1, 3])
def test_copies(dtype, heads, dim, page, layers):
    shape = (11, page, heads, dim) if layers == 0 else (layers, 11, page, heads, dim)
    k, v = cache(1, shape, dtype), cache(2, shape, dtype)
    list_ = [(3, 0, page), (4, 1, 1), (4, 2, page - 1), (5, 6, 7), (-1, 7, 5), (3, 11, 5), (11, 8, 5), (9, 9, 5), (10, 8, 0), (10, 7, -4),
             (3, 10, page + 99), (0, 9, 3)]
    want = [bits(x).clone() for x in (k, v)]
    for w in want:
        w = w if layers else w[None]
        for a, b, rows in list_[:11]:
            if 0 <= a < 11 and 0 <= b < 11:
                w[:, b, :max(0, min(rows, page))] = w[:, a, :max(0, min(rows, page))].clone()
    B.dbsa_pages_copy(k, v, dev(list_), dev([11]))
    torch.cuda.synchronize()
    assert torch.equal(bits(k), want[0]) and torch.equal(bits(v), want[1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.uint8])
def test_copies_with_strides(dtype):
    """Heads first in a page; K and V interleaved; tokens further apart than their heads fill."""
    base = cache(3, (2, 9, 4, 32, 2, 64), dtype)          # [layer, page, head, token, k or v, D]
    want = bits(base).view(2, 9, 4, 32, 2, -1).clone()
    k, v = base[:, :, :, :, 0].transpose(2, 3), base[:, :, :, :, 1].transpose(2, 3)
    B.dbsa_pages_copy(k, v, dev([(0, 8, 32), (1, 7, 13)]), dev([2]))
    want[:, 8] = want[:, 0]
    want[:, 7, :, :13] = want[:, 1, :, :13]
    torch.cuda.synchronize()
    assert torch.equal(bits(base).view_as(want), want)


@pytest.mark.parametrize("count,done", [(0, 0), (-5, 0), (2, 2), (99, 3)])
def test_copies_that_count(count, done):
    k, v = cache(4, (8, 16, 2, 64), torch.float32), cache(5, (8, 16, 2, 64), torch.float32)
    want = k.clone()
    for a, b in [(0, 5), (1, 6), (2, 7)][:done]:
        want[b] = want[a]
    B.dbsa_pages_copy(k, v, dev([(0, 5, 16), (1, 6, 16), (2, 7, 16)]), dev([count]))
    assert torch.equal(bits(k), bits(want))


def test_many_copies_in_many_layers():
    k, v = cache(6, (5, 700, 16, 2, 64), torch.bfloat16), cache(7, (5, 700, 16, 2, 64), torch.bfloat16)
    want = [x.clone() for x in (k, v)]
    rng = np.random.default_rng(8)
    to = rng.permutation(350) + 350
    list_ = [(int(rng.integers(0, 350)), int(t), int(rng.integers(1, 17))) for t in to]
    for x in want:
        orc.copy_rows(x, list_)
    B.dbsa_pages_copy(k, v, dev(list_), dev([350]))
    assert torch.equal(bits(k), bits(want[0])) and torch.equal(bits(v), bits(want[1]))


# ---- together --------------------------------------------------------------------------------------------------

def attend(lay, q, pool, k, v, table, n):
    return B.dbsa_chunk_attn(lay, q, pool[0], pool[1], k, v, table, n, 0.125)


def test_a_conversation_that_branches():
    """Prompts come in, answers branch, proposed tokens are attended, checked and cut back, the arena is tidied up: after each step the
    attention over the shared pages gives, bit for bit, what it gives over pages of each question's own."""
    b, heads, dim, page, pages, columns, vocab = 6, 2, 64, 16, 64, 9, 300
    gen = torch.Generator(device="cuda").manual_seed(11)
    randn = lambda *s: torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16)  # noqa: E731
    pool = randn(34, heads, dim), randn(34, heads, dim)
    k, v = randn(1, pages, page, heads, dim), randn(1, pages, page, heads, dim)
    table = torch.full((b, columns), -1, dtype=torch.int32, device="cuda")
    refs, n = torch.zeros(pages, dtype=torch.int32, device="cuda"), torch.zeros(b, dtype=torch.int32, device="cuda")
    truth = [[] for _ in range(b)]  # (k, v) of each question's tokens
    own_table = torch.arange(b * columns, dtype=torch.int32, device="cuda").view(b, columns)

    def chunk(new):
        """New tokens: room, keys, attention."""
        got, copies, count = B.dbsa_pages_reserve(table, refs, n, dev(new), page)
        assert got.tolist() == list(new)
        B.dbsa_pages_copy(k, v, copies, count)
        length = n.tolist()
        for u in range(b):
            for j in range(length[u] - new[u], length[u]):
                truth[u].append((randn(heads, dim), randn(heads, dim)))
                at = int(table[u, j // page])
                k[0, at, j % page], v[0, at, j % page] = truth[u][-1]
        cu = np.concatenate([[0], np.cumsum(new)])
        lay = B.dbsa_layout_build_chunk(4, [4, 14, 34], [0, 1, 2], cu_qlens=cu, sel_ptr=np.arange(b + 1), sel_idx=[0, 1] * (b // 2), n_q_heads=4,
                                        n_kv_heads=heads, own_tokens=length)
        q = randn(int(cu[-1]), 4, dim)
        return lay, q, compare(lay, q)

    def compare(lay, q):
        k2, v2 = torch.zeros(b * columns, page, heads, dim, dtype=k.dtype, device="cuda"), torch.zeros(b * columns, page, heads, dim, dtype=k.dtype, device="cuda")
        for u in range(b):
            for j, (x, y) in enumerate(truth[u]):
                k2[u * columns + j // page, j % page], v2[u * columns + j // page, j % page] = x, y
        here = attend(lay, q, pool, k[0], v[0], table, n)
        want = attend(lay, q, pool, k2, v2, own_table, n)
        assert torch.equal(bits(here), bits(want))
        return here

    chunk([21, 1, 37, 1, 30, 1])
    source = [0, 0, 2, 0, 2, 2]
    B.dbsa_pages_fork(table, refs, n, dev(source), page)
    truth = [list(truth[s]) for s in source]
    for step in range(5):
        new = [4, 3, 1, 4, 2, 4]
        lay, q, o = chunk(new)
        # the model's scores are whatever comes of the attention
        logits = (o.float().reshape(o.shape[0], -1) @ torch.randn((4 * dim, vocab), generator=gen, device="cuda"))
        cu = dev(np.concatenate([[0], np.cumsum(new)]))
        tokens = torch.randint(0, vocab, (o.shape[0],), generator=gen, device="cuda", dtype=torch.int32)
        likely = logits.argmax(1).to(torch.int32)
        tokens[1:] = torch.where(torch.rand(o.shape[0] - 1, generator=gen, device="cuda") < 0.7, likely[:-1], tokens[1:])
        uniform = torch.rand(o.shape[0], generator=gen, device="cuda")
        out, accepted = B.dbsa_draft_verify(logits, tokens, cu, uniform, temperature=torch.zeros(b, device="cuda"), self_len=n, new_len=n)
        want = orc.draft_verify(logits.double().cpu().numpy(), tokens.tolist(), cu.tolist(), uniform.tolist(), temperature=[0.0] * b)
        assert out.tolist() == want["out"].tolist() and accepted.tolist() == want["accepted"].tolist()
        truth = [x[:len(x) - (t - 1 - a)] for x, t, a in zip(truth, new, accepted.tolist())]
        assert n.tolist() == [len(x) for x in truth]
        B.dbsa_pages_trim(table, refs, n, page)
        if step == 2:
            B.dbsa_pages_fork(table, refs, n, dev([0, 5, 2, 1, 4, 3]), page)
            truth = [list(truth[s]) for s in (0, 5, 2, 1, 4, 3)]
        if step >= 2:
            copies, counts, _ = B.dbsa_pages_compact(refs, table, page)
            B.dbsa_pages_copy(k, v, copies, counts)
            assert (refs[:int(counts[1])] > 0).all() and (refs[int(counts[1]):] == 0).all()
        named = table[table >= 0].cpu().numpy()
        assert (np.bincount(named, minlength=pages) == refs.cpu().numpy()).all()
        lay = B.dbsa_layout_build_chunk(4, [4, 14, 34], [0, 1, 2], cu_qlens=np.arange(b + 1), sel_ptr=np.arange(b + 1), sel_idx=[0, 1] * (b // 2),
                                        n_q_heads=4, n_kv_heads=heads, own_tokens=n.tolist())
        compare(lay, randn(b, 4, dim))


def test_a_step_as_a_graph():
    """fork, reserve, copy, trim, compact, copy recorded once, replayed with other books, eager calls between."""
    b, columns, pages, page = 12, 20, 400, 16
    start = [books(s, b, columns, pages, page, stray=False) for s in range(4)]
    live = books(9, b, columns, pages, page, stray=False)
    k, v = cache(1, (2, pages, page, 2, 64), torch.bfloat16), cache(2, (2, pages, page, 2, 64), torch.bfloat16)
    source, add = dev(np.arange(b)), dev(np.zeros(b))
    kept = dict(got=dev(np.zeros(b)), copies=dev(np.zeros((b, 3))), n_copies=dev([0]), workspace=dev(np.zeros(pages)))
    moves = dict(copies=dev(np.zeros((pages // 2, 3))), counts=dev([0, 0]), new_place=dev(np.zeros(pages)))

    def step():
        B.dbsa_pages_fork(live.table, live.refs, live.self_len, source, page)
        B.dbsa_pages_reserve(live.table, live.refs, live.self_len, add, page, **kept)
        B.dbsa_pages_copy(k, v, kept["copies"], kept["n_copies"])
        live.self_len.sub_(5).clamp_(min=0)
        B.dbsa_pages_trim(live.table, live.refs, live.self_len, page)
        B.dbsa_pages_compact(live.refs, live.table, page, **moves)
        B.dbsa_pages_copy(k, v, moves["copies"], moves["counts"])

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
    stream.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    rng = np.random.default_rng(4)
    for turn in range(6):
        first = start[turn % 4]
        live.want = orc.Books(first.want.table, first.want.refs, first.want.self_len, page)
        for x in ("table", "refs", "self_len"):
            getattr(live, x).copy_(dev(getattr(first.want, x)))
        s, a = rng.integers(0, b, b), rng.integers(0, 20, b)
        source.copy_(dev(s))
        add.copy_(dev(a))
        want = [x.clone() for x in (k, v)]
        (g.replay if turn % 3 else step)()
        live.want.fork(s)
        got, copies = live.want.reserve(a)
        live.want.self_len = np.maximum(live.want.self_len - 5, 0)
        live.want.trim()
        more, _, _ = live.want.compact()
        for x in want:
            orc.copy_rows(x, copies)
            orc.copy_rows(x, more)
        live.check(f"turn {turn}")
        assert torch.equal(bits(k), bits(want[0])) and torch.equal(bits(v), bits(want[1]))


def test_books_give_the_rows_the_chunk_attention_reads():
    """The oracle of the chunk attention and the books agree where token j of a question lies."""
    k = books(21, 5, 7, 60, 16, stray=False)
    k.reserve([9, 1, 30, 2, 5])
    for u in range(5):
        rows, j = chunk_oracle.own_rows(k.table[u].tolist(), int(k.self_len[u]), 16, 60)
        assert len(j) == int(k.self_len[u]) and (rows // 16 == k.want.table[u][j // 16]).all()
