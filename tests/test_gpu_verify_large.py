"""Verification in the forms that large batches take, against the fp64 oracle: many questions (decided in a launch of their own, drawn in
another), and many values (statistics in pieces of 8192, the draw's walk through such a piece).  What has to be equal: as in
test_gpu_verify.py; of a random number of 1 see `alike`."""
import numpy as np
import pytest
import torch

from oracle import steps_oracle as orc
from paper_2503_08640_amd import binding as B
from test_gpu_verify import call, dev, make, same, wanted

pytestmark = pytest.mark.gpu


def workgroups(b, vocab, draft):
    """Of the draw from logits: above 1536 of them the decision has a launch of its own."""
    shares = -(-vocab // 512)
    most = -(-shares // 4)
    each = 4 * (-(-b * most // 2048) if draft else most)
    return b * -(-shares // each)


def values(c):
    """Looked at by the statistics: from 2^25 on in pieces of 8192."""
    return c["x"].numel() * (1 if c["y"] is None else 2)


def spoil(c, seed):
    """Proposals that are none, certain ones, equal distributions that stand throughout or are refused without a weight left."""
    rng = np.random.default_rng(seed)
    n = len(c["tokens"])
    c["tokens"][rng.random(n) < 0.05] = -1
    c["uniform"][rng.random(n) < 0.2] = 0.0
    c["uniform"][rng.random(n) < 0.05] = 1.0 - 2.0 ** -24
    rows = np.diff(c["cu"])
    if c["y"] is not None:
        for u in np.nonzero(rng.random(len(rows)) < 0.2)[0]:
            k = rows[u] - 1
            if k > 0:
                c["y"][u, :k] = c["x"][c["cu"][u]:c["cu"][u] + k]
        c["uniform"][rng.random(n) < 0.05] = 1.0
    return c


def alike(c):
    """Questions that a number of 1 refuses or not by what 64 bits round away.  The kernel holds p and q to 2.1e-12 of them (the
    exponential 2e-12, each sum, inverse and product a few 1e-16), the oracle to 1e-15, so that q - p can have either sign where
    |q - p| <= 2.2e-12 (p + q) <= 4.4e-12 of the larger, as between two distributions that are 1 at one token and e-100 beside it: twice
    that is left out.  Rows that are equal bit by bit give equal p and q on both sides.  (A random number below 1 comes as near to
    p / q with a probability of 1e-11.)"""
    out = np.zeros(len(c["cu"]) - 1, bool)
    if c["y"] is None:
        return out
    for u in range(len(out)):
        heat = 1.0 if c["heat"] is None else float(c["heat"][u])
        for a, row in enumerate(range(c["cu"][u], c["cu"][u + 1] - 1)):
            x = int(c["tokens"][row + 1])
            if c["uniform"][row] != 1.0 or x < 0 or not heat > 0 or torch.equal(c["x"][row], c["y"][u, a]):
                continue
            p, q = (orc.distribution(z.double().numpy(), heat, False)[0][x] for z in (c["x"][row], c["y"][u, a]))
            out[u] |= abs(p - q) <= 8e-12 * max(p, q)
    return out


def check(c, what):
    """The oracle's outcome; at most one question in a hundred may be left out."""
    got, want, out = call(c), wanted(c), alike(c)
    assert out.mean() <= 0.01
    for u in np.nonzero(out)[0]:
        lo, hi = c["cu"][u], c["cu"][u + 1]
        for key in ("out", "logp"):
            want[key][lo:hi] = got[key][lo:hi]
        want["accepted"][u] = got["accepted"][u]
    same(got, want, c, what)


def heats(seed, b):
    return [float(x) for x in np.random.default_rng(seed).choice([0.0, 0.6, 1.0, 1.3, float("nan"), 1e-3], b)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("heat", [None, "mixed", "greedy"])
def test_many_questions(dtype, draft, heat):
    """A workgroup to each question's draw; some have no rows."""
    b = 1700
    rows = [int(x) for x in np.random.default_rng(b).integers(0, 5, b)]
    c = spoil(make(400, rows, 301, dtype, draft=draft, heat={None: None, "mixed": heats(1, b), "greedy": [0.0] * b}[heat]), 2)
    assert workgroups(b, 301, draft) > 1536
    check(c, f"1700 questions {dtype} draft {draft} heat {heat}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_questions_with_several_workgroups_each(dtype):
    b, vocab = 400, 10007
    rows = [int(x) for x in np.random.default_rng(b).integers(0, 5, b)]
    c = spoil(make(410, rows, vocab, dtype, heat=heats(3, b)), 4)
    assert workgroups(b, vocab, True) > 1536 > b
    check(c, f"400 questions of 10007 words {dtype}")


VOCAB = 300001  # (no multiple of any piece)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b", [15, 40])
def test_many_values(b, dtype):
    """Proposals with distributions; with and without a launch for the decisions."""
    c = spoil(make(420 + b, [4] * (b - 1) + [1], VOCAB, dtype, heat=heats(5, b), spread=1.0), 6)
    assert values(c) >= 1 << 25 and (workgroups(b, VOCAB, True) > 1536) == (b == 40)
    check(c, f"{b} questions of {VOCAB} words {dtype}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [[1] * 120, [4, 3] * 17, [0, 9, 1] * 12])
def test_many_values_without_distributions(rows, dtype):
    """Tokens drawn one to a question, and looked-up proposals that stand, are refused or have all there is: each draw walks through the
    shares of one piece, from sums with or without the proposal."""
    b = len(rows)
    for heat in (None, heats(7, b)):
        c = spoil(make(430, rows, VOCAB, dtype, draft=False, heat=heat, spread=0.5), 8)
        assert values(c) >= 1 << 25
        rng = np.random.default_rng(9)
        for u in np.nonzero((np.array(rows) > 1) & (rng.random(b) < 0.7))[0]:
            row = int(c["cu"][u])  # the first proposal has nearly everything, or everything, and is refused now and then
            x = int(c["tokens"][row + 1])
            if x < 0:
                continue
            if rng.random() < 0.3:
                c["x"][row] = -float("inf")
            c["x"][row, x] = float(rng.choice([9.0, 25.0, 60.0]))
            c["uniform"][row] = rng.choice([0.5, 1.0 - 2.0 ** -24, 1.0])
        check(c, f"looked up, {b} questions of {VOCAB} words {dtype} heat {heat is not None}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [True, False])
def test_many_values_masked(dtype, draft):
    """Whole stretches without a value, or with the type's lowest, infinite values, rows of no numbers: pieces that are gone through
    once more."""
    b, inf = 32, float("inf")
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    c = make(440, [4] * b, VOCAB, dtype, draft=draft, heat=heats(10, b), spread=1.0)
    assert values(c) >= 1 << 25
    rng = np.random.default_rng(11)
    for row in range(0, 4 * b, 3):
        hide = torch.from_numpy(rng.random(VOCAB) < 0.999)
        c["x"][row, hide] = [-inf, low, -1e9, -1e4][row // 3 % 4]
        c["x"][row, :VOCAB // 2] = [-inf, low, -1e9, -1e4][row // 3 % 4]
    c["x"][5, 250000:] = inf
    c["x"][9], c["x"][13] = float("nan"), -inf
    c["x"][18, 123456] = 3e5
    c["x"][22] = c["x"][22].clamp_min(-10) * 1e30
    if draft:
        c["y"][1, 1], c["y"][2, 0], c["y"][7, 2, :200000] = low, float("nan"), low
        c["y"][4, 0] = c["y"][4, 0] + 3e6
    check(c, f"masked {VOCAB} words {dtype} draft {draft}")


def test_replayed_with_one_workspace():
    """Both forms recorded, replayed in turn with other numbers, an eager call of another batch over the same workspace between."""
    batches = [make(450, [int(x) for x in np.random.default_rng(1).integers(0, 4, 1600)], 301, "f32", heat=heats(12, 1600)),
               make(451, [4] * 15, VOCAB, "bf16"), make(452, [1] * 120, VOCAB, "f32", draft=False)]
    assert workgroups(1600, 301, True) > 1536 and min(values(c) for c in batches[1:]) >= 1 << 25
    ws = torch.empty(max(B.dbsa_draft_verify_workspace_bytes(c["x"].shape[0], len(c["cu"]) - 1, c["x"].shape[1]) for c in batches),
                     dtype=torch.uint8, device="cuda")
    made = []
    for c in batches:
        t = {x: dev(c[x]) for x in ("x", "y", "tokens", "cu", "uniform", "heat")}
        t["out"], t["acc"] = torch.empty_like(t["tokens"]), torch.empty_like(t["cu"][1:])
        run = lambda t=t: B.dbsa_draft_verify(t["x"], t["tokens"], t["cu"], t["uniform"], draft=t["y"], temperature=t["heat"],  # noqa: E731
                                              out=t["out"], accepted=t["acc"], workspace=ws)
        run()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        made.append((c, t, g, run))
    for turn in range(3):
        for i, (c, t, g, _) in enumerate(made):
            c["uniform"] = np.random.default_rng(turn).random(len(c["uniform"])).astype(np.float32)
            t["uniform"].copy_(torch.from_numpy(c["uniform"]))
            t["out"].fill_(-5)
            g.replay()
            made[(i + 1) % 3][3]()
            want = wanted(c)
            torch.cuda.synchronize()
            assert (t["out"].cpu().numpy() == want["out"]).all() and (t["acc"].cpu().numpy() == want["accepted"]).all(), (turn, i)
