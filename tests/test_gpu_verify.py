"""Verification of drafted tokens on the GPU against the float64 oracle.

What comes out are tokens, which have to be equal.  A decision can go the other way only where it is nearer to its
border than the probabilities are exact: an exponential is fp32 (2^-22 of itself, and of its exponent x log2(e), |x| up
to 40, two roundings of 2^-24 each: 2^-24 * 40 * 2 ln 2 < 2^-17 for the smallest, whose mass is e^-40, and 2^-21 for those
that count), sums are 64-bit: probabilities and running sums are right to 2^-20 of 1, and the two of a difference to 2^-19.
Where max(p - q, 0) is drawn from, its total is smaller than 1: the margin in units of it counts 20 times, as the tests'
distributions differ by 5% or more.  So decisions with a margin above 20 * 2^-19 = 4e-5 have to agree; the others are counted.
"""
import numpy as np
import pytest

from oracle import pipo_oracle as O

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def _api():
    import paper_2605_27255_amd as P
    return P


def _rows(rng, n, V, peaks=10):
    """A broad floor, and in long rows a few tokens that hold nearly all of the probability."""
    x = 1.5 * rng.standard_normal((n, V))
    for r in range(n):
        x[r, rng.integers(0, V, min(peaks, V))] += 3 * rng.random(min(peaks, V)) + (np.log(V) + 3 if V > 100 else 0)
    return x


def _case(seed, R, K, V, dtype, near=0.5):
    """float64 values of the type: target rows [R (K + 1), V], drafter rows [R, K, V], drafts, random numbers."""
    rng = np.random.default_rng(seed)
    rnd = lambda x: torch.tensor(x).to(dtype).double().numpy()  # noqa: E731
    p = rnd(_rows(rng, R * (K + 1), V))
    q = rnd(p.reshape(R, K + 1, V)[:, :K] + near * rng.standard_normal((R, K, V)))
    e = np.exp(q - q.max(2, keepdims=True))
    cum = np.cumsum(e / e.sum(2, keepdims=True), 2)
    drafts = (rng.random((R, K, 1)) > cum).sum(2).clip(max=V - 1)
    return p, q, drafts, rng.random((R, K + 1)).astype(np.float32)


def _run(p, q, drafts, u, dtype, starts=None, temperature=1.0, pad=0):
    def gpu(x):
        y = torch.full((*x.shape[:-1], x.shape[-1] + pad), float("nan"), dtype=dtype, device="cuda")
        y[..., :x.shape[-1]] = torch.tensor(x).to(dtype).cuda()
        return y[..., :x.shape[-1]]
    i32 = lambda x: None if x is None else torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")  # noqa: E731
    t, a = _api().verify_drafts(gpu(p), i32(drafts), torch.tensor(u, dtype=torch.float32).cuda(), None if q is None else gpu(q),
                                i32(starts), temperature)
    torch.cuda.synchronize()
    return t.cpu().numpy(), a.cpu().numpy()


def _check(p, q, drafts, u, dtype, starts=None, temperature=1.0, pad=0, most=0.2):
    want, accepted, margin = O.verify_drafts(p, drafts, u.astype(np.float64), q, starts, temperature)
    t, a = _run(p, q, drafts, u, dtype, starts, temperature, pad)
    sure = margin > 4e-5
    np.testing.assert_array_equal(a[sure], accepted[sure])
    np.testing.assert_array_equal(t[sure], want[sure])
    assert (~sure).mean() <= most, (~sure).mean()
    for r in range(len(a)):             # in any case: the drafts up to the accepted number, one token, nothing behind
        assert (t[r, :a[r]] == drafts[r, :a[r]]).all() and (t[r, a[r] + 1:] == -1).all()
    return t, a


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 17, 1000, 8191, 8192, 8193, 20011])
@pytest.mark.parametrize("K", [0, 1, 4])
@pytest.mark.parametrize("drafter", [True, False])
def test_verify(dtype, V, K, drafter):
    p, q, d, u = _case([V, K], 24, K, V, dtype)
    _check(p, q if drafter else None, d, u, dtype, pad=V % 3, most=0.35)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_verify_the_whole_vocabulary(dtype):
    p, q, d, u = _case(5, 3, 2, 151936, dtype)
    _check(p, q, d, u, dtype, temperature=0.6, most=0.7)
    p, q, d, u = _case(6, 1, 1, 524288, dtype)
    _check(p, q, d, u, dtype, most=1.0)


@pytest.mark.parametrize("temperature", [0.3, 0.6, 1.0, 2.5])
def test_verify_temperatures(temperature):
    p, q, d, u = _case(7, 40, 3, 500, torch.float32)
    _check(p, q, d, u, torch.float32, temperature=temperature)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [5, 1000, 30000])
def test_verify_greedy(dtype, V):
    p, q, d, u = _case([8, V], 20, 5, V, dtype)
    d[:, :3] = p.reshape(20, 6, V)[:, :3].argmax(2)
    d[::4, 3:] = p.reshape(20, 6, V)[::4, 3:5].argmax(2)
    p[7, :] = 2.0                       # ties: the lowest id
    want, accepted, _ = O.verify_drafts(p, d, u, q, None, 0.0)
    for temperature in (0.0, -1.0):
        t, a = _run(p, q, d, u, dtype, None, temperature)
        np.testing.assert_array_equal(t, want)
        np.testing.assert_array_equal(a, accepted)
    assert accepted.max() == 5 and len(set(accepted)) > 1


def test_verify_63_drafts():
    p, q, d, u = _case(9, 5, 63, 50, torch.float32, near=0.05)
    t, a = _check(p, q, d, u, torch.float32, most=0.6)
    d[0, 40:], d[1, 0] = -1, -1
    _check(p, q, d, u, torch.float32, most=0.6)


def test_verify_ragged_rows():
    """Rows by starts: requests without rows, with fewer rows than drafts, with more; drafts that end early."""
    p, q, d, u = _case(10, 6, 3, 300, torch.float32)
    starts = np.array([0, 4, 4, 6, 7, 13, 15])
    p = p[:20]
    d[0, 1] = -1
    d[5] = -1
    t, a = _check(p, q, d, u, torch.float32, starts=starts, most=0.5)
    assert a[1] == 0 and (t[1] == -1).all() and a[2] <= 1 and a[3] == 0 and a[5] == 0 and (t[[0, 2, 3, 4, 5], 0] >= 0).all()
    for bad in ([0, 4, 2 ** 31 - 1, 3, 7, -5, 100], [19, 21, 30, 40, 50, 60, 70]):      # nonsense: nothing out of bounds
        _run(p, q, d, u, torch.float32, starts=np.array(bad))


def test_verify_masked_logits_and_bad_rows():
    p, q, d, u = _case(11, 8, 2, 400, torch.float32)
    p[:, 100:] = -np.inf                # the target allows only some tokens
    q[:, :, 50:60] = -np.inf
    d = np.minimum(d, 399)
    _check(p, q, d, u, torch.float32, most=0.5)
    lowest = float(torch.finfo(torch.float32).min)
    p2 = np.where(np.isinf(p), lowest, p)
    _check(p2, q, d, u, torch.float32, most=0.5)
    for bad in (np.nan, np.inf, None):
        p2, q2 = p.copy(), q.copy()
        if bad is None:
            p2[0], p2[4], q2[2, 0] = -np.inf, -np.inf, -np.inf
        else:
            p2[0, 5], p2[4, 7], q2[2, 0, 9] = bad, bad, bad
        t, a = _check(p2, q2, d, u, torch.float32, most=0.5)
        assert a[0] == 0 and t[0, 0] == -1 and a[2] == 0 and t[2, 0] == -1


def test_verify_logits_of_any_magnitude():
    p, q, d, u = _case(12, 10, 2, 300, torch.float32)
    for shift, size in ((1e6, 1.0), (-3e4, 1.0), (0.0, 1e30), (3e38, 0.0)):
        a = (p * size + shift).astype(np.float32).astype(np.float64)
        b = (q * size + shift).astype(np.float32).astype(np.float64)
        _check(a, b, d, u, torch.float32, most=0.5)


def test_verify_numbers_at_the_ends():
    """Drafts outside the vocabulary, random numbers of 0, 1 and NaN, a draft that is certain, p = q."""
    p, q, d, u = _case(13, 6, 1, 100, torch.float32)
    d[0], u[0, 1] = 100, 0.0
    d[1], u[1, 0], u[1, 1] = 2 ** 31 - 1, 0.0, 1.0
    q[2] = p[4]                         # p = q: every number below 1 accepts
    u[2, 0] = np.float32(0.999)
    u[3, 0], u[3, 1] = np.nan, np.nan   # NaN accepts nothing and draws the last token of positive mass
    t, a = _run(p, q, d, u, torch.float32)
    want, accepted, _ = O.verify_drafts(p, d, u.astype(np.float64), q)
    np.testing.assert_array_equal(a[[0, 1, 2, 3]], [0, 0, 1, 0])
    assert t[0, 0] == want[0, 0] and t[1, 0] == np.flatnonzero(_left(p[2], q[1, 0]))[-1]
    assert t[3, 0] == np.flatnonzero(_left(p[6], q[3, 0]))[-1]
    # p nowhere above q (here: equal, and the number says no): drawn from p itself
    q[2], u[2, 0] = p[4], 1.0
    t, a = _run(p, q, d, u, torch.float32)
    want, _, margin = O.verify_drafts(p, d, u.astype(np.float64), np.concatenate([q[:2], p[4][None, None], q[3:]]))
    assert a[2] == 0 and 0 <= t[2, 0] < 100
    # not drawn, and certain: rejected only by a number of 1, then there is nothing else
    p[0] = -np.inf
    p[0, 42], d[0], u[0, 0] = 1.0, 42, 0.999
    assert _run(p, None, d, u, torch.float32)[1][0] == 1
    u[0, 0] = 1.0
    t, a = _run(p, None, d, u, torch.float32)
    assert a[0] == 0 and t[0, 0] == 42


def _left(p, q):
    e, f = np.exp(p - p.max()), np.exp(q - q.max())
    x = e / e.sum() - f / f.sum()
    return np.where(x > 1e-9, x, 0)


def test_verified_tokens_are_distributed_as_the_target():
    """20000 requests with the same rows: the first token's frequencies are p's (each within 5 standard deviations)."""
    n, V = 20000, 7
    rng = np.random.default_rng(14)
    p, q = rng.standard_normal(V) * 1.5, rng.standard_normal(V) * 1.5
    P, Q = np.exp(p) / np.exp(p).sum(), np.exp(q) / np.exp(q).sum()
    d = rng.choice(V, size=(n, 1), p=Q)
    u = rng.random((n, 2))
    for drafter in (True, False):
        t, _ = _run(np.broadcast_to(p, (2 * n, V)).copy(), np.broadcast_to(q, (n, 1, V)).copy() if drafter else None, d, u,
                    torch.float32)
        # (without the drafter's logits a draft counts as certain, whatever it is: the same distribution)
        f = np.bincount(t[:, 0], minlength=V) / n
        assert (np.abs(f - P) <= 5 * np.sqrt(P * (1 - P) / n)).all()


def test_verify_captured_into_a_graph_and_on_two_streams():
    cases = [_case([15, i], 16, 3, 5000, torch.bfloat16) for i in range(3)]
    want = [_run(*c, torch.bfloat16) for c in cases]
    gpu = [[torch.tensor(x).to(y).cuda() for x, y in zip(c, (torch.bfloat16, torch.bfloat16, torch.int32, torch.float32))] for c in cases]
    hold = [x.clone() for x in gpu[0]]
    A = _api()
    A.verify_drafts(hold[0], hold[2], hold[3], hold[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = A.verify_drafts(hold[0], hold[2], hold[3], hold[1])
    for i in (1, 0, 2, 1):
        for x, y in zip(hold, gpu[i]):
            x.copy_(y)
        graph.replay()
        A.verify_drafts(gpu[2][0], gpu[2][2], gpu[2][3], gpu[2][1])
        torch.cuda.synchronize()
        for x, y in zip(out, want[i]):
            np.testing.assert_array_equal(x.cpu().numpy(), y)
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(A.verify_drafts(gpu[i][0], gpu[i][2], gpu[i][3], gpu[i][1]))
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i]:
            for y, z in zip(x, want[i]):
                np.testing.assert_array_equal(y.cpu().numpy(), z)


def test_python_calls_refuse_what_does_not_fit():
    A = _api()
    z, d, u = torch.zeros((8, 50), device="cuda"), torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 4), device="cuda")
    q = torch.zeros((2, 3, 50), device="cuda")
    bad = [lambda: A.verify_drafts(z[:7], d, u), lambda: A.verify_drafts(z, d.long(), u), lambda: A.verify_drafts(z, d, u[:, :3]),
           lambda: A.verify_drafts(z, d, None), lambda: A.verify_drafts(z, d, u.double()), lambda: A.verify_drafts(z, d, u, q[:, :2]),
           lambda: A.verify_drafts(z, d, u, q.bfloat16()), lambda: A.verify_drafts(z, d, u, q[:, :1].expand(2, 3, 50)),
           lambda: A.verify_drafts(z, d, u, starts=d[0, :2]), lambda: A.verify_drafts(z, d, u, temperature=float("nan")),
           lambda: A.verify_drafts(z, d, u, temperature=1e-7), lambda: A.verify_drafts(z.half(), d, u),
           lambda: A.verify_drafts(torch.zeros((130, 5), device="cuda"), torch.zeros((2, 64), dtype=torch.int32, device="cuda"),
                                   torch.zeros((2, 65), device="cuda"))]
    for call in bad:
        with pytest.raises(A.PipoError):
            call()
    t, a = A.verify_drafts(z[:0], d[:0], u[:0])
    assert t.shape == (0, 4) and a.shape == (0,)
