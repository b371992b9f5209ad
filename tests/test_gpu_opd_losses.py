"""GPU parity of the OPD losses (teacher's top logits, distillation, clipped
policy loss) and their gradients against the float64 oracle.

Tolerances.  A log-probability is a logit, exact in fp64, minus the log of a sum
of exponentials of up to V terms.  Each term is 2^x of a difference with three
fp32 roundings (difference, product, fma), each at most 2^-24 of an exponent of
at most 30 (terms further down weigh less than e^-20 of the sum), plus the
exponential's own 2^-23: 3 * 30 * 2^-24 + 2^-23 = 5.5e-6.  A sum of fp32 adds
passes at most 512 terms in one thread (V = 524288 over 1024 threads) and 16
merges: 528 * 2^-24 = 3.1e-5 in the worst order, 1.1e-5 for the rows of up to
152000 tokens that most tests use.  So |error of log p| <= DELTA, and every
output is at most its derivative in log p times DELTA off, plus the rounding of
the output itself (half a step of its type)."""
import numpy as np
import pytest

from oracle import pipo_oracle as O

pytestmark = pytest.mark.gpu

DELTA = 5.5e-6 + 1.1e-5
DELTA_LONG = 5.5e-6 + 3.1e-5
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}


@pytest.fixture(scope="module")
def torch():
    import torch as t
    assert t.cuda.is_available(), "GPU tests need a GPU"
    return t


def _rows(torch, T, V, dtype, seed, pad=0, raised=8):
    """Logit rows with some tokens raised, as a view of padded storage (pad
    columns hold a sentinel), and their values in float64."""
    rng = np.random.default_rng(seed)
    z = 2.0 * rng.standard_normal((T, V + pad), dtype=np.float32)
    for t in range(T):
        at = rng.integers(0, V, raised)
        z[t, at] += 12.0 * rng.random(raised, dtype=np.float32)
    z[:, V:] = 1e4
    d = torch.from_numpy(z).cuda().to(getattr(torch, dtype))[:, :V]
    return d, d.double().cpu().numpy()


def _close(got, ref, tol, what=""):
    got = got.double().cpu().numpy()
    bad = np.isnan(ref) != np.isnan(got)
    assert not bad.any(), (what, "NaN", np.argwhere(bad)[:4])
    with np.errstate(invalid="ignore"):
        over = (np.abs(got - ref) > tol) & (got != ref) & ~np.isnan(ref)
    assert not over.any(), (what, np.argwhere(over)[:4], got[over][:4], ref[over][:4], np.broadcast_to(tol, ref.shape)[over][:4])


# ---- top logits ------------------------------------------------------------------------------------------------

def _check_top(torch, d, z, k, temperature=1.0, delta=DELTA):
    from paper_2605_27255_amd import opd_top_logits
    ids, logp, tail = opd_top_logits(d, k, temperature)
    torch.cuda.synchronize()
    r_ids, r_logp, r_tail = O.opd_top_logits(z, k, temperature)
    np.testing.assert_array_equal(ids.cpu().numpy(), r_ids)
    _close(logp, r_logp, delta + HALF["float32"] * np.abs(r_logp), "logp")
    # the mass outside and the whole are two such sums; with nothing outside, -inf exactly
    _close(tail, r_tail, 2 * delta + HALF["float32"] * np.abs(r_tail), "tail")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V,k,pad", [(1, 1, 1, 0), (3, 7, 7, 2), (2, 9, 1, 0), (5, 255, 128, 1), (2, 1000, 256, 0),
                                       (4, 2041, 255, 3), (7, 4096, 32, 0), (3, 16384, 20, 0), (3, 16385, 20, 5),
                                       (2, 50021, 100, 0), (3, 151936, 32, 0), (2, 151937, 256, 1)])
def test_top_logits(torch, T, V, k, pad, dtype):
    d, z = _rows(torch, T, V, dtype, seed=V + k, pad=pad)
    _check_top(torch, d, z, k, temperature=1.0 if k % 2 else 1.6)


def test_top_logits_longest_rows_and_many_rows(torch):
    d, z = _rows(torch, 2, 1 << 19, "bfloat16", seed=1)
    _check_top(torch, d, z, 64, delta=DELTA_LONG)
    d, z = _rows(torch, 700, 1201, "float32", seed=2)
    _check_top(torch, d, z, 17)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("V", [300, 4099, 70001])
def test_top_logits_of_crowded_rows(torch, V, dtype):
    """Constant rows, sorted rows, one value on more entries than are ranked,
    zeros of either sign, masked rows with fewer tokens than k."""
    k, rows = 50, []
    ramp = np.arange(V, dtype=np.float32) / V * 20
    rows += [np.full(V, 3.0, np.float32), ramp, ramp[::-1].copy(), np.zeros(V, np.float32)]
    rows[-1][::2] = -0.0
    crowd = np.random.default_rng(V).standard_normal(V).astype(np.float32)
    crowd[V // 20:] = 2.5                                  # most of the row at one value
    crowd[V // 3] = 9.0
    rows.append(crowd)
    lowest = np.full(V, float(torch.finfo(getattr(torch, dtype)).min), np.float32)
    rows.append(lowest.copy())                             # everything masked with the lowest value: uniform
    lowest[5:25] = 1.0
    rows.append(lowest)
    few = np.full(V, -np.inf, np.float32)
    few[7:290:13] = np.arange(22, dtype=np.float32)        # 22 tokens, k of 50
    rows.append(few)
    d = torch.from_numpy(np.stack(rows)).cuda().to(getattr(torch, dtype))
    _check_top(torch, d, d.double().cpu().numpy(), k)


@pytest.mark.parametrize("V", [300, 4099, 70001])
def test_top_logits_of_rows_of_all_ones_bits(torch, V):
    """Memory filled with ones is NaNs whose bits come last in any order: NaN
    log-probabilities, ids different and in range, split rows or not."""
    from paper_2605_27255_amd import opd_top_logits
    k = 50
    for bits, dtype in ((torch.int32, torch.float32), (torch.int16, torch.bfloat16)):
        d = torch.full((3, V), -1, dtype=bits, device="cuda").view(dtype)
        d[1, 5:25] = 1.0                                    # fewer than k others
        d[2, 100:200] = torch.arange(100, device="cuda").to(dtype)
        ids, logp, tail = opd_top_logits(d, k)
        torch.cuda.synchronize()
        assert logp.isnan().all() and tail.isnan().all()
        for row in ids.tolist():
            assert len(set(row)) == k and 0 <= min(row) and max(row) < V


def test_top_logits_of_rows_without_a_distribution(torch):
    """All -inf, a NaN, a +inf: NaN log-probabilities, ids different and in range; other rows as ever."""
    from paper_2605_27255_amd import opd_top_logits
    for V in (40, 40000):
        d, z = _rows(torch, 6, V, "float32", seed=8)
        d[1] = -float("inf")
        d[2, 3] = float("nan")
        d[3, V - 1] = float("inf")
        d[4] = float("nan")
        bad = torch.tensor([1, 2, 3, 4])
        ids, logp, tail = opd_top_logits(d, 24)
        torch.cuda.synchronize()
        assert logp[bad].isnan().all() and tail[bad].isnan().all()
        for r in ids.cpu().numpy():
            assert len(set(r.tolist())) == 24 and r.min() >= 0 and r.max() < V
        r_ids, r_logp, _ = O.opd_top_logits(z[[0, 5]], 24)
        np.testing.assert_array_equal(ids[[0, 5]].cpu().numpy(), r_ids)
        _close(logp[[0, 5]], r_logp, DELTA + HALF["float32"] * np.abs(r_logp))


@pytest.mark.parametrize("dtype,V", [("float32", 90001), ("bfloat16", 170003), ("float32", 4097), ("bfloat16", 20011)])
def test_top_logits_of_many_crowded_rows(torch, dtype, V):
    """Rows enough that none is split: ties, masks and NaNs among ordinary
    rows, whole-row kernels of every size; the copies of a row agree."""
    from paper_2605_27255_amd import opd_top_logits
    pad = -V % 8                              # every row lies alike
    d, z = _rows(torch, 8, V, dtype, seed=V, pad=pad)
    d[1] = 2.0
    d[2, V // 2:] = d[2].max()
    d[3, 30:] = -float("inf")
    d[4, 5] = float("nan")
    d[5, ::2] = float(torch.finfo(d.dtype).min)
    z = d.double().cpu().numpy()
    many = d._base.repeat(13, 1)[:, :V]
    ids, logp, tail = opd_top_logits(many, 40)
    torch.cuda.synchronize()
    for i in range(1, 13):
        assert torch.equal(ids[:8], ids[8 * i:8 * i + 8])
        assert torch.equal(logp[:8].nan_to_num(7), logp[8 * i:8 * i + 8].nan_to_num(7))
    keep = [0, 1, 2, 3, 5, 6, 7]
    r_ids, r_logp, r_tail = O.opd_top_logits(z[keep], 40)
    np.testing.assert_array_equal(ids[:8][keep].cpu().numpy(), r_ids)
    _close(logp[:8][keep], r_logp, DELTA + HALF["float32"] * np.abs(r_logp), "logp")
    _close(tail[:8][keep], r_tail, 2 * DELTA + HALF["float32"] * np.abs(r_tail), "tail")
    assert logp[4].isnan().all() and tail[4].isnan()
    row = ids[4].cpu().numpy()
    assert len(set(row.tolist())) == 40 and row.min() >= 0 and row.max() < V


def test_top_logits_split_rows_without_a_distribution(torch):
    """NaN, +inf and -inf rows, and ties across segments, in rows that are split."""
    from paper_2605_27255_amd import opd_top_logits
    V = 100003
    d, z = _rows(torch, 6, V, "float32", seed=8)
    d[1] = -float("inf")
    d[2, 90000] = float("nan")
    d[3, 3] = float("inf")
    d[4, 1::5] = 50.0                         # 20001 equal values in every segment
    ids, logp, tail = opd_top_logits(d, 24)
    torch.cuda.synchronize()
    for t in (1, 2, 3):
        assert logp[t].isnan().all() and tail[t].isnan()
        r = ids[t].cpu().numpy()
        assert len(set(r.tolist())) == 24 and r.min() >= 0 and r.max() < V
    keep = [0, 4, 5]
    r_ids, r_logp, r_tail = O.opd_top_logits(d.double().cpu().numpy()[keep], 24)
    np.testing.assert_array_equal(ids[keep].cpu().numpy(), r_ids)
    _close(logp[keep], r_logp, DELTA + HALF["float32"] * np.abs(r_logp), "logp")
    _close(tail[keep], r_tail, 2 * DELTA + HALF["float32"] * np.abs(r_tail), "tail")


# ---- distillation ------------------------------------------------------------------------------------------------

def _teacher(torch, z, k, temperature, seed, noise=0.7):
    rng = np.random.default_rng(seed)
    ids, logp, tail = O.opd_top_logits(z + noise * rng.standard_normal(z.shape), k, temperature)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a)).cuda().to(t)  # noqa: E731
    ids, logp, tail = dev(ids, torch.int32), dev(logp, torch.float32), dev(tail, torch.float32)
    return ids, logp, tail


def _host(*ts):
    return [None if t is None else t.cpu().numpy().astype(np.float64 if t.is_floating_point() else np.int64) for t in ts]


def _check_distill(torch, d, z, ids, logp, tail=None, rows=None, labels=None, scale=None, grad=True, delta=DELTA, **kw):
    from paper_2605_27255_amd import opd_distill
    loss, g = opd_distill(d, ids, logp, tail, rows=rows, labels=labels, scale=scale, grad=grad, **kw)
    torch.cuda.synchronize()
    h_ids, h_logp, h_tail, h_rows, h_labels, h_scale = _host(ids, logp, tail, rows, labels, scale)
    r_loss, r_grad, size = O.opd_distill(z, h_ids, h_logp, h_tail, h_rows, h_labels, scale=h_scale, **kw)
    unit = O.opd_distill(z, h_ids, h_logp, h_tail, h_rows, h_labels, **kw)[2].sum(1) * kw.get("temperature", 1.0)
    # each entry's term moves by at most (|a| + 2 P) DELTA (its a is P df/dP), and size sums just that
    _close(loss, r_loss, delta * unit + HALF["float32"] * np.abs(r_loss), "loss")
    if grad is not None:
        name = str(d.dtype).split(".")[1]
        # a product of an exponential of its own (DELTA again) and of sums that carry DELTA; 1e-38: denormals flush
        _close(g, r_grad, 4 * delta * size + HALF[name] * np.abs(r_grad) + 1e-37, "grad")
    return loss, g


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("kind", ["forward", "reverse", "jsd"])
@pytest.mark.parametrize("T,V,k,pad,with_tail", [(1, 1, 1, 0, False), (2, 2, 1, 0, True), (3, 9, 9, 1, True),
                                                 (4, 513, 100, 0, True), (5, 4096, 32, 0, False), (3, 16384, 3, 3, True),
                                                 (2, 16387, 256, 0, True), (4, 50021, 20, 7, False), (2, 151936, 32, 0, True)])
def test_distill(torch, T, V, k, pad, with_tail, kind, dtype):
    d, z = _rows(torch, T, V, dtype, seed=V + k, pad=pad)
    temperature = 1.0 if V % 2 else 1.7
    ids, logp, tail = _teacher(torch, z, k, temperature, seed=5)
    scale = torch.linspace(0.3, -1.2, T).cuda()
    _check_distill(torch, d, z, ids, logp, tail if with_tail else None, scale=scale, kind=kind, beta=0.3,
                   temperature=temperature)


@pytest.mark.parametrize("V", [1000, 40001])
def test_distill_rows_labels_and_slots(torch, V):
    """A row map, unscored positions, empty slots in odd places, and flagged
    positions (no teacher row, an id out of range, an id listed twice) that
    leave the others alone."""
    T, k = 12, 40
    d, z = _rows(torch, T, V, "float32", seed=V)
    ids, logp, tail = _teacher(torch, z[:8], k, 1.0, seed=6)
    rows = torch.tensor([0, 1, 1, 2, 3, 8, -1, 4, 5, 6, 7, 7], dtype=torch.int32).cuda()     # 8 and -1: no such row
    labels = torch.tensor([1, 1, -1, 1, 1, 1, 1, 1, 1, 1, -5, 2 ** 31 - 1], dtype=torch.int32).cuda()
    ids[2, ::3] = -1
    ids[3, :] = -7                       # nothing listed
    ids[4, 5] = V
    ids[5, 39] = ids[5, 0]
    ids[6, 0] = 2 ** 31 - 1
    for tl in (tail, None):
        for kind in ("forward", "reverse", "jsd"):
            loss, g = _check_distill(torch, d, z, ids, logp, tl, rows=rows, labels=labels, kind=kind)
            flagged = [5, 6, 7, 8, 9]
            assert loss[flagged].isnan().all() and g[flagged].isnan().all()
            assert not loss[[2, 10]].any() and not g[[2, 10]].any()


def test_distill_masked_logits(torch):
    """Students with masked tokens (-inf, the lowest value), everything listed
    but masked, tails without mass, and rows without any token."""
    V = 3001
    d, z = _rows(torch, 8, V, "float32", seed=2)
    ids, logp, tail = _teacher(torch, z, 16, 1.0, seed=3)
    out = torch.ones(V, dtype=torch.bool, device="cuda")
    out[ids[1].long()] = False
    d[0, ::2] = -float("inf")
    d[1, out] = -float("inf")            # the student has nothing outside the list
    d[2, ids[2].long()] = -float("inf")  # ... and nothing on it
    d[3] = -float("inf")
    d[4, 1::2] = float(torch.finfo(torch.float32).min)
    d[5, 77] = float("nan")
    d[6, 78] = float("inf")
    d[7] = float(torch.finfo(torch.float32).min)
    z = d.double().cpu().numpy()
    for kind in ("reverse", "jsd"):
        with np.errstate(all="ignore"):
            loss, g = _check_distill(torch, d, z, ids, logp, tail, kind=kind)
        assert loss[[3, 5, 6]].isnan().all() and g[[3, 5, 6]].isnan().all()
        assert loss[[0, 1, 2, 4, 7]].isfinite().all() and g[[0, 1, 2, 4, 7]].isfinite().all()
    from paper_2605_27255_amd import opd_distill
    loss, _ = opd_distill(d, ids, logp, tail, kind="forward", grad=True)
    assert torch.isposinf(loss[[0, 1, 2]]).all() and loss[[3, 5, 6]].isnan().all()   # teacher mass where there is none


def test_distill_near_teacher_and_sharp_student(torch):
    """A student that is its teacher (nothing left but rounding), and one with
    all but 1e-9 of its mass on one listed token: the rest's mass is exact."""
    V, k = 20011, 8
    d, z = _rows(torch, 3, V, "float32", seed=4)
    d[1] = 0
    d[1, 17] = 30.0
    d[2, :] = -50.0
    d[2, 3] = 45.0                       # the rest holds e^-85 of the mass, below fp32 normals
    z = d.double().cpu().numpy()
    ids, logp, tail = _teacher(torch, z, k, 1.0, seed=9, noise=0.0)
    for kind in ("forward", "reverse", "jsd"):
        _check_distill(torch, d, z, ids, logp, tail, kind=kind)
    ids, logp, tail = _teacher(torch, z, k, 1.0, seed=9, noise=0.5)
    for kind in ("forward", "reverse", "jsd"):
        _check_distill(torch, d, z, ids, logp, tail, kind=kind)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V,pad", [(3, 777, 0), (40, 70003, 5), (300, 20001, 0)])
def test_gradients_in_place_and_beside(torch, T, V, pad, dtype):
    """The gradient of the same rows in a new tensor, in a buffer of another
    stride and alignment, beside the logits in one buffer, and over them: the
    same values, and nothing written outside the rows.  (Rows that lie
    differently are summed in another order: each view has its own values.)"""
    from paper_2605_27255_amd import opd_distill, opd_policy
    d, z = _rows(torch, T, V, dtype, seed=11, pad=pad)
    ids, logp, tail = _teacher(torch, z[:3], 12, 1.0, seed=2)
    rows = (torch.arange(T, dtype=torch.int32) % 3).cuda()
    y = ids[rows.long(), 0].contiguous()
    y[T // 2] = -1
    adv = torch.linspace(-1, 1, T).cuda()
    for call in (lambda x, g: opd_distill(x, ids, logp, tail, rows=rows, labels=y, grad=g)[-1],
                 lambda x, g: opd_policy(x, y, adv, grad=g)[-1]):
        want = call(d, True)
        other = torch.full((T, V + 9), 7.0, device="cuda", dtype=d.dtype)
        call(d, other[:, 3:3 + V])
        assert torch.equal(other[:, 3:3 + V], want) and (other[:, :3] == 7).all() and (other[:, 3 + V:] == 7).all()
        both = torch.full((T, 2 * V + 3), 7.0, device="cuda", dtype=d.dtype)
        both[:, :V] = d
        want = call(both[:, :V], True)
        call(both[:, :V], both[:, V + 1:2 * V + 1])
        assert torch.equal(both[:, V + 1:2 * V + 1], want) and torch.equal(both[:, :V], d)
        assert (both[:, V] == 7).all() and (both[:, 2 * V + 1:] == 7).all()
        store = torch.full((T, V + 6), 7.0, device="cuda", dtype=d.dtype)
        store[:, 1:V + 1] = d
        x = store[:, 1:V + 1]
        want = call(x, True)
        assert call(x, x) is x
        assert torch.equal(x, want) and (store[:, 0] == 7).all() and (store[:, V + 1:] == 7).all()


def test_distill_gradient_against_differences(torch):
    """Along random directions: (loss(z + h u) - loss(z - h u)) / 2h against the
    gradient.  The two losses carry at most DELTA_SMALL (901 tokens: 4 terms a
    thread and 10 merges, 14 * 2^-24 beside the exponentials' 5.5e-6) times
    their terms' slopes each; the quotient's own error is h^2 / 6 times the third
    derivative, which three powers of u's largest element and the terms bound."""
    from paper_2605_27255_amd import opd_distill
    delta, T, V, k, h = 5.5e-6 + 14 * 2.0 ** -24, 6, 901, 10, 2e-2
    d, z = _rows(torch, T, V, "float32", seed=21)
    ids, logp, tail = _teacher(torch, z, k, 1.0, seed=22)
    for kind in ("forward", "reverse", "jsd"):
        _, grad = opd_distill(d, ids, logp, tail, kind=kind, grad=True)
        h_ids, h_logp, h_tail = _host(ids, logp, tail)
        slopes = O.opd_distill(z, h_ids, h_logp, h_tail, kind=kind)[2].sum(1)
        for seed in range(3):
            u = torch.from_numpy(np.random.default_rng(seed).standard_normal((T, V)).astype(np.float32)).cuda()
            u = u / u.abs().amax(1, keepdim=True)
            up = opd_distill((d.double() + h * u.double()).float(), ids, logp, tail, kind=kind)[0].double()
            down = opd_distill((d.double() - h * u.double()).float(), ids, logp, tail, kind=kind)[0].double()
            got = ((up - down) / (2 * h)).cpu().numpy()
            want = (grad.double() * u.double()).sum(1).cpu().numpy()
            # inputs round too: 2^-24 of logits up to 20 moves each loss by 20 * 2^-24 of its slopes
            tol = slopes * ((2 * delta + 40 * 2.0 ** -24) / (2 * h) + 8 * h * h / 6)
            assert (np.abs(got - want) <= tol).all(), (kind, got, want, tol)


# rows of 16-byte pieces on both sides of each size at which another kernel variant takes over (256 pieces a slab)
SLABS = [0.01, 1, 3, 5, 7, 9, 13, 17, 21, 26, 30, 35, 40, 46, 82, 110]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("slabs", SLABS)
@pytest.mark.parametrize("side", [-1, 1])
def test_distill_row_lengths(torch, slabs, side, dtype):
    """Enough rows that none is split (and, for the longest, that a workgroup
    takes several): copies of six, among them unscored and flagged ones."""
    from paper_2605_27255_amd import opd_distill
    N = 4 if dtype == "float32" else 8
    V = max(13, int(slabs * 256) * N + side * 3)
    pad, copies = -V % N, 50 if slabs < 82 else 51
    d, z = _rows(torch, 6, V, dtype, seed=V, pad=pad)
    ids, logp, tail = _teacher(torch, z, 7, 1.0, seed=3)
    ids[4, 1] = ids[4, 0]                     # flagged by its list
    y = torch.tensor([1, -1, 1, 1, 1, 1], dtype=torch.int32).cuda()
    rows = torch.tensor([0, 1, 2, 9, 4, 5], dtype=torch.int32).cuda()      # position 3: no such teacher row
    scale = torch.linspace(0.5, 2, 6).cuda()
    many = lambda a: a.repeat(copies, *[1] * (a.dim() - 1))  # noqa: E731
    x = many(d._base)[:, :V]
    loss, g = opd_distill(x, ids, logp, tail, rows=many(rows), labels=many(y), scale=many(scale), grad=True)
    only, none = opd_distill(x, ids, logp, tail, rows=many(rows), labels=many(y))
    torch.cuda.synchronize()
    assert none is None
    for i in range(1, copies):
        part = slice(6 * i, 6 * i + 6)
        assert torch.equal(loss[:6].nan_to_num(7), loss[part].nan_to_num(7)), i
        assert torch.equal(g[:6].nan_to_num(7), g[part].nan_to_num(7)), i
    h = _host(ids, logp, tail, rows, y, scale)
    r_loss, r_grad, size = O.opd_distill(z, *h[:5], scale=h[5])
    unit = O.opd_distill(z, *h[:5])[2].sum(1)
    delta = DELTA_LONG
    for got in (loss[:6], only[:6], only[-6:]):
        _close(got, r_loss, delta * unit + HALF["float32"] * np.abs(r_loss), "loss")
    _close(g[:6], r_grad, 4 * delta * size + HALF[dtype] * np.abs(r_grad) + 1e-37, "grad")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V", [(2, 3001), (2, 20011), (100, 70001), (2, 151936)])
def test_rows_whose_beginning_is_masked(torch, T, V, dtype):
    """Rows that start with masked tokens, or with tokens far below the others:
    no sum may depend on where a row's large values stand."""
    from paper_2605_27255_amd import opd_distill
    d, z = _rows(torch, 6, V, dtype, seed=V, pad=-V % 8)
    d[0, :V - V // 50] = -float("inf")
    d[1, :V - V // 50] -= 300.0
    d[2, :V // 2] = float(torch.finfo(d.dtype).min)
    d[3, : V - 1] = -float("inf")
    d[4, V - 5] = 200.0
    z = d.double().cpu().numpy()
    ids, logp, tail = _teacher(torch, np.where(np.isfinite(z) & (np.abs(z) < 1e30), z, 0.0), 9, 1.0, seed=1)
    many = lambda a: a.repeat((T + 5) // 6, *[1] * (a.dim() - 1))[:T]  # noqa: E731
    x = many(d._base)[:, :V]
    zz = z[np.arange(T) % 6][:6]
    loss, g = opd_distill(x, many(ids), many(logp), many(tail), kind="jsd", grad=True)
    only, _ = opd_distill(x, many(ids), many(logp), many(tail), kind="jsd")
    torch.cuda.synchronize()
    n = len(zz)
    h = _host(ids[:n], logp[:n], tail[:n])
    with np.errstate(all="ignore"):
        r_loss, r_grad, size = O.opd_distill(zz, *h, kind="jsd")
    for got in (loss[:n], only[:n]):
        _close(got, r_loss, DELTA * size.sum(1) + HALF["float32"] * np.abs(r_loss), "loss")
    _close(g[:n], r_grad, 4 * DELTA * size + HALF[dtype] * np.abs(r_grad) + 1e-37, "grad")


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T", [3, 98])
def test_longest_rows(torch, T, dtype):
    """524288 tokens, split over workgroups and not, with 256 entries."""
    from paper_2605_27255_amd import opd_distill
    V = 1 << 19
    d, z = _rows(torch, 3, V, dtype, seed=V)
    ids, logp, tail = _teacher(torch, z, 256, 1.3, seed=4)
    rows = (torch.arange(T, dtype=torch.int32) % 3).cuda()
    x = d.repeat(33, 1)[:T]
    kw = dict(rows=rows, kind="reverse", temperature=1.3)
    loss, g = opd_distill(x, ids, logp, tail, grad=True, **kw)
    only, _ = opd_distill(x, ids, logp, tail, **kw)
    torch.cuda.synchronize()
    r_loss, r_grad, size = O.opd_distill(z, *_host(ids, logp, tail), temperature=1.3)
    unit = size.sum(1) * 1.3
    for got in (loss[:3], only[:3], loss[-1:]):
        at = (T - 1) % 3 if len(got) == 1 else slice(0, 3)
        _close(got, np.atleast_1d(r_loss[at]), DELTA_LONG * np.atleast_1d(unit[at]) + HALF["float32"] * np.abs(np.atleast_1d(r_loss[at])))
    _close(g[:3], r_grad, 4 * DELTA_LONG * size + HALF[dtype] * np.abs(r_grad) + 1e-37, "grad")
    _close(g[-1], r_grad[(T - 1) % 3], (4 * DELTA_LONG * size + HALF[dtype] * np.abs(r_grad) + 1e-37)[(T - 1) % 3], "grad")


def test_calls_without_a_work_array(torch):
    """The C entries with d_work NULL: one workgroup a row, the same results to rounding."""
    import ctypes
    from paper_2605_27255_amd import load_library, opd_distill, opd_top_logits
    lib, V, T, k = load_library(), 151936, 3, 20
    d, z = _rows(torch, T, V, "float32", seed=5)
    ids, logp, tail = opd_top_logits(d, k)
    i2, l2, t2 = torch.empty_like(ids), torch.empty_like(logp), torch.empty_like(tail)
    stream = torch.cuda.current_stream().cuda_stream
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    assert lib.pipo_opd_top_logits(T, V, p(d), V, 1.0, k, p(i2), p(l2), p(t2), None, 0, stream) == 0
    torch.cuda.synchronize()
    assert torch.equal(ids, i2)
    r = O.opd_top_logits(z, k)
    _close(l2, r[1], DELTA + HALF["float32"] * np.abs(r[1]))
    _close(t2, r[2], 2 * DELTA + HALF["float32"] * np.abs(r[2]))
    t_ids, t_logp, t_tail = _teacher(torch, z, k, 1.0, seed=2)
    loss, g = torch.empty(T, device="cuda"), torch.empty_like(d)
    assert lib.pipo_opd_distill(T, V, p(d), V, T, k, p(t_ids), p(t_logp), p(t_tail), None, None, 1, 0.5, 1.0, None, p(loss),
                                p(g), V, None, 0, stream) == 0
    torch.cuda.synchronize()
    r_loss, r_grad, size = O.opd_distill(z, *_host(t_ids, t_logp, t_tail))
    _close(loss, r_loss, DELTA * size.sum(1) + HALF["float32"] * np.abs(r_loss), "loss")
    _close(g, r_grad, 4 * DELTA * size + HALF["float32"] * np.abs(r_grad) + 1e-37, "grad")
    again = opd_distill(d, t_ids, t_logp, t_tail, grad=True)
    assert all(torch.equal(a, b) for a, b in zip(again, opd_distill(d, t_ids, t_logp, t_tail, grad=True)))


# ---- policy loss ---------------------------------------------------------------------------------------------------

def _check_policy(torch, d, z, y, adv, old=None, ref=None, scale=None, grad=True, delta=DELTA, **kw):
    from paper_2605_27255_amd import opd_policy
    loss, logp, kl, g = opd_policy(d, y, adv, old_logp=old, ref_logp=ref, scale=scale, grad=grad, **kw)
    torch.cuda.synchronize()
    h_y, h_adv, h_old, h_ref, h_scale = _host(y, adv, old, ref, scale)
    r_loss, r_logp, r_kl, r_grad, slope = O.opd_policy(z, h_y, h_adv, h_old, h_ref, scale=h_scale, **kw)
    eps = HALF["float32"]
    _close(logp, r_logp, delta + eps * np.abs(r_logp), "logp")
    _close(loss, r_loss, delta * slope + eps * np.abs(r_loss), "loss")
    if ref is None:
        assert kl is None
    else:
        u = np.where(h_y >= 0, h_ref - r_logp, 0)
        _close(kl, r_kl, delta * np.abs(np.expm1(u)) + delta ** 2 + eps * np.abs(r_kl), "kl")
    if grad is not None:
        T, V = z.shape
        name = str(d.dtype).split(".")[1]
        w = np.abs(h_scale if h_scale is not None else np.ones(T)) / kw.get("temperature", 1.0)
        p = np.stack([np.exp(O._log_softmax_row(r, kw.get("temperature", 1.0))) for r in z])
        hot = np.zeros((T, V))
        for t in range(T):
            if 0 <= h_y[t] < V:
                hot[t, int(h_y[t])] = 1
        # the factor moves by slope * DELTA, each probability by itself * 2 DELTA (its own exponential and the sum)
        tol = (w * slope)[:, None] * (p + hot * (1 - p)) * 4 * delta + HALF[name] * np.abs(r_grad) + 1e-37
        _close(g, r_grad, tol, "grad")
    return loss, logp, kl, g


def _rollout(torch, z, temperature, seed):
    """Labels the row likes, and old and reference log-probabilities whose
    ratios stay 1e-3 from the clip's edges (the gradient jumps there)."""
    rng = np.random.default_rng(seed)
    T, V = z.shape
    y = np.array([int(np.argsort(-z[t], kind="stable")[min(V - 1, rng.integers(0, 6))]) for t in range(T)])
    lp = O.opd_policy(z, y, np.ones(T), temperature=temperature)[1]
    ratio = np.exp(0.3 * rng.standard_normal(T))
    for edge in (0.8, 1.3):
        ratio = np.where(np.abs(ratio - edge) < 1e-3, edge + 2e-3, ratio)
    dev = lambda a: torch.from_numpy(a.astype(np.float32)).cuda()  # noqa: E731
    return (torch.from_numpy(y.astype(np.int32)).cuda(), dev(rng.standard_normal(T)), dev(lp - np.log(ratio)),
            dev(lp + 0.3 * rng.standard_normal(T)))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V,pad", [(1, 1, 0), (3, 2, 1), (5, 777, 0), (9, 4096, 0), (4, 16384, 4), (6, 16385, 0),
                                     (5, 50021, 3), (3, 151936, 0)])
def test_policy(torch, T, V, pad, dtype):
    d, z = _rows(torch, T, V, dtype, seed=V, pad=pad)
    temperature = 1.0 if V % 2 else 0.7
    y, adv, old, ref = _rollout(torch, z, temperature, seed=V)
    scale = torch.linspace(1.0, 0.2, T).cuda()
    if T > 3:
        y[1] = -1
        y[3] = V                        # no such token: flagged
    kw = dict(clip=(0.2, 0.3), temperature=temperature)
    loss, logp, _, g = _check_policy(torch, d, z, y, adv, old, ref, scale, kl_coef=0.1, **kw)
    if T > 3:
        assert loss[3].isnan() and g[3].isnan().all() and loss[1] == 0 and logp[1] == 0 and not g[1].any()
    _check_policy(torch, d, z, y, adv, old, None, None, **kw)
    _check_policy(torch, d, z, y, adv, None, ref, None, kl_coef=0.0, grad=None, **kw)
    _check_policy(torch, d, z, y, adv, None, None, scale, **kw)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V", [(1, 33333), (257, 20011), (1100, 9001), (1100, 40003)])
def test_policy_without_a_gradient(torch, T, V, dtype):
    """Rows from workgroups of four, eight and sixteen waves."""
    d, z = _rows(torch, T, V, dtype, seed=V)
    rng = np.random.default_rng(1)
    y = torch.from_numpy(rng.integers(0, V, T).astype(np.int32)).cuda()
    _check_policy(torch, d, z, y, torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda(), grad=None)


def test_policy_sharp_rows_and_masks(torch):
    """A label with all but 1e-12 of the mass keeps the gradient of that rest;
    masked tokens get none; rows without a token, or with a NaN, are NaN."""
    V = 9001
    d, z = _rows(torch, 6, V, "float32", seed=3)
    d[0] = 0
    d[0, 5] = 37.0
    d[1, ::2] = -float("inf")
    d[2] = -float("inf")
    d[3, 9] = float("nan")
    d[4] = float(torch.finfo(torch.float32).min)
    d[5, 100:] = float(torch.finfo(torch.float32).min)
    z = d.double().cpu().numpy()
    y = torch.tensor([5, 1, 0, 0, 7, 50], dtype=torch.int32).cuda()
    adv = torch.tensor([1.0, -1, 1, 1, 2, 1]).cuda()
    with np.errstate(all="ignore"):
        loss, _, _, g = _check_policy(torch, d, z, y, adv)
    assert g[0, 5] < 0 and abs(g[0, 5].item()) < 1e-10 and not g[1, ::2].any() and not g[5, 100:].any()
    assert loss[[2, 3]].isnan().all() and g[[2, 3]].isnan().all()


# ---- together, streams, graphs, far offsets --------------------------------------------------------------------------

def test_training_chunk_end_to_end(torch):
    """A chunk as a training loop runs it: PAD-compacted teacher rows, the
    teacher's list, the OPD targets, distillation into the logits' place, and a
    policy step whose advantages are the sampled KL terms."""
    from paper_2605_27255_amd import opd_distill, opd_policy, opd_targets, opd_teacher_rows, opd_top_logits
    rng = np.random.default_rng(31)
    T, V, k = 96, 8192, 32
    tok = rng.integers(0, V - 1, T).astype(np.int32)
    tok[rng.random(T) < 0.25] = V - 1
    tok[0] = 1
    Tt = int(np.count_nonzero(tok != V - 1))
    s, zs = _rows(torch, T, V, "bfloat16", seed=32)
    te, zt = _rows(torch, Tt, V, "bfloat16", seed=33)
    y = rng.integers(0, V - 1, T).astype(np.int32)
    y[rng.random(T) < 0.1] = -1
    labels = torch.from_numpy(y).cuda()
    rows = opd_teacher_rows(torch.from_numpy(tok).cuda(), V - 1)
    ids, logp, tail = opd_top_logits(te, k)
    kl, _, _ = opd_targets(s.contiguous(), te.contiguous(), labels, rows)
    loss, g = opd_distill(s, ids, logp, tail, rows=rows, labels=labels, kind="reverse", scale=torch.full((T,), 1 / T).cuda(),
                          grad=True)
    adv = -kl
    p_loss, p_logp, _, p_grad = opd_policy(s, labels, adv, grad=s)
    torch.cuda.synchronize()
    assert p_grad is s
    o_rows = O.opd_teacher_rows(tok, V - 1)
    o_ids, o_logp, o_tail = O.opd_top_logits(zt, k)
    np.testing.assert_array_equal(ids.cpu().numpy(), o_ids)
    o_loss, o_grad, size = O.opd_distill(zs, o_ids, o_logp, o_tail, o_rows, y, scale=np.full(T, 1 / T))
    unit = O.opd_distill(zs, o_ids, o_logp, o_tail, o_rows, y)[2].sum(1)
    # the teacher's numbers carry DELTA as well
    _close(loss, o_loss, 3 * DELTA * unit + 2.0 ** -24 * np.abs(o_loss), "loss")
    _close(g, o_grad, 8 * DELTA * size + HALF["bfloat16"] * np.abs(o_grad) + 1e-37, "grad")
    o = O.opd_policy(zs, y, adv.cpu().numpy())
    _close(p_loss, o[0], DELTA * o[4] + 2.0 ** -24 * np.abs(o[0]), "policy loss")
    p = np.stack([np.exp(O._log_softmax_row(r, 1.0)) for r in zs])
    hot = (np.arange(V)[None] == y[:, None]) * 1.0
    _close(p_grad, o[3], o[4][:, None] * (p + hot) * 4 * DELTA + HALF["bfloat16"] * np.abs(o[3]) + 1e-37, "policy grad")


@pytest.mark.parametrize("T,V", [(3, 60001), (400, 20000)])
def test_streams_and_graphs(torch, T, V):
    """The calls on a side stream, and captured in two graphs whose replays
    interleave with eager calls and new inputs, give the eager results."""
    from paper_2605_27255_amd import opd_distill, opd_policy, opd_top_logits
    gen = torch.Generator(device="cuda").manual_seed(1)
    fresh = lambda: 3 * torch.randn((T, V), generator=gen, device="cuda")  # noqa: E731
    s, te = fresh(), fresh()
    adv, y = torch.randn(T, generator=gen, device="cuda"), torch.randint(0, V, (T,), generator=gen, device="cuda").int()

    def step():
        ids, logp, tail = opd_top_logits(te, 16)
        return (ids, logp, tail) + opd_distill(s, ids, logp, tail, labels=y, grad=True)

    def policy():
        loss, logp, _, g = opd_policy(s, y, adv, grad=True)
        return loss, logp, g

    side = torch.cuda.Stream()
    want = [t.clone() for t in step() + policy()]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step() + policy()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs, outs = [], []
    for fn in (step, policy):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(fn())
        graphs.append(g)
    for i in range(4):
        s.copy_(fresh())
        te.copy_(fresh())
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay()
        want = step() + policy()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[0] + outs[1], want)), i


def test_rows_far_apart(torch):
    """Row offsets beyond 2^32 bytes and 2^31 elements."""
    V, ld, T = 5003, (1 << 30) + 3, 4
    store = torch.empty(ld * (T - 1) + V, dtype=torch.bfloat16, device="cuda")
    d = store.as_strided((T, V), (ld, 1))
    src, z = _rows(torch, T, V, "bfloat16", seed=7)
    d.copy_(src)
    _check_top(torch, d, z, 30)
    ids, logp, tail = _teacher(torch, z, 8, 1.0, seed=1)
    _check_distill(torch, d, z, ids, logp, tail, kind="reverse", grad=d)


def test_python_refusals(torch):
    from paper_2605_27255_amd import PIPO_EINVAL, PipoError, opd_distill, opd_policy, opd_top_logits
    d, z = _rows(torch, 4, 100, "float32", seed=1)
    ids, logp, tail = _teacher(torch, z, 5, 1.0, seed=1)
    y, adv = torch.zeros(4, dtype=torch.int32).cuda(), torch.zeros(4).cuda()
    calls = [lambda: opd_top_logits(d, 0), lambda: opd_top_logits(d, 101), lambda: opd_top_logits(d[0], 1),
             lambda: opd_top_logits(d.half(), 5), lambda: opd_top_logits(d.t(), 2), lambda: opd_top_logits(d, 5, 0.0),
             lambda: opd_top_logits(d[:1].expand(4, 100), 5),
             lambda: opd_distill(d, ids, logp, tail, kind="kl"), lambda: opd_distill(d, ids.long(), logp),
             lambda: opd_distill(d, ids, logp[:, :3]), lambda: opd_distill(d, ids, logp.cpu()),
             lambda: opd_distill(d, ids, logp, tail[:3]), lambda: opd_distill(d, ids, logp, rows=y[:3]),
             lambda: opd_distill(d, ids, logp, grad=torch.empty(4, 99, device="cuda")),
             lambda: opd_distill(d, ids, logp, grad=d.bfloat16()), lambda: opd_distill(d, ids, logp, kind="jsd", beta=1.0),
             lambda: opd_distill(d[:, :50], ids, logp, grad=d[:, 25:75]),
             lambda: opd_policy(d, y, adv[:2]), lambda: opd_policy(d, y.long(), adv), lambda: opd_policy(d, y, adv, kl_coef=0.1),
             lambda: opd_policy(d, y, adv, clip=(1.5, 0.2)), lambda: opd_policy(d, y, adv, temperature=float("nan")),
             lambda: opd_policy(d, y, adv, scale=torch.ones(4, 1, device="cuda"))]
    for i, call in enumerate(calls):
        with pytest.raises(PipoError) as e:
            call()
        assert e.value.code == PIPO_EINVAL, i
    empty = d[:0]
    assert opd_top_logits(empty, 5)[0].shape == (0, 5)
    loss, g = opd_distill(empty, ids, logp, tail, grad=True)
    assert loss.shape == (0,) and g.shape == (0, 100)
    assert opd_policy(empty, y[:0], adv[:0], grad=True)[3].shape == (0, 100)


# ---- split rows, masks and magnitudes ----------------------------------------------------------------------------------

def _is_split(call, T, V, k, dtype):
    from paper_2605_27255_amd import load_library
    return load_library().pipo_opd_work_bytes(call, T, V, k, dtype == "bfloat16") > 0


@pytest.mark.parametrize("temperature", [0.7, 1.0, 2.0])
@pytest.mark.parametrize("T,V,dtype,grad", [(3, 60001, "float32", True), (2, 151936, "bfloat16", True),
                                            (16, 151936, "float32", None)])
def test_split_rows_with_nothing_outside(torch, T, V, dtype, grad, temperature):
    """Everything but the list (or the label) masked with -inf, in rows that are
    split: the tokens outside have no mass, and nothing is NaN."""
    d, z = _rows(torch, T, V, dtype, seed=V)
    ids, logp, tail = _teacher(torch, z, 9, temperature, seed=1)
    for x in (ids.long(), ids[:, :1].long()):
        assert _is_split(2 if grad else 1, T, V, x.shape[1], dtype)
        only = torch.full_like(d, -float("inf")).scatter_(1, x, d.gather(1, x))
        oz = only.double().cpu().numpy()
        if x.shape[1] == 1:
            y, adv, ref = ids[:, 0].contiguous(), torch.linspace(-1, 1, T).cuda(), torch.full((T,), -0.3).cuda()
            out = _check_policy(torch, only, oz, y, adv, None, ref, grad=grad, kl_coef=0.1, temperature=temperature)
            assert all(t is None or t.isfinite().all() for t in out)
            continue
        for kind in ("reverse", "jsd", "forward"):
            loss, g = _check_distill(torch, only, oz, ids, logp, tail, grad=grad, kind=kind, temperature=temperature)
            # (a teacher with mass where the student has none is infinitely far in the forward direction)
            assert torch.isposinf(loss).all() if kind == "forward" else loss.isfinite().all()
            assert grad is None or g.isfinite().all()


# A row's gradient sums to zero.  An unlisted one's exponent is at most 30 (less weighs under 2^-30) and rounded once, 21 *
# 2^-24 of the value; its exponential 2^-23, coefficient and product 2^-24 each: 25 * 2^-24.  The sum behind the coefficient
# has exponentials as exact, once more where threads are merged (46 * 2^-24), and adds: up to 20 in a thread, 16 in merges.
ZERO_SUM = 107 * 2.0 ** -24


@pytest.mark.parametrize("offset,temperature", [(1000.0, 0.7), (-1000.0, 0.7), (10000.0, 1.0), (20.0, 0.05), (20.0, 1e-3),
                                                (0.0, 1e-5), (3.0, 1e-5)])
@pytest.mark.parametrize("T,V", [(4, 2001), (3, 70001), (100, 5003)])
def test_gradients_of_rows_with_an_offset(torch, T, V, offset, temperature):
    """softmax does not change with an offset of the row, nor with logits and
    temperature scaled together: nor does the gradient's accuracy."""
    rng = np.random.default_rng(V)
    z = (offset + temperature * 3.0 * rng.standard_normal((T, V))).astype(np.float32)
    d, z = torch.from_numpy(z).cuda(), z.astype(np.float64)
    ids, logp, tail = O.opd_top_logits(z + temperature * rng.standard_normal(z.shape), 9, temperature)
    ids, logp, tail = (torch.from_numpy(a).cuda().to(t) for a, t in ((ids, torch.int32), (logp, torch.float32), (tail, torch.float32)))
    y = torch.from_numpy(rng.integers(0, V, T).astype(np.int32)).cuda()
    grads = [_check_distill(torch, d, z, ids, logp, tail, kind=kind, temperature=temperature)[1] for kind in ("forward", "jsd")]
    grads.append(_check_policy(torch, d, z, y, torch.linspace(0.5, 1.5, T).cuda(), temperature=temperature)[3])
    for g in grads:
        off = (g.double().sum(1).abs() / g.double().abs().sum(1)).cpu().numpy()
        assert (off <= ZERO_SUM).all(), off


@pytest.mark.parametrize("level,temperature", [(14.5361, 1e-5), (20.0, 1e-5), (50.0, 1e-5), (200.0, 1e-5), (1000.0, 1e-5),
                                               (1000.0, 1e-3), (-200.0, 1e-5)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V", [(3, 3001), (2, 130001), (100, 20011)])
def test_gradients_of_level_rows_at_small_temperatures(torch, T, V, dtype, level, temperature):
    """Thousands of equal tokens far from 0 in units of the temperature: what a
    reference of the exponentials cannot hold is not left out of the gradient."""
    d = torch.full((T, V), level, device="cuda", dtype=getattr(torch, dtype))
    d[:, 1::7] -= 1.5 * temperature             # (another level, where the type can tell it)
    z = d.double().cpu().numpy()
    ids, logp, tail = _teacher(torch, z, 9, temperature, seed=1, noise=temperature)
    _check_distill(torch, d, z, ids, logp, tail, kind="jsd", temperature=temperature)
    _check_policy(torch, d, z, ids[:, 0].contiguous(), torch.ones(T).cuda(), temperature=temperature)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("mask,temperature", [(-1e4, 1.0), (-1e9, 0.7), (-1e9, 1.1), (-1e10, 1.0), (-1e10, 0.5), (-3e20, 1.0),
                                              (-1e30, 1.4), (-1e32, 1.0), (-1e9, 1e-3)])
@pytest.mark.parametrize("T,V", [(6, 3001), (6, 140001), (102, 20011)])
def test_tokens_masked_with_finite_values(torch, T, V, dtype, mask, temperature):
    """Masks of every magnitude weigh nothing beside a token that is not masked,
    and alike where all are, or where all tokens outside the list are."""
    d, z = _rows(torch, 6, V, dtype, seed=V)
    ids, logp, tail = _teacher(torch, z, 9, temperature, seed=2)
    d[0, 1::2] = mask
    d[1, : V - V // 10] = mask
    d[2, V // 10:] = mask
    listed = ids[3:4].long()
    d[3:4] = torch.full_like(d[3:4], mask).scatter_(1, listed, d[3:4].gather(1, listed))
    d[4] = mask
    z = d.double().cpu().numpy()
    for k in (1, 9, 40) if temperature >= 0.5 else ():
        _check_top(torch, d, z, k, temperature)
    many = lambda a: a.repeat((T + 5) // 6, *[1] * (a.dim() - 1))[:T]  # noqa: E731
    zz = np.tile(z, ((T + 5) // 6, 1))[:T]
    for kind in ("forward", "jsd"):
        _check_distill(torch, many(d), zz, many(ids), many(logp), many(tail), kind=kind, temperature=temperature)
        _check_distill(torch, many(d), zz, many(ids), many(logp), None, kind=kind, temperature=temperature, grad=None)
    y = torch.tensor([2, V - 1, 0, int(listed[0, 0]), 5, 1], dtype=torch.int32).cuda()
    _check_policy(torch, many(d), zz, many(y), torch.linspace(0.5, 1.5, T).cuda(), temperature=temperature)


# exponents on both sides of 2^22, where rows are summed by differences instead, in one row and apart
@pytest.mark.parametrize("offset,temperature", [(1e6, 1.0), (-1e6, 1.0), (2907270.0, 1.0), (-2907270.0, 1.0), (2e7, 3.0),
                                                (1e10, 500.0), (-1e10, 500.0), (29.0727, 1e-5), (-30.0, 1e-5), (3e12, 1e5)])
@pytest.mark.parametrize("T,V", [(3, 3001), (3, 70001), (100, 5003)])
def test_rows_far_from_zero(torch, T, V, offset, temperature):
    """Finite logits of any magnitude: only their differences count."""
    rng = np.random.default_rng(V)
    z = (offset + temperature * 3.0 * rng.standard_normal((T, V))).astype(np.float32)
    d, z = torch.from_numpy(z).cuda(), z.astype(np.float64)
    for k in (9, 150):
        _check_top(torch, d, z, k, temperature)
    ids, logp, tail = _teacher(torch, z, 9, temperature, seed=2, noise=temperature)
    for kind in ("forward", "reverse", "jsd"):
        _check_distill(torch, d, z, ids, logp, tail, kind=kind, temperature=temperature)
    _check_policy(torch, d, z, ids[:, 3].contiguous(), torch.linspace(0.5, 1.5, T).cuda(), temperature=temperature)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("T,V,k", [(9, 3001, 9), (9, 140001, 9), (9, 140001, 100), (99, 20011, 9), (3, 40, 40), (9, 257, 256)])
def test_top_logits_with_little_outside(torch, T, V, k, dtype):
    """The mass outside the list to its own precision however small it is, also
    where no float holds it: sharp rows, small temperatures, masks."""
    d, _ = _rows(torch, 9, V, dtype, seed=V + k)
    at = torch.randperm(V, generator=torch.Generator().manual_seed(k))[:k].cuda()
    top = torch.linspace(0, 5, k).cuda().to(d.dtype)
    d[1] -= 150.0
    d[2] -= 500.0
    d[3] = -1e4
    d[4] = -1e9
    d[5] = float(torch.finfo(d.dtype).min)
    d[6] = -float("inf")
    d[7] = -float("inf")
    d[7, V // 3] = -700.0                      # one segment has something outside, or it is on the list
    for t in range(1, 8):
        d[t, at] = top + (3000.0 if t == 2 else 0.0)
    z = d.double().cpu().numpy()
    many = lambda a: a.repeat((T + 8) // 9, *[1] * (a.dim() - 1))[:T]  # noqa: E731
    from paper_2605_27255_amd import opd_distill, opd_top_logits
    for temperature in (1.0, 1e-3, 30.0):
        ids, logp, tail = opd_top_logits(many(d), k, temperature)
        r_ids, r_logp, r_tail = (np.tile(r, ((T + 8) // 9,) + (1,) * (r.ndim - 1))[:T] for r in O.opd_top_logits(z, k, temperature))
        np.testing.assert_array_equal(ids.cpu().numpy(), r_ids)
        # what is below the least float32 (masks over 1e-3) is -inf in float32
        r_logp, r_tail = (np.where(r < -3.4028235e38, -np.inf, r) for r in (r_logp, r_tail))
        _close(logp, r_logp, DELTA + HALF["float32"] * np.abs(r_logp), "logp")
        _close(tail, r_tail, 2 * DELTA + HALF["float32"] * np.abs(r_tail), "tail")
    if V > k:
        # a student that has that mass is finitely far from such a teacher
        ids, logp, tail = opd_top_logits(d[:5], k)
        loss, _ = opd_distill(torch.zeros_like(d[:5]), ids, logp, tail, kind="reverse")
        assert loss.isfinite().all() and tail.isfinite().all()


@pytest.mark.parametrize("V", [777, 140001])
def test_policy_of_a_masked_label(torch, V):
    """A label of probability 0: the ratio of an on-policy call is 1 all the
    same, and a KL estimate of a token that the reference can draw is infinite."""
    from paper_2605_27255_amd import opd_policy
    d, _ = _rows(torch, 3, V, "float32", seed=V)
    y = torch.tensor([4, V - 1, 9], dtype=torch.int32).cuda()
    d[torch.arange(3), y.long()] = -float("inf")
    z, adv = d.double().cpu().numpy(), torch.tensor([1.5, -0.5, 2.0]).cuda()
    for grad in (True, None):
        loss, logp, _, g = _check_policy(torch, d, z, y, adv, grad=grad)
        assert torch.equal(loss, -adv) and torch.isneginf(logp).all()
        assert grad is None or torch.equal(g[torch.arange(3), y.long()], -adv)
        ref = torch.full((3,), -4.0).cuda()
        loss, _, kl, _ = opd_policy(d, y, adv, ref_logp=ref, grad=grad)
        assert torch.equal(loss, -adv) and torch.isposinf(kl).all()
        loss, _, kl, _ = opd_policy(d, y, adv, ref_logp=ref, kl_coef=0.1, grad=grad)
        assert torch.isposinf(loss).all() and torch.isposinf(kl).all()
        # ... of rollouts that another policy drew: ratio 0, clipped where the advantage is negative
        loss, _, _, _ = opd_policy(d, y, adv, old_logp=ref, grad=grad)
        assert torch.equal(loss, torch.where(adv < 0, -adv * 0.8, 0.0))


@pytest.mark.parametrize("T,V", [(5, 9001), (5, 60001)])
def test_policy_label_with_almost_all_mass(torch, T, V):
    """What the label's own gradient and log-probability lack to 0 is the mass of
    the other tokens, to its relative precision, however small that is."""
    d = torch.zeros((T, V), device="cuda")
    height = torch.tensor([10.0, 20.0, 37.0, 60.0, 80.0], device="cuda")
    d[:, 5] = height
    y, adv = torch.full((T,), 5, dtype=torch.int32).cuda(), torch.linspace(0.5, 1.5, T).cuda()
    from paper_2605_27255_amd import opd_policy
    _, logp, _, g = opd_policy(d, y, adv, grad=True)
    rest = (V - 1) * torch.exp(-height.double())
    want = -adv.double() * rest / (1 + rest)
    # the rest's sum carries DELTA, as does each gradient; half a step of the output
    assert ((g[:, 5].double() - want).abs() <= (DELTA + 2.0 ** -24) * want.abs()).all(), (g[:, 5], want)
    lp = -torch.log1p(rest)
    assert ((logp.double() - lp).abs() <= (DELTA + 2.0 ** -24) * lp.abs()).all(), (logp, lp)
    others = g.double().sum(1) - g[:, 5].double()
    assert ((g[:, 5].double() + others).abs() <= 2 * DELTA * want.abs()).all()


def test_gradient_over_the_logits_and_autograd(torch):
    """Writing the gradient over logits that a backward pass still needs is seen
    by autograd, as any other write is; over a leaf it is refused like one."""
    from paper_2605_27255_amd import PipoError, opd_distill, opd_policy
    gen = torch.Generator(device="cuda").manual_seed(3)
    h = torch.randn((6, 32), generator=gen, device="cuda")
    w = torch.randn((32, 700), generator=gen, device="cuda", requires_grad=True)
    y, adv = torch.arange(6, dtype=torch.int32).cuda(), torch.ones(6).cuda()
    ids, logp = torch.arange(24, dtype=torch.int32).cuda().view(6, 4), torch.full((6, 4), -1.5).cuda()
    for call in (lambda x, g: opd_distill(x, ids, logp, grad=g), lambda x, g: opd_policy(x, y, adv, grad=g)):
        x = h @ w                           # whose backward pass does not need its result
        x.backward(call(x, True)[-1])
        want, w.grad = w.grad, None
        x = h @ w
        x.backward(call(x, x)[-1])
        assert torch.equal(w.grad, want)
        w.grad = None
        x = 5 * torch.tanh(h @ w)
        capped = torch.tanh(h @ w)          # whose backward pass reads its result
        call(x, x)                          # (the factor's backward pass does not)
        g = call(capped, capped)[-1]
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            capped.backward(g)
        w.grad = None
        part = torch.tanh(h @ w)
        call(part.detach(), part.detach())  # the same memory by another tensor
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            part.sum().backward()
        w.grad = None
        leaf = (h @ w).detach().requires_grad_()
        before = leaf.detach().clone()
        for target in (leaf, leaf[:]):
            with pytest.raises(PipoError):
                call(leaf, target)
        assert torch.equal(leaf, before)
        with torch.no_grad():
            assert call(leaf, leaf)[-1] is leaf and not torch.equal(leaf, before)
        with torch.inference_mode():
            x = h @ w
            assert call(x, x)[-1] is x


def test_empty_chunk_with_an_empty_list(torch):
    """A chunk of nothing: no positions, no teacher rows."""
    from paper_2605_27255_amd import PipoError, opd_distill, opd_top_logits
    for dtype in (torch.float32, torch.bfloat16):
        z = torch.empty((0, 100), dtype=dtype, device="cuda")
        ids, logp, tail = opd_top_logits(z, 5)
        loss, g = opd_distill(z, ids, logp, tail, grad=True)
        assert loss.shape == (0,) and g.shape == (0, 100)
        with pytest.raises(PipoError):
            opd_distill(torch.zeros((2, 100), dtype=dtype, device="cuda"), ids, logp, tail)


# Rows that are split, by type and call: with the gradient, the loss alone, the top logits.
SPLIT = [("float32", 70001, True), ("bfloat16", 110001, True), ("float32", 151936, None), ("bfloat16", 210001, None)]


@pytest.mark.parametrize("dtype,V,grad", SPLIT)
def test_split_rows_labels_and_slots(torch, dtype, V, grad):
    """A row map, unscored positions, empty slots and flagged positions in split rows."""
    T, k = 12, 40
    assert _is_split(2 if grad else 1, T, V, k, dtype)
    d, z = _rows(torch, T, V, dtype, seed=V)
    ids, logp, tail = _teacher(torch, z[:8], k, 1.0, seed=6)
    rows = torch.tensor([0, 1, 1, 2, 3, 8, -1, 4, 5, 6, 7, 7], dtype=torch.int32).cuda()     # 8 and -1: no such row
    labels = torch.tensor([1, 1, -1, 1, 1, 1, 1, 1, 1, 1, -5, 2 ** 31 - 1], dtype=torch.int32).cuda()
    ids[2, ::3] = -1
    ids[3, :] = -7                       # nothing listed
    ids[4, 5] = V
    ids[5, 39] = ids[5, 0]
    ids[6, 0] = 2 ** 31 - 1
    flagged = [5, 6, 7, 8, 9]
    for tl in (tail, None):
        for kind in ("forward", "reverse", "jsd"):
            loss, g = _check_distill(torch, d, z, ids, logp, tl, rows=rows, labels=labels, kind=kind, grad=grad)
            assert loss[flagged].isnan().all() and not loss[[2, 10]].any()
            assert grad is None or (g[flagged].isnan().all() and not g[[2, 10]].any())
    y = torch.arange(T, dtype=torch.int32).cuda()
    y[1], y[3], y[5] = -1, V, V - 1
    adv, old, ref = torch.linspace(-1, 1, T).cuda(), torch.full((T,), -9.0).cuda(), torch.full((T,), -8.0).cuda()
    out = _check_policy(torch, d, z, y, adv, old, ref, torch.linspace(1, 2, T).cuda(), grad=grad, kl_coef=0.1)
    assert all(t is None or (t[3].isnan().all() and not t[1].any()) for t in out)


@pytest.mark.parametrize("dtype,V,grad", SPLIT)
def test_split_rows_with_masks_and_without_a_distribution(torch, dtype, V, grad):
    """Masked segments, a rest or a list without mass, lowest values, NaN and infinities in split rows."""
    assert _is_split(2 if grad else 1, 9, V, 16, dtype)
    d, z = _rows(torch, 9, V, dtype, seed=2)
    ids, logp, tail = _teacher(torch, z, 16, 1.0, seed=3)
    out = torch.ones(V, dtype=torch.bool, device="cuda")
    out[ids[1].long()] = False
    low = float(torch.finfo(d.dtype).min)
    d[0, ::2] = -float("inf")
    d[1, out] = -float("inf")            # the student has nothing outside the list
    d[2, ids[2].long()] = -float("inf")  # ... and nothing on it
    d[3] = -float("inf")
    d[4, V // 3: V - V // 3] = low       # whole segments of the lowest value
    d[5, 77] = float("nan")
    d[6, V - 78] = float("inf")
    d[7] = low
    d[8, : V // 2] = -float("inf")       # whole segments of nothing
    z = d.double().cpu().numpy()
    for kind in ("reverse", "jsd"):
        for tl in (tail, None):
            with np.errstate(all="ignore"):
                loss, g = _check_distill(torch, d, z, ids, logp, tl, kind=kind, grad=grad)
            assert loss[[3, 5, 6]].isnan().all() and loss[[0, 1, 2, 4, 7, 8]].isfinite().all()
            if grad:
                assert g[[3, 5, 6]].isnan().all() and g[[0, 1, 2, 4, 7, 8]].isfinite().all()
    y = torch.tensor([1, int(ids[1, 3]), 0, 0, 7, 5, 5, 9, V - 1], dtype=torch.int32).cuda()
    with np.errstate(all="ignore"):
        loss, logp, _, g = _check_policy(torch, d, z, y, torch.linspace(0.5, 1.5, 9).cuda(), torch.full((9,), -5.0).cuda(), grad=grad)
    assert loss[[3, 5, 6]].isnan().all() and loss[[0, 1, 2, 4, 7, 8]].isfinite().all()


@pytest.mark.parametrize("dtype,V", [("float32", 70001), ("bfloat16", 110001)])
def test_split_near_teacher_and_sharp_student(torch, dtype, V):
    k = 8
    assert _is_split(2, 3, V, k, dtype)
    d, z = _rows(torch, 3, V, dtype, seed=4)
    d[1] = 0
    d[1, 17] = 30.0
    d[2, :] = -50.0
    d[2, 3] = 45.0
    z = d.double().cpu().numpy()
    for noise in (0.0, 0.5):
        ids, logp, tail = _teacher(torch, z, k, 1.0, seed=9, noise=noise)
        for kind in ("forward", "reverse", "jsd"):
            _check_distill(torch, d, z, ids, logp, tail, kind=kind)
            _check_distill(torch, d, z, ids, logp, None, kind=kind, temperature=0.8)


@pytest.mark.parametrize("T", [95, 96, 97])
def test_rows_on_both_sides_of_the_split(torch, T):
    """The same rows in calls that split them and that do not: the same results to rounding, masked or not."""
    from paper_2605_27255_amd import opd_distill
    V = 50001
    assert _is_split(2, T, V, 9, "float32") == (T <= 96)
    d, z = _rows(torch, 5, V, "float32", seed=7)
    ids, logp, tail = _teacher(torch, z, 9, 1.0, seed=8)
    d[1, V // 2:] = -float("inf")
    only = ids[2:3].long()
    d[2:3] = torch.full_like(d[2:3], -float("inf")).scatter_(1, only, d[2:3].gather(1, only))
    d[3] = float(torch.finfo(torch.float32).min)
    z = d.double().cpu().numpy()
    pick = torch.arange(T).cuda() % 5
    loss, g = opd_distill(d[pick], ids[pick], logp[pick], tail[pick], kind="jsd", grad=True)
    torch.cuda.synchronize()
    r_loss, r_grad, size = O.opd_distill(z, *_host(ids, logp, tail), kind="jsd")
    for t in (0, 5, T - 5):
        at = (np.arange(5) + t) % 5
        _close(loss[t:t + 5], r_loss[at], (DELTA * size.sum(1) + HALF["float32"] * np.abs(r_loss))[at], "loss")
        _close(g[t:t + 5], r_grad[at], (4 * DELTA * size + HALF["float32"] * np.abs(r_grad) + 1e-37)[at], "grad")


def test_split_streams_and_graphs(torch):
    """Split top logits and losses on a side stream, and captured in two graphs replayed between eager calls."""
    from paper_2605_27255_amd import opd_distill, opd_policy, opd_top_logits
    T, V = 3, 70001
    assert all(_is_split(call, T, V, k, "float32") for call, k in ((0, 16), (2, 16), (2, 1)))
    gen = torch.Generator(device="cuda").manual_seed(1)
    fresh = lambda: 3 * torch.randn((T, V), generator=gen, device="cuda")  # noqa: E731
    s, te = fresh(), fresh()
    adv, y = torch.randn(T, generator=gen, device="cuda"), torch.randint(0, V, (T,), generator=gen, device="cuda").int()

    def step():
        ids, logp, tail = opd_top_logits(te, 16)
        return (ids, logp, tail) + opd_distill(s, ids, logp, tail, labels=y, grad=True)

    def policy():
        loss, logp, _, g = opd_policy(s, y, adv, grad=True)
        return opd_top_logits(s, 5) + (loss, logp, g)

    side = torch.cuda.Stream()
    want = [t.clone() for t in step() + policy()]
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step() + policy()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs, outs = [], []
    for fn in (step, policy):
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(fn())
        graphs.append(g)
    for i in range(4):
        s.copy_(fresh())
        te.copy_(fresh())
        for g in graphs if i % 2 else graphs[::-1]:
            g.replay()
        want = step() + policy()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs[0] + outs[1], want)), i


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("level", [0.0, -2907280.0, -2907200.0, -1e9])
@pytest.mark.parametrize("mask", [-float("inf"), -3e38])
@pytest.mark.parametrize("T,V", [(100, 40001), (3, 3001), (3, 110001)])
def test_rows_whose_beginning_and_list_are_masked(torch, T, V, mask, level, dtype):
    """No reference for the sum at the row's beginning nor on its list, and
    tokens at any level behind them (exponents on both sides of 2^22)."""
    d, _ = _rows(torch, 3, V, "float32", seed=V, pad=-V % 8)
    d += level
    d = d.to(getattr(torch, dtype))
    listed = torch.arange(0, 90, 10).int().cuda().repeat(3, 1)
    d[:, : V - 300] = mask
    z = d.double().cpu().numpy()
    logp, tail = torch.full((3, 9), -4.0).cuda(), torch.full((3,), -0.2).cuda()
    many = lambda a: a.repeat((T + 2) // 3, *[1] * (a.dim() - 1))[:T]  # noqa: E731
    zz = np.tile(z, ((T + 2) // 3, 1))[:T]
    for kind in ("reverse", "jsd"):
        for grad in (True, None):
            loss, g = _check_distill(torch, many(d), zz, many(listed), many(logp), many(tail), kind=kind, grad=grad)
            assert loss.isfinite().all()
    y = torch.tensor([V - 1, V - 300, V - 7], dtype=torch.int32).cuda()
    loss, _, _, g = _check_policy(torch, many(d), zz, many(y), torch.linspace(0.5, 1.5, T).cuda())
    assert loss.isfinite().all() and g.isfinite().all()


def test_split_calls_on_two_streams_at_once(torch):
    """Calls that overlap on two streams work in arrays of their own."""
    from paper_2605_27255_amd import opd_distill, opd_policy, opd_top_logits
    T, V = 8, 151936
    gen = torch.Generator(device="cuda").manual_seed(4)
    sets = []
    for _ in range(2):
        z = 3 * torch.randn((T, V), generator=gen, device="cuda")
        sets.append((z, torch.randint(0, V, (T,), generator=gen, device="cuda").int(), torch.randn(T, generator=gen, device="cuda")))

    def chain(z, y, adv):
        ids, logp, tail = opd_top_logits(z, 20)
        return (ids, logp, tail) + opd_distill(z, ids, logp, tail, kind="jsd", grad=True) + opd_policy(z, y, adv, grad=True)[:2]

    want = [[t.clone() for t in chain(*s)] for s in sets]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], [[], []]
    for _ in range(10):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(chain(*sets[i]))
    torch.cuda.synchronize()
    for i in range(2):
        for outs in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(outs, want[i]))
