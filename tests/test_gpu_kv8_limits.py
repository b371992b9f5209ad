"""The serving operators at the ends of what their calls allow: starts that hold anything, rows without a slot inside a
block, value and key scales, queries and scores of any magnitude.  Helpers, the oracle and the tolerances are those of
test_gpu_kv8."""
import numpy as np
import pytest

from oracle import pipo_oracle as O
from test_gpu_kv8 import _api, _append_both, _i32, _kv, _paged, assert_same_cache, random_cache, to_gpu
import test_gpu_verify as verify

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

INT_MAX, INT_MIN = 2 ** 31 - 1, -2 ** 31


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


# ---- starts that hold anything ------------------------------------------------------------------------------------------

WRAPPING = [[0, INT_MAX, -2, 3], [5, INT_MIN, 2, 4], [INT_MAX, INT_MIN, INT_MAX, INT_MIN], [2, -2 ** 30, 2 ** 30, -2 ** 30],
            [INT_MIN, INT_MAX, INT_MIN, 1], [1, INT_MIN + 1, INT_MAX - 1, INT_MIN + 2]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n_q,n_kv", [(9, 4, 2), (9, 16, 1), (1024, 64, 8)])      # (1024: prompts beside requests of few rows)
@pytest.mark.parametrize("starts", WRAPPING)
def test_attention_starts_whose_difference_wraps(dtype, rows, n_q, n_kv, starts):
    """Rows that are read and written stay inside the call's: NaN rows around the queries, guards around the output."""
    rng = np.random.default_rng(1)
    total = [50, 60, 3000]
    c, tables = _paged(rng, total, n_kv, 32, 64)
    x = torch.full((rows + 128, n_q, 64), float("nan"), dtype=dtype, device="cuda")
    x[64:64 + rows] = torch.tensor(rng.standard_normal((rows, n_q, 64))).to(dtype)
    y = torch.full((rows + 128, n_q, 64), 7.0, dtype=dtype, device="cuda")
    _api().kv8_attention(x[64:64 + rows], to_gpu(c), _i32(tables), _i32(starts), _i32(total), out=y[64:64 + rows])
    torch.cuda.synchronize()
    assert (y[:64] == 7.0).all() and (y[64 + rows:] == 7.0).all() and torch.isfinite(y.float()).all()


@pytest.mark.parametrize("starts", WRAPPING)
def test_verify_starts_whose_difference_wraps(starts):
    R, K, V, rows = 3, 3, 300, 12
    p, q, d, u = verify._case(2, R, K, V, torch.float32)
    x = torch.full((rows + 64, V), float("nan"), device="cuda")
    x[32:32 + rows] = torch.tensor(p).float()
    t, a = _api().verify_drafts(x[32:32 + rows], _i32(d), torch.tensor(u).cuda(), torch.tensor(q).float().cuda(), _i32(starts))
    t, a = t.cpu().numpy(), a.cpu().numpy()
    for r in range(R):
        mine = range(rows)[max(starts[r], 0):max(starts[r + 1], 0)]
        if not mine:
            assert a[r] == 0 and (t[r] == -1).all()
            continue
        want, accepted, margin = O.verify_drafts(p, d[r:r + 1], u[r:r + 1].astype(np.float64), q[r:r + 1],
                                                 np.array([mine[0], mine[-1] + 1]))
        if margin[0] > 4e-5:
            assert a[r] == accepted[0] and (t[r] == want[0]).all()


# ---- rows without a slot inside a block's run ---------------------------------------------------------------------------

def _with_holes(rng, slots, gaps):
    """The slots with runs of rows without one among them, of lengths drawn from `gaps`."""
    out = []
    for s in slots:
        out.append(int(s))
        if rng.random() < 0.4:
            hole = [-1, -2 ** 31, 2 ** 31 - 1][rng.integers(3)]
            out += [hole] * int(rng.choice(gaps))
    return np.array(out)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("slots,D", [([64, -1, 65], 64), ([64, -1, -1, 66, 65], 128), ([-1, 97, -1, 98, 96], 64),
                                     ([-1] * 70 + [40] + [-1] * 70 + [41, 42] + [-1] * 70, 64),
                                     ([33, 34] + [-1] * 61 + [35] + [-1] * 2000 + [36, 64] + [-1] * 1100 + [65], 128)])
def test_append_holes_inside_a_block(dtype, slots, D):
    rng = np.random.default_rng(len(slots))
    c = random_cache(rng, 4, 2, 32, D)
    k, v = _kv(rng, len(slots), 2, D, dtype, size=3.0)
    assert_same_cache(_append_both(c, k, v, np.array(slots), dtype), c)


@pytest.mark.parametrize("tokens,n_kv", [(40, 1), (300, 2), (3000, 2), (2500, 8)])     # (one to 64 rows a workgroup)
@pytest.mark.parametrize("gaps", [[1], [1, 3, 62, 63, 64, 65], [1, 1, 1, 1, 1500]])
def test_append_holes_anywhere(tokens, n_kv, gaps):
    rng = np.random.default_rng([tokens, n_kv, len(gaps)])
    block, D = 64, 64
    if len(gaps) == 5:
        tokens //= 8
    blocks = rng.permutation(tokens)
    slots, b = [], 0
    while len(slots) < tokens:          # runs from anywhere in a block, some backwards or with a slot twice
        at = int(rng.integers(0, block))
        run = list(range(at, int(rng.integers(at, block)) + 1))
        if rng.random() < 0.2:
            run = run[::-1] + run[:1]
        slots += [int(blocks[b]) * block + t for t in run]
        b += 1
    slots = _with_holes(rng, slots, gaps)
    c = random_cache(rng, tokens, n_kv, block, D)
    k, v = _kv(rng, len(slots), n_kv, D, torch.bfloat16)
    assert_same_cache(_append_both(c, k, v, slots, torch.bfloat16), c)
