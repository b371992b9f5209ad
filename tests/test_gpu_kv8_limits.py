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


# ---- scales, queries and scores of any magnitude ------------------------------------------------------------------------

def _rows_in_64_bits(q, c, table, pos, scale):
    """One request's rows q [n, n_q, D] (float64) at positions pos: output, sum p |v|, the largest p s and |score|s' size."""
    n, n_q, D = q.shape
    G = n_q // c.n_kv
    L = int(max(pos)) + 1
    at = np.arange(L)
    blk, off = table[at // c.block], at % c.block
    sc = c.scales.astype(np.float64)
    out, size, most, reach = (np.zeros((n, n_q, D)), np.zeros((n, n_q, D)), np.zeros((n, n_q)), np.zeros((n, n_q)))
    for h in range(n_q):
        k = (c.codes[0, blk, h // G, off].astype(np.float64) - 128) * sc[blk, h // G, 0][:, None]
        v = (c.codes[1, blk, h // G, off].astype(np.float64) - 128) * sc[blk, h // G, 1][:, None]
        s = q[:, h] @ k.T * scale
        s = np.where(at[None, :] <= np.asarray(pos)[:, None], s, -np.inf)
        p = np.exp(s - s.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        out[:, h], size[:, h] = p @ v, p @ np.abs(v)
        most[:, h] = (p * sc[blk, h // G, 1]).max(1)
        reach[:, h] = (np.abs(q[:, h]) @ np.abs(k).T).max(1) * abs(scale)
    return out, size, most, reach


def _close(got, ref, n, D, dtype):
    """Errors of a token's weight count by what it carries: the relative ones (test_gpu_kv8's, and 2^-17 for the log of a
    scale up to 2^126) with sum p |v|; fp16's smallest step, 2^-25 in units of 2^5 at least a token's largest weight times
    scale, with 128 of these for each of n tokens (bf16; the lower halves of fp32 probabilities: 2^-25 of 2^14)."""
    out, size, most, reach = ref
    e, half = 2.0 ** -24, dtype is torch.bfloat16
    rel = (2 * reach * (D + 8) * e + 16 * e + n / 8 * e + (2.0 ** -11 + 2.0 ** -17 if half else 0))[:, :, None]
    tol = rel * size + (n * 2.0 ** (-30 if half else -39) * 128 * most)[:, :, None]
    tol = tol * (1 + 2.0 ** -8) + np.abs(out) * (2.0 ** -8 if half else e) + 2.0 ** (-133 if half else -149)
    assert np.isfinite(got).all()
    assert (np.abs(got - out) <= tol).all(), (np.abs(got - out) / tol).max()


# one token; several heads' tokens (two tiles of rows a wave); a prompt's rows, whose waves share the tiles
SHAPES = {"one": (1, 4, 1), "rows": (6, 8, 2), "prompt": (600, 64, 8)}


def _attend(q, c, table, dtype, scale=None):
    """The GPU's rows and those of 64 bits: the request's last tokens, all of them or (of a prompt) some."""
    rows, n_q, D = q.shape
    total = int(table.shape[0]) * c.block
    x = torch.tensor(q).to(dtype)
    got = _api().kv8_attention(x.cuda(), to_gpu(c), _i32(table[None]), _i32([0, rows]), _i32([total]), scale=scale)
    some = np.arange(rows) if rows < 40 else np.concatenate([np.arange(0, rows, 71), [rows - 1]])
    ref = _rows_in_64_bits(x.double().numpy()[some], c, table, some + total - rows, D ** -0.5 if scale is None else scale)
    return got.double().cpu().numpy()[some], ref


CHAINS = {"falling": [1e15, 1e-4, 1e-18], "falling far": [1e30, 1e12, 1e-6], "to nothing": [1.0, 1e-18, 1e-36],
          "from above": [1e17, 1.0, 1e-18], "rising": [1e-18, 1e-4, 1e15], "rising far": [1e-36, 1e-18, 1.0, 1e18, 1e30],
          "both": [1.0, 1e-30, 1.0, 1e30, 1e-30, 1e10], "again and again": [1e12, 1e-6] * 6, "near": [1.0, 0.3, 0.01, 3.0, 40.0, 0.2],
          "zeros": [0.0, 1e-3, 0.0, 1e9, 0.0], "subnormal": [1e-40, 1e-44, 1e-39], "subnormal beside": [1e-3, 1e-40, 1e-3],
          "largest": [2.6e36, 1e-37, 2.6e36]}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("chain", sorted(CHAINS))
def test_attention_value_scales_in_steps(dtype, shape, chain):
    """A wave that takes blocks whose value scales rise and fall by many powers of two (the quarters of a range alike)."""
    rows, n_q, n_kv = SHAPES[shape]
    rng = np.random.default_rng(len(chain))
    steps = CHAINS[chain] * 4
    c = random_cache(rng, max(len(steps), 19), n_kv, 32, 64)
    table = rng.permutation(c.blocks)
    for i, b in enumerate(table):
        c.scales[b, :, 1] = steps[i % len(steps)]
    got, ref = _attend(rng.standard_normal((rows, n_q, 64)), c, table, dtype)
    _close(got, ref, len(table) * 32, 64, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tiles", [13, 140])
def test_attention_value_scales_at_random(dtype, tiles):
    for seed in range(6):
        rng = np.random.default_rng([seed, tiles])
        c = random_cache(rng, tiles, 2, 32, 128)
        c.scales[:, :, 1] = (10.0 ** rng.uniform(-30, 30, c.scales[:, :, 1].shape)).astype(np.float32)
        got, ref = _attend(rng.standard_normal((2, 8, 128)), c, rng.permutation(tiles), dtype)
        _close(got, ref, tiles * 32, 128, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("order", [[0, 1], [1, 0], [0, 1, 0], [0, 1, 2, 1, 0], [2, 0, 1], [0, 0, 2, 1, 1], [1, 2, 0]])
def test_attention_large_values_that_weigh_nothing(dtype, shape, order):
    """Blocks of huge values whose scores leave them no weight (e^-400), beside ones of small values: the output is
    the small ones', to its own precision.  (0: huge, 1: small, 2: huge too, by another 2^60.)"""
    rows, n_q, n_kv = SHAPES[shape]
    rng = np.random.default_rng(5)
    order = order * 4
    c = random_cache(rng, max(len(order), 20), n_kv, 32, 64)
    table = rng.permutation(c.blocks)
    for i, b in enumerate(table):
        kind = order[i % len(order)]
        c.scales[b, :, 1] = [1e18, 1e-5, 1e-18][kind] if kind != 2 else 1e36
        if kind != 1:
            c.codes[0, b] = 28
        c.scales[b, :, 0] = 0.5 if kind != 1 else 0.01
    got, ref = _attend(np.full((rows, n_q, 64), 1.0) + 0.1 * rng.standard_normal((rows, n_q, 64)), c, table, dtype)
    assert ref[1][-1].max() < 1e-2          # (a prompt's first rows may see huge ones only)
    _close(got, ref, len(table) * 32, 64, dtype)


def _key_case(rng, n_kv, D, key_scale, blocks=20):
    c = random_cache(rng, blocks, n_kv, 32, D)
    c.scales[:, :, 0] = key_scale * (0.5 + rng.random((blocks, n_kv))).astype(np.float32)
    return c, rng.permutation(blocks)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("q_size,key_scale,scale", [(3e37, 1e-39, None), (1e37, 2e-37, 0.01), (2e35, 1e-36, None), (1e-38, 1e36, None),
                                                    (1e-40, 1e36, 30.0), (1.0, 0.02, 1e-38), (1e-3, 1e-30, 1e33), (1e33, 1e3, 1e-36),
                                                    (1e30, 1e-35, 3e5)])
def test_attention_queries_and_keys_of_any_size(dtype, shape, q_size, key_scale, scale):
    """Queries, key scales and the scale of the scores far from 1, whose product is not: no step between passes 32 bits."""
    rows, n_q, n_kv = SHAPES[shape]
    rng = np.random.default_rng(7)
    c, table = _key_case(rng, n_kv, 64, key_scale)
    got, ref = _attend(q_size * np.clip(rng.standard_normal((rows, n_q, 64)), -3, 3), c, table, dtype, scale)
    _close(got, ref, len(table) * 32, 64, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", sorted(SHAPES))
@pytest.mark.parametrize("size", [1e6, 1e8, 1e9, 1e12, 1e20, 1e30])
def test_attention_scores_far_above_a_float_s_unit(dtype, shape, size):
    """Scores whose neighbours among floats are more than 1 apart: a token that is ahead by more than that takes all."""
    rows, n_q, n_kv = SHAPES[shape]
    rng = np.random.default_rng(9)
    c, table = _key_case(rng, n_kv, 64, 0.02)
    q = size * (1.0 + 0.1 * rng.standard_normal((rows, n_q, 64)))
    c.codes[0] = np.clip(c.codes[0], 100, 156)
    c.codes[0, table[0], :, 5] = 200            # its score is twice the others' in every row, and some are below 0
    got, ref = _attend(q, c, table, dtype)
    out, spread, most, _ = ref
    want = (c.codes[1, table[0], :, 5].astype(np.float64) - 128) * c.scales[table[0], :, 1][:, None]
    want = np.repeat(want, n_q // n_kv, 0)[None]
    np.testing.assert_allclose(out, np.broadcast_to(want, out.shape), rtol=1e-12)
    _close(got, (out, spread, most, np.zeros_like(most)), len(table) * 32, 64, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_codes_near_zero_beside_large_scales(dtype):
    """A block whose scale goes by one large key that the query does not see (its dimension is 0 there): the others'
    scores are 0, whatever cancels in them, and their average comes out to the roundings of 128 |q| scale."""
    rng = np.random.default_rng(10)
    for size in (1.0, 1e5, 1e9):
        c, table = _key_case(rng, 1, 64, 0.02 * size)
        c.codes[0] = 128
        c.codes[0, :, :, 3, 0] = 255
        q = rng.standard_normal((2, 4, 64))
        q[:, :, 0] = 0.0
        got, ref = _attend(q, c, table, dtype)
        assert np.isfinite(got).all()
        e = 2.0 ** -24 * 66 * 2 * 128 * 0.03 * size * np.abs(q).sum(2) / 8 if dtype is torch.bfloat16 else np.zeros((2, 4))
        out, spread, most, _ = ref
        tol = np.minimum(2 * np.expm1(np.minimum(e, 30.0)) + 2.0 ** -10, 2.0)[:, :, None] * np.maximum(spread, 4 * most[:, :, None] * 128)
        assert (np.abs(got - out) <= tol).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("total,new,n_q,n_kv", [([3000, 700, 45], [3, 1, 2], 8, 2), ([500, 400], [9, 3], 16, 2), ([900, 2300], [600, 1], 64, 8)])
def test_attention_same_bits_of_every_form(dtype, total, new, n_q, n_kv):
    """Key ranges and their join, several tiles of rows, prompts beside a request of few rows; scales that move units."""
    rng = np.random.default_rng(17)
    c, tables = _paged(rng, total, n_kv, 64, 128)
    c.scales[::3, :, 1] *= 100.0
    q = torch.tensor(rng.standard_normal((sum(new), n_q, 128))).to(dtype).cuda()
    args = to_gpu(c), _i32(tables), _i32(np.concatenate([[0], np.cumsum(new)])), _i32(total)
    first = _api().kv8_attention(q, *args)
    for _ in range(5):
        assert torch.equal(_api().kv8_attention(q, *args), first)
