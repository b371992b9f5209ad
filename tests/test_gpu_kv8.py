"""The paged 8-bit cache on the GPU against the float64 oracle: blocks and slots of a step's tokens, keys and values
into the cache and back, attention over it.

Whole numbers (tables, slots, codes) and scales have to be equal.  Attention's tolerance counts its roundings, for
A = the largest |v| and S = the largest sum |q k| scale that a row sees:
  fp32: queries as fp16 pairs, 2^-22 of each (and 2^-24 of the sum's 4 fp32 roundings a dimension's product chain), so
        S (2^-22 + D 2^-24) in every score, twice (numerator and sum), the exponential's argument
        (2^-24 of S each for product, difference, shift) and its own 2^-22, pairs of probabilities 2^-22, sums of n terms
        in chains of n / 32 additions 2^-24 each, joined: A (2 (S (2^-22 + (D + 4) 2^-24)) + 2^-20 + n / 8 2^-24);
  bf16: the same, a probability's fp16 rounding 2^-11 A, and half a step of the output, 2^-8 of the value.
"""
import os

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


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _bits(x, dtype):
    """float64 values of x rounded to the type."""
    return torch.tensor(x).to(dtype).double().numpy()


def to_gpu(c):
    """A Kv8Cache with the oracle cache's contents."""
    tiles = []
    for w in (0, 1):
        flat = np.empty((c.blocks, c.n_kv, c.block * c.D), dtype=np.uint8)
        flat[:, :, O.kv8_place(c.block, c.D, w)] = c.codes[w]
        last = (c.block // 16, c.D // 64) if w == 0 else (c.block // 32, c.D // 32)
        tiles.append(torch.tensor(flat.reshape(c.blocks, c.n_kv, *last, 64, 16)).cuda())
    return _api().Kv8Cache(*tiles, torch.tensor(c.scales).cuda())


def codes_of(cache):
    out = []
    for w, x in enumerate((cache.keys, cache.values)):
        flat = x.cpu().numpy().reshape(cache.blocks, cache.n_kv, -1)
        out.append(flat[:, :, O.kv8_place(cache.block, cache.head_dim, w)])
    return np.stack(out)


def random_cache(rng, blocks, n_kv, block, D):
    codes = np.clip(np.rint(128 + 40 * rng.standard_normal((2, blocks, n_kv, block, D))), 1, 255).astype(np.uint8)
    return O.Kv8Oracle(codes, (0.01 + 0.03 * rng.random((blocks, n_kv, 2))).astype(np.float32))


def assert_same_cache(cache, want):
    torch.cuda.synchronize()
    np.testing.assert_array_equal(cache.scales.cpu().numpy(), want.scales)
    np.testing.assert_array_equal(codes_of(cache), want.codes)


# ---- blocks and slots -------------------------------------------------------------------------------------------------

def _state(rng, lens, block, width, spare):
    held = np.array([-(-max(int(x), 0) // block) for x in lens])
    held = np.minimum(held, width)
    P = int(held.sum()) + spare
    ids = rng.permutation(P)
    tables = np.full((len(lens), width), -1)
    at = 0
    for r, h in enumerate(held):
        tables[r, :h] = ids[at:at + h]
        at += h
    free = np.concatenate([ids[at:], np.full(at, 7)])
    return tables, held, free, P - at


def check_plan(lens, new, state, rows, block):
    tables, held, free, n_free = state
    want = O.kv8_plan(lens, new, tables, held, free, n_free, rows, block)
    t, h, f, n = _i32(tables), _i32(held), _i32(free), _i32([n_free])
    got = _api().kv8_plan(_i32(lens), _i32(new), t, h, f, n, rows=rows, block=block)
    torch.cuda.synchronize()
    for name, x, y in zip(("starts", "total", "slots", "positions"), got, want[3:]):
        np.testing.assert_array_equal(x.cpu().numpy(), y, err_msg=name)
    np.testing.assert_array_equal(t.cpu().numpy(), want[0], err_msg="tables")
    np.testing.assert_array_equal(h.cpu().numpy(), want[1], err_msg="held")
    assert n.item() == len(want[2])
    np.testing.assert_array_equal(f.cpu().numpy()[:n.item()], want[2], err_msg="free")
    return want


@pytest.mark.parametrize("R", [1, 2, 63, 64, 65, 257, 1024, 1500])
@pytest.mark.parametrize("block", [32, 256])
@pytest.mark.parametrize("most", [1, 5, 300])
def test_plan(R, block, most):
    rng = np.random.default_rng([R, block, most])
    lens = rng.integers(0, 700, R)
    new = rng.integers(0, most + 1, R)
    new[rng.random(R) < 0.2] = -1
    width = -(-1000 // block) + 1
    rows = int(np.maximum(new, 0).sum()) + 3
    check_plan(lens, new, _state(rng, lens, block, width, -(-most // block) * R + 5), rows, block)


def test_plan_step_by_step_reuses_blocks():
    rng = np.random.default_rng(5)
    R, block, width, P = 7, 32, 9, 60
    tables, held, free, n_free = np.full((R, width), -1), np.zeros(R, int), np.arange(P), P
    lens = np.zeros(R, int)
    for step in range(20):
        new = rng.integers(0, 60, R)
        new[rng.random(R) < 0.25] = -1
        new = np.minimum(new, np.maximum(width * block - lens, 0))
        t, h, stack, _, total, _, _ = check_plan(lens, new, (tables, held, free, n_free), int(np.maximum(new, 0).sum()), block)
        tables, held, n_free = t, h, len(stack)
        free = np.concatenate([stack, np.full(P - n_free, 0)])
        lens = np.maximum(total - rng.integers(0, 3, R), 0)         # drafts are rejected: fewer than the blocks hold
        used = [b for r in range(R) for b in tables[r, :held[r]]]
        assert sorted(used + list(stack)) == list(range(P))         # every block once


@pytest.mark.parametrize("R", [9, 1300])
def test_plan_refuses_requests_one_by_one(R):
    rng = np.random.default_rng(R)
    block, width = 64, 6
    lens, new = rng.integers(0, 200, R), rng.integers(0, 150, R)
    lens[1], lens[2], new[3], new[4] = -5, width * block, 0, 0
    new[2] = 1                                                      # beyond its table
    state = _state(rng, lens, block, width, R // 2)                 # too few blocks
    check_plan(lens, new, state, int(np.maximum(new, 0).sum()), block)
    check_plan(lens, new, state, int(np.maximum(new, 0).sum()) // 2, block)     # nor rows
    check_plan(lens, new, state, 0, block)
    tables, held, free, _ = state
    check_plan(lens, new, (tables, held, free, 0), 4 * R, block)


def test_plan_of_more_requests_than_lds_holds():
    rng = np.random.default_rng(7)
    R = 5000
    lens, new = rng.integers(0, 90, R), rng.integers(0, 4, R)
    new[rng.random(R) < 0.1] = -1
    check_plan(lens, new, _state(rng, lens, 32, 4, R), int(np.maximum(new, 0).sum()) + 1, 32)


def test_plan_long_prompts():
    rng = np.random.default_rng(6)
    lens, new = np.array([0, 100, 4096, 7]), np.array([70001, 1, 30000, 0])
    check_plan(lens, new, _state(rng, lens, 64, 1200, 2000), 100010, 64)


# ---- into the cache and back --------------------------------------------------------------------------------------------

def _append_both(c, k, v, slots, dtype, wide=0):
    """Appends on both sides; k, v float64 already of the type's values. Returns the GPU's cache."""
    cache = to_gpu(c)
    n, H, D = k.shape
    x = torch.full((n, 2 * H + wide, D), float("nan"), dtype=dtype, device="cuda")
    x[:, :H], x[:, H:2 * H] = torch.tensor(k).to(dtype).cuda(), torch.tensor(v).to(dtype).cuda()
    _api().kv8_append(cache, x[:, :H], x[:, H:2 * H], _i32(slots))
    c.append(k, v, slots)
    return cache


def _kv(rng, n, H, D, dtype, size=1.0):
    return [_bits(size * rng.standard_normal((n, H, D)) * np.exp(0.5 * rng.standard_normal((n, H, 1))), dtype) for _ in "kv"]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block", [32, 64, 128, 256])
def test_append_prompts_and_tokens(dtype, D, block):
    rng = np.random.default_rng([D, block])
    H = 3
    c = random_cache(rng, 9, H, block, D)
    order = rng.permutation(9)
    # a prompt from a block's start over its border, one from inside a block, single tokens, rows that go nowhere
    slots = np.concatenate([order[0] * block + np.arange(block), order[1] * block + np.arange(block // 2 + 1),
                            order[2] * block + np.arange(block // 3, block), order[3] * block + np.arange(5),
                            [order[4] * block], [-1, -1], [order[5] * block + block - 1], [order[6] * block + 17],
                            [9 * block, 2 ** 31 - 1]])
    k, v = _kv(rng, len(slots), H, D, dtype)
    cache = _append_both(c, k, v, slots, dtype, wide=1)
    assert_same_cache(cache, c)
    # the same tokens again: nothing changes; then smaller and larger ones, which grow the scale
    for size in (1.0, 0.01, 30.0):
        k2, v2 = [_bits(size * x, dtype) for x in (k, v)]
        at = np.concatenate([order[3] * block + np.arange(5, 8), [order[4] * block + 1], [order[1] * block + block - 1]])
        cache = _append_both(c, k2[:5], v2[:5], at, dtype)
        assert_same_cache(cache, c)
    got = _api().kv8_read(cache, _i32(np.concatenate([slots, [-7]])), dtype=dtype)
    for w in (0, 1):
        want = torch.tensor(c.rows(w, np.concatenate([slots, [-7]]))).float().to(dtype)     # (exact in fp32: 8 x 24 bits rounded once)
        assert torch.equal(got[w].cpu(), want)


@pytest.mark.parametrize("rows", [1, 2, 64, 65, 255, 256, 257, 700, 1024, 1025, 4095, 4096, 5000])
def test_append_many_rows(rows):
    """Row counts on both sides of where a workgroup takes several rows, single tokens and prompts among them."""
    rng = np.random.default_rng(rows)
    block, H, D = 32, 2, 64
    slots, b = [], 0
    order = rng.permutation(rows + 1)
    while len(slots) < rows:
        n = min(int(rng.choice([1, 1, 3, 32, 90])), rows - len(slots))
        at = int(rng.integers(0, block))
        for i in range(n):
            slots.append(int(order[b + (at + i) // block]) * block + (at + i) % block)
        b += (at + n - 1) // block + 1
    c = random_cache(rng, rows + 1, H, block, D)
    k, v = _kv(rng, rows, H, D, torch.float32)
    assert_same_cache(_append_both(c, k, v, np.array(slots), torch.float32), c)


def test_append_one_token_after_the_other_is_what_the_rule_says():
    rng = np.random.default_rng(8)
    H, D, block = 2, 128, 64
    c = random_cache(rng, 3, H, block, D)
    cache = to_gpu(c)
    k, v = _kv(rng, 130, H, D, torch.bfloat16)
    for t in range(130):
        slots = np.array([(t // block) * block + t % block])
        _api().kv8_append(cache, torch.tensor(k[t:t + 1]).bfloat16().cuda(), torch.tensor(v[t:t + 1]).bfloat16().cuda(), _i32(slots))
        c.append(k[t:t + 1], v[t:t + 1], slots)
    assert_same_cache(cache, c)
    # every rounding was half a step of the scale then; the scale only grew: at most half a step each time it did
    got = _api().kv8_read(cache, _i32(np.arange(128)))
    for w, x in enumerate((k, v)):
        s = cache.scales[:2, :, w].cpu().numpy().repeat(block, 0)[:, :, None]
        assert (np.abs(got[w].cpu().numpy() - x[:128]) <= 0.5 * (1 + 20) * s).all()


def test_append_ties_round_to_even_and_repeated_slots_take_the_last_row():
    H, D, block = 1, 64, 32
    c = O.Kv8Oracle(np.full((2, 2, H, block, D), 9, np.uint8), np.ones((2, H, 2), np.float32))
    k = np.zeros((4, H, D))
    k[0, 0, :8] = [127, 0.5, 1.5, -2.5, 2.5, -0.5, 126.5, -127]         # scale 1: exact ties
    k[1], k[2], k[3] = 1000.0, 2.0, 3.0                                 # rows 1 and 2 have one slot: the later one counts
    slots = np.array([0, 1, 1, 2])
    cache = _append_both(c, k, k, slots, torch.float32)
    assert_same_cache(cache, c)
    assert c.scales[0, 0, 0] == 1.0 and list(c.codes[0, 0, 0, 0, :8]) == [255, 128, 130, 126, 130, 128, 254, 1]
    # the scale doubles: what was odd is a tie again
    k2 = np.zeros((1, H, D))
    k2[0, 0, 0] = 254
    cache = _append_both(c, k2, k2, np.array([5]), torch.float32)
    assert_same_cache(cache, c)
    assert list(c.codes[0, 0, 0, 0, :8]) == [192, 128, 129, 127, 129, 128, 191, 64]


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_append_of_what_is_not_finite_makes_the_head_of_the_block_nan(bad):
    rng = np.random.default_rng(3)
    H, D, block = 2, 64, 32
    c = random_cache(rng, 3, H, block, D)
    k, v = _kv(rng, 3, H, D, torch.bfloat16)
    k[1, 1, 5] = bad
    cache = _append_both(c, k, v, np.array([33, 34, 35]), torch.bfloat16)
    torch.cuda.synchronize()
    s = cache.scales.cpu().numpy()
    assert np.isnan(s[1, 1, 0]) and np.isfinite(np.delete(s.ravel(), (1 * H + 1) * 2)).all()
    got = _api().kv8_read(cache, _i32([32, 34, 63, 0]))[0].cpu().numpy()
    assert np.isnan(got[:3, 1]).all() and np.isfinite(got[:3, 0]).all() and np.isfinite(got[3]).all()
    cache2 = _append_both(c, k[:1], v[:1], np.array([36]), torch.bfloat16)          # still
    assert np.isnan(cache2.scales.cpu().numpy()[1, 1, 0])
    cache3 = _append_both(c, k[:1], v[:1], np.array([32]), torch.bfloat16)          # until the block begins anew
    assert np.isfinite(cache3.scales.cpu().numpy()).all()


def test_append_of_tiny_and_huge_values():
    H, D, block = 2, 64, 32
    for size in (0.0, 1e-44, 2.0 ** -126, 126.9 * 2.0 ** -126, 1e-30, 1e38):
        c = O.Kv8Oracle(np.full((2, 1, H, block, D), 77, np.uint8), np.full((1, H, 2), 5.0, np.float32))
        k = _bits(size * np.linspace(-1, 1, 3 * H * D).reshape(3, H, D), torch.float32)
        assert_same_cache(_append_both(c, k, k[::-1].copy(), np.array([0, 1, 2]), torch.float32), c)


# ---- attention ----------------------------------------------------------------------------------------------------------

def _paged(rng, totals, n_kv, block, D, spare=2, width=None):
    need = [-(-max(int(t), 0) // block) for t in totals]
    P = max(sum(need) + spare, 1)
    ids, tables, at = rng.permutation(P), np.full((len(totals), max(width or 0, max(need), 1)), -1), 0
    for r, n in enumerate(need):
        tables[r, :n] = ids[at:at + n]
        at += n
    return random_cache(rng, P, n_kv, block, D), tables


def _tolerance(want, size, top, D, n, dtype):
    e = 2.0 ** -24
    t = top * (2 * size * (4 * e + (D + 4) * e) + 16 * e + n / 8 * e)
    if dtype is torch.bfloat16:
        return (t + top * 2.0 ** -11)[:, :, None] * (1 + 2.0 ** -8) + np.abs(want) * 2.0 ** -8
    return t[:, :, None] + np.abs(want) * e


def check_attention(q, c, tables, starts, total, dtype, scale=None, max_len=None, cache=None, wide=0):
    rows, n_q, D = q.shape
    x = torch.full((rows, n_q + wide, D), float("nan"), dtype=dtype, device="cuda")
    x[:, :n_q] = torch.tensor(q).to(dtype).cuda()
    y = torch.full((rows, n_q + wide, D), 7.0, dtype=dtype, device="cuda")
    out = _api().kv8_attention(x[:, :n_q], cache or to_gpu(c), _i32(tables), _i32(starts), _i32(total), scale=scale,
                               max_len=max_len, out=y[:, :n_q])
    torch.cuda.synchronize()
    want, size, top = O.kv8_attention(q, c, tables, starts, total, scale, max_len)
    got = out.double().cpu().numpy()
    assert (y[:, n_q:] == 7.0).all()
    covered = np.zeros(rows, bool)
    covered[starts[0]:starts[-1]] = True
    assert (got[~covered] == 7.0).all()                     # rows behind the last request stay as they were
    err, tol = np.abs(got - want)[covered], _tolerance(want, size, top, D, tables.shape[1] * c.block, dtype)[covered]
    assert np.isfinite(got).all() and (err <= tol).all(), (err / np.maximum(tol, 1e-300)).max()
    return out


PATTERNS = {
    "one": ([1], [1]), "two": ([31, 2], [1, 2]), "borders": ([32, 33, 64, 65, 96], [1, 1, 1, 1, 1]),
    "verify": ([500, 70, 3, 129], [5, 4, 3, 1]), "prompt": ([150], [150]), "chunk": ([333, 40], [77, 40]),
    "mixed": ([700, 1, 90, 260], [1, 1, 60, 9]),
}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("pattern", sorted(PATTERNS))
@pytest.mark.parametrize("heads", [(2, 2), (4, 1), (15, 3), (14, 2), (16, 1)])
def test_attention(dtype, D, pattern, heads):
    n_q, n_kv = heads
    total, new = PATTERNS[pattern]
    rng = np.random.default_rng([D, n_q, len(pattern), total[0]])
    block = int(rng.choice([32, 64, 128, 256]))
    c, tables = _paged(rng, total, n_kv, block, D)
    starts = np.concatenate([[0], np.cumsum(new)])
    q = _bits(1.5 * rng.standard_normal((starts[-1] + 2, n_q, D)), dtype)
    check_attention(q, c, tables, starts, np.array(total), dtype, wide=3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block", [32, 64, 128, 256])
def test_attention_long_contexts_are_split(dtype, block):
    rng = np.random.default_rng(block)
    total, new = [4100, 1, 2049, 1023], [1, 1, 2, 3]
    c, tables = _paged(rng, total, 2, block, 128)
    starts = np.concatenate([[0], np.cumsum(new)])
    q = _bits(rng.standard_normal((7, 8, 128)), dtype)
    check_attention(q, c, tables, starts, np.array(total), dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_many_rows_take_a_group_each(dtype):
    """Enough row groups that the waves of a workgroup take different ones, beside requests of a few rows, which get
    key ranges: no rows, one token of many, the most rows that count as few and one more."""
    rng = np.random.default_rng(12)
    total, new = [700, 5000, 2300, 0, 3100, 900, 40], [600, 1, 2200, 2, 4, 5, 0]        # (8 heads: 32 and 40 rows)
    c, tables = _paged(rng, total, 8, 64, 64)
    starts = np.concatenate([[0], np.cumsum(new)])
    n = starts[-1]
    q = _bits(rng.standard_normal((n, 64, 64)), dtype)
    x = torch.tensor(q).to(dtype).cuda()
    out = _api().kv8_attention(x, to_gpu(c), _i32(tables), _i32(starts), _i32(total)).double().cpu().numpy()
    assert (out[starts[3]:starts[4]] == 0).all()
    for rows in (range(0, 5), range(597, 603), range(1500, 1503), range(n - 14, n)):        # (the oracle is slow)
        for i in rows:
            r = int(np.searchsorted(starts, i, side="right")) - 1
            if total[r] == 0:
                continue
            pos = total[r] - starts[r + 1] + i
            want, size, top = O.kv8_attention(q[i:i + 1], c, tables[r:r + 1], np.array([0, 1]), np.array([pos + 1]))
            tol = _tolerance(want, size, top, 64, 5000, dtype)
            assert (np.abs(out[i:i + 1] - want) <= tol).all(), i


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_rows_that_see_nothing_and_blocks_that_are_not_there(dtype):
    rng = np.random.default_rng(4)
    total, new = [0, 200, 2, 100, 64], [3, 2, 4, 1, 0]      # no tokens, more rows than tokens, no rows
    c, tables = _paged(rng, total, 2, 32, 64, width=9)
    tables[1, 2], tables[1, 4], tables[3, 0] = -1, c.blocks, 2 ** 31 - 1        # holes: their tokens are not there
    starts = np.concatenate([[0], np.cumsum(new)])
    q = _bits(rng.standard_normal((11, 4, 64)), dtype)
    out = check_attention(q, c, tables, starts, np.array(total), dtype)
    assert (out[:3] == 0).all() and (out[5:7] == 0).all()
    check_attention(q, c, tables, starts, np.array([-5, 2 ** 31 - 1, -2 ** 31, 100, 64]), dtype)     # lengths cut off at the table
    check_attention(q, c, tables, starts, np.array(total), dtype, max_len=70)
    tables[:] = -1
    assert (check_attention(q, c, tables, starts, np.array(total), dtype)[:10] == 0).all()


@pytest.mark.parametrize("R", [63, 64, 65, 300, 4097, 5000])
def test_attention_of_many_requests(R):
    """A lane looks at one request, or at the first of several: both sides of 64 and of 64 x 64."""
    rng = np.random.default_rng(R)
    total, new = rng.integers(0, 5, R), rng.integers(0, 3, R)
    total[R // 2], new[R // 2], new[0] = 90, 7, 1
    c, tables = _paged(rng, total, 1, 32, 64)
    starts = np.concatenate([[0], np.cumsum(new)])
    q = _bits(rng.standard_normal((starts[-1], 2, 64)), torch.bfloat16)
    check_attention(q, c, tables, starts, total, torch.bfloat16)


def test_attention_starts_that_leave_rows_out():
    rng = np.random.default_rng(9)
    c, tables = _paged(rng, [50, 60], 2, 32, 64)
    q = _bits(rng.standard_normal((9, 4, 64)), torch.float32)
    check_attention(q, c, tables, np.array([3, 5, 6]), np.array([50, 60]), torch.float32)
    x, y = torch.tensor(q).float().cuda(), torch.full((9, 4, 64), 7.0, device="cuda")
    for starts in ([0, 2 ** 31 - 1, 4], [-3, 2, 1], [5, 3, 100], [2 ** 31 - 1, 0, -2 ** 31]):        # nonsense: nothing out of bounds
        out = _api().kv8_attention(x, to_gpu(c), _i32(tables), _i32(starts), _i32([50, 60]), out=y)
        torch.cuda.synchronize()
        assert out.shape == q.shape


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_attention_a_bad_block_spoils_only_who_sees_it(dtype):
    rng = np.random.default_rng(11)
    total, new = [70, 70], [40, 1]
    c, tables = _paged(rng, total, 2, 32, 64)
    q = _bits(rng.standard_normal((41, 4, 64)), dtype)
    starts = np.array([0, 40, 41])
    clean = check_attention(q, c, tables, starts, np.array(total), dtype)
    for w in (0, 1):
        c2 = O.Kv8Oracle(c.codes, c.scales.copy())
        c2.scales[tables[0, 2], 1, w] = np.nan              # positions 64 .. of request 0, KV head 1
        got = _api().kv8_attention(torch.tensor(q).to(dtype).cuda(), to_gpu(c2), _i32(tables), _i32(starts), _i32(total))
        nan = torch.isnan(got)
        assert nan[34:40, 2:].all() and not nan[:34].any() and not nan[:, :2].any() and not nan[40].any()
        assert torch.equal(got[~nan], clean[~nan])
    # a query with a NaN or infinity spoils its own row and head
    q2 = q.copy()
    q2[3, 1, 0], q2[5, 2, 7] = np.nan, np.inf
    got = _api().kv8_attention(torch.tensor(q2).to(dtype).cuda(), to_gpu(c), _i32(tables), _i32(starts), _i32(total))
    nan = torch.isnan(got)
    assert nan[3, 1].all() and nan[5, 2].all()
    nan[3, 1], nan[5, 2] = False, False
    assert not nan.any()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("q_size,scale", [(1e-30, 1e28), (3e4, 1e-5), (1e30, 1e-31), (0.0, None), (1.0, 0.0), (1.0, -0.125), (40.0, None)])
def test_attention_scales(dtype, q_size, scale):
    rng = np.random.default_rng(13)
    c, tables = _paged(rng, [300], 1, 64, 128)
    q = _bits(q_size * rng.standard_normal((2, 4, 128)), dtype)
    check_attention(q, c, tables, np.array([0, 2]), np.array([300]), dtype, scale=scale)


def test_attention_scales_of_blocks_that_differ_widely():
    rng = np.random.default_rng(14)
    c, tables = _paged(rng, [400], 1, 32, 64)
    c.scales[:, :, 1] = (10.0 ** rng.uniform(-30, 30, c.scales[:, :, 1].shape)).astype(np.float32)
    c.scales[tables[0, 3], 0, :] = 0.0
    c.scales[tables[0, 4], 0, 0] *= 200.0
    q = _bits(rng.standard_normal((1, 4, 64)), torch.float32)
    check_attention(q, c, tables, np.array([0, 1]), np.array([400]), torch.float32)


def test_attention_far_blocks_of_a_large_cache():
    """Offsets beyond 32 bits: the request's blocks lie behind 4 GiB of keys and of values."""
    rng = np.random.default_rng(15)
    n_kv, D, block = 8, 128, 256
    P = (1 << 32) // (n_kv * D * block) + 40
    A = _api()
    cache = A.Kv8Cache(torch.empty((P, n_kv, block // 16, 2, 64, 16), dtype=torch.uint8, device="cuda"),
                       torch.empty((P, n_kv, block // 32, 4, 64, 16), dtype=torch.uint8, device="cuda"),
                       torch.zeros((P, n_kv, 2), device="cuda"))
    c = random_cache(rng, 40, n_kv, block, D)
    slots = (P - 40) * block + np.arange(600)
    k, v = _kv(rng, 600, n_kv, D, torch.bfloat16)
    A.kv8_append(cache, torch.tensor(k).bfloat16().cuda(), torch.tensor(v).bfloat16().cuda(), _i32(slots))
    c.append(k, v, np.arange(600))
    got = A.kv8_read(cache, _i32(slots[::37]))
    for w in (0, 1):
        assert torch.equal(got[w].cpu(), torch.tensor(c.rows(w, np.arange(600)[::37])).float())
    q = _bits(rng.standard_normal((1, 16, D)), torch.bfloat16)
    near = np.arange(3)[None]
    want, size, top = O.kv8_attention(q, c, near, np.array([0, 1]), np.array([600]))
    out = A.kv8_attention(torch.tensor(q).bfloat16().cuda(), cache, _i32(near + P - 40), _i32([0, 1]), _i32([600]))
    assert (np.abs(out.double().cpu().numpy() - want) <= _tolerance(want, size, top, D, 768, torch.bfloat16)).all()


def test_attention_without_a_work_array_and_with_a_small_one():
    """The C entry: NULL works (no split over workgroups), too small a work array is refused."""
    import ctypes
    from paper_2605_27255_amd import pipo
    rng = np.random.default_rng(16)
    c, tables = _paged(rng, [3000], 2, 64, 64)
    q = _bits(rng.standard_normal((1, 4, 64)), torch.float32)
    cache, lib = to_gpu(c), pipo.load_library()
    x, out = torch.tensor(q).float().cuda(), torch.zeros((1, 4, 64), device="cuda")
    t, s, n = _i32(tables), _i32([0, 1]), _i32([3000])
    need = lib.pipo_kv8_attention_work_bytes(ctypes.byref(cache.c), 1, 1, 4, 3000, 0)
    assert need > 0
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    call = lambda w, b: lib.pipo_kv8_attention(ctypes.byref(cache.c), 1, 1, 4, x.data_ptr(), 256, t.data_ptr(),  # noqa: E731
                                               tables.shape[1], s.data_ptr(), n.data_ptr(), 3000, 0.125, out.data_ptr(),
                                               256, w, b, torch.cuda.current_stream().cuda_stream)
    assert call(work.data_ptr(), need - 1) == pipo.PIPO_EINVAL
    want, size, top = O.kv8_attention(q, c, tables, np.array([0, 1]), np.array([3000]))
    for w, b in ((None, 0), (work.data_ptr(), need)):
        out.zero_()
        assert call(w, b) == pipo.PIPO_OK
        torch.cuda.synchronize()
        assert (np.abs(out.double().cpu().numpy() - want) <= _tolerance(want, size, top, 64, 3008, torch.float32)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [1, 3, 5])
def test_rows_at_any_element(dtype, shift):
    """Keys, values, queries and outputs that begin off the 16-byte grid, in rows of odd stride."""
    rng = np.random.default_rng(20)
    total, new, D = [70, 45], [3, 2], 64
    c, tables = _paged(rng, total, 2, 32, D)
    k, v = _kv(rng, 5, 2, D, dtype)
    q = _bits(rng.standard_normal((5, 4, D)), dtype)
    slots = np.array([tables[0, t // 32] * 32 + t % 32 for t in (67, 68, 69)] + [tables[1, t // 32] * 32 + t % 32 for t in (43, 44)])

    def at(x):
        n, h, _ = x.shape
        ld = h * D + 7
        flat = torch.full((n * ld + 16,), 7.0, dtype=dtype, device="cuda")
        y = flat.as_strided((n, h, D), (ld, D, 1), shift)
        y.copy_(torch.tensor(x).to(dtype))
        return y

    cache = to_gpu(c)
    _api().kv8_append(cache, at(k), at(v), _i32(slots))
    c.append(k, v, slots)
    assert_same_cache(cache, c)
    out = at(np.zeros_like(q))
    _api().kv8_attention(at(q), cache, _i32(tables), _i32([0, 3, 5]), _i32(total), out=out)
    want, size, top = O.kv8_attention(q, c, tables, np.array([0, 3, 5]), np.array(total))
    assert (np.abs(out.double().cpu().numpy() - want) <= _tolerance(want, size, top, D, 96, dtype)).all()
    assert (out._base.as_strided((4, 7), (4 * D + 7, 1), shift + 4 * D) == 7.0).all()      # nothing between the rows


def test_appends_on_two_streams_to_different_blocks():
    rng = np.random.default_rng(21)
    c = random_cache(rng, 40, 2, 64, 128)
    cache = to_gpu(c)
    parts = []
    for i in range(2):
        slots = np.concatenate([np.arange(64 * b, 64 * b + 64) for b in range(20 * i, 20 * i + 20)])
        parts.append((slots, *_kv(rng, len(slots), 2, 128, torch.bfloat16)))
    gpu = [(_i32(s), torch.tensor(k).bfloat16().cuda(), torch.tensor(v).bfloat16().cuda()) for s, k, v in parts]
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(torch.cuda.Stream()):
            _api().kv8_append(cache, gpu[i][1], gpu[i][2], gpu[i][0])
    for s, k, v in parts:
        c.append(k, v, s)
    assert_same_cache(cache, c)


def test_python_calls_refuse_what_does_not_fit():
    A = _api()
    cache = A.Kv8Cache.new(4, 2, 64)
    assert (cache.blocks, cache.n_kv, cache.block, cache.head_dim) == (4, 2, 64, 64)
    x = torch.zeros((3, 2, 64), device="cuda")
    q, i = torch.zeros((3, 4, 64), device="cuda"), lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    t, s, n = i(1, 2), i(2), i(1)
    bad = [lambda: A.Kv8Cache(cache.keys, cache.values[:3], cache.scales), lambda: A.Kv8Cache(cache.keys[:, :, ::2], cache.values, cache.scales),
           lambda: A.Kv8Cache(cache.keys.char(), cache.values, cache.scales), lambda: A.Kv8Cache(cache.keys.cpu(), cache.values, cache.scales),
           lambda: A.kv8_append(cache, x, x[:2], i(3)), lambda: A.kv8_append(cache, x, x.bfloat16(), i(3)),
           lambda: A.kv8_append(cache, x.half(), x.half(), i(3)), lambda: A.kv8_append(cache, x, x, i(4)),
           lambda: A.kv8_append(cache, x, x, i(3).long()), lambda: A.kv8_append(cache, x[:, :1], x[:, :1], i(3)),
           lambda: A.kv8_append(cache, x.transpose(1, 2), x, i(3)), lambda: A.kv8_append(cache, x[:1].expand(3, 2, 64), x, i(3)),
           lambda: A.kv8_read(cache, i(3), dtype=torch.float16), lambda: A.kv8_read(cache, i(3).cpu()),
           lambda: A.kv8_attention(q[:, :3], cache, t, s, n), lambda: A.kv8_attention(q.half(), cache, t, s, n),
           lambda: A.kv8_attention(q, cache, t, i(3), n), lambda: A.kv8_attention(q, cache, t, s, i(2)),
           lambda: A.kv8_attention(q, cache, t, s, n, max_len=129), lambda: A.kv8_attention(q, cache, t, s, n, max_len=0),
           lambda: A.kv8_attention(q, cache, t, s, n, scale=float("nan")), lambda: A.kv8_attention(q, cache, t, s, n, out=q[:2]),
           lambda: A.kv8_attention(q, cache, t, s, n, out=q.bfloat16()),
           lambda: A.kv8_attention(q, cache, t, s, n, out=torch.zeros_like(q, requires_grad=True)),
           lambda: A.kv8_plan(i(2), i(2), i(2, 3), i(2), i(5), i(1), rows=4, block=48), lambda: A.kv8_plan(i(2), i(3), i(2, 3), i(2), i(5), i(1), rows=4, block=32),
           lambda: A.kv8_plan(i(2), i(2), i(2, 3), i(2), i(5), i(1), rows=-1, block=32)]
    for call in bad:
        with pytest.raises(A.PipoError):
            call()
    # nothing to do is no error
    A.kv8_append(cache, x[:0], x[:0], i(0))
    assert A.kv8_read(cache, i(0))[0].shape == (0, 2, 64) and A.kv8_attention(q[:0], cache, t, s, n).shape == (0, 4, 64)


@pytest.mark.parametrize("total,new", [([3000, 40], [3, 1]), ([2200, 700], [2200, 600])])
def test_attention_over_its_own_queries(total, new):
    """Short and split rows, and a prompt's: the output in place of the queries, in a wider tensor."""
    rng = np.random.default_rng(19)
    c, tables = _paged(rng, total, 8, 64, 64)
    cache, args = to_gpu(c), (_i32(tables), _i32(np.concatenate([[0], np.cumsum(new)])), _i32(total))
    x = torch.tensor(rng.standard_normal((sum(new), 70, 64))).bfloat16().cuda()
    want = _api().kv8_attention(x[:, 3:67], cache, *args)
    rest = x[:, 67:].clone(), x[:, :3].clone()
    _api().kv8_attention(x[:, 3:67], cache, *args, out=x[:, 3:67])
    assert torch.equal(x[:, 3:67], want) and torch.equal(x[:, 67:], rest[0]) and torch.equal(x[:, :3], rest[1])
    with pytest.raises(_api().PipoError):
        _api().kv8_attention(x[:, 3:67], cache, *args, out=x[:, 4:68])


def test_attention_same_bits_every_time():
    rng = np.random.default_rng(17)
    total, new = [3000, 700, 45], [3, 1, 2]
    c, tables = _paged(rng, total, 2, 64, 128)
    q = torch.tensor(rng.standard_normal((6, 8, 128))).float().cuda()
    args = to_gpu(c), _i32(tables), _i32([0, 3, 4, 6]), _i32(total)
    first = _api().kv8_attention(q, *args)
    for _ in range(5):
        assert torch.equal(_api().kv8_attention(q, *args), first)


# ---- together ---------------------------------------------------------------------------------------------------------------

def test_two_streams_at_once():
    rng = np.random.default_rng(18)
    total, new = [3000, 700], [3, 1]
    c, tables = _paged(rng, total, 2, 64, 128)
    cache, args = to_gpu(c), (_i32(tables), _i32([0, 3, 4]), _i32(total))
    qs = [torch.tensor(rng.standard_normal((4, 8, 128))).bfloat16().cuda() for _ in range(2)]
    want = [_api().kv8_attention(q, cache, *args) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(_api().kv8_attention(qs[i], cache, *args))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


class _Server:
    """A toy target model's serving state: its 'layer' makes keys, values and queries from token and position tables."""

    def __init__(self, seed, R, K, V, n_q, n_kv, D, block, width, blocks):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        self.R, self.K, self.V, self.block = R, K, V, block
        self.tok = rnd(V, n_q + 2 * n_kv, D).bfloat16()
        self.head = (0.2 * rnd(n_q * D, V))
        self.shape = n_q, n_kv, D
        self.cache = _api().Kv8Cache.new(blocks, n_kv, D, block)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.tables, self.held = torch.full((R, width), -1, **i32), torch.zeros(R, **i32)
        self.free, self.n_free = torch.arange(blocks, **i32), torch.full((1,), blocks, **i32)
        self.lens, self.last = torch.zeros(R, **i32), torch.arange(R, **i32)

    def step(self, tokens, new, rows):
        """tokens [rows] flat: what each request's step feeds (its known token, then drafts)."""
        A, (n_q, n_kv, D) = _api(), self.shape
        starts, total, slots, positions = A.kv8_plan(self.lens, new, self.tables, self.held, self.free, self.n_free,
                                                     rows=rows, block=self.block)
        x = self.tok[tokens.long()] * (1.0 + 0.01 * positions.clamp(min=0)[:, None, None]).bfloat16()
        A.kv8_append(self.cache, x[:, n_q:n_q + n_kv], x[:, n_q + n_kv:], slots)
        o = A.kv8_attention(x[:, :n_q], self.cache, self.tables, starts, total)
        logits = o.reshape(rows, -1).float() @ self.head
        self.seen = x, o
        return starts, logits


def _serve(seed, steps, graph):
    """Verified decoding of three requests, of which one draft list is shorter; returns every step's outputs."""
    A = _api()
    R, K, V = 3, 3, 97
    s = _Server(seed, R, K, V, 4, 2, 64, 32, 12, 40)
    g = torch.Generator().manual_seed(seed)
    new = _i32([K + 1, K + 1, K])
    drafts = torch.zeros((R, K), dtype=torch.int32, device="cuda")
    u = torch.zeros((R, K + 1), device="cuda")
    rows = 3 * K + 2
    out = {}

    def one():
        flat = torch.cat([s.last[0:1], drafts[0], s.last[1:2], drafts[1], s.last[2:3], drafts[2, :K - 1]])
        starts, logits = s.step(flat, new, rows)
        tokens, accepted = A.verify_drafts(logits, drafts, u, starts=starts, temperature=0.0)
        out.update(tokens=tokens, accepted=accepted, logits=logits)
        s.lens.add_(accepted).add_(1)
        s.last.copy_(tokens.gather(1, accepted.long()[:, None])[:, 0])

    seen, plan = [], None
    for step in range(steps):
        drafts.copy_(torch.randint(0, V, (R, K), generator=g).int())
        if seen:        # drafts of which some are right: what the greedy target said last time for these contexts
            drafts[:, 0] = seen[-1][0][:, 0].cuda().clamp(min=0)
        drafts[2, K - 1] = -1
        if not graph or step < 2:
            one()
        else:
            if plan is None:
                torch.cuda.synchronize()
                keep = [x.clone() for x in (s.tables, s.held, s.free, s.n_free, s.lens, s.last)]
                plan = torch.cuda.CUDAGraph()
                with torch.cuda.graph(plan):
                    one()
                for x, y in zip((s.tables, s.held, s.free, s.n_free, s.lens, s.last), keep):
                    x.copy_(y)
            plan.replay()
        torch.cuda.synchronize()
        seen.append([x.cpu().clone() for x in (out["tokens"], out["accepted"], out["logits"], s.lens, drafts, *s.seen)])
    return s, seen


def test_a_run_of_all_operators_captured_and_eager():
    s, eager = _serve(1, 24, False)
    _, replayed = _serve(1, 24, True)
    for step, (a, b) in enumerate(zip(eager, replayed)):
        for x, y in zip(a, b):
            assert torch.equal(x, y), step
    held = s.held.cpu().numpy()
    assert (held >= -(-s.lens.cpu().numpy() // 32)).all() and held.sum() + s.n_free.item() == 40


def test_a_run_of_all_operators_is_the_oracles():
    """Every step's blocks, cache, attention and verdicts, the oracle fed with what each layer made of the tokens."""
    s, seen = _serve(2, 12, False)
    n_q, n_kv, D = s.shape
    R, K, V, rows = s.R, s.K, s.V, 3 * s.K + 2
    c = O.Kv8Oracle(np.zeros((2, 40, n_kv, 32, D), np.uint8), np.zeros((40, n_kv, 2), np.float32))
    tables, held, free, n_free = np.full((R, 12), -1), np.zeros(R, int), np.arange(40), 40
    lens, rejected = np.zeros(R, int), 0
    for tokens, accepted, logits, after, drafts, x, o in seen:
        tables, held, stack, starts, total, slots, _ = O.kv8_plan(lens, [K + 1, K + 1, K], tables, held, free, n_free, rows, 32)
        free, n_free = np.array(stack + [0] * (40 - len(stack))), len(stack)
        x, o = x.double().numpy(), o.double().numpy()
        c.append(x[:, n_q:n_q + n_kv], x[:, n_q + n_kv:], slots)
        want, size, top = O.kv8_attention(x[:, :n_q], c, tables, starts, total)
        assert (np.abs(o - want) <= _tolerance(want, size, top, D, 12 * 32, torch.bfloat16)).all()
        t, a, _ = O.verify_drafts(logits.double().numpy(), drafts.numpy(), np.zeros((R, K + 1)), None, starts, 0.0)
        np.testing.assert_array_equal(tokens.numpy(), t)
        np.testing.assert_array_equal(accepted.numpy(), a)
        lens = lens + a + 1
        rejected += int((total - lens).sum())
        np.testing.assert_array_equal(after.numpy(), lens)
    assert rejected > 0
    np.testing.assert_array_equal(s.tables.cpu().numpy(), tables)
    assert_same_cache(s.cache, c)
