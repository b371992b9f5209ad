"""The serving operators on the CPU: the oracle's rules in small cases worked out by hand, and the refusals of the C
entries and of the Python calls, which all come before any device work."""
import ctypes
import os

import numpy as np
import pytest

from oracle import pipo_oracle as O


@pytest.fixture(scope="module")
def lib():
    from paper_2605_27255_amd import pipo, build
    if not os.path.exists(pipo.LIB_PATH):
        build.build()
    return pipo.load_library()


# ---- the oracle -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("block", [32, 64, 128, 256])
@pytest.mark.parametrize("D", [64, 128])
def test_oracle_tiles_hold_every_element_once(block, D):
    for values in (False, True):
        at = O.kv8_place(block, D, values)
        assert sorted(at.ravel()) == list(range(block * D))
    # a key tile's 16 bytes are one token's dimensions; a value tile's are two dimensions of eight tokens
    assert (np.diff(O.kv8_place(block, D, False).reshape(block, D // 16, 16), axis=2) == 1).all()
    at = O.kv8_place(block, D, True)
    assert list(at[[0, 1, 2, 3, 16, 17, 18, 19], 0]) == list(range(8)) and at[0, 16] == 8 and at[4, 0] == 256


def test_oracle_append_by_hand():
    c = O.Kv8Oracle(np.full((2, 1, 1, 32, 64), 128, np.uint8), np.zeros((1, 1, 2), np.float32))
    x = np.zeros((2, 1, 64))
    x[0, 0, 0], x[1, 0, 0] = 127.0, -63.5
    c.append(x, 2 * x, [0, 1])
    assert list(c.scales[0, 0]) == [1.0, 2.0] and list(c.codes[:, 0, 0, :2, 0].ravel()) == [255, 64, 255, 64]
    x[0, 0, 0] = 254.0                  # the scale doubles: -64 becomes -32; a token beyond the others is kept as well
    c.append(x[:1], x[:1], [2])
    assert list(c.scales[0, 0]) == [2.0, 2.0] and list(c.codes[0, 0, 0, :3, 0]) == [192, 96, 255]
    np.testing.assert_array_equal(c.rows(0, [0, 1, 2, -1])[:, 0, 0], [128.0, -64.0, 254.0, 0.0])
    x[0, 0, 0] = 1.0                    # the first slot: the block begins anew
    c.append(x[:1], x[:1], [0])
    assert c.scales[0, 0, 0] == np.float32(1) / np.float32(127)


def test_oracle_plan_by_hand():
    tables, held = [[5, -1, -1], [3, 1, -1], [-1, -1, -1]], [1, 2, 0]
    t, h, stack, starts, total, slots, pos = O.kv8_plan([31, 40, 0], [2, -1, 33], tables, held, [0, 2, 4, 9], 3, 40, 32)
    # request 1 ends: 3 on top of 1; request 0 takes 3, request 2 takes 1 and 4
    assert t.tolist() == [[5, 3, -1], [-1, -1, -1], [1, 4, -1]] and list(h) == [2, 0, 2] and stack == [0, 2]
    assert starts.tolist() == [0, 2, 2, 35] and total.tolist() == [33, 0, 33]
    assert slots[:3].tolist() == [191, 96, 32] and slots[34] == 128 and (slots[35:] == -1).all()
    assert pos[:3].tolist() == [31, 32, 0] and pos[34] == 32 and (pos[35:] == -1).all()
    # no blocks for request 2, which leaves request 0 as it is
    t, h, stack, _, total, slots, _ = O.kv8_plan([31, 40, 0], [2, 0, 33], tables, held, [0], 1, 40, 32)
    assert total.tolist() == [33, 40, 0] and stack == [] and (slots[2:] == -1).all() and list(h) == [2, 2, 0]


def test_oracle_attention_is_the_softmax_of_its_tokens():
    rng = np.random.default_rng(1)
    codes = rng.integers(1, 256, (2, 3, 1, 32, 64)).astype(np.uint8)
    c = O.Kv8Oracle(codes, np.full((3, 1, 2), 0.01, np.float32))
    q = rng.standard_normal((3, 2, 64))
    out, size, top = O.kv8_attention(q, c, np.array([[2, 0]]), np.array([0, 3]), np.array([40]))
    x = (codes.astype(float) - 128) * np.float32(0.01)
    k, v = (np.concatenate([x[w, 2, 0], x[w, 0, 0]]) for w in (0, 1))
    for i in range(3):
        e = np.exp(k[:38 + i] @ q[i, 1] / 8)
        np.testing.assert_allclose(out[i, 1], e @ v[:38 + i] / e.sum(), rtol=1e-12)
    assert (np.abs(out) <= top[:, :, None]).all() and (size > 0).all()


def test_oracle_verification_by_hand():
    log = np.log
    p = log(np.array([[0.5, 0.3, 0.2], [0.1, 0.2, 0.7]]))
    q = log(np.array([[[0.25, 0.25, 0.5]]]))
    # token 2: p / q = 0.4; accepted below it, replaced above it by max(p - q, 0) = (0.25, 0.05, 0)
    t, a, m = O.verify_drafts(p, np.array([[2]]), np.array([[0.39, 0.25]]), q)
    assert t.tolist() == [[2, 1]] and a[0] == 1 and m[0] == pytest.approx(0.2 - 0.39 * 0.5)
    for u, token in ((0.8, 0), (0.85, 1)):
        t, a, _ = O.verify_drafts(p, np.array([[2]]), np.array([[0.41, u]]), q)
        assert t.tolist() == [[token, -1]] and a[0] == 0
    # not drawn: accepted below p, else from the others
    assert O.verify_drafts(p, np.array([[2]]), np.array([[0.19, 0.0]]))[0].tolist() == [[2, 0]]
    assert O.verify_drafts(p, np.array([[0]]), np.array([[0.51, 0.59]]))[0].tolist() == [[1, -1]]
    assert O.verify_drafts(p, np.array([[0]]), np.array([[0.51, 0.61]]))[0].tolist() == [[2, -1]]
    assert O.verify_drafts(p, np.array([[0]]), np.array([[0.9, 0.9]]), temperature=0.0)[0].tolist() == [[0, 2]]
    assert O.verify_drafts(p, np.array([[-1]]), np.array([[0.9, 0.9]]))[0].tolist() == [[2, -1]]


# ---- refusals -------------------------------------------------------------------------------------------------------------

A = 1 << 20            # never read: every call below is refused


def _kv8(**kw):
    from paper_2605_27255_amd import pipo
    a = dict(keys=A, values=A, scales=A, blocks=4, n_kv=2, head_dim=64, block=64)
    a.update(kw)
    return pipo.PipoKv8(*a.values())


CACHES = [dict(keys=None), dict(values=None), dict(scales=None), dict(keys=A + 8), dict(values=A + 1), dict(scales=A + 4),
          dict(blocks=0), dict(n_kv=0), dict(n_kv=257), dict(head_dim=96), dict(block=16), dict(block=48), dict(block=512),
          dict(blocks=1 << 25, block=64)]


def _call(lib, name, base, kw):
    a = dict(base)
    a.update(kw)
    if "cache" in a and a["cache"] is not None:
        a["cache"] = ctypes.byref(_kv8(**a["cache"]))
    return getattr(lib, name)(*a.values())


def test_struct_layout(tmp_path):
    import subprocess
    from paper_2605_27255_amd import pipo
    header = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "pipo.h")
    src = tmp_path / "layout.c"
    src.write_text(f'#include <stdio.h>\n#include <stddef.h>\n#include "{header}"\nint main(void) {{ printf("%zu %zu %zu\\n", '
                   "sizeof(pipo_kv8), offsetof(pipo_kv8, scales), offsetof(pipo_kv8, block)); return 0; }\n")
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "layout")], check=True)
    got = subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True).stdout.split()
    assert [int(x) for x in got] == [ctypes.sizeof(pipo.PipoKv8), pipo.PipoKv8.scales.offset, pipo.PipoKv8.block.offset]


def test_plan_refusals(lib):
    from paper_2605_27255_amd import PIPO_EINVAL
    base = dict(R=2, width=4, block=64, blocks=8, lens=A, new=A, tables=A, held=A, free=A, n_free=A, rows=5, starts=A,
                total=A, slots=A, positions=A, stream=None)
    for kw in [dict(R=0), dict(R=(1 << 20) + 1), dict(width=0), dict(width=1 << 25), dict(block=0), dict(block=16),
               dict(block=96), dict(blocks=0), dict(blocks=1 << 25), dict(rows=-1), dict(rows=(1 << 20) + 1),
               dict(width=1 << 20, block=256, blocks=1 << 24)] + [{k: v} for k in (
                   "lens", "new", "tables", "held", "free", "n_free", "starts", "total", "slots", "positions") for v in (None, A + 2)]:
        assert _call(lib, "pipo_kv8_plan", base, kw) == PIPO_EINVAL, kw


@pytest.mark.parametrize("dt", ["", "_bf16"])
def test_cache_refusals(lib, dt):
    from paper_2605_27255_amd import PIPO_EINVAL, PIPO_OK
    rows = dict(cache={}, rows=3, k=A, ldk=128, v=A, ldv=128, slots=A, stream=None)
    read = dict(cache={}, rows=3, slots=A, k=A, v=A, stream=None)
    for kw in [dict(cache=c) for c in CACHES] + [dict(cache=None), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(k=None),
                                                 dict(v=None), dict(slots=None), dict(ldk=127), dict(ldv=127), dict(k=A + 1),
                                                 dict(v=A + 1), dict(slots=A + 2), dict(ldk=1 << 40)]:
        assert _call(lib, "pipo_kv8_append" + dt, rows, kw) == PIPO_EINVAL, kw
    for kw in [dict(cache=c) for c in CACHES] + [dict(cache=None), dict(rows=-1), dict(k=None), dict(v=A + 8), dict(slots=None)]:
        assert _call(lib, "pipo_kv8_read" + dt, read, kw) == PIPO_EINVAL, kw
    assert _call(lib, "pipo_kv8_append" + dt, rows, dict(rows=0, k=None, v=None, slots=None)) == PIPO_OK
    assert _call(lib, "pipo_kv8_read" + dt, read, dict(rows=0, k=None, v=None, slots=None)) == PIPO_OK


@pytest.mark.parametrize("dt", ["", "_bf16"])
def test_attention_refusals(lib, dt):
    from paper_2605_27255_amd import PIPO_EINVAL, PIPO_OK
    base = dict(cache={}, R=2, rows=3, n_q=8, q=A, ld=512, tables=A, width=2, starts=A, total=A, max_len=128, scale=0.125,
                out=2 * A, ldo=512, work=None, bytes=0, stream=None)
    for kw in [dict(cache=c) for c in CACHES] + [
            dict(cache=None), dict(R=0), dict(rows=-1), dict(n_q=0), dict(n_q=7), dict(n_q=34), dict(q=None), dict(q=A + 1),
            dict(ld=511), dict(ldo=511), dict(tables=None), dict(width=0), dict(starts=None), dict(total=None), dict(max_len=0),
            dict(max_len=129), dict(out=A + 64), dict(out=A, ldo=513), dict(scale=float("nan")), dict(scale=1e300),
            dict(out=None), dict(rows=(1 << 20) + 1)]:
        assert _call(lib, "pipo_kv8_attention" + dt, base, kw) == PIPO_EINVAL, kw
    long = dict(width=200, max_len=200 * 64)
    need = lib.pipo_kv8_attention_work_bytes(ctypes.byref(_kv8()), 2, 3, 8, 200 * 64, dt != "")
    assert need > 0
    for kw in (dict(work=A, bytes=need - 1), dict(work=A + 8, bytes=need)):
        assert _call(lib, "pipo_kv8_attention" + dt, base, {**long, **kw}) == PIPO_EINVAL, kw
    assert _call(lib, "pipo_kv8_attention" + dt, base, dict(rows=0, q=None, out=None)) == PIPO_OK
    assert lib.pipo_kv8_attention_work_bytes(ctypes.byref(_kv8(block=16)), 2, 3, 8, 200, 0) == 0


@pytest.mark.parametrize("dt", ["", "_bf16"])
def test_verify_refusals(lib, dt):
    from paper_2605_27255_amd import PIPO_EINVAL, PIPO_OK
    need = lib.pipo_verify_work_bytes(2, 3, 50)
    assert lib.pipo_verify_work_bytes(65535, 63, 1 << 19) == 0     # more workgroups than a launch has
    assert need > 0 and lib.pipo_verify_work_bytes(2, 64, 50) == 0 and lib.pipo_verify_work_bytes(-1, 3, 50) == 0
    base = dict(R=2, K=3, V=50, rows=8, z=A, ld=50, starts=None, drafts=A, d=A, lr=150, ln=50, u=A, t=1.0, tokens=A, accepted=A,
                work=A, bytes=need, stream=None)
    for kw in [dict(R=-1), dict(R=65536), dict(K=-1), dict(K=64), dict(V=0), dict(V=(1 << 19) + 1), dict(rows=7), dict(rows=-1),
               dict(z=None), dict(z=A + 1), dict(ld=49), dict(starts=A + 2), dict(drafts=None), dict(d=A + 1), dict(lr=49),
               dict(ln=49), dict(lr=-150), dict(u=None), dict(t=float("nan")), dict(t=1e6), dict(t=1e-9), dict(tokens=None),
               dict(accepted=None), dict(work=None), dict(work=A + 8), dict(bytes=need - 1)]:
        assert _call(lib, "pipo_verify_drafts" + dt, base, kw) == PIPO_EINVAL, kw
    assert _call(lib, "pipo_verify_drafts" + dt, base, dict(R=0, rows=0, z=None, drafts=None, u=None, tokens=None, accepted=None,
                                                            work=None, bytes=0)) == PIPO_OK


def test_python_calls_refuse_host_tensors(lib):
    import torch
    from paper_2605_27255_amd import Kv8Cache, PipoError, kv8_append, kv8_attention, kv8_plan, kv8_read, verify_drafts
    i, z = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 8)
    for call in (lambda: Kv8Cache.new(4, 2, 64, device="cpu"), lambda: Kv8Cache.new(4, 2, 64, block=16),
                 lambda: Kv8Cache.new(4, 2, 80), lambda: Kv8Cache(z, z, z), lambda: kv8_append(None, z, z, i),
                 lambda: kv8_read(z, i), lambda: kv8_attention(z, None, i, i, i), lambda: verify_drafts(z, i[:, None], z),
                 lambda: kv8_plan(i, i, i[:, None], i, i, i, 4, 64)):
        with pytest.raises(PipoError):
            call()


def test_oracle_append_runs_go_over_rows_without_a_slot():
    x = np.zeros((4, 1, 64))
    x[:, 0, 0] = 127.0, 1e6, 254.0, 508.0
    a, b = (O.Kv8Oracle(np.full((2, 3, 1, 32, 64), 128, np.uint8), np.ones((3, 1, 2), np.float32)) for _ in "ab")
    a.append(x, x, [33, -1, 34, 35])
    b.append(x[[0, 2, 3]], x[[0, 2, 3]], [33, 34, 35])
    np.testing.assert_array_equal(a.codes, b.codes)
    np.testing.assert_array_equal(a.scales, b.scales)
    assert a.scales[1, 0, 0] == 4.0 and list(a.codes[0, 1, 0, 1:4, 0]) == [160, 192, 255]       # 31.75 to the nearest
