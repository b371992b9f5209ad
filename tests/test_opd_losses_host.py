"""OPD losses on the CPU: the oracle's formulas against differences and closed
forms, and the refusals of the C entries and of the Python calls, which all
come before any device work."""
import ctypes
import os

import numpy as np
import pytest

from oracle import pipo_oracle as O

KINDS = ("forward", "reverse", "jsd")


def _lists(T, V, k, seed, temperature=1.0):
    rng = np.random.default_rng(seed)
    z = 2.0 * rng.standard_normal((T, V))
    t = z + 0.7 * rng.standard_normal((T, V))
    return z, O.opd_top_logits(t, k, temperature)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("with_tail", [True, False])
@pytest.mark.parametrize("temperature", [1.0, 1.7])
def test_oracle_distill_gradient_is_the_difference_quotient(kind, with_tail, temperature):
    T, V, k = 3, 23, 6
    z, (ids, logp, tail) = _lists(T, V, k, seed=3, temperature=temperature)
    ids[1, 2] = -1                      # an empty slot
    scale = np.array([0.5, 2.0, -1.0])
    kw = dict(tail=tail if with_tail else None, kind=kind, beta=0.3, temperature=temperature)
    _, grad, _ = O.opd_distill(z, ids, logp, scale=scale, **kw)
    h = 1e-5                            # truncation h^2 ~ 1e-10, rounding 1e-16 / h ~ 1e-11 per unit of loss
    for v in range(V):
        d = np.zeros((T, V))
        d[:, v] = h
        up, down = (O.opd_distill(z + s * d, ids, logp, **kw)[0] for s in (1, -1))
        np.testing.assert_allclose(grad[:, v], scale * (up - down) / (2 * h), atol=1e-8)


def test_oracle_policy_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(4)
    T, V = 6, 11
    z = rng.standard_normal((T, V))
    y = rng.integers(0, V, T)
    y[5] = -1
    lp = O.opd_policy(z, y, np.ones(T), temperature=0.8)[1]
    old = lp - np.array([0.05, 0.5, -0.5, 0.5, -0.5, 0.0])     # inside; above and below the clip for either sign
    adv = np.array([1.0, 1.5, 1.5, -0.5, -0.5, 1.0])
    kw = dict(old_logp=old, ref_logp=lp + 0.3, clip=(0.2, 0.3), kl_coef=0.1, temperature=0.8)
    loss, _, kl, grad, _ = O.opd_policy(z, y, adv, scale=np.full(T, 2.0), **kw)
    assert kl[:5] == pytest.approx(np.exp(0.3) - 1.3) and loss[5] == 0 and not grad[5].any()
    for v in range(V):
        d = np.zeros((T, V))
        d[:, v] = 1e-5
        up, down = (O.opd_policy(z + s * d, y, adv, **kw)[0] for s in (1, -1))
        np.testing.assert_allclose(grad[:, v], 2.0 * (up - down) / 2e-5, atol=1e-8)
    # clipped where the ratio has moved the way the advantage wants: only the KL term is left
    only_kl = O.opd_policy(z, y, 0 * adv, scale=np.full(T, 2.0), **kw)[3]
    for t, clipped in enumerate((False, True, False, False, True)):
        assert np.allclose(grad[t], only_kl[t], atol=1e-12) == clipped, t


def test_oracle_distill_closed_forms():
    T, V = 4, 17
    z, (ids, logp, tail) = _lists(T, V, V, seed=5)          # the whole vocabulary listed
    ls = np.stack([O._log_softmax_row(r, 1.0) for r in z])
    lq = np.zeros((T, V))
    np.put_along_axis(lq, ids, logp, 1)
    assert np.all(np.isneginf(tail))
    np.testing.assert_allclose(O.opd_distill(z, ids, logp, kind="forward")[0], np.sum(np.exp(lq) * (lq - ls), 1))
    np.testing.assert_allclose(O.opd_distill(z, ids, logp, tail, kind="reverse")[0], np.sum(np.exp(ls) * (ls - lq), 1))
    np.testing.assert_allclose(O.opd_distill(z, ids, logp, kind="forward")[1], np.exp(ls) - np.exp(lq), atol=1e-14)
    # a student equal to its teacher: no divergence and no gradient, whatever is listed
    ids, logp, tail = O.opd_top_logits(z, 5)
    for kind in KINDS:
        loss, grad, _ = O.opd_distill(z, ids, logp, tail, kind=kind)
        assert np.abs(loss).max() < 1e-14 and np.abs(grad).max() < 1e-14
    # a gradient in the logits sums to zero over the row when every token is in some entry
    z2 = z + np.random.default_rng(6).standard_normal(z.shape)
    for kind in KINDS:
        assert np.abs(O.opd_distill(z2, ids, logp, tail, kind=kind)[1].sum(1)).max() < 1e-14


def test_oracle_top_logits_orders_ties_by_id():
    z = np.array([[1.0, 3.0, -0.0, 3.0, 0.0, -np.inf]])
    ids, logp, tail = O.opd_top_logits(z, 5)
    assert ids.tolist() == [[1, 3, 0, 2, 4]] and np.isneginf(tail[0])
    assert np.exp(logp).sum() == pytest.approx(1.0)


@pytest.fixture(scope="module")
def lib():
    from paper_2605_27255_amd import pipo, build
    if not os.path.exists(pipo.LIB_PATH):
        build.build()
    return pipo.load_library()


A, B = ctypes.c_void_p(1 << 20), ctypes.c_void_p(1 << 24)      # never read: every call below is refused
NAN = float("nan")


def _top(lib, dt, **kw):
    a = dict(T=4, V=8, z=A, ld=8, temperature=1.0, k=2, ids=B, logp=B, tail=None, work=None, nw=0, stream=None)
    a.update(kw)
    return getattr(lib, "pipo_opd_top_logits" + dt)(*a.values())


def _distill(lib, dt, **kw):
    a = dict(T=4, V=8, z=A, ld=8, Tt=4, k=2, ids=B, logp=B, tail=None, rows=None, labels=None, kind=0, beta=0.5,
             temperature=1.0, scale=None, loss=B, grad=None, ldg=0, work=None, nw=0, stream=None)
    a.update(kw)
    return getattr(lib, "pipo_opd_distill" + dt)(*a.values())


def _policy(lib, dt, **kw):
    a = dict(T=4, V=8, z=A, ld=8, labels=B, adv=B, old=None, ref=None, lo=0.2, hi=0.2, kl_coef=0.0, temperature=1.0,
             scale=None, loss=B, logp=None, kl=None, grad=None, ldg=0, work=None, nw=0, stream=None)
    a.update(kw)
    return getattr(lib, "pipo_opd_policy" + dt)(*a.values())


ROWS = [dict(T=-1), dict(T=1 << 22), dict(V=0), dict(V=(1 << 19) + 1), dict(ld=7), dict(ld=1 << 40), dict(z=None), dict(z=ctypes.c_void_p((1 << 20) + 1)),
        dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=NAN), dict(temperature=float("inf")),
        dict(temperature=1e-200)]
LOSS = ROWS + [dict(loss=None), dict(grad=ctypes.c_void_p((1 << 21) + 1), ldg=8), dict(grad=ctypes.c_void_p(1 << 21), ldg=7),
               dict(grad=ctypes.c_void_p((1 << 20) + 16), ldg=8), dict(grad=A, ldg=9),
               dict(ld=14, grad=ctypes.c_void_p((1 << 20) + 4 * 7), ldg=14)]


@pytest.mark.parametrize("dt", ["", "_bf16"])
def test_bad_arguments_are_refused_before_device_work(lib, dt):
    from paper_2605_27255_amd import PIPO_EINVAL
    for kw in ROWS + [dict(k=0), dict(k=9), dict(V=1000, ld=1000, k=257), dict(ids=None), dict(logp=None)]:
        assert _top(lib, dt, **kw) == PIPO_EINVAL, kw
    for kw in LOSS + [dict(Tt=0), dict(k=0), dict(k=257), dict(ids=None), dict(logp=None), dict(kind=-1), dict(kind=3),
                      dict(kind=2, beta=0.0), dict(kind=2, beta=1.0), dict(kind=2, beta=NAN)]:
        assert _distill(lib, dt, **kw) == PIPO_EINVAL, kw
    for kw in LOSS + [dict(labels=None), dict(adv=None), dict(lo=-0.1), dict(lo=1.1), dict(lo=NAN), dict(hi=-0.1),
                      dict(hi=float("inf")), dict(kl_coef=0.1), dict(kl=B), dict(ref=B, kl_coef=NAN)]:
        assert _policy(lib, dt, **kw) == PIPO_EINVAL, kw


def test_work_arrays_are_checked(lib):
    """Calls that use a work array say how large; a smaller or misaligned one is refused."""
    from paper_2605_27255_amd import PIPO_EINVAL
    long = dict(T=4, V=151936, ld=151936)
    for bf16, dt in enumerate(("", "_bf16")):
        for call, fn, extra in ((0, _top, {}), (1, _distill, {}), (2, _distill, dict(grad=ctypes.c_void_p(1 << 30), ldg=151936)),
                                (2, _policy, dict(grad=ctypes.c_void_p(1 << 30), ldg=151936))):
            need = lib.pipo_opd_work_bytes(call, 4, 151936, 1 if fn is _policy else 2, bf16)
            if need == 0:
                continue
            assert fn(lib, dt, work=B, nw=need - 1, **long, **extra) == PIPO_EINVAL
            assert fn(lib, dt, work=ctypes.c_void_p((1 << 24) + 8), nw=need, **long, **extra) == PIPO_EINVAL
        assert lib.pipo_opd_work_bytes(0, 4, 151936, 2, bf16) > 0 and lib.pipo_opd_work_bytes(2, 4, 151936, 2, bf16) > 0
    for bad in ((0, 0, 100, 1, 0), (0, 4, 0, 1, 0), (0, 4, (1 << 19) + 1, 1, 0), (0, 4, 100, 0, 0), (2, 4, 100, 257, 0)):
        assert lib.pipo_opd_work_bytes(*bad) == 0


def test_empty_calls_need_no_arrays(lib):
    from paper_2605_27255_amd import PIPO_OK
    for dt in ("", "_bf16"):
        assert _top(lib, dt, T=0, z=None, ids=None, logp=None) == PIPO_OK
        assert _distill(lib, dt, T=0, z=None, ids=None, logp=None, loss=None) == PIPO_OK
        assert _policy(lib, dt, T=0, z=None, labels=None, adv=None, loss=None) == PIPO_OK


def test_python_calls_refuse_host_tensors(lib):
    import torch
    from paper_2605_27255_amd import PipoError, opd_distill, opd_policy, opd_top_logits
    z = torch.zeros(2, 8)
    i, f = torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    for call in (lambda: opd_top_logits(z, 2), lambda: opd_distill(z, i[:, None], f[:, None]),
                 lambda: opd_policy(z, i, f)):
        with pytest.raises(PipoError):
            call()


def test_empty_calls_with_empty_lists(lib):
    """No positions and no teacher rows: a chunk of nothing but prompt."""
    from paper_2605_27255_amd import PIPO_EINVAL, PIPO_OK
    for dt in ("", "_bf16"):
        nothing = dict(T=0, z=None, ids=None, logp=None, loss=None)
        assert _distill(lib, dt, Tt=0, **nothing) == PIPO_OK
        assert _distill(lib, dt, Tt=-1, **nothing) == PIPO_EINVAL
        assert _distill(lib, dt, Tt=0, k=0, **nothing) == PIPO_EINVAL
        assert _distill(lib, dt, Tt=0) == PIPO_EINVAL


def test_build_reads_the_compilers_report_of_spills():
    from paper_2605_27255_amd import build
    report = ("a.hip:1:1: remark:     ScratchSize [bytes/lane]: 0 [-Rpass-analysis=kernel-resource-usage]\n"
              "a.hip:9:1: remark:     ScratchSize [bytes/lane]: 188 [-Rpass-analysis=kernel-resource-usage]\n")
    assert build.spilled(report) == 188 > build.SPILL_LIMIT and build.spilled("") == 0
