"""Heads normalised and rotated, the gated recurrence and the optimiser's step without a GPU: what their C calls refuse before they touch a device, and the memory they ask for."""
from ctypes import byref, c_longlong, c_size_t

import numpy as np
import pytest

from paper_1912_12055_amd import binding as nb

P = 1 << 12  # stands for a pointer: every call here is refused before it is used
Q, R, S = 2 * P, 3 * P, 4 * P
F32, BF16, F16 = nb.NNA_F32, nb.NNA_BF16, nb.NNA_F16
ARG, SHAPE, UNSUPPORTED = nb.NNA_ERR_INVALID_ARG, nb.NNA_ERR_SHAPE, nb.NNA_ERR_UNSUPPORTED
THREE, TWO = (c_longlong * 3)(640, 64, 8), (c_longlong * 2)(640, 64)


def rotate(q=P, qs=THREE, heads=8, k=Q, ks=THREE, kheads=8, type=F32, B=1, T=10, width=8, freqs=P, pairs=4, at=None, steps=None, offset=0, norm=1, eps=1e-6, w=None,
           yq=R, yk=S):
    return nb.lib().nna_rotate_heads(q, qs, heads, k, ks, kheads, type, B, T, width, freqs, pairs, 0, at, steps, offset, norm, eps, w, None, yq, yk, -1, None)


def rotate_back(g=P, gk=Q, q=P, qs=THREE, k=Q, kheads=8, type=F32, width=8, norm=1, w=None, hq=R, hk=S, gw=R, ws=P, size=1 << 30):
    return nb.lib().nna_rotate_heads_backward(g, gk, q, qs, 8, k, qs, kheads, type, 1, 10, width, P, 4, 0, None, None, 0, norm, 1e-6, w, None, hq, hk, gw, None, ws, size, -1, None)


def scan(x=P, xs=TWO, f=Q, fs=TWO, i=None, is_=None, type=F32, B=1, T=10, C=64, out=R):
    return nb.lib().nna_gated_scan(x, xs, f, fs, i, is_, type, B, T, C, None, None, None, out, None, P << 20, 1 << 40, -1, None)


def scan_back(g=S, kept=S, x=P, f=Q, i=None, type=F32, C=64, gx=R, gf=5 * P, gi=None):
    return nb.lib().nna_gated_scan_backward(g, kept, x, TWO, f, TWO, i, TWO if i else None, type, 1, 10, C, None, None, gx, gf, gi, None, P << 20, 1 << 40, -1, None)


def step(x=P, f=Q, state=S, out=R, type=F32, B=1, C=64):
    return nb.lib().nna_gated_scan_step(x, 64, f, 64, None, 0, type, B, C, state, out, -1, None)


def adamw(rows=((P, Q, 100, F32),), m=R, v=S, ms=None, vs=None, master=None, size=1 << 20, t=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, count=None):
    p, g, n, types = (np.array([r[k] for r in rows], dtype) for k, dtype in enumerate((np.uint64, np.uint64, np.int64, np.int32)))
    return nb.lib().nna_adamw(*(a.ctypes.data if len(rows) else None for a in (p, g, n, types)), len(rows) if count is None else count, m, v, ms, vs, master, size, t, None, lr, None, b1,
                              b2, eps, wd, -1, None)


def moment(c=P, s=Q, n=256, out=R):
    return nb.lib().nna_adamw_moment(c, 0, s, n, out, -1, None)


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("call,status", [
    (lambda: rotate(q=None), ARG), (lambda: rotate(yq=None), ARG), (lambda: rotate(k=None), ARG), (lambda: rotate(yk=None), ARG), (lambda: rotate(qs=None), ARG),
    (lambda: rotate(ks=None), ARG), (lambda: rotate(type=5), ARG), (lambda: rotate(heads=0), SHAPE), (lambda: rotate(kheads=-1), SHAPE), (lambda: rotate(B=-1), SHAPE),
    (lambda: rotate(T=-1), SHAPE), (lambda: rotate(width=0), SHAPE), (lambda: rotate(width=257), UNSUPPORTED), (lambda: rotate(pairs=5), SHAPE), (lambda: rotate(pairs=-1), SHAPE),
    (lambda: rotate(freqs=None), ARG), (lambda: rotate(at=P), ARG), (lambda: rotate(offset=1 << 53), ARG), (lambda: rotate(eps=-1.0), ARG), (lambda: rotate(eps=NAN), ARG),
    (lambda: rotate(norm=0, w=P), ARG), (lambda: rotate(yk=R), ARG), (lambda: rotate(heads=1 << 17), SHAPE), (lambda: rotate(B=1 << 30, T=1 << 30), SHAPE),
    (lambda: rotate_back(g=None), ARG), (lambda: rotate_back(gk=None), ARG), (lambda: rotate_back(q=None), ARG), (lambda: rotate_back(hq=None), ARG),
    (lambda: rotate_back(hk=None), ARG), (lambda: rotate_back(qs=None), ARG), (lambda: rotate_back(ws=None), ARG), (lambda: rotate_back(ws=P + 4), ARG),
    (lambda: rotate_back(size=8), ARG), (lambda: rotate_back(norm=0), ARG), (lambda: rotate_back(norm=0, gw=None, w=P), ARG), (lambda: rotate_back(hk=R), ARG),
    (lambda: rotate_back(width=300), UNSUPPORTED), (lambda: rotate_back(type=-1), ARG),
    (lambda: scan(x=None), ARG), (lambda: scan(f=None), ARG), (lambda: scan(out=None), ARG), (lambda: scan(xs=None), ARG), (lambda: scan(fs=None), ARG),
    (lambda: scan(i=P, is_=None), ARG), (lambda: scan(type=3), ARG), (lambda: scan(C=0), SHAPE), (lambda: scan(T=-1), SHAPE), (lambda: scan(B=-1), SHAPE),
    (lambda: scan(B=1 << 40), SHAPE), (lambda: scan(C=1 << 29), SHAPE), (lambda: scan(B=(1 << 21) + 1), SHAPE), (lambda: scan(B=1 << 20, C=192), SHAPE), (lambda: scan(T=1 << 31), SHAPE),
    (lambda: scan_back(g=None), ARG), (lambda: scan_back(kept=None), ARG), (lambda: scan_back(x=None), ARG), (lambda: scan_back(gx=None), ARG), (lambda: scan_back(gf=None), ARG),
    (lambda: scan_back(gi=P), ARG), (lambda: scan_back(i=P), ARG), (lambda: scan_back(C=0), SHAPE),
    (lambda: step(x=None), ARG), (lambda: step(state=None), ARG), (lambda: step(out=None), ARG), (lambda: step(C=0), SHAPE), (lambda: step(type=4), ARG),
    (lambda: adamw(t=0), ARG), (lambda: adamw(b1=1.0), ARG), (lambda: adamw(b2=-0.1), ARG), (lambda: adamw(eps=NAN), ARG), (lambda: adamw(eps=INF), ARG), (lambda: adamw(lr=NAN), ARG),
    (lambda: adamw(wd=INF), ARG), (lambda: adamw(m=None), ARG), (lambda: adamw(v=None), ARG), (lambda: adamw(m=S), ARG), (lambda: adamw(ms=P), ARG), (lambda: adamw(vs=P), ARG),
    (lambda: adamw(ms=5 * P, vs=5 * P), ARG), (lambda: adamw(master=R), ARG), (lambda: adamw(ms=5 * P, vs=6 * P, master=6 * P), ARG),
    (lambda: adamw(rows=(), count=1), ARG), (lambda: adamw(count=-1), ARG), (lambda: adamw(size=100), ARG), (lambda: adamw(size=-1), ARG),
    (lambda: adamw(rows=[(0, Q, 100, F32)]), ARG), (lambda: adamw(rows=[(P, P, 100, F32)]), ARG), (lambda: adamw(rows=[(P, Q, -1, F32)]), SHAPE),
    (lambda: adamw(rows=[(P, Q, 1 << 40, F32)]), SHAPE), (lambda: adamw(rows=[(P, Q, 100, 9)]), ARG), (lambda: adamw(rows=[(P, Q, 129, F32), (R, S, 5, F32)], size=256), ARG),
    (lambda: adamw(rows=[(P, 0, 129, F32), (R, S, 5, F32)], size=256), ARG),
    (lambda: adamw(rows=[(P, Q, 100, F32), (P + 396, S, 5, F32)]), ARG), (lambda: adamw(rows=[(P + 200, Q, 100, F32), (P, S, 101, BF16)]), ARG),
    (lambda: moment(c=None), ARG), (lambda: moment(s=None), ARG), (lambda: moment(out=None), ARG), (lambda: moment(n=100), SHAPE), (lambda: moment(n=-128), SHAPE),
])
def test_refusals(call, status):
    assert call() == status, nb.nna_last_error()
    assert nb.nna_last_error() and "HIP device" not in nb.nna_last_error()  # (nor for the device, which comes last)


@pytest.mark.parametrize("call", [rotate, rotate_back, scan, scan_back, step, adamw, moment, lambda: rotate(k=None, ks=None, kheads=0, yk=None), lambda: rotate(B=0, q=None),
                                  lambda: adamw(rows=[(P, Q, 100, F32), (P + 400, S, 5, F32)]), lambda: adamw(rows=[(P + 202, Q, 100, F32), (P, S, 101, BF16)]),
                                  lambda: adamw(ms=5 * P, vs=6 * P, master=7 * P), lambda: adamw(rows=()), lambda: adamw(rows=[(0, 0, 100, F32), (P, S, 5, F32)], size=256), lambda: adamw(rows=[(P, 0, 100, F32), (P, S, 5, F32)])])
def test_no_device(call):
    """Arguments that would do get as far as the device."""
    assert call() == ARG and "device" in nb.nna_last_error()


def test_memory():
    n = c_size_t()
    assert nb.nna_rotate_heads_backward_workspace(2, 50, 64) == 100 * 2 * 64 * 4
    assert nb.nna_rotate_heads_backward_workspace(20, 5000, 64) == 512 * 2 * 64 * 4
    assert nb.nna_rotate_heads_backward_workspace(0, 0, 64) == 2 * 64 * 4
    assert nb.lib().nna_rotate_heads_backward_workspace(1, 1, 300, byref(n)) == UNSUPPORTED
    assert nb.lib().nna_rotate_heads_backward_workspace(1, 1, 64, None) == ARG
    assert nb.lib().nna_gated_scan_workspace(1, 1, 0, byref(n)) == SHAPE
    assert nb.lib().nna_gated_scan_workspace(1, 1, 8, None) == ARG
    for B, T, C in ((0, 5000, 64), (1, 0, 64), (1, 1, 1), (1, 64, 512), (64, 5000, 512)):
        assert nb.nna_gated_scan_workspace(B, T, C) == 0
    assert nb.nna_gated_scan_workspace(2, 5000, 64) >= 2 * 2 * 2 * 64 * 4


def test_where_states_begin():
    at, size = nb.nna_adamw_places([1, 128, 129, 0, 5])
    assert at.tolist() == [0, 128, 256, 512, 512] and size == 640
    assert nb.nna_adamw_places([])[1] == 0


def test_frequencies():
    f = nb.nna_rotary_freqs(8, base=100.0, scale=4.0, device=None)
    assert f.tolist() == pytest.approx([1 / 4, 100 ** -0.25 / 4, 100 ** -0.5 / 4, 100 ** -0.75 / 4], rel=1e-15)
    assert nb.nna_rotary_freqs(0, device=None).numel() == 0
    for bad in (dict(width=7), dict(width=8, base=0.0), dict(width=8, scale=NAN), dict(width=8, scale=-1.0)):
        with pytest.raises(ValueError):
            nb.nna_rotary_freqs(**bad, device=None)
