"""The operators on top of the frames (layer norm, 8-bit blocks, linear attention) without a GPU: what their C calls refuse before they touch a
device, and the memory they ask for."""
from ctypes import byref, c_longlong, c_size_t

import pytest

from paper_1912_12055_amd import binding as nb

P = 4096  # stands for a pointer: every call here is refused before it is used
F32, BF16, F16 = nb.NNA_F32, nb.NNA_BF16, nb.NNA_F16
ARG, SHAPE, UNSUPPORTED = nb.NNA_ERR_INVALID_ARG, nb.NNA_ERR_SHAPE, nb.NNA_ERR_UNSUPPORTED


def norm(x=P, xt=F32, rows=3, width=8, step=8, w=P, b=P, eps=1e-5, y=P, yt=F32, stats=None, codes=None, scales=None):
    return nb.lib().nna_layer_norm(x, xt, rows, width, step, w, b, eps, y, yt, stats, codes, scales, -1, None)


def frames(x=P, B=2, width=8, T=5, eps=1e-5, y=P, yt=F32):
    return nb.lib().nna_layer_norm_frames(x, B, width, T, None, None, eps, y, yt, None, -1, None)


def back(g=P, gt=F32, x=P, xt=F32, rows=3, width=8, codes=None, scales=None, stats=P, gx=2 * P, gw=P, gb=P, ws=P, size=1 << 30):
    return nb.lib().nna_layer_norm_backward(g, gt, x, xt, rows, width, width, codes, scales, stats, None, gx, gw, gb, ws, size, -1, None)


def strides(*s):
    return (c_longlong * 3)(*s)


def attend(q=P, qs=strides(640, 64, 8), type=F32, B=1, T=10, H=8, dk=8, dv=8, decay=P, scale=1.0, out=P, ws=P, size=1 << 40):
    return nb.lib().nna_decay_attention(q, qs, P, strides(640, 64, 8), P, strides(640, 64, 8), type, B, T, H, dk, dv, decay, scale, None, None, None, out, ws, size,
                                        -1, None)


def attend_back(g=P, gk=P, gv=P, type=F32, T=10, dv=8, scale=1.0, ws=P, size=1 << 40):
    s = strides(640, 64, 8)
    return nb.lib().nna_decay_attention_backward(g, P, s, P, s, P, s, type, 1, T, 8, 8, dv, P, scale, None, None, None, None, gk, gv, None, ws, size, -1, None)


def step(q=P, state=P, type=F32, H=8, dk=8, scale=1.0):
    s = (c_longlong * 2)(64, 8)
    return nb.lib().nna_decay_attention_step(q, s, P, s, P, s, type, 1, H, dk, 8, P, scale, state, P, -1, None)


@pytest.mark.parametrize("call,status", [
    (lambda: norm(x=None), ARG), (lambda: norm(y=None), ARG), (lambda: norm(xt=9), ARG), (lambda: norm(xt=BF16), ARG), (lambda: norm(eps=-1.0), ARG),
    (lambda: norm(eps=float("nan")), ARG), (lambda: norm(rows=-1), SHAPE), (lambda: norm(width=0), SHAPE), (lambda: norm(width=16385), UNSUPPORTED),
    (lambda: norm(rows=1 << 60), SHAPE), (lambda: norm(codes=P), ARG), (lambda: norm(scales=P), ARG), (lambda: norm(yt=BF16, codes=P, scales=P), UNSUPPORTED),
    (lambda: frames(x=None), ARG), (lambda: frames(width=2113), UNSUPPORTED), (lambda: frames(T=-1), SHAPE), (lambda: frames(B=1 << 40, T=1 << 20), SHAPE),
    (lambda: back(g=None), ARG), (lambda: back(x=None), ARG), (lambda: back(stats=None), ARG), (lambda: back(ws=None), ARG), (lambda: back(size=16), ARG),
    (lambda: back(ws=P + 4), ARG), (lambda: back(gx=P), ARG), (lambda: back(gt=F16, xt=BF16), ARG), (lambda: back(width=0), SHAPE),
    (lambda: attend(q=None), ARG), (lambda: attend(out=None), ARG), (lambda: attend(qs=None), ARG), (lambda: attend(decay=None), ARG), (lambda: attend(scale=0.0), ARG),
    (lambda: attend(scale=float("inf")), ARG), (lambda: attend(type=F16), UNSUPPORTED), (lambda: attend(type=7), ARG), (lambda: attend(dk=129), UNSUPPORTED),
    (lambda: attend(dv=0), SHAPE), (lambda: attend(H=0), SHAPE), (lambda: attend(T=-1), SHAPE), (lambda: attend(B=1 << 40), SHAPE), (lambda: attend(B=1 << 19), SHAPE),
    (lambda: attend(qs=strides(0, (1 << 24) + 1, 8)), SHAPE), (lambda: attend(qs=strides(0, -8, 8)), SHAPE), (lambda: attend(T=20000, ws=None, size=0), ARG),
    (lambda: attend(T=20000, size=256), ARG), (lambda: attend(T=20000, ws=P + 16), ARG),
    (lambda: attend_back(g=None), ARG), (lambda: attend_back(gk=None), ARG), (lambda: attend_back(gv=None), ARG), (lambda: attend_back(type=F16), UNSUPPORTED),
    (lambda: attend_back(dv=300), UNSUPPORTED), (lambda: attend_back(scale=float("nan")), ARG), (lambda: attend_back(T=20000, ws=None, size=0), ARG),
    (lambda: step(q=None), ARG), (lambda: step(state=None), ARG), (lambda: step(type=F16), UNSUPPORTED), (lambda: step(H=0), SHAPE), (lambda: step(dk=200), UNSUPPORTED),
    (lambda: step(scale=0.0), ARG),
])
def test_refusals(call, status):
    assert call() == status, nb.nna_last_error()
    assert nb.nna_last_error()


@pytest.mark.parametrize("call", [norm, frames, back, attend, attend_back, step])
def test_no_device(call):
    assert call() not in (nb.NNA_OK, SHAPE, UNSUPPORTED)
    assert "device" in nb.nna_last_error()


def test_memory_of_linear_attention():
    """Both directions' states, 256-byte multiples; nothing where the sequences fill the card or are short."""
    one = nb.nna_decay_attention_workspace(1, 5000, 8, 64, 64)
    assert one and one % (8 * 64 * 64 * 4) == 0
    assert nb.nna_decay_attention_backward_workspace(1, 5000, 8, 64, 64) % (2 * 8 * 64 * 64 * 4) == 0
    for B, T in ((1, 0), (1, 1), (1, 400), (0, 5000), (64, 5000)):
        assert nb.nna_decay_attention_workspace(B, T, 8, 64, 64) == 0
        assert nb.nna_decay_attention_backward_workspace(B, T, 8, 64, 64) == 0
    n = c_size_t()
    assert nb.lib().nna_decay_attention_workspace(1, 10, 8, 64, 129, byref(n)) == UNSUPPORTED
    assert nb.lib().nna_decay_attention_workspace(1, 10, 8, 64, 64, None) == ARG
    assert nb.lib().nna_decay_attention_backward_workspace(1, 10, 8, 64, 64, None) == ARG
    assert nb.lib().nna_layer_norm_backward_workspace(10, 0, 0, 0, byref(n)) == SHAPE


def test_the_step_between_frames_is_checked_where_there_are_two():
    for s in (strides(640, 1 << 40, 8), strides(640, -8, 8)):
        assert attend(qs=s, T=2) == SHAPE
        for T in (0, 1):
            assert attend(qs=s, T=T) == ARG and "device" in nb.nna_last_error()
