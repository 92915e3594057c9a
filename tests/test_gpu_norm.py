"""Layer norm of rows and frames and values kept in 8 bits, forward and backward, against plain implementations in 64 bits.

Tolerances.  A float32 sum over a row, taken in lanes of at most 16 values and a tree of at most ten joins, is off by at most 26 * 2^-24 of the
sum of magnitudes, and each elementary step by 2^-24 of its result; the mean's error and the rounding of x - mean count against the magnitudes
|x| + |mean|, which r carries into h.  An output is off by at most 64 * 2^-24 of the magnitudes that enter it, and half a unit of its
type.  A weight gradient is a sum over the rows of a workgroup and then over the workgroups: at most rows / groups + 64 + 26 terms deep.
"""
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0**-24
HALF = {torch.float32: 2.0**-24, torch.bfloat16: 2.0**-8, torch.float16: 2.0**-11}  # half a unit in the last place of 24, 8 and 11 bits, against the value
EPS = 1e-5


@pytest.fixture(scope="module")
def nb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import binding
    binding.lib()
    return binding


def _say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _inputs(shape, dtype, seed=0):
    g = _gen(seed)
    x = torch.randn(shape, device=DEV, generator=g) * 2 + 3 * torch.randn((*shape[:-1], 1), device=DEV, generator=g)
    w, b = 1 + 0.3 * torch.randn(shape[-1], device=DEV, generator=g), torch.randn(shape[-1], device=DEV, generator=g)
    return x.to(dtype), w, b, torch.randn(shape, device=DEV, generator=g)


def _exact(x, w, b, gout=None, stats_of=None):
    """y, and the gradients of sum(gout y), in 64 bits; `stats_of`: the values the mean and r are of, where x only stands for them"""
    x = x.double()
    s = x if stats_of is None else stats_of.double()
    m = s.mean(-1, keepdim=True)
    r = 1 / (((s - m) ** 2).mean(-1, keepdim=True) + EPS).sqrt()
    h = (x - m) * r
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else w.double()
    y = h * w + (0 if b is None else b.double())
    if gout is None:
        return y, m, r, h
    g = gout.double()
    gh = g * w
    gx = r * (gh - gh.mean(-1, keepdim=True) - h * (gh * h).mean(-1, keepdim=True))
    rows = tuple(range(x.dim() - 1))
    return gx, (g * h).sum(rows), g.sum(rows), m, r, h, gh


def _close(got, ref, bound, what):
    assert got.shape == ref.shape, what
    d = (got.double() - ref).abs()
    assert torch.isfinite(got).all(), what
    worst = float((d / bound).max()) if d.numel() else 0.0
    assert worst <= 1, (what, worst)


def _check_y(y, x, w, b):
    ref, m, r, h = _exact(x, w, b)
    aw = 1 if w is None else w.double().abs()
    most = x.double().abs().amax(-1, keepdim=True)
    bound = HALF[y.dtype] * ref.abs() + 64 * U32 * (aw * ((most + m.abs()) * r + h.abs()) + ref.abs()) + 1e-30 + (2.0**-25 if y.dtype == torch.float16 else 0)
    _close(y, ref, bound, "y")


def _check_grads(gx, gw, gb, x, w, gout, stats_of=None):
    rgx, rgw, rgb, m, r, h, gh = _exact(x, w, None, gout, stats_of)
    most = (x if stats_of is None else stats_of).double().abs().amax(-1, keepdim=True)
    eh = 64 * U32 * ((most + m.abs()) * r + h.abs())  # of h
    ah = h.abs()
    eg = (gh.abs().mean(-1, keepdim=True) + (ah + eh) * (gh.abs() * (ah + 2 * eh)).mean(-1, keepdim=True) + gh.abs()) * r
    e2 = r * (eh * (gh * h).abs().mean(-1, keepdim=True) + ah * (gh.abs() * eh).mean(-1, keepdim=True))
    bound = HALF[gx.dtype] * rgx.abs() + 64 * U32 * eg + e2 + 1e-30 + (2.0**-25 if gx.dtype == torch.float16 else 0)
    _close(gx, rgx, bound, "gx")
    rows = tuple(range(x.dim() - 1))
    depth = x[..., 0].numel() / 64 + 64 + 26
    a = gout.double().abs()
    _close(gw, rgw, (a * eh).sum(rows) + depth * U32 * (a * ah).sum(rows) + 1e-30, "gw")
    _close(gb, rgb, depth * U32 * a.sum(rows) + 1e-30, "gb")


TYPES = [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.float32, torch.bfloat16),
         (torch.float32, torch.float16)]
WIDTHS = [1, 2, 7, 8, 9, 64, 127, 128, 129, 250, 256, 257, 512, 513, 1000, 1024, 1025, 2048, 2051, 4096, 4100, 8192, 8193, 16384]


@pytest.mark.parametrize("width", WIDTHS)
def test_rows_of_every_width_and_type(nb, width):
    for k, (tx, ty) in enumerate(TYPES):
        for rows in (1, 5, 67):
            _say("norm", width, tx, ty, rows)
            x, w, b, g = _inputs((rows, width), tx, seed=width + k)
            g = g.to(ty)
            y, kept = nb.nna_layer_norm(x, w, b, eps=EPS, out_dtype=ty, keep=32)
            assert y.dtype == ty and torch.equal(y, nb.nna_layer_norm(x, w, b, eps=EPS, out_dtype=ty))
            _check_y(y, x, w, b)
            gx, gw, gb = nb.nna_layer_norm_backward(g, kept, w)
            assert gx.dtype == tx
            _check_grads(gx, gw, gb, x, w, g)


@pytest.mark.parametrize("rows,width", [(5000, 128), (70001, 9), (3000, 512), (9001, 1024), (4099, 2048)])
def test_more_rows_than_the_launch_has_workgroups(nb, rows, width):
    _say("many rows", rows, width)
    x, w, b, g = _inputs((rows, width), torch.float32, seed=3)
    y, kept = nb.nna_layer_norm(x, w, b, eps=EPS, keep=32)
    _check_y(y, x, w, b)
    grads = nb.nna_layer_norm_backward(g, kept, w)
    _check_grads(*grads, x, w, g)
    for a, c in zip(grads, nb.nna_layer_norm_backward(g, kept, w)):
        assert torch.equal(a, c)  # no order that changes from call to call
    only_x = nb.nna_layer_norm_backward(g, kept, w, want_gw=False)
    only_w = nb.nna_layer_norm_backward(g, kept, w, want_gx=False)
    assert only_x[1] is None and only_w[0] is None and torch.equal(only_x[0], grads[0]) and torch.equal(only_w[1], grads[1]) and torch.equal(only_w[2], grads[2])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_row_strides_and_starts(nb, dtype):
    big = _inputs((3, 11, 700), dtype)[0]
    w, b = _inputs((1, 301), dtype)[1:3]
    for x in (big[:, :, 1:302], big[1, 2:9, 399:700], big[:, 3:4, 7:308], big[2, 4, 5:306].expand(6, 301)):
        _say("strides", tuple(x.shape), x.stride(), x.storage_offset())
        y, kept = nb.nna_layer_norm(x, w, b, eps=EPS, keep=32)
        _check_y(y, x, w, b)
        g = _inputs(tuple(x.shape), dtype, seed=9)[3].to(dtype)
        _check_grads(*nb.nna_layer_norm_backward(g, kept, w), x, w, g)


@pytest.mark.parametrize("shape", [(2, 1, 5), (3, 40, 1), (1, 128, 216), (2, 129, 31), (3, 84, 33), (2, 257, 64), (1, 513, 50), (2, 558, 35),
                                   (1, 559, 17), (2, 1025, 43), (1, 1088, 16), (1, 1089, 9), (1, 2049, 23), (2, 2112, 8), (40, 128, 900)])
def test_frames(nb, shape):
    for ty in (torch.float32, torch.bfloat16, torch.float16):
        _say("frames", shape, ty)
        rows, w, b, g = _inputs((shape[0], shape[2], shape[1]), torch.float32, seed=shape[1])
        spec = rows.transpose(1, 2).contiguous()
        x = spec.transpose(1, 2)
        g = g.to(ty)
        y, kept = nb.nna_layer_norm(x, w, b, eps=EPS, out_dtype=ty, keep=32)
        assert y.is_contiguous() and torch.equal(y, nb.nna_layer_norm(x, w, b, eps=EPS, out_dtype=ty))
        _check_y(y, x, w, b)
        gx, gw, gb = nb.nna_layer_norm_backward(g, kept, w)
        if min(shape[1:]) > 1:
            assert gx.transpose(1, 2).is_contiguous()
        _check_grads(gx, gw, gb, x, w, g)
        for a, c in zip((gx, gw, gb), nb.nna_layer_norm_backward(g, kept, w)):
            assert torch.equal(a, c)


def test_without_weights_and_without_rows(nb):
    x, w, b, g = _inputs((4, 96), torch.float32)
    y, kept = nb.nna_layer_norm(x, eps=EPS, keep=32)
    _check_y(y, x, None, None)
    _check_grads(*nb.nna_layer_norm_backward(g, kept), x, None, g)
    for shape in ((0, 96), (3, 0, 96)):
        y, kept = nb.nna_layer_norm(torch.empty(shape, device=DEV), w, b, keep=8)
        gx, gw, gb = nb.nna_layer_norm_backward(torch.empty(shape, device=DEV), kept, w)
        assert y.shape == gx.shape == shape and not gw.any() and not gb.any()
    frames = torch.empty((2, 96, 0), device=DEV).transpose(1, 2)
    assert nb.nna_layer_norm(frames, w, b).shape == (2, 0, 96)


def test_rows_of_one_value_and_of_huge_values(nb):
    x = torch.tensor([[5.0] * 32, [0.0] * 32, [1e18] * 16 + [-1e18] * 16, [1e-30] * 31 + [-1e-30]], device=DEV)
    y = nb.nna_layer_norm(x, eps=EPS)
    ref = _exact(x, None, None)[0]
    assert torch.isfinite(y).all() and torch.allclose(y.double(), ref, rtol=1e-5, atol=1e-5)


def test_a_value_that_is_not_finite_stays_in_its_row(nb):
    x, w, b, g = _inputs((9, 300), torch.float32)
    clean, kc = nb.nna_layer_norm(x, w, b, keep=32)
    bad = x.clone()
    bad[2, 7], bad[5, 299] = float("nan"), float("inf")
    frames = bad.T.contiguous()[None].transpose(1, 2)
    for y in (nb.nna_layer_norm(bad, w, b), nb.nna_layer_norm(frames, w, b)[0]):
        assert torch.isnan(y[[2, 5]]).all()
        keep = [0, 1, 3, 4, 6, 7, 8]
        assert torch.allclose(y[keep], clean[keep], rtol=1e-5, atol=1e-5)
    y, k8 = nb.nna_layer_norm(bad, w, b, keep=8)
    gx = nb.nna_layer_norm_backward(g, k8, w)[0]
    assert torch.isnan(gx[[2, 5]]).any(-1).all() and torch.isfinite(gx[keep]).all()


def test_gradients_against_differences(nb):
    """<gx, d> against (L(x + e d) - L(x - e d)) / 2e, L = sum gout y of the kernel's own y.  With |d| = |x| / sqrt(n)-sized steps e = 2^-6 the
    third-order term is below e^2 |L'''| ~ 2^-12 of sum |gout h| and y's rounding gives 2^-24 |y| per value over 2e."""
    for frames in (False, True):
        x, w, b, g = _inputs((23, 200), torch.float32, seed=21)
        d = _inputs((23, 200), torch.float32, seed=22)[3]
        call = (lambda v: nb.nna_layer_norm(v.T.contiguous()[None].transpose(1, 2), w, b, keep=32)) if frames else (lambda v: nb.nna_layer_norm(v, w, b, keep=32))
        kept = call(x)[1]
        gx = nb.nna_layer_norm_backward(g[None].contiguous() if frames else g, kept, w)[0]
        e = 2.0**-6
        up, down = call(x + e * d)[0].double(), call(x - e * d)[0].double()
        diff = float((g.double() * (up - down)).sum()) / (2 * e)
        scale = float((g.double().abs() * w.double().abs() * (1 + up.abs())).sum())
        assert abs(float((gx.double().reshape(g.shape) * d.double()).sum()) - diff) <= scale * (2.0**-11 + 64 * U32 / e) / np.sqrt(g.numel()) * 8


# ---- 8 bits ----------------------------------------------------------------------------------------------------------
def _codes(x):
    """float32 arithmetic of the definition, in numpy"""
    rows, width = x.shape
    blocks = -(-width // 128)
    v = np.zeros((rows, blocks * 128), np.float32)
    v[:, :width] = x
    v = v.reshape(rows, blocks, 128)
    most = np.abs(v).max(-1)
    with np.errstate(all="ignore"):
        bad = ~np.isfinite(most)
        zero = most < np.float32(2.0**-100)
        up = np.where(zero | bad, np.float32(0), np.float32(127) / np.where(zero | bad, np.float32(1), most))
        codes = np.rint(np.where(bad[..., None], np.float32(0), v * up[..., None]).astype(np.float32))
        scales = np.where(zero, np.float32(0), most * np.float32(1 / 127)).astype(np.float32)
    scales[bad] = np.nan
    return codes.reshape(rows, -1)[:, :width].astype(np.int8), scales


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,width", [(1, 1), (1, 127), (3, 128), (2, 129), (5, 1000), (1, 100003), (700, 257)])
def test_codes_are_the_definitions_bit_for_bit(nb, dtype, rows, width):
    _say("pack8", dtype, rows, width)
    x = (_inputs((rows, width), torch.float32, seed=width)[0] * torch.exp(torch.randn(rows, 1, device=DEV, generator=_gen(1)))).to(dtype)
    codes, scales = nb.nna_pack8(x)
    rc, rs = _codes(x.float().cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), rc) and np.array_equal(scales.cpu().numpy(), rs)
    back = nb.nna_unpack8(codes, scales)
    values = (rc.astype(np.float32) * np.repeat(rs, 128, 1)[:, :width]).astype(np.float32)
    assert np.array_equal(back.cpu().numpy(), values)
    # half a code, and four roundings of at most the largest value
    assert (back.double() - x.double()).abs().max() <= float(x.double().abs().max()) * (1 / 254 + 4 * U32)
    for t in (torch.bfloat16, torch.float16):
        assert torch.equal(nb.nna_unpack8(codes, scales, dtype=t), back.to(t))


def test_codes_of_blocks_that_are_zero_tiny_or_not_finite(nb):
    x = torch.zeros((6, 256), device=DEV)
    x[1] = 2.0**-120
    x[2, 5], x[2, 200] = float("inf"), 1.0
    x[3, 130] = float("nan")
    x[3, 127] = -3.0
    x[4] = torch.linspace(-1, 1, 256, device=DEV) * 3e38
    x[5, 255] = -float("inf")
    x[5, 0] = float("nan")
    codes, scales = nb.nna_pack8(x)
    rc, rs = _codes(x.cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), rc) and np.array_equal(scales.cpu().numpy(), rs, equal_nan=True)
    back = nb.nna_unpack8(codes, scales)
    assert not back[:2].any() and torch.isnan(back[2, :128]).all() and torch.isnan(back[3, 128:]).all() and torch.isnan(back[5]).all()
    assert back[2, 200] == 1 and abs(float(back[3, 127]) + 3) < 1e-6 and torch.isfinite(back[4]).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("rows,width", [(3, 1), (4, 100), (7, 128), (5, 300), (33, 512), (9, 1000), (3, 2049), (2, 5000), (2, 9000), (4001, 256)])
def test_layer_norm_that_keeps_8_bits(nb, dtype, rows, width):
    _say("norm8", dtype, rows, width)
    x, w, b, g = _inputs((rows, width), dtype, seed=rows + width)
    g = g.to(dtype)
    y, kept = nb.nna_layer_norm(x, w, b, eps=EPS, keep=8)
    assert kept.x is None and torch.equal(y, nb.nna_layer_norm(x, w, b, eps=EPS))
    codes, scales = nb.nna_pack8(x)
    assert torch.equal(codes, kept.codes) and torch.equal(scales, kept.scales)
    _check_grads(*nb.nna_layer_norm_backward(g, kept, w), nb.nna_unpack8(codes, scales), w, g, stats_of=x)


def test_pack8_of_strided_rows_and_of_nothing(nb):
    big = _inputs((6, 500), torch.bfloat16)[0]
    x = big[1:5, 3:262]
    codes, scales = nb.nna_pack8(x)
    rc, rs = _codes(x.float().cpu().numpy())
    assert np.array_equal(codes.cpu().numpy(), rc) and np.array_equal(scales.cpu().numpy(), rs)
    codes, scales = nb.nna_pack8(torch.empty((0, 40), device=DEV))
    assert nb.nna_unpack8(codes, scales).shape == (0, 40)


# ---- refusals, streams, graphs -------------------------------------------------------------------------------------------
def test_refusals(nb):
    x, w, b, g = _inputs((4, 96), torch.float32)
    y, kept = nb.nna_layer_norm(x, w, b, keep=32)
    for bad in (lambda: nb.nna_layer_norm(x.cpu()), lambda: nb.nna_layer_norm(x.double()), lambda: nb.nna_layer_norm(x, w[:95]),
                lambda: nb.nna_layer_norm(x, w.bfloat16()), lambda: nb.nna_layer_norm(x.bfloat16(), out=torch.empty_like(x)),
                lambda: nb.nna_layer_norm(x[:, ::2]), lambda: nb.nna_layer_norm(x.bfloat16().expand(2, 4, 96).transpose(1, 2)),
                lambda: nb.nna_layer_norm(x[None].transpose(1, 2), keep=8), lambda: nb.nna_layer_norm_backward(g.bfloat16(), kept, w),
                lambda: nb.nna_layer_norm_backward(g[:3], kept, w), lambda: nb.nna_layer_norm_backward(g.T.contiguous().T, kept, w),
                lambda: nb.nna_pack8(x.T), lambda: nb.nna_unpack8(x, x), lambda: nb.nna_layer_norm(torch.tensor(1.0, device=DEV))):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        nb.nna_layer_norm(x, keep=16)
    for bad, status in ((lambda: nb.nna_layer_norm(x, eps=-1.0), nb.NNA_ERR_INVALID_ARG), (lambda: nb.nna_layer_norm(x, eps=float("nan")), nb.NNA_ERR_INVALID_ARG),
                        (lambda: nb.nna_layer_norm(x.half(), out_dtype=torch.bfloat16), nb.NNA_ERR_INVALID_ARG),
                        (lambda: nb.nna_layer_norm(torch.empty((2, 16385), device=DEV)), nb.NNA_ERR_UNSUPPORTED),
                        (lambda: nb.nna_layer_norm(torch.empty((1, 2113, 4), device=DEV).transpose(1, 2)), nb.NNA_ERR_UNSUPPORTED),
                        (lambda: nb.nna_layer_norm(x, out_dtype=torch.bfloat16, keep=8), nb.NNA_ERR_UNSUPPORTED),
                        (lambda: nb.nna_layer_norm(torch.empty((2, 0), device=DEV)), nb.NNA_ERR_SHAPE),
                        (lambda: nb.nna_layer_norm_backward(g, kept, w, want_gx=False, want_gw=False), nb.NNA_ERR_INVALID_ARG),
                        (lambda: nb.nna_layer_norm_backward(g, kept, w, workspace=torch.empty(16, dtype=torch.uint8, device=DEV)), nb.NNA_ERR_INVALID_ARG)):
        with pytest.raises(nb.NnaError) as e:
            bad()
        assert e.value.status == status


def test_on_another_stream_and_in_a_graph(nb):
    x, w, b, g = _inputs((300, 640), torch.bfloat16)
    g = g.to(x.dtype)
    spec = _inputs((2, 50, 130), torch.float32)[0].transpose(1, 2).contiguous()

    def step(stream=None):
        y, kept = nb.nna_layer_norm(x, w, b, keep=8, stream=stream)
        f, kf = nb.nna_layer_norm(spec.transpose(1, 2), keep=32, stream=stream)
        return (y, *nb.nna_layer_norm_backward(g, kept, w, stream=stream), f, *nb.nna_layer_norm_backward(f, kf, stream=stream))

    eager = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = step(stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(eager, out))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for k in range(3):
        x.copy_(torch.randn_like(x, dtype=torch.float32))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        assert all(torch.equal(a, c) for a, c in zip(step(), got)), k


def test_rows_normalised_in_place(nb):
    """y over x is right where x is not what is kept, and refused where it is: the gradients would be those of y."""
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        for width in (40, 640, 5000):
            _say("in place", dtype, width)
            x, w, b, g = _inputs((37, width), dtype, seed=width)
            g = g.to(dtype)
            y, kept = nb.nna_layer_norm(x, w, b, keep=8)
            ref = nb.nna_layer_norm_backward(g, kept, w)
            z = x.clone()
            assert nb.nna_layer_norm(z, w, b, out=z) is z and torch.equal(z, y)
            z = x.clone()
            z, kept = nb.nna_layer_norm(z, w, b, keep=8, out=z)
            assert torch.equal(z, y) and all(torch.equal(a, c) for a, c in zip(nb.nna_layer_norm_backward(g, kept, w), ref))
            z = x.clone()
            for out in (z, z.view(-1)[:x.numel()].view(x.shape)):
                with pytest.raises(ValueError):
                    nb.nna_layer_norm(z, w, b, keep=32, out=out)
            two = torch.cat([x, x])
            with pytest.raises(ValueError):
                nb.nna_layer_norm(two[:37], w, b, keep=32, out=two[36:73])
            assert torch.equal(two, torch.cat([x, x]))
            out, kept = nb.nna_layer_norm(two[:37], w, b, keep=32, out=two[37:])  # beside it: nothing is shared
            assert torch.equal(two[37:], y) and torch.equal(kept.x, x)


def test_outputs_over_inputs_are_refused(nb):
    """Where other workgroups still read what one writes: frames in place, other strides or types, part of the input, the weights."""
    buf = torch.zeros(40 * 64, device=DEV)
    x, w = buf[:1280].view(20, 64), torch.ones(64, device=DEV)
    frames = buf[:1280].view(1, 64, 20).transpose(1, 2)
    wide = buf.view(20, 128)[:, :64]
    scales = torch.ones(20, 1, device=DEV)
    for bad in (lambda: nb.nna_layer_norm(frames, out=buf[:1280].view(1, 20, 64)), lambda: nb.nna_layer_norm(wide, out=buf[:1280].view(20, 64)),
                lambda: nb.nna_layer_norm(x, out=buf[64:1344].view(20, 64)), lambda: nb.nna_layer_norm(x[:1].expand(20, 64), out=x),
                lambda: nb.nna_layer_norm(x, out_dtype=torch.bfloat16, out=buf.view(torch.bfloat16)[:1280].view(20, 64)),
                lambda: nb.nna_layer_norm(torch.ones(1, 64, device=DEV), w, out=w[None]), lambda: nb.nna_layer_norm(torch.ones(1, 64, device=DEV), None, w, out=w[None]),
                lambda: nb.nna_unpack8(buf.view(torch.int8)[-1280:].view(20, 64), scales, out=buf[-1280:].view(20, 64))):
        with pytest.raises(ValueError):
            bad()
    p, st = buf.data_ptr(), torch.cuda.current_stream().cuda_stream
    stats, ws = torch.zeros(64, device=DEV), torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    norm, back = nb.lib().nna_layer_norm, nb.lib().nna_layer_norm_backward
    for status in (nb.lib().nna_layer_norm_frames(p, 1, 64, 20, None, None, 1e-5, p, nb.NNA_F32, None, 0, st),
                   norm(p, nb.NNA_F32, 20, 64, 128, None, None, 1e-5, p, nb.NNA_F32, None, None, None, 0, st),
                   norm(p, nb.NNA_F32, 20, 64, 64, None, None, 1e-5, p, nb.NNA_BF16, None, None, None, 0, st),
                   nb.lib().nna_layer_norm_frames_backward(p, nb.NNA_F32, p + 5120, 1, 64, 20, stats.data_ptr(), None, p, None, None, None, 0, 0, st),
                   back(p, nb.NNA_BF16, p + 5120, nb.NNA_F32, 20, 64, 64, None, None, stats.data_ptr(), None, p, None, None, None, 0, 0, st)):
        assert status == nb.NNA_ERR_INVALID_ARG
    # over gout where nothing else is read of it: allowed, and right
    x, w, b, g = _inputs((300, 640), torch.float32)
    kept = nb.nna_layer_norm(x, w, b, keep=32)[1]
    gx = nb.nna_layer_norm_backward(g, kept, w, want_gw=False)[0]
    assert back(g.data_ptr(), nb.NNA_F32, x.data_ptr(), nb.NNA_F32, 300, 640, 640, None, None, kept.stats.data_ptr(), w.data_ptr(), g.data_ptr(), None, None, None, 0, 0, st) == nb.NNA_OK
    assert torch.equal(g, gx)


def test_weights_that_are_no_tensors_are_refused_with_a_given_output_too(nb):
    x = torch.ones(3, 8, device=DEV)
    for bad in ([1.0] * 8, np.ones(8, np.float32)):
        for kw in (dict(weight=bad), dict(bias=bad)):
            for out in (None, torch.empty_like(x)):
                with pytest.raises(TypeError):
                    nb.nna_layer_norm(x, out=out, **kw)
