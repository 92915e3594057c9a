"""Queries and keys normalised and rotated in one pass against the definition in 64 bits, forward and backward.

Tolerances, in units of U = 2^-24 of a row's sums of magnitudes.  A sum of squares over a head is off by at most width / lanes + 8 roundings, its root and reciprocal by 3, a value by
2 more; cos and sin are off by 2 U of one (the remainder of the angle 1, the functions 1), a turned pair by 4 U of its magnitudes: 64 U of the row's largest magnitude holds for all
heads up to 256 values here.  A row's gradient takes one more sum over the head: its terms are bounded by r (|g w| + |h| mean |g w h|).  Weights' gradients are sums over rows: (rows + 64) U
of the sums of magnitudes.  A 16-bit result is rounded once more, by half a step of its value.
"""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0**-24
TYPES = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def nb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import binding
    binding.lib()
    return binding


def _say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def exact(x, freqs, positions, weight, eps, interleaved, g=None):
    """(y, its tolerance, gx, its tolerance, gw, its tolerance) in 64 bits on the CPU, x [B, T, H, width], positions [B, T]"""
    x, freqs, positions, weight, g = (None if t is None else t.double().cpu() for t in (x, freqs, positions, weight, g))
    n, width = freqs.numel(), x.shape[-1]
    angle = positions[..., None, None] * freqs
    cos, sin = torch.cos(angle), torch.sin(angle)
    first = torch.arange(n) * 2 if interleaved else torch.arange(n)
    second = first + 1 if interleaved else first + n

    def turn(v, sin):
        out = v.clone()
        out[..., first] = v[..., first] * cos - v[..., second] * sin
        out[..., second] = v[..., first] * sin + v[..., second] * cos
        return out

    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) if eps is not None else torch.ones_like(x[..., :1])
    h = x * r
    w = weight if weight is not None else torch.ones(width, dtype=torch.float64)
    y = turn(h * w, sin)
    most = (h * w).abs().amax(-1, keepdim=True)
    out = [y, 64 * U * most.expand_as(y)]
    if g is None:
        return out
    back = turn(g, -sin)
    if eps is None:
        return out + [back, 64 * U * back.abs().amax(-1, keepdim=True).expand_as(y), None, None]
    gw = (back * h).sum((0, 1, 2))
    size = (back.abs().amax(-1, keepdim=True) * h.abs()).sum((0, 1, 2))
    t = back * w
    gx = r * (t - h * (t * h).mean(-1, keepdim=True))
    bound = r * (t.abs().amax(-1, keepdim=True) + h.abs() * (t * h).abs().mean(-1, keepdim=True))
    rows = x[..., 0].numel()
    return out + [gx, 64 * U * bound, gw, (rows + 64) * U * size]


def near(name, got, value, tolerance):
    got = got.cpu()
    if got.dtype != torch.float32:
        tolerance = tolerance + torch.finfo(got.dtype).eps / 2 * torch.clamp(value.abs() + tolerance, min=torch.finfo(got.dtype).tiny)
    off = (got.double() - value).abs()
    worst = float((off / tolerance.clamp(min=1e-300)).max()) if off.numel() else 0.0
    assert worst <= 1, (name, worst)


def inputs(B, T, H, K, width, pairs, dtype, seed=0, far=False, weights=True):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*s):
        return torch.randn(*s, device=DEV, generator=g)

    q, gq = normal(B, T, H, width).to(dtype), normal(B, T, H, width).to(dtype)
    k, gk = (normal(B, T, K, width).to(dtype), normal(B, T, K, width).to(dtype)) if K else (None, None)
    freqs = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64, device=DEV) / max(1, pairs))
    positions = torch.randint(-(1 << 31) if far else -100, (1 << 31) - 1 if far else 1000, (B, T), device=DEV, generator=g).to(torch.int32)
    wq, wk = (1 + 0.3 * normal(width), 1 + 0.3 * normal(width)) if weights else (None, None)
    return q, k, gq, gk, freqs, positions, wq, wk if K else None


def check(nb, q, k, gq, gk, freqs, positions, wq, wk, eps, interleaved, offset=0):
    B, T = q.shape[:2]
    how = dict(positions=positions, offset=offset, q_weight=wq, k_weight=wk, eps=eps, interleaved=interleaved)
    at = positions if positions is not None else offset + torch.arange(T, device=DEV).expand(B, T)
    yq, yk = nb.nna_rotate_heads(q, k, freqs, **how)
    hq, hk, gqw, gkw = nb.nna_rotate_heads_backward(gq, gk, q, k, freqs, **how)
    for x, y, g, h, w, gw in ((q, yq, gq, hq, wq, gqw), (k, yk, gk, hk, wk, gkw)):
        if x is None:
            assert y is None and h is None and gw is None
            continue
        want = exact(x, freqs, at, w, eps, interleaved, g)
        near("y", y, *want[:2])
        near("gx", h, *want[2:4])
        if eps is None:
            assert gw is None
        else:
            near("gw", gw, *want[4:])
    return yq, yk, hq, hk, gqw, gkw


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("width,pairs", [(64, 32), (64, 16), (64, 5), (64, 0), (128, 64), (128, 24), (48, 24), (80, 20), (33, 16), (33, 3), (1, 0), (2, 1), (3, 1), (16, 8), (40, 20), (96, 36),
                                         (127, 63), (128, 1), (256, 128), (256, 64), (255, 127), (131, 30), (200, 100), (129, 0)])
def test_heads(nb, width, pairs, interleaved, dtype):
    _say(width, pairs, interleaved, dtype)
    for H, K, eps, weights in ((3, 2, 1e-6, True), (4, 4, None, False), (1, 0, 1e-3, False)):
        check(nb, *inputs(2, 5, H, K, width, pairs, dtype, seed=width, weights=weights), eps, interleaved)


@pytest.mark.parametrize("B,T,H,K", [(1, 1, 1, 1), (1, 1, 16, 16), (7, 1, 8, 2), (1, 300, 5, 1), (3, 101, 8, 8), (2, 64, 1, 0), (2, 40, 70, 3), (1, 9, 300, 1), (2, 3, 4100, 1), (1, 50, 1, 130)])
def test_shapes(nb, B, T, H, K):
    for dtype, width in ((torch.bfloat16, 64), (torch.float32, 48), (torch.float32, 6)):
        check(nb, *inputs(B, T, H, K, width, width // 2, dtype, seed=T), 1e-6, False)


def test_many_rows(nb):
    """More tokens than the backward pass has workgroups."""
    check(nb, *inputs(4, 2500, 8, 2, 16, 8, torch.float32), 1e-6, True)


def test_far_positions(nb):
    """Any int32 position, and offsets of 2^40: the angle's own 64 bits are what limits it (2^-53 of 2^31, 2^40 turns: nothing, and 2^-13 of a float32's step)."""
    for dtype in TYPES:
        check(nb, *inputs(2, 33, 2, 2, 64, 32, dtype, far=True), 1e-6, False)
    q, k, gq, gk, freqs, _, wq, wk = inputs(1, 33, 2, 2, 64, 32, torch.float32)
    slow = freqs * 2.0**-12
    check(nb, q, k, gq, gk, slow, None, wq, wk, 1e-6, True, offset=1 << 40)
    check(nb, q, k, gq, gk, freqs, None, wq, wk, 1e-6, True, offset=-12345)


def test_strides_and_one_frame(nb):
    """Slices of one projection, misaligned; heads before frames; keys shared by heads; positions of one sequence for all; and frames on their own."""
    for dtype in TYPES:
        q, k, gq, gk, freqs, positions, wq, wk = inputs(3, 50, 4, 4, 40, 10, dtype)
        want = check(nb, q, k, gq, gk, freqs, positions, wq, wk, 1e-5, False)
        qkv = torch.zeros(3, 50, 1 + 8 * 40, dtype=dtype, device=DEV)
        q2, k2 = qkv[..., 1 : 1 + 160].view(3, 50, 4, 40), qkv[..., 161:].view(3, 50, 4, 40)
        q2.copy_(q)
        k2.copy_(k.transpose(2, 1).contiguous().transpose(2, 1))
        got = check(nb, q2, k.transpose(2, 1).contiguous().transpose(2, 1), gq, gk, freqs, positions.t().contiguous().t(), wq, wk, 1e-5, False)
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        check(nb, q, k2[:, :, :1].expand(3, 50, 4, 40), gq, gk, freqs, positions[:1].expand(3, 50), wq, wk, 1e-5, False)
        yq, yk = nb.nna_rotate_heads(q[:, 7], k[:, 7], freqs, positions=positions[:, 7], q_weight=wq, k_weight=wk, eps=1e-5)
        assert torch.equal(yq, want[0][:, 7]) and torch.equal(yk, want[1][:, 7])
        back = nb.nna_rotate_heads_backward(gq[:, 7].contiguous(), gk[:, 7].contiguous(), q[:, 7], k[:, 7], freqs, positions=positions[:, 7], q_weight=wq, k_weight=wk, eps=1e-5)
        assert torch.equal(back[0], want[2][:, 7]) and torch.equal(back[1], want[3][:, 7])


def test_what_is_not_finite_stays_in_its_row(nb):
    q, k, gq, gk, freqs, positions, wq, wk = inputs(2, 40, 4, 4, 64, 32, torch.bfloat16)
    clean = nb.nna_rotate_heads(q, k, freqs, positions=positions, q_weight=wq, k_weight=wk, eps=1e-6)
    for value in (float("nan"), float("inf")):
        spoilt = q.clone()
        spoilt[1, 3, 2, 5] = value
        y = nb.nna_rotate_heads(spoilt, k, freqs, positions=positions, q_weight=wq, k_weight=wk, eps=1e-6)
        touched = torch.zeros_like(q, dtype=torch.bool)
        touched[1, 3, 2] = True
        assert torch.equal(y[0][~touched], clean[0][~touched]) and torch.equal(y[1], clean[1])
        assert y[0][1, 3, 2].isnan().any()


def test_rows_of_zeros(nb):
    """With eps = 0 a row of zeros is not a number, with eps it is zero, and its gradient is g w / sqrt(eps)."""
    q, k, gq, gk, freqs, positions, wq, wk = inputs(1, 4, 2, 0, 32, 16, torch.float32)
    q[0, 2, 1] = 0
    check(nb, q, None, gq, None, freqs, positions, wq, None, 1e-6, False)
    y, _ = nb.nna_rotate_heads(q, None, freqs, positions=positions, eps=1e-6)
    assert not y[0, 2, 1].any()


def test_gradients_against_differences(nb):
    """Both sides' differences in 64 bits along random directions: off by h^2 / 6 of the third derivative (below 1,000 here: 2e-6) and 2^-18 of the terms."""
    q, _, gq, _, freqs, positions, wq, _ = inputs(2, 5, 2, 0, 12, 4, torch.float32, seed=4)
    hq, _, gqw, _ = nb.nna_rotate_heads_backward(gq, None, q, None, freqs, positions=positions, q_weight=wq, eps=1e-2)

    def loss(q, w):
        return float((exact(q, freqs, positions, w, 1e-2, False)[0] * gq.double().cpu()).sum())

    for leaf, grad in ((0, hq), (1, gqw)):
        x = [q.double(), wq.double()]
        d = torch.randn_like(x[leaf])
        up, down = ([t + s * 1e-4 * d if j == leaf else t for j, t in enumerate(x)] for s in (1, -1))
        want = (loss(*up) - loss(*down)) / 2e-4
        assert abs(float((grad.double() * d).sum()) - want) <= 1e-5 * float((grad.double() * d).abs().sum())


def test_same_bits(nb):
    args = inputs(4, 2500, 8, 2, 64, 32, torch.bfloat16)
    q, k, gq, gk, freqs, positions, wq, wk = args
    how = dict(positions=positions, q_weight=wq, k_weight=wk, eps=1e-6)
    one, two = (nb.nna_rotate_heads_backward(gq, gk, q, k, freqs, **how) for _ in range(2))
    for a, b in zip(one, two):
        assert torch.equal(a, b)


def test_empty(nb):
    for B, T in ((0, 3), (2, 0)):
        q = torch.empty(B, T, 4, 8, device=DEV)
        freqs = nb.nna_rotary_freqs(8)
        y, _ = nb.nna_rotate_heads(q, None, freqs, eps=1e-6)
        h, _, gw, _ = nb.nna_rotate_heads_backward(q, None, q, None, freqs, eps=1e-6)
        assert y.shape == q.shape == h.shape and not gw.any()


def test_refusals(nb):
    q, k, gq, gk, freqs, positions, wq, wk = inputs(2, 5, 4, 2, 16, 8, torch.float32)
    call = nb.nna_rotate_heads
    bad = [
        lambda: call(q.cpu(), k, freqs), lambda: call(q, k.cpu(), freqs), lambda: call(q, k.half(), freqs), lambda: call(q.double(), None, freqs), lambda: call(q, k[:, :4], freqs),
        lambda: call(q, k[..., :8], freqs), lambda: call(q, k[:, 0], freqs), lambda: call(q[0, 0], None, freqs), lambda: call(q, k, freqs.float()), lambda: call(q, k, freqs.cpu()),
        lambda: call(q, k, freqs[::2]), lambda: call(q, k, torch.cat([freqs, freqs])), lambda: call(q, k, freqs, positions=positions.long()),
        lambda: call(q, k, freqs, positions=positions[:1]), lambda: call(q, k, freqs, positions=positions.cpu()), lambda: call(q, k, freqs, positions=positions, offset=3),
        lambda: call(q, k, freqs, q_weight=wq), lambda: call(q, k, freqs, q_weight=wq[:8], eps=1e-6), lambda: call(q, k, freqs, eps=-1.0), lambda: call(q, k, freqs, out=(q, k)),
        lambda: call(q, k, freqs, out=(torch.empty_like(q), None)), lambda: call(q, k, freqs, out=(torch.empty_like(q).half(), torch.empty_like(k))),
        lambda: call(q.transpose(2, 3), None, freqs[:1]), lambda: call(torch.empty(1, 1, 1, 257, device=DEV), None, freqs),
        lambda: nb.nna_rotate_heads_backward(gq, None, q, k, freqs), lambda: nb.nna_rotate_heads_backward(gq[:1], gk, q, k, freqs),
        lambda: nb.nna_rotate_heads_backward(gq.half(), gk, q, k, freqs), lambda: nb.nna_rotate_heads_backward(gq.transpose(0, 1), gk, q, k, freqs),
    ]
    for n, c in enumerate(bad):
        with pytest.raises((TypeError, ValueError, nb.NnaError)):
            c()
            pytest.fail(f"call {n} was not refused")


def test_out_another_stream_and_a_graph(nb):
    q, k, gq, gk, freqs, positions, wq, wk = inputs(2, 300, 4, 2, 64, 32, torch.bfloat16)
    how = dict(positions=positions, q_weight=wq, k_weight=wk, eps=1e-6)

    def call():
        return (*nb.nna_rotate_heads(q, k, freqs, **how), *nb.nna_rotate_heads_backward(gq, gk, q, k, freqs, **how))

    want = call()
    out = torch.empty_like(q), torch.empty_like(k)
    version = out[0]._version
    assert nb.nna_rotate_heads(q, k, freqs, **how, out=out)[0] is out[0] and out[0]._version > version
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = nb.nna_rotate_heads(q, k, freqs, **how, stream=side.cuda_stream)
    back = nb.nna_rotate_heads_backward(gq, gk, q, k, freqs, **how, stream=side.cuda_stream)
    side.synchronize()
    for a, b in zip(want, (*got, *back)):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for _ in range(3):
        q.copy_(torch.randn_like(q))
        positions.add_(17)
        graph.replay()
        got = [t.clone() for t in held]
        for a, b in zip(got, call()):
            assert torch.equal(a, b)
        torch.cuda.synchronize()


def test_far_apart(nb):
    """Sequences whose elements' offsets pass 32 bits."""
    q, k, gq, gk, freqs, positions, wq, wk = inputs(2, 9, 2, 2, 64, 32, torch.bfloat16)
    memory = torch.empty((1 << 32) + 9 * 2 * 64 * 2, dtype=torch.bfloat16, device=DEV)
    far_q, far_k = (memory[at:].as_strided((2, 9, 2, 64), (1 << 32, 128, 64, 1)) for at in (0, 9 * 128))
    far_q.copy_(q)
    far_k.copy_(k)
    how = dict(positions=positions, q_weight=wq, k_weight=wk, eps=1e-6)
    for a, b in zip(nb.nna_rotate_heads(q, k, freqs, **how), nb.nna_rotate_heads(far_q, far_k, freqs, **how)):
        assert torch.equal(a, b)
    for a, b in zip(nb.nna_rotate_heads_backward(gq, gk, q, k, freqs, **how), nb.nna_rotate_heads_backward(gq, gk, far_q, far_k, freqs, **how)):
        assert torch.equal(a, b)
