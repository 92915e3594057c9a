"""Layer norm and linear attention where counts of threads and of bytes pass 32 bits."""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32 = 2.0**-24


@pytest.fixture(scope="module")
def nb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import binding
    binding.lib()
    return binding


def test_more_frames_than_a_launch_has_threads_for(nb):
    """Four bins: y = (x - m) r, with m and r of four values; three roundings of sums and one each of r, the difference and the product, and m's
    own error against a difference, all below 64 units of a value of at most 2 plus what m's error (of |x| <= 8) is times r (x has a spread of 1 at least)."""
    T = (1 << 27) + (1 << 20) + 5  # more than 2^22 tiles of 32
    print("[case] frames", T, file=sys.stderr, flush=True)
    x = torch.empty((1, 4, T), device=DEV)
    for d, low in enumerate((-6.0, -2.0, 2.0, 5.0)):  # apart by construction
        x[0, d].uniform_(low, low + 1.0)
    y, kept = nb.nna_layer_norm(x.transpose(1, 2), keep=32)
    gx, _, _ = nb.nna_layer_norm_backward(y, kept, want_gw=False)
    assert y.shape == (1, T, 4)
    for at in (0, (1 << 27) - 4096, 1 << 27, T - 5000):
        v = x[0, :, at:at + 5000].T.double()
        n = v.shape[0]
        m = v.mean(1, keepdim=True)
        r = ((v - m) ** 2).mean(1, keepdim=True).add(1e-5).rsqrt()
        h = (v - m) * r
        assert (y[0, at:at + n].double() - h).abs().max() <= 64 * U32 * 8
        g = y[0, at:at + n].double()
        ref = r * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        assert (gx[0, at:at + n].double() - ref).abs().max() <= 64 * U32 * 8
    assert torch.isfinite(gx).all()


def test_as_many_heads_as_a_launch_takes(nb):
    """One value a head: products of two and three float32, a sum of two, each rounded once: exact to 8 units of the sum of magnitudes."""
    B, H = 1 << 18, 8
    print("[case] heads", B * H, file=sys.stderr, flush=True)
    g = torch.Generator(device=DEV).manual_seed(3)
    q, k, v, go = (torch.randn((B, 2, H, 1), device=DEV, generator=g) for _ in range(4))
    decay = torch.rand(H, device=DEV, generator=g)
    o, last = nb.nna_decay_attention(q, k, v, decay, want_state=True)
    gq, gk, gv, _ = nb.nna_decay_attention_backward(go, q, k, v, decay)
    l, Q, K, V, G = decay.double()[None, :, None], *(x.double() for x in (q, k, v, go))
    kv = K * V
    states = kv[:, 0], l * kv[:, 0] + kv[:, 1]
    most = kv[:, 0].abs(), l * kv[:, 0].abs() + kv[:, 1].abs()
    bound = (2 + 192 + 256) * U32  # the operator's own: dk + dv + 192 products, and the powers
    for t in (0, 1):
        assert ((o[:, t].double() - Q[:, t] * states[t]).abs() <= bound * (Q[:, t].abs() * most[t]) + 1e-37).all()
        assert ((gq[:, t].double() - G[:, t] * states[t]).abs() <= bound * (G[:, t].abs() * most[t]) + 1e-37).all()
    assert ((last[..., 0].double() - states[1]).abs() <= bound * most[1] + 1e-37).all()
    qg = Q * G
    for t, ref, size in ((1, qg[:, 1], qg[:, 1].abs()), (0, qg[:, 0] + l * qg[:, 1], qg[:, 0].abs() + l * qg[:, 1].abs())):
        assert ((gk[:, t].double() - V[:, t] * ref).abs() <= bound * (V[:, t].abs() * size) + 1e-37).all()
        assert ((gv[:, t].double() - K[:, t] * ref).abs() <= bound * (K[:, t].abs() * size) + 1e-37).all()
    state = torch.zeros((B, H, 1, 1), device=DEV)
    one = nb.nna_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, state)
    assert ((one.double() - Q[:, 0] * kv[:, 0]).abs() <= 8 * U32 * (Q[:, 0] * kv[:, 0]).abs() + 1e-37).all()
