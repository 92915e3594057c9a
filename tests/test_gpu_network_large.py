"""Arrays of more than 2^31 values: rotated heads, the gated recurrence and AdamW at their far ends against the same calls on those ends alone."""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def nb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import binding
    binding.lib()
    yield binding
    torch.cuda.empty_cache()


def _say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def test_rotated_heads(nb):
    T, tail = (1 << 24) + 77, 300
    _say("rotate", T)
    q = torch.randn(1, T, 1, 128, dtype=torch.bfloat16, device=DEV)
    freqs, w = nb.nna_rotary_freqs(128), 1 + 0.1 * torch.randn(128, device=DEV)
    y, _ = nb.nna_rotate_heads(q, None, freqs, q_weight=w, eps=1e-6)
    want, _ = nb.nna_rotate_heads(q[:, -tail:], None, freqs, offset=T - tail, q_weight=w, eps=1e-6)
    assert torch.equal(y[:, -tail:], want)
    h, _, gw, _ = nb.nna_rotate_heads_backward(y, None, q, None, freqs, q_weight=w, eps=1e-6)
    want = nb.nna_rotate_heads_backward(y[:, -tail:].contiguous(), None, q[:, -tail:], None, freqs, offset=T - tail, q_weight=w, eps=1e-6)[0]
    assert torch.equal(h[:, -tail:], want)
    # the gradient of w is the sum over rows of y turned back, w h, times h = w h^2: its sum over a head is that over all values, 2^24 rows of some 128
    assert gw.isfinite().all() and float(gw.mean()) == pytest.approx(T, rel=0.2)


def test_gated_recurrence(nb):
    T, C, tail = (1 << 22) + 130, 512, 1000
    _say("scan", T)
    x, f = (torch.randn(1, T, C, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    h, last, kept = nb.nna_gated_scan(x, f, want_state=True, keep=True)
    first = nb.nna_gated_scan(x[:, T - tail - 500 : T - tail], f[:, T - tail - 500 : T - tail], want_state=True)[1]  # (500 frames of gates about a half leave nothing of what was before)
    want, want_last, want_kept = nb.nna_gated_scan(x[:, -tail:], f[:, -tail:], state=first, want_state=True, keep=True)
    # (other segments, other roundings: a bfloat16 apart at most)
    assert float((h[:, -tail:].float() - want.float()).norm()) <= 2.0**-8 * float(want.float().norm()) and float((last - want_last).norm()) <= 1e-5 * float(last.norm())
    gx, gf, _, _ = nb.nna_gated_scan_backward(h, kept, x, f)
    wx, wf, _, _ = nb.nna_gated_scan_backward(h[:, -tail:].contiguous(), want_kept, x[:, -tail:], f[:, -tail:])
    for a, b in ((gx, wx), (gf, wf)):
        assert float((a[:, -tail:].float() - b.float()).norm()) <= 2.0**-8 * float(b.float().norm())
    assert gx[:, :tail].float().norm() > 0


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(nb, bits):
    n, tail = (1 << 31) + 300, 128 * 50 + 44
    _say("adamw", n, bits)
    p, g = torch.empty(n, dtype=torch.bfloat16, device=DEV).normal_(), torch.empty(n, dtype=torch.bfloat16, device=DEV).normal_()
    start = n - tail  # (a multiple of 128)
    assert start % 128 == 0
    _, size = nb.nna_adamw_places([n])

    def states(size):
        s = dict(m=torch.zeros(size, dtype=torch.float32 if bits == 32 else torch.int8, device=DEV), v=torch.zeros(size, dtype=torch.float32 if bits == 32 else torch.uint8, device=DEV))
        if bits == 8:
            s["m_scales"], s["v_scales"] = torch.zeros(size // 128, device=DEV), torch.zeros(size // 128, device=DEV)
        return s

    s, twin = states(size), p[start:].clone()
    t = states(nb.nna_adamw_places([tail])[1])
    for step in (1, 2):
        nb.nna_adamw([p], [g], step=step, **s)
        nb.nna_adamw([twin], [g[start:].clone()], step=step, **t)
        if step == 1:
            assert torch.equal(p[start:], twin)
    assert torch.equal(s["m"][start : start + tail], t["m"][:tail])
    if bits == 8:
        # (the additive sequence goes with the place: of another place the second moments are rounded otherwise, by a code at most)
        assert torch.equal(s["m_scales"][start // 128 :], t["m_scales"]) and int((s["v"][start:].int() - t["v"].int()).abs().max()) <= 2
        assert nb.nna_adamw_moment(s["v"], s["v_scales"])[start : start + tail].gt(0).all()
    else:
        assert torch.equal(s["v"][start : start + tail], t["v"][:tail]) and torch.equal(p[start:], twin)
