"""AdamW where gradients are so small that a float32 product may be none, with an eps of nothing or nearly; and many tensors in several launches, states in 8 bits.

Tolerances, U = 2^-24.  An update is one quotient: 20 U of its largest size, as for any gradient; a moment below 2^-126 is held to 2^-149, and two of them are rounded so: 2 2^-149 of it for the
first and half of that share for the second's root.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U, LEAST = 2.0**-24, 2.0**-149


@pytest.fixture(scope="module")
def nb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import binding
    binding.lib()
    return binding


def states(nb, sizes, bits):
    _, size = nb.nna_adamw_places(sizes)
    s = dict(m=torch.zeros(size, device=DEV, dtype=torch.float32 if bits == 32 else torch.int8), v=torch.zeros(size, device=DEV, dtype=torch.float32 if bits == 32 else torch.uint8))
    if bits == 8:
        s["m_scales"], s["v_scales"] = torch.zeros(size // 128, device=DEV), torch.zeros(size // 128, device=DEV)
    return s


def values(s):
    """(m, v) in 64 bits"""
    if "m_scales" not in s:
        return s["m"].double(), s["v"].double()
    m, v = s["m"].double() / 127, s["v"].double() / 255
    return m * m.abs() * s["m_scales"].double().repeat_interleave(128), v**4 * s["v_scales"].double().repeat_interleave(128)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("size,eps", [(1e-18, 0.0), (1e-18, 1e-20), (3e-18, 0.0), (1e-17, 0.0), (1e-15, 0.0), (1e-15, 1e-20), (1e-10, 0.0), (1.0, 0.0), (1e-33, 1e-20), (1e-36, 1e-20), (1e-30, 1e-20)])
def test_weights_of_faint_gradients(nb, bits, size, eps):
    """Steps of 16 blocks whose history is far above this step's own part of the moments: what the codes hold has to reach the weight."""
    n, betas, lr = 2048, (0.9, 0.99), 1.0
    g0 = torch.Generator(device=DEV).manual_seed(3)
    s = states(nb, [n], bits)
    for t in (1, 2, 3, 100):
        # (no gradient far below the others: where v is nothing in float32 the quotient with an eps of zero is none)
        g = size * (1 + torch.rand(n, device=DEV, generator=g0)) * (0.1 if t == 3 else 1.0)
        p, (om, ov) = torch.zeros(n, device=DEV), values(s)
        nb.nna_adamw([p], [g], step=t, **s, lr=lr, betas=betas, eps=eps, weight_decay=0.0)
        d = g.double()
        m, v = betas[0] * om + (1 - betas[0]) * d, betas[1] * ov + (1 - betas[1]) * d * d
        seen = v > 0.5 * LEAST  # (float32 has v)
        root = (v / (1 - betas[1] ** t)).sqrt() + eps
        rate = lr / (1 - betas[0] ** t)
        share = 20 * U + 2 * LEAST / m.abs() + torch.where(v > 64 * LEAST, LEAST / v, 1.0) * (1 - eps / root)
        assert bool(((p.double() + rate * m / root).abs() <= rate * m.abs() / root * share)[seen | (eps > 0)].all()), t


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.float32, torch.bfloat16, torch.float16)])
def test_many_tensors_in_8_bits(nb, dtypes):
    """More tensors than a launch takes, against the same steps one tensor at a time: weights, first moments and scales are equal.  Second moments' codes go with the place: the definition's."""
    sizes = [1 + 37 * n % 1000 for n in range(333)]
    g0 = torch.Generator(device=DEV).manual_seed(4)
    params = [torch.randn(n, device=DEV, generator=g0).to(dtypes[k % len(dtypes)]) for k, n in enumerate(sizes)]
    grads = [torch.randn(n, device=DEV, generator=g0).to(p.dtype) for n, p in zip(sizes, params)]
    how = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.05, step=5)
    places, _ = nb.nna_adamw_places(sizes)
    s = states(nb, sizes, 8)
    whole = [p.clone() for p in params]
    nb.nna_adamw(whole, grads, **s, **how)
    for k, n in enumerate(sizes):
        one, alone = params[k].clone(), states(nb, [n], 8)
        nb.nna_adamw([one], [grads[k]], **alone, **how)
        at, blocks = int(places[k]), -(-n // 128)
        assert torch.equal(one, whole[k]), k
        assert torch.equal(alone["m"], s["m"][at : at + 128 * blocks]), k
        for name in ("m_scales", "v_scales"):
            assert torch.equal(alone[name], s[name][at // 128 : at // 128 + blocks]), (k, name)
    v = torch.zeros(s["v"].numel(), device=DEV, dtype=torch.float64)
    for k, n in enumerate(sizes):
        v[int(places[k]) : int(places[k]) + n] = (1 - how["betas"][1]) * grads[k].double() ** 2
    most = s["v_scales"].double().repeat_interleave(128)
    shift = (((torch.arange(v.numel(), device=DEV) * 0x9E3779B9 + 5 * 0xB504F333) & 0xFFFFFFFF) >> 8).double() * 2.0**-24
    codes = torch.floor(255 * (v / torch.where(most > 0, most, 1)) ** 0.25 + shift).clamp(max=255)
    assert torch.equal(s["v"].double(), torch.where(v > 0, codes.clamp(min=1), 0))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-38, 1e-40, 1e-45, 1e-60])
def test_no_gradient_and_an_eps_below_float32(nb, bits, eps):
    """Nothing over an eps that has no normal float32 is nothing, and not a NaN."""
    p, s = torch.ones(300, device=DEV), states(nb, [300], bits)
    g = torch.zeros(300, device=DEV)
    g[7] = 1.0
    for t in (1, 2):
        nb.nna_adamw([p], [g], step=t, **s, lr=0.25, betas=(0.9, 0.99), eps=eps, weight_decay=0.0)
    rest = torch.ones(300, dtype=torch.bool, device=DEV)
    rest[7] = False
    assert bool((p[rest] == 1).all()) and abs(float(p[7]) - 0.5) <= 40 * U
