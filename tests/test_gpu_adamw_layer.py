"""The optimiser layer's state: each tensor's own number of steps, float32 copies after a load, calls that are refused, groups' options.

Tolerances against a loop in 64 bits are those of a step in 32 bits: a step of one tensor is off by 20 U of its largest size (3.2 lr at most) and 3 U of the weight (U = 2^-24), and the next
steps take both over.
"""
import copy

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0**-24


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import layers as L
    return L


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _reference(params, **how):
    twins = [torch.nn.Parameter(p.detach().double()) for p in params]
    return twins, torch.optim.AdamW(twins, foreach=False, fused=False, **how)


@pytest.mark.parametrize("capturable", [False, True])
def test_each_tensor_counts_its_own_steps(layers, capturable):
    """A tensor that is unfrozen late, one whose branch is taken now and then, and one that is always there, against torch's own count of each in 64 bits."""
    how = dict(lr=1e-2, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)
    params = [torch.nn.Parameter(torch.randn(n, device=DEV, generator=_gen(n))) for n in (300, 5, 129, 1000)]
    twins, other = _reference(params, **how)
    optimiser = layers.AdamW(params, **how, capturable=capturable)
    for t in range(24):
        g = _gen(1000 + t)
        for n, (p, q) in enumerate(zip(params, twins)):
            grad = 1 + 0.2 * torch.randn(p.shape, device=DEV, generator=g)
            if (n == 1 and t < 15) or (n == 2 and t % 5) or (n == 3 and t == 20):
                p.grad = q.grad = None
            else:
                p.grad, q.grad = grad, grad.double()
        optimiser.step()
        other.step()
        for n, (p, q) in enumerate(zip(params, twins)):
            bound = (t + 1) * (3 * U * 2 * float(q.detach().abs().max()) + 20 * U * 3.2 * 1e-2)
            assert float((p.detach().double() - q.detach()).abs().max()) <= bound, (t, n)


def test_each_tensor_counts_its_own_steps_in_a_graph(layers):
    """Two recorded steps, of all tensors and of some, replayed in any order, against the same steps run one by one."""
    def make():
        params = [torch.nn.Parameter(torch.randn(n, device=DEV, generator=_gen(n))) for n in (300, 5, 129)]
        return params, layers.AdamW(params, lr=1e-2, bits=8, capturable=True), [torch.zeros_like(p) for p in params]

    def step(params, optimiser, grads, live):
        for n, (p, g) in enumerate(zip(params, grads)):
            p.grad = g if n in live else None
        optimiser.step()

    mine, eager = make(), make()
    for one in (mine, eager):
        for n, g in enumerate(one[2]):
            g.normal_(generator=_gen(50 + n))
        step(*one, (0, 1, 2))
    graphs = {}
    torch.cuda.synchronize()
    for live in ((0, 1, 2), (0, 2)):
        graphs[live] = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graphs[live]):
            step(*mine, live)
    for n, live in enumerate([(0, 2), (0, 2), (0, 1, 2), (0, 2), (0, 1, 2)]):
        for one in (mine, eager):
            for k, g in enumerate(one[2]):
                g.normal_(generator=_gen(100 * n + k))
        graphs[live].replay()
        step(*eager, live)
        torch.cuda.synchronize()
        for p, q in zip(mine[0], eager[0]):
            assert torch.equal(p, q), (n, live)
    assert mine[1].param_groups[0]["steps"].tolist() == [6, 3, 6] and int(mine[1].param_groups[0]["step"]) == 6


@pytest.mark.parametrize("bits", [32, 8])
def test_counts_are_part_of_the_state(layers, bits):
    params = [torch.nn.Parameter(torch.randn(n, device=DEV, generator=_gen(n))) for n in (300, 5)]
    a = layers.AdamW(params, lr=1e-2, bits=bits)

    def step(optimiser, params, t):
        for n, p in enumerate(params):
            p.grad = torch.randn(p.shape, device=DEV, generator=_gen(10 * t + n)) if n == 0 or t > 2 else None
        optimiser.step()

    for t in range(5):
        step(a, params, t)
    saved, twins = copy.deepcopy(a.state_dict()), [torch.nn.Parameter(p.detach().clone()) for p in params]
    assert saved["param_groups"][0]["steps"] == [5, 2]
    b = layers.AdamW(twins, lr=1e-2, bits=bits)
    b.load_state_dict(saved)
    for t in range(5, 8):
        step(a, params, t)
        step(b, twins, t)
    for p, q in zip(params, twins):
        assert torch.equal(p, q)
