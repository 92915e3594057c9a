"""The optimiser layer's state: each tensor's own number of steps, float32 copies after a load, calls that are refused, groups' options.

Tolerances against a loop in 64 bits are those of a step in 32 bits: a step of one tensor is off by 20 U of its largest size (3.2 lr at most) and 3 U of the weight (U = 2^-24), and the next
steps take both over.
"""
import copy
import pickle

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


def _stepped(layers, value=1.0, steps=3):
    """A bfloat16 parameter and its optimiser, whose float32 copy is between two bfloat16 values"""
    p = torch.nn.Parameter(torch.full((300,), value, device=DEV, dtype=torch.bfloat16))
    optimiser = layers.AdamW([p], lr=1e-4, weight_decay=0.0)
    for _ in range(steps):
        p.grad = torch.ones_like(p)
        optimiser.step()
    return p, optimiser


@pytest.mark.parametrize("way", ["loaded", "copied", "pickled"])
@pytest.mark.parametrize("write", [None, "all", "some", "same"])
def test_weights_written_behind_a_load(layers, way, write):
    """A 16-bit weight that is not what its float32 copy rounds to has been written by something else: the step goes on from it.  One that is keeps its copy."""
    p, optimiser = _stepped(layers)
    if way == "loaded":
        q = torch.nn.Parameter(p.detach().clone())
        other = layers.AdamW([q], lr=1e-4, weight_decay=0.0)
        other.load_state_dict(copy.deepcopy(optimiser.state_dict()))
    else:
        q, other = copy.deepcopy((p, optimiser)) if way == "copied" else pickle.loads(pickle.dumps((p, optimiser)))
        q = other.param_groups[0]["params"][0]
    was = other.param_groups[0]["copies"][:300].clone()
    assert float(was[0]) == float(optimiser.param_groups[0]["copies"][0]) and float(was[0]) != float(q.detach()[0])
    start = was.double()
    with torch.no_grad():
        if write == "all":
            q.fill_(0.5)
            start = q.double()
        elif write == "some":
            q[7:9] = 0.25
            start = q.double()
        elif write == "same":
            q.copy_(q.clone())  # (its own values again: other weights' loading, as a checkpoint does it)
    q.grad = torch.ones_like(q)
    other.step()
    got = other.param_groups[0]["copies"][:300].double()
    # a steady gradient's step is lr: 1e-4 off by 2^-20 of itself, the copy by half a step of a value below 1
    assert float((got - (start - 1e-4)).abs().max()) <= 2.0**-25 + 1e-4 * 2.0**-20
    assert torch.equal(q.detach(), got.bfloat16())


def test_a_load_is_not_recorded(layers):
    """Behind a load the copies are compared with the weights first: not in a graph, whose replays would do it again."""
    p = torch.nn.Parameter(torch.ones(5, device=DEV, dtype=torch.bfloat16))
    optimiser = layers.AdamW([p], lr=1e-4, capturable=True)
    p.grad = torch.ones_like(p)
    optimiser.step()
    optimiser.load_state_dict(copy.deepcopy(optimiser.state_dict()))
    torch.cuda.synchronize()
    tick, refused = torch.zeros(1, device=DEV), False
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        tick.add_(1)
        try:
            optimiser.step()
        except RuntimeError as e:
            refused = "not recorded" in str(e)
    assert refused


@pytest.mark.parametrize("capturable", [False, True])
def test_a_refused_step_does_not_count(layers, capturable):
    p, q = (torch.nn.Parameter(torch.ones(300, device=DEV)) for _ in range(2))
    a, b = (layers.AdamW([x], lr=1e-2, bits=8, capturable=capturable) for x in (p, q))
    for t in range(4):
        grad = torch.randn(300, device=DEV, generator=_gen(t))
        for x in (p, q):
            x.grad = grad.clone()
        # (a rate that is no number, and a decay that is none)
        for name in ("lr", "weight_decay") if t != 1 else ():
            was = a.param_groups[0][name]
            a.param_groups[0][name] = float("nan")
            with pytest.raises(Exception):
                a.step()
            a.param_groups[0][name] = was
        p.grad = torch.ones(300, device=DEV).to_sparse()
        with pytest.raises(TypeError):
            a.step()
        p.grad = grad.clone()
        a.step()
        b.step()
        assert torch.equal(p, q) and int(a.param_groups[0]["step"]) == t + 1, t
    for name in ("m", "v", "m_scales", "v_scales"):
        assert torch.equal(a.param_groups[0][name], b.param_groups[0][name])


def test_a_step_is_recorded_whole_or_not_at_all(layers):
    """Groups of which one may not be recorded: nothing of the others is."""
    p, q = (torch.nn.Parameter(torch.ones(300, device=DEV)) for _ in range(2))
    optimiser = layers.AdamW([dict(params=[p]), dict(params=[q], capturable=False)], lr=1e-2, capturable=True)
    for x in (p, q):
        x.grad = torch.ones_like(x)
    optimiser.step()
    was, tick, refused = p.detach().clone(), torch.zeros(1, device=DEV), False
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tick.add_(1)
        try:
            optimiser.step()
        except RuntimeError as e:
            refused = "not recorded" in str(e)
    graph.replay()
    torch.cuda.synchronize()
    assert refused and torch.equal(p.detach(), was) and int(optimiser.param_groups[0]["step"]) == 1


@pytest.mark.parametrize("bits", [16, 4, 0, None, "8"])
def test_bits_of_a_group(layers, bits):
    p, q = (torch.nn.Parameter(torch.ones(3, device=DEV)) for _ in range(2))
    with pytest.raises(ValueError, match="bits"):
        layers.AdamW([dict(params=[p], bits=bits)])
    optimiser = layers.AdamW([dict(params=[p], bits=8)])
    with pytest.raises(ValueError, match="bits"):
        optimiser.add_param_group(dict(params=[q], bits=bits))
    assert len(optimiser.param_groups) == 1
    optimiser.add_param_group(dict(params=[q], bits=32))


def test_frequencies_are_constants(layers):
    """No gradient is taken of them: one that is asked for is refused."""
    f = torch.ones(4, device=DEV, dtype=torch.float64).requires_grad_()
    with pytest.raises(ValueError, match="constant"):
        layers.RotaryHeads(8, freqs=f)
    with pytest.raises(ValueError, match="constant"):
        layers.RotaryHeads(8, freqs=torch.nn.Parameter(torch.ones(4)))
    with torch.no_grad():
        layers.RotaryHeads(8, freqs=f.detach())


def test_a_load_into_16_bit_weights_makes_their_copies(layers):
    """States saved of float32 weights have no copies: a 16-bit model that loads them gets its own, and keeps small steps."""
    p = torch.nn.Parameter(torch.ones(300, device=DEV))
    a = layers.AdamW([p], lr=1e-4, weight_decay=0.0)
    p.grad = torch.ones_like(p)
    a.step()
    q = torch.nn.Parameter(torch.ones(300, device=DEV, dtype=torch.bfloat16))
    b = layers.AdamW([q], lr=1e-4, weight_decay=0.0)
    b.load_state_dict(copy.deepcopy(a.state_dict()))
    for _ in range(60):
        q.grad = torch.ones_like(q)
        b.step()
    # 60 steps of lr: 1e-4 off by 2^-20 of itself each, the copy by half a step of a value below 1
    got = b.param_groups[0]["copies"][:300].double()
    assert float((got - (1 - 60e-4)).abs().max()) <= 60 * (2.0**-25 + 1e-4 * 2.0**-20) and torch.equal(q.detach(), got.bfloat16())


def test_a_rate_in_device_memory_is_loaded_there(layers):
    """A recorded step reads its rate where it is: one that a load brought in host memory would be a constant of the graph."""
    p = torch.nn.Parameter(torch.ones(5, device=DEV))
    a = layers.AdamW([p], lr=torch.tensor(1e-2, device=DEV), weight_decay=0.0, capturable=True)
    p.grad = torch.ones_like(p)
    a.step()
    saved = copy.deepcopy(a.state_dict())
    saved["param_groups"][0]["lr"] = saved["param_groups"][0]["lr"].cpu()
    a.load_state_dict(saved)
    rate = a.param_groups[0]["lr"]
    assert rate.is_cuda and float(rate) == float(torch.tensor(1e-2))
