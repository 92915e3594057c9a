"""Rotated heads, the gated recurrence and AdamW as layers and an optimiser: through autograd, in a block with linear attention, recorded into a graph, and in the example that runs them together."""
import copy
import importlib.util
import os
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import layers as L
    return L


def _say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _near(got, ref, rel):
    assert got.shape == ref.shape
    assert (got.double() - ref).norm() <= rel * ref.norm()


def rotated(x, weight, freqs, positions, eps, interleaved):
    """The definition in 64 bits, differentiable: x [B, T, H, width]"""
    v = x if eps is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * weight
    n, angle = freqs.numel(), positions[..., None, None].double() * freqs
    a, b, rest = (v[..., 0 : 2 * n : 2], v[..., 1 : 2 * n : 2], v[..., 2 * n :]) if interleaved else (v[..., :n], v[..., n : 2 * n], v[..., 2 * n :])
    a, b = a * angle.cos() - b * angle.sin(), a * angle.sin() + b * angle.cos()
    return torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), rest], -1)


def scanned(x, f, i, state, lengths):
    """The definition in 64 bits, differentiable: (h, last)"""
    a, u = torch.sigmoid(f), torch.sigmoid(-f if i is None else i)
    h, out = state, []
    for t in range(x.shape[1]):
        here = (t < lengths)[:, None]
        h = torch.where(here, a[:, t] * h + u[:, t] * x[:, t], h)
        out.append(torch.where(here, h, 0.0))
    return torch.stack(out, 1), h


def attended(q, k, v, decay):
    T = q.shape[1]
    t = torch.arange(T, device=q.device)
    gap = t[:, None] - t
    weight = torch.where(gap >= 0, decay[:, None, None] ** gap.clamp(min=0), 0.0)
    scores = torch.einsum("bthd,bshd->bhts", q, k) * q.shape[-1] ** -0.5 * weight
    return torch.einsum("bhts,bshd->bthd", scores, v)


@pytest.mark.parametrize("eps,interleaved,keys", [(1e-5, False, True), (1e-5, True, False), (None, True, True)])
def test_rotary_heads_train(layers, eps, interleaved, keys):
    """float32: 2^-18 of the norm is 64 units of 2^-24, what a row may be off by"""
    g = _gen(1)
    layer = layers.RotaryHeads(24, rotary=16, eps=eps, interleaved=interleaved)
    if eps is not None:
        with torch.no_grad():
            layer.q_weight.add_(0.3 * torch.randn(24, device=DEV, generator=g))
            layer.k_weight.add_(0.3 * torch.randn(24, device=DEV, generator=g))
    q, k = torch.randn(2, 9, 4, 24, device=DEV, generator=g).requires_grad_(), torch.randn(2, 9, 2, 24, device=DEV, generator=g).requires_grad_()
    positions = torch.randint(0, 1000, (2, 9), device=DEV, generator=g).to(torch.int32)
    out = layer(q, k, positions=positions) if keys else (layer(q, positions=positions),)
    gouts = [torch.randn(o.shape, device=DEV, generator=g) for o in out]
    torch.autograd.backward(out, gouts)
    q64, k64, wq, wk = (t if t is None else t.detach().double().requires_grad_() for t in (q, k, layer.q_weight, layer.k_weight))
    want = [rotated(q64, wq, layer._freqs, positions, eps, interleaved)] + ([rotated(k64, wk, layer._freqs, positions, eps, interleaved)] if keys else [])
    torch.autograd.backward(want, [x.double() for x in gouts])
    for a, b in zip(out, want):
        _near(a, b.detach(), 2.0**-18)
    _near(q.grad, q64.grad, 2.0**-18)
    if keys:
        _near(k.grad, k64.grad, 2.0**-18)
    else:
        assert k.grad is None and (eps is None or layer.k_weight.grad is None)
    if eps is not None:
        _near(layer.q_weight.grad, wq.grad, 2.0**-18)
        if keys:
            _near(layer.k_weight.grad, wk.grad, 2.0**-18)
    # one of the outputs alone
    if keys:
        gk, = torch.autograd.grad(layer(q, k, positions=positions)[1], k, gouts[1])
        _near(gk, k64.grad, 2.0**-18)


@pytest.mark.parametrize("gated", [False, True])
def test_gated_recurrence_trains(layers, gated):
    """float32, 70 frames: 20 (70 + 10) units of 2^-24 at most"""
    g = _gen(2)
    layer = layers.GatedRecurrence()
    x, f, i = (torch.randn(3, 70, 20, device=DEV, generator=g).requires_grad_() for _ in range(3))
    i = i if gated else None
    state = torch.randn(3, 20, device=DEV, generator=g).requires_grad_()
    lengths = torch.tensor([70, 0, 33], dtype=torch.int32, device=DEV)
    leaves = [t for t in (x, f, i, state) if t is not None]
    h, last = layer(x, f, i, state=state, lengths=lengths, return_state=True)
    gout, glast = torch.randn(h.shape, device=DEV, generator=g), torch.randn(last.shape, device=DEV, generator=g)
    got = torch.autograd.grad((h, last), leaves, (gout, glast))
    twins = [t.detach().double().requires_grad_() for t in leaves]
    by = iter(twins)
    wh, wlast = scanned(next(by), next(by), next(by) if gated else None, next(by), lengths)
    want = torch.autograd.grad((wh, wlast), twins, (gout.double(), glast.double()))
    for a, b in zip((h, last, *got), (wh.detach(), wlast.detach(), *want)):
        _near(a, b, 1600 * 2.0**-24)
    # each output alone; without a state
    for n, out in ((0, gout), (1, glast)):
        a = torch.autograd.grad(layer(x, f, i, state=state, lengths=lengths, return_state=True)[n], leaves, out)
        b = torch.autograd.grad(scanned(*twins[:2], twins[2] if gated else None, twins[-1], lengths)[n], twins, out.double(), allow_unused=True)
        for p, q in zip(a, b):
            _near(p, q, 1600 * 2.0**-24)
    assert torch.equal(layer(x, f, i), layer(x, f, i, state=torch.zeros_like(state)))


def test_a_block_of_them(layers):
    """Norm, rotation, linear attention and the recurrence after one another, and two optimiser steps, against the same in 64 bits: some two hundred roundings of 2^-24 a value, the worst of them
    in the gates' sums over 50 frames; an AdamW step's size is at most 3.2 lr whatever the gradient, so weights are held to that times what the gradients are off by."""
    g = _gen(3)
    B, T, H, d = 2, 50, 2, 16
    W = 2 * H * d
    norm, turn, mix, remember = layers.LayerNorm(W), layers.RotaryHeads(d, rotary=8), layers.DecayAttention(H), layers.GatedRecurrence()
    params = [torch.nn.Parameter(torch.randn(W, 3 * H * d + 2 * W, device=DEV, generator=g) * W**-0.5), norm.weight, norm.bias, turn.q_weight, turn.k_weight]
    x = torch.randn(B, T, W, device=DEV, generator=g)
    gout = torch.randn(B, T, H * d + W, device=DEV, generator=g)
    optimiser = layers.AdamW(params, lr=1e-2, weight_decay=0.1)
    twins = [p.detach().double().requires_grad_() for p in params]
    other = torch.optim.AdamW(twins, lr=1e-2, weight_decay=0.1, foreach=False)

    def run():
        y = norm(x) @ params[0]
        q, k, v = (t.unflatten(-1, (H, d)) for t in y[..., : 3 * H * d].chunk(3, -1))
        q, k = turn(q, k, offset=7)
        return torch.cat([mix(q, k, v).flatten(-2), remember(*y[..., 3 * H * d :].chunk(2, -1))], -1)

    def definition():
        w, nw, nb, wq, wk = twins
        v = x.double()
        h = (v - v.mean(-1, keepdim=True)) / (v.var(-1, correction=0, keepdim=True) + norm.eps).sqrt() * nw + nb
        y = h @ w
        q, k, v = (t.unflatten(-1, (H, d)) for t in y[..., : 3 * H * d].chunk(3, -1))
        at = torch.arange(T, device=DEV).expand(B, T) + 7
        q, k = rotated(q, wq, turn._freqs, at, 1e-6, False), rotated(k, wk, turn._freqs, at, 1e-6, False)
        a, f = y[..., 3 * H * d :].chunk(2, -1)
        return torch.cat([attended(q, k, v, mix.decay.double()).flatten(-2), scanned(a, f, None, torch.zeros(B, W, dtype=torch.float64, device=DEV), torch.tensor([T] * B, device=DEV))[0]], -1)

    for step in range(2):
        out, want = run(), definition()
        _near(out, want.detach(), 2e-5)
        optimiser.zero_grad()
        other.zero_grad()
        out.backward(gout)
        want.backward(gout.double())
        for p, t in zip(params, twins):
            _near(p.grad, t.grad, 2e-5)
        optimiser.step()
        other.step()
        for p, t in zip(params, (t.detach() for t in twins)):
            # (a first step is lr times the gradient's sign, but for those near eps: 1e-8 beside gradients off by 1e-5)
            assert float((p.detach().double() - t).norm()) <= 1e-3 * 1e-2 * t.numel() ** 0.5


def test_second_derivatives_and_forward_mode_are_refused(layers):
    from torch.autograd import forward_ad
    turn, bare, scan = layers.RotaryHeads(8), layers.RotaryHeads(8, eps=None), layers.GatedRecurrence()
    q = torch.randn(1, 5, 2, 8, device=DEV).requires_grad_()
    x = torch.randn(1, 5, 8, device=DEV).requires_grad_()
    w = torch.ones((), device=DEV).requires_grad_()
    for call, t in ((lambda t: turn(t), q), (lambda t: turn(t, t)[1], q), (lambda t: scan(t, t), x), (lambda t: scan(x.detach(), t), x)):
        gx, = torch.autograd.grad(call(t * w).square().sum(), t, create_graph=True)
        with pytest.raises(RuntimeError, match="no second derivative"):
            gx.square().sum().backward()
    # linear calls' gradients are constants: those have a derivative, and it is theirs
    for call, t in ((lambda t: bare(t), q), (lambda t: scan(t, x.detach(), x.detach()), x)):
        gx, = torch.autograd.grad(call(t * w).sum(), t, create_graph=True)
        gw, = torch.autograd.grad(gx.sum(), w)
        assert torch.allclose(gw, gx.detach().sum(), rtol=1e-4, atol=1e-4)
    state = torch.zeros(1, 8, device=DEV)
    with forward_ad.dual_level():
        dual_q, dual_x, dual_s = (forward_ad.make_dual(t.detach(), torch.ones_like(t)) for t in (q, x, state))
        for call in (lambda: turn(dual_q), lambda: bare(dual_q), lambda: scan(dual_x, x.detach()), lambda: scan(x.detach(), dual_x), lambda: scan(x.detach(), x.detach(), state=dual_s),
                     lambda: scan.step(dual_x[:, 0], x[:, 0].detach(), state), lambda: scan.step(x[:, 0].detach(), x[:, 0].detach(), dual_s)):
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises((NotImplementedError, RuntimeError)):
                    call()


def test_what_is_changed_before_a_backward_pass_is_noticed(layers):
    turn, scan = layers.RotaryHeads(8), layers.GatedRecurrence()
    for make in ("q", "positions", "f", "lengths", "step"):
        q = torch.randn(1, 5, 2, 8, device=DEV).requires_grad_() * 1
        positions, lengths = torch.arange(5, device=DEV, dtype=torch.int32)[None].clone(), torch.tensor([5], dtype=torch.int32, device=DEV)
        x, f = (torch.randn(1, 5, 8, device=DEV).requires_grad_() * 1 for _ in range(2))
        state = torch.zeros(1, 8, device=DEV)
        out = turn(q, positions=positions).sum() + scan(x, f, lengths=lengths).sum() + (state * x[:, 0]).sum()
        with torch.no_grad():
            if make == "step":
                scan.step(x[:, 0], f[:, 0], state)
            else:
                dict(q=q, positions=positions, f=f, lengths=lengths)[make].add_(1)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.backward()


def test_layers_refuse(layers):
    with pytest.raises(ValueError):
        layers.RotaryHeads(8, rotary=7)
    with pytest.raises(ValueError):
        layers.RotaryHeads(8, rotary=10)
    with pytest.raises(ValueError):
        layers.RotaryHeads(8)(torch.zeros(1, 2, 3, 9, device=DEV))
    with pytest.raises(RuntimeError, match="no derivative"):
        x = torch.zeros(1, 8, device=DEV).requires_grad_()
        layers.GatedRecurrence().step(x, x, torch.zeros(1, 8, device=DEV))
    p = torch.nn.Parameter(torch.zeros(4, 6, device=DEV))
    for bad in (dict(params=[torch.nn.Parameter(torch.zeros(3))]), dict(params=[torch.nn.Parameter(p.detach().t())]), dict(params=[torch.nn.Parameter(p.detach().double())]), dict(params=[p], bits=4)):
        with pytest.raises(ValueError):
            layers.AdamW(**bad)
    half = layers.RotaryHeads(8).bfloat16()  # (the weights are the norm's, in float32; the angles are no parameters)
    assert half._freqs.dtype == torch.float64
    with pytest.raises(TypeError):
        half(torch.zeros(1, 2, 3, 8, device=DEV))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_goes_on_from_its_state(layers, bits):
    """state_dict and back, groups of different rates, gradients that are missing or lie otherwise, a schedule."""
    g = _gen(5)
    shapes = [(40, 30), (7,), (300,)]
    kinds = [torch.float32, torch.bfloat16, torch.float16]
    params = [torch.nn.Parameter(torch.randn(s, device=DEV, generator=g).to(t)) for s, t in zip(shapes, kinds)]

    def make(params):
        return layers.AdamW([dict(params=params[:2], lr=1e-2), dict(params=params[2:], weight_decay=0.0)], lr=1e-3, bits=bits)

    a = make(params)
    schedule = torch.optim.lr_scheduler.StepLR(a, 2, 0.5)

    def step(optimiser, params, n):
        for k, p in enumerate(params):
            grad = torch.randn(p.shape[::-1], device=DEV, generator=_gen(100 * n + k)).to(p.dtype)
            p.grad = grad.t() if p.dim() == 2 else grad
            if k == 2 and n == 1:
                p.grad = None
        optimiser.step()

    for n in range(3):
        step(a, params, n)
        schedule.step()
    saved, at = copy.deepcopy(a.state_dict()), [p.detach().clone() for p in params]
    assert saved["param_groups"][0]["step"] == 3 and saved["param_groups"][1]["step"] == 2
    for n in range(3, 6):
        step(a, params, n)
    twins = [torch.nn.Parameter(p) for p in at]
    b = make(twins)
    b.load_state_dict(saved)
    b.param_groups[0]["lr"] = torch.tensor(b.param_groups[0]["lr"], dtype=torch.float64)  # (in host memory: read as a number)
    for n in range(3, 6):
        step(b, twins, n)
    for p, q in zip(params, twins):
        assert torch.equal(p, q)
    for x, y in zip(a.param_groups, b.param_groups):
        for name in ("m", "v", "m_scales", "v_scales", "copies"):
            assert (x[name] is None and y[name] is None) or torch.equal(x[name], y[name])


def test_small_steps_of_16_bit_weights_are_not_lost(layers):
    """A thousand steps of 10^-5 on a bfloat16 one, whose own distance is 2^-8: with a float32 copy they are there; a weight that something else writes starts from there."""
    for master, want in ((True, 0.99), (False, 1.0)):
        p = torch.nn.Parameter(torch.ones(5, device=DEV, dtype=torch.bfloat16))
        optimiser = layers.AdamW([p], lr=1e-5, weight_decay=0.0, master=master)
        for _ in range(1000):
            p.grad = torch.ones_like(p)
            optimiser.step()
        assert float(p.detach()[0]) == float(torch.tensor(want).bfloat16())
        with torch.no_grad():
            p.fill_(0.5)
        p.grad = torch.ones_like(p)
        optimiser.step()
        assert float(p.detach()[0]) == 0.5


@pytest.mark.parametrize("case", ["first", "counted", "written", "fine"])
def test_what_may_not_be_recorded(layers, case):
    """A first step would zero its states in each replay, one counted in host memory repeat its number, and one behind a write take the float32 copies from rounded weights."""
    p = torch.nn.Parameter(torch.ones(5, device=DEV, dtype=torch.bfloat16))
    p.grad = torch.ones_like(p)
    optimiser = layers.AdamW([p], lr=1e-5, weight_decay=0.0, capturable=case != "counted")
    if case != "first":
        optimiser.step()
    if case == "written":
        with torch.no_grad():
            p.fill_(1.0)
    tick = torch.zeros(1, device=DEV)
    torch.cuda.synchronize()
    graph, refused = torch.cuda.CUDAGraph(), False
    with torch.cuda.graph(graph):
        tick.add_(1)
        try:
            optimiser.step()
        except RuntimeError as e:
            refused = "not recorded" in str(e)
    assert refused == (case != "fine")
    if case == "first":
        assert "m" not in optimiser.param_groups[0]
        return
    if case == "written":
        optimiser.step()
        with torch.cuda.graph(graph := torch.cuda.CUDAGraph()):
            optimiser.step()
    if case in ("written", "fine"):
        before = optimiser.param_groups[0]["copies"][:5].clone()
        for n in range(3):  # steps of 1e-5, which a bfloat16 one would lose
            graph.replay()
            torch.cuda.synchronize()
            moved = (before - optimiser.param_groups[0]["copies"][:5]).double()
            # (a float32 below one holds its value to 2^-25 and a step is off by 2^-20 of itself: each of them)
            assert float((moved - (n + 1) * 1e-5).abs().max()) <= (n + 1) * (2.0**-25 + 2.0**-20 * 1e-5) + 2.0**-25


def test_the_kernels_of_a_transform_are_trained(layers):
    """The library's own copy of a layer's weights follows the steps."""
    layer = layers.STFT(n_fft=256, hop_length=64, trainable=True, output_format="Power")
    optimiser = layers.AdamW(layer.parameters(), lr=1e-2)
    wave = torch.randn(2, 2000, device=DEV, generator=_gen(6))
    before = layer(wave)
    before.sum().backward()
    optimiser.step()
    after = layer(wave).detach()
    fresh = layers.STFT(n_fft=256, hop_length=64, trainable=True, output_format="Power")
    with torch.no_grad():
        fresh.wsin_wcos.copy_(layer.wsin_wcos)
    assert not torch.equal(after, before) and torch.equal(after, fresh(wave))


RECORDED = """
import torch
from paper_1912_12055_amd import layers
g = torch.Generator(device="cuda:0").manual_seed(1)
def make():
    torch.manual_seed(0)
    w = torch.nn.Parameter(torch.randn(32, 5 * 32, device="cuda:0", dtype=torch.bfloat16) * 32 ** -0.5)
    turn, mix, scan = layers.RotaryHeads(16), layers.DecayAttention(2), layers.GatedRecurrence()
    optimiser = layers.AdamW([w, *turn.parameters()], lr=torch.tensor(1e-2, device="cuda:0"), bits=8, capturable=True)
    def step(x):
        y = x @ w
        q, k, v = (t.unflatten(-1, (2, 16)) for t in y[..., :96].chunk(3, -1))
        q, k = turn(q, k)
        out = mix(q, k, v).flatten(-2) + scan(*y[..., 96:].chunk(2, -1))
        loss = out.float().square().mean()
        optimiser.zero_grad(set_to_none=True)
        loss.backward()
        optimiser.step()
        return loss.detach()
    return step, [w, *turn.parameters()], optimiser
x = torch.randn(2, 400, 32, device="cuda:0", generator=g).bfloat16()
step, params, optimiser = make()
side = torch.cuda.Stream()
side.wait_stream(torch.cuda.current_stream())
with torch.cuda.stream(side):
    step(x)
torch.cuda.current_stream().wait_stream(side)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    loss = step(x)
eager, twins, other = make()
eager(x)
for n in range(4):
    x.copy_(torch.randn(x.shape, device="cuda:0", generator=g))
    for o in (optimiser, other):
        o.param_groups[0]["lr"].fill_(1e-2 / (n + 1))
    graph.replay()
    torch.cuda.synchronize()
    want = eager(x)
    assert torch.equal(loss, want), (n, loss, want)
    assert all(torch.equal(a, b) for a, b in zip(params, twins)), n
    assert int(optimiser.param_groups[0]["step"]) == n + 2
print("the same")
"""


def test_a_training_step_recorded_into_a_graph(layers):
    """Forward, backward and the optimiser's step, replayed with other inputs and rates, against the same steps run one by one."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", RECORDED], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0 and "the same" in done.stdout, done.stderr[-2000:]


def test_the_example_runs_and_streams(layers):
    path = os.path.join(os.path.dirname(__file__), "..", "examples")
    sys.path.insert(0, path)
    try:
        spec = importlib.util.spec_from_file_location("frame_recurrence", os.path.join(path, "frame_recurrence.py"))
        example = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(example)
    finally:
        sys.path.remove(path)
    torch.manual_seed(0)
    model = example.RecurrentFrameModel()
    before = [p.detach().clone() for p in model.parameters()]
    losses = example.train(model, 3)
    assert all(v == v and v < 100 for v in losses)
    for p, b in zip(model.parameters(), before):
        assert p.grad is not None and p.grad.isfinite().all() and not torch.equal(p, b)
    with torch.no_grad():
        wave, _, _ = example.clips(3, _gen(7), seconds=1.0)
        tokens = model.tokens(wave)
        whole, states = model(tokens)
    assert all(s.isfinite().all() for s in states)
    # bfloat16 weights and states in one, float32 states in the other: a few roundings of 2^-9 between them
    assert (example.stream(model, tokens, prompt=17) - whole).norm() <= 0.02 * whole.norm()
