"""The layers of networks on the transforms' frames through autograd, products kept in 8 bits, and the example that runs them together."""
import importlib.util
import os
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


@pytest.mark.parametrize("kind", ["rows", "frames", "every other", "bfloat16"])
def test_layer_norm_layer_trains(layers, kind):
    """gradients of weight, bias and input against the same in 64 bits (float32: sums of a few thousand terms, 2^-24 each at most; 2^-8 for bfloat16)"""
    _say("LayerNorm", kind)
    g = _gen(1)
    layer = layers.LayerNorm(60)
    with torch.no_grad():
        layer.weight.add_(0.3 * torch.randn(60, device=DEV, generator=g))
        layer.bias.add_(torch.randn(60, device=DEV, generator=g))
    base = torch.randn(4, 60, 70, device=DEV, generator=g).requires_grad_()
    view = {"rows": lambda t: t.transpose(1, 2).contiguous(), "frames": lambda t: t.transpose(1, 2), "every other": lambda t: t.transpose(1, 2)[:, ::2],
            "bfloat16": lambda t: t.transpose(1, 2).contiguous().bfloat16()}[kind]
    y = layer(view(base))
    assert y.is_contiguous()
    gout = torch.randn(y.shape, device=DEV, generator=g).to(y.dtype)
    y.backward(gout)
    x64, w64, b64 = base.detach().double().requires_grad_(), layer.weight.detach().double().requires_grad_(), layer.bias.detach().double().requires_grad_()
    v = view(x64) if kind != "bfloat16" else x64.transpose(1, 2).float().bfloat16().double()
    m = v.mean(-1, keepdim=True)
    ref = (v - m) / ((v - m).square().mean(-1, keepdim=True) + layer.eps).sqrt() * w64 + b64
    ref.backward(gout.double())
    rel = 2.0**-8 if kind == "bfloat16" else 1e-5
    for got, want in ((y, ref.detach()), (base.grad, x64.grad), (layer.weight.grad, w64.grad), (layer.bias.grad, b64.grad)):
        _near(got, want, rel)


def test_layer_norm_layer_that_keeps_8_bits(layers):
    from paper_1912_12055_amd import binding as nb
    g = _gen(2)
    x = torch.randn(50, 300, device=DEV, generator=g).requires_grad_()
    full, small = layers.LayerNorm(300), layers.LayerNorm(300, kept_bits=8)
    gout = torch.randn(50, 300, device=DEV, generator=g)
    grads = []
    for layer in (full, small):
        x.grad = None
        layer(x).backward(gout)
        grads.append((x.grad.clone(), layer.weight.grad.clone(), layer.bias.grad.clone()))
    y, kept = nb.nna_layer_norm(x.detach(), small.weight.detach(), small.bias.detach(), keep=8)
    for a, b in zip(grads[1], nb.nna_layer_norm_backward(gout, kept, small.weight.detach())):
        assert torch.equal(a, b)
    # h is off by at most a / 254 of r, a the largest of 128 values: below 1/40 for these; gw follows it, gx by its part along h alone
    assert (grads[1][1] - grads[0][1]).abs().max() <= (gout.abs() / 40).sum(0).max() and torch.equal(grads[1][2], grads[0][2])
    assert (grads[1][0] - grads[0][0]).norm() <= 0.02 * grads[0][0].norm()
    with torch.no_grad():
        assert torch.equal(small(x), full(x))
    frames = torch.randn(2, 300, 33, device=DEV, generator=g)
    assert torch.allclose(small(frames.transpose(1, 2).requires_grad_()), full(frames.transpose(1, 2)), rtol=1e-4, atol=1e-5)  # rows are made of them


def test_an_input_changed_before_its_backward_pass_is_noticed(layers):
    x = torch.randn(8, 64, device=DEV)
    layer = layers.LayerNorm(64)
    y = layer(x)
    x.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_decay_attention_layer_trains(layers):
    _say("DecayAttention")
    g = _gen(3)
    B, T, H, dk, dv = 2, 90, 3, 32, 40
    layer = layers.DecayAttention(H)
    proj = torch.randn(B, T, H * (dk + dv), device=DEV, generator=g).requires_grad_()
    k1 = torch.randn(B, T, 1, dk, device=DEV, generator=g).requires_grad_()  # keys that the heads share
    state = torch.randn(B, H, dk, dv, device=DEV, generator=g).requires_grad_()
    lengths = torch.tensor([90, 37], dtype=torch.int32, device=DEV)

    def inputs(p, k):
        return p[..., :H * dk].unflatten(-1, (H, dk)), k.expand(B, T, H, dk), p[..., H * dk:].unflatten(-1, (H, dv))

    o, last = layer(*inputs(proj, k1), state=state, lengths=lengths, return_state=True)
    go, gl = torch.randn(o.shape, device=DEV, generator=g), torch.randn(last.shape, device=DEV, generator=g)
    (o * go).sum().add((last * gl).sum()).backward()
    p64, k64, s64 = (t.detach().double().requires_grad_() for t in (proj, k1, state))
    q, k, v = inputs(p64, k64)
    S, outs, lasts, loss = s64, [], [None] * B, 0.0
    for t in range(T):
        S = layer.decay.double()[:, None, None] * S + k[:, t, :, :, None] * v[:, t, :, None, :]
        ot = (q[:, t, :, :, None] * S).sum(-2) * dk**-0.5
        here = (t < lengths).double()[:, None, None]
        loss = loss + (ot * here * go[:, t].double()).sum()
        for b in range(B):
            if t + 1 == int(lengths[b]):
                loss = loss + (S[b] * gl[b].double()).sum()
    loss.backward()
    for got, want in ((proj.grad, p64.grad), (k1.grad, k64.grad), (state.grad, s64.grad)):
        _near(got, want, 1e-5)
    # the outputs alone, and the last state alone
    proj.grad = None
    layer(*inputs(proj, k1)).sum().backward()
    assert proj.grad.abs().sum() > 0
    proj.grad = None
    layer(*inputs(proj, k1), return_state=True)[1].sum().backward()
    assert not proj.grad[..., :H * dk].any() and proj.grad[..., H * dk:].abs().sum() > 0


def test_layers_refuse(layers):
    q = torch.randn(1, 4, 2, 8, device=DEV)
    mix = layers.DecayAttention(2)
    state = torch.zeros(1, 2, 8, 8, device=DEV)
    with pytest.raises(RuntimeError):
        mix.step(q[:, 0].clone().requires_grad_(), q[:, 0], q[:, 0], state)
    for bad in (lambda: layers.DecayAttention(2, decay=[0.5]), lambda: layers.DecayAttention(2, decay=[0.5, 1.5]), lambda: layers.DecayAttention(1, decay=[float("nan")]),
                lambda: layers.DecayAttention(1, decay=torch.tensor([0.5], requires_grad=True)), lambda: layers.LayerNorm(8, kept_bits=4),
                lambda: layers.LayerNorm(9)(q), lambda: layers.STFT(n_fft=256, hop_length=64, trainable=True, kept_bits=16),
                lambda: layers.LayerNorm(8, device="cpu")):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.parametrize("make", [lambda L, b: L.STFT(n_fft=512, hop_length=128, trainable=True, output_format="Power", kept_bits=b),
                                  lambda L, b: L.MelSpectrogram(sr=16000, n_fft=512, hop_length=128, n_mels=40, trainable_mel=True, trainable_STFT=True, kept_bits=b),
                                  lambda L, b: L.CQT1992v2(sr=16000, hop_length=128, fmin=220.0, n_bins=24, trainable=True, output_format="Power", kept_bits=b)])
def test_trainable_layers_that_keep_their_products_in_8_bits(layers, make):
    """The outputs are the same; the gradients those of products off by at most 1/254 of the largest of 128: sqrt(128) / 254 < 0.045 of a block's norm."""
    g = _gen(4)
    x = (0.3 * torch.randn(3, 9001, device=DEV, generator=g)).requires_grad_()
    outs, grads, held = [], [], []
    for bits in (32, 8):
        layer = make(layers, bits)
        _say(type(layer).__name__, bits)
        x.grad = None
        y = layer(x)
        held.append(sum(t.numel() * t.element_size() for t in y.grad_fn.saved_tensors) - x.numel() * 4)
        gout = torch.randn(y.shape, device=DEV, generator=_gen(5))
        y.backward(gout)
        outs.append(y.detach())
        grads.append([x.grad.clone()] + [p.grad.clone() for p in layer.parameters()])
    assert torch.equal(*outs)
    assert 0 < held[1] <= held[0] * (1 / 4 + 1 / 128) + 64
    for a, b in zip(*grads):
        assert torch.isfinite(b).all() and 0 < (a - b).norm() <= 0.045 * a.norm()


def test_the_example_learns_and_streams(layers):
    spec = importlib.util.spec_from_file_location("frame_model", os.path.join(os.path.dirname(__file__), "..", "examples", "frame_model.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    torch.manual_seed(0)
    model = example.FrameModel()
    losses = example.train(model, 25)
    _say("losses", losses[0], losses[-1])
    assert losses[-1] < 0.5 * losses[0]
    with torch.no_grad():
        wave, _, _ = example.clips(3, _gen(7), seconds=1.0)
        tokens = model.tokens(wave)
        whole, state = model(tokens)
    assert torch.isfinite(state).all()
    # bfloat16 weights and states in one, float32 states in the other: a few roundings of 2^-9 between them
    assert (example.stream(model, tokens, prompt=17) - whole).norm() <= 0.02 * whole.norm()


def test_what_the_calls_write_in_place_is_noticed(layers):
    """A tensor that a recorded call holds for its backward pass, written by a later call through its pointer: a state by `step`, outputs that are given."""
    from paper_1912_12055_amd import binding as nb
    g = _gen(8)
    q = torch.randn(2, 6, 2, 16, device=DEV, generator=g).requires_grad_()
    mix, state = layers.DecayAttention(2), torch.randn(2, 2, 16, 16, device=DEV, generator=g)
    o = mix(q, q, q, state=state)
    with torch.no_grad():
        mix.step(q[:, 0], q[:, 0], q[:, 0], state)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()
    for inference in (False, True):  # nothing else changes
        with torch.inference_mode(inference):
            s = torch.zeros(2, 2, 16, 16, device=DEV)
            mix.step(q[:, 0].detach(), q[:, 0].detach(), q[:, 0].detach(), s)
            assert s.any()

    x = torch.randn(5, 16, device=DEV, generator=g).requires_grad_()
    codes, scales = nb.nna_pack8(x.detach())
    for write in (lambda out: nb.nna_layer_norm(x.detach(), out=out), lambda out: nb.nna_unpack8(codes, scales, out=out),
                  lambda out: nb.nna_decay_attention(*3 * [out.new_ones(1, 5, 1, 16)], mix.decay[:1], out=out.view(1, 5, 1, 16)),
                  lambda out: nb.nna_decay_attention_step(*3 * [out.new_ones(5, 1, 16)], mix.decay[:1], out.new_zeros(5, 1, 16, 16), out=out.view(5, 1, 16))):
        held = torch.randn(5, 16, device=DEV, generator=g)
        y = (x * held).sum()
        write(held)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    layer = layers.STFT(n_fft=512, hop_length=128, trainable=True, output_format="Power")
    wave = torch.randn(2, 4000, device=DEV, generator=g)
    kept = torch.zeros(nb.nna_kept_bytes(layer.plan, 2, 4000), dtype=torch.uint8, device=DEV)
    nb.nna_forward_keep(layer.plan, wave, kept=kept)
    assert kept._version == 1


def test_results_are_memory_of_the_stream_they_are_written_on(layers):
    """With a stream's handle: what a call allocates is that stream's (memory that torch's current stream has freed and may still read is not written), and is
    not handed out again while the current stream, which gets it, is still at work."""
    from paper_1912_12055_amd import binding as nb
    g = _gen(9)
    x, w = torch.randn(4096, 512, device=DEV, generator=g), torch.ones(512, device=DEV)
    spec = torch.randn(2, 64, 300, device=DEV, generator=g)
    q = torch.randn(2, 3000, 4, 64, device=DEV, generator=g)
    decay, first = torch.full((4,), 0.9, device=DEV), torch.randn(2, 4, 64, 64, device=DEV, generator=g)
    side = torch.cuda.Stream()

    def calls(stream, state):
        y, kept = nb.nna_layer_norm(x, w, keep=8, stream=stream)
        f, kf = nb.nna_layer_norm(spec.transpose(1, 2), keep=32, stream=stream)
        out = [y, kept.stats, kept.codes, kept.scales, f, kf.stats, *nb.nna_layer_norm_backward(x, kept, w, stream=stream), *nb.nna_layer_norm_backward(f, kf, stream=stream)]
        codes, scales = nb.nna_pack8(x, stream=stream)
        out += [codes, scales, nb.nna_unpack8(codes, scales, stream=stream)]
        out += nb.nna_decay_attention(q, q, q, decay, state=first, want_state=True, stream=stream)
        out += nb.nna_decay_attention_backward(q, q, q, q, decay, state=first, gstate=first, want_gstate=True, stream=stream)
        return out + [nb.nna_decay_attention_step(q[:, 0], q[:, 0], q[:, 0], decay, state, stream=stream)]

    states = first.clone(), first.clone()
    ref = [t.clone() for t in calls(None, states[0])]
    torch.cuda.synchronize()
    out = calls(side.cuda_stream, states[1])
    torch.cuda.synchronize()
    segments = torch.cuda.memory_snapshot()
    for k, (a, b) in enumerate(zip(out, ref)):
        assert torch.equal(a, b), k
        owner = [s["stream"] for s in segments if s["address"] <= a.data_ptr() < s["address"] + s["total_size"]]
        assert owner == [side.cuda_stream], k
    assert torch.equal(*states)
    y = nb.nna_layer_norm(x, w, stream=side.cuda_stream)
    at, size = y.data_ptr(), y.numel()
    torch.cuda.current_stream().wait_stream(side)
    a = torch.randn(8192, 8192, device=DEV, generator=g)
    torch.cuda.synchronize()
    for _ in range(10):
        a = a @ a  # the current stream is busy, and has y to read after it
    z = y.sum()
    del y
    with torch.cuda.stream(side):
        again = torch.empty(size, device=DEV)
    busy = not torch.cuda.current_stream().query()
    assert not busy or again.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.isfinite(z)


def _penalty(call, x, weight):
    """the gradient of a call behind a product with `weight`, differentiated"""
    y = call(x * weight)
    gx, = torch.autograd.grad(y.square().sum(), x, create_graph=True)
    return gx


@pytest.mark.parametrize("kind", ["norm", "norm without weights", "attention", "state", "stft", "mel", "cqt", "complex"])
def test_a_second_derivative_is_refused(layers, kind):
    """Not left out: the gradients themselves are right under create_graph, and differentiating them raises."""
    g = _gen(10)
    mix = layers.DecayAttention(2)
    zeros = torch.zeros(2, 2, 16, 16, device=DEV)
    call, shape = {
        "norm": (layers.LayerNorm(16), (4, 16)), "norm without weights": (layers.LayerNorm(16, affine=False), (4, 16)),
        "attention": (lambda h: mix(h, h, h), (2, 6, 2, 16)), "state": (lambda h: mix(h.detach(), h.detach(), h.detach(), state=zeros + h.sum()), (2, 6, 2, 16)),
        "stft": (layers.STFT(n_fft=512, hop_length=128, trainable=True, output_format="Power"), (1, 2000)),
        "mel": (layers.MelSpectrogram(sr=16000, n_fft=512, hop_length=128, n_mels=40, trainable_STFT=True), (1, 2000)),
        "cqt": (layers.CQT1992v2(sr=16000, hop_length=128, fmin=440.0, n_bins=12, trainable=True), (1, 4000)),
        "complex": (layers.STFT(n_fft=512, hop_length=128, trainable=True, output_format="Complex"), (1, 2000))}[kind]
    _say("second derivative", kind)
    x = torch.randn(shape, device=DEV, generator=g).requires_grad_()
    weight = torch.ones((), device=DEV).requires_grad_()
    gx = _penalty(call, x, weight)
    y = call(x * weight)
    first, = torch.autograd.grad(y.square().sum(), x)
    assert (gx.detach() - first).norm() <= 1e-5 * first.norm()  # (the transforms' sums in another order: some units of 2^-24)
    with pytest.raises(RuntimeError, match="no second derivative"):
        gx.square().sum().backward()


def test_gradients_that_are_constants_stay_constants(layers):
    """A gradient that depends on nothing with a gradient of its own has no second derivative to leave out."""
    g = _gen(11)
    q, k, v = (torch.randn(2, 6, 2, 16, device=DEV, generator=g) for _ in range(3))
    first, w = torch.randn(2, 2, 16, 16, device=DEV, generator=g), torch.full((), 3.0, device=DEV).requires_grad_()
    mix, norm = layers.DecayAttention(2), layers.LayerNorm(16)
    stft = layers.STFT(n_fft=512, hop_length=128, trainable=True, output_format="Complex")
    stft.wsin_wcos.requires_grad_(False)
    wave = torch.randn(1, 2000, device=DEV, generator=g)
    for call, x in ((lambda t: mix(q, k, t, state=first), v), (lambda t: mix(t, k, v), q), (lambda t: mix(q, t, v), k), (stft, wave)):
        x = x.clone().requires_grad_()
        gx, = torch.autograd.grad(call(x * w).sum(), x, create_graph=True)  # w times a constant
        plain = x.detach().requires_grad_()
        c, = torch.autograd.grad(call(plain).sum(), plain)
        gw, = torch.autograd.grad(gx.sum(), w)
        assert torch.allclose(gw, c.sum(), rtol=1e-5, atol=1e-5 * float(c.abs().sum()))
    y = norm(q)
    grads = torch.autograd.grad(y.sum(), (norm.weight, norm.bias), create_graph=True)
    assert not any(t.requires_grad for t in grads)


def test_forward_mode_is_refused(layers):
    """a dual tensor's tangent is not dropped"""
    from torch.autograd import forward_ad
    g = _gen(12)
    q = torch.randn(2, 6, 2, 16, device=DEV, generator=g)
    state = torch.zeros(2, 2, 16, 16, device=DEV)
    mix, norm, bare = layers.DecayAttention(2), layers.LayerNorm(16), layers.LayerNorm(16, affine=False)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(q, torch.ones_like(q))
        dual_state = forward_ad.make_dual(state, torch.ones_like(state))
        for call in (lambda: bare(dual), lambda: norm(dual), lambda: mix(dual, q, q), lambda: mix(q, q, dual), lambda: mix(q, q, q, state=dual_state),
                     lambda: mix.step(dual[:, 0], q[:, 0], q[:, 0], state), lambda: mix.step(q[:, 0], q[:, 0], q[:, 0], dual_state)):
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises((NotImplementedError, RuntimeError)):
                    call()
        assert not state.any()
        with torch.no_grad():  # others are as ever
            assert mix(q, q, q).shape == norm(q).shape == q.shape


@pytest.mark.parametrize("bins", [2112, 2113, 4097])
def test_layer_norm_layer_on_wide_frames(layers, bins):
    """More bins than are read as frames (an STFT of 8,192 samples has 4,097): rows are made of them; values and gradients as of rows, and against 64 bits."""
    _say("wide frames", bins)
    g = _gen(13)
    layer = layers.LayerNorm(bins)
    with torch.no_grad():
        layer.weight.add_(0.3 * torch.randn(bins, device=DEV, generator=g))
    spec = torch.randn(2, bins, 21, device=DEV, generator=g).requires_grad_()
    y = layer(spec.transpose(1, 2))
    gout = torch.randn(y.shape, device=DEV, generator=g)
    y.backward(gout)
    x, w = spec.detach().double().transpose(1, 2).requires_grad_(), layer.weight.detach().double().requires_grad_()
    d = x - x.mean(-1, keepdim=True)
    ref = d / (d.square().mean(-1, keepdim=True) + layer.eps).sqrt() * w
    ref.backward(gout.double())
    for got, want in ((y, ref.detach()), (spec.grad, x.grad.transpose(1, 2)), (layer.weight.grad, w.grad)):
        _near(got, want, 1e-5)
    with torch.no_grad():
        assert torch.equal(layer(spec.transpose(1, 2)), y)
        if bins > 2112:
            assert torch.equal(layer(spec.transpose(1, 2).contiguous()), y)


LAYERS8 = {"stft": lambda L, b: L.STFT(n_fft=512, hop_length=128, trainable=True, output_format="Power", kept_bits=b),
           "mel": lambda L, b: L.MelSpectrogram(sr=16000, n_fft=512, hop_length=128, n_mels=40, trainable_mel=True, trainable_STFT=True, kept_bits=b),
           "cqt": lambda L, b: L.CQT1992v2(sr=16000, hop_length=128, fmin=220.0, n_bins=24, trainable=True, output_format="Power", kept_bits=b)}


@pytest.mark.parametrize("kind", sorted(LAYERS8))
@pytest.mark.parametrize("length", [9001, 6000, 16384])
def test_products_in_8_bits_of_a_clip_know_no_other_clip(layers, kind, length):
    """A clip between two others that is NaN in one sample, or a million times as loud: the others' gradients are those of 8 bits by themselves, off by at most
    sqrt(128) / 254 < 0.045 of a block's norm (whatever its neighbour)."""
    _say("clips in 8 bits", kind, length)
    g = _gen(14)
    clean = 0.3 * torch.randn(3, length, device=DEV, generator=g)
    gout = None
    grads = {}
    for bits in (32, 8):
        layer = LAYERS8[kind](layers, bits)
        for what in ("clean", "nan", "loud"):
            x = clean.clone()
            if what == "nan":
                x[1, length // 2] = float("nan")
            elif what == "loud":
                x[1] *= 1e3  # its powers a million times
            x.requires_grad_()
            y = layer(x)
            gout = torch.randn(y.shape, device=DEV, generator=_gen(15)) if gout is None else gout
            y.backward(gout)
            grads[bits, what] = x.grad
    for what in ("nan", "loud"):
        for b in (0, 2):
            full, small, alone = grads[32, "clean"][b], grads[8, what][b], grads[8, "clean"][b]
            assert torch.isfinite(small).all(), what
            assert (small - full).norm() <= 0.045 * full.norm(), what
            assert (small - alone).norm() <= 1e-5 * alone.norm(), what
    assert not torch.isfinite(grads[8, "nan"][1]).all()


@pytest.mark.parametrize("kind", sorted(LAYERS8))
@pytest.mark.parametrize("batch,frames", [(1, 15), (40, 15), (1, 16), (5, 16), (2, 32), (3, 33), (1, 64), (4, 128), (2, 129)])
def test_products_in_8_bits_of_any_number_of_frames(layers, kind, batch, frames):
    _say("frames in 8 bits", kind, batch, frames)
    if kind == "cqt":  # one second at least: its longest kernel
        frames += 25
    x = (0.3 * torch.randn(batch, 128 * (frames - 1), device=DEV, generator=_gen(16))).requires_grad_()
    grads = []
    for bits in (32, 8):
        layer = LAYERS8[kind](layers, bits)
        x.grad = None
        y = layer(x)
        assert y.shape[-1] == frames
        held = [t for t in y.grad_fn.saved_tensors if t is not x]
        assert len(held) == (2 if bits == 8 and frames >= 16 else 1)
        y.backward(torch.randn(y.shape, device=DEV, generator=_gen(17)))
        grads.append([x.grad.clone()] + [p.grad.clone() for p in layer.parameters()])
    for a, b in zip(*grads):
        assert torch.isfinite(b).all() and (a - b).norm() <= 0.045 * a.norm()


FIRST_CALLS = """
import sys
import torch
from paper_1912_12055_amd import binding as nb
g = torch.Generator(device="cuda:0").manual_seed(1)
x, w = torch.randn(64, 200, device="cuda:0", generator=g), torch.ones(200, device="cuda:0")
spec, q = torch.randn(2, 50, 40, device="cuda:0", generator=g), torch.randn(1, 900, 2, 64, device="cuda:0", generator=g)
decay, state = torch.full((2,), 0.9, device="cuda:0"), torch.zeros(1, 2, 64, 64, device="cuda:0")

def step():
    y, kept = nb.nna_layer_norm(x, w, keep=8)
    f, kf = nb.nna_layer_norm(spec.transpose(1, 2), keep=32)
    o, last = nb.nna_decay_attention(q, q, q, decay, state=state, want_state=True)
    return [y, *nb.nna_layer_norm_backward(x, kept, w), f, *nb.nna_layer_norm_backward(f, kf), o, last, *nb.nna_decay_attention_backward(o, q, q, q, decay)[:3],
            nb.nna_unpack8(*nb.nna_pack8(x))]

torch.mm(x, x.T)  # (torch's own set-up)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = step()
for k in range(3):
    x.copy_(torch.randn_like(x)), q.copy_(torch.randn_like(q))
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in out]
    assert all(torch.equal(a, b) for a, b in zip(got, step())), k
print("the same")
"""


def test_first_calls_of_a_process_inside_a_graph(layers):
    """The kernels' set-up is done at the first call that needs it, also where that call is recorded."""
    import subprocess

    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=100)
    assert done.returncode == 0 and "the same" in done.stdout, done.stderr[-2000:]
