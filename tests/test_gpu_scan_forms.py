"""The gated recurrence in each of the forms that a call's sizes choose, and where thousands of frames' products have to be exact.

A gate is off by 6 roundings of 2^-24 of itself, a frame's step by 3 more of the state, and both are forgotten with the state: the bounds here follow the recurrence itself, each frame's
own error (10 U of the magnitudes, twice that where two such values meet) carried on by its gate, and not the number of frames.
"""
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0**-24


@pytest.fixture(scope="module")
def nb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import binding
    binding.lib()
    return binding


def _say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def exact(x, f, i, go, first, glast, lengths):
    """{name: (value, bound of a float32 form's error)} in 64 bits on the GPU.  Of each sequence its value, its sum of magnitudes, and its error: e <- a e + 10 U magnitude."""
    B, T, C = x.shape
    n = torch.full((B,), T, device=DEV) if lengths is None else lengths.clamp(0, T)
    x, f, go, first, glast, i = (None if t is None else t.double() for t in (x, f, go, first, glast, i))
    a, u = torch.sigmoid(f), torch.sigmoid(-f if i is None else i)
    na, nu = torch.sigmoid(-f), torch.sigmoid(f if i is None else -i)
    here = torch.arange(T, device=DEV)[None, :, None] < n[:, None, None]
    h, size, off = first, first.abs(), torch.zeros_like(first)
    hs, sizes, offs, before = [], [], [], []
    for t in range(T):
        before.append((h, size, off))
        now = a[:, t] * h + u[:, t] * x[:, t], a[:, t] * size + u[:, t] * x[:, t].abs()
        now = *now, a[:, t] * off + 10 * U * now[1]
        h, size, off = (torch.where(here[:, t], new, old) for new, old in zip(now, (h, size, off)))
        hs.append(h), sizes.append(size), offs.append(off)
    h, off = (torch.where(here, torch.stack(v, 1), 0.0) for v in (hs, offs))
    out = dict(h=(h, off), last=(hs[-1], offs[-1]))
    bh, bs, bo = (torch.stack(v, 1) for v in zip(*before))
    e, size, off = glast, glast.abs(), torch.zeros_like(glast)
    es, sizes, offs = [None] * T, [None] * T, [None] * T
    for t in reversed(range(T)):
        e, size = (torch.where(here[:, t], s + g, s) for s, g in ((e, go[:, t]), (size, go[:, t].abs())))
        es[t], sizes[t], offs[t] = e, size, off
        e, off = torch.where(here[:, t], a[:, t] * e, e), torch.where(here[:, t], a[:, t] * off + 10 * U * size, off)
        size = torch.where(here[:, t], a[:, t] * size, size)
    out["gfirst"] = e, off + 10 * U * size
    es, sizes, offs = (torch.stack(v, 1) for v in (es, sizes, offs))
    taken, taken_size = (bh - x, bs + x.abs()) if i is None else (bh, bs)
    out["gx"] = u * es, u * (offs + 10 * U * sizes)
    out["gf"] = a * na * es * taken, a * na * (offs * taken_size + sizes * bo + 20 * U * sizes * taken_size)
    if i is not None:
        out["gi"] = u * nu * es * x, u * nu * x.abs() * (offs + 20 * U * sizes)
    return {k: (torch.where(here, v, 0.0) if v.dim() == 3 else v, bound) for k, (v, bound) in out.items()}


def near(name, got, value, bound):
    bound = bound + 2.0**-126 * (1 + value.abs().amax())
    if got.dtype != torch.float32:
        bound = bound + torch.finfo(got.dtype).eps / 2 * torch.clamp(value.abs() + bound, min=torch.finfo(got.dtype).tiny)
    worst = float(((got.double() - value).abs() / bound).max())
    assert worst <= 1, (name, worst)


# (sequences, frames, channels of float32): rows of 16 lanes; of 32 with several rounds; segments of several rounds; and of one
FORMS = [(4, 300, 1024), (4, 700, 1009), (13, 513, 250), (16, 431, 512), (23, 300, 257), (1, 2100, 2047), (2, 1300, 1000), (1, 3001, 300), (3, 300, 64)]


@pytest.mark.parametrize("B,T,C", FORMS)
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_forms(nb, B, T, C, gated, dtype):
    if dtype != torch.float32:
        C *= 2  # (a lane takes two channels of 16 bits: the same form)
    _say(B, T, C, gated, dtype)
    g = torch.Generator(device=DEV).manual_seed(T + C)

    def normal(*s):
        return torch.randn(*s, device=DEV, generator=g)

    # a projection's slices; channels that remember from a few frames to thousands
    wide = normal(B, T, (2 + gated) * C)
    wide[..., C : 2 * C] += 9 * torch.rand(C, device=DEV, generator=g)
    wide = wide.to(dtype)
    x, f, i = wide[..., :C], wide[..., C : 2 * C], wide[..., 2 * C :] if gated else None
    go, first, glast = normal(B, T, C).to(dtype), normal(B, C), normal(B, C)
    ragged = torch.randint(0, T + 1, (B,), device=DEV, generator=g).to(torch.int32)
    ragged[0] = T
    ragged[-1] = T - T // 3
    for lengths in (None, ragged):
        want = exact(x, f, i, go, first, glast, lengths)
        h, last, kept = nb.nna_gated_scan(x, f, i, state=first, lengths=lengths, want_state=True, keep=True)
        gx, gf, gi, gfirst = nb.nna_gated_scan_backward(go, kept, x, f, i, lengths=lengths, gstate=glast, want_gstate=True)
        for name, got in dict(h=h, last=last, gx=gx, gf=gf, gi=gi, gfirst=gfirst).items():
            if got is not None:
                near(name, got, *want[name])
                if lengths is not None and got.dim() == 3:
                    assert not got[torch.arange(T, device=DEV) >= ragged[:, None]].any(), name


@pytest.mark.parametrize("B,C", [(1, 64), (4, 1024), (16, 512)])
@pytest.mark.parametrize("gated", [False, True])
def test_steady_gates(nb, B, C, gated):
    """A decay for each channel, the same in every frame, over 16,384 frames: what is left of a first state, of a constant input, and the gradients that come all the way.  A run's 1 - A is off by
    6 U for the gate (exponential 3, its sum, the reciprocal and the product 1 each), 5 for its own sum (eight additions of a sum that grows to it), 1 for what they add and 2 for each time that
    runs are joined: 16 U at most, if all had one sign, of a sum over all frames of ten at most: 9.6e-6; a state's own steps, 1,024 roundings of up to U / 2, are a walk of less than 4e-7: below 1e-5 together.
    In half of the channels the sum is below 0.6: the median is below 2e-6."""
    T = 16384
    f = torch.linspace(7.4, 13, C, device=DEV)
    a, q = torch.sigmoid(f.double()), torch.sigmoid(-f.double())
    left = torch.exp(T * torch.log1p(-q))
    some = -torch.expm1(T * torch.log1p(-q))
    f = f.expand(B, T, C)
    one, zero = torch.ones(1, 1, C, device=DEV).expand(B, T, C), torch.zeros(1, 1, C, device=DEV).expand(B, T, C)
    first = 0.5 + torch.rand(B, C, device=DEV, generator=torch.Generator(device=DEV).manual_seed(C))

    def held(name, got, want):
        off = ((got.double() - want) / want).abs()
        _say(name, float(off.max()), float(off.median()))
        assert float(off.max()) <= 1e-5 and float(off.median()) <= 2e-6, (name, float(off.max()), float(off.median()))

    # (a gate of the input's own that is open as far as the other's is closed)
    i = -f.contiguous() if gated else None
    _, last, kept = nb.nna_gated_scan(zero, f, i, state=first, want_state=True, keep=True)
    held("left", last, left * first.double())
    h, last = nb.nna_gated_scan(one, f, i, want_state=True)
    held("of ones", last, some.expand(B, C))
    held("of ones, the last frame", h[:, -1], some.expand(B, C))
    gx, gf, gi, gfirst = nb.nna_gated_scan_backward(torch.zeros(B, T, C, device=DEV), kept, zero, f, i, gstate=first, want_gstate=True)
    held("first state's gradient", gfirst, left * first.double())
    held("first frame's", gx[:, 0], q * torch.exp((T - 1) * torch.log1p(-q)) * first.double())
    # gf: a (1 - a) e h, the state left of the first one so far times the gradient left of the last one: the same in all frames
    held("gates'", gf[:, 5000], q * left * first.double() ** 2)
    gx, _, _, gfirst = nb.nna_gated_scan_backward(one.contiguous(), kept, zero, f, i, want_gstate=True)
    held("of ones, first state's", gfirst, (a * some / q).expand(B, C))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,C", [(1, 128), (4, 2048), (16, 1024)])
def test_steady_gates_of_16_bits(nb, B, C, dtype):
    """The same of 16-bit gates, whose exponential's argument (up to 11 where the sum is large) is one float32: 6 U for its rounding, 2 for its factor's, 2 for the exponential and 3 as above, and 10
    for the sums: 23 U of a sum of ten: 1.4e-5, and the walk: 1.5e-5."""
    T = 16384
    f = torch.linspace(7.41, 13, C, device=DEV).to(dtype)
    q = torch.sigmoid(-f.double())
    left, some, f = torch.exp(T * torch.log1p(-q)), -torch.expm1(T * torch.log1p(-q)), f.expand(B, T, C)
    first = 0.5 + torch.rand(B, C, device=DEV, generator=torch.Generator(device=DEV).manual_seed(C))
    zero, one = torch.zeros(1, 1, C, device=DEV, dtype=dtype).expand(B, T, C), torch.ones(1, 1, C, device=DEV, dtype=dtype).expand(B, T, C)
    _, last, kept = nb.nna_gated_scan(zero, f, state=first, want_state=True, keep=True)
    ones = nb.nna_gated_scan(one, f, want_state=True)[1]
    gfirst = nb.nna_gated_scan_backward(zero.contiguous(), kept, zero, f, gstate=first, want_gstate=True)[3]
    for name, got, want in (("left", last, left * first.double()), ("of ones", ones, some.expand(B, C)), ("gradient", gfirst, left * first.double())):
        off = ((got.double() - want) / want).abs()
        _say(name, dtype, float(off.max()), float(off.median()))
        assert float(off.max()) <= 1.5e-5 and float(off.median()) <= 2e-6, (name, float(off.max()), float(off.median()))
