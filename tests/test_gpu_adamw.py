"""AdamW steps over many tensors against the definition in 64 bits, states in 32 bits and in 8.

Tolerances, U = 2^-24.  A moment in 32 bits is two products and a sum of terms: 5 U of the sum of their magnitudes (the factor 1 - b is rounded too).  An update divides one by the
root of the other: the quotient is off by 5 + 3 + 6 U of itself (first moment, half of the second's, root, product, sum, quotient, rate, its product); the weight, kept and
summed, by 3 U more.  With g and m of either sign the first moment's own error counts by its terms, not by itself.  8-bit codes are equal: their borders are met in 64 bits here and there,
and the moments before them are sums of the same products (g^2 first): b s + (1 - b) g is often halfway between two scales.
"""
import math
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0**-24
HOW = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.05)


@pytest.fixture(scope="module")
def nb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import binding
    binding.lib()
    return binding


def _say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


SHAPES = [(1,), (7,), (128,), (129,), (300, 5), (0,), (2048,), (2049,), (64, 64), (10000,), (3, 1, 5), (70000,), (127,), (8192,), (8193,)]


def tensors(dtypes, seed=0, shapes=SHAPES):
    g = torch.Generator(device=DEV).manual_seed(seed)
    params, grads = [], []
    for n, s in enumerate(shapes):
        dtype = dtypes[n % len(dtypes)]
        params.append(torch.randn(s, device=DEV, generator=g).to(dtype))
        # gradients of very different sizes, some of them zero
        v = torch.randn(s, device=DEV, generator=g) * torch.exp(3 * torch.randn(s, device=DEV, generator=g)) * 1e-2
        grads.append(torch.where(torch.rand(s, device=DEV, generator=g) < 0.1, 0, v).to(dtype))
    return params, grads


def states(nb, params, bits, master=False):
    _, size = nb.nna_adamw_places([p.numel() for p in params])
    s = dict(m=torch.zeros(size, device=DEV, dtype=torch.float32 if bits == 32 else torch.int8), v=torch.zeros(size, device=DEV, dtype=torch.float32 if bits == 32 else torch.uint8))
    if bits == 8:
        s["m_scales"], s["v_scales"] = torch.zeros(size // 128, device=DEV), torch.zeros(size // 128, device=DEV)
    if master:
        s["master"] = torch.full((size,), 7.0, device=DEV)
        for p, part in zip(params, parts(nb, s["master"], params)):
            if p.dtype != torch.float32:
                part.copy_(p.flatten())
    return s


def parts(nb, flat, params, unit=1):
    at, _ = nb.nna_adamw_places([p.numel() for p in params])
    return [flat[a // unit : (a + p.numel() + unit - 1) // unit] for a, p in zip(at.tolist(), params)]


def near(name, got, value, tolerance):
    off = (got.double() - value).abs()
    worst = float((off / tolerance.clamp(min=1e-300)).max()) if off.numel() else 0.0
    assert worst <= 1, (name, worst)


def expect(p, g, m, v, t, lr, betas, eps, weight_decay):
    """(p, m, v and the tolerances of a float32 form) in 64 bits; p, g, m, v of 64 bits"""
    b1, b2 = betas
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * (g * g)
    size = b1 * m.abs() + (1 - b1) * g.abs()
    root = (v1 / (1 - b2**t)).sqrt() + eps
    rate = lr / (1 - b1**t)
    new = (1 - lr * weight_decay) * p - rate * m1 / root
    return new, m1, v1, 3 * U * (p.abs() + new.abs()) + 20 * U * rate * size / root, 5 * U * size + 1e-45, 6 * U * v1 + 1e-44


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16,), (torch.float16, torch.float32), (torch.bfloat16, torch.float32, torch.float16)])
@pytest.mark.parametrize("master", [False, True])
def test_32_bits(nb, dtypes, master):
    _say(dtypes, master)
    params, grads = tensors(dtypes)
    s = states(nb, params, 32, master)
    for t in (1, 2, 3, 1000):
        if t == 3:
            grads = [None if n in (1, 9) else g for n, g in enumerate(grads)]
        before = [x.clone() for x in params], {k: x.clone() for k, x in s.items()}
        nb.nna_adamw(params, grads, step=t, **s, **HOW)
        for n, (p, g) in enumerate(zip(params, grads)):
            was = before[0][n]
            m, v, old_m, old_v = (parts(nb, x, params)[n] for x in (s["m"], s["v"], before[1]["m"], before[1]["v"]))
            if g is None:
                assert torch.equal(p, was) and torch.equal(m, old_m) and torch.equal(v, old_v)
                continue
            narrow = p.dtype != torch.float32
            old = parts(nb, before[1]["master"], params)[n] if master and narrow else was.flatten()
            new, m1, v1, tp, tm, tv = expect(old.double(), g.flatten().double(), old_m.double(), old_v.double(), t, **HOW)
            near("m", m, m1, tm)
            near("v", v, v1, tv)
            if narrow:
                if master:
                    copy = parts(nb, s["master"], params)[n]
                    near("master", copy, new, tp)
                    assert torch.equal(copy.to(p.dtype), p.flatten())
                tp = tp + torch.finfo(p.dtype).eps / 2 * torch.clamp(new.abs() + tp, min=torch.finfo(p.dtype).tiny)
            near("p", p.flatten(), new, tp)
    if master:  # (float32 tensors have no copies, and what lies between tensors is left as it is)
        used = torch.zeros_like(s["master"], dtype=torch.bool)
        for p, part in zip(params, parts(nb, used, params)):
            if p.dtype != torch.float32:
                part.fill_(True)
        assert bool((s["master"][~used] == 7).all())
    for flat in (s["m"], s["v"]):
        used = torch.zeros_like(flat, dtype=torch.bool)
        for part in parts(nb, used, params):
            part.fill_(True)
        assert not flat[~used].any()


def first_values(codes, scales):
    c = codes.double()
    return (c / 127) * (c / 127).abs() * scales.double().repeat_interleave(128)[: c.numel()]


def second_values(codes, scales):
    return (codes.double() / 255) ** 4 * scales.double().repeat_interleave(128)[: codes.numel()]


def packed(x, levels, power, shift):
    """(codes' magnitudes, scales) of x >= 0 in 64 bits; blocks whose largest is no normal float32 are zero"""
    n = x.numel()
    blocks = torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128)
    scales = blocks.amax(-1).float()
    scales = torch.where(scales >= 2.0**-126, scales, 0)
    most = scales.double().repeat_interleave(128)[:n]
    y = torch.where(most > 0, x / torch.where(most > 0, most, 1), 0) ** (1 / power) * levels + shift
    codes = torch.floor(y).clamp(max=levels)
    if power == 4:
        codes = torch.where((x > 0) & (most > 0), codes.clamp(min=1), torch.where(x > 0, codes, 0))
    return torch.where(most > 0, codes, 0), scales


@pytest.mark.parametrize("dtypes", [(torch.float32,), (torch.bfloat16, torch.float32, torch.float16)])
def test_8_bits(nb, dtypes):
    params, grads = tensors(dtypes, seed=1)
    torch.manual_seed(1)
    s = states(nb, params, 8, master=True)
    places, _ = nb.nna_adamw_places([p.numel() for p in params])
    for t in (1, 2, 3, 4, 500):
        grads = [(g.float() * (1 + 0.3 * torch.randn_like(g.float()))).to(g.dtype) for g in grads]
        before = [x.clone() for x in params], {k: x.clone() for k, x in s.items()}
        nb.nna_adamw(params, grads, step=t, **s, **HOW)
        for n, (p, g) in enumerate(zip(params, grads)):
            def of(x, unit=1):
                return parts(nb, x, params, unit)[n]

            narrow = p.dtype != torch.float32
            old = of(before[1]["master"]) if narrow else before[0][n].flatten()
            om, ov = first_values(of(before[1]["m"]), of(before[1]["m_scales"], 128)), second_values(of(before[1]["v"]), of(before[1]["v_scales"], 128))
            new, m1, v1, tp, _, _ = expect(old.double(), g.flatten().double(), om, ov, t, **HOW)
            copy = of(s["master"]) if narrow else p.flatten()
            near("weight", copy, new, tp)
            if narrow:
                assert torch.equal(copy.to(p.dtype), p.flatten())
            codes, scales = packed(m1.abs(), 127, 2, 0.5)
            assert torch.equal(of(s["m"]).double(), codes * m1.sign()) and torch.equal(of(s["m_scales"], 128), scales)
            at = torch.arange(p.numel(), device=DEV) + int(places[n])
            shift = (((at * 0x9E3779B9 + t * 0xB504F333) & 0xFFFFFFFF) >> 8).double() * 2.0**-24
            codes, scales = packed(v1, 255, 4, shift)
            assert torch.equal(of(s["v"]).double(), codes) and torch.equal(of(s["v_scales"], 128), scales)
    for codes, scales, values in ((s["m"], s["m_scales"], first_values), (s["v"], s["v_scales"], second_values)):
        got, want = nb.nna_adamw_moment(codes, scales).double(), values(codes, scales)
        assert float((got - want).abs().max()) <= U * float(want.abs().max()) and torch.equal(got != 0, want != 0)
        assert bool(((got - want).abs() <= 2 * U * want.abs() + 1e-45).all())


@pytest.mark.parametrize("kind", ["cancel", "tiny", "faint", "same", "steep"])
def test_8_bits_where_float32_says_little(nb, kind):
    """Moments that cancel to 10^-4 of their terms (64 bits' own roundings are 10^-12 of what is left), gradients whose squares are below float32, blocks of one value, and values 2^-40 apart: the codes are those of 64 bits."""
    torch.manual_seed(7)
    p = torch.zeros(128 * 40, device=DEV)
    s = states(nb, [p], 8)
    g = torch.randn_like(p)
    if kind == "same":
        g = torch.randn(40, 1, device=DEV).expand(40, 128).flatten().contiguous()
    if kind == "tiny":
        g *= 10.0 ** -torch.linspace(10, 25, g.numel(), device=DEV).view(128, 40).t().flatten()
    if kind == "faint":
        g *= 10.0 ** -torch.linspace(8, 22, 40, device=DEV).repeat_interleave(128)
    if kind == "steep":
        g *= 2.0 ** -torch.randint(0, 40, g.shape, device=DEV)
    for t in (1, 2, 3):
        before = {k: x.clone() for k, x in s.items()}
        om, ov = first_values(before["m"], before["m_scales"]), second_values(before["v"], before["v_scales"])
        if kind == "cancel" and t > 1:
            g = (-9 * om * (1 + 1e-4 * torch.randn_like(om))).float()
        nb.nna_adamw([p], [g], step=t, **s, **HOW)
        _, m1, v1, *_ = expect(p.double(), g.double(), om, ov, t, **HOW)
        codes, scales = packed(m1.abs(), 127, 2, 0.5)
        assert torch.equal(s["m_scales"], scales) and torch.equal(s["m"].double(), codes * m1.sign())
        shift = (((torch.arange(p.numel(), device=DEV) * 0x9E3779B9 + t * 0xB504F333) & 0xFFFFFFFF) >> 8).double() * 2.0**-24
        codes, scales = packed(v1, 255, 4, shift)
        assert torch.equal(s["v_scales"], scales) and torch.equal(s["v"].double(), codes)


def test_second_moments_in_8_bits_follow_their_decay(nb):
    """Rounded to the nearest, codes whose distance is wider than 1 - b2 would stay for good where the block's largest is fed anew.  After 200 steps without a gradient (0.82 of where it began) a
    value's code is still above 56: a rounding there is off by less than one code, 4 / 56 of the value.  Every step adds one, most of one sign cancelled by the sequence's next: five left over
    are 36 %, and the mean over 12,700 values, each with its own place in the sequence, is off by 1 % at most (five roundings' spread of 4 / 56 / sqrt(12) each, over the root of 12,700: 0.05 %,
    and the root's curve, half of the spread squared: 0.5 %)."""
    p, g = torch.zeros(12800, device=DEV), torch.zeros(12800, device=DEV)
    s = states(nb, [p], 8)
    s["v"].copy_(torch.randint(60, 255, (12800,), device=DEV))
    s["v"][::128] = 255
    s["v_scales"].fill_(1.0)
    begin = second_values(s["v"], s["v_scales"])
    g[::128] = 1.0  # (keeps the blocks' scales where they are)
    for t in range(1, 201):
        nb.nna_adamw([p], [g], step=t, **s, lr=0.0, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0)
    end = second_values(s["v"], s["v_scales"])
    rest = torch.ones(12800, dtype=torch.bool, device=DEV)
    rest[::128] = False
    ratio = (end / begin)[rest] / 0.999**200
    assert float((ratio.log().mean()).abs()) <= 0.01 and float(ratio.max()) <= 1.4 and float(ratio.min()) >= 1 / 1.4


def test_what_is_not_finite(nb):
    """Of 32 bits its own value, of 8 its block, whose neighbours' weights of that step are right still; and the block stays marked."""
    for bits in (32, 8):
        params, grads = tensors((torch.float32,), shapes=[(300,), (300,)])
        s = states(nb, params, bits)
        twin, t = [p.clone() for p in params], {k: x.clone() for k, x in s.items()}
        nb.nna_adamw(twin, grads, step=1, **t, **HOW)
        for value in (float("nan"), float("inf")):
            mine, u = [p.clone() for p in params], {k: x.clone() for k, x in s.items()}
            spoilt = [grads[0], grads[1].clone()]
            spoilt[1][130] = value
            nb.nna_adamw(mine, spoilt, step=1, **u, **HOW)
            assert torch.equal(mine[0], twin[0])
            bad = ~mine[1].isfinite()
            assert bad.nonzero().flatten().tolist() == [130]
            assert torch.equal(mine[1][~bad], twin[1][~bad])
            nb.nna_adamw(mine, grads, step=2, **u, **HOW)
            assert (~mine[1].isfinite()).nonzero().flatten().tolist() == ([130] if bits == 32 else list(range(128, 256)))


def test_zero_and_tiny_blocks(nb):
    """Blocks of zeros, of values whose squares are below float32's, and of its largest: nothing is divided by zero."""
    g = torch.zeros(6 * 128, device=DEV)
    g[128:256] = 1e-30
    g[256:384] = 1e-20
    g[384:512] = 1e18
    g[512] = 1e-3
    p = torch.ones_like(g)
    s = states(nb, [p], 8)
    for t in (1, 2, 3):
        nb.nna_adamw([p], [g], step=t, **s, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0)
        assert p.isfinite().all() and s["m_scales"].isfinite().all() and s["v_scales"].isfinite().all()
    assert bool((p[:128] == 1).all()) and float(p[400]) == pytest.approx(1 - 3e-3, rel=1e-3) and bool((p[513:640] == 1).all())


def test_against_a_plain_loop(nb):
    """Twenty steps on one problem, 32 bits: torch's own loop in 64 bits, off by the steps' own roundings (20 times a step's tolerance, and what they do to the next)."""
    p = torch.randn(5000, device=DEV)
    ref = p.double().clone().requires_grad_(True)
    mine, s = p.clone(), states(nb, [p], 32)
    optimiser = torch.optim.AdamW([ref], lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1, foreach=False, fused=False)
    for t in range(1, 21):
        g = torch.randn(5000, device=DEV)
        ref.grad = g.double()
        optimiser.step()
        nb.nna_adamw([mine], [g], step=t, **s, lr=1e-2, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.1)
    assert float((mine.double() - ref.detach()).abs().max()) <= 20 * (3 * U * 2 * float(p.abs().max()) + 20 * U * 1e-2 * 20)


def test_many_tensors(nb):
    """More than one launch takes; the same step one tensor at a time gives the same bits."""
    shapes = [(1 + 37 * n % 1000,) for n in range(333)]
    params, grads = tensors((torch.float32, torch.bfloat16), shapes=shapes)
    for bits in (32, 8):
        one, s = [p.clone() for p in params], states(nb, params, bits)
        nb.nna_adamw(one, grads, step=5, **s, **HOW)
        if bits == 32:
            for p, g, whole in zip(params, grads, one):
                p = p.clone()
                nb.nna_adamw([p], [g], step=5, **states(nb, [p], bits), **HOW)
                assert torch.equal(p, whole)


@pytest.mark.parametrize("live,behind", [(80, 1), (80, 100), (79, 3), (160, 2), (81, 1)])
def test_tensors_without_a_gradient_behind_a_full_launch(nb, live, behind):
    """80 tensors go into a launch: what lies behind them without a gradient asks for none."""
    params, grads = tensors((torch.float32, torch.bfloat16), shapes=[(1 + 37 * n % 300,) for n in range(live + behind)])
    mine, s = [p.clone() for p in params], states(nb, params, 32)
    nb.nna_adamw(mine, [*grads[:live], *[None] * behind], step=3, **s, **HOW)
    twin = [p.clone() for p in params[:live]]
    nb.nna_adamw(twin, grads[:live], step=3, **states(nb, twin, 32), **HOW)
    for n, p in enumerate(mine):
        assert torch.equal(p, twin[n] if n < live else params[n]), n


def test_views_at_any_place(nb):
    for bits in (32, 8):
        for dtype in (torch.float32, torch.bfloat16):
            memory, gradient = torch.randn(2, 5000, device=DEV).to(dtype).unbind(0)
            p, g = memory[1:4001], gradient[3:4003]
            rest = memory[4001:].clone(), memory[0].clone()
            q = p.clone()
            for x, y in ((p, g), (q, g.clone())):
                nb.nna_adamw([x], [y], step=1, **states(nb, [x], bits), **HOW)
            assert torch.equal(p, q) and torch.equal(memory[4001:], rest[0]) and torch.equal(memory[0], rest[1])


def test_step_and_rate_in_device_memory_and_a_graph(nb):
    params, grads = tensors((torch.float32, torch.bfloat16))
    for bits in (32, 8):
        mine, s = [p.clone() for p in params], states(nb, params, bits)
        twin, t = [p.clone() for p in params], {k: x.clone() for k, x in s.items()}
        step, lr = torch.zeros(1, dtype=torch.int64, device=DEV), torch.tensor(1e-3, device=DEV)
        how = {k: v for k, v in HOW.items() if k != "lr"}
        nb.nna_adamw(mine, grads, step=step + 1, lr=lr, **s, **how)  # (not recorded: sets nothing up, and takes part)
        nb.nna_adamw(twin, grads, step=1, lr=float(lr), **t, **how)
        step.fill_(1)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step.add_(1)
            nb.nna_adamw(mine, grads, step=step, lr=lr, **s, **how)
        for n in range(2, 6):
            lr.fill_(n * 1e-3)
            for g in grads:
                g.mul_(0.7)
            graph.replay()
            nb.nna_adamw(twin, grads, step=n, lr=float(lr), **t, **how)
            torch.cuda.synchronize()
            for a, b in zip(mine, twin):
                assert torch.equal(a, b), n
            for k in s:
                assert torch.equal(s[k], t[k]), (n, k)


def test_versions_and_streams(nb):
    params, grads = tensors((torch.float32,), shapes=[(300,), (5,)])
    s = states(nb, params, 32)
    at = [p._version for p in params]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    nb.nna_adamw(params, [grads[0], None], step=1, **s, **HOW, stream=side.cuda_stream)
    side.synchronize()
    assert params[0]._version > at[0] and params[1]._version == at[1] and s["m"]._version > 0


def test_refusals(nb):
    p, g = torch.zeros(300, device=DEV), torch.ones(300, device=DEV)
    s = states(nb, [p], 32)
    s8 = states(nb, [p], 8)

    def call(params=(p,), grads=(g,), step=1, s=s, **more):
        nb.nna_adamw(list(params), list(grads), step=step, **{**s, **more})

    bad = [
        lambda: call(grads=()), lambda: call(params=(p.cpu(),)), lambda: call(grads=(g.cpu(),)), lambda: call(grads=(g.half(),)), lambda: call(grads=(g[:200],)),
        lambda: call(params=(p.double(),), grads=(g.double(),)), lambda: call(params=(p.view(2, 150).t(),), grads=(g.view(2, 150).t(),)), lambda: call(step=0), lambda: call(step=-1),
        lambda: call(step=torch.ones(1, device=DEV)), lambda: call(step=torch.ones(1, dtype=torch.int64)), lambda: call(step=torch.ones(2, dtype=torch.int64, device=DEV)),
        lambda: call(lr=float("nan")), lambda: call(lr=torch.ones(1, dtype=torch.float64, device=DEV)), lambda: call(betas=(1.0, 0.9)), lambda: call(betas=(0.9, 1.0)),
        lambda: call(eps=-1.0), lambda: call(weight_decay=float("inf")), lambda: call(m=s["m"][:256]), lambda: call(m=s["m"].half()), lambda: call(v=s["v"].cpu()), lambda: call(m=s["v"]),
        lambda: call(s=s8, m_scales=None), lambda: call(s=s8, v_scales=s8["v_scales"][:1]), lambda: call(s=s8, v=s8["m"]), lambda: call(m_scales=s8["m_scales"], v_scales=s8["v_scales"]),
        lambda: call(params=(p, p), grads=(g, g), s=states(nb, [p, p], 32)), lambda: call(params=(p, p[100:200]), grads=(g, g[:100]), s=states(nb, [p, p[:100]], 32)),
        lambda: call(master=s["m"][:256]), lambda: call(grads=(p,)), lambda: call(params=("x",)), lambda: nb.nna_adamw_moment(s["m"], s8["m_scales"]),
        lambda: nb.nna_adamw_moment(s8["m"], s8["m_scales"][:1]), lambda: nb.nna_adamw_moment(s8["m"][:100], s8["m_scales"]), lambda: nb.nna_adamw_moment(s8["m"], s8["m_scales"], out=s["m"].half()),
    ]
    for n, c in enumerate(bad):
        with pytest.raises((TypeError, ValueError, nb.NnaError)):
            c()
            pytest.fail(f"call {n} was not refused")
    assert not p.any() and not s["m"].any()
    nb.nna_adamw([], [], torch.empty(0, device=DEV), torch.empty(0, device=DEV), 1)
