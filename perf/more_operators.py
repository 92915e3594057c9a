"""The work that the speed of this library's further operators of networks on the frames is measured on: queries and keys normalised
and rotated by their frames' positions, the gated linear recurrence, and AdamW steps over all of a network's tensors.

Every case is one call, or one training step's forward and backward call, that such a network makes over and over.  ``own`` chooses between
the library's calls and their plain form in elementary torch operations; both take the same state.  The listed sizes go from one frame of one
stream to long training sequences, and from a small network's tensors to some hundred million parameters; ``draw`` spreads further ones over the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-6
BLOCK = 128  # a tensor's values that share a scale; tensors' states begin at multiples of it
LR, BETAS, ADAM_EPS, DECAY = 1e-3, (0.9, 0.999), 1e-8, 0.01
SIZE = {"float32": 4, "bfloat16": 2, "float16": 2}


def listed():
    return [
        # the new frame of one stream: launch and host time count
        dict(name="rotate_token", kind="rotate", train=False, batch=1, frames=0, heads=8, kheads=8, width=64, rotary=64, norm=True,
             interleaved=False, far=False, dtype="bfloat16"),
        # training on 16 clips of ten seconds, float32, pairs of neighbours
        dict(name="rotate_clips", kind="rotate", train=True, batch=16, frames=431, heads=8, kheads=8, width=64, rotary=64, norm=True,
             interleaved=True, far=False, dtype="float32"),
        # prompts far into their recordings, a position for each frame, keys shared by groups of heads, half of an odd-sized head rotated, no norm
        dict(name="rotate_far", kind="rotate", train=False, batch=3, frames=7001, heads=12, kheads=4, width=80, rotary=40, norm=False,
             interleaved=False, far=True, dtype="float16"),
        # training on long sequences
        dict(name="rotate_long", kind="rotate", train=True, batch=4, frames=16384, heads=16, kheads=16, width=128, rotary=128, norm=True,
             interleaved=False, far=False, dtype="bfloat16"),
        # one new frame of each of 256 streams through the recurrence
        dict(name="scan_streams", kind="scan_step", batch=256, width=2048, gates=1, dtype="bfloat16"),
        # a recording of three minutes (hop 256 at 22.05 kHz) as the prompt of a stream: outputs and the state to go on from
        dict(name="scan_song", kind="scan", train=False, batch=1, frames=15504, width=512, gates=1, ragged=False, state=True, dtype="bfloat16"),
        # training on 16 clips of up to ten seconds, lengths differ, float32, a gate of its own for the input, states carried over
        dict(name="scan_clips", kind="scan", train=True, batch=16, frames=431, width=512, gates=2, ragged=True, state=True, dtype="float32"),
        # training on long sequences
        dict(name="scan_long", kind="scan", train=True, batch=4, frames=16384, width=2048, gates=1, ragged=False, state=False, dtype="bfloat16"),
        # the tensors of a small network on Mel frames
        dict(name="adam_small", kind="adam", blocks=2, width=256, mels=80, n_fft=0, bits=32, dtype="float32"),
        # a trainable Mel layer (its kernels and its filters) with four blocks on top, states in 8 bits
        dict(name="adam8_layers", kind="adam", blocks=4, width=512, mels=128, n_fft=2048, bits=8, dtype="float32"),
        # a large network in bfloat16 with float32 copies of its weights
        dict(name="adam_large", kind="adam", blocks=16, width=1024, mels=128, n_fft=0, bits=32, dtype="bfloat16"),
        # the same with states in 8 bits
        dict(name="adam8_large", kind="adam", blocks=16, width=1024, mels=128, n_fft=0, bits=8, dtype="bfloat16"),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotate", "rotate", "rotate", "scan", "scan", "scan", "scan_step", "adam", "adam"])
    dtype = rng.choice(["float32", "bfloat16", "bfloat16", "float16"])
    if kind == "rotate":
        heads = rng.choice([1, 2, 3, 4, 8, 12, 16])
        kheads = rng.choice([n for n in (1, 2, 4, 8, 12, 16, heads) if heads % n == 0])
        width = rng.choice([32, 48, 64, 64, 80, 96, 128, rng.randint(16, 128)])
        rotary = rng.choice([width // 2 * 2, width // 2 * 2, width // 4 * 2, width // 8 * 2])
        train = rng.random() < 0.6
        frames = rng.choice([0, _log_between(rng, 1, 16384), _log_between(rng, 1, 16384)]) if not train else _log_between(rng, 1, 16384)
        most = (1 << (27 if dtype != "float32" else 26)) // (max(1, frames) * heads * width)
        return dict(kind=kind, train=train, batch=_log_between(rng, 1, max(1, min(256, most))), frames=frames, heads=heads, kheads=kheads,
                    width=width, rotary=rotary, norm=rng.random() < 0.7, interleaved=rng.random() < 0.5, far=rng.random() < 0.5, dtype=dtype)
    if kind == "scan_step":
        return dict(kind=kind, batch=_log_between(rng, 1, 256), width=_log_between(rng, 64, 4096), gates=rng.choice([1, 2]), dtype=dtype)
    if kind == "scan":
        width = rng.choice([_log_between(rng, 64, 4096), 64 * _log_between(rng, 1, 64)])
        frames = _log_between(rng, 1, 16384)
        gates = rng.choice([1, 2])
        most = (1 << (27 if dtype != "float32" else 25)) // (width * frames * gates)
        return dict(kind=kind, train=rng.random() < 0.7, batch=_log_between(rng, 1, max(1, min(64, most))), frames=frames, width=width,
                    gates=gates, ragged=rng.random() < 0.5, state=rng.random() < 0.5, dtype=dtype)
    width = rng.choice([64, 96, 128, 200, 256, 384, 512, 768, 1000, 1024])
    n_fft = rng.choice([0, 512, 1024, 2048])
    return dict(kind=kind, blocks=_log_between(rng, 1, max(1, min(24, 15 * 1024 * 1024 // width**2))), width=width, mels=rng.choice([40, 80, 84, 128, 229]),
                n_fft=n_fft, bits=rng.choice([8, 32]), dtype=rng.choice(["float32", "bfloat16"]))


# ---- a network's tensors -----------------------------------------------------------------------------------------------


def _shapes(case):
    """(the matrices and their biases, of the network's type; norms and a trainable Mel layer's weights, float32)"""
    w, mels = case["width"], case["mels"]
    network = [(w, mels), (w,)]
    for _ in range(case["blocks"]):
        network += [(3 * w, w), (3 * w,), (w, w), (w,), (4 * w, w), (4 * w,), (w, 4 * w), (w,)]
    exact = [(mels,), (mels,)] + [(w,)] * (4 * case["blocks"])
    if case["n_fft"]:
        bins = case["n_fft"] // 2 + 1
        exact += [(2 * bins, case["n_fft"]), (mels, bins)]
    return network, exact


def _padded(shapes):
    return [-(-math.prod(s) // BLOCK) * BLOCK for s in shapes]


def _flat(g, shapes, dtype, std):
    """Normal values in one piece of memory with a view for each tensor; zero between them."""
    sizes = _padded(shapes)
    flat = torch.zeros(sum(sizes), device=DEVICE, dtype=dtype)
    views, at = [], 0
    for shape, size in zip(shapes, sizes):
        n = math.prod(shape)
        flat[at : at + n].normal_(generator=g).mul_(std / math.sqrt(shape[-1]) if len(shape) > 1 else std)
        views.append(flat[at : at + n].view(shape))
        at += size
    return flat, views


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    s = dict(case)

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=g)

    kind, dtype = case["kind"], getattr(torch, case["dtype"])
    if kind == "rotate":
        B, T, H, K, d = case["batch"], max(1, case["frames"]), case["heads"], case["kheads"], case["width"]
        # queries and keys as one projection of the frames gives them, with the values in between; some channels larger than others
        gain = torch.exp(0.4 * normal((H + 2 * K) * d))
        qkv = (normal(B, T, (H + 2 * K) * d) * gain).to(dtype)
        s["q"], s["k"] = qkv[..., : H * d].view(B, T, H, d), qkv[..., H * d : (H + K) * d].view(B, T, K, d)
        # angles for long contexts: the base's exponent over the rotated part, positions interpolated by 4
        s["freqs"] = 10000.0 ** (-torch.arange(case["rotary"] // 2, dtype=torch.float64, device=DEVICE) / max(1, case["rotary"] // 2)) / 4
        start = torch.randint(0, 1 << 20 if case["far"] else 1 << 12, (B, 1), device=DEVICE, generator=g)
        s["positions"] = (start + torch.arange(T, device=DEVICE)).to(torch.int32) if case["far"] or not case["frames"] else None
        s["wq"], s["wk"] = (1 + 0.2 * normal(d), 1 + 0.2 * normal(d)) if case["norm"] else (None, None)
        if case["train"]:
            s["gq"], s["gk"] = normal(B, T, H, d).to(dtype), normal(B, T, K, d).to(dtype)
        if not case["frames"]:
            s["q"], s["k"], s["positions"] = s["q"][:, 0], s["k"][:, 0], s["positions"][:, 0].contiguous()
    elif kind in ("scan", "scan_step"):
        B, C, n = case["batch"], case["width"], 1 + case["gates"]
        T = case.get("frames", 1)
        # the input and its gates as one projection of the frames gives them; channels that remember from two frames to some thousands
        both = normal(B, T, n * C)
        both[..., C : 2 * C] += 1 + 7 * torch.rand(C, device=DEVICE, generator=g)
        both = both.to(dtype)
        s["x"], s["forget"] = both[..., :C], both[..., C : 2 * C]
        s["input"] = both[..., 2 * C :] if n == 3 else None
        if kind == "scan_step":
            s["x"], s["forget"], s["input"] = (t if t is None else t[:, 0] for t in (s["x"], s["forget"], s["input"]))
            s["state"] = normal(B, C)
        else:
            s["state0"] = normal(B, C) if case["state"] else None
            s["gstate"] = normal(B, C) if case["state"] and case["train"] else None
            s["lengths"] = None
            if case["ragged"]:
                s["lengths"] = (T * (0.3 + 0.7 * torch.rand(B, device=DEVICE, generator=g))).round().to(torch.int32)
            s["gout"] = normal(B, T, C).to(dtype) if case["train"] else None
    else:
        network, exact_ones = _shapes(case)
        s["p"], params = _flat(g, network, dtype, 1.0)
        s["g"], grads = _flat(g, network, dtype, 0.02)
        s["p32"], params32 = _flat(g, exact_ones, torch.float32, 1.0)
        s["g32"], grads32 = _flat(g, exact_ones, torch.float32, 0.02)
        s["params"], s["grads"] = params + params32, grads + grads32
        s["cut"] = s["p"].numel()
        s["master"] = None
        if dtype != torch.float32:
            # weights between two bfloat16 ones
            s["master"] = torch.cat([s["p"].float(), s["p32"]])
            s["master"][: s["cut"]] *= 1 + 2.0**-10 * (torch.rand(s["cut"], device=DEVICE, generator=g) - 0.5)
        every = torch.cat([s["g"].float(), s["g32"]])
        # what some hundred steps on gradients like these leave: the first moment noisy, the second one near the gradients' squares
        m = every * 0.3 * torch.rand(every.numel(), device=DEVICE, generator=g)
        v = every.square() * (0.02 + torch.rand(every.numel(), device=DEVICE, generator=g))
        s["step"] = 400
        if case["bits"] == 8:
            m, s["m_scales"] = _pack_first(m)
            v, s["v_scales"] = _pack_second(v, s["step"])
        else:
            s["m_scales"] = s["v_scales"] = None
        s["m"], s["v"] = m, v
    return s


# ---- the library's calls ---------------------------------------------------------------------------------------------


def _run_own(s):
    from paper_1912_12055_amd import binding as nb

    kind = s["kind"]
    if kind == "rotate":
        how = dict(positions=s["positions"], q_weight=s["wq"], k_weight=s["wk"], eps=EPS if s["norm"] else None, interleaved=s["interleaved"])
        out = nb.nna_rotate_heads(s["q"], s["k"], s["freqs"], **how)
        if not s["train"]:
            return out
        return (*out, *nb.nna_rotate_heads_backward(s["gq"], s["gk"], s["q"], s["k"], s["freqs"], **how))
    if kind == "scan_step":
        return nb.nna_gated_scan_step(s["x"], s["forget"], s["state"], input=s["input"]), s["state"]
    if kind == "scan":
        how = dict(input=s["input"], lengths=s["lengths"])
        if not s["train"]:
            return nb.nna_gated_scan(s["x"], s["forget"], state=s["state0"], want_state=True, **how)
        h, last, kept = nb.nna_gated_scan(s["x"], s["forget"], state=s["state0"], want_state=True, keep=True, **how)
        return (h, last, *nb.nna_gated_scan_backward(s["gout"], kept, s["x"], s["forget"], gstate=s["gstate"], want_gstate=s["state"], **how))
    s["step"] += 1
    nb.nna_adamw(s["params"], s["grads"], s["m"], s["v"], s["step"], lr=LR, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, m_scales=s["m_scales"],
                 v_scales=s["v_scales"], master=s["master"])
    m, v = s["m"], s["v"]
    if s["bits"] == 8:
        m, v = nb.nna_adamw_moment(m, s["m_scales"]), nb.nna_adamw_moment(v, s["v_scales"])
    return s["p"], s["p32"], s["master"], m, v


# ---- their plain form ------------------------------------------------------------------------------------------------


def _angles(s, frames):
    """cos and sin [B, T, 1, pairs]; the angles in 64 bits, since far positions leave nothing of them in 32"""
    at = s["positions"]
    if at is None:
        at = torch.arange(frames, device=DEVICE)[None]
    angle = at.reshape(-1, frames, 1, 1).double() * s["freqs"]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _pairs(x, n, interleaved):
    """(first, second) of each of the n pairs at the head's start, and what stays as it is"""
    if interleaved:
        return x[..., 0 : 2 * n : 2], x[..., 1 : 2 * n : 2], x[..., 2 * n :]
    return x[..., :n], x[..., n : 2 * n], x[..., 2 * n :]


def _rotate(x, cos, sin, interleaved):
    n = cos.shape[-1]
    a, b, rest = _pairs(x, n, interleaved)
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1)
    return torch.cat([turned, rest], -1)


def _plain_head(x, gout, weight, cos, sin, s):
    """(rotated norm of x, and with gout the gradients of x and the weight)"""
    v = x.float()
    if s["norm"]:
        r = 1 / torch.sqrt(v.square().mean(-1, keepdim=True) + EPS)
        h = v * r
        v = h * weight
    y = _rotate(v, cos, sin, s["interleaved"]).to(x.dtype)
    if gout is None:
        return y, None, None
    g = _rotate(gout.float(), cos, -sin, s["interleaved"])
    if not s["norm"]:
        return y, g.to(x.dtype), None
    gw = (g * h).sum(tuple(range(g.dim() - 1)))
    g = g * weight
    return y, (r * (g - h * (g * h).mean(-1, keepdim=True))).to(x.dtype), gw


def _plain_rotate(s):
    q, k = s["q"], s["k"]
    if not s["frames"]:
        cos, sin = (t[:, 0] for t in _angles(s, 1))
    else:
        cos, sin = _angles(s, s["frames"])
    yq, gq, gwq = _plain_head(q, s["gq"] if s["train"] else None, s["wq"], cos, sin, s)
    yk, gk, gwk = _plain_head(k, s["gk"] if s["train"] else None, s["wk"], cos, sin, s)
    return (yq, yk, gq, gk, gwq, gwk) if s["train"] else (yq, yk)


def _plain_scan_all(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis, h_{-1} = 0, by doubling.  In 64 bits: products of thousands of numbers near one"""
    n, d = a.shape[0], 1
    while d < n:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _frames_first(x):
    return x.double().transpose(0, 1)  # [T, B, C]


def _plain_gates(s):
    """(a, u) in 64 bits: what stays of the state, what is taken of the input"""
    f = _frames_first(s["forget"])
    return 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(f if s["input"] is None else -_frames_first(s["input"])))


def _plain_scan(s):
    x, (a, u) = _frames_first(s["x"]), _plain_gates(s)
    T, B, C = x.shape
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device=DEVICE)
    here = (torch.arange(T, device=DEVICE)[:, None] < n)[..., None]
    # behind a sequence's end the state stays what it is
    a, x = torch.where(here, a, 1), torch.where(here, x, 0)
    first = s["state0"].double() if s["state0"] is not None else torch.zeros(B, C, dtype=torch.float64, device=DEVICE)
    b = u * x
    h = _plain_scan_all(a, torch.cat([b[:1] + a[:1] * first, b[1:]]))
    out = torch.where(here, h, 0).transpose(0, 1).to(s["x"].dtype)
    last = h[-1].float()
    if not s["train"]:
        return out, last
    g = torch.where(here, _frames_first(s["gout"]), 0)
    if s["gstate"] is not None:
        g[-1] += s["gstate"]
    # e_t = g_t + a_{t+1} e_{t+1}
    e = _plain_scan_all(torch.cat([torch.zeros_like(a[:1]), a.flip(0)[:-1]]), g.flip(0)).flip(0)
    before = torch.cat([first[None], h[:-1]])
    taken = before - x if s["input"] is None else before
    grads = [torch.where(here, u * e, 0), torch.where(here, a * (1 - a) * e * taken, 0)]
    if s["input"] is not None:
        grads.append(torch.where(here, u * (1 - u) * e * x, 0))
    grads = [t.transpose(0, 1).to(s["x"].dtype) for t in grads]
    if s["input"] is None:
        grads.append(None)
    return (out, last, *grads, (a[0] * e[0]).float() if s["state"] else None)


def _plain_scan_step(s):
    x, f = s["x"].float(), s["forget"].float()
    a, u = 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(f if s["input"] is None else -s["input"].float()))
    s["state"].mul_(a).add_(u * x)
    return s["state"].to(s["x"].dtype), s["state"]


def _blocks(x):
    """(values by blocks, the blocks' scales in 32 bits)"""
    x = x.view(-1, BLOCK)
    return x, x.abs().amax(-1).float()


def _first_values(codes, scales):
    t = codes.view(-1, BLOCK).double() / 127
    return (t * t.abs() * scales[:, None]).view(-1)


def _second_values(codes, scales):
    t = (codes.view(-1, BLOCK).double() / 255).square()
    return (t * t * scales[:, None]).view(-1)


def _parts(x, scales):
    most = scales[:, None].double()
    return torch.where(most > 0, x.abs() / torch.where(most > 0, most, 1), 0)


def _pack_first(m):
    """First moments in 8 bits, the square of a code standing for a value: finer towards zero.  (Borders between codes are met in 64 bits.)"""
    m, scales = _blocks(m.double())
    codes = torch.round(127 * torch.sqrt(_parts(m, scales))) * torch.sign(m)
    return codes.to(torch.int8).view(-1), scales


def _dither(n, step):
    """A number in [0, 1) for each place and step: an additive sequence"""
    at = torch.arange(n, device=DEVICE) * 0x9E3779B9 + step * 0xB504F333
    return ((at & 0xFFFFFFFF) >> 8) * 2.0**-24


def _pack_second(v, step):
    """Second moments in 8 bits, the fourth power of a code standing for a value, rounded up or down by the place and the step; none that is not zero becomes zero"""
    v, scales = _blocks(v.double())
    codes = torch.floor(255 * torch.sqrt(torch.sqrt(_parts(v, scales))) + _dither(v.numel(), step).view(v.shape)).clamp(max=255)
    codes = torch.where(v > 0, codes.clamp(min=1), 0)
    return codes.to(torch.uint8).view(-1), scales


def _plain_adam(s):
    s["step"] += 1
    t, cut = s["step"], s["cut"]
    g = torch.cat([s["g"].float(), s["g32"]])
    if s["bits"] == 8:
        m, v = _first_values(s["m"], s["m_scales"]), _second_values(s["v"], s["v_scales"])
    else:
        m, v = s["m"], s["v"]
    g = g.to(m.dtype)
    m = m * BETAS[0] + g * (1 - BETAS[0])
    v = v * BETAS[1] + (g * g) * (1 - BETAS[1])
    p = s["master"] if s["master"] is not None else torch.cat([s["p"].float(), s["p32"]])
    by = m.float() / (torch.sqrt(v.float()) * (1 / math.sqrt(1 - BETAS[1] ** t)) + ADAM_EPS)
    p = p * (1 - LR * DECAY) - by * (LR / (1 - BETAS[0] ** t))
    s["p"].copy_(p[:cut])
    if s["master"] is not None:
        s["master"][:cut] = p[:cut]
        # (weights that are float32 themselves have no copy)
        p = s["p32"] * (1 - LR * DECAY) - by[cut:] * (LR / (1 - BETAS[0] ** t))
        s["p32"].copy_(p)
    else:
        s["p32"].copy_(p[cut:])
    if s["bits"] == 8:
        for name, (codes, scales) in (("m", _pack_first(m)), ("v", _pack_second(v, t))):
            s[name].copy_(codes)
            s[name + "_scales"].copy_(scales)
        m, v = _first_values(s["m"], s["m_scales"]).float(), _second_values(s["v"], s["v_scales"]).float()
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
        m, v = s["m"], s["v"]
    return s["p"], s["p32"], s["master"], m, v


def run(state):
    if own:
        return _run_own(state)
    return {"rotate": _plain_rotate, "scan": _plain_scan, "scan_step": _plain_scan_step, "adam": _plain_adam}[state["kind"]](state)


def work(case):
    kind = case["kind"]
    if kind == "rotate":
        n = case["batch"] * max(1, case["frames"]) * (case["heads"] + case["kheads"]) * case["width"]
        # q and k read, written; in training their gradients' way back, and they once more
        return dict(bytes=n * SIZE[case["dtype"]] * (2 + 3 * case["train"]), flops=n * (6 + 12 * case["train"]))
    if kind == "scan_step":
        n = case["batch"] * case["width"]
        return dict(bytes=n * (8 + SIZE[case["dtype"]] * (2 + case["gates"])), flops=n * 12)
    if kind == "scan":
        n = case["batch"] * case["frames"] * case["width"] * (0.65 if case["ragged"] else 1)
        arrays = 2 + case["gates"]  # the input, its gates and the output
        if case["train"]:
            arrays += 1 + 2 * (1 + case["gates"])  # the output's gradient; the input and its gates again, and their gradients
        return dict(bytes=n * SIZE[case["dtype"]] * arrays + case["batch"] * case["width"] * 8 * case["state"] * (1 + case["train"]),
                    flops=n * (14 + 24 * case["train"]))
    network, exact_ones = (sum(math.prod(x) for x in shapes) for shapes in _shapes(case))
    states = 16 if case["bits"] == 32 else 4 + 16 / BLOCK + 2 + 8  # read and written; in 8 bits also the values that the codes stand for
    narrow = case["dtype"] != "float32"  # gradient read, weight written, and its float32 copy read and written
    return dict(bytes=network * ((SIZE[case["dtype"]] * 2 + 8 if narrow else 12) + states) + exact_ones * (12 + states), flops=(network + exact_ones) * 16)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------


def _exact_rotate(s):
    """As products of complex numbers, gradients by autograd"""
    B = s["q"].shape[0]
    T = max(1, s["frames"])
    where = s["positions"].double().view(B, T) if s["positions"] is not None else torch.arange(T, device=DEVICE).double().expand(B, T)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE), where[..., None, None] * s["freqs"])
    pairs = s["freqs"].numel()

    def forward(x, w):
        v = x.view(B, T, -1, x.shape[-1])
        if s["norm"]:
            v = v / (v.pow(2).mean(-1, keepdim=True) + EPS).sqrt() * w
        head, rest = v[..., : 2 * pairs], v[..., 2 * pairs :]
        if s["interleaved"]:
            z = torch.view_as_real(torch.complex(head[..., 0::2].contiguous(), head[..., 1::2].contiguous()) * turn).flatten(-2)
        else:
            z = torch.complex(head[..., :pairs].contiguous(), head[..., pairs:].contiguous()) * turn
            z = torch.cat([z.real, z.imag], -1)
        return torch.cat([z, rest], -1).view(x.shape)

    outs, gxs, gws = [], [], []
    for name in "qk":
        x = s[name].double().contiguous().requires_grad_(s["train"])
        w = s["w" + name].double().requires_grad_(s["train"]) if s["norm"] else None
        y = forward(x, w)
        if s["train"]:
            got = torch.autograd.grad(y, [x] + ([w] if s["norm"] else []), s["g" + name].double())
            gxs.append(got[0])
            gws.append(got[1] if s["norm"] else None)
        outs.append(y.detach())
        del x, y
    return (*outs, *gxs, *gws)


def _exact_scan(s):
    """Frame by frame"""
    B, T, C = s["x"].shape
    count = s["lengths"] if s["lengths"] is not None else torch.full((B,), T, dtype=torch.int32, device=DEVICE)
    h = s["state0"].double() if s["state0"] is not None else torch.zeros(B, C, dtype=torch.float64, device=DEVICE)
    coupled = s["input"] is None

    def at(t):
        f = s["forget"][:, t].double()
        i = -f if coupled else s["input"][:, t].double()
        return s["x"][:, t].double(), torch.sigmoid(f), torch.sigmoid(i), torch.sigmoid(-f), torch.sigmoid(-i), (t < count)[:, None]

    out = torch.zeros(B, T, C, dtype=torch.float64, device=DEVICE)
    past = []
    for t in range(T):
        x, a, u, _, _, live = at(t)
        if s["train"]:
            past.append(h)
        h = torch.where(live, torch.addcmul(u * x, a, h), h)
        out[:, t] = torch.where(live, h, 0.0)
    if not s["train"]:
        return out, h
    gx, gf = torch.zeros_like(out), torch.zeros_like(out)
    gi = None if coupled else torch.zeros_like(out)
    e = s["gstate"].double() if s["gstate"] is not None else torch.zeros_like(h)
    for t in reversed(range(T)):
        x, a, u, na, nu, live = at(t)
        e = torch.where(live, e + s["gout"][:, t].double(), e)
        gx[:, t] = torch.where(live, u * e, 0.0)
        gf[:, t] = torch.where(live, e * a * na * ((past[t] - x) if coupled else past[t]), 0.0)
        if not coupled:
            gi[:, t] = torch.where(live, e * u * nu * x, 0.0)
        e = torch.where(live, a * e, e)
    return out, h, gx, gf, gi, e if s["state"] else None


def _exact_adam(s):
    t, cut = s["step"] + 1, s["cut"]
    b1, b2 = BETAS
    g = torch.cat([s["g"].double(), s["g32"].double()])
    m, v = s["m"].double(), s["v"].double()
    if s["bits"] == 8:
        m = (m / 127).square().mul(m.sign()) * s["m_scales"].double().repeat_interleave(BLOCK)
        v = (v / 255).pow(4) * s["v_scales"].double().repeat_interleave(BLOCK)
    m, v = torch.lerp(g, m, b1), torch.lerp(g.square(), v, b2)
    p = torch.cat([s["p"].double() if s["master"] is None else s["master"][:cut].double(), s["p32"].double()])
    p = p - LR * DECAY * p - LR * (m / (1 - b1**t)) / ((v / (1 - b2**t)).sqrt() + ADAM_EPS)
    if s["bits"] == 8:
        def kept(x, power, levels, shift):
            top = x.abs().reshape(-1, BLOCK).max(-1).values.float().double().repeat_interleave(BLOCK)
            y = (x.abs() / top).nan_to_num(0.0).pow(1 / power) * levels
            y = torch.floor(y + shift).clamp(max=levels)
            return y if power == 2 else torch.where(x > 0, y.clamp(min=1), y), top

        n = m.numel()
        shift = torch.remainder(torch.arange(n, device=DEVICE) * 0x9E3779B9 + t * 0xB504F333, 1 << 32).div(256, rounding_mode="floor").double() / 2**24
        c, top = kept(m, 2, 127, 0.5)
        m = m.sign() * (c / 127) ** 2 * top
        c, top = kept(v, 4, 255, shift)
        v = (c / 255) ** 4 * top
    master = None if s["master"] is None else torch.cat([p[:cut], s["master"][cut:].double()])
    return p[:cut], p[cut:], master, m, v


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "rotate":
        return _exact_rotate(s)
    if kind == "adam":
        return _exact_adam(s)
    if kind == "scan":
        return _exact_scan(s)
    f = s["forget"].double()
    h = s["state"].double() * torch.sigmoid(f) + s["x"].double() * torch.sigmoid(-f if s["input"] is None else s["input"].double())
    return h, h
