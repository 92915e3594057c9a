"""The work that the speed of this library's sequence operators is measured on: layer norm, activation checkpoints in
8 bits, and linear attention with a decay for each head.

Every case is one call, or one training step, that a network on top of the spectrogram layers makes over and over.  ``own``
chooses between the library's calls and their plain form in elementary torch operations; both take the same state.  The
listed sizes go from a single frame of a stream to long training sequences; ``draw`` spreads further ones over the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-5
BLOCK = 128  # values that share a scale
CHUNK = 64   # frames the plain form of the attention takes at a time


def listed():
    return [
        # one frame of a stream through a layer norm: launch and host time count
        dict(name="norm_frame", kind="norm", train=False, rows=1, width=512, dtype="bfloat16"),
        # 64 clips of five seconds, 128 Mel bands [B, bins, T], to tokens of a bfloat16 network, and back
        dict(name="norm_mel", kind="norm_frames", train=True, batch=64, width=128, frames=216, out="bfloat16"),
        # the bins of a 2,048-sample STFT, ten seconds of 16 tracks, float32 throughout
        dict(name="norm_stft", kind="norm_frames", train=True, batch=16, width=1025, frames=431, out="float32"),
        # a wide network's tokens
        dict(name="norm_wide", kind="norm", train=True, rows=65536, width=2048, dtype="bfloat16"),
        # the tokens of 16 tracks of ten seconds, their activations kept in 8 bits for the backward pass
        dict(name="norm8_tracks", kind="norm8", train=True, rows=6896, width=512, dtype="float32"),
        # a large training batch, kept in 8 bits
        dict(name="norm8_batch", kind="norm8", train=True, rows=131072, width=1024, dtype="bfloat16"),
        # what a trainable STFT layer keeps of 16 clips (float32 products of all kernels, flat), to 8 bits and back
        dict(name="pack8_kept", kind="pack8", rows=1, width=3063808, dtype="float32"),
        # one new frame of one stream
        dict(name="step_one", kind="step", batch=1, heads=8, dk=64, dv=64, dtype="bfloat16"),
        # one new frame of each of 256 streams
        dict(name="step_streams", kind="step", batch=256, heads=16, dk=128, dv=128, dtype="bfloat16"),
        # a recording of three minutes (hop 256 at 22.05 kHz) as the prompt of a stream: outputs and the state to go on from
        dict(name="decay_song", kind="decay", train=False, batch=1, heads=8, frames=15504, dk=64, dv=64, dtype="bfloat16",
             ragged=False, state=True),
        # training on 16 clips of up to ten seconds, lengths differ, float32, states carried from the clips' earlier parts
        dict(name="decay_clips", kind="decay", train=True, batch=16, heads=8, frames=431, dk=64, dv=64, dtype="float32",
             ragged=True, state=True),
        # training on long sequences
        dict(name="decay_long", kind="decay", train=True, batch=4, heads=16, frames=16384, dk=128, dv=128, dtype="bfloat16",
             ragged=False, state=False),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm_frames", "norm8", "norm8", "pack8", "step", "decay", "decay", "decay"])
    dtype = rng.choice(["float32", "bfloat16"])
    if kind in ("norm", "norm8"):
        width = rng.choice([_log_between(rng, 64, 4096), 64 * _log_between(rng, 1, 64)])
        rows = _log_between(rng, 1, (1 << 27 if dtype == "bfloat16" else 1 << 26) // width)
        return dict(kind=kind, train=kind == "norm8" or rng.random() < 0.7, rows=rows, width=width, dtype=dtype)
    if kind == "norm_frames":
        # Mel bands, constant-Q bins or Fourier bins of clips of one second to a minute
        width = rng.choice([40, 64, 80, 84, 128, 168, 229, 256, 257, 513, 1025])
        frames = _log_between(rng, 20, 2600)
        batch = _log_between(rng, 1, max(1, (1 << 25) // (width * frames)))
        return dict(kind=kind, train=True, batch=batch, width=width, frames=frames, out=dtype)
    if kind == "pack8":
        return dict(kind=kind, rows=rng.choice([1, 1, _log_between(rng, 2, 500)]), width=_log_between(rng, 1000, 100000), dtype=dtype)
    heads = rng.choice([1, 2, 4, 8, 12, 16])
    dk, dv = rng.choice([32, 48, 64, 64, 96, 128]), rng.choice([32, 48, 64, 64, 96, 128])
    if kind == "step":
        return dict(kind=kind, batch=_log_between(rng, 1, 256), heads=heads, dk=dk, dv=dv, dtype=dtype)
    frames = _log_between(rng, 10, 16000)
    most = (1 << 27 if dtype == "bfloat16" else 1 << 25) // (heads * frames * max(dk, dv))
    return dict(kind=kind, train=rng.random() < 0.7, batch=_log_between(rng, 1, max(1, min(64, most))), heads=heads, frames=frames, dk=dk,
                dv=dv, dtype=dtype, ragged=rng.random() < 0.5, state=rng.random() < 0.5)


def _activations(g, rows, width):
    """Values of a residual stream: channels of different scale and offset, a few of them much larger."""
    gain = torch.exp(0.5 * torch.randn(width, device=DEVICE, generator=g))
    gain = torch.where(torch.rand(width, device=DEVICE, generator=g) < 0.01, 20 * gain, gain)
    return torch.randn(rows, width, device=DEVICE, generator=g) * gain + 0.3 * torch.randn(width, device=DEVICE, generator=g)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(int(seed))
    s = dict(case)

    def normal(*shape):
        return torch.randn(*shape, device=DEVICE, generator=g)

    kind = case["kind"]
    if kind in ("norm", "norm8", "norm_frames"):
        width = case["width"]
        s["weight"], s["bias"] = 1 + 0.2 * normal(width), 0.1 * normal(width)
        if kind == "norm_frames":
            # a power spectrogram on a logarithmic scale [B, bins, T], as the layers write it: neighbouring frames alike, less power higher up
            shape = (case["batch"], width, case["frames"])
            spec = 2 * normal(*shape) + 2 * normal(shape[0], 1, shape[2]) - torch.linspace(0, 8, width, device=DEVICE)[:, None]
            s["x"] = spec.transpose(1, 2)
            s["out_dtype"] = getattr(torch, case["out"])
            s["gout"] = normal(shape[0], shape[2], width).to(s["out_dtype"])
        else:
            dtype = getattr(torch, case["dtype"])
            s["x"] = _activations(g, case["rows"], width).to(dtype)
            s["out_dtype"] = dtype
            s["gout"] = normal(case["rows"], width).to(dtype)
    elif kind == "pack8":
        s["x"] = _activations(g, 1, case["width"]).expand(case["rows"], -1).mul(normal(case["rows"], 1)).to(getattr(torch, case["dtype"]))
    else:
        B, H, dk, dv, dtype = case["batch"], case["heads"], case["dk"], case["dv"], getattr(torch, case["dtype"])
        T = case.get("frames", 1)
        # queries, keys and values as one projection of the frames gives them
        qkv = normal(B, T, H * (2 * dk + dv)).to(dtype)
        s["q"] = qkv[..., : H * dk].view(B, T, H, dk)
        s["k"] = qkv[..., H * dk : 2 * H * dk].view(B, T, H, dk)
        s["v"] = qkv[..., 2 * H * dk :].view(B, T, H, dv)
        # heads that remember from about 30 frames to some thousands
        s["decay"] = 1 - torch.exp2(-5 - 7 * (torch.arange(H, device=DEVICE) + torch.rand(H, device=DEVICE, generator=g)) / H)
        if kind == "step":
            s["q"], s["k"], s["v"] = s["q"][:, 0], s["k"][:, 0], s["v"][:, 0]
            s["state"] = 3 * normal(B, H, dk, dv)
        else:
            s["state0"] = 3 * normal(B, H, dk, dv) if case["state"] else None
            s["gstate"] = normal(B, H, dk, dv) if case["state"] and case["train"] else None
            s["lengths"] = None
            if case["ragged"]:
                s["lengths"] = (T * (0.3 + 0.7 * torch.rand(B, device=DEVICE, generator=g))).round().to(torch.int32)
            s["gout"] = normal(B, T, H, dv).to(dtype) if case["train"] else None
    return s


# ---- the library's calls ---------------------------------------------------------------------------------------------


def _run_own(s):
    from paper_1912_12055_amd import binding as nb

    kind = s["kind"]
    if kind in ("norm", "norm8", "norm_frames"):
        if not s["train"]:
            return nb.nna_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, out_dtype=s["out_dtype"])
        y, kept = nb.nna_layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, out_dtype=s["out_dtype"], keep=8 if kind == "norm8" else 32)
        return (y, *nb.nna_layer_norm_backward(s["gout"], kept, s["weight"]))
    if kind == "pack8":
        codes, scales = nb.nna_pack8(s["x"])
        return nb.nna_unpack8(codes, scales, dtype=s["x"].dtype), scales
    if kind == "step":
        return nb.nna_decay_attention_step(s["q"], s["k"], s["v"], s["decay"], s["state"]), s["state"]
    q, k, v, decay, state, lengths = s["q"], s["k"], s["v"], s["decay"], s["state0"], s["lengths"]
    o, last = nb.nna_decay_attention(q, k, v, decay, state=state, lengths=lengths, want_state=True) if s["state"] else (
        nb.nna_decay_attention(q, k, v, decay, lengths=lengths), None)
    if not s["train"]:
        return o, last
    return (o, last, *nb.nna_decay_attention_backward(s["gout"], q, k, v, decay, state=state, lengths=lengths, gstate=s["gstate"],
                                                      want_gstate=s["state"]))


# ---- their plain form ------------------------------------------------------------------------------------------------


def _plain_norm(s):
    x, w, b = s["x"].float(), s["weight"], s["bias"]
    mean = x.mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt((x - mean).square().mean(-1, keepdim=True) + EPS)
    y = ((x - mean) * rstd * w + b).to(s["out_dtype"])
    if not s["train"]:
        return y
    kept = _plain_unpack8(*_plain_pack8(x)) if s["kind"] == "norm8" else x
    h, g = (kept - mean) * rstd, s["gout"].float()
    gh = g * w
    gx = rstd * (gh - gh.mean(-1, keepdim=True) - h * (gh * h).mean(-1, keepdim=True))
    rows = tuple(range(g.dim() - 1))
    return y, gx.to(s["x"].dtype), (g * h).sum(rows), g.sum(rows)


def _plain_pack8(x):
    rows, width = x.shape
    blocks = -(-width // BLOCK)
    v = torch.nn.functional.pad(x.float(), (0, blocks * BLOCK - width)).view(rows, blocks, BLOCK)
    most = v.abs().amax(-1, keepdim=True)
    fine = most >= 2.0**-100
    codes = torch.where(fine, torch.round(v * (torch.full_like(most, 127) / most)), 0).to(torch.int8).view(rows, -1)[:, :width]
    return codes, torch.where(fine, most * (1 / 127), 0)[..., 0]


def _plain_unpack8(codes, scales):
    return codes.float() * scales.repeat_interleave(BLOCK, 1)[:, : codes.shape[1]]


def _heads_first(x):
    return x.float().transpose(1, 2).contiguous()  # [B, H, T, D]


def _plain_mix(a, b, c, decay):
    """sum over j <= i of decay^(i-j) (a_i . b_j) c_j, a chunk of frames at a time: within chunks by their products, across them by the
    chunks' states."""
    B, H, T, _ = a.shape
    n = -(-T // CHUNK)
    a, b, c = (torch.nn.functional.pad(x, (0, 0, 0, n * CHUNK - T)).view(B, H, n, CHUNK, -1) for x in (a, b, c))
    i = torch.arange(CHUNK, device=a.device)
    d = decay[:, None]
    apart = i[:, None] - i
    within = torch.where(apart >= 0, d[..., None] ** apart.clamp(min=0), 0)  # [H, C, C]
    o = ((a @ b.transpose(-1, -2).contiguous()) * within[:, None]) @ c
    state = (b * (d ** (CHUNK - 1 - i))[:, None, :, None]).transpose(-1, -2).contiguous() @ c  # of each chunk alone
    m = torch.arange(n, device=a.device)
    gap = m[:, None] - 1 - m
    across = torch.where(gap >= 0, (d**CHUNK)[..., None] ** gap.clamp(min=0), 0)  # [H, n, n]
    before = (across @ state.view(B, H, n, -1)).view(state.shape)
    o = o + (a * (d ** (i + 1))[:, None, :, None]) @ before
    return o.view(B, H, n * CHUNK, -1)[:, :, :T]


def _flip(x):
    return torch.flip(x, (2,))


def _plain_decay(s):
    q, k, v, decay = _heads_first(s["q"]), _heads_first(s["k"]), _heads_first(s["v"]), s["decay"]
    B, H, T, dk = q.shape
    q = q * dk**-0.5
    t = torch.arange(T, device=q.device)
    n = s["lengths"].long() if s["lengths"] is not None else torch.full((B,), T, device=q.device)
    here = (t < n[:, None])[:, None, :, None]  # [B, 1, T, 1]
    q, k, v = (torch.where(here, x, 0) for x in (q, k, v))
    d = decay[:, None]
    since = (d ** (t + 1))[None, :, :, None]                                  # of the first state, at each frame
    left = torch.where(here, (d ** (n[:, None, None] - 1 - t).clamp(min=0))[..., None], 0)  # of each frame, in the last state
    whole = (d ** n[:, None, None])[..., None]                                # of the first state, in the last
    o = _plain_mix(q, k, v, decay)
    last = None
    if s["state0"] is not None:
        o = o + (q * since) @ s["state0"]
        last = whole * s["state0"] + (k * left).transpose(-1, -2).contiguous() @ v
    out = [o.transpose(1, 2).to(s["q"].dtype), last]
    if not s["train"]:
        return tuple(out)
    g = torch.where(here, _heads_first(s["gout"]), 0)
    gq = _plain_mix(g, v, k, decay)
    gk = _flip(_plain_mix(_flip(v), _flip(g), _flip(q), decay))
    gv = _flip(_plain_mix(_flip(k), _flip(q), _flip(g), decay))
    gfirst = None
    if s["state0"] is not None:
        gq = gq + (g * since) @ s["state0"].transpose(-1, -2).contiguous()
        gk = gk + (v * left) @ s["gstate"].transpose(-1, -2).contiguous()
        gv = gv + (k * left) @ s["gstate"]
        gfirst = whole * s["gstate"] + (q * since).transpose(-1, -2).contiguous() @ g
    grads = [x.transpose(1, 2).to(s["q"].dtype) for x in (gq * dk**-0.5, gk, gv)]
    return (*out, *grads, gfirst)


def _plain_step(s):
    q, k, v = s["q"].float() * s["q"].shape[-1] ** -0.5, s["k"].float(), s["v"].float()
    s["state"].mul_(s["decay"][:, None, None]).add_(k[..., None] * v[..., None, :])
    return (q[..., None] * s["state"]).sum(-2).to(s["q"].dtype), s["state"]


def run(state):
    if own:
        return _run_own(state)
    if state["kind"] in ("norm", "norm8", "norm_frames"):
        return _plain_norm(state)
    if state["kind"] == "pack8":
        codes, scales = _plain_pack8(state["x"])
        return _plain_unpack8(codes, scales).to(state["x"].dtype), scales
    return _plain_step(state) if state["kind"] == "step" else _plain_decay(state)


def work(case):
    kind = case["kind"]
    size = {"float32": 4, "bfloat16": 2}
    if kind in ("norm", "norm8"):
        n, e = case["rows"] * case["width"], size[case["dtype"]]
        # x and y; in training gy, x again (or its 8 bits, written and read) and gx
        moved = 2 * e + (3 * e if kind == "norm" else 2 * e + 2 * (1 + 4 / BLOCK)) * case["train"]
        return dict(bytes=n * moved + 8 * case["width"], flops=n * (8 + 14 * case["train"]))
    if kind == "norm_frames":
        n, e = case["batch"] * case["frames"] * case["width"], size[case["out"]]
        return dict(bytes=n * (4 + e + (e + 8) * case["train"]) + 8 * case["width"], flops=n * (8 + 14 * case["train"]))
    if kind == "pack8":
        n, e = case["rows"] * case["width"], size[case["dtype"]]
        return dict(bytes=n * (2 * e + 2 * (1 + 4 / BLOCK)), flops=4 * n)
    heads, dk, dv, e = case["batch"] * case["heads"], case["dk"], case["dv"], size[case["dtype"]]
    if kind == "step":
        return dict(bytes=heads * (8 * dk * dv + e * (2 * dk + 2 * dv)), flops=heads * 5 * dk * dv)
    tokens = heads * case["frames"] * (0.65 if case["ragged"] else 1)
    moved, flops = tokens * e * (2 * dk + 2 * dv), tokens * 4 * dk * dv  # by the recurrence: the fewest operations
    if case["train"]:
        moved, flops = moved + tokens * e * (4 * dk + 3 * dv), flops + tokens * 10 * dk * dv
    return dict(bytes=moved + heads * (8 + 8 * case["train"]) * dk * dv * case["state"], flops=flops)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------


def _exact_blocks(x):
    """(values the codes stand for, scales) of rows in 64 bits."""
    rows, width = x.shape
    blocks = (width + BLOCK - 1) // BLOCK
    v = torch.zeros(rows, blocks * BLOCK, dtype=torch.float64, device=x.device)
    v[:, :width] = x
    v = v.reshape(rows, blocks, BLOCK)
    scale = v.abs().max(-1).values / 127
    return (torch.round(v / scale[..., None]).nan_to_num(0.0) * scale[..., None]).reshape(rows, -1)[:, :width], scale


def _exact_norm(s):
    x = s["x"].double()
    var, mean = torch.var_mean(x, -1, correction=0, keepdim=True)
    r = (var + EPS).rsqrt()
    y = torch.addcmul(s["bias"].double(), (x - mean) * r, s["weight"].double())
    if not s["train"]:
        return y
    if s["kind"] == "norm8":
        x = _exact_blocks(x)[0]
    h, g = (x - mean) * r, s["gout"].double()
    D = h.shape[-1]
    a = g * s["weight"].double()
    gx = (D * a - a.sum(-1, keepdim=True) - h * (a * h).sum(-1, keepdim=True)) * r / D
    return y, gx, (g * h).flatten(0, -2).sum(0), g.flatten(0, -2).sum(0)


def _exact_decay(s):
    """Each (sequence, head) by itself: all pairs of its frames."""
    B, T, H, dk = s["q"].shape
    dv = s["v"].shape[-1]
    zeros = lambda n: torch.zeros(B, T, H, n, dtype=torch.float64, device=DEVICE)  # noqa: E731
    o, gq, gk, gv = zeros(dv), zeros(dk), zeros(dk), zeros(dv)
    last = torch.zeros(B, H, dk, dv, dtype=torch.float64, device=DEVICE)
    gfirst = torch.zeros_like(last)
    lengths = s["lengths"].tolist() if s["lengths"] is not None else [T] * B
    for h in range(H):
        decay = float(s["decay"][h])
        power = torch.tensor(decay, dtype=torch.float64, device=DEVICE) ** torch.arange(T + 1, device=DEVICE)
        for b, n in enumerate(lengths):
            q, k, v = (s[x][b, :n, h].double() for x in "qkv")
            q = q / math.sqrt(dk)
            t = torch.arange(n, device=DEVICE)
            gap = t[:, None] - t
            D = torch.where(gap < 0, 0.0, power[gap.clamp(min=0)])
            first = s["state0"][b, h].double() if s["state0"] is not None else torch.zeros_like(last[0, 0])
            since, left = power[1 : n + 1, None], power[:n].flip(0)[:, None]
            A = (q @ k.T).mul_(D)
            o[b, :n, h] = A @ v + since * (q @ first)
            last[b, h] = power[n] * first + (left * k).T @ v
            if s["train"]:
                g = s["gout"][b, :n, h].double()
                glast = s["gstate"][b, h].double() if s["gstate"] is not None else torch.zeros_like(first)
                gv[b, :n, h] = A.T @ g + left * (k @ glast)
                A = (g @ v.T).mul_(D)
                gq[b, :n, h] = (A @ k + since * (g @ first.T)) / math.sqrt(dk)
                gk[b, :n, h] = A.T @ q + left * (v @ glast.T)
                gfirst[b, h] = power[n] * glast + (since * q).T @ g
    has = s["state0"] is not None
    return (o, last if has else None) + ((gq, gk, gv, gfirst if has else None) if s["train"] else ())


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("norm", "norm8", "norm_frames"):
        return _exact_norm(s)
    if kind == "pack8":
        return _exact_blocks(s["x"].double())
    if kind == "step":
        state = s["decay"].double()[:, None, None] * s["state"].double() + s["k"].double()[..., None] * s["v"].double()[..., None, :]
        return (s["q"].double()[..., None] * state).sum(-2) / math.sqrt(case["dk"]), state
    return _exact_decay(s)
