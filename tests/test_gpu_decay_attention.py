"""Linear attention with a decay for each head against its definition in 64 bits (all pairs of frames), forward, backward and frame by frame.

Tolerances.  With M the same sums over magnitudes, float32 results are off by at most C 2^-24 M: C counts the products summed one after the other
(dk + dv + 192 in a chunk and two a chunk after it) and the powers (an exponent of up to 126 is rounded twice: 256).  With bfloat16 the weights and the
state are rounded once where they are multiplied (2^-8 of M at most), and so is the result (2^-8 of it); over many values of either
sign the roundings add as squares: together at most 2^-8 of the result's norm.
"""
import math
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32, U16 = 2.0**-24, 2.0**-8


@pytest.fixture(scope="module")
def nb():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU (there is no CPU fallback)")
    from paper_1912_12055_amd import binding
    binding.lib()
    return binding


def _say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def _inputs(B, T, H, dk, dv, dtype, seed=0, state=True):
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*s):
        return torch.randn(*s, device=DEV, generator=g)

    q, k, v, go = (normal(B, T, H, d).to(dtype) for d in (dk, dk, dv, dv))
    decay = 1 - 2.0 ** (-1 - 8 * torch.rand(H, device=DEV, generator=g))
    first, glast = (normal(B, H, dk, dv), normal(B, H, dk, dv)) if state else (None, None)
    return q, k, v, go, decay, first, glast


def _exact(q, k, v, decay, first=None, lengths=None, go=None, glast=None, scale=None):
    """{name: (value, magnitude)} by the definition, each (sequence, head) over all pairs of its frames"""
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    scale = dk**-0.5 if scale is None else scale
    lengths = [T] * B if lengths is None else [min(max(int(n), 0), T) for n in lengths]
    shape = dict(o=(B, T, H, dv), gq=(B, T, H, dk), gk=(B, T, H, dk), gv=(B, T, H, dv), last=(B, H, dk, dv), gfirst=(B, H, dk, dv))
    out = {name: (torch.zeros(s, dtype=torch.float64, device=DEV), torch.zeros(s, dtype=torch.float64, device=DEV)) for name, s in shape.items()}
    for b, n in enumerate(lengths):
        for h in range(H):
            for m, fn in enumerate((lambda x: x, torch.abs)):
                l = float(decay[h])
                Q, K, V = (fn(x[b, :n, h].double()) for x in (q, k, v))
                S = torch.zeros(dk, dv, dtype=torch.float64, device=DEV) if first is None else fn(first[b, h].double())
                t = torch.arange(n, device=DEV)
                gap = (t[:, None] - t).double()
                D = torch.where(gap >= 0, torch.tensor(l, dtype=torch.float64, device=DEV) ** gap.clamp(min=0), 0)
                L = torch.tensor(l, dtype=torch.float64, device=DEV)
                since, left = (L ** (t + 1).double())[:, None], (L ** (n - 1 - t).double())[:, None]
                sc = scale if m == 0 else abs(scale)
                W = sc * (Q @ K.T) * D
                out["o"][m][b, :n, h] = W @ V + sc * since * (Q @ S)
                out["last"][m][b, h] = L**n * S + (left * K).T @ V
                if go is not None:
                    G = fn(go[b, :n, h].double())
                    GS = torch.zeros_like(S) if glast is None else fn(glast[b, h].double())
                    out["gv"][m][b, :n, h] = W.T @ G + left * (K @ GS)
                    W = sc * (G @ V.T) * D
                    out["gq"][m][b, :n, h] = W @ K + sc * since * (G @ S.T)
                    out["gk"][m][b, :n, h] = W.T @ Q + left * (V @ GS.T)
                    out["gfirst"][m][b, h] = L**n * GS + sc * (since * Q).T @ G
    return out


def _close(got, exact, name, T, dk, dv):
    ref, most = exact[name]
    assert got.shape == ref.shape, name
    assert torch.isfinite(got).all(), name
    d = (got.double() - ref).abs()
    bound = (dk + dv + 192 + 2 * (T // 64) + 256) * U32 * most + 1e-37
    if got.dtype == torch.bfloat16:
        bound = bound + U16 * (ref.abs() + 1.01 * most)
        if got.numel() > 1000:
            assert d.norm() <= U16 * ref.norm(), (name, float(d.norm() / ref.norm()))
    worst = float((d / bound).max()) if d.numel() else 0.0
    assert worst <= 1, (name, worst)


def _check(nb, q, k, v, go, decay, first, glast, lengths=None, scale=None):
    B, T, H, dk = q.shape
    dv = v.shape[-1]
    e = _exact(q, k, v, decay, first, lengths, go, glast, scale)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device=DEV)
    o, last = nb.nna_decay_attention(q, k, v, decay, scale=scale, state=first, lengths=n, want_state=True)
    gq, gk, gv, gfirst = nb.nna_decay_attention_backward(go, q, k, v, decay, scale=scale, state=first, lengths=n, gstate=glast, want_gstate=True)
    assert {x.dtype for x in (o, gq, gk, gv)} == {q.dtype}
    for name, x in dict(o=o, last=last, gq=gq, gk=gk, gv=gv, gfirst=gfirst).items():
        _close(x, e, name, T, dk, dv)
    return o, last, gq, gk, gv, gfirst


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [1, 2, 15, 63, 64, 65, 128, 129, 200, 431])
def test_every_length(nb, dtype, T):
    for state in (True, False):
        _say("T", T, dtype, state)
        _check(nb, *_inputs(2, T, 3, 64, 64, dtype, seed=T, state=state))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dk,dv", [(1, 1), (3, 5), (16, 32), (32, 7), (64, 128), (128, 64), (65, 63), (48, 96), (100, 128), (128, 128), (127, 33)])
def test_every_head_size(nb, dtype, dk, dv):
    _say("heads", dk, dv, dtype)
    _check(nb, *_inputs(2, 150, 2, dk, dv, dtype, seed=dk + dv))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,H,dk,dv", [(1, 5000, 1, 64, 64), (1, 2111, 3, 128, 128), (3, 1025, 5, 64, 128), (2, 3000, 4, 40, 24), (600, 70, 2, 32, 32)])
def test_long_sequences_in_segments_and_many_short_ones(nb, dtype, B, T, H, dk, dv):
    _say("segments", B, T, H, dk, dv, dtype, nb.nna_decay_attention_workspace(B, T, H, dk, dv))
    args = _inputs(B, T, H, dk, dv, dtype, seed=T)
    args[4][0] = 1 - 2.0**-11  # a head that remembers across segments
    _check(nb, *args)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,lengths", [(200, [0, 200, 1, 64, 65, 199, 128]), (2000, [2000, 0, 700, 1999, 512, 1]), (70, [-3, 1000, 64, 5])])
def test_lengths_and_what_lies_past_them(nb, dtype, T, lengths):
    _say("lengths", T, lengths, dtype)
    q, k, v, go, decay, first, glast = _inputs(len(lengths), T, 2, 64, 96, dtype, seed=T)
    whole = _check(nb, q, k, v, go, decay, first, glast, lengths)
    for b, n in enumerate(lengths):  # infinities and NaN past the end change nothing
        for x in (q, k, v, go):
            x[b, max(n, 0):] = float("nan")
            x[b, max(n, 0)::2] = float("inf")
    n = torch.tensor(lengths, dtype=torch.int32, device=DEV)
    again = (*nb.nna_decay_attention(q, k, v, decay, state=first, lengths=n, want_state=True),
             *nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, lengths=n, gstate=glast, want_gstate=True))
    assert all(torch.equal(a, c) for a, c in zip(whole, again))
    for b, n in enumerate(lengths):
        n = min(max(n, 0), T)
        assert not any(x[b, n:].any() for x in (whole[0], *whole[2:5]))
        if n == 0:
            assert torch.equal(whole[1][b], first[b])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_shared_heads_and_orders(nb, dtype):
    B, T, H, dk, dv = 2, 130, 4, 40, 56
    g = torch.Generator(device=DEV).manual_seed(2)
    wide = torch.randn(B, T, 1 + H * (2 * dk + dv) + 3, device=DEV, generator=g).to(dtype)
    q = wide[..., 1:1 + H * dk].unflatten(-1, (H, dk))
    k = wide[..., 1 + H * dk:1 + 2 * H * dk].unflatten(-1, (H, dk))
    v = wide[..., 1 + 2 * H * dk:1 + H * (2 * dk + dv)].unflatten(-1, (H, dv))
    _, _, _, go, decay, first, glast = _inputs(B, T, H, dk, dv, dtype)
    _check(nb, q, k, v, go, decay, first, glast)  # parts of one projection, no start aligned
    hq, hk, hv = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (q, k, v))
    _check(nb, hq, hk, hv, go, decay, first, glast)  # [B, H, T, d] in memory
    shared = k[:, :, :1].expand(B, T, H, dk), v[:, :, 1:2].expand(B, T, H, dv)
    _check(nb, q, *shared, go, decay, first, glast)  # keys and values that the heads share
    _check(nb, q[:1].expand(B, T, H, dk), k, v, go, decay, first, glast)  # queries that the sequences share
    _check(nb, q.flip(1)[:, ::2], k[:, ::2], v[:, 1::2], go[:, :65].contiguous(), decay, first, glast)


def test_gradients_of_shared_heads_through_autograd_sums(nb):
    """what autograd makes of an expanded input: the sum of the heads' gradients"""
    q, k, v, go, decay, _, _ = _inputs(1, 90, 4, 32, 32, torch.float32, state=False)
    k1 = k[:, :, :1]
    gk = nb.nna_decay_attention_backward(go, q, k1.expand(-1, -1, 4, -1), v, decay)[1].sum(2, keepdim=True)
    e = _exact(q, k1.expand(-1, -1, 4, -1), v, decay, go=go)["gk"]
    assert ((gk.double() - e[0].sum(2, keepdim=True)).abs() <= 800 * U32 * e[1].sum(2, keepdim=True)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decays_of_zero_one_and_near_them(nb, dtype):
    q, k, v, go, decay, first, glast = _inputs(1, 300, 6, 64, 64, dtype, seed=4)
    decay[:] = torch.tensor([0.0, 1.0, 1e-30, 1 - 2.0**-24, 0.5, 1e-3], device=DEV)
    _check(nb, q, k, v, go, decay, first, glast)
    o = nb.nna_decay_attention(q, k, v, decay)[:, :, 0]
    alone = (q[:, :, 0].double() * k[:, :, 0].double()).sum(-1, keepdim=True) * v[:, :, 0].double() / 8  # a head without memory
    assert (o.double() - alone).norm() <= U16 * alone.norm()


@pytest.mark.parametrize("scale", [1.0, -0.3, 7.5])
def test_scales(nb, scale):
    _check(nb, *_inputs(2, 100, 2, 32, 32, torch.float32, seed=8), scale=scale)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [100, 1500])
def test_a_value_that_is_not_finite_reaches_no_frame_before_it(nb, dtype, T):
    q, k, v, go, decay, first, glast = _inputs(2, T, 2, 64, 64, dtype, seed=6)
    clean = (*nb.nna_decay_attention(q, k, v, decay, state=first, want_state=True), *nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, gstate=glast, want_gstate=True))
    at = 77
    for x, value in ((v, float("nan")), (v, float("inf")), (k, float("nan")), (k, -float("inf")), (q, float("nan"))):
        _say("not finite", "qkv"[[id(q), id(k), id(v)].index(id(x))], value, dtype, T)
        keep = x.clone()
        x[1, at, 0, 5] = value
        o, last = nb.nna_decay_attention(q, k, v, decay, state=first, want_state=True)
        assert torch.equal(o[0], clean[0][0]) and torch.equal(o[:, :, 1], clean[0][:, :, 1]) and torch.equal(o[1, :at], clean[0][1, :at])
        assert not torch.isfinite(o[1, at, 0]).all()
        if x is q:
            assert torch.equal(o[1, at + 1:], clean[0][1, at + 1:]) and torch.equal(last, clean[1])
        else:
            assert not torch.isfinite(o[1, T - 1, 0]).all() and not torch.isfinite(last[1, 0]).all()
        if x is v:
            assert torch.isnan(o[1, at:, 0]).all() and torch.isnan(last[1, 0]).all()
        x.copy_(keep)
    go[1, at, 0, 3] = float("inf")  # the gradients of frames after it do not know it
    gq, gk, gv, gfirst = nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, gstate=glast, want_gstate=True)
    for got, ref in zip((gk, gv), clean[3:5]):
        assert torch.equal(got[1, at + 1:], ref[1, at + 1:]) and torch.equal(got[0], ref[0])
    others = [t for t in range(T) if t != at]
    assert torch.equal(gq[1, others], clean[2][1, others]) and torch.isnan(gv[1, at, 0]).all()


def test_the_same_inputs_give_the_same_bits(nb):
    q, k, v, go, decay, first, glast = _inputs(2, 3000, 4, 64, 64, torch.bfloat16)
    for _ in range(2):
        runs = [(*nb.nna_decay_attention(q, k, v, decay, state=first, want_state=True), *nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, gstate=glast, want_gstate=True)) for _ in range(2)]
        assert all(torch.equal(a, c) for a, c in zip(*runs))


def test_gradients_against_differences(nb):
    """out and the last state are linear in each of q, k and v: the difference along a direction is exact but for rounding, C 2^-24 of the
    magnitudes at either end."""
    q, k, v, go, decay, first, glast = _inputs(2, 150, 2, 32, 40, torch.float32, seed=12)
    go, glast = go.contiguous(), glast.contiguous()

    def loss(q, k, v, first):
        o, last = nb.nna_decay_attention(q, k, v, decay, state=first, want_state=True)
        return float((go.double() * o.double()).sum() + (glast.double() * last.double()).sum())

    gq, gk, gv, gfirst = nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, gstate=glast, want_gstate=True)
    e = _exact(q, k, v, decay, first, None, go, glast)
    size = float((e["o"][1] * go.abs()).sum() + (e["last"][1] * glast.abs()).sum())
    g = torch.Generator(device=DEV).manual_seed(1)
    args = dict(q=q, k=k, v=v, first=first)
    for name, grad in (("q", gq), ("k", gk), ("v", gv), ("first", gfirst)):
        d = torch.randn(args[name].shape, device=DEV, generator=g)
        up, down = (loss(**{**args, name: args[name] + s * d}) for s in (1, -1))
        got = float((grad.double() * d.double()).sum())
        assert abs(got - (up - down) / 2) <= 1000 * U32 * 4 * size, name


# ---- frame by frame ----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,H,dk,dv", [(1, 1, 1, 1), (1, 8, 64, 64), (3, 2, 33, 31), (2, 3, 128, 128), (5, 4, 96, 50), (300, 2, 64, 128)])
def test_frames_one_by_one(nb, dtype, B, H, dk, dv):
    _say("step", B, H, dk, dv, dtype)
    T = 20
    q, k, v, go, decay, first, _ = _inputs(B, T, H, dk, dv, dtype, seed=B + dk)
    e = _exact(q, k, v, decay, first)
    state = first.clone()
    for t in range(T):
        o = nb.nna_decay_attention_step(q[:, t], k[:, t], v[:, t], decay, state)
        ref, most = e["o"][0][:, t], e["o"][1][:, t]
        bound = (dk + 64) * U32 * most + 1e-37 + (U16 * ref.abs() if dtype == torch.bfloat16 else 0)
        assert float(((o.double() - ref).abs() / bound).max()) <= 1, t
    assert ((state.double() - e["last"][0]).abs() <= 64 * U32 * e["last"][1] + 1e-37).all()


def test_a_prompt_and_then_frames_one_by_one(nb):
    q, k, v, _, decay, _, _ = _inputs(2, 500, 4, 64, 64, torch.float32, state=False)
    whole, last = nb.nna_decay_attention(q, k, v, decay, want_state=True)
    e = _exact(q, k, v, decay)
    o, state = nb.nna_decay_attention(q[:, :450], k[:, :450], v[:, :450], decay, want_state=True)
    assert torch.equal(o, whole[:, :450])
    for t in range(450, 500):
        step = nb.nna_decay_attention_step(q[:, t], k[:, t], v[:, t], decay, state)
        assert ((step.double() - e["o"][0][:, t]).abs() <= 800 * U32 * e["o"][1][:, t]).all()
    assert ((state.double() - last.double()).abs() <= 800 * U32 * e["last"][1]).all()
    # in pieces: the state of one is the first of the next
    state, pieces = None, []
    for a, b in ((0, 1), (1, 64), (64, 200), (200, 500)):
        o, state = nb.nna_decay_attention(q[:, a:b], k[:, a:b], v[:, a:b], decay, state=state, want_state=True)
        pieces.append(o)
    assert ((torch.cat(pieces, 1).double() - e["o"][0]).abs() <= 800 * U32 * e["o"][1]).all()


# ---- refusals, nothing to do, streams, graphs --------------------------------------------------------------------------------
def test_nothing_to_do(nb):
    q, k, v, go, decay, first, glast = _inputs(2, 0, 3, 16, 24, torch.float32)
    o, last = nb.nna_decay_attention(q, k, v, decay, state=first, want_state=True)
    assert o.shape == (2, 0, 3, 24) and torch.equal(last, first)
    gfirst = nb.nna_decay_attention_backward(go, q, k, v, decay, gstate=glast, want_gstate=True)[3]
    assert torch.allclose(gfirst, glast, rtol=1e-6, atol=0)
    q, k, v, go, decay, first, glast = _inputs(0, 50, 3, 16, 24, torch.float32)
    assert nb.nna_decay_attention(q, k, v, decay, state=first, want_state=True)[1].shape == (0, 3, 16, 24)
    assert nb.nna_decay_attention_backward(go, q, k, v, decay)[0].shape == q.shape
    assert nb.nna_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, first).shape == (0, 3, 24)


def test_refusals(nb):
    q, k, v, go, decay, first, glast = _inputs(2, 10, 3, 16, 24, torch.float32)
    call = nb.nna_decay_attention
    for bad in (lambda: call(q.cpu(), k, v, decay), lambda: call(q.half(), k.half(), v.half(), decay), lambda: call(q, k.bfloat16(), v, decay),
                lambda: call(q[0], k[0], v[0], decay), lambda: call(q, k[..., :15], v, decay), lambda: call(q, k, v[:, :9], decay),
                lambda: call(q[..., ::2], k[..., ::2], v, decay), lambda: call(q, k, v, decay[:2]), lambda: call(q, k, v, decay.double()),
                lambda: call(q, k, v, decay, state=first.bfloat16()), lambda: call(q, k, v, decay, state=first[:, :, :, :5]),
                lambda: call(q, k, v, decay, lengths=torch.tensor([1, 2], device=DEV)), lambda: call(q, k, v, decay, lengths=torch.tensor([1, 2], dtype=torch.int32)),
                lambda: call(q, k, v, decay, out=torch.empty_like(q)), lambda: nb.nna_decay_attention_backward(go.bfloat16(), q, k, v, decay),
                lambda: nb.nna_decay_attention_backward(go[:, :5], q, k, v, decay), lambda: nb.nna_decay_attention_step(q, k, v, decay, first),
                lambda: nb.nna_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, None)):
        with pytest.raises(TypeError):
            bad()
    wide = torch.empty((1, 4, 1, 129), device=DEV)
    long = _inputs(1, 5000, 1, 64, 64, torch.float32)
    for bad, status in ((lambda: call(q, k, v, decay, scale=0.0), nb.NNA_ERR_INVALID_ARG), (lambda: call(q, k, v, decay, scale=float("nan")), nb.NNA_ERR_INVALID_ARG),
                        (lambda: call(wide, wide, wide, decay[:1]), nb.NNA_ERR_UNSUPPORTED),
                        (lambda: call(*long[:3], long[4], workspace=torch.empty(256, dtype=torch.uint8, device=DEV)), nb.NNA_ERR_INVALID_ARG)):
        with pytest.raises(nb.NnaError) as e:
            bad()
        assert e.value.status == status


def test_on_another_stream_and_in_a_graph(nb):
    q, k, v, go, decay, first, glast = _inputs(1, 3000, 2, 64, 64, torch.bfloat16)
    assert nb.nna_decay_attention_workspace(1, 3000, 2, 64, 64)

    def step(stream=None):
        return (*nb.nna_decay_attention(q, k, v, decay, state=first, want_state=True, stream=stream),
                *nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, gstate=glast, want_gstate=True, stream=stream))

    eager = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    out = step(stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(eager, out))
    state = first.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
        one = nb.nna_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, state)
    check = first.clone()
    for i in range(3):
        q.copy_(torch.randn_like(q))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, one, state)]
        want = nb.nna_decay_attention_step(q[:, 0], k[:, 0], v[:, 0], decay, check)
        assert all(torch.equal(a, c) for a, c in zip((*step(), want, check), got)), i


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,H,dk,dv", [(13, 1100, 10, 16, 16), (16, 800, 4, 33, 17), (4, 1100, 25, 40, 100), (16, 4160, 4, 16, 80), (2, 520, 3, 64, 64)])
def test_segments_of_either_direction(nb, dtype, B, T, H, dk, dv):
    """Many heads are cut forward alone, some neither way, some in one type only."""
    _say("directions", B, T, H, dk, dv, dtype, nb.nna_decay_attention_workspace(B, T, H, dk, dv), nb.nna_decay_attention_backward_workspace(B, T, H, dk, dv))
    args = _inputs(B, T, H, dk, dv, dtype, seed=T + H)
    args[4][0] = 1 - 2.0**-11
    _check(nb, *args)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,d", [(100, 64), (1500, 64), (100, 128), (1500, 100)])
def test_gradients_of_keys_and_values_alone(nb, dtype, T, d):
    """Without gq the others have the same bits."""
    from ctypes import c_longlong

    q, k, v, go, decay, first, glast = _inputs(2, T, 3, d, d, dtype, seed=d)
    _say("no gq", T, d, dtype)
    _, gk, gv, gfirst = nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, gstate=glast, want_gstate=True)
    alone = torch.full_like(k, float("nan")), torch.full_like(v, float("nan")), torch.full_like(first, float("nan"))
    strides = (c_longlong * 3)(T * 3 * d, 3 * d, d)
    need = nb.nna_decay_attention_backward_workspace(2, T, 3, d, d)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    status = nb.lib().nna_decay_attention_backward(
        go.data_ptr(), q.data_ptr(), strides, k.data_ptr(), strides, v.data_ptr(), strides, nb.NNA_F32 if dtype == torch.float32 else nb.NNA_BF16, 2, T, 3, d, d,
        decay.data_ptr(), d**-0.5, None, first.data_ptr(), glast.data_ptr(), None, alone[0].data_ptr(), alone[1].data_ptr(), alone[2].data_ptr(),
        ws.data_ptr() if need else None, need, 0, torch.cuda.current_stream().cuda_stream)
    assert status == nb.NNA_OK
    for a, b in zip(alone, (gk, gv, gfirst)):
        assert torch.equal(a, b)


SIZES = [(2, 200, 2, 64, 64), (1, 431, 2, 128, 128), (2, 150, 2, 100, 33), (1, 3000, 2, 64, 64), (1, 2111, 2, 128, 64)]


def _all_of(nb, q, k, v, go, decay, first, glast):
    o, last = nb.nna_decay_attention(q, k, v, decay, state=first, want_state=True)
    gq, gk, gv, gfirst = nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, gstate=glast, want_gstate=True)
    return dict(o=o, gq=gq, gk=gk, gv=gv, last=last, gfirst=gfirst)


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("B,T,H,dk,dv", SIZES)
def test_bfloat16_results_are_off_by_their_own_rounding_alone(nb, B, T, H, dk, dv, given):
    """A float32 sum that is an operand again (weights, state) is held to 2^-17 at least, so what comes before the last rounding is off by some units of
    2^-17 of the result's norm (roundings of either sign add as squares), a 64th of the 2^-9 that the rounding takes or less; a rounding of a value that is off by e
    is off by at most 2 e more than that of the value: 1 + 2 / 64 of the exact result's own rounding, and 1.05 is allowed."""
    _say("own rounding", B, T, H, dk, dv, given)
    q, k, v, go, decay, first, glast = _inputs(B, T, H, dk, dv, torch.bfloat16, seed=T + 1)
    e = _exact(q, k, v, decay, first, None, go, glast)
    if given:
        got = _all_of(nb, q, k, v, go, decay, first, glast)
    else:  # no state is given back
        gq, gk, gv, _ = nb.nna_decay_attention_backward(go, q, k, v, decay, state=first, gstate=glast)
        got = dict(o=nb.nna_decay_attention(q, k, v, decay, state=first), gq=gq, gk=gk, gv=gv)
    for name in ("o", "gq", "gk", "gv"):
        ref = e[name][0]
        own = (ref.bfloat16().double() - ref).norm()
        assert (got[name].double() - ref).norm() <= 1.05 * own, (name, float((got[name].double() - ref).norm() / own))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,H,dk,dv", SIZES)
def test_float32_results_hold_float32(nb, B, T, H, dk, dv, dtype):
    """Roundings of either sign add as squares: a product of planes leaves out or rounds off some 2^-24, its power of the decay two of them, and the sums some ten
    roundings of partial sums: 16 units, 1e-6 of the norm.  Operands of two planes alone would be off by 2^-17 / sqrt(3) = 4.4e-6 each."""
    _say("float32", B, T, H, dk, dv, dtype)
    args = _inputs(B, T, H, dk, dv, dtype, seed=T + 2)
    q, k, v, go, decay, first, glast = args
    e = _exact(q, k, v, decay, first, None, go, glast)
    for name, x in _all_of(nb, *args).items():
        if x.dtype == torch.float32:
            ref = e[name][0]
            assert (x.double() - ref).norm() <= 1e-6 * ref.norm(), (name, float((x.double() - ref).norm() / ref.norm()))


def _of_head(name, x, h):
    return x[:, h] if name in ("last", "gfirst") else x[:, :, h]


@pytest.mark.parametrize("T,dk,dv", [(100, 64, 64), (1500, 64, 64), (100, 128, 128), (100, 65, 63), (100, 7, 100)])
def test_the_largest_float32_values_are_values(nb, T, dk, dv):
    """float32's largest is above bfloat16's: what it enters is what it would be times 1 (powers of two throughout), and no frame before it knows it."""
    _say("largest", T, dk, dv)
    most, at = torch.finfo(torch.float32).max, 77
    q, k, v, go, decay, first, glast = _inputs(1, T, 2, dk, dv, torch.float32, seed=T + dk, state=False)
    clean = _all_of(nb, q, k, v, go, decay, None, None)
    for name, x in (("v", v), ("k", k), ("q", q), ("go", go)):
        for last in (False, True):
            keep, d = x.clone(), x.shape[-1] - 1 if last else 0
            x[0, at, 0, d] = most
            got = _all_of(nb, q, k, v, go, decay, None, None)
            for out in ("o", "gq") if name != "go" else ("o",):
                assert torch.equal(got[out][0, :at], clean[out][0, :at]), (name, out)
            for out in ("gk", "gv") if name in ("go", "q") else ():
                assert torch.equal(got[out][0, at + 1:], clean[out][0, at + 1:]), (name, out)
            for out in got:
                assert torch.equal(_of_head(out, got[out], 1), _of_head(out, clean[out], 1)), (name, out)
            x.copy_(keep)
    # one value through a state and weights: 2^-7 of it everywhere
    q, k, v = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    q[..., 0], k[0, at, 0, 0], v[0, at, 0, dv - 1] = 2.0**-7, 1.0, most
    one = torch.ones_like(decay)
    o, state = nb.nna_decay_attention(q, k, v, one, scale=1.0, want_state=True)
    assert (o[0, at:, 0, dv - 1] == most * 2.0**-7).all() and not o[0, :at].any() and not o[0, :, :, :dv - 1].any()
    assert state[0, 0, 0, dv - 1] == most and int((state != 0).sum()) == 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,dk,dv", [(100, 128, 128), (1500, 128, 128), (100, 65, 63), (1500, 33, 100), (40, 5, 3)])
def test_a_value_that_is_not_finite_in_heads_of_other_sizes(nb, dtype, T, dk, dv):
    """no output before it, no gradient of keys and values after a go or q that has one, no other head; in the first column and in the last"""
    _say("not finite", T, dk, dv, dtype)
    q, k, v, go, decay, first, glast = _inputs(2, T, 2, dk, dv, dtype, seed=dk)
    clean, at = _all_of(nb, q, k, v, go, decay, first, glast), 35
    for name, x in (("v", v), ("k", k), ("q", q), ("go", go)):
        for value in (float("nan"), float("inf")):
            for d in (0, x.shape[-1] - 1):
                keep = x.clone()
                x[1, at, 0, d] = value
                got = _all_of(nb, q, k, v, go, decay, first, glast)
                before = ("o", "gq") if name != "go" else ("o",)
                after = ("gk", "gv") if name in ("go", "q") else ()
                for out in got:
                    a, b = got[out], clean[out]
                    assert torch.equal(a[0], b[0]), (name, out)
                    assert torch.equal(_of_head(out, a, 1), _of_head(out, b, 1)), (name, out)
                    if out in before:
                        assert torch.equal(a[1, :at], b[1, :at]), (name, out)
                    if out in after:
                        assert torch.equal(a[1, at + 1:], b[1, at + 1:]), (name, out)
                assert not torch.isfinite(torch.cat([t[1].flatten() for t in got.values()])).all()
                x.copy_(keep)


def test_outputs_over_inputs_are_refused(nb):
    from ctypes import c_longlong

    q, k, v, go, decay, first, glast = _inputs(2, 10, 3, 16, 16, torch.float32)
    one = [x[:, 0].contiguous() for x in (q, k, v)]
    for x in (q, k, v):
        with pytest.raises(ValueError):
            nb.nna_decay_attention(q, k, v, decay, out=x)
    for x in one:
        with pytest.raises(ValueError):
            nb.nna_decay_attention_step(*one, decay, first, out=x)
    with pytest.raises(ValueError):
        nb.nna_decay_attention_step(*one, decay, first, out=first.view(-1)[:96].view(2, 3, 16))
    both = torch.zeros(21 * 48, device=DEV)
    with pytest.raises(ValueError):
        nb.nna_decay_attention(both[:960].view(2, 10, 3, 16), k, v, decay, out=both[48:].view(2, 10, 3, 16))
    s, s2, st = (c_longlong * 3)(480, 48, 16), (c_longlong * 2)(48, 16), torch.cuda.current_stream().cuda_stream
    P = [x.data_ptr() for x in (q, k, v)]
    new = [torch.zeros_like(x).data_ptr() for x in (q, k, v)]
    qkv, step = (P[0], s, P[1], s, P[2], s, nb.NNA_F32, 2, 10, 3, 16, 16, decay.data_ptr(), 1.0), (P[0], s2, P[1], s2, P[2], s2, nb.NNA_F32, 2, 3, 16, 16, decay.data_ptr(), 1.0)
    for p in P:
        assert nb.lib().nna_decay_attention(*qkv, None, None, None, p, None, 0, 0, st) == nb.NNA_ERR_INVALID_ARG
        assert nb.lib().nna_decay_attention_step(*step, first.data_ptr(), p, 0, st) == nb.NNA_ERR_INVALID_ARG
    g, f, l = go.data_ptr(), first.data_ptr(), glast.data_ptr()
    for outs in ((P[0], new[1], new[2], None), (new[0], P[1], new[2], None), (new[0], new[1], g, None), (*new, f), (*new, l)):
        assert nb.lib().nna_decay_attention_backward(g, *qkv, None, f, l, *outs, None, 0, 0, st) == nb.NNA_ERR_INVALID_ARG


def test_one_frame_from_memory_of_any_order(nb):
    """of [T, B, H, d] in memory, the distance from one frame to the next is no matter where there is one frame"""
    q, k, v, go, decay, first, glast = _inputs(3, 1, 2, 16, 24, torch.float32, seed=2)
    want = _all_of(nb, q, k, v, go, decay, first, glast)
    far = [torch.as_strided(x, x.shape, (x.stride(0), 1 << 40, x.stride(2), 1)) for x in (q, k, v)]
    got = _all_of(nb, *far, go, decay, first, glast)
    assert all(torch.equal(got[name], want[name]) for name in want)
