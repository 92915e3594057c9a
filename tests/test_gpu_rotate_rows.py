"""The weights' gradients of rotated heads over many rows: every workgroup's share of them has to be there.

Gradients that go with the outputs: every row's part of a weight's gradient, g' h, is then positive (h^2 w), and a share left out, or taken twice, shows as itself.
The kernel adds a lane's rows one after the other, then a workgroup's lanes, then 512 workgroups: rows / (512 workgroups x 16 lanes and more) + 256 + 512 roundings at most, each of half a unit of
2^-24 of the sum, and 64 units of a row's own values (cos, sin, the norm): below 2^-13 of a sum of positive terms; one workgroup's share is 2^-9.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("B,T,H,K,width,pairs,interleaved", [(4, 2500, 8, 2, 16, 8, True), (3, 7001, 12, 4, 80, 20, False), (1, 20011, 1, 1, 64, 32, False), (2, 4099, 2, 0, 33, 10, True),
                                                            (5, 3000, 3, 6, 256, 128, False), (40, 431, 8, 8, 64, 0, False)])
def test_many_rows(B, T, H, K, width, pairs, interleaved, dtype):
    from paper_1912_12055_amd import binding as nb
    g = torch.Generator(device=DEV).manual_seed(T)
    q = torch.randn(B, T, H, width, device=DEV, generator=g).to(dtype)
    k = torch.randn(B, T, K, width, device=DEV, generator=g).to(dtype) if K else None
    freqs = 100.0 ** (-torch.arange(pairs, dtype=torch.float64, device=DEV) / max(1, pairs))
    wq, wk = (0.5 + torch.rand(width, device=DEV, generator=g) for _ in range(2))
    how = dict(eps=1e-6, interleaved=interleaved, q_weight=wq, k_weight=wk if K else None)
    yq, yk = nb.nna_rotate_heads(q, k, freqs, **how)
    gw = nb.nna_rotate_heads_backward(yq, yk, q, k, freqs, **how)[2:]
    for x, w, got in ((q, wq, gw[0]), (k, wk, gw[1])):
        if x is None:
            assert got is None
            continue
        v = x.double()
        want = (v.square() / (v.square().mean(-1, keepdim=True) + 1e-6)).sum((0, 1, 2)) * w.double()
        # (the outputs that stand for gradients are rounded once, up or down: B T H of them, of which a walk is left; half a step of the largest of a row, 8 times h, beside a mean of h^2 of one)
        walk = 8 * torch.finfo(dtype).eps / 2 * (B * T * x.shape[2]) ** -0.5 * 4
        assert float(((got.double() - want).abs() / want).max()) <= 2.0**-13 + (walk if dtype != torch.float32 else 0), dtype
