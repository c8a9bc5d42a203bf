"""Gradients through RotaryPositions.apply: the transposed rotation, recorded as any torch operation's."""
import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from paper_2609_34606_b200 import hsa
from test_rope import FP32_WORK, HALF_STEP

pytestmark = pytest.mark.gpu


def turned(w, pos, r, pairs, layout, scaling, factor, transpose):
    f, a = O.frequencies(pairs, 1e4, scaling, factor)
    return O.rope(w.double().cpu().numpy(), pos, pairs, f, a, layout, transpose), a


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("transpose", [False, True])
@pytest.mark.parametrize("tokens,H,d,pairs,scaling", [(1, 1, 128, (64,), "none"), (37, 3, 64, (8, 7, 9), "bands"), (130, 5, 40, (20,), "linear")])
def test_gradient_of_apply(cuda_device, dtype, layout, transpose, tokens, H, d, pairs, scaling):
    g = torch.Generator().manual_seed(tokens)
    rand = lambda: torch.randn(tokens, H, d, generator=g).to(dtype).to(cuda_device)
    factor = 1.0 if scaling == "none" else 4.0
    r = hsa.RotaryPositions(d, 2 * sum(pairs), layout, axis_pairs=pairs, scaling=scaling, factor=factor, device=cuda_device)
    pos = torch.randint(0, 50000, (len(pairs), tokens), generator=g).to(torch.int32)
    x, w = rand().requires_grad_(), rand()
    y = r.apply(x, pos.to(cuda_device), transpose=transpose)
    assert torch.equal(y.detach(), r.apply(x.detach(), pos.to(cuda_device), transpose=transpose))
    got, = torch.autograd.grad(y, x, w, retain_graph=True)
    assert got.dtype == dtype and torch.equal(got, r.apply(w, pos.to(cuda_device), transpose=not transpose))
    ref, a = turned(w, pos.numpy(), r, pairs, layout, scaling, factor, not transpose)
    # |w| <= 5: fp32 work on a pair, half a step of the result, the smallest steps of the type
    bound = FP32_WORK * a * 10 + HALF_STEP[dtype] * (np.abs(ref) + FP32_WORK * a * 10) + torch.finfo(dtype).smallest_normal
    assert (np.abs(got.double().cpu().numpy() - ref) <= bound).all()
    # a gradient that is one number everywhere, without memory of its own; the same leaf twice
    x.grad = None
    (y.sum() + r.apply(x, pos.to(cuda_device), transpose=transpose).sum()).backward()
    ones, _ = turned(torch.ones(tokens, H, d), pos.numpy(), r, pairs, layout, scaling, factor, not transpose)
    size = 4 * a
    bound = 2 * (FP32_WORK * size + HALF_STEP[dtype] * size) + HALF_STEP[dtype] * 2 * size
    assert np.abs(x.grad.double().cpu().numpy() - 2 * ones).max() <= bound


def test_gradient_against_differences_and_twice(cuda_device):
    g = torch.Generator().manual_seed(1)
    x = torch.randn(5, 2, 32, generator=g).to(cuda_device).requires_grad_()
    r = hsa.RotaryPositions(32, device=cuda_device)              # positions: 0, 1, ...
    w = torch.randn(5, 2, 32, generator=g).to(cuda_device)
    f = lambda z: (r.apply(z) ** 2 * w).sum()
    first, = torch.autograd.grad(f(x), x, create_graph=True)
    for i, j, k in ((0, 0, 0), (1, 1, 7), (4, 0, 31), (3, 1, 16)):
        up, down = x.detach().clone(), x.detach().clone()
        up[i, j, k] += 0.25
        down[i, j, k] -= 0.25
        # f is quadratic: differences are exact but for fp32 sums of 320 terms below 64
        assert abs((f(up) - f(down)).item() / 0.5 - first[i, j, k].item()) < 320 * 64 * 2.0 ** -23
    v = torch.randn(5, 2, 32, generator=g).to(cuda_device)
    second, = torch.autograd.grad((first * v).sum(), x)
    want = r.apply(2 * w * r.apply(v), transpose=True)           # the Hessian 2 R^T diag(w) R times v
    assert (second - want).abs().max() < 1e-4


def test_strided_gradient_and_refusals(cuda_device):
    r = hsa.RotaryPositions(64, device=cuda_device)
    pos = torch.arange(9, dtype=torch.int32, device=cuda_device)
    x = torch.randn(9, 2, 64, device=cuda_device, requires_grad=True)
    w = torch.randn(9, 2, 64, device=cuda_device)
    odd = torch.empty(9 * 128 + 1, device=cuda_device)[1:].view(9, 2, 64).copy_(w)          # 4-byte aligned
    for g in (w.transpose(1, 2).contiguous().transpose(1, 2), w.repeat(1, 1, 2)[..., :64], odd, w[:, :1].expand(9, 2, 64)):
        got, = torch.autograd.grad(r.apply(x, pos), x, g)
        assert torch.equal(got, r.apply(g.contiguous().clone(), pos, transpose=True))
    for out in (torch.empty_like(w), x):
        with pytest.raises(ValueError, match="gradient"):
            r.apply(x, pos, out=out)
    with torch.no_grad():
        assert r.apply(x, pos, out=torch.empty_like(w)).grad_fn is None and r.apply(x, pos).grad_fn is None
    y = r.apply(x, pos)
    pos += 1                                                      # the positions that the gradient needs are gone
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_captured_with_its_gradient(cuda_device):
    r = hsa.RotaryPositions(64, device=cuda_device)
    pos = torch.arange(33, dtype=torch.int32, device=cuda_device)
    x = torch.randn(33, 2, 64, device=cuda_device, requires_grad=True)
    w = torch.randn(33, 2, 64, device=cuda_device)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(r.apply(x, pos), x, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = r.apply(x, pos)
        got, = torch.autograd.grad(y, x, w)
    with torch.no_grad():
        x.mul_(-2)
    w.add_(1)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y.detach(), r.apply(x.detach(), pos)) and torch.equal(got, r.apply(w, pos, transpose=True))
