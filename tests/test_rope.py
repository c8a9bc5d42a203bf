"""Rotary positions: the table and the refusals on the host, the kernel against the fp64 reference on the GPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from paper_2609_34606_b200 import hsa

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
# fp32 work on the way: the sine and cosine are each off by at most 2^-24 (series and reduction below half a step,
# one rounding), times the amplitude one more, and the two products and their sum two roundings: four half steps of
# 2^-24 of |a| + |b|, and half of that again for the angle's own 2^-32 of a turn and the amplitude's rounding.
FP32_WORK = 6 * 2.0 ** -24


def config(head_dim=128, rot_dim=128, layout=0, pairs=(64,), scaling=0, base=1e4, factor=1.0, trained=4096.0, fast=32.0,
           slow=1.0):
    return hsa.hsa_rope_config(head_dim, rot_dim, layout, len(pairs), (C.c_int32 * 3)(*pairs), scaling, base, factor, trained,
                               fast, slow)


# ------------------------------------------------------------------ host
@pytest.mark.parametrize("scaling", ["none", "linear", "base", "bands"])
@pytest.mark.parametrize("pairs", [(64,), (22, 21, 21), (1,), (1, 0, 1), (3, 5)])
def test_table(pairs, scaling):
    factor = 1.0 if scaling == "none" else 6.5
    turns, amplitude = hsa.hsa_rope_table(config(rot_dim=2 * sum(pairs), pairs=pairs, scaling=hsa._SCALINGS[scaling],
                                                 factor=factor))
    f, a = O.frequencies(pairs, 1e4, scaling, factor)
    got = turns.numpy().view(np.uint64).astype(np.float64) / 2.0 ** 64 * (2 * math.pi)
    assert got.shape == f.shape
    assert np.abs(got / f.astype(np.float64) - 1).max() < 1e-14 and abs(amplitude - a) < 1e-6
    if scaling == "base" and pairs[0] > 1:   # the slowest pair is stretched by the factor, the fastest not at all
        assert got[0] == pytest.approx(1.0) and got[pairs[0] - 1] * factor == pytest.approx(1e4 ** (-(pairs[0] - 1) / pairs[0]))


@pytest.mark.parametrize("bad", [dict(rot_dim=3, pairs=(1,)), dict(rot_dim=0, pairs=(0,)), dict(rot_dim=130, pairs=(65,)),
                                 dict(layout=2), dict(pairs=(63,)), dict(pairs=(65, -1)), dict(head_dim=12, rot_dim=8, pairs=(4,)),
                                 dict(head_dim=520), dict(scaling=4), dict(scaling=1, factor=0.5), dict(scaling=1, factor=math.nan),
                                 dict(base=1.0), dict(base=math.inf), dict(scaling=3, factor=2.0, fast=1.0, slow=1.0),
                                 dict(scaling=3, factor=2.0, trained=0.0)])
def test_table_refusals(bad):
    with pytest.raises(hsa.HSAError) as e:
        hsa.hsa_rope_table(config(**bad))
    assert e.value.code == hsa.HSA_ERR_INVALID_ARG


def test_call_refusals_on_host():
    """Every refusal comes before a CUDA call: made-up addresses are never followed."""
    ok = dict(x=0x1000, out=0x2000, type=0, n=4, H=2, d=128, ts=256, hs=128, ots=256, ohs=128, flags=0)
    rope = dict(rot=128, layout=0, axes=1, pairs=(64,), amplitude=1.0, turns=0x3000, pos=0x4000, stride=4)

    def call(r=None, **kw):
        a, q = {**ok, **kw}, {**rope, **(r or {})}
        pairs = (C.c_int32 * 3)(*q["pairs"])
        args = hsa.hsa_rope_args(q["rot"], q["layout"], q["axes"], pairs, q["amplitude"], q["turns"], q["pos"], q["stride"])
        return hsa._lib.hsa_rope(a["x"], a["out"], a["type"], a["n"], a["H"], a["d"], a["ts"], a["hs"], a["ots"], a["ohs"],
                                 C.byref(args), a["flags"], None)

    assert call(n=0) == hsa.HSA_OK
    for kw in [dict(x=None), dict(out=None), dict(x=0x1008), dict(out=0x2008), dict(type=3), dict(n=-1), dict(H=0), dict(d=100),
               dict(ts=255), dict(hs=64), dict(ots=132), dict(ohs=100), dict(flags=2), dict(out=0x1000, ots=512), dict(d=64)]:
        assert call(**kw) == hsa.HSA_ERR_INVALID_ARG, kw
    for r in [dict(turns=None), dict(turns=0x3004), dict(pos=0x4002), dict(rot=127), dict(rot=0), dict(layout=2), dict(axes=0),
              dict(axes=4), dict(pairs=(63,)), dict(axes=2, pairs=(32, 31)), dict(axes=2, pairs=(65, -1)),
              dict(axes=2, pairs=(32, 32), stride=3), dict(amplitude=math.inf), dict(amplitude=math.nan)]:
        assert call(r) == hsa.HSA_ERR_INVALID_ARG, r
    assert hsa._lib.hsa_rope(0x1000, 0x2000, 0, 4, 2, 128, 256, 128, 256, 128, None, 0, None) == hsa.HSA_ERR_INVALID_ARG


def test_wrapper_refusals_on_host():
    with pytest.raises(ValueError):
        hsa.RotaryPositions(128, layout="spiral", device="cpu")
    with pytest.raises(ValueError):
        hsa.RotaryPositions(128, axis_pairs=(16, 16, 16, 16), device="cpu")
    r = hsa.RotaryPositions(64, device="cpu")
    with pytest.raises(ValueError):
        r.apply(torch.zeros(2, 3, 64))                       # not a CUDA tensor
    with pytest.raises(ValueError):
        r.apply(torch.zeros(2, 3, 128))                      # another head size
    with pytest.raises(ValueError):
        r.args(torch.zeros(5, dtype=torch.int64), 5)
    with pytest.raises(ValueError):
        r.args(torch.zeros(4, dtype=torch.int32), 5)
    with pytest.raises(ValueError):
        r.args(torch.zeros(1, 10, dtype=torch.int32)[:, ::2], 5)


# ------------------------------------------------------------------ GPU
def check(got, x, pos, pairs, layout, scaling="none", factor=1.0, transpose=False):
    f, a = O.frequencies(pairs, 1e4, scaling, factor)
    X = x.double().cpu().numpy()
    ref = O.rope(X, pos, pairs, f, a, layout, transpose)
    half = sum(pairs)
    size = np.abs(X)                              # |a| + |b| of the pair each value belongs to
    if layout == "half":
        both = size[..., :half] + size[..., half:2 * half]
        size = np.concatenate([both, both, np.zeros_like(size[..., 2 * half:])], -1)
    else:
        both = size[..., 0:2 * half:2] + size[..., 1:2 * half:2]
        size = np.concatenate([np.repeat(both, 2, -1), np.zeros_like(size[..., 2 * half:])], -1)
    work = FP32_WORK * a * size
    tiny = torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps
    bound = work + HALF_STEP[x.dtype] * (np.abs(ref) + work) + tiny
    d = np.abs(got.double().cpu().numpy() - ref)
    assert (d <= bound).all(), (d - bound).max()
    assert torch.equal(got[..., 2 * half:], x[..., 2 * half:])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,pairs", [(128, (64,)), (128, (22, 21, 21)), (64, (32,)), (128, (24,)), (64, (1,)), (128, (57,)),
                                     (40, (20,)), (8, (4,)), (128, (3, 5)), (512, (256,))])
def test_rotation_and_its_transpose(cuda_device, dtype, layout, d, pairs):
    g = torch.Generator().manual_seed(d + sum(pairs))
    for tokens, H in ((1, 1), (7, 5), (130, 3)):
        x = torch.randn(tokens, H, d, generator=g).to(dtype).to(cuda_device)
        pos = torch.randint(-5, 2 ** 31 - 1, (len(pairs), tokens), generator=g, dtype=torch.int64).to(torch.int32)
        pos[:, 0] = 0
        r = hsa.RotaryPositions(d, 2 * sum(pairs), layout, axis_pairs=pairs, device=cuda_device)
        for transpose in (False, True):
            y = r.apply(x, pos.to(cuda_device), transpose=transpose)
            check(y, x, pos.numpy(), pairs, layout, transpose=transpose)


@pytest.mark.gpu
@pytest.mark.parametrize("scaling,factor", [("linear", 4.0), ("base", 8.0), ("bands", 16.0)])
def test_scaled_positions_in_place_and_strided(cuda_device, scaling, factor):
    pairs = (16, 8, 8)
    g = torch.Generator().manual_seed(3)
    wide = torch.randn(70, 6, 3, 64, generator=g).to(torch.bfloat16).to(cuda_device)
    x = wide[:, ::2, 1]                              # [70, 3, 64] with strides (1152, 384, 1)
    pos = torch.randint(0, 60000, (3, 90), generator=g, dtype=torch.int64).to(torch.int32).to(cuda_device)[:, 11:81]
    r = hsa.RotaryPositions(64, 64, "interleaved", axis_pairs=pairs, scaling=scaling, factor=factor, device=cuda_device)
    before, keep = x.clone(), wide.clone()
    y = r.apply(x, pos)
    check(y, before, pos.cpu().numpy(), pairs, "interleaved", scaling, factor)
    assert r.apply(x, pos, out=x) is x and torch.equal(x, y)
    keep[:, ::2, 1] = y
    assert torch.equal(wide, keep)                   # nothing beside the rows was touched


@pytest.mark.gpu
def test_many_heads_and_default_positions(cuda_device):
    """Enough work that a thread takes several heads, with a share that does not divide them."""
    g = torch.Generator().manual_seed(4)
    x = torch.randn(6000, 13, 64, generator=g).to(torch.bfloat16).to(cuda_device)
    for layout in ("half", "interleaved"):
        y = hsa.RotaryPositions(64, layout=layout, device=cuda_device).apply(x)
        check(y, x, np.arange(6000)[None], (32,), layout)


@pytest.mark.gpu
def test_gradient(cuda_device):
    """The transposed map against autograd through the formula and against differences."""
    pairs, d = (10, 6), 40
    g = torch.Generator().manual_seed(5)
    x = torch.randn(9, 2, d, generator=g, dtype=torch.float64)
    w = torch.randn(9, 2, d, generator=g, dtype=torch.float64)
    pos = torch.randint(0, 5000, (2, 9), generator=g, dtype=torch.int64).to(torch.int32)
    r = hsa.RotaryPositions(d, 32, "half", axis_pairs=pairs, scaling="bands", factor=4.0, device=cuda_device)
    got = r.apply(w.float().to(cuda_device), pos.to(cuda_device), transpose=True).double().cpu()
    f, a = O.frequencies(pairs, 1e4, "bands", 4.0)
    fn = lambda z: O.rope(z, pos.numpy(), pairs, f, a, "half")
    ref = O.rope(w.float().double().numpy(), pos.numpy(), pairs, f, a, "half", transpose=True)
    # |w| <= 4.5 here: FP32_WORK * amplitude * 2 |w| and half a step of the result
    assert np.abs(got.numpy() - ref).max() < FP32_WORK * a * 9 + 2.0 ** -24 * 9
    z, step = x.numpy(), 1e-3
    for i, j, k in ((0, 0, 0), (3, 1, 17), (8, 0, 31), (5, 1, 35)):
        up, down = z.copy(), z.copy()
        up[i, j, k] += step
        down[i, j, k] -= step
        diff = ((fn(up) - fn(down)) * w.numpy()).sum() / (2 * step)     # the map is linear: exact but for fp64
        assert abs(diff - got[i, j, k].item()) < 1e-5
    # forward, then transposed: amplitude^2 times the input
    y = r.apply(r.apply(x.float().to(cuda_device), pos.to(cuda_device)), pos.to(cuda_device), transpose=True)
    back = x.clone()
    back[..., :32] *= a * a
    assert (y.double().cpu() - back).abs().max() < 4 * FP32_WORK * a * a * 9


@pytest.mark.gpu
def test_captured_and_on_another_stream(cuda_device):
    x = torch.randn(33, 4, 128, device=cuda_device, dtype=torch.bfloat16)
    pos = torch.arange(33, dtype=torch.int32, device=cuda_device)
    r = hsa.RotaryPositions(128, device=cuda_device)
    want = r.apply(x, pos)
    out = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r.apply(x, pos, out=out)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.apply(x, pos, out=out)
    pos += 7
    x.neg_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, r.apply(x, pos))
