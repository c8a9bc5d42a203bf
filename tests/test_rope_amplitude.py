"""Amplitudes: the scaling's own, and one that the caller sets, in the rotation and in the append."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from paper_2609_34606_b200 import hsa
from test_kv8 import Case, dev_i32
from test_rope import FP32_WORK, HALF_STEP


def test_amplitude_on_host():
    bands = dict(scaling="bands", factor=8.0, device="cpu")
    assert hsa.RotaryPositions(64, **bands).amplitude == pytest.approx(0.1 * math.log(8.0) + 1, rel=1e-7)
    assert hsa.RotaryPositions(64, device="cpu").amplitude == 1.0
    r = hsa.RotaryPositions(64, amplitude=1.0, **bands)
    assert r.amplitude == 1.0 and r.args(None, 3).amplitude == 1.0
    assert torch.equal(r.turns, hsa.RotaryPositions(64, **bands).turns)
    for bad in (math.nan, math.inf):
        with pytest.raises(ValueError):
            hsa.RotaryPositions(64, amplitude=bad, device="cpu")


@pytest.mark.gpu
@pytest.mark.parametrize("amplitude", [None, 1.0, 0.7, -3.0])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rotation_with_amplitude(cuda_device, amplitude, layout):
    g = torch.Generator().manual_seed(7)
    x = torch.randn(40, 3, 64, generator=g)
    r = hsa.RotaryPositions(64, 48, layout, scaling="bands", factor=8.0, device=cuda_device, amplitude=amplitude)
    f, a = O.frequencies((24,), 1e4, "bands", 8.0)
    a = a if amplitude is None else amplitude
    for transpose in (False, True):
        y = r.apply(x.to(cuda_device), transpose=transpose)
        ref = O.rope(x.numpy(), np.arange(40)[None], (24,), f, a, layout, transpose)
        # |x| < 5: fp32 work on a pair and half a step of the result
        assert np.abs(y.double().cpu().numpy() - ref).max() < (FP32_WORK + 2 * HALF_STEP[torch.float32]) * abs(a) * 10


@pytest.mark.gpu
@pytest.mark.parametrize("amplitude", [None, 1.0, 5.0])
@pytest.mark.parametrize("layout,rot", [("half", 128), ("half", 36), ("interleaved", 128), ("interleaved", 36)])
def test_append_with_amplitude(cuda_device, amplitude, layout, rot):
    c = Case(cuda_device, 2, 2, 128, [300, 300], sums=True, seed=41)
    r = hsa.RotaryPositions(128, rot, layout, scaling="bands", factor=16.0, device=cuda_device, amplitude=amplitude)
    f, a = O.frequencies((rot // 2,), 1e4, "bands", 16.0)
    a = a if amplitude is None else amplitude
    for counts in ([100, 3], [130, 200]):
        starts, held = np.concatenate([[0], np.cumsum(counts)]), list(c.held)
        k, v = c.append(counts, rope=r, twin=False)
        at = np.concatenate([np.arange(h, h + m) for h, m in zip(held, counts)])[None]
        K, V = O.rope(k.double().numpy(), at, (rot // 2,), f, a, layout), v.double().numpy()
        cut = lambda x: [x[starts[i]:starts[i + 1]] for i in range(2)]
        O.append(c.state, c.table.numpy(), held, cut(K), cut(V))
        c.check_state(exact=False)
    assert c.cache.device_status() == 0
