"""Attention over the 8-bit cache where weights and scores lie far apart: a dominant key before a long tail, scores that
leave fp32 no fraction, ties at any size."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from test_kv8 import Case

pytestmark = pytest.mark.gpu

# (query heads, key heads, tokens of the sequence): each instance of the kernel for few rows, then the other kernel
ROWS = [(2, 2, 1), (4, 1, 1), (7, 1, 1), (5, 5, 8), (4, 2, 6), (16, 1, 1), (2, 2, 17), (2, 2, 130), (1, 1, 300)]


def reference(c, q, causal):
    return O.attend([q.double().numpy()], c.state, c.table.numpy(), c.held, causal, c.cache.cfg.softmax_scale or None)[0]


def check(got, lse, ref, score, lost=2.0 ** -33):
    """out: half a step of bf16 for the result, 2^-8 for the weights, `score` (in nats) for numerator and denominator, and
    `lost` of the largest weight, which the sum of weights is no smaller than, for each key."""
    out, lse_ref, spread, size = ref
    d = np.abs(got.double().cpu().numpy() - out)
    bound = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 * 1.02 + 2 * score) * spread + lost * size
    assert (d <= bound).all(), ((d / np.maximum(bound, 1e-300)).max(), np.argwhere(~(d <= bound))[:4])
    e = np.abs(lse.double().cpu().numpy() - lse_ref)
    assert (e <= score + 2.0 ** -20 * (1 + np.abs(lse_ref))).all(), np.nanmax(e)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", ROWS)
@pytest.mark.parametrize("nats", [8.0, 15.0, 18.0])
@pytest.mark.parametrize("tail", [1500, 6000])
def test_a_dominant_key_leaves_the_others_their_weight(cuda_device, d, Hq, Hkv, n, nats, tail):
    """One key far above all others whose value is next to nothing: the result is made of the others."""
    c = Case(cuda_device, Hq, Hkv, d, [tail], seed=d + n, max_tokens=tail)
    k, v = c.randn(tail, Hkv, d, scale=0.05), 1 + c.randn(tail, Hkv, d, scale=0.5)
    k[:, :, 0] = 0
    k[5, :, 0] = nats * math.sqrt(d)
    v[5] *= 2.0 ** -20
    q = c.randn(n, Hq, d)
    q[:, :, 0] = 1
    c.append([tail], k=k, v=v, twin=False)
    c.take_gpu_state()
    _, got, lse = c.attend([n], True, q=q, check=False)
    # products exact or short by 2^-17 of max|q| |k|_1, sums in fp32: 2^-16 together
    score = 2.0 ** -16 * float(q.abs().max()) * float(k.double().abs().sum(-1).max()) * 1.07 / math.sqrt(d) + 2.0 ** -20
    check(got, lse, reference(c, q, True), score)
    assert c.cache.device_status() == 0
