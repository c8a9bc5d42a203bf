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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", ROWS)
@pytest.mark.parametrize("power", [12, 22, 28, 38, 50, math.inf])
def test_one_huge_key(cuda_device, d, Hq, Hkv, n, power):
    """A key whose scores pass 2^power: rows that it points at get its value alone, rows that it points away from the others'
    result.  (inf: as it is stored, 2^60.)"""
    c = Case(cuda_device, Hq, Hkv, d, [700], seed=21)
    k, v = c.randn(700, Hkv, d), c.randn(700, Hkv, d)
    for b in range(0, 700, 64):
        v[b:b + 64] *= 2.0 ** (b // 64 % 5 * 3 - 6)
    k[70] *= 2.0 ** min(power, 50)
    k[70, :, 0] = 2.0 ** power * 40
    q = c.randn(n, Hq, d)
    q[..., 0] = torch.where(torch.rand(n, Hq, generator=c.g) < 0.5, -4.0, 4.0)
    c.append([700], k=k, v=v, twin=False)
    assert c.cache.device_status() == (0 if power < 60 else -7)
    c.take_gpu_state()
    _, got, lse = c.attend([n], True, q=q, check=False)
    ref = reference(c, q, True)
    k[70] = 0
    score = 2.0 ** -16 * float(q.abs().max()) * float(k.double().abs().sum(-1).max()) * 1.07 / math.sqrt(d) + 2.0 ** -20
    # rows that the huge key points at: nothing else counts; its score is off by 2^-14 of itself (short products, sums of 128 terms)
    hit = np.abs(ref[1]) > 1000
    assert hit.any() and not hit.all() or n * Hq < 4
    part = lambda rows: (got.cpu()[rows], lse.cpu()[rows], [x[rows] for x in ref])
    check(*part(~hit), score)
    o, l, mine = part(hit)
    check(o, torch.from_numpy(mine[1]), mine, 0.0)
    assert (np.abs(l.double().numpy() - mine[1]) <= 2.0 ** -14 * np.abs(mine[1])).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", ROWS)
@pytest.mark.parametrize("power,q_power", [(0, 0), (21, 0), (30, 0), (45, 0), (59, 0), (59, 45)])
@pytest.mark.parametrize("tokens", [650, 9000])
def test_ties_of_any_size(cuda_device, d, Hq, Hkv, n, power, q_power, tokens):
    """All keys alike: every row is the mean of the values it sees, whatever the scores are, over pages of different value scales."""
    c = Case(cuda_device, Hq, Hkv, d, [tokens], seed=22, max_tokens=tokens)
    k, v = c.randn(1, Hkv, d) * 2.0 ** power, 1 + c.randn(tokens, Hkv, d, scale=0.5)
    k = k.clamp(-2.0 ** 59, 2.0 ** 59).expand(tokens, Hkv, d).contiguous()
    for b in range(0, tokens, 64):
        v[b:b + 64] *= 2.0 ** (b // 64 % 5 * 3 - 6)
    q = c.randn(n, Hq, d) * 2.0 ** q_power
    c.append([tokens], k=k, v=v, twin=False)
    c.take_gpu_state()
    _, got, lse = c.attend([n], True, q=q, check=False)
    ref = reference(c, q, True)
    check(got, torch.from_numpy(ref[1]), ref, 0.0)
    size = float(q.double().abs().max()) * float(k.double().abs().sum(-1).max()) * 1.07 / math.sqrt(d)
    assert (np.abs(lse.double().cpu().numpy() - ref[1]) <= 2.0 ** -16 * size + 2.0 ** -20 * (1 + np.abs(ref[1]))).all()
    assert c.cache.device_status() == 0


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", ROWS)
@pytest.mark.parametrize("high", [0, 1])
@pytest.mark.parametrize("power", [21, 24, 25, 26])
def test_scores_one_step_of_fp32_apart(cuda_device, d, Hq, Hkv, n, high, power):
    """Scores of 1.5 * 2^power, in powers of two, where fp32 steps by 2^(power - 23): a few keys are one step above the others."""
    c = Case(cuda_device, Hq, Hkv, d, [900], seed=23, softmax_scale=math.log(2))
    k, v = torch.zeros(900, Hkv, d, dtype=torch.bfloat16), 1 + c.randn(900, Hkv, d, scale=0.5)
    k[:, :, 0] = 1.5 * 2.0 ** (power - 10)
    few = torch.arange(900) % 128 == 77 if high else torch.arange(900) // 64 == 6
    k[few, :, 1] = 2.0 ** (power - 23)
    q = torch.zeros(n, Hq, d, dtype=torch.bfloat16)
    q[:, :, 0], q[:, :, 1] = 2 ** 10, 1
    c.append([900], k=k, v=v, twin=False)
    c.take_gpu_state()
    _, got, lse = c.attend([n], False, q=q, check=False)
    ref = reference(c, q, False)
    check(got, torch.from_numpy(ref[1]), ref, 0.0)
    assert (np.abs(lse.double().cpu().numpy() - ref[1]) <= 2.0 ** -22 * np.abs(ref[1])).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,n", ROWS)
@pytest.mark.parametrize("tokens", [500, 9000])
def test_rows_beside_far_ones_keep_their_bits(cuda_device, d, Hq, Hkv, n, tokens):
    """Rows whose scores are ordinary give the same bits whether or not rows beside them have scores of 2^40."""
    c = Case(cuda_device, Hq, Hkv, d, [tokens], seed=24, max_tokens=tokens)
    k, v = c.randn(tokens, Hkv, d), c.randn(tokens, Hkv, d)
    k[:, :, 0] = 0
    k[70, :, 0], k[300, :, 0] = 2.0 ** 40, -2.0 ** 41
    q = c.randn(n, Hq, d)
    q[..., 0] = 0
    far = torch.rand(n, Hq, generator=c.g) < 0.3
    other = q.clone()
    other[..., 0][far] = 1
    c.append([tokens], k=k, v=v, twin=False)
    _, want, want_lse = c.attend([n], True, q=q, check=False)
    _, got, lse = c.attend([n], True, q=other, check=False)
    keep = ~far
    assert torch.equal(got.cpu()[keep], want.cpu()[keep]) and torch.equal(lse.cpu()[keep], want_lse.cpu()[keep])
    assert not far.any() or (lse.cpu()[far] > 1e9).all()
    assert c.cache.device_status() == 0
