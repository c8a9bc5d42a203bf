"""The 8-bit paged cache: refusals on the host; append, attention and a run of the three operators together against
the fp64 reference on the GPU."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import kv8_oracle as O
from paper_2609_34606_b200 import hsa


# ------------------------------------------------------------------ host
CFG = dict(num_heads=8, num_kv_heads=2, head_dim=128, page_tokens=64, max_pages=16, max_blocks=8, max_batch=4, max_tokens=512,
           softmax_scale=0.0, flags=0)


def test_sizes_and_config_refusals():
    s = hsa.hsa_kv8_query_sizes(hsa.hsa_kv8_config(*CFG.values()))
    assert s.k_pool == s.v_pool == 16 * 2 * 64 * 128 and s.k_scale == s.v_scale == 16 * 2 * 4
    assert s.page_table == 4 * 8 * 4 and s.ksum == 4 * 2 * 8 * 128 * 4 and s.workspace > 0
    for bad in [dict(num_heads=0), dict(num_heads=7), dict(num_heads=2048, num_kv_heads=1), dict(num_kv_heads=0), dict(head_dim=96),
                dict(page_tokens=32), dict(max_pages=0), dict(max_blocks=0), dict(max_batch=0), dict(max_batch=5000),
                dict(max_tokens=0), dict(softmax_scale=-1.0), dict(softmax_scale=math.inf), dict(softmax_scale=math.nan), dict(flags=1),
                dict(max_pages=1 << 28), dict(max_blocks=1 << 25)]:
        with pytest.raises(hsa.HSAError) as e:
            hsa.hsa_kv8_query_sizes(hsa.hsa_kv8_config(*{**CFG, **bad}.values()))
        assert e.value.code == hsa.HSA_ERR_INVALID_ARG, bad


def test_create_refusals_on_host():
    lib, h = hsa._lib, C.c_void_p()
    cfg = hsa.hsa_kv8_config(*CFG.values())
    ok = [0x10000, 0x20000, 0x30000, 0x40000, 0x50000, 0x60000, 0x70000]
    for i, v in [(0, None), (1, None), (2, None), (3, None), (4, None), (6, None), (0, 0x10080), (1, 0x20010), (2, 0x30004),
                 (3, 0x40008), (4, 0x50004), (5, 0x60008), (6, 0x70080)]:
        b = list(ok)
        b[i] = v
        assert lib.hsa_kv8_create(C.byref(h), C.byref(cfg), C.byref(hsa.hsa_kv8_buffers(*b))) == hsa.HSA_ERR_INVALID_ARG, (i, v)
    assert lib.hsa_kv8_create(None, None, None) == hsa.HSA_ERR_INVALID_ARG
    assert lib.hsa_kv8_create(C.byref(h), None, None) == hsa.HSA_ERR_INVALID_ARG and h.value is None
    assert lib.hsa_kv8_destroy(None) == hsa.HSA_ERR_INVALID_ARG
    assert lib.hsa_kv8_append(None, 1, 1, 1, 1, 128, 128, None, 1, 1, None, None) == hsa.HSA_ERR_INVALID_ARG
    assert lib.hsa_kv8_attend(None, 1, 1, 1, 128, 128, None, 1, 1, 0, None, None, 0, 1, 128, 128, None, None) == hsa.HSA_ERR_INVALID_ARG
    assert lib.hsa_kv8_device_status(None, None) == hsa.HSA_ERR_INVALID_ARG and lib.hsa_kv8_last_cuda_error(None) == 0
    assert "not finite" in hsa.hsa_status_string(hsa.HSA_ERR_DEVICE_NONFINITE)


# ------------------------------------------------------------------ GPU
def dev_i32(x, device):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device=device)


class Case:
    """A cache, its twin in fp64, and the tokens that went in."""

    def __init__(self, device, Hq, Hkv, d, lengths, spare=0, sums=False, max_tokens=4096, seed=0, softmax_scale=0.0):
        self.device, self.Hq, self.Hkv, self.d, self.batch = device, Hq, Hkv, d, len(lengths)
        self.g = torch.Generator().manual_seed(seed)
        blocks = max(1, max(-(-n // 64) for n in lengths))
        pages = self.batch * blocks + 3
        order = torch.randperm(pages, generator=self.g)[:self.batch * blocks]
        self.table = order.view(self.batch, blocks).to(torch.int32)
        self.cache = hsa.KV8Cache(Hq, Hkv, d, pages, blocks, self.batch, max_tokens, softmax_scale, device=device, key_sums=sums,
                                  page_table=self.table.to(device))
        c = self.cache
        for t in (c.k_codes, c.v_codes):         # what nobody wrote is NaN
            t.view(torch.uint8).fill_(0xFF)
        c.k_scale.fill_(float("nan"))
        c.v_scale.fill_(float("nan"))
        if c.ksum is not None:
            c.ksum.fill_(float("nan"))
        nan = lambda *s: np.full(s, np.nan)
        self.state = {"k_codes": nan(pages, Hkv, 64, d), "v_codes": nan(pages, Hkv, 64, d), "k_scale": nan(pages, Hkv),
                      "v_scale": nan(pages, Hkv), "sums": nan(self.batch, Hkv, blocks, d) if sums else None}
        self.held = [0] * self.batch

    def randn(self, *shape, scale=1.0):
        return (torch.randn(*shape, generator=self.g) * scale).to(torch.bfloat16)

    def append(self, counts, rope=None, positions=None, scale=1.0, k=None, v=None, twin=True, max_new=None):
        n = sum(counts)
        k = self.randn(n, self.Hkv, self.d, scale=scale) if k is None else k
        v = self.randn(n, self.Hkv, self.d, scale=scale) if v is None else v
        starts = np.concatenate([[0], np.cumsum(counts)])
        pos = None if positions is None else dev_i32(positions, self.device)
        self.cache.append(k.to(self.device), v.to(self.device), dev_i32(self.held, self.device),
                          token_start=dev_i32(starts, self.device), max_new=max_new or max(counts), rope=rope, positions=pos)
        if twin:
            K, V = k.double().numpy(), v.double().numpy()
            if rope is not None:
                c = rope.cfg
                pairs = list(c.axis_pairs)[:c.n_axes]
                at = positions if positions is not None else np.concatenate(
                    [np.arange(h, h + m) for h, m in zip(self.held, counts)])[None].repeat(c.n_axes, 0)
                f, a = O.frequencies(pairs, c.base)
                K = O.rope(K, at, pairs, f, a, "half" if c.layout == 0 else "interleaved")
            cut = lambda x: [x[starts[i]:starts[i + 1]] for i in range(self.batch)]
            O.append(self.state, self.table.numpy(), self.held, cut(K), cut(V))
        self.held = [h + m for h, m in zip(self.held, counts)]
        return k, v

    def written(self):
        return [(s, b, int(self.table[s, b])) for s in range(self.batch) for b in range(-(-self.held[s] // 64))]

    def take_gpu_state(self):
        """The twin holds what the cache holds (attention is judged on the same codes)."""
        c = self.cache
        self.state["k_codes"], self.state["v_codes"] = (t.float().double().cpu().numpy() for t in (c.k_codes, c.v_codes))
        self.state["k_scale"], self.state["v_scale"] = (t.double().cpu().numpy() for t in (c.k_scale, c.v_scale))

    def check_state(self, exact):
        """exact: no rotation, so that every code is determined.  Else the rotated value is off by some 2^-21 of its pair,
        which may move a code to the neighbour of the nearest, or a scale across its border."""
        c = self.cache
        for name in ("k", "v"):
            codes = getattr(c, name + "_codes").float().double().cpu().numpy()
            scale = getattr(c, name + "_scale").double().cpu().numpy()
            for s, b, page in self.written():
                ref, ref_scale = self.state[name + "_codes"][page], self.state[name + "_scale"][page]
                if exact or name == "v":
                    assert np.array_equal(scale[page], ref_scale), (name, s, b)
                    assert np.array_equal(codes[page], ref), (name, s, b)
                    continue
                assert np.isin(scale[page] / ref_scale, (0.5, 1.0, 2.0)).all()
                got, want = codes[page] * scale[page][:, None, None], ref * ref_scale[:, None, None]
                # neighbours in e4m3: 2^-3 of the value, or the subnormal step of the scale
                assert (np.abs(got - want) <= np.maximum(2.0 ** -3 * np.abs(want) * 1.01, 2.0 ** -8 * ref_scale[:, None, None])).all()
                assert (got != want).mean() < 1e-2, "far more than lie that near a border"
        unwritten = sorted(set(range(c.max_pages)) - {p for _, _, p in self.written()})
        for t in (c.k_codes, c.v_codes):
            assert (t.view(torch.uint8)[unwritten] == 0xFF).all()
        assert c.k_scale[unwritten].isnan().all() and c.v_scale[unwritten].isnan().all()
        if c.ksum is not None:
            got = c.ksum.double().cpu().numpy()
            for s, b, page in self.written():
                ref, size = self.state["sums"][s, :, b], np.abs(self.state["k_codes"][page] * self.state["k_scale"][page][:, None, None])
                # 64 values in fp32, summed in two stages: at most 20 roundings of 2^-24 deep; rotated ones are off by 2^-20 of
                # the largest; stored ones may be a neighbouring code
                slack = 0.0 if exact else 2.0 ** -3
                bound = 20 * 2.0 ** -24 * size.sum(1) * 1.07 + (2.0 ** -18 * size.max() * 64 if not exact else 0) + slack * size.max(1)
                assert (np.abs(got[s, :, b] - ref) <= bound).all()

    def attend(self, counts, causal, sel=None, lengths=None, with_lse=True, out=None, q=None, max_q=None, q_scale=1.0, check=True):
        n = sum(counts)
        q = self.randn(n, self.Hq, self.d, scale=q_scale) if q is None else q
        starts = np.concatenate([[0], np.cumsum(counts)])
        lengths = self.held if lengths is None else lengths
        args = {}
        if sel is not None:
            most = max(1, max(len(x) for s in sel for x in s))
            idx = np.full((self.batch, self.Hkv, most), -7)
            for s in range(self.batch):
                for h in range(self.Hkv):
                    idx[s, h, :len(sel[s][h])] = sel[s][h]
            args = dict(sel_idx=dev_i32(idx, self.device), sel_cnt=dev_i32([[len(x) for x in s] for s in sel], self.device))
        got, lse = self.cache.attend(q.to(self.device), dev_i32(lengths, self.device), token_start=dev_i32(starts, self.device),
                                     max_q=max_q or max(1, max(counts)), causal=causal, with_lse=True, out=out, **args)
        if check:
            Q = q.double().numpy()
            ref = O.attend([Q[starts[i]:starts[i + 1]] for i in range(self.batch)], self.state, self.table.numpy(), lengths, causal,
                           self.cache.cfg.softmax_scale or None, sel)
            size = [float(np.abs(self.state["k_codes"][p] * self.state["k_scale"][p][..., None, None]).sum(-1).max(initial=0.0))
                    for p in [[int(self.table[s, b]) for b in range(-(-lengths[s] // 64))] for s in range(self.batch)]]
            for i in range(self.batch):
                at = slice(int(starts[i]), int(starts[i + 1]))
                assert_attention(got[at], lse[at], ref[i], Q[at], size[i])
        return q, got, lse


def assert_attention(got, lse, ref, q, k_size):
    """out: half a step of bf16 (2^-8); every weight w_j off by 2^-8 of itself or 2^-21 of the largest one, which the sum of
    weights is no smaller than, so that sum_j |dw_j| |v_j| / sum_j w_j <= 2^-8 spread + 2^-21 size (twice that with the fp32
    sums); and by its score's error: products exact or short by 2^-17 of max|q| |k|_1, sums of 128 terms in fp32, taken as 2^-16
    together, which moves numerator and denominator by as much each.  lse: the same score error, and fp32 logarithms."""
    out, lse_ref, spread, size = ref
    score = 2.0 ** -16 * np.abs(q).max(initial=0.0) * k_size / math.sqrt(q.shape[-1]) + 2.0 ** -20
    empty = np.isneginf(lse_ref)
    d = np.abs(got.double().cpu().numpy() - out)
    bound = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 * 1.02 + 2 * score) * spread + 2.0 ** -20 * size + 1e-30
    assert (d <= bound).all(), ((d - bound).max(), np.argwhere(d > bound)[:4])
    got_lse = lse.double().cpu().numpy()
    assert np.array_equal(np.isneginf(got_lse), empty)
    assert (got.float().cpu().numpy()[empty] == 0).all()
    e = np.abs(got_lse[~empty] - lse_ref[~empty])
    assert (e <= score + 2.0 ** -20 * (1 + np.abs(lse_ref[~empty]))).all(), e.max()


SHAPES = [(1, 1, 64), (12, 12, 128), (8, 2, 128), (6, 1, 64), (40, 8, 64), (5, 5, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sums", [False, True])
@pytest.mark.parametrize("counts", [[1], [63], [64], [65], [200], [1, 0, 64, 129], [3, 70, 1, 0, 0, 500]])
def test_append_without_positions(cuda_device, d, sums, counts):
    """Codes, scales and sums bit for bit, over appends that begin and end anywhere in a page and whose sizes grow."""
    c = Case(cuda_device, 3, 3, d, [3 * n + 140 for n in counts], sums=sums, seed=d + len(counts))
    for scale, more in ((1.0, counts), (0.01, [min(1, n) for n in counts]), (300.0, [2 if n else 0 for n in counts]), (1e-9, counts),
                        (1.0, [1] * len(counts)), (2.0, [64] * len(counts))):
        if sum(more):
            c.append(more, scale=scale)
            c.check_state(exact=True)
    assert c.cache.device_status() == 0


@pytest.mark.gpu
def test_append_token_by_token(cuda_device):
    c = Case(cuda_device, 2, 2, 64, [140, 140], sums=True, seed=1)
    for i in range(140):
        c.append([1, 1], scale=1.0 if i % 50 else 20.0)
    c.check_state(exact=True)


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,pairs", [(128, (64,)), (128, (22, 21, 21)), (64, (32,)), (64, (31,)), (128, (9,)), (64, (5, 0, 8)), (128, (40,))])
def test_append_with_positions(cuda_device, layout, d, pairs):
    c = Case(cuda_device, 2, 2, d, [400, 400, 400], sums=True, seed=len(pairs) + d)
    rope = hsa.RotaryPositions(d, 2 * sum(pairs), layout, axis_pairs=pairs, device=cuda_device)
    c.append([100, 1, 64], rope=rope)
    c.check_state(exact=False)
    pos = torch.randint(-9, 1 << 20, (len(pairs), 37 + 5 + 150), generator=c.g).numpy()
    c.append([37, 5, 150], rope=rope, positions=pos)
    c.check_state(exact=False)
    assert c.cache.device_status() == 0


@pytest.mark.gpu
def test_append_many_heads_to_a_block(cuda_device):
    """Enough blocks that a CTA takes several heads, the last share a short one."""
    c = Case(cuda_device, 13, 13, 64, [20000], sums=True, seed=5, max_tokens=20000)
    rope = hsa.RotaryPositions(64, 64, "half", device=cuda_device)
    k, v = c.append([20000], rope=rope, twin=False)
    ref = Case(cuda_device, 13, 13, 64, [20000], sums=True, seed=5, max_tokens=20000)
    y = rope.apply(k.to(cuda_device))                      # rounds to bf16: keys that stay as they are
    ref.append([20000], k=y.cpu(), v=v, twin=False)
    a, b = (x.cache.k_codes.float() * x.cache.k_scale[..., None, None] for x in (c, ref))
    pages = [p for _, _, p in c.written()]
    a, b = a[pages], b[pages]
    # y is off by half a step of bf16, its code by half a step of e4m3: 2^-8 + 2 * 2^-4 of the value, or a subnormal step
    assert ((a - b).abs() <= (2.0 ** -8 + 2.0 ** -3) * torch.maximum(a.abs(), b.abs()) + 2.0 ** -9 * ref.cache.k_scale[pages][..., None, None]).all()
    assert torch.equal(c.cache.v_codes.view(torch.uint8)[pages], ref.cache.v_codes.view(torch.uint8)[pages])


@pytest.mark.gpu
def test_append_again_leaves_the_same_bits(cuda_device):
    c = Case(cuda_device, 2, 2, 128, [300, 300], sums=True, seed=6)
    c.append([70, 130])
    rope = hsa.RotaryPositions(128, device=cuda_device)
    before = list(c.held)
    k, v = c.append([100, 9], rope=rope, scale=5.0)
    first = [t.clone() for t in (c.cache.k_codes.view(torch.uint8), c.cache.v_codes.view(torch.uint8), c.cache.k_scale,
                                 c.cache.v_scale, c.cache.ksum)]
    c.held = before
    c.append([100, 9], rope=rope, k=k, v=v, twin=False)
    for x, y in zip(first, (c.cache.k_codes.view(torch.uint8), c.cache.v_codes.view(torch.uint8), c.cache.k_scale, c.cache.v_scale,
                            c.cache.ksum)):
        assert torch.equal(x.nan_to_num(7.0) if x.is_floating_point() else x, y.nan_to_num(7.0) if y.is_floating_point() else y)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 3e38])
def test_append_of_what_cannot_be_stored(cuda_device, value):
    """NaN becomes 0, the others 2^60, the status word says so, and other pages know nothing of it."""
    c = Case(cuda_device, 2, 2, 64, [128], sums=True)
    k, v = c.randn(128, 2, 64), c.randn(128, 2, 64)
    k[70, 1, 5] = value
    v[3, 0, 9] = value
    c.append([128], k=k, v=v)
    c.check_state(exact=True)
    assert c.cache.device_status() == hsa.HSA_ERR_DEVICE_NONFINITE
    assert c.cache.device_status() == 0
    c.attend([1], causal=True)


@pytest.mark.gpu
def test_append_extremes(cuda_device):
    """Zeros, the smallest and the largest values that are stored; strided rows."""
    c = Case(cuda_device, 2, 2, 64, [256], sums=True, max_tokens=256)
    k = torch.zeros(256, 2, 64, dtype=torch.bfloat16)
    v = c.randn(256, 2, 64)
    v[0:64] = 0
    v[64:128] *= 2.0 ** -45
    v[128:192] *= 2.0 ** 57
    v[192:256] = 448.0
    c.append([256], k=k, v=v)
    c.check_state(exact=True)
    assert c.cache.device_status() == 0
    wide = torch.zeros(100, 5, 3, 64, dtype=torch.bfloat16, device=cuda_device).normal_()
    x, y = Case(cuda_device, 2, 2, 64, [100], seed=1), Case(cuda_device, 2, 2, 64, [100], seed=1)
    held = dev_i32([0], cuda_device)
    x.cache.append(wide[:, 0:4:2, 1], wide[:, 1:4:2, 2], held)
    y.cache.append(wide[:, 0:4:2, 1].contiguous(), wide[:, 1:4:2, 2].contiguous(), held)
    assert torch.equal(x.cache.k_codes.view(torch.uint8), y.cache.k_codes.view(torch.uint8))
    assert torch.equal(x.cache.v_codes.view(torch.uint8), y.cache.v_codes.view(torch.uint8))


@pytest.mark.gpu
def test_append_leaves_out_what_does_not_fit(cuda_device):
    """Sequences whose rows or lengths do not fit, and pages outside the pools, are left alone and reported; the others
    are served."""
    dev = cuda_device

    def fresh():
        c = Case(dev, 1, 1, 64, [128, 128, 128], max_tokens=64)
        return c, c.randn(30, 1, 64).to(dev)

    for starts, held, good in [([0, 10, 8, 30], [0, 0, 0], [0, 2]), ([0, 10, 20, 31], [0, 0, 0], [0, 1]), ([-1, 10, 20, 30], [0, 0, 0], [1, 2]),
                               ([0, 10, 20, 30], [0, -1, 0], [0, 2]), ([0, 10, 20, 30], [119, 0, 0], [1, 2]), ([0, 26, 28, 30], [0, 0, 0], [1, 2])]:
        c, k = fresh()
        c.cache.append(k, k, dev_i32(held, dev), token_start=dev_i32(starts, dev), max_new=25 if starts[1] == 26 else 30)
        assert c.cache.device_status() == hsa.HSA_ERR_DEVICE_BOUNDS, (starts, held)
        touched = {int(p) for p in (c.cache.k_scale[:, 0] == c.cache.k_scale[:, 0]).nonzero()}
        assert touched == {int(c.table[s, held[s] // 64]) for s in good}, (starts, held)
    for page in (-1, 9, 1 << 30):
        c, k = fresh()
        c.cache.page_table[1, 0] = page
        c.cache.append(k, k, dev_i32([0, 0, 0], dev))
        assert c.cache.device_status() == hsa.HSA_ERR_DEVICE_BOUNDS
        touched = {int(p) for p in (c.cache.k_scale[:, 0] == c.cache.k_scale[:, 0]).nonzero()}
        assert touched == {int(c.table[0, 0]), int(c.table[2, 0])}


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
@pytest.mark.parametrize("causal", [False, True])
def test_attend_single_tokens(cuda_device, Hq, Hkv, d, causal):
    """A token of each sequence, histories from one token to some that are split over the device."""
    lengths = [1, 64, 65, 777, 130, 1, 2000]
    c = Case(cuda_device, Hq, Hkv, d, lengths, seed=Hq)
    c.append(lengths)
    c.take_gpu_state()
    c.attend([1] * len(lengths), causal)
    c.attend([1, 0, 1, 0, 0, 1, 1], causal)
    assert c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("counts", [[2, 3, 5, 1], [17, 64, 0, 33], [129, 40, 200, 256], [300, 1, 31, 2]])
def test_attend_chunks(cuda_device, Hq, Hkv, d, causal, counts):
    """Ragged queries at the end of ragged histories; as many queries as tokens, and one more of either."""
    for past in ([0, 0, 0, 0], [1, 63, 65, 300]):
        lengths = [a + b for a, b in zip(past, counts)]
        c = Case(cuda_device, Hq, Hkv, d, [max(1, n) for n in lengths], seed=sum(counts))
        c.append(lengths)
        c.take_gpu_state()
        c.attend(counts, causal)
        assert c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[1, 1], [20, 3], [150, 70]])
@pytest.mark.parametrize("causal", [False, True])
def test_attend_with_nothing_to_see(cuda_device, counts, causal):
    """More queries than tokens: the first ones stand before the sequence; a length of zero leaves all of them empty."""
    c = Case(cuda_device, 4, 2, 128, [200, 200], seed=2)
    c.append([200, 200])
    c.take_gpu_state()
    c.attend(counts, causal, lengths=[0, 0])
    c.attend(counts, causal, lengths=[1, 0])
    c.attend(counts, causal, lengths=[max(0, counts[0] - 1), counts[1] // 2])
    c.attend(counts, causal, lengths=[199, 64])          # shorter than what the pages hold


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d", SHAPES)
@pytest.mark.parametrize("counts", [[1, 1], [9, 30], [140, 300]])
@pytest.mark.parametrize("causal", [False, True])
def test_attend_lists(cuda_device, Hq, Hkv, d, counts, causal):
    """Block lists of every length, in any order, an entry twice, blocks behind the length, an empty list."""
    lengths = [700, 450]
    c = Case(cuda_device, Hq, Hkv, d, lengths, seed=7)
    c.append(lengths)
    c.take_gpu_state()
    rng = np.random.default_rng(3)
    some = lambda n, k: list(rng.permutation(n)[:k])
    sel = [[some(11, 1 + h % 5) for h in range(Hkv)], [some(8, (3 * h) % 8) for h in range(Hkv)]]
    c.attend(counts, causal, sel=sel)
    sel = [[[4, 4, 1, 10] for _ in range(Hkv)], [[10, 7, 9, 0] if h % 2 else [] for h in range(Hkv)]]
    c.attend(counts, causal, sel=sel)
    assert c.cache.device_status() == 0


@pytest.mark.gpu
def test_attend_bad_lists_and_pages(cuda_device):
    """Entries outside the table and pages outside the pools count as not seen, and are reported."""
    for counts in ([1], [5], [140]):
        c = Case(cuda_device, 4, 2, 128, [500], seed=8)
        c.append([500])
        c.take_gpu_state()
        n = sum(counts)
        q = c.randn(n, 4, 128)
        idx = torch.tensor([[[0, -1, 3, 8], [99, 2, 1 << 30, 5]]], dtype=torch.int32, device=cuda_device)
        cnt = torch.tensor([[4, 9]], dtype=torch.int32, device=cuda_device)
        call = lambda i, m: c.cache.attend(q.to(cuda_device), dev_i32([500], cuda_device), causal=True, sel_idx=i, sel_cnt=m, with_lse=True)
        got = call(idx, cnt)
        assert c.cache.device_status() == hsa.HSA_ERR_DEVICE_BOUNDS
        good = torch.tensor([[[0, 3, 3, 3], [2, 5, 5, 5]]], dtype=torch.int32, device=cuda_device)
        want = call(good, torch.full_like(cnt, 2))
        assert c.cache.device_status() == 0
        assert torch.allclose(got[0].float(), want[0].float(), atol=2e-2, rtol=1e-2) and torch.allclose(got[1], want[1], atol=1e-4)
        assert call(idx, -cnt)[1].isneginf().all()
        before = c.cache.page_table.clone()
        c.cache.page_table[0, 1], c.cache.page_table[0, 6] = -5, c.cache.max_pages
        got = c.cache.attend(q.to(cuda_device), dev_i32([500], cuda_device), causal=True, with_lse=True)
        assert c.cache.device_status() == hsa.HSA_ERR_DEVICE_BOUNDS
        c.cache.page_table.copy_(before)
        six = torch.tensor([[[0, 2, 3, 4, 5, 7]] * 2], dtype=torch.int32, device=cuda_device)
        want = call(six, torch.full_like(cnt, 6))
        assert torch.allclose(got[0].float(), want[0].float(), atol=2e-2, rtol=1e-2) and torch.allclose(got[1], want[1], atol=1e-4)
        assert c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("big", [False, True])
def test_attend_leaves_other_rows_alone(cuda_device, big):
    """Rows behind the last sequence, between sequences and of sequences that do not fit stay as they were."""
    f = 20 if big else 1
    dev = cuda_device
    c = Case(dev, 4, 2, 64, [300, 300, 300], seed=9)
    c.append([300, 300, 300])
    c.take_gpu_state()
    n = 20 * f
    q = c.randn(n, 4, 64).to(dev)
    for starts, lengths, served in [([2 * f, 5 * f, 9 * f, 12 * f], [300, 200, 100], [0, 1, 2]), ([0, 5 * f, 4 * f, 12 * f], [300, 200, 100], [0, 2]),
                                    ([0, 5 * f, 9 * f, 21 * f], [300, 200, 100], [0, 1]), ([0, 4 * f, 8 * f, 12 * f], [300, -1, 321], [0])]:
        out = torch.full_like(q, 7.0)
        c.cache.attend(q, dev_i32(lengths, dev), token_start=dev_i32(starts, dev), max_q=9 * f, causal=True, out=out)
        assert c.cache.device_status() == (0 if len(served) == 3 else hsa.HSA_ERR_DEVICE_BOUNDS)
        mine = torch.zeros(n, dtype=torch.bool)
        for s in served:
            mine[starts[s]:starts[s + 1]] = True
        assert (out[~mine.to(dev)] == 7.0).all()
        assert (out[mine.to(dev)] != 7.0).any(-1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[1, 1], [3, 40], [200, 260]])
def test_rows_are_independent_of_infinities_and_of_stale_values(cuda_device, counts):
    """A query that is Inf or NaN spoils its own row alone; so do huge stored values that it does not see."""
    c = Case(cuda_device, 4, 2, 128, [400, 400], seed=10)
    v = c.randn(800, 2, 128)
    v[390:400] *= 2.0 ** 50                    # the last tokens of the first sequence
    c.append([400, 400], v=v, k=c.randn(800, 2, 128))
    c.take_gpu_state()
    n = sum(counts)
    q = c.randn(n, 4, 128)
    lengths = [390, 400]
    _, want, want_lse = c.attend(counts, True, lengths=lengths, q=q)
    bad = q.clone()
    bad[0, 1, 3], bad[n - 1, 3, 0] = math.nan, math.inf
    _, got, lse = c.attend(counts, True, lengths=lengths, q=bad, check=False)
    keep = torch.ones(n, 4, dtype=torch.bool)
    keep[0, 1] = keep[n - 1, 3] = False
    assert torch.equal(got.cpu()[keep], want.cpu()[keep]) and torch.equal(lse.cpu()[keep], want_lse.cpu()[keep])
    assert got.cpu()[0, 1].isnan().all() and got.cpu()[n - 1, 3].isnan().any()


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[1], [6], [130]])
@pytest.mark.parametrize("q_scale", [0.0, 1e-6, 30.0, 1e4])
def test_attend_flat_and_peaked(cuda_device, counts, q_scale):
    """Weights all alike, and weights that rise for as long as the history goes on, pages of very different size."""
    c = Case(cuda_device, 2, 2, 64, [900], seed=11)
    k, v = c.randn(900, 2, 64), c.randn(900, 2, 64)
    k[:, :, 0] += torch.linspace(-3, 3, 900)[:, None]
    for b in range(0, 900, 64):
        v[b:b + 64] *= 2.0 ** ((b // 64 * 7) % 23 - 11)
    c.append([900], k=k, v=v)
    c.take_gpu_state()
    c.attend(counts, False, q_scale=q_scale)
    c.attend(counts, True, q_scale=q_scale)


@pytest.mark.gpu
def test_attend_scale_and_equal_shares(cuda_device):
    c = Case(cuda_device, 4, 4, 128, [333, 90, 5], seed=12, softmax_scale=0.25)
    c.append([333, 90, 5])
    c.take_gpu_state()
    q, got, _ = c.attend([4, 4, 4], True)
    again = c.cache.attend(q.to(cuda_device), dev_i32(c.held, cuda_device))       # no token_start: equal shares
    assert torch.equal(got, again)
    wide = torch.zeros(12, 2, 4, 2, 128, dtype=torch.bfloat16, device=cuda_device)
    wide[:, 1, :, 0] = q.to(cuda_device)
    out = torch.zeros(12, 8, 128, dtype=torch.bfloat16, device=cuda_device)[:, ::2]
    assert torch.equal(c.cache.attend(wide[:, 1, :, 0], dev_i32(c.held, cuda_device), out=out), got)


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[1, 1, 1], [5, 40, 2], [300, 150, 400]])
def test_attend_twice_gives_the_same_bits_captured_or_not(cuda_device, counts):
    """Work that is split over CTAs is joined in a fixed order; a replayed graph follows lengths and tables."""
    dev = cuda_device
    c = Case(dev, 8, 2, 128, [3000, 3000, 3000], seed=13, max_tokens=9000)
    c.append([3000, 2000, 2500])
    c.take_gpu_state()
    q, want, want_lse = c.attend(counts, True, check=False)
    for _ in range(3):
        _, got, lse = c.attend(counts, True, q=q, check=False)
        assert torch.equal(got, want) and torch.equal(lse, want_lse)
    qd, out = q.to(dev), torch.empty_like(want)
    lengths, starts = dev_i32(c.held, dev), dev_i32(np.concatenate([[0], np.cumsum(counts)]), dev)
    call = lambda o: c.cache.attend(qd, lengths, token_start=starts, max_q=max(counts), causal=True, out=o)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    lengths -= 501
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, call(None)) and not torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call(None)
    side.synchronize()
    assert torch.equal(out, got)


@pytest.mark.gpu
def test_parts_of_a_history_join_through_their_lse(cuda_device):
    """Attention over two disjoint lists, joined by their lse, is attention over both."""
    c = Case(cuda_device, 4, 2, 128, [640], seed=14)
    c.append([640])
    c.take_gpu_state()
    q = c.randn(30, 4, 128)
    a, b = [[[0, 3, 5, 9]] * 2], [[[1, 2, 4, 6, 7, 8]] * 2]
    _, o1, l1 = c.attend([30], False, sel=a, q=q)
    _, o2, l2 = c.attend([30], False, sel=b, q=q)
    _, o, l = c.attend([30], False, q=q)
    both = torch.logaddexp(l1, l2)
    joined = o1.float() * (l1 - both).exp()[..., None] + o2.float() * (l2 - both).exp()[..., None]
    # |v| < 4.5: each side off by 2^-8 of its output and 2^-8 of its weights' mean
    assert (joined - o.float()).abs().max() < 4 * 2.0 ** -8 * 4.5 and (both - l).abs().max() < 1e-4


@pytest.mark.gpu
def test_call_refusals_with_a_context(cuda_device):
    dev = cuda_device
    c = Case(dev, 4, 2, 64, [128, 128], max_tokens=64)
    k, q = torch.zeros(10, 2, 64, dtype=torch.bfloat16, device=dev), torch.zeros(10, 4, 64, dtype=torch.bfloat16, device=dev)
    held = dev_i32([0, 0], dev)
    lib, ctx = hsa._lib, c.cache.ctx

    def append(**kw):
        a = {**dict(k=k.data_ptr(), v=k.data_ptr(), n=10, batch=2, ts=128, hs=64, start=None, most=5, held=held.data_ptr()), **kw}
        return lib.hsa_kv8_append(ctx, a["k"], a["v"], a["n"], a["batch"], a["ts"], a["hs"], a["start"], a["most"], a["held"], None, None)

    def attend(**kw):
        a = {**dict(q=q.data_ptr(), n=10, batch=2, ts=256, hs=64, start=None, most=5, len=held.data_ptr(), idx=None, cnt=None, topk=0,
                    out=q.data_ptr(), ots=256, ohs=64, lse=None), **kw}
        return lib.hsa_kv8_attend(ctx, a["q"], a["n"], a["batch"], a["ts"], a["hs"], a["start"], a["most"], a["len"], 1, a["idx"], a["cnt"],
                                  a["topk"], a["out"], a["ots"], a["ohs"], a["lse"], None)

    bad = hsa.HSA_ERR_INVALID_ARG
    for kw in [dict(k=None), dict(v=None), dict(k=k.data_ptr() + 8), dict(n=-1), dict(n=65), dict(batch=0), dict(batch=3), dict(ts=60),
               dict(ts=132), dict(hs=32), dict(most=0), dict(most=4), dict(most=11), dict(held=None), dict(held=held.data_ptr() + 2)]:
        assert append(**kw) == bad, kw
    for kw in [dict(q=None), dict(out=None), dict(q=q.data_ptr() + 8), dict(n=65), dict(batch=0), dict(batch=3), dict(ts=60), dict(hs=100),
               dict(ots=60), dict(ohs=4), dict(most=0), dict(most=4), dict(len=None), dict(idx=held.data_ptr()), dict(cnt=held.data_ptr()),
               dict(idx=held.data_ptr(), cnt=held.data_ptr(), topk=0), dict(lse=held.data_ptr() + 1)]:
        assert attend(**kw) == bad, kw
    assert append(n=0) == attend(n=0) == hsa.HSA_OK
    cache = c.cache
    for call in [lambda: cache.append(k.float(), k.float(), held), lambda: cache.append(k, k[:5], held), lambda: cache.append(q, q, held),
                 lambda: cache.append(k, k, held.long()), lambda: cache.append(k, k, held, token_start=held),
                 lambda: cache.append(k, k, held, positions=held), lambda: cache.append(k.cpu(), k, held),
                 lambda: cache.append(k, k, held, rope=hsa.RotaryPositions(128, device=dev)),
                 lambda: cache.attend(k, held), lambda: cache.attend(q.half(), held), lambda: cache.attend(q, held.cpu()),
                 lambda: cache.attend(q, held, out=k), lambda: cache.attend(q, held, sel_idx=held),
                 lambda: cache.attend(q, held, sel_idx=torch.zeros(2, 4, 3, dtype=torch.int32, device=dev),
                                      sel_cnt=torch.zeros(2, 4, dtype=torch.int32, device=dev))]:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        hsa.KV8Cache(4, 2, 64, 9, 2, 2, 64, device=dev, page_table=torch.zeros(2, 3, dtype=torch.int32, device=dev))
    assert cache.device_status() == 0


@pytest.mark.gpu
def test_rollout_positions_append_select_attend(cuda_device):
    """The operators as a layer uses them: chunks of tokens with frame, row and column positions go into the cache, each
    head selects blocks by the cache's key sums, and the chunk attends to them; then one sequence goes on token by token."""
    dev, H, d, chunk, chunks, topk = cuda_device, 3, 128, 200, 6, 5
    total = chunk * chunks + 70
    c = Case(dev, H, H, d, [total], sums=True, seed=15)
    rope = hsa.RotaryPositions(d, d, "interleaved", axis_pairs=(22, 21, 21), device=dev)
    f, _ = O.frequencies((22, 21, 21), 1e4)
    place = lambda t: np.stack([t // 50, t % 50 // 10, t % 10])
    for i in range(chunks):
        t = np.arange(i * chunk, (i + 1) * chunk)
        c.append([chunk], rope=rope, positions=place(t))
        c.check_state(exact=False)
        q = c.randn(chunk, H, d)
        qr = rope.apply(q.to(dev), dev_i32(place(t), dev))
        n = c.held[0]
        idx, cnt = torch.zeros(H, 1, topk, dtype=torch.int32, device=dev), torch.zeros(H, 1, dtype=torch.int32, device=dev)
        budgets = torch.full((H,), topk, dtype=torch.int32, device=dev)
        hsa.hsa_select_blocks_noalloc(qr, c.cache.ksum[0], n, n, False, 0.0, budgets, idx, cnt)
        # the lists are the best blocks by the reference's scores, but for scores as near as the key sums are off
        mean_q = qr.double().cpu().numpy().mean(0)
        blocks = -(-n // 64)
        sums = c.cache.ksum[0, :, :blocks].double().cpu().numpy()
        score = np.einsum("hd,hbd->hb", mean_q, sums / np.array([min(64, n - 64 * b) for b in range(blocks)])[None, :, None])
        for h in range(H):
            mine = idx[h, 0, :int(cnt[h, 0])].cpu().numpy()
            assert len(mine) == min(topk, blocks)
            rest = np.setdiff1d(np.arange(blocks), mine)
            assert not len(rest) or score[h, mine].min() >= score[h, rest].max() - 1e-5
        c.take_gpu_state()
        out, lse = c.cache.attend(qr, dev_i32([n], dev), causal=False, sel_idx=idx.view(1, H, topk), sel_cnt=cnt.view(1, H), with_lse=True)
        sel = [[idx[h, 0, :int(cnt[h, 0])].tolist() for h in range(H)]]
        ref = O.attend([qr.double().cpu().numpy()], c.state, c.table.numpy(), [n], False, sel=sel)[0]
        k_size = float(np.abs(c.state["k_codes"] * c.state["k_scale"][..., None, None])[[p for _, _, p in c.written()]].sum(-1).max())
        assert_attention(out, lse, ref, qr.double().cpu().numpy(), k_size)
    for i in range(70):
        c.append([1], rope=rope, positions=place(np.array([c.held[0]])), twin=False)
        if i % 23 == 0:
            c.take_gpu_state()
            c.attend([1], True)
    assert c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("n", [1, 17])
def test_attend_more_sequences_than_a_plan_lists(cuda_device, n):
    """5600 (sequence, head) pairs: every CTA has more of them than its list of runs holds, for one query and for many."""
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in rng.integers(n, 140, 700)]
    lengths[5] = lengths[699] = n
    c = Case(cuda_device, 8, 8, 64, lengths, seed=16, max_tokens=sum(lengths))
    c.append(lengths, twin=False)
    c.take_gpu_state()
    c.attend([n] * 700, True)
    c.attend([n if i % 3 else 0 for i in range(700)], False)
    assert c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts", [[1], [30], [150]])
@pytest.mark.parametrize("far", [-120.0, 120.0])
def test_value_scales_far_apart(cuda_device, d, counts, far):
    """Pages whose values differ by 2^80: a page of huge values that nothing points at (`far` < 0) leaves the others their
    precision, and one that everything points at gives the result whatever the others hold."""
    c = Case(cuda_device, 2, 2, d, [256], seed=17)
    k, v = c.randn(256, 2, d), c.randn(256, 2, d)
    k[:, :, 0] = 0
    k[64:128, :, 0] = far * math.log(2) * math.sqrt(d)      # with a query of 1 there: weights of 2^far
    v[64:128] *= 2.0 ** 45
    v[128:192] *= 2.0 ** -35
    q = c.randn(sum(counts), 2, d)
    q[:, :, 0] = 1
    c.append([256], k=k, v=v)
    c.take_gpu_state()
    _, got, lse = c.attend(counts, False, q=q)
    ref = O.attend([q.double().numpy()], c.state, c.table.numpy(), [256], False)[0]
    # the pages that weigh: half a step of bf16 for the result and 2^-8 for the weights; scores as in assert_attention
    score = 2.0 ** -16 * float(q.abs().max()) * float(k.double().abs().sum(-1).max()) / math.sqrt(d) + 2.0 ** -20
    if far < 0:
        bound = 2.0 ** -8 * np.abs(ref[0]) + (2.0 ** -8 * 1.02 + 2 * score) * ref[2] + 2.0 ** -20 * 256 * 6
        assert (np.abs(got.double().cpu().numpy() - ref[0]) <= bound).all()
    else:
        bound = 2.0 ** -8 * np.abs(ref[0]) + (2.0 ** -8 * 1.02 + 2 * score) * ref[2] + 2.0 ** -20 * ref[3]
        assert (np.abs(got.double().cpu().numpy() - ref[0]) <= bound).all()
    assert c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [[100], [20, 3], [128, 128]])
def test_a_tile_of_rows_shared_by_both_halves_of_the_kernel(cuda_device, counts):
    """Items of at most 128 rows, whose pages two groups of warps take in turn: histories of one page, of two, of an odd
    number, and long ones that are split over the device."""
    for lengths in ([128 + 0, 128], [129, 200], [64 * 7, 64 * 9 + 1], [9000, 6001]):
        lengths = lengths[:len(counts)]
        for d, Hq, Hkv in ((128, 2, 2), (64, 5, 1) if max(counts) <= 20 else (64, 1, 1)):
            c = Case(cuda_device, Hq, Hkv, d, lengths, seed=18, max_tokens=16000)
            c.append(lengths, twin=False)
            c.take_gpu_state()
            c.attend(counts, True)
            c.attend(counts, False)
            assert c.cache.device_status() == 0
