"""The 8-bit paged cache at its edges: waits that run out, instances and calls that the other tests pass by."""
import numpy as np
import pytest
import torch

from paper_2609_34606_b200 import hsa
from test_kv8 import Case, dev_i32


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,counts,lengths", [(2, 2, [1], [20000]), (4, 2, [2, 7], [300, 9000]), (16, 1, [1, 1, 0], [5000, 70, 9]),
                                                   (4, 4, [20, 100], [2000, 3001]), (4, 2, [300, 1, 200], [9000, 1, 200]),
                                                   (3, 3, [1] * 200, [700] * 200), (2, 2, [40] * 160, [200] * 160)])
@pytest.mark.parametrize("listed", [False, True])
def test_attention_that_gives_up_leaves_the_context_usable(cuda_device, d, Hq, Hkv, counts, lengths, listed):
    """Waits of the attention kernels run out with copies and products in flight: the kernel ends by itself and says so, and the
    next call gives the usual bits."""
    c = Case(cuda_device, Hq, Hkv, d, lengths, seed=31, max_tokens=sum(lengths))
    c.append(lengths, twin=False)
    sel = None
    if listed:
        sel = [[list(c_) for c_ in [range(h % 2, -(-n // 64), 2)] * Hkv] for h, n in enumerate(lengths)]
    q, want, want_lse = c.attend(counts, True, sel=sel, check=False)
    assert c.cache.device_status() == 0
    for limit in (1, 1, 300, 1000, 3000, 10000, 20_000):
        c.cache.set_wait_limit_ns(limit)
        _, got, lse = c.attend(counts, True, sel=sel, q=q, check=False)
        status = c.cache.device_status()
        assert status == hsa.HSA_ERR_DEVICE_TIMEOUT or limit > 1 and status == 0
        if status == 0:
            assert torch.equal(got, want) and torch.equal(lse, want_lse)
    c.cache.set_wait_limit_ns(2_000_000_000)
    for _ in range(2):
        _, got, lse = c.attend(counts, True, sel=sel, q=q, check=False)
        assert c.cache.device_status() == 0 and torch.equal(got, want) and torch.equal(lse, want_lse)


# (query heads, key heads, tokens of each sequence): rows of a key head up to 2, 4, 8 and 16, each instance full and not
FEW = [(3, 3, [2, 1, 2]), (3, 1, [1, 1, 0]), (4, 4, [3, 4, 1]), (8, 1, [1, 1, 1]), (5, 1, [1, 0, 1]), (2, 2, [7, 8, 1]),
       (16, 1, [1, 1, 1]), (9, 1, [1, 1, 0]), (8, 2, [4, 3, 2]), (4, 4, [16, 9, 12]), (5, 1, [3, 2, 1])]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,counts", FEW)
def test_few_rows_of_every_instance(cuda_device, d, Hq, Hkv, counts):
    """Against the reference: whole histories and lists, causal and not, parts of an item on several SMs, rows that see nothing."""
    lengths = [16, 777, 5000]
    c = Case(cuda_device, Hq, Hkv, d, lengths, seed=32, max_tokens=6000)
    c.append(lengths, twin=False)
    c.take_gpu_state()
    rng = np.random.default_rng(4)
    for causal in (True, False):
        c.attend(counts, causal)
        c.attend(counts, causal, sel=[[list(rng.permutation(-(-n // 64))[:1 + (3 * h) % 7]) for h in range(Hkv)] for n in lengths])
        c.attend(counts, causal, sel=[[[]] * Hkv, [[12, 3, 3, 0]] * Hkv, [list(range(78, -1, -1))] * Hkv])
        c.attend(counts, causal, lengths=[0, 1, max(0, counts[2] - 1)])
    assert c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,most", [(2, 2, 1), (4, 2, 2), (4, 2, 4), (4, 2, 8), (6, 1, 2)])
def test_few_rows_leave_other_rows_alone(cuda_device, d, Hq, Hkv, most):
    """Rows behind the last sequence, between sequences and of sequences that do not fit stay as they were, those of lse too."""
    c = Case(cuda_device, Hq, Hkv, d, [300, 300, 300], seed=33)
    c.append([300, 300, 300], twin=False)
    n, m = 5 * most, most
    q = c.randn(n, Hq, d).to(cuda_device)
    i32 = lambda x: dev_i32(x, cuda_device)
    for starts, lengths, served in [([1, 1 + m, 1 + 2 * m, 1 + 3 * m], [300, 200, 100], [0, 1, 2]), ([0, 2 * m + 1, m, 3 * m], [300, 200, 100], []),
                                    ([m, 2 * m, 3 * m, 5 * m + 1], [300, 200, 100], [0, 1]), ([0, m, 2 * m, 3 * m], [300, -1, 321], [0]),
                                    ([-1, m - 1, m, 3 * m + 1], [300, 200, 100], [1])]:
        out, lse = torch.full_like(q, 7.0), torch.full((n, Hq), 7.0, device=cuda_device)
        hsa.hsa_kv8_attend(c.cache.ctx, q, 3, i32(starts), m, i32(lengths), True, None, None, out, lse)
        assert c.cache.device_status() == (0 if len(served) == 3 else hsa.HSA_ERR_DEVICE_BOUNDS)
        mine = torch.zeros(n, dtype=torch.bool, device=cuda_device)
        for s in served:
            mine[starts[s]:starts[s + 1]] = True
        assert (out[~mine] == 7.0).all() and (lse[~mine] == 7.0).all()
        assert (out[mine] != 7.0).any(-1).all() and (lse[mine] != 7.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hq,Hkv,counts", FEW)
def test_few_rows_are_independent(cuda_device, d, Hq, Hkv, counts):
    """A query that is not finite spoils its own row alone; pages outside the pools and entries outside the table are not seen;
    twice the same call, the same bits, in a graph too."""
    c = Case(cuda_device, Hq, Hkv, d, [400, 400, 9000], seed=34, max_tokens=10000)
    c.append([400, 400, 9000], twin=False)
    n = sum(counts)
    q, want, want_lse = c.attend(counts, True, check=False)
    bad = q.clone()
    bad[0, Hq - 1, 3], bad[n - 1, 0, 0] = float("nan"), float("inf")
    _, got, lse = c.attend(counts, True, q=bad, check=False)
    keep = torch.ones(n, Hq, dtype=torch.bool)
    keep[0, Hq - 1] = keep[n - 1, 0] = False
    assert torch.equal(got.cpu()[keep], want.cpu()[keep]) and torch.equal(lse.cpu()[keep], want_lse.cpu()[keep])
    assert got.cpu()[0, Hq - 1].isnan().all()
    qd, starts, lengths, out = q.to(cuda_device), dev_i32(np.concatenate([[0], np.cumsum(counts)]), cuda_device), dev_i32(c.held, cuda_device), torch.empty_like(want)
    call = lambda o, **kw: c.cache.attend(qd, lengths, token_start=starts, max_q=max(counts), out=o, **kw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and c.cache.device_status() == 0
    idx = torch.tensor([[[0, -1, 3, 141]], [[99999, 2, 1 << 30, 5]], [[7, 8, -5, 9]]], dtype=torch.int32, device=cuda_device).expand(3, Hkv, 4).contiguous()
    cnt = torch.full((3, Hkv), 4, dtype=torch.int32, device=cuda_device)
    call(out, sel_idx=idx, sel_cnt=cnt)
    assert c.cache.device_status() == hsa.HSA_ERR_DEVICE_BOUNDS
    good = torch.tensor([[[0, 3, 3]], [[2, 5, 5]], [[7, 8, 9]]], dtype=torch.int32, device=cuda_device).expand(3, Hkv, 3).contiguous()
    only = call(torch.empty_like(out), sel_idx=good, sel_cnt=torch.tensor([[2] * Hkv, [2] * Hkv, [3] * Hkv], dtype=torch.int32, device=cuda_device))
    # the same keys in other places of a step: fp32 sums in another order, a bf16 step apart at most
    assert torch.allclose(out.float(), only.float(), atol=2.0 ** -12, rtol=2.0 ** -7) and c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("d,n", [(128, 1), (128, 40), (64, 5)])
def test_pages_behind_four_gigabytes(cuda_device, d, n):
    """Pools of more than 2^32 bytes: pages at their far end give the bits that the same pages at the begin of small pools give."""
    H, tokens = 12, 700
    blocks, far = 11, (1 << 32) // (H * 64 * d) + 40
    g = torch.Generator(device=cuda_device).manual_seed(51)
    rand = lambda *s: torch.randn(*s, generator=g, device=cuda_device).to(torch.bfloat16)
    k, v, q = rand(tokens, H, d), rand(tokens, H, d), rand(n, H, d)
    rope = hsa.RotaryPositions(d, device=cuda_device)
    res = []
    for pages, table in ((blocks, torch.arange(blocks)), (far, far - 1 - torch.arange(blocks))):
        c = hsa.KV8Cache(H, H, d, pages, blocks, 1, tokens, device=cuda_device, key_sums=True,
                         page_table=table.to(torch.int32)[None].to(cuda_device))
        c.append(k[:300], v[:300], dev_i32([0], cuda_device), rope=rope)
        c.append(k[300:], v[300:], dev_i32([300], cuda_device), rope=rope)
        out, lse = c.attend(q, dev_i32([tokens], cuda_device), with_lse=True)
        assert c.device_status() == 0
        at = table.to(cuda_device)
        res.append([t.clone() for t in (c.k_codes.view(torch.uint8)[at], c.v_codes.view(torch.uint8)[at], c.k_scale[at], c.v_scale[at], c.ksum,
                                        out, lse)])
        c.destroy()
        del c
    assert all(torch.equal(x, y) for x, y in zip(*res))
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("counts", [[1, 1], [3, 1], [20, 100], [300, 260]])
def test_heads_before_tokens_and_in_place(cuda_device, d, counts):
    """Tensors that keep the tokens of a head together, results over the queries, and both."""
    c, twin = (Case(cuda_device, 4, 2, d, [5000, 700], seed=52, max_tokens=6000) for _ in range(2))
    k, v = c.append([5000, 700], twin=False)
    flip = lambda t: t.to(cuda_device).transpose(0, 1).contiguous().transpose(0, 1)
    held, starts = dev_i32([0, 0], cuda_device), dev_i32([0, 5000, 5700], cuda_device)
    twin.cache.append(flip(k), flip(v), held, token_start=starts, max_new=5000)
    pages = [p for _, _, p in c.written()]
    for name in ("k_codes", "v_codes"):
        a, b = (getattr(x.cache, name).view(torch.uint8)[pages] for x in (c, twin))
        assert torch.equal(a, b), name
    q, want, _ = c.attend(counts, True, check=False)
    lengths, starts = dev_i32(c.held, cuda_device), dev_i32(np.concatenate([[0], np.cumsum(counts)]), cuda_device)
    call = lambda x, out: c.cache.attend(x, lengths, token_start=starts, max_q=max(counts), out=out)
    x = flip(q)
    assert torch.equal(call(x, None), want) and torch.equal(call(x, torch.empty_like(x)), want)
    assert call(x, x) is x and torch.equal(x, want)
    y = q.to(cuda_device)
    assert torch.equal(call(y, y), want) and c.cache.device_status() == 0


@pytest.mark.gpu
@pytest.mark.parametrize("Hq,Hkv,d,n", [(4, 2, 128, 1), (2, 2, 64, 30)])
def test_captured_step_follows_the_lengths(cuda_device, Hq, Hkv, d, n):
    """Rotation, append and attention captured once; replays grow the sequences, whose lengths the graph itself counts up."""
    steps, start = 70 if n == 1 else 8, [100, 64, 1]
    room = [s + (steps + 2) * n for s in start]
    eager, other = (Case(cuda_device, Hq, Hkv, d, room, seed=53, sums=True, max_tokens=1000) for _ in range(2))
    g = torch.Generator().manual_seed(54)
    past = [torch.randn(sum(start), Hkv, d, generator=g).to(torch.bfloat16) for _ in range(2)]
    rope = hsa.RotaryPositions(d, device=cuda_device)
    for c in (eager, other):
        c.append(start, rope=rope, k=past[0], v=past[1], twin=False)
    new = [torch.randn(steps, 3 * n, h, d, generator=g).to(torch.bfloat16).to(cuda_device) for h in (Hkv, Hkv, Hq)]
    k, v, q = (torch.empty_like(t[0]) for t in new)
    out, held = torch.empty_like(q), dev_i32(start, cuda_device)
    pos = torch.empty(3 * n, dtype=torch.int32, device=cuda_device)
    row = torch.arange(n, dtype=torch.int32, device=cuda_device).repeat(3)

    def step(c, held):
        pos.copy_(held.repeat_interleave(n, output_size=3 * n) + row)
        c.cache.append(k, v, held, rope=rope, positions=pos)
        c.cache.attend(rope.apply(q, pos), held + n, out=out)
        held += n

    side = torch.cuda.Stream()
    graph, held_g = torch.cuda.CUDAGraph(), held.clone()
    for t, x in zip((k, v, q), new):
        t.copy_(x[0])
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(other, held_g)
    for i in range(steps):
        for t, x in zip((k, v, q), new):
            t.copy_(x[i])
        step(eager, held)
        want = out.clone()
        graph.replay()
        assert torch.equal(out, want), i
    assert held.tolist() == held_g.tolist() == [s + steps * n for s in start]
    assert eager.cache.device_status() == other.cache.device_status() == 0
    eager.held = held.tolist()
    pages = [p for _, _, p in eager.written()]
    for name in ("k_codes", "v_codes"):
        a, b = (getattr(x.cache, name).view(torch.uint8)[pages] for x in (eager, other))
        assert torch.equal(a, b), name
