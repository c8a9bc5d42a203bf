"""The history in 8 bits: rotary positions, the append that applies them, and attention over the cache.

Three operators that follow one another in a layer whose history is held in 8 bits:

    rope     x -> rotated x.  Pair p of a row turns by position * frequency[p]; the transposed rotation is
             the operator's gradient.
    append   new keys and values -> pages of the cache.  Keys are rotated on the way; a page of 64 tokens
             of one head holds e4m3 codes and one scale, a power of two; the sum of a page's keys is kept
             for block selection where the caller asks for it.
    attend   queries, cache -> softmax attention of each query over the tokens its sequence holds, over all
             blocks or those of a list per head; causal or not; one token per sequence or many.

`run` computes them in plain torch operations, or, where `own` is set, through the framework's calls.
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 64
E4M3_TOP = 448.0
FRAME, COLS = 1560, 52   # tokens of a latent frame and of a row of it (832 x 480 video)
BASE = 10000.0
BANDS = (32.0, 1.0)      # turns over the trained length above which a pair keeps its frequency, below which it is stretched
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def listed():
    return [
        # one token of a rollout far into a sequence: launch and latency
        dict(name="rope_token", op="rope", tokens=1, H=12, d=128, rot=128, layout="half", axes=1, dtype="bf16", pos=1000003,
             factor=1.0, transpose=False),
        # the queries of a video chunk: frame, row and column each turn their share of the pairs
        dict(name="rope_chunk", op="rope", tokens=4680, H=12, d=128, rot=128, layout="interleaved", axes=3, dtype="bf16",
             pos=4680, factor=1.0, transpose=False),
        # the gradient of a part of the head, in 32 bits, of a context stretched eight times
        dict(name="rope_grad", op="rope", tokens=20011, H=8, d=128, rot=96, layout="half", axes=1, dtype="fp32", pos=131072,
             factor=8.0, transpose=True),
        # a token of each of 48 sequences
        dict(name="append_step", op="append", batch=48, new_lo=1, new_hi=1, held_lo=300, held_hi=8000, H=8, d=128, rot=128,
             layout="half", axes=1, sums=False),
        # a video chunk behind nine others, with the key sums that block selection reads; it starts inside a page
        dict(name="append_chunk", op="append", batch=1, new_lo=4680, new_hi=4680, held_lo=42120, held_hi=42120, H=12, d=128,
             rot=128, layout="interleaved", axes=3, sums=True),
        # ragged prompts, heads of 64, no positions
        dict(name="append_prompts", op="append", batch=16, new_lo=500, new_hi=8000, held_lo=0, held_hi=700, H=16, d=64, rot=0,
             layout="half", axes=1, sums=False),
        # one token, a short history
        dict(name="attend_short", op="attend", batch=1, q_lo=1, q_hi=1, keys_lo=777, keys_hi=777, Hq=12, Hkv=12, d=128,
             causal=True, topk=0),
        # a token of each of 48 sequences, four query heads to a key head
        dict(name="attend_batch", op="attend", batch=48, q_lo=1, q_hi=1, keys_lo=300, keys_hi=8000, Hq=32, Hkv=8, d=128,
             causal=True, topk=0),
        # a token against the history of a long video
        dict(name="attend_long", op="attend", batch=1, q_lo=1, q_hi=1, keys_lo=280800, keys_hi=280800, Hq=12, Hkv=12, d=128,
             causal=True, topk=0),
        # a video chunk against all of its history
        dict(name="attend_chunk", op="attend", batch=1, q_lo=4680, q_hi=4680, keys_lo=46800, keys_hi=46800, Hq=12, Hkv=12,
             d=128, causal=False, topk=0),
        # the same against the 64 blocks that each head selected
        dict(name="attend_selected", op="attend", batch=1, q_lo=4680, q_hi=4680, keys_lo=46800, keys_hi=46800, Hq=12, Hkv=12,
             d=128, causal=False, topk=64),
        # ragged prompts, some continuing a history, heads of 64
        dict(name="attend_prompts", op="attend", batch=6, q_lo=129, q_hi=2500, keys_lo=400, keys_hi=4100, Hq=16, Hkv=4, d=64,
             causal=True, topk=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, one token to tens of thousands, one sequence to 64, both head sizes."""
    top = max(_cost(c) for c in listed())
    while True:
        d = rng.choice([64, 128, 128])
        op = rng.choice(["rope", "append", "append", "attend", "attend", "attend"])
        if op == "rope":
            axes = rng.choice([1, 1, 3])
            c = dict(op=op, tokens=_log_int(rng, 1, 24000), H=rng.choice([1, 3, 8, 12, 16, 32]), d=d,
                     rot=rng.choice([d, d, d - 16, d // 2, 2 * rng.randint(3, d // 2)]), layout=rng.choice(["half", "interleaved"]),
                     axes=axes, dtype=rng.choice(["bf16", "bf16", "fp16", "fp32"]), factor=rng.choice([1.0, 1.0, 4.0, 10.0]),
                     transpose=rng.random() < 0.4)
            c["pos"] = c["tokens"] + _log_int(rng, 1, 4000000)
        elif op == "append":
            batch = _log_int(rng, 1, 64)
            lo = _log_int(rng, 1, max(1, 6000 // batch))
            held = rng.choice([0, _log_int(rng, 1, 40000 // batch)])
            c = dict(op=op, batch=batch, new_lo=lo, new_hi=rng.choice([lo, 2 * lo + 1]), held_lo=held, held_hi=2 * held,
                     H=rng.choice([1, 2, 8, 12, 16]), d=d, rot=rng.choice([0, d, d, d // 2, d - 2]),
                     layout=rng.choice(["half", "interleaved"]), axes=rng.choice([1, 1, 3]), sums=rng.random() < 0.5)
        else:
            batch = rng.choice([1, 1, _log_int(rng, 2, 64)])
            Hkv = rng.choice([1, 2, 4, 8, 12])
            keys = _log_int(rng, 1, 280000 // batch)
            q = min(keys, rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 10, 4680)]))
            c = dict(op=op, batch=batch, q_lo=max(1, q // 2), q_hi=q, keys_lo=max(q, keys // 3), keys_hi=max(q, keys),
                     Hq=Hkv * rng.choice([1, 1, 2, 4, 5, 8]), Hkv=Hkv, d=d, causal=rng.random() < 0.6, topk=0)
            if rng.random() < 0.3:
                c["topk"] = _log_int(rng, 1, 128)
        if _cost(c) <= top and _memory(c) <= 24e9:
            return c


# ------------------------------------------------------------------ sizes
def _spread(lo, hi, n, shift=0):
    """n sizes between lo and hi, evenly spread over their logarithm in a mixed order."""
    lo1, hi1 = lo + 1, hi + 1
    return [int(round(lo1 * (hi1 / lo1) ** (((i + shift) * 0.618034 + 0.5) % 1.0))) - 1 for i in range(n)]


def _sequences(case):
    """(new tokens or queries, tokens in the cache with them) of every sequence."""
    n = case["batch"]
    if case["op"] == "append":
        new = _spread(case["new_lo"], case["new_hi"], n)
        held = _spread(case["held_lo"], case["held_hi"], n, 3)
        return new, [a + b for a, b in zip(new, held)]
    q = _spread(case["q_lo"], case["q_hi"], n)
    return q, [max(a, b) for a, b in zip(q, _spread(case["keys_lo"], case["keys_hi"], n, 3))]


def _blocks(tokens):
    return (tokens + BLOCK - 1) // BLOCK


def _memory(case):
    """Bytes the plain form's largest intermediate takes."""
    if case["op"] != "attend":
        return 0
    q, keys = _sequences(case)
    top = min(case["topk"] or 1 << 30, _blocks(max(keys))) * BLOCK
    return 4.0 * case["batch"] * max(case["Hq"] * max(q), 2 * case["Hkv"] * case["d"]) * top


def _pairs(rot, axes):
    """Pairs of each axis."""
    n = rot // 2
    if axes == 1:
        return [n]
    rest = n // 3
    return [n - 2 * rest, rest, rest]


def work(case):
    """Bytes (every input once, every output once) and operations of one pass."""
    if case["op"] == "rope":
        size = {"bf16": 2, "fp16": 2, "fp32": 4}[case["dtype"]]
        n = case["tokens"] * case["H"]
        return {"bytes": 2 * n * case["d"] * size + 4 * case["tokens"] * case["axes"], "flops": 3 * n * case["rot"]}
    new, keys = _sequences(case)
    if case["op"] == "append":
        row = case["H"] * case["d"]
        b = sum(new) * row * 6
        # a page that tokens stand in already: its scale may grow, which its codes then follow
        b += sum(8 * case["H"] * (_blocks(k) - (k - n) // BLOCK) for n, k in zip(new, keys))
        if case["sums"]:
            b += sum(4 * row * (_blocks(k) - (k - n) // BLOCK) for n, k in zip(new, keys))
        return {"bytes": b, "flops": 3 * sum(new) * case["H"] * (case["rot"] + case["d"])}
    rows = case["Hq"] * case["d"]
    b, f = 0, 0
    for n, k in zip(new, keys):
        seen = k
        if case["topk"]:
            seen = min(k, case["topk"] * BLOCK)
        b += seen * case["Hkv"] * case["d"] * 2 + n * rows * 4
        pairs = n * seen
        if case["causal"]:
            pairs = (n * k - n * (n - 1) // 2) * (seen / k)
        f += 4 * pairs * rows
    return {"bytes": int(b), "flops": int(f)}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 250)


# ------------------------------------------------------------------ state
def _frequencies(rot, axes, factor, trained):
    """Radians per position of each pair, in 64 bits, and what the rotated values are multiplied by."""
    out = []
    for n in _pairs(rot, axes):
        f = BASE ** (-torch.arange(n, dtype=torch.float64) / n)
        if factor != 1.0:
            fast, slow = BANDS
            keep = ((trained * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1)
            f = f * (keep + (1 - keep) / factor)
        out.append(f)
    return torch.cat(out), 1.0 if factor == 1.0 else 0.1 * math.log(factor) + 1.0


def _positions(first, count, axes, dev):
    t = torch.arange(first, first + count, device=dev, dtype=torch.int64)
    if axes == 1:
        return t[None].to(torch.int32)
    return torch.stack([t // FRAME, t % FRAME // COLS, t % COLS]).to(torch.int32)


def _quantise(x):
    """e4m3 codes and power-of-two scales of [..., 64, d] pages."""
    top = x.abs().amax(dim=(-1, -2)).clamp(min=2.0 ** -40)
    m, e = torch.frexp(top)                      # top = m 2^e, 0.5 <= m < 1; 448 = 0.875 2^9
    e = e - 9 + (m > 0.875).to(e.dtype)
    scale = torch.ldexp(torch.ones_like(top), e)
    return (x / scale[..., None, None]).to(torch.float8_e4m3fn), scale


def _rope_handle(case):
    from paper_2609_34606_b200 import hsa
    factor = case.get("factor", 1.0)
    return hsa.RotaryPositions(case["d"], rot_dim=case["rot"], layout=case["layout"], base=BASE,
                               axis_pairs=_pairs(case["rot"], case["axes"]), scaling="bands" if factor != 1.0 else "none",
                               factor=factor, trained_tokens=4096, device="cuda")


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    rand = lambda *shape: torch.randn(*shape, generator=g, device=dev)
    s = {"case": dict(case)}
    if case["op"] == "rope":
        dtype = TYPES[case["dtype"]]
        s["x"] = rand(case["tokens"], case["H"], case["d"]).to(dtype)
        s["out"] = torch.empty_like(s["x"])
        s["pos"] = _positions(case["pos"] - case["tokens"], case["tokens"], case["axes"], dev)
        if own:
            s["rope"] = _rope_handle(case)
        else:
            f, s["amplitude"] = _frequencies(case["rot"], case["axes"], case["factor"], 4096)
            s["freq"] = f.to(dev)
        return s
    d, batch = case["d"], case["batch"]
    new, keys = _sequences(case)
    n_blocks = [_blocks(k) for k in keys]
    per_seq, used = max(n_blocks), sum(n_blocks)
    pages = used + 3                             # a few that nobody holds
    order = torch.randperm(pages, generator=g, device=dev)[:used].to(torch.int32)
    table = torch.zeros(batch, per_seq, dtype=torch.int32, device=dev)
    n_blk = torch.tensor(n_blocks, device=dev)
    table[torch.arange(per_seq, device=dev)[None] < n_blk[:, None]] = order
    s["table"] = table
    s["starts"] = torch.tensor([0] + new, device=dev).cumsum(0).to(torch.int32)
    s["total"], s["max_new"] = sum(new), max(new)
    Hkv = case["H"] if case["op"] == "append" else case["Hkv"]
    # the history: what stands in a page before the first append is never read
    k, v = rand(pages, Hkv, BLOCK, d), rand(pages, Hkv, BLOCK, d)
    s["k_codes"], s["k_scale"] = _quantise(k)
    s["v_codes"], s["v_scale"] = _quantise(v)
    del k, v
    if case["op"] == "append":
        s["k"], s["v"] = (rand(s["total"], Hkv, d).to(torch.bfloat16) for _ in range(2))
        s["held"] = torch.tensor([b - a for a, b in zip(new, keys)], dtype=torch.int32, device=dev)
        s["sums"] = torch.zeros(batch, Hkv, per_seq, d, device=dev) if case["sums"] else None
        if case["rot"]:
            s["pos"] = torch.cat([_positions(b - a, a, case["axes"], dev) for a, b in zip(new, keys)], 1)
            if own:
                s["rope"] = _rope_handle(case)
            else:
                s["freq"] = _frequencies(case["rot"], case["axes"], 1.0, 0)[0].to(dev)
    else:
        s["q"] = rand(s["total"], case["Hq"], d).to(torch.bfloat16)
        s["lengths"] = torch.tensor(keys, dtype=torch.int32, device=dev)
        if case["topk"]:
            # distinct blocks of every head's own choice, ascending, as the selection leaves them
            score = torch.rand(batch, Hkv, per_seq, generator=g, device=dev)
            score = score.masked_fill(torch.arange(per_seq, device=dev) >= n_blk[:, None, None], -1.0)
            n = min(case["topk"], per_seq)
            idx = score.topk(n, dim=-1).indices.sort(dim=-1).values
            cnt = n_blk[:, None].clamp(max=n).expand(batch, Hkv)
            # (sequences with fewer blocks than the list is long: theirs come first)
            s["sel_idx"], s["sel_cnt"] = idx.to(torch.int32).contiguous(), cnt.to(torch.int32).contiguous()
    if own:
        from paper_2609_34606_b200 import hsa
        s["cache"] = hsa.KV8Cache(case.get("Hq", Hkv), Hkv, d, max_pages=pages, max_blocks=per_seq, max_batch=batch,
                                  max_tokens=s["total"], device=dev, page_table=table, k_codes=s["k_codes"],
                                  v_codes=s["v_codes"], k_scale=s["k_scale"], v_scale=s["v_scale"], key_sums=s.get("sums"))
        s["out"] = torch.empty_like(s["q"]) if "q" in s else None
    return s


# ------------------------------------------------------------------ the plain forms
def _rotate(x, pos, freq, case, sign=1.0, amplitude=1.0):
    """[tokens, H, d] in 32 bits; angles in 64 (positions reach millions), sines and cosines rounded once."""
    rot, half = case["rot"], case["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(case["axes"], device=x.device),
                                   torch.tensor(_pairs(rot, case["axes"]), device=x.device), output_size=half)
    angle = pos.to(torch.float64)[axis].T * freq             # [tokens, pairs]
    cos = (angle.cos() * amplitude).float()[:, None]
    sin = (angle.sin() * (sign * amplitude)).float()[:, None]
    x = x.float()
    if case["layout"] == "half":
        a, b = x[..., :half], x[..., half:rot]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(s):
    case, dev = s["case"], s["k"].device
    n, Hkv, d, batch = s["total"], case["H"], case["d"], case["batch"]
    k, v = s["k"].float(), s["v"].float()
    if case["rot"]:
        k = _rotate(s["k"], s["pos"], s["freq"], case)
    starts, held = s["starts"].long(), s["held"].long()
    t = torch.arange(n, device=dev)
    b = torch.searchsorted(starts[1:], t, right=True)
    at = held[b] + t - starts[b]                             # place in the sequence
    first = held // BLOCK                                    # first page that is written, of each sequence
    last = (held + (starts[1:] - starts[:-1]) - 1) // BLOCK
    per = int(s["max_new"] + 2 * BLOCK - 2) // BLOCK         # pages of a sequence that a call can reach
    blk = first[:, None] + torch.arange(per, device=dev)
    live = blk <= last[:, None]
    page = s["table"].long().gather(1, blk.clamp(max=s["table"].shape[1] - 1))
    pos = blk[..., None] * BLOCK + torch.arange(BLOCK, device=dev)
    older = (pos < held[:, None, None])[:, :, None, :, None]  # rows that earlier calls wrote
    touched = ((first * BLOCK < held)[:, None] & (torch.arange(per, device=dev) == 0))[:, :, None]
    sums = None
    for x, codes, scale, is_k in ((k, s["k_codes"], s["k_scale"], True), (v, s["v_codes"], s["v_scale"], False)):
        new = torch.zeros(batch * per * BLOCK, Hkv, d, device=dev)
        new[(b * per + at // BLOCK - first[b]) * BLOCK + at % BLOCK] = x
        new = new.view(batch, per, BLOCK, Hkv, d).transpose(2, 3)      # [batch, pages, Hkv, 64, d]
        old_scale = scale[page]
        old = torch.where(older, codes[page].float() * old_scale[..., None, None], 0.0)
        top = new.abs().amax(dim=(-1, -2)).clamp(min=2.0 ** -40)
        m, e = torch.frexp(top)
        grown = torch.ldexp(torch.ones_like(top), e - 9 + (m > 0.875).to(e.dtype))
        grown = torch.where(touched, torch.maximum(grown, old_scale), grown)
        c = ((new + old) / grown[..., None, None]).to(torch.float8_e4m3fn)
        # rows behind a page's last token: zeros where the page is new, as they were where it is not
        written = (pos >= held[:, None, None]) & (pos < (held + starts[1:] - starts[:-1])[:, None, None])
        keep = ~(written[:, :, None] | older[..., 0]) & touched[..., None]
        rest = (codes[page].float() * old_scale[..., None, None] / grown[..., None, None]).to(torch.float8_e4m3fn)
        c = torch.where(keep[..., None], rest.view(torch.uint8), c.view(torch.uint8)).view(torch.float8_e4m3fn)
        codes.view(torch.uint8)[page[live]] = c.view(torch.uint8)[live]
        scale[page[live]] = grown[live]
        if is_k and s["sums"] is not None:
            stored = torch.where(older, c.float() * grown[..., None, None], 0.0)
            sums = (stored + new).sum(3)
    if sums is not None:
        where = torch.arange(batch, device=dev)[:, None].expand(batch, per)
        s["sums"].transpose(1, 2)[where[live], blk[live]] = sums[live]


def _plain_attend(s):
    case, q, dev = s["case"], s["q"], s["q"].device
    batch, Hq, Hkv, d = case["batch"], case["Hq"], case["Hkv"], case["d"]
    group = Hq // Hkv
    starts, lengths, table = s["starts"].long(), s["lengths"].long(), s["table"].long()
    n_q = starts[1:] - starts[:-1]
    i = torch.arange(s["max_new"], device=dev)
    row = (starts[:-1, None] + i).clamp(max=s["total"] - 1)             # [batch, max_q]
    real = i < n_q[:, None]
    if case["topk"]:
        blk = s["sel_idx"].long()                                       # [batch, Hkv, n]
        live = torch.arange(blk.shape[-1], device=dev) < s["sel_cnt"][..., None]
    else:
        blk = torch.arange(table.shape[1], device=dev).expand(batch, 1, -1)
        live = torch.ones_like(blk, dtype=torch.bool)
    n = blk.shape[-1]
    page = table[torch.arange(batch, device=dev)[:, None, None], blk]
    head = torch.arange(Hkv, device=dev)[:, None]
    k = (s["k_codes"][page, head].float() * s["k_scale"][page, head][..., None, None]).flatten(2, 3)   # [batch, Hkv, keys, d]
    v = (s["v_codes"][page, head].float() * s["v_scale"][page, head][..., None, None]).flatten(2, 3)
    at = (blk[..., None] * BLOCK + torch.arange(BLOCK, device=dev)).flatten(2)                          # [batch, Hkv or 1, keys]
    seen = (at < lengths[:, None, None]) & live.repeat_interleave(BLOCK, -1)
    qs = q[row].float().view(batch, -1, Hkv, group, d).permute(0, 2, 3, 1, 4)                           # [batch, Hkv, group, max_q, d]
    scores = torch.matmul(qs.flatten(2, 3), k.transpose(-1, -2)).view(batch, Hkv, group, -1, n * BLOCK)
    scores *= d ** -0.5
    seen = seen[:, :, None, None]
    if case["causal"]:
        mine = (lengths - n_q)[:, None] + i
        seen = seen & (at[:, :, None, None] <= mine[:, None, None, :, None])
    scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    scores -= top
    scores.exp_()
    total = scores.sum(-1, keepdim=True)
    out = torch.matmul(scores.flatten(2, 3), v).view(batch, Hkv, group, -1, d)
    out = torch.where(total > 0, out / total, 0.0)
    lse = torch.where(total > 0, top + total.log(), -math.inf)
    out = out.permute(0, 3, 1, 2, 4).reshape(batch, -1, Hq, d)[real]
    return {"out": out.to(q.dtype), "lse": lse.permute(0, 3, 1, 2, 4).reshape(batch, -1, Hq)[real]}


def run(s):
    case = s["case"]
    if case["op"] == "rope":
        if own:
            return s["rope"].apply(s["x"], s["pos"], transpose=case["transpose"], out=s["out"])
        y = _rotate(s["x"], s["pos"], s["freq"], case, -1.0 if case["transpose"] else 1.0, s["amplitude"])
        return y.to(s["x"].dtype)
    if case["op"] == "append":
        if own:
            s["cache"].append(s["k"], s["v"], s["held"], token_start=s["starts"], max_new=s["max_new"],
                              rope=s.get("rope"), positions=s.get("pos"))
        else:
            _plain_append(s)
        res = {"k_codes": s["k_codes"], "k_scale": s["k_scale"], "v_codes": s["v_codes"], "v_scale": s["v_scale"]}
        if s["sums"] is not None:
            res["sums"] = s["sums"]
        return res
    if own:
        out, lse = s["cache"].attend(s["q"], s["lengths"], token_start=s["starts"], max_q=s["max_new"], causal=case["causal"],
                                     sel_idx=s.get("sel_idx"), sel_cnt=s.get("sel_cnt"), out=s["out"], with_lse=True)
        return {"out": out, "lse": lse}
    return _plain_attend(s)


# ------------------------------------------------------------------ from the definitions, in 64 bits
def _e4m3(x):
    """The nearest e4m3 value (ties to the even one) of values up to 448, in 64 bits."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -30)))
    e = torch.where(x.abs() < torch.exp2(e), e - 1, e)
    e = torch.where(x.abs() >= torch.exp2(e + 1), e + 1, e).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _turn64(x, pos, case, transpose=False):
    """Each pair as a complex number times exp(i angle)."""
    f, amplitude = _frequencies(case["rot"], case["axes"], case.get("factor", 1.0), 4096)
    rot, half, n, at = case["rot"], case["rot"] // 2, _pairs(case["rot"], case["axes"]), 0
    angle = torch.empty(x.shape[0], half, dtype=torch.float64, device=x.device)
    for axis, count in enumerate(n):
        angle[:, at:at + count] = pos[axis].double()[:, None] * f[at:at + count].to(x.device)
        at += count
    z = x.double()
    if case["layout"] == "half":
        pairs = torch.complex(z[..., :half], z[..., half:rot])
    else:
        pairs = torch.view_as_complex(z[..., :rot].reshape(*z.shape[:-1], half, 2).contiguous())
    w = torch.polar(torch.full_like(angle, amplitude), -angle if transpose else angle)
    y = torch.view_as_real(pairs * w[:, None])
    out = z.clone()
    out[..., :rot] = torch.cat([y[..., 0], y[..., 1]], -1) if case["layout"] == "half" else y.flatten(-2)
    return out


def _append64(s, case):
    new, keys = _sequences(case)
    k = _turn64(s["k"], s["pos"], case) if case["rot"] else s["k"].double()
    res = {"k_codes": s["k_codes"].double(), "k_scale": s["k_scale"].double(), "v_codes": s["v_codes"].double(),
           "v_scale": s["v_scale"].double()}
    if s["sums"] is not None:
        res["sums"] = s["sums"].double()
    table, first = s["table"].tolist(), 0
    for b, (n, end) in enumerate(zip(new, keys)):
        held = end - n
        for blk in range(held // BLOCK, _blocks(end)):
            lo, hi = max(held, blk * BLOCK), min(end, (blk + 1) * BLOCK)
            r0, r1, page = lo - blk * BLOCK, hi - blk * BLOCK, table[b][blk]
            for name, x in (("k", k), ("v", s["v"].double())):
                codes, scale = res[name + "_codes"][page], res[name + "_scale"][page]     # [H, 64, d], [H]
                rows = x[first + lo - held:first + hi - held].transpose(0, 1)
                top = rows.abs().amax((1, 2)).clamp(min=2.0 ** -40)
                fit = torch.exp2(torch.ceil(torch.log2(top / E4M3_TOP)))
                if r0:
                    fit = torch.maximum(fit, scale)
                    codes.copy_(_e4m3(codes * (scale / fit)[:, None, None]))
                else:
                    codes.zero_()
                codes[:, r0:r1] = _e4m3(rows / fit[:, None, None])
                scale.copy_(fit)
                if name == "k" and "sums" in res:
                    res["sums"][b, :, blk] = rows.sum(1) + (codes[:, :r0] * fit[:, None, None]).sum(1)
        first += n
    return res


def _attend64(s, case):
    new, keys = _sequences(case)
    group, d = case["Hq"] // case["Hkv"], case["d"]
    out = torch.zeros(s["total"], case["Hq"], d, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((s["total"], case["Hq"]), -math.inf, dtype=torch.float64, device=s["q"].device)
    first = 0
    for b, (n, length) in enumerate(zip(new, keys)):
        for h in range(case["Hkv"]):
            blocks = torch.arange(_blocks(length), device=out.device)
            if case["topk"]:
                blocks = s["sel_idx"][b, h, :int(s["sel_cnt"][b, h])].long()
            page = s["table"][b].long()[blocks]
            k = (s["k_codes"][page, h].double() * s["k_scale"][page, h].double()[:, None, None]).reshape(-1, d)
            v = (s["v_codes"][page, h].double() * s["v_scale"][page, h].double()[:, None, None]).reshape(-1, d)
            at = (blocks[:, None] * BLOCK + torch.arange(BLOCK, device=out.device)).reshape(-1)
            for r in range(h * group, (h + 1) * group):
                x = s["q"][first:first + n, r].double() @ k.T / math.sqrt(d)
                hidden = (at >= length).expand(n, -1)
                if case["causal"]:
                    hidden = hidden | (at > length - n + torch.arange(n, device=out.device)[:, None])
                x.masked_fill_(hidden, -math.inf)
                lse[first:first + n, r] = total = torch.logsumexp(x, 1)
                out[first:first + n, r] = torch.where(total[:, None] > -math.inf, (x - total[:, None]).exp_(), 0.0) @ v
        first += n
    return {"out": out, "lse": lse}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _turn64(s["x"], s["pos"], case, case["transpose"])
    if case["op"] == "append":
        return _append64(s, case)
    return _attend64(s, case)
