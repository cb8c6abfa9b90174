"""Performance cases of the operators around the verification step, through the
Python binding: rotary positions with the write into the cache, attention of a
chunk of new tokens over that cache, and sampling.

A serving program makes these calls beside the verification: a prompt (or the
tokens of an accepted block) is rotated and appended to the cache, its queries
attend over the cache under the block-causal mask of a block-diffusion model,
and the drafter draws its tokens from filtered logits.  Head counts, head sizes,
vocabulary, pages and lengths are those of the workloads in ``synth/configs.py``
and generic ones between them.

Ops:
  rotary  queries and keys turned at given positions (the new slots of a step)
  append  queries turned, keys turned and written with the values to the cache
  attend  attention of a ragged chunk over the cache, block-causal
  sample  a token for each row of logits, with temperature, top-k, top-p, min-p
"""

from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
VOCAB = 151936
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # The new slots of one batch-1 verification step at their RoPE-copy
        # positions: the smallest call, host time and one launch.
        {"name": "rotary-step", "op": "rotary", "dtype": "bf16", "tokens": 8, "hq": 16, "hkv": 8, "d": 128,
         "rot": 128, "interleaved": False, "fused": False, "far": 1024, "factor": 1.0},
        # A decode round's tokens with half of each head turned, interleaved
        # pairs, far positions, FP32.
        {"name": "rotary-part-f32", "op": "rotary", "dtype": "f32", "tokens": 1021, "hq": 32, "hkv": 8, "d": 128,
         "rot": 64, "interleaved": True, "fused": False, "far": 1000000, "factor": 1.0},
        # Chunks of a ragged batch into a paged cache, from a fused projection's
        # output, positions scaled for long contexts.
        {"name": "append-ragged-paged", "op": "append", "dtype": "bf16", "batch": 24, "q_lo": 1, "q_hi": 351,
         "lo": 101, "hi": 6007, "pad": 5, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "fused": True, "factor": 4.0, "page": 16},
        # Long prompts of a batch, written to a contiguous cache.
        {"name": "append-long-prompts", "op": "append", "dtype": "bf16", "batch": 8, "q_lo": 4096, "q_hi": 4096,
         "lo": 0, "hi": 0, "pad": 0, "hq": 32, "hkv": 8, "d": 128, "rot": 128, "interleaved": False,
         "fused": True, "factor": 1.0, "page": 0},
        # One block of a small model at batch 1 without drafts: few rows against
        # a prefix, where latency counts.
        {"name": "attend-block", "op": "attend", "dtype": "bf16", "batch": 1, "q_lo": 4, "q_hi": 4, "lo": 1024,
         "hi": 1024, "pad": 0, "hq": 16, "hkv": 8, "d": 128, "mask_block": 4, "page": 0},
        # Single tokens of a full serving batch with uneven lengths, paged.
        {"name": "attend-single-tokens", "op": "attend", "dtype": "bf16", "batch": 64, "q_lo": 1, "q_hi": 1,
         "lo": 512, "hi": 32767, "pad": 0, "hq": 32, "hkv": 8, "d": 128, "mask_block": 1, "page": 16},
        # Chunks and single tokens mixed in one batch, paged, blocks of 8.
        {"name": "attend-mixed-paged", "op": "attend", "dtype": "bf16", "batch": 24, "q_lo": 1, "q_hi": 351,
         "lo": 101, "hi": 6007, "pad": 5, "hq": 32, "hkv": 8, "d": 128, "mask_block": 8, "page": 64},
        # The prompt of one request in FP32, the paper's own precision.
        {"name": "attend-prompt-f32", "op": "attend", "dtype": "f32", "batch": 1, "q_lo": 1000, "q_hi": 1000,
         "lo": 24, "hi": 24, "pad": 0, "hq": 32, "hkv": 8, "d": 128, "mask_block": 8, "page": 0},
        # The last chunks of long prompts: the largest products.
        {"name": "attend-long-chunks", "op": "attend", "dtype": "bf16", "batch": 4, "q_lo": 2048, "q_hi": 2048,
         "lo": 14336, "hi": 14336, "pad": 0, "hq": 32, "hkv": 8, "d": 128, "mask_block": 32, "page": 16},
        # Drafted tokens of a batch-1 block.
        {"name": "sample-block", "op": "sample", "dtype": "bf16", "rows": 4, "vocab": VOCAB, "params": "one",
         "temperature": 1.0, "top_k": 50, "top_p": 0.95, "min_p": 0.0, "banned": 0.0},
        # A tokenizer whose size is no multiple of a vector load, FP32 logits,
        # nothing filtered but the far tail.
        {"name": "sample-odd-vocab-f32", "op": "sample", "dtype": "f32", "rows": 61, "vocab": 50001,
         "params": "one", "temperature": 0.8, "top_k": 0, "top_p": 1.0, "min_p": 0.02, "banned": 0.0},
        # Every slot of a large batch of long blocks, requests with their own
        # settings.
        {"name": "sample-mixed-rows", "op": "sample", "dtype": "bf16", "rows": 512, "vocab": VOCAB,
         "params": "rows", "temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, "banned": 0.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choices(["rotary", "append", "attend", "attend_f32", "sample"], [2, 3, 5, 2, 4])[0]
    while True:
        hkv = rng.choice([1, 2, 4, 8, 8])
        c = {"op": op.split("_")[0], "dtype": "f32" if op == "attend_f32" else rng.choice(["bf16", "bf16", "f32"])}
        if op == "sample":
            c["rows"] = _log_int(rng, 1, 512)
            c["vocab"] = VOCAB if rng.random() < 0.4 else _log_int(rng, 1000, VOCAB)
            c["params"] = rng.choice(["one", "rows"])
            c["temperature"] = rng.choice([0.0, 0.6, 1.0, 1.0, 1.3])
            c["top_k"] = rng.choice([0, 1, 20, 50, 1000])
            c["top_p"] = rng.choice([1.0, 0.5, 0.9, 0.95])
            c["min_p"] = rng.choice([0.0, 0.0, 0.05])
            c["banned"] = rng.choice([0.0, 0.0, 0.9])
        elif op in ("rotary", "append"):
            c["hq"], c["hkv"], c["d"] = hkv * rng.choice([1, 2, 4, 4]), hkv, rng.choice([64, 128, 128])
            c["rot"] = rng.choice([c["d"], c["d"], c["d"] // 2])
            c["interleaved"], c["fused"] = rng.random() < 0.3, rng.random() < 0.6
            c["factor"] = rng.choice([1.0, 1.0, 4.0, 16.0])
            if op == "rotary":
                c["tokens"], c["far"] = _log_int(rng, 1, 32768), _log_int(rng, 64, 1000000)
            else:
                c["batch"], c["q_hi"] = _log_int(rng, 1, 64), _log_int(rng, 1, 4096)
                c["q_lo"], c["hi"] = rng.choice([1, c["q_hi"]]), _log_int(rng, 1, 16384)
                c["lo"] = rng.choice([0, c["hi"]])
                c["pad"], c["page"] = rng.choice([0, 0, 3]), rng.choice([0, 16, 16, 64])
        else:
            c["hq"], c["hkv"], c["d"] = hkv * rng.choice([1, 2, 4, 4, 8]), hkv, rng.choice([64, 128, 128, 128])
            c["batch"], c["q_hi"] = _log_int(rng, 1, 64), _log_int(rng, 1, 4096)
            if rng.random() < 0.25:
                c["q_hi"] = 1
            c["q_lo"], c["hi"] = rng.choice([1, c["q_hi"]]), _log_int(rng, 1, 32000)
            c["lo"] = rng.choice([0, c["hi"]])
            c["mask_block"], c["pad"] = rng.choice([0, 1, 1, 4, 8, 32]), rng.choice([0, 0, 3])
            c["page"] = rng.choice([0, 16, 16, 64])
        w = work(c)
        # No dearer than the largest listed case of the operator, in the plain
        # form too: its padded scores and keys stay in the range of theirs.
        if c["op"] == "attend":
            kv = c["hi"] + c["q_hi"]
            padded = c["batch"] * c["hq"] * c["q_hi"] * kv
            f32 = c["dtype"] == "f32"
            fits = (w["bytes"] < (1e9 if f32 else 4.5e9) and w["flops"] < (6e10 if f32 else 2e12)
                    and padded < 4e9 and c["batch"] * kv * c["hkv"] * c["d"] < 2e9)
        elif c["op"] == "sample":
            fits = c["rows"] * c["vocab"] <= (8e6 if c["dtype"] == "f32" else 7.8e7)
        else:
            fits = w["bytes"] < 8e8 and c.get("batch", 1) * (c.get("hi", 0) + c.get("q_hi", 0)) < 1.5e5
        if fits:
            return c


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _spread(lo, hi, n):
    """n lengths spread evenly over [lo, hi], the mean of both for one."""
    if n == 1:
        return torch.tensor([(lo + hi + 1) // 2])
    return torch.linspace(lo, hi, n, dtype=torch.float64).round().long()


def _lens(c, cpu):
    """Chunk and cached lengths of the sequences, each in an order of its own."""
    b = c["batch"]
    q = _spread(c["q_lo"], c["q_hi"], b)[torch.randperm(b, generator=cpu)]
    kv = _spread(c["lo"], c["hi"], b)[torch.randperm(b, generator=cpu)] + q
    return q, kv


def _cache(c, kv, cpu):
    """Shape of the cache, and the block table of a paged one (pages in a random
    order out of a pool that holds any pairing of the lengths; unused entries
    point to a spare page)."""
    most, page = c["hi"] + c["q_hi"], c["page"]
    if not page:
        return (c["batch"], most, c["hkv"], c["d"]), None
    per = -(-kv // page)
    pool = sum(int((-(-_spread(c[lo], c[hi], c["batch"]) // page)).sum()) for lo, hi in (("lo", "hi"), ("q_lo", "q_hi")))
    used = torch.arange(-(-most // page)) < per[:, None]
    table = torch.full(used.shape, pool)
    table[used] = torch.randperm(pool, generator=cpu)[:int(per.sum())]
    return (pool + 1, page, c["hkv"], c["d"]), table.to(torch.int32).to(DEV)


def _frequencies(c):
    """Angle a position of each pair [rot/2] in 64 bits; scaled (factor > 1): the
    pairs that turn less than once in the original context are slowed down by
    the factor, those that turn 32 times or more are left, and those between
    are blended; and the factor on the rotated values."""
    half = c["rot"] // 2
    f = 1000000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
    if c["factor"] == 1.0:
        return f.to(DEV), 1.0
    turns = f * 8192 / (2 * math.pi)
    keep = ((turns - 1) / 31).clamp(0, 1)
    return (f * keep + f / c["factor"] * (1 - keep)).to(DEV), 0.1 * math.log(c["factor"]) + 1.0


def _heads(c, tokens, gpu):
    """q, k, v [tokens, heads, d]: parts of one projection's output, or alone."""
    dt, d, hq, hkv = DTYPES[c["dtype"]], c["d"], c["hq"], c["hkv"]
    new = lambda *shape: torch.randn(shape, generator=gpu, device=DEV, dtype=dt)  # noqa: E731
    if c["fused"]:
        return new(tokens, hq + 2 * hkv, d).split([hq, hkv, hkv], 1)
    return new(tokens, hq, d), new(tokens, hkv, d), new(tokens, hkv, d)


def prepare(case, seed):
    c = dict(case)
    gpu = torch.Generator(device=DEV).manual_seed(seed)
    cpu = torch.Generator().manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] == "sample":
        n, V = c["rows"], c["vocab"]
        x = torch.randn((n, V), generator=gpu, device=DEV).mul_(2.0)
        # Six rows of ten have a clear favourite among the flat rest, with a few
        # close seconds, as a model's rows have.
        at = torch.randint(0, V, (n, 4), generator=gpu, device=DEV)
        raised = 12.5 - 1.5 * torch.arange(4, device=DEV, dtype=torch.float32)
        sure = (torch.rand(n, generator=cpu) < 0.6).to(DEV)
        x.scatter_(1, at, torch.where(sure[:, None], raised, x.gather(1, at)))
        if c["banned"]:
            x.masked_fill_(torch.rand((n, V), generator=gpu, device=DEV) < c["banned"], -math.inf)
        s["logits"] = x.to(dt)
        s["uniforms"] = torch.rand(n, generator=cpu).to(DEV)
        if c["params"] == "rows":
            pick = lambda *v: torch.tensor(v)[torch.randint(0, len(v), (n,), generator=cpu)].to(DEV)  # noqa: E731
            s["temperature"], s["top_p"] = pick(0.0, 0.7, 1.0, 1.0, 1.3), pick(1.0, 1.0, 0.8, 0.95)
            s["top_k"], s["min_p"] = pick(0, 0, 20, 50, 1000).to(torch.int32), pick(0.0, 0.0, 0.05)
        else:
            s.update({p: c[p] for p in ("temperature", "top_k", "top_p", "min_p")})
        return s
    if c["op"] == "rotary":
        s["q"], s["k"], _ = _heads(c, c["tokens"], gpu)
        s["positions"] = torch.randint(0, c["far"], (c["tokens"],), generator=cpu, dtype=torch.int32).to(DEV)
        s["freq"], s["attn_factor"] = _frequencies(c)
        return s
    q_len, kv = _lens(c, cpu)
    tokens = int(q_len.sum()) + c["pad"]               # `pad` rows behind the last sequence
    starts = torch.cat([torch.zeros(1, dtype=torch.long), q_len.cumsum(0)])
    shape, s["block_table"] = _cache(c, kv, cpu)
    s["q_starts"], s["kv_lens"] = starts.to(torch.int32).to(DEV), kv.to(torch.int32).to(DEV)
    s["tokens"], s["used"], s["max_q"], s["max_kv"] = tokens, int(q_len.sum()), c["q_hi"], c["hi"] + c["q_hi"]
    if c["op"] == "append":
        s["q"], s["k"], s["v"] = _heads(c, tokens, gpu)
        s["freq"], s["attn_factor"] = _frequencies(c)
        s["k_cache"] = torch.zeros(shape, device=DEV, dtype=dt)
        s["v_cache"] = torch.zeros(shape, device=DEV, dtype=dt)
    else:
        s["q"] = torch.randn((tokens, c["hq"], c["d"]), generator=gpu, device=DEV, dtype=dt)
        s["k_cache"] = torch.randn(shape, generator=gpu, device=DEV, dtype=dt)
        s["v_cache"] = torch.randn(shape, generator=gpu, device=DEV, dtype=dt)
        s["lse"] = torch.zeros((c["hq"], tokens), device=DEV)
    s["out"] = torch.zeros((tokens, c["hq"], c["d"]), device=DEV, dtype=dt)
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _turn(c, s, x, pos):
    """x [tokens, heads, d] turned by pos [tokens], in 32 bits (angles in 64)."""
    angle = pos.double()[:, None] * s["freq"]
    cos, sin = (angle.cos() * s["attn_factor"]).float()[:, None], (angle.sin() * s["attn_factor"]).float()[:, None]
    part, rest = x[..., :c["rot"]].float(), x[..., c["rot"]:]
    if c["interleaved"]:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = part[..., :c["rot"] // 2], part[..., c["rot"] // 2:]
        part = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([part.to(x.dtype), rest], -1)


def _token_rows(s):
    """Sequence of each token, its place in the chunk and in the cache."""
    starts = s["q_starts"].long()
    token = torch.arange(s["used"], device=DEV)
    seq = torch.searchsorted(starts, token, right=True) - 1
    place = token - starts[seq]
    return seq, place, s["kv_lens"].long()[seq] - (starts[seq + 1] - starts[seq]) + place


def _plain_append(c, s):
    n = s["used"]
    seq, _, at = _token_rows(s)
    s["out"][:n] = _turn(c, s, s["q"][:n], at)
    k = _turn(c, s, s["k"][:n], at)
    first = s["block_table"].long()[seq, at // c["page"]] if c["page"] else seq
    second = at % c["page"] if c["page"] else at
    s["k_cache"][first, second] = k
    s["v_cache"][first, second] = s["v"][:n]
    return s["out"], s["k_cache"], s["v_cache"]


def _plain_attend(c, s):
    b, hq, hkv, d, nq, nk = c["batch"], c["hq"], c["hkv"], c["d"], s["max_q"], s["max_kv"]
    g, n, starts, kv = hq // hkv, s["used"], s["q_starts"].long(), s["kv_lens"].long()
    seq, place, _ = _token_rows(s)
    # Queries and keys padded to one length a sequence.
    slot = torch.arange(nq, device=DEV)
    q_len = starts[1:] - starts[:-1]
    rows = (starts[:-1, None] + slot).clamp(max=s["tokens"] - 1)
    q = s["q"][rows].float().view(b, nq, hkv, g, d).permute(0, 2, 3, 1, 4).reshape(b, hkv, g * nq, d)
    key = torch.arange(nk, device=DEV)
    held = key < kv[:, None]
    if c["page"]:
        page = s["block_table"].long()[:, key // c["page"]]
        k, v = (s[t][page, key % c["page"]] for t in ("k_cache", "v_cache"))
    else:
        k, v = s["k_cache"][:, :nk], s["v_cache"][:, :nk]
    k = k.permute(0, 2, 3, 1).float().contiguous()
    v = v.permute(0, 2, 1, 3).float().masked_fill_(~held[:, None, :, None], 0.0)
    x = torch.matmul(q, k).mul_(1.0 / math.sqrt(d)).view(b, hq, nq, nk)
    pos = (kv - q_len)[:, None] + slot
    m = c["mask_block"]
    sees = torch.minimum((pos // m + 1) * m, kv[:, None]) if m else kv[:, None].expand(b, nq)
    x.masked_fill_((key >= sees[..., None])[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(b, hkv, g * nq, nk), v).view(b, hq, nq, d).div_(total)
    s["out"][:n] = o[seq, :, place].to(s["out"].dtype)
    s["lse"][:, :n] = (top + total.log())[seq, :, place, 0].t()
    return s["out"], s["lse"]


def _plain_sample(s):
    logits = s["logits"]
    n, V = logits.shape
    row = lambda p: torch.as_tensor(s[p], device=DEV).expand(n)[:, None]  # noqa: E731
    number = lambda p: row(p).float().double()  # noqa: E731  the parameters are 32-bit numbers
    T, top_p, min_p, k = number("temperature"), number("top_p"), number("min_p"), row("top_k").long()
    # Falling logits, the lowest index first among equal ones; weights in 64
    # bits, since the running sums decide the token.
    x, order = torch.sort(logits.float(), dim=1, descending=True, stable=True)
    x = x.double()
    gap = x - x[:, :1]
    greedy = T <= 0
    w = (gap / torch.where(greedy, 1.0, T)).exp()
    w = w * torch.where(greedy, gap == 0, gap >= -700.0 * T)
    rank = torch.arange(V, device=DEV)
    k = torch.where(greedy, 1, torch.where((k <= 0) | (k > V), V, k))
    w = w * (rank < k)
    run_sum = w.cumsum(1)
    enough = top_p * run_sum[:, -1:]
    w = w * ((top_p >= 1) | (rank == 0) | (run_sum - w < enough))
    w = w * (w >= min_p.clamp(max=1.0))
    run_sum = w.cumsum(1)
    at = (run_sum <= s["uniforms"].double()[:, None] * run_sum[:, -1:]).sum(1, keepdim=True)
    token = order.gather(1, at)[:, 0].to(torch.int32)
    return token, (w.gather(1, at) / run_sum[:, -1:])[:, 0].float(), (w > 0).sum(1).to(torch.int32)


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2606_02544_amd import binding
        if c["op"] == "sample":
            return binding.sample(s["logits"], s["uniforms"], temperature=s["temperature"], top_k=s["top_k"],
                                  top_p=s["top_p"], min_p=s["min_p"])
        if c["op"] == "attend":
            return binding.chunk_attention(
                s["q"], s["k_cache"], s["v_cache"], s["block_table"], s["q_starts"], s["kv_lens"],
                max_q_len=s["max_q"], max_kv_len=s["max_kv"], page_size=c["page"], mask_block=c["mask_block"],
                out=s["out"], lse=s["lse"])
        if c["op"] == "append":
            q = binding.rotary_append(
                s["q"], s["k"], s["v"], s["k_cache"], s["v_cache"], s["block_table"], s["q_starts"], s["kv_lens"],
                s["freq"], max_kv_len=s["max_kv"], page_size=c["page"], interleaved=c["interleaved"],
                attn_factor=s["attn_factor"], q_out=s["out"])
            return q, s["k_cache"], s["v_cache"]
        return binding.rotary(s["q"], s["k"], s["positions"], s["freq"], interleaved=c["interleaved"],
                              attn_factor=s["attn_factor"])
    if c["op"] == "sample":
        return _plain_sample(s)
    if c["op"] == "attend":
        return _plain_attend(c, s)
    if c["op"] == "append":
        return _plain_append(c, s)
    return _turn(c, s, s["q"], s["positions"]), _turn(c, s, s["k"], s["positions"])


# ---------------------------------------------------------------------------
# What a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "sample":
        n = c["rows"] * c["vocab"]
        return {"bytes": n * e + c["rows"] * 32, "flops": 4 * n}
    if c["op"] == "rotary":
        n = c["tokens"] * (c["hq"] + c["hkv"])
        return {"bytes": 2 * n * c["d"] * e + 4 * c["tokens"] + 4 * c["rot"], "flops": 3 * n * c["rot"]}
    q = _spread(c["q_lo"], c["q_hi"], c["batch"])
    tokens = int(q.sum())
    if c["op"] == "append":
        heads = c["hq"] + 2 * c["hkv"]
        return {"bytes": 2 * tokens * heads * c["d"] * e + 12 * c["batch"] + 4 * c["rot"],
                "flops": 3 * tokens * (c["hq"] + c["hkv"]) * c["rot"]}
    before = _spread(c["lo"], c["hi"], c["batch"])
    keys = int(before.sum()) + tokens
    # Visible pairs: the keys before the chunk (their mean length: lengths and
    # chunks are paired at random), and half of the chunk with itself.
    m = c["mask_block"]
    inside = float((q.double() ** 2).sum()) if not m else float((q.double() * (q.double() + min(m, int(q.max())))).sum()) / 2
    pairs = tokens * float(before.double().mean()) + inside
    moved = 2 * keys * c["hkv"] * c["d"] * e + tokens * c["hq"] * (2 * c["d"] * e + 4)
    return {"bytes": moved, "flops": 4 * c["hq"] * c["d"] * pairs}


# ---------------------------------------------------------------------------
# The same results in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c = s["case"]

    def rotated(x, pos):
        """As complex numbers times e^(i angle)."""
        turn = torch.polar(torch.full((), s["attn_factor"], dtype=torch.float64, device=DEV),
                           pos.double()[:, None] * s["freq"])[:, None]
        y = x.double()
        half = c["rot"] // 2
        pair = (y[..., :c["rot"]].unflatten(-1, (half, 2)) if c["interleaved"]
                else y[..., :c["rot"]].unflatten(-1, (2, half)).transpose(-1, -2))
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        y[..., :c["rot"]] = (z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        return y

    if c["op"] == "rotary":
        return rotated(s["q"], s["positions"]), rotated(s["k"], s["positions"])
    if c["op"] == "sample":
        tokens, probs, kept = [], [], []
        for i in range(c["rows"]):
            value = lambda p: float(s[p][i]) if isinstance(s[p], torch.Tensor) else float(torch.tensor(s[p]).float())  # noqa: E731
            T, k, top_p, min_p = (value(p) for p in ("temperature", "top_k", "top_p", "min_p"))
            x = s["logits"][i].double()
            best = x.max()
            if T <= 0:
                tokens.append(int((x == best).nonzero()[0, 0]))
                probs.append(1.0)
                kept.append(1)
                continue
            idx = torch.argsort(-x, stable=True)[:int(k) if 0 < k < c["vocab"] else c["vocab"]]
            y = x[idx] - best
            idx, y = idx[y >= -700 * T], y[y >= -700 * T]
            p = (y / T).exp()
            if top_p < 1:
                idx, p = (t[:1 + int((p.cumsum(0) < top_p * p.sum()).sum())] for t in (idx, p))
            many = max(1, int((p >= min(min_p, 1.0)).sum()))
            idx, p = idx[:many], p[:many]
            n = int(torch.searchsorted(p.cumsum(0), s["uniforms"][i].double() * p.cumsum(0)[-1], right=True))
            tokens.append(int(idx[n]))
            probs.append(float(p[n] / p.cumsum(0)[-1]))
            kept.append(len(idx))
        return (torch.tensor(tokens, dtype=torch.int32), torch.tensor(probs, dtype=torch.float64),
                torch.tensor(kept, dtype=torch.int32))

    starts, lens = s["q_starts"].tolist(), s["kv_lens"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    if c["op"] == "append":
        caches = [torch.zeros(s["k_cache"].shape, dtype=torch.float64, device=DEV) for _ in range(2)]
    else:
        lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    for i in range(c["batch"]):
        a, b = starts[i], starts[i + 1]
        n = lens[i]
        pos = torch.arange(n - (b - a), n, device=DEV)
        pages = s["block_table"][i].long() if c["page"] else None
        if c["op"] == "append":
            out[a:b] = rotated(s["q"][a:b], pos)
            new = (rotated(s["k"][a:b], pos), s["v"][a:b].double())
            for cache, x in zip(caches, new):
                if c["page"]:
                    cache.view(-1, c["hkv"], c["d"])[pages[pos // c["page"]] * c["page"] + pos % c["page"]] = x
                else:
                    cache[i, pos] = x
            continue
        if c["page"]:
            k, v = (s[t][pages[:-(-n // c["page"])]].reshape(-1, c["hkv"], c["d"])[:n] for t in ("k_cache", "v_cache"))
        else:
            k, v = s["k_cache"][i, :n], s["v_cache"][i, :n]
        g, m = c["hq"] // c["hkv"], c["mask_block"]
        blind = torch.arange(n, device=DEV) // m > (pos // m)[:, None] if m else None
        for h in range(c["hkv"]):
            kh, vh = k[:, h].double().t().contiguous(), v[:, h].double()
            for j in range(h * g, h * g + g):
                x = s["q"][a:b, j].double() @ kh / math.sqrt(c["d"])
                if m:
                    x.masked_fill_(blind, -math.inf)
                z = torch.logsumexp(x, 1)
                lse[j, a:b] = z
                out[a:b, j] = x.sub_(z[:, None]).exp_() @ vh
    return (out, *caches) if c["op"] == "append" else (out, lse)
