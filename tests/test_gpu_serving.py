"""Rotary positions, chunk attention, sampling and the verification step run together,
as a serving program does: prompts prefilled in chunks into a paged cache, a block
drafted by sampling, verified over that cache, and the accepted block appended."""

import numpy as np
import pytest
import torch

import oracle.chunk
import oracle.rotary

pytestmark = pytest.mark.gpu
THETA, B, HQ, HKV, D, PAGE, V = 10000.0, 8, 8, 2, 64, 16, 5000
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Layer:
    """One attention layer's projections of a ragged batch, as random numbers, and its
    paged cache."""

    def __init__(self, dtype, lens, seed):
        self.dt, self.lens = DT[dtype], lens
        self.g = torch.Generator().manual_seed(seed)
        per = 16
        self.table = torch.randperm(len(lens) * per, generator=self.g).view(len(lens), per).to(torch.int32).cuda()
        self.k_cache = torch.full((len(lens) * per, PAGE, HKV, D), float("nan"), dtype=self.dt, device="cuda")
        self.v_cache = self.k_cache.clone()
        self.cap = per * PAGE
        # every token's query, key and value, by sequence
        self.qkv = [torch.randn((n + 3 * B, HQ + 2 * HKV, D), generator=self.g).to(self.dt) for n in lens]
        self.have = [0] * len(lens)

    def step(self, new, freq, mask_block=B, **kw):
        """Appends the next `new` tokens of each sequence and attends over the cache."""
        from paper_2606_02544_amd import binding
        rows = torch.cat([x[h:h + n] for x, h, n in zip(self.qkv, self.have, new)]).cuda()
        q, k, v = rows.split([HQ, HKV, HKV], 1)
        self.have = [h + n for h, n in zip(self.have, new)]
        starts, kv = i32([0] + list(np.cumsum(new))), i32(self.have)
        q = binding.rotary_append(q, k, v, self.k_cache, self.v_cache, self.table, starts, kv, freq,
                                  max_kv_len=self.cap, page_size=PAGE)
        return binding.chunk_attention(q, self.k_cache, self.v_cache, self.table, starts, kv, max_q_len=max(new),
                                       max_kv_len=self.cap, page_size=PAGE, mask_block=mask_block, **kw)

    def want(self, b, first, last, mask_block=B):
        """The oracle's attention of tokens [first, last) of sequence b, all of whose
        blocks' keys are cached."""
        freq, _ = oracle.rotary.frequencies(D, THETA)
        x = self.qkv[b][:last].double().numpy()
        pos = np.arange(last)
        q = oracle.rotary.rotate(x[:, :HQ], pos, freq)[first:]
        k = oracle.rotary.rotate(x[:, HQ:HQ + HKV], pos, freq)
        return oracle.chunk.chunk_attention(q, k[None], x[None, :, HQ + HKV:], None, [0, last - first], [last],
                                            mask_block=mask_block)


def near(got, want, lse, wl, dtype):
    # bf16: rotated queries and keys are rounded (2^-8 of each, so a score by 2^-7 of
    # its size), weights and the output once more: as the parity tests bound it, 2e-2 of
    # the row's largest; fp32: 1e-5 and, for the log-sum-exp, 1e-4 of its size.
    g = got.double().cpu().numpy()
    if dtype == "bf16":
        assert (np.abs(g - want).max(-1) <= 2e-2 * np.abs(want).max(-1)).all()
    else:
        assert np.abs(g - want).max() <= 1e-5
        assert np.abs(lse.double().cpu().numpy() - wl).max() <= 1e-4 * max(1.0, np.abs(wl).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_prompts_drafts_and_verification(dtype):
    from paper_2606_02544_amd import binding
    lens = [40, 8, 136]                                        # whole blocks of prompt
    layer = Layer(dtype, lens, 1)
    freq, _ = binding.rope_frequencies(D, THETA)
    # The prompts in two chunks, cut at block borders; a sequence that has none left
    # takes part with no rows.
    for new in ([24, 8, 64], [16, 0, 72]):
        before = list(layer.have)
        out, lse = layer.step(new, freq)
        at = 0
        for b, n in enumerate(new):
            if n:
                want, wl, _, _ = layer.want(b, before[b], before[b] + n)
                near(out[at:at + n], want, lse[:, at:at + n], wl, dtype)
            at += n
    # The drafter's block: logits of each slot, one token each.
    b = len(lens)
    logits = (2.0 * torch.randn((b, B, V), generator=layer.g)).to(layer.dt).cuda()
    u = torch.rand(b * B, generator=layer.g).cuda()
    token, prob, kept = binding.sample(logits.view(b * B, V), u, temperature=0.8)
    assert bool((kept == V).all())
    # Verified with the target's logits: the drafter's own make every draft pass, and
    # its probabilities are those it was drawn with.
    step = torch.stack([torch.randperm(B, generator=layer.g) + 1 for _ in lens]).to(torch.int32)
    order = step.argsort(1)
    drafts = torch.gather(token.view(b, B).cpu(), 1, order)
    rows = torch.gather(logits.cpu(), 1, order[:, :, None].expand(b, B, V)).cuda()
    p_target, p_draft, accepted, correction = binding.verify_accept_sampled(
        logits, rows, drafts.to(torch.int32).cuda(), step.cuda(), i32([B] * b),
        torch.rand((b, B + 1), generator=layer.g).cuda(), temperature=0.8)
    assert accepted.tolist() == [B] * b and correction.tolist() == [-1] * b
    torch.testing.assert_close(p_draft, torch.gather(prob.view(b, B), 1, order.cuda()), rtol=1e-4, atol=0)
    # The target's attention of the block over the cache filled above, its own rotary
    # embedding fused, against the same block appended and attended to as a chunk: with
    # no drafts the block's slots see each other and the prefix.
    new = torch.stack([x[n:n + B] for x, n in zip(layer.qkv, lens)]).cuda()
    q, k, v = (t.contiguous() for t in new.split([HQ, HKV, HKV], 2))
    out, lse = binding.verify_attention(
        q, k, v, layer.k_cache, layer.v_cache, layer.table, i32(lens), torch.ones((b, B), dtype=torch.int32, device="cuda"),
        i32([0] * b), block_size=B, max_ref=0, max_prefix_len=layer.cap, page_size=PAGE, rope_theta=THETA)
    chunk, chunk_lse = layer.step([B] * b, freq)
    for i, n in enumerate(lens):
        want, wl, _, _ = layer.want(i, n, n + B)
        near(out[i], want, lse[i], wl, dtype)
        near(chunk[i * B:(i + 1) * B], want, chunk_lse[:, i * B:(i + 1) * B], wl, dtype)
    # Single tokens after it, causal.
    out, lse = layer.step([1] * b, freq, mask_block=1, kv_chunk=64)
    for i, n in enumerate(lens):
        want, wl, _, _ = layer.want(i, n + B, n + B + 1, 1)
        near(out[i:i + 1], want, lse[:, i:i + 1], wl, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_captured_and_replayed(dtype):
    """Append, attention (ranges joined) and sampling of a decode step in one graph,
    replayed while the cache grows, eager calls on other data between the replays."""
    from paper_2606_02544_amd import binding
    b, cap = 3, 300
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda *s: torch.randn(s, generator=g, device="cuda").to(DT[dtype])  # noqa: E731
    rows = new(b, HQ + 2 * HKV, D)
    caches = [new(b, cap, HKV, D), new(b, cap, HKV, D)]
    logits, u = new(b, V), torch.rand(b, generator=g, device="cuda")
    starts, kv = i32([0, 1, 2, 3]), i32([200, 1, 64])
    freq, _ = binding.rope_frequencies(D, THETA)

    def step(kc, vc):
        q, k, v = rows.split([HQ, HKV, HKV], 1)
        q = binding.rotary_append(q, k, v, kc, vc, None, starts, kv, freq, max_kv_len=cap)
        out, lse = binding.chunk_attention(q, kc, vc, None, starts, kv, max_q_len=1, max_kv_len=cap, kv_chunk=64)
        return (out, lse, *binding.sample(logits, u, temperature=0.9, top_k=40, top_p=0.9))

    other = [c.clone() for c in caches]
    step(*other)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*caches)
    for _ in range(4):
        mine = [c.clone() for c in caches]
        want = step(*mine)
        graph.replay()
        step(*other)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip((*got, *caches), (*want, *mine)))
        kv += 1
        rows.copy_(new(b, HQ + 2 * HKV, D))
        logits.copy_(new(b, V))
        u.copy_(torch.rand(b, generator=g, device="cuda"))
