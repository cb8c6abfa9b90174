"""Far addresses and many tokens in every kernel of windowed attention and of the 4-bit
cache, on the GPU: caches whose tokens lie past 2^32 bytes give the bits of dense ones; the
append of thousands of tokens, for every kind of rotary dims, against the float64 oracle
(as tests/test_gpu_fp4.py does); values by 64-bit indices, exact."""

import ctypes

import numpy as np
import pytest
import torch

import oracle.rotary as rope
import span_cases as S
from test_gpu_fp4 import append, f64, random_cache, same_codes, to_gpu

pytestmark = pytest.mark.gpu
KEYS, HKV = 140, 2                                             # cached tokens
STEP = (2 ** 32 // (KEYS - 1) // 256 + 1) * 256                # bytes between them: the last lies past 2^32


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def far(x, step):
    """x [1, KEYS, HKV, width] with `step` bytes between tokens."""
    e = x.element_size()
    space = torch.empty(step * KEYS, dtype=torch.uint8, device="cuda").view(x.dtype)
    return torch.as_strided(space, x.shape, (0, step // e, x.shape[3], 1)).copy_(x)


def caches(form, d):
    """The same keys and values dense and far, [1, KEYS, HKV, width] each.  4 bits: scales
    at a sixteenth of the codes' strides, and at the codes' own."""
    g = torch.Generator().manual_seed(d)
    if form == "fp4":
        dense = [to_gpu(x) for x in random_cache((1, KEYS, HKV), d, g, head_inner=True)]
    else:
        dense = [torch.randn((1, KEYS, HKV, d), generator=g).to(torch.float32 if form == "f32" else torch.bfloat16).cuda() for _ in range(2)]
    kinds = [(STEP, STEP, STEP // 16, STEP // 16), (STEP,) * 4] if form == "fp4" else [(STEP,) * 2]
    return dense, [[far(x, step) for x, step in zip(dense, steps)] for steps in kinds]


def placed(cache, paged, n):
    """A cache of n sequences that are all the one given, and its block table: a page a
    token, or contiguous."""
    if paged:
        return [x.transpose(0, 1) for x in cache], torch.arange(KEYS, dtype=torch.int32, device="cuda").repeat(n, 1)
    return [x.expand(n, -1, -1, -1) for x in cache], None


def equal(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("form,d", [("bf16", 128), ("bf16", 64), ("fp4", 128), ("fp4", 64), ("f32", 128), ("f32", 64)])
def test_chunks_past_32_bits(form, d, paged):
    from paper_2606_02544_amd import binding
    dense, fars = caches(form, d)
    for tokens in S.TOKENS:
        q = torch.randn((tokens, 16, d), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(torch.float32 if form == "f32" else torch.bfloat16)
        for window, sinks in ((60, 3),) + (((0, 0),) if form == "fp4" else ()):
            def run(cache):
                held, table = placed(cache, paged, 2)
                kw = dict(max_q_len=70, max_kv_len=KEYS, page_size=int(paged), window=window, sinks=sinks,
                          out=torch.zeros_like(q), lse=torch.zeros((16, tokens), device="cuda"))
                rest = (table, i32(0, 70, 71), i32(KEYS, KEYS - 9))
                if form == "fp4":
                    return binding.chunk_attention_fp4(q, binding.Fp4Cache(*held), *rest, **kw)
                return binding.chunk_attention(q, *held, *rest, **kw)

            want = run(dense)
            assert bool(want[0][:71].any(-1).all())
            assert all(equal(run(x), want) for x in fars), (tokens, window)


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("form,d", [("bf16", 128), ("bf16", 64), ("fp4", 128), ("fp4", 64)])
def test_verifications_past_32_bits(form, d, paged):
    from paper_2606_02544_amd import binding
    dense, fars = caches(form, d)
    B, L, hq = 8, 8, 32
    for n in S.COPIES:
        g = torch.Generator(device="cuda").manual_seed(n)
        q, k, v = (torch.randn((n, B + L, h, d), generator=g, device="cuda").bfloat16() for h in (hq, HKV, HKV))
        steps = torch.arange(1, B + 1, dtype=torch.int32, device="cuda").repeat(n, 1)
        lens, refs = torch.full((n,), KEYS, dtype=torch.int32, device="cuda"), torch.full((n,), L, dtype=torch.int32, device="cuda")
        for window, sinks in ((60, 3),) + (((0, 0),) if form == "fp4" else ()):
            def run(cache):
                held, table = placed(cache, paged, n)
                kw = dict(block_size=B, max_ref=L, max_prefix_len=KEYS, page_size=int(paged), window=window, sinks=sinks)
                if form == "fp4":
                    return binding.verify_attention_fp4(q, k, v, binding.Fp4Cache(*held), table, lens, steps, refs, **kw)
                return binding.verify_attention(q, k, v, *held, table, lens, steps, refs, **kw)

            want = run(dense)
            assert bool(want[0].any(-1).all())
            assert all(equal(run(x), want) for x in fars), (n, window)


@pytest.mark.parametrize("d,rot,interleaved", [(64, 64, True), (64, 36, False), (64, 6, True), (128, 128, False)])
@pytest.mark.parametrize("page", [0, 24])
def test_append_of_many_tokens(d, rot, interleaved, page):
    """Four tokens a work-group, the last one's not all there; a ragged batch with tokens of
    no sequence at either end."""
    from paper_2606_02544_amd import binding
    first, lens, kv = 5, [4000, 1, 0, 4195], [4100, 1, 7, 4195]
    T, hq, hkv, cap = first + sum(lens) + 6, 2, 1, 4195
    g = torch.Generator().manual_seed(rot)
    x = torch.randn((T, hq + 2 * hkv, d), generator=g).bfloat16()
    q, k, v = x.cuda().split([hq, hkv, hkv], 1)
    starts = torch.tensor([first] + list(np.cumsum(lens) + first), dtype=torch.int32)
    per = -(-cap // page) if page else 0
    n = (len(lens) * per + 1, page) if page else (len(lens), cap)
    table = torch.randperm(len(lens) * per, generator=g).view(len(lens), per).to(torch.int32) if page else None
    where = (table.cuda() if page else None, starts.cuda(), i32(*kv))
    freq, _ = binding.rope_frequencies(rot, 10000.0)
    cache = binding.fp4_cache(*n, hkv, d)
    for t in cache:
        t.fill_(77)
    out, want = (torch.full((T, hq, d), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    append(q, k, v, cache, *where, freq, cap, page, interleaved=interleaved, attn_factor=1.25, q_out=out)
    bf = [torch.zeros((*n, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    binding.rotary_append(q, k, v, *bf, *where, freq, max_kv_len=cap, page_size=page, interleaved=interleaved, attn_factor=1.25, q_out=want)
    assert torch.equal(out, want)                              # queries: the bits that the bf16 append gives
    rows = rope.cache_rows(starts.tolist(), kv, T)
    live = [t for t in range(T) if rows[t][0] >= 0 and rows[t][1] >= 0]
    assert len(live) == sum(lens)
    at = [((int(table[b, i // page]), i % page) if page else (b, i)) for b, i in (rows[t] for t in live)]
    seq, tok = map(np.array, zip(*at))
    c = [t.cpu().numpy() for t in cache]
    turned = rope.rotate(f64(k)[live], np.array([rows[t][1] for t in live]), freq.cpu().numpy(), interleaved=interleaved, factor=1.25)
    same_codes(c[0][seq, tok], c[2][seq, tok], turned, True)
    same_codes(c[1][seq, tok], c[3][seq, tok], f64(v)[live], False)
    for a in c:
        a[seq, tok] = 77
        assert (a == 77).all(), "rows of no token were written"


def test_values_by_64_bit_indices():
    """2^27 heads and more of 128 (34 GB of keys): one sequence's, many times over."""
    from paper_2606_02544_amd import binding
    n, tokens, hkv, d = 2 ** 13 + 1, 2048, 8, 128
    g = torch.Generator().manual_seed(4)
    one = binding.Fp4Cache(*map(to_gpu, random_cache((1, tokens, hkv), d, g)))
    want = binding.fp4_values(one)[0]
    desc = binding.Fp4ValuesDesc(n, tokens, hkv, d, 0, one.k.stride(1), one.k.stride(2))
    pointers = binding.Fp4Pointers(*[x.data_ptr() for x in one], 0, one.k_scales.stride(1), one.k_scales.stride(2))
    out = torch.empty((n, tokens, hkv, d), dtype=torch.bfloat16, device="cuda")
    status = binding.lib().simsd_fp4_values(ctypes.byref(desc), ctypes.byref(pointers), out.data_ptr(), None,
                                            torch.cuda.current_stream().cuda_stream)
    assert status == 0
    for part in out.split(512):
        assert torch.equal(part, want.expand(part.shape[0], -1, -1, -1))
