"""Rotary positions and the write into the cache on the GPU, against the float64
oracle.

Tolerance: the result's own rounding is off by half a step at most,
finfo.eps / 2 of its value.  Before it, in fp32: the reduced angle as a float of
at most half a turn is off by pi * 2^-24, sine and cosine by 2 * 2^-24, their
product with the factor, the two products and the sum by 2^-24 each of a term at
most: 10 * 2^-24 of factor * (|x1| + |x2|) holds it all; the fp64 angle adds
three roundings of |position * freq| <= |position|."""

import numpy as np
import pytest
import torch

import oracle.rotary as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def bound(x, want, freq, pos, interleaved, factor, dt):
    half = len(freq)
    pair = np.zeros(x.shape)
    for i in range(half):
        i1, i2 = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        s = np.abs(x[..., i1]) + np.abs(x[..., i2])
        pair[..., i1] = pair[..., i2] = s
    angle = np.abs(np.asarray(pos, np.float64))[:, None, None] * 3 * 2.0 ** -53
    return torch.finfo(dt).eps / 2 * np.abs(want) + factor * pair * (10 * 2.0 ** -24 + angle) * 1.01


def check(got, x, pos, freq, interleaved, factor):
    x64 = x.double().cpu().numpy()
    want = ref.rotate(x64, pos, freq, interleaved=interleaved, factor=factor)
    err = np.abs(got.double().cpu().numpy() - want)
    # (rows from rotary_dim on are copies: their bound is the copy's own rounding, 0 here)
    rot = 2 * len(freq)
    assert np.array_equal(got.cpu()[..., rot:].float().numpy(), x.cpu()[..., rot:].float().numpy())
    tol = bound(x64, want, freq, pos, interleaved, factor, got.dtype)
    assert (err <= tol)[..., :rot].all(), (err - tol).max()


def make(tokens, heads, d, dt, gen, fused=False):
    x = torch.randn((tokens, sum(heads), d), generator=gen).to(dt).cuda()
    parts = x.split(heads, 1)
    return parts if fused else [p.contiguous() for p in parts]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,hq,hkv,d,rot", [
    (1, 1, 1, 64, 64), (8, 16, 8, 128, 128), (33, 5, 1, 128, 64), (7, 4, 2, 128, 6), (3, 2, 2, 8, 2),
    (5, 3, 3, 72, 40), (2, 1, 1, 512, 512), (8200, 2, 1, 64, 32), (8195, 1, 1, 64, 6)])
def test_rotary(dtype, interleaved, tokens, hq, hkv, d, rot):
    from paper_2606_02544_amd import binding
    gen = torch.Generator().manual_seed(tokens * 7 + rot)
    q, k = make(tokens, [hq, hkv], d, DT[dtype], gen, fused=True)
    pos = torch.randint(-5, 100000, (tokens,), generator=gen, dtype=torch.int32)
    freq, factor = binding.rope_frequencies(rot, 10000.0)
    qo, ko = binding.rotary(q, k, pos.cuda(), freq, interleaved=interleaved, attn_factor=1.25)
    for got, x in ((qo, q), (ko, k)):
        check(got, x, pos.numpy(), freq.cpu().numpy(), interleaved, 1.25)
    only, none = binding.rotary(None, k, pos.cuda(), freq, interleaved=interleaved, attn_factor=1.25)[::-1]
    assert none is None and torch.equal(only, ko)


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_far_positions_and_scaled_frequencies(scaling):
    from paper_2606_02544_amd import binding
    kw = dict(scaling=scaling, factor=8.0, original_context=4096)
    freq, factor = binding.rope_frequencies(128, 500000.0, **kw)
    want, extra = ref.frequencies(128, 500000.0, **kw)
    np.testing.assert_allclose(freq.cpu().numpy(), want, rtol=1e-14)
    assert factor == np.float32(extra)
    gen = torch.Generator().manual_seed(3)
    (q,) = make(9, [4], 128, torch.float32, gen)
    pos = torch.tensor([0, 1, 4095, 4096, 131071, 10 ** 6 + 1, 2 ** 24 + 1, 2 ** 30 + 7, 2 ** 31 - 1], dtype=torch.int32)
    out, _ = binding.rotary(q, None, pos.cuda(), freq, attn_factor=factor)
    check(out, q, pos.numpy(), freq.cpu().numpy(), False, factor)


@pytest.mark.parametrize("dtype,interleaved,rot", [("bf16", False, 128), ("bf16", True, 64), ("f32", False, 10)])
def test_in_place_and_heads_outermost(dtype, interleaved, rot):
    from paper_2606_02544_amd import binding
    gen = torch.Generator().manual_seed(5)
    pos = torch.arange(40, dtype=torch.int32).cuda()
    freq, _ = binding.rope_frequencies(rot, 1e6)
    x = torch.randn((40, 12, 128), generator=gen).to(DT[dtype]).cuda()
    q, k = x[:, :8], x[:, 8:10]
    want = binding.rotary(q, k, pos, freq, interleaved=interleaved)
    before = x[:, 10:].clone()
    h = torch.zeros((8, 40, 128), dtype=DT[dtype], device="cuda").transpose(0, 1)
    binding.rotary(q, None, pos, freq, interleaved=interleaved, q_out=h)
    assert torch.equal(h, want[0])
    binding.rotary(q, k, pos, freq, interleaved=interleaved, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, 10:], before)


def ragged(lens, tokens, first=0):
    starts = torch.tensor([first] + list(np.cumsum(lens) + first), dtype=torch.int32)
    assert int(starts[-1]) <= tokens
    return starts


@pytest.mark.parametrize("dtype,d,interleaved", [("bf16", 128, False), ("f32", 64, True)])
@pytest.mark.parametrize("page", [0, 1, 16, 24])
@pytest.mark.parametrize("lens,kv,first,pad", [
    ([1], [1], 0, 0), ([3, 0, 5, 1], [3, 0, 100, 77], 0, 0), ([0, 0], [5, 0], 2, 3),
    ([1] * 70, list(range(1, 71)), 1, 2),
    ([i % 3 for i in range(4200)], [i % 3 + i % 131 for i in range(4200)], 2, 1), ([65, 7, 130], [65, 107, 131], 0, 9)])
def test_append(dtype, d, interleaved, page, lens, kv, first, pad):
    from paper_2606_02544_amd import binding
    hq, hkv, cap = 4, 2, 136
    tokens = first + sum(lens) + pad
    gen = torch.Generator().manual_seed(11)
    q, k, v = make(tokens, [hq, hkv, hkv], d, DT[dtype], gen, fused=True)
    starts = ragged(lens, tokens, first)
    b = len(lens)
    if page:
        per = -(-cap // page)
        table = torch.randperm(b * per, generator=gen).view(b, per).to(torch.int32)
        shape = (b * per, page, hkv, d)
    else:
        table, shape = None, (b, cap, hkv, d)
    kc = torch.full(shape, 7.0, dtype=DT[dtype], device="cuda")
    vc = torch.full(shape, -7.0, dtype=DT[dtype], device="cuda")
    q_out = torch.full((tokens, hq, d), 3.0, dtype=DT[dtype], device="cuda")
    freq, _ = binding.rope_frequencies(d, 10000.0)
    got = binding.rotary_append(q, k, v, kc, vc, None if table is None else table.cuda(), starts.cuda(),
                                torch.tensor(kv, dtype=torch.int32).cuda(), freq, max_kv_len=cap,
                                page_size=page, interleaved=interleaved, q_out=q_out)
    assert got is q_out
    rows = ref.cache_rows(starts.tolist(), kv, tokens)
    live = [t for t in range(tokens) if rows[t][0] >= 0]
    want_k, want_v = torch.full(shape, 7.0, dtype=DT[dtype]), torch.full(shape, -7.0, dtype=DT[dtype])
    at = []
    for t in live:
        s, i = rows[t]
        at.append((int(table[s, i // page]), i % page) if page else (s, i))
        want_v[at[-1]] = v[t].cpu()
    assert torch.equal(vc.cpu(), want_v)
    pos = np.array([rows[t][1] for t in live])
    if live:
        check(q_out[live], q[live], pos, freq.cpu().numpy(), interleaved, 1.0)
        new_k = torch.stack([kc[a] for a in at])
        check(new_k, k[live], pos, freq.cpu().numpy(), interleaved, 1.0)
        for a in at:
            kc[a] = 7.0
    assert torch.equal(kc.cpu(), want_k)                       # nothing else was written
    dead = [t for t in range(tokens) if rows[t][0] < 0]
    assert bool((q_out[dead] == 3.0).all())


def test_append_skips_what_has_no_row():
    """Indices outside [0, max_kv_len) and pages outside the pool are not written;
    positions of their own turn queries and keys."""
    from paper_2606_02544_amd import binding
    gen = torch.Generator().manual_seed(2)
    q, k, v = make(12, [2, 1, 1], 64, torch.float32, gen)
    starts = torch.tensor([0, 4, 8, 12], dtype=torch.int32).cuda()
    kv = torch.tensor([2, 34, 20], dtype=torch.int32).cuda()      # -2.., 30..33, 16..19
    table = torch.tensor([[0, 1], [-1, 2], [3, 9]], dtype=torch.int32).cuda()
    kc = torch.zeros((4, 16, 1, 64), device="cuda")
    vc = torch.zeros_like(kc)
    pos = torch.arange(100, 112, dtype=torch.int32).cuda()
    freq, _ = binding.rope_frequencies(64, 10000.0)
    out = binding.rotary_append(q, k, v, kc, vc, table, starts, kv, freq, max_kv_len=32, page_size=16, positions=pos)
    check(out, q, pos.cpu().numpy(), freq.cpu().numpy(), False, 1.0)
    want = torch.zeros((4, 16, 1, 64))
    want[0, 0], want[0, 1] = v[2].cpu(), v[3].cpu()
    want[2, 14], want[2, 15] = v[4].cpu(), v[5].cpu()
    assert torch.equal(vc.cpu(), want)
    assert torch.equal(kc[0, 0], binding.rotary(None, k, pos, freq)[1][2])


def test_append_replayed_from_a_graph():
    from paper_2606_02544_amd import binding
    gen = torch.Generator().manual_seed(4)
    q, k, v = make(6, [4, 2, 2], 128, torch.bfloat16, gen)
    starts = torch.tensor([0, 2, 6], dtype=torch.int32).cuda()
    kv = torch.tensor([2, 4], dtype=torch.int32).cuda()
    kc = torch.zeros((2, 64, 2, 128), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    freq, _ = binding.rope_frequencies(128, 10000.0)
    call = lambda a, b: binding.rotary_append(q, k, v, a, b, None, starts, kv, freq, max_kv_len=64)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(kc, vc)
    for _ in range(3):
        ke, ve = kc.clone(), vc.clone()
        eager = call(ke, ve)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(kc, ke) and torch.equal(vc, ve)
        kv += torch.tensor([3, 9], dtype=torch.int32, device="cuda")
        q.mul_(0.5)


def test_another_stream():
    from paper_2606_02544_amd import binding
    q = torch.randn((1000, 8, 128), device="cuda")
    pos = torch.arange(1000, dtype=torch.int32, device="cuda")
    freq, _ = binding.rope_frequencies(128, 10000.0)
    want, _ = binding.rotary(q, None, pos, freq)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, _ = binding.rotary(q, None, pos, freq, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)


def test_no_tokens():
    from paper_2606_02544_amd import binding
    freq, _ = binding.rope_frequencies(128, 10000.0)
    out, _ = binding.rotary(torch.zeros((0, 4, 128), device="cuda"), None,
                            torch.zeros(0, dtype=torch.int32, device="cuda"), freq)
    assert out.shape == (0, 4, 128)


def test_turned_keys_serve_the_verification():
    """Keys and queries of the new slots turned here, at their RoPE-copy positions,
    give what the verification's own rotation gives (both bf16: two roundings of
    keys and queries, so as its parity tests compare it, 2e-2 of the row)."""
    from gpu_util import DeviceInputs
    from paper_2606_02544_amd import binding
    from synth import CONFIGS, generate
    cfg = CONFIGS[2].replace(prefix=200)
    inp = generate(cfg)
    d = DeviceInputs(inp)
    call = lambda q, k, theta: binding.verify_attention(  # noqa: E731
        q, k, d.v_new, d.k_cache, d.v_cache, None, d.prefix_lens, d.step_map, d.num_ref,
        block_size=4, max_ref=4, max_prefix_len=200, rope_theta=theta)[0]
    step = inp.step_map[0]
    pos = [200 + i for i in range(4)] + [200 + int(np.flatnonzero(step == r + 1)[0]) for r in range(4)]
    freq, _ = binding.rope_frequencies(128, 10000.0)
    q, k = binding.rotary(d.q[0], d.k_new[0], torch.tensor(pos, dtype=torch.int32).cuda(), freq)
    a, b = call(q[None], k[None], 0.0).float(), call(d.q, d.k_new, 10000.0).float()
    assert bool(((a - b).abs().amax(-1) <= 2e-2 * b.abs().amax(-1)).all())
