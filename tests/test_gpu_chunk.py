"""Chunk attention on the GPU against the float64 oracle.

Tolerances, A = sum p |v| / sum p of a row and dim, S = the largest
scale * sum |q_i k_i| of the row, n its keys:
  * a score is off by (d + 16) 2^-24 S at most (fp32 sum of d products, the scale,
    the exponent's FMA), so a weight by as much relatively, and the quotient by
    twice that of A;
  * fp32 sums of n products: n 2^-24 A, and n 2^-24 of the weights' sum;
  * bf16: each weight is rounded to bf16, 2^-8 A; the output half a step, 2^-8 |o|
    (fp32: two roundings of the quotient, 2^-23 |o|).
The log-sum-exp: the score's error, n 2^-24, and 2^-22 of the hardware logarithm,
2^-23 of its own size."""

import numpy as np
import pytest
import torch

import oracle.chunk as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(lens, hq, hkv, d, dtype, page, seed, first=0, pad=0, spare=float("nan"), cap=None, order="thd"):
    """lens: (new, kv) of each sequence.  Cache entries past kv hold `spare`."""
    g = torch.Generator().manual_seed(seed)
    b, cap = len(lens), cap or max(max(kv for _, kv in lens), 1)
    n = [x for x, _ in lens]
    T = first + sum(n) + pad
    starts = torch.tensor([first] + list(np.cumsum(n) + first), dtype=torch.int32)
    kv = torch.tensor([x for _, x in lens], dtype=torch.int32)
    q = torch.randn((T, hq, d), generator=g).to(DT[dtype])
    per = -(-cap // page) if page else 0
    shape = (b * per + 1, page, hkv, d) if page else (b, cap, hkv, d)
    k, v = (torch.randn(shape, generator=g).to(DT[dtype]) for _ in range(2))
    table = None
    if page:
        table = torch.randperm(b * per, generator=g).view(b, per).to(torch.int32)
        held = torch.zeros(shape[:2], dtype=torch.bool)
        for i, x in enumerate(kv.tolist()):
            for t in range(x):
                held[int(table[i, t // page]), t % page] = True
            table[i, -(-x // page):] = b * per                  # unused entries: a spare page
    else:
        held = torch.arange(cap) < kv[:, None]
    k[~held] = spare
    v[~held] = spare
    if order == "htd":                                          # heads outside tokens in memory
        k, v = (x.transpose(1, 2).contiguous().transpose(1, 2) for x in (k, v))
    return dict(q=q, k=k, v=v, table=table, starts=starts, kv=kv, cap=cap, page=page, max_q=max(n))


def call(s, dev=True, **kw):
    from paper_2606_02544_amd import binding
    x = [s[n].cuda() if s[n] is not None else None for n in ("q", "k", "v", "table", "starts", "kv")]
    kw.setdefault("max_q_len", s["max_q"])
    out, lse = binding.chunk_attention(*x, max_kv_len=s["cap"], page_size=s["page"], **kw)
    return out, lse


def check(s, out, lse, mask_block, scale=0.0):
    f = lambda x: x.double().numpy()  # noqa: E731
    want, wl, size, S = ref.chunk_attention(f(s["q"]), f(s["k"]), f(s["v"]), s["table"], s["starts"].tolist(),
                                            s["kv"].tolist(), mask_block=mask_block, page=s["page"], scale=scale)
    rows = ~np.isnan(wl[0])
    d, n = s["q"].shape[2], s["cap"]
    bf16 = s["q"].dtype == torch.bfloat16
    S = S.T[:, :, None]
    score = (d + 16) * 2.0 ** -24 * S
    tol = (2 * score + n * 2.0 ** -23 + (2.0 ** -8 if bf16 else 0)) * size + (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(want)
    got, gl = f(out.cpu()), f(lse.cpu())
    err = np.abs(got - want)[rows]
    assert np.isfinite(got[rows]).all()
    assert (err <= tol[rows] + 1e-30).all(), float((err - tol[rows]).max())
    assert np.array_equal(np.isneginf(gl[:, rows]), np.isneginf(wl[:, rows]))
    fin = rows[None] & ~np.isneginf(wl)
    lt = (score[:, :, 0].T + n * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -23 * np.abs(wl))[fin]
    assert (np.abs(gl[fin] - wl[fin]) <= lt).all()


SHAPES = [
    ([(1, 1)], 1, 1), ([(1, 64)], 4, 2), ([(1, 65), (1, 1000), (1, 3)], 8, 2), ([(5, 5)], 4, 4),
    ([(64, 64), (1, 130), (0, 50), (17, 140)], 8, 2), ([(100, 300)], 3, 1), ([(33, 33), (70, 200)], 16, 1),
    ([(0, 0), (3, 3), (0, 7)], 2, 1), ([(300, 300)], 4, 1),
]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("lens,hq,hkv", SHAPES)
def test_shapes(dtype, d, page, lens, hq, hkv):
    s = make(lens, hq, hkv, d, dtype, page, 1)
    for mask_block in (1, 8, 0):
        check(s, *call(s, mask_block=mask_block), mask_block)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page", [0, 1, 4, 5, 24, 64, 100, 128, 256])
@pytest.mark.parametrize("kv_chunk", [0, 64, 128])
def test_pages_and_key_ranges(dtype, d, page, kv_chunk):
    """Page sizes that divide a tile, hold several, end inside one or share none of
    its factors; ranges of keys joined by the second kernel."""
    s = make([(7, 450), (40, 257), (1, 64)], 4, 2, d, dtype, page, 2)
    check(s, *call(s, mask_block=4, kv_chunk=kv_chunk), 4)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask_block", [1, 2, 3, 32, 100, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("kv_chunk", [0, 64])
def test_mask_blocks(dtype, mask_block, kv_chunk):
    s = make([(150, 290), (130, 130)], 2, 1, 64, dtype, 0, 3)
    check(s, *call(s, mask_block=mask_block, kv_chunk=kv_chunk), mask_block)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("max_q", [1, 20, 40, 500])
def test_every_group_shape(dtype, d, max_q):
    """The kernel chosen by max_q_len serves sequences of any length."""
    s = make([(9, 70), (1, 333), (90, 200)], 8, 2, d, dtype, 16, 4)
    for kv_chunk in (0, 128):
        check(s, *call(s, mask_block=8, max_q_len=max_q, kv_chunk=kv_chunk), 8)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", [16, 64])
@pytest.mark.parametrize("lens", [[(130, 150)], [(256, 256)], [(300, 320)], [(512, 512)], [(900, 900)],
                                  [(200, 230), (0, 40), (100, 100)], [(64, 64)] * 7 + [(33, 500)]])
def test_blocks_that_share_a_unit(dtype, heads, lens):
    """Between one and two row blocks of whole rows a compute unit, in which case they
    are dealt out by length: every block once."""
    s = make(lens, heads, heads, 64, dtype, 0, 15)
    check(s, *call(s, mask_block=8, kv_chunk=1024), 8)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page", [0, 1, 5, 16, 96])
@pytest.mark.parametrize("lens,hq,hkv", [([(1500, 1700)], 32, 8), ([(700, 2000), (1, 900), (400, 400), (90, 2100)], 32, 8)])
def test_large(dtype, d, page, lens, hq, hkv):
    """Enough rows for the largest work-groups (pages of one token: more of them than a
    work-group holds); a sample of the rows is compared, one by one, and one with the
    value of a later key infinite."""
    s = make(lens, hq, hkv, d, dtype, page, 14)
    out, lse = call(s, mask_block=8)
    f = lambda x: x.double().numpy()  # noqa: E731
    g = np.random.RandomState(5)
    starts, kv = s["starts"].tolist(), s["kv"].tolist()
    tokens = sorted(set(g.randint(0, s["q"].shape[0], 60).tolist() + [0, starts[-1] - 1] + starts[:-1]))
    for t in tokens:
        b = max(i for i in range(len(kv)) if starts[i] <= t < starts[i + 1])
        n = ref.seen(kv[b], starts[b + 1] - starts[b], t - starts[b], 8)
        one = dict(s, q=s["q"][t:t + 1], starts=torch.tensor([0] * (b + 1) + [1] * (len(kv) - b)),
                   kv=torch.tensor([n if i == b else 0 for i in range(len(kv))]))
        check(one, out[t:t + 1], lse[:, t:t + 1], 0)
    # A value that only rows from its block on see.
    at = kv[0] - 300
    where = (int(s["table"][0, at // page]), at % page) if page else (0, at)
    s["v"][where[0], where[1], 0, 3] = float("inf")
    wild, wild_lse = call(s, mask_block=8)
    first = starts[1] - (kv[0] - at // 8 * 8)                  # first token that sees it
    heads = hq // hkv
    assert bool(torch.isinf(wild[first:starts[1], :heads, 3]).all())
    wild[first:starts[1], :heads, 3] = out[first:starts[1], :heads, 3]
    assert torch.equal(wild, out) and torch.equal(wild_lse, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_new_tokens_than_cached(dtype):
    """Rows at negative positions see nothing."""
    s = make([(10, 4), (3, 0), (2, 5)], 4, 2, 128, dtype, 0, 5)
    for mask_block in (0, 1, 4):
        check(s, *call(s, mask_block=mask_block), mask_block)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_chunk", [0, 64])
def test_rows_outside_the_batch_stay(dtype, kv_chunk):
    s = make([(4, 100), (0, 3), (30, 190)], 4, 1, 128, dtype, 16, 6, first=3, pad=7)
    out = torch.full(s["q"].shape, 9.0, dtype=DT[dtype], device="cuda")
    lse = torch.full((4, s["q"].shape[0]), 9.0, device="cuda")
    got = call(s, mask_block=1, out=out, lse=lse, kv_chunk=kv_chunk)
    assert got[0] is out and got[1] is lse
    check(s, out, lse, 1)
    rows = torch.tensor([i for i in range(out.shape[0]) if i < 3 or i >= 37])
    assert bool((out[rows] == 9.0).all()) and bool((lse[:, rows] == 9.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("batch,first", [(64, 3), (65, 3), (150, 0), (130, 1), (4161, 2)])
def test_many_sequences_and_strides(dtype, page, batch, first):
    lens = [(i % 4, i % 4 + (37 * i) % 90) for i in range(batch)]
    s = make(lens, 4, 2, 64, dtype, page, 7, first=first, pad=first, order="htd")
    for kv_chunk in (0, 64):
        check(s, *call(s, mask_block=1, kv_chunk=kv_chunk), 1)


def test_one_cache_for_all_sequences():
    """A cache expanded over the batch (stride 0): a shared prompt."""
    s = make([(3, 80), (2, 80)], 4, 2, 64, "bf16", 0, 15)
    s["k"], s["v"] = (x[:1].expand(2, -1, -1, -1) for x in (s["k"], s["v"]))
    from paper_2606_02544_amd import binding
    k, v = (s[n][:1].cuda().expand(2, -1, -1, -1) for n in ("k", "v"))
    out, lse = binding.chunk_attention(s["q"].cuda(), k, v, None, s["starts"].cuda(), s["kv"].cuda(), max_q_len=3,
                                       max_kv_len=80)
    check(s, out, lse, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_chunk", [0, 64])
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), "both"])
def test_values_and_keys_that_are_no_numbers(dtype, kv_chunk, value):
    """What a row does not see has no part in it; what it sees has."""
    for lens, hq, hkv in (([(90, 150)], 2, 1), ([(12, 70), (200, 333)], 4, 1)):
        s = make(lens, hq, hkv, 128, dtype, 0, 8)
        kv, n = lens[-1][1], lens[-1][0]
        b = len(lens) - 1
        clean = {k: (x.clone() if isinstance(x, torch.Tensor) else x) for k, x in s.items()}
        at = kv - 30                                           # a key that the last rows see
        if value == "both":
            s["v"][b, at, 0, 5], s["v"][b, at + 1, 0, 5] = float("inf"), float("-inf")
            s["v"][b, at, 0, 64] = float("-inf")
        else:
            s["v"][b, at, 0, 5] = s["v"][b, kv - 1, 0, 100] = value
        for mask_block in (1, 4):
            out, lse = call(s, mask_block=mask_block, kv_chunk=kv_chunk)
            base, base_lse = call(clean, mask_block=mask_block, kv_chunk=kv_chunk)
            f = lambda x: x.double().numpy()  # noqa: E731
            want = ref.chunk_attention(f(s["q"]), f(s["k"]), f(s["v"]), None, s["starts"].tolist(),
                                       s["kv"].tolist(), mask_block=mask_block)[0]
            got = f(out.cpu())
            wild = ~np.isfinite(want)
            assert wild.any() and np.array_equal(np.isnan(want), np.isnan(got))
            assert np.array_equal(want[wild & ~np.isnan(want)], got[wild & ~np.isnan(want)])
            assert torch.equal(lse, base_lse)
            keep = torch.from_numpy(~wild)
            assert torch.equal(out.cpu()[keep], base.cpu()[keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_that_are_no_numbers(dtype):
    s = make([(60, 100)], 2, 1, 64, dtype, 0, 9)
    base, base_lse = call(s, mask_block=1)
    s["k"][0, 80] = float("nan")
    s["v"][0, 99] = float("nan")
    out, lse = call(s, mask_block=1)
    assert torch.equal(out[:40], base[:40]) and torch.equal(lse[:, :40], base_lse[:, :40])
    assert bool(torch.isnan(out[40:]).all()) and bool(torch.isnan(lse[:, 40:]).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores_and_given_scale(dtype):
    s = make([(20, 90)], 2, 1, 64, dtype, 0, 10)
    check(s, *call(s, mask_block=1, scale=0.5), 1, 0.5)
    s["q"] = (s["q"] * 40).to(s["q"].dtype)
    check(s, *call(s, mask_block=1), 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """Caches whose tokens, heads or pages lie far apart (element offsets beyond
    2^32): a large buffer seen through strides."""
    d, n = 64, 40
    e = 2 if dtype == "bf16" else 4
    stride = (2 ** 32 // n // 8 + 1024) * 8                    # elements between tokens
    s = make([(2, n)], 1, 1, d, dtype, 0, 11, spare=0.0)
    assert (n - 1) * stride * e > 2 ** 32
    dense = call(s, mask_block=1)
    from paper_2606_02544_amd import binding
    k, v = (torch.as_strided(torch.empty(stride * (n - 1) + d, dtype=DT[dtype], device="cuda"),
                             (1, n, 1, d), (stride * n, stride, d, 1)) for _ in range(2))
    k.copy_(s["k"].cuda())
    v.copy_(s["v"].cuda())
    out, lse = binding.chunk_attention(s["q"].cuda(), k, v, None, s["starts"].cuda(), s["kv"].cuda(),
                                       max_q_len=2, max_kv_len=n)
    assert torch.equal(out, dense[0]) and torch.equal(lse, dense[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_replays_of_two_graphs(dtype):
    """Graphs captured one after the other keep workspaces of their own: replayed
    at once on two streams, and between eager calls, each gives its own result."""
    from paper_2606_02544_amd import binding
    sets, graphs, outs = [], [], []
    for seed in (1, 2):
        s = make([(3, 500), (1, 700)], 4, 2, 128, dtype, 0, 20 + seed, spare=0.0)
        s = {k: (x.cuda() if isinstance(x, torch.Tensor) else x) for k, x in s.items()}
        sets.append(s)
    run = lambda s: binding.chunk_attention(s["q"], s["k"], s["v"], None, s["starts"], s["kv"],  # noqa: E731
                                            max_q_len=3, max_kv_len=s["cap"], kv_chunk=64)
    eager = [run(s) for s in sets]
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(s))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(4):
        for o in outs:
            o[0].fill_(5.0)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        run(sets[0])
        torch.cuda.synchronize()
        for o, e in zip(outs, eager):
            assert torch.equal(o[0], e[0]) and torch.equal(o[1], e[1])


def test_no_tokens_no_keys_and_another_stream():
    from paper_2606_02544_amd import binding
    q = torch.randn((5, 2, 64), device="cuda", dtype=torch.bfloat16)
    starts = torch.tensor([0, 5], dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, dtype=torch.int32, device="cuda")
    out, lse = binding.chunk_attention(q, None, None, None, starts, zero, max_q_len=5, max_kv_len=0)
    assert not out.any() and bool(torch.isneginf(lse).all())
    out, lse = binding.chunk_attention(q[:0], None, None, None, zero.repeat(2), zero, max_q_len=0, max_kv_len=0)
    assert out.shape == (0, 2, 64)
    s = make([(3, 500)], 4, 2, 128, "bf16", 0, 12, spare=0.0)
    want = call(s, kv_chunk=64)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = call(s, kv_chunk=64, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_prompt_as_the_verification_sees_it(dtype):
    """A block of mask tokens without drafts, as a chunk over a cache that holds its
    own keys, is the verification attention of that block."""
    from paper_2606_02544_amd import binding
    B, n = 8, 200
    s = make([(B, n + B)], 4, 2, 64, dtype, 0, 13)
    out, lse = call(s, mask_block=0)
    dev = {k: s[k].cuda() for k in ("q", "k", "v")}
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    want, wl = binding.verify_attention(
        dev["q"][None], dev["k"][:, n:].contiguous(), dev["v"][:, n:].contiguous(), dev["k"], dev["v"], None,
        i32(n), torch.ones((1, B), dtype=torch.int32, device="cuda"), i32(0), block_size=B, max_ref=0,
        max_prefix_len=n)
    check(s, out, lse, 0)
    check(s, want[0], wl[0], 0)
