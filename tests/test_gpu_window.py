"""Chunk attention under a sliding window with sinks, on the GPU against the float64
oracle; tolerances as derived for chunk attention (tests/test_gpu_chunk.py), n the
keys of the cache."""

import numpy as np
import pytest
import torch

import oracle.window as ref
from test_gpu_chunk import DT, call, make

pytestmark = pytest.mark.gpu
INF = float("inf")
TYPES = [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)]


def near(got, gl, want, wl, size, S, d, n, bf16):
    """Outputs [..., d] and log-sum-exps [...] within the tolerance; S as wl."""
    score = (d + 16) * 2.0 ** -24 * S
    tol = ((2 * score + n * 2.0 ** -23)[..., None] + (2.0 ** -8 if bf16 else 0)) * size \
        + (2.0 ** -8 if bf16 else 2.0 ** -23) * np.abs(want)
    err = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (err <= tol + 1e-30).all(), float((err - tol).max())
    assert np.array_equal(np.isneginf(gl), np.isneginf(wl))
    fin = ~np.isneginf(wl)
    lt = (score + n * 2.0 ** -24 + 2.0 ** -22 + 2.0 ** -23 * np.abs(np.where(fin, wl, 0)))[fin]
    assert (np.abs(gl[fin] - wl[fin]) <= lt).all()


def check(s, out, lse, mask_block, window, sinks, scale=0.0):
    f = lambda x: x.double().cpu().numpy()  # noqa: E731
    want, wl, size, S = ref.chunk_attention(f(s["q"]), f(s["k"]), f(s["v"]), s["table"], s["starts"].tolist(),
                                            s["kv"].tolist(), mask_block=mask_block, window=window, sinks=sinks,
                                            page=s["page"], scale=scale)
    rows = ~np.isnan(wl[0])
    near(f(out)[rows], f(lse).T[rows], want[rows], wl.T[rows], size[rows], S.T[rows], s["q"].shape[2], s["cap"],
         s["q"].dtype == torch.bfloat16)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (7, 3), (64, 0), (65, 4), (100, 64), (33, 130), (1000, 5)])
def test_windows(dtype, d, window, sinks):
    """Single tokens, chunks and prompts; windows shorter than a tile and longer than the
    cache, sinks that meet the window and that do not, longer than a tile and than the
    cache; a sequence without new tokens."""
    s = make([(1, 1), (1, 65), (1, 400), (5, 5), (0, 50), (40, 300), (90, 90)], 8, 2, d, dtype, 16, 1)
    for mask_block in (1, 8):
        check(s, *call(s, mask_block=mask_block, window=window, sinks=sinks), mask_block, window, sinks)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [0, 1, 5, 24, 64, 100, 256])
@pytest.mark.parametrize("kv_chunk", [0, 64, 128])
def test_pages_and_key_ranges(dtype, d, page, kv_chunk):
    s = make([(7, 450), (40, 257), (1, 64), (1, 449)], 4, 2, d, dtype, page, 2)
    for window, sinks in ((150, 4), (40, 70)):
        check(s, *call(s, mask_block=4, kv_chunk=kv_chunk, window=window, sinks=sinks), 4, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask_block", [1, 3, 32, 100, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 2 ** 31 - 1), (50, 2), (1, 0)])
def test_mask_blocks(dtype, mask_block, window, sinks):
    """Blocks of any size, whose tokens all see the same keys; windows and sinks up to
    the largest number."""
    s = make([(150, 290), (130, 130)], 2, 1, 64, dtype, 0, 3)
    for kv_chunk in (0, 64):
        check(s, *call(s, mask_block=mask_block, window=window, sinks=sinks, kv_chunk=kv_chunk), mask_block, window, sinks)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("max_q", [1, 4, 20, 40, 500])
@pytest.mark.parametrize("page", [0, 16])
def test_every_group_shape(dtype, d, max_q, page):
    s = make([(9, 70), (1, 333), (90, 400), (70, 70)], 8, 2, d, dtype, page, 4)
    for kv_chunk in (0, 128):
        check(s, *call(s, mask_block=1, max_q_len=max_q, kv_chunk=kv_chunk, window=77, sinks=9), 1, 77, 9)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [0, 16])
def test_large(dtype, d, page):
    """The largest work-groups: rows by rows against a call of single rows' keys."""
    s = make([(1500, 1700), (1, 900), (400, 2000)], 32, 8, d, dtype, page, 14)
    out, lse = call(s, mask_block=8, window=600, sinks=20)
    g = np.random.RandomState(5)
    starts, kv = s["starts"].tolist(), s["kv"].tolist()
    f = lambda x: x.double().cpu().numpy()  # noqa: E731
    for t in sorted(set(g.randint(0, s["q"].shape[0], 24).tolist() + [0, starts[-1] - 1] + starts[:-1])):
        b = max(i for i in range(len(kv)) if starts[i] <= t < starts[i + 1])
        n = starts[b + 1] - starts[b]
        seen = ref.keys(kv[b], n, t - starts[b], 8, 600, 20)
        k, v = (f(ref.gather(s[x], s["table"], b, kv[b], page) if not page else
                  torch.stack([s[x][int(s["table"][b, i // page]), i % page] for i in range(kv[b])])) for x in ("k", "v"))
        for h in (0, 13, 31):
            want, wl, size, S = ref.row(f(s["q"][t, h]), k[seen, h // 4], v[seen, h // 4], d ** -0.5)
            near(f(out[t, h])[None], f(lse[h, t])[None], want[None], np.array([wl]), size[None], np.array([S]), d, s["cap"],
                 dtype == "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_negative_positions(dtype):
    s = make([(10, 4), (3, 0), (80, 75)], 4, 2, 128, dtype, 0, 5)
    for mask_block in (1, 4):
        for window, sinks in ((2, 1), (30, 0)):
            check(s, *call(s, mask_block=mask_block, window=window, sinks=sinks), mask_block, window, sinks)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_chunk", [0, 64])
def test_rows_outside_the_batch_stay(dtype, kv_chunk):
    s = make([(4, 300), (0, 3), (30, 190)], 4, 1, 128, dtype, 16, 6, first=3, pad=7)
    out = torch.full(s["q"].shape, 9.0, dtype=DT[dtype], device="cuda")
    lse = torch.full((4, s["q"].shape[0]), 9.0, device="cuda")
    call(s, mask_block=1, out=out, lse=lse, kv_chunk=kv_chunk, window=100, sinks=4)
    check(s, out, lse, 1, 100, 4)
    rows = torch.tensor([i for i in range(out.shape[0]) if i < 3 or i >= 37])
    assert bool((out[rows] == 9.0).all()) and bool((lse[:, rows] == 9.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,first", [(64, 3), (65, 3), (4161, 2)])
def test_many_sequences_and_strides(dtype, batch, first):
    s = make([(i % 4, i % 4 + (37 * i) % 190) for i in range(batch)], 4, 2, 64, dtype, 16, 7, first=first, pad=first, order="htd")
    for kv_chunk in (0, 64):
        check(s, *call(s, mask_block=1, kv_chunk=kv_chunk, window=30, sinks=2), 1, 30, 2)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("kv_chunk", [0, 64])
@pytest.mark.parametrize("max_q", [1, 20, 40, 500])
def test_what_a_row_does_not_see(dtype, d, kv_chunk, max_q):
    """Infinities and NaN before the window, behind the row and between the sinks and the
    window change nothing; those inside it do what they do in the formula."""
    window, sinks = 90, 5
    s = make([(60, 350), (1, 300)], 4, 2, d, dtype, 16, 31)
    base, base_lse = call(s, mask_block=1, kv_chunk=kv_chunk, max_q_len=max_q, window=window, sinks=sinks)

    def at(b, t):
        return int(s["table"][b, t // 16]), t % 16

    # Token i of the first sequence sees [201 + i, 291 + i) and [0, 5); the other [210, 300).
    for b, t, dim, value in ((0, 5, 3, INF), (0, 200, 4, float("nan")), (1, 209, 3, INF), (1, 5, 6, float("nan")),
                             (0, 4, 7, -INF), (0, 220, 9, INF), (0, 345, 11, float("nan")), (1, 0, 5, INF), (1, 299, 8, -INF)):
        s["v"][(*at(b, t), 1, dim)] = value
    s["k"][(*at(0, 150), 1)] = float("nan")
    s["k"][(*at(1, 100), 1)] = INF
    out, lse = call(s, mask_block=1, kv_chunk=kv_chunk, max_q_len=max_q, window=window, sinks=sinks)
    want = base.clone()
    want[:60, 2:, 7] = -INF
    want[:20, 2:, 9] = INF                                     # 220 >= 201 + i
    want[55:60, 2:, 11] = float("nan")                         # 345 < 291 + i
    want[60, 2:, 5], want[60, 2:, 8] = INF, -INF
    same = (out == want) | (out.isnan() & want.isnan())
    assert bool(same.all()), (~same).nonzero()[:8]
    assert torch.equal(lse, base_lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_given_away(dtype):
    """Pages none of whose keys are seen may hold other sequences' tokens, or anything:
    their entries point to a page of NaN here."""
    s = make([(1, 500), (3, 700), (1, 90)], 4, 2, 64, dtype, 16, 9)
    want = call(s, mask_block=1, window=100, sinks=6)
    table = s["table"].clone()
    spare = s["k"].shape[0] - 1
    for b, (n, kv) in enumerate(((1, 500), (3, 700), (1, 90))):
        for g in range(1, max(1, (kv - n - 99) // 16)):
            table[b, g] = spare
    assert bool(torch.isnan(s["k"][spare].float()).all()) and int((table == spare).sum()) > int((s["table"] == spare).sum())
    got = call(dict(s, table=table), mask_block=1, window=100, sinks=6)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_window_past_the_cache_is_none(dtype):
    """To the tolerance: the divisions of the keys may differ."""
    s = make([(30, 200), (1, 333)], 4, 2, 128, dtype, 16, 10)
    out, lse = call(s, mask_block=4, window=10 ** 6, sinks=3)
    check(s, out, lse, 4, 0, 0)
    check(s, *call(s, mask_block=4), 4, 0, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    from paper_2606_02544_amd import binding
    d, n = 64, 140
    e = 2 if dtype == "bf16" else 4
    stride = (2 ** 32 // n // 8 + 1024) * 8
    s = make([(2, n)], 1, 1, d, dtype, 0, 11, spare=0.0)
    assert (n - 1) * stride * e > 2 ** 32
    dense = call(s, window=40, sinks=2)
    k, v = (torch.as_strided(torch.empty(stride * (n - 1) + d, dtype=DT[dtype], device="cuda"),
                             (1, n, 1, d), (stride * n, stride, d, 1)) for _ in range(2))
    k.copy_(s["k"].cuda())
    v.copy_(s["v"].cuda())
    out, lse = binding.chunk_attention(s["q"].cuda(), k, v, None, s["starts"].cuda(), s["kv"].cuda(),
                                       max_q_len=2, max_kv_len=n, window=40, sinks=2)
    assert torch.equal(out, dense[0]) and torch.equal(lse, dense[1])


def test_replays_of_two_graphs_and_another_stream():
    from paper_2606_02544_amd import binding
    sets, graphs, outs = [], [], []
    for seed in (1, 2):
        s = make([(3, 500), (1, 700)], 4, 2, 128, "bf16", 0, 20 + seed, spare=0.0)
        sets.append({k: (x.cuda() if isinstance(x, torch.Tensor) else x) for k, x in s.items()})
    run = lambda s, **kw: binding.chunk_attention(s["q"], s["k"], s["v"], None, s["starts"], s["kv"],  # noqa: E731
                                                  max_q_len=3, max_kv_len=s["cap"], kv_chunk=64, window=300, sinks=4, **kw)
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
    streams[0].wait_stream(torch.cuda.current_stream())
    got = run(sets[0], stream=streams[0])
    torch.cuda.synchronize()
    assert torch.equal(got[0], eager[0][0]) and torch.equal(got[1], eager[0][1])
