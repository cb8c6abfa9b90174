"""The verification step's attention under a sliding window with sinks and over a 4-bit
prefix, on the GPU against the float64 oracle; tolerances as derived for bf16 chunk
attention (tests/test_gpu_chunk.py), n the keys of prefix and new slots."""

import numpy as np
import pytest
import torch

import oracle.window as ref
from test_gpu_fp4 import decoded, random_cache, to_gpu
from test_gpu_window import near

pytestmark = pytest.mark.gpu
FORMS = ["bf16", "fp4"]


def make(form, prefix, B, L, hq, hkv, d, page, seed, mode="mixed"):
    g = torch.Generator().manual_seed(seed)
    b, n, cap = len(prefix), B + L, max(max(prefix), 1)
    new = lambda *s: torch.randn(s, generator=g).bfloat16()  # noqa: E731
    s = dict(form=form, q=new(b, n, hq, d), k=new(b, n, hkv, d), v=new(b, n, hkv, d), B=B, L=L, page=page, cap=max(prefix),
             prefix=torch.tensor(prefix, dtype=torch.int32), table=None)
    per = -(-cap // page) if page else 0
    shape = (b * per + 1, page, hkv) if page else (b, cap, hkv)
    held = torch.arange(cap) < s["prefix"][:, None]
    if page:
        s["table"] = torch.randperm(b * per, generator=g).view(b, per).to(torch.int32)
        held = torch.zeros(shape[:2], dtype=torch.bool)
        for i, x in enumerate(prefix):
            for t in range(x):
                held[int(s["table"][i, t // page]), t % page] = True
            s["table"][i, -(-x // page):] = b * per
    if form == "fp4":
        s["cache"] = random_cache(shape, d, g)
        s["cache"][2][~held] = 255
        s["cache"][3][~held] = 255
    else:
        s["cache"] = [new(*shape, d) for _ in range(2)]
        for x in s["cache"]:
            x[~held] = float("nan")
    # Steps: 1..gamma in a random order; the rest committed, not drafted, or padding.
    gamma = [int(torch.randint(0, L + 1, (1,), generator=g)) if mode == "mixed" else L for _ in prefix]
    steps = torch.zeros((b, B), dtype=torch.int32)
    for i, m in enumerate(gamma):
        order = torch.randperm(B, generator=g)
        steps[i, order[:m]] = torch.arange(1, m + 1, dtype=torch.int32)
        if mode == "mixed":
            steps[i, order[m:]] = torch.tensor([0, m + 1, -1, -3], dtype=torch.int32)[torch.randint(0, 4, (B - m,), generator=g)]
    s["steps"], s["gamma"] = steps, torch.tensor(gamma, dtype=torch.int32)
    return s


def call(s, dev=None, **kw):
    from paper_2606_02544_amd import binding
    c = lambda x: None if x is None else x.cuda()  # noqa: E731
    cache = [to_gpu(x) for x in s["cache"]]
    sizes = dict(block_size=s["B"], max_ref=s["L"], max_prefix_len=s["cap"], page_size=s["page"])
    new, rest = (c(s["q"]), c(s["k"]), c(s["v"])), (c(s["table"]), c(s["prefix"]), c(s["steps"]), c(s["gamma"]))
    if s["form"] == "fp4":
        return binding.verify_attention_fp4(*new, binding.Fp4Cache(*cache), *rest, **sizes, **kw)
    return binding.verify_attention(*new, *cache, *rest, **sizes, **kw)


def check(s, out, lse, window, sinks, scale=0.0):
    f = lambda x: x.double().cpu().numpy()  # noqa: E731
    k, v = decoded(s["cache"]) if s["form"] == "fp4" else (f(x) for x in s["cache"])
    want, wl, size, S = ref.verify_attention(f(s["q"]), f(s["k"]), f(s["v"]), k, v, s["table"], s["prefix"], s["steps"].numpy(),
                                             s["gamma"], window=window, sinks=sinks, page=s["page"], scale=scale)
    got = f(out)
    dead = np.isneginf(wl).transpose(0, 2, 1)
    assert not got[dead].any()
    near(got, f(lse).transpose(0, 2, 1), want, wl.transpose(0, 2, 1), size, S.transpose(0, 2, 1), s["q"].shape[3],
         s["cap"] + s["B"] + s["L"], True)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("B,L,hq,hkv", [(1, 0, 1, 1), (4, 4, 4, 2), (8, 8, 8, 2), (7, 3, 6, 2), (32, 32, 4, 1), (16, 9, 32, 2), (64, 0, 2, 2)])
def test_shapes(form, d, page, B, L, hq, hkv):
    """Row blocks of each size, one sequence without a prefix."""
    s = make(form, [200, 0, 65, 1], B, L, hq, hkv, d, page, B + L)
    for window, sinks in ((60, 3),) if form == "bf16" else ((0, 0), (60, 3)):
        check(s, *call(s, window=window, sinks=sinks), window, sinks)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 70), (64, 0), (65, 4), (100, 64), (10 ** 6, 5), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("kv_chunk", [0, 64, 128])
def test_windows(form, window, sinks, kv_chunk):
    s = make(form, [300, 64, 127, 500], 8, 8, 8, 2, 64, 24, 3)
    check(s, *call(s, window=window, sinks=sinks, kv_chunk=kv_chunk), window, sinks)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("page", [0, 1, 5, 64, 100, 256])
@pytest.mark.parametrize("kv_chunk", [0, 64])
def test_pages_and_key_ranges(form, page, kv_chunk):
    s = make(form, [450, 257, 64, 0], 4, 4, 4, 2, 128, page, 4)
    check(s, *call(s, window=200, sinks=4, kv_chunk=kv_chunk), 200, 4)
    if form == "fp4":
        check(s, *call(s, kv_chunk=kv_chunk), 0, 0)


@pytest.mark.parametrize("form", FORMS)
def test_no_prefix_at_all(form):
    s = make(form, [0, 0], 8, 8, 4, 2, 128, 0, 5)
    for x in s["cache"]:
        x.fill_(0)
    check(s, *call(s, window=50, sinks=2), 50, 2)


@pytest.mark.parametrize("page", [0, 16])
def test_a_window_past_the_prefix_is_the_step_without(page):
    """Both within the tolerance of the oracle."""
    s = make("bf16", [300, 90], 8, 8, 8, 2, 128, page, 6)
    check(s, *call(s, window=10 ** 6), 0, 0)
    check(s, *call(s), 0, 0)


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("kv_chunk", [0, 64])
def test_what_a_slot_does_not_see(form, kv_chunk):
    """NaN in the prefix outside window and sinks, and in padded and hidden new slots."""
    s = make(form, [300, 200], 6, 6, 4, 2, 64, 16, 7)
    s["steps"] = torch.tensor([[1, 2, 3, -1, 0, 5], [2, 1, -1, -1, 3, 4]], dtype=torch.int32)
    s["gamma"] = torch.tensor([3, 4], dtype=torch.int32)
    base, base_lse = call(s, window=80, sinks=4, kv_chunk=kv_chunk)
    for b, prefix in ((0, 300), (1, 200)):
        for t in (4, 50, prefix - 80):
            at = (int(s["table"][b, t // 16]), t % 16)
            for x in s["cache"][2:] if form == "fp4" else s["cache"]:
                x[at] = 255 if form == "fp4" else float("nan")
    for x in (s["k"], s["v"]):
        x[0, 3], x[1, 2], x[1, 3] = (float("nan"),) * 3        # padded block slots
        x[0, 6 + 3:], x[1, 6 + 4:] = float("nan"), float("inf")   # padded reference slots
    s["v"][0, 6 + 2, 1, 5] = float("inf")                      # draft 3's slot: seen by itself and label 4 on
    out, lse = call(s, window=80, sinks=4, kv_chunk=kv_chunk)
    want = base.clone()
    for slot in (8, 5):                                        # itself, and the undrafted slot (label 4)
        want[0, slot, 2:, 5] = float("inf")
    assert torch.equal(out, want) and torch.equal(lse, base_lse)


@pytest.mark.parametrize("form", FORMS)
def test_given_scale_and_large_scores(form):
    s = make(form, [90], 8, 8, 2, 1, 64, 0, 8, mode="full")
    check(s, *call(s, window=40, sinks=1, scale=0.5), 40, 1, 0.5)
    s["q"] = (s["q"] * 40).bfloat16()
    check(s, *call(s, window=40, sinks=1), 40, 1)


def test_a_large_batch():
    """More sequences than the chip holds work-groups, ranges and none."""
    s = make("fp4", [(i * 37) % 190 for i in range(300)], 4, 4, 4, 2, 64, 16, 9)
    for kv_chunk in (0, 64):
        check(s, *call(s, kv_chunk=kv_chunk, window=90, sinks=2), 90, 2)


@pytest.mark.parametrize("page", [0, 16])
def test_order_of_the_prefixes(page):
    """Lengths that rise, fall, repeat and are 0: each sequence has its own outputs."""
    for prefix in ([5, 300, 0, 64, 300, 17, 0], [700, 400, 100], [1, 2, 3, 500], list(range(64))):
        s = make("fp4", prefix, 4, 2, 4, 2, 64, page, len(prefix))
        for kv_chunk in (0, 128):
            check(s, *call(s, kv_chunk=kv_chunk), 0, 0)


@pytest.mark.parametrize("form", FORMS)
def test_blocks_that_end_inside_a_slot(form):
    s = make(form, [90, 0, 200], 7, 4, 15, 1, 64, 16, 12)
    for kv_chunk in (0, 64):
        check(s, *call(s, kv_chunk=kv_chunk, window=70, sinks=2), 70, 2)
        if form == "fp4":
            check(s, *call(s, kv_chunk=kv_chunk), 0, 0)


@pytest.mark.parametrize("form", FORMS)
def test_replays_of_a_graph_and_another_stream(form):
    from paper_2606_02544_amd import binding
    sets = [make(form, [500, 300], 8, 8, 8, 2, 128, 16, 20 + i) for i in range(2)]
    gpu = []
    for s in sets:
        c = {k: (x.cuda() if isinstance(x, torch.Tensor) else x) for k, x in s.items()}
        gpu.append(dict(c, cache=[to_gpu(x) for x in s["cache"]]))

    def run(s, **kw):
        kw |= dict(block_size=s["B"], max_ref=s["L"], max_prefix_len=s["cap"], page_size=s["page"], window=400, sinks=4, kv_chunk=64)
        rest = (s["table"], s["prefix"], s["steps"], s["gamma"])
        if form == "fp4":
            return binding.verify_attention_fp4(s["q"], s["k"], s["v"], binding.Fp4Cache(*s["cache"]), *rest, **kw)
        return binding.verify_attention(s["q"], s["k"], s["v"], *s["cache"], *rest, **kw)

    eager = [run(s) for s in gpu]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(gpu[0])
    for _ in range(4):
        got[0].fill_(5.0)
        graph.replay()
        other = run(gpu[1])
        torch.cuda.synchronize()
        assert torch.equal(got[0], eager[0][0]) and torch.equal(got[1], eager[0][1])
        assert torch.equal(other[0], eager[1][0])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    again = run(gpu[0], stream=st)
    torch.cuda.synchronize()
    assert torch.equal(again[0], eager[0][0]) and torch.equal(again[1], eager[0][1])
