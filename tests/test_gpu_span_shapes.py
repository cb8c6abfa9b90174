"""Every row-block shape of attention under a window with sinks and over a 4-bit cache, on
the GPU against the float64 oracle: chunks in bf16, fp32 and over 4 bits, verifications in
bf16 and over 4 bits, each with finite values and with such that some rows see and others
do not (infinities and NaN; over 4 bits scales of 255).  Tolerances as derived in
tests/test_gpu_chunk.py, n the keys; what is not finite is equal."""

import functools

import numpy as np
import pytest
import torch

import oracle.window as ref
import span_cases as S
import test_gpu_chunk
import test_gpu_fp4
import test_gpu_verify_span
from test_gpu_fp4 import decoded, to_gpu
from test_gpu_window import near

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
N = max(kv for _, kv in S.LENS)


def f64(x):
    return x.double().cpu().numpy()


def same(got, gl, want, wl, size, spread, d, n, bf16):
    """Outputs [rows..., d] and log-sum-exps [rows...] against the oracle's."""
    wild, lost = ~np.isfinite(want), np.isnan(wl)
    assert np.array_equal(got[wild], want[wild], equal_nan=True), np.argwhere(wild & ~((got == want) | np.isnan(got) & np.isnan(want)))[:5]
    assert np.array_equal(np.isnan(gl), lost)
    zero = lambda x, where: np.where(where, 0.0, x)  # noqa: E731
    near(zero(got, wild), zero(gl, lost), zero(want, wild), zero(wl, lost), zero(size, wild), zero(spread, lost), d, n, bf16)


def spoil(form, place, k, v, hkv, keys, values):
    """NaN, inf or -inf in turn in values of the last KV head, NaN in keys of the first."""
    for i, (b, t) in enumerate(values):
        if form == "fp4":
            v[(*place(b, t), hkv - 1, i % v.shape[3])] = 255
        else:
            v[(*place(b, t), hkv - 1, (5 * i + 3) % v.shape[3])] = (NAN, INF, -INF)[i % 3]
    for b, t in keys:
        k[(*place(b, t), 0)] = 255 if form == "fp4" else NAN


@functools.lru_cache(maxsize=4)
def chunk_data(form, d, hq, hkv, page, wild):
    if form == "fp4":
        s = test_gpu_fp4.make(S.LENS, hq, hkv, d, page, 3)
    else:
        s = test_gpu_chunk.make(S.LENS, hq, hkv, d, form, page, 3)
        s["cache"] = [s["k"], s["v"]]
    if wild:
        place = (lambda b, t: (int(s["table"][b, t // page]), t % page)) if page else (lambda b, t: (b, t))
        at = s["cache"][2:] if form == "fp4" else s["cache"]
        spoil(form, place, *at, hkv, [(0, 340), (1, 120)],
              [(0, 10), (0, 200), (0, 320), (0, 345), (1, 299), (1, 250), (2, 3), (3, 30), (0, 100), (1, 5)])
    return s


@functools.lru_cache(maxsize=64)
def chunk_oracle(form, d, hq, hkv, page, wild, window, sinks, m):
    s = chunk_data(form, d, hq, hkv, page, wild)
    k, v = decoded(s["cache"]) if form == "fp4" else map(f64, s["cache"])
    with np.errstate(invalid="ignore"):
        want, wl, size, spread = ref.chunk_attention(f64(s["q"]), k, v, s["table"], s["starts"].tolist(), s["kv"].tolist(),
                                                     mask_block=m, window=window, sinks=sinks, page=page)
    return want, wl.T, size, spread.T


def chunks(form, d, hq, hkv, page, wild, ranges):
    from paper_2606_02544_amd import binding
    s = chunk_data(form, d, hq, hkv, page, wild)
    cache = [to_gpu(x) for x in s["cache"]]
    where = (None if s["table"] is None else s["table"].cuda(), s["starts"].cuda(), s["kv"].cuda())
    for tokens in S.TOKENS:
        q = torch.full((tokens, hq, d), NAN, dtype=s["q"].dtype, device="cuda")
        q[:S.NEW] = s["q"].cuda()
        for window, sinks, m in S.windows(form):
            for kv_chunk in ranges:
                out, lse = torch.full_like(q, 9.0), torch.full((hq, tokens), 9.0, device="cuda")
                kw = dict(max_q_len=max(n for n, _ in S.LENS), max_kv_len=N, page_size=page, mask_block=m, kv_chunk=kv_chunk,
                          window=window, sinks=sinks, out=out, lse=lse)
                if form == "fp4":
                    binding.chunk_attention_fp4(q, binding.Fp4Cache(*cache), *where, **kw)
                else:
                    binding.chunk_attention(q, *cache, *where, **kw)
                assert bool((out[S.NEW:] == 9.0).all()) and bool((lse[:, S.NEW:] == 9.0).all()), "rows of no sequence"
                same(f64(out[:S.NEW]), f64(lse[:, :S.NEW]).T, *chunk_oracle(form, d, hq, hkv, page, wild, window, sinks, m), d, N,
                     form != "f32")


@pytest.mark.parametrize("form", ["bf16", "fp4", "f32"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("hq,hkv", S.HEADS)
@pytest.mark.parametrize("page", [0, 24])
def test_chunks(form, d, hq, hkv, page):
    chunks(form, d, hq, hkv, page, False, (0, 64))


@pytest.mark.parametrize("form", ["bf16", "fp4", "f32"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("page", [0, 16])
def test_chunks_with_values_that_are_not_finite(form, d, page):
    chunks(form, d, 16, 2, page, True, (0, 128))


@functools.lru_cache(maxsize=4)
def step_data(form, B, L, hq, hkv, d, page, wild):
    s = test_gpu_verify_span.make(form, S.PREFIXES, B, L, hq, hkv, d, page, B + d)
    if wild:
        place = (lambda b, t: (int(s["table"][b, t // page]), t % page)) if page else (lambda b, t: (b, t))
        at = s["cache"][2:] if form == "fp4" else s["cache"]
        spoil(form, place, *at, hkv, [(0, 230)], [(0, 3), (0, 150), (0, 299), (2, 96), (2, 60), (2, 0)])
        for i in range(len(S.PREFIXES)):                       # values of new slots: seen by those whom the mask lets
            s["v"][i, i, hkv - 1, 7], s["v"][i, B + L - 1, hkv - 1, 9] = NAN, INF
    return s


@functools.lru_cache(maxsize=64)
def step_oracle(form, B, L, hq, hkv, d, page, wild, window, sinks):
    s = step_data(form, B, L, hq, hkv, d, page, wild)
    k, v = decoded(s["cache"]) if form == "fp4" else map(f64, s["cache"])
    with np.errstate(invalid="ignore"):
        want, wl, size, spread = ref.verify_attention(f64(s["q"]), f64(s["k"]), f64(s["v"]), k, v, s["table"], s["prefix"],
                                                      s["steps"].numpy(), s["gamma"], window=window, sinks=sinks, page=page)
    return want, wl.transpose(0, 2, 1), size, spread.transpose(0, 2, 1)


def steps(form, B, L, hq, hkv, d, page, wild, ranges):
    """Copies of a batch in a larger one: each as the first, to the bit."""
    from paper_2606_02544_amd import binding
    s = step_data(form, B, L, hq, hkv, d, page, wild)
    b = len(S.PREFIXES)
    for n in S.COPIES:
        many = lambda x: x.cuda().repeat(n, *[1] * (x.dim() - 1))  # noqa: E731
        new, rest = [many(s[x]) for x in ("q", "k", "v")], [many(s[x]) for x in ("prefix", "steps", "gamma")]
        cache = [to_gpu(x) if page else many(x) for x in s["cache"]]
        table = many(s["table"]) if page else None
        for window, sinks in {w[:2] for w in S.windows(form)}:
            for kv_chunk in ranges:
                kw = dict(block_size=B, max_ref=L, max_prefix_len=max(S.PREFIXES), page_size=page, kv_chunk=kv_chunk,
                          window=window, sinks=sinks)
                if form == "fp4":
                    out, lse = binding.verify_attention_fp4(*new, binding.Fp4Cache(*cache), table, *rest, **kw)
                else:
                    out, lse = binding.verify_attention(*new, *cache, table, *rest, **kw)
                bits = out.view(torch.int16).view(n, -1), lse.view(torch.int32).view(n, -1)
                assert all(torch.equal(x, x[:1].expand_as(x)) for x in bits), "copies differ"
                same(f64(out[:b]), f64(lse[:b]).transpose(0, 2, 1), *step_oracle(form, B, L, hq, hkv, d, page, wild, window, sinks), d,
                     max(S.PREFIXES) + B + L, True)


@pytest.mark.parametrize("form", ["bf16", "fp4"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,L,hq,hkv", S.STEPS)
@pytest.mark.parametrize("page", [0, 24])
def test_verifications(form, d, B, L, hq, hkv, page):
    steps(form, B, L, hq, hkv, d, page, False, (0, 64))


@pytest.mark.parametrize("form", ["bf16", "fp4"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,L,hq,hkv", S.STEPS[:2])
@pytest.mark.parametrize("page", [0, 16])
def test_verifications_with_values_that_are_not_finite(form, d, B, L, hq, hkv, page):
    steps(form, B, L, hq, hkv, d, page, True, (0, 64))
