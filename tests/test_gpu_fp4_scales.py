"""The largest scales of a 4-bit cache in its attentions, on the GPU against the float64
oracle.

At 2^126 (a scale byte of 253) the codes 4 and 6 are past bf16's range and infinite, at
2^127 (254) those from 2 on; the others are numbers like any.  The queries are zero, so
that every key a row sees has the same weight and a sum holds one such number, below
2^128, at most.  Tolerance: the weights' and the output's rounding to bf16 and n
additions in fp32, with scores that are exact."""

import numpy as np
import pytest
import torch

import oracle.window as ref
import test_gpu_fp4 as chunks
import test_gpu_verify_span as steps

pytestmark = pytest.mark.gpu


def held(cache):
    """The cache's values as bf16 holds them."""
    return [np.where(np.abs(x) >= 2.0 ** 128, np.copysign(np.inf, x), x) for x in chunks.decoded(cache)]


def compare(got, want, size, n):
    wild = ~np.isfinite(want)
    assert np.array_equal(got[wild], want[wild], equal_nan=True)
    assert np.isfinite(got[~wild]).all()
    got, want, size = got[~wild], want[~wild], size[~wild]
    err, tol = np.abs(got - want), (n * 2.0 ** -23 + 2.0 ** -8) * size + 2.0 ** -8 * np.abs(want)
    assert (err <= tol).all(), (int((err > tol).sum()), float((err - tol).max()))
    return int(wild.sum()), float(np.abs(want).max())


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("kv_chunk", [0, 64])
@pytest.mark.parametrize("tokens", [61, 1000, 2000, 3000, 4000, 8000])
def test_chunks(d, kv_chunk, tokens):
    """In tiles that every row sees whole and in such that some rows do not see, in row
    blocks of every size (which go by `tokens`, most of them of no sequence)."""
    s = chunks.make([(60, 350), (1, 300)], 16, 2, d, 16, 31, pad=tokens - 61)
    s["q"].zero_()
    # sequence, key, KV head, group of 32 dims, scale; a head and group once a sequence
    for b, t, head, group, scale in ((0, 10, 0, 0, 253), (0, 320, 1, 0, 254), (0, 320, 0, 1, 253), (0, 345, 1, 1, 254),
                                     (1, 299, 0, 0, 254), (1, 298, 0, 1, 253), (1, 3, 1, 0, 253), (1, 290, 1, 1, 254)):
        s["cache"][3][int(s["table"][b, t // 16]), t % 16, head, group] = scale
    k, v = held(s["cache"])
    for window, sinks in ((0, 0), (100, 12), (345, 0)):
        out, lse = chunks.call(s, mask_block=1, kv_chunk=kv_chunk, window=window, sinks=sinks)
        with np.errstate(invalid="ignore"):
            want, _, size, _ = ref.chunk_attention(chunks.f64(s["q"][:61]), k, v, s["table"], s["starts"].tolist(),
                                                   s["kv"].tolist(), mask_block=1, window=window, sinks=sinks, page=16)
        wild, largest = compare(chunks.f64(out[:61]), want, size, 350)
        assert wild > 0 and largest > 2.0 ** 117               # (2^126 / 350 and more)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,L,hq", [(4, 4, 4), (8, 8, 32), (32, 32, 8)])
@pytest.mark.parametrize("copies", [1, 24, 48, 96])
def test_verifications(d, B, L, hq, copies):
    """Among the sinks, at the window's beginning and at the prefix's end; copies of the
    batch take the row blocks from the smallest to the largest."""
    s = steps.make("fp4", [300, 90], B, L, hq, 2, d, 16, 7, mode="full")
    s["q"].zero_()
    for b, t, head, group, scale in ((0, 2, 0, 0, 253), (0, 222, 1, 0, 254), (0, 299, 0, 1, 254), (0, 260, 1, 1, 253),
                                     (1, 1, 0, 0, 254), (1, 12, 1, 0, 253), (1, 89, 0, 1, 253), (1, 50, 1, 1, 254)):
        s["cache"][3][int(s["table"][b, t // 16]), t % 16, head, group] = scale
    k, v = held(s["cache"])
    many = dict(s, **{x: s[x].repeat(copies, *[1] * (s[x].dim() - 1)) for x in ("q", "k", "v", "table", "prefix", "steps", "gamma")})
    f = lambda x: x.double().cpu().numpy()  # noqa: E731
    for window, sinks in ((0, 0), (80, 5)):
        with np.errstate(invalid="ignore"):
            want, _, size, _ = ref.verify_attention(f(s["q"]), f(s["k"]), f(s["v"]), k, v, s["table"], s["prefix"],
                                                    s["steps"].numpy(), s["gamma"], window=window, sinks=sinks, page=16)
        for kv_chunk in (0, 64):
            out, lse = steps.call(many, window=window, sinks=sinks, kv_chunk=kv_chunk)
            assert torch.equal(out.view(copies, -1)[:1].expand(copies, -1).isnan(), out.view(copies, -1).isnan())
            wild, largest = compare(f(out[:2]), want, size, 300 + B + L)
            assert wild > 0 and largest > 2.0 ** 117
            wild, largest = compare(f(out[-2:]), want, size, 300 + B + L)
