"""The oracles of rotary positions, chunk attention and sampling against other ways to
the same numbers (CPU)."""

import math

import numpy as np
import pytest
import torch

from oracle import chunk, rotary, sampling
from oracle.rope import rotate as verify_rotate


def test_rotary_as_complex_numbers():
    g = np.random.RandomState(1)
    x = g.randn(5, 3, 20)
    pos = np.array([0, 1, 7, 100, 12345])
    freq, _ = rotary.frequencies(12, 10000.0)
    turn = 1.5 * np.exp(1j * pos[:, None] * freq)[:, None]
    half = (x[..., :6] + 1j * x[..., 6:12]) * turn
    want = np.concatenate([half.real, half.imag, x[..., 12:]], -1)
    np.testing.assert_allclose(rotary.rotate(x, pos, freq, factor=1.5), want, atol=1e-11)
    pairs = (x[..., 0:12:2] + 1j * x[..., 1:12:2]) * turn
    want = np.concatenate([np.stack([pairs.real, pairs.imag], -1).reshape(5, 3, 12), x[..., 12:]], -1)
    np.testing.assert_allclose(rotary.rotate(x, pos, freq, interleaved=True, factor=1.5), want, atol=1e-11)


def test_rotary_as_the_verification_rotates():
    g = np.random.RandomState(2)
    x = g.randn(4, 2, 64)
    pos = np.array([3, 9, 200, 201])
    freq, _ = rotary.frequencies(64, 10000.0)
    want = np.stack([verify_rotate(x[i], np.full(x[i].shape[:-1], pos[i]), 10000.0) for i in range(4)])
    np.testing.assert_allclose(rotary.rotate(x, pos, freq), want, atol=1e-12)


@pytest.mark.parametrize("mask_block", [0, 1, 3, 8, 100])
def test_chunk_as_dense_masked_attention(mask_block):
    g = np.random.RandomState(3)
    lens = [(5, 9), (7, 7), (1, 20), (4, 2)]
    q = g.randn(17, 4, 8)
    k, v = g.randn(4, 20, 2, 8), g.randn(4, 20, 2, 8)
    starts = np.cumsum([0] + [n for n, _ in lens])
    out, lse, _, _ = chunk.chunk_attention(q, k, v, None, starts, [m for _, m in lens], mask_block=mask_block)
    for b, (n, m) in enumerate(lens):
        pos = torch.arange(m - n, m)
        key = torch.arange(20)
        block = (lambda p: torch.div(p, mask_block, rounding_mode="floor")) if mask_block else (lambda p: p * 0)
        sees = (key < m) & (block(key) <= block(pos)[:, None]) & (pos >= 0)[:, None]
        for h in range(4):
            x = torch.from_numpy(q[starts[b]:starts[b] + n, h]) @ torch.from_numpy(k[b, :, h // 2]).T / math.sqrt(8)
            x = x.masked_fill(~sees, -math.inf)
            want = torch.nan_to_num(torch.softmax(x, -1)) @ torch.from_numpy(v[b, :, h // 2])
            np.testing.assert_allclose(out[starts[b]:starts[b] + n, h], want.numpy(), atol=1e-12)
            np.testing.assert_allclose(lse[h, starts[b]:starts[b] + n], torch.logsumexp(x, -1).numpy(), atol=1e-12)


def test_chunk_as_the_verification_without_drafts():
    """A block without drafts, all of it undrafted: bidirectional attention over the
    prefix and the block (SDPA in float64)."""
    g = np.random.RandomState(4)
    q, k, v = g.randn(6, 2, 8), g.randn(1, 30, 1, 8), g.randn(1, 30, 1, 8)
    out = chunk.chunk_attention(q, k, v, None, [0, 6], [30], mask_block=0)[0]
    t = lambda x: torch.from_numpy(x)  # noqa: E731
    want = torch.nn.functional.scaled_dot_product_attention(
        t(q).transpose(0, 1), t(k[0]).transpose(0, 1).expand(2, 30, 8), t(v[0]).transpose(0, 1).expand(2, 30, 8))
    np.testing.assert_allclose(out, want.transpose(0, 1).numpy(), atol=1e-12)


def test_sampling_frequencies():
    """Tokens drawn with evenly spread numbers come out in proportion to the kept
    softmax."""
    x = np.array([1.0, 3.0, -2.0, 3.0, 0.5, -np.inf, np.nan, 2.0])
    u = (np.arange(40000) + 0.5) / 40000
    for T, k, p, m in ((1.0, 0, 1.0, 0.0), (0.7, 3, 1.0, 0.0), (1.0, 0, 0.8, 0.0), (1.0, 0, 1.0, 0.2), (2.0, 4, 0.9, 0.3)):
        w = np.where(np.isfinite(x), np.exp((np.nan_to_num(x, nan=-1e9, neginf=-1e9) - 3.0) / T), 0.0)
        order = sorted(range(8), key=lambda i: (-w[i], i))
        keep = [i for i in order if w[i] > 0][:k or None]
        total, run, cut = sum(w[i] for i in keep), 0.0, []
        for i in keep:
            if run < p * total or not cut:
                cut.append(i)
            run += w[i]
        cut = [i for i in cut if w[i] >= m]
        z = sum(w[i] for i in cut)
        draws = [sampling.sample_row(x, y, T, k, p, m) for y in u]
        assert {d[2] for d in draws} == {len(cut)}
        for i in range(8):
            share = np.mean([d[0] == i for d in draws])
            assert abs(share - (w[i] / z if i in cut else 0.0)) <= 1.0 / 40000
            assert all(abs(d[1] - w[i] / z) < 1e-12 for d in draws if d[0] == i)


def test_sampling_edges():
    row = lambda x, *a: sampling.sample_row(np.array(x, float), *a)  # noqa: E731
    assert row([-np.inf, np.nan], 0.5) == (-1, 0.0, 0)
    assert row([0.0, 5.0, 5.0], 0.9, 0.0) == (1, 1.0, 1)
    assert row([-0.0, 0.0, -0.0], 0.5)[0] == 1
    assert row([np.inf, 1.0, np.inf], 0.7)[0] == 2
    assert row([0.0, 800.0], 0.999999)[2] == 1 and row([0.0, 600.0], 0.999999)[2] == 2
