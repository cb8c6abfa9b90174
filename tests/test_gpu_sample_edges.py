"""Sampling where rows are unlike most: the largest logits outside a row's 16-byte
vectors, zeros of one sign only, counts past 16 bits beside NaN, long vocabularies.

Tokens and kept counts equal the float64 oracle's.  A probability is one rounding to
fp32 (2^-24) of a quotient whose sum is off by half a fixed-point unit a token, V *
2^-(S + 1) with S = 62 - ceil(log2 V), of the largest weight at most; 2^-40 holds the
oracle's own roundings."""

import numpy as np
import pytest
import torch

import oracle.sampling as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def run(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    from paper_2606_02544_amd import binding
    token, prob, kept = binding.sample(x.cuda(), u.cuda(), temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    want = ref.sample(x.cpu().double().numpy(), u.numpy(), np.float32(temperature), top_k, np.float32(top_p), np.float32(min_p))
    assert kept.cpu().tolist() == want[2].tolist()
    assert token.cpu().tolist() == want[0].tolist()
    V = x.shape[1]
    sums = V * 2.0 ** -(63 - (V - 1).bit_length())
    np.testing.assert_allclose(prob.cpu().numpy(), want[1], rtol=2.0 ** -24 + sums + 2.0 ** -40, atol=0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1025, 5001, 50257, 151643, 155651])
@pytest.mark.parametrize("k", [1, 2, 3, 50])
def test_largest_logits_outside_the_vectors(dtype, V, k):
    """Rows of an odd length start at every alignment: the largest logits are the
    first and the last of a row, the others far apart."""
    g = torch.Generator().manual_seed(V + k)
    x = torch.randn((9, V), generator=g).clamp(max=3.0)
    at = torch.linspace(V // 60, V - V // 60, k + 2).long()
    x[:, at] = 20.0 - 0.125 * torch.arange(k + 2)
    x[:, V - 1] = 22.0
    x[4:, 0] = 21.0
    u = torch.rand(9, generator=g)
    run(x.to(DT[dtype]), u, 4.0, k)
    run(x.to(DT[dtype]), u, 4.0, k, 0.9)
    run(x.to(DT[dtype]), u, 4.0, k, 1.0, 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1025, 5003, 151936, 200003])
def test_negative_zeros_without_positive_ones(dtype, V):
    """Every zero of a row is -0: all entries, the largest one with the rest near or far
    below, some below positive ones, and none but entries that are never kept beside."""
    g = torch.Generator().manual_seed(V)
    x = -torch.randn((7, V), generator=g).abs() - 0.25
    x[0] = -0.0
    x[1, V // 3] = -0.0
    x[2] -= 60.0
    x[2, 5::701] = -0.0
    x[3, ::5] = -0.0
    x[3, 1::5] = 1.5
    x[4] = float("-inf")
    x[4, 3::11] = -0.0
    x[5] = torch.randn(V, generator=g)
    x[5, 7::13] = -0.0
    x[6] = float("nan")
    x[6, ::2] = -0.0
    assert not (x.view(torch.int32) == 0).any()
    x, u = x.to(DT[dtype]), torch.rand(7, generator=g)
    run(x, u)
    run(x, u, 1.0, 0, 0.9)
    run(x, u, 0.7, 1000, 0.8)
    run(x, u, 1.0, 0, 0.95, 0.01)
    run(x, u, 0.0)


@pytest.mark.parametrize("V", [65537, 151936, 2 ** 22])
@pytest.mark.parametrize("n", [65535, 65536, 65537, 131072])
def test_counts_of_negative_zeros_past_16_bits(V, n):
    g = torch.Generator().manual_seed(n)
    x = -torch.randn((2, V), generator=g).abs() - 0.25
    x[:, torch.randperm(V, generator=g)[:n]] = -0.0
    x[1, V - 1] = 1.0
    x, u = x.bfloat16(), torch.rand(2, generator=g)
    run(x, u)
    run(x, u, 1.0, 0, 0.3)


def patterns(*parts):
    """A bf16 row of the given (16-bit pattern, count) parts."""
    bits = torch.cat([torch.full((n,), p - 65536 if p > 32767 else p, dtype=torch.int16) for p, n in parts])
    return bits.view(torch.bfloat16)


@pytest.mark.parametrize("nan,count", [(0xff81, 1), (0xff81, 2), (0xff81, 70000), (0xffff, 9), (0x7f81, 1), (0xffc0, 65537)])
@pytest.mark.parametrize("equal", [0x3f80, 0x3f81, 0x8000, 0xff80])
def test_counts_past_16_bits_beside_nan(nan, count, equal):
    """NaN of any payload is never kept, and hides no count that wraps: 70000 and 140000
    equal entries beside it, in the order of their patterns and in any."""
    g = torch.Generator().manual_seed(equal + count)
    for n in (70000, 140000):
        row = patterns((equal, n), (nan, count), (0xbf80, 3000), (0x3f00, 7))
        x = torch.stack([row, row[torch.randperm(len(row), generator=g)]] * 2)
        u = torch.tensor([0.0, 0.5, 0.25, 0.9999])
        run(x, u)
        run(x, u, 0.5, 0, 0.9)
        run(x, u, 1.0, 2000, 0.9)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [2 ** 18, 2 ** 20 - 3, 2 ** 22])
def test_sums_of_long_vocabularies(dtype, V):
    """A tail of equal tokens whose weights, near an odd number of half units, are all
    rounded one way: in fp32 the sums are off by nearly as much as they may be (2e-6 of
    the largest weight at 2^22)."""
    unit = 2.0 ** -(62 - (V - 1).bit_length())
    x = torch.empty((4, V))
    for i, w in enumerate((0.45, 0.55, 1.45, 2.55)):
        x[i] = float(np.log(w * unit))
    x[:, V // 2] = 0.0
    x = x.to(DT[dtype])
    u = torch.tensor([0.0, 0.5, 0.25, 0.75])
    run(x, u)
    run(x, u, 1.0, 0, 0.5)
