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
