"""Values of a 4-bit cache for heads of every size, with scales at any address and
stride, on the GPU; exact."""

import numpy as np
import pytest
import torch

import oracle.fp4 as fp4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [32, 64, 96, 160, 192, 224, 256, 384, 512])
@pytest.mark.parametrize("offset,gap", [(0, 0), (1, 0), (2, 1), (3, 5)])
def test_heads_and_places_of_scales(d, offset, gap):
    """`offset`: bytes before the first scale; `gap`: between one head's scales and the next's."""
    from paper_2606_02544_amd import binding
    n, tokens, hkv, groups = 3, 7, 2, d // 32
    g = torch.Generator().manual_seed(d + offset)
    codes = [torch.randint(0, 256, (n, tokens, hkv, d // 2), generator=g, dtype=torch.uint8) for _ in range(2)]
    scales = []
    for _ in range(2):
        row = groups + gap
        space = torch.randint(0, 256, (offset + n * tokens * hkv * row,), generator=g, dtype=torch.uint8).cuda()
        scales.append(torch.as_strided(space, (n, tokens, hkv, groups), (tokens * hkv * row, hkv * row, row, 1), offset))
    k, v = binding.fp4_values(binding.Fp4Cache(codes[0].cuda(), codes[1].cuda(), *scales))
    for got, c, s in zip((k, v), codes, scales):
        with np.errstate(over="ignore"):                       # (past bf16's range, infinite)
            want = torch.from_numpy(fp4.decode(c.numpy(), s.cpu().numpy()).astype(np.float32)).bfloat16()
        got = got.cpu()
        assert got.shape == (n, tokens, hkv, d)
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[~got.isnan()], want[~want.isnan()])
