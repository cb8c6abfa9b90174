"""What simsd_fp4_values asks of a cache's scales: nothing of their place, whatever the
head's size (CPU; no kernel is launched)."""

import ctypes

import pytest

from paper_2606_02544_amd import binding
from paper_2606_02544_amd.binding import Fp4Pointers, Fp4ValuesDesc
from test_operator_checks import FAKE, chunk_desc, no_gpu  # noqa: F401 (no_gpu: a fixture)

HIP, ALIGNMENT = 7, 4                                          # (past the checks there is no device here)


def values(d, at, strides):
    desc = Fp4ValuesDesc(num=2, tokens=3, num_kv_heads=4, head_dim=d, cache_stride_seq=6 * d, cache_stride_token=2 * d,
                         cache_stride_head=(d // 2 + 15) // 16 * 16)
    cache = Fp4Pointers(0x10000, 0x20000, at, at + 0x1001, *strides)
    return binding.lib().simsd_fp4_values(ctypes.byref(desc), ctypes.byref(cache), FAKE, ctypes.c_void_p(0x90000), None)


@pytest.mark.parametrize("d", range(32, 513, 32))
def test_scales_at_any_place(no_gpu, d):  # noqa: F811
    for at in (0x30000, 0x30001, 0x30002, 0x30003, 0x30100):
        for strides in ((1000, 100, d // 32), (1001, 103, 17), (0, 0, 0)):
            assert values(d, at, strides) == HIP, (at, strides)
    assert values(d, 0x30000, (-1, 0, 0)) == 2 and values(d, 0x30000, (0, 2 ** 48 + 1, 0)) == 2


def test_an_attention_reads_them_as_words(no_gpu):  # noqa: F811
    def run(**kw):
        c = dict(k=0x10000, v=0x10000, k_scales=0x20004, v_scales=0x20004, scale_stride_seq=512, scale_stride_token=16, scale_stride_head=4)
        c.update(kw)
        return binding.lib().simsd_chunk_attention_fp4(ctypes.byref(chunk_desc(head_dim=128)), 8, 2, FAKE, ctypes.byref(Fp4Pointers(**c)),
                                                       *[FAKE] * 6, 0, None)

    assert run() != ALIGNMENT
    for kw in (dict(k_scales=0x20002), dict(v_scales=0x20001), dict(scale_stride_token=6), dict(scale_stride_seq=1)):
        assert run(**kw) == ALIGNMENT, kw


def test_outputs_past_one_launch(no_gpu):  # noqa: F811
    """More than 2^37 - 8192 elements (256 GiB) of keys or values are refused by their size."""
    def run(num, tokens, heads, d):
        desc = Fp4ValuesDesc(num=num, tokens=tokens, num_kv_heads=heads, head_dim=d, cache_stride_seq=0, cache_stride_token=0,
                             cache_stride_head=0)
        cache = Fp4Pointers(0x10000, 0x20000, 0x30000, 0x40000, 0, 0, 0)
        return binding.lib().simsd_fp4_values(ctypes.byref(desc), ctypes.byref(cache), FAKE, ctypes.c_void_p(0x90000), None)

    for d in range(32, 513, 32):
        rows = (2 ** 37 - 8192) // d
        heads = next(h for h in range(1, 4096) if rows // h < 2 ** 31)
        tokens = rows // heads                                 # the most that are taken
        assert run(1, tokens, heads, d) == HIP and run(1, tokens + 1, heads, d) == 2, d
    assert run(2 ** 20, 2 ** 16, 1, 512) == 2 and run(2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1, 32) == 2
