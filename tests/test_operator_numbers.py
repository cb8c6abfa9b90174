"""Numbers that a descriptor's 32-bit fields cannot hold are refused by the operators'
entry points (CPU; nothing is launched)."""

import contextlib
import types

import pytest
import torch

from paper_2606_02544_amd import binding

BF, I32 = torch.bfloat16, torch.int32
WRAPPED = [2 ** 31, 2 ** 32, 2 ** 32 + 1, 2 ** 32 + 20, -2 ** 32 + 20, -2 ** 31 - 1, 2 ** 64 + 1]


@pytest.fixture(autouse=True)
def launch_on_the_host(monkeypatch):
    monkeypatch.setattr(binding, "_Launch",
                        lambda device, stream: contextlib.nullcontext(types.SimpleNamespace(handle=None)))


def z(*shape, dtype=BF):
    return torch.zeros(shape, dtype=dtype)


@pytest.mark.parametrize("x", WRAPPED)
def test_sample(x):
    with pytest.raises(ValueError, match="top_k"):
        binding.sample(z(3, 9), z(3, dtype=torch.float32), top_k=x)


@pytest.mark.parametrize("x", WRAPPED)
@pytest.mark.parametrize("name", ["max_q_len", "max_kv_len", "mask_block", "kv_chunk", "page_size"])
def test_chunk_attention(name, x):
    kw = dict(max_q_len=6, max_kv_len=20, mask_block=1, kv_chunk=0, page_size=0)
    kw[name] = x
    with pytest.raises(ValueError, match=f"{name}|holds 20|page_size is"):
        binding.chunk_attention(z(6, 4, 64), z(2, 20, 2, 64), z(2, 20, 2, 64), None, z(3, dtype=I32),
                                z(2, dtype=I32), **kw)


@pytest.mark.parametrize("x", WRAPPED)
@pytest.mark.parametrize("name", ["max_kv_len", "page_size"])
def test_append(name, x):
    """(A length of -2^32 + 20 would pass for none here and for 20 in the library.)"""
    kw = dict(max_kv_len=20, page_size=0)
    kw[name] = x
    with pytest.raises(ValueError, match=f"{name}|holds 20|page_size is"):
        binding.rotary_append(z(6, 4, 64), z(6, 2, 64), z(6, 2, 64), z(2, 20, 2, 64), z(2, 20, 2, 64), None,
                              z(3, dtype=I32), z(2, dtype=I32), z(32, dtype=torch.float64), **kw)


@pytest.mark.parametrize("x", WRAPPED)
def test_frequencies(x):
    with pytest.raises(ValueError, match="original_context"):
        binding.rope_frequencies(64, 10000.0, scaling="yarn", factor=2.0, original_context=x, device="cpu")
    with pytest.raises(ValueError, match="rotary_dim"):
        binding.rope_frequencies(x, 10000.0, device="cpu")


@pytest.mark.parametrize("scale", [1e-46, -1e-50, 5e-324])
def test_scale_that_vanishes(scale):
    """(0 stands for the default.)"""
    with pytest.raises(ValueError, match="scale"):
        binding.chunk_attention(z(6, 4, 64), z(2, 20, 2, 64), z(2, 20, 2, 64), None, z(3, dtype=I32), z(2, dtype=I32),
                                max_q_len=6, max_kv_len=20, scale=scale)
