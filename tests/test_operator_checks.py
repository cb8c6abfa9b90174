"""What rotary positions, chunk attention and sampling refuse, and the layout of their
descriptors (CPU; no kernel is launched: every call fails a check)."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

import oracle.rotary
from paper_2606_02544_amd import binding
from paper_2606_02544_amd.binding import ChunkDesc, RotaryDesc, SampleDesc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BF, I32 = torch.bfloat16, torch.int32
FAKE = ctypes.c_void_p(0x10000)     # aligned, never dereferenced
NULL = None


@pytest.fixture
def no_gpu():
    if torch.cuda.is_available():
        pytest.skip("fake pointers only without a visible GPU")


# --- descriptors ------------------------------------------------------------
@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
def test_descriptor_layouts(tmp_path):
    kinds = {"simsd_rotary_desc": RotaryDesc, "simsd_chunk_desc": ChunkDesc, "simsd_sample_desc": SampleDesc}
    lines = []
    for name, cls in kinds.items():
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
        lines.append(f'printf("%zu\\n", sizeof({name}));')
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "simsd.h"\nint main(void) {' + "\n".join(lines) + "return 0; }")
    exe = str(tmp_path / "layout")
    subprocess.run(["gcc", "-I" + os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    want = []
    for cls in kinds.values():
        want += [getattr(cls, f[0]).offset for f in cls._fields_] + [ctypes.sizeof(cls)]
    assert got == want


def rotary_desc(**kw):
    d = dict(num_tokens=4, num_q_heads=4, num_kv_heads=2, head_dim=64, rotary_dim=64, interleaved=0, batch=2,
             max_kv_len=32, page_size=0, max_pages_per_seq=0, num_pages=0, attn_factor=1.0, q_stride_token=256,
             q_stride_head=64, k_stride_token=128, k_stride_head=64, v_stride_token=128, v_stride_head=64,
             q_out_stride_token=256, q_out_stride_head=64, k_out_stride_token=128, k_out_stride_head=64,
             cache_stride_seq=4096, cache_stride_token=128, cache_stride_head=64, dtype=1)
    d.update(kw)
    return RotaryDesc(**d)


ROTARY_ARGS = ("q", "k", "positions", "freq", "q_out", "k_out")
APPEND_ARGS = ("q", "k", "v", "positions", "freq", "q_out", "k_cache", "v_cache", "block_table", "q_starts", "kv_lens")


def rotary(desc, **over):
    fn = binding.lib().simsd_rotary
    return fn(desc and ctypes.byref(desc), *(over.get(n, FAKE) for n in ROTARY_ARGS), None)


def append(desc, **over):
    fn = binding.lib().simsd_rotary_append
    return fn(desc and ctypes.byref(desc), *(over.get(n, FAKE) for n in APPEND_ARGS), None)


@pytest.mark.parametrize("field,value,status", [
    ("num_tokens", -1, 2), ("num_tokens", 2 ** 25, 2), ("num_q_heads", -1, 2), ("head_dim", 0, 3), ("head_dim", 68, 3),
    ("head_dim", 520, 3), ("rotary_dim", 0, 2), ("rotary_dim", 7, 2), ("rotary_dim", 66, 2), ("interleaved", 2, 2),
    ("attn_factor", 0.0, 2), ("attn_factor", float("nan"), 2), ("attn_factor", float("inf"), 2), ("dtype", 7, 3),
    ("q_stride_token", -8, 2), ("q_stride_head", 12, 4), ("k_stride_token", 2 ** 41, 2), ("q_out_stride_head", 32, 2),
    ("q_out_stride_token", 64, 2), ("k_out_stride_token", 0, 2)])
def test_rotary_descriptor(no_gpu, field, value, status):
    assert rotary(rotary_desc(**{field: value})) == status
    assert binding.lib().simsd_last_error()


@pytest.mark.parametrize("field,value,status", [
    ("num_kv_heads", 0, 2), ("batch", 0, 2), ("batch", 70000, 2), ("max_kv_len", -1, 2), ("page_size", -1, 2),
    ("v_stride_token", 4, 4), ("cache_stride_token", 4, 4), ("cache_stride_seq", -8, 2), ("num_pages", -1, 2),
    ("max_pages_per_seq", 1, 2)])
def test_append_descriptor(no_gpu, field, value, status):
    paged = field in ("num_pages", "max_pages_per_seq")
    base = dict(page_size=16, max_pages_per_seq=2, num_pages=9) if paged else {}
    assert append(rotary_desc(**{**base, field: value})) == status


def test_rotary_pointers(no_gpu):
    d = rotary_desc()
    assert rotary(None) == 1 and append(None) == 1
    for n in ROTARY_ARGS:
        assert rotary(d, **{n: NULL}) == 1, n
    for n in ("q", "k", "v", "freq", "q_out", "k_cache", "v_cache", "q_starts", "kv_lens"):
        assert append(d, **{n: NULL}) == 1, n
    assert append(rotary_desc(page_size=16, max_pages_per_seq=2, num_pages=4), block_table=NULL) == 1
    for n, at in (("q", 8), ("k_out", 8), ("freq", 4), ("positions", 2)):
        assert rotary(d, **{n: ctypes.c_void_p(0x10000 + at)}) == 4, n
    for n, at in (("v", 8), ("k_cache", 8), ("freq", 4), ("positions", 2), ("q_starts", 1), ("kv_lens", 2)):
        assert append(d, **{n: ctypes.c_void_p(0x10000 + at)}) == 4, n
    # in place with other strides
    wide = rotary_desc(q_stride_token=512)
    assert rotary(wide) == 2 and append(wide) == 2
    # nothing to do
    none = rotary_desc(num_tokens=0)
    assert rotary(none, q=NULL, k=NULL, positions=NULL) == 0 and append(none, k=NULL) == 0


def chunk_desc(**kw):
    d = dict(num_tokens=4, batch=2, num_q_heads=4, num_kv_heads=2, head_dim=64, max_q_len=3, max_kv_len=32,
             mask_block=1, page_size=0, max_pages_per_seq=0, kv_chunk=0, cache_stride_seq=4096,
             cache_stride_token=128, cache_stride_head=64, scale=0.0, dtype=1)
    d.update(kw)
    return ChunkDesc(**d)


CHUNK_ARGS = ("q", "k_cache", "v_cache", "block_table", "q_starts", "kv_lens", "out", "lse")


def chunk(desc, ws=FAKE, nbytes=1 << 40, **over):
    fn = binding.lib().simsd_chunk_attention
    return fn(desc and ctypes.byref(desc), *(over.get(n, FAKE) for n in CHUNK_ARGS), ws, nbytes, None)


@pytest.mark.parametrize("field,value,status", [
    ("num_tokens", -1, 2), ("num_tokens", 2 ** 24, 2), ("batch", 0, 2), ("batch", 65536, 2), ("num_q_heads", 5, 2),
    ("num_kv_heads", 0, 2), ("num_q_heads", 34, 3), ("head_dim", 96, 3), ("max_q_len", -1, 2), ("max_kv_len", -1, 2),
    ("max_kv_len", 2 ** 30 + 1, 2), ("mask_block", -1, 2), ("page_size", -1, 2), ("page_size", 16, 2), ("kv_chunk", 32, 2),
    ("kv_chunk", -64, 2), ("cache_stride_head", 4, 4), ("cache_stride_token", -8, 2), ("scale", -1.0, 2),
    ("scale", float("nan"), 2), ("dtype", 9, 3)])
def test_chunk_descriptor(no_gpu, field, value, status):
    d = chunk_desc(**{field: value})
    assert chunk(d) == status
    assert binding.lib().simsd_last_error()
    assert binding.chunk_workspace_size(d) == 0


def test_chunk_pointers_and_workspace(no_gpu):
    assert chunk(None) == 1
    d = chunk_desc()
    for n in ("q", "k_cache", "v_cache", "q_starts", "kv_lens", "out"):
        assert chunk(d, **{n: NULL}) == 1, n
    assert chunk(chunk_desc(page_size=16, max_pages_per_seq=2), block_table=NULL) == 1
    for n in ("q", "k_cache", "out"):
        assert chunk(d, **{n: ctypes.c_void_p(0x10008)}) == 4, n
    assert chunk(d, lse=ctypes.c_void_p(0x10002)) == 4
    split = chunk_desc(max_kv_len=256, kv_chunk=64)
    size = binding.chunk_workspace_size(split)
    assert size == 4 * 4 * 4 * (64 + 2) * 4                    # ranges, tokens, heads, output and two numbers
    assert chunk(split, ws=NULL, nbytes=0) == 5
    assert chunk(split, nbytes=size - 1) == 5
    assert chunk(split, ws=ctypes.c_void_p(0x10004), nbytes=size) == 4
    assert binding.chunk_workspace_size(chunk_desc(max_kv_len=256, kv_chunk=256)) == 0
    assert chunk(chunk_desc(num_tokens=0), q=NULL, ws=NULL, nbytes=0) == 0


def sample_desc(**kw):
    d = dict(rows=3, vocab=100, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, dtype=1)
    d.update(kw)
    return SampleDesc(**d)


SAMPLE_ARGS = ("logits", "uniforms", "temperatures", "top_ks", "top_ps", "min_ps", "token", "prob", "kept")


def sample(desc, **over):
    return binding.lib().simsd_sample(desc and ctypes.byref(desc), *(over.get(n, FAKE) for n in SAMPLE_ARGS), None)


@pytest.mark.parametrize("field,value,status", [
    ("rows", -1, 2), ("rows", 2 ** 22, 2), ("vocab", 0, 2), ("vocab", 2 ** 22 + 1, 2), ("temperature", -0.5, 2),
    ("temperature", float("inf"), 2), ("temperature", float("nan"), 2), ("top_k", -1, 2), ("top_p", -0.1, 2),
    ("top_p", 1.5, 2), ("top_p", float("nan"), 2), ("min_p", -0.1, 2), ("min_p", 2.0, 2), ("dtype", 5, 3)])
def test_sample_descriptor(no_gpu, field, value, status):
    assert sample(sample_desc(**{field: value})) == status


def test_sample_pointers(no_gpu):
    assert sample(None) == 1
    for n in ("logits", "uniforms", "token"):
        assert sample(sample_desc(), **{n: NULL}) == 1, n
    assert sample(sample_desc(), logits=ctypes.c_void_p(0x10001)) == 4
    assert sample(sample_desc(dtype=0), logits=ctypes.c_void_p(0x10002)) == 4
    assert sample(sample_desc(), top_ks=ctypes.c_void_p(0x10002)) == 4
    assert sample(sample_desc(rows=0), logits=NULL) == 0


# --- frequencies --------------------------------------------------------------
@pytest.mark.parametrize("rot,theta", [(2, 10000.0), (64, 10000.0), (128, 1e6), (96, 500000.0)])
@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
def test_frequencies(rot, theta, scaling):
    if scaling == "ntk" and rot == 2:
        pytest.skip("refused")
    for factor, context, fast, slow in ((1.0, 4096, 32.0, 1.0), (8.0, 4096, 32.0, 1.0), (4.0, 64, 40.0, 40.0), (16.0, 1, 2.0, 0.5)):
        kw = dict(scaling=scaling, factor=factor, original_context=context, beta_fast=fast, beta_slow=slow)
        freq, extra = binding.rope_frequencies(rot, theta, device="cpu", **kw)
        want, want_extra = oracle.rotary.frequencies(rot, theta, **kw)
        np.testing.assert_allclose(freq.numpy(), want, rtol=1e-13)
        assert extra == np.float32(want_extra)


def test_frequencies_refused():
    for kw in (dict(rotary_dim=3), dict(rotary_dim=0), dict(theta=1.0), dict(theta=float("nan")),
               dict(scaling="linear", factor=0.5), dict(scaling="ntk", rotary_dim=2),
               dict(scaling="yarn", original_context=0), dict(scaling="yarn", original_context=10, beta_fast=1.0, beta_slow=2.0)):
        args = dict(rotary_dim=64, theta=10000.0)
        args.update(kw)
        with pytest.raises(binding.SimsdError):
            binding.rope_frequencies(args.pop("rotary_dim"), args.pop("theta"), device="cpu", **args)
    with pytest.raises(ValueError, match="scaling"):
        binding.rope_frequencies(64, 10000.0, scaling="other", device="cpu")


# --- the binding's own checks ----------------------------------------------------
def base():
    z = lambda *s, dtype=BF: torch.zeros(s, dtype=dtype)  # noqa: E731
    return dict(q=z(6, 4, 64), k=z(6, 2, 64), v=z(6, 2, 64), pos=z(6, dtype=I32), freq=z(32, dtype=torch.float64),
                kc=z(2, 20, 2, 64), vc=z(2, 20, 2, 64), table=None, starts=z(3, dtype=I32), kv=z(2, dtype=I32), page=0)


def paged():
    a = base()
    a.update(kc=torch.zeros(9, 16, 2, 64, dtype=BF), vc=torch.zeros(9, 16, 2, 64, dtype=BF),
             table=torch.zeros(2, 2, dtype=I32), page=16)
    return a


def call_rotary(a, **kw):
    return binding.rotary(a["q"], a["k"], a["pos"], a["freq"], **kw)


def call_append(a, **kw):
    return binding.rotary_append(a["q"], a["k"], a["v"], a["kc"], a["vc"], a["table"], a["starts"], a["kv"], a["freq"],
                                 max_kv_len=20, page_size=a["page"], **kw)


def call_chunk(a, **kw):
    return binding.chunk_attention(a["q"], a["kc"], a["vc"], a["table"], a["starts"], a["kv"], max_q_len=6,
                                   max_kv_len=20, page_size=a["page"], **kw)


@pytest.mark.parametrize("call", [call_rotary, call_append, call_chunk])
@pytest.mark.parametrize("make", [base, paged])
def test_tensors_off_the_gpu(call, make):
    with pytest.raises(ValueError, match="on a GPU"):
        call(make())


@pytest.mark.parametrize("change,match", [
    (dict(q=torch.zeros(6, 4, 64)), "q_?k?|k must be"), (dict(q=torch.zeros(5, 4, 64, dtype=BF)), "shape|positions"),
    (dict(k=torch.zeros(6, 2, 32, dtype=BF)), "k has shape"), (dict(q=torch.zeros(6, 64, 4, dtype=BF).transpose(1, 2)), "unit stride"),
    (dict(q=torch.zeros(6, 64, dtype=BF)), "3-D"), (dict(pos=torch.zeros(6, dtype=torch.int64)), "positions"),
    (dict(pos=torch.zeros(7, dtype=I32)), "positions"), (dict(freq=torch.zeros(32)), "freq"), (dict(freq=[1.0]), "freq"),
    (dict(q=torch.zeros(6, 4, 64, dtype=torch.float16), k=torch.zeros(6, 2, 64, dtype=torch.float16)), "bfloat16 or float32")])
def test_rotary_tensors(change, match):
    a = base()
    a.update(change)
    with pytest.raises(ValueError, match=match):
        call_rotary(a)


def test_rotary_outputs():
    a = base()
    for kw in (dict(q_out=torch.zeros(6, 4, 64)), dict(k_out=torch.zeros(6, 4, 64, dtype=BF))):
        with pytest.raises(ValueError, match="_out"):
            call_rotary(a, **kw)
    a["q"] = None
    with pytest.raises(ValueError, match="q_out without q"):
        call_rotary(a, q_out=torch.zeros(6, 4, 64, dtype=BF))


CACHE = [
    (dict(kc=torch.zeros(2, 20, 2, 64)), "k_cache must be"), (dict(vc=torch.zeros(2, 20, 2, 32, dtype=BF)), "v_cache"),
    (dict(kc=torch.zeros(1, 20, 2, 64, dtype=BF), vc=torch.zeros(1, 20, 2, 64, dtype=BF)), "batch"),
    (dict(kc=torch.zeros(2, 19, 2, 64, dtype=BF), vc=torch.zeros(2, 19, 2, 64, dtype=BF)), "holds 19"),
    (dict(vc=torch.zeros(2, 30, 2, 64, dtype=BF)[:, :20]), "strides differ"),
    (dict(starts=torch.zeros(2, dtype=I32)), "q_starts"), (dict(starts=torch.zeros(3, dtype=torch.int64)), "q_starts"),
    (dict(kv=torch.zeros(2)), "kv_lens"), (dict(kv=torch.zeros(0, dtype=I32)), "kv_lens"), (dict(kv=None), "kv_lens"),
]
PAGES = [
    (dict(table=None), "block_table"), (dict(table=torch.zeros(2, 1, dtype=I32)), "too few pages"),
    (dict(table=torch.zeros(3, 2, dtype=I32)), "block_table"), (dict(table=torch.zeros(2, 2)), "block_table"),
    (dict(kc=torch.zeros(9, 8, 2, 64, dtype=BF), vc=torch.zeros(9, 8, 2, 64, dtype=BF)), "page_size"),
]


@pytest.mark.parametrize("call", [call_append, call_chunk])
@pytest.mark.parametrize("make,change,match", [(base, *c) for c in CACHE] + [(paged, *c) for c in PAGES])
def test_cache_tensors(call, make, change, match):
    a = make()
    a.update(change)
    with pytest.raises(ValueError, match=match):
        call(a)


def test_append_tensors():
    a = base()
    a["v"] = torch.zeros(6, 1, 64, dtype=BF)
    with pytest.raises(ValueError, match="v has shape"):
        call_append(a)
    a = base()
    a["kc"] = a["vc"] = torch.zeros(1, 1, 2, 64, dtype=BF).expand(2, 20, 2, 64)
    with pytest.raises(ValueError, match="expanded"):
        call_append(a)
    with pytest.raises(ValueError, match="positions"):
        call_append(base(), positions=torch.zeros(5, dtype=I32))


def test_chunk_tensors():
    a = base()
    a["q"] = torch.zeros(6, 8, 64, dtype=BF)[:, ::2]
    with pytest.raises(ValueError, match="contiguous"):
        call_chunk(a)
    for kw in (dict(out=torch.zeros(6, 4, 64)), dict(lse=torch.zeros(6, 4))):
        with pytest.raises(ValueError):
            call_chunk(base(), **kw)
    with pytest.raises(TypeError):
        call_chunk(base(), mask_block=1.5)


@pytest.mark.parametrize("kw,match", [
    (dict(logits=torch.zeros(3, 9, dtype=torch.float16)), "bfloat16 or float32"), (dict(logits=torch.zeros(3)), "2-D"),
    (dict(logits=torch.zeros(3, 18)[:, ::2]), "contiguous"), (dict(uniforms=torch.zeros(4)), "uniforms"),
    (dict(uniforms=torch.zeros(3, dtype=torch.float64)), "uniforms"), (dict(temperature=torch.ones(2)), "temperature"),
    (dict(top_k=torch.ones(3)), "top_k"), (dict(top_p=torch.ones(3, dtype=BF)), "top_p"),
    (dict(), "on a GPU")])
def test_sample_tensors(kw, match):
    a = dict(logits=torch.zeros(3, 9), uniforms=torch.zeros(3))
    a.update(kw)
    with pytest.raises(ValueError, match=match):
        binding.sample(a.pop("logits"), a.pop("uniforms"), **a)
    with pytest.raises(TypeError):
        binding.sample(torch.zeros(3, 9), torch.zeros(3), top_k=1.5)
