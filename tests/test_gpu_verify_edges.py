"""Verifications under a window that holds no cached key, on the GPU against the float64
oracle (tolerances as derived for bf16 chunk attention, tests/test_gpu_chunk.py); the
lists themselves are gone through on the CPU (tests/test_verify_list_host.py)."""

import pytest

from test_gpu_verify_span import FORMS, call, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("B,L,hq,hkv,d", [(4, 4, 4, 2, 64), (8, 8, 8, 2, 128), (32, 32, 4, 1, 64), (32, 32, 4, 1, 128)])
@pytest.mark.parametrize("page,prefix", [(16, [16, 48, 80, 32]), (24, [24, 72, 120]), (1, [33, 1, 64]), (0, [96, 100, 100]), (0, [65, 65])])
def test_a_window_of_one_key(form, B, L, hq, hkv, d, page, prefix):
    """Prefixes that end with a page inside a tile, and that fill a contiguous cache: the
    slots see the sinks and each other."""
    s = make(form, prefix, B, L, hq, hkv, d, page, len(prefix))
    for sinks in (0, 1, 20, 64, 90):
        for kv_chunk in (0, 64):
            check(s, *call(s, window=1, sinks=sinks, kv_chunk=kv_chunk), 1, sinks)
