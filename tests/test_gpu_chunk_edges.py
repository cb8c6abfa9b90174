"""Chunk attention of values that are not finite in keys that every row sees."""

import pytest
import torch

from test_gpu_chunk import DT, call, make

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("max_q", [1, 20, 40, 500])
@pytest.mark.parametrize("kv_chunk", [0, 64])
def test_in_whole_tiles_and_in_masked_ones(dtype, d, page, max_q, kv_chunk):
    """Keys 10 and 70 (whole tiles of every row), 330 and 340 (masked ones of the first
    sequence): the element of every row that sees the value is it, or NaN where two meet,
    and all others are what they were."""
    s = make([(60, 350), (1, 200)], 8, 2, d, dtype, page, 31)

    def at(b, t):
        return (int(s["table"][b, t // page]), t % page) if page else (b, t)

    base, base_lse = call(s, mask_block=1, max_q_len=max_q, kv_chunk=kv_chunk)
    for b, t, dim, value in ((0, 10, 3, INF), (0, 70, 5, -INF), (0, 330, 7, INF), (0, 340, 7, -INF),
                             (0, 70, 9, float("nan")), (1, 10, 4, -INF), (1, 199, 11, INF)):
        s["v"][(*at(b, t), 1, dim)] = value
    out, lse = call(s, mask_block=1, max_q_len=max_q, kv_chunk=kv_chunk)
    want = base.clone()
    want[:60, 4:, 3], want[:60, 4:, 5], want[:60, 4:, 9] = INF, -INF, float("nan")
    want[40:60, 4:, 7], want[50:60, 4:, 7] = INF, float("nan")        # token i sees 291 + i keys
    want[60, 4:, 4], want[60, 4:, 11] = -INF, INF
    assert torch.equal(lse, base_lse)
    same = (out == want) | (out.isnan() & want.isnan())
    assert bool(same.all()), (~same).nonzero()[:8]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_q", [1, 40, 500])
@pytest.mark.parametrize("kv_chunk", [0, 64])
def test_with_weights_that_vanish(dtype, max_q, kv_chunk):
    """A value whose key weighs 0 beside the row's others: infinity, or NaN as 0 times it
    is (which of them may differ by the division of the keys), and nothing else changes."""
    s = make([(60, 350)], 4, 1, 64, dtype, 0, 32)
    s["q"][:, :, 0] = 30.0
    s["k"][:, :, :, 0] = 30.0
    for t in (10, 130, 300):
        s["k"][0, t, 0, 0] = -30.0                             # 225 below the others, e^-225 of their weight
    base, base_lse = call(s, mask_block=1, max_q_len=max_q, kv_chunk=kv_chunk)
    for t, dim in ((10, 3), (130, 5), (300, 7)):
        s["v"][0, t, 0, dim] = INF
    out, lse = call(s, mask_block=1, max_q_len=max_q, kv_chunk=kv_chunk)
    sees = torch.zeros(out.shape, dtype=torch.bool)
    sees[:, :, 3] = sees[:, :, 5] = True
    sees[10:, :, 7] = True                                     # token i sees 291 + i keys
    hit = out.cpu()[sees]
    assert bool((hit.isnan() | (hit == INF)).all())
    assert torch.equal(out.cpu()[~sees], base.cpu()[~sees]) and torch.equal(lse, base_lse)


def test_threads_that_share_a_stream():
    """Calls with key ranges from several host threads on the default stream."""
    import threading
    from paper_2606_02544_amd import binding
    sets = [make([(2, 900), (1, 700)], 8, 2, 128, "bf16", 16, 50 + i) for i in range(3)]
    dev = [[s[n].cuda() for n in ("q", "k", "v", "table", "starts", "kv")] for s in sets]
    one = lambda i: binding.chunk_attention(*dev[i], max_q_len=2, max_kv_len=sets[i]["cap"], page_size=16,  # noqa: E731
                                            kv_chunk=64)
    want = [one(i) for i in range(3)]
    got = [[], [], []]

    def thread(i):
        for _ in range(40):
            got[i].append(one(i))

    threads = [threading.Thread(target=thread, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(3):
        assert len(got[i]) == 40
        for out, lse in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])
