"""Host threads that call an operator with scratch on one stream: its kernels are
enqueued call by call (CPU; the library is stood in for)."""

import contextlib
import threading
import time
import types

import torch

from paper_2606_02544_amd import binding

BF, I32 = torch.bfloat16, torch.int32


def test_two_threads_on_one_stream(monkeypatch):
    inside, most, buffers = [], [], []

    def call(*args):
        inside.append(1)
        most.append(len(inside))
        buffers.append(args[-3])
        time.sleep(0.02)                                       # (the interpreter runs the other threads)
        inside.pop()
        return 0

    real = binding.lib()
    stand_in = types.SimpleNamespace(
        simsd_chunk_attention=call,
        simsd_chunk_attention_workspace_size=real.simsd_chunk_attention_workspace_size)
    monkeypatch.setattr(binding, "lib", lambda: stand_in)
    monkeypatch.setattr(binding, "_Launch",
                        lambda device, stream: contextlib.nullcontext(types.SimpleNamespace(handle=0)))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(binding, "WORKSPACES", binding._Workspaces())
    z = lambda *s, dtype=BF: torch.zeros(s, dtype=dtype)  # noqa: E731
    cache = z(2, 256, 2, 64)

    def thread():
        for _ in range(3):
            binding.chunk_attention(z(6, 4, 64), cache, cache, None, z(3, dtype=I32), z(2, dtype=I32), max_q_len=6,
                                    max_kv_len=256, kv_chunk=64)

    threads = [threading.Thread(target=thread) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(buffers) == 12 and None not in buffers
    assert max(most) == 1
