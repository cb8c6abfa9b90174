"""Windows, 4-bit caches and the verification step as a server runs them: prompts in
ragged chunks, blocks that are verified and partly accepted, single tokens, over pages
that the sequences take as they grow; every step against the float64 oracle over the
cache as it then is (tolerances as derived in tests/test_gpu_chunk.py)."""

import numpy as np
import pytest
import torch

import oracle.fp4 as fp4
import oracle.window as ref
from test_gpu_window import near

pytestmark = pytest.mark.gpu
HQ, HKV, D, PAGE, CAP, WINDOW, SINKS = 8, 2, 64, 16, 240, 70, 5
B, L = 4, 3                                                    # block and reference slots of a verification
ROUNDS = [[70, 1, 33], [0, 64, 50], [41, 30, 0]]               # the prompts' chunks


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Server:
    def __init__(self, form, seed):
        from paper_2606_02544_amd import binding
        self.binding, self.form = binding, form
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        n, per = len(ROUNDS[0]), -(-CAP // PAGE)
        self.cache = binding.fp4_cache(n * per, PAGE, HKV, D) if form == "fp4" else \
            [torch.zeros((n * per, PAGE, HKV, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.table = torch.randperm(n * per, generator=self.g, device="cuda").view(n, per).to(torch.int32)
        self.freq, _ = binding.rope_frequencies(D, 10000.0)
        self.kv = [0] * n
        self.log = [[] for _ in range(n)]                      # k and v rows of each sequence, before rotation

    def rows(self, *shape):
        return torch.randn((*shape, D), generator=self.g, device="cuda").bfloat16()

    def held(self):
        """The caches' values in float64, as the oracle takes them."""
        if self.form == "fp4":
            c = [x.cpu().numpy() for x in self.cache]
            return fp4.decode(c[0], c[2]), fp4.decode(c[1], c[3])
        return [x.double().cpu().numpy() for x in self.cache]

    def append(self, q, k, v, n, cache=None, kv=None):
        where = (self.table, i32(*np.cumsum([0] + n)), i32(*(kv or self.kv)), self.freq)
        kw = dict(max_kv_len=CAP, page_size=PAGE)
        c = cache or self.cache
        return self.binding.rotary_append_fp4(q, k, v, c, *where, **kw) if self.form == "fp4" else \
            self.binding.rotary_append(q, k, v, *c, *where, **kw)

    def forward(self, n, mask_block, window, sinks):
        """A step of n[b] new tokens of each sequence: appended, then attended to."""
        q, k, v = self.rows(sum(n), HQ), self.rows(sum(n), HKV), self.rows(sum(n), HKV)
        for i, at in enumerate(np.cumsum([0] + n)[:-1]):
            self.log[i].append((k[at:at + n[i]], v[at:at + n[i]]))
            self.kv[i] += n[i]
        q = self.append(q, k, v, n)
        starts, kv = i32(*np.cumsum([0] + n)), i32(*self.kv)
        kw = dict(max_q_len=max(n), max_kv_len=CAP, page_size=PAGE, mask_block=mask_block, window=window, sinks=sinks)
        where = (self.table, starts, kv)
        out, lse = self.binding.chunk_attention_fp4(q, self.cache, *where, **kw) if self.form == "fp4" else \
            self.binding.chunk_attention(q, *self.cache, *where, **kw)
        f = lambda x: x.double().cpu().numpy()  # noqa: E731
        want, wl, size, S = ref.chunk_attention(f(q), *self.held(), self.table.cpu(), starts.tolist(), self.kv,
                                                mask_block=mask_block, window=window, sinks=sinks, page=PAGE)
        near(f(out), f(lse).T, want, wl.T, size, S.T, D, CAP, True)

    def verify(self, window, sinks):
        b, n = len(self.kv), B + L
        q, k, v = self.rows(b, n, HQ), self.rows(b, n, HKV), self.rows(b, n, HKV)
        steps, refs = i32([1, 2, 3, 0], [3, 1, 0, 2], [0, 1, -1, 2]), i32(3, 3, 2)
        kw = dict(block_size=B, max_ref=L, max_prefix_len=CAP, page_size=PAGE, window=window, sinks=sinks)
        where = (self.table, i32(*self.kv), steps, refs)
        out, lse = self.binding.verify_attention_fp4(q, k, v, self.cache, *where, **kw) if self.form == "fp4" else \
            self.binding.verify_attention(q, k, v, *self.cache, *where, **kw)
        f = lambda x: x.double().cpu().numpy()  # noqa: E731
        want, wl, size, S = ref.verify_attention(f(q), f(k), f(v), *self.held(), self.table.cpu(), self.kv, steps.cpu().numpy(),
                                                 refs.tolist(), window=window, sinks=sinks, page=PAGE)
        t = lambda x: x.transpose(0, 2, 1)  # noqa: E731
        near(f(out), t(f(lse)), want, t(wl), size, t(S), D, CAP + n, True)


@pytest.mark.parametrize("form,window,sinks", [("fp4", 0, 0), ("fp4", WINDOW, SINKS), ("bf16", WINDOW, SINKS)])
def test_a_server(form, window, sinks):
    s = Server(form, 3)
    for n in ROUNDS:
        s.forward(n, 1, window, sinks)
    for accepted in ([4, 0, 2], [1, 4, 3]):
        s.verify(window, sinks)
        s.forward(accepted, 4, window, sinks)                  # the accepted tokens, seen as one block
    for _ in range(3):
        s.forward([1, 1, 1], 1, window, sinks)
    # The cache holds what one append of each sequence's whole would have written.
    whole = [torch.zeros_like(x) for x in s.cache]
    whole = s.binding.Fp4Cache(*whole) if form == "fp4" else whole
    k, v = (torch.cat([r[j] for log in s.log for r in log]) for j in range(2))
    s.append(None, k, v, list(s.kv), whole)
    assert all(torch.equal(x, y) for x, y in zip(s.cache, whole))


def test_a_cache_as_a_plain_tuple():
    s = Server("fp4", 4)
    k, v = s.rows(6, HKV), s.rows(6, HKV)
    s.append(None, k, v, [3, 1, 2], kv=[3, 1, 2])
    again = tuple(torch.zeros_like(x) for x in s.cache)
    s.append(None, k, v, [3, 1, 2], again, kv=[3, 1, 2])
    assert all(torch.equal(x, y) for x, y in zip(s.cache, again))
