"""Sampling on the GPU against the float64 oracle: tokens and kept counts are
equal.  (The kernel's running sums are off by 4e-9 of the largest weight at worst;
no uniform number here falls that near a boundary of the oracle's, or it would
differ from it by the oracle's own rounding too.)  Probabilities are rounded to
fp32 once after sums exact to 1e-8: 2^-24 + 1e-8 of the value."""

import numpy as np
import pytest
import torch

import oracle.sampling as ref

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def f32(v):
    return np.float32(v) if not isinstance(v, torch.Tensor) else v.cpu().numpy()


def run(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, prob, kept) of the kernel, checked against the oracle's."""
    from paper_2606_02544_amd import binding
    par = dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    put = {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in par.items()}
    token, prob, kept = binding.sample(logits.cuda() if not logits.is_cuda else logits, u.cuda(), **put)
    want = ref.sample(logits.cpu().double().numpy(), u.numpy(), f32(temperature),
                      top_k if not isinstance(top_k, torch.Tensor) else top_k.numpy(), f32(top_p), f32(min_p))
    assert token.cpu().tolist() == want[0].tolist()
    assert kept.cpu().tolist() == want[2].tolist()
    np.testing.assert_allclose(prob.cpu().numpy(), want[1], rtol=2.0 ** -24 + 1e-8, atol=0)
    return token, prob, kept


def rows(n, V, dt, seed, sigma=2.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, V), generator=g) * sigma).to(dt), torch.rand(n, generator=g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 8, 9, 63, 511, 1000, 4097, 50001, 151936, 155647, 155649, 200003])
def test_sizes_unfiltered_and_filtered(dtype, V):
    n = 5 if V < 100000 else 3
    x, u = rows(n, V, DT[dtype], V)
    run(x, u)
    run(x, u, 0.7, 50, 0.9, 0.01)
    run(x, u, 0.0)


FILTERS = [dict(top_k=1), dict(top_k=3), dict(top_k=999), dict(top_k=1000), dict(top_k=1001), dict(top_p=0.0),
           dict(top_p=1e-6), dict(top_p=0.5), dict(top_p=0.95), dict(top_p=0.9999), dict(min_p=1.0),
           dict(min_p=0.3), dict(min_p=1e-3), dict(min_p=1e-30), dict(top_k=20, top_p=0.9),
           dict(top_k=20, top_p=0.9, min_p=0.2), dict(top_p=0.9, min_p=0.01), dict(top_k=200, min_p=0.002),
           dict(temperature=0.01), dict(temperature=1e-30), dict(temperature=100.0, top_p=0.5),
           dict(temperature=1e30, top_k=7), dict(temperature=0.3, top_k=500, top_p=0.7, min_p=0.001)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("params", FILTERS, ids=str)
def test_filters(dtype, params):
    x, u = rows(16, 1000, DT[dtype], 77)
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    run(x, u, **params)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_parameters_a_row(dtype):
    x, u = rows(64, 3001, DT[dtype], 5)
    g = torch.Generator().manual_seed(6)
    pick = lambda v: torch.tensor(v)[torch.randint(0, len(v), (64,), generator=g)]  # noqa: E731
    run(x, u, pick([0.0, 0.5, 1.0, 1.7, -1.0]), pick([0, 1, 40, 5000, -3]).to(torch.int32),
        pick([1.0, 0.6, 0.97, 0.0, 1.5]), pick([0.0, 0.05, 1.0, -0.5]))


def test_parameters_that_are_no_numbers():
    from paper_2606_02544_amd import binding
    x, u = rows(3, 500, torch.float32, 8)
    nan = torch.full((3,), float("nan"))
    inf = torch.full((3,), float("inf"))
    plain = run(x, u)
    got = binding.sample(x.cuda(), u.cuda(), top_p=nan.cuda(), min_p=nan.cuda())
    assert all(torch.equal(a, b) for a, b in zip(got, plain))
    assert torch.equal(binding.sample(x.cuda(), u.cuda(), temperature=nan.cuda())[0].cpu().long(), x.argmax(1))
    got = binding.sample(x.cuda(), u.cuda(), temperature=inf.cuda())
    assert got[2].tolist() == [500] * 3
    # u outside [0, 1) stays inside the row
    bad = torch.tensor([1.0, -3.0, float("nan")])
    token = binding.sample(x.cuda(), bad.cuda())[0].cpu()
    assert token[0] == x[0].argmin() and token[1] == x[1].argmax() and token[2] == x[2].argmax()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [100, 65536, 151936, 200003])
def test_equal_logits(dtype, V):
    """Ties in the order of the index; counts past 16 bits."""
    u = torch.tensor([0.0, 0.25, 0.5, 0.999999])
    for value in (0.0, 1.0078125, -3.0, -3.015625):
        x = torch.full((4, V), value, dtype=DT[dtype])
        run(x, u)
        run(x, u, top_k=V // 2 + 1, top_p=0.5)
    x[:, V // 3] = 5.0
    x[:, V // 2:] = 2.0
    x[:, -1] = -2.0
    run(x, u, 0.9)
    run(x, u, 0.9, top_p=0.75)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fill", [float("-inf"), float("nan"), "lowest"])
@pytest.mark.parametrize("V", [64, 151936])
def test_masked_logits(dtype, fill, V):
    x, u = rows(4, V, DT[dtype], 12)
    g = torch.Generator().manual_seed(1)
    value = torch.finfo(DT[dtype]).min if fill == "lowest" else fill
    x[torch.rand(x.shape, generator=g) < 0.95] = value
    x[3] = value
    run(x, u)
    run(x, u, 0.8, 30, 0.9, 0.02)
    run(x, u, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_and_signed_zero_logits(dtype):
    x, u = rows(4, 300, DT[dtype], 13)
    x[0, 100] = x[0, 200] = float("inf")
    x[1] = float("inf")
    x[2, :] = torch.where(torch.arange(300) % 2 == 0, 0.0, -0.0).to(DT[dtype])
    x[3, :] = -1.0
    x[3, 5::7] = -0.0
    x[3, 6::7] = 0.0
    run(x, u)
    run(x, u, 0.0)
    run(x, u, 1.0, 70, 0.6, 0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5003, 151936])
def test_logits_of_one_sign(dtype, V):
    """Log-probabilities (nothing positive), few positive entries, a NaN among them,
    and the largest entry at either end of the row."""
    x, u = rows(6, V, DT[dtype], 40)
    x[0] -= 40.0
    x[1] = torch.log_softmax(x[1].float(), 0).to(DT[dtype])
    x[2, 10:] = -x[2, 10:].abs() - 0.5
    x[3, V // 2] = float("nan")
    x[4, 0] = 30.0
    x[5, V - 1] = 30.0
    run(x, u)
    run(x, u, 0.8, 40, 0.9)
    run(x, u, 1.0, 0, 1.0, 0.05)
    run(x, u, 1.0, 0, 0.9)
    run(x, u, 0.0)


def test_every_bf16_pattern():
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    g = torch.Generator().manual_seed(3)
    x = torch.stack([bits[torch.randperm(65536, generator=g)].view(torch.bfloat16) for _ in range(4)])
    x[2:][torch.isinf(x[2:])] = 0.0
    u = torch.tensor([0.1, 0.9, 0.3, 0.7])
    run(x, u)
    run(x, u, 1e38, 20000)
    run(x, u, 1e37, 0, 0.7, 0.001)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_start_anywhere(dtype):
    x, u = rows(7, 1003, DT[dtype], 21)
    flat = torch.zeros(7 * 1003 + 3, dtype=DT[dtype], device="cuda")
    for shift in (1, 2, 3):
        y = flat[shift:shift + 7 * 1003].view(7, 1003)
        y.copy_(x)
        run(y, u, 0.9, 100, 0.9)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_same_on_every_run_and_from_a_graph(dtype):
    from paper_2606_02544_amd import binding
    x, u = rows(9, 20011, DT[dtype], 30)
    x, u = x.cuda(), u.cuda()
    call = lambda: binding.sample(x, u, temperature=0.9, top_k=400, top_p=0.9, min_p=0.001)  # noqa: E731
    first = call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for _ in range(3):
        graph.replay()
        eager = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))
        if _ == 0:
            assert all(torch.equal(a, b) for a, b in zip(out, first))
        u.copy_(torch.rand(9, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_largest_vocabulary(dtype):
    """2^22 entries: flat, masked with the lowest value, and few of them possible."""
    x, u = rows(3, 2 ** 22, DT[dtype], 31)
    x[1] = torch.finfo(DT[dtype]).min
    x[1, 12345::70001] = 3.0
    x[2] = 1.0
    run(x, u)
    run(x, u, 0.9, 300, 0.9, 0.01)
    run(x, u, 0.5, 0, 0.3)


def test_a_row_past_32_bits_of_offset():
    """Logits of more than 2^32 bytes: the last rows are read where they lie."""
    from paper_2606_02544_amd import binding
    V, n = 2 ** 22, 520
    x = torch.zeros((n, V), dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 31
    x[n - 1, 77] = x[n - 2, V - 1] = 50.0
    token, prob, kept = binding.sample(x, torch.full((n,), 0.5, device="cuda"), top_k=5)
    assert token[n - 1] == 77 and token[n - 2] == V - 1 and kept[0] == 5 and token[0] == 2
    assert prob[n - 1] == 1.0 and abs(float(prob[0]) - 0.2) < 1e-6


def test_given_outputs_and_no_rows():
    from paper_2606_02544_amd import binding
    x, u = rows(2, 100, torch.float32, 1)
    t = torch.empty(2, dtype=torch.int32, device="cuda")
    got = binding.sample(x.cuda(), u.cuda(), token=t, stream=torch.cuda.current_stream())
    assert got[0] is t
    empty = binding.sample(torch.zeros((0, 5), device="cuda"), torch.zeros(0, device="cuda"))
    assert [e.shape for e in empty] == [(0,)] * 3
