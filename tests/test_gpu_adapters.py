"""Low-rank adapters of many requests (ordermoe_adapters) against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2607_17154_gb300 import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF16 = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    B.lib()


@pytest.fixture(autouse=True)
def _no_device_error():
    yield
    assert B.ordermoe_device_error()[0] == 0


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rnd(g, *shape, std=1.0, pad=0):
    """bf16 values whose rows lie `pad` and what is missing to a multiple of 8 apart; NaN between them."""
    w = shape[-1]
    ld = (w + 7) // 8 * 8 + pad
    t = torch.full((*shape[:-1], ld), math.nan, dtype=BF16, device=DEV)[..., :w]
    return t.copy_((torch.randn(*shape, device=DEV, generator=g) * std).to(BF16))


def reference(X, A, Bw, ids, scale, rank, residual, out):
    """Y and its bound in 64 bits. h: products are exact, K of them summed in fp32 (2^-23 a sum, the tensor cores may
    cut); its two bf16 parts are within 2^-16 of it; R products of each part, again 2^-23 a sum; scale, residual and the
    rounding to Y (2^-8, or 2^-24) once each."""
    T, N = out.shape
    y = torch.zeros(T, N, dtype=torch.double, device=DEV)
    far = torch.zeros_like(y)
    n, R, K = A.shape
    for a in range(n):
        t = (ids == a).nonzero()[:, 0]
        if not len(t):
            continue
        r = R if rank is None else int(rank[a])
        s = 1.0 if scale is None else float(scale[a])
        x, d, u = X[t].double(), A[a, :r].double(), Bw[a, :, :r].double()
        h, habs = x @ d.T, x.abs() @ d.abs().T
        y[t] = s * (h @ u.T)
        far[t] = abs(s) * (habs @ u.abs().T * (K + 40) * 2.0 ** -23 + h.abs() @ u.abs().T * (2.0 ** -16 + (2 * R + 8) * 2.0 ** -23))
    if residual is not None:
        y += residual.double()
    step = 2.0 ** -24 if out.dtype == torch.float32 else 2.0 ** -8
    return y, far + y.abs() * (step + 2.0 ** -23) + (0 if residual is None else residual.double().abs() * 2.0 ** -23) + 2.0 ** -120


def call(X, A, Bw, ids, Y, **kw):
    T, K = X.shape
    ws = torch.empty(B.ordermoe_adapters_workspace_bytes(T, K, Y.shape[1], A.shape[1]), dtype=torch.uint8, device=DEV).fill_(255)
    B.ordermoe_adapters(X, A, Bw, ids, Y, ws, **kw)


def check(X, A, Bw, ids, Y, scale=None, rank=None, residual=None):
    keep = None if residual is None else residual.clone()
    call(X, A, Bw, ids, Y, scale=scale, rank=rank, residual=residual)
    y, far = reference(X, A, Bw, ids, scale, rank, keep, Y)
    assert bool(((Y.double() - y).abs() <= far).all()), float(((Y.double() - y).abs() - far).max())


SIZES = [  # T, K, N, R, adapters
    (1, 64, 64, 8, 1), (1, 4096, 4096, 16, 3), (2, 1, 1, 8, 2), (5, 63, 9, 24, 4), (16, 100, 300, 32, 2), (17, 512, 257, 64, 1),
    (33, 1999, 1009, 40, 7), (64, 128, 256, 128, 64), (127, 320, 100, 16, 3), (128, 1024, 512, 64, 32), (129, 72, 520, 8, 200),
    (300, 2048, 130, 120, 5), (1000, 96, 64, 48, 2), (4096, 256, 264, 16, 8), (3, 14336, 64, 8, 2), (200, 300, 700, 128, 12), (128, 64, 1500, 72, 3), (40, 33, 65, 16, 40), (4100, 64, 9000, 72, 3), (45000, 32, 200, 8, 5)]


@pytest.mark.parametrize("T,K,N,R,n", SIZES)
@pytest.mark.parametrize("f32", [False, True])
def test_sizes(T, K, N, R, n, f32):
    g = gen(T + K)
    X, A, Bw = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1)
    ids = torch.randint(-1, n, (T,), dtype=torch.int32, device=DEV, generator=g)
    Y = torch.full((T, N), math.nan, dtype=torch.float32 if f32 else BF16, device=DEV)
    check(X, A, Bw, ids, Y, scale=torch.randn(n, device=DEV, generator=g), residual=rnd(g, T, N))


@pytest.mark.parametrize("order", ["runs", "one", "none", "alternating", "descending"])
def test_orders_of_tokens(order):
    T, K, N, R, n = 400, 200, 300, 32, 9
    g = gen(7)
    t = torch.arange(T, dtype=torch.int32, device=DEV)
    ids = {"runs": t // 50, "one": 0 * t + 4, "none": 0 * t - 1, "alternating": t % n, "descending": (T - 1 - t) // 50}[order].int()
    X, A, Bw = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1)
    check(X, A, Bw, ids, torch.empty(T, N, dtype=BF16, device=DEV), residual=rnd(g, T, N))
    check(X, A, Bw, ids, torch.empty(T, N, dtype=torch.float32, device=DEV))  # no residual, no scale


def test_ranks_and_what_is_behind_them():
    T, K, N, R, n = 150, 130, 70, 32, 5
    g = gen(8)
    X, A, Bw = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1)
    rank = torch.tensor([0, 1, 15, 17, 32], dtype=torch.int32, device=DEV)
    for a, r in enumerate(rank.tolist()):
        A[a, r:] = math.nan
        Bw[a, :, r:] = math.nan
    ids = torch.randint(-1, n, (T,), dtype=torch.int32, device=DEV, generator=g)
    check(X, A, Bw, ids, torch.empty(T, N, dtype=BF16, device=DEV), rank=rank, residual=rnd(g, T, N))


def test_one_tokens_values_do_not_reach_another():
    T, K, N, R, n = 40, 64, 64, 16, 2
    g = gen(9)
    X, A, Bw = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1)
    ids = (torch.arange(T, device=DEV) % 3 - 1).int()
    X[1], X[20] = math.nan, math.inf
    A[1, 3, 5] = math.nan  # tokens of adapter 1 alone
    Y = torch.zeros(T, N, dtype=torch.float32, device=DEV)
    res = rnd(g, T, N)
    call(X, A, Bw, ids, Y, residual=res)
    hit = (ids == 1)
    hit[1], bad0 = True, (ids == 0) & (torch.arange(T, device=DEV) != 1)
    assert bool(torch.isnan(Y[hit]).all())
    assert torch.equal(Y[ids == -1], res[ids == -1].float())
    y, far = reference(X[bad0], A, Bw, ids[bad0], None, None, res[bad0], Y[bad0])
    assert bool(((Y[bad0].double() - y).abs() <= far).all())


@pytest.mark.parametrize("pad", [8, 40])
def test_wider_buffers_and_in_place(pad):
    T, K, N, R, n = 77, 90, 110, 24, 3
    g = gen(10)
    X, A, Bw = rnd(g, T, K, pad=pad), rnd(g, n, R, K, std=0.05, pad=pad), rnd(g, n, N, R, std=0.1, pad=pad)
    ids = torch.randint(-1, n, (T,), dtype=torch.int32, device=DEV, generator=g)
    for shift in (0, 1):  # rows of Y and residual at odd addresses too
        wide = torch.full((T, N + pad + 1), 5.0, dtype=BF16, device=DEV)
        Y = wide[:, shift:shift + N]
        Y.copy_(torch.randn(T, N, device=DEV, generator=g).to(BF16))
        check(X, A, Bw, ids, Y, residual=Y)
        assert bool((wide[:, :shift] == 5.0).all()) and bool((wide[:, shift + N:] == 5.0).all())


def test_far_adapters():
    """Adapters whose addresses pass 2^31 values."""
    K, N, R = 4096, 64, 128
    n = (1 << 31) // (R * K) + 2
    A = torch.zeros(n, R, K, dtype=BF16, device=DEV)
    g = gen(11)
    A[-1] = torch.randn(R, K, device=DEV, generator=g) * 0.05
    Bw = torch.zeros(n, N, R, dtype=BF16, device=DEV)
    Bw[-1] = torch.randn(N, R, device=DEV, generator=g) * 0.1
    X = rnd(g, 3, K)
    ids = torch.tensor([n - 1, -1, n - 1], dtype=torch.int32, device=DEV)
    Y = torch.empty(3, N, dtype=BF16, device=DEV)
    call(X, A, Bw, ids, Y)
    y, far = reference(X, A[-1:], Bw[-1:], (ids == n - 1).int() - 1, None, None, None, Y)
    assert bool(((Y.double() - y).abs() <= far).all())


def test_bad_ids_and_ranks_are_reported():
    T, K, N, R, n = 6, 64, 64, 16, 2
    g = gen(12)
    X, A, Bw, res = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1), rnd(g, T, N)
    Y, want = (torch.empty(T, N, dtype=BF16, device=DEV) for _ in range(2))
    for bad in (n, -2, 2 ** 31 - 1):
        ids = torch.tensor([0, 1, 0, bad, 1, 0], dtype=torch.int32, device=DEV)
        call(X, A, Bw, ids, Y, residual=res)
        assert B.ordermoe_device_error() == (B.DEV_BAD_INDEX, 3)
        ids[3] = -1
        call(X, A, Bw, ids, want, residual=res)
        assert torch.equal(Y, want)
    call(X, A, Bw, ids, Y, residual=res, rank=torch.tensor([-1, R + 1], dtype=torch.int32, device=DEV))
    assert B.ordermoe_device_error()[0] == B.DEV_BAD_INDEX
    call(X, A, Bw, ids, want, residual=res, rank=torch.tensor([0, R], dtype=torch.int32, device=DEV))
    assert torch.equal(Y, want)


def test_captured_with_ids_that_change_and_on_a_stream():
    T, K, N, R, n = 130, 256, 128, 16, 4
    g = gen(13)
    X, A, Bw, res = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1), rnd(g, T, N)
    ids = torch.zeros(T, dtype=torch.int32, device=DEV)
    Y, want = (torch.empty(T, N, dtype=BF16, device=DEV) for _ in range(2))
    ws = torch.empty(B.ordermoe_adapters_workspace_bytes(T, K, N, R), dtype=torch.uint8, device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.ordermoe_adapters(X, A, Bw, ids, Y, ws, residual=res)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            B.ordermoe_adapters(X, A, Bw, ids, Y, ws, residual=res)
    for i in range(4):
        ids.copy_(torch.randint(-1, n, (T,), dtype=torch.int32, device=DEV, generator=g))
        graph.replay()
        check(X, A, Bw, ids, want, residual=res)
        assert torch.equal(Y, want)


@pytest.mark.parametrize("rows", [16, 17, 33, 65, 128])
@pytest.mark.parametrize("N", [1, 31, 129, 383, 640])
def test_tokens_of_one_adapter_over_slices_of_columns(rows, N):
    """Every share of the warps between tokens and columns, over several slices, with rows in any place and in vectors."""
    T, K, R, n = 300, 72, 40, 2
    g = gen(rows + N)
    X, A, Bw = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1)
    ids = torch.full((T,), -1, dtype=torch.int32, device=DEV)
    ids[5:5 + rows] = 1
    ids[200:299:3] = 0
    for dt in (BF16, torch.float32):
        check(X, A, Bw, ids, torch.empty(T, N, dtype=dt, device=DEV), residual=rnd(g, T, N))
        check(X, A, Bw, ids, torch.empty(T, N + 3, dtype=dt, device=DEV)[:, :N])


@pytest.mark.parametrize("T", [3, 128, 1000, 4096])
def test_results_in_32_bits_over_a_long_k(T):
    """In the 2-norm: a sum of 512 of K is 32 products of 16. Where each is cut instead of rounded, by 2^-24 of the running
    sum in the mean, and that grows as the root of their number, the sum is off by 2^-24 * 32 * 2 / 3 < 2^-19 of itself;
    what follows is rounded. (One running sum over K = 14336 would be off by 28 times that.)"""
    K, N, R, n = 14336, 128, 128, 2
    g = gen(T)
    X, A, Bw = rnd(g, T, K), rnd(g, n, R, K, std=0.02), rnd(g, n, N, R, std=0.1)
    ids = (torch.arange(T, dtype=torch.int32, device=DEV) // 64 % n).int()
    Y = torch.empty(T, N, dtype=torch.float32, device=DEV)
    call(X, A, Bw, ids, Y)
    y, _ = reference(X, A, Bw, ids, None, None, None, Y)
    assert float((Y.double() - y).norm() / y.norm()) <= 2.0 ** -19


def test_inputs_written_by_the_kernels_before():
    """Ids, weights, ranks, the residual (a product's result) and X change right before each call, nothing waits in between:
    the same bits as with a wait after every step."""
    T, K, N, R, n = 150, 512, 1024, 32, 6
    g = gen(14)
    W = rnd(g, N, K, std=0.02)
    X, A, Bw = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1)
    ids, rank = torch.zeros(T, dtype=torch.int32, device=DEV), torch.full((n,), R, dtype=torch.int32, device=DEV)
    Y = torch.empty(T, N, dtype=BF16, device=DEV)
    ws = torch.empty(B.ordermoe_adapters_workspace_bytes(T, K, N, R), dtype=torch.uint8, device=DEV)
    sets = [(rnd(g, T, K), rnd(g, n, N, R, std=0.1), torch.randint(-1, n, (T,), dtype=torch.int32, device=DEV, generator=g),
             torch.randint(0, R + 1, (n,), dtype=torch.int32, device=DEV, generator=g)) for _ in range(24)]

    def steps(wait):
        out = []
        for x, b, i, r in sets:
            for to, what in ((X, x), (Bw, b), (ids, i), (rank, r)):
                to.copy_(what)
                wait()
            B.ordermoe_linear(X, W, Y)
            wait()
            B.ordermoe_adapters(X, A, Bw, ids, Y, ws, rank=rank, residual=Y)
            wait()
            out.append(Y.clone())
        return out

    want = steps(torch.cuda.synchronize)
    for _ in range(4):
        for a, b in zip(steps(lambda: None), want):
            assert torch.equal(a, b)


def test_on_another_stream():
    T, K, N, R, n = 130, 256, 320, 16, 4
    g = gen(15)
    X, A, Bw, res = rnd(g, T, K), rnd(g, n, R, K, std=0.05), rnd(g, n, N, R, std=0.1), rnd(g, T, N)
    ids = torch.randint(-1, n, (T,), dtype=torch.int32, device=DEV, generator=g)
    ws = torch.empty(B.ordermoe_adapters_workspace_bytes(T, K, N, R), dtype=torch.uint8, device=DEV)
    Y, want, s = torch.zeros(T, N, dtype=BF16, device=DEV), torch.zeros(T, N, dtype=BF16, device=DEV), torch.cuda.Stream()
    check(X, A, Bw, ids, want, residual=res)
    s.wait_stream(torch.cuda.current_stream())
    B.ordermoe_adapters(X, A, Bw, ids, Y, ws, residual=res, stream=s)
    s.synchronize()
    assert torch.equal(Y, want)
