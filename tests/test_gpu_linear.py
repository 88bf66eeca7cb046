"""ordermoe_linear against Y = act(X W^T + bias) + residual in 64 bits, and dense layers in a
stack.

Tolerance: the fp32 sum of K products and the bias is off by at most (K + 8) 2^-24 of the sum
of magnitudes S = |x| |w| + |b| (one rounding or truncation of the running sum for each product,
twice the half-step for truncation: (K + 8) 2^-23 S); an activation's slope is at most
1.13 (GELU) and its own fp32 evaluation within 2^-20 of its value; the residual adds one
rounding of 2^-24. Then one rounding to Y: 2^-8 of its value in bf16, 2^-24 in fp32."""
import math

import numpy as np
import pytest
import torch

import oracle
from paper_2607_17154_gb300 import binding as B
from paper_2607_17154_gb300 import synth
from paper_2607_17154_gb300.layer import DenseFFN, LayerStack, exact_tables
from paper_2607_17154_gb300.layer import build_tables, calibrate_stack

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    B.lib()
    yield
    code, detail = B.ordermoe_device_error()
    assert code == 0, (code, detail)


def rows(n, w, std, seed, pad=0, odd=False, dt=torch.bfloat16, offset=0):
    ld = (w if odd else (w + 7) // 8 * 8) + pad
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    buf = torch.randn(n * ld + offset, generator=g, device=DEV) * std
    return buf.to(dt)[offset:].view(n, ld)[:, :w]


def act64(v, act):
    if act == "relu":
        return v.clamp(min=0.0)
    if act == "gelu":
        return v * 0.5 * torch.special.erfc(-v / math.sqrt(2.0))
    if act == "gelu_tanh":
        # 0.5 (1 + tanh u) = sigmoid(2 u): the sum loses the tail (u = -32: 1e-28) even in 64 bits
        return v * torch.sigmoid(2.0 * math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3))
    return v * torch.sigmoid(v) if act == "silu" else v


def check(X, W, Y, bias=None, act="none", residual=None):
    res = None if residual is None else residual.double().clone()
    keep = None
    if Y._base is not None:
        keep = Y._base.clone()
    B.ordermoe_linear(X, W, Y, bias=bias, act=act, residual=residual)
    torch.cuda.synchronize()
    v = X.double() @ W.double().T
    S = X.double().abs() @ W.double().abs().T
    if bias is not None:
        v, S = v + bias.double(), S + bias.double().abs()
    ref = act64(v, act)
    err = 1.13 * (X.shape[1] + 8) * 2.0 ** -23 * S + 2.0 ** -20 * ref.abs()
    if res is not None:
        ref = ref + res
        err = err + 2.0 ** -24 * ref.abs()
    half = 2.0 ** -24 if Y.dtype == torch.float32 else 2.0 ** -8
    off = (Y.double() - ref).abs()
    assert (off <= half * ref.abs() + (1 + half) * err + 1e-38).all(), (off / (half * ref.abs() + err + 1e-38)).max()
    if keep is not None:  # what lies between the rows is as it was
        Y2 = Y.clone()
        Y.copy_(torch.as_strided(keep, Y.shape, Y.stride(), Y.storage_offset()))
        same = Y._base.view(torch.uint8) == keep.view(torch.uint8)
        assert same.all()
        Y.copy_(Y2)


SIZES = [(1, 1, 1), (1, 4096, 4096), (1, 7, 2048), (3, 129, 65), (16, 256, 256), (17, 1000, 520), (33, 5632, 2048),
         (64, 128, 72), (100, 2049, 1999), (128, 640, 4096), (129, 300, 100), (255, 257, 8), (300, 4096, 1024)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("f32", [False, True])
def test_split(M, N, K, f32):
    X, W = rows(M, K, 1.0, 1), rows(N, K, 0.05, 2)
    Y = torch.empty(M, N, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    check(X, W, Y)


# at least 48 tiles of 256 x 256: CTA pairs
PAIRS = [(1021, 4096, 512), (1500, 2561, 328), (4100, 1024, 200), (257, 6300, 64), (8192, 512, 136)]


@pytest.mark.parametrize("M,N,K", PAIRS)
@pytest.mark.parametrize("f32", [False, True])
def test_pairs(M, N, K, f32):
    X, W = rows(M, K, 1.0, 3), rows(N, K, 0.05, 4)
    Y = torch.empty(M, N, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    check(X, W, Y, bias=rows(1, N, 0.5, 5)[0].contiguous(), residual=rows(M, N, 1.0, 6, odd=True))


@pytest.mark.parametrize("M,N,K", [(64, 12289, 264), (101, 14000, 136), (128, 32003, 72), (256, 12050, 328),
                                   (300, 12161, 200), (511, 24700, 64), (66, 19456, 64)])
@pytest.mark.parametrize("f32", [False, True])
def test_pairs_of_narrow_column_tiles(M, N, K, f32):
    """One or two row tiles: the column tiles as wide as the rounds ask for (the last size: 256)."""
    X, W = rows(M, K, 1.0, 31), rows(N, K, 0.05, 32)
    dt = torch.float32 if f32 else torch.bfloat16
    check(X, W, rows(M, N, 1.0, 33, pad=5, odd=True, dt=dt), bias=rows(1, N, 0.5, 34)[0].contiguous(), act="silu")
    W[:, :] = float("nan")  # no column reads another's weights
    W[N // 2] = 0.5
    Y = torch.empty(M, N, dtype=dt, device=DEV)
    B.ordermoe_linear(X, W, Y)
    assert torch.equal(torch.isnan(Y).all(0), torch.arange(N, device=DEV) != N // 2)
    assert torch.isfinite(Y[:, N // 2]).all()


# fewer tiles, many K blocks: two pairs share K, or four (the last two)
PAIR_SPLIT = [(300, 4096, 2056), (512, 4000, 2048), (257, 8100, 2200), (333, 2999, 4096), (200, 8100, 2200),
              (150, 1280, 2048), (300, 700, 2048), (290, 643, 3000), (300, 4096, 6200), (512, 4000, 6144),
              (400, 2000, 2048), (257, 5000, 6400)]


# (The kernels of the sizes above are what the rules give; the sizes below say theirs and check it.)
@pytest.mark.parametrize("M,N,K", PAIR_SPLIT)
def test_pairs_that_share_k(M, N, K):
    X, W = rows(M, K, 1.0, 25), rows(N, K, 0.05, 26)
    Y = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    check(X, W, Y)
    check(X, W, Y, rows(1, N, 0.5, 27)[0].contiguous(), "gelu", rows(M, N, 1.0, 28, odd=True))
    ref = Y.clone()
    B.ordermoe_linear(X, W, Y, bias=rows(1, N, 0.5, 27)[0].contiguous(), act="gelu",
                      residual=rows(M, N, 1.0, 28, odd=True))
    assert torch.equal(Y, ref)
    check(X, W, torch.empty(M, N, device=DEV))


@pytest.mark.parametrize("split,M,N,K", [
    (2, 690, 768, 2048), (2, 401, 2003, 2111), (2, 999, 1001, 2300), (2, 1021, 517, 4100), (2, 330, 1030, 2304),
    (2, 513, 2500, 6150), (2, 260, 3900, 6200), (4, 300, 700, 2048), (4, 290, 643, 3000), (4, 930, 250, 2500),
    (2, 257, 1281, 2057), (4, 320, 600, 2300)])
def test_pairs_that_share_k_in_clusters(split, M, N, K):
    """Ragged products of the kernel whose pairs share K, two and four to a cluster: K blocks that the pairs
    do not share evenly, tiles that end past M and N."""
    plan = B.ordermoe_selftest_linear_plan(M, N, K)
    if split == 4 and plan["kernel"] == "split":
        pytest.skip("fewer than 15 clusters of eight CTAs fit this device: it never takes them")
    assert (plan["kernel"], plan["split"]) == ("pair_split", split), plan
    X, W = rows(M, K, 1.0, 25), rows(N, K, 0.05, 26)
    Y = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    check(X, W, Y)
    bias, R = rows(1, N, 0.5, 27)[0].contiguous(), rows(M, N, 1.0, 28, odd=True)
    for act in ("gelu", "silu"):
        check(X, W, Y, bias, act, R)
    ref, Z = Y.clone(), R.clone()
    B.ordermoe_linear(X, W, Z, bias=bias, act="silu", residual=Z)  # in place, and again
    assert torch.equal(Z, ref)
    wide = rows(M, N, 1.0, 29, pad=13, odd=True, offset=1)
    check(X, W, wide, bias, "relu", R)
    W[:, :] = float("nan")  # no column reads another's weights
    W[N // 2] = 0.5
    B.ordermoe_linear(X, W, Y)
    assert torch.equal(torch.isnan(Y).all(0), torch.arange(N, device=DEV) != N // 2)


@pytest.mark.parametrize("kernel,M,N,K", [
    ("split", 1, 1, 1), ("split", 17, 1000, 520), ("split", 255, 257, 8), ("split", 200, 8100, 2200),
    ("split", 150, 1280, 2048), ("pair", 300, 4096, 1024), ("pair", 300, 4096, 2056), ("pair", 333, 2999, 4096),
    ("pair", 1021, 4096, 512), ("pair", 257, 5000, 6400)])
def test_kernels_of_the_other_sizes(kernel, M, N, K):
    assert B.ordermoe_selftest_linear_plan(M, N, K)["kernel"] == kernel
    X, W = rows(M, K, 1.0, 35), rows(N, K, 0.05, 36)
    check(X, W, torch.empty(M, N, dtype=torch.bfloat16, device=DEV), act="silu", residual=rows(M, N, 1.0, 37))


# How far an fp32 result is off in the 2-norm, of random operands. An MMA adds 16 products to a sum and truncates
# it: half a unit of the last place is lost on average, toward zero; a unit is 0.72 2^-23 of the value (the mean
# over a binade). After j of the n = 32 MMAs of 512 of K the sum's norm is sqrt(j / n) of what it ends with, and the
# losses along them add up to 0.36 2^-23 n / sqrt(3) = 6.6 2^-23 of it; from one 512 of K to the next they are
# independent, as the sums are. Their random part (0.21 2^-23 sqrt(n / 2)) and the additions of the 512s' sums
# (0.21 2^-23 sqrt(28 / 2) for 28 of them) are 0.8 2^-23 each: 6.8 2^-23 = 8.1e-7 in all, for K up to 14336. One
# accumulator over K = 2048 loses 0.36 2^-23 128 / sqrt(3) = 3.2e-6.
F32_OFF = 1e-6


@pytest.mark.parametrize("kernel,M,N", [("split", 1, 4096), ("split", 48, 1000), ("split", 130, 700), ("pair", 300, 4100),
                                        ("pair", 70, 12300)])
@pytest.mark.parametrize("K", [1000, 2048, 6400, 14336])
def test_fp32_results_are_fp32_sums(kernel, M, N, K):
    assert B.ordermoe_selftest_linear_plan(M, N, K, f32=True)["kernel"] == kernel
    X, W = rows(M, K, 1.0, 45), rows(N, K, 0.05, 46)
    Y = torch.empty(M, N, device=DEV)
    B.ordermoe_linear(X, W, Y)
    v = X.double() @ W.double().T
    off = (Y.double() - v).norm()
    assert off <= F32_OFF * v.norm(), float(off / v.norm())
    bias, R = rows(1, N, 0.5, 47)[0].contiguous(), rows(M, N, 1.0, 48)
    B.ordermoe_linear(X, W, Y, bias=bias, residual=R)
    u = v + bias.double()
    off = (Y.double() - (u + R.double())).norm()
    assert off <= F32_OFF * v.norm() + 2.0 ** -24 * (u.norm() + (u + R.double()).norm())


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("M,N,K", [(5, 200, 96), (130, 515, 264), (2048, 2048, 128)])
def test_epilogue(act, M, N, K):
    X, W, b = rows(M, K, 2.0, 7), rows(N, K, 0.1, 8), rows(1, N, 1.0, 9)[0].contiguous()
    R = rows(M, N, 1.0, 10, odd=True)
    for bias in (None, b):
        for res in (None, R):
            for dt in (torch.bfloat16, torch.float32):
                check(X, W, torch.empty(M, N, dtype=dt, device=DEV), bias, act, res)


@pytest.mark.parametrize("M,N,K", [(9, 130, 100), (200, 1023, 512), (1100, 4099, 136)])
def test_strides_and_odd_addresses(M, N, K):
    """Rows inside wider buffers; Y and residual at addresses and strides that no 8-byte access fits."""
    for pad, offset in ((8, 0), (13, 0), (24, 4), (5, 1)):
        X, W = rows(M, K, 1.0, 11, pad=pad // 8 * 8), rows(N, K, 0.1, 12, pad=16)
        R = rows(M, N, 1.0, 13, pad=pad, odd=True, offset=offset)
        for dt in (torch.bfloat16, torch.float32):
            Y = rows(M, N, 1.0, 14, pad=pad, odd=True, dt=dt, offset=offset)
            check(X, W, Y, act="silu", residual=R)


@pytest.mark.parametrize("M,N,K", [(1, 512, 512), (77, 300, 1000), (1500, 2048, 256)])
def test_in_place_and_again(M, N, K):
    """Y may be the residual; the same call gives the same bits."""
    X, W = rows(M, K, 1.0, 15), rows(N, K, 0.1, 16)
    R = rows(M, N, 1.0, 17, pad=8)
    Y = R.clone()
    B.ordermoe_linear(X, W, Y, act="gelu", residual=R)
    for _ in range(3):
        H = R.clone()
        B.ordermoe_linear(X, W, H, act="gelu", residual=H)
        assert torch.equal(H, Y)


@pytest.mark.parametrize("M", [4, 1100])
def test_infinities_and_nan_stay_in_their_rows_and_columns(M):
    N, K = 2600, 128
    X, W = rows(M, K, 1.0, 18), rows(N, K, 0.1, 19)
    Y, Z = (torch.empty(M, N, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    B.ordermoe_linear(X, W, Y, act="relu")
    X[1, 3], W[5, 7], W[9, 0] = float("nan"), float("nan"), float("inf")
    B.ordermoe_linear(X, W, Z, act="relu")
    torch.cuda.synchronize()
    keep = torch.ones(M, N, dtype=torch.bool, device=DEV)
    keep[1], keep[:, 5], keep[:, 9] = False, False, False
    assert torch.equal(Y[keep], Z[keep])
    assert Z[1].isnan().all() and Z[:, 5].isnan().all()
    want = torch.relu(X[:, 0].double() * float("inf"))
    assert torch.equal(Z[[0, 2, 3], 9].double(), want[[0, 2, 3]])


@pytest.mark.parametrize("kernel,N,K", [("split", 8, 8), ("pair", 4100, 8), ("pair_split", 768, 2048)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_tails_of_the_activations(kernel, N, K, f32, act):
    """Sums of one product (exact) from -105 to 105: an activation's negative tail down to the smallest normal
    number of either type (2^-126) is as near as any other value. The exponent s is off by 2^-21 |s| (roundings of the
    cubic or of the square and of the constants: s up to 88) and a bf16 result's fast exponential by (2 + 1.2 |s|) 2^-23 of
    its value: 2^-14 covers them beside the rounding; SiLU's s in fp32 is exact, 2^-20."""
    if kernel == "pair_split" and f32:
        kernel = "pair" if B.ordermoe_selftest_linear_plan(690, N, K, True)["kernel"] == "pair" else "split"
    v = torch.cat([torch.arange(-105.0, -16.0, 0.5), torch.arange(-16.0, 16.0, 0.0625)])
    v = torch.cat([v, torch.arange(16.0, 105.5, 0.5)]).to(DEV)
    v = v[torch.randperm(len(v), generator=torch.Generator().manual_seed(1)).to(DEV)][:690]
    M = len(v)
    assert M == 690 and B.ordermoe_selftest_linear_plan(M, N, K, f32)["kernel"] == kernel
    X, W = torch.zeros(M, K, dtype=torch.bfloat16, device=DEV), torch.zeros(N, K, dtype=torch.bfloat16, device=DEV)
    X[:, 0], W[:, 0] = v.to(torch.bfloat16), 1.0
    assert torch.equal(X[:, 0].float(), v)
    Y = torch.empty(M, N, dtype=torch.float32 if f32 else torch.bfloat16, device=DEV)
    B.ordermoe_linear(X, W, Y, act=act)
    ref = act64(v.double(), act)[:, None]
    tol = (2.0 ** -24 if f32 else 2.0 ** -8) + (2.0 ** -20 if f32 and act == "silu" else 2.0 ** -14)
    normal = (ref.abs() >= 2.0 ** -126).expand(M, N)
    off = (Y.double() - ref).abs()
    assert (off <= tol * ref.abs())[normal].all(), (off / ref.abs())[normal].max()
    assert (Y.double().abs() <= 2.0 ** -125)[~normal].all()


def test_extreme_values():
    """Sums beyond bf16's range, tails of the activations, and zeros."""
    X = torch.tensor([[1.0] * 8, [3e38] * 8, [-3e38] * 8, [0.0] * 8], device=DEV).to(torch.bfloat16)
    W = torch.tensor([[1.0] + [0.0] * 7, [-9.0] + [0.0] * 7, [-1e-3] + [0.0] * 7, [1.0] * 8], device=DEV).to(torch.bfloat16)
    for act in ("none", "relu", "gelu", "gelu_tanh", "silu"):
        Y = torch.empty(4, 4, dtype=torch.float32, device=DEV)
        B.ordermoe_linear(X, W, Y, act=act)
        v = X.float() @ W.float().T
        ref = act64(v.double(), act).float()
        # a value past fp32's range in the cube of gelu_tanh, and inf * 0 in the tails, are torch's NaN too
        ok = torch.isfinite(ref)
        assert torch.allclose(Y[ok], ref[ok], rtol=1e-5, atol=1e-37), (act, Y, ref)
        assert not torch.isnan(Y[torch.isposinf(v)]).any() and (Y[torch.isposinf(v)] > 1e38).all()
        assert torch.equal(Y[3], torch.zeros(4, device=DEV))


def test_no_rows_and_no_others():
    W = rows(64, 64, 0.1, 20)
    Y = torch.empty(0, 64, dtype=torch.bfloat16, device=DEV)
    B.ordermoe_linear(torch.empty(0, 64, dtype=torch.bfloat16, device=DEV), W, Y)
    big = torch.full((9, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    X = rows(6, 64, 1.0, 21)
    B.ordermoe_linear(X, W, big[:6])
    torch.cuda.synchronize()
    assert (big[6:] == 3.0).all()


def test_another_stream_and_a_graph():
    X, W, b = rows(40, 512, 1.0, 22), rows(704, 512, 0.1, 23), rows(1, 704, 1.0, 24)[0].contiguous()
    Y = torch.empty(40, 704, dtype=torch.bfloat16, device=DEV)
    check(X, W, Y, b, "silu")
    ref = Y.clone()
    s = torch.cuda.Stream()
    Z = torch.zeros_like(Y)
    torch.cuda.synchronize()
    B.ordermoe_linear(X, W, Z, bias=b, act="silu", stream=s)
    s.synchronize()
    assert torch.equal(Z, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.ordermoe_linear(X, W, Z, bias=b, act="silu")
        B.ordermoe_linear(Z, W[:, :].T.contiguous(), X[:, :], residual=X)
    X0 = X.clone()
    Z.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(Z, ref)
    want = X0.double() + ref.double() @ W.double()
    assert (X.double() - want).norm() <= 2.0 ** -8 * want.norm()


@pytest.mark.parametrize("T", [2, 16, 70])
@pytest.mark.parametrize("few", [False, True])
def test_stack_of_moe_and_dense_layers(T, few):
    """MoE and dense layers in turn on the residual map, eager and as a graph, against the same
    layers in 64 bits from each layer's own bf16 inputs. A layer's sum is off by the roundings of
    its inner activations (2^-8 each of the expert outputs and of H) and h_out by one: 4 * 2^-8
    of the update and 2^-8 of the stream bound its 2-norm."""
    d, E, k, dff, M, L = 512, 8, 2, 256, 2, 4
    layers, tabs = [], []
    for l in range(L):
        W1, W3, W2 = synth.ffn_weights(E, d, dff, 100 * l, device=DEV)
        if l % 2:
            layers.append(DenseFFN(W1[0], W2[0], T, b1=rows(1, dff, 0.1, l)[0].contiguous(),
                                   b2=rows(1, d, 0.1, l + 9)[0].contiguous()))
        else:
            layers.append({"W_r": synth.router_weights(E, d, 2, l, device=DEV), "W1": W1, "W3": W3, "W2": W2})
            tabs.append(exact_tables(E, M, DEV))
    st = LayerStack(layers, tabs, k, T, DEV, few=few)
    home = torch.zeros(T, dtype=torch.uint8, device=DEV)
    loc, q = home.clone(), torch.zeros(T, device=DEV)
    hs = [synth.hidden(T, d, 5, DEV)] + [torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in range(L)]
    xs = [torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in range(L + 1)]
    st.step_residual(hs, xs, home, loc, q)
    torch.cuda.synchronize()
    for l, lay in enumerate(layers):
        x, h = xs[l].double(), hs[l].double()
        if isinstance(lay, DenseFFN):
            y = torch.relu(x @ lay.W1.double().T + lay.b1.double()) @ lay.W2.double().T + lay.b2.double()
        else:
            w, idx = torch.topk(torch.softmax(x @ lay["W_r"].double().T, 1), k, dim=1)
            w = w / w.sum(1, keepdim=True)
            y = torch.zeros_like(x)
            for t in range(T):
                for j in range(k):
                    e = idx[t, j]
                    a = lay["W1"][e].double() @ x[t]
                    y[t] += w[t, j] * (lay["W2"][e].double() @ (a * torch.sigmoid(a) * (lay["W3"][e].double() @ x[t])))
        want = h + y
        off = (hs[l + 1].double() - want).norm()
        assert off <= 2.0 ** -8 * (want.norm() + 4 * y.norm()), l
        n = hs[l + 1].double()
        n = n / (n.square().mean(1, keepdim=True) + B.NORM_EPS).sqrt()
        assert ((xs[l + 1].double() - n).abs() <= 2.0 ** -7 * n.abs() + 1e-30).all()
    eager = [v.clone() for v in hs]
    g = st.capture_residual(hs, xs, home, loc, q, prologue=lambda: (loc.copy_(home), q.zero_()))
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(eager, hs))


@pytest.mark.parametrize("T,d,dff", [(1, 64, 100), (6, 64, 9), (70, 256, 501), (300, 512, 1001), (5, 64, 1)])
def test_dense_layers_of_any_width(T, d, dff):
    """A d_ff that is no multiple of 8. H is rounded once (2^-8) and carries the first product's bound; y is
    off by W2 times that and by its own sum's and rounding's."""
    W1, W2 = rows(dff, d, 0.1, 70, odd=True).clone(), rows(d, dff, 0.1, 71, odd=True).clone()
    b1, b2 = rows(1, dff, 0.5, 72)[0].contiguous(), rows(1, d, 0.5, 73)[0].contiguous()
    x, h = rows(T, d, 1.0, 74), rows(T, d, 1.0, 75)
    y = torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    DenseFFN(W1, W2, T, b1=b1, b2=b2).forward(x, y, residual=h)
    X, A1, A2 = x.double(), W1.double(), W2.double()
    g = X @ A1.T + b1.double()
    S = X.abs() @ A1.abs().T + b1.double().abs()
    H = g.clamp(min=0.0)
    dH = 2.0 ** -8 * H + (1 + 2.0 ** -8) * (d + 8) * 2.0 ** -23 * S
    ref = H @ A2.T + b2.double() + h.double()
    mag = (H + dH) @ A2.abs().T + b2.double().abs()
    err = dH @ A2.abs().T + (dff + 8) * 2.0 ** -23 * mag + 2.0 ** -24 * ref.abs()
    off = (y.double() - ref).abs()
    assert (off <= 2.0 ** -8 * ref.abs() + (1 + 2.0 ** -8) * err).all(), (off / (2.0 ** -8 * ref.abs() + err)).max()


@pytest.mark.parametrize("few", [False, True])
def test_stack_of_dense_layers_alone(few):
    """No MoE layer: a step and its graph give what the layers give one by one."""
    T, d, dff, L = 5, 256, 384, 3
    dense = [DenseFFN(rows(dff, d, 0.1, 80 + l), rows(d, dff, 0.1, 90 + l), T, act="gelu") for l in range(L)]
    st = LayerStack(dense, [], 1, T, DEV, few=few)
    hs = [synth.hidden(T, d, 6, DEV)] + [torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in range(L)]
    xs = [torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in range(L + 1)]
    home = torch.zeros(T, dtype=torch.uint8, device=DEV)
    st.step_residual(hs, xs, home, None, None)
    want = [hs[0].clone()]
    x = torch.zeros_like(hs[0])
    B.ordermoe_rmsnorm(want[0], T, d, B.NORM_EPS, x)
    for lay in dense:
        want.append(torch.zeros_like(hs[0]))
        lay.forward_residual(x.clone(), want[-2], want[-1], x)
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(hs, want)) and torch.equal(xs[-1], x)
    g = st.capture_residual(hs, xs, home, None, None)
    for h in hs[1:]:
        h.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(hs, want))


@pytest.mark.parametrize("kinds", ["MDMDM", "DMM", "MD", "DMDDMD"])
def test_a_stack_with_dense_layers_is_calibrated(kinds):
    """Similarities, counts and transitions are those of the MoE layers, from each one's own inputs, in the
    order of LayerStack's tables and P; then the stack runs with them and looks ahead."""
    d, E, k, dff, M, N = 512, 8, 2, 256, 2, 700
    layers = []
    for l, kind in enumerate(kinds):
        W1, W3, W2 = synth.ffn_weights(E, d, dff, 200 * l, device=DEV)
        layers.append(DenseFFN(W1[0], W2[0], 4) if kind == "D" else
                      {"W_r": synth.router_weights(E, d, 2, l, device=DEV), "W1": W1, "W3": W3, "W2": W2})
    moe = [l for l, kind in enumerate(kinds) if kind == "M"]
    L = len(moe)
    cal = calibrate_stack(layers, synth.calibration(N, d, 7, device=DEV), k, M)
    torch.cuda.synchronize()
    assert len(cal["hs"]) == len(cal["xs"]) == len(kinds) + 1
    assert cal["sim"].shape == (L, E, E) and cal["counts"].shape == (L, E) and cal["logits"].shape == (L, N, E)
    assert cal["P"].shape == cal["tcount"].shape == (L - 1, E, E)
    logits = cal["logits"].cpu().numpy()
    for i, l in enumerate(moe):
        x, Wr = cal["xs"][l], layers[l]["W_r"]
        ref, mag = x.double() @ Wr.double().T, x.double().abs() @ Wr.double().abs().T
        assert ((cal["logits"][i].double() - ref).abs() <= (d + 8) * 2.0 ** -23 * mag).all()
        o_sim = oracle.similarity(synth.bits(Wr), synth.bits(x))
        np.testing.assert_allclose(cal["sim"][i].cpu().numpy(), o_sim, atol=2e-5)
        assert cal["counts"][i].sum() == N * k
    for l, kind in enumerate(kinds):
        if kind == "D":  # it ran, in its place
            x, W1, W2 = cal["xs"][l].double(), layers[l].W1.double(), layers[l].W2.double()
            y = torch.relu(x @ W1.T) @ W2.T
            want = cal["hs"][l].double() + y
            assert (cal["hs"][l + 1].double() - want).norm() <= 2.0 ** -8 * (want.norm() + 4 * y.norm())
    if L > 1:
        ref_c, ref_P = oracle.transitions(np.ascontiguousarray(logits.transpose(1, 0, 2)), k)
        np.testing.assert_array_equal(cal["tcount"].cpu().numpy(), ref_c)
        np.testing.assert_array_equal(cal["P"].cpu().numpy().view(np.uint32), ref_P.view(np.uint32))
    # the plan's tables from these similarities, and two steps with the horizon that P allows
    stride = B.ordermoe_tables_bytes(E, M)
    tabs = torch.zeros(L * stride, dtype=torch.uint8, device=DEV)
    place = np.zeros((M, E), np.uint8)
    place[np.arange(E) % M, np.arange(E)] = 1
    for i in range(L):
        build_tables(cal["sim"][i], (np.arange(E) // 4).astype(np.int32), place, 0.1, 0.3,
                     synth.server_params(M, d, dff, 0), DEV, out=tabs[i * stride:(i + 1) * stride])
    T = 4
    home = torch.as_tensor(synth.homes(T, M, 1)).to(DEV)
    out = []
    for few in (False, True):
        st = LayerStack(layers, tabs, k, T, DEV, H=3, stride=stride, P=cal["P"], few=few)
        hs = [cal["hs"][0][:T].clone()] + [torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in kinds]
        xs = [torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in range(len(kinds) + 1)]
        st.step_residual(hs, xs, home, home.clone(), torch.zeros(T, device=DEV))
        torch.cuda.synchronize()
        out.append(hs)
    for l, (u, v) in enumerate(zip(*out)):  # as test_stack_of_few_tokens: 2^-8 of H, Y, h a layer
        assert (u.double() - v.double()).norm() <= 4 * 2.0 ** -8 * max(l, 1) * u.double().norm()


def test_short_products_behind_long_ones_on_two_streams():
    """Every kernel behind every other, launched eagerly, two streams side by side: TMEM of a CTA is free when it asks."""
    sizes = [(1021, 4096, 512), (1, 256, 64), (300, 2048, 2048), (16, 256, 256), (4096, 128, 64), (128, 2048, 4096),
             (1, 2048, 8192), (100, 12289, 128)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    sets = [[(rows(M, K, 1.0, 40 + i), rows(N, K, 0.05, 60 + i), torch.empty(M, N, dtype=dt, device=DEV))
             for i, (M, N, K) in enumerate(sizes)] for dt in (torch.bfloat16, torch.float32)]
    torch.cuda.synchronize()
    for turn in range(20):
        for i in range(len(sizes)):
            for st, work in zip(streams, sets):
                with torch.cuda.stream(st):
                    B.ordermoe_linear(*work[(i * (turn % 7 + 1) + turn) % len(sizes)])
    torch.cuda.synchronize()
    for work in sets:
        for X, W, Y in work:
            first = Y.clone()
            check(X, W, Y)
            assert torch.equal(first, Y)
