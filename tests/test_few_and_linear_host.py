"""What needs no GPU of the few-token layer and of the matrix product: the C ABI's refusals, found
before anything is enqueued (addresses that are passed are not read), sizes of the workspace,
the binding's checks, and barriers read from the sources."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2607_17154_gb300 import binding as B

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2607_17154_gb300", "csrc")
OK, ARG, SHAPE = B.OK, B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED_SHAPE
AT = 1 << 20  # an aligned address that a refused call never reads
N = None


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_17154_gb300 import build
    build.build()


def desc(**over):
    v = dict(T_max=1, E=8, d=256, dff=512, k=2, renorm=1, W_r=AT, W1=AT, W3=AT, W2=AT, tables=AT,
             tables_bytes=1 << 16, scratch=N, scratch_bytes=0, lookahead_H=1, tables_stride=0, P=N)
    v.update(over)
    return B.LayerDesc(**v)


def few(d=None, T=4, X=AT, home=AT, loc=N, qhat=N, y=AT, ws=AT, nbytes=1 << 30):
    rc = B.lib().ordermoe_layer_few(ctypes.byref(d or desc()), T, X, home, loc, qhat, y, N, ws, nbytes, N)
    return rc, B.lib().ordermoe_last_error().decode()


@pytest.mark.parametrize("over,code", [
    (dict(E=0), SHAPE), (dict(E=65), SHAPE), (dict(k=0), SHAPE), (dict(k=9, E=16), SHAPE), (dict(k=9), SHAPE),
    (dict(d=128), SHAPE), (dict(d=0), SHAPE), (dict(d=33024), SHAPE), (dict(dff=64), SHAPE), (dict(dff=0), SHAPE),
    (dict(E=64, dff=1 << 26), SHAPE), (dict(lookahead_H=5), SHAPE),
    (dict(W_r=N), ARG), (dict(W1=N), ARG), (dict(W3=N), ARG), (dict(W2=N), ARG), (dict(tables=N), ARG),
    (dict(W_r=AT + 8), ARG), (dict(W1=AT + 2), ARG), (dict(W2=AT + 8), ARG), (dict(tables=AT + 8), ARG),
    (dict(tables_bytes=100), ARG)])
def test_layers_that_layer_few_refuses(over, code):
    for T in (4, 0):  # also where there is nothing to do
        rc, msg = few(desc(**over), T=T)
        assert rc == code and msg.startswith("layer_few:"), (over, rc, msg)


@pytest.mark.parametrize("call,code", [
    (dict(T=-1), ARG), (dict(T=17), SHAPE), (dict(X=N), ARG), (dict(home=N), ARG), (dict(y=N), ARG), (dict(X=AT + 8), ARG),
    (dict(y=AT + 2), ARG), (dict(loc=AT), ARG), (dict(qhat=AT), ARG), (dict(ws=N), ARG), (dict(ws=AT + 16), ARG),
    (dict(nbytes=1000), ARG)])
def test_calls_that_layer_few_refuses(call, code):
    rc, msg = few(**call)
    assert rc == code and msg.startswith("layer_few:"), (call, rc, msg)


@pytest.mark.parametrize("over", [dict(P=N), dict(tables_stride=0), dict(tables_stride=100),
                                  dict(tables_stride=4104)])
@pytest.mark.parametrize("T", [4, 0])
def test_look_ahead_is_refused_before_anything_is_enqueued(over, T):
    """The decisions of a look-ahead are prepared by a copy of their own on the stream: without a GPU that
    copy fails, so a refusal that came behind it would be another error."""
    rc, msg = few(desc(**dict(dict(lookahead_H=2, tables_stride=4096, P=AT), **over)), T=T)
    assert rc == ARG and msg.startswith("layer_few:"), (rc, msg)


def test_no_tokens():
    assert few(T=0, X=N, home=N, y=N, ws=N, nbytes=0)[0] == OK
    assert B.lib().ordermoe_layer_few(N, 0, N, N, N, N, N, N, N, 0, N) == ARG


def test_layer_few_residual_refuses():
    d = desc()

    def call(T=4, x=AT, h=AT, eps=1e-6, h_out=AT, x_out=AT):
        return B.lib().ordermoe_layer_few_residual(ctypes.byref(d), T, x, AT, AT, N, N, eps, h_out, x_out, N, AT, 0, N) \
            if h else B.lib().ordermoe_layer_few_residual(ctypes.byref(d), T, x, N, AT, N, N, eps, h_out, x_out, N, AT, 0, N)
    for kw in (dict(h=N), dict(x_out=N), dict(h_out=N), dict(x=N), dict(eps=0.0), dict(eps=-1.0),
               dict(eps=float("nan")), dict(x_out=AT + 8), dict(h_out=AT + 8), dict()):  # the last: no workspace
        assert call(**kw) == ARG, kw
        assert B.lib().ordermoe_last_error().decode().startswith("layer_few_residual:")


def test_workspace_sizes():
    size = B.ordermoe_layer_few_workspace_bytes
    for shape in ((8, 256, 512, 2), (64, 2048, 1408, 6), (8, 4096, 14336, 2)):
        sizes = [size(T, *shape) for T in range(1, 17)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:])) and sizes[0] > 0  # enough for every smaller T
        E, d, dff, k = shape
        assert sizes[-1] >= min(E, 16 * k) * 16 * dff * 2
    for bad in ((0, 8, 256, 512, 2), (17, 8, 256, 512, 2), (4, 65, 256, 512, 2), (4, 8, 0, 512, 2), (4, 8, 256, 512, 9),
                (4, 2, 256, 512, 3)):
        assert size(*bad) == 0
    assert B.lib().ordermoe_layer_few_init(N, 1 << 20, N) == ARG
    assert B.lib().ordermoe_layer_few_init(AT, 128, N) == ARG
    assert B.lib().ordermoe_layer_few_init(AT + 64, 1 << 20, N) == ARG


def test_a_workspace_is_ready_for_any_stream_when_it_is_returned(monkeypatch):
    """The counters are cleared on the stream that is current where it is made; a first call on another
    stream is ordered behind nothing. So the clearing has ended before anyone has the workspace."""
    from contextlib import nullcontext

    from paper_2607_17154_gb300 import layer
    done, capturing = [], [False]

    class Stream:
        def synchronize(self):
            done.append("wait")
    monkeypatch.setattr(B, "ordermoe_layer_few_init", lambda ws, stream=None: done.append("clear"))
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, device=None, **kw: empty(*a, **kw))
    monkeypatch.setattr(torch.cuda, "device", lambda d: nullcontext())
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing[0])
    layer.few_workspace(4, 8, 256, 512, 2, "cuda:0")
    assert done == ["clear", "wait"]
    capturing[0] = True  # nothing to wait for
    layer.few_workspace(4, 8, 256, 512, 2, "cuda:0")
    assert done == ["clear", "wait", "clear"]


def test_what_replaces_a_layers_tensors_reaches_its_few_token_calls(monkeypatch):
    """forward() reads a layer's weights, tables and buffers at every call; so must forward_few(), whose
    descriptors are made before (a plan made again puts new tables in place of the old)."""
    from paper_2607_17154_gb300 import layer
    seen = []
    monkeypatch.setattr(layer, "few_workspace", lambda *a: torch.zeros(1 << 12, dtype=torch.uint8))
    monkeypatch.setattr(B, "ordermoe_layer_few", lambda desc, T, X, home, loc, qhat, y, ws, out, stream: seen.append((desc, out)))
    monkeypatch.setattr(B, "_ptr", lambda t: t.data_ptr() if t is not None else None)
    bf = torch.bfloat16
    Wr, W1, W2 = torch.zeros(4, 256, dtype=bf), torch.zeros(4, 128, 256, dtype=bf), torch.zeros(4, 256, 128, dtype=bf)
    tables = torch.zeros(B.ordermoe_tables_bytes(4, 1), dtype=torch.uint8)
    m = layer.MoELayer(Wr, W1, W1.clone(), W2, tables, 2, 4, few=True)
    x = torch.zeros(4, 256, dtype=bf)
    for name in ("tables", "W_r", "W1", "W3", "W2"):
        old = getattr(m, name)
        setattr(m, name, old.clone())
        m.forward_few(x, None, None, None, x)
        assert getattr(seen[-1][0], name) == getattr(m, name).data_ptr() != old.data_ptr(), name
    for name, field in (("logits", "logits"), ("topk_idx", "topk_idx"), ("topk_w", "topk_w"), ("chosen", "chosen_expert"),
                        ("server", "chosen_server"), ("kind", "kind"), ("counters", "counters")):
        setattr(m, name, getattr(m, name).clone())
        m.forward_few(x, None, None, None, x)
        assert getattr(seen[-1][1], field) == getattr(m, name).data_ptr(), name
    m.renorm, m.k = 0, 1
    m.forward_few(x, None, None, None, x)
    assert (seen[-1][0].renorm, seen[-1][0].k) == (0, 1)


def linear(X=AT, ldx=64, W=AT, ldw=64, bias=N, act=0, residual=N, ldr=0, M=4, n=32, K=64, Y=AT, ldy=32, f32=0):
    rc = B.lib().ordermoe_linear(X, ldx, W, ldw, bias, act, residual, ldr, M, n, K, Y, ldy, f32, N)
    return rc, B.lib().ordermoe_last_error().decode()


@pytest.mark.parametrize("call,code", [
    (dict(M=-1), ARG), (dict(n=0), ARG), (dict(K=0), ARG), (dict(act=-1), ARG), (dict(act=5), ARG),
    (dict(ldx=56), ARG), (dict(ldw=63), ARG), (dict(ldy=31), ARG), (dict(residual=AT, ldr=31), ARG),
    (dict(ldx=65), SHAPE), (dict(ldw=68), SHAPE), (dict(ldx=1 << 38), SHAPE), (dict(ldw=1 << 40), SHAPE),
    (dict(X=N), ARG), (dict(W=N), ARG), (dict(Y=N), ARG), (dict(X=AT + 8), ARG), (dict(W=AT + 2), ARG),
    (dict(Y=AT + 1), ARG), (dict(Y=AT + 2, f32=1), ARG), (dict(bias=AT + 1), ARG), (dict(residual=AT + 1, ldr=32), ARG)])
def test_calls_that_linear_refuses(call, code):
    rc, msg = linear(**call)
    assert rc == code and msg.startswith("linear:"), (call, rc, msg)


@pytest.mark.parametrize("call,code", [
    (dict(residual=AT, ldr=32, f32=1), ARG),            # each row of floats covers two of the residual's
    (dict(residual=AT, ldr=40), ARG),
    (dict(M=2 ** 31 - 100), SHAPE), (dict(n=2 ** 31 - 300, ldy=2 ** 32), SHAPE),
    (dict(K=2 ** 31 - 60, ldx=2 ** 32, ldw=2 ** 32), SHAPE)])
def test_results_in_place_and_sizes_that_linear_refuses(call, code):
    rc, msg = linear(**call)
    assert rc == code and msg.startswith("linear:"), (call, rc, msg)


GB300 = (152, 76, 36, 16)  # SMs, CTA pairs, clusters of two pairs and of four that are resident at once


@pytest.mark.parametrize("sizes,kernel,split", [
    ((1, 4096, 4096), "split", 8), ((33, 5632, 2048), "split", None), ((64, 128, 72), "split", 1),
    ((200, 8100, 2200), "split", 2), ((64, 12289, 264), "pair", 1), ((300, 4096, 2056), "pair", 1),
    ((1021, 4096, 14336), "pair", 1), ((690, 768, 2048), "pair_split", 2), ((401, 2003, 2111), "pair_split", 2),
    ((300, 700, 2048), "pair_split", 4), ((930, 250, 2500), "pair_split", 4), ((513, 2500, 6150), "pair_split", 2)])
def test_kernels_that_the_product_takes(sizes, kernel, split):
    p = B.ordermoe_selftest_linear_plan(*sizes, device=GB300)
    assert p["kernel"] == kernel and (split is None or p["split"] == split), p


@pytest.mark.parametrize("device", [GB300, (152, 76, 38, 19), (152, 76, 30, 0), (148, 74, 33, 14), (2, 1, 0, 0)])
@pytest.mark.parametrize("f32", [False, True])
def test_tiles_of_the_product(device, f32):
    """For sizes over the whole range: the tiles cover Y once and no row or column of tiles is empty, a
    tile's accumulator and sums fit, and the grid is what the kernel's index arithmetic takes."""
    rng = __import__("random").Random(17)
    sms, pairs, c2, c4 = device
    kinds = set()
    for _ in range(4000):
        M, n, K = (int(round(a * (b / a) ** rng.random())) for a, b in ((1, 20000), (1, 70000), (1, 40000)))
        p = B.ordermoe_selftest_linear_plan(M, n, K, f32, device)
        kinds.add((p["kernel"], p["split"]))
        blocks = (K + 63) // 64
        assert (p["row_tiles"] - 1) * p["rows"] < M <= p["row_tiles"] * p["rows"], (M, n, K, p)
        assert (p["col_tiles"] - 1) * p["cols"] < n <= p["col_tiles"] * p["cols"], (M, n, K, p)
        tiles = p["row_tiles"] * p["col_tiles"]
        if p["kernel"] == "split":
            assert p["rows"] % 16 == 0 and p["rows"] <= (64 if f32 else 128) and p["cols"] % 16 == 0 and 80 <= p["cols"] <= 128
            assert p["split"] in (1, 2, 4, 8) and p["split"] <= blocks and p["grid"] == tiles * p["split"]
            stage = (p["rows"] + p["cols"]) * 128  # bytes; the last one's weights are read as 128 rows
            assert 1 <= p["stages"] <= 12 and p["stages"] * stage >= p["rows"] * 512
            assert p["stages"] * stage + max(0, 128 * 128 - stage) + 1024 <= 221 * 1024
        elif p["kernel"] == "pair":
            assert p["rows"] % 32 == 0 and p["rows"] <= (128 if f32 else 256) and p["cols"] % 16 == 0 and p["cols"] <= 256
            assert p["grid"] == 2 * min(tiles, pairs) and M >= 64
        else:
            assert not f32 and p["rows"] % 32 == 0 and p["rows"] <= 256 and p["cols"] == 256 and M > 256
            assert p["split"] in (2, 4) and tiles <= (c2 if p["split"] == 2 else c4)
            assert p["grid"] == 2 * p["split"] * tiles and p["split"] <= blocks
    if sms > 100:
        assert {("split", 1), ("split", 2), ("split", 4), ("split", 8), ("pair", 1)} <= kinds
        assert f32 or ("pair_split", 2) in kinds and (c4 == 0 or ("pair_split", 4) in kinds)


def test_linear_plan_refuses():
    plan = (ctypes.c_int * 8)()
    call = B.lib().ordermoe_selftest_linear_plan
    for args in ((0, 1, 1, 0, N, plan), (1, 0, 1, 0, N, plan), (1, 1, 0, 0, N, plan), (1, 1, 1, 0, N, N),
                 (1, 1, 1, 0, (ctypes.c_int * 4)(1, 1, 0, 0), plan), (1, 1, 1, 0, (ctypes.c_int * 4)(152, 0, 0, 0), plan)):
        assert call(*args) == ARG
        assert B.lib().ordermoe_last_error().decode().startswith("selftest_linear_plan:")
    big = (2 ** 31 - 600, 2 ** 31 - 600, 64, 0, (ctypes.c_int * 4)(*GB300), plan)
    assert call(*big) == SHAPE


def test_bound_of_fp32_results_sees_the_length_of_an_accumulator():
    """The bound on sums that are truncated as above, on the host: 512 of K a sum within it, all of K not."""
    from tests.test_gpu_linear import F32_OFF
    rng = np.random.default_rng(3)
    for K in (2048, 6400):
        x, w = (rng.standard_normal((300, K)).astype(np.float32) for _ in range(2))
        steps = (x.astype(np.float64) * w).reshape(300, K // 16, 16).sum(2)
        ref = steps.sum(1)

        def trunc(v):
            f = v.astype(np.float32)
            return np.where(np.abs(f.astype(np.float64)) > np.abs(v), np.nextafter(f, np.float32(0)), f)

        def off(per):
            total = np.zeros(300, np.float32)
            for c in range(0, K // 16, per):
                acc = np.zeros(300, np.float32)
                for j in range(c, min(c + per, K // 16)):
                    acc = trunc(acc.astype(np.float64) + steps[:, j])
                total = total + acc
            return np.linalg.norm(total - ref) / np.linalg.norm(ref)
        assert off(32) <= F32_OFF < off(K // 16)


def test_linear_of_no_rows():
    assert linear(M=0, X=N, W=N, Y=N)[0] == OK


def test_binding_refuses_host_tensors_types_and_shapes(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    bf = torch.bfloat16
    X, W, Y = torch.zeros(4, 64, dtype=bf), torch.zeros(32, 64, dtype=bf), torch.zeros(4, 32, dtype=bf)
    for args, err in (((X, W, Y), ValueError),                                     # not on the GPU
                      ((X.float(), W, Y), TypeError), ((X[0], W, Y), TypeError),
                      ((X, W, None), TypeError)):
        with pytest.raises(err):
            B.ordermoe_linear(*args)
    with pytest.raises(ValueError):
        B.ordermoe_linear(X, W, Y, act="tanh")

    class Fake:  # a device tensor
        def __init__(self, device, stride=(64, 1), dtype=bf):
            self.dtype, self.shape, self.device_, self.stride_ = dtype, (4, 64), device, stride

        def get_device(self):
            return self.device_

        def stride(self, i):
            return self.stride_[i]

        def data_ptr(self):
            return AT
    assert B._matrix(Fake(0), "X", (4, 64), 0) == (AT, 64)
    assert B._matrix(Fake(0, (80, 1)), "X", (4, 64), 0) == (AT, 80)
    for t, shape, err, what in ((Fake(1), (4, 64), ValueError, "current device"), (Fake(0), (4, 63), ValueError, "must be"),
                                (Fake(0, dtype=torch.float16), (4, 64), TypeError, "must be"),
                                (Fake(0, (1, 4)), (4, 64), ValueError, "contiguous"),
                                (Fake(0, (0, 1)), (4, 64), ValueError, "overlap")):
        with pytest.raises(err, match=what):
            B._matrix(t, "X", shape, 0)
    with pytest.raises(ValueError):
        B._entries(X, "X", bf, 4 * 64, 0)
    with pytest.raises(TypeError):
        B._entries(X, "X", torch.float32, 1, 0)
    assert B._entries(None, "loc", torch.uint8, 4, 0) is None
    with pytest.raises(ValueError):
        u8 = torch.zeros(1 << 12, dtype=torch.uint8)
        B.ordermoe_layer_few(desc(), 4, X, u8, None, None, X, u8)


@pytest.mark.parametrize("d,dff", [(64, 100), (64, 1), (72, 9), (20, 36), (64, 128)])
def test_dense_layers_hand_on_rows_that_the_product_takes(monkeypatch, d, dff):
    """Whatever d_ff is, both products of a DenseFFN get weights and activations whose rows start at
    multiples of 16 bytes, with the caller's values."""
    from paper_2607_17154_gb300 import layer
    bf, calls = torch.bfloat16, []
    W1, W2 = torch.randn(dff, d).to(bf), torch.randn(d, dff).to(bf)
    monkeypatch.setattr(B, "ordermoe_linear", lambda X, W, Y, **kw: calls.append((X, W, Y, kw)))
    m = layer.DenseFFN(W1, W2, 5)
    x, y = torch.zeros(5, (d + 7) // 8 * 8, dtype=bf)[:, :d], torch.zeros(5, d, dtype=bf)
    m.forward(x, y, residual=y)
    (X, V1, H, k1), (H2, V2, Y, k2) = calls
    for t in (V1, V2, H, H2):
        assert t.stride(0) % 8 == 0 and t.data_ptr() % 16 == 0 and (t.shape[1] == 1 or t.stride(1) == 1)
    assert torch.equal(V1, W1) and torch.equal(V2, W2)
    assert H.shape == H2.shape == (5, dff) and H.data_ptr() == H2.data_ptr() and H.stride() == H2.stride()
    assert X is x and Y is y and k1["act"] == "relu" and k2["residual"] is y
    if d % 8 == 0 and dff % 8 == 0:  # nothing is copied
        assert V1 is W1 and V2 is W2


@pytest.mark.parametrize("few", [False, True])
def test_a_stack_of_dense_layers_alone(monkeypatch, few):
    from paper_2607_17154_gb300 import layer
    bf, calls = torch.bfloat16, []
    monkeypatch.setattr(B, "ordermoe_linear", lambda X, W, Y, **kw: calls.append((X, W, Y, kw["residual"] if "residual" in kw else None)))
    monkeypatch.setattr(B, "ordermoe_rmsnorm", lambda h, T, d, eps, x, stream: calls.append((h, x)))
    dense = [layer.DenseFFN(torch.zeros(128, 64, dtype=bf), torch.zeros(64, 128, dtype=bf), 4) for _ in range(2)]
    st = layer.LayerStack(dense, [], 0, 4, "cpu", few=few)
    xs, hs = [torch.zeros(4, 64, dtype=bf) for _ in range(3)], [torch.zeros(4, 64, dtype=bf) for _ in range(3)]
    st.step(xs[:2], None, None, None, hs[:2])
    assert [c[2] is y for c, y in zip(calls[1::2], hs)] == [True, True] and len(calls) == 4
    calls.clear()
    st.step_residual(hs, xs, None, None, None)
    assert len(calls) == 7 and calls[0] == (hs[0], xs[0]) and calls[3] == (hs[1], xs[1]) and calls[6] == (hs[2], xs[2])
    assert calls[1][0] is xs[0] and calls[2][3] is hs[0] and calls[2][2] is hs[1]
    with pytest.raises(ValueError):
        layer.LayerStack([], [], 2, 4, "cpu")


def test_calibration_counts_the_moe_layers_of_a_stack(monkeypatch):
    """Of MoE, dense, MoE: each MoE layer's own inputs and logits, in order; the dense one with room for all
    calibration tokens."""
    from paper_2607_17154_gb300 import layer
    bf, N, d, E, seen = torch.bfloat16, 9, 64, 4, {}

    class Stack:
        def __init__(self, layers, tables, k, T_max, device):
            seen.update(layers=layers, tables=tables)

        def step_residual(self, hs, xs, home, loc, qhat, logits, eps):
            seen.update(hs=hs, xs=xs, logits=logits)
    monkeypatch.setattr(layer, "LayerStack", Stack)
    monkeypatch.setattr(layer, "exact_tables", lambda *a: "tables")
    monkeypatch.setattr(B, "ordermoe_similarity_no_logits", lambda W, x, *a: seen.setdefault("sim", []).append((W, x)))
    monkeypatch.setattr(B, "ordermoe_transitions_strided", lambda lg, *a: seen.update(trans=(lg, a)))
    dense = layer.DenseFFN(torch.ones(128, d, dtype=bf), torch.ones(d, 128, dtype=bf), 2)
    lays = [{"W1": torch.zeros(E, 128, d), "W_r": torch.zeros(E, d)} for _ in range(2)]
    cal = layer.calibrate_stack([lays[0], dense, lays[1]], torch.zeros(N, d, dtype=bf), 2, 1)
    assert seen["tables"] == ["tables"] * 2 and seen["layers"][0] is lays[0] and seen["layers"][2] is lays[1]
    assert seen["layers"][1].T_max == N and torch.equal(seen["layers"][1].W1, dense.W1)
    assert len(seen["hs"]) == len(seen["xs"]) == 4 and seen["logits"][1] is None
    lg = cal["logits"]
    assert lg.shape == (2, N, E) and [t.data_ptr() for t in (seen["logits"][0], seen["logits"][2])] == [t.data_ptr() for t in lg]
    assert [(w is l["W_r"]) for (w, _), l in zip(seen["sim"], lays)] == [True, True]
    assert seen["sim"][0][1] is seen["xs"][0] and seen["sim"][1][1] is seen["xs"][2]
    assert seen["trans"][0] is lg and seen["trans"][1][:3] == (N, 2, E)
    assert cal["sim"].shape == (2, E, E) and cal["P"].shape == (1, E, E)
    with pytest.raises(ValueError):
        layer.calibrate_stack([dense], torch.zeros(N, d, dtype=bf), 2, 1)


def kernel(path, name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())
    start = text.index("{", text.index(name + "("))
    depth = 0
    for i in range(start, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if depth == 0:
            return text[start:i]


def test_cluster_barriers_around_the_accesses_to_a_peer():
    """The peers' shared memory is reached through helpers: behind a cluster barrier (every CTA runs),
    and no CTA leaves before another barrier."""
    for path, name, helper in (("linear.cu", "linear_split_kernel", "load_rank("),
                               ("linear.cu", "linear_pair_kernel", "lead_barrier("),
                               ("linear.cu", "linear_pair_split_kernel", "pair_barrier("),
                               ("linear.cu", "linear_pair_split_kernel", "load_rank("),
                               ("few_tokens.cu", "few_tokens_kernel", "store_both(")):
        body = kernel(path, name)
        assert "mapa_shared(" not in body
        first, last = body.index(helper), body.rindex(helper)
        assert 0 <= body.find("cluster_sync()") < first, name
        assert body.find("cluster_sync()", last) > last, name


def test_waits_of_the_new_kernels_are_bounded():
    """Every wait goes through a helper that takes a limit; no loop tries a barrier by itself."""
    for path in ("few_tokens.cu", "linear.cu"):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, path)).read())
        assert "mbar_try_wait" not in text
        assert all("limit_ns" in m for m in re.findall(r"mbar_wait\((.*?)\)\)?[;,)]", text, flags=re.S))
        assert text.count("while (true)") == text.count("for (;;)") == 0
    body = kernel("few_tokens.cu", "bool grid_wait")
    assert "limit_ns" in body and "return false" in body
