"""The few-token layer (ordermoe_layer_few, ordermoe_layer_few_residual) against the
oracle's decisions on its own logits and the experts' formulas in 64 bits.

Tolerance of y = bf16(sum_j w_j W2 H_j), H = silu(g) u in two bf16. g and u are fp32 sums of d
products: off by at most d 2^-24 of their sums of magnitudes, G and U, and H by 1.1 |u| dg +
|silu(g)| du + 1.1 dg du (|silu'| <= 1.1) and 2^-20 |H| of its evaluation. The two parts leave 2^-16 |H|
(half a step of the second), the sum over the experts' d_ff and k at most k d_ff 2^-24 of S =
sum_j w_j sum_f |W2| |H_j|. Then one rounding, 2^-8 |y|. As a whole, the rounding is at most 2^-8 in the
2-norm, and the rest, whose terms are independent and mostly far below their bounds, an eighth of that."""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_17154_gb300 import binding as B
from paper_2607_17154_gb300 import synth
from paper_2607_17154_gb300.layer import LayerStack, MoELayer, build_tables, few_workspace
from tests.helpers import check_layer_integers_full

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = B.NORM_EPS
STEP = 2.0 ** -8  # half a bf16 step

# d, E, k, dff, M, clusters
TINY = (256, 8, 2, 512, 4, 2)
SHAPES = {
    "tiny": TINY,
    "one expert": (256, 1, 1, 128, 1, 1),
    "all experts": (512, 8, 8, 128, 3, 2),
    "odd experts": (768, 40, 3, 640, 5, 8),
    "many": (2048, 64, 6, 1408, 8, 8),
    "many, top-8": (1024, 64, 8, 256, 32, 8),
    "wide": (1024, 16, 4, 4096, 6, 4),
    "five experts": (256, 5, 3, 384, 2, 1),
    "long rows": (8192, 3, 2, 128, 2, 1),
    "longest rows": (32768, 2, 1, 128, 1, 1),
}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    B.lib()
    yield
    code, detail = B.ordermoe_device_error()
    assert code == 0, (code, detail)


class Case:
    def __init__(self, shape, T, seed=0, qbar=0.1, few=True, T_max=None, renorm=1):
        d, E, k, dff, M, K = shape
        self.d, self.E, self.k, self.dff, self.M, self.T = d, E, k, dff, M, T
        self.X = synth.hidden(T, d, seed)
        self.Wr = synth.router_weights(E, d, K, seed + 101)
        self.W1, self.W3, self.W2 = synth.ffn_weights(E, d, dff, seed + 202)
        rng = np.random.default_rng(seed + 1)
        sim = self.Wr.double()
        sim = sim / sim.norm(dim=1, keepdim=True)
        sim = (sim @ sim.T).float().numpy()
        np.fill_diagonal(sim, 1.0)
        group = (np.arange(E) // (E // K)).astype(np.int32)
        x = (rng.random((M, E)) < 0.3 / M).astype(np.uint8)
        x[rng.permutation(E) % M, np.arange(E)] = 1
        sp = synth.server_params(M, d, dff, seed)
        self.o_tab = oracle.tables(sim, group, x, 0.5, qbar, sp.F, sp.B, sp.tau, sp.z, sp.c,
                                   sp.omega_T, sp.omega_Q)
        self.tab = build_tables(sim, group, x, 0.5, qbar, sp, DEV)
        self.home = synth.homes(T, M, seed)
        self.loc0 = np.where(rng.random(T) < 0.4, rng.integers(0, M, T), self.home).astype(np.uint8)
        self.q0 = (rng.random(T) * 0.6 * qbar).astype(np.float32)
        g = lambda t: t.to(DEV)  # noqa: E731
        self.renorm = renorm
        self.layer = MoELayer(g(self.Wr), g(self.W1), g(self.W3), g(self.W2), self.tab, k, T_max or T,
                              renorm=renorm, few=few)

    def experts(self, t, chosen, w):
        """sum_j w_j W2 (silu(W1 x) * (W3 x)) of token t in 64 bits, and how far off its fp32 sum may be."""
        x = self.X[t].double()
        y, slack = torch.zeros(self.d, dtype=torch.float64), torch.zeros(self.d, dtype=torch.float64)
        eps, rest = self.d * 2.0 ** -24, 2.0 ** -16 + 2.0 ** -20 + self.k * self.dff * 2.0 ** -24
        for e, wj in zip(chosen, w):
            g, u = self.W1[e].double() @ x, self.W3[e].double() @ x
            dg, du = eps * (self.W1[e].double().abs() @ x.abs()), eps * (self.W3[e].double().abs() @ x.abs())
            silu = g / (1 + torch.exp(-g))
            dh = 1.1 * u.abs() * dg + silu.abs() * du + 1.1 * dg * du
            y += float(wj) * (self.W2[e].double() @ (silu * u))
            slack += float(wj) * (self.W2[e].double().abs() @ (dh + rest * (silu * u).abs()))
        return y.numpy(), slack.numpy()

    def run(self, state, residual=False, h=None, T=None):
        T = self.T if T is None else T
        m = self.layer
        m.counters.zero_()
        X, home = self.X[:T].to(DEV), torch.as_tensor(self.home[:T]).to(DEV)
        loc = torch.as_tensor(self.loc0[:T]).to(DEV) if state else None
        q = torch.as_tensor(self.q0[:T]).to(DEV) if state else None
        y = torch.full((T, self.d), 7.0, dtype=torch.bfloat16, device=DEV)
        x_out = torch.full_like(y, 7.0)
        if residual:
            m.forward_few_residual(X, h[:T].to(DEV), home, loc, q, y, x_out)
        else:
            m.forward_few(X, home, loc, q, y)
        torch.cuda.synchronize()
        c = lambda a: a[:T].cpu().numpy()  # noqa: E731
        gpu = dict(idx=c(m.topk_idx), w=c(m.topk_w), chosen=c(m.chosen), server=c(m.server), kind=c(m.kind))
        gpu["loc"], gpu["qhat"] = (loc.cpu().numpy(), q.cpu().numpy()) if state else (None, None)
        return y.float().cpu().numpy().astype(np.float64), x_out, gpu, c(m.logits)

    def check_decisions(self, gpu, logits, state):
        T = logits.shape[0]
        loc = self.loc0[:T] if state else self.home[:T]
        q = self.q0[:T] if state else np.zeros(T, np.float32)
        if not state:  # nothing was returned to compare with
            idx, _ = oracle.topk(logits, self.k, self.renorm)
            r = oracle.select(idx, self.o_tab, self.home[:T], loc.copy(), q.copy())
            gpu = dict(gpu, loc=r[3], qhat=r[4])
        _, w, chosen = check_layer_integers_full(logits, gpu, self.o_tab, self.home[:T], loc, q, self.k,
                                                 self.E, renorm=self.renorm)
        np.testing.assert_array_equal(np.bincount(gpu["kind"].reshape(-1), minlength=4),
                                      self.layer.counters.cpu().numpy())
        ref = self.X[:T].double() @ self.Wr.double().T
        mag = self.X[:T].double().abs() @ self.Wr.double().abs().T
        assert (np.abs(logits - ref.numpy()) <= self.d * 2.0 ** -24 * mag.numpy()).all()
        return chosen, w


def assert_y(got, ref, slack, base=None):
    """got against base + ref by the bound above."""
    want = ref if base is None else base + ref
    off = np.abs(got - want)
    bound = STEP * np.abs(want) + (1 + STEP) * slack + 1e-30
    assert (off <= bound).all(), (off / bound).max()
    assert np.linalg.norm(off) <= 1.125 * STEP * np.linalg.norm(np.abs(want))


@pytest.mark.parametrize("T", [1, 2, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("shape", ["tiny", "odd experts", "many"])
def test_layer_few(shape, T):
    c = Case(SHAPES[shape], T, seed=T)
    y, _, gpu, logits = c.run(state=T % 2 == 1)
    chosen, w = c.check_decisions(gpu, logits, T % 2 == 1)
    for t in range(T):
        assert_y(y[t], *c.experts(t, chosen[t], w[t]))


@pytest.mark.parametrize("shape", ["one expert", "all experts", "many, top-8", "wide", "five experts", "long rows",
                                   "longest rows"])
@pytest.mark.parametrize("T", [3, 16])
def test_layer_few_residual(shape, T):
    c = Case(SHAPES[shape], T, seed=3 * T)
    h = synth.hidden(T, c.d, 99)
    y, x_out, gpu, logits = c.run(state=True, residual=True, h=h)
    chosen, w = c.check_decisions(gpu, logits, True)
    for t in range(T):
        assert_y(y[t], *c.experts(t, chosen[t], w[t]), base=h[t].double().numpy())
    # the norm of the bf16 stream it wrote: fp32 sums within 2^-20, one rounding
    ref = y / np.sqrt((y ** 2).mean(1, keepdims=True) + EPS)
    got = x_out.float().cpu().numpy()
    assert (np.abs(got - ref) <= STEP * (1 + 2.0 ** -8) * np.abs(ref) + 1e-30).all()


@pytest.mark.parametrize("T", [2, 12])
def test_gate_weights_as_they_are(T):
    """renorm = 0: the softmax's own weights, whose sum is below 1."""
    c = Case(SHAPES["odd experts"], T, seed=50 + T, renorm=0)
    y, _, gpu, logits = c.run(state=True)
    chosen, w = c.check_decisions(gpu, logits, True)
    assert (w.sum(1) < 0.99).all()
    for t in range(T):
        assert_y(y[t], *c.experts(t, chosen[t], w[t]))


def test_undecided_tokens_with_look_ahead():
    """Horizon 2: a token with a NaN logit and one with a home that is no server, after a call that
    decided them: their rows are left, the others are the ones of the call before."""
    c = Case(TINY, 5, seed=60)
    stride = c.tab.numel()
    tabs = torch.cat([c.tab, c.tab])
    P = torch.full((1, c.E, c.E), 1.0 / c.E, device=DEV)
    m = c.layer
    desc = B.make_layer_desc(5, m.W_r, m.W1, m.W3, m.W2, tabs, c.k, m.ws, lookahead_H=2, tables_stride=stride, P=P)

    def run(X, home):
        y = torch.full((5, c.d), 7.0, dtype=torch.bfloat16, device=DEV)
        B.ordermoe_layer_few(desc, 5, X.to(DEV), torch.as_tensor(home).to(DEV), None, None, y, m.few_ws, m.few_out)
        torch.cuda.synchronize()
        return y
    y = run(c.X, c.home)
    assert B.ordermoe_device_error() == (0, 0) and not (y == 7.0).all(1).any()
    X, home = c.X.clone(), c.home.copy()
    X[1, 0] = float("nan")
    y2 = run(X, home)
    assert B.ordermoe_device_error() == (B.DEV_NAN_LOGIT, 1)
    assert (y2[1] == 7.0).all() and torch.equal(y2[[0, 2, 3, 4]], y[[0, 2, 3, 4]])
    home[3] = 200
    y3 = run(c.X, home)
    assert B.ordermoe_device_error() == (B.DEV_BAD_INDEX, 3)
    assert (y3[3] == 7.0).all() and torch.equal(y3[[0, 1, 2, 4]], y[[0, 1, 2, 4]])


def test_same_bits_again_and_with_fewer_tokens_in_the_buffers():
    c = Case(TINY, 11, seed=5, T_max=16)
    y, _, gpu, logits = c.run(state=True)
    for _ in range(3):
        y2, _, gpu2, logits2 = c.run(state=True)
        assert np.array_equal(y, y2) and np.array_equal(logits, logits2)
        assert all(np.array_equal(gpu[n], gpu2[n]) for n in gpu)
    for T in (16, 1, 7):  # other sizes in the same workspace
        c2 = Case(TINY, T, seed=5)
        c2.layer.few_ws = c.layer.few_ws
        y2, _, gpu2, logits2 = c2.run(state=False)
        chosen, w = c2.check_decisions(gpu2, logits2, False)
        for t in range(T):
            assert_y(y2[t], *c2.experts(t, chosen[t], w[t]))
    assert not c.layer.few_ws[:12].any()  # the counters are back at zero


@pytest.mark.parametrize("T", [3, 8, 16])
def test_weights_of_other_experts_do_not_reach_a_token(T):
    """Infinities and NaN in an expert's weights show in the tokens that use it, and in no other."""
    c = Case(SHAPES["odd experts"], T, seed=T + 20)
    y, _, gpu, logits = c.run(state=False)
    used = np.unique(gpu["chosen"][0])
    bad = int(used[0])
    m = c.layer
    for W, v in ((m.W1, float("nan")), (m.W3, float("inf")), (m.W2, float("-inf"))):
        keep = W[bad].clone()
        W[bad] = v
        y2 = c.run(state=False)[0]
        W[bad] = keep
        users = (gpu["chosen"] == bad).any(1)
        assert users[0] and not np.isfinite(y2[users]).all(1).any()
        assert np.array_equal(y2[~users], y[~users])
    assert np.array_equal(c.run(state=False)[0], y)


def test_a_token_that_is_not_decided_is_left_unwritten():
    c = Case(TINY, 6, seed=8)
    h = synth.hidden(6, c.d, 98)
    y, x, gpu, _ = c.run(state=True, residual=True, h=h)
    keep = c.X.clone()
    c.X[2, 5] = float("nan")
    y2, x2, gpu2, _ = c.run(state=True, residual=True, h=h)
    assert B.ordermoe_device_error() == (B.DEV_NAN_LOGIT, 2)
    rest = [0, 1, 3, 4, 5]
    assert (y2[2] == 7.0).all() and (x2[2] == 7.0).all()
    assert np.array_equal(y2[rest], y[rest]) and torch.equal(x2[rest], x[rest])
    assert (gpu2["idx"][2] == -1).all() and (gpu2["w"][2] == 0).all()
    assert gpu2["loc"][2] == c.loc0[2] and gpu2["qhat"][2] == c.q0[2]
    assert np.array_equal(gpu2["loc"][rest], gpu["loc"][rest])
    c.X = keep
    c.home = c.home.copy()
    c.home[4] = c.M  # no such server
    y3 = c.run(state=True)[0]
    assert B.ordermoe_device_error() == (B.DEV_BAD_INDEX, 4)
    assert (y3[4] == 7.0).all() and np.isfinite(y3).all() and not (y3[[0, 1, 2, 3, 5]] == 7.0).all(1).any()
    c.X = torch.full_like(keep, float("nan"))  # none is decided
    assert (c.run(state=True)[0] == 7.0).all()
    assert B.ordermoe_device_error()[0] == B.DEV_NAN_LOGIT
    c.X, c.home[4] = keep, 0
    assert (c.run(state=True)[0] != 7.0).any()


def test_tables_of_another_layer_are_reported():
    c = Case(TINY, 2, seed=8)
    d = Case((256, 7, 2, 512, 4, 1), 2, seed=8)
    m = c.layer
    desc = B.make_layer_desc(2, m.W_r, m.W1, m.W3, m.W2, torch.cat([d.tab, d.tab, c.tab]), 2, m.ws)
    y = torch.full((2, c.d), 7.0, dtype=torch.bfloat16, device=DEV)
    B.ordermoe_layer_few(desc, 2, c.X.to(DEV), torch.zeros(2, dtype=torch.uint8, device=DEV), None, None, y,
                         m.few_ws)
    torch.cuda.synchronize()
    assert B.ordermoe_device_error()[0] == B.DEV_BAD_INDEX
    assert (y == 7.0).all()


def test_no_tokens_and_no_outputs():
    c = Case(TINY, 4, seed=9)
    y, _, _, _ = c.run(state=False)
    X, home = c.X.to(DEV), torch.as_tensor(c.home).to(DEV)
    out = torch.zeros(4, c.d, dtype=torch.bfloat16, device=DEV)
    B.ordermoe_layer_few(c.layer.few_desc, 0, X, home, None, None, out, c.layer.few_ws)
    torch.cuda.synchronize()
    assert not out.any()
    B.ordermoe_layer_few(c.layer.few_desc, 4, X, home, None, None, out, c.layer.few_ws)  # no `out`
    torch.cuda.synchronize()
    assert np.array_equal(out.float().cpu().numpy(), y)


def test_another_stream_and_two_graphs_on_one_workspace():
    a, b = Case(TINY, 4, seed=30), Case(TINY, 9, seed=31)
    ya, yb = a.run(state=False)[0], b.run(state=False)[0]
    ws = few_workspace(16, a.E, a.d, a.dff, a.k, DEV)
    outs, graphs = [], []
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for c in (a, b):
        X, home = c.X.to(DEV), torch.as_tensor(c.home).to(DEV)
        y = torch.zeros(c.T, c.d, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            B.ordermoe_layer_few(c.layer.few_desc, c.T, X, home, None, None, y, ws)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            B.ordermoe_layer_few(c.layer.few_desc, c.T, X, home, None, None, y, ws)
        outs.append((y, X, home))
        graphs.append(g)
    for i in (0, 1, 1, 0, 1):
        outs[i][0].zero_()
        graphs[i].replay()
    torch.cuda.synchronize()
    assert np.array_equal(outs[0][0].float().cpu().numpy(), ya)
    assert np.array_equal(outs[1][0].float().cpu().numpy(), yb)


def test_two_calls_at_once():
    """Calls in two streams, a workspace each: neither waits for the other's CTAs for ever."""
    a, b = Case(SHAPES["many"], 7, seed=40), Case(SHAPES["many"], 16, seed=41)
    ya, yb = a.run(state=False)[0], b.run(state=False)[0]
    args = []
    for c in (a, b):
        args.append((c, torch.cuda.Stream(), c.X.to(DEV), torch.as_tensor(c.home).to(DEV),
                     torch.zeros(c.T, c.d, dtype=torch.bfloat16, device=DEV)))
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, X, home, y in args:
            B.ordermoe_layer_few(c.layer.few_desc, c.T, X, home, None, None, y, c.layer.few_ws, stream=s)
    torch.cuda.synchronize()
    assert np.array_equal(args[0][4].float().cpu().numpy(), ya)
    assert np.array_equal(args[1][4].float().cpu().numpy(), yb)


def test_first_call_on_another_stream():
    """Layers made behind work that is still under way, on memory that it leaves full of ones, whose
    first call is on a stream that nobody ordered behind it."""
    a = Case(TINY, 6, seed=45)
    ya = a.run(state=False)[0]
    X, home = a.X.to(DEV), torch.as_tensor(a.home).to(DEV)
    y = torch.zeros(6, a.d, dtype=torch.bfloat16, device=DEV)
    m, s = a.layer, torch.cuda.Stream()
    big = torch.ones(1 << 28, device=DEV)
    torch.cuda.synchronize()
    for _ in range(3):
        dirty = torch.empty(m.few_ws.numel(), dtype=torch.uint8, device=DEV)
        for _ in range(20):
            big.mul_(1.0)
        dirty.fill_(1)
        del dirty
        b = MoELayer(m.W_r, m.W1, m.W3, m.W2, m.tables, m.k, 6, few=True)
        b.forward_few(X, home, None, None, y, stream=s)
        s.synchronize()
        assert np.array_equal(y.float().cpu().numpy(), ya)
        assert not b.few_ws[:12].any()
        y.zero_()
        torch.cuda.synchronize()


@pytest.mark.parametrize("H", [1, 3])
@pytest.mark.parametrize("T", [1, 13, 17])
def test_stack_of_few_tokens(H, T):
    """A stack with few=True against the same stack by the larger layers' launches: the decisions
    of every layer (near ties apart: none here) and the residual stream within the
    roundings of the other (an expert output's, H's and the stream's, 2^-8 each, a layer)."""
    L, E, k, M, d, dff = 3, 8, 2, 4, 512, 256
    layers, sims = [], []
    for l in range(L):
        W1, W3, W2 = synth.ffn_weights(E, d, dff, 1000 * l, device=DEV)
        Wr = synth.router_weights(E, d, 2, 7 + 1000 * l, device=DEV)
        layers.append({"W_r": Wr, "W1": W1, "W3": W3, "W2": W2})
        S = torch.nn.functional.normalize(Wr.double(), dim=1)
        S = (S @ S.T).float().cpu().numpy()
        np.fill_diagonal(S, 1.0)
        sims.append(S)
    rng = np.random.default_rng(3)
    place = np.zeros((M, E), np.uint8)
    place[np.arange(E) % M, np.arange(E)] = 1
    stride = B.ordermoe_tables_bytes(E, M)
    tabs = torch.zeros(L * stride, dtype=torch.uint8, device=DEV)
    sp = synth.server_params(M, d, dff, 0)
    for l in range(L):
        build_tables(sims[l], (np.arange(E) // 4).astype(np.int32), place, 0.5, 0.3, sp, DEV,
                     out=tabs[l * stride:(l + 1) * stride])
    P = rng.random((L - 1, E, E)).astype(np.float32)
    P = torch.as_tensor(P / P.sum(-1, keepdims=True)).to(DEV)
    home = torch.as_tensor(synth.homes(T, M, 1)).to(DEV)
    got = []
    for few in (False, True):
        st = LayerStack(layers, tabs, k, T, DEV, H=H, stride=stride, P=P, few=few)
        hs = [synth.hidden(T, d, 4, DEV)] + [torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in range(L)]
        xs = [torch.zeros(T, d, dtype=torch.bfloat16, device=DEV) for _ in range(L + 1)]
        loc, q = home.clone(), torch.zeros(T, device=DEV)
        logits = torch.zeros(L, T, E, device=DEV)
        st.step_residual(hs, xs, home, loc, q, logits=logits)
        g = st.capture_residual(hs, xs, home, loc, q, prologue=lambda: (loc.copy_(home), q.zero_()))
        eager = [h.clone() for h in hs]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(eager, hs))
        got.append((hs, loc.cpu(), q.cpu(), logits))
    assert torch.equal(got[0][1], got[1][1]) and torch.equal(got[0][2], got[1][2])
    for l in range(L + 1):
        u, v = got[0][0][l].double(), got[1][0][l].double()
        assert (u - v).norm() <= 4 * STEP * max(l, 1) * u.norm()
    if T > B.FEW_TOKENS:  # more tokens than it takes: the same launches
        assert all(torch.equal(u, v) for u, v in zip(got[0][0], got[1][0]))
