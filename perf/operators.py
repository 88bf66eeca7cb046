"""Performance cases of two operators of a decoder's feed-forward half when it serves few tokens, and
of its dense products.

  few     a whole MoE layer for at most 16 tokens: router, softmax, top-k, server-expert selection
          (Alg. 2, H = 1), the chosen experts' SwiGLU and the weighted combine, alone or on the
          residual map (h + y and its RMSNorm)
  linear  Y = act(X W^T + bias) + residual: the dense products around the experts (attention
          projections, dense feed-forward layers, output heads)

`run` computes them in elementary torch operations, or with `own` by the framework's calls.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
EPS = 1e-6

# layer shapes of synth.WORKLOADS (d, experts, routed, d_ff, servers, clusters, budget, homes)
TINY = dict(d=256, E=8, k=2, dff=512, M=4, K=2, qbar=0.05, home="uniform")
WIDE = dict(d=4096, E=8, k=2, dff=14336, M=4, K=4, qbar=0.5, home="uniform")
FINE = dict(d=2048, E=64, k=6, dff=1408, M=8, K=8, qbar=0.5, home="zipf1.1")
# between them: a number of experts that is no power of two, and a middle one
ODD = dict(d=1024, E=40, k=3, dff=640, M=5, K=8, qbar=0.1, home="zipf1.1")
MID = dict(d=1024, E=16, k=4, dff=4096, M=6, K=4, qbar=0.1, home="uniform")


def listed():
    return [
        # the smallest layer: one launch's latency
        dict(name="few_tiny", kind="few", T=4, residual=False, state=False, **TINY),
        # one sequence decoding on 64 narrow experts, a layer of a stack
        dict(name="few_fine_1", kind="few", T=1, residual=True, state=True, **FINE),
        # a few sequences (a ragged batch) on 64 narrow experts
        dict(name="few_fine_7", kind="few", T=7, residual=True, state=False, **FINE),
        # one sequence on 8 wide experts
        dict(name="few_wide_1", kind="few", T=1, residual=True, state=True, **WIDE),
        # the largest few-token batch: all wide experts' weights are read
        dict(name="few_wide_16", kind="few", T=16, residual=False, state=False, **WIDE),
        # one token's output projection, added to the residual stream
        dict(name="linear_1", kind="linear", M=1, N=4096, K=4096, act="none", bias=False, res=True,
             f32=False, pad=0),
        # a decode batch through the first product of a dense feed-forward layer
        dict(name="linear_33", kind="linear", M=33, N=5632, K=2048, act="gelu", bias=True, res=False,
             f32=False, pad=0),
        # a decode batch's logits over a ragged vocabulary, kept in 32 bits
        dict(name="linear_head", kind="linear", M=128, N=32003, K=2048, act="none", bias=False,
             res=False, f32=True, pad=0),
        # odd sizes, rows inside wider buffers
        dict(name="linear_odd", kind="linear", M=301, N=1009, K=1999, act="silu", bias=True, res=True,
             f32=False, pad=24),
        # a chunk of a prompt through the second product of a dense feed-forward layer
        dict(name="linear_1021", kind="linear", M=1021, N=4096, K=14336, act="none", bias=True,
             res=True, f32=False, pad=0),
        # a full prefill batch through the first product
        dict(name="linear_4096", kind="linear", M=4096, N=14336, K=4096, act="relu", bias=True,
             res=False, f32=False, pad=0),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    if rng.random() < 0.5:
        shape = dict(rng.choice([TINY, WIDE, FINE, FINE, ODD, MID]))
        return dict(kind="few", T=rng.randint(1, 16), residual=rng.random() < 0.5,
                    state=rng.random() < 0.5, **shape)
    M, N, K = _log_int(rng, 1, 4096), _log_int(rng, 64, 16384), _log_int(rng, 64, 14336)
    while M * N * K > 4096 * 14336 * 4096:
        M, N, K = M // 2, N // 2, K // 2
    return dict(kind="linear", M=M, N=N, K=K, act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]),
                bias=rng.random() < 0.5, res=rng.random() < 0.5, f32=rng.random() < 0.25,
                pad=rng.choice([0, 0, 8, 40]))


# ----------------------------------------------------------------- inputs
def _normal(g, std, *shape, dt=torch.bfloat16):
    x = torch.empty(shape, dtype=dt, device=DEV)
    return x.normal_(0.0, std, generator=g)


def _few_inputs(c, seed):
    """A layer's weights, its selection data (similarities, groups, a placement with a copy of
    every expert and some replicas, server parameters) and the tokens."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    rng = np.random.default_rng(seed + 77)
    T, d, E, M, K, dff = c["T"], c["d"], c["E"], c["M"], c["K"], c["dff"]
    s = {"case": c}
    cluster = np.arange(E) // (E // K)
    cent = _normal(g, 0.02, K, d, dt=torch.float32)
    s["W_r"] = (cent[torch.as_tensor(cluster).to(DEV)]
                + _normal(g, 0.005, E, d, dt=torch.float32)).to(torch.bfloat16)
    s["W1"], s["W3"] = _normal(g, 0.02, E, dff, d), _normal(g, 0.02, E, dff, d)
    s["W2"] = _normal(g, 0.02, E, d, dff)
    s["X"] = _normal(g, 1.0, T, d)
    if c["residual"]:  # the layer reads the normalised residual stream
        s["h"] = s["X"]
        s["X"] = _rms(s["h"].float()).to(torch.bfloat16)
    W = s["W_r"].double()
    W = W / W.norm(dim=1, keepdim=True)
    sim = (W @ W.T).float()
    s["sim"] = sim.fill_diagonal_(1.0)
    s["group"] = torch.as_tensor(cluster.astype(np.int32)).to(DEV)
    x = (rng.random((M, E)) < 0.33 / M).astype(np.uint8)
    x[rng.permutation(E) % M, np.arange(E)] = 1
    s["place"] = torch.as_tensor(x).to(DEV)
    F = rng.uniform(20e12, 110e12, size=M)
    B, tau = rng.uniform(1.0, 10.0, size=(M, M)) / 8 * 1e9, rng.uniform(0.2e-3, 20e-3, size=(M, M))
    np.fill_diagonal(B, 1.0)
    np.fill_diagonal(tau, 0.0)
    s["F"], s["B"], s["tau"] = (torch.as_tensor(v).to(DEV) for v in (F, B, tau))
    p = (np.arange(M) + 1.0) ** (-1.1 if c["home"] == "zipf1.1" else 0.0)
    home = rng.choice(M, size=T, p=p / p.sum())
    s["home"] = torch.as_tensor(home.astype(np.uint8)).to(DEV)
    if c["state"]:  # tokens in the middle of a stack: some moved, part of their budget spent
        loc = np.where(rng.random(T) < 0.4, rng.integers(0, M, T), home).astype(np.uint8)
        s["loc0"] = torch.as_tensor(loc).to(DEV)
        s["q0"] = torch.as_tensor((rng.random(T) * 0.6 * c["qbar"]).astype(np.float32)).to(DEV)
    return s


def _plan(s):
    """The selection's tables (Eqs. 7, 18, 37, 38) as tensors: a layer keeps them."""
    c = s["case"]
    E = c["E"]
    q = 0.5 * (1.0 - s["sim"].clamp(max=1.0))
    s["Q"] = q.fill_diagonal_(0.0)
    s["qbar"] = float(np.float32(c["qbar"]))
    s["on"] = s["place"].bool().T[None]
    s["Cq"] = (0.5 * q.double() / float(np.float32(c["qbar"]))).float()
    s["sub"] = (s["group"][:, None] == s["group"][None]) & (s["sim"] >= 0.5) & ~torch.eye(
        E, dtype=torch.bool, device=DEV)
    comp = 6.0 * c["d"] * c["dff"] / s["F"]
    link = (2.0 * c["d"] / s["B"] + s["tau"]).fill_diagonal_(0.0)
    s["A"] = (0.5 * (link + comp[None])[None] / comp[:, None, None]).float()  # [home][from][to]


def prepare(case, seed):
    if case["kind"] == "linear":
        return _linear_inputs(case, seed)
    s = _few_inputs(case, seed)
    c = case
    T, d = c["T"], c["d"]
    _plan(s)
    if c["state"]:
        s["loc"], s["qhat"] = s["loc0"].clone(), s["q0"].clone()
    s["y"] = torch.empty(T, d, dtype=torch.bfloat16, device=DEV)
    s["x_out"] = torch.empty_like(s["y"])
    if own:  # the layer object that a user's program keeps
        from paper_2607_17154_gb300 import binding as B
        from paper_2607_17154_gb300.layer import MoELayer
        t = torch.zeros(B.ordermoe_tables_bytes(c["E"], c["M"]), dtype=torch.uint8, device=DEV)
        B.ordermoe_build_tables(s["sim"], s["group"], s["place"], 0.5, c["qbar"], s["F"], s["B"],
                                s["tau"], 2.0 * d, 6.0 * d * c["dff"], 0.5, 0.5, t)
        s["layer"] = MoELayer(s["W_r"], s["W1"], s["W3"], s["W2"], t, c["k"], T, few=True)
    return s


def _linear_inputs(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    M, N, K, pad = c["M"], c["N"], c["K"], c["pad"]

    def rows(n, w, std, odd):
        # rows of w values, 16-byte aligned unless `odd`, inside wider ones where pad > 0
        ld = (w if odd else (w + 7) // 8 * 8) + pad
        return _normal(g, std, n, ld)[:, :w]

    s = {"case": c, "X": rows(M, K, 1.0, False), "W": rows(N, K, 0.02, False)}
    s["bias"] = _normal(g, 0.5, N) if c["bias"] else None
    s["res"] = rows(M, N, 1.0, True) if c["res"] else None
    s["Y"] = torch.empty(M, N + pad, dtype=torch.float32 if c["f32"] else torch.bfloat16,
                         device=DEV)[:, :N]
    return s


# ------------------------------------------------------------------- runs
def _rms(v):
    return v * torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)


def _select(s, idx, a, loc, q):
    """Alg. 2 per slot in rank order: the cheapest (expert, server) of the target and the
    substitutes that the budget allows; ties: exact, the current server, lower server, expert."""
    c = s["case"]
    T, k, E, M = idx.shape[0], c["k"], c["E"], c["M"]
    rows, ar = torch.arange(T, device=DEV), torch.arange
    taken = torch.zeros(T, E, dtype=torch.bool, device=DEV).scatter_(1, idx, True)
    here, picks = loc, []
    for j in range(k):
        r = idx[:, j]
        qn = q[:, None] + s["Q"][r]
        ok = (s["sub"][r] & ~taken & (qn <= s["qbar"])).scatter_(1, r[:, None], True)
        cost = s["A"][a, loc][:, None, :] + s["Cq"][r][:, :, None]  # [T][E][M]
        cost = torch.where(ok[:, :, None] & s["on"], cost, math.inf)
        key = cost.view(torch.int32).long() << 32
        key |= (ar(E, device=DEV)[None] != r[:, None]).long()[:, :, None] << 31
        key |= (ar(M, device=DEV)[None] != loc[:, None]).long()[:, None, :] << 30
        key |= ar(M, device=DEV)[None, None, :] << 8
        key |= ar(E, device=DEV)[None, :, None]
        best = key.reshape(T, -1).amin(1)
        e, m = best & 0xFF, (best >> 8) & 0xFF
        picks.append((e, m, 2 * (m != loc).long() + (e != r).long()))
        q = qn[rows, e]
        taken[rows, e] = True
        here = m if j == 0 else here
    chosen, server, kind = (torch.stack(v, 1) for v in zip(*picks))
    return chosen, server, kind, here, q


def _experts(s, x, chosen, w):
    """sum_j w_j W2_e (silu(W1_e x) * (W3_e x)) over a token's experts, in 32 bits."""
    c = s["case"]
    T, k, E = x.shape[0], c["k"], c["E"]
    if T * k < E:  # the entries' own experts
        e = chosen.flatten()
        v = x.repeat_interleave(k, 0)[:, :, None]
        h = torch.bmm(s["W1"][e].float(), v)
        h = h * torch.sigmoid(h) * torch.bmm(s["W3"][e].float(), v)
        y = torch.bmm(s["W2"][e].float(), h)[:, :, 0]
        return (y.view(T, k, -1) * w[:, :, None]).sum(1)
    gate = torch.zeros(T, E, device=DEV).scatter_(1, chosen, w)
    v = x.T[None].expand(E, -1, -1)
    h = torch.bmm(s["W1"].float(), v)
    h = h * torch.sigmoid(h) * torch.bmm(s["W3"].float(), v)
    y = torch.bmm(s["W2"].float(), h)  # [E][d][T]
    return (y * gate.T[:, None, :]).sum(0).T


def _act(v, act):
    if act == "relu":
        return v.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * v * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (v + 0.044715 * v * v * v)))
    return v * torch.sigmoid(v) if act == "silu" else v


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    if c["kind"] == "linear":
        v = s["X"].float() @ s["W"].float().T
        v = _act(v if s["bias"] is None else v + s["bias"].float(), c["act"])
        v = v if s["res"] is None else v + s["res"].float()
        s["Y"].copy_(v)
        return s["Y"]
    x = s["X"].float()
    logits = s["X"].double() @ s["W_r"].double().T  # 64 bits: the ranks are decided on them
    order = torch.sort(logits, dim=1, descending=True, stable=True).indices
    idx = order[:, :c["k"]]
    p = torch.exp(logits - logits.amax(1, keepdim=True))
    w = p.gather(1, idx)
    w = (w / w.sum(1, keepdim=True)).float()
    home = s["home"].long()
    if c["state"]:
        chosen, server, kind, loc, q = _select(s, idx, home, s["loc0"].long(), s["q0"])
    else:
        chosen, server, kind, loc, q = _select(s, idx, home, home, torch.zeros(c["T"], device=DEV))
    y = _experts(s, x, chosen, w)
    out = {"logits": logits.float(), "topk": idx.int(), "topk_w": w, "chosen": chosen.int(),
           "server": server.to(torch.uint8), "kind": kind.to(torch.uint8)}
    if c["state"]:
        out.update(loc=loc.to(torch.uint8), qhat=q)
    if not c["residual"]:
        return dict(out, y=y.to(torch.bfloat16))
    h = (s["h"].float() + y).to(torch.bfloat16)
    return dict(out, h=h, x=_rms(h.float()).to(torch.bfloat16))


def _run_own(s, c):
    if c["kind"] == "linear":
        from paper_2607_17154_gb300 import binding as B
        B.ordermoe_linear(s["X"], s["W"], s["Y"], bias=s["bias"], act=c["act"], residual=s["res"])
        return s["Y"]
    m, loc, q = s["layer"], None, None
    if c["state"]:
        loc, q = s["loc"], s["qhat"]
        loc.copy_(s["loc0"])
        q.copy_(s["q0"])
    if c["residual"]:
        m.forward_few_residual(s["X"], s["h"], s["home"], loc, q, s["y"], s["x_out"])
        out = {"h": s["y"], "x": s["x_out"]}
    else:
        m.forward_few(s["X"], s["home"], loc, q, s["y"])
        out = {"y": s["y"]}
    if c["state"]:
        out.update(loc=loc, qhat=q)
    return dict(out, logits=m.logits, topk=m.topk_idx, topk_w=m.topk_w, chosen=m.chosen,
                server=m.server, kind=m.kind)


def work(case):
    """Each input read and each output written once; an expert's weights only when a token is
    expected to reach it (each token takes k distinct experts of E)."""
    c = case
    if c["kind"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        nbytes = 2.0 * (M * K + N * K) + (4.0 if c["f32"] else 2.0) * M * N
        nbytes += (2.0 * N if c["bias"] else 0.0) + (2.0 * M * N if c["res"] else 0.0)
        return {"bytes": nbytes, "flops": 2.0 * M * N * K}
    T, d, E, k = c["T"], c["d"], c["E"], c["k"]
    hit = E * (1.0 - (1.0 - k / E) ** T)
    return {"bytes": 6.0 * hit * d * c["dff"] + 2.0 * E * d + 2.0 * T * d * (4 if c["residual"] else 2)
            + T * (14.0 * k + 4 * E + 16) + 8.0 * E * E,
            "flops": 6.0 * T * k * d * c["dff"] + 2.0 * T * d * E}


# ------------------------------------------------------- the same in 64 bits
def _exact_select(c, t, sim, group, place, F, B, tau, target, home, loc, q):
    """Alg. 2 of one token on numpy values; costs and losses in the interface's 32 bits."""
    f4 = np.float32
    d_ref = 6.0 * c["d"] * c["dff"] / F[home]
    taken, first, picks = set(target), None, []
    for r in target:
        best = None
        for e in [r] + [e for e in range(c["E"]) if e != r and group[e] == group[r]
                        and sim[r, e] >= 0.5 and e not in taken]:
            loss = f4(0.0) if e == r else f4(0.5) * (f4(1.0) - min(f4(1.0), sim[r, e]))
            if e != r and f4(q + loss) > f4(c["qbar"]):
                continue
            quality = f4(0.5 * float(loss) / float(f4(c["qbar"])))
            for m in np.flatnonzero(place[:, e]):
                delay = 6.0 * c["d"] * c["dff"] / F[m]
                if m != loc:
                    delay += 2.0 * c["d"] / B[loc, m] + tau[loc, m]
                rank = (f4(f4(0.5 * delay / d_ref) + quality), e != r, m != loc, m, e, loss)
                best = rank if best is None or rank[:5] < best[:5] else best
        _, sub, away, m, e, loss = best
        taken.add(e)
        q = f4(q + loss) if sub else q
        first = m if first is None else first
        picks.append(e)
    return picks, first, q


def exact(case, seed):
    c = case
    if c["kind"] == "linear":
        s = _linear_inputs(c, seed)
        v = s["X"].double() @ s["W"].double().T
        if c["bias"]:
            v += s["bias"].double()
        if c["act"] == "relu":
            v = torch.relu(v)
        elif c["act"] == "silu":
            v = torch.nn.functional.silu(v)
        elif c["act"] != "none":
            v = torch.nn.functional.gelu(v, approximate="tanh" if c["act"] == "gelu_tanh" else "none")
        return v + s["res"].double() if c["res"] else v
    s = _few_inputs(c, seed)
    x = s["X"].double()
    logits = torch.nn.functional.linear(x, s["W_r"].double())
    w, idx = torch.topk(torch.softmax(logits, 1), c["k"], dim=1)
    w = w / w.sum(1, keepdim=True)
    host = {n: s[n].cpu().numpy() for n in ("sim", "group", "place", "F", "B", "tau", "home")}
    home, target = host.pop("home").astype(int), idx.tolist()
    loc = s["loc0"].cpu().numpy().astype(int) if c["state"] else home
    q = s["q0"].cpu().numpy() if c["state"] else np.zeros(c["T"], np.float32)
    y, qhat = torch.zeros_like(x), np.zeros(c["T"])
    for t in range(c["T"]):
        picks, _, qhat[t] = _exact_select(c, t, target=target[t], home=home[t], loc=loc[t], q=q[t], **host)
        for j, e in enumerate(picks):
            h = torch.nn.functional.silu(s["W1"][e].double() @ x[t]) * (s["W3"][e].double() @ x[t])
            y[t] += w[t, j] * (s["W2"][e].double() @ h)
    out = {"logits": logits, "topk": None, "topk_w": w, "chosen": None, "server": None, "kind": None}
    if c["state"]:
        out.update(loc=None, qhat=qhat)
    if not c["residual"]:
        return dict(out, y=y)
    h = s["h"].double() + y
    hb = h.to(torch.bfloat16).double()  # the residual stream is a bf16 tensor of the interface
    return dict(out, h=h, x=hb / torch.sqrt(hb.square().mean(1, keepdim=True) + EPS))
