"""One OrderMoE MoE layer on the GPU: device buffers from torch, every step
through the C ABI (route_select -> dispatch -> expert_ffn -> combine)."""
import torch

from . import binding as B


class MoELayer:
    """Holds a layer's weights, tables and scratch for up to T_max tokens. Its calls share the scratch:
    they may not overlap on the GPU (one stream, or one ordered behind the other)."""

    def __init__(self, W_r, W1, W3, W2, tables, k, T_max, renorm=1, device=None, few=False):
        """few: also keep the workspace of forward_few (calls of up to B.FEW_TOKENS tokens)."""
        self.device = device or W1.device
        self.W_r, self.W1, self.W3, self.W2 = W_r, W1, W3, W2
        self.E, self.dff, self.d = W1.shape
        self.k, self.renorm, self.tables = k, renorm, tables
        self.T_max = T_max
        R = T_max * k
        dev = self.device
        self.logits = torch.empty(T_max, self.E, dtype=torch.float32, device=dev)
        self.topk_idx = torch.empty(T_max, k, dtype=torch.int32, device=dev)
        self.topk_w = torch.empty(T_max, k, dtype=torch.float32, device=dev)
        self.chosen = torch.empty(T_max, k, dtype=torch.int32, device=dev)
        self.server = torch.empty(T_max, k, dtype=torch.uint8, device=dev)
        self.kind = torch.empty(T_max, k, dtype=torch.uint8, device=dev)
        self.counters = torch.zeros(4, dtype=torch.int32, device=dev)
        self.offsets = torch.empty(self.E + 1, dtype=torch.int32, device=dev)
        self.row_token = torch.empty(R, dtype=torch.int32, device=dev)
        self.row_of = torch.empty(T_max, k, dtype=torch.int32, device=dev)
        self.X_perm = torch.empty(R, self.d, dtype=torch.bfloat16, device=dev)
        self.H = torch.empty(R, self.dff, dtype=torch.bfloat16, device=dev)
        self.Y_perm = torch.empty(R, self.d, dtype=torch.bfloat16, device=dev)
        ws = B.ordermoe_dispatch_workspace_bytes(T_max, k, self.E)
        self.ws = torch.empty(ws, dtype=torch.uint8, device=dev)
        self.few_ws = None
        if few:
            self.few_ws = few_workspace(min(T_max, B.FEW_TOKENS), self.E, self.d, self.dff, k, dev)

    # What forward_few's descriptors point to: forward() reads these at every call, so a new plan's
    # tables, new weights or another buffer put in their place have to reach forward_few too.
    _DESCRIBED = frozenset(("W_r", "W1", "W3", "W2", "tables", "k", "renorm", "logits", "topk_idx",
                            "topk_w", "chosen", "server", "kind", "counters"))
    _few = None

    def __setattr__(self, name, value):
        object.__setattr__(self, name, value)
        if name in self._DESCRIBED:
            object.__setattr__(self, "_few", None)

    def _described(self):
        if self._few is None:
            self._few = (B.make_layer_desc(self.T_max, self.W_r, self.W1, self.W3, self.W2,
                                           self.tables, self.k, self.ws, self.renorm),
                         B.make_few_out(self.logits, self.topk_idx, self.topk_w, self.chosen,
                                        self.server, self.kind, self.counters))
        return self._few

    @property
    def few_desc(self):
        return self._described()[0]

    @property
    def few_out(self):
        return self._described()[1]

    def forward(self, X, home, loc, qhat, y, T=None, logits_in=None, stream=None):
        """y[:T] = MoE(X[:T]); loc/qhat are updated in place (Eq. 44)."""
        T = X.shape[0] if T is None else T
        assert T <= self.T_max
        R = T * self.k
        B.ordermoe_route_select(X, self.W_r, logits_in, T, self.E, self.d, self.k, self.renorm,
                                self.tables, home, loc, qhat, self.logits, self.topk_idx,
                                self.topk_w, self.chosen, self.server, self.kind, self.counters,
                                stream)
        B.ordermoe_dispatch(self.chosen, X, T, self.k, self.E, self.d, self.offsets,
                            self.row_token, self.row_of, self.X_perm, self.ws, stream)
        B.ordermoe_expert_ffn(self.X_perm, self.offsets, R, self.W1, self.W3, self.W2, self.E,
                              self.d, self.dff, self.H, self.Y_perm, stream)
        B.ordermoe_combine(self.Y_perm, self.row_of, self.topk_w, T, self.k, self.d, y, stream)
        return y

    def forward_residual(self, x, h, home, loc, qhat, h_out, x_out, T=None, eps=B.NORM_EPS,
                         stream=None):
        """One layer of a stack on the residual map: the layer runs on x
        (= RMSNorm(h)), then h_out = h + y and x_out = RMSNorm(h_out), the next
        layer's inputs. Router logits, decisions and the permutation stay in
        this object's buffers."""
        T = x.shape[0] if T is None else T
        assert T <= self.T_max
        R = T * self.k
        B.ordermoe_route_select(x, self.W_r, None, T, self.E, self.d, self.k, self.renorm,
                                self.tables, home, loc, qhat, self.logits, self.topk_idx,
                                self.topk_w, self.chosen, self.server, self.kind, self.counters,
                                stream)
        B.ordermoe_dispatch(self.chosen, x, T, self.k, self.E, self.d, self.offsets,
                            self.row_token, self.row_of, self.X_perm, self.ws, stream)
        B.ordermoe_expert_ffn(self.X_perm, self.offsets, R, self.W1, self.W3, self.W2, self.E,
                              self.d, self.dff, self.H, self.Y_perm, stream)
        B.ordermoe_combine_residual_norm(self.Y_perm, self.row_of, self.topk_w, h, T, self.k,
                                         self.d, eps, h_out, x_out, stream)
        return h_out, x_out


    def forward_few(self, X, home, loc, qhat, y, T=None, stream=None):
        """forward() of at most B.FEW_TOKENS tokens in one launch: the decisions in the same
        buffers, y rounded once (neither H nor the experts' outputs are bf16 on the way)."""
        T = X.shape[0] if T is None else T
        assert T <= self.T_max and self.few_ws is not None
        B.ordermoe_layer_few(self.few_desc, T, X, home, loc, qhat, y, self.few_ws, self.few_out,
                             stream)
        return y

    def forward_few_residual(self, x, h, home, loc, qhat, h_out, x_out, T=None, eps=B.NORM_EPS,
                             stream=None):
        """forward_residual() of at most B.FEW_TOKENS tokens in one launch."""
        T = x.shape[0] if T is None else T
        assert T <= self.T_max and self.few_ws is not None
        B.ordermoe_layer_few_residual(self.few_desc, T, x, h, home, loc, qhat, eps, h_out, x_out,
                                      self.few_ws, self.few_out, stream)
        return h_out, x_out


def few_workspace(T, E, d, dff, k, device):
    """The workspace of ordermoe_layer_few calls of up to T tokens, prepared."""
    ws = torch.empty(B.ordermoe_layer_few_workspace_bytes(T, E, d, dff, k), dtype=torch.uint8,
                     device=device)
    with torch.cuda.device(device):
        B.ordermoe_layer_few_init(ws)
    _settle(device)
    return ws


def _settle(device):
    """Waits for the current stream: buffers that were made and cleared there may then be used on any
    other. (While it is being captured nothing runs, and only the graph may use them.)"""
    if torch.device(device).type != "cuda":
        return
    with torch.cuda.device(device):
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.current_stream().synchronize()


def build_tables(sim, group, placement, theta, qbar, sp, device, out=None):
    """Device tables for one layer from host arrays (sim, group, placement) and
    server parameters sp (synth.ServerParams); written into `out` (a uint8
    device tensor, e.g. one slice of a stack of layers' tables) when given."""
    E = sim.shape[0]; M = placement.shape[0]
    t = out if out is not None else torch.zeros(B.ordermoe_tables_bytes(E, M), dtype=torch.uint8,
                                                device=device)
    f = lambda a, dt: torch.as_tensor(a).to(device=device, dtype=dt).contiguous()
    B.ordermoe_build_tables(f(sim, torch.float32), f(group, torch.int32), f(placement, torch.uint8),
                            theta, qbar, f(sp.F, torch.float64), f(sp.B, torch.float64),
                            f(sp.tau, torch.float64), sp.z, sp.c, sp.omega_T, sp.omega_Q, t)
    return t


def _rows16(W):
    """The matrix W as ordermoe_linear takes it, rows at multiples of 16 bytes: itself, or a copy."""
    n, w = W.shape
    if W.data_ptr() % 16 == 0 and (w <= 1 or W.stride(1) == 1) and (n <= 1 or W.stride(0) % 8 == 0):
        return W
    return torch.empty(n, (w + 7) // 8 * 8, dtype=W.dtype, device=W.device)[:, :w].copy_(W)


class DenseFFN:
    """A dense feed-forward layer (every second layer of Switch-Base-8E is one, with ReLU):
    y = act(x W1^T + b1) W2^T + b2 through ordermoe_linear, for up to T_max tokens.
    W1 [dff, d], W2 [d, dff], b1 [dff], b2 [d] bf16 (the biases may be None). Weights whose rows do not
    start at multiples of 16 bytes (a d_ff that is no multiple of 8) are copied once to rows that do; x
    of more than one row needs such rows itself. Calls share H: they may not overlap on the GPU."""

    def __init__(self, W1, W2, T_max, b1=None, b2=None, act="relu"):
        self.W1, self.W2, self.b1, self.b2, self.act = _rows16(W1), _rows16(W2), b1, b2, act
        self.dff, self.d = W1.shape
        self.T_max = T_max
        self.H = torch.empty(T_max, (self.dff + 7) // 8 * 8, dtype=torch.bfloat16,
                             device=W1.device)[:, :self.dff]
        _settle(W1.device)

    def forward(self, x, y, residual=None, stream=None):
        """y = the layer of x [T, d], added to residual [T, d] when given (y may be it)."""
        T = x.shape[0]
        assert T <= self.T_max
        B.ordermoe_linear(x, self.W1, self.H[:T], bias=self.b1, act=self.act, stream=stream)
        B.ordermoe_linear(self.H[:T], self.W2, y, bias=self.b2, residual=residual, stream=stream)
        return y

    def forward_residual(self, x, h, h_out, x_out, eps=B.NORM_EPS, stream=None):
        """On the residual map: h_out = h + y, x_out = RMSNorm(h_out)."""
        self.forward(x, h_out, residual=h, stream=stream)
        B.ordermoe_rmsnorm(h_out, x.shape[0], self.d, eps, x_out, stream)
        return h_out, x_out


class LayerStack:
    """L MoE layers run through ordermoe_layer_forward with the token state
    (location, accumulated loss; Eqs. 36 and 44) carried from layer to layer, and
    DenseFFN layers between them. Steps, and the graphs captured from them, share
    the scratch: they may not overlap on the GPU."""

    def __init__(self, layers, tables, k, T_max, device, H=1, stride=0, P=None, few=False):
        """layers: dicts with W_r, W1, W3, W2 (device bf16). tables: a list of
        per-layer device buffers, or (for look-ahead, H > 1) one device buffer
        holding all layers' tables `stride` bytes apart; P [L-1, E, E] the
        transition matrices. Layer l looks min(H, L - l) - 1 layers ahead. few: steps of at most
        B.FEW_TOKENS tokens run each MoE layer in one launch (ordermoe_layer_few). Myopic steps
        of 1 to 8 tokens gain by it (64 narrow experts, us a layer: 1 token 50 -> 39, 8 tokens 125 ->
        113), 16 tokens do not (168 -> 173); with H = 3, whose decisions keep launches of their own, only
        wide experts do (1 token 148 -> 144; 64 narrow experts 104 -> 107, 16 tokens 227 -> 243). A
        DenseFFN in `layers` runs in its place; tables, P and L then count the MoE layers
        alone, in order (a stack may have none: tables, k, P and few say nothing then)."""
        dense = {l: lay for l, lay in enumerate(layers) if isinstance(lay, DenseFFN)}
        layers = [lay for lay in layers if not isinstance(lay, DenseFFN)]
        if not layers and not dense:
            raise ValueError("a stack needs a layer")
        E, dff, d = layers[0]["W1"].shape if layers else (0, 0, next(iter(dense.values())).d)
        L = len(layers)
        self.scratch = torch.empty(B.ordermoe_layer_scratch_bytes(T_max, E, d, dff, k) if layers else 0,
                                   dtype=torch.uint8, device=device)
        self.descs = []
        for l, lay in enumerate(layers):
            if isinstance(tables, torch.Tensor):
                t = tables[l * stride:]
                Hl = min(H, L - l)
                Pl = P[l:l + Hl - 1].contiguous() if Hl > 1 else None
            else:
                t, Hl, Pl = tables[l], 1, None
            self.descs.append(B.make_layer_desc(T_max, lay["W_r"], lay["W1"], lay["W3"], lay["W2"],
                                                t, k, self.scratch, lookahead_H=Hl,
                                                tables_stride=stride, P=Pl))
        for l, lay in dense.items():
            self.descs.insert(l, lay)
        self.d, self.T_max = d, T_max
        self.few_ws = None
        if few and layers:
            self.few_ws = few_workspace(min(T_max, B.FEW_TOKENS), E, d, dff, k, device)

    def _few(self, T):
        return self.few_ws is not None and T <= B.FEW_TOKENS

    def step(self, X_layers, home, loc, qhat, y_layers, counters=None, stream=None):
        """Layer l reads X_layers[l] and writes y_layers[l]; loc/qhat carry the
        trajectory (set loc = home, qhat = 0 before the first layer)."""
        T = X_layers[0].shape[0]
        out = B.make_few_out(counters=counters) if self._few(T) and counters is not None else None
        for desc, X, y in zip(self.descs, X_layers, y_layers):
            if isinstance(desc, DenseFFN):
                desc.forward(X, y, stream=stream)
                continue
            if self._few(T):
                B.ordermoe_layer_few(desc, T, X, home, loc, qhat, y, self.few_ws, out, stream)
                continue
            B.ordermoe_layer_forward(desc, T, X, home, loc, qhat, y, counters, 0, stream)

    def step_residual(self, hs, xs, home, loc, qhat, counters=None, logits=None,
                      eps=B.NORM_EPS, stream=None):
        """One pass over the stack on the residual map: xs[0] = RMSNorm(hs[0]),
        then layer l runs on xs[l] and writes hs[l + 1] = hs[l] + y_l and
        xs[l + 1] = RMSNorm(hs[l + 1]). hs, xs: L + 1 device buffers [T, d]
        bf16 (hs[0] is the input); logits: optional [L, T, E] f32 receiving each
        layer's router logits (layer-major; a dense layer leaves its own), or a
        list of [T, E] buffers (None: not wanted)."""
        T = hs[0].shape[0]
        B.ordermoe_rmsnorm(hs[0], T, self.d, eps, xs[0], stream)
        for l, desc in enumerate(self.descs):
            if isinstance(desc, DenseFFN):
                desc.forward_residual(xs[l], hs[l], hs[l + 1], xs[l + 1], eps, stream)
                continue
            if self._few(T):
                out = B.make_few_out(logits=None if logits is None else logits[l], counters=counters)
                B.ordermoe_layer_few_residual(desc, T, xs[l], hs[l], home, loc, qhat, eps, hs[l + 1],
                                              xs[l + 1], self.few_ws, out, stream)
                continue
            B.ordermoe_layer_forward_residual(desc, T, xs[l], hs[l], home, loc, qhat, eps,
                                              hs[l + 1], xs[l + 1],
                                              None if logits is None else logits[l], counters,
                                              stream)

    def capture(self, X_layers, home, loc, qhat, y_layers, counters=None, prologue=None):
        """Records one step (every layer's kernels, after the optional prologue,
        e.g. resetting loc and qhat) as a CUDA graph over these buffers, so a
        step is one graph launch. Returns the torch.cuda.CUDAGraph; replay()
        runs the step on the buffers' current contents."""
        return self._capture(lambda s: self.step(X_layers, home, loc, qhat, y_layers, counters,
                                                 stream=s), prologue)

    def capture_residual(self, hs, xs, home, loc, qhat, counters=None, prologue=None,
                         eps=B.NORM_EPS):
        """capture() of step_residual over these buffers."""
        return self._capture(lambda s: self.step_residual(hs, xs, home, loc, qhat, counters,
                                                          eps=eps, stream=s), prologue)

    def _capture(self, body, prologue):
        s = torch.cuda.Stream(device=self.scratch.device)
        s.wait_stream(torch.cuda.current_stream(self.scratch.device))
        with torch.cuda.stream(s):  # one eager step first: per-device set-up outside the capture
            if prologue is not None:
                prologue()
            body(s)
        torch.cuda.current_stream(self.scratch.device).wait_stream(s)
        torch.cuda.synchronize(self.scratch.device)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            if prologue is not None:
                prologue()
            body(s)
        return g


def exact_tables(E, M, device):
    """Selection tables that keep every routed expert (no substitutes: the
    threshold 2 exceeds any cosine; every expert on every server): the
    unmodified model, which a stack's calibration pass runs."""
    sim = torch.eye(E, dtype=torch.float32, device=device)
    group = torch.arange(E, dtype=torch.int32, device=device)
    x = torch.ones(M, E, dtype=torch.uint8, device=device)
    t = torch.zeros(B.ordermoe_tables_bytes(E, M), dtype=torch.uint8, device=device)
    f64 = lambda *sh: torch.ones(*sh, dtype=torch.float64, device=device)
    B.ordermoe_build_tables(sim, group, x, 2.0, 1.0, f64(M), f64(M, M), f64(M, M) * 0, 1.0, 1.0,
                            0.5, 0.5, t)
    return t


def calibrate_stack(layers, h_cal, k_freq, M, eps=B.NORM_EPS):
    """Offline statistics of a stack on the residual map (Section III-B on the
    representations each layer actually sees): the calibration tokens h_cal
    [N, d] pass through the unmodified stack (every routed expert kept), and
    layer l's similarity and counts (Eqs. 3-5) are taken over its own inputs
    x_l = RMSNorm(h_l), its transitions (Eq. 41) between the router logits of
    consecutive layers along the same pass. DenseFFN layers run in their place,
    and what is returned counts the MoE layers alone, in order, as LayerStack's
    tables and P do. Returns a dict: sim [L, E, E], counts [L, E],
    P [L-1, E, E], tcount [L-1, E, E], logits [L, N, E] (f32 device) of the L
    MoE layers, hs and xs (the residual states and normalised inputs of all
    layers, one more than there are)."""
    dev = h_cal.device
    N, d = h_cal.shape
    moe = [l for l, lay in enumerate(layers) if not isinstance(lay, DenseFFN)]
    L = len(moe)
    if L == 0:
        raise ValueError("calibrate_stack: no MoE layer")
    E = layers[moe[0]]["W1"].shape[0]
    # (more tokens than a dense layer serves: its weights, with room for these)
    run = [lay if not isinstance(lay, DenseFFN) or lay.T_max >= N
           else DenseFFN(lay.W1, lay.W2, N, lay.b1, lay.b2, lay.act) for lay in layers]
    tab = exact_tables(E, M, dev)
    stack = LayerStack(run, [tab] * L, k_freq, N, dev)
    hs = [h_cal] + [torch.empty_like(h_cal) for _ in layers]
    xs = [torch.empty_like(h_cal) for _ in range(len(layers) + 1)]
    home = torch.zeros(N, dtype=torch.uint8, device=dev)
    logits = torch.empty(L, N, E, dtype=torch.float32, device=dev)
    of = [None] * len(layers)  # a layer's logits
    for i, l in enumerate(moe):
        of[l] = logits[i]
    stack.step_residual(hs, xs, home, None, None, logits=of, eps=eps)
    sim = torch.empty(L, E, E, dtype=torch.float32, device=dev)
    counts = torch.empty(L, E, dtype=torch.int32, device=dev)
    ws = torch.empty(B.ordermoe_similarity_workspace_bytes(1, E, N), dtype=torch.uint8, device=dev)
    for i, l in enumerate(moe):
        B.ordermoe_similarity_no_logits(layers[l]["W_r"], xs[l], 1, E, d, N, k_freq, sim[i],
                                        counts[i], ws)
    P = torch.empty(max(L - 1, 1), E, E, dtype=torch.float32, device=dev)
    tcount = torch.empty(max(L - 1, 1), E, E, dtype=torch.int32, device=dev)
    if L >= 2:
        B.ordermoe_transitions_strided(logits, N, L, E, k_freq, E, N * E, tcount, P)
    return {"sim": sim, "counts": counts, "P": P[:L - 1], "tcount": tcount[:L - 1],
            "logits": logits, "xs": xs, "hs": hs}
