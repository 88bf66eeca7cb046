"""Performance cases of the attention half of a decoder block that serves many requests, and of the
per-request corrections of its projections.

  append    new tokens' keys and values into a paged cache, rotary positions on queries and keys
  attend    attention of one new token a sequence over the cache (grouped heads, ragged lengths),
            alone or adding up the weight that each cached token received
  evict     the cache cut to a budget of slots a head: the newest, the first and the most attended
            tokens stay
  adapters  low-rank corrections of many requests' own adapters, added to a shared projection

`run` computes them in elementary torch operations, or with `own` by the framework's calls.
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
BF16 = torch.bfloat16

# heads of queries, heads of the cache, width of a head
TINY = dict(Hq=4, H=4, D=64)       # d 256
WIDE = dict(Hq=32, H=8, D=128)     # d 4096, four query heads a cached one
FINE = dict(Hq=16, H=16, D=128)    # d 2048, every head its own keys
ONE = dict(Hq=16, H=1, D=128)      # all query heads on one cached head
ODD = dict(Hq=21, H=3, D=64)       # groups of seven
BIG = dict(Hq=8, H=4, D=256)       # wide heads


def listed():
    return [
        # one sequence of a tiny model, a short context: the latency of a call
        dict(name="attend_tiny", kind="attend", S=1, lo=0, hi=100, page=16, mass=False, **TINY),
        # one long document, one user
        dict(name="attend_long", kind="attend", S=1, lo=0, hi=131071, page=16, mass=False, **WIDE),
        # a decode batch of 128 requests of any age, one just begun
        dict(name="attend_batch", kind="attend", S=128, lo=1, hi=8191, page=32, mass=False, **WIDE),
        # a batch that keeps count of what is attended, for eviction; an idle row in it
        dict(name="attend_mass", kind="attend", S=17, lo=0, hi=4097, page=64, mass=True, **FINE),
        # one decoding token
        dict(name="append_1", kind="append", S=1, lo=1, hi=1, past=1000, page=16, adjacent=False,
             keep=False, **WIDE),
        # chunks of prompts of several requests, far positions
        dict(name="append_prompt", kind="append", S=5, lo=0, hi=1638, past=100000, page=64,
             adjacent=True, keep=True, **WIDE),
        # every decode step of a full cache: one token too many in each head
        dict(name="evict_step", kind="evict", S=32, lo=1025, hi=1025, budget=1024, recent=256, sinks=4,
             page=16, **WIDE),
        # prompts cut to a quarter and less; one request is below its budget
        dict(name="evict_prompt", kind="evict", S=8, lo=1500, hi=16383, budget=2048, recent=512, sinks=0,
             page=64, **WIDE),
        # one request's output projection
        dict(name="adapters_1", kind="adapters", T=1, K=4096, N=4096, R=16, n=1, run=1, f32=False,
             pad=0, ragged=False),
        # a decode batch of 128 requests on 32 adapters of several ranks, some requests without one
        dict(name="adapters_batch", kind="adapters", T=128, K=4096, N=6144, R=64, n=32, run=1, f32=False,
             pad=0, ragged=True),
        # odd sizes, rows inside wider buffers, results in 32 bits
        dict(name="adapters_odd", kind="adapters", T=301, K=1999, N=1009, R=24, n=7, run=5, f32=True,
             pad=24, ragged=True),
        # prompts of a few requests
        dict(name="adapters_prompt", kind="adapters", T=4096, K=4096, N=14336, R=64, n=8, run=512,
             f32=False, pad=0, ragged=False),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "append", "evict", "adapters", "adapters"])
    if kind == "adapters":
        n = _log_int(rng, 1, 200)
        T, K, N = _log_int(rng, 1, 4096), _log_int(rng, 64, 14336), _log_int(rng, 64, 14336)
        return dict(kind=kind, T=T, K=K, N=N, R=8 * rng.randint(1, 8 if n > 32 else 16), n=n,
                    run=_log_int(rng, 1, 512), f32=rng.random() < 0.25, pad=rng.choice([0, 0, 8, 40]),
                    ragged=rng.random() < 0.5)
    shape = dict(rng.choice([TINY, WIDE, WIDE, FINE, ONE, ODD, BIG]))
    page = rng.choice([8, 16, 32, 64, 128])
    most = 1 << 19  # slots times heads times width / 1024 of a cache, all sequences together
    S = _log_int(rng, 1, 256)
    if kind == "attend":
        hi = _log_int(rng, 1, 131072)
        while S * hi * shape["H"] * shape["D"] > most * 960:
            S, hi = (S + 1) // 2, (hi + 1) // 2
        return dict(kind=kind, S=S, lo=rng.choice([0, 1, hi // 2, hi]), hi=hi, page=page,
                    mass=rng.random() < 0.4, **shape)
    if kind == "append":
        S, hi = min(S, 64), rng.choice([1, _log_int(rng, 1, 2048)])
        while S * hi > 4096:
            S, hi = (S + 1) // 2, (hi + 1) // 2
        return dict(kind=kind, S=S, lo=rng.choice([0, 1, hi]) if hi > 1 else 1, hi=hi,
                    past=_log_int(rng, 1, 100000), page=page, adjacent=rng.random() < 0.5,
                    keep=rng.random() < 0.5, **shape)
    budget = _log_int(rng, 8, 4096)
    hi = budget + _log_int(rng, 1, 12288)
    while S * hi * shape["H"] * shape["D"] > most * 256:
        S = (S + 1) // 2
        if S == 1:
            hi = min(hi, budget + 4096)
            break
    return dict(kind=kind, S=S, lo=rng.choice([0, budget, budget + 1, hi]), hi=hi, budget=budget,
                recent=budget // rng.choice([2, 4, 8]), sinks=rng.choice([0, 1, 4]), page=page, **shape)


# ----------------------------------------------------------------- inputs
def _counts(c):
    """Lengths (attend, evict) or new tokens (append) of the sequences, evenly from lo to hi."""
    S, lo, hi = c["S"], c["lo"], c["hi"]
    return [hi] if S == 1 else [lo + (hi - lo) * i // (S - 1) for i in range(S)]


def _past(c):
    """Cached slots of the sequences before new tokens come: some of them hold a short past only, and
    a long one of tokens is behind them (positions do not count slots where a cache was cut)."""
    return [min(c["past"], 37 + 101 * i) for i in range(c["S"])]


def _normal(g, std, *shape, dt=BF16):
    return torch.empty(shape, dtype=dt, device=DEV).normal_(0.0, std, generator=g)


def _cache(c, g, order, lens):
    """A pool of pages, the pages of each sequence anywhere in it."""
    S, H, D, page = c["S"], c["H"], c["D"], c["page"]
    width = max(1, max((n + page - 1) // page for n in lens))
    pool = sum((n + page - 1) // page for n in lens) + 3
    free = order.sample(range(pool), pool)
    table = torch.zeros(S, width, dtype=torch.int32)
    for i, n in enumerate(lens):
        for j in range((n + page - 1) // page):
            table[i, j] = free.pop()
    return {"case": c, "lens": lens, "k": _normal(g, 1.0, pool, H, page, D),
            "v": _normal(g, 1.0, pool, H, page, D), "table": table.to(DEV),
            "len": torch.tensor(lens, dtype=torch.int32, device=DEV), "slots": width * page}


def _freq(D):
    return 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) * 2 / D)


def _inputs(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    order = random.Random(seed)
    if c["kind"] == "adapters":
        return _adapter_inputs(c, g, order)
    S, Hq, H, D = c["S"], c["Hq"], c["H"], c["D"]
    new = _counts(c)
    if c["kind"] != "append":
        order.shuffle(new)
    lens = new if c["kind"] != "append" else [a + b for a, b in zip(_past(c), new)]
    s = _cache(c, g, order, lens)
    slots = s["slots"]
    if c["kind"] == "append":
        T = sum(new)
        s["T"], s["new"] = T, new
        qkv = _normal(g, 1.0, T, (Hq + 2 * H) * D)  # one product's rows
        s["q"], s["nk"], s["nv"] = qkv.split([Hq * D, H * D, H * D], dim=1)
        s["starts"] = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int().to(DEV)
        base = [order.randint(0, c["past"]) for _ in range(S)]
        s["position"] = torch.tensor([b + j for b, n in zip(base, new) for j in range(n)],
                                     dtype=torch.int32, device=DEV)
        s["freq"] = _freq(D)
        s["q_out"] = torch.zeros(T, Hq * D, dtype=BF16, device=DEV)
        if c["keep"]:
            s["mass"] = _normal(g, 1.0, S, H, slots, dt=torch.float32).abs_()
            s["pos"] = torch.zeros(S, H, slots, dtype=torch.int32, device=DEV)
        return s
    if c["kind"] == "attend":
        s["q"] = _normal(g, 1.0, S, Hq * D)
        s["out"] = torch.zeros(S, Hq * D, dtype=BF16, device=DEV)
        s["lse"] = torch.zeros(S, Hq, dtype=torch.float32, device=DEV)
        if c["mass"]:
            s["mass0"] = _normal(g, 0.1, S, H, slots, dt=torch.float32).abs_()
            s["mass"] = s["mass0"].clone()
            s["pos"] = torch.zeros(S, H, slots, dtype=torch.int32, device=DEV)
        return s
    # weights as attention leaves them: a few tokens hold most; many of the rest have nothing at all
    m = torch.exp(_normal(g, 3.0, S, H, slots, dt=torch.float32))
    s["mass0"] = torch.where(m < 0.05, torch.zeros_like(m), m)
    # positions: one token a slot, in an order of its own for every head (an earlier cut moved them)
    far = _normal(g, 1.0, S, H, slots, dt=torch.float32)
    far.masked_fill_(torch.arange(slots, device=DEV) >= s["len"][:, None, None], math.inf)
    s["pos0"] = far.argsort(dim=2, stable=True).argsort(dim=2).int() + 1000 * (c["sinks"] == 0)
    s["newest"] = s["len"] - 1 + 1000 * (c["sinks"] == 0)
    s["mass"], s["pos"] = s["mass0"].clone(), s["pos0"].clone()
    s["len_out"] = torch.zeros_like(s["len"])
    return s


def _adapter_inputs(c, g, order):
    T, K, N, R, n, pad = c["T"], c["K"], c["N"], c["R"], c["n"], c["pad"]

    def rows(*shape, odd=False, std=1.0):
        w = shape[-1]
        ld = (w if odd else (w + 7) // 8 * 8) + pad
        return _normal(g, std, *shape[:-1], ld)[..., :w]

    s = {"case": c, "X": rows(T, K), "A": rows(n, R, K, std=0.02), "B": _normal(g, 0.1, n, N, R),
         "res": rows(T, N, odd=True)}
    # runs of tokens of one request; with more requests than adapters of some length, in any order
    ids, picks = [], list(range(n))
    order.shuffle(picks)
    while len(ids) < T:
        a = picks[(len(ids) // c["run"]) % n] if not c["ragged"] else order.randrange(-1, n)
        ids += [a] * c["run"]
    s["ids"] = torch.tensor(ids[:T], dtype=torch.int32, device=DEV)
    s["rank_host"] = [order.randint(1, R) if c["ragged"] else R for _ in range(n)]
    s["rank"] = torch.tensor(s["rank_host"], dtype=torch.int32, device=DEV)
    s["scale"] = 0.5 + torch.rand(n, device=DEV, generator=g)
    s["Y"] = torch.zeros(T, N + pad, dtype=torch.float32 if c["f32"] else BF16, device=DEV)[:, :N]
    return s


def prepare(case, seed):
    s, c = _inputs(case, seed), case
    if own:
        from paper_2607_17154_gb300 import binding as B
        if c["kind"] == "adapters":
            nbytes = B.ordermoe_adapters_workspace_bytes(c["T"], c["K"], c["N"], c["R"])
        else:
            s["cache"] = B.make_cache(s["k"], s["v"], s["table"], s["len"], s.get("mass"), s.get("pos"))
            nbytes = 0
            if c["kind"] == "attend":
                nbytes = B.ordermoe_attention_paged_workspace_bytes(s["cache"], c["Hq"], weights=c["mass"])
            elif c["kind"] == "evict":
                nbytes = B.ordermoe_cache_evict_workspace_bytes(s["cache"], c["budget"])
        s["ws"] = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------- runs
def _append(s, c):
    Hq, H, D, page, T = c["Hq"], c["H"], c["D"], c["page"], s["T"]
    a = s["position"].double()[:, None] * s["freq"]
    cos, sin = torch.cos(a).float()[:, None], torch.sin(a).float()[:, None]

    def turn(x, heads):
        x = x.reshape(T, heads, D).float()
        u, w = (x[..., 0::2], x[..., 1::2]) if c["adjacent"] else (x[..., :D // 2], x[..., D // 2:])
        u, w = u * cos - w * sin, u * sin + w * cos
        return (torch.stack((u, w), 3) if c["adjacent"] else torch.cat((u, w), 2)).reshape(T, heads, D)

    starts = s["starts"].long()
    t = torch.arange(T, device=DEV)
    seq = (t[:, None] >= starts[None, 1:]).sum(1)
    slot = s["len"].long()[seq] - (starts[seq + 1] - starts[seq]) + t - starts[seq]
    pages = s["table"][seq, slot // page].long()
    s["k"][pages, :, slot % page] = turn(s["nk"], H).to(BF16)
    s["v"][pages, :, slot % page] = s["nv"].reshape(T, H, D)
    s["q_out"].copy_(turn(s["q"], Hq).reshape(T, Hq * D))
    if c["keep"]:
        s["mass"][seq, :, slot] = 0.0
        s["pos"][seq, :, slot] = s["position"][:, None].expand(T, H)


def _attend(s, c):
    S, Hq, H, D, slots = c["S"], c["Hq"], c["H"], c["D"], s["slots"]
    pages = s["table"].long()
    k = s["k"][pages].transpose(1, 2).reshape(S * H, slots, D).float()
    x = torch.bmm(s["q"].view(S * H, Hq // H, D).float(), k.transpose(1, 2)) * (1.0 / math.sqrt(D))
    del k
    behind = torch.arange(slots, device=DEV) >= s["len"][:, None]  # [S][slots]
    x = x.view(S, H, Hq // H, slots).masked_fill_(behind[:, None, None], -math.inf)
    top = x.amax(3, keepdim=True)
    p = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(3, keepdim=True)  # 0: nothing is attended
    p = p / torch.where(total == 0.0, 1.0, total)
    v = s["v"][pages].transpose(1, 2).reshape(S * H, slots, D).float()
    s["out"].copy_(torch.bmm(p.view(S * H, Hq // H, slots), v).view(S, Hq * D))
    s["lse"].copy_((top + torch.log(total)).view(S, Hq))
    if c["mass"]:
        s["mass"] += p.sum(2)


def _evict(s, c):
    page, budget, slots = c["page"], c["budget"], s["slots"]
    s["len_out"].copy_(s["len"].clamp(max=budget))
    slot = torch.arange(slots, device=DEV)
    held = (slot < s["len"][:, None])[:, None]  # [S][1][slots]
    stays = (s["pos"] < c["sinks"]) | (s["pos"] > (s["newest"] - c["recent"])[:, None, None])
    key = torch.where(stays, math.inf, s["mass"]).masked_fill_(~held, -math.inf)
    order = torch.sort(key, dim=2, descending=True, stable=True).indices[..., :budget]
    kept = torch.zeros_like(stays).scatter_(2, order, True) & held
    full = (s["len"] > budget)[:, None, None]  # sequences that have too many
    i, h, to = (~kept & full & (slot < budget)).nonzero(as_tuple=True)
    fr = (kept & full & (slot >= budget)).nonzero(as_tuple=True)[2]
    for x in (s["mass"], s["pos"]):
        x[i, h, to] = x[i, h, fr]
    a, b = s["table"][i, to // page].long(), s["table"][i, fr // page].long()
    for x in (s["k"], s["v"]):
        x[a, h, to % page] = x[b, h, fr % page]


def _adapters(s):
    n, R, K = s["A"].shape
    low = (s["X"].float() @ s["A"].reshape(n * R, K).float().T).view(-1, n, R)  # of every adapter
    own_one = s["ids"][:, None] == torch.arange(n, device=DEV)
    used = torch.arange(R, device=DEV) < s["rank"][:, None]
    low = torch.where(own_one[:, :, None] & used, low * s["scale"][:, None], 0.0)
    y = low.view(-1, n * R) @ s["B"].transpose(0, 1).reshape(-1, n * R).float().T
    s["Y"].copy_(s["res"].float() + y)


def _outputs(s, c):
    names = {"append": ("q_out", "k", "v") + (("mass", "pos") if c.get("keep") else ()),
             "attend": ("out", "lse") + (("mass",) if c.get("mass") else ()),
             "evict": ("k", "v", "mass", "pos", "len_out"), "adapters": ("Y",)}[c["kind"]]
    return {n: s[n] for n in names}


def run(state):
    s, c = state, state["case"]
    kind = c["kind"]
    # what a pass changes begins as it was, so that every pass does the same work
    if kind == "attend" and c["mass"]:
        s["mass"].copy_(s["mass0"])
    if kind == "evict":
        s["mass"].copy_(s["mass0"])
        s["pos"].copy_(s["pos0"])
    if own:
        from paper_2607_17154_gb300 import binding as B
        if kind == "append":
            B.ordermoe_cache_append(s["cache"], s["nk"], s["nv"], q=s["q"], q_out=s["q_out"],
                                    starts=s["starts"], position=s["position"], inv_freq=s["freq"],
                                    adjacent=c["adjacent"])
        elif kind == "attend":
            B.ordermoe_attention_paged(s["cache"], s["q"], s["out"], s["ws"], lse=s["lse"],
                                       weights=c["mass"])
        elif kind == "evict":
            B.ordermoe_cache_evict(s["cache"], c["budget"], s["len_out"], s["ws"], newest=s["newest"],
                                   recent=c["recent"], sinks=c["sinks"])
        else:
            B.ordermoe_adapters(s["X"], s["A"], s["B"], s["ids"], s["Y"], s["ws"], scale=s["scale"],
                                rank=s["rank"], residual=s["res"])
    elif kind == "append":
        _append(s, c)
    elif kind == "attend":
        _attend(s, c)
    elif kind == "evict":
        _evict(s, c)
    else:
        _adapters(s)
    return _outputs(s, c)


def work(case):
    """Each input read and each output written once."""
    c = case
    if c["kind"] == "adapters":
        T, K, N, R, n = c["T"], c["K"], c["N"], c["R"], c["n"]
        picks = (T + c["run"] - 1) // c["run"]  # runs of tokens; the adapters they are expected to reach
        n_any = n + 1 if c["ragged"] else n
        hit = n * (1.0 - (1.0 - 1.0 / n_any) ** picks) if c["ragged"] else min(n, picks)
        r = (R + 1) / 2.0 if c["ragged"] else R
        rows = T * (n / n_any)
        return {"bytes": 2.0 * hit * r * (K + N) + 2.0 * rows * K + (6.0 if c["f32"] else 4.0) * T * N + 4.0 * T,
                "flops": 2.0 * rows * r * (K + N)}
    H, D, n = c["H"], c["D"], _counts(c)
    if c["kind"] == "append":
        T = sum(n)
        return {"bytes": 4.0 * T * (c["Hq"] + 2 * H) * D + T * (4 + (8.0 * H if c["keep"] else 0.0)),
                "flops": 3.0 * T * (c["Hq"] + H) * D}
    if c["kind"] == "attend":
        return {"bytes": sum(n) * H * (4.0 * D + (8.0 if c["mass"] else 0.0)) + 4.0 * c["S"] * c["Hq"] * (D + 1),
                "flops": 4.0 * sum(n) * c["Hq"] * D}
    # rows that move: those kept among the slots behind the budget, in the mean of any order
    b = c["budget"]
    moved = sum(b * (x - b) / x for x in n if x > b)
    return {"bytes": H * (sum(8.0 * x for x in n if x > b) + moved * (8.0 * D + 8.0)) + 8.0 * c["S"],
            "flops": 4.0 * H * sum(x for x in n if x > b)}


# ------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    c, s = case, _inputs(case, seed)
    f64 = torch.float64
    if c["kind"] == "adapters":
        y = s["res"].to(f64)
        for t0 in range(0, c["T"], 512):  # tokens of a slice, adapter after adapter, by masks
            ids = s["ids"][t0:t0 + 512]
            x = s["X"][t0:t0 + 512].to(f64)
            for a, r in enumerate(s["rank_host"]):
                on = (ids == a).to(f64)
                if not bool(on.any()):
                    continue
                low = torch.einsum("tk,rk->tr", x * on[:, None], s["A"][a, :r].to(f64))
                y[t0:t0 + 512] += torch.einsum("tr,nr->tn", low, s["B"][a, :, :r].to(f64)) * float(s["scale"][a])
        return {"Y": y}
    S, Hq, H, D, page = c["S"], c["Hq"], c["H"], c["D"], c["page"]
    if c["kind"] == "append":
        k, v = s["k"].to(f64), s["v"].to(f64)
        z = torch.polar(torch.ones((), dtype=f64, device=DEV),
                        s["position"].to(f64)[:, None] * s["freq"])[:, None]

        def turn(x, heads):
            x = x.reshape(s["T"], heads, D).to(f64)
            x = x.view(s["T"], heads, D // 2, 2) if c["adjacent"] else x.view(s["T"], heads, 2, D // 2).transpose(2, 3)
            y = torch.view_as_real(torch.view_as_complex(x.contiguous()) * z)
            return (y if c["adjacent"] else y.transpose(2, 3)).reshape(s["T"], heads, D)

        nk, nv, table, t = turn(s["nk"], H), s["nv"].reshape(s["T"], H, D).to(f64), s["table"].cpu(), 0
        pos = s["position"].cpu()
        for i, n in enumerate(s["new"]):
            for j in range(n):
                at = s["lens"][i] - n + j
                k[int(table[i, at // page]), :, at % page] = nk[t]
                v[int(table[i, at // page]), :, at % page] = nv[t]
                if c["keep"]:
                    s["mass"][i, :, at] = 0.0
                    s["pos"][i, :, at] = int(pos[t])
                t += 1
        out = {"q_out": turn(s["q"], Hq).reshape(s["T"], Hq * D), "k": k, "v": v}
        return dict(out, mass=s["mass"].to(f64), pos=s["pos"]) if c["keep"] else out
    if c["kind"] == "attend":
        out = torch.zeros(S, H, Hq // H, D, dtype=f64, device=DEV)
        lse = torch.full((S, H, Hq // H), -math.inf, dtype=f64, device=DEV)
        mass = s["mass0"].to(f64) if c["mass"] else None
        for i, n in enumerate(s["lens"]):
            if n == 0:
                continue
            slot = torch.arange(n, device=DEV)
            at = s["table"][i].long()[slot // page]
            k, v = s["k"][at, :, slot % page].to(f64), s["v"][at, :, slot % page].to(f64)  # [n][H][D]
            x = torch.einsum("hgd,nhd->hgn", s["q"][i].view(H, Hq // H, D).to(f64), k) / math.sqrt(D)
            p = torch.softmax(x, 2)
            out[i] = torch.einsum("hgn,nhd->hgd", p, v)
            lse[i] = torch.logsumexp(x, 2)
            if c["mass"]:
                mass[i, :, :n] += p.sum(1)
        res = {"out": out.reshape(S, Hq * D), "lse": lse.reshape(S, Hq)}
        return dict(res, mass=mass) if c["mass"] else res
    # a cut changes no number, it moves them: sorted on the host, head by head
    b = c["budget"]
    k, v, table = s["k"], s["v"], s["table"].long()
    mass, pos = s["mass0"].cpu(), s["pos0"].cpu()
    newest = s["newest"].tolist()
    src, dst = ([], [], []), ([], [], [])
    for i, n in enumerate(s["lens"]):
        for h in range(H if n > b else 0):
            m, p = mass[i, h, :n].tolist(), pos[i, h, :n].tolist()
            rank = [(0 if p[x] < c["sinks"] or p[x] > newest[i] - c["recent"] else 1, -m[x], x) for x in range(n)]
            rank = sorted((a, w if a else 0.0, x) for a, w, x in rank)
            kept = {x for _, _, x in rank[:b]}
            to = [x for x in range(b) if x not in kept]
            fr = sorted(x for x in kept if x >= b)
            for x, y in zip(to, fr):
                mass[i, h, x], pos[i, h, x] = m[y], p[y]
            for at, xs in ((dst, to), (src, fr)):
                at[0].extend([i] * len(xs))
                at[1].extend([h] * len(xs))
                at[2].extend(xs)
    si, sh, sx = (torch.tensor(a, dtype=torch.long, device=DEV) for a in src)
    di, dh, dx = (torch.tensor(a, dtype=torch.long, device=DEV) for a in dst)
    for a in (k, v):
        a[table[di, dx // page], dh, dx % page] = a[table[si, sx // page], sh, sx % page]
    return {"k": k.to(f64), "v": v.to(f64), "mass": mass.to(DEV).to(f64), "pos": pos.to(DEV), "len_out": s["len"].clamp(max=b)}
