"""The paged cache on the GPU: append, attention of one new token a sequence, eviction, each against the
definition in 64 bits, and a stack that runs them together."""
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


def make(lens, H, D, page, seed=0, extra=1, width=None, weights=False, fill=math.nan):
    """A cache of random pages in random order; every slot that no sequence holds is `fill`."""
    g, S = gen(seed), len(lens)
    n = width or max(1, max((x + page - 1) // page for x in lens)) + extra
    pool = S * n + 2
    k = torch.full((pool, H, page, D), fill, dtype=BF16, device=DEV)
    v = torch.full_like(k, fill)
    order = torch.randperm(pool, generator=torch.Generator().manual_seed(seed))
    table = order[:S * n].view(S, n).int().to(DEV)
    for s, x in enumerate(lens):
        i = torch.arange(x, device=DEV)
        at = table[s].long()[i // page]
        k[at, :, i % page] = torch.randn(x, H, D, device=DEV, generator=g).to(BF16)
        v[at, :, i % page] = torch.randn(x, H, D, device=DEV, generator=g).to(BF16)
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)
    mass = pos = None
    if weights:
        mass = torch.rand(S, H, n * page, device=DEV, generator=g)
        pos = torch.arange(n * page, dtype=torch.int32, device=DEV).expand(S, H, n * page).contiguous()
    return B.make_cache(k, v, table, length, mass, pos)


def rows(cache, s, which):
    """[slots, heads, dim] of sequence s in 64 bits."""
    k, v, table, length, _, _ = cache._keep
    i = torch.arange(max(0, min(int(length[s]), cache.slots)), device=DEV)
    t = k if which == "k" else v
    return t[table[s].long()[i // cache.page], :, i % cache.page].double()


def workspace(cache, hq, weights=False):
    return torch.empty(B.ordermoe_attention_paged_workspace_bytes(cache, hq, weights), dtype=torch.uint8, device=DEV)


def reference(cache, q, hq, scale=None):
    """out, lse and the weights per head of the cache in 64 bits, and their bounds.

    x: products of bf16 values are exact in fp32; D of them are summed in fp32, each sum off by 2^-23 at most (the
    tensor cores may cut instead of rounding), then the scale and its change to powers of two, 2^-22 of x. A change d of
    every x changes p = softmax(x) by 2 d of itself. exp2 is within 2^-21 of its value, p's two parts within 2^-16, sums
    of n + 64 terms (slots, and the joins' parts) within 2^-23 each. out is rounded once more, by 2^-8 of itself."""
    S, H, D = cache.seqs, cache.heads, cache.dim
    scale = D ** -0.5 if scale is None else scale
    out, lse = torch.zeros(S, hq, D, dtype=torch.double, device=DEV), torch.full((S, hq), -math.inf, dtype=torch.double, device=DEV)
    out_b, lse_b, ps = torch.zeros_like(out), torch.zeros_like(lse), []
    for s in range(S):
        k, v = rows(cache, s, "k"), rows(cache, s, "v")
        n = k.shape[0]
        if n == 0:
            ps.append(None)
            continue
        qs = q[s].double().view(H, hq // H, D)
        x = torch.einsum("hgd,nhd->hgn", qs, k) * scale
        dx = (torch.einsum("hgd,nhd->hgn", qs.abs(), k.abs()) * scale * (D + 8) * 2.0 ** -23 + x.abs() * 2.0 ** -22).amax(2)
        p = torch.softmax(x, 2)
        rel = 2 * dx + 2.0 ** -21 + (n + 64) * 2.0 ** -22
        out[s] = torch.einsum("hgn,nhd->hgd", p, v).reshape(hq, D)
        out_b[s] = (torch.einsum("hgn,nhd->hgd", p, v.abs()) * (rel + 2.0 ** -16)[..., None]).reshape(hq, D)
        lse[s] = torch.logsumexp(x, 2).reshape(hq)
        lse_b[s] = (dx + (n + 64) * 2.0 ** -23 + 2.0 ** -20 + lse[s].view(H, -1).abs() * 2.0 ** -21).reshape(hq)
        ps.append((p.sum(1), (p * rel[..., None]).sum(1) + hq // H * 2.0 ** -23 * p.sum(1)))
    out_b += out.abs() * 2.0 ** -8 + 2.0 ** -120
    return out.reshape(S, -1), out_b.reshape(S, -1), lse, lse_b, ps


def check(cache, q, out, lse, hq, scale=None):
    o, ob, l, lb, _ = reference(cache, q, hq, scale)
    assert bool(((out.double() - o).abs() <= ob).all()), float(((out.double() - o).abs() - ob).max())
    none = torch.isinf(l)
    assert bool((lse[none] == -math.inf).all())
    assert bool(((lse.double() - l).abs() <= lb)[~none].all()), float(((lse.double() - l).abs() - lb)[~none].max())


def attend(cache, q, hq, scale=None, weights=False, ws=None):
    out = torch.full_like(q, math.nan)
    lse = torch.full((cache.seqs, hq), math.nan, device=DEV)
    B.ordermoe_attention_paged(cache, q, out, workspace(cache, hq, weights) if ws is None else ws, scale=scale, lse=lse,
                               weights=weights)
    return out, lse


EDGE = [0, 1, 2, 7, 8, 9, 15, 16, 17, 31, 33, 64, 100, 0, 257, 1000]
SHAPES = [(4, 4, 64, 8), (4, 4, 64, 1), (21, 3, 64, 16), (16, 1, 64, 2), (32, 8, 128, 16), (16, 16, 128, 64), (16, 1, 128, 32),
          (40, 2, 128, 4), (9, 1, 128, 1024), (7, 7, 128, 256), (33, 1, 128, 16), (8, 4, 256, 16), (9, 1, 256, 8), (20, 2, 256, 128)]


@pytest.mark.parametrize("hq,H,D,page", SHAPES)
def test_attention_at_edges(hq, H, D, page):
    cache = make(EDGE, H, D, page, seed=hq)
    q = torch.randn(len(EDGE), hq * D, device=DEV, generator=gen(1)).to(BF16)
    out, lse = attend(cache, q, hq)
    check(cache, q, out, lse, hq)


@pytest.mark.parametrize("lens,hq,H,D,page", [
    ([70001], 32, 8, 128, 16), ([40000], 8, 1, 64, 64), ([1], 32, 8, 128, 16), ([5], 8, 4, 256, 16), ([20000, 3, 0], 8, 4, 256, 32),
    ([3, 9000, 0, 1, 4097, 12], 16, 1, 128, 16), ([i % 4 for i in range(1100)], 4, 2, 64, 8), ([0] * 700 + [50], 8, 8, 128, 16),
    ([100], 4, 4, 64, 16), ([17, 0, 300], 32, 8, 128, 16), ([480, 495], 33, 1, 128, 8), ([1, 129], 20, 2, 256, 16),
    ([0] * 1000 + [70] + [0] * 40 + [1, 90] + [0] * 500, 4, 2, 64, 16), ([33 if i % 37 == 0 else 0 for i in range(3000)], 8, 4, 64, 64),
    ([0, 0, 0], 4, 4, 64, 16), ([1200 - i for i in range(40)], 32, 8, 128, 16)])
def test_attention_of_long_and_many_sequences(lens, hq, H, D, page):
    cache = make(lens, H, D, page, seed=3)
    q = torch.randn(len(lens), hq * D, device=DEV, generator=gen(2)).to(BF16)
    ws = workspace(cache, hq).fill_(255)  # whatever it holds
    out, lse = attend(cache, q, hq, ws=ws)
    check(cache, q, out, lse, hq)
    again, _ = attend(cache, q, hq, ws=ws)
    assert torch.equal(again, out)


@pytest.mark.parametrize("scale,size", [(1.0, 6.0), (1e-3, 1.0), (0.7, 0.0)])
def test_attention_of_sharp_and_flat_scores(scale, size):
    cache = make([513, 40, 17], 2, 128, 16, seed=5)
    q = (torch.randn(3, 8 * 128, device=DEV, generator=gen(3)) * size).to(BF16)
    out, lse = attend(cache, q, 8, scale=scale)
    check(cache, q, out, lse, 8, scale)


@pytest.mark.parametrize("lens", [[0, 1, 50, 700, 3001], [33, 0, 200]])
@pytest.mark.parametrize("hq,H,D,page", [(4, 4, 64, 8), (32, 8, 128, 16), (40, 2, 128, 64), (16, 1, 128, 16), (9, 1, 256, 32)])
def test_weights_add_up_in_mass(hq, H, D, page, lens):
    cache = make(lens, H, D, page, seed=6, weights=True)
    q = torch.randn(len(lens), hq * D, device=DEV, generator=gen(4)).to(BF16)
    mass = cache._keep[4]
    before = mass.double()
    ws = workspace(cache, hq, True)
    out, lse = attend(cache, q, hq, weights=True, ws=ws)
    check(cache, q, out, lse, hq)
    ps = reference(cache, q, hq)[4]
    attend(cache, q, hq, weights=True, ws=ws)
    for s, p in enumerate(ps):
        n = 0 if p is None else p[0].shape[1]
        assert torch.equal(mass[s, :, n:].double(), before[s, :, n:])
        if n:
            want = before[s, :, :n] + 2 * p[0]
            assert bool(((mass[s, :, :n].double() - want).abs() <= 2 * p[1] + want * 2.0 ** -23).all())


def test_rows_in_wider_buffers_and_out_in_place():
    hq, H, D = 8, 2, 64
    lens = [30, 0, 500, 77]
    cache = make(lens, H, D, 16, seed=7)
    wide = torch.randn(4, hq * D + 24, device=DEV, generator=gen(5)).to(BF16)
    q = wide[:, 8:8 + hq * D]
    keep = wide.clone()
    res = torch.full((4, hq * D + 8), 7.0, dtype=BF16, device=DEV)
    lse = torch.empty(4, hq, device=DEV)
    B.ordermoe_attention_paged(cache, q, res[:, :hq * D], workspace(cache, hq), lse=lse)
    check(cache, q.contiguous(), res[:, :hq * D], lse, hq)
    assert bool((res[:, hq * D:] == 7.0).all()) and torch.equal(wide, keep)
    B.ordermoe_attention_paged(cache, q, q, workspace(cache, hq))
    assert torch.equal(q, res[:, :hq * D])
    assert torch.equal(wide[:, :8], keep[:, :8]) and torch.equal(wide[:, 8 + hq * D:], keep[:, 8 + hq * D:])


def test_scores_of_minus_infinity_and_values_that_are_no_numbers():
    cache = make([40, 40, 40], 1, 64, 16, seed=8)
    k, v, table = cache._keep[:3]
    q = torch.ones(3, 64, dtype=BF16, device=DEV)
    for j in range(3):  # every key of sequence 0: x = -inf; one of 1; one NaN key of 2
        k[table[0, j].long()] = -math.inf
    k[table[1, 0].long(), 0, 3] = -math.inf
    k[table[2, 0].long(), 0, 3, 5] = math.nan
    out, lse = attend(cache, q, 1)
    assert bool((out[0] == 0).all()) and float(lse[0, 0]) == -math.inf
    assert bool(torch.isnan(out[2]).all()) and math.isnan(float(lse[2, 0]))
    kk, vv = rows(cache, 1, "k")[:, 0], rows(cache, 1, "v")[:, 0]
    p = torch.softmax(kk.sum(1) / 8, 0)
    assert bool(torch.isfinite(out[1]).all())
    assert bool(((out[1].double() - p @ vv).abs() <= 2.0 ** -8 * (p @ vv).abs() + 2.0 ** -12 * (p @ vv.abs())).all())


def test_shared_pages_and_offsets_beyond_32_bits():
    H, D, page = 8, 128, 64
    pages = (1 << 31) // (H * page * D) + 40  # more than 2^31 values
    k = torch.zeros(pages, H, page, D, dtype=BF16, device=DEV)
    v = torch.zeros(pages, H, page, D, dtype=BF16, device=DEV)
    k[-16:] = torch.randn(16, H, page, D, device=DEV, generator=gen(9)).to(BF16)
    v[-16:] = torch.randn(16, H, page, D, device=DEV, generator=gen(10)).to(BF16)
    table = torch.tensor([[pages - 1 - i for i in range(10)], [pages - 1, pages - 3, pages - 16] + [0] * 7],
                         dtype=torch.int32, device=DEV)
    cache = B.make_cache(k, v, table, torch.tensor([10 * page - 3, 3 * page - 9], dtype=torch.int32, device=DEV))
    q = torch.randn(2, 16 * D, device=DEV, generator=gen(11)).to(BF16)
    out, lse = attend(cache, q, 16)
    check(cache, q, out, lse, 16)
    # and appended there
    length = cache._keep[3]
    length += 1
    nk, nv = (torch.randn(2, H * D, device=DEV, generator=gen(12 + i)).to(BF16) for i in range(2))
    with pytest.raises(ValueError):
        B.ordermoe_cache_append(cache, nk, nv, q_out=q)
    B.ordermoe_cache_append(cache, nk, nv)
    at = int(length[0]) - 1
    assert torch.equal(k[table[0, at // page].long(), :, at % page], nk[0].view(H, D))
    assert torch.equal(v[table[0, at // page].long(), :, at % page], nv[0].view(H, D))


def test_bad_pages_and_lengths_are_reported_and_read_as_zeros():
    for page in (8, 32):
        cache = make([70, 70, 70], 2, 64, page, seed=13)
        k, v, table, length = cache._keep[:4]
        q = torch.randn(3, 4 * 64, device=DEV, generator=gen(14)).to(BF16)
        good, _ = attend(cache, q, 4)
        bad = table.clone()
        table[1, 1] = -5
        out, _ = attend(cache, q, 4)
        assert B.ordermoe_device_error() == (B.DEV_BAD_INDEX, 1)
        assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2]) and bool(torch.isfinite(out[1]).all())
        table.copy_(bad)
        table[2, 0] = k.shape[0]
        attend(cache, q, 4)
        assert B.ordermoe_device_error() == (B.DEV_BAD_INDEX, 2)
        table.copy_(bad)
        k[torch.isnan(k)] = 0
        v[torch.isnan(v)] = 0
        length[0], length[1] = -3, cache.slots + 100
        out, lse = attend(cache, q, 4)
        assert B.ordermoe_device_error()[0] == B.DEV_BAD_INDEX
        assert bool((out[0] == 0).all())
        length[0], length[1] = 0, cache.slots
        assert torch.equal(attend(cache, q, 4)[0], out)


def test_a_captured_call_follows_the_lengths_and_two_graphs_share_a_workspace():
    hq, H, D = 16, 4, 128
    cache = make([900, 30, 0, 411], H, D, 16, seed=15, weights=True, fill=0.5)
    length = cache._keep[3]
    q = torch.randn(4, hq * D, device=DEV, generator=gen(16)).to(BF16)
    ws = workspace(cache, hq, True)
    outs = [torch.zeros_like(q) for _ in range(2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(s):
        for i in range(2):
            B.ordermoe_attention_paged(cache, q, outs[i], ws, weights=bool(i))
        s.synchronize()
        for i in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                B.ordermoe_attention_paged(cache, q, outs[i], ws, weights=bool(i))
            graphs.append(g)
    torch.cuda.synchronize()
    for lens in ([900, 30, 0, 411], [17, 0, 900, 1], [0, 0, 0, 0], [911, 911, 911, 911]):
        length.copy_(torch.tensor(lens))
        for g in graphs:
            g.replay()
        want, _ = attend(cache, q, hq)
        for o in outs:
            assert torch.equal(o, want)


def test_calls_on_another_stream():
    cache = make([300, 44], 2, 64, 16, seed=17)
    q = torch.randn(2, 4 * 64, device=DEV, generator=gen(18)).to(BF16)
    want, _ = attend(cache, q, 4)
    out, ws, s = torch.zeros_like(q), workspace(cache, 4), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    B.ordermoe_attention_paged(cache, q, out, ws, stream=s)
    s.synchronize()
    assert torch.equal(out, want)


# ------------------------------------------------------------------------- append
@pytest.mark.parametrize("hq,H,D,page,adjacent,rot", [
    (32, 8, 128, 16, False, 128), (4, 4, 64, 8, True, 64), (21, 3, 64, 1, False, 32), (8, 4, 256, 64, True, 16), (1, 1, 128, 16, False, 0),
    (64, 64, 256, 16, False, 256)])
def test_append(hq, H, D, page, adjacent, rot):
    past, new = [0, 5, 31, 1000, 16], [3, 0, 1, 40, 17]
    S, T, pad = 5, sum(new), 4
    cache = make([a + b for a, b in zip(past, new)], H, D, page, seed=20, weights=True, fill=0.25)
    k, v, table, length, mass, pos = cache._keep
    g = gen(21)
    qkv = torch.randn(T + pad, (hq + 2 * H) * D, device=DEV, generator=g).to(BF16)
    q, nk, nv = qkv.split([hq * D, H * D, H * D], dim=1)
    starts = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int().to(DEV)
    position = torch.randint(0, 1000000, (T + pad,), dtype=torch.int32, device=DEV, generator=g)
    position[:3] = torch.tensor([0, -5, (1 << 24) - 1], dtype=torch.int32)
    freq = 10000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) * 2 / max(rot, 1))
    want_k, want_v, want_mass, want_pos = k.clone(), v.clone(), mass.clone(), pos.clone()
    q_out = torch.full((T + pad, hq * D), 9.0, dtype=BF16, device=DEV)
    B.ordermoe_cache_append(cache, nk, nv, q=q, q_out=q_out, starts=starts, position=position,
                            inv_freq=freq if rot else None, adjacent=adjacent)

    def turned(x, heads):
        """The turn in 64 bits, and its bound: cos and sin within 2^-22, three roundings, one to bf16."""
        x = x[:T].double().reshape(T, heads, D).clone()
        part = x[..., :rot]
        a, b = (part[..., 0::2], part[..., 1::2]) if adjacent else (part[..., :rot // 2], part[..., rot // 2:])
        a, b = a.clone(), b.clone()
        th = position[:T].double()[:, None, None] * freq
        u, w = a * th.cos() - b * th.sin(), a * th.sin() + b * th.cos()
        far = torch.zeros_like(x)
        both = (a.abs() + b.abs()) * 2.0 ** -21
        if adjacent:
            x[..., 0:rot:2], x[..., 1:rot:2] = u, w
            far[..., 0:rot:2], far[..., 1:rot:2] = both, both
        else:
            x[..., :rot // 2], x[..., rot // 2:rot] = u, w
            far[..., :rot // 2], far[..., rot // 2:rot] = both, both
        far[..., :rot] += x[..., :rot].abs() * 2.0 ** -8
        return x, far

    x, far = turned(q, hq)
    assert bool(((q_out[:T].double().view(T, hq, D) - x).abs() <= far).all())
    assert bool((q_out[T:] == 9.0).all())
    x, far = turned(nk, H)
    t = 0
    for s in range(S):
        for j in range(new[s]):
            slot = past[s] + j
            p = int(table[s, slot // page])
            assert bool(((k[p, :, slot % page].double() - x[t]).abs() <= far[t]).all())
            want_k[p, :, slot % page] = k[p, :, slot % page]
            want_v[p, :, slot % page] = nv[t].view(H, D)
            want_mass[s, :, slot] = 0
            want_pos[s, :, slot] = position[t]
            t += 1
    assert torch.equal(k, want_k) and torch.equal(v, want_v) and torch.equal(mass, want_mass) and torch.equal(pos, want_pos)


def test_append_in_place_by_slot_and_bad_places():
    H, D, page = 2, 64, 16
    cache = make([17, 40, 3, 20], H, D, page, seed=22, fill=0.5)
    k, v, table, length = cache._keep[:4]
    nk, nv = (torch.randn(4, H * D, device=DEV, generator=gen(23 + i)).to(BF16) for i in range(2))
    q = torch.randn(4, 4 * D, device=DEV, generator=gen(25)).to(BF16)
    freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) * 2 / D)
    out = torch.empty_like(q)
    B.ordermoe_cache_append(cache, nk, nv, q=q, q_out=out, inv_freq=freq, position=(length - 1).contiguous())
    same = q.clone()
    B.ordermoe_cache_append(cache, nk, nv, q=same, q_out=same, inv_freq=freq)  # positions are slots
    assert torch.equal(same, out)
    before = k.clone(), v.clone()
    length[0] = 0  # idle: left out without a word
    left = torch.full_like(q, 3.0)
    B.ordermoe_cache_append(cache, nk, nv, q=q, q_out=left, inv_freq=freq)
    assert B.ordermoe_device_error()[0] == 0
    assert bool((left[0] == 3.0).all()) and torch.equal(left[1:], out[1:]) and torch.equal(k, before[0])
    length[0], length[1], length[2] = -1, cache.slots + 1, 3
    table[2, 0] = k.shape[0] + 7
    left = torch.full_like(q, 3.0)
    B.ordermoe_cache_append(cache, nk, nv, q=q, q_out=left, inv_freq=freq)
    assert B.ordermoe_device_error()[0] == B.DEV_BAD_INDEX
    assert bool((left[:3] == 3.0).all()) and torch.equal(left[3], out[3])
    assert torch.equal(k, before[0]) and torch.equal(v, before[1])


# -------------------------------------------------------------------------- evict
def evicted(cache, budget, recent, sinks, newest):
    """The cache after a cut, slot by slot on the host: k, v, mass, pos, length."""
    k, v, table, length, mass, pos = (None if t is None else t.cpu() for t in cache._keep)
    k, v, mass = k.clone(), v.clone(), mass.clone()
    pos = None if pos is None else pos.clone()
    out = length.clone()
    for s in range(cache.seqs):
        n = int(length[s])
        if n <= budget:
            continue
        out[s] = budget
        for h in range(cache.heads):
            p = list(range(n)) if pos is None else pos[s, h, :n].tolist()
            m = [0.0 if x != x else x for x in mass[s, h, :n].tolist()]
            last = n - 1 if newest is None else int(newest[s])
            order = sorted(range(n), key=lambda i: (0, 0.0, i) if p[i] < sinks or p[i] > last - recent else (1, -m[i], i))
            kept = set(order[:budget])
            to = [i for i in range(budget) if i not in kept]
            fr = [i for i in range(budget, n) if i in kept]
            for x, y in zip(to, fr):
                a, b = (int(table[s, x // cache.page]), x % cache.page), (int(table[s, y // cache.page]), y % cache.page)
                k[a[0], h, a[1]], v[a[0], h, a[1]] = k[b[0], h, b[1]], v[b[0], h, b[1]]
                mass[s, h, x] = mass[s, h, y]
                if pos is not None:
                    pos[s, h, x] = pos[s, h, y]
    return k, v, mass, pos, out


def cut(cache, budget, recent=0, sinks=0, newest=None):
    k, v, _, length, mass, pos = cache._keep
    want = evicted(cache, budget, recent, sinks, newest)
    out = torch.full_like(length, -1)
    ws = torch.empty(B.ordermoe_cache_evict_workspace_bytes(cache, budget), dtype=torch.uint8, device=DEV).fill_(255)
    B.ordermoe_cache_evict(cache, budget, out, ws, newest=newest, recent=recent, sinks=sinks)
    for n, got, w in zip("k v mass pos length".split(), (k, v, mass, pos, out), want):
        if w is not None:
            same = torch.equal(got.cpu().view(torch.int16), w.view(torch.int16)) if w.dtype == BF16 else \
                torch.equal(torch.nan_to_num(got.cpu().double(), 1e30), torch.nan_to_num(w.double(), 1e30))
            assert same, n


@pytest.mark.parametrize("H,D,page,lens,budget,recent,sinks", [
    (2, 64, 8, [0, 1, 15, 16, 17, 18, 40], 16, 4, 2), (3, 128, 16, [700, 33, 5], 32, 32, 0), (1, 256, 4, [1000, 999], 1, 1, 0),
    (8, 128, 64, [1025] * 3, 1024, 256, 4), (2, 64, 16, [2500, 3000], 2049, 100, 1), (1, 64, 16, [60000], 777, 10, 3),
    (4, 128, 8, [1025, 1030, 1024], 1024, 100, 2), (2, 256, 1, [40, 64], 30, 3, 1), (2, 64, 16, [4095, 4000], 4060, 64, 0),
    (2, 128, 16, [5000, 700, 701], 700, 10, 3), (1, 64, 32, [16384], 9000, 0, 0), (1, 64, 16, [20000, 16385], 3000, 100, 4)])
def test_evict(H, D, page, lens, budget, recent, sinks):
    cache = make(lens, H, D, page, seed=30, weights=True)
    length, mass, pos = cache._keep[3:]
    g = gen(31)
    perm = torch.rand(pos.shape, device=DEV, generator=g)  # any order of positions, one token a slot
    perm.masked_fill_(torch.arange(cache.slots, device=DEV) >= length[:, None, None], 9.0)
    pos.copy_(perm.argsort(dim=2, stable=True).argsort(dim=2))
    mass[..., ::3] = 0.0  # ties
    cut(cache, budget, recent, sinks, newest=(length - 1).contiguous())


@pytest.mark.parametrize("fill", ["zeros", "equal", "signs", "nan"])
def test_evict_of_ties_signs_and_values_that_are_no_numbers(fill):
    cache = make([500, 64, 333], 2, 64, 16, seed=32, weights=True)
    mass = cache._keep[4]
    if fill in ("zeros", "equal"):
        mass.fill_(0.0 if fill == "zeros" else 2.5)
        mass[0, 0, 7] = -0.0 if fill == "zeros" else 2.5
    else:
        mass.copy_(torch.randn(mass.shape, device=DEV, generator=gen(33)).round())
        mass[0, 0, 9], mass[0, 0, 11] = math.inf, -math.inf
        if fill == "nan":
            mass[:, :, ::7] = math.nan
    cut(cache, 100)


def test_evict_without_positions_and_protected_ties():
    cache = make([200, 90], 2, 64, 16, seed=34, weights=True)
    k, v, table, length, mass, _ = cache._keep
    cut(B.make_cache(k, v, table, length, mass), 50, recent=20, sinks=5)
    cache = make([200], 2, 64, 16, seed=35, weights=True)
    cache._keep[5].fill_(3)  # one position for all: everything is protected, the lowest slots stay
    cut(cache, 50, recent=20, sinks=5, newest=torch.tensor([3], dtype=torch.int32, device=DEV))


def test_evict_reports_bad_pages_and_lengths():
    cache = make([60, 60], 1, 64, 16, seed=36, weights=True)
    k, v, table, length, mass, pos = cache._keep
    mass.copy_(torch.arange(cache.slots, device=DEV).float().expand_as(mass))  # the last ones stay
    before = k.clone()
    table[0, 3] = -1
    out = torch.zeros_like(length)
    ws = torch.empty(B.ordermoe_cache_evict_workspace_bytes(cache, 16), dtype=torch.uint8, device=DEV)
    B.ordermoe_cache_evict(cache, 16, out, ws)
    assert B.ordermoe_device_error() == (B.DEV_BAD_INDEX, 0)
    assert out.tolist() == [16, 16]
    i = torch.arange(44, 60, device=DEV)
    assert torch.equal(k[table[1, 0].long(), 0], before[table[1].long()[i // 16], 0, i % 16])
    length[1] = 10 ** 6
    B.ordermoe_cache_evict(cache, cache.slots, out, torch.empty(1 << 20, dtype=torch.uint8, device=DEV))
    assert B.ordermoe_device_error() == (B.DEV_BAD_INDEX, 1) and out.tolist() == [60, cache.slots]


# ----------------------------------------------------------------------- together
def test_steps_of_append_attention_and_eviction():
    """Sequences that grow a token a step and are cut whenever they pass a budget, beside a host's model in 64 bits that
    keeps what the cache keeps."""
    S, hq, H, D, page, budget = 3, 8, 2, 64, 8, 40
    g = gen(40)
    from paper_2607_17154_gb300.layer import PagedCache
    c = PagedCache(S, budget + 1, H, D, DEV, page=page, weights=True)
    freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) * 2 / D)
    ws = workspace(c.cache, hq, True)
    out, lse = torch.empty(S, hq * D, dtype=BF16, device=DEV), torch.empty(S, hq, device=DEV)
    for step in range(60):
        qkv = torch.randn(S, (hq + 2 * H) * D, device=DEV, generator=g).to(BF16)
        q, k, v = qkv.split([hq * D, H * D, H * D], dim=1)
        c.advance()
        B.ordermoe_cache_append(c.cache, k, v, q=q, q_out=q, position=c.position, inv_freq=freq)
        B.ordermoe_attention_paged(c.cache, q, out, ws, lse=lse, weights=True)
        check(c.cache, q, out, lse, hq)
        total = c.mass[:, :, :int(c.length[0])].double()
        # a slot's newest token has its weights, what was cut took its own along: no more than one a step and query head
        assert bool((total.sum(2) <= (step + 1) * hq // H * (1 + 2.0 ** -15)).all())
        want = evicted(c.cache, budget, 8, 2, c.position.cpu())
        c.length.copy_(c.cut(budget, recent=8, sinks=2))
        assert torch.equal(c.k.cpu(), want[0]) and torch.equal(c.mass.cpu(), want[2]) and torch.equal(c.pos.cpu(), want[3])
        assert torch.equal(c.length.cpu(), want[4])
    for s in range(S):
        for h in range(H):
            held = set(c.pos[s, h, :budget].tolist())
            assert len(held) == budget and {0, 1} <= held and set(range(52, 60)) <= held


def test_a_stack_with_attention_and_adapters_in_a_graph():
    """Decoding steps of attention, dense and MoE layers: the same bits eagerly and replayed, and the attention layer's
    own arithmetic against 64 bits."""
    from paper_2607_17154_gb300 import synth
    from paper_2607_17154_gb300.layer import DecodeAttention, DenseFFN, LayerStack, PagedCache, exact_tables
    S, d, hq, H, D, R, n = 4, 256, 4, 2, 64, 16, 3
    w = synth.workload("tiny")
    inp = synth.layer_inputs(w, seed=1)
    moe = {"W_r": inp["Wr"].to(DEV), **{x: inp[x].to(DEV) for x in ("W1", "W3", "W2")}}
    g = gen(50)
    rnd = lambda *s, std=0.05: (torch.randn(*s, device=DEV, generator=g) * std).to(BF16)
    wide = (hq + 2 * H) * D
    ad = {"A_qkv": rnd(n, R, d), "B_qkv": rnd(n, wide, R), "A_o": rnd(n, R, hq * D), "B_o": rnd(n, d, R),
          "scale": torch.tensor([1.0, 0.5, 2.0], device=DEV), "rank": torch.tensor([16, 3, 9], dtype=torch.int32, device=DEV)}
    freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) * 2 / D)
    Wqkv, Wo = [rnd(wide, d) for _ in range(2)], [rnd(d, hq * D) for _ in range(2)]
    dense = DenseFFN(rnd(512, d), rnd(d, 512), S)

    def stack():
        first = PagedCache(S, 40, H, D, DEV, page=16)
        second = PagedCache(S, 40, H, D, DEV, page=16, share=first, weights=True)
        at = [DecodeAttention(Wqkv[i], Wo[i], c, hq, inv_freq=freq, weights=bool(i), adapters=ad if i == 0 else None)
              for i, c in enumerate((first, second))]
        at[0].ids.copy_(torch.tensor([2, -1, 0, 1]))
        tab = exact_tables(w.E, w.M, DEV)
        return first, second, at, LayerStack([at[0], moe, at[1], dense], [tab], w.k, S, DEV)

    def buffers():
        return [torch.zeros(S, d, dtype=BF16, device=DEV) for _ in range(5)], \
               [torch.zeros(S, d, dtype=BF16, device=DEV) for _ in range(5)]

    tokens = [rnd(S, d, std=1.0) for _ in range(6)]
    home = torch.zeros(S, dtype=torch.uint8, device=DEV)
    first, second, at, st = stack()
    hs, xs = buffers()
    eager = []
    for x in tokens:
        hs[0].copy_(x)
        first.advance()
        st.step_residual(hs, xs, home, None, None)
        eager.append(hs[4].clone())
    # the last step's first layer in 64 bits, from the layer's own rounded q, o
    a = at[0]
    o, ob, _, _, _ = reference(first.cache, a.q, hq)
    assert bool(((a.o.double() - o).abs() <= ob).all())
    y = a.o.double() @ Wo[0].double().T
    sum_y = a.o.double().abs() @ Wo[0].double().abs().T
    mid = hs[0].double() + y
    low = torch.zeros_like(y)
    for s, i in enumerate(a.ids.tolist()):
        if i >= 0:
            r = int(ad["rank"][i])
            low[s] = float(ad["scale"][i]) * ad["B_o"][i, :, :r].double() @ (ad["A_o"][i, :r].double() @ a.o[s].double())
    bound = 2.0 ** -8 * mid.abs() * (1 + 2.0 ** -8) + 2.0 ** -8 * (mid + low).abs() + 2.0 ** -12 * (sum_y + low.abs()) + 2.0 ** -14
    assert bool(((hs[1].double() - mid - low).abs() <= bound).all())
    # replayed
    first, second, at, st = stack()
    hs, xs = buffers()
    graph = st.capture_residual(hs, xs, home, None, None, prologue=first.advance)
    first.length.zero_()
    first.position.fill_(-1)
    second.mass.zero_()
    for x, want in zip(tokens, eager):
        hs[0].copy_(x)
        graph.replay()
        assert torch.equal(hs[4], want)
    assert first.length.tolist() == [6] * S


def test_layers_refuse_other_batches_and_calibration():
    from paper_2607_17154_gb300.layer import DecodeAttention, PagedCache, calibrate_stack
    c = PagedCache(2, 16, 1, 64, DEV, page=16)
    z = lambda *s: torch.zeros(*s, dtype=BF16, device=DEV)
    a = DecodeAttention(z(192, 64), z(64, 64), c, 1)
    with pytest.raises(ValueError, match="2 sequences"):
        a.forward(z(3, 64), z(3, 64))
    with pytest.raises(ValueError, match="attention"):
        calibrate_stack([a], z(8, 64), 1, 1)
    with pytest.raises(ValueError):
        DecodeAttention(z(192, 64), z(64, 128), c, 1)
    with pytest.raises(ValueError):
        PagedCache(3, 16, 1, 64, DEV, page=16, share=c)


def test_a_captured_cut_follows_lengths_and_weights():
    for slots, budget in ((1040, 1024), (2992, 300), (20000, 500)):  # by itself, with a second launch, long rows
        H, D, page = 2, 64, 16
        cache = make([min(slots, 40)] * 2, H, D, page, seed=60, width=slots // page, extra=0, weights=True, fill=0.5)
        k, v, table, length, mass, pos = cache._keep
        out, newest = torch.zeros_like(length), torch.zeros_like(length)
        ws = torch.empty(B.ordermoe_cache_evict_workspace_bytes(cache, budget), dtype=torch.uint8, device=DEV)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            B.ordermoe_cache_evict(cache, budget, out, ws, newest=newest, recent=9, sinks=1)
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                B.ordermoe_cache_evict(cache, budget, out, ws, newest=newest, recent=9, sinks=1)
        torch.cuda.synchronize()
        for i, lens in enumerate(([slots, 7], [budget + 1, budget], [slots - 5, slots])):
            length.copy_(torch.tensor(lens))
            newest.copy_(length - 1)
            mass.copy_(torch.rand(mass.shape, device=DEV, generator=gen(61 + i)))
            k.copy_(torch.randn(k.shape, device=DEV, generator=gen(71 + i)).to(BF16))
            want = evicted(cache, budget, 9, 1, newest.cpu())
            g.replay()
            for got, w in zip((k, v, mass, pos, out), want):
                assert torch.equal(got.cpu(), w)
            pos.copy_(torch.arange(cache.slots, dtype=torch.int32, device=DEV).expand_as(pos))


def test_lengths_and_queries_written_by_the_kernels_before():
    """Lengths, queries and the cache change right before each call, nothing waits in between: the same bits as with a wait
    after every step."""
    hq, H, D = 16, 4, 128
    cache = make([2000, 2000, 2000], H, D, 16, seed=80, weights=True, fill=0.5)
    k, v, table, length, mass, pos = cache._keep
    ws = workspace(cache, hq, True)
    q = torch.zeros(3, hq * D, dtype=BF16, device=DEV)
    out = torch.zeros_like(q)
    g = gen(81)
    sets = [(torch.randint(0, 2001, (3,), dtype=torch.int32, device=DEV, generator=g), torch.randn(q.shape, device=DEV, generator=g).to(BF16),
             torch.randn(3, 2 * H * D, device=DEV, generator=g).to(BF16)) for _ in range(24)]

    def steps(wait):
        k0, v0, res = k.clone(), v.clone(), []
        mass.zero_()
        for n, x, kv in sets:
            length.copy_(n)
            wait()
            q.copy_(x)
            wait()
            B.ordermoe_cache_append(cache, kv[:, :H * D], kv[:, H * D:])
            wait()
            B.ordermoe_attention_paged(cache, q, out, ws, weights=True)
            wait()
            res += [out.clone(), mass.clone()]
        k.copy_(k0)
        v.copy_(v0)
        return res

    want = steps(torch.cuda.synchronize)
    for _ in range(4):
        for a, b in zip(steps(lambda: None), want):
            assert torch.equal(a, b)


def filled(seqs, slots, H=2, D=64, seed=120):
    """A PagedCache whose sequences are full, weights and values random."""
    from paper_2607_17154_gb300.layer import PagedCache
    c = PagedCache(seqs, slots, H, D, DEV, page=16, weights=True)
    fill(c, seed)
    return c


def fill(c, seed):
    g = gen(seed)
    for t in (c.k, c.v, c.mass):
        t.copy_(torch.rand(t.shape, device=DEV, generator=g))
    c.pos.copy_(torch.arange(c.cache.slots, dtype=torch.int32, device=DEV).expand_as(c.pos))
    c.length.fill_(c.cache.slots)
    c.position.fill_(c.cache.slots - 1)


def same_cache(c, out, want):
    return all(torch.equal(a.cpu(), b) for a, b in zip((c.k, c.v, c.mass, c.pos, out), want))


def test_cuts_of_other_budgets_leave_a_captured_one_its_memory():
    """A captured cut is replayed after cuts with other budgets, when what those could have given back to the allocator is
    in use by others."""
    c = filled(3, 208)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        first = c.cut(64, recent=4, sinks=2)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            assert c.cut(64, recent=4, sinks=2).data_ptr() == first.data_ptr()
    torch.cuda.synchronize()
    for budget in (32, 150, 208, 10 ** 6):  # the last two cut nothing
        fill(c, budget)
        want = evicted(c.cache, budget, 4, 2, c.position.cpu())
        assert same_cache(c, c.cut(budget, recent=4, sinks=2), want)
    del first
    others = [torch.full((n,), 7, dtype=torch.uint8, device=DEV) for n in [512] * 64 + [4096] * 64 + [65536] * 16]
    fill(c, 121)
    want = evicted(c.cache, 64, 4, 2, c.position.cpu())
    graph.replay()
    assert same_cache(c, c.cut(208), want[:4] + (c.length.cpu(),))  # (nothing more to cut)
    assert all(bool((o == 7).all()) for o in others)


def test_cut_on_another_stream():
    """The buffers of a cut that runs behind pending work on a stream of its own are nobody else's."""
    c, s = filled(3, 208), torch.cuda.Stream()
    want = evicted(c.cache, 50, 0, 0, c.position.cpu())
    busy = torch.zeros(1 << 26, device=DEV)
    torch.cuda.synchronize()
    for _ in range(20):
        busy += 1  # pending on the current stream, with temporary memory that it gives back
        (busy[:4096] * 2).sum()
    with torch.cuda.stream(s):
        for _ in range(20):
            busy.square()
    out = c.cut(50, stream=s)
    s.synchronize()
    assert same_cache(c, out, want)
    torch.cuda.synchronize()


def test_a_cache_without_weights_is_not_cut():
    from paper_2607_17154_gb300.layer import PagedCache
    with pytest.raises(B.OrderMoEError, match="mass"):
        PagedCache(2, 32, 1, 64, DEV, page=16).cut(8)


def attention_stack(S, slots, seed):
    """Two layers of attention that share lengths (the second keeps weights) and a dense one."""
    from paper_2607_17154_gb300.layer import DecodeAttention, DenseFFN, LayerStack, PagedCache
    d, hq, H, D, g = 256, 4, 2, 64, gen(seed)
    rnd = lambda *s: (torch.randn(*s, device=DEV, generator=g) * 0.05).to(BF16)
    freq = 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64, device=DEV) * 2 / D)
    first = PagedCache(S, slots, H, D, DEV, page=16)
    second = PagedCache(S, slots, H, D, DEV, page=16, share=first, weights=True)
    layers = [DecodeAttention(rnd((hq + 2 * H) * D, d), rnd(d, hq * D), c, hq, inv_freq=freq, weights=c is second)
              for c in (first, second)]
    layers.append(DenseFFN(rnd(512, d), rnd(d, 512), S))
    hs, xs = ([torch.zeros(S, d, dtype=BF16, device=DEV) for _ in range(4)] for _ in range(2))
    return (first, second), LayerStack(layers, [], 1, S, DEV), hs, xs


def state(caches):
    return [t.clone() for c in caches for t in (c.k, c.v, c.mass, c.pos, c.length, c.position) if t is not None]


@pytest.mark.parametrize("inside", [True, False])
def test_a_capture_leaves_the_caches_as_they_are(inside):
    """Requests are held while the step is captured, one of them with a full cache and one idle: what the caches hold
    stays, and the graph then goes on where the eager steps ended. The step's advance is captured, or called before each
    replay."""
    S, slots, steps = 4, 16, 5
    tokens = [torch.randn(S, 256, device=DEV, generator=gen(110 + i)).to(BF16) for i in range(2 * steps)]
    home = torch.zeros(S, dtype=torch.uint8, device=DEV)
    results = []
    for captured in (False, True):
        caches, stack, hs, xs = attention_stack(S, slots, 100)
        c, got = caches[0], []

        def run(step, x):
            hs[0].copy_(x)
            step()
            got.append(hs[3].clone())

        def eager():
            c.advance()
            stack.step_residual(hs, xs, home, None, None)

        for x in tokens[:steps]:
            run(eager, x)
        step = eager
        if captured:
            length, position = c.length.clone(), c.position.clone()
            c.length[1], c.length[2] = slots, 0  # a full one and an idle one, for the capture alone
            before = state(caches)
            graph = stack.capture_residual(hs, xs, home, None, None, prologue=c.advance if inside else None)
            for a, b in zip(state(caches), before):
                assert torch.equal(a, b)
            c.length.copy_(length)
            c.position.copy_(position)
            step = graph.replay if inside else lambda: (c.advance(), graph.replay())
        for x in tokens[steps:]:
            run(step, x)
        results.append(got + state(caches))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert c.length.tolist() == [2 * steps] * S and c.position.tolist() == [2 * steps - 1] * S


def test_a_capture_whose_prologue_cuts():
    """A prologue that cuts the cache before it advances: nothing is cut while the step is captured."""
    S, slots, budget = 3, 16, 8
    caches, stack, hs, xs = attention_stack(S, slots, 101)
    first, second = caches
    home = torch.zeros(S, dtype=torch.uint8, device=DEV)

    def prologue():
        first.length.copy_(second.cut(budget, recent=2, sinks=1))
        first.advance()

    for i in range(12):
        hs[0].copy_(torch.randn(S, 256, device=DEV, generator=gen(130 + i)).to(BF16))
        first.advance()
        stack.step_residual(hs, xs, home, None, None)
    before = state(caches)
    graph = stack.capture_residual(hs, xs, home, None, None, prologue=prologue)
    for a, b in zip(state(caches), before):
        assert torch.equal(a, b)
    want = evicted(second.cache, budget, 2, 1, second.position.cpu())
    graph.replay()
    assert first.length.tolist() == [budget + 1] * S
    assert torch.equal(second.pos[:, :, :budget].cpu(), want[3][:, :, :budget])


def held(cache, x):
    """Places of sequence s's first x[s] slots: pages and rows in them."""
    table = cache._keep[2].long()
    return [(table[s][(i := torch.arange(n, device=DEV)) // cache.page], i % cache.page) for s, n in enumerate(x)]


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("lens,H", [([40, 0, 500], 2), ([5000], 1), ([16] * 2000 + [9000], 1)])
def test_values_behind_scores_of_minus_infinity_alone_say_nothing(lens, H, bad):
    """Every score of a sequence is -inf: 0 and -inf, whatever its values hold. Rows that a warp, a CTA's warps and CTAs share."""
    cache = make(lens, H, 64, 16, seed=92, weights=True)
    k, v = cache._keep[:2]
    for at, row in held(cache, lens):
        k[at, :, row] = -math.inf
        v[at, :, row] = bad
    q = torch.ones(len(lens), 2 * H * 64, dtype=BF16, device=DEV)
    before = cache._keep[4].clone()
    out, lse = attend(cache, q, 2 * H, weights=True)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())
    assert torch.equal(cache._keep[4], before)


BORDERS = [([70001], 32, 8, 128, 16), ([40000], 8, 1, 64, 64), ([20000, 3, 0], 8, 4, 256, 32), ([3, 9000, 0, 1, 4097, 12], 16, 1, 128, 16),
           ([480, 495], 33, 1, 128, 8), ([1200 - i for i in range(40)], 32, 8, 128, 16), ([2000, 17], 9, 1, 256, 4), ([5000], 40, 2, 128, 16)]


@pytest.mark.parametrize("steps", [False, True])
@pytest.mark.parametrize("lens,hq,H,D,page", BORDERS)
def test_every_unit_of_slots_counts_once(lens, hq, H, D, page, steps):
    """One slot of each unit of 16 holds the value 1 in a column of its own, all others are 0: a unit that is lost or
    counted twice between warps and CTAs changes an output from p to 0 or 2 p. Keys are equal, or (steps) their scores are
    integers in powers of two that rise and fall from unit to unit, so that partial results are joined with other maxima.

    Equal keys: x = 0 and all sums are whole numbers, so p = 1 / n is off by a division (2^-24) and out by its rounding (2^-8);
    lse = log2f(n) ln 2 by 2^-22 of itself (log2f 1 ulp, the constant and the product half each), less than a slot more or
    less would change it. Steps: x up to 6, off by 2^-20 (the scale's roundings, 6 * 2^-23), exp2f 2^-22, and sums of at most 2^9 terms
    after one another (units of a warp, warps, CTAs), 2^-15: less than 2^-14 together."""
    cache = make(lens, H, D, page, seed=90)
    k, v = cache._keep[:2]
    places = held(cache, lens)
    q = torch.zeros(len(lens), hq * D, dtype=BF16, device=DEV)
    level = []
    for (at, row), n in zip(places, lens):
        unit = torch.arange(n, device=DEV) // 16
        e = torch.where(unit // 5 % 2 == 0, unit // 3 % 7, 6 - unit % 7) if steps else 0 * unit
        level.append(e.double())
        k[at, :, row] = 0
        k[at, :, row, 0] = e.to(BF16)[:, None]
        v[at, :, row] = 0
    q.view(-1, hq, D)[:, :, 0] = 1
    total = [float((2.0 ** e).sum()) for e in level]
    lse_far = 2.0 ** -14 if steps else 0.0
    far = 2.0 ** -8 + (2.0 ** -14 if steps else 2.0 ** -23)
    ws, empty = workspace(cache, hq), v.clone()
    for turn in range((max(lens) + 16 * D - 1) // (16 * D)):  # D units of every sequence at a time
        want = torch.zeros(len(lens), D, dtype=torch.double, device=DEV)
        v.copy_(empty)
        for s, ((at, row), n) in enumerate(zip(places, lens)):
            unit = torch.arange((n + 15) // 16, device=DEV)[turn * D:(turn + 1) * D]
            slot = (unit * 16 + (unit * 7 + turn) % 16).clamp(max=n - 1)
            v[at[slot], :, row[slot], unit - turn * D] = 1
            want[s, unit - turn * D] = 2.0 ** level[s][slot] / max(total[s], 1.0)
        out, lse = attend(cache, q, hq, scale=math.log(2.0), ws=ws)
        off = (out.double().view(-1, hq, D) - want[:, None]).abs()
        assert bool((off <= want[:, None] * far).all()), float((off / want[:, None]).nan_to_num().max())
        for s, t in enumerate(total):
            if lens[s] == 0:
                assert bool((lse[s] == -math.inf).all())
            else:
                assert bool(((lse[s].double() - math.log(t)).abs() <= math.log(t) * 2.0 ** -22 + lse_far).all())


@pytest.mark.parametrize("lens,hq,H,D,page", [b for b in BORDERS if max(b[0]) < 10000])
def test_every_slot_has_its_weight(lens, hq, H, D, page):
    """Equal keys: each slot of a sequence gets 1 / n (off by 2^-24) from every query head of the group, whose sum is off by
    2^-24 a head."""
    cache = make(lens, H, D, page, seed=91, weights=True)
    mass = cache._keep[4].zero_()
    q = torch.zeros(len(lens), hq * D, dtype=BF16, device=DEV)
    attend(cache, q, hq, weights=True)
    for s, n in enumerate(lens):
        want = hq // H / max(n, 1)
        assert bool(((mass[s, :, :n].double() - want).abs() <= want * (hq // H + 2) * 2.0 ** -24).all())
        assert bool((mass[s, :, n:] == 0).all())


@pytest.mark.parametrize("S", [129, 300, 1024, 1500])
def test_append_to_many_sequences(S):
    """Sequences without new tokens at the beginning, in runs and at the end; rows of padding behind the last token."""
    H, D, page, pad = 1, 64, 8, 7
    new = [0 if i < 9 or i >= S - 11 or i // 6 % 3 == 1 else 1 + i % 3 for i in range(S)]
    past = [i * 5 % 14 for i in range(S)]
    T = sum(new)
    cache = make([a + b for a, b in zip(past, new)], H, D, page, seed=93, extra=0, weights=True, fill=0.25)
    k, v, table, length, mass, pos = cache._keep
    nk, nv, q = (torch.randn(T + pad, n * D, device=DEV, generator=gen(94 + n)).to(BF16) for n in (H, H, 2 * H))
    starts = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).int().to(DEV)
    position = torch.arange(T + pad, dtype=torch.int32, device=DEV) + 100
    want = [x.clone() for x in (k, v, mass, pos)]
    seq = torch.repeat_interleave(torch.arange(S), torch.tensor(new)).to(DEV)
    t = torch.arange(T, device=DEV)
    slot = torch.tensor(past, device=DEV)[seq] + t - starts.long()[seq]
    at = table.long()[seq, slot // page]
    want[0][at, :, slot % page] = nk[:T].view(T, H, D)
    want[1][at, :, slot % page] = nv[:T].view(T, H, D)
    want[2][seq, :, slot] = 0
    want[3][seq, :, slot] = position[:T, None]
    q_out = torch.full_like(q, 9.0)
    B.ordermoe_cache_append(cache, nk, nv, q=q, q_out=q_out, starts=starts, position=position)
    for got, w in zip((k, v, mass, pos), want):
        assert torch.equal(got, w)
    assert torch.equal(q_out[:T], q[:T]) and bool((q_out[T:] == 9.0).all())


def test_append_and_cut_on_another_stream():
    H, D, budget = 2, 64, 40
    nk, nv = (torch.randn(3, H * D, device=DEV, generator=gen(95 + i)).to(BF16) for i in range(2))
    results = []
    for s in (None, torch.cuda.Stream()):
        cache = make([90, 17, 41], H, D, 16, seed=97, weights=True, fill=0.5)
        out = torch.zeros_like(cache._keep[3])
        ws = torch.empty(B.ordermoe_cache_evict_workspace_bytes(cache, budget), dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        B.ordermoe_cache_append(cache, nk, nv, stream=s)
        B.ordermoe_cache_evict(cache, budget, out, ws, stream=s)
        torch.cuda.synchronize()
        results.append([x.clone() for x in cache._keep] + [out])
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert results[0][-1].tolist() == [40, 17, 40]


def test_a_capture_that_raises_leaves_the_caches_as_they_are():
    S, slots = 3, 16
    caches, stack, hs, xs = attention_stack(S, slots, 102)
    home = torch.zeros(S, dtype=torch.uint8, device=DEV)
    for i in range(4):
        hs[0].copy_(torch.randn(S, 256, device=DEV, generator=gen(150 + i)).to(BF16))
        caches[0].advance()
        stack.step_residual(hs, xs, home, None, None)
    before = state(caches)

    def prologue():
        caches[0].advance()
        raise KeyError("no such request")

    with pytest.raises(KeyError):
        stack.capture_residual(hs, xs, home, None, None, prologue=prologue)
    for a, b in zip(state(caches), before):
        assert torch.equal(a, b)
    wrong = [torch.zeros(S + 1, 256, dtype=BF16, device=DEV) for _ in range(4)]  # refused within the step
    with pytest.raises(ValueError):
        stack.capture_residual(wrong, [w.clone() for w in wrong], home, None, None, prologue=caches[0].advance)
    for a, b in zip(state(caches), before):
        assert torch.equal(a, b)
