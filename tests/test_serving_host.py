"""What needs no GPU of the paged cache, the attention over it and the adapters: refusals before
anything is enqueued (addresses that are passed are not read) and sizes of the workspaces."""
import ctypes

import pytest
import torch

from paper_2607_17154_gb300 import binding as B

OK, ARG, SHAPE = B.OK, B.ERR_INVALID_ARG, B.ERR_UNSUPPORTED_SHAPE
AT = 1 << 20  # an aligned address that a refused call never reads
N = None


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_2607_17154_gb300 import build
    build.build()


def cache(**over):
    v = dict(k=AT, v=AT, pages=100, page=16, heads=2, dim=64, seqs=3, seq_pages=4, table=AT, ld_table=4, length=AT, mass=AT, pos=AT)
    v.update(over)
    return B.Cache(**v)


def run(name, *args):
    rc = getattr(B.lib(), name)(*args)
    return rc, B.lib().ordermoe_last_error().decode()


def append(c=N, k=AT, ldk=128, v=AT, ldv=128, q=AT, ldq=256, qo=AT, ldqo=256, T=3, hq=4, starts=N, position=N, freq=AT, rot=64):
    c = cache() if c is N else c
    return run("ordermoe_cache_append", ctypes.byref(c), k, ldk, v, ldv, q, ldq, qo, ldqo, T, hq, starts, position, freq, rot, 0, N)


def attend(c=N, q=AT, ldq=256, hq=4, scale=0.1, out=AT, ldo=256, lse=AT, weights=0, ws=AT, nbytes=1 << 40):
    c = cache() if c is N else c
    return run("ordermoe_attention_paged", ctypes.byref(c), q, ldq, hq, scale, out, ldo, lse, weights, ws, nbytes, N)


def evict(c=N, budget=8, sinks=1, recent=2, newest=AT, out=AT * 2, ws=AT, nbytes=1 << 40):
    c = cache() if c is N else c
    return run("ordermoe_cache_evict", ctypes.byref(c), budget, sinks, recent, newest, out, ws, nbytes, N)


CALLS = [(append, "cache_append:"), (attend, "attention_paged:"), (evict, "cache_evict:")]


@pytest.mark.parametrize("call,prefix", CALLS, ids=[p for _, p in CALLS])
@pytest.mark.parametrize("over,code", [
    (dict(seqs=-1), ARG), (dict(pages=-1), ARG), (dict(seq_pages=0), ARG), (dict(ld_table=3), ARG), (dict(dim=96), SHAPE),
    (dict(dim=0), SHAPE), (dict(page=0), SHAPE), (dict(page=12), SHAPE), (dict(page=2048), SHAPE), (dict(heads=0), SHAPE),
    (dict(heads=1025), SHAPE), (dict(seqs=65536), SHAPE), (dict(pages=1 << 31), SHAPE), (dict(seq_pages=(1 << 26) + 1, ld_table=1 << 27), SHAPE),
    (dict(k=N), ARG), (dict(v=N), ARG), (dict(table=N), ARG), (dict(length=N), ARG), (dict(k=AT + 8), ARG), (dict(v=AT + 2), ARG),
    (dict(table=AT + 2), ARG), (dict(length=AT + 1), ARG), (dict(mass=AT + 2), ARG), (dict(pos=AT + 2), ARG)])
def test_caches_that_are_refused(call, prefix, over, code):
    rc, msg = call(cache(**over))
    assert rc == code and msg.startswith(prefix), (rc, msg)


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), ARG), (dict(T=2), ARG), (dict(q=N), ARG), (dict(qo=N), ARG), (dict(hq=0), SHAPE), (dict(hq=5000), SHAPE),
    (dict(rot=-16), SHAPE), (dict(rot=80), SHAPE), (dict(rot=24), SHAPE), (dict(freq=N), ARG), (dict(k=N), ARG), (dict(v=N), ARG),
    (dict(k=AT + 8), ARG), (dict(v=AT + 2), ARG), (dict(q=AT + 8), ARG), (dict(qo=AT + 8), ARG), (dict(ldk=120), ARG), (dict(ldv=132), ARG),
    (dict(ldq=248), ARG), (dict(ldqo=260), ARG), (dict(ldqo=264), ARG), (dict(ldk=1 << 38), ARG), (dict(starts=AT + 2), ARG),
    (dict(position=AT + 1), ARG), (dict(freq=AT + 4), ARG)])
def test_calls_that_append_refuses(over, code):
    rc, msg = append(**over)
    assert rc == code and msg.startswith("cache_append:"), (rc, msg)


@pytest.mark.parametrize("over,code", [
    (dict(hq=3), SHAPE), (dict(hq=0), SHAPE), (dict(hq=4098), SHAPE), (dict(scale=0.0), ARG), (dict(scale=-1.0), ARG),
    (dict(scale=float("nan")), ARG), (dict(scale=float("inf")), ARG), (dict(q=N), ARG), (dict(out=N), ARG), (dict(q=AT + 8), ARG),
    (dict(out=AT + 2), ARG), (dict(lse=AT + 2), ARG), (dict(ldq=248), ARG), (dict(ldo=257), ARG), (dict(ldo=264), ARG), (dict(ws=N), ARG),
    (dict(ws=AT + 128), ARG), (dict(nbytes=1000), ARG), (dict(c=cache(mass=N), weights=1), ARG)])
def test_calls_that_attention_refuses(over, code):
    rc, msg = attend(**over)
    assert rc == code and msg.startswith("attention_paged:"), (rc, msg)


@pytest.mark.parametrize("over,code", [
    (dict(budget=0), ARG), (dict(sinks=-1), ARG), (dict(recent=-1), ARG), (dict(sinks=5, recent=4), ARG), (dict(budget=(1 << 30) + 1), SHAPE),
    (dict(c=cache(mass=N)), ARG), (dict(out=N), ARG), (dict(out=AT), ARG), (dict(newest=N), ARG), (dict(newest=AT + 2), ARG),
    (dict(out=AT + 2), ARG), (dict(ws=N), ARG), (dict(ws=AT + 16), ARG), (dict(nbytes=100), ARG)])
def test_calls_that_evict_refuses(over, code):
    rc, msg = evict(**over)
    assert rc == code and msg.startswith("cache_evict:"), (rc, msg)


def test_null_cache_and_nothing_to_do():
    for name, args in (("ordermoe_cache_append", [N] * 1 + [N, 0, N, 0, N, 0, N, 0, 0, 0, N, N, N, 0, 0, N]),
                       ("ordermoe_attention_paged", [N, N, 0, 4, 0.1, N, 0, N, 0, N, 0, N]),
                       ("ordermoe_cache_evict", [N, 8, 0, 0, N, N, N, 0, N])):
        assert run(name, *args)[0] == ARG
    none = cache(seqs=0, k=N, v=N, table=N, length=N, mass=N, pos=N)
    assert append(none, T=0)[0] == OK and append(none, T=1)[0] == ARG
    assert attend(none, q=N, out=N, ws=N, nbytes=0)[0] == OK
    assert evict(none, out=N, ws=N, nbytes=0)[0] == OK
    assert append(T=0, starts=AT)[0] == OK


GOOD = dict(X=AT, ldx=128, A=AT, sa=128 * 16, lda=128, Bw=AT, sb=64 * 16, ldb=16, ids=AT, rank=AT, scale=AT, n=4, R=16, res=AT, ldr=64,
            T=8, N=64, K=128, Y=AT * 2, ldy=64, f32=0, ws=AT, nbytes=1 << 40, stream=N)


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), ARG), (dict(N=0), ARG), (dict(K=0), ARG), (dict(n=0), ARG), (dict(R=0), SHAPE), (dict(R=12), SHAPE), (dict(R=136), SHAPE),
    (dict(K=(1 << 30) + 1, ldx=1 << 31, lda=1 << 31), SHAPE), (dict(N=2 ** 31 - 1, ldy=1 << 31, ldr=1 << 31), SHAPE), (dict(T=2 ** 31 - 1), SHAPE),
    (dict(ldx=120), ARG), (dict(lda=120), ARG), (dict(ldb=8), ARG), (dict(ldy=63), ARG), (dict(ldr=63), ARG), (dict(sa=-8), ARG), (dict(sb=-8), ARG),
    (dict(ldx=132), SHAPE), (dict(lda=132), SHAPE), (dict(ldb=20), SHAPE), (dict(sa=4), SHAPE), (dict(sb=12), SHAPE), (dict(ldx=1 << 38), SHAPE),
    (dict(X=N), ARG), (dict(A=N), ARG), (dict(Bw=N), ARG), (dict(ids=N), ARG), (dict(Y=N), ARG), (dict(X=AT + 8), ARG), (dict(A=AT + 8), ARG),
    (dict(Bw=AT + 8), ARG), (dict(Y=AT + 1), ARG), (dict(Y=AT + 2, f32=1), ARG), (dict(res=AT + 1), ARG), (dict(ids=AT + 2), ARG),
    (dict(rank=AT + 2), ARG), (dict(scale=AT + 2), ARG), (dict(res=AT * 2, ldr=72), ARG), (dict(res=AT * 2, f32=1), ARG), (dict(ws=N), ARG),
    (dict(ws=AT + 16), ARG), (dict(nbytes=16), ARG)])
def test_calls_that_adapters_refuses(over, code):
    rc, msg = run("ordermoe_adapters", *dict(GOOD, **over).values())
    assert rc == code and msg.startswith("adapters:"), (over, rc, msg)


def test_no_tokens_need_nothing():
    assert run("ordermoe_adapters", *dict(GOOD, T=0, X=N, Y=N, ws=N, nbytes=0).values())[0] == OK


def test_sizes_of_workspaces():
    L = B.lib()
    f = L.ordermoe_attention_paged_workspace_bytes
    assert f(4, 8, 3, 64, 100, 0) == 0 and f(4, 8, 4, 96, 100, 0) == 0 and f(4, 8, 4, 64, 0, 0) == 0
    plain, kept = f(4, 8, 4, 64, 1000, 0), f(4, 8, 4, 64, 1000, 1)
    assert 0 < plain and kept >= plain + 4 * 8 * 1000 * 4  # a score a query head and slot at least
    assert f(0, 8, 4, 64, 100, 1) > 0
    e = L.ordermoe_cache_evict_workspace_bytes
    assert e(4, 2, 100) >= 4 * 2 * (2 * 100 + 1) * 4 and e(4, 0, 100) == 0 and e(4, 2, 0) == 0
    a = L.ordermoe_adapters_workspace_bytes
    assert a(10, 4096, 4096, 16) >= 10 * 16 * 4 and a(0, 64, 64, 8) == 0 and a(10, 64, 64, 12) == 0


def test_the_binding_refuses_other_tensors():
    k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    table, length = torch.zeros(3, 1, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        B.make_cache(k, k.clone(), table, length)
    with pytest.raises(ValueError):
        B.make_cache(k, k[:2], table, length)
    with pytest.raises(TypeError):
        B.make_cache(k.float(), k.float(), table, length)


def test_a_budget_above_the_slots_asks_for_the_slots_workspace():
    c = cache()
    slots = c.seq_pages * c.page
    need = B.lib().ordermoe_cache_evict_workspace_bytes(c.seqs, c.heads, slots)
    for budget in (slots, slots + 1, 1 << 30):
        rc, msg = evict(c, budget=budget, nbytes=need - 1)
        assert rc == ARG and "workspace" in msg


@pytest.mark.parametrize("at", [AT, AT + 4, AT + 8, AT - 8])
def test_evict_refuses_new_lengths_over_what_it_reads(at):
    """Three sequences: any of the twelve bytes of length, or of newest."""
    far = AT * 4
    for over in (dict(newest=far), dict(c=cache(length=far))):
        rc, msg = evict(out=at, **over)
        assert rc == ARG and "overlap" in msg, (over, rc, msg)
