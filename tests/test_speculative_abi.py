"""Refusals of the operators of speculative rollouts and distillation: every bad argument is turned down on the host, before a
launch (no GPU needed)."""
import pytest

from test_abi import E_ALIGN, E_ARG, E_NULL, E_SIZE, E_WS, ODD, OK, L, P, _FakeTensor  # noqa: F401

NAN, INF = float("nan"), float("inf")


def _attend(L, q=P, qs=512, k=P, v=P, pages=9, ps=4096, ts=256, hs=64, bt=P, w=4, off=P, ln=P, out=P, lse=P, T=6, B=2, H=8, Hk=4, d=64, page=16,
            mn=6, ml=64, scale=0.1, ws=P, wsb=1 << 30):
    return L.rlcs_chunk_attention_bf16(q, qs, k, v, pages, ps, ts, hs, bt, w, off, ln, out, lse, T, B, H, Hk, d, page, mn, ml, scale, ws, wsb, None)


def test_chunk_attention_refusals(L):
    f = lambda **k: _attend(L, **k)
    assert f(T=0) == OK and f(H=0, Hk=0, qs=0) == OK and f(B=0) == OK and f(mn=0) == OK
    for bad in (dict(T=-1), dict(B=-1), dict(H=-8), dict(Hk=3), dict(Hk=0), dict(d=4), dict(d=60), dict(d=136), dict(page=0), dict(page=32769),
                dict(mn=-1), dict(ml=-1), dict(ml=2 ** 31), dict(pages=-1), dict(pages=2 ** 31), dict(w=-1), dict(qs=511), dict(ps=-8), dict(ts=-8),
                dict(hs=-8), dict(B=2 ** 21), dict(T=2 ** 25), dict(H=8192, Hk=1, qs=2 ** 20)):
        assert f(**bad) == E_SIZE, bad
    for v in (0.0, -1.0, NAN, INF):
        assert f(scale=v) == E_ARG
    for name in ("q", "k", "v", "bt", "off", "ln", "out"):
        assert f(**{name: None}) == E_NULL, name
    for name in ("bt", "off", "ln", "lse"):
        assert f(**{name: ODD}) == E_ALIGN, name
    for name in ("q", "k", "v", "out", "ws"):
        assert f(**{name: P + 8}) == E_ALIGN, name
    for name in ("qs", "ps", "ts", "hs"):
        assert f(**{name: 516}) == E_ALIGN, name
    sizes = (6, 2, 8, 4, 64, 16, 6, 64)
    need = L.rlcs_chunk_attention_workspace_bytes(*sizes)
    if need:
        assert f(wsb=need - 1) == E_WS and f(ws=None) == E_WS
    for other in ((0, 2, 8, 4, 64, 16, 6, 64), (6, 2, 8, 3, 64, 16, 6, 64), (6, 0, 8, 4, 64, 16, 6, 64), (6, 2, 8, 4, 64, 16, 0, 64)):
        assert L.rlcs_chunk_attention_workspace_bytes(*other) == 0


def test_chunk_attention_workspace_of_a_long_context(L):
    need = L.rlcs_chunk_attention_workspace_bytes(4, 1, 32, 8, 128, 64, 4, 32768)
    assert need > 0
    assert _attend(L, T=4, B=1, H=32, Hk=8, d=128, qs=4096, page=64, mn=4, ml=32768, wsb=need - 1) == E_WS


def _verify(L, x=P, ld=8, y=P, ldd=8, tok=P, off=P, u=P, du=P, t=None, ta=1.0, out=P, lp=P, acc=P, T=6, B=2, A=8, ws=P, wsb=1 << 20, bf16=False):
    fn = L.rlcs_verify_drafts_bf16 if bf16 else L.rlcs_verify_drafts
    return fn(x, ld, y, ldd, tok, off, u, du, t, ta, out, lp, acc, T, B, A, ws, wsb, None)


@pytest.mark.parametrize("bf16", [False, True])
def test_verify_refusals(L, bf16):
    f = lambda **k: _verify(L, bf16=bf16, **k)
    assert f(B=0) == OK and f(B=0, off=None) == OK
    for bad in (dict(T=-1), dict(B=-1), dict(A=-1), dict(A=0), dict(ld=7), dict(ldd=7), dict(A=2 ** 22 + 1, ld=2 ** 23, ldd=2 ** 23), dict(T=2 ** 25),
                dict(B=2 ** 25), dict(T=2 ** 24, ld=2 ** 20)):
        assert f(**bad) == E_SIZE, bad
    for name in ("x", "tok", "off", "u", "du", "out", "lp", "acc"):
        assert f(**{name: None}) == E_NULL, name
    for name in ("tok", "off", "u", "du", "t", "out", "lp", "acc"):
        assert f(**{name: ODD}) == E_ALIGN, name
    assert f(x=P + 1) == E_ALIGN and f(y=P + 1) == E_ALIGN and f(ws=P + 8) == E_ALIGN
    assert f(ta=NAN) == E_ARG
    need = L.rlcs_verify_drafts_workspace_bytes(6, 2)
    assert need > 0 and f(wsb=need - 1) == E_WS and f(ws=None) == E_WS
    assert L.rlcs_verify_drafts_workspace_bytes(0, 2) == 0 and L.rlcs_verify_drafts_workspace_bytes(6, 0) == 0


def _distill(L, x=P, ld=8, ids=P, t=P, mask=None, loss=P, dx=P, ldd=8, R=4, A=8, K=3, T=1.0, s=1.0, bf16=False):
    fn = L.rlcs_distill_grad_bf16 if bf16 else L.rlcs_distill_grad
    return fn(x, ld, ids, t, mask, loss, dx, ldd, R, A, K, T, s, None)


@pytest.mark.parametrize("bf16", [False, True])
def test_distill_refusals(L, bf16):
    f = lambda **k: _distill(L, bf16=bf16, **k)
    assert f(R=0) == OK
    for bad in (dict(R=-1), dict(A=0), dict(A=-1), dict(K=-1), dict(K=1025), dict(ld=7), dict(ldd=7), dict(A=2 ** 22 + 1, ld=2 ** 23, ldd=2 ** 23),
                dict(R=2 ** 30, ld=2 ** 12)):
        assert f(**bad) == E_SIZE, bad
    for v in (0.0, -1.0, NAN, INF, 1e-45):
        assert f(T=v) == E_ARG
    assert f(s=NAN) == E_ARG and f(s=INF) == E_ARG
    for name in ("x", "ids", "t"):
        assert f(**{name: None}) == E_NULL, name
    assert f(loss=None, dx=None) == E_NULL
    for name in ("ids", "t", "loss"):
        assert f(**{name: ODD}) == E_ALIGN, name
    assert f(x=P + 1) == E_ALIGN and f(dx=P + 1) == E_ALIGN


def _fork(L, t=P, ln=P, src=P, fr=P, new=P, a=P, b=P, used=P, B=4, N=5, w=8, F=9, page=16, ws=None, wsb=0):
    return L.rlcs_fork_block_tables(t, ln, src, fr, new, a, b, used, B, N, w, F, page, ws, wsb, None)


def test_fork_refusals(L):
    f = lambda **k: _fork(L, **k)
    for bad in (dict(B=-1), dict(N=-1), dict(w=-1), dict(F=-1), dict(page=-1), dict(B=2 ** 24), dict(N=2 ** 24), dict(F=2 ** 31), dict(page=2 ** 25)):
        assert f(**bad) == E_SIZE, bad
    assert f(page=0) == E_ARG
    for name in ("t", "ln", "src", "fr", "new", "a", "b", "used"):
        assert f(**{name: None}) == E_NULL, name
        assert f(**{name: ODD}) == E_ALIGN, name
    assert L.rlcs_fork_block_tables_workspace_bytes(4096, 4096) == 0
    need = L.rlcs_fork_block_tables_workspace_bytes(5000, 5)
    assert need > 0 and f(B=5000) == E_WS and f(B=5000, ws=P, wsb=need - 1) == E_WS and f(B=5000, ws=P + 8, wsb=need) == E_ALIGN


def _copy(L, k=P, v=P, pages=9, ps=4096, ts=256, hs=64, a=P, b=P, N=4, page=16, Hk=4, d=64):
    return L.rlcs_copy_pages_bf16(k, v, pages, ps, ts, hs, a, b, N, page, Hk, d, None)


def test_copy_refusals(L):
    f = lambda **k: _copy(L, **k)
    assert f(N=0) == OK and f(pages=0) == OK and f(d=0) == OK
    for bad in (dict(N=-1), dict(pages=-1), dict(page=-1), dict(Hk=-1), dict(d=-8), dict(d=60), dict(ps=-8), dict(ts=-8), dict(hs=-8),
                dict(pages=2 ** 31), dict(N=2 ** 31)):
        assert f(**bad) == E_SIZE, bad
    for name in ("k", "a", "b"):
        assert f(**{name: None}) == E_NULL, name
    for name, bad in (("k", P + 8), ("v", P + 8), ("a", ODD), ("b", ODD), ("ps", 516), ("ts", 4), ("hs", 4)):
        assert f(**{name: bad}) == E_ALIGN, name


def _free(L, t=P, ln=P, pt=P, pl=P, out=P, n=P, B=4, w=8, G=2, pw=3, pages=100, page=16, ws=P, wsb=1 << 20):
    return L.rlcs_free_pages(t, ln, pt, pl, out, n, B, w, G, pw, pages, page, ws, wsb, None)


def test_free_refusals(L):
    f = lambda **k: _free(L, **k)
    for bad in (dict(B=-1), dict(w=-1), dict(G=-1), dict(pw=-1), dict(pages=-1), dict(page=-1), dict(B=2 ** 24), dict(G=2 ** 24), dict(pages=2 ** 31),
                dict(page=2 ** 25)):
        assert f(**bad) == E_SIZE, bad
    assert f(page=0) == E_ARG
    for name in ("t", "ln", "pt", "pl", "out", "n"):
        assert f(**{name: None}) == E_NULL, name
        assert f(**{name: ODD}) == E_ALIGN, name
    need = L.rlcs_free_pages_workspace_bytes(100)
    assert need > 0 and f(wsb=need - 1) == E_WS and f(ws=None) == E_WS and f(ws=P + 8) == E_ALIGN
    assert L.rlcs_free_pages_workspace_bytes(0) == 0 and L.rlcs_free_pages_workspace_bytes(-1) == 0


def test_binding_checks():
    import torch
    from paper_2608_17641_b200 import api, binding
    binding.lib()
    i = torch.zeros(2, dtype=torch.int32)
    x, q = torch.zeros(2, 8), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    cache = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    for call in (lambda: api.chunk_attention(q, cache, cache, i.view(1, 2), i, i[:1]), lambda: api.verify_drafts(x, i, i, x[:, 0], x[:1, 0]),
                 lambda: api.compute_distillation(x, i.view(2, 1), x[:, :1]), lambda: api.copy_pages(cache, cache, i, i),
                 lambda: api.fork_block_tables(i.view(1, 2), i[:1], i, i, page_size=4), lambda: api.list_free_pages(i.view(1, 2), i[:1], num_pages=4, page_size=4)):
        with pytest.raises(TypeError):
            call()                                            # CUDA tensors only
    with pytest.raises(TypeError):
        api.verify_drafts(x.double(), i, i, x[:, 0], x[:1, 0])
    with pytest.raises(ValueError):
        api.chunk_attention(q[0], cache, cache, i.view(1, 2), i, i[:1])
    with pytest.raises(ValueError):
        api.list_free_pages(i.view(1, 2), i[:1], num_pages=4, page_size=4, prefix_table=i.view(1, 2))
