"""Refusals of the rollout and policy operators: every bad argument is turned down on the host, before a launch (no GPU needed)."""
import pytest

from test_abi import E_ALIGN, E_ARG, E_NULL, E_SIZE, E_WS, ODD, OK, L, P, _FakeTensor  # noqa: F401

NAN, INF = float("nan"), float("inf")


def _sample(L, x=P, ld=8, u=P, t=None, k=None, p=None, m=None, ta=1.0, ka=0, pa=1.0, ma=0.0, a=P, lp=P, kp=P, R=4, A=8, bf16=False):
    fn = L.rlcs_sample_actions_bf16 if bf16 else L.rlcs_sample_actions
    return fn(x, ld, u, t, k, p, m, ta, ka, pa, ma, a, lp, kp, R, A, None)


@pytest.mark.parametrize("bf16", [False, True])
def test_sample_refusals(L, bf16):
    f = lambda **k: _sample(L, bf16=bf16, **k)
    assert f(R=0) == OK and f(R=0, x=None) == OK
    assert f(R=-1) == E_SIZE and f(A=0) == E_SIZE and f(A=-1) == E_SIZE and f(ld=7) == E_SIZE
    assert f(A=2 ** 22 + 1, ld=2 ** 23) == E_SIZE and f(R=2 ** 30, ld=2 ** 12) == E_SIZE
    for name in ("x", "u", "a", "lp", "kp"):
        assert f(**{name: None}) == E_NULL
    assert f(ta=NAN) == E_ARG and f(pa=NAN) == E_ARG and f(ma=NAN) == E_ARG
    for name in ("u", "t", "k", "p", "m", "a", "lp", "kp"):
        assert f(**{name: ODD}) == E_ALIGN
    assert f(x=P + 1) == E_ALIGN


def _policy(L, x=P, ld=8, a=P, mask=None, adv=P, old=None, loss=P, lp=P, h=P, dx=P, ldd=8, R=4, A=8, T=1.0, clip=0.2, c=0.0, s=1.0, bf16=False):
    fn = L.rlcs_policy_grad_bf16 if bf16 else L.rlcs_policy_grad
    return fn(x, ld, a, mask, adv, old, loss, lp, h, dx, ldd, R, A, T, clip, c, s, None)


@pytest.mark.parametrize("bf16", [False, True])
def test_policy_refusals(L, bf16):
    f = lambda **k: _policy(L, bf16=bf16, **k)
    assert f(R=0) == OK
    assert f(R=-1) == E_SIZE and f(A=0) == E_SIZE and f(ld=7) == E_SIZE and f(ldd=7) == E_SIZE and f(A=2 ** 22 + 1, ld=2 ** 23, ldd=2 ** 23) == E_SIZE
    assert f(R=2 ** 30, ld=2 ** 12) == E_SIZE
    for v in (0.0, -1.0, NAN, INF, 1e-45):
        assert f(T=v) == E_ARG
    assert f(clip=-0.1) == E_ARG and f(clip=NAN) == E_ARG and f(c=NAN) == E_ARG and f(s=INF) == E_ARG
    for name in ("x", "a", "lp", "h", "adv"):
        assert f(**{name: None}) == E_NULL
    assert f(adv=None, loss=None, dx=None, old=P) == E_NULL
    for name in ("a", "adv", "old", "loss", "lp", "h"):
        assert f(**{name: ODD}) == E_ALIGN
    assert f(x=P + 1) == E_ALIGN and f(dx=P + 1) == E_ALIGN


def _attend(L, q=P, qs=512, k=P, v=P, pages=9, ps=4096, ts=256, hs=64, pt=P, pw=4, pl=P, go=P, bt=P, ow=4, ln=P, out=P, lse=P, B=2, H=8, Hk=4,
            d=64, page=16, G=1, mp=64, ml=64, scale=0.1, ws=P, wsb=1 << 30):
    return L.rlcs_prefix_attention_bf16(q, qs, k, v, pages, ps, ts, hs, pt, pw, pl, go, bt, ow, ln, out, lse, B, H, Hk, d, page, G, mp, ml,
                                        scale, ws, wsb, None)


def test_attention_refusals(L):
    f = lambda **k: _attend(L, **k)
    assert f(B=0) == OK and f(H=0, Hk=0, qs=0) == OK
    for bad in (dict(B=-1), dict(H=-8), dict(Hk=3), dict(Hk=0), dict(d=4), dict(d=60), dict(d=136), dict(page=0), dict(page=32769), dict(G=-1),
                dict(mp=-1), dict(ml=-1), dict(ml=2 ** 31), dict(pages=-1), dict(pages=2 ** 31), dict(pw=-1), dict(ow=-1), dict(qs=511),
                dict(ps=-8), dict(B=2 ** 21)):
        assert f(**bad) == E_SIZE, bad
    for v in (0.0, -1.0, NAN, INF):
        assert f(scale=v) == E_ARG
    for name in ("q", "k", "v", "pt", "pl", "go", "bt", "ln", "out"):
        assert f(**{name: None}) == E_NULL, name
    for name in ("pt", "pl", "go", "bt", "ln", "lse"):
        assert f(**{name: ODD}) == E_ALIGN, name
    for name in ("q", "k", "v", "out", "ws"):
        assert f(**{name: P + 8}) == E_ALIGN, name
    for name in ("qs", "ps", "ts", "hs"):
        assert f(**{name: 516}) == E_ALIGN, name
    need = L.rlcs_prefix_attention_workspace_bytes(2, 8, 4, 64, 16, 1, 64, 64)
    assert need > 0 and f(wsb=need - 1) == E_WS and f(ws=None) == E_WS
    assert L.rlcs_prefix_attention_workspace_bytes(0, 8, 4, 64, 16, 1, 64, 64) == 0
    assert L.rlcs_prefix_attention_workspace_bytes(2, 8, 3, 64, 16, 1, 64, 64) == 0


def _tables(L, c=P, a=P, f=P, t=P, s=P, p=P, o=P, po=P, B=4, w=8, F=9, n=5, page=16):
    return L.rlcs_block_tables(c, a, f, t, s, p, o, po, B, w, F, n, page, None)


def test_tables_refusals(L):
    f = lambda **k: _tables(L, **k)
    for bad in (dict(B=-1), dict(w=-1), dict(F=-1), dict(n=-1), dict(page=-1), dict(B=2 ** 24), dict(F=2 ** 31), dict(n=2 ** 31), dict(page=2 ** 25)):
        assert f(**bad) == E_SIZE, bad
    assert f(page=0) == E_ARG
    for name in ("c", "a", "f", "t", "s", "p", "o", "po"):
        assert f(**{name: None}) == E_NULL, name
        assert f(**{name: ODD}) == E_ALIGN, name
    assert f(s=P + 4) == E_ALIGN


def test_binding_checks(monkeypatch):
    import torch
    from paper_2608_17641_b200 import api, binding
    binding.lib()
    x, a = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: api.sample_actions(x, torch.zeros(2)), lambda: api.compute_policy_gradient(x, a, torch.zeros(2)),
                 lambda: api.build_block_tables(a, a, a, a.view(1, 2), page_size=4, num_slots=2)):
        with pytest.raises(TypeError):
            call()                                            # CUDA tensors only
    with pytest.raises(TypeError):
        api.sample_actions(x.double(), torch.zeros(2))
    monkeypatch.setattr(binding, "_current_device", lambda: 0)

    class Rows(_FakeTensor):
        def __init__(self, dtype, shape, strides):
            super().__init__(0, dtype, shape)
            self._s = strides

        def dim(self):
            return len(self.shape)

        def stride(self, i=None):
            return self._s if i is None else self._s[i]

    assert binding._rows(Rows(torch.float32, (2, 8), (11, 1)), "f32", "logits", 0)[1] == 11
    assert binding._rows(Rows(torch.float32, (1, 8), (0, 1)), "f32", "logits", 0)[1] == 8
    for strides in ((8, 2), (7, 1), (0, 1)):
        with pytest.raises(ValueError):
            binding._rows(Rows(torch.float32, (2, 8), strides), "f32", "logits", 0)
    with pytest.raises(TypeError):
        binding._rows(Rows(torch.bfloat16, (2, 8), (8, 1)), "f32", "logits", 0)
    with pytest.raises(ValueError):
        binding._rows(Rows(torch.float32, (2, 8), (8, 1)), "f32", "dlogits", 0, (2, 9))
    with pytest.raises(ValueError):
        binding._typed(_FakeTensor(0, torch.int32, (3,)), "i32", (2,), "actions", 0)
    with pytest.raises(TypeError):
        binding._typed(_FakeTensor(0, torch.int64, (2,)), "i32", (2,), "actions", 0)


class _FakeLibrary:
    """The C library's functions by name, type and kind of result; none of them does anything."""

    def __getattr__(self, name):
        from paper_2608_17641_b200 import binding
        argtypes, restype = binding.SIGNATURES[name]

        def call(*args):
            return 4096 if restype is binding._sz else OK
        call.argtypes, call.restype, call.__name__ = argtypes, restype, name
        return call


class _Rows(_FakeTensor):
    """A contiguous stand-in for a CUDA tensor of any shape."""

    def dim(self):
        return len(self.shape)

    def stride(self, i=None):
        steps = [1]
        for n in self.shape[:0:-1]:
            steps.insert(0, steps[0] * n)
        return tuple(steps) if i is None else steps[i]

    def numel(self):
        n = 1
        for d in self.shape:
            n *= d
        return n

    def element_size(self):
        return self.dtype.itemsize

    def record_stream(self, stream):
        pass


def _attention_args():
    import torch
    t = lambda dtype, *shape: _Rows(0, dtype, shape)
    i32, bf16 = torch.int32, torch.bfloat16
    cache = t(bf16, 9, 16, 2, 64)
    return (t(bf16, 4, 8, 64), cache, cache, t(i32, 1, 4), t(i32, 1), t(i32, 2), t(i32, 4, 4), t(i32, 4))


@pytest.mark.parametrize("case", ["attention", "attention, given room", "normalised GAE", "sampling", "policy", "tables"])
def test_prepared_calls_hold_what_their_wrapper_made(monkeypatch, case):
    """A prepared call repeats raw pointers: everything that the wrapper allocated stays until the prepared call itself is dropped."""
    import gc
    import weakref
    import torch
    from paper_2608_17641_b200 import binding
    made = []

    def alloc(shape, dtype, device):
        shape = shape if isinstance(shape, tuple) else (shape,)
        t = _Rows(0, dtype, shape)
        made.append(weakref.ref(t))
        return t

    monkeypatch.setattr(binding, "_lib", _FakeLibrary())
    monkeypatch.setattr(binding, "_alloc", alloc)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda stream=None: 1234)
    t = lambda dtype, *shape: _Rows(0, dtype, shape)
    f32, i32 = torch.float32, torch.int32
    x, u8 = t(f32, 2, 8), t(torch.uint8, 2, 8)
    prepare = binding.prepare
    if case.startswith("attention"):
        room = dict(workspace=lambda nbytes: alloc((nbytes,), torch.uint8, 0)) if "room" in case else {}
        step = prepare(binding.rlcs_prefix_attention_bf16, *_attention_args(), scale=0.1, **room)
        assert len(made) == 3
    elif case == "normalised GAE":
        step = prepare(binding.rlcs_gae_normalized, x, x, u8, gamma=0.9, lam=0.9)
        assert len(made) == 3
    elif case == "sampling":
        step = prepare(binding.rlcs_sample_actions, x, t(f32, 2))
        assert len(made) == 3
    elif case == "policy":
        step = prepare(binding.rlcs_policy_grad, x, t(i32, 2), t(f32, 2))
        assert len(made) == 4
    else:
        step = prepare(binding.rlcs_block_tables, t(i32, 4), t(i32, 4), t(i32, 9), t(i32, 4, 8), page_size=16, num_slots=5)
        assert len(made) == 4
    gc.collect()
    assert all(m() is not None for m in made)
    step()
    step.outputs = None
    gc.collect()
    assert all(m() is not None for m in made)
    assert getattr(binding._recording, "held", None) is None and getattr(binding._recording, "calls", None) is None
    del step
    gc.collect()
    assert all(m() is None for m in made)


def test_attention_calls_share_no_workspace(monkeypatch):
    """A call is several launches that hand results on through the workspace: another thread's call on the same stream, made while
    the first is being enqueued, must not get the same one; and none is kept behind the calls' backs."""
    import gc
    import threading
    import weakref
    from paper_2608_17641_b200 import api, binding
    made, seen = [], []

    class Memory(_Rows):
        def data_ptr(self):
            return id(self)

    def alloc(shape, dtype, device):
        t = Memory(0, dtype, shape if isinstance(shape, tuple) else (shape,))
        made.append(weakref.ref(t))
        return t

    class Library(_FakeLibrary):
        def __getattr__(self, name):
            fn = super().__getattr__(name)
            if name != "rlcs_prefix_attention_bf16":
                return fn

            def call(*args):
                seen.append(args[-3])
                if len(seen) == 1:
                    t = threading.Thread(target=lambda: api.shared_prefix_attention(*_attention_args()))
                    t.start()
                    t.join()
                return OK
            return call

    monkeypatch.setattr(binding, "_lib", Library())
    monkeypatch.setattr(binding, "_alloc", alloc)
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda stream=None: 1234)
    api.shared_prefix_attention(*_attention_args())
    assert len(seen) == 2 and seen[0] != seen[1]
    gc.collect()
    assert all(m() is None for m in made)


def test_attention_workspace_is_checked(monkeypatch):
    """A workspace in host memory, or with gaps, is refused: its pointer and size go to the kernels as they are."""
    import torch
    from paper_2608_17641_b200 import api, binding
    monkeypatch.setattr(binding, "_lib", _FakeLibrary())
    monkeypatch.setattr(binding, "_alloc", lambda shape, dtype, device: _Rows(0, dtype, shape))
    monkeypatch.setattr(binding, "_current_device", lambda: 0)
    monkeypatch.setattr(binding, "_stream", lambda stream=None: 1234)
    with pytest.raises(TypeError):
        api.shared_prefix_attention(*_attention_args(), workspace=torch.zeros(1 << 20, dtype=torch.uint8))
    with pytest.raises(TypeError):
        api.shared_prefix_attention(*_attention_args(), workspace=4096)
    with pytest.raises(ValueError):
        api.shared_prefix_attention(*_attention_args(), workspace=_Rows(1, torch.uint8, (1 << 20,)))
    gaps = _Rows(0, torch.uint8, (1 << 20,))
    gaps.is_contiguous = lambda: False
    with pytest.raises(ValueError):
        api.shared_prefix_attention(*_attention_args(), workspace=gaps)
    api.shared_prefix_attention(*_attention_args(), workspace=_Rows(0, torch.uint8, (1 << 20,)))
