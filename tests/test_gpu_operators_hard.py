"""Rollout and policy operators on the GPU where a value, a size or a call's surroundings are hard: NaN rows, sums of a
million terms, calls that are prepared, captured or cut short.  Tolerances are those of test_gpu_operators.py."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_operators import BF16, F32, api, check_policy, plain_policy, policy_inputs, rule_sample, up  # noqa: E402,F401

INF, NAN = math.inf, float("nan")


def near_log_probs(got, want):
    want = torch.as_tensor(want, dtype=torch.float64, device=got.device)
    return ((got.double() - want).abs() <= 1e-5 + 2.0 ** -22 * want.abs()).all()


# ------------------------------------------------------------------------------------------ sampling
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,A", [(600, 5000), (3, 40000)])
@pytest.mark.parametrize("numbers", [1, 5, 40])
def test_sample_top_k_above_the_numbers_of_a_row(api, R, A, numbers, dtype):
    """Fewer numbers than top_k, the rest NaN, right behind a call that leaves the multiprocessors' shared memory full of words that
    would pass for keys of logits far above the row's own."""
    g = torch.Generator(device="cuda").manual_seed(numbers)
    full = torch.full((1200, 32768), -3.0, dtype=BF16, device="cuda")
    some = torch.zeros(1200, dtype=torch.int32, device="cuda")
    x = torch.full((R, A), NAN, device="cuda")
    at = torch.rand(R, A, device="cuda", generator=g).argsort(1)[:, :numbers]
    x.scatter_(1, at, torch.randn(R, numbers, device="cuda", generator=g) - 6)
    x = x.to(dtype)
    one, u = torch.ones(R, device="cuda"), torch.rand(R, device="cuda", generator=g)
    for k in (50, 192):
        for p in (1.0, 0.8):
            ks = torch.full((R,), k, dtype=torch.int32, device="cuda")
            want = rule_sample(x, u, one, ks, one * p, 0 * one)
            api.compute_log_probs(full, some)
            got = api.sample_actions(x, u, top_k=k, top_p=p)
            assert torch.equal(got[0], want[0])
            assert near_log_probs(got[1], want[1]) and near_log_probs(got[2], want[2])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sample_log_probs_of_long_even_rows(api, dtype):
    """Enough rows for one block each, of logits that are all alike but a few: the softmax's sum has 2048 equal terms a thread, whose
    roundings in 32 bits have one sign (3e-5 of the sum)."""
    R, A = 600, 1 << 19
    x = torch.zeros(R, A, dtype=dtype, device="cuda")
    x[:, 77] = 2.8125
    u = torch.zeros(R, device="cuda")
    for k, others in ((0, 0), (30, 40)):
        x[:, 100:100 + others] = 2.0
        z = 1.0 + others * math.exp(2.0 - 2.8125) + (A - 1 - others) * math.exp(-2.8125)
        for kw in (dict(temperature=0.0), dict(top_k=1), dict(min_p=0.5), dict(top_p=0.5), dict(top_p=0.5, min_p=0.01), dict(top_k=300), dict())[:7 if k == 0 else 1] \
                + ((dict(top_k=k),) if k else ()):
            a, lp, _ = api.sample_actions(x, u, **kw)
            at = x.gather(1, a[:, None].long())[:, 0].double()
            assert near_log_probs(lp, at - 2.8125 - math.log(z)), kw


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R", [1, 600])
def test_sample_log_probs_count_what_cannot_be_drawn(api, R, dtype):
    """A million actions 22.5 below the most likely one: each weighs nothing, together they hold 1.8e-4 of the probability."""
    A = (1 << 20) + 3
    x = torch.full((R, A), -22.5, dtype=dtype, device="cuda")
    x[:, 5] = 0
    want = -math.log(1.0 + (A - 1) * math.exp(-22.5))
    u = torch.full((R,), 0.5, device="cuda")
    for kw in (dict(), dict(temperature=0.0), dict(top_k=50), dict(top_k=500), dict(top_p=0.9), dict(min_p=0.01), dict(top_k=500, min_p=0.01)):
        a, lp, kp = api.sample_actions(x, u, **kw)
        assert (a == 5).all() and near_log_probs(lp, want), kw
        assert (kp.abs() <= 1e-6).all(), kw


@pytest.mark.parametrize("A", [9, 300, 3000])
def test_sample_top_k_of_any_whole_number(api, A):
    """Numbers of no limit do not become one when they are cut to 32 bits."""
    x = torch.randn(40, A, generator=torch.Generator().manual_seed(1)).cuda()
    u = torch.rand(40, generator=torch.Generator().manual_seed(2)).cuda()
    want = api.sample_actions(x, u)
    for k in (-1, -2 ** 31, -2 ** 32 + 1, -2 ** 40 + 2, 2 ** 31, 2 ** 32 + 1, 2 ** 40):
        for v, w in zip(api.sample_actions(x, u, top_k=k), want):
            assert torch.equal(v, w), k


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [9, 100, 1000, 5000])
def test_sample_infinite_temperature(api, A, dtype):
    """Every allowed action alike, disallowed ones still never drawn."""
    g = torch.Generator(device="cuda").manual_seed(A)
    x = torch.randn(200, A, device="cuda", generator=g).to(dtype)
    x[:, 1::2] = -INF
    x[::7, 2] = torch.finfo(dtype).min
    n = (A + 1) // 2
    u = torch.rand(200, device="cuda", generator=g)
    for kw in (dict(), dict(top_k=n), dict(min_p=0.5), dict(top_p=1 - 2.0 ** -24)):
        a, lp, kp = api.sample_actions(x, u, temperature=INF, **kw)
        assert (a % 2 == 0).all() and (a >= 0).all(), kw
        assert near_log_probs(lp, -math.log(n)) and near_log_probs(kp, -math.log(n)), kw


# ------------------------------------------------------------------------------------------ policy loss
# one size (actions, type) for each way through the policy kernels: a thread, eight lanes, a warp in registers, a warp in two passes, a
# cluster that stages its rows, a cluster that reads them twice
POLICY_WAYS = [(6, F32), (64, BF16), (70, F32), (300, BF16), (1500, F32), (3000, BF16), (3500, F32), (8000, BF16), (5000, F32), (20000, BF16),
               (140001, F32), (600000, BF16)]


def nan_rows(A, dtype):
    """Twelve rows: two ordinary ones, then rows without a number in all their kinds, one of -inf alone, one left out."""
    x, a, adv, _ = policy_inputs(12, A, dtype, 3)
    x[2:9] = -INF
    x[2] = NAN
    x[3, ::2] = NAN
    x[4, 1::2] = NAN
    x[5, 0] = NAN
    x[6, A - 1] = NAN
    x[7, A // 2] = NAN
    x[9, A // 3] = INF
    x[10] = NAN
    mask = torch.ones(12, dtype=torch.uint8)
    mask[10] = 0
    return x, a, adv, mask, [2, 3, 4, 5, 6, 7, 9], [8, 10], [0, 1, 11]


@pytest.mark.parametrize("A,dtype", POLICY_WAYS)
def test_policy_rows_of_nan_are_not_left_out(api, A, dtype):
    x, a, adv, mask, broken, out, fine = nan_rows(A, dtype)
    xd, ad, advd, maskd = up(x), up(a), up(adv), up(mask)
    old = torch.zeros(12, device="cuda")
    clean = api.compute_policy_gradient(up(x[fine]), up(a[fine]), up(adv[fine]), entropy_coef=0.1)
    for got in (api.compute_policy_gradient(xd, ad, advd, mask=maskd, entropy_coef=0.1),
                api.compute_policy_gradient(xd, ad, advd, mask=maskd),
                api.compute_policy_gradient(xd, ad, advd, mask=maskd, entropy_coef=0.1, old_log_probs=old),
                api.compute_log_probs(xd, ad, mask=maskd)):
        for v in got:
            assert torch.isnan(v[broken]).all(), [i for i in broken if not torch.isnan(v[i]).all()]
            assert (v[out] == 0).all()
            assert torch.isfinite(v[fine]).all()
    got = api.compute_policy_gradient(xd, ad, advd, mask=maskd, entropy_coef=0.1)
    for v, w in zip(got, clean):
        assert ((v[fine].double() - w.double()).abs() <= 1e-5 + 2.0 ** -7 * w.double().abs()).all()


@pytest.mark.parametrize("A,dtype", POLICY_WAYS)
def test_policy_nan_in_the_acting_log_probs_is_seen(api, A, dtype):
    """A ratio or an advantage that is NaN makes the row's loss and gradient NaN (not its log-probability and entropy); a ratio past the
    largest float against an advantage of 0 does not."""
    x, a, adv, _ = policy_inputs(8, A, dtype, 4)
    x[5, a[5]] = -INF                                         # probability 0, and acted with probability 0
    old = plain_policy(x, a, adv, None, None, 1.0, 0.2, 0, 1)[1].float()
    old[1] = NAN
    adv[2] = NAN
    old[3], adv[3] = -200.0, 0.0
    old[4], adv[4] = -200.0, -1.0                             # the ratio overflows: as far as the formula goes
    old[5] = -INF
    loss, lp, ent, grad = api.compute_policy_gradient(up(x), up(a), up(adv), old_log_probs=up(old), entropy_coef=0.1)
    for r in (1, 2, 5):
        assert torch.isnan(loss[r]) and torch.isnan(grad[r]).all(), r
    assert torch.isfinite(ent).all() and torch.isfinite(lp[[0, 1, 2, 3, 4, 6, 7]]).all() and lp[5] == -INF
    for r in (0, 3, 6, 7):
        assert torch.isfinite(loss[r]) and torch.isfinite(grad[r]).all(), r
    assert abs(float(loss[3] + 0.1 * ent[3])) <= 1e-6
    assert loss[4] == INF


@pytest.mark.parametrize("A,dtype", POLICY_WAYS)
def test_policy_masks_of_any_low_value(api, A, dtype):
    """Disallowed actions marked by a low number instead of -inf, two thirds and all but eight of a row, whole stretches of them among the
    allowed ones, and rows that lie far from 0 altogether."""
    R = 7
    lowest = torch.finfo(dtype).min
    for low in (-1e4, -1e9, -1e10, -3e20, -9e28, -1e30, -1.2e30, -1e35, lowest):
        for share in (0.66, 1.0):
            x, a, adv, g = policy_inputs(R, A, dtype, 5)
            off = torch.rand(R, A, generator=g) < share
            off[:, A // 3:A // 2] = True
            off[torch.arange(R)[:, None], torch.randint(0, A, (R, 8), generator=g)] = False
            off[torch.arange(R), a.long()] = False
            x[off] = low
            x[0] += 3e5
            x[1, ~off[1]] += 2.0 ** 40
            x[2, ~off[2]] -= 2.0 ** 33
            got = check_policy(api, x, a, adv, T=0.8, c=0.05, in_place=share == 1.0)
            assert all(torch.isfinite(v).all() for v in got)


# ------------------------------------------------------------------------------------------ prepared, captured and concurrent calls
def plain_memory(monkeypatch):
    """Memory of torch's own allocator, which hands out again what is dropped (the harness's guard bands keep everything)."""
    from paper_2608_17641_b200 import binding
    monkeypatch.setattr(binding, "_alloc", lambda shape, dtype, device: torch.empty(shape, dtype=dtype, device="cuda"))


def attention_inputs(B=8, prompt=700, own=300, seed=0):
    """Two groups of rows, with every key in its own page order: what shared_prefix_attention() takes, and its lengths' bounds."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    page, Hk, d = 16, 2, 64
    wp, wo = -(-prompt // page), -(-own // page)
    ids = torch.randperm(2 * wp + B * wo, device="cuda", generator=g).int()
    k, v = (torch.randn(ids.numel(), page, Hk, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    q = torch.randn(B, 8, d, device="cuda", generator=g).bfloat16()
    return ((q, k, v, ids[:2 * wp].view(2, wp), i32(prompt, prompt // 2), i32(0, B // 2, B), ids[2 * wp:].view(B, wo),
             torch.randint(0, own + 1, (B,), device="cuda", generator=g, dtype=torch.int32)), dict(max_prefix_len=prompt, max_len=own))


def test_prepared_attention_keeps_its_workspace(monkeypatch):
    """The workspace that the wrapper made is not handed to anybody else while the prepared call lives."""
    from paper_2608_17641_b200 import binding
    plain_memory(monkeypatch)
    args, bounds = attention_inputs()
    want = binding.rlcs_prefix_attention_bf16(*args, scale=0.125, **bounds)
    need = binding.lib().rlcs_prefix_attention_workspace_bytes(8, 8, 2, 64, 16, 2, 700, 300)
    step = binding.prepare(binding.rlcs_prefix_attention_bf16, *args, scale=0.125, **bounds)
    others = [torch.full((need,), 85, dtype=torch.uint8, device="cuda") for _ in range(4)]
    for _ in range(3):
        got = step()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert all((t == 85).all() for t in others)


def test_prepared_sampling_and_policy_repeat_the_direct_call():
    from paper_2608_17641_b200 import binding
    x = torch.randn(9, 5000, generator=torch.Generator().manual_seed(0)).cuda()
    u, adv = torch.rand(9, generator=torch.Generator().manual_seed(1)).cuda(), torch.arange(9.0).cuda()
    sample = binding.prepare(binding.rlcs_sample_actions, x, u, top_k=30)
    learn = binding.prepare(binding.rlcs_policy_grad, x, sample.outputs[0], adv, entropy_coef=0.1)
    for seed in (2, 3):
        x.copy_(torch.randn(9, 5000, generator=torch.Generator().manual_seed(seed)))
        got = (*sample(), *learn())
        want = binding.rlcs_sample_actions(x, u, top_k=30)
        for v, w in zip(got, (*want, *binding.rlcs_policy_grad(x, want[0], adv, entropy_coef=0.1))):
            assert torch.equal(v, w)


def test_attention_in_graphs_shares_no_workspace(api, monkeypatch):
    """Captured without a workspace of the caller's, the first call of its stream among them; larger calls in between and other
    tensors in the memory that they leave; two graphs of one capture stream replayed side by side."""
    plain_memory(monkeypatch)
    sets = [attention_inputs(seed=s) for s in (1, 2)]
    want = [api.shared_prefix_attention(*args, **bounds) for args, bounds in sets]
    large, large_bounds = attention_inputs(B=64, prompt=6000, own=2000, seed=3)
    side = torch.cuda.Stream()
    graphs, out = [torch.cuda.CUDAGraph() for _ in sets], []
    torch.cuda.synchronize()
    for graph, (args, bounds) in zip(graphs, sets):
        with torch.cuda.graph(graph, stream=side):
            out.append(api.shared_prefix_attention(*args, **bounds))
    with torch.cuda.stream(side):
        large_want = api.shared_prefix_attention(*large, **large_bounds)
        others = [torch.full((n << 20,), 85, dtype=torch.uint8, device="cuda") for n in (1, 1, 2, 4, 8)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(50):
        for stream, graph in zip(streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay()
    with torch.cuda.stream(side):
        large_got = api.shared_prefix_attention(*large, **large_bounds)
    torch.cuda.synchronize()
    for got, exp in zip((*out, large_got), (*want, large_want)):
        assert torch.equal(got[0], exp[0]) and torch.equal(got[1], exp[1])
    assert all((t == 85).all() for t in others)


# ------------------------------------------------------------------------------------------ waits that run out
@pytest.fixture
def wait_polls():
    from paper_2608_17641_b200 import binding
    yield binding.rlcs_debug_set_wait_polls
    binding.rlcs_debug_set_wait_polls(-1)


@pytest.mark.parametrize("page", [16, 48])                    # copied by boxes, and piece by piece
@pytest.mark.parametrize("rows", [4, 30, 70])                 # 16, 128 and 256 rows of a prompt at a time
@pytest.mark.parametrize("d", [64, 128])
def test_attention_waits_that_run_out(api, wait_polls, rows, page, d):
    """Waits that give up at once or early: the call ends by itself, its rows are NaN or (where no wait of theirs ran out) right, and
    nothing of it is still on its way: calls right behind it are as ever."""
    g = torch.Generator(device="cuda").manual_seed(d)
    prompt, own = 1500, 130
    wp, wo = -(-prompt // page), -(-own // page)
    ids = torch.randperm(wp + rows * wo, device="cuda", generator=g).int()
    k, v = (torch.randn(ids.numel(), page, 1, d, device="cuda", generator=g).bfloat16() for _ in range(2))
    i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device="cuda")
    q = torch.randn(rows, 4, d, device="cuda", generator=g).bfloat16()
    lens = torch.randint(0, own + 1, (rows,), device="cuda", generator=g, dtype=torch.int32)
    call = lambda: api.shared_prefix_attention(q, k, v, ids[:wp].view(1, wp), i32(prompt), i32(0, rows), ids[wp:].view(rows, wo), lens)
    want, want_lse = call()
    for polls in (0, 0, 1, 2, 5, 20, 100):
        wait_polls(polls)
        out, lse = call()
        wait_polls(-1)
        again, again_lse = call()
        broken = torch.isnan(lse)
        assert torch.isnan(out[broken]).all()
        assert torch.equal(out[~broken], want[~broken]) and torch.equal(lse[~broken], want_lse[~broken])
        assert torch.equal(again, want) and torch.equal(again_lse, want_lse)
        if polls == 0 and (page == 16 or rows > 4):           # small tiles copied piece by piece have no waits of this kind
            assert broken.all()


@pytest.mark.parametrize("R,A,dtype", [(700, 5000, F32), (700, 32768, BF16), (40, 40000, F32), (300, 140001, BF16), (9, 600000, BF16), (3, 20011, F32)])
def test_policy_waits_that_run_out(api, wait_polls, R, A, dtype):
    """The same for the policy loss, one block and clusters of 2 to 8 a row, more rows than run at once, rows left out among them, and
    rows that take the second way of summing."""
    g = torch.Generator(device="cuda").manual_seed(A)
    x = torch.randn(R, A, device="cuda", generator=g).to(dtype)
    x[::5] = torch.finfo(dtype).min
    a = torch.randint(0, A, (R,), device="cuda", generator=g, dtype=torch.int32)
    adv, mask = torch.randn(R, device="cuda", generator=g), torch.rand(R, device="cuda", generator=g) < 0.8
    call = lambda: api.compute_policy_gradient(x, a, adv, mask=mask, entropy_coef=0.1)
    want = call()
    for polls in (0, 0, 1, 2, 5, 20, 100):
        wait_polls(polls)
        got = call()
        wait_polls(-1)
        again = call()
        for v, w in zip(got, want):
            broken = torch.isnan(v)
            assert not broken[~mask].any() and torch.equal(v[~broken], w[~broken])
            if polls == 0 and v.dim() == 1:                   # (the second way of summing waits for nothing but its cluster)
                ordinary = mask.clone()
                ordinary[::5] = False
                assert broken[ordinary].all()
        for v, w in zip(again, want):
            assert torch.equal(v, w)


