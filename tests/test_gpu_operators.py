"""Rollout and policy operators on the GPU against plain 64-bit implementations: action sampling, policy loss and its
gradient, attention over a shared paged prefix, block tables.

Tolerances.  fp32 logits scaled by 1/T carry a relative rounding of 2^-23, so a difference d to the row's maximum is off by at
most |d| 2^-22 and exp(d) by the same factor; |d| <= 30 in what still counts, hence 1e-5 on log-probabilities, entropies and
(relative) probabilities, plus 2^-22 of the value for its own rounding.  bfloat16 results add half a last place, 2^-8 of the value.
Attention: the weights enter as two bfloat16 parts (2^-17 of each), scores of up to 30 are off by 30 * 2^-22: 2^-15 of the
largest |v| covers both."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _util import guarded_empty, guarded_upload  # noqa: E402

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def api():
    from paper_2608_17641_b200 import api as a
    return a


def up(t, offset=0):
    return guarded_upload(t.cpu(), offset)


def strided_rows(x, pad, offset=0):
    """A device copy of x [R, A] whose rows are `pad` elements apart beyond A, guarded."""
    R, A = x.shape
    big = torch.full((R, A + pad), float("nan"), dtype=x.dtype)
    big[:, :A] = x
    return up(big, offset)[:, :A]


# ------------------------------------------------------------------------------------------ sampling
def plain_sample(x, u, t, k, p, low):
    """The rule of the header row by row: whole weights from the device's own fp32 exponentials (so that whole numbers can be
    compared), everything after them in Python integers and 64-bit floats."""
    x = x.float()
    actions, full, part = [], [], []
    for r in range(x.shape[0]):
        row = torch.where(torch.isnan(x[r]), torch.tensor(-math.inf), x[r])
        top = row.max()
        if top == -math.inf:
            actions.append(-1), full.append(-math.inf), part.append(-math.inf)
            continue
        tr = torch.tensor(float(t[r]), dtype=F32)
        greedy = not bool(tr > 0)
        inv = torch.tensor(1.0) if greedy else (torch.ones(1, device="cuda") / tr.cuda()).cpu()[0]
        d = torch.where(row == top, torch.zeros(()), (row - top) * inv)
        e = torch.exp(d.cuda()).cpu()
        w = [math.floor(v * 2.0 ** 31 + 0.5) for v in e.double().tolist()]
        order = sorted(range(len(w)), key=lambda j: (-float(row[j]), j))
        lowest = torch.tensor(float(low[r]), dtype=F32)
        n = 1 if greedy else (int(k[r]) if int(k[r]) > 0 else len(w))
        kept = [j for i, j in enumerate(order[:n]) if i == 0 or not bool(lowest > 0) or bool(e[j] >= lowest)]
        pr = float(torch.tensor(float(p[r]), dtype=F32))
        if pr < 1:
            enough, before, some = pr * float(sum(w[j] for j in kept)), 0, []
            for i, j in enumerate(kept):
                if i == 0 or float(before) < enough:
                    some.append(j)
                before += w[j]
            kept = some
        total = sum(w[j] for j in kept)
        target = min(math.floor(float(torch.tensor(float(u[r]), dtype=F32)) * float(total)), total - 1)
        run = 0
        for j in sorted(kept):
            run += w[j]
            if run > target:
                break
        z = torch.exp((row.double() - top.double()) / (1.0 if greedy else float(tr)))
        z = torch.where(row == top, torch.ones((), dtype=torch.float64), z)
        dj = 0.0 if row[j] == top else float(row[j].double() - top.double()) / (1.0 if greedy else float(tr))
        actions.append(j), full.append(dj - math.log(float(z.sum()))), part.append(dj - math.log(float(z[kept].sum())))
    return np.array(actions), np.array(full), np.array(part)


def check_sample(api, x, u, t=None, k=None, p=None, low=None, pad=0, offset=0, stream=None):
    R = x.shape[0]
    every = lambda v, d: torch.full((R,), d) if v is None else v if isinstance(v, torch.Tensor) else torch.full((R,), v)
    want = plain_sample(x, u, every(t, 1.0), every(k, 0), every(p, 1.0), every(low, 0.0))
    dev = lambda v: up(v) if isinstance(v, torch.Tensor) else v
    got = api.sample_actions(strided_rows(x, pad, offset), up(u), temperature=dev(t), top_k=dev(k), top_p=dev(p), min_p=dev(low), stream=stream)
    a, lp, kp = (v.cpu().numpy() for v in got)
    assert a.dtype == np.int32 and np.array_equal(a, want[0]), (a, want[0])
    for g, w in ((lp, want[1]), (kp, want[2])):
        there = np.isfinite(w)
        assert np.array_equal(g[~there], w[~there].astype(np.float32))
        assert (np.abs(g[there] - w[there]) <= 1e-5 + 2.0 ** -22 * np.abs(w[there])).all(), np.abs(g - w)[there].max()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [1, 2, 7, 31, 32, 33, 64, 65, 255, 1000, 1024, 1025, 2049, 4099, 20011])
def test_sample_sizes_and_filters(api, A, dtype):
    g = torch.Generator().manual_seed(A)
    R = 12 if A < 5000 else 6
    x = (torch.randn(R, A, generator=g) * 3).to(dtype)
    u = torch.rand(R, generator=g)
    check_sample(api, x, u, pad=A % 3)
    check_sample(api, x, u, t=0.7, k=torch.randint(0, max(2, A), (R,), generator=g, dtype=torch.int32),
                 p=torch.rand(R, generator=g) * 1.1, low=torch.rand(R, generator=g) * 0.2, offset=1)
    check_sample(api, x, u, t=torch.rand(R, generator=g) * 2, p=0.9, pad=5)
    check_sample(api, x, u, k=5, low=0.01)


@pytest.mark.parametrize("A", [40, 3000])
def test_sample_extremes_of_the_uniform(api, A):
    x = torch.randn(8, A, generator=torch.Generator().manual_seed(1)) * 2
    u = torch.tensor([0.0, 1 - 2.0 ** -24, 2.0 ** -30, 0.5, 0.25, 1.0, float("nan"), 1e-45])
    fine = torch.nan_to_num(u).clamp(max=1 - 2.0 ** -24)
    got = api.sample_actions(up(x), up(u), top_p=0.99)
    want = api.sample_actions(up(x), up(fine), top_p=0.99)
    assert torch.equal(got[0][:5], want[0][:5]) and got[0].min() >= 0 and got[0].max() < A
    check_sample(api, x[:5], u[:5], k=17)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [6, 100, 5000])
def test_sample_ties_go_to_the_lowest_index(api, A, dtype):
    x = torch.zeros(6, A, dtype=dtype)
    x[1, A // 2:] = 1
    x[2, ::2] = -0.0
    x[3] = (torch.arange(A) % 5).to(dtype)
    x[4] = -math.inf
    x[4, 3] = 2
    x[5, A - 1] = 3
    u = torch.tensor([0.999, 0.999, 0.5, 0.7, 0.3, 0.9])
    for k in (1, 2, 3, A - 1, A, A + 5):
        check_sample(api, x, u, k=k)
        check_sample(api, x, u, k=k, p=0.5)
    for p in (0.0, 1e-6, 0.3, 0.6, 1.0 - 2.0 ** -24):
        check_sample(api, x, u, p=p)
    check_sample(api, x, u, t=0.0)
    check_sample(api, x, u, low=1.0)
    check_sample(api, x, u, low=2.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [9, 1500])
def test_sample_empty_masked_and_infinite_rows(api, A, dtype):
    g = torch.Generator().manual_seed(3)
    x = torch.randn(9, A, generator=g).to(dtype)
    x[0] = -math.inf
    x[1] = float("nan")
    x[2, ::2] = float("nan")
    x[3, 1:] = -math.inf
    x[4, :] = torch.finfo(dtype).min
    x[5, 1:] = torch.finfo(dtype).min
    x[6, 2] = math.inf
    x[7, 2] = x[7, 5] = math.inf
    x[8, ::3] = -math.inf
    u = torch.rand(9, generator=g)
    check_sample(api, x, u)
    check_sample(api, x, u, t=0.5, k=4, p=0.8, low=0.05)
    check_sample(api, x, u, t=0.0)
    check_sample(api, x, u, t=1e-30)
    check_sample(api, x, u, t=1e30)


def rule_sample(x, u, t, k, p, low):
    """The same rule as plain_sample() for wide rows, on the GPU: a stable sort and exact 64-bit sums."""
    x = torch.where(torch.isnan(x.float()), -math.inf, x.float())
    R, A = x.shape
    top = x.amax(1, keepdim=True)
    greedy = ~(t > 0)
    inv = (1.0 / torch.where(greedy, 1.0, t))[:, None]
    e = torch.exp(torch.where(x == top, 0.0, (x - top) * inv))
    w = torch.floor(e.double() * 2.0 ** 31 + 0.5).long()
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    rank = torch.arange(A, device=x.device)[None]
    limit = torch.where(greedy, 1, torch.where(k > 0, k.long(), A))[:, None]
    keep = (rank < limit) & ((rank == 0) | ~(low > 0)[:, None] | (e.gather(1, order) >= low[:, None]))
    ws = torch.where(keep, w.gather(1, order), 0)
    before = torch.cumsum(ws, 1) - ws
    keep &= (rank == 0) | ~(p < 1)[:, None] | (before.double() < p.double()[:, None] * ws.sum(1, keepdim=True).double())
    kept = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, 0))
    total = kept.sum(1)
    target = torch.minimum(torch.floor(u.double() * total.double()).long(), total - 1)
    a = (torch.cumsum(kept, 1) <= target[:, None]).sum(1)
    d = torch.where(x == top, 0.0, (x - top) * inv).double()
    z = torch.exp(d)
    at = d.gather(1, a[:, None])[:, 0]
    return a.int(), at - z.sum(1).log(), at - torch.where(kept > 0, z, 0.0).sum(1).log()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R,A", [(1, 131072), (3, 262143), (40, 33001), (130, 9000), (300, 8200), (700, 1200), (2, 1000001)])
@pytest.mark.parametrize("kind", ["peaked", "flat", "steps"])
def test_sample_wide_rows(api, R, A, dtype, kind):
    """Every cluster size and way through the large-row kernel: equal to the rule, whatever the settings."""
    g = torch.Generator(device="cuda").manual_seed(A + R)
    rand = lambda: torch.rand(R, device="cuda", generator=g)
    x = torch.randn(R, A, device="cuda", generator=g) * {"peaked": 3.0, "flat": 0.05, "steps": 4.0}[kind]
    if kind == "steps":
        x = x.round()                                        # thousands of equal logits at every cut
    x = x.to(dtype)
    one = torch.ones(R, device="cuda")
    none = torch.zeros(R, device="cuda", dtype=torch.int32)
    ks = torch.randint(1, 400, (R,), device="cuda", generator=g, dtype=torch.int32)
    for t, k, p, low in ((one, none, one, 0 * one), (rand() + 0.3, ks, one, 0 * one), (rand() + 0.5, none, rand(), 0 * one),
                         (rand() * 3 + 0.1, ks * 40, rand() * 0.3 + 0.7, rand() * 0.02), (one, none, one, rand() * 0.1), (0 * one, none, one, 0 * one),
                         (one * 0.05, ks, rand(), rand() * 0.2)):
        u = rand()
        want = rule_sample(x, u, t, k, p, low)
        got = api.sample_actions(x, u, temperature=t, top_k=k, top_p=p, min_p=low)
        assert torch.equal(got[0], want[0]), (got[0] != want[0]).sum()
        for v, r in zip(got[1:], want[1:]):
            assert ((v.double() - r).abs() <= 1e-5 + 2.0 ** -22 * r.abs()).all()


def test_sample_parameters_that_limit_nothing(api):
    x = torch.randn(5, 300, generator=torch.Generator().manual_seed(9))
    u = torch.rand(5, generator=torch.Generator().manual_seed(8))
    base = api.sample_actions(up(x), up(u))
    nan = torch.full((5,), float("nan"))
    other = api.sample_actions(up(x), up(u), top_k=up(torch.full((5,), -3, dtype=torch.int32)), top_p=up(nan), min_p=up(nan))
    for a, b in zip(base, other):
        assert torch.equal(a, b)


def test_sample_follows_the_distribution(api):
    """Frequencies over evenly spaced uniforms are the probabilities, to one part in the number of draws each."""
    n, A = 20000, 11
    row = torch.randn(A, generator=torch.Generator().manual_seed(2)) * 2
    x = row.repeat(n, 1)
    a, lp, _ = api.sample_actions(up(x), up((torch.arange(n) + 0.5) / n))
    want = torch.softmax(row.double(), 0)
    got = torch.bincount(a.cpu().long(), minlength=A).double() / n
    assert (got - want).abs().max() <= 2 / n + 1e-6
    assert (lp.cpu().double().exp() - want[a.cpu().long()]).abs().max() < 1e-5


def test_sample_leading_shape_stream_and_repeat(api):
    x = torch.randn(4, 5, 333, generator=torch.Generator().manual_seed(4))
    u = torch.rand(4, 5, generator=torch.Generator().manual_seed(5))
    xd, ud = up(x), up(u)
    one = api.sample_actions(xd, ud, top_k=20)
    assert one[0].shape == (4, 5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    two = api.sample_actions(xd, ud, top_k=20, stream=s)
    s.synchronize()
    for a, b in zip(one, two):
        assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------ policy loss
def plain_policy(x, a, adv, old, mask, T, clip, c, scale):
    """64-bit definition; rows left out give zeros."""
    x = x.double() / T
    R, A = x.shape
    live = (torch.ones(R, dtype=torch.bool) if mask is None else mask.bool()) & (a >= 0) & (a < A)
    live &= (x > -math.inf).any(1)
    pick = a.long().clamp(0, A - 1)
    x = torch.where(live[:, None], x, torch.zeros((), dtype=torch.float64))
    lp = torch.log_softmax(x, 1)
    p = lp.exp()
    safe = torch.where(p > 0, lp, torch.zeros((), dtype=torch.float64))
    h = -(p * safe).sum(1)
    la = lp.gather(1, pick[:, None])[:, 0]
    adv = torch.zeros(R, dtype=torch.float64) if adv is None else adv.double()
    if old is None:
        gain, s = adv * la, adv
    else:
        rho = (la - old.double()).exp()
        free, held = rho * adv, rho.clamp(1 - clip, 1 + clip) * adv
        gain, s = torch.minimum(free, held), torch.where(free <= held, free, torch.zeros((), dtype=torch.float64))
    hot = torch.zeros_like(p).scatter_(1, pick[:, None], 1.0)
    grad = scale / T * (s[:, None] * (p - hot) + c * p * (safe + h[:, None]))
    z = lambda v: torch.where(live, v, torch.zeros((), dtype=torch.float64))
    return z(-scale * (gain + c * h)), z(la), z(h), torch.where(live[:, None], grad, torch.zeros((), dtype=torch.float64))


def check_policy(api, x, a, adv, old=None, mask=None, T=1.0, clip=0.2, c=0.0, scale=1.0, pad=0, offset=0, in_place=False):
    want = plain_policy(x, a, adv, old, mask, T, clip, c, scale)
    dev = lambda v: None if v is None else up(v)
    xd = strided_rows(x, pad, offset)
    got = [v.cpu().double() for v in api.compute_policy_gradient(
        xd, dev(a), dev(adv), old_log_probs=dev(old), mask=dev(mask), temperature=T, clip=clip, entropy_coef=c, scale=scale,
        in_place=in_place)]
    s = 1.0 if old is None else (want[1] - old.double()).exp().clamp(max=1e4)      # the ratio magnifies what lp is off by
    size = adv.double().abs()
    near = lambda g, w, tol: ((g - w).abs() <= tol) | (g == w)
    assert near(got[1], want[1], 1e-5 + 2.0 ** -22 * want[1].abs()).all()
    assert near(got[2], want[2], 1e-5 + 2.0 ** -22 * want[2].abs()).all()
    assert near(got[0], want[0], scale * (size * s + c) * 2e-5 + 2.0 ** -20 * want[0].abs()).all()
    tol = (scale / T * (size * s + c * (want[2] + 1)) * 2e-5)[:, None] + 2.0 ** -20 * want[3].abs()
    if x.dtype == BF16:
        tol = tol + 2.0 ** -8 * want[3].abs() + 1e-38
    assert near(got[3], want[3], tol).all(), (got[3] - want[3]).abs().max()
    if not in_place:
        assert torch.equal(xd.cpu().nan_to_num(), x.nan_to_num())
    return got


def policy_inputs(R, A, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(R, A, generator=g) * 3).to(dtype)
    return x, torch.randint(0, A, (R,), generator=g, dtype=torch.int32), torch.randn(R, generator=g), g


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [1, 2, 3, 8, 17, 18, 32, 33, 64, 96, 129, 500, 1024, 2047, 2048, 2049, 4095, 10007, 40000])
def test_policy_sizes(api, A, dtype):
    R = 37 if A < 3000 else 5
    x, a, adv, g = policy_inputs(R, A, dtype, A)
    check_policy(api, x, a, adv, pad=A % 4)
    check_policy(api, x, a, adv, T=0.7, c=0.05, scale=1 / R, offset=A % 3)
    noise = torch.where(torch.rand(R, generator=g) < 0.5, torch.rand(R, generator=g) * 0.3 - 0.15, (torch.rand(R, generator=g) - 0.5) * 3)
    old = (plain_policy(x, a, adv, None, None, 1.3, 0.2, 0, 1)[1] + noise).float()
    check_policy(api, x, a, adv, old=old, mask=torch.rand(R, generator=g) < 0.7, T=1.3, c=0.01, pad=1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [65, 128, 255, 257, 600, 1030, 4097, 8200, 16390, 33000, 140001, 262144, 700001])
def test_policy_sizes_of_every_way(api, A, dtype):
    """Lanes, warps, one block and clusters of 2 to 8 a row, kept on the chip or read twice; rows at odd addresses, disallowed actions and
    rows left out between the others, more rows than clusters run at once."""
    R = 9 if A < 20000 else 3
    x, a, adv, g = policy_inputs(R, A, dtype, A)
    x[torch.rand(R, A, generator=g) < 0.2] = -math.inf
    x[torch.arange(R), a.long()] = 1.5
    mask = torch.ones(R, dtype=torch.bool)
    mask[1] = False
    for pad, offset, in_place in ((0, 0, False), (A % 3 + 1, 1, False), (0, 3, True)):
        check_policy(api, x, a, adv, mask=mask, T=0.8, c=0.05, scale=1 / R, pad=pad, offset=offset, in_place=in_place)


def test_policy_gradient_into_a_buffer_of_another_alignment():
    from paper_2608_17641_b200 import binding
    for A in (50, 300, 3000, 9000):
        x, a, adv, _ = policy_inputs(6, A, BF16, A)
        want = binding.rlcs_policy_grad_bf16(up(x), up(a), up(adv), entropy_coef=0.2)
        out = strided_rows(torch.zeros(6, A, dtype=BF16), 3, 1)
        got = binding.rlcs_policy_grad_bf16(up(x), up(a), up(adv), entropy_coef=0.2, dlogits=out)
        for v, w in zip(got, want):
            assert torch.equal(v, w)


def test_policy_more_rows_than_run_at_once(api):
    """The persistent clusters of the wide kernel take several rows each, dead ones among them."""
    R, A = 1300, 10001
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(R, A, device="cuda", generator=g).bfloat16()
    a = torch.randint(0, A, (R,), device="cuda", generator=g, dtype=torch.int32)
    adv, mask = torch.randn(R, device="cuda", generator=g), torch.rand(R, device="cuda", generator=g) < 0.7
    loss, lp, h, grad = api.compute_policy_gradient(x, a, adv, mask=mask, entropy_coef=0.1)
    ref = torch.log_softmax(x.double(), 1)
    p = ref.exp()
    ent = -(p * ref).sum(1)
    la = ref.gather(1, a[:, None].long())[:, 0]
    live = mask.double()
    assert ((lp - la * live).abs() <= 2e-5).all() and ((h - ent * live).abs() <= 2e-5).all()
    hot = torch.zeros_like(p).scatter_(1, a[:, None].long(), 1.0)
    want = live[:, None] * (adv.double()[:, None] * (p - hot) + 0.1 * p * (ref + ent[:, None]))
    assert ((grad - want).abs() <= 2.0 ** -8 * want.abs() + 1e-6).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("R", [1, 7, 8, 9, 1000, 4099])
def test_policy_row_counts(api, R, dtype):
    x, a, adv, _ = policy_inputs(R, 18, dtype, R)
    check_policy(api, x, a, adv, c=0.02)
    x, a, adv, _ = policy_inputs(R, 129, dtype, R)
    check_policy(api, x, a, adv, c=0.02, in_place=True)


@pytest.mark.parametrize("A", [5, 70, 3001])
def test_policy_rows_left_out_may_hold_anything(api, A):
    x, a, adv, _ = policy_inputs(9, A, F32, 6)
    x[0], x[1], x[2], x[3] = float("nan"), math.inf, -math.inf, float("nan")
    mask = torch.tensor([0, 0, 1, 1, 1, 1, 2, 255, 0], dtype=torch.uint8)
    a[3], a[4], a[5] = -1, A, 2 ** 31 - 1
    adv[0] = float("nan")
    adv_ref = adv.nan_to_num()
    want = plain_policy(x.nan_to_num(posinf=0.0), a, adv_ref, None, mask, 1.0, 0.2, 0.1, 1.0)
    got = [v.cpu().double() for v in api.compute_policy_gradient(up(x), up(a), up(adv), mask=up(mask), entropy_coef=0.1)]
    dead = [0, 1, 2, 3, 4, 5, 8]
    for v in got:
        assert (v[dead] == 0).all()
    for v, w in zip(got, want):
        assert (v[6:8] - w[6:8]).abs().max() < 1e-4


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [4, 70, 5000])
def test_policy_disallowed_actions(api, A, dtype):
    x, a, adv, g = policy_inputs(11, A, dtype, 8)
    off = torch.rand(11, A, generator=g) < 0.5
    off[torch.arange(11), a.long()] = False
    x[off] = -math.inf
    x[0] = torch.finfo(dtype).min
    x[1] = -math.inf
    x[1, a[1]] = 5
    got = check_policy(api, x, a, adv, c=0.1, T=0.9 if dtype == F32 else 1.0)
    assert (got[3][off & (torch.arange(11)[:, None] > 1)] == 0).all()
    # an action of probability 0: log-probability -inf, everything else finite
    x, a, adv, g = policy_inputs(3, A, dtype, 8)
    x[0, a[0]] = -math.inf
    loss, lp, h, grad = (v.cpu() for v in api.compute_policy_gradient(up(x), up(a), up(adv)))
    assert lp[0] == -math.inf and torch.isfinite(h).all() and torch.isfinite(grad).all()


@pytest.mark.parametrize("A", [6, 70, 5000])
def test_policy_nan_stays_in_its_row(api, A):
    x, a, adv, _ = policy_inputs(4, A, F32, 2)
    clean = [v.cpu() for v in api.compute_policy_gradient(up(x), up(a), up(adv), entropy_coef=0.1)]
    for at in (0, A // 2, A - 1):
        y = x.clone()
        y[2, at] = float("nan")
        got = [v.cpu() for v in api.compute_policy_gradient(up(y), up(a), up(adv), entropy_coef=0.1)]
        for c, v in zip(clean, got):
            assert torch.isnan(v[2]).all()
            assert torch.equal(c[[0, 1, 3]], v[[0, 1, 3]])


def test_policy_gradient_against_differences(api):
    """The kernel's gradient against central differences of the 64-bit loss (h = 1e-4: the third derivative's h^2 and the
    rounding's 1e-16 / h both stay below 1e-7; the kernel itself is within 2e-5)."""
    x, a, adv, g = policy_inputs(6, 9, F32, 12)
    old = plain_policy(x, a, adv, None, None, 0.8, 0.2, 0, 1)[1].float() + torch.tensor([0.05, -0.1, 0.6, -0.6, 0.6, -0.6])
    for o in (None, old):
        got = api.compute_policy_gradient(up(x), up(a), up(adv), old_log_probs=None if o is None else up(o), temperature=0.8,
                                          entropy_coef=0.3)[3].cpu().double()
        for j in range(9):
            d = torch.zeros(6, 9, dtype=torch.float64)
            d[:, j] = 1e-4
            up_, down = (plain_policy(x.double() + s * d, a, adv, o, None, 0.8, 0.2, 0.3, 1.0)[0] for s in (1, -1))
            assert ((up_ - down) / 2e-4 - got[:, j]).abs().max() < 2e-5


def test_policy_scoring_and_shapes(api):
    x, a, adv, _ = policy_inputs(12, 50, BF16, 3)
    want = plain_policy(x, a, adv, None, None, 1.0, 0.2, 0, 1)
    lp, h = api.compute_log_probs(up(x.view(3, 4, 50)), up(a.view(3, 4)))
    assert lp.shape == (3, 4) and (lp.cpu().view(-1).double() - want[1]).abs().max() < 1e-5 and (h.cpu().view(-1).double() - want[2]).abs().max() < 1e-5
    out = api.compute_policy_gradient(up(x.view(3, 4, 50)), up(a.view(3, 4)), up(adv.view(3, 4)))
    assert out[3].shape == (3, 4, 50) and out[3].dtype == BF16 and (out[1] == lp).all()


def test_policy_sampled_log_probs_agree(api):
    """What sample_actions says of its action is what scoring says of it, for the whole softmax at that temperature."""
    for A in (18, 3000):
        x, _, _, g = policy_inputs(40, A, F32, 21)
        act, lp, _ = api.sample_actions(up(x), up(torch.rand(40, generator=g)), temperature=0.6, top_k=10)
        assert (api.compute_log_probs(up(x), act, temperature=0.6)[0] - lp).abs().max() < 2e-5


# ------------------------------------------------------------------------------------------ attention
class Cache:
    """A paged cache whose unused places hold NaN."""

    def __init__(self, seed, prefix_lens, own_lens, page, Hk, d, layout="tokens", spare=2):
        g = torch.Generator().manual_seed(seed)
        wp = max([-(-n // page) for n in prefix_lens] + [1])
        wo = max([-(-n // page) for n in own_lens] + [1])
        need = sum(-(-n // page) for n in prefix_lens) + sum(-(-n // page) for n in own_lens)
        ids = torch.randperm(need + spare, generator=g).tolist()
        self.k = torch.full((need + spare, page, Hk, d), float("nan"), dtype=BF16)
        self.v = self.k.clone()
        self.prefix_table = torch.full((len(prefix_lens), wp), 2 ** 30, dtype=torch.int32)
        self.own_table = torch.full((len(own_lens), wo), -7, dtype=torch.int32)
        self.keys = {}
        for name, lens, table in (("p", prefix_lens, self.prefix_table), ("o", own_lens, self.own_table)):
            for i, n in enumerate(lens):
                k, v = (torch.randn(n, Hk, d, generator=g).to(BF16) for _ in range(2))
                self.keys[name, i] = k, v
                for j in range(-(-n // page)):
                    table[i, j] = ids.pop()
                    part = k[j * page:(j + 1) * page]
                    self.k[table[i, j], :part.shape[0]] = part
                    self.v[table[i, j], :part.shape[0]] = v[j * page:(j + 1) * page]
        if layout == "heads":                                # [pages, Hk, page, d] in memory
            self.kd, self.vd = (up(t.permute(0, 2, 1, 3).contiguous()).permute(0, 2, 1, 3) for t in (self.k, self.v))
        else:
            self.kd, self.vd = up(self.k), up(self.v)


def plain_attention(q, cache, offsets, scale, n_rows, n_groups):
    B, H, d = q.shape
    Hk = cache.k.shape[2]
    out, lse = torch.zeros(B, H, d, dtype=torch.float64), torch.full((B, H), -math.inf, dtype=torch.float64)
    for b in range(B):
        parts = [cache.keys["p", g] for g in range(n_groups) if offsets[g] <= b < offsets[g + 1]] + [cache.keys["o", b]]
        k = torch.cat([x[0] for x in parts]).double().repeat_interleave(H // Hk, 1)
        v = torch.cat([x[1] for x in parts]).double().repeat_interleave(H // Hk, 1)
        if k.shape[0]:
            c = torch.einsum("hd,lhd->hl", q[b].double(), k) * scale
            lse[b] = torch.logsumexp(c, 1)
            out[b] = torch.einsum("hl,lhd->hd", torch.softmax(c, 1), v)
    return out, lse


def check_attention(api, prefix_lens, sizes, own_lens, H, Hk, d, page, seed=0, layout="tokens", q_pad=0, slack=0, bounds=True, first=0, stream=None):
    cache = Cache(seed, prefix_lens, own_lens, page, Hk, d, layout)
    g = torch.Generator().manual_seed(seed + 1)
    B = len(own_lens)
    q = torch.randn(B, H, d, generator=g).to(BF16)
    offsets = [first]
    for n in sizes:
        offsets.append(offsets[-1] + n)
    scale = 1.7 / math.sqrt(d)
    want, want_lse = plain_attention(q, cache, offsets, scale, B, len(prefix_lens))
    big = torch.full((B, H * d + q_pad), float("nan"), dtype=BF16)
    big[:, :H * d] = q.view(B, -1)
    qd = up(big)[:, :H * d].view(B, H, d) if q_pad == 0 else up(big)[:, :H * d].unflatten(1, (H, d))
    grouped = len(prefix_lens) > 0
    kw = dict(max_prefix_len=max(prefix_lens, default=0) + slack, max_len=max(own_lens) + slack) if bounds else {}
    out, lse = api.shared_prefix_attention(
        qd, cache.kd, cache.vd, up(cache.prefix_table) if grouped else None,
        up(torch.tensor(prefix_lens, dtype=torch.int32)) if grouped else None,
        up(torch.tensor(offsets, dtype=torch.int32)) if grouped else None, up(cache.own_table),
        up(torch.tensor(own_lens, dtype=torch.int32)), scale=scale, stream=stream, **kw)
    if stream is not None:
        stream.synchronize()
    out, lse = out.cpu().double(), lse.cpu().double()
    empty = want_lse == -math.inf
    assert torch.equal(lse == -math.inf, empty) and (out[empty] == 0).all()
    assert ((lse - want_lse)[~empty].abs() <= 1e-5 + 2.0 ** -22 * want_lse[~empty].abs()).all()
    most = max([float(v.abs().max()) for _, v in cache.keys.values() if v.numel()] + [0.0])
    assert ((out - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15 * most).all(), (out - want).abs().max()


@pytest.mark.parametrize("H,Hk,d", [(8, 8, 64), (8, 2, 128), (28, 4, 64), (20, 1, 128), (4, 4, 8), (6, 2, 40), (33, 1, 80), (4, 1, 96)])
@pytest.mark.parametrize("page", [1, 7, 16, 64, 100])
def test_attention_heads_and_pages(api, H, Hk, d, page):
    check_attention(api, [65, 130, 1], [3, 1, 2], [0, 5, 64, 63, 129, 1], H, Hk, d, page, seed=page)


@pytest.mark.parametrize("prefix", [0, 1, 15, 16, 17, 63, 64, 65, 127, 128, 129, 1000, 5000])
@pytest.mark.parametrize("own", [0, 1, 64, 700])
def test_attention_lengths(api, prefix, own):
    check_attention(api, [prefix], [5], [own, 0, own // 2, own, 1], 8, 2, 64, 16, seed=prefix + own)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_many_rows_share_a_prompt(api, d):
    check_attention(api, [700, 90], [70, 30], [(7 * i) % 50 for i in range(100)], 8, 2, d, 32)
    check_attention(api, [3000], [33], [i for i in range(33)], 16, 2, d, 64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 8, 24, 64, 128])
@pytest.mark.parametrize("prefix", [1, 64, 65, 640, 1500])
def test_attention_blocks_of_128_and_256_rows(api, prefix, page, d):
    """One and two row tiles a block, the second one partly filled or empty; pages copied by boxes and piece by piece."""
    check_attention(api, [prefix, max(1, prefix // 2)], [20, 28], [i % 3 for i in range(48)], 4, 1, d, page, seed=prefix)       # 80, 112 rows
    check_attention(api, [prefix, max(1, prefix // 3)], [40, 73], [i % 3 for i in range(113)], 4, 1, d, page, seed=prefix)      # 160, 292 rows


@pytest.mark.parametrize("d", [8, 40, 72, 104])
@pytest.mark.parametrize("page", [16, 48])
def test_attention_many_rows_with_few_dimensions(api, d, page):
    check_attention(api, [200, 77], [30, 9], [i % 7 for i in range(39)], 8, 1, d, page, seed=d)


@pytest.mark.parametrize("page", [16, 48, 64])
@pytest.mark.parametrize("rows", [10, 40])
def test_attention_missing_prefix_pages_of_many_rows(api, rows, page):
    """Pages that are not there in a prefix that 80 and 320 query rows share, whole and partial tiles."""
    n = 5 * page + 3
    cache, cut = (Cache(5, [n], [4] * rows, page, 1, 64) for _ in range(2))
    q = torch.randn(rows, 8, 64, generator=torch.Generator().manual_seed(6)).to(BF16)
    cache.prefix_table[0, 1] = -1
    cache.prefix_table[0, 4] = cache.k.shape[0] + 5
    keep = [i for i in range(n) if i // page not in (1, 4)]
    cut.keys["p", 0] = tuple(t[keep] for t in cut.keys["p", 0])
    want, want_lse = plain_attention(q, cut, [0, rows], 0.125, rows, 1)
    i32 = lambda *v: up(torch.tensor(v, dtype=torch.int32))
    out, lse = api.shared_prefix_attention(up(q), cache.kd, cache.vd, up(cache.prefix_table), i32(n), i32(0, rows), up(cache.own_table), i32(*[4] * rows))
    most = max(float(v.abs().max()) for _, v in cut.keys.values())
    assert ((out.cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -15 * most).all()
    assert ((lse.cpu().double() - want_lse).abs() <= 1e-5 + 2.0 ** -22 * want_lse.abs()).all()


def test_attention_groups_of_any_size_and_rows_outside(api):
    check_attention(api, [40, 0, 33, 70], [0, 4, 1, 0], [3, 1, 0, 9, 12], 8, 4, 64, 16)
    check_attention(api, [40, 33], [2, 2], [3, 1, 0, 9, 12, 0, 5], 8, 4, 64, 16, first=2)      # rows before and after
    check_attention(api, [], [], [3, 1, 0, 9, 200], 8, 4, 128, 16)                             # no prefixes at all


def test_attention_strides_layouts_and_bounds(api):
    check_attention(api, [100, 30], [2, 2], [30, 1, 64, 100], 8, 2, 128, 16, layout="heads")
    check_attention(api, [100, 30], [2, 2], [30, 1, 64, 100], 8, 2, 64, 16, q_pad=24)
    check_attention(api, [100, 30], [2, 2], [30, 1, 64, 100], 8, 2, 64, 16, slack=5000)
    check_attention(api, [100, 30], [2, 2], [30, 1, 64, 100], 8, 2, 64, 16, bounds=False)
    check_attention(api, [100, 30], [2, 2], [30, 1, 64, 100], 8, 2, 64, 16, stream=torch.cuda.Stream())


def test_attention_pages_that_are_not_there(api):
    """A page number outside the cache holds no keys: as if the tokens of that page were left out."""
    cache = Cache(5, [64], [48, 48], 16, 2, 64)
    cut = Cache(5, [64], [48, 48], 16, 2, 64)
    q = torch.randn(2, 4, 64, generator=torch.Generator().manual_seed(6)).to(BF16)
    cache.prefix_table[0, 1] = -1
    cache.own_table[1, 0] = cache.k.shape[0]
    cache.own_table[0, :] = torch.iinfo(torch.int32).min
    drop = lambda kv, a, b: tuple(torch.cat([t[:a], t[b:]]) for t in kv)
    cut.keys["p", 0] = drop(cut.keys["p", 0], 16, 32)
    cut.keys["o", 1] = drop(cut.keys["o", 1], 0, 16)
    cut.keys["o", 0] = drop(cut.keys["o", 0], 0, 48)
    want, want_lse = plain_attention(q, cut, [0, 2], 0.125, 2, 1)
    i32 = lambda *v: up(torch.tensor(v, dtype=torch.int32))
    out, lse = api.shared_prefix_attention(up(q), cache.kd, cache.vd, up(cache.prefix_table), i32(64), i32(0, 2), up(cache.own_table), i32(48, 48))
    assert (out.cpu().double() - want).abs().max() < 2e-2 and (lse.cpu().double() - want_lse).abs().max() < 1e-4


def test_attention_large_scores_and_one_key_wins(api):
    cache = Cache(7, [200], [90], 16, 1, 64)
    q = (torch.randn(1, 2, 64, generator=torch.Generator().manual_seed(1)) * 60).to(BF16)
    want, want_lse = plain_attention(q, cache, [0, 1], 1.0, 1, 1)
    i32 = lambda *v: up(torch.tensor(v, dtype=torch.int32))
    out, lse = api.shared_prefix_attention(up(q), cache.kd, cache.vd, up(cache.prefix_table), i32(200), i32(0, 1), up(cache.own_table), i32(90), scale=1.0)
    # scores of thousands are themselves off by their fp32 rounding
    assert ((lse.cpu().double() - want_lse).abs() <= 2.0 ** -21 * want_lse.abs()).all()
    assert (out.cpu().double() - want).abs().max() < 2.0 ** -6


def test_attention_offsets_past_32_bits(api):
    """Pages whose elements lie beyond 2^32 of the cache's start."""
    d, Hk, page = 64, 1, 16
    stride = 1 << 22                                         # elements between pages: page 1040 starts past 2^32
    flat = torch.zeros((1041 << 22) + page * d, dtype=BF16, device="cuda")
    k = flat.as_strided((1042, page, Hk, d), (stride, d, d, 1))
    g = torch.Generator().manual_seed(0)
    content = torch.randn(page, Hk, d, generator=g).to(BF16)
    k[1040] = content.cuda()
    k[3] = torch.randn(page, Hk, d, generator=g).to(BF16).cuda()
    q = torch.randn(1, 2, d, generator=g).to(BF16)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    for table in ((None, None, None, i32(1040).view(1, 1), i32(page)), (i32(1040).view(1, 1), i32(page), i32(0, 1), i32(3).view(1, 1), i32(0))):
        out, lse = api.shared_prefix_attention(q.cuda(), k, k, *table, scale=0.1)
        c = torch.einsum("hd,ld->hl", q[0].double(), content[:, 0].double()) * 0.1
        want = torch.softmax(c, 1) @ content[:, 0].double()
        assert (out[0].cpu().double() - want).abs().max() < 2e-2 and (lse[0].cpu().double() - torch.logsumexp(c, 1)).abs().max() < 1e-4


# ------------------------------------------------------------------------------------------ block tables
def plain_tables(cached, added, free, table, page, n):
    table, B, width = table.copy(), *table.shape
    slots, positions = np.full(n, -1, np.int64), np.full(n, -1, np.int32)
    offsets, pages = np.zeros(B + 1, np.int32), np.zeros(B + 1, np.int32)
    t = used = 0
    for b in range(B):
        c, a = max(int(cached[b]), 0), max(int(added[b]), 0)
        have, need = min(-(-c // page), width), min(-(-(c + a) // page), width)
        for j in range(have, width):
            table[b, j] = -1
            if j < need:
                table[b, j] = free[used] if used < len(free) else -1
                used += 1
        for i in range(a):
            if t < n:
                j = (c + i) // page
                positions[t] = c + i
                if j < width and table[b, j] >= 0:
                    slots[t] = int(table[b, j]) * page + (c + i) % page
            t += 1
        offsets[b + 1], pages[b + 1] = t, used
    return slots, positions, offsets, pages, table


def check_tables(cached, added, page, width, free_count, n, seed=0):
    from paper_2608_17641_b200 import binding
    g = np.random.RandomState(seed)
    B = len(cached)
    table = g.randint(0, 1000, (B, width)).astype(np.int32)
    free = (g.permutation(free_count) + 5000).astype(np.int32)
    cached, added = np.array(cached, np.int32), np.array(added, np.int32)
    want = plain_tables(cached, added, free, table, page, n)
    td = guarded_upload(table)
    got = binding.rlcs_block_tables(guarded_upload(cached), guarded_upload(added), guarded_upload(free), td, page_size=page, num_slots=n)
    for a, b in zip((*got, td), want):
        assert a.cpu().numpy().dtype == b.dtype and np.array_equal(a.cpu().numpy(), b)


@pytest.mark.parametrize("B", [1, 2, 31, 33, 256, 1000, 1025, 3000, 9001])
@pytest.mark.parametrize("page", [1, 16, 100])
def test_tables_sizes(B, page):
    g = np.random.RandomState(B + page)
    cached, added = g.randint(0, 150, B), g.randint(0, 40, B)
    need = int((-(-(cached + added) // page) + (cached // -page)).sum())
    total, width = int(added.sum()), -(-190 // page)
    check_tables(cached, added, page, width, need + 3, total)
    check_tables(cached, np.ones(B, int), page, width, B, B)
    check_tables(np.zeros(B, int), added, page, width, int((-(-added // page)).sum()), total + 5)


def test_tables_edges():
    check_tables([], [], 16, 4, 3, 2)                                     # no rows
    check_tables([0, 0, 0], [0, 0, 0], 16, 2, 4, 0)                       # nothing to do
    check_tables([0, 0, 7, 0], [0, 5, 0, 0], 16, 2, 4, 9)                 # empty rows around
    check_tables([5, 30, 2], [40, 40, 1], 16, 3, 2, 81)                   # the list runs out
    check_tables([5, 30, 2], [40, 40, 1], 16, 3, 0, 81)                   # there is no list
    check_tables([100, 3], [50, 90], 16, 4, 20, 140)                      # longer than the table is wide
    check_tables([-4, 3], [6, -9], 16, 4, 20, 6)                          # negative lengths
    check_tables([15, 16, 17], [1, 1, 1], 16, 4, 4, 3)                    # page boundaries
    check_tables([3, 9], [6, 8], 16, 4, 20, 5)                            # more tokens than slots
    check_tables([3, 9], [6, 8], 16, 0, 20, 14)                           # no table


def test_tables_repeat_is_the_same_and_large_pages():
    from paper_2608_17641_b200 import binding
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    table = i32(3, -1, -1, 4, -1, -1).view(2, 3)
    free = i32(2 ** 31 - 1, 9)
    args = dict(page_size=1 << 20, num_slots=4)
    one = binding.rlcs_block_tables(i32(1 << 20, 5), i32(3, 1), free, table, **args)
    first = table.clone()
    two = binding.rlcs_block_tables(i32(1 << 20, 5), i32(3, 1), free, table, **args)
    assert torch.equal(first, table)
    for a, b in zip(one, two):
        assert torch.equal(a, b)
    base = (2 ** 31 - 1) << 20
    assert one[0].tolist() == [base, base + 1, base + 2, (4 << 20) + 5]       # slots past 32 bits


# ------------------------------------------------------------------------------------------ together
def test_operators_work_together_in_the_example():
    """The example's policy acts, is credited and learns: its reward rises well above chance (one in six), the same on a second run."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "token_rollout.py")
    spec = importlib.util.spec_from_file_location("token_rollout", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history = example.train(iterations=25, say=None)
    assert abs(history[0] - 1 / 6) < 0.08 and sum(history[-3:]) / 3 > 0.4, history
    assert example.train(iterations=3, say=None) == history[:3]


def test_outputs_belong_to_the_stream_that_writes_them(api):
    """A call on a side stream, right behind a long pending use of freed memory on the current one: its outputs must not lie there."""
    from paper_2608_17641_b200 import binding
    plain = binding._alloc
    binding._alloc = lambda shape, dtype, device: torch.empty(shape, dtype=dtype, device="cuda")
    try:
        g = torch.Generator(device="cuda").manual_seed(0)
        x = torch.randn(64, 4000, device="cuda", generator=g)
        a = torch.randint(0, 4000, (64,), device="cuda", generator=g, dtype=torch.int32)
        adv = torch.randn(64, device="cuda", generator=g)
        want = [v.clone() for v in api.compute_policy_gradient(x, a, adv)]
        big = torch.randn(6000, 6000, device="cuda", generator=g)
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        for _ in range(3):
            gone = torch.empty(64, 4000, device="cuda")
            for _ in range(4):
                big @ big                                     # keeps the current stream busy
            gone.fill_(7.0)                                   # pending when its memory is given back
            del gone
            got = api.compute_policy_gradient(x, a, adv, stream=side)
            torch.cuda.synchronize()
            for v, w in zip(got, want):
                assert torch.equal(v, w)
    finally:
        binding._alloc = plain


def test_operators_in_a_graph(api):
    """Captured with caller-owned outputs and workspace, replayed on new inputs in the same buffers."""
    from paper_2608_17641_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(7, 5000, device="cuda", generator=g).bfloat16()
    u, adv = torch.rand(7, device="cuda", generator=g), torch.randn(7, device="cuda", generator=g)

    def work():
        a, lp, kp = api.sample_actions(x, u, top_k=30, top_p=0.9)
        return (a, lp, kp, *api.compute_policy_gradient(x, a, adv, entropy_coef=0.1))

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        work()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    plain = binding._alloc
    binding._alloc = lambda shape, dtype, device: torch.empty(shape, dtype=dtype, device="cuda")      # guard bands are filled outside a capture only
    try:
        with torch.cuda.graph(graph):
            out = work()
    finally:
        binding._alloc = plain
    for seed in (1, 2):
        x.copy_(torch.randn(7, 5000, device="cuda", generator=g))
        u.copy_(torch.rand(7, device="cuda", generator=g))
        graph.replay()
        for got, want in zip(out, work()):
            assert torch.equal(got, want)
