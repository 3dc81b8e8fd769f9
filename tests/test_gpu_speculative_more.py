"""Operators of speculative rollouts and distillation on the GPU: what a call's company must not change, pages shared by cut-back branches,
and rows and weights at the edges of what the formulas say.

Tolerances count roundings: a bfloat16 result is off by at most 2^-8 of its value (half a step), a fp32 one by 2^-24."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _util import guarded_empty  # noqa: E402
from test_gpu_operators import BF16, F32, up  # noqa: E402
from test_gpu_speculative import I32, Paged, api, check_verify, ints, plain_chunks, plain_weights, verify_inputs  # noqa: E402,F401


# ------------------------------------------------------------------------------------------ attention of chunks
@pytest.mark.parametrize("H,Hk,d,page", [(8, 2, 128, 64), (14, 2, 64, 16), (4, 4, 64, 24), (6, 2, 40, 128)])
def test_chunk_weights_keep_sixteen_bits_whatever_else_is_in_the_step(api, H, Hk, d, page):
    """The same tokens alone, under close bounds, and in a step of long tables and long chunks: tiles of 16 rows and blocks of 128.  Softmax
    weights as two bfloat16 parts are off by 2^-16 of themselves, scores (up to 30) by 2^-17: the output by 2^-15 sum_j p_j |v_j|, by 2^-15
    of the largest |v| for the sums, and by half a step of its own."""
    lens, counts = [300, 650, 410], [2, 300, 77]
    cache = Paged(d + page, lens, page, Hk, d)
    offsets = [0, 2, 302, 379]
    q = torch.randn(379, H, d, generator=torch.Generator().manual_seed(7)).to(BF16)
    scale = 1.7 / math.sqrt(d)
    want, want_lse, size = plain_chunks(q, cache.keys, lens, offsets, scale, max(lens))
    most = max(float(v.abs().max()) for _, v in cache.keys)
    wide = torch.cat([cache.table, torch.full((3, -(-1000 // page)), -1, dtype=I32)], 1)
    together = api.chunk_attention(up(q), cache.kd, cache.vd, up(wide), up(ints(offsets)), up(ints(lens)), scale=scale)
    alone = api.chunk_attention(up(q[:2]), cache.kd, cache.vd, up(cache.table[:1].contiguous()), up(ints([0, 2])), up(ints(lens[:1])), scale=scale,
                                max_new=2, max_len=300)
    for (out, lse), n in ((together, 379), (alone, 2)):
        out, lse = out.cpu().double(), lse.cpu().double()
        assert ((lse - want_lse[:n]).abs() <= 1e-5 + 2.0 ** -22 * want_lse[:n].abs()).all()
        err = (out - want[:n]).abs() - 2.0 ** -8 * want[:n].abs() - 2.0 ** -15 * (size[:n] + most)
        assert (err <= 0).all(), err.max()


# ------------------------------------------------------------------------------------------ pages
def plain_fork_by_page(table, lens, sources, free, page):
    """A part-filled page belongs to the first new row that ends in it, and to none where a new row has it whole."""
    B, width = table.shape
    rows, ends, whole, first = [], [], set(), {}
    for i, s in enumerate(sources):
        row, end = [-1] * width, -1
        if 0 <= s < B:
            n = max(int(lens[s]), 0)
            need = -(-n // page)
            row[:min(need, width)] = [int(v) for v in table[s, :min(need, width)]]
            whole.update(row[:min(n // page, width)])
            if n % page and need <= width and row[need - 1] >= 0:
                end = need - 1
                first.setdefault(row[end], i)
        rows.append(row), ends.append(end)
    come, go, used = [-1] * len(rows), [-1] * len(rows), 0
    for i, (row, end) in enumerate(zip(rows, ends)):
        if end >= 0 and (row[end] in whole or first[row[end]] != i):
            new = max(int(free[used]), -1) if used < len(free) else -1
            come[i], go[i], row[end] = (row[end] if new >= 0 else -1), new, new
            used += 1
    return rows, come, go, used


@pytest.mark.parametrize("B,N,width", [(1, 3, 4), (5, 9, 3), (40, 40, 7), (300, 200, 20), (1000, 1500, 33), (4096, 4096, 9), (700, 5000, 6), (6000, 6000, 5), (5000, 3, 4),
                                       (2048, 3001, 40), (4096, 4096, 26), (3, 13, 9000), (4000, 5, 26)])
def test_fork_goes_by_the_page_that_is_shared(api, B, N, width):
    """Tables whose rows share pages with one another at any place, as whole pages, as part-filled ones and as both."""
    page = 16
    g = torch.Generator().manual_seed(B + N)
    table = torch.randperm(4 * B * width, generator=g)[:B * width].to(I32).view(B, width)
    like = torch.randint(0, B, (B,), generator=g)
    upto = torch.randint(0, width + 1, (B,), generator=g)
    for _ in range(2):                                                 # branches, and branches of branches
        table = torch.where(torch.arange(width)[None] < upto[:, None], table[like], table)
    some = torch.rand(B, generator=g) < 0.1                            # and pages at another place than their owner's
    table[some, width - 1] = table[like[some], 0]
    lens = torch.randint(0, width * page + 20, (B,), generator=g, dtype=I32)
    sources = torch.randint(-1, B + 1, (N,), generator=g, dtype=I32)
    if N == B:
        sources = torch.arange(B, dtype=I32)                           # every row continues itself
    for free in (torch.arange(4 * B * width, 4 * B * width + N, dtype=I32), torch.arange(4 * B * width, 4 * B * width + N // 4, dtype=I32)):
        want = plain_fork_by_page(table, lens.tolist(), sources.tolist(), free.tolist(), page)
        got = api.fork_block_tables(up(table), up(lens), up(sources), up(free), page_size=page)
        for a, b in zip(got, want[:3] + ([want[3]],)):
            assert torch.equal(a.cpu(), torch.tensor(b, dtype=I32).view(a.shape))
        # with pages enough nobody can write into what another row has
        if N == len(free):
            ends = {}
            new = got[0].tolist()
            for i, s in enumerate(sources.tolist()):
                n = max(int(lens[s]), 0) if 0 <= s < B else 0
                if n % page and -(-n // page) <= width:
                    ends[i] = new[i][n // page]
            for i, s in enumerate(sources.tolist()):
                n = max(int(lens[s]), 0) if 0 <= s < B else 0
                for j, p in enumerate(new[i][:min(-(-n // page), width)]):
                    new[i][j] = (p, j == n // page)
            owners = {}
            for i, p in ends.items():
                assert owners.setdefault(p, i) == i                    # one row a part-filled page
            assert not any(p in owners and not last for row in new for p, last in (v for v in row if isinstance(v, tuple)))


def test_branches_cut_back_into_a_shared_page_grow_apart(api):
    """Fork, lower both branches into a page that they share, fork again, add tokens: every row keeps its own keys."""
    page, width, Hk, d = 16, 6, 1, 64
    pages = 40
    k = torch.zeros(pages, page, Hk, d, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    table = torch.full((4, width), -1, dtype=I32, device="cuda")
    lens = torch.zeros(4, dtype=I32, device="cuda")
    texts = [[] for _ in range(4)]                                     # a number a token

    def add(counts, values):
        nonlocal lens
        free, _ = api.list_free_pages(table, lens, num_pages=pages, page_size=page)
        slots, _, _, _ = api.build_block_tables(lens, up(ints(counts)), free, table, page_size=page, num_slots=sum(counts))
        assert len(set(slots.tolist())) == sum(counts)                 # no two tokens in one place
        k.view(-1, Hk, d)[slots] = up(torch.tensor(values, dtype=F32).to(BF16))[:, None, None].expand(-1, Hk, d)
        v.view(-1, Hk, d)[slots] = -k.view(-1, Hk, d)[slots]
        lens = lens + up(ints(counts))
        at = 0
        for b, n in enumerate(counts):
            texts[b] = texts[b] + values[at:at + n]
            at += n

    def cut(to):
        nonlocal lens
        lens = torch.minimum(lens, up(ints(to)))
        for b, n in enumerate(to):
            texts[b] = texts[b][:n]

    def fork(sources):
        nonlocal table, lens, texts
        free, _ = api.list_free_pages(table, lens, num_pages=pages, page_size=page)
        table, come, go, _ = api.fork_block_tables(table, lens, up(ints(sources)), free, page_size=page)
        api.copy_pages(k, v, come, go)
        lens, texts = lens[up(ints(sources)).long()], [list(texts[s]) for s in sources]
        return [c for c in come.tolist() if c >= 0]

    def check():
        for b, text in enumerate(texts):
            assert int(lens[b]) == len(text)
            at = [int(table[b, i // page]) * page + i % page for i in range(len(text))]
            assert k.view(-1, d)[at, 0].tolist() == text and (v.view(-1, d)[at, 0] == -k.view(-1, d)[at, 0]).all()

    add([40, 3, 0, 0], [float(i) for i in range(43)])
    fork([0, 0, 0, 1])                                                 # three rows of 40, one of 3
    check()
    cut([20, 24, 40, 3])                                               # two end in the second page, which the third has whole
    assert len(fork([0, 1, 2, 3])) == 2
    check()
    add([15, 9, 5, 20], [float(100 + i) for i in range(49)])
    check()
    fork([0, 0, 1, 2])
    cut([25, 22, 30, 35])                                              # two end in a page that nobody has whole, one of them may stay
    assert len(fork([0, 1, 2, 3])) == 1
    add([20, 20, 7, 2], [float(160 + i) for i in range(49)])
    check()


def test_fork_of_no_rows_into_many(api):
    new, come, go, used = api.fork_block_tables(torch.zeros(0, 3, dtype=I32, device="cuda"), up(ints([])), up(torch.zeros(20000, dtype=I32)), up(ints([1])),
                                                page_size=16)
    assert (new == -1).all() and new.shape == (20000, 3) and (come == -1).all() and (go == -1).all() and used.tolist() == [0]


def test_fork_captured_twice_and_replayed(api):
    """Two graphs of forks of more rows than one block holds share nothing."""
    g = torch.Generator().manual_seed(1)
    graphs = []
    for n in (300, 5000):
        table, lens = up(torch.randperm(4 * n, generator=g).to(I32).view(n, 4)), up(torch.randint(0, 65, (n,), generator=g, dtype=I32))
        sources, free = up(torch.randint(0, n, (n,), generator=g, dtype=I32)), up(torch.arange(4 * n, 5 * n, dtype=I32))
        api.fork_block_tables(table, lens, sources, free, page_size=16)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = api.fork_block_tables(table, lens, sources, free, page_size=16)
        graphs.append((graph, got, (table, lens, sources, free)))
    for _ in range(2):
        for _, _, (table, lens, sources, free) in graphs:
            lens.copy_(torch.randint(0, 65, lens.shape, generator=g, dtype=I32))
        for graph, _, _ in graphs:
            graph.replay()
        for _, got, (table, lens, sources, free) in graphs:
            for a, b in zip(got, api.fork_block_tables(table, lens, sources, free, page_size=16)):
                assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------ distillation
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A,K,times", [(3, 2, 1), (18, 5, 40), (100, 40, 1), (700, 20, 1), (1500, 300, 1), (6000, 9, 70), (6000, 9, 1), (70001, 33, 1), (600000, 4, 1)])
def test_distill_gradient_of_excluded_logits_is_the_formulas(api, A, K, times, dtype):
    """Logits of -inf, named by the teacher (once, twice, with no probability) and not: scale / T (0 - sum p), to a rounding of p and the
    result's own; in short rows, rows of a block, and rows of a cluster."""
    g = torch.Generator().manual_seed(A)
    R, T, scale = 6, 1.3, 0.7
    x = (torch.randn(R, A, generator=g) * 2).to(dtype)
    ids = torch.stack([torch.randperm(A, generator=g)[:K] for _ in range(R)]).to(I32)
    teacher = torch.randn(R, K, generator=g)
    other = torch.rand(R, A, generator=g) < 0.3
    other.scatter_(1, ids.long(), False)
    x[other] = -math.inf
    for r in range(R):
        x[r, ids[r, r % K].long()] = -math.inf
    ids[3, 1] = ids[3, 0]
    x[3, ids[3, 0].long()] = -math.inf
    teacher[4, 4 % K] = -math.inf                                      # named, but with no probability
    if A == 3:
        x[:, [a for a in range(3) if a not in ids[0].tolist()]] = 0.5
    some = (x > -math.inf).any(1)
    p = torch.softmax(teacher.double() / T, 1)
    dense = torch.zeros(R, A, dtype=torch.float64).scatter_add_(1, ids.long(), p)
    want = scale / T * (torch.softmax(x.double() / T, 1) - dense)
    loss, grad = api.compute_distillation(up(x.repeat(times, 1)), up(ids.repeat(times, 1)), up(teacher.repeat(times, 1)), temperature=T, scale=scale)
    loss, grad = loss.cpu().view(times, R), grad.cpu().double().view(times, R, A)
    out = (x == -math.inf) & some[:, None]
    assert (grad[:, out & (dense == 0)] == 0).all()
    bound = (1e-5 + (2.0 ** -8 if dtype == BF16 else 2.0 ** -22)) * want.abs()
    assert ((grad - want)[:, out].abs() <= bound[out]).all()
    named = out & (dense > 0)
    assert torch.equal(loss[0] == math.inf, named.any(1)) and (loss == loss[0]).all()


# ------------------------------------------------------------------------------------------ verification
def nearest(n, d):
    """n / d (whole numbers) rounded to 53 bits, ties to even, as a fraction of whole numbers: by long division alone."""
    if n == 0:
        return 0, 1
    down = n.bit_length() - d.bit_length() - 54                        # the quotient has 54 or 55 bits
    q, rest = divmod(n << max(-down, 0), d << max(down, 0))
    over = q.bit_length() - 53
    low, q = q & ((1 << over) - 1), q >> over
    half = 1 << (over - 1)
    if low > half or (low == half and (rest or q & 1)):
        q += 1
    return (q << max(down + over, 0)), (1 << max(-down - over, 0))


def test_nearest_is_what_it_says():
    for n, d in ((2 ** 40, 3), (2 ** 40, 5071373719), (1, 7), (2 ** 60 + 1, 1), (2 ** 54 + 2, 1), (2 ** 54 + 6, 1), (10 ** 18 + 1, 10 ** 3)):
        a, b = nearest(n, d)
        assert a / b == n / d


def shares(weights, total, rounded):
    """Shares of 2^40: the header's (quotient and product rounded) or the exact floors."""
    if not rounded:
        return [w * 2 ** 40 // total for w in weights]
    a, b = nearest(2 ** 40, total)
    return [n // d for n, d in (nearest(w * a, b) for w in weights)]


def test_verify_difference_is_rounded_as_the_header_says(api):
    """Rows where the header's shares draw another token than exact floors would: a draft policy with one more, weak entry, so that the
    difference is a few thousand units in which every single one can be drawn."""
    g = torch.Generator().manual_seed(11)
    R, A = 60000, 8
    x = -torch.rand(R, A, generator=g)
    x[:, 0] = 0.0
    drafts = x.clone()
    x[:, 7], drafts[:, 7] = -math.inf, -16.0 - torch.rand(R, generator=g)
    weights = [(torch.exp(up(v)).cpu().double() * 2.0 ** 31 + 0.5).floor().long().tolist() for v in (x, drafts)]
    rows, u, want, other = [], [], [], []
    for r, (w, v) in enumerate(zip(*weights)):
        sums = []
        for rounded in (True, False):
            left = [max(0, a - b) for a, b in zip(shares(w, sum(w), rounded), shares(v, sum(v), rounded))]
            sums.append([sum(left[:j + 1]) for j in range(A)])
        if sums[0] == sums[1] or not 0 < sums[0][-1] < 2 ** 20:
            continue
        draw = lambda s, c: next(j for j in range(A) if s[j] > math.floor(c * s[-1]))
        for j in range(A - 1):                                         # uniforms on both sides of every border
            for at in (sums[0][j] - 0.5, sums[0][j] + 0.5):
                c = float(torch.tensor(at / sums[0][-1], dtype=F32))
                if 0 <= c < 1 and draw(sums[0], c) != draw(sums[1], c):
                    rows.append(r), u.append(c), want.append(draw(sums[0], c)), other.append(draw(sums[1], c))
    assert len(rows) >= 5
    n = len(rows)
    pick = torch.tensor(rows).repeat_interleave(2)                     # a draft of entry 7, which the target never takes, and the last row
    tokens = ints([0, 7] * n)
    out, _, acc = api.verify_drafts(up(x[pick]), up(tokens), up(ints(list(range(0, 2 * n + 1, 2)))), up(torch.full((2 * n,), 0.5)),
                                    up(torch.tensor(u, dtype=F32)), draft_logits=up(drafts[pick]))
    assert (acc == 0).all() and out[::2].tolist() == want and want != other


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_verify_log_probs_of_rows_that_keep_rising(api, dtype):
    """Rows whose maximum rises with every load of every thread, by steps of 1e-8 to 0.01 (bfloat16: powers of two): 1e-5 and 2^-22 of the value."""
    R, A = 300, 1 << 22
    each = 4096 if dtype == F32 else 8192
    place = torch.arange(A, device="cuda") // each
    rise = 1e-8 * 1.047 ** torch.arange(R, device="cuda") if dtype == F32 else 2.0 ** -(4 + torch.arange(R, device="cuda") % 4).float()
    x = (place[None] * rise[:, None]).to(dtype)
    g = torch.Generator(device="cuda").manual_seed(2)
    du = torch.rand(R, device="cuda", generator=g)
    out, lp, acc = api.verify_drafts(x, torch.zeros(R, dtype=I32, device="cuda"), torch.arange(R + 1, dtype=I32, device="cuda"), torch.zeros(R, device="cuda"), du)
    for r in range(R):
        want = torch.log_softmax(x[r].double(), 0)[out[r].long()]
        assert abs(float(lp[r] - want)) <= 1e-5 + 2.0 ** -22 * abs(float(want)), (r, float(lp[r] - want))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A,top", [(20000, 3.0), (70003, 30.0)])
def test_verify_uniforms_at_the_border_of_rising_rows(api, A, top, dtype):
    x, tokens, offsets, u, du, drafts = verify_inputs([3, 2], A, dtype, A, near=0.1)
    x = (x.float() * 0.02 + torch.linspace(0, top, A)).to(dtype)
    drafts = (drafts.float() * 0.02 + torch.linspace(0, top, A)).to(dtype)
    tokens[1:] = torch.tensor([A - 5, A // 2 + A // 3, A - 100, A - 1], dtype=I32)
    for drawn in (True, False):
        for step in (-1, 0, 1):
            for t in range(len(u) - 1):
                w, v = plain_weights(x[t], 1.0)[0], plain_weights(drafts[t], 1.0)[0]
                tok = int(tokens[t + 1])
                at = w[tok] * sum(v) / max(1, v[tok] * sum(w)) if drawn else w[tok] / sum(w)
                edge = np.float32(min(at, 1 - 2.0 ** -24))
                if step:
                    edge = np.nextafter(edge, np.float32(step * 2))
                u[t] = min(float(edge), 1 - 2.0 ** -24)
            check_verify(api, x, tokens, offsets, u, du, drafts if drawn else None)


def test_verify_follows_a_filtered_target(api):
    """Drafts drawn with top_k, both policies' rows -inf outside it: tokens follow the filtered target, five standard deviations."""
    B, A, K = 40000, 9, 3
    g = torch.Generator(device="cuda").manual_seed(6)
    rand = lambda n: torch.rand(n, device="cuda", generator=g)
    p, q = torch.randn(A, device="cuda", generator=g) * 1.5, torch.randn(A, device="cuda", generator=g) * 1.5
    p_kept, q_kept = (v.masked_fill(v < v.topk(K).values[-1], -math.inf) for v in (p, q))
    tokens, _, kept = api.sample_actions(q.repeat(2 * B, 1), rand(2 * B), top_k=K)
    assert (kept - torch.log_softmax(q_kept, 0)[tokens.long()]).abs().max() < 1e-5
    out, lp, acc = api.verify_drafts(p_kept.repeat(2 * B, 1), tokens, torch.arange(0, 2 * B + 1, 2, device="cuda", dtype=I32), rand(2 * B), rand(B),
                                     draft_logits=q_kept.repeat(2 * B, 1))
    want = torch.softmax(p_kept, 0)
    share = torch.bincount(out[::2].long(), minlength=A) / B
    assert ((share - want).abs() <= 5 * (want * (1 - want) / B).sqrt()).all()
    keep = float(torch.minimum(want, torch.softmax(q_kept, 0)).sum())
    assert abs(float(acc.float().mean()) - keep) <= 5 * math.sqrt(keep * (1 - keep) / B)
    assert (lp[::2] - torch.log(want)[out[::2].long()]).abs().max() < 1e-5
