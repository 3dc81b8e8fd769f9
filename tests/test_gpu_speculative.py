"""Operators of speculative rollouts and distillation on the GPU against plain 64-bit implementations: attention of chunks over a
paged cache, verification of drafts, distillation, and the pages of a cache.

Tolerances.  Attention: the output's own rounding is half a last place, 2^-8 of its value; the weights enter the second product
as bfloat16, each off by at most 2^-8 of itself, which moves the output by at most 2^-8 sum_j p_j |v_j|; scores of up to 30 are
off by 30 * 2^-22, below 2^-15 of the largest |v|.  lse: 1e-5 for the same scores, 2^-22 of the value for its rounding.
Log-probabilities and losses: fp32 logits scaled by 1/T carry 2^-23, a difference d <= 30 to the maximum is off by 2^-22 |d|,
hence 1e-5, and 2^-22 of the value.  Gradients: probabilities are off by 1e-5 of their value, 30 * 2^-22; bfloat16 results add 2^-8 of the value."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _util import guarded_empty, guarded_upload  # noqa: E402
from test_gpu_operators import BF16, F32, strided_rows, up  # noqa: E402

I32 = torch.int32


@pytest.fixture(scope="module")
def api():
    from paper_2608_17641_b200 import api as a
    return a


def ints(values):
    return torch.tensor(values, dtype=I32)


# ------------------------------------------------------------------------------------------ attention of chunks
class Paged:
    """Trajectories in a paged cache whose unused places hold NaN."""

    def __init__(self, seed, lens, page, Hk, d, layout="tokens", spare=2):
        g = torch.Generator().manual_seed(seed)
        need = sum(-(-n // page) for n in lens)
        ids = torch.randperm(need + spare, generator=g).tolist()
        self.k = torch.full((need + spare, page, Hk, d), float("nan"), dtype=BF16)
        self.v = self.k.clone()
        self.table = torch.full((len(lens), max([-(-n // page) for n in lens] + [1])), 2 ** 30, dtype=I32)
        self.keys = []
        for i, n in enumerate(lens):
            k, v = (torch.randn(n, Hk, d, generator=g).to(BF16) for _ in range(2))
            self.keys.append([k, v])
            for j in range(-(-n // page)):
                self.table[i, j] = at = ids.pop()
                part = slice(j * page, (j + 1) * page)
                self.k[at, :k[part].shape[0]], self.v[at, :k[part].shape[0]] = k[part], v[part]
        if layout == "heads":                                # [pages, Hk, page, d] in memory
            self.kd, self.vd = (up(t.permute(0, 2, 1, 3).contiguous()).permute(0, 2, 1, 3) for t in (self.k, self.v))
        else:
            self.kd, self.vd = up(self.k), up(self.v)


def plain_chunks(q, keys, lens, offsets, scale, max_len, missing=None):
    """out, lse and the sum of p |v| of every token; NaN where no trajectory has the token."""
    T, H, d = q.shape
    out, lse, size = torch.full((T, H, d), math.nan, dtype=torch.float64), torch.full((T, H), math.nan, dtype=torch.float64), None
    size = torch.zeros_like(out)
    for b, (k, v) in enumerate(keys):
        r = H // k.shape[1]
        kd, vd = (x.double().repeat_interleave(r, 1) for x in (k, v))
        n = offsets[b + 1] - offsets[b]
        seen = torch.arange(k.shape[0])[None, :] <= torch.arange(lens[b] - n, lens[b])[:, None]
        seen &= torch.arange(k.shape[0])[None, :] < max_len
        if missing is not None:
            seen &= ~missing[b][None, :k.shape[0]]
        rows = slice(offsets[b], offsets[b + 1])
        c = torch.einsum("thd,lhd->thl", q[rows].double(), kd) * scale
        c = c.masked_fill(~seen[:, None, :], -math.inf)
        top = torch.logsumexp(c, 2) if k.shape[0] else torch.full((n, H), -math.inf, dtype=torch.float64)
        p = torch.where(top[..., None] == -math.inf, 0.0, torch.exp(c - top[..., None]))
        lse[rows], out[rows], size[rows] = top, torch.einsum("thl,lhd->thd", p, vd), torch.einsum("thl,lhd->thd", p, vd.abs())
    return out, lse, size


def compare_chunks(got, lse, want, want_lse, size, most):
    got, lse = got.cpu().double(), lse.cpu().double()
    there = ~torch.isnan(want_lse)
    assert (got[~there] == 123).all() and (lse[~there] == 123).all()            # left as they were
    empty = want_lse == -math.inf
    assert torch.equal(lse[there] == -math.inf, empty[there]) and (got[empty] == 0).all()
    some = there & ~empty
    assert ((lse - want_lse)[some].abs() <= 1e-5 + 2.0 ** -22 * want_lse[some].abs()).all(), (lse - want_lse)[some].abs().max()
    err = (got - want)[some].abs() - 2.0 ** -8 * (want[some].abs() + size[some]) - 2.0 ** -15 * most
    assert not torch.isnan(got[some]).any() and (err <= 0).all(), err.max()


def check_chunks(lens, counts, H, Hk, d, page, seed=0, layout="tokens", q_pad=0, first=0, behind=0, bounds=True, cut=None, width=0, factor=1.0,
                 stream=None):
    from paper_2608_17641_b200 import binding
    cache = Paged(seed, lens, page, Hk, d, layout)
    g = torch.Generator().manual_seed(seed + 1)
    offsets = [first]
    for n in counts:
        offsets.append(offsets[-1] + n)
    T = offsets[-1] + behind
    q = (torch.randn(T, H, d, generator=g) * factor).to(BF16)
    scale = 1.7 / math.sqrt(d)
    max_len = max(lens + [0]) if cut is None else cut
    want, want_lse, size = plain_chunks(q, cache.keys, lens, offsets, scale, max_len)
    big = torch.full((T, H * d + q_pad), float("nan"), dtype=BF16)
    big[:, :H * d] = q.view(T, -1)
    qd = up(big)[:, :H * d].unflatten(1, (H, d))
    out, lse = guarded_empty((T, H, d), BF16).fill_(123), guarded_empty((T, H), F32).fill_(123)
    table = cache.table
    if width:
        table = torch.cat([table, torch.full((len(lens), width), 2 ** 30, dtype=I32)], 1)
    kw = dict(max_new=max(counts + [0]), max_len=max_len) if bounds else {} if cut is None else dict(max_len=cut)
    got = binding.rlcs_chunk_attention_bf16(qd, cache.kd, cache.vd, up(table), up(ints(offsets)), up(ints(lens)), scale=scale, out=out, lse=lse,
                                            stream=stream, **kw)
    if stream is not None:
        stream.synchronize()
    assert got[0] is out and got[1] is lse
    compare_chunks(out, lse, want, want_lse, size, max([float(v.abs().max()) for _, v in cache.keys if v.numel()] + [0.0]))


@pytest.mark.parametrize("H,Hk,d", [(8, 8, 64), (8, 2, 128), (28, 4, 64), (20, 1, 128), (4, 4, 8), (6, 2, 40), (33, 1, 80), (4, 1, 96)])
@pytest.mark.parametrize("page", [1, 7, 16, 64, 100, 256])
def test_chunk_heads_and_pages(H, Hk, d, page):
    check_chunks([65, 130, 1, 9], [3, 1, 1, 9], H, Hk, d, page, seed=page)
    check_chunks([65, 130, 200], [40, 0, 33], H, Hk, d, page, seed=page + 1)


@pytest.mark.parametrize("cached", [0, 1, 15, 63, 64, 65, 127, 129, 1000, 5000])
@pytest.mark.parametrize("new", [1, 2, 5, 17, 64, 65, 130, 300])
def test_chunk_lengths(cached, new):
    check_chunks([cached + new, new, cached + 1], [new, new, 1], 8, 2, 64, 16, seed=cached + new)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 8, 16, 24, 32, 64, 128, 192, 256])
@pytest.mark.parametrize("r", [1, 4, 7])
def test_chunk_blocks_of_many_rows(r, page, d):
    """Blocks of one and two row tiles, the last of each partly filled; key tiles that start, end and are missing inside pages."""
    check_chunks([500, 257, 300], [400, 257, 20], 2 * r, 2, d, page, seed=page)
    check_chunks([700], [131], r, 1, d, page, seed=page + 5)


@pytest.mark.parametrize("d", [8, 40, 72, 104])
@pytest.mark.parametrize("page", [16, 48, 128])
def test_chunk_many_rows_with_few_dimensions(d, page):
    check_chunks([200, 300, 77], [70, 300, 1], 8, 2, d, page, seed=d)


def test_chunk_long_context_is_cut_and_joined():
    check_chunks([9000], [40], 4, 1, 128, 64)
    check_chunks([9000, 10], [200, 10], 8, 2, 128, 64)
    check_chunks([20000], [3], 4, 1, 64, 16)
    check_chunks([3000, 40, 1], [2500, 1, 1], 4, 2, 128, 64)


def test_chunk_single_tokens_and_chunks_in_one_step():
    check_chunks([100, 1, 700, 33, 900, 64], [1, 1, 300, 1, 5, 64], 8, 2, 128, 32)
    check_chunks([100, 1, 700, 33, 900, 64], [1, 1, 300, 1, 5, 64], 8, 2, 128, 32, bounds=False)


def test_chunk_rows_without_keys():
    """Chunks longer than their trajectory: the first tokens see nothing.  Empty chunks, empty trajectories."""
    check_chunks([0, 3, 0, 10], [2, 5, 0, 0], 4, 2, 64, 16)
    check_chunks([0, 30, 0, 10], [50, 70, 0, 0], 8, 2, 128, 16)
    check_chunks([0], [3], 4, 2, 64, 16)
    check_chunks([0, 0], [300, 3], 4, 2, 64, 16)


def test_chunk_tokens_outside_every_trajectory_are_left():
    check_chunks([20, 30], [4, 2], 4, 2, 64, 16, first=3, behind=5)
    check_chunks([200, 300], [100, 230], 8, 2, 128, 64, first=40, behind=50)
    check_chunks([200, 300], [100, 230], 8, 2, 128, 64, first=40, behind=300, bounds=False)


def test_chunk_layouts_strides_and_bounds():
    for new in (3, 200):
        check_chunks([300, 210], [new, 7], 8, 2, 64, 32, layout="heads")
        check_chunks([300, 210], [new, 7], 8, 2, 128, 64, layout="heads", q_pad=24)
        check_chunks([300, 210], [new, 7], 8, 2, 128, 64, bounds=False, width=40)
        check_chunks([300, 210], [new, 7], 8, 2, 128, 64, cut=130)
        check_chunks([300, 210], [new, 7], 8, 2, 128, 64, cut=0)
        check_chunks([300, 210], [new, 7], 8, 2, 128, 20, factor=6.0)


def test_chunk_many_trajectories():
    """More trajectories than the lookup goes through level by level, of all sizes, some of them empty."""
    g = torch.Generator().manual_seed(4)
    counts = [int(c) for c in torch.randint(0, 4, (200,), generator=g)]
    counts[7], counts[100], counts[199] = 90, 33, 200
    check_chunks([c + int(k) for c, k in zip(counts, torch.randint(0, 60, (200,), generator=g))], counts, 8, 2, 64, 16, first=1, behind=2)
    counts = [int(c) for c in torch.randint(0, 3, (150,), generator=g)]
    check_chunks([c + int(k) for c, k in zip(counts, torch.randint(0, 60, (150,), generator=g))], counts, 4, 2, 128, 16)


def check_wide(lens, counts, H, Hk, d, page, **more):
    """The same calls with a table for longer trajectories, where rows go in blocks of 128."""
    check_chunks(lens, counts, H, Hk, d, page, bounds=False, width=-(-800 // page), **more)


@pytest.mark.parametrize("H,Hk,d", [(8, 8, 64), (8, 2, 128), (28, 4, 64), (20, 1, 128), (4, 4, 8), (6, 2, 40), (33, 1, 80), (4, 1, 96)])
@pytest.mark.parametrize("page", [1, 7, 16, 64, 100, 256])
def test_chunk_long_tables_heads_and_pages(H, Hk, d, page):
    check_wide([65, 130, 1, 9], [3, 1, 1, 9], H, Hk, d, page, seed=page)
    check_wide([65, 130, 200], [40, 0, 33], H, Hk, d, page, seed=page + 1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [1, 8, 16, 24, 32, 64, 128, 192, 256])
@pytest.mark.parametrize("r", [1, 4, 7])
def test_chunk_long_tables_blocks_of_many_rows(r, page, d):
    check_wide([500, 257, 300], [400, 257, 20], 2 * r, 2, d, page, seed=page)
    check_wide([700], [131], r, 1, d, page, seed=page + 5)


@pytest.mark.parametrize("new", [17, 64, 65, 130, 300])
@pytest.mark.parametrize("cached", [0, 1, 15, 63, 64, 65, 127, 129])
def test_chunk_long_tables_lengths(cached, new):
    check_wide([cached + new, new, cached + 1], [new, new, 1], 8, 2, 64, 16, seed=cached + new)


def test_chunk_long_tables_empty_outside_and_strided():
    check_wide([0, 30, 0, 10], [50, 70, 0, 0], 8, 2, 128, 16)
    check_wide([0, 0], [300, 3], 4, 2, 64, 16)
    check_wide([200, 300], [100, 230], 8, 2, 128, 64, first=40, behind=50)
    check_wide([300, 210], [200, 7], 8, 2, 64, 32, layout="heads")
    check_wide([300, 210], [200, 7], 8, 2, 128, 64, layout="heads", q_pad=24)
    check_wide([300, 210], [200, 7], 8, 2, 128, 20, factor=6.0)
    check_wide([200, 300, 77], [70, 300, 1], 8, 2, 72, 48)


@pytest.mark.parametrize("page", [7, 16, 64])
def test_chunk_long_tables_pages_that_are_not_there(api, page):
    lens, counts = [400, 333], [150, 150]
    cache = Paged(4, lens, page, 2, 64)
    table, missing = cache.table.clone(), [torch.zeros(400, dtype=torch.bool) for _ in lens]
    for b, j, what in ((0, 0, -1), (0, 2, 2 ** 31 - 1), (1, 1, -2 ** 31), (1, (332 // page), cache.k.shape[0])):
        table[b, j] = what
        missing[b][j * page:(j + 1) * page] = True
    table = torch.cat([table, torch.full((2, -(-800 // page)), -1, dtype=I32)], 1)
    q = torch.randn(300, 4, 64, generator=torch.Generator().manual_seed(9)).to(BF16)
    want = plain_chunks(q, cache.keys, lens, [0, 150, 300], 0.2, 400, missing)
    out, lse = api.chunk_attention(up(q), cache.kd, cache.vd, up(table), up(ints([0, 150, 300])), up(ints(lens)), scale=0.2)
    compare_chunks(out, lse, *want, 5.0)
    out, lse = api.chunk_attention(up(q), cache.kd, cache.vd, up(torch.full_like(table, -1)), up(ints([0, 150, 300])), up(ints(lens)), scale=0.2)
    assert (out == 0).all() and (lse == -math.inf).all()


def test_chunk_lengths_out_of_all_proportion(api):
    """Lengths beyond the table, up to the largest number: what the table holds is seen; negative ones: nothing."""
    for new in (2, 100):
        cache = Paged(5, [320], 16, 2, 64)
        q = torch.randn(new, 4, 64, generator=torch.Generator().manual_seed(9)).to(BF16)
        args = (up(q), cache.kd, cache.vd, up(cache.table), up(ints([0, new])))
        want = api.chunk_attention(*args, up(ints([320 + new])))
        got = api.chunk_attention(*args, up(ints([2 ** 31 - 1])))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        out, lse = api.chunk_attention(*args, up(ints([-2 ** 31])))
        assert (out == 0).all() and (lse == -math.inf).all()


def test_chunk_longer_than_max_new_is_cut(api):
    from paper_2608_17641_b200 import binding
    for most, new in ((2, 6), (90, 300)):
        cache = Paged(1, [400, 50], 16, 2, 64)
        q = up(torch.randn(new + 2, 4, 64, generator=torch.Generator().manual_seed(3)).to(BF16))
        args = (cache.kd, cache.vd, up(cache.table), up(ints([0, new, new + 2])), up(ints([400, 50])))
        want, want_lse = binding.rlcs_chunk_attention_bf16(q, *args, scale=0.1)
        out, lse = guarded_empty((new + 2, 4, 64), BF16).fill_(5), guarded_empty((new + 2, 4), F32).fill_(5)
        binding.rlcs_chunk_attention_bf16(q, *args, scale=0.1, max_new=most, out=out, lse=lse)
        assert (out[most:new] == 5).all() and (lse[most:new] == 5).all()
        there = [i for i in range(new + 2) if not most <= i < new]
        assert (lse[there] - want_lse[there]).abs().max() < 1e-4 and (out[there].float() - want[there].float()).abs().max() < 0.05


@pytest.mark.parametrize("new", [3, 150])
@pytest.mark.parametrize("page", [7, 16, 64])
def test_chunk_pages_that_are_not_there(api, new, page):
    lens, counts = [400, 333], [new, min(new, 333)]
    cache = Paged(4, lens, page, 2, 64)
    table, missing = cache.table.clone(), [torch.zeros(400, dtype=torch.bool) for _ in lens]
    for b, j, what in ((0, 0, -1), (0, 2, 2 ** 31 - 1), (1, 1, -2 ** 31), (1, (332 // page), cache.k.shape[0])):
        table[b, j] = what
        missing[b][j * page:(j + 1) * page] = True
    g = torch.Generator().manual_seed(9)
    offsets = [0, counts[0], counts[0] + counts[1]]
    q = torch.randn(offsets[-1], 4, 64, generator=g).to(BF16)
    want = plain_chunks(q, cache.keys, lens, offsets, 0.2, 400, missing)
    out, lse = api.chunk_attention(up(q), cache.kd, cache.vd, up(table), up(ints(offsets)), up(ints(lens)), scale=0.2)
    compare_chunks(out, lse, *want, 5.0)
    # no page at all
    out, lse = api.chunk_attention(up(q), cache.kd, cache.vd, up(torch.full_like(table, -1)), up(ints(offsets)), up(ints(lens)), scale=0.2)
    assert (out == 0).all() and (lse == -math.inf).all()


def test_chunk_tables_narrower_than_the_lengths(api):
    """Keys at places beyond the table's width are not there."""
    for new in (4, 100):
        cache = Paged(4, [320], 16, 2, 64)
        q = torch.randn(new, 4, 64, generator=torch.Generator().manual_seed(9)).to(BF16)
        missing = [torch.arange(320) >= 160]
        want = plain_chunks(q, cache.keys, [320], [0, new], 0.2, 320, missing)
        out, lse = api.chunk_attention(up(q), cache.kd, cache.vd, up(cache.table[:, :10].contiguous()), up(ints([0, new])), up(ints([320])), scale=0.2)
        compare_chunks(out, lse, *want, 5.0)


def test_chunk_offsets_past_32_bits(api):
    """A cache of more than 2^31 elements whose trajectory lies in its last pages."""
    page, Hk, d = 64, 8, 128
    pages = (1 << 31) // (page * Hk * d) + 40
    k = torch.empty(pages, page, Hk, d, dtype=BF16, device="cuda")
    v = torch.empty_like(k)
    small = Paged(3, [500], page, Hk, d)
    for new in (2, 300):
        table = small.table + (pages - small.k.shape[0])
        k[pages - small.k.shape[0]:], v[pages - small.k.shape[0]:] = small.kd, small.vd
        q = up(torch.randn(new, 16, d, generator=torch.Generator().manual_seed(1)).to(BF16))
        want = api.chunk_attention(q, small.kd, small.vd, up(small.table), up(ints([0, new])), up(ints([500])))
        got = api.chunk_attention(q, k, v, up(table), up(ints([0, new])), up(ints([500])))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # and copies of pages there
    src, dst = ints([pages - 1, 0]), ints([pages - 20, 1])
    k[0], v[0] = 1, 2
    k[pages - 1], v[pages - 1] = 3, 4
    api.copy_pages(k, v, up(src), up(dst))
    assert (k[pages - 20] == 3).all() and (v[pages - 20] == 4).all() and (k[1] == 1).all() and (v[1] == 2).all()


def test_chunk_of_one_token_agrees_with_the_shared_prefix_operator(api):
    cache = Paged(8, [300, 45, 1], 16, 2, 128)
    q = up(torch.randn(3, 8, 128, generator=torch.Generator().manual_seed(2)).to(BF16))
    a = api.chunk_attention(q, cache.kd, cache.vd, up(cache.table), up(ints([0, 1, 2, 3])), up(ints([300, 45, 1])))
    b = api.shared_prefix_attention(q, cache.kd, cache.vd, None, None, None, up(cache.table), up(ints([300, 45, 1])))
    assert (a[1] - b[1]).abs().max() < 2e-5 and (a[0].float() - b[0].float()).abs().max() <= 2.0 ** -7 * float(b[0].float().abs().max())


def test_chunk_on_another_stream_and_twice_the_same(api):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check_chunks([300, 40], [90, 2], 8, 2, 128, 64, stream=s)
    cache = Paged(8, [3000, 45], 64, 2, 128)
    q = up(torch.randn(345, 8, 128, generator=torch.Generator().manual_seed(2)).to(BF16))
    args = (q, cache.kd, cache.vd, up(cache.table), up(ints([0, 300, 345])), up(ints([3000, 45])))
    a, b = api.chunk_attention(*args), api.chunk_attention(*args)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("polls", [0, 1, 3])
@pytest.mark.parametrize("new,page", [(2, 16), (100, 64), (300, 64), (300, 24)])
def test_chunk_waits_that_run_out(api, polls, new, page):
    """A wait that gives up leaves NaN or the right value, nothing else, and the next call is right."""
    from paper_2608_17641_b200 import binding
    cache = Paged(8, [900], page, 2, 128)
    q = up(torch.randn(new, 8, 128, generator=torch.Generator().manual_seed(2)).to(BF16))
    args = (q, cache.kd, cache.vd, up(cache.table), up(ints([0, new])), up(ints([900])))
    want = api.chunk_attention(*args)
    binding.rlcs_debug_set_wait_polls(polls)
    try:
        got = api.chunk_attention(*args)
        torch.cuda.synchronize()
    finally:
        binding.rlcs_debug_set_wait_polls(-1)
    for g, w in zip(got, want):
        assert (torch.isnan(g) | (g == w)).all()
    again = api.chunk_attention(*args)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


# ------------------------------------------------------------------------------------------ verification
def plain_weights(row, t):
    """Weights of one row of logits from the device's own fp32 exponentials, and its log-probabilities in 64 bits."""
    row = torch.where(torch.isnan(row.float()), -math.inf, row.float())
    top = row.max()
    if top == -math.inf:
        return None, None
    tr = torch.tensor(t, dtype=F32)
    greedy = not bool(tr > 0)
    inv = torch.tensor(1.0) if greedy else (torch.ones(1, device="cuda") / tr.cuda()).cpu()[0]
    e = torch.exp(torch.where(row == top, torch.zeros(()), (row - top) * inv).cuda()).cpu()
    w = [math.floor(v * 2.0 ** 31 + 0.5) for v in e.double().tolist()]
    d = torch.where(row == top, torch.zeros((), dtype=torch.float64), (row.double() - top.double()) / (1.0 if greedy else float(tr)))
    if greedy:
        w = [int(j == int(row.argmax())) for j in range(len(w))]
    return w, d - torch.log(torch.exp(d).sum())


def plain_verify(x, tokens, offsets, u, du, drafts, temps):
    T, A = x.shape
    out, lps, acc = [None] * T, [None] * T, []
    for b in range(len(offsets) - 1):
        lo, hi = offsets[b], offsets[b + 1]
        for t in range(lo, hi):
            out[t], lps[t] = -1, -math.inf
        acc.append(0)
        for t in range(lo, hi):
            w, lp = plain_weights(x[t], temps[b])
            if w is None:
                break
            greedy, last, tok = not temps[b] > 0, t == hi - 1, int(tokens[t + 1]) if t + 1 < hi else -1
            v = None
            if not last:
                if drafts is not None and not greedy:
                    v = plain_weights(drafts[t], temps[b])[0]
                vx, V = (float(v[tok]) if v and 0 <= tok < A else 0.0, float(sum(v)) if v else 0.0) if drafts is not None and not greedy else (1.0, 1.0)
                ok = 0 <= tok < A and (w[tok] == 1 if greedy else float(u[t]) * (vx * float(sum(w))) < float(w[tok]) * V)
                if ok:
                    out[t], lps[t] = tok, float(lp[tok])
                    acc[b] += 1
                    continue
            rest = list(w)
            if not last and not greedy:
                if drafts is not None:
                    unit, less = 2.0 ** 40 / float(sum(w)), 2.0 ** 40 / float(sum(v)) if v else 0.0
                    rest = [max(0, math.floor(float(a) * unit) - (math.floor(float(c) * less) if v else 0)) for a, c in zip(w, v or [0] * A)]
                elif 0 <= tok < A:
                    rest[tok] = 0
            if sum(rest) == 0:
                rest = list(w)
            target = min(math.floor(float(du[b]) * float(sum(rest))), sum(rest) - 1)
            pick = int(np.searchsorted(np.cumsum(np.array(rest, dtype=np.int64)), target, side="right"))
            out[t], lps[t] = pick, float(lp[pick])
            break
    return out, lps, acc


def check_verify(api, x, tokens, offsets, u, du, drafts=None, temps=1.0, pad=0, lead=0, stream=None):
    from paper_2608_17641_b200 import binding
    B = len(offsets) - 1
    each = [float(torch.tensor(t, dtype=F32)) for t in (temps if isinstance(temps, list) else [temps] * B)]
    want = plain_verify(x, tokens, offsets, u, du, drafts, each)
    fn = binding.rlcs_verify_drafts if x.dtype == F32 else binding.rlcs_verify_drafts_bf16
    T = x.shape[0]
    out, lp, acc = guarded_empty((T,), I32).fill_(77), guarded_empty((T,), F32).fill_(77), guarded_empty((B,), I32).fill_(77)
    fn(strided_rows(x, pad, lead), up(tokens), up(ints(offsets)), up(u), up(du), draft_logits=None if drafts is None else strided_rows(drafts, pad + 1, lead),
       temperature=up(torch.tensor(temps)) if isinstance(temps, list) else temps, out_tokens=out, log_probs=lp, accepted=acc, stream=stream)
    if stream is not None:
        stream.synchronize()
    out, lp = out.tolist(), lp.tolist()
    assert acc.tolist() == want[2]
    for t in range(T):
        if want[0][t] is None:
            assert out[t] == 77 and lp[t] == 77
            continue
        assert out[t] == want[0][t], (t, out[t], want[0][t])
        if want[1][t] == -math.inf:
            assert lp[t] == -math.inf
        else:
            assert abs(lp[t] - want[1][t]) <= 1e-5 + 2.0 ** -22 * abs(want[1][t]), (t, lp[t], want[1][t])
    return want


def verify_inputs(counts, A, dtype, seed, near=0.7, first=0, behind=0):
    g = torch.Generator().manual_seed(seed)
    offsets = [first]
    for n in counts:
        offsets.append(offsets[-1] + n)
    T = offsets[-1] + behind
    x = (torch.randn(T, A, generator=g) * 3).to(dtype)
    drafts = (x.float() + near * torch.randn(T, A, generator=g)).to(dtype)
    tokens = torch.zeros(T, dtype=I32)
    for t in range(T - 1):
        tokens[t + 1] = int(torch.multinomial(torch.softmax(drafts[t].float(), 0), 1, generator=g))
    return x, tokens, offsets, torch.rand(T, generator=g), torch.rand(len(counts), generator=g), drafts


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [1, 2, 7, 31, 33, 64, 65, 255, 1000, 1025, 4099, 20011])
def test_verify_sizes(api, A, dtype):
    x, tokens, offsets, u, du, drafts = verify_inputs([4, 1, 0, 9, 3], A, dtype, A)
    check_verify(api, x, tokens, offsets, u, du, drafts)
    check_verify(api, x, tokens, offsets, u, du, None, pad=A % 3, lead=1)
    check_verify(api, x, tokens, offsets, u, du, drafts, temps=[0.7, 0.0, 1.0, 1.3, -1.0], pad=5)
    check_verify(api, x, tokens, offsets, u, du, None, temps=0.0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A,B", [(70001, 2), (150000, 1), (3001, 300)])
def test_verify_wide_rows_and_many_trajectories(api, A, B, dtype):
    counts = [3, 6] if B == 2 else [4] if B == 1 else [1 + i % 3 for i in range(B)]
    x, tokens, offsets, u, du, drafts = verify_inputs(counts, A, dtype, A, near=0.4)
    want = check_verify(api, x, tokens, offsets, u, du, drafts, temps=0.9, pad=1)
    assert B < 100 or (any(a == 0 for a in want[2]) and any(a == 2 for a in want[2]))
    check_verify(api, x, tokens, offsets, u, du, None, temps=1.1)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A,times", [(1500, 100), (9001, 130), (20245, 50), (130000, 9), (147000, 9), (200003, 8)])
def test_verify_more_trajectories_than_run_at_once(api, A, times, dtype):
    """Some trajectories against the plain form, and many times over in one call, which may split a row otherwise: the same tokens."""
    x, tokens, offsets, u, du, drafts = verify_inputs([3, 1, 2, 0, 4], A, dtype, A, near=0.5)
    x[5, : A // 2] = -math.inf
    x[6] = -math.inf
    temps = [0.8, 1.0, 1.3, 1.0, 0.0]
    for q, pad in ((drafts, A % 3), (None, 0)):
        check_verify(api, x, tokens, offsets, u, du, q, temps=temps, pad=pad)
        rows, results = x.shape[0], []
        for n in (1, times):
            starts = ints([k * rows + o for k in range(n) for o in offsets[:-1]] + [n * rows])
            out, lp, acc = api.verify_drafts(strided_rows(x.repeat(n, 1), pad, 0), up(tokens.repeat(n)), up(starts), up(u.repeat(n)), up(du.repeat(n)),
                                             draft_logits=None if q is None else up(q.repeat(n, 1)), temperature=up(torch.tensor(temps * n)))
            results.append((out.cpu().view(n, rows), lp.cpu().view(n, rows), acc.cpu().view(n, 5)))
        (out, lp, acc), (outs, lps, accs) = results
        assert (outs == out).all() and (accs == acc).all()
        assert ((lps - lp).abs().nan_to_num(0.0) <= 3e-5).all()        # twice what one may be off; nan: -inf on both sides


@pytest.mark.parametrize("drawn", [True, False])
def test_verify_rows_too_wide_for_shared_memory(api, drawn):
    x, tokens, offsets, u, du, drafts = verify_inputs([3], 500001, BF16, 2, near=0.3)
    check_verify(api, x, tokens, offsets, u, du, drafts if drawn else None, pad=3)


@pytest.mark.parametrize("A", [9, 3000])
def test_verify_rows_outside_and_long_runs(api, A):
    x, tokens, offsets, u, du, drafts = verify_inputs([40, 2, 700] if A == 9 else [40, 2], A, F32, 3, near=0.05, first=2, behind=3)
    check_verify(api, x, tokens, offsets, u, du, drafts)
    check_verify(api, x, tokens, offsets, u * 0, du, x)                # the draft policy is the target: everything stays


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [5, 300, 9000])
def test_verify_masked_infinite_and_nan_logits(api, A, dtype):
    x, tokens, offsets, u, du, drafts = verify_inputs([3, 3, 3, 3, 3, 3, 3], A, dtype, 17, near=0.2)
    g = torch.Generator().manual_seed(1)
    x[torch.rand(x.shape, generator=g) < 0.3] = -math.inf
    drafts[torch.rand(x.shape, generator=g) < 0.3] = torch.finfo(dtype).min
    x[4] = -math.inf                                                   # allows nothing
    x[6, :] = float("nan")
    x[9, A // 2] = math.inf
    drafts[12] = -math.inf                                             # a draft from nowhere
    x[15, ::2] = float("nan")
    drafts[18, 1:] = float("nan")
    check_verify(api, x, tokens, offsets, u, du, drafts)
    check_verify(api, x, tokens, offsets, u, du, None, temps=[1.0, 0.0, 0.5, 0.0, 2.0, 0.0, 1.0])


@pytest.mark.parametrize("drawn", [False, True])
def test_verify_tokens_that_are_none(api, drawn):
    x, tokens, offsets, u, du, drafts = verify_inputs([4, 4, 4, 4], 50, F32, 5, near=0.0)
    u *= 0.01
    tokens[1], tokens[6], tokens[11], tokens[12] = -1, 50, 2 ** 31 - 1, -2 ** 31
    got = check_verify(api, x, tokens, offsets, u, du, drafts if drawn else None)
    assert got[2][0] == 0 and got[2][1] <= 1


def test_verify_extreme_uniforms(api):
    x, tokens, offsets, u, du, drafts = verify_inputs([4] * 6, 300, F32, 5, near=0.3)
    top = 1 - 2.0 ** -24
    for a in (0.0, top, 1e-30):
        for c in (0.0, top, 0.5):
            check_verify(api, x, tokens, offsets, torch.full_like(u, a), torch.full_like(du, c), drafts)
            check_verify(api, x, tokens, offsets, torch.full_like(u, a), torch.full_like(du, c), None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [40, 3000, 20000])
def test_verify_uniforms_at_the_border(api, A, dtype):
    """Uniforms within a few places of w V / (v W), where the verdict takes the whole weights' own sums."""
    x, tokens, offsets, u, du, drafts = verify_inputs([6, 9, 2], A, dtype, A, near=0.5)
    for drawn in (True, False):
        for step in (-2, -1, 0, 1, 2):
            for t in range(len(u) - 1):
                w, v = plain_weights(x[t], 1.0)[0], plain_weights(drafts[t], 1.0)[0]
                tok = int(tokens[t + 1])
                at = w[tok] * sum(v) / max(1, v[tok] * sum(w)) if drawn else w[tok] / sum(w)
                edge = np.float32(min(at, 1 - 2.0 ** -24))
                for _ in range(abs(step)):
                    edge = np.nextafter(edge, np.float32(step))
                u[t] = min(float(edge), 1 - 2.0 ** -24)
            check_verify(api, x, tokens, offsets, u, du, drafts if drawn else None)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [7, 700, 9000])
def test_verify_infinite_and_tiny_temperatures(api, A, dtype):
    """An infinite temperature makes all allowed tokens alike and no other one possible; a tiny one all but decides."""
    x, tokens, offsets, u, du, _ = verify_inputs([3, 4, 1, 2], A, dtype, A)
    off = torch.rand(x.shape, generator=torch.Generator().manual_seed(1)) < 0.5
    off[:, 0] = False
    x[off] = -math.inf
    x[2, A // 2] = float("nan")
    out, lp, acc = api.verify_drafts(up(x), up(tokens), up(ints(offsets)), up(u), up(du), temperature=math.inf)
    allowed = (x > -math.inf)
    out, lp = out.tolist(), lp.tolist()
    for t, tok in enumerate(out):
        if tok >= 0:
            assert allowed[t, tok] and abs(lp[t] + math.log(int(allowed[t].sum()))) < 1e-5
    assert max(out) >= 0
    out, lp, acc = api.verify_drafts(up(x), up(tokens), up(ints(offsets)), up(u), up(du), temperature=1e-30)
    best = torch.where(torch.isnan(x.float()), -math.inf, x.float()).max(1)
    for t, tok in enumerate(out.tolist()):
        if tok >= 0:
            assert float(x[t, tok]) == float(best.values[t])


def test_verify_turned_down_draft_that_is_certain(api):
    """Nothing is left of the difference (p = q, turned down by u = 1) and of a certain, given draft: the target's own probabilities."""
    x = torch.full((4, 40), -math.inf)
    x[:, 7] = 1.0
    tokens, offsets = ints([0, 7, 0, 7]), [0, 2, 4]
    u, du = torch.ones(4), torch.tensor([0.3, 0.9])
    for drafts in (None, x):
        check_verify(api, x, tokens, offsets, u, du, drafts)


def test_verify_follows_the_target(api):
    """What comes out is distributed as the target: 40000 trajectories of one draft, five standard deviations."""
    B, A = 40000, 6
    g = torch.Generator(device="cuda").manual_seed(4)
    p_log, q_log = torch.tensor([0.5, -1.0, 2.0, 0.0, -3.0, 1.0], device="cuda"), torch.tensor([1.5, 0.0, 0.0, 0.5, 1.0, -2.0], device="cuda")
    drafts = q_log.repeat(2 * B, 1)
    tokens = torch.multinomial(torch.softmax(q_log, 0).repeat(2 * B, 1), 1, generator=g)[:, 0].to(I32)
    rand = lambda n: torch.rand(n, device="cuda", generator=g)
    out, lp, acc = api.verify_drafts(p_log.repeat(2 * B, 1), tokens, torch.arange(0, 2 * B + 1, 2, device="cuda", dtype=I32), rand(2 * B), rand(B),
                                     draft_logits=drafts)
    p, q = torch.softmax(p_log, 0), torch.softmax(q_log, 0)
    share = torch.bincount(out[::2].long(), minlength=A) / B
    assert ((share - p).abs() < 5 * (p * (1 - p) / B).sqrt()).all()
    keep = float(torch.minimum(p, q).sum())
    assert abs(float(acc.float().mean()) - keep) < 5 * math.sqrt(keep * (1 - keep) / B)
    assert (lp[::2] - torch.log(p)[out[::2].long()]).abs().max() < 1e-5


def test_verify_streams_and_repeats(api):
    s = torch.cuda.Stream()
    x, tokens, offsets, u, du, drafts = verify_inputs([4, 2, 8], 5000, BF16, 6)
    s.wait_stream(torch.cuda.current_stream())
    check_verify(api, x, tokens, offsets, u, du, drafts, stream=s)
    args = (up(x), up(tokens), up(ints(offsets)), up(u), up(du))
    a, b = (api.verify_drafts(*args, draft_logits=up(drafts)) for _ in range(2))
    for v, w in zip(a, b):
        assert torch.equal(v, w)


def test_verify_without_trajectories_or_rows(api):
    none = torch.zeros(0, device="cuda")
    out, lp, acc = api.verify_drafts(torch.zeros(0, 5, device="cuda"), none.to(I32), up(ints([0, 0, 0])), none, torch.zeros(2, device="cuda"))
    assert out.numel() == 0 and lp.numel() == 0 and acc.tolist() == [0, 0]
    out, lp, acc = api.verify_drafts(torch.zeros(3, 5, device="cuda"), up(ints([1, 2, 3])), up(ints([0])), up(torch.zeros(3)), none)
    assert acc.numel() == 0


# ------------------------------------------------------------------------------------------ distillation
def plain_distill(x, ids, teacher, mask, T, scale):
    R, A = x.shape
    lq = torch.log_softmax(x.double() / T, 1)
    loss, grad = torch.zeros(R, dtype=torch.float64), torch.zeros(R, A, dtype=torch.float64)
    for r in range(R):
        there = [(int(i), float(t)) for i, t in zip(ids[r], teacher[r]) if 0 <= int(i) < A]
        if (mask is not None and not mask[r]) or not there or max(t for _, t in there) == -math.inf or bool((x[r] == -math.inf).all()):
            continue
        p = torch.softmax(torch.tensor([t for _, t in there], dtype=torch.float64) / T, 0)
        grad[r] = torch.exp(lq[r])
        for (i, _), w in zip(there, p):
            if w > 0:
                loss[r] += w * (torch.log(w) - lq[r, i])
                grad[r, i] -= w
    return scale * loss, scale / T * grad, scale / T * torch.exp(lq)


def distill_inputs(R, A, K, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(R, A, generator=g) * 3).to(dtype)
    ids = torch.stack([torch.randperm(A, generator=g)[:K] if K <= A else torch.randint(0, A, (K,), generator=g) for _ in range(R)]).to(I32).view(R, K)
    return x, ids, torch.randn(R, K, generator=g) * 2, g


def check_distill(api, x, ids, teacher, mask=None, T=1.0, scale=1.0, pad=0, lead=0, in_place=False, stream=None):
    want, want_grad, prob = plain_distill(x, ids, teacher, mask, T, scale)
    xd = strided_rows(x, pad, lead)
    loss, grad = api.compute_distillation(xd, up(ids), up(teacher), mask=None if mask is None else up(mask), temperature=T, scale=scale,
                                          in_place=in_place, stream=stream)
    if stream is not None:
        stream.synchronize()
    if in_place:
        assert grad.data_ptr() == xd.data_ptr()
    loss, got = loss.cpu().double(), grad.cpu().double()
    assert ((loss - want).abs() <= scale * 1e-5 + 2.0 ** -22 * want.abs()).all(), (loss - want).abs().max()
    # a gradient is the difference of two probabilities, each 1e-5 of itself off
    bound = 1e-5 * (prob + (prob - want_grad).abs()) + (2.0 ** -8 if x.dtype == BF16 else 2.0 ** -22) * want_grad.abs() + 1e-38
    assert ((got - want_grad).abs() <= bound * 1.01).all(), ((got - want_grad).abs() - bound).max()
    return loss, got


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [1, 2, 7, 18, 63, 64, 65, 100, 257, 1000, 1025, 2049, 4099, 9001, 20011, 70003])
def test_distill_sizes(api, A, dtype):
    R = 9 if A < 5000 else 4
    for K, pad, lead, in_place in ((1, 0, 0, False), (min(A, 20), A % 3 + 1, 1, False), (min(A, 64), 0, 3, True), (min(A, 200), 8, 0, False)):
        x, ids, teacher, _ = distill_inputs(R, A, K, dtype, A + K)
        check_distill(api, x, ids, teacher, T=1.3, scale=0.7, pad=pad, lead=lead, in_place=in_place)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A,K", [(5, 300), (700, 1024), (30000, 1024), (150001, 33)])
def test_distill_many_entries_and_wide_rows(api, A, K, dtype):
    x, ids, teacher, _ = distill_inputs(3, A, K, dtype, K)
    check_distill(api, x, ids, teacher, T=0.8)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A,K", [(3, 40), (7, 17), (11, 16), (16, 4), (23, 33), (33, 64), (70, 9)])
def test_distill_short_rows(api, A, K, dtype):
    for R, pad, lead in ((1, 0, 0), (515, 0, 1), (130, 5, 3)):
        x, ids, teacher, g = distill_inputs(R, A, K, dtype, A + R)
        ids[R // 2] = ids[R // 2, 0]
        ids[R // 3, K // 2:] = -1
        check_distill(api, x, ids, teacher, torch.rand(R, generator=g) < 0.9, T=0.7, pad=pad, lead=lead, in_place=pad == 0)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [3, 40, 500, 12000])
def test_distill_entries_named_twice_or_absent(api, A, dtype):
    x, ids, teacher, g = distill_inputs(8, A, 12, dtype, A)
    ids[0] = ids[0, 0]                                                 # all of one token
    ids[1, 1::2] = ids[1, ::2]
    ids[2, 3:] = -1
    ids[3] = -1                                                        # no teacher
    ids[4, 0], ids[4, 1], ids[4, 2] = A, 2 ** 31 - 1, -2 ** 31
    teacher[2, 3:] = float("nan")                                      # of absent entries
    teacher[5, 1:] = -math.inf
    teacher[6] = -math.inf
    mask = torch.ones(8, dtype=torch.bool)
    loss, grad = check_distill(api, x, ids, teacher, mask)
    assert loss[3] == 0 and (grad[3] == 0).all() and loss[6] == 0 and (grad[6] == 0).all()
    mask[::2] = False
    check_distill(api, x, ids, teacher, mask, scale=0.25)


@pytest.mark.parametrize("A", [5, 70, 3001, 9000])
def test_distill_rows_left_out_may_hold_anything(api, A):
    x, ids, teacher, _ = distill_inputs(7, A, 4, F32, 6)
    clean = [v.cpu() for v in api.compute_distillation(up(x), up(ids), up(teacher))]
    x[0], x[1], x[2] = float("nan"), math.inf, -math.inf
    teacher[3] = float("nan")
    mask = torch.tensor([0, 0, 1, 0, 1, 255, 1], dtype=torch.uint8)
    loss, grad = (v.cpu() for v in api.compute_distillation(up(x), up(ids), up(teacher), mask=up(mask)))
    assert (loss[:4] == 0).all() and (grad[:4] == 0).all()
    assert torch.equal(loss[4:], clean[0][4:]) and torch.equal(grad[4:], clean[1][4:])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [6, 70, 900, 9000])
def test_distill_masked_and_nan_logits(api, A, dtype):
    x, ids, teacher, g = distill_inputs(9, A, 3, dtype, 8)
    off = torch.rand(9, A, generator=g) < 0.4
    off.scatter_(1, ids.long(), False)
    x[off] = -math.inf
    x[1][off[1]] = torch.finfo(dtype).min
    x[2][off[2]] = -1e9
    _, grad = check_distill(api, x, ids, teacher, T=1.0)
    assert (grad[off] == 0).all()
    # a teacher that wants what the student excludes: loss +inf, gradient finite; NaN and +inf stay in their rows
    clean = [v.cpu() for v in api.compute_distillation(up(x), up(ids), up(teacher))]
    x[3, ids[3, 0].long()] = -math.inf
    x[4, A // 2] = float("nan")
    x[5, 0] = math.inf
    teacher[6, 1] = float("nan")
    teacher[7, 0] = math.inf
    loss, grad = (v.cpu() for v in api.compute_distillation(up(x), up(ids), up(teacher)))
    assert loss[3] == math.inf and torch.isfinite(grad[3]).all()
    assert torch.isnan(loss[4:8]).all() and torch.isnan(grad[4:8]).all()
    for r in (0, 1, 2, 8):
        assert loss[r] == clean[0][r] and torch.equal(grad[r], clean[1][r])


@pytest.mark.parametrize("A", [50, 900, 9000])
def test_distill_logits_far_from_zero(api, A):
    """A common offset of the logits changes nothing: 1e8 and 1e30 are exact multiples of the logits' own spacing there."""
    x, ids, teacher, g = distill_inputs(4, A, 6, F32, 3)
    x[0] = torch.randint(0, 4, (A,), generator=g) * 8.0 + 2.0 ** 27
    x[1] = -2.0 ** 100
    x[2] = torch.randint(0, 4, (A,), generator=g) * 8.0 - 2.0 ** 27
    x[3, ::2] = -1e30
    check_distill(api, x, ids, teacher)


@pytest.mark.parametrize("R", [1, 7, 129, 1000, 4099])
@pytest.mark.parametrize("A", [18, 129, 1500])
def test_distill_row_counts(api, R, A):
    x, ids, teacher, g = distill_inputs(R, A, 5, BF16, R)
    mask = torch.rand(R, generator=g) < 0.8
    check_distill(api, x, ids, teacher, mask, scale=1.0 / R)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A,K", [(2049, 2), (4095, 600), (4097, 9), (6001, 1024), (8192, 33), (8194, 5), (12345, 520), (16384, 12), (16390, 300)])
def test_distill_many_rows_of_middle_width(api, A, K, dtype):
    """More than two rows a multiprocessor, of 8 to 64 KB; the rows that are checked hold what can go wrong, the others repeat them."""
    x, ids, teacher, g = distill_inputs(10, A, K, dtype, A)
    ids[0] = ids[0, 0]
    ids[1, K // 2:] = -1
    ids[2] = -1
    ids[3, 0], ids[3, 1] = A, -2 ** 31
    teacher[4, 1:] = -math.inf
    teacher[5] = -math.inf
    off = torch.rand(10, A, generator=g) < 0.4
    off.scatter_(1, ids.clamp(0, A - 1).long(), False)
    x[6][off[6]], x[7][off[7]] = -math.inf, torch.finfo(dtype).min
    mask = torch.ones(10, dtype=torch.bool)
    mask[8] = False
    want, want_grad, prob = plain_distill(x, ids, teacher, mask, 1.2, 0.9)
    loss, grad = api.compute_distillation(strided_rows(x.repeat(31, 1), K % 3, A % 2), up(ids.repeat(31, 1)), up(teacher.repeat(31, 1)),
                                          mask=up(mask.repeat(31)), temperature=1.2, scale=0.9, in_place=K % 2 == 0)
    loss, grad = loss.cpu().view(31, 10), grad.cpu().view(31, 10, A)
    assert ((loss[0].double() - want).abs() <= 1e-5 + 2.0 ** -22 * want.abs()).all()
    bound = 1e-5 * (prob + (prob - want_grad).abs()) + (2.0 ** -8 if dtype == BF16 else 2.0 ** -22) * want_grad.abs() + 1e-38
    assert ((grad[0].double() - want_grad).abs() <= bound * 1.01).all()
    if A % 8 == 0 and K % 3 == 0:                                      # rows at the same alignment: the same bits
        assert (loss == loss[0]).all() and (grad == grad[0]).all()
    else:
        assert ((loss.double() - want).abs() <= 1e-5 + 2.0 ** -22 * want.abs()).all()
        assert ((grad.double() - want_grad).abs() <= bound * 1.01).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("A", [4100, 8190])
def test_distill_nan_in_many_rows_of_middle_width(api, A, dtype):
    x, ids, teacher, _ = distill_inputs(6, A, 3, dtype, 8)
    again = lambda: [v.cpu().view(60, 6, -1) for v in api.compute_distillation(up(x.repeat(60, 1)), up(ids.repeat(60, 1)), up(teacher.repeat(60, 1)))]
    clean = again()
    x[1, A // 2] = float("nan")
    x[2, A - 1] = math.inf
    teacher[3, 1] = float("nan")
    teacher[4] = torch.tensor([-math.inf, -math.inf, float("nan")])
    x[5, ids[5, 0].long()] = -math.inf
    loss, grad = again()
    assert torch.isnan(loss[:, 1:5]).all() and torch.isnan(grad[:, 1:5]).all()
    assert (loss[:, 5] == math.inf).all() and torch.isfinite(grad[:, 5]).all()
    assert (loss[:, 0] == clean[0][:, 0]).all() and (grad[:, 0] == clean[1][:, 0]).all()


def test_distill_more_rows_than_run_at_once(api):
    R, A, K = 1300, 10001, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn(R, A, device="cuda", generator=g).bfloat16()
    ids = torch.argsort(torch.rand(R, A, device="cuda", generator=g), 1)[:, :K].to(I32).contiguous()
    teacher, mask = torch.randn(R, K, device="cuda", generator=g), torch.rand(R, device="cuda", generator=g) < 0.7
    loss, grad = api.compute_distillation(x, ids, teacher, mask=mask)
    lq, p = torch.log_softmax(x.double(), 1), torch.softmax(teacher.double(), 1)
    want = (p * (torch.log(p) - lq.gather(1, ids.long()))).sum(1) * mask
    assert ((loss - want).abs() <= 2e-5).all()
    dense = lq.exp().scatter_add(1, ids.long(), -p) * mask[:, None]
    assert ((grad - dense).abs() <= 2.0 ** -8 * dense.abs() + 1e-5).all()


def test_distill_gradient_against_differences(api):
    """The kernel's gradient against central differences of the 64-bit loss (h = 1e-4: h^2 and 1e-16 / h stay below 1e-7; the kernel
    itself is within 2e-5)."""
    x, ids, teacher, _ = distill_inputs(6, 9, 4, F32, 12)
    ids[2, 1] = ids[2, 0]
    got = api.compute_distillation(up(x), up(ids), up(teacher), temperature=0.8)[1].cpu().double()
    for j in range(9):
        d = torch.zeros(6, 9, dtype=torch.float64)
        d[:, j] = 1e-4
        more, less = (plain_distill(x.double() + s * d, ids, teacher, None, 0.8, 1.0)[0] for s in (1, -1))
        assert ((more - less) / 2e-4 - got[:, j]).abs().max() < 2e-5


def test_distill_towards_itself_is_zero_and_shapes(api):
    """The student's own logits as the teacher, all of them: loss and gradient vanish, to rounding."""
    x, _, _, _ = distill_inputs(6, 50, 3, F32, 4)
    ids = torch.arange(50, dtype=I32).repeat(6, 1)
    loss, grad = api.compute_distillation(up(x.view(2, 3, 50)), up(ids.view(2, 3, 50)), up(x.view(2, 3, 50)), temperature=1.4)
    assert loss.shape == (2, 3) and grad.shape == (2, 3, 50) and loss.abs().max() < 1e-5 and grad.abs().max() < 1e-5


@pytest.mark.parametrize("polls", [0, 1, 3])
@pytest.mark.parametrize("R,A,dtype", [(2, 9000, F32), (400, 70000, BF16), (40, 150000, BF16)])
def test_distill_waits_that_run_out(api, polls, R, A, dtype):
    """A wait that gives up leaves NaN, the right value or nothing written, and the next call is right."""
    from paper_2608_17641_b200 import binding
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(R, A, device="cuda", generator=g).to(dtype)
    ids = torch.randint(0, A, (R, 7), device="cuda", generator=g, dtype=I32)
    teacher = torch.randn(R, 7, device="cuda", generator=g)
    want = api.compute_distillation(x, ids, teacher)
    fn = binding.rlcs_distill_grad if dtype == F32 else binding.rlcs_distill_grad_bf16
    loss, grad = guarded_empty((R,), F32).fill_(77), guarded_empty((R, A), dtype).fill_(77)
    binding.rlcs_debug_set_wait_polls(polls)
    try:
        fn(x, ids, teacher, loss=loss, dlogits=grad)
        torch.cuda.synchronize()
    finally:
        binding.rlcs_debug_set_wait_polls(-1)
    for got, w in zip((loss, grad), want):
        assert (torch.isnan(got) | (got == w) | (got == 77)).all()
    again = api.compute_distillation(x, ids, teacher)
    assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1])


def test_distill_into_a_buffer_and_on_a_stream(api):
    from paper_2608_17641_b200 import binding
    s = torch.cuda.Stream()
    for A in (50, 300, 3000, 9000):
        x, ids, teacher, _ = distill_inputs(6, A, 5, BF16, A)
        want = binding.rlcs_distill_grad_bf16(up(x), up(ids), up(teacher))
        got = binding.rlcs_distill_grad_bf16(up(x), up(ids), up(teacher), dlogits=strided_rows(torch.zeros(6, A, dtype=BF16), 3, 1))
        only = binding.rlcs_distill_grad_bf16(up(x), up(ids), up(teacher), want_grad=False)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(only, want[0])
        s.wait_stream(torch.cuda.current_stream())
        check_distill(api, x, ids, teacher, stream=s)


# ------------------------------------------------------------------------------------------ pages
def plain_fork(table, lens, sources, free, page):
    B, width = table.shape
    new, come, go, used, seen = [], [], [], 0, set()
    for s in sources:
        row = [-1] * width
        a = b = -1
        if 0 <= s < B:
            n = max(int(lens[s]), 0)
            need = -(-n // page)
            row[:min(need, width)] = [int(v) for v in table[s, :min(need, width)]]
            if s in seen and n % page and need <= width and row[need - 1] >= 0:
                b = max(int(free[used]), -1) if used < len(free) else -1
                a = row[need - 1] if b >= 0 else -1
                row[need - 1] = b
                used += 1
            seen.add(s)
        new.append(row), come.append(a), go.append(b)
    return new, come, go, used


def check_fork(api, table, lens, sources, free, page):
    want = plain_fork(table, lens, sources.tolist(), free.tolist(), page)
    got = api.fork_block_tables(up(table), up(lens), up(sources), up(free), page_size=page)
    assert got[0].shape == (sources.numel(), table.shape[1])
    for g, w in zip(got, (want[0], want[1], want[2], [want[3]])):
        assert np.array_equal(g.cpu().numpy().reshape(-1), np.array(w, dtype=np.int64).reshape(-1))


@pytest.mark.parametrize("page", [1, 3, 16, 100])
@pytest.mark.parametrize("B,N", [(1, 1), (1, 50), (7, 7), (300, 300), (300, 20), (33, 1000), (4096, 4096), (5000, 300), (300, 5000), (5001, 5003)])
def test_fork_sizes(api, B, N, page):
    g = torch.Generator().manual_seed(B + N + page)
    width = 9
    lens = torch.randint(0, width * page + 1, (B,), generator=g, dtype=I32)
    table = torch.randperm(B * width, generator=g).to(I32).view(B, width)
    sources = torch.randint(-1, B + 1, (N,), generator=g, dtype=I32)
    check_fork(api, table, lens, sources, torch.arange(B * width, B * width + N, dtype=I32), page)
    check_fork(api, table, lens, sources, torch.arange(B * width, B * width + N // 5, dtype=I32), page)


def test_fork_edges(api):
    table = ints([[3, 4, 5], [6, 7, 8], [-1, -1, -1], [9, -1, 11]])
    lens = ints([40, 100, 20, 25])                       # longer than the table, missing pages
    for sources in ([0, 0, 0], [1, 1], [2, 2, 2], [3, 3, 3], [-5, 2 ** 31 - 1, 4], [0, 1, 2, 3, 3, 2, 1, 0]):
        check_fork(api, table, lens, ints(sources), ints([20, -1, 22, 23]), 16)
    check_fork(api, table, -lens, ints([0, 1]), ints([]), 16)
    check_fork(api, table, lens, ints([]), ints([1]), 16)
    check_fork(api, torch.zeros(0, 3, dtype=I32), ints([]), ints([0, 1]), ints([1]), 16)
    check_fork(api, torch.zeros(2, 0, dtype=I32), ints([5, 6]), ints([0, 0]), ints([1]), 16)


@pytest.mark.parametrize("layout", ["tokens", "heads", "strided", "gaps"])
@pytest.mark.parametrize("page,Hk,d", [(1, 1, 8), (16, 2, 64), (7, 3, 40), (64, 8, 128), (100, 4, 80)])
def test_copy_pages(api, layout, page, Hk, d):
    g = torch.Generator().manual_seed(page)
    pages = 40
    k, v = (torch.randn(pages, page, Hk, d, generator=g).to(BF16) for _ in range(2))

    def device(t):
        if layout == "heads":
            return up(t.permute(0, 2, 1, 3).contiguous()).permute(0, 2, 1, 3)
        if layout == "strided":
            return up(torch.cat([t, t + 1], 3))[..., :d]
        if layout == "gaps":
            return up(torch.cat([t, t + 1], 0).view(2, pages, page, Hk, d).transpose(0, 1).contiguous())[:, 0]
        return up(t)

    order = torch.randperm(pages, generator=g)
    come, go = order[:15].to(I32), order[15:30].to(I32)
    come[3], go[5], come[7], go[8] = -1, -1, pages, 2 ** 31 - 1
    go[9] = come[9]                                      # onto itself
    want_k, want_v = k.clone(), v.clone()
    for a, b in zip(come.tolist(), go.tolist()):
        if 0 <= a < pages and 0 <= b < pages:
            want_k[b], want_v[b] = k[a], v[a]
    kd, vd = device(k), device(v)
    got = api.copy_pages(kd, vd, up(come), up(go))
    assert got[0] is kd and torch.equal(kd.cpu(), want_k) and torch.equal(vd.cpu(), want_v)
    kd = device(k)
    api.copy_pages(kd, None, up(come), up(go))
    assert torch.equal(kd.cpu(), want_k)


def test_copy_many_pages(api):
    """More pairs than a block lists at a time, most of them none."""
    k = torch.arange(6000, device="cuda")[:, None, None, None].expand(6000, 2, 1, 8).to(BF16).contiguous()
    g = torch.Generator().manual_seed(2)
    order = torch.randperm(6000, generator=g).to(I32)
    come, go = order[:3000].clone(), order[3000:].clone()
    come[torch.rand(3000, generator=g) < 0.7] = -1
    want = k.clone()
    want[go[come >= 0].long().cuda()] = k[come[come >= 0].long().cuda()]
    v = k.clone()
    api.copy_pages(k, v, up(come), up(go))
    assert torch.equal(k, want) and torch.equal(v, want)
    api.copy_pages(k, v, up(ints([])), up(ints([])))


def plain_free(tables, pages, page):
    named = set()
    for table, lens in tables:
        for row, n in zip(table.tolist(), lens.tolist()):
            named.update(row[:-(-max(n, 0) // page)])
    return [p for p in range(pages) if p not in named]


def check_free(api, table, lens, pages, page, prefix=None):
    want = plain_free([(table, lens)] + ([prefix] if prefix is not None else []), pages, page)
    kw = dict(prefix_table=up(prefix[0]), prefix_lens=up(prefix[1])) if prefix is not None else {}
    free, count = api.list_free_pages(up(table), up(lens), num_pages=pages, page_size=page, **kw)
    assert free.shape == (pages,) and count.tolist() == [len(want)]
    assert np.array_equal(free.cpu().numpy(), np.array(want + [-1] * (pages - len(want)), dtype=np.int32))


@pytest.mark.parametrize("page", [1, 16, 100])
@pytest.mark.parametrize("B,pages", [(1, 1), (1, 31), (3, 32), (3, 33), (7, 64), (40, 1000), (300, 5000), (1000, 70001), (5000, 300000)])
def test_free_sizes(api, B, pages, page):
    g = torch.Generator().manual_seed(B + pages)
    width = max(1, min(40, pages // B))
    table = torch.randperm(max(pages, B * width), generator=g)[:B * width].to(I32).view(B, width)
    lens = torch.randint(0, width * page + 2, (B,), generator=g, dtype=I32)
    check_free(api, table, lens, pages, page)
    check_free(api, table, lens, pages, page, (table[: max(1, B // 3)].flip(1).contiguous(), lens[: max(1, B // 3)].contiguous()))
    check_free(api, table, torch.zeros_like(lens), pages, page)


def test_free_edges(api):
    table = ints([[0, 0, 5], [5, -1, 2 ** 31 - 1], [9, 8, 7], [40, 64, -2 ** 31]])
    for pages in (0, 1, 6, 32, 40, 41, 63, 64, 65, 5000):
        check_free(api, table, ints([48, 48, 17, 48]), pages, 16)
        check_free(api, table, ints([-1, 2 ** 31 - 1, 1, 0]), pages, 16)
        check_free(api, torch.zeros(0, 3, dtype=I32), ints([]), pages, 16)
        check_free(api, torch.zeros(2, 0, dtype=I32), ints([5, 6]), pages, 16)


def test_freed_pages_serve_tables_and_forks(api):
    """The list as it is, -1 at its end: what is beyond the free pages has none."""
    table = ints([[0, 1, -1], [2, 3, -1]])
    free, count = api.list_free_pages(up(table), up(ints([20, 32])), num_pages=6, page_size=16)
    assert count.item() == 2 and free.tolist() == [4, 5, -1, -1, -1, -1]
    td = up(table)
    slots, _, _, used = api.build_block_tables(up(ints([20, 32])), up(ints([13, 1])), free, td, page_size=16, num_slots=14)
    assert used.item() == 2 and td.tolist() == [[0, 1, 4], [2, 3, 5]]
    new, come, go, used = api.fork_block_tables(td, up(ints([33, 33])), up(ints([0, 0, 1, 1])), free[2:].contiguous(), page_size=16)
    assert used.item() == 2 and go.tolist() == [-1] * 4 and come.tolist() == [-1] * 4
    assert new.tolist() == [[0, 1, 4], [0, 1, -1], [2, 3, 5], [2, 3, -1]]


# ------------------------------------------------------------------------------------------ together
def test_speculative_operators_in_a_graph(api):
    """A step of all of them, captured once and replayed on new inputs: what direct calls give.  Two graphs share nothing."""
    def inputs(seed):
        cache = Paged(seed, [150, 90], 16, 2, 64, spare=30)
        x, tokens, offsets, u, du, drafts = verify_inputs([5, 3], 700, F32, seed)
        q = torch.randn(8, 4, 64, generator=torch.Generator().manual_seed(seed)).to(BF16)
        _, ids, teacher, _ = distill_inputs(8, 700, 9, F32, seed)
        k, v = cache.k.nan_to_num(), cache.v.nan_to_num()
        return [t.cuda() for t in (q, k, v, cache.table.clamp(0, 45), ints([150, 90]), x, tokens, ints(offsets), u, du, drafts, ids, teacher)]

    def step(q, k, v, table, lens, x, tokens, offsets, u, du, drafts, ids, teacher):
        out, lse = api.chunk_attention(q, k, v, table, offsets, lens, max_new=5)
        new, lp, acc = api.verify_drafts(x, tokens, offsets, u, du, draft_logits=drafts)
        loss, grad = api.compute_distillation(drafts, ids, teacher)
        kept = lens - 4 + acc
        free, count = api.list_free_pages(table, kept, num_pages=k.shape[0], page_size=16)
        forked, come, go, used = api.fork_block_tables(table, kept, acc % 2, free, page_size=16)
        k2, v2 = k.clone(), v.clone()
        api.copy_pages(k2, v2, come, go)
        return out, lse, new, lp, acc, loss, grad, free, count, forked, come, go, used, k2, v2

    fixed = [inputs(1), inputs(2)]
    graphs = []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for f in fixed:
            step(*f)
    torch.cuda.current_stream().wait_stream(side)
    for f in fixed:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = step(*f)
        graphs.append((g, got))
    for seeds in ((3, 4), (5, 6)):
        for f, seed in zip(fixed, seeds):
            for a, b in zip(f, inputs(seed)):
                a.copy_(b)
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for f, (_, got) in zip(fixed, graphs):
            for a, b in zip(got, step(*f)):
                assert torch.equal(a, b)


def test_prepared_calls_repeat_the_direct_ones(api):
    from paper_2608_17641_b200 import binding
    cache = Paged(3, [150, 90], 16, 2, 64)
    x, tokens, offsets, u, du, drafts = verify_inputs([5, 3], 700, F32, 1)
    q = up(torch.randn(8, 4, 64, generator=torch.Generator().manual_seed(7)).to(BF16))
    _, ids, teacher, _ = distill_inputs(8, 700, 9, F32, 2)
    o, table, lens = up(ints(offsets)), up(cache.table), up(ints([150, 90]))
    for fn, args, kw in ((binding.rlcs_chunk_attention_bf16, (q, cache.kd, cache.vd, table, o, lens), dict(scale=0.2)),
                         (binding.rlcs_verify_drafts, (up(x), up(tokens), o, up(u), up(du)), dict(draft_logits=up(drafts))),
                         (binding.rlcs_distill_grad, (up(x), up(ids), up(teacher)), dict(temperature=1.2)),
                         (binding.rlcs_fork_block_tables, (table, lens, up(ints([1, 1, 0])), up(ints([30, 31]))), dict(page_size=16)),
                         (binding.rlcs_free_pages, (table, lens), dict(num_pages=90, page_size=16))):
        call = binding.prepare(fn, *args, **kw)
        want = fn(*args, **kw)
        for _ in range(2):
            for a, b in zip(call(), want):
                assert torch.equal(a, b)


# ------------------------------------------------------------------------------------------ the example
def test_operators_work_together_in_the_example(api):
    """Two rounds of generation: the log-probabilities that verification reported along the way, through pages given back and
    tables forked, against a dense recomputation from the tokens alone.  Logits of up to 10 are bfloat16 on both sides, off by 2^-8 of
    themselves each, from hidden states that are bfloat16 too: 0.16 a token bounds it, a wrong page costs whole units."""
    import os
    import sys
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import speculative_rollout as ex
    generator = torch.Generator(device="cuda").manual_seed(1)
    target, draft = ex.Target(generator), ex.Draft(generator)
    for _ in range(2):
        prompts = torch.randint(0, ex.VOCAB, (ex.ROWS, ex.PROMPT), device="cuda", generator=generator, dtype=torch.int32)
        texts, total, kept, losses = ex.generate(target, draft, prompts, generator, rate=2.0)
        assert len(kept) == len(losses) and all(math.isfinite(v) for v in losses) and 0 <= min(kept) <= max(kept) <= ex.DRAFTS
        for b in range(ex.ROWS):
            text = torch.tensor(texts[b], device="cuda")
            x = target.embed[text].float()
            q = (x @ target.wq.float()).view(-1, ex.HEADS, ex.DIM)
            k, v = (t.repeat_interleave(ex.HEADS // ex.KV_HEADS, 1) for t in (x @ target.wkv.float()).view(-1, 2, ex.KV_HEADS, ex.DIM).unbind(1))
            c = torch.einsum("ihd,jhd->hij", q, k) * ex.DIM ** -0.5
            c = c.masked_fill(torch.ones(len(text), len(text), device="cuda").triu(1).bool(), -math.inf)
            a = torch.einsum("hij,jhd->ihd", torch.softmax(c, -1), v).reshape(len(text), -1)
            lp = torch.log_softmax(torch.tanh(x + a @ target.wo.float()) @ target.out.float(), 1)
            new = torch.arange(ex.PROMPT, len(text), device="cuda")
            want = lp[new - 1, text[new]].sum()
            assert abs(float(total[b] - want)) <= 0.16 * len(new), (b, float(total[b]), float(want))
    # the draft policy's gradient against autograd
    before, last = (torch.randint(0, ex.VOCAB, (20,), device="cuda", generator=generator) for _ in range(2))
    teacher = torch.randn(20, ex.VOCAB, device="cuda", generator=generator)
    top, ids = teacher.topk(ex.TOP, 1)
    features = draft.features(before, last)
    out = draft.out.double().requires_grad_()
    lq = torch.log_softmax(features.double() @ out, 1)
    p = torch.softmax(top.double(), 1)
    ((p * (p.log() - lq.gather(1, ids))).sum() / 20).backward()
    _, grad = api.compute_distillation(features @ draft.out, ids.int(), top, scale=1 / 20)
    # products of 256 fp32 terms: 2^-16 of their size
    assert (features.t() @ grad - out.grad).abs().max() <= 2.0 ** -15 * out.grad.abs().max() + 1e-6
