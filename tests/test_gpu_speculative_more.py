"""Operators of speculative rollouts and distillation on the GPU: what a call's company must not change, pages shared by cut-back branches,
and rows and weights at the edges of what the formulas say.

Tolerances count roundings: a bfloat16 result is off by at most 2^-8 of its value (half a step), a fp32 one by 2^-24."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _util import guarded_empty  # noqa: E402
from test_gpu_operators import BF16, F32, up  # noqa: E402
from test_gpu_speculative import I32, Paged, api, ints, plain_chunks  # noqa: E402,F401


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
