"""The sensitivity map's operators at sizes and values on both sides of where their kernels change what they do."""
import pytest
import torch

import map_reference as ref
import paper_2303_10837_b200 as he
import synthetic_inputs as si
from test_gpu_map_operators import check_log_probs, gen, logits_of, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return he.he_ctx_create(8192, list(si.PRIMES_N8192), 40)


def widths_about(threads, dtype):
    """Columns of rows that a block of so many threads, each with 64 bytes, just holds at once, and of the next ones."""
    per = 16 // ref.DTYPES[dtype].itemsize
    full = threads * 4 * per
    if threads == 32:
        return list(range(full - 2 * per, full + 2))
    return [full - 2 * per, full - per - 1, full - per + 1, full - 1, full, full + 1]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("threads", [32, 64, 96, 128, 256])
def test_alternatives_of_rows_that_just_fill_a_piece(ctx, dtype, threads):
    """Rows at every distance from 16 bytes: whether a row fills a block's piece depends on it."""
    for V in widths_about(threads, dtype):
        z, y = logits_of(4, V, dtype, 31 * V, False)
        few = z.round().masked_fill(torch.rand(4, V, generator=gen(V), device="cuda") < 0.9, float("-inf"))
        ids = [ref.log_probs(t, y, 64)[4] for t in (z, few)]
        per = 16 // z.element_size()
        for shift in range(per):
            views = [ref.strided(t, -V % per + per, shift) for t in (z, few)]
            for top in (31, 32, 33, 64):
                for view, want in zip(views, ids):
                    got = he.he_token_log_probs(ctx, view, y, top=top)[4]
                    assert torch.equal(got, want[:, :top]), (V, shift, top)
            if V % per == per - 1:
                check_log_probs(ctx, views[0], y, 64)
