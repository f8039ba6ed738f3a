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


@pytest.mark.parametrize("size", [1e17, 1e19, 1e30, 2.0 ** 117])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_gradients_of_the_entropy_and_masked_logits(ctx, dtype, size):
    """p_j (ln p_j + H) is 0 where p_j is, whatever gradient it is multiplied by."""
    z, y = logits_of(5, 3000, dtype, 19, True)
    z[1:, 1::7] = torch.finfo(z.dtype).min
    lse, entropy, ids = check_log_probs(ctx, z, y, 3)
    g = gen(6)
    dlogp, dent, dtop = randn(g, 5) * size, randn(g, 5) * size, randn(g, 5, 3) * size
    hit = torch.zeros_like(z, dtype=torch.bool).scatter_(1, y.clamp(min=0)[:, None], True).scatter_(1, ids, True)
    for top in ({}, {"top_ids": ids, "dtop": dtop}):
        got = he.he_token_log_probs_backward(ctx, z, y, lse, dlogp, entropy=entropy, dentropy=dent, **top)
        want, tol = ref.log_probs_grad(z, y, lse, dlogp, entropy, dent, top.get("top_ids"), top.get("dtop"))
        # a p below 2^-126 may count as 0, and with it what it is multiplied by: at most 100 times 5 sizes, or 2^9
        ref.close(got, want, tol + ref.rounding(want, z.dtype) + 2.0 ** -117 * size, "dlogits")
        assert (got[(z < -1e30) & ~hit] == 0).all()


def test_alternatives_outside_the_vocabulary(ctx):
    """Their gradients flow off the other logits, as the formula says, and reach none."""
    z, y = logits_of(3, 700, "f32", 4, False)
    y[:] = torch.tensor([3, -1, 699])
    _, lse, _, _, ids = he.he_token_log_probs(ctx, z, y, top=4)
    dlogp, dtop = randn(gen(1), 3), randn(gen(2), 3, 4)
    ids[0, 1], ids[1, 2], ids[2, 3] = -1, 700, 2 ** 40
    got = he.he_token_log_probs_backward(ctx, z, y, lse, dlogp, top_ids=ids, dtop=dtop)
    # as many columns more as it takes, with p = 0
    inside = torch.where((ids < 0) | (ids >= 700), torch.full_like(ids, 700), ids)
    more = torch.cat([z, torch.full((3, 1), float("-inf"), device="cuda")], 1)
    want, tol = ref.log_probs_grad(more, y, lse, dlogp, None, None, inside, dtop)
    ref.close(got, want[:, :700], (tol + ref.rounding(want, z.dtype) + 2.0 ** -126)[:, :700], "dlogits")


@pytest.mark.parametrize("alone", [False, True])
def test_linear_map_of_infinities(ctx, alone):
    """16-bit ones give infinite entries, those of fp32 entries that are not numbers; either in their own rows and columns alone."""
    g = gen(8)
    x, dy = torch.randint(1, 4, (50, 40), generator=g, device="cuda").float(), torch.randint(1, 4, (50, 24), generator=g, device="cuda").float()
    x[7, 3] = float("inf")
    dy[30, 5] = -float("inf")
    cuts = None if alone else torch.tensor([0, 20, 45], dtype=torch.int32, device="cuda")
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        w, b = he.he_linear_sensitivity(ctx, x.to(dtype), dy.to(dtype), samples=cuts)
        hit = torch.zeros_like(w, dtype=torch.bool)
        hit[:, 3] = hit[5, :] = True
        assert torch.isfinite(w[~hit]).all() and b[5] == float("inf") and torch.isfinite(b[:5]).all() and torch.isfinite(b[6:]).all()
        assert (torch.isnan(w[hit]) if dtype == torch.float32 else torch.isinf(w[hit])).all()


@pytest.mark.parametrize("exponent", [-109, -121, -129])
def test_linear_map_of_the_smallest_values(ctx, exponent):
    """Three pieces of bf16 hold a value of 2^-110 or more, and smaller ones to half of bf16's smallest step, 2^-134."""
    g = gen(11)
    dy = (torch.rand(64, 32, generator=g, device="cuda") + 1) * 2.0 ** -60 * 2.0 ** (exponent + 60)
    x = (torch.rand(64, 48, generator=g, device="cuda") + 1) * 2.0 ** 60
    for cuts in (None, [0, 20, 20, 64]):
        got = he.he_linear_sensitivity(ctx, x, dy, samples=None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device="cuda"))[0]
        want, tol = ref.linear(x, dy, cuts)[0]
        ref.close(got, want, tol + 2.0 ** -134 * x.double().sum(0), "map")
