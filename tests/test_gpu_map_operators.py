"""The sensitivity map's operators against their definitions in 64 bits."""
import pytest
import torch

import map_reference as ref
import paper_2303_10837_b200 as he
import synthetic_inputs as si

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def ctx():
    return he.he_ctx_create(8192, list(si.PRIMES_N8192), 40)


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def logits_of(rows, V, dtype, seed, masked):
    g = gen(seed)
    z = randn(g, rows, V) * 3
    if masked:
        z.masked_fill_(torch.rand(rows, V, generator=g, device="cuda") < 0.4, -INF)
        z[0].fill_(-INF)
    y = torch.randint(0, V, (rows,), generator=g, device="cuda")
    y[rows // 2] = -100
    return z.to(ref.DTYPES[dtype]), y


def check_log_probs(ctx, z, y, top):
    logp, lse, entropy, top_logp, ids = he.he_token_log_probs(ctx, z, y, top=top)
    w_logp, w_lse, w_entropy, w_top, w_ids = ref.log_probs(z, y, top)
    tl, te = ref.log_probs_tolerance(z, w_lse, w_entropy)
    ref.close(lse, w_lse, tl, "lse")
    ref.close(logp, w_logp, tl, "logp")
    ref.close(entropy, w_entropy, te, "entropy")
    if top:
        assert torch.equal(ids, w_ids)
        ref.close(top_logp, w_top, tl[:, None].expand_as(w_top), "top_logp")
    else:
        assert top_logp is None and ids is None
    return lse, entropy, ids


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V,top", [(1, 1, 1), (3, 7, 7), (5, 100, 20), (2, 255, 64), (33, 1000, 5), (300, 1024, 0), (4, 8193, 32), (1, 50257, 64),
                                        (7, 65536, 8), (1, 131072, 20), (700, 4097, 3)])
@pytest.mark.parametrize("masked", [False, True])
def test_log_probs(ctx, dtype, rows, V, top, masked):
    z, y = logits_of(rows, V, dtype, 100 + V + rows, masked)
    check_log_probs(ctx, z, y, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (3, 0), (8, 8), (5, 3)])
def test_log_probs_of_strided_rows(ctx, dtype, pad, shift):
    z, y = logits_of(9, 2049, dtype, 7, False)
    check_log_probs(ctx, ref.strided(z, pad, shift), y, 6)
    check_log_probs(ctx, z[:1].expand(5, -1), y[:5].contiguous(), 6)


@pytest.mark.parametrize("V", [40, 5000, 40000])
def test_alternatives_of_equal_and_of_sorted_values(ctx, V):
    y = torch.zeros(6, dtype=torch.int64, device="cuda")
    z = torch.zeros(6, V, device="cuda")
    z[1] = torch.arange(V, device="cuda")                          # every value is a new best one
    z[2] = -torch.arange(V, device="cuda").float()
    z[3] = torch.arange(V, device="cuda") % 3
    z[4] = -INF
    z[4, V // 2] = 1.0
    z[5] = torch.where(torch.arange(V, device="cuda") % 2 == 0, 0.0, -0.0)
    for top in (1, 17, 32):
        check_log_probs(ctx, z, y, top)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,V,top", [(3, 100, 64), (5, 9000, 20), (2, 131072, 64), (900, 5003, 8), (1, 20000, 1)])
def test_alternatives_among_few_values(ctx, dtype, rows, V, top):
    """Masks that leave fewer tokens than alternatives, equal logits, logits of few sizes: the lowest indices of equal ones."""
    g, t = gen(V + top), ref.DTYPES[dtype]
    z = randn(g, rows, V) * 2
    y = torch.randint(0, V, (rows,), generator=g, device="cuda")
    sparse = torch.rand(rows, V, generator=g, device="cuda") < 1 - 30 / V
    late = torch.arange(V, device="cuda").expand(rows, V) < V - 5
    for x in (z.masked_fill(sparse, -INF), z.masked_fill(sparse, torch.finfo(t).min), z.masked_fill(late, -INF), torch.full_like(z, 0.5),
              z.round(), z.clamp(max=0.0), torch.where(late, -0.0, 0.0), z.masked_fill(late, float("nan")).masked_fill(~late, 1.0)):
        x = x.to(t)
        for view in (x, ref.strided(x, 3, 1)):
            _, _, _, _, ids = he.he_token_log_probs(ctx, view, y, top=top)
            assert torch.equal(ids, ref.log_probs(x, y, top)[4])
        if not torch.isnan(x).any():
            check_log_probs(ctx, x, y, top)


def test_log_probs_of_rows_that_are_not_finite(ctx):
    z, y = logits_of(5, 3000, "f32", 3, False)
    y[:] = 5
    z[0, 17] = float("nan")
    z[1, 2999] = INF
    z[2].fill_(-INF)
    z[3] += 1e30
    logp, lse, entropy, top_logp, ids = he.he_token_log_probs(ctx, z, y, top=4)
    for t in (logp, lse, entropy):
        assert torch.isnan(t[0]) and torch.isnan(t[1])
    assert torch.isnan(top_logp[:2]).all()
    check_log_probs(ctx, z[2:], y[2:], 4)
    assert ((ids >= 0) & (ids < 3000)).all() and 17 not in ids[0].tolist()
    # a target outside the vocabulary shows
    y[4] = 3000
    assert torch.isnan(he.he_token_log_probs(ctx, z, y)[0][4])


def test_log_probs_keep_their_digits_far_from_zero(ctx):
    z, y = logits_of(4, 4000, "f32", 12, False)
    near = he.he_token_log_probs(ctx, z, y)
    far = he.he_token_log_probs(ctx, (z * 64).round() / 64 + 4096.0, y)
    base = he.he_token_log_probs(ctx, (z * 64).round() / 64, y)
    assert torch.equal(far[0], base[0]) and torch.equal(far[2], base[2])
    assert near[0].shape == (4,)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 9), (6, 1000), (40, 8193), (2, 50257), (1, 131072)])
@pytest.mark.parametrize("form", ["logp", "entropy", "top", "all"])
def test_log_probs_gradient(ctx, dtype, rows, V, form):
    z, y = logits_of(rows, V, dtype, 900 + V + rows, masked=V > 1 and rows > 1)
    g = gen(5)
    top = min(V, 6) if form in ("top", "all") else 0
    _, lse, entropy, _, ids = he.he_token_log_probs(ctx, z, y, top=top)
    dlogp = randn(g, rows)
    dent = randn(g, rows) if form in ("entropy", "all") else None
    dtop = randn(g, rows, top) if top else None
    want, tol = ref.log_probs_grad(z, y, lse, dlogp, entropy, dent, ids if top else None, dtop)
    args = dict(entropy=entropy, dentropy=dent, top_ids=ids if top else None, dtop=dtop)
    got = he.he_token_log_probs_backward(ctx, z, y, lse, dlogp, **args)
    ref.close(got, want, tol + ref.rounding(want, z.dtype) + 2.0 ** -126, "dlogits")
    # rows at other alignments, and in place
    for pad, shift in ((0, 1), (5, 2)):
        zs = ref.strided(z, pad, shift)
        assert torch.equal(he.he_token_log_probs_backward(ctx, zs, y, lse, dlogp, **args), got)
        out = he.he_token_log_probs_backward(ctx, zs, y, lse, dlogp, out=zs, **args)
        assert out is zs and torch.equal(zs, got)


def test_log_probs_gradient_of_an_alternative_named_twice_and_of_the_target(ctx):
    z, y = logits_of(3, 500, "f32", 8, False)
    y[:] = torch.tensor([4, 9, -1])
    ids = torch.tensor([[4, 4, 4], [1, 9, 1], [499, 0, 499]], device="cuda")
    dtop, dlogp = randn(gen(1), 3, 3), randn(gen(2), 3)
    _, lse, entropy, _, _ = he.he_token_log_probs(ctx, z, y)
    want, tol = ref.log_probs_grad(z, y, lse, dlogp, entropy, None, ids, dtop)
    ref.close(he.he_token_log_probs_backward(ctx, z, y, lse, dlogp, top_ids=ids, dtop=dtop), want, tol + ref.rounding(want, z.dtype), "dlogits")


def test_log_probs_gradient_where_nothing_flows(ctx):
    z, y = logits_of(4, 700, "f32", 8, False)
    y[:] = torch.tensor([3, -100, 5, 6])
    z[1].fill_(float("nan"))                  # a padded row
    z[2].fill_(-INF)
    _, lse, _, _, _ = he.he_token_log_probs(ctx, z, y)
    d = he.he_token_log_probs_backward(ctx, z, y, lse, torch.ones(4, device="cuda"))
    assert (d[1] == 0).all() and (d[2] == 0).all() and (d[0] != 0).any()
    y[3] = 700
    assert torch.isnan(he.he_token_log_probs_backward(ctx, z, y, lse, torch.ones(4, device="cuda"))[3]).all()


def test_log_probs_gradient_against_differences(ctx):
    rows, V, h = 6, 300, 2.0 ** -6
    z, y = logits_of(rows, V, "f32", 21, False)
    v = randn(gen(3), rows, V)
    _, lse, entropy, _, _ = he.he_token_log_probs(ctx, z, y)
    one = torch.ones(rows, device="cuda")
    up, down = he.he_token_log_probs(ctx, z + h * v, y), he.he_token_log_probs(ctx, z - h * v, y)
    d = (he.he_token_log_probs_backward(ctx, z, y, lse, one).double() * v.double()).sum(1)
    e = (he.he_token_log_probs_backward(ctx, z, y, lse, 0 * one, entropy=entropy, dentropy=one).double() * v.double()).sum(1)
    # a central difference is off by h^2 / 6 of a third derivative (twice that of the definition here), and by 1e-5 / h: values are off by at most 1e-5
    at = lambda c, i: ref.log_probs(z.double() + c * h * v.double(), y, 1)[i]   # noqa: E731
    for i, g in ((0, d), (2, e)):
        third = (at(2, i) - 2 * at(1, i) + 2 * at(-1, i) - at(-2, i)) / (2 * h ** 3)
        off = ((up[i] - down[i]).double() / (2 * h) - g).abs()
        assert bool((off <= 2 * third.abs() * h * h / 6 + h ** 4 * 1e3 + 1e-5 / h).all())


# ---------------------------------------------------------------- layer norm

WIDTHS = [(1, 1), (5, 2), (3, 7), (17, 32), (9, 100), (2, 257), (33, 768), (130, 1024), (3, 4096), (2, 5000), (2, 8192), (1, 10001), (2, 40000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", WIDTHS)
@pytest.mark.parametrize("weights", ["f32", "own", "none"])
def test_layer_norm(ctx, dtype, rows, width, weights):
    g, t = gen(width), ref.DTYPES[dtype]
    x = (randn(g, rows, width) * 2 + 0.5).to(t)
    kind = torch.float32 if weights == "f32" else t
    w = None if weights == "none" else randn(g, width).to(kind)
    b = None if weights == "none" else randn(g, width).to(kind)
    (y, ty), (m, tm), (r, tr) = ref.norm(x, w, b, 1e-5)
    for case in (x, ref.strided(x, 0, 1), ref.strided(x, 16, 0), ref.strided(x, 3, 2)):
        gy, gm, gr = he.he_layer_norm(ctx, case, w, b, eps=1e-5)
        ref.close(gm, m, tm + 2.0 ** -140, "mean")
        ref.close(gr, r, tr + ref.rounding(r, torch.float32), "rstd")
        ref.close(gy, y, ty + ref.rounding(y, t), "y")
    same = x.clone()
    out, _, _ = he.he_layer_norm(ctx, same, w, b, eps=1e-5, out=same)
    assert out is same and torch.equal(same, he.he_layer_norm(ctx, x, w, b, eps=1e-5)[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", [(30000, 520), (28500, 1024), (20000, 1032), (19001, 2048), (14300, 2056), (14300, 4096)])
def test_layer_norm_of_many_rows(ctx, dtype, rows, width):
    g, t = gen(rows + width), ref.DTYPES[dtype]
    x = (randn(g, rows, width) * 2 + randn(g, width)).to(t)
    w, b = randn(g, width), randn(g, width).to(t)
    for weight, bias in ((w, w), (None, b), (None, None)):
        y, mean, rstd = he.he_layer_norm(ctx, x, weight, bias)
        for lo in range(0, rows, 5000):
            (wy, ty), (wm, tm), (wr, tr) = ref.norm(x[lo:lo + 5000], weight, bias, 1e-5)
            ref.close(y[lo:lo + 5000], wy, ty + ref.rounding(wy, t), "y")
            ref.close(mean[lo:lo + 5000], wm, tm, "mean")
            ref.close(rstd[lo:lo + 5000], wr, tr, "rstd")
    out, _, _ = he.he_layer_norm(ctx, x, w, w)
    room = torch.zeros(rows, width + 8, dtype=t, device="cuda")
    room[:, :width] = x
    got = he.he_layer_norm(ctx, room[:, :width], w, w, out=room[:, :width])[0]
    assert torch.equal(got, out) and (room[:, width:] == 0).all()


def test_layer_norm_of_equal_values_and_of_rows_that_are_not_finite(ctx):
    x = torch.full((4, 300), 3.0, device="cuda")
    x[1, 5], x[2, 7] = float("nan"), INF
    y, m, r = he.he_layer_norm(ctx, x, eps=1e-5)
    assert (y[0] == 0).all() and (y[3] == 0).all() and float(m[0]) == 3.0
    assert torch.isnan(y[1]).all() and torch.isnan(y[2]).all()
    empty = he.he_layer_norm(ctx, x[:0])
    assert empty[0].shape == (0, 300) and empty[1].shape == (0,)


def cuts_of(kind, rows):
    if kind == "all":
        return None
    if kind == "one":
        return [0, rows]
    if kind == "rows":
        return list(range(rows + 1))
    if kind == "padded":                                       # rows before, empty samples, rows behind
        a = min(3, rows)
        return [a, a, a + (rows - a) // 3, a + (rows - a) // 3, a + (rows - a) // 3, rows - min(2, rows - a)]
    if kind == "none":
        return [0]
    g = torch.Generator()
    g.manual_seed(rows)
    n = max(1, rows // 5)
    return [0] + torch.randint(0, rows + 1, (n,), generator=g).sort().values.tolist() + [rows]


def offsets(cuts):
    return None if cuts is None else torch.tensor(cuts, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,width", WIDTHS + [(2000, 64), (1500, 257), (700, 1024), (5000, 8)])
@pytest.mark.parametrize("kind", ["all", "one", "rows", "padded", "ragged", "none"])
def test_layer_norm_backward(ctx, dtype, rows, width, kind):
    g, t = gen(width + rows), ref.DTYPES[dtype]
    x, dy, w = (randn(g, rows, width) * 2 + 0.5).to(t), randn(g, rows, width).to(t), randn(g, width)
    cuts = cuts_of(kind, rows)
    _, mean, rstd = he.he_layer_norm(ctx, x, w, None)
    (dx, tx), (dw, tw), (db, tb) = ref.norm_grad(dy, x, mean, rstd, w, cuts)
    for pad, shift in ((0, 0), (0, 1), (16, 0)):
        xs, ds = (x, dy) if (pad, shift) == (0, 0) else (ref.strided(x, pad, shift), ref.strided(dy, pad, shift))
        gx, gw, gb = he.he_layer_norm_backward(ctx, ds, xs, mean, rstd, w, samples=offsets(cuts))
        ref.close(gx, dx, tx, "dx")
        ref.close(gw, dw, tw + ref.rounding(dw, torch.float32), "dweight")
        ref.close(gb, db, tb + ref.rounding(db, torch.float32), "dbias")


def test_layer_norm_backward_without_weight_and_in_the_inputs_type(ctx):
    g = gen(4)
    x, dy, w = (randn(g, 50, 640).bfloat16() for _ in range(3))
    _, mean, rstd = he.he_layer_norm(ctx, x)
    for weight in (None, w[0].contiguous()):
        got = he.he_layer_norm_backward(ctx, dy, x, mean, rstd, weight)
        for a, (b, tol) in zip(got, ref.norm_grad(dy, x, mean, rstd, weight, None)):
            ref.close(a, b, tol, "gradient")
    dx, dw, db = he.he_layer_norm_backward(ctx, dy[:0], x[:0], mean[:0], rstd[:0])
    assert dx.shape == (0, 640) and (dw == 0).all() and (db == 0).all()


def test_padding_does_not_reach_the_sums(ctx):
    g = gen(6)
    x, dy = randn(g, 200, 96), randn(g, 200, 96)
    cuts = [4, 60, 60, 151]
    _, mean, rstd = he.he_layer_norm(ctx, x)
    _, dw, db = he.he_layer_norm_backward(ctx, dy, x, mean, rstd, samples=offsets(cuts))
    sw, sb = he.he_linear_sensitivity(ctx, x, dy, samples=offsets(cuts))
    x[:4], x[151:], dy[:4], dy[151:] = float("nan"), INF, -INF, float("nan")
    _, dw2, db2 = he.he_layer_norm_backward(ctx, dy, x, mean, rstd, samples=offsets(cuts))
    sw2, sb2 = he.he_linear_sensitivity(ctx, x, dy, samples=offsets(cuts))
    for a, b in ((dw, dw2), (db, db2), (sw, sw2), (sb, sb2)):
        assert torch.equal(a, b)


def test_layer_norm_gradient_against_differences(ctx):
    rows, width, h = 4, 50, 2.0 ** -7
    g = gen(9)
    x, w, b, dy, v = randn(g, rows, width), randn(g, width), randn(g, width), randn(g, rows, width), randn(g, rows, width)
    _, mean, rstd = he.he_layer_norm(ctx, x, w, b)
    dx, dw, db = he.he_layer_norm_backward(ctx, dy, x, mean, rstd, w)
    value = lambda *a: float((he.he_layer_norm(ctx, *a)[0].double() * dy.double()).sum())   # noqa: E731
    # off by h^2 / 6 of the third derivative (twice that of the definition here; in the weights there is none), and by 1e-4 / h: values are off by at most 1e-4
    at = lambda c: float((ref.norm(x.double() + c * h * v.double(), w, b, 1e-5)[0][0] * dy.double()).sum())   # noqa: E731
    slack = 1e-4 / h
    third = abs(at(2) - 2 * at(1) + 2 * at(-1) - at(-2)) / (2 * h ** 3)
    assert abs((value(x + h * v, w, b) - value(x - h * v, w, b)) / (2 * h) - float((dx.double() * v.double()).sum())) < 2 * third * h * h / 6 + h ** 4 * 1e4 + slack
    assert abs((value(x, w + h * v[0], b) - value(x, w - h * v[0], b)) / (2 * h) - float((dw.double() * v[0].double()).sum())) < slack
    assert abs((value(x, w, b + h * v[0]) - value(x, w, b - h * v[0])) / (2 * h) - float((db.double() * v[0].double()).sum())) < slack


# ---------------------------------------------------------------- linear layers

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,inputs,outputs", [(1, 1, 1), (7, 3, 5), (40, 64, 64), (100, 65, 130), (65, 128, 256), (200, 333, 101), (129, 256, 128), (600, 264, 520),
                                                 (33, 1000, 8)])
@pytest.mark.parametrize("kind", ["all", "one", "rows", "padded", "ragged", "none"])
def test_linear_sensitivity(ctx, dtype, rows, inputs, outputs, kind):
    g, t = gen(rows + inputs), ref.DTYPES[dtype]
    x, dy = randn(g, rows, inputs).to(t), randn(g, rows, outputs).to(t)
    cuts = cuts_of(kind, rows)
    (w, tw), (b, tb) = ref.linear(x, dy, cuts)
    for pad, shift in ((0, 0), (0, 1), (16, 0)):
        xs, ds = (x, dy) if (pad, shift) == (0, 0) else (ref.strided(x, pad, shift), ref.strided(dy, pad, shift))
        gw, gb = he.he_linear_sensitivity(ctx, xs, ds, samples=offsets(cuts))
        ref.close(gw, w, tw, "weight")
        ref.close(gb, b, tb, "bias")
    # added to a part of a map that is not aligned
    room = torch.full((outputs * inputs + 1,), 2.0, device="cuda")
    out = room[1:].view(outputs, inputs)
    out_bias = torch.full((outputs,), 3.0, device="cuda")
    he.he_linear_sensitivity(ctx, x, dy, samples=offsets(cuts), out=out, out_bias=out_bias, accumulate=True)
    ref.close(out, w + 2.0, tw + ref.rounding(w + 2.0, torch.float32), "added weight")
    ref.close(out_bias, b + 3.0, tb + ref.rounding(b + 3.0, torch.float32), "added bias")
    assert float(room[0]) == 2.0
    only, none = he.he_linear_sensitivity(ctx, x, dy, samples=offsets(cuts), bias=False)
    assert none is None
    ref.close(only, w, tw, "weight alone")


def test_linear_sensitivity_of_a_long_sample(ctx):
    g = gen(31)
    x, dy = randn(g, 5000, 192).bfloat16(), randn(g, 5000, 160).bfloat16()
    for cuts in ([0, 5000], [0, 10, 4100, 4990], None):
        (w, tw), (b, tb) = ref.linear(x, dy, cuts)
        gw, gb = he.he_linear_sensitivity(ctx, x, dy, samples=offsets(cuts))
        ref.close(gw, w, tw, "weight")
        ref.close(gb, b, tb, "bias")
        # and as near as fp32 sums are on the whole
        assert float((gw.double() - w).norm() / w.norm()) < 2e-6


@pytest.mark.parametrize("inputs,outputs", [(512, 512), (4096, 1024), (640, 2000), (2048, 129)])
@pytest.mark.parametrize("lengths", [[300, 600, 64, 520, 600], [17, 128, 300, 520, 64, 33, 600, 1, 16, 15], [1, 2, 3, 16, 17], [128], [2000, 5, 700]])
def test_linear_sensitivity_of_many_samples_is_exact_in_whole_numbers(ctx, inputs, outputs, lengths):
    """Sums of whole numbers below 2^24 have no rounding: every order of the work gives the same, whatever waits for what inside the kernel."""
    import random
    rng = random.Random(len(lengths) + inputs)
    lens = [rng.choice(lengths) for _ in range(min(60, 20000 // max(lengths) + 8))]
    g = gen(inputs)
    x = torch.randint(-2, 3, (sum(lens), inputs), generator=g, device="cuda").bfloat16()
    dy = torch.randint(-2, 3, (sum(lens), outputs), generator=g, device="cuda").bfloat16()
    cuts = [0]
    for n in lens:
        cuts.append(cuts[-1] + n)
    want = torch.zeros(outputs, inputs, device="cuda")
    for lo, hi in zip(cuts, cuts[1:]):
        want += (dy[lo:hi].float().T @ x[lo:hi].float()).abs()
    for _ in range(4):
        assert torch.equal(he.he_linear_sensitivity(ctx, x, dy, samples=offsets(cuts))[0], want)
    alone = (dy.float().abs().T @ x.float().abs())
    assert torch.equal(he.he_linear_sensitivity(ctx, x, dy)[0], alone)
    assert he.he_ctx_status(ctx) == 0


def test_linear_sensitivity_of_no_rows(ctx):
    x, dy = torch.empty(0, 8, device="cuda"), torch.empty(0, 5, device="cuda")
    for samples in (None, offsets([0]), offsets([0, 0, 0])):
        w, b = he.he_linear_sensitivity(ctx, x, dy, samples=samples)
        assert w.shape == (5, 8) and (w == 0).all() and (b == 0).all()


def test_offsets_that_make_no_sense_stay_in_bounds(ctx):
    """Unspecified sums, but no access outside: the kernels clamp what they read (in their row loops)."""
    g = gen(2)
    x, dy = randn(g, 50, 40), randn(g, 50, 24)
    _, mean, rstd = he.he_layer_norm(ctx, x)
    for bad in ([0, 1000, 20], [-5, 10, 50], [30, 10, 0], [50, 50, 2147483647], [-2147483648, 7, 3]):
        w, b = he.he_linear_sensitivity(ctx, x, dy, samples=offsets(bad))
        assert w.shape == (24, 40) and b.shape == (24,)
        he.he_layer_norm_backward(ctx, x, x, mean, rstd, samples=offsets(bad))
    torch.cuda.synchronize()
    want, tol = ref.linear(x, dy, [0, 50])[0]
    ref.close(he.he_linear_sensitivity(ctx, x, dy, samples=offsets([0, 50]))[0], want, tol, "weight")


# ---------------------------------------------------------------- streams, graphs, repeated calls

def all_calls(ctx, s):
    logp, lse, entropy, top_logp, ids = he.he_token_log_probs(ctx, s["z"], s["y"], top=5)
    d = he.he_token_log_probs_backward(ctx, s["z"], s["y"], lse, s["one"], entropy=entropy, dentropy=s["one"])
    y, mean, rstd = he.he_layer_norm(ctx, s["x"], s["w"], s["w"])
    back = he.he_layer_norm_backward(ctx, s["dy"], s["x"], mean, rstd, s["w"], samples=s["cuts"])
    linear = he.he_linear_sensitivity(ctx, s["x"], s["dy"], samples=s["cuts"])
    return [logp, lse, entropy, top_logp, ids, d, y, mean, rstd, *back, *linear]


def state(seed, dtype=torch.bfloat16):
    g = gen(seed)
    return {"z": randn(g, 300, 2000).to(dtype), "y": torch.randint(0, 2000, (300,), generator=g, device="cuda"), "one": torch.ones(300, device="cuda"),
            "x": randn(g, 300, 256).to(dtype), "dy": randn(g, 300, 256).to(dtype), "w": randn(g, 256), "cuts": offsets([0, 50, 51, 200, 290])}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_same_bits_again_on_another_stream_and_from_a_graph(ctx, dtype):
    s = state(1, dtype)
    want = [t.clone() for t in all_calls(ctx, s)]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(want, all_calls(ctx, s)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = all_calls(ctx, s)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = all_calls(ctx, s)
    other = state(2, dtype)
    for k in s:
        s[k].copy_(other[k])
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, all_calls(ctx, s)))


def test_two_streams_at_once(ctx):
    states = [state(3), state(4)]
    want = [[t.clone() for t in all_calls(ctx, s)] for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for _ in range(5):
        got = []
        for s, st in zip(states, streams):
            with torch.cuda.stream(st):
                got.append(all_calls(ctx, s))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
