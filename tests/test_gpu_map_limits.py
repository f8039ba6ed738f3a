"""The sensitivity map's operators at the ends of what their calls allow: offsets past 32 bits, long rows, many rows, the type's lowest value,
first calls inside a capture and from other threads."""
import math
import subprocess
import sys
import threading

import pytest
import torch

import map_reference as ref
import paper_2303_10837_b200 as he
import synthetic_inputs as si
from test_gpu_map_operators import all_calls, check_log_probs, gen, logits_of, offsets, randn, state

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return he.he_ctx_create(8192, list(si.PRIMES_N8192), 40)


def far_apart(t, unit):
    """The matrix with rows so far apart, at multiples of `unit`, that the last ones begin past 2^32 elements."""
    rows, cols = t.shape
    stride = (2 ** 32 // (rows - 1) + 8 + unit - 1) // unit * unit
    room = torch.empty((rows - 1) * stride + cols, dtype=t.dtype, device="cuda")
    view = room.as_strided((rows, cols), (stride, 1))
    view.copy_(t)
    return view


@pytest.mark.parametrize("unit", [1, 8])
def test_rows_past_32_bits(ctx, unit):
    g = gen(1)
    z, y = logits_of(4, 5000, "bf16", 2, True)
    far, one = far_apart(z, unit), torch.ones(4, device="cuda")
    lse, _, _ = check_log_probs(ctx, far, y, 7)
    want, tol = ref.log_probs_grad(z, y, lse, one, None, None, None, None)
    assert he.he_token_log_probs_backward(ctx, far, y, lse, one, out=far) is far
    ref.close(far, want, tol + ref.rounding(want, z.dtype) + 2.0 ** -126, "dlogits")
    del far
    x, dy = randn(g, 4, 1000).bfloat16(), randn(g, 4, 1000).bfloat16()
    cuts = [0, 1, 4]
    for width in (1000, 999):
        x, dy = x[:, :width].contiguous(), dy[:, :width].contiguous()
        far = far_apart(x, unit)
        _, mean, rstd = he.he_layer_norm(ctx, x)
        for got, (want, tol) in zip(he.he_layer_norm_backward(ctx, dy, far, mean, rstd, samples=offsets(cuts)), ref.norm_grad(dy, x, mean, rstd, None, cuts)):
            ref.close(got, want, tol, "backward")
        for c in (cuts, None):
            want, tol = ref.linear(x, dy, c)[0]
            ref.close(he.he_linear_sensitivity(ctx, far, dy, samples=offsets(c) if c else None)[0], want, tol, "map")
        want, tol = ref.norm(x, None, None, 1e-5)[0]
        ref.close(he.he_layer_norm(ctx, far, out=far)[0], want, tol + ref.rounding(want, x.dtype), "norm")
        del far


def test_a_row_of_many_values(ctx):
    """2^28 values and some, of thirteen sizes: their numbers give the results."""
    V = 2 ** 28 + 13
    kind = torch.arange(V, device="cuda").remainder_(13)
    z = ((kind - 9).float() * 0.5).bfloat16()
    z[V - 1] = 4.0
    z[12345] = 3.5
    count = torch.bincount(kind, minlength=13).double()
    del kind
    value = (torch.arange(13, device="cuda").double() - 9) * 0.5
    for at, was in ((V - 1, (V - 1) % 13), (12345, 12345 % 13)):
        count[was] -= 1
    value = torch.cat([value, torch.tensor([4.0, 3.5], dtype=torch.float64, device="cuda")])
    count = torch.cat([count, torch.ones(2, dtype=torch.float64, device="cuda")])
    lse = (count * value.exp()).sum().log()
    p = (value - lse).exp()
    entropy = -(count * p * (value - lse)).sum()
    y = torch.tensor([V - 1], device="cuda")
    logp, got_lse, got_entropy, top_logp, ids = he.he_token_log_probs(ctx, z[None], y, top=3)
    # each of 2048 threads adds 2^28 / 2048 / 2 terms in a row, of either half of a pair
    tol = (V / 4096 + 64) * ref.U
    assert abs(float(got_lse) - float(lse)) < tol and abs(float(logp) - float(4.0 - lse)) < tol
    assert abs(float(got_entropy) - float(entropy)) < 3 * tol * (1 + math.log(V))
    assert ids[0].tolist() == [V - 1, 12345, 12]
    d = he.he_token_log_probs_backward(ctx, z[None], y, got_lse, torch.ones(1, device="cuda"), out=z[None])[0]
    assert abs(float(d[V - 1]) - 1.0) < 2 ** -8
    # p is off by the lse and by a rounding to bf16 (subnormal ones too: the type's smallest step)
    for j in (0, 11, 12344, 12345, 12346, V // 2, V - 2):
        v = 3.5 if j == 12345 else (j % 13 - 9) * 0.5
        assert abs(float(d[j]) + math.exp(v - float(lse))) <= math.exp(v - float(lse)) * (tol + 2 ** -8)


@pytest.mark.parametrize("dtype,V", [("bf16", 57344), ("f32", 28672), ("f16", 7 * 8192 - 3), ("bf16", 32768), ("bf16", 16384)])
def test_pieces_that_a_cluster_has_not_all(ctx, dtype, V):
    """A row of as many pieces as would make one more block than the row has pieces."""
    for rows in (1, 5):
        z, y = logits_of(rows, V, dtype, V, False)
        check_log_probs(ctx, z, y, 64)
        check_log_probs(ctx, ref.strided(z, 1, 1), y, 3)


@pytest.mark.parametrize("dtype,rows,V,top", [("f16", 700, 860, 32), ("bf16", 500, 300, 64), ("bf16", 300, 1100, 33), ("f32", 900, 70, 64), ("f16", 40, 4100, 64),
                                              ("bf16", 3, 33000, 64)])
def test_rows_that_do_not_fill_a_piece(ctx, dtype, rows, V, top):
    z, y = logits_of(rows, V, dtype, V + top, False)
    check_log_probs(ctx, z, y, top)
    check_log_probs(ctx, ref.strided(z, 1, 3), y, top)


def test_many_rows(ctx):
    g = gen(3)
    rows = 150001
    z, y = logits_of(rows, 40, "bf16", 4, True)
    lse, entropy, _ = check_log_probs(ctx, z, y, 2)
    dlogp = randn(g, rows)
    want, tol = ref.log_probs_grad(z, y, lse, dlogp, entropy, None, None, None)
    ref.close(he.he_token_log_probs_backward(ctx, z, y, lse, dlogp), want, tol + ref.rounding(want, z.dtype) + 2.0 ** -126, "dlogits")
    x, dy = randn(g, rows, 24).bfloat16(), randn(g, rows, 24).bfloat16()
    n, mean, rstd = he.he_layer_norm(ctx, x)
    want, t = ref.norm(x, None, None, 1e-5)[0]
    ref.close(n, want, t + ref.rounding(want, n.dtype), "norm")
    cuts = [0, 1, 3000, 3000, 100000, rows - 7]
    back = he.he_layer_norm_backward(ctx, dy, x, mean, rstd, samples=offsets(cuts))
    for got, (want, t) in zip(back, ref.norm_grad(dy, x, mean, rstd, None, cuts)):
        ref.close(got, want, t, "backward")
    for c in (cuts, None):
        for got, (want, t) in zip(he.he_linear_sensitivity(ctx, x, dy, samples=offsets(c) if c else None), ref.linear(x, dy, c)):
            ref.close(got, want, t, "map")


def test_many_samples(ctx):
    """More samples than a list of stages holds, empty ones among them, in whole numbers."""
    g = gen(9)
    x, dy = (torch.randint(-2, 3, (9000, 200), generator=g, device="cuda").half() for _ in range(2))
    cuts = torch.arange(9001, device="cuda", dtype=torch.int32).repeat_interleave(3)
    got, bias = he.he_linear_sensitivity(ctx, x, dy, samples=cuts)
    assert torch.equal(got, dy.float().abs().T @ x.float().abs()) and torch.equal(bias, dy.float().abs().sum(0))
    _, mean, rstd = he.he_layer_norm(ctx, x)
    _, dw, db = he.he_layer_norm_backward(ctx, dy, x, mean, rstd, samples=cuts)
    assert torch.equal(db, bias)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_masks_of_the_types_lowest_value(ctx, dtype):
    """Values that are finite but far below all others count nothing, whatever gradient they meet."""
    z, y = logits_of(6, 3000, dtype, 17, False)
    z[:, ::3] = torch.finfo(z.dtype).min
    z[4] = torch.finfo(z.dtype).min
    y[:] = torch.tensor([1, 2, -100, 4, 5, 7])
    lse, entropy, ids = check_log_probs(ctx, z[[0, 1, 2, 3, 5]], y[[0, 1, 2, 3, 5]], 5)
    _, lse, entropy, _, _ = he.he_token_log_probs(ctx, z, y)
    # a row of nothing else has them all alike
    assert abs(float(entropy[4]) - math.log(3000)) < 1e-5
    dlogp, dent = torch.full((6,), 1e6, device="cuda"), torch.full((6,), 1e9, device="cuda")
    got = he.he_token_log_probs_backward(ctx, z.float(), y, lse, dlogp, entropy=entropy, dentropy=dent)
    keep = [0, 1, 2, 3, 5]
    want, tol = ref.log_probs_grad(z.float()[keep], y[keep], lse[keep], dlogp[keep], entropy[keep], dent[keep], None, None)
    ref.close(got[keep], want, tol + ref.rounding(want, torch.float32) + 2.0 ** -126, "dlogits")


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_what_follows_a_call_finds_it_done(ctx, bias, dtype):
    """A call's kernels overlap one another, not what comes before or behind the call on its stream."""
    g = gen(77)
    x, dy = (torch.randint(-2, 3, (3000, 512), generator=g, device="cuda").to(dtype) for _ in range(2))
    alone = dy.float().abs().T @ x.float().abs()
    cuts, source = offsets(list(range(0, 3001, 2))), (x.clone(), dy.clone())
    pairs = (dy.float().view(1500, 2, 512).permute(0, 2, 1) @ x.float().view(1500, 2, 512)).abs().sum(0)
    column = dy.float().view(1500, 2, 512).sum(1).abs().sum(0), dy.float().abs().sum(0)
    _, mean, rstd = he.he_layer_norm(ctx, x)
    back = [t.clone() for t in he.he_layer_norm_backward(ctx, dy, x, mean, rstd, samples=cuts)]
    torch.cuda.synchronize()
    for _ in range(10):
        for samples, want in ((None, alone), (cuts, pairs)):
            x.copy_(source[0])
            dy.copy_(source[1])
            w, b = he.he_linear_sensitivity(ctx, x, dy, samples=samples, bias=bias)
            copy = w.clone(), None if b is None else b.clone()
            x.fill_(9.0)
            dy.fill_(9.0)
            w.zero_()
            assert torch.equal(copy[0], want)
            if bias:
                assert torch.equal(copy[1], column[samples is None])
        x.copy_(source[0])
        dy.copy_(source[1])
        got = [t.clone() for t in he.he_layer_norm_backward(ctx, dy, x, mean, rstd, samples=cuts)]
        x.fill_(9.0)
        dy.fill_(9.0)
        assert all(torch.equal(a, b) for a, b in zip(got, back))


def test_first_calls_inside_a_capture():
    code = """
import torch, sys
sys.path[:0] = ["tests"]
import paper_2303_10837_b200 as he, synthetic_inputs as si
from test_gpu_map_operators import all_calls, state
ctx = he.he_ctx_create(8192, list(si.PRIMES_N8192), 40)
s = state(1)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    held = all_calls(ctx, s)
graph.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(held, all_calls(ctx, s)))
"""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_calls_from_several_threads(ctx):
    states = [state(20 + i) for i in range(4)]
    want = [[t.clone() for t in all_calls(ctx, s)] for s in states]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(10):
                got = all_calls(ctx, states[i])
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(want[i], got)):
                    wrong.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
