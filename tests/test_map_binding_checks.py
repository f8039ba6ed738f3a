"""Refusals of the sensitivity map's operators, on the host: wrong sizes, types and layouts raise HeError before anything is launched,
and calls that are right as far as the host can see reach the device check (TypeError: host tensors)."""
import ctypes

import pytest
import torch

import paper_2303_10837_b200 as he


@pytest.fixture()
def ctx():
    return he.Ctx(0, 8192, 3, 40)           # handle 0: never used, never destroyed


def refused(call):
    with pytest.raises(he.HeError) as ei:
        call()
    assert ei.value.code == he.HE_ERR_INVALID_ARG


def reaches_device_check(call):
    with pytest.raises(TypeError):
        call()


def f(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def i64(n):
    return torch.zeros(n, dtype=torch.int64)


def i32(n):
    return torch.zeros(n, dtype=torch.int32)


def test_log_probs(ctx):
    go = he.he_token_log_probs
    refused(lambda: go(ctx, f(4, 10, dtype=torch.float64), i64(4)))
    refused(lambda: go(ctx, f(40), i64(4)))                              # not a matrix
    refused(lambda: go(ctx, f(10, 4).t(), i64(4)))                       # rows that do not lie together
    refused(lambda: go(ctx, f(4, 10), i64(3)))
    refused(lambda: go(ctx, f(4, 10), i32(4)))
    refused(lambda: go(ctx, f(4, 10), i64(8)[::2]))
    refused(lambda: go(ctx, f(4, 0), i64(4)))
    refused(lambda: go(ctx, f(4, 10), i64(4), top=11))
    refused(lambda: go(ctx, f(4, 100), i64(4), top=he.HE_MAX_TOP + 1))
    refused(lambda: go(ctx, f(4, 10), i64(4), top=-1))
    reaches_device_check(lambda: go(ctx, f(4, 10), i64(4), top=10))
    reaches_device_check(lambda: go(ctx, f(1, 10).expand(4, 10), i64(4)))


def test_log_probs_backward(ctx):
    go = he.he_token_log_probs_backward
    refused(lambda: go(ctx, f(4, 10), i64(4), f(3), f(4)))
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(5)))
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), dentropy=f(4)))            # without the entropy
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), entropy=f(4), dentropy=f(3)))
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), top_ids=torch.zeros(4, 2, dtype=torch.int64)))
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), top_ids=torch.zeros(4, 2, dtype=torch.int64), dtop=f(4, 3)))
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), top_ids=torch.zeros(4, 2, dtype=torch.int32), dtop=f(4, 2)))
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), out=f(4, 9)))
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), out=f(4, 10, dtype=torch.float16)))
    refused(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), out=f(1, 10).expand(4, 10)))   # every row would be the same memory
    reaches_device_check(lambda: go(ctx, f(4, 10), i64(4), f(4), f(4), entropy=f(4), dentropy=f(4)))


def test_layer_norm(ctx):
    go = he.he_layer_norm
    refused(lambda: go(ctx, f(4, 10, dtype=torch.int32)))
    refused(lambda: go(ctx, f(4, 10), f(9)))
    refused(lambda: go(ctx, f(4, 10), f(10), f(10, dtype=torch.bfloat16)))
    refused(lambda: go(ctx, f(4, 10, dtype=torch.bfloat16), f(10), f(10, dtype=torch.bfloat16)))   # weights of two types
    refused(lambda: go(ctx, f(4, 10), eps=-1.0))
    refused(lambda: go(ctx, f(4, 10), eps=float("nan")))
    refused(lambda: go(ctx, f(4, 0)))
    refused(lambda: go(ctx, f(4, 10), out=f(3, 10)))
    refused(lambda: go(ctx, f(2, 4, 10)))
    reaches_device_check(lambda: go(ctx, f(4, 10), f(10), f(10)))


def test_layer_norm_backward(ctx):
    go = he.he_layer_norm_backward
    refused(lambda: go(ctx, f(4, 9), f(4, 10), f(4), f(4)))
    refused(lambda: go(ctx, f(4, 10, dtype=torch.float16), f(4, 10), f(4), f(4)))        # dy of another type
    refused(lambda: go(ctx, f(4, 10), f(4, 10), f(3), f(4)))
    refused(lambda: go(ctx, f(4, 10), f(4, 10), f(4), f(4), f(11)))
    refused(lambda: go(ctx, f(4, 10), f(4, 10), f(4), f(4), samples=i64(3)))
    refused(lambda: go(ctx, f(4, 10), f(4, 10), f(4), f(4), samples=i32(0)))
    refused(lambda: go(ctx, f(4, 10), f(4, 10), f(4), f(4), samples=i32(6)[::2]))
    reaches_device_check(lambda: go(ctx, f(4, 10), f(4, 10), f(4), f(4), f(10), samples=i32(3)))


def test_linear_sensitivity(ctx):
    go = he.he_linear_sensitivity
    refused(lambda: go(ctx, f(4, 10), f(5, 3)))
    refused(lambda: go(ctx, f(4, 10), f(4, 3, dtype=torch.bfloat16)))
    refused(lambda: go(ctx, f(4, 10), f(4, 0)))
    refused(lambda: go(ctx, f(4, 10), f(4, 3), samples=i64(2)))
    refused(lambda: go(ctx, f(4, 10), f(4, 3), out=f(10, 3)))
    refused(lambda: go(ctx, f(4, 10), f(4, 3), out=f(3, 12)[:, :10]))
    refused(lambda: go(ctx, f(4, 10), f(4, 3), out=f(3, 10, dtype=torch.float64)))
    refused(lambda: go(ctx, f(4, 10), f(4, 3), out_bias=f(4)))
    refused(lambda: go(ctx, f(4, 10), f(4, 3), accumulate=True))                         # nothing to add to
    refused(lambda: go(ctx, f(4, 10), f(4, 3), out=f(3, 10), accumulate=True))
    reaches_device_check(lambda: go(ctx, f(4, 10), f(4, 3), out=f(3, 10), out_bias=f(3), accumulate=True))
    reaches_device_check(lambda: go(ctx, f(4, 10), f(4, 3), out=f(3, 10), accumulate=True, bias=False))


def test_a_tensor_on_another_device_is_refused(monkeypatch):
    class Far:
        is_cuda = True

        def __init__(self, device):
            self.device = device

        def get_device(self):
            return self.device

    monkeypatch.setattr(he, "_raw_device", lambda: 1)
    assert he._on_gpu(Far(1), None, Far(1)) == 1
    for tensors in ((Far(0),), (Far(1), None, Far(0))):
        refused(lambda: he._on_gpu(*tensors))


def test_c_entry_points_refuse_a_missing_context():
    lib, null = he._lib, None
    assert lib.he_token_log_probs(null, null, 0, 1, 1, 1, null, 0, null, null, null, null, null, null) == he.HE_ERR_INVALID_ARG
    assert lib.he_token_log_probs_backward(null, null, 0, 1, 1, 1, null, null, null, null, null, 0, null, null, null, 1, null) == he.HE_ERR_INVALID_ARG
    assert lib.he_layer_norm(null, null, 0, 1, 1, 1, null, null, 0, 1e-5, null, 1, null, null, null) == he.HE_ERR_INVALID_ARG
    assert lib.he_layer_norm_backward(null, null, 1, null, 1, 0, 1, 1, null, null, null, 0, null, 0, null, 1, null, null, null, 0, null) == he.HE_ERR_INVALID_ARG
    assert lib.he_linear_sensitivity(null, null, 1, null, 1, 0, 1, 1, 1, null, 0, 0, null, null, null, 0, null) == he.HE_ERR_INVALID_ARG
    assert lib.he_layer_norm_backward_work_bytes(null, 1, 1) == 0 and lib.he_linear_sensitivity_work_bytes(null, 0, 1, 1, 1, 0, 0) == 0
    assert isinstance(lib, ctypes.CDLL)
