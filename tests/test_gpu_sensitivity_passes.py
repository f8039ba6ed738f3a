"""A model's pass in sensitivity_map beside the model's own, and what it raises."""
import pytest
import torch
from torch import nn

import paper_2303_10837_b200 as he
import synthetic_inputs as si
from paper_2303_10837_b200.sensitivity import sensitivity_map
from test_gpu_sensitivity import Model, batches, by_samples

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    return he.he_ctx_create(8192, list(si.PRIMES_N8192), 40)


def test_layer_norms_under_autocast_are_those_of_torch(ctx):
    """fp32 inside and out, whatever their inputs and weights are."""
    torch.manual_seed(9)
    data = batches(12, count=1)
    for kind in (torch.float32, torch.bfloat16):
        model = Model().cuda()
        for m in model.modules():
            if isinstance(m, nn.LayerNorm):
                m.to(kind)
        seen = []
        hooks = [m.register_forward_hook(lambda m, args, out: seen.append(out.detach())) for m in model.modules() if isinstance(m, nn.LayerNorm)]
        with torch.autocast("cuda", dtype=torch.bfloat16):
            model(data[0][0])
            there, seen[:] = list(seen), []
            got = sensitivity_map(ctx, model, data)
        for h in hooks:
            h.remove()
        assert len(there) == len(seen) == 5
        for a, b in zip(there, seen):
            # behind five layers at most, of which each may round a value of up to 4 the other way
            assert a.dtype == b.dtype == torch.float32 and float((a - b).abs().max()) < 0.1
        assert float((seen[0] - there[0]).abs().max()) < 1e-5
        want = by_samples(model, data)
        assert float((got.map - want).norm() / want.norm()) < 5e-2


def test_a_layer_norm_behind_a_linear_layer_under_autocast(ctx):
    """Its input is of autocast's type, its output is not."""
    torch.manual_seed(10)
    model = nn.Sequential(nn.Linear(20, 33), nn.LayerNorm(33), nn.Linear(33, 7)).cuda()
    x, y = torch.randn(9, 4, 20, device="cuda"), torch.randint(0, 7, (9, 4), device="cuda")
    seen = []
    model[1].register_forward_hook(lambda m, args, out: seen.append((args[0].detach(), out.detach())))
    for dtype in (torch.bfloat16, torch.float16):
        seen.clear()
        with torch.autocast("cuda", dtype=dtype):
            model(x)
            got = sensitivity_map(ctx, model, [(x, y)])
        (a_in, a), (b_in, b) = seen
        assert torch.equal(a_in, b_in) and a_in.dtype == dtype and a.dtype == b.dtype == torch.float32
        assert float((a - b).abs().max()) < 1e-5             # of values up to 6: a few roundings of fp32
        want = torch.zeros_like(got.map, dtype=torch.float64)
        m = nn.Sequential(nn.Linear(20, 33), nn.LayerNorm(33), nn.Linear(33, 7)).cuda().double()
        m.load_state_dict(model.state_dict())
        for i in range(9):
            m.zero_grad()
            torch.log_softmax(m(x[i].double()), -1).gather(1, y[i][:, None]).sum().backward()
            want += torch.cat([p.grad.reshape(-1).abs() for p in m.parameters()]) / 9
        assert float((got.map - want).norm() / want.norm()) < 5e-2


def test_an_error_inside_a_kernel_is_raised(ctx, monkeypatch):
    from paper_2303_10837_b200 import sensitivity as sv
    model, data = Model().cuda(), batches(2, count=1)
    # one that is there: an encryption of what is not finite leaves it in the context
    keys = he.he_keygen(ctx, 3)
    he.he_encrypt(ctx, keys, he.he_pack(ctx, None, torch.full((8,), float("nan"), device="cuda"))[0], 1, 0)
    with pytest.raises(he.HeError) as ei:
        sensitivity_map(ctx, model, data)
    assert ei.value.code == he.HE_ERR_OVERFLOW
    sensitivity_map(ctx, model, data)                        # and it is no longer
    monkeypatch.setattr(sv, "he_ctx_status", lambda c: he.HE_ERR_CUDA, raising=False)
    with pytest.raises(he.HeError) as ei:
        sensitivity_map(ctx, model, data)
    assert ei.value.code == he.HE_ERR_CUDA


def test_a_layer_of_no_rows(ctx):
    """A model with a part that a batch gives nothing to."""
    class Parts(nn.Module):
        def __init__(self):
            super().__init__()
            self.a, self.n, self.b = nn.Linear(6, 6), nn.LayerNorm(6), nn.Linear(6, 5)

        def forward(self, x):
            return self.b(torch.cat([x, self.n(self.a(x[:, :0]))], 1))

    torch.manual_seed(3)
    model, x, y = Parts().cuda(), torch.randn(4, 3, 6, device="cuda"), torch.randint(0, 5, (4, 3), device="cuda")
    got = sensitivity_map(ctx, model, [(x, y)]).map
    head = nn.Sequential(model.b)
    assert (got[:54] == 0).all() and torch.equal(got[54:], sensitivity_map(ctx, head, [(x, y)]).map)


def test_parts_of_a_model_that_autocast_leaves_alone(ctx):
    """Are differentiated in fp32 too: the pass backward is not under the caller's autocast."""
    class Plain(nn.Module):
        def __init__(self):
            super().__init__()
            self.net = Model()

        def forward(self, t):
            with torch.autocast("cuda", enabled=False):
                return self.net(t)

    torch.manual_seed(11)
    model, data = Plain().cuda(), batches(5)
    want = sensitivity_map(ctx, model, data)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        got = sensitivity_map(ctx, model, data)
    assert torch.equal(got.map, want.map) and got[1:] == want[1:]


def test_layers_that_a_model_runs_on_another_stream(ctx):
    """What they add to the map is there when it is divided, however late their stream comes to it."""
    class Aside(nn.Module):
        def __init__(self):
            super().__init__()
            self.a, self.n, self.b = nn.Linear(20, 33), nn.LayerNorm(33), nn.Linear(33, 7)
            self.stream, self.wait = torch.cuda.Stream(), 0

        def forward(self, x):
            here = torch.cuda.current_stream()
            self.stream.wait_stream(here)
            with torch.cuda.stream(self.stream):
                y = self.n(self.a(x))
                if self.wait and y.requires_grad:
                    y.register_hook(self.late)
            here.wait_stream(self.stream)
            return self.b(y)

        def late(self, g):
            torch.cuda._sleep(self.wait)                     # clocks
            return g

    torch.manual_seed(12)
    model = Aside().cuda()
    data = [(torch.randn(9, 4, 20, device="cuda"), torch.randint(0, 7, (9, 4), device="cuda")) for _ in range(3)]
    plain = nn.Sequential(model.a, model.n, model.b)
    want = sensitivity_map(ctx, plain, data)
    for wait in (0, 20_000_000):
        model.wait = wait
        torch.cuda.synchronize()
        got = sensitivity_map(ctx, model, data)
        assert torch.equal(got.map, want.map) and got[1:] == want[1:]


def test_64_bits_are_refused_under_autocast_too(ctx):
    model = nn.Sequential(nn.LayerNorm(6), nn.Linear(6, 5)).cuda().double()
    x, y = torch.randn(4, 3, 6, device="cuda", dtype=torch.float64), torch.randint(0, 5, (4, 3), device="cuda")
    for enabled in (False, True):
        with torch.autocast("cuda", dtype=torch.bfloat16, enabled=enabled), pytest.raises(he.HeError) as ei:
            sensitivity_map(ctx, model, [(x, y)])
        assert ei.value.code == he.HE_ERR_INVALID_ARG and "float64" in str(ei.value)
