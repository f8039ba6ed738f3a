"""The sensitivity map of small models against per-sample gradients in 64 bits, and the whole mask calculation and round that it begins."""
import copy

import numpy as np
import pytest
import torch
from torch import nn

import paper_2303_10837_b200 as he
import synthetic_inputs as si
from paper_2303_10837_b200.sensitivity import sensitivity_map

pytestmark = pytest.mark.gpu


class Block(nn.Module):
    """A transformer's layer, of the modules that get scores and of functions."""

    def __init__(self, d, ff):
        super().__init__()
        self.n1, self.qkv, self.out = nn.LayerNorm(d), nn.Linear(d, 3 * d), nn.Linear(d, d, bias=False)
        self.n2, self.up, self.down = nn.LayerNorm(d), nn.Linear(d, ff), nn.Linear(ff, d)

    def forward(self, x):
        q, k, v = self.qkv(self.n1(x)).chunk(3, -1)
        a = torch.softmax(q @ k.transpose(-1, -2) / q.shape[-1] ** 0.5, -1)
        x = x + self.out(a @ v)
        return x + self.down(torch.tanh(self.up(self.n2(x))))


class Model(nn.Module):
    def __init__(self, vocab=97, d=48, ff=80, layers=2):
        super().__init__()
        self.words = nn.Embedding(vocab, d)
        self.words.weight.requires_grad_(False)
        self.blocks = nn.Sequential(*[Block(d, ff) for _ in range(layers)])
        self.norm, self.head = nn.LayerNorm(d), nn.Linear(d, vocab)

    def forward(self, t):
        return self.head(self.norm(self.blocks(self.words(t))))


def batches(seed, count=2, samples=5, tokens=11, vocab=97):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for _ in range(count):
        t = torch.randint(0, vocab, (samples, tokens), generator=g, device="cuda")
        y = torch.randint(0, vocab, (samples, tokens), generator=g, device="cuda")
        y[1, 6:] = -100                                      # a shorter sample
        out.append((t, y))
    return out


def by_samples(model, data):
    """The definition: each sample's gradient by itself, in 64 bits."""
    m = copy.deepcopy(model).double()
    total = torch.zeros(sum(p.numel() for p in m.parameters()), dtype=torch.float64, device="cuda")
    k = 0
    for t, y in data:
        for i in range(t.shape[0]):
            m.zero_grad(set_to_none=True)
            lp = torch.log_softmax(m(t[i:i + 1])[0], -1)
            keep = y[i] >= 0
            lp[keep].gather(1, y[i][keep][:, None]).sum().backward()
            total += torch.cat([(torch.zeros_like(p) if p.grad is None else p.grad).reshape(-1).abs() for p in m.parameters()])
            k += 1
    return total / k


@pytest.fixture(scope="module")
def ctx():
    return he.he_ctx_create(8192, list(si.PRIMES_N8192), 40)


# fp32 passes through a dozen layers of up to 97 terms are off by some 100 u = 6e-6 of a score; bf16 activations by 100 times 2^-9 at most, and
# by its root on the whole
@pytest.mark.parametrize("dtype,rel", [(torch.float32, 1e-4), (torch.bfloat16, 5e-2)])
def test_map_is_the_mean_of_the_samples_magnitudes(ctx, dtype, rel):
    torch.manual_seed(1)
    model = Model().cuda().to(dtype)
    data = batches(3)
    got = sensitivity_map(ctx, model, data)
    want = by_samples(model, data)
    assert got.map.shape == want.shape and got.map.dtype == torch.float32
    assert got.samples == 10 and got.tokens == sum(int((y >= 0).sum()) for _, y in data)
    assert float((got.map.double() - want).norm() / want.norm()) < rel
    assert (got.map[:model.words.weight.numel()] == 0).all()
    assert -20 < got.log_prob < 0 and 0 < got.entropy < np.log(97) + 1e-3
    # nothing is left behind: gradients, patched layers
    assert all(p.grad is None for p in model.parameters()) and all("forward" not in m.__dict__ for m in model.modules())


def test_one_logit_row_for_each_sample(ctx):
    torch.manual_seed(2)
    model = nn.Sequential(nn.Linear(20, 33), nn.LayerNorm(33), nn.Linear(33, 7)).cuda()
    x, y = torch.randn(9, 20, device="cuda"), torch.randint(0, 7, (9,), device="cuda")
    got = sensitivity_map(ctx, model, [(x, y)]).map.double()
    m = copy.deepcopy(model).double()
    want = torch.zeros_like(got)
    for i in range(9):
        m.zero_grad()
        torch.log_softmax(m(x[i:i + 1].double()), -1)[0, y[i]].backward()
        want += torch.cat([p.grad.reshape(-1).abs() for p in m.parameters()]) / 9
    assert float((got - want).norm() / want.norm()) < 1e-5


def test_a_layer_used_twice_is_refused(ctx):
    inner = nn.Linear(8, 8)
    model = nn.Sequential(inner, inner).cuda()
    with pytest.raises(he.HeError):
        sensitivity_map(ctx, model, [(torch.randn(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda"))])


def test_a_weight_used_outside_its_layer_is_refused(ctx):
    class Outside(nn.Linear):
        pass

    class Uses(nn.Module):
        def __init__(self):
            super().__init__()
            self.a = nn.Linear(8, 8)

        def forward(self, x):
            return self.a(x) @ self.a.weight

    x, y = torch.randn(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    for model in (Uses().cuda(), Outside(8, 8).cuda()):
        with pytest.raises(he.HeError):
            sensitivity_map(ctx, model, [(x, y)])
        assert all(p.grad is None for p in model.parameters())


def test_frozen_parameters_and_layers_without_a_bias(ctx):
    torch.manual_seed(5)
    model = nn.Sequential(nn.Linear(16, 24, bias=False), nn.LayerNorm(24, bias=False), nn.Linear(24, 24), nn.LayerNorm(24), nn.Linear(24, 9)).cuda()
    model[2].requires_grad_(False)
    model[3].weight.requires_grad_(False)
    model[4].bias.requires_grad_(False)
    x, y = torch.randn(4, 5, 16, device="cuda"), torch.randint(0, 9, (4, 5), device="cuda")
    got = sensitivity_map(ctx, model, [(x[:3], y[:3]), (x[:0], y[:0]), (x[3:], y[3:])])
    m = copy.deepcopy(model).double()
    want = torch.zeros_like(got.map, dtype=torch.float64)
    for i in range(4):
        m.zero_grad(set_to_none=True)
        torch.log_softmax(m(x[i].double()), -1).gather(1, y[i][:, None]).sum().backward()
        want += torch.cat([(torch.zeros_like(p) if p.grad is None else p.grad).reshape(-1).abs() for p in m.parameters()]) / 4
    assert got.samples == 4 and got.tokens == 20
    assert float((got.map - want).norm() / want.norm()) < 1e-5
    assert ((got.map == 0) == (want == 0)).all()


def test_under_autocast_and_another_stream(ctx):
    torch.manual_seed(6)
    model, data = Model().cuda(), batches(8, count=1)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream), torch.autocast("cuda", dtype=torch.bfloat16):
        got = sensitivity_map(ctx, model, data)
    stream.synchronize()
    want = by_samples(model, data)
    assert float((got.map - want).norm() / want.norm()) < 5e-2


def test_mask_calculation_and_round_from_the_maps(ctx):
    """Stages 2 and 3 of the protocol: two clients' maps, their encrypted weighted sum, the mask of the most sensitive parameters, a round with it."""
    torch.manual_seed(4)
    model, alpha = Model().cuda(), [0.4, 0.6]
    keys = he.he_keygen(ctx, 7)
    maps = [sensitivity_map(ctx, model, batches(10 + i)).map for i in range(2)]
    P = maps[0].numel()
    cts = [he.he_encrypt(ctx, keys, he.he_pack(ctx, None, m)[0], 5, i) for i, m in enumerate(maps)]
    score = he.he_unpack(ctx, None, he.he_decrypt(ctx, keys, he.he_weighted_aggregate(ctx, cts, alpha)), None, P)
    plain = sum(a * m.double() for a, m in zip(alpha, maps))
    assert float((score - plain).abs().max()) < 1e-6         # the scheme's noise
    k = P // 10
    mask = he.he_select_mask(ctx, score.float(), k)
    idx = he.he_mask_indices(mask).long()
    assert mask.k == k and float(score.float()[idx].min()) >= float(torch.topk(score.float(), k).values[-1])
    updates = [torch.randn(P, device="cuda") * 0.01 for _ in range(2)]
    packed = [he.he_pack(ctx, mask, u) for u in updates]
    agg = he.he_weighted_aggregate(ctx, [he.he_encrypt(ctx, keys, s, 6, i) for i, (s, _) in enumerate(packed)], alpha)
    rest = he.he_plain_aggregate(ctx, [r for _, r in packed], alpha)
    out = he.he_unpack(ctx, mask, he.he_decrypt(ctx, keys, agg), rest, P)
    assert float((out - sum(a * u.double() for a, u in zip(alpha, updates))).abs().max()) < 1e-6
    assert he.he_ctx_status(ctx) == 0
