"""What sensitivity_map refuses before it touches a GPU: layers that it has no scores for, shared parameters, layers used twice."""
import pytest
import torch
from torch import nn

import paper_2303_10837_b200 as he
from paper_2303_10837_b200 import sensitivity as sv


def places(model):
    return sv._parts(model, torch.zeros(sum(p.numel() for p in model.parameters())))


def refused(call, word):
    with pytest.raises(he.HeError) as ei:
        call()
    assert ei.value.code == he.HE_ERR_INVALID_ARG and word in str(ei.value)


def test_places_follow_the_flattened_model():
    model = nn.Sequential(nn.Linear(3, 4), nn.LayerNorm(4), nn.Linear(4, 2, bias=False))
    flat = torch.arange(sum(p.numel() for p in model.parameters()), dtype=torch.float32)
    parts = sv._parts(model, flat)
    got = torch.cat([t.reshape(-1) for _, p in parts for t in (p.weight, p.bias) if t is not None])
    assert torch.equal(got, flat) and len(parts) == 3 and parts[2][1].bias is None


def test_untrained_layers_are_left_out_and_others_refused():
    model = nn.Sequential(nn.Embedding(7, 3), nn.Linear(3, 4))
    refused(lambda: places(model), "Embedding")
    model[0].weight.requires_grad_(False)
    assert [p.name for _, p in places(model)] == ["1"]
    model[1].weight.requires_grad_(False)
    refused(lambda: places(model), "bias")
    model[1].bias.requires_grad_(False)
    refused(lambda: places(model), "no trained")
    refused(lambda: places(nn.LayerNorm((2, 3))), "dimensions")
    refused(lambda: places(nn.MultiheadAttention(4, 2)), "MultiheadAttention")


def test_shared_parameters_are_refused():
    a, b = nn.Linear(3, 3), nn.Linear(3, 3)
    b.weight = a.weight
    refused(lambda: places(nn.Sequential(a, b)), "shared")


def test_a_layer_used_twice_or_without_the_samples_dimension():
    state = sv._Pass(he.Ctx(0, 8192, 3, 40), 4, torch.device("cpu"))
    part = sv._Part("x", None, None)
    state.enter(part, torch.Size((4, 7)))
    refused(lambda: state.enter(part, torch.Size((4, 7))), "twice")
    for shape in ((12, 7), (3, 4, 7), (4,)):
        refused(lambda: state.enter(sv._Part("y", None, None), torch.Size(shape)), "first dimension")
    assert state.samples(4) is None and state.samples(12).tolist() == [0, 3, 6, 9, 12]


def test_layers_get_their_own_forward_back():
    model = nn.Sequential(nn.Linear(2, 2), nn.LayerNorm(2))
    state = sv._Pass(he.Ctx(0, 8192, 3, 40), 1, torch.device("cpu"))
    with pytest.raises(ZeroDivisionError):
        with sv._layers_of(places(model), state):
            assert "forward" in model[0].__dict__
            raise ZeroDivisionError
    assert "forward" not in model[0].__dict__ and "forward" not in model[1].__dict__


def test_a_model_on_the_host_is_refused():
    with pytest.raises(TypeError):
        sv.sensitivity_map(he.Ctx(0, 8192, 3, 40), nn.Linear(2, 2), [])
