"""How sensitivity_map takes a model's layers over for a pass, and what it refuses there; no GPU is touched."""
import threading

import pytest
import torch
from torch import nn

import paper_2303_10837_b200 as he
from paper_2303_10837_b200 import sensitivity as sv
from test_sensitivity_refusals import places, refused


def a_pass(count=3):
    return sv._Pass(he.Ctx(0, 8192, 3, 40), count, torch.device("cpu"))


def in_a_thread(call):
    """What a call gives, or raises, in another thread."""
    got = []

    def work():
        try:
            got.append(call())
        except Exception as e:
            got.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    return got[0]


def test_calls_of_another_thread_are_refused_and_leave_the_pass_alone():
    model, x = nn.Sequential(nn.Linear(4, 4), nn.Linear(4, 2)), torch.randn(3, 4)
    want = model(x)
    with sv._layers_of(places(model), a_pass()):
        got = in_a_thread(lambda: model(x))
        assert isinstance(got, he.HeError) and got.code == he.HE_ERR_INVALID_ARG and "thread" in str(got)
        assert torch.equal(model(x), want)
    assert torch.equal(in_a_thread(lambda: model(x)), want)


def test_two_passes_at_once_are_refused_and_the_layers_come_back():
    model, x = nn.Sequential(nn.Linear(4, 4), nn.Linear(4, 2)), torch.randn(3, 4)
    want = model(x)

    def enter(which):
        with sv._layers_of(which, a_pass()):
            pass

    for other in (model, nn.Sequential(model[1])):           # one layer in common is enough
        with sv._layers_of(places(model), a_pass()):
            refused(lambda: enter(places(other)), "already")
            got = in_a_thread(lambda: enter(places(other)))
            assert isinstance(got, he.HeError) and "already" in str(got)
            assert torch.equal(model(x), want)
        assert all("forward" not in m.__dict__ for m in model)
    enter(places(model))


def test_a_layer_with_a_forward_of_its_own_is_refused():
    model = nn.Sequential(nn.Linear(4, 4), nn.Linear(4, 2))
    plain = model[1].forward
    model[1].forward = lambda x: plain(x) * 2

    def enter():
        with sv._layers_of(places(model), a_pass()):
            pass

    for _ in range(2):
        refused(enter, "forward of its own")
    assert "forward" in model[1].__dict__ and "forward" not in model[0].__dict__
    del model[1].forward
    enter()


def test_a_trained_layer_without_a_gradient_is_refused():
    class Stops(nn.Module):
        def __init__(self):
            super().__init__()
            self.a, self.b = nn.Linear(4, 4), nn.Linear(4, 2)

        def forward(self, x):
            with torch.no_grad():
                x = self.a(x)
            return self.b(x)

    model, x = Stops(), torch.randn(3, 4)
    with sv._layers_of(places(model), a_pass()):
        refused(lambda: model(x), "no_grad")
    model.a.requires_grad_(False)
    with sv._layers_of(places(model), a_pass()):
        assert model(x).requires_grad


def test_a_layer_of_no_rows():
    state = a_pass()
    state.enter(sv._Part("x", None, None), torch.Size((3, 0, 7)))
    assert state.samples(0).tolist() == [0, 0, 0, 0] and state.samples(0).dtype == torch.int32
