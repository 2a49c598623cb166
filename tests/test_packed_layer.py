"""Host-only checks of layer.PackedLayer: sizes and weights that a run would refuse half way through are refused when it is made, and
arguments of a run before anything is called."""
import pytest
import torch

import paper_2509_22323_amd as ra
from paper_2509_22323_amd import layer as layer_module
from test_joint_layer import weights

SIZES = dict(H=2, D=64, image=77, text=9, documents=3)


@pytest.fixture(autouse=True)
def no_calls(monkeypatch):
    monkeypatch.setattr(layer_module._b, "rapid_quantize_rows", lambda w, q, s: (q, s))


def make(first=None, second=None, **kw):
    return ra.PackedLayer((first or weights(F=144), second or weights(F=64)), **{**SIZES, **kw})


def test_a_layer_is_made_on_the_weights_device():
    layer = make(weights(F=160, mod_b=None, qkv_b=None, q_norm=None, k_norm=None, out_b=None, ff_in_b=None, ff_out_b=None), axes=[ra.RopeAxis(32)])
    assert [tuple(t.shape) for t in layer.f] == [(77, 160), (9, 64)] and tuple(layer.table.shape) == (86, 16, 2)
    assert not any(k in layer.small[0] for k in layer.PRODUCTS)


@pytest.mark.parametrize("kw", [
    dict(image=0), dict(image=-128), dict(text=0), dict(H=0), dict(H=1, D=128), dict(D=96), dict(layout="halves"), dict(eps=-1e-6), dict(documents=0),
    dict(first=weights(F=136)), dict(second=weights(F=8)), dict(second=weights(F=64, C=64)), dict(second=weights(F=64, out_w=None)),
    dict(second=weights(F=64, ff_out_w=(64, 128)))], ids=lambda kw: " ".join(kw))
def test_sizes_that_do_not_fit(kw):
    with pytest.raises(ValueError):
        make(**kw)


@pytest.mark.parametrize("kw", [
    dict(conditioning=torch.zeros(4, 128)), dict(conditioning=torch.zeros(0, 128)), dict(conditioning=torch.zeros(128)), dict(positions=torch.zeros(86, 1)),
    dict(document=torch.zeros(85)), dict(document=torch.zeros(1, 86)), dict(order=torch.zeros(77)), dict(cap=-1.0), dict(cap=float("inf")),
    dict(cap=float("nan"))], ids=lambda kw: " ".join(kw))
def test_arguments_of_a_run(kw, monkeypatch):
    layer = make()
    monkeypatch.setattr(layer_module, "_b", None)
    args = dict(conditioning=torch.zeros(3, 128), document=torch.zeros(86))
    with pytest.raises(ValueError):
        layer.run(torch.zeros(77, 128), torch.zeros(9, 128), **{**args, **kw})


def test_positions_are_needed_for_a_rotation():
    with pytest.raises(ValueError):
        make(axes=[ra.RopeAxis(64)]).run(torch.zeros(77, 128), torch.zeros(9, 128), torch.zeros(3, 128), torch.zeros(86))
