"""Host-only checks of layer.JointLayer: sizes and weights that a run would refuse half way through are refused when it is made."""
import pytest
import torch

import paper_2509_22323_amd as ra
from paper_2509_22323_amd import layer as layer_module

SIZES = dict(B=2, H=2, D=64, image=256, text=9)


def weights(C=128, D=64, F=136, **other):
    """(zeros on the CPU: enough for what is checked before any call)"""
    shapes = dict(mod_w=(6 * C, C), mod_b=(6 * C,), qkv_w=(3 * C, C), qkv_b=(3 * C,), q_norm=(D,), k_norm=(D,), out_w=(C, C), out_b=(C,),
                  ff_in_w=(F, C), ff_in_b=(F,), ff_out_w=(C, F), ff_out_b=(C,))
    assert set(shapes) == set(layer_module.WEIGHTS)
    shapes.update(other)
    return {k: None if s is None else torch.zeros(s, dtype=torch.bfloat16) for k, s in shapes.items()}


def make(first=None, second=None, **kw):
    return ra.JointLayer((first or weights(), second or weights(F=64)), **{**SIZES, **kw})


def test_a_layer_is_made_on_the_weights_device():
    layer = make(weights(mod_b=None, qkv_b=None, q_norm=None, k_norm=None, out_b=None, ff_in_b=None, ff_out_b=None))
    assert [tuple(t.shape) for t in layer.f] == [(2, 256, 136), (2, 9, 64)]


@pytest.mark.parametrize("kw", [
    dict(image=200), dict(image=64), dict(image=0), dict(image=-128), dict(text=0), dict(text=-5), dict(B=0), dict(H=0), dict(H=1, D=128), dict(D=32),
    dict(D=96), dict(layout="halves"), dict(eps=-1e-6), dict(eps=float("nan")), dict(first=weights(F=132)), dict(second=weights(F=4)),
    dict(second=weights(C=64)), dict(first=weights(D=32)), dict(first=weights(mod_w=(5 * 128, 128))), dict(first=weights(qkv_w=(128, 384))),
    dict(second=weights(out_w=None)), dict(second=weights(ff_out_b=(136,))), dict(second=weights(ff_out_w=(128, 64)))], ids=lambda kw: " ".join(kw))
def test_sizes_that_do_not_fit(kw):
    with pytest.raises(ValueError):
        make(**kw)


@pytest.mark.parametrize("shape", [(264, 2), (265, 1), (265, 3), (1, 265, 2), (3, 265, 2), (2, 264, 2), (2, 1, 265, 2), (265,)], ids=str)
def test_positions_that_do_not_fit(shape):
    with pytest.raises(ValueError):
        make(positions=torch.zeros(shape, dtype=torch.int32), axes=[ra.RopeAxis(32), ra.RopeAxis(32)])


def test_one_stream_is_no_layer():
    with pytest.raises(ValueError):
        ra.JointLayer((weights(),), **SIZES)


@pytest.mark.parametrize("a_sparse", [-1, 4, 17])
def test_actions_that_there_are_not(a_sparse, monkeypatch):
    """refused before anything is called"""
    layer = make()
    monkeypatch.setattr(layer_module, "_b", None)
    with pytest.raises(ValueError):
        layer.run(torch.zeros(2, 256, 128), torch.zeros(2, 9, 128), torch.zeros(2, 128), a_sparse)


class Current:
    """Stands in for torch's current device: 0, or what the innermost `with` names."""
    def __init__(self, monkeypatch):
        self.device = 0
        current = self

        class Guard:
            def __init__(self, device):
                self.to = device

            def __enter__(self):
                self.before, current.device = current.device, self.to

            def __exit__(self, *_):
                current.device = self.before

        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current.device, raising=False)
        monkeypatch.setattr(torch.cuda, "device", Guard)


@pytest.mark.parametrize("device", [0, 1])
@pytest.mark.parametrize("a_sparse", [0, 3])
def test_calls_are_made_with_the_layers_device_current(device, a_sparse, monkeypatch):
    """The calls that launch on the current device find the layer's one there, and the caller's is current again behind a run."""
    layer, current, made = make(), Current(monkeypatch), []
    layer.device = device

    class Calls:
        def __getattr__(self, name):
            return lambda *a, **k: made.append((name, current.device))

    monkeypatch.setattr(layer_module, "_b", Calls())
    layer.run(torch.zeros(2, 256, 128), torch.zeros(2, 9, 128), torch.zeros(2, 128), a_sparse)
    assert current.device == 0 and {d for _, d in made} == {device}
    attention = "rapid_attn_joint" if a_sparse == 0 else "rapid_attn_joint_select"
    assert [name for name, _ in made].count(attention) == 1 and len([1 for name, _ in made if name == "rapid_linear"]) == 10


def test_a_trace_is_played_with_the_layers_device_current(monkeypatch):
    from paper_2509_22323_amd import sampler
    layer, current, made = make(), Current(monkeypatch), []
    layer.device = 1
    monkeypatch.setattr(sampler, "_run_layer_trace", lambda *a: made.append(current.device))
    sampler.run_action_trace([(0, 0)], None, None, None, None, 1, 128, None, None, *torch.zeros(3, 2, 8), layer=layer)
    assert made == [1] and current.device == 0


@pytest.mark.parametrize("which", [(0, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1)], ids=str)
def test_a_trace_of_layers_needs_tensors_of_its_own(which, monkeypatch):
    from paper_2509_22323_amd import sampler
    Current(monkeypatch)
    monkeypatch.setattr(sampler, "_run_layer_trace", lambda *a: pytest.fail("played"))
    t = torch.zeros(2, 2, 8)
    with pytest.raises(ValueError):
        sampler.run_action_trace([(0, 0)], None, None, None, None, 1, 128, None, None, *(t[i] for i in which), layer=make())
