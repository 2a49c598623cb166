"""Host-only checks of what calls on packed sequences refuse: numbers that fp32 does not hold, and what a layer would refuse half way."""
import pytest
import torch

import paper_2509_22323_amd as ra
from paper_2509_22323_amd import layer as layer_module
from test_joint_layer import weights
from test_packed_abi import A, ALIGN, SHAPE, norm
from test_packed_layer import make, no_calls  # noqa: F401


@pytest.mark.parametrize("kw", [dict(cap=1e-46), dict(scale=1e-46), dict(cap=5e-324, scale=1.0)], ids=str)
def test_caps_and_scales_that_fp32_holds_as_zero(kw):
    """0 would be no cap, or the usual scale: refused before the tensors are looked at"""
    q = torch.zeros((1, 2, 4, 64), dtype=torch.bfloat16)
    for workspace in (None, torch.zeros(4096, dtype=torch.uint8)):
        with pytest.raises(ValueError):
            ra.rapid_attn_packed([(q, q, q, q)], torch.zeros(4, dtype=torch.int32), workspace=workspace, **kw)
    with pytest.raises(TypeError):
        ra.rapid_attn_packed([(q, q, q, q)], torch.zeros(4, dtype=torch.int32), cap=1e-44, scale=1e-44)


@pytest.mark.parametrize("cap", [1e-46, 4e38, 3.4028235677973366e38])
def test_caps_of_a_layer(cap, monkeypatch):
    layer = make()
    monkeypatch.setattr(layer_module, "_b", None)
    with pytest.raises(ValueError):
        layer.run(torch.zeros(77, 128), torch.zeros(9, 128), torch.zeros(3, 128), torch.zeros(86), cap=cap)


def test_a_norm_takes_finite_eps_alone():
    """1 / sqrt(infinity) by Newton's steps would be NaN, not 0 (an unaligned row: nothing is launched)"""
    odd = (A + 8, 0, 64)
    assert norm(eps=float("inf"), x=odd) == SHAPE and norm(eps=3.4e38, x=odd) == ALIGN


@pytest.mark.parametrize("eps", [float("inf"), 1e39, 3.4028235677973366e38, float("nan")])
def test_a_layer_takes_finite_eps_alone(eps):
    with pytest.raises(ValueError):
        make(eps=eps)


@pytest.mark.parametrize("kw", [dict(second=dict(F=2 ** 17)), dict(first=dict(F=2 ** 17)), dict(first=dict(F=16, C=257 * 64), second=dict(F=16, C=257 * 64), H=257)], ids=str)
def test_widths_that_a_run_would_refuse(kw):
    """A product of 2^17 inputs was refused behind the attention's, that is with the image's states half way"""
    with torch.device("meta"):
        streams = [weights(**{"F": 64, **kw.get(name, {})}) for name in ("first", "second")]
    with pytest.raises(ValueError):
        make(*streams, H=kw.get("H", 2))


@pytest.mark.parametrize("kw", [dict(image=torch.zeros(76, 128)), dict(image=torch.zeros(77, 64)), dict(text=torch.zeros(1, 9, 128)), dict(text=torch.zeros(1, 128).expand(9, 128)),
                                dict(image=torch.zeros(77 * 64 + 64).as_strided((77, 128), (64, 1)))], ids=lambda kw: " ".join(kw))
def test_states_that_a_run_would_refuse(kw, monkeypatch):
    """Text whose rows lie upon each other was refused behind the image's last product"""
    layer = make()
    monkeypatch.setattr(layer_module, "_b", None)
    args = dict(image=torch.zeros(77, 128), text=torch.zeros(9, 128), conditioning=torch.zeros(3, 128), document=torch.zeros(86))
    with pytest.raises(ValueError):
        layer.run(**{**args, **kw})
