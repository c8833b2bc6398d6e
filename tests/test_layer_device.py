"""Resident layers on a device that is not the current one, without a GPU: every call of the library that
goes to the current device's stream finds the layer's device current."""
import pytest
import torch

from dmoe_synth import TINY, layer_inputs
from paper_2605_30876_gb300 import layer as L

CURRENT_DEVICE_CALLS = ("dmoe_router", "dmoe_dispatch", "dmoe_router_prepare", "dmoe_layer_forward",
                        "dmoe_q4_swiglu", "dmoe_q4_linear", "dmoe_combine_rows", "dmoe_q4_quantize")


@pytest.fixture
def calls(monkeypatch):
    """(call, the current device) of each library call; device 0 is current, host tensors stand for others."""
    at, seen = [0], []

    class on:
        def __init__(self, device):
            self.index = device.index

        def __enter__(self):
            self.before, at[0] = at[0], self.index

        def __exit__(self, *_):
            at[0] = self.before
    monkeypatch.setattr(torch.cuda, "current_device", lambda: at[0])
    monkeypatch.setattr(torch.cuda, "device", on)
    for name in CURRENT_DEVICE_CALLS:
        monkeypatch.setattr(L, name, lambda *a, _n=name, **k: seen.append((_n, at[0])))
    return seen


@pytest.mark.parametrize("kind", ["MoELayer", "MoELayerQ4"])
@pytest.mark.parametrize("shared", [0, 128, 256])
def test_a_layer_runs_on_its_own_device(calls, kind, shared):
    shape = TINY.with_(d_ff_shared=shared)
    layer = getattr(L, kind).from_shape(shape, layer_inputs(shape, seed=0, device="cpu"), device="cpu")
    del calls[:]
    x = torch.zeros(shape.T, shape.d_model, dtype=torch.bfloat16)
    for index in (1, 0):
        layer.device = torch.device("cuda", index)
        layer.prepare()
        layer.forward(x)
        assert len(calls) >= 2 and all(at == index for _, at in calls), calls
        del calls[:]
    assert torch.cuda.current_device() == 0


def test_cuda_is_the_device_that_was_current():
    assert L._indexed("cuda:2").index == 2 and L._indexed("cpu").type == "cpu"


def test_cuda_without_a_number(calls):
    assert L._indexed("cuda") == torch.device("cuda", 0)
    with torch.cuda.device(torch.device("cuda", 1)):
        assert L._indexed("cuda") == torch.device("cuda", 1)


def test_weights_elsewhere_are_refused(calls):
    weights = layer_inputs(TINY, seed=0, device="cpu")
    with pytest.raises(ValueError, match="w_r"):
        L.MoELayerQ4.from_shape(TINY, weights, device="cuda:1")
    with pytest.raises(ValueError, match="workspace"):
        L.MoELayerQ4.from_shape(TINY, weights, device="cpu", workspace=torch.empty(1, device="meta"))
    assert calls == []


def test_other_shapes_are_refused_before_any_call(calls):
    """Fewer tokens than the layer's (the router would read behind them), an output of half the rows (its
    slots would be taken for twice as many), another width, another device."""
    layer = L.MoELayerQ4.from_shape(TINY, layer_inputs(TINY, seed=0, device="cpu"), device="cpu")
    del calls[:]
    T, d = TINY.T, TINY.d_model
    good = torch.zeros(T, d, dtype=torch.bfloat16)
    for bad in (good[:-1], good[: T // 2], good[:, :-8], good[None], good.to("meta"), torch.cat([good, good])):
        with pytest.raises(ValueError, match="x: expected"):
            layer.forward(bad)
        with pytest.raises(ValueError, match="y: expected"):
            layer.forward(good, bad)
    assert calls == []
    assert layer.forward(good, good.clone()) is not None and len(calls) >= 5
