"""What the Python face of AdamW over tensor lists does on the host: order of calls, refusals (no GPU)."""
import pytest
import torch

from paper_2403_03507_amd import binding as gb
from paper_2403_03507_amd.hooks import PerLayerGaLore


class _Recorder:
    """Stands in for the library's two optimizers of a PerLayerGaLore and notes the calls."""

    def __init__(self, error=None):
        self.calls, self.error = [], error

    def join(self):
        self.calls.append("join")

    def step(self, weights, grads, lr, stats=None):
        self.calls.append("step")
        if self.error:
            raise self.error


def _driver(others, error=None):
    drv = object.__new__(PerLayerGaLore)
    drv.opt = drv.others_opt = _Recorder(error)
    drv.others, drv.others_lr, drv._others_array = others, 1e-3, None
    return drv


def _params(n):
    params = [torch.nn.Parameter(torch.ones(3)) for _ in range(n)]
    for p in params:
        p.grad = torch.ones(3)
    return params


def test_finish_joins_the_streams_when_it_raises():
    # the hooks have started GaLore steps on the library's streams: whatever finish() refuses, they are ordered first
    params = _params(3)
    params[1].grad = None
    drv = _driver(params)
    with pytest.raises(ValueError):
        drv.finish()
    assert drv.opt.calls == ["join"]                                             # and nothing was stepped
    assert params[0].grad is not None and params[2].grad is not None
    for error in (ValueError("a gradient of another kind"), gb.GaloreError(1, "refused")):
        params = _params(2)
        drv = _driver(params, error)
        with pytest.raises(type(error)):
            drv.finish()
        assert drv.opt.calls == ["step", "join"] and all(p.grad is not None for p in params)


def test_finish_steps_and_joins():
    params = _params(2)
    drv = _driver(params)
    drv.finish()
    assert drv.opt.calls == ["step", "join"] and all(p.grad is None for p in params)
    drv = _driver([])
    drv.finish()
    assert drv.opt.calls == ["join"]


def test_rates_that_no_step_could_take_are_refused():
    plain, captured = gb.GaLoreAdamW([], device="cpu"), gb.GaLoreAdamW([], device="cpu", capturable=True)
    with pytest.raises(ValueError):
        plain.set_lr(1e-3)                                                       # has no rate on the device
    with pytest.raises(ValueError):
        plain.step([], [])                                                       # nor one of its own
    assert plain.t == 0
    for bad in (float("nan"), float("inf"), -float("inf")):
        with pytest.raises(ValueError):
            captured.set_lr(bad)
        with pytest.raises(ValueError):
            captured.step([], [], bad)
        assert not captured.clock.any()
    captured.set_lr(0.25)
    assert float(captured.clock[8:12].view(torch.float32)) == 0.25
    captured.set_lr(torch.tensor(0.5))                                           # a schedule's tensor is not looked at
    assert float(captured.clock[8:12].view(torch.float32)) == 0.5


def _described(monkeypatch):
    """param_desc of host tensors as if they were the device's: only what happens before a launch is looked at."""
    monkeypatch.setattr(gb, "param_desc", lambda t: gb.galore_tensor(1 << 20, 1, t.numel(), t.numel(), gb.GALORE_F32))


def test_states_on_another_device_than_the_weights_are_refused(monkeypatch):
    _described(monkeypatch)
    w = torch.zeros(8)
    for options in ({}, {"moments": "q8"}, {"capturable": True}):
        with pytest.raises(ValueError, match="device"):
            gb.GaLoreAdamW([w], device="meta", **options)
    assert gb.GaLoreAdamW([w], device="cpu").M_flat.device == w.device


def test_a_step_on_another_device_than_the_states_is_refused(monkeypatch):
    _described(monkeypatch)
    calls = []
    monkeypatch.setattr(gb, "galore_adamw", lambda *a: calls.append(a))
    opt = gb.GaLoreAdamW([torch.zeros(8)], device="cpu")                         # where get_device() is -1
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    array = gb.tensor_array([gb.galore_tensor(1 << 20, 1, 8, 8, gb.GALORE_F32)])
    with pytest.raises(ValueError, match="device"):
        opt.step(array, array, 1e-3)
    assert not calls and opt.t == 0
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    opt.step(array, array, 1e-3)
    assert len(calls) == 1 and opt.t == 1


def test_a_workspace_that_is_no_device_memory_is_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(gb, "_stats_ptr", lambda stats: 1 << 20)
    need = gb.galore_grad_norm_workspace_bytes(1)
    array = gb.tensor_array([gb.galore_tensor(1 << 20, 1, 8, 8, gb.GALORE_F32)])
    with pytest.raises(ValueError, match="workspace"):
        gb.galore_grad_norm(array, 1.0, 1.0, None, torch.zeros(need, dtype=torch.uint8))


def test_buffers_whose_addresses_the_states_hold_cannot_be_replaced(monkeypatch):
    # a loaded state is copied into them: an assignment would leave the library with the address of freed memory
    _described(monkeypatch)
    opt = gb.GaLoreAdamW([torch.zeros(8), torch.zeros(300)], moments="q8", device="cpu", capturable=True)
    for name in ("M_flat", "V_flat", "M_scale_flat", "V_scale_flat", "master_flat"):
        before = getattr(opt, name)
        with pytest.raises(AttributeError):
            setattr(opt, name, torch.zeros(1024, dtype=torch.uint8))
        assert getattr(opt, name) is before
    assert opt.M_flat.shape == (768,) and opt.M_scale_flat.shape == (3,) and opt.master_flat is None
    opt.M_flat.copy_(torch.full((768,), 7, dtype=torch.uint8))                   # tensors start at multiples of 256
    assert opt.M[1].shape == (300,) and bool((opt.M[1] == 7).all())


@pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64])
def test_states_do_not_follow_the_default_dtype(default, monkeypatch):
    # the library is told fp32: buffers of the default type would be too short
    monkeypatch.setattr(gb, "param_desc", lambda t: gb.galore_tensor(1 << 20, 1, t.numel(), t.numel(), gb.GALORE_BF16))
    w = torch.zeros(300, dtype=torch.bfloat16)
    torch.set_default_dtype(default)
    try:
        q8 = gb.GaLoreAdamW([w], moments="q8", master=True, device="cpu", capturable=True)
        plain = gb.GaLoreAdamW([w], master=True, device="cpu")
        norm = gb.GaLoreGradNorm(1, device="cpu")
    finally:
        torch.set_default_dtype(torch.float32)
    assert q8.M_scale_flat.dtype == q8.V_scale_flat.dtype == q8.master_flat.dtype == torch.float32
    assert plain.M_flat.dtype == plain.V_flat.dtype == plain.master_flat.dtype == norm.stats.dtype == torch.float32
    assert q8.M_flat.dtype == q8.V_flat.dtype == q8.clock.dtype == norm.workspace.dtype == torch.uint8
