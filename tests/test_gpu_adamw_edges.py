"""AdamW over tensor lists, gradient norm and scaling on the GPU at their edges: second moments beyond fp32.

Tolerances count roundings (u = 2^-24, half a step of fp32; 2^-8 for a weight stored in bf16).  W = (1 - lr wd) W - lr n: the
factor of W, its product and the sum are 2u |W| + u |W'|.  n differs from the oracle's by 11u |n| (the oracle rounds m c1, the
square root, the sum and the quotient: 4u; the step its square root and reciprocal by one unit in the last place, 2u each, and
lr c1, the sum and a product: 7u); with fp32 moments it is the oracle's own expression, and lr n is rounded: u |lr n|."""
import numpy as np
import pytest
import torch

from helpers import TDT, f32, to64
from oracle import q8_oracle as q8
from paper_2403_03507_amd import binding as gb

pytestmark = pytest.mark.gpu

U, TINY = 2.0 ** -24, 2.0 ** -149
B1, B2, EPS, LR, WD = f32(0.9), f32(0.999), f32(1e-8), f32(1e-3), f32(0.1)


def _same(got, want, bound):
    """NaN where the oracle has NaN, finite and within the bound elsewhere."""
    bad = np.isnan(want)
    assert np.array_equal(np.isnan(got), bad), (int(np.isnan(got).sum()), int(bad.sum()))
    err = np.abs(got[~bad] - want[~bad])
    assert np.all(err <= bound[~bad] + TINY), float((err / (bound[~bad] + TINY)).max())


def _weight_bound(before, n, want, dtype):
    dw = 2 * U * np.abs(before) + LR * 11 * U * np.abs(n) + U * np.abs(want)
    return dw + (2.0 ** -8 * (np.abs(want) + dw) if dtype == "bf16" else 0.0)


@pytest.mark.parametrize("wdt,gdt,master", [("f32", "f32", False), ("bf16", "bf16", False), ("bf16", "f32", True), ("bf16", "bf16", True)])
@pytest.mark.parametrize("size", [7e20, 1e21, 1e30, 3e38])
def test_eight_bit_second_moment_that_overflows(size, wdt, gdt, master):
    # One finite gradient whose square leaves fp32, among ordinary ones.  In that step its weight only decays; its block's
    # scale is infinite then, and what the block's codes stand for is no number any more: NaN in its 256 weights, never a
    # finite step of m / eps.  Every other block as if nothing had happened.
    rng = np.random.default_rng(21)
    shape, n = (3, 700), 2100
    w = torch.from_numpy(rng.standard_normal(shape)).to(TDT[wdt]).cuda()
    opt = gb.GaLoreAdamW([w], moments="q8", master=master, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    Mc, Vc, Ms, Vs = np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros(9, np.float32), np.zeros(9, np.float32)
    spike, block = 300, slice(256, 512)
    others = np.r_[0:256, 512:n]
    for k in range(1, 7):
        g = torch.from_numpy(rng.standard_normal(n) * 1e-3).to(TDT[gdt])
        if k == 2:
            g[spike] = size
        before = to64(opt.master[0] if master else w).reshape(-1)
        opt.step([w], [g.view(shape).cuda()], LR)
        step_n = q8.adam_q8(g.float().numpy(), Mc, Vc, Ms, Vs, B1, B2, EPS, k).astype(np.float64)
        want = (1 - LR * WD) * before - LR * step_n
        after = opt.master[0] if master else w
        _same(to64(after).reshape(-1), want, _weight_bound(before, step_n, want, "f32" if master else wdt))
        if master:
            assert torch.equal(torch.isnan(w), torch.isnan(after)) and torch.equal(w[~torch.isnan(w)], after.bfloat16()[~torch.isnan(w)])
        assert np.array_equal(opt.V[0].cpu().numpy().reshape(-1)[others], Vc[others])
        assert np.array_equal(np.delete(opt.V_scale[0].cpu().numpy(), 1), np.delete(Vs, 1))
        assert np.array_equal(opt.M_scale[0].cpu().numpy(), Ms)
        got = to64(after).reshape(-1)
        if k == 2:
            assert step_n[spike] == 0.0 and np.isfinite(got).all() and np.isinf(float(opt.V_scale[0][1]))
        if k > 2:
            assert np.isnan(got[block]).all() and np.isfinite(got[others]).all()
            assert not np.isfinite(float(opt.V_scale[0][1]))                     # a check of the states sees it as well


@pytest.mark.parametrize("scale", [float("inf"), float("nan")])
def test_eight_bit_state_whose_scale_is_no_number(scale):
    # a state that was loaded with such a scale: its block shows it
    rng = np.random.default_rng(22)
    w = torch.from_numpy(rng.standard_normal((5, 300))).float().cuda()
    g = torch.from_numpy(rng.standard_normal((5, 300)) * 1e-3).float().cuda()
    opt, ref = (gb.GaLoreAdamW([x], moments="q8", beta1=B1, beta2=B2, eps=EPS) for x in (w, w.clone()))
    clean = w.clone()
    opt.V_scale[0][2] = scale
    opt.step([w], [g], LR)
    ref.step([clean], [g], LR)
    w, clean = w.view(-1), clean.view(-1)
    assert torch.isnan(w[512:768]).all()
    assert torch.equal(w[:512], clean[:512]) and torch.equal(w[768:], clean[768:])


@pytest.mark.parametrize("size", [7e20, 1e30])
def test_fp32_second_moment_that_overflows(size):
    # only the weight of that gradient is touched by it, and that one decays from then on
    rng = np.random.default_rng(23)
    shape = (3, 700)
    w = torch.from_numpy(rng.standard_normal(shape)).float().cuda()
    clean = w.clone()
    opt, ref = (gb.GaLoreAdamW([x], beta1=B1, beta2=B2, eps=EPS, weight_decay=WD) for x in (w, clean))
    for k in range(1, 6):
        g = torch.from_numpy(rng.standard_normal(shape) * 1e-3).float().cuda()
        ref.step([clean], [g], LR)
        if k == 2:
            g.view(-1)[300] = size
        before = float(w.view(-1)[300])
        opt.step([w], [g], LR)
        if k >= 2:
            want = (1 - LR * WD) * before                                        # n = m / inf
            assert abs(float(w.view(-1)[300]) - want) <= 3 * U * abs(before)
        same = torch.ones(2100, dtype=torch.bool, device="cuda")
        same[300] = False
        assert torch.equal(w.view(-1)[same], clean.view(-1)[same])
