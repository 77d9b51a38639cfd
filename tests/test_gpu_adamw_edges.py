"""AdamW over tensor lists, gradient norm and scaling on the GPU at their edges: second moments beyond fp32, memory next to
the tensors, ends around a workgroup's elements, lists of many workgroups, the stream that the calls go to, steps
that are left out.

Tolerances count roundings (u = 2^-24, half a step of fp32; 2^-8 for a weight stored in bf16).  W = (1 - lr wd) W - lr n: the
factor of W, its product and the sum are 2u |W| + u |W'|.  n differs from the oracle's by 11u |n| (the oracle rounds m c1, the
square root, the sum and the quotient: 4u; the step its square root and reciprocal by one unit in the last place, 2u each, and
lr c1, the sum and a product: 7u).  Bounds for fp32 moments stand at their tests."""
import numpy as np
import pytest
import torch

from helpers import TDT, f32, to64
from oracle import adamw_oracle as ao
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


# ---- memory next to the tensors --------------------------------------------------------------------

# ends around 8 elements, a block of 256, and what a workgroup takes (512 elements; with 8-bit moments 1024)
SIZES = [(1, 1), (1, 7), (5, 1), (1, 9), (3, 85), (1, 255), (1, 257), (1, 511), (1, 512), (1, 513), (1, 1023), (1, 1024), (1, 1025),
         (7, 73), (2, 511), (3, 513), (2, 1023), (33, 31), (9, 1025), (1, 2047), (5, 2049)]


def _placed(rng, shape, dtype, gap, offset):
    """A matrix in a buffer that holds numbers everywhere: none of them may change but the matrix's own."""
    rows, cols = shape
    buf = torch.from_numpy(rng.uniform(0.5, 2.0, offset + rows * (cols + gap) + 40) * rng.choice([-1.0, 1.0])).to(TDT[dtype]).cuda()
    return buf, buf[offset:offset + rows * (cols + gap)].view(rows, cols + gap)[:, :cols]


def _around(buf, view):
    """The buffer with the view's own elements out of it."""
    inside = torch.zeros(buf.numel(), dtype=torch.bool, device="cuda")
    inside.as_strided(view.shape, view.stride(), view.storage_offset())[:] = True
    return buf[~inside]


@pytest.mark.parametrize("gaps", [True, False])
@pytest.mark.parametrize("moments", ["f32", "q8"])
@pytest.mark.parametrize("wdt,gdt,master", [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "bf16", False), ("bf16", "f32", False),
                                            ("bf16", "bf16", True), ("bf16", "f32", True)])
def test_a_step_changes_nothing_next_to_its_tensors(wdt, gdt, master, moments, gaps):
    rng = np.random.default_rng(31)
    W = [_placed(rng, s, wdt, gaps * (i % 4) * 3, (0, 1, 3)[i % 3]) for i, s in enumerate(SIZES)]
    G = [_placed(rng, s, gdt, gaps * (i % 3), i % 2) for i, s in enumerate(SIZES)]
    weights, grads = [w for _, w in W], [g for _, g in G]
    opt = gb.GaLoreAdamW(weights, moments=moments, master=master, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    states = [opt.M_flat, opt.V_flat] + ([opt.master_flat] if master else [])
    own = torch.zeros(opt.M_flat.numel(), dtype=torch.bool, device="cuda")
    for m in opt.M:
        own[m.storage_offset():m.storage_offset() + m.numel()] = True
    for s in states:
        s[~own] = 77                                                             # between two tensors' states
    keep_w, keep_g, before = [_around(*w).clone() for w in W], [b.clone() for b, _ in G], [w.clone() for w in weights]
    for _ in range(2):
        opt.step(weights, grads, LR)
    for i in range(len(SIZES)):
        assert torch.equal(_around(*W[i]), keep_w[i]), SIZES[i]
        assert torch.equal(G[i][0], keep_g[i]), SIZES[i]
        # and every element of its own was stepped: by about lr twice, which bf16 may round away
        if wdt == "f32":
            assert bool((weights[i] != before[i]).all()), SIZES[i]
        assert bool((opt.M[i] != 0).all()), SIZES[i]
    for s in states:
        assert bool((s[~own] == 77).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("finite", [1.0, 0.0])
def test_scaling_changes_nothing_next_to_its_tensors(dtype, finite):
    rng = np.random.default_rng(32)
    sizes = SIZES + [(3, 5000), (700, 9), (1, 4096), (1, 4097)]
    G = [_placed(rng, s, dtype, (i % 4) * 3, (0, 1, 3)[i % 3]) for i, s in enumerate(sizes)]
    keep, before = [_around(*g).clone() for g in G], [g.clone() for _, g in G]
    norm = gb.GaLoreGradNorm(len(G))
    norm.scale([g for _, g in G], torch.tensor([1.0, 0.5 * finite, finite, 0.0], device="cuda"))
    for i, (buf, view) in enumerate(G):
        assert torch.equal(_around(buf, view), keep[i]), sizes[i]
        assert torch.equal(view, before[i] * 0.5 if finite else torch.zeros_like(view)), sizes[i]     # halves are exact


# ---- lists of many workgroups ----------------------------------------------------------------------

@pytest.mark.parametrize("moments,wdt", [("f32", "f32"), ("f32", "bf16"), ("q8", "bf16"), ("q8", "f32")])
@pytest.mark.parametrize("gap", [0, 3])
def test_every_element_of_a_list_of_many_workgroups(moments, wdt, gap):
    # From 4096 workgroups (2.1M elements, with 8-bit moments 4.2M) on a launch numbers them by XCD.  All elements of two full
    # groups and a rest of such workgroups, against calls on pieces that are too short for that (multiples of 256 elements).
    rng = np.random.default_rng(33)
    shapes = [(1, 2500001), (1, 33), (700, 2001), (1, 4100000), (1100, 1101)]
    total = sum(m * n for m, n in shapes)
    assert 2 * 4096 * 512 < total and 2 * 4096 * 1024 < total < 3 * 4096 * 1024
    gen = torch.Generator("cuda").manual_seed(4)
    rand = lambda m, n: torch.randn(m, n + gap, generator=gen, device="cuda").to(TDT[wdt])[:, :n]
    W, G = [rand(*s) for s in shapes], [rand(*s) for s in shapes]
    pieces_w, pieces_g, at = [], [], []
    for i, (w, g) in enumerate(zip(W, G)):
        flat_w, flat_g = w.reshape(-1).clone(), g.reshape(-1).clone()
        for a in range(0, flat_w.numel(), 1 << 20):
            pieces_w.append(flat_w[a:a + (1 << 20)])
            pieces_g.append(flat_g[a:a + (1 << 20)])
            at.append((i, a))
    opt = gb.GaLoreAdamW(W, moments=moments, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    singles = [gb.GaLoreAdamW([w], moments=moments, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD) for w in pieces_w]
    start = [to64(w) for w in W]
    for _ in range(2):
        opt.step(W, G, LR)
        for o, w, g in zip(singles, pieces_w, pieces_g):
            o.step([w], [g], LR)
    for (i, a), o, w in zip(at, singles, pieces_w):
        cut = lambda t: t.reshape(-1)[a:a + w.numel()]
        assert torch.equal(cut(W[i]), w) and torch.equal(cut(opt.M[i]), o.M[0]) and torch.equal(cut(opt.V[i]), o.V[0]), (i, a)
        if moments == "q8":
            blocks = slice(a // 256, a // 256 + o.M_scale[0].numel())
            assert torch.equal(opt.M_scale[i][blocks], o.M_scale[0]) and torch.equal(opt.V_scale[i][blocks], o.V_scale[0]), (i, a)
    if moments == "f32":
        # Both ways could be wrong together: the weights against the oracle.  With one gradient in both steps every sum has terms of
        # one sign: m is off by 2u, v by 3u; the corrections and their products are 2u each, so that sqrt(v c2) + eps is off by
        # 5u / 2 + 2u and n by 2u + 2u + 4.5u + u < 10u; the weight's factor, its product and the sum are 3u of it.  The 20u
        # below leave room for |W'| <= |W| + lr.
        for i, g in enumerate(G):
            m, v, w = 0.0, 0.0, start[i]
            for k in (1, 2):
                before = w
                w, m, v, n = ao.adamw(w, to64(g), m, v, B1, B2, EPS, LR, WD, k)
            largest = np.maximum(np.abs(start[i]), np.abs(before))
            bound = 2 * (3 * U * largest + LR * 20 * U * np.abs(n) + TINY)
            if wdt == "bf16":
                bound = bound + 2 * 2.0 ** -8 * (np.maximum(largest, np.abs(w)) + LR) * 1.01
            assert np.all(np.abs(to64(W[i]) - w) <= bound)


# ---- the stream ------------------------------------------------------------------------------------

@pytest.mark.parametrize("call", ["measure", "scale", "step_f32", "step_q8", "tick"])
def test_a_call_waits_for_its_own_stream(call):
    # what it reads is written at the end of long work on a stream of the caller's: a call on any other stream would read
    # what was there before.  All results are exact: powers of two.
    n = 1 << 20
    g, w, before = torch.empty(n, device="cuda"), torch.zeros(n, device="cuda"), torch.tensor([7.0, 7.0, 0.0, 0.0], device="cuda")
    big = torch.ones(1 << 28, device="cuda")                                     # 1 GiB: a pass over it takes about 0.4 ms
    norm = gb.GaLoreGradNorm(1, max_norm=1024.0)
    opt = gb.GaLoreAdamW([w], moments="q8" if call == "step_q8" else "f32", beta1=0.5, beta2=0.75, eps=0.0, capturable=call == "tick")
    ready = torch.tensor([2048.0, 0.5, 1.0, 0.0], device="cuda")
    side = torch.cuda.Stream()
    for _ in range(2):
        g.fill_(1.0)
        norm.stats.copy_(before)
        opt.M_flat.zero_(); opt.V_flat.zero_(); opt.t = 0
        if opt.clock is not None:
            opt.clock.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(60):
                big.mul_(1.0)
            g.fill_(2.0)
            if call == "measure":
                out = norm.measure([g]).clone()
            elif call == "scale":
                norm.stats.copy_(ready)
                norm.scale([g])
                out = g.clone()
            elif call == "tick":
                opt.clock[:8].view(torch.int64).fill_(4)
                gb.galore_adamw_tick(opt.clock, 0.5, 0.75)
                out = opt.clock.clone()
            else:
                opt.step([w], [g], 0.5)
                out = torch.cat([(opt.M_scale_flat if call == "step_q8" else opt.M_flat), (opt.V_scale_flat if call == "step_q8" else opt.V_flat)])
        side.synchronize()
        if call == "measure":
            assert out.tolist() == [2048.0, 0.5, 1.0, 0.0]                       # sqrt(4 * 2^20); 1024 / 2048.000001 in fp32
        elif call == "scale":
            assert bool((out == 1.0).all())
        elif call == "tick":
            assert int(out[:8].view(torch.int64)) == 5
        else:
            half = out.numel() // 2
            assert bool((out[:half] == 1.0).all()) and bool((out[half:] == 1.0).all())    # g / 2 and g^2 / 4


# ---- steps that are left out -----------------------------------------------------------------------

@pytest.mark.parametrize("moments", ["f32", "q8"])
def test_hooks_with_the_count_on_the_device_leave_out_steps_that_are_not_finite(moments):
    # others_options={"capturable": True}: a step whose gradients were not finite neither moves anything nor counts
    from paper_2403_03507_amd.hooks import PerLayerGaLore

    gen = torch.Generator("cuda").manual_seed(9)
    fresh = lambda: [torch.randn(s, generator=gen, device="cuda") for s in ((48, 64), (64,), (5, 7))]
    start = fresh()
    mat, vec, emb = (torch.nn.Parameter(x.clone()) for x in start)
    drv = PerLayerGaLore([[mat]], 8, 1e-2, update_gap=100, refresh_iters=3, others=[vec, emb], others_lr=3e-2,
                         others_options={"moments": moments, "weight_decay": 0.1, "capturable": True})
    ref_w = [x.clone() for x in start[1:]]
    ref = gb.GaLoreAdamW(ref_w, moments=moments, weight_decay=0.1)
    norm, ref_norm = gb.GaLoreGradNorm(2, max_norm=1.0), gb.GaLoreGradNorm(2, max_norm=1.0)
    for i in range(5):
        g = fresh()
        if i in (0, 3):
            g[2][4, 6] = float("inf")
        sum((p * x).sum() for p, x in zip((mat, vec, emb), g)).backward()
        drv.finish(norm.measure([vec.grad, emb.grad]))
        if i not in (0, 3):
            ref.step(ref_w, g[1:], 3e-2, ref_norm.measure(g[1:]))
        torch.cuda.synchronize()
        assert torch.equal(vec.data, ref_w[0]) and torch.equal(emb.data, ref_w[1]), i
        assert drv.others_opt.count() == ref.t
    drv.close()
