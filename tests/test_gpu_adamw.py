"""AdamW over tensor lists on the GPU against the fp64 oracle.

Tolerances count roundings (u = 2^-24, half a step of fp32; 2^-8 for a weight stored in bf16).  With g = s G:
  m = fma(b1, m, (1-b1) g): g, the product and the sum are rounded             |dm| <= 3u (|b1 m| + |(1-b1) g|)
  v: g twice, two products, the sum; all terms positive                        |dv| <= 5u v
  n = (m c1) / (sqrt(v c2) + eps): c1, c2, two products, square root, sum, quotient, and half of v's error
                                                                               |dn| <= c1 |dm| / den + 10u |n|
  W: 1 - lr wd, its product, the sum                                           |dW| <= 2u |W| + lr |dn| + u |W'|
Smaller numbers than fp32's normal ones are allowed one of its smallest steps."""
import numpy as np
import pytest
import torch

from helpers import TDT, f32, to64
from oracle import adamw_oracle as ao
from oracle import q8_oracle as q8
from paper_2403_03507_amd import binding as gb

pytestmark = pytest.mark.gpu

U, TINY = 2.0 ** -24, 2.0 ** -149
B1, B2, EPS, LR, WD = f32(0.9), f32(0.999), f32(1e-8), f32(1e-2), f32(0.1)
STORED = {torch.float32: 0.0, torch.bfloat16: 2.0 ** -8}

# one element, less than a vector, vectors and a rest, lengths around powers of two from the blocks of 256 on
SIZES = [(1, 1), (1, 3), (3, 1), (1, 255), (1, 256), (1, 257), (7, 5), (33, 1023), (2, 1024), (1, 2047), (1, 2049), (64, 129), (5, 8193), (1, 16384)]


def _rand(rng, *shape, wide=4.0):
    """Values of unequal size, zeros among them."""
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-wide, 1, shape))
    return np.where(rng.random(shape) < 0.05, 0.0, x)


def _place(x, dtype, ld_pad=0, offset=0):
    """x on the GPU: rows `ld_pad` further apart than their length, from an element offset on; NaN around it."""
    rows, cols = x.shape
    buf = torch.full((offset + rows * (cols + ld_pad) + 9,), float("nan"), dtype=dtype, device="cuda")
    view = buf[offset:offset + rows * (cols + ld_pad)].view(rows, cols + ld_pad)[:, :cols]
    view.copy_(torch.from_numpy(x))
    return buf, view


def _outside_is_nan(buf, view):
    keep = buf.clone()
    off = view.storage_offset()
    rows, cols = view.shape
    keep[off:off + rows * view.stride(0)].view(rows, view.stride(0))[:, :cols] = float("nan") if rows * view.stride(0) + off <= keep.numel() else 0
    return bool(torch.isnan(keep).all())


def _stats(scale, finite=1.0):
    return torch.tensor([123.0, scale, finite, 0.0], device="cuda")


def _bounds(w, g, m, v, k, scale, wd, lr=LR):
    """Oracle results of one step and the bounds above (fp64)."""
    gs = scale * g
    w1, m1, v1, n = ao.adamw(w, gs, m, v, B1, B2, EPS, lr, wd, k)
    dm = 3 * U * (np.abs(B1 * m) + np.abs((1 - B1) * gs)) + TINY
    dv = 5 * U * v1 + 2 * TINY
    c1, den = 1 / (1 - B1 ** k), np.sqrt(v1 / (1 - B2 ** k)) + EPS
    dn = c1 * dm / den + 10 * U * np.abs(n) + TINY
    dw = 2 * U * np.abs(w) + lr * dn + U * np.abs(w1) + TINY
    return (w1, m1, v1), (dw, dm, dv)


def _within(got, want, bound, dtype=torch.float32):
    got = got if isinstance(got, np.ndarray) else to64(got)
    err = np.abs(got - want)
    ok = err <= bound + STORED[dtype] * (np.abs(want) + bound) + TINY
    assert np.all(ok), (float(err.max()), float((err / np.maximum(bound + STORED[dtype] * np.abs(want), 1e-300)).max()), int((~ok).sum()))


@pytest.mark.parametrize("gaps", [True, False])
@pytest.mark.parametrize("scale", [None, 0.37])
@pytest.mark.parametrize("wdt,gdt,master", [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "bf16", False), ("bf16", "f32", False),
                                            ("bf16", "bf16", True), ("bf16", "f32", True)])
def test_one_step_of_a_list_of_all_sizes(wdt, gdt, master, scale, gaps):
    rng = np.random.default_rng(11)
    stats = None if scale is None else _stats(scale)
    s = 1.0 if scale is None else f32(scale)
    W, G, decay, start = [], [], [], []
    for i, shape in enumerate(SIZES):
        pad, off = ((0, 0), (3, 0), (0, 1), (5, 3))[i % 4]
        W.append(_place(_rand(rng, *shape), TDT[wdt], pad * gaps, off))
        G.append(_place(_rand(rng, *shape), TDT[gdt], (i % 3) * 2 * gaps, i % 2))
        decay.append(WD if i % 2 else 0.0)
    opt = gb.GaLoreAdamW([w for _, w in W], master=master, beta1=B1, beta2=B2, eps=EPS, weight_decay=decay)
    opt.t = 6
    for i, shape in enumerate(SIZES):
        opt.M[i].copy_(torch.from_numpy(_rand(rng, *shape)))
        opt.V[i].copy_(torch.from_numpy(_rand(rng, *shape) ** 2))
        if master:
            opt.master[i].copy_(torch.from_numpy(_rand(rng, *shape)))
        start.append((to64(opt.master[i] if master else W[i][1]), to64(G[i][1]), to64(opt.M[i]), to64(opt.V[i])))
    opt.step([w for _, w in W], [g for _, g in G], LR, stats)
    torch.cuda.synchronize()
    for i in range(len(SIZES)):
        (w1, m1, v1), (dw, dm, dv) = _bounds(*start[i], 7, s, decay[i])
        _within(opt.M[i], m1, dm)
        _within(opt.V[i], v1, dv)
        if master:
            _within(opt.master[i], w1, dw)
            assert torch.equal(W[i][1], opt.master[i].to(torch.bfloat16))
        else:
            _within(W[i][1], w1, dw, TDT[wdt])
        assert _outside_is_nan(*W[i])                                  # nothing written around the weight
        assert np.array_equal(to64(G[i][1]), start[i][1])
    for flat, parts in ((opt.M_flat, opt.M), (opt.V_flat, opt.V)):      # nor between two states
        rest = flat.clone()
        for p in parts:
            at = p.storage_offset()
            rest[at:at + p.numel()] = 0
        assert not rest.any()


@pytest.mark.parametrize("master,gaps", [(False, True), (False, False), (True, True)])
def test_eight_bit_moments_equal_the_format_bit_for_bit(master, gaps):
    # codes and scales against the oracle that replays the fp32 operations of the format; the weight follows from its N
    rng = np.random.default_rng(5)
    sizes = SIZES + [(40, 512), (3, 771), (9, 20000)]
    for wdt, gdt in (("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32"), ("f32", "bf16")):
        if master and wdt == "f32":
            continue
        W, G, ref = [], [], []
        for i, shape in enumerate(sizes):
            W.append(_place(_rand(rng, *shape), TDT[wdt], (i % 3) * 4 * gaps, i % 2))
            G.append(_place(_rand(rng, *shape), TDT[gdt], (i % 2) * 3 * gaps, (i % 4)))
        opt = gb.GaLoreAdamW([w for _, w in W], moments="q8", master=master, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
        for shape in sizes:
            n = shape[0] * shape[1]
            ref.append((np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros(-(-n // 256), np.float32), np.zeros(-(-n // 256), np.float32)))
        for k in range(1, 5):
            scale = f32(0.6) if k % 2 else 1.0
            for i, shape in enumerate(sizes):
                g = _rand(rng, *shape)
                if k == 3:
                    g[:, :300] = 0.0                                    # blocks of zero gradients
                G[i][1].copy_(torch.from_numpy(g))
            before = [to64(opt.master[i] if master else W[i][1]) for i in range(len(sizes))]
            opt.step([w for _, w in W], [g for _, g in G], LR, _stats(scale) if k % 2 else None)
            torch.cuda.synchronize()
            for i, shape in enumerate(sizes):
                Mc, Vc, Ms, Vs = ref[i]
                g = (np.float32(scale) * G[i][1].float().cpu().numpy().reshape(-1)).astype(np.float32)
                n = q8.adam_q8(g, Mc, Vc, Ms, Vs, B1, B2, EPS, k).astype(np.float64).reshape(shape)
                got = opt.M[i].cpu().numpy().reshape(-1)
                assert np.array_equal(np.where(got == 0x80, 0, got), np.where(Mc == 0x80, 0, Mc)), (i, k)   # the zero's sign is free
                assert np.array_equal(opt.V[i].cpu().numpy().reshape(-1), Vc), (i, k)
                assert np.array_equal(opt.M_scale[i].cpu().numpy(), Ms) and np.array_equal(opt.V_scale[i].cpu().numpy(), Vs), (i, k)
                # n once more with other roundings.  The oracle rounds m c1, the square root, the sum and the quotient (u
                # each); the kernel's square root and reciprocal are good to one unit in the last place (2u each), and it
                # rounds lr c1, the sum and m times the reciprocal: 4u + 4u + 3u = 11u of n
                want = (1 - LR * WD) * before[i] - LR * n
                dw = 2 * U * np.abs(before[i]) + LR * 11 * U * np.abs(n) + U * np.abs(want)
                if master:
                    _within(opt.master[i], want, dw)
                    assert torch.equal(W[i][1], opt.master[i].to(torch.bfloat16))
                else:
                    _within(W[i][1], want, dw, TDT[wdt])
        for i in range(len(sizes)):
            assert _outside_is_nan(*W[i])


@pytest.mark.parametrize("size", [1e-38, 1e-25, 1e-20, 1e-10, 1e6, 1e12, 1e18])
def test_eight_bit_moments_at_extreme_magnitudes(size):
    # scales that are subnormal or zero (reciprocals beyond fp32), and second moments beyond 2^31 times their codes' range
    rng = np.random.default_rng(6)
    w = torch.from_numpy(rng.standard_normal((3, 700))).float().cuda()
    opt = gb.GaLoreAdamW([w], moments="q8", beta1=B1, beta2=B2, eps=EPS)
    n = w.numel()
    Mc, Vc, Ms, Vs = np.zeros(n, np.uint8), np.zeros(n, np.uint8), np.zeros(9, np.float32), np.zeros(9, np.float32)
    for k in range(1, 4):
        g = (rng.standard_normal(n) * size).astype(np.float32)
        before = to64(w).reshape(-1)
        opt.step([w], [torch.from_numpy(g).view(3, 700).cuda()], LR)
        want_n = q8.adam_q8(g, Mc, Vc, Ms, Vs, B1, B2, EPS, k).astype(np.float64)
        got = opt.M[0].cpu().numpy().reshape(-1)
        assert np.array_equal(np.where(got == 0x80, 0, got), np.where(Mc == 0x80, 0, Mc)), k
        assert np.array_equal(opt.V[0].cpu().numpy().reshape(-1), Vc), k
        assert np.array_equal(opt.M_scale[0].cpu().numpy(), Ms) and np.array_equal(opt.V_scale[0].cpu().numpy(), Vs), k
        want = before - LR * want_n
        # as in the test above; a square root below 1.1e-19 counts as that, 1.1e-11 of the smallest denominator eps
        _within(to64(w).reshape(-1), want, 2 * U * np.abs(before) + LR * 12 * U * np.abs(want_n) + U * np.abs(want))


def test_blocks_of_256_are_those_of_the_low_rank_state():
    # a matrix with rows of a multiple of 256 elements: the same codes and scales as galore_adam_q8 leaves
    rng = np.random.default_rng(3)
    g = torch.from_numpy(_rand(rng, 24, 768)).float().cuda()
    w = torch.zeros(24, 768, device="cuda")
    opt = gb.GaLoreAdamW([w], moments="q8")
    Mc, Vc = torch.zeros(24, 768, dtype=torch.uint8, device="cuda"), torch.zeros(24, 768, dtype=torch.uint8, device="cuda")
    Ms, Vs = torch.zeros(24, 3, device="cuda"), torch.zeros(24, 3, device="cuda")
    N = torch.empty_like(g)
    for k in range(1, 4):
        opt.step([w], [g], 1e-3)
        gb.galore_adam_q8(g, Mc, Vc, Ms, Vs, N, False, 0.9, 0.999, 1e-8, k)
    assert torch.equal(opt.V[0], Vc) and torch.equal(opt.M[0] & 0x7F, Mc & 0x7F)
    assert torch.equal(opt.M_scale[0], Ms.view(-1)) and torch.equal(opt.V_scale[0], Vs.view(-1))


@pytest.mark.parametrize("moments", ["f32", "q8"])
def test_long_lists_and_splits_of_a_list_give_the_same_bits(moments):
    # 200 tensors: several launches; the same tensors one call each, and those in a list with one that has gaps between rows
    rng = np.random.default_rng(2)
    shapes = [(1, int(n)) for n in rng.integers(1, 3000, 200)]
    W0 = [torch.from_numpy(_rand(rng, *s)).float().cuda() for s in shapes]
    G = [torch.from_numpy(_rand(rng, *s)).bfloat16().cuda() for s in shapes]
    Wa, Wb = [w.clone() for w in W0], [w.clone() for w in W0]
    a = gb.GaLoreAdamW(Wa, moments=moments, weight_decay=0.1)
    singles = [gb.GaLoreAdamW([w], moments=moments, weight_decay=0.1) for w in Wb]
    for _ in range(2):
        a.step(Wa, G, 1e-2)
        for o, w, g in zip(singles, Wb, G):
            o.step([w], [g], 1e-2)
    Wc = [w.clone() for w in W0] + [torch.zeros(5, 9, device="cuda")[:, :7]]
    c = gb.GaLoreAdamW(Wc, moments=moments, weight_decay=0.1)
    for _ in range(2):
        c.step(Wc, G + [torch.ones(5, 7, device="cuda")], 1e-2)
    for i, o in enumerate(singles):
        assert torch.equal(Wa[i], Wb[i]) and torch.equal(a.M[i], o.M[0]) and torch.equal(a.V[i], o.V[0]), i
        assert torch.equal(Wa[i], Wc[i]) and torch.equal(a.M[i], c.M[i]) and torch.equal(a.V[i], c.V[i]), i


def test_both_state_formats_and_both_types_in_one_call():
    rng = np.random.default_rng(4)
    shapes = [(5, 300), (1, 77), (4, 256), (2, 1000)]
    W = [torch.from_numpy(_rand(rng, *s)).to(torch.bfloat16 if i % 2 else torch.float32).cuda() for i, s in enumerate(shapes)]
    G = [torch.from_numpy(_rand(rng, *s)).to(torch.float32 if i > 1 else torch.bfloat16).cuda() for i, s in enumerate(shapes)]
    mixed, apart = [w.clone() for w in W], [w.clone() for w in W]
    opts = [gb.GaLoreAdamW([w], moments="q8" if i in (0, 3) else "f32") for i, w in enumerate(W)]
    refs = [gb.GaLoreAdamW([w], moments="q8" if i in (0, 3) else "f32") for i, w in enumerate(W)]
    gb.galore_adamw(mixed, G, [o._states[0] for o in opts], 0.9, 0.999, 1e-8, 1e-2, 1)
    for o, w, g in zip(refs, apart, G):
        o.step([w], [g], 1e-2)
    for i in range(4):
        assert torch.equal(mixed[i], apart[i]) and torch.equal(opts[i].M[0], refs[i].M[0]) and torch.equal(opts[i].V[0], refs[i].V[0])


@pytest.mark.parametrize("moments", ["f32", "q8"])
def test_a_step_whose_gradients_were_not_finite_changes_nothing(moments):
    W = [torch.randn(3, 700, device="cuda"), torch.randn(50, device="cuda").bfloat16()]
    G = [torch.full_like(w, float("nan")) for w in W]
    opt = gb.GaLoreAdamW(W, moments=moments, weight_decay=0.1)
    opt.step(W, [torch.randn_like(w) for w in W], 1e-2)
    keep = [t.clone() for t in W + [opt.M_flat, opt.V_flat]]
    opt.step(W, G, 1e-2, _stats(0.0, finite=0.0))
    for x, y in zip(keep, W + [opt.M_flat, opt.V_flat]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_without_stats_non_finite_gradients_show(bad):
    for moments in ("f32", "q8"):
        w = torch.ones(1, 1000, device="cuda")
        g = torch.full((1, 1000), 0.5, device="cuda")
        g[0, 300] = bad                                                 # second block of 256
        opt = gb.GaLoreAdamW([w], moments=moments)
        opt.step([w], [g], 1e-2)
        assert torch.isnan(w[0, 300]) and torch.isfinite(w[0, :300]).all() and torch.isfinite(w[0, 301:]).all()
        if moments == "f32":
            assert not torch.isfinite(opt.M[0][0, 300]) and not torch.isfinite(opt.V[0][0, 300])
        else:
            assert not torch.isfinite(opt.M_scale[0][1]) and not torch.isfinite(opt.V_scale[0][1])
            assert torch.isfinite(opt.M_scale[0][[0, 2, 3]]).all()
        g[0, 300] = 0.5
        opt.step([w], [g], 1e-2)                                         # the next step: still visible, elsewhere unharmed
        assert torch.isnan(w[0, 300]) and torch.isfinite(w[0, :256]).all() and torch.isfinite(w[0, 512:]).all()


def test_zero_moments_and_gradients_leave_the_weight():
    # v = 0: n = 0 / (0 + eps)
    for moments in ("f32", "q8"):
        w = torch.randn(7, 333, device="cuda")
        want = w.clone()
        opt = gb.GaLoreAdamW([w], moments=moments)
        opt.step([w], [torch.zeros_like(w)], 1e-2)
        assert torch.equal(w, want) and not opt.M_flat.any() and not opt.V_flat.any()


def test_extreme_magnitudes():
    # gradients whose squares are subnormal or near the largest fp32 number
    rng = np.random.default_rng(8)
    for size in (1e-25, 1e-19, 1e-10, 1e10, 1e18):
        g = (rng.standard_normal((4, 500)) * size).astype(np.float32)
        w = rng.standard_normal((4, 500)).astype(np.float32)
        W = torch.from_numpy(w).cuda()
        opt = gb.GaLoreAdamW([W], beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
        opt.step([W], [torch.from_numpy(g).cuda()], LR)
        z = np.zeros_like(g, dtype=np.float64)
        (w1, m1, v1), (dw, dm, dv) = _bounds(w.astype(np.float64), g.astype(np.float64), z, z, 1, 1.0, WD)
        _within(opt.M[0], m1, dm)
        _within(opt.V[0], v1, dv + 4 * TINY)
        _within(W, w1, dw)


def test_parameters_of_any_rank():
    shapes = [(), (5,), (3, 4), (2, 3, 5), (2, 2, 2, 3)]
    W = [torch.randn(s, device="cuda") for s in shapes]
    W0 = [to64(w).reshape(1, -1) for w in W]
    G = [torch.randn(s, device="cuda") for s in shapes]
    opt = gb.GaLoreAdamW(W, beta1=B1, beta2=B2, eps=EPS)
    opt.step(W, G, LR)
    for w, w0, g in zip(W, W0, G):
        z = np.zeros_like(w0)
        (w1, _, _), (dw, _, _) = _bounds(w0, to64(g).reshape(1, -1), z, z, 1, 1.0, 0.0)
        _within(to64(w).reshape(1, -1), w1, dw)
    with pytest.raises(ValueError):
        gb.param_desc(torch.randn(8, device="cuda")[::2])
    with pytest.raises(ValueError):
        gb.param_desc(torch.randn(4, 6, 8, device="cuda").transpose(0, 1))
    with pytest.raises(ValueError):
        gb.param_desc(torch.randn(4, 6, device="cuda").t())
    with pytest.raises(ValueError):
        gb.param_desc(torch.zeros(4, 6, dtype=torch.float16, device="cuda"))
    w = torch.ones(3, 4, device="cuda")
    one = gb.GaLoreAdamW([w])
    with pytest.raises(gb.GaloreError) as e:                                  # a broadcast gradient has no rows of its own
        one.step([w], [torch.ones(1, 4, device="cuda").expand(3, 4)], LR)
    assert e.value.status == 2 and one.t == 0 and bool((w == 1).all())


@pytest.mark.parametrize("moments,gdt", [("q8", "bf16"), ("f32", "f32")])
def test_more_than_2_to_the_31_elements(moments, gdt):
    # offsets beyond 32 bits: the last rows, and rows on both sides of element 2^31, against the oracle
    rows, cols = (1 << 15) + 3, (1 << 16) + 5
    W = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    G = torch.zeros(rows, cols, dtype=TDT[gdt], device="cuda")
    at = [0, (1 << 31) // cols - 1, (1 << 31) // cols, rows - 1]
    gen = torch.Generator("cuda").manual_seed(1)
    for r in at:
        W[r] = torch.randn(cols, generator=gen, device="cuda").bfloat16()
        G[r] = torch.randn(cols, generator=gen, device="cuda").to(G.dtype)
    W0, opt = W[at].clone(), gb.GaLoreAdamW([W], moments=moments, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    norm = gb.GaLoreGradNorm(1)
    stats = norm.measure([G])
    opt.step([W], [G], LR, stats)
    torch.cuda.synchronize()
    total = float(G[at].double().square().sum().sqrt())
    assert abs(float(stats[0]) - total) <= 2.0 ** -23 * total and float(stats[1]) == 1.0
    z = np.zeros((1, cols))
    for j, r in enumerate(at):
        (w1, _, _), (dw, _, _) = _bounds(to64(W0[j:j + 1]), to64(G[r:r + 1]), z, z, 1, 1.0, WD)
        _within(to64(W[r:r + 1]), w1, dw, torch.bfloat16)
    rest = torch.ones(rows, dtype=torch.bool, device="cuda")
    rest[at] = False
    assert not W[rest].any()
    norm.scale([G], _stats(0.5))
    assert abs(float(norm.measure([G])[0]) - 0.5 * total) <= 2.0 ** -7 * total


@pytest.mark.parametrize("moments,rows,cols", [("f32", (1 << 16) + 1, (1 << 16) + 4), ("q8", (1 << 17) + 1, (1 << 16) + 4)])
def test_more_elements_than_one_launch_takes(moments, rows, cols):
    # 2^23 workgroups of 512 (8-bit moments: 1024) elements are one launch; rows on both sides of that, and the last one
    if torch.cuda.mem_get_info()[0] < 72 << 30:
        pytest.skip("needs 60 GB of device memory")
    split = (1 << 23) * (512 if moments == "f32" else 1024)
    assert rows * cols > split
    W = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    G = torch.zeros_like(W)
    at = [0, split // cols - 1, split // cols, split // cols + 1, rows - 1]
    gen = torch.Generator("cuda").manual_seed(2)
    for r in at:
        W[r] = torch.randn(cols, generator=gen, device="cuda").bfloat16()
        G[r] = torch.randn(cols, generator=gen, device="cuda").bfloat16()
    W0, opt = W[at].clone(), gb.GaLoreAdamW([W], moments=moments, beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    opt.step([W], [G], LR)
    torch.cuda.synchronize()
    z = np.zeros((1, cols))
    for j, r in enumerate(at):
        (w1, _, _), (dw, _, _) = _bounds(to64(W0[j:j + 1]), to64(G[r:r + 1]), z, z, 1, 1.0, WD)
        _within(to64(W[r:r + 1]), w1, dw, torch.bfloat16)
        W[r] = 0
    assert int(torch.count_nonzero(W)) == 0
    del W, G, opt
    torch.cuda.empty_cache()


@pytest.mark.parametrize("moments", ["f32", "q8"])
def test_captured_calls_replay(moments):
    # norm, scaling of one part, AdamW of the other, captured once and replayed between eager work; the graph keeps its k
    torch.manual_seed(0)
    W = [torch.randn(37, 515, device="cuda").bfloat16(), torch.randn(900, device="cuda")]
    G = [torch.empty_like(w) for w in W]
    Wr = [w.clone() for w in W]
    opt, ref = gb.GaLoreAdamW(W, moments=moments, weight_decay=0.1), gb.GaLoreAdamW(Wr, moments=moments, weight_decay=0.1)
    norm, norm_r = gb.GaLoreGradNorm(2, max_norm=0.5), gb.GaLoreGradNorm(2, max_norm=0.5)

    def pass_(o, n, weights, grads):
        stats = n.measure(grads)
        o.step(weights, grads, 1e-2, stats)
        o.t = 4
        n.scale(grads)

    opt.t = ref.t = 4
    side = torch.cuda.Stream()
    for g in G:
        g.copy_(torch.randn_like(g))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        pass_(opt, norm, W, G)
    for i in range(5):
        torch.manual_seed(100 + i)
        fresh = [torch.randn_like(g) for g in G]
        for g, x in zip(G, fresh):
            g.copy_(x)
        graph.replay()
        Gr = [x.clone() for x in fresh]
        pass_(ref, norm_r, Wr, Gr)
        torch.cuda.synchronize()
        assert torch.equal(norm.stats, norm_r.stats)
        for x, y in zip(W + G + [opt.M_flat, opt.V_flat], Wr + Gr + [ref.M_flat, ref.V_flat]):
            assert torch.equal(x, y), i


@pytest.mark.parametrize("moments", ["f32", "q8"])
def test_replays_count_their_steps_on_the_device(moments):
    # norm, tick and AdamW captured once: every replay is the next step with the current rate, and a gradient that is not
    # finite leaves a step out and does not count; against eager calls with host counts
    torch.manual_seed(1)
    W = [torch.randn(33, 260, device="cuda"), torch.randn(900, device="cuda").bfloat16()]
    G = [torch.zeros_like(w) for w in W]
    Wr = [w.clone() for w in W]
    opt = gb.GaLoreAdamW(W, moments=moments, weight_decay=0.1, capturable=True)
    ref = gb.GaLoreAdamW(Wr, moments=moments, weight_decay=0.1)
    norm, norm_r = gb.GaLoreGradNorm(2, max_norm=1.0), gb.GaLoreGradNorm(2, max_norm=1.0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        opt.step(W, G, stats=norm.measure(G))
    assert opt.count() == 0
    for i in range(7):
        torch.manual_seed(40 + i)
        for g in G:
            g.copy_(torch.randn_like(g))
        if i == 3:
            G[1][5] = float("nan")
        opt.set_lr(1e-2 / (i + 1))
        graph.replay()
        if i != 3:
            ref.step(Wr, G, 1e-2 / (i + 1), norm_r.measure(G))
        torch.cuda.synchronize()
        assert opt.count() == ref.t
        for x, y in zip(W + [opt.M_flat, opt.V_flat], Wr + [ref.M_flat, ref.V_flat]):
            assert torch.equal(x, y), i
    opt.step(W, G, 1e-3)                                                  # eager, behind the replays
    ref.step(Wr, G, 1e-3)
    assert opt.count() == ref.t == 7 and all(torch.equal(x, y) for x, y in zip(W, Wr))


@pytest.mark.parametrize("beta1,beta2", [(0.9, 0.999), (0.0, 0.95), (0.99, 0.99999)])
def test_bias_corrections_of_the_device_clock(beta1, beta2):
    clock = torch.zeros(24, dtype=torch.uint8, device="cuda")
    for t in (0, 1, 2, 9, 99, 4567, 10 ** 6, 1 << 40):
        clock[:8].view(torch.int64).fill_(t)
        gb.galore_adamw_tick(clock, beta1, beta2)
        assert int(clock[:8].view(torch.int64)) == t + 1
        got = clock[12:20].view(torch.float32).double().cpu().numpy()
        want = [1.0 / (1.0 - f32(b) ** (t + 1)) for b in (beta1, beta2)]
        # rounded once from 64 bits: half a step, and what 64 bits lose where 1 - b^t cancels (at most 2^17 times 2^-52)
        assert np.all(np.abs(got - want) <= (U + 2.0 ** -35) * np.asarray(want)), t
    clock.zero_()
    gb.galore_adamw_tick(clock, 0.9, 0.999, _stats(1.0, finite=0.0))
    assert not clock.any()


def test_calls_run_on_the_current_stream():
    w, g = torch.zeros(1 << 20, device="cuda"), torch.zeros(1 << 20, device="cuda")
    opt = gb.GaLoreAdamW([w], eps=0.0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(20):
            g.add_(0.05)                                                  # finished before the step reads it only if in order
        opt.step([w], [g], 1e-2)
    side.synchronize()
    # first step: n = 1 up to rounding (m c1 = g, sqrt(v c2) = g)
    assert float((w + 1e-2).abs().max()) <= 1e-2 * 16 * U


def test_two_calls_at_once_on_two_streams():
    # no state is shared between calls: two lists, two norms, two streams, no ordering between them
    torch.manual_seed(2)
    lists = [[torch.randn(300, 1000, device="cuda"), torch.randn(77, device="cuda")] for _ in range(2)]
    grads = [[torch.randn_like(w) for w in ws] for ws in lists]
    start = [[w.clone() for w in ws] for ws in lists]
    opts = [gb.GaLoreAdamW(ws, moments=m, weight_decay=0.1) for ws, m in zip(lists, ("f32", "q8"))]
    norms = [gb.GaLoreGradNorm(2, max_norm=1.0) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                opts[i].step(lists[i], grads[i], 1e-2, norms[i].measure(grads[i]))
    torch.cuda.synchronize()
    for i, m in enumerate(("f32", "q8")):
        ref, norm = gb.GaLoreAdamW(start[i], moments=m, weight_decay=0.1), gb.GaLoreGradNorm(2, max_norm=1.0)
        for _ in range(5):
            ref.step(start[i], grads[i], 1e-2, norm.measure(grads[i]))
        for a, b in zip(start[i], lists[i]):
            assert torch.equal(a, b)
        assert torch.equal(ref.M_flat, opts[i].M_flat) and torch.equal(ref.V_flat, opts[i].V_flat)


def test_training_descends_as_torch_does_it():
    # 20 steps on one quadratic, against the oracle's trajectory in fp64 (fp32 weights)
    rng = np.random.default_rng(1)
    target, w64 = rng.standard_normal((4, 129)), rng.standard_normal((4, 129)).astype(np.float32).astype(np.float64)
    W = torch.from_numpy(w64).float().cuda()
    opt = gb.GaLoreAdamW([W], beta1=B1, beta2=B2, eps=EPS, weight_decay=WD)
    m, v = np.zeros_like(w64), np.zeros_like(w64)
    for k in range(1, 21):
        opt.step([W], [(W - torch.from_numpy(target).float().cuda())], LR)
        w64, m, v, _ = ao.adamw(w64, w64 - target, m, v, B1, B2, EPS, LR, WD, k)
    # an error of a weight enters the next gradients; 20 steps of at most 30 roundings of numbers under 8 each
    assert np.abs(to64(W) - w64).max() <= 20 * 30 * 8 * U


@pytest.mark.parametrize("moments", ["f32", "q8"])
def test_hooks_step_the_other_parameters(moments):
    # a training loop with GaLore matrices and norm weights through PerLayerGaLore, against the same steps by hand
    from paper_2403_03507_amd.hooks import PerLayerGaLore

    class Block(torch.nn.Module):
        def __init__(self):
            super().__init__()
            self.scale = torch.nn.Parameter(torch.ones(64, device="cuda"))
            self.up = torch.nn.Linear(64, 192, bias=False, device="cuda")
            self.down = torch.nn.Linear(192, 64, bias=True, device="cuda")

        def forward(self, x):
            return x + self.down(torch.nn.functional.silu(self.up(x * self.scale)))

    def model():
        torch.manual_seed(5)
        return torch.nn.Sequential(Block(), Block())

    xs = [torch.randn(32, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(50 + s)) for s in range(3)]
    mats = lambda net: [[b.up.weight, b.down.weight] for b in net]
    rest = lambda net: [p for b in net for p in (b.scale, b.down.bias)]
    hooked = model()
    drv = PerLayerGaLore(mats(hooked), 8, 1e-2, update_gap=2, refresh_iters=3, others=rest(hooked), others_lr=3e-2,
                         others_options={"moments": moments, "weight_decay": [0.0, 0.1, 0.0, 0.1]})
    norm = gb.GaLoreGradNorm(4, max_norm=0.01)
    for i, x in enumerate(xs):
        hooked(x).pow(2).mean().backward()
        drv.finish(norm.measure([p.grad for p in rest(hooked)]) if i else None)
        assert all(p.grad is None for p in hooked.parameters())
    manual = model()
    flat, others = [p for l in mats(manual) for p in l], rest(manual)
    opt = gb.GaLore([p.data for p in flat], 8, update_gap=2, refresh_iters=3)
    adamw = gb.GaLoreAdamW(others, moments=moments, weight_decay=[0.0, 0.1, 0.0, 0.1])
    for i, x in enumerate(xs):
        manual(x).pow(2).mean().backward()
        for li in (1, 0):
            ps = flat[2 * li:2 * li + 2]
            opt.step([p.data for p in ps], [p.grad for p in ps], 1e-2, first=2 * li)
        adamw.step([p.data for p in others], [p.grad for p in others], 3e-2, norm.measure([p.grad for p in others]) if i else None)
        for p in manual.parameters():
            p.grad = None
    torch.cuda.synchronize()
    for a, b in zip(hooked.parameters(), manual.parameters()):
        assert torch.equal(a, b)
    hooked(xs[0]).pow(2).mean().backward()
    rest(hooked)[0].grad = None
    with pytest.raises(ValueError):
        drv.finish()
    drv.opt.join()
    drv.close()
    opt.close()
