"""Global gradient norm, clip factor and scaling on the GPU against the fp64 oracle.

The norm is formed in 64 bits and stored in 32: off by half a step of fp32 (2^-24) and the 64-bit sum's own error, which
is beyond that; the factor likewise.  Scaled entries are rounded once: 2^-24 of the product for fp32, and for bf16 that
and half a step of bf16 (2^-8)."""
import numpy as np
import pytest
import torch

from helpers import TDT, f32, to64
from oracle import adamw_oracle as ao
from paper_2403_03507_amd import binding as gb

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -24 * (1 + 2.0 ** -10)
SIZES = [(1, 1), (1, 2), (1, 7), (3, 1), (1, 255), (5, 63), (33, 1023), (1, 4096), (1, 4097), (700, 9), (9, 700), (3, 50000)]


def _grads(rng, sizes, dtypes, pads=(0,), offsets=(0,)):
    out = []
    for i, (m, n) in enumerate(sizes):
        dt, pad, off = TDT[dtypes[i % len(dtypes)]], pads[i % len(pads)], offsets[i % len(offsets)]
        buf = torch.full((off + m * (n + pad) + 3,), float("nan"), dtype=dt, device="cuda")
        view = buf[off:off + m * (n + pad)].view(m, n + pad)[:, :n]
        view.copy_(torch.from_numpy(rng.standard_normal((m, n)) * np.exp(rng.uniform(-3, 3))))
        out.append(view)
    return out


def _check(stats, grads, scale, max_norm):
    norm, factor, finite = ao.grad_stats([to64(g) for g in grads], scale, max_norm)
    got = [float(x) for x in stats]
    assert abs(got[0] - norm) <= HALF * norm and abs(got[1] - factor) <= HALF * abs(factor) and got[2] == finite and got[3] == 0.0, (got, norm, factor)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_of_one_gradient(size, dtype):
    rng = np.random.default_rng(size[0] * 7 + size[1])
    for pad, off in ((0, 0), (0, 1), (5, 2), (1, 0)):
        G = _grads(rng, [size], [dtype], [pad], [off])
        norm = gb.GaLoreGradNorm(1, max_norm=1.5)
        _check(norm.measure(G), G, 1.0, 1.5)


@pytest.mark.parametrize("scale,max_norm", [(1.0, float("inf")), (1.0, 0.25), (0.125, 3.0), (-2.0, 1.0), (1.0, 1e30), (0.0, 1.0)])
def test_norm_of_lists(scale, max_norm):
    rng = np.random.default_rng(4)
    sizes = SIZES * 25                                                      # 300 tensors: three launches
    G = _grads(rng, sizes, ["f32", "bf16", "bf16"], [0, 3, 0, 7], [0, 1, 3])
    norm = gb.GaLoreGradNorm(len(G), max_norm=max_norm)
    first = norm.measure(G, scale).clone()
    _check(first, G, scale, f32(max_norm))
    assert torch.equal(first, norm.measure(G, scale))                       # the order of the sum is fixed


def test_norm_of_more_than_the_cache_holds():
    # 600 MiB of bf16 gradients: loads past the caches, and spans of 154 thousand elements
    rng = np.random.default_rng(1)
    one = torch.from_numpy(rng.standard_normal(1 << 20)).bfloat16().cuda()
    G = [one.repeat(150), one.repeat(150)[1:]]
    total = 300 * float(one.double().square().sum()) - float(one[0]) ** 2
    stats = gb.GaLoreGradNorm(2, max_norm=1.0).measure(G)
    assert abs(float(stats[0]) - total ** 0.5) <= HALF * total ** 0.5


def test_scaling_of_more_than_one_launch_takes():
    # 2^23 workgroups of 2048 bf16 elements are one launch
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 40 GB of device memory")
    n = (1 << 34) + 70000
    G = torch.zeros(n // 10000, 10000, dtype=torch.bfloat16, device="cuda")
    rows = [0, (1 << 34) // 10000, G.shape[0] - 1]
    for r in rows:
        G[r] = r % 7 + 1
    norm = gb.GaLoreGradNorm(1, max_norm=1.0)
    total = 100.0 * sum((r % 7 + 1) ** 2 for r in rows) ** 0.5
    stats = norm.measure([G])
    assert abs(float(stats[0]) - total) <= HALF * total
    norm.scale([G], torch.tensor([1.0, 0.5, 1.0, 0.0], device="cuda"))
    for r in rows:
        assert bool((G[r] == (r % 7 + 1) / 2).all())
        G[r] = 0
    assert int(torch.count_nonzero(G)) == 0
    del G
    torch.cuda.empty_cache()


def test_more_gradients_than_the_workspace_is_for():
    norm = gb.GaLoreGradNorm(2)
    G = [torch.ones(4, device="cuda") for _ in range(200)]
    with pytest.raises(gb.GaloreError) as e:
        norm.measure(G)
    assert e.value.status == 6
    norm.stats.copy_(torch.tensor([1.0, 0.5, 1.0, 0.0]))
    with pytest.raises(gb.GaloreError) as e:
        norm.scale([G[0], G[0]])                                                # the same tensor twice
    assert e.value.status == 1 and bool((G[0] == 1).all())


def test_norm_of_nothing():
    norm = gb.GaLoreGradNorm(0, max_norm=2.0)
    assert norm.measure([]).tolist() == [0.0, 1.0, 1.0, 0.0]


@pytest.mark.parametrize("value", [3e38, 1e-38, 1e-30, 1e25])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_entries_whose_squares_leave_fp32(value, dtype):
    G = [torch.full((3, 1001), value, dtype=TDT[dtype], device="cuda")]
    norm = gb.GaLoreGradNorm(1, max_norm=1.0)
    stats = [float(x) for x in norm.measure(G)]
    want, factor, _ = ao.grad_stats([to64(G[0])], 1.0, 1.0)
    assert stats[2] == 1.0                                                   # every entry is finite
    if want < 3.4e38:
        assert abs(stats[0] - want) <= HALF * want + 2.0 ** -149
    else:
        assert stats[0] == float("inf")                                       # the norm itself is beyond fp32
    assert abs(stats[1] - factor) <= HALF * factor + 2.0 ** -149


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", [(0, 0), (1, 12345), (2, 6)])
def test_one_entry_that_is_not_finite(bad, where):
    G = [torch.ones(1, 300, device="cuda"), torch.ones(1, 20000, device="cuda", dtype=torch.bfloat16), torch.ones(1, 7, device="cuda")]
    G[where[0]][0, where[1]] = bad
    norm = gb.GaLoreGradNorm(3, max_norm=1.0)
    stats = norm.clip(G)
    assert stats[1] == 0.0 and stats[2] == 0.0
    assert all(not g.any() for g in G)                                        # zeros, not 0 * inf


@pytest.mark.parametrize("factor", [0.3, 1.0, 2.0, -1.0, 0.0])
def test_scaling_of_lists(factor):
    rng = np.random.default_rng(9)
    G = _grads(rng, SIZES * 12, ["bf16", "f32", "f32"], [0, 2, 0, 9], [0, 3, 1])
    before = [to64(g) for g in G]
    norm = gb.GaLoreGradNorm(len(G))
    norm.scale(G, torch.tensor([1.0, factor, 1.0, 0.0], device="cuda"))
    for g, b in zip(G, before):
        want, got = f32(factor) * b, to64(g)
        # fp32 product, then the stored type: a bf16 number's half step is relative to the rounded product
        bound = HALF * np.abs(want) + (2.0 ** -8 * np.abs(want) * (1 + HALF) if g.dtype == torch.bfloat16 else 0.0)
        assert np.all(np.abs(got - want) <= bound)
        base = g._base if g._base is not None else g
        inside = torch.zeros(base.numel(), dtype=torch.bool, device="cuda")
        inside.as_strided(g.shape, g.stride(), g.storage_offset())[:] = True
        assert torch.isnan(base.view(-1)[~inside]).all()                        # nothing around it


def test_clipped_galore_step_equals_a_step_on_clipped_gradients():
    # the operators together with the low-rank step: one norm over GaLore matrices and the others
    from paper_2403_03507_amd import workloads as wl
    shapes = [(128, 344), (344, 128)]
    W = [wl.make_weight(m, n, i, "bf16").cuda() for i, (m, n) in enumerate(shapes)]
    vec = torch.ones(128, device="cuda")
    G = [wl.GradientSource(m, n, 9 + i, "lowrank", dtype="bf16").grad(0).cuda() for i, (m, n) in enumerate(shapes)]
    gvec = torch.randn(128, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    Wr, vr = [w.clone() for w in W], vec.clone()

    def optimizers(weights, v):
        gal = gb.GaLore(weights, 16, auto_refresh=False)
        for i, (m, n) in enumerate(shapes):
            gal.proj[i].copy_(wl.random_orthonormal(min(m, n), 16, 60 + i).bfloat16())
        return gal, gb.GaLoreAdamW([v], weight_decay=0.0)

    gal, adamw = optimizers(W, vec)
    norm = gb.GaLoreGradNorm(3, max_norm=0.5)
    grads = [g.clone() for g in G]
    stats = norm.measure(grads + [gvec])
    norm.scale(grads)
    gal.step(W, grads, 1e-2)
    adamw.step([vec], [gvec], 1e-2, stats)
    torch.cuda.synchronize()
    total, factor, _ = ao.grad_stats([to64(g) for g in G] + [to64(gvec)], 1.0, 0.5)
    assert factor < 1.0 and abs(float(stats[0]) - total) <= HALF * total

    gal_r, adamw_r = optimizers(Wr, vr)
    gal_r.step(Wr, [(g.float() * stats[1]).bfloat16() for g in G], 1e-2)
    adamw_r.step([vr], [gvec * stats[1]], 1e-2)
    torch.cuda.synchronize()
    for a, b in zip(W + [vec], Wr + [vr]):
        assert torch.equal(a, b)
    gal.close()
    gal_r.close()
