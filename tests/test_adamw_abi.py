"""AdamW over tensor lists, gradient norm and scaling: refusals (on the host, before anything is launched; no GPU) and
the oracle's pins."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import adamw_oracle as ao
from oracle import q8_oracle as q8
from paper_2403_03507_amd import binding as gb

T = gb.galore_tensor
F32, BF16, U8 = gb.GALORE_F32, gb.GALORE_BF16, gb.GALORE_U8
NONE = T(None, 0, 0, 0, F32)
BASE = 1 << 20


class Call:
    """A valid call on made-up addresses (nothing is launched: every test spoils it)."""

    def __init__(self, n=2, rows=3, cols=100, dtype=F32, moments=F32, master=False):
        at = iter(range(BASE, BASE + (1 << 24), 1 << 14))
        t = lambda dt, r=rows, c=cols: T(next(at), r, c, c, dt)
        blocks = -(-rows * cols // 256)
        self.W = [t(dtype) for _ in range(n)]
        self.G = [t(dtype) for _ in range(n)]
        self.S = [gb.galore_adamw_state(t(moments), t(moments), t(F32, 1, blocks) if moments == U8 else NONE,
                                        t(F32, 1, blocks) if moments == U8 else NONE, t(F32) if master else NONE, 0.01) for _ in range(n)]
        self.scalars = dict(beta1=0.9, beta2=0.999, eps=1e-8, lr=1e-3, k=1)
        self.stats, self.count, self.clock = None, n, None

    def status(self, **kw):
        a = dict(self.scalars, **kw)
        n = len(self.W)
        arr = lambda items, typ: None if items is None else (typ * n)(*items)
        return gb.lib().galore_adamw(arr(self.W, T), arr(self.G, T), arr(self.S, gb.galore_adamw_state), self.count,
                                     a["beta1"], a["beta2"], a["eps"], a["lr"], a["k"], self.clock, self.stats, None)


def test_adamw_refuses_bad_scalars():
    for bad in (dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=float("nan")),
                dict(lr=float("inf")), dict(lr=float("nan")), dict(k=0), dict(k=-3)):
        assert Call().status(**bad) == 1, bad
    c = Call(); c.count = -1
    assert c.status() == 1
    c = Call(); c.S[1].weight_decay = -1.0
    assert c.status() == 1
    for bad in (float("nan"), float("inf")):
        c = Call(); c.S[1].weight_decay = bad
        assert c.status() == 1
    c = Call(); c.stats = BASE + 4
    assert c.status() == 5
    c = Call(); c.clock = BASE + 4
    assert c.status() == 5
    tick = gb.lib().galore_adamw_tick
    assert tick(None, 0.9, 0.999, None, None) == 1
    assert tick(BASE, 1.0, 0.999, None, None) == 1 and tick(BASE, 0.9, float("nan"), None, None) == 1
    assert tick(BASE + 4, 0.9, 0.999, None, None) == 5 and tick(BASE, 0.9, 0.999, BASE + 8, None) == 5


def test_adamw_refuses_missing_and_misshapen_tensors():
    L = gb.lib()
    assert L.galore_adamw(None, None, None, 1, 0.9, 0.999, 1e-8, 1e-3, 1, None, None, None) == 1
    assert L.galore_adamw(None, None, None, 0, 0.9, 0.999, 1e-8, 1e-3, 1, None, None, None) == 0      # an empty list is a step
    for field in ("W", "G"):
        c = Call(); getattr(c, field)[1].data = None
        assert c.status() == 1, field
        c = Call(); getattr(c, field)[1].rows = 0
        assert c.status() == 2, field
        c = Call(); getattr(c, field)[1].cols += 1; getattr(c, field)[1].ld += 1
        assert c.status() in (2, 7), field                                                          # G: shape, W: its state
        c = Call(); getattr(c, field)[1].ld -= 1
        assert c.status() == 2, field
        c = Call(); getattr(c, field)[1].dtype = U8
        assert c.status() == 3, field
        c = Call(); getattr(c, field)[1].data += 2
        assert c.status() == 5, field
        c = Call(dtype=BF16); getattr(c, field)[1].data += 1
        assert c.status() == 5, field
    for field in ("m", "v"):
        c = Call(); getattr(c.S[0], field).data = None
        assert c.status() == 1, field
        c = Call(); getattr(c.S[0], field).dtype = BF16
        assert c.status() == 3, field
        c = Call(); getattr(c.S[0], field).ld += 1
        assert c.status() == 7, field
        c = Call(); getattr(c.S[0], field).rows += 1
        assert c.status() == 7, field
        c = Call(); getattr(c.S[0], field).data += 8
        assert c.status() == 5, field


def test_adamw_refuses_malformed_8bit_and_master_states():
    c = Call(moments=U8); c.S[0].v.dtype = F32                              # one moment 8-bit, the other fp32
    assert c.status() == 3
    c = Call(); c.S[0].v.dtype = U8
    assert c.status() == 3
    for field in ("m_scale", "v_scale"):
        c = Call(moments=U8); getattr(c.S[1], field).data = None
        assert c.status() == 1
        c = Call(moments=U8); getattr(c.S[1], field).dtype = BF16
        assert c.status() == 3
        c = Call(moments=U8); getattr(c.S[1], field).cols = getattr(c.S[1], field).ld = 1       # 300 elements: two blocks
        assert c.status() == 7
        c = Call(moments=U8); getattr(c.S[1], field).data += 2
        assert c.status() == 5
    c = Call(dtype=BF16, master=True); c.S[0].master.dtype = BF16
    assert c.status() == 3
    c = Call(dtype=BF16, master=True); c.S[0].master.cols = c.S[0].master.ld = 99
    assert c.status() == 7
    c = Call(dtype=BF16, master=True); c.S[0].master.data += 4
    assert c.status() == 5
    c = Call(dtype=F32, master=True)                                         # an fp32 weight is its own master
    assert c.status() == 3


def test_adamw_refuses_the_same_tensor_twice():
    c = Call(); c.W[1].data = c.W[0].data
    assert c.status() == 1 and b"same address" in gb.lib().galore_last_error(None)
    c = Call(); c.S[1].m.data = c.S[0].v.data
    assert c.status() == 1
    c = Call(); c.S[0].v.data = c.S[0].m.data
    assert c.status() == 1
    c = Call(moments=U8); c.S[0].v_scale.data = c.S[0].m_scale.data
    assert c.status() == 1
    c = Call(dtype=BF16, master=True); c.S[0].master.data = c.S[1].master.data
    assert c.status() == 1


def test_adamw_refuses_a_gradient_that_it_would_overwrite():
    c = Call(); c.G[0].data = c.W[1].data
    assert c.status() == 1
    c = Call(); c.G[1].data = c.S[0].m.data
    assert c.status() == 1


def test_gradient_calls_refuse_bad_arguments():
    L = gb.lib()
    need = gb.galore_grad_norm_workspace_bytes(2)
    assert need % 256 == 0 and need >= 8 * 2
    assert L.galore_grad_norm_workspace_bytes(-1, ctypes.byref(ctypes.c_size_t())) == 1
    assert L.galore_grad_norm_workspace_bytes(1, None) == 1

    def norm(G=None, count=2, scale=1.0, max_norm=1.0, stats=BASE, ws=BASE, nbytes=need):
        G = G if G is not None else [T(BASE, 3, 100, 100, F32), T(BASE + 4096, 3, 100, 100, BF16)]
        return L.galore_grad_norm((T * len(G))(*G), count, scale, max_norm, stats, ws, nbytes, None)
    assert norm(count=-1) == 1
    assert norm(scale=float("nan")) == 1 and norm(scale=float("inf")) == 1
    assert norm(max_norm=0.0) == 1 and norm(max_norm=-1.0) == 1 and norm(max_norm=float("nan")) == 1
    assert norm(stats=None) == 1 and norm(stats=BASE + 8) == 5
    assert norm(ws=None) == 6 and norm(ws=BASE + 16) == 5 and norm(nbytes=need // 2) == 6
    bad = lambda **kw: [T(*[kw.get(f, d) for f, d in (("data", BASE), ("rows", 3), ("cols", 100), ("ld", 100), ("dtype", F32))])]
    assert norm(bad(data=None), 1) == 1 and norm(bad(rows=0), 1) == 2 and norm(bad(ld=99), 1) == 2
    assert norm(bad(dtype=U8), 1) == 3 and norm(bad(data=BASE + 2), 1) == 5
    assert L.galore_grad_norm(None, 1, 1.0, 1.0, BASE, BASE, need, None) == 1

    def scale(G, count=None, stats=BASE):
        return L.galore_scale_grads((T * len(G))(*G), len(G) if count is None else count, stats, None)
    assert scale(bad(), stats=None) == 1 and scale(bad(), stats=BASE + 4) == 5 and scale(bad(), count=-1) == 1
    assert scale(bad(dtype=U8)) == 3 and scale(bad(data=BASE + 1)) == 5
    assert scale(bad() * 2) == 1                                              # twice in place
    assert L.galore_scale_grads(None, 0, BASE, None) == 0


def test_python_face_refuses_what_the_library_cannot_see():
    w = torch.zeros(4, 4)
    with pytest.raises(ValueError):
        gb.param_desc(w)                                                      # host memory
    with pytest.raises(ValueError):
        gb.GaLoreAdamW([w], device="cpu")
    with pytest.raises(ValueError):
        gb.GaLoreAdamW([], moments="q4", device="cpu")
    with pytest.raises(ValueError):
        gb.GaLoreAdamW([], weight_decay=[0.1], device="cpu")
    with pytest.raises(ValueError):
        gb._stats_ptr(torch.zeros(4))
    with pytest.raises(ValueError):
        gb._clock_ptr(torch.zeros(24, dtype=torch.uint8))
    with pytest.raises(ValueError):
        gb.galore_adamw((T * 1)(), (T * 2)(), [], 0.9, 0.999, 1e-8, 1e-3, 1)


# ---- the oracle ------------------------------------------------------------------------------------

def test_oracle_adamw_by_hand():
    # b1 = 1/2, b2 = 3/4, k = 1 from zero: m = g/2, v = g^2/4; corrected g and g^2; n = g / (|g| + eps)
    w, m, v, n = ao.adamw(np.array([2.0, -1.0]), np.array([3.0, -4.0]), np.zeros(2), np.zeros(2), 0.5, 0.75, 1.0, 0.5, 0.25, 1)
    assert np.allclose(m, [1.5, -2.0], rtol=0, atol=0) and np.allclose(v, [2.25, 4.0], rtol=0, atol=0)
    assert np.allclose(n, [0.75, -0.8], rtol=1e-15)
    assert np.allclose(w, [2.0 * 0.875 - 0.375, -0.875 + 0.4], rtol=1e-15)
    # k = 2: m = 1.5/2 + g/2, corrected by 1 - 1/4; v = 3/4 * 2.25 + g^2/4, corrected by 1 - 9/16
    w, m, v, n = ao.adamw(np.array([0.0]), np.array([1.0]), np.array([1.5]), np.array([2.25]), 0.5, 0.75, 0.0, 1.0, 0.0, 2)
    assert m[0] == 1.25 and v[0] == 1.9375
    assert np.allclose(n, (1.25 / 0.75) / np.sqrt(1.9375 / 0.4375), rtol=1e-15) and w[0] == -n[0]


def test_oracle_adamw_is_the_gradient_step_of_the_low_rank_rule_at_full_rank():
    # with beta1 = beta2 = 0 the update is the sign of the gradient
    g = np.array([3.0, -2.0, 0.5])
    w, _, _, n = ao.adamw(np.zeros(3), g, np.ones(3), np.ones(3), 0.0, 0.0, 0.0, 0.1, 0.0, 7)
    assert np.allclose(n, np.sign(g), rtol=1e-15) and np.allclose(w, -0.1 * np.sign(g), rtol=1e-15)


def test_oracle_grad_stats_by_hand():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    assert ao.grad_stats(g, 1.0, np.inf) == (5.0, 1.0, 1.0)
    norm, factor, finite = ao.grad_stats(g, 0.5, 1.0)
    assert norm == 2.5 and finite == 1.0 and abs(factor - 0.5 * 1.0 / 2.500001) < 1e-15
    assert ao.grad_stats([np.array([1.0, np.inf])], 1.0, 1.0)[1:] == (0.0, 0.0)
    assert ao.grad_stats([], 1.0, 1.0) == (0.0, 1.0, 1.0)


def test_first_moment_codes_are_e4m3_numbers():
    # what the kernels' conversions rely on: code c stands for 2^-8 times the OCP e4m3 number with the bits of c, and
    # rounding to the nearest e4m3 number is the format's rounding (checked with torch's own type)
    c = torch.arange(0, 121, dtype=torch.uint8)
    table = torch.from_numpy(q8.decode_table(False))
    assert torch.equal(c.view(torch.float8_e4m3fn).double() * 2.0 ** -8, table[:121])
    y = torch.cat([torch.rand(200000, generator=torch.Generator().manual_seed(1)) ** 4,
                   torch.from_numpy(q8.midpoints(False)).float(), torch.tensor([0.0, 1.0, 2.0 ** -18, 2.0 ** -17])]).clamp(max=1.0)
    want = q8.encode(y.numpy(), np.float32(1.0), False)
    assert np.array_equal((y * 256).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), want)
