"""The layer operators on every kind of product kernel, at sizes that take it.

A product runs as tiles whose contraction 1, 2, 4 or 8 blocks share, or on pairs of SMs with 128 or 256 accumulator columns, in one go or split
and joined; each for plain and gated forward products, for dx and for weight gradients, with float32 or rounded results.  `KINDS` has a size for
each of those that the sizes of test_gpu_layers.py leave out.  Next to the elementwise bounds of the definition, the norm of the error is held, which
shows what a bound that grows with the contraction lets pass.
"""
import pytest
import torch

import tests.layer_reference as R
from paper_2012_05396_b200 import layers as L
from tests.test_gpu_layers import DT, check, gen, normal, weights
from tests.test_layer_error_norms import F32_NORM

pytestmark = pytest.mark.gpu

# (operator, type, gradient type, rows, in, out)
KINDS = [("gated_backward", "bf16", "bf16", 1164, 72, 4136), ("gated_backward", "bf16", "bf16", 1295, 4792, 8), ("gated_backward", "bf16", "bf16", 5415, 72, 1265),
         ("gated_backward", "bf16", "bf16", 5987, 8, 40), ("gated_backward", "bf16", "f32", 19, 8, 112), ("gated_backward", "bf16", "f32", 19, 8, 3328),
         ("gated_backward", "bf16", "f32", 2345, 8, 8), ("gated_backward", "bf16", "f32", 2607, 1560, 144), ("gated_backward", "bf16", "f32", 3097, 136, 3408),
         ("gated_backward", "f32", "bf16", 17, 8, 104), ("gated_backward", "f32", "bf16", 2309, 8, 8), ("gated_backward", "f32", "bf16", 2856, 1592, 144),
         ("gated_backward", "f32", "f32", 17, 4904, 8), ("gated_backward", "f32", "f32", 18, 2440, 8), ("gated_backward", "f32", "f32", 18, 72, 5288),
         ("gated_backward", "f32", "f32", 3385, 8, 112), ("gated_backward", "f32", "f32", 534, 3814, 8), ("gated_backward", "bf16", "bf16", 20000, 1000, 1000),
         ("gated_forward", "bf16", "", 144, 5656, 696), ("gated_forward", "bf16", "", 57, 5384, 8), ("gated_forward", "bf16", "", 500, 16384, 1024),
         ("gated_forward", "f32", "", 17, 2832, 528), ("gated_forward", "f32", "", 26, 192, 5288), ("gated_forward", "f32", "", 393, 5088, 16),
         ("linear_backward", "bf16", "bf16", 135, 2960, 3160), ("linear_backward", "bf16", "bf16", 17, 1928, 3352), ("linear_backward", "bf16", "bf16", 3635, 2776, 136),
         ("linear_backward", "bf16", "bf16", 5601, 8, 64), ("linear_backward", "bf16", "f32", 1104, 5832, 8), ("linear_backward", "bf16", "f32", 17, 672, 3368),
         ("linear_backward", "bf16", "f32", 2430, 8, 8), ("linear_backward", "bf16", "f32", 2465, 1544, 264), ("linear_backward", "bf16", "f32", 49, 8, 5936),
         ("linear_backward", "f32", "bf16", 17, 4016, 568), ("linear_backward", "f32", "bf16", 2232, 1648, 328), ("linear_backward", "f32", "bf16", 2311, 8, 8),
         ("linear_backward", "f32", "bf16", 573, 3816, 8), ("linear_backward", "f32", "f32", 17, 4080, 552), ("linear_backward", "f32", "f32", 19, 8, 1040),
         ("linear_backward", "f32", "f32", 5346, 2408, 32), ("linear_backward", "bf16", "bf16", 20000, 1000, 1000),
         ("linear_forward", "bf16", "", 1133, 8, 5688), ("linear_forward", "bf16", "", 2470, 5432, 72), ("linear_forward", "bf16", "", 61, 5456, 8),
         ("linear_forward", "bf16", "", 256, 16384, 4096), ("linear_forward", "f32", "", 1458, 25, 1750), ("linear_forward", "f32", "", 26, 2728, 744),
         ("linear_forward", "f32", "", 26, 386, 5734), ("linear_forward", "f32", "", 3073, 1224, 136), ("linear_forward", "f32", "", 100, 2048, 1000)]

# float32 forward products whose work would take the few-row kernel longer: both sides of that rule
KINDS += [("gated_forward", "f32", "", *s) for s in ((17, 9, 3186), (2966, 11, 18), (3559, 94, 9), (309, 775, 25), (148, 8, 2608), (194, 4180, 24), (130, 8, 4840),
                                                      (3255, 1112, 72), (100, 2048, 1000), (2000, 64, 64), (24, 704, 1920))]
KINDS += [("linear_forward", "f32", "", *s) for s in ((34, 9, 5831), (3866, 9, 34), (1232, 314, 9), (1247, 908, 8), (129, 8, 5064), (298, 3358, 28), (387, 8, 5088),
                                                       (57, 3712, 2408), (8000, 8, 1000), (1000, 64, 1000), (2000, 64, 64), (7000, 1000, 8))]

# two to sixteen bfloat16 rows, forward and backward, both sides of where the tensor cores take them
KINDS += [(op, "bf16", "", *s) for op in ("linear_forward", "gated_forward")
          for s in ((8, 8192, 520), (2, 20000, 8), (16, 16384, 64), (9, 4112, 1000), (5, 4752, 10304), (16, 3104, 4096), (8, 6152, 129), (3, 6136, 129))]
KINDS += [(op, "bf16", g, *s) for op in ("linear_backward", "gated_backward") for g in ("f32", "bf16")
          for s in ((16, 2304, 2304), (9, 2056, 8200), (8, 2304, 2304), (12, 2308, 2304), (16, 8192, 6200), (13, 64, 16384))]


@pytest.mark.parametrize("act", [0, 2])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_every_kind_of_product(kind, act):
    op, dtype, grad, rows, d, f = kind
    t, g = DT[dtype], gen(rows + act)
    x, w = normal(g, rows, d, dtype=t), weights(g, f, d, t)
    w2 = weights(g, f, d, t) if op.startswith("gated") else None
    if op == "linear_forward":
        b, r = normal(g, f, dtype=torch.float32), normal(g, rows, f, dtype=t)
        y, z = L.ssd_linear_forward(x, w, bias=b, residual=r, act=act, keep=True)
        ref = R.linear_forward(x, w, b, r, act)
        got = {"y": y, "z": z}
    elif op == "gated_forward":
        bg, bu = normal(g, f, dtype=torch.float32), normal(g, f, dtype=torch.float32)
        ref = R.gated_forward(x, w, w2, bg, bu, act)
        got = dict(zip(("h", "gate", "up"), L.ssd_gated_forward(x, w, w2, bg, bu, act=act, keep=True)))
    else:
        dy, z, u = (normal(g, rows, f, dtype=t) for _ in range(3))
        if op == "linear_backward":
            ref = R.linear_backward(dy, x, w, z, act, DT[grad])
            got = dict(zip(("dx", "dw0", "db0"), L.ssd_linear_backward(dy, x, w, z if act else None, act=act, grad_dtype=DT[grad])))
        else:
            ref = R.gated_backward(dy, x, w, w2, z, u, act, DT[grad])
            got = dict(zip(("dx", "dw0", "dw1", "db0", "db1"), L.ssd_gated_backward(dy, x, w, w2, z, u, act=act, grad_dtype=DT[grad])))
    for k, v in got.items():
        check(v, ref[k], k)


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


# float32 results of 2048 and more products each: few rows, tiles by clusters of 8, pairs split and not
@pytest.mark.parametrize("size", [(2, 4096, 1000), (16, 2304, 1000), (100, 2048, 1000), (300, 4096, 700), (2048, 2304, 2048), (256, 5632, 264)], ids=str)
def test_norm_of_the_error_of_float32_products(size):
    rows, d, f = size
    g = gen(rows)
    x, w, w2 = normal(g, rows, d, dtype=torch.float32), weights(g, f, d, torch.float32), weights(g, f, d, torch.float32)
    y, _ = L.ssd_linear_forward(x, w)
    _, gate, up = L.ssd_gated_forward(x, w, w2, keep=True)
    errors = [off(y, x.double() @ w.double().t()), off(gate, x.double() @ w.double().t()), off(up, x.double() @ w2.double().t())]
    assert max(errors) <= F32_NORM, errors


# (rows, in, out): 2048 and more products in dx (linear: out, gated: 2 out), in the weight gradients (rows), or in both
@pytest.mark.parametrize("size", [(12, 300, 4096), (256, 512, 2300), (2304, 200, 2400), (4099, 520, 264), (2304, 2304, 2304)], ids=str)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_norm_of_the_error_of_float32_gradients(size, dtype):
    rows, d, f = size
    t, g = DT[dtype], gen(rows)
    x, w, w2 = normal(g, rows, d, dtype=t), weights(g, f, d, t), weights(g, f, d, t)
    dy, a, u = (normal(g, rows, f, dtype=t) for _ in range(3))
    xd, wd, w2d, dyd, ad, ud = (v.double() for v in (x, w, w2, dy, a, u))
    errors = {}
    dx, dw, db = L.ssd_linear_backward(dy, x, w)
    if dtype == "f32":
        errors["linear dx"] = off(dx, dyd @ wd)
    errors["linear dw"], errors["linear db"] = off(dw, dyd.t() @ xd), off(db, dyd.sum(0))
    dx, dwg, dwu, dbg, dbu = L.ssd_gated_backward(dy, x, w, w2, a, u, act=0)
    dg, du = dyd * ud, dyd * ad
    if dtype == "f32":
        errors["gated dx"] = off(dx, dg @ wd + du @ w2d)
    errors.update({"dw gate": off(dwg, dg.t() @ xd), "dw up": off(dwu, du.t() @ xd), "db gate": off(dbg, dg.sum(0)), "db up": off(dbu, du.sum(0))})
    assert max(errors.values()) <= F32_NORM, errors


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("size", [(300, 520, 520), (1458, 25, 1750), (2048, 512, 2048), (100, 2048, 1000)], ids=str)
def test_special_values_of_float32_operands_in_parts(size, gated):
    """A NaN or infinity reaches the outputs that depend on it and no others, also through operands in three parts; the largest numbers pass."""
    rows, d, f = size
    g = gen(rows)
    x, w, w2 = normal(g, rows, d, dtype=torch.float32), weights(g, f, d, torch.float32), weights(g, f, d, torch.float32)

    def call(x, w):
        return L.ssd_gated_forward(x, w, w2, keep=True)[1] if gated else L.ssd_linear_forward(x, w)[0]

    clean = call(x, w)
    for bad in (float("nan"), float("inf"), float("-inf")):
        x2, w2_ = x.clone(), w.clone()
        x2[rows // 2, 3] = bad
        w2_[5, 7] = bad
        w2_[f - 1, d - 1] = bad
        y = call(x2, w2_)
        hit = torch.zeros(rows, f, dtype=torch.bool, device="cuda")
        hit[rows // 2] = True
        hit[:, 5] = True
        hit[:, f - 1] = True
        assert not bool(torch.isfinite(y[hit]).any()) and torch.equal(y[~hit], clean[~hit])
    # one product each, of numbers whose first part would round up to infinity, and of the smallest normal ones
    for v in (3.4e38, -3.4e38, 3.3961775e38, 1.2e-38, -1.2e-38):
        x3, w3 = torch.zeros_like(x), torch.zeros_like(w)
        x3[:, d // 2] = v
        w3[:, d // 2] = 1.0
        y = call(x3, w3)
        assert torch.allclose(y.double(), torch.full_like(y, float(torch.tensor(v)), dtype=torch.float64), rtol=2.0 ** -22, atol=2.0 ** -134)
        y = call(w3.new_zeros(rows, d).index_fill_(1, torch.tensor([d // 2], device="cuda"), 1.0), torch.zeros_like(w).index_fill_(1, torch.tensor([d // 2], device="cuda"), v))
        assert torch.allclose(y.double(), torch.full_like(y, float(torch.tensor(v)), dtype=torch.float64), rtol=2.0 ** -22, atol=2.0 ** -134)
    # overflow of the sum
    y = call(torch.full_like(x, 1e38), torch.ones_like(w))
    assert not bool(torch.isfinite(y).any())
    # a gradient's operands: infinities stay in their column of dx and row of dw
    dy = normal(g, rows, f, dtype=torch.float32)
    base = L.ssd_linear_backward(dy, x, w)
    dy2 = dy.clone()
    dy2[rows - 1, 2] = float("inf")
    dx, dw, db = L.ssd_linear_backward(dy2, x, w)
    assert not bool(torch.isfinite(dx[rows - 1]).any()) and torch.equal(dx[:rows - 1], base[0][:rows - 1])
    keep = torch.arange(f, device="cuda") != 2
    assert not bool(torch.isfinite(dw[2]).any()) and torch.equal(dw[keep], base[1][keep])
    assert not bool(torch.isfinite(db[2])) and torch.equal(db[keep], base[2][keep])
