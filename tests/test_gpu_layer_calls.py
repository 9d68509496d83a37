"""Calls of the layer operators at the ends of what their contract allows: pitches, workspaces, row counts, kernels taken."""
import ctypes as C

import pytest
import torch

import tests.layer_reference as R
from paper_2012_05396_b200 import binding as B
from paper_2012_05396_b200 import layers as L
from tests.test_gpu_layers import DT, check, gen, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_row_over_its_residual_whatever_the_pitches(dtype):
    """With one row a pitch means nothing, so the residual may be the result whatever pitch each is given with."""
    g, t = gen(1), DT[dtype]
    x, w, r = normal(g, 1, 72, dtype=t), normal(g, 40, 72, dtype=t, std=0.1), normal(g, 1, 40, dtype=t)
    ref = R.linear_forward(x, w, None, r.clone(), 2)
    code = B.SSD_F32 if dtype == "f32" else B.SSD_BF16
    a = L.ssd_linear_fwd(1, 72, 40, code, L.SSD_ACT_GELU, x.data_ptr(), 0, w.data_ptr(), 72, None, r.data_ptr(), 40, r.data_ptr(), 1000)
    assert L.lib().ssd_linear_forward(C.byref(a), None, 0, torch.cuda.current_stream().cuda_stream) == B.SSD_OK
    check(r, ref["y"], "y over its residual")
