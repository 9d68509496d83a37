"""Calls of the layer operators at the ends of what their contract allows: pitches, workspaces, row counts, kernels taken."""
import ctypes as C
import os
import subprocess
import sys

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


# Calls that take every kind of room from a workspace, (op, rows, in, out, dtype): sums of a contraction split over pairs, and over pairs for weight
# gradients; operands in parts; rows that are copied; column sums; strips of dx of a few rows.
ROOM = [("linear_forward", 256, 25088, 4096, "bf16"), ("linear_forward", 300, 4001, 600, "bf16"), ("linear_forward", 260, 2048, 1000, "f32"),
        ("gated_forward", 300, 2100, 500, "bf16"), ("gated_forward", 256, 1024, 512, "f32"), ("linear_backward", 256, 4096, 1000, "f32"),
        ("linear_backward", 2000, 600, 700, "bf16"), ("gated_backward", 300, 520, 700, "f32"), ("gated_backward", 1100, 264, 333, "bf16"),
        ("linear_backward", 7, 500, 900, "f32")]


@pytest.mark.parametrize("at", [0, 16, 48, 112])
@pytest.mark.parametrize("case", ROOM, ids=str)
def test_workspaces_on_any_16_bytes(case, at):
    """Exactly the bytes that were asked for, on an odd multiple of 16: the same bits as anywhere else, and nothing written beside them."""
    op, rows, d, f, dtype = case
    g, t = gen(2), DT[dtype]
    code = B.SSD_F32 if dtype == "f32" else B.SSD_BF16
    x, w, w2 = normal(g, rows, d, dtype=t), normal(g, f, d, dtype=t, std=d ** -0.5), normal(g, f, d, dtype=t, std=d ** -0.5)
    dy, z, u = (normal(g, rows, f, dtype=t) for _ in range(3))

    def empty(*shape, dt=t):
        return torch.empty(*shape, device="cuda", dtype=dt)

    if op == "linear_forward":
        outs = [empty(rows, f)]
        a = L.ssd_linear_fwd(rows, d, f, code, 2, x.data_ptr(), d, w.data_ptr(), d, None, None, 0, outs[0].data_ptr(), f)
        want = L.ssd_linear_forward(x, w, act=2)[:1]
    elif op == "gated_forward":
        outs = [empty(rows, f)]
        a = L.ssd_gated_fwd(rows, d, f, code, 3, x.data_ptr(), d, w.data_ptr(), d, w2.data_ptr(), d, None, None, outs[0].data_ptr(), f)
        want = L.ssd_gated_forward(x, w, w2)[:1]
    elif op == "linear_backward":
        outs = [empty(rows, d), empty(f, d, dt=torch.float32), empty(f, dt=torch.float32)]
        a = L.ssd_linear_bwd(rows, d, f, code, 2, B.SSD_F32, 0, dy.data_ptr(), f, x.data_ptr(), d, w.data_ptr(), d, z.data_ptr(), f, outs[0].data_ptr(), d,
                             outs[1].data_ptr(), d, outs[2].data_ptr())
        want = L.ssd_linear_backward(dy, x, w, z, act=2)
    else:
        outs = [empty(rows, d), empty(f, d, dt=torch.float32), empty(f, d, dt=torch.float32), empty(f, dt=torch.float32), empty(f, dt=torch.float32)]
        a = L.ssd_gated_bwd(rows, d, f, code, 3, B.SSD_F32, 0, dy.data_ptr(), f, x.data_ptr(), d, w.data_ptr(), d, w2.data_ptr(), d, z.data_ptr(), f,
                            u.data_ptr(), f, outs[0].data_ptr(), d, outs[1].data_ptr(), d, outs[2].data_ptr(), d, outs[3].data_ptr(), outs[4].data_ptr())
        want = L.ssd_gated_backward(dy, x, w, w2, z, u)
    n = C.c_int64()
    assert getattr(L.lib(), f"ssd_{op}_workspace")(C.byref(a), C.byref(n)) == B.SSD_OK and n.value > 0
    room = torch.full((n.value + 256,), 0x5A, device="cuda", dtype=torch.uint8)
    assert room.data_ptr() % 32 == 0
    assert getattr(L.lib(), f"ssd_{op}")(C.byref(a), room.data_ptr() + at, n.value, torch.cuda.current_stream().cuda_stream) == B.SSD_OK
    assert all(torch.equal(p, q) for p, q in zip(outs, want))
    assert bool((room[:at] == 0x5A).all()) and bool((room[at + n.value:] == 0x5A).all())
    # and the same through the torch interface
    if op == "linear_forward":
        assert torch.equal(L.ssd_linear_forward(x, w, act=2, workspace=room[at:at + n.value])[0], want[0])
        with pytest.raises(B.SsdError):
            L.ssd_linear_forward(x, w, act=2, workspace=room[at:at + n.value - 1])


@pytest.mark.parametrize("rows", [65535 * 8, 65535 * 8 + 1, 600000, 1048577])
@pytest.mark.parametrize("width", [(8, 8), (3, 5), (10, 10)], ids=str)
def test_more_rows_than_a_grid_is_high(rows, width):
    """Small float32 layers over very many rows: eight rows a block, and a grid is at most 65535 blocks high."""
    g, (d, f) = gen(3), width
    x, w, w2 = normal(g, rows, d, dtype=torch.float32), normal(g, f, d, dtype=torch.float32), normal(g, f, d, dtype=torch.float32)
    b, r = normal(g, f, dtype=torch.float32), normal(g, rows, f, dtype=torch.float32)
    y, z = L.ssd_linear_forward(x, w, bias=b, residual=r, act=2, keep=True)
    ref = R.linear_forward(x, w, b, r, 2)
    check(y, ref["y"], "y")
    check(z, ref["z"], "z")
    h, gate, up = L.ssd_gated_forward(x, w, w2, b, keep=True)
    ref = R.gated_forward(x, w, w2, b, None, 3)
    for got, k in ((h, "h"), (gate, "gate"), (up, "up")):
        check(got, ref[k], k)


BITS = """
import hashlib, sys, torch
from paper_2012_05396_b200 import layers as L
g = torch.Generator(device="cuda")

def call(rows, d, f, dtype, gated=False):
    g.manual_seed(rows * 7919 + d)
    x, w, w2 = (torch.empty(*s, device="cuda", dtype=dtype).normal_(0, 1, generator=g) for s in ((rows, d), (f, d), (f, d)))
    y = L.ssd_gated_forward(x, w, w2)[0] if gated else L.ssd_linear_forward(x, w)[0]
    return hashlib.sha256(y.view(torch.uint8).cpu().numpy().tobytes()).hexdigest()

f32, bf16 = torch.float32, torch.bfloat16
calls = [(1, 4096, 4096, f32), (2, 2048, 2048, f32), (4, 4096, 1000, f32), (8, 2048, 3001, f32), (8, 2049, 3000, f32), (1, 4096, 4096, bf16),
         (4, 1001, 2003, bf16), (8, 2048, 4096, bf16), (16, 1024, 4096, bf16), (1, 2048, 2048, f32, True), (8, 2048, 2048, f32, True), (5, 2048, 2048, bf16, True)]
first = int(sys.argv[1])
order = calls[first:] + calls[:first]
sums = {c: call(*c) for c in order}
print("\\n".join(sums[c] for c in calls))
"""


def test_same_bits_whatever_a_process_called_before():
    """A few-row call's bits follow from its sizes and alignment, not from which call a process made first."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    runs = [subprocess.run([sys.executable, "-c", BITS, str(first)], cwd=root, capture_output=True, text=True, timeout=600) for first in (0, 3, 6, 8)]
    assert all(r.returncode == 0 for r in runs), [r.stderr[-500:] for r in runs]
    lines = [r.stdout.split() for r in runs]
    assert len(lines[0]) == 12
    assert all(other == lines[0] for other in lines[1:]), [[i for i, (a, b) in enumerate(zip(lines[0], o)) if a != b] for o in lines]


def test_numbers_beyond_32_bits_are_refused():
    """They do not wrap around into a valid one."""
    g = gen(6)
    x, w = normal(g, 4, 8, dtype=torch.float32), normal(g, 6, 8, dtype=torch.float32)
    y, z = L.ssd_linear_forward(x, w, act=2, keep=True)
    a = torch.zeros(64, device="cuda")
    lst = L.GradList([a])
    calls = [lambda v: L.ssd_linear_forward(x, w, act=v), lambda v: L.ssd_gated_forward(x, w, w.clone(), act=v), lambda v: L.ssd_linear_backward(y, x, w, z, act=v),
             lambda v: L.ssd_gated_backward(y, x, w, w.clone(), z, z.clone(), act=v), lambda v: L.ssd_clip_grad_norm(lst, 1.0, nonfinite=v),
             lambda v: L.GradList([a], groups=[v]), lambda v: L.GradList([a], num_groups=v)]
    for call in calls:
        for v in (1 << 32, (1 << 32) + 1, -(1 << 32), 1 << 63, 1 << 70):
            with pytest.raises(B.SsdError) as e:
                call(v)
            assert e.value.status == B.SSD_ERR_ARG


def test_running_out_of_memory_is_torchs_error():
    """A result that no card holds (1.4 TB): what torch's own operators raise, and the next call works."""
    x, w = torch.ones(600000, 1, device="cuda"), torch.ones(600000, 1, device="cuda")
    with pytest.raises(torch.OutOfMemoryError):
        L.ssd_linear_forward(x, w)
    y, _ = L.ssd_linear_forward(x[:3], w[:5])
    assert bool((y == 1.0).all())
