"""Calls of the layer operators that are refused although every argument by itself is a good one.  No GPU: nothing is enqueued."""
import ctypes as C

import pytest

from paper_2012_05396_b200 import binding as B
from paper_2012_05396_b200 import build as libbuild
from paper_2012_05396_b200 import layers as L
from tests.test_layers_abi import BASE, STEP, args_of, large, need, status


@pytest.fixture(scope="module", autouse=True)
def built():
    libbuild.build_library()


@pytest.mark.parametrize("dtype", [B.SSD_BF16, B.SSD_F32])
@pytest.mark.parametrize("victim", ["x", "weight"])
@pytest.mark.parametrize("rows", [8, 64])
def test_only_the_residual_may_be_the_result(rows, victim, dtype):
    """A result over its residual is allowed; over another input that is the residual too it is not (x = act(x W^T) + x in place)."""
    a = args_of("linear_forward", rows=rows, in_features=64, out_features=64, dtype=dtype, **{n: 64 for n, t in L.ssd_linear_fwd._fields_ if n.startswith("ld")})
    if victim == "weight":
        a.rows = 64
    p = getattr(a, victim)
    a.residual = a.y = p
    assert status("linear_forward", a) == B.SSD_ERR_ARG
    a.z = None
    assert status("linear_forward", a) == B.SSD_ERR_ARG
    # and the same of a vector that the result lies over
    a = args_of("linear_forward", rows=1, in_features=64, out_features=64, dtype=B.SSD_F32, **{n: 64 for n, t in L.ssd_linear_fwd._fields_ if n.startswith("ld")})
    a.residual = a.y = a.bias
    assert status("linear_forward", a) == B.SSD_ERR_ARG


@pytest.mark.parametrize("op", ["linear_forward", "linear_backward", "gated_forward", "gated_backward"])
def test_workspaces_count_the_room_to_align_them(op):
    """A workspace may start on any 16 bytes; what calls take from it are multiples of 256 bytes on 32, so 16 more are asked for."""
    st, n = need(op, large(op, dtype=B.SSD_F32))
    assert st == B.SSD_OK and n > 0 and n % 256 == 16
    for at in (0, 16):
        assert status(op, large(op, dtype=B.SSD_F32), workspace=BASE + 100 * STEP + at, size=n - 1) == B.SSD_ERR_ARG
        assert status(op, large(op, dtype=B.SSD_F32), workspace=BASE + 100 * STEP + at + 8, size=n + 64) == B.SSD_ERR_ALIGN


def room(rows, d, f, op="linear_forward"):
    a = args_of(op, rows=rows, in_features=d, out_features=f, dtype=B.SSD_F32)
    for n, t in a._fields_:
        if n.startswith("ld"):
            setattr(a, n, d if n in ("ldx", "ldw", "ldwg", "ldwu") else f)
    st, n = need(op, a)
    assert st == B.SSD_OK
    return n


def test_which_float32_calls_take_their_operands_apart():
    """The kernel for a few rows needs no workspace.  It takes small calls; wide, shallow ones of many rows, where it is up to nine times slower, go to
    the tensor cores, whatever the number of their weights."""
    for small in ((1, 4096, 4096), (16, 1024, 1024), (64, 512, 512), (24, 1024, 1024), (1024, 64, 10), (1000, 1000, 8), (60, 1000, 1000)):
        assert room(*small) == 0, small
    for shallow in ((8000, 8, 1000), (1000, 64, 1000), (1000, 8, 1000), (250, 500, 500), (100000, 1, 64), (1463, 6, 1600), (846, 64, 512)):
        assert room(*shallow) > 0, shallow
        assert room(*shallow, op="gated_forward") > 0, shallow


def backward_room(rows, d, f, dtype, grad, op="linear_backward"):
    a = args_of(op, rows=rows, in_features=d, out_features=f, dtype=dtype, grad_dtype=grad)
    for n, t in a._fields_:
        if n.startswith("ld"):
            setattr(a, n, d if n in ("ldx", "ldw", "ldwg", "ldwu", "lddx", "lddw", "lddwg", "lddwu") else f)
    st, n = need(op, a)
    assert st == B.SSD_OK
    return n


def test_room_of_a_few_rows_through_many_weights():
    """The few-row kernel keeps a part of dx for every strip of weight rows, half a gigabyte for 16 rows of a vocabulary's width; from where the tensor
    cores are faster, the room does not grow with the weights."""
    for grad in (B.SSD_F32, B.SSD_BF16):
        for op in ("linear_backward", "gated_backward"):
            assert backward_room(16, 4096, 128256, B.SSD_BF16, grad, op) < 1 << 26
            assert backward_room(9, 32768, 8192, B.SSD_BF16, grad, op) < 1 << 26
    # small ones keep to it
    strips = -(-1024 // -(-1024 // 444))
    assert backward_room(16, 1024, 1024, B.SSD_BF16, B.SSD_F32) < strips * 16 * 1024 * 4 + (1 << 20)
