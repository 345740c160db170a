"""CPU-only checks of what the header says about the largest sizes of the microscaled operators and of the norm."""
import ctypes
import os
import re

import pytest

from paper_1804_01526_amd import hbfp

L = hbfp._lib
ref = ctypes.byref
MOST_ROWS, MOST_K = 0x7FFFFFFF, 0x7FFFFF00
HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "hbfp.h")


def test_the_header_names_the_limits_of_a_plan():
    text = open(HEADER).read()
    said = re.search(r"hbfp_mx4_plan \(host only\).*?rows above (0x[0-9a-f]+), kdim above (0x[0-9a-f]+)", text, re.S)
    assert said, "the limits are not in the header"
    rows, kdim = (int(n, 16) for n in said.groups())
    d = hbfp.Mx4Desc()
    assert L.hbfp_mx4_plan(rows, 1, ref(d)) == hbfp.OK and L.hbfp_mx4_plan(rows + 1, 1, ref(d)) == hbfp.ERR_ARG
    assert L.hbfp_mx4_plan(1, kdim, ref(d)) == hbfp.OK and L.hbfp_mx4_plan(1, kdim + 1, ref(d)) == hbfp.ERR_ARG
    assert (rows, kdim) == (MOST_ROWS, MOST_K)


@pytest.mark.parametrize("rows,kdim", [(MOST_ROWS, 1), (1, MOST_K), (MOST_ROWS, MOST_K)])
def test_a_plan_at_its_limits(rows, kdim):
    d = hbfp.mx4_plan(rows, kdim)
    assert d.groups == (kdim + 255) // 256 and d.groups * 256 < 1 << 31 and d.scale_rows == (rows + 15) // 16 * 16
    assert d.code_bytes == d.groups * rows * 128 and d.scale_bytes == d.groups * d.scale_rows * 8


def test_products_and_norms_have_the_same_limits():
    n = ctypes.c_size_t(0)
    for size in (L.hbfp_gemm_mx4_workspace, L.hbfp_linear_mx4_workspace):
        for at in ((MOST_ROWS, 1, 1), (1, MOST_ROWS, 1), (1, 1, MOST_K)):
            assert size(*at, ref(n)) == hbfp.OK
            assert size(*(v + (v > 1) for v in at), ref(n)) == hbfp.ERR_ARG
    for at in ((MOST_ROWS, 1), (1, MOST_K)):
        assert L.hbfp_norm_grad_workspace(*at, ref(n)) == hbfp.OK
        assert L.hbfp_norm_grad_workspace(*(v + (v > 1) for v in at), ref(n)) == hbfp.ERR_ARG


def test_a_source_s_rows_are_a_contraction_where_it_is_converted_down_its_columns():
    """A source of more rows than a contraction may have has no plan for that operand; along its rows it has one."""
    rows = MOST_K + 1
    assert L.hbfp_mx4_plan(rows, 200, ref(hbfp.Mx4Desc())) == hbfp.OK
    assert L.hbfp_mx4_plan(200, rows, ref(hbfp.Mx4Desc())) == hbfp.ERR_ARG
