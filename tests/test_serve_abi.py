"""CPU-only checks of the serving operators' C ABI: geometry, sizes and refusals, all before a GPU is touched."""
import ctypes

import numpy as np
import pytest

from paper_1804_01526_amd import hbfp
from tests import serve_ref

L = hbfp._lib
P = 0x100000          # a device address that nothing reads: every call below is refused on the host


def _cache(batch=2, heads=2, capacity=100, dim=64):
    c = hbfp.cache_plan(batch, heads, capacity, dim)
    c.k, c.v, c.k_exps, c.v_exps = P, P + (1 << 24), P + (2 << 24), P + (3 << 24)
    return c


def _h(dtype=1, data=P, st=(1024, 256, 64)):
    return hbfp.Heads(data, dtype, 0, *st)


def test_struct_sizes():
    assert ctypes.sizeof(hbfp.CacheDesc) == 96 and ctypes.sizeof(hbfp.Heads) == 40


@pytest.mark.parametrize("batch,heads,capacity,dim,slots,nblk", [
    (1, 1, 1, 1, 64, 1), (2, 3, 64, 32, 64, 1), (2, 3, 65, 33, 128, 2), (4, 8, 8192, 128, 8192, 4), (1, 1, 100, 256, 128, 8)])
def test_cache_geometry(batch, heads, capacity, dim, slots, nblk):
    c = hbfp.cache_plan(batch, heads, capacity, dim)
    assert (c.slots, c.nblk) == (slots, nblk) and c.code_bytes == batch * heads * slots * 16 * nblk
    assert c.exp_bytes == batch * heads * slots * nblk and c.k is None


def test_cache_plan_refusals():
    c = hbfp.CacheDesc()
    plan = lambda *a: L.hbfp_cache_plan(*a, ctypes.byref(c))
    for bad in ((0, 1, 1, 1), (1, 0, 1, 1), (1, 1, 0, 1), (1, 1, 1, 0), (-1, 1, 1, 1)):
        assert plan(*bad) == hbfp.ERR_ARG
    assert plan(1, 1, 10, 257) == hbfp.ERR_FORMAT and plan(1, 1, 1 << 24, 256) == hbfp.ERR_FORMAT
    assert plan(1, 1, (1 << 24) - 64, 256) == hbfp.OK and plan(1 << 31, 1, 1, 1) == hbfp.ERR_FORMAT
    assert L.hbfp_cache_plan(1, 1, 1, 1, None) == hbfp.ERR_ARG


def test_append_and_read_refusals():
    ref = ctypes.byref
    append = lambda c, k, v, t=1, n=P, vals=None: L.hbfp_cache_append(ref(c) if c else None, ref(k) if k else None, ref(v) if v else None, t, n, vals, None, None)
    c = _cache()
    assert append(None, _h(), _h()) == hbfp.ERR_ARG and append(c, None, _h()) == hbfp.ERR_ARG and append(c, _h(), None) == hbfp.ERR_ARG
    assert append(c, _h(), _h(), t=0) == hbfp.ERR_ARG and append(c, _h(), _h(), n=None) == hbfp.ERR_ARG and append(c, _h(), _h(), n=P + 2) == hbfp.ERR_ARG
    assert append(c, _h(3), _h(3)) == hbfp.ERR_FORMAT and append(c, _h(1), _h(2)) == hbfp.ERR_FORMAT
    assert append(c, _h(data=None), _h()) == hbfp.ERR_ARG and append(c, _h(0, P + 2), _h(0)) == hbfp.ERR_ARG
    assert append(c, _h(st=(1, -1, 1)), _h()) == hbfp.ERR_ARG and append(c, _h(), _h(), vals=P + 1) == hbfp.ERR_ARG
    bad = _cache()
    bad.slots += 64
    assert append(bad, _h(), _h()) == hbfp.ERR_LAYOUT
    for name, at in (("k", None), ("v_exps", P + 8)):
        bad = _cache()
        setattr(bad, name, at)
        assert append(bad, _h(), _h()) == hbfp.ERR_ARG
    bad = _h()
    bad.reserved = 1
    assert append(c, bad, _h()) == hbfp.ERR_ARG
    read = lambda dtype, n, k, v: L.hbfp_cache_read(ref(c), n, dtype, k, v, None)
    assert read(2, P, P, P) == hbfp.ERR_FORMAT and read(0, None, P, P) == hbfp.ERR_ARG and read(0, P, None, None) == hbfp.ERR_ARG
    assert read(0, P, P + 2, P) == hbfp.ERR_ARG


def test_attend_and_weigh_refusals():
    ref, c = ctypes.byref, _cache(capacity=9000)
    need = hbfp.cache_attend_workspace(c, 1, 8)
    assert need > 0 and need % 256 == 0 and hbfp.cache_attend_workspace(c, 1, 8, longest=64) == 0

    def attend(cache=c, q=_h(), t=1, h=8, n=P, longest=0, causal=1, out=_h(), lse=P, ws=P, size=need):
        return L.hbfp_cache_attend(ref(cache), ref(q), t, h, n, longest, 0.1, causal, ref(out), lse, ws, size, None)

    assert attend(h=7) == hbfp.ERR_ARG and attend(h=0) == hbfp.ERR_ARG and attend(t=0) == hbfp.ERR_ARG and attend(t=1 << 30, h=8) == hbfp.ERR_ARG
    assert attend(n=None) == hbfp.ERR_ARG and attend(lse=None) == hbfp.ERR_ARG and attend(longest=-1) == hbfp.ERR_ARG and attend(causal=2) == hbfp.ERR_ARG
    assert attend(q=_h(2)) == hbfp.ERR_FORMAT and attend(q=_h(5), out=_h(5)) == hbfp.ERR_FORMAT
    assert attend(out=_h(st=(1024, 256, 0))) == hbfp.ERR_ARG and attend(out=_h(st=(511, 512, 64))) == hbfp.ERR_ARG      # elements that meet
    assert attend(ws=None) == hbfp.ERR_WORKSPACE and attend(size=need - 1) == hbfp.ERR_WORKSPACE and attend(ws=P + 16) == hbfp.ERR_WORKSPACE
    n = ctypes.c_size_t(0)
    assert L.hbfp_cache_attend_workspace(ref(c), 1, 8, 3, 0, ref(n)) == hbfp.ERR_FORMAT
    assert L.hbfp_cache_attend_workspace(ref(c), 1, 9, 1, 0, ref(n)) == hbfp.ERR_ARG
    assert L.hbfp_cache_attend_workspace(ref(c), 1, 8, 1, 0, None) == hbfp.ERR_ARG

    def weigh(q=_h(), t=1, h=8, lse=P, w=P, out=P, ld=9000, causal=1):
        return L.hbfp_cache_weigh(ref(c), ref(q), t, h, P, 0.1, causal, lse, 1.0, w, out, ld, None)

    assert weigh(ld=8999) == hbfp.ERR_ARG and weigh(w=None) == hbfp.ERR_ARG and weigh(out=None) == hbfp.ERR_ARG and weigh(lse=None) == hbfp.ERR_ARG
    assert weigh(out=P + 400) == hbfp.ERR_ARG and weigh(h=3) == hbfp.ERR_ARG and weigh(q=_h(4)) == hbfp.ERR_FORMAT and weigh(causal=-1) == hbfp.ERR_ARG


def test_evict_refusals():
    ref, src = ctypes.byref, _cache()
    dst = _cache(capacity=50)
    for i, name in enumerate(("k", "v", "k_exps", "v_exps")):
        setattr(dst, name, P + ((8 + i) << 24))
    far = P + (20 << 24)

    def evict(s=src, d=dst, w=far, ld=100, n=far + 4096, keep=50, recent=5, w_out=far + 8192, ld_out=50, kept=far + 16384, n_out=far + 32768):
        return L.hbfp_cache_evict(ref(s), w, ld, n, keep, recent, ref(d), w_out, ld_out, kept, n_out, None)

    assert evict(keep=0) == hbfp.ERR_ARG and evict(keep=51) == hbfp.ERR_ARG and evict(recent=-1) == hbfp.ERR_ARG
    assert evict(ld=99) == hbfp.ERR_ARG and evict(ld_out=49) == hbfp.ERR_ARG
    for name in ("w", "n", "w_out", "kept", "n_out"):
        assert evict(**{name: None}) == hbfp.ERR_ARG
    assert evict(d=_cache(dim=32)) == hbfp.ERR_LAYOUT and evict(d=_cache(batch=1)) == hbfp.ERR_LAYOUT
    assert evict(d=src) == hbfp.ERR_ARG and evict(w_out=far) == hbfp.ERR_ARG and evict(n_out=far + 4096) == hbfp.ERR_ARG


def test_product_refusals():
    n, kp = ctypes.c_size_t(0), ctypes.c_int64(0)
    assert L.hbfp_rows_plan(3, 129, ctypes.byref(kp), ctypes.byref(n)) == hbfp.OK and (kp.value, n.value) == (256, 768)
    assert L.hbfp_rows_plan(0, 1, None, None) == hbfp.ERR_ARG and L.hbfp_rows_plan(1, 0, None, None) == hbfp.ERR_ARG
    quant = lambda src=P, dtype=0, r=4, c=8, ld=8, codes=P, scales=P: L.hbfp_quant_rows(src, dtype, r, c, ld, codes, scales, None)
    assert quant(src=None) == hbfp.ERR_ARG and quant(dtype=7) == hbfp.ERR_FORMAT and quant(ld=7) == hbfp.ERR_ARG and quant(codes=P + 4) == hbfp.ERR_ARG
    assert quant(scales=None) == hbfp.ERR_ARG and quant(r=0) == hbfp.ERR_ARG and quant(src=P + 2) == hbfp.ERR_ARG
    assert L.hbfp_linear_i8_workspace(4, 8, 133145, ctypes.byref(n)) == hbfp.ERR_RANGE and L.hbfp_linear_i8_workspace(4, 8, 133144, ctypes.byref(n)) == hbfp.OK
    assert 133144 * 127 ** 2 < 2 ** 31 <= 133145 * 127 ** 2
    assert L.hbfp_linear_i8_workspace(4, 0, 8, ctypes.byref(n)) == hbfp.ERR_ARG and L.hbfp_gemm_rows_workspace(4, 8, 8, None) == hbfp.ERR_ARG
    assert L.hbfp_linear_i8_workspace(4, 8, 16, ctypes.byref(n)) == hbfp.OK
    lin = lambda x=P, dtype=1, m=4, k=16, ldx=16, b=P, sb=P, bias=None, cols=8, y=P, ldy=8, ws=P, size=n.value: L.hbfp_linear_i8(
        x, dtype, m, k, ldx, b, sb, bias, cols, y, ldy, ws, size, None)
    assert lin(x=None) == hbfp.ERR_ARG and lin(ldx=15) == hbfp.ERR_ARG and lin(dtype=9) == hbfp.ERR_FORMAT and lin(b=P + 8) == hbfp.ERR_ARG
    assert lin(sb=None) == hbfp.ERR_ARG and lin(bias=P + 1) == hbfp.ERR_ARG and lin(y=None) == hbfp.ERR_ARG and lin(ldy=7) == hbfp.ERR_ARG
    assert lin(ws=None) == hbfp.ERR_WORKSPACE and lin(size=n.value - 1) == hbfp.ERR_WORKSPACE and lin(ws=P + 128) == hbfp.ERR_WORKSPACE
    gemm = lambda a=P, sa=P, b=P, sb=P, m=4, cols=8, k=16, y=P, dtype=0, ldy=8: L.hbfp_gemm_rows(a, sa, b, sb, None, m, cols, k, y, dtype, ldy, None, 0, None)
    assert gemm(a=P + 8) == hbfp.ERR_ARG and gemm(sa=None) == hbfp.ERR_ARG and gemm(k=200000) == hbfp.ERR_RANGE and gemm(dtype=3) == hbfp.ERR_FORMAT
    assert gemm(ldy=4) == hbfp.ERR_ARG and gemm(y=None) == hbfp.ERR_ARG and gemm(m=0) == hbfp.ERR_ARG


def test_the_definitions_that_the_gpu_tests_use():
    """Hand-worked numbers for the reference itself."""
    got = serve_ref.cached(np.array([[4, 0.5, 1.5, 2.5, -3.5, 7.4, 0, 0]]))
    np.testing.assert_array_equal(got, [[4, 0, 2, 2, -4, 7, 0, 0]])
    np.testing.assert_array_equal(serve_ref.cached(np.array([7.5, 1.0, 3.0, -7.0])), [8, 0, 4, -8])      # 1 / 2 and 3 / 2 are ties
    np.testing.assert_array_equal(serve_ref.cached(np.array([2.0 ** -128, 2.0 ** -129])), [2.0 ** -128, 0])
    assert serve_ref.evict(np.array([1, 3, 3, 0, 9, 2.0]), 6, 4, 1) == [1, 2, 4, 5]
    assert serve_ref.evict(np.array([1, 1, 1, 1.0]), 4, 2, 0) == [0, 1] and serve_ref.evict(np.array([1.0]), 1, 4, 0) == [0]
    codes, scale = serve_ref.rows(np.array([[127, -63.5, 0.5, 1.5], [0, 0, 0, 0]]))
    np.testing.assert_array_equal(codes, [[127, -64, 0, 2], [0, 0, 0, 0]])
    np.testing.assert_array_equal(scale, [np.float32(127) * np.float32(1 / 127), 0])
