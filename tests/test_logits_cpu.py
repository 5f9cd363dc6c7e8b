"""CPU-side checks of include/class_logits.h: exported symbols, sizes, and arguments that are refused before anything is launched."""
import ctypes as ct
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
i64, i32, u32, f32 = ct.c_int64, ct.c_int, ct.c_uint32, ct.c_float
NULL, ONE, ODD = ct.c_void_p(0), ct.c_void_p(256), ct.c_void_p(257)  # never read: the checks come first


@pytest.fixture(scope="module")
def ks():
    import paper_2102_06025_amd as ks
    if not os.path.exists(ks.lib_path()):
        from paper_2102_06025_amd.build import build
        build()
    ks.lib()
    return ks


def test_header_symbols_are_exported(ks):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "class_logits.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(class_[a-z0-9_]+)\s*\(", src))
    assert names == {"class_codes_bytes", "class_quantize_rows", "class_logits_int8", "class_logits_adjust"}
    assert all(hasattr(ks.lib(), n) and hasattr(ks, n) for n in names)


@pytest.mark.parametrize("n,D,rows,classes", [(1, 1, 32, False), (1, 1, 64, True), (33, 64, 64, False), (128, 65, 128, True), (129, 512, 192, True),
                                              (10_000, 128, 10_048, True)])
def test_bytes_of_codes(ks, n, D, rows, classes):
    assert ks.class_codes_bytes(n, D, classes) == rows * ((D + 31) // 32 * 32)


def test_bytes_of_refused_sizes(ks):
    assert [ks.class_codes_bytes(*a) for a in ((0, 8), (8, 0), (8, 65_537), (-1, 8))] == [0] * 4
    assert ks.class_codes_bytes(4_000_000, 65_536, True) == 4_000_000 * 65_536


def test_quantize_refuses(ks):
    def call(V=ONE, dtype=1, n=5, D=8, ldv=8, flags=0, codes=ONE, scale=ONE):
        return ks.lib().class_quantize_rows(V, i32(dtype), i64(n), i32(D), i64(ldv), u32(flags), codes, scale, NULL)
    for bad in (dict(V=NULL), dict(codes=NULL), dict(codes=ODD), dict(scale=NULL), dict(n=0), dict(n=1 << 31), dict(D=0), dict(ldv=7), dict(dtype=3),
                dict(flags=4), dict(dtype=2), dict(dtype=2, scale=NULL, flags=2), dict(V=ODD)):
        assert call(**bad) == ks.KS_INVALID_ARG, bad
    assert call(D=65_537, ldv=65_537) == ks.KS_UNSUPPORTED


def test_product_refuses(ks):
    def call(xq=ONE, xs=ONE, wq=ONE, ws=ONE, C=5, D=8, B=3, out=ONE, dtype=1, ldl=5):
        return ks.lib().class_logits_int8(xq, xs, wq, ws, NULL, i64(C), i32(D), i32(B), f32(1.0), out, i32(dtype), i64(ldl), NULL)
    for bad in (dict(xq=NULL), dict(xs=NULL), dict(wq=NULL), dict(ws=NULL), dict(out=NULL), dict(xq=ODD), dict(wq=ODD), dict(out=ODD),
                dict(out=ct.c_void_p(258)), dict(C=0), dict(C=1 << 31, ldl=1 << 31), dict(D=0), dict(B=0), dict(ldl=4), dict(dtype=2)):
        assert call(**bad) == ks.KS_INVALID_ARG, bad
    assert call(D=65_537) == ks.KS_UNSUPPORTED
    assert call(B=4_194_241) == ks.KS_UNSUPPORTED


def test_adjust_refuses(ks):
    def call(z=ONE, ldl=100, out=ONE, ldo=100, dtype=1, C=100, c0=0, Cg=100, B=2, so=NULL, si=NULL, slen=0, smax=0, bo=NULL, bi=NULL, bv=NULL,
             blen=0, bmax=0, al=NULL, lda=4, nm=2, mr=NULL):
        return ks.lib().class_logits_adjust(z, i64(ldl), out, i64(ldo), i32(dtype), i64(C), i64(c0), i64(Cg), i32(B), so, si, i64(slen), i32(smax),
                                            NULL, NULL, NULL, NULL, bo, bi, bv, i64(blen), i32(bmax), al, i64(lda), i32(nm), mr, NULL, NULL)
    for bad in (dict(z=NULL), dict(out=NULL), dict(B=0), dict(C=0, Cg=0), dict(c0=-1), dict(c0=1), dict(Cg=1 << 31), dict(ldl=99), dict(ldo=99),
                dict(ldo=101), dict(dtype=2), dict(out=ODD), dict(z=ct.c_void_p(258)), dict(so=ONE, slen=4, smax=4), dict(smax=-1), dict(bmax=-1),
                dict(slen=-1), dict(bo=ONE, bi=ONE, blen=4, bmax=4), dict(bo=ONE, bv=ONE, blen=4, bmax=4), dict(smax=1 << 29, bmax=1 << 29),
                dict(al=ONE, lda=3), dict(al=ONE, nm=0), dict(al=ONE, nm=1)):
        assert call(**bad) == ks.KS_INVALID_ARG, bad
    assert call() == ks.KS_OK  # in place with nothing to do: nothing is launched


def test_binding_refuses_host_tensors(ks):
    with pytest.raises(TypeError):
        ks.class_quantize_rows(torch.zeros(4, 8))
    with pytest.raises(TypeError):
        ks.class_logits_int8(torch.zeros(1024, dtype=torch.int8), torch.zeros(1), torch.zeros(4096, dtype=torch.int8), torch.zeros(1), 1.0)
    with pytest.raises(TypeError):
        ks.class_logits_adjust(torch.zeros(2, 8))


def test_adjust_refuses_a_first_class_near_the_largest_number(ks):
    L, p = ks.lib(), 256
    for c0, Cg in (((1 << 63) - 1, 100), ((1 << 63) - 50, 100), (0, -(1 << 63)), (1 << 62, 1 << 30)):
        assert L.class_logits_adjust(p, 100, p, 100, 1, 100, c0, Cg, 2, None, None, 0, 0, None, None, None, None, None, None, None, 0, 0, None, 4, 2,
                                     None, None, None) == ks.KS_INVALID_ARG, (c0, Cg)


def test_bytes_of_sizes_beyond_a_c_int(ks):
    """Sizes that no call takes have no codes, not the codes of their low 32 bits."""
    assert [ks.class_codes_bytes(*a) for a in ((8, (1 << 32) + 8), (8, 8 - (1 << 32)), (1 << 31, 8), (1 << 62, 65_536), ((1 << 64) + 8, 8))] == [0] * 5
    assert ks.class_codes_bytes((1 << 31) - 1, 8) == (1 << 31) * 32
