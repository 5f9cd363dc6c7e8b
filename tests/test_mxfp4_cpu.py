"""CPU-side checks of include/class_mxfp4.h: exported symbols, sizes, and arguments that are refused before anything is launched."""
import ctypes as ct
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, ONE, ODD = None, 256, 257  # never read: the checks come first


@pytest.fixture(scope="module")
def ks():
    import paper_2102_06025_amd as ks
    if not os.path.exists(ks.lib_path()):
        from paper_2102_06025_amd.build import build
        build()
    ks.lib()
    return ks


def test_header_symbols_are_exported(ks):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "class_mxfp4.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(class_[a-z0-9_]+)\s*\(", src))
    assert names == {"class_mxfp4_bytes", "class_quantize_mxfp4", "class_dequantize_mxfp4", "class_logits_mxfp4"}
    assert all(hasattr(ks.lib(), n) and hasattr(ks, n) for n in names)


@pytest.mark.parametrize("n,D,groups,classes", [(1, 1, 1, False), (1, 1, 2, True), (33, 64, 2, False), (128, 65, 4, True), (129, 512, 6, True),
                                                (10_000, 333, 314, True)])
def test_bytes_of_codes(ks, n, D, groups, classes):
    pieces = (D + 63) // 64
    assert ks.class_mxfp4_bytes(n, D, classes) == groups * (1024 * pieces + 256 * ((pieces + 3) // 4))


def test_bytes_of_refused_sizes(ks):
    assert [ks.class_mxfp4_bytes(*a) for a in ((0, 8), (8, 0), (8, 65_537), (-1, 8), (1 << 31, 8), (8, (1 << 32) + 8), ((1 << 64) + 8, 8))] == [0] * 7
    assert ks.lib().class_mxfp4_bytes(8, 8, 2) == 0
    assert ks.class_mxfp4_bytes((1 << 31) - 1, 65_536, True) == (1 << 26) * (1024 * 1024 + 256 * 256)


@pytest.mark.parametrize("name", ["class_quantize_mxfp4", "class_dequantize_mxfp4"])
def test_rows_refuse(ks, name):
    def call(V=ONE, dtype=1, n=5, D=8, ldv=8, flags=0, codes=ONE):
        if name == "class_quantize_mxfp4":
            return ks.lib().class_quantize_mxfp4(V, dtype, n, D, ldv, flags, codes, NULL)
        return ks.lib().class_dequantize_mxfp4(codes, n, D, flags, V, dtype, ldv, NULL)
    for bad in (dict(V=NULL), dict(codes=NULL), dict(codes=ODD), dict(codes=264), dict(n=0), dict(n=-1), dict(n=1 << 31), dict(D=0), dict(ldv=7),
                dict(dtype=2), dict(dtype=-1), dict(flags=2), dict(V=ODD), dict(V=258), dict(V=257, dtype=0)):
        assert call(**bad) == ks.KS_INVALID_ARG, bad
    assert call(D=65_537, ldv=65_537) == ks.KS_UNSUPPORTED


def test_product_refuses(ks):
    def call(x=ONE, w=ONE, C=5, D=8, B=3, out=ONE, dtype=1, ldl=5):
        return ks.lib().class_logits_mxfp4(x, w, NULL, C, D, B, 1.0, out, dtype, ldl, NULL)
    for bad in (dict(x=NULL), dict(w=NULL), dict(out=NULL), dict(x=ODD), dict(w=264), dict(out=ODD), dict(out=258), dict(C=0), dict(C=1 << 31, ldl=1 << 31),
                dict(D=0), dict(B=0), dict(B=-1), dict(ldl=4), dict(dtype=2)):
        assert call(**bad) == ks.KS_INVALID_ARG, bad
    assert call(D=65_537) == ks.KS_UNSUPPORTED
    assert call(B=4_194_241) == ks.KS_UNSUPPORTED


def test_binding_refuses(ks):
    with pytest.raises(TypeError):
        ks.class_quantize_mxfp4(torch.zeros(4, 8))
    with pytest.raises(TypeError):
        ks.class_dequantize_mxfp4(torch.zeros(1280, dtype=torch.uint8), 4, 8)
    with pytest.raises(TypeError):
        ks.class_logits_mxfp4(torch.zeros(1280, dtype=torch.uint8), torch.zeros(2560, dtype=torch.uint8), 4, 8, 8, 1.0)
    for sizes, code in (((0, 8, 8), ks.KS_INVALID_ARG), ((1, 1 << 31, 8), ks.KS_INVALID_ARG), ((1, 8, (1 << 32) + 8), ks.KS_INVALID_ARG),
                        ((1, 8, 65_537), ks.KS_UNSUPPORTED), ((4_194_241, 8, 8), ks.KS_UNSUPPORTED)):
        with pytest.raises(ks.KsError) as e:
            ks.class_logits_mxfp4(torch.zeros(1280, dtype=torch.uint8), torch.zeros(2560, dtype=torch.uint8), *sizes, 1.0)
        assert e.value.code == code
    for sizes, code in (((0, 8), ks.KS_INVALID_ARG), ((1 << 31, 8), ks.KS_INVALID_ARG), ((4, 65_537), ks.KS_UNSUPPORTED)):
        with pytest.raises(ks.KsError) as e:
            ks.class_dequantize_mxfp4(torch.zeros(1280, dtype=torch.uint8), *sizes)
        assert e.value.code == code
