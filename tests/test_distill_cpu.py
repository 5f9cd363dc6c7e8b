"""CPU-side checks of include/class_distill.h: exported symbols, sizes, and arguments that are refused before anything is launched; the
formulas of its gradient against differences, in 64 bits."""
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ks():
    import paper_2102_06025_amd as ks
    if not os.path.exists(ks.lib_path()):
        from paper_2102_06025_amd.build import build
        build()
    ks.lib()
    return ks


def test_header_symbols_are_exported(ks):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "class_distill.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(class_[a-z0-9_]+)\s*\(", src))
    assert names == {"class_distill_fwd_bwd", "class_distill_workspace"}
    assert all(hasattr(ks.lib(), n) and hasattr(ks, n) for n in names)


def test_workspace(ks):
    assert [ks.class_distill_workspace(*a) for a in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 31, 1, 1), ((1 << 32) + 8, 1, 1), (8, (1 << 32) + 1, 1), (8, 1, 4_097),
                                                     (8, 1, (1 << 32) + 1), (-1, 1, 1))] == [0] * 9
    assert 0 < ks.class_distill_workspace(1, 1, 1) <= 1_024
    assert 0 < ks.class_distill_workspace(390_625, 1_024, 128) < 1 << 20


def test_refusals(ks):
    def call(z=256, ldl=100, dtype=1, C=100, B=2, ids=256, t=256, tt=1, K=4, T=1.0, lo=256, lm=256, dz=512, ldd=100, ws=256, size=1 << 20, st=None):
        return ks.lib().class_distill_fwd_bwd(z, ldl, dtype, C, B, ids, t, tt, K, T, 1.0, lo, lm, dz, ldd, ws, size, st, None)
    for bad in (dict(z=None), dict(ids=None), dict(t=None), dict(lo=None), dict(lm=None), dict(dz=None), dict(ws=None), dict(ldl=99), dict(ldd=99), dict(dtype=2),
                dict(tt=2), dict(C=0), dict(C=1 << 31, ldl=1 << 31, ldd=1 << 31), dict(B=0), dict(B=-1), dict(K=0), dict(T=0.0), dict(T=-1.0),
                dict(T=float("nan")), dict(T=float("inf")), dict(T=1e-31), dict(T=1e-45), dict(T=1e31), dict(z=258), dict(dz=258), dict(z=257, dtype=0), dict(t=258), dict(t=257, tt=0), dict(ids=258),
                dict(lo=257), dict(lm=257), dict(ws=260), dict(st=258), dict(z=512, ldl=101)):
        assert call(**bad) == ks.KS_INVALID_ARG, bad
    assert call(K=4_097) == ks.KS_UNSUPPORTED
    assert call(size=255) == ks.KS_WORKSPACE_TOO_SMALL


def test_binding_refuses_host_tensors(ks):
    with pytest.raises(TypeError):
        ks.class_distill_fwd_bwd(torch.zeros(2, 8), torch.zeros(2, 3, dtype=torch.int32), torch.zeros(2, 3))


@pytest.mark.parametrize("T", [0.7, 1.0, 3.0])
def test_the_formula_of_the_gradient(T):
    """T^2 sum q (log q - log p) has the gradient T (p - q): differences of 64-bit losses."""
    gen = torch.Generator().manual_seed(1)
    z, q = torch.randn(9, generator=gen, dtype=torch.float64), torch.zeros(9, dtype=torch.float64)
    q[torch.tensor([2, 5, 7])] = torch.softmax(torch.randn(3, generator=gen, dtype=torch.float64) / T, 0)

    def loss(z):
        return T * T * (torch.xlogy(q, q) - q * torch.log_softmax(z / T, 0)).sum()
    eps = 1e-5
    for c in range(9):
        d = torch.zeros(9, dtype=torch.float64)
        d[c] = eps
        # third derivatives are below 1 / T, so differences are off by eps^2 / (6 T), and by roundings of 1e-15 / eps
        assert abs((loss(z + d) - loss(z - d)) / (2 * eps) - T * (torch.softmax(z / T, 0)[c] - q[c])) < 1e-9
