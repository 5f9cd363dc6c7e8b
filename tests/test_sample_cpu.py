"""CPU-side checks of include/class_sample.h: exported symbols, sizes, and arguments that are refused before anything is launched."""
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
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "class_sample.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(class_[a-z0-9_]+)\s*\(", src))
    assert names == {"class_sample", "class_sample_workspace"}
    assert all(hasattr(ks.lib(), n) and hasattr(ks, n) for n in names)


def test_workspace(ks):
    assert [ks.class_sample_workspace(*a) for a in ((0, 1), (1, 0), (1 << 31, 1), ((1 << 32) + 8, 1), (8, (1 << 32) + 1), (-1, 1))] == [0] * 6
    assert ks.class_sample_workspace(1, 1) == 768
    assert ks.class_sample_workspace(390_625, 256) >= 256 * 12
    assert 0 < ks.class_sample_workspace((1 << 31) - 1, 1) <= 4_096 * 12 + 2_048 * 12 + 4_096 * 8 + 2_048  # parts grow with the row


def test_refusals(ks):
    def call(z=256, ldl=100, dtype=1, C=100, B=2, u=256, t=None, k=None, p=None, m=None, ids=256, lp=None, ws=256, size=1 << 20):
        return ks.lib().class_sample(z, ldl, dtype, C, B, u, t, k, p, m, ids, lp, ws, size, None)
    for bad in (dict(z=None), dict(u=None), dict(ids=None), dict(ws=None), dict(ldl=99), dict(dtype=2), dict(C=0), dict(C=1 << 31, ldl=1 << 31), dict(B=0),
                dict(B=-1), dict(z=258), dict(z=257, dtype=0), dict(ws=260), dict(u=257), dict(t=257), dict(k=258), dict(p=257), dict(m=259), dict(ids=258),
                dict(lp=257)):
        assert call(**bad) == ks.KS_INVALID_ARG, bad
    assert call(size=767) == ks.KS_WORKSPACE_TOO_SMALL


def test_binding_refuses_host_tensors(ks):
    with pytest.raises(TypeError):
        ks.class_sample(torch.zeros(2, 8), torch.zeros(2))
