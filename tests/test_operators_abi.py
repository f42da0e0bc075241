"""Host-side checks of the embedding and orthogonalisation entry points that need no GPU."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__ as ge
    ge.build()
    import paper_2506_20818_b200 as p
    p.load_library()
    return p


def test_struct_layouts(pkg):
    assert C.sizeof(pkg.Matrix) == 16 and pkg.Matrix.rows.offset == 8
    assert C.sizeof(pkg.MuonDesc) == 12 * 8 + 2 * 4 and pkg.MuonDesc.coeffs.offset == 32 and pkg.MuonDesc.steps.offset == 100
    assert pkg.LP_NO_PADDING == -2**31


def test_null_context_is_rejected(pkg):
    lib = pkg.load_library()
    assert lib.lp_embed(None, 0, None, 1, 1, 1, None, 0, 0, 1.0, 0, None, 1) == -1
    assert lib.lp_embed_grad(None, 0, None, 1, None, 0, 0, 1.0, 1, 1, 0, None, 1, 0) == -1
    assert lib.lp_orthogonalize(None, 0, 1, 1, 1, None, 1, 1, 5, None, 1e-7, None, 1, 1) == -1
    assert lib.lp_muon_step(None, None, None, 0, 0, None, None, None, None, 1, None, None, None) == -1


def test_entry_points_have_their_argument_counts(pkg):
    """The ctypes signatures follow the header's parameter lists."""
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "lp.h")).read(), flags=re.S)
    lib = pkg.load_library()
    for name in ("lp_embed", "lp_embed_grad", "lp_orthogonalize", "lp_muon_step"):
        params = re.search(name + r"\s*\(([^;]*)\);", text).group(1).split(",")
        kinds = [C.c_void_p if "*" in p else C.c_double if "double" in p else C.c_int64 if "int64_t" in p else C.c_int32 for p in params]
        assert getattr(lib, name).argtypes == kinds
