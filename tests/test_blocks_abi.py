"""Host-side checks of the residual-block entry points that need no GPU."""
import ctypes as C
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = ("lp_dropout", "lp_residual_norm", "lp_residual_norm_grad", "lp_grouped_linear", "lp_grouped_weight_grad")


@pytest.fixture(scope="module")
def pkg():
    import __graft_entry__ as ge
    ge.build()
    import paper_2506_20818_b200 as p
    p.load_library()
    return p


def header():
    return re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lp.h")).read(), flags=re.S)


def test_null_context_is_rejected(pkg):
    lib = pkg.load_library()
    for name in NAMES:
        f = getattr(lib, name)
        assert f(None, *[None if t is C.c_void_p else 0 for t in f.argtypes[1:]]) == -1


def test_entry_points_follow_the_header(pkg):
    lib, text = pkg.load_library(), header()
    for name in NAMES:
        params = re.search(name + r"\s*\(([^;]*)\);", text).group(1).split(",")
        kinds = [C.c_void_p if "*" in p else C.c_double if "double" in p else C.c_uint64 if "uint64_t" in p else C.c_int64 if "int64_t" in p else C.c_int32 for p in params]
        assert getattr(lib, name).argtypes == kinds


def test_descriptor_follows_the_header(pkg):
    body = re.search(r"typedef struct \{([^}]*)\} lp_residual_desc;", header()).group(1)
    want = []
    for line in body.split(";"):
        m = re.match(r"\s*(?:const )?(\w+)\s+(.*)", line.strip(), flags=re.S)
        if m:
            for name in m.group(2).split(","):
                ptr = "*" in name
                kind = C.c_void_p if ptr else {"int64_t": C.c_int64, "int32_t": C.c_int32, "uint64_t": C.c_uint64, "double": C.c_double}[m.group(1)]
                want.append((name.strip().lstrip("*"), kind))
    assert [tuple(f) for f in pkg.ResidualDesc._fields_] == want


def test_packed_descriptor_is_the_structure(pkg):
    from paper_2506_20818_b200 import binding
    values = (5, 6, 1, 0, 2, 1, 1e-5, 0.5, 0.25, 2**64 - 1, 3, 9, 11, 12, 13, 14, 15, 16)
    packed = binding._RESIDUAL.pack(*values)
    assert len(packed) == C.sizeof(pkg.ResidualDesc)
    d = pkg.ResidualDesc.from_buffer_copy(packed)
    assert tuple(getattr(d, name) for name, _ in pkg.ResidualDesc._fields_) == values
