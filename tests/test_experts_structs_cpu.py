"""Every struct of sky_experts.h and sky_optim.h has its ctypes form in _lib: the same fields in the same
order, each of the same kind and size."""
import ctypes as C
import os
import re

import pytest

from paper_2202_11836_gb300 import _lib as L

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KIND = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float, "sky_dtype": C.c_int, "sky_route_weights": C.c_int,
        "sky_state_type": C.c_int}


def structs():
    for h in ("sky_experts.h", "sky_optim.h"):
        src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", h)).read(), flags=re.S)
        for body, name in re.findall(r"typedef\s+struct\s*\{([^}]*)\}\s*(\w+)\s*;", src):
            fields = []
            for line in filter(None, (s.strip() for s in body.split(";"))):
                kind, names = re.match(r"((?:const\s+)?\w+)\s*(.*)", line, re.S).groups()
                for n in names.split(","):
                    n = n.strip()
                    fields.append((n.lstrip("* "), C.c_void_p if n.startswith("*") else KIND[kind]))
            yield name, fields


@pytest.mark.parametrize("name,fields", list(structs()), ids=lambda v: v if isinstance(v, str) else None)
def test_struct(name, fields):
    t = getattr(L, "".join(p.capitalize() for p in name.split("_")))
    assert [n.rstrip("_") for n, _ in t._fields_] == [n for n, _ in fields]
    assert [k for _, k in t._fields_] == [k for _, k in fields]


def test_all_are_found():
    assert {n for n, _ in structs()} == {"sky_route_shape", "sky_rows_shape", "sky_grouped_shape", "sky_adamw_tensor",
                                         "sky_adamw_config", "sky_adamw_now"}
