"""The key-value cache's structs and constants are the same in include/msi.h and
in the binding."""
import ctypes
import os
import subprocess

import pytest

from paper_2608_23805_gb300 import native as N

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
STRUCTS = (N.msi_kv_desc, N.msi_kv_attention_args)


@pytest.fixture(scope="module")
def c_values(tmp_path_factory):
    exprs = ["MSI_KV_Q8", "MSI_KV_E4M3", "MSI_KV_OBSERVE"]
    for s in STRUCTS:
        exprs.append("sizeof(%s)" % s.__name__)
        for f in s._fields_:
            exprs += ["offsetof(%s, %s)" % (s.__name__, f[0]), "sizeof(((%s*)0)->%s)" % (s.__name__, f[0])]
    d = tmp_path_factory.mktemp("abi")
    src = d / "v.c"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"msi.h\"\nint main(void) {\n"
                   + "".join('  printf("%%lld\\n", (long long)(%s));\n' % e for e in exprs) + "  return 0;\n}\n")
    subprocess.run(["gcc", "-I", INCLUDE, str(src), "-o", str(d / "v")], check=True)
    out = subprocess.run([str(d / "v")], check=True, capture_output=True, text=True).stdout.split()
    return dict(zip(exprs, map(int, out)))


def test_constants(c_values):
    for name in ("MSI_KV_Q8", "MSI_KV_E4M3", "MSI_KV_OBSERVE"):
        assert getattr(N, name) == c_values[name]


@pytest.mark.parametrize("struct", STRUCTS, ids=lambda s: s.__name__)
def test_layout(c_values, struct):
    assert ctypes.sizeof(struct) == c_values["sizeof(%s)" % struct.__name__]
    for f in struct._fields_:
        got = getattr(struct, f[0])
        assert (got.offset, got.size) == (c_values["offsetof(%s, %s)" % (struct.__name__, f[0])],
                                          c_values["sizeof(((%s*)0)->%s)" % (struct.__name__, f[0])]), f[0]
