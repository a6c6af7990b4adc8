"""The binding's struct is the header's: names, order, offsets and types of the
fields as a C compiler has them."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

import paper_2608_17995_gb300 as av

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def header_fields():
    text = open(os.path.join(ROOT, "include", "avits.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} avits_kv_cache;", text).group(1)
    fields = []
    for line in filter(None, (x.strip() for x in body.split(";"))):
        kind, names = re.match(r"((?:const )?\w+\s*\*?)\s*(.*)", line, re.S).groups()
        fields += [(n.strip(), re.sub(r"\s", "", kind)) for n in names.split(",")]
    return fields


def test_names_and_types():
    kinds = {"void*": ctypes.c_void_p, "constint32_t*": ctypes.c_void_p, "int32_t*": ctypes.c_void_p,
             "float*": ctypes.c_void_p, "int64_t": ctypes.c_int64, "int32_t": ctypes.c_int32}
    got = header_fields()
    assert len(got) == 21
    assert [(n, kinds[k]) for n, k in got] == list(av._CacheStruct._fields_)


def test_sizes_and_offsets(tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    names = [n for n, _ in header_fields()]
    src = tmp_path / "offsets.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "avits.h"\nint main(void) {\n'
                   '  printf("%zu\\n", sizeof(avits_kv_cache));\n' +
                   "".join('  printf("%%zu %%zu\\n", offsetof(avits_kv_cache, %s), '
                           'sizeof(((avits_kv_cache*)0)->%s));\n' % (n, n) for n in names) +
                   "  return 0;\n}\n")
    exe = str(tmp_path / "offsets")
    subprocess.check_call([cc, str(src), "-I" + os.path.join(ROOT, "include"), "-o", exe])
    out = subprocess.check_output([exe], text=True).split("\n")
    assert int(out[0]) == ctypes.sizeof(av._CacheStruct)
    for n, line in zip(names, out[1:]):
        field = getattr(av._CacheStruct, n)
        assert [field.offset, field.size] == [int(x) for x in line.split()], n
