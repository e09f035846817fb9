"""Host-only checks of include/gwtf_stage.h: exported symbols, constants,
struct layouts, and calls refused before a device is touched."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2509_21221_amd import mcf, stage

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gwtf_stage.h")


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def declared():
    return sorted(set(re.findall(r"\b(gwtf_stage_\w+)\s*\(", text())))


def test_every_declared_function_is_exported_and_bound():
    lib = mcf.load_library()
    names = declared()
    assert len(names) == 10
    for name in names:
        assert hasattr(lib, name), name
        assert callable(getattr(stage, name)), name


def test_constants_match_the_header():
    found = dict(re.findall(r"\b(GWTF_(?:TYPE|TOKEN|NORM)_\w+)\s*=\s*(\d+)", text()))
    found.update(re.findall(r"#define (GWTF_\w+) (\d+)", text()))
    assert len(found) == 11
    for name, value in found.items():
        assert getattr(stage, name) == int(value), name


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a C compiler")
def test_struct_layouts_match_the_header(tmp_path):
    structs = {c.__name__: c for c in [*stage._CALLS.values(), stage.gwtf_stage_shape_t]}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "gwtf_stage.h"', "int main(void) {"]
    for name, c in structs.items():
        lines.append(f'printf("{name} %zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {f}));' for f, _ in c._fields_]
        lines.append('printf("\\n");')
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    for line in subprocess.check_output([str(exe)], text=True).splitlines():
        name, size, *offsets = line.split()
        c = structs[name]
        assert ctypes.sizeof(c) == int(size), name
        assert [getattr(c, f).offset for f, _ in c._fields_] == [int(o) for o in offsets], name


def test_null_arguments_fail_cleanly():
    lib = stage._library()
    for name in stage._CALLS:
        assert getattr(lib, "gwtf_stage_" + name)(None, None) == mcf.GWTF_ERR_INVALID_ARG
        assert "handle is NULL" in stage.gwtf_stage_last_error(None)
    lib.gwtf_stage_destroy(None)
    out = ctypes.c_void_p(1)
    assert lib.gwtf_stage_create(None, None, ctypes.byref(out)) == mcf.GWTF_ERR_INVALID_ARG
    assert out.value is None
    assert lib.gwtf_stage_create(None, None, None) == mcf.GWTF_ERR_INVALID_ARG
    for bad in [(0, 1, 1), (1, 0, 1), (1, 1, 0), (1 << 31, 1, 1), (1, (1 << 20) + 1, 1), (1, 1, 1 << 31)]:
        with pytest.raises(mcf.GwtfError, match="range"):
            stage.gwtf_stage_create(*bad)
