"""Host-only checks of include/gwtf_learn.h: exported symbols, constants,
struct layouts, and calls refused before a device is touched."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from paper_2509_21221_amd import learn, mcf

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "gwtf_learn.h")


def text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_every_declared_function_is_exported_and_bound():
    lib = mcf.load_library()
    names = sorted(set(re.findall(r"\b(gwtf_learn_\w+)\s*\(", text())))
    assert len(names) == 8
    for name in names:
        assert hasattr(lib, name), name
        assert callable(getattr(learn, name)), name


def test_constants_match_the_header():
    found = dict(re.findall(r"\b(GWTF_(?:UNIFORM|STATE)_\w+)\s*=\s*(\d+)", text()))
    found.update(re.findall(r"#define (GWTF_\w+) (\d+)", text()))
    assert len(found) == 6
    for name, value in found.items():
        assert getattr(learn, name) == int(value), name


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs a C compiler")
def test_struct_layouts_match_the_header(tmp_path):
    structs = {c.__name__: c for c in [*learn._CALLS.values(), learn.gwtf_learn_tensor_t]}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "gwtf_learn.h"', "int main(void) {"]
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
    lib = learn._library()
    for name in learn._CALLS:
        assert getattr(lib, "gwtf_learn_" + name)(None, None) == mcf.GWTF_ERR_INVALID_ARG
        assert "handle is NULL" in learn.gwtf_learn_last_error(None)
    lib.gwtf_learn_destroy(None)
    out = ctypes.c_void_p(1)
    assert lib.gwtf_learn_create(-1, None, ctypes.byref(out)) == mcf.GWTF_ERR_INVALID_ARG
    assert out.value is None
    assert lib.gwtf_learn_create(0, None, None) == mcf.GWTF_ERR_INVALID_ARG
    out = ctypes.c_void_p(1)
    assert lib.gwtf_learn_list_create(None, 0, None, 0, ctypes.byref(out)) == mcf.GWTF_ERR_INVALID_ARG
    assert out.value is None
    lib.gwtf_learn_list_destroy(None)


def test_parts_of_one_memory_are_refused():
    """The check needs no device: spans of tensors are compared by address."""
    import torch

    apart = learn.LearnOps._apart
    base = torch.zeros(64)
    apart(None, [(base[:8], "params"), (base[8:16], "m"), (base[:0], "v")], [base[16:24], base[16:24], base[20:28]])
    for written, read in (([(base[:8], "params"), (base[7:9], "m")], []), ([(base[:8], "params")], [base[4:12]]),
                          ([(base[20:24], "params")], [base[16:40]]), ([(base[30:32], "v")], [base[0:40], base[2:4]]),
                          ([(base[:8], "params"), (base[:8], "params")], [])):
        with pytest.raises(ValueError, match="shares memory"):
            apart(None, written, read)
