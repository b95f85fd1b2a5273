"""The argument blocks of the attention-layer calls, which the binding packs field by field, are laid out as include/fi.h declares
them: a C program says where every field lies."""
import ctypes
import os
import subprocess

import pytest

from paper_2002_02645_b200 import binding as fb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KINDS = [fb.fi_pages_config_t, fb.fi_pages_extend_t, fb.fi_head_norm_rope_t, fb.fi_kv_config_t, fb.fi_kv_append_t, fb.fi_kv_attend_t]


@pytest.fixture(scope="module")
def declared(tmp_path_factory):
    where = tmp_path_factory.mktemp("layout")
    lines = []
    for kind in KINDS:
        name = kind.__name__
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        for field, _ in kind._fields_:
            lines.append(f'printf("{name}.{field} %zu %zu\\n", offsetof({name}, {field}), sizeof((({name} *)0)->{field}));')
    source = where / "layout.c"
    source.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "fi.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(where / "layout"), str(source)], check=True)
    out = subprocess.run([str(where / "layout")], check=True, stdout=subprocess.PIPE, text=True).stdout
    return {line.split()[0]: [int(x) for x in line.split()[1:]] for line in out.splitlines()}


@pytest.mark.parametrize("kind", KINDS, ids=lambda k: k.__name__)
def test_fields_lie_where_the_header_says(declared, kind):
    assert declared[kind.__name__] == [ctypes.sizeof(kind)]
    end = 0
    for field, _ in kind._fields_:
        at = getattr(kind, field)
        assert declared[f"{kind.__name__}.{field}"] == [at.offset, at.size], field
        assert 0 <= at.offset - end < 8                          # no field of the header is missing in between
        end = at.offset + at.size
    assert fb._packer(kind).size == ctypes.sizeof(kind)


def test_null_arguments_are_refused_without_a_device():
    lib, h = fb.load_library(), ctypes.c_void_p()
    assert lib.fi_pages_create(None, ctypes.byref(h)) == fb.FI_ERR_INVALID_ARG and not h.value
    assert lib.fi_kv_create(None, ctypes.byref(h)) == fb.FI_ERR_INVALID_ARG and not h.value
    for call in (lib.fi_pages_extend, lib.fi_kv_append, lib.fi_kv_attend):
        assert call(None, None, None) == fb.FI_ERR_INVALID_ARG
    for call in (lib.fi_head_norm_rope, lib.fi_head_norm_rope_backward):
        assert call(None, None) == fb.FI_ERR_INVALID_ARG
    assert lib.fi_kv_poll_status(None) == fb.FI_ERR_INVALID_ARG and lib.fi_kv_set_wait_limit(None, 1) == fb.FI_ERR_INVALID_ARG
    assert lib.fi_pages_destroy(None) == 0 and lib.fi_kv_destroy(None) == 0
