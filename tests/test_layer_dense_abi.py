"""The argument blocks of the layer's products, row norm and shared pages are laid out as include/fi.h declares them, and calls that cannot be
right are refused before any device is needed."""
import ctypes
import os
import subprocess

import pytest

from paper_2002_02645_b200 import binding as fb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KINDS = [fb.fi_linear_t, fb.fi_linear_backward_t, fb.fi_layer_norm_t, fb.fi_pages_fork_t, fb.fi_pages_free_t, fb.fi_pages_compact_t]


@pytest.fixture(scope="module")
def declared(tmp_path_factory):
    where = tmp_path_factory.mktemp("layout")
    lines = []
    for kind in KINDS:
        name = kind.__name__
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        for field, _ in kind._fields_:
            lines.append(f'printf("{name}.{field} %zu %zu\\n", offsetof({name}, {field}), sizeof((({name} *)0)->{field}));')
    for name, value in fb.FI_ACTIVATIONS.items():
        lines.append(f'printf("act.{name} %d\\n", (int)FI_ACT_{name.upper()});')
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


def test_activations_are_numbered_as_in_the_header(declared):
    assert {n: declared[f"act.{n}"][0] for n in fb.FI_ACTIVATIONS} == fb.FI_ACTIVATIONS


def test_refusals_need_no_device():
    lib = fb.load_library()
    for call in (lib.fi_linear, lib.fi_linear_backward, lib.fi_layer_norm, lib.fi_layer_norm_backward):
        assert call(None, None) == fb.FI_ERR_INVALID_ARG
    for call in (lib.fi_pages_fork, lib.fi_pages_free, lib.fi_pages_compact):
        assert call(None, None, None) == fb.FI_ERR_INVALID_ARG
    assert lib.fi_kv_copy_pages(None, None, 0, None, None) == fb.FI_ERR_INVALID_ARG

    def linear(**kw):
        a = fb.fi_linear_t(x=1 << 20, weight=1 << 21, out=1 << 22, x_stride=64, weight_stride=64, out_stride=32, tokens=4, in_dim=64, out_dim=32,
                           activation=0, out_dtype=fb.FI_BF16)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.fi_linear(bytes(a), None)

    assert linear(tokens=0) == fb.FI_OK and linear(rows=1 << 23, out_rows=0) == fb.FI_OK      # nothing to do
    for bad in (dict(in_dim=60), dict(in_dim=0), dict(out_dim=36), dict(tokens=-1), dict(tokens=1 << 31), dict(tokens=(1 << 30) + 1),
                dict(in_dim=(1 << 30) + 8, x_stride=1 << 31, weight_stride=1 << 31), dict(out_dim=(1 << 30) + 8, out_stride=1 << 31), dict(activation=5), dict(activation=-1),
                dict(out_dtype=2), dict(x=None), dict(weight=None), dict(out=None), dict(x=8), dict(x_stride=60), dict(x_stride=56),
                dict(weight_stride=32), dict(out_stride=31), dict(out=(1 << 22) + 1), dict(residual=1 << 23, residual_stride=8), dict(bias=2),
                dict(preact=1 << 23, preact_stride=8), dict(wait_limit=-1), dict(rows=1 << 23, out_rows=-1)):
        assert linear(**bad) == fb.FI_ERR_INVALID_ARG, bad

    def norm(backward=False, **kw):
        a = fb.fi_layer_norm_t(x=1 << 20, dy=1 << 21, out=1 << 22, x_stride=64, dy_stride=64, out_stride=64, tokens=4, dim=64, eps=1e-5)
        for k, v in kw.items():
            setattr(a, k, v)
        return (lib.fi_layer_norm_backward if backward else lib.fi_layer_norm)(bytes(a), None)

    assert norm(tokens=0) == fb.FI_OK
    for bad in (dict(dim=0), dict(dim=16385), dict(tokens=-1), dict(x=None), dict(out=None), dict(x=(1 << 20) + 2), dict(x_stride=63), dict(out_stride=8),
                dict(x_dtype=3), dict(y_dtype=-1), dict(weight=2), dict(rows=1 << 23, x_rows=-1)):
        assert norm(**bad) == fb.FI_ERR_INVALID_ARG, bad
    for bad in (dict(dy=None), dict(rows=1 << 23, x_rows=4), dict(tokens_dev=1 << 23), dict(dweight=1 << 23), dict(dy_stride=8), dict(dy=(1 << 21) + 2)):
        assert norm(True, **bad) == fb.FI_ERR_INVALID_ARG, bad
    assert lib.fi_layer_norm_workspace(0) == 0 and lib.fi_layer_norm_workspace(16385) == 0 and lib.fi_layer_norm_workspace(100) > 0
    assert lib.fi_linear_backward_workspace(10, 64, 0) == 0 and lib.fi_linear_backward_workspace(10, 64, 4) >= 1280
    for dim, ctas in ((8, 444), (1024, 444), (2048, 592), (4096, 296), (16384, 148)):     # sums of as many CTAs as run at one time
        assert 2 * 4 * dim * ctas <= lib.fi_layer_norm_workspace(dim) <= 21 << 20
    assert lib.fi_pages_compact_workspace(-1) == 0 and lib.fi_pages_compact_workspace(1000) >= 4 * 1000
