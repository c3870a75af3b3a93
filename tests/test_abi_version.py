"""The header, the binding's structs and the library agree, and a library of another version is refused (CPU only)."""
import ctypes as C
import os
import subprocess
import types

import pytest

import paper_2609_34370_b200 as spx
from paper_2609_34370_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = {"spx_attn_args_t": binding.AttnArgs, "spx_sample_args_t": binding.SampleArgs, "spx_kv_append_args_t": binding.KvAppendArgs,
           "spx_logprob_args_t": binding.LogprobArgs, "spx_conf_args_t": binding.ConfArgs, "spx_lm_head_args_t": binding.LmHeadArgs}


def test_structs_have_the_headers_layout(tmp_path):
    """A C program against the header prints every struct's size and every field's offset."""
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "spx.h"', "int main(void) {", 'printf("%d\\n", SPX_ABI_VERSION);']
    for name, struct in STRUCTS.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        for field, *_ in struct._fields_:
            lines.append(f'printf("{name}.{field} %zu\\n", offsetof({name}, {field}));')
    source, program = tmp_path / "layout.c", tmp_path / "layout"
    source.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(program), str(source)], check=True)
    version, *rows = subprocess.run([str(program)], check=True, capture_output=True, text=True).stdout.split("\n")
    assert int(version) == binding.ABI_VERSION
    want = dict(row.rsplit(" ", 1) for row in rows if row)
    for name, struct in STRUCTS.items():
        assert C.sizeof(struct) == int(want[name]), name
        for field, *_ in struct._fields_:
            assert getattr(struct, field).offset == int(want[f"{name}.{field}"]), (name, field)


def test_the_library_has_the_bindings_version():
    build.build()
    assert spx.load_library().spx_abi_version() == binding.ABI_VERSION


@pytest.mark.parametrize("stale", [types.SimpleNamespace(), types.SimpleNamespace(spx_abi_version=lambda: binding.ABI_VERSION + 1)])
def test_a_library_of_another_version_is_refused(stale, monkeypatch):
    build.build()
    monkeypatch.setattr(binding, "_lib", None)
    monkeypatch.setattr(binding.C, "CDLL", lambda path: stale)
    with pytest.raises(spx.SpxError):
        spx.load_library()
