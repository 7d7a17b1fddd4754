"""The structures of the calls in front of the head, as a C compiler lays them out and as the binding passes them."""
import os
import subprocess

import pytest

from paper_2510_11062_amd import api

INCLUDE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
MIRRORS = {"at_grpo_rows": api._Rows, "at_grpo_rope": api._Rope, "at_grpo_norm_rope": api._NormRope, "at_grpo_kv": api._KV}


@pytest.mark.parametrize("compiler,std", [("gcc", "-std=c99"), ("g++", "-std=c++17")])
def test_struct_layout(tmp_path, compiler, std):
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "at_grpo.h"', "int main(void) {"]
    want = []
    for name, mirror in MIRRORS.items():
        lines.append(f'  printf("%zu\\n", sizeof({name}));')
        want.append(api.C.sizeof(mirror))
        for field in (f[0] for f in mirror._fields_):
            lines.append(f'  printf("%zu\\n", offsetof({name}, {field}));')
            want.append(getattr(mirror, field).offset)
    src = tmp_path / ("layout.c" if compiler == "gcc" else "layout.cpp")
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    exe = tmp_path / "layout"
    subprocess.run([compiler, std, "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    assert [int(x) for x in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()] == want


def test_enumerators_of_the_binding(tmp_path):
    names = ["AT_GRPO_CALL_QK_NORM_ROPE_BWD"]
    src = tmp_path / "e.c"
    src.write_text('#include <stdio.h>\n#include "at_grpo.h"\nint main(void) {\n' + "".join(f'  printf("%d\\n", (int){n});\n' for n in names) + "  return 0;\n}\n")
    exe = tmp_path / "e"
    subprocess.run(["gcc", "-std=c99", "-I", INCLUDE, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split() == [str(api.CALL_QK_NORM_ROPE_BWD)]


@pytest.mark.parametrize("call", ["qk_norm_rope", "qk_norm_rope_bwd", "kv_append", "prefix_attention"])
def test_without_the_extension_a_call_says_so(monkeypatch, call):
    import torch
    monkeypatch.setattr(api, "_binding", None)

    def missing():
        raise api.AtGrpoError("extension not built")

    monkeypatch.setattr(api, "load_binding", missing)
    x = torch.zeros(1, 1, 8)
    args = {"qk_norm_rope": (x, x, None, None), "qk_norm_rope_bwd": (x, x, x, x, None, None), "kv_append": (None, x, x, x, None), "prefix_attention": (None, x)}
    with pytest.raises(api.AtGrpoError, match="not built"):
        getattr(api, "at_grpo_" + call)(*args[call])
