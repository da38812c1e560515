"""The calls of shared prefixes, attention weights and kept tokens without a GPU: the struct's layout against the
header, and the refusals that need no device."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lv():
    from paper_2606_22983_gb300 import build
    build()
    from paper_2606_22983_gb300 import lv as module
    return module


def test_struct_layout(lv, tmp_path):
    src = tmp_path / "layout.c"
    names = [n for n, _ in lv.lv_weights._fields_]
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"lv.h\"\nint main(void) {\n"
                   '  printf("size %zu\\n", sizeof(lv_weights));\n' + "".join(
                       f'  printf("{n} %zu\\n", offsetof(lv_weights, {n}));\n' for n in names) + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    out = dict(line.split() for line in
               subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(out["size"]) == ctypes.sizeof(lv.lv_weights)
    for n in names:
        assert int(out[n]) == getattr(lv.lv_weights, n).offset, n


def test_null_arguments(lv):
    L = lv.lib()
    q, w = lv.lv_heads(), lv.lv_weights()
    bad = lv.LV_ERR_INVALID
    assert L.lv_batch_share(None, 1) == bad
    assert L.lv_batch_plan_shared(None, None, None, None, None, None, 0, 0, 0, None) == bad
    assert L.lv_attention_weights(None, 0, ctypes.byref(q), None, ctypes.byref(w), 0, 1.0, None) == bad
    assert L.lv_select_kept(None, ctypes.byref(w), None, None, 0, 0, 0, None, 1, None) == bad
    assert L.lv_kv_compact(None, None, None, 0, None, 1, None, None, None) == bad
    assert L.lv_session_truncate(None, None, None, 0, None) == bad
    with pytest.raises(lv.LvError) as e:
        lv.lv_session_truncate(None, None, None, 0, 0)
    assert e.value.status == bad
