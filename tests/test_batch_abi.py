"""The serving-step calls of the C ABI without a GPU: struct layouts against the header, and the
refusals that need no device."""
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


def test_struct_layouts(lv, tmp_path):
    src = tmp_path / "layout.c"
    fields = {T: [n for n, _ in getattr(lv, T)._fields_] for T in ("lv_batch_desc", "lv_heads")}
    src.write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"lv.h\"\nint main(void) {\n" + "".join(
        f'  printf("{T} %zu\\n", sizeof({T}));\n' + "".join(
            f'  printf("{T}.{n} %zu\\n", offsetof({T}, {n}));\n' for n in names) for T, names in fields.items()) +
        '  printf("types %d %d %d\\n", LV_BF16, LV_F16, LV_F32);\n  return 0;\n}\n')
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o",
                    str(exe)], check=True)
    out = dict(line.split(" ", 1) for line in
               subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.splitlines())
    for T, names in fields.items():
        struct = getattr(lv, T)
        assert int(out[T]) == ctypes.sizeof(struct)
        for n in names:
            assert int(out[f"{T}.{n}"]) == getattr(struct, n).offset, (T, n)
    assert out["types"] == f"{lv.LV_BF16} {lv.LV_F16} {lv.LV_F32}"


def test_null_arguments(lv):
    L = lv.lib()
    h, d, x = ctypes.c_void_p(7), lv.lv_batch_desc(), lv.lv_heads()
    assert L.lv_batch_create(None, ctypes.byref(d), ctypes.byref(h)) == lv.LV_ERR_INVALID
    assert not h.value                      # cleared, as a refused creation leaves it
    assert L.lv_batch_create(None, None, None) == lv.LV_ERR_INVALID
    assert L.lv_batch_destroy(None, None) == lv.LV_ERR_INVALID
    assert L.lv_batch_plan(None, None, None, None, 0, 0, 0, None) == lv.LV_ERR_INVALID
    assert L.lv_kv_write(None, 0, ctypes.byref(x), ctypes.byref(x), None) == lv.LV_ERR_INVALID
    assert L.lv_attention(None, 0, ctypes.byref(x), ctypes.byref(x), None, 1.0, None) == lv.LV_ERR_INVALID
    with pytest.raises(lv.LvError) as e:
        lv.lv_batch_destroy(None, 0)
    assert e.value.status == lv.LV_ERR_INVALID
