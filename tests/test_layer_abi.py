"""include/ob_layer.h without a device: it is plain C, its structures and constants are the binding's, every call it declares is
exported, and what the host can refuse it refuses."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ob():
    import paper_2104_06069_amd as ob
    if not os.path.exists(ob.lib_path()):
        from paper_2104_06069_amd.build import build
        build()
    return ob


def test_every_declared_call_is_exported_and_bound(ob):
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ob_layer.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ob_(?:norm|linear8|clip)_[a-z0-9_]+)\s*\(", src)))
    assert len(names) == 22
    for name in names:
        call = getattr(ob.lib(), name)
        assert call.argtypes is not None, name
        declared = re.search(re.escape(name) + r"\s*\(([^)]*)\)", src).group(1)
        assert len(call.argtypes) == len(declared.split(",")), name


def test_layouts_and_constants(ob, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    structs = {"ob_norm_config": ob.ObNormConfig, "ob_linear8_config": ob.ObLinear8Config, "ob_clip_config": ob.ObClipConfig}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ob_layer.h"', 'int main(void) {']
    want = []
    for cname, ct in structs.items():
        lines.append(f'  printf("%zu\\n", sizeof({cname}));')
        want.append(C.sizeof(ct))
        for f, _ in ct._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({cname}, {f}));')
            want.append(getattr(ct, f).offset)
    for c in ("OB_E4M3", "OB_E5M2", "OB_BLOCK_ROWS", "OB_BLOCK_SQUARE", "OB_LINEAR8_FEW_ROWS"):
        lines.append(f'  printf("%d\\n", (int){c});')
        want.append(getattr(ob, c))
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    assert [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()] == want


def test_create_refuses(ob):
    L, out = ob.lib(), C.c_void_p()
    nan, inf = float("nan"), float("inf")
    good = dict(n=64, dtype=ob.OB_BF16, res_dtype=ob.OB_BF16, weight_dtype=ob.OB_F32, eps=1e-6)
    for field, value in (("n", 0), ("n", 16385), ("dtype", 3), ("res_dtype", ob.OB_F16), ("weight_dtype", -1), ("eps", -1.0), ("eps", nan), ("eps", inf)):
        assert L.ob_norm_create(C.byref(ob.ObNormConfig(**dict(good, **{field: value}))), C.byref(out)) == -2 and not out.value, field
    for k, n, rows in ((0, 1, 1), (1, 0, 1), (1 << 21, 1, 1), (1, 1 << 21, 1), (1, 1, -1), (1, 1, (1 << 22) + 1)):
        assert L.ob_linear8_create(C.byref(ob.ObLinear8Config(k, n, rows)), C.byref(out)) == -2 and not out.value
    for offs, eps, scale in (([0, 5, 3], 0, 1), ([1, 5], 0, 1), ([0, 5], -1, 1), ([0, 5], nan, 1), ([0, 5], 0, 0), ([0, 5], 0, nan), ([0, 5], 0, inf),
                             ([0, (1 << 35) + 1], 0, 1)):
        cfg = ob.ObClipConfig(len(offs) - 1, (C.c_int64 * len(offs))(*offs), eps, scale)
        assert L.ob_clip_create(C.byref(cfg), C.byref(out)) == -2 and not out.value, (offs, eps, scale)
    assert L.ob_clip_create(C.byref(ob.ObClipConfig(0, (C.c_int64 * 1)(0), 0, 1)), C.byref(out)) == -2
    assert L.ob_clip_create(C.byref(ob.ObClipConfig(1, None, 0, 1)), C.byref(out)) == -1
    for create, cfg in ((L.ob_norm_create, ob.ObNormConfig(**good)), (L.ob_linear8_create, ob.ObLinear8Config(1, 1, 1))):
        assert create(None, C.byref(out)) == -1 and create(C.byref(cfg), None) == -1
    assert L.ob_clip_create(None, C.byref(out)) == -1


def test_null_contexts(ob):
    L = ob.lib()
    one = C.c_float(0)
    p = C.addressof(one)
    assert L.ob_norm_forward(None, p, 1, None, 0, None, 1, None, 0, p, 1, None, 0, None, 0, 0, None, None) == -1
    assert L.ob_norm_backward(None, p, 1, p, 1, p, None, None, 0, 1, p, 1, None, 0, None) == -1
    assert L.ob_linear8_quantize(None, p, 0, 1, 1, 1, 0, 0, 0, p, 128, p, 4, None, 0, None, 0, None) == -1
    assert L.ob_linear8_forward(None, p, 128, p, 4, 0, p, 128, p, 4, 1, p, 1, 0, None) == -1
    assert L.ob_linear8_forward_few(None, p, 0, 1, 0, p, 128, p, 4, 1, p, 1, 0, None) == -1
    assert L.ob_linear8_input_grad(None, p, 128, p, 4, 0, p, 128, p, 4, 1, p, 1, 0, None) == -1
    assert L.ob_linear8_weight_grad(None, p, 128, p, 4, 0, p, 128, p, 4, 1, p, 1, 0, 0, None) == -1
    assert L.ob_clip_norm(None, p, 0, p, None, None) == -1
    assert L.ob_clip_apply(None, p, 0, p, 1.0, p, 0, None) == -1
    assert L.ob_clip_norm_apply(None, p, 0, 1.0, p, None, p, 0, None) == -1
    for kind in ("norm", "linear8", "clip"):
        getattr(L, f"ob_{kind}_destroy")(None)
        assert getattr(ob, f"ob_{kind}_workspace_bytes")(None) == 0
        assert getattr(L, f"ob_{kind}_last_hip_error")(None) == b""
