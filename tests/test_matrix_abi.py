"""include/ob_matrix.h without a device: it is plain C, its structures and constants are the binding's, every call it declares
is exported, and what the host can refuse it refuses."""
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
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "ob_matrix.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ob_(?:experts|muon)_[a-z_]+)\s*\(", src)))
    assert len(names) == 13
    for name in names:
        assert getattr(ob.lib(), name).argtypes is not None, name


def test_layouts_and_constants(ob, tmp_path):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    structs = {"ob_experts_config": ob.ObExpertsConfig, "ob_muon_config": ob.ObMuonConfig}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "ob_matrix.h"', 'int main(void) {']
    want = []
    for cname, ct in structs.items():
        lines.append(f'  printf("%zu\\n", sizeof({cname}));')
        want.append(C.sizeof(ct))
        for f, _ in ct._fields_:
            lines.append(f'  printf("%zu\\n", offsetof({cname}, {f}));')
            want.append(getattr(ct, f).offset)
    for c in ("OB_EXPERTS_KN", "OB_EXPERTS_NK"):
        lines.append(f'  printf("%d\\n", (int){c});')
        want.append(getattr(ob, c))
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]) + "\n")
    subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    assert [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout.split()] == want


def test_experts_create_refuses(ob):
    L, out = ob.lib(), C.c_void_p()
    assert L.ob_experts_create(None, C.byref(out)) == -1
    good = dict(num_groups=4, dtype=ob.OB_BF16, w_layout=0, reserved=0, k=64, n=32, max_rows=100, w_stride=0)
    for field, value in (("num_groups", 0), ("num_groups", 65537), ("dtype", ob.OB_F32), ("dtype", 7), ("w_layout", 2), ("reserved", 1), ("k", 0),
                         ("k", 1 << 21), ("n", -1), ("max_rows", -1), ("max_rows", 1 << 31), ("w_stride", 64 * 32 - 1), ("w_stride", -1)):
        cfg = ob.ObExpertsConfig(**dict(good, **{field: value}))
        assert L.ob_experts_create(C.byref(cfg), C.byref(out)) == -2 and not out.value, field
    assert L.ob_experts_create(C.byref(ob.ObExpertsConfig(**good)), None) == -1


def test_muon_create_refuses(ob):
    L, out = ob.lib(), C.c_void_p()
    offs, rows, coef = (C.c_int64 * 3)(0, 12, 20), (C.c_int64 * 2)(3, 0), (C.c_float * 3)(3.4, -4.8, 2.0)
    scale = (C.c_float * 2)(1.0, float("inf"))

    def create(**kw):
        d = dict(num_layers=2, layer_offsets=offs, layer_rows=rows, layer_scale=None, coefficients=coef, num_coefficients=1, steps=5, eps=1e-7,
                 beta=0.9, weight_decay=0.0, nesterov=1, precision=ob.OB_F32)
        cfg = ob.ObMuonConfig(**dict(d, **kw))
        return L.ob_muon_create(C.byref(cfg), C.byref(out))
    assert L.ob_muon_create(None, C.byref(out)) == -1
    for field in ("layer_offsets", "layer_rows", "coefficients"):
        assert create(**{field: None}) == -1, field
    nan = float("nan")
    for field, value in (("num_layers", 0), ("steps", 0), ("steps", 65), ("num_coefficients", 0), ("num_coefficients", 6), ("eps", -1.0), ("eps", nan),
                         ("beta", 1.0), ("beta", -0.1), ("beta", nan), ("weight_decay", -1.0), ("precision", ob.OB_BF16), ("layer_scale", scale),
                         ("coefficients", (C.c_float * 3)(1.0, nan, 0.0)), ("layer_rows", (C.c_int64 * 2)(5, 0)), ("layer_rows", (C.c_int64 * 2)(-3, 0)),
                         ("layer_rows", (C.c_int64 * 2)(0, 0)), ("layer_offsets", (C.c_int64 * 3)(0, 24, 20)), ("layer_offsets", (C.c_int64 * 3)(1, 12, 20))):
        assert create(**{field: value}) == -2 and not out.value, field
    assert create(layer_offsets=(C.c_int64 * 3)(0, 1 << 21, 1 << 21), layer_rows=(C.c_int64 * 2)(1, 0)) == -6


def test_null_contexts(ob):
    L = ob.lib()
    one = C.c_float(0)
    p = C.addressof(one)
    assert L.ob_experts_forward(None, p, 1, p, p, 1, p, 1, 1, None) == -1
    assert L.ob_experts_input_grad(None, p, 1, p, p, 1, p, 1, 1, None) == -1
    assert L.ob_experts_weight_grad(None, p, 1, p, 1, p, 1, p, 1, 0, None) == -1
    assert L.ob_muon_orthogonalize(None, p, 0, p, 0, None) == -1
    assert L.ob_muon_step(None, p, p, p, 0, 1.0, 1.0, None, 0, None) == -1
    L.ob_experts_destroy(None)
    L.ob_muon_destroy(None)
    assert ob.ob_muon_workspace_bytes(None) == 0 and ob.ob_experts_workspace_bytes(None) == 0
