"""What the compiler made of the kernels of a layer's operators, which results show rarely or not at all: built for gfx950, no device."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", params=("ob_norm", "ob_linear8", "ob_clip"))
def text(request, tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    asm = tmp_path_factory.mktemp("asm") / "m.s"
    subprocess.run([hipcc, "-O3", "--offload-arch=gfx950", "--offload-device-only", "-S", "-std=c++17", "-ffp-contract=off", "-Xclang",
                    "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "paper_2104_06069_amd", "csrc", request.param + ".hip"), "-o", str(asm)], check=True, capture_output=True)
    return request.param, asm.read_text()


def test_no_memory_for_spills_and_no_packed_binary32(text):
    name, text = text
    counts = re.findall(r"\.name:\s+(_ZN3obl\w+).*?\.private_segment_fixed_size:\s+(\d+).*?\.vgpr_spill_count:\s+(\d+)", text, re.S)
    assert len(counts) >= {"ob_norm": 50, "ob_linear8": 40, "ob_clip": 20}[name]
    assert [c for c in counts if c[1:] != ("0", "0")] == []
    assert not re.findall(r"v_pk_(?:add|mul|fma)_f32", text)


def function(text, part):
    start = re.search(r"^(_ZN3obl\w*" + part + r"\w*):", text, re.M)
    return text[start.end():text.index(".Lfunc_end", start.end())]


@pytest.mark.parametrize("variant,stores,products", [("ILi0ELi2", 32, 64), ("ILi1ELi1", 32, 64), ("ILi0ELi0", 64, 256), ("ILi1ELi0", 64, 256), ("ILi0ELi3", 64, 256)])
def test_stores_are_counted_with_the_loads(text, variant, stores, products):
    """k_product8_flow waits for loads by how many loads and stores are behind them: a tile's stores are as many whatever part of the tile exists, in
    one piece without branches, its loop has 18 loads a slab, and nothing else goes to memory."""
    name, text = text
    if name != "ob_linear8":
        pytest.skip("of the products")
    code = [line.split(";")[0].strip() for line in function(text, "k_product8_flow" + variant).split("\n")]
    code = [line for line in code if line]
    at = [i for i, line in enumerate(code) if line.startswith("buffer_store")]
    assert len(at) == stores
    assert not [line for line in code[at[0]:at[-1]] if line.startswith((".LBB", "s_cbranch", "s_branch"))]
    old = [line for line in code if line.startswith("buffer_load") and "lds" not in line]      # (what results are added to: waited for, and with it all before)
    assert len(old) == (64 if variant.endswith("Li3") else 0)
    assert len([line for line in code if line.startswith("v_mfma")]) == 2 * products
    assert len([line for line in code if line.startswith("buffer_load") and "lds" in line]) == 36 + 2 * 18
    assert not [line for line in code if line.startswith(("scratch", "global_", "flat_"))]


def test_a_tensors_sum_is_there_before_the_arrival(text):
    """k_clip_norm counts workgroups that are done, from a single thread: each of the four wavefronts that store a tensor's sum waits for
    that store before the barrier that thread is behind, and the count follows the barrier."""
    name, text = text
    if name != "ob_clip":
        pytest.skip("of the clipping")
    code = [line.split(";")[0].strip() for line in function(text, "k_clip_norm").split("\n")]
    arrival = next(i for i, line in enumerate(code) if line.startswith("global_atomic_add"))
    barrier = max(i for i, line in enumerate(code[:arrival]) if line.startswith("s_barrier"))
    stores = [i for i, line in enumerate(code[:barrier]) if line.startswith("global_store")]
    assert stores
    assert [line for line in code[stores[-1]:barrier] if re.match(r"s_waitcnt vmcnt\(0\)", line)]
    after = [line for line in code[stores[0]:stores[-1]] if line.startswith("s_cbranch")]      # (around the norm's store, where there is none to write)
    for line in after:
        label = line.split()[-1] + ":"
        assert code[:barrier].index(label) <= next(i for i in range(stores[-1], barrier) if re.match(r"s_waitcnt vmcnt\(0\)", code[i])), line


@pytest.mark.parametrize("variant,stores,products", [("ILi0ELi1", 32, 64), ("ILi1ELi2", 32, 64), ("ILi1ELi3", 64, 256)])
def test_the_other_variants_count_the_same(text, variant, stores, products):
    """The results' types and formats that the list above leaves out."""
    test_stores_are_counted_with_the_loads(text, variant, stores, products)
