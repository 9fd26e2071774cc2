"""What the compiler made of the matrix operators' kernels, which results show rarely or not at all: built for gfx950, no device."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def text(tmp_path_factory):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not (os.path.exists(hipcc) or shutil.which(hipcc)):
        pytest.skip("no hipcc")
    asm = tmp_path_factory.mktemp("asm") / "m.s"
    subprocess.run([hipcc, "-O3", "--offload-arch=gfx950", "--offload-device-only", "-S", "-std=c++17", "-ffp-contract=off", "-Xclang",
                    "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "paper_2104_06069_amd", "csrc", "ob_matrix.hip"), "-o", str(asm)], check=True, capture_output=True)
    return asm.read_text()


def test_no_spills(text):
    counts = re.findall(r"\.name:\s+(_ZN3obm\w+).*?\.private_segment_fixed_size:\s+(\d+).*?\.sgpr_spill_count:\s+(\d+).*?\.vgpr_spill_count:\s+(\d+)",
                        text, re.S)
    assert len(counts) > 60
    assert [c for c in counts if c[1:] != ("0", "0", "0")] == []


def test_first_and_second_terms_come_from_one_number(text):
    """No product is rounded to binary16 without being rounded to binary32 first (split4)."""
    assert "v_fma_mix" not in text and "v_mad_mix" not in text


def test_no_packed_binary32(text):
    assert not re.findall(r"v_pk_(?:add|mul|fma)_f32", text)
