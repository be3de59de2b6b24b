"""Properties of the device code of the operators that fill gradient buffers (CPU
only: compiles their sources to AMDGPU assembly with the library's own flags).

* no packed fp32 arithmetic (the library is built without it);
* fp32 subnormals are kept, as the checkpoints' small steps need;
* no register spills and no private memory;
* the weight gradient's products are bf16 matrix instructions on operands that
  transposing LDS reads deliver;
* results are stored through the hardware's bf16 conversion.
"""
import importlib.util
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1909_08029_amd", "csrc")
SOURCES = ["rip_embed", "rip_ckpt", "rip_wgrad", "rip_loss"]


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    spec = importlib.util.spec_from_file_location(
        "rip_build", os.path.join(ROOT, "paper_1909_08029_amd", "build.py"))
    b = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(b)
    flags = [f for f in b.COMMON if f not in ("-fPIC", "-shared")]
    out = tmp_path_factory.mktemp("asm")
    jobs = [subprocess.Popen(
        [b.HIPCC, *flags, "--cuda-device-only", "-S", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
         "-x", "hip", os.path.join(CSRC, s + ".hip"), "-o", str(out / (s + ".s"))],
        stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for s in SOURCES]
    for s, j in zip(SOURCES, jobs):
        text, _ = j.communicate(timeout=600)
        assert j.returncode == 0, (s, text)
    return {s: (out / (s + ".s")).read_text() for s in SOURCES}


@pytest.mark.parametrize("source", SOURCES)
def test_arithmetic_and_registers(asm, source):
    text = asm[source]
    assert not re.search(r"^\s+v_pk_(add|mul|fma)_f32", text, flags=re.M)
    assert set(re.findall(r"\.amdhsa_float_denorm_mode_32\s+(\d+)", text)) == {"3"}
    assert set(re.findall(r"\.vgpr_spill_count:\s+(\d+)", text)) == {"0"}
    assert set(re.findall(r"\.private_segment_fixed_size:\s+(\d+)", text)) == {"0"}
    assert "v_cvt_pk_bf16_f32" in text


def test_matrix_instructions(asm):
    text = asm["rip_wgrad"]
    assert "v_mfma_f32_32x32x16_bf16" in text and "ds_read_b64_tr_b16" in text
    assert not re.findall(r"v_mfma_(?!f32_32x32x16_bf16)\w+", text)
