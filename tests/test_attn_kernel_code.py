"""Properties of the device code of attention and AdamW (CPU only: compiles their sources
to AMDGPU assembly with the library's own flags).

* no packed fp32 arithmetic, fp32 subnormals kept;
* attention's products are matrix instructions, of bf16 on operands that transposing LDS
  reads deliver, and of fp32 for the widest heads alone;
* no private memory but for the widest fp32 heads, whose rows and sums alone take 384
  registers, and at most sixteen values of loops' surroundings in others.
"""
import importlib.util
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1909_08029_amd", "csrc")
SOURCES = ["rip_adamw", "rip_attn", "rip_attn_forward", "rip_attn_backward"]


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
        text, _ = j.communicate(timeout=900)
        assert j.returncode == 0, (s, text)
    return {s: (out / (s + ".s")).read_text() for s in SOURCES}


@pytest.mark.parametrize("source", SOURCES)
def test_arithmetic_and_registers(asm, source):
    text = asm[source]
    assert not re.search(r"^\s+v_pk_(add|mul|fma)_f32", text, flags=re.M)
    assert set(re.findall(r"\.amdhsa_float_denorm_mode_32\s+(\d+)", text)) == {"3"}
    kernels = re.findall(r"\.name:\s+(_Z\S+)\s.*?\.private_segment_fixed_size:\s+(\d+)", text, flags=re.S)
    assert kernels
    for name, private in kernels:
        if not re.search(r"(forward|dq|dkv)_kernelILi3ELi256E", name):   # (fp32, 256)
            assert int(private) <= (64 if "attn_" in source else 0), name


def test_matrix_instructions(asm):
    forms = {"v_mfma_f32_32x32x16_bf16", "v_mfma_f32_32x32x2_f32"}
    for source in ("rip_attn_forward", "rip_attn_backward"):
        assert set(re.findall(r"v_mfma_\w+", asm[source])) == forms
        assert "ds_read_b64_tr_b16" in asm[source] and "v_cvt_pk_bf16_f32" in asm[source]


def test_every_kernel_is_found_by_its_name():
    """Names that the host registers in the built library are names of its device code (one
    that is not ends the process at its first launch)."""
    data = open(os.path.join(ROOT, "paper_1909_08029_amd", "librip.so"), "rb").read()
    names = set(re.findall(rb"\0(_Z[A-Za-z0-9_$]*_kernel[A-Za-z0-9_$]*)(?=\0)", data))
    kernels = set(re.findall(rb"\0(_Z[A-Za-z0-9_$]*_kernel[A-Za-z0-9_$]*)\.kd(?=\0)", data))
    assert len(kernels) > 100
    stubs = {n for n in names if b"__device_stub__" in n}
    assert names - stubs == kernels, sorted(names - stubs ^ kernels)[:4]
