"""Loads straight to LDS in the device assembly: they take their place from M0, and a scalar
write of M0 needs one wait state (any instruction) before the load that reads it.  Hazards
are the source's own business where both stand in one block of inline assembly, so the
compiled code is looked at."""
import glob
import os
import re
import shutil
import subprocess

import pytest

from paper_2609_20734_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = [f for f in sorted(glob.glob(os.path.join(B.PKG, "csrc", "*.hip"))) if "load_lds" in open(f).read()]


def hazards(assembly):
    """(writes of M0, loads to LDS that directly follow one)."""
    lines = [ln.split(";")[0].strip() for ln in assembly.splitlines()]
    code = [ln for ln in lines if ln and not ln.startswith(".") and not ln.endswith(":")]
    writes = [i for i, ln in enumerate(code) if re.match(r"s_\w+\s+m0\b", ln)]
    return len(writes), [code[i + 1] for i in writes if re.match(r"(global|buffer)_load", code[i + 1]) and "lds" in code[i + 1]]


def test_the_search_finds_them():
    text = "\ts_mov_b32 m0, s4\n.Lx:\n\t;;#ASM\n\tglobal_load_lds_dwordx4 v[0:1], off\n"
    assert hazards(text) == (1, ["global_load_lds_dwordx4 v[0:1], off"])
    assert hazards(text.replace(".Lx:", "s_nop 0")) == (1, [])


@pytest.mark.parametrize("source", SOURCES, ids=os.path.basename)
def test_a_wait_state_between_m0_and_the_load(source, tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    out = str(tmp_path / "device.s")
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    res = subprocess.run([hipcc, *flags, "--cuda-device-only", "-S", "-I", os.path.join(ROOT, "include"), "-I",
                          os.path.join(B.PKG, "csrc"), source, "-o", out], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-4000:]
    writes, found = hazards(open(out).read())
    assert writes > 0 and not found, found
