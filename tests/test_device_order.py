"""The built device code of the distillation calls: no floating-point atomics, whose order the results would depend on."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_07409_amd import binding as B

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"


@pytest.mark.skipif(not os.path.exists(OBJDUMP), reason="no llvm-objdump")
def test_no_float_atomics_in_distillation(tmp_path):
    lib = shutil.copy(B.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([OBJDUMP, "--offloading", lib], cwd=tmp_path, check=True, capture_output=True)
    kernels, found = set(), {}
    for o in sorted(p for p in tmp_path.iterdir() if "gfx950" in p.name):
        name = "?"
        with subprocess.Popen([OBJDUMP, "-d", "--no-show-raw-insn", o], stdout=subprocess.PIPE, text=True) as p:
            for line in p.stdout:
                m = re.match(r"[0-9a-f]+ <(.+)>:", line)
                if m:
                    name = m[1]
                    if "k_head_" in name or "k_distill_" in name:
                        kernels.add(name)
                elif name in kernels and re.search(r"\t(ds|global_atomic|buffer_atomic)\w*add\w*_(f32|f16|bf16|f64)", line):
                    found[name] = line.strip()
        assert p.returncode == 0
    assert len(kernels) > 15, kernels
    assert not found, found
