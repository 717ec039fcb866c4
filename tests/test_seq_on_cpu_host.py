"""The losses of whole sequences on the CPU (no GPU): seq_on_cpu.cpp compiles the C entries and the
kernels of vpce_seq.hip as they stand, with the header under cpu_hip/ in place of HIP's, and runs
them over arrays that end or begin at a page that faults."""
import os
import platform
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CXX = shutil.which("g++")

pytestmark = [pytest.mark.skipif(CXX is None, reason="no g++"),
              pytest.mark.skipif(platform.machine() != "x86_64", reason="cpu_hip switches stacks of x86-64")]


@pytest.fixture(scope="module")
def seq_on_cpu(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("seq") / "seq_on_cpu")
    subprocess.run([CXX, "-std=c++17", "-O2", "-w", "-I", os.path.join(HERE, "cpu_hip"),
                    "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2609_14306_amd", "csrc"),
                    "-x", "c++", os.path.join(HERE, "seq_on_cpu.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("mode", ["ordered", "disordered", "longer", "no tokens", "runs"])
def test_kernels_on_the_cpu(seq_on_cpu, mode):
    out = subprocess.run([seq_on_cpu, mode], stdout=subprocess.PIPE, text=True, timeout=240)
    assert out.returncode == 0, out.stdout
