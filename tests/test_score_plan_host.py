"""What the scoring calls would launch, on the CPU (no GPU): score_plan_check.cpp holds 1500 random
scoring forwards, and with plan_check.cpp's own checks 600 random gradients with an entropy term, to
covering the problem once inside the workspace."""
import os
import shutil
import subprocess

import pytest

import paper_2609_14306_amd as vp

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CXX = shutil.which("g++")

pytestmark = [pytest.mark.skipif(CXX is None, reason="no g++"),
              pytest.mark.skipif(not os.path.exists(vp.LIB_PATH),
                                 reason="libvpce.so not built (run __graft_entry__.build())")]


def test_scoring_plans_cover_the_problem(tmp_path):
    with open(os.path.join(HERE, "plan_check.cpp")) as f:
        text = f.read()
    for old, new in [("../paper_2609_14306_amd", os.path.join(ROOT, "paper_2609_14306_amd")),
                     ("vp_ce_backward(&pr, H, W.data(), (const int64_t*)64, (const float*)64, (const float*)64,",
                      "vp_score_backward(&pr, H, W.data(), (const int64_t*)64, (const float*)64, (const float*)64, "
                      "(const float*)64, (const float*)64,"),
                     ("int main(", "static int plan_check_main(")]:
        assert text.count(old) == 1, old
        text = text.replace(old, new)
    copy, exe = str(tmp_path / "plan_check_score.cpp"), str(tmp_path / "score_plan_check")
    with open(copy, "w") as f:
        f.write(text)
    subprocess.run([CXX, "-D__HIP_PLATFORM_AMD__", "-std=c++17", "-O1", "-Wall", f'-DPLAN_CHECK="{copy}"',
                    "-I", os.path.join(ROOT, "include"), "-I", "/opt/rocm/include",
                    os.path.join(HERE, "score_plan_check.cpp"), "-o", exe, vp.LIB_PATH,
                    "-L/opt/rocm/lib", "-lamdhip64",
                    f"-Wl,-rpath,/opt/rocm/lib:{os.path.dirname(vp.LIB_PATH)}"], check=True)
    for seed in ("3", "8"):
        out = subprocess.run([exe, seed], stdout=subprocess.PIPE, text=True, timeout=120)
        assert out.returncode == 0, out.stdout
        print(out.stdout)
