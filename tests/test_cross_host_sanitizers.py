"""Cross attention's plan and launch rules under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import shutil
import subprocess

import pytest

from paper_2503_07680_amd import build as B

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plan_and_rules_are_clean_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "host_sanitize_cross")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
                    "-fno-sanitize-recover=all", "-I", B.INCLUDE, "-I", B.CSRC, os.path.join(HERE, "host_sanitize_cross_main.cpp"),
                    os.path.join(B.CSRC, "plan.cpp"), "-o", exe], check=True, stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0")
    r = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, env=env, timeout=300)
    assert r.returncode == 0 and r.stdout.decode().strip().endswith("ok"), r.stdout.decode()[-3000:]
