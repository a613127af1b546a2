"""The tables of attention's tile kernels, on the CPU under AddressSanitizer and UndefinedBehaviorSanitizer."""
import os
import subprocess

from conftest import ROOT


def test_tables_hold_every_pair_once(tmp_path):
    csrc, exe = os.path.join(ROOT, "paper_1606_07676_amd", "csrc"), str(tmp_path / "tables")
    subprocess.check_call(["g++", "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan",
                           "-static-libubsan", "-I", csrc, "-I", os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "tile_tables_driver.cpp"),
                           os.path.join(csrc, "iso_plan.cpp"), "-o", exe])
    # the sanitizer runtimes are linked statically: a preloaded library may then come first
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0")
    out = subprocess.run([exe], env=env, stdout=subprocess.PIPE, stderr=subprocess.PIPE, text=True, timeout=600)
    assert out.returncode == 0, (out.returncode, out.stdout[-2000:], out.stderr[-2000:])
    assert "tables ok" in out.stdout
