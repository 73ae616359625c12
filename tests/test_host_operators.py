"""The stage executor's host code with rotary positions, norm joins, norms without a mean and distillation, built with g++ under AddressSanitizer and
UndefinedBehaviorSanitizer (tests/host/sanitize_operators.cpp); and a build without their launchers, which links and refuses them."""
import subprocess

from tests.test_host_sanitizers import build, run_clean

SOURCES = ["tests/host/sanitize_operators.cpp", "tests/host/operator_stubs.cpp", "tests/host/kernel_stubs.cpp", "paper_2410_14312_amd/csrc/stage.cpp"]


def test_layers_are_clean_under_sanitizers(tmp_path_factory):
    run_clean(build(tmp_path_factory, "sanitize_operators", SOURCES))


def test_a_build_without_them_refuses(tmp_path_factory):
    src = tmp_path_factory.mktemp("without") / "main.cpp"
    src.write_text("""#include "tmps.h"
#include <stdio.h>
int main() {
    tmps_stage_cfg c = {1, 2, 2, 2, 0, 0, 0.1f, 0.9f};
    tmps_layer_desc r = {TMPS_ROTARY, {4, 8, 2}, 0}, n = {TMPS_LAYERNORM, {8, 1}, TMPS_FLAG_RMS}, j[2] = {{TMPS_LINEAR, {8, 8, 0, 1}, 0}, {TMPS_NORMJOIN, {8, 1, 2}, 0}};
    tmps_layer_desc d[2] = {{TMPS_LINEAR, {8, 8, 0, 1}, 0}, {TMPS_DISTILL, {8, 1, 2, 0x3f800000, 0x3f800000}, 0}};
    tmps_stage_cfg last = c;
    last.is_last = 1;
    size_t s;
    printf("%d %d %d %d\\n", tmps_stage_bytes(&r, 1, &c, &s, &s, &s, &s), tmps_stage_bytes(&n, 1, &c, &s, &s, &s, &s), tmps_stage_bytes(j, 2, &c, &s, &s, &s, &s),
           tmps_stage_bytes(d, 2, &last, &s, &s, &s, &s));
}
""")
    import os
    from tests.test_host_sanitizers import ROOT
    exe = str(src.parent / "without")
    cmd = ["g++", "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-pthread", str(src),
           os.path.join(ROOT, "tests/host/kernel_stubs.cpp"), os.path.join(ROOT, "paper_2410_14312_amd/csrc/stage.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert subprocess.run([exe], capture_output=True, text=True, timeout=60).stdout.split() == ["-7"] * 4
