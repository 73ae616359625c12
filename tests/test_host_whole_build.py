"""The library's launchers are strong symbols, and a build that is meant to be whole does not link without one."""
import os
import subprocess

from paper_2410_14312_amd import binding
from tests.test_host_sanitizers import ROOT

LAUNCHERS = ["rotary", "norm_join_forward", "norm_join_backward", "norm_join_part_elems", "distill", "distill_workspace_elems", "check_distill"]


def test_launchers_are_strong_symbols():
    binding.load_library()
    out = subprocess.run(["nm", "-DC", "--defined-only", os.path.join(ROOT, "paper_2410_14312_amd", "libtmps.so")], capture_output=True, text=True)
    assert out.returncode == 0, out.stderr
    kinds = {line.split(None, 2)[2].split("(")[0]: line.split(None, 2)[1] for line in out.stdout.splitlines()}
    assert [kinds["tmps::" + n] for n in LAUNCHERS] == ["T"] * len(LAUNCHERS)


def test_a_missing_source_is_an_error_of_the_link(tmp_path):
    src = tmp_path / "main.cpp"
    src.write_text('#include "tmps.h"\nint main() { size_t s; tmps_layer_desc d = {}; tmps_stage_cfg c = {}; return tmps_stage_bytes(&d, 1, &c, &s, &s, &s, &s); }\n')
    cmd = ["g++", "-std=c++17", "-DTMPS_WHOLE", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-pthread", str(src),
           os.path.join(ROOT, "tests/host/kernel_stubs.cpp"), os.path.join(ROOT, "paper_2410_14312_amd/csrc/stage.cpp"), "-o", str(tmp_path / "main")]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode != 0 and all("undefined reference to `tmps::%s(" % n in r.stderr for n in LAUNCHERS if n != "check_distill"), r.stderr
