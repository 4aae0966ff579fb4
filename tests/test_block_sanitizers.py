"""The host code of the decoder block's operators under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU): plans, workspace layouts, grids and argument checks, linked
into a driver that stubs out the kernel launchers."""
import os
import subprocess

from tests.test_sanitizers import CSRC, ROOT, SAN, _env, pytestmark  # noqa: F401


def test_plans_grids_and_entry_checks_are_clean(tmp_path):
    exe = str(tmp_path / "host_block")
    subprocess.run(
        ["g++", "-std=c++17", "-g", "-O1", *SAN, "-D__HIP_PLATFORM_AMD__",
         "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
         os.path.join(ROOT, "tests", "sanitize", "host_block.cpp"),
         os.path.join(CSRC, "gbla_plan.cpp"), os.path.join(CSRC, "gbla_delta_plan.cpp"),
         os.path.join(CSRC, "gbla_delta_api.cpp"), os.path.join(CSRC, "gbla_norm_api.cpp"), "-o", exe],
        check=True)
    run = subprocess.run([exe], capture_output=True, text=True, env=_env(), timeout=300)
    assert run.returncode == 0, run.stderr[-4000:]
    assert "host block ok" in run.stdout
    assert "runtime error" not in run.stderr
