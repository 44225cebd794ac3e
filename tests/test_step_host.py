"""The C-ABI layer of xattn_prefill, xattn_rope_kvcache and xbeam_logprobs on the CPU: csrc/xattn_step_api.cpp built with g++ against a
stand-in for the HIP runtime and the launches (tests/host/step_main.cpp)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_14686_amd", "csrc")
SOURCES = [os.path.join(ROOT, "tests", "host", "step_main.cpp")] + \
    [os.path.join(CSRC, f) for f in ("xattn_api.cpp", "xattn_step_api.cpp", "xattn_error.cpp")]


def test_workspaces_axes_and_cuts(tmp_path):
    exe = os.path.join(str(tmp_path), "step_host")
    res = subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-pthread", "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                          "-fsanitize=undefined", "-fno-sanitize-recover=all"] + SOURCES + ["-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and "all scenarios ran" in run.stdout, run.stdout + run.stderr
