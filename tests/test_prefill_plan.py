"""How xattn_prefill's work is cut, on the CPU: csrc/xattn_prefill_plan.h in tests/host/prefill_plan_main.cpp."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_bounds_and_parts(tmp_path):
    exe = os.path.join(str(tmp_path), "prefill_plan")
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                          os.path.join(ROOT, "tests", "host", "prefill_plan_main.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert run.returncode == 0 and "all batches ran" in run.stdout, run.stdout + run.stderr
