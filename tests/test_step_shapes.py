"""Launch shapes of the operators around decode attention at the ends of their ranges, on the CPU (tests/host/step_shapes_main.cpp)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_threads_of_the_largest_calls(tmp_path):
    exe = os.path.join(str(tmp_path), "step_shapes")
    res = subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-fsanitize=undefined",
                          "-fno-sanitize-recover=all", os.path.join(ROOT, "tests", "host", "step_shapes_main.cpp"), "-o", exe],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and "all scenarios ran" in run.stdout, run.stdout + run.stderr
