"""The paged cache's calls on the host, once a batch is set (paged_calls.cpp: launches that do nothing)."""
import os
import subprocess


def test_calls(tmp_path):
    """Under the address and undefined-behaviour sanitizers."""
    here = os.path.dirname(os.path.abspath(__file__))
    exe = str(tmp_path / "paged_calls")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-D__HIP_PLATFORM_AMD__", "-I", rocm + "/include", os.path.join(here, "paged_calls.cpp"), "-o", exe],
                   check=True)
    r = subprocess.run([exe], capture_output=True, text=True, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0 and r.stdout.split() == ["ok"], r.stdout + r.stderr
