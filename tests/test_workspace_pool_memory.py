"""The scratch-buffer pool when the host's memory runs out (CPU only, fake backend): an error code, no exception."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_no_host_memory_is_an_error_code(tmp_path):
    src = os.path.join(ROOT, "tests", "cpp", "workspace_pool_memory_test.cpp")
    exe = str(tmp_path / "workspace_pool_memory_test")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-pthread", "-o", exe, src])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "ok", out.stdout + out.stderr
