"""The operators' C ABI used from plain C (tests/c/ops_c.c): compiles as C11
against gockpt_ops.h alone, and on the GPU agrees with its own sums on the host."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2511_07035_amd")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def _build(out_dir) -> str:
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    exe = os.path.join(str(out_dir), "ops_c")
    cmd = [cc, "-std=c11", "-O2", "-Wall", "-Werror", "-ffp-contract=off", "-D__HIP_PLATFORM_AMD__",
           f"-I{ROCM}/include", f"-I{ROOT}/include", os.path.join(ROOT, "tests", "c", "ops_c.c"), "-o", exe,
           f"-L{PKG}", "-lgockpt", f"-L{ROCM}/lib", "-lamdhip64", "-lm", f"-Wl,-rpath,{PKG}",
           f"-Wl,-rpath,{ROCM}/lib"]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    return exe


def test_c_consumer_compiles_against_the_header(tmp_path):
    _build(tmp_path)


@pytest.mark.gpu
def test_c_consumer_agrees_with_the_host(tmp_path):
    r = subprocess.run([_build(tmp_path)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.startswith("ok"), (r.returncode, r.stdout, r.stderr)
