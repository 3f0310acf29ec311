"""Host code of the packed plans, the pages and the shared-prefix attention
under AddressSanitizer and UBSan (CPU only): tests/c_abi/kvc_serving_checks
against the instrumented library that the other host checks build."""
import importlib.util
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


def test_serving_host_code_under_sanitizers(tmp_path):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present: the checks pass fake device addresses")
    spec = importlib.util.spec_from_file_location("kvc_build_host_checks",
                                                  os.path.join(HERE, "c_abi", "build_host_checks.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    mod.build(force=False)
    exe = str(tmp_path / "kvc_serving_checks")
    subprocess.run(["/opt/rocm/llvm/bin/clang", "-std=c11", "-O1", "-g", "-Wall", "-Wextra", "-Werror",
                    *mod.DRIVER_SANITIZERS, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(mod.ROOT, "include"), os.path.join(HERE, "c_abi", "kvc_serving_checks.c"),
                    "-L" + mod.PKG, "-l:libkvc_hostsan.so", "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath," + mod.PKG,
                    "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True, capture_output=True, text=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    assert r.returncode == 0, r.stdout + r.stderr[-4000:]
    assert "serving checks ok" in r.stdout
