"""The training operators' host validation layer (csrc/abi_train.hip, with csrc/abi.hip) built under
AddressSanitizer and UndefinedBehaviorSanitizer on the host side only and driven by
tests/sanitize/train_abi_harness.cpp, whose stub launchers record their arguments: no GPU is used. Every
refusal of the entry points is made here, on the CPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_05448_amd", "csrc")
HARNESS = os.path.join(ROOT, "tests", "sanitize", "train_abi_harness.cpp")
ROCM = "/opt/rocm"


def test_training_validation_layer_is_clean_under_asan_and_ubsan(tmp_path):
    hipcc = shutil.which("hipcc") or os.path.join(ROCM, "bin", "hipcc")
    clang = os.path.join(ROCM, "llvm", "bin", "clang++")
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("ROCm compilers not found")
    flags = ["-O1", "-g", "-fno-omit-frame-pointer", "-std=c++17", "--offload-arch=gfx950",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host",
             "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
             f"-I{os.path.join(ROOT, 'include')}"]
    objs = []
    for src in (os.path.join(CSRC, "abi.hip"), os.path.join(CSRC, "abi_train.hip"), HARNESS):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run([hipcc, *flags, "-x", "hip", "-c", src, "-o", obj], capture_output=True,
                           text=True)
        assert r.returncode == 0, r.stdout + r.stderr
        objs.append(obj)
    exe = str(tmp_path / "train_abi_harness")
    r = subprocess.run([clang, "-fsanitize=address,undefined", *objs, f"-L{ROCM}/lib", "-lamdhip64",
                        f"-Wl,-rpath,{ROCM}/lib", "-lpthread", "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:halt_on_error=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    print(r.stdout, r.stderr)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "all checks passed" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr
    r = subprocess.run([exe, "--plant-overflow"], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode != 0 and "heap-buffer-overflow" in r.stderr
