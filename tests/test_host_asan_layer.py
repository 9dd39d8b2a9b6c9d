"""The host code of the calls around a reduced activation under AddressSanitizer (CPU
only): their argument checks and launchers are rebuilt with the host half
instrumented (`-Xarch_host -fsanitize=address`; device code is unaffected), linked
with the other objects into a private copy of libxred.so and driven by
tests/c/layer_validation.c.  Runs only where no GPU is visible: its pointers are not
real device memory."""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

import pytest

torch = pytest.importorskip("torch")
ROOT = Path(__file__).resolve().parents[1]
SRC = ROOT / "tests" / "c" / "layer_validation.c"
CLANG = "/opt/rocm/llvm/bin/clang"
REBUILT = ("xred_layer", "xred_norm", "xred_route", "xred_experts")


def test_host_code_under_asan(tmp_path):
    from paper_2510_20171_amd import build
    if torch.cuda.device_count() > 0:
        pytest.skip("a GPU is visible: the driver's pointers are not device memory")
    if not Path(CLANG).exists() or not Path(build.HIPCC).exists():
        pytest.skip("no ROCm clang / hipcc")
    if not list(build.BUILD.glob("*.o")):
        build.build()

    def rebuild(name):
        obj = tmp_path / f"{name}.o"
        subprocess.run([build.HIPCC, *build.HIPFLAGS, "-Xarch_host", "-fsanitize=address",
                        "-Xarch_host", "-fno-omit-frame-pointer", "-c",
                        str(build.CSRC / f"{name}.hip"), "-o", str(obj)],
                       check=True, capture_output=True, text=True)
        return str(obj)

    with ThreadPoolExecutor(4) as pool:
        objs = list(pool.map(rebuild, REBUILT))
    objs += [str(o) for o in sorted(build.BUILD.glob("*.o")) if o.stem not in REBUILT]
    lib, exe = tmp_path / "libxred.so", tmp_path / "layer_validation"
    subprocess.run([build.HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *objs, "-o", str(lib)],
                   check=True, capture_output=True, text=True)
    subprocess.run([CLANG, "-std=c11", "-Wall", "-Werror", "-fsanitize=address",
                    "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    f"-I{ROOT / 'include'}", str(SRC), f"-L{tmp_path}", "-lxred",
                    "-L/opt/rocm/lib", "-lamdhip64", f"-Wl,-rpath,{tmp_path}",
                    "-Wl,-rpath,/opt/rocm/lib", "-o", str(exe)],
                   check=True, capture_output=True, text=True)
    env = {**os.environ, "ASAN_OPTIONS": "detect_leaks=0:halt_on_error=1"}
    env.pop("XRED_TRACE", None)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "all layer checks passed" in r.stdout, r.stdout + r.stderr
    assert "AddressSanitizer" not in r.stderr, r.stderr
