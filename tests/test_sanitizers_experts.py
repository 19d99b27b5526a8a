"""Host-side sanitizers on the refusals of the calls on tokens sorted by expert and of the loss (no GPU involved): the library's host code
is rebuilt with AddressSanitizer and UndefinedBehaviorSanitizer, without its device code, which those tests never reach."""
import os
import subprocess

import pytest

from test_sanitizers import run_child


def test_host_checks_under_asan_and_ubsan(tmp_path):
    from paper_2512_19720_amd import build as b
    runtime = b.sanitizer_runtime()
    if not runtime or not os.path.exists(runtime):
        pytest.skip("the ROCm toolchain ships no shared AddressSanitizer runtime")
    so, stub = tmp_path / "libpdelta_san.so", tmp_path / "device_code.so"
    b.build_library(jobs=8, lib_path=str(so), obj_dir=str(tmp_path / "obj"), extra_compile=[*b.SANITIZE_COMPILE, "--offload-host-only"],
                    extra_link=b.SANITIZE_LINK)
    # the names under which host code looks for its device code, with nothing behind them
    names = [line.split()[-1] for line in subprocess.run(["nm", "-D", "--undefined-only", str(so)], capture_output=True, text=True, check=True).stdout.splitlines()]
    names = [n for n in names if n.startswith("__hip_fatbin")]
    assert names
    source = tmp_path / "device_code.c"
    source.write_text("".join(f"const char {n}[4096] = {{0}};\n" for n in names))
    subprocess.run(["gcc", "-shared", "-fPIC", "-o", str(stub), str(source)], check=True)
    run_child(["test_experts_host.py"], ["--pdelta-lib", str(so), "-m", "not gpu"], f"{runtime}:{stub}", tmp_path)
