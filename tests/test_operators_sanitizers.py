"""The operators' host side (validation, sizes) under AddressSanitizer and UBSan, driven by a C11 program, which also proves that the
header is C.  The device code is compiled as always and never launched."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


def run(cmd, **kw):
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, **kw)
    assert r.returncode == 0, f"{' '.join(cmd)}\n{r.stdout[-4000:]}"
    return r.stdout


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_host_side_validation_of_the_operators_is_clean_under_sanitizers(tmp_path):
    from paper_2111_00705_amd import build as B
    drv, obj, exe = (str(tmp_path / f) for f in ("operators_validation.o", "operators_san.o", "operators_validation"))
    run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-c", "-I", os.path.join(ROOT, "include"), "-o", drv,
         os.path.join(ROOT, "tests", "c", "operators_validation.c")])
    host_san = []
    for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-g"):
        host_san += ["-Xarch_host", f]
    flags = [f for f in B.HIPCC_FLAGS if f not in ("-O3", "-shared", "-fPIC")]
    run([HIPCC, "-O1", *flags, *host_san, "-c", "-o", obj, B.SOURCES[1]])
    run([HIPCC, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-Wno-option-ignored", "-o", exe, obj, drv, "-lm"])
    out = run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1"))
    assert "operators validation: 0 failures" in out
    assert "ERROR" not in out and "runtime error" not in out
