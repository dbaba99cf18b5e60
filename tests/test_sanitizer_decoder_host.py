"""The host code of the decoder's entry points under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU involved): their
sources built with the sanitizers on the host side, and tests/sanitize/decoder_abi_driver.c run against them."""
import os

import pytest

from test_sanitizer_host import ENV, ROOT, SAN, run

SOURCES = ("qk_rows.hip", "cache_attention.hip", "causal.hip")


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="hipcc not found")
def test_decoder_abi_validation_under_sanitizers(tmp_path):
    from paper_2208_08124_amd import build
    lib = str(tmp_path / "libdecoder_san.so")
    host_san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                "-Xarch_host", "-fno-sanitize-recover=undefined"]
    flags = [f for f in build.HIPCC_FLAGS if f != "-O3"]
    alone = os.path.join(ROOT, "tests", "sanitize", "host_error_alone.cpp")
    run(["/opt/rocm/bin/hipcc", *flags, "-O1", "-g", *host_san, "-o", lib, alone, *[os.path.join(build.CSRC, s) for s in SOURCES]])
    exe = str(tmp_path / "decoder_abi_driver")
    run(["/opt/rocm/llvm/bin/clang", *SAN, "-I" + os.path.join(ROOT, "include"), "-o", exe,
         os.path.join(ROOT, "tests", "sanitize", "decoder_abi_driver.c"), lib, "-lm",
         "-Wl,-rpath," + str(tmp_path), "-Wl,-rpath,/opt/rocm/lib"])
    out = run([exe], env=ENV)
    assert out.strip().endswith("ok")
