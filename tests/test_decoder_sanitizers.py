"""AddressSanitizer and UndefinedBehaviorSanitizer build of the host code of cross attention and of
a decoder's operators (CPU only): seq_abi.hip, decoder_abi.hip and monarch_attn.hip, sanitizers on
their host pass, with tests/sanitize/decoder_main.cpp."""
import os

import pytest

from test_sanitizers import HIPCC, ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2505_18698_amd", "csrc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_decoder_host_code_under_asan_ubsan(tmp_path):
    common = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
              "-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=all",
              "-fno-omit-frame-pointer", '-DMA_BUILD_ID="0123456789abcdef"', "-I", os.path.join(ROOT, "include")]
    objs = [str(tmp_path / x) for x in ("abi.o", "seq.o", "decoder.o", "main.o")]
    for unit, obj in zip(("monarch_attn", "seq_abi", "decoder_abi"), objs):
        _run(common + ["-c", os.path.join(CSRC, unit + ".hip"), "-o", obj])
    _run(common + ["--cuda-host-only", "-x", "hip", "-c", os.path.join(SAN, "decoder_main.cpp"), "-o", objs[3]])
    exe = str(tmp_path / "decoder_san")
    _run([HIPCC, "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address,undefined", *objs, "-o", exe])
    assert "ok" in _run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1"))
