"""AddressSanitizer and UndefinedBehaviorSanitizer build of the host code of the exact
attention over sequences and of the paged cache (CPU only): seq_abi.hip and
monarch_attn.hip, sanitizers on their host pass, with tests/sanitize/sequences_main.cpp."""
import os

import pytest

from test_sanitizers import HIPCC, ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2505_18698_amd", "csrc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_sequences_host_code_under_asan_ubsan(tmp_path):
    common = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
              "-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=all",
              "-fno-omit-frame-pointer", '-DMA_BUILD_ID="0123456789abcdef"', "-I", os.path.join(ROOT, "include")]
    objs = [str(tmp_path / x) for x in ("abi.o", "seq.o", "main.o")]
    _run(common + ["-c", os.path.join(CSRC, "monarch_attn.hip"), "-o", objs[0]])
    _run(common + ["-c", os.path.join(CSRC, "seq_abi.hip"), "-o", objs[1]])
    _run(common + ["--cuda-host-only", "-x", "hip", "-c", os.path.join(SAN, "sequences_main.cpp"), "-o", objs[2]])
    exe = str(tmp_path / "seq_san")
    _run([HIPCC, "--offload-arch=gfx950", "-Xarch_host", "-fsanitize=address,undefined", *objs, "-o", exe])
    assert "ok" in _run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1"))
