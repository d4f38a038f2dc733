"""The host sides of the paged cache in 8 bits and of the page calls under AddressSanitizer and UBSan, their launches replaced by checks of what they
would be given."""
import os

from test_sanitize_paged import ROOT, run


def test_calls_stay_in_their_workspace_and_launch_limits(tmp_path):
    from paper_2502_09888_amd import build as hb
    hipcc, flags = hb._hipcc(), [f for f in hb.FLAGS if f != "-fPIC"]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    objs = [str(tmp_path / name) for name in ("paged8.o", "pages.o", "driver.o")]
    run([hipcc, *flags, *san, "-c", os.path.join(hb.CSRC, "paged8_api.hip"), "-o", objs[0]])
    run([hipcc, *flags, *san, "-c", os.path.join(hb.CSRC, "pages_api.hip"), "-o", objs[1]])
    run([hipcc, *flags, *san, "-x", "hip", "--offload-host-only", "-c", os.path.join(ROOT, "tests", "sanitize", "pages_driver.cpp"), "-o", objs[2]])
    exe = str(tmp_path / "pages_san")
    run([hipcc, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize", "-o", exe, *objs])
    out = run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert "bad=0" in out
