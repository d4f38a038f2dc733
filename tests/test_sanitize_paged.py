"""The paged cache's host side under AddressSanitizer and UBSan, its launches replaced by checks of what they would be given."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=600, **kw)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    return r.stdout


def test_paged_calls_stay_in_their_workspace_and_launch_limits(tmp_path):
    from paper_2502_09888_amd import build as hb
    hipcc, flags = hb._hipcc(), [f for f in hb.FLAGS if f != "-fPIC"]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    objs = [str(tmp_path / "api.o"), str(tmp_path / "driver.o")]
    run([hipcc, *flags, *san, "-c", os.path.join(hb.CSRC, "paged_api.hip"), "-o", objs[0]])
    run([hipcc, *flags, *san, "-x", "hip", "--offload-host-only", "-c", os.path.join(ROOT, "tests", "sanitize", "paged_driver.cpp"), "-o", objs[1]])
    exe = str(tmp_path / "paged_san")
    run([hipcc, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize", "-o", exe, *objs])
    out = run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert "bad=0" in out
