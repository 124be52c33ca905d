"""The host side of layer norm, linear attention and the clipping of gradients under AddressSanitizer and UndefinedBehaviorSanitizer; device code as the library
has it.  No GPU is involved."""
import concurrent.futures
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.slow
def test_host_side_under_sanitizers(tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc not found")
    from paper_2202_13638_amd import build
    build.build()
    units = ["bagel_api.hip", "clip.hip", "layer_norm.hip", *build.MATRIX_16_SOURCES]
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
    sources = [os.path.join(build.CSRC, u) for u in units] + [os.path.join(ROOT, "tests", "sanitize", "more_operators_driver.cpp")]

    def compiled(source):
        obj = str(tmp_path / (os.path.basename(source) + ".o"))
        r = subprocess.run(["hipcc", *build.FLAGS, "-g", "-x", "hip", *san, "-c", source, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        return obj

    with concurrent.futures.ThreadPoolExecutor(len(sources)) as pool:
        objs = list(pool.map(compiled, sources))
    objs += [os.path.join(build.BUILD, s.replace(".hip", ".o")) for s in build.SOURCES if s not in units]
    exe = str(tmp_path / "more_operators_san")
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-fno-gpu-sanitize", "-fsanitize=address", "-fsanitize=undefined", "-o", exe, *objs],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    # the HIP runtime keeps allocations of its own to the end
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "more operators sanitizer driver: ok" in out, out
    assert "ERROR: AddressSanitizer" not in out and "runtime error" not in out, out
