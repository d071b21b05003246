"""The paged cache's host code under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only; device code is not instrumented)."""
import os
import subprocess

from paper_2512_24086_amd import build as b
from tests.test_host_sanitized import ROOT, SAN


def test_paged_abi_is_clean_under_asan_and_ubsan(tmp_path):
    build_dir = os.path.join(b.PKG, "_build")
    others = [os.path.join(build_dir, os.path.splitext(s)[0] + ".o") for s in b.SOURCES if s != "rf2_paged.cpp"]
    if not all(os.path.exists(o) for o in others):
        b.build(verbose=False)
    objects = []
    for source in (os.path.join(b.CSRC, "rf2_paged.cpp"), os.path.join(ROOT, "tests", "paged_abi_sanitized.cpp")):
        objects.append(str(tmp_path / (os.path.basename(source) + ".o")))
        subprocess.run([b.hipcc(), *b.FLAGS, *SAN, "-c", source, "-o", objects[-1]], check=True, capture_output=True)
    exe = str(tmp_path / "paged_abi_sanitized")
    subprocess.run([b.hipcc(), "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize", *objects, *others,
                    "-o", exe], check=True, capture_output=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:verify_asan_link_order=0:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    out = run.stdout + run.stderr
    assert run.returncode == 0, out[-3000:]
    assert "PAGED ABI CHECK PASSED" in run.stdout
    assert "AddressSanitizer" not in out and "runtime error" not in out and "LeakSanitizer" not in out, out[-3000:]
