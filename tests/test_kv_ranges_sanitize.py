"""The host layer of the paged cache's calls for long contexts under AddressSanitizer and UndefinedBehaviorSanitizer (CPU
only): the entry points, and the launchers that plan their workspaces, rebuilt with both on their host code, every other object
unchanged, and linked into tests/sanitize/kv_ranges_host_checks.cpp."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/llvm/bin/clang++"

pytestmark = pytest.mark.slow


def test_kv_ranges_host_layer_under_asan_and_ubsan(tmp_path):
    from paper_2609_29029_amd import build as B
    if not os.path.exists(CLANG):
        pytest.skip("no ROCm clang++ in this image")
    if not all(os.path.exists(os.path.join(B.BUILD, s.replace(".hip", ".o"))) for s in B.SOURCES):
        B.build()
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-omit-frame-pointer"]
    checked = ("capi.hip", "kv_capi.hip", "kv_bounds.hip", "kv_ranges.hip")
    objs = [str(tmp_path / s.replace(".hip", ".o")) for s in checked]
    builds = [subprocess.Popen([B.hipcc(), "-O1", "-g", "-std=c++17", f"--offload-arch={B.ARCH}", "-fPIC", *san,
                                "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                                "-c", os.path.join(B.CSRC, s), "-o", o], stderr=subprocess.PIPE, text=True)
              for s, o in zip(checked, objs)]
    errors = [b.communicate()[1] for b in builds]
    assert all(b.returncode == 0 for b in builds), errors
    host_san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]
    others = [os.path.join(B.BUILD, s.replace(".hip", ".o")) for s in B.SOURCES if s not in checked]
    driver, exe = str(tmp_path / "driver.o"), str(tmp_path / "kv_ranges_host_checks")
    for command in ([CLANG, "-O1", "-g", "-std=c++17", *host_san, "-c",
                     os.path.join(ROOT, "tests", "sanitize", "kv_ranges_host_checks.cpp"), "-o", driver],
                    [CLANG, *host_san, driver, *objs, *others, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]):
        r = subprocess.run(command, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="abort_on_error=1:detect_leaks=1",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    print(r.stdout, r.stderr[-4000:])
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert " 0 failed" in r.stdout
