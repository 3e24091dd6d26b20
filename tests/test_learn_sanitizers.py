"""Host code of the learner's library under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only): the library is built with the sanitizers
on its host code, and the refusals run against it in a child process."""
import os
import subprocess

import pytest

from test_sanitizers import HIPCC, ROOT, _run_child


def test_refusals_under_asan_ubsan(tmp_path):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not available")
    clang_rt = None
    for root, _, names in os.walk("/opt/rocm/llvm/lib/clang"):
        if "libclang_rt.asan-x86_64.so" in names:
            clang_rt = os.path.join(root, "libclang_rt.asan-x86_64.so")
    if clang_rt is None:
        pytest.skip("clang AddressSanitizer runtime not available")
    from paper_2606_11440_amd.build import CSRC, LEARN_SOURCES
    host = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops", *host, "-Xarch_host", "-fno-omit-frame-pointer", "-I", os.path.join(ROOT, "include"),
             "-I", CSRC]
    procs, objs = [], []
    for src in LEARN_SOURCES:
        obj = str(tmp_path / (src + ".o"))
        objs.append(obj)
        procs.append(subprocess.Popen([HIPCC, *flags, "-c", os.path.join(CSRC, src), "-o", obj],
                                      stdout=subprocess.DEVNULL, stderr=subprocess.PIPE))
    for p in procs:
        _, err = p.communicate(timeout=900)
        assert p.returncode == 0, err.decode()[-2000:]
    lib = str(tmp_path / "liblearn_san.so")
    subprocess.check_call([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", *host, "-o", lib, *objs])
    code = ("import sys; sys.path.insert(0, %r); import paper_2606_11440_amd.learn as L; L.LEARN_PATH = %r; import pytest; "
            "sys.exit(pytest.main(['-x', '-q', '-p', 'no:cacheprovider', 'tests/test_learn_refusals.py']))" % (ROOT, lib))
    out = _run_child(["-c", code], {"LD_PRELOAD": clang_rt})
    assert " passed" in out
