"""The paged calls' host-side code (argument checks, plans, workspace queries) under AddressSanitizer
(CPU only), as test_abi_asan.py has it for the other entry points; undefined arithmetic (overflow,
division by zero) ends the run too."""
import os
import subprocess
import sys

import pytest

asan = pytest.importorskip("test_abi_asan")


def test_paged_host_code_is_clean(tmp_path):
    try:
        hipcc = asan.eb_build.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not found")
    rt = asan._asan_runtime()
    if rt is None:
        pytest.skip("ASan runtime not found")
    lib = str(tmp_path / "libeb_asan.so")
    host = [f for flag in ("-fsanitize=address", "-fsanitize=signed-integer-overflow",
                           "-fsanitize=integer-divide-by-zero", "-fsanitize=shift",
                           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer")
            for f in ("-Xarch_host", flag)]
    cmd = [hipcc, *asan.eb_build.HIPCC_FLAGS, *host, "-shared-libasan",
           "-I", os.path.join(asan.ROOT, "include"),
           *[os.path.join(asan.eb_build.CSRC, s) for s in asan.eb_build.SOURCES], "-o", lib]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
    assert res.returncode == 0, res.stderr[-2000:]
    driver = tmp_path / "run_abi.py"
    driver.write_text(
        "import sys\n"
        f"sys.path.insert(0, {asan.ROOT!r})\n"
        "import pytest\n"
        "import paper_2609_16450_amd.binding as B\n"
        f"B._LIB_PATH = {lib!r}\n"
        "code = pytest.main(['-q', '-x', '-p', 'no:cacheprovider', '-m', 'not gpu',\n"
        f"                   {os.path.join(asan.ROOT, 'tests', 'test_paged_abi.py')!r}])\n"
        "import ctypes\n"
        "ctypes.CDLL(None).__asan_init  # the ASan runtime is loaded\n"
        "sys.exit(int(code))\n")
    env = dict(os.environ, LD_PRELOAD=rt, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1")
    res = subprocess.run([sys.executable, str(driver)], capture_output=True, text=True,
                         timeout=600, env=env, cwd=str(tmp_path))
    out = res.stdout + res.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
    assert res.returncode == 0, out[-4000:]
    assert " passed" in out
