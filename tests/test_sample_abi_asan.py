"""The host-side code of eb_lmhead_logits, eb_sample and eb_kv_assign (argument checks, workspace sizes,
launch shapes) under AddressSanitizer (CPU only), as test_abi_asan.py has it for other entry points;
undefined arithmetic ends the run too.  The sources are compiled side by side."""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest

asan = pytest.importorskip("test_abi_asan")


def test_host_code_is_clean(tmp_path):
    try:
        hipcc = asan.eb_build.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not found")
    rt = asan._asan_runtime()
    if rt is None:
        pytest.skip("ASan runtime not found")
    host = [f for flag in ("-fsanitize=address", "-fsanitize=signed-integer-overflow",
                           "-fsanitize=integer-divide-by-zero", "-fsanitize=shift",
                           "-fno-sanitize-recover=all", "-fno-omit-frame-pointer")
            for f in ("-Xarch_host", flag)]
    common = [hipcc, *asan.eb_build.HIPCC_FLAGS, *host, "-shared-libasan"]

    def run(cmd):
        res = subprocess.run(cmd, capture_output=True, text=True, timeout=900)
        assert res.returncode == 0, res.stderr[-2000:]

    def compiled(source):
        out = str(tmp_path / (source + ".o"))
        flags = [f for f in common if f != "-shared"]
        run([*flags, "-I", os.path.join(asan.ROOT, "include"), "-c",
             os.path.join(asan.eb_build.CSRC, source), "-o", out])
        return out

    with ThreadPoolExecutor(4) as pool:
        objects = list(pool.map(compiled, asan.eb_build.SOURCES))
    lib = str(tmp_path / "libeb_asan.so")
    run([*common, *objects, "-o", lib])
    driver = tmp_path / "run_abi.py"
    driver.write_text(
        "import sys\n"
        f"sys.path.insert(0, {asan.ROOT!r})\n"
        "import pytest\n"
        "import paper_2609_16450_amd.binding as B\n"
        f"B._LIB_PATH = {lib!r}\n"
        "code = pytest.main(['-q', '-x', '-p', 'no:cacheprovider', '-m', 'not gpu',\n"
        f"                   {os.path.join(asan.ROOT, 'tests', 'test_sample_abi.py')!r}])\n"
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
