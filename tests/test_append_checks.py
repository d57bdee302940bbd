"""What the append calls' checked mode costs the host (CPU only)."""
import os
import subprocess

import pytest

from paper_2609_39819_amd import kvt

from test_abi import no_gpu_only

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.dirname(kvt.LIB_PATH)


@no_gpu_only
@pytest.mark.parametrize("tokens", [16, 1000, 14336])
def test_the_table_of_targets_is_made_once(tmp_path, tokens):
    """The search for two tokens in one slot sizes its table for the call's tokens: growing it as they come in makes
    it again and again (7 times for 14336 tokens)."""
    exe = str(tmp_path / "append_allocs")
    r = subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(os.path.dirname(HERE), "include"),
                        os.path.join(HERE, "append_allocs.cpp"), "-o", exe, "-L", PKG, "-lkvt",
                        f"-Wl,-rpath,{PKG}", "-Wl,--allow-shlib-undefined"], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe, str(tokens)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stderr
    plain, n_plain, turned, n_turned = map(int, r.stdout.split())
    assert plain == turned == kvt.KVT_ERR_OUT_OF_RANGE
    assert n_plain <= 1 and n_turned <= 1, r.stdout
