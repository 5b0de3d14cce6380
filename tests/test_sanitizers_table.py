"""The host validation of the embedding table, the loss over many classes and
AdamW under AddressSanitizer and UBSan (CPU), on the library's
objects that test_sanitizers.py builds."""
import glob
import os
import subprocess

import pytest


def test_table_validation_under_asan_and_ubsan(tmp_path):
    base = pytest.importorskip("tests.test_sanitizers")
    if not os.path.exists(base.HIPCC):
        pytest.skip("hipcc not found")
    objs = os.path.join(base.CACHE, base._sources_hash())
    if not os.path.exists(os.path.join(objs, "abi_driver")):
        base.test_abi_validation_under_asan_and_ubsan()
    drv, exe = str(tmp_path / "driver.o"), str(tmp_path / "abi_table_driver")
    subprocess.run([base.HIPCC, "--offload-arch=gfx950", "-g", "-Xarch_host", base.SAN, "-I", base.INCLUDE, "-x", "c",
                    os.path.join(base.HERE, "abi_table_driver.c"), "-c", "-o", drv], check=True, capture_output=True)
    library = [o for o in glob.glob(os.path.join(objs, "*.o")) if os.path.basename(o) != "driver.o"]
    subprocess.run([base.HIPCC, "--offload-arch=gfx950", "-Xarch_host", base.SAN, "-o", exe, *library, drv], check=True,
                   capture_output=True)
    env = dict(base.ENV, ASAN_OPTIONS="detect_leaks=0")
    assert "abi table driver: ok" in base._run(exe, env)
