"""Host-side checks of pages of bytes and of shared prefixes, which need no GPU."""
import ctypes
import os
import shutil
import subprocess

import pytest

from tests.conftest import REPO


@pytest.fixture(scope="module")
def lib():
    from paper_2609_03675_gb300 import build, kv
    build.build()
    return kv._load()


def test_sizes_and_constants_match_the_binding(tmp_path):
    from paper_2609_03675_gb300 import kv
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    src = tmp_path / "sizes.c"
    src.write_text('#include "cofie_kv.h"\n#include <stdio.h>\nint main(void) { printf("%zu %u", sizeof(cofie_kv_prefix), COFIE_KV_INT8); return 0; }\n')
    exe = tmp_path / "sizes"
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(REPO, "include"), str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    size, int8 = subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()
    assert int(size) == ctypes.sizeof(kv._Prefix) == kv._PREFIX.size and int(int8) == kv._BITS["int8"][1]


@pytest.mark.parametrize("field,value,msg", [("bits", 0x107, b"bits"), ("bits", 0x110, b"bits"), ("bits", 0x104, b"bits"), ("k_scales", None, b"required"),
                                             ("v_scales", 4098, b"aligned"), ("k_pages", 4104, b"aligned")])
def test_caches_of_bytes_are_checked_without_a_gpu(lib, field, value, msg):
    from paper_2609_03675_gb300 import _abi, kv
    p = kv._KVParams(4, 16, 8, 2, 64, 0, 0x108, -1, 4096, 4096, 4096, 4096)
    setattr(p, field, value)
    h = ctypes.c_void_p()
    assert lib.cofie_kv_create(ctypes.byref(p), ctypes.byref(h)) == _abi.EINVAL
    assert msg in lib.cofie_kv_last_error(None) and not h.value


def test_shared_without_a_handle(lib):
    from paper_2609_03675_gb300 import _abi
    assert lib.cofie_kv_attend_shared(None, None, None, None, None, None, 0, 1, 0.0, None) == _abi.EINVAL
