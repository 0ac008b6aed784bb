"""The entry points of include/cofie_kv.h: exported, declared once, C99, and
their host-side checks, which need no GPU."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest

from tests.conftest import REPO

HEADER = os.path.join(REPO, "include", "cofie_kv.h")


@pytest.fixture(scope="module")
def lib():
    from paper_2609_03675_gb300 import build, kv
    build.build()
    return kv._load()


def test_exports_every_declared_symbol(lib):
    from paper_2609_03675_gb300 import kv
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(cofie_(?:rotary|kv)_[a-z_]+)\s*\(", text)))
    assert sorted(kv.EXPORTS) == names, "binding and header disagree"
    for n in names:
        assert hasattr(lib, n), f"{n} not exported"


def test_header_is_c99_and_struct_sizes_match_the_binding(tmp_path):
    from paper_2609_03675_gb300 import kv
    if shutil.which("gcc") is None:
        pytest.skip("no gcc")
    src = tmp_path / "sizes.c"
    src.write_text('#include "cofie_kv.h"\n#include <stdio.h>\nint main(void) { printf("%zu %zu %zu %zu", sizeof(cofie_rotary_params), '
                   'sizeof(cofie_rows), sizeof(cofie_kv_params), sizeof(cofie_kv_batch)); return 0; }\n')
    exe = tmp_path / "sizes"
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(REPO, "include"), str(src), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    sizes = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]
    assert sizes == [ctypes.sizeof(x) for x in (kv._RotaryParams, kv._Rows, kv._KVParams, kv._Batch)]


def test_null_arguments(lib):
    from paper_2609_03675_gb300 import _abi
    h = ctypes.c_void_p()
    assert lib.cofie_rotary_create(None, ctypes.byref(h)) == _abi.EINVAL
    assert lib.cofie_kv_create(None, ctypes.byref(h)) == _abi.EINVAL
    assert lib.cofie_rotary_run(None, None, 1, 1, None, 0, 0, None) == _abi.EINVAL
    assert lib.cofie_kv_append(None, None, None, None, None, None, None, None) == _abi.EINVAL
    assert lib.cofie_kv_read(None, None, None, None, None) == _abi.EINVAL
    assert lib.cofie_kv_attend(None, None, None, None, None, 0, 1, 0.0, None) == _abi.EINVAL
    assert lib.cofie_kv_status(None, None) == _abi.EINVAL
    lib.cofie_rotary_destroy(None)
    lib.cofie_kv_destroy(None)
    assert b"NULL" in lib.cofie_kv_last_error(None)


def test_rotary_checks_its_rows_on_the_host(lib):
    from paper_2609_03675_gb300 import Rotary, _abi, kv
    r = Rotary(64)
    rows = (kv._Rows * 1)(kv._Rows(4096, 8192, 2, 128, 64, 128, 64))
    for change, args, msg in (({}, (rows, 0, 4, 4096, 0), b"1 to 4"), ({}, (rows, 5, 4, 4096, 0), b"1 to 4"), ({}, (rows, 1, 4, 4096, 3), b"dtype"),
                              ({}, (rows, 1, 4, None, 0), b"positions"), ({"src": 4097}, (rows, 1, 4, 4096, 0), b"aligned"),
                              ({"out": None}, (rows, 1, 4, 4096, 0), b"NULL"), ({"heads": 0}, (rows, 1, 4, 4096, 0), b"heads"),
                              ({"out": 4096, "out_token": 64}, (rows, 1, 4, 4096, 0), b"in place")):
        x = kv._Rows(4096, 8192, 2, 128, 64, 128, 64)
        for k, v in change.items():
            setattr(x, k, v)
        rows[0] = x
        assert lib.cofie_rotary_run(r._h, ctypes.addressof(rows), *args[1:4], args[4], 0, None) == _abi.EINVAL
        assert msg in lib.cofie_rotary_last_error(r._h), msg
    assert lib.cofie_rotary_run(r._h, ctypes.addressof(rows), 1, 0, None, 0, 0, None) == _abi.OK  # no tokens


@pytest.mark.parametrize("field,value,msg", [
    ("n_pages", 0, b"n_pages"), ("page_size", 48, b"page_size"), ("page_size", 512, b"page_size"), ("n_heads", 0, b"n_heads"),
    ("n_kv_heads", 3, b"divide"), ("head_dim", 96, b"head_dim"), ("dtype", 2, b"dtype"), ("bits", 8, b"bits"),
    ("k_pages", None, b"required"), ("v_scales", None, b"required"), ("v_pages", 4100, b"aligned"),
])
def test_cache_rejects_bad_params_without_a_gpu(lib, field, value, msg):
    from paper_2609_03675_gb300 import _abi, kv
    p = kv._KVParams(4, 16, 8, 2, 64, 0, 4, -1, 4096, 4096, 4096, 4096)
    setattr(p, field, value)
    h = ctypes.c_void_p()
    assert lib.cofie_kv_create(ctypes.byref(p), ctypes.byref(h)) == _abi.EINVAL
    assert msg in lib.cofie_kv_last_error(None)
    assert not h.value


def test_frequencies_of_the_oracle_follow_the_formulas():
    """The oracle's own pins: no scaling gives base^(-2 i / d); yarn leaves fast pairs and divides slow ones."""
    from tests import kv_oracle as K
    f, m = K.frequencies(8, 10000.0)
    assert f == pytest.approx([1.0, 0.1, 0.01, 0.001]) and m == 1.0
    assert K.frequencies(8, 10000.0, "linear", 4.0)[0] == pytest.approx([0.25, 0.025, 0.0025, 0.00025])
    y, m = K.frequencies(128, 1e6, "yarn", 4.0, 32768)
    n, _ = K.frequencies(128, 1e6)
    assert y[0] == n[0] and y[-1] == pytest.approx(n[-1] / 4) and m == pytest.approx(1.1386294)
    # base scaling: the slowest pair turns factor times slower, the fastest as before
    b, _ = K.frequencies(128, 1e6, "base", 4.0)
    assert b[0] == 1.0 and b[-1] == pytest.approx(n[-1] / 4)


def test_codes_of_the_oracle():
    import torch
    from tests import kv_oracle as K
    x = torch.zeros(64)
    x[:4] = torch.tensor([15.0, 0.5, 1.5, 14.4])
    n, s, z = K.quantise(x)
    assert float(s[0]) == 1.0 and int(z[0]) == 0 and n[:4].tolist() == [15, 1, 2, 14]
    back, _ = K.unpack(*K.pack(n, s, z))
    assert back[:4].tolist() == [15.0, 1.0, 2.0, 14.0]
    n, s, z = K.quantise(torch.linspace(-3, 4.2, 64))  # 7.2 / 15 = 0.48 -> 0.5
    assert float(s[0]) == 0.5 and int(z[0]) == 6
