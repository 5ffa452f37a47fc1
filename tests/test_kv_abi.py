"""include/aj_kv.h: the library exports what it declares, the binding covers it, and creation checks its arguments
without a device."""
import ctypes
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def built():
    from paper_2504_20039_b200 import build as b

    return b.build()


def _declared():
    text = open(os.path.join(ROOT, "include", "aj_kv.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(aj_kv_[a-z_0-9]+)\s*\(", text)))


def test_symbols_and_binding(built):
    from paper_2504_20039_b200 import kv

    lib = ctypes.CDLL(built)
    assert sorted(kv.EXPORTS) == _declared()
    for n in _declared():
        assert hasattr(lib, n), n


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "aj_kv.h"\nint main(void) { return (int)AJ_KV_FLAG_FORCE_SIMT - 1; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "t.o")], check=True)


def test_creation_checks_need_no_device(built):
    import torch

    import paper_2504_20039_b200 as aj

    ok = (0, 2, 4, 8, 2, 128, 16)

    def status(*args):
        with pytest.raises(aj.AjError) as e:
            aj.KvHandle(*args)
        return e.value.status

    for i, bad in [(0, -1), (1, 0), (1, 5000), (2, 0), (3, 0), (3, 7), (4, 0), (5, 0)]:
        args = list(ok)
        args[i] = bad
        assert status(*args) == aj.AJ_ERR_INVALID_ARG, args
    for i, bad in [(5, 12), (5, 264), (6, 8), (6, 24), (6, 256)]:
        args = list(ok)
        args[i] = bad
        assert status(*args) == aj.AJ_ERR_UNSUPPORTED, args
    assert status(*ok, 7) == aj.AJ_ERR_INVALID_ARG
    assert status(*ok, aj.AJ_BF16, 2) == aj.AJ_ERR_INVALID_ARG
    if not torch.cuda.is_available():  # no device: creation fails cleanly, there is no CPU fallback
        assert status(*ok) == aj.AJ_ERR_CUDA
