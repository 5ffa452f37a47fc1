"""include/aj_score.h: the library exports what it declares, the binding covers it, and calls check their arguments without a device."""
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
    text = open(os.path.join(ROOT, "include", "aj_score.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(aj_(?:score|add)_[a-z_0-9]+)\s*\(", text)))


def test_symbols_and_binding(built):
    from paper_2504_20039_b200 import score

    lib = ctypes.CDLL(built)
    assert sorted(score.EXPORTS) == _declared()
    for n in _declared():
        assert hasattr(lib, n), n


def test_header_is_plain_c(tmp_path):
    src = tmp_path / "t.c"
    src.write_text('#include "aj_score.h"\nint main(void) { return (int)AJ_SCORE_FLAG_FORCE_SIMT - 1 + AJ_E4M3 - 2; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(src), "-o", str(tmp_path / "t.o")], check=True)


def test_creation_checks_need_no_device(built):
    import torch

    import paper_2504_20039_b200 as aj

    def status(*args):
        with pytest.raises(aj.AjError) as e:
            aj.ScoreHandle(*args)
        return e.value.status

    ok = (0, 4, 64, 1000, aj.AJ_BF16, 5, 0)
    for i, bad in [(0, -1), (1, 0), (2, 0), (3, 0), (4, 3), (4, -1), (5, -1), (5, 33), (6, 2)]:
        args = list(ok)
        args[i] = bad
        assert status(*args) == aj.AJ_ERR_INVALID_ARG, args
    for i, bad in [(2, 65537), (3, 2**21 + 1)]:
        args = list(ok)
        args[i] = bad
        assert status(*args) == aj.AJ_ERR_UNSUPPORTED, args
    if not torch.cuda.is_available():  # no device: creation fails cleanly, there is no CPU fallback
        assert status(*ok) == aj.AJ_ERR_CUDA


def test_the_argument_structures_are_eight_bytes_a_field(tmp_path):
    """What the binding packs is what the header declares."""
    from paper_2504_20039_b200 import score

    src = tmp_path / "t.c"
    src.write_text('#include <stdio.h>\n#include "aj_score.h"\n'
                   'int main(void) { printf("%d %d %d %d %d %d\\n", (int)sizeof(aj_norm_args), (int)offsetof(aj_norm_args, eps), (int)offsetof(aj_norm_args, cuda_stream),'
                   ' (int)sizeof(aj_score_args), (int)offsetof(aj_score_args, inv_temperature), (int)offsetof(aj_score_args, cuda_stream)); return 0; }\n')
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "t")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [score._NORM_ARGS.size, 48, 17 * 8, score._SCORE_ARGS.size, 72, 15 * 8]


def test_the_argument_structures_are_checked(built):
    from paper_2504_20039_b200 import score

    import paper_2504_20039_b200 as aj

    p = 1 << 20
    ok = [0, p, 64, p, 64, p, 1e-5, 0, 64, 0, 1 << 22, 64, p, 64, p, 64, p, 0]
    f = score._lib()["aj_add_norm_call"]
    assert f(score._NORM_ARGS.pack(*ok)) == aj.AJ_OK  # no rows
    for i, bad in ((0, -1), (0, 1 << 32), (2, 63), (6, -1.0), (7, -1), (8, 0), (8, 1 << 32), (9, 7), (9, 1 << 33)):
        args = list(ok)
        args[7] = 4
        args[i] = bad
        assert f(score._NORM_ARGS.pack(*args)) == aj.AJ_ERR_INVALID_ARG, (i, bad)
    assert f(None) == aj.AJ_ERR_INVALID_ARG
    g = score._lib()["aj_score_call"]
    assert g(None, score._SCORE_ARGS.pack(*([p] * 6), 1, 4, 1, 1.0, *([p] * 5), 0)) == aj.AJ_ERR_INVALID_ARG and g(None, None) == aj.AJ_ERR_INVALID_ARG


def test_norm_checks_need_no_device(built):
    from paper_2504_20039_b200 import score

    import paper_2504_20039_b200 as aj

    f = score._lib()["aj_add_norm"]
    p = ctypes.c_void_p(1 << 20)
    #     device x  xs  r  rs  w  eps  rows d  dtype ro ros out os o8 o8s scale stream
    ok = [0, p, 64, p, 64, p, 1e-5, 4, 64, 0, ctypes.c_void_p(1 << 22), 64, p, 64, p, 64, p, None]
    for changes in [{0: -1}, {1: None}, {2: 63}, {4: 63}, {5: None}, {6: -1.0}, {6: float("nan")}, {7: -1}, {8: 0}, {9: 2}, {9: 7}, {11: 63}, {13: 63}, {15: 63},
                    {12: None, 14: None, 16: None}, {14: None}, {16: None}, {1: ctypes.c_void_p(3)}, {5: ctypes.c_void_p(6)}, {12: ctypes.c_void_p(1 << 21), 10: ctypes.c_void_p(1 << 21)}]:
        args = list(ok)
        for i, v in changes.items():
            args[i] = v
        assert f(*args) == aj.AJ_ERR_INVALID_ARG, changes
    args = list(ok)
    args[8], args[2], args[4], args[11], args[13], args[15] = 32769, 40000, 40000, 40000, 40000, 40000
    assert f(*args) == aj.AJ_ERR_UNSUPPORTED
    args = list(ok)
    args[7] = 0
    assert f(*args) == aj.AJ_OK  # no rows


def test_the_binding_refuses_tensors_of_other_kinds(built):
    import torch

    import paper_2504_20039_b200 as aj

    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64)
    for kw in [{}, {"out": torch.zeros(4, 64)}, {"out": torch.zeros(3, 64, dtype=torch.bfloat16)}]:  # tensors of the CPU; other type; other extent
        assert aj.add_norm(x, w, check=False, **({"out": torch.zeros_like(x)} | kw)) == aj.AJ_ERR_INVALID_ARG
    with pytest.raises(aj.AjError):
        aj.add_norm(x[0], w, out=x[0])
