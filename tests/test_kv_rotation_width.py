"""The binding of aj_kv_append refuses a rotation of another width than its table's.  No device: the call is recorded instead of made."""
import pytest
import torch

import paper_2504_20039_b200 as aj


@pytest.mark.parametrize("rot_dim,ok", [(None, True), (32, True), (0, True), (30, False), (34, False), (16, False), (64, False)])
def test_a_rotation_of_another_width_than_its_table(rot_dim, ok):
    """The library takes rot_dim for the length of a table's rows: another one would rotate by other positions' angles, or read past the table."""
    h = object.__new__(aj.KvHandle)
    h._h, calls = None, []
    h._append = lambda *a: calls.append(a) or aj.AJ_OK
    if hasattr(h, "_take"):
        h._take(-1, 2, 3, 4, 2, 64, 16, aj.AJ_BF16, False)
    bf, i32 = torch.bfloat16, torch.int32
    pages = torch.zeros(5, 2, 16, 64, dtype=bf)
    args = (torch.zeros(6, 256, dtype=bf), torch.zeros(6, 128, dtype=bf), torch.zeros(6, 128, dtype=bf), pages, pages, torch.zeros(2, 2, dtype=i32),
            torch.zeros(2, dtype=i32), torch.zeros(6, 256, dtype=bf), 2, 3, torch.zeros(40, 32))
    if ok:
        assert h.append(*args, rot_dim=rot_dim) == aj.AJ_OK and len(calls) == 1
    else:
        with pytest.raises(aj.AjError) as e:
            h.append(*args, rot_dim=rot_dim)
        assert e.value.status == aj.AJ_ERR_INVALID_ARG
        assert h.append(*args, rot_dim=rot_dim, check=False) == aj.AJ_ERR_INVALID_ARG and not calls
