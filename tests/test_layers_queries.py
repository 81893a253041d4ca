"""The workspace queries of the layers without a GPU: sizes for what the calls take, 0 for what they refuse."""
import os

import pytest

torch = pytest.importorskip("torch")
D = pytest.importorskip("paper_2605_12683_amd")
from paper_2605_12683_amd import _binding as _b  # noqa: E402

if not os.path.exists(_b.LIB_PATH):
    pytest.skip("libdeer.so is not built (run __graft_entry__.build())", allow_module_level=True)

GOOD = dict(B=2, T=16, H=4, Hk=2, Dk=8, Dv=8)
FAR = 1 << 32     # a count that 32 bits hold as the one before it is added


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("op", [_b.DEER_OP_SOLVE, _b.DEER_OP_ADJOINT])
def test_linattn(dtype, op):
    assert D.deer_linattn_workspace_bytes(**GOOD, op=op, dtype=dtype) > 0
    for name in GOOD:
        for bad in (0, -1, GOOD[name] + FAR, GOOD[name] - FAR):
            assert D.deer_linattn_workspace_bytes(**{**GOOD, name: bad}, op=op, dtype=dtype) == 0, (name, bad)
    for other in (torch.float64, torch.int32, torch.float8_e4m3fn):
        assert D.deer_linattn_workspace_bytes(**GOOD, op=op, dtype=other) == 0
    assert D.deer_linattn_workspace_bytes(**GOOD, op=op + FAR, dtype=dtype) == 0


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_layernorm(dtype):
    good = dict(rows=8, G=4, D=16)
    assert D.deer_layernorm_workspace_bytes(**good, dtype=dtype) > 0
    for name, far in (("rows", 1 << 64), ("G", FAR), ("D", FAR)):
        for bad in (0, -4, good[name] + far, good[name] - far):
            assert D.deer_layernorm_workspace_bytes(**{**good, name: bad}, dtype=dtype) == 0, (name, bad)
    assert D.deer_layernorm_workspace_bytes(**good, dtype=torch.float64) == 0
