"""Bias tables that are not aligned for their type are refused; one that is reaches the device, wherever it lies (tested there)."""
import pytest

from paper_2401_09135_b200 import binding as B
from test_ops_host import PTR, attn_desc, bwd, fwd


@pytest.mark.parametrize("dtype,shifts", [(0, (1, 2, 3)), (1, (1, 3))])
def test_misaligned_tables_are_refused(dtype, shifts):
    for s in shifts:
        d = attn_desc(table_dtype=dtype)
        assert fwd(desc=d, table=PTR + s) == B.E_ARG
        assert bwd(desc=d, table=PTR + s) == B.E_ARG and bwd(desc=d, dtable=PTR + s) == B.E_ARG
