"""What the header of the layers in 8 bits (include/aif_q8.h) says of a call's arguments, held without a GPU."""
import pytest

from paper_2511_12934_amd import binding as B
from test_q8_host import call, ctx, lib, linear_args, rows_args  # noqa: F401  (ctx and lib are fixtures)


@pytest.mark.parametrize("name,make", [("aif_q8_rows", rows_args), ("aif_q8_linear", linear_args)])
@pytest.mark.parametrize("reserved", [1, -1, 1 << 30])
def test_reserved_fields_are_zero(lib, ctx, name, make, reserved):  # noqa: F811
    """Of calls without rows too: a field that is given a meaning later must not have been taken with another."""
    before = lib.host_launches()
    for n_rows in (5, 0):
        assert call(lib, ctx, name, make(n_rows=n_rows, reserved=reserved)) == B.AIF_EINVAL
        assert b"reserved" in lib.aif_q8_last_error(ctx)
    assert lib.host_launches() == before
    assert call(lib, ctx, name, make(reserved=0)) == B.AIF_OK
