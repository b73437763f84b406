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


def test_products_refuse_codes_whose_padding_lies_behind_their_storage():
    """A row that a product reads is read up to a multiple of 16 bytes: they have to be the tensor's, as a row's scales up to a multiple of four have to be."""
    import torch
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    bare = lambda rows, width, block=1: B.Q8Matrix(u8(rows, width), u8(rows if block == 1 else -(-rows // 128), 4), block)  # noqa: E731
    out = torch.zeros(1, 8, dtype=torch.bfloat16)
    w = B.q8_empty(8, 24, "cpu", 128)
    B.Q8Linear(B.q8_empty(1, 24, "cpu"), w, out)
    # one row of 24, which its storage ends with: for a, w and up
    with pytest.raises(ValueError, match="multiple of 16"):
        B.Q8Linear(bare(1, 24), w, out)
    a, one = B.q8_empty(1, 24, "cpu"), B.q8_empty(1, 24, "cpu", 128)
    for kw in (dict(w=bare(1, 24, 128)), dict(w=one, up=bare(1, 24, 128))):
        with pytest.raises(ValueError, match="multiple of 16"):
            B.Q8Linear(a, out=torch.zeros(1, 1, dtype=torch.bfloat16), **kw)
    # the last row of a matrix whose rows lie apart; with the bytes behind it there it is taken
    wide = u8(4 * 32)
    with pytest.raises(ValueError, match="multiple of 16"):
        B.Q8Linear(B.Q8Matrix(wide[:3 * 32 + 24].clone().as_strided((4, 24), (32, 1)), u8(4, 4)), w, torch.zeros(4, 8, dtype=torch.bfloat16))
    B.Q8Linear(B.Q8Matrix(wide.as_strided((4, 24), (32, 1)), u8(4, 4)), w, torch.zeros(4, 8, dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="multiple of 16"):
        B.Q8Linear(B.Q8Matrix(wide.as_strided((3, 24), (32, 1), 40), u8(3, 4)), w, torch.zeros(3, 8, dtype=torch.bfloat16))
    # a whole number of 16 bytes, no rows, and matrices that are written
    B.Q8Linear(bare(1, 32), B.q8_empty(8, 32, "cpu", 128), out)
    B.Q8Linear(bare(0, 24), w, torch.zeros(0, 8, dtype=torch.bfloat16))
    B.Q8Linear(B.q8_empty(1, 24, "cpu"), B.q8_empty(24, 24, "cpu", 128), bare(1, 24))
    B.Q8Rows(torch.zeros(1, 24), q=bare(1, 24))
