"""What a linear layer's workspace holds, on the CPU: room for what the passes of its size use, no
more.  Few tokens are read where they lie, so that a plan for single tokens does not cost its weights' size."""
import pytest

import block_paths
from paper_2411_17866_amd import dsm
from test_block_host import show  # noqa: F401

F32, BF16 = dsm.DSM_F32, dsm.DSM_BF16
NONE, SILU = dsm.DSM_ACT_NONE, dsm.DSM_ACT_SILU


def up(n, to):
    return -(-n // to) * to


def regions(*sizes):
    """Of regions in bytes, each on a line of 256."""
    return sum(up(n, 256) for n in sizes)


def asked(tokens, dim, wide, dtype, act, dw, grads):
    return dsm.dsm_linear_workspace(dsm.dsm_linear_problem(tokens, dim, wide, dtype, act, dw, grads))


SIZES = [size for size, *_ in block_paths.FORWARD + block_paths.BACKWARD] + [
    (1, 6400, 1600), (1, 1600, 6400), (24, 6400, 1600), (32, 64, 64), (33, 64, 64), (64, 6400, 6400), (65, 6400, 1600), (128, 96, 70), (129, 96, 70)]


@pytest.mark.parametrize("act", [NONE, SILU], ids=["none", "silu"])
@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_workspace(show, size, types, act):  # noqa: F811
    tokens, dim, wide = size
    dtype, dw = types
    q = {k: v if "form" in k else int(v) for k, v in show(*size, dtype, act, dw).items()}
    number = 4 if dtype == F32 else 2
    parts = regions(q["splits"] * tokens * up(wide, 8) * 4) if q["splits"] > 1 else 0
    # Rows of x and w that do not lie as the tiles' loads want them are copied.
    row = up(dim, 64) * number
    copies = regions(tokens * row, wide * row)
    powers = regions(tokens * 4, wide * 4)
    forward = parts if q["few"] else copies + parts + (powers if q["form"] == "halves" else 0)
    assert asked(*size, dtype, act, dw, 0) == forward
    halves = q["back_form"] == "halves"
    rows = up(tokens, 64)
    dz = rows * up(wide, 64) * number * (2 if q["dz_halves"] else 1)
    dbias = (-(-tokens // q["split_rows"]) if halves else rows // 64) * wide * 4
    back = regions(dbias)
    back += regions(q["dx_splits"] * tokens * up(dim, 8) * 4) if q["dx_splits"] > 1 else 0
    back += regions(q["dw_splits"] * wide * up(dim, 8) * 4) if q["dw_splits"] > 1 else 0
    if not (q["back_few"] and dtype == BF16 and act == NONE):  # (dz is dy, read where it lies)
        back += regions(dz)
    if not q["back_few"]:
        back += regions((2 * rows if q["dz_halves"] else tokens) * row, wide * row)
    if halves:
        back += powers + regions(tokens * 4, 512 * 4, rows // q["split_rows"] * 4)
    if not q["few"] and q["dz_halves"]:  # (the passes' copies of x lie at the same place)
        forward += regions(2 * rows * row) - regions(tokens * row)
    assert asked(*size, dtype, act, dw, 1) == max(forward, back)


@pytest.mark.parametrize("size,dtype,bytes_", [((1, 6400, 1600), F32, 5 * 1600 * 4), ((24, 6400, 1600), BF16, 0), ((1, 1600, 6400), BF16, 0)], ids=str)
def test_single_tokens_ask_for_no_copy_of_the_weights(size, dtype, bytes_):
    assert asked(*size, dtype, SILU, dtype, 0) == bytes_
