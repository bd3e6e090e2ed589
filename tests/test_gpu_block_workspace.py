"""The linear layer's passes on the GPU stay within the workspace that their size asks for, whatever it holds:
rows that are read in place and rows that are copied, through every tile and part."""
import pytest

torch = pytest.importorskip("torch")

import block_paths  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# (Those of fewer than 2^31 products, and borders of few tokens.)
SIZES = sorted({size for size, *_ in block_paths.FORWARD + block_paths.BACKWARD if size[0] * size[1] * size[2] < 2 ** 31} |
               {(1, 6400, 1600), (1, 64, 64), (33, 64, 64), (64, 64, 64), (65, 64, 64), (128, 64, 64), (129, 64, 64)})


@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (BF16, F32)], ids=["f32", "bf16", "mixed"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_nothing_around_the_workspace_is_touched(size, types):
    from paper_2411_17866_amd import ops
    tokens, dim, wide = size
    dtype, dw_dtype = types
    gen = torch.Generator(device="cuda").manual_seed(sum(size))

    def rows(n, cols, apart):
        """Rows of n x cols, that far behind each other's ends."""
        t = torch.empty(n, cols + apart, device="cuda").normal_(0, 1, generator=gen).to(dtype)
        return t[:, :cols]

    for act in ("none", "silu"):
        for apart in (0, 3):  # (read in place where their width allows it; never)
            x, w, dy, z = rows(tokens, dim, apart), rows(wide, dim, apart), rows(tokens, wide, apart), rows(tokens, wide, apart)
            bias = torch.empty(wide, device="cuda").normal_(0, 1, generator=gen)
            for grads in (True, False):
                plan = ops.Linear(tokens, dim, wide, dtype=dtype, act=act, dw_dtype=dw_dtype, grads=grads)
                seen = []
                for fill in (0, 255):
                    room = torch.full((256 + plan.workspace_bytes + 4096 + 256,), fill, dtype=torch.uint8, device="cuda")
                    first = 256 - room.data_ptr() % 256
                    plan.workspace = room[first:first + plan.workspace_bytes]
                    out = dict(plan(x, w, bias=bias))
                    if grads:
                        out.update(plan.backward(dy, x, w, z=None if act == "none" else z))
                    assert (room[:first] == fill).all() and (room[first + plan.workspace_bytes:] == fill).all()
                    seen.append(out)
                assert all(torch.equal(seen[0][k], seen[1][k]) for k in seen[0])
