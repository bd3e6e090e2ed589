"""dsm_grad_clip on the GPU over tensors that lie in pieces: every kind of width, distance and first element,
pieces longer and shorter than a chunk, with NaN between them, against 64-bit values."""
import math

import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402
from paper_2411_17866_amd import dsm  # noqa: E402

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16

# first, numel, block, stride; a chunk is 16384 elements.
PLACES = [(0, 1, 1, 1), (0, 5000, 1, 3), (3, 20000, 7, 9), (0, 40000, 767, 832), (5, 40000, 768, 832), (0, 40000, 768, 771), (8, 33333, 1600, 1608),
          (1, 2047, 2048, 4096), (0, 16385, 1601, 1601), (0, 50000, 16383, 16390), (0, 50000, 16384, 16385), (7, 70000, 16385, 16392),
          (8, 100000, 40000, 40008), (13, 100001, 40001, 40003), (4, 50001, 100, 128), (24, 300, 8, 11), (16384, 40000, 24576, 30001),
          (0, 2303, 255, 257), (0, 2304, 255, 257), (0, 2305, 255, 257), (2, 255, 2, 2), (2, 257, 3, 4)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("place", PLACES, ids=str)
def test_pieces(place, dtype):
    first, numel, block, stride = place
    e = first + torch.arange(numel, device="cuda")
    at = e // block * stride + e % block
    gen = torch.Generator(device="cuda").manual_seed(sum(place))
    g = torch.empty(numel, device="cuda").normal_(0, 1, generator=gen).to(dtype)
    room = torch.full((int(at.max()) + 100,), float("nan"), device="cuda", dtype=dtype)
    gaps = torch.ones_like(room, dtype=torch.bool)
    gaps[at] = False
    kind = dsm.DSM_F32 if dtype == F32 else dsm.DSM_BF16
    for skip in (0, 1):  # (from an odd address too)
        big = torch.cat([room[:skip], room])
        data = big[skip:]
        data[at] = g
        table = (dsm.dsm_clip_tensor * 1)(dsm.dsm_clip_tensor(data.data_ptr(), first, numel, block, stride, kind, 0))
        size = dsm.dsm_clip_workspace(table, 1)
        workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
        norm = torch.empty(1, device="cuda")
        (want,), (clipped,) = O.clip([g], [0], math.inf)
        for most, limit in ((math.inf, None), (0.5 * want, 0.5 * want)):
            dsm.dsm_grad_clip(table, 1, most, norm.data_ptr(), workspace.data_ptr(), size, 1e-6,
                              torch.cuda.current_stream().cuda_stream)
            assert abs(float(norm) - want) <= 4 * O.U * want
            if limit is None:
                assert torch.equal(data[at], g)
            else:
                clipped = O.clip([g], [0], float(torch.tensor(limit).float()))[1][0]
                assert ((data[at].double() - clipped).abs() <= (O.HALF[dtype] + 2 ** -50) * clipped.abs()).all()
            assert torch.isnan(data[gaps]).all()
