"""The linear layer and its gradients along each of the ways that the library's rules take
(block_paths), against 64-bit values within a priori bounds."""
import pytest

torch = pytest.importorskip("torch")

import block_oracle as O  # noqa: E402
import block_paths  # noqa: E402
from test_gpu_linear import BF16, F32, TYPES, _backward, _forward, _inputs  # noqa: E402

pytestmark = pytest.mark.gpu


@TYPES
@pytest.mark.parametrize("size", [s for s, *_ in block_paths.FORWARD], ids=str)
def test_forward(size, dtype):
    k = sum(size)
    _forward(_inputs(*size, dtype, seed=k), O.ACTS[k % 5])


@pytest.mark.parametrize("kind", [(F32, F32), (BF16, BF16), (BF16, F32)], ids=["f32", "bf16", "bf16_f32"])
@pytest.mark.parametrize("size", [s for s, *_ in block_paths.BACKWARD], ids=str)
def test_backward(size, kind):
    _backward(_inputs(*size, kind[0], seed=sum(size)), "silu", dw_dtype=kind[1])


# Without an activation dz is dy, read where it lies where its rows are whole; dbias's sums run
# beside the products.
@TYPES
@pytest.mark.parametrize("size", [(1, 70, 900), (5, 1917, 515), (20, 1600, 2304), (47, 65, 1030), (64, 128, 192), (192, 1000, 128), (1536, 1601, 704), (3200, 1504, 1216)], ids=str)
def test_backward_without_an_activation(size, dtype):
    _backward(_inputs(*size, dtype, seed=sum(size)), "none")
