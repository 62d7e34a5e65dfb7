"""The operators of include/paraanya_ops.h on the device where a value, a width or a stride is at the edge of
what a kernel's main path takes."""
import math

import pytest

from test_gpu_ops import BF16, _check_lora, _lora_case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _lib(gpu_lib):
    return gpu_lib


# ------------------------------------------------------------------ projection with adapters
# Sizes that take the projection of up to 64 rows, 64 x 64, 128 x 128 and 256 x 256 tiles, rows of whole
# pieces, of an even and of an odd length, and both kernels of the first product.
TILES = [(24, 64, 96), (64, 71, 70), (300, 64, 96), (300, 71, 96), (4200, 136, 1030), (1300, 135, 1400), (8200, 72, 2050),
         (8200, 70, 2050), (17000, 70, 70)]


@pytest.mark.parametrize("Rk", [5, 16, 40])
@pytest.mark.parametrize("M,K,N", TILES)
def test_lora_linear_weights_that_are_not_finite_stay_with_their_request(M, K, N, Rk):
    """NaN and infinities in B and in A of two adapters, beside requests of others and without one."""
    x, w, a, b, s, bias = _lora_case(M, K, N, Rk, 4, BF16)
    b[1] = math.nan
    b[2, N // 2, Rk // 2] = math.inf
    b[2, N - 1, 0] = -math.inf
    a[3, Rk - 1, K // 3] = math.inf
    cuts = [0, 1, 3, 7, M // 3, M // 3 + 2, M // 2, M // 2, M - 7, M - 6, M - 2]
    _check_lora(x, w, a, b, cuts, [0, 1, -1, 2, 0, 1, 2, 0, 3, 0], s, bias)


@pytest.mark.parametrize("Rk", [1, 5, 8, 20, 24, 100])
@pytest.mark.parametrize("M,K,N", [(24, 64, 96), (300, 71, 96), (1300, 136, 1400), (17000, 70, 70)])
def test_lora_linear_a_row_that_is_not_finite(M, K, N, Rk):
    """An infinity in x, with weights above 0, makes its row infinite (not NaN) and no other."""
    x, w, a, b, s, bias = _lora_case(M, K, N, Rk, 3, BF16)
    x[5, K // 2] = math.inf
    x[M - 3, 0] = -math.inf
    x[M // 2, 1] = math.nan
    _check_lora(x, w.abs(), a.abs(), b.abs(), [0, 2, 11, M // 2, M], [0, 1, -1, 2], s, bias)
