"""Every kernel of the 8-bit products on the GPU (fp8_sizes.py), for both types of result and both heights of the weights' blocks."""
import numpy as np
import pytest

from fp8_sizes import PRODUCTS
from oracle import ops
from test_gpu_fp8 import gpu_gemm, up

pytestmark = pytest.mark.gpu

each_kernel = pytest.mark.parametrize("size", [p[0] for p in PRODUCTS], ids=lambda s: "x".join(map(str, s[:3])))
each_form = pytest.mark.parametrize("out,w_rows", [("f32", 128), ("f32", 1), ("bf16", 128), ("bf16", 1)])


@each_form
@each_kernel
def test_large_products_that_cancel_leave_the_small_ones(size, out, w_rows):
    """Each block of K has 448 * 448 - 448 * 448 and six products of -1, 0 or 1 in one group of eight: every partial sum is a
    whole number below 2^18, so FP32 sums are exact in any order, and so is the result, at most 6 * 33 times a power of two, as a BF16 number."""
    m, n, k, workspace = size
    rng = np.random.default_rng(m + n + k)
    unit, large = ops.e4m3(np.array([-1.0, 0.0, 1.0])), ops.e4m3(np.array([448.0, -448.0]))
    a, w = np.zeros((m, k), dtype=np.uint8), np.zeros((n, k), dtype=np.uint8)
    blocks = up(k, 128) // 128
    for b in range(blocks):
        groups = (min(k, 128 * b + 128) - 128 * b) // 8
        if groups == 0:
            continue
        p = 128 * b + 8 * int(rng.integers(groups))
        a[:, p:p + 2], w[:, p:p + 2] = large[0], large
        a[:, p + 2:p + 8], w[:, p + 2:p + 8] = rng.choice(unit, (m, 6)), rng.choice(unit, (n, 6))
    sa = np.tile(2.0 ** rng.integers(-3, 4, m), (blocks, 1)).astype(np.float32)
    sw = np.tile(2.0 ** rng.integers(-3, 4, up(n, w_rows) // w_rows), (blocks, 1)).astype(np.float32)
    got = gpu_gemm(a, sa, w, sw, w_rows, out, workspace=workspace)
    want = (ops.TABLE[a] @ ops.TABLE[w].T) * sa[0][:, None] * sw[0][np.arange(n) // w_rows]
    assert np.array_equal(got, want), f"{(got != want).sum()} of {got.size}, the first at {np.argwhere(got != want)[:4].tolist()}"
