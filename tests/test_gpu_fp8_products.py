"""Every kernel of the 8-bit products on the GPU (fp8_sizes.py), for both types of result and both heights of the weights' blocks."""
import numpy as np
import pytest

from fp8_sizes import PRODUCTS
from oracle import ops
from paper_2603_17435_amd import binding, inputs
from test_gpu_fp8 import gpu_gemm, operands, up

pytestmark = pytest.mark.gpu

each_kernel = pytest.mark.parametrize("size", [p[0] for p in PRODUCTS], ids=lambda s: "x".join(map(str, s[:3])))
each_form = pytest.mark.parametrize("out,w_rows", [("f32", 128), ("f32", 1), ("bf16", 128), ("bf16", 1)])


def some(n, step, rng):
    """The first and last rows (or columns), both sides of a tile's borders, and some others."""
    at = np.concatenate([[0, n - 1, n - 2], np.arange(step, n, step), np.arange(step, n, step) - 1, rng.integers(0, n, 40)])
    return np.unique(at[(at >= 0) & (at < n)])


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


def check_some(got, a, sa, w, sw, w_rows, out, step=128):
    """Within FP32's bounds (those of test_gpu_fp8.py, without what 8-bit instructions would lose) on the first and last rows and
    columns, both sides of the tiles' borders, and some others."""
    rng = np.random.default_rng(1)
    rows, cols = some(a.shape[0], 64, rng), some(w.shape[0], step, rng)
    ref, total = ops.fp8_gemm(a[rows], sa[:, rows], w[cols], sw[:, cols // w_rows], 1)
    bound = (131 + sa.shape[0]) * 2.0 ** -23 * total
    if out == "bf16":
        bound += 2.0 ** -8 * (np.abs(ref) + bound)
    off = np.abs(got[np.ix_(rows, cols)] - ref)
    assert (off <= bound).all(), f"{(off > bound).sum()} of {off.size}, worst {np.nanmax(off / np.maximum(bound, 1e-300))} at {np.argwhere(off > bound)[:4].tolist()}"


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_more_than_the_usual_workspace(out):
    """A product that splits K with 128 MB and does not with 32: partial results behind the first 32 MB, the same bits again."""
    args = operands(473, 8901, 13272, 128, 4)
    got = gpu_gemm(*args, 128, out, workspace=128 << 20)
    check_some(got, *args, 128, out)
    assert np.array_equal(got, gpu_gemm(*args, 128, out, workspace=128 << 20))
    check_some(gpu_gemm(*args, 128, out), *args, 128, out)


@each_form
@each_kernel
def test_every_kernel(size, out, w_rows):
    """Any codes and scales; everything behind K, the last row and the last column is NaN or has to be left alone."""
    m, n, k, workspace = size
    args = operands(m, n, k, w_rows, m + k)
    got = gpu_gemm(*args, w_rows, out, pad=1, workspace=workspace)
    check_some(got, *args, w_rows, out)
    assert np.array_equal(got, gpu_gemm(*args, w_rows, out, workspace=workspace))  # other strides, the same bits


@each_form
@each_kernel
def test_special_values_in_every_kernel(size, out, w_rows):
    """A NaN code reaches its row or column and nothing else, a zero scale clears its block, an infinite one gives what the
    definition gives.  (What the infinite scale meets are whole multiples of 2^-9 below 2^13: zero in FP32 where it is zero.)"""
    m, n, k, workspace = size
    a, sa, w, sw = operands(m, n, k, w_rows, k)
    last = sa.shape[0] - 1
    column = sw.shape[1] // 2
    cols = np.arange(n)[np.arange(n) // w_rows == column]
    a[0, k - 1] = 0x7F
    w[n - 1, 0] = 0xFF
    w[np.ix_(cols, range(128 * last, k))] = ops.e4m3(np.array([1.0]))[0]
    sa[0, m - 1] = 0.0
    sw[last, column] = np.inf
    got = gpu_gemm(a, sa, w, sw, w_rows, out, workspace=workspace)
    ref, _ = ops.fp8_gemm(a, sa, w, sw, w_rows)
    assert np.isnan(ref[0]).all() and np.isnan(ref[:, n - 1]).all() and np.isinf(ref[1:, cols]).any() == (m > 1)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    inf = np.isinf(ref)
    assert np.array_equal(np.isinf(got), inf) and np.array_equal(got[inf], ref[inf])
    if m > 1:
        keep = np.array([j for j in range(n - 1) if j // w_rows != column])
        check_some(got[1:, keep], a[1:], sa[:, 1:], w[keep], sw[:, keep // w_rows], 1, out)


@each_form
@pytest.mark.parametrize("m", [5, 70])
def test_scales_whose_product_leaves_the_normal_range(m, out, w_rows):
    """The product of two scales is a number in FP32, subnormal or infinite ones too; a sum that is a whole number is multiplied by it
    and rounded once (and to BF16)."""
    n, k = 200, 100
    rng = np.random.default_rng(m)
    a, w = ops.e4m3(rng.integers(-16, 17, (m, k))), ops.e4m3(rng.integers(-16, 17, (n, k)))
    a[1] = 0
    sa = (rng.uniform(1, 2, (1, m)) * 2.0 ** -70).astype(np.float32)
    sw = (rng.uniform(1, 2, (1, up(n, w_rows) // w_rows)) * 2.0 ** -70).astype(np.float32)
    sa[0, :3] = 2.0 ** 100, 2.0 ** 100, 1.5
    sw[0, -1] = 2.0 ** 100
    with np.errstate(over="ignore", invalid="ignore"):
        scale = sa[0][:, None] * sw[0][np.arange(n) // w_rows][None, :]
        want = ((ops.TABLE[a] @ ops.TABLE[w].T) * scale.astype(np.float64)).astype(np.float32)
    assert (np.abs(scale[3:, 0]) < 2.0 ** -126).all() and np.isinf(scale[0, -1]) and np.isnan(want[1, -1])
    if out == "bf16":
        want = inputs.bf16_to_f32(inputs.f32_to_bf16(want))
    assert np.array_equal(gpu_gemm(a, sa, w, sw, w_rows, out), want, equal_nan=True)


def test_results_behind_2_to_31_elements():
    """Small whole numbers, so that every sum is exact; operands' rows far apart."""
    import torch
    m, n, k, ld = 70000, 33000, 130, 65536
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    gen = torch.Generator(device="cuda").manual_seed(m)
    codes = torch.from_numpy(ops.e4m3(np.arange(-4, 4))).cuda()
    a, w = (torch.empty(rows, ld, dtype=torch.uint8, device="cuda") for rows in (m, n))
    for x in (a, w):
        x[:, :k] = codes[torch.randint(0, 8, (x.shape[0], k), generator=gen, device="cuda")]
    sa, sw = torch.full((2, m), 0.5, device="cuda"), torch.full((2, up(n, 128) // 128), 2.0, device="cuda")
    c = torch.empty(m, n, device="cuda")
    binding.zs_fp8_gemm(a, sa, w, sw, c, m, n, k, lda=ld, ldw=ld)
    value = torch.float8_e4m3fn
    wv = w[:, :k].view(value).double()
    for rows in (slice(0, 200), slice(32700, 32800), slice(65000, 65100), slice(m - 200, m)):
        assert torch.equal(c[rows].double(), a[rows, :k].view(value).double() @ wv.t())


@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_more_blocks_than_a_launch_has_workgroups(transpose):
    """2^20 workgroups of sixteen blocks of a row, or of a tile of 128 x 128, are what a launch takes at a time."""
    import torch
    r, c = ((1 << 27) + 77, 1) if transpose else ((1 << 24) + 33, 3)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = (torch.randn(r, c, generator=gen, device="cuda") * 3).to(torch.bfloat16)
    rows, cols = (c, r) if transpose else (r, c)
    q = torch.full((rows, up(cols, 16)), 0xAA, dtype=torch.uint8, device="cuda")
    s = torch.full((up(cols, 128) // 128, rows), -7.0, device="cuda")
    binding.zs_fp8_quantize(x, binding.ZS_TYPE_BF16, r, c, q, s, transpose=transpose)
    blocks = torch.zeros(rows, up(cols, 128), device="cuda")
    blocks[:, :cols] = x.t() if transpose else x
    blocks = blocks.view(rows, -1, 128)
    peak = blocks.abs().amax(2)
    mantissa, exponent = torch.frexp(peak)  # 448 = 0.875 2^9
    e = torch.where(peak == 0, 0, torch.where(mantissa <= 0.875, exponent - 9, exponent - 8).clamp_min(-126))
    scale = torch.ldexp(torch.ones_like(peak), e)
    assert torch.equal(s, scale.t())
    codes = (blocks / scale[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(rows, -1)
    assert torch.equal(q, codes[:, :q.shape[1]])
