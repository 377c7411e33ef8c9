"""The 8-bit products on the GPU against their definitions in 64 bits (oracle/ops.py).

Tolerances, derived: codes and scales are equal bit for bit.  A product's block sum of 128 terms, its two scales and
the sum over the blocks are in FP32: with a relative error of 2^-23 for each of the 128 + blocks + 3 operations
(twice a rounding's half step, so that a matrix core that cuts instead of rounding passes as well) the result is off by at
most (131 + blocks) 2^-23 S, S the sum of magnitudes.  BF16 results round once more: 2^-8 of the value, and they
may come from the 8-bit matrix instructions, which cut small products: ops.fp8_cut says by how much."""
import numpy as np
import pytest

from oracle import ops
from paper_2603_17435_amd import binding, inputs

pytestmark = pytest.mark.gpu


def up(x, step):
    return -(-x // step) * step


def dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def gpu_quantize(x, block_rows=1, transpose=False, ldx=None, ldq=None, lds=None, bf16=True):
    """x: uint16 patterns or float32.  Returns the whole code and scale arrays, filled with 0xAA / -7 beforehand."""
    import torch
    r, c = x.shape
    rows, cols = (c, r) if transpose else (r, c)
    wide = np.full((r, ldx or c), 0x7FC0 if bf16 else np.nan, dtype=x.dtype)
    wide[:, :c] = x
    ldq = ldq or up(cols, 16)
    lds = lds or up(rows, block_rows) // block_rows
    q = torch.full((rows + 1, ldq), 0xAA, dtype=torch.uint8, device="cuda")
    s = torch.full((up(cols, 128) // 128 + 1, lds), -7.0, device="cuda")
    t = binding.ZS_TYPE_BF16 if bf16 else binding.ZS_TYPE_F32
    binding.zs_fp8_quantize(dev(wide.view(np.int16) if bf16 else wide), t, r, c, q, s, ldx=ldx, ldq=ldq, lds=lds, block_rows=block_rows,
                            transpose=transpose)
    torch.cuda.synchronize()
    return q.cpu().numpy(), s.cpu().numpy()


def check_quantize(x, block_rows, transpose, **kw):
    values = inputs.bf16_to_f32(x) if x.dtype == np.uint16 else x
    q, s = gpu_quantize(x, block_rows, transpose, bf16=x.dtype == np.uint16, **kw)
    want_q, want_s = ops.quantize(values.T if transpose else values, block_rows)
    rows, cols = want_q.shape
    got = q[:rows, :cols]
    nan = want_q == 127
    assert ((got[nan] & 127) == 127).all() and np.array_equal(got[~nan], want_q[~nan])
    assert np.array_equal(s[:want_s.shape[0], :want_s.shape[1]], want_s)
    assert (q[:rows, cols:up(cols, 16)] == 0).all()
    assert (q[:rows, up(cols, 16):] == 0xAA).all() and (q[rows:] == 0xAA).all()
    assert (s[want_s.shape[0]:] == -7).all() and (s[:, want_s.shape[1]:] == -7).all()


MODES = [(1, False), (1, True), (128, False), (128, True)]


@pytest.mark.parametrize("rows,transpose", MODES)
@pytest.mark.parametrize("r,c", [(1, 1), (1, 128), (3, 130), (127, 16), (128, 128), (129, 257), (33, 1000), (300, 77)])
def test_quantize(rows, transpose, r, c):
    rng = np.random.default_rng(r * 1000 + c)
    x = (rng.standard_normal((r, c)) * np.exp(rng.uniform(-20, 20, (r, 1)))).astype(np.float32)
    check_quantize(inputs.f32_to_bf16(x), rows, transpose)
    check_quantize(x, rows, transpose)


@pytest.mark.parametrize("rows,transpose", MODES)
def test_quantize_strides(rows, transpose):
    x = inputs.activations(130, 260, 5)
    cols, height = (130, 260) if transpose else (260, 130)
    check_quantize(x, rows, transpose, ldx=264, ldq=up(cols, 16) + 32, lds=height + 5)
    check_quantize(x, rows, transpose, ldx=261)
    check_quantize(inputs.bf16_to_f32(x), rows, transpose, ldx=263)


@pytest.mark.parametrize("rows,transpose", MODES)
def test_quantize_values_at_the_borders(rows, transpose):
    """Ties, magnitudes on both sides of a scale's step, subnormal and the largest numbers, zeros, NaN and Inf."""
    rng = np.random.default_rng(9)
    bits = rng.integers(0, 1 << 16, (256, 384), dtype=np.uint16)  # any BF16 pattern, NaN and Inf among them
    check_quantize(bits, rows, transpose)
    x = np.zeros((256, 384), dtype=np.float32)
    check_quantize(x, rows, transpose)
    peaks = np.array([448, 448.00003, 447.99997, 224, 3.4028235e38, 1e-45, 1.17549435e-38, 2.0 ** -118, 7 * 2.0 ** -120, 1], dtype=np.float32)
    mid = (ops.POSITIVE[:-1] + ops.POSITIVE[1:]).astype(np.float32) / 2
    for i, p in enumerate(peaks):
        x[i] = rng.choice(mid, 384) * (p / np.float32(512))
        x[i, ::128] = p
        x[i, 5] = -0.0
    x[20, 7] = np.nan
    x[21, 300] = -np.inf
    x[22, :] = np.nan
    check_quantize(x, rows, transpose)
    check_quantize(np.ascontiguousarray(x.T), rows, transpose)


# ---- products ------------------------------------------------------------------------------


def operands(m, n, k, w_rows, seed, scale_bits=True):
    """Random codes (every finite one) and scales of any mantissa."""
    rng = np.random.default_rng(seed)
    finite = np.array([c for c in range(256) if (c & 127) != 127], dtype=np.uint8)
    small = np.array([c for c in finite if abs(ops.TABLE[c]) <= 16], dtype=np.uint8)
    a, w = rng.choice(small, (m, k)), rng.choice(small, (n, k))
    a[rng.integers(0, m, 8), rng.integers(0, k, 8)] = rng.choice(finite, 8)
    w[rng.integers(0, n, 8), rng.integers(0, k, 8)] = rng.choice(finite, 8)
    kb = up(k, 128) // 128
    sa = rng.uniform(0.5, 2.0, (kb, m)).astype(np.float32)
    sw = (rng.uniform(0.5, 2.0, (kb, up(n, w_rows) // w_rows)) * 2.0 ** rng.integers(-12, 4, (kb, 1))).astype(np.float32)
    return a, sa, w, sw


def padded(x, ld, fill):
    out = np.full((x.shape[0], ld), fill, dtype=x.dtype)
    out[:, :x.shape[1]] = x
    return out


def gpu_gemm(a, sa, w, sw, w_rows, out="f32", pad=0, workspace=binding.ZS_FP8_WORKSPACE_BYTES, stream=None):
    """Everything behind the operands' columns is NaN codes and NaN scales."""
    import torch
    m, k = a.shape
    n = w.shape[0]
    ld = up(k, 16) + 16 * pad
    da, dw = dev(padded(a, ld, 0x7F)), dev(padded(w, ld, 0x7F))
    dsa, dsw = dev(padded(sa, sa.shape[1] + pad, np.nan)), dev(padded(sw, sw.shape[1] + pad, np.nan))
    ldc = up(n, 4) + 8 * pad
    c = torch.full((m + 1, ldc), 77.0, dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    ws = torch.full((max(workspace, 1),), 0xFF, dtype=torch.uint8, device="cuda") if workspace else None
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    fn = binding.zs_fp8_gemm if out == "f32" else binding.zs_fp8_gemm_bf16
    fn(da, dsa, dw, dsw, c, m, n, k, w_rows=w_rows, lda=ld, ldw=ld, ldsa=dsa.shape[1], ldsw=dsw.shape[1], ldc=ldc, workspace_dev=ws,
       workspace_bytes=workspace, stream=stream)
    torch.cuda.synchronize()
    got = c.float().cpu().numpy()
    assert (got[m:] == 77).all() and (got[:, n:] == 77).all()  # nothing else was written
    return got[:m, :n]


def check_gemm(got, a, sa, w, sw, w_rows, out):
    ref, total = ops.fp8_gemm(a, sa, w, sw, w_rows)
    bound = (131 + sa.shape[0]) * 2.0 ** -23 * total
    if out == "bf16":
        bound += ops.fp8_cut(a, sa, w, sw, w_rows)
        bound += 2.0 ** -8 * (np.abs(ref) + bound)
    off = np.abs(got - ref)
    assert (off <= bound).all(), f"{(off > bound).sum()} of {off.size}, worst {np.nanmax(off / np.maximum(bound, 1e-300))} at {np.argwhere(off > bound)[:4].tolist()}"


SIZES = [(1, 1, 1), (1, 16, 128), (1, 1000, 4096), (2, 130, 129), (5, 64, 1000), (15, 100, 257), (16, 256, 512), (17, 257, 383), (32, 512, 4100),
         (33, 129, 640), (64, 384, 2048), (65, 70, 300), (100, 1024, 1024), (128, 128, 128), (129, 333, 777), (200, 500, 1500), (255, 260, 256),
         (256, 512, 1024), (257, 300, 2000), (300, 1000, 130), (513, 769, 640), (1000, 64, 4096), (1024, 1024, 512), (7, 5003, 8100)]


@pytest.mark.parametrize("w_rows", [128, 1])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_gemm(m, n, k, w_rows):
    args = operands(m, n, k, w_rows, m * 7 + n + k)
    out = "bf16" if (m + n) % 2 else "f32"
    check_gemm(gpu_gemm(*args, w_rows, out), *args, w_rows, out)
    out = "f32" if out == "bf16" else "bf16"
    check_gemm(gpu_gemm(*args, w_rows, out, pad=1, workspace=0), *args, w_rows, out)


@pytest.mark.parametrize("m", [1, 3, 16, 20, 40, 64, 80, 130, 260])
def test_gemm_each_workspace_size_and_repeats(m):
    """Less scratch splits less: other orders of the sums, the same result within the bound; and the same bits on a second call."""
    args = operands(m, 320, 3000, 128, m)
    for room in (0, 256, 100 << 10, 3 << 20):
        got = gpu_gemm(*args, 128, "f32", workspace=room)
        check_gemm(got, *args, 128, "f32")
        assert np.array_equal(got, gpu_gemm(*args, 128, "f32", workspace=room))


@pytest.mark.parametrize("m", [1, 20, 100, 300])
def test_gemm_special_values(m):
    """A NaN code reaches its row or column and nothing else; a zero scale clears its block, an infinite one gives what
    the definition gives."""
    n, k = 140, 400
    a, sa, w, sw = operands(m, n, k, 1, 3)
    a[0, 399] = 0x7F
    w[139, 0] = 0xFF
    sa[1, m - 1] = 0.0
    sw[2, 5] = np.inf
    ref, _ = ops.fp8_gemm(a, sa, w, sw, 1)
    got = gpu_gemm(a, sa, w, sw, 1)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert np.isnan(ref[0]).all() and np.isnan(ref[:, 139]).all() and not np.isnan(ref[1:, :5]).any()
    inf = np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf]) and np.array_equal(inf, np.isinf(got))
    keep = [j for j in range(n - 1) if j != 5]
    check_gemm(got[1:, keep], a[1:], sa[:, 1:], w[keep], sw[:, keep], 1, "f32") if m > 1 else None


def test_gemm_adds_exactly_where_it_can():
    """Small whole numbers: every sum is exact, whatever its order."""
    rng = np.random.default_rng(1)
    for m, n, k in [(1, 64, 4096), (16, 48, 1024), (60, 100, 640), (130, 150, 1000), (300, 260, 512)]:
        a, w = ops.e4m3(rng.integers(-8, 9, (m, k))), ops.e4m3(rng.integers(-8, 9, (n, k)))
        kb = up(k, 128) // 128
        sa, sw = 2.0 ** rng.integers(-1, 2, (kb, m)).astype(np.float32), 2.0 ** rng.integers(-1, 2, (kb, up(n, 128) // 128)).astype(np.float32)
        ref, _ = ops.fp8_gemm(a, sa, w, sw, 128)
        assert np.array_equal(gpu_gemm(a, sa, w, sw, 128), ref.astype(np.float32))


def test_gemm_on_another_stream():
    import torch
    args = operands(50, 300, 1000, 128, 11)
    check_gemm(gpu_gemm(*args, 128, "bf16", stream=torch.cuda.Stream()), *args, 128, "bf16")


def test_gemm_on_two_streams_at_a_time():
    """Calls with a workspace each do not disturb one another."""
    import torch
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    jobs = []
    for i, (m, n, k) in enumerate([(40, 700, 3000), (300, 520, 2500)] * 3):
        args = operands(m, n, k, 128, 50 + i)
        a, w = dev(padded(args[0], up(k, 16), 0)), dev(padded(args[2], up(k, 16), 0))
        jobs.append((args, a, dev(args[1]), w, dev(args[3]), torch.empty(m, n, device="cuda"), torch.empty(8 << 20, dtype=torch.uint8, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(3):
        for i, (args, a, sa, w, sw, c, ws) in enumerate(jobs):
            binding.zs_fp8_gemm(a, sa, w, sw, c, a.shape[0], w.shape[0], args[0].shape[1], workspace_dev=ws, workspace_bytes=ws.numel(),
                                stream=streams[i % 2])
    torch.cuda.synchronize()
    for args, *_, c, ws in jobs:
        check_gemm(c.cpu().numpy(), *args, 128, "f32")


@pytest.mark.parametrize("m,n,k,ldw", [(1, 32700, 100000, 140000), (2, 70000, 65500, 65536), (70, 70000, 65500, 65536)])
def test_gemm_weights_of_more_than_4_gib(m, n, k, ldw):
    """Small whole numbers again, so that sums of any order are exact; features from all over the matrix."""
    import torch
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    gen = torch.Generator(device="cuda").manual_seed(m)
    codes = dev(ops.e4m3(np.arange(-4, 4)))
    w = codes[torch.randint(0, 8, (n, ldw), generator=gen, device="cuda", dtype=torch.uint8).int()]
    a = codes[torch.randint(0, 8, (m, ldw), generator=gen, device="cuda").int()]
    kb = up(k, 128) // 128
    sa, sw = torch.full((kb, m), 0.5, device="cuda"), torch.full((kb, up(n, 128) // 128), 2.0, device="cuda")
    c = torch.empty(m, up(n, 4), device="cuda")
    binding.zs_fp8_gemm(a, sa, w, sw, c, m, n, k, lda=ldw, ldw=ldw)
    at = torch.tensor([0, 1, 12345, n // 2, 32767 if n > 40000 else 77, n - 130, n - 2, n - 1], device="cuda")
    value = torch.float8_e4m3fn
    ref = a[:, :k].view(value).double() @ w[at][:, :k].view(value).double().t()
    assert torch.equal(c[:, at].double(), ref)


# the layers of the benchmark, checked on sampled features (the oracle's time)
@pytest.mark.parametrize("m,n,k", [(1, 1024, 4096), (16, 28672, 4096), (48, 4096, 14336), (200, 4096, 14336), (2048, 6144, 4096)])
def test_gemm_layer_sizes(m, n, k):
    rng = np.random.default_rng(k + m)
    x = inputs.activations(m, k, m)
    w = inputs.gaussian_weights(n, k, n)
    qa, sa = gpu_quantize(x)
    qw, sw = gpu_quantize(w, 128)
    a, sa, w, sw = qa[:m], sa[:-1], qw[:n], sw[:-1]
    got = gpu_gemm(a, sa, w, sw, 128)
    rows, cols = np.unique(rng.integers(0, m, 64)), np.unique(np.concatenate([rng.integers(0, n, 200), [0, n - 1]]))
    check_gemm(got[np.ix_(rows, cols)], a[rows], sa[:, rows], w[cols], sw[:, cols // 128], 1, "f32")


# ---- gradients -----------------------------------------------------------------------------


def test_gradients_against_the_formula_and_differences():
    """dX = dY W and dW = dY^T X as products of transposed codes, for L = sum of dY * (X W^T)."""
    m, n, k = 70, 200, 330
    x, w, dy = inputs.activations(m, k, 1), inputs.gaussian_weights(n, k, 2, sigma=1.0), inputs.activations(m, n, 3)

    def codes(v, rows, transpose):
        q, s = gpu_quantize(v, rows, transpose)
        return np.ascontiguousarray(q[:-1, :v.shape[0 if transpose else 1]]), s[:-1]
    dyq, wt = codes(dy, 1, False), codes(w, 128, True)
    dx = gpu_gemm(*dyq, *wt, 128)
    check_gemm(dx, *dyq, *wt, 128, "f32")
    # the transposed weights are the weights: blocks of 128 x 128 look the same from both sides
    wq = codes(w, 128, False)
    assert np.array_equal(wt[0], wq[0].T) and np.array_equal(wt[1], wq[1].T)
    dyt, xt = codes(dy, 1, True), codes(x, 1, True)
    dw = gpu_gemm(*dyt, *xt, 1)
    check_gemm(dw, *dyt, *xt, 1, "f32")
    # differences of L along some elements of X: the product itself says how much L moves
    xq, xs = codes(x, 1, False)
    g = ops.TABLE[dyq[0]] * ops.spread(dyq[1], 1, m, n)
    base = (g * gpu_gemm(xq, xs, *wq, 128)).sum()
    sums = (np.abs(g) * ops.fp8_gemm(xq, xs, *wq, 128)[1]).sum()
    for i, j in [(0, 0), (3, 100), (m - 1, k - 1)]:
        moved = xq.copy()
        moved[i, j] ^= 0x88 if (moved[i, j] & 0x78) not in (0x70, 0x78) else 0x80  # another sign and exponent
        step = (ops.TABLE[moved[i, j]] - ops.TABLE[xq[i, j]]) * xs[j // 128, i]
        found = (g * gpu_gemm(moved, xs, *wq, 128)).sum() - base
        # both L's are off by their products' bound; the gradient by its own, times the step
        tol = 2 * (131 + 3) * 2.0 ** -23 * sums * 1.5 + abs(step) * (131 + 2) * 2.0 ** -23 * ops.fp8_gemm(*dyq, *wt, 128)[1][i, j]
        assert abs(found - step * dx[i, j]) <= tol


# ---- graphs ---------------------------------------------------------------------------------


@pytest.mark.parametrize("m", [1, 24, 200])
def test_quantize_and_gemm_replay_from_a_graph(m):
    import torch
    n, k = 520, 1300
    w = inputs.gaussian_weights(n, k, 5)
    qw, sw = gpu_quantize(w, 128)
    qw, sw = dev(qw[:n]), dev(sw[:-1])
    xs = [inputs.activations(m, k, s) for s in (1, 2)]
    x = dev(xs[0].view(np.int16))
    qa = torch.zeros(m, up(k, 16), dtype=torch.uint8, device="cuda")
    sa = torch.zeros(up(k, 128) // 128, m, device="cuda")
    c = torch.zeros(m, n, device="cuda")
    ws = torch.zeros(binding.ZS_FP8_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")

    def step():
        binding.zs_fp8_quantize(x, binding.ZS_TYPE_BF16, m, k, qa, sa)
        binding.zs_fp8_gemm(qa, sa, qw, sw, c, m, n, k, workspace_dev=ws, workspace_bytes=ws.numel())
    eager = []
    for v in xs:
        x.copy_(dev(v.view(np.int16)))
        step()
        torch.cuda.synchronize()
        eager.append(c.cpu().numpy())
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        step()
    torch.cuda.synchronize()
    for i in (0, 1, 0, 1):
        x.copy_(dev(xs[i].view(np.int16)))
        c.fill_(float("nan"))
        qa.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(c.cpu().numpy(), eager[i])
