"""The embedding operators on the GPU against their definitions (oracle/ops.py).

Lookups are equal bit for bit: one FP32 product, one rounding.  A gradient's row is the FP32 sum of its
count of tokens, in any order, times the scale: off by at most (count + 1) 2^-24 of the sum of magnitudes (one more
rounding where it is added to what was there)."""
import numpy as np
import pytest

from oracle import ops
from paper_2603_17435_amd import binding, inputs

pytestmark = pytest.mark.gpu


def dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def same(got, want):
    """Bit patterns of BF16: equal, or both NaN."""
    nan = (want & 0x7FFF) > 0x7F80
    return np.array_equal(got[~nan], want[~nan]) and ((got[nan] & 0x7FFF) > 0x7F80).all()


def lookup(fn, ids, k, ldy=None, **kw):
    import torch
    ldy = ldy or k
    y = torch.full((len(ids) + 1, ldy), 0x5A5A, dtype=torch.int16, device="cuda")
    fn(dev(ids), ids.itemsize, len(ids), y, ldy=ldy, **kw)
    torch.cuda.synchronize()
    y = y.cpu().numpy().view(np.uint16)
    assert (y[len(ids):] == 0x5A5A).all() and (y[:, k:] == 0x5A5A).all()
    return y[:len(ids), :k]


def want_rows(w, ids, scale):
    return inputs.f32_to_bf16(ops.embed(inputs.bf16_to_f32(w), ids, scale))


@pytest.mark.parametrize("kind", ["gauss", "rowscale", "specials", "zeros", "wide"])
@pytest.mark.parametrize("n,k", [(64, 64), (256, 192), (128, 320)])
def test_packed_lookup(kind, n, k):
    if kind == "zeros":
        w = np.zeros((n, k), dtype=np.uint16)
    elif kind == "wide":  # mostly fallbacks
        w = np.random.default_rng(n).integers(0, 1 << 16, (n, k), dtype=np.uint16)
    else:
        w = inputs.make_weights(kind, n, k, 3)
    blob, d = binding.zs_encode(w)
    blob = dev(blob)
    rng = np.random.default_rng(k)
    for ids in (np.arange(n), rng.permutation(n).astype(np.int32), rng.integers(-3, n + 3, 301), np.array([n - 1]), np.array([0, 0, 0, -1, n, 1 << 40]),
                np.array([-1 << 31, (1 << 31) - 1, 5], dtype=np.int32)):
        for scale, ldy in ((1.0, k), (8.0, k + 8), (0.3, k + 1)):
            got = lookup(lambda *a, **kw: binding.zs_embed(d, blob, *a, **kw), ids, k, ldy=ldy, scale=scale)
            assert same(got, want_rows(w, ids, scale))


def test_packed_lookup_of_every_bit_pattern():
    w = np.random.default_rng(4).permutation(np.arange(65536, dtype=np.uint16)).reshape(256, 256)
    blob, d = binding.zs_encode(w)
    got = lookup(lambda *a, **kw: binding.zs_embed(d, dev(blob), *a, **kw), np.arange(256), 256)
    assert same(got, w)


def test_packed_lookup_of_a_vocabulary():
    """The LM head's table of the benchmark, packed on the GPU; many tokens, repeated ones among them."""
    import torch
    n, k, t = 128256, 4096, 3001
    gen = torch.Generator(device="cuda").manual_seed(1)
    w = (torch.randn(n, k, generator=gen, device="cuda") * 0.02).to(torch.bfloat16)
    cap = binding.zs_encode_bound(n, k)
    blob = torch.empty(cap, dtype=torch.uint8, device="cuda")
    scratch = torch.empty(binding.ZS_ENCODE_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    d = binding.zs_encode_device(w, n, k, blob, cap, scratch)
    ids = torch.randint(0, n, (t,), generator=gen, device="cuda")
    ids[:3] = torch.tensor([0, n - 1, n - 1])
    y = torch.empty(t, k, dtype=torch.bfloat16, device="cuda")
    binding.zs_embed(d, blob, ids, 8, t, y, scale=64.0)
    assert torch.equal(y, (w[ids].float() * 64).to(torch.bfloat16))


def test_lookup_in_tables_of_more_than_4_gib():
    import torch
    n, k = 1 << 20, 4096
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GB")
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = torch.empty(n, k, dtype=torch.bfloat16, device="cuda").normal_(0, 0.02, generator=gen)
    ids = torch.tensor([n - 1, 0, 524288, 524287, n - 64, -1, 700001], device="cuda", dtype=torch.int32)
    want = torch.where((ids >= 0)[:, None], w[ids.clamp_min(0).long()], torch.zeros((), dtype=torch.bfloat16, device="cuda"))
    y = torch.empty(len(ids), k, dtype=torch.bfloat16, device="cuda")
    binding.zs_dense_embed(w, n, k, ids, 4, len(ids), y)
    assert torch.equal(y, want)
    cap = binding.zs_encode_bound(n, k)
    blob = torch.empty(cap, dtype=torch.uint8, device="cuda")
    d = binding.zs_encode_device(w, n, k, blob, cap, torch.empty(binding.ZS_ENCODE_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda"))
    assert d.total_bytes > 1 << 32
    y.fill_(7)
    binding.zs_embed(d, blob, ids, 4, len(ids), y)
    assert torch.equal(y, want)


@pytest.mark.parametrize("n,k,ldw", [(1, 1, 1), (5, 7, 9), (100, 64, 64), (77, 129, 130), (300, 1000, 1008), (50, 2049, 2049)])
def test_dense_lookup(n, k, ldw):
    rng = np.random.default_rng(k)
    w = rng.integers(0, 1 << 16, (n, ldw), dtype=np.uint16)
    table = dev(w.view(np.int16))
    for ids in (np.arange(n), rng.integers(-2, n + 2, 130).astype(np.int32), np.array([n - 1, -1])):
        for scale, ldy in ((1.0, k), (0.7, k + 3)):
            got = lookup(lambda *a, **kw: binding.zs_dense_embed(table, n, k, *a, ldw=ldw, **kw), ids, k, ldy=ldy, scale=scale)
            assert same(got, want_rows(w[:, :k], ids, scale))


def test_infinite_table_and_padding():
    """A padded position is zero also with a scale or table that is not finite."""
    w = np.full((64, 64), 0x7F80, dtype=np.uint16)
    ids = np.array([3, -1, 64])
    blob, d = binding.zs_encode(w)
    for got in (lookup(lambda *a, **kw: binding.zs_embed(d, dev(blob), *a, **kw), ids, 64, scale=float("inf")),
                lookup(lambda *a, **kw: binding.zs_dense_embed(dev(w.view(np.int16)), 64, 64, *a, **kw), ids, 64, scale=float("inf"))):
        assert (got[0] == 0x7F80).all() and not got[1:].any()


# ---- gradient --------------------------------------------------------------------------------


def gpu_grad(ids, dy, n, scale=1.0, lddy=None, lddw=None, base=None, workspace_fill=0xFF):
    """dy: uint16 patterns or float32; base: what is there and is added to."""
    import torch
    t, k = dy.shape
    bf16 = dy.dtype == np.uint16
    wide = np.full((t, lddy or k), 0x7FC0 if bf16 else np.nan, dtype=dy.dtype)
    wide[:, :k] = dy
    lddw = lddw or k
    dw = np.full((n + 1, lddw), 55.0, dtype=np.float32)
    if base is not None:
        dw[:n, :k] = base
    dw = dev(dw)
    need = binding.zs_embed_grad_workspace(t, n, k)
    ws = torch.full((max(need, 1),), workspace_fill, dtype=torch.uint8, device="cuda")
    binding.zs_embed_grad(dev(ids), ids.itemsize, t, dev(wide.view(np.int16) if bf16 else wide), binding.ZS_TYPE_BF16 if bf16 else binding.ZS_TYPE_F32,
                          dw, n, k, scale=scale, lddy=lddy or k, lddw=lddw, accumulate=base is not None, workspace_dev=ws, workspace_bytes=need)
    torch.cuda.synchronize()
    dw = dw.cpu().numpy()
    assert (dw[n:] == 55).all() and (dw[:, k:] == 55).all()
    return dw[:n, :k]


def check_grad(ids, dy, n, scale=1.0, base=None, **kw):
    got = gpu_grad(ids, dy, n, scale, base=base, **kw)
    values = inputs.bf16_to_f32(dy) if dy.dtype == np.uint16 else dy
    ref, total, count = ops.embed_grad(ids, values, n, scale)
    bound = (count[:, None] + 1) * 2.0 ** -24 * total
    if base is not None:
        ref = ref + base
        bound = bound + 2.0 ** -24 * np.abs(ref) * 1.001
        assert np.array_equal(got[count == 0], base[count == 0])
    else:
        assert not got[count == 0].any()
    off = np.abs(got - ref)
    assert (off <= bound).all(), (np.argwhere(off > bound)[:4].tolist(), np.max(off / np.maximum(bound, 1e-300)))
    assert np.array_equal(got, gpu_grad(ids, dy, n, scale, base=base, workspace_fill=0, **kw))  # the same bits again
    return got


@pytest.mark.parametrize("t,n,k", [(1, 1, 1), (2, 5, 3), (31, 10, 64), (32, 1000, 8), (33, 3, 130), (100, 50, 513), (1000, 100, 72),
                                    (1025, 4000, 40), (3000, 7, 16), (4096, 900, 5), (4097, 900, 5), (9, 40, 2500), (4500, 40, 1100)])
def test_grad(t, n, k):
    rng = np.random.default_rng(t + k)
    ids = rng.integers(-1, n + 1, t)
    dy = rng.standard_normal((t, k)).astype(np.float32)
    check_grad(ids, dy, n, 0.7)
    check_grad(ids.astype(np.int32), inputs.f32_to_bf16(dy), n, 3.0, lddy=k + 3, lddw=k + 5)
    base = rng.standard_normal((n, k)).astype(np.float32)
    check_grad(ids, dy, n, 0.7, base=base)


@pytest.mark.parametrize("t", [64, 777, 17000, 300000])
def test_grad_long_runs(t):
    """All tokens alike, a few ids, none at all; more tokens than one merge takes."""
    rng = np.random.default_rng(t)
    k = 8
    dy = rng.standard_normal((t, k)).astype(np.float32)
    for ids in (np.full(t, 3), np.full(t, -1), rng.integers(0, 2, t), np.sort(rng.integers(0, 9, t))[::-1].copy(),
                rng.integers(0, 1 << 17, t) % 131, np.where(np.arange(t) % 32 < 31, 4, 2)):
        check_grad(ids.astype(np.int64), dy, 200)


@pytest.mark.parametrize("t,k", [(6000, 5), (6000, 300), (12000, 1000)])
def test_grad_runs_of_every_length(t, k):
    """Runs of less and more than sixteen chunks (of 8 or 16 tokens), which begin at each place of a workgroup's eight chunks."""
    lengths = [3, 16, 33, 136, 137, 1, 150, 270, 290, 64, 8 * 129 + 3, 5, 300, 7, 1500, 129, 128, 2, 145]
    ids = np.concatenate([np.full(n, 2 * i) for i, n in enumerate(lengths * 3)])[:t]
    rng = np.random.default_rng(k)
    dy = rng.standard_normal((t, k)).astype(np.float32)
    ids = np.concatenate([ids, np.full(t - len(ids), -1)])
    check_grad(rng.permutation(ids), dy, 120, 0.5)


def test_no_tokens():
    base = np.arange(12, dtype=np.float32).reshape(4, 3)
    none = np.zeros(0, dtype=np.int64)
    assert not gpu_grad(none, np.zeros((0, 3), dtype=np.float32), 4).any()
    assert np.array_equal(gpu_grad(none, np.zeros((0, 3), dtype=np.float32), 4, base=base), base)


def test_grad_of_padded_and_infinite_rows():
    """What stands in a padded position does not reach the table; Inf and NaN reach their own row."""
    t, n, k = 200, 20, 72
    ids = np.arange(t) % 23 - 2                     # -2, -1 and 20 have no row
    dy = np.ones((t, k), dtype=np.float32)
    dy[(ids < 0) | (ids >= n)] = np.nan
    dy[ids == 3] = np.inf
    dy[np.nonzero(ids == 4)[0][1], 5] = np.nan
    got = gpu_grad(ids, dy, n)
    count = np.bincount(ids[(ids >= 0) & (ids < n)], minlength=n).astype(np.float32)
    want = np.broadcast_to(count[:, None], (n, k)).copy()
    want[3] = np.inf
    want[4, 5] = np.nan
    assert np.array_equal(got, want, equal_nan=True)


def test_grad_of_a_large_table():
    """Rows behind 2^31 elements."""
    import torch
    n, k, t = 600000, 4096, 100
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("needs 20 GB")
    ids = torch.tensor([n - 1, 524288, 0, 524287, n - 1] * 20, device="cuda")
    dy = torch.randn(t, k, device="cuda")
    dw = torch.full((n, k), 3.0, device="cuda")
    need = binding.zs_embed_grad_workspace(t, n, k)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    binding.zs_embed_grad(ids, 8, t, dy, binding.ZS_TYPE_F32, dw, n, k, workspace_dev=ws, workspace_bytes=need)
    for row, at in ((n - 1, (0, 4)), (524288, (1,)), (0, (2,)), (524287, (3,))):
        pick = torch.zeros(5, dtype=torch.bool, device="cuda")
        pick[list(at)] = True
        mine = dy[pick.repeat(20)].double()
        assert ((dw[row] - mine.sum(0)).abs() <= 41 * 2.0 ** -24 * mine.abs().sum(0)).all()
    dw[[n - 1, 524288, 0, 524287]] = 0
    assert not dw.any()


def test_grad_against_differences():
    """L = sum of G * scale * W[ids] is linear in W: moving one weight moves L by the gradient times the step."""
    rng = np.random.default_rng(2)
    n, k, t = 64, 64, 90
    w = inputs.gaussian_weights(n, k, 1, sigma=1.0)
    ids = rng.integers(0, 40, t)
    g = rng.standard_normal((t, k)).astype(np.float32)
    dw = gpu_grad(ids, g, n, 2.0)  # (a power of two: scaling a BF16 number is exact)

    def loss(table):
        blob, d = binding.zs_encode(table)
        y = lookup(lambda *a, **kw: binding.zs_embed(d, dev(blob), *a, **kw), ids, k, scale=2.0)
        return (g.astype(np.float64) * inputs.bf16_to_f32(y)).sum()
    start = loss(w)
    for v, c in [(ids[0], 0), (ids[5], 63), (ids[89], 17), (50, 3)]:
        moved = w.copy()
        moved[v, c] = inputs.f32_to_bf16(np.array([2.5], dtype=np.float32))[0]
        step = float(inputs.bf16_to_f32(moved[v:v + 1, c:c + 1])[0, 0]) - float(inputs.bf16_to_f32(w[v:v + 1, c:c + 1])[0, 0])
        _, total, count = ops.embed_grad(ids, g, n, 2.0)
        # the losses are sums in 64 bits; the gradient is off by its bound
        assert abs(loss(moved) - start - step * dw[v, c]) <= abs(step) * (count[v] + 1) * 2.0 ** -24 * total[v, c] + 1e-10


def test_grad_replays_from_a_graph():
    import torch
    n, k, t = 300, 96, 2500
    rng = np.random.default_rng(3)
    batches = [(rng.integers(-1, n, t), rng.standard_normal((t, k)).astype(np.float32)) for _ in range(2)]
    ids, dy = dev(batches[0][0]), dev(batches[0][1])
    dw, more = torch.empty(n, k, device="cuda"), torch.empty(n, k, device="cuda")
    need = binding.zs_embed_grad_workspace(t, n, k)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")

    def step():
        for out, add in ((dw, False), (more, True)):
            binding.zs_embed_grad(ids, 8, t, dy, binding.ZS_TYPE_F32, out, n, k, accumulate=add, workspace_dev=ws, workspace_bytes=need)

    def run(i, go):
        ids.copy_(dev(batches[i][0]))
        dy.copy_(dev(batches[i][1]))
        dw.fill_(float("nan"))
        more.fill_(1.0)
        torch.cuda.synchronize()
        go()
        torch.cuda.synchronize()
        return dw.cpu().numpy(), more.cpu().numpy()
    eager = [run(i, step) for i in (0, 1)]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream), torch.cuda.graph(graph, stream=stream):
        step()
    torch.cuda.synchronize()
    for i in (0, 1, 1, 0):
        assert all(np.array_equal(a, b) for a, b in zip(run(i, graph.replay), eager[i]))


# ---- together --------------------------------------------------------------------------------


def test_tokens_to_logits_with_one_packed_table():
    """As a server uses them: embeddings out of the packed table, an 8-bit layer, logits by zs_gemm on the same blob."""
    import torch
    import oracle
    vocab, hidden, t = 512, 256, 37
    table, layer = inputs.gaussian_weights(vocab, hidden, 1, sigma=1.0), inputs.gaussian_weights(hidden, hidden, 2, sigma=0.1)
    ids = np.random.default_rng(5).integers(-1, vocab, t)
    w = dev(table.view(np.int16))
    cap = binding.zs_encode_bound(vocab, hidden)
    blob = torch.empty(cap, dtype=torch.uint8, device="cuda")
    d = binding.zs_encode_device(w, vocab, hidden, blob, cap, torch.empty(binding.ZS_ENCODE_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda"))
    codes = {name: torch.zeros(rows, hidden, dtype=torch.uint8, device="cuda") for name, rows in (("w", hidden), ("x", t))}
    sw, sx = torch.empty(2, 2, device="cuda"), torch.empty(2, t, device="cuda")
    binding.zs_fp8_quantize(dev(layer.view(np.int16)), binding.ZS_TYPE_BF16, hidden, hidden, codes["w"], sw, block_rows=128)
    ws = torch.zeros(max(binding.zs_gemm_workspace(d, t), 256), dtype=torch.uint8, device="cuda")
    scratch = torch.empty(binding.ZS_FP8_WORKSPACE_BYTES, dtype=torch.uint8, device="cuda")
    x, h = torch.empty(t, hidden, dtype=torch.int16, device="cuda"), torch.empty(t, hidden, dtype=torch.int16, device="cuda")
    logits = torch.empty(t, vocab, device="cuda")
    binding.zs_embed(d, blob, dev(ids), 8, t, x, scale=16.0)
    binding.zs_fp8_quantize(x, binding.ZS_TYPE_BF16, t, hidden, codes["x"], sx)
    binding.zs_fp8_gemm_bf16(codes["x"], sx, codes["w"], sw, h, t, hidden, hidden, workspace_dev=scratch, workspace_bytes=scratch.numel())
    binding.zs_gemm(d, blob, h, logits, t, workspace_dev=ws, workspace_bytes=ws.numel())
    torch.cuda.synchronize()
    got_x, got_h = x.cpu().numpy().view(np.uint16), h.cpu().numpy().view(np.uint16)
    assert same(got_x, want_rows(table, ids, 16.0))
    qx, qs = ops.quantize(inputs.bf16_to_f32(got_x), 1)
    qw, qws = ops.quantize(inputs.bf16_to_f32(layer), 128)
    ref, total = ops.fp8_gemm(qx, qs, qw, qws, 128)
    assert (np.abs(inputs.bf16_to_f32(got_h) - ref) <= 133 * 2.0 ** -23 * total + 2.0 ** -8 * np.abs(ref) * 1.01).all()
    assert not got_h[ids < 0].any()
    ref, total = oracle.gemm(got_h, table)
    assert (np.abs(logits.cpu().numpy() - ref) <= 1e-3 * total + 1e-6).all()
