"""The 8-bit products and the embedding operators, as cases that can be timed and whose outputs can be compared.

Entry points: zs_fp8_quantize, zs_fp8_gemm (FP32 output), zs_fp8_gemm_bf16, zs_embed (rows out of a compressed
table), zs_dense_embed, zs_embed_grad.  Shapes are the LLaMA-3.1 layers of paper_2603_17435_amd/inputs.py and the
128256 x 4096 LM head of the benchmark, whose table a tied embedding shares.

`own` says which side run() computes: the library's entry points, or the same operators in elementary torch
operations in 32 bits.  A case is a dict of plain values; "op" names the operator.
"""
import math
import struct

import torch

own = False

E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0

# no drawn case costs more than the largest listed one of its kind
MAX_MACS = 4096 * 28672 * 4096
MAX_WEIGHT = 28672 * 8192
MAX_QUANT = 28672 * 4096
MAX_TABLE = 128256 * 4096
MAX_ROWS = 16384 * 4096

# scratch that a program keeps for the calls that can use some: the products' sums over parts of K
PRODUCT_SCRATCH = 32 << 20


def _gemm(name, m, n, k, out, w_rows=128, op="gemm"):
    return {"name": name, "op": op, "M": m, "N": n, "K": k, "out": out, "w_rows": w_rows}


def _quant(name, r, c, rows, transpose, dtype="bf16"):
    return {"name": name, "op": "quantize", "R": r, "C": c, "block_rows": rows, "transpose": transpose, "dtype": dtype}


def _embed(name, op, v, k, t, law, index):
    return {"name": name, "op": op, "V": v, "K": k, "T": t, "law": law, "index": index}


def _grad(name, v, k, t, dtype, index):
    return {"name": name, "op": "embed_grad", "V": v, "K": k, "T": t, "dtype": dtype, "index": index}


def listed():
    return [
        # the smallest product of a decode step: the K (or V) projection of a single sequence; latency
        _gemm("gemm_kv_m1", 1, 1024, 4096, "f32"),
        # the widest layer of a block for 16 sequences: the weights are read once and little else happens
        _gemm("gemm_gate_up_m16", 16, 28672, 4096, "bf16"),
        # a short prompt through one layer as a model calls it: BF16 activations to codes, then the product
        _gemm("linear_down_m200", 200, 4096, 14336, "bf16", op="linear"),
        # a prefill chunk through the widest layer: the matrix cores
        _gemm("gemm_gate_up_m4096", 4096, 28672, 4096, "bf16"),
        # the weight gradient of the QKV layer over a ragged batch of tokens: both sides with a scale for each row's 128
        _gemm("gemm_dw_qkv_5003", 6144, 4096, 5003, "f32", w_rows=1),
        # what that gradient multiplies: activations along the tokens, transposed on the way
        _quant("quantize_t_2051", 2051, 14336, 1, True),
        # a layer's weights to codes when a model is loaded
        _quant("quantize_gate_up", 28672, 4096, 128, False),
        # the embeddings of one decode step, out of the compressed table that the LM head multiplies by
        _embed("embed_packed_32", "embed", 128256, 4096, 32, "gauss", "i64"),
        # a long prompt's, table with rows of differing scale (a third of the elements are fallbacks)
        _embed("embed_packed_5000", "embed", 128256, 4096, 5000, "rowscale", "i32"),
        # a training batch's, from an uncompressed table
        _embed("embed_dense_16384", "dense_embed", 128256, 4096, 16384, "gauss", "i64"),
        # the gradient of a small table for one short sequence
        _grad("grad_8192_t509", 8192, 1024, 509, "f32", "i64"),
        # the gradient of the whole table for a training batch
        _grad("grad_128256_t16384", 128256, 4096, 16384, "bf16", "i64"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["gemm"] * 5 + ["linear"] * 2 + ["quantize"] * 3 + ["embed"] * 2 + ["dense_embed", "embed_grad", "embed_grad"])
    if op in ("gemm", "linear"):
        while True:
            n, k = _log(rng, 64, 57344), _log(rng, 64, 28672)
            if rng.random() < 0.5:  # most layers' sizes are multiples of 128, a shard's or a small head's need not be
                n, k = max(128, n // 128 * 128), max(128, k // 128 * 128)
            if n * k <= MAX_WEIGHT:
                break
        m = min(_log(rng, 1, 8192), max(1, MAX_MACS // (n * k)))
        return {"op": op, "M": m, "N": n, "K": k, "out": rng.choice(["f32", "bf16"]), "w_rows": 1 if op == "gemm" and rng.random() < 0.25 else 128}
    if op == "quantize":
        r = _log(rng, 1, 32768)
        c = min(_log(rng, 64, 28672), MAX_QUANT // r)
        return {"op": op, "R": r, "C": c, "block_rows": rng.choice([1, 1, 128]), "transpose": rng.random() < 0.4, "dtype": rng.choice(["bf16", "bf16", "f32"])}
    index = rng.choice(["i32", "i64"])
    if op == "embed":
        k = 64 * _log(rng, 4, 128)
        v = max(1, min(_log(rng, 1024, 128256), MAX_TABLE // k) // 64) * 64
        return {"op": op, "V": v, "K": k, "T": _log(rng, 1, 5000), "law": rng.choice(["gauss", "gauss", "rowscale"]), "index": index}
    k = _log(rng, 64, 8192)
    if rng.random() < 0.7:
        k = k // 8 * 8
    v = min(_log(rng, 1024, 128256), MAX_TABLE // k)
    t = min(_log(rng, 1, 65536), MAX_ROWS // k)
    if op == "dense_embed":
        return {"op": op, "V": v, "K": k, "T": t, "law": "gauss", "index": index}
    return {"op": op, "V": v, "K": k, "T": t, "dtype": rng.choice(["bf16", "f32"]), "index": index}


def _up(x, step):
    return (x + step - 1) // step * step


def _weights(n, k, law, gen):
    """[n, k] BF16 weights of scale 0.02; "rowscale": row scales log-uniform over three decades."""
    w = torch.randn(n, k, generator=gen, device="cuda")
    if law == "rowscale":
        w *= torch.exp(torch.rand(n, 1, generator=gen, device="cuda") * math.log(1e3) - math.log(1e3))
    return w.mul_(0.02).to(torch.bfloat16)


def _activations(r, c, dtype, gen):
    """Activations of a transformer: a few channels are much larger than the others."""
    x = torch.randn(r, c, generator=gen, device="cuda")
    x *= torch.where(torch.rand(1, c, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    return x.to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def _padded_blocks(x, rows):
    """[R, C] as [row blocks, rows, column blocks, 128], zeros behind the last row and column."""
    r, c = x.shape
    y = torch.zeros(_up(r, rows), _up(c, 128), dtype=x.dtype, device=x.device)
    y[:r, :c] = x
    return y.view(y.shape[0] // rows, rows, y.shape[1] // 128, 128)


def _stored(x, rows):
    """Codes with scales as a checkpoint holds them: scale = largest magnitude / 448, in 32 bits, of any mantissa.
    Codes' rows are padded to 128 bytes; scales lie by blocks of 128 columns: S[column block, row block]."""
    r, c = x.shape
    b = _padded_blocks(x.float(), rows)
    s = b.abs().amax((1, 3)).div_(E4M3_MAX).clamp_min_(1e-30)
    q = (b / s[:, None, :, None]).to(E4M3).view(torch.uint8).view(b.shape[0] * rows, b.shape[2] * 128)
    return q[:r].contiguous(), s.t().contiguous()


def _ids(t, v, index, gen):
    """Token ids as text has them: log-uniform (a frequent token takes several percent), 3 % of padding at the end."""
    u = torch.rand(t, generator=gen, device="cuda", dtype=torch.float64)
    ids = torch.exp(u * math.log(v)).long().sub_(1).clamp_(0, v - 1)
    if t >= 64:
        ids[t - t // 32:] = -1
    return ids.to(torch.int64 if index == "i64" else torch.int32)


DESC = "<IIqqiIQQQQQQQQQII"  # zs_desc of include/zipserv.h


def _pack(w):
    """The matrix in the layout of include/zipserv.h, for prepare(): blob on the GPU, fields of the descriptor."""
    n, k = w.shape
    n_bt = (n // 64) * (k // 64)
    bits = w.view(torch.int16)
    step = max(1, (1 << 24) // (64 * k))  # strips at a time
    strips = n // 64

    def chunk(s0):
        x = bits[64 * s0:64 * min(strips, s0 + step)].to(torch.int32) & 0xFFFF
        x = x.view(-1, 4, 2, 8, k // 64, 2, 4, 8).permute(0, 4, 5, 1, 6, 2, 3, 7)
        return x.reshape(-1, 4096)  # [BlockTile, element in storage order]

    hist = torch.zeros(256, dtype=torch.int64, device="cuda")
    for s0 in range(0, strips, step):
        e = (bits[64 * s0:64 * min(strips, s0 + step)].reshape(-1).to(torch.int32) >> 7) & 255
        hist += torch.bincount(e, minlength=256)
    total = torch.cat([hist.new_zeros(1), hist.cumsum(0)])
    cover = total[7:257] - total[0:250]
    base = int((cover == cover.max()).nonzero()[0]) - 1
    weight = 2.0 ** torch.arange(8, device="cuda")
    planes = torch.empty(n_bt, 64, 3, 8, dtype=torch.uint8, device="cuda")
    counts = torch.empty(n_bt, dtype=torch.int64, device="cuda")
    high, low = [], []
    per_strip = k // 64
    for s0 in range(0, strips, step):
        x = chunk(s0)
        b0 = s0 * per_strip
        code = ((x >> 7) & 255) - base
        code = torch.where((code >= 1) & (code <= 7), code, 0)
        for j in range(3):
            bit = ((code >> j) & 1).float().view(-1, 64, 8, 8)
            planes[b0:b0 + x.shape[0], :, j] = (bit * weight).sum(-1).to(torch.uint8)
        inside = code > 0
        counts[b0:b0 + x.shape[0]] = inside.sum(1)
        high.append((((x >> 8) & 0x80) | (x & 0x7F)).to(torch.uint8)[inside])
        low.append(x.to(torch.int16)[~inside])
    h_units, l_units = (counts + 15) // 16, (2 * (4096 - counts) + 15) // 16
    offsets = torch.zeros(n_bt + 1, 2, dtype=torch.int64, device="cuda")
    offsets[1:, 0], offsets[1:, 1] = h_units.cumsum(0), l_units.cumsum(0)

    def spread(parts, count, first, size):
        """The compacted elements, each BlockTile's at its own start."""
        flat = torch.cat(parts)
        out = torch.zeros(size, dtype=flat.dtype, device="cuda")
        shift = first - (count.cumsum(0) - count)
        for s0 in range(0, n_bt, 4096):
            part = count[s0:s0 + 4096]
            a = int(count[:s0].sum())
            at = torch.arange(a, a + int(part.sum()), device="cuda") + shift[s0:s0 + 4096].repeat_interleave(part)
            out[at] = flat[a:a + at.numel()]
        return out

    h_bytes, l_bytes = 16 * int(offsets[-1, 0]), 16 * int(offsets[-1, 1])
    h = spread(high, counts, 16 * offsets[:-1, 0], h_bytes)
    lo = spread(low, 4096 - counts, 8 * offsets[:-1, 1], l_bytes // 2)
    off_offsets = _up(n_bt * 1536, 256)
    off_h = _up(off_offsets + 8 * (n_bt + 1), 256)
    off_l = _up(off_h + h_bytes, 256)
    size = _up(off_l + l_bytes, 256)
    blob = torch.zeros(size, dtype=torch.uint8, device="cuda")
    blob[:n_bt * 1536] = planes.view(-1)
    blob[off_offsets:off_offsets + 8 * (n_bt + 1)] = offsets.to(torch.int32).view(torch.uint8).view(-1)
    blob[off_h:off_h + h_bytes] = h
    blob[off_l:off_l + l_bytes] = lo.view(torch.uint8)
    n_high = int(counts.sum())
    fields = [0x45425A53, 1, n, k, base, 1, n_high, n * k - n_high, 0, off_offsets, off_h, off_l, h_bytes, l_bytes, size,
              int(h_units.max()), int(l_units.max())]
    return blob, fields


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]
    if op in ("gemm", "linear"):
        m, n, k, rows = case["M"], case["N"], case["K"], case["w_rows"]
        s = {"case": case, "ws": torch.empty(PRODUCT_SCRATCH, dtype=torch.uint8, device="cuda"),
             "C": torch.empty(m, _up(n, 8), dtype=torch.float32 if case["out"] == "f32" else torch.bfloat16, device="cuda")}
        s["W"], s["SW"] = _stored(_weights(n, k, "rowscale" if rows == 1 else "gauss", gen), rows)
        x = _activations(m, k, "bf16", gen)
        if op == "gemm":
            s["A"], s["SA"] = _stored(x, 1)
        else:
            s["X"] = x
            s["A"] = torch.empty(m, _up(k, 128), dtype=torch.uint8, device="cuda")
            s["SA"] = torch.empty(_up(k, 128) // 128, m, device="cuda")
        return s
    if op == "quantize":
        r, c, rows = case["R"], case["C"], case["block_rows"]
        qr, qc = (c, r) if case["transpose"] else (r, c)
        x = _weights(r, c, "rowscale", gen) if rows == 128 else _activations(r, c, "f32", gen)
        return {"case": case, "X": x.to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32),
                "Q": torch.zeros(qr, _up(qc, 128), dtype=torch.uint8, device="cuda"),
                "S": torch.empty(_up(qc, 128) // 128, _up(qr, rows) // rows, device="cuda")}
    v, k, t = case["V"], case["K"], case["T"]
    if op == "embed_grad":
        dy = torch.randn(t, k, generator=gen, device="cuda").mul_(1e-3).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
        return {"case": case, "ids": _ids(t, v, case["index"], gen), "dY": dy, "dW": torch.empty(v, k, device="cuda"),
                "ws": torch.empty((1 << 20) + 64 * t + t * k // 2 + 64 * k, dtype=torch.uint8, device="cuda")}
    w = _weights(v, k, case["law"], gen)
    s = {"case": case, "ids": _ids(t, v, case["index"], gen), "Y": torch.empty(t, k, dtype=torch.bfloat16, device="cuda")}
    if op == "dense_embed":
        return {**s, "W": w}
    s["blob"], s["fields"] = _pack(w)
    s["desc"] = bytearray(struct.pack(DESC, *s["fields"]))
    return s


# ---- the library's calls ----------------------------------------------------------------


def _run_own(s):
    from paper_2603_17435_amd import binding as zs
    case = s["case"]
    op = case["op"]
    if op in ("gemm", "linear"):
        m, n, k = case["M"], case["N"], case["K"]
        if op == "linear":
            zs.zs_fp8_quantize(s["X"], zs.ZS_TYPE_BF16, m, k, s["A"], s["SA"], ldq=s["A"].shape[1])
        gemm = zs.zs_fp8_gemm if case["out"] == "f32" else zs.zs_fp8_gemm_bf16
        gemm(s["A"], s["SA"], s["W"], s["SW"], s["C"], m, n, k, w_rows=case["w_rows"], lda=s["A"].shape[1], ldw=s["W"].shape[1],
             ldc=s["C"].shape[1], workspace_dev=s["ws"], workspace_bytes=PRODUCT_SCRATCH)
        return s["C"][:, :n]
    if op == "quantize":
        r, c = case["R"], case["C"]
        zs.zs_fp8_quantize(s["X"], zs.ZS_TYPE_BF16 if case["dtype"] == "bf16" else zs.ZS_TYPE_F32, r, c, s["Q"], s["S"],
                           ldq=s["Q"].shape[1], block_rows=case["block_rows"], transpose=case["transpose"])
        return {"codes": s["Q"][:, :r if case["transpose"] else c].view(E4M3), "scales": s["S"]}
    v, k, t, size = case["V"], case["K"], case["T"], 8 if case["index"] == "i64" else 4
    if op == "embed":
        zs.zs_embed(zs.ZsDesc.from_buffer(s["desc"]), s["blob"], s["ids"], size, t, s["Y"], scale=math.sqrt(k))
        return s["Y"]
    if op == "dense_embed":
        zs.zs_dense_embed(s["W"], v, k, s["ids"], size, t, s["Y"], scale=math.sqrt(k))
        return s["Y"]
    zs.zs_embed_grad(s["ids"], size, t, s["dY"], zs.ZS_TYPE_BF16 if case["dtype"] == "bf16" else zs.ZS_TYPE_F32, s["dW"], v, k,
                     scale=math.sqrt(k), workspace_dev=s["ws"], workspace_bytes=s["ws"].numel())
    return s["dW"]


# ---- the plain forms: elementary torch operations, 32 bits -------------------------------


def _quantized(x, rows):
    """Blocks of rows x 128 with the smallest power of two for a scale that keeps the largest finite magnitude within 448."""
    r, c = x.shape
    b = _padded_blocks(x.float(), rows)
    a = torch.where(b.isfinite(), b.abs(), 0.0).amax((1, 3))
    mantissa, exponent = torch.frexp(a)  # a = mantissa 2^exponent, 448 = 0.875 2^9
    e = torch.where(mantissa <= 0.875, exponent - 9, exponent - 8).clamp_min_(-126)
    s = torch.ldexp(torch.ones_like(a), torch.where(a == 0, 0, e))
    q = (b / s[:, None, :, None]).to(E4M3).view(torch.uint8).view(b.shape[0] * rows, b.shape[2] * 128)
    return q[:r, :c].contiguous(), s.t().contiguous()


def _values(q, s, rows, r, c):
    """Codes times scales, in 32 bits."""
    s = s.t().repeat_interleave(rows, 0)[:r].repeat_interleave(128, 1)[:, :c]
    return q[:r, :c].view(E4M3).float() * s


def _popcount(x):
    """Ones in each 64-bit integer."""
    x = x - ((x >> 1) & 0x5555555555555555)
    x = (x & 0x3333333333333333) + ((x >> 2) & 0x3333333333333333)
    x = (x + (x >> 4)) & 0x0F0F0F0F0F0F0F0F
    return ((x * 0x0101010101010101) >> 56) & 0x7F


def _rows_of_blob(s, ids):
    """BF16 patterns of the table's rows `ids`, [T, K], decoded as include/zipserv.h describes the blob."""
    f, blob = s["fields"], s["blob"]
    n, k, base = f[2], f[3], f[4]
    off_offsets, off_h, off_l, h_bytes, l_bytes = f[9:14]
    kb, n_bt = k // 64, (n // 64) * (k // 64)
    planes = blob[:n_bt * 1536].view(torch.int64).view(n_bt, 64, 3)
    offsets = blob[off_offsets:off_offsets + 8 * (n_bt + 1)].view(torch.int32).view(-1, 2)
    h, lo = blob[off_h:off_h + h_bytes], blob[off_l:off_l + l_bytes].view(torch.int16)
    row = ids % 64
    bt = (ids // 64 * kb)[:, None] + torch.arange(kb, device="cuda")
    p = planes[bt]  # [T, kb, 64 FragTiles, 3]
    mask = p[..., 0] | p[..., 1] | p[..., 2]
    count = _popcount(mask)
    before = count.cumsum(-1) - count
    j = torch.arange(8, device="cuda")  # the row's FragTiles, in the order of the columns
    tile = ((j // 4 * 4 + (row // 16)[:, None]) * 8 + j % 4 * 2 + (row % 16 // 8)[:, None])[:, None].expand(-1, kb, -1)  # [T, kb, 8]
    shift = (8 * (row % 8))[:, None, None]
    mask, before = mask.gather(-1, tile), before.gather(-1, tile)
    p = p.gather(2, tile[..., None].expand(-1, -1, -1, 3))
    below = before + _popcount(mask & ((1 << shift) - 1))
    bits = ((mask >> shift)[..., None] >> j) & 1  # [T, kb, 8 FragTiles, 8 columns]
    hi = below[..., None] + bits.cumsum(-1) - bits
    li = 64 * tile[..., None] + shift[..., None] + j - hi
    plane_bits = ((p >> shift[..., None])[..., None, :] >> j[:, None]) & 1
    code = plane_bits[..., 0] + 2 * plane_bits[..., 1] + 4 * plane_bits[..., 2]
    start = offsets[bt].long()[:, :, None, None]
    hb = h[(16 * start[..., 0] + hi).clamp_max_(max(0, h_bytes - 1))].long() if h_bytes else torch.zeros_like(hi)
    raw = lo[(8 * start[..., 1] + li).clamp_max_(max(0, l_bytes // 2 - 1))].long() if l_bytes else torch.zeros_like(hi)
    value = torch.where(bits > 0, (hb & 0x80) << 8 | (base + code) << 7 | hb & 0x7F, raw & 0xFFFF)
    return torch.where(value > 32767, value - 65536, value).to(torch.int16).view(len(ids), k).view(torch.bfloat16)


def _run_plain(s):
    case = s["case"]
    op = case["op"]
    if op in ("gemm", "linear"):
        m, n, k = case["M"], case["N"], case["K"]
        a, sa = _quantized(s["X"], 1) if op == "linear" else (s["A"], s["SA"])
        c = _values(a, sa, 1, m, k) @ _values(s["W"], s["SW"], case["w_rows"], n, k).t()
        return c.to(s["C"].dtype)
    if op == "quantize":
        q, scales = _quantized(s["X"].t() if case["transpose"] else s["X"], case["block_rows"])
        return {"codes": q.view(E4M3), "scales": scales}
    ids = s["ids"].long()
    known = (ids >= 0) & (ids < case["V"])
    ids = torch.where(known, ids, 0)
    scale = math.sqrt(case["K"])
    if op == "embed_grad":
        rows = torch.where(known[:, None], s["dY"].float() * scale, 0.0)
        return torch.zeros(case["V"], case["K"], device="cuda").index_add_(0, ids, rows)
    rows = s["W"][ids] if op == "dense_embed" else _rows_of_blob(s, ids)
    return torch.where(known[:, None], rows.float() * scale, 0.0).to(torch.bfloat16)


def run(state):
    return _run_own(state) if own else _run_plain(state)


def exact(case, seed):
    """The operators' definitions in 64 bits, from the tensors that the inputs were made of."""
    s = prepare(case, seed)
    op = case["op"]
    table = torch.arange(256, device="cuda", dtype=torch.int64)
    fraction, exponent = (table & 7).double(), (table >> 3) & 15
    table = torch.where(exponent == 0, fraction * 2.0 ** -9, (8 + fraction) * 2.0 ** (exponent - 10).double()) * torch.where(table > 127, -1.0, 1.0)

    powers = torch.tensor([2.0 ** e for e in range(-126, 129)], dtype=torch.float64, device="cuda")

    def block_scale(x, rows):
        r, c = x.shape
        peak = torch.zeros(_up(r, rows), _up(c, 128), dtype=torch.float64, device="cuda")
        peak[:r, :c] = x.abs()
        peak = peak.view(_up(r, rows) // rows, rows, -1, 128).amax(3).amax(1)
        return torch.where(peak > 0, powers[torch.searchsorted(E4M3_MAX * powers, peak)], 1.0)  # the least 2^e with peak <= 448 2^e

    def spread(scale, rows, r, c):
        return scale[torch.arange(r, device="cuda") // rows][:, torch.arange(c, device="cuda") // 128]

    if op in ("gemm", "linear"):
        m, n, k, rows = case["M"], case["N"], case["K"], case["w_rows"]
        w = table[s["W"][:n, :k].int()] * spread(s["SW"].t().double(), rows, n, k)
        if op == "gemm":
            a = table[s["A"][:m, :k].int()] * spread(s["SA"].t().double(), 1, m, k)
        else:  # the codes are part of the definition: nearest number with four bits, ties to even
            x = s["X"].double()
            scale = spread(block_scale(x, 1), 1, m, k)
            q = x / scale
            unit = powers[torch.searchsorted(powers, q.abs().clamp_min(2.0 ** -6), right=True) - 1] / 8
            a = torch.round(q / unit) * unit * scale
        return a @ w.t()
    if op == "quantize":
        x = (s["X"].t() if case["transpose"] else s["X"]).double()
        scale = block_scale(x, case["block_rows"])
        return {"codes": x / spread(scale, case["block_rows"], *x.shape), "scales": scale.t().contiguous()}
    gen = torch.Generator(device="cuda").manual_seed(seed)
    v, k = case["V"], case["K"]
    ids = s["ids"].long()
    known = (ids >= 0) & (ids < v)
    if op == "embed_grad":
        out = torch.zeros(v, k, dtype=torch.float64, device="cuda")
        order = ids[known].argsort(stable=True)
        out.index_add_(0, ids[known][order], s["dY"][known][order].double())
        return out * math.sqrt(k)
    w = _weights(v, k, case["law"], gen)
    out = torch.zeros(len(ids), k, dtype=torch.float64, device="cuda")
    out[known] = w[ids[known]].double() * math.sqrt(k)
    return out


def work(case):
    """Each input read once, each output written once."""
    op = case["op"]
    if op in ("gemm", "linear"):
        m, n, k, rows = case["M"], case["N"], case["K"], case["w_rows"]
        kb = _up(k, 128) // 128
        size = n * k + 4 * kb * (_up(n, rows) // rows) + m * n * (4 if case["out"] == "f32" else 2)
        size += 2 * m * k if op == "linear" else m * k + 4 * kb * m
        return {"bytes": size, "flops": 2 * m * n * k}
    if op == "quantize":
        r, c = case["R"], case["C"]
        return {"bytes": r * c * (3 if case["dtype"] == "bf16" else 5), "flops": 2 * r * c}
    v, k, t = case["V"], case["K"], case["T"]
    index = t * (8 if case["index"] == "i64" else 4)
    if op == "embed_grad":
        return {"bytes": index + t * k * (2 if case["dtype"] == "bf16" else 4) + 4 * v * k, "flops": t * k}
    if op == "dense_embed":
        return {"bytes": index + 2 * 2 * t * k, "flops": t * k}
    # of each BlockTile that a row meets: its planes and start, the row's own bytes
    return {"bytes": index + t * (k // 64) * (1536 + 8 + 64 + 128), "flops": t * k}
