"""The 8-bit products and embedding operators without a GPU: the oracle's own pins, refusals (all of them are
decided on the host before anything is launched), and the generated code of the kernels."""
import os
import re
import subprocess

import numpy as np
import pytest

from oracle import ops
from paper_2603_17435_amd import binding, build as zs_build
from test_isa_hazards import WIDE_STORE, kernels, wide_store_hazards

P = 1 << 20  # an address that nothing reads: the calls below are refused first


def test_oracle_e4m3():
    torch = pytest.importorskip("torch")
    table = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(table, ops.TABLE, equal_nan=True)
    fine = ~np.isnan(ops.TABLE)
    assert np.array_equal(ops.e4m3(ops.TABLE[fine]), np.arange(256)[fine])
    mid = (ops.POSITIVE[:-1] + ops.POSITIVE[1:]) / 2
    assert (ops.e4m3(mid) % 2 == 0).all()
    assert np.array_equal(ops.e4m3(mid * (1 + 2.0 ** -30)), np.arange(1, 127)) and np.array_equal(ops.e4m3(mid * (1 - 2.0 ** -30)), np.arange(126))
    q, s = ops.quantize(np.array([[448.0, 1.0], [449.0, 0.0], [0.0, 0.0], [np.inf, -3.5]]), 1)
    assert s.tolist() == [[1.0, 2.0, 1.0, 2.0 ** -7]] and q[3].tolist() == [127, 254]


def refused(fn, status, *args, **kw):
    with pytest.raises(binding.ZsError) as e:
        fn(*args, stream=0, **kw)
    assert e.value.status == status


ARG, SHAPE, SIZE, FORMAT, CONFIG = -1, -2, -3, -4, -6


def test_quantize_refusals():
    def q(status, x=P, t=binding.ZS_TYPE_BF16, r=4, c=256, out=P, s=P, **kw):
        refused(binding.zs_fp8_quantize, status, x, t, r, c, out, s, **kw)
    q(ARG, x=None)
    q(ARG, out=None)
    q(ARG, s=None)
    q(ARG, x=P + 1)
    q(ARG, x=P + 2, t=binding.ZS_TYPE_F32)
    q(ARG, out=P + 8)
    q(ARG, s=P + 2)
    q(CONFIG, t=2)
    q(CONFIG, block_rows=64)
    q(CONFIG, block_rows=0)
    q(SHAPE, r=0)
    q(SHAPE, c=0)
    q(SHAPE, r=1 << 31)
    q(SHAPE, ldx=255)
    q(SHAPE, ldq=240)
    q(SHAPE, ldq=264)
    q(SHAPE, lds=3)
    q(SHAPE, lds=1, block_rows=128, transpose=True)
    q(SHAPE, ldq=0, transpose=True)


@pytest.mark.parametrize("fn", [binding.zs_fp8_gemm, binding.zs_fp8_gemm_bf16])
def test_gemm_refusals(fn):
    def g(status, a=P, sa=P, w=P, sw=P, c=P, m=3, n=200, k=300, **kw):
        refused(fn, status, a, sa, w, sw, c, m, n, k, **kw)
    for name in ("a", "sa", "w", "sw", "c"):
        g(ARG, **{name: None})
    for name in ("a", "w", "c"):
        g(ARG, **{name: P + 8})
    g(ARG, sa=P + 1)
    g(ARG, sw=P + 2)
    g(ARG, workspace_dev=P + 128, workspace_bytes=1 << 20)
    g(CONFIG, w_rows=64)
    g(CONFIG, w_rows=0)
    for name in ("m", "n", "k"):
        g(SHAPE, **{name: 0})
        g(SHAPE, **{name: -1})
        g(SHAPE, **{name: 1 << 31})
    g(SHAPE, lda=(1 << 23) + 16)
    g(SHAPE, ldw=(1 << 23) + 16)
    g(SHAPE, lda=288)
    g(SHAPE, lda=300)
    g(SHAPE, ldw=288)
    g(SHAPE, ldw=312)
    g(SHAPE, ldc=196)
    g(SHAPE, ldc=202)
    g(SHAPE, ldsa=2)
    g(SHAPE, ldsw=1)
    g(SHAPE, ldsw=199, w_rows=1)


def test_embed_refusals():
    _, d = binding.zs_encode(np.zeros((128, 192), dtype=np.uint16))

    def e(status, desc=d, blob=P, ids=P, size=8, t=5, y=P, **kw):
        refused(binding.zs_embed, status, desc, blob, ids, size, t, y, **kw)
    e(ARG, blob=None)
    e(ARG, blob=P + 128)
    e(ARG, ids=None)
    e(ARG, ids=P + 4)
    e(ARG, y=None)
    e(ARG, y=P + 1)
    e(CONFIG, size=2)
    e(SHAPE, t=-1)
    e(SHAPE, t=1 << 31)
    e(SHAPE, ldy=191)
    bad = binding.ZsDesc.from_buffer_copy(d)
    bad.off_H += 1
    e(FORMAT, desc=bad)
    assert binding.lib().zs_embed(None, P, P, 8, 5, 1.0, P, 192, None) == ARG

    def x(status, w=P, n=100, k=50, ids=P, size=4, t=5, y=P, **kw):
        refused(binding.zs_dense_embed, status, w, n, k, ids, size, t, y, **kw)
    x(ARG, w=None)
    x(ARG, w=P + 1)
    x(ARG, ids=None)
    x(ARG, ids=P + 2)
    x(ARG, y=None)
    x(CONFIG, size=0)
    x(SHAPE, n=0)
    x(SHAPE, k=0)
    x(SHAPE, n=1 << 31)
    x(SHAPE, ldw=49)
    x(SHAPE, ldy=49)
    x(SHAPE, t=-1)
    binding.zs_embed(d, P, None, 8, 0, None, stream=0)  # no tokens: nothing to do
    binding.zs_dense_embed(P, 100, 50, None, 8, 0, None, stream=0)


def test_embed_grad_refusals_and_workspace():
    need = binding.zs_embed_grad_workspace(1000, 500, 64)
    assert need >= 16 * 1000 and need % 256 == 0
    assert binding.zs_embed_grad_workspace(0, 500, 64) == 0 and binding.zs_embed_grad_workspace(-1, 500, 64) == 0
    assert binding.zs_embed_grad_workspace(10, 0, 64) == 0

    def g(status, ids=P, size=8, t=1000, dy=P, kind=binding.ZS_TYPE_F32, dw=P, n=500, k=64, ws=P, room=need, **kw):
        refused(binding.zs_embed_grad, status, ids, size, t, dy, kind, dw, n, k, workspace_dev=ws, workspace_bytes=room, **kw)
    g(ARG, ids=None)
    g(ARG, ids=P + 4)
    g(ARG, dy=None)
    g(ARG, dy=P + 2)
    g(ARG, dw=None)
    g(ARG, dw=P + 2)
    g(ARG, ws=None)
    g(ARG, ws=P + 64)
    g(SIZE, room=need - 1)
    g(CONFIG, size=16)
    g(CONFIG, kind=7)
    g(SHAPE, t=-1)
    g(SHAPE, t=1 << 31)
    g(SHAPE, n=0)
    g(SHAPE, n=1 << 31)
    g(SHAPE, k=0)
    g(SHAPE, lddy=63)
    g(SHAPE, lddw=63)


@pytest.fixture(scope="module")
def asm_of(tmp_path_factory):
    out = tmp_path_factory.mktemp("ops_isa")
    texts = {}
    for src in zs_build.operator_sources():
        to = out / (os.path.basename(src) + ".s")
        cmd = [zs_build.HIPCC, "-S", "--cuda-device-only", src, "-o", str(to)] + \
              [f for f in zs_build.COMMON if f != "-fPIC"] + zs_build.DEVICE
        subprocess.run(cmd, check=True, capture_output=True)
        texts[os.path.basename(src)] = to.read_text()
    return texts


def test_no_private_memory_no_packed_fp32_and_no_lost_store(asm_of):
    seen = 0
    for source, asm in asm_of.items():
        for name, size in re.findall(r"\.amdhsa_kernel (\w+)\n(?:.*\n)*?\s*\.amdhsa_private_segment_fixed_size (\d+)", asm):
            seen += 1
            assert int(size) == 0, f"{source}: {name}: {size} bytes"
        assert not re.search(r"^\s*(scratch_(load|store)|v_pk_(add|mul|fma)_f32)", asm, re.M), source
        stores = 0
        for name, ins in kernels(asm):
            stores += sum(1 for t, _ in ins if WIDE_STORE.match(t))
            found = wide_store_hazards(ins)
            assert not found, f"{source}: {name}: {list(found.values())[:4]}"
        assert stores
    assert seen >= 10
