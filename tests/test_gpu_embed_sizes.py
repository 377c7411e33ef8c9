"""The embedding operators where the amount of work takes another way through their kernels: four BlockTiles to a wave, more work than
workgroups in a launch.  Definitions and tolerances as in test_gpu_embed.py."""
import numpy as np
import pytest

from paper_2603_17435_amd import binding, inputs
from test_gpu_embed import check_grad, dev, lookup, same, want_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["rowscale", "wide"])
@pytest.mark.parametrize("n,k,t", [(64, 64, 33000), (256, 320, 7000), (256, 384, 5500), (128, 448, 4800)])
def test_packed_lookup_with_four_block_tiles_to_a_wave(kind, n, k, t):
    """One, five, six and seven BlockTiles to a row, padded positions among the tokens (a wave takes four where there are 32768 or more in all)."""
    assert t * (k // 64) >= 32768
    w = inputs.make_weights(kind, n, k, 3) if kind != "wide" else np.random.default_rng(n).integers(0, 1 << 16, (n, k), dtype=np.uint16)
    blob, d = binding.zs_encode(w)
    blob = dev(blob)
    ids = np.random.default_rng(k).integers(-3, n + 3, t)
    ids[-1] = n - 1
    for of in (ids, ids.astype(np.int32)):
        for scale, ldy in ((1.0, k), (0.3, k + 1)):
            got = lookup(lambda *a, **kw: binding.zs_embed(d, blob, *a, **kw), of, k, ldy=ldy, scale=scale)
            assert same(got, want_rows(w, of, scale))


def test_more_tokens_than_workgroups():
    """A launch has 2^20 workgroups at most."""
    import torch
    n, k, t = 192, 64, (1 << 20) + 77
    w = inputs.make_weights("gauss", n, k, 9)
    blob, d = binding.zs_encode(w)
    table = dev(w.view(np.int16))
    gen = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(-1, n, (t,), generator=gen, device="cuda", dtype=torch.int32)
    want = torch.where((ids >= 0)[:, None], table[ids.clamp_min(0).long()], torch.zeros((), dtype=torch.int16, device="cuda"))
    y = torch.full((t, k), 7, dtype=torch.int16, device="cuda")
    binding.zs_embed(d, dev(blob), ids, 4, t, y)
    assert torch.equal(y, want)


def test_dense_lookup_of_more_pieces_than_threads():
    """2^28 pieces of eight columns are what a launch takes at a time."""
    import torch
    n, k, t = 500, 2048, (1 << 20) + 5
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB")
    gen = torch.Generator(device="cuda").manual_seed(2)
    w = torch.randn(n, k, generator=gen, device="cuda").to(torch.bfloat16)
    ids = torch.randint(0, n, (t,), generator=gen, device="cuda", dtype=torch.int32)
    y = torch.empty(t, k, dtype=torch.bfloat16, device="cuda")
    binding.zs_dense_embed(w, n, k, ids, 4, t, y)
    assert torch.equal(y, w[ids.long()])


def test_grad_of_more_chunks_than_workgroups():
    """2^24 tokens and some: four rounds of merges, in which the workgroups go round, as they do for the sums."""
    n, t = 3000, (1 << 24) + 1000
    rng = np.random.default_rng(6)
    ids = np.minimum(np.exp(rng.random(t) * np.log(n + 2)).astype(np.int32) - 1, n)  # (n has no row)
    check_grad(ids, rng.standard_normal((t, 1), dtype=np.float32), n, 0.5)
