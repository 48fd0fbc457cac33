"""The tests' definitions of attention on packed batches agree with one another (no GPU)."""
import numpy as np
import pytest


@pytest.mark.parametrize("lens,H,Hkv,dh", [([5, 0, 33, 1, 70], 6, 2, 32), ([64], 3, 1, 64), ([1, 17], 4, 4, 128)])
def test_attention_by_torch_is_attention_by_numpy(lens, H, Hkv, dh):
    import packedlib as pl
    rng = np.random.default_rng(3)
    qkv = rng.standard_normal((sum(lens), (H + 2 * Hkv) * dh)).astype(np.float32)
    dO = rng.standard_normal((sum(lens), H * dh)).astype(np.float32)
    for a, b in zip(pl.attention(lens, H, Hkv, dh, qkv, dO, 2.0 ** -8), pl.attention_on("cpu", lens, H, Hkv, dh, qkv, dO, 2.0 ** -8)):
        assert a.shape == b.shape and np.abs(a - b).max() <= 1e-12


@pytest.mark.parametrize("lens,heads,want", [([900, 11], (66, 2, 64), (64, 128, 7)), ([1200, 9], (64, 8, 128), (128, 256, 4)), ([40, 3], (4, 2, 64), (64, 64, 0))])
def test_blocks_are_read_from_the_lists(lens, heads, want):
    import packedlib as pl
    assert pl.blocks(lens, *heads) == want
