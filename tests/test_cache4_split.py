"""Which attentions over the 4-bit cache are cut along the keys: the workspace says so (no GPU)."""

import pytest


def _bytes(B, n, G=1, hq=32, hkv=8, hd=128, dtype=0, fresh=0):
    from paper_2608_08086_amd import archer as a
    return a.lib.archer_op_attention_cache4_ws_bytes(dtype, B, G, hq, hkv, hd, n, fresh)


@pytest.mark.parametrize("B", [1, 2, 16, 20, 32, 64, 200, 256])
@pytest.mark.parametrize("heads", [(32, 8), (28, 4), (32, 32), (7, 1)])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", [0, 1])
def test_a_long_sequence_is_cut_in_any_batch(B, heads, hd, dtype):
    """max_cached may be one sequence's length alone, and the others short."""
    n = _bytes(B, 131072, hq=heads[0], hkv=heads[1], hd=hd, dtype=dtype)
    # partial results of at most as many chunks as a round of workgroups, or two a sequence
    assert 0 < n <= max(2 * B, 1024 // heads[1]) * heads[0] * (hd + 2) * 4 + 512


def test_short_sequences_and_large_batches_are_not():
    assert _bytes(64, 1000) == 0 and _bytes(257, 131072) == 0
    assert _bytes(16, 131072, G=256, hkv=32) == 0        # many rows: the row kernel takes a sequence whole
    # every sequence has a round of workgroups of its own
    assert _bytes(20, 131072, G=256, hkv=32, dtype=1) == 0 and _bytes(20, 131072, G=240, hkv=32, dtype=1) > 0
    assert _bytes(256, 2**31 - 1) == 0                  # more steps in all than 32 bits count
