"""What the calls on packed batches refuse before any launch (CPU)."""
import os

import pytest

import paper_2306_09782_amd as L


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.library_path()):
        from paper_2306_09782_amd.build import build
        build(verbose=False)
    return L.load_library()


def test_clear_padding_arguments(lib):
    call = lambda x, off, T, B, width: lib.lomo_clear_padding(x, off, T, B, width, None)
    for T, B, width in ((-1, 1, 8), (4, -1, 8), (4, 1, -8), (4, 1, 12), (1 << 31, 1, 8), (4, 1, 1 << 31)):
        assert call(16, 16, T, B, width) == 2
    assert call(None, 16, 4, 1, 8) == 1 and call(16, None, 4, 1, 8) == 1
    assert call(None, None, 0, 1, 8) == 0 and call(None, None, 4, 1, 0) == 0
    with pytest.raises(L.LomoError):
        L.binding._check(call(24, 16, 4, 1, 8))
    with pytest.raises(L.LomoError):
        L.binding._check(call(16, 18, 4, 1, 8))


def test_a_sequence_longer_than_the_rotary_tables(lib):
    """Positions that the batch counts by itself have to be in the tables: pairs beyond them would stay unturned."""
    import torch
    from paper_2306_09782_amd.chain import PackedAttention
    packed = PackedAttention("cpu", 100, 2, 1, 64)
    qkv, o, lse = torch.zeros(100, 256, dtype=torch.float16), torch.zeros(100, 128, dtype=torch.float16), torch.zeros(100, 2)
    cos, sin = torch.ones(40, 32), torch.zeros(40, 32)
    packed.set_batch([30, 41, 2])
    with pytest.raises(L.LomoError, match="41 tokens"):
        packed.forward(qkv, cos, sin, o, lse)
    for lengths, positions in (([40, 40], None), ([], None), ([100], torch.full((1, 100), 39, dtype=torch.int32)), ([100], torch.full((1, 100), -1, dtype=torch.int32))):
        packed.set_batch(lengths, positions)
        with pytest.raises(L.LomoError, match="x is on cpu"):      # taken, up to the device
            packed.forward(qkv, cos, sin, o, lse)


def test_axes_of_pairs_from_any_sequence():
    """Lists, tuples, bytes, tensors and arrays of any whole type name the same axes; numbers that are no axes are refused."""
    import numpy as np
    import torch
    from paper_2306_09782_amd.chain import PackedAttention
    want = bytes([0, 1] * 16)
    for given in (want, bytearray(want), list(want), tuple(want), np.array(list(want)), np.array(list(want), dtype=np.int32),
                  np.array(list(want), dtype=np.uint8), torch.tensor(list(want))):
        packed = PackedAttention("cpu", 8, 2, 1, 64, pair_axis=given)
        assert packed.pair_axis == want and packed.positions.shape == (2, 8)
    for bad in (32, [0, -1] * 16, [0, 256] * 16, ["a"] * 32, 1.5):
        with pytest.raises(L.LomoError):
            PackedAttention("cpu", 8, 2, 1, 64, pair_axis=bad)
