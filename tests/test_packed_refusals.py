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
