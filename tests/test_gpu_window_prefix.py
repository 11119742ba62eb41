"""Attention with a window: what a query does not see does not change a bit of its result, large finite scores of its neighbours included."""
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def L():
    import paper_2306_09782_amd as L
    if not os.path.exists(L.library_path()):
        from paper_2306_09782_amd.build import build
        build(verbose=False)
    L.load_library()
    return L


def run(L, qkv, do, h, g, window, sinks):
    n, d = qkv.shape[0], do.shape[1] // h
    off = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    o, lse, dqkv = torch.empty_like(do), torch.empty(n, h, device=DEV), torch.empty_like(qkv)
    ws = torch.full((L.lomo_window_attention_workspace_bytes(n, 1, h, g, d, sinks),), 255, dtype=torch.uint8, device=DEV)
    L.lomo_window_attention_forward(qkv, o, lse, off, h, g, window, sinks)
    L.lomo_window_attention_backward(qkv, o, do, lse, dqkv, off, h, g, window, sinks, ws)
    return o, lse, dqkv[:, :h * d].contiguous()


def inputs(seed, n, h, g, d, sharp):
    rng = np.random.default_rng(seed)
    qkv = rng.standard_normal((n, (h + 2 * g) * d)).astype(np.float16)
    qkv[:, :h * d] *= np.float16(sharp)
    return torch.from_numpy(qkv).to(DEV), torch.from_numpy(rng.standard_normal((n, h * d)).astype(np.float16)).to(DEV)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,window,sinks", [(900, 5000, 0), (900, 200, 4)])
def test_a_prefix_has_the_bits_of_the_whole(L, d, n, window, sinks):
    h, g = 4, 2
    qkv, do = inputs(n + window, n, h, g, d, 4.0)      # scores of 4: references move
    whole = run(L, qkv, do, h, g, window, sinks)
    for m in (1, 37, 128, 333, 640, 899):
        for x, y in zip(whole, run(L, qkv[:m].contiguous(), do[:m].contiguous(), h, g, window, sinks)):
            assert torch.equal(x[:m], y), m


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window,sinks,key", [(5000, 0, 333), (100, 3, 333), (100, 3, 1)])
def test_a_large_key_changes_those_that_see_it_alone(L, d, window, sinks, key):
    """A key whose scores are large, finite or +inf: queries that do not see it keep every bit of o, lse and dq."""
    n, h, g = 600, 4, 2
    qkv, do = inputs(key, n, h, g, d, 1.0)
    clean = run(L, qkv, do, h, g, window, sinks)
    i = torch.arange(n, device=DEV)
    hit = (i >= key) & ((i - key < window) | (key < sinks))
    for column, value in (slice(0, None), 40.0), (slice(0, None), -40.0), (3, 60000.0), (3, float("inf")):
        x = qkv.clone()
        x.view(n, h + 2 * g, d)[key, h:h + g, column] = value
        for got, was in zip(run(L, x, do, h, g, window, sinks), clean):
            assert torch.equal(got[~hit], was[~hit]), value
            assert not torch.equal(got[hit], was[hit]), value
