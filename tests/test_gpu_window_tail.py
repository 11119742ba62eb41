"""Attention backward: the rows behind a sequence's last query, which fill up its last tile, add nothing to any key."""
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


@pytest.mark.parametrize("n,window,sinks,key", [(60, 60, 0, 5), (64, 64, 0, 5), (700, 5000, 0, 70), (704, 5000, 0, 70), (500, 90, 6, 5), (512, 90, 6, 5),
                                                (200, 100, 0, 190), (333, 40, 0, 330)])
@pytest.mark.parametrize("d", [64, 128])
def test_a_key_that_no_query_takes_has_no_gradient(L, d, n, window, sinks, key):
    """One infinite element of a key that every query scores with -inf: P = 0 and dS = 0 there, so dk and dv of the key are 0, whether the
    sequence ends with a whole tile or not; all other keys have the gradients that they have where the key is finite and far away."""
    h, g, col = 2, 1, 9
    rng = np.random.default_rng(n + key)
    qkv = rng.standard_normal((n, (h + 2 * g) * d)).astype(np.float16)
    do = (3 * rng.standard_normal((n, h * d))).astype(np.float16)
    for a in range(h):
        qkv[:, a * d + col] = -np.abs(qkv[:, a * d + col]) - np.float16(0.5)
    got = []
    for value in (np.inf, 60000.0):      # -60000 * 0.5 / sqrt(d): a probability of 0 as well
        qkv[key, h * d + col] = value
        x, u = torch.from_numpy(qkv).to(DEV), torch.from_numpy(do).to(DEV)
        off = torch.tensor([0, n], dtype=torch.int32, device=DEV)
        o, lse, dqkv = torch.empty_like(u), torch.empty(n, h, device=DEV), torch.empty_like(x)
        ws = torch.full((L.lomo_window_attention_workspace_bytes(n, 1, h, g, d, sinks),), 255, dtype=torch.uint8, device=DEV)
        L.lomo_window_attention_forward(x, o, lse, off, h, g, window, sinks)
        L.lomo_window_attention_backward(x, o, u, lse, dqkv, off, h, g, window, sinks, ws)
        got.append(dqkv.view(n, h + 2 * g, d)[:, h:])
        assert bool(lse.isfinite().all())
    assert not bool(got[0][key].any()) and torch.equal(got[0], got[1])
