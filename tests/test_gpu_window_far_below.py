"""Attention with a window: many keys far below the largest score, which together carry what the result is."""
import math
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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("score", [9.0, 11.5, 13.0, 13.7])
@pytest.mark.parametrize("first", [True, False])
def test_keys_far_below_the_largest(L, d, score, first):
    """One key with v = 0 scores `score` more than all others, whose v is 1: o is their share of the softmax.  Their probabilities, e^-score of the largest,
    are normal fp16 numbers in the kernel down to 2^-21 of it: half a step of 2^-11 for them, another for o, 2^-17 for fp32.
    Where o itself is below the normal range, 2^-14 (the first queries: e^-13 and less), its steps are 2^-24 and its rounding is off by up to 2^-25."""
    n, key = 6000, 0 if first else 5000
    qkv = torch.zeros(n, 3 * d, dtype=torch.float16, device=DEV)
    qkv[:, 0], qkv[key, d], qkv[:, 2 * d:] = 8.0, score * math.sqrt(d) / 8, 1.0
    qkv[key, 2 * d:] = 0.0
    s = 8.0 * float(qkv[key, d]) / math.sqrt(d)
    off = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    o, lse = torch.empty(n, d, dtype=torch.float16, device=DEV), torch.empty(n, 1, device=DEV)
    L.lomo_window_attention_forward(qkv, o, lse, off, 1, 1, n, 0)
    i = np.arange(n)
    others, has = np.where(i >= key, i, i + 1).astype(np.float64), i >= key
    want = np.where(has, others * np.exp(-s) / (1 + others * np.exp(-s)), 1.0)
    got = o[:, d // 2].double().cpu().numpy()
    share = np.abs(got - want) / ((2.0 ** -10 + 2.0 ** -17) * want + 2.0 ** -25)
    assert bool((o == o[:, :1]).all()) and share.max() <= 1, (share.max(), share.argmax())
    np.testing.assert_allclose(lse[:, 0].cpu().numpy(), np.where(has, s + np.log1p(others * np.exp(-s)), np.log(i + 1.0)), rtol=0, atol=1e-5)
