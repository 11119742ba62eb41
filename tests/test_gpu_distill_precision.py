"""Distillation where fp32 exponents are long: large logits, small temperatures; and teachers that are not finite."""
import os

import numpy as np
import pytest
import torch

from oracle import student as S

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


def run(L, z, ids, teacher, targets, scale, tau, w):
    f = lambda a, t: torch.from_numpy(np.ascontiguousarray(a, dtype=t)).to(DEV)
    zd = f(z, np.float16)
    loss, dz = torch.full((len(z),), 5.0, device=DEV), torch.full_like(zd, 5.0)
    L.lomo_distill(zd, f(ids, np.int32), f(teacher, np.float16), f(targets, np.int32), scale, tau, w, loss, dz)
    return loss.cpu().numpy().astype(np.float64), dz.cpu().numpy().astype(np.float64)


def rows(seed, T, V, K):
    rng = np.random.default_rng(seed)
    z, teacher = rng.standard_normal((T, V)).astype(np.float16), rng.standard_normal((T, K)).astype(np.float16)
    ids = rng.integers(0, V, (T, K))
    return z, ids, teacher, ids[:, 0]


@pytest.mark.parametrize("tau", [1.0, 2.0])
def test_a_teacher_without_weight_does_not_matter(L, tau):
    z, ids, teacher, targets = rows(5, 5, 520, 4)
    clean = run(L, z, ids, teacher, targets, 16.0, tau, 0.0)
    for t, value in enumerate((np.nan, np.inf, -np.inf)):
        teacher[t, 2] = value
    teacher[3] = np.nan
    got = run(L, z, ids, teacher, targets, 16.0, tau, 0.0)
    assert np.array_equal(got[0], clean[0]) and np.array_equal(got[1], clean[1]) and np.isfinite(clean[1]).all()
