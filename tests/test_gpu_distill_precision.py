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


def definition(z, ids, teacher, target, tau, w):
    """One token: loss, gradient, and the size of what their errors are relative to."""
    z, t = z.astype(np.float64), teacher.astype(np.float64)
    log_p = (t - t.max()) / tau - np.log(np.exp((t - t.max()) / tau).sum())
    log_q = (z - z.max()) / tau - np.log(np.exp((z - z.max()) / tau).sum())
    log_1 = (z - z.max()) - np.log(np.exp(z - z.max()).sum())
    p = np.exp(log_p)
    loss = -(1 - w) * log_1[target] + w * tau ** 2 * (p * (log_p - log_q[ids])).sum()
    size = (1 - w) * (1 - log_1[target]) + w * tau ** 2 * (1 + (p * (abs(log_p) + abs(log_q[ids]))).sum())
    grad = (1 - w) * np.exp(log_1) + w * tau * np.exp(log_q)
    grad[target] -= 1 - w
    np.subtract.at(grad, ids, w * tau * p)
    return loss, grad, size


# fp32 arguments of exponentials of up to 64 (what is below adds nothing), 2^-24 of each, and sums of 2^10 terms: 2^-17 covers them
NEAR = 2.0 ** -17


@pytest.mark.parametrize("tau,shift,step", [(2.0 ** -10, 60000.0, 32.0), (2.0 ** -6, 20.0, 2.0 ** -6), (2.0 ** -8, 1000.0, 1.0), (2.0, 30000.0, 16.0),
                                            (2.0 ** 10, 30000.0, 16.0)])
@pytest.mark.parametrize("w", [0.6, 1.0])
def test_differences_of_large_teacher_logits(L, tau, shift, step, w):
    T, V, K = 8, 64, 9
    rng = np.random.default_rng(3)
    z = rng.standard_normal((T, V)).astype(np.float16) * np.float16(min(tau, 1.0))
    ids = np.stack([rng.permutation(V)[:K] for _ in range(T)])
    teacher = (shift + step * rng.integers(-3, 1, (T, K))).astype(np.float16)
    teacher[0] = teacher[0, 0]                       # all alike
    targets, scale = ids[:, 1], 8.0 / min(tau, 1.0)
    loss, dz = run(L, z, ids, teacher, targets, scale, tau, w)
    for t in range(T):
        want, grad, size = definition(z[t], ids[t], teacher[t], targets[t], tau, w)
        grad, most = scale * grad, scale * ((1 - w) + w * tau)
        assert abs(loss[t] - want) <= NEAR * size, (t, loss[t], want)
        assert (np.abs(dz[t] - grad) <= S.H16 * np.abs(grad) + NEAR * most + S.TINY16).all(), t


@pytest.mark.parametrize("shift", [0.0, 1000.0, 30000.0, 60000.0, -60000.0])
@pytest.mark.parametrize("w,tau", [(0.0, 2.0), (0.5, 1.0), (0.5, 4.0)])
def test_loss_of_large_logits(L, shift, w, tau):
    T, V, K = 6, 1000, 5
    rng = np.random.default_rng(4)
    z = (shift + 2 * rng.standard_normal((T, V))).astype(np.float16)
    ids = np.stack([rng.permutation(V)[:K] for _ in range(T)])
    teacher, targets = rng.standard_normal((T, K)).astype(np.float16), ids[:, 2]
    loss, dz = run(L, z, ids, teacher, targets, 64.0, tau, w)
    for t in range(T):
        want, grad, size = definition(z[t], ids[t], teacher[t], targets[t], tau, w)
        assert abs(loss[t] - want) <= NEAR * size, (t, loss[t], want)
        assert (np.abs(dz[t] - 64 * grad) <= (S.H16 + NEAR) * np.abs(64 * grad) + 64 * NEAR * tau + S.TINY16).all(), t


@pytest.mark.parametrize("w", [0.5, 1.0])
@pytest.mark.parametrize("K", [1, 4, 700])
def test_a_teacher_of_nothing_but_nan_is_seen(L, w, K):
    z, ids, teacher, targets = rows(6, 4, 520, K)
    clean = run(L, z, ids, teacher, targets, 16.0, 2.0, w)
    teacher[1], teacher[2, 1:] = np.nan, -np.inf      # all NaN; one listed
    teacher[3, -1] = np.nan
    got = run(L, z, ids, teacher, targets, 16.0, 2.0, w)
    assert got[0][0] == clean[0][0] and np.array_equal(got[1][0], clean[1][0])
    for t in (1, 3):
        assert not np.isfinite(got[0][t]) and not np.isfinite(got[1][t]).all(), t
    assert np.isfinite(got[0][2]) and np.isfinite(got[1][2]).all()
