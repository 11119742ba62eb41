"""Distillation from a teacher's top logits on the GPU against oracle/student.py, element by element within the bounds that it derives."""
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


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def inputs(seed, T, V, K):
    rng = np.random.default_rng(seed)
    z = (2 * rng.standard_normal((T, V))).astype(np.float16)
    ids = rng.integers(0, V, (T, K)).astype(np.int32)
    teacher = np.sort(6 + 3 * rng.standard_normal((T, K)).astype(np.float16), axis=1)[:, ::-1].copy()
    for t in range(T):
        z[t, ids[t]] = teacher[t] + rng.standard_normal(K).astype(np.float16)
    targets = ids[:, 0].copy()
    targets[rng.random(T) < 0.3] = rng.integers(0, V)
    return z, ids, teacher, targets


def run(L, z, ids, teacher, targets, scale, tau, w, in_place=False):
    zd = dev(z)
    loss, dz = torch.full((len(z),), 5.0, device=DEV), zd if in_place else torch.full_like(zd, 5.0)
    L.lomo_distill(zd, dev(ids), dev(teacher), dev(targets), scale, tau, w, loss, dz)
    return loss.cpu().numpy(), dz.cpu().numpy()


def check(got, want):
    (loss, dz), (el, eg) = want[:2], want[2:]
    for name, a, b, e in (("loss", got[0], loss, el), ("dlogits", got[1], dz, eg)):
        off = np.abs(S.f64(a) - b)
        print(name, "worst share of the bound", np.max(off / np.maximum(e, 1e-300)))
        assert np.isfinite(a).all() and (off <= e).all(), name


@pytest.mark.parametrize("T,V,K,tau,w", [(1, 8, 1, 1.0, 1.0), (5, 16, 3, 2.0, 0.5), (9, 1000, 16, 2.0, 0.0), (7, 4104, 65, 0.5, 0.9), (6, 32000, 64, 1.5, 1.0),
                                         (4, 32008, 1000, 4.0, 0.3), (3, 70008, 1024, 2.0, 0.7), (2, 131080, 127, 1.0, 0.5), (2, 300000, 5, 3.0, 0.9)])
def test_against_the_definition(L, T, V, K, tau, w):
    z, ids, teacher, targets = inputs(T + V, T, V, K)
    scale = 1024.0 / T
    want = S.distill(z, ids, teacher, targets, scale, tau, w)
    got = run(L, z, ids, teacher, targets, scale, tau, w)
    check(got, want)
    again = run(L, z, ids, teacher, targets, scale, tau, w, in_place=True)
    assert np.array_equal(again[0], got[0]) and np.array_equal(again[1].view(np.uint16), got[1].view(np.uint16))


@pytest.mark.parametrize("w", [0.4, 1.0])
def test_what_a_token_may_lack(L, w):
    """Targets and ids outside the vocabulary, ids listed twice, teacher logits of -inf, masked logits of -inf."""
    z, ids, teacher, targets = inputs(1, 12, 264, 9)
    targets[0], targets[1], targets[2] = -100, 264, 263
    ids[3], ids[4, 2:5], ids[5, ::2] = -1, [264, -7, 2 ** 31 - 1], ids[5, 1]
    ids[6], targets[6] = 11, 11                                  # one token, nine times, and the target
    teacher[7], teacher[8, 3:] = -np.inf, -np.inf                # nothing listed; three listed
    z[9] = -np.inf
    z[9, ids[9]], z[9, targets[9]] = 1.0, 2.0                    # all else is masked out of the student
    z[10], teacher[10] = 1.5, 2.5                                # everything alike
    z[11, 5], targets[11] = 60000.0, 5                           # as sure as can be
    with np.errstate(invalid="ignore"):
        want = S.distill(z, ids, teacher, targets, 16.0, 2.0, w)
    want[3][9][z[9] == -np.inf] = S.TINY16                       # their bounds have an infinite logit times a probability of 0
    got = run(L, z, ids, teacher, targets, 16.0, 2.0, w)
    check(got, want)
    assert not got[1][:2].any() and not got[0][:2].any() and not got[1][9][z[9] == -np.inf].any()
    if w == 1.0:
        assert not got[1][3].any() and not got[1][7].any() and got[0][3] == got[0][7] == 0.0


def test_not_finite_stays_in_its_row(L):
    z, ids, teacher, targets = inputs(2, 6, 520, 4)
    clean = run(L, z, ids, teacher, targets, 8.0, 2.0, 0.5)
    z[1, 7], z[3, 9], teacher[4, 1] = np.inf, np.nan, np.nan
    got = run(L, z, ids, teacher, targets, 8.0, 2.0, 0.5)
    for t in (0, 2, 5):
        assert got[0][t] == clean[0][t] and np.array_equal(got[1][t], clean[1][t])
    for t in (1, 3, 4):
        assert not np.isfinite(got[0][t]) and not np.isfinite(got[1][t]).all()


def test_mean(L):
    T, V, K = 200, 1000, 8
    z, ids, teacher, targets = inputs(4, T, V, K)
    targets[::3] = -100
    n, scale = int((targets >= 0).sum()), 4096.0
    want = S.distill(z, ids, teacher, targets, float(np.float32(scale / n)), 2.0, 0.8)
    loss, dz, stats = torch.zeros(T, device=DEV), torch.zeros(T, V, dtype=torch.float16, device=DEV), torch.zeros(3, dtype=torch.float64, device=DEV)
    args = dev(ids), dev(teacher), dev(targets), scale, 2.0, 0.8
    L.lomo_distill_mean(dev(z), *args, loss, dz, stats)
    check((loss.cpu().numpy(), dz.cpu().numpy()), want)
    assert stats[1].item() == n
    assert stats[0].item() == pytest.approx(loss.double().sum().item() / n, rel=1e-12)
    none = torch.full((T,), -100, dtype=torch.int32, device=DEV)
    L.lomo_distill_mean(dev(z), args[0], args[1], none, scale, 2.0, 0.8, loss, dz, stats)
    assert stats[:2].tolist() == [0.0, 0.0] and not bool(dz.any()) and not bool(loss.any())


def test_refusals_stream_and_graph(L):
    T, V, K = 30, 4096, 12
    z, ids, teacher, targets = (dev(x) for x in inputs(8, T, V, K))
    loss, dz = torch.zeros(T, device=DEV), torch.zeros_like(z)
    for bad in (lambda: L.lomo_distill(z.float(), ids, teacher, targets, 1.0, 2.0, 0.5, loss, dz),
                lambda: L.lomo_distill(z, ids.long(), teacher, targets, 1.0, 2.0, 0.5, loss, dz),
                lambda: L.lomo_distill(z, ids, teacher[:, :5], targets, 1.0, 2.0, 0.5, loss, dz),
                lambda: L.lomo_distill(z, ids[:5], teacher[:5], targets, 1.0, 2.0, 0.5, loss, dz),
                lambda: L.lomo_distill(z[:, ::2], ids, teacher, targets, 1.0, 2.0, 0.5, loss, dz[:, ::2]),
                lambda: L.lomo_distill(z, ids, teacher, targets.cpu(), 1.0, 2.0, 0.5, loss, dz),
                lambda: L.lomo_distill(z, ids, teacher, targets, 1.0, 0.0, 0.5, loss, dz),
                lambda: L.lomo_distill(z, ids, teacher, targets, 1.0, 1.0, 1.5, loss, dz)):
        with pytest.raises(L.LomoError):
            bad()
    L.lomo_distill(z, ids, teacher, targets, 2.0, 2.0, 0.5, loss, dz)
    want = loss.clone(), dz.clone()
    side = torch.cuda.Stream()
    for x in (loss, dz):
        x.zero_()
    side.wait_stream(torch.cuda.current_stream())
    L.lomo_distill(z, ids, teacher, targets, 2.0, 2.0, 0.5, loss, dz, stream=side)
    side.synchronize()
    assert torch.equal(loss, want[0]) and torch.equal(dz, want[1])
    stats = torch.zeros(3, dtype=torch.float64, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lomo_distill_mean(z, ids, teacher, targets, 64.0, 2.0, 0.5, loss, dz, stats)
    for _ in range(3):
        z.mul_(-0.5)
        for x in (loss, dz, stats):
            x.zero_()
        graph.replay()
        a, b, c = torch.zeros_like(loss), torch.zeros_like(dz), torch.zeros_like(stats)
        L.lomo_distill_mean(z, ids, teacher, targets, 64.0, 2.0, 0.5, a, b, c)
        torch.cuda.synchronize()
        assert torch.equal(loss, a) and torch.equal(dz, b) and torch.equal(stats[:2], c[:2])


def test_rows_beyond_32_bits(L):
    V, K = 131072, 4
    T = (1 << 31) // V + 50
    z = torch.zeros(T, V, dtype=torch.float16, device=DEV)
    ids, teacher = torch.randint(0, V, (T, K), dtype=torch.int32, device=DEV), torch.randn(T, K, device=DEV).half()
    targets = torch.full((T,), -100, dtype=torch.int32, device=DEV)
    z[T - 1], targets[T - 1] = torch.randn(V, device=DEV).half(), 77
    one = [x[T - 1:].clone() for x in (z, ids, teacher, targets)]
    loss, dz = torch.zeros(1, device=DEV), torch.zeros(1, V, dtype=torch.float16, device=DEV)
    L.lomo_distill(*one, 64.0, 2.0, 0.5, loss, dz)
    all_loss = torch.ones(T, device=DEV)
    L.lomo_distill(z, ids, teacher, targets, 64.0, 2.0, 0.5, all_loss, z)
    assert torch.equal(z[T - 1:], dz) and torch.equal(all_loss[T - 1:], loss) and bool(dz.any())
    assert not bool(all_loss[:T - 1].any()) and not bool(z[:T - 1:97].any())
