"""oracle/student.py: gradients against differences, definitions against their special cases, and what the calls refuse (no GPU work)."""
import ctypes
import os

import numpy as np
import pytest
import torch

import paper_2306_09782_amd as L
from oracle import attn_chain as A
from oracle import loss as CE
from oracle import student as S


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(L.library_path()):
        from paper_2306_09782_amd.build import build
        build(verbose=False)
    return L.load_library()


def test_rope_with_one_position_on_all_axes_is_the_plain_step():
    rng = np.random.default_rng(0)
    s, nh, d = 12, 2, 128
    cos, sin = A.rope_tables(s, d)
    x = rng.standard_normal((s, nh * d))
    pos = np.tile(np.arange(s), (3, 1))
    axes = rng.integers(0, 3, d // 2)
    y, _ = S.rope_axes(x, cos, sin, pos, axes, nh, d)
    np.testing.assert_allclose(y, A.rope_rotate(x, cos, sin, s, nh), atol=1e-12)
    back, _ = S.rope_axes(y, cos, sin, pos, axes, nh, d, inverse=True)
    np.testing.assert_allclose(back, x, atol=1e-6)      # the tables are fp32: cos^2 + sin^2 = 1 to 2^-23
    same, _ = S.rope_axes(x, cos, sin, pos + s, axes, nh, d)      # no such position
    np.testing.assert_array_equal(same, x)


def test_window_attention_without_a_limit_is_causal_attention():
    rng = np.random.default_rng(1)
    s, nh, d = 64, 2, 128
    qkv = rng.standard_normal((2 * s, 3 * nh * d)).astype(np.float16)
    o, lse, _, _ = S.window_attention_forward(qkv, [0, s, 2 * s], nh, nh, 10 ** 9, 0)
    want = A.attention_forward_stored(qkv, s, nh)
    np.testing.assert_allclose(lse, want["lse"], rtol=2e-7, atol=2e-7)
    assert np.abs(o - S.f64(want["o"])).max() <= 2.0 ** -9 * np.abs(o).max()


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (5, 0), (100, 4)])
def test_window_attention_gradient_against_differences(window, sinks):
    rng = np.random.default_rng(window)
    h, g, d, off = 4, 2, 8, [0, 7, 7, 16]
    qkv, do = rng.standard_normal((18, (h + 2 * g) * d)), rng.standard_normal((18, h * d))
    f = lambda x: np.nansum(S.window_attention_forward(x, off, h, g, window, sinks)[0] * do)
    o, lse, _, _ = S.window_attention_forward(qkv, off, h, g, window, sinks)
    grad, _ = S.window_attention_backward(qkv, o, do, lse, off, h, g, window, sinks)
    assert np.isnan(grad[16:]).all() and not np.isnan(grad[:16]).any()
    for r, c in zip(rng.integers(0, 16, 40), rng.integers(0, qkv.shape[1], 40)):
        step = np.zeros_like(qkv)
        step[r, c] = 1e-5
        assert grad[r, c] == pytest.approx((f(qkv + step) - f(qkv - step)) / 2e-5, abs=2e-8)


@pytest.mark.parametrize("tau,w", [(1.0, 1.0), (2.0, 0.5), (0.7, 0.9), (3.0, 0.0)])
def test_distill_gradient_against_differences(tau, w):
    rng = np.random.default_rng(7)
    T, V, K = 5, 16, 4
    z, teacher = rng.standard_normal((T, V)), rng.standard_normal((T, K))
    ids = rng.integers(0, V, (T, K))
    ids[1, 2], ids[2], teacher[3, 1] = ids[1, 0], -1, -np.inf      # listed twice, nothing listed, no share
    targets = np.array([3, 0, 5, -100, 15])
    f = lambda x: S.distill(x, ids, teacher, targets, 1.0, tau, w)[0].sum()
    grad = S.distill(z, ids, teacher, targets, 2.0, tau, w)[1]
    assert not grad[3].any() and (w == 1.0) == (not grad[2].any())
    np.testing.assert_allclose(grad.sum(1), 0.0, atol=1e-12)
    for r in range(T):
        for c in range(V):
            step = np.zeros_like(z)
            step[r, c] = 1e-5
            assert grad[r, c] == pytest.approx((f(z + step) - f(z - step)) / 1e-5, abs=1e-8)


def test_distill_without_a_teachers_weight_is_cross_entropy():
    rng = np.random.default_rng(3)
    z, targets = rng.standard_normal((6, 24)), np.array([0, 23, -100, 5, 24, 7])
    want = CE.cross_entropy(z, targets, 8.0)
    loss, grad, _, _ = S.distill(z, rng.integers(0, 24, (6, 3)), rng.standard_normal((6, 3)), targets, 8.0 / want["n"], 2.0, 0.0)
    np.testing.assert_allclose(loss, want["token_losses"], atol=1e-12)
    np.testing.assert_allclose(grad, want["dlogits"], atol=1e-12)


def test_distill_from_a_teacher_that_lists_everything_is_the_whole_divergence():
    rng = np.random.default_rng(4)
    z, t, tau = rng.standard_normal((3, 8)), rng.standard_normal((3, 8)), 1.7
    log = lambda x: x / tau - np.log(np.exp(x / tau).sum(1, keepdims=True))
    loss = S.distill(z, np.tile(np.arange(8), (3, 1)), t, np.zeros(3), 1.0, tau, 1.0)[0]
    np.testing.assert_allclose(loss, tau ** 2 * (np.exp(log(t)) * (log(t) - log(z))).sum(1), atol=1e-12)


# ------------------------------------------------------------------------------------------------------- refusals

OK, NULL, SHAPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4
P = None
A16, ODD, ODD4 = 64, 72, 66      # addresses of nothing: every check comes before the first launch


def test_rope_axes_refusals(lib):
    axes = bytes(64)

    def call(x=P, ldx=256, y=P, ldy=256, cos=P, sin=P, rows=4, pos=P, n_axes=1, axes=axes, T=4, heads=2, d=128):
        return lib.lomo_rope_axes(x, ldx, y, ldy, cos, sin, rows, pos, n_axes, axes, T, heads, d, 0, P)

    for bad in (dict(T=-1), dict(rows=-1), dict(n_axes=0), dict(n_axes=9), dict(heads=-1), dict(d=24), dict(d=8), dict(d=272), dict(ldx=248),
                dict(ldy=255), dict(ldx=260), dict(axes=bytes([1] * 64)), dict(x=A16, y=A16, ldx=264)):
        assert call(**bad) == SHAPE, bad
    assert call(axes=P) == NULL and call() == NULL and call(x=A16, y=A16, pos=A16) == NULL
    full = dict(x=A16, y=A16, cos=A16, sin=A16, pos=A16)
    for name, at in (("x", ODD), ("y", ODD), ("cos", ODD4), ("sin", ODD4), ("pos", ODD4)):
        assert call(**{**full, name: at}) == ALIGN, name
    assert call(T=0) == OK and call(heads=0) == OK


def test_window_attention_refusals(lib):
    def forward(qkv=P, o=P, lse=P, off=P, T=100, B=2, h=4, g=2, d=128, window=8, sinks=4):
        return lib.lomo_window_attention_forward(qkv, o, lse, off, T, B, h, g, d, window, sinks, P)

    def backward(qkv=P, o=P, do=P, lse=P, dqkv=P, off=P, T=100, B=2, h=4, g=2, d=128, window=8, sinks=4, ws=P, n=0):
        return lib.lomo_window_attention_backward(qkv, o, do, lse, dqkv, off, T, B, h, g, d, window, sinks, ws, n, P)

    for bad in (dict(T=-1), dict(B=-1), dict(h=0), dict(g=0), dict(h=5), dict(d=96), dict(d=256), dict(window=0), dict(window=-3), dict(sinks=-1),
                dict(sinks=65), dict(T=(1 << 30) + 1), dict(B=(1 << 24) + 1), dict(h=1 << 17), dict(T=1 << 30, h=512)):
        assert forward(**bad) == SHAPE and backward(**bad) == SHAPE, bad
    assert forward() == NULL and backward() == NULL
    for empty in (dict(T=0), dict(B=0)):
        assert forward(**empty) == OK and backward(**empty) == OK
    full = dict(qkv=A16, o=A16, lse=A16, off=A16)
    for name, at in (("qkv", ODD), ("o", ODD), ("lse", ODD4), ("off", ODD4)):
        assert forward(**{**full, name: at}) == ALIGN, name
    full.update(do=A16, dqkv=A16)
    for name, at in (("do", ODD), ("dqkv", ODD), ("ws", ODD)):
        assert backward(**{**full, name: at}) == ALIGN, name
    need = lib.lomo_window_attention_workspace_bytes(100, 2, 4, 2, 128, 4)
    assert need >= 4 * 100 * 4 and backward(**full) == WORKSPACE and backward(**full, ws=A16, n=need - 1) == WORKSPACE
    size = lambda *a: lib.lomo_window_attention_workspace_bytes(*a)
    assert size(0, 2, 4, 2, 128, 4) == size(100, 0, 4, 2, 128, 4) == size(100, 2, 4, 3, 128, 4) == size(100, 2, 4, 2, 128, 65) == 0
    assert size(1 << 20, 1, 64, 64, 128, 64) > 1 << 32


def test_distill_refusals(lib):
    def call(z=P, ids=P, teacher=P, targets=P, tau=2.0, w=0.5, loss=P, dz=P, T=4, V=16, K=3):
        return lib.lomo_distill(z, ids, teacher, targets, 1.0, tau, w, loss, dz, T, V, K, P)

    def mean(z=P, ids=P, teacher=P, targets=P, tau=2.0, w=0.5, loss=P, dz=P, T=4, V=16, K=3, scale=1.0, stats=P):
        return lib.lomo_distill_mean(z, ids, teacher, targets, scale, tau, w, loss, dz, stats, T, V, K, P)

    nan, inf = float("nan"), float("inf")
    for bad in (dict(T=-1), dict(V=-8), dict(V=12), dict(V=0), dict(K=0), dict(K=1025), dict(tau=0.0), dict(tau=-1.0), dict(tau=nan), dict(tau=inf),
                dict(w=-0.1), dict(w=1.1), dict(w=nan), dict(T=1 << 31)):
        assert call(**bad) == SHAPE and mean(**bad) == SHAPE, bad
    assert call() == NULL and mean() == NULL and mean(scale=0.0) == SHAPE and mean(scale=nan) == SHAPE and call(T=0) == OK and mean(T=0) == NULL
    full = dict(z=A16, ids=A16, teacher=A16, targets=A16, loss=A16, dz=A16)
    for name, at in (("z", ODD), ("ids", ODD4), ("teacher", 65), ("targets", ODD4), ("loss", ODD4), ("dz", ODD)):
        assert call(**{**full, name: at}) == ALIGN and mean(**{**full, name: at}) == ALIGN, name
    assert mean(**full) == NULL and mean(**full, stats=68) == ALIGN


def test_binding_refuses_what_it_cannot_pass_on():
    half, single, whole = (lambda *s, t=t: torch.zeros(*s, dtype=t) for t in (torch.float16, torch.float32, torch.int32))
    with pytest.raises(L.LomoError, match="current device"):
        L.lomo_rope_axes(half(4, 128), half(4, 128), single(4, 64), single(4, 64), whole(1, 4), [0] * 64, 1, 128)
    with pytest.raises(L.LomoError, match="current device"):
        L.lomo_window_attention_forward(half(4, 384), half(4, 128), single(4, 1), whole(2), 1, 1, 4)
    with pytest.raises(L.LomoError, match="current device"):
        L.lomo_distill(half(4, 16), whole(4, 2), half(4, 2), whole(4), 1.0, 1.0, 0.5, single(4), half(4, 16))


def test_refusals_of_what_no_launch_holds(lib):
    """Launches of 2^32 threads and more, temperatures at which fp32 exponents of fp16 logits mean nothing: before anything is launched."""
    window = lib.lomo_window_attention_forward
    assert window(A16, A16, A16, A16, 100, 1 << 24, 4, 2, 128, 8, 4, P) == SHAPE
    assert lib.lomo_window_attention_workspace_bytes(100, 1 << 24, 4, 2, 128, 4) == 0
    assert lib.lomo_rope_axes(A16, 256, A16, 256, A16, A16, 4, A16, 1, bytes(128), 1 << 28, 1, 256, 0, P) == SHAPE
    for tau, T in ((2.0 ** -11, 4), (2.0 ** 11, 4), (1.0, 1 << 22)):
        assert lib.lomo_distill(A16, A16, A16, A16, 1.0, tau, 0.5, A16, A16, T, 16, 3, P) == SHAPE
        assert lib.lomo_distill_mean(A16, A16, A16, A16, 1.0, tau, 0.5, A16, A16, A16, T, 16, 3, P) == SHAPE


def test_packed_attention_wants_a_batch_first(lib):
    from paper_2306_09782_amd.chain import PackedAttention
    packed = PackedAttention("cpu", 10, 2, 1, 64, window=4)
    half = lambda *s: torch.zeros(*s, dtype=torch.float16)
    with pytest.raises(L.LomoError, match="set_batch"):
        packed.forward(half(10, 256), torch.zeros(10, 32), torch.zeros(10, 32), half(10, 128), torch.zeros(10, 2))
    for lengths in ([11], [5, -1], [1] * 65):
        with pytest.raises(L.LomoError, match="sequences"):
            packed.set_batch(lengths)
