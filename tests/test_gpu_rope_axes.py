"""Rotary positions with several axes on the GPU against oracle/student.py."""
import os

import numpy as np
import pytest
import torch

from oracle import attn_chain as A
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


def tables(P, d, base=1e6):
    angle = np.arange(P)[:, None] * base ** (-np.arange(d // 2) / (d // 2))[None, :]
    return np.cos(angle).astype(np.float32), np.sin(angle).astype(np.float32)


@pytest.mark.parametrize("T,heads,d,axes,P,wide", [(1, 1, 128, 1, 5, 0), (37, 3, 64, 3, 900, 64), (130, 10, 128, 3, 300, 256), (77, 5, 16, 2, 50, 8),
                                                   (65, 33, 256, 8, 1000, 0), (300, 2, 96, 2, 70000, 16)])
@pytest.mark.parametrize("inverse", [False, True])
def test_against_the_definition(L, T, heads, d, axes, P, wide, inverse):
    rng = np.random.default_rng(T + d)
    cos, sin = tables(P, d)
    x = rng.standard_normal((T, heads * d + wide)).astype(np.float16)
    pos = rng.integers(0, P, (axes, T)).astype(np.int32)
    pos[rng.random((axes, T)) < 0.05] = rng.choice([-1, P, 2 ** 31 - 1, -2 ** 31])      # outside the tables: not turned
    for axis in (np.sort(rng.integers(0, axes, d // 2)), rng.integers(0, axes, d // 2), np.zeros(d // 2, int)):
        want, bound = S.rope_axes(x, cos, sin, pos, axis, heads, d, inverse)
        y = torch.full((T, heads * d + wide), 5.0, dtype=torch.float16, device=DEV)
        L.lomo_rope_axes(dev(x), y, dev(cos), dev(sin), dev(pos), [int(a) for a in axis], heads, d, inverse=inverse)
        got = y.cpu().numpy()
        assert (np.abs(S.f64(got[:, :heads * d]) - want) <= bound).all()
        assert (got[:, heads * d:] == 5.0).all()
        z = dev(x)
        L.lomo_rope_axes(z, z, dev(cos), dev(sin), dev(pos), [int(a) for a in axis], heads, d, inverse=inverse)      # in place
        assert torch.equal(z[:, :heads * d], y[:, :heads * d]) and np.array_equal(z[:, heads * d:].cpu().numpy(), x[:, heads * d:])


def test_rows_of_wider_buffers_and_one_axis_as_the_plain_step(L):
    rng = np.random.default_rng(3)
    s, nh, d = 48, 2, 128
    cos, sin = (dev(t) for t in A.rope_tables(s, d))
    qkv = dev(rng.standard_normal((2 * s, 3 * nh * d)).astype(np.float16))
    want = qkv.clone()
    L.lomo_rope_forward(want, cos, sin, s, nh)
    pos = dev(np.tile(np.arange(s, dtype=np.int32), (3, 2)))
    got = torch.zeros(2 * s, 5 * nh * d, dtype=torch.float16, device=DEV)
    L.lomo_rope_axes(qkv, got[:, 8:8 + 2 * nh * d], cos, sin, pos, [c % 3 for c in range(64)], 2 * nh, d)
    # each is within the bound of the definition, so they are within two of each other (the compiler rounds some of the plain step's sums to fp32
    # before it rounds them to fp16, and others at once)
    _, bound = S.rope_axes(qkv.cpu().numpy(), cos.cpu().numpy(), sin.cpu().numpy(), pos.cpu().numpy(), [c % 3 for c in range(64)], 2 * nh, d)
    off = (got[:, 8:8 + 2 * nh * d].double() - want[:, :2 * nh * d].double()).abs().cpu().numpy()
    assert (off <= 2 * bound).all() and (off == 0).mean() > 0.99
    assert not bool(got[:, :8].any()) and not bool(got[:, 8 + 2 * nh * d:].any())


def test_turning_back_is_the_gradient(L):
    rng = np.random.default_rng(5)
    T, heads, d = 20, 2, 64
    cos, sin = tables(40, d)
    pos, axis = rng.integers(0, 40, (3, T)).astype(np.int32), rng.integers(0, 3, d // 2)
    f = lambda x: S.rope_axes(x, cos, sin, pos, axis, heads, d)[0]
    dy = rng.standard_normal((T, heads * d)).astype(np.float16)
    x = rng.standard_normal((T, heads * d))
    dx = torch.empty(T, heads * d, dtype=torch.float16, device=DEV)
    L.lomo_rope_axes(dev(dy), dx, dev(cos), dev(sin), dev(pos), [int(a) for a in axis], heads, d, inverse=True)
    for r, c in zip(rng.integers(0, T, 30), rng.integers(0, heads * d, 30)):
        step = np.zeros_like(x)
        step[r, c] = 0.5      # the step is linear
        want = ((f(x + step) - f(x - step)) * S.f64(dy)).sum()
        assert abs(float(dx[r, c]) - want) <= 2.0 ** -11 * abs(want) + 1e-6


def test_refusals_empty_calls_stream_and_graph(L):
    T, d = 50, 128
    x = torch.randn(T, 2 * d, device=DEV).half()
    cos, sin = (dev(t) for t in tables(60, d))
    pos = torch.arange(T, dtype=torch.int32, device=DEV)[None].contiguous()
    y, axis = torch.zeros_like(x), [0] * 64
    for bad in (lambda: L.lomo_rope_axes(x.float(), y, cos, sin, pos, axis, 2, d), lambda: L.lomo_rope_axes(x, y[:40], cos, sin, pos, axis, 2, d),
                lambda: L.lomo_rope_axes(x, y, cos, sin[:59], pos, axis, 2, d), lambda: L.lomo_rope_axes(x, y, cos, sin, pos.long(), axis, 2, d),
                lambda: L.lomo_rope_axes(x, y, cos, sin, pos, axis[:63], 2, d), lambda: L.lomo_rope_axes(x, y, cos, sin, pos, [1] * 64, 2, d),
                lambda: L.lomo_rope_axes(x, y, cos, sin, pos, axis, 3, d), lambda: L.lomo_rope_axes(x, y, cos.cpu(), sin, pos, axis, 2, d),
                lambda: L.lomo_rope_axes(x.t().contiguous().t(), y, cos, sin, pos, axis, 2, d),
                lambda: L.lomo_rope_axes(x[:, 1:], y, cos, sin, pos, axis, 1, d)):
        with pytest.raises(L.LomoError):
            bad()
    L.lomo_rope_axes(x[:0], y[:0], cos, sin, pos[:, :0].contiguous(), axis, 2, d)
    L.lomo_rope_axes(x, y, cos, sin, pos, axis, 2, d)
    want = y.clone()
    side = torch.cuda.Stream()
    y.zero_()
    side.wait_stream(torch.cuda.current_stream())
    L.lomo_rope_axes(x, y, cos, sin, pos, axis, 2, d, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lomo_rope_axes(x, y, cos, sin, pos, axis, 2, d)
    for _ in range(3):
        x.mul_(-1)
        y.zero_()
        graph.replay()
        L.lomo_rope_axes(x, want, cos, sin, pos, axis, 2, d)
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_tables_without_rows_and_rows_beyond_32_bits(L):
    x = torch.randn(10, 128, device=DEV).half()
    none, y = torch.empty(0, 64, device=DEV), torch.zeros_like(x)
    L.lomo_rope_axes(x, y, none, none, torch.zeros(1, 10, dtype=torch.int32, device=DEV), bytes(64), 1, 128)
    assert torch.equal(x, y)
    heads, d = 48, 128
    T = (1 << 31) // (heads * d) + 100
    cos, sin = (dev(t) for t in tables(50, d))
    big = torch.zeros(T, heads * d, dtype=torch.float16, device=DEV)
    big[T - 10:] = torch.randn(10, heads * d, device=DEV).half()
    pos = torch.randint(0, 50, (2, T), dtype=torch.int32, device=DEV)
    axis = bytes([0] * 20 + [1] * 44)
    want = torch.empty(10, heads * d, dtype=torch.float16, device=DEV)
    L.lomo_rope_axes(big[T - 10:].contiguous(), want, cos, sin, pos[:, T - 10:].contiguous(), axis, heads, d)
    L.lomo_rope_axes(big, big, cos, sin, pos, axis, heads, d)
    assert torch.equal(big[T - 10:], want) and not bool(big[:T - 10:997].any())
