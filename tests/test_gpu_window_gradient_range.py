"""Gradients of attention with a window over the range of what comes in: dO far below and above 1, of one size or of many.  dq, dk and dv against
the definition in fp64, relative to their norms."""
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


def normal(seed, *shape):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape).astype(np.float32)).to(DEV)


def run(L, qkv, do, h, g, window, sinks):
    n, d = qkv.shape[0], do.shape[1] // h
    off = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    o, lse, dqkv = torch.empty_like(do), torch.empty(n, h, device=DEV), torch.empty_like(qkv)
    ws = torch.full((L.lomo_window_attention_workspace_bytes(n, 1, h, g, d, sinks),), 255, dtype=torch.uint8, device=DEV)
    L.lomo_window_attention_forward(qkv, o, lse, off, h, g, window, sinks)
    L.lomo_window_attention_backward(qkv, o, do, lse, dqkv, off, h, g, window, sinks, ws)
    return o, lse, dqkv


def sees(n, window, sinks):
    i = torch.arange(n, device=DEV)
    gap = i[:, None] - i[None, :]
    return (gap >= 0) & ((gap < window) | (i[None, :] < sinks))


def gradients(qkv, do, o, lse, h, g, window, sinks):
    """[n x (h + 2 g) x d] in fp64, with o and lse as the forward left them."""
    n, d = qkv.shape[0], do.shape[1] // h
    see = sees(n, window, sinks)
    x, u, w = qkv.view(n, h + 2 * g, d).double(), do.view(n, h, d).double(), o.view(n, h, d).double()
    grad = torch.zeros_like(x)
    for a in range(h):
        b = a // (h // g)
        q, k, v = x[:, a], x[:, h + b], x[:, h + g + b]
        p = ((q @ k.t().contiguous()) / d ** 0.5 - lse[:, a, None].double()).exp() * see
        ds = p * (u[:, a] @ v.t().contiguous() - (u[:, a] * w[:, a]).sum(1, keepdim=True)) / d ** 0.5
        grad[:, a] = ds @ k
        grad[:, h + b] += ds.t().contiguous() @ q
        grad[:, h + g + b] += p.t().contiguous() @ u[:, a]
    return grad


def check(got, want, what, rows=False):
    """Roundings of half a step of P or dS and of the result that are independent: 2^-11 / sqrt(3) each, relative to the norm of the sum's terms
    (random signs: that of the sum), together 2^-11 * 0.82; twice that.  Below 2^-14 the result itself is off by up to half a step of 2^-24."""
    dims = dict(dim=-1) if rows else {}
    off, size = (got - want).norm(**dims), want.norm(**dims)
    allowed = 2.0 ** -11 * 1.64 * size + 2.0 ** -25 * (want.shape[-1] if rows else want.numel()) ** 0.5
    print(what, "relative", float((off / size.clamp_min(1e-300)).max()), "share of what is allowed", float((off / allowed).max()))
    assert bool(torch.isfinite(got).all()) and bool((off <= allowed).all()), what


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sigma", [100.0, 1.0, 1e-2, 1e-3])
@pytest.mark.parametrize("n,window,sinks", [(6001, 4096, 4), (3000, 1000, 40)])
def test_size_of_the_incoming_gradient(L, n, window, sinks, sigma, d):
    h, g = 2, 1
    qkv, do = normal(n + d, n, (h + 2 * g) * d).half(), (sigma * normal(7, n, h * d)).half()
    o, lse, dqkv = run(L, qkv, do, h, g, window, sinks)
    want, got = gradients(qkv, do, o, lse, h, g, window, sinks), dqkv.view(n, h + 2 * g, d).double()
    for part, name in enumerate(("dq 0", "dq 1", "dk", "dv")):
        check(got[:, part], want[:, part], name)


@pytest.mark.parametrize("d", [64, 128])
def test_beyond_the_range_of_fp16(L, d):
    """dS of more than 65504, whose products with small q and k are within the range."""
    n, h, g, window, sinks = 700, 2, 1, 3, 0
    x = normal(1, n, h + 2 * g, d)
    x[:, :h + g] *= 0.01
    x[:, h + g:] *= 40
    qkv, do = x.half().view(n, -1), (6000 * normal(2, n, h * d)).half()
    o, lse, dqkv = run(L, qkv, do, h, g, window, sinks)
    want, got = gradients(qkv, do, o, lse, h, g, window, sinks), dqkv.view(n, h + 2 * g, d).double()
    assert bool(want.abs().max() < 65504)
    for part, name in enumerate(("dq 0", "dq 1", "dk", "dv")):
        check(got[:, part], want[:, part], name)


@pytest.mark.parametrize("d", [64, 128])
def test_every_query_at_its_own_size(L, d):
    """Queries whose dO differ by up to a factor of a million: each row of dq is as exact as it would be alone."""
    n, h, g, window, sinks = 2500, 2, 1, 1500, 4
    x = normal(3, n, h + 2 * g, d)
    x[:, h] *= 8                                                             # so that small rows of dq are not all below the normal range
    x[:, :h] /= 8
    size = 10 ** (6 * torch.rand(n, 1, device=DEV, generator=torch.Generator(DEV).manual_seed(1)) - 4)
    qkv, do = x.half().view(n, -1), (size * normal(4, n, h * d)).half()
    o, lse, dqkv = run(L, qkv, do, h, g, window, sinks)
    want, got = gradients(qkv, do, o, lse, h, g, window, sinks), dqkv.view(n, h + 2 * g, d).double()
    for part in range(h):
        check(got[1:, part], want[1:, part], "dq %d" % part, rows=True)      # the first query has a single key: dq is 0 but for o's rounding
    check(got[:, h], want[:, h], "dk")
    check(got[:, h + g], want[:, h + g], "dv")


@pytest.mark.parametrize("d", [64, 128])
def test_a_large_gradient_stays_with_its_query(L, d):
    """Keys that a query with a huge dO does not see, and the other queries, keep every bit of their gradients."""
    n, h, g, window, sinks, big = 900, 4, 2, 130, 3, 400
    qkv, do = normal(5, n, (h + 2 * g) * d).half(), (1e-3 * normal(6, n, h * d)).half()
    clean = run(L, qkv, do, h, g, window, sinks)[2]
    do[big] = 30000.0
    got = run(L, qkv, do, h, g, window, sinks)[2]
    assert torch.equal(torch.cat((got[:big], got[big + 1:]))[:, :h * d], torch.cat((clean[:big], clean[big + 1:]))[:, :h * d])
    hidden = ~sees(n, window, sinks)[big]
    assert torch.equal(got[hidden, h * d:], clean[hidden, h * d:]) and not torch.equal(got[~hidden, h * d:], clean[~hidden, h * d:])
