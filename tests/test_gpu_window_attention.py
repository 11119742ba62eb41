"""Attention with a sliding window and sinks on the GPU against oracle/student.py, element by element within the bounds that it derives."""
import os

import numpy as np
import pytest
import torch

from oracle import student as S

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MARK = 77.0      # what rows of no sequence hold, before and after


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


def offsets_of(lengths, start=0):
    return [start + int(n) for n in np.concatenate(([0], np.cumsum(lengths)))]


def run(L, qkv, do, offsets, h, g, window, sinks, stream=None, o=None, lse=None):
    """o, lse, dqkv of the forward and the backward, on buffers filled with MARK and a workspace filled with NaN."""
    T, d = qkv.shape[0], qkv.shape[1] // (h + 2 * g)
    off = torch.tensor(offsets, dtype=torch.int32, device=DEV)
    o = torch.full((T, h * d), MARK, dtype=torch.float16, device=DEV)
    lse = torch.full((T, h), MARK, device=DEV)
    dqkv = torch.full_like(qkv, MARK)
    ws = torch.full((L.lomo_window_attention_workspace_bytes(T, len(offsets) - 1, h, g, d, sinks),), 255, dtype=torch.uint8, device=DEV)
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())
    L.lomo_window_attention_forward(qkv, o, lse, off, h, g, window, sinks, stream)
    L.lomo_window_attention_backward(qkv, o, do, lse, dqkv, off, h, g, window, sinks, ws, stream)
    torch.cuda.synchronize()
    return o, lse, dqkv


def inputs(seed, T, h, g, d, sharp=1.0):
    rng = np.random.default_rng(seed)
    qkv = rng.standard_normal((T, (h + 2 * g) * d)).astype(np.float16)
    qkv[:, :h * d] *= np.float16(sharp)
    return qkv, (3 * rng.standard_normal((T, h * d))).astype(np.float16)


def within(got, want, bound, what):
    got, rows = got.float().cpu().numpy().astype(np.float64), ~np.isnan(want[:, 0])
    assert (got[~rows] == MARK).all(), what
    off = np.abs(got[rows] - want[rows])
    worst = np.max(off / bound[rows]) if off.size else 0.0
    print(what, "worst share of the bound", worst)
    assert np.isfinite(got[rows]).all() and worst <= 1.0, what


CASES = [
    # lengths, heads, key heads, width, window, sinks, sharpness, first row
    ([1], 1, 1, 128, 1, 0, 1.0, 0),
    ([1], 2, 1, 64, 5, 4, 1.0, 3),
    ([64], 2, 2, 128, 64, 0, 1.0, 0),
    ([65, 1, 0, 127, 128, 129, 0, 200], 4, 2, 64, 50, 4, 1.0, 5),
    ([65, 1, 0, 127, 128, 129, 0, 200], 4, 2, 128, 50, 4, 1.0, 5),
    ([300], 8, 2, 128, 1, 1, 1.0, 0),                 # a window of the token itself
    ([700], 4, 1, 128, 100, 64, 1.0, 0),              # as many sinks as there may be, half of them inside the window of many
    ([700], 4, 1, 64, 30, 64, 1.0, 0),                # more sinks than the window has keys
    ([513], 2, 2, 64, 512, 33, 2.0, 0),               # the last query alone has left one behind
    ([1300, 70], 4, 4, 128, 256, 5, 0.3, 0),          # pieces of the far queries
    ([1100], 2, 1, 128, 5000, 4, 1.0, 0),             # no limit
    ([1537], 7, 1, 128, 520, 40, 3.0, 0),             # seven heads of one key head
    ([3] * 70, 2, 1, 64, 2, 1, 1.0, 1),               # more sequences than a wave has lanes
]


@pytest.mark.parametrize("lengths,h,g,d,window,sinks,sharp,start", CASES)
def test_against_the_definition(L, lengths, h, g, d, window, sinks, sharp, start):
    off = offsets_of(lengths, start)
    qkv, do = inputs(sum(lengths) + window, off[-1] + 6, h, g, d, sharp)
    o, lse, dqkv = run(L, dev(qkv), dev(do), off, h, g, window, sinks)
    want, want_lse, bound, bound_lse = S.window_attention_forward(qkv, off, h, g, window, sinks)
    within(lse, want_lse, bound_lse, "lse")
    within(o, want, bound, "o")
    grad, bound = S.window_attention_backward(qkv, o.cpu().numpy(), do, lse.cpu().numpy(), off, h, g, window, sinks)
    n = d * h
    for name, sl in (("dq", slice(0, n)), ("dk", slice(n, n + g * d)), ("dv", slice(n + g * d, None))):
        within(dqkv[:, sl], grad[:, sl], bound[:, sl], name)


@pytest.mark.parametrize("window,sinks", [(4096, 0), (1000, 4)])
def test_long_sequence(L, window, sinks):
    """9001 tokens against the definition in fp64 on the GPU; a random entry in a thousand of the gradient against the same."""
    n, h, g, d = 9001, 2, 1, 128
    qkv, do = (dev(x) for x in inputs(n, n, h, g, d))
    o, lse, dqkv = run(L, qkv, do, [0, n], h, g, window, sinks)
    i = torch.arange(n, device=DEV)
    gap = i[:, None] - i[None, :]
    hidden = (gap < 0) | ((gap >= window) & (i[None, :] >= sinks))
    x = qkv.view(n, h + 2 * g, d).double()
    grad = torch.zeros_like(x)
    for a in range(h):
        q, k, v = x[:, a], x[:, h], x[:, h + 1]
        s = ((q @ k.t().contiguous()) / d ** 0.5).masked_fill(hidden, -float("inf"))
        p = torch.softmax(s, 1)
        u = do.view(n, h, d)[:, a].double()
        assert (torch.logsumexp(s, 1) - lse[:, a]).abs().max() <= 1e-5
        want = p @ v
        # every probability and the result to half a step of fp16, the rest of the bound a tenth of that
        assert ((o.view(n, h, d)[:, a].double() - want).abs() <= 2.0 ** -11 * want.abs() + 1.1 * 2.0 ** -11 * (p @ v.abs()) + 2e-5).all()
        p = (s - lse[:, a, None].double()).exp()
        ds = p * (u @ v.t().contiguous() - (u * o.view(n, h, d)[:, a].double()).sum(1, keepdim=True)) / d ** 0.5
        grad[:, a] = ds @ k
        grad[:, h] += ds.t().contiguous() @ q
        grad[:, h + 1] += p.t().contiguous() @ u
    got = dqkv.view(n, h + 2 * g, d).double()
    for part in range(h + 2 * g):
        # roundings of half a step of P or dS and of the result that are independent: 2^-11 / sqrt(3) each, relative to the norm of the sum's terms
        # (random signs: that of the sum), together 2^-11 * 0.82; twice that
        off = (got[:, part] - grad[:, part]).norm() / grad[:, part].norm()
        assert off <= 2.0 ** -11 * 1.64, (part, float(off))


def test_rows_do_not_depend_on_the_batch(L):
    h, g, d, window, sinks = 4, 2, 128, 200, 4
    lengths = [130, 700, 1, 0, 333]
    off = offsets_of(lengths, 7)
    qkv, do = (dev(x) for x in inputs(2, off[-1] + 5, h, g, d))
    whole = run(L, qkv, do, off, h, g, window, sinks)
    for a, b in zip(off, off[1:]):
        if a == b:
            continue
        alone = run(L, qkv[a:b].contiguous(), do[a:b].contiguous(), [0, b - a], h, g, window, sinks)
        for x, y in zip(whole, alone):
            assert torch.equal(x[a:b], y)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_hidden_values_stay_hidden(L, d, value):
    """A row of inf or NaN, in a sequence, before it, behind it, in another: whoever does not see it keeps every bit."""
    h, g, window, sinks, n, bad = 4, 2, 70, 3, 400, 200
    off = offsets_of([50, n, 60], 4)
    qkv, do = inputs(9, off[-1] + 3, h, g, d)
    clean = run(L, dev(qkv), dev(do), off, h, g, window, sinks)
    s0 = off[1]
    outside = [0, off[-1] + 1]
    for part in ("k and v", "v", "k", "q", "do"):
        x, y = qkv.copy(), do.copy()
        rows = outside + [off[0] + 7, s0 + bad]
        cols = {"k and v": slice(h * d, None), "v": slice((h + g) * d, None), "k": slice(h * d, (h + g) * d), "q": slice(0, h * d), "do": None}[part]
        for r in rows:
            if cols is None:
                y[r] = value
            else:
                x[r, cols] = value
        got = run(L, dev(x), dev(y), off, h, g, window, sinks)
        see = S.visible(n, window, sinks)
        hit = np.zeros(n, bool)      # queries that meet the value
        if part in ("q", "do"):
            hit[bad] = True
        else:
            hit = see[:, bad].copy()
        keys = see[hit].any(0)       # keys whose gradients they reach
        keep_q = torch.from_numpy(np.flatnonzero(~hit) + s0).to(DEV)
        keep_k = torch.from_numpy(np.flatnonzero(~keys) + s0).to(DEV)
        if part != "do":
            assert torch.equal(got[0][keep_q], clean[0][keep_q]) and torch.equal(got[1][keep_q], clean[1][keep_q]), part
        assert torch.equal(got[2][keep_q, :h * d], clean[2][keep_q, :h * d]), part
        assert torch.equal(got[2][keep_k, h * d:], clean[2][keep_k, h * d:]), part
        last = slice(off[2], off[3])      # a sequence without any, and rows of none
        for a, b in zip(got, clean):
            assert torch.equal(a[last], b[last]) and bool((a[off[-1]:] == MARK).all()) and bool((a[:4] == MARK).all()), part
        met = torch.from_numpy(np.flatnonzero(hit) + s0).to(DEV)
        reached = got[2][met, :h * d].isfinite().all(1) if part != "v" else got[0][met].isfinite().all(1)
        assert not bool(reached.any()), part      # and whoever sees it shows it


def test_one_infinite_value_reaches_its_column_alone(L):
    h, g, d, n, window = 2, 1, 128, 100, 40
    qkv, do = inputs(4, n, h, g, d)
    qkv[50, (h + g) * d + 9] = np.inf
    o, lse, _ = run(L, dev(qkv), dev(do), [0, n], h, g, window, 0)
    got = o.view(n, h, d).isfinite().cpu().numpy()
    want = np.ones((n, h, d), bool)
    want[50:90, :, 9] = False
    np.testing.assert_array_equal(got, want)
    assert bool((o.view(n, h, d)[50:90, :, 9] == float("inf")).all()) and bool(lse.isfinite().all())


@pytest.mark.parametrize("n,window,sinks,key", [(300, 90, 2, 0), (300, 90, 2, 131), (700, 5000, 0, 70), (60, 60, 0, 5)])
@pytest.mark.parametrize("d", [64, 128])
def test_gradient_of_queries_that_score_minus_infinity(L, d, n, window, sinks, key):
    """A key with one infinite element: queries whose score is -inf have a finite lse, P = 0 there, and 0 * inf = NaN in that column of dq alone;
    the others meet +inf and have nothing finite."""
    h, g, col = 2, 1, 9
    qkv, do = inputs(n + key, n, h, g, d)
    qkv[:, col] = -np.abs(qkv[:, col]) - np.float16(0.1)      # head 0 scores -inf
    qkv[:, d + col] = np.abs(qkv[:, d + col]) + np.float16(0.1)
    finite = qkv.copy()
    qkv[key, h * d + col] = np.inf
    o, lse, dqkv = run(L, dev(qkv), dev(do), [0, n], h, g, window, sinks)
    see = S.visible(n, window, sinks)
    hit = see[:, key]
    dq = dqkv.view(n, h + 2 * g, d)[:, :h].float().cpu().numpy()
    want = np.ones((n, d), bool)
    want[hit, col] = False
    got = np.isfinite(dq[:, 0])
    rows = np.arange(n) != (0 if key == 0 else -1)      # a query that sees nothing else has no lse, and nothing finite
    np.testing.assert_array_equal(got[rows], want[rows])
    assert not np.isfinite(dq[hit, 1]).any() and np.isfinite(dq[~hit, 1]).all()
    # the finite entries of head 0, with the key's share taken out
    q, v, u = (x.astype(np.float64) for x in (finite[:, :d], finite[:, (h + g) * d:], do[:, :d]))
    k = finite[:, h * d:(h + 1) * d].astype(np.float64)
    w, e = o[:, :d].cpu().numpy().astype(np.float64), lse[:, 0].cpu().numpy().astype(np.float64)
    left = see.copy()
    left[:, key] = False
    with np.errstate(all="ignore"):
        p = np.where(left, np.exp(q @ k.T / d ** 0.5 - e[:, None]), 0.0)
        grad = (p * (u @ v.T - (u * w).sum(1, keepdims=True)) / d ** 0.5) @ k
        _, bound = S.window_attention_backward(finite, o.cpu().numpy(), do, lse.cpu().numpy(), [0, n], h, g, window, sinks)
    ok = want & rows[:, None]
    assert (np.abs(dq[:, 0] - grad)[ok] <= bound[:, :d][ok]).all()


def test_offsets_that_do_not_ascend_stay_in_bounds(L):
    """No results are promised; rows before and behind the buffers' own are not touched."""
    h, g, d, T = 2, 1, 64, 300
    for off in ([0, 400, 300], [-50, 100, 300], [0, 200, 100, 300], [250, 250, -7], [2 ** 31 - 1, 0]):
        big = [torch.full((T + 128, w), MARK, dtype=t, device=DEV) for w, t in ((4 * d, torch.float16), (2 * d, torch.float16), (2, torch.float32),
                                                                               (4 * d, torch.float16))]
        qkv, o, lse, dqkv = (x[64:64 + T] for x in big)
        qkv.copy_(dev(inputs(1, T, h, g, d)[0]))
        o_off = torch.tensor(off, dtype=torch.int32, device=DEV)
        size = L.lomo_window_attention_workspace_bytes(T, len(off) - 1, h, g, d, 4)
        ws = torch.full((size + 512,), 255, dtype=torch.uint8, device=DEV)
        L.lomo_window_attention_forward(qkv, o, lse, o_off, h, g, 40, 4)
        L.lomo_window_attention_backward(qkv, o, o.clone(), lse, dqkv, o_off, h, g, 40, 4, ws[256:256 + size])
        torch.cuda.synchronize()
        for x in big[1:]:
            assert bool((x[:64] == MARK).all()) and bool((x[64 + T:] == MARK).all()), off
        assert bool((ws[:256] == 255).all()) and bool((ws[256 + size:] == 255).all()), off


def test_empty_calls_and_bad_tensors(L):
    half = dict(dtype=torch.float16, device=DEV)
    off = torch.zeros(2, dtype=torch.int32, device=DEV)
    L.lomo_window_attention_forward(torch.empty(0, 384, **half), torch.empty(0, 128, **half), torch.empty(0, 1, device=DEV), off, 1, 1, 4)
    qkv, o, lse = torch.zeros(8, 384, **half), torch.full((8, 128), MARK, **half), torch.zeros(8, 1, device=DEV)
    L.lomo_window_attention_forward(qkv, o, lse, off, 1, 1, 4)      # one sequence without rows
    torch.cuda.synchronize()
    assert bool((o == MARK).all())
    for bad in (lambda: L.lomo_window_attention_forward(qkv.float(), o, lse, off, 1, 1, 4),
                lambda: L.lomo_window_attention_forward(qkv, o, lse, off.long(), 1, 1, 4),
                lambda: L.lomo_window_attention_forward(torch.zeros(8, 768, **half)[:, ::2], o, lse, off, 1, 1, 4),
                lambda: L.lomo_window_attention_forward(qkv, o, lse, off.cpu(), 1, 1, 4),
                lambda: L.lomo_window_attention_forward(qkv, o, lse, off, 1, 1, 0),
                lambda: L.lomo_window_attention_backward(qkv, o, o, lse, qkv.clone(), off, 1, 1, 4, 4, torch.empty(16, dtype=torch.uint8, device=DEV)),
                lambda: L.lomo_window_attention_backward(qkv, o, o[:4], lse, qkv.clone(), off, 1, 1, 4, 4, lse)):
        with pytest.raises(L.LomoError):
            bad()


def test_other_stream_and_graph(L):
    h, g, d, window, sinks = 4, 1, 128, 90, 4
    off = offsets_of([300, 41, 650])
    qkv, do = (dev(x) for x in inputs(6, off[-1], h, g, d))
    want = run(L, qkv, do, off, h, g, window, sinks)
    for x, y in zip(run(L, qkv, do, off, h, g, window, sinks, stream=torch.cuda.Stream()), want):
        assert torch.equal(x, y)
    offsets = torch.tensor(off, dtype=torch.int32, device=DEV)
    o, lse, dqkv = (torch.zeros_like(x) for x in want)
    ws = torch.zeros(L.lomo_window_attention_workspace_bytes(off[-1], 3, h, g, d, sinks), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.lomo_window_attention_forward(qkv, o, lse, offsets, h, g, window, sinks)
        L.lomo_window_attention_backward(qkv, o, do, lse, dqkv, offsets, h, g, window, sinks, ws)
    first = qkv.clone()
    other = dev(inputs(7, off[-1], h, g, d)[0])
    for k in range(4):
        qkv.copy_(other if k % 2 else first)
        ws.fill_(255)
        for x in (o, lse, dqkv):
            x.zero_()
        graph.replay()
        eager = run(L, qkv, do, off, h, g, window, sinks)
        for x, y in zip((o, lse, dqkv), eager):
            assert torch.equal(x, y), k


def test_rows_beyond_32_bits(L):
    """The last sequence of buffers of more than 2^31 elements, 4 GiB: as at the beginning of small ones."""
    h, g, d, window, sinks, n = 32, 8, 128, 100, 4, 300
    T = (1 << 31) // ((h + 2 * g) * d) + n + 1000
    small = [dev(x) for x in inputs(3, n, h, g, d)]
    want = run(L, *small, [0, n], h, g, window, sinks)
    qkv, do = torch.zeros(T, (h + 2 * g) * d, dtype=torch.float16, device=DEV), torch.zeros(T, h * d, dtype=torch.float16, device=DEV)
    qkv[T - n:], do[T - n:] = small
    got = run(L, qkv, do, [T - n, T], h, g, window, sinks)
    for x, y in zip(got, want):
        assert torch.equal(x[T - n:], y) and bool((x[:T - n:997] == MARK).all())


def test_two_calls_at_once(L):
    h, g, d, window, sinks, n = 8, 2, 128, 300, 4, 2000
    data = [[dev(x) for x in inputs(seed, n, h, g, d)] for seed in (1, 2)]
    want = [run(L, *x, [0, n], h, g, window, sinks) for x in data]
    off = torch.tensor([0, n], dtype=torch.int32, device=DEV)
    size = L.lomo_window_attention_workspace_bytes(n, 1, h, g, d, sinks)
    streams, got = [torch.cuda.Stream() for _ in data], []
    for (qkv, do), w in zip(data, want):
        got.append([torch.zeros_like(x) for x in w] + [torch.empty(size, dtype=torch.uint8, device=DEV)])
    torch.cuda.synchronize()
    for _ in range(4):
        for (qkv, do), (o, lse, dqkv, ws), st in zip(data, got, streams):
            L.lomo_window_attention_forward(qkv, o, lse, off, h, g, window, sinks, st)
            L.lomo_window_attention_backward(qkv, o, do, lse, dqkv, off, h, g, window, sinks, ws, st)
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        for x, y in zip(a, b):
            assert torch.equal(x, y)
