"""Steps on packed sequences, recorded once as a HIP graph and replayed on other batches: other lengths, other numbers of tokens."""
import os

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


H16 = dict(dtype=torch.float16)
V, F, EPS = 264, 384, 1e-5


def model(h, g, d, n_layers=2, seed=3):
    gen = torch.Generator().manual_seed(seed)
    H = h * d
    f = lambda *s, sigma: (sigma * torch.randn(*s, generator=gen)).half().to(DEV)
    gain = lambda: (1 + 0.1 * torch.randn(H, generator=gen)).half().to(DEV)
    layers = [{"w1": gain(), "W_qkv": f((h + 2 * g) * d, H, sigma=1.5 * H ** -0.5), "W_o": f(H, H, sigma=H ** -0.5), "w2": gain(),
               "W_gu": f(2 * F, H, sigma=H ** -0.5), "W_d": f(H, F, sigma=F ** -0.5)} for _ in range(n_layers)]
    return {"W_emb": f(V, H, sigma=1.0), "layers": layers, "w_f": gain(), "W_lm": f(V, H, sigma=1.5 * H ** -0.5)}


def tensors(m):
    return [m["W_emb"], m["w_f"], m["W_lm"]] + [p[k] for p in m["layers"] for k in sorted(p)]


def copied(m):
    return {"W_emb": m["W_emb"].clone(), "w_f": m["w_f"].clone(), "W_lm": m["W_lm"].clone(),
            "layers": [{k: v.clone() for k, v in p.items()} for p in m["layers"]]}


def tables(d, n=300):
    angle = torch.arange(n)[:, None] * 1e4 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))[None, :]
    return angle.cos().float().to(DEV), angle.sin().float().to(DEV)


class Problem:
    """Tokens, targets and a teacher in fixed buffers, as a captured step needs them."""

    def __init__(self, T, K=5):
        self.T, self.K = T, K
        self.ids, self.targets = (torch.zeros(T, dtype=torch.int32, device=DEV) for _ in range(2))
        self.top, self.logits = torch.zeros(T, K, dtype=torch.int32, device=DEV), torch.zeros(T, K, device=DEV, **H16)

    def set(self, seed, lengths):
        gen = torch.Generator().manual_seed(seed)
        self.ids.copy_(torch.randint(0, V, (self.T,), generator=gen, dtype=torch.int32))
        targets = torch.randint(0, V, (self.T,), generator=gen, dtype=torch.int32)
        targets[sum(lengths):] = -100
        self.targets.copy_(targets)
        self.top.copy_(torch.randint(0, V, (self.T, self.K), generator=gen, dtype=torch.int32))
        self.logits.copy_(torch.randn(self.T, self.K, generator=gen).half())


BATCHES = [[40, 0, 1, 70], [120, 30], [9], [150], [], [64, 64], [33, 44, 55]]


def near(a, b):
    """The step size may differ in its last bit, since the norm's sum is atomic: nearly all weights have the same bits, and none is far off."""
    same = (a.view(torch.int16) == b.view(torch.int16)).float().mean().item()
    return same > 0.999 and bool((a.float() - b.float()).abs().max() <= 2.0 ** -9 * a.float().abs().max())


@pytest.mark.parametrize("norm,checkpoint,keep,distil", [("global", True, False, False), ("global", True, False, True),
                                                         ("grouped", True, False, True), ("global", False, True, True)])
@pytest.mark.parametrize("h,g,d", [(4, 2, 64), (2, 1, 128)])
def test_replays_take_other_batches(L, h, g, d, norm, checkpoint, keep, distil):
    from paper_2306_09782_amd.chain import LomoFineTuneStep, PackedAttention, Teacher
    T, lr, scale = 150, 2.0, 512.0
    cos, sin = tables(d)
    data, start = Problem(T), model(h, g, d)

    def make():
        packed = PackedAttention(DEV, T, h, g, d, 20, 3, max_sequences=5)
        step = LomoFineTuneStep(DEV, 1, T, h * d, F, h, 2, V, norm=norm, checkpoint=checkpoint, keep_handons=keep, packed=packed)
        teacher = Teacher(data.top, data.logits) if distil else None
        return packed, step, lambda m: step.step(data.ids, data.targets, m, cos, sin, lr, scale, max_norm=1e9, teacher=teacher)

    packed, step, run = make()
    m = copied(start)
    side = torch.cuda.Stream()
    data.set(0, BATCHES[0])
    packed.set_batch(BATCHES[0])
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run(m)                                   # outside of the recording: kernels' attributes, workspaces
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(m)
    eager_packed, eager_step, eager_run = make()
    for k, lengths in enumerate(BATCHES):
        data.set(k + 1, lengths)
        for w, w0 in zip(tensors(m), tensors(start)):
            w.copy_(w0)
        packed.set_batch(lengths)
        graph.replay()
        torch.cuda.synchronize()
        got = step.result()
        other = copied(start)
        eager_packed.set_batch(lengths)
        eager_run(other)
        torch.cuda.synchronize()
        want = eager_step.result()
        assert got["loss"] == want["loss"] and got["overflow"] == want["overflow"], (k, lengths)
        for i, (a, b) in enumerate(zip(tensors(m), tensors(other))):
            assert near(a, b), (k, lengths, i)
        for a, b in zip(step.chain.attn, eager_step.chain.attn):      # gradients: every bit
            assert torch.equal(a.dqkv, b.dqkv) and torch.equal(a.dxn, b.dxn), (k, lengths)


@pytest.mark.parametrize("distil", [False, True])
def test_norm_pass_on_a_second_stream(L, distil):
    """`packed` with overlap_norm_pass: the weights of the step on one stream."""
    from paper_2306_09782_amd.chain import LomoFineTuneStep, PackedAttention, Teacher
    h, g, d, T = 4, 2, 64, 150
    cos, sin = tables(d)
    data, start = Problem(T), model(h, g, d)
    out = []
    for overlap in (False, True):
        packed = PackedAttention(DEV, T, h, g, d, 20, 3, max_sequences=5)
        step = LomoFineTuneStep(DEV, 1, T, h * d, F, h, 2, V, checkpoint=False, keep_handons=True, overlap_norm_pass=overlap, packed=packed)
        m, got = copied(start), []
        for k, lengths in enumerate(BATCHES[:4]):
            data.set(k, lengths)
            packed.set_batch(lengths)
            step.step(data.ids, data.targets, m, cos, sin, 2.0, 512.0, max_norm=1e9, teacher=Teacher(data.top, data.logits) if distil else None)
            torch.cuda.synchronize()
            res = step.result()
            assert not res["overflow"]
            got.append(res["loss"])
        out.append((got, m))
    assert out[0][0] == pytest.approx(out[1][0], rel=1e-3)
    for a, b in zip(tensors(out[0][1]), tensors(out[1][1])):
        assert near(a, b)


@pytest.mark.parametrize("off", [[0, 50], [0, 0], [3, 20, 20, 41], [7], [50, 50], [0, 49], [-4, 60], [30, 10], [60, 70], [20, 2 ** 31 - 1], [-9, -3]])
@pytest.mark.parametrize("width", [8, 264, 1536])
def test_clear_padding(L, off, width):
    """Rows of no sequence become zeros, the others and what is around the buffer stay; offsets out of order stay in bounds."""
    T = 50
    big = torch.full((T + 20, width), 7.0, device=DEV, **H16)
    L.lomo_clear_padding(big[10:10 + T], torch.tensor(off, dtype=torch.int32, device=DEV))
    first = min(max(off[0], 0), T)
    end = min(max(off[-1], first), T)
    want = torch.full_like(big, 7.0)
    want[10:10 + first] = 0
    want[10 + end:10 + T] = 0
    assert torch.equal(big, want)


def test_clear_padding_beyond_32_bits(L):
    T, width = (1 << 20) + 10, 4096
    x = torch.ones(T, width, device=DEV, **H16)
    L.lomo_clear_padding(x, torch.tensor([2, T - 3], dtype=torch.int32, device=DEV))
    assert not bool(x[:2].any()) and not bool(x[T - 3:].any()) and bool((x[2:T - 3:1009] == 1).all()) and bool((x[T - 4] == 1).all())


def test_clear_padding_refusals(L):
    x, off = torch.ones(6, 16, device=DEV, **H16), torch.tensor([0, 3], dtype=torch.int32, device=DEV)
    L.lomo_clear_padding(x[:0], off)
    for bad in (lambda: L.lomo_clear_padding(x.float(), off), lambda: L.lomo_clear_padding(x, off.long()), lambda: L.lomo_clear_padding(x, off.cpu()),
                lambda: L.lomo_clear_padding(x.cpu(), off), lambda: L.lomo_clear_padding(x[:, ::2], off), lambda: L.lomo_clear_padding(x, off[:0]),
                lambda: L.lomo_clear_padding(torch.ones(4, 12, device=DEV, **H16), off), lambda: L.lomo_clear_padding(x.view(-1), off)):
        with pytest.raises(L.LomoError):
            bad()
    assert bool((x == 1).all())
