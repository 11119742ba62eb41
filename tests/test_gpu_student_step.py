"""Whole fine-tuning steps of a student: packed sequences, shared key heads, a window with sinks, rotary positions on three axes, a teacher,
through LomoFineTuneStep and LomoTrainer, against automatic differentiation of the same model in fp64."""
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


def make_model(gen, V, H, F, width, n_layers):
    f = lambda *s, sigma: (sigma * torch.randn(*s, generator=gen)).half()
    gain = lambda: (1 + 0.1 * torch.randn(H, generator=gen)).half()
    layers = [{"w1": gain(), "W_qkv": f(width, H, sigma=1.5 * H ** -0.5), "W_o": f(H, H, sigma=H ** -0.5), "w2": gain(),
               "W_gu": f(2 * F, H, sigma=H ** -0.5), "W_d": f(H, F, sigma=F ** -0.5)} for _ in range(n_layers)]
    return {"W_emb": f(V, H, sigma=1.0), "layers": layers, "w_f": gain(), "W_lm": f(V, H, sigma=1.5 * H ** -0.5)}


def tensors(m):
    return [m["W_emb"], m["w_f"], m["W_lm"]] + [p[k] for p in m["layers"] for k in sorted(p)]


def mapped(m, f):
    return {"W_emb": f(m["W_emb"]), "w_f": f(m["w_f"]), "W_lm": f(m["W_lm"]), "layers": [{k: f(v) for k, v in p.items()} for p in m["layers"]]}


def reference(m, ids, targets, lengths, positions, pair_axis, cos, sin, h, g, d, window, sinks, eps, teacher):
    """Mean loss and the gradients of all tensors, fp64."""
    m = mapped(m, lambda t: t.double().requires_grad_())
    n = sum(lengths)
    norm = lambda x, w: x / (x.square().mean(1, keepdim=True) + eps).sqrt() * w
    pair = torch.arange(d // 2)
    where = positions.long()[torch.tensor(list(pair_axis))][:, :n].t()
    c, s = (t.double()[where, pair][:, None] for t in (cos, sin))

    def turn(x):
        a, b = x.view(n, -1, d).chunk(2, 2)
        return torch.cat((a * c - b * s, b * c + a * s), 2)

    x = m["W_emb"][ids[:n].long()]
    for p in m["layers"]:
        q, k, v = (norm(x, p["w1"]) @ p["W_qkv"].t()).split([h * d, g * d, g * d], 1)
        q, k, v = turn(q), turn(k), v.view(n, g, d)
        out, at = [], 0
        for length in lengths:
            i = torch.arange(length)
            gap = i[:, None] - i[None, :]
            hidden = (gap < 0) | ((gap >= window) & (i[None, :] >= sinks))
            rows, o = slice(at, at + length), []
            for a in range(h):
                b = a // (h // g)
                o.append(torch.softmax((q[rows, a] @ k[rows, b].t() / d ** 0.5).masked_fill(hidden, -float("inf")), 1) @ v[rows, b])
            out.append(torch.cat(o, 1))
            at += length
        x = x + torch.cat(out) @ p["W_o"].t()
        gate, up = (norm(x, p["w2"]) @ p["W_gu"].t()).chunk(2, 1)
        x = x + (torch.nn.functional.silu(gate) * up) @ p["W_d"].t()
    z = norm(x, m["w_f"]) @ m["W_lm"].t()
    count = (targets[:n] >= 0) & (targets[:n] < z.shape[1])
    z, t = z[count], targets[:n][count].long()
    loss = -torch.log_softmax(z, 1)[torch.arange(len(t)), t]
    if teacher is not None:
        tau, w = teacher[2:]
        log_p = torch.log_softmax(teacher[1][:n][count].double() / tau, 1)
        log_q = torch.log_softmax(z / tau, 1).gather(1, teacher[0][:n][count].long())
        loss = (1 - w) * loss + w * tau ** 2 * (log_p.exp() * (log_p - log_q)).sum(1)
    loss.mean().backward()
    return float(loss.detach().mean()), [t.grad for t in tensors(m)]


def problem(seed, H, F, V, h, g, d, lengths, padding, axes, K):
    gen = torch.Generator().manual_seed(seed)
    T = sum(lengths) + padding
    m = make_model(gen, V, H, F, (h + 2 * g) * d, 2)
    ids = torch.randint(0, V, (T,), generator=gen, dtype=torch.int32)
    targets = torch.roll(ids, -1)
    targets[sum(lengths):] = -100
    at = 0
    for n in lengths:
        at += n
        if n:
            targets[at - 1] = -100
    angle = torch.arange(300)[:, None] * 1e4 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))[None, :]
    positions = torch.randint(0, 300, (axes, T), generator=gen, dtype=torch.int32)
    teacher = (torch.randint(0, V, (T, K), generator=gen, dtype=torch.int32), (2 * torch.randn(T, K, generator=gen)).half(), 2.0, 0.7)
    return m, ids, targets, angle.cos().float(), angle.sin().float(), positions, teacher


@pytest.mark.parametrize("norm,checkpoint,keep,d,h,g", [("global", True, False, 64, 4, 2), ("grouped", True, False, 128, 2, 1),
                                                        ("global", False, True, 128, 2, 2)])
@pytest.mark.parametrize("distil", [False, True])
def test_step_against_differentiation(L, norm, checkpoint, keep, d, h, g, distil):
    from paper_2306_09782_amd.chain import LomoFineTuneStep, LomoTrainer, PackedAttention, Teacher
    H, F, V, window, sinks, lengths, padding = h * d, 384, 264, 20, 3, [40, 0, 1, 70], 17
    pair_axis = [c % 3 for c in range(d // 2)]
    m, ids, targets, cos, sin, positions, teacher = problem(d + h + g, H, F, V, h, g, d, lengths, padding, 3, 6)
    want_loss, grads = reference(m, ids, targets, lengths, positions, pair_axis, cos, sin, h, g, d, window, sinks, 1e-5,
                                 teacher if distil else None)
    T = sum(lengths) + padding
    packed = PackedAttention(DEV, T, h, g, d, window, sinks, max_sequences=9, pair_axis=pair_axis)
    packed.set_batch(lengths, positions.to(DEV))
    step = LomoFineTuneStep(DEV, 1, T, H, F, h, 2, V, norm=norm, checkpoint=checkpoint, keep_handons=keep, packed=packed)
    dm = mapped(m, lambda t: t.to(DEV).clone())
    lr = 3.0
    trainer = LomoTrainer(step, lr=lr, loss_scale=1024.0, max_norm=1e9)      # the grouped norm's coefficients would differ
    res = trainer.train_step(ids.to(DEV), targets.to(DEV), dm, cos.to(DEV), sin.to(DEV),
                             teacher=Teacher(teacher[0].to(DEV), teacher[1].to(DEV), *teacher[2:]) if distil else None)
    assert not res["overflow"] and abs(res["loss"] - want_loss) <= 2e-3 * want_loss
    for before, after, grad in zip(tensors(m), tensors(dm), grads):
        after = after.cpu().double()
        moved, want = after - before.double(), -lr * grad
        # some 48 roundings to fp16 on the way to a gradient, 2^-11 / sqrt(3) each and independent: 0.2 per cent; five times that; and the rounding
        # of the weights themselves
        allowed = 0.01 * want.norm() + 1.5 * 2.0 ** -11 / 3 ** 0.5 * after.norm()
        print(tuple(before.shape), "share of what is allowed", float((moved - want).norm() / allowed))
        assert (moved - want).norm() <= allowed, tuple(before.shape)
    # the padding's tokens do not matter, nor what its rows held
    again = mapped(m, lambda t: t.to(DEV).clone())
    other = ids.clone()
    other[sum(lengths):] = (other[sum(lengths):] + 5) % V
    LomoTrainer(step, lr=lr, loss_scale=1024.0, max_norm=1e9).train_step(
        other.to(DEV), targets.to(DEV), again, cos.to(DEV), sin.to(DEV),
        teacher=Teacher(teacher[0].to(DEV), teacher[1].to(DEV), *teacher[2:]) if distil else None)
    for a, b in zip(tensors(dm), tensors(again)):
        assert torch.equal(a, b)


def test_a_shorter_batch_after_a_longer_one(L):
    """The same step object: rows that were tokens of the last batch are padding of this one."""
    from paper_2306_09782_amd.chain import LomoFineTuneStep, PackedAttention
    h, g, d, F, V, T = 2, 1, 64, 384, 264, 150
    m, ids, targets, cos, sin, positions, _ = problem(5, h * d, F, V, h, g, d, [60, 90], 0, 1, 1)
    cos, sin, ids = cos.to(DEV), sin.to(DEV), ids.to(DEV)

    def run(batches):
        packed = PackedAttention(DEV, T, h, g, d, 30, 2, max_sequences=2)
        step = LomoFineTuneStep(DEV, 1, T, h * d, F, h, 2, V, packed=packed)
        for lengths in batches:
            dm = mapped(m, lambda t: t.to(DEV).clone())
            packed.set_batch(lengths)
            t = targets.clone()
            t[sum(lengths):] = -100
            step.step(ids, t.to(DEV), dm, cos, sin, 1.0, 512.0, max_norm=1e9)
            torch.cuda.synchronize()
            assert not step.result()["overflow"]
        return dm

    for a, b in zip(tensors(run([[60, 90], [40]])), tensors(run([[40]]))):
        assert torch.equal(a, b)


def test_without_a_limit_it_is_the_plain_step(L):
    """Equal sequences, no window, one axis: the losses and updates of the step's own attention, up to roundings."""
    from paper_2306_09782_amd.chain import LomoFineTuneStep, PackedAttention
    h, d, F, V, batch, seq = 2, 128, 384, 264, 2, 128
    m, ids, targets, cos, sin, _, _ = problem(6, h * d, F, V, h, h, d, [seq] * batch, 0, 1, 1)
    out = []
    for packed in (None, PackedAttention(DEV, batch * seq, h, h, d)):
        if packed is not None:
            packed.set_batch([seq] * batch)
        step = LomoFineTuneStep(DEV, batch, seq, h * d, F, h, 2, V, packed=packed)
        dm = mapped(m, lambda t: t.to(DEV).clone())
        step.step(ids.to(DEV), targets.to(DEV), dm, cos[:seq].to(DEV).contiguous(), sin[:seq].to(DEV).contiguous(), 3.0, 1024.0, max_norm=1e9)
        torch.cuda.synchronize()
        out.append((step.result()["loss"], [(a.cpu().double() - b.double()) for a, b in zip(tensors(dm), tensors(m))]))
    assert abs(out[0][0] - out[1][0]) <= 2e-3 * out[0][0]
    for before, a, b in zip(tensors(m), out[0][1], out[1][1]):
        # as above, each of the two
        assert (a - b).norm() <= 2 * (0.01 * a.norm() + 1.5 * 2.0 ** -11 / 3 ** 0.5 * before.double().norm())


def test_refusals(L):
    from paper_2306_09782_amd.chain import LomoFineTuneStep, PackedAttention
    for bad in ((100, 4, 3, 64), (100, 4, 2, 96)):
        with pytest.raises(L.LomoError):
            PackedAttention(DEV, *bad)
    with pytest.raises(L.LomoError):
        PackedAttention(DEV, 100, 4, 2, 64, 10, 65)
    packed = PackedAttention(DEV, 100, 4, 2, 64, 10, 2, max_sequences=3, pair_axis=[0, 1] * 16)
    for lengths in ([50, 51], [1, 1, 1, 1], [-1, 5]):
        with pytest.raises(L.LomoError):
            packed.set_batch(lengths)
    with pytest.raises(L.LomoError):
        packed.set_batch([10], torch.zeros(3, 100, dtype=torch.int32, device=DEV))
    packed.set_batch([])
    packed.set_batch([10, 20])
    assert packed.offsets.tolist() == [0, 10, 30, 30] and packed.positions[:, :30].tolist() == [list(range(10)) + list(range(20))] * 2
    for batch, seq, H, n_heads in ((1, 99, 256, 4), (1, 100, 512, 4), (1, 100, 256, 2)):
        with pytest.raises(L.LomoError):
            LomoFineTuneStep(DEV, batch, seq, H, 384, n_heads, 1, 264, packed=packed)
