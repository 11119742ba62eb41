"""Measured cases of the operators for fine-tuning a student model on long packed sequences: rotary positions with several axes,
attention with a sliding window and sinks and its gradient, distillation from a teacher's top logits.

  "rope"      the rotary step on the q and k heads of a fused projection, every pair of channels turned by the position on its own
              axis (time, height, width); `inverse` turns back, as the gradient needs it.
  "forward"   softmax attention over packed sequences: a query sees the `window` last tokens of its sequence, itself among them,
              and the first `sinks` tokens.  Query heads share key and value heads in equal groups.  Outputs o and log-sum-exp.
  "backward"  the gradient of the above from the saved o and log-sum-exp, with respect to the fused q | k | v.
  "distill"   token losses and logit gradient: cross-entropy with the target mixed with the divergence from a teacher that is
              known by its top logits, at a temperature.

Head widths, head counts, token counts and vocabularies are those that the package is configured and tested with, their halves
and generic ones; sequences run from one token to 16384, odd lengths among them.  Storage is fp16, as everywhere in the package.
"""
from __future__ import annotations

import math

import torch

own = False      # set by whoever measures: the framework's entry points instead of the plain forms

DEVICE = "cuda:0"
HALF = dict(dtype=torch.float16, device=DEVICE)
SINGLE = dict(dtype=torch.float32, device=DEVICE)
WORKSPACE = 128 << 20      # bytes of scratch memory, as a program keeps it for all its calls


# --------------------------------------------------------------------------------------------------------- cases


def _attention(name, kind, lengths, heads, kv_heads, width, window, sinks, behind=0):
    """lengths: of the packed sequences; behind: rows of the buffers that belong to none (padding of the batch)."""
    return {"name": name, "kind": kind, "lengths": ",".join(str(n) for n in lengths), "heads": heads, "kv_heads": kv_heads,
            "width": width, "window": window, "sinks": sinks, "behind": behind}


def _rope(name, tokens, heads, kv_heads, width, axes, inverse):
    return {"name": name, "kind": "rope", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "width": width, "axes": axes,
            "inverse": inverse}


def _distill(name, tokens, vocab, top, temperature, soft_weight):
    return {"name": name, "kind": "distill", "tokens": tokens, "vocab": vocab, "top": top, "temperature": temperature,
            "soft_weight": soft_weight}


def listed():
    return [
        # a few short sequences of a small model: the smallest calls, where launches and latency are the time
        _attention("forward_short", "forward", [57, 1, 90, 33], 8, 2, 64, 64, 4),
        # a fine-tuning batch from which padding has been removed: documents of mixed lengths packed into 4096 rows
        _attention("forward_packed", "forward", [511, 1300, 77, 1, 960, 640, 600], 32, 8, 128, 1024, 4, 7),
        # heads that share nothing, an odd length and a window that no tile divides
        _attention("forward_odd", "forward", [4095], 32, 32, 128, 1000, 1),
        # long context: one sequence, where the window saves most of the work
        _attention("forward_long", "forward", [16384], 32, 8, 128, 4096, 4),
        # the gradients of the same kinds of batch
        _attention("backward_short", "backward", [57, 1, 90, 33], 8, 2, 64, 64, 4),
        _attention("backward_packed", "backward", [511, 1300, 77, 1, 960, 640, 600], 32, 8, 128, 1024, 4, 7),
        _attention("backward_long", "backward", [16384], 32, 8, 128, 2048, 4),
        # one short prompt with a picture in it
        _rope("rope_short", 333, 8, 2, 64, 3, False),
        # a long batch of text, pictures and video, on the way back
        _rope("rope_long_inverse", 16384, 32, 8, 128, 3, True),
        # one short answer
        _distill("distill_short", 37, 32000, 16, 2.0, 0.5),
        # a batch of the fine-tuning configurations, a vocabulary with eight added tokens
        _distill("distill_batch", 4096, 32008, 64, 2.0, 0.9),
        # a large vocabulary, an odd number of tokens and of kept logits
        _distill("distill_large_vocabulary", 4001, 131080, 127, 1.5, 1.0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_lengths(rng, tokens):
    cuts = sorted({0, tokens, *(rng.randrange(1, tokens) for _ in range(rng.choice([0, 0, 1, 3, 8])) if tokens > 1)})
    return [b - a for a, b in zip(cuts, cuts[1:])]


def draw(rng):
    """Another case of the same ranges: token counts, windows and vocabularies over their logarithm, odd ones among them."""
    heads = [(8, 2, 64), (8, 8, 64), (32, 8, 64), (8, 8, 128), (16, 4, 128), (28, 4, 128), (32, 8, 128), (32, 32, 128)]
    while True:
        kind = rng.choice(["forward", "backward", "forward", "backward", "rope", "distill"])
        h, g, d = rng.choice(heads)
        if kind == "rope":
            case = _rope("", _log_int(rng, 200, 16384), h, g, d, rng.choice([2, 3, 3]), rng.random() < 0.5)
        elif kind == "distill":
            case = _distill("", _log_int(rng, 30, 8192), 8 * _log_int(rng, 500, 16400), _log_int(rng, 1, 256),
                            rng.choice([1.0, 1.5, 2.0, 4.0]), rng.choice([0.3, 0.5, 0.9, 1.0]))
        else:
            case = _attention("", kind, _draw_lengths(rng, _log_int(rng, 100, 16384)), h, g, d, _log_int(rng, 16, 4096),
                              rng.choice([0, 1, 4, 4, 16, 64]), rng.choice([0, 0, 5]))
        del case["name"]
        like = [c for c in listed() if c["kind"] == kind]
        cost = lambda c: max(work(c)["bytes"], work(c)["flops"] / 50)
        if cost(case) <= max(cost(c) for c in like):
            return case


# -------------------------------------------------------------------------------------------------------- inputs


def _lengths(case):
    return [int(n) for n in case["lengths"].split(",")]


def _offsets(case):
    out = [0]
    for n in _lengths(case):
        out.append(out[-1] + n)
    return out


def _generator(seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(int(seed))
    return gen


def _normal(gen, shape, sigma=1.0):
    return torch.randn(shape, generator=gen, **HALF).mul_(sigma)


def _prepare_attention(case, seed):
    gen = _generator(seed)
    h, g, d = case["heads"], case["kv_heads"], case["width"]
    offsets = _offsets(case)
    T = offsets[-1] + case["behind"]
    qkv = _normal(gen, (T, (h + 2 * g) * d))
    state = {"case": case, "qkv": qkv, "offsets": torch.tensor(offsets, dtype=torch.int32, device=DEVICE)}
    if case["kind"] == "forward":
        # rows behind the last sequence stay as they are
        return {**state, "o": torch.zeros(T, h * d, **HALF), "lse": torch.zeros(T, h, **SINGLE)}
    o, lse = _plain_forward(state)
    return {**state, "o": o, "lse": lse, "do": _normal(gen, (T, h * d)), "dqkv": torch.zeros_like(qkv),
            "ws": torch.empty(WORKSPACE, dtype=torch.uint8, device=DEVICE)}


def _positions(tokens, axes, seed):
    """[axes x tokens]: runs of text, where all axes advance together, between pictures and clips on a grid of patches."""
    gen = torch.Generator().manual_seed(int(seed))
    pick = lambda lo, hi: int(torch.randint(lo, hi, (1,), generator=gen))
    runs, filled, at = [], 0, pick(0, 2000)
    while filled < tokens:
        n = pick(20, 400)
        runs.append((torch.arange(n) + at).expand(axes, n))
        filled, at = filled + n, at + n
        t, y, x = pick(1, 6), pick(4, 24), pick(4, 24)
        grid = torch.stack(torch.meshgrid(torch.arange(t), torch.arange(y), torch.arange(x), indexing="ij")).reshape(3, -1)
        runs.append(grid[3 - axes:] + at)
        filled, at = filled + t * y * x, at + max(t, y, x)
    return torch.cat(runs, 1)[:, :tokens].to(torch.int32).contiguous()


def _pair_axis(case):
    """Which axis turns which pair: sections of neighbouring pairs, the first the shortest."""
    half, axes = case["width"] // 2, case["axes"]
    first = half // (axes + 1)
    return [0] * first + [1 + (i * (axes - 1)) // (half - first) for i in range(half - first)]


def _prepare_rope(case, seed):
    gen = _generator(seed)
    T, d, n = case["tokens"], case["width"], case["heads"] + case["kv_heads"]
    positions = _positions(T, case["axes"], seed)
    angle = (torch.arange(int(positions.max()) + 1, device=DEVICE, dtype=torch.float64)[:, None]
             * 1e6 ** (-torch.arange(d // 2, device=DEVICE, dtype=torch.float64) / (d // 2))[None, :])
    return {"case": case, "x": _normal(gen, (T, (n + case["kv_heads"]) * d)), "y": torch.empty(T, n * d, **HALF),
            "cos": angle.cos().float(), "sin": angle.sin().float(), "positions": positions.to(DEVICE), "pair_axis": _pair_axis(case)}


def _prepare_distill(case, seed):
    gen = _generator(seed)
    T, V, K = case["tokens"], case["vocab"], case["top"]
    logits = _normal(gen, (T, V), 2.0)
    # K different tokens, spread over the vocabulary
    draw_int = lambda hi: torch.randint(0, hi, (T, 1), generator=gen, device=DEVICE)
    ids = ((draw_int(V) + (1 + draw_int(V // K)) * torch.arange(K, device=DEVICE)) % V).int()
    teacher = 14.0 - 1.5 * torch.arange(1, K + 1, **SINGLE).log() + torch.randn(T, K, generator=gen, **SINGLE)
    teacher = teacher.sort(dim=1, descending=True).values
    # the student has learnt some of it
    logits.scatter_(1, ids.long(), (teacher + 1.5 * torch.randn(T, K, generator=gen, **SINGLE)).half())
    targets = ids[:, 0].clone()
    targets[torch.rand(T, generator=gen, **SINGLE) < 0.1] = -100      # prompts and padding are not counted
    return {"case": case, "logits": logits, "ids": ids, "teacher": teacher.half(), "targets": targets,
            "scale": 65536.0 / T, "loss": torch.empty(T, **SINGLE), "dlogits": torch.empty(T, V, **HALF)}


def prepare(case, seed):
    return {"rope": _prepare_rope, "distill": _prepare_distill}.get(case["kind"], _prepare_attention)(case, seed)


# --------------------------------------------------------------------------------------------------- plain forms


class _Band:
    """Attention by blocks of as many tokens as the window has: the keys of a block's queries are those of the block and of
    the one before, and the sinks of all sequences beside them."""

    def __init__(self, state):
        case, qkv, off = state["case"], state["qkv"], state["offsets"].long()
        self.h, self.g, self.d = case["heads"], case["kv_heads"], case["width"]
        self.T, self.used, self.B = qkv.shape[0], int(sum(_lengths(case))), off.numel() - 1
        self.bs = min(case["window"], max(_lengths(case)))
        self.nb = -(-self.T // self.bs)
        token = torch.arange(self.nb * self.bs, device=DEVICE)
        seq = torch.bucketize(token, off[1:], right=True)               # B: behind the last sequence
        pos = token - off[seq.clamp(max=self.B - 1)]
        before = lambda x, fill: torch.cat((torch.cat((x.new_full((1, self.bs), fill), x.view(self.nb, self.bs)[:-1])),
                                            x.view(self.nb, self.bs)), 1)
        sq, pq = seq.view(self.nb, self.bs, 1), pos.view(self.nb, self.bs, 1)
        sk, pk = before(seq, -1)[:, None, :], before(pos, 0)[:, None, :]
        self.near = (sq == sk) & (sq < self.B) & (pk <= pq) & (pq - pk < case["window"])
        s = max(1, case["sinks"])
        sink_seq = torch.arange(self.B, device=DEVICE).repeat_interleave(s)
        sink_pos = torch.arange(s, device=DEVICE).repeat(self.B)
        self.sink_rows = (off[sink_seq] + sink_pos).clamp(max=self.T - 1)
        self.far = (sq == sink_seq) & (pq - sink_pos >= case["window"]) & (sink_pos < case["sinks"])

    def queries(self, x):      # [T x h d] -> [g, block, query heads of the group and rows, d]
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, self.nb * self.bs - self.T))
        x = x.view(self.nb, self.bs, self.g, self.h // self.g, self.d)
        return x.permute(2, 0, 3, 1, 4).reshape(self.g, self.nb, -1, self.d)

    def tokens(self, x):       # and back: [T x h d]
        x = x.view(self.g, self.nb, self.h // self.g, self.bs, -1).permute(1, 3, 0, 2, 4)
        return x.reshape(self.nb * self.bs, -1)[:self.T]

    def keys(self, x):         # [T x g d] -> the two blocks' keys [g, block, 2 bs, d], the sinks [g, 1, B s, d]
        x = x.float().view(self.T, self.g, self.d).transpose(0, 1)
        blocks = torch.nn.functional.pad(x, (0, 0, 0, self.nb * self.bs - self.T)).reshape(self.g, self.nb, self.bs, self.d)
        return (torch.cat((torch.cat((torch.zeros_like(blocks[:, :1]), blocks[:, :-1]), 1), blocks), 2),
                x[:, self.sink_rows][:, None].contiguous())

    def key_tokens(self, near, far):      # the sums of the two blocks' and the sinks' gradients: [T x g d]
        x = near[:, :, self.bs:].clone()
        x[:, :-1] += near[:, 1:, :self.bs]
        x = x.reshape(self.g, -1, self.d)[:, :self.T]
        x = x.index_add(1, self.sink_rows, far)
        return x.transpose(0, 1).reshape(self.T, -1)

    def masked(self, near, far, value):
        rep = lambda m: m.repeat(1, self.h // self.g, 1)[None]
        return near.masked_fill_(~rep(self.near), value), far.masked_fill_(~rep(self.far), value)

    def split(self, qkv):
        return qkv.split([self.h * self.d, self.g * self.d, self.g * self.d], 1)


def _times(x, keys):      # [g, block, m, d] with [g, block or 1, n, d]
    return x @ keys.transpose(-1, -2).contiguous()


def _plain_forward(state):
    band = _Band(state)
    q, k, v = band.split(state["qkv"])
    q, (kn, kf), (vn, vf) = band.queries(q) * band.d ** -0.5, band.keys(k), band.keys(v)
    near, far = band.masked(_times(q, kn), _times(q, kf), -math.inf)
    top = torch.maximum(near.amax(-1, True), far.amax(-1, True))
    top = top.masked_fill(top == -math.inf, 0.0)                        # rows behind the last sequence
    near, far = near.sub_(top).exp_(), far.sub_(top).exp_()
    total = near.sum(-1, True) + far.sum(-1, True)
    o = band.tokens((near @ vn + far @ vf) / total)
    lse = band.tokens(top + total.log())
    o[band.used:], lse[band.used:] = 0.0, 0.0
    return o.half(), lse.contiguous()


def _plain_backward(state):
    band = _Band(state)
    q, k, v = band.split(state["qkv"])
    q, (kn, kf), (vn, vf) = band.queries(q), band.keys(k), band.keys(v)
    do, o = band.queries(state["do"]), band.queries(state["o"])
    T, h, rows = band.T, band.h, band.nb * band.bs
    lse = torch.nn.functional.pad(state["lse"], (0, 0, 0, rows - T)).view(band.nb, band.bs, band.g, h // band.g)
    lse = lse.permute(2, 0, 3, 1).reshape(band.g, band.nb, -1, 1)
    delta, scale = (do * o).sum(-1, True), band.d ** -0.5
    pn, pf = band.masked(_times(q, kn).mul_(scale).sub_(lse).exp_(), _times(q, kf).mul_(scale).sub_(lse).exp_(), 0.0)
    merged = lambda p, x: (p.transpose(-1, -2).contiguous() @ x)        # [g, block, keys, d]
    dv = band.key_tokens(merged(pn, do), merged(pf, do).sum(1))
    dn = _times(do, vn).sub_(delta).mul_(pn).mul_(scale)
    df = _times(do, vf).sub_(delta).mul_(pf).mul_(scale)
    del pn, pf
    dq = band.tokens(dn @ kn + df @ kf)
    dk = band.key_tokens(merged(dn, q), merged(df, q).sum(1))
    dqkv = torch.cat((dq, dk, dv), 1)
    dqkv[band.used:] = 0.0
    return dqkv.half()


def _plain_rope(state):
    case, T = state["case"], state["case"]["tokens"]
    d, n = case["width"], case["heads"] + case["kv_heads"]
    pos = state["positions"].long()[torch.tensor(state["pair_axis"], device=DEVICE)]      # [d / 2 x T]
    pair = torch.arange(d // 2, device=DEVICE)
    cos = state["cos"][pos.t(), pair][:, None]
    sin = state["sin"][pos.t(), pair][:, None] * (-1.0 if case["inverse"] else 1.0)
    x = state["x"][:, :n * d].float().view(T, n, d)
    a, b = x[..., :d // 2], x[..., d // 2:]
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).view(T, n * d).half()


def _plain_distill(state):
    case, z = state["case"], state["logits"].float()
    tau, mix, V = case["temperature"], case["soft_weight"], case["vocab"]
    ids, targets = state["ids"].long(), state["targets"].long()
    counted = (targets >= 0) & (targets < V)
    at = targets.clamp(0, V - 1)[:, None]
    log_p = state["teacher"].float() / tau
    log_p = log_p - log_p.amax(1, True)
    log_p = log_p - log_p.exp().sum(1, True).log()
    top = z.amax(1, True)
    hard, soft = (z - top).exp(), ((z - top) / tau).exp()
    hard_sum, soft_sum = hard.sum(1, True), soft.sum(1, True)
    log_q = (z.gather(1, ids) - top) / tau - soft_sum.log()
    divergence = tau * tau * (log_p.exp() * (log_p - log_q)).sum(1)
    cross = (top + hard_sum.log() - z.gather(1, at))[:, 0]
    loss = torch.where(counted, (1.0 - mix) * cross + mix * divergence, torch.zeros_like(cross))
    # 1 - probability of the target without cancellation, as far as 32 bits of a sum allow
    grad = (1.0 - mix) / hard_sum * hard.scatter_add(1, at, -hard_sum) + mix * tau / soft_sum * soft.scatter_add(
        1, ids, -log_p.exp() * soft_sum)
    grad *= counted[:, None] * state["scale"]
    return loss, grad.half()


def run(state):
    case = state["case"]
    kind = case["kind"]
    if not own:
        if kind == "rope":
            return {"y": _plain_rope(state)}
        if kind == "distill":
            return dict(zip(("loss", "dlogits"), _plain_distill(state)))
        if kind == "forward":
            return dict(zip(("o", "lse"), _plain_forward(state)))
        return {"dqkv": _plain_backward(state)}
    import paper_2306_09782_amd as L
    if kind == "rope":
        L.lomo_rope_axes(state["x"], state["y"], state["cos"], state["sin"], state["positions"], state["pair_axis"],
                         case["heads"] + case["kv_heads"], case["width"], inverse=case["inverse"])
        return {"y": state["y"]}
    if kind == "distill":
        L.lomo_distill(state["logits"], state["ids"], state["teacher"], state["targets"], state["scale"], case["temperature"],
                       case["soft_weight"], state["loss"], state["dlogits"])
        return {"loss": state["loss"], "dlogits": state["dlogits"]}
    if kind == "forward":
        L.lomo_window_attention_forward(state["qkv"], state["o"], state["lse"], state["offsets"], case["heads"], case["kv_heads"],
                                        case["window"], case["sinks"])
        return {"o": state["o"], "lse": state["lse"]}
    L.lomo_window_attention_backward(state["qkv"], state["o"], state["do"], state["lse"], state["dqkv"], state["offsets"],
                                     case["heads"], case["kv_heads"], case["window"], case["sinks"], state["ws"])
    return {"dqkv": state["dqkv"]}


# ---------------------------------------------------------------------------------------------------------- work


def _visible(n, window, sinks):
    """Pairs of a query and a key that it sees, in a sequence of n tokens."""
    full = min(n, window)
    pairs = full * (full + 1) // 2 + (n - full) * window
    reach = min(sinks, max(0, n - window))              # queries that have left 1, 2, .. first tokens behind them
    return pairs + reach * (reach + 1) // 2 + (max(0, n - window) - reach) * sinks


def work(case):
    """Bytes: every input read once and every output written once.  Flops: the products over the visible pairs, two of them
    forwards and five backwards; of the others the arithmetic per element."""
    if case["kind"] == "rope":
        T, n, d = case["tokens"], case["heads"] + case["kv_heads"], case["width"]
        return {"bytes": 4.0 * T * n * d + 4.0 * case["axes"] * T + 4.0 * T * d, "flops": 3.0 * T * n * d}
    if case["kind"] == "distill":
        T, V, K = case["tokens"], case["vocab"], case["top"]
        return {"bytes": 4.0 * T * V + 6.0 * T * K + 8.0 * T, "flops": 12.0 * T * V}
    h, g, d = case["heads"], case["kv_heads"], case["width"]
    T = sum(_lengths(case))
    pairs = float(sum(_visible(n, case["window"], case["sinks"]) for n in _lengths(case)))
    if case["kind"] == "forward":
        return {"bytes": 2.0 * T * (2 * h + 2 * g) * d + 4.0 * T * h, "flops": 4.0 * d * h * pairs}
    return {"bytes": 2.0 * T * (4 * h + 4 * g) * d + 4.0 * T * h, "flops": 10.0 * d * h * pairs}


# --------------------------------------------------------------------------------------- definitions in 64 bits


def _exact_attention(state):
    """Sequence by sequence and head by head over the whole square of scores."""
    case, backward = state["case"], state["case"]["kind"] == "backward"
    h, g, d = case["heads"], case["kv_heads"], case["width"]
    off = _offsets(case)
    T = state["qkv"].shape[0]
    double = dict(dtype=torch.float64, device=DEVICE)
    o, lse, grad = torch.zeros(T, h, d, **double), torch.zeros(T, h, **double), torch.zeros(T, h + 2 * g, d, **double)
    x = state["qkv"].view(T, h + 2 * g, d)
    for a, b in zip(off, off[1:]):
        i = torch.arange(b - a, device=DEVICE)
        gap = i[:, None] - i[None, :]
        hidden = (gap < 0) | ((gap >= case["window"]) & (i[None, :] >= case["sinks"]))
        del gap
        for n in range(h):
            q, k, v = (x[a:b, c].double() for c in (n, h + n // (h // g), h + g + n // (h // g)))
            s = (q @ k.t().contiguous()).div_(math.sqrt(d)).masked_fill_(hidden, -math.inf)
            if not backward:
                lse[a:b, n] = torch.logsumexp(s, 1)
                o[a:b, n] = torch.softmax(s, 1) @ v
                continue
            p = s.sub_(state["lse"][a:b, n, None].double()).exp_()
            do, out = (state[w].view(T, h, d)[a:b, n].double() for w in ("do", "o"))
            grad[a:b, h + g + n // (h // g)] += p.t().contiguous() @ do
            ds = (do @ v.t().contiguous()).sub_((do * out).sum(1, keepdim=True)).mul_(p).div_(math.sqrt(d))
            grad[a:b, n] = ds @ k
            grad[a:b, h + n // (h // g)] += ds.t().contiguous() @ q
    return {"dqkv": grad.view(T, -1)} if backward else {"o": o.view(T, -1), "lse": lse}


def _exact_rope(state):
    case, T, d = state["case"], state["case"]["tokens"], state["case"]["width"]
    n, half = case["heads"] + case["kv_heads"], d // 2
    y = torch.empty(T, n, d, dtype=torch.float64, device=DEVICE)
    x = state["x"].view(T, -1, d)[:, :n].double()
    for c, axis in enumerate(state["pair_axis"]):
        at = state["positions"][axis].long()
        turn = torch.complex(state["cos"][at, c].double(), state["sin"][at, c].double())
        pair = torch.complex(x[:, :, c], x[:, :, c + half]) * (turn.conj() if case["inverse"] else turn)[:, None]
        y[:, :, c], y[:, :, c + half] = pair.real, pair.imag
    return {"y": y.view(T, n * d)}


def _exact_distill(state):
    case = state["case"]
    T, V, tau, mix = case["tokens"], case["vocab"], case["temperature"], case["soft_weight"]
    loss = torch.zeros(T, dtype=torch.float64, device=DEVICE)
    grad = torch.zeros(T, V, dtype=torch.float64, device=DEVICE)
    for a in range(0, T, 512):
        rows = slice(a, min(T, a + 512))
        z, target = state["logits"][rows].double(), state["targets"][rows].long()
        index = torch.arange(z.shape[0], device=DEVICE)
        p = torch.softmax(state["teacher"][rows].double() / tau, 1)
        want = torch.zeros_like(z).index_put_((index[:, None], state["ids"][rows].long()), p, accumulate=True)
        log_q, log_h = torch.log_softmax(z / tau, 1), torch.log_softmax(z, 1)
        counted = (target >= 0) & (target < V)
        target = target.where(counted, torch.zeros_like(target))
        soft = (p * p.log()).sum(1) - (want * log_q).sum(1)
        loss[rows] = torch.where(counted, mix * tau * tau * soft - (1 - mix) * log_h[index, target], 0.0)
        one = torch.zeros_like(z).index_put_((index, target), torch.ones_like(loss[rows]))
        grad[rows] = ((1 - mix) * (log_h.exp() - one) + mix * tau * (log_q.exp() - want)) * counted[:, None] * state["scale"]
    return {"loss": loss, "dlogits": grad}


def exact(case, seed):
    state = prepare(case, seed)
    return {"rope": _exact_rope, "distill": _exact_distill}.get(case["kind"], _exact_attention)(state)
