"""What the operators of token sequence models are timed on, and their plain forms.

Three operators, for layers that train or run beside the spiking ones:

  glr    a gated linear recurrence over [T][batch][n]: a = sigmoid(z), h_t = a_t h_{t-1} + (1 - a_t) x_t, and its backward pass from
         states kept every 128 steps.  z is what a projection gives for the gate, about +2 with a spread of 1.5 (a memory of some ten
         steps, now and then of hundreds).  `ragged`: sequences of a batch have lengths of their own, down to one step.
         call: "forward" (h, last state, kept states), "backward" (dz, dx, dh0), "packed" (backward from z and x in 8 bits).
  pack   activations [rows][cols] to 8 bits and back: blocks of 32 along a row share a power of two as their step.
  vocab  softmax cross entropy of rows h against a vocabulary w [vocab][d], one target per row (-1: none; about 5 % of the rows).
         call: "loss" (evaluation: the loss of each row), "train" (the losses, and the gradients of h and w of their mean).
         h has unit entries and w a spread of 3 / sqrt(d), so that logits spread over about +-10.

`dtype` is the type of activations and weights; states and losses are float32 in either.
"""
import math

import torch

own = False

BLOCK = 32      # elements of a row that share a step in 8 bits
INTERVAL = 128  # steps between the states that the forward pass keeps
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "bfloat16": 2}


def _glr(name, call, dtype, T, batch, n, ragged=False):
    c = dict(op="glr", call=call, dtype=dtype, T=T, batch=batch, n=n, ragged=ragged)
    return dict(c, name=name) if name else c


def _pack(name, dtype, rows, cols):
    c = dict(op="pack", dtype=dtype, rows=rows, cols=cols)
    return dict(c, name=name) if name else c


def _vocab(name, call, dtype, rows, d, vocab):
    c = dict(op="vocab", call=call, dtype=dtype, rows=rows, d=d, vocab=vocab)
    return dict(c, name=name) if name else c


def listed():
    return [
        # serving: one new token for each of 64 sequences, the state carried from call to call
        _glr("glr_token", "forward", "bfloat16", 1, 64, 2048),
        # a small layer whose sizes fit no tile, sequences of different lengths
        _glr("glr_forward_ragged", "forward", "float32", 333, 13, 75, ragged=True),
        # the forward pass of a layer in training
        _glr("glr_forward", "forward", "bfloat16", 4096, 8, 2048),
        # backward pass of a wide layer in 32 bits on a padded batch
        _glr("glr_backward_f32", "backward", "float32", 1000, 32, 1024, ragged=True),
        # backward pass over one long document: the batch leaves few channels
        _glr("glr_backward_long", "backward", "bfloat16", 32768, 1, 1024),
        # the training case again with its gate and drive kept in 8 bits
        _glr("glr_backward_packed", "packed", "bfloat16", 4096, 8, 2048),
        # checkpoints of a small layer with an odd width
        _pack("pack_ragged", "float32", 4329, 1501),
        # checkpoints of a layer's activations over a whole batch
        _pack("pack_batch", "bfloat16", 32768, 4096),
        # the readout of a small model on one time step of a batch
        _vocab("vocab_small", "train", "float32", 32, 256, 1000),
        # evaluation of a validation batch
        _vocab("vocab_eval", "loss", "bfloat16", 4096, 2048, 50021),
        # a training step of a model kept in 32 bits
        _vocab("vocab_train_f32", "train", "float32", 2000, 1024, 20011),
        # a training step with a large vocabulary: batch 8 of 1024 steps
        _vocab("vocab_train", "train", "bfloat16", 8192, 2048, 128000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Half of them multiples of 64, the others as they come."""
    n = _log_int(rng, lo, hi)
    return max(lo, n // 64 * 64) if rng.random() < 0.5 else n


def _draw(rng):
    dtype = rng.choice(list(TYPES))
    op = rng.choice(["glr", "glr", "pack", "vocab"])
    if op == "glr":
        call = rng.choice(["forward", "backward", "packed"])
        T = 1 if call == "forward" and rng.random() < 0.2 else _log_int(rng, 2, 32768)
        return _glr(None, call, dtype, T, _log_int(rng, 1, 64), _width(rng, 16, 4096), ragged=rng.random() < 0.4)
    if op == "pack":
        return _pack(None, dtype, _log_int(rng, 1, 32768), _width(rng, 16, 8192))
    return _vocab(None, rng.choice(["loss", "train"]), dtype, _log_int(rng, 1, 8192), _width(rng, 64, 2048), _width(rng, 64, 128000))


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        top[c["op"]] = max(top.get(c["op"], (0, 0)), (w["bytes"], w["flops"]))
    while True:
        c = _draw(rng)
        w = work(c)
        # 32 bits cost about six times the matrix time of 16
        flops = w["flops"] * (6 if c["op"] == "vocab" and c["dtype"] == "float32" else 1)
        if w["bytes"] <= top[c["op"]][0] and flops <= top[c["op"]][1]:
            return c


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 17)
    t = TYPES[case["dtype"]]
    if case["op"] == "pack":
        # activations spread over some orders of magnitude from row to row
        x = _normal(g, case["rows"], case["cols"]) * torch.exp(_normal(g, case["rows"], 1))
        return dict(case=case, x=x.to(t))
    if case["op"] == "vocab":
        rows, d, vocab = case["rows"], case["d"], case["vocab"]
        h = _normal(g, rows, d).to(t)
        w = (_normal(g, vocab, d) * (3.0 / math.sqrt(d))).to(t)
        target = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
        none = torch.rand((rows,), generator=g, device="cuda") < 0.05
        none[0] = False
        return dict(case=case, h=h, w=w, target=torch.where(none, torch.full_like(target, -1), target))
    T, B, n = case["T"], case["batch"], case["n"]
    s = dict(case=case, z=(2.0 + 1.5 * _normal(g, T, B, n)).to(t), x=_normal(g, T, B, n).to(t), h0=0.5 * _normal(g, B, n), lengths=None)
    if case["ragged"]:
        s["lengths"] = torch.randint(1, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    if case["call"] == "forward":
        return s
    s["dh"] = _normal(g, T, B, n).to(t)
    if case["call"] == "packed":
        s["z"], s["x"] = _to_bytes(s["z"]), _to_bytes(s["x"])
        z, x = _values(s["z"], torch.float32, n), _values(s["x"], torch.float32, n)
    else:
        z, x = s["z"].float(), s["x"].float()
    s["kept"] = _states(z, x, s["h0"], s["lengths"])[2]
    return s


# ---- plain forms ---------------------------------------------------------------------------------
def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the first axis from zero, by doubling the steps that each entry spans."""
    k = 1
    while k < a.shape[0]:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _held(T, lengths):
    """[T][B][1]: steps behind the end of a sequence."""
    return torch.arange(T, device=lengths.device)[:, None, None] >= lengths[None, :, None]


def _states(z, x, h0, lengths):
    """h with the state held behind a sequence's end, the last state, the states before the steps 0, 128, 256, ..."""
    a, b = torch.sigmoid(z), torch.sigmoid(-z) * x
    if lengths is not None:
        held = _held(z.shape[0], lengths)
        a, b = torch.where(held, 1.0, a), torch.where(held, 0.0, b)
    b = torch.cat([b[:1] + a[:1] * h0, b[1:]])
    h = _scan(a, b)
    return h, h[-1], torch.cat([h0[None], h[:-1]])[::INTERVAL].contiguous()


def _glr_forward(s):
    h, last, kept = _states(s["z"].float(), s["x"].float(), s["h0"], s["lengths"])
    if s["lengths"] is not None:
        h = torch.where(_held(h.shape[0], s["lengths"]), 0.0, h)
    return h.to(s["z"].dtype), last, kept


def _glr_backward(s, z, x, dtype):
    a, c, lengths = torch.sigmoid(z), torch.sigmoid(-z), s["lengths"]
    dh, h0 = s["dh"].float(), s["kept"][0]
    h = _states(z, x, h0, lengths)[0]
    before = torch.cat([h0[None], h[:-1]])
    hold = a
    if lengths is not None:
        held = _held(z.shape[0], lengths)
        hold, dh = torch.where(held, 1.0, a), torch.where(held, 0.0, dh)
    ahead = torch.cat([hold[1:], torch.ones_like(hold[:1])])
    g = _scan(ahead.flip(0), dh.flip(0)).flip(0)
    dz, dx = a * c * (before - x) * g, c * g
    if lengths is not None:
        dz, dx = torch.where(held, 0.0, dz), torch.where(held, 0.0, dx)
    return dz.to(dtype), dx.to(dtype), hold[0] * g[0]


def _to_bytes(x):
    """Codes and the exponent byte of each block: its step is the smallest power of two (from 2^-126) that no code exceeds 127 with."""
    n = x.shape[-1]
    v = torch.nn.functional.pad(x.float(), (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = v.abs().amax(-1)
    m, e = torch.frexp(top)
    k = torch.where(torch.round(m * 128) > 127, e - 6, e - 7).clamp(min=-126)
    exps = torch.where(top == 0, 0, k + 127).to(torch.uint8)
    step = torch.where(top == 0, 1.0, _steps(exps))
    return torch.round(v / step[..., None]).to(torch.int8).flatten(-2)[..., :n].contiguous(), exps


def _steps(exps):
    return (exps.to(torch.int32) << 23).view(torch.float32)


def _values(p, dtype, n):
    codes, exps = p
    return (codes.float() * _steps(exps).repeat_interleave(BLOCK, -1)[..., :n]).to(dtype)


def _vocab_plain(s):
    h, w, target = s["h"].float(), s["w"].float(), s["target"].long()
    counted = target >= 0
    label = target.clamp(min=0)[:, None]
    logits = h @ w.T
    top = logits.amax(1, keepdim=True)
    e = torch.exp(logits - top)
    total = e.sum(1, keepdim=True)
    loss = torch.where(counted, (torch.log(total) + top - logits.gather(1, label))[:, 0], 0.0)
    if s["case"]["call"] == "loss":
        return loss
    G = e / total
    G.scatter_add_(1, label, torch.full_like(total, -1.0))
    G *= (counted / counted.sum())[:, None]
    return loss, (G @ w).to(s["h"].dtype), (G.T @ h).to(s["w"].dtype)


def _run_plain(s):
    case = s["case"]
    if case["op"] == "pack":
        return _values(_to_bytes(s["x"]), s["x"].dtype, case["cols"])
    if case["op"] == "vocab":
        return _vocab_plain(s)
    if case["call"] == "forward":
        return _glr_forward(s)
    if case["call"] == "packed":
        return _glr_backward(s, _values(s["z"], torch.float32, case["n"]), _values(s["x"], torch.float32, case["n"]), s["dh"].dtype)
    return _glr_backward(s, s["z"].float(), s["x"].float(), s["dh"].dtype)


def _run_own(s):
    import paper_2412_11810_amd as snn

    case = s["case"]
    if case["op"] == "pack":
        return snn.snn_unpack(snn.snn_pack(s["x"]), s["x"].dtype)
    if case["op"] == "vocab":
        loss, state = snn.snn_vocab_loss(s["h"], s["w"], s["target"])
        if case["call"] == "loss":
            return loss
        return loss, *snn.snn_vocab_loss_grad(s["h"], s["w"], s["target"], state)
    if case["call"] == "forward":
        return snn.snn_glr_forward(s["z"], s["x"], s["h0"], lengths=s["lengths"], keep=True)
    z, x = (snn.Packed(*s["z"]), snn.Packed(*s["x"])) if case["call"] == "packed" else (s["z"], s["x"])
    return snn.snn_glr_backward(z, x, s["kept"], s["dh"], lengths=s["lengths"])


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    s = SIZE[case["dtype"]]
    if case["op"] == "pack":
        x = case["rows"] * case["cols"]
        codes = x + case["rows"] * -(-case["cols"] // BLOCK)
        return {"bytes": 2 * (s * x + codes), "flops": 4 * x}  # to 8 bits and back
    if case["op"] == "vocab":
        rows, d, vocab = case["rows"], case["d"], case["vocab"]
        train = case["call"] == "train"
        return {"bytes": (2 if train else 1) * s * (rows + vocab) * d + 8 * rows, "flops": (6 if train else 2) * rows * d * vocab}
    channels = case["batch"] * case["n"]
    x, kept = case["T"] * channels, -(-case["T"] // INTERVAL) * channels
    if case["call"] == "forward":
        return {"bytes": 3 * s * x + 4 * (2 * channels + kept), "flops": 10 * x}
    read = 2 * (x + case["T"] * case["batch"] * -(-case["n"] // BLOCK)) if case["call"] == "packed" else 2 * s * x
    return {"bytes": read + 3 * s * x + 4 * (channels + kept), "flops": 25 * x}


# ---- the definitions in 64 bits, step by step ----------------------------------------------------
def _exact_values(p, n):
    codes, exps = (v.double() for v in p)
    return codes * torch.exp2(exps - 127).repeat_interleave(BLOCK, -1)[..., :n]


def _exact_glr(s):
    case = s["case"]
    T, n = case["T"], case["n"]
    z, x = (_exact_values(s[k], n) if case["call"] == "packed" else s[k].double() for k in ("z", "x"))
    a = 1 / (1 + torch.exp(-z))
    c = 1 / (1 + torch.exp(z))
    live = torch.ones((T, case["batch"], 1), dtype=torch.float64, device=z.device)
    if s["lengths"] is not None:
        live = (torch.arange(1, T + 1, device=z.device)[:, None] <= s["lengths"][None, :])[..., None].double()
    u = c * live  # how far a step moves the state towards its drive
    state = (s["h0"] if case["call"] == "forward" else s["kept"][0]).double()
    before = torch.empty_like(z)
    for t in range(T):
        before[t] = state
        state = torch.addcmul(state, u[t], x[t] - state)
    if case["call"] == "forward":
        return (before + u * (x - before)) * live, state, before[::INTERVAL].clone()
    g, dh = torch.zeros_like(state), s["dh"].double() * live
    back = torch.empty_like(z)
    for t in range(T - 1, -1, -1):
        g = g + dh[t]
        back[t] = g
        g = torch.addcmul(g, u[t], g, value=-1)
    return a * u * (before - x) * back, u * back, g


def exact(case, seed):
    if case["op"] == "glr" and case["T"] * case["batch"] * case["n"] > 1 << 28:
        return None
    s = prepare(case, seed)
    if case["op"] == "glr":
        return _exact_glr(s)
    if case["op"] == "pack":
        x = s["x"].double()
        v = torch.nn.functional.pad(x, (0, -case["cols"] % BLOCK)).unflatten(-1, (-1, BLOCK))
        top = v.abs().amax(-1, keepdim=True)
        # rounded to even, top / step is at most 127 where it is below 127.5
        k = (torch.floor(torch.log2(top.clamp(min=2.0 ** -149) / 127.5)) + 1).clamp(min=-126)
        step = torch.exp2(k)
        return (torch.round(v / step) * step).flatten(-2)[..., :case["cols"]]
    h, w, target = s["h"].double(), s["w"].double(), s["target"].long()
    counted = (target >= 0).double()
    label = target.clamp(min=0)
    logits = torch.mm(h, w.t())
    lse = torch.logsumexp(logits, 1)
    loss = (lse - logits[torch.arange(len(label)), label]) * counted
    if case["call"] == "loss":
        return loss
    p = torch.exp(logits - lse[:, None])
    p[torch.arange(len(label)), label] -= 1
    p *= (counted / counted.sum())[:, None]
    return loss, torch.mm(p, w), torch.mm(p.t(), h)
