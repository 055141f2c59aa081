"""What the layer, the norm and the optimizer step of token sequence models are timed on, and their plain forms.

Three operators, for models whose other parts are the recurrence, the 8-bit activations and the vocabulary loss that the library has:

  delta  a gated delta rule, a layer whose state is a matrix per head: over [T][batch][heads]
           S_t = a_t S_{t-1} + k_t u_t^T,  u_t = beta_t (v_t - a_t S_{t-1}^T k_t),  o_t = scale S_t^T q_t,  a_t = exp(g_t).
         Keys have length one and something in common, as behind a nonlinearity; decays make memories of a few to some hundred steps.
         `key_heads` divides `heads`: queries and keys are shared by consecutive heads.  `ragged`: sequences of a batch have lengths of their own.
         call: "forward" (o, the last state, states kept every 256 steps), "backward" (dq, dk, dv, dg, dbeta, ds0).
  norm   rows s = x + residual (or x), y = w s / sqrt(mean(s^2) + eps).
         call: "forward" (y, s), "packed" (y in 8 bits: blocks of 32 along a row share a power of two), "backward" (dx, dw).
  adamw  a step of AdamW over all tensors of a model: `layers` times four matrices [width][width], one [width][4 width] and back, and two vectors,
         then, with vocab > 0, a table [vocab][width].  "bfloat16": gradients in bfloat16, weights in float32 with a copy in bfloat16.
         bits: 32 (m and v), or 8 (m and the root of v, blocks of 32 elements with a power of two as their step, rounded up or
         down by a threshold that a lattice over elements and steps gives).

`dtype` is the type of activations and their gradients (norm: of w as well); states, gates and moments are float32.
"""
import math

import torch

own = False

CHUNK = 64      # steps that the plain form takes at once
KEPT = 256      # steps between the states that the forward pass keeps
BLOCK = 32      # elements that share a step in 8 bits
EPS = 1e-6      # of the norm
STEP = 1000     # of the optimizer
LR, BETA1, BETA2, ADAM_EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.1
LATTICE = 0xC13FA9A9, 0x91E10DA5  # 2^32 times 1 / r and 1 / r^2, r^3 = r + 1
TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16}
SIZE = {"float32": 4, "bfloat16": 2}


def _named(name, c):
    return dict(c, name=name) if name else c


def _delta(name, call, dtype, T, batch, heads, key_heads, dk, dv, ragged=False):
    return _named(name, dict(op="delta", call=call, dtype=dtype, T=T, batch=batch, heads=heads, key_heads=key_heads, dk=dk, dv=dv, ragged=ragged))


def _norm(name, call, dtype, rows, n, residual=True):
    return _named(name, dict(op="norm", call=call, dtype=dtype, rows=rows, n=n, residual=residual))


def _adamw(name, dtype, bits, layers, width, vocab):
    return _named(name, dict(op="adamw", dtype=dtype, bits=bits, layers=layers, width=width, vocab=vocab))


def listed():
    return [
        # serving: one new token for each of 64 sequences, the state carried from call to call
        _delta("delta_token", "forward", "bfloat16", 1, 64, 16, 16, 128, 128),
        # a small layer whose sizes fit no tile, keys shared by three heads, sequences of different lengths
        _delta("delta_forward_ragged", "forward", "float32", 333, 5, 6, 2, 48, 75, ragged=True),
        # the forward pass of a layer in training
        _delta("delta_forward", "forward", "bfloat16", 4096, 8, 16, 16, 128, 128),
        # its backward pass
        _delta("delta_backward", "backward", "bfloat16", 4096, 8, 16, 16, 128, 128),
        # backward pass over a long document in 32 bits, keys shared by two heads: the batch leaves few heads
        _delta("delta_backward_long", "backward", "float32", 16384, 1, 8, 4, 64, 128),
        # serving: the norm of one token of 64 sequences
        _norm("norm_token", "forward", "bfloat16", 64, 2048),
        # rows of odd width in 32 bits
        _norm("norm_ragged", "forward", "float32", 4329, 1501),
        # training: the norm before a projection that takes 8 bits
        _norm("norm_packed", "packed", "bfloat16", 32768, 4096),
        # and the backward pass of one
        _norm("norm_backward", "backward", "bfloat16", 32768, 4096),
        # a small model kept in 32 bits
        _adamw("adamw_small", "float32", 32, 2, 75, 1000),
        # a model whose moments are kept in 8 bits
        _adamw("adamw_8_bits", "bfloat16", 8, 8, 1024, 50021),
        # a model with a large vocabulary
        _adamw("adamw_large", "bfloat16", 32, 2, 2048, 128000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi, by=64):
    """Half of them multiples of `by`, the others as they come."""
    n = _log_int(rng, lo, hi)
    return max(lo, n // by * by) if rng.random() < 0.5 else n


def _draw(rng):
    dtype = rng.choice(list(TYPES))
    op = rng.choice(["delta", "delta", "norm", "adamw"])
    if op == "delta":
        call = rng.choice(["forward", "backward"])
        T = 1 if call == "forward" and rng.random() < 0.2 else _log_int(rng, 2, 16384)
        key_heads = _log_int(rng, 1, 16)
        return _delta(None, call, dtype, T, _log_int(rng, 1, 64), key_heads * rng.choice([1, 1, 2, 3]), key_heads,
                      _width(rng, 16, 128, 16), _width(rng, 16, 256, 16), ragged=rng.random() < 0.4)
    if op == "norm":
        return _norm(None, rng.choice(["forward", "packed", "backward"]), dtype, _log_int(rng, 1, 32768), _width(rng, 16, 8192), rng.random() < 0.7)
    return _adamw(None, dtype, rng.choice([8, 32]), rng.randint(1, 8), _width(rng, 16, 2048), rng.choice([0, _log_int(rng, 64, 128000)]))


def draw(rng):
    top = {}
    for c in listed():
        w = work(c)
        top[c["op"]] = max(top.get(c["op"], (0, 0)), (w["bytes"], w["flops"]))
    while True:
        c = _draw(rng)
        w = work(c)
        # 32 bits cost about six times the matrix time of 16
        flops = w["flops"] * (6 if c["op"] == "delta" and c["dtype"] == "float32" else 1)
        if w["bytes"] <= top[c["op"]][0] and flops <= top[c["op"]][1]:
            return c


# ---- inputs --------------------------------------------------------------------------------------
def _normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _shapes(case):
    d = case["width"]
    layer = [(d, d)] * 4 + [(d, 4 * d), (4 * d, d), (d,), (d,)]
    return layer * case["layers"] + ([(case["vocab"], d)] if case["vocab"] else [])


def _prepare_delta(case, g, t):
    T, B, H, K, dk, dv = (case[k] for k in ("T", "batch", "heads", "key_heads", "dk", "dv"))
    q, k = _normal(g, T, B, K, dk), _normal(g, T, B, K, dk) + 0.5 * _normal(g, 1, B, K, dk)
    q, k = (x / x.norm(dim=-1, keepdim=True) for x in (q, k))
    s = dict(case=case, q=q.to(t), k=k.to(t), v=_normal(g, T, B, H, dv).to(t), lengths=None, s0=0.5 * _normal(g, B, H, dk, dv),
             # a softplus with a rate per head: about 0.3 to 0.003
             g=-torch.log1p(torch.exp(_normal(g, T, B, H) - 1.0)) * torch.exp(-3.0 * torch.rand((H,), generator=g, device="cuda")),
             beta=torch.sigmoid(_normal(g, T, B, H)))
    if case["ragged"]:
        s["lengths"] = torch.randint(1, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    if case["call"] == "backward":
        s["do"] = _normal(g, T, B, H, dv).to(t)
        s["ds_last"] = _normal(g, B, H, dk, dv)
        s["kept"] = _delta_plain(s, out=False)[2]
    return s


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 6007 + 29)
    t = TYPES[case["dtype"]]
    if case["op"] == "delta":
        return _prepare_delta(case, g, t)
    if case["op"] == "norm":
        rows, n = case["rows"], case["n"]
        # rows whose sizes differ, weights around one
        s = dict(case=case, x=(_normal(g, rows, n) * torch.exp(0.5 * _normal(g, rows, 1))).to(t), w=(1 + 0.2 * _normal(g, n)).to(t))
        if case["call"] == "backward":
            s["dy"] = _normal(g, rows, n).to(t)
        s["r"] = _normal(g, rows, n).to(t) if case["residual"] else None  # (backwards: what comes past the norm)
        return s
    shapes = _shapes(case)
    counts = [math.prod(x) for x in shapes]
    # gradients of a spread over tensors; moments as after many such steps: m a tenth of a gradient's size, the root of v about that size
    size = torch.exp(_normal(g, len(shapes))).tolist()
    s = dict(case=case, g=[(1e-3 * a * _normal(g, *x)).to(t) for a, x in zip(size, shapes)], copy=None)
    parts = {"p": [0.02 * _normal(g, n) for n in counts], "m": [3e-4 * a * _normal(g, n) for a, n in zip(size, counts)],
             "v": [1e-3 * a * (0.5 + torch.rand((n,), generator=g, device="cuda")) for a, n in zip(size, counts)]}
    if case["bits"] == 32:
        parts["v"] = [x * x for x in parts["v"]]
    if t != torch.float32:
        parts["copy"] = [x.to(t) for x in parts["p"]]
    for name, x in parts.items():
        # one array for all tensors, each from a whole block on
        whole = torch.cat([torch.nn.functional.pad(y, (0, -y.numel() % BLOCK)) for y in x])
        if name in "mv" and case["bits"] == 8:
            s[name + "_all"] = _to_bytes(whole, 0.5)
            codes, exps = (_parts(y, counts, by) for y, by in zip(s[name + "_all"], (1, BLOCK)))
            s[name] = list(zip(codes, exps))
        else:
            s[name + "_all"] = whole
            s[name] = [y.view(z) for y, z in zip(_parts(whole, counts, 1), shapes)]
    return s


def _parts(x, counts, by):
    """Each tensor's part of an array for all, which has an entry for `by` elements."""
    parts = x.split([-(-n // BLOCK) * BLOCK // by for n in counts])
    return [y[:n] if by == 1 else y for y, n in zip(parts, counts)]


# ---- plain forms: delta --------------------------------------------------------------------------
def _live(s, T):
    """[T][B]: steps that are there."""
    return torch.arange(T, device=s["q"].device)[:, None] < (T if s["lengths"] is None else s["lengths"][None, :].long())


def _chunks(x, heads, live):
    """[T][B][h][...] in 32 bits as [chunks][B][heads][CHUNK][...], zeros where nothing is there."""
    T = x.shape[0]
    if live is not None:
        x = torch.where(live.view(*live.shape, *[1] * (x.dim() - 2)), x, 0)
    x = x.float().repeat_interleave(heads // x.shape[2], 2) if x.shape[2] != heads else x.float()
    x = torch.cat([x, x.new_zeros(-T % CHUNK, *x.shape[1:])]).unflatten(0, (-1, CHUNK))
    return x.movedim(1, 3).contiguous()


def _steps_of(x, T):
    """The other way."""
    return x.movedim(3, 1).flatten(0, 1)[:T]


def _delta_maps(s):
    """What a chunk's steps are to each other."""
    case = s["case"]
    T, H = case["T"], case["heads"]
    live = None if s["lengths"] is None else _live(s, T)
    m = {k: _chunks(s[k], H, live) for k in ("q", "k", "v", "g", "beta")}
    m["q"] = m["q"] * case["dk"] ** -0.5
    G = m["g"].double().cumsum(-1)
    low = torch.ones(CHUNK, CHUNK, dtype=torch.bool, device=G.device).tril()
    D = torch.exp(torch.where(low, G[..., :, None] - G[..., None, :], -math.inf)).float()
    m["D"], m["low"] = D, low.tril(-1)
    m["gam"], m["end"], m["tail"] = torch.exp(G).float()[..., None], torch.exp(G[..., -1:, None]).float(), torch.exp(G[..., -1:] - G).float()[..., None]
    m["kk"] = m["k"] @ m["k"].transpose(-1, -2) * D * m["low"]
    # the inverse of 1 + L as the product of 1 + (-L)^(2^i), in 64 bits
    power = -(m["beta"][..., None] * m["kk"]).double()
    inv = torch.eye(CHUNK, device=G.device, dtype=torch.float64) + power
    for _ in range(5):
        power = power @ power
        inv = inv + inv @ power
    m["A"] = inv.float() * m["beta"][..., None, :]
    m["P"] = m["q"] @ m["k"].transpose(-1, -2) * D
    return m


def _delta_walk(s, m, out):
    """The state before each chunk and the last one, u, o."""
    state, before, us, os = s["s0"] if "s0" in s else s["kept"][0], [], [], []
    for c in range(m["k"].shape[0]):
        before.append(state)
        u = m["A"][c] @ (m["v"][c] - m["gam"][c] * (m["k"][c] @ state))
        if out:
            os.append(m["gam"][c] * (m["q"][c] @ state) + m["P"][c] @ u)
        us.append(u)
        state = m["end"][c] * state + (m["tail"][c] * m["k"][c]).transpose(-1, -2) @ u
    return torch.stack(before), state, torch.stack(us), torch.stack(os) if out else None


def _delta_plain(s, out=True):
    T = s["case"]["T"]
    before, last, _, o = _delta_walk(s, _delta_maps(s), out)
    return _steps_of(o, T).to(s["v"].dtype) if out else None, last, before[::KEPT // CHUNK].contiguous()


def _delta_plain_back(s):
    case, m = s["case"], _delta_maps(s)
    T, H, K = case["T"], case["heads"], case["key_heads"]
    live = None if s["lengths"] is None else _live(s, T)
    before, _, u, _ = _delta_walk(dict(s, s0=s["kept"][0]), m, False)
    do, ds = _chunks(s["do"], H, live), s["ds_last"]
    after, du, de = [None] * len(u), [None] * len(u), [None] * len(u)
    for c in reversed(range(len(u))):
        after[c] = ds
        du[c] = m["P"][c].transpose(-1, -2) @ do[c] + m["tail"][c] * (m["k"][c] @ ds)
        de[c] = m["A"][c].transpose(-1, -2) @ du[c]
        ds = m["end"][c] * ds + (m["gam"][c] * m["q"][c]).transpose(-1, -2) @ do[c] - (m["gam"][c] * m["k"][c]).transpose(-1, -2) @ de[c]
    after, du, de = torch.stack(after), torch.stack(du), torch.stack(de)
    e = m["v"] - m["gam"] * (m["k"] @ before)
    raw = e - m["kk"] @ u  # u / beta
    across = de @ raw.transpose(-1, -2)
    dp = do @ u.transpose(-1, -2) * m["D"]
    dm = -across * m["beta"][..., None, :] * m["D"] * m["low"]
    back = before.transpose(-1, -2)
    to_q, to_k, of_u = m["gam"] * (do @ back), m["gam"] * (de @ back), m["tail"] * (u @ after.transpose(-1, -2))
    dq = to_q + dp @ m["k"]
    dk = of_u - to_k + dp.transpose(-1, -2) @ m["q"] + dm @ m["k"] + dm.transpose(-1, -2) @ m["k"]
    dbeta = (raw * du).sum(-1) - (m["kk"] * across).sum(-2)
    # a decay lies between all that was written before it and all that is read from it on
    z = (m["q"] @ m["k"].transpose(-1, -2) * dp + m["k"] @ m["k"].transpose(-1, -2) * dm).double()
    read, wrote = (m["q"] * to_q - m["k"] * to_k).double().sum(-1), (m["k"] * of_u).double().sum(-1)
    total = (m["end"] * before * after).double().sum((-1, -2))[..., None]
    on = read + z.sum(-1) - z.sum(-2)
    dg = total + on.flip(-1).cumsum(-1).flip(-1) + wrote.cumsum(-1) - wrote
    if live is not None:
        dg = torch.where(_chunks(live[..., None].expand(T, case["batch"], H), H, None) > 0, dg, 0)
    t = s["v"].dtype
    dq, dk = (_steps_of(x, T).unflatten(2, (K, H // K)).sum(3) for x in (dq * case["dk"] ** -0.5, dk))
    return dq.to(t), dk.to(t), _steps_of(de, T).to(t), _steps_of(dg, T).float(), _steps_of(dbeta, T).float(), ds


# ---- plain forms: norm and 8 bits ----------------------------------------------------------------
def _to_bytes(x, threshold):
    """Codes and exponent bytes: a block's step is the smallest power of two (from 2^-126) that its largest element is at most 127 times;
    an element's code is the multiple below it, or the next one where it is nearer to that than `threshold` says (0.5: to nearest, ties to even,
    and a step that 127.49 still fits)."""
    n = x.shape[-1]
    v = torch.nn.functional.pad(x, (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = v.abs().amax(-1)
    f, e = torch.frexp(top)
    nearest = isinstance(threshold, float)
    over = torch.round(f * 128) > 127 if nearest else f * 128 > 127
    k = torch.where(over, e - 6, e - 7).clamp(min=-126)
    exps = torch.where(top == 0, 0, k + 127).to(torch.uint8)
    x_ = v / torch.where(top == 0, 1.0, _steps(exps))[..., None]
    codes = torch.round(x_) if nearest else torch.floor(x_ + torch.nn.functional.pad(threshold, (0, -n % BLOCK)).view(x_.shape))
    return codes.to(torch.int8).flatten(-2)[..., :n].contiguous(), exps


def _steps(exps):
    return (exps.to(torch.int32) << 23).view(torch.float32)


def _values(codes, exps, dtype=torch.bfloat16):
    """(codes have 7 bits: exact in bfloat16)"""
    return (codes.float() * _steps(exps).repeat_interleave(BLOCK, -1)[..., :codes.shape[-1]]).to(dtype)


def _norm_plain(s):
    t = s["x"].dtype
    x = s["x"].float()
    call = s["case"]["call"]
    if call != "backward" and s["r"] is not None:
        x = x + s["r"].float()
    inv = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    if call == "backward":
        dy, hat = s["dy"].float(), x * inv
        mine = dy * s["w"].float()
        dx = inv * (mine - hat * (mine * hat).mean(-1, keepdim=True))
        if s["r"] is not None:
            dx = dx + s["r"].float()
        return dx.to(t), (dy * hat).sum(0).to(t)
    y = x * inv * s["w"].float()
    y = _values(*_to_bytes(y, 0.5)) if call == "packed" else y.to(t)
    return (y, x.to(t)) if s["r"] is not None else (y,)


# ---- plain forms: adamw --------------------------------------------------------------------------
def _threshold(n, a, b, device):
    i = torch.arange(n, device=device)
    return (((i * a + STEP * b) & 0xFFFFFFFF) >> 16).float() * 2.0 ** -16


def _adamw_plain(s):
    eight = s["case"]["bits"] == 8
    c1, c2 = 1 / (1 - BETA1 ** STEP), 1 / math.sqrt(1 - BETA2 ** STEP)
    for i, p in enumerate(s["p"]):
        g = s["g"][i].float()
        m, v = s["m"][i], s["v"][i]
        if eight:
            m, v = _values(*m, torch.float32).view(p.shape), _values(*v, torch.float32).view(p.shape) ** 2
        m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g * g
        p.copy_(p * (1 - LR * DECAY) - LR * (m * c1) / (v.sqrt() * c2 + ADAM_EPS))
        if s["copy"]:
            s["copy"][i].copy_(p)
        if eight:
            root = v.sqrt().flatten()
            codes, exps = _to_bytes(m.flatten(), _threshold(p.numel(), *LATTICE, p.device))
            s["m"][i][0].copy_(codes)
            s["m"][i][1].copy_(exps)
            codes, exps = _to_bytes(root, _threshold(p.numel(), *LATTICE[::-1], p.device))
            s["v"][i][0].copy_(torch.where(root > 0, codes.clamp(min=1), codes))  # what is not nothing stays so
            s["v"][i][1].copy_(exps)
        else:
            s["m"][i].copy_(m)
            s["v"][i].copy_(v)
    moments = [_values(*s[k + "_all"]) for k in "mv"] if eight else [s["m_all"], s["v_all"]]
    return s["p_all"], s.get("copy_all"), *moments


def _run_plain(s):
    case = s["case"]
    if case["op"] == "delta":
        return _delta_plain(s) if case["call"] == "forward" else _delta_plain_back(s)
    return _norm_plain(s) if case["op"] == "norm" else _adamw_plain(s)


# ---- the library's calls -------------------------------------------------------------------------
def _run_own(s):
    import paper_2412_11810_amd as snn

    case = s["case"]
    if case["op"] == "delta":
        inputs = [s[k] for k in ("q", "k", "v", "g", "beta")]
        if case["call"] == "forward":
            return snn.snn_delta_forward(*inputs, s["s0"], lengths=s["lengths"], keep=True)
        return snn.snn_delta_backward(*inputs, s["kept"], s["do"], s["ds_last"], lengths=s["lengths"])
    if case["op"] == "norm":
        if case["call"] == "backward":
            return snn.snn_norm_backward(s["x"], s["w"], s["dy"], dtotal=s["r"], eps=EPS)
        y, total = snn.snn_norm_forward(s["x"], s["w"], residual=s["r"], eps=EPS, packed=case["call"] == "packed")
        if case["call"] == "packed":
            y = snn.snn_unpack(y, torch.bfloat16)
        return (y, total) if s["r"] is not None else (y,)
    if "plan" not in s:  # kept by a program as long as its weights
        m, v = ([snn.Packed(*x) for x in s[k]] if case["bits"] == 8 else s[k] for k in "mv")
        s["plan"] = snn.snn_adamw_plan(s["p"], m, v, copies=s["copy"])
    snn.snn_adamw_step(s["plan"], s["g"], STEP, lr=LR, betas=(BETA1, BETA2), eps=ADAM_EPS, weight_decay=DECAY)
    moments = [snn.snn_unpack(snn.Packed(*s[k + "_all"]), torch.bfloat16) for k in "mv"] if case["bits"] == 8 else [s["m_all"], s["v_all"]]
    return s["p_all"], s.get("copy_all"), *moments


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    s = SIZE[case["dtype"]]
    if case["op"] == "delta":
        T, B, H, K, dk, dv = (case[k] for k in ("T", "batch", "heads", "key_heads", "dk", "dv"))
        steps, state = T * B, 4 * B * H * dk * dv
        x = s * (2 * K * dk + 2 * H * dv) + 8 * H  # q, k, v, o, g, beta
        # a step by itself: three products of a vector and the state; in chunks those and, among CHUNK steps, four, half of them needed
        among = min(T, CHUNK)
        flops = H * (6 * dk * dv + 2 * among * (dk + dv))
        if case["call"] == "forward":
            return {"bytes": steps * x + state * (2 + -(-T // KEPT)), "flops": steps * flops}
        return {"bytes": steps * (2 * x - s * H * dv) + state * (2 + -(-T // KEPT)), "flops": steps * (H * 4 * dk * dv + 2.5 * flops)}
    if case["op"] == "norm":
        rows, n = case["rows"], case["n"]
        x = rows * n
        if case["call"] == "backward":
            return {"bytes": s * (x * (4 if case["residual"] else 3) + 2 * n), "flops": 10 * x}
        y = s * x if case["call"] == "forward" else 2 * (x + rows * -(-n // BLOCK)) + 2 * x  # packed: written, and read for its values
        return {"bytes": s * x * (3 if case["residual"] else 1) + y + s * n, "flops": 5 * x}
    n = sum(math.prod(x) for x in _shapes(case))
    moments = 16 * n if case["bits"] == 32 else 2 * (3 * (n + -(-n // BLOCK)) + 2 * n)  # in 8 bits: read, written, and read for their values
    return {"bytes": moments + 8 * n + (4 if case["dtype"] == "float32" else 2 + 2) * n, "flops": 15 * n}


# ---- the definitions in 64 bits, step by step ----------------------------------------------------
def _exact_delta(s):
    case = s["case"]
    T, H, K, scale = case["T"], case["heads"], case["key_heads"], case["dk"] ** -0.5
    own_head = torch.arange(H, device="cuda") // (H // K)
    live = _live(s, T).double().expand(T, case["batch"])
    on = live[..., None, None]
    q, k = (torch.where(on > 0, s[n].double(), 0.0)[:, :, own_head] for n in ("q", "k"))
    v = torch.where(on > 0, s["v"].double(), 0.0)
    a, beta = torch.exp(torch.where(on[..., 0] > 0, s["g"].double(), 0.0))[..., None, None], torch.where(on[..., 0] > 0, s["beta"].double(), 0.0)[..., None]

    def forth(t, S):
        held = a[t] * S
        e = v[t] - (held * k[t][..., None]).sum(-2)
        return held, e, torch.addcmul(held, k[t][..., None], (beta[t] * e)[..., None, :])

    S = (s["s0"] if case["call"] == "forward" else s["kept"][0]).double()
    o, kept = torch.empty_like(v), []
    every = KEPT if case["call"] == "forward" else CHUNK
    for t in range(T):
        if t % every == 0:
            kept.append(S)
        S = forth(t, S)[2]
        if case["call"] == "forward":
            o[t] = scale * (S * q[t][..., None]).sum(-2)
    if case["call"] == "forward":
        return o, S, torch.stack(kept)
    do, dS = torch.where(on > 0, s["do"].double(), 0.0), s["ds_last"].double()
    dq, dk, dv, dg, db = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(a[..., 0, 0]), torch.zeros_like(beta[..., 0])
    for first in reversed(range(0, T, every)):
        states = [kept[first // every]]
        for t in range(first, min(first + every, T)):
            states.append(forth(t, states[-1])[2])
        for t in reversed(range(first, min(first + every, T))):
            held, e, S = forth(t, states[t - first])
            dq[t] = scale * (S * do[t][..., None, :]).sum(-1)
            dS = torch.addcmul(dS, q[t][..., None], scale * do[t][..., None, :])
            du = (dS * k[t][..., None]).sum(-2)
            db[t], de = (du * e).sum(-1), beta[t] * du
            dv[t] = de
            dk[t] = (dS * (beta[t] * e)[..., None, :]).sum(-1) - (held * de[..., None, :]).sum(-1)
            dS = torch.addcmul(dS, k[t][..., None], de[..., None, :], value=-1)
            dg[t] = (dS * held).sum((-1, -2))
            dS = a[t] * dS
    shared = lambda x: (x * on).unflatten(2, (K, H // K)).sum(3)  # noqa: E731
    return shared(dq), shared(dk), dv * on, dg * live[..., None], db * live[..., None], dS


def _exact_bytes(x, lattice=None):
    """Values of elements in 8 bits, and the codes' least step."""
    n = x.shape[-1]
    v = torch.nn.functional.pad(x, (0, -n % BLOCK)).unflatten(-1, (-1, BLOCK))
    top = v.abs().amax(-1, keepdim=True).clamp(min=2.0 ** -149)
    if lattice is None:
        step = torch.exp2((torch.floor(torch.log2(top / 127.5)) + 1).clamp(min=-126))
        return (torch.round(v / step) * step).flatten(-2)[..., :n]
    step = torch.exp2(torch.ceil(torch.log2(top / 127)).clamp(min=-126))
    i = torch.arange(v.numel(), device=x.device).view(v.shape)
    u = ((i * lattice[0] + STEP * lattice[1]) % 2 ** 32 // 2 ** 16).double() / 2 ** 16
    return (torch.floor(v / step + u) * step).flatten(-2)[..., :n], step.expand_as(v).flatten(-2)[..., :n]


def _exact_norm(s):
    x, w, r = s["x"].double(), s["w"].double(), s["r"]
    call = s["case"]["call"]
    if r is not None and call != "backward":
        x = x + r.double()
    size = torch.sqrt(torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / x.shape[-1] + EPS)
    if call != "backward":
        y = x / size * w
        y = _exact_bytes(y) if call == "packed" else y
        return (y, x) if r is not None else (y,)
    dy = s["dy"].double()
    dx = dy * w / size - x * torch.linalg.vecdot(dy * w, x)[:, None] / (x.shape[-1] * size ** 3)
    return dx if r is None else dx + r.double(), torch.mv((dy * x).t(), 1 / size[:, 0])


def _exact_adamw(s):
    eight = s["case"]["bits"] == 8
    after = []
    for i, p in enumerate(s["p"]):
        g = s["g"][i].double().flatten()
        m, v = s["m"][i], s["v"][i]
        if eight:
            m, v = (codes.double() * torch.exp2(exps.double() - 127).repeat_interleave(BLOCK)[:len(g)] for codes, exps in (m, v))
            v = v * v
        m, v = (x.double().flatten() for x in (m, v))
        m, v = m + (g - m) * (1 - BETA1), v + (g * g - v) * (1 - BETA2)
        move = m / (1 - BETA1 ** STEP) / (torch.sqrt(v / (1 - BETA2 ** STEP)) + ADAM_EPS)
        p = p.double().flatten() * (1 - LR * DECAY) - LR * move
        if eight:
            root = torch.sqrt(v)
            (m, _), (v, least) = _exact_bytes(m, LATTICE), _exact_bytes(root, LATTICE[::-1])
            v = torch.where(root > 0, torch.maximum(v, least), v)
        after.append([torch.nn.functional.pad(x, (0, -len(x) % BLOCK)) for x in (p, m, v)])
    p, m, v = (torch.cat(x) for x in zip(*after))
    return p, p if s["copy"] else None, m, v


def exact(case, seed):
    s = prepare(case, seed)
    return {"delta": _exact_delta, "norm": _exact_norm, "adamw": _exact_adamw}[case["op"]](s)
