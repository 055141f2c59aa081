"""Operators of token sequence models (snn_glr_*, snn_pack / snn_unpack, snn_vocab_*) against plain implementations in 64 bits on the
CPU, through the Python binding.  Refusals that need no GPU run everywhere.

Tolerances count roundings.  E32 = 2^-23 covers the two or three roundings and the last-place errors of the hardware's exponential
and reciprocal that a step makes; results in bf16 are off by half a step, 2^-8 of the value, on top."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2412_11810_amd as snn
from paper_2412_11810_amd import ops

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
E32 = 2.0 ** -23
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


# ---- plain implementations ------------------------------------------------------------------------
def glr_forward(z, x, h0, lengths):
    T, B, n = z.shape
    h, state, kept = torch.zeros(T, B, n, dtype=torch.float64), h0.clone(), []
    for t in range(T):
        if t % 128 == 0:
            kept.append(state.clone())
        on = (t < lengths)[:, None]
        a = 1 / (1 + torch.exp(-z[t]))
        new = a * state + x[t] / (1 + torch.exp(z[t]))
        state = torch.where(on, new, state)
        h[t] = torch.where(on, new, 0.0)
    return h, state, torch.stack(kept) if kept else torch.zeros(0, B, n, dtype=torch.float64)


def glr_backward(z, x, h0, lengths, dh, dh_last):
    T, B, n = z.shape
    before, state = torch.zeros(T, B, n, dtype=torch.float64), h0.clone()
    a, c = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
    for t in range(T):
        before[t] = state
        state = torch.where((t < lengths)[:, None], a[t] * state + c[t] * x[t], state)
    dz, dx, g, most = torch.zeros_like(z), torch.zeros_like(z), dh_last.clone(), dh_last.abs().max().item()
    for t in reversed(range(T)):
        on = (t < lengths)[:, None]
        g = torch.where(on, g + dh[t], g)
        most = max(most, g.abs().max().item())
        dx[t] = torch.where(on, c[t] * g, 0.0)
        dz[t] = torch.where(on, a[t] * c[t] * (before[t] - x[t]) * g, 0.0)
        g = torch.where(on, a[t] * g, g)
    return dz, dx, g, most


def to_bytes(x):
    """Codes and exponents of rows of numpy floats, block by block."""
    rows, n = x.shape
    codes, exps = np.zeros((rows, n), np.int8), np.zeros((rows, -(-n // 32)), np.uint8)
    for r in range(rows):
        for b in range(exps.shape[1]):
            v = x[r, 32 * b:32 * b + 32].astype(np.float64)
            if not np.all(np.isfinite(v)):
                exps[r, b] = 255
            elif np.any(v):
                k = -126
                while k < 121 and np.abs(np.round(np.ldexp(v, -k))).max() > 127:
                    k += 1
                codes[r, 32 * b:32 * b + 32], exps[r, b] = np.clip(np.round(np.ldexp(v, -k)), -127, 127), k + 127
    return codes, exps


def from_bytes(codes, exps):
    step = np.where(exps == 255, np.nan, np.where(exps == 0, 0.0, np.ldexp(1.0, exps.astype(int) - 127)))
    return codes.astype(np.float64) * np.repeat(step, 32, -1)[..., :codes.shape[-1]]


def vocab_loss(h, w, target):
    rows = len(target)
    logits = h @ w.T
    on = (target >= 0) & (target < w.shape[0])
    y = torch.where(on, target, 0)
    lse = torch.logsumexp(logits, 1)
    others = logits.clone()
    others[torch.arange(rows), y] = -math.inf
    miss = torch.exp(torch.logsumexp(others, 1) - lse)  # 1 - softmax of the target, as a sum
    loss = torch.where(on, torch.where(miss < 0.5, -torch.log1p(-miss), lse - logits[torch.arange(rows), y]), 0.0)
    return logits, lse, miss, on, y, loss


def vocab_grads(h, w, target, dloss):
    logits, lse, miss, on, y, _ = vocab_loss(h, w, target)
    G = torch.exp(logits - lse[:, None])
    G[torch.arange(len(y)), y] = -miss
    G = torch.where(on[:, None], G * dloss[:, None], 0.0)
    return G, G @ w, G.T @ h


def near(got, want, tol, what):
    """|got - want| <= tol + half a step of got's type, everywhere."""
    got_, want = got.double().cpu(), want.double()
    assert got_.shape == want.shape, what
    off = (got_ - want).abs() - (tol + HALF[got.dtype] * want.abs())
    assert not torch.isnan(off).any() and off.max().item() <= 0 if off.numel() else True, (what, off.max().item())


# ---- gated linear recurrence ------------------------------------------------------------------------
def glr_inputs(T, B, n, dtype, ragged, seed=1, halves=False):
    g = torch.Generator().manual_seed(seed)
    z = (2 + 1.5 * torch.randn(T, B, n, generator=g)).clamp(-6, 6).to(dtype)
    x, dh = torch.randn(T, B, n, generator=g).to(dtype), torch.randn(T, B, n, generator=g).to(dtype)
    h0, dlast = torch.randn(B, n, generator=g), torch.randn(B, n, generator=g)
    lengths = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32) if ragged else torch.full((B,), T, dtype=torch.int32)
    if ragged:
        lengths[0] = T
        lengths[-1] = 0
        pad = torch.arange(T)[:, None] >= lengths[None, :]
        for a in (z, x, dh):
            a[pad] = math.nan  # nothing may read these
    if halves:
        zx = torch.cat([z, x], -1).cuda()
        return zx[..., :n], zx[..., n:], dh.cuda(), h0.cuda(), dlast.cuda(), lengths.cuda()
    return z.cuda(), x.cuda(), dh.cuda(), h0.cuda(), dlast.cuda(), lengths.cuda()


def bounds(z, x, h0, lengths):
    """Largest |z|, least b = sigmoid(-z), largest |x| or |h0| of what is read."""
    live = torch.arange(z.shape[0])[:, None] < lengths[None, :]
    z, x = z[live], x[live]
    if not z.numel():
        return 0.0, 0.5, max(h0.abs().max().item(), 1e-30)
    return z.abs().max().item(), 1 / (1 + math.exp(z.max().item())), max(x.abs().max().item(), h0.abs().max().item())


GLR = [(0, 2, 5, False), (1, 1, 1, False), (1, 64, 130, False), (2, 3, 7, True), (15, 2, 64, False), (16, 3, 66, True), (17, 2, 33, True),
       (127, 1, 10, False), (128, 2, 128, True), (129, 5, 31, True), (300, 3, 75, True), (1000, 1, 2, False), (300, 33, 1024, False),
       (700, 1, 12800, False), (260, 64, 1024, True)]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,B,n,ragged", GLR)
def test_glr_forward(T, B, n, ragged, dtype):
    z, x, _, h0, _, lengths = glr_inputs(T, B, n, dtype, ragged, halves=n % 2 == 1)
    h, last, kept = snn.snn_glr_forward(z, x, h0, lengths=lengths if ragged else None, keep=True)
    zc, xc, hc, lc = z.double().cpu(), x.double().cpu(), h0.double().cpu(), lengths.cpu()
    want = glr_forward(zc, xc, hc, lc)
    zmax, bmin, M = bounds(zc, xc, hc, lc)
    # e_t <= (1 - b) e_{t-1} + 2 M E32 (b (|z| + 4) + 1), and the joins of 16-step maps as much again
    tol = 4 * M * E32 * (zmax + 4 + 1 / bmin)
    for got, ref, what in zip((h, last, kept), want, ("h", "last", "kept")):
        near(got, ref, tol, what)
    if T:
        near(snn.snn_glr_forward(z, x, None, lengths=lengths if ragged else None)[0], glr_forward(zc, xc, 0 * hc, lc)[0], tol, "from zero")


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,B,n,ragged", GLR)
@pytest.mark.parametrize("packed", [False, True])
def test_glr_backward(T, B, n, ragged, dtype, packed):
    z, x, dh, h0, dlast, lengths = glr_inputs(T, B, n, dtype, ragged, seed=2, halves=n % 2 == 1)
    zc, xc = z.double().cpu(), x.double().cpu()
    zi, xi = z, x
    if packed:
        zi, xi = snn.snn_pack(z), snn.snn_pack(x)
        zc = torch.from_numpy(from_bytes(zi.codes.cpu().numpy(), zi.exps.cpu().numpy()))
        xc = torch.from_numpy(from_bytes(xi.codes.cpu().numpy(), xi.exps.cpu().numpy()))
    hc, dc, lc = h0.double().cpu(), dlast.double().cpu(), lengths.cpu()
    kept = glr_forward(zc, xc, hc, lc)[2].float().cuda()
    dhc = dh.double().cpu()
    wide = torch.full((T, B, 2 * n), 7.0, dtype=dtype, device="cuda")
    dz, dx, dh0 = snn.snn_glr_backward(zi, xi, kept, dh, dlast, lengths=lengths if ragged else None, dz=wide[..., :n], dx=wide[..., n:])
    want = glr_backward(zc, xc, hc, lc, dhc, dc)
    zmax, bmin, M = bounds(zc, xc, hc, lc)
    G = max(want[3], 1e-30)
    e_h, e_g = 4 * M * E32 * (zmax + 4 + 1 / bmin), 4 * G * E32 * (zmax + 4 + 1 / bmin)
    near(dx, want[1], e_g + G * (zmax + 4) * E32, "dx")
    near(dz, want[0], 0.25 * (2 * M * e_g + G * e_h) + 2 * M * G * (zmax + 6) * E32, "dz")
    near(dh0, want[2], e_g, "dh0")
    none = snn.snn_glr_backward(zi, xi, kept, dh, None, lengths=lengths if ragged else None)
    zero = glr_backward(zc, xc, hc, lc, dhc, 0 * dc)
    near(none[1], zero[1], e_g + G * (zmax + 4) * E32, "dx without dh_last")
    near(none[2], zero[2], e_g, "dh0 without dh_last")


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,B,n", [(1, 64, 130), (20, 40, 65), (33, 7, 97), (18, 9, 63), (40, 11, 64), (16, 300, 3), (40, 160, 130), (40, 170, 128),
                                   (20, 200, 160)])
def test_glr_backward_from_bytes_is_that_of_their_values(T, B, n, dtype):
    # rows that end anywhere in a wavefront's channels; steps are powers of two: the same products, hence the same bits
    z, x, dh, h0, dlast, _ = glr_inputs(T, B, n, dtype, False, seed=9)
    z *= torch.exp(torch.randn(B, n, device="cuda")).to(dtype)
    pz, px = snn.snn_pack(z), snn.snn_pack(x)
    z, x = snn.snn_unpack(pz, dtype), snn.snn_unpack(px, dtype)
    kept = snn.snn_glr_forward(z, x, h0, keep=True)[2]
    assert same(snn.snn_glr_backward(pz, px, kept, dh, dlast), snn.snn_glr_backward(z, x, kept, dh, dlast))


@gpu
def test_glr_state_in_place_is_a_sequence_cut_anywhere():
    z, x, dh, h0, _, _ = glr_inputs(300, 3, 50, torch.float32, False)
    whole, last, _ = snn.snn_glr_forward(z, x, h0)
    state = h0.clone()
    parts = [snn.snn_glr_forward(z[a:b], x[a:b], state, h_last=state)[0] for a, b in ((0, 1), (1, 2), (2, 150), (150, 300))]
    tol = 4 * 5 * E32 * (10 + 500)  # |x|, |h0| < 5, |z| <= 6: as above
    near(torch.cat(parts), whole.cpu(), tol, "h")
    near(state, last.cpu(), tol, "state")


@gpu
def test_glr_lengths_outside_count_as_the_nearer_end():
    z, x, dh, h0, _, _ = glr_inputs(200, 4, 70, torch.float32, False)
    lengths = torch.tensor([-5, 207, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
    inside = torch.tensor([0, 200, 200, 0], dtype=torch.int32, device="cuda")
    got, want = (snn.snn_glr_forward(z, x, h0, lengths=v, keep=True) for v in (lengths, inside))
    assert same(got, want) and same(*(snn.snn_glr_backward(z, x, want[2], dh, lengths=v) for v in (lengths, inside)))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,B,n", [(40, 3, 66), (700, 2, 70)])
def test_glr_rows_of_wider_arrays(T, B, n, dtype):
    z, x, dh, h0, dlast, _ = glr_inputs(T, B, n, dtype, False, seed=4)
    wide = torch.full((T, B, 5 * n + 2), math.nan, dtype=dtype, device="cuda")
    parts = [wide[..., i * n:(i + 1) * n] for i in range(5)]
    for to, v in zip(parts, (z, x, dh)):
        to.copy_(v)
    h, last, kept = snn.snn_glr_forward(z, x, h0, keep=True)
    assert same(snn.snn_glr_forward(parts[0], parts[1], h0, keep=True, h=parts[3]), [h, last, kept])
    want = snn.snn_glr_backward(z, x, kept, dh, dlast)
    assert same(snn.snn_glr_backward(parts[0], parts[1], kept, parts[2], dlast, dz=parts[3], dx=parts[4]), want)
    assert torch.isnan(wide[..., 5 * n:]).all()


@gpu
@pytest.mark.parametrize("T", [20, 1000])
def test_glr_gradient_of_the_state_in_place(T):
    z, x, dh, h0, dlast, _ = glr_inputs(T, 3, 50, torch.float32, False, seed=6)
    kept = snn.snn_glr_forward(z, x, h0, keep=True)[2]
    want = snn.snn_glr_backward(z, x, kept, dh, dlast)
    dz, dx, state = torch.empty_like(z), torch.empty_like(z), dlast.clone()
    p = ops.snn_glr(T, 3, 50, 0, 0, 0, 0, 0, 0, None)
    work = snn.lib().snn_glr_workspace(C.byref(p))
    space = torch.empty(max(work, 1), dtype=torch.uint8, device="cuda")
    at = ops.snn_launch(0, torch.cuda.current_stream().cuda_stream, space.data_ptr(), work)
    ops._run("snn_glr_backward", C.byref(at), C.byref(p), *(a.data_ptr() for a in (z, x, kept, dh, state, dz, dx, state)))
    assert same([dz, dx, state], want)


@gpu
def test_glr_many_segments():
    z, x, dh, h0, dlast, lengths = glr_inputs(20000, 1, 3, torch.float32, False, seed=8)
    zc, xc, hc, lc = z.double().cpu(), x.double().cpu(), h0.double().cpu(), lengths.cpu()
    h, last, kept = snn.snn_glr_forward(z, x, h0, keep=True)
    want, back = glr_forward(zc, xc, hc, lc), glr_backward(zc, xc, hc, lc, dh.double().cpu(), dlast.double().cpu())
    zmax, bmin, M = bounds(zc, xc, hc, lc)
    tol = 4 * M * E32 * (zmax + 4 + 1 / bmin)
    for got, ref, what in zip((h, last, kept), want, ("h", "last", "kept")):
        near(got, ref, tol, what)
    dx, dh0 = snn.snn_glr_backward(z, x, kept, dh, dlast)[1:]
    e_g = 4 * back[3] * E32 * (zmax + 4 + 1 / bmin)
    near(dx, back[1], e_g + back[3] * (zmax + 4) * E32, "dx")
    near(dh0, back[2], e_g, "dh0")


@gpu
def test_glr_long_memory_keeps_its_drive():
    # gates so near one that 1 - a in 32 bits would be off by 30 %: the state still tends to its drive, 1
    T = 4096
    z, x = torch.full((T, 1, 64), 15.0, device="cuda"), torch.ones((T, 1, 64), device="cuda")
    h = snn.snn_glr_forward(z, x)[0]
    b = 1 / (1 + math.exp(15.0))
    want = 1 - (1 - b) ** T
    # b is off by (15 + 4) E32 of itself, a step's rounding by 2^-24 of h <= want
    assert abs(h[-1].double().cpu() - want).max().item() <= want * (20 * E32 + T * 2.0 ** -24)


@gpu
def test_glr_saturated_gates_and_values_that_are_not_finite():
    inf, nan = math.inf, math.nan
    z = torch.tensor([200.0, -200.0, inf, -inf, nan, 0.0, 0.0], device="cuda").repeat(20, 1, 1)
    x = torch.tensor([1.0, 3.0, 1.0, 3.0, 1.0, nan, inf], device="cuda").repeat(20, 1, 1)
    h0 = torch.full((1, 7), 2.0, device="cuda")
    h, last, kept = snn.snn_glr_forward(z, x, h0, keep=True)
    assert h[:, 0, :4].cpu().tolist() == [[2.0, 3.0, 2.0, 3.0]] * 20 and torch.isnan(h[1:, 0, 4:]).all()
    dz, dx, dh0 = snn.snn_glr_backward(z, x, kept, torch.ones_like(z))
    assert torch.isfinite(dz[:, 0, :4]).all() and torch.isfinite(dx[:, 0, :4]).all()
    assert dh0[0, :4].cpu().tolist() == [20.0, 0.0, 20.0, 0.0]


# ---- 8 bits -------------------------------------------------------------------------------------
@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n", [(1, 1), (3, 7), (2, 8), (5, 31), (4, 32), (3, 33), (9, 75), (300, 264), (2, 5001)])
def test_pack_and_unpack(rows, n, dtype):
    g = torch.Generator().manual_seed(n)
    x = (torch.randn(rows, n, generator=g) * torch.exp(3 * torch.randn(rows, 1, generator=g))).to(dtype)
    wide = torch.full((rows, n + 3), math.nan, dtype=dtype)
    wide[:, 1:n + 1] = x
    codes, exps = to_bytes(x.float().numpy())
    for given in (x.cuda(), wide.cuda()[:, 1:n + 1]):
        p = snn.snn_pack(given)
        assert np.array_equal(p.codes.cpu().numpy(), codes) and np.array_equal(p.exps.cpu().numpy(), exps)
    for out in (torch.float32, torch.bfloat16):  # a code has 7 bits: exact in both
        assert np.array_equal(snn.snn_unpack(p, out).double().cpu().numpy(), from_bytes(codes, exps))


@gpu
def test_pack_borders():
    top = torch.finfo(torch.float32).max
    rows = [[0.0] * 40, [127.0, 1.0] * 20, [127.49, -127.4, 0.5, 1.5, 2.5] * 8, [127.5] * 40, [255.0, 1.0] * 20, [top, -top, 1.0, 0.0] * 10,
            [1e-45, -3e-39] * 20, [2.0 ** -126 * 127] * 40, [2.0 ** -126 * 128, 0.0] * 20, [-0.0] * 40, [math.inf] + [1.0] * 39,
            [1.0] * 35 + [math.nan] * 5]
    x = torch.tensor(rows, dtype=torch.float32)
    codes, exps = to_bytes(x.numpy())
    p = snn.snn_pack(x.cuda())
    assert np.array_equal(p.codes.cpu().numpy(), codes) and np.array_equal(p.exps.cpu().numpy(), exps)
    back = snn.snn_unpack(p).double().cpu().numpy()
    assert np.array_equal(back, from_bytes(codes, exps), equal_nan=True)
    assert np.isnan(back[10, :32]).all() and np.isfinite(back[10, 32:]).all() and np.isnan(back[11, 32:]).all()
    step = np.repeat(np.ldexp(1.0, exps[:10].astype(int) - 127), 32, -1)[:, :40]
    # the largest float, 2^128 less 2^104, would be 128 of the largest step, 2^121, whose product is no float: 127 of them are less than one step off
    limit = np.where(np.arange(10) == 5, 1.0, 0.5)[:, None]
    assert (np.abs(back[:10] - x[:10].double().numpy()) <= limit * step).all()


# ---- cross entropy over a vocabulary --------------------------------------------------------------
def vocab_inputs(rows, d, vocab, dtype, seed=3, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    h, w = torch.randn(rows, d, generator=g).to(dtype), (spread / math.sqrt(d) * torch.randn(vocab, d, generator=g)).to(dtype)
    t = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int32)
    t[torch.rand(rows, generator=g) < 0.1] = -1
    return h, w, t, torch.rand(rows, generator=g) + 0.1


def check_vocab(h, w, t, dloss, given_h=None, given_w=None):
    """Losses and gradients against 64 bits.  A logit is a sum of d (fp32: 6 d) products in some order: off by at most that many roundings of
    the sum of their magnitudes."""
    rows, d = h.shape
    dtype, vocab = h.dtype, w.shape[0]
    gh, gw, gt = (h.cuda() if given_h is None else given_h), (w.cuda() if given_w is None else given_w), t.cuda()
    loss, state = snn.snn_vocab_loss(gh, gw, gt)
    H, W, t64 = h.double(), w.double(), t.long()
    logits, lse, miss, on, y, want = vocab_loss(H, W, t64)
    terms = (1 if dtype == torch.bfloat16 else 6) * d + 8
    e_l = terms * E32 * (H.abs() @ W.abs().T).amax(1) + 4 * E32 * logits.abs().amax(1)  # of each row's logits
    # a loss moves by no more than its logits do; the sum of vocab exponentials adds vocab roundings of one, at worst
    count = 64 + vocab / 64  # of the longest chain of additions: 64 in a lane, then one per block
    near(loss, want, (2 * e_l + count * E32) * torch.where(miss < 0.5, 2 * miss, 1.0) + 8 * E32 * want.abs() + 1e-30, "loss")
    assert (loss.cpu()[~on] == 0).all()
    for given in (None, dloss):
        scale = torch.where(on, 1.0 / max(1, int(on.sum())), 0.0).double() if given is None else given.double()
        dh, dw = snn.snn_vocab_loss_grad(gh, gw, gt, state, None if given is None else given.cuda())
        G, want_h, want_w = vocab_grads(H, W, t64, scale)
        rel = 4 * e_l + (count + 16) * E32 + (2.0 ** -8 if dtype == torch.bfloat16 else 0)  # of an element of G, to itself
        A = G.abs() * rel[:, None]
        sums = (1 if dtype == torch.bfloat16 else 6) * E32
        near(dh, want_h, A @ W.abs() + sums * (vocab + 8) * (G.abs() @ W.abs()) + 1e-30, "dh")
        near(dw, want_w, A.T @ H.abs() + sums * (rows + 8) * (G.abs().T @ H.abs()) + 1e-30, "dw")
    return loss, state


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,d,vocab", [(1, 1, 1), (1, 64, 2), (3, 5, 7), (2, 64, 1000), (33, 100, 129), (257, 128, 513), (300, 72, 1025),
                                          (64, 256, 128), (31, 1000, 300), (600, 320, 2500), (700, 40, 3), (5000, 33, 17)])
def test_vocab(rows, d, vocab, dtype):
    check_vocab(*vocab_inputs(rows, d, vocab, dtype))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_vocab_in_several_pieces(dtype):
    check_vocab(*vocab_inputs(66000, 24, 4500, dtype))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("d", [64, 70])
def test_vocab_rows_of_wider_arrays(d, dtype):
    h, w, t, dloss = vocab_inputs(100, d, 300, dtype)
    wide_h, wide_w = torch.full((100, d + 5), math.nan, dtype=dtype), torch.full((300, d + 8), math.nan, dtype=dtype)
    wide_h[:, 3:3 + d], wide_w[:, 8:] = h, w
    check_vocab(h, w, t, dloss, wide_h.cuda()[:, 3:3 + d], wide_w.cuda()[:, 8:])


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_vocab_gradients_of_the_losses_of_any_size(dtype):
    # rows' factors from 1e-12 to 1e6, of either sign, and none: relative to the largest of them nothing is lost
    h, w, t, _ = vocab_inputs(130, 96, 400, dtype)
    g = torch.Generator().manual_seed(1)
    dloss = 10 ** (torch.rand(130, generator=g) * 18 - 12) * torch.sign(torch.randn(130, generator=g))
    dloss[::7] = 0
    h[7] = math.nan  # a row whose loss has no gradient takes no part
    t[7] = 5
    gh, gw, gt = h.cuda(), w.cuda(), t.cuda()
    state = snn.snn_vocab_loss(gh, gw, gt)[1]
    dh, dw = snn.snn_vocab_loss_grad(gh, gw, gt, state, dloss.cuda())
    H = torch.where(dloss[:, None] == 0, 0.0, h.double())
    G, want_h, want_w = vocab_grads(H, w.double(), t.long(), dloss.double())
    # logits of 96 products (fp32: 6 each) of up to 12 in magnitude, then the roundings of G; sums of 400 and 130 terms
    rel = 4 * 600 * E32 * (H.abs() @ w.double().abs().T).amax() + (2.0 ** -8 if dtype == torch.bfloat16 else 0)
    near(dh, want_h, (rel + 6 * 408 * E32) * (G.abs() @ w.double().abs()) + 1e-36, "dh")
    near(dw, want_w, (rel + 6 * 138 * E32) * (G.abs().T @ H.abs()) + 1e-36, "dw")


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_vocab_nearly_certain_and_hopeless_targets(dtype):
    # the targets' logits stand out by up to 60 either way: losses from 1e-24 to 60
    h = torch.eye(64).to(dtype)
    w = torch.zeros(300, 64).to(dtype)
    t = torch.arange(64, dtype=torch.int32) * 4
    for r in range(64):
        w[4 * r, r] = 60.0 * (r - 31) / 32
    loss, _ = check_vocab(h, w, t, torch.rand(64) + 0.5)
    assert 0 < loss[63].item() < 1e-20 and loss[0].item() > 50


@gpu
def test_vocab_without_targets_and_targets_outside():
    h, w, t, dloss = vocab_inputs(40, 64, 100, torch.bfloat16)
    t[:] = -1
    t[::3], t[1::3] = 100, 2 ** 31 - 1
    loss, state = snn.snn_vocab_loss(h.cuda(), w.cuda(), t.cuda())
    dh, dw = snn.snn_vocab_loss_grad(h.cuda(), w.cuda(), t.cuda(), state)
    assert not loss.any() and not dh.any() and not dw.any()
    h[5] = math.nan  # a row that has no target takes no part, whatever it holds
    t[0] = 3
    loss, state = snn.snn_vocab_loss(h.cuda(), w.cuda(), t.cuda())
    dh, dw = snn.snn_vocab_loss_grad(h.cuda(), w.cuda(), t.cuda(), state)
    assert loss[0] > 0 and not loss[1:].any() and dh[0].any() and not dh[1:].any() and torch.isfinite(dw).all()


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_vocab_no_rows(dtype):
    h, w, t = torch.zeros(0, 8, dtype=dtype, device="cuda"), torch.ones(5, 8, dtype=dtype, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")
    loss, state = snn.snn_vocab_loss(h, w, t)
    dh, dw = snn.snn_vocab_loss_grad(h, w, t, state)
    assert loss.numel() == 0 and dh.shape == (0, 8) and dw.shape == (5, 8) and not dw.any()


@gpu
def test_vocab_values_that_are_not_finite_show():
    h, w, t, _ = vocab_inputs(300, 64, 700, torch.float32)
    t[:] = torch.arange(300, dtype=torch.int32)
    h[7] = math.inf
    h[9, 3] = math.nan
    loss, state = snn.snn_vocab_loss(h.cuda(), w.cuda(), t.cuda())
    dh, dw = snn.snn_vocab_loss_grad(h.cuda(), w.cuda(), t.cuda(), state)
    bad = torch.zeros(300, dtype=torch.bool)
    bad[[7, 9]] = True
    assert torch.equal(torch.isnan(loss).cpu(), bad) and torch.equal(torch.isnan(dh).all(1).cpu(), bad)
    assert torch.isfinite(dh.cpu()[~bad]).all() and torch.isnan(dw).any(1).all()


# ---- together ---------------------------------------------------------------------------------
def model_loss(p, tokens, targets, h0):
    """Losses of a one-layer model in 64 bits: an embedding, gate and drive by one projection, the recurrence, the vocabulary again."""
    zx = p["embed"][tokens] @ p["project"].T
    n = zx.shape[-1] // 2
    state, h = h0, []
    for t in range(zx.shape[0]):
        state = state + torch.sigmoid(-zx[t, :, :n]) * (zx[t, :, n:] - state)
        h.append(state)
    logits = torch.stack(h).flatten(0, 1) @ p["embed"].T
    return torch.nn.functional.cross_entropy(logits, targets.flatten(), ignore_index=-1)


@gpu
@pytest.mark.parametrize("packed", [False, True])
def test_a_training_step_of_a_model(packed):
    """Gradients of an embedding that is also the readout, and of the projection between, against autograd in 64 bits and against differences."""
    T, B, n, vocab = 150, 3, 48, 333
    g = torch.Generator().manual_seed(5)
    p64 = {"embed": torch.randn(vocab, n, generator=g, dtype=torch.float64) * 0.5,
           "project": torch.randn(2 * n, n, generator=g, dtype=torch.float64) * 0.3}
    p64 = {k: v.float().double().requires_grad_() for k, v in p64.items()}
    tokens, targets = torch.randint(0, vocab, (T, B), generator=g), torch.randint(-1, vocab, (T, B), generator=g)
    h0 = torch.randn(B, n, generator=g, dtype=torch.float64).float().double()
    want = model_loss(p64, tokens, targets, h0)
    want.backward()

    embed, project = (p64[k].detach().float().cuda() for k in ("embed", "project"))
    tk, tg = tokens.cuda(), targets.to(torch.int32).cuda().flatten()
    e = embed[tk]
    zx = (e.flatten(0, 1) @ project.T).view(T, B, 2 * n)
    h, _, kept = snn.snn_glr_forward(zx[..., :n], zx[..., n:], h0.float().cuda(), keep=True)
    saved = (snn.snn_pack(zx[..., :n]), snn.snn_pack(zx[..., n:])) if packed else (zx[..., :n], zx[..., n:])
    loss, state = snn.snn_vocab_loss(h.flatten(0, 1), embed, tg)
    dh, d_embed = snn.snn_vocab_loss_grad(h.flatten(0, 1), embed, tg, state)
    dzx = torch.empty_like(zx)
    snn.snn_glr_backward(*saved, kept, dh.view(T, B, n), dz=dzx[..., :n], dx=dzx[..., n:])
    flat = dzx.flatten(0, 1)
    d_project = flat.T @ e.flatten(0, 1)
    d_embed = d_embed.index_add(0, tk.flatten(), flat @ project)
    mean = loss.sum() / (tg >= 0).sum()
    assert abs(mean.item() - want.item()) < 1e-5 * want.item()
    # in 32 bits the sums of up to 450 terms are off by 1e-5 of the largest gradient at most; 8 bits move z and x by 2^-7 of
    # a block's largest, 4 here, hence a gradient by a few hundredths of the largest
    tol = 0.05 if packed else 1e-5
    for got, k in ((d_embed, "embed"), (d_project, "project")):
        ref = p64[k].grad
        assert (got.double().cpu() - ref).abs().max() <= tol * ref.abs().max(), k
        direction = torch.randn(ref.shape, generator=g, dtype=torch.float64)
        with torch.no_grad():
            ends = [model_loss({**p64, k: p64[k] + s * direction}, tokens, targets, h0) for s in (1e-5, -1e-5)]
        slope = ((ends[0] - ends[1]) / 2e-5).item()
        assert abs((got.double().cpu() * direction).sum().item() - slope) <= tol * (ref.abs().max() * direction.abs().sum()).item() + 1e-6


# ---- calls ------------------------------------------------------------------------------------
def every_operator(seed=7):
    """A function that runs every operator once, and its inputs."""
    z, x, dh, h0, dlast, lengths = glr_inputs(400, 3, 70, torch.bfloat16, True, seed=seed)
    live = torch.arange(400, device="cuda")[:, None] < lengths[None, :]
    z, x, dh = (torch.where(live[..., None], a, 0.0) for a in (z, x, dh))
    h, w, t, dloss = (a.cuda() for a in vocab_inputs(200, 96, 1500, torch.float32, seed=seed))

    def run():
        out, last, kept = snn.snn_glr_forward(z, x, h0, lengths=lengths, keep=True)
        pz, px = snn.snn_pack(z), snn.snn_pack(x)
        loss, state = snn.snn_vocab_loss(h, w, t)
        return [out, last, kept, *snn.snn_glr_backward(z, x, kept, dh, dlast, lengths=lengths),
                *snn.snn_glr_backward(pz, px, kept, dh, dlast, lengths=lengths), snn.snn_unpack(pz), loss, state,
                *snn.snn_vocab_loss_grad(h, w, t, state, dloss)]
    return run, [z, x, dh, h0, dlast, h, w, dloss]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b)) and len(a) == len(b)


@gpu
def test_calls_on_other_streams_give_the_same_bits():
    run, _ = every_operator()
    other, _ = every_operator(seed=8)
    want, want_other = run(), other()
    assert same(run(), want)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(3):  # both at once
        for s, f, to in zip(streams, (run, other), got):
            with torch.cuda.stream(s):
                to.append(f())
    torch.cuda.synchronize()
    assert all(same(a, want) for a in got[0]) and all(same(a, want_other) for a in got[1])


@gpu
def test_calls_in_a_graph():
    run, inputs = every_operator()
    want = run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for _ in range(3):
        for o in got:
            o.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, want)
        inputs[0].mul_(0.5)  # other values in the same arrays
        want = run()
        torch.cuda.synchronize()


@gpu
def test_calls_from_two_threads():
    import threading
    runs = [every_operator(seed)[0] for seed in (11, 12)]
    want = [f() for f in runs]
    torch.cuda.synchronize()
    wrong = []

    def work(f, ref):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(5):
                got = f()
                torch.cuda.current_stream().synchronize()
                if not same(got, ref):
                    wrong.append(1)
                try:  # a refusal of one thread's is not another's
                    snn.snn_glr_forward(torch.zeros(2, 1, 1 << 26, device="cuda"), torch.zeros(2, 1, 1 << 26, device="cuda"))
                except snn.SnnError as e:
                    if "channels" not in str(e):
                        wrong.append(str(e))

    threads = [threading.Thread(target=work, args=a) for a in zip(runs, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


# ---- offsets beyond 32 bits ---------------------------------------------------------------------
@gpu
def test_glr_arrays_beyond_4_gb():
    T, n, tail = 70016, 32768, 256  # 4.6 GB each in bf16
    g = torch.Generator(device="cuda").manual_seed(1)
    z = torch.empty((T, 1, n), dtype=torch.bfloat16, device="cuda").normal_(2.0, 1.0, generator=g)
    x, dh = (torch.empty_like(z).normal_(generator=g) for _ in range(2))
    h, last, kept = snn.snn_glr_forward(z, x, keep=True)
    dz, dx, _ = snn.snn_glr_backward(z, x, kept, dh)
    a = T - tail  # a multiple of 128: the last steps by themselves, from the state before them
    part, part_last, _ = snn.snn_glr_forward(z[a:], x[a:], kept[a // 128])
    part_dz, part_dx, _ = snn.snn_glr_backward(z[a:], x[a:], kept[a // 128:], dh[a:])
    # in other groups, hence joined differently: a rounding of bf16, or of the states before it
    for got, want in ((h[a:], part), (dz[a:], part_dz), (dx[a:], part_dx)):
        assert ((got.float() - want.float()).abs() <= 2.0 ** -7 * want.float().abs() + 1e-3).all()
    assert (last - part_last).abs().max() < 1e-3 and h[a].abs().max() > 0.1 and dz[a].abs().max() > 0.01


@gpu
def test_pack_beyond_4_gb():
    x = torch.empty((1 << 17, 33000), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    p = snn.snn_pack(x)
    codes, exps = to_bytes(x[-2:].float().cpu().numpy())
    assert np.array_equal(p.codes[-2:].cpu().numpy(), codes) and np.array_equal(p.exps[-2:].cpu().numpy(), exps)
    assert np.array_equal(snn.snn_unpack(p, torch.bfloat16)[-2:].double().cpu().numpy(), from_bytes(codes, exps))


@gpu
def test_vocab_beyond_4_gb():
    rows, d, vocab = 8, 2048, 1_200_000  # w and dw: 4.9 GB each
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda").normal_(0.0, 0.05, generator=g)
    t = torch.arange(vocab - rows, vocab, dtype=torch.int32, device="cuda")
    loss, state = snn.snn_vocab_loss(h, w, t)
    dh, dw = snn.snn_vocab_loss_grad(h, w, t, state)
    logits = torch.cat([h.float() @ w[a:a + 100000].float().T for a in range(0, vocab, 100000)], 1).double()
    want = torch.logsumexp(logits, 1) - logits[torch.arange(rows), t.long()]
    assert (loss.double() - want).abs().max() < 1e-4  # 2048 products in 32 bits, logits up to 12
    G = torch.softmax(logits, 1)
    G[torch.arange(rows), t.long()] -= 1
    G /= rows
    for a in (0, vocab - 64):  # an element of G is rounded to bf16, a sum of eight and the result too
        ref = G[:, a:a + 64].T @ h.double()
        assert ((dw[a:a + 64].double() - ref).abs() <= 2.0 ** -7 * (G[:, a:a + 64].abs().T @ h.double().abs()) + 1e-12).all()
    ref = sum(G[:, a:a + 100000].float() @ w[a:a + 100000].float() for a in range(0, vocab, 100000)).double()
    bound = sum(G[:, a:a + 100000].abs().float() @ w[a:a + 100000].abs().float() for a in range(0, vocab, 100000)).double()
    assert ((dh.double() - ref).abs() <= 2.0 ** -7 * bound).all()


# ---- refusals -----------------------------------------------------------------------------------
def refused(call, text):
    with pytest.raises(snn.SnnError) as e:
        call()
    assert e.value.status == snn.SNN_E_INVAL and text in str(e.value), str(e.value)


def test_c_entry_points_refuse_what_they_cannot_run():
    """No GPU needed: shapes and pointers are looked at before anything else happens."""
    L, at = snn.lib(), ops.snn_launch(0, None, None, 0)
    here = C.cast(C.create_string_buffer(4096), C.c_void_p).value

    def glr(**k):
        p = dict(T=10, batch=2, n=8, dtype=0)
        return C.byref(ops.snn_glr(**{**p, **k}))

    def forward(p, launch=C.byref(at), z=here):
        ops._run("snn_glr_forward", launch, p, z, here, None, here, None, None)

    refused(lambda: forward(glr(), None), "no device")
    refused(lambda: forward(None), "no shape")
    refused(lambda: forward(glr(dtype=7)), "unknown type 7")
    refused(lambda: forward(glr(T=-1)), "T = -1")
    refused(lambda: forward(glr(batch=0)), "batch 0")
    refused(lambda: forward(glr(batch=1 << 16, n=1 << 16)), "channels")
    refused(lambda: forward(glr(ld_z=7)), "7 elements")
    refused(lambda: forward(glr(ld_dx=-8)), "-8 elements")
    refused(lambda: forward(glr(ld_h=1 << 40)), "at most")
    refused(lambda: forward(glr(), z=None), "z is NULL")
    refused(lambda: forward(glr(), z=here + 1), "z is not aligned")
    refused(lambda: forward(glr()), "not in device memory" if not torch.cuda.is_available() else "not in")
    assert L.snn_glr_workspace(glr(n=0)) == 0 and L.snn_glr_workspace(glr()) == 0 and L.snn_glr_workspace(glr(T=4096)) > 0
    packed = ops.snn_packed(here, here, 0, 0)

    def backward_packed(p, z=packed):
        ops._run("snn_glr_backward_packed", C.byref(at), p, C.byref(z) if z else None, C.byref(packed), *[here] * 6)

    refused(lambda: backward_packed(glr(), None), "without codes")
    refused(lambda: backward_packed(glr(), ops.snn_packed(here, None, 0, 0)), "without codes")
    refused(lambda: backward_packed(glr(), ops.snn_packed(here, here, 7, 0)), "7 codes")
    refused(lambda: backward_packed(glr(n=33), ops.snn_packed(here, here, 0, 1)), "1 codes or exponents")
    refused(lambda: backward_packed(glr(n=-5)), "n -5")
    for name in ("snn_pack", "snn_unpack"):
        def pack(dtype=0, rows=2, cols=8, ld=0, x=here):
            ops._run(name, C.byref(at), dtype, rows, cols, ld, x, here, here)
        refused(lambda: pack(dtype=2), "unknown type")
        refused(lambda: pack(rows=-1), "rows")
        refused(lambda: pack(cols=0), "rows of 0")
        refused(lambda: pack(rows=1 << 30, cols=1 << 30), "rows of")
        refused(lambda: pack(ld=7), "fewer")
        refused(lambda: pack(), "not in")

    def vocab(**k):
        return C.byref(ops.snn_vocab(**{**dict(rows=4, d=8, vocab=10, dtype=0), **k}))

    def loss(p):
        ops._run("snn_vocab_loss", C.byref(at), p, *[here] * 5)

    refused(lambda: loss(None), "no shape")
    refused(lambda: loss(vocab(dtype=-1)), "unknown type")
    for bad in (dict(rows=-1), dict(d=0), dict(vocab=0), dict(rows=1 << 23), dict(d=1 << 17), dict(vocab=1 << 25)):
        refused(lambda: loss(vocab(**bad)), "2^22")
    refused(lambda: loss(vocab(ld_w=7)), "7 elements")
    refused(lambda: loss(vocab()), "not in")
    assert L.snn_vocab_workspace(vocab(vocab=0), 0) == 0 and L.snn_vocab_workspace(vocab(), 1) > L.snn_vocab_workspace(vocab(), 0) > 0


def test_binding_refuses_tensors_that_do_not_fit():
    f = torch.zeros
    for call, kind in (
            (lambda: snn.snn_glr_forward(f(4, 2, 3), f(4, 2, 3)), ValueError),                          # on the CPU
            (lambda: snn.snn_glr_forward(f(4, 3), f(4, 3)), ValueError),
            (lambda: snn.snn_glr_forward(f(4, 2, 3, dtype=torch.float64), f(4, 2, 3, dtype=torch.float64)), TypeError),
            (lambda: snn.snn_glr_forward(f(4, 2, 3), f(4, 2, 3, dtype=torch.bfloat16)), TypeError),
            (lambda: snn.snn_glr_forward(f(4, 2, 3), f(4, 2, 4)), ValueError),
            (lambda: snn.snn_glr_forward(f(4, 2, 3), f(4, 3, 2).mT), ValueError),
            (lambda: snn.snn_glr_forward(f(4, 1, 3).expand(4, 2, 3), f(4, 2, 3)), ValueError),
            (lambda: snn.snn_glr_forward(f(2, 4, 3).transpose(0, 1), f(4, 2, 3)), ValueError),
            (lambda: snn.snn_glr_forward(f(4, 2, 3), f(4, 2, 3), f(2, 3, dtype=torch.bfloat16)), TypeError),
            (lambda: snn.snn_glr_forward(f(4, 2, 3), f(4, 2, 3), lengths=f(2, dtype=torch.int64)), TypeError),
            (lambda: snn.snn_glr_backward(f(4, 2, 3), f(4, 2, 3), f(2, 2, 3), f(4, 2, 3)), ValueError),
            (lambda: snn.snn_glr_backward(snn.Packed(f(4, 2, 3), f(4, 2, 1)), f(4, 2, 3), f(1, 2, 3), f(4, 2, 3)), TypeError),
            (lambda: snn.snn_pack(f(())), ValueError),
            (lambda: snn.snn_pack(f(4, 0)), ValueError),
            (lambda: snn.snn_pack(f(4, 3, dtype=torch.int32)), TypeError),
            (lambda: snn.snn_pack(f(4, 8)[:, ::2]), ValueError),
            (lambda: snn.snn_unpack(snn.Packed(f(4, 33, dtype=torch.int8), f(4, 1, dtype=torch.uint8))), ValueError),
            (lambda: snn.snn_vocab_loss(f(4, 3), f(5, 4), f(4, dtype=torch.int32)), ValueError),
            (lambda: snn.snn_vocab_loss(f(4, 3), f(5, 3), f(4, dtype=torch.int64)), TypeError),
            (lambda: snn.snn_vocab_loss(f(4, 3), f(5, 3), f(3, dtype=torch.int32)), ValueError),
            (lambda: snn.snn_vocab_loss_grad(f(4, 3), f(5, 3), f(4, dtype=torch.int32), f(4, 2)), ValueError)):
        with pytest.raises(kind):
            call()


@gpu
def test_workspaces_and_host_arrays_are_checked():
    z = torch.zeros(1000, 1, 64, device="cuda")
    p = ops.snn_glr(1000, 1, 64, 0, 0, 0, 0, 0, 0, None)
    need = snn.lib().snn_glr_workspace(C.byref(p))
    assert need > 0
    space = torch.empty(need + 512, dtype=torch.uint8, device="cuda")
    args = [z.data_ptr(), z.data_ptr(), None, torch.empty_like(z).data_ptr(), None, None]

    def call(work, size, device=0, arrays=args):
        ops._run("snn_glr_forward", C.byref(ops.snn_launch(device, None, work, size)), C.byref(p), *arrays)

    call(space.data_ptr(), need)
    torch.cuda.synchronize()
    refused(lambda: call(space.data_ptr(), need - 1), f"{need} are needed")
    refused(lambda: call(None, need), "workspace has 0")
    refused(lambda: call(space.data_ptr() + 4, need), "aligned")
    refused(lambda: call(space.data_ptr(), need, device=1), "device 1")
    host = torch.zeros(1000, 1, 64)
    refused(lambda: call(space.data_ptr(), need, arrays=[host.data_ptr(), *args[1:]]), "z is not in")
    pinned = torch.zeros(1000, 1, 64, pin_memory=True)
    refused(lambda: call(space.data_ptr(), need, arrays=[pinned.data_ptr(), *args[1:]]), "z is not in")


# ---- as many rows as there may be -----------------------------------------------------------------
@gpu
@pytest.mark.parametrize("d,vocab", [(64, 300), (250, 60)])
def test_vocab_weight_gradients_of_many_rows(d, vocab):
    # rows of G the other way round are 6 * rows bytes in fp32: 256 of them in a tile are more than 4 GB
    rows = 2_900_000
    g = torch.Generator(device="cuda").manual_seed(4)
    h = torch.empty((rows, d), device="cuda").normal_(generator=g).abs_()
    w = torch.empty((vocab, d), device="cuda").normal_(0.0, 2 / math.sqrt(d), generator=g)
    t = torch.zeros(rows, dtype=torch.int32, device="cuda")
    state = snn.snn_vocab_loss(h, w, t)[1]
    dw = snn.snn_vocab_loss_grad(h, w, t, state)[1]
    want, W = torch.zeros((vocab, d), dtype=torch.float64, device="cuda"), w.double()
    for a in range(0, rows, 290_000):
        H = h[a:a + 290_000].double()
        G = torch.softmax(H @ W.T, 1)
        G[:, 0] = -G[:, 1:].sum(1)
        want += G.T @ H / rows
    # every term of a sum has the sign of the others: 16 products at least are added at a time, hence rows / 16 roundings at most; logits
    # of up to 6 d products of up to 5 * 10 / sqrt(d)
    near(dw, want.cpu(), ((rows / 16 + 16) * E32 + 4 * (6 * d + 8) * E32) * want.abs().cpu(), "dw")


@gpu
def test_pack_more_rows_than_a_grid_has_threads():
    rows = (1 << 30) + 77
    x = torch.empty((rows, 1), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(5))
    p = snn.snn_pack(x)
    back = snn.snn_unpack(p, torch.bfloat16)
    for part in (slice(0, 1000), slice((1 << 29) - 500, (1 << 29) + 500), slice((1 << 30) - 500, rows)):
        codes, exps = to_bytes(x[part].float().cpu().numpy())
        assert np.array_equal(p.codes[part].cpu().numpy(), codes) and np.array_equal(p.exps[part].cpu().numpy(), exps)
        assert np.array_equal(back[part].double().cpu().numpy(), from_bytes(codes, exps))
    a = rows // 2  # (an element by itself keeps its 7 bits)
    assert ((back[a:].float() - x[a:].float()).abs_() <= 2.0 ** -7 * x[a:].float().abs_()).all()


@gpu
@pytest.mark.parametrize("d,vocab,gradients", [(64, 131072, False), (1024, 2100, True)])
def test_vocab_more_tiles_and_elements_than_a_grid_has_threads(d, vocab, gradients):
    rows = 1 << 22
    g = torch.Generator(device="cuda").manual_seed(6)
    h = torch.empty((rows, d), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.empty((vocab, d), dtype=torch.bfloat16, device="cuda").normal_(0.0, 2 / math.sqrt(d), generator=g)
    t = torch.randint(0, vocab, (rows,), dtype=torch.int32, device="cuda", generator=g)
    loss, state = snn.snn_vocab_loss(h, w, t)
    some = torch.cat([torch.arange(0, 40), torch.arange(rows // 2, rows // 2 + 40), torch.arange(rows - 40, rows)]).cuda()
    H, W, y = h[some].double().cpu(), w.double().cpu(), t[some].long().cpu()
    logits, lse, miss, on, _, want = vocab_loss(H, W, y)
    e_l = (d + 8) * E32 * (H.abs() @ W.abs().T).amax(1) + 4 * E32 * logits.abs().amax(1)
    count = 64 + vocab / 64
    near(loss[some], want, 2 * e_l + count * E32 + 8 * E32 * want, "loss")
    if gradients:
        dh = snn.snn_vocab_loss_grad(h, w, t, state, torch.ones(rows, device="cuda"))[0]
        G, want_h, _ = vocab_grads(H, W, y, torch.ones(len(y), dtype=torch.float64))
        A = G.abs() * (4 * e_l + (count + 16) * E32 + 2.0 ** -8)[:, None]
        near(dh[some], want_h, A @ W.abs() + E32 * (vocab + 8) * (G.abs() @ W.abs()), "dh")


def test_vocab_refuses_more_elements_than_a_grid_reaches():
    with pytest.raises(snn.SnnError, match="2\\^35 in all"):
        ops._run("snn_vocab_loss", C.byref(ops.snn_launch(0, None, None, 0)), C.byref(ops.snn_vocab(1 << 22, (1 << 13) + 1, 10, 1)), *[None] * 5)


# ---- gates that are closed or nearly so -----------------------------------------------------------
def relative_bounds(z, x, h0, dh, dlast):
    """What h, dz, dx and dh0 may be off by, in terms of the magnitudes of what they are sums of: of each step's gate s = min(a, 1 - a), off
    by (|z| + 8) E32 of itself and 2^-126, and of three roundings; twice that, for steps that are joined to maps before they are applied."""
    T = z.shape[0]
    a, c = torch.sigmoid(z), torch.sigmoid(-z)
    e_s = torch.minimum(a, c) * (z.abs() + 8) * E32 + 2.0 ** -126
    m, e, offs = h0.abs(), torch.zeros_like(h0), []
    before_m, before_e = [], []
    for t in range(T):
        before_m.append(m)
        before_e.append(e)
        e = a[t] * e + e_s[t] * (m + x[t].abs())
        m = a[t] * m + c[t] * x[t].abs()
        e = e + 3 * E32 * m
        offs.append(e)
    gm, ge = dlast.abs(), torch.zeros_like(h0)
    tol_z, tol_x = torch.zeros_like(z), torch.zeros_like(z)
    for t in reversed(range(T)):
        gm = gm + dh[t].abs()
        ge = ge + E32 * gm
        off = before_m[t] + x[t].abs()
        tol_x[t] = c[t] * ge + (e_s[t] + 2 * E32 * c[t]) * gm
        tol_z[t] = a[t] * c[t] * (off * ge + gm * (before_e[t] + 5 * E32 * off)) + 2 * e_s[t] * off * gm
        ge = a[t] * ge + (e_s[t] + 2 * E32 * a[t]) * gm
        gm = a[t] * gm
    return [2 * v + 1e-36 for v in (torch.stack(offs), tol_z, tol_x, ge)]


@gpu
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("T,low,high", [(1, -30, -5), (1, -40, 15), (3, -16, -10), (40, -25, 5), (128, -3, 0), (300, -25, 15), (40, 86, 90), (300, 80, 88.8), (300, -90, -86), (300, -200, 200), (5000, -14, 14)])
def test_glr_closed_gates_keep_their_digits(T, low, high, packed):
    # a state and a gradient far above what drives them: what a closed gate lets through of them counts beside that
    g = torch.Generator().manual_seed(T)
    z = low + (high - low) * torch.rand(T, 2, 66, generator=g)
    x, dh = 1e-3 * torch.randn(T, 2, 66, generator=g), 1e-3 * torch.randn(T, 2, 66, generator=g)
    h0, dlast = 1e4 * torch.randn(2, 66, generator=g), 1e4 * torch.randn(2, 66, generator=g)
    zg, xg, dhg, hg, dg = (v.cuda() for v in (z, x, dh, h0, dlast))
    zi, xi = (snn.snn_pack(zg), snn.snn_pack(xg)) if packed else (zg, xg)
    if packed:
        zg, xg = snn.snn_unpack(zi), snn.snn_unpack(xi)
        z, x = zg.cpu(), xg.cpu()
    h, _, kept = snn.snn_glr_forward(zg, xg, hg, keep=True)
    dz, dx, dh0 = snn.snn_glr_backward(zi, xi, kept, dhg, dg)
    z, x, dh, h0, dlast = (v.double() for v in (z, x, dh, h0, dlast))
    all_steps = torch.full((2,), T)
    tol = relative_bounds(z, x, h0, dh, dlast)
    near(h, glr_forward(z, x, h0, all_steps)[0], tol[0], "h")
    for got, want, t, what in zip((dz, dx, dh0), glr_backward(z, x, h0, all_steps, dh, dlast), tol[1:], ("dz", "dx", "dh0")):
        near(got, want, t, what)


@gpu
def test_glr_gates_shut_altogether():
    z = torch.tensor([[[-200.0, -20.0]]], device="cuda")
    h = snn.snn_glr_forward(z, torch.tensor([[[1.0, 1e-3]]], device="cuda"), torch.tensor([[1e8, 1e4]], device="cuda"))[0].cpu()
    assert h[0, 0, 0] == 1 and abs(h[0, 0, 1].item() - (1e-3 + math.exp(-20) * 1e4)) < 1e-3 * 40 * E32


@gpu
@pytest.mark.parametrize("steps", [1, 16, 128])
def test_glr_long_memory_from_call_to_call(steps):
    z, x, state = torch.full((steps, 1, 64), 15.0, device="cuda"), torch.ones((steps, 1, 64), device="cuda"), torch.zeros((1, 64), device="cuda")
    for _ in range(2048 // steps):
        snn.snn_glr_forward(z, x, state, h_last=state)
    want = 1 - (1 - 1 / (1 + math.exp(15.0))) ** 2048
    # as for one call: the gate's digits, and a rounding of the state per step at most
    assert abs(state.double().cpu() - want).max().item() <= want * (20 * E32 + 2048 * 2.0 ** -24)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T", [30, 700])
def test_glr_padded_steps_have_no_gradient_whatever_that_of_the_state(T, dtype):
    z, x, dh, h0, dlast, _ = glr_inputs(T, 4, 66, dtype, False, seed=12)
    lengths = torch.tensor([T, 0, T // 2, 1], dtype=torch.int32, device="cuda")
    kept = snn.snn_glr_forward(z, x, h0, lengths=lengths, keep=True)[2]
    want = snn.snn_glr_backward(z, x, kept, dh, dlast, lengths=lengths)
    dlast[1:, ::2] = torch.tensor([math.inf, math.nan, -math.inf], device="cuda")[:, None]
    dz, dx, dh0 = snn.snn_glr_backward(z, x, kept, dh, dlast, lengths=lengths)
    held = torch.arange(T, device="cuda")[:, None] >= lengths[None, :]
    assert not dz[held].any() and not dx[held].any()
    assert not torch.isfinite(dx[0, 2:, ::2]).any() and not torch.isfinite(dh0[1:, ::2]).any()
    for got, ref in zip((dz, dx, dh0), want):  # the other channels
        assert torch.equal(got[..., 1::2], ref[..., 1::2]) and torch.equal(got[..., 0, :], ref[..., 0, :])


@gpu
def test_a_refused_device_leaves_no_error_behind():
    p = ops.snn_glr(0, 1, 8, 0, 0, 0, 0, 0, 0, None)
    with pytest.raises(snn.SnnError):
        ops._run("snn_glr_forward", C.byref(ops.snn_launch(63, None, None, 0)), C.byref(p), *[None] * 6)
    assert (torch.zeros(3, device="cuda") + 1).sum().item() == 3 and torch.cuda.current_device() == 0
    snn.snn_glr_forward(torch.zeros(1, 1, 8, device="cuda"), torch.zeros(1, 1, 8, device="cuda"))


@gpu
@pytest.mark.parametrize("sign", [1, -1])
def test_vocab_logits_up_to_2_to_the_30(sign):
    # of some rows one logit's neighbours, 2^-24 of it away, are much further off than 1: a loss is a difference of logits, each off by 2^-24
    sizes = torch.tensor([1e3, 1e6, 3.1e7, 1.7e8, 5.5e8, 1.07e9, 1.08e9, 3.4e9, 1e10, 1.1e10, 1e30], dtype=torch.float32)
    h, w = sizes[:, None], sign * torch.tensor([[1.0], [1.5], [0.5], [1.5]])
    for y in range(4):
        t = torch.full((11,), y, dtype=torch.int32)
        loss, state = snn.snn_vocab_loss(h.cuda(), w.cuda(), t.cuda())
        dh = snn.snn_vocab_loss_grad(h.cuda(), w.cuda(), t.cuda(), state, torch.ones(11, device="cuda"))[0].cpu()
        _, _, _, _, _, want = vocab_loss(h.double(), w.double(), t.long())
        beyond = (h[:, 0] * (1.5 if sign > 0 else 0.5)) >= 2.0 ** 30  # the largest logit's magnitude
        assert torch.isnan(loss.cpu()[beyond]).all() and torch.isnan(dh[beyond]).all() and torch.isfinite(dh[~beyond]).all()
        # (both logits times log2(e), their difference, times log(2); the logarithm of a sum of two)
        near(loss[~beyond.cuda()], want[~beyond], 8 * E32 * (want[~beyond] + 1), "loss")


@gpu
@pytest.mark.parametrize("rows,d,vocab", [(1, 64, 7), (1, 512, 1000), (2, 70, 300), (31, 130, 1025), (32, 64, 129), (17, 200, 2500), (32, 96, 5003), (5, 24, 4100)])
def test_vocab_gradients_of_few_rows_lose_nothing_but_their_own_rounding(rows, d, vocab):
    # sums of few terms, or of few that count: each element of G is off by its logits and 2^-16, nothing of the size of a rounding to bf16
    h, w, t, dloss = vocab_inputs(rows, d, vocab, torch.bfloat16, seed=rows)
    t[0] = vocab // 2
    gh, gw, gt = h.cuda(), w.cuda(), t.cuda()
    state = snn.snn_vocab_loss(gh, gw, gt)[1]
    H, W, t64 = h.double(), w.double(), t.long()
    e_l = (d + 8) * E32 * (H.abs() @ W.abs().T).amax(1) + 4 * E32 * (H @ W.T).abs().amax(1)
    for given in (None, dloss):
        on = (t >= 0).double()
        G, want_h, want_w = vocab_grads(H, W, t64, on / on.sum() if given is None else given.double())
        dh, dw = snn.snn_vocab_loss_grad(gh, gw, gt, state, None if given is None else given.cuda())
        A = G.abs() * (4 * e_l + (80 + vocab / 64) * E32 + 2.0 ** -16)[:, None]
        near(dh, want_h, A @ W.abs() + (vocab + 8) * E32 * (G.abs() @ W.abs()) + 1e-30, "dh")
        near(dw, want_w, A.T @ H.abs() + (rows + 8) * E32 * (G.abs().T @ H.abs()) + 1e-30, "dw")
