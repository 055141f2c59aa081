"""Norm, optimizer step and delta rule of token sequence models (snn_norm_*, snn_adamw_step, snn_delta_*) against plain implementations in 64 bits
on the CPU, through the Python binding.  Refusals that need no GPU run everywhere.

Tolerances count roundings: U = 2^-24 is what one in 32 bits is off by at most, relative to its result; results in bf16 are off by half
a step, 2^-8 of the value, on top."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2412_11810_amd as snn
from paper_2412_11810_amd import ops

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}
TYPES = [torch.float32, torch.bfloat16]


def near(got, want, tol, what):
    """|got - want| <= tol + half a step of got's type, everywhere."""
    got_, want = got.double().cpu(), want.double().cpu()
    assert got_.shape == want.shape, what
    off = (got_ - want).abs() - (tol + HALF[got.dtype] * want.abs())
    assert not torch.isnan(off).any() and off.max().item() <= 0 if off.numel() else True, (what, off.max().item())


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def rows_of(shape, dtype, seed, wide=0, spread=0.5):
    """Rows on the GPU, those of a wider array (NaN beside them) with `wide`."""
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(*shape[:-1], 1, generator=g))).to(dtype)
    if wide:
        w = torch.full((*shape[:-1], shape[-1] + wide), math.nan, dtype=dtype, device="cuda")
        w[..., 1:shape[-1] + 1] = x.cuda()
        return w[..., 1:shape[-1] + 1]
    return x.cuda()


# ---- norm ---------------------------------------------------------------------------------------
NORM = [(1, 1), (2200, 2000), (130, 1000), (1030, 600), (3, 2), (5, 8), (70, 31), (64, 64), (9, 75), (1000, 128), (3, 500), (33, 513), (7, 1024), (5, 1501), (64, 2048), (3, 2049), (4, 4096),
        (2, 8191), (3, 8200), (2, 16385), (1, 32768), (5000, 40), (2100, 1100)]
ROUNDINGS = 64  # of a sum over a row: 32 elements in a lane, 6 exchanges, 16 wavefronts, and the square root, the quotient and three products


def norm_plain(x, r, w, eps):
    s = x.double().cpu() + (0 if r is None else r.double().cpu())
    i = 1 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    return s, i, s * i * (1 if w is None else w.double().cpu())


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", NORM)
def test_norm_forward(rows, n, dtype):
    x, r = rows_of((rows, n), dtype, 1, wide=n % 2 * 3), rows_of((rows, n), dtype, 2)
    w = rows_of((1, n), dtype, 3)[0]
    s, i, want = norm_plain(x, r, w, 1e-6)
    y, total = snn.snn_norm_forward(x, w, residual=r, eps=1e-6)
    near(total, s, U * s.abs(), "total")
    near(y, want, ROUNDINGS * U * want.abs(), "y")
    want = norm_plain(x, None, None, 0.25)[2]
    y, total = snn.snn_norm_forward(x, eps=0.25)
    assert total is x
    near(y, want, ROUNDINGS * U * want.abs(), "y without residual and weights")
    # in place, and into a part of a wider array
    wide, stream = torch.full((rows, 2 * n), 7.0, dtype=dtype, device="cuda"), r.clone()
    y2, total2 = snn.snn_norm_forward(x, w, residual=stream, eps=1e-6, y=wide[:, n:], total=stream)
    assert total2 is stream
    assert same([y2, total2], snn.snn_norm_forward(x, w, residual=r, eps=1e-6)) and (wide[:, :n] == 7).all()


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", NORM)
def test_norm_forward_packed(rows, n, dtype):
    x, r = rows_of((rows, n), dtype, 4, wide=n % 2), rows_of((rows, n), dtype, 5)
    w = rows_of((1, n), dtype, 6)[0]
    want = norm_plain(x, r, w, 1e-6)[2]
    p, total = snn.snn_norm_forward(x, w, residual=r, eps=1e-6, packed=True)
    assert same([total], snn.snn_norm_forward(x, w, residual=r, eps=1e-6)[1:])
    blocks = torch.nn.functional.pad(want, (0, -n % 32)).unflatten(-1, (-1, 32))
    off = ROUNDINGS * U
    top, step = blocks.abs().amax(-1), torch.exp2(p.exps.cpu().double() - 127)
    # the smallest step that fits, but for what the largest element may be off by
    assert (top <= 127.5 * step * (1 + off)).all() and (top * (1 + off) > 127.5 * step / 2).all()
    codes = torch.nn.functional.pad(p.codes.cpu().double(), (0, -n % 32)).unflatten(-1, (-1, 32))
    assert ((codes * step[..., None] - blocks).abs() <= 0.5 * step[..., None] + off * blocks.abs()).all()
    if dtype == torch.float32:  # y is not rounded before: its codes are those of snn_pack
        assert same(p, snn.snn_pack(snn.snn_norm_forward(x, w, residual=r, eps=1e-6)[0]))


def norm_back_plain(s, w, dy, ds, eps):
    s, dy = s.double().cpu(), dy.double().cpu()
    mine = dy if w is None else dy * w.double().cpu()
    i = 1 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    hat = s * i
    dx = i * (mine - hat * (mine * hat).mean(-1, keepdim=True)) + (0 if ds is None else ds.double().cpu())
    size = i * (mine.abs() + hat.abs() * (mine * hat).abs().mean(-1, keepdim=True))
    return dx, size, (dy * hat).sum(0), (dy * hat).abs().sum(0)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", NORM)
def test_norm_backward(rows, n, dtype):
    s, dy, ds = rows_of((rows, n), dtype, 7), rows_of((rows, n), dtype, 8, wide=n % 2 * 2), rows_of((rows, n), dtype, 9)
    w = rows_of((1, n), dtype, 10)[0]
    dx, size, dw, terms = norm_back_plain(s, w, dy, ds, 1e-6)
    got, got_w = snn.snn_norm_backward(s, w, dy, dtotal=ds, eps=1e-6)
    near(got, dx, 3 * ROUNDINGS * U * size + U * ds.double().cpu().abs(), "dx")
    # a sum over rows: those of a lane one after the other (1024 workgroups take turns), then up to 1024 in 32 strands
    near(got_w, dw, (ROUNDINGS + rows / 1024 + 80) * U * terms, "dw")
    free, none = snn.snn_norm_backward(s, None, dy, eps=1e-6)
    plain = norm_back_plain(s, None, dy, None, 1e-6)
    assert none is None
    near(free, plain[0], 3 * ROUNDINGS * U * plain[1], "dx without weights")
    place = dy.clone()
    assert same(snn.snn_norm_backward(s, w, place, dtotal=ds, eps=1e-6, dx=place), [got, got_w])
    place = ds.clone()
    assert same(snn.snn_norm_backward(s, w, dy, dtotal=place, eps=1e-6, dx=place), [got, got_w])


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n", NORM)
def test_norm_results_in_the_place_of_inputs(rows, n, dtype):
    x, r, dy = (rows_of((rows, n), dtype, k, wide=n % 2) for k in (31, 32, 33))
    w = rows_of((1, n), dtype, 34)[0]
    want, back = snn.snn_norm_forward(x, w, residual=r), snn.snn_norm_backward(x, w, dy, dtotal=r)
    for total, y in ((0, 1), (1, 0), (None, 0), (None, 1)):
        place = [rows_of((rows, n), dtype, k, wide=n % 2) for k in (31, 32)]
        got = snn.snn_norm_forward(place[0], w, residual=place[1], total=None if total is None else place[total], y=place[y])
        assert got[0] is place[y] and (total is None or got[1] is place[total]) and same(got, want)
    place = x.clone()
    assert same(snn.snn_norm_backward(place, w, dy, dtotal=r, dx=place), back)


@gpu
def test_norm_refuses_results_in_other_places():
    wide, w = torch.zeros((9, 40), device="cuda"), torch.ones(40, device="cuda")
    x, r = wide[1:], torch.zeros((8, 40), device="cuda")
    for call in (lambda: snn.snn_norm_forward(x, w, residual=r, total=wide[:-1]), lambda: snn.snn_norm_forward(x, w, y=wide[:-1]),
                 lambda: snn.snn_norm_forward(x, w, residual=r, total=x, y=x), lambda: snn.snn_norm_forward(x, wide[3], y=x),
                 lambda: snn.snn_norm_backward(x, w, r, dx=wide[:-1]), lambda: snn.snn_norm_backward(r, wide[4], r, dx=x)):
        refused(call, "share elements")
    assert (wide == 0).all()


@gpu
def test_norm_gradients_are_differences():
    s, dy, w = (rows_of(x, torch.float32, k) for k, x in enumerate(((5, 33), (5, 33), (1, 33))))
    dx, dw = snn.snn_norm_backward(s, w[0], dy, eps=1e-3)
    f = lambda a, b: (norm_plain(a, None, b, 1e-3)[2] * dy.double().cpu()).sum()  # noqa: E731
    d, S, W = 1e-6, s.double().cpu(), w[0].double().cpu()
    for r, c in ((0, 0), (2, 17), (4, 32)):
        e = torch.zeros_like(S)
        e[r, c] = d
        # (a third derivative of size 30 d^2, and 1e-16 of f over d)
        assert abs((f(S + e, W) - f(S - e, W)) / (2 * d) - dx[r, c].item()) < 1e-5 * max(1, dx.abs().max().item())
        assert abs((f(S, W + e[r]) - f(S, W - e[r])) / (2 * d) - dw[c].item()) < 1e-5 * max(1, dw.abs().max().item())


@gpu
@pytest.mark.parametrize("n", [40, 600, 3000, 9000])
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_numbers_of_any_size(n, dtype):
    x = rows_of((8, n), dtype, 11, spread=0)
    scale = torch.tensor([1e36, 1e30, 1e25, 1.0, 1e-18, 1e-25, 1e-36, 0.0], device="cuda")[:, None]
    x = (x.float() * scale).to(dtype)
    w, dy = rows_of((1, n), dtype, 12)[0], rows_of((8, n), dtype, 13)
    for eps in (0.0, 1e-6):
        live = slice(0, 7) if eps == 0 else slice(0, 8)  # (0 / 0 is NaN)
        y = snn.snn_norm_forward(x, w, eps=eps)[0]
        want = norm_plain(x, None, w, eps)[2]
        near(y[live], want[live], ROUNDINGS * U * want[live].abs() + 2.0 ** -133, "y")
        got = snn.snn_norm_backward(x[live], w, dy[live], eps=eps)
        dx, size, dw, terms = norm_back_plain(x[live], w, dy[live], None, eps)
        fits = size.amax(1) < 1e37  # a row of 1e-36 has gradients of 1e36
        near(got[0][fits.cuda()], dx[fits], (3 * ROUNDINGS * U * size + 2.0 ** -133)[fits], "dx")
        near(got[1], dw, (ROUNDINGS + 80) * U * terms + 2.0 ** -133, "dw")
        if eps == 0:
            assert torch.isnan(y[7]).all()


@gpu
def test_norm_values_that_are_not_finite_stay_in_their_rows():
    x = rows_of((6, 100), torch.float32, 14)
    clean, w = x.clone(), torch.ones(100, device="cuda")
    x[1, 3], x[4, 99] = math.inf, math.nan
    y, p = snn.snn_norm_forward(x, w)[0], snn.snn_norm_forward(x, w, packed=True)[0]
    want = snn.snn_norm_forward(clean, w)[0]
    rest = [0, 2, 3, 5]
    assert torch.equal(y[rest], want[rest]) and torch.isnan(y[4]).all() and torch.isnan(y[1, 3]) and (y[1, :3] == 0).all()
    assert same([p.codes[rest], p.exps[rest]], [z[rest] for z in snn.snn_pack(want)])
    assert (p.exps[4] == 255).all() and p.exps[1].tolist() == [255, 0, 0, 0]


@gpu
def test_norm_of_no_rows():
    x, w = torch.zeros((0, 70), device="cuda"), torch.ones(70, device="cuda")
    assert snn.snn_norm_forward(x, w, residual=x)[0].shape == (0, 70) and snn.snn_norm_forward(x, w, packed=True)[0].exps.shape == (0, 3)
    dx, dw = snn.snn_norm_backward(x, w, x)
    assert dx.shape == (0, 70) and (dw == 0).all()


@gpu
def test_norm_beyond_4_gb():
    rows, n = 70000, 32768  # 4.6 GB in bf16
    x = torch.empty((rows, n), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    y, total = snn.snn_norm_forward(x, None, residual=x)
    at = slice(rows - 3, rows)
    want = norm_plain(x[at], x[at], None, 1e-6)
    near(y[at], want[2], ROUNDINGS * U * want[2].abs(), "y")
    assert torch.equal(total, 2 * x)


# ---- AdamW --------------------------------------------------------------------------------------
C1, C2 = 0xC13FA9A9, 0x91E10DA5


def adamw_plain(p, g, m, v, t, lr, betas, eps, decay):
    """New p, m, v, and what they may be off by in 32 bits."""
    a, b = betas
    m1, v1 = a * m + (1 - a) * g, b * v + (1 - b) * g * g
    em, ev = 4 * U * (a * m.abs() + (1 - a) * g.abs()), 5 * U * v1
    root = torch.sqrt(v1 / (1 - b ** t)) + eps
    move = lr * m1 / (1 - a ** t) / root
    p1 = p * (1 - lr * decay) - move
    # half of v's error, six factors and quotients
    return p1, m1, v1, 2 * U * p.abs() + lr * em / (1 - a ** t) / root + 10 * U * move.abs(), em, ev


def values(p):
    return p.codes.cpu().double().flatten() * torch.exp2(p.exps.cpu().double() - 127).repeat_interleave(32)[:p.codes.numel()]


def check_codes(p, want, tol, t, c1, c2, root):
    """The codes of a moment in 8 bits: floor(x / step + u) of an x within tol of `want`."""
    n = len(want)
    pad = lambda x: torch.nn.functional.pad(x, (0, -n % 32)).view(-1, 32)  # noqa: E731
    step = torch.exp2(p.exps.cpu().double() - 127)[:, None]
    x, e, codes = pad(want), pad(tol), pad(p.codes.cpu().double().flatten())
    top = x.abs().amax(1)
    assert ((top - e.amax(1)) <= 127 * step[:, 0]).all()
    assert ((top + e.amax(1) > 63.5 * step[:, 0]) | (p.exps.cpu() <= 1)).all()
    assert ((p.exps.cpu() == 0) == (top == 0)).all()
    i = torch.arange(x.numel()).view(x.shape)
    u = (((i * c1 + t * c2) % 2 ** 32) // 2 ** 16).double() / 2 ** 16
    at = x / step + u
    lowest = torch.where(x > 0, 1.0, -127.0) if root else torch.full_like(x, -127.0)
    assert (codes <= torch.maximum(at + e / step + 2.0 ** -16, lowest)).all() and (codes >= lowest).all()  # (x / step + u has 24 bits)
    assert (codes > at - 1 - e / step - 2.0 ** -16).all()


SHAPES = [(1,), (7, 5), (32,), (33,), (0,), (4, 64), (8192,), (8193,), (5, 3001), (1025, 64)]


def adamw_inputs(shapes, bits, kinds, seed=1):
    g = torch.Generator().manual_seed(seed)
    params = [(0.1 * torch.randn(x, generator=g)).to(k).cuda() for x, (k, _) in zip(shapes, kinds)]
    grads = [(0.01 * torch.exp(2 * torch.randn((), generator=g)) * torch.randn(x, generator=g)).to(k).cuda() for x, (_, k) in zip(shapes, kinds)]
    copies = [torch.full(p.shape, 7.0, dtype=torch.bfloat16, device="cuda") if p.dtype == torch.float32 and i % 3 else None for i, p in enumerate(params)]
    return params, grads, copies, *snn.snn_adamw_moments(params, bits)


@gpu
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("many", [False, True])
def test_adamw_steps(bits, many):
    shapes = SHAPES * (9 if many else 1)  # more tensors than a launch takes
    kinds = [(TYPES[i % 2], TYPES[i // 2 % 2]) for i in range(len(shapes))]
    params, grads, copies, m, v = adamw_inputs(shapes, bits, kinds)
    plan = snn.snn_adamw_plan(params, m, v, copies)
    how = dict(lr=3e-3, betas=(0.85, 0.98), eps=1e-7, weight_decay=0.2)
    for t in (1, 2, 3, 50, 1000003):
        flat = lambda x: values(x) if bits == 8 else x.cpu().double().flatten()  # noqa: E731
        before = [(p.cpu().double().flatten(), g.cpu().double().flatten(), flat(a), flat(b) ** (2 if bits == 8 else 1)) for p, g, a, b in zip(params, grads, m, v)]
        snn.snn_adamw_step(plan, grads, t, **how)
        for k, (x, p, a, b, c) in enumerate(zip(before, params, m, v, copies)):
            p1, m1, v1, ep, em, ev = adamw_plain(*x, t, how["lr"], how["betas"], how["eps"], how["weight_decay"])
            near(p.flatten(), p1, ep, ("p", k, t))
            if c is not None:
                assert torch.equal(c, p.to(torch.bfloat16))
            if not len(p1):
                continue
            if bits == 32:
                near(a.flatten(), m1, em, ("m", k, t))
                near(b.flatten(), v1, ev, ("v", k, t))
            else:
                check_codes(a, m1, em, t, C1, C2, False)
                root = torch.sqrt(v1)
                check_codes(b, root, 4 * U * root, t, C2, C1, True)
        grads = [g * 0.5 for g in grads]


@gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_of_parts_of_arrays(bits):
    # at any address, and nothing beside them is touched
    shapes, kinds = [(37,), (8200,), (1,), (3, 50)], [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)] * 2
    params, grads, copies, m, v = adamw_inputs(shapes, bits, kinds)
    wide, at = [], 0

    def part(x):
        nonlocal at
        at += 1
        w = torch.full((x.numel() + 16,), 99, dtype=x.dtype, device="cuda")
        first = 1 + at % 7
        w[first:first + x.numel()] = x.flatten()
        wide.append((w, first, x.numel()))
        return w[first:first + x.numel()].view(x.shape)

    of = lambda x: snn.Packed(*map(part, x)) if bits == 8 else part(x)  # noqa: E731
    plans = [snn.snn_adamw_plan([part(x) for x in params], [of(x) for x in m], [of(x) for x in v], [x if x is None else part(x) for x in copies])]
    theirs = [part(g) for g in grads]
    plans.append(snn.snn_adamw_plan(params, m, v, copies))
    for t in (1, 2, 3):
        snn.snn_adamw_step(plans[0], theirs, t)
        snn.snn_adamw_step(plans[1], grads, t)
    assert same(plans[0].memory, plans[1].memory)
    for w, first, n in wide:
        assert (w[:first] == 99).all() and (w[first + n:] == 99).all()


@gpu
def test_adamw_in_8_bits_follows_moments_that_change_little_at_a_time():
    # gradients that stop: a root changes by 1/2000 of itself at a time, a twentieth of a code at most
    params = [torch.zeros(4096, device="cuda")]
    m, v = snn.snn_adamw_moments(params, 8)
    plan, g = snn.snn_adamw_plan(params, m, v), torch.linspace(0.5, 1.0, 4096, device="cuda")
    for t in range(1, 101):
        snn.snn_adamw_step(plan, [g], t)
    for t in range(101, 1101):
        snn.snn_adamw_step(plan, [0 * g], t)
    want = g.double().cpu() * math.sqrt(1 - 0.999 ** 100) * 0.999 ** 500
    step = torch.exp2(v[0].exps.cpu().double() - 127).repeat_interleave(32)
    # a sum of N errors floor(x + u) - x over multiples of an irrational number grows with the logarithm of N: 3 + log2 N is more than any
    assert ((values(v[0]) - want).abs() <= (3 + math.log2(1100)) * step).all()
    # and cancels over the elements: their mean is off by a part of a step
    assert abs((values(v[0]) - want).mean().item()) <= 0.25 * step.max().item()


@gpu
def test_adamw_first_steps_of_elements_of_very_different_sizes():
    # a root that has no code of its own has the smallest: its element moves less than in 32 bits, never more
    g = torch.full((64,), 1e-6, device="cuda")
    g[::32] = 1.0
    params = [torch.zeros(64, device="cuda")]
    plan = snn.snn_adamw_plan(params, *snn.snn_adamw_moments(params, 8))
    for t in range(1, 20):
        before = params[0].clone()
        snn.snn_adamw_step(plan, [g], t, lr=1.0, weight_decay=0.0)
        # its m is at most rounded up to a step, 1 / 63.5 of the block's largest, its root 1 / 127 of that one's at least: a quotient of 2 and its
        # own 1e-6; the largest element's is 1
        assert ((params[0] - before).abs() <= 2.1).all()
    assert (plan.v[0].codes > 0).all()


@gpu
def test_adamw_scale_of_gradients_and_step_on_the_device():
    kinds = [(torch.float32, torch.bfloat16)] * len(SHAPES)
    both = [adamw_inputs(SHAPES, 8, kinds) for _ in range(2)]
    plans = [snn.snn_adamw_plan(x[0], x[3], x[4], x[2]) for x in both]
    step, scale = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.full((1,), 0.25, device="cuda")
    for t in (1, 2, 3):
        snn.snn_adamw_step(plans[0], both[0][1], t)
        snn.snn_adamw_step(plans[1], [g * 4 for g in both[1][1]], step, grad_scale=scale)
        assert step.item() == t
    for a, b in zip(both[0][0] + both[0][2], both[1][0] + both[1][2]):
        # (the device's pow() and the host's may differ in their last bit of 64)
        assert a is None or torch.allclose(a.float(), b.float(), rtol=4 * U if a.dtype == torch.float32 else 2.0 ** -7, atol=1e-9)


@gpu
def test_adamw_in_a_graph():
    kinds = [(torch.float32, torch.float32)] * len(SHAPES)
    (params, grads, copies, m, v), (other, _, _, om, ov) = (adamw_inputs(SHAPES, 32, kinds) for _ in range(2))
    plan, eager = snn.snn_adamw_plan(params, m, v, copies), snn.snn_adamw_plan(other, om, ov)
    step, eager_step = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        snn.snn_adamw_step(plan, grads, step)
    for t in range(1, 5):
        for g in grads:
            g.mul_(0.9)
        graph.replay()
        torch.cuda.synchronize()
        snn.snn_adamw_step(eager, grads, eager_step)
        assert step.item() == t and same(params, other) and same(m, om) and same(v, ov)


@gpu
def test_adamw_of_more_elements_than_32_bits_count():
    n = 2 ** 32 + 100
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 2 ** 31 - 1, 2 ** 31, 2 ** 32 - 1, 2 ** 32, n - 1], device="cuda")
    g[at] = torch.arange(1, 7, device="cuda").to(torch.bfloat16)
    m, v = snn.snn_adamw_moments([p], 8)
    snn.snn_adamw_step(snn.snn_adamw_plan([p], m, v), [g], 1, lr=0.5, weight_decay=0.0)
    assert (p[at] == -0.5).all() and p.count_nonzero().item() == 6
    assert (v[0].codes[at] > 0).all() and v[0].codes.count_nonzero().item() == 6


@gpu
def test_adamw_refuses_arrays_that_share_elements():
    x = torch.zeros(200, device="cuda")
    m, v = snn.snn_adamw_moments([x, x])
    g = [torch.ones(200, device="cuda")] * 2
    for params, grads, moments in (([x, x], g, (m, v)), ([x[:100], x[99:199]], [g[0][:100]] * 2, ([y[:100] for y in m], [y[:100] for y in v])),
                                   ([x], [x], (m[:1], v[:1])), ([x], g[:1], (m[:1], m[:1])), ([x], [m[0]], (m[:1], v[:1]))):
        with pytest.raises(snn.SnnError) as e:
            snn.snn_adamw_step(snn.snn_adamw_plan(params, *moments), grads, 1)
        assert e.value.status == snn.SNN_E_INVAL and "shares" in str(e.value) or "share" in str(e.value)
    assert (x == 0).all()
    y = torch.zeros(100, device="cuda")
    snn.snn_adamw_step(snn.snn_adamw_plan([x[:100], y], *snn.snn_adamw_moments([y, y])), [g[0][:100]] * 2, 1)  # one gradient for two is none


@gpu
def test_adamw_gradients_that_are_not_finite():
    p = [torch.zeros(96, device="cuda")]
    m, v = snn.snn_adamw_moments(p, 8)
    g = torch.ones(96, device="cuda")
    g[40] = math.nan
    snn.snn_adamw_step(snn.snn_adamw_plan(p, m, v), [g], 1)
    assert m[0].exps.tolist()[1] == v[0].exps.tolist()[1] == 255 and torch.isnan(p[0]).nonzero().tolist() == [[40]]
    assert torch.isfinite(values(m[0])[:32]).all() and torch.isfinite(values(m[0])[64:]).all()


@gpu
def test_adamw_moves_the_weights_of_a_network():
    import synth
    w = synth.config(0)
    d = synth.generate(w)
    net = snn.from_workload(w, d, device=0)
    kinds = [(snn.SNN_W_IN, 0), (snn.SNN_W_REC, 0), (snn.SNN_W_OUT, 0)]
    params = [torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda() for x in (d["W_in"][0], d["W_rec"][0], d["W_out"])]
    plan = snn.snn_adamw_plan(params, *snn.snn_adamw_moments(params))
    net.snn_bind_inputs(d["in_spikes"], d["labels"], w.T)
    for t in (1, 2):
        net.snn_bptt(snn.SNN_CHUNK, 0, 16)
        grads = [net.snn_grads(*k) for k in kinds]
        before = [p.cpu().double() for p in params]
        moments = [(a.cpu().double(), b.cpu().double()) for a, b in zip(plan.m, plan.v)]
        snn.snn_adamw_step(plan, [torch.from_numpy(g).cuda() for g in grads], t, lr=1e-4)
        for p, x, g, (a, b), k in zip(params, before, grads, moments, kinds):
            want = adamw_plain(x, torch.from_numpy(g).double(), a, b, t, 1e-4, (0.9, 0.999), 1e-8, 0.01)
            near(p, want[0], want[3], "weights")
            net.snn_set_weights(*k, p)
    net.snn_bptt(snn.SNN_CHUNK, 0, 16)
    assert not np.array_equal(net.snn_grads(*kinds[0]), grads[0])
    net.snn_destroy()


# ---- gated delta rule ---------------------------------------------------------------------------
def delta_plain(q, k, v, g, beta, s0, lengths, scale):
    """Step by step, differentiable."""
    T, B, H = g.shape
    heads = torch.arange(H) // (H // q.shape[2])
    S, o, kept = s0, [], []
    for t in range(T):
        if t % 256 == 0:
            kept.append(S)
        on = (t < lengths)[:, None, None, None]
        kt, qt = k[t][:, heads], q[t][:, heads]
        held = torch.exp(g[t])[..., None, None] * S
        u = beta[t][..., None] * (v[t] - (held * kt[..., None]).sum(-2))
        S = torch.where(on, held + kt[..., None] * u[..., None, :], S)
        o.append(torch.where(on[..., 0], scale * (S * qt[..., None]).sum(-2), 0.0))
    return torch.stack(o) if T else torch.zeros_like(v), S, torch.stack(kept) if T else S[None][:0]


def delta_inputs(T, B, H, K, dk, dv, dtype, ragged=False, seed=1):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *x: torch.randn(x, generator=g)  # noqa: E731
    q, k = rand(T, B, K, dk), rand(T, B, K, dk) + 0.5 * rand(1, B, K, dk)
    q, k = ((x / x.norm(dim=-1, keepdim=True)).to(dtype) for x in (q, k))
    x = dict(q=q, k=k, v=rand(T, B, H, dv).to(dtype), g=-torch.nn.functional.softplus(rand(T, B, H) - 1) * torch.exp(-3 * torch.rand(H, generator=g)),
             beta=torch.sigmoid(rand(T, B, H)))
    s0, do, ds = rand(B, H, dk, dv), rand(T, B, H, dv).to(dtype), rand(B, H, dk, dv)
    lengths = torch.full((B,), T, dtype=torch.int32)
    if ragged:
        lengths = torch.randint(0, T + 1, (B,), generator=g, dtype=torch.int32)
        lengths[0], lengths[-1] = T, 0
        pad = torch.arange(T)[:, None] >= lengths[None, :]
        for a in (*x.values(), do):
            a[pad] = math.nan  # nothing may read these
    return [a.cuda() for a in x.values()], s0.cuda(), do.cuda(), ds.cuda(), lengths.cuda()


def clean(a, lengths):
    """In 64 bits on the CPU, zeros behind the ends."""
    a = a.cpu().double()
    return torch.where((torch.arange(a.shape[0])[:, None] < lengths.cpu()[None, :]).view(*a.shape[:2], *[1] * (a.dim() - 2)), a, 0.0)


def delta_tol(T, dk, times):
    """What results may be off by, to their 2-norm.  Roundings of either sign add up as the root of their number: sums over dk and over 64 steps, twice
    each, and those of up to 16 chunks that a state remembers.  Four times that, for what adds up in one direction; `times` as much where such results
    are factors again."""
    return times * 4 * U * math.sqrt(2 * (dk + 64) * min(T / 64 + 1, 16))


def close(got, want, tol, what):
    """To the 2-norm, and each element to 30 times the root mean square besides its own rounding.  Results in bf16 come of factors in two parts, each off by
    2^-17 at most, two of them."""
    got_, want = got.double().cpu(), want.double()
    assert got_.shape == want.shape, what
    if not want.numel():
        return
    if got.dtype == torch.bfloat16:
        tol += 2.0 ** -16
    off, norm = (got_ - want).norm().item(), want.norm().item()
    assert off <= (tol + HALF[got.dtype]) * norm, (what, off / max(norm, 1e-300), tol)
    rest = ((got_ - want).abs() - HALF[got.dtype] * want.abs()).max().item()
    assert rest <= 30 * tol * norm / math.sqrt(want.numel()), (what, rest, norm)


DELTA = [(0, 2, 3, 3, 5, 7, False), (1, 2, 3, 3, 5, 7, False), (1, 64, 4, 2, 128, 128, False), (3, 2, 2, 1, 65, 130, True), (16, 2, 4, 4, 128, 64, True),
         (17, 1, 2, 2, 16, 16, False), (63, 2, 1, 1, 1, 1, False), (64, 2, 2, 2, 64, 64, False), (65, 3, 3, 1, 48, 75, True), (130, 3, 2, 2, 33, 31, True),
         (256, 1, 2, 2, 128, 128, False), (257, 3, 2, 1, 64, 100, True), (300, 5, 4, 2, 128, 40, True), (700, 1, 1, 1, 100, 256, False),
         (200, 4, 6, 2, 72, 33, True), (128, 8, 8, 8, 32, 96, False), (8, 2, 3, 1, 100, 70, True), (12, 64, 4, 2, 24, 40, True), (32, 64, 4, 4, 70, 20, False),
         (70, 1, 2, 1, 128, 1024, False), (2, 1, 3, 3, 17, 1000, False), (40, 300, 6, 2, 5, 3, True), (90, 2, 40, 5, 16, 33, True),
         (1100, 3, 2, 1, 64, 40, True), (1500, 2, 2, 2, 100, 33, True), (2600, 1, 1, 1, 16, 16, False), (1030, 1, 4, 2, 128, 130, False)]


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,B,H,K,dk,dv,ragged", DELTA)
def test_delta_forward(T, B, H, K, dk, dv, ragged, dtype):
    x, s0, _, _, lengths = delta_inputs(T, B, H, K, dk, dv, dtype, ragged)
    given = lengths if ragged else None
    o, last, kept = snn.snn_delta_forward(*x, s0, lengths=given, keep=True)
    c, tol = [clean(a, lengths) for a in x], delta_tol(T, dk, 1)
    want = delta_plain(*c, s0.cpu().double(), lengths.cpu(), dk ** -0.5)
    for got, ref, what in zip((o, last, kept), want, ("o", "last", "kept")):
        close(got, ref, tol, what)
    assert (o[torch.arange(T, device="cuda")[:, None] >= lengths[None, :]] == 0).all()
    if T:
        close(snn.snn_delta_forward(*x, None, lengths=given, scale=2.0)[0], delta_plain(*c, 0 * s0.cpu().double(), lengths.cpu(), 2.0)[0], tol, "from zero")


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,B,H,K,dk,dv,ragged", DELTA)
def test_delta_backward(T, B, H, K, dk, dv, ragged, dtype):
    x, s0, do, ds, lengths = delta_inputs(T, B, H, K, dk, dv, dtype, ragged, seed=2)
    given = lengths if ragged else None
    c = [clean(a, lengths).requires_grad_() for a in x]
    S = s0.cpu().double().requires_grad_()
    o, last, kept = delta_plain(*c, S, lengths.cpu(), dk ** -0.5)
    f = (o * clean(do, lengths)).sum()
    got = snn.snn_delta_backward(*x, kept.detach().float().cuda(), do, ds, lengths=given)
    want = torch.autograd.grad(f + (last * ds.cpu().double()).sum(), (*c, S), retain_graph=True, allow_unused=True)
    tol = delta_tol(T, dk, 3)
    for a, b, y, what in zip(got, want, (*c, S), ("dq", "dk", "dv", "dg", "dbeta", "ds0")):
        close(a, torch.zeros_like(y) if b is None else b, tol, what)
    behind = torch.arange(T, device="cuda")[:, None] >= lengths[None, :]
    assert all((a[behind] == 0).all() for a in got[:5])
    if T:
        none = snn.snn_delta_backward(*x, kept.detach().float().cuda(), do, lengths=given)
        for a, b, what in zip(none, torch.autograd.grad(f, (*c, S)), ("dq", "dk", "dv", "dg", "dbeta", "ds0")):
            close(a, b, tol, what + " without ds_last")


@gpu
def test_delta_gradients_are_differences():
    T, B, H, K, dk, dv = 70, 1, 2, 1, 6, 5
    x, s0, do, ds, lengths = delta_inputs(T, B, H, K, dk, dv, torch.float32, seed=3)
    c, S = [clean(a, lengths) for a in x], s0.cpu().double()
    kept = snn.snn_delta_forward(*x, s0, keep=True)[2]
    got = snn.snn_delta_backward(*x, kept, do, ds)

    def f(*a):
        o, last, _ = delta_plain(*a, lengths.cpu(), dk ** -0.5)
        return ((o * do.cpu().double()).sum() + (last * ds.cpu().double()).sum()).item()

    every, d = [*c, S], 1e-5
    for i, a in enumerate(got):
        for at in (0, every[i].numel() // 2, every[i].numel() - 1):
            e = torch.zeros_like(every[i]).flatten()
            e[at] = d
            e = e.view(every[i].shape)
            diff = (f(*every[:i], every[i] + e, *every[i + 1:]) - f(*every[:i], every[i] - e, *every[i + 1:])) / (2 * d)
            # (a third derivative of up to 1e3 gradients times d^2, and 1e-14 of f over d)
            assert abs(diff - a.flatten()[at].item()) <= 1e-5 * max(1.0, a.abs().max().item()), (i, at)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_delta_state_in_place_is_a_sequence_cut_anywhere(dtype):
    x, s0, _, _, lengths = delta_inputs(300, 2, 4, 2, 72, 90, dtype, seed=4)
    whole, last, _ = snn.snn_delta_forward(*x, s0)
    state = s0.clone()
    parts = [snn.snn_delta_forward(*[y[a:b].contiguous() for y in x], state, s_last=state)[0] for a, b in ((0, 1), (1, 2), (2, 20), (20, 100), (100, 300))]
    tol = 2 * delta_tol(300, 72, 1)
    close(torch.cat(parts), whole.cpu(), tol + HALF[dtype], "o")
    close(state, last.cpu(), tol, "state")


@gpu
@pytest.mark.parametrize("T", [1, 100, 1800])
def test_delta_states_in_place(T):
    x, s0, do, ds, lengths = delta_inputs(T, 2, 4, 2, 40, 70, torch.float32, ragged=True, seed=6)
    state = s0.clone()
    got, want = snn.snn_delta_forward(*x, state, lengths=lengths, s_last=state), snn.snn_delta_forward(*x, s0, lengths=lengths, keep=True)
    assert got[1] is state and same(got[:2], want[:2])
    # ds0 in the place of ds_last, by the C entry point
    grads = snn.snn_delta_backward(*x, want[2], do, ds, lengths=lengths)
    p = ops.snn_delta(T, 2, 4, 2, 40, 70, ops.SNN_F32, 40 ** -0.5, lengths=lengths.data_ptr())
    at, space = ops._launch(ds.device, snn.lib().snn_delta_workspace(C.byref(p), 1))
    out, d = [torch.empty_like(y) for y in grads[:5]], ds.clone()
    q, k, v, g, beta = (y.data_ptr() for y in x)
    assert snn.lib().snn_delta_backward(C.byref(at), C.byref(p), q, k, v, g, beta, want[2].data_ptr(), do.data_ptr(), d.data_ptr(),
                                        *[y.data_ptr() for y in out], d.data_ptr()) == 0
    assert same([*out, d], grads)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,H,K,dk,dv", [(6, 3, 3, 40, 40), (150, 4, 2, 24, 40), (300, 2, 2, 128, 128), (1700, 2, 1, 40, 64)])
def test_delta_results_in_the_place_of_inputs(T, H, K, dk, dv, dtype):
    x, s0, do, ds, lengths = delta_inputs(T, 2, H, K, dk, dv, dtype, ragged=True, seed=23)
    want = snn.snn_delta_forward(*x, s0, lengths=lengths, keep=True)
    back = snn.snn_delta_backward(*x, want[2], do, ds, lengths=lengths)
    q, k, v, g, beta = (a.clone() for a in x)
    got = snn.snn_delta_forward(q, k, v, g, beta, s0, lengths=lengths, keep=True, o=v)
    assert got[0] is v and same(got, want)
    v.copy_(x[2])
    got = snn.snn_delta_backward(q, k, v, g, beta, want[2], do, ds, lengths=lengths, dq=q, dk=k, dv=v)
    assert got[0] is q and got[1] is k and got[2] is v and same(got, back)
    # dg and dbeta by the C entry point
    (q, k, v, g, beta), ds0 = (a.clone() for a in x), ds.clone()
    p = ops.snn_delta(T, 2, H, K, dk, dv, ops._type(q, "q"), dk ** -0.5, lengths=lengths.data_ptr())
    at, space = ops._launch(ds.device, snn.lib().snn_delta_workspace(C.byref(p), 1))
    inputs = [a.data_ptr() for a in (q, k, v, g, beta)]
    assert snn.lib().snn_delta_backward(C.byref(at), C.byref(p), *inputs, want[2].data_ptr(), do.data_ptr(), ds0.data_ptr(), *inputs, ds0.data_ptr()) == 0
    assert same([q, k, v, g, beta, ds0], back)


@gpu
def test_delta_refuses_results_in_other_places():
    x, s0, do, ds, _ = delta_inputs(100, 2, 2, 2, 40, 40, torch.float32, seed=24)
    kept, before = snn.snn_delta_forward(*x, s0, keep=True)[2], do.clone()
    wide = torch.zeros((101, 2, 2, 40), device="cuda")
    for call in (lambda: snn.snn_delta_backward(*x, kept, do, ds, dv=do), lambda: snn.snn_delta_backward(*x, kept, do, ds, dq=do),
                 lambda: snn.snn_delta_backward(*x, kept, do, ds, dq=x[1]), lambda: snn.snn_delta_backward(*x, kept, do, ds, dq=wide[1:], dk=wide[:-1]),
                 lambda: snn.snn_delta_forward(*x, s0, o=x[0]), lambda: snn.snn_delta_forward(*x[:2], wide[1:], *x[3:], s0, o=wide[:-1])):
        refused(call, "share elements")
    assert torch.equal(do, before) and (wide == 0).all()


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [5, 150])
def test_delta_parts_of_a_projection(T, dtype):
    B, H, K, dk, dv = 3, 4, 2, 24, 40
    x, s0, do, ds, lengths = delta_inputs(T, B, H, K, dk, dv, dtype, seed=5)
    want = snn.snn_delta_forward(*x, s0, keep=True)
    back = snn.snn_delta_backward(*x, want[2], do, ds)
    sizes = [K * dk, K * dk, H * dv, H * dv, 3]
    wide, grads = (torch.full((T, B, sum(sizes)), math.nan, dtype=dtype, device="cuda") for _ in range(2))
    part = lambda w: [p.view(T, B, n, -1) for p, n in zip(w.split(sizes, -1), (K, K, H, H))]  # noqa: E731
    q, k, v, o = part(wide)
    for to, y in zip((q, k, v), x):
        to.copy_(y)
    assert same(snn.snn_delta_forward(q, k, v, *x[3:], s0, keep=True, o=o), want)
    dq, dk_, dv_, do_ = part(grads)
    do_.copy_(do)
    assert same(snn.snn_delta_backward(q, k, v, *x[3:], want[2], do_, ds, dq=dq, dk=dk_, dv=dv_), back)
    assert torch.isnan(wide[..., -3:]).all() and torch.isnan(grads[..., -3:]).all()


@gpu
def test_delta_lengths_outside_count_as_the_nearer_end():
    for T in (10, 100):
        x, s0, do, ds, _ = delta_inputs(T, 4, 2, 2, 20, 30, torch.float32, seed=6)
        lengths = torch.tensor([-5, T + 7, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device="cuda")
        inside = torch.tensor([0, T, T, 0], dtype=torch.int32, device="cuda")
        got, want = (snn.snn_delta_forward(*x, s0, lengths=v, keep=True) for v in (lengths, inside))
        assert same(got, want) and same(*(snn.snn_delta_backward(*x, want[2], do, ds, lengths=v) for v in (lengths, inside)))


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [12, 200])
def test_delta_equal_keys(T, dtype):
    # one key again and again with beta = 1: a step writes over what the last one wrote, and reads its own value
    x, s0, _, _, lengths = delta_inputs(T, 2, 2, 2, 32, 48, dtype, seed=7)
    key = torch.zeros(32, dtype=dtype, device="cuda")
    key[:4] = 0.5
    x[0][:], x[1][:] = key, key
    x[3].zero_()
    x[4].fill_(1.0)
    o, last, _ = snn.snn_delta_forward(*x, None, scale=1.0)
    # differences of neighbouring values, each off by a few roundings
    near(o, x[2].cpu(), (16 * U if dtype == torch.float32 else 16 * U + 2.0 ** -16) * 2 * x[2].cpu().double().abs().max(), "o")


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [20, 250])
def test_delta_small_values_in_the_place_of_large_ones(T, dtype):
    # beta = 1 and keys that do not meet: each step reads its own value, as the difference of what was held and what is taken from it
    x, _, _, _, _ = delta_inputs(T, 2, 2, 2, 32, 48, dtype, seed=21)
    x[0][:] = x[1][:] = torch.eye(32, device="cuda")[torch.arange(T) % 32][:, None, None]
    x[3].zero_()
    x[4].fill_(1.0)
    s0 = 4096 * torch.randn((2, 2, 32, 48), generator=torch.Generator().manual_seed(22)).cuda()
    x[2][:T // 2] *= 512
    o = snn.snn_delta_forward(*x, s0, scale=1.0)[0]
    held = max(s0.abs().max().item(), x[2].abs().max().item())
    near(o, x[2].cpu(), 16 * U * held, "o")


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_delta_gates_at_their_ends(dtype):
    # decays that forget all (minus infinity, and sums of them that 32 bits would round), none at all, beta 0 and 1
    T = 150
    x, s0, do, ds, lengths = delta_inputs(T, 2, 3, 3, 40, 40, dtype, seed=8)
    g, beta = x[3], x[4]
    g[::7] = -60.0
    g[30], g[100, 0] = -math.inf, -math.inf
    g[5:9], g[70:90] = 0.0, -1e-4
    beta[::3], beta[1::5] = 0.0, 1.0
    o, last, kept = snn.snn_delta_forward(*x, s0, keep=True)
    c = [clean(a, lengths) for a in x]
    tol = delta_tol(T, 40, 1)
    want = delta_plain(*c, s0.cpu().double(), lengths.cpu(), 40 ** -0.5)
    close(o, want[0], tol, "o")
    close(last, want[1], tol, "last")
    c[3] = c[3].clamp(min=-1e4)  # (exp of it is 0; the gradient of minus infinity would be 0 times infinity)
    c = [a.requires_grad_() for a in c]
    S = s0.cpu().double().requires_grad_()
    o, last, _ = delta_plain(*c, S, lengths.cpu(), 40 ** -0.5)
    want = torch.autograd.grad((o * do.cpu().double()).sum() + (last * ds.cpu().double()).sum(), (*c, S))
    for a, b, what in zip(snn.snn_delta_backward(*x, kept, do, ds), want, ("dq", "dk", "dv", "dg", "dbeta", "ds0")):
        close(a, b, 3 * tol, what)


@gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("K,dk,dv", [(7, 40, 40), (1, 40, 70), (7, 100, 33), (1, 128, 64)])
def test_delta_gradients_of_gates_behind_strong_decays(K, dk, dv, dtype):
    # What goes past a decay is all that its gate's gradient is made of, however little that is beside what was written before it and read after it: heads that
    # forget nearly all at every step, and single strong decays among mild ones, each compared to its own size.
    T, H = 200, 7
    x, s0, do, ds, lengths = delta_inputs(T, 1, H, K, dk, dv, dtype, seed=20)
    g, strong = x[3], [-5.0, -10.0, -20.0, -60.0, -20.0, -30.0]
    for h in range(4):
        g[:, 0, h] = strong[h]
    g[::9, 0, 4] = strong[4]
    g[[63, 64, 100, 101, 150], 0, 5] = strong[5]
    kept = snn.snn_delta_forward(*x, s0, keep=True)[2]
    c = [clean(a, lengths).requires_grad_() for a in x]
    S = s0.cpu().double().requires_grad_()
    o, last, _ = delta_plain(*c, S, lengths.cpu(), dk ** -0.5)
    want = torch.autograd.grad((o * do.cpu().double()).sum() + (last * ds.cpu().double()).sum(), (c[3], c[4]))
    got = snn.snn_delta_backward(*x, kept, do, ds)[3:5]
    for a, b, what in zip(got, want, ("dg", "dbeta")):
        for h in range(H):
            # (the exponent of a decay has 24 bits: the decay is off by |g| U, and twice that by its multiplication with log2 e)
            at = g[:, 0, h] < -4.9
            for part in (at, ~at):
                off = 2 * U * -strong[h] if h < 6 and part is at else 0
                close(a[part, 0, h], b[part.cpu(), 0, h], delta_tol(T, dk, 3) + off, (what, h))


@gpu
@pytest.mark.parametrize("T", [4, 90, 2000])
def test_delta_values_that_are_not_finite_stay_in_their_heads(T):
    x, s0, do, ds, _ = delta_inputs(T, 3, 4, 2, 20, 30, torch.float32, seed=9)
    want = snn.snn_delta_forward(*x, s0, keep=True)
    back = snn.snn_delta_backward(*x, want[2], do, ds)
    x[2][2, 1, 3, 4] = math.nan
    s0[0, 2, 3, 5] = math.inf
    got = snn.snn_delta_forward(*x, s0, keep=True)
    bad = torch.zeros(3, 4, dtype=torch.bool, device="cuda")
    bad[1, 3] = bad[0, 2] = True
    assert torch.equal(got[0][:, ~bad], want[0][:, ~bad]) and torch.equal(got[1][~bad], want[1][~bad])
    assert not torch.isfinite(got[1][1, 3, :, 4]).any()
    grads = snn.snn_delta_backward(*x, got[2], do, ds)
    keys = ~bad.view(3, 2, 2).any(2)
    assert all(torch.equal(a[:, keys], b[:, keys]) for a, b in zip(grads[:2], back[:2]))
    assert all(torch.equal(a[:, ~bad], b[:, ~bad]) for a, b in zip(grads[2:5], back[2:5])) and torch.equal(grads[5][~bad], back[5][~bad])


@gpu
def test_delta_no_gradient_behind_an_end_whatever_that_of_the_state():
    x, s0, do, ds, _ = delta_inputs(100, 2, 2, 2, 20, 30, torch.float32, seed=10)
    lengths = torch.tensor([70, 0], dtype=torch.int32, device="cuda")
    kept = snn.snn_delta_forward(*x, s0, lengths=lengths, keep=True)[2]
    ds[:, 0] = math.inf
    grads = snn.snn_delta_backward(*x, kept, do, ds, lengths=lengths)
    assert all((a[70:, 0] == 0).all() and (a[:, 1] == 0).all() for a in grads[:5]) and torch.equal(grads[5][1], ds[1])


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_delta_pieces_of_long_sequences(dtype):
    # more than the workspace holds at once: the same bits as calls for parts of the sequence, which fit
    T, B, H = 64 * 160, 2, 32
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *x: torch.randn(x, generator=g, device="cuda")  # noqa: E731
    q, k = (torch.nn.functional.normalize(rand(T, B, H, 128), dim=-1).to(dtype) for _ in range(2))
    x = [q, k, rand(T, B, H, 64).to(dtype), -0.1 * rand(T, B, H).abs(), torch.sigmoid(rand(T, B, H))]
    do, ds = rand(T, B, H, 64).to(dtype), rand(B, H, 128, 64)
    p = ops.snn_delta(T, B, H, H, 128, 64, ops.SNN_BF16 if dtype == torch.bfloat16 else ops.SNN_F32, 1.0)
    half = ops.snn_delta(512, B, H, H, 128, 64, p.dtype, 1.0)
    size = snn.lib().snn_delta_workspace
    assert size(C.byref(p), 0) < 20 * size(C.byref(half), 0) and size(C.byref(p), 1) < 20 * size(C.byref(half), 1)
    o, last, kept = snn.snn_delta_forward(*x, keep=True)
    grads = snn.snn_delta_backward(*x, kept, do, ds)
    cuts = list(range(0, T, 512))
    state = None
    for a in cuts:
        part = [y[a:a + 512] for y in x]
        oo, state, kk = snn.snn_delta_forward(*part, state, keep=True)
        assert torch.equal(oo, o[a:a + 512]) and torch.equal(kk, kept[a // 256:a // 256 + 2]), a
    assert torch.equal(state, last)
    for a in reversed(cuts):
        part = snn.snn_delta_backward(*[y[a:a + 512] for y in x], kept[a // 256:a // 256 + 2].contiguous(), do[a:a + 512], ds)
        ds = part[5]
        assert same(part[:5], [y[a:a + 512] for y in grads[:5]]), a
    assert torch.equal(ds, grads[5])


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_delta_ends_in_any_piece(dtype):
    # a sequence that ends long before the others: the same bits as if they all ended there, whatever piece that is in
    T, B, H = 64 * 160, 2, 32
    g = torch.Generator(device="cuda").manual_seed(5)
    rand = lambda *x: torch.randn(x, generator=g, device="cuda")  # noqa: E731
    q, k = (torch.nn.functional.normalize(rand(T, B, H, 128), dim=-1).to(dtype) for _ in range(2))
    x = [q, k, rand(T, B, H, 64).to(dtype), -0.1 * rand(T, B, H).abs(), torch.sigmoid(rand(T, B, H))]
    do, ds = rand(T, B, H, 64).to(dtype), rand(B, H, 128, 64)
    for n in (70, 64 * 128, 64 * 150 + 1):
        lengths = torch.tensor([T, n], dtype=torch.int32, device="cuda")
        for y in (*x, do):
            y[n:, 1] = math.nan
        o, last, kept = snn.snn_delta_forward(*x, lengths=lengths, keep=True)
        grads = snn.snn_delta_backward(*x, kept, do, ds, lengths=lengths)
        short = [y[:n] for y in x]
        want = snn.snn_delta_forward(*short, keep=True)
        back = snn.snn_delta_backward(*short, want[2], do[:n], ds)
        of_one = lambda a: a[:, 1]  # noqa: E731
        assert same(map(of_one, (o[:n], kept[:len(want[2])], *(y[:n] for y in grads[:5]))), map(of_one, (want[0], want[2], *back[:5]))), n
        assert torch.equal(last[1], want[1][1]) and torch.equal(grads[5][1], back[5][1])
        assert all((y[n:, 1] == 0).all() for y in (o, *grads[:5])) and (kept[len(want[2]):, 1] == last[1]).all()
        assert all(torch.isfinite(y).all() for y in (o, last, *grads))
        for y in (*x, do):  # (the next end is further on)
            y[n:, 1] = y[n:, 0]


@gpu
@pytest.mark.parametrize("dtype,chunks", [(torch.float32, 700), (torch.bfloat16, 1500)])
def test_delta_segments_of_pieces(dtype, chunks):
    # few heads and more steps than the workspace holds at once: pieces, whose walks take segments side by side.  Calls for parts of 20 chunks, which have one
    # segment and one piece, sum in another order
    T, H, dk, dv, part = 64 * chunks + 17, 16, 128, 64, 1280
    g = torch.Generator(device="cuda").manual_seed(7)
    rand = lambda *x: torch.randn(x, generator=g, device="cuda")  # noqa: E731
    q, k = (torch.nn.functional.normalize(rand(T, 1, H, dk), dim=-1).to(dtype) for _ in range(2))
    x = [q, k, rand(T, 1, H, dv).to(dtype), -0.02 * rand(T, 1, H).abs(), torch.sigmoid(rand(T, 1, H))]
    do, s0, ds = rand(T, 1, H, dv).to(dtype), rand(1, H, dk, dv), rand(1, H, dk, dv)
    size = lambda n, back: snn.lib().snn_delta_workspace(C.byref(ops.snn_delta(n, 1, H, H, dk, dv, ops._type(q, "q"), 1.0)), back)  # noqa: E731
    assert all(size(T, back) < 0.8 * chunks / 100 * size(6400, back) for back in (0, 1))
    o, last, kept = snn.snn_delta_forward(*x, s0, keep=True)
    grads = snn.snn_delta_backward(*x, kept, do, ds)
    tol = 2 * delta_tol(T, dk, 1)
    off = lambda a: HALF[dtype] if a.dtype == dtype else 0  # noqa: E731  (both are rounded)
    cuts, state = list(range(0, T, part)), s0
    for a in cuts:
        oo, state, kk = snn.snn_delta_forward(*[y[a:a + part] for y in x], state, keep=True)
        close(o[a:a + part], oo.cpu(), tol + off(oo), ("o", a))
        close(kept[a // 256:(a + part) // 256], kk.cpu(), tol, ("kept", a))
    close(last, state.cpu(), tol, "last")
    for a in reversed(cuts):
        back = snn.snn_delta_backward(*[y[a:a + part] for y in x], kept[a // 256:(a + part) // 256].contiguous(), do[a:a + part], ds)
        ds = back[5]
        for y, z, what in zip(grads, back[:5], ("dq", "dk", "dv", "dg", "dbeta")):
            close(y[a:a + part], z.cpu(), 3 * tol + off(z), (what, a))
    close(grads[5], ds.cpu(), 3 * tol, "ds0")


@gpu
def test_delta_beyond_4_gb():
    T, B, H, dv = 32768 + 16, 8, 64, 128  # 2^31 elements and more of v, of o
    g = torch.Generator(device="cuda").manual_seed(4)
    q, k = (torch.nn.functional.normalize(torch.randn((T, B, 1, 32), generator=g, device="cuda"), dim=-1).bfloat16() for _ in range(2))
    v = torch.empty((T, B, H, dv), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    gates = -0.2 * torch.rand((T, B, H), generator=g, device="cuda")
    beta = torch.rand((T, B, H), generator=g, device="cuda")
    x = [q, k, v, gates, beta]
    o, last, _ = snn.snn_delta_forward(*x)
    # the last 16 steps by themselves, from a state 500 steps back: nothing that is older is left of it
    first = [y[T - 516:T - 16] for y in x]
    state = snn.snn_delta_forward(*first)[1]
    end, state, _ = snn.snn_delta_forward(*[y[T - 16:] for y in x], state)
    tol = 2 * delta_tol(500, 32, 1)
    close(o[T - 16:], end.cpu(), tol + HALF[torch.bfloat16], "o")
    close(last, state.cpu(), tol, "last")


@gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_delta_token_of_a_large_batch(dtype):
    # more than 2^25 bytes of v: the same bits as for parts of the batch
    B, H, K, dk, dv = 1 << 15, 16, 2, 8, 64
    g = torch.Generator(device="cuda").manual_seed(6)
    rand = lambda *x: torch.randn(x, generator=g, device="cuda")  # noqa: E731
    x = [rand(1, B, K, dk).to(dtype), rand(1, B, K, dk).to(dtype), rand(1, B, H, dv).to(dtype), -rand(1, B, H).abs(), torch.sigmoid(rand(1, B, H))]
    state = rand(B, H, dk, dv)
    o, last, _ = snn.snn_delta_forward(*x, state)
    for at in range(0, B, B // 4):
        at = slice(at, at + B // 4)
        part = snn.snn_delta_forward(*[y[:, at] for y in x], state[at])
        assert torch.equal(part[0], o[:, at]) and torch.equal(part[1], last[at])
    # and rows that are far apart
    wide = torch.full((1, 3, 1 << 24), 7.0, dtype=dtype, device="cuda")
    n = H * dv
    q, k, v, to = (wide[..., i * n:i * n + w * c].unflatten(-1, (w, c)) for i, (w, c) in enumerate(((K, dk), (K, dk), (H, dv), (H, dv))))
    for y, z in zip((q, k, v), x):
        y.copy_(z[:, :3])
    got = snn.snn_delta_forward(q, k, v, x[3][:, :3], x[4][:, :3], state[:3], o=to)
    assert torch.equal(to, o[:, :3]) and torch.equal(got[1], last[:3]) and (wide[..., 4 * n:] == 7).all()


@gpu
@pytest.mark.parametrize("T", [1, 100, 1600])
def test_delta_in_a_graph(T):
    x, s0, do, ds, lengths = delta_inputs(T, 3, 4, 2, 40, 50, torch.bfloat16, ragged=T > 1, seed=11)
    state = s0.clone()

    def run():
        o, last, kept = snn.snn_delta_forward(*x, state, lengths=lengths, keep=True)
        return o, last, kept, *snn.snn_delta_backward(*x, kept, do, ds, lengths=lengths)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(3):
        state.mul_(0.5)
        x[2].mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        assert same(got, run())


@gpu
def test_delta_on_another_stream_and_from_two_threads():
    import threading
    cases = [delta_inputs(200, 2, 4, 4, 64, 64, torch.bfloat16, seed=s) for s in (12, 13)]

    def run(case):
        x, s0, do, ds, _ = case
        o, last, kept = snn.snn_delta_forward(*x, s0, keep=True)
        return o, last, *snn.snn_delta_backward(*x, kept, do, ds)

    want, got = [run(c) for c in cases], [None, None]
    torch.cuda.synchronize()

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(10):
                got[i] = run(cases[i])
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert all(same(a, b) for a, b in zip(got, want))


# ---- all of them together -------------------------------------------------------------------------
@gpu
def test_a_model_of_norms_delta_rule_and_vocabulary_takes_a_step():
    T, B, H, dk, dv, d, vocab = 80, 2, 2, 16, 24, 40, 101
    g = torch.Generator().manual_seed(5)
    rand = lambda *x: torch.randn(x, generator=g)  # noqa: E731
    sizes = [H * dk, H * dk, H * dv, H, H]
    params = [p.cuda() for p in (rand(vocab, d), 1 + 0.1 * rand(d), rand(d, sum(sizes)) / d ** 0.5, rand(H * dv, d) / 7, 1 + 0.1 * rand(d))]
    tokens = torch.randint(0, vocab, (T + 1, B), generator=g).cuda()
    targets = tokens[1:].flatten().int()

    def gates(z):
        q, k, v, a, b = z.split(sizes, -1)
        q, k = (torch.nn.functional.normalize(y.unflatten(-1, (H, dk)), dim=-1) for y in (q, k))
        return q, k, v.unflatten(-1, (H, dv)), -torch.nn.functional.softplus(a), torch.sigmoid(b)

    def plain(table, w1, up, down, w2):
        norm = lambda s, w: w * s / torch.sqrt((s * s).mean(-1, keepdim=True) + 1e-6)  # noqa: E731
        x = table[tokens[:-1].cpu()]
        o = delta_plain(*gates(norm(x, w1) @ up), torch.zeros(B, H, dk, dv, dtype=torch.float64), torch.full((B,), T), dk ** -0.5)[0]
        y = norm(x + o.flatten(2) @ down, w2).flatten(0, 1)
        return torch.nn.functional.cross_entropy(y @ table.T, targets.cpu().long())

    # the library's calls, and torch for the products between
    table, w1, up, down, w2 = params
    x = table[tokens[:-1]]
    y1, _ = snn.snn_norm_forward(x, w1)
    z = (y1 @ up).requires_grad_()
    layer = gates(z)
    held = [y.detach().contiguous() for y in layer]
    o, _, kept = snn.snn_delta_forward(*held, keep=True)
    y2, total = snn.snn_norm_forward(o.flatten(2) @ down, w2, residual=x)
    loss, state = snn.snn_vocab_loss(y2.flatten(0, 1), table, targets)
    dy2, dtable = snn.snn_vocab_loss_grad(y2.flatten(0, 1), table, targets, state)
    dtotal, dw2 = snn.snn_norm_backward(total, w2, dy2.view_as(total))
    ddown = o.flatten(2).flatten(0, 1).T @ dtotal.flatten(0, 1)
    back = snn.snn_delta_backward(*held, kept, (dtotal @ down.T).view_as(o))
    dz, = torch.autograd.grad(layer, z, back[:5])
    dup = y1.flatten(0, 1).T @ dz.flatten(0, 1)
    dx, dw1 = snn.snn_norm_backward(x, w1, dz @ up.T, dtotal=dtotal)
    dtable = dtable.index_add(0, tokens[:-1].flatten(), dx.flatten(0, 1))
    grads = [dtable, dw1, dup, ddown, dw2]
    double = [p.cpu().double().requires_grad_() for p in params]
    want = plain(*double)
    assert abs(loss.double().mean().item() - want.item()) <= 2e-5 * want.item()  # (the root mean square of its logits' errors is 1e-6)
    reference = torch.autograd.grad(want, double)
    for a, b, what in zip(grads, reference, ("table", "w1", "up", "down", "w2")):
        close(a, b, 3 * delta_tol(T, d, 3), what)
    # and the step that they make
    plan = snn.snn_adamw_plan(params, *snn.snn_adamw_moments(params))
    before = [p.cpu().double() for p in params]
    snn.snn_adamw_step(plan, grads, 1, lr=1e-2)
    for p, x, a in zip(params, before, grads):
        want = adamw_plain(x, a.cpu().double(), 0 * x, 0 * x, 1, 1e-2, (0.9, 0.999), 1e-8, 0.01)
        near(p, want[0], want[3], "step")


# ---- refusals -----------------------------------------------------------------------------------
def refused(call, text):
    with pytest.raises(snn.SnnError) as e:
        call()
    assert e.value.status == snn.SNN_E_INVAL and text in str(e.value), str(e.value)


def test_c_entry_points_of_norm_and_adamw_refuse_what_they_cannot_run():
    L, at = snn.lib(), ops.snn_launch(0, None, None, 0)
    here = C.cast(C.create_string_buffer(4096), C.c_void_p).value

    def norm(**k):
        return C.byref(ops.snn_norm(**{**dict(rows=4, n=8, dtype=0, eps=1e-6), **k}))

    for name, count in (("snn_norm_forward", 5), ("snn_norm_forward_packed", 6), ("snn_norm_backward", 6)):
        def call(p, launch=C.byref(at), first=here):
            ops._run(name, launch, p, first, *[here] * (count - 1))
        refused(lambda: call(norm(), None), "no device")
        refused(lambda: call(None), "no shape")
        refused(lambda: call(norm(dtype=2)), "unknown type 2")
        for bad in (dict(n=0), dict(n=32769), dict(rows=-1), dict(rows=1 << 40)):
            refused(lambda: call(norm(**bad)), "2^15")
        for bad in (-1.0, math.nan, math.inf):
            refused(lambda: call(norm(eps=bad)), "eps")
        refused(lambda: call(norm(ld_dx=7)), "7 elements")
        refused(lambda: call(norm(), first=None), "is NULL")
        refused(lambda: call(norm(), first=here + 2), "not aligned")
        refused(lambda: call(norm()), "not in")
    assert L.snn_norm_workspace(norm(n=0)) == 0 and L.snn_norm_workspace(norm()) > 0

    def adamw(**k):
        return C.byref(ops.snn_adamw(**{**dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=1), **k}))

    def step(how, launch=C.byref(at), count=1, **k):
        t = ops.snn_adamw_tensor(**{**dict(p=here, g=here, m=here, v=here, n=8), **k})
        ops._run("snn_adamw_step", launch, how, C.byref(t), count)

    refused(lambda: step(adamw(), None), "no device")
    refused(lambda: step(None), "no step")
    refused(lambda: step(adamw(), count=-1), "no tensors")
    for bad in (dict(lr=math.nan), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(weight_decay=math.inf)):
        refused(lambda: step(adamw(**bad)), "betas")
    refused(lambda: step(adamw(step=0)), "the first one is 1")
    refused(lambda: step(adamw(), n=-1), "-1 elements")
    refused(lambda: step(adamw(), dtype_g=3), "unknown type")
    refused(lambda: step(adamw(), m_exps=here), "one without")
    refused(lambda: step(adamw(), copy=here, dtype_p=1), "copy")
    refused(lambda: step(adamw(), p=None), "p is NULL")
    refused(lambda: step(adamw()), "not in")
    assert L.snn_adamw_workspace(adamw()) == 0 < L.snn_adamw_workspace(adamw(step_on_device=here))


def test_binding_of_norm_and_adamw_refuses_tensors_that_do_not_fit():
    f, b = torch.zeros, torch.bfloat16
    m, v = snn.snn_adamw_moments([f(40)], 8)
    assert m[0].codes.shape == (40,) and v[0].exps.shape == (2,) and [x.shape for x in snn.snn_adamw_moments([f(3, 5)])[0]] == [(3, 5)]
    plan = snn.snn_adamw_plan([f(40)], m, v)
    for call, kind in (
            (lambda: snn.snn_norm_forward(f(4, 8)), ValueError),                                # on the CPU
            (lambda: snn.snn_norm_forward(f(())), ValueError),
            (lambda: snn.snn_norm_forward(f(4, 8, dtype=torch.float16)), TypeError),
            (lambda: snn.snn_norm_forward(f(4, 8), f(8, dtype=b)), TypeError),
            (lambda: snn.snn_norm_forward(f(4, 8), f(7)), ValueError),
            (lambda: snn.snn_norm_forward(f(4, 8), residual=f(4, 7)), ValueError),
            (lambda: snn.snn_norm_forward(f(4, 8), residual=f(8, 4).T), ValueError),
            (lambda: snn.snn_norm_forward(f(4, 8), total=f(4, 8)), ValueError),
            (lambda: snn.snn_norm_backward(f(4, 8), f(8), f(4, 9)), ValueError),
            (lambda: snn.snn_norm_backward(f(4, 8), f(8), f(4, 8), dtotal=f(4, 8, dtype=b)), TypeError),
            (lambda: snn.snn_adamw_moments([f(4)], 16), ValueError),
            (lambda: snn.snn_adamw_plan([f(4)], [f(4)], []), ValueError),
            (lambda: snn.snn_adamw_plan([f(4)], [f(5)], [f(4)]), ValueError),
            (lambda: snn.snn_adamw_plan([f(4)], [f(4, dtype=b)], [f(4)]), TypeError),
            (lambda: snn.snn_adamw_plan([f(40)], m, [f(40)]), TypeError),
            (lambda: snn.snn_adamw_plan([f(41)], m, v), ValueError),
            (lambda: snn.snn_adamw_plan([f(40)], [snn.Packed(m[0].codes, f(1, dtype=torch.uint8))], v), ValueError),
            (lambda: snn.snn_adamw_plan([f(4, dtype=b)], [f(4)], [f(4)], [f(4, dtype=b)]), TypeError),
            (lambda: snn.snn_adamw_plan([f(4, 4).T[:2]], [f(2, 4)], [f(2, 4)]), ValueError),
            (lambda: snn.snn_adamw_step(plan, [], 1), ValueError),
            (lambda: snn.snn_adamw_step(plan, [f(40, dtype=torch.float64)], 1), TypeError),
            (lambda: snn.snn_adamw_step(plan, [f(39)], 1), ValueError),
            (lambda: snn.snn_adamw_step(plan, [f(80)[::2]], 1), ValueError),
            (lambda: snn.snn_adamw_step(plan, [f(40)], f(1)), TypeError),
            (lambda: snn.snn_adamw_step(plan, [f(40)], 1), ValueError)):                        # on the CPU
        with pytest.raises(kind):
            call()


def test_a_plan_is_of_the_memory_that_its_tensors_had():
    import weakref
    p = torch.nn.Parameter(torch.zeros(40))
    m, v = snn.snn_adamw_moments([p])
    plan = snn.snn_adamw_plan([p], m, v)
    old = plan.memory[0]
    assert old.data_ptr() == p.data_ptr() == plan.tensors[0].p
    p.data = torch.ones(40)
    assert (old == 0).all() and old.data_ptr() == plan.tensors[0].p
    with pytest.raises(ValueError, match="other memory"):
        snn.snn_adamw_step(plan, [torch.zeros(40)], 1)
    held = weakref.ref(plan.memory[0])
    del old, plan
    assert held() is None


@pytest.mark.parametrize("bits,which,name", [(32, "m", "m"), (32, "v", "v"), (8, "m.codes", "the codes of m"), (8, "m.exps", "the exponents of m"),
                                             (8, "v.codes", "the codes of v"), (8, "v.exps", "the exponents of v"), (8, "copies", "copies"), (32, "params", "params")])
def test_a_plan_is_of_the_memory_that_its_moments_and_copies_had(bits, which, name):
    params = [torch.zeros(40), torch.zeros(0), torch.zeros(3, 50)]
    m, v = snn.snn_adamw_moments(params, bits)
    copies = [None, None, torch.zeros(3, 50, dtype=torch.bfloat16)]
    plan = snn.snn_adamw_plan(params, m, v, copies)
    x, part = dict(m=m, v=v, copies=copies, params=params)[which.split(".")[0]][2], which.split(".")[1:]
    x = getattr(x, part[0]) if part else x
    old, grads = x.detach(), [torch.zeros_like(p) for p in params]
    with pytest.raises(ValueError, match="run on a GPU"):
        snn.snn_adamw_step(plan, grads, 1)  # (as far as it comes here)
    x.data = x.clone()  # moments that were loaded, say
    with pytest.raises(ValueError, match=rf"^{name}\[2\] has other memory"):
        snn.snn_adamw_step(plan, grads, 1)
    x.data = old
    with pytest.raises(ValueError, match="run on a GPU"):
        snn.snn_adamw_step(plan, grads, 1)


def test_c_entry_points_of_the_delta_rule_refuse_what_they_cannot_run():
    L, at = snn.lib(), ops.snn_launch(0, None, None, 0)
    here = C.cast(C.create_string_buffer(4096), C.c_void_p).value

    def shape(**k):
        return C.byref(ops.snn_delta(**{**dict(T=20, batch=2, heads=4, key_heads=2, dk=8, dv=8, dtype=0, scale=1.0), **k}))

    for name, count in (("snn_delta_forward", 9), ("snn_delta_backward", 14)):
        def call(p, launch=C.byref(at), first=here):
            ops._run(name, launch, p, first, *[here] * (count - 1))
        refused(lambda: call(shape(), None), "no device")
        refused(lambda: call(None), "no shape")
        refused(lambda: call(shape(dtype=2)), "unknown type 2")
        refused(lambda: call(shape(T=-1)), "T = -1")
        for bad in (dict(key_heads=3), dict(heads=0), dict(key_heads=0), dict(key_heads=-2)):
            refused(lambda: call(shape(**bad)), "multiple")
        for bad in (dict(dk=0), dict(dk=129), dict(dv=0), dict(dv=1025)):
            refused(lambda: call(shape(**bad)), "1024")
        for bad in (dict(batch=0), dict(batch=1 << 20), dict(batch=1 << 17, dv=1024)):
            refused(lambda: call(shape(**bad)), "2^20")
        refused(lambda: call(shape(scale=math.inf)), "scale")
        for bad in (dict(ld_q=15), dict(ld_v=31), dict(ld_dv=-1), dict(ld_o=(1 << 22) + 1), dict(batch=1 << 18, dv=16)):
            refused(lambda: call(shape(**bad)), "elements from row to row")
        refused(lambda: call(shape(), first=None), "q is NULL")
        refused(lambda: call(shape(), first=here + 2), "not aligned")
        refused(lambda: call(shape()), "not in")
    assert L.snn_delta_workspace(shape(dk=0), 0) == 0 and L.snn_delta_workspace(shape(), 1) > L.snn_delta_workspace(shape(), 0) > 0
    assert L.snn_delta_workspace(shape(T=1), 0) == 0


def test_binding_of_the_delta_rule_refuses_tensors_that_do_not_fit():
    f = torch.zeros
    x = dict(q=f(4, 2, 2, 8), k=f(4, 2, 2, 8), v=f(4, 2, 4, 6), g=f(4, 2, 4), beta=f(4, 2, 4))
    wide = f(4, 2, 2, 16)[..., ::2]
    for change, kind in ((dict(), ValueError), (dict(q=f(4, 2, 16)), ValueError), (dict(k=f(4, 2, 2, 7)), ValueError), (dict(v=f(4, 3, 4, 6)), ValueError),
                         (dict(v=f(4, 2, 4, 6, dtype=torch.bfloat16)), TypeError), (dict(g=f(4, 2, 2)), ValueError),
                         (dict(beta=f(4, 2, 4, dtype=torch.bfloat16)), TypeError), (dict(q=wide), ValueError), (dict(k=f(4, 2, 2, 16)[..., :8]), ValueError),
                         (dict(q=f(2, 4, 2, 8).transpose(0, 1)), ValueError), (dict(s0=f(2, 4, 6, 8)), ValueError), (dict(s_last=f(2, 4, 8, 5)), ValueError),
                         (dict(lengths=f(2)), TypeError), (dict(o=f(4, 2, 4, 7)), ValueError)):
        with pytest.raises(kind):
            snn.snn_delta_forward(**{**x, **change})
    for change, kind in ((dict(), ValueError), (dict(kept=f(2, 2, 4, 8, 6)), ValueError), (dict(do=f(4, 2, 4, 5)), ValueError),
                         (dict(ds_last=f(2, 4, 8, 6, dtype=torch.float64)), TypeError), (dict(dk=f(4, 2, 2, 9)), ValueError)):
        with pytest.raises(kind):
            snn.snn_delta_backward(**{**x, **dict(kept=f(1, 2, 4, 8, 6), do=f(4, 2, 4, 6)), **change})
