"""Dropout, root-mean-square norms and gated blocks at the ends of what their arguments may be.

U is half a step of fp32 relative to the value, HALF half a step of the storage type."""
import math

import pytest
import torch

from tests.layers_util import ACTS, DEV, HALF, U, Act, Model, act64, dtype_of, generator, within, workspace

pytestmark = pytest.mark.gpu


# ---- activations at every size of their argument ---------------------------------------------------------------------------
SIZES = [0.0, 1e-30, 1e-3, 0.3, 1.0, 2.5, 5.0, 12.0, 30.0, 200.0, 1e4, 1e9, 1e12, 1.2e13, 1e15, 1e18, 2e19, 1e25, 1e38, 3e38]


def _slopes(act, storage, values):
    """(f, slope) of the values, from a backward pass whose gate's weight is 1 and whose up's is 0: dx = dg, and dWu = du^T x with x = 1."""
    n = len(values)
    m = Model(1, [(8, 8), (8, 8)], storage, generator(0))
    m.w[0][1].copy_(torch.eye(8, device=DEV).to(m.dt))
    m.w[1][1].zero_()
    rows = [n]
    x, g, u, da, dx = (Act(rows, 8, m.dt) for _ in range(5))
    for t in (x, u, da):
        t[0].fill_(1.0)
    g[0].copy_(torch.tensor(values, device=DEV, dtype=torch.float32).to(m.dt)[:, None].expand(n, 8))
    work = workspace(m.ctx.gated_backward_bytes(0, 1, rows, 8))
    m.ctx.gated_backward(0, 1, rows, 8, x.at, g.at, u.at, da.at, dx.at, activation=ACTS[act], accumulate=False, workspace=work.data_ptr(),
                         workspace_bytes=work.numel())
    torch.cuda.synchronize()
    out = g[0][:, 0].double(), dx[0].double()
    m.close()
    return out


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("act", list(ACTS))
def test_slopes_of_large_arguments(act, storage):
    """From 200 on the slope is 1 or 0 to the bit: what is left of it, e^-200 of the argument, is below fp32's least value. Below, 16 roundings of the slope's
    terms, each at most 1 + |g|, and one to the storage type."""
    g, slope = _slopes(act, storage, SIZES + [-v for v in SIZES])
    want = act64(act, g)[1]
    want = torch.where(g.abs() > 150.0, (g > 0).double(), want)
    bound = torch.where(g.abs() > 150.0, 0.0, 16 * U * (1 + g.abs()) + HALF[dtype_of(storage)] * want.abs())
    for j in range(8):
        within(slope[:, j], want, bound, (act, j))


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_small_values_of_an_activation_keep_their_bits(act):
    """a = f(v) for v = -12 to -0.01, in fp32, within roundings of the VALUE: forms that subtract from 1 lose all of it.

    The value goes with exp(-|z|), z being v, v^2 / 2 or sqrt(8 / pi) (v + 0.044715 v^3): a relative error d of z's own is |z| d of the value. z is made in
    six roundings at most (0.044715, that times v, times v again, the sum, sqrt(8 / pi), the product; gelu: v / sqrt(2) in two, and erfc moves 2 x^2 + 1
    times as much as x does, which is less than six times v^2 / 2 + 1). 24 for the exponential or erfc (a few steps of 2 U), the division and the products.
    A factor 1 / (1 + exp(-z)) below 2^-126, fp32's least normal number, may be off by as much as it is."""
    values = [-12.0 + 0.0625 * i for i in range(192)]
    m = Model(1, [(8, 8), (8, 8)], "f32", generator(0))
    m.w[0][1].zero_(), m.w[1][1].zero_()
    m.w[0][1][0, :, 0] = 1.0                                 # g = x[0]
    m.w[1][1][0, :, 1] = 1.0                                 # u = x[1]
    rows = [len(values)]
    x, a = Act(rows, 8, m.dt), Act(rows, 8, m.dt)
    x[0].zero_()
    x[0][:, 0] = torch.tensor(values, device=DEV)
    x[0][:, 1] = 1.0
    m.ctx.gated(0, 1, rows, 8, x.at, a.at, activation=ACTS[act])
    torch.cuda.synchronize()
    v = x[0][:, 0].double()
    if act == "silu":
        want, moves = v * torch.sigmoid(v), v.abs()
    elif act == "gelu":
        want, moves = 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0)), v * v / 2 + 1
    else:
        z = math.sqrt(8 / math.pi) * (v + 0.044715 * v ** 3)
        want, moves = v * torch.sigmoid(z), z.abs()
    for j in range(8):
        within(a[0][:, j], want, (24 + 6 * moves) * U * want.abs() + v.abs() * 2.0 ** -126, (act, j))
    m.close()


# ---- rows that overlap ----------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,stride", [([40, 37], 8), ([70, 1], 0), ([50, 33], 56), ([1, 1], 64), ([1, 0], 0), ([300, 290], 8), ([20, 3], 8)])
def test_weight_gradients_of_overlapping_rows_with_an_infinity(rows, stride, storage):
    """Windows of a sequence, one row for all, single rows: an infinity counts in the columns where a row has it, and nowhere else."""
    dt, gen, K, cols, wide, most = dtype_of(storage), generator(41), len(rows), 64, 48, max(rows)
    m = Model(K, [(wide, cols), (wide, cols)], storage, gen)
    own = (most - 1) * stride + cols
    x = torch.randn(K, own, generator=gen, device=DEV).to(dt)
    view = x.as_strided((K, most, cols), (own, stride, 1))
    for k, n in enumerate(rows):
        if n:
            view[k, n - 1, -1] = float("inf")               # the last element that this replica reads
    g, u, da = (Act(rows, wide, dt, "dense", gen) for _ in range(3))
    work = workspace(m.ctx.gated_backward_bytes(0, 1, rows, cols))
    m.ctx.gated_backward(0, 1, rows, cols, (x.data_ptr(), own, stride), g.at, u.at, da.at, None, accumulate=False, workspace=work.data_ptr(),
                         workspace_bytes=work.numel())
    torch.cuda.synchronize()
    for k, n in enumerate(rows):
        f, slope = act64("silu", g.d(k))
        xk = view[k, :n].double()
        there = xk.isfinite().all(0)                        # columns without one
        for which, d, o in ((0, da.d(k) * u.d(k) * slope, (16 * U * (1 + g.d(k).abs()) + HALF[dt] * slope.abs()) * (da.d(k) * u.d(k)).abs()),
                            (1, da.d(k) * f, (16 * U * (f.abs() + g.d(k).abs()) + HALF[dt] * f.abs()) * da.d(k).abs())):
            o = o + 4 * U * d.abs()
            got, xs = m.grad(which, k)[:, there], xk[:, there]
            want = d.T @ xs
            bound = o.T @ xs.abs() + 2 * (n + 2) * U * ((d.abs() + o).T @ xs.abs())
            within(got, want, bound + HALF[dt] * (want.abs() + bound), ("gate", "up")[which])
            if n == 1:
                one = m.grad(which, k)[:, -1].double()
                assert torch.equal(one, torch.where(d[0] > 0, math.inf, -math.inf).double())
            elif n:
                assert bool((~m.grad(which, k)[:, ~there].isfinite()).all())
    m.close()


# ---- quotients next to a border of e4m3 -----------------------------------------------------------------------------------------
def test_quotients_next_to_a_border_are_rounded_by_way_of_fp32():
    """Every border between two values of e4m3, with products gain * h that are closer to it than half a step of fp32, on either side: 48 bits make the
    quotient, whose scale is a power of two (the largest element is 448 times it), so it is known to the bit. To fp32 it becomes the border, and
    then goes to its even side."""
    q8 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()             # 0 to 448
    lower, upper = q8[:-1], q8[1:]
    border = (lower + upper) / 2
    e, f = 2.0 ** -13, 2.0 ** -12
    # (1 + e)(1 - e) = 1 - 2^-26,   (1 + f)(1 - f + f^2) = 1 + 2^-36;  border has five bits, so both factors are fp32 values
    h = torch.cat([border * (1 + e), border * (1 + f)])
    w = torch.cat([torch.full_like(border, 1 - e), torch.full_like(border, 1 - f + f * f)])
    even = torch.where((torch.arange(126) & 1) == 0, lower, upper)
    want = torch.cat([even, even])
    assert torch.equal((h * w).float().double(), torch.cat([border, border])) and bool((h * w != torch.cat([border, border])).all())
    assert torch.equal(h.float().double(), h) and torch.equal(w.float().double(), w)
    h, w, want = (torch.cat([t, t.new_tensor([s])]) for t, s in ((h, 448.0), (w, 1.0), (want, 448.0)))
    cols = h.numel()
    assert cols == 253                                       # eight bytes at a time, and one by one behind them
    for K, pad in ((1, 0), (2, 3)):
        width = cols + pad
        gain, rows = torch.ones(width, dtype=torch.float64), [4] * K
        gain[:cols] = w
        m = Model(K, [(width,)], "f32", generator(0))
        x = torch.zeros(K, 4, width, dtype=torch.float64)
        x[:, :, :cols] = h
        for r in range(4):
            x[:, r] *= (-1.0) ** r * 2.0 ** (3 * r - 4)
        x = x.float().to(DEV)
        for k in range(K):
            m.weight(0, k).copy_(gain.float().to(DEV))
        q, s = torch.zeros(K, 4, width, dtype=torch.uint8, device=DEV), torch.zeros(K, 4, device=DEV)
        m.ctx.rms_norm(0, rows, (x.data_ptr(), 4 * width, width), (q.data_ptr(), 4 * width, width), scales=(s.data_ptr(), 4, 1), eps=0.0)
        torch.cuda.synchronize()
        got = q.view(torch.float8_e4m3fn).double().cpu()
        for k in range(K):
            for r in range(4):
                assert torch.equal(got[k, r, :cols] * (-1.0) ** r, want), (K, k, r, int((got[k, r, :cols] * (-1.0) ** r != want).sum()))
                assert bool((got[k, r, cols:] == 0).all())
        m.close()


# ---- more rows than a launch has threads for ------------------------------------------------------------------------------------
def test_a_norm_of_more_rows_than_one_launch_holds():
    """2^28 + 2^20 + 7 rows of eight columns, sixteen threads each: the second launch goes on where the first ends."""
    gen, period, times, tail = generator(51), 1 << 20, 257, 7
    m = Model(1, [(8,)], "bf16", gen, plus=1.0)
    n = period * times + tail
    part = torch.randn(period, 8, generator=gen, device=DEV).bfloat16()
    want, y = torch.empty_like(part), torch.full((n + 1, 8), 77.0, dtype=torch.bfloat16, device=DEV)
    m.ctx.rms_norm(0, [period], (part.data_ptr(), 0, 8), (want.data_ptr(), 0, 8))
    x = torch.empty(n, 8, dtype=torch.bfloat16, device=DEV)
    x[: period * times].view(times, period, 8).copy_(part.expand(times, period, 8))
    x[period * times:] = part[:tail]
    m.ctx.rms_norm(0, [n], (x.data_ptr(), 0, 8), (y.data_ptr(), 0, 8))
    torch.cuda.synchronize()
    for i in range(times):
        assert torch.equal(y[i * period: (i + 1) * period], want), i
    assert torch.equal(y[period * times: n], want[:tail]) and bool((y[n] == 77.0).all())
    m.close()
