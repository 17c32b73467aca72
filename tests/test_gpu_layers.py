"""Dropout, root-mean-square norms and gated blocks of K replicas on the GPU, against the same in 64 bits: sizes, layouts and types
where they can go wrong, rows that are not there, what lies around the outputs, graphs, streams.

Tolerances count roundings: U is half a step of fp32 relative to the value, HALF half a step of the storage type."""
import math

import numpy as np
import pytest
import torch

from paper_2203_13085_amd import binding as B
from tests.layers_util import (ACTS, DEV, HALF, U, Act, Model, act64, dtype_of, generator, mask_of, philox, scale_of, within, workspace,
                               workspace_kept)

pytestmark = pytest.mark.gpu
SEED, CALL = 0x1234567890ABCDEF, 0x3FFFFFFFF          # a call number beyond 32 bits


def test_philox_known_answers():
    """The vectors published with the generator."""
    assert philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


# ---- dropout ---------------------------------------------------------------------------------------------------------------
DROPS = [  # rows, cols, layout
    ([7, 7, 7], 260, "dense"),
    ([1], 1, "dense"),
    ([1, 0, 3], 8, "padded"),
    ([5, 9], 1023, "odd"),
    ([33, 1, 64, 0], 64, "turned"),
    ([3, 2], 2056, "padded"),
    ([2, 300], 24, "dense"),
]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", DROPS)
@pytest.mark.parametrize("p", [0.1, 0.5])
def test_dropout_is_its_definition_to_the_bit(rows, cols, layout, p, storage):
    dt, gen, K = dtype_of(storage), generator(1), len(rows)
    m = Model(K, [(8,)], storage, gen)
    x, res, y, z = Act(rows, cols, dt, layout, gen), Act(rows, cols, dt, "dense", gen), Act(rows, cols, dt, layout), Act(rows, cols, dt, "padded")
    m.ctx.dropout(rows, cols, x.at, y.at, p, residual=res.at, seed=SEED, call=CALL)
    m.ctx.dropout(rows, cols, x.at, z.at, p, seed=SEED, call=CALL)
    torch.cuda.synchronize()
    s = torch.tensor(scale_of(p), dtype=torch.float32, device=DEV)
    for k in range(K):
        stays = mask_of(k, rows[k], cols, p, SEED, CALL).to(DEV)
        kept = torch.where(stays, x[k].float() * s, 0.0)
        assert torch.equal(y[k], (res[k].float() + kept).to(dt))
        assert torch.equal(z[k], kept.to(dt))
    assert y.untouched_outside() and z.untouched_outside()
    m.close()


def test_dropout_drops_its_share():
    """Of 2^21 elements 0.1 are dropped, within six standard deviations; columns, rows and halves of words alike."""
    m = Model(2, [(8,)], "f32", generator(0))
    x, y = torch.ones(2, 1024, 1024, device=DEV), torch.empty(2, 1024, 1024, device=DEV)
    m.ctx.dropout([1024] * 2, 1024, (x.data_ptr(), 1 << 20, 1024), (y.data_ptr(), 1 << 20, 1024), 0.1, seed=3, call=5)
    torch.cuda.synchronize()
    q = round(0.1 * 65536) / 65536
    dropped = (y == 0).double()
    for part in (dropped, dropped[0], dropped[1], *(dropped[:, :, j::8] for j in range(8)), dropped[:, ::2], dropped[0] * dropped[1]):
        n, want = part.numel(), q * q if part is not dropped and part.shape == (1024, 1024) and float(part.mean()) < 0.05 else q
        assert abs(float(part.mean()) - want) < 6 * math.sqrt(want * (1 - want) / n)
    assert set(y.unique().tolist()) == {0.0, float(np.float32(65536 / (65536 - 6554)))}
    m.close()


def test_masks_depend_on_the_place_and_the_call_alone():
    """Other layouts, fewer replicas or rows, another stream, another call in between: the same mask. Another call, seed or counter: another."""
    m4, m2 = Model(4, [(8,)], "f32", generator(0)), Model(2, [(8,)], "bf16", generator(0))

    def mask(m, rows, layout, seed=SEED, call=CALL, counter=None):
        dt = m.dt
        x = Act(rows, 200, dt, layout)
        for k, n in enumerate(rows):
            x.t[k, :n] = 1.0
        y = Act(rows, 200, dt, "dense")
        m.ctx.dropout(rows, 200, x.at, y.at, 0.3, seed=seed, call=call, counter=counter)
        torch.cuda.synchronize()
        return [(y[k] != 0).cpu() for k in range(len(rows))]
    a = mask(m4, [50, 60, 70, 80], "dense")
    b = mask(m4, [60, 80, 0, 9], "turned")
    c = mask(m2, [50, 70], "odd")
    assert torch.equal(a[0], b[0][:50]) and torch.equal(a[1], b[1][:60]) and torch.equal(a[3][:9], b[3])
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1][:60])
    for other in (dict(call=CALL + 1), dict(call=CALL - (1 << 33)), dict(seed=SEED + 1), dict(seed=SEED ^ (1 << 63))):
        assert not torch.equal(a[0], mask(m4, [50, 60, 70, 80], "dense", **other)[0])
    assert not torch.equal(a[0], a[1][:50])
    counter = torch.tensor([7], dtype=torch.int64, device=DEV)
    assert torch.equal(a[0], mask(m4, [50, 60, 70, 80], "dense", call=CALL - 7, counter=counter.data_ptr())[0])
    m4.close(), m2.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_dropout_edges(storage):
    """p = 0 and 1, in place, a dropped infinity or NaN counts 0, a broadcast input."""
    dt, gen = dtype_of(storage), generator(2)
    m = Model(2, [(8,)], storage, gen)
    rows, cols = [6, 4], 48
    x, res, y = Act(rows, cols, dt, "dense", gen), Act(rows, cols, dt, "dense", gen), Act(rows, cols, dt)
    m.ctx.dropout(rows, cols, x.at, y.at, 0.0, residual=res.at)
    for k in range(2):
        assert torch.equal(y[k], (res[k].float() + x[k].float()).to(dt))
    x[0][0, :] = float("nan")
    x[1][1, :] = float("inf")
    m.ctx.dropout(rows, cols, x.at, y.at, 1.0, residual=res.at)
    assert torch.equal(y[0], res[0]) and torch.equal(y[1], res[1])
    m.ctx.dropout(rows, cols, x.at, y.at, 0.5, seed=1, call=2)
    stays = mask_of(0, 6, cols, 0.5, 1, 2).to(DEV)
    assert torch.equal(y[0][0].isnan(), stays[0]) and bool((y[0][0][~stays[0]] == 0).all())
    want = y.t.clone()
    m.ctx.dropout(rows, cols, x.at, x.at, 0.5, seed=1, call=2)                    # in place
    for k in range(2):
        assert torch.equal(x[k].nan_to_num(5.0), want[k, : rows[k]].nan_to_num(5.0))
    one = torch.randn(cols, device=DEV).to(dt)
    m.ctx.dropout(rows, cols, (one.data_ptr(), 0, 0), y.at, 0.0)                  # every row the same
    assert all(torch.equal(y[k], one.expand(rows[k], cols)) for k in range(2))
    m.close()


@pytest.mark.parametrize("storage,K,n,cols", [("bf16", 3, 4096, 4096), ("f32", 2, 4096, 4104)])
def test_calls_beyond_the_cache_give_the_same_bits(storage, K, n, cols):
    """Accesses with the streaming hint (over 256 MiB a call), against the replicas one by one, without: dropout, a norm in either output, its backward pass."""
    dt, gen = dtype_of(storage), generator(22)
    m = Model(K, [(cols,)], storage, gen, plus=1.0)
    x, res = (torch.randn(K, n, cols, generator=gen, device=DEV).to(dt) for _ in range(2))
    at = lambda t: (t.data_ptr(), t.stride(0), t.stride(1))  # noqa: E731

    def all_of(masks):
        out = {name: torch.zeros(K, n, cols, dtype=torch.uint8 if name == "q" else dt, device=DEV) for name in ("d", "h", "y", "q", "dx", "dr")}
        scales = torch.zeros(K, n, device=DEV)
        for rows in masks:
            drop = dict(p=0.3, seed=SEED, call=CALL)
            m.ctx.dropout(rows, cols, at(x), at(out["d"]), 0.3, residual=at(res), seed=SEED, call=CALL)
            m.ctx.rms_norm(0, rows, at(x), at(out["y"]), residual=at(res), sum=at(out["h"]), **drop)
            m.ctx.rms_norm(0, rows, at(x), at(out["q"]), residual=at(res), scales=(scales.data_ptr(), n, 1), **drop)
            work = workspace(m.ctx.rms_norm_backward_bytes(0, rows))
            m.ctx.rms_norm_backward(0, rows, at(out["h"]), at(out["y"]), at(out["dx"]), dsum=at(x), dresidual=at(out["dr"]), workspace=work.data_ptr(),
                                    workspace_bytes=work.numel(), **drop)
            torch.cuda.synchronize()
        return [*out.values(), scales]
    for a, b in zip(all_of([[n] * K]), all_of([[n if k == i else 0 for k in range(K)] for i in range(K)])):
        assert torch.equal(a, b)
    m.close()


# ---- norms -------------------------------------------------------------------------------------------------------------------
NORMS = [  # rows, cols, layout: every shape of the kernels, and columns on either side of their limits
    ([1], 1, "dense"),
    ([3, 0, 2], 7, "odd"),
    ([40, 17], 128, "dense"),
    ([5, 4], 136, "turned"),
    ([9, 2, 1], 511, "padded"),
    ([3, 4], 1024, "dense"),
    ([7, 1], 1023, "odd"),
    ([5, 5], 2048, "padded"),
    ([3, 2], 2049, "dense"),
    ([2, 3], 4096, "turned"),
    ([2, 2], 8192, "dense"),
    ([1, 2], 8200, "odd"),
    ([3], 16384, "dense"),
]
DEPTH = 40        # roundings on the way of a norm's sum: at most 32 of a thread, its squares' and six to eight across threads counted among them


def _norm64(x, res, factor, w, eps):
    h = x * factor + (res if res is not None else 0.0)
    rho = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    return h, rho, w * h * rho


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", NORMS)
@pytest.mark.parametrize("p,with_res", [(0.0, True), (0.0, False), (0.25, True)])
def test_rms_norm(rows, cols, layout, p, with_res, storage):
    dt, gen, K, eps = dtype_of(storage), generator(3), len(rows), 1e-5
    m = Model(K, [(5,), (cols,)], storage, gen, plus=1.0)
    x, res = Act(rows, cols, dt, layout, gen), Act(rows, cols, dt, "padded", gen, 3.0) if with_res else None
    h, y = Act(rows, cols, dt, "padded"), Act(rows, cols, dt, layout)
    m.ctx.rms_norm(1, rows, x.at, y.at, residual=res.at if res else None, sum=h.at, eps=eps, p=p, seed=SEED, call=CALL)
    torch.cuda.synchronize()
    e = float(np.float32(eps))
    for k in range(K):
        f = mask_of(k, rows[k], cols, p, SEED, CALL).to(DEV).double() * scale_of(p)
        w = m.weight(1, k).double()
        h64, rho, y64 = _norm64(x.d(k), res.d(k) if res else None, f, w, e)
        off = U * (2 * (x.d(k) * f).abs() + h64.abs())                 # of h: scale, product, sum
        if p == 0.0 and not with_res:
            assert torch.equal(h[k], x[k])
        within(h[k], h64, off + HALF[dt] * (h64.abs() + off), "sum")
        # rho moves with the root of the mean square: half of (DEPTH roundings, and what the elements are off by)
        rel = 0.5 * (DEPTH * U + 2 * off.norm(dim=1, keepdim=True) / h64.norm(dim=1, keepdim=True).clamp(min=1e-30)) + 4 * U
        bound = (w * rho).abs() * off + y64.abs() * (rel + 2 * U)
        within(y[k], y64, bound + HALF[dt] * (y64.abs() + bound), "y")
    assert h.untouched_outside() and y.untouched_outside() and m.gaps_untouched()
    m.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", [([1], 1, "dense"), ([3, 0, 2], 7, "odd"), ([9, 5], 512, "dense"), ([4, 3], 2048, "turned"),
                                              ([2, 2], 4100, "padded"), ([2], 16384, "dense")])
def test_rms_norm_in_8_bits(rows, cols, layout, storage):
    """A row of zeros too. Each value is within half a step of e4m3 (2^-4 relative, or half the least step, 2^-10) of the exact quotient."""
    dt, gen, K, eps = dtype_of(storage), generator(4), len(rows), 1e-6
    m = Model(K, [(cols,)], storage, gen, plus=1.0)
    x = Act(rows, cols, dt, layout, gen)
    x[0][0] = 0.0
    R = max(max(rows), 1)
    q = torch.full((K, R, cols + 8), 0x55, dtype=torch.uint8, device=DEV)
    scales = torch.full((K, R), -1.0, device=DEV)
    m.ctx.rms_norm(0, rows, x.at, (q.data_ptr(), q.stride(0), q.stride(1)), scales=(scales.data_ptr(), R, 1), eps=eps)
    torch.cuda.synchronize()
    for k, n in enumerate(rows):
        _, _, y64 = _norm64(x.d(k), None, 1.0, m.weight(0, k).double(), float(np.float32(eps)))
        rel = (0.5 * DEPTH + 8) * U                                                     # of y in fp32
        most = y64.abs().amax(1)
        s = scales[k, :n].double()
        within(s, (most / 448).clamp(min=2.0 ** -126), most / 448 * (rel + U), "scale")
        v = q[k, :n, :cols].contiguous().view(torch.float8_e4m3fn).double()
        want = y64 / s[:, None]
        within(v, want, want.abs() * (2.0 ** -4 * (1 + 4 * rel) + 4 * rel) + 2.0 ** -10, "quotient")
        assert bool((q[k, n:] == 0x55).all()) and bool((q[k, :n, cols:] == 0x55).all()) and bool((scales[k, n:] == -1).all())
        if n and k:
            assert bool((v.abs().amax(1) == 448).all())
    assert float(scales[0, 0]) == 2.0 ** -126 and bool((q[0, 0, :cols] & 0x7F == 0).all())
    m.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
def test_rms_norm_in_8_bits_takes_the_nearest_value(storage):
    """Every one of 2^21 values, with a residual and a mask: the quotients are made in 64 bits, so what lies next to a border goes to its side."""
    dt, gen, rows, cols, p = dtype_of(storage), generator(21), [512, 512], 2048, 0.125
    m = Model(2, [(cols,)], storage, gen, plus=1.0)
    x, res, h = Act(rows, cols, dt, "dense", gen), Act(rows, cols, dt, "dense", gen), Act(rows, cols, dt)
    q, scales = torch.zeros(2, 512, cols, dtype=torch.uint8, device=DEV), torch.zeros(2, 512, device=DEV)
    m.ctx.rms_norm(0, rows, x.at, (q.data_ptr(), 512 * cols, cols), residual=res.at, sum=h.at, scales=(scales.data_ptr(), 512, 1), eps=1e-6, p=p, seed=SEED, call=CALL)
    torch.cuda.synchronize()
    for k in range(2):
        f = mask_of(k, 512, cols, p, SEED, CALL).to(DEV).double() * scale_of(p)
        h64, _, y64 = _norm64(x.d(k), res.d(k), f, m.weight(0, k).double(), float(np.float32(1e-6)))
        s64 = y64.abs().amax(1, keepdim=True) / 448
        assert torch.equal(q[k].view(torch.float8_e4m3fn).float(), (y64 / s64).float().to(torch.float8_e4m3fn).float())
        within(scales[k], s64[:, 0], U * s64[:, 0] * 1.001, "scale")
        within(h[k], h64, HALF[dt] * h64.abs() * 1.001 + U * h64.abs(), "sum")
    m.close()


def test_rms_norm_without_numbers():
    """An infinity or a NaN stays in its row; a row of zeros gives zeros."""
    gen = generator(5)
    m = Model(1, [(96,)], "f32", gen)
    x, y = Act([4], 96, torch.float32, "dense", gen), Act([4], 96, torch.float32)
    x[0][1, 3], x[0][2, 5], x[0][3] = float("nan"), float("inf"), 0.0
    m.ctx.rms_norm(0, [4], x.at, y.at, eps=1e-6)
    assert bool(y[0][0].isfinite().all()) and bool(y[0][1].isnan().all()) and bool(y[0][3].eq(0).all())
    assert bool(y[0][2, 5].isnan()) and bool(torch.cat([y[0][2, :5], y[0][2, 6:]]).eq(0).all())      # infinity times 1 / infinity; finite ones times it
    q, s = torch.zeros(4, 96, dtype=torch.uint8, device=DEV), torch.zeros(4, device=DEV)
    m.ctx.rms_norm(0, [4], x.at, (q.data_ptr(), 0, 96), scales=(s.data_ptr(), 0, 1), eps=1e-6)
    assert bool(s[1].isnan()) and bool(q[1].view(torch.float8_e4m3fn).float().isnan().all()) and bool(s[0].isfinite())
    m.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,layout", NORMS + [([700, 300], 40, "dense"), ([2500], 72, "padded")])
@pytest.mark.parametrize("p,accumulate", [(0.0, True), (0.25, False)])
def test_rms_norm_backward(rows, cols, layout, p, accumulate, storage):
    dt, gen, K, eps = dtype_of(storage), generator(6), len(rows), 1e-5
    m = Model(K, [(cols,), (3,)], storage, gen, plus=1.0)
    h, dy = Act(rows, cols, dt, layout, gen, 2.0), Act(rows, cols, dt, "padded", gen)
    dsum = Act(rows, cols, dt, "dense", gen) if p else None
    dres, dx = Act(rows, cols, dt, "padded"), Act(rows, cols, dt, layout)
    before = [m.grad(0, k).double() for k in range(K)]
    nbytes = m.ctx.rms_norm_backward_bytes(0, rows)
    work = workspace(nbytes)
    m.ctx.rms_norm_backward(0, rows, h.at, dy.at, dx.at, dsum=dsum.at if dsum else None, dresidual=dres.at, eps=eps, p=p, seed=SEED, call=CALL,
                            accumulate=accumulate, workspace=work.data_ptr(), workspace_bytes=nbytes)
    torch.cuda.synchronize()
    e = float(np.float32(eps))
    for k, n in enumerate(rows):
        f = mask_of(k, n, cols, p, SEED, CALL).to(DEV).double() * scale_of(p)
        w, hk, dyk = m.weight(0, k).double(), h.d(k), dy.d(k)
        rho = 1 / torch.sqrt((hk * hk).mean(1, keepdim=True) + e)
        hat = hk * rho
        mean = (hat * w * dyk).mean(1, keepdim=True)
        add = dsum.d(k) if dsum else torch.zeros_like(hk)
        dh = rho * (w * dyk - hat * mean) + add
        # the two parts and the mean, each with DEPTH roundings at most of its terms' size, and a few of rho
        size = rho * ((w * dyk).abs() + hat.abs() * (hat * w * dyk).abs().mean(1, keepdim=True)) + add.abs()
        off = (2 * DEPTH + 10) * U * size
        within(dres[k], dh, off + HALF[dt] * (dh.abs() + off), "dresidual")
        off2 = (off + 2 * U * (dh.abs() + off)) * f
        within(dx[k], dh * f, off2 + HALF[dt] * ((dh * f).abs() + off2), "dx")
        dw = (dyk * hat).sum(0) + (before[k] if accumulate else 0.0)
        terms = (dyk * hat).abs().sum(0) + before[k].abs()
        off = (n + DEPTH) * U * terms                      # any order of n additions, and hat's own
        within(m.grad(0, k), dw, off + HALF[dt] * (dw.abs() + off), "gain")
    assert dres.untouched_outside() and dx.untouched_outside() and m.gaps_untouched() and workspace_kept(work, nbytes)
    m.close()


def test_rms_norm_backward_is_the_slope():
    """The gradient along a direction against differences of the forward pass in 64 bits; and what is not wanted, or in place."""
    gen, rows, cols, eps = generator(7), [5, 3], 96, 1e-3
    m = Model(2, [(cols,)], "f32", gen, plus=1.0)
    h, dy, dx = Act(rows, cols, torch.float32, "dense", gen), Act(rows, cols, torch.float32, "dense", gen), Act(rows, cols, torch.float32)
    m.ctx.zero_grads()
    work = workspace(m.ctx.rms_norm_backward_bytes(0, rows))
    m.ctx.rms_norm_backward(0, rows, h.at, dy.at, dx.at, eps=eps, workspace=work.data_ptr(), workspace_bytes=work.numel())
    e = float(np.float32(eps))
    for k in range(2):
        w, v = m.weight(0, k).double(), torch.randn(rows[k], cols, generator=gen, device=DEV).double()
        vw = torch.randn(cols, generator=gen, device=DEV).double()

        def loss(t):
            return float((_norm64(h.d(k) + t * v, None, 1.0, w + t * vw, e)[2] * dy.d(k)).sum())
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        ours = float((dx.d(k) * v).sum() + (m.grad(0, k).double() * vw).sum())
        size = float((dx.d(k) * v).abs().sum() + (m.grad(0, k).double() * vw).abs().sum())
        assert abs(slope - ours) <= 1e-5 * size          # (2 DEPTH + 10) U = 5.4e-6 of the terms, and the difference's 1e-10
    gain = m.grad(0, 0).clone()
    want = dx.t.clone()
    m.ctx.rms_norm_backward(0, rows, h.at, dy.at, None, eps=eps, accumulate=False, workspace=work.data_ptr(), workspace_bytes=work.numel())
    assert torch.equal(m.grad(0, 0), gain)
    m.ctx.rms_norm_backward(0, rows, h.at, dy.at, dy.at, eps=eps, accumulate=False, workspace=work.data_ptr(), workspace_bytes=work.numel())
    assert all(torch.equal(dy[k], want[k, : rows[k]]) for k in range(2))
    m.close()


def test_gradients_of_replicas_without_rows():
    """accumulate: they stay; otherwise they are replaced, by zeros."""
    gen = generator(8)
    m = Model(3, [(40,), (24, 40), (24, 40)], "bf16", gen)
    empty = Act([0, 0, 0], 40, m.dt, "dense", gen)
    wide = Act([0, 0, 0], 24, m.dt, "dense", gen)
    before = [g[0].clone() for g in m.g]
    m.ctx.rms_norm_backward(0, [0] * 3, empty.at, empty.at, empty.at, workspace=None)
    m.ctx.gated_backward(1, 2, [0] * 3, 40, empty.at, wide.at, wide.at, wide.at, empty.at)
    m.ctx.rms_norm(0, [0] * 3, empty.at, empty.at)
    m.ctx.gated(1, 2, [0] * 3, 40, empty.at, wide.at)
    m.ctx.dropout([0] * 3, 40, empty.at, empty.at, 0.5)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b[0]) for a, b in zip(before, m.g))
    m.ctx.rms_norm_backward(0, [0] * 3, empty.at, empty.at, empty.at, accumulate=False)
    m.ctx.gated_backward(1, 2, [0] * 3, 40, empty.at, wide.at, wide.at, wide.at, empty.at, accumulate=False)
    torch.cuda.synchronize()
    assert all(bool(m.grad(i, k).eq(0).all()) for i in range(3) for k in range(3)) and m.gaps_untouched()
    assert empty.untouched_outside() and wide.untouched_outside()
    m.close()


# ---- gated blocks ------------------------------------------------------------------------------------------------------------
GATED = [  # rows, cols, wide, layout
    ([1], 1, 1, "dense"),
    ([1, 1, 1, 1], 256, 192, "dense"),
    ([3, 0, 2], 33, 17, "odd"),
    ([5, 16], 64, 40, "padded"),
    ([65, 130], 128, 96, "dense"),
    ([70, 1, 64], 515, 103, "turned"),
    ([200], 192, 264, "padded"),
    ([257, 31], 72, 520, "dense"),
    ([300, 0, 512], 256, 384, "dense"),
    ([17], 1032, 1000, "turned"),
]


LARGE = [  # what only many tiles or many bytes take: tiles of 256 and, unaligned, of 128; weights beyond the cache with few rows
    ([512, 300, 0, 511] + [257] * 60, 1032, 1000, "dense", "silu"),
    ([256, 129, 0, 255] + [200] * 12, 2051, 1030, "odd", "gelu"),
    ([3, 0, 16] + [5] * 61, 1032, 1024, "dense", "relu"),
    ([40, 64, 0] + [17] * 61, 1032, 1024, "turned", "gelu_tanh"),
]


def _product_off(deep, storage):
    """Roundings of a sum of `deep` products, in any order; twice that, for what the matrix units do not round to nearest."""
    return 2 * (deep + 2) * U


def _block(rows, cols, wide, layout, act, storage, seed=9, packed=False):
    dt, gen, K = dtype_of(storage), generator(seed), len(rows)
    shapes = [(2, wide, cols)] if packed else [(wide, cols), (3,), (wide, cols)]
    m = Model(K, shapes, storage, gen, scales=[cols ** -0.5] * 3)
    x = Act(rows, cols, dt, layout, gen)
    g, u, a = Act(rows, wide, dt, "padded"), Act(rows, wide, dt, layout), Act(rows, wide, dt, layout)
    i, j = (0, 0) if packed else (0, 2)
    m.ctx.gated(i, j, rows, cols, x.at, a.at, g=g.at, u=u.at, activation=ACTS[act])
    weights = [(m.weight(0, k)[0], m.weight(0, k)[1]) if packed else (m.weight(0, k), m.weight(2, k)) for k in range(K)]
    grads = [(m.grad(0, k)[0], m.grad(0, k)[1]) if packed else (m.grad(0, k), m.grad(2, k)) for k in range(K)]
    return m, (i, j), x, g, u, a, weights, grads


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,wide,layout", GATED)
@pytest.mark.parametrize("act,packed", [("silu", False), ("gelu", True), ("gelu_tanh", False), ("relu", False)])
def test_gated(rows, cols, wide, layout, act, packed, storage):
    check_gated(rows, cols, wide, layout, act, packed, storage)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,wide,layout,act", LARGE)
def test_gated_large(rows, cols, wide, layout, act, storage):
    check_gated(rows, cols, wide, layout, act, False, storage)


def check_gated(rows, cols, wide, layout, act, packed, storage):
    m, (i, j), x, g, u, a, weights, _ = _block(rows, cols, wide, layout, act, storage, packed=packed)
    dt, off = m.dt, _product_off(cols, storage)
    alone = Act(rows, wide, dt, "dense")
    m.ctx.gated(i, j, rows, cols, x.at, alone.at, activation=ACTS[act])
    torch.cuda.synchronize()
    for k in range(len(rows)):
        wg, wu = (w.double() for w in weights[k])
        g64, u64 = x.d(k) @ wg.T, x.d(k) @ wu.T
        og, ou = off * (x.d(k).abs() @ wg.abs().T), off * (x.d(k).abs() @ wu.abs().T)
        within(g[k], g64, og + HALF[dt] * (g64.abs() + og), "g")
        within(u[k], u64, ou + HALF[dt] * (u64.abs() + ou), "u")
        f, _ = act64(act, g64)
        # no activation is steeper than 1.13; its own error: 16 roundings, of its value or (where 1 + erf or tanh cancels) of its argument
        of = 1.13 * og + 16 * U * (f.abs() + g64.abs())
        bound = of * (u64.abs() + ou) + f.abs() * ou + U * (f * u64).abs()
        within(a[k], f * u64, bound + HALF[dt] * ((f * u64).abs() + bound), "a")
        assert torch.equal(a[k], alone[k])
    assert all(t.untouched_outside() for t in (g, u, a, alone)) and m.gaps_untouched()
    m.close()


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,wide,layout", GATED)
@pytest.mark.parametrize("act,packed,accumulate", [("silu", False, False), ("gelu", True, True), ("gelu_tanh", False, True), ("relu", False, False)])
def test_gated_backward(rows, cols, wide, layout, act, packed, accumulate, storage):
    check_gated_backward(rows, cols, wide, layout, act, packed, accumulate, storage)


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("rows,cols,wide,layout,act", LARGE)
def test_gated_backward_large(rows, cols, wide, layout, act, accumulate, storage):
    check_gated_backward(rows, cols, wide, layout, act, False, accumulate, storage)


def check_gated_backward(rows, cols, wide, layout, act, packed, accumulate, storage):
    m, (i, j), x, g, u, a, weights, grads = _block(rows, cols, wide, layout, act, storage, packed=packed)
    dt, gen = m.dt, generator(10)
    da, dx = Act(rows, wide, dt, layout, gen), Act(rows, cols, dt, layout)
    before = [tuple(t.double() for t in p) for p in grads]
    nbytes = m.ctx.gated_backward_bytes(i, j, rows, cols)
    work = workspace(nbytes)
    m.ctx.gated_backward(i, j, rows, cols, x.at, g.at, u.at, da.at, dx.at, activation=ACTS[act], accumulate=accumulate,
                         workspace=work.data_ptr(), workspace_bytes=nbytes)
    torch.cuda.synchronize()
    for k, n in enumerate(rows):
        wg, wu = (w.double() for w in weights[k])
        f, slope = act64(act, g.d(k))
        dg, du = da.d(k) * u.d(k) * slope, da.d(k) * f
        # 16 roundings of the activation or its slope (of their terms where those cancel), two products, and one to the storage type
        og = (16 * U * (1 + g.d(k).abs()) + HALF[dt] * slope.abs()) * (da.d(k) * u.d(k)).abs() + 4 * U * dg.abs()
        ou = (16 * U * (f.abs() + g.d(k).abs()) + HALF[dt] * f.abs()) * da.d(k).abs() + 2 * U * du.abs()
        want = dg @ wg + du @ wu
        size = (dg.abs() + og) @ wg.abs() + (du.abs() + ou) @ wu.abs()
        bound = og @ wg.abs() + ou @ wu.abs() + _product_off(2 * wide, storage) * size
        within(dx[k], want, bound + HALF[dt] * (want.abs() + bound), "dx")
        for which, d, o in ((0, dg, og), (1, du, ou)):
            want = d.T @ x.d(k)
            bound = o.T @ x.d(k).abs() + _product_off(n, storage) * ((d.abs() + o).T @ x.d(k).abs())
            if accumulate:
                want = want + before[k][which]
                bound = bound + U * want.abs()
            within(grads[k][which], want, bound + HALF[dt] * (want.abs() + bound), ("gate", "up")[which])
    assert dx.untouched_outside() and m.gaps_untouched() and workspace_kept(work, nbytes)
    # without dx the gradients are the same
    kept = [g_[0].clone() for g_ in m.g]
    if not accumulate:
        m.ctx.gated_backward(i, j, rows, cols, x.at, g.at, u.at, da.at, None, activation=ACTS[act], accumulate=False,
                             workspace=work.data_ptr(), workspace_bytes=nbytes)
        torch.cuda.synchronize()
        assert all(torch.equal(c, g_[0]) for c, g_ in zip(kept, m.g))
    m.close()


@pytest.mark.parametrize("act", list(ACTS))
def test_gated_backward_is_the_slope(act):
    rows, cols, wide = [6, 4], 40, 24
    m, (i, j), x, g, u, a, weights, grads = _block(rows, cols, wide, "dense", act, "f32", seed=11)
    gen = generator(12)
    da, dx = Act(rows, wide, torch.float32, "dense", gen), Act(rows, cols, torch.float32)
    work = workspace(m.ctx.gated_backward_bytes(i, j, rows, cols))
    m.ctx.gated_backward(i, j, rows, cols, x.at, g.at, u.at, da.at, dx.at, activation=ACTS[act], accumulate=False,
                         workspace=work.data_ptr(), workspace_bytes=work.numel())
    torch.cuda.synchronize()
    for k in range(2):
        wg, wu = (w.double() for w in weights[k])
        vx, vg, vu = (torch.randn(*s, generator=gen, device=DEV).double() for s in ((rows[k], cols), (wide, cols), (wide, cols)))

        def loss(t):
            f, _ = act64(act, (x.d(k) + t * vx) @ (wg + t * vg).T)
            return float((f * ((x.d(k) + t * vx) @ (wu + t * vu).T) * da.d(k)).sum())
        slope = (loss(1e-6) - loss(-1e-6)) / 2e-6
        parts = [(dx.d(k) * vx), grads[k][0].double() * vg, grads[k][1].double() * vu]
        size = sum(float(q.abs().sum()) for q in parts)
        # 2 (2 wide + 2) U = 6e-6 of the terms, which cancel in the results by less than a factor of ten; differences: 1e-9 (relu: no corner
        # within 1e-6 of a value, which the size of g makes sure of: 240 values, a corner is 1e-5 of one's range)
        assert abs(slope - sum(float(q.sum()) for q in parts)) <= 6e-5 * size
    m.close()


def test_gated_with_shared_and_broadcast_inputs():
    """One batch for all replicas (stride 0), and one row for all."""
    gen, rows, cols, wide = generator(13), [20, 20], 64, 48
    m = Model(2, [(wide, cols), (wide, cols)], "bf16", gen, scales=[0.1, 0.1])
    x = torch.randn(20, cols, generator=gen, device=DEV).bfloat16()
    full = x.expand(2, 20, cols).contiguous()
    a, b = Act(rows, wide, m.dt), Act(rows, wide, m.dt)
    m.ctx.gated(0, 1, rows, cols, (x.data_ptr(), 0, cols), a.at)
    m.ctx.gated(0, 1, rows, cols, (full.data_ptr(), 20 * cols, cols), b.at)
    assert torch.equal(a.t, b.t)
    m.ctx.gated(0, 1, rows, cols, (x.data_ptr(), 0, 0), a.at)
    assert torch.equal(a[0], b[0][:1].expand(20, wide)) and torch.equal(a[1], b[1][:1].expand(20, wide))
    m.close()


# ---- streams, graphs, many replicas -------------------------------------------------------------------------------------------
def _sublayer(m, rows, cols, wide, x, res, out, stream, counter=None, call=1):
    ctx, s = m.ctx, stream.cuda_stream
    ctx.rms_norm(0, rows, x.at, out["y"].at, residual=res.at, sum=out["h"].at, p=0.2, seed=9, call=call, counter=counter, stream=s)
    ctx.gated(1, 2, rows, cols, out["y"].at, out["a"].at, g=out["g"].at, u=out["u"].at, stream=s)
    ctx.gated_backward(1, 2, rows, cols, out["y"].at, out["g"].at, out["u"].at, out["a"].at, out["dy"].at, accumulate=False,
                       workspace=out["w1"].data_ptr(), workspace_bytes=out["w1"].numel(), stream=s)
    ctx.rms_norm_backward(0, rows, out["h"].at, out["dy"].at, out["dx"].at, dresidual=out["dres"].at, p=0.2, seed=9, call=call, counter=counter,
                          accumulate=False, workspace=out["w2"].data_ptr(), workspace_bytes=out["w2"].numel(), stream=s)


def _outputs(m, rows, cols, wide):
    out = {n: Act(rows, cols, m.dt) for n in ("y", "h", "dy", "dx", "dres")}
    out.update({n: Act(rows, wide, m.dt) for n in ("a", "g", "u")})
    out["w1"] = workspace(m.ctx.gated_backward_bytes(1, 2, rows, cols))
    out["w2"] = workspace(m.ctx.rms_norm_backward_bytes(0, rows))
    return out


def _copies(m, out):
    return [out[n].buf.clone() for n in ("y", "h", "dy", "dx", "dres", "a", "g", "u")] + [g.clone() for g, _ in m.g]


@pytest.mark.parametrize("storage", ["f32", "bf16"])
@pytest.mark.parametrize("K,rows,cols,wide", [(3, [40, 0, 7], 136, 88), (64, [2] * 64, 64, 40), (2, [300, 256], 512, 384)])
def test_a_recorded_pass_repeats_the_eager_one(K, rows, cols, wide, storage):
    """Forward and backward in one graph, replayed with other inputs, other masks from the counter, and eager work of its own in between."""
    gen = generator(14)
    m = Model(K, [(cols,), (wide, cols), (wide, cols)], storage, gen, scales=[1.0, cols ** -0.5, cols ** -0.5])
    x, res = Act(rows, cols, m.dt, "dense", gen), Act(rows, cols, m.dt, "dense", gen)
    eager, rec = _outputs(m, rows, cols, wide), _outputs(m, rows, cols, wide)
    counter = torch.zeros(1, dtype=torch.int64, device=DEV)
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        _sublayer(m, rows, cols, wide, x, res, rec, torch.cuda.current_stream(), counter.data_ptr(), call=100)
    for turn in range(4):
        for k, n in enumerate(rows):
            x.t[k, :n] = torch.randn(n, cols, generator=gen, device=DEV).to(m.dt)
        counter.fill_(turn * 10)
        graph.replay()
        torch.cuda.synchronize()
        got = _copies(m, rec)
        _sublayer(m, rows, cols, wide, x, res, eager, torch.cuda.current_stream(), call=100 + turn * 10)
        torch.cuda.synchronize()
        for a, b in zip(got, _copies(m, eager)):
            assert torch.equal(a, b)
    m.close()


def test_two_passes_at_once_on_two_streams():
    """One context, two streams, outputs and workspaces of their own (only one of them writes gradients)."""
    gen, rows, cols, wide = generator(15), [256, 192], 512, 640
    m = Model(2, [(cols,), (wide, cols), (wide, cols)], "bf16", gen, scales=[1.0, cols ** -0.5, cols ** -0.5])
    x, res = Act(rows, cols, m.dt, "dense", gen), Act(rows, cols, m.dt, "dense", gen)
    alone, one, two = (_outputs(m, rows, cols, wide) for _ in range(3))
    _sublayer(m, rows, cols, wide, x, res, alone, torch.cuda.current_stream())
    torch.cuda.synchronize()
    want = _copies(m, alone)
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        _sublayer(m, rows, cols, wide, x, res, one, s1)
        m.ctx.rms_norm(0, rows, x.at, two["y"].at, residual=res.at, sum=two["h"].at, p=0.2, seed=9, call=1, stream=s2.cuda_stream)
        m.ctx.gated(1, 2, rows, cols, two["y"].at, two["a"].at, g=two["g"].at, u=two["u"].at, stream=s2.cuda_stream)
    torch.cuda.synchronize()
    for a, b in zip(want, _copies(m, one)):
        assert torch.equal(a, b)
    assert all(torch.equal(two[n].buf, alone[n].buf) for n in ("y", "h", "a", "g", "u"))
    m.close()


def test_gradients_go_where_the_step_reads_them():
    """Backward into the bound buffers, then the library's own step: the update of these gradients."""
    gen, rows, cols, wide = generator(16), [33, 20], 64, 48
    m = Model(2, [(cols,), (wide, cols), (wide, cols)], "f32", gen, scales=[1.0, 0.1, 0.1])
    x, res = Act(rows, cols, m.dt, "dense", gen), Act(rows, cols, m.dt, "dense", gen)
    out = _outputs(m, rows, cols, wide)
    before = [w.double() for _, w in m.w]
    _sublayer(m, rows, cols, wide, x, res, out, torch.cuda.current_stream())
    m.ctx.local_step(0.5)
    torch.cuda.synchronize()
    for i in range(3):
        want = before[i] - 0.5 * 1.9 * m.g[i][1].double()           # Nesterov momentum 0.9 from a buffer of zeros
        within(m.w[i][1], want, 4 * U * (before[i].abs() + m.g[i][1].double().abs()), str(i))
    m.close()


def test_offsets_beyond_32_bits():
    """Rows a GiB and replicas 4 GiB apart, all activations between each other in one buffer: the same as from dense ones."""
    K, n, cols, wide, gen = 2, 3, 64, 48, generator(23)
    buf = torch.empty((1 << 31) + 2 * (1 << 29) + 16 * 4096, dtype=torch.bfloat16, device=DEV)
    m = Model(K, [(cols,), (wide, cols), (wide, cols)], "bf16", gen, scales=[1.0, 0.1, 0.1])
    place = {}

    def far(name, width):
        place[name] = place.get(name, len(place))
        return buf.as_strided((K, n, width), (1 << 31, 1 << 29, 1), 4096 * place[name])

    def dense(name, width):
        place[name] = place.get(name) if isinstance(place.get(name), torch.Tensor) else torch.zeros(K, n, width, dtype=torch.bfloat16, device=DEV)
        return place[name]
    x0, r0, d0 = (torch.randn(K, n, cols, generator=gen, device=DEV).bfloat16() for _ in range(3))
    at = lambda t: (t.data_ptr(), t.stride(0), t.stride(1))  # noqa: E731
    results = []
    for make in (dense, far):
        place.clear()
        m.ctx.zero_grads()
        rows = [n] * K
        x, r, dy = make("x", cols), make("r", cols), make("dy", cols)
        x.copy_(x0), r.copy_(r0), dy.copy_(d0)
        out = {name: make(name, wide if name in ("a", "g", "u") else cols) for name in ("d", "h", "y", "a", "g", "u", "dx", "dr", "dz")}
        work = workspace(max(m.ctx.rms_norm_backward_bytes(0, rows), m.ctx.gated_backward_bytes(1, 2, rows, cols)))
        m.ctx.dropout(rows, cols, at(x), at(out["d"]), 0.5, residual=at(r), seed=1, call=2)
        m.ctx.rms_norm(0, rows, at(x), at(out["y"]), residual=at(r), sum=at(out["h"]), p=0.5, seed=1, call=2)
        m.ctx.rms_norm_backward(0, rows, at(out["h"]), at(dy), at(out["dx"]), dsum=at(r), dresidual=at(out["dr"]), p=0.5, seed=1, call=2,
                                workspace=work.data_ptr(), workspace_bytes=work.numel())
        m.ctx.gated(1, 2, rows, cols, at(x), at(out["a"]), g=at(out["g"]), u=at(out["u"]))
        m.ctx.gated_backward(1, 2, rows, cols, at(x), at(out["g"]), at(out["u"]), at(out["a"]), at(out["dz"]), workspace=work.data_ptr(),
                             workspace_bytes=work.numel())
        torch.cuda.synchronize()
        results.append([t.clone() for t in out.values()] + [g.float() for _, g in m.g])
    for i, (a, b) in enumerate(zip(*results)):
        # rows this far apart take the other kernels of the products: the same sums in another order, and a rounding may fall the other way
        assert torch.equal(a, b) if i < 3 or i in (6, 7) else torch.allclose(a.float(), b.float(), rtol=2.0 ** -6, atol=2.0 ** -9), i
    m.close()
