"""The channel norm, the 8-bit checkpoints, and the log probabilities of labels with their gradient and loss, against plain
implementations in 64 bits, at the sizes, layouts and values where they can go wrong."""
import pathlib
import subprocess
import sys
import threading

import numpy as np
import pytest
import torch

import paper_2409_09083_b200 as ftp
from _operators import (GUARD, HALF_STEP, TINY, TYPES, U, close, eight_bits, guarded, like, logprob, norm_backward,
                        norm_forward, rows)

pytestmark = pytest.mark.gpu
EPS = 1e-5

# (shape, elements between samples beyond dense, start off a 256-byte boundary): rows of one value to more than a block holds, odd
# ones, planes that vectors divide and do not, channels from one to more than stay in registers
SHAPES = [
    ((1, 1), 0, 0), ((3, 2), 0, 0), ((5, 7), 0, 0), ((33, 32), 0, 0), ((9, 33), 3, 1), ((1, 1024), 0, 0), ((17, 1000), 24, 0),
    ((6, 1111), 2, 3), ((300, 64), 0, 0), ((4, 4096), 0, 0), ((3, 5001), 0, 0), ((2, 9000), 0, 0), ((2, 20000), 0, 5), ((1, 40000), 8, 0),
    ((1, 70001), 0, 0), ((700, 257), 1, 0), ((333, 372), 0, 0), ((1300, 1111), 2, 0), ((19, 4097), 0, 1), ((2500, 68), 3, 2), ((9, 2047), 6, 7),
    ((2, 3, 1, 2), 0, 0), ((1, 8, 13, 13), 0, 0), ((3, 32, 13, 13), 0, 0), ((2, 64, 16, 24), 0, 0), ((2, 21, 10, 6), 4, 2), ((1, 512, 7, 7), 0, 0),
    ((400, 9001), 1, 3), ((160, 16384), 0, 0), ((2, 100, 8, 8), 8, 8), ((1, 1030, 5, 4), 0, 0), ((1, 2100, 3, 11), 5, 1), ((40, 5, 1, 3), 0, 0), ((2, 4, 64, 70), 0, 0),
]


def _ids(s):
    return "x".join(map(str, s[0])) + (f"+{s[1]}" if s[1] else "") + (f"@{s[2]}" if s[2] else "")


def _normal(shape, seed, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _run(shape):
    p = int(np.prod(shape[2:])) if len(shape) > 2 else 1
    return shape[1] if p == 1 else p


def _rows_of(shape):
    return (shape[0],) + tuple(shape[2:])


# ---- norm -----------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", SHAPES, ids=_ids)
def test_norm_forward(case, dtype):
    shape, pad, shift = case
    x = _normal(shape, 1, dtype) + torch.tensor(0.5, dtype=dtype)
    w, b = _normal(shape[1:2], 2), _normal(shape[1:2], 3)
    xd, xg = guarded(x, pad, shift)
    yd, yg = guarded(torch.zeros_like(x), pad, shift)
    mean, rstd = (torch.full(_rows_of(shape), GUARD, device="cuda") for _ in range(2))
    ckpt = torch.empty(ftp.ftp_ckpt_bytes(x), dtype=torch.uint8, device="cuda")
    ftp.ftp_norm_forward(xd, w.cuda(), b.cuda(), yd, mean, rstd, eps=EPS)
    y, m, r = norm_forward(x, w, b, EPS)
    # mean: a sum of c terms in a tree of at most 16 + 5 + 5 levels and one division; 32 half-units of the mean magnitude.  hat: that error
    # and the ones of variance (the same tree), root and quotient.
    xr = rows(x)
    size = xr.abs().mean(1)
    close(mean, m, 32 * U * size, "mean")
    err = 64 * U * (1 + (size * r) ** 2)                       # relative error of rstd: the mean's error enters the variance
    close(rstd, r, err * r, "rstd")
    hat = (xr.abs() + size[:, None]) * r[:, None]
    bound = HALF_STEP[dtype] * y.abs() + TINY[dtype] + (64 * U + err[:, None]) * (hat * w.double().abs() + b.double().abs())
    close(like(rows(yd), shape), like(y, shape), like(bound, shape), "y")
    xg(), yg()
    # the same results with the checkpoint on the side, whose bytes are those of the separate call
    y2, _ = guarded(torch.zeros_like(x), pad, shift)
    mean2, rstd2 = torch.empty_like(mean), torch.empty_like(rstd)
    ftp.ftp_norm_forward(xd, w.cuda(), b.cuda(), y2, mean2, rstd2, eps=EPS, ckpt=ckpt)
    separate = torch.empty_like(ckpt)
    ftp.ftp_ckpt_save(xd, separate)
    assert torch.equal(ckpt, separate)
    close(rows(y2), y, rows(like(bound, shape)), "y beside a checkpoint")
    # in place, no weight, no statistics
    y3, _, _ = norm_forward(x, None, None, EPS)
    ftp.ftp_norm_forward(xd, None, None, xd, eps=EPS)
    close(rows(xd), y3, HALF_STEP[dtype] * y3.abs() + TINY[dtype] + (64 * U + err[:, None]) * hat, "in place")
    xg()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("from_ckpt", [False, True])
@pytest.mark.parametrize("case", SHAPES, ids=_ids)
def test_norm_backward(case, from_ckpt, dtype):
    shape, pad, shift = case
    x = _normal(shape, 4, dtype)
    dy = _normal(shape, 5, dtype)
    w = _normal(shape[1:2], 6)
    xd, xg = guarded(x, pad, shift)
    dyd, dyg = guarded(dy, pad, shift)
    dxd, dxg = guarded(torch.zeros_like(x), pad, shift)
    _, m, r = norm_forward(x, w, None, EPS)
    mean, rstd = m.float().cuda(), r.float().cuda()
    dw, db = (torch.full(shape[1:2], GUARD, device="cuda") for _ in range(2))
    ws = torch.full((ftp.ftp_norm_workspace_bytes(x),), 255, dtype=torch.uint8, device="cuda")      # NaNs, if read before written
    src = xd
    x64 = x
    ckpt = None
    if from_ckpt:
        ckpt = torch.empty(ftp.ftp_ckpt_bytes(x), dtype=torch.uint8, device="cuda")
        ftp.ftp_ckpt_save(xd, ckpt)
        x64 = torch.from_numpy(eight_bits(x, _run(shape))[0])
        src = None
    ftp.ftp_norm_backward(src, dyd, w.cuda(), mean, rstd, dxd, dw, db, ws, ckpt=ckpt)
    dx, dw64, db64, dx_size, dw_size, db_size = norm_backward(x64, dy, w, mean, rstd)
    # row sums: trees of at most 8 + 8 + 5 + 5 levels, then five operations: 64 half-units of the terms' magnitude.  Column sums: at most
    # one thread adds all rows (and the vector's pixels) in turn.
    close(rows(dxd), dx, HALF_STEP[dtype] * dx.abs() + TINY[dtype] + 64 * U * dx_size, "dx")
    n = int(np.prod(_rows_of(shape)))
    close(dw, dw64, (n + 32) * U * dw_size, "dweight")
    close(db, db64, (n + 32) * U * db_size, "dbias")
    xg(), dyg(), dxg()
    # dx in dy's place; dx alone; the sums alone: the same bits
    dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
    ftp.ftp_norm_backward(src, dyd, w.cuda(), mean, rstd, None, dw2, db2, ws, ckpt=ckpt)
    assert torch.equal(dw, dw2) and torch.equal(db, db2)
    dx2 = torch.empty_like(dxd)
    if pad == 0 and shift == 0:
        ftp.ftp_norm_backward(src, dyd, w.cuda(), mean, rstd, dx2, None, None, None, ckpt=ckpt)
        assert torch.equal(dx2, dxd)
    ftp.ftp_norm_backward(src, dyd, w.cuda(), mean, rstd, dyd, dw2, db2, ws, ckpt=ckpt)
    assert torch.equal(dyd, dxd) and torch.equal(dw, dw2)
    dyg()


# maps of a whole tile and a part of one, whose channels leave the last warp of a block fewer than the others have (from 15 channels in
# two warps to 1000 in 32)
UNEVEN = [((1, 15, 11, 12), 0, 0), ((2, 31, 7, 10), 0, 0), ((1, 60, 11, 12), 0, 0), ((2, 125, 7, 10), 0, 0), ((2, 250, 7, 10), 0, 0),
          ((2, 500, 7, 10), 0, 0), ((2, 500, 7, 10), 2, 1), ((1, 1000, 7, 10), 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", UNEVEN, ids=_ids)
def test_norm_of_maps_whose_last_warp_has_fewer_channels(case, dtype):
    test_norm_forward(case, dtype)
    for from_ckpt in (False, True):
        test_norm_backward(case, from_ckpt, dtype)


# two pixels a lane in 16 bits with more than 128 channels, and maps of 513 to 1024 channels, which the forward pass gives to a block
# of up to 32 warps
WIDE = [((3, 160, 7, 10), 0, 0), ((2, 300, 7, 10), 0, 0), ((1, 512, 7, 10), 4, 2), ((1, 640, 9, 9), 3, 1), ((1, 700, 7, 10), 0, 0), ((1, 1024, 6, 12), 0, 0)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", WIDE, ids=_ids)
def test_norm_of_maps_of_many_channels(case, dtype):
    test_norm_forward(case, dtype)
    for from_ckpt in (False, True):
        test_norm_backward(case, from_ckpt, dtype)
    test_ckpt_is_defined_to_the_bit(case, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", SHAPES + UNEVEN + WIDE, ids=_ids)
def test_norm_backward_in_the_place_of_x(case, dtype):
    """dx written over x: the same bits as in a place of its own, in each form of the kernel."""
    shape, pad, shift = case
    x, dy, w = _normal(shape, 13, dtype), _normal(shape, 14, dtype), _normal(shape[1:2], 15).cuda()
    (xd, xg), (dyd, _), (dx, _) = guarded(x, pad, shift), guarded(dy, pad, shift), guarded(torch.zeros_like(x), pad, shift)
    _, m, r = norm_forward(x, w, None, EPS)
    ws = torch.empty(ftp.ftp_norm_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    sums = [torch.empty_like(w) for _ in range(4)]
    for to, dw, db in ((dx, *sums[:2]), (xd, *sums[2:])):
        ftp.ftp_norm_backward(xd, dyd, w, m.float().cuda(), r.float().cuda(), to, dw, db, ws)
    assert torch.equal(xd, dx) and torch.equal(sums[0], sums[2]) and torch.equal(sums[1], sums[3])
    xg()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", [((7, 65, 1, 1), 3, 1), ((300, 24, 1, 1), 0, 0)], ids=_ids)
def test_maps_of_one_pixel_are_rows(case, dtype):
    test_norm_forward(case, dtype)
    for from_ckpt in (False, True):
        test_norm_backward(case, from_ckpt, dtype)
    test_ckpt_is_defined_to_the_bit(case, dtype)
    test_logprob(case, dtype)
    test_logprob_backward(case, dtype)
    test_loss_logprob(case, dtype)


@pytest.mark.parametrize("shape", [(6, 40), (2, 6, 5, 3)])
def test_norm_gradients_against_differences(shape):
    """dx, dweight and dbias against central differences of sum(y t) of the plain forward pass in 64 bits."""
    x, t, w, b = _normal(shape, 7), _normal(shape, 8), _normal(shape[1:2], 9), _normal(shape[1:2], 10)
    mean, rstd = (torch.empty(_rows_of(shape), device="cuda") for _ in range(2))
    y, dx = torch.empty(shape, device="cuda"), torch.empty(shape, device="cuda")
    dw, db = torch.empty(shape[1], device="cuda"), torch.empty(shape[1], device="cuda")
    ws = torch.empty(ftp.ftp_norm_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    ftp.ftp_norm_forward(x.cuda(), w.cuda(), b.cuda(), y, mean, rstd, eps=EPS)
    ftp.ftp_norm_backward(x.cuda(), t.cuda(), w.cuda(), mean, rstd, dx, dw, db, ws)
    f = lambda x, w, b: float((norm_forward(x, w, b, EPS)[0] * rows(t)).sum())          # noqa: E731
    h = 1e-4                                                   # the quotient is off by order h^2 and 2^-53 / h: below 1e-6
    for name, value, got in (("x", x.double(), dx), ("w", w.double(), dw), ("b", b.double(), db)):
        flat, args = value.reshape(-1), {"x": x.double(), "w": w.double(), "b": b.double()}
        for i in range(0, flat.numel(), max(1, flat.numel() // 12)):
            up, down = flat.clone(), flat.clone()
            up[i] += h
            down[i] -= h
            d = (f(**{**args, name: up.view(value.shape)}) - f(**{**args, name: down.view(value.shape)})) / (2 * h)
            assert abs(d - float(got.reshape(-1)[i])) <= 2e-5 * max(1.0, float(got.abs().max())), (name, i)


@pytest.mark.parametrize("shape", [(5, 300), (2, 12, 9, 4)])
def test_norm_keeps_a_nan_in_its_row(shape):
    x = _normal(shape, 11)
    x.reshape(-1)[7] = float("nan")
    y = torch.empty(shape, device="cuda")
    ftp.ftp_norm_forward(x.cuda(), None, None, y, eps=EPS)
    assert torch.equal(torch.isnan(rows(y)).any(1), torch.isnan(rows(x)).any(1))
    assert torch.equal(torch.isnan(rows(y)).all(1), torch.isnan(rows(x)).any(1))


def test_norm_of_rows_far_from_zero():
    """(x - mean)^2 is summed, not x^2 - mean^2: values 1000 +- 1 keep their variance."""
    for shape in ((8, 512), (2, 32, 6, 6)):
        x = _normal(shape, 12) + 1000
        mean, rstd = (torch.empty(_rows_of(shape), device="cuda") for _ in range(2))
        y = torch.empty(shape, device="cuda")
        ftp.ftp_norm_forward(x.cuda(), None, None, y, mean, rstd, eps=EPS)
        y64, _, r = norm_forward(x, None, None, EPS)
        # the mean is off by 32 half-units of 1000, 2e-3, in units of the deviation: squared in the variance
        close(rstd, r, 1e-5 * r, "rstd")
        close(rows(y), y64, 32 * U * 1000 * 2 + 1e-4, "y")


def _same(a, b):
    """Equal values, NaN in the same places (an fp16 drawn here may be infinite, and comes back as NaN)."""
    a, b = a.cpu(), b.cpu()
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a[~torch.isnan(a)], b[~torch.isnan(b)])


# ---- checkpoint -----------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", SHAPES, ids=_ids)
def test_ckpt_is_defined_to_the_bit(case, dtype):
    shape, pad, shift = case
    x = (_normal(shape, 20) * torch.exp2(6 * _normal(shape, 21))).to(dtype)
    flat = x.reshape(-1)
    flat[::13] = 0
    xd, xg = guarded(x, pad, shift)
    ckpt = torch.full((ftp.ftp_ckpt_bytes(x) + 64,), 77, dtype=torch.uint8, device="cuda")
    ftp.ftp_ckpt_save(xd, ckpt)
    values, q, exponents = eight_bits(x, _run(shape))
    raw = ckpt.cpu().numpy()
    assert np.array_equal(raw[:q.size].view(np.int8), q.reshape(-1))
    assert np.array_equal(raw[q.size:q.size + exponents.size], exponents)
    assert (raw[q.size + exponents.size:] == 77).all() and q.size + exponents.size == ftp.ftp_ckpt_bytes(x)
    back, bg = guarded(torch.zeros_like(x), pad, shift)
    ftp.ftp_ckpt_load(ckpt, back)
    want = torch.from_numpy(values).to(dtype)
    assert _same(back, want)
    xg(), bg()
    for other in TYPES:
        o = torch.empty(shape, dtype=other, device="cuda")
        ftp.ftp_ckpt_load(ckpt, o)
        assert _same(o, torch.from_numpy(values).float().to(other))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("run", [(4, 96), (3, 45), (2, 2500), (3, 5003), (1, 9001), (2, 3, 7, 9)])
def test_ckpt_special_values(run, shift, dtype):
    """Blocks with infinities, NaNs and the largest values, from the call and from the norm's forward pass in place."""
    x = _normal(run, 22).to(dtype)
    f = x.reshape(-1)
    top = torch.finfo(dtype).max
    f[0], f[5], f[11] = float("inf"), float("nan"), -float("inf")
    f[33], f[34] = top, -top
    f[35] = torch.finfo(dtype).tiny
    f[-1], f[f.numel() // 2] = float("nan"), float("inf")
    xd, xg = guarded(x, 0, shift)
    ckpt = torch.empty(ftp.ftp_ckpt_bytes(x), dtype=torch.uint8, device="cuda")
    ftp.ftp_ckpt_save(xd, ckpt)
    there, tg = guarded(x, 0, shift)
    beside = torch.empty_like(ckpt)
    ftp.ftp_norm_forward(there, None, None, there, ckpt=beside)
    assert torch.equal(ckpt, beside)
    tg()
    back, bg = guarded(torch.zeros_like(x), 0, shift)
    ftp.ftp_ckpt_load(ckpt, back)
    xg(), bg()
    want = torch.from_numpy(eight_bits(x, _run(run))[0]).to(dtype)
    assert _same(back, want)
    assert torch.isfinite(back.cpu()[torch.isfinite(x)]).all()


def test_ckpt_of_the_smallest_values():
    x = torch.tensor([2.0 ** -126, 2.0 ** -127, 2.0 ** -128, 3 * 2.0 ** -127, 2.0 ** -149, 0.0, -(2.0 ** -126)]).reshape(1, 7)
    ckpt = torch.empty(ftp.ftp_ckpt_bytes(x), dtype=torch.uint8, device="cuda")
    ftp.ftp_ckpt_save(x.cuda(), ckpt)
    back = torch.empty((1, 7), device="cuda")
    ftp.ftp_ckpt_load(ckpt, back)
    assert torch.equal(back.cpu(), torch.from_numpy(eight_bits(x, 7)[0]).float())


# ---- log probabilities ----------------------------------------------------------------------------------------------

CLASSES = [
    ((1, 1), 0, 0), ((4, 2), 0, 0), ((3, 5), 2, 1), ((65, 32), 0, 0), ((9, 33), 0, 0), ((1, 1000), 0, 0), ((40, 1000), 8, 0), ((7, 1025), 0, 3),
    ((5, 2049), 0, 0), ((3, 4097), 1, 1), ((2, 20011), 0, 0), ((1, 32000), 0, 0), ((310, 5000), 0, 0), ((1, 131072), 0, 0), ((2, 131071), 0, 0),
    ((1, 260000), 0, 1), ((1800, 2500), 0, 0), ((1777, 2311), 0, 1), ((24, 93590), 8, 0), ((30, 22001), 0, 0),
    ((150, 10007), 1, 0), ((1184, 2100), 0, 0), ((90, 40001), 1, 5), ((450, 33001), 0, 5),
    ((1, 2, 1, 3), 0, 0), ((2, 21, 8, 8), 0, 0), ((2, 80, 13, 13), 0, 0), ((1, 300, 9, 12), 8, 0), ((3, 70, 5, 5), 3, 1), ((1, 1500, 3, 4), 0, 0),
]


def _logits(shape, seed, dtype):
    """Logits with equal values among them, ruled-out classes, rows of one value, of the lowest value, and with nothing left."""
    z = (3 * _normal(shape, seed)).to(dtype)
    r = z.movedim(1, -1).reshape(-1, shape[1]).clone()
    gen = torch.Generator().manual_seed(seed + 1)
    r[torch.rand(r.shape, generator=gen) < 0.1] = -float("inf")
    n = r.shape[0]
    if n >= 4:
        r[1] = 2.5                                            # all equal
        r[2] = -float("inf")                                  # nothing left
        r[3] = torch.finfo(dtype).min                         # masked with the lowest value
    if n >= 8:
        r[4, : max(1, shape[1] // 2)] = torch.finfo(dtype).min
        r[5] = (torch.arange(shape[1]) % 3).to(dtype)         # many equal ones
    labels = torch.randint(0, shape[1], (n,), generator=gen)
    labels[::5] = -1
    if n >= 8:
        labels[6] = shape[1]                                  # out of range
    return like(r, shape).contiguous(), labels.reshape(_rows_of(shape))


def _lse_bound(z, d):
    """Half-units: the difference z - m, its product with log2 e (relative to the exponent, weighted with p), the exponential (2 units), a
    tree of 32 + 16 levels, the logarithm; and for lse the rounding of the sum with m."""
    return 128 * U


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CLASSES, ids=_ids)
def test_logprob(case, dtype):
    shape, pad, shift = case
    z, labels = _logits(shape, 30, dtype)
    zd, zg = guarded(z, pad, shift)
    out = {k: torch.full(_rows_of(shape), GUARD, device="cuda") for k in ("logp", "lse", "entropy")}
    top = min(shape[1], 20 if shape[0] % 2 else 7)
    tshape = (shape[0], top) + tuple(shape[2:])
    tl, ti = torch.full(tshape, GUARD, device="cuda"), torch.full(tshape, -5, dtype=torch.int64, device="cuda")
    ftp.ftp_logprob(zd, labels.cuda(), top_logp=tl, top_index=ti, **out)
    want, d, p = logprob(z, labels, top)
    assert torch.equal(rows(ti).long(), want["top_index"]), "top_index"
    e = _lse_bound(z, d)
    fin = torch.where(torch.isfinite(want["lse"]), want["lse"].abs(), torch.zeros(()).double())
    close(out["lse"], want["lse"], e + U * fin, "lse")
    lab = torch.where(torch.isfinite(want["logp"]), want["logp"].abs(), torch.zeros(()).double())
    close(out["logp"], want["logp"], e + 2 * U * lab, "logp")
    # entropy = log s - (t / s) log 2: each part up to log c and the mean exponent, 32 + 16 levels
    spread = torch.where(p > 0, p * d.abs(), 0.0).sum(1) + np.log(shape[1]) + 1
    close(out["entropy"], want["entropy"], e * spread, "entropy")
    tfin = torch.where(torch.isfinite(want["top_logp"]), want["top_logp"].abs(), torch.zeros(()).double())
    close(rows(tl), want["top_logp"], e + 2 * U * tfin, "top_logp")
    zg()
    # each output alone, and no best classes
    for k, v in out.items():
        alone = torch.full_like(v, GUARD)
        ftp.ftp_logprob(zd, labels.cuda() if k == "logp" else None, **{k: alone})
        close(alone, v, 0 if len(shape) == 2 else 2 * e * (1 + v.double().abs().nan_to_num(0, 0, 0)), k)
    one = torch.empty((shape[0], 1) + tuple(shape[2:]), dtype=torch.int64, device="cuda")
    ftp.ftp_logprob(zd, None, top_index=one)
    assert torch.equal(one.cpu(), ti[:, :1].cpu())


@pytest.mark.parametrize("shape", [(4, 100), (4, 6000), (1, 140000), (1, 12, 2, 2)])
def test_logprob_of_rows_with_nan_or_infinity(shape):
    z = 3 * _normal(shape, 31)
    r = z.movedim(1, -1).reshape(-1, shape[1]).clone()
    r[0, shape[1] // 2] = float("nan")
    if r.shape[0] > 1:
        r[1, 3] = float("inf")
    z = like(r, shape).contiguous()
    labels = torch.zeros(_rows_of(shape), dtype=torch.int64)
    out = {k: torch.empty(_rows_of(shape), device="cuda") for k in ("logp", "lse", "entropy")}
    ti = torch.empty((shape[0], 5) + tuple(shape[2:]), dtype=torch.int64, device="cuda")
    ftp.ftp_logprob(z.cuda(), labels.cuda(), top_index=ti, **out)
    want, _, _ = logprob(z, labels, 5)
    for k, v in out.items():
        assert torch.equal(torch.isnan(v.cpu().reshape(-1)), torch.isnan(want[k])), k
    assert torch.equal(rows(ti).long(), want["top_index"])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CLASSES, ids=_ids)
def test_logprob_backward(case, dtype):
    shape, pad, shift = case
    z, labels = _logits(shape, 32, dtype)
    r = z.movedim(1, -1).reshape(-1, shape[1])
    if r.shape[0] >= 4:
        r[3] = 1.0                                            # (an lse of the lowest value holds no log c: see the header)
        if r.shape[0] >= 8:
            r[4] = 0.5
        z = like(r, shape).contiguous()
    want, d, p = logprob(z, labels, 1)
    zd, zg = guarded(z, pad, shift)
    dz, dg = guarded(torch.zeros_like(z), pad, shift)
    lse, h = want["lse"].float(), want["entropy"].float()
    gl, gh = _normal((r.shape[0],), 33), _normal((r.shape[0],), 34)
    dev = lambda v: v.reshape(_rows_of(shape)).cuda()         # noqa: E731
    ftp.ftp_logprob_backward(zd, labels.cuda(), dev(lse), dev(h), dev(gl), dev(gh), dz)
    lab = labels.reshape(-1)
    wl = torch.where(lab < 0, 0.0, torch.where(lab >= shape[1], torch.nan, gl.double()))[:, None]
    hit = torch.arange(shape[1])[None] == lab[:, None]
    zr = rows(z)
    lp = torch.where(torch.isinf(lse[:, None]), -torch.inf, zr - lse.double()[:, None])
    pp = torch.exp(lp)
    want_d = torch.where(hit, wl, 0.0) - pp * wl - gh.double()[:, None] * torch.where(pp > 0, pp * (lp + h.double()[:, None]), 0.0)
    want_d = torch.where(torch.isinf(lse)[:, None], 0.0, torch.where(torch.isnan(wl), torch.nan, want_d))
    # z - lse is off by half a unit of the larger of them, the exponent by that and half a unit of itself, the exponential by two units
    lpf = torch.where(torch.isfinite(lp), lp, 0.0)
    rel = U * (8 + 2 * lse.double().abs().nan_to_num(0, 0, 0)[:, None] + 3 * lpf.abs())
    size = hit * wl.abs().nan_to_num() + pp * (wl.abs().nan_to_num() + gh.double().abs()[:, None] * (lpf.abs() + h.double()[:, None] + 1))
    close(rows(dz), want_d, HALF_STEP[dtype] * want_d.abs().nan_to_num() + TINY[dtype] + 2 * rel * size + 2.0 ** -140, "dlogits")
    zg(), dg()
    # one of the deltas alone, in place
    ftp.ftp_logprob_backward(zd, None, dev(lse), dev(h), None, dev(gh), dz)
    only = torch.where(torch.isinf(lse)[:, None], 0.0, -gh.double()[:, None] * torch.where(pp > 0, pp * (lp + h.double()[:, None]), 0.0))
    close(rows(dz), only, HALF_STEP[dtype] * only.abs() + TINY[dtype] + 2 * rel * size + 2.0 ** -140, "dentropy alone")
    ftp.ftp_logprob_backward(zd, None, dev(lse), dev(h), None, dev(gh), zd)
    assert torch.equal(zd, dz)
    zg()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", CLASSES + [((5000, 10), 0, 0), ((3, 4, 60, 61), 0, 0)], ids=_ids)
def test_loss_logprob(case, dtype):
    shape, pad, shift = case
    z, labels = _logits(shape, 35, dtype)
    n = labels.numel()
    lab = labels.reshape(-1)
    lab[lab >= shape[1]] = 0
    if n >= 4:
        lab[2] = -1                                           # a row with nothing left would make the loss infinite
    r = z.movedim(1, -1).reshape(-1, shape[1])
    for i in range(n):
        if lab[i] >= 0 and r[i, lab[i]] < -1e30:
            lab[i] = int(r[i].argmax())                       # nor a label that is ruled out
    zd, zg = guarded(z, pad, shift)
    dz, dg = guarded(torch.zeros_like(z), pad, shift)
    loss = torch.full((1,), GUARD, device="cuda")
    ws = torch.full((ftp.ftp_loss_logprob_workspace_bytes(z),), 255, dtype=torch.uint8, device="cuda")
    scale = 1024.0
    ftp.ftp_loss_logprob(zd, labels.cuda(), dz, loss, ws, scale=scale)
    want, d, p = logprob(z, labels, 1)
    known = lab >= 0
    m = max(1, int(known.sum()))
    hit = torch.arange(shape[1])[None] == lab[:, None]
    want_d = torch.where(known[:, None], (p - hit.double()) * (scale / m), 0.0)
    df = torch.where(torch.isfinite(d), d, 0.0)
    bound = HALF_STEP[dtype] * want_d.abs() + TINY[dtype] + U * (64 + 4 * df.abs()) * (p + hit) * known[:, None] * (scale / m) + 2.0 ** -140
    close(rows(dz), want_d, bound, "dlogits")
    terms = want["logp"][known].abs().sum() / m
    close(loss[0], -want["logp"][known].sum() / m, (128 + 16 + n) * U * (terms + 1), "loss")
    zg(), dg()
    # loss alone, delta alone, delta in the logits' place: the same bits
    loss2, dz2 = torch.empty_like(loss), torch.empty_like(dz)
    ftp.ftp_loss_logprob(zd, labels.cuda(), None, loss2, ws, scale=scale)
    ftp.ftp_loss_logprob(zd, labels.cuda(), zd, None, ws, scale=scale)
    assert torch.equal(loss, loss2) and torch.equal(zd, dz)
    zg()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape, shift", [((5000, 10), 0), ((3001, 33), 1), ((2000, 479), 0), ((700, 1000), 3), ((300, 2048), 0), ((90, 5003), 1),
                                          ((9, 40001), 0), ((2, 21, 40, 50), 0), ((3, 70, 9, 9), 1), ((1, 700, 8, 6), 0)])
def test_loss_and_delta_in_the_logits_place_in_one_call(shape, shift, dtype):
    """The loss reads the label's logit where another thread writes its delta: the same bits as with a place for the delta."""
    z = (3 * _normal(shape, 38)).to(dtype)
    labels = torch.randint(0, shape[1], _rows_of(shape), generator=torch.Generator().manual_seed(8)).cuda()
    zd, zg = guarded(z, 0, shift)
    dz, dg = guarded(torch.zeros_like(z), 0, shift)
    ws = torch.empty(ftp.ftp_loss_logprob_workspace_bytes(z), dtype=torch.uint8, device="cuda")
    loss, want = torch.full((1,), GUARD, device="cuda"), torch.full((1,), GUARD, device="cuda")
    ftp.ftp_loss_logprob(zd, labels, dz, want, ws, scale=64.0)
    for _ in range(8):
        zd.copy_(z)
        ftp.ftp_loss_logprob(zd, labels, zd, loss, ws, scale=64.0)
        assert torch.equal(loss, want) and torch.equal(zd, dz)
    zg(), dg()


def test_loss_without_a_labelled_row_and_with_ruled_out_ones():
    for shape in ((6, 50), (2, 5, 3, 3)):
        z = _normal(shape, 36).cuda()
        none = torch.full(_rows_of(shape), -1, dtype=torch.int64, device="cuda")
        ws = torch.empty(ftp.ftp_loss_logprob_workspace_bytes(z), dtype=torch.uint8, device="cuda")
        loss, dz = torch.full((1,), GUARD, device="cuda"), torch.full(shape, GUARD, device="cuda")
        ftp.ftp_loss_logprob(z, none, dz, loss, ws)
        assert loss.item() == 0.0 and not dz.any()
        z.movedim(1, -1)[0].reshape(-1, shape[1])[:] = -float("inf")
        if len(shape) == 4:
            z[0] = -float("inf")
        ftp.ftp_loss_logprob(z, none + 1, dz, loss, ws)
        assert loss.item() == float("inf") and torch.isfinite(dz).all() and not dz[0].any()
        ftp.ftp_loss_logprob(z, none + 1 + shape[1], dz, loss, ws)
        assert torch.isnan(loss).all() and torch.isnan(dz).all()


@pytest.mark.parametrize("shape", [(5, 9), (1, 4, 3, 2)])
def test_loss_gradient_against_differences(shape):
    z = _normal(shape, 37)
    labels = torch.randint(0, shape[1], _rows_of(shape), generator=torch.Generator().manual_seed(1))
    dz, loss = torch.empty(shape, device="cuda"), torch.empty(1, device="cuda")
    ws = torch.empty(ftp.ftp_loss_logprob_workspace_bytes(z), dtype=torch.uint8, device="cuda")
    ftp.ftp_loss_logprob(z.cuda(), labels.cuda(), dz, loss, ws)
    f = lambda v: -float(logprob(v.view(shape), labels, 1)[0]["logp"].mean())       # noqa: E731
    flat, h = z.double().reshape(-1), 1e-4
    for i in range(flat.numel()):
        up, down = flat.clone(), flat.clone()
        up[i] += h
        down[i] -= h
        assert abs((f(up) - f(down)) / (2 * h) - float(dz.reshape(-1)[i])) <= 1e-6


def test_backward_ckpt_is_load_forward_backward():
    from paper_2409_09083_b200 import synth
    for precision in (0, 1):
        plan = ftp.ftp_plan([synth.conv(16, 8, 3), synth.pool()], 2, 16, 20, 28, (2, 2), ((1, 2),), precision=precision)
        x, params, ws = _normal(plan.shape, 50).cuda(), 0.3 * _normal((plan.param_floats,), 51).cuda(), plan.new_workspace()
        dy = _normal((plan.out_floats,), 52).cuda()
        ckpt = torch.empty(ftp.ftp_ckpt_bytes(x), dtype=torch.uint8, device="cuda")
        ftp.ftp_ckpt_save(x, ckpt)
        got, want = ([torch.empty_like(x), torch.empty_like(x), torch.empty_like(params)] for _ in range(2))
        ftp.ftp_backward_ckpt(plan, ckpt, got[0], dy, params, got[1], got[2], ws)
        ftp.ftp_ckpt_load(ckpt, want[0])
        ftp.ftp_forward(plan, want[0], params, None, ws)
        ftp.ftp_backward(plan, want[0], dy, params, want[1], want[2], ws)
        for a, b in zip(got, want):
            assert torch.equal(a, b)


# ---- streams, graphs, order -----------------------------------------------------------------------------------------

def _everything(x, dy, w, labels, out):
    ftp.ftp_norm_forward(x, w, w, out["y"], out["mean"], out["rstd"], ckpt=out["ckpt"])
    ftp.ftp_loss_logprob(out["y"], labels, out["dz"], out["loss"], out["lws"])
    ftp.ftp_logprob(out["y"], labels, out["logp"], out["lse"], out["entropy"], out["tl"], out["ti"])
    ftp.ftp_logprob_backward(out["y"], labels, out["lse"], out["entropy"], dy[:, 0], out["logp"], out["dz2"])
    ftp.ftp_norm_backward(None, out["dz"], w, out["mean"], out["rstd"], out["dx"], out["dw"], out["db"], out["nws"], ckpt=out["ckpt"])
    ftp.ftp_ckpt_load(out["ckpt"], out["back"])


def _buffers(x, labels):
    rs = labels.shape
    out = {k: torch.empty_like(x) for k in ("y", "dz", "dz2", "dx", "back")}
    out |= {k: torch.empty(rs, device="cuda") for k in ("mean", "rstd", "logp", "lse", "entropy")}
    out |= {"tl": torch.empty((x.shape[0], 4) + x.shape[2:], device="cuda"),
            "ti": torch.empty((x.shape[0], 4) + x.shape[2:], device="cuda", dtype=torch.int64),
            "loss": torch.empty(1, device="cuda"), "dw": torch.empty(x.shape[1], device="cuda"), "db": torch.empty(x.shape[1], device="cuda"),
            "ckpt": torch.empty(ftp.ftp_ckpt_bytes(x), device="cuda", dtype=torch.uint8),
            "nws": torch.empty(ftp.ftp_norm_workspace_bytes(x), device="cuda", dtype=torch.uint8),
            "lws": torch.empty(ftp.ftp_loss_logprob_workspace_bytes(x), device="cuda", dtype=torch.uint8)}
    return out


_RESULTS = ("y", "dz", "dz2", "dx", "back", "mean", "rstd", "logp", "lse", "entropy", "tl", "ti", "loss", "dw", "db", "ckpt")


@pytest.mark.parametrize("shape", [(600, 1003), (3, 5000), (1, 130000), (3, 40, 19, 19)])
def test_graph_side_stream_and_repeat_give_the_same_bits(shape):
    labels = torch.randint(-1, shape[1], _rows_of(shape), generator=torch.Generator().manual_seed(2)).cuda()
    w = _normal(shape[1:2], 40).cuda()
    x, dy = _normal(shape, 41).cuda(), _normal(shape, 42).cuda()
    dy0 = dy.select(1, 0).contiguous()
    pack = dy0.unsqueeze(1)                                   # dy[:, 0] of _everything: one delta for each row
    first = _buffers(x, labels)
    _everything(x, pack, w, labels, first)
    again = _buffers(x, labels)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _everything(x, pack, w, labels, again)
    torch.cuda.synchronize()
    held = _buffers(x, labels)
    xs = torch.zeros_like(x)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _everything(xs, pack, w, labels, held)
    xs.copy_(x)
    g.replay()
    torch.cuda.synchronize()
    for k in _RESULTS:
        assert torch.equal(first[k], again[k]), k
        assert torch.equal(first[k], held[k]), k


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(6, 372), (40, 1111), (3, 5001), (2, 9001), (2, 40, 10, 6)])
def test_arrays_of_different_alignment(shape, dtype):
    """Every array another distance off the 16-byte grid, and another stride between samples: the same results as dense ones."""
    x, dy, w = _normal(shape, 60, dtype), _normal(shape, 61, dtype), _normal(shape[1:2], 62).cuda()
    labels = torch.randint(-1, shape[1], _rows_of(shape), generator=torch.Generator().manual_seed(3)).cuda()
    dense = _buffers(x.cuda(), labels)
    ftp.ftp_norm_forward(x.cuda(), w, w, dense["y"], dense["mean"], dense["rstd"])
    ftp.ftp_norm_backward(x.cuda(), dy.cuda(), w, dense["mean"], dense["rstd"], dense["dx"], dense["dw"], dense["db"], dense["nws"])
    ftp.ftp_logprob(x.cuda(), labels, dense["logp"], dense["lse"], dense["entropy"])
    ftp.ftp_loss_logprob(x.cuda(), labels, dense["dz"], dense["loss"], dense["lws"], scale=100.0)
    ftp.ftp_logprob_backward(x.cuda(), labels, dense["lse"], dense["entropy"], dense["mean"], dense["rstd"], dense["dz2"])
    xd, xg = guarded(x, 3, 1)
    dyd, dyg = guarded(dy, 6, 2)
    outs = [guarded(torch.zeros_like(x), pad, shift) for pad, shift in ((0, 3), (5, 0), (1, 5), (2, 6))]
    (y, yg), (dx, dxg), (dz, dzg), (dz2, dz2g) = outs
    got = _buffers(x.cuda(), labels)
    u = HALF_STEP[dtype]
    ftp.ftp_norm_forward(xd, w, w, y, got["mean"], got["rstd"])
    ftp.ftp_norm_backward(xd, dyd, w, dense["mean"], dense["rstd"], dx, got["dw"], got["db"], got["nws"])
    ftp.ftp_loss_logprob(xd, labels, dz, got["loss"], got["lws"], scale=100.0)
    ftp.ftp_logprob_backward(xd, labels, dense["lse"], dense["entropy"], dense["mean"], dense["rstd"], dz2)
    # other kernels, other orders of the same sums: both are within 64 half-units of the terms' magnitude and half a step of the type
    for a, b, size in ((y, dense["y"], 8.0), (dx, dense["dx"], 30.0), (dz, dense["dz"], 100.0 / max(1, int((labels >= 0).sum()))), (dz2, dense["dz2"], 30.0)):
        a, b = a.cpu().double(), b.cpu().double()
        assert ((a - b).abs() <= 2 * (u * b.abs() + TINY[dtype] + 64 * U * size)).all()
    terms = float((dy.double().abs()).sum())
    assert (got["dw"] - dense["dw"]).abs().max() <= 2e-5 * terms and (got["db"] - dense["db"]).abs().max() <= 2e-5 * terms
    assert abs(got["loss"].item() - dense["loss"].item()) <= 1e-5 * (1 + abs(dense["loss"].item()))
    for check in (xg, dyg, yg, dxg, dzg, dz2g):
        check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", [(6, 372), (40, 1111), (3, 5001), (2, 9001), (700, 33), (2, 40, 10, 6), (3, 33, 5, 7)])
def test_column_sums_and_loss_of_arrays_of_different_alignment(shape, dtype):
    """Every array another distance off the 16-byte grid: each column's sums to the rounding of its own terms, the loss to that of its rows."""
    x, dy, w = _normal(shape, 63, dtype), _normal(shape, 64, dtype), _normal(shape[1:2], 65)
    labels = torch.randint(-1, shape[1], _rows_of(shape), generator=torch.Generator().manual_seed(4))
    _, m, r = norm_forward(x, w, None, EPS)
    mean, rstd = m.float().cuda(), r.float().cuda()
    n = labels.numel()
    want, d, p = logprob(x, labels, 1)
    known = labels.reshape(-1) >= 0
    count = max(1, int(known.sum()))
    hit = torch.arange(shape[1])[None] == labels.reshape(-1, 1)
    for (px, sx), (py, sy), (po, so) in (((3, 1), (6, 2), (5, 0)), ((0, 0), (1, 3), (2, 6)), ((2, 5), (0, 0), (0, 1)), ((1, 7), (8, 7), (3, 4))):
        (xd, xg), (dyd, dyg), (dx, dxg) = guarded(x, px, sx), guarded(dy, py, sy), guarded(torch.zeros_like(x), po, so)
        dw, db, loss = torch.full(shape[1:2], GUARD, device="cuda"), torch.full(shape[1:2], GUARD, device="cuda"), torch.full((1,), GUARD, device="cuda")
        ws = torch.full((ftp.ftp_norm_workspace_bytes(x),), 255, dtype=torch.uint8, device="cuda")
        ftp.ftp_norm_backward(xd, dyd, w.cuda(), mean, rstd, dx, dw, db, ws)
        dx64, dw64, db64, dx_size, dw_size, db_size = norm_backward(x, dy, w, mean, rstd)
        # (the bounds of the aligned arrays: row sums in trees, at most one thread adds all rows of a column in turn)
        close(rows(dx), dx64, HALF_STEP[dtype] * dx64.abs() + TINY[dtype] + 64 * U * dx_size, "dx")
        close(dw, dw64, (n + 32) * U * dw_size, "dweight")
        close(db, db64, (n + 32) * U * db_size, "dbias")
        lws = torch.full((ftp.ftp_loss_logprob_workspace_bytes(x),), 255, dtype=torch.uint8, device="cuda")
        dz, dzg = guarded(torch.zeros_like(x), po, so)
        ftp.ftp_loss_logprob(xd, labels.cuda(), dz, loss, lws)
        want_d = torch.where(known[:, None], (p - hit.double()) / count, 0.0)
        bound = HALF_STEP[dtype] * want_d.abs() + TINY[dtype] + U * (64 + 4 * d.abs()) * (p + hit) * known[:, None] / count + 2.0 ** -140
        close(rows(dz), want_d, bound, "dlogits")
        terms = want["logp"][known].abs().sum() / count
        close(loss[0], -want["logp"][known].sum() / count, (128 + 16 + n) * U * (terms + 1), "loss")
        for check in (xg, dyg, dxg, dzg):
            check()


def test_offsets_past_32_bits():
    """Five samples 2^29 + 8 values apart: the last one starts past 2^31 values and 2^32 bytes."""
    stride, n = (1 << 29) + 8, 5
    whole = torch.empty((n - 1) * stride + 4096, dtype=torch.float16, device="cuda")
    for shape in ((n, 1003), (n, 12, 10, 9)):
        per = int(np.prod(shape[1:]))
        view = torch.as_strided(whole, (n, per), (stride, 1))
        view = view if len(shape) == 2 else view.unflatten(1, shape[1:])
        x = _normal(shape, 70).half()
        view.copy_(x)
        labels = torch.zeros(_rows_of(shape), dtype=torch.int64, device="cuda")
        want, got = _buffers(x.cuda(), labels), _buffers(x.cuda(), labels)
        for out, src in ((want, x.cuda()), (got, view)):
            ftp.ftp_ckpt_save(src, out["ckpt"])
            ftp.ftp_logprob(src, labels, out["logp"], out["lse"], out["entropy"], out["tl"], out["ti"])
            ftp.ftp_norm_forward(src, None, None, src, out["mean"], out["rstd"])
            out["y"].copy_(src)
            ftp.ftp_norm_backward(None, src, None, out["mean"], out["rstd"], src, out["dw"], out["db"], out["nws"], ckpt=out["ckpt"])
            out["dx"].copy_(src)
            ftp.ftp_loss_logprob(src, labels, src, out["loss"], out["lws"])
            out["dz"].copy_(src)
            ftp.ftp_ckpt_load(out["ckpt"], src)
            out["back"].copy_(src)
        for k in ("ckpt", "logp", "lse", "entropy", "tl", "ti", "mean", "rstd", "y", "dx", "dw", "db", "loss", "dz", "back"):
            close(got[k], want[k], 1e-2 * (1 + want[k].double().abs()) if k in ("y", "dx", "dz", "loss", "dw", "db") else 4e-6 * (1 + want[k].double().abs()), k)


def test_two_streams_at_once():
    """Calls that share nothing but their inputs, on two streams with workspaces of their own."""
    shape = (700, 4000)
    x, dy, w = _normal(shape, 80).cuda(), _normal(shape, 81).cuda(), _normal(shape[1:2], 82).cuda()
    labels = torch.randint(0, shape[1], (shape[0],), generator=torch.Generator().manual_seed(5)).cuda()
    pack = dy[:, :1].contiguous()
    alone = _buffers(x, labels)
    _everything(x, pack, w, labels, alone)
    torch.cuda.synchronize()
    both = [_buffers(x, labels) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for out, s in zip(both, streams):
            with torch.cuda.stream(s):
                _everything(x, pack, w, labels, out)
    torch.cuda.synchronize()
    for out in both:
        for k in _RESULTS:
            assert torch.equal(out[k], alone[k]), k


def test_empty_arrays():
    w = torch.full((6,), GUARD, device="cuda")
    for shape in ((0, 6), (2, 6, 0, 3)):
        x = torch.empty(shape, device="cuda")
        labels = torch.empty(_rows_of(shape), dtype=torch.int64, device="cuda")
        stat = torch.empty(_rows_of(shape), device="cuda")
        ws = torch.empty(ftp.ftp_norm_workspace_bytes(x), dtype=torch.uint8, device="cuda")
        assert ftp.ftp_ckpt_bytes(x) == 0
        ftp.ftp_norm_forward(x, w, None, x, stat, stat)
        dw, db = w.clone(), w.clone()
        ftp.ftp_norm_backward(x, x, w, stat, stat, x, dw, db, ws)
        assert not dw.any() and not db.any()
        ftp.ftp_norm_backward(x, x, w, stat, stat, x, None, None, None)
        ftp.ftp_loss_logprob(x, labels, x, None, torch.empty(ftp.ftp_loss_logprob_workspace_bytes(x), dtype=torch.uint8, device="cuda"))
        ftp.ftp_logprob(x, labels, stat)
        ftp.ftp_logprob_backward(x, labels, stat, None, stat, None, x)
        loss = torch.full((1,), GUARD, device="cuda")
        ftp.ftp_loss_logprob(x, labels, x, loss, torch.empty(ftp.ftp_loss_logprob_workspace_bytes(x), dtype=torch.uint8, device="cuda"))
        assert loss.item() == 0.0


def test_the_first_calls_of_a_process_can_be_captured():
    """Launch sizes that a process asks the runtime for once, attributes and lazily loaded kernels: none needs a call before the capture."""
    code = """
import torch
import paper_2409_09083_b200 as ftp
gen = torch.Generator().manual_seed(5)
new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device="cuda")
z = torch.randn((90, 40001), generator=gen).cuda()
labels = torch.randint(0, 40001, (90,), generator=gen).cuda()
x, dy = torch.randn((60, 700), generator=gen).cuda(), torch.randn((60, 700), generator=gen).cuda()
ws, lws = (new(n, dtype=torch.uint8) for n in (ftp.ftp_norm_workspace_bytes(x), ftp.ftp_loss_logprob_workspace_bytes(z)))
def run(o):
    ftp.ftp_norm_forward(x, None, None, o[0], o[1], o[2], ckpt=o[3])
    ftp.ftp_ckpt_load(o[3], o[4])
    ftp.ftp_norm_backward(x, dy, None, o[1], o[2], o[5], o[6], o[7], ws)
    ftp.ftp_logprob(z, labels, logp=o[8], lse=o[9], top_logp=o[10], top_index=o[11])
    ftp.ftp_loss_logprob(z, labels, o[12], o[13], lws)
def outs():
    k = new(ftp.ftp_ckpt_bytes(x), dtype=torch.uint8)
    return [new(60, 700), new(60), new(60), k, new(60, 700), new(60, 700), new(700), new(700), new(90), new(90), new(90, 5),
            new(90, 5, dtype=torch.int64), new(90, 40001), new(1)]
held, eager = outs(), outs()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    run(held)
g.replay()
run(eager)
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(held, eager))
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=pathlib.Path(__file__).resolve().parents[1], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def _logprob_call(shape):
    z = _normal(shape, 90).cuda()
    labels = torch.randint(0, shape[1], shape[:1], generator=torch.Generator().manual_seed(6)).cuda()
    logp, index = torch.zeros(shape[0], device="cuda"), torch.zeros((shape[0], 4), dtype=torch.int64, device="cuda")
    return (logp, index), lambda: ftp.ftp_logprob(z, labels, logp, top_index=index)


def _loss_call(shape):
    z = _normal(shape, 91).cuda()
    labels = torch.randint(0, shape[1], shape[:1], generator=torch.Generator().manual_seed(7)).cuda()
    dz, loss = torch.zeros_like(z), torch.zeros(1, device="cuda")
    ws = torch.empty(ftp.ftp_loss_logprob_workspace_bytes(z), dtype=torch.uint8, device="cuda")
    return (dz, loss), lambda: ftp.ftp_loss_logprob(z, labels, dz, loss, ws)


def _norm_backward_call(shape):
    x, dy, w = _normal(shape, 92, torch.bfloat16).cuda(), _normal(shape, 93, torch.bfloat16).cuda(), _normal(shape[1:2], 94).cuda()
    mean, rstd = torch.zeros(shape[0], device="cuda"), torch.ones(shape[0], device="cuda")
    dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w)
    ws = torch.empty(ftp.ftp_norm_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    return (dx, dw, db), lambda: ftp.ftp_norm_backward(x, dy, w, mean, rstd, dx, dw, db, ws)


@pytest.mark.parametrize("make, shapes", [(_logprob_call, ((600, 4100), (80, 9000))), (_loss_call, ((600, 4100), (80, 9000))),
                                          (_norm_backward_call, ((40, 16384), (3, 8200)))], ids=["logprob", "loss", "norm backward"])
def test_two_host_threads_call_one_kernel_with_much_and_little_shared_memory(make, shapes, monkeypatch):
    """Calls of two threads share nothing but what both are given: what one asks of a kernel must not refuse the other one's launch.
    The threads loop over the C entry itself; the binding's own work would leave them little time next to one another."""
    want, threads, found, marshalled = [], [], [], []
    for shape in shapes:
        out, call = make(shape)
        call()
        want.append(out)
    start = threading.Barrier(2, timeout=60)

    def loop(entry, args, stream):
        start.wait()
        found.append([entry(*args, stream.cuda_stream) for _ in range(20000)])
    results = []
    for shape in shapes:
        out, call = make(shape)
        with monkeypatch.context() as m:
            m.setattr(ftp.binding, "_call", lambda entry, x, name, stream, *args: marshalled.append((entry, args)))
            call()
        results.append((out, call))                           # (the call holds its inputs)
        threads.append(threading.Thread(target=loop, args=marshalled[-1] + (torch.cuda.Stream(),)))
    torch.cuda.synchronize()
    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-5)                               # (about the length of a call)
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(interval)
    torch.cuda.synchronize()
    assert len(found) == 2
    refused = [sum(rc != 0 for rc in codes) for codes in found]
    assert refused == [0, 0], refused
    for (out, _), first in zip(results, want):
        assert all(torch.equal(a, b) for a, b in zip(out, first))


def test_a_refused_call_leaves_no_error_for_the_next_one():
    """The default stream takes nothing while another one is captured (in the mode that forbids it), and the capture is lost; the calls that
    follow are good ones.  In a process of its own, for the lost capture's sake."""
    code = """
import ctypes
import torch
import paper_2409_09083_b200 as ftp
z = torch.randn((90, 40001), device="cuda")
labels = torch.zeros(90, dtype=torch.int64, device="cuda")
dz, loss, none = torch.empty_like(z), torch.empty(1, device="cuda"), torch.empty((0, 40001), device="cuda")
lws = torch.empty(ftp.ftp_loss_logprob_workspace_bytes(z), dtype=torch.uint8, device="cuda")
nws = torch.empty(ftp.ftp_norm_workspace_bytes(z), dtype=torch.uint8, device="cuda")
dw, db, stat = torch.empty(40001, device="cuda"), torch.empty(40001, device="cuda"), torch.empty(0, device="cuda")
x, back = torch.randn((40, 70), device="cuda"), torch.empty((40, 70), device="cuda")
ckpt = torch.empty(ftp.ftp_ckpt_bytes(x), dtype=torch.uint8, device="cuda")
calls = [lambda: ftp.ftp_loss_logprob(z, labels, dz, loss, lws), lambda: ftp.ftp_loss_logprob(none, labels[:0], none, loss, lws),
         lambda: ftp.ftp_norm_backward(none, none, None, stat, stat, None, dw, db, nws)]
for call in calls:
    call()
torch.cuda.synchronize()
for call in calls:
    graph, handle = torch.cuda.CUDAGraph(), ctypes.c_void_p()
    torch.cuda.cudart().cudaStreamCreate(ctypes.addressof(handle))            # (torch's own do not stand back behind the default stream)
    side = torch.cuda.ExternalStream(handle.value)
    with torch.cuda.stream(side):
        graph.capture_begin()
    try:
        call()
        raise SystemExit("the call was not refused")
    except ftp.FtpError:
        pass
    with torch.cuda.stream(side):
        try:
            graph.capture_end()
        except RuntimeError:
            pass
    ftp.ftp_ckpt_save(x, ckpt)
    ftp.ftp_ckpt_load(ckpt, back)
    call()
    torch.cuda.synchronize()
    assert (back - x).abs().max() <= x.abs().max() / 127
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=pathlib.Path(__file__).resolve().parents[1], capture_output=True, text=True, timeout=300)
    assert done.returncode == 0, done.stderr[-2000:]


def test_one_dimension_is_one_row_and_the_stream_may_be_given():
    """x of shape [c], on a stream that is not the current one, given as an object and as its handle: the bits of the [1, c] call."""
    c = 1234
    x, dy, w = _normal((1, c), 100).cuda(), _normal((1, c), 101).cuda(), _normal((c,), 102).cuda()
    labels = torch.tensor([77], device="cuda")
    side = torch.cuda.Stream()

    def everything(x, dy, top, **on):
        new = lambda n, dtype=torch.float32: torch.full((n,), 3, dtype=dtype, device="cuda")            # noqa: E731
        y, dx, dz, dz2, back = (torch.empty_like(x) for _ in range(5))
        mean, rstd, logp, lse, h, loss, dw, db = new(1), new(1), new(1), new(1), new(1), new(1), new(c), new(c)
        tl, ti = torch.empty(top, device="cuda"), torch.empty(top, dtype=torch.int64, device="cuda")
        ckpt, nws, lws = (new(n, torch.uint8) for n in (ftp.ftp_ckpt_bytes(x), ftp.ftp_norm_workspace_bytes(x), ftp.ftp_loss_logprob_workspace_bytes(x)))
        torch.cuda.synchronize()
        ftp.ftp_norm_forward(x, w, w, y, mean, rstd, ckpt=ckpt, **on)
        ftp.ftp_norm_backward(None, dy, w, mean, rstd, dx, dw, db, nws, ckpt=ckpt, **on)
        ftp.ftp_ckpt_save(y, ckpt, **on)
        ftp.ftp_ckpt_load(ckpt, back, **on)
        ftp.ftp_logprob(y, labels, logp, lse, h, tl, ti, **on)
        ftp.ftp_logprob_backward(y, labels, lse, h, logp, rstd, dz, **on)
        ftp.ftp_loss_logprob(y, labels, dz2, loss, lws, **on)
        torch.cuda.synchronize()
        return [t.flatten() for t in (y, mean, rstd, ckpt, dx, dw, db, back, logp, lse, h, tl, ti, dz, loss, dz2)]
    want = everything(x, dy, (1, 4))
    for on in (dict(stream=side), dict(stream=side.cuda_stream)):
        assert all(torch.equal(a, b) for a, b in zip(everything(x[0], dy[0], (4,), **on), want))


@pytest.mark.parametrize("shape", [(6, 50), (5, 3001), (2, 9, 5, 3)])
def test_gradient_of_a_row_with_nothing_left_is_zero_whatever_its_label(shape):
    z = _normal(shape, 110)
    r = z.movedim(1, -1).reshape(-1, shape[1]).clone()
    r[:3] = -float("inf")
    z = like(r, shape).contiguous().cuda()
    labels = torch.zeros(r.shape[0], dtype=torch.int64)
    labels[1], labels[2], labels[4] = -1, shape[1], shape[1] + 7
    labels = labels.reshape(_rows_of(shape)).cuda()
    lse, h = torch.empty(_rows_of(shape), device="cuda"), torch.empty(_rows_of(shape), device="cuda")
    ftp.ftp_logprob(z, None, lse=lse, entropy=h)
    dz = torch.full(shape, GUARD, device="cuda")
    ftp.ftp_logprob_backward(z, labels, lse, h, torch.ones_like(lse), torch.ones_like(lse), dz)
    d = rows(dz)
    assert not d[:3].any() and torch.isnan(d[4]).all() and torch.isfinite(d[torch.arange(len(d)) != 4]).all()
