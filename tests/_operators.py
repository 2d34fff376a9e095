"""Plain implementations in 64 bits of the operators between and behind the stacks, and arrays with guard values around them."""
import numpy as np
import torch

U = 2.0 ** -24                                   # half a unit in the last place of fp32, relative
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}     # half of the least step
TYPES = (torch.float32, torch.bfloat16, torch.float16)
GUARD = 123.0


def rows(a):
    """[n, c, ...] as [rows, c] in 64 bits."""
    a = a.detach().cpu().double()
    return a.movedim(1, -1).reshape(-1, a.shape[1])


def like(r, shape):
    """[rows, c] back to [n, c, ...]."""
    return r.reshape((shape[0],) + tuple(shape[2:]) + (r.shape[1],)).movedim(-1, 1)


def guarded(value, pad=0, shift=0):
    """A CUDA array with the values of `value` ([n, c, ...]), `pad` guard elements behind each sample and its start `shift` elements
    behind a 256-byte boundary; returns (array, check) where check() asserts that no guard was written."""
    n = value.shape[0]
    per = value[0].numel()
    whole = torch.full((64 + shift + n * (per + pad) + 64,), GUARD, dtype=value.dtype, device="cuda")
    body = whole[64 + shift:64 + shift + n * (per + pad)].view(n, per + pad)
    view = body[:, :per]
    view = view.unflatten(1, value.shape[1:]) if value.dim() > 2 else view
    view.copy_(value)
    seen = torch.ones_like(whole, dtype=torch.bool)
    seen[64 + shift:64 + shift + n * (per + pad)].view(n, per + pad)[:, :per] = False

    def check():
        assert bool((whole[seen] == GUARD).all()), "elements outside the array were written"
    return view, check


def norm_forward(x, w, b, eps):
    """y, mean, rstd (rows) in 64 bits."""
    x = rows(x)
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w.cpu().double()
    b = torch.zeros(x.shape[1], dtype=torch.float64) if b is None else b.cpu().double()
    return (x - mean) * rstd * w + b, mean[:, 0], rstd[:, 0]


def norm_backward(x, dy, w, mean, rstd):
    """dx, dw, db in 64 bits for given statistics, and what the terms of each amount to in magnitude."""
    x, dy, mean, rstd = rows(x), rows(dy), mean.cpu().double().reshape(-1, 1), rstd.cpu().double().reshape(-1, 1)
    w = torch.ones(x.shape[1], dtype=torch.float64) if w is None else w.cpu().double()
    hat = (x - mean) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True))
    size = (x.abs() + mean.abs()) * rstd                       # of hat, before its difference is taken
    dx_size = rstd * (g.abs() + g.abs().mean(1, keepdim=True) + size * (g.abs() * size).mean(1, keepdim=True))
    return dx, (dy * hat).sum(0), dy.sum(0), dx_size, (dy.abs() * size).sum(0), dy.abs().sum(0)


def eight_bits(x, run):
    """(values, q, exponent bytes) of the checkpoint of an array as numpy, run by run."""
    a = x.detach().cpu().double().numpy().reshape(-1, run)
    blocks = -(-run // 32)
    room = np.zeros((a.shape[0], blocks * 32))
    room[:, :run] = a
    room = room.reshape(-1, 32)
    finite = np.isfinite(room)
    big = np.where(finite, np.abs(room), 0).max(1)
    k = np.full(len(big), -126)
    for e in range(-126, 122):                                 # the least step whose 127-fold reaches
        k = np.where(127 * 2.0 ** e < big, e + 1, k)
    step = (2.0 ** k)[:, None]
    most = np.full_like(step, 127)
    top = {torch.float32: 122, torch.bfloat16: 122, torch.float16: 10}[x.dtype]
    most[k == top] = 63
    q = np.where(finite, np.clip(np.rint(np.where(finite, room, 0) / step), -most, most), -128)
    v = np.where(finite, q * step, np.nan)
    return v.reshape(a.shape[0], -1)[:, :run].reshape(x.shape), q.astype(np.int8).reshape(a.shape[0], -1), (k + 127).astype(np.uint8)


def logprob(z, labels, top):
    """Dict of lse, logp, entropy, top_logp, top_index (rows) in 64 bits by the stated rules."""
    z = rows(z)
    r, c = z.shape
    labels = labels.cpu().reshape(-1)
    bad = (torch.isnan(z) | (z == torch.inf)).any(1)
    empty = (z == -torch.inf).all(1)
    m = z.amax(1, keepdim=True)
    s = torch.exp(torch.where(empty[:, None], -torch.inf, z - torch.where(empty[:, None], 0.0, m))).sum(1, keepdim=True)
    d = torch.where(empty[:, None], -torch.inf, z - m) - torch.log(torch.where(s > 0, s, 1.0))          # log p
    p = torch.exp(d)
    out = {"lse": (torch.where(empty, -torch.inf, m[:, 0] + torch.log(s[:, 0]))),
           "entropy": -torch.where(p > 0, p * d, 0.0).sum(1),
           "logp": torch.where(labels < 0, 0.0, torch.where(labels >= c, torch.nan, d[torch.arange(r), labels.clamp(0, c - 1)]))}
    order = torch.argsort(-torch.where(torch.isnan(z), -torch.inf, z), dim=1, stable=True)[:, :top]
    out["top_index"], out["top_logp"] = order, d.gather(1, order)
    for k in ("lse", "entropy", "top_logp"):
        out[k][bad] = torch.nan
    out["logp"][bad & (labels >= 0)] = torch.nan
    return out, d, p


def close(got, want, bound, what):
    """|got - want| <= bound element by element; NaN and infinities in the same places."""
    got, want, bound = (torch.as_tensor(v).detach().cpu().double() for v in (got, want, bound))
    got = got.reshape(want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]) and torch.equal(torch.isinf(got), inf), f"{what}: infinities differ"
    fine = torch.isfinite(want)
    off = (got - want).abs()[fine] - bound.expand(want.shape)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, f"{what}: {float(off.max())} beyond the bound"
