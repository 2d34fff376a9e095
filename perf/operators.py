"""What the speed of the operators around a stack is measured on: the channel norm between two plans, the 8-bit checkpoints
of maps that a training step keeps instead of the maps, and the log probabilities of class labels with their gradient.

All of them read arrays [n, c] (n rows of c values) or [n, c, h, w] (n maps of c channels); statistics, probabilities and
alternatives run along c.  Sizes are those of the stacks' maps (32 to 512 channels, 13 x 13 to 416 x 416 pixels), of
classifiers' heads, and plain matrices of rows in 16 bits.

`run` has two forms: elementary torch operations in 32 bits, and (`own`) the framework's calls.
"""
import math

import torch

own = False

EPS = 1e-5
_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}
_BLOCK = 32


def _case(name, op, kind, n, c, h=0, w=0, pad=0, top=0):
    """h = w = 0: rows [n, c], `pad` elements between the end of a row and the next; else maps [n, c, h, w], `pad` elements
    between the end of a sample and the next."""
    return {"name": name, "op": op, "type": kind, "n": n, "c": c, "h": h, "w": w, "pad": pad, "top": top}


def listed():
    return [
        # channel norm of one row: an answer to one sample, all latency
        _case("norm_fwd_bf16_row", "norm_fwd", "bf16", 1, 1024),
        # of the first pooled map of 16 images of 608 x 608, the largest map a stack hands on
        _case("norm_fwd_f32_map", "norm_fwd", "f32", 16, 32, 304, 304),
        # backward pass at the narrow end of the 23-layer stack, planes of 169 pixels that no vector divides
        _case("norm_bwd_f32_map_odd", "norm_bwd", "f32", 8, 512, 13, 13),
        # backward pass of rows of an odd length, cut out of wider ones
        _case("norm_bwd_f16_ragged", "norm_bwd", "f16", 6001, 1111, pad=2),
        # forward pass that leaves the 8-bit checkpoint of its input, then the backward pass that reads it: the joint behind
        # the second pool of 8 images of 416 x 416 (training on small memory)
        _case("norm_ckpt_f32_map", "norm_ckpt", "f32", 8, 64, 208, 208),
        # the same for a matrix of rows, a large batch of hidden vectors
        _case("norm_ckpt_bf16_rows", "norm_ckpt", "bf16", 4096, 4096),
        # a map put away in 8 bits and taken back: the third group boundary of 16 images of 608 x 608
        _case("ckpt_f32_map", "ckpt", "f32", 16, 128, 76, 76),
        # rows of a length that fills no block
        _case("ckpt_bf16_ragged", "ckpt", "bf16", 777, 5001),
        # the answer of a classifier to one image: log probability of a class, entropy, the five best
        _case("logprob_f32_one", "logprob", "f32", 1, 1000, top=5),
        # a batch of rows over many classes with the eight best of each
        _case("logprob_bf16_rows", "logprob", "bf16", 4096, 32000, top=8),
        # gradient of log probabilities and entropies over the most classes
        _case("logprob_bwd_bf16", "logprob_bwd", "bf16", 515, 131072),
        # loss and delta of a class for each pixel, the last map of a dense head
        _case("loss_f32_map", "loss", "f32", 8, 21, 416, 416),
    ]


def _log_uniform(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))


def draw(rng):
    """One more case of the same ranges: any operator, type and layout, rows of up to 16384 values (131072 classes), maps of up
    to 1024 channels and 1 to 416 pixels a side; it moves no more bytes than its operator's largest listed case."""
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), work(c)["bytes"])
    most["logprob_bwd"] = max(most["logprob_bwd"], most["loss"])
    while True:
        op = rng.choice(["norm_fwd", "norm_bwd", "norm_ckpt", "ckpt", "logprob", "logprob_bwd", "loss"])
        kind = rng.choice(["f32", "bf16", "f16"])
        classes = op in ("logprob", "logprob_bwd", "loss")
        # of two values a norm leaves the signs alone, and the delta of that is rounding and nothing else
        least = 4 if op in ("norm_bwd", "norm_ckpt") else 1
        pad = rng.choice([0, 0, 0, 1, 8, rng.randint(1, 64)])
        if rng.random() < 0.5:
            c = _case("drawn", op, kind, _log_uniform(rng, 1, 16384), _log_uniform(rng, least, 131072 if classes else 16384), pad=pad)
        else:
            c = _case("drawn", op, kind, _log_uniform(rng, 1, 32), _log_uniform(rng, least, 1024), _log_uniform(rng, 1, 416),
                      _log_uniform(rng, 1, 416), pad=pad)
        if op == "logprob":
            c["top"] = rng.randint(0, min(20, c["c"]))
        if work(c)["bytes"] <= most[op] and work(c)["bytes"] > 4096:
            del c["name"]
            return c


def _pixels(case):
    return max(1, case["h"] * case["w"])


def _shape(case, c=None):
    c = case["c"] if c is None else c
    return (case["n"], c) if case["h"] == 0 else (case["n"], c, case["h"], case["w"])


def _run(case):
    """Length of the runs that a checkpoint cuts into blocks: a row, or a plane of more than one pixel."""
    return case["c"] if _pixels(case) == 1 else _pixels(case)


def _sums(case):
    """Shape of what there is one of for each row or pixel."""
    return (case["n"],) if case["h"] == 0 else (case["n"], case["h"], case["w"])


def _array(case, fill=None):
    """An array of the case's shape, type and stride between samples."""
    n, per = case["n"], case["c"] * _pixels(case)
    whole = torch.zeros(n * (per + case["pad"]), device="cuda", dtype=_TYPES[case["type"]])
    a = whole.view(n, per + case["pad"])[:, :per]
    a = a if case["h"] == 0 else a.view(_shape(case)) if case["pad"] == 0 else a.unflatten(1, _shape(case)[1:])
    if fill is not None:
        a.copy_(fill)
    return a


def prepare(case, seed):
    """Inputs of the distributions that the calls meet: activations behind a leaky ReLU with channels of different scales,
    deltas, norm weights around 1, logits over some ten units with a few classes ruled out (-inf) and rows without a label;
    and the buffers that a program keeps from step to step."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)     # noqa: E731
    shape, c, op = _shape(case), case["c"], case["op"]
    s = {"case": case}
    along = (1, c) + (1,) * (len(shape) - 2)
    if op in ("norm_fwd", "norm_bwd", "norm_ckpt", "ckpt"):
        x = normal(*shape) * (0.25 + torch.rand(along, device="cuda", generator=gen)) + 0.3 * normal(*along)
        s["x"] = _array(case, torch.where(x > 0, x, 0.1 * x))
        if op != "ckpt":
            s["w"], s["b"] = 1 + 0.2 * normal(c), 0.1 * normal(c)
            s["mean"], s["rstd"] = (torch.empty(_sums(case), device="cuda") for _ in range(2))
            s["y"] = _array(case)
        if op in ("norm_bwd", "norm_ckpt"):
            s["dy"] = _array(case, normal(*shape))
            s["dx"], s["dw"], s["db"] = _array(case), torch.empty(c, device="cuda"), torch.empty(c, device="cuda")
        if op == "norm_bwd":
            wide = s["x"].float()
            s["mean"].copy_(wide.mean(1))
            s["rstd"].copy_(1 / torch.sqrt(((wide - wide.mean(1, keepdim=True)) ** 2).mean(1) + EPS))
        if op == "ckpt":
            s["back"] = _array(case)
    else:
        z = 3 * normal(*shape)
        labels = torch.randint(0, c, _sums(case), device="cuda", generator=gen)
        classes = torch.arange(c, device="cuda").view(along)
        out = (torch.rand(*shape, device="cuda", generator=gen) < 0.02) & (classes != labels.unsqueeze(1)) & (classes > 0)
        s["labels"] = torch.where(torch.rand(_sums(case), device="cuda", generator=gen) < 0.1, -1, labels)
        s["logits"] = _array(case, torch.where(out, -math.inf, z))
        if op == "logprob":
            s["logp"], s["lse"], s["entropy"] = (torch.empty(_sums(case), device="cuda") for _ in range(3))
            if case["top"]:
                s["top_logp"] = torch.empty(_shape(case, case["top"]), device="cuda")
                s["top_index"] = torch.empty(_shape(case, case["top"]), device="cuda", dtype=torch.int64)
        else:
            s["dlogits"] = _array(case)
        if op == "logprob_bwd":
            wide = s["logits"].float()
            s["lse"] = torch.log(torch.exp(wide - wide.amax(1, keepdim=True)).sum(1)) + wide.amax(1)
            lp = wide - s["lse"].unsqueeze(1)
            s["entropy"] = -torch.where(lp > -math.inf, torch.exp(lp) * lp, 0.0).sum(1)
            s["dlogp"], s["dentropy"] = normal(*_sums(case)), 0.1 * normal(*_sums(case))
        if op == "loss":
            s["loss"] = torch.empty(1, device="cuda")
    if own:
        import paper_2409_09083_b200 as ftp
        if op in ("norm_bwd", "norm_ckpt"):
            s["ws"] = torch.empty(ftp.ftp_norm_workspace_bytes(s["x"]), device="cuda", dtype=torch.uint8)
        if op == "loss":
            s["ws"] = torch.empty(ftp.ftp_loss_logprob_workspace_bytes(s["logits"]), device="cuda", dtype=torch.uint8)
        if op in ("norm_ckpt", "ckpt"):
            s["ckpt"] = torch.empty(ftp.ftp_ckpt_bytes(s["x"]), device="cuda", dtype=torch.uint8)
    return s


def _loss_scale(case):
    """What the loss is multiplied with before its delta is rounded to the logits' type."""
    return 65536.0 if case["type"] == "f16" else 1.0


# The operators in their plain form -----------------------------------------------------------------------------------

def _channels(v, like):
    return v.view((1, -1) + (1,) * (like.dim() - 2))


def _norm_forward(x, w, b):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    return (x - mean) * rstd * _channels(w, x) + _channels(b, x), mean.squeeze(1), rstd.squeeze(1)


def _norm_backward(x, dy, w, mean, rstd):
    x, dy, mean, rstd = x.float(), dy.float(), mean.unsqueeze(1), rstd.unsqueeze(1)
    hat = (x - mean) * rstd
    g = dy * _channels(w, x)
    dx = (g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True)) * rstd
    rest = [0] + list(range(2, x.dim()))
    return dx, (dy * hat).sum(rest), dy.sum(rest)


def _eight_bits(x, case):
    """The values that the checkpoint of x stands for: blocks of 32 along the innermost run of a row or plane share the
    smallest power of two whose 127-fold reaches the block's largest magnitude; values are its nearest multiples."""
    run = _run(case)
    v = x.float().reshape(-1, run)
    v = torch.cat([v, v.new_zeros(v.shape[0], -run % _BLOCK)], 1).view(v.shape[0], -1, _BLOCK)
    largest = v.abs().amax(2, keepdim=True)
    part, exponent = torch.frexp(largest)                     # largest = part * 2^exponent, 1/2 <= part < 1
    k = torch.clamp(exponent - 7 + (part > 127 / 128), min=-126)
    step = ((k + 127).int() << 23).view(torch.float32)        # 2^k to the bit
    q = torch.clamp(torch.round(v / step), -127, 127)
    return (q * step).view(v.shape[0], -1)[:, :run].reshape(x.shape)


def _log_softmax(z):
    z = z.float()
    top = z.amax(1, keepdim=True)
    lse = torch.log(torch.exp(z - top).sum(1, keepdim=True)) + top
    return z - lse, lse.squeeze(1)


def _at(logp, labels):
    return torch.where(labels >= 0, logp.gather(1, labels.clamp(min=0).unsqueeze(1)).squeeze(1), 0.0)


def _entropy(logp):
    return -torch.where(logp > -math.inf, torch.exp(logp) * logp, 0.0).sum(1)


def _hit(logp, labels):
    return torch.arange(logp.shape[1], device=logp.device).view((1, -1) + (1,) * (logp.dim() - 2)) == labels.unsqueeze(1)


def _run_plain(s):
    case = s["case"]
    op, kind = case["op"], _TYPES[case["type"]]
    if op == "norm_fwd":
        y, mean, rstd = _norm_forward(s["x"], s["w"], s["b"])
        return {"y": y.to(kind), "mean": mean, "rstd": rstd}
    if op == "norm_bwd":
        dx, dw, db = _norm_backward(s["x"], s["dy"], s["w"], s["mean"], s["rstd"])
        return {"dx": dx.to(kind), "dw": dw, "db": db}
    if op == "norm_ckpt":
        y, mean, rstd = _norm_forward(s["x"], s["w"], s["b"])
        dx, dw, db = _norm_backward(_eight_bits(s["x"], case), s["dy"], s["w"], mean, rstd)
        return {"y": y.to(kind), "dx": dx.to(kind), "dw": dw, "db": db}
    if op == "ckpt":
        return {"back": _eight_bits(s["x"], case).to(kind)}
    logp, lse = _log_softmax(s["logits"])
    labels = s["labels"]
    if op == "logprob":
        out = {"logp": _at(logp, labels), "lse": lse, "entropy": _entropy(logp)}
        if case["top"]:
            order = torch.sort(s["logits"], dim=1, descending=True, stable=True)[1][:, :case["top"]].contiguous()
            out["top_logp"], out["top_index"] = logp.gather(1, order), order
        return out
    if op == "logprob_bwd":
        logp = s["logits"].float() - s["lse"].unsqueeze(1)
        p = torch.exp(logp)
        surprise = torch.where(p > 0, p * (logp + s["entropy"].unsqueeze(1)), 0.0)
        labelled = torch.where(labels >= 0, s["dlogp"], 0.0).unsqueeze(1)
        d = labelled * (_hit(logp, labels).float() - p) - s["dentropy"].unsqueeze(1) * surprise
        return {"dlogits": d.to(kind)}
    labelled = (labels >= 0).unsqueeze(1)
    count = (labels >= 0).sum().clamp(min=1)
    d = torch.where(labelled, torch.exp(logp) - _hit(logp, labels).float(), 0.0) * (_loss_scale(case) / count)
    return {"loss": (-_at(logp, labels).sum() / count).view(1), "dlogits": d.to(kind)}


def run(state):
    s = state
    if not own:
        return _run_plain(s)
    import paper_2409_09083_b200 as ftp
    op = s["case"]["op"]
    if op == "norm_fwd":
        ftp.ftp_norm_forward(s["x"], s["w"], s["b"], s["y"], s["mean"], s["rstd"], eps=EPS)
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if op == "norm_bwd":
        ftp.ftp_norm_backward(s["x"], s["dy"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], s["ws"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if op == "norm_ckpt":
        ftp.ftp_norm_forward(s["x"], s["w"], s["b"], s["y"], s["mean"], s["rstd"], eps=EPS, ckpt=s["ckpt"])
        ftp.ftp_norm_backward(None, s["dy"], s["w"], s["mean"], s["rstd"], s["dx"], s["dw"], s["db"], s["ws"], ckpt=s["ckpt"])
        return {"y": s["y"], "dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if op == "ckpt":
        ftp.ftp_ckpt_save(s["x"], s["ckpt"])
        ftp.ftp_ckpt_load(s["ckpt"], s["back"])
        return {"back": s["back"]}
    if op == "logprob":
        out = {"logp": s["logp"], "lse": s["lse"], "entropy": s["entropy"]}
        if s["case"]["top"]:
            out["top_logp"], out["top_index"] = s["top_logp"], s["top_index"]
        ftp.ftp_logprob(s["logits"], s["labels"], **out)
        return out
    if op == "logprob_bwd":
        ftp.ftp_logprob_backward(s["logits"], s["labels"], s["lse"], s["entropy"], s["dlogp"], s["dentropy"], s["dlogits"])
        return {"dlogits": s["dlogits"]}
    ftp.ftp_loss_logprob(s["logits"], s["labels"], s["dlogits"], s["loss"], s["ws"], scale=_loss_scale(s["case"]))
    return {"loss": s["loss"], "dlogits": s["dlogits"]}


def work(case):
    """Bytes: every input once and every output once, a checkpoint written and read (33 bytes for 32 values).  Operations:
    those on each value, an exponential counted as one."""
    size, rows = _SIZE[case["type"]], case["n"] * _pixels(case)
    values = rows * case["c"]
    run = _run(case)
    eight = (values // run) * -(-run // _BLOCK) * (_BLOCK + 1)
    op = case["op"]
    if op == "norm_fwd":
        return {"bytes": 2 * size * values + 8 * rows + 8 * case["c"], "flops": 8 * values}
    if op == "norm_bwd":
        return {"bytes": 3 * size * values + 8 * rows + 12 * case["c"], "flops": 14 * values}
    if op == "norm_ckpt":
        return {"bytes": 4 * size * values + 2 * eight + 16 * rows + 20 * case["c"], "flops": 26 * values}
    if op == "ckpt":
        return {"bytes": 2 * size * values + 2 * eight, "flops": 6 * values}
    if op == "logprob":
        return {"bytes": size * values + (20 + 12 * case["top"]) * rows, "flops": 6 * values}
    if op == "logprob_bwd":
        return {"bytes": 2 * size * values + 24 * rows, "flops": 7 * values}
    return {"bytes": 2 * size * values + 8 * rows, "flops": 8 * values}


# The operators from their definitions, in 64 bits: rows [rows, c], a part of them at a time ----------------------------

def _rows(a):
    """[n, c, ...] as rows of c values in 64 bits."""
    return a.movedim(1, -1).reshape(-1, a.shape[1]).double()


def _as_map(rows, shape):
    return rows.view((shape[0],) + tuple(shape[2:]) + (rows.shape[1],)).movedim(-1, 1).contiguous()


def _exact_eight_bits(x, run):
    """Block by block through integers: the exponent is found by counting the powers of two that do not reach."""
    flat = x.double().reshape(-1, run)
    blocks = -(-run // _BLOCK)
    room = torch.zeros(flat.shape[0], blocks * _BLOCK, dtype=torch.float64, device=x.device)
    room[:, :run] = flat
    room = room.view(-1, _BLOCK)
    powers = torch.tensor([2.0 ** k for k in range(-126, 123)], dtype=torch.float64, device=x.device)
    step = powers[torch.searchsorted(127 * powers[:-1], room.abs().amax(1))].unsqueeze(1)
    return (torch.round(room / step) * step).view(flat.shape[0], -1)[:, :run].reshape(x.shape)


def exact(case, seed):
    s = prepare(case, seed)
    op, shape = case["op"], _shape(case)
    if op == "ckpt":
        return {"back": _exact_eight_bits(s["x"], _run(case))}
    if op.startswith("norm"):
        x, w, b = _rows(s["x"]), s["w"].double(), s["b"].double()
        spread, mean = torch.var_mean(x, dim=1, correction=0)
        rstd = torch.rsqrt(spread + EPS)
        out = {}
        if op != "norm_bwd":
            out["y"] = _as_map(torch.addcmul(b, (x - mean[:, None]) * rstd[:, None], w), shape)
        if op == "norm_fwd":
            return out | {"mean": mean.view(_sums(case)), "rstd": rstd.view(_sums(case))}
        if op == "norm_bwd":
            mean, rstd = s["mean"].double().reshape(-1), s["rstd"].double().reshape(-1)
        else:
            x = _rows(_exact_eight_bits(s["x"], _run(case)))
        dy = _rows(s["dy"])
        hat = (x - mean[:, None]) * rstd[:, None]
        g = dy * w
        c = case["c"]
        dx = (c * g - g.sum(1, keepdim=True) - hat * (g * hat).sum(1, keepdim=True)) * (rstd / c)[:, None]
        return out | {"dx": _as_map(dx, shape), "dw": torch.einsum("rc,rc->c", dy, hat), "db": dy.sum(0)}
    z, labels = _rows(s["logits"]), s["labels"].reshape(-1)
    r = torch.arange(z.shape[0], device=z.device)
    if op == "logprob_bwd":
        lse, h = s["lse"].double().reshape(-1, 1), s["entropy"].double().reshape(-1, 1)
    else:
        lse = torch.logsumexp(z, 1, keepdim=True)
    p = torch.exp(z - lse)
    known = labels >= 0
    if op == "logprob":
        out = {"logp": torch.where(known, z[r, labels.clamp(min=0)] - lse[:, 0], 0.0).view(_sums(case)), "lse": lse.view(_sums(case)),
               "entropy": -torch.xlogy(p, p).sum(1).view(_sums(case))}
        if case["top"]:
            order = torch.argsort(-z, dim=1, stable=True)[:, :case["top"]]
            out["top_logp"] = _as_map(z.gather(1, order) - lse, shape)
            out["top_index"] = _as_map(order, shape)
        return out
    if op == "logprob_bwd":
        gl = torch.where(known, s["dlogp"].double().reshape(-1), 0.0)
        ge = s["dentropy"].double().reshape(-1, 1)
        d = -p * gl[:, None] - ge * (torch.where(p > 0, p * (z - lse), 0.0) + p * h)
        d[r[known], labels[known]] += gl[known]
        return {"dlogits": _as_map(d, shape)}
    count = max(1, int(known.sum()))
    loss = (lse[known, 0] - z[r[known], labels[known]]).sum() / count
    p[r[known], labels[known]] -= 1
    p[~known] = 0
    return {"loss": loss.view(1), "dlogits": _as_map(p, shape) * (_loss_scale(case) / count)}
