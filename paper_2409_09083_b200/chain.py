"""Chains: a network of several plans with a channel norm between each two, trained on class labels.

A plan keeps every map of its layers between its forward and its backward pass.  The paper counts those maps as what fills a
device (Section 5.2, "feature maps dominate") and divides them over tiles and devices; a chain divides them over time: its plans
share ONE workspace, and what outlives a plan's forward pass is the joint behind it, in 8 bits:

  forward   plan -> norm (`ftp_norm_forward`, which leaves the checkpoint of what it normalised) -> checkpoint of what the next plan
            gets (`ftp_ckpt_save`) -> next plan -> ... -> loss and delta of the last map (`ftp_loss_logprob`)
  backward  the last plan's maps are still there; for the joints before it the norm's backward pass reads its checkpoint, and the plan
            runs its forward pass once more from its own (`ftp_backward_ckpt`).

So the forward pass, the loss and the last plan's gradients are those of the network itself; the gradients before the last joint are
taken at maps that are off by at most 1/127 of the largest magnitude among 32 neighbours.

A joint is kept twice, as what its norm got and as what the next plan got.  A chain has one workspace and one set of maps and checkpoints:
its calls follow one another on one stream, or one after the other by the caller's care; two streams at once want two chains.

Parameters are one flat vector: plan 0, weight and bias of the norm behind it, plan 1, ...
"""
import functools

import torch

from . import binding as ftp
from . import synth


def _on_its_device(run):
    """A chain's calls with its device current: the plans' calls take that one's current stream, as the operators between them do."""
    @functools.wraps(run)
    def call(self, *args, **kwargs):
        if self.workspace.is_cuda:
            with torch.cuda.device(self.workspace.device):
                return run(self, *args, **kwargs)
        return run(self, *args, **kwargs)
    return call


class Chain:
    def __init__(self, plans, eps=1e-5, device="cuda"):
        """plans: ftp plans in order (one may come several times, with parameters of its own in each place); the output map of each
        has the shape of the next one's input."""
        if not plans:
            raise ValueError("a chain needs at least one plan")
        self.plans, self.eps, self.device = list(plans), eps, torch.device(device)
        self.shapes = []                                      # of each plan's output map
        for p in self.plans:
            n, c, h, w = p.shape
            self.shapes.append((n,) + tuple(synth.map_shapes(p.layers, c, h, w)[-1]))
        for i, p in enumerate(self.plans[1:]):
            if tuple(p.shape) != self.shapes[i]:
                raise ValueError(f"plan {i} gives a map {self.shapes[i]}, plan {i + 1} takes {tuple(p.shape)}")
        self.slices, at = [], 0                               # (plan, weight, bias) of each joint, (plan,) of the last
        for i, (p, s) in enumerate(zip(self.plans, self.shapes)):
            sizes = [p.param_floats] if i + 1 == len(self.plans) else [p.param_floats, s[1], s[1]]
            self.slices.append([slice(at + sum(sizes[:k]), at + sum(sizes[:k + 1])) for k in range(len(sizes))])
            at += sum(sizes)
        self.param_floats = at
        empty = lambda size, dtype=torch.uint8: torch.empty(size, dtype=dtype, device=self.device)          # noqa: E731
        joints = self.shapes[:-1]
        self.workspace = empty(max(p.workspace_bytes for p in self.plans))
        most = max(_count(s) for s in self.shapes)
        self.maps = [empty(most, torch.float32) for _ in range(3)]
        self.norm_ckpt = [empty(ftp.ftp_ckpt_bytes(s)) for s in joints]       # what each norm got
        self.plan_ckpt = [empty(ftp.ftp_ckpt_bytes(s)) for s in joints]       # what the next plan got
        self.mean, self.rstd = ([empty(s[0] * s[2] * s[3], torch.float32) for s in joints] for _ in range(2))
        self.norm_ws = empty(max([ftp.ftp_norm_workspace_bytes(s) for s in joints] + [16]))
        self.loss_ws = empty(ftp.ftp_loss_logprob_workspace_bytes(self.shapes[-1]))

    @property
    def kept_bytes(self):
        """What a step keeps between the plans: checkpoints and statistics."""
        return sum(t.numel() * t.element_size() for ts in (self.norm_ckpt, self.plan_ckpt, self.mean, self.rstd) for t in ts)

    def init_norms(self, params):
        """Weights 1 and biases 0 for the norms in a flat parameter vector."""
        for sl in self.slices[:-1]:
            params[sl[1]].fill_(1.0)
            params[sl[2]].zero_()

    def _map(self, k, i):
        s = self.shapes[i]
        return self.maps[k][:_count(s)].view(s)

    @_on_its_device
    def forward(self, x, params, y=None, keep=False, stream=None):
        """Logits of the last plan ([N, classes, H, W]), in `y` or a buffer of the chain; keep: the checkpoints for a backward pass."""
        self._check(x, params, y=y)
        cur = x
        for i, plan in enumerate(self.plans):
            sl, last = self.slices[i], i + 1 == len(self.plans)
            out = y if last and y is not None else self._map(i % 2, i)
            ftp.ftp_forward(plan, cur, params[sl[0]], out, self.workspace, stream=stream)
            if not last:
                ftp.ftp_norm_forward(out, params[sl[1]], params[sl[2]], out, self.mean[i] if keep else None, self.rstd[i] if keep else None,
                                     eps=self.eps, ckpt=self.norm_ckpt[i] if keep else None, stream=stream)
                if keep:
                    ftp.ftp_ckpt_save(out, self.plan_ckpt[i], stream=stream)
                cur = out
        return out

    @_on_its_device
    def answer(self, x, params, top_logp, top_index, entropy=None, stream=None):
        """The best classes of every pixel with their log probabilities ([N, k, H, W]), and the entropies."""
        ftp.ftp_logprob(self.forward(x, params, stream=stream), None, entropy=entropy, top_logp=top_logp, top_index=top_index, stream=stream)

    @_on_its_device
    def step_grad(self, x, labels, params, dparams, loss_out, dx=None, stream=None):
        """Loss (mean over the labelled pixels of -log p) and gradient of one batch; labels: int64 [N, H, W] of the last map."""
        self._check(x, params, labels=labels, dparams=dparams, loss_out=loss_out, dx=dx)
        if dparams.numel() != self.param_floats:
            raise ValueError(f"dparams has {dparams.numel()} elements, the chain needs {self.param_floats}")
        last, ws = len(self.plans) - 1, self.workspace
        logits = self.forward(x, params, keep=True, stream=stream)
        ftp.ftp_loss_logprob(logits, labels, logits, loss_out, self.loss_ws, stream=stream)
        # the last map and the last plan's input hold a buffer each; the delta travels through the third, and from then on all are free
        delta = 2
        source = x if last == 0 else self._map((last - 1) % 2, last - 1)
        sl = self.slices[last]
        ftp.ftp_backward(self.plans[last], source, logits, params[sl[0]], dx if last == 0 else self._map(delta, last - 1), dparams[sl[0]], ws, stream=stream)
        free = [0, 1]
        for i in range(last - 1, -1, -1):
            sl, d = self.slices[i], self._map(delta, i)
            ftp.ftp_norm_backward(None, d, params[sl[1]], self.mean[i], self.rstd[i], d, dparams[sl[1]], dparams[sl[2]], self.norm_ws,
                                  ckpt=self.norm_ckpt[i], stream=stream)
            if i > 0:
                to = free[1]
                ftp.ftp_backward_ckpt(self.plans[i], self.plan_ckpt[i - 1], self._map(free[0], i - 1), d, params[sl[0]], self._map(to, i - 1),
                                      dparams[sl[0]], ws, stream=stream)
                delta, free = to, [free[0], delta]
            else:
                ftp.ftp_forward(self.plans[0], x, params[sl[0]], None, ws, stream=stream)
                ftp.ftp_backward(self.plans[0], x, d, params[sl[0]], dx, dparams[sl[0]], ws, stream=stream)

    @_on_its_device
    def step(self, x, labels, params, dparams, lr, loss_out, dx=None, stream=None):
        """One training step: step_grad, then params -= lr dparams."""
        self.step_grad(x, labels, params, dparams, loss_out, dx=dx, stream=stream)
        ftp.ftp_sgd(params, dparams, lr, stream=stream)

    def _check(self, x, params, **others):
        if params.numel() != self.param_floats:
            raise ValueError(f"params has {params.numel()} elements, the chain needs {self.param_floats}")
        if x.numel() != self.plans[0].in_floats:
            raise ValueError(f"x has {x.numel()} elements, the chain needs {self.plans[0].in_floats}")
        for name, t in (("x", x), ("params", params), *others.items()):
            if t is not None and t.device != self.workspace.device:
                raise ValueError(f"{name} is on {t.device}, the chain on {self.workspace.device}")


def _count(shape):
    n = 1
    for e in shape:
        n *= e
    return n
