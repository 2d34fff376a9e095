"""Chains of plans with channel norms between them: loss and gradients against the 64-bit oracle with the norms, the 8-bit
checkpoints and the class loss in 64 bits; the same bits from a graph; and that training goes through."""
import numpy as np
import pytest
import torch

import paper_2409_09083_b200 as ftp
from oracle import reference as orc
from paper_2409_09083_b200 import chain as chains
from paper_2409_09083_b200 import synth
from _operators import U, logprob, norm_backward, norm_forward, rows, like

EPS = 1e-5


def _plans(n=2, h=24, w=32, precision=0):
    a = [synth.conv(3, 8, 3), synth.pool(), synth.conv(8, 16, 3)]
    b = [synth.conv(16, 24, 3), synth.pool()]
    c = [synth.conv(24, 12, 1), synth.conv(12, 10, 3)]
    at, plans = (3, h, w), []
    for layers in (a, b, c):
        plans.append(ftp.ftp_plan(layers, n, *at, (2, 2), ((1, len(layers)),), precision=precision))
        at = synth.map_shapes(layers, *at)[-1]
    return plans


def _batch(chain, seed=0):
    gen = torch.Generator().manual_seed(seed)
    n, c, h, w = chain.plans[0].shape
    x = torch.rand((n, c, h, w), generator=gen)
    params = 0.3 * torch.randn(chain.param_floats, generator=gen)
    for sl in chain.slices[:-1]:
        params[sl[1]] = 1 + 0.2 * torch.randn(params[sl[1]].shape, generator=gen)
    s = chain.shapes[-1]
    labels = torch.randint(-1, s[1], (s[0],) + s[2:], generator=gen)
    return x, params, labels


def test_shapes_have_to_fit():
    plans = _plans()
    with pytest.raises(ValueError, match="plan 0 gives a map"):
        chains.Chain([plans[0], plans[2]], device="cpu")
    with pytest.raises(ValueError, match="at least one"):
        chains.Chain([], device="cpu")
    chain = chains.Chain(plans, device="cpu")
    assert chain.param_floats == sum(p.param_floats for p in plans) + 2 * (16 + 24)
    params = torch.zeros(chain.param_floats)
    chain.init_norms(params)
    assert params.sum() == 16 + 24
    with pytest.raises(ValueError, match="params has 3"):
        chain.forward(torch.zeros(plans[0].in_floats), params[:3])
    with pytest.raises(ValueError, match="x has 5"):
        chain.step_grad(torch.zeros(5), None, params, params, None)
    with pytest.raises(ValueError, match="dparams has"):
        chain.step_grad(torch.zeros(plans[0].in_floats), None, params, params[1:], None)
    # what outlives a plan's forward pass: two bytes and a thirty-second for each value of a joint, and two floats a pixel
    joints = sum(int(np.prod(s)) for s in chain.shapes[:-1])
    assert 2 * 33 / 32 * joints <= chain.kept_bytes <= 2.5 * joints + 8 * 2 * (12 * 16 + 6 * 8)


@pytest.mark.gpu
def test_loss_and_gradients_against_the_oracle():
    plans = _plans()
    chain = chains.Chain(plans)
    x, params, labels = _batch(chain)
    dparams, loss, dx = torch.empty(chain.param_floats, device="cuda"), torch.empty(1, device="cuda"), torch.empty(plans[0].shape, device="cuda")
    chain.step_grad(x.cuda(), labels.cuda(), params.cuda(), dparams, loss, dx=dx)
    p64 = params.double().numpy()
    # forward in 64 bits
    cur, tapes, stats = x.double().numpy(), [], []
    for i, plan in enumerate(plans):
        sl = chain.slices[i]
        maps, tape = orc.forward(plan.layers, cur, p64[sl[0]])
        tapes.append((maps, tape))
        cur = maps[-1]
        if i < 2:
            y, mean, rstd = norm_forward(torch.from_numpy(cur), torch.from_numpy(p64[sl[1]]), torch.from_numpy(p64[sl[2]]), EPS)
            stats.append((mean, rstd))
            cur = like(y, chain.shapes[i]).contiguous().numpy()
    known = labels.reshape(-1) >= 0
    want, d, p = logprob(torch.from_numpy(cur), labels, 1)
    m = int(known.sum())
    assert abs(loss.item() + float(want["logp"][known].sum()) / m) <= 1e-5 * abs(loss.item())
    delta = torch.where(known[:, None], p - (torch.arange(p.shape[1])[None] == labels.reshape(-1, 1)).double(), 0.0) / m
    delta = like(delta, chain.shapes[-1]).contiguous().numpy()
    # backward in 64 bits, at the values of the checkpoints that the step kept
    got = dparams.cpu().double().numpy()

    def check(part, want, what, tol=1e-4):
        assert np.abs(got[part] - want).max() <= tol * np.abs(want).max(), what
    for i in (2, 1, 0):
        sl = chain.slices[i]
        if i < 2:
            kept = torch.empty(chain.shapes[i], device="cuda")
            ftp.ftp_ckpt_load(chain.norm_ckpt[i], kept)
            dx64, dw, db, _, _, _ = norm_backward(kept, torch.from_numpy(delta), torch.from_numpy(p64[sl[1]]), chain.mean[i], chain.rstd[i])
            check(sl[1], dw.numpy(), f"weight of norm {i}")
            check(sl[2], db.numpy(), f"bias of norm {i}")
            delta = like(dx64, chain.shapes[i]).contiguous().numpy()
        if i == 1:
            kept = torch.empty(plans[1].shape, device="cuda")
            ftp.ftp_ckpt_load(chain.plan_ckpt[0], kept)
            maps, tape = orc.forward(plans[1].layers, kept.cpu().double().numpy(), p64[sl[0]])
        else:
            maps, tape = tapes[i]
        delta, dparams64, _ = orc.backward(plans[i].layers, maps, tape, p64[sl[0]], delta)
        check(sl[0], dparams64, f"plan {i}", 1e-3)               # (a near-tie of a pool or of a sign may fall the other way)
    assert np.abs(dx.cpu().double().numpy() - delta).max() <= 1e-3 * np.abs(delta).max()
    assert np.isfinite(got).all()


@pytest.mark.gpu
@pytest.mark.parametrize("precision", [0, 1])
def test_steps_in_a_graph_are_the_same_bits_and_training_goes_through(precision):
    chain = chains.Chain(_plans(precision=precision))
    x, params, labels = _batch(chain, 1)
    x, labels = x.cuda(), labels.cuda()
    eager, held = params.cuda(), params.cuda()
    dparams, loss = torch.empty(chain.param_floats, device="cuda"), torch.empty(1, device="cuda")
    losses = []
    for _ in range(3):
        chain.step(x, labels, eager, dparams, 0.02, loss)
        losses.append(loss.item())
    assert all(np.isfinite(losses))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        chain.step(x, labels, held, dparams, 0.02, loss)
    replayed = []
    for _ in range(3):
        g.replay()
        torch.cuda.synchronize()
        replayed.append(loss.item())
    assert replayed == losses and torch.equal(eager, held)


@pytest.mark.gpu
def test_answer():
    chain = chains.Chain(_plans())
    x, params, labels = _batch(chain, 2)
    n, c, h, w = chain.shapes[-1]
    tl, ti = torch.empty((n, 3, h, w), device="cuda"), torch.empty((n, 3, h, w), dtype=torch.int64, device="cuda")
    e = torch.empty((n, h, w), device="cuda")
    chain.answer(x.cuda(), params.cuda(), tl, ti, e)
    logits = chain.forward(x.cuda(), params.cuda())
    want, _, _ = logprob(logits, labels, 3)
    assert torch.equal(rows(ti).long(), want["top_index"])
    assert (rows(tl) - want["top_logp"]).abs().max() <= 256 * U * (1 + want["top_logp"].abs().max())
    assert (e.cpu().double().reshape(-1) - want["entropy"]).abs().max() <= 1e-4


@pytest.mark.gpu
def test_one_plan_is_a_chain_too():
    plan = ftp.ftp_plan([synth.conv(3, 10, 3)], 2, 3, 12, 16, (1, 1), ((1, 1),))
    chain = chains.Chain([plan])
    x, params, labels = _batch(chain, 3)
    dparams, loss, dx = torch.empty(chain.param_floats, device="cuda"), torch.empty(1, device="cuda"), torch.empty(plan.shape, device="cuda")
    chain.step_grad(x.cuda(), labels.cuda(), params.cuda(), dparams, loss, dx=dx)
    y, dy, again, dx2 = (torch.empty(s, device="cuda") for s in (chain.shapes[0], chain.shapes[0], dparams.shape, plan.shape))
    ws = plan.new_workspace()
    ftp.ftp_forward(plan, x.cuda(), params.cuda(), y, ws)
    loss2 = torch.empty(1, device="cuda")
    ftp.ftp_loss_logprob(y, labels.cuda(), dy, loss2, chain.loss_ws)
    ftp.ftp_backward(plan, x.cuda(), dy, params.cuda(), dx2, again, ws)
    assert torch.equal(dparams, again) and torch.equal(dx, dx2) and torch.equal(loss, loss2)


def test_inputs_of_another_device():
    plans = _plans()
    chain = chains.Chain(plans, device="cpu")
    x, params = torch.zeros(plans[0].in_floats), torch.zeros(chain.param_floats)
    with pytest.raises(ValueError, match="x is on meta, the chain on cpu"):
        chain.forward(x.to("meta"), params)
    with pytest.raises(ValueError, match="params is on meta"):
        chain.answer(x, params.to("meta"), None, None)


def _odd_plans(n=2, h=10, w=14, precision=0):
    """13 channels at every joint, so that no part of the parameters after the first starts on 16 bytes."""
    def make(layers, c):
        return ftp.ftp_plan(layers, n, c, h, w, (2, 2), ((1, len(layers)),), precision=precision)
    return make([synth.conv(3, 13, 3)], 3), lambda: make([synth.conv(13, 13, 3)], 13)


def test_a_plan_in_two_places_has_parameters_in_each():
    first, middle = _odd_plans()
    again = middle()
    chain = chains.Chain([first, again, again], device="cpu")
    assert [len(sl) for sl in chain.slices] == [3, 3, 1]
    assert chain.param_floats == first.param_floats + 2 * again.param_floats + 4 * 13
    assert chain.slices[1][0].stop - chain.slices[1][0].start == chain.slices[2][0].stop - chain.slices[2][0].start == again.param_floats


@pytest.mark.gpu
@pytest.mark.parametrize("precision", [0, 1])
def test_parameters_off_the_16_byte_grid_and_a_plan_in_two_places(precision):
    first, middle = _odd_plans(precision=precision)
    again = middle()
    chain, apart = chains.Chain([first, again, again]), chains.Chain([first, middle(), middle()])
    x, params, labels = _batch(chain, 4)
    x, params, labels = x.cuda(), params.cuda(), labels.cuda()
    assert any(sl[0].start % 4 for sl in chain.slices)
    grads, losses = [], []
    for c in (chain, apart):
        dparams, loss = torch.full((c.param_floats,), float("nan"), device="cuda"), torch.empty(1, device="cuda")
        c.step_grad(x, labels, params, dparams, loss)
        grads.append(dparams)
        losses.append(loss)
    assert torch.equal(grads[0], grads[1]) and torch.equal(losses[0], losses[1]) and torch.isfinite(grads[0]).all()
    # the same calls, the norms' checkpoints among them (without, their sums have another order), with every part of the parameters in
    # an array of its own
    cur, ws = x, torch.empty(chain.workspace.numel(), dtype=torch.uint8, device="cuda")
    for i, plan in enumerate(chain.plans):
        part, out = [params[s].clone() for s in chain.slices[i]], torch.empty(chain.shapes[i], device="cuda")
        ftp.ftp_forward(plan, cur, part[0], out, ws)
        if i < 2:
            ftp.ftp_norm_forward(out, part[1], part[2], out, eps=EPS, ckpt=torch.empty_like(chain.norm_ckpt[i]))
            cur = out
    assert torch.equal(out, chain.forward(x, params, keep=True))
    delta, loss = torch.empty_like(out), torch.empty(1, device="cuda")
    ftp.ftp_loss_logprob(out, labels, delta, loss, chain.loss_ws)
    grad = torch.empty(again.param_floats, device="cuda")
    ftp.ftp_backward(again, cur, delta, part[0], None, grad, ws)
    assert torch.equal(grad, grads[0][chain.slices[2][0]]) and torch.equal(loss, losses[0])


@pytest.mark.parametrize("name", ["dparams", "dx", "labels", "loss_out"])
def test_what_a_step_writes_and_reads_is_on_the_chains_device(name):
    plans = _plans()
    chain = chains.Chain(plans, device="cpu")
    x, params = torch.zeros(plans[0].in_floats), torch.zeros(chain.param_floats)
    n, _, h, w = chain.shapes[-1]
    given = dict(labels=torch.zeros((n, h, w), dtype=torch.int64), dparams=params.clone(), loss_out=torch.zeros(1), dx=x.clone())
    given[name] = given[name].to("meta")
    with pytest.raises(ValueError, match=f"{name} is on meta, the chain on cpu"):
        chain.step_grad(x, params=params, **given)
    with pytest.raises(ValueError, match=f"{name} is on meta, the chain on cpu"):
        chain.step(x, params=params, lr=0.1, **given)


def test_a_chains_output_is_on_its_device():
    plans = _plans()
    chain = chains.Chain(plans, device="cpu")
    x, params = torch.zeros(plans[0].in_floats), torch.zeros(chain.param_floats)
    with pytest.raises(ValueError, match="y is on meta, the chain on cpu"):
        chain.forward(x, params, y=torch.empty(chain.shapes[-1], device="meta"))


@pytest.mark.gpu
def test_a_chain_on_a_stream_that_is_given():
    x, params, labels = (t.cuda() for t in _batch(chains.Chain(_plans()), 5))
    results = []
    for stream in (None, torch.cuda.Stream()):
        chain = chains.Chain(_plans())
        p, dparams, loss = params.clone(), torch.empty_like(params), torch.empty(1, device="cuda")
        s = chain.shapes[-1]
        tl, ti = torch.empty((s[0], 2) + s[2:], device="cuda"), torch.empty((s[0], 2) + s[2:], dtype=torch.int64, device="cuda")
        torch.cuda.synchronize()
        for _ in range(2):
            chain.step(x, labels, p, dparams, 0.02, loss, stream=stream)
        chain.answer(x, p, tl, ti, stream=stream)
        torch.cuda.synchronize()
        results.append((p, dparams, loss, tl, ti))
    assert all(torch.equal(a, b) for a, b in zip(*results))
