"""What the operators between and behind the stacks refuse, before anything reaches the GPU: through the binding, and at the C-ABI itself.
Everything here runs on the CPU."""
import ctypes

import pytest
import torch

import paper_2409_09083_b200 as ftp
from paper_2409_09083_b200 import binding

ARG, TOO_LARGE = -1, -9
lib = binding._lib
SOME = 1 << 20                                      # an address that no refused call touches


def _d(n, c, p=1, type_=0, size=None):
    return ctypes.byref(binding.ftp_dims(ctypes.sizeof(binding.ftp_dims) if size is None else size, type_, n, c, p))


def test_sizes():
    assert ftp.ftp_ckpt_bytes((3, 64)) == 3 * 2 * 33
    assert ftp.ftp_ckpt_bytes((3, 65)) == 3 * 3 * 33
    assert ftp.ftp_ckpt_bytes((2, 5, 13, 13)) == 2 * 5 * 6 * 33
    assert ftp.ftp_ckpt_bytes((2, 5, 1, 1)) == 2 * 33                   # one pixel: rows of c values
    assert ftp.ftp_ckpt_bytes((70,)) == 3 * 33
    assert ftp.ftp_ckpt_bytes((0, 5)) == 0
    assert ftp.ftp_norm_workspace_bytes((7, 10)) >= 2 * 10 * 4
    assert ftp.ftp_loss_logprob_workspace_bytes((7, 10)) > 0


@pytest.mark.parametrize("dims, code", [((1, 0, 1), ARG), ((-1, 4, 1), ARG), ((1, 4, -1), ARG), ((1 << 30, 4, 1), TOO_LARGE),
                                        ((1, 1 << 30, 1), TOO_LARGE), ((1, 4, 1 << 30), TOO_LARGE), ((1 << 29, 1 << 20, 1), TOO_LARGE)])
def test_dims_are_checked_by_every_entry(dims, code):
    d, n = _d(*dims), ctypes.c_size_t()
    assert lib.ftp_ckpt_bytes(d, ctypes.byref(n)) == code
    assert lib.ftp_norm_workspace(d, ctypes.byref(n)) == code
    assert lib.ftp_loss_logprob_workspace(d, ctypes.byref(n)) == code
    assert lib.ftp_ckpt_save(d, SOME, 0, SOME, None) == code
    assert lib.ftp_ckpt_load(d, SOME, SOME, 0, None) == code
    assert lib.ftp_norm_forward(d, SOME, 0, None, None, 1e-5, SOME, 0, None, None, None, None) == code
    assert lib.ftp_norm_backward(d, SOME, 0, None, SOME, 0, None, SOME, SOME, SOME, 0, None, None, None, 0, None) == code
    assert lib.ftp_logprob(d, SOME, 0, SOME, SOME, None, None, 0, None, None, None) == code
    assert lib.ftp_logprob_backward(d, SOME, 0, SOME, SOME, None, SOME, None, SOME, 0, None) == code
    assert lib.ftp_loss_logprob(d, SOME, 0, SOME, 1.0, SOME, 0, SOME, SOME, 1 << 20, None) == code


def test_struct_size_and_type():
    n = ctypes.c_size_t()
    assert lib.ftp_ckpt_bytes(None, ctypes.byref(n)) == ARG
    assert lib.ftp_ckpt_bytes(_d(1, 4), None) == ARG
    assert lib.ftp_ckpt_bytes(_d(1, 4, size=8), ctypes.byref(n)) == ARG
    assert lib.ftp_ckpt_bytes(_d(1, 4, type_=3), ctypes.byref(n)) == ARG


def _norm_forward(d=None, x=SOME, xs=0, w=None, b=None, eps=1e-5, y=SOME, ys=0, m=None, r=None, k=None):
    return lib.ftp_norm_forward(d or _d(4, 8), x, xs, w, b, eps, y, ys, m, r, k, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(y=None), dict(xs=7), dict(ys=7), dict(xs=-8), dict(xs=1 << 45), dict(x=SOME + 2), dict(y=SOME + 1),
                                 dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(w=SOME + 2), dict(b=SOME + 1),
                                 dict(m=SOME + 2), dict(r=SOME + 2), dict(k=SOME + 8), dict(d=_d(4, 8, 3), xs=23)])
def test_norm_forward_refuses(bad):
    assert _norm_forward(**bad) == ARG


def _norm_backward(d=None, x=SOME, xs=0, k=None, dy=SOME, dys=0, w=None, m=SOME, r=SOME, dx=SOME, dxs=0, dw=SOME, db=SOME, ws=SOME, n=1 << 30):
    return lib.ftp_norm_backward(d or _d(4, 8), x, xs, k, dy, dys, w, m, r, dx, dxs, dw, db, ws, n, None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(k=SOME), dict(x=None, k=SOME + 8), dict(dy=None), dict(m=None), dict(r=None), dict(dw=None),
                                 dict(db=None), dict(dx=None, dw=None, db=None), dict(ws=None), dict(ws=SOME + 8), dict(n=2 * 148 * 2 * 8 * 4 - 1),
                                 dict(xs=7), dict(dys=7), dict(dxs=7), dict(dy=SOME + 2), dict(dx=SOME + 2), dict(w=SOME + 2),
                                 dict(dw=SOME + 2), dict(db=SOME + 2), dict(m=SOME + 2), dict(r=SOME + 2)])
def test_norm_backward_refuses(bad):
    assert _norm_backward(**bad) == ARG


@pytest.mark.parametrize("bad", [(None, 0, SOME), (SOME, 0, None), (SOME, 7, SOME), (SOME, 0, SOME + 8), (SOME + 2, 0, SOME)])
def test_ckpt_refuses(bad):
    x, stride, k = bad
    assert lib.ftp_ckpt_save(_d(4, 8), x, stride, k, None) == ARG
    assert lib.ftp_ckpt_load(_d(4, 8), k, x, stride, None) == ARG


def _logprob(d=None, z=SOME, zs=0, lab=SOME, lp=SOME, lse=SOME, h=SOME, top=2, tl=SOME, ti=SOME):
    return lib.ftp_logprob(d or _d(4, 8), z, zs, lab, lp, lse, h, top, tl, ti, None)


@pytest.mark.parametrize("bad", [dict(z=None), dict(zs=7), dict(lab=None), dict(top=-1), dict(top=21, d=_d(4, 80)), dict(top=9), dict(top=0),
                                 dict(tl=None, ti=None), dict(lp=None, lse=None, h=None, top=0, tl=None, ti=None), dict(z=SOME + 2),
                                 dict(lab=SOME + 4), dict(lp=SOME + 2), dict(lse=SOME + 2), dict(h=SOME + 2), dict(tl=SOME + 2), dict(ti=SOME + 4)])
def test_logprob_refuses(bad):
    assert _logprob(**bad) == ARG


def test_too_many_classes_or_rows():
    d = _d(2, 260001)
    assert _logprob(d=d) == TOO_LARGE
    assert lib.ftp_logprob_backward(d, SOME, 0, SOME, SOME, SOME, SOME, SOME, SOME, 0, None) == TOO_LARGE
    assert lib.ftp_loss_logprob(d, SOME, 0, SOME, 1.0, SOME, 0, SOME, SOME, 1 << 20, None) == TOO_LARGE
    assert lib.ftp_loss_logprob(_d(1 << 20, 2, 1 << 12), SOME, 0, SOME, 1.0, SOME, 0, SOME, SOME, 1 << 20, None) == TOO_LARGE


def _logprob_backward(z=SOME, zs=0, lab=SOME, lse=SOME, h=SOME, gl=SOME, gh=SOME, dz=SOME, dzs=0):
    return lib.ftp_logprob_backward(_d(4, 8), z, zs, lab, lse, h, gl, gh, dz, dzs, None)


@pytest.mark.parametrize("bad", [dict(z=None), dict(dz=None), dict(lse=None), dict(lab=None), dict(h=None), dict(zs=7), dict(dzs=7), dict(z=SOME + 2),
                                 dict(dz=SOME + 2), dict(lab=SOME + 4), dict(lse=SOME + 2), dict(h=SOME + 2), dict(gl=SOME + 2), dict(gh=SOME + 2)])
def test_logprob_backward_refuses(bad):
    assert _logprob_backward(**bad) == ARG


def _loss(z=SOME, zs=0, lab=SOME, scale=1.0, dz=SOME, dzs=0, loss=SOME, ws=SOME, n=1 << 20):
    return lib.ftp_loss_logprob(_d(4, 8), z, zs, lab, scale, dz, dzs, loss, ws, n, None)


@pytest.mark.parametrize("bad", [dict(z=None), dict(lab=None), dict(dz=None, loss=None), dict(ws=None), dict(ws=SOME + 8), dict(n=100), dict(zs=7),
                                 dict(dzs=7), dict(scale=float("nan")), dict(scale=float("inf")), dict(z=SOME + 2), dict(dz=SOME + 2),
                                 dict(lab=SOME + 4), dict(loss=SOME + 2)])
def test_loss_refuses(bad):
    assert _loss(**bad) == ARG


# ---- the binding ----------------------------------------------------------------------------------------------------

def _t(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype)


def test_binding_refuses_shapes_types_and_devices():
    x = _t(4, 8)
    stat, w = _t(4), _t(8)
    with pytest.raises(ValueError, match="CUDA"):
        ftp.ftp_norm_forward(x, w, w, x, stat, stat)
    with pytest.raises(ValueError, match="y is"):
        ftp.ftp_norm_forward(x, w, w, _t(4, 9))
    with pytest.raises(ValueError, match="y is"):
        ftp.ftp_norm_forward(x, w, w, x.half())
    with pytest.raises(ValueError, match="float32, bfloat16 or float16"):
        ftp.ftp_norm_forward(x.double(), w, w, x.double())
    with pytest.raises(ValueError, match="weight has 7"):
        ftp.ftp_norm_forward(x, _t(7), w, x)
    with pytest.raises(ValueError, match="weight must be"):
        ftp.ftp_norm_forward(x, w.half(), w, x)
    with pytest.raises(ValueError, match="mean has 5"):
        ftp.ftp_norm_forward(x, w, w, x, _t(5), stat)
    with pytest.raises(ValueError, match="ckpt holds"):
        ftp.ftp_norm_forward(x, w, w, x, ckpt=_t(4 * 33 - 1, dtype=torch.uint8))
    with pytest.raises(ValueError, match="exactly one"):
        ftp.ftp_norm_backward(None, x, w, stat, stat, x, w, w, None)
    with pytest.raises(ValueError, match="workspace"):
        ftp.ftp_norm_backward(x, x, w, stat, stat, x, w, w, None)
    with pytest.raises(ValueError, match="workspace holds"):
        ftp.ftp_norm_backward(x, x, w, stat, stat, x, w, w, _t(3))
    with pytest.raises(ValueError, match="dx is"):
        ftp.ftp_norm_backward(x, x, w, stat, stat, _t(4, 4), w, w, None)
    with pytest.raises(ValueError, match="dense within"):
        ftp.ftp_ckpt_save(_t(4, 8, 3)[:, ::2], _t(1000, dtype=torch.uint8))
    with pytest.raises(ValueError, match="overlap"):
        ftp.ftp_ckpt_save(_t(1, 8).expand(4, 8), _t(1000, dtype=torch.uint8))
    with pytest.raises(ValueError, match="dense"):
        ftp.ftp_ckpt_save(_t(16)[::2], _t(1000, dtype=torch.uint8))
    with pytest.raises(ValueError, match="ckpt holds"):
        ftp.ftp_ckpt_load(_t(3, dtype=torch.uint8), x)
    labels = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="labels must be"):
        ftp.ftp_logprob(x, labels.int(), stat)
    with pytest.raises(ValueError, match="labels has 3"):
        ftp.ftp_logprob(x, labels[:3], stat)
    with pytest.raises(ValueError, match="top_index is for 9"):
        ftp.ftp_logprob(x, labels, top_index=torch.zeros(4, 9, dtype=torch.int64))
    with pytest.raises(ValueError, match="top_logp and top_index"):
        ftp.ftp_logprob(x, labels, top_logp=_t(4, 2), top_index=torch.zeros(4, 3, dtype=torch.int64))
    with pytest.raises(ValueError, match="entropy must not be None"):
        ftp.ftp_logprob_backward(x, labels, stat, None, None, stat, x)
    with pytest.raises(ValueError, match="dlogits is"):
        ftp.ftp_loss_logprob(x, labels, _t(4, 7), None, None)
    with pytest.raises(ValueError, match="loss_out has 2"):
        ftp.ftp_loss_logprob(x, labels, x, _t(2), None)
    with pytest.raises(ValueError, match="CUDA"):
        ftp.ftp_loss_logprob(x, labels, x, _t(1), _t(1 << 14, dtype=torch.uint8))
    with pytest.raises(ftp.FtpError):
        ftp.ftp_ckpt_bytes(_t(4, 0))


def test_backward_ckpt_checks_its_sizes():
    from paper_2409_09083_b200 import synth
    wl = synth.workload("C0")
    plan = ftp.ftp_plan(wl.layers, wl.N, wl.C, wl.H, wl.W, wl.grid, wl.groups)
    ws = torch.zeros(plan.workspace_bytes, dtype=torch.uint8)
    x, dy, p = _t(plan.in_floats), _t(plan.out_floats), _t(plan.param_floats)
    with pytest.raises(ValueError, match="x has 3"):
        ftp.ftp_backward_ckpt(plan, ws, _t(3), dy, p, None, p, ws)
    with pytest.raises(ValueError, match="CUDA"):
        ftp.ftp_backward_ckpt(plan, ws, x, dy, p, None, p, ws)
    h = plan._h
    for bad in ((None, SOME, SOME, SOME, SOME, SOME, SOME, SOME), (h, None, SOME, SOME, SOME, SOME, SOME, SOME),
                (h, SOME, None, SOME, SOME, None, SOME, SOME), (h, SOME, SOME, SOME, SOME, SOME, SOME, SOME),       # dx = x
                (h, SOME, SOME, None, SOME, None, SOME, SOME), (h, SOME, SOME, SOME, None, None, SOME, SOME),
                (h, SOME, SOME, SOME, SOME, None, None, SOME), (h, SOME, SOME, SOME, SOME, None, SOME, SOME + 8),
                (h, SOME + 8, SOME, SOME, SOME, None, SOME, SOME)):
        assert lib.ftp_backward_ckpt(*bad, None) == ARG


def test_backward_ckpt_refuses_a_delta_in_the_place_that_it_fills():
    """x receives the checkpoint's values before the delta is read: where input and output maps have one size, they could be one array."""
    from paper_2409_09083_b200 import synth
    plan = ftp.ftp_plan([synth.conv(4, 4, 3)], 1, 4, 8, 8, (1, 1), ((1, 1),))
    assert plan.in_floats == plan.out_floats
    h, x = plan._h, SOME + (1 << 16)
    assert lib.ftp_backward_ckpt(h, SOME, x, x, SOME, None, SOME, SOME, None) == ARG


class _OnGpu:
    """A float32 tensor's outside, on a device that this machine need not have."""
    dtype, is_cuda = torch.float32, True

    def __init__(self, count, device):
        self.count, self.device = count, torch.device(device)

    def numel(self):
        return self.count

    def element_size(self):
        return 4

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return SOME

    def get_device(self):
        return self.device.index


def test_backward_ckpt_runs_on_its_arrays_device(monkeypatch):
    """As the other operators do: with x's device current, on that device's stream, and not with arrays of several devices."""
    from paper_2409_09083_b200 import synth
    plan = ftp.ftp_plan([synth.conv(4, 8, 3)], 1, 4, 8, 8, (1, 1), ((1, 1),))
    counts = dict(ckpt=ftp.ftp_ckpt_bytes(plan.shape), x=plan.in_floats, dy=plan.out_floats, params=plan.param_floats, dx=plan.in_floats,
                  dparams=plan.param_floats, workspace=plan.workspace_bytes)
    arrays = {k: _OnGpu(n, "cuda:1") for k, n in counts.items()}
    seen = []
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: pytest.fail("the current device's stream was taken"))
    monkeypatch.setattr(binding, "_call", lambda fn, x, name, stream, *args: seen.append((x, name, stream, args)))
    ftp.ftp_backward_ckpt(plan, **arrays)
    x, name, stream, args = seen[0]
    assert x is arrays["x"] and name == "x" and stream is None
    assert [getattr(a, "value", a) for a in args] == [plan._h.value] + 7 * [SOME]
    for k in counts:
        if k != "x":
            with pytest.raises(ValueError, match=f"{k} (is|must be a contiguous tensor) on cuda:"):
                ftp.ftp_backward_ckpt(plan, **{**arrays, k: _OnGpu(counts[k], "cuda:0")})
