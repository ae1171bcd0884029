"""Host-side checks of the state space and distillation entry points: bad
arguments are refused, with a message, before anything is launched."""

import ctypes

import pytest

from paper_1907_05701_amd import binding as bd

PTR = ctypes.c_void_p(256)   # never read: every call here is refused on the host


def _dims(**over):
    return bd.make_ssm_dims(**dict(dict(T=5, B=3, D=12, N=4, G=2, W=4, precision="bf16"), **over))


def _scan_in(dims, **over):
    a = bd.SsmScanIn(256, 256, 256, 256, 256, dims.D, dims.D, dims.G * dims.N, dims.G * dims.N, dims.D, 256, 256, 256,
                     256, None, bd.SSM_SOFTPLUS)
    for k, v in over.items():
        setattr(a, k, v)
    return a


def _refused(rc, code):
    assert rc == code
    assert len(bd.lib().blstm_last_error()) > 10


@pytest.mark.parametrize("over,code", [
    (dict(T=0), -1), (dict(B=-1), -1), (dict(N=0), -1), (dict(W=0), -1), (dict(G=5), -1), (dict(N=65), -2),
    (dict(W=9), -2), (dict(T=1 << 13, B=1 << 12), -2), (dict(D=(1 << 20) + 2), -2), (dict(precision=3), -1)])
def test_bad_ssm_dims(over, code):
    with pytest.raises(bd.BlstmError) as e:
        bd.ssm_workspace_bytes(_dims(**over))
    assert e.value.code == code
    L, d = bd.lib(), _dims(**over)
    ok = _dims()
    _refused(L.ssm_scan_fwd(ctypes.byref(d), ctypes.byref(_scan_in(ok)), PTR, 1 << 30, None, None, PTR, None), code)
    _refused(L.ssm_conv_fwd(ctypes.byref(d), PTR, 1 << 30, PTR, None, None, None, PTR, 1 << 30, None, 0, None), code)


def test_scans_of_more_threads_than_a_launch_has_are_refused():
    for over in (dict(T=1, B=1 << 24, D=512, G=1), dict(T=1 << 10, B=1 << 10, D=64, N=64, G=64)):
        with pytest.raises(bd.BlstmError) as e:
            bd.ssm_workspace_bytes(_dims(**over))
        assert e.value.code == bd.BLSTM_EUNSUPPORTED
    L, d = bd.lib(), _dims(T=1, B=1 << 24, D=512, G=1)
    i = ctypes.byref(_scan_in(d))
    _refused(L.ssm_scan_step(ctypes.byref(d), i, None, 1 << 24, PTR, PTR, 512, None), bd.BLSTM_EUNSUPPORTED)
    _refused(L.ssm_conv_step(ctypes.byref(d), PTR, 512, PTR, None, None, 1 << 24, PTR, PTR, 512, 0, None),
             bd.BLSTM_EUNSUPPORTED)


def test_workspaces_hold_a_state_for_every_eight_frames():
    a = bd.ssm_workspace_bytes(_dims(T=8, N=16))
    b = bd.ssm_workspace_bytes(_dims(T=9, N=16))
    assert a["saved"] == 3 * 12 * 16 * 4 and b["saved"] == 2 * a["saved"]
    # states are held in whole lanes
    assert bd.ssm_workspace_bytes(_dims(T=8, N=13))["saved"] == a["saved"]


@pytest.mark.parametrize("field", ["x", "dt", "Bm", "Cm", "A"])
def test_scan_needs_its_inputs(field):
    L, d = bd.lib(), _dims()
    bad = _scan_in(d, **{field: None})
    _refused(L.ssm_scan_fwd(ctypes.byref(d), ctypes.byref(bad), PTR, 12, None, None, PTR, None), bd.BLSTM_EINVAL)
    one = _dims(T=1)
    _refused(L.ssm_scan_step(ctypes.byref(one), ctypes.byref(bad), None, 3, PTR, PTR, 12, None), bd.BLSTM_EINVAL)


@pytest.mark.parametrize("field", ["ldx", "lddt", "ldb", "ldc", "ldz"])
def test_scan_refuses_short_pitches(field):
    L, d = bd.lib(), _dims()
    bad = _scan_in(d, **{field: 7})
    _refused(L.ssm_scan_fwd(ctypes.byref(d), ctypes.byref(bad), PTR, 12, None, None, PTR, None), bd.BLSTM_EINVAL)


def test_scan_refusals():
    L, d, one = bd.lib(), _dims(), _dims(T=1)
    i = _scan_in(d)
    _refused(L.ssm_scan_fwd(ctypes.byref(d), ctypes.byref(i), None, 12, None, None, PTR, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_scan_fwd(ctypes.byref(d), ctypes.byref(i), PTR, 11, None, None, PTR, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_scan_fwd(ctypes.byref(d), ctypes.byref(_scan_in(d, flags=4)), PTR, 12, None, None, PTR, None),
             bd.BLSTM_EINVAL)
    _refused(L.ssm_scan_step(ctypes.byref(d), ctypes.byref(i), None, 3, PTR, PTR, 12, None), bd.BLSTM_EINVAL)   # T
    _refused(L.ssm_scan_step(ctypes.byref(one), ctypes.byref(i), None, 2, PTR, PTR, 12, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_scan_step(ctypes.byref(one), ctypes.byref(i), PTR, 0, PTR, PTR, 12, None), bd.BLSTM_EINVAL)
    g = bd.SsmScanGrads(256, 256, 256, 256, None, 12, 12, 8, 8, 12, 256, None, None, None)   # z given, dz not
    _refused(L.ssm_scan_bwd(ctypes.byref(d), ctypes.byref(i), PTR, 12, None, PTR, ctypes.byref(g), PTR, None),
             bd.BLSTM_EINVAL)
    g.dz, g.lddb = 256, 3
    _refused(L.ssm_scan_bwd(ctypes.byref(d), ctypes.byref(i), PTR, 12, None, PTR, ctypes.byref(g), PTR, None),
             bd.BLSTM_EINVAL)


def test_scan_refuses_misaligned_buffers():
    L, d = bd.lib(), _dims()
    i = ctypes.byref(_scan_in(d))
    odd = ctypes.c_void_p(264)
    _refused(L.ssm_scan_fwd(ctypes.byref(d), i, PTR, 12, None, odd, PTR, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_scan_fwd(ctypes.byref(d), i, PTR, 12, None, None, odd, None), bd.BLSTM_EINVAL)
    g = bd.SsmScanGrads(256, 256, 256, 256, 256, 12, 12, 8, 8, 12, 256, None, None, None)
    _refused(L.ssm_scan_bwd(ctypes.byref(d), i, PTR, 12, None, odd, ctypes.byref(g), PTR, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_scan_bwd(ctypes.byref(d), i, PTR, 12, None, PTR, ctypes.byref(g), odd, None), bd.BLSTM_EINVAL)


def test_conv_refusals():
    L, d, one = bd.lib(), _dims(), _dims(T=1)
    r = ctypes.byref(d)
    _refused(L.ssm_conv_fwd(r, None, 12, PTR, None, None, None, PTR, 12, None, 0, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_conv_fwd(r, PTR, 11, PTR, None, None, None, PTR, 12, None, 0, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_conv_fwd(r, PTR, 12, PTR, None, None, PTR, PTR, 12, PTR, 0, None), bd.BLSTM_EINVAL)   # state_out is state
    _refused(L.ssm_conv_fwd(r, PTR, 12, PTR, None, None, None, PTR, 12, None, 1, None), bd.BLSTM_EINVAL)   # flags
    _refused(L.ssm_conv_bwd(r, PTR, 12, PTR, None, None, None, PTR, 12, None, PTR, 12, None, None, None, PTR, 0, None),
             bd.BLSTM_EINVAL)
    _refused(L.ssm_conv_step(r, PTR, 12, PTR, None, None, 3, PTR, PTR, 12, 0, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_conv_step(ctypes.byref(one), PTR, 12, PTR, None, None, 2, PTR, PTR, 12, 0, None), bd.BLSTM_EINVAL)
    _refused(L.ssm_conv_step(ctypes.byref(one), PTR, 12, PTR, None, None, 3, None, PTR, 12, 0, None), bd.BLSTM_EINVAL)


def _topk(M=4, K=10, ld=10, prec=1, k=3, tau=1.0, top=PTR):
    return bd.lib().softmax_topk_rows(PTR, ld, M, K, prec, k, ctypes.c_float(tau), top, PTR, None, None)


@pytest.mark.parametrize("over,code", [
    (dict(M=0), -1), (dict(K=0), -1), (dict(ld=9), -1), (dict(prec=2), -1), (dict(k=0), -1), (dict(k=11), -1),
    (dict(k=257, K=300, ld=300), -2), (dict(K=(1 << 18) + 1, ld=1 << 19), -2), (dict(tau=0.0), -1),
    (dict(tau=float("nan")), -1), (dict(tau=float("inf")), -1), (dict(tau=-1.0), -1), (dict(top=None), -1)])
def test_topk_refusals(over, code):
    _refused(_topk(**over), code)


@pytest.mark.parametrize("over,code", [
    (dict(top=None), -1), (dict(idx=None), -1), (dict(k=0), -1), (dict(k=300), -2), (dict(temperature=0.0), -1),
    (dict(soft=float("inf")), -1), (dict(hard=float("nan")), -1)])
def test_distill_refusals(over, code):
    t = bd.SoftmaxTeacher(256, 256, None, None, None, 3, 1.0, 1.0, 0.0)
    for k, v in over.items():
        setattr(t, k, v)
    L, F = bd.lib(), ctypes.c_float(1.0)
    _refused(L.softmax_distill_rows(PTR, 10, 4, 10, 1, ctypes.byref(t), F, PTR, ctypes.c_void_p(512), 10, None), code)
    d = bd.make_dims(1, 8, 64, 8, 10, 2, 2, "fp32")
    _refused(L.softmax_distill_fwd_bwd(ctypes.byref(d), PTR, None, PTR, ctypes.byref(t), F, PTR, PTR, PTR, PTR, None), code)


def test_distill_buffers():
    t = bd.SoftmaxTeacher(256, 256, None, None, None, 3, 1.0, 1.0, 0.0)
    L, F, other = bd.lib(), ctypes.c_float(1.0), ctypes.c_void_p(512)
    _refused(L.softmax_distill_rows(PTR, 10, 4, 10, 1, ctypes.byref(t), F, None, other, 10, None), -1)
    _refused(L.softmax_distill_rows(PTR, 10, 4, 10, 1, ctypes.byref(t), F, PTR, other, 9, None), -1)
    _refused(L.softmax_distill_rows(PTR, 10, 4, 10, 1, ctypes.byref(t), F, other, PTR, 12, None), -1)   # in place, other pitch
    d = bd.make_dims(1, 8, 64, 8, 10, 2, 2, "bf16")
    _refused(L.softmax_topk(ctypes.byref(d), PTR, None, PTR, 3, F, PTR, PTR, None, PTR, None), -1)      # no theta_lp
    _refused(L.softmax_topk(ctypes.byref(d), PTR, PTR, PTR, 11, F, PTR, PTR, None, PTR, None), -1)


def test_the_binding_refuses_host_tensors():
    import torch
    d = bd.make_ssm_dims(T=1, B=1, D=4, N=1, precision="fp32")
    x = torch.zeros(1, 1, 4)
    with pytest.raises(ValueError):
        bd.ssm_conv_fwd(d, x, x, None, x)
    with pytest.raises(ValueError):
        bd.softmax_topk_rows(torch.zeros(2, 4), torch.zeros(2, 1), torch.zeros(2, 1, dtype=torch.int32))


@pytest.mark.parametrize("n", ["T", "B", "D", "K"])
def test_a_teacher_of_another_shape_is_refused(n):
    from types import SimpleNamespace

    from paper_1907_05701_amd.train import Trainer
    shape = dict(T=3, B=2, D=4, K=10)
    step = SimpleNamespace(shape=shape, device="cpu")
    teacher = SimpleNamespace(shape=dict(shape, **{n: 11}))
    with pytest.raises(ValueError, match=f"teacher's {n} is 11"):
        Trainer(step, [], 0.1, 4, teacher=teacher)


# -------------------------------------------------------- limits by direction ---
def _sizes(d, *names):
    """ssm_workspace_bytes of some buffers alone: (code, their sizes)."""
    v = {n: ctypes.c_size_t() for n in names}
    args = [ctypes.byref(v[n]) if n in v else None for n in ("saved", "fwd", "bwd", "conv_bwd")]
    return bd.lib().ssm_workspace_bytes(ctypes.byref(d), *args), {n: x.value for n, x in v.items()}


def test_a_forward_is_not_held_to_the_backwards_limits():
    """The launch that sums the backward's partials, and its lanes, are the backward's alone."""
    L = bd.lib()
    # 2 T B G N past a launch's threads; states on four lanes in the backward where the forward has two
    for over in (dict(T=1 << 10, B=1 << 10, D=64, N=64, G=64), dict(T=1, B=1 << 24, D=64, N=16, G=1)):
        d = _dims(**over)
        assert _sizes(d, "saved", "fwd")[0] == 0
        _refused(_sizes(d, "bwd")[0], bd.BLSTM_EUNSUPPORTED)
        i = _scan_in(d)
        # past the limits, to the next check (nothing is launched: y, then dy are missing)
        _refused(L.ssm_scan_fwd(ctypes.byref(d), ctypes.byref(i), None, d.D, None, None, PTR, None), bd.BLSTM_EINVAL)
        g = bd.SsmScanGrads(256, 256, 256, 256, 256, d.D, d.D, d.G * d.N, d.G * d.N, d.D, 256, None, None, None)
        _refused(L.ssm_scan_bwd(ctypes.byref(d), ctypes.byref(i), None, d.D, None, PTR, ctypes.byref(g), PTR, None),
                 bd.BLSTM_EUNSUPPORTED)


def test_a_convolution_is_not_held_to_the_scans_limits():
    d = _dims(T=1, B=1 << 24, D=512, G=1, N=1)
    rc, n = _sizes(d, "conv_bwd")
    assert rc == 0 and n["conv_bwd"] > 0
    _refused(_sizes(d, "fwd")[0], bd.BLSTM_EUNSUPPORTED)


def test_the_binding_asks_for_the_sizes_of_its_call():
    big = dict(T=1 << 10, B=1 << 10, D=64, N=64, G=64)
    assert bd._ssm_bytes(_dims(**big), "saved") > 0
    with pytest.raises(bd.BlstmError):
        bd._ssm_bytes(_dims(**big), "bwd")
    d = _dims()
    assert {n: bd._ssm_bytes(d, n) for n in ("saved", "fwd", "bwd", "conv_bwd")} == bd.ssm_workspace_bytes(d)
    d.T = 50   # other values of the same object
    assert bd._ssm_bytes(d, "saved") == bd.ssm_workspace_bytes(d)["saved"]


# ------------------------------------------------------------------ refusals ---
def test_a_gate_gradient_without_a_gate_is_refused():
    """There is none to write: dz would stay as it was."""
    L, d = bd.lib(), _dims()
    i = _scan_in(d, z=None)
    g = bd.SsmScanGrads(256, 256, 256, 256, 256, 12, 12, 8, 8, 12, 256, None, None, None)
    # lddx is short, too: refused either way, but for the gate first
    g.lddx = 3
    _refused(L.ssm_scan_bwd(ctypes.byref(d), ctypes.byref(i), PTR, 12, None, PTR, ctypes.byref(g), PTR, None),
             bd.BLSTM_EINVAL)
    assert b"dz" in L.blstm_last_error()


def test_a_stream_of_another_device_is_refused():
    from types import SimpleNamespace

    import torch
    other = SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0)
    with pytest.raises(ValueError, match="stream"):
        bd._call("softmax_topk_rows", 0, other)


# ------------------------------------------------- calls that have no teacher ---
def test_a_trainer_calls_a_step_without_a_teacher_as_before(monkeypatch):
    """A step object whose step() takes the rate and the flags alone."""
    import numpy as np
    import torch

    from paper_1907_05701_amd.train import Trainer
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: None)

    class Step:
        shape, device = dict(T=3, B=2, D=4, K=10), torch.device("cpu")
        x, labels, loss = torch.zeros(3, 2, 4), torch.zeros(3, 2, dtype=torch.int32), torch.ones(1)
        calls = []

        def step(self, lr, flags=0):
            self.calls.append((lr, flags))

        def check_recurrence(self):
            pass

    got = Trainer(Step(), [(np.zeros((3, 2, 4), np.float32), np.zeros((3, 2), np.int32))], 0.1, 2, warmup_epochs=1,
                  flags=2).run(2)
    assert len(Step.calls) == 2 and all(f == 2 for _, f in Step.calls) and [h[2] for h in got] == [1.0, 1.0]


def test_a_learner_step_calls_its_own_methods_as_before(monkeypatch):
    """A learner whose gradient() and step() take what they took before there were teachers."""
    import contextlib

    import torch

    from paper_1907_05701_amd.step import LearnerStep
    calls = []

    class Own(LearnerStep):
        def gradient(self):
            calls.append("gradient")

        def update(self, lr, flags=0, grads=None, scale=1.0):
            calls.append("update")

    shape = dict(L=1, D=4, H=16, P=8, K=10, T=2, B=2, precision="fp32", device="cpu")
    Own(**shape).step(0.1)
    assert calls == ["gradient", "update"]

    class Stepping(LearnerStep):
        def step(self, lr, flags=0):
            calls.append((lr, flags))

    monkeypatch.setattr(torch.cuda, "CUDAGraph", lambda: "graph")
    monkeypatch.setattr(torch.cuda, "graph", lambda g: contextlib.nullcontext())
    assert Stepping(**shape).capture(0.5, steps=2, flags=3) == "graph"
    assert calls[2:] == [(0.5, 3), (0.5, 3)]
