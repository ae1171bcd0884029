"""Host-side checks of the scoring and 8-bit entry points: bad arguments are
refused, with a message, before anything is launched."""

import ctypes

import pytest
import torch

from paper_1907_05701_amd import binding as bd

PTR = ctypes.c_void_p(256)   # never read: every call here is refused on the host
ODD = ctypes.c_void_p(264)
EINVAL, EUNSUPPORTED = bd.BLSTM_EINVAL, bd.BLSTM_EUNSUPPORTED


def _refused(rc, code):
    assert rc == code
    assert len(bd.lib().blstm_last_error()) > 10


def _scores(**over):
    q = bd.SoftmaxScores(256, 256, 256, 256, 256, 3, 5, 1.0)
    for k, v in over.items():
        setattr(q, k, v)
    return q


def _grads(**over):
    g = bd.SoftmaxScoreGrads(256, 256, 256, 3, 1.0)
    for k, v in over.items():
        setattr(g, k, v)
    return g


BAD_SCORES = [
    (dict(ids=None), EINVAL), (dict(logprob=None), EINVAL), (dict(top=None), EINVAL), (dict(idx=None), EINVAL),
    (dict(n=-1), EINVAL), (dict(k=-1), EINVAL), (dict(k=101), EINVAL), (dict(n=257), EUNSUPPORTED),
    (dict(k=257), EUNSUPPORTED), (dict(n=0, k=0, entropy=None), EINVAL), (dict(temperature=0.0), EINVAL),
    (dict(temperature=-1.0), EINVAL), (dict(temperature=float("nan")), EINVAL), (dict(temperature=float("inf")), EINVAL)]


@pytest.mark.parametrize("over,code", BAD_SCORES)
def test_what_is_asked_of_rows(over, code):
    L, q = bd.lib(), ctypes.byref(_scores(**over))
    _refused(L.softmax_logprob_rows(PTR, 100, 4, 100, 1, q, None), code)
    d = bd.make_dims(2, 40, 64, 32, 100, 21, 8, "bf16")
    _refused(L.softmax_logprob(ctypes.byref(d), PTR, PTR, PTR, q, PTR, None), code)
    _refused(L.int8_logprob_rows(PTR, 64, 4, 64, 1, PTR, 64, PTR, 100, 64, None, q, PTR, None), code)


@pytest.mark.parametrize("over,code", [
    (dict(ids=None), EINVAL), (dict(dlogprob=None), EINVAL), (dict(n=-1), EINVAL), (dict(n=257), EUNSUPPORTED),
    (dict(n=0, dentropy=None), EINVAL), (dict(temperature=0.0), EINVAL), (dict(temperature=float("nan")), EINVAL)])
def test_gradients_that_are_given(over, code):
    L, g = bd.lib(), ctypes.byref(_grads(**over))
    _refused(L.softmax_logprob_bwd_rows(PTR, 100, 4, 100, 1, g, PTR, 100, None), code)
    d = bd.make_dims(2, 40, 64, 32, 100, 21, 8, "bf16")
    _refused(L.softmax_logprob_bwd(ctypes.byref(d), PTR, PTR, PTR, g, PTR, PTR, PTR, None), code)


def test_rows_of_logits():
    L, q, g = bd.lib(), ctypes.byref(_scores()), ctypes.byref(_grads())
    for args, code in [((None, 100, 4, 100, 1), EINVAL), ((PTR, 99, 4, 100, 1), EINVAL), ((PTR, 100, 0, 100, 1), EINVAL),
                       ((PTR, 100, 4, 0, 1), EINVAL), ((PTR, 100, 4, 100, 2), EINVAL),
                       ((PTR, 100, 1 << 22, 100, 1), EUNSUPPORTED),
                       ((PTR, 1 << 19, 4, (1 << 18) + 1, 1), EUNSUPPORTED)]:
        _refused(L.softmax_logprob_rows(*args, q, None), code)
        _refused(L.softmax_logprob_bwd_rows(*args, g, PTR, 1 << 19, None), code)
    _refused(L.softmax_logprob_rows(PTR, 100, 4, 100, 1, None, None), EINVAL)
    _refused(L.softmax_logprob_bwd_rows(PTR, 100, 4, 100, 1, None, PTR, 100, None), EINVAL)
    _refused(L.softmax_logprob_bwd_rows(PTR, 100, 4, 100, 1, g, None, 100, None), EINVAL)
    _refused(L.softmax_logprob_bwd_rows(PTR, 100, 4, 100, 1, g, PTR, 99, None), EINVAL)     # also: over logits
    _refused(L.softmax_logprob_bwd_rows(PTR, 100, 4, 100, 1, g, PTR, 104, None), EINVAL)    # over logits, another pitch


def test_head_needs_its_inputs():
    L, d = bd.lib(), ctypes.byref(bd.make_dims(2, 40, 64, 32, 100, 21, 8, "bf16"))
    q, g = ctypes.byref(_scores()), ctypes.byref(_grads())
    for at in range(4):
        a = [PTR] * 4
        a[at] = None
        _refused(L.softmax_logprob(d, a[0], a[1], a[2], q, a[3], None), EINVAL)
        _refused(L.softmax_logprob_bwd(d, a[0], a[1], a[2], g, PTR, PTR, a[3], None), EINVAL)
    _refused(L.softmax_logprob_bwd(d, PTR, PTR, PTR, g, None, PTR, PTR, None), EINVAL)
    _refused(L.softmax_logprob_bwd(d, PTR, PTR, PTR, g, PTR, None, PTR, None), EINVAL)


def test_quantize_refusals():
    L = bd.lib()
    ok = [PTR, 60, 4, 60, 1, PTR, 64, 64, PTR, None]
    for at, v, code in [(0, None, EINVAL), (1, 59, EINVAL), (2, 0, EINVAL), (2, 1 << 22, EUNSUPPORTED), (3, 0, EINVAL),
                        (3, 65, EINVAL), (4, 7, EINVAL), (5, None, EINVAL), (5, ODD, EINVAL), (6, 48, EINVAL),
                        (6, 72, EINVAL), (6, (1 << 22) + 16, EUNSUPPORTED), (7, 60, EINVAL), (7, 48, EINVAL),
                        (8, None, EINVAL)]:
        a = list(ok)
        a[at] = v
        _refused(L.int8_quantize_rows(*a), code)
    _refused(L.int8_quantize_rows(PTR, 1 << 20, 4, 1 << 17, 1, PTR, 1 << 17, 1 << 17, PTR, None), EUNSUPPORTED)


def test_linear_refusals():
    L = bd.lib()
    #       q    ldq xs  M  w    ldw  ws   N   K  bias  y   ldy prec
    ok = [PTR, 64, PTR, 4, PTR, 64, PTR, 30, 64, None, PTR, 30, 1, None]
    for at, v, code in [(0, None, EINVAL), (0, ODD, EINVAL), (1, 48, EINVAL), (1, 72, EINVAL), (2, None, EINVAL),
                        (3, 0, EINVAL), (3, 1 << 22, EUNSUPPORTED), (4, None, EINVAL), (4, ODD, EINVAL), (5, 56, EINVAL),
                        (5, 1 << 23, EUNSUPPORTED), (6, None, EINVAL), (7, 0, EINVAL), (8, 60, EINVAL), (8, 0, EINVAL),
                        (10, None, EINVAL), (11, 29, EINVAL), (12, 5, EINVAL)]:
        a = list(ok)
        a[at] = v
        _refused(L.int8_linear(*a), code)
    _refused(L.int8_linear(PTR, 1 << 17, PTR, 4, PTR, 1 << 17, PTR, 30, 1 << 17, None, PTR, 30, 1, None), EUNSUPPORTED)
    _refused(L.int8_linear(PTR, 64, PTR, 4, PTR, 64, PTR, 1 << 24, 64, None, PTR, 1 << 24, 1, None), EUNSUPPORTED)
    _refused(L.int8_linear(PTR, 64, PTR, 1 << 21, PTR, 64, PTR, 1 << 21, 64, None, PTR, 1 << 21, 1, None), EUNSUPPORTED)


def test_linear_of_tokens_refusals():
    L = bd.lib()
    #       x   ldx M  K  prec w    ldw ws_   N   Kw bias  y   ldy ws
    ok = [PTR, 60, 4, 60, 1, PTR, 64, PTR, 30, 64, None, PTR, 30, PTR, None]
    for at, v, code in [(0, None, EINVAL), (1, 59, EINVAL), (2, 0, EINVAL), (2, 1 << 22, EUNSUPPORTED), (3, 0, EINVAL),
                        (3, 65, EINVAL), (4, 3, EINVAL), (5, None, EINVAL), (5, ODD, EINVAL), (6, 48, EINVAL), (7, None, EINVAL),
                        (8, 0, EINVAL), (9, 60, EINVAL), (11, None, EINVAL), (12, 29, EINVAL), (13, None, EINVAL),
                        (13, ODD, EINVAL)]:
        a = list(ok)
        a[at] = v
        _refused(L.int8_linear_rows(*a), code)
    q = ctypes.byref(_scores())
    #       x   ldx M  P  prec w    ldw ws_    K   Kw bias scores ws
    ok = [PTR, 60, 4, 60, 1, PTR, 64, PTR, 100, 64, None, q, PTR, None]
    for at, v, code in [(0, None, EINVAL), (1, 59, EINVAL), (2, 0, EINVAL), (2, 1 << 22, EUNSUPPORTED), (3, 0, EINVAL),
                        (3, 65, EINVAL), (4, 3, EINVAL), (5, None, EINVAL), (5, ODD, EINVAL), (6, 48, EINVAL), (7, None, EINVAL),
                        (8, 0, EINVAL), (8, (1 << 18) + 1, EUNSUPPORTED), (9, 60, EINVAL), (11, None, EINVAL),
                        (12, None, EINVAL), (12, ODD, EINVAL)]:
        a = list(ok)
        a[at] = v
        _refused(L.int8_logprob_rows(*a), code)


def test_workspace_sizes():
    assert bd.int8_linear_ws_bytes(1, 16) >= 16 + 4
    assert bd.int8_linear_ws_bytes(1000, 1024) >= 1000 * 1028
    assert bd.int8_logprob_ws_bytes(1000, 32000, 256) >= bd.int8_linear_ws_bytes(1000, 256)
    for bad in [(0, 16), (4, 0), (1 << 22, 16), (4, 1 << 17)]:
        with pytest.raises(bd.BlstmError):
            bd.int8_linear_ws_bytes(*bad)
    for bad in [(0, 100, 16), (4, 0, 16), (4, 100, 0), (1 << 22, 100, 16), (4, (1 << 18) + 1, 16), (4, 100, 1 << 17)]:
        with pytest.raises(bd.BlstmError):
            bd.int8_logprob_ws_bytes(*bad)


def test_tensors_have_to_be_on_the_gpu():
    f, i = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.int8)
    with pytest.raises(ValueError):
        bd.softmax_logprob_rows(f, entropy=torch.zeros(4))
    with pytest.raises(ValueError):
        bd.softmax_logprob_bwd_rows(f, f, dentropy=torch.zeros(4))
    with pytest.raises(ValueError):
        bd.int8_quantize_rows(f, i, torch.zeros(4))
    with pytest.raises(ValueError):
        bd.int8_linear(i, torch.zeros(4), i, torch.zeros(4), f)
    with pytest.raises(ValueError):
        bd.int8_linear_rows(f, i, torch.zeros(4), torch.zeros(4, 4), torch.zeros(1 << 16, dtype=torch.uint8))


def test_head_workspaces_are_bounded():
    """Frames past a part of about 180 MB are taken in turn."""
    for M in (1, 2688, 30000, 1 << 20, (1 << 22) - 1):
        for K in (100, 9001, 32000, 1 << 18):
            if (M + 127) // 128 * ((K + 127) // 128) >= 1 << 22:
                continue   # refused
            for Kw in (16, 256, 1024):
                assert bd.int8_logprob_ws_bytes(M, K, Kw) < 200 << 20, (M, K, Kw)


@pytest.mark.parametrize("call", ["softmax_logprob_rows", "softmax_logprob_bwd_rows", "int8_quantize_rows", "int8_linear",
                                  "int8_linear_rows", "int8_logprob_rows", "softmax_topk_rows"])
def test_the_first_tensor_is_required(call):
    n = {"softmax_logprob_rows": 0, "softmax_logprob_bwd_rows": 1, "int8_quantize_rows": 2, "int8_linear": 4,
         "int8_linear_rows": 4, "int8_logprob_rows": 3, "softmax_topk_rows": 2}[call]
    with pytest.raises(ValueError, match="required"):
        getattr(bd, call)(None, *[None] * n)


def test_rows_that_are_not_there():
    """int8_linear takes its sizes from y."""
    for name in ("x", "y", "logits"):
        with pytest.raises(ValueError, match=f"{name} is required"):
            bd._floats(name, None, 0)


def test_calls_ask_for_the_device_by_torch_s_public_name(monkeypatch):
    """With nothing private to find it by, a call reaches the library, which refuses these arguments."""
    monkeypatch.delattr(torch._C, "_cuda_getDevice", raising=False)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    stream = type("Stream", (), {"cuda_stream": 0, "device": torch.device("cuda", 0)})()
    with pytest.raises(bd.BlstmError):
        bd._call("int8_quantize_rows", 0, stream, None, 64, 4, 64, 1, PTR, 64, 64, PTR)


@pytest.mark.parametrize("M", [17, 32, 64])
def test_head_plans_for_the_workgroups_that_run_at_a_time(M):
    """512 columns of few frames leave LDS for one workgroup a CU: 256 ranges of 131072 classes, 16 bytes a frame each,
    beside tokens and group maxima (1024 pairs of tiles, 4 a wave along the classes)."""
    waves = 4 if M <= 32 else 2
    up = lambda n: -(-n // 256) * 256  # noqa: E731
    most = up(M * 512) + up(M * 4) + up(M * 256 * 16) + up(M * 1024 * waves * 4 * 4)
    assert bd.int8_logprob_ws_bytes(M, 131072, 512) <= most


@pytest.mark.parametrize("K,Kw", [(100, 16), (1000, 256), (9001, 512), (32000, 256), (32000, 1024), (131072, 512), (1 << 18, 32), (5000, 1040)])
def test_a_workspace_for_some_frames_is_enough_for_fewer(K, Kw):
    """As a program keeps it that calls with batches of several sizes."""
    sizes = [bd.int8_logprob_ws_bytes(M, K, Kw) for M in (*range(1, 400), *range(400, 6000, 37), 20000, 100000)]
    assert sizes == sorted(sizes)
    sizes = [bd.int8_linear_ws_bytes(M, Kw) for M in range(1, 400)]
    assert sizes == sorted(sizes)
