"""Layer norm, matrix product and their gradients: what the calls refuse, before anything is launched (no GPU needed)."""
import copy
import ctypes
import pickle
import sys
import threading
import types

import pytest
import torch

from paper_2609_32420_b200 import build as cbuild
from paper_2609_32420_b200 import carnator as cn

P, BIG = 1 << 20, 1 << 40       # a 256-byte aligned address that is never read, a workspace size that suffices


@pytest.fixture(scope="module", autouse=True)
def _built():
    cbuild.build_library()


def norm_shape(**kw):
    x = torch.empty((2, 3, 40, 128), dtype=torch.bfloat16)
    s = cn.make_norm_shape(x, x)
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(s, k)[v[0]] = v[1]
        else:
            setattr(s, k, v)
    return s


def linear_shape(**kw):
    x, w, y = (torch.empty(n, dtype=torch.bfloat16) for n in ((2, 40, 128), (64, 128), (2, 40, 64)))
    s = cn.make_linear_shape(x, w, y, Z=y, dX=x, dW=w)
    for k, v in kw.items():
        if isinstance(v, tuple):
            getattr(s, k)[v[0]] = v[1]
        else:
            setattr(s, k, v)
    return s


def call_norm(s, X=P, Y=P, weight=P, mean=P, rstd=P):
    return cn.lib().carnator_layer_norm(X, weight, P, P, P, ctypes.byref(s), Y, mean, rstd, None)


def call_norm_backward(s, dY=P, X=P, mean=P, dX=P, dw=P, ws=P, ws_bytes=BIG):
    return cn.lib().carnator_layer_norm_backward(dY, X, mean, P, P, P, P, ctypes.byref(s), dX, dw, P, P, P, ws, ws_bytes, None)


def call_linear(s, X=P, W=P, bias=P, gate=P, residual=P, Y=P, Z=P, ws=P, ws_bytes=BIG):
    return cn.lib().carnator_linear(X, W, bias, gate, residual, ctypes.byref(s), Y, Z, ws, ws_bytes, None)


def call_linear_backward(s, dY=P, X=P, W=P, Z=P, gate=P, dX=P, dW=P, db=P, dg=P, ws=P, ws_bytes=BIG):
    return cn.lib().carnator_linear_backward(dY, X, W, Z, gate, ctypes.byref(s), dX, dW, db, dg, ws, ws_bytes, None)


def expect(call, status, **kw):
    before = cn.kernel_launches()
    assert call(**kw) == status
    assert cn.kernel_launches() == before


NORM_BAD = [
    (dict(B=0), cn.ERR_INVALID_ARG), (dict(N=0), cn.ERR_INVALID_ARG), (dict(C=0), cn.ERR_INVALID_ARG), (dict(H=-1), cn.ERR_INVALID_ARG),
    (dict(C=16385), cn.ERR_UNSUPPORTED), (dict(B=65536), cn.ERR_UNSUPPORTED), (dict(H=1 << 16, N=1 << 15), cn.ERR_UNSUPPORTED),
    (dict(x_dtype=2), cn.ERR_INVALID_ARG), (dict(y_dtype=-1), cn.ERR_INVALID_ARG), (dict(weight_dtype=7), cn.ERR_INVALID_ARG),
    (dict(mod_dtype=9), cn.ERR_INVALID_ARG), (dict(eps=-1e-6), cn.ERR_INVALID_ARG), (dict(eps=float("nan")), cn.ERR_INVALID_ARG),
    (dict(eps=float("inf")), cn.ERR_INVALID_ARG), (dict(scale_stride=-1), cn.ERR_INVALID_ARG),
    (dict(x_stride=(2, 132)), cn.ERR_INVALID_ARG), (dict(x_stride=(0, -8)), cn.ERR_INVALID_ARG), (dict(x_stride=(0, 1 << 39)), cn.ERR_INVALID_ARG),
]


@pytest.mark.parametrize("kw,status", NORM_BAD)
def test_norm_refuses_bad_records(kw, status):
    s = norm_shape(**kw)
    expect(lambda: call_norm(s), status)
    expect(lambda: call_norm_backward(s), status)


def test_norm_refuses_bad_pointers_and_overlapping_outputs():
    for kw in (dict(X=None), dict(Y=None), dict(X=P + 2), dict(Y=P + 8), dict(mean=None), dict(rstd=None), dict(weight=P + 2 * 0 + 1)):
        expect(lambda **k: call_norm(norm_shape(), **k), cn.ERR_INVALID_ARG, **kw)
    for st in ((2, 64), (2, 0), (1, 128), (0, 40 * 128)):           # rows of Y that share channels, heads or entries that share rows
        expect(lambda: call_norm(norm_shape(y_stride=st)), cn.ERR_INVALID_ARG)
        expect(lambda: call_norm_backward(norm_shape(dx_stride=st)), cn.ERR_INVALID_ARG)
    for kw in (dict(dY=None), dict(X=None), dict(mean=None), dict(dX=None), dict(dX=P + 4), dict(dw=P + 2)):
        expect(lambda **k: call_norm_backward(norm_shape(), **k), cn.ERR_INVALID_ARG, **kw)
    for kw in (dict(ws=None), dict(ws=P + 64), dict(ws_bytes=100)):
        expect(lambda **k: call_norm_backward(norm_shape(), **k), cn.ERR_WORKSPACE, **kw)


LINEAR_BAD = [
    (dict(B=0), cn.ERR_INVALID_ARG), (dict(N=-3), cn.ERR_INVALID_ARG), (dict(in_features=0), cn.ERR_INVALID_ARG), (dict(out_features=0), cn.ERR_INVALID_ARG),
    (dict(activation=4), cn.ERR_INVALID_ARG), (dict(activation=-1), cn.ERR_INVALID_ARG), (dict(y_dtype=2), cn.ERR_INVALID_ARG),
    (dict(bias_dtype=3), cn.ERR_INVALID_ARG), (dict(gate_dtype=3), cn.ERR_INVALID_ARG), (dict(gate_stride=-8), cn.ERR_INVALID_ARG),
    (dict(B=1 << 15, N=1 << 16), cn.ERR_UNSUPPORTED), (dict(B=70000, N=1), cn.ERR_UNSUPPORTED), (dict(N=1 << 27), cn.ERR_UNSUPPORTED),
    (dict(in_features=(1 << 27) + 1), cn.ERR_UNSUPPORTED), (dict(out_features=(1 << 27) + 1), cn.ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("kw,status", LINEAR_BAD)
def test_linear_refuses_bad_records(kw, status):
    s = linear_shape(**kw)
    expect(lambda: call_linear(s), status)
    expect(lambda: call_linear_backward(s), status)
    assert cn.linear_workspace_bytes(s) == 0 and cn.linear_backward_workspace_bytes(s) == 0


def test_linear_refuses_bad_strides_and_pointers():
    for kw in (dict(x_stride=(1, 132)), dict(x_stride=(1, 64)), dict(x_stride=(0, 0)), dict(w_stride=124), dict(w_stride=64), dict(y_stride=(1, 0)),
               dict(y_stride=(0, 64)), dict(y_stride=(1, 60)), dict(residual_stride=(1, 32)), dict(z_stride=(0, 64))):
        expect(lambda: call_linear(linear_shape(**kw)), cn.ERR_INVALID_ARG)
    for kw in (dict(X=None), dict(W=None), dict(Y=None), dict(X=P + 8), dict(W=P + 2), dict(Y=P + 8), dict(Z=P + 4), dict(residual=P + 8),
               dict(bias=P + 1), dict(gate=P + 2)):
        s = linear_shape()
        expect(lambda **k: call_linear(s, **k), cn.ERR_INVALID_ARG, **kw)
    for kw in (dict(ws=None), dict(ws=P + 128), dict(ws_bytes=255)):
        expect(lambda **k: call_linear(linear_shape(), **k), cn.ERR_WORKSPACE, **kw)
    for kw in (dict(dY=None), dict(dY=P + 8), dict(X=None), dict(W=None), dict(dX=P + 8), dict(dW=P + 2), dict(gate=None), dict(db=P + 2)):
        expect(lambda **k: call_linear_backward(linear_shape(), **k), cn.ERR_INVALID_ARG, **kw)
    s = linear_shape(activation=cn.ACT_SILU)
    expect(lambda: call_linear_backward(s, Z=None, dg=None), cn.ERR_INVALID_ARG)       # the slope of the activation wants z
    expect(lambda: call_linear_backward(linear_shape(), Z=None), cn.ERR_INVALID_ARG)   # so does the gate's gradient
    for kw in (dict(dx_stride=(1, 64)), dict(dx_stride=(0, 128)), dict(dw_stride=64), dict(x_stride=(0, 0))):
        expect(lambda: call_linear_backward(linear_shape(**kw)), cn.ERR_INVALID_ARG)
    need = cn.linear_backward_workspace_bytes(linear_shape())
    assert need >= 256 + 2 * 40 * 64 * 2
    expect(lambda: call_linear_backward(linear_shape(), ws_bytes=need - 1), cn.ERR_WORKSPACE)


def test_calls_without_a_gpu_fail_loudly():
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for st in (call_norm(norm_shape()), call_norm_backward(norm_shape()), call_linear(linear_shape()), call_linear_backward(linear_shape())):
        assert st in (cn.ERR_UNSUPPORTED, cn.ERR_CUDA)


def test_python_calls_check_tensors_against_the_record():
    bf = torch.bfloat16
    x, w, y = torch.empty((1, 6, 64), dtype=bf), torch.empty((32, 64), dtype=bf), torch.empty((1, 6, 32), dtype=bf)
    s = cn.make_linear_shape(x, w, y)
    bad = [
        lambda: cn.linear(x.float(), w, s, Y=y), lambda: cn.linear(x, w, s, Y=y.float()), lambda: cn.linear(x[:, :5], w, s, Y=y),
        lambda: cn.linear(x, w[:16], s, Y=y), lambda: cn.linear(torch.empty((1, 6, 128), dtype=bf)[..., :64], w, s, Y=y),
        lambda: cn.linear(x, w, s, Y=y, bias=torch.empty(32, dtype=bf)),             # the record has fp32 biases unless it was given one
        lambda: cn.linear(x, w, s, Y=y, bias=torch.empty(31)), lambda: cn.linear(x, w, s, Y=y, gate=torch.empty((2, 32))),
        lambda: cn.linear(x, w, s, Y=y, bias=torch.empty(64)[::2]), lambda: cn.linear(x.half(), w, s, Y=y),
        lambda: cn.make_linear_shape(x, w[:, :32], y), lambda: cn.make_linear_shape(x, w, x), lambda: cn.make_linear_shape(x[0], w, y),
        lambda: cn.make_linear_shape(x.mT.contiguous().mT, w, y),
    ]
    t = torch.empty((1, 1, 6, 64), dtype=bf)
    ns = cn.make_norm_shape(t, t)
    st = torch.empty((1, 1, 6))
    bad += [
        lambda: cn.layer_norm(t.float(), ns, Y=t), lambda: cn.layer_norm(t, ns, Y=t, weight=torch.empty(63)), lambda: cn.layer_norm(t[:, :, :5], ns, Y=t),
        lambda: cn.layer_norm(t, ns, Y=t, scale=torch.empty((2, 64))), lambda: cn.layer_norm(t, ns, Y=t, mean=st.double(), rstd=st),
        lambda: cn.layer_norm_backward(t, t, st, st[:, :, :5], ns), lambda: cn.make_norm_shape(t[0], t[0]), lambda: cn.make_norm_shape(t.double(), t),
    ]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    if not torch.cuda.is_available():
        with pytest.raises(cn.CarnatorError):
            cn.linear(x, w, s, Y=y)
        with pytest.raises(cn.CarnatorError):
            cn.layer_norm(t, ns)


# ---- records: copied, shared, used again -----------------------------------------------------------------
DEVICE = "cuda" if torch.cuda.is_available() else "cpu"


class Library:
    """In the place of the library: keeps the record that each call was given and launches nothing."""

    def __init__(self):
        self.records = []

    def __getattr__(self, name):
        def call(*args):
            record = next(a._obj for a in args if hasattr(a, "_obj"))
            self.records.append(type(record).from_buffer_copy(record))
            return 256 if name.endswith("_workspace_bytes") else cn.OK
        return call


@pytest.fixture
def library(monkeypatch):
    fake = Library()
    monkeypatch.setattr(cn, "lib", lambda: fake)
    return fake


def norm_call(s=None, packed=False):
    x, y = (torch.empty((1, 2, 4, 72), dtype=torch.bfloat16, device=DEVICE) for _ in range(2))
    s = s or cn.make_norm_shape(x, y)
    return s, lambda r=s: cn.layer_norm(x, r, Y=None if packed else y)


def norm_backward_call(packed=False):
    x, y = (torch.empty((1, 2, 4, 72), dtype=torch.bfloat16, device=DEVICE) for _ in range(2))
    stat = torch.empty((1, 2, 4), device=DEVICE)
    s = cn.make_norm_shape(x, y)
    return s, lambda r=s: cn.layer_norm_backward(y, x, stat, stat, r, dX=None if packed else torch.empty_like(x))


def linear_call(packed=False):
    x, w, y = (torch.empty(n, dtype=torch.bfloat16, device=DEVICE) for n in ((1, 4, 64), (40, 64), (1, 4, 40)))
    s = cn.make_linear_shape(x, w, y, activation=cn.ACT_GELU)
    return s, lambda r=s: cn.linear(x, w, r, Y=None if packed else y)


def linear_backward_call(packed=False):
    x, w, y = (torch.empty(n, dtype=torch.bfloat16, device=DEVICE) for n in ((1, 4, 64), (40, 64), (1, 4, 40)))
    s = cn.make_linear_shape(x, w, y, Z=y, dX=x, dW=w, activation=cn.ACT_GELU)
    return s, lambda r=s: cn.linear_backward(y, x, w, r, Z=y, dX=torch.empty_like(x), dW=torch.empty_like(w))


CALLS = [norm_call, norm_backward_call, linear_call, linear_backward_call]


@pytest.mark.parametrize("make", CALLS)
@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda s: pickle.loads(pickle.dumps(s))], ids=["copy", "deepcopy", "pickle"])
def test_a_copied_record_stands_for_itself(library, make, how):
    """A copy of a record that has been used: its calls pass what it says, whatever becomes of the original."""
    s, call = make()
    call()
    t = how(s)
    said = bytes(t)
    s.N = 4000
    if hasattr(s, "activation"):
        s.activation = cn.ACT_SILU
    s.x_stride[1] = 1 << 30
    call(t)
    assert bytes(t) == said and bytes(library.records[-1]) == said
    with pytest.raises(ValueError):
        call(s)


@pytest.mark.parametrize("make", CALLS)
def test_calls_leave_the_record_as_it_is(library, make):
    s, call = make(packed=True)
    for name in ("y_stride", "dx_stride"):          # of a tensor that the call does not get: its own output has strides of its own
        if make in (norm_backward_call, linear_backward_call) and name == "y_stride":
            continue
        getattr(s, name)[0], getattr(s, name)[1] = 7777, 88
    if make is linear_backward_call:                # has no output of its own
        s.dx_stride[:] = [4 * 64, 64]
    before = bytes(s)
    call()
    assert bytes(s) == before
    passed = library.records[-1]
    if make is norm_call:
        assert list(passed.y_stride) == [2 * 4 * 72, 4 * 72, 72]
    if make is norm_backward_call:
        assert list(passed.dx_stride) == [2 * 4 * 72, 4 * 72, 72]
    if make is linear_call:
        assert list(passed.y_stride) == [4 * 40, 40]


@pytest.mark.parametrize("make", [norm_call, linear_call])
@pytest.mark.parametrize("packed", [False, True])
def test_threads_share_a_record(library, make, packed):
    """Four threads whose first call with a new record is the same moment."""
    errors, interval = [], sys.getswitchinterval()
    sys.setswitchinterval(1e-6)

    def work(call, gate):
        gate.wait()
        try:
            for _ in range(3):
                call()
        except Exception as e:  # noqa: BLE001
            errors.append(e)
    try:
        for i in range(200):
            s, call = make(packed=packed)
            if make is linear_call:
                s.gate_stride = 8 * i          # a record that nothing has seen
            else:
                s.eps = 1e-6 * (i + 1)
            gate = threading.Barrier(4)
            threads = [threading.Thread(target=work, args=(call, gate)) for _ in range(4)]
            for t in threads:
                t.start()
            for t in threads:
                t.join()
    finally:
        sys.setswitchinterval(interval)
    assert not errors, errors[:3]


# ---- where the tensors are --------------------------------------------------------------------------------
def test_tensors_in_host_memory_are_refused_where_there_is_a_gpu(library, monkeypatch):
    """The kernels would be given addresses of the host.  (A machine without a GPU checks arguments and launches nothing.)"""
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x, w, y = (torch.empty(n, dtype=torch.bfloat16) for n in ((1, 4, 64), (64, 64), (1, 4, 64)))
    t, stat = x[:, None], torch.empty((1, 1, 4))
    ns, ls = cn.make_norm_shape(t, t), cn.make_linear_shape(x, w, y, dX=x, dW=w)
    for call in (lambda **k: cn.layer_norm(t, ns, Y=t, **k), lambda **k: cn.layer_norm_backward(t, t, stat, stat, ns, dX=t, **k),
                 lambda **k: cn.linear(x, w, ls, Y=y, **k), lambda **k: cn.linear_backward(y, x, w, ls, dX=x, dW=w, **k)):
        for stream in (None, types.SimpleNamespace(cuda_stream=0)):
            with pytest.raises(ValueError, match="cpu"):
                call(stream=stream)
    assert not library.records


def test_workspaces_are_where_the_tensors_are(library):
    x, w, y = (torch.empty(n, dtype=torch.bfloat16, device=DEVICE) for n in ((1, 4, 64), (64, 64), (1, 4, 64)))
    t, stat = x[:, None], torch.empty((1, 1, 4), device=DEVICE)
    ns, ls = cn.make_norm_shape(t, t), cn.make_linear_shape(x, w, y, dX=x, dW=w)
    for ws in (torch.empty(1 << 16, dtype=torch.uint8, device="meta"), torch.empty(1, dtype=torch.uint8, device=DEVICE).expand(1 << 16),
               torch.empty(1 << 16, dtype=torch.uint8, device=DEVICE)[::2]):
        for call in (lambda: cn.layer_norm_backward(t, t, stat, stat, ns, dX=t, ws=ws), lambda: cn.linear(x, w, ls, Y=y, ws=ws),
                     lambda: cn.linear_backward(y, x, w, ls, dX=x, dW=w, ws=ws)):
            with pytest.raises(ValueError, match="ws"):
                call()
    assert not library.records


# ---- as wide as the C calls ---------------------------------------------------------------------------------
def test_a_norm_may_have_a_bias_only(library):
    x = torch.empty((1, 1, 4, 64), dtype=torch.bfloat16, device=DEVICE)
    stat = torch.empty((1, 1, 4), device=DEVICE)
    for dtype, code in ((torch.bfloat16, cn.DTYPE_BF16), (torch.float32, cn.DTYPE_F32)):
        bias = torch.empty(64, dtype=dtype, device=DEVICE)
        s = cn.make_norm_shape(x, x, bias=bias)
        assert s.weight_dtype == code
        cn.layer_norm(x, s, bias=bias, Y=x)
        g = cn.layer_norm_backward(x, x, stat, stat, s, bias=bias)
        assert g.dbias.shape == (64,) and g.dweight is None
        assert cn.layer_norm_backward(x, x, stat, stat, s, bias=bias, want=()).dbias is None
    assert cn.make_norm_shape(x, x, torch.empty(64, dtype=torch.bfloat16, device=DEVICE)).weight_dtype == cn.DTYPE_BF16


def test_gradients_want_only_what_they_read(library):
    x, w, y = (torch.empty(n, dtype=torch.bfloat16, device=DEVICE) for n in ((1, 4, 64), (40, 64), (1, 4, 40)))
    s = cn.make_linear_shape(x, w, y, Z=y, dX=x, dW=w)
    cn.linear_backward(y, None, w, s, Z=y, dX=x)
    cn.linear_backward(y, x, None, s, Z=y, dW=w)
    cn.linear_backward(y, None, None, s, Z=y)
    calls = len(library.records)
    for bad in (lambda: cn.linear_backward(y, None, w, s, Z=y, dW=w), lambda: cn.linear_backward(y, x, None, s, Z=y, dX=x)):
        with pytest.raises(ValueError):
            bad()
    assert len(library.records) == calls
