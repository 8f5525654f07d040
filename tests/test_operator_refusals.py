"""What the gated linear, the rotary positions and the AdamW step refuse before anything is launched: needs no GPU."""
import ctypes

import pytest
import torch

import paper_2202_13808_b200 as dropit
from paper_2202_13808_b200 import _lib, build as build_mod

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
NULL, A, ODD = ctypes.c_void_p(0), ctypes.c_void_p(1 << 20), ctypes.c_void_p((1 << 20) + 8)


@pytest.fixture(scope="module")
def lib():
    build_mod.build()
    return _lib.load()


def test_gated_linear(lib):
    def forward(x=A, w=A, b=A, M=4, C=16, H=8, dtype=0, gate=0, h=A, gu=A):
        return lib.dropit_gated_linear(x, w, b, M, C, H, dtype, gate, h, gu, NULL, NULL)
    assert forward(M=0, x=NULL, h=NULL) == OK
    for bad in (dict(x=NULL), dict(w=NULL), dict(h=NULL), dict(x=ODD), dict(w=ODD), dict(b=ODD), dict(h=ODD), dict(gu=ODD), dict(M=-1), dict(C=0),
                dict(H=0), dict(dtype=2), dict(dtype=-1), dict(gate=3), dict(gate=-1), dict(M=2 ** 31), dict(M=2 ** 27, C=16),
                dict(H=2 ** 30), dict(H=2 ** 26, C=16), dict(C=2 ** 62, H=2 ** 62, M=2 ** 62)):
        assert forward(**bad) == INVALID, bad
    size = ctypes.c_size_t(7)
    assert lib.dropit_gated_linear_backward_workspace(-1, 8, 0, ctypes.byref(size)) == INVALID
    assert lib.dropit_gated_linear_backward_workspace(4, 0, 0, ctypes.byref(size)) == INVALID
    assert lib.dropit_gated_linear_backward_workspace(4, 8, 0, None) == INVALID

    def backward(dh=A, gu=A, M=4, H=8, dtype=0, gate=0, dgu=A, db=NULL, ws=NULL, bytes_=0):
        return lib.dropit_gated_linear_backward(dh, gu, M, H, dtype, gate, dgu, db, ws, bytes_, NULL)
    assert backward(M=0, dh=NULL) == OK
    for bad in (dict(dh=NULL), dict(gu=ODD), dict(dgu=NULL), dict(db=ODD), dict(M=-1), dict(H=0), dict(gate=9), dict(dtype=5), dict(db=A), dict(db=A, ws=ODD),
                dict(M=2 ** 28)):
        assert backward(**bad) == INVALID, bad
    assert backward(db=A, ws=A, bytes_=8) == WORKSPACE

    def input_grad(d=A, w=A, M=4, C=16, H=8, dtype=0, dx=A):
        return lib.dropit_gated_input_grad(d, w, M, C, H, dtype, dx, NULL, NULL)
    assert input_grad(M=0, d=NULL) == OK
    for bad in (dict(d=NULL), dict(w=ODD), dict(dx=NULL), dict(M=-1), dict(C=0), dict(H=0), dict(dtype=3)):
        assert input_grad(**bad) == INVALID, bad


class _Plan(ctypes.Structure):
    _fields_ = [("head_dim", ctypes.c_int32), ("pairs", ctypes.c_int32), ("axes", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("turns", ctypes.c_uint64 * 256), ("axis", ctypes.c_uint8 * 256)]


class _Rotated(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("strides", ctypes.c_int64 * 6), ("heads", ctypes.c_int32)]


def _plan(lib, head_dim, sections, theta=100.0, shared=0, interleaved=0):
    plan = _Plan()
    code = lib.dropit_rotary_make_plan(head_dim, (ctypes.c_int * max(len(sections), 1))(*sections), len(sections), theta, shared, interleaved,
                                       ctypes.byref(plan))
    return code, plan


def test_rotary_plans(lib):
    code, plan = _plan(lib, 40, (16, 0, 8))
    assert code == OK and (plan.head_dim, plan.pairs, plan.axes) == (40, 12, 3)
    assert list(plan.axis[:12]) == [0] * 8 + [2] * 4
    # turns per position: theta^-e / 2 pi; the first pair of each axis makes one radian a step
    for j, e in ((0, 0.0), (1, 2 / 16), (8, 0.0), (11, 6 / 8)):
        assert abs(plan.turns[j] / 2 ** 64 - 100.0 ** -e / (2 * 3.141592653589793)) < 2.0 ** -50
    _, ladder = _plan(lib, 40, (16, 0, 8), shared=1)
    assert abs(ladder.turns[11] / 2 ** 64 - 100.0 ** -(22 / 24) / (2 * 3.141592653589793)) < 2.0 ** -50
    for bad in ((1, (2,)), (16, (3,)), (16, (18,)), (16, (0,)), (16, ()), (16, (-2, 8)), (16, (2,) * 9), (16, (8,), 0.5), (16, (8,), float("nan")),
                (16, (8,), float("inf"))):
        assert _plan(lib, *bad)[0] == INVALID, bad
    assert _plan(lib, 1024, (514,))[0] == UNSUPPORTED
    for bad in (dict(head_dim=16, sections=(6, 3)), dict(head_dim=16, sections=()), dict(head_dim=16, sections=(20,)), dict(head_dim=16, sections=(8,), theta=0)):
        with pytest.raises(ValueError):
            dropit.dropit_rotary_plan(**bad)
    with pytest.raises(dropit.DropITError):
        dropit.dropit_rotary_plan(1024, (514,))


def test_rotary(lib):
    _, plan = _plan(lib, 16, (8, 8))
    def call(plan=plan, batch=2, length=3, q=_Rotated(1 << 20, 1 << 20, heads=2), k=None, positions=A, kind=0, dtype=0):
        ref = lambda t: None if t is None else ctypes.byref(t)
        return lib.dropit_rotary(ref(plan), batch, length, ref(q), ref(k), positions, kind, 6, 2, 1, dtype, 0, NULL)
    assert call(batch=0) == OK and call(length=0) == OK and call(q=_Rotated(heads=0)) == OK
    broken = _Plan.from_buffer_copy(plan)
    broken.pairs = 300
    wide = _Plan.from_buffer_copy(plan)
    wide.pairs = 9
    for bad in (dict(plan=None), dict(q=None), dict(batch=-1), dict(length=-1), dict(length=2 ** 31), dict(positions=NULL), dict(positions=ctypes.c_void_p(6)),
                dict(positions=ctypes.c_void_p(12), kind=1), dict(kind=3), dict(dtype=2), dict(q=_Rotated(0, 1 << 20, heads=2)),
                dict(q=_Rotated(1 << 20, 1, heads=2)), dict(q=_Rotated(1 << 20, 1 << 20, heads=-1)), dict(k=_Rotated(2, 0, heads=1)), dict(plan=broken),
                dict(plan=wide), dict(q=_Rotated(2, 2, heads=2), dtype=1), dict(batch=2 ** 62, length=2 ** 30)):
        assert call(**bad) == INVALID, bad
    assert call(q=_Rotated(1 << 20, 1 << 20, heads=1 << 20)) == UNSUPPORTED


class _Tensor(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p), ("lr_device", ctypes.c_void_p), ("n", ctypes.c_int64), ("first_block", ctypes.c_int64),
                ("ordinal", ctypes.c_int32), ("lr", ctypes.c_float), ("weight_decay", ctypes.c_float)]


class _Options(ctypes.Structure):
    _fields_ = [("param_dtype", ctypes.c_int), ("grad_dtype", ctypes.c_int), ("state_bits", ctypes.c_int32), ("dither", ctypes.c_int32),
                ("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("seed", ctypes.c_uint32)]


class _State(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("m", "v", "m_scale", "v_scale", "master", "steps", "ticket", "grad_factor")]


def test_adamw(lib):
    at = 1 << 20

    def call(count=1, tensors=True, options=True, tensor=(at, at, None, 10, 0, 0, 1e-3, 0.0), state=None, **o):
        o = dict(dict(param_dtype=1, grad_dtype=1, state_bits=32, beta1=0.9, beta2=0.999, eps=1e-8), **o)
        s = dict(dict(m=at, v=at, steps=at, ticket=at), **(state or {}))
        return lib.dropit_adamw_step(ctypes.byref(_Tensor(*tensor)) if tensors else None, count, ctypes.byref(_Options(**o)) if options else None,
                                     ctypes.byref(_State(**s)), NULL)
    nothing = (None, None, None, 0, 0, 0, 1e-3, 0.0)
    assert call(count=0, tensors=False) == OK and call(tensor=nothing, state=dict(m=None)) == OK
    inf, nan = float("inf"), float("nan")
    for bad in (dict(count=-1), dict(tensors=False), dict(options=False), dict(param_dtype=2), dict(grad_dtype=-1), dict(state_bits=16), dict(beta1=1.0),
                dict(beta1=nan), dict(beta2=-0.1), dict(eps=-1.0), dict(eps=nan), dict(tensor=(None, at, None, 10, 0, 0, 1e-3, 0.0)),
                dict(tensor=(at, at + 2, None, 10, 0, 0, 1e-3, 0.0)), dict(tensor=(at, at, None, -1, 0, 0, 1e-3, 0.0)),
                dict(tensor=(at, at, None, 2 ** 31, 0, 0, 1e-3, 0.0)), dict(tensor=(at, at, None, 10, -1, 0, 1e-3, 0.0)),
                dict(tensor=(at, at, None, 10, 2 ** 40, 0, 1e-3, 0.0)), dict(tensor=(at, at, None, 10, 0, -1, 1e-3, 0.0)),
                dict(tensor=(at, at, None, 10, 0, 0, inf, 0.0)), dict(tensor=(at, at, None, 10, 0, 0, 1e-3, nan)),
                dict(state=dict(m=None)), dict(state=dict(v=at + 8)), dict(state=dict(steps=None)), dict(state=dict(ticket=None)),
                dict(state=dict(master=at)), dict(state_bits=8), dict(state_bits=8, state=dict(m_scale=at, v_scale=at + 2)),
                dict(param_dtype=0, state=dict(master=at + 4))):
        assert call(**bad) == INVALID, bad


def test_the_bindings_refuse_cpu_tensors(lib):
    x, w = torch.zeros(4, 16), torch.zeros(16, 16)
    with pytest.raises(ValueError):
        dropit.dropit_gated_linear(x, w)
    with pytest.raises(ValueError):
        dropit.dropit_gated_linear_backward(x, torch.zeros(4, 32))
    with pytest.raises(ValueError):
        dropit.dropit_gated_input_grad(x, w)
    with pytest.raises(ValueError):
        dropit.DropITGatedLinear(16, 8)(x)
    with pytest.raises(ValueError):
        dropit.DropITGatedLinear(16, 8, gate="tanh")
    with pytest.raises(ValueError):
        dropit.dropit_rotary(torch.zeros(1, 4, 2, 16), None, torch.zeros(4, 1, dtype=torch.int32), dropit.dropit_rotary_plan(16, (16,)))
    p = torch.nn.Parameter(torch.zeros(4))
    p.grad = torch.ones(4)
    with pytest.raises(ValueError):
        dropit.DropITAdamW([p]).step()
