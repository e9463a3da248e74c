"""include/aspis_optim.h without a GPU: every declared entry point is exported, lists
are made and refused, and the device calls refuse bad arguments before anything
is enqueued.  Addresses are fake and never read."""
import ctypes
import os
import re

import pytest

from conftest import ROOT

ap = pytest.importorskip("paper_2108_02416_gb300")
P, f32 = ctypes.c_void_p, ctypes.c_float
AT = 1 << 30                       # a fake device address, 16-byte aligned


def tensors(*rows):
    items = (ap._Tensor * max(1, len(rows)))()
    for item, row in zip(items, rows):
        item.data, item.numel, item.type = row[:3]
        item.out, item.out_type = row[3:] if len(row) > 3 else (None, 0)
    return items


def make(*rows, n=None):
    h = P()
    st = ap.lib.aspis_tensors_create(tensors(*rows), len(rows) if n is None else n, ctypes.byref(h))
    return st, h


def param(**k):
    x = ap._Param(param=AT, master=None, grad=AT + 0x10000, exp_avg=AT + 0x20000, exp_avg_sq=AT + 0x30000, numel=100,
                  param_type=ap.F32, grad_type=ap.F32, weight_decay=0.1, reserved=0)
    for name, value in k.items():
        setattr(x, name, value)
    return x


def make_params(*items):
    h = P()
    a = (ap._Param * max(1, len(items)))(*items)
    return ap.lib.aspis_params_create(a, len(items), ctypes.byref(h)), h


def args(**k):
    x = ap._AdamwArgs(1e-3, 0.9, 0.999, 1e-8, 1, 1.0, 1.0, 0, 0)
    for name, value in k.items():
        setattr(x, name, value)
    return x


def test_every_declared_call_is_exported():
    src = open(os.path.join(ROOT, "include", "aspis_optim.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    names = set(re.findall(r"\b(aspis_[a-z_]+)\s*\(", src))
    assert names == {"aspis_tensors_create", "aspis_tensors_destroy", "aspis_params_create", "aspis_params_destroy",
                     "aspis_grad_norm", "aspis_clip_grads", "aspis_adamw"}
    lib = ctypes.CDLL(ap.LIB_PATH)
    assert all(hasattr(lib, n) for n in names)
    assert f"ASPIS_NORM_WORKSPACE_BYTES {ap.NORM_WORKSPACE_BYTES}\n" in src


def test_struct_sizes():
    assert ctypes.sizeof(ap._Tensor) == 32
    assert ctypes.sizeof(ap._Param) == 64
    assert ctypes.sizeof(ap._AdamwArgs) == 56


@pytest.mark.parametrize("row,code", [
    ((AT, 5, ap.F32), ap.OK),
    ((AT + 4, 5, ap.F32), ap.OK),
    ((AT + 2, 5, ap.BF16), ap.OK),
    ((None, 0, ap.F16), ap.OK),                          # empty: no address needed
    ((AT, 5, ap.F32, AT + 64, ap.BF16), ap.OK),
    ((None, 5, ap.F32), ap.E_INVAL),
    ((AT, -1, ap.F32), ap.E_INVAL),
    ((AT, 5, 3), ap.E_INVAL),
    ((AT, 5, -1), ap.E_INVAL),
    ((AT, 5, ap.F32, AT + 64, 7), ap.E_INVAL),
    ((AT + 2, 5, ap.F32), ap.E_ALIGN),
    ((AT + 1, 5, ap.F16), ap.E_ALIGN),
    ((AT, 5, ap.F32, AT + 63, ap.BF16), ap.E_ALIGN),
    ((AT, (1 << 40) + 1, ap.F32), ap.E_RANGE),
    ((AT, (1 << 38) + 1, ap.BF16), ap.E_RANGE),
])
def test_tensor_lists(row, code):
    st, h = make(row)
    assert st == code and bool(h) == (code == ap.OK)
    ap.lib.aspis_tensors_destroy(h)


def test_list_counts_and_pointers():
    assert make(n=0)[0] == ap.OK
    assert make((AT, 1, ap.F32), n=-1)[0] == ap.E_INVAL
    assert make((AT, 1, ap.F32), n=1 << 25)[0] == ap.E_RANGE      # refused before the array is read
    h = P()
    assert ap.lib.aspis_tensors_create(None, 1, ctypes.byref(h)) == ap.E_INVAL
    assert ap.lib.aspis_tensors_create(None, 0, ctypes.byref(h)) == ap.OK
    ap.lib.aspis_tensors_destroy(h)
    assert ap.lib.aspis_tensors_create(tensors((AT, 1, ap.F32)), 1, None) == ap.E_INVAL
    ap.lib.aspis_tensors_destroy(None)
    ap.lib.aspis_params_destroy(None)


@pytest.mark.parametrize("n", [1, 119, 120, 121, 499, 500, 501, 1000, 1001, 2500])
def test_lists_of_many_tensors(n):
    st, h = make(*[(AT + 64 * i, i % 17, ap.F32) for i in range(n)])
    assert st == ap.OK
    ap.lib.aspis_tensors_destroy(h)
    st, h = make_params(*[param(param=AT + 64 * i, grad=AT + (1 << 20) + 64 * i, exp_avg=AT + (2 << 20) + 64 * i,
                                exp_avg_sq=AT + (3 << 20) + 64 * i, numel=i % 17) for i in range(n)])
    assert st == ap.OK
    ap.lib.aspis_params_destroy(h)


@pytest.mark.parametrize("rows,clip", [
    ([(AT, 16, ap.F32), (AT + 64, 16, ap.F32)], True),                    # neighbours
    ([(AT, 16, ap.F32), (AT + 60, 16, ap.F32)], False),                   # the last value twice
    ([(AT, 16, ap.F32), (AT, 16, ap.F32)], False),                        # the same tensor twice
    ([(AT + 4096, 4, ap.F32), (AT, 2000, ap.F32)], False),                # one inside another
    ([(AT, 16, ap.F32), (AT, 0, ap.F32)], True),                          # an empty one anywhere
    ([(AT, 16, ap.F32, AT + 4096, ap.F32), (AT, 16, ap.F32, AT + 8192, ap.F32)], True),   # read twice
    ([(AT, 16, ap.F32, AT + 4096, ap.F32), (AT + 64, 16, ap.F32, AT + 4100, ap.F32)], False),
    ([(AT, 16, ap.F32, AT + 32, ap.F32)], False),                         # output over its own input
    ([(AT, 16, ap.F32, AT, ap.F32)], True),                               # ... exactly: in place
    ([(AT, 16, ap.F32, AT, ap.BF16)], False),                             # ... of another type
    ([(AT, 16, ap.F32, AT + 4096, ap.F32), (AT + 4096, 16, ap.F32, AT + 8192, ap.F32)], False),
])
def test_overlaps_are_refused_by_clipping_alone(rows, clip):
    st, h = make(*rows)
    assert st == ap.OK                                   # the norm may be taken
    # E_ALIGN of the norm's address comes only after the other checks: nothing is enqueued either way
    got = ap.lib.aspis_clip_grads(h, 1.0, 1.0, P(AT + 2), P(AT), None)
    assert got == (ap.E_ALIGN if clip else ap.E_INVAL)
    ap.lib.aspis_tensors_destroy(h)


@pytest.mark.parametrize("change,code", [
    ({}, ap.OK),
    ({"numel": 0, "param": None, "grad": None, "exp_avg": None, "exp_avg_sq": None}, ap.OK),
    ({"param_type": ap.BF16, "master": AT + 0x40000}, ap.OK),
    ({"param_type": ap.F16}, ap.OK),
    ({"grad_type": ap.BF16, "grad": AT + 0x10002}, ap.OK),
    ({"param": None}, ap.E_INVAL),
    ({"grad": None}, ap.E_INVAL),
    ({"exp_avg": None}, ap.E_INVAL),
    ({"exp_avg_sq": None}, ap.E_INVAL),
    ({"master": AT + 0x40000}, ap.E_INVAL),              # fp32 parameters take no master
    ({"numel": -5}, ap.E_INVAL),
    ({"param_type": 9}, ap.E_INVAL),
    ({"grad_type": 3}, ap.E_INVAL),
    ({"weight_decay": -0.1}, ap.E_INVAL),
    ({"weight_decay": float("nan")}, ap.E_INVAL),
    ({"weight_decay": float("inf")}, ap.E_INVAL),
    ({"reserved": 1}, ap.E_INVAL),
    ({"grad": AT + 0x10002}, ap.E_ALIGN),
    ({"exp_avg": AT + 0x20001}, ap.E_ALIGN),
    ({"param_type": ap.BF16, "master": AT + 0x40002}, ap.E_ALIGN),
    ({"grad": AT}, ap.E_INVAL),                          # overlaps
    ({"grad": AT + 396}, ap.E_INVAL),
    ({"exp_avg_sq": AT + 0x20000}, ap.E_INVAL),
    ({"exp_avg": AT - 4}, ap.E_INVAL),
    ({"numel": (1 << 40) + 1}, ap.E_RANGE),
])
def test_param_lists(change, code):
    st, h = make_params(param(**change))
    assert st == code and bool(h) == (code == ap.OK)
    ap.lib.aspis_params_destroy(h)


def test_params_may_share_a_gradient_and_nothing_else():
    far = dict(param=AT + 0x100000, exp_avg=AT + 0x120000, exp_avg_sq=AT + 0x130000)
    st, h = make_params(param(), param(**far))
    assert st == ap.OK
    ap.lib.aspis_params_destroy(h)
    for name in far:                                     # tied parameters or moments
        st, h = make_params(param(), param(**{k: v for k, v in far.items() if k != name}))
        assert st == ap.E_INVAL and not h


def test_norm_and_clip_refuse():
    st, h = make((AT, 5, ap.F32))
    norm, clip, work = ap.lib.aspis_grad_norm, ap.lib.aspis_clip_grads, P(AT)
    bad = [0.0, -1.0, float("nan"), float("inf")]
    assert norm(None, 1.0, P(AT), None, work, None) == ap.E_INVAL
    assert norm(h, 1.0, None, None, work, None) == ap.E_INVAL
    assert norm(h, 1.0, P(AT), None, None, None) == ap.E_INVAL
    assert norm(h, 1.0, P(AT + 2), None, work, None) == ap.E_ALIGN
    assert norm(h, 1.0, P(AT), P(AT + 3), work, None) == ap.E_ALIGN
    assert norm(h, 1.0, P(AT), None, P(AT + 8), None) == ap.E_ALIGN
    for s in bad:
        assert norm(h, s, P(AT), None, work, None) == ap.E_INVAL
        assert clip(h, 1.0, s, P(AT), work, None) == ap.E_INVAL
    assert clip(None, 1.0, 1.0, P(AT), work, None) == ap.E_INVAL
    assert clip(h, 1.0, 1.0, None, work, None) == ap.E_INVAL
    assert clip(h, -1.0, 1.0, P(AT), work, None) == ap.E_INVAL
    assert clip(h, float("nan"), 1.0, P(AT), work, None) == ap.E_INVAL
    assert clip(h, 1.0, 1.0, P(AT), P(AT + 8), None) == ap.E_ALIGN
    ap.lib.aspis_tensors_destroy(h)


@pytest.mark.parametrize("change", [
    {"lr": float("nan")}, {"lr": float("inf")}, {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": 1.0}, {"beta2": float("nan")},
    {"eps": -1e-8}, {"eps": float("inf")}, {"eps": float("nan")}, {"step": 0}, {"step": -3}, {"max_norm": float("nan")},
    {"scale": 0.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"reserved": 1}])
def test_adamw_refuses(change):
    st, h = make_params(param())
    assert ap.lib.aspis_adamw(h, ctypes.byref(args(**change)), P(AT), P(AT), None) == ap.E_INVAL
    ap.lib.aspis_params_destroy(h)


def test_adamw_refuses_pointers():
    st, h = make_params(param())
    call = ap.lib.aspis_adamw
    a, plain, skip = args(), args(max_norm=-1.0), args(max_norm=-1.0, skip_nonfinite=1)
    assert call(None, ctypes.byref(a), P(AT), P(AT), None) == ap.E_INVAL
    assert call(h, None, P(AT), P(AT), None) == ap.E_INVAL
    assert call(h, ctypes.byref(a), None, P(AT), None) == ap.E_INVAL
    assert call(h, ctypes.byref(a), P(AT + 2), P(AT), None) == ap.E_ALIGN
    assert call(h, ctypes.byref(a), P(AT), P(AT + 8), None) == ap.E_ALIGN
    assert call(h, ctypes.byref(plain), None, P(AT), None) == ap.E_INVAL
    assert call(h, ctypes.byref(skip), None, None, None) == ap.E_INVAL
    ap.lib.aspis_params_destroy(h)


def test_python_refuses_host_tensors():
    torch = pytest.importorskip("torch")
    x = [torch.zeros(4) for _ in range(4)]
    with pytest.raises(ValueError):
        ap.TensorList(x[:1])
    with pytest.raises(ValueError):
        ap.ParamList(x[:1], x[1:2], x[2:3], x[3:])
    with pytest.raises(ValueError):
        ap.TensorList([], out=x)
    with pytest.raises(ValueError):
        ap.ParamList([], [], [], [], weight_decay=[0.1])
    with pytest.raises(ValueError):
        ap.aspis_adamw(ap.ParamList([], [], [], []), 1, 1e-3, max_norm=-1.0)
