"""CPU-only checks of the recurrence, the products grouped by expert and the gradient norm: structures, workspace sizes and refusals.  No
kernel is launched: every call here is refused, or has nothing to do."""
from __future__ import annotations

import ctypes as C
import os

import pytest
import torch

from paper_2302_12445_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EALIGN, ETOOBIG = 0, -1, -5, -6
SPACE = 1 << 20  # an aligned address that is never read: the calls here return before
BIG = 1 << 60


class Steps(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("step", C.c_int64)]


class Recurrence(C.Structure):
    _fields_ = [("batch", C.c_int32), ("width", C.c_int32), ("steps", C.c_int64), ("dtype", C.c_int32), ("reserved", C.c_int32),
                ("lens", C.c_void_p), ("x", Steps), ("gate", Steps), ("state", C.c_void_p), ("kept", C.c_void_p), ("h", Steps),
                ("last", C.c_void_p), ("dh", Steps), ("dlast", C.c_void_p), ("dx", Steps), ("dgate", Steps), ("dstate", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class Experts(C.Structure):
    _fields_ = [("rows", C.c_int64), ("experts", C.c_int32), ("outs", C.c_int32), ("ins", C.c_int32), ("dtype", C.c_int32),
                ("ends", C.c_void_p), ("x", C.c_void_p), ("x_stride", C.c_int64), ("weight", C.c_void_p), ("dy", C.c_void_p),
                ("dy_stride", C.c_int64), ("out", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class Grad(C.Structure):
    _fields_ = [("data", C.c_void_p), ("out", C.c_void_p), ("elements", C.c_int64), ("dtype", C.c_int32), ("out_dtype", C.c_int32)]


def recurrence(**change):
    r = Recurrence(batch=2, width=64, steps=300, dtype=1, workspace=SPACE, workspace_bytes=BIG, state=SPACE, kept=SPACE, last=SPACE, dlast=SPACE,
                   dstate=SPACE)
    for name in ("x", "gate", "h", "dh", "dx", "dgate"):
        setattr(r, name, Steps(SPACE, 300 * 64, 64))
    for name, value in change.items():
        setattr(r, name, Steps(*value) if isinstance(value, tuple) else value)
    return bytes(r)


def experts(**change):
    x = Experts(rows=20, experts=3, outs=24, ins=40, dtype=1, ends=SPACE, x=SPACE, x_stride=40, weight=SPACE, dy=SPACE, dy_stride=24, out=SPACE,
                workspace=SPACE, workspace_bytes=BIG)
    for name, value in change.items():
        setattr(x, name, value)
    return bytes(x)


def grads(*rows):
    return b"".join(bytes(Grad(*r)) for r in rows)


def test_structures_are_the_header_s():
    assert C.sizeof(Recurrence) == ops._RECURRENCE.size and C.sizeof(Experts) == ops._EXPERTS.size
    assert C.sizeof(Grad) == ops._grad_layout(1).size and C.sizeof(Grad) * 7 == ops._grad_layout(7).size
    r = Recurrence.from_buffer_copy(ops._RECURRENCE.pack(*range(1, ops._RECURRENCE_MEMBERS + 1)))
    assert (r.batch, r.width, r.steps, r.dtype, r.reserved, r.lens) == (1, 2, 3, 4, 5, 6)
    assert (r.x.data, r.x.batch, r.x.step, r.gate.data, r.state, r.kept, r.h.data, r.last) == (7, 8, 9, 10, 13, 14, 15, 18)
    assert (r.dh.data, r.dlast, r.dx.data, r.dgate.data, r.dstate, r.workspace, r.workspace_bytes) == (19, 22, 23, 26, 29, 30, 31)
    x = Experts.from_buffer_copy(ops._EXPERTS.pack(*range(1, ops._EXPERTS_MEMBERS + 1)))
    assert [getattr(x, n) for n, _ in Experts._fields_] == list(range(1, ops._EXPERTS_MEMBERS + 1))
    assert "#define DEAR_RECURRENCE_KEPT %d" % ops.KEPT in open(os.path.join(ROOT, "include", "dear_ops.h")).read()


BAD_RECURRENCE = [
    (dict(batch=-1), EINVAL), (dict(width=0), EINVAL), (dict(width=(1 << 24) + 1), EINVAL), (dict(steps=-1), EINVAL),
    (dict(steps=(1 << 30) + 1), EINVAL), (dict(dtype=2), EINVAL), (dict(reserved=1), EINVAL), (dict(x=(0, 19200, 64)), EINVAL),
    (dict(gate=(0, 19200, 64)), EINVAL), (dict(x=(SPACE, -1, 64)), EINVAL), (dict(gate=(SPACE, 19200, -64)), EINVAL),
    (dict(x=(SPACE + 1, 19200, 64)), EALIGN), (dict(x=(SPACE, 19200, 1 << 22)), ETOOBIG), (dict(lens=SPACE + 2), EALIGN),
    (dict(state=SPACE + 2), EALIGN), (dict(kept=SPACE + 1), EALIGN), (dict(last=SPACE + 3), EALIGN), (dict(dlast=SPACE + 2), EALIGN),
    (dict(dstate=SPACE + 2), EALIGN), (dict(workspace=0), EINVAL), (dict(workspace=SPACE + 128), EALIGN), (dict(workspace_bytes=2047), ETOOBIG),
    (dict(batch=1 << 28), ETOOBIG),
]


@pytest.mark.parametrize("change,status", BAD_RECURRENCE)
def test_recurrence_refusals(change, status):
    lib, packed = ops.load_library(), recurrence(**change)
    assert lib.dear_recurrence(packed, None) == status and lib.dear_recurrence_backward(packed, None) == status


def test_recurrence_refuses_outputs_without_places_of_their_own():
    lib = ops.load_library()
    for bad in ((SPACE, 0, 64), (SPACE, 19200, 0), (SPACE, 19200, 63), (SPACE, 19199, 64), (SPACE, 64, 64), (SPACE, 64, 127), (0, 19200, 64)):
        assert lib.dear_recurrence(recurrence(h=bad), None) == EINVAL, bad
        assert lib.dear_recurrence_backward(recurrence(dx=bad), None) == EINVAL, bad
        assert lib.dear_recurrence_backward(recurrence(dgate=bad), None) == EINVAL, bad
    assert lib.dear_recurrence_backward(recurrence(kept=0), None) == EINVAL
    assert lib.dear_recurrence_backward(recurrence(dh=(0, 19200, 64)), None) == EINVAL
    assert lib.dear_recurrence(None, None) == EINVAL and lib.dear_recurrence_backward(None, None) == EINVAL


def test_recurrence_of_nothing_launches_nothing():
    lib, nothing = ops.load_library(), bytes(Recurrence(batch=0, width=64, steps=300, dtype=1))
    assert lib.dear_recurrence(nothing, None) == OK and lib.dear_recurrence_backward(nothing, None) == OK
    same = bytes(Recurrence(batch=2, width=64, steps=0, dtype=1, state=SPACE, last=SPACE, dlast=SPACE, dstate=SPACE))
    assert lib.dear_recurrence(same, None) == OK and lib.dear_recurrence_backward(same, None) == OK


def test_recurrence_workspace():
    lib, n = ops.load_library(), C.c_int64(-1)
    f = lib.dear_recurrence_workspace
    assert f(recurrence(), C.byref(n)) == OK and n.value >= 2 * 2 * 64 * 8  # two tiles' maps of either sequence
    assert f(recurrence(steps=256), C.byref(n)) == OK and n.value == 0
    assert f(recurrence(batch=0), C.byref(n)) == OK and n.value == 0
    assert f(recurrence(batch=1 << 20), C.byref(n)) == OK and n.value >= (1 << 20) * 2 * 64 * 8
    assert f(recurrence(), None) == EINVAL and f(None, C.byref(n)) == EINVAL and f(recurrence(width=0), C.byref(n)) == EINVAL


@pytest.mark.parametrize("batch,width,steps", [
    (1 << 30, 1 << 20, 1 << 27), ((1 << 31) - 1, 1 << 24, 1 << 30), (1 << 24, 1 << 22, 1 << 30), (1 << 28, 1 << 22, 1 << 30), (1, 1 << 24, 1 << 23),
    ((1 << 31) - 1, 64, 1), (1 << 17, 1 << 12, 256), (1 << 30, (1 << 21) + 64, 1 << 27)])
def test_recurrence_refuses_sizes_whose_products_pass_64_bits(batch, width, steps):
    """Workgroups, and bytes of workspace, of more than a launch has threads, also where their number, or its bits below 2^64, would fit."""
    lib, n, step = ops.load_library(), C.c_int64(-1), min(width, (1 << 22) - 1)
    change = dict(batch=batch, width=width, steps=steps, workspace_bytes=(1 << 63) - 1)
    assert lib.dear_recurrence_workspace(recurrence(**change), C.byref(n)) == ETOOBIG and n.value == -1
    if width < 1 << 22:  # (outputs that are wider than steps lie apart have no places of their own)
        tensors = {name: (SPACE, steps * step, step) for name in ("x", "gate", "h", "dh", "dx", "dgate")}
        assert lib.dear_recurrence(recurrence(**change, **tensors), None) == ETOOBIG
        assert lib.dear_recurrence_backward(recurrence(**change, **tensors), None) == ETOOBIG


def test_recurrence_refuses_tensors_that_pass_64_bits():
    lib = ops.load_library()
    for batch, stride in ((3, 1 << 62), (2, (1 << 63) - 1), (5, 1 << 61), (1 << 20, 1 << 45)):
        far = (SPACE, stride, 64)
        for name in ("x", "gate", "h"):
            assert lib.dear_recurrence(recurrence(batch=batch, **{name: far}), None) == EINVAL, (name, batch, stride)
        for name in ("x", "gate", "dh", "dx", "dgate"):
            assert lib.dear_recurrence_backward(recurrence(batch=batch, **{name: far}), None) == EINVAL, (name, batch, stride)


BAD_EXPERTS = [
    (dict(rows=-1), EINVAL), (dict(rows=1 << 31), EINVAL), (dict(experts=0), EINVAL), (dict(experts=(1 << 16) + 1), EINVAL),
    (dict(outs=0), EINVAL), (dict(ins=0), EINVAL), (dict(outs=(1 << 20) + 1), EINVAL), (dict(ins=(1 << 20) + 1), EINVAL),
    (dict(dtype=2), EINVAL), (dict(ends=0), EINVAL), (dict(out=0), EINVAL), (dict(ends=SPACE + 2), EALIGN), (dict(out=SPACE + 1), EALIGN),
]


@pytest.mark.parametrize("change,status", BAD_EXPERTS)
def test_expert_refusals(change, status):
    lib, packed = ops.load_library(), experts(**change)
    for name in ("linear", "input_grad", "weight_grad"):
        assert getattr(lib, "dear_expert_" + name)(packed, None) == status


def test_expert_refusals_of_each():
    lib = ops.load_library()
    x = ((dict(x=0), EINVAL), (dict(x_stride=39), EINVAL), (dict(x=SPACE + 1), EALIGN))
    dy = ((dict(dy=0), EINVAL), (dict(dy_stride=23), EINVAL), (dict(dy=SPACE + 1), EALIGN))
    weight = ((dict(weight=0), EINVAL), (dict(weight=SPACE + 1), EALIGN))
    many = ((dict(rows=(1 << 31) - 1, outs=1 << 20, ins=1 << 20, x_stride=1 << 20, dy_stride=1 << 20), ETOOBIG),)
    for name, bad in (("linear", x + weight + many), ("input_grad", dy + weight + many), ("weight_grad", x + dy + ((dict(out=SPACE + 2), EALIGN),)),
                      ("weight_grad", ((dict(outs=1 << 20, ins=1 << 20, x_stride=1 << 20, dy_stride=1 << 20), ETOOBIG),))):
        f = getattr(lib, "dear_expert_" + name)
        for change, status in bad:
            assert f(experts(**change), None) == status, (name, change)
        assert f(None, None) == EINVAL
    n = C.c_int64(-1)
    for name in ("linear", "input_grad", "weight_grad"):
        f = getattr(lib, "dear_expert_%s_workspace" % name)
        assert f(experts(), C.byref(n)) == OK and n.value >= 0
        assert f(experts(outs=0), C.byref(n)) == EINVAL and f(experts(), None) == EINVAL and f(None, C.byref(n)) == EINVAL
    none = bytes(Experts(rows=0, experts=3, outs=24, ins=40, dtype=1))
    assert lib.dear_expert_linear(none, None) == OK and lib.dear_expert_input_grad(none, None) == OK


def test_gradient_refusals():
    lib = ops.load_library()
    n = C.c_int64(-1)
    assert lib.dear_grad_norm_workspace(400, C.byref(n)) == OK and n.value >= 8 * 2048
    assert lib.dear_grad_norm_workspace(-1, C.byref(n)) == EINVAL and lib.dear_grad_norm_workspace(4, None) == EINVAL
    assert lib.dear_grad_norm_workspace((1 << 20) + 1, C.byref(n)) == EINVAL
    good = (SPACE, SPACE, 100, 0, 0)
    for rows, status in ((((0, SPACE, 100, 0, 0),), EINVAL), (((SPACE, SPACE, -1, 0, 0),), EINVAL), (((SPACE, SPACE, 100, 2, 0),), EINVAL),
                         (((SPACE + 2, SPACE, 100, 0, 0),), EALIGN), (((SPACE + 1, SPACE, 100, 1, 0),), EALIGN),
                         (((SPACE, SPACE, (1 << 56) + 1, 0, 0),), EINVAL), (((SPACE, SPACE, 1 << 56, 0, 0), good), EINVAL)):
        assert lib.dear_grad_norm(grads(*rows), len(rows), SPACE, SPACE, BIG, None) == status, rows
        assert lib.dear_clip_grads(grads(*rows), len(rows), 1.0, SPACE, SPACE, BIG, None) == status, rows
    for rows, status in ((((SPACE, 0, 100, 0, 0),), EINVAL), (((SPACE, SPACE, 100, 0, 3),), EINVAL), (((SPACE, SPACE + 402, 100, 0, 0),), EALIGN),
                         (((SPACE, SPACE, 100, 0, 1),), EINVAL),                          # in place, of another type
                         (((SPACE, SPACE + 4, 100, 0, 0),), EINVAL),                      # half on itself
                         ((good, good), EINVAL), ((good, (SPACE + 4096, SPACE + 396, 100, 0, 0)), EINVAL),
                         ((good, (SPACE + 8, SPACE + 4096, 4, 0, 0)), EINVAL)):           # an output on another tensor's input
        assert lib.dear_clip_grads(grads(*rows), len(rows), 1.0, SPACE, SPACE, BIG, None) == status, rows
    one = grads(good)
    for args, status in (((one, 1, 0.0, SPACE, SPACE, BIG), EINVAL), ((one, 1, -1.0, SPACE, SPACE, BIG), EINVAL), ((one, 1, float("nan"), SPACE, SPACE, BIG), EINVAL),
                         ((one, 1, 1.0, None, SPACE, BIG), EINVAL), ((one, 1, 1.0, SPACE, None, BIG), EINVAL), ((one, -1, 1.0, SPACE, SPACE, BIG), EINVAL),
                         ((None, 1, 1.0, SPACE, SPACE, BIG), EINVAL), ((one, 1, 1.0, SPACE + 2, SPACE, BIG), EALIGN),
                         ((one, 1, 1.0, SPACE, SPACE + 8, BIG), EALIGN), ((one, 1, 1.0, SPACE, SPACE, 100), ETOOBIG)):
        assert lib.dear_clip_grads(*args, None) == status, args[1:]


def test_python_refusals():
    t, f = torch.zeros(2, 5, 8, dtype=torch.bfloat16), torch.zeros(4, 8)
    with pytest.raises(ValueError, match="not on a GPU"):
        ops.recurrence(t, t)
    with pytest.raises(ValueError, match="not on a GPU"):
        ops.recurrence_backward(t, t, t, f)
    for call in (lambda: ops.expert_linear(f, f[None], torch.zeros(1, dtype=torch.int32)),
                 lambda: ops.expert_input_grad(f, f[None], torch.zeros(1, dtype=torch.int32)),
                 lambda: ops.expert_weight_grad(f, f, torch.zeros(1, dtype=torch.int32)), lambda: ops.grad_norm([f]), lambda: ops.clip_grads([f], 1.0)):
        with pytest.raises(ValueError, match="not on a GPU"):
            call()
    with pytest.raises(ValueError, match="no tensors"):
        ops.grad_norm([])
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(ValueError, match="max_norm"):
            ops.clip_grads([f], bad)
    with pytest.raises(ValueError, match="2 tensors and 1"):
        ops.clip_grads([f, f], 1.0, [f])
