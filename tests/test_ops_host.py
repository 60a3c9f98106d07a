"""CPU-only checks of libdear_ops: exports, the argument structure, workspace sizes and refusals.  No kernel is launched:
every call here is refused, or has nothing to do."""
from __future__ import annotations

import ctypes as C
import os
import re

import pytest
import torch

import paper_2302_12445_amd as dear
from paper_2302_12445_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, EALIGN, ETOOBIG = 0, -1, -5, -6
SPACE = 1 << 20  # an aligned address that is never read: the calls here return before


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "dear_ops.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(dear_[a-z_]+)\s*\(", header))
    assert declared == set(ops.EXPORTS)
    lib = ops.load_library()
    for name in declared:
        assert hasattr(lib, name), name
    assert "#define DEAR_CHECKPOINT_GROUP %d" % ops.GROUP in header
    assert "#define DEAR_NORM_MAX_COLS %d" % ops.NORM_MAX_COLS in header


def attention_bytes(batch=2, q_heads=4, kv_heads=2, head_dim=64, q_len=16, kv_len=24, dtype=1, causal=0, scale=0.125, lse=SPACE,
                    workspace=SPACE, workspace_bytes=1 << 30, **tensors):
    def strides(heads, n):
        return (SPACE, n * heads * head_dim, heads * head_dim, head_dim)
    t = {"q": strides(q_heads, q_len), "k": strides(kv_heads, kv_len), "v": strides(kv_heads, kv_len), "out": strides(q_heads, q_len)}
    t.update(dout=t["q"], dq=t["q"], dk=t["k"], dv=t["k"])
    t.update(tensors)
    return ops._ATTENTION.pack(batch, q_heads, kv_heads, head_dim, q_len, kv_len, dtype, causal, scale, 0, 0, 0, *t["q"], *t["k"],
                               *t["v"], *t["out"], lse, *t["dout"], *t["dq"], *t["dk"], *t["dv"], workspace, workspace_bytes)


def test_attention_structure_is_the_header_s():
    """Sizes of the C structure, member by member."""
    class Heads(C.Structure):
        _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]

    class Attention(C.Structure):
        _fields_ = [("batch", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                    ("q_len", C.c_int64), ("kv_len", C.c_int64), ("dtype", C.c_int32), ("causal", C.c_int32), ("scale", C.c_float),
                    ("reserved", C.c_int32), ("q_lens", C.c_void_p), ("kv_lens", C.c_void_p), ("q", Heads), ("k", Heads), ("v", Heads),
                    ("out", Heads), ("lse", C.c_void_p), ("dout", Heads), ("dq", Heads), ("dk", Heads), ("dv", Heads),
                    ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]
    assert C.sizeof(Attention) == ops._ATTENTION.size
    a = Attention.from_buffer_copy(attention_bytes(batch=3, lse=77, workspace_bytes=99, dv=(1, 2, 3, 4)))
    assert (a.batch, a.q_heads, a.kv_heads, a.head_dim, a.q_len, a.kv_len, a.dtype, a.lse, a.workspace_bytes) == (3, 4, 2, 64, 16, 24, 1, 77, 99)
    assert (a.dv.data, a.dv.batch, a.dv.token, a.dv.head) == (1, 2, 3, 4) and a.scale == 0.125


BAD_ATTENTION = [
    (dict(batch=-1), EINVAL), (dict(q_heads=0), EINVAL), (dict(kv_heads=0), EINVAL), (dict(q_heads=3), EINVAL), (dict(kv_heads=8), EINVAL),
    (dict(head_dim=0), EINVAL), (dict(head_dim=63), EINVAL), (dict(head_dim=4), EINVAL), (dict(head_dim=136), EINVAL),
    (dict(q_len=-1), EINVAL), (dict(kv_len=-1), EINVAL), (dict(q_len=(1 << 30) + 1), EINVAL), (dict(kv_len=1 << 40), EINVAL),
    (dict(dtype=2), EINVAL), (dict(causal=2), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=-1.0), EINVAL),
    (dict(scale=float("nan")), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(lse=0), EINVAL), (dict(lse=SPACE + 2), EALIGN),
    (dict(q=(0, 4096, 256, 64)), EINVAL), (dict(q=(SPACE + 8, 4096, 256, 64)), EALIGN), (dict(k=(SPACE, 1536, 132, 64)), EALIGN),
    (dict(v=(SPACE, 1536, 128, 60)), EALIGN), (dict(v=(SPACE, -1536, 128, 64)), EINVAL), (dict(q_len=1 << 30, batch=64), ETOOBIG),
]


@pytest.mark.parametrize("change,status", BAD_ATTENTION)
def test_attention_refusals(change, status):
    lib = ops.load_library()
    packed = attention_bytes(**change)
    assert lib.dear_attention(packed, None) == status
    assert lib.dear_attention_backward(packed, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(out=(SPACE, 0, 256, 64)), EINVAL), (dict(out=(SPACE, 4096, 0, 64)), EINVAL), (dict(out=(SPACE, 4096, 256, 0)), EINVAL),
    (dict(out=(0, 4096, 256, 64)), EINVAL)])
def test_attention_refuses_outputs_without_places_of_their_own(change, status):
    assert ops.load_library().dear_attention(attention_bytes(**change), None) == status


@pytest.mark.parametrize("change,status", [
    (dict(workspace=0), EINVAL), (dict(workspace=SPACE + 16), EALIGN), (dict(workspace_bytes=511), ETOOBIG), (dict(dout=(0, 0, 0, 0)), EINVAL),
    (dict(dq=(SPACE, 4096, 0, 64)), EINVAL), (dict(dk=(SPACE, 0, 128, 64)), EINVAL), (dict(dv=(SPACE, 1536, 128, 0)), EINVAL),
    (dict(dk=(SPACE + 4, 1536, 128, 64)), EALIGN), (dict(kv_len=1 << 30, q_len=1, batch=128), ETOOBIG)])
def test_attention_backward_refusals(change, status):
    assert ops.load_library().dear_attention_backward(attention_bytes(**change), None) == status


def test_attention_of_nothing_launches_nothing():
    lib = ops.load_library()
    none = (0, 0, 0, 0)
    nothing = dict(q=none, k=none, v=none, out=none, dout=none, dq=none, dk=none, dv=none, lse=0, workspace=0, workspace_bytes=0)
    assert lib.dear_attention(attention_bytes(batch=0, **nothing), None) == OK
    assert lib.dear_attention_backward(attention_bytes(batch=0, **nothing), None) == OK
    assert lib.dear_attention_backward(attention_bytes(q_len=0, kv_len=0, **nothing), None) == OK
    assert lib.dear_attention(attention_bytes(q_len=0, **dict(nothing, k=(SPACE, 1536, 128, 64), v=(SPACE, 1536, 128, 64))), None) == OK


def test_workspaces():
    lib, n = ops.load_library(), C.c_int64(-1)
    assert lib.dear_attention_backward_workspace(attention_bytes(), C.byref(n)) == OK and n.value >= 2 * 4 * 16 * 4
    assert lib.dear_attention_workspace(attention_bytes(), C.byref(n)) == OK and n.value >= 0
    assert lib.dear_attention_workspace(attention_bytes(head_dim=5), C.byref(n)) == EINVAL
    assert lib.dear_attention_backward_workspace(attention_bytes(), None) == EINVAL
    assert lib.dear_attention_workspace(None, C.byref(n)) == EINVAL and lib.dear_attention(None, None) == EINVAL
    assert lib.dear_checkpoint_weight_grad_workspace(1, 5, 7, 9, C.byref(n)) == OK and n.value >= 0
    assert lib.dear_checkpoint_weight_grad_workspace(1, 1 << 40, 1 << 24, 1 << 24, C.byref(n)) == OK and n.value >= 0
    for bad in ((2, 5, 7, 9), (1, -1, 7, 9), (1, 5, 0, 9), (1, 5, 7, 0), (1, 5, (1 << 24) + 1, 9), (1, (1 << 40) + 1, 7, 9)):
        assert lib.dear_checkpoint_weight_grad_workspace(*bad, C.byref(n)) == EINVAL
    assert lib.dear_add_rms_norm_backward_workspace(0, 100, 1024, C.byref(n)) == OK and n.value >= 4096
    for bad in ((2, 5, 7), (1, -1, 7), (1, 5, 0), (1, 5, 32769)):
        assert lib.dear_add_rms_norm_backward_workspace(*bad, C.byref(n)) == EINVAL


def test_checkpoint_refusals():
    lib, p = ops.load_library(), SPACE
    enc, dec = lib.dear_checkpoint_encode, lib.dear_checkpoint_decode
    assert enc(None, 1, 0, 8, 8, None, None, None) == OK and dec(None, None, 0, 8, 1, None, None) == OK
    for args, status in (((0, 1, 4, 8, 8, p, p), EINVAL), ((p, 2, 4, 8, 8, p, p), EINVAL), ((p, 1, -1, 8, 8, p, p), EINVAL),
                         ((p, 1, 4, 0, 8, p, p), EINVAL), ((p, 1, 4, 8, 7, p, p), EINVAL), ((p, 1, 4, 8, 8, 0, p), EINVAL),
                         ((p, 1, 4, 8, 8, p, 0), EINVAL), ((p + 1, 1, 4, 8, 8, p, p), EALIGN), ((p + 2, 0, 4, 8, 8, p, p), EALIGN),
                         ((p, 1, 4, 8, 8, p + 8, p), EALIGN), ((p, 1, 1 << 40, 1 << 20, 1 << 20, p, p), ETOOBIG),
                         ((p, 1, 4, 1 << 31, 1 << 31, p, p), EINVAL)):
        assert enc(*args, None) == status, args
    for args, status in (((0, p, 4, 8, 1, p), EINVAL), ((p, 0, 4, 8, 1, p), EINVAL), ((p, p, 4, 8, 1, 0), EINVAL),
                         ((p, p, 4, 8, 3, p), EINVAL), ((p, p, -4, 8, 1, p), EINVAL), ((p, p, 4, 0, 1, p), EINVAL),
                         ((p + 4, p, 4, 8, 1, p), EALIGN), ((p, p, 4, 8, 0, p + 2), EALIGN), ((p, p, 1 << 40, 1 << 20, 1, p), ETOOBIG)):
        assert dec(*args, None) == status, args


def test_weight_grad_refusals():
    f, p = ops.load_library().dear_checkpoint_weight_grad, SPACE
    big = 1 << 40
    for args, status in (((0, 1, 8, p, p, 4, 8, 8, p, p, big), EINVAL), ((p, 3, 8, p, p, 4, 8, 8, p, p, big), EINVAL),
                         ((p, 1, 7, p, p, 4, 8, 8, p, p, big), EINVAL), ((p, 1, 8, 0, p, 4, 8, 8, p, p, big), EINVAL),
                         ((p, 1, 8, p, 0, 4, 8, 8, p, p, big), EINVAL), ((p, 1, 8, p, p, -1, 8, 8, p, p, big), EINVAL),
                         ((p, 1, 8, p, p, 4, 0, 8, p, p, big), EINVAL), ((p, 1, 8, p, p, 4, 8, 0, p, p, big), EINVAL),
                         ((p, 1, 8, p, p, 4, 8, 8, 0, p, big), EINVAL), ((p + 1, 1, 8, p, p, 4, 8, 8, p, p, big), EALIGN),
                         ((p, 1, 8, p + 8, p, 4, 8, 8, p, p, big), EALIGN), ((p, 1, 8, p, p, 4, 8, 8, p + 4, p, big), EALIGN)):
        assert f(*args, None) == status, args
    # a long sum over few outputs is split, and needs its workspace
    n = C.c_int64()
    assert ops.load_library().dear_checkpoint_weight_grad_workspace(1, 1 << 16, 64, 64, C.byref(n)) == OK and n.value > 0
    assert f(p, 1, 64, p, p, 1 << 16, 64, 64, p, 0, n.value, None) == EINVAL
    assert f(p, 1, 64, p, p, 1 << 16, 64, 64, p, p, n.value - 1, None) == ETOOBIG
    assert f(p, 1, 64, p, p, 1 << 16, 64, 64, p, p + 64, n.value, None) == EALIGN


def test_norm_refusals():
    lib, p = ops.load_library(), SPACE
    ok = dict(x=p, xs=8, r=p, rs=8, w=p, t=1, rows=4, cols=8, eps=1e-5, h=p, y=p, c=p, e=p, rstd=p)
    def call(**change):
        a = dict(ok, **change)
        return lib.dear_add_rms_norm(a["x"], a["xs"], a["r"], a["rs"], a["w"], a["t"], a["rows"], a["cols"], a["eps"], a["h"], a["y"],
                                     a["c"], a["e"], a["rstd"], None)
    assert call(rows=0, x=0, r=0, w=0, h=0, y=0, c=0, e=0, rstd=0) == OK
    for change, status in ((dict(x=0), EINVAL), (dict(xs=7), EINVAL), (dict(rs=7), EINVAL), (dict(w=0), EINVAL), (dict(t=5), EINVAL),
                           (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL), (dict(cols=32769, xs=32769, rs=32769), EINVAL),
                           (dict(eps=-1.0), EINVAL), (dict(eps=float("nan")), EINVAL), (dict(h=0), EINVAL), (dict(r=0), EINVAL),
                           (dict(c=0), EINVAL), (dict(e=0), EINVAL), (dict(rstd=0), EINVAL), (dict(x=p + 1), EALIGN), (dict(h=p + 1), EALIGN),
                           (dict(y=p + 1), EALIGN), (dict(w=p + 2), EALIGN), (dict(c=p + 8), EALIGN), (dict(rstd=p + 2), EALIGN),
                           (dict(rows=1 << 32), ETOOBIG)):
        assert call(**change) == status, change
    ok = dict(dy=p, dys=8, h=p, hs=8, dh=p, dhs=8, w=p, rstd=p, t=1, rows=4, cols=8, dx=p, dw=p, ws=p, n=1 << 30)
    def back(**change):
        a = dict(ok, **change)
        return lib.dear_add_rms_norm_backward(a["dy"], a["dys"], a["h"], a["hs"], a["dh"], a["dhs"], a["w"], a["rstd"], a["t"], a["rows"],
                                              a["cols"], a["dx"], a["dw"], a["ws"], a["n"], None)
    for change, status in ((dict(dy=0), EINVAL), (dict(dys=7), EINVAL), (dict(h=0), EINVAL), (dict(hs=7), EINVAL), (dict(dhs=7), EINVAL),
                           (dict(w=0), EINVAL), (dict(rstd=0), EINVAL), (dict(t=7), EINVAL), (dict(rows=-1), EINVAL), (dict(cols=0), EINVAL),
                           (dict(dx=0), EINVAL), (dict(dw=0), EINVAL), (dict(ws=0), EINVAL), (dict(ws=p + 16), EALIGN), (dict(n=1), ETOOBIG),
                           (dict(dy=p + 1), EALIGN), (dict(dh=p + 1), EALIGN), (dict(dw=p + 2), EALIGN)):
        assert back(**change) == status, change


def test_tensors_off_the_gpu_are_refused():
    q, w = torch.zeros(1, 4, 2, 64), torch.ones(64)
    kept = ops.Checkpoint(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 2, dtype=torch.uint8), 64)
    for f in (lambda: ops.attention(q, q, q), lambda: ops.attention_backward(q, q, q, q, q, w), lambda: ops.checkpoint_encode(w),
              lambda: ops.checkpoint_decode(kept), lambda: ops.checkpoint_weight_grad(q[0, :, 0], kept),
              lambda: ops.add_rms_norm(q, q, w), lambda: ops.add_rms_norm_backward(q, q, w, w)):
        with pytest.raises(ValueError):
            f()


def test_errors_are_described():
    assert "align" in dear.strerror(EALIGN)


def test_attention_of_more_threads_than_a_launch_takes():
    """2^24 workgroups of 256 threads, or 2^23 of 512, are refused before anything is launched."""
    lib, room = ops.load_library(), 1 << 60
    many = dict(batch=1 << 20, q_heads=16, kv_heads=16, q_len=16, kv_len=24, workspace_bytes=room)
    assert lib.dear_attention(attention_bytes(**many), None) == ETOOBIG
    assert lib.dear_attention_backward(attention_bytes(**many), None) == ETOOBIG
    keys = dict(batch=1 << 16, q_heads=16, kv_heads=16, q_len=16, kv_len=512, workspace_bytes=room)
    assert lib.dear_attention_backward(attention_bytes(**dict(keys, head_dim=128)), None) == ETOOBIG
    assert lib.dear_attention_backward(attention_bytes(**dict(keys, kv_len=1024, dtype=0)), None) == ETOOBIG


def test_weight_grad_of_more_threads_than_a_launch_takes():
    """2^24 tiles of 256 threads are refused before anything is launched."""
    f, p, big = ops.load_library().dear_checkpoint_weight_grad, SPACE, 1 << 60
    assert f(p, 1, 1 << 19, p, p, 4, 1 << 19, 1 << 19, p, p, big, None) == ETOOBIG
    assert f(p, 0, 1 << 24, p, p, 4, 1 << 24, 1 << 14, p, p, big, None) == ETOOBIG


# batch 2, 4 query and 2 key heads of 64 values, 16 queries and 24 keys; (data, batch, token, head) strides
OVERLAPPING = [(64, 64), (64, 128), (128, 64), (256, 128), (64, 512), (192, 64)]  # token, head
APART = [(4096, 64, 1024), (8192, 256, 64), (64 * 16 * 4, 64, 64 * 16), (1 << 20, 1 << 10, 64), (64, 512, 128), (256, 512, 64), (8192, 264, 64)]


@pytest.mark.parametrize("token,head", OVERLAPPING)
@pytest.mark.parametrize("name", ["out", "dq"])
def test_attention_refuses_outputs_whose_elements_share_a_place(name, token, head):
    """Strides that are each long enough by themselves, and still lead two elements to one place."""
    call = ops.load_library().dear_attention if name == "out" else ops.load_library().dear_attention_backward
    few = dict(kv_len=8192, workspace_bytes=0)  # a call that needs a workspace, which is looked at last
    assert call(attention_bytes(**{name: (SPACE, 1 << 20, token, head)}, **few), None) == EINVAL
    assert call(attention_bytes(**{name: (SPACE, 512, 256, 64)}, **few), None) == EINVAL  # batches
    assert call(attention_bytes(**{name: (SPACE, 64, 1 << 10, 1 << 20)}, **few), None) == ETOOBIG


def test_attention_takes_outputs_of_any_order():
    """Refused for their workspace alone."""
    lib = ops.load_library()
    for batch, token, head in APART:
        change = dict(dq=(SPACE, batch, token, head), workspace_bytes=0)
        assert lib.dear_attention_backward(attention_bytes(**change), None) == ETOOBIG, (batch, token, head)
    # axes of one element: their strides say nothing
    one = dict(batch=1, q_heads=1, kv_heads=1, q_len=1, workspace_bytes=0)
    assert lib.dear_attention_backward(attention_bytes(dq=(SPACE, 0, 0, 0), **one), None) == ETOOBIG


def test_attention_refuses_what_is_reserved():
    lib, at = ops.load_library(), 4 * 4 + 2 * 8 + 2 * 4 + 4  # behind scale
    packed = bytearray(attention_bytes(kv_len=8192, workspace_bytes=0))
    n = C.c_int64()
    assert lib.dear_attention_workspace(bytes(packed), C.byref(n)) == OK and n.value > 0
    packed[at] = 1
    for f in (lib.dear_attention, lib.dear_attention_backward):
        assert f(bytes(packed), None) == EINVAL
    for f in (lib.dear_attention_workspace, lib.dear_attention_backward_workspace):
        assert f(bytes(packed), C.byref(n)) == EINVAL


@pytest.mark.parametrize("scale", [1e39, -1e39, 3.5e38])
def test_a_scale_that_fp32_does_not_hold_is_a_value_error(monkeypatch, scale):
    monkeypatch.setattr(ops, "_dtype", lambda t, what: 0)  # (tensors here are on the CPU)
    q = torch.zeros(1, 4, 2, 64)
    ops._ATTENTION.pack(*ops._attention_sizes(q, q, q, False, 3.4e38, None, None)[2], *([0] * 35))
    with pytest.raises(ValueError):
        ops._attention_sizes(q, q, q, False, scale, None, None)
