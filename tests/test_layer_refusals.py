"""What the entry points around the sparse attention refuse before anything is launched, without a GPU: through the C ABI, so that the
binding's own checks are not in the way."""
import ctypes as C

import numpy as np
import pytest

from paper_2508_21058_b200 import MocCross, MocError, MocRope, load_library
from paper_2508_21058_b200.binding import _CrossProblem, _Rows

NULL, SHAPE, TABLE, ALIGN, WORKSPACE = -1, -2, -3, -4, -5


def _code(f, *a, **kw):
    with pytest.raises(MocError) as e:
        f(*a, **kw)
    return e.value.code


def test_rope_problem():
    assert _code(MocRope, 96) == SHAPE
    assert _code(MocRope, 64, [0] * 33, [1.0] * 33) == SHAPE
    assert _code(MocRope, 64, [0] * 12, [1.0] * 12, halves=True) == SHAPE          # not a multiple of eight pairs
    assert _code(MocRope, 64, [0, 4], [1.0, 1.0], n_axes=5) == SHAPE
    assert _code(MocRope, 64, [0, 2], [1.0, 1.0], n_axes=2) == SHAPE
    assert _code(MocRope, 64, [0, -1], [1.0, 1.0], n_axes=2) == SHAPE
    assert _code(MocRope, 64, [0], [float("nan")]) == SHAPE
    assert _code(MocRope, 64, [0], [float("inf")]) == SHAPE
    assert _code(MocRope, 64, [0], [1.0, 2.0]) == SHAPE
    assert _code(MocRope, 64, eps=-1.0) == SHAPE
    assert _code(MocRope, 64, eps=float("nan")) == SHAPE
    assert _code(MocRope.from_axes, 64, (16, 3)) == SHAPE
    assert _code(MocRope.from_axes, 64, (32, 34)) == SHAPE
    assert MocRope(64).workspace_bytes() > 0 and MocRope.from_axes(128, (44, 42, 42)).n_axes == 3


def test_rope_calls():
    lib, op = load_library(), MocRope.from_axes(64, (16, 24, 24))
    addr = 1 << 20                                       # never followed: every call here is refused before a launch

    def rows(head=64, tok=256, data=addr):
        return C.byref(_Rows(data, head, tok))

    def fwd(x_type=0, L=8, hq=4, hk=0, pos=addr, q=None, w=addr, out=None):
        return lib.moc_norm_rope(op._h, x_type, L, hq, hk, pos, q or rows(), w, out or rows(), None, None, None, None)

    assert lib.moc_norm_rope(None, 0, 8, 4, 0, addr, rows(), None, rows(), None, None, None, None) == NULL
    assert fwd(x_type=2) == SHAPE and fwd(L=-1) == SHAPE and fwd(hq=0) == SHAPE and fwd(hq=70000) == SHAPE and fwd(hk=-1) == SHAPE
    assert fwd(pos=None) == NULL and fwd(pos=addr + 2) == ALIGN
    assert fwd(q=rows(data=None)) == NULL and fwd(q=rows(data=addr + 8)) == ALIGN and fwd(w=addr + 1) == ALIGN
    assert fwd(q=rows(head=0)) == SHAPE and fwd(q=rows(tok=0)) == SHAPE              # broadcast tensors
    assert fwd(q=rows(head=68, tok=512)) == ALIGN
    assert fwd(q=rows(head=64, tok=192)) == SHAPE                                    # a token's heads reach into the next token
    assert fwd(q=rows(head=64 * 7, tok=64)) == SHAPE                                 # a head's tokens reach into the next head
    assert fwd(q=rows(head=-64)) == SHAPE and fwd(q=rows(head=1 << 40)) == SHAPE
    assert fwd(out=rows(tok=64)) == SHAPE
    assert fwd(hk=2) == NULL                                                         # keys without tensors

    def bwd(ws=addr, w=addr, dw=addr, x=None):
        return lib.moc_norm_rope_bwd(op._h, 0, 8, 4, 0, addr, x or rows(), w, rows(), rows(), dw, None, None, None, None, None, ws, None)

    assert bwd(ws=None) == WORKSPACE and bwd(ws=addr + 16) == ALIGN
    assert bwd(dw=None) == NULL and bwd(w=None) == SHAPE and bwd(x=rows(data=None)) == NULL


@pytest.mark.parametrize("kw,code", [
    (dict(n_heads=0), SHAPE), (dict(n_heads=4, n_kv_heads=3), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(head_dim=80), SHAPE),
    (dict(softmax_scale=-1.0), SHAPE), (dict(softmax_scale=float("nan")), SHAPE), (dict(softmax_scale=float("inf")), SHAPE),
    (dict(q_off=[1, 5]), TABLE), (dict(k_off=[1, 5]), TABLE), (dict(q_off=[0, 5, 4], k_off=[0, 5, 6]), TABLE),
    (dict(q_off=[0, 5, 6], k_off=[0, 5, 4]), TABLE), (dict(k_len=[6]), TABLE), (dict(k_len=[-1]), TABLE),
    (dict(q_off=[0, 5, 6]), TABLE), (dict(k_len=[1, 1]), TABLE), (dict(q_off=[0, 2**30]), SHAPE), (dict(k_off=[0, 2**30]), SHAPE),
])
def test_cross_problem(kw, code):
    args = dict(n_heads=2, n_kv_heads=2, head_dim=64, q_off=[0, 5], k_off=[0, 5])
    args.update(kw)
    assert _code(MocCross, **args) == code


def test_cross_null_arguments():
    lib, h = load_library(), C.c_void_p(0)
    off = np.array([0, 4], np.int32)
    assert lib.moc_cross_create(None, C.byref(h)) == NULL
    assert lib.moc_cross_create(C.byref(_CrossProblem(1, 1, 64, 1, 0.0, None, off.ctypes.data, None)), C.byref(h)) == NULL
    assert lib.moc_cross_create(C.byref(_CrossProblem(1, 1, 64, -1, 0.0, off.ctypes.data, off.ctypes.data, None)), C.byref(h)) == SHAPE
    assert lib.moc_cross_destroy(None) == NULL and lib.moc_rope_destroy(None) == NULL
    assert lib.moc_cross_attend(None, None, None, None, None, None, None, None) == NULL
    n = C.c_size_t(0)
    assert lib.moc_cross_workspace_bytes(None, 0, C.byref(n)) == NULL and lib.moc_rope_workspace_bytes(None, C.byref(n)) == NULL
