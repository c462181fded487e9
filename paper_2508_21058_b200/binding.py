"""ctypes binding of ``libmoc.so``.  Same names as the C entry points (include/moc.h);
argument marshalling only.  torch supplies device memory and the stream."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np
import torch

_DIR = os.path.dirname(os.path.abspath(__file__))
FLAG_CAUSAL = 0x1
WHOLE_SHOT = -1


class MocError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(what)
        self.code = code


class _Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("head_stride", C.c_int64), ("token_stride", C.c_int64)]


class _RopeProblem(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("n_pairs", C.c_int32), ("n_axes", C.c_int32), ("flags", C.c_uint32), ("eps", C.c_float),
                ("pair_axis", C.c_void_p), ("pair_freq", C.c_void_p)]


class _CrossProblem(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("n_segments", C.c_int32),
                ("softmax_scale", C.c_float), ("q_off", C.c_void_p), ("k_off", C.c_void_p), ("k_len", C.c_void_p)]


class _Problem(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("n_tokens", C.c_int32), ("head_dim", C.c_int32),
                ("n_chunks", C.c_int32), ("top_k", C.c_int32), ("win_back", C.c_int32), ("win_fwd", C.c_int32),
                ("flags", C.c_uint32), ("softmax_scale", C.c_float),
                ("chunk_off", C.c_void_p), ("chunk_shot", C.c_void_p), ("chunk_mod", C.c_void_p)]


_lib = None


def lib_path() -> str:
    """The library this process loads: libmoc.so beside this file, or (MOC_LIBRARY=debug) the build with
    index checks, libmoc_debug.so."""
    return os.path.join(_DIR, "libmoc_debug.so" if os.environ.get("MOC_LIBRARY") == "debug" else "libmoc.so")


def load_library():
    """dlopen the CUDA library.  Raises if it has not been built: nothing else can run the path."""
    global _lib
    if _lib is not None:
        return _lib
    path = lib_path()
    if not os.path.exists(path):
        raise MocError(-100, f"{path} is missing: build it with `python -m paper_2508_21058_b200.build` "
                             "(there is no fallback implementation)")
    lib = C.CDLL(path)
    vp, i32, sz = C.c_void_p, C.c_int, C.c_size_t
    lib.moc_plan_create.argtypes = [C.POINTER(_Problem), C.POINTER(vp)]
    lib.moc_plan_destroy.argtypes = [vp]
    lib.moc_workspace_bytes.argtypes = [vp, i32, C.POINTER(sz)]
    lib.moc_chunk_pool.argtypes = [vp, vp, vp, vp, vp]
    lib.moc_chunk_pool_noalloc.argtypes = [vp, vp, vp, vp]
    lib.moc_plan_set_workspace_budget.argtypes = [vp, sz]
    lib.moc_route.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.moc_lists_from_sel.argtypes = [vp, vp, vp, vp]
    lib.moc_outer_num_shots.argtypes = [vp, C.POINTER(C.c_int32)]
    lib.moc_outer_route.argtypes = [vp, vp, vp, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp, vp, vp]
    lib.moc_outer_reduced_layout.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                             vp, vp, vp, vp]
    lib.moc_gather_tokens.argtypes = [vp, vp, vp, C.c_int32, vp, vp]
    lib.moc_context_drop.argtypes = [vp, vp, C.c_float, C.c_float, C.c_uint64, vp, vp]
    # test hooks (exported, not in the public header)
    lib.moc_debug_use_cuda_core_attention.argtypes = [vp, i32]
    lib.moc_debug_set_wait_limit_us.argtypes = [vp, C.c_uint]
    lib.moc_debug_wait_probe.argtypes = [vp, vp, i32, vp]
    lib.moc_debug_wait_probe_form.argtypes = [vp, vp, i32, i32, vp]
    lib.moc_debug_shared_key_tiles.argtypes = [C.POINTER(_Problem), i32, i32, C.POINTER(i32), vp, vp, C.POINTER(sz)]
    lib.moc_attend.argtypes = [vp] * 9
    lib.moc_attend_bwd.argtypes = [vp] * 13
    rows = C.POINTER(_Rows)
    lib.moc_rope_create.argtypes = [C.POINTER(_RopeProblem), C.POINTER(vp)]
    lib.moc_rope_destroy.argtypes = [vp]
    lib.moc_rope_workspace_bytes.argtypes = [vp, C.POINTER(sz)]
    lib.moc_norm_rope.argtypes = [vp, i32, C.c_int32, C.c_int32, C.c_int32, vp] + [rows, vp, rows] * 2 + [vp]
    lib.moc_norm_rope_bwd.argtypes = [vp, i32, C.c_int32, C.c_int32, C.c_int32, vp] + [rows, vp, rows, rows, vp] * 2 + [vp, vp]
    lib.moc_cross_create.argtypes = [C.POINTER(_CrossProblem), C.POINTER(vp)]
    lib.moc_cross_destroy.argtypes = [vp]
    lib.moc_cross_workspace_bytes.argtypes = [vp, i32, C.POINTER(sz)]
    lib.moc_cross_attend.argtypes = [vp] + [rows] * 4 + [vp] * 3
    lib.moc_cross_attend_bwd.argtypes = [vp] + [rows] * 4 + [vp] + [rows] * 4 + [vp] * 2
    lib.moc_cross_get_status.argtypes = [vp, vp, vp, C.POINTER(i32), C.POINTER(i32)]
    lib.moc_debug_rope_split.argtypes = [i32, i32, i32, C.c_int64, i32, i32, i32, C.POINTER(C.c_int64)]
    lib.moc_debug_cross_plan.argtypes = [C.POINTER(_CrossProblem), i32, C.POINTER(C.c_int64)]
    lib.moc_selected_pairs.argtypes = [vp, vp, vp, C.POINTER(C.c_int64)]
    lib.moc_get_status.argtypes = [vp, vp, vp, C.POINTER(i32), C.POINTER(i32)]
    lib.moc_launch_count.restype = C.c_int64
    lib.moc_strerror.restype = C.c_char_p
    lib.moc_strerror.argtypes = [i32]
    lib.moc_last_cuda_error.restype = C.c_char_p
    _lib = lib
    return lib


def launch_count() -> int:
    return int(load_library().moc_launch_count())


def _check(code: int):
    if code != 0:
        lib = load_library()
        msg = lib.moc_strerror(code).decode()
        if code == -7:
            msg += ": " + lib.moc_last_cuda_error().decode()
        raise MocError(code, f"moc error {code}: {msg}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _stream():
    """The current stream's handle, without building a torch.cuda.Stream object for it (5 us a call)."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _problem(n_heads, n_tokens, head_dim, chunk_off, chunk_shot, chunk_mod, top_k, win_back, win_fwd, causal, softmax_scale):
    """The C problem statement, and the host arrays it points to."""
    off = np.ascontiguousarray(chunk_off, np.int32)
    shot = np.ascontiguousarray(chunk_shot, np.int32)
    mod = np.ascontiguousarray(chunk_mod, np.uint8)
    if len(off) != len(shot) + 1 or len(mod) != len(shot):
        raise MocError(-3, "moc error -3: chunk tables have inconsistent lengths")
    pr = _Problem(int(n_heads), int(n_tokens), int(head_dim), len(shot), int(top_k), int(win_back), int(win_fwd),
                  FLAG_CAUSAL if causal else 0, float(softmax_scale), off.ctypes.data, shot.ctypes.data, mod.ctypes.data)
    return pr, (off, shot, mod)


def debug_shared_key_tiles(wl, n_sm):
    """Test hook, host only: for each long key tile of a head in the dK/dV launch on n_sm SMs, the tiles of query rows that have it as
    an anchor and the blocks that share it; and the bytes there are for the counters of all heads' tiles."""
    lay = wl.layout
    pr, tables = _problem(wl.n_heads, lay.n_tokens, wl.head_dim, lay.chunk_off, lay.chunk_shot, lay.chunk_mod, wl.top_k, wl.win_back,
                          wl.win_fwd, wl.causal, 0.0)
    cap = lay.n_tokens // 128 + lay.n_chunks
    n, room, query_tiles, blocks = C.c_int(0), C.c_size_t(0), np.zeros(cap, np.int32), np.zeros(cap, np.int32)
    _check(load_library().moc_debug_shared_key_tiles(C.byref(pr), int(n_sm), cap, C.byref(n), query_tiles.ctypes.data, blocks.ctypes.data,
                                                     C.byref(room)))
    return query_tiles[:n.value], blocks[:n.value], room.value


class MocPlan:
    """Owns a ``moc_plan``.  Methods mirror the C entry points and take torch CUDA tensors."""

    def __init__(self, n_heads, n_tokens, head_dim, chunk_off, chunk_shot, chunk_mod, top_k,
                 win_back=0, win_fwd=0, causal=True, scalar_attend=False, softmax_scale=0.0):
        self._lib = load_library()
        self._h = C.c_void_p(0)
        pr, tables = _problem(n_heads, n_tokens, head_dim, chunk_off, chunk_shot, chunk_mod, top_k, win_back, win_fwd, causal,
                              softmax_scale)
        _check(self._lib.moc_plan_create(C.byref(pr), C.byref(self._h)))
        self.H, self.L, self.d, self.C, self.k = int(n_heads), int(n_tokens), int(head_dim), pr.n_chunks, int(top_k)
        if scalar_attend:       # test hook: the in-library CUDA-core cross-check of the attention kernels
            _check(self._lib.moc_debug_use_cuda_core_attention(self._h, 1))

    @classmethod
    def from_workload(cls, wl, n_heads=None, **kw):
        lay = wl.layout
        return cls(wl.n_heads if n_heads is None else n_heads, lay.n_tokens, wl.head_dim, lay.chunk_off,
                   lay.chunk_shot, lay.chunk_mod, wl.top_k, wl.win_back, wl.win_fwd, wl.causal, **kw)

    def close(self):
        if self._h:
            self._lib.moc_plan_destroy(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self, with_bwd=False) -> int:
        n = C.c_size_t(0)
        _check(self._lib.moc_workspace_bytes(self._h, int(with_bwd), C.byref(n)))
        return int(n.value)

    def moc_plan_set_workspace_budget(self, max_bytes: int):
        _check(self._lib.moc_plan_set_workspace_budget(self._h, C.c_size_t(int(max_bytes))))

    def new_workspace(self, with_bwd=False, device="cuda") -> torch.Tensor:
        return torch.empty(self.workspace_bytes(with_bwd), dtype=torch.uint8, device=device)

    def moc_chunk_pool(self, K, desc, ws):
        _check(self._lib.moc_chunk_pool(self._h, _ptr(K), _ptr(desc), _ptr(ws), _stream()))

    def moc_chunk_pool_noalloc(self, K, desc):
        """Descriptors without a workspace: scratch is a fixed array inside the library (small
        problems only; raises MocError -9 beyond its size).  Calls sharing a GPU must not overlap."""
        _check(self._lib.moc_chunk_pool_noalloc(self._h, _ptr(K), _ptr(desc), _stream()))

    def moc_route(self, Q, desc, sel_idx, ws):
        _check(self._lib.moc_route(self._h, _ptr(Q), _ptr(desc), _ptr(sel_idx), _ptr(ws), _stream()))

    def moc_lists_from_sel(self, sel_idx, ws):
        _check(self._lib.moc_lists_from_sel(self._h, _ptr(sel_idx), _ptr(ws), _stream()))

    def moc_context_drop(self, sel_idx, p_max, lam, seed, ws):
        _check(self._lib.moc_context_drop(self._h, _ptr(sel_idx), float(p_max), float(lam), int(seed), _ptr(ws), _stream()))

    def moc_attend(self, Q, K, V, sel_idx, O, lse, ws):
        _check(self._lib.moc_attend(self._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(sel_idx), _ptr(O), _ptr(lse), _ptr(ws),
                                    _stream()))

    def moc_attend_bwd(self, Q, K, V, O, lse, dO, sel_idx, dQ, dK, dV, ws):
        _check(self._lib.moc_attend_bwd(self._h, _ptr(Q), _ptr(K), _ptr(V), _ptr(O), _ptr(lse), _ptr(dO),
                                        _ptr(sel_idx), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(ws), _stream()))

    def moc_selected_pairs(self, ws) -> int:
        n = C.c_int64(0)
        _check(self._lib.moc_selected_pairs(self._h, _ptr(ws), _stream(), C.byref(n)))
        return int(n.value)

    def moc_get_status(self, ws):
        st, det = C.c_int(0), C.c_int(0)
        _check(self._lib.moc_get_status(self._h, _ptr(ws), _stream(), C.byref(st), C.byref(det)))
        return int(st.value), int(det.value)

    def moc_outer_num_shots(self) -> int:
        n = C.c_int32(0)
        _check(self._lib.moc_outer_num_shots(self._h, C.byref(n)))
        return int(n.value)

    def moc_outer_route(self, Xq, desc, q_tok0, q_tok1, top_m, shot_desc, scores, sel_shot, ws):
        _check(self._lib.moc_outer_route(self._h, _ptr(Xq), _ptr(desc), int(q_tok0), int(q_tok1), int(top_m), _ptr(shot_desc),
                                         _ptr(scores), _ptr(sel_shot), _ptr(ws), _stream()))

    def moc_outer_reduced_layout(self, sel_shot, q_tok0, q_tok1):
        """Host only: (chunk_off, chunk_shot, chunk_mod, tok_map) of the reduced stream for one row of sel_shot."""
        sel = np.ascontiguousarray(sel_shot, np.int32).reshape(-1)
        # only what the call fills in is touched, and no part is copied: clearing and copying a map of 264k tokens took longer than making it
        off = np.empty(self.C + 1, np.int32)
        shot = np.empty(self.C, np.int32)
        mod = np.empty(self.C, np.uint8)
        tok = np.empty(self.L, np.int32)
        nc, nt = C.c_int32(0), C.c_int32(0)
        _check(self._lib.moc_outer_reduced_layout(self._h, sel.ctypes.data, len(sel), int(q_tok0), int(q_tok1), C.byref(nc),
                                                  C.byref(nt), off.ctypes.data, shot.ctypes.data, mod.ctypes.data, tok.ctypes.data))
        return off[:nc.value + 1], shot[:nc.value], mod[:nc.value], tok[:nt.value]

    def moc_gather_tokens(self, X, tok_map, out):
        _check(self._lib.moc_gather_tokens(self._h, _ptr(X), _ptr(tok_map), int(tok_map.numel()), _ptr(out), _stream()))

    # test hooks
    def debug_set_wait_limit_us(self, us: int):
        _check(self._lib.moc_debug_set_wait_limit_us(self._h, int(us)))

    def debug_wait_probe(self, ws, code: int, form: int = 0):
        _check(self._lib.moc_debug_wait_probe_form(self._h, _ptr(ws), int(form), int(code), _stream()))

    # convenience: allocate outputs and run the forward path
    def forward(self, Q, K, V, ws=None):
        dev = Q.device
        ws = self.new_workspace(False, dev) if ws is None else ws
        desc = torch.empty((self.H, self.C, self.d), dtype=torch.float32, device=dev)
        sel = torch.empty((self.H, self.L, self.k), dtype=torch.int32, device=dev)
        O = torch.empty_like(Q)
        lse = torch.empty((self.H, self.L), dtype=torch.float32, device=dev)
        self.moc_chunk_pool(K, desc, ws)
        self.moc_route(Q, desc, sel, ws)
        self.moc_attend(Q, K, V, sel, O, lse, ws)
        return desc, sel, O, lse, ws


def _rows(t, heads, tokens, d, dtype, name, dev, spare=False):
    """A [heads][tokens][d] tensor of any strides as the library takes it; `spare`: it may have more tokens."""
    if t is None:
        raise MocError(-1, f"moc error -1: {name} is missing")
    shape = t.shape
    if t.dtype is dtype and t.get_device() == dev and len(shape) == 3 and shape[0] == heads and shape[2] == d and (
            shape[1] == tokens or (spare and shape[1] > tokens)):
        head, tok, one = t.stride()
        if one == 1:
            return _Rows(t.data_ptr(), head, tok)
        raise MocError(-2, f"moc error -2: the channels of {name} are not consecutive")
    _on_current(t, name, dev)
    raise MocError(-2, f"moc error -2: {name} is {t.dtype} {tuple(shape)}, not {dtype} {(heads, tokens, d)}")


def _on_current(t, name, dev):
    if t.get_device() != dev:                                   # (-1 on the CPU)
        raise MocError(-6, f"moc error -6: {name} is on {t.device}, which is not the current device")


def _table(t, shape, dtype, name, dev):
    """The address of a contiguous tensor, or NULL."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise MocError(-2, f"moc error -2: {name} is {t.dtype} {tuple(t.shape)}, not contiguous {dtype} {shape}")
    _on_current(t, name, dev)
    return t.data_ptr()


def _scratch(ws, n_bytes, dev):
    if ws is None or ws.numel() * ws.element_size() < n_bytes or not ws.is_contiguous():
        raise MocError(-5, f"moc error -5: a contiguous workspace of {n_bytes} bytes is needed")
    _on_current(ws, "the workspace", dev)
    return ws.data_ptr()


def debug_rope_split(fp32, bwd, head_dim, n_tokens, n_q, n_k, n_sm=148):
    """Test hook, host only: how a call of MocRope deals out its work on n_sm SMs."""
    out = (C.c_int64 * 7)()
    _check(load_library().moc_debug_rope_split(int(fp32), int(bwd), int(head_dim), int(n_tokens), int(n_q), int(n_k), int(n_sm), out))
    return dict(zip(("by_token", "q_units", "k_units", "per_warp", "n_split", "items", "warps"), out))


class MocRope:
    """Owns a ``moc_rope``: the norm of every query and key head with the position rotation in one pass.  Queries, keys and their
    outputs are [head][token][d] tensors of any strides (the channels consecutive), for instance parts of a fused projection
    [token][head][d], transposed.

    pair_axis, pair_freq: of every turned pair of channels the axis of its position, and radians per step."""

    def __init__(self, head_dim, pair_axis=(), pair_freq=(), n_axes=None, eps=1e-6, halves=False):
        self._lib = load_library()
        self._h = C.c_void_p(0)
        axis = _int32(pair_axis, "pair_axis")
        freq = np.ascontiguousarray(pair_freq, np.float64)
        if axis.shape != freq.shape or axis.ndim != 1:
            raise MocError(-2, "moc error -2: pair_axis and pair_freq are lists of the same length")
        if n_axes is None:
            n_axes = int(axis.max()) + 1 if len(axis) else 0
        pr = _RopeProblem(int(head_dim), len(axis), int(n_axes), 0x1 if halves else 0, float(eps), axis.ctypes.data, freq.ctypes.data)
        _check(self._lib.moc_rope_create(C.byref(pr), C.byref(self._h)))
        self.d, self.n_axes = int(head_dim), int(n_axes) if len(axis) else 0
        n = C.c_size_t(0)
        _check(self._lib.moc_rope_workspace_bytes(self._h, C.byref(n)))
        self._ws_bytes = int(n.value)

    @classmethod
    def from_axes(cls, head_dim, axis_dims, theta=10000.0, **kw):
        """Axis a turns axis_dims[a] channels (an even number), its pair m by theta ** (-2 m / axis_dims[a]) a step; the axes' pairs
        follow one another, and the channels behind them are not turned."""
        if any(int(n) < 0 or int(n) % 2 for n in axis_dims):
            raise MocError(-2, "moc error -2: an axis turns an even number of channels")
        axis = [a for a, n in enumerate(axis_dims) for _ in range(int(n) // 2)]
        freq = [float(theta) ** (-2.0 * m / int(n)) for n in axis_dims for m in range(int(n) // 2)]
        return cls(head_dim, axis, freq, n_axes=len(axis_dims), **kw)

    def close(self):
        if self._h:
            self._lib.moc_rope_destroy(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self) -> int:
        return self._ws_bytes

    def new_workspace(self, device="cuda") -> torch.Tensor:
        return torch.empty(self._ws_bytes, dtype=torch.uint8, device=device)

    def _common(self, pos, q, k, dev):
        if q is None:
            raise MocError(-1, "moc error -1: q is missing")
        if q.dim() != 3 or q.dtype not in (torch.bfloat16, torch.float32):
            raise MocError(-2, f"moc error -2: queries are [head][token][d], bf16 or fp32, not {q.dtype} {tuple(q.shape)}")
        if k is not None and k.dim() != 3:
            raise MocError(-2, f"moc error -2: keys are [head][token][d], not {tuple(k.shape)}")
        hq, L, _ = q.shape
        return (1 if q.dtype is torch.float32 else 0, L, hq, 0 if k is None else k.shape[0],
                _table(pos, (L, self.n_axes), torch.int32, "pos", dev) if self.n_axes else None)

    def moc_norm_rope(self, pos, q, w_q, q_out, k=None, w_k=None, k_out=None):
        """q_out (and k_out) <- norm and rotation of q (and k); pos: int32 [token][axis]; w_q, w_k: fp32 [d], or None for no norm."""
        dev, d, b16, f32 = torch._C._cuda_getDevice(), self.d, torch.bfloat16, torch.float32
        x_type, L, hq, hk, at = self._common(pos, q, k, dev)
        rk = (None,) * 3
        if hk:
            rk = (_rows(k, hk, L, d, q.dtype, "k", dev), _table(w_k, (d,), f32, "w_k", dev), _rows(k_out, hk, L, d, b16, "k_out", dev))
        code = self._lib.moc_norm_rope(self._h, x_type, L, hq, hk, at, _rows(q, hq, L, d, q.dtype, "q", dev), _table(w_q, (d,), f32, "w_q", dev),
                                       _rows(q_out, hq, L, d, b16, "q_out", dev), *rk, torch._C._cuda_getCurrentRawStream(dev))
        if code:
            _check(code)

    def moc_norm_rope_bwd(self, pos, q, w_q, dq_out, dq, dw_q, ws, k=None, w_k=None, dk_out=None, dk=None, dw_k=None):
        """dq, dw_q (and dk, dw_k) <- from dq_out (and dk_out), the gradients of moc_norm_rope's outputs."""
        dev, d, b16, f32 = torch._C._cuda_getDevice(), self.d, torch.bfloat16, torch.float32
        x_type, L, hq, hk, at = self._common(pos, q, k, dev)
        rk = (None,) * 5
        if hk:
            rk = (_rows(k, hk, L, d, q.dtype, "k", dev), _table(w_k, (d,), f32, "w_k", dev), _rows(dk_out, hk, L, d, b16, "dk_out", dev),
                  _rows(dk, hk, L, d, q.dtype, "dk", dev), _table(dw_k, (d,), f32, "dw_k", dev))
        code = self._lib.moc_norm_rope_bwd(self._h, x_type, L, hq, hk, at, _rows(q, hq, L, d, q.dtype, "q", dev), _table(w_q, (d,), f32, "w_q", dev),
                                           _rows(dq_out, hq, L, d, b16, "dq_out", dev), _rows(dq, hq, L, d, q.dtype, "dq", dev),
                                           _table(dw_q, (d,), f32, "dw_q", dev), *rk, _scratch(ws, self._ws_bytes, dev),
                                           torch._C._cuda_getCurrentRawStream(dev))
        if code:
            _check(code)


def _int32(values, name):
    """A table of whole numbers for the library; one that does not fit is refused, where a cast would wrap or cut it."""
    t = np.asarray(values)
    if t.size and (t.dtype.kind not in "biuf" or not (t.min() >= -2**31 and t.max() < 2**31) or (t != np.floor(t)).any()):
        raise MocError(-2, f"moc error -2: {name} is a list of whole numbers below 2^31")
    return np.ascontiguousarray(t, np.int32)


def _cross_problem(n_heads, n_kv_heads, head_dim, q_off, k_off, k_len, softmax_scale):
    """The C problem statement, and the host arrays it points to."""
    qo, ko = _int32(q_off, "q_off"), _int32(k_off, "k_off")
    kl = None if k_len is None else _int32(k_len, "k_len")
    if qo.ndim != 1 or len(qo) < 1 or ko.shape != qo.shape or (kl is not None and kl.shape != (len(qo) - 1,)):
        raise MocError(-3, "moc error -3: segment tables have inconsistent lengths")
    pr = _CrossProblem(int(n_heads), int(n_kv_heads), int(head_dim), len(qo) - 1, float(softmax_scale), qo.ctypes.data, ko.ctypes.data,
                       None if kl is None else kl.ctypes.data)
    return pr, (qo, ko, kl)


def debug_cross_plan(n_heads, n_kv_heads, head_dim, q_off, k_off, k_len=None, n_sm=148):
    """Test hook, host only: what MocCross of the same arguments launches on n_sm SMs: items of the forward's three kernels, rows of
    partial results, items of dQ, pieces of dK/dV and slots of their sums; key tiles that a CTA walks at most and in the mean."""
    pr, tables = _cross_problem(n_heads, n_kv_heads, head_dim, q_off, k_off, k_len, 0.0)
    out = (C.c_int64 * 14)()
    _check(load_library().moc_debug_cross_plan(C.byref(pr), int(n_sm), out))
    return dict(zip(("two_tile", "one_tile", "few", "part_rows", "dq", "pieces", "slots", "two_tile_walk", "two_tile_mean", "one_tile_walk",
                     "one_tile_mean", "dq_walk", "dq_mean", "two_tile_wait"), out))


class MocCross:
    """Owns a ``moc_cross``: attention of a stream's segments (shots, or sequences of a batch) to encoder states of another
    length.  q_off, k_off: [segments + 1] where each segment's queries and states begin; k_len: how many of them it has
    (default: up to the next one's).  Tensors are [head][token][d], bf16, of any strides (the channels consecutive)."""

    def __init__(self, n_heads, n_kv_heads, head_dim, q_off, k_off, k_len=None, softmax_scale=0.0):
        self._lib = load_library()
        self._h = C.c_void_p(0)
        pr, (qo, ko, _) = _cross_problem(n_heads, n_kv_heads, head_dim, q_off, k_off, k_len, softmax_scale)
        _check(self._lib.moc_cross_create(C.byref(pr), C.byref(self._h)))
        self.H, self.Hkv, self.d = int(n_heads), int(n_kv_heads), int(head_dim)
        self.n_queries, self.n_states = int(qo[-1]), int(ko[-1])
        self._ws_bytes = []
        for with_bwd in (0, 1):
            n = C.c_size_t(0)
            _check(self._lib.moc_cross_workspace_bytes(self._h, with_bwd, C.byref(n)))
            self._ws_bytes.append(int(n.value))

    def close(self):
        if self._h:
            self._lib.moc_cross_destroy(self._h)
            self._h = C.c_void_p(0)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def workspace_bytes(self, with_bwd=False) -> int:
        return self._ws_bytes[1 if with_bwd else 0]

    def new_workspace(self, with_bwd=False, device="cuda") -> torch.Tensor:
        return torch.empty(self.workspace_bytes(with_bwd), dtype=torch.uint8, device=device)

    # (tensors may have more rows than the segments: those behind the last one's are left alone)
    def moc_cross_attend(self, Q, K, V, O, lse, ws):
        """O, lse (fp32 [head][query]) <- attention of every segment's queries to its states."""
        dev, H, kv, n, m, d, b16 = torch._C._cuda_getDevice(), self.H, self.Hkv, self.n_queries, self.n_states, self.d, torch.bfloat16
        code = self._lib.moc_cross_attend(self._h, _rows(Q, H, n, d, b16, "Q", dev, True), _rows(K, kv, m, d, b16, "K", dev, True),
                                          _rows(V, kv, m, d, b16, "V", dev, True), _rows(O, H, n, d, b16, "O", dev, True),
                                          _table(lse, (H, n), torch.float32, "lse", dev), _scratch(ws, self._ws_bytes[0], dev),
                                          torch._C._cuda_getCurrentRawStream(dev))
        if code:
            _check(code)

    def moc_cross_attend_bwd(self, Q, K, V, O, lse, dO, dQ, dK, dV, ws):
        """dQ, dK, dV <- from dO, the gradient of O; O, lse: the forward's."""
        dev, H, kv, n, m, d, b16 = torch._C._cuda_getDevice(), self.H, self.Hkv, self.n_queries, self.n_states, self.d, torch.bfloat16
        code = self._lib.moc_cross_attend_bwd(self._h, _rows(Q, H, n, d, b16, "Q", dev, True), _rows(K, kv, m, d, b16, "K", dev, True),
                                              _rows(V, kv, m, d, b16, "V", dev, True), _rows(O, H, n, d, b16, "O", dev, True),
                                              _table(lse, (H, n), torch.float32, "lse", dev), _rows(dO, H, n, d, b16, "dO", dev, True),
                                              _rows(dQ, H, n, d, b16, "dQ", dev, True), _rows(dK, kv, m, d, b16, "dK", dev, True),
                                              _rows(dV, kv, m, d, b16, "dV", dev, True), _scratch(ws, self._ws_bytes[1], dev),
                                              torch._C._cuda_getCurrentRawStream(dev))
        if code:
            _check(code)

    def moc_cross_get_status(self, ws):
        st, det = C.c_int(0), C.c_int(0)
        _check(self._lib.moc_cross_get_status(self._h, _ptr(ws), _stream(), C.byref(st), C.byref(det)))
        return int(st.value), int(det.value)
