"""Binding of libmate.so (same names as the C entry points; marshalling only): ctypes for what is called
once per plan, a native module (csrc/binding.cpp) for what is called once per layer."""
import ctypes as C
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libmate.so")

IMPL_AUTO, IMPL_SIMT, IMPL_TCGEN05 = 0, 1, 2
FLAG_VIEW_ORDER, FLAG_BULK_TILES, FLAG_GATHER_TILES = 4, 8, 16   # or-ed to the implementation choice (see mate.h)
VIEW_ROW, VIEW_COL, VIEW_EITHER = 0, 1, 2   # (either: of a Cache only)
ID_TEXT = 0x7FFFFFFF   # ids of a cached or new token that belongs to the text, wherever it stands (see mate.h)
_BF16, _F32 = 0, 1

_lib = None
_cache_calls = None   # the native module, once the library is loaded


class MateError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (where, _status_string(status), status))


def library_path() -> str:
    """MATE_LIB (read when the library is first loaded) selects another build of the same library:
    the profiling build, libmate_trace.so."""
    return os.environ.get("MATE_LIB") or _LIB_PATH


def _load():
    """Loads the CUDA library; there is no fallback: a missing library is an error."""
    global _lib, _cache_calls
    if _lib is not None:
        return _lib
    path = library_path()
    if not os.path.exists(path):
        raise ImportError(
            "libmate.so is not built: run `python -m paper_2109_04312_b200.build` "
            "(needs nvcc); there is no CPU or PyTorch fallback")
    lib = C.CDLL(path)
    vp, i32, u32, f32, sz = C.c_void_p, C.c_int, C.c_uint, C.c_float, C.c_size_t
    lib.mate_status_string.restype = C.c_char_p
    lib.mate_status_string.argtypes = [i32]
    lib.mate_plan.restype = i32
    lib.mate_plan.argtypes = [vp, vp, i32, i32, i32, vp, i32, i32, i32, vp, C.POINTER(vp)]
    lib.mate_plan_bucketed.restype = i32
    lib.mate_plan_bucketed.argtypes = [vp, vp, i32, i32, i32, vp, i32, i32, i32, i32, vp, C.POINTER(vp)]
    lib.mate_plan_varlen.restype = i32
    lib.mate_plan_varlen.argtypes = [vp, vp, i32, i32, vp, vp, i32, i32, i32, i32, vp, C.POINTER(vp)]
    lib.mate_plan_packed.restype = i32
    lib.mate_plan_packed.argtypes = [vp, vp, i32, vp, vp, vp, i32, i32, i32, vp, C.POINTER(vp)]
    lib.mate_plan_bucketed_global.restype = i32
    lib.mate_plan_bucketed_global.argtypes = [vp, vp, i32, i32, vp, vp, vp, i32, i32, i32, i32, vp, C.POINTER(vp)]
    lib.mate_plan_sat.restype = i32
    lib.mate_plan_sat.argtypes = [vp, vp, i32, i32, i32, i32, i32, i32, vp, C.POINTER(vp)]
    lib.mate_plan_get.restype = i32
    lib.mate_plan_get.argtypes = [vp, i32, vp, vp, vp]
    lib.mate_plan_useful_pairs.restype = i32
    lib.mate_plan_useful_pairs.argtypes = [vp, vp]
    lib.mate_plan_status.restype = i32
    lib.mate_plan_status.argtypes = [vp, vp]
    lib.mate_debug_expire_wait.restype = i32
    lib.mate_debug_expire_wait.argtypes = [vp, vp]
    lib.mate_plan_destroy.restype = i32
    lib.mate_plan_destroy.argtypes = [vp]
    lib.mate_attn_workspace_bytes.restype = i32
    lib.mate_attn_workspace_bytes.argtypes = [vp, i32, i32, u32, C.POINTER(sz), C.POINTER(sz)]
    lib.mate_attn_fwd.restype = i32
    lib.mate_attn_fwd.argtypes = [vp, vp, vp, vp, i32, i32, f32, vp, vp, vp, sz, u32, vp]
    lib.mate_attn_bwd.restype = i32
    lib.mate_attn_bwd.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, vp, vp, vp, vp, sz, u32, vp]
    lib.mate_cell_mean.restype = i32
    lib.mate_cell_mean.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.mate_attn_bwd_noalloc.restype = i32
    lib.mate_attn_bwd_noalloc.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, f32, vp, vp, vp, vp]
    try:
        from . import _native
    except ImportError as e:
        raise ImportError("the native binding is not built: run `python -m paper_2109_04312_b200.build`") from e
    _native.bind(*(C.cast(f, C.c_void_p).value for f in (lib.mate_attn_workspace_bytes, lib.mate_attn_fwd,
                                                         lib.mate_attn_bwd, lib.mate_cell_mean)), MateError)
    entries = (lib.mate_rope, lib.mate_cache_extend, lib.mate_cache_append, lib.mate_cache_fork, lib.mate_cache_free,
               lib.mate_cache_compact, lib.mate_cache_workspace_bytes, lib.mate_cache_status, lib.mate_attn_decode)
    _native.bind_cache(*(C.cast(f, C.c_void_p).value for f in entries))
    _cache_calls = _native
    _lib = lib
    return lib


def _status_string(status):
    try:
        return _load().mate_status_string(status).decode()
    except Exception:
        return "?"


def _check(status, where):
    if status != 0:
        raise MateError(status, where)


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return _BF16
    if t.dtype == torch.float32:
        return _F32
    raise TypeError("libmate takes bfloat16 or float32 tensors, got %s" % t.dtype)


def _dev(t, name):
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.is_contiguous()):
        raise ValueError("%s must be a contiguous CUDA tensor" % name)
    return C.c_void_p(t.data_ptr())


class Plan:
    """Owner of a mate_plan_t*: the pre-computed per-view order (see mate_plan)."""

    def __init__(self, handle, B, N, P, H, max_row_id, max_col_id, device, T=None):
        self._h = handle
        self.B, self.N, self.P, self.H = B, N, P, H
        self.max_id = (max_row_id, max_col_id)
        self.device = device
        self.T = T             # packed plans: total number of tokens (tensors are [H, T, d])
        from . import _native
        self._native = _native
        # what the native calls need of the plan, and the workspaces they keep for it
        self._info = _native.plan_info(handle.value, B, N, H, -1 if T is None else T, max_row_id + 1, max_col_id + 1,
                                       device.index if device.index is not None else torch.cuda.current_device())

    def _split(self, Q):
        """Checks a tensor's shape against the plan; returns (d, shape of the row statistic)."""
        if self.T is not None:
            if Q.dim() != 3 or tuple(Q.shape[:2]) != (self.H, self.T):
                raise ValueError("a packed plan takes [H, T, d] tensors")
            return Q.shape[2], (self.H, self.T)
        if Q.dim() != 4 or tuple(Q.shape[:3]) != (self.B, self.H, self.N):
            raise ValueError("tensor shapes do not match the plan")
        return Q.shape[3], (self.B, self.H, self.N)

    def get(self, view):
        """(perm, inv_perm, seg_off) of one view as numpy int32 arrays."""
        perm = np.empty((self.B, self.N), np.int32)
        inv = np.empty((self.B, self.N), np.int32)
        seg = np.empty((self.B, self.max_id[view] + 2), np.int32)
        _check(_load().mate_plan_get(self._h, view, perm.ctypes.data, inv.ctypes.data, seg.ctypes.data),
               "mate_plan_get")
        return perm, inv, seg

    def useful_pairs(self):
        out = np.empty((self.B, self.H), np.int64)
        _check(_load().mate_plan_useful_pairs(self._h, out.ctypes.data), "mate_plan_useful_pairs")
        return out

    def status(self):
        _check(_load().mate_plan_status(self._h, _stream()), "mate_plan_status")

    def debug_expire_wait(self):
        """Test hook: makes a bounded device wait give up (see mate_debug_expire_wait in mate.h)."""
        _check(_load().mate_debug_expire_wait(self._h, _stream()), "mate_debug_expire_wait")

    def destroy(self):
        if self._h is not None:
            self._native.drop(self._info)
            _lib.mate_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass


def mate_plan_bucketed(row_ids, col_ids, prefix_len, head_view, radius, max_row_id=None, max_col_id=None) -> Plan:
    """Plan of the bucketed variant (see mate_plan_bucketed in mate.h); radius = 0 is the exact pattern."""
    return mate_plan(row_ids, col_ids, prefix_len, head_view, max_row_id, max_col_id, radius=radius)


def mate_plan_packed(row_ids, col_ids, cu_seqlens, prefix_lens, head_view, max_row_id=None, max_col_id=None) -> Plan:
    """Plan of a packed batch (see mate_plan_packed in mate.h): row_ids, col_ids are int32 CUDA tensors [T],
    example b owning the tokens cu_seqlens[b] .. cu_seqlens[b + 1] - 1; Q, K, V, O and the gradients are then
    [H, T, d] and LSE is [H, T]."""
    if row_ids.dtype != torch.int32 or col_ids.dtype != torch.int32 or row_ids.shape != col_ids.shape \
            or row_ids.dim() != 1:
        raise ValueError("row_ids / col_ids must be int32 tensors of the same [T] shape")
    cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
    pf = np.ascontiguousarray(np.asarray(prefix_lens, dtype=np.int32))
    B = int(pf.shape[0])
    if cu.shape != (B + 1,) or int(cu[-1]) != int(row_ids.shape[0]):
        raise ValueError("cu_seqlens must have B + 1 entries and end at T")
    hv = np.ascontiguousarray(np.asarray(head_view, dtype=np.uint8))
    if max_row_id is None:
        max_row_id = max(int(row_ids.max().item()), 0) if row_ids.numel() else 0
    if max_col_id is None:
        max_col_id = max(int(col_ids.max().item()), 0) if col_ids.numel() else 0
    handle = C.c_void_p()
    with torch.cuda.device(row_ids.device):
        _check(_load().mate_plan_packed(_dev(row_ids, "row_ids"), _dev(col_ids, "col_ids"), B, cu.ctypes.data,
                                        pf.ctypes.data, hv.ctypes.data, int(hv.shape[0]), int(max_row_id),
                                        int(max_col_id), _stream(), C.byref(handle)), "mate_plan_packed")
    n_max = max(int(np.diff(cu).max()), 1)
    return Plan(handle, B, n_max, pf.tolist(), int(hv.shape[0]), int(max_row_id), int(max_col_id), row_ids.device,
                T=int(cu[-1]))


def mate_plan_varlen(row_ids, col_ids, prefix_lens, head_view, radius=0, max_row_id=None, max_col_id=None) -> Plan:
    """Plan with one prefix length per example (see mate_plan_varlen in mate.h): prefix_lens has B entries."""
    return mate_plan(row_ids, col_ids, [int(x) for x in prefix_lens], head_view, max_row_id, max_col_id,
                     radius=radius)


def mate_plan(row_ids, col_ids, prefix_len, head_view, max_row_id=None, max_col_id=None, radius=0) -> Plan:
    """row_ids, col_ids: int32 CUDA tensors [B, N]; head_view: sequence of 0 (row) / 1 (column);
    prefix_len: one int, or a list of B ints (one per example)."""
    if row_ids.dtype != torch.int32 or col_ids.dtype != torch.int32 or row_ids.shape != col_ids.shape \
            or row_ids.dim() != 2:
        raise ValueError("row_ids / col_ids must be int32 tensors of the same [B, N] shape")
    B, N = row_ids.shape
    hv = np.ascontiguousarray(np.asarray(head_view, dtype=np.uint8))
    if max_row_id is None:
        max_row_id = max(int(row_ids.max().item()), 0)
    if max_col_id is None:
        max_col_id = max(int(col_ids.max().item()), 0)
    handle = C.c_void_p()
    with torch.cuda.device(row_ids.device):
        lib = _load()
        common = (_dev(row_ids, "row_ids"), _dev(col_ids, "col_ids"), B, N)
        tail = (hv.ctypes.data, int(hv.shape[0]), int(max_row_id), int(max_col_id))
        if isinstance(prefix_len, (list, tuple, np.ndarray)):
            pf = np.ascontiguousarray(np.asarray(prefix_len, dtype=np.int32))
            if pf.shape != (B,):
                raise ValueError("prefix_len must have one entry per example")
            _check(lib.mate_plan_varlen(*common, pf.ctypes.data, *tail, int(radius), _stream(), C.byref(handle)),
                   "mate_plan_varlen")
            prefix_len = pf.tolist()
        elif radius:
            _check(lib.mate_plan_bucketed(*common, int(prefix_len), *tail, int(radius), _stream(),
                                          C.byref(handle)), "mate_plan_bucketed")
        else:
            _check(lib.mate_plan(*common, int(prefix_len), *tail, _stream(), C.byref(handle)), "mate_plan")
    return Plan(handle, B, N, prefix_len, int(hv.shape[0]), int(max_row_id), int(max_col_id), row_ids.device)


def mate_plan_bucketed_global(row_ids, col_ids, prefix_lens, global_lens, head_view, radius, max_row_id=None,
                              max_col_id=None) -> Plan:
    """Bucketed plan whose global section (global_lens[b] >= prefix_lens[b] positions of every head's own order)
    may reach beyond the prefix (see mate_plan_bucketed_global in mate.h).  Scalars are taken for every example."""
    B, N = row_ids.shape
    pf = np.ascontiguousarray(np.broadcast_to(np.asarray(prefix_lens, dtype=np.int32), (B,)))
    gl = np.ascontiguousarray(np.broadcast_to(np.asarray(global_lens, dtype=np.int32), (B,)))
    hv = np.ascontiguousarray(np.asarray(head_view, dtype=np.uint8))
    if max_row_id is None:
        max_row_id = max(int(row_ids.max().item()), 0)
    if max_col_id is None:
        max_col_id = max(int(col_ids.max().item()), 0)
    handle = C.c_void_p()
    with torch.cuda.device(row_ids.device):
        _check(_load().mate_plan_bucketed_global(_dev(row_ids, "row_ids"), _dev(col_ids, "col_ids"), B, N, pf.ctypes.data,
                                                 gl.ctypes.data, hv.ctypes.data, int(hv.shape[0]), int(max_row_id),
                                                 int(max_col_id), int(radius), _stream(), C.byref(handle)),
               "mate_plan_bucketed_global")
    return Plan(handle, B, N, pf.tolist(), int(hv.shape[0]), int(max_row_id), int(max_col_id), row_ids.device)


def mate_plan_sat(row_ids, col_ids, prefix_len, n_heads, max_row_id=None, max_col_id=None) -> Plan:
    """Plan of the head-independent row-or-column pattern (see mate_plan_sat in mate.h)."""
    if row_ids.dtype != torch.int32 or col_ids.dtype != torch.int32 or row_ids.shape != col_ids.shape \
            or row_ids.dim() != 2:
        raise ValueError("row_ids / col_ids must be int32 tensors of the same [B, N] shape")
    B, N = row_ids.shape
    if max_row_id is None:
        max_row_id = max(int(row_ids.max().item()), 0)
    if max_col_id is None:
        max_col_id = max(int(col_ids.max().item()), 0)
    handle = C.c_void_p()
    with torch.cuda.device(row_ids.device):
        _check(_load().mate_plan_sat(_dev(row_ids, "row_ids"), _dev(col_ids, "col_ids"), B, N, int(prefix_len),
                                     int(n_heads), int(max_row_id), int(max_col_id), _stream(), C.byref(handle)),
               "mate_plan_sat")
    return Plan(handle, B, N, prefix_len, int(n_heads), int(max_row_id), int(max_col_id), row_ids.device)


def mate_attn_workspace_bytes(plan, d, dtype, impl=IMPL_AUTO):
    f, b = C.c_size_t(0), C.c_size_t(0)
    _check(_load().mate_attn_workspace_bytes(plan._h, int(d), dtype, impl, C.byref(f), C.byref(b)),
           "mate_attn_workspace_bytes")
    return f.value, b.value


def mate_attn_fwd(plan, Q, K, V, scale=None, impl=IMPL_AUTO, out=None, lse=None, workspace=None):
    """Q, K, V: [B, H, N, d] CUDA tensors (bf16 or f32), or [H, T, d] for a packed plan.  Returns (O, LSE)
    in original token order."""
    return plan._native.attn_fwd(plan._info, Q, K, V, scale, impl, out, lse, workspace)


def mate_attn_bwd(plan, Q, K, V, O, LSE, dO, scale=None, impl=IMPL_AUTO, workspace=None):
    """Returns (dQ, dK, dV)."""
    return plan._native.attn_bwd(plan._info, Q, K, V, O, LSE, dO, scale, impl, workspace)


def mate_cell_mean(plan, logits, col_ids, want_count=True, out=None):
    """Mean of the token logits per table cell (see mate_cell_mean in mate.h).  logits: float32 [B, N];
    col_ids: the int32 [B, N] tensor the plan was made from.  Returns (mean, count) of shape
    [B, max_row_id + 1, max_col_id + 1] (count is None when not wanted).  out: (mean, count) tensors of an
    earlier call, written in place."""
    mean, count = (None, None) if out is None else out
    return plan._native.cell_mean(plan._info, logits, col_ids, want_count, mean, count)


def mate_attn_bwd_noalloc(plan, Q, K, V, O, LSE, dO, dQ, dK, dV, scale=None):
    """Backward for callers that may not allocate device memory (for example inside a loop whose
    framework owns every byte of the device): the caller passes the three output tensors and the
    library uses its built-in scratch array, so neither this function nor the C entry point
    allocates anything.  B*H*N is limited to 1,048,576.  Calls must not overlap on the GPU."""
    d, _ = plan._split(Q)
    for t in (K, V, O, dO, dQ, dK, dV):
        if t.shape != Q.shape or t.dtype != Q.dtype:
            raise ValueError("K, V, O, dO, dQ, dK, dV must match Q in shape and dtype")
    if LSE.dtype != torch.float32 or LSE.numel() * d < Q.numel():
        raise ValueError("LSE must be a float32 tensor with one element per row")
    if scale is None:
        scale = 1.0 / float(d) ** 0.5
    with torch.cuda.device(Q.device):
        _check(_load().mate_attn_bwd_noalloc(plan._h, _dev(Q, "Q"), _dev(K, "K"), _dev(V, "V"),
                                             _dev(O, "O"), _dev(LSE, "LSE"), _dev(dO, "dO"), d,
                                             _dtype_code(Q), float(scale), _dev(dQ, "dQ"),
                                             _dev(dK, "dK"), _dev(dV, "dV"), _stream()),
               "mate_attn_bwd_noalloc")
    return dQ, dK, dV


def mate_rope_freqs(rot, base=10000.0, factor=1.0, original_len=None, low=1.0, high=4.0, device="cuda"):
    """Radians per position of the rot / 2 pairs, base ** (-2 i / rot), as a float64 tensor.  factor stretches them for contexts
    `factor` times as long: all of them, or, where original_len is given, by how often a pair turns within it -- those with at least
    `high` turns are kept, those with at most `low` are stretched, between them the two are mixed."""
    if rot < 0 or rot % 2 or not factor > 0 or not high > low:
        raise ValueError("rot must be even, factor positive, high larger than low")
    f = base ** (-np.arange(0, rot, 2, dtype=np.float64) / max(rot, 1))
    keep = 0.0 if original_len is None else np.clip((original_len * f / (2 * np.pi) - low) / (high - low), 0.0, 1.0)
    return torch.from_numpy(f * keep + f / factor * (1 - keep)).to(device)


def mate_rope(Q, positions, freqs, K=None, interleaved=False, mscale=1.0, backward=False, out=None):
    """Rotary positions (see mate_rope in mate.h).  Q, and K with heads of its own: [B, H, N, d] (or [H, T, d]) CUDA tensors, bf16 or
    f32, of any strides with contiguous rows, for example views of a fused projection's output.  positions: int32 [B, N], or [N] for
    all examples; freqs: float64 [rot / 2] (mate_rope_freqs).  backward: gradients of the inputs from those of the outputs.
    out: where the result goes (a pair with K), any strides: the inputs themselves, or tensors that share no memory with them or with
    one another; else new contiguous tensors.  Returns Q' or (Q', K')."""
    if _lib is None:
        _load()
    if K is not None and out is not None and not (isinstance(out, (tuple, list)) and len(out) == 2):
        raise ValueError("out must be a pair of tensors where Q and K are given")
    q, k = (out, None) if K is None else out or (None, None)
    return _cache_calls.rope(Q, K, positions, freqs, interleaved, mscale, backward, q, k)


class Cache:
    """A paged cache of keys and values (see mate_cache_t in mate.h): the caller's tensors, which the calls read and write.

    k, v: [layers, pages, kv_heads, page_size, d] bf16 or f32 (a cache laid out slot by slot is passed as a transposed view);
    row_ids, col_ids: int32 [pages, page_size]; table: int32 [seqs, width]; lens, prefix: int32 [seqs]; refs: int32 [pages];
    head_view: VIEW_ROW, VIEW_COL or VIEW_EITHER for every query head.  The calls go by the tensors given here: change them in
    place (cache.prefix[s] = 128), not for others."""

    def __init__(self, k, v, row_ids, col_ids, table, lens, prefix, refs, head_view):
        _load()
        self.k, self.v, self.row_ids, self.col_ids = k, v, row_ids, col_ids
        self.table, self.lens, self.prefix, self.refs = table, lens, prefix, refs
        self.head_view = np.ascontiguousarray(np.asarray(head_view, dtype=np.uint8))
        self.status_word = torch.zeros(1, dtype=torch.int32, device=k.device)
        self._native = _cache_calls
        self._info = _cache_calls.cache_info(k, v, row_ids, col_ids, table, lens, prefix, refs, self.status_word, self.head_view.tobytes())

    @classmethod
    def empty(cls, pages, page_size, kv_heads, d, seqs, width, head_view, layers=1, dtype=torch.bfloat16, device="cuda"):
        """A cache without a token: `pages` pages of `page_size` slots, up to `seqs` sequences of up to `width` pages."""
        def ints(*shape, value=0):
            return torch.full(shape, value, dtype=torch.int32, device=device)
        k, v = (torch.zeros((layers, pages, kv_heads, page_size, d), dtype=dtype, device=device) for _ in range(2))
        return cls(k, v, ints(pages, page_size), ints(pages, page_size), ints(seqs, width, value=-1), ints(seqs), ints(seqs), ints(pages),
                   head_view)

    def status(self):
        """Waits, and raises MateError if a call found something out of range, or no free page, since the last time."""
        self._native.cache_status(self._info)


def mate_cache_extend(cache, seqs, counts, granted=None):
    """Room for counts[i] more tokens of sequence seqs[i] (None: i): pages are handed out and lens grow (see
    mate_cache_extend in mate.h).  int32 CUDA tensors [n].  Returns granted: counts[i], or 0 where there was no room."""
    return cache._native.cache_extend(cache._info, seqs, counts, granted)


def mate_cache_append(cache, K, V, seqs=None, counts=None, row_ids=None, col_ids=None, layer=0, freqs=None, positions=None,
                      interleaved=False, mscale=1.0, Q=None, out=None):
    """The last counts[i] (None: N) tokens of sequence seqs[i] (None: i) into one layer of the cache (see mate_cache_append in mate.h).
    K, V: [B, kv_heads, N, d] with contiguous rows; row_ids, col_ids: int32 [B, N], None for further layers.  With freqs
    K is rotated on the way, and Q [B, heads, N, d] too, which is returned (out: where it goes, Q itself or a tensor that shares no
    memory with Q, K and V)."""
    return cache._native.cache_append(cache._info, layer, K, V, seqs, counts, row_ids, col_ids, positions, freqs, interleaved, mscale, Q,
                                      out)


def mate_cache_fork(cache, parents, children):
    """children[i], which must be empty, becomes a copy of parents[i]: full pages are shared, a last one that is filled in part is
    copied in all layers (see mate_cache_fork in mate.h).  int32 CUDA tensors [n]."""
    cache._native.cache_fork(cache._info, parents, children)


def mate_cache_free(cache, seqs=None):
    """The sequences (None: all) become empty, their pages lose a reference (see mate_cache_free in mate.h)."""
    cache._native.cache_free(cache._info, seqs)


def mate_cache_compact(cache, n_live=None):
    """Moves the pages in use to the front (see mate_cache_compact in mate.h); returns their number, an int32 CUDA tensor."""
    return cache._native.cache_compact(cache._info, n_live)


def mate_attn_decode(cache, Q, row_ids, col_ids, seqs=None, layer=0, scale=None, max_len=None, out=None, lse=None):
    """Attention of one new token per sequence over what is cached (see mate_attn_decode in mate.h).  Q: [B, heads, d]; row_ids,
    col_ids: int32 [B], the new tokens' ids (ID_TEXT: text, and new tokens of the prefix); seqs: int32 [B] (None: 0 .. B - 1);
    max_len: an upper bound of the sequences' lengths, by which the work is split (None: what the table holds, which short sequences
    in a wide table pay for).  out, lse: where the results go, contiguous (out may be Q itself; otherwise they share no memory).
    Returns (O, LSE)."""
    return cache._native.attn_decode(cache._info, layer, Q, seqs, row_ids, col_ids, scale, max_len, out, lse)
