"""Thin ctypes binding of libdynakv.so: same names as the C ABI, argument marshalling only.

torch owns device memory and streams; every step of the path runs in the library's kernels.  There is
no fallback: if the library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdynakv.so")

DTYPES = {"f32": 0, "f16": 1, "bf16": 2}
TORCH_DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
ERR_TOKENS, ERR_CLUSTERS, ERR_SPLIT_SIZE, ERR_SELECT, ERR_INIT, ERR_IMPORT, ERR_PLACE = 1, 2, 4, 8, 16, 32, 64
OK, EINVAL, ECAPACITY, ESTATE, EHIP, ENOMEM = range(6)
SEARCH_STORAGE, SEARCH_MEAN = 0, 1
UPDATE_ADAPTIVE, UPDATE_STATIC, UPDATE_TOKENS, UPDATE_LOCAL = 0, 1, 2, 3
LAUNCH_SEPARATE, LAUNCH_SPLIT_KERNEL = 1 << 16, 1 << 17


def launch_shape(kv_splits: int = 0, att_waves: int = 0, flags: int = 0) -> int:
    """The value of Config.launch (DYNAKV_LAUNCH in the header)."""
    return (kv_splits & 255) | ((att_waves & 255) << 8) | flags


class _Cfg(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("n_units", "group_size", "head_dim", "dtype", "n_clusters_init",
                                          "max_clusters", "max_tokens", "kmeans_iters", "buffer_max",
                                          "group_reduce")] + \
               [(k, C.c_float) for k in ("var_alpha", "size_factor", "softmax_scale")] + \
               [(k, C.c_int32) for k in ("search_copy", "score_round", "update_mode", "launch", "local_window", "local_clusters")]


_STATE_FIELDS = ("n_clusters", "n_tokens", "error", "tau", "centroids", "size", "buffered", "flag", "m2", "offsets",
                 "members", "scores", "n_selected", "selected", "n_gathered", "gathered", "last_assign", "counters",
                 "keys", "values", "first_page")
# what dynakv_import_state reads
IMPORT_FIELDS = ("n_clusters", "n_tokens", "tau", "centroids", "size", "buffered", "flag", "m2", "offsets", "members",
                 "keys", "values", "n_selected", "selected")


class _State(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in _STATE_FIELDS]


class _Heads(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("dtype", "n_seqs", "n_tokens", "n_kv_heads", "group_size", "head_dim", "rotary_dim",
                                          "interleaved")] + [("eps", C.c_float)] + \
               [(k, C.c_int64) for k in ("q_seq_stride", "q_token_stride", "k_seq_stride", "k_token_stride", "v_seq_stride",
                                          "v_token_stride")]


class _Packed(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("n_units", "capacity", "head_dim", "dtype", "bits")] + \
               [(k, C.c_void_p) for k in ("k_codes", "k_scales", "v_codes", "v_scales")]


@dataclass
class Config:
    n_units: int
    group_size: int
    dtype: str
    n_clusters_init: int
    max_clusters: int
    max_tokens: int
    kmeans_iters: int = 10
    buffer_max: int = 16
    group_reduce: int = 0
    var_alpha: float = 0.0
    size_factor: float = 0.0
    softmax_scale: float = 0.0
    head_dim: int = 128
    search_copy: int = SEARCH_STORAGE
    score_round: int = 0
    update_mode: int = UPDATE_ADAPTIVE
    launch: int = 0
    local_window: int = 0
    local_clusters: int = 0


_lib = None


def load():
    """Loads the built library; raises if it is missing (build it with paper_2511_07427_amd/build.py)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("libdynakv.so is not built: run `python paper_2511_07427_amd/build.py`")
        lib = C.CDLL(LIB_PATH)
        vp, i32 = C.c_void_p, C.c_int32
        lib.dynakv_workspace_bytes.restype = C.c_size_t
        lib.dynakv_workspace_bytes.argtypes = [C.POINTER(_Cfg)]
        lib.dynakv_create.argtypes = [C.POINTER(_Cfg), vp, C.c_size_t, C.POINTER(vp)]
        lib.dynakv_destroy.argtypes = [vp]
        lib.dynakv_build_index.argtypes = [vp, vp, vp, i32, vp, vp]
        lib.dynakv_extend_index.argtypes = [vp, vp, vp, i32, vp]
        lib.dynakv_place_by_coretrieval.argtypes = [vp, vp, vp, i32, vp, i32, i32, vp, vp, vp]
        lib.dynakv_retrieve_attend.argtypes = [vp, vp, i32, vp, vp, vp]
        lib.dynakv_retrieve_attend_static.argtypes = [vp, vp, i32, vp, vp, vp]
        lib.dynakv_append.argtypes = [vp, vp, vp, vp]
        lib.dynakv_split.argtypes = [vp, vp]
        lib.dynakv_decode_step.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp]
        lib.dynakv_export_state.argtypes = [vp, C.POINTER(_State), vp]
        lib.dynakv_import_state.argtypes = [vp, C.POINTER(_State), vp]
        lib.dynakv_norm_rope.argtypes = [C.POINTER(_Heads)] + [vp] * 11
        lib.dynakv_packed_write.argtypes = [C.POINTER(_Packed), vp, vp, i32, vp, vp, vp]
        lib.dynakv_packed_read.argtypes = [C.POINTER(_Packed), vp, i32, vp, vp, vp]
        lib.dynakv_tree_scratch_bytes.restype = C.c_size_t
        lib.dynakv_tree_scratch_bytes.argtypes = [i32, i32, i32]
        lib.dynakv_attend_tree.argtypes = [vp, vp, i32, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        lib.dynakv_packed_attend.argtypes = [C.POINTER(_Packed), vp, vp, i32, i32, vp, vp, vp, C.c_float, vp, vp, vp, C.c_size_t, vp]
        lib.dynakv_profile_enable.argtypes = [vp, i32]
        lib.dynakv_profile_sample.argtypes = [vp, i32, i32]
        lib.dynakv_profile_read.argtypes = [vp, C.POINTER(i32), C.POINTER(C.c_double)]
        lib.dynakv_profiled_kernel.restype = C.c_char_p
        lib.dynakv_profiled_kernel.argtypes = [vp]
        lib.dynakv_strerror.restype = C.c_char_p
        lib.dynakv_strerror.argtypes = [C.c_int]
        _lib = lib
    return _lib


def _check(rc, what):
    if rc != 0:
        raise RuntimeError("%s: %s" % (what, load().dynakv_strerror(rc).decode()))


def _cfg(cfg: Config) -> _Cfg:
    return _Cfg(cfg.n_units, cfg.group_size, cfg.head_dim, DTYPES[cfg.dtype], cfg.n_clusters_init, cfg.max_clusters,
                cfg.max_tokens, cfg.kmeans_iters, cfg.buffer_max, cfg.group_reduce, cfg.var_alpha, cfg.size_factor,
                cfg.softmax_scale, cfg.search_copy, cfg.score_round, cfg.update_mode, cfg.launch, cfg.local_window,
                cfg.local_clusters)


def dynakv_workspace_bytes(cfg: Config) -> int:
    return load().dynakv_workspace_bytes(C.byref(_cfg(cfg)))


def _stream() -> int:
    return torch.cuda.current_stream().cuda_stream


def _dev(t: torch.Tensor, dtype, shape=None) -> int:
    assert t.is_cuda and t.is_contiguous() and t.dtype == dtype, (t.device, t.dtype, dtype)
    if shape is not None:
        assert tuple(t.shape) == tuple(shape), (tuple(t.shape), tuple(shape))
    return t.data_ptr()


def _raw_stream(index: int) -> int:
    return torch.cuda.current_stream(index).cuda_stream


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", _raw_stream)      # the same without making a Stream object (1 us)


def _enqueue(index: int, name: str, call, *args):
    """call(*args, stream) with the tensors' device current, on that device's current stream."""
    if index == torch.cuda.current_device():
        rc = call(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = call(*args, _raw_stream(index))
    if rc:
        _check(rc, name)


def _on_device(t, index: int, dtype, shape) -> int:
    """Address of an operand of the operators beside the index; ValueError where it does not fit."""
    if t.get_device() != index or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError("expected a contiguous %s tensor %s on GPU %d, got %s %s on %s%s" % (
            dtype, tuple(shape), index, t.dtype, tuple(t.shape), t.device, "" if t.is_contiguous() else ", not contiguous"))
    return t.data_ptr()


def _gpu(t: torch.Tensor) -> int:
    if not t.is_cuda:
        raise ValueError("expected a tensor on a GPU, got one on %s" % t.device)
    return t.get_device()


# ---- operators beside the index ---------------------------------------------------------------------
_CODES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


def dynakv_norm_rope(q, k, v, positions, q_out, k_out, v_out, q_weight=None, k_weight=None, inv_freq=None, eps=1e-6,
                     interleaved=False):
    """Norms, rotates and lays out a layer's projected rows by unit (see the header).

    q [B, T, H * G, 128], k and v [B, T, H, 128]: views whose last two dimensions are contiguous (parts of one fused projection
    are); any of them may be None together with its output.  positions int32 [B, T], negative: padding, left as it is.
    q_out [B * H, T, G, 128], k_out and v_out [B * H, T, 128]; q_weight, k_weight [128] or None: no norm; inv_freq float32
    [rotary_dim / 2] or None: no rotation."""
    if (q is None) != (q_out is None) or (k is None) != (k_out is None) or (v is None) != (v_out is None):
        raise ValueError("queries, keys and values each come with their output")
    given = q if q is not None else k if k is not None else v
    if given is None:
        raise ValueError("no rows are given")
    index, dtype = _gpu(given), given.dtype
    if dtype not in _CODES:
        raise ValueError("rows of %s are not supported" % dtype)
    if positions.dim() != 2 or given.dim() != 4:
        raise ValueError("positions are [sequences, tokens], rows [sequences, tokens, heads, 128]")
    B, T = positions.shape
    kv = k if k is not None else v
    H = kv.shape[2] if kv is not None else q_out.shape[0] // max(1, B)
    heads = H if q is None else q.shape[2]
    if H < 1 or heads < 1 or heads % H:
        raise ValueError("%d query heads do not go with %d KV heads" % (heads, H))
    G = heads // H

    def rows(x, n, name):                  # address, stride of a sequence, of a token
        if x is None:
            return None, 0, 0
        st = x.stride()
        # (a dimension of one element may have any stride)
        if x.get_device() != index or x.dtype is not dtype or x.shape != (B, T, n, 128) or st[3] != 1 or (st[2] != 128 and n > 1):
            raise ValueError("%s: expected %s [%d, %d, %d, 128] on GPU %d with contiguous heads, got %s %s, strides %s, on %s" % (
                name, dtype, B, T, n, index, x.dtype, tuple(x.shape), st, x.device))
        return x.data_ptr(), st[0] if B > 1 else 0, st[1] if T > 1 else 0

    qp, q0, q1 = rows(q, heads, "q")
    kp, k0, k1 = rows(k, H, "k")
    vp, v0, v1 = rows(v, H, "v")
    pos = _on_device(positions, index, torch.int32, (B, T))
    qo = None if q is None else _on_device(q_out, index, dtype, (B * H, T, G, 128))
    ko = None if k is None else _on_device(k_out, index, dtype, (B * H, T, 128))
    vo = None if v is None else _on_device(v_out, index, dtype, (B * H, T, 128))
    wq = None if q_weight is None else _on_device(q_weight, index, dtype, (128,))
    wk = None if k_weight is None else _on_device(k_weight, index, dtype, (128,))
    pairs = 0 if inv_freq is None else inv_freq.numel()
    freq = None if inv_freq is None else _on_device(inv_freq, index, torch.float32, (pairs,))
    c = _Heads(_CODES[dtype], B, T, H, G, 128, 2 * pairs, 1 if interleaved else 0, eps, q0, q1, k0, k1, v0, v1)
    _enqueue(index, "dynakv_norm_rope", load().dynakv_norm_rope, C.byref(c), qp, kp, vp, wq, wk, freq, pos, qo, ko, vo)


def dynakv_tree_scratch_bytes(n_units: int, n_nodes: int, group_size: int) -> int:
    return load().dynakv_tree_scratch_bytes(n_units, n_nodes, group_size)


def tree_scratch(n_units: int, n_nodes: int, group_size: int, device="cuda:0") -> torch.Tensor:
    """Scratch for dynakv_attend_tree and dynakv_packed_attend of these sizes.  Calls that may overlap (two streams, two graphs)
    need one each."""
    n = dynakv_tree_scratch_bytes(n_units, n_nodes, group_size)
    if n == 0:
        raise ValueError("dynakv: no tree of %d nodes with %d query heads on %d units" % (n_nodes, group_size, n_units))
    return torch.empty(n, dtype=torch.uint8, device=device)


def _tree_operands(index, dtype, U, Q, k_tree, v_tree, tree, out, lse, scratch):
    """Addresses of what the two attentions of drafted tokens share: (sizes and queries to tree), (out to scratch)."""
    if Q.dim() != 4 or (k_tree is None) != (v_tree is None):
        raise ValueError("Q is [units, nodes, query heads, 128]; drafted keys and values come together")
    _, T, G, _ = shape = Q.shape
    if shape[0] != U or shape[3] != 128:
        raise ValueError("Q: expected [%d, nodes, query heads, 128], got %s" % (U, tuple(shape)))
    q, o = _on_device(Q, index, dtype, shape), _on_device(out, index, dtype, shape)
    k = v = t = l = None
    if k_tree is not None:
        k, v = _on_device(k_tree, index, dtype, (U, T, 128)), _on_device(v_tree, index, dtype, (U, T, 128))
    if tree is not None:
        t = _on_device(tree, index, torch.int64, (U, T))
    if lse is not None:
        l = _on_device(lse, index, torch.float32, (U, T, G))
    if scratch.get_device() != index or scratch.dtype is not torch.uint8 or not scratch.is_contiguous():
        raise ValueError("scratch: expected contiguous bytes on GPU %d" % index)
    return T, G, (q, k, v, t), (o, l, scratch.data_ptr(), scratch.numel())


class PackedCache:
    """A packed cache (dynakv_packed_t) over four uint8 tensors that it keeps alive: codes [U, capacity, 128 * bits / 8] and
    scales [U, capacity, 4] of keys and of values; dtype "f32", "f16" or "bf16": of what is written and read."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales, dtype: str):
        self._lib = load()
        self.index = _gpu(k_codes)
        if k_codes.dim() != 3 or k_codes.shape[2] not in (128, 64) or dtype not in DTYPES:
            raise ValueError("codes are [units, capacity, 128 or 64] of dtype f32, f16 or bf16, got %s, %s" % (tuple(k_codes.shape), dtype))
        U, cap, width = k_codes.shape
        self.n_units, self.capacity, self.bits, self.dtype = U, cap, width // 16, TORCH_DTYPES[dtype]
        u8 = torch.uint8
        self.tensors = (k_codes, k_scales, v_codes, v_scales)
        self._c = _Packed(U, cap, 128, DTYPES[dtype], self.bits, _on_device(k_codes, self.index, u8, (U, cap, width)),
                          _on_device(k_scales, self.index, u8, (U, cap, 4)), _on_device(v_codes, self.index, u8, (U, cap, width)),
                          _on_device(v_scales, self.index, u8, (U, cap, 4)))
        self._ref = C.byref(self._c)

    @classmethod
    def zeros(cls, n_units: int, capacity: int, dtype: str, bits: int, device="cuda:0"):
        if bits not in (8, 4):
            raise ValueError("a packed cache has 8 or 4 bits, not %r" % (bits,))
        t = [torch.zeros(n_units, capacity, w, dtype=torch.uint8, device=device) for w in (16 * bits, 4, 16 * bits, 4)]
        return cls(*t, dtype=dtype)

    def _rows(self, K, V):
        if K.dim() != 3:
            raise ValueError("rows are [units, tokens, 128], got %s" % (tuple(K.shape),))
        n = K.shape[1]
        shape = (self.n_units, n, 128)
        return n, _on_device(K, self.index, self.dtype, shape), _on_device(V, self.index, self.dtype, shape)

    def _per_unit(self, t):
        return None if t is None else _on_device(t, self.index, torch.int32, (self.n_units,))

    def dynakv_packed_write(self, K: torch.Tensor, V: torch.Tensor, start: torch.Tensor | None = None, count: torch.Tensor | None = None):
        """Row i < count[u] of K, V [U, n, 128] goes to position start[u] + i (int32 [U]; None: 0 and n)."""
        n, kp, vp = self._rows(K, V)
        _enqueue(self.index, "dynakv_packed_write", self._lib.dynakv_packed_write, self._ref, kp, vp, n, self._per_unit(start),
                 self._per_unit(count))

    def dynakv_packed_read(self, positions: torch.Tensor | None, K: torch.Tensor, V: torch.Tensor):
        """The rows at positions (int32 [U, n]; None: the first n) into K, V [U, n, 128]."""
        n, kp, vp = self._rows(K, V)
        pp = None if positions is None else _on_device(positions, self.index, torch.int32, (self.n_units, n))
        _enqueue(self.index, "dynakv_packed_read", self._lib.dynakv_packed_read, self._ref, pp, n, kp, vp)

    def dynakv_packed_attend(self, lengths, Q, k_tree, v_tree, tree, out, lse, scratch, softmax_scale: float = 0.0):
        """Attention of a tree of drafted tokens over rows 0..lengths[u]-1 (int32 [U]; None: all); operands as those of
        Index.dynakv_attend_tree."""
        T, G, before, after = _tree_operands(self.index, self.dtype, self.n_units, Q, k_tree, v_tree, tree, out, lse, scratch)
        q, k, v, t = before
        _enqueue(self.index, "dynakv_packed_attend", self._lib.dynakv_packed_attend, self._ref, self._per_unit(lengths), q, T, G, k, v, t,
                 softmax_scale, *after)


class Index:
    """One index (dynakv_index_t) over a workspace tensor it keeps alive.  Work goes to torch's current stream."""

    def __init__(self, cfg: Config, device="cuda:0"):
        self.cfg = cfg
        self._lib = load()
        self._c = _cfg(cfg)
        nbytes = self._lib.dynakv_workspace_bytes(C.byref(self._c))
        if nbytes == 0:
            raise ValueError("dynakv: invalid configuration %r" % (cfg,))
        self.device = torch.device(device)
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        h = C.c_void_p()
        _check(self._lib.dynakv_create(C.byref(self._c), self.workspace.data_ptr(), nbytes, C.byref(h)), "dynakv_create")
        self._h = h
        self._tdtype = TORCH_DTYPES[cfg.dtype]

    def __del__(self):
        if getattr(self, "_h", None):
            self._lib.dynakv_destroy(self._h)
            self._h = None

    # ---- the four calls ---------------------------------------------------------------------
    def dynakv_build_index(self, K: torch.Tensor, V: torch.Tensor, init_idx: torch.Tensor):
        c = self.cfg
        n = K.shape[1]
        kp = _dev(K, self._tdtype, (c.n_units, n, c.head_dim))
        vp = _dev(V, self._tdtype, (c.n_units, n, c.head_dim))
        ip = _dev(init_idx, torch.int32, (c.n_units, c.n_clusters_init))
        _check(self._lib.dynakv_build_index(self._h, kp, vp, n, ip, _stream()), "dynakv_build_index")

    def dynakv_extend_index(self, K: torch.Tensor, V: torch.Tensor):
        c = self.cfg
        n = K.shape[1]
        kp = _dev(K, self._tdtype, (c.n_units, n, c.head_dim))
        vp = _dev(V, self._tdtype, (c.n_units, n, c.head_dim))
        _check(self._lib.dynakv_extend_index(self._h, kp, vp, n, _stream()), "dynakv_extend_index")

    def dynakv_retrieve_attend(self, Q: torch.Tensor, token_budget: int, out: torch.Tensor, lse: torch.Tensor | None):
        c = self.cfg
        qp = _dev(Q, self._tdtype, (c.n_units, c.group_size, c.head_dim))
        op = _dev(out, torch.float32, (c.n_units, c.group_size, c.head_dim))
        lp = _dev(lse, torch.float32, (c.n_units, c.group_size)) if lse is not None else None
        _check(self._lib.dynakv_retrieve_attend(self._h, qp, int(token_budget), op, lp, _stream()),
               "dynakv_retrieve_attend")

    def dynakv_place_by_coretrieval(self, K: torch.Tensor, V: torch.Tensor, Qref: torch.Tensor, token_budget: int):
        """Returns (P [U, M0, M0] float32: Eq. 8's co-retrieval probabilities, order [U, M0] int32: the placement chain),
        both device tensors; the index's pages are laid out afresh in chain order."""
        c = self.cfg
        n, r = K.shape[1], Qref.shape[0]
        kp = _dev(K, self._tdtype, (c.n_units, n, c.head_dim))
        vp = _dev(V, self._tdtype, (c.n_units, n, c.head_dim))
        qp = _dev(Qref, self._tdtype, (r, c.n_units, c.group_size, c.head_dim))
        P = torch.empty(c.n_units, c.n_clusters_init, c.n_clusters_init, dtype=torch.float32, device=self.device)
        order = torch.empty(c.n_units, c.n_clusters_init, dtype=torch.int32, device=self.device)
        _check(self._lib.dynakv_place_by_coretrieval(self._h, kp, vp, n, qp, r, int(token_budget), P.data_ptr(),
                                                      order.data_ptr(), _stream()), "dynakv_place_by_coretrieval")
        return P, order

    def dynakv_retrieve_attend_static(self, Q: torch.Tensor, token_budget: int, out: torch.Tensor, lse: torch.Tensor | None):
        """The same retrieval with the split-KV scratch in the library's static device array; returns the status
        (ECAPACITY if the configuration needs more scratch than the array holds) instead of raising on it."""
        c = self.cfg
        qp = _dev(Q, self._tdtype, (c.n_units, c.group_size, c.head_dim))
        op = _dev(out, torch.float32, (c.n_units, c.group_size, c.head_dim))
        lp = _dev(lse, torch.float32, (c.n_units, c.group_size)) if lse is not None else None
        rc = self._lib.dynakv_retrieve_attend_static(self._h, qp, int(token_budget), op, lp, _stream())
        if rc not in (OK, ECAPACITY):
            _check(rc, "dynakv_retrieve_attend_static")
        return rc

    def dynakv_append(self, k_new: torch.Tensor, v_new: torch.Tensor):
        c = self.cfg
        kp = _dev(k_new, self._tdtype, (c.n_units, c.head_dim))
        vp = _dev(v_new, self._tdtype, (c.n_units, c.head_dim))
        _check(self._lib.dynakv_append(self._h, kp, vp, _stream()), "dynakv_append")

    def dynakv_split(self):
        _check(self._lib.dynakv_split(self._h, _stream()), "dynakv_split")

    def dynakv_decode_step(self, Q: torch.Tensor, token_budget: int, out: torch.Tensor, lse: torch.Tensor | None,
                           k_new: torch.Tensor, v_new: torch.Tensor):
        c = self.cfg
        qp = _dev(Q, self._tdtype, (c.n_units, c.group_size, c.head_dim))
        op = _dev(out, torch.float32, (c.n_units, c.group_size, c.head_dim))
        lp = _dev(lse, torch.float32, (c.n_units, c.group_size)) if lse is not None else None
        kp = _dev(k_new, self._tdtype, (c.n_units, c.head_dim))
        vp = _dev(v_new, self._tdtype, (c.n_units, c.head_dim))
        _check(self._lib.dynakv_decode_step(self._h, qp, int(token_budget), op, lp, kp, vp, _stream()),
               "dynakv_decode_step")

    def dynakv_attend_tree(self, Q, k_tree, v_tree, tree, out, lse, scratch):
        """Attention of a tree of drafted tokens over what the last retrieval gathered, and over the tree.

        Q, out [U, nodes, G, 128]; k_tree, v_tree [U, nodes, 128] or None; tree int64 [U, nodes] of which bit j says that the
        node sees drafted token j, or None: a chain; lse float32 [U, nodes, G] or None; scratch: tree_scratch(U, nodes, G)."""
        index = self.workspace.get_device()
        T, G, before, after = _tree_operands(index, self._tdtype, self.cfg.n_units, Q, k_tree, v_tree, tree, out, lse, scratch)
        if G != self.cfg.group_size:
            raise ValueError("the index has %d query heads per unit, Q %d" % (self.cfg.group_size, G))
        q, k, v, t = before
        _enqueue(index, "dynakv_attend_tree", self._lib.dynakv_attend_tree, self._h, q, T, k, v, t, *after)

    def decode_step_ptrs(self, q_ptr: int, budget: int, out_ptr: int, lse_ptr: int, k_ptr: int, v_ptr: int, stream: int):
        """dynakv_decode_step on raw device addresses, without per-call tensor checks, for loops where
        interpreter time would otherwise dominate."""
        rc = self._lib.dynakv_decode_step(self._h, q_ptr, budget, out_ptr, lse_ptr, k_ptr, v_ptr, stream)
        if rc:
            _check(rc, "decode step")

    # ---- timing aid ---------------------------------------------------------------------------
    def dynakv_profile_enable(self, max_launches: int):
        _check(self._lib.dynakv_profile_enable(self._h, int(max_launches)), "dynakv_profile_enable")

    def dynakv_profile_sample(self, every: int, run: int = 1):
        _check(self._lib.dynakv_profile_sample(self._h, int(every), int(run)), "dynakv_profile_sample")

    def dynakv_profile_read(self):
        n, ms = C.c_int32(), C.c_double()
        _check(self._lib.dynakv_profile_read(self._h, C.byref(n), C.byref(ms)), "dynakv_profile_read")
        return n.value, ms.value

    def dynakv_profiled_kernel(self) -> str:
        return self._lib.dynakv_profiled_kernel(self._h).decode()

    # ---- snapshot -------------------------------------------------------------------------------
    def _state_spec(self):
        c = self.cfg
        U, M, N, d = c.n_units, c.max_clusters, c.max_tokens, c.head_dim
        i32, f32, f64, i64 = torch.int32, torch.float32, torch.float64, torch.int64
        return dict(n_clusters=((U,), i32), n_tokens=((U,), i32), error=((U,), i32), tau=((U,), f64),
                    centroids=((U, M, d), f32), size=((U, M), i32), buffered=((U, M), i32), flag=((U, M), i32),
                    m2=((U, M), f64), offsets=((U, M + 1), i32), members=((U, N), i32), scores=((U, M), f32),
                    n_selected=((U,), i32), selected=((U, M), i32), n_gathered=((U,), i32), gathered=((U, N), i32),
                    last_assign=((U,), i32), counters=((U, 8), i64), keys=((U, N, d), self._tdtype),
                    values=((U, N, d), self._tdtype), first_page=((U, M), i32))

    def dynakv_export_state(self, fields=_STATE_FIELDS[:-3], to_cpu=True):
        """Returns the requested parts of the state (the call waits for the stream), as CPU tensors unless
        to_cpu is False.  A set error word does not raise: the returned status is kept in `self.export_status`
        (ECAPACITY in that case) and the words are in the "error" field."""
        spec = self._state_spec()
        # the library writes these from end to end; the others only as far as there are tokens
        partly = ("members", "gathered", "keys", "values")
        bufs = {k: (torch.zeros if k in partly else torch.empty)(spec[k][0], dtype=spec[k][1], device=self.device) for k in fields}
        st = _State(**{k: (bufs[k].data_ptr() if k in bufs else None) for k in _STATE_FIELDS})
        rc = self._lib.dynakv_export_state(self._h, C.byref(st), _stream())
        self.export_status = rc
        if rc not in (OK, ECAPACITY):
            _check(rc, "dynakv_export_state")
        return {k: v.cpu() for k, v in bufs.items()} if to_cpu else bufs

    def dynakv_import_state(self, state: dict):
        """state: device tensors by field name (the fields of IMPORT_FIELDS; n_selected / selected optional), shaped
        like those dynakv_export_state returns."""
        spec = self._state_spec()
        ptrs = {}
        for k in IMPORT_FIELDS:
            if k in state:
                ptrs[k] = _dev(state[k], spec[k][1], spec[k][0])
        st = _State(**{k: ptrs.get(k) for k in _STATE_FIELDS})
        _check(self._lib.dynakv_import_state(self._h, C.byref(st), _stream()), "dynakv_import_state")
