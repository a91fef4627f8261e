"""Thin Python binding of libkvr (include/kvr.h) over ctypes.

Argument marshalling only: every step of the decode path runs in the CUDA
kernels of libkvr.so.  Functions keep the C names; torch tensors are passed by
their data pointers, and the stream defaults to torch's current CUDA stream.
Importing this module fails loudly if libkvr.so has not been built.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libkvr.so")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"libkvr.so not found at {LIB_PATH}: build it with "
        "`python -c 'import __graft_entry__ as g; g.build()'` (there is no "
        "fallback implementation)")

lib = ctypes.CDLL(LIB_PATH)

KVR_OK, KVR_EINVAL, KVR_ENOMEM, KVR_ECAPACITY, KVR_ECUDA, KVR_EDEVICE, \
    KVR_ESTATE = range(7)
STATUS_NAMES = {0: "KVR_OK", 1: "KVR_EINVAL", 2: "KVR_ENOMEM",
                3: "KVR_ECAPACITY", 4: "KVR_ECUDA", 5: "KVR_EDEVICE",
                6: "KVR_ESTATE"}
KVR_BF16, KVR_F32 = 0, 1
DTYPES = {"bf16": KVR_BF16, "f32": KVR_F32}
TORCH_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


class KvrError(RuntimeError):
    def __init__(self, status: int, where: str, msg: str):
        super().__init__(f"{where}: {STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class kvr_cache_desc(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int), ("n_layers", ctypes.c_int),
                ("n_kv_heads", ctypes.c_int), ("group", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("capacity", ctypes.c_int),
                ("kv_dtype", ctypes.c_int), ("out_dtype", ctypes.c_int),
                ("softmax_scale", ctypes.c_float)]


_P = ctypes.c_void_p
_I = ctypes.c_int
_S = ctypes.c_int

_SIGS = {
    "kvr_cache_required_bytes": (ctypes.c_size_t, [ctypes.POINTER(kvr_cache_desc)]),
    "kvr_cache_create": (_S, [ctypes.POINTER(kvr_cache_desc), _P, ctypes.c_size_t,
                              _P, ctypes.POINTER(_P)]),
    "kvr_cache_destroy": (None, [_P]),
    "kvr_cache_load": (_S, [_P, _I, _P, _P, _I, _I, _P]),
    "kvr_decode_attend_score": (_S, [_P, _I, _I, _P, _P, _P, _P, _P]),
    "kvr_decode_attend_score_noalloc": (_S, [_P, _I, _I, _P, _P, _P, _P, _P]),
    "kvr_evict_compact": (_S, [_P, _I, _I, _I, _I, _P]),
    "kvr_decode_step": (_S, [_P, _I, _I, _P, _P, _P, _P, _I, _I, _P]),
    "kvr_decode_step_rkv": (_S, [_P, _I, _I, _P, _P, _P, _P, _I, _I,
                                 ctypes.c_float, _P]),
    "kvr_decode_step_host": (_S, [_P, _I, _I, _P, _P, _P, _P, _P, _P, _P, _P,
                                  _I, _I, _P]),
    "kvr_absorb_chunk": (_S, [_P, _I, _I, _I, _P, _P, _P, _P, _I, _I, _I, _P]),
    "kvr_cache_copy_sequences": (_S, [_P, _P, _P, _P, _I, _P]),
    "kvr_evict_compact_rkv": (_S, [_P, _I, _I, _I, _I, ctypes.c_float, _P]),
    "kvr_cache_export": (_S, [_P, _I, _P, _P, _P, _P, _P, _P, _P]),
    "kvr_cache_import": (_S, [_P, _I, _P, _P, _P, _P, _P, _P, _P]),
    "kvr_cache_lengths": (_S, [_P, _P]),
    "kvr_cache_launch_count": (_S, [_P, _P]),
    "kvr_cache_set_fused": (_S, [_P, _I]),
    "kvr_cache_set_wait_limit": (_S, [_P, ctypes.c_uint64]),
    "kvr_cache_set_hold_first_unit": (_S, [_P, _I]),
    "kvr_cache_set_fused_tuning": (_S, [_P, _I, _I]),
    "kvr_cache_set_chunk_tuning": (_S, [_P, _I, _I]),
    "kvr_fork_set_kernel": (_S, [_P, _I]),
    "kvr_fork_last_kernel": (_I, [_P]),
    "kvr_cache_set_absorb_kernel": (_S, [_P, _I]),
    "kvr_cache_last_absorb_kernel": (_I, [_P]),
    "kvr_cache_last_chunk_groups": (_I, [_P, _P]),
    "kvr_cache_scores": (_S, [_P, _P, _P, _P, _P]),
    "kvr_cache_rows": (_S, [_P, _P, _P]),
    "kvr_sync_status": (_S, [_P, _P]),
    "kvr_last_error": (ctypes.c_char_p, []),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def kvr_last_error() -> str:
    return lib.kvr_last_error().decode()


def _check(status: int, where: str):
    if status != KVR_OK:
        raise KvrError(status, where, kvr_last_error())


# A call's marshalling is most of what a small step costs on the host (one
# sequence, one call a layer, 28 calls: 304 us a token with c_void_p objects
# and torch.cuda.current_stream(), 184 without), so pointers go to ctypes as plain integers and
# the current stream is read without building a torch.cuda.Stream.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(_raw_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _ptr(t):
    if isinstance(t, torch.Tensor):
        if not t.is_contiguous():
            raise ValueError("tensors passed to libkvr must be contiguous")
        return t.data_ptr()
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        if not t.flags["C_CONTIGUOUS"]:
            raise ValueError("arrays passed to libkvr must be C-contiguous")
        return t.ctypes.data_as(ctypes.c_void_p)
    return int(t)


def make_desc(n_seq, n_layers, n_kv_heads, group, head_dim, capacity,
              kv_dtype="bf16", out_dtype="bf16", softmax_scale=0.0):
    return kvr_cache_desc(n_seq, n_layers, n_kv_heads, group, head_dim,
                          capacity, DTYPES[kv_dtype], DTYPES[out_dtype],
                          float(softmax_scale))


def kvr_cache_required_bytes(desc: kvr_cache_desc) -> int:
    return int(lib.kvr_cache_required_bytes(ctypes.byref(desc)))


def kvr_cache_create(desc, dev_buf, nbytes, stream=None):
    h = ctypes.c_void_p()
    _check(lib.kvr_cache_create(ctypes.byref(desc), _ptr(dev_buf), nbytes,
                                _stream(stream), ctypes.byref(h)),
           "kvr_cache_create")
    return h


def kvr_cache_destroy(h):
    lib.kvr_cache_destroy(h)


def kvr_cache_load(h, seq, k, v, n_rows, first_pos=0, stream=None):
    _check(lib.kvr_cache_load(h, seq, _ptr(k), _ptr(v), n_rows, first_pos,
                              _stream(stream)), "kvr_cache_load")


def kvr_decode_attend_score(h, layer_begin, layer_end, q, k_new, v_new, out,
                            stream=None):
    _check(lib.kvr_decode_attend_score(h, layer_begin, layer_end, _ptr(q),
                                       _ptr(k_new), _ptr(v_new), _ptr(out),
                                       _stream(stream)),
           "kvr_decode_attend_score")


def kvr_decode_attend_score_noalloc(h, layer_begin, layer_end, q, k_new,
                                    v_new, out, stream=None):
    _check(lib.kvr_decode_attend_score_noalloc(h, layer_begin, layer_end,
                                               _ptr(q), _ptr(k_new),
                                               _ptr(v_new), _ptr(out),
                                               _stream(stream)),
           "kvr_decode_attend_score_noalloc")


def kvr_evict_compact(h, layer_begin, layer_end, budget, window, stream=None):
    _check(lib.kvr_evict_compact(h, layer_begin, layer_end, budget, window,
                                 _stream(stream)), "kvr_evict_compact")


def kvr_decode_step(h, layer_begin, layer_end, q, k_new, v_new, out, budget,
                    window, stream=None):
    _check(lib.kvr_decode_step(h, layer_begin, layer_end, _ptr(q), _ptr(k_new),
                               _ptr(v_new), _ptr(out), budget, window,
                               _stream(stream)), "kvr_decode_step")


def kvr_decode_step_rkv(h, layer_begin, layer_end, q, k_new, v_new, out,
                        budget, window, lam, stream=None):
    _check(lib.kvr_decode_step_rkv(h, layer_begin, layer_end, _ptr(q),
                                   _ptr(k_new), _ptr(v_new), _ptr(out), budget,
                                   window, float(lam), _stream(stream)),
           "kvr_decode_step_rkv")


def kvr_decode_step_host(h, layer_begin, layer_end, q_host, k_new_host,
                         v_new_host, out_host, q_dev, k_new_dev, v_new_dev,
                         out_dev, budget, window, stream=None):
    _check(lib.kvr_decode_step_host(
        h, layer_begin, layer_end, _ptr(q_host), _ptr(k_new_host),
        _ptr(v_new_host), _ptr(out_host), _ptr(q_dev), _ptr(k_new_dev),
        _ptr(v_new_dev), _ptr(out_dev), budget, window, _stream(stream)),
        "kvr_decode_step_host")


def kvr_absorb_chunk(h, layer_begin, layer_end, chunk, q, k_new, v_new, out,
                     budget, window, evict=True, stream=None):
    _check(lib.kvr_absorb_chunk(h, layer_begin, layer_end, chunk, _ptr(q),
                                _ptr(k_new), _ptr(v_new), _ptr(out), budget,
                                window, 1 if evict else 0, _stream(stream)),
           "kvr_absorb_chunk")


def kvr_evict_compact_rkv(h, layer_begin, layer_end, budget, window, lam,
                          stream=None):
    _check(lib.kvr_evict_compact_rkv(h, layer_begin, layer_end, budget, window,
                                     float(lam), _stream(stream)),
           "kvr_evict_compact_rkv")


def kvr_cache_copy_sequences(dst, dst_seqs, src, src_seqs, stream=None):
    d = np.ascontiguousarray(dst_seqs, dtype=np.int32)
    s = np.ascontiguousarray(src_seqs, dtype=np.int32)
    if d.shape != s.shape or d.ndim != 1:
        raise ValueError("dst_seqs and src_seqs must be 1-D of one length")
    _check(lib.kvr_cache_copy_sequences(dst, _ptr(d), src, _ptr(s), len(d),
                                        _stream(stream)),
           "kvr_cache_copy_sequences")


def kvr_cache_import(h, seq, host_k, host_v, host_score, host_pos, host_len,
                     host_next_pos, stream=None):
    _check(lib.kvr_cache_import(h, seq, _ptr(host_k), _ptr(host_v),
                                _ptr(host_score), _ptr(host_pos),
                                _ptr(host_len), _ptr(host_next_pos),
                                _stream(stream)), "kvr_cache_import")


def kvr_cache_export(h, seq, host_k, host_v, host_score, host_pos, host_len,
                     host_next_pos, stream=None):
    _check(lib.kvr_cache_export(h, seq, _ptr(host_k), _ptr(host_v),
                                _ptr(host_score), _ptr(host_pos),
                                _ptr(host_len), _ptr(host_next_pos),
                                _stream(stream)), "kvr_cache_export")


def kvr_cache_lengths(h, host_len):
    _check(lib.kvr_cache_lengths(h, _ptr(host_len)), "kvr_cache_lengths")


def kvr_cache_launch_count(h) -> int:
    n = ctypes.c_uint64()
    _check(lib.kvr_cache_launch_count(h, ctypes.byref(n)),
           "kvr_cache_launch_count")
    return int(n.value)


def kvr_cache_set_fused(h, enable: bool):
    _check(lib.kvr_cache_set_fused(h, 1 if enable else 0), "kvr_cache_set_fused")


def kvr_cache_set_fused_tuning(h, groups: int, group_warps: int = 0):
    _check(lib.kvr_cache_set_fused_tuning(h, groups, group_warps),
           "kvr_cache_set_fused_tuning")


def kvr_fork_set_kernel(h, kernel: int):
    _check(lib.kvr_fork_set_kernel(h, kernel), "kvr_fork_set_kernel")


def kvr_fork_last_kernel(h) -> int:
    return int(lib.kvr_fork_last_kernel(h))


def kvr_cache_set_chunk_tuning(h, groups: int, stages: int = 0):
    _check(lib.kvr_cache_set_chunk_tuning(h, groups, stages),
           "kvr_cache_set_chunk_tuning")


def kvr_sync_status(h, stream=None):
    _check(lib.kvr_sync_status(h, _stream(stream)), "kvr_sync_status")


class Cache:
    """Owner of one kvr_cache handle and the torch buffer it lives in."""

    def __init__(self, n_seq, n_layers, n_kv_heads, group, head_dim, capacity,
                 kv_dtype="bf16", out_dtype="bf16", softmax_scale=0.0,
                 device="cuda", stream=None, buf=None):
        """buf: an optional caller-owned uint8 device tensor of at least
        kvr_cache_required_bytes (256-byte aligned); by default one is
        allocated."""
        self.desc = make_desc(n_seq, n_layers, n_kv_heads, group, head_dim,
                              capacity, kv_dtype, out_dtype, softmax_scale)
        self.S, self.L, self.H, self.G, self.d = (n_seq, n_layers, n_kv_heads,
                                                  group, head_dim)
        self.cap = capacity
        self.kv_dtype, self.out_dtype = kv_dtype, out_dtype
        self._rows = self._scores = None  # views of the buffer, once asked for
        self.nbytes = kvr_cache_required_bytes(self.desc)
        if self.nbytes == 0:
            raise KvrError(KVR_EINVAL, "Cache", "invalid descriptor")
        if buf is None:
            buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        elif buf.numel() < self.nbytes or buf.dtype != torch.uint8:
            raise ValueError("buf must be uint8 with at least "
                             f"{self.nbytes} bytes")
        self.buf = buf
        self.handle = kvr_cache_create(self.desc, self.buf, self.nbytes, stream)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            kvr_cache_destroy(h)
            self.handle = None

    @property
    def kv_torch_dtype(self):
        return TORCH_DTYPES[self.kv_dtype]

    @property
    def out_torch_dtype(self):
        return TORCH_DTYPES[self.out_dtype]

    def load(self, seq, k, v, first_pos=0, stream=None):
        k = k.contiguous()
        v = v.contiguous()
        kvr_cache_load(self.handle, seq, k, v, k.shape[2], first_pos, stream)

    def _layers(self, layers):
        return (0, self.L) if layers is None else layers

    def new_out(self, nl):
        return torch.empty(self.S, nl, self.H * self.G, self.d,
                           dtype=self.out_torch_dtype, device=self.buf.device)

    def attend_score(self, q, k_new, v_new, out=None, layers=None, stream=None):
        lb, le = self._layers(layers)
        out = self.new_out(le - lb) if out is None else out
        kvr_decode_attend_score(self.handle, lb, le, q, k_new, v_new, out,
                                stream)
        return out

    def evict(self, budget, window, layers=None, stream=None):
        lb, le = self._layers(layers)
        kvr_evict_compact(self.handle, lb, le, budget, window, stream)

    def step(self, q, k_new, v_new, budget, window, out=None, layers=None,
             stream=None):
        lb, le = self._layers(layers)
        out = self.new_out(le - lb) if out is None else out
        kvr_decode_step(self.handle, lb, le, q, k_new, v_new, out, budget,
                        window, stream)
        return out

    def step_rkv(self, q, k_new, v_new, budget, window, lam=0.1, out=None,
                 layers=None, stream=None):
        """A decode step with the R-KV eviction (kvr_decode_step_rkv)."""
        lb, le = self._layers(layers)
        out = self.new_out(le - lb) if out is None else out
        kvr_decode_step_rkv(self.handle, lb, le, q, k_new, v_new, out, budget,
                            window, lam, stream)
        return out

    def absorb(self, q, k_new, v_new, budget=0, window=0, evict=True,
               out=None, layers=None, stream=None):
        """q [S][nl][c][H*G][d], k_new/v_new [S][nl][c][H][d] -> out
        [S][nl][c][H*G][d] (kvr_absorb_chunk)."""
        lb, le = self._layers(layers)
        c = q.shape[2]
        if out is None:
            out = torch.empty(self.S, le - lb, c, self.H * self.G, self.d,
                              dtype=self.out_torch_dtype, device=self.buf.device)
        kvr_absorb_chunk(self.handle, lb, le, c, q, k_new, v_new, out, budget,
                         window, evict, stream)
        return out

    def evict_rkv(self, budget, window, lam=0.1, layers=None, stream=None):
        """Eviction with the R-KV score (App. C), mix weight lam."""
        lb, le = self._layers(layers)
        kvr_evict_compact_rkv(self.handle, lb, le, budget, window, lam, stream)

    def copy_from(self, src: "Cache", src_seqs, dst_seqs, stream=None):
        """Sequence dst_seqs[i] takes the whole state of src's sequence
        src_seqs[i] (App. C: forking a candidate by copy, or committing the
        chosen one)."""
        kvr_cache_copy_sequences(self.handle, dst_seqs, src.handle, src_seqs,
                                 stream)

    def lengths(self):
        a = np.zeros((self.S, self.L), np.int32)
        kvr_cache_lengths(self.handle, a)
        return a

    def export(self, seq, kv=True, stream=None):
        """Host copy of one sequence: dict of numpy arrays (K/V as float32)."""
        rows = (self.L, self.H, self.cap)
        score = np.zeros(rows, np.float32)
        pos = np.zeros(rows, np.int32)
        ln = np.zeros(rows[:2], np.int32)
        npos = np.zeros(rows[:2], np.int32)
        hk = hv = None
        if kv:
            hk = torch.empty(*rows, self.d, dtype=self.kv_torch_dtype).contiguous()
            hv = torch.empty_like(hk)
        kvr_cache_export(self.handle, seq, hk, hv, score, pos, ln, npos, stream)
        res = {"score": score, "pos": pos, "len": ln, "next_pos": npos}
        if kv:
            res["K"] = hk.float().numpy()
            res["V"] = hv.float().numpy()
        return res

    def import_state(self, seq, state, stream=None):
        """Replace sequence seq with a state dict in the form export(seq,
        kv=True) returns (kvr_cache_import); K/V are cast to kv_dtype."""
        hk, hv = (torch.from_numpy(np.ascontiguousarray(state[x], np.float32))
                  .to(self.kv_torch_dtype).contiguous() for x in ("K", "V"))
        arr = {x: np.ascontiguousarray(state[x], t) for x, t in (
            ("score", np.float32), ("pos", np.int32), ("len", np.int32),
            ("next_pos", np.int32))}
        kvr_cache_import(self.handle, seq, hk, hv, arr["score"], arr["pos"],
                         arr["len"], arr["next_pos"], stream)

    def scores_view(self):
        """(score, pos, state) as device tensors viewing the cache buffer (no
        copy): score and pos [S][L][H][row_stride], state [S][L][H][4]."""
        if self._scores is None:  # the buffer stays where it is
            self._scores = self._view_scores()
        return self._scores

    def _view_scores(self):
        sp, pp, stp = _P(), _P(), _P()
        stride = ctypes.c_int64()
        _check(lib.kvr_cache_scores(self.handle, ctypes.byref(sp), ctypes.byref(pp),
                                    ctypes.byref(stp), ctypes.byref(stride)),
               "kvr_cache_scores")
        base = self.buf.data_ptr()
        rows = self.S * self.L * self.H * stride.value

        def view(ptr, n, dtype):
            off = ptr.value - base
            return self.buf[off:off + 4 * n].view(dtype)

        shape = (self.S, self.L, self.H, stride.value)
        return (view(sp, rows, torch.float32).view(shape),
                view(pp, rows, torch.int32).view(shape),
                view(stp, self.S * self.L * self.H * 4, torch.int32).view(
                    self.S, self.L, self.H, 4))

    def rows_view(self):
        """(K, V) as device tensors viewing the cache buffer (no copy), each
        [S][L][H][capacity][d] (kvr_cache_rows)."""
        if self._rows is None:  # the buffer stays where it is
            self._rows = self._view_rows()
        return self._rows

    def _view_rows(self):
        kp, vp = _P(), _P()
        _check(lib.kvr_cache_rows(self.handle, ctypes.byref(kp),
                                  ctypes.byref(vp)), "kvr_cache_rows")
        shape = (self.S, self.L, self.H, self.cap, self.d)
        es = 2 if self.kv_dtype == "bf16" else 4
        n = int(np.prod(shape)) * es
        base = self.buf.data_ptr()
        return tuple(self.buf[p.value - base:p.value - base + n]
                     .view(self.kv_torch_dtype).view(shape) for p in (kp, vp))

    def set_absorb_kernel(self, kernel: int):
        """kvr_absorb_chunk's one-launch kernel: 0 tcgen05, 1 mma.sync."""
        _check(lib.kvr_cache_set_absorb_kernel(self.handle, kernel),
               "kvr_cache_set_absorb_kernel")

    def last_chunk_groups(self):
        """(groups per SM, warps a group) of the last step on the chunked
        kernel (kvr_cache_last_chunk_groups), (0, 0) before the first."""
        warps = ctypes.c_int()
        groups = lib.kvr_cache_last_chunk_groups(self.handle,
                                                 ctypes.byref(warps))
        return int(groups), warps.value

    def last_absorb_kernel(self) -> int:
        """How the last absorb ran (kvr_cache_last_absorb_kernel): 0 tcgen05,
        1 mma.sync, 2 token by token, 3 in blocks, -1 before the first."""
        return int(lib.kvr_cache_last_absorb_kernel(self.handle))

    def set_fused(self, enable: bool):
        kvr_cache_set_fused(self.handle, enable)

    def set_wait_limit(self, ns: int):
        """Bound of the step kernels' waits on copies (0: the 2 s default)."""
        _check(lib.kvr_cache_set_wait_limit(self.handle, int(ns)),
               "kvr_cache_set_wait_limit")

    def set_hold_first_unit(self, enable: bool):
        """Testing hook: the step kernels' first unit is never loaded, so
        its bounded wait runs out (kvr_cache_set_hold_first_unit)."""
        _check(lib.kvr_cache_set_hold_first_unit(self.handle, 1 if enable
                                                 else 0),
               "kvr_cache_set_hold_first_unit")

    def set_chunk_tuning(self, groups: int, stages: int = 0):
        """groups -1 keeps the chunked kernel off (older per-unit kernels)."""
        kvr_cache_set_chunk_tuning(self.handle, groups, stages)

    def launch_count(self):
        return kvr_cache_launch_count(self.handle)

    def sync_status(self, stream=None):
        kvr_sync_status(self.handle, stream)


# ---- candidates -------------------------------------------------------------

for _name, (_res, _args) in {
    "kvr_fork_required_bytes": (ctypes.c_size_t, [_P, _I, _I]),
    "kvr_fork_candidates": (_S, [_P, _I, _I, _P, ctypes.c_size_t, _P,
                                 ctypes.POINTER(_P)]),
    "kvr_fork_decode_attend_score": (_S, [_P, _I, _I, _P, _P, _P, _P, _P]),
    "kvr_fork_commit": (_S, [_P, _P, _I, _I, _P]),
    "kvr_fork_export": (_S, [_P, _I, _I, _P, _P, _P, _P, _P, _P, _P]),
    "kvr_fork_destroy": (None, [_P]),
}.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def kvr_fork_required_bytes(parent, n_cand, tail_cap) -> int:
    return int(lib.kvr_fork_required_bytes(parent, n_cand, tail_cap))


def kvr_fork_candidates(parent, n_cand, tail_cap, dev_buf, nbytes, stream=None):
    h = ctypes.c_void_p()
    _check(lib.kvr_fork_candidates(parent, n_cand, tail_cap, _ptr(dev_buf),
                                   nbytes, _stream(stream), ctypes.byref(h)),
           "kvr_fork_candidates")
    return h


def kvr_fork_decode_attend_score(fork, layer_begin, layer_end, q, k_new, v_new,
                                 out, stream=None):
    _check(lib.kvr_fork_decode_attend_score(fork, layer_begin, layer_end,
                                            _ptr(q), _ptr(k_new), _ptr(v_new),
                                            _ptr(out), _stream(stream)),
           "kvr_fork_decode_attend_score")


def kvr_fork_commit(fork, chosen, budget, window, stream=None):
    chosen = np.ascontiguousarray(chosen, dtype=np.int32)
    _check(lib.kvr_fork_commit(fork, _ptr(chosen), budget, window,
                               _stream(stream)), "kvr_fork_commit")


def kvr_fork_export(fork, cand, seq, prefix_score, tail_k, tail_v, tail_score,
                    tail_pos, tail_len, stream=None):
    _check(lib.kvr_fork_export(fork, cand, seq, _ptr(prefix_score), _ptr(tail_k),
                               _ptr(tail_v), _ptr(tail_score), _ptr(tail_pos),
                               _ptr(tail_len), _stream(stream)),
           "kvr_fork_export")


def kvr_fork_destroy(fork):
    lib.kvr_fork_destroy(fork)


class Fork:
    """N candidates of a Cache sharing its live rows (owner of the buffer)."""

    def __init__(self, cache: Cache, n_cand: int, tail_cap: int, stream=None,
                 kernel: int = 0, buf=None):
        """kernel: 0 the library's choice, 1 candidate-batched, 2 chunked,
        3 one CTA per unit, 4 generic, 5 candidate-batched on 5th-generation
        tensor cores (kvr_fork_set_kernel).  buf: an
        optional caller-owned uint8 device tensor of at least
        kvr_fork_required_bytes."""
        self.cache, self.N, self.tcap = cache, n_cand, tail_cap
        self.nbytes = kvr_fork_required_bytes(cache.handle, n_cand, tail_cap)
        if self.nbytes == 0:
            raise KvrError(KVR_EINVAL, "Fork", "invalid fork arguments")
        if buf is None:
            buf = torch.empty(self.nbytes, dtype=torch.uint8,
                              device=cache.buf.device)
        elif buf.numel() < self.nbytes or buf.dtype != torch.uint8:
            raise ValueError("buf must be uint8 with at least "
                             f"{self.nbytes} bytes")
        self.buf = buf
        self.handle = kvr_fork_candidates(cache.handle, n_cand, tail_cap,
                                          self.buf, self.nbytes, stream)
        if kernel:
            kvr_fork_set_kernel(self.handle, kernel)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            kvr_fork_destroy(h)
            self.handle = None

    def attend_score(self, q, k_new, v_new, out=None, layers=None, stream=None):
        c = self.cache
        lb, le = (0, c.L) if layers is None else layers
        if out is None:
            out = torch.empty(self.N, c.S, le - lb, c.H * c.G, c.d,
                              dtype=c.out_torch_dtype, device=c.buf.device)
        kvr_fork_decode_attend_score(self.handle, lb, le, q, k_new, v_new, out,
                                     stream)
        return out

    def commit(self, chosen, budget, window, stream=None):
        kvr_fork_commit(self.handle, chosen, budget, window, stream)

    def last_kernel(self) -> int:
        """The kernel that ran the last candidate step (kvr_fork_last_kernel)."""
        return kvr_fork_last_kernel(self.handle)

    def export(self, cand, seq, kv=False, stream=None):
        c = self.cache
        ps = np.zeros((c.L, c.H, c.cap), np.float32)
        ts = np.zeros((c.L, c.H, self.tcap), np.float32)
        tp = np.zeros((c.L, c.H, self.tcap), np.int32)
        tl = np.zeros((c.L, c.H), np.int32)
        tk = tv = None
        if kv:
            tk = torch.empty(c.L, c.H, self.tcap, c.d, dtype=c.kv_torch_dtype)
            tv = torch.empty_like(tk)
        kvr_fork_export(self.handle, cand, seq, ps, tk, tv, ts, tp, tl, stream)
        res = {"prefix_score": ps, "tail_score": ts, "tail_pos": tp,
               "tail_len": tl}
        if kv:
            res["tail_K"] = tk.float().numpy()
            res["tail_V"] = tv.float().numpy()
        return res


# ---- full-context decode ----------------------------------------------------

for _name, (_res, _args) in {
    "kvr_decode_attend_workspace_bytes": (ctypes.c_size_t, [_P, _I, _I, _I]),
    "kvr_decode_attend": (_S, [_P, _I, _I, _P, _P, _P, _P, _I, _P,
                               ctypes.c_size_t, _P]),
}.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def kvr_decode_attend_workspace_bytes(h, layer_begin, layer_end, n_splits=0):
    return int(lib.kvr_decode_attend_workspace_bytes(h, layer_begin, layer_end,
                                                     n_splits))


def kvr_decode_attend(h, layer_begin, layer_end, q, k_new, v_new, out,
                      n_splits, workspace, workspace_bytes, stream=None):
    _check(lib.kvr_decode_attend(h, layer_begin, layer_end, _ptr(q),
                                 _ptr(k_new), _ptr(v_new), _ptr(out), n_splits,
                                 _ptr(workspace), workspace_bytes,
                                 _stream(stream)), "kvr_decode_attend")


def attend_full(cache: Cache, q, k_new, v_new, out=None, layers=None,
                n_splits=0, workspace=None, stream=None):
    """Full-context decode step on `cache` (no scores, no eviction)."""
    lb, le = (0, cache.L) if layers is None else layers
    out = cache.new_out(le - lb) if out is None else out
    need = kvr_decode_attend_workspace_bytes(cache.handle, lb, le, n_splits)
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8,
                                device=cache.buf.device)
    kvr_decode_attend(cache.handle, lb, le, q, k_new, v_new, out, n_splits,
                      workspace, workspace.numel(), stream)
    return out


# ---- degeneration detector: the entropy test --------------------------------

class kvr_entropy_desc(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int), ("vocab", ctypes.c_int),
                ("window", ctypes.c_int), ("guard", ctypes.c_int),
                ("tau", ctypes.c_float), ("temperature", ctypes.c_float),
                ("logits_dtype", ctypes.c_int)]


for _name, (_res, _args) in {
    "kvr_entropy_required_bytes": (ctypes.c_size_t,
                                   [ctypes.POINTER(kvr_entropy_desc)]),
    "kvr_entropy_create": (_S, [ctypes.POINTER(kvr_entropy_desc), _P,
                                ctypes.c_size_t, _P, ctypes.POINTER(_P)]),
    "kvr_entropy_reset": (_S, [_P, _I, _I, _P]),
    "kvr_entropy_step": (_S, [_P, _P, ctypes.c_int64, _P, _P, _P, _P]),
    "kvr_entropy_export": (_S, [_P, _P, _P, _P, _P]),
    "kvr_entropy_sync_status": (_S, [_P, _P]),
    "kvr_entropy_launch_count": (_S, [_P, _P]),
    "kvr_entropy_set_kernel": (_S, [_P, _I]),
    "kvr_entropy_destroy": (None, [_P]),
}.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def kvr_entropy_required_bytes(desc: kvr_entropy_desc) -> int:
    return int(lib.kvr_entropy_required_bytes(ctypes.byref(desc)))


def kvr_entropy_create(desc, dev_buf, nbytes, stream=None):
    h = _P()
    _check(lib.kvr_entropy_create(ctypes.byref(desc), _ptr(dev_buf), nbytes,
                                  _stream(stream), ctypes.byref(h)),
           "kvr_entropy_create")
    return h


def kvr_entropy_reset(h, row_begin, row_end, stream=None):
    _check(lib.kvr_entropy_reset(h, row_begin, row_end, _stream(stream)),
           "kvr_entropy_reset")


def kvr_entropy_step(h, logits, row_stride, entropy=None, mean=None,
                     stopped=None, stream=None):
    _check(lib.kvr_entropy_step(h, _ptr(logits), int(row_stride),
                                _ptr(entropy), _ptr(mean), _ptr(stopped),
                                _stream(stream)), "kvr_entropy_step")


def kvr_entropy_export(h, host_hist, host_count, host_stopped, stream=None):
    _check(lib.kvr_entropy_export(h, _ptr(host_hist), _ptr(host_count),
                                  _ptr(host_stopped), _stream(stream)),
           "kvr_entropy_export")


def kvr_entropy_sync_status(h, stream=None):
    _check(lib.kvr_entropy_sync_status(h, _stream(stream)),
           "kvr_entropy_sync_status")


def kvr_entropy_launch_count(h) -> int:
    n = ctypes.c_uint64()
    _check(lib.kvr_entropy_launch_count(h, ctypes.byref(n)),
           "kvr_entropy_launch_count")
    return n.value


def kvr_entropy_destroy(h):
    lib.kvr_entropy_destroy(h)


class EntropyDetector:
    """Owner of one kvr_entropy handle and the torch buffer it lives in
    (Sec. 3.2 entropy test; App. C tau 7.0, window 12, guard 24)."""

    def __init__(self, rows, vocab, window=12, guard=24, tau=7.0,
                 temperature=1.0, logits_dtype="bf16", device="cuda",
                 stream=None):
        self.desc = kvr_entropy_desc(rows, vocab, window, guard, float(tau),
                                     float(temperature), DTYPES[logits_dtype])
        self.rows, self.vocab, self.window = rows, vocab, window
        self.logits_dtype = logits_dtype
        self.nbytes = kvr_entropy_required_bytes(self.desc)
        if self.nbytes == 0:
            raise KvrError(KVR_EINVAL, "EntropyDetector", "invalid descriptor")
        self.buf = torch.empty(self.nbytes, dtype=torch.uint8, device=device)
        self.handle = kvr_entropy_create(self.desc, self.buf, self.nbytes,
                                         stream)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            kvr_entropy_destroy(h)
            self.handle = None

    def reset(self, begin=0, end=None, stream=None):
        kvr_entropy_reset(self.handle, begin, self.rows if end is None else end,
                          stream)

    def step(self, logits, entropy=None, mean=None, stopped=None, stream=None):
        """One generated token: logits [rows][>= vocab] (row stride taken
        from the tensor).  Returns (entropy, mean, stopped) device tensors."""
        if logits.dim() != 2 or logits.shape[0] != self.rows or \
                logits.shape[1] < self.vocab or logits.stride(1) != 1:
            raise ValueError("logits must be [rows][>= vocab] with unit "
                             "column stride")
        if logits.dtype != TORCH_DTYPES[self.logits_dtype]:
            raise ValueError("logits dtype does not match the descriptor")
        dev = logits.device
        entropy = torch.empty(self.rows, dtype=torch.float32, device=dev) \
            if entropy is None else entropy
        mean = torch.empty(self.rows, dtype=torch.float32, device=dev) \
            if mean is None else mean
        stopped = torch.empty(self.rows, dtype=torch.int32, device=dev) \
            if stopped is None else stopped
        _check(lib.kvr_entropy_step(self.handle,
                                    ctypes.c_void_p(logits.data_ptr()),
                                    int(logits.stride(0)), _ptr(entropy),
                                    _ptr(mean), _ptr(stopped),
                                    _stream(stream)), "kvr_entropy_step")
        return entropy, mean, stopped

    def export(self, stream=None):
        hist = np.zeros((self.rows, self.window), np.float32)
        count = np.zeros(self.rows, np.int32)
        stopped = np.zeros(self.rows, np.int32)
        kvr_entropy_export(self.handle, hist, count, stopped, stream)
        return hist, count, stopped

    def set_kernel(self, kernel: int):
        """0: the library's choice, 1: persistent streaming kernel, 2: one CTA
        per piece of a row."""
        _check(lib.kvr_entropy_set_kernel(self.handle, kernel),
               "kvr_entropy_set_kernel")

    def launch_count(self):
        return kvr_entropy_launch_count(self.handle)

    def sync_status(self, stream=None):
        kvr_entropy_sync_status(self.handle, stream)


# ---- the full context held in 4 bits ----------------------------------------

for _name, (_res, _args) in {
    "kvr_kv4_required_bytes": (ctypes.c_size_t,
                               [ctypes.POINTER(kvr_cache_desc)]),
    "kvr_kv4_create": (_S, [ctypes.POINTER(kvr_cache_desc), _P,
                            ctypes.c_size_t, _P, ctypes.POINTER(_P)]),
    "kvr_kv4_destroy": (None, [_P]),
    "kvr_kv4_load": (_S, [_P, _I, _P, _P, _I, _P]),
    "kvr_kv4_append": (_S, [_P, _I, _I, _I, _P, _P, _P, _P]),
    "kvr_kv4_truncate": (_S, [_P, _P]),
    "kvr_kv4_lengths": (_S, [_P, _P]),
    "kvr_kv4_read": (_S, [_P, _I, _I, _I, _P, _P, _P, _P]),
    "kvr_kv4_attend_workspace_bytes": (ctypes.c_size_t, [_P, _I, _I, _I]),
    "kvr_kv4_attend": (_S, [_P, _I, _I, _I, _P, _P, _P, _I, _P,
                            ctypes.c_size_t, _P]),
    "kvr_kv4_evict": (_S, [_P, _P, _I, _I, _P]),
    "kvr_kv4_scores": (_S, [_P, _P, _P]),
    "kvr_kv4_launch_count": (_S, [_P, _P]),
    "kvr_kv4_sync_status": (_S, [_P, _P]),
}.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args


def _empty(shape, dtype, device, stream):
    """Device memory that a call on `stream` writes, from that stream's own pool:
    what another stream gave back it may still be working on."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(stream)) if int(stream) else \
            torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _on_device(x, what, device=None):
    """The GPU that x lies on; a ValueError where that is none, or not `device`:
    an address of another memory must not reach a kernel."""
    at = x.get_device()
    if at < 0 or device is not None and at != device:
        raise ValueError(f"{what} must lie on the GPU"
                         + ("" if device is None else f" cuda:{device}")
                         + f", not on {x.device}")
    return at


def _given_workspace(x, device):
    _on_device(x, "workspace", device)
    if not x.is_contiguous():
        raise ValueError("workspace must be contiguous")


def _scratch(nbytes, device, stream):
    """Device scratch for one call on `stream`."""
    return _empty(max(nbytes, 16), torch.uint8, device, stream)


def _stream_of(cache, stream):
    """A call's stream; a ValueError where kernels would run on another device
    than the cache's."""
    if _raw_device is not None:
        now = _raw_device()
        if now != cache._device:
            raise ValueError(f"the cache lies on cuda:{cache._device}, the "
                             f"current device is cuda:{now}")
        if stream is None and _raw_stream is not None:
            return _raw_stream(now)
    return _stream(stream)


class Kv4Cache:
    """A full-context cache held in 4 bits (kvr_kv4_*; the format stands in
    include/kvr.h): owner of the handle and of the torch buffer it lives in.
    What a call allocates, outputs that it was not given among them, belongs to
    the call's stream, as tensors do that are made under torch.cuda.stream.
    Calls run on the current device, which has to be the cache's."""

    _at = _stream_of

    def __init__(self, n_seq, n_layers, n_kv_heads, group, head_dim, capacity,
                 dtype="bf16", out_dtype="bf16", softmax_scale=0.0,
                 device="cuda", stream=None, buf=None):
        """dtype: element type of q, k and v.  buf: an optional caller-owned
        uint8 device tensor of at least kvr_kv4_required_bytes (256-byte
        aligned); by default one is allocated."""
        self.desc = make_desc(n_seq, n_layers, n_kv_heads, group, head_dim,
                              capacity, dtype, out_dtype, softmax_scale)
        self.S, self.L, self.H, self.G, self.d = (n_seq, n_layers, n_kv_heads,
                                                  group, head_dim)
        self.cap = capacity
        self.dtype, self.out_dtype = dtype, out_dtype
        self._io, self._out = TORCH_DTYPES[dtype], TORCH_DTYPES[out_dtype]
        self._all, self._scores = (0, n_layers), None
        self.nbytes = int(lib.kvr_kv4_required_bytes(ctypes.byref(self.desc)))
        if self.nbytes == 0:
            raise KvrError(KVR_EINVAL, "Kv4Cache", "invalid descriptor")
        if buf is None:
            buf = _empty(self.nbytes, torch.uint8, device, stream)
        elif buf.numel() < self.nbytes or buf.dtype != torch.uint8:
            raise ValueError("buf must be uint8 with at least "
                             f"{self.nbytes} bytes")
        self.buf = buf
        self._device = _on_device(buf, "buf")
        h = _P()
        _check(lib.kvr_kv4_create(ctypes.byref(self.desc), _ptr(buf),
                                  self.nbytes, self._at(stream),
                                  ctypes.byref(h)), "kvr_kv4_create")
        self.handle = h

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            lib.kvr_kv4_destroy(h)
            self.handle = None

    def _rows(self, x, shape, what):
        """The address of x, a dense tensor of the cache's element type on the
        cache's device."""
        if x.shape != shape or x.dtype is not self._io or \
                not x.is_contiguous():
            raise ValueError(f"{what} must be contiguous {self.dtype} "
                             f"{list(shape)}, not {x.dtype} {list(x.shape)}")
        if x.get_device() != self._device:
            _on_device(x, what, self._device)  # raises
        return x.data_ptr()

    def _counts(self, x, what="counts"):
        """A host int32 array of one value a sequence, or None."""
        if x is None:
            return None
        a = np.ascontiguousarray(x, dtype=np.int32)
        if a.shape != (self.S,):
            raise ValueError(f"{what} must be {self.S} whole numbers")
        return a

    def load(self, seq, k, v, stream=None):
        """Replace a sequence: k, v [L][H][n][d] (kvr_kv4_load)."""
        shape = (self.L, self.H, k.shape[2], self.d)
        _check(lib.kvr_kv4_load(self.handle, seq, self._rows(k, shape, "k"),
                                self._rows(v, shape, "v"), shape[2],
                                self._at(stream)), "kvr_kv4_load")

    def append(self, k, v, counts=None, layers=None, stream=None):
        """Append tokens: k, v [S][nl][n][H][d]; counts: how many of them each
        sequence has (kvr_kv4_append)."""
        lb, le = layers or self._all
        shape = (self.S, le - lb, k.shape[2], self.H, self.d)
        counts = self._counts(counts)
        _check(lib.kvr_kv4_append(
            self.handle, lb, le, shape[2],
            None if counts is None else counts.ctypes.data,
            self._rows(k, shape, "k"), self._rows(v, shape, "v"),
            self._at(stream)), "kvr_kv4_append")

    def truncate(self, lens):
        """Each sequence keeps its first lens[s] rows (kvr_kv4_truncate)."""
        lens = self._counts(lens, "lens")
        _check(lib.kvr_kv4_truncate(
            self.handle, None if lens is None else lens.ctypes.data),
            "kvr_kv4_truncate")

    def lengths(self):
        a = np.zeros((self.S, self.L), np.int32)
        _check(lib.kvr_kv4_lengths(self.handle, _ptr(a)), "kvr_kv4_lengths")
        return a

    def read_newest(self, n, counts=None, layers=None, stream=None):
        """What the newest n rows stand for: (k, v) [S][nl][H][n][d]
        (kvr_kv4_read)."""
        lb, le = layers or self._all
        counts = self._counts(counts)
        shape = (self.S, le - lb, self.H, n, self.d)
        k, v = (_empty(shape, self._io, self.buf.device, stream)
                for _ in range(2))
        _check(lib.kvr_kv4_read(self.handle, lb, le, n,
                                None if counts is None else counts.ctypes.data,
                                k.data_ptr(), v.data_ptr(), self._at(stream)),
               "kvr_kv4_read")
        return k, v

    def attend_workspace(self, n_q, layers=None):
        """A workspace for attend() of up to n_q tokens over these layers."""
        lb, le = layers or self._all
        n = int(lib.kvr_kv4_attend_workspace_bytes(self.handle, lb, le, n_q))
        return torch.empty(n, dtype=torch.uint8, device=self.buf.device)

    def attend(self, q, out=None, counts=None, layers=None, scores=False,
               workspace=None, stream=None):
        """Attention of the newest tokens: q [S][nl][n][H*G][d] -> out, the
        same shape in out_dtype; scores: add each row's accumulated attention
        weight (kvr_kv4_attend)."""
        lb, le = layers or self._all
        shape = (self.S, le - lb, q.shape[2], self.H * self.G, self.d)
        qp = self._rows(q, shape, "q")
        counts = self._counts(counts)
        if out is None:
            out = _empty(shape, self._out, q.device, stream)
        elif out.shape != shape or out.dtype is not self._out or \
                not out.is_contiguous():
            raise ValueError(f"out must be contiguous {self.out_dtype} "
                             f"{list(shape)}")
        elif out.get_device() != self._device:
            _on_device(out, "out", self._device)  # raises
        if workspace is None:
            workspace = _scratch(int(lib.kvr_kv4_attend_workspace_bytes(
                self.handle, lb, le, shape[2])), q.device, stream)
        else:
            _given_workspace(workspace, self._device)
        _check(lib.kvr_kv4_attend(
            self.handle, lb, le, shape[2],
            None if counts is None else counts.ctypes.data, qp,
            out.data_ptr(), 1 if scores else 0, workspace.data_ptr(),
            workspace.nbytes, self._at(stream)), "kvr_kv4_attend")
        return out

    def evict_into(self, cache: Cache, budget, window, stream=None):
        """Cut every sequence into an evicted cache (kvr_kv4_evict)."""
        if not isinstance(cache, Cache):
            raise ValueError(f"the destination must be a Cache, not {cache!r}")
        _on_device(cache.buf, "the destination", self._device)
        _check(lib.kvr_kv4_evict(self.handle, cache.handle, budget, window,
                                 self._at(stream)), "kvr_kv4_evict")

    def scores_view(self):
        """The scores as a device tensor viewing the buffer,
        [S][L][H][capacity]; it may be written."""
        if self._scores is None:  # the buffer stays where it is
            p, stride = _P(), ctypes.c_int64()
            _check(lib.kvr_kv4_scores(self.handle, ctypes.byref(p),
                                      ctypes.byref(stride)), "kvr_kv4_scores")
            off = p.value - self.buf.data_ptr()
            n = self.S * self.L * self.H * stride.value
            self._scores = self.buf[off:off + 4 * n].view(torch.float32).view(
                self.S, self.L, self.H, stride.value)[..., :self.cap]
        return self._scores

    def launch_count(self):
        n = ctypes.c_uint64()
        _check(lib.kvr_kv4_launch_count(self.handle, ctypes.byref(n)),
               "kvr_kv4_launch_count")
        return int(n.value)

    def sync_status(self, stream=None):
        _check(lib.kvr_kv4_sync_status(self.handle, self._at(stream)),
               "kvr_kv4_sync_status")


# ---- the full context in pages ----------------------------------------------

class kvr_paged_desc(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int), ("n_layers", ctypes.c_int),
                ("n_kv_heads", ctypes.c_int), ("group", ctypes.c_int),
                ("head_dim", ctypes.c_int), ("n_pages", ctypes.c_int),
                ("page_rows", ctypes.c_int), ("table_pages", ctypes.c_int),
                ("kv_dtype", ctypes.c_int), ("out_dtype", ctypes.c_int),
                ("softmax_scale", ctypes.c_float)]


for _name, (_res, _args) in {
    "kvr_paged_required_bytes": (ctypes.c_size_t,
                                 [ctypes.POINTER(kvr_paged_desc)]),
    "kvr_paged_create": (_S, [ctypes.POINTER(kvr_paged_desc), _P,
                              ctypes.c_size_t, _P, ctypes.POINTER(_P)]),
    "kvr_paged_destroy": (None, [_P]),
    "kvr_paged_plan": (_S, [_P, _P, _I, _P, _P]),
    "kvr_paged_append": (_S, [_P, _I, _I, _I, _I, _P, _P, _P, _P]),
    "kvr_paged_attend_workspace_bytes": (ctypes.c_size_t, [_P, _I, _I]),
    "kvr_paged_attend": (_S, [_P, _I, _I, _P, _P, _P, ctypes.c_size_t, _P]),
    "kvr_paged_attend_pages_workspace_bytes": (ctypes.c_size_t,
                                               [_P, _I, _I, _I, _I]),
    "kvr_paged_attend_pages": (_S, [_P, _I, _I, _P, _I, _I, _P, _P, _P,
                                    ctypes.c_size_t, _P]),
    "kvr_paged_tables": (_S, [_P, _P, _P, _P, _P]),
    "kvr_paged_rows": (_S, [_P, _P, _P, _P]),
    "kvr_paged_launch_count": (_S, [_P, _P]),
    "kvr_paged_sync_status": (_S, [_P, _P]),
}.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args


class PagedCache:
    """Full contexts in pages of a shared pool (kvr_paged_*; include/kvr.h says
    how they are kept): owner of the handle and of the torch buffer it lives in.
    What a call allocates belongs to the call's stream, as with Kv4Cache.
    Calls run on the current device, which has to be the cache's."""

    @staticmethod
    def make_desc(n_seq, n_layers, n_kv_heads, group, head_dim, n_pages,
                  page_rows=64, table_pages=None, dtype="bf16",
                  out_dtype="bf16", softmax_scale=0.0):
        """table_pages: pages a sequence may hold, by default the whole pool.
        Workspaces of attend_pages grow with it, and a call of few sequences is
        faster where it is no more than they need."""
        return kvr_paged_desc(
            n_seq, n_layers, n_kv_heads, group, head_dim, n_pages, page_rows,
            n_pages if table_pages is None else table_pages, DTYPES[dtype],
            DTYPES[out_dtype], float(softmax_scale))

    @staticmethod
    def required_bytes(*args, **kw):
        """Bytes of the buffer, for __init__'s arguments up to softmax_scale."""
        d = PagedCache.make_desc(*args, **kw)
        return int(lib.kvr_paged_required_bytes(ctypes.byref(d)))

    def __init__(self, n_seq, n_layers, n_kv_heads, group, head_dim, n_pages,
                 page_rows=64, table_pages=None, dtype="bf16",
                 out_dtype="bf16", softmax_scale=0.0, device="cuda",
                 stream=None, buf=None):
        """dtype: element type of q, k and v.  buf: an optional caller-owned
        uint8 device tensor of at least required_bytes(...) (256-byte aligned);
        by default one is allocated."""
        self.desc = self.make_desc(n_seq, n_layers, n_kv_heads, group,
                                   head_dim, n_pages, page_rows, table_pages,
                                   dtype, out_dtype, softmax_scale)
        self.S, self.L, self.H, self.G, self.d = (n_seq, n_layers, n_kv_heads,
                                                  group, head_dim)
        self._hg = n_kv_heads * group
        self.n_pages, self.page_rows = n_pages, page_rows
        self.table_pages = self.desc.table_pages
        self.dtype, self.out_dtype = dtype, out_dtype
        self._io, self._out = TORCH_DTYPES[dtype], TORCH_DTYPES[out_dtype]
        self._all, self._tables, self._pool = (0, n_layers), None, None
        self.nbytes = int(lib.kvr_paged_required_bytes(ctypes.byref(self.desc)))
        if self.nbytes == 0:
            raise KvrError(KVR_EINVAL, "PagedCache", "invalid descriptor")
        if buf is None:
            buf = _empty(self.nbytes, torch.uint8, device, stream)
        elif buf.numel() < self.nbytes or buf.dtype != torch.uint8 or \
                not buf.is_contiguous():
            raise ValueError("buf must be contiguous uint8 with at least "
                             f"{self.nbytes} bytes")
        self.buf = buf
        self._device = _on_device(buf, "buf")
        h = _P()
        _check(lib.kvr_paged_create(ctypes.byref(self.desc), _ptr(buf),
                                    self.nbytes, self._at(stream),
                                    ctypes.byref(h)), "kvr_paged_create")
        self.handle = h

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            lib.kvr_paged_destroy(h)
            self.handle = None

    _at = _stream_of

    def _tensor(self, x, shape, dtype, what):
        """The address of x, a dense tensor of this shape on the cache's
        device."""
        if x.shape != shape or x.dtype is not dtype or not x.is_contiguous():
            raise ValueError(f"{what} must be contiguous {dtype} "
                             f"{list(shape)}, not {x.dtype} {list(x.shape)}")
        if x.get_device() != self._device:
            _on_device(x, what, self._device)  # raises
        return x.data_ptr()

    def plan(self, lens, n_new=0, slots=None, stream=None):
        """The sequences' lengths become lens (int32 [S] on the device); returns
        the slots [S][n_new] of the tokens they grow by, None where n_new is 0
        (kvr_paged_plan).  Where one grows by more than n_new tokens or the free
        pages do not reach, nothing changes, every slot is -1, and
        sync_status() raises."""
        at = self._at(stream)
        want = self._tensor(lens, (self.S,), torch.int32, "lens")
        if n_new < 0 or n_new > 1 << 24:
            raise ValueError(f"{n_new} new tokens")
        if slots is None and n_new:
            slots = _empty((self.S, n_new), torch.int32, self.buf.device,
                           stream)
        to = None if slots is None else self._tensor(
            slots, (self.S, n_new), torch.int32, "slots")
        _check(lib.kvr_paged_plan(self.handle, want, n_new,
                                  to if n_new else None, at), "kvr_paged_plan")
        return slots

    def append(self, k, v, slots, layers=None, stream=None):
        """New tokens' keys and values: k, v [n][nl][n_new][H][d], slots int32
        [n][n_new], rows of a plan's (kvr_paged_append)."""
        lb, le = layers or self._all
        n, n_new = slots.shape
        shape = (n, le - lb, n_new, self.H, self.d)
        _check(lib.kvr_paged_append(
            self.handle, lb, le, n, n_new,
            self._tensor(slots, (n, n_new), torch.int32, "slots"),
            self._tensor(k, shape, self._io, "k"),
            self._tensor(v, shape, self._io, "v"), self._at(stream)),
            "kvr_paged_append")

    def _workspace(self, name, *args):
        n = int(getattr(lib, name)(self.handle, *args))
        if n == 0:
            raise KvrError(KVR_EINVAL, name, "invalid arguments")
        return torch.empty(n, dtype=torch.uint8, device=self.buf.device)

    def attend_workspace(self, layers=None):
        """A workspace for attend() over these layers."""
        return self._workspace("kvr_paged_attend_workspace_bytes",
                               *(layers or self._all))

    def attend_pages_workspace(self, budget, window=1, layers=None):
        """A workspace for attend_pages() with this choice over these layers."""
        return self._workspace("kvr_paged_attend_pages_workspace_bytes",
                               *(layers or self._all), budget, window)

    def _outputs(self, q, out, shape, stream):
        """The output tensor: `out`, or a new one.  (A call a layer spends its time
        on the host, so what is usual is asked without another call.)"""
        at = self._device
        if q.shape != shape or q.dtype is not self._io or \
                not q.is_contiguous() or q.get_device() != at:
            self._tensor(q, shape, self._io, "q")  # raises
        if out is None:
            return _empty(shape, self._out, q.device, stream)
        if out.shape != shape or out.dtype is not self._out or \
                not out.is_contiguous() or out.get_device() != at:
            self._tensor(out, shape, self._out, "out")  # raises
        return out

    def _given(self, workspace):
        if workspace.get_device() != self._device or \
                not workspace.is_contiguous():
            _given_workspace(workspace, self._device)  # raises
        return workspace

    def attend(self, q, out=None, layers=None, workspace=None, stream=None):
        """Attention of each sequence's newest token: q [S][nl][H*G][d] -> out,
        the same shape in out_dtype (kvr_paged_attend)."""
        lb, le = layers or self._all
        at = self._at(stream)
        out = self._outputs(q, out, (self.S, le - lb, self._hg, self.d),
                            stream)
        workspace = self._given(workspace) if workspace is not None else \
            _scratch(int(lib.kvr_paged_attend_workspace_bytes(
                self.handle, lb, le)), q.device, stream)
        st = lib.kvr_paged_attend(self.handle, lb, le, q.data_ptr(),
                                  out.data_ptr(), workspace.data_ptr(),
                                  workspace.nbytes, at)
        if st:
            _check(st, "kvr_paged_attend")
        return out

    def attend_pages(self, q, budget, window=1, out=None, pages=None,
                     layers=None, workspace=None, stream=None):
        """The same over each unit's window newest pages and the budget others
        of the greatest score (kvr_paged_attend_pages); pages: an int32 tensor
        [S][nl][H][budget + window] for the choice."""
        lb, le = layers or self._all
        at = self._at(stream)
        out = self._outputs(q, out, (self.S, le - lb, self._hg, self.d),
                            stream)
        to = None if pages is None else self._tensor(
            pages, (self.S, le - lb, self.H, budget + window), torch.int32,
            "pages")
        workspace = self._given(workspace) if workspace is not None else \
            _scratch(int(lib.kvr_paged_attend_pages_workspace_bytes(
                self.handle, lb, le, budget, window)), q.device, stream)
        st = lib.kvr_paged_attend_pages(
            self.handle, lb, le, q.data_ptr(), budget, window, out.data_ptr(),
            to, workspace.data_ptr(), workspace.nbytes, at)
        if st:
            _check(st, "kvr_paged_attend_pages")
        return out

    def tables_view(self):
        """(table [S][table_pages], lens [S], free pages [1]) as device tensors
        viewing the buffer, to be read only."""
        if self._tables is None:  # the buffer stays where it is
            p = [_P() for _ in range(3)]
            stride = ctypes.c_int64()
            _check(lib.kvr_paged_tables(
                self.handle, ctypes.byref(p[0]), ctypes.byref(stride),
                ctypes.byref(p[1]), ctypes.byref(p[2])), "kvr_paged_tables")
            self._tables = tuple(
                self._view(at, shape, torch.int32)
                for at, shape in zip(p, ((self.S, stride.value), (self.S,),
                                         (1,))))
        return self._tables

    def _view(self, at, shape, dtype):
        off = at.value - self.buf.data_ptr()
        n = int(np.prod(shape, dtype=np.int64)) * dtype.itemsize
        return self.buf.view(-1)[off:off + n].view(dtype).view(shape)

    def _views(self):
        if self._pool is None:
            p = [_P() for _ in range(3)]
            _check(lib.kvr_paged_rows(self.handle, *map(ctypes.byref, p)),
                   "kvr_paged_rows")
            lead = (self.L, self.n_pages, self.H)
            self._pool = tuple(
                self._view(at, (*lead, rows, self.d), self._io)
                for at, rows in zip(p, (self.page_rows, self.page_rows, 2)))
        return self._pool

    def rows_view(self):
        """(K, V) as device tensors viewing the buffer, each
        [L][n_pages][H][page_rows][d], to be read only."""
        return self._views()[:2]

    def bounds_view(self):
        """The least and greatest keys of full pages, [L][n_pages][H][2][d], as
        a device tensor viewing the buffer, to be read only."""
        return self._views()[2]

    def launch_count(self):
        n = ctypes.c_uint64()
        _check(lib.kvr_paged_launch_count(self.handle, ctypes.byref(n)),
               "kvr_paged_launch_count")
        return int(n.value)

    def sync_status(self, stream=None):
        _check(lib.kvr_paged_sync_status(self.handle, self._at(stream)),
               "kvr_paged_sync_status")


# ---- verification of drafted tokens -----------------------------------------

class kvr_verify_desc(ctypes.Structure):
    _fields_ = [("n_seq", ctypes.c_int), ("n_draft", ctypes.c_int),
                ("vocab", ctypes.c_int), ("temperature", ctypes.c_float),
                ("logits_dtype", ctypes.c_int)]


for _name, (_res, _args) in {
    "kvr_verify_workspace_bytes": (ctypes.c_size_t,
                                   [ctypes.POINTER(kvr_verify_desc)]),
    "kvr_verify_drafts": (_S, [ctypes.POINTER(kvr_verify_desc), _P,
                               ctypes.c_int64, _P, ctypes.c_int64, _P, _P, _P,
                               _P, _P, _P, _P, ctypes.c_size_t, _P]),
}.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args

_LOGITS = {torch.bfloat16: KVR_BF16, torch.float32: KVR_F32}


def verify_workspace(n_seq, n_draft, vocab, device="cuda"):
    """A workspace for verify_drafts() of these sizes."""
    d = kvr_verify_desc(n_seq, n_draft, vocab, 1.0, KVR_BF16)
    n = int(lib.kvr_verify_workspace_bytes(ctypes.byref(d)))
    if n == 0:
        raise KvrError(KVR_EINVAL, "verify_workspace", "invalid descriptor")
    return torch.empty(n, dtype=torch.uint8, device=device)


def _logit_rows(x, what):
    """Row stride of logits [S][n][V]: a row's logits side by side, the rows one
    stride apart, which is V at least where there is more than one of them."""
    S, n, V = x.shape
    if x.is_contiguous():
        return V
    rows, col = x.stride()[1:] if n > 1 else (x.stride(0), x.stride(2))
    if col != 1 and V > 1 or S > 1 and x.stride(0) != n * rows:
        raise ValueError(f"{what}: rows must lie one stride apart")
    if S * n > 1 and rows < V:
        raise ValueError(f"{what}: rows must not overlap (stride {rows} of "
                         f"{V} logits)")
    return max(rows, V)


def verify_drafts(target, draft, tokens, u, race, n_draft=None,
                  temperature=1.0, accepted=None, out_tokens=None,
                  workspace=None, stream=None):
    """Accept or reject drafted tokens (kvr_verify_drafts): target logits
    [S][T + 1][V], draft logits [S][T][V], tokens int32 and u fp32 [S][T], race
    fp32 [S][V] (exponential, > 0), n_draft int32 [S] or None; temperature > 0
    (0 is refused).  Returns (accepted [S], tokens [S][T + 1]) on the device;
    where they are not given they belong to the call's stream."""
    S, n, V = target.shape
    T = n - 1
    if draft.shape != (S, T, V) or draft.dtype is not target.dtype or \
            target.dtype not in _LOGITS:
        raise ValueError(f"target and draft must be bf16 or f32 {[S, n, V]} "
                         f"and {[S, T, V]}")
    device = _on_device(target, "target")
    if T and draft.get_device() != device:
        _on_device(draft, "draft", device)  # raises
    ts = _logit_rows(target, "target")
    ds = _logit_rows(draft, "draft") if T else V
    for x, name, shape, dt in (
            (tokens, "tokens", (S, T), torch.int32),
            (u, "u", (S, T), torch.float32),
            (race, "race", (S, V), torch.float32),
            (n_draft, "n_draft", (S,), torch.int32),
            (accepted, "accepted", (S,), torch.int32),
            (out_tokens, "out_tokens", (S, n), torch.int32)):
        if x is None:
            continue
        if x.shape != shape or x.dtype is not dt or not x.is_contiguous():
            raise ValueError(f"{name} must be contiguous {dt} {list(shape)}")
        if x.get_device() != device and x.numel():  # (no drafts: empty)
            _on_device(x, name, device)  # raises
    dev = target.device
    if accepted is None:
        accepted = _empty(S, torch.int32, dev, stream)
    if out_tokens is None:
        out_tokens = _empty((S, n), torch.int32, dev, stream)
    d = kvr_verify_desc(S, T, V, temperature, _LOGITS[target.dtype])
    if workspace is None:
        workspace = _scratch(int(lib.kvr_verify_workspace_bytes(
            ctypes.byref(d))), dev, stream)
    else:
        _given_workspace(workspace, device)
    _check(lib.kvr_verify_drafts(
        ctypes.byref(d), target.data_ptr(), ts, draft.data_ptr(), ds,
        tokens.data_ptr(), u.data_ptr(), race.data_ptr(),
        None if n_draft is None else n_draft.data_ptr(), accepted.data_ptr(),
        out_tokens.data_ptr(), workspace.data_ptr(), workspace.nbytes,
        _stream(stream)), "kvr_verify_drafts")
    return accepted, out_tokens
