"""ctypes binding of the LESS C-ABI library (include/less.h).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  The functions carry the C names.  There is no CPU fallback: loading
fails loudly when the library has not been built, and nothing here computes.
torch is used for device memory and streams.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os
from typing import Dict, Optional, Sequence

import numpy as np
import torch

from . import build as _build

LESS_OK = 0
LESS_SCORE_NORM_SPARSE = 1
LESS_NO_STATE = 2
LESS_POLICY_LAMBDA = 4
LESS_POLICY_TOVA = 8
LESS_WITH_PARALLEL_FORM = 16
LESS_OUT_F16 = 32

EXPORTED = [
    "less_arena_bytes", "less_create", "less_prefill", "less_decode_step", "less_position",
    "less_state_record_bytes", "less_export_state", "less_import_state",
    "less_read_feature_maps", "less_poll_status", "less_launch_count", "less_strerror",
    "less_destroy", "less_decode_step_host", "less_profile", "less_profile_read",
    "less_prompt_scores_noalloc", "less_masked_attention", "less_kernel_variant",
    "less_last_status_where", "less_selftest_wait_timeout",
    "less_pages_workspace_bytes", "less_pages_reset", "less_pages_resize", "less_pages_fork",
    "less_pages_trim", "less_pages_compact", "less_pages_write", "less_pages_attention",
    "less_pages_poll_status",
]
LESS_NOALLOC_MAX_ROWS = 65536
LESS_ERR_NOALLOC_TOO_LARGE = -12
LESS_ERR_PAGES_EXHAUSTED = -13
LESS_PAGES_E4M3 = 1
LESS_PAGES_BF16 = 2
LESS_PAGE_BLOCK = 16

KERNEL_NAMES = ["feature_map", "decode", "rowstat", "colsum", "attn_out", "select", "build", "finalize",
                "psi", "gather", "masked_pack", "masked_out"]


class less_config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("layers", C.c_int32), ("heads", C.c_int32),
                ("head_dim", C.c_int32), ("rank", C.c_int32), ("hidden", C.c_int32),
                ("heavy", C.c_int32), ("recent", C.c_int32), ("max_prompt", C.c_int32),
                ("max_prefill_layers", C.c_int32), ("flags", C.c_uint32), ("group", C.c_int32)]


class less_weights(C.Structure):
    _fields_ = [("w_phi1", C.c_void_p), ("w_phi2", C.c_void_p), ("w_psi1", C.c_void_p),
                ("w_psi2", C.c_void_p), ("w_psi3", C.c_void_p), ("psi_scale", C.c_void_p)]


class less_pages(C.Structure):
    _fields_ = [("layers", C.c_int32), ("heads", C.c_int32), ("group", C.c_int32), ("head_dim", C.c_int32),
                ("page_tokens", C.c_int32), ("pages", C.c_int32), ("seqs", C.c_int32), ("seq_pages", C.c_int32),
                ("flags", C.c_uint32), ("codes", C.c_void_p), ("amax", C.c_void_p), ("table", C.c_void_p),
                ("lens", C.c_void_p), ("refs", C.c_void_p), ("workspace", C.c_void_p),
                ("workspace_bytes", C.c_size_t)]


class LessError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {less_strerror(code)} ({code})")


_lib = None


def lib() -> C.CDLL:
    """Loads libless_b200.so (built in-tree).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.LIB_PATH
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is missing: build it with `python -m paper_2402_09398_b200.build` "
            "(there is no CPU fallback)")
    L = C.CDLL(path)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    L.less_arena_bytes.restype = sz
    L.less_arena_bytes.argtypes = [C.POINTER(less_config)]
    L.less_state_record_bytes.restype = sz
    L.less_state_record_bytes.argtypes = [C.POINTER(less_config)]
    L.less_create.restype = C.c_int
    L.less_create.argtypes = [C.POINTER(less_config), C.POINTER(less_weights), vp, sz, C.POINTER(vp)]
    L.less_prefill.restype = C.c_int
    L.less_prefill.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp]
    L.less_decode_step.restype = C.c_int
    L.less_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    L.less_decode_step_host.restype = C.c_int
    L.less_decode_step_host.argtypes = [vp, vp, vp, vp, vp, vp]
    L.less_profile.restype = C.c_int
    L.less_profile.argtypes = [vp, C.c_int]
    L.less_profile_read.restype = C.c_int
    L.less_profile_read.argtypes = [vp, vp, vp]
    L.less_prompt_scores_noalloc.restype = C.c_int
    L.less_prompt_scores_noalloc.argtypes = [vp, vp, i32, i32, vp, vp]
    L.less_position.restype = i64
    L.less_position.argtypes = [vp]
    L.less_launch_count.restype = i64
    L.less_launch_count.argtypes = [vp]
    L.less_export_state.restype = C.c_int
    L.less_export_state.argtypes = [vp, vp, i32, vp, sz, vp]
    L.less_import_state.restype = C.c_int
    L.less_import_state.argtypes = [vp, vp, i32, vp, sz, vp]
    L.less_masked_attention.restype = C.c_int
    L.less_masked_attention.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    L.less_read_feature_maps.restype = C.c_int
    L.less_read_feature_maps.argtypes = [vp, vp, vp, vp]
    L.less_poll_status.restype = C.c_int
    L.less_poll_status.argtypes = [vp, vp]
    L.less_strerror.restype = C.c_char_p
    L.less_strerror.argtypes = [C.c_int]
    L.less_destroy.restype = C.c_int
    L.less_destroy.argtypes = [vp]
    L.less_kernel_variant.restype = C.c_char_p
    L.less_kernel_variant.argtypes = [vp, C.c_int]
    L.less_last_status_where.restype = C.c_int
    L.less_last_status_where.argtypes = [vp]
    L.less_selftest_wait_timeout.restype = C.c_int
    L.less_selftest_wait_timeout.argtypes = [vp, C.c_uint32, vp]
    pg = C.POINTER(less_pages)
    L.less_pages_workspace_bytes.restype = sz
    L.less_pages_workspace_bytes.argtypes = [pg]
    for name, args in (("reset", [vp]), ("resize", [i32, vp, vp, vp]), ("fork", [i32, vp, vp, vp]),
                       ("trim", [i32, vp, i32, i32, vp]), ("compact", [vp]),
                       ("write", [i32, i32, i32, vp, vp, i32, vp, i64, vp, i64, vp]),
                       ("attention", [i32, i32, i32, vp, vp, i32, i32, vp, i64, i32, i32, C.c_float, vp, vp]),
                       ("poll_status", [vp])):
        fn = getattr(L, "less_pages_" + name)
        fn.restype = C.c_int
        fn.argtypes = [pg] + args
    _lib = L
    return L


# --------------------------------------------------------------------------- #
# the C calls, same names
# --------------------------------------------------------------------------- #
def less_strerror(code: int) -> str:
    return lib().less_strerror(int(code)).decode()


def less_arena_bytes(cfg: less_config) -> int:
    return int(lib().less_arena_bytes(C.byref(cfg)))


def less_state_record_bytes(cfg: less_config) -> int:
    return int(lib().less_state_record_bytes(C.byref(cfg)))


def less_create(cfg: less_config, weights: less_weights, arena_ptr: int, arena_bytes: int):
    out = C.c_void_p()
    rc = lib().less_create(C.byref(cfg), C.byref(weights), arena_ptr, arena_bytes, C.byref(out))
    return rc, out


def less_prefill(ctx, layer_begin, layer_count, prompt_len, Q, K, V, attn_out, stream) -> int:
    return lib().less_prefill(ctx, layer_begin, layer_count, prompt_len, Q, K, V, attn_out, stream)


def less_decode_step(ctx, q, k, v, out, evicted_pos, stream) -> int:
    return lib().less_decode_step(ctx, q, k, v, out, evicted_pos, stream)


def less_decode_step_host(ctx, q_host, k_host, v_host, out_host, stream) -> int:
    return lib().less_decode_step_host(ctx, q_host, k_host, v_host, out_host, stream)


def less_profile(ctx, enable: int) -> int:
    return lib().less_profile(ctx, int(enable))


def less_profile_read(ctx, ms_ptr, launches_ptr) -> int:
    return lib().less_profile_read(ctx, ms_ptr, launches_ptr)


def less_prompt_scores_noalloc(Q, K, n_inst, prompt_len, acc_out, stream) -> int:
    """H2O prompt scores for callers that cannot allocate device memory (a
    process whose pool owns the GPU, a plugin handed only buffers and a stream):
    the scratch lives in a fixed array inside the library.  Device pointers in,
    return code out; at most LESS_NOALLOC_MAX_ROWS rows (n_inst * prompt_len);
    calls that may overlap on the GPU race on the shared array."""
    return lib().less_prompt_scores_noalloc(Q, K, n_inst, prompt_len, acc_out, stream)


def less_position(ctx) -> int:
    return int(lib().less_position(ctx))


def less_launch_count(ctx) -> int:
    return int(lib().less_launch_count(ctx))


def less_export_state(ctx, inst_ptr, n, host_ptr, nbytes, stream) -> int:
    return lib().less_export_state(ctx, inst_ptr, n, host_ptr, nbytes, stream)


def less_import_state(ctx, inst_ptr, n, host_ptr, nbytes, stream) -> int:
    return lib().less_import_state(ctx, inst_ptr, n, host_ptr, nbytes, stream)


def less_masked_attention(ctx, layer_begin, layer_count, seq_len, Q, K, V, exact_until, out, stream) -> int:
    return lib().less_masked_attention(ctx, layer_begin, layer_count, seq_len, Q, K, V, exact_until, out, stream)


def less_read_feature_maps(ctx, phi_ptr, psi_ptr, stream) -> int:
    return lib().less_read_feature_maps(ctx, phi_ptr, psi_ptr, stream)


def less_poll_status(ctx, stream) -> int:
    return lib().less_poll_status(ctx, stream)


def less_destroy(ctx) -> int:
    return lib().less_destroy(ctx)


def less_kernel_variant(ctx, kernel_id: int) -> str:
    return lib().less_kernel_variant(ctx, int(kernel_id)).decode()


def less_last_status_where(ctx) -> int:
    return int(lib().less_last_status_where(ctx))


def less_selftest_wait_timeout(ctx, polls: int, stream) -> int:
    return lib().less_selftest_wait_timeout(ctx, int(polls), stream)


def less_pages_workspace_bytes(cache: less_pages) -> int:
    return int(lib().less_pages_workspace_bytes(C.byref(cache)))


def less_pages_reset(cache: less_pages, stream) -> int:
    return lib().less_pages_reset(cache, stream)


def less_pages_resize(cache: less_pages, n, seqs, lens, stream) -> int:
    return lib().less_pages_resize(cache, n, seqs, lens, stream)


def less_pages_fork(cache: less_pages, n, src, dst, stream) -> int:
    return lib().less_pages_fork(cache, n, src, dst, stream)


def less_pages_trim(cache: less_pages, n, seqs, sinks, window, stream) -> int:
    return lib().less_pages_trim(cache, n, seqs, sinks, window, stream)


def less_pages_compact(cache: less_pages, stream) -> int:
    return lib().less_pages_compact(cache, stream)


def less_pages_write(cache: less_pages, layer_begin, layer_count, n, seqs, starts, rows, k, k_stride, v, v_stride,
                     stream) -> int:
    return lib().less_pages_write(cache, layer_begin, layer_count, n, seqs, starts, rows, k, k_stride, v, v_stride,
                                  stream)


def less_pages_attention(cache: less_pages, layer_begin, layer_count, n, seqs, starts, rows, max_new, q, q_stride,
                         window, sinks, scale, out, stream) -> int:
    return lib().less_pages_attention(cache, layer_begin, layer_count, n, seqs, starts, rows, max_new, q, q_stride,
                                      window, sinks, scale, out, stream)


def less_pages_poll_status(cache: less_pages, stream) -> int:
    return lib().less_pages_poll_status(cache, stream)


# --------------------------------------------------------------------------- #
# convenience holder: owns the torch buffers the context borrows
# --------------------------------------------------------------------------- #
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _check(rc: int, where: str) -> None:
    if rc != LESS_OK:
        raise LessError(rc, where)


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream


class LessContext:
    """Allocates the arena with torch, keeps the weights alive, forwards calls."""

    def __init__(self, batch, layers, heads, head_dim, rank, hidden, heavy, recent, max_prompt,
                 weights: Dict[str, torch.Tensor], max_prefill_layers: int = 1, flags: int = 0,
                 psi_scale: Optional[torch.Tensor] = None, device="cuda", group: int = 1):
        if not torch.cuda.is_available():
            raise RuntimeError("the LESS library needs a CUDA device (there is no CPU path)")
        lib()
        self.device = torch.device(device)
        self.cfg = less_config(batch, layers, heads, head_dim, rank, hidden, heavy, recent,
                               max_prompt, max_prefill_layers, flags, group)
        nbytes = less_arena_bytes(self.cfg)
        if nbytes == 0:
            raise LessError(-1, "less_arena_bytes")
        self.weights = {k: v.to(self.device).contiguous() for k, v in weights.items()}
        self.psi_scale = None if psi_scale is None else psi_scale.to(self.device, torch.float32).contiguous()
        self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        w = less_weights(*(self.weights[n].data_ptr() for n in
                           ("w_phi1", "w_phi2", "w_psi1", "w_psi2", "w_psi3")), _ptr(self.psi_scale))
        torch.cuda.synchronize()
        rc, ctx = less_create(self.cfg, w, self.arena.data_ptr(), nbytes)
        _check(rc, "less_create")
        self.ctx = ctx
        self.instances = batch * layers * heads
        self.group = max(1, group)
        self.N = heavy + recent
        self.record_bytes = less_state_record_bytes(self.cfg)
        self.out_dtype = torch.float16 if flags & LESS_OUT_F16 else torch.float32

    # -- hot path ---------------------------------------------------------- #
    def prefill(self, Q, K, V, layer_begin=0, attn_out=None, stream=None):
        B, Lc, H, S, D = Q.shape
        assert Q.dtype == K.dtype == V.dtype == torch.float16
        assert Q.is_contiguous() and K.is_contiguous() and V.is_contiguous()
        _check(less_prefill(self.ctx, layer_begin, Lc, S, _ptr(Q), _ptr(K), _ptr(V), _ptr(attn_out),
                            _stream_ptr(stream)), "less_prefill")

    def masked_attention(self, Q, K, V, exact_until, layer_begin=0, out=None, stream=None):
        """The parallel form: Q fp16 [B, Lc, H * group, S, D], K, V fp16 [B, Lc, H, S, D], exact_until int32
        [B, Lc, H, S]; the result has Q's shape."""
        B, Lc, _, S, D = Q.shape
        assert Q.dtype == K.dtype == V.dtype == torch.float16 and exact_until.dtype == torch.int32
        assert Q.is_contiguous() and K.is_contiguous() and V.is_contiguous() and exact_until.is_contiguous()
        if out is None:
            out = torch.empty(Q.shape, dtype=torch.float32, device=Q.device)
        _check(less_masked_attention(self.ctx, layer_begin, Lc, S, _ptr(Q), _ptr(K), _ptr(V), _ptr(exact_until),
                                     _ptr(out), _stream_ptr(stream)), "less_masked_attention")
        return out

    def reset(self, layer_begin=0, layer_count=None, stream=None):
        n = self.cfg.layers - layer_begin if layer_count is None else layer_count
        _check(less_prefill(self.ctx, layer_begin, n, 0, None, None, None, None, _stream_ptr(stream)),
               "less_prefill(reset)")

    def decode_step(self, q, k, v, out=None, evicted_pos=None, stream=None):
        assert q.dtype == k.dtype == v.dtype == torch.float16
        if out is None:
            out = torch.empty(q.shape, dtype=self.out_dtype, device=q.device)
        assert out.dtype == self.out_dtype
        _check(less_decode_step(self.ctx, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(evicted_pos),
                                _stream_ptr(stream)), "less_decode_step")
        return out

    def decode_step_host(self, q, k, v, out, stream=None):
        """q, k, v, out: host tensors (pinned for speed); synchronous."""
        _check(less_decode_step_host(self.ctx, _ptr(q), _ptr(k), _ptr(v), _ptr(out),
                                     _stream_ptr(stream)), "less_decode_step_host")
        return out

    def profile(self, enable: bool):
        _check(less_profile(self.ctx, 1 if enable else 0), "less_profile")

    def profile_read(self):
        ms = np.zeros(len(KERNEL_NAMES), dtype=np.float32)
        n = np.zeros(len(KERNEL_NAMES), dtype=np.int64)
        _check(less_profile_read(self.ctx, ms.ctypes.data, n.ctypes.data), "less_profile_read")
        return {k: (float(a), int(b)) for k, a, b in zip(KERNEL_NAMES, ms, n)}

    # -- state ------------------------------------------------------------- #
    @property
    def position(self) -> int:
        return less_position(self.ctx)

    @property
    def launches(self) -> int:
        return less_launch_count(self.ctx)

    def _record_views(self, buf: np.ndarray, i: int):
        N, D, R = self.N, self.cfg.head_dim, self.cfg.rank
        rec = buf[i * self.record_bytes:(i + 1) * self.record_bytes]
        off = 16
        views = {"header": rec[:16].view(np.int32)}
        for name, dt, shape in (("pos", np.int32, (N,)), ("acc", np.float32, (N,)),
                                ("K", np.float16, (N, D)), ("V", np.float16, (N, D)),
                                ("psi", np.float32, (N, R)), ("H", np.float32, (R, D)),
                                ("z", np.float32, (R,))):
            n = int(np.prod(shape)) * np.dtype(dt).itemsize
            views[name] = rec[off:off + n].view(dt).reshape(shape)
            off += n
        return views

    def export_state(self, instances: Sequence[int], stream=None):
        inst = np.ascontiguousarray(instances, dtype=np.int32)
        buf = np.zeros(len(inst) * self.record_bytes, dtype=np.uint8)
        _check(less_export_state(self.ctx, inst.ctypes.data, len(inst), buf.ctypes.data, buf.nbytes,
                                 _stream_ptr(stream)), "less_export_state")
        out = []
        for i in range(len(inst)):
            v = self._record_views(buf, i)
            cnt = int(v["header"][0])
            out.append({"count": cnt, "t": int(v["header"][1]), "pos": v["pos"][:cnt].copy(),
                        "acc": v["acc"][:cnt].copy(), "K": v["K"][:cnt].copy(),
                        "V": v["V"][:cnt].copy(), "psi": v["psi"][:cnt].copy(),
                        "H": v["H"].copy(), "z": v["z"].copy()})
        return out

    def import_state(self, instances: Sequence[int], records, stream=None):
        inst = np.ascontiguousarray(instances, dtype=np.int32)
        buf = np.zeros(len(inst) * self.record_bytes, dtype=np.uint8)
        for i, r in enumerate(records):
            v = self._record_views(buf, i)
            cnt = int(r["count"])
            v["header"][0] = cnt
            v["header"][1] = int(r["t"])
            for name in ("pos", "acc", "K", "V", "psi"):
                v[name][:cnt] = r[name]
            v["H"][...] = r["H"]
            v["z"][...] = r["z"]
        _check(less_import_state(self.ctx, inst.ctypes.data, len(inst), buf.ctypes.data, buf.nbytes,
                                 _stream_ptr(stream)), "less_import_state")

    def read_feature_maps(self, stream=None):
        R = self.cfg.rank
        phi = np.zeros((self.instances * self.group, R), dtype=np.float32)
        psi = np.zeros((self.instances, R), dtype=np.float32)
        _check(less_read_feature_maps(self.ctx, phi.ctypes.data, psi.ctypes.data, _stream_ptr(stream)),
               "less_read_feature_maps")
        return phi, psi

    def poll_status(self, stream=None) -> int:
        return less_poll_status(self.ctx, _stream_ptr(stream))

    def kernel_variant(self, kernel: str) -> str:
        """Name of the kernel variant last launched under a KERNEL_NAMES id."""
        return less_kernel_variant(self.ctx, KERNEL_NAMES.index(kernel))

    def status_where(self) -> int:
        return less_last_status_where(self.ctx)

    def selftest_wait_timeout(self, polls: int, stream=None) -> int:
        return less_selftest_wait_timeout(self.ctx, polls, _stream_ptr(stream))

    def close(self):
        if getattr(self, "ctx", None) is not None:
            less_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def from_workload(w, weights=None, device="cuda", max_prefill_layers=1, flags=0, psi_scale=None,
                  heavy=None, recent=None, max_prompt=None) -> LessContext:
    """Context shaped like a `workloads.Workload`."""
    from . import workloads as wl
    if weights is None:
        weights = wl.make_weights(w, device)
    return LessContext(w.batch, w.layers, w.heads, w.head_dim, w.rank, w.hidden,
                       w.heavy if heavy is None else heavy, w.recent if recent is None else recent,
                       w.prompt if max_prompt is None else max_prompt, weights,
                       max_prefill_layers=max_prefill_layers, flags=flags, psi_scale=psi_scale,
                       device=device, group=getattr(w, "group", 1))


class PagedCache:
    """The paged 8-bit cache (less_pages): holds its torch buffers and forwards calls.

    Sequences are rows of `table`; lists of them and of lengths are int32 tensors on the cache's device.  `buffers`
    gives the cache tensors that exist already (codes, amax, table, lens, refs), contiguous, in the shapes below;
    without it the cache starts empty.  Calls are asynchronous on the current stream or on `stream`, and what they are
    given may be dropped when they return: memory that `stream` still reads is not handed out again before it has.
    (As with any call, `stream` has to wait for the stream that wrote the inputs.)  `poll_status` tells what the device
    found wrong; until then calls that change the cache do nothing (write and trim go on with what is not refused)."""

    def __init__(self, layers, heads, head_dim, pages, seqs, seq_pages, group=1, page_tokens=64, fmt="int8",
                 dtype=torch.float16, device="cuda", buffers: Optional[Dict[str, torch.Tensor]] = None):
        if fmt not in ("int8", "e4m3"):
            raise ValueError(f"fmt is 'int8' or 'e4m3', not {fmt!r}")
        if dtype not in (torch.float16, torch.bfloat16):
            raise ValueError(f"dtype is torch.float16 or torch.bfloat16, not {dtype}")
        self.fmt, self.dtype = fmt, dtype
        flags = (LESS_PAGES_E4M3 if fmt == "e4m3" else 0) | (LESS_PAGES_BF16 if dtype == torch.bfloat16 else 0)
        desc = less_pages(layers, heads, group, head_dim, page_tokens, pages, seqs, seq_pages, flags)
        nbytes = less_pages_workspace_bytes(desc)
        if nbytes == 0:
            raise LessError(-1, "less_pages_workspace_bytes")
        if not torch.cuda.is_available():
            raise RuntimeError("the LESS library needs a CUDA device (there is no CPU path)")
        shapes = {"codes": ((layers, pages, heads, 2, page_tokens * head_dim), torch.uint8),
                  "amax": ((layers, pages, heads, 2, page_tokens // LESS_PAGE_BLOCK), torch.float32),
                  "table": ((seqs, seq_pages), torch.int32), "lens": ((seqs,), torch.int32),
                  "refs": ((pages,), torch.int32)}
        if buffers is None:
            buffers = {n: torch.empty(s, dtype=t, device=device) for n, (s, t) in shapes.items()}
            empty = True
        else:
            empty = False
            for n, (s, t) in shapes.items():
                b = buffers[n]
                if tuple(b.shape) != s or b.dtype != t or not b.is_contiguous() or not b.is_cuda:
                    raise ValueError(f"{n}: a contiguous CUDA tensor {s} of {t} is wanted, "
                                     f"got {tuple(b.shape)} of {b.dtype} on {b.device}")
        self.codes, self.amax, self.table, self.lens, self.refs = (buffers[n] for n in shapes)
        self.device = self.codes.device
        if any(b.device != self.device for b in (self.amax, self.table, self.lens, self.refs)):
            raise ValueError("the buffers of a cache are on one device")
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=self.device)
        for n in shapes:
            setattr(desc, n, buffers[n].data_ptr())
        desc.workspace, desc.workspace_bytes = self.workspace.data_ptr(), nbytes
        self.desc = desc
        self.scale = head_dim ** -0.5
        self.layers, self.heads, self.group, self.head_dim = layers, heads, group, head_dim
        self._index = self.device.index
        self._streams = set()                            # those that the buffers are recorded on
        self._lib = lib()
        if empty:
            self.reset()

    # -- helpers (a call takes a few microseconds on the host: the checks below are the cheap forms) ---------- #
    def _call(self, fn, where, *args, stream=None, keep=()):
        if stream is not None:
            for t in keep:
                if t is not None:
                    t.record_stream(stream)
            if stream.cuda_stream not in self._streams:
                self._streams.add(stream.cuda_stream)
                for t in (self.codes, self.amax, self.table, self.lens, self.refs, self.workspace):
                    t.record_stream(stream)
        if torch._C._cuda_getDevice() == self._index:
            rc = fn(self.desc, *args, torch._C._cuda_getCurrentRawStream(self._index) if stream is None
                    else stream.cuda_stream)
        else:
            with torch.cuda.device(self._index):
                rc = fn(self.desc, *args, torch._C._cuda_getCurrentRawStream(self._index) if stream is None
                        else stream.cuda_stream)
        if rc != LESS_OK:
            raise LessError(rc, where)

    def _list(self, t: torch.Tensor, name: str, n: Optional[int] = None) -> int:
        if t.dtype is not torch.int32 or t.get_device() != self._index or t.dim() != 1 or not t.is_contiguous():
            raise ValueError(f"{name}: a contiguous 1-d int32 tensor on {self.device} is wanted")
        if n is not None and t.shape[0] != n:
            raise ValueError(f"{name}: {n} values are wanted, got {t.shape[0]}")
        return t.data_ptr()

    def _rows(self, t: torch.Tensor, name: str, heads: int):
        if t.dtype is not self.dtype or t.get_device() != self._index or t.dim() != 4:
            raise ValueError(f"{name}: a [rows, layers, heads, D] tensor of {self.dtype} on {self.device} is wanted")
        rows, layers, h, dim = t.shape
        if h != heads or dim != self.head_dim or layers > self.layers:
            raise ValueError(f"{name}: [rows, layers, {heads}, {self.head_dim}] is wanted, got {tuple(t.shape)}")
        if rows <= 1 or t.is_contiguous():
            stride = layers * h * dim
            if rows == 0 or t.is_contiguous():
                return rows, layers, stride
        else:
            stride = t.stride(0)
        if t.stride(3) != 1 or (h > 1 and t.stride(2) != dim) or (layers > 1 and t.stride(1) != h * dim):
            raise ValueError(f"{name}: everything but the rows has to be contiguous")
        return rows, layers, stride

    # -- the maps ---------------------------------------------------------- #
    def reset(self, stream=None):
        """Empties the cache."""
        self._call(self._lib.less_pages_reset, "less_pages_reset", stream=stream)

    def resize(self, seqs, lens, stream=None):
        """Sequences get new lengths: pages are taken or released (0 frees a sequence)."""
        n = seqs.shape[0]
        self._call(self._lib.less_pages_resize, "less_pages_resize", n, self._list(seqs, "seqs"),
                   self._list(lens, "lens", n), stream=stream, keep=(seqs, lens))

    def fork(self, src, dst, stream=None):
        """The empty sequences dst become copies of src (whole pages shared)."""
        n = src.shape[0]
        self._call(self._lib.less_pages_fork, "less_pages_fork", n, self._list(src, "src"), self._list(dst, "dst", n),
                   stream=stream, keep=(src, dst))

    def trim(self, seqs, sinks, window, stream=None):
        """Releases the pages between the first `sinks` tokens and the last `window`."""
        self._call(self._lib.less_pages_trim, "less_pages_trim", seqs.shape[0], self._list(seqs, "seqs"), sinks, window,
                   stream=stream, keep=(seqs,))

    def compact(self, stream=None):
        """Moves the pages in use to the front of the pool."""
        self._call(self._lib.less_pages_compact, "less_pages_compact", stream=stream)

    # -- contents ---------------------------------------------------------- #
    def write(self, k, v, seqs, starts=None, layer_begin=0, stream=None):
        """k, v [rows, layers, heads, D]: the last tokens of the listed sequences (rows starts[i] .. starts[i + 1]
        belong to seqs[i]; without starts one row each)."""
        n = seqs.shape[0]
        rows, layers, ks = self._rows(k, "k", self.heads)
        vrows, vlayers, vs = self._rows(v, "v", self.heads)
        if (vrows, vlayers) != (rows, layers):
            raise ValueError("k and v have the same shape")
        self._call(self._lib.less_pages_write, "less_pages_write", layer_begin, layers, n, self._list(seqs, "seqs"),
                   None if starts is None else self._list(starts, "starts", n + 1), rows, k.data_ptr(), ks,
                   v.data_ptr(), vs, stream=stream, keep=(k, v, seqs, starts))

    def attention(self, q, seqs, starts=None, max_new=None, layer_begin=0, window=0, sinks=0, scale=None, out=None,
                  stream=None):
        """q [rows, layers, heads * group, D]: attention of the last tokens of the listed sequences over the cache.
        max_new: the most new tokens of a sequence, as far as the host knows (default: all rows)."""
        n = seqs.shape[0]
        rows, layers, qs = self._rows(q, "q", self.heads * self.group)
        if out is None:                                  # memory of the stream that writes it
            with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
                out = torch.empty_like(q, memory_format=torch.contiguous_format)
        elif out.shape != q.shape or out.dtype != self.dtype or out.device != self.device or not out.is_contiguous():
            raise ValueError("out: a contiguous tensor of q's shape and type is wanted")
        self._call(self._lib.less_pages_attention, "less_pages_attention", layer_begin, layers, n,
                   self._list(seqs, "seqs"), None if starts is None else self._list(starts, "starts", n + 1), rows,
                   max(1, rows if max_new is None else max_new), q.data_ptr(), qs, window, sinks,
                   self.scale if scale is None else scale, out.data_ptr(), stream=stream, keep=(q, seqs, starts, out))
        return out

    def poll_status(self, stream=None) -> int:
        """What the device found wrong since the last poll (0 = nothing); clears it."""
        with torch.cuda.device(self._index):
            return less_pages_poll_status(self.desc, _stream_ptr(stream))
