"""ctypes binding of libbaklava: argument marshalling only.

Every step of the hot path runs inside the library's HIP kernels; nothing here
computes.  PyTorch tensors are used as device memory (`.data_ptr()`) and for
the current stream.  Importing this module does not load the library; the
first call does, and fails loudly if the library has not been built.
"""
from __future__ import annotations

import array
import ctypes as C
import os
from typing import List, Optional, Sequence

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libbaklava.so")

OK, EINVAL, EINFEASIBLE, ECAPACITY, EHIP, ESTATE, ENOMEM = range(7)
BF16, F32, MXFP4 = 0, 1, 2
POLICY_SCORE, POLICY_STREAMING = 0, 1
OPT_CHUNK_TOKENS, OPT_KERNEL, OPT_TIME_KERNEL, OPT_CHUNK_TOKENS_WHOLE, OPT_TARGET_ITEMS, OPT_TARGET_ITEMS_WHOLE = 1, 2, 3, 4, 5, 6
OPT_TRACK_SCORES, OPT_TILED_SELECT_ROWS = 7, 8
KERNEL_AUTO, KERNEL_VALU, KERNEL_MFMA = 0, 1, 2

EXPORTS = [
    "baklava_strerror", "baklava_last_hip_error", "baklava_alloc_proportional",
    "baklava_alloc_threshold", "baklava_layout", "baklava_plan_schedule", "baklava_workspace_bytes",
    "baklava_create",
    "baklava_destroy", "baklava_set_option", "baklava_reset", "baklava_set_lengths",
    "baklava_append", "baklava_decode_attn", "baklava_append_decode_attn", "baklava_compact", "baklava_lengths", "baklava_profile_read",
    "baklava_stream_probe", "baklava_profile_workspace_bytes", "baklava_profile_similarity", "baklava_kv_importance", "baklava_prefill_scores", "baklava_layer_workspace_bytes", "baklava_layer_similarity",
    "baklava_alloc_two_level", "baklava_layer_similarity_static", "baklava_append_decode_attn_replay",
    "baklava_sync_lengths", "baklava_flush_scores",
    "baklava_qk_norm_rope", "baklava_prompt_attn", "baklava_append_prompt", "baklava_read_rows",
    "baklava_tree_workspace_bytes", "baklava_tree_attn", "baklava_verify_workspace_bytes", "baklava_verify_draft", "baklava_append_accepted",
]


class BaklavaError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: status {status} ({strerror(status)})")


class Desc(C.Structure):
    _fields_ = [
        ("L", C.c_int32), ("Hq", C.c_int32), ("Hkv", C.c_int32), ("D", C.c_int32), ("batch", C.c_int32),
        ("dtype", C.c_int32), ("sink", C.c_int32), ("recent", C.c_int32), ("policy", C.c_int32),
        ("track_scores", C.c_int32),
        ("k", C.c_void_p), ("v", C.c_void_p), ("score", C.c_void_p), ("pos", C.c_void_p),
        ("off", C.c_void_p), ("cap", C.c_void_p), ("len", C.c_void_p), ("budget", C.c_void_p),
        ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("kv_scale", C.c_void_p),
    ]


class WorkItem(C.Structure):
    _fields_ = [("cache", C.c_int32), ("start", C.c_int32), ("count", C.c_int32), ("slot", C.c_int32),
                ("nsplit", C.c_int32), ("reserved", C.c_int32), ("row0", C.c_int64)]


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            f"{LIB_PATH} is missing: build it first (python -m paper_2502_13176_amd.build). "
            "There is no fallback path.")
    L = C.CDLL(LIB_PATH)
    i32p, i64p, f64p = C.POINTER(C.c_int32), C.POINTER(C.c_int64), C.POINTER(C.c_double)
    L.baklava_strerror.restype = C.c_char_p
    L.baklava_strerror.argtypes = [C.c_int]
    L.baklava_last_hip_error.restype = C.c_int
    L.baklava_alloc_proportional.argtypes = [f64p, C.c_int32, C.c_int64, C.c_int32, C.c_int32, i32p]
    L.baklava_alloc_threshold.argtypes = [f64p, C.c_int32, i32p, C.c_double, C.c_double, i32p]
    L.baklava_layout.argtypes = [i32p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, i64p, i32p, i64p]
    L.baklava_plan_schedule.argtypes = [i64p, i32p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                        C.c_int64, C.POINTER(WorkItem), i64p]
    L.baklava_workspace_bytes.restype = C.c_size_t
    L.baklava_workspace_bytes.argtypes = [C.POINTER(Desc), i32p, i32p]
    L.baklava_create.argtypes = [C.POINTER(Desc), i64p, i32p, i32p, i32p, C.POINTER(C.c_void_p)]
    L.baklava_destroy.argtypes = [C.c_void_p]
    L.baklava_set_option.argtypes = [C.c_void_p, C.c_int32, C.c_int64]
    L.baklava_reset.argtypes = [C.c_void_p, C.c_void_p]
    L.baklava_set_lengths.argtypes = [C.c_void_p, i32p, C.c_void_p]
    L.baklava_append.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
    L.baklava_append_decode_attn.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_int32,
                                             C.c_void_p, C.c_void_p, C.c_void_p]
    L.baklava_append_decode_attn_replay.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                                    C.c_void_p, C.c_void_p, C.c_void_p]
    L.baklava_sync_lengths.argtypes = [C.c_void_p, C.c_void_p]
    L.baklava_flush_scores.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]
    L.baklava_decode_attn.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    L.baklava_compact.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
    L.baklava_lengths.argtypes = [C.c_void_p, i32p]
    L.baklava_profile_read.argtypes = [C.c_void_p, f64p, i64p]
    L.baklava_stream_probe.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p]
    L.baklava_profile_workspace_bytes.restype = C.c_size_t
    L.baklava_profile_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32]
    L.baklava_profile_similarity.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                             C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.c_size_t, C.c_void_p]
    L.baklava_layer_workspace_bytes.restype = C.c_size_t
    L.baklava_layer_workspace_bytes.argtypes = [C.c_int32, C.c_int32]
    L.baklava_layer_similarity.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
    L.baklava_layer_similarity_static.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                                  C.c_void_p, C.c_void_p, C.c_void_p]
    L.baklava_alloc_two_level.argtypes = [f64p, f64p, C.c_int32, C.c_int32, C.c_int64, C.c_int32, C.c_int32,
                                          C.c_double, C.c_double, i32p]
    L.baklava_prefill_scores.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32,
                                         C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
    L.baklava_kv_importance.argtypes = [f64p, C.c_int32, C.c_int32, C.c_int32, f64p]
    # (baklava_rows and the arrays of lengths travel as addresses: see _Rows and _ints)
    vp = C.c_void_p
    L.baklava_qk_norm_rope.argtypes = [vp, vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp, vp, C.c_float, vp,
                                       C.c_int32, C.c_char_p, vp, C.c_int32, C.c_int32, vp, vp, vp]
    L.baklava_prompt_attn.argtypes = [vp, vp, vp, C.c_int32, vp, vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32, vp, vp, vp]
    L.baklava_append_prompt.argtypes = [vp, C.c_int32, vp, vp, vp, vp, vp, vp]
    L.baklava_read_rows.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
    L.baklava_tree_workspace_bytes.restype = C.c_size_t
    L.baklava_tree_workspace_bytes.argtypes = [vp, C.c_int32, C.c_int32]
    L.baklava_tree_attn.argtypes = [vp, C.c_int32, C.c_int32, vp, vp, C.c_int32, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
    L.baklava_verify_workspace_bytes.restype = C.c_size_t
    L.baklava_verify_workspace_bytes.argtypes = [C.c_int32] * 4
    L.baklava_verify_draft.argtypes = [vp, C.c_int64, vp, C.c_int64] + [C.c_int32] * 4 + [vp] * 9 + [C.c_size_t, vp]
    L.baklava_append_accepted.argtypes = [vp, C.c_int32, C.c_int32, vp, vp, C.c_int32] + [vp] * 6
    for name in EXPORTS:
        if name not in ("baklava_tree_workspace_bytes", "baklava_verify_workspace_bytes", "baklava_strerror", "baklava_workspace_bytes", "baklava_profile_workspace_bytes",
                        "baklava_layer_workspace_bytes"):
            getattr(L, name).restype = C.c_int
    _lib = L
    return L


def strerror(status: int) -> str:
    return lib().baklava_strerror(int(status)).decode()


def _check(status: int, what: str) -> None:
    if status != OK:
        raise BaklavaError(status, what)


def _i32(a) -> np.ndarray:
    return np.ascontiguousarray(a, dtype=np.int32)


def _p(a: np.ndarray, ctype):
    return a.ctypes.data_as(C.POINTER(ctype))


# ---------------------------------------------------------------------------
# host-only calls
# ---------------------------------------------------------------------------

def alloc_proportional(importance: Sequence[float], global_budget: int, lo: int, hi: int) -> List[int]:
    imp = np.ascontiguousarray(importance, dtype=np.float64)
    out = np.zeros(len(imp), dtype=np.int32)
    _check(lib().baklava_alloc_proportional(_p(imp, C.c_double), len(imp), int(global_budget), int(lo),
                                            int(hi), _p(out, C.c_int32)), "baklava_alloc_proportional")
    return out.tolist()


def alloc_threshold(importance: Sequence[float], size_in: Sequence[int], t: float, r: float) -> List[int]:
    imp = np.ascontiguousarray(importance, dtype=np.float64)
    size = _i32(size_in)
    out = np.zeros(len(imp), dtype=np.int32)
    _check(lib().baklava_alloc_threshold(_p(imp, C.c_double), len(imp), _p(size, C.c_int32), float(t),
                                         float(r), _p(out, C.c_int32)), "baklava_alloc_threshold")
    return out.tolist()


def layout(budget: Sequence[int], L: int, Hkv: int, batch: int, slack: int):
    b = _i32(budget)
    n = L * Hkv * batch
    off = np.zeros(n, dtype=np.int64)
    cap = np.zeros(n, dtype=np.int32)
    total = C.c_int64(0)
    _check(lib().baklava_layout(_p(b, C.c_int32), L, Hkv, batch, slack, _p(off, C.c_int64),
                                _p(cap, C.c_int32), C.byref(total)), "baklava_layout")
    return off, cap, int(total.value)


def plan_schedule(off, cap, L: int, caches_per_layer: int, chunk: int, whole_model: bool, max_items=None,
                  target_items: int = 0):
    """baklava_plan_schedule: list of (cache, start, count, slot, nsplit, row0) in launch order."""
    off = np.ascontiguousarray(off, dtype=np.int64)
    cap = _i32(cap)
    n = C.c_int64(0)
    args = (_p(off, C.c_int64), _p(cap, C.c_int32), L, caches_per_layer, chunk, int(target_items),
            int(bool(whole_model)))
    _check(lib().baklava_plan_schedule(*args, 0, None, C.byref(n)), "baklava_plan_schedule")
    cap_items = int(n.value) if max_items is None else int(max_items)
    items = (WorkItem * max(1, cap_items))()
    _check(lib().baklava_plan_schedule(*args, cap_items, items, C.byref(n)), "baklava_plan_schedule")
    return [(it.cache, it.start, it.count, it.slot, it.nsplit, it.row0) for it in items[: int(n.value)]]


# ---------------------------------------------------------------------------
# device context
# ---------------------------------------------------------------------------

def _stream_ptr(stream=None) -> int:
    """The handle of `stream`, or of torch's current one.  Building a Stream object to ask it for its handle takes 2.9
    us, nearly half of a small attention call (6.8 us on the host, 4.1 without); torch also gives the bare handle, though
    under names that it does not promise to keep."""
    import torch
    if stream is not None:
        return int(stream.cuda_stream)
    if torch.cuda.is_initialized():
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            pass
    return int(torch.cuda.current_stream().cuda_stream)


class Arena:
    """Device memory of a ragged KV arena plus a libbaklava context over it.

    Holds torch tensors only to keep the memory alive; all work goes through
    the C-ABI calls.
    """

    def __init__(self, L: int, Hq: int, Hkv: int, D: int, batch: int, dtype: str, budget: Sequence[int],
                 slack: int, sink: int, recent: int, policy: int = POLICY_SCORE, track_scores: bool = False,
                 device: str = "cuda:0", workspace_fill: int = 0):
        import torch
        self.torch = torch
        self.L, self.Hq, self.Hkv, self.D, self.batch = L, Hq, Hkv, D, batch
        self.G = Hq // Hkv
        self.dtype = dtype
        self.device = torch.device(device)
        self.budget_host = _i32(budget)
        self.off_host, self.cap_host, self.total_tokens = layout(budget, L, Hkv, batch, slack)
        self.n_caches = L * batch * Hkv
        mx = self.mx = dtype == "mxfp4"  # rows of D / 2 bytes of codes, their scales in a plane of their own
        tdt = torch.uint8 if mx else torch.bfloat16 if dtype == "bf16" else torch.float32
        dev = self.device
        self.k = torch.zeros((self.total_tokens, D // 2 if mx else D), dtype=tdt, device=dev)
        self.v = torch.zeros_like(self.k)
        self.gpu = self.k.get_device()
        self.kv_scale = torch.full((self.total_tokens, D // 16), 2, dtype=torch.uint8, device=dev) if mx else None
        self.score = torch.zeros((self.total_tokens,), dtype=torch.float32, device=dev)
        self.pos = torch.zeros((self.total_tokens,), dtype=torch.int32, device=dev)
        self.off = torch.from_numpy(self.off_host).to(dev)
        self.cap = torch.from_numpy(self.cap_host).to(dev)
        self.len = torch.zeros((self.n_caches,), dtype=torch.int32, device=dev)
        self.budget = torch.from_numpy(self.budget_host).to(dev)

        d = Desc()
        d.L, d.Hq, d.Hkv, d.D, d.batch = L, Hq, Hkv, D, batch
        d.dtype = MXFP4 if mx else BF16 if dtype == "bf16" else F32
        d.sink, d.recent, d.policy, d.track_scores = sink, recent, policy, int(bool(track_scores))
        ws_bytes = lib().baklava_workspace_bytes(C.byref(d), _p(self.cap_host, C.c_int32),
                                                 _p(self.budget_host, C.c_int32))
        if ws_bytes == 0:
            raise BaklavaError(EINVAL, "baklava_workspace_bytes")
        # the library does not rely on the workspace's initial contents; tests fill it with 0xFF bytes
        self.workspace = torch.full((ws_bytes,), int(workspace_fill), dtype=torch.uint8, device=dev)
        d.k, d.v = self.k.data_ptr(), self.v.data_ptr()
        d.kv_scale = self.kv_scale.data_ptr() if mx else None
        d.score, d.pos = self.score.data_ptr(), self.pos.data_ptr()
        d.off, d.cap, d.len, d.budget = (self.off.data_ptr(), self.cap.data_ptr(), self.len.data_ptr(),
                                         self.budget.data_ptr())
        d.workspace, d.workspace_bytes = self.workspace.data_ptr(), ws_bytes
        self.desc = d
        torch.cuda.synchronize(dev)
        ctx = C.c_void_p()
        _check(lib().baklava_create(C.byref(d), _p(self.off_host, C.c_int64), _p(self.cap_host, C.c_int32),
                                    None, _p(self.budget_host, C.c_int32), C.byref(ctx)), "baklava_create")
        self.ctx = ctx

    def close(self) -> None:
        if getattr(self, "ctx", None):
            lib().baklava_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- thin wrappers with the C names ------------------------------------------------
    def set_option(self, option: int, value: int) -> None:
        _check(lib().baklava_set_option(self.ctx, option, int(value)), "baklava_set_option")

    def reset(self, stream=None) -> None:
        _check(lib().baklava_reset(self.ctx, _stream_ptr(stream)), "baklava_reset")

    def set_lengths(self, len_host: Sequence[int], stream=None) -> None:
        a = _i32(len_host)
        _check(lib().baklava_set_lengths(self.ctx, _p(a, C.c_int32), _stream_ptr(stream)), "baklava_set_lengths")

    def _expect_bf16(self, *rows) -> None:
        """Rows for caches in 4 bits: codes in their place would be read as rows four times as long."""
        for t in rows:
            if t.dtype is not self.torch.bfloat16:
                raise ValueError("queries and new rows of an mxfp4 arena are bf16")

    def append(self, layer_begin: int, layer_count: int, k_new, v_new, token_pos: int, stream=None) -> None:
        if self.mx:
            self._expect_bf16(k_new, v_new)
        _check(lib().baklava_append(self.ctx, layer_begin, layer_count, k_new.data_ptr(), v_new.data_ptr(),
                                    int(token_pos), _stream_ptr(stream)), "baklava_append")

    def append_decode_attn(self, layer_begin: int, layer_count: int, k_new, v_new, token_pos: int, q, out,
                           stream=None) -> None:
        if self.mx:
            self._expect_bf16(k_new, v_new, q)
        _check(lib().baklava_append_decode_attn(self.ctx, layer_begin, layer_count, k_new.data_ptr(),
                                                v_new.data_ptr(), int(token_pos), q.data_ptr(), out.data_ptr(),
                                                _stream_ptr(stream)), "baklava_append_decode_attn")

    def append_decode_attn_replay(self, layer_begin: int, layer_count: int, k_new, v_new, token_pos_dev, q, out,
                                  stream=None) -> None:
        if self.mx:
            self._expect_bf16(k_new, v_new, q)
        _check(lib().baklava_append_decode_attn_replay(self.ctx, layer_begin, layer_count, k_new.data_ptr(),
                                                       v_new.data_ptr(), token_pos_dev.data_ptr(), q.data_ptr(),
                                                       out.data_ptr(), _stream_ptr(stream)),
               "baklava_append_decode_attn_replay")

    def sync_lengths(self, stream=None) -> None:
        _check(lib().baklava_sync_lengths(self.ctx, _stream_ptr(stream)), "baklava_sync_lengths")

    def flush_scores(self, layer_begin: int, layer_count: int, stream=None) -> None:
        _check(lib().baklava_flush_scores(self.ctx, layer_begin, layer_count, _stream_ptr(stream)),
               "baklava_flush_scores")

    def append_prompt(self, layer: int, k, v, lens: Sequence[int], pos0: Optional[Sequence[int]] = None, scores=None,
                      stream=None) -> None:
        """baklava_append_prompt: k, v [tokens, Hkv, D] (the sequences of `lens` tokens in a row) or [batch, Hkv, T, D]
        (padded), of any strides with contiguous rows; scores [Hkv, tokens] or [batch, Hkv, T] fp32, or None (zeros)."""
        if len(lens) != self.batch or (pos0 is not None and len(pos0) != self.batch):
            raise ValueError("one length (and position) per sequence expected")
        n, n_at, total, most = _ints(lens)
        dt = self.torch.bfloat16 if self.dtype in ("bf16", "mxfp4") else self.torch.float32
        rows = _Rows(self.torch)
        if rows.device != self.gpu:
            raise ValueError("the arena's GPU must be the current one")
        k_at = rows.add(k, "k", self.batch, total, most, self.Hkv, self.D, dt)
        v_at = rows.add(v, "v", self.batch, total, most, self.Hkv, self.D, dt)
        s_at = rows.add_values(scores, "scores", self.batch, total, most, self.Hkv) if scores is not None else None
        p0, p0_at, _, _ = _ints(pos0) if pos0 is not None else (None, None, 0, 0)
        st = lib().baklava_append_prompt(self.ctx, int(layer), k_at, v_at, n_at, p0_at, s_at, _stream_ptr(stream))
        _check(st, "baklava_append_prompt")

    def read_rows(self, layer_begin: int, layer_count: int, n: int, stream=None):
        """baklava_read_rows: the last n rows of every cache of the range as values, (k, v) [caches, n, D]."""
        if n < 1 or layer_count < 1:
            raise ValueError("at least one row of one layer expected")
        if stream is None and _current_device() != self.gpu:
            raise ValueError("the arena's GPU must be the current one, or a stream of it be given")
        dt = self.torch.bfloat16 if self.dtype in ("bf16", "mxfp4") else self.torch.float32
        shape = (layer_count * self.batch * self.Hkv, n, self.D)
        k, v = (_empty_on(stream, self.torch.empty, shape, dtype=dt, device=self.device) for _ in range(2))
        _check(lib().baklava_read_rows(self.ctx, int(layer_begin), int(layer_count), int(n), k.data_ptr(), v.data_ptr(),
                                       _stream_ptr(stream)), "baklava_read_rows")
        _hold_until_stream_passes((k, v), stream)
        return k, v

    def tree_attn(self, layer_begin: int, layer_count: int, k, v, parent, q, n_nodes=None, out=None, lse=None,
                  want_lse: bool = False, stream=None):
        """baklava_tree_attn: parent int32 [batch, N], n_nodes int32 [batch] or None (N); q [tokens, Hq, D], k and v [tokens,
        Hkv, D] (N tokens of every sequence in a row, the sequences of the first layer first) or [layers * batch, H, N, D], of any
        strides with contiguous rows.  Returns out (like q; places of absent nodes are not written), and with want_lse or lse given
        also lse (fp32 [Hq, tokens] or [layers * batch, Hq, N]).  No gradient: tensors that require one are refused outside
        torch.no_grad()."""
        torch = self.torch
        _refuse_grad(torch, q, k, v)
        rows = _Rows(torch)
        if rows.device != self.gpu:
            raise ValueError("the arena's GPU must be the current one")
        N, n_seq = _per_node(parent, "parent"), layer_count * self.batch
        _expect(rows, parent, torch.int32, "parent", (self.batch, N))
        if n_nodes is not None:
            _expect(rows, n_nodes, torch.int32, "n_nodes", (self.batch,))
        dt = torch.float32 if self.dtype not in ("bf16", "mxfp4") else torch.bfloat16
        k_at = rows.add(k, "k", n_seq, n_seq * N, N, self.Hkv, self.D, dt)
        v_at = rows.add(v, "v", n_seq, n_seq * N, N, self.Hkv, self.D, dt)
        q_at = rows.add(q, "q", n_seq, n_seq * N, N, self.Hq, self.D, dt)
        if out is None:
            out = q.new_empty(q.shape) if stream is None else _empty_on(stream, q.new_empty, q.shape)
        if lse is None and want_lse:
            lse = _empty_on(stream, q.new_empty, (self.Hq, q.shape[0]) if q.dim() == 3 else q.shape[:3], dtype=torch.float32)
        out_at = rows.add(out, "out", n_seq, n_seq * N, N, self.Hq, self.D, dt)
        lse_at = rows.add_values(lse, "lse", n_seq, n_seq * N, N, self.Hq) if lse is not None else None
        nbytes = lib().baklava_tree_workspace_bytes(self.ctx, int(layer_count), N)
        ws = _empty_on(stream, parent.new_empty, max(nbytes, 256), dtype=torch.uint8)
        _check(lib().baklava_tree_attn(self.ctx, int(layer_begin), int(layer_count), k_at, v_at, N, parent.data_ptr(),
                                       n_nodes.data_ptr() if n_nodes is not None else None, q_at, out_at, lse_at, ws.data_ptr(),
                                       nbytes, _stream_ptr(stream)), "baklava_tree_attn")
        _hold_until_stream_passes((out, lse), stream)
        return (out, lse) if lse is not None else out

    def append_accepted(self, layer_begin: int, layer_count: int, k, v, path, n_path, pos0, q=None, lse=None, stream=None) -> None:
        """baklava_append_accepted: path int32 [batch, N], n_path and pos0 int32 [batch]; k, v (and q, lse, which an arena that
        tracks scores needs) as tree_attn took and gave them.  sync_lengths comes before the next call that takes its position
        by value.  No gradient: tensors that require one are refused outside torch.no_grad()."""
        torch = self.torch
        _refuse_grad(torch, k, v, q, lse)
        rows = _Rows(torch)
        if rows.device != self.gpu:
            raise ValueError("the arena's GPU must be the current one")
        N, n_seq = _per_node(path, "path"), layer_count * self.batch
        _expect(rows, path, torch.int32, "path", (self.batch, N))
        _expect(rows, n_path, torch.int32, "n_path", (self.batch,))
        _expect(rows, pos0, torch.int32, "pos0", (self.batch,))
        if (q is None) != (lse is None):
            raise ValueError("q and lse go together")
        dt = torch.float32 if self.dtype not in ("bf16", "mxfp4") else torch.bfloat16
        k_at = rows.add(k, "k", n_seq, n_seq * N, N, self.Hkv, self.D, dt)
        v_at = rows.add(v, "v", n_seq, n_seq * N, N, self.Hkv, self.D, dt)
        q_at = rows.add(q, "q", n_seq, n_seq * N, N, self.Hq, self.D, dt) if q is not None else None
        lse_at = rows.add_values(lse, "lse", n_seq, n_seq * N, N, self.Hq) if lse is not None else None
        _check(lib().baklava_append_accepted(self.ctx, int(layer_begin), int(layer_count), k_at, v_at, N, path.data_ptr(),
                                             n_path.data_ptr(), pos0.data_ptr(), q_at, lse_at, _stream_ptr(stream)),
               "baklava_append_accepted")

    def decode_attn(self, layer_begin: int, layer_count: int, q, out, stream=None) -> None:
        if self.mx:
            self._expect_bf16(q)
        _check(lib().baklava_decode_attn(self.ctx, layer_begin, layer_count, q.data_ptr(), out.data_ptr(),
                                         _stream_ptr(stream)), "baklava_decode_attn")

    def compact(self, layer_begin: int, layer_count: int, kept_idx_out=None, stream=None) -> None:
        ptr = kept_idx_out.data_ptr() if kept_idx_out is not None else None
        _check(lib().baklava_compact(self.ctx, layer_begin, layer_count, ptr, _stream_ptr(stream)),
               "baklava_compact")

    def profile_read(self):
        ms, n = C.c_double(0.0), C.c_int64(0)
        _check(lib().baklava_profile_read(self.ctx, C.byref(ms), C.byref(n)), "baklava_profile_read")
        return float(ms.value), int(n.value)

    def lengths(self) -> np.ndarray:
        out = np.zeros(self.n_caches, dtype=np.int32)
        _check(lib().baklava_lengths(self.ctx, _p(out, C.c_int32)), "baklava_lengths")
        return out


def stream_probe(dst, src, nbytes: int, mode: int, stream=None) -> None:
    """baklava_stream_probe on two torch device tensors (mode 0: copy, 1: read only, 2: read only with non-temporal loads, 3: mode 2 on 64 workgroups)."""
    _check(lib().baklava_stream_probe(dst.data_ptr(), src.data_ptr(), int(nbytes), int(mode),
                                      _stream_ptr(stream)), "baklava_stream_probe")


def _empty_on(stream, make, *shape, **kw):
    """make(*shape, **kw), an allocation for kernels of `stream` (None: torch's current one).  It has to come from that stream's
    part of the caching allocator: a block of the current stream's part may have been dropped while kernels of the current
    stream still use it, and nothing would order another stream's kernels behind those."""
    if stream is None:
        return make(*shape, **kw)
    import torch
    with torch.cuda.stream(stream):
        return make(*shape, **kw)


def _hold_until_stream_passes(tensors, stream) -> None:
    """Tensors that kernels enqueued on another stream than torch's current one use, and that the caller may use on the current
    one: the caching allocator must not hand their memory out again before both have passed their use.  (A workspace that comes
    from the other stream's part and is used there alone needs none of this.)"""
    if stream is None:
        return
    import torch
    here = torch.cuda.current_stream()
    for t in tensors:
        if t is not None:
            t.record_stream(stream)
            t.record_stream(here)


def kv_importance(similarity, L: int, Hq: int, Hkv: int) -> np.ndarray:
    """baklava_kv_importance: [L, Hq] head similarities -> [L, Hkv] KV-cache importances (host only)."""
    sim = np.ascontiguousarray(similarity, dtype=np.float64).reshape(-1)
    if sim.size != L * Hq:
        raise ValueError("similarity must hold L * Hq values")
    out = np.zeros(L * Hkv, dtype=np.float64)
    _check(lib().baklava_kv_importance(_p(sim, C.c_double), L, Hq, Hkv, _p(out, C.c_double)), "baklava_kv_importance")
    return out.reshape(L, Hkv)


def profile_workspace_bytes(batch: int, Hq: int, T: int) -> int:
    return int(lib().baklava_profile_workspace_bytes(batch, Hq, T))


def profile_similarity(q, k, v, want_cos: bool = True, want_lse: bool = False, stream=None):
    """baklava_profile_similarity on torch device tensors q [batch, Hq, T, D], k / v [batch, Hkv, T, D]
    (bf16).  Returns (sim [batch, Hq], cos [batch, Hq, T] or None) as torch fp32 device tensors, and
    the per-token log2-sum-exp [batch, Hq, T] as a third value when want_lse is set."""
    import torch
    batch, Hq, T, D = q.shape
    Hkv = k.shape[1]
    if k.shape != (batch, Hkv, T, D) or v.shape != k.shape:
        raise ValueError("k and v must be [batch, Hkv, T, D]")
    if q.dtype != torch.bfloat16 or k.dtype != torch.bfloat16 or v.dtype != torch.bfloat16:
        raise ValueError("bf16 tensors expected")
    if not (q.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
        raise ValueError("contiguous tensors expected")
    sim = _empty_on(stream, torch.empty, (batch, Hq), dtype=torch.float32, device=q.device)
    cos = _empty_on(stream, torch.empty, (batch, Hq, T), dtype=torch.float32, device=q.device) if want_cos else None
    lse = _empty_on(stream, torch.empty, (batch, Hq, T), dtype=torch.float32, device=q.device) if want_lse else None
    nbytes = profile_workspace_bytes(batch, Hq, T)
    ws = _empty_on(stream, torch.empty, (max(nbytes, 256),), dtype=torch.uint8, device=q.device)
    _check(lib().baklava_profile_similarity(q.data_ptr(), k.data_ptr(), v.data_ptr(), batch, Hq, Hkv, T, D, BF16,
                                            cos.data_ptr() if want_cos else None, sim.data_ptr(),
                                            lse.data_ptr() if want_lse else None, ws.data_ptr(),
                                            nbytes, _stream_ptr(stream)), "baklava_profile_similarity")
    _hold_until_stream_passes((sim, cos, lse), stream)
    return (sim, cos, lse) if want_lse else (sim, cos)


def prefill_scores(q, k_plane, lse, score_plane, batch: int, Hq: int, Hkv: int, T: int, row_off=None, stream=None):
    """baklava_prefill_scores: q [batch, Hq, T, 128] bf16, lse [batch, Hq, T] fp32, k_plane a bf16 tensor of
    rows of 128 elements (an arena's K plane: of a "bf16" arena, 4-bit rows are none), score_plane fp32, one value per row of
    k_plane, row_off an int64 device tensor [batch * Hkv] or None (dense).  Contiguous tensors."""
    import torch
    if q.dtype is not torch.bfloat16 or k_plane.dtype is not torch.bfloat16 or k_plane.dim() < 1 or k_plane.shape[-1] != 128:
        raise ValueError("q and k_plane must hold bf16 rows of 128 elements")
    if lse.dtype is not torch.float32 or score_plane.dtype is not torch.float32:
        raise ValueError("lse and score_plane must be fp32")
    if not (q.is_contiguous() and k_plane.is_contiguous() and lse.is_contiguous() and score_plane.is_contiguous()):
        raise ValueError("contiguous tensors expected")
    rows = batch * Hkv * T if row_off is None else T  # (at least: with row_off the rows of a sequence lie where it says)
    if q.numel() < batch * Hq * T * 128 or lse.numel() < batch * Hq * T or k_plane.numel() < rows * 128 or score_plane.numel() < rows:
        raise ValueError("tensors too small for batch, heads and T")
    if row_off is not None and (row_off.dtype is not torch.int64 or not row_off.is_contiguous() or row_off.numel() < batch * Hkv):
        raise ValueError("row_off must be a contiguous int64 tensor of one row per sequence and KV head")
    _check(lib().baklava_prefill_scores(q.data_ptr(), k_plane.data_ptr(), lse.data_ptr(),
                                        row_off.data_ptr() if row_off is not None else None, batch, Hq, Hkv, T, 128,
                                        BF16, score_plane.data_ptr(), _stream_ptr(stream)), "baklava_prefill_scores")


def alloc_two_level(layer_importance, head_importance, global_budget: int, lo: int, hi: int, t: float, r: float):
    """baklava_alloc_two_level: head_importance [L, Hkv] -> list of L * Hkv budgets (host only)."""
    himp = np.ascontiguousarray(head_importance, dtype=np.float64)
    L, Hkv = himp.shape
    limp = np.ascontiguousarray(layer_importance, dtype=np.float64)
    if limp.size != L:
        raise ValueError("one importance per layer expected")
    out = np.zeros(L * Hkv, dtype=np.int32)
    _check(lib().baklava_alloc_two_level(_p(limp, C.c_double), _p(himp.reshape(-1), C.c_double), L, Hkv,
                                         int(global_budget), lo, hi, float(t), float(r), _p(out, C.c_int32)),
           "baklava_alloc_two_level")
    return out.tolist()


def layer_similarity(x_in, x_out, want_cos: bool = True, stream=None):
    """baklava_layer_similarity on torch device tensors [n_seq, T, hidden] (bf16).
    Returns (sim [n_seq], cos [n_seq, T] or None) as torch fp32 device tensors."""
    import torch
    n_seq, T, hidden = x_in.shape
    if x_out.shape != x_in.shape or x_in.dtype != torch.bfloat16 or x_out.dtype != torch.bfloat16:
        raise ValueError("two bf16 tensors of equal shape expected")
    if not (x_in.is_contiguous() and x_out.is_contiguous()):
        raise ValueError("contiguous tensors expected")
    sim = _empty_on(stream, torch.empty, (n_seq,), dtype=torch.float32, device=x_in.device)
    cos = _empty_on(stream, torch.empty, (n_seq, T), dtype=torch.float32, device=x_in.device) if want_cos else None
    nbytes = int(lib().baklava_layer_workspace_bytes(n_seq, T))
    ws = _empty_on(stream, torch.empty, (max(nbytes, 256),), dtype=torch.uint8, device=x_in.device)
    _check(lib().baklava_layer_similarity(x_in.data_ptr(), x_out.data_ptr(), n_seq, T, hidden, BF16,
                                          cos.data_ptr() if want_cos else None, sim.data_ptr(), ws.data_ptr(), nbytes,
                                          _stream_ptr(stream)), "baklava_layer_similarity")
    _hold_until_stream_passes((sim, cos), stream)
    return sim, cos



LAYER_STATIC_MAX_TILES = 65536


def layer_similarity_static(x_in, x_out, sim, cos=None, stream=None) -> None:
    """baklava_layer_similarity_static: as layer_similarity, but the caller passes the outputs (sim [n_seq],
    cos [n_seq, T] or None, fp32 device tensors) and nothing is allocated, here or in the library."""
    n_seq, T, hidden = x_in.shape
    _check(lib().baklava_layer_similarity_static(x_in.data_ptr(), x_out.data_ptr(), n_seq, T, hidden, BF16,
                                                 cos.data_ptr() if cos is not None else None, sim.data_ptr(),
                                                 _stream_ptr(stream)), "baklava_layer_similarity_static")


# ---------------------------------------------------------------------------
# prompts
# ---------------------------------------------------------------------------

def _current_device() -> int:
    import torch
    try:
        return torch._C._cuda_getDevice()
    except AttributeError:
        return torch.cuda.current_device()


def _ints(values):
    """int32 array of host integers: (the array, which has to outlive the call, its address, sum, maximum)."""
    a = array.array("i", values)
    return a, a.buffer_info()[0], sum(a), max(a, default=0)


def _refuse_grad(torch, *tensors) -> None:
    """The library has no backward passes: a result without a graph would end a gradient silently."""
    if torch.is_grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                raise ValueError("no gradient is computed here: call under torch.no_grad() or with detached tensors")


class _Rows:
    """Up to five baklava_rows in one array of 64-bit words; each is handed over by its address, which add() returns.

    These wrappers run once per layer and step, where a small call takes some 5 us on the GPU: hence the care for what they
    cost on the host."""

    __slots__ = ("words", "at", "n", "device", "f32")

    def __init__(self, torch):
        self.words = (C.c_int64 * 20)()
        self.at = C.addressof(self.words)
        self.n = 0
        self.device = _current_device() if torch.cuda.is_initialized() else -1  # (no tensor is on a GPU then)
        self.f32 = torch.float32

    def on_device(self, t, name: str) -> None:
        if not t.is_cuda or t.get_device() != self.device:
            raise ValueError(f"{name} must be on the current GPU")

    def _put(self, t, seq, tok, head) -> int:
        i, at = self.n, self.at
        self.words[i:i + 4] = t.data_ptr(), seq, tok, head
        self.n = i + 4
        self.at = at + 32
        return at

    def add(self, t, name: str, n_seq: int, total: int, most: int, heads: int, D: int, dtype) -> int:
        """Rows of D elements: [tokens, heads, D] packed, or [batch, heads, T, D]."""
        shape = t.shape
        if len(shape) == 3 and shape[0] >= total and shape[1] == heads and shape[2] == D:
            tok, head, one = t.stride()
            seq = 0
        elif len(shape) == 4 and shape[0] == n_seq and shape[1] == heads and shape[2] >= most and shape[3] == D:
            seq, head, tok, one = t.stride()
            if n_seq > 1 and seq == 0:
                raise ValueError(f"{name}: sequences must not share their memory")
        else:
            raise ValueError(f"{name} must be [tokens, {heads}, {D}] or [batch, {heads}, T, {D}] and hold all tokens")
        if one != 1 or t.dtype is not dtype:
            raise ValueError(f"{name}: contiguous rows of {dtype} expected")
        if not t.is_cuda or t.get_device() != self.device:
            raise ValueError(f"{name} must be on the current GPU")
        return self._put(t, seq, tok, head)

    def add_values(self, t, name: str, n_seq: int, total: int, most: int, heads: int) -> int:
        """One fp32 value per token and head: [heads, tokens] packed, or [batch, heads, T]."""
        shape = t.shape
        if len(shape) == 2 and shape[0] == heads and shape[1] >= total:
            head, tok = t.stride()
            seq = 0
        elif len(shape) == 3 and shape[0] == n_seq and shape[1] == heads and shape[2] >= most:
            seq, head, tok = t.stride()
            if n_seq > 1 and seq == 0:
                raise ValueError(f"{name}: sequences must not share their memory")
        else:
            raise ValueError(f"{name} must be [{heads}, tokens] or [batch, {heads}, T] and hold all tokens")
        if t.dtype is not self.f32:
            raise ValueError(f"{name}: float32 expected")
        self.on_device(t, name)
        return self._put(t, seq, tok, head)


def _expect(rows: _Rows, t, dtype, name: str, shape) -> None:
    """A contiguous tensor of that type and shape on the current GPU."""
    if t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor {list(shape)}")
    if not t.is_cuda or t.get_device() != rows.device:
        raise ValueError(f"{name} must be on the current GPU")


def _per_node(t, name: str) -> int:
    """Nodes of a tree, from a tensor [sequences, nodes]."""
    if t.dim() != 2 or t.shape[1] < 1:
        raise ValueError(f"{name} must be [sequences, nodes], of at least one node")
    return t.shape[1]


def verify_draft(logits, token, parent, u, draft_logits=None, temperature=None, n_nodes=None, stream=None):
    """baklava_verify_draft: logits (and draft_logits) [batch, N, V] or [batch * N, V] bf16 or fp32, rows of any one stride with
    contiguous elements; token and parent int32 [batch, N], u fp32 [batch, N], temperature fp32 [batch] or None (1), n_nodes int32
    [batch] or None (N).  Returns (path [batch, N], n_path [batch], next_token [batch]), int32: whole numbers, which no gradient goes
    through, whatever the logits require."""
    import torch
    rows = _Rows(torch)
    N, batch = _per_node(parent, "parent"), parent.shape[0]
    if batch < 1:
        raise ValueError("at least one sequence expected")
    _expect(rows, parent, torch.int32, "parent", (batch, N))
    _expect(rows, token, torch.int32, "token", (batch, N))
    _expect(rows, u, torch.float32, "u", (batch, N))
    if n_nodes is not None:
        _expect(rows, n_nodes, torch.int32, "n_nodes", (batch,))
    if temperature is not None:
        _expect(rows, temperature, torch.float32, "temperature", (batch,))
    dt, V = logits.dtype, logits.shape[-1]
    if dt is not torch.bfloat16 and dt is not torch.float32:
        raise ValueError("bf16 or fp32 logits expected")
    at = []
    for t, name in ((logits, "logits"), (draft_logits, "draft_logits")):
        if t is None:
            at.append((None, 0))
            continue
        shape = t.shape
        if shape != (batch, N, V) and shape != (batch * N, V):
            raise ValueError(f"{name} must be [{batch}, {N}, {V}] or [{batch * N}, {V}]")
        if t.dtype is not dt or (V > 1 and t.stride(-1) != 1) or (len(shape) == 3 and N > 1 and batch > 1 and t.stride(0) != N * t.stride(1)):
            raise ValueError(f"{name}: contiguous rows of {dt}, at one distance, expected")
        rows.on_device(t, name)
        at.append((t.data_ptr(), t.stride(0) if len(shape) == 2 or N == 1 else t.stride(1)))
    nbytes = lib().baklava_verify_workspace_bytes(batch, N, V, int(draft_logits is not None))
    if stream is None:
        path, n_path, token_out = parent.new_empty((batch, N)), parent.new_empty(batch), parent.new_empty(batch)
    else:
        path, n_path, token_out = (_empty_on(stream, parent.new_empty, n) for n in ((batch, N), batch, batch))
    ws = _empty_on(stream, parent.new_empty, max(nbytes, 256), dtype=torch.uint8)
    _check(lib().baklava_verify_draft(at[0][0], at[0][1], at[1][0], at[1][1], BF16 if dt is torch.bfloat16 else F32, batch, N, V,
                                      token.data_ptr(), parent.data_ptr(), n_nodes.data_ptr() if n_nodes is not None else None,
                                      temperature.data_ptr() if temperature is not None else None, u.data_ptr(), path.data_ptr(),
                                      n_path.data_ptr(), token_out.data_ptr(), ws.data_ptr(), nbytes, _stream_ptr(stream)),
           "baklava_verify_draft")
    _hold_until_stream_passes((path, n_path, token_out), stream)
    return path, n_path, token_out


def prompt_attn(q, k, v, lens: Sequence[int], kv_lens: Optional[Sequence[int]] = None, out=None, lse=None,
                want_lse: bool = False, stream=None):
    """baklava_prompt_attn on torch device tensors (bf16): q [tokens, Hq, D], k and v [keys, Hkv, D] (the sequences in a row)
    or q [batch, Hq, T, D], k and v [batch, Hkv, T', D] (padded); lens query tokens and kv_lens keys of every sequence.
    Returns out (like q; places past a sequence's length are not written), and with want_lse or lse given also lse (fp32
    [Hq, tokens] or [batch, Hq, T]).  No gradient: tensors that require one are refused outside torch.no_grad()."""
    import torch
    _refuse_grad(torch, q, k, v)
    q_shape, k_shape = q.shape, k.shape
    if len(q_shape) not in (3, 4) or len(k_shape) not in (3, 4) or k_shape != v.shape:
        raise ValueError("q, k, v of three or four dimensions expected, k and v alike")
    n_seq = len(lens)
    if n_seq == 0 or (kv_lens is not None and len(kv_lens) != n_seq):
        raise ValueError("one length per sequence expected")
    n_q, q_at, total, most = _ints(lens)
    n_k, k_at, k_total, k_most = _ints(kv_lens) if kv_lens is not None else (n_q, None, total, most)
    if min(n_q) < 0 or min(n_k) < 0:
        raise ValueError("lengths must not be negative")
    Hq, Hkv, D = q_shape[1], k_shape[1], q_shape[-1]
    dt = torch.bfloat16
    rows = _Rows(torch)
    at = [rows.add(q, "q", n_seq, total, most, Hq, D, dt), rows.add(k, "k", n_seq, k_total, k_most, Hkv, D, dt),
          rows.add(v, "v", n_seq, k_total, k_most, Hkv, D, dt)]
    if out is None:
        out = q.new_empty(q_shape) if stream is None else _empty_on(stream, q.new_empty, q_shape)
    if lse is None and want_lse:
        lse = _empty_on(stream, q.new_empty, (Hq, q_shape[0]) if len(q_shape) == 3 else q_shape[:3], dtype=torch.float32)
    at.append(rows.add(out, "out", n_seq, total, most, Hq, D, dt))
    at.append(rows.add_values(lse, "lse", n_seq, total, most, Hq) if lse is not None else None)
    _check(lib().baklava_prompt_attn(at[0], at[1], at[2], n_seq, q_at, k_at, Hq, Hkv, D, BF16, at[3], at[4],
                                     _stream_ptr(stream)), "baklava_prompt_attn")
    _hold_until_stream_passes((out, lse), stream)
    return (out, lse) if lse is not None else out


def _axes(sections, axis_of_pair, n_freq: int, axes: int) -> Optional[bytes]:
    """The axis of every pair, a byte each; None: axis 0 for all."""
    if sections is not None:
        if axis_of_pair is not None or sum(sections) != n_freq or len(sections) > axes or min(sections, default=0) < 0:
            raise ValueError("sections must add up to the number of pairs, at most one for each axis")
        return b"".join([bytes((a,)) * n for a, n in enumerate(sections)]) if len(sections) > 1 else None
    if axis_of_pair is not None:
        if len(axis_of_pair) != n_freq or any(not 0 <= a < axes for a in axis_of_pair):
            raise ValueError("axis_of_pair must name an axis for every pair")
        return bytes(list(axis_of_pair))  # (an array's own bytes are those of its words)
    return None


def qk_norm_rope(q, k, pos, inv_freq: Sequence[float], q_weight=None, k_weight=None, eps: float = 1e-6,
                 sections: Optional[Sequence[int]] = None, axis_of_pair: Optional[Sequence[int]] = None,
                 interleaved: bool = False, q_out=None, k_out=None, stream=None):
    """baklava_qk_norm_rope on torch device tensors: q [tokens, Hq, D], k [tokens, Hkv, D] or [batch, H, T, D] (either may be
    None), bf16 or fp32, of any strides with contiguous rows; pos int32 [tokens] or [axes, tokens] ([axes, batch, T] in any
    shape of as many values); inv_freq one frequency per pair of rotated elements (empty: no rotation, pos is not looked at).
    The axis of every pair is given by axis_of_pair, or by sections: pairs of axis 0, of axis 1, ...  Weights [D] or None (not
    normed).  q_out, k_out may be q and k.  Returns (q_out, k_out).  No gradient: tensors that require one are refused outside
    torch.no_grad()."""
    import torch
    _refuse_grad(torch, q, k, q_weight, k_weight)
    t0 = q if q is not None else k
    if t0 is None or (q is not None and k is not None and q.dim() != k.dim()):
        raise ValueError("q or k of three or four dimensions expected, both alike")
    shape, dtype = t0.shape, t0.dtype
    if len(shape) == 3:
        n_seq, T = 1, shape[0]
    elif len(shape) == 4:
        n_seq, T = shape[0], shape[2]
    else:
        raise ValueError("q or k of three or four dimensions expected, both alike")
    if dtype is not torch.bfloat16 and dtype is not torch.float32:
        raise ValueError("bf16 or fp32 tensors expected")
    D, tokens = shape[-1], n_seq * T
    if k is not None and ((1, k.shape[0]) if len(shape) == 3 else (k.shape[0], k.shape[2])) != (n_seq, T):
        raise ValueError("q and k must hold the same tokens")
    if tokens == 0:
        return tuple(None if t is None else o if o is not None else torch.empty_like(t) for t, o in ((q, q_out), (k, k_out)))
    rows = _Rows(torch)
    freq = array.array("d", inv_freq)
    n_freq, axes, pos_at = len(freq), 1, None
    if n_freq:
        n_pos = pos.numel()
        if pos.dtype is not torch.int32 or not pos.is_contiguous() or n_pos == 0 or n_pos % tokens:
            raise ValueError("pos must be a contiguous int32 tensor with one value per axis and token")
        rows.on_device(pos, "pos")
        axes, pos_at = n_pos // tokens, pos.data_ptr()
    axis = _axes(sections, axis_of_pair, n_freq, axes)
    in_at, out_at, w_at, outs, heads = [None, None], [None, None], [None, None], [None, None], [0, 0]
    for i, (t, name, w, o) in enumerate(((q, "q", q_weight, q_out), (k, "k", k_weight, k_out))):
        if t is None:
            if w is not None or o is not None:
                raise ValueError(f"no {name} given")
            continue
        h = heads[i] = t.shape[1]
        in_at[i] = rows.add(t, name, n_seq, tokens, T, h, D, dtype)
        if w is not None:
            if w.dtype is not dtype or w.shape != (D,) or not w.is_contiguous():
                raise ValueError(f"{name}_weight must be a contiguous [{D}] tensor of the rows' type")
            rows.on_device(w, f"{name}_weight")
            w_at[i] = w.data_ptr()
        if o is None:
            o = t.new_empty(t.shape) if stream is None else _empty_on(stream, t.new_empty, t.shape)
        elif o.shape != t.shape:
            raise ValueError(f"{name}_out must have the shape of {name}")
        out_at[i], outs[i] = rows.add(o, f"{name}_out", n_seq, tokens, T, h, D, dtype), o
    _check(lib().baklava_qk_norm_rope(in_at[0], in_at[1], n_seq, T, heads[0], heads[1], D,
                                      BF16 if dtype is torch.bfloat16 else F32, w_at[0], w_at[1], float(eps), pos_at, axes, axis,
                                      freq.buffer_info()[0], 2 * n_freq, 1 if interleaved else 0, out_at[0], out_at[1],
                                      _stream_ptr(stream)), "baklava_qk_norm_rope")
    _hold_until_stream_passes(outs, stream)
    return outs[0], outs[1]
