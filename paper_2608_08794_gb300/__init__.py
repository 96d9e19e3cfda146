"""Python binding of libapack, the GB300 (sm_103a) A-PACK inner-LLM prune step.

Argument marshalling only: every computation runs in the CUDA kernels of
``libapack.so`` behind the C ABI declared in ``include/apack.h``.  The
functions keep the C names (``apack_score``, ``apack_select``,
``apack_compact``, ``apack_prune_step``, ...).  Device buffers are passed as
torch CUDA tensors (their data pointers) and streams as torch streams;
PyTorch only provides memory and streams.

Importing this package loads the library and raises if it has not been
built (``__graft_entry__.build()`` or ``python -m paper_2608_08794_gb300._build``).
There is no fallback.
"""

import ctypes
import math
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libapack.so")

APACK_OK, APACK_EINVAL, APACK_ECUDA, APACK_EWORKSPACE, APACK_ETIMEOUT, APACK_EDEVICE, APACK_EUNSUPPORTED = range(7)
APACK_MOD_OTHER, APACK_MOD_AUDIO, APACK_MOD_VISUAL = 0, 1, 2
APACK_SELECT_PER_MODALITY, APACK_SELECT_JOINT = 0, 1
APACK_SOFTMAX_MM, APACK_SOFTMAX_CAUSAL_ROW = 0, 1
APACK_HEAD_DIM = 128
APACK_BF16, APACK_FP16, APACK_FP32 = 0, 1, 2
APACK_ROTARY_HALF, APACK_ROTARY_PAIRS = 0, 1
APACK_ROTARY_NONE, APACK_ROTARY_LINEAR, APACK_ROTARY_NTK, APACK_ROTARY_YARN = range(4)

EXPORTED = ("apack_workspace_size", "apack_keep_counts", "apack_score", "apack_select", "apack_compact",
            "apack_prune_step", "apack_device_error", "apack_launch_count", "apack_status_string",
            "apack_score_static", "apack_frame_alignment_workspace_size", "apack_frame_alignment",
            "apack_decode_workspace_size", "apack_decode_attention", "apack_prune_schedule",
            "apack_prune_schedule_graph", "apack_graph_launch", "apack_graph_destroy",
            "apack_rotary_frequencies", "apack_rotary", "apack_rotary_append", "apack_paged_decode_workspace_size",
            "apack_paged_decode_attention", "apack_paged_compact", "apack_copy_pages")


class ApackError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class apack_seqs(ctypes.Structure):
    _fields_ = [("num_seqs", ctypes.c_int32),
                ("cu_seqlens_h", ctypes.POINTER(ctypes.c_int32)),
                ("cu_qlens_h", ctypes.POINTER(ctypes.c_int32)),
                ("n_audio_h", ctypes.POINTER(ctypes.c_int32)),
                ("n_visual_h", ctypes.POINTER(ctypes.c_int32)),
                ("modality", ctypes.c_void_p),
                ("num_q_heads", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32),
                ("softmax_domain", ctypes.c_int32),
                ("q_start_h", ctypes.POINTER(ctypes.c_int32))]


class apack_plane(ctypes.Structure):
    _fields_ = [("src", ctypes.c_void_p), ("dst", ctypes.c_void_p),
                ("src_plane_stride", ctypes.c_int64), ("dst_plane_stride", ctypes.c_int64),
                ("src_row_stride", ctypes.c_int64), ("dst_row_stride", ctypes.c_int64),
                ("row_bytes", ctypes.c_int64), ("num_planes", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class apack_step(ctypes.Structure):
    _fields_ = [("layer", ctypes.c_int32), ("q", ctypes.c_void_p),
                ("keep_count_h", ctypes.POINTER(ctypes.c_int32)), ("keep_ratio_h", ctypes.POINTER(ctypes.c_float)),
                ("k_out", ctypes.c_void_p), ("v_out", ctypes.c_void_p), ("kv_out_layer_stride", ctypes.c_int64),
                ("hidden_out", ctypes.c_void_p), ("extra_planes_h", ctypes.POINTER(apack_plane)),
                ("num_extra", ctypes.c_int32), ("modality_out", ctypes.c_void_p), ("keep_idx", ctypes.c_void_p),
                ("new_cu_seqlens_h", ctypes.POINTER(ctypes.c_int32)), ("new_cu_seqlens", ctypes.c_void_p)]


class apack_paged_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("layer_stride", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("token_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("num_layers", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32),
                ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("page_table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("num_seqs", ctypes.c_int32),
                ("max_pages", ctypes.c_int32)]


class apack_rotary_spec(ctypes.Structure):
    _fields_ = [("layout", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("num_axes", ctypes.c_int32),
                ("section", ctypes.c_int32 * 3), ("magnitude", ctypes.c_float),
                ("freq_h", ctypes.POINTER(ctypes.c_double))]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"libapack.so is not built ({LIB_PATH}); run __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    P, I32, I64, SZ, VP = ctypes.POINTER, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_void_p
    PI32 = VP                     # host arrays go in as plain addresses (see _host)
    lib.apack_workspace_size.argtypes = [P(apack_seqs), P(SZ)]
    lib.apack_keep_counts.argtypes = [P(apack_seqs), VP, I32, PI32, PI32]
    lib.apack_score.argtypes = [P(apack_seqs), VP, VP, I64, VP, VP, SZ, VP]
    lib.apack_select.argtypes = [P(apack_seqs), VP, VP, PI32, I32, VP, VP, VP, VP, VP, SZ, VP]
    lib.apack_compact.argtypes = [VP, I64, P(apack_plane), I32, VP, VP]
    lib.apack_prune_step.argtypes = [P(apack_seqs), I32, I32, VP, VP, VP, I64, VP, I64, VP, PI32,
                                     I32, VP, VP, I64, VP, P(apack_plane), I32, VP, VP, PI32, VP, VP, VP, SZ,
                                     P(VP), VP]
    lib.apack_device_error.argtypes = [VP, VP, PI32, I32]
    lib.apack_score_static.argtypes = [P(apack_seqs), VP, VP, I64, VP, VP, VP]
    lib.apack_frame_alignment_workspace_size.argtypes = [I32, I64, P(SZ)]
    lib.apack_frame_alignment.argtypes = [VP, VP, I32, I32, I32, I64, I32, ctypes.c_float, ctypes.c_float, VP, VP,
                                          VP, VP, VP, SZ, VP]
    lib.apack_decode_workspace_size.argtypes = [I32, PI32, I32, I32, P(SZ)]
    lib.apack_decode_attention.argtypes = [I32, PI32, VP, VP, VP, I64, I32, I32, VP, VP, SZ, VP]
    lib.apack_prune_schedule.argtypes = [P(apack_seqs), I32, VP, VP, I64, VP, I64, I32, P(apack_step), I32, VP, VP,
                                         SZ, P(VP), VP]
    lib.apack_prune_schedule_graph.argtypes = [P(apack_seqs), I32, VP, VP, I64, VP, I64, I32, P(apack_step), I32,
                                               VP, VP, SZ, P(VP)]
    lib.apack_graph_launch.argtypes = [VP, VP]
    lib.apack_graph_destroy.argtypes = [VP]
    F32, F64 = ctypes.c_float, ctypes.c_double
    lib.apack_rotary_frequencies.argtypes = [I32, F64, I32, F64, I64, F64, F64, VP, P(F32)]
    lib.apack_rotary.argtypes = [VP, I32, I64, I32, I32, VP, I64, VP, I64, VP, I64, I32, VP]
    lib.apack_rotary_append.argtypes = [VP, VP, I32, I64, VP, I64, VP, I64, I32, VP, I64, VP, I64, VP, I64, VP, VP,
                                        VP, VP]
    lib.apack_paged_decode_workspace_size.argtypes = [VP, I32, P(SZ)]
    lib.apack_paged_decode_attention.argtypes = [VP, I32, VP, VP, I64, I32, F32, VP, I32, VP, VP, SZ, VP]
    lib.apack_paged_compact.argtypes = [VP, VP, I32, I32, I32, VP, VP, VP, I64, VP, VP]
    lib.apack_copy_pages.argtypes = [VP, VP, I64, VP, VP]
    lib.apack_launch_count.argtypes = []
    lib.apack_launch_count.restype = ctypes.c_uint64
    lib.apack_status_string.argtypes = [I32]
    lib.apack_status_string.restype = ctypes.c_char_p
    for name in EXPORTED:
        if name not in ("apack_launch_count", "apack_status_string"):
            getattr(lib, name).restype = I32
    return lib


_lib = _load()


def status_string(status):
    return _lib.apack_status_string(int(status)).decode()


def _check(status, where):
    if status != APACK_OK:
        raise ApackError(status, where)


def _ptr(t):
    """Device address of a torch tensor (or None -> NULL)."""
    return None if t is None else t.data_ptr()


def _current_stream():
    """The current device's current stream, as an address.  torch.cuda.current_stream() builds a
    Stream object on every call; its raw handle is the same."""
    import torch
    if torch.cuda.is_initialized():
        try:
            return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
        except AttributeError:
            pass
    return torch.cuda.current_stream().cuda_stream


def _stream(stream):
    if stream is None:
        return _current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _i32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.int32))


def _f32(a):
    return np.ascontiguousarray(np.asarray(a, dtype=np.float32))


def _host(a):
    """Address of a contiguous host array (or None -> NULL); the caller keeps the array alive."""
    return None if a is None else a.ctypes.data


def _planes(planes):
    return (apack_plane * len(planes))(*planes) if len(planes) else None


class Seqs:
    """A packed batch: host offsets and counts plus the device modality mask.

    Keeps the host arrays alive for as long as the ``apack_seqs`` struct is used."""

    def __init__(self, cu_seqlens, cu_qlens, n_audio, n_visual, modality, num_q_heads, num_kv_heads,
                 head_dim=APACK_HEAD_DIM, softmax_domain=0, q_start=None):
        self.cu_seqlens = _i32(cu_seqlens)
        self.cu_qlens = _i32(cu_qlens)
        self.n_audio = _i32(n_audio)
        self.n_visual = _i32(n_visual)
        self.q_start = None if q_start is None else _i32(q_start)
        self.modality = modality
        I32P = ctypes.POINTER(ctypes.c_int32)
        self.struct = apack_seqs(
            num_seqs=len(self.cu_seqlens) - 1,
            cu_seqlens_h=self.cu_seqlens.ctypes.data_as(I32P),
            cu_qlens_h=self.cu_qlens.ctypes.data_as(I32P),
            n_audio_h=self.n_audio.ctypes.data_as(I32P),
            n_visual_h=self.n_visual.ctypes.data_as(I32P),
            modality=None if modality is None else modality.data_ptr(),
            num_q_heads=num_q_heads, num_kv_heads=num_kv_heads, head_dim=head_dim,
            softmax_domain=int(softmax_domain),
            q_start_h=None if self.q_start is None else self.q_start.ctypes.data_as(I32P))
        self.softmax_domain = int(softmax_domain)

    @property
    def num_seqs(self):
        return len(self.cu_seqlens) - 1

    @property
    def total_tokens(self):
        return int(self.cu_seqlens[-1])

    def ref(self):
        return ctypes.byref(self.struct)


def apack_workspace_size(seqs):
    n = ctypes.c_size_t(0)
    _check(_lib.apack_workspace_size(seqs.ref(), ctypes.byref(n)), "apack_workspace_size")
    return n.value


def apack_keep_counts(seqs, keep_ratio, select_mode=APACK_SELECT_PER_MODALITY):
    """Keep counts [B, 2] and new offsets [B+1] (host numpy) from keep ratios [B, 2]."""
    r = np.ascontiguousarray(np.asarray(keep_ratio, dtype=np.float32).reshape(seqs.num_seqs, 2))
    k = np.zeros((seqs.num_seqs, 2), np.int32)
    cu = np.zeros(seqs.num_seqs + 1, np.int32)
    _check(_lib.apack_keep_counts(seqs.ref(), _host(r), select_mode, _host(k), _host(cu)), "apack_keep_counts")
    return k, cu


def apack_score(seqs, q, k, k_token_stride, scores, ws, stream=None):
    _check(_lib.apack_score(seqs.ref(), _ptr(q), _ptr(k), int(k_token_stride), _ptr(scores), _ptr(ws),
                            ws.numel() * ws.element_size(), _stream(stream)), "apack_score")


def apack_select(seqs, scores, keep_count, keep_idx, ws, select_mode=APACK_SELECT_PER_MODALITY,
                 modality_out=None, dst_of_src=None, new_cu_seqlens=None, stream=None, keep_ratio=None):
    """keep_count: [B, 2] counts, or None with keep_ratio [B, 2] (ratios 1-P of Eq. inner)."""
    kc = None if keep_count is None else _i32(keep_count)
    kr = None if keep_ratio is None else _f32(keep_ratio)
    _check(_lib.apack_select(seqs.ref(), _ptr(scores), _host(kr), _host(kc), select_mode, _ptr(keep_idx), _ptr(modality_out), _ptr(dst_of_src),
                             _ptr(new_cu_seqlens), _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "apack_select")


def make_plane(src, dst, row_bytes, num_planes=1, src_plane_stride=0, dst_plane_stride=0, src_row_stride=None,
               dst_row_stride=None):
    """Descriptor of a group of per-token planes (byte strides)."""
    return apack_plane(src=src.data_ptr(), dst=dst.data_ptr(), src_plane_stride=src_plane_stride,
                       dst_plane_stride=dst_plane_stride,
                       src_row_stride=row_bytes if src_row_stride is None else src_row_stride,
                       dst_row_stride=row_bytes if dst_row_stride is None else dst_row_stride,
                       row_bytes=row_bytes, num_planes=num_planes, reserved=0)


def apack_compact(keep_idx, n_out, planes, ws=None, stream=None):
    _check(_lib.apack_compact(_ptr(keep_idx), int(n_out), _planes(planes), len(planes), _ptr(ws), _stream(stream)),
           "apack_compact")


def apack_prune_step(seqs, layer, num_layers, q, k_cache, v_cache, kv_layer_stride, hidden, hidden_dim,
                     keep_ratio=None, keep_count=None, select_mode=APACK_SELECT_PER_MODALITY, k_out=None,
                     v_out=None, kv_out_layer_stride=0, hidden_out=None, extra_planes=(), modality_out=None,
                     keep_idx=None, new_cu_seqlens=None, scores=None, ws=None, stage_events=None, stream=None):
    """One pruning step; returns the new packed offsets (host numpy [B+1])."""
    B = seqs.num_seqs
    ratio = None
    if keep_ratio is not None:
        ratio = np.ascontiguousarray(np.asarray(keep_ratio, dtype=np.float32).reshape(B, 2))
    kc = None if keep_count is None else _i32(keep_count)
    new_cu = np.zeros(B + 1, np.int32)
    ev = None
    if stage_events is not None:
        handles = [e.cuda_event if hasattr(e, "cuda_event") else e for e in stage_events]
        if len(handles) != 4 or not all(handles):
            raise ValueError("stage_events: four created CUDA events (record a torch event once to create it)")
        ev = (ctypes.c_void_p * 4)(*handles)
    st = _lib.apack_prune_step(
        seqs.ref(), int(layer), int(num_layers), _ptr(q), _ptr(k_cache), _ptr(v_cache), int(kv_layer_stride),
        _ptr(hidden), int(hidden_dim), _host(ratio), _host(kc), select_mode, _ptr(k_out), _ptr(v_out),
        int(kv_out_layer_stride), _ptr(hidden_out), _planes(extra_planes), len(extra_planes), _ptr(modality_out),
        _ptr(keep_idx), _host(new_cu), _ptr(new_cu_seqlens), _ptr(scores), _ptr(ws),
        0 if ws is None else ws.numel() * ws.element_size(), ev, _stream(stream))
    _check(st, "apack_prune_step")
    return new_cu


def _event_handles(events, n, what):
    if events is None:
        return None
    handles = [0 if e is None else (e.cuda_event if hasattr(e, "cuda_event") else e) for e in events]
    if len(handles) != n:
        raise ValueError(f"{what}: {n} events expected")
    return (ctypes.c_void_p * n)(*handles)


def apack_prune_schedule(seqs, num_layers, k_cache, v_cache, kv_layer_stride, hidden, hidden_dim, steps,
                         select_mode=APACK_SELECT_PER_MODALITY, scores=None, ws=None, stage_events=None, stream=None,
                         capture=False):
    """A whole progressive schedule (one apack_prune_step per entry of `steps`, each
    reading the previous step's outputs).  steps: dicts with layer, q, keep_count or
    keep_ratio, k_out, v_out, kv_out_layer_stride, hidden_out, modality_out, keep_idx
    and optionally new_cu_seqlens (device) and extra_planes.  stage_events: None or
    4 * len(steps) created events.  Returns the new host offsets of every step."""
    B = seqs.num_seqs
    n = len(steps)
    I32P = ctypes.POINTER(ctypes.c_int32)
    keep = []                           # host arrays referenced by the call
    arr = (apack_step * n)()
    new_cus = []
    for i, d in enumerate(steps):
        st = arr[i]
        st.layer = int(d["layer"])
        st.q = _ptr(d["q"])
        if d.get("keep_count") is not None:
            kc = _i32(d["keep_count"]).reshape(-1)
            keep.append(kc)
            st.keep_count_h = kc.ctypes.data_as(I32P)
        else:
            r = np.ascontiguousarray(np.asarray(d["keep_ratio"], dtype=np.float32).reshape(B, 2))
            keep.append(r)
            st.keep_ratio_h = r.ctypes.data_as(ctypes.POINTER(ctypes.c_float))
        st.k_out, st.v_out = _ptr(d["k_out"]), _ptr(d["v_out"])
        st.kv_out_layer_stride = int(d["kv_out_layer_stride"])
        st.hidden_out = _ptr(d.get("hidden_out"))
        extra = d.get("extra_planes", ())
        if extra:
            ep = (apack_plane * len(extra))(*extra)
            keep.append(ep)
            st.extra_planes_h = ctypes.cast(ep, ctypes.POINTER(apack_plane))
        st.num_extra = len(extra)
        st.modality_out = _ptr(d["modality_out"])
        st.keep_idx = _ptr(d["keep_idx"])
        cu = np.zeros(B + 1, np.int32)
        new_cus.append(cu)
        st.new_cu_seqlens_h = cu.ctypes.data_as(I32P)
        st.new_cu_seqlens = _ptr(d.get("new_cu_seqlens"))
    head = (seqs.ref(), int(num_layers), _ptr(k_cache), _ptr(v_cache), int(kv_layer_stride), _ptr(hidden),
            int(hidden_dim), int(select_mode), arr, n, _ptr(scores), _ptr(ws),
            0 if ws is None else ws.numel() * ws.element_size())
    if capture:
        g = ctypes.c_void_p()
        _check(_lib.apack_prune_schedule_graph(*head, ctypes.byref(g)), "apack_prune_schedule_graph")
        # the graph replays on these device buffers: keep them alive with it
        buffers = [t for t in (k_cache, v_cache, hidden, scores, ws, seqs.modality) if t is not None]
        for d in steps:
            buffers += [v for v in d.values() if hasattr(v, "data_ptr")]
        return new_cus, ScheduleGraph(g, buffers)
    stage = _event_handles(stage_events, 4 * n, "stage_events")
    _check(_lib.apack_prune_schedule(*head, stage, _stream(stream)), "apack_prune_schedule")
    return new_cus


class ScheduleGraph:
    """An executable CUDA graph of one schedule (apack_prune_schedule_graph);
    launch() replays it, the graph is freed with the object.  The graph reads
    and writes the device buffers it was captured on, so the object holds
    references to them (inputs, outputs, scores, workspace) until it is closed."""

    def __init__(self, handle, buffers=()):
        self._h = handle
        self._buffers = list(buffers)

    def launch(self, stream=None):
        _check(_lib.apack_graph_launch(self._h, _stream(stream)), "apack_graph_launch")

    def close(self):
        if self._h is not None and self._h.value:
            _check(_lib.apack_graph_destroy(self._h), "apack_graph_destroy")
        self._h = None
        self._buffers = []

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def apack_prune_schedule_graph(seqs, num_layers, k_cache, v_cache, kv_layer_stride, hidden, hidden_dim, steps,
                               select_mode=APACK_SELECT_PER_MODALITY, scores=None, ws=None):
    """Captures the schedule of apack_prune_schedule (same arguments) into a CUDA
    graph.  Returns (new host offsets of every step, ScheduleGraph)."""
    return apack_prune_schedule(seqs, num_layers, k_cache, v_cache, kv_layer_stride, hidden, hidden_dim, steps,
                                select_mode=select_mode, scores=scores, ws=ws, capture=True)


def apack_score_static(seqs, q, k, k_token_stride, scores, device_error_out=None, stream=None):
    """apack_score without a workspace, for callers that cannot allocate device
    memory (the library's fixed 8 MiB scratch array is used instead)."""
    _check(_lib.apack_score_static(seqs.ref(), _ptr(q), _ptr(k), int(k_token_stride), _ptr(scores),
                                   _ptr(device_error_out), _stream(stream)), "apack_score_static")


def apack_frame_alignment_workspace_size(n_frames, dim):
    n = ctypes.c_size_t(0)
    _check(_lib.apack_frame_alignment_workspace_size(int(n_frames), int(dim), ctypes.byref(n)),
           "apack_frame_alignment_workspace_size")
    return n.value


def apack_frame_alignment(visual, audio, n_frames, tokens_per_frame, n_audio, dim, c_out, s_out, ws, window=3,
                          tau=0.78, beta=0.90, dnorm_out=None, cbar_out=None, stream=None):
    """Pre-LLM windowed CKA c_f and gated score s_f per frame (Sec. 3.1)."""
    _check(_lib.apack_frame_alignment(_ptr(visual), _ptr(audio), int(n_frames), int(tokens_per_frame), int(n_audio),
                                      int(dim), int(window), float(tau), float(beta), _ptr(c_out), _ptr(s_out),
                                      _ptr(dnorm_out), _ptr(cbar_out), _ptr(ws), ws.numel() * ws.element_size(),
                                      _stream(stream)), "apack_frame_alignment")


def apack_decode_workspace_size(cu_seqlens, num_q_heads, num_kv_heads):
    cu = _i32(cu_seqlens)
    n = ctypes.c_size_t(0)
    _check(_lib.apack_decode_workspace_size(len(cu) - 1, _host(cu), int(num_q_heads),
                                            int(num_kv_heads), ctypes.byref(n)), "apack_decode_workspace_size")
    return n.value


def apack_decode_attention(cu_seqlens, q, k, v, kv_token_stride, num_q_heads, num_kv_heads, out, ws, stream=None):
    """Attention of one decode token per sequence over its KV cache (Sec. 3.2)."""
    cu = _i32(cu_seqlens)
    _check(_lib.apack_decode_attention(len(cu) - 1, _host(cu), _ptr(q), _ptr(k), _ptr(v),
                                       int(kv_token_stride), int(num_q_heads), int(num_kv_heads), _ptr(out),
                                       _ptr(ws), ws.numel() * ws.element_size(), _stream(stream)),
           "apack_decode_attention")


# ---------------------------------------------------------------- paged caches


_DTYPES = {"torch.bfloat16": APACK_BF16, "torch.float16": APACK_FP16, "torch.float32": APACK_FP32}
_CODES = {}                       # torch type -> code, filled as types are met


def _dtype_code(dtype):
    code = _CODES.get(dtype)
    if code is None:
        code = _DTYPES.get(str(dtype))
        if code is None:
            raise ValueError(f"{dtype}: bfloat16, float16 or float32 expected")
        _CODES[dtype] = code
    return code


_cuda = None                      # (current device, current stream of a device), looked up once CUDA is there
_int32_type = None                # torch.int32, likewise


# The calls of a decode step take the host longer than the device.  So their wrappers test what is usual in a few plain
# comparisons, and leave what is not (the unusual that is right, and the messages) to the functions below.


def _on_device(tensors, stream):
    """The calls run on the current device: tensors elsewhere are refused (without a device the library's own checks
    answer).  Returns the address of the stream, the device's current one when None."""
    global _cuda, _int32_type
    if _cuda is None:
        import torch
        _int32_type = torch.int32
        if torch.cuda.is_initialized() or torch.cuda.is_available():
            torch.cuda.current_device()              # initialises
            try:
                _cuda = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
            except AttributeError:
                _cuda = torch.cuda.current_device, lambda dev: torch.cuda.current_stream(dev).cuda_stream
    dev = -1 if _cuda is None else _cuda[0]()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"a tensor on device {t.get_device()}; the current device is {dev}")
    return _cuda[1](dev) if stream is None and _cuda is not None else _stream(stream)


def _int32(t, what, shape=None):
    if str(t.dtype) != "torch.int32" or not t.is_contiguous() or (shape is not None and t.shape != shape):
        raise ValueError(f"{what}: contiguous int32{'' if shape is None else f' of shape {shape}'} expected, "
                         f"not {t.dtype} {tuple(t.shape)}")


def _head_rows(t, what, dtype=None, shape=None):
    """A [tokens, heads, D] tensor whose heads are back to back; returns its token stride in elements."""
    dims, stride = t.shape, t.stride()
    if dtype is not None and t.dtype != dtype:
        raise ValueError(f"{what}: {dtype} expected, not {t.dtype}")
    if shape is not None and dims != shape:
        raise ValueError(f"{what}: shape {tuple(shape)} expected, not {tuple(dims)}")
    if len(dims) != 3 or stride[2] != 1 or (stride[1] != dims[2] and dims[1] > 1):
        raise ValueError(f"{what}: [tokens, heads, D] with heads back to back expected")
    return stride[0] if dims[0] > 1 else dims[1] * dims[2]


class PagedCache:
    """A pool of key-value pages and the page tables of a batch (apack_paged_cache).

    k, v: [layers, pages, page_tokens, Hkv, D] bfloat16 or float16 tensors of equal strides, D contiguous; any
    order of the other dimensions in memory (permute a [layers, pages, Hkv, page_tokens, D] pool).  page_table:
    int32 [num_seqs, max_pages].  Holds the tensors."""

    def __init__(self, k, v, page_table):
        import torch
        if k.dim() != 5 or k.shape != v.shape or k.stride() != v.stride() or k.dtype != v.dtype or k.stride(4) != 1:
            raise ValueError("k and v: [layers, pages, page_tokens, heads, D] of one shape, type and strides expected")
        if page_table.dtype != torch.int32 or page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
            raise ValueError("page_table: int32 [sequences, pages] with contiguous rows expected")
        if not k.get_device() == v.get_device() == page_table.get_device():
            raise ValueError("k, v and page_table: one device expected")
        self._tensors = k, v, page_table
        self.dtype, self._device = k.dtype, k.get_device()
        size = k.element_size()
        layers, pages, tokens, heads, dim = k.shape
        seqs, columns = page_table.shape
        self.num_kv_heads, self.head_dim, self.num_seqs, self.num_layers = heads, dim, seqs, layers
        self._scale = 1.0 / math.sqrt(dim)
        # a stride of an extent of one says nothing, and may be anything
        stride = [k.stride(i) * size if k.shape[i] > 1 else 0 for i in range(4)]
        self.struct = apack_paged_cache(
            k=k.data_ptr(), v=v.data_ptr(), layer_stride=stride[0], page_stride=stride[1], token_stride=stride[2],
            head_stride=stride[3], num_layers=layers, num_pages=pages, page_tokens=tokens, num_kv_heads=heads,
            head_dim=dim, dtype=_dtype_code(k.dtype), page_table=page_table.data_ptr(),
            table_stride=page_table.stride(0) if seqs > 1 else columns, num_seqs=seqs, max_pages=columns)
        self._address = ctypes.addressof(self.struct)

    # struct holds their addresses: other tensors take another PagedCache
    k = property(lambda self: self._tensors[0])
    v = property(lambda self: self._tensors[1])
    page_table = property(lambda self: self._tensors[2])

    def get_device(self):
        return self._device


class Rotary:
    """Rotary positions (apack_rotary_spec): frequencies of a form of scaling, or given ones.

    scaling: "none", "linear", "ntk" or "yarn" (see apack_rotary_frequencies); frequencies: radians per position
    of the rotary_dim / 2 pairs, in the place of base and scaling.  sections: pairs per position axis (2 or 3
    axes).  interleaved: pairs of neighbouring elements, else of the two halves.  The attributes that say what it was
    made with are read-only."""

    def __init__(self, rotary_dim, base=10000.0, interleaved=False, scaling="none", factor=1.0, original_len=0,
                 beta_fast=32.0, beta_slow=1.0, sections=None, magnitude=None, frequencies=None):
        modes = {"none": APACK_ROTARY_NONE, "linear": APACK_ROTARY_LINEAR, "ntk": APACK_ROTARY_NTK,
                 "yarn": APACK_ROTARY_YARN}
        if scaling not in modes:
            raise ValueError(f"scaling {scaling!r}: one of {', '.join(modes)} expected")
        pairs = max(1, int(rotary_dim) // 2)
        m = ctypes.c_float(1.0)
        if frequencies is None:
            frequencies = np.zeros(pairs, np.float64)
            _check(_lib.apack_rotary_frequencies(int(rotary_dim), float(base), modes[scaling], float(factor),
                                                 int(original_len), float(beta_fast), float(beta_slow),
                                                 _host(frequencies), ctypes.byref(m)), "apack_rotary_frequencies")
        else:
            frequencies = np.array(frequencies, np.float64)
            if frequencies.shape != (pairs,):
                raise ValueError(f"frequencies: {pairs} expected")
        self._frequencies = frequencies          # struct holds its address
        sec = [] if sections is None else [int(x) for x in sections]
        if len(sec) > 3:
            raise ValueError("sections: at most three axes")
        self._magnitude = float(m.value if magnitude is None else magnitude)
        self.struct = apack_rotary_spec(
            layout=APACK_ROTARY_PAIRS if interleaved else APACK_ROTARY_HALF, rotary_dim=int(rotary_dim),
            num_axes=max(1, len(sec)), section=(ctypes.c_int32 * 3)(*(sec + [0] * (3 - len(sec)))),
            magnitude=self._magnitude,
            freq_h=frequencies.ctypes.data_as(ctypes.POINTER(ctypes.c_double)))
        self._axes = self.struct.num_axes
        self._address = ctypes.addressof(self.struct)

    frequencies = property(lambda self: self._frequencies)
    rotary_dim = property(lambda self: self.struct.rotary_dim)
    magnitude = property(lambda self: self._magnitude)
    num_axes = property(lambda self: self._axes)

    def _positions(self, positions, n):
        """Checks int32 [n] or [axes, n] (expanded from one axis, where all share it); returns the stride between axes."""
        dims, stride = positions.shape, positions.stride()
        if str(positions.dtype) != "torch.int32" or not (
                dims == (self.num_axes, n) or (self.num_axes == 1 and dims == (n,))) or (stride[-1] != 1 and n > 1):
            raise ValueError(f"positions: int32 [{self.num_axes}, {n}], tokens contiguous, expected, not "
                             f"{positions.dtype} {tuple(dims)}")
        return stride[0] if self.num_axes > 1 else n


def apack_rotary(rotary, x, positions, out, transpose=False, stream=None):
    """Rotary positions of x [tokens, heads, D] into out (out is x: in place); transpose: the gradient."""
    if _cuda is None:
        stream = _on_device((x, positions, out), stream)
    else:
        dev = _cuda[0]()
        if x.get_device() != dev or positions.get_device() != dev or out.get_device() != dev:
            _on_device((x, positions, out), stream)
        stream = _cuda[1](dev) if stream is None else _stream(stream)
    dtype, shape, xs = x.dtype, x.shape, x.stride()
    code = _CODES.get(dtype)
    if code is None:
        code = _dtype_code(dtype)
    if len(shape) != 3 or xs[2] != 1 or xs[1] != shape[2]:
        xs = (_head_rows(x, "x"),)
    n, heads, dim = shape
    xs = xs[0] if n > 1 else heads * dim
    if out is x:
        outs = xs
    else:
        outs = out.stride()
        if out.dtype is not dtype or out.shape != shape or outs[2] != 1 or outs[1] != dim:
            outs = (_head_rows(out, "out", dtype, shape),)
        outs = outs[0] if n > 1 else heads * dim
    axes, axis = rotary._axes, positions.stride()
    if positions.dtype is _int32_type and positions.shape == ((axes, n) if axes > 1 else (n,)) and axis[-1] == 1:
        axis = axis[0] if axes > 1 else n
    else:
        axis = rotary._positions(positions, n)
    size = 4 if code == APACK_FP32 else 2
    status = _lib.apack_rotary(rotary._address, code, n, heads, dim, x.data_ptr(), size * xs, out.data_ptr(), size * outs,
                               positions.data_ptr(), axis, 1 if transpose else 0, stream)
    if status:
        raise ApackError(status, "apack_rotary")


def apack_rotary_append(rotary, cache, layer, q, k, v, q_out, positions, rows, seqs=None, ws=None, stream=None):
    """Rotates new tokens' queries into q_out and their keys into the pages of `layer`, with their values.
    rotary None: no rotation; q (and q_out) None: keys and values alone."""
    if _cuda is None:
        stream = _on_device((cache, k, v, rows, q, q_out, positions, seqs, ws), stream)
    else:
        dev = _cuda[0]()
        if (cache._device != dev or k.get_device() != dev or v.get_device() != dev or rows.get_device() != dev or
                (q is not None and q.get_device() != dev) or (q_out is not None and q_out.get_device() != dev) or
                (positions is not None and positions.get_device() != dev) or
                (seqs is not None and seqs.get_device() != dev) or (ws is not None and ws.get_device() != dev)):
            _on_device((cache, k, v, rows, q, q_out, positions, seqs, ws), stream)
        stream = _cuda[1](dev) if stream is None else _stream(stream)
    n = k.shape[0]
    dtype, dim = cache.dtype, cache.head_dim
    shape = (n, cache.num_kv_heads, dim)
    ks, vs = k.stride(), v.stride()
    if k.dtype is not dtype or k.shape != shape or ks[1] != dim or ks[2] != 1:
        ks = (_head_rows(k, "k", dtype, shape),)
    if v.dtype is not dtype or v.shape != shape or vs[1] != dim or vs[2] != 1:
        vs = (_head_rows(v, "v", dtype, shape),)
    ks, vs = (ks[0], vs[0]) if n > 1 else (shape[1] * dim, shape[1] * dim)
    q_at = q_out_at = spec = pos_at = None
    qs = qos = heads = axis = 0
    if (q is None) != (q_out is None):
        raise ValueError("q and q_out: both or neither expected")
    if q is not None:
        heads = q.shape[1]
        shape = (n, heads, dim)
        qs, qos = q.stride(), q_out.stride()
        if q.dtype is not dtype or q.shape != shape or qs[1] != dim or qs[2] != 1:
            qs = (_head_rows(q, "q", dtype, shape),)
        if q_out.dtype is not dtype or q_out.shape != shape or qos[1] != dim or qos[2] != 1:
            qos = (_head_rows(q_out, "q_out", dtype, shape),)
        qs, qos = (qs[0], qos[0]) if n > 1 else (heads * dim, heads * dim)
        q_at, q_out_at = q.data_ptr(), q_out.data_ptr()
    if rotary is not None:
        if positions is None:
            raise ValueError("positions: expected with a rotation")
        axes, axis = rotary._axes, positions.stride()
        if positions.dtype is _int32_type and positions.shape == ((axes, n) if axes > 1 else (n,)) and axis[-1] == 1:
            axis = axis[0] if axes > 1 else n
        else:
            axis = rotary._positions(positions, n)
        spec, pos_at = rotary._address, positions.data_ptr()
    if not (rows.dtype is _int32_type and rows.shape == (n,) and rows.is_contiguous()):
        _int32(rows, "rows", (n,))
    if seqs is not None and not (seqs.dtype is _int32_type and seqs.shape == (n,) and seqs.is_contiguous()):
        _int32(seqs, "seqs", (n,))
    status = _lib.apack_rotary_append(
        spec, cache._address, int(layer), n, q_at, 2 * qs, q_out_at, 2 * qos, heads, k.data_ptr(), 2 * ks, v.data_ptr(),
        2 * vs, pos_at, axis, rows.data_ptr(), None if seqs is None else seqs.data_ptr(),
        None if ws is None else ws.data_ptr(), stream)
    if status:
        raise ApackError(status, "apack_rotary_append")


def apack_paged_decode_workspace_size(cache, num_q_heads):
    n = ctypes.c_size_t(0)
    _check(_lib.apack_paged_decode_workspace_size(cache._address, int(num_q_heads), ctypes.byref(n)),
           "apack_paged_decode_workspace_size")
    return n.value


def apack_paged_decode_attention(cache, layer, seqlens, q, out, ws, scale=None, lse=None, stream=None):
    """Attention of one decode token per sequence over its pages; seqlens: int32 [num_seqs] on the device.
    q [num_seqs, Hq, D]; out: the same shape, contiguous, of q's type or float32; lse: float32 [num_seqs, Hq]."""
    if _cuda is None:
        stream = _on_device((cache, seqlens, q, out, ws, lse), stream)
    else:
        dev = _cuda[0]()
        if (cache._device != dev or seqlens.get_device() != dev or q.get_device() != dev or out.get_device() != dev or
                ws.get_device() != dev or (lse is not None and lse.get_device() != dev)):
            _on_device((cache, seqlens, q, out, ws, lse), stream)
        stream = _cuda[1](dev) if stream is None else _stream(stream)
    seqs, dim, dtype, qs = cache.num_seqs, cache.head_dim, cache.dtype, q.stride()
    heads = q.shape[1]
    shape = (seqs, heads, dim)
    if q.dtype is not dtype or q.shape != shape or qs[1] != dim or qs[2] != 1:
        qs = (_head_rows(q, "q", dtype, shape),)
    qs = qs[0] if seqs > 1 else heads * dim
    if not (seqlens.dtype is _int32_type and seqlens.shape == (seqs,) and seqlens.is_contiguous()):
        _int32(seqlens, "seqlens", (seqs,))
    if out.shape != shape or not out.is_contiguous():
        raise ValueError(f"out: contiguous {shape} expected")
    if lse is not None and (str(lse.dtype) != "torch.float32" or lse.shape != (seqs, heads) or not lse.is_contiguous()):
        raise ValueError(f"lse: contiguous float32 {shape[:2]} expected")
    code = _CODES.get(out.dtype)
    status = _lib.apack_paged_decode_attention(
        cache._address, int(layer), seqlens.data_ptr(), q.data_ptr(), 2 * qs, heads,
        cache._scale if scale is None else scale, out.data_ptr(), _dtype_code(out.dtype) if code is None else code,
        None if lse is None else lse.data_ptr(), ws.data_ptr(), ws.nbytes, stream)
    if status:
        raise ApackError(status, "apack_paged_decode_attention")


def apack_paged_compact(src, dst, cu_dst, n_out, keep_idx=None, cu_src=None, src_layer=0, dst_layer=0,
                        num_layers=None, ws=None, stream=None):
    """The kept rows of every sequence of pool src, in order, to the first rows of its pages in dst (src is dst:
    in place).  cu_dst, cu_src: int32 [num_seqs + 1] on the device; keep_idx: n_out entries at least (the call cannot
    see cu_dst); num_layers: all that both have by default."""
    stream = _on_device((src, dst, cu_dst, keep_idx, cu_src, ws), stream)
    _int32(cu_dst, "cu_dst", (dst.num_seqs + 1,))
    if cu_src is not None:
        _int32(cu_src, "cu_src", (src.num_seqs + 1,))
    if keep_idx is not None:
        _int32(keep_idx, "keep_idx")
        if keep_idx.numel() < n_out:
            raise ValueError(f"keep_idx: {n_out} entries expected, not {keep_idx.numel()}")
    if num_layers is None:
        num_layers = min(src.num_layers - src_layer, dst.num_layers - dst_layer)
    _check(_lib.apack_paged_compact(src._address, dst._address, int(src_layer), int(dst_layer), int(num_layers),
                                    _ptr(keep_idx), _ptr(cu_src), cu_dst.data_ptr(), int(n_out), _ptr(ws),
                                    stream), "apack_paged_compact")


def apack_copy_pages(cache, pairs, ws=None, stream=None):
    """Copies page pairs[i, 0] to page pairs[i, 1] in every layer; pairs: int32 [n, 2] on the device."""
    if _cuda is None:
        stream = _on_device((cache, pairs, ws), stream)
    else:
        dev = _cuda[0]()
        if cache._device != dev or pairs.get_device() != dev or (ws is not None and ws.get_device() != dev):
            _on_device((cache, pairs, ws), stream)
        stream = _cuda[1](dev) if stream is None else _stream(stream)
    n = pairs.shape[0]
    if not (pairs.dtype is _int32_type and pairs.shape == (n, 2) and pairs.is_contiguous()):
        _int32(pairs, "pairs", (n, 2))
    status = _lib.apack_copy_pages(cache._address, pairs.data_ptr(), n, None if ws is None else ws.data_ptr(), stream)
    if status:
        raise ApackError(status, "apack_copy_pages")


def apack_device_error(ws, stream=None, clear=True):
    code = ctypes.c_int32(0)
    _check(_lib.apack_device_error(_ptr(ws), _stream(stream), ctypes.byref(code), 1 if clear else 0),
           "apack_device_error")
    return code.value


def apack_launch_count():
    return int(_lib.apack_launch_count())


def library_path():
    return LIB_PATH
