"""ctypes binding of libvideomla.so (include/videomla.h), same names as the C ABI.

Argument marshalling only: every step of the cache append and of the
attention runs in the library's CUDA kernels. PyTorch supplies device memory
and streams. There is no fallback: if the library is missing or a call
fails, these functions raise.
"""

import ctypes
import os

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libvideomla.so")

MLA_OK = 0
MLA_ERR_ARG = -1
MLA_ERR_UNSUPPORTED = -2
MLA_ERR_RANGE = -3
MLA_ERR_CUDA = -4
MLA_ERR_TIMEOUT = -5
MLA_ERR_TOO_LARGE = -6
MLA_NOALLOC_SCRATCH_BYTES = 8 * 1024 * 1024

MLA_FLAG_NO_RMSNORM = 1
MLA_FLAG_SIMT = 2
MLA_FLAG_ROTATE_AT_USE = 4

MLA_ROPE_INTERLEAVED = 0
MLA_ROPE_HALF = 1
MLA_ROPE_SCALE_NONE = 0
MLA_ROPE_SCALE_LINEAR = 1
MLA_ROPE_SCALE_NTK = 2
MLA_ROPE_SCALE_YARN = 3
_DTYPES = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}  # MLA_DTYPE_*

# Every symbol include/videomla.h declares.
EXPORTS = ("mla_rope_table_bytes", "mla_rope_table_fill", "mla_config_check",
           "mla_cache_reset", "mla_cache_append", "mla_attention_forward",
           "mla_absorb_weights", "mla_query_workspace_bytes", "mla_query_prologue",
           "mla_query_prologue_noalloc", "mla_output_projection", "mla_dense_attention_forward",
           "mla_window_workspace_bytes", "mla_attention_window_forward", "mla_decompress_window",
           "mla_rope_scaled_table_fill", "mla_rope_apply", "mla_paged_check",
           "mla_pages_plan_bytes", "mla_pages_resize", "mla_pages_fork", "mla_pages_copy",
           "mla_pages_compact", "mla_paged_append", "mla_paged_workspace_bytes",
           "mla_paged_attention",
           "mla_selftest_bounded_wait", "mla_status_string", "mla_last_cuda_error", "mla_device_status",
           "mla_debug_rescale_count", "mla_version")


class mla_config(ctypes.Structure):
    _fields_ = [
        ("hidden", ctypes.c_int), ("heads", ctypes.c_int), ("head_dim", ctypes.c_int),
        ("d_c", ctypes.c_int), ("d_r", ctypes.c_int), ("d_q", ctypes.c_int),
        ("rope_pairs_t", ctypes.c_int), ("rope_pairs_h", ctypes.c_int),
        ("rope_pairs_w", ctypes.c_int),
        ("rope_dim_t", ctypes.c_int), ("rope_dim_h", ctypes.c_int), ("rope_dim_w", ctypes.c_int),
        ("rope_theta", ctypes.c_double), ("rope_table_len", ctypes.c_int),
        ("tokens_per_frame", ctypes.c_int), ("window_frames", ctypes.c_int),
        ("batch", ctypes.c_int), ("rms_eps", ctypes.c_float), ("flags", ctypes.c_uint),
        ("sink_frames", ctypes.c_int),
    ]


class mla_cache(ctypes.Structure):
    _fields_ = [
        ("c", ctypes.c_void_p), ("kr", ctypes.c_void_p), ("rope_table", ctypes.c_void_p),
        ("frames_written", ctypes.c_longlong), ("cfg", mla_config),
    ]


class mla_rope(ctypes.Structure):
    _fields_ = [
        ("table", ctypes.c_void_p), ("table_len", ctypes.c_int),
        ("pairs_t", ctypes.c_int), ("pairs_h", ctypes.c_int), ("pairs_w", ctypes.c_int),
        ("axes", ctypes.c_int), ("offset", ctypes.c_int), ("layout", ctypes.c_int),
    ]


class mla_paged_cache(ctypes.Structure):
    _fields_ = [
        ("c", ctypes.c_void_p), ("kr", ctypes.c_void_p), ("table", ctypes.c_void_p),
        ("lens", ctypes.c_void_p), ("refs", ctypes.c_void_p), ("plan", ctypes.c_void_p),
        ("layers", ctypes.c_int), ("pages", ctypes.c_int), ("page_tokens", ctypes.c_int),
        ("seqs", ctypes.c_int), ("max_pages", ctypes.c_int), ("d_c", ctypes.c_int),
        ("d_r", ctypes.c_int),
    ]


class MlaError(RuntimeError):
    def __init__(self, fn, code, lib):
        self.code = code
        msg = lib.mla_status_string(code).decode()
        if code == MLA_ERR_CUDA:
            msg += f" (cudaError {lib.mla_last_cuda_error()})"
        super().__init__(f"{fn} failed: {msg} [{code}]")


_lib = None


def load():
    """Load the in-tree library once; raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
    lib = ctypes.CDLL(LIB_PATH)
    P, VP, I, LL = ctypes.POINTER, ctypes.c_void_p, ctypes.c_int, ctypes.c_longlong
    lib.mla_rope_table_bytes.argtypes = [P(mla_config)]
    lib.mla_rope_table_bytes.restype = ctypes.c_ulonglong
    lib.mla_rope_table_fill.argtypes = [P(mla_config), P(ctypes.c_float)]
    lib.mla_config_check.argtypes = [P(mla_config)]
    lib.mla_cache_reset.argtypes = [P(mla_cache), VP]
    lib.mla_cache_append.argtypes = [P(mla_cache), VP, VP, VP, VP, VP, LL, I, VP]
    lib.mla_attention_forward.argtypes = [P(mla_cache), VP, VP, VP, I, VP, VP]
    lib.mla_status_string.argtypes = [I]
    lib.mla_status_string.restype = ctypes.c_char_p
    lib.mla_last_cuda_error.argtypes = []
    lib.mla_device_status.argtypes = [P(I), I]
    lib.mla_debug_rescale_count.argtypes = [P(ctypes.c_ulonglong), I]
    lib.mla_version.argtypes = []
    lib.mla_absorb_weights.argtypes = [P(mla_config), VP, VP, VP, VP, VP, VP, VP, VP, VP]
    lib.mla_query_workspace_bytes.argtypes = [P(mla_config), I]
    lib.mla_query_workspace_bytes.restype = ctypes.c_ulonglong
    lib.mla_query_prologue.argtypes = [P(mla_config), VP, VP, VP, I, VP, ctypes.c_ulonglong, VP,
                                       VP, VP]
    lib.mla_output_projection.argtypes = [P(mla_config), VP, VP, I, VP, VP]
    lib.mla_query_prologue_noalloc.argtypes = [P(mla_config), VP, VP, VP, I, VP, VP, VP]
    lib.mla_dense_attention_forward.argtypes = [P(mla_config), VP, VP, VP, I, I, I, VP, VP]
    lib.mla_decompress_window.argtypes = [P(mla_cache), VP, VP, VP, VP, VP]
    lib.mla_selftest_bounded_wait.argtypes = [ctypes.c_ulonglong, VP]
    lib.mla_window_workspace_bytes.argtypes = [P(mla_config), I]
    lib.mla_window_workspace_bytes.restype = ctypes.c_ulonglong
    lib.mla_attention_window_forward.argtypes = [P(mla_cache), VP, VP, VP, I, VP, VP,
                                                 ctypes.c_ulonglong, VP, VP]
    D = ctypes.c_double
    lib.mla_rope_scaled_table_fill.argtypes = [I, I, D, I, D, I, D, D, P(ctypes.c_float)]
    lib.mla_rope_apply.argtypes = [P(mla_rope), VP, VP, VP, I, LL, I, I, LL, LL, LL, LL, I, VP]
    lib.mla_paged_check.argtypes = [P(mla_paged_cache)]
    lib.mla_pages_plan_bytes.argtypes = [P(mla_paged_cache)]
    lib.mla_pages_plan_bytes.restype = ctypes.c_ulonglong
    lib.mla_pages_resize.argtypes = [P(mla_paged_cache), VP, VP]
    lib.mla_pages_fork.argtypes = [P(mla_paged_cache), VP, VP, I, VP]
    lib.mla_pages_copy.argtypes = [P(mla_paged_cache), VP, VP, I, VP]
    lib.mla_pages_compact.argtypes = [P(mla_paged_cache), VP, VP, VP]
    lib.mla_paged_append.argtypes = [P(mla_paged_cache), I, VP, VP, I, VP, VP, P(mla_rope), VP]
    lib.mla_paged_workspace_bytes.argtypes = [P(mla_paged_cache)]
    lib.mla_paged_workspace_bytes.restype = ctypes.c_ulonglong
    lib.mla_paged_attention.argtypes = [P(mla_paged_cache), I, VP, VP, I, I, VP, I, I, VP,
                                        ctypes.c_ulonglong, VP, VP]
    for name in ("mla_paged_attention", "mla_rope_scaled_table_fill", "mla_rope_apply", "mla_paged_check",
                 "mla_pages_resize", "mla_pages_fork", "mla_pages_copy", "mla_pages_compact",
                 "mla_paged_append"):
        getattr(lib, name).restype = I
    for name in ("mla_rope_table_fill", "mla_config_check", "mla_cache_reset", "mla_cache_append",
                 "mla_attention_forward", "mla_last_cuda_error", "mla_device_status",
                 "mla_version", "mla_absorb_weights", "mla_query_prologue",
                 "mla_query_prologue_noalloc", "mla_output_projection",
                 "mla_dense_attention_forward", "mla_attention_window_forward",
                 "mla_decompress_window", "mla_selftest_bounded_wait",
                 "mla_debug_rescale_count"):
        getattr(lib, name).restype = I
    _lib = lib
    return lib


def _check(fn, code):
    if code != MLA_OK:
        raise MlaError(fn, code, load())


def make_config(w, flags=0):
    """mla_config from a synth.Workload-like object (a workload with sink
    frames keeps k^R unrotated: the long-rollout window of App. D.4-D.5)."""
    sink = getattr(w, "sink_frames", 0)
    if sink:
        flags |= MLA_FLAG_ROTATE_AT_USE
    return mla_config(
        hidden=w.hidden, heads=w.heads, head_dim=w.head_dim, d_c=w.d_c, d_r=w.d_r, d_q=w.d_q,
        rope_pairs_t=w.rope_pairs[0], rope_pairs_h=w.rope_pairs[1], rope_pairs_w=w.rope_pairs[2],
        rope_dim_t=w.rope_axis_dims[0], rope_dim_h=w.rope_axis_dims[1],
        rope_dim_w=w.rope_axis_dims[2], rope_theta=w.rope_theta,
        rope_table_len=w.rope_table_len, tokens_per_frame=w.tokens_per_frame,
        window_frames=w.window_frames, batch=w.batch, rms_eps=w.rms_eps, flags=flags,
        sink_frames=sink)


def mla_config_check(cfg):
    return load().mla_config_check(ctypes.byref(cfg))


def mla_rope_table_fill(cfg):
    """The RoPE cos/sin table as a float32 NumPy array [L, d_r/2, 2]."""
    lib = load()
    nbytes = lib.mla_rope_table_bytes(ctypes.byref(cfg))
    if nbytes == 0:
        raise MlaError("mla_rope_table_bytes", MLA_ERR_ARG, lib)
    out = np.empty((cfg.rope_table_len, cfg.d_r // 2, 2), dtype=np.float32)
    _check("mla_rope_table_fill",
           lib.mla_rope_table_fill(ctypes.byref(cfg),
                                   out.ctypes.data_as(ctypes.POINTER(ctypes.c_float))))
    return out


def _stream_ptr(stream):
    if stream is None:
        # the handle of torch.cuda.current_stream() without the Stream object,
        # which costs as much as a small call's launch
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return ctypes.c_void_p(stream.cuda_stream)


def _dev(t, dtype, shape, name):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _ptr(t, dtype, shape, name):
    """_dev for calls that take microseconds: the address as an int."""
    if type(t) is torch.Tensor and t.is_cuda and t.dtype is dtype and t.shape == shape \
            and t.is_contiguous():
        return t.data_ptr()
    return _dev(t, dtype, shape, name)


class LatentCache:
    """Device buffers of one layer's sliding-window latent cache + the C struct.

    c  bf16 [B, W*T, d_c]; kr bf16 [B, W*T, d_r]; rope fp32 [L, d_r/2, 2].
    """

    def __init__(self, cfg, device="cuda"):
        self.cfg = cfg
        slots = cfg.tokens_per_frame * cfg.window_frames
        self.c = torch.zeros(cfg.batch, slots, cfg.d_c, dtype=torch.bfloat16, device=device)
        self.kr = torch.zeros(cfg.batch, slots, cfg.d_r, dtype=torch.bfloat16, device=device)
        self.rope = torch.from_numpy(mla_rope_table_fill(cfg)).to(device)
        self.struct = mla_cache(c=self.c.data_ptr(), kr=self.kr.data_ptr(),
                                rope_table=self.rope.data_ptr(), frames_written=0, cfg=cfg)

    @property
    def frames_written(self):
        return self.struct.frames_written

    @frames_written.setter
    def frames_written(self, v):
        self.struct.frames_written = int(v)

    @property
    def slots(self):
        return self.cfg.tokens_per_frame * self.cfg.window_frames

    def n_valid(self):
        held = min(self.frames_written, self.cfg.window_frames)
        return held * self.cfg.tokens_per_frame


def mla_cache_reset(cache, stream=None):
    _check("mla_cache_reset",
           load().mla_cache_reset(ctypes.byref(cache.struct), _stream_ptr(stream)))


def mla_cache_append(cache, x, w_dkv, gamma_kv, w_kr, pos, first_frame, n_frames, stream=None):
    cfg = cache.cfg
    n_tok = n_frames * cfg.tokens_per_frame
    bf = torch.bfloat16
    args = (
        _dev(x, bf, (cfg.batch, n_tok, cfg.hidden), "x"),
        _dev(w_dkv, bf, (cfg.d_c, cfg.hidden), "w_dkv"),
        None if gamma_kv is None else _dev(gamma_kv, bf, (cfg.d_c,), "gamma_kv"),
        _dev(w_kr, bf, (cfg.d_r, cfg.hidden), "w_kr"),
        None if pos is None and cfg.flags & MLA_FLAG_ROTATE_AT_USE
        else _dev(pos, torch.int32, (cfg.batch, n_tok, 3), "pos"),
    )
    _check("mla_cache_append",
           load().mla_cache_append(ctypes.byref(cache.struct), *args, int(first_frame),
                                   int(n_frames), _stream_ptr(stream)))


def mla_attention_forward(cache, q_c, q_r, q_pos, o_lat, stream=None):
    cfg = cache.cfg
    Nq = q_c.shape[1]
    bf = torch.bfloat16
    args = (
        _dev(q_c, bf, (cfg.batch, Nq, cfg.heads, cfg.d_c), "q_c"),
        _dev(q_r, bf, (cfg.batch, Nq, cfg.heads, cfg.d_r), "q_r"),
        _dev(q_pos, torch.int32, (cfg.batch, Nq, 3), "q_pos"),
    )
    out = _dev(o_lat, bf, (cfg.batch, Nq, cfg.heads, cfg.d_c), "o_lat")
    _check("mla_attention_forward",
           load().mla_attention_forward(ctypes.byref(cache.struct), *args, int(Nq), out,
                                        _stream_ptr(stream)))


def mla_window_workspace_bytes(cfg, Nq):
    return int(load().mla_window_workspace_bytes(ctypes.byref(cfg), int(Nq)))


def mla_attention_window_forward(cache, q_c, q_r, q_pos, frame_hw, workspace, o_lat, stream=None):
    """Attention over the assembled sink + FIFO window with window-relative
    RoPE (App. D.4, D.5); q_pos holds absolute frames, frame_hw [T, 2] the
    (h, w) of every token of a latent frame."""
    cfg = cache.cfg
    Nq = q_c.shape[1]
    bf = torch.bfloat16
    if not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.is_contiguous()):
        raise TypeError("workspace must be a contiguous CUDA tensor")
    _check("mla_attention_window_forward",
           load().mla_attention_window_forward(
               ctypes.byref(cache.struct),
               _dev(q_c, bf, (cfg.batch, Nq, cfg.heads, cfg.d_c), "q_c"),
               _dev(q_r, bf, (cfg.batch, Nq, cfg.heads, cfg.d_r), "q_r"),
               _dev(q_pos, torch.int32, (cfg.batch, Nq, 3), "q_pos"), int(Nq),
               _dev(frame_hw, torch.int32, (cfg.tokens_per_frame, 2), "frame_hw"),
               ctypes.c_void_p(workspace.data_ptr()),
               workspace.numel() * workspace.element_size(),
               _dev(o_lat, bf, (cfg.batch, Nq, cfg.heads, cfg.d_c), "o_lat"),
               _stream_ptr(stream)))


def mla_decompress_window(cache, w_uk, w_uv, k, v, stream=None):
    """Expand the latent cache into per-head keys [W_up^K c | k] and values
    W_up^V c, both [B, H, W*T, head_dim] (the decompress-then-dense form)."""
    cfg = cache.cfg
    H, dh, dr, dc = cfg.heads, cfg.head_dim, cfg.d_r, cfg.d_c
    shape = (cfg.batch, H, cache.slots, dh)
    bf = torch.bfloat16
    _check("mla_decompress_window",
           load().mla_decompress_window(
               ctypes.byref(cache.struct), _dev(w_uk, bf, (H, dh - dr, dc), "w_uk"),
               _dev(w_uv, bf, (H, dh, dc), "w_uv"), _dev(k, bf, shape, "k"),
               _dev(v, bf, shape, "v"), _stream_ptr(stream)))


def absorbed_weight_shapes(cfg):
    """Shapes of (w_qcat, w_b) that mla_absorb_weights writes."""
    return ((cfg.heads * (cfg.d_c + cfg.d_r), cfg.d_q), (cfg.hidden, cfg.heads * cfg.d_c))


def mla_absorb_weights(cfg, w_uq, w_uk, w_qr, gamma_q, w_uv, w_o, stream=None):
    """Absorbed query and output weights (App. E) as new bf16 CUDA tensors."""
    H, dc, dr, dq, d, dh = cfg.heads, cfg.d_c, cfg.d_r, cfg.d_q, cfg.hidden, cfg.head_dim
    dn = dh - dr
    bf = torch.bfloat16
    args = (
        _dev(w_uq, bf, (H, dn, dq), "w_uq"), _dev(w_uk, bf, (H, dn, dc), "w_uk"),
        _dev(w_qr, bf, (H, dr, dq), "w_qr"),
        None if gamma_q is None else _dev(gamma_q, bf, (dq,), "gamma_q"),
        _dev(w_uv, bf, (H, dh, dc), "w_uv"), _dev(w_o, bf, (d, H * dh), "w_o"),
    )
    sq, sb = absorbed_weight_shapes(cfg)
    w_qcat = torch.empty(sq, dtype=bf, device=w_uq.device)
    w_b = torch.empty(sb, dtype=bf, device=w_uq.device)
    _check("mla_absorb_weights",
           load().mla_absorb_weights(ctypes.byref(cfg), *args, ctypes.c_void_p(w_qcat.data_ptr()),
                                     ctypes.c_void_p(w_b.data_ptr()), _stream_ptr(stream)))
    return w_qcat, w_b


def mla_query_workspace_bytes(cfg, Nq):
    return int(load().mla_query_workspace_bytes(ctypes.byref(cfg), int(Nq)))


def mla_query_prologue(cfg, x, w_dq, w_qcat, workspace, q_c, q_r, stream=None):
    Nq = x.shape[1]
    bf = torch.bfloat16
    H, dc, dr, dq, d = cfg.heads, cfg.d_c, cfg.d_r, cfg.d_q, cfg.hidden
    if not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.is_contiguous()):
        raise TypeError("workspace must be a contiguous CUDA tensor")
    _check("mla_query_prologue",
           load().mla_query_prologue(
               ctypes.byref(cfg), _dev(x, bf, (cfg.batch, Nq, d), "x"),
               _dev(w_dq, bf, (dq, d), "w_dq"), _dev(w_qcat, bf, (H * (dc + dr), dq), "w_qcat"),
               int(Nq), ctypes.c_void_p(workspace.data_ptr()),
               workspace.numel() * workspace.element_size(),
               _dev(q_c, bf, (cfg.batch, Nq, H, dc), "q_c"),
               _dev(q_r, bf, (cfg.batch, Nq, H, dr), "q_r"), _stream_ptr(stream)))


def mla_query_prologue_noalloc(cfg, x, w_dq, w_qcat, q_c, q_r, stream=None):
    """The query prologue for callers that cannot allocate device memory: the
    intermediate buffer is the library's fixed scratch (see the C header for
    its size limit and the rule that overlapping calls race on it)."""
    Nq = x.shape[1]
    bf = torch.bfloat16
    H, dc, dr, dq, d = cfg.heads, cfg.d_c, cfg.d_r, cfg.d_q, cfg.hidden
    _check("mla_query_prologue_noalloc",
           load().mla_query_prologue_noalloc(
               ctypes.byref(cfg), _dev(x, bf, (cfg.batch, Nq, d), "x"),
               _dev(w_dq, bf, (dq, d), "w_dq"), _dev(w_qcat, bf, (H * (dc + dr), dq), "w_qcat"),
               int(Nq), _dev(q_c, bf, (cfg.batch, Nq, H, dc), "q_c"),
               _dev(q_r, bf, (cfg.batch, Nq, H, dr), "q_r"), _stream_ptr(stream)))


def mla_output_projection(cfg, o_lat, w_b, y, stream=None):
    Nq = o_lat.shape[1]
    bf = torch.bfloat16
    _check("mla_output_projection",
           load().mla_output_projection(
               ctypes.byref(cfg), _dev(o_lat, bf, (cfg.batch, Nq, cfg.heads, cfg.d_c), "o_lat"),
               _dev(w_b, bf, (cfg.hidden, cfg.heads * cfg.d_c), "w_b"), int(Nq),
               _dev(y, bf, (cfg.batch, Nq, cfg.hidden), "y"), _stream_ptr(stream)))


def mla_dense_attention_forward(cfg, q, k, v, n_valid, o, stream=None):
    """Dense per-head baseline: q [B, Nq, H, d_h], k/v [B, H, slots, d_h]."""
    B, Nq, H, dh = cfg.batch, q.shape[1], cfg.heads, cfg.head_dim
    slots = k.shape[2]
    bf = torch.bfloat16
    _check("mla_dense_attention_forward",
           load().mla_dense_attention_forward(
               ctypes.byref(cfg), _dev(q, bf, (B, Nq, H, dh), "q"),
               _dev(k, bf, (B, H, slots, dh), "k"), _dev(v, bf, (B, H, slots, dh), "v"),
               int(slots), int(n_valid), int(Nq), _dev(o, bf, (B, Nq, H, dh), "o"),
               _stream_ptr(stream)))


def mla_rope_scaled_table_fill(rot_dim, table_len, theta=10000.0, scaling=MLA_ROPE_SCALE_NONE,
                               factor=1.0, native_len=0, beta_fast=32.0, beta_slow=1.0):
    """cos/sin of one coordinate, frequencies scaled for a long context, as a
    float32 NumPy array [table_len, rot_dim/2, 2]."""
    if rot_dim < 2 or table_len < 1:
        raise MlaError("mla_rope_scaled_table_fill", MLA_ERR_ARG, load())
    out = np.empty((table_len, rot_dim // 2, 2), dtype=np.float32)
    _check("mla_rope_scaled_table_fill",
           load().mla_rope_scaled_table_fill(
               int(rot_dim), int(table_len), float(theta), int(scaling), float(factor),
               int(native_len), float(beta_fast), float(beta_slow),
               out.ctypes.data_as(ctypes.POINTER(ctypes.c_float))))
    return out


class Rope:
    """A rotation: its table (float32 CUDA tensor [len, pairs, 2]) + the C struct.

    pairs = (t, h, w) complex pairs per coordinate. (m, 0, 0) turns all pairs
    with one coordinate, pos [tokens, 1], unless axes=3 says that tokens carry
    three; offset is the first rotated channel of a head, half the layout that
    pairs channel i with i + m instead of 2i with 2i + 1.
    """

    def __init__(self, table, pairs, offset=0, half=False, axes=None):
        pairs = tuple(int(v) for v in pairs)
        if len(pairs) != 3:
            raise ValueError("pairs must be (t, h, w)")
        self.table = table
        self.pairs = pairs
        self.axes = (3 if pairs[1] or pairs[2] else 1) if axes is None else int(axes)
        _dev(table, torch.float32, (table.shape[0], sum(pairs), 2), "table")
        self.struct = mla_rope(table=table.data_ptr(), table_len=table.shape[0],
                               pairs_t=pairs[0], pairs_h=pairs[1], pairs_w=pairs[2],
                               axes=self.axes, offset=int(offset),
                               layout=MLA_ROPE_HALF if half else MLA_ROPE_INTERLEAVED)
        self.ref = ctypes.byref(self.struct)


def mla_rope_apply(rope, x, pos, y, inverse=False, stream=None):
    """Rotate part of every head of x [tokens, heads, head_dim] into y (which
    may be x); bf16, fp16 or fp32, channels contiguous, other strides free."""
    for t, name in ((x, "x"), (y, "y")):
        if not isinstance(t, torch.Tensor) or not t.is_cuda:
            raise TypeError(f"{name} must be a CUDA tensor")
    shape, dtype = x.shape, _DTYPES.get(x.dtype)
    if dtype is None or y.dtype is not x.dtype:
        raise TypeError(f"x and y must both be bfloat16, float16 or float32, got {x.dtype}, {y.dtype}")
    if y.shape != shape:
        raise ValueError(f"y must have shape {tuple(shape)}, got {tuple(y.shape)}")
    if len(shape) != 3 or shape[2] < 1:
        raise ValueError("x and y must be [tokens, heads, head_dim]")
    tokens, heads, dim = shape
    xt, xh, xc = x.stride()
    yt, yh, yc = y.stride()
    if dim > 1 and (xc != 1 or yc != 1):
        raise ValueError("x and y must have contiguous channels")
    _check("mla_rope_apply",
           load().mla_rope_apply(
               rope.ref, x.data_ptr(), _ptr(pos, torch.int32, (tokens, rope.axes), "pos"),
               y.data_ptr(), dtype, tokens, heads, dim, xt, xh, yt, yh, 1 if inverse else 0,
               _stream_ptr(stream)))


class PagedCache:
    """A latent cache in pages over the caller's CUDA tensors + the C struct.

    c bf16 [layers, pages, page_tokens, d_c]; kr bf16 [..., d_r]; table int32
    [seqs, max_pages]; lens int32 [seqs]; refs int32 [pages]. PagedCache.empty()
    allocates them for a pool without streams.
    """

    def __init__(self, c, kr, table, lens, refs):
        if c.dim() != 4 or kr.dim() != 4 or table.dim() != 2:
            raise ValueError("c and kr must be [layers, pages, page_tokens, width], table "
                             "[seqs, max_pages]")
        layers, pages, tokens, d_c = c.shape
        seqs, max_pages = table.shape
        bf, i32 = torch.bfloat16, torch.int32
        self.c, self.kr, self.table, self.lens, self.refs = c, kr, table, lens, refs
        self.seqs, self.d_c, self.d_r = seqs, d_c, kr.shape[3]
        self.struct = mla_paged_cache(
            c=_dev(c, bf, c.shape, "c"),
            kr=_dev(kr, bf, (layers, pages, tokens, kr.shape[3]), "kr"),
            table=_dev(table, i32, table.shape, "table"), lens=_dev(lens, i32, (seqs,), "lens"),
            refs=_dev(refs, i32, (pages,), "refs"), layers=layers, pages=pages,
            page_tokens=tokens, seqs=seqs, max_pages=max_pages, d_c=d_c, d_r=kr.shape[3])
        self.ref = ctypes.byref(self.struct)
        nbytes = load().mla_pages_plan_bytes(self.ref)
        if nbytes == 0:
            raise MlaError("mla_pages_plan_bytes", MLA_ERR_ARG, load())
        self.plan = torch.empty(nbytes // 4, dtype=i32, device=c.device)
        self.struct.plan = self.plan.data_ptr()

    @classmethod
    def empty(cls, layers, pages, page_tokens, seqs, max_pages, d_c, d_r, device="cuda"):
        bf, i32 = torch.bfloat16, torch.int32
        return cls(torch.zeros(layers, pages, page_tokens, d_c, dtype=bf, device=device),
                   torch.zeros(layers, pages, page_tokens, d_r, dtype=bf, device=device),
                   torch.full((seqs, max_pages), -1, dtype=i32, device=device),
                   torch.zeros(seqs, dtype=i32, device=device),
                   torch.zeros(pages, dtype=i32, device=device))


def mla_pages_resize(cache, new_lens, stream=None):
    """Give streams new lengths (int32 [seqs], -1: leave it): pages are given
    back or added, a shared last page that grows is copied first."""
    _check("mla_pages_resize",
           load().mla_pages_resize(cache.ref,
                                   _ptr(new_lens, torch.int32, (cache.seqs,), "new_lens"),
                                   _stream_ptr(stream)))


def _pairs_of(src, dst):
    n = src.shape[0] if isinstance(src, torch.Tensor) and src.dim() == 1 else 0
    return _ptr(src, torch.int32, (n,), "src"), _ptr(dst, torch.int32, (n,), "dst"), n


def mla_pages_fork(cache, src, dst, stream=None):
    """Branch stream src[i] as the empty stream dst[i]; all pages are shared."""
    _check("mla_pages_fork",
           load().mla_pages_fork(cache.ref, *_pairs_of(src, dst), _stream_ptr(stream)))


def mla_pages_copy(cache, src, dst, stream=None):
    """Copy page src[i] to page dst[i] in every layer."""
    _check("mla_pages_copy",
           load().mla_pages_copy(cache.ref, *_pairs_of(src, dst), _stream_ptr(stream)))


def mla_pages_compact(cache, new_table, new_refs, stream=None):
    """Pack the pool's pages in use to its front; the metadata afterwards goes
    to new_table and new_refs (the cache's own, or buffers that replace them)."""
    i32 = torch.int32
    _check("mla_pages_compact",
           load().mla_pages_compact(cache.ref,
                                    _ptr(new_table, i32, cache.table.shape, "new_table"),
                                    _ptr(new_refs, i32, cache.refs.shape, "new_refs"),
                                    _stream_ptr(stream)))


def mla_paged_append(cache, layer, c_new, kr_new, q_start, pos, rope, stream=None):
    """Write new tokens, the streams' newest, into their pages of one layer:
    c_new [total, d_c] as is, kr_new [total, d_r] rotated at pos."""
    bf, i32 = torch.bfloat16, torch.int32
    total = c_new.shape[0] if isinstance(c_new, torch.Tensor) and c_new.dim() == 2 else 0
    _check("mla_paged_append",
           load().mla_paged_append(
               cache.ref, layer, _ptr(c_new, bf, (total, cache.d_c), "c_new"),
               _ptr(kr_new, bf, (total, cache.d_r), "kr_new"), total,
               _ptr(q_start, i32, (cache.seqs + 1,), "q_start"),
               _ptr(pos, i32, (total, rope.axes), "pos"), rope.ref, _stream_ptr(stream)))


def mla_paged_workspace_bytes(cache):
    return int(load().mla_paged_workspace_bytes(cache.ref))


def mla_paged_attention(cache, layer, q_c, q_r, q_start, head_dim, causal_block, workspace, o,
                        stream=None):
    """Attention of the streams' newest tokens (q_c [total, heads, d_c], q_r
    [total, heads, d_r] rotated; rows of stream s from q_start[s]) over the
    pages of one layer. causal_block 0: every held token is seen; b: those
    before the end of the token's own block of b."""
    bf = torch.bfloat16
    if not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.is_contiguous()):
        raise TypeError("workspace must be a contiguous CUDA tensor")
    total, heads, _ = q_c.shape
    _check("mla_paged_attention",
           load().mla_paged_attention(
               cache.ref, layer, _ptr(q_c, bf, (total, heads, cache.d_c), "q_c"),
               _ptr(q_r, bf, (total, heads, cache.d_r), "q_r"), total, heads,
               _ptr(q_start, torch.int32, (cache.seqs + 1,), "q_start"), head_dim,
               causal_block, workspace.data_ptr(), workspace.nbytes,
               _ptr(o, bf, (total, heads, cache.d_c), "o"), _stream_ptr(stream)))


def mla_selftest_bounded_wait(limit_ns, stream=None):
    """Make one bounded device wait run out (nothing arrives on its barrier)."""
    _check("mla_selftest_bounded_wait",
           load().mla_selftest_bounded_wait(int(limit_ns), _stream_ptr(stream)))


def mla_device_status(clear=True):
    st = ctypes.c_int(0)
    _check("mla_device_status", load().mla_device_status(ctypes.byref(st), int(bool(clear))))
    return st.value


def mla_debug_rescale_count(clear=True):
    """Rows whose online softmax rescaled its output (debug build only; a
    release build raises MlaError with MLA_ERR_UNSUPPORTED)."""
    n = ctypes.c_ulonglong(0)
    _check("mla_debug_rescale_count",
           load().mla_debug_rescale_count(ctypes.byref(n), int(bool(clear))))
    return n.value
