"""ctypes binding of the C-ABI in ``include/longlive.h``: argument marshalling only.

Every step of the hot path runs in the HIP library.  There is no fallback: if the
library is missing or a call fails, an exception is raised.  torch is used for
device memory and streams only.
"""
from __future__ import annotations

import ctypes as C
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "liblonglive.so")
_lib = None

LL_OK, LL_ERR_INVALID_ARG, LL_ERR_STATE, LL_ERR_BUFFER_TOO_SMALL, LL_ERR_UNSUPPORTED, LL_ERR_HIP = range(6)
STATUS_NAMES = {0: "LL_OK", 1: "LL_ERR_INVALID_ARG", 2: "LL_ERR_STATE", 3: "LL_ERR_BUFFER_TOO_SMALL",
                4: "LL_ERR_UNSUPPORTED", 5: "LL_ERR_HIP"}

# name -> (restype, argtypes); mirrors include/longlive.h
_vp, _i, _i64, _sz = C.c_void_p, C.c_int, C.c_int64, C.c_size_t
SIGNATURES = {
    "ll_cache_bytes": (_sz, [_i] * 7),
    "ll_cache_create": (_i, [_i] * 9 + [C.c_float, _vp, _sz, C.POINTER(_vp)]),
    "ll_cache_bytes_fp8": (_sz, [_i] * 7),
    "ll_cache_create_fp8": (_i, [_i] * 9 + [C.c_float, _i, _i, _vp, _sz, C.POINTER(_vp)]),
    "ll_cache_destroy": (_i, [_vp]),
    "ll_cache_reset": (_i, [_vp, _i]),
    "ll_chunk_append": (_i, [_vp, _i, _i64, _i, _vp, _vp, _vp, _vp, _vp]),
    "ll_sink_window_attn": (_i, [_vp, _i, _vp, _vp, _vp]),
    "ll_sink_window_attn_unrotated": (_i, [_vp, _i, _vp, _vp, _vp]),
    "ll_recache_prefill": (_i, [_vp, _i, _i, _i64, _i, _vp, _vp, _vp, _vp, _vp]),
    "ll_recache_prefill_static": (_i, [_vp, _i, _i, _i64, _i, _vp, _vp, _vp, _vp, _vp]),
    "ll_cache_live_frames": (_i, [_vp, _i, C.POINTER(_i64), _i, C.POINTER(_i)]),
    "ll_cache_slot_of_frame": (_i, [_vp, _i, _i64, C.POINTER(_i64)]),
    "ll_cache_live_ranges": (_i, [_vp, _i, C.POINTER(_i64), _i, C.POINTER(_i)]),
    "ll_cache_read_frame": (_i, [_vp, _i, _i64, _vp, _vp, _vp]),
    "ll_cache_set_sink_relative": (_i, [_vp, _i]),
    "ll_prompt_bytes": (_sz, [_i] * 4),
    "ll_prompt_create": (_i, [_i] * 4 + [_vp, _sz, C.POINTER(_vp)]),
    "ll_prompt_destroy": (_i, [_vp]),
    "ll_prompt_recache": (_i, [_vp, _i, _vp, _vp, _i, _vp]),
    "ll_prompt_tokens": (_i, [_vp, _i, C.POINTER(_i)]),
    "ll_cross_attn": (_i, [_vp, _i, _vp, _i, _vp, _vp]),
    "ll_cross_attn_out": (_i, [_vp, _i, _vp, _i, _vp, _vp, _vp, _vp]),
    "ll_out_proj_pack_weight": (_i, [_i, _i, _vp, _vp, _vp]),
    "ll_cross_attn_out_workspace_bytes": (C.c_size_t, [_i, _i, _i]),
    "ll_clip_bytes": (_sz, [_i] * 7),
    "ll_clip_create": (_i, [_i] * 9 + [C.c_float, _vp, _sz, C.POINTER(_vp)]),
    "ll_clip_destroy": (_i, [_vp]),
    "ll_clip_forward": (_i, [_vp, _i64, _i, _i, _vp, _vp, _vp, _vp, _vp]),
    "ll_clip_backward": (_i, [_vp, _vp, _vp, _vp, _vp, _vp]),
    "ll_clip_chunk_key_ranges": (_i, [_vp, _i, C.POINTER(_i64), _i, C.POINTER(_i)]),
    "ll_paged_bytes": (_sz, [_i] * 6),
    "ll_paged_create": (_i, [_i] * 11 + [C.c_float, _vp, _sz, C.POINTER(_vp)]),
    "ll_paged_destroy": (_i, [_vp]),
    "ll_paged_append": (_i, [_vp, _i, _i, _i, _vp, _vp, _vp, _i, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64, _vp]),
    "ll_paged_attn_workspace_bytes": (_sz, [_vp, _i, _i, _i64, _i, _i]),
    "ll_paged_attn": (_i, [_vp, _i, _i, _i, _i, _i64, _vp, _vp, _vp, _i, _i64, _i, _i, _vp, _i64, _vp, _i64, _vp, _sz, _vp]),
    "ll_linear_packed_bytes": (_sz, [_i, _i]),
    "ll_linear_pack_weight": (_i, [_i, _i, _vp, _i64, _vp, _vp]),
    "ll_linear": (_i, [_i, _i, _i, _vp, _i64, _vp, _vp, _i, _vp, _i64, _vp, _i64, _vp]),
    "ll_set_attn_variant": (_i, [_i]),
    "ll_attn_variant_name": (C.c_char_p, [_i]),
    "ll_attn_key_groups": (_i, [_i] * 3 + [C.POINTER(_i)] * 3),
    "ll_attn_split": (_i, [_i] * 5 + [C.POINTER(_i)] * 2),
    "ll_attn_key_groups_fp8": (_i, [_i] * 3 + [C.POINTER(_i)] * 3),
    "ll_attn_clip_tail": (_i, [_i] * 3 + [C.POINTER(_i)] * 4),
    "ll_hold_split_slots": (_i, [_i] * 3),
    "ll_split_slots_taken": (_i, [C.POINTER(_i)]),
    "ll_probe_mfma_rate": (_i, [C.c_void_p, C.c_size_t, _i, _i, _i, C.POINTER(C.c_double), C.POINTER(C.c_double), C.c_void_p]),
    "ll_probe_mfma_mix": (_i, [C.c_void_p, C.c_size_t, _i, _i, _i, _i, _i, C.POINTER(C.c_double), C.POINTER(C.c_double), C.c_void_p]),
    "ll_status_string": (C.c_char_p, [_i]),
    "ll_last_error": (C.c_char_p, []),
}


class LongLiveError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


def lib() -> C.CDLL:
    """Load liblonglive.so (built by ``paper_2509_22622_amd.build``); raise if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not built: run `python -m paper_2509_22622_amd.build`")
        # torch first: it ships its own copy of the HIP runtime, and the library must bind to the copy that owns
        # the process's device memory and streams.  Loaded the other way round, the process holds two runtimes and
        # the library's own one finds no device.
        import torch  # noqa: F401
        L = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(status: int) -> None:
    if status != LL_OK:
        raise LongLiveError(status, lib().ll_last_error().decode())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def cache_bytes(layers, heads, head_dim, tokens_per_frame, sink_frames, window_frames, chunk_frames, kv_format="bf16") -> int:
    fn = lib().ll_cache_bytes_fp8 if kv_format == "fp8_e4m3" else lib().ll_cache_bytes
    return fn(layers, heads, head_dim, tokens_per_frame, sink_frames, window_frames, chunk_frames)


def set_attn_variant(variant: int) -> None:
    _check(lib().ll_set_attn_variant(variant))


def attn_key_groups(head_dim, heads, chunks) -> int:
    """Key groups the default bf16 kernels take for a launch of ``chunks``, (query rows, blocks of 32 keys) each."""
    rows, kblocks = ((C.c_int * len(chunks))(*x) for x in zip(*chunks))
    groups = C.c_int()
    _check(lib().ll_attn_key_groups(head_dim, heads, len(chunks), rows, kblocks, C.byref(groups)))
    return groups.value


def attn_split(head_dim, heads, rows, kblocks, kv_format="bf16"):
    """(groups, splits) of a streamed chunk with ``kblocks`` blocks of 32 keys (8-bit cache: 64) in a full window."""
    groups, splits = C.c_int(), C.c_int()
    _check(lib().ll_attn_split(head_dim, int(kv_format == "fp8_e4m3"), heads, rows, kblocks, C.byref(groups), C.byref(splits)))
    return groups.value, splits.value


def attn_key_groups_fp8(head_dim, heads, chunks) -> int:
    """4 where a re-prefill launch of an 8-bit cache deals its tiles' keys to groups of waves, else 1; ``chunks``: (query rows,
    blocks of 64 keys) each, all of which would split when streamed."""
    rows, kblocks = ((C.c_int * len(chunks))(*x) for x in zip(*chunks))
    groups = C.c_int()
    _check(lib().ll_attn_key_groups_fp8(head_dim, heads, len(chunks), rows, kblocks, C.byref(groups)))
    return groups.value


def attn_clip_tail(head_dim, heads, chunks):
    """(tiles per head, splits) of the last round that a clip's forward pass launches by itself; ``chunks``: (query rows, blocks of
    32 keys) each, the latest first."""
    rows, kblocks = ((C.c_int * len(chunks))(*x) for x in zip(*chunks))
    tiles, splits = C.c_int(), C.c_int()
    _check(lib().ll_attn_clip_tail(head_dim, heads, len(chunks), rows, kblocks, C.byref(tiles), C.byref(splits)))
    return tiles.value, splits.value


def hold_split_slots(first: int, n: int, hold: bool) -> None:
    """Take slots for partial results out of use, or give them back (a test instrument; synchronises)."""
    _check(lib().ll_hold_split_slots(first, n, int(hold)))


def split_slots_taken() -> int:
    """Places of the pool of partial results that are taken while no call is at work (a test instrument; synchronises)."""
    taken = C.c_int()
    _check(lib().ll_split_slots_taken(C.byref(taken)))
    return taken.value


def probe_mfma_rate(workgroups: int = 256, iters: int = 20000, random_operands: bool = True):
    """(TFLOP/s, core clock in GHz) of a pure 32x32x16 bf16 MFMA stream on the current device."""
    import torch
    scratch = torch.empty(workgroups * 2048 + 16, dtype=torch.uint8, device="cuda")
    tflops, ghz = C.c_double(), C.c_double()
    _check(lib().ll_probe_mfma_rate(C.c_void_p(scratch.data_ptr()), scratch.numel(), workgroups, iters,
                                    int(random_operands), C.byref(tflops), C.byref(ghz), _stream()))
    return tflops.value, ghz.value


PROBE_COMPANIONS = {0: "none", 1: "v_add_f32", 2: "v_exp_f32", 3: "v_cvt_pk_bf16_f32", 4: "v_dot2c_f32_bf16",
                    5: "v_max3_f32", 6: "ds_read_b128", 7: "16x16x32 MFMAs, no companion"}
PROBE_FP8_KINDS = {8: "fp8 32x32x64 MFMAs alone", 9: "+ the 8-bit kernel's vector and LDS work per MFMA",
                   10: "+ its vector work only (4 exp2, 4 add, 2 cvt, 2 max3)", 11: "+ its LDS reads only (2 x 16 B)"}


def probe_mfma_mix(companion: int, per_mfma: int = 1, workgroups: int = 256, iters: int = 20000, random_operands: bool = True):
    """(MFMA TFLOP/s, core clock in GHz) with `per_mfma` companion instructions behind every MFMA (see the header)."""
    import torch
    scratch = torch.empty(workgroups * 2048 + 16, dtype=torch.uint8, device="cuda")
    tflops, ghz = C.c_double(), C.c_double()
    _check(lib().ll_probe_mfma_mix(C.c_void_p(scratch.data_ptr()), scratch.numel(), workgroups, iters, int(random_operands),
                                   companion, per_mfma, C.byref(tflops), C.byref(ghz), _stream()))
    return tflops.value, ghz.value


def attn_variant_names() -> dict:
    out, v = {}, 1
    while True:
        n = lib().ll_attn_variant_name(v)
        if n is None:
            return out
        out[v] = n.decode()
        v += 1


class Cache:
    """Handle on ``layers`` rolling KV caches.  ``device=None`` makes an index-only handle.

    ``kv_format="fp8_e4m3"`` makes the 8-bit cache (``ll_cache_create_fp8``): q_out of ``chunk_append`` and the
    tensors of ``read_frame`` are then uint8 (E4M3 codes) of the same shape; everything else stays bfloat16.
    """

    def __init__(self, layers, heads, head_dim, grid_h, grid_w, chunk_frames, sink_frames, window_frames,
                 rope_theta=10000.0, device="cuda", kv_format="bf16", k_exp=0, v_exp=0):
        if kv_format not in ("bf16", "fp8_e4m3"):
            raise ValueError(f"kv_format {kv_format!r}")
        self.kv_format = kv_format
        self.layers, self.heads, self.head_dim = layers, heads, head_dim
        self.grid_h, self.grid_w = grid_h, grid_w
        self.P = grid_h * grid_w
        self.C, self.S, self.W = chunk_frames, sink_frames, window_frames
        self._h = C.c_void_p()
        self.buffer = None
        nbytes = cache_bytes(layers, heads, head_dim, self.P, sink_frames, window_frames, chunk_frames, kv_format)
        if device is not None:
            import torch
            if nbytes == 0:
                raise LongLiveError(1, "invalid shape")
            self.buffer = torch.empty(nbytes, dtype=torch.uint8, device=device)
            ptr, size = C.c_void_p(self.buffer.data_ptr()), nbytes
        else:
            ptr, size = None, 0
        if kv_format == "fp8_e4m3":
            _check(lib().ll_cache_create_fp8(layers, heads, head_dim, self.P, sink_frames, window_frames, chunk_frames,
                                             grid_h, grid_w, rope_theta, k_exp, v_exp, ptr, size, C.byref(self._h)))
        else:
            _check(lib().ll_cache_create(layers, heads, head_dim, self.P, sink_frames, window_frames, chunk_frames,
                                         grid_h, grid_w, rope_theta, ptr, size, C.byref(self._h)))

    def close(self):
        if self._h:
            lib().ll_cache_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_sink_relative(self, on: bool) -> None:
        """Sink at a fixed rotary distance from the window (see ``ll_cache_set_sink_relative``)."""
        _check(lib().ll_cache_set_sink_relative(self._h, int(bool(on))))

    def reset(self, layer=-1):
        _check(lib().ll_cache_reset(self._h, layer))

    def chunk_append(self, layer, frame_start, n_frames, q=None, k=None, v=None, q_out=None):
        """q and q_out None with k, v given: keys and values only (the queries go to sink_window_attn_unrotated)."""
        stream = _stream() if k is not None else None
        _check(lib().ll_chunk_append(self._h, layer, frame_start, n_frames, _ptr(q), _ptr(k), _ptr(v), _ptr(q_out), stream))

    def sink_window_attn(self, layer, q_roped, out):
        _check(lib().ll_sink_window_attn(self._h, layer, _ptr(q_roped), _ptr(out), _stream()))

    def sink_window_attn_unrotated(self, layer, q, out):
        """The same attention from the chunk's unrotated, unscaled queries (the kernel turns them on load)."""
        _check(lib().ll_sink_window_attn_unrotated(self._h, layer, _ptr(q), _ptr(out), _stream()))

    def recache_prefill(self, layer, include_sink, win_start, n_win, q=None, k=None, v=None, out=None):
        stream = _stream() if q is not None else None
        _check(lib().ll_recache_prefill(self._h, layer, int(include_sink), win_start, n_win, _ptr(q), _ptr(k), _ptr(v),
                                        _ptr(out), stream))

    def recache_prefill_static(self, layer, include_sink, win_start, n_win, q=None, k=None, v=None, out=None):
        stream = _stream() if q is not None else None
        _check(lib().ll_recache_prefill_static(self._h, layer, int(include_sink), win_start, n_win, _ptr(q), _ptr(k),
                                               _ptr(v), _ptr(out), stream))

    def live_frames(self, layer):
        cap = self.S + self.W + self.C + 1
        buf, n = (C.c_int64 * cap)(), C.c_int()
        _check(lib().ll_cache_live_frames(self._h, layer, buf, cap, C.byref(n)))
        return list(buf[: n.value])

    def slot_of_frame(self, layer, frame):
        s = C.c_int64()
        _check(lib().ll_cache_slot_of_frame(self._h, layer, frame, C.byref(s)))
        return s.value

    def live_ranges(self, layer):
        buf, n = (C.c_int64 * 16)(), C.c_int()
        _check(lib().ll_cache_live_ranges(self._h, layer, buf, 8, C.byref(n)))
        return [(buf[2 * i], buf[2 * i + 1]) for i in range(n.value)]

    def read_frame(self, layer, frame, k_out, v_out):
        _check(lib().ll_cache_read_frame(self._h, layer, frame, _ptr(k_out), _ptr(v_out), _stream()))


class Prompt:
    """Handle on the per-layer keys and values of the active prompt (``ll_prompt_*``, ``ll_cross_attn``).
    ``device=None`` makes an index-only handle."""

    def __init__(self, layers, heads, head_dim, max_tokens, device="cuda"):
        self.layers, self.heads, self.head_dim, self.max_tokens = layers, heads, head_dim, max_tokens
        self._h = C.c_void_p()
        self.buffer = None
        nbytes = lib().ll_prompt_bytes(layers, heads, head_dim, max_tokens)
        if device is not None:
            import torch
            if nbytes == 0:
                raise LongLiveError(1, "invalid shape")
            self.buffer = torch.empty(nbytes, dtype=torch.uint8, device=device)
            ptr, size = C.c_void_p(self.buffer.data_ptr()), nbytes
        else:
            ptr, size = None, 0
        _check(lib().ll_prompt_create(layers, heads, head_dim, max_tokens, ptr, size, C.byref(self._h)))

    def close(self):
        if self._h:
            lib().ll_prompt_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def recache(self, layer, k, v, n_tokens=None):
        """Replace the layer's prompt keys and values: k, v bf16 [n_tokens, H, D] on the device."""
        if n_tokens is None:
            n_tokens = k.shape[0]
        if self.buffer is not None:
            _check(lib().ll_prompt_recache(self._h, layer, _ptr(k), _ptr(v), n_tokens, _stream()))
        else:
            _check(lib().ll_prompt_recache(self._h, layer, None, None, n_tokens, None))

    def tokens(self, layer) -> int:
        n = C.c_int()
        _check(lib().ll_prompt_tokens(self._h, layer, C.byref(n)))
        return n.value

    def cross_attn(self, layer, q, out, n_q=None):
        """out = softmax(q k^T / sqrt(D)) v over the layer's prompt; q, out bf16 [n_q, H, D] on the device."""
        if n_q is None:
            n_q = q.shape[0]
        if self.buffer is not None:
            _check(lib().ll_cross_attn(self._h, layer, _ptr(q), n_q, _ptr(out), _stream()))
        else:
            _check(lib().ll_cross_attn(self._h, layer, None, n_q, None, None))

    def pack_out_weight(self, w_out, w_packed):
        """The layer's output weight (bf16 [H*D, H*D], [output feature][input feature]) in the projection's order."""
        _check(lib().ll_out_proj_pack_weight(self.heads, self.head_dim, _ptr(w_out), _ptr(w_packed), _stream()))

    def cross_attn_out_workspace_bytes(self, n_q) -> int:
        return lib().ll_cross_attn_out_workspace_bytes(self.heads, self.head_dim, n_q)

    def cross_attn_out(self, layer, q=None, w_packed=None, workspace=None, y=None, n_q=None):
        """Cross-attention followed by the output projection y = concat_heads(attention output) w_out^T; w_packed from
        pack_out_weight, workspace of cross_attn_out_workspace_bytes(n_q) bytes."""
        if q is not None:
            n_q = q.shape[0]
            _check(lib().ll_cross_attn_out(self._h, layer, _ptr(q), n_q, _ptr(w_packed), _ptr(workspace), _ptr(y), _stream()))
        else:
            _check(lib().ll_cross_attn_out(self._h, layer, None, n_q, None, None, None, None))


class Clip:
    """Handle on one layer's training step: attention of a supervised clip over sink + detached window + itself
    (``ll_clip_forward``) and its gradients (``ll_clip_backward``).  ``device=None`` makes an index-only handle."""

    def __init__(self, heads, head_dim, grid_h, grid_w, chunk_frames, sink_frames, window_frames, clip_frames,
                 rope_theta=10000.0, device="cuda"):
        self.heads, self.head_dim, self.P = heads, head_dim, grid_h * grid_w
        self._h = C.c_void_p()
        self.buffer = None
        nbytes = lib().ll_clip_bytes(heads, head_dim, self.P, sink_frames, window_frames, clip_frames, chunk_frames)
        if device is not None:
            import torch
            if nbytes == 0:
                raise LongLiveError(1, "invalid shape")
            self.buffer = torch.empty(nbytes, dtype=torch.uint8, device=device)
            ptr, size = C.c_void_p(self.buffer.data_ptr()), nbytes
        else:
            ptr, size = None, 0
        _check(lib().ll_clip_create(heads, head_dim, self.P, sink_frames, window_frames, clip_frames, chunk_frames,
                                    grid_h, grid_w, rope_theta, ptr, size, C.byref(self._h)))

    def close(self):
        if self._h:
            lib().ll_clip_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def forward(self, ctx_start, n_ctx, n_clip, q=None, k=None, v=None, out=None):
        stream = _stream() if self.buffer is not None else None
        _check(lib().ll_clip_forward(self._h, ctx_start, n_ctx, n_clip, _ptr(q), _ptr(k), _ptr(v), _ptr(out), stream))

    def chunk_key_ranges(self, chunk):
        """Key set of one chunk of the last forward: [(begin, end)] token-slot ranges into the resident frames."""
        buf, n = (C.c_int64 * 4)(), C.c_int()
        _check(lib().ll_clip_chunk_key_ranges(self._h, chunk, buf, 2, C.byref(n)))
        return [(buf[2 * i], buf[2 * i + 1]) for i in range(n.value)]

    def backward(self, dout=None, dq=None, dk=None, dv=None):
        stream = _stream() if self.buffer is not None else None
        _check(lib().ll_clip_backward(self._h, _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), stream))


ROPES = {"none": 0, "pairs": 1, "halves": 2, "grid": 3}
ACTIVATIONS = {"none": 0, "gelu_tanh": 1, "gelu": 2, "silu": 3}


def _rows(t, name, dtype, shape, index):
    """Elements from one row of ``t`` to the next; raises ValueError unless it has this type and shape, lies on GPU ``index`` (-1: the CPU) and
    each row's numbers lie one after the other.  A single row's stride is a row's length."""
    if t.dtype is not dtype or t.shape != shape or t.get_device() != index:
        raise ValueError(f"{name}: {dtype} {list(shape)} on GPU {index} is needed, got {t.dtype} {list(t.shape)} on {t.device}")
    row = 1
    for n in shape[1:]:
        row *= n
    if t.is_contiguous():
        return row
    dense, steps = 1, t.stride()
    for i in range(len(shape) - 1, 0, -1):
        if steps[i] != dense and shape[i] != 1:
            raise ValueError(f"{name}: a row's numbers must lie one after the other, got strides {list(steps)}")
        dense *= shape[i]
    return steps[0] if shape[0] > 1 else row


def _ints(t, name, shape, index):
    """The address of a contiguous int32 array of this shape, or None."""
    import torch
    if t is None:
        return None
    if t.dtype is not torch.int32 or t.shape != shape or t.get_device() != index or not t.is_contiguous():
        raise ValueError(f"{name}: contiguous int32 {list(shape)} on GPU {index} is needed, got {t.dtype} {list(t.shape)} on {t.device}, strides {list(t.stride())}")
    return t.data_ptr()


def _call_on(index, fn, *args):
    """fn(*args, stream) with GPU ``index`` current and its current stream.  The stream is asked for as torch's generated code does: 0.1 us where
    a Stream object takes 1.1, of the 9 that a small call takes the host."""
    import torch
    stream = torch._C._cuda_getCurrentRawStream(index)
    if torch.cuda.current_device() == index:
        _check(fn(*args, stream))
    else:
        with torch.cuda.device(index):
            _check(fn(*args, stream))


class PagedCache:
    """Handle on ``layers`` paged caches of ``n_pages`` pages that many sequences share (``ll_paged_*``).  ``device=None`` makes an
    index-only handle.

    ``rope``: "none", "pairs", "halves" or "grid"; ``rope_dim`` None turns whole heads.  The tensors of a call are on the cache's device, and
    its work goes to that device's current stream."""

    def __init__(self, layers, q_heads, kv_heads, head_dim, page_tokens, n_pages, rope="none", rope_dim=None, rope_theta=10000.0,
                 kv_format="bf16", k_exp=0, v_exp=0, device="cuda"):
        if kv_format not in ("bf16", "fp8_e4m3"):
            raise ValueError(f"kv_format {kv_format!r}")
        if rope not in ROPES:
            raise ValueError(f"rope {rope!r}")
        if rope_dim is None:
            rope_dim = 0 if rope == "none" else head_dim
        fmt = int(kv_format == "fp8_e4m3")
        self.layers, self.q_heads, self.kv_heads, self.head_dim = layers, q_heads, kv_heads, head_dim
        self.page_tokens, self.n_pages, self.kv_format, self.rope = page_tokens, n_pages, kv_format, rope
        self._h = C.c_void_p()
        self.buffer = None
        self._views = {}
        nbytes = lib().ll_paged_bytes(layers, kv_heads, head_dim, page_tokens, n_pages, fmt)
        ptr, size = None, 0
        if device is not None:
            import torch
            if torch.device(device).type != "cuda":
                raise ValueError(f"device {device}: the pool must be on a GPU")
            if nbytes == 0:
                raise LongLiveError(1, "invalid shape")
            self.buffer = torch.empty(nbytes, dtype=torch.uint8, device=device)
            ptr, size = C.c_void_p(self.buffer.data_ptr()), nbytes
        args = (layers, q_heads, kv_heads, head_dim, page_tokens, n_pages, fmt, k_exp, v_exp, ROPES[rope], rope_dim, rope_theta, ptr, size, C.byref(self._h))
        if self.buffer is None:
            _check(lib().ll_paged_create(*args))
        else:
            self._index = self.buffer.get_device()
            with torch.cuda.device(self._index):
                _check(lib().ll_paged_create(*args))

    def close(self):
        if self._h:
            lib().ll_paged_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _gpu(self):
        """The index of the cache's GPU."""
        if self.buffer is None:
            raise LongLiveError(1, "an index-only handle has no memory")
        return self._index

    def _images(self, layer):
        """The layer's numbers as [page, kv head, K or V, granule of 16 tokens, piece, 4, 16, ...] (the layout in longlive.h)."""
        import torch
        self._gpu()
        if not 0 <= layer < self.layers:
            raise LongLiveError(1, f"layer {layer} out of range [0, {self.layers})")
        dtype = torch.bfloat16 if self.kv_format == "bf16" else torch.float8_e4m3fn
        numbers = self.n_pages * self.kv_heads * 2 * self.page_tokens * self.head_dim
        pool = self.buffer[: self.buffer.numel() - self.head_dim // 2 * 8].view(dtype)[layer * numbers:(layer + 1) * numbers]
        return pool.view(self.n_pages, self.kv_heads, 2, self.page_tokens // 16, -1, 4, 16, 8 if dtype == torch.bfloat16 else 16)

    def keys(self, layer):
        """The layer's keys where they lie: a view whose elements, taken in order, are [n_pages, page_tokens, kv_heads, head_dim] (8 dimensions,
        or 7 for bfloat16; ``.reshape`` copies, ``.copy_`` fills the cache)."""
        if ("k", layer) not in self._views:
            x = self._images(layer)[:, :, 0]                                          # page, head, granule, c, g, r, rest
            if self.kv_format == "bf16":
                x = x.permute(0, 2, 5, 1, 3, 4, 6)                                    # page, granule, r, head, c, g, e
            else:
                x = x.unflatten(-1, (2, 8)).permute(0, 2, 5, 1, 3, 6, 4, 7)           # page, granule, r, head, c, s, g, e
            self._views["k", layer] = x
        return self._views["k", layer]

    def values(self, layer):
        """The layer's values where they lie, as ``keys`` has the keys (8 dimensions)."""
        if ("v", layer) not in self._views:
            x = self._images(layer)[:, :, 1].unflatten(-1, (-1, 4))                   # page, head, granule, c, g, r, h, j
            self._views["v", layer] = x.permute(0, 2, 4, 7, 1, 3, 6, 5)               # page, granule, g, j, head, c, h, r
        return self._views["v", layer]

    def _batch(self, seq_lens, page_table, cu_tokens):
        """(n_seqs, cu_tokens, seq_lens, page_table, columns, row stride) as the calls take them."""
        import torch
        i = self._gpu()
        n = page_table.shape[0]
        cols = page_table.shape[-1]
        stride = _rows(page_table, "page_table", torch.int32, (n, cols), i)
        return n, _ints(cu_tokens, "cu_tokens", (n + 1,), i), _ints(seq_lens, "seq_lens", (n,), i), page_table.data_ptr(), cols, stride

    def append(self, layer, seq_lens, page_table, k, v, q=None, q_out=None, cu_tokens=None, positions=None):
        """New tokens' keys and values into their pages, and q_out = turned, scaled q (``ll_paged_append``).  k, v bf16 [n_tokens, kv_heads, D],
        q, q_out bf16 [n_tokens, q_heads, D] or None; positions int32 [n_tokens] ([n_tokens, 3] for "grid") or None."""
        import torch
        i, bf16 = self._gpu(), torch.bfloat16
        n_seqs, cu, lens, table, cols, stride = self._batch(seq_lens, page_table, cu_tokens)
        rows = k.shape[0]
        kv, queries = (rows, self.kv_heads, self.head_dim), (rows, self.q_heads, self.head_dim)
        k_stride, v_stride = _rows(k, "k", bf16, kv, i), _rows(v, "v", bf16, kv, i)
        if (q is None) != (q_out is None):
            raise ValueError("q and q_out come together")
        q_at = out_at = None
        q_stride = out_stride = 0
        if q is not None:
            q_stride, out_stride = _rows(q, "q", bf16, queries, i), _rows(q_out, "q_out", bf16, queries, i)
            q_at, out_at = q.data_ptr(), q_out.data_ptr()
        at = _ints(positions, "positions", (rows, 3) if self.rope == "grid" else (rows,), i)
        _call_on(i, lib().ll_paged_append, self._h, layer, n_seqs, rows, cu, lens, table, cols, stride, at, q_at, q_stride, k.data_ptr(), k_stride,
                 v.data_ptr(), v_stride, out_at, out_stride)

    def attn_workspace_bytes(self, n_seqs, max_new=1, max_len=None, sink_tokens=0, window_tokens=0) -> int:
        """Bytes of ``attn``'s workspace for these sizes; max_len None: as much as the pool holds, which is right for one sequence that fills it and costs
        time for shorter ones (16384 tokens in a pool of 524288: 81 us, with their own length 17)."""
        return lib().ll_paged_attn_workspace_bytes(self._h, n_seqs, max_new, self._max_len(max_len), sink_tokens, window_tokens)

    def attn_workspace(self, n_seqs, max_new=1, max_len=None, sink_tokens=0, window_tokens=0):
        """A workspace of that many bytes on the cache's device, for one ``attn`` call at a time."""
        import torch
        return torch.empty(self.attn_workspace_bytes(n_seqs, max_new, max_len, sink_tokens, window_tokens), dtype=torch.uint8,
                           device=torch.device("cuda", self._gpu()))

    def _max_len(self, max_len):
        return min(self.n_pages * self.page_tokens, 1 << 30) if max_len is None else max_len

    def attn(self, layer, seq_lens, page_table, q, out, workspace=None, cu_tokens=None, max_new=1, max_len=None, sink_tokens=0, window_tokens=0):
        """Attention of the new tokens' queries over their sequences' pages (``ll_paged_attn``).  q as ``append`` left it in q_out, out like it; the
        workspace from ``attn_workspace`` with the same sizes.  max_len: the longest sequence's length, as near as it is known (None: see
        ``attn_workspace_bytes``); max_new: the most rows that a sequence brings by ``cu_tokens``, later ones are left alone."""
        import torch
        i = self._gpu()
        n_seqs, cu, lens, table, cols, stride = self._batch(seq_lens, page_table, cu_tokens)
        shape = (q.shape[0], self.q_heads, self.head_dim)
        q_stride, out_stride = _rows(q, "q", torch.bfloat16, shape, i), _rows(out, "out", torch.bfloat16, shape, i)
        size = 0
        if workspace is not None:
            size = workspace.numel()
            _rows(workspace, "workspace", torch.uint8, (size,), i)
            if size > 1 and workspace.stride(0) != 1:
                raise ValueError("workspace must be contiguous")
        _call_on(i, lib().ll_paged_attn, self._h, layer, n_seqs, shape[0], max_new, self._max_len(max_len), cu, lens, table, cols, stride, sink_tokens,
                 window_tokens, q.data_ptr(), q_stride, out.data_ptr(), out_stride, workspace.data_ptr() if size else None, size)


class Linear:
    """A weight laid out for ``ll_linear``: w bf16 [n_out, n_in] on the GPU, n_in a multiple of 8.  Keeps its own copy, in ``packed``, which is written on the
    stream that is current here: other streams wait for it before their first ``forward``, as for any tensor."""

    def __init__(self, w):
        import torch
        self._index = w.get_device()
        if self._index < 0:
            raise ValueError("w must be on a GPU")
        self.n_out, self.n_in = w.shape
        stride = _rows(w, "w", torch.bfloat16, (self.n_out, self.n_in), self._index)
        nbytes = lib().ll_linear_packed_bytes(self.n_out, self.n_in)
        if nbytes == 0:
            raise LongLiveError(1, f"no kernel for a weight of {self.n_out} x {self.n_in}")
        self.packed = torch.empty(nbytes, dtype=torch.uint8, device=w.device)
        _call_on(self._index, lib().ll_linear_pack_weight, self.n_out, self.n_in, w.data_ptr(), stride, self.packed.data_ptr())

    def forward(self, x, y, bias=None, activation="none", residual=None):
        """y = activation(x w^T + bias) + residual: x bf16 [m, n_in], y and residual bf16 [m, n_out], bias bf16 [n_out].  y may be the residual."""
        import torch
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation {activation!r}")
        i, bf16, m, n, k = self._index, torch.bfloat16, x.shape[0], self.n_out, self.n_in
        x_stride, y_stride = _rows(x, "x", bf16, (m, k), i), _rows(y, "y", bf16, (m, n), i)
        bias_at = residual_at = None
        residual_stride = 0
        if bias is not None:
            _rows(bias, "bias", bf16, (n,), i)
            if not bias.is_contiguous():
                raise ValueError("bias must be contiguous")
            bias_at = bias.data_ptr()
        if residual is not None:
            residual_stride = _rows(residual, "residual", bf16, (m, n), i)
            residual_at = residual.data_ptr()
        _call_on(i, lib().ll_linear, m, n, k, x.data_ptr(), x_stride, self.packed.data_ptr(), bias_at, ACTIVATIONS[activation], residual_at,
                 residual_stride, y.data_ptr(), y_stride)
