"""Thin Python binding of the C-ABI library (argument marshalling only).

Every step of the method runs in the CUDA kernels of libmvsparse.so; this module only
turns torch tensors into raw pointers, allocates the caller-owned workspace and checks
status codes.  There is no CPU fallback: if the library has not been built, importing
`load()` raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmvsparse.so")
LIB_DEBUG_PATH = os.path.join(_HERE, "libmvsparse_debug.so")     # the checked build, see MvContext.debug_status

MV_OK = 0
MV_ERR_INVALID_ARG = -1
MV_ERR_WORKSPACE = -2
MV_ERR_CUDA = -3
MV_ERR_TOO_LARGE = -4
MV_ERR_TIMEOUT = -5
MV_SELECT_STATIC_MAX_D = 1 << 24
MV_MODE_AUTO = 0
MV_MODE_GENERAL = 1
MV_MODE_TRACK = 2
MV_F32, MV_BF16, MV_F16, MV_I32, MV_I64 = 0, 1, 2, 3, 4
MV_TOP_MAX = 64
MV_DBG_CAND_OVERFLOW, MV_DBG_WINDOW_OVERFLOW, MV_DBG_FALLBACK, MV_DBG_LIST_OVERFLOW = 1, 2, 4, 8
MV_DBG_PICK_RANGE, MV_DBG_LIST_RANGE, MV_DBG_OUT_RANGE, MV_DBG_GATHER_RANGE, MV_DBG_INTERNAL = 16, 32, 64, 128, 256

_lib = None
_lib_debug = None


class MvError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


def load() -> ctypes.CDLL:
    """Loads libmvsparse.so (built in-tree by paper_2011_06495_b200.build); raises if absent."""
    global _lib
    if _lib is None:
        _lib = _open(LIB_PATH, "python -m paper_2011_06495_b200.build")
    return _lib


def load_debug() -> ctypes.CDLL:
    """Loads the checked build libmvsparse_debug.so (same ABI; its kernels report clamped or refused
    indices through mv_debug_status); raises if absent."""
    global _lib_debug
    if _lib_debug is None:
        _lib_debug = _open(LIB_DEBUG_PATH, "python -m paper_2011_06495_b200.build --debug")
    return _lib_debug


def _open(path: str, how: str) -> ctypes.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `{how}` (there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    c_vp, c_i, c_i64, c_sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
    lib.mv_workspace_bytes.restype = c_sz
    lib.mv_workspace_bytes.argtypes = [c_i, c_i64, c_i64]
    lib.mv_create.restype = c_i
    lib.mv_create.argtypes = [ctypes.POINTER(c_vp), c_vp, c_vp, c_sz]
    lib.mv_destroy.restype = c_i
    lib.mv_destroy.argtypes = [c_vp]
    lib.mv_set_mode.restype = c_i
    lib.mv_set_mode.argtypes = [c_vp, c_i]
    lib.mv_sparse_step.restype = c_i
    lib.mv_sparse_step.argtypes = [c_vp, c_vp, c_vp, c_i, c_i64, c_i64, c_vp, c_vp]
    lib.mv_vote.restype = c_i
    lib.mv_vote.argtypes = [c_vp, c_vp, c_vp, c_i, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp]
    lib.mv_select.restype = c_i
    lib.mv_select.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_vp, c_vp]
    lib.mv_ad_step.restype = c_i
    lib.mv_ad_step.argtypes = [c_vp, c_vp, c_vp, c_vp, c_i, c_i64, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp, c_vp]
    lib.mv_topk_union_step.restype = c_i
    lib.mv_topk_union_step.argtypes = [c_vp, c_vp, c_vp, c_i, c_i64, c_i64, c_vp, c_vp, c_i64, c_vp]
    lib.mv_select_static.restype = c_i
    lib.mv_select_static.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_vp, c_vp]
    lib.mv_aggregate.restype = c_i
    lib.mv_aggregate.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_vp, c_vp]
    lib.mv_sparse_step_host.restype = c_i
    lib.mv_sparse_step_host.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_vp, c_vp, c_vp, c_vp, c_vp, c_vp]
    lib.mv_read_diag.restype = c_i
    lib.mv_read_diag.argtypes = [c_vp, c_i, c_vp]
    lib.mv_set_kernel_timing.restype = c_i
    lib.mv_set_kernel_timing.argtypes = [c_vp, c_i]
    lib.mv_read_kernel_timing.restype = c_i
    lib.mv_read_kernel_timing.argtypes = [c_vp, ctypes.POINTER(ctypes.c_float), ctypes.POINTER(c_i)]
    lib.mv_set_phase_timing.restype = c_i
    lib.mv_set_phase_timing.argtypes = [c_vp, c_i]
    lib.mv_read_phase_times.restype = c_i
    lib.mv_read_phase_times.argtypes = [c_vp, ctypes.POINTER(ctypes.c_float), c_i, ctypes.POINTER(c_i)]
    lib.mv_last_launches.restype = c_i
    lib.mv_last_launches.argtypes = [c_vp]
    lib.mv_status_string.restype = ctypes.c_char_p
    lib.mv_status_string.argtypes = [c_i]
    c_u64 = ctypes.c_uint64
    lib.mv_select_rs.restype = c_i
    lib.mv_select_rs.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_u64, c_u64, c_vp, c_vp]
    lib.mv_rs_step.restype = c_i
    lib.mv_rs_step.argtypes = [c_vp, c_vp, c_vp, c_i, c_i64, c_i64, c_u64, c_u64, c_vp, c_vp]
    lib.mv_aggregate_partial.restype = c_i
    lib.mv_aggregate_partial.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_vp, c_vp]
    lib.mv_finish_mean.restype = c_i
    lib.mv_finish_mean.argtypes = [c_vp, c_vp, c_i64, c_i, c_vp]
    # wire formats (include/mv_wire.h)
    lib.mv_pos_offset_bits.restype = c_i
    lib.mv_pos_offset_bits.argtypes = [c_i64]
    lib.mv_pos_stream_bits.restype = c_i64
    lib.mv_pos_stream_bits.argtypes = [c_i64, c_i64, c_i64]
    lib.mv_pos_decode_workspace_bytes.restype = c_sz
    lib.mv_pos_decode_workspace_bytes.argtypes = [c_i64, c_i64]
    lib.mv_pos_encode.restype = c_i
    lib.mv_pos_encode.argtypes = [c_vp, c_vp, c_i64, c_i64, c_i64, c_vp]
    lib.mv_pos_decode.restype = c_i
    lib.mv_pos_decode.argtypes = [c_vp, c_vp, c_i64, c_i64, c_i64, c_vp, c_i64, c_vp, c_vp, c_sz]
    lib.mv_quant_stream_words.restype = c_i64
    lib.mv_quant_stream_words.argtypes = [c_i64, c_i]
    lib.mv_quant_workspace_bytes.restype = c_sz
    lib.mv_quant_workspace_bytes.argtypes = [c_i]
    lib.mv_quantize.restype = c_i
    lib.mv_quantize.argtypes = [c_vp, c_vp, c_i64, c_i, c_vp, c_vp, c_vp, c_sz]
    lib.mv_dequantize.restype = c_i
    lib.mv_dequantize.argtypes = [c_vp, c_vp, c_i64, c_i, c_vp]
    # language-model operators (include/mv_lm.h)
    c_f = ctypes.c_float
    lib.mv_embed.restype = c_i
    lib.mv_embed.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_i64, c_vp, c_i, c_i64, c_f, c_vp, c_i, c_i64]
    lib.mv_embed_grad_workspace_bytes.restype = c_sz
    lib.mv_embed_grad_workspace_bytes.argtypes = [c_i64, c_i64, c_i64]
    lib.mv_embed_grad.restype = c_i
    lib.mv_embed_grad.argtypes = [c_vp, c_vp, c_i, c_i64, c_vp, c_i, c_i64, c_i64, c_i64, c_f, c_i64, c_i, c_vp, c_i64, c_vp, c_sz]
    lib.mv_token_logprob.restype = c_i
    lib.mv_token_logprob.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_i64, c_vp, c_i, c_f, c_i, c_vp, c_vp, c_vp, c_vp, c_vp]
    lib.mv_token_logprob_grad.restype = c_i
    lib.mv_token_logprob_grad.argtypes = [c_vp, c_vp, c_i, c_i64, c_i64, c_i64, c_vp, c_i, c_f, c_vp, c_vp, c_vp, c_vp, c_vp, c_i64]
    lib.mv_clip_workspace_bytes.restype = c_sz
    lib.mv_clip_workspace_bytes.argtypes = [c_vp, c_i, c_i]
    lib.mv_clip_create.restype = c_i
    lib.mv_clip_create.argtypes = [ctypes.POINTER(c_vp), c_vp, c_vp, c_vp, c_vp, c_vp, c_i, c_i, c_vp, c_sz]
    lib.mv_clip_destroy.restype = c_i
    lib.mv_clip_destroy.argtypes = [c_vp]
    lib.mv_clip_status.restype = c_i
    lib.mv_clip_status.argtypes = [c_vp, c_vp]
    lib.mv_clip_set_polls.restype = c_i
    lib.mv_clip_set_polls.argtypes = [c_vp, c_i]
    lib.mv_clip_norm.restype = c_i
    lib.mv_clip_norm.argtypes = [c_vp, c_vp, c_vp]
    lib.mv_clip_scale.restype = c_i
    lib.mv_clip_scale.argtypes = [c_vp, c_vp, c_f, c_vp]
    lib.mv_clip_pack.restype = c_i
    lib.mv_clip_pack.argtypes = [c_vp, c_vp, c_f, c_vp, c_i64, c_vp]
    lib.mv_set_tail_kernel.restype = c_i
    lib.mv_set_tail_kernel.argtypes = [c_vp, c_i]
    lib.mv_fallback_count.restype = c_i
    lib.mv_fallback_count.argtypes = [c_vp, ctypes.POINTER(ctypes.c_uint32)]
    lib.mv_debug_status.restype = c_i
    lib.mv_debug_status.argtypes = [c_vp, ctypes.POINTER(c_i)]
    lib.mv_debug_build.restype = c_i
    lib.mv_debug_build.argtypes = []
    return lib


def status_string(status: int) -> str:
    return load().mv_status_string(int(status)).decode()


def workspace_bytes(N: int, d: int, K: int) -> int:
    return int(load().mv_workspace_bytes(int(N), int(d), int(K)))


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _check(status: int, where: str):
    if status != MV_OK:
        raise MvError(status, where)


def mv_select_static(votes, N: int, K: int, out_idx, mask_bits=None, stream: Optional[torch.cuda.Stream] = None):
    """mv_select without a context or a workspace (scratch is an array built into the library);
    for callers that may not allocate device memory.  d is limited to MV_SELECT_STATIC_MAX_D."""
    st = stream if stream is not None else torch.cuda.current_stream(votes.device)
    _check(load().mv_select_static(ctypes.c_void_p(st.cuda_stream), _ptr(votes), int(N), votes.numel(), int(K),
                                   _ptr(out_idx), _ptr(mask_bits)), "mv_select_static")


def _stream_ptr(t: torch.Tensor, stream: Optional[torch.cuda.Stream]):
    st = stream if stream is not None else torch.cuda.current_stream(t.device)
    return ctypes.c_void_p(st.cuda_stream)


def pos_offset_bits(B: int) -> int:
    return int(load().mv_pos_offset_bits(int(B)))


def pos_stream_bits(d: int, B: int, K: int) -> int:
    return int(load().mv_pos_stream_bits(int(d), int(B), int(K)))


def pos_decode_workspace_bytes(nbits: int, B: int) -> int:
    return int(load().mv_pos_decode_workspace_bytes(int(nbits), int(B)))


def quant_stream_words(K: int, q: int) -> int:
    return int(load().mv_quant_stream_words(int(K), int(q)))


def quant_workspace_bytes(q: int) -> int:
    return int(load().mv_quant_workspace_bytes(int(q)))


def mv_pos_encode(idx, d: int, B: int, words, stream: Optional[torch.cuda.Stream] = None):
    """Position stream of an ascending int32 index list into `words` (uint32/int32, caller-sized)."""
    _check(load().mv_pos_encode(_stream_ptr(words, stream), _ptr(idx), idx.numel(), int(d), int(B), _ptr(words)),
           "mv_pos_encode")


def mv_pos_decode(words, nbits: int, d: int, B: int, idx, result, workspace, stream: Optional[torch.cuda.Stream] = None):
    _check(load().mv_pos_decode(_stream_ptr(words, stream), _ptr(words), int(nbits), int(d), int(B), _ptr(idx),
                                idx.numel(), _ptr(result), _ptr(workspace), workspace.numel() * workspace.element_size()),
           "mv_pos_decode")


def mv_quantize(v, q: int, words, workspace, value_range=None, stream: Optional[torch.cuda.Stream] = None):
    _check(load().mv_quantize(_stream_ptr(words, stream), _ptr(v), v.numel(), int(q), _ptr(words), _ptr(value_range),
                              _ptr(workspace), workspace.numel() * workspace.element_size()), "mv_quantize")


def mv_dequantize(words, K: int, q: int, out, stream: Optional[torch.cuda.Stream] = None):
    _check(load().mv_dequantize(_stream_ptr(words, stream), _ptr(words), int(K), int(q), _ptr(out)), "mv_dequantize")


_TYPES = {torch.float32: MV_F32, torch.bfloat16: MV_BF16, torch.float16: MV_F16, torch.int32: MV_I32, torch.int64: MV_I64}
_VALUES, _IDS, _FLOAT = (MV_F32, MV_BF16, MV_F16), (MV_I32, MV_I64), (MV_F32,)
_raw_current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)     # absent from a torch without CUDA


def _need(ok: bool, where: str):
    """Shapes, types and devices that the raw pointers of the C call no longer show."""
    if not ok:
        raise MvError(MV_ERR_INVALID_ARG, where)


def _raw_stream(device_index: int, stream: Optional[torch.cuda.Stream]):
    return stream.cuda_stream if stream is not None else _raw_current_stream(device_index)


def _matrix(t: torch.Tensor, kinds, where: str):
    """(address, type code, rows, columns, row pitch, device) of a 2-d CUDA tensor whose rows are contiguous."""
    code, shape, stride, dev = _TYPES.get(t.dtype, -1), t.shape, t.stride(), t.get_device()
    if len(shape) != 2 or code not in kinds or dev < 0 or (stride[1] != 1 and shape[1] != 1):
        raise MvError(MV_ERR_INVALID_ARG, where)
    rows, cols = shape
    return t.data_ptr(), code, rows, cols, stride[0] if rows > 1 else cols, dev


def _vector(t: Optional[torch.Tensor], n: int, kinds, dev: int, where: str):
    """(address, type code) of a contiguous 1-d tensor of n elements on that device; (None, first kind) for None."""
    if t is None:
        return None, kinds[0]
    code = _TYPES.get(t.dtype, -1)
    if code not in kinds or t.dim() != 1 or t.numel() != n or t.get_device() != dev or not t.is_contiguous():
        raise MvError(MV_ERR_INVALID_ARG, where)
    return t.data_ptr(), code


def mv_embed(weight, ids, out, scale: float = 1.0, stream: Optional[torch.cuda.Stream] = None):
    """out[t] = scale * weight[ids[t]]; weight [V, D], ids [T], out [T, D]."""
    w, w_type, V, D, ldw, dev = _matrix(weight, _VALUES, "mv_embed")
    o, o_type, T, Do, ldo, dev_o = _matrix(out, _VALUES, "mv_embed")
    i, i_type = _vector(ids, T, _IDS, dev, "mv_embed")
    _need(Do == D and dev_o == dev, "mv_embed")
    _check(load().mv_embed(_raw_stream(dev, stream), w, w_type, V, D, ldw, i, i_type, T, float(scale), o, o_type, ldo), "mv_embed")


def embed_grad_workspace_bytes(T: int, V: int, D: int) -> int:
    return int(load().mv_embed_grad_workspace_bytes(int(T), int(V), int(D)))


def mv_embed_grad(dout, ids, dweight, workspace, scale: float = 1.0, pad_id: int = -1, accumulate: bool = False,
                  stream: Optional[torch.cuda.Stream] = None):
    """dweight[v] (+)= scale * sum of dout over the tokens with id v; dout [T, D], ids [T], dweight float [V, D]."""
    x, x_type, T, D, ldd, dev = _matrix(dout, _VALUES, "mv_embed_grad")
    d, _, V, Dw, ldw, dev_w = _matrix(dweight, _FLOAT, "mv_embed_grad")
    i, i_type = _vector(ids, T, _IDS, dev, "mv_embed_grad")
    _need(Dw == D and dev_w == dev and workspace.get_device() == dev and workspace.is_contiguous(), "mv_embed_grad")
    _check(load().mv_embed_grad(_raw_stream(dev, stream), x, x_type, ldd, i, i_type, T, V, D, float(scale), int(pad_id), bool(accumulate), d, ldw,
                                workspace.data_ptr(), workspace.numel() * workspace.element_size()), "mv_embed_grad")


def mv_token_logprob(logits, targets=None, scale: float = 1.0, logprob=None, entropy=None, lse=None, top_logprob=None, top_id=None,
                     stream: Optional[torch.cuda.Stream] = None):
    """Log probabilities of targets [T] under softmax(scale * logits), logits [T, V]; logprob, entropy, lse: float [T];
    top_logprob float [T, k], top_id int32 [T, k].  An output that is None is not computed."""
    where = "mv_token_logprob"
    x, x_type, T, V, ld, dev = _matrix(logits, _VALUES, where)
    y, i_type = _vector(targets, T, _IDS, dev, where)
    lp, h, l = _vector(logprob, T, _FLOAT, dev, where)[0], _vector(entropy, T, _FLOAT, dev, where)[0], _vector(lse, T, _FLOAT, dev, where)[0]
    k, tops = None, [None, None]
    for j, (t, kind) in enumerate(((top_logprob, torch.float32), (top_id, torch.int32))):
        if t is not None:
            n, width = t.shape if t.dim() == 2 else (-1, 0)
            _need(n == T and t.dtype == kind and t.get_device() == dev and t.is_contiguous() and k in (None, width), where)
            k, tops[j] = width, t.data_ptr()
    _check(load().mv_token_logprob(_raw_stream(dev, stream), x, x_type, T, V, ld, y, i_type, float(scale), k or 0, lp, h, l, tops[0], tops[1]), where)


def mv_token_logprob_grad(logits, targets, lse, g_logprob, dlogits, scale: float = 1.0, entropy=None, g_entropy=None,
                          stream: Optional[torch.cuda.Stream] = None):
    """dlogits [T, V] of sum(g_logprob * logprob + g_entropy * entropy); dlogits may be logits.  g_logprob (with targets)
    or g_entropy (with entropy) may be None."""
    where = "mv_token_logprob_grad"
    x, x_type, T, V, ld, dev = _matrix(logits, _VALUES, where)
    d, d_type, Td, Vd, ldg, dev_d = _matrix(dlogits, _VALUES, where)
    y, i_type = _vector(targets, T, _IDS, dev, where)
    l, h = _vector(lse, T, _FLOAT, dev, where)[0], _vector(entropy, T, _FLOAT, dev, where)[0]
    g1, g2 = _vector(g_logprob, T, _FLOAT, dev, where)[0], _vector(g_entropy, T, _FLOAT, dev, where)[0]
    _need(d_type == x_type and Td == T and Vd == V and dev_d == dev, where)
    _check(load().mv_token_logprob_grad(_raw_stream(dev, stream), x, x_type, T, V, ld, y, i_type, float(scale), l, h, g1, g2, d, ldg), where)


class MvClip:
    """A plan over a fixed list of contiguous tensors, which it keeps alive with its workspace; `groups` (ascending) says
    which tensors share a norm (None: all of them).  Calls may go to any stream, one after the other; the plan and the tensors
    may be dropped before they have run."""

    def __init__(self, tensors, groups=None, n_groups: Optional[int] = None, stream: Optional[torch.cuda.Stream] = None, device=None):
        self.handle = None
        self.lib = load()
        self.tensors = list(tensors)
        n = len(self.tensors)
        dev = torch.device(device) if device is not None else self.tensors[0].device if n else torch.device("cuda")
        if dev.type == "cuda" and dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        groups = [0] * n if groups is None else [int(g) for g in groups]
        self.n_groups = int(n_groups) if n_groups is not None else (max(groups) + 1 if n else 1)
        lengths = [0] * max(self.n_groups, 1)
        for t, g in zip(self.tensors, groups):
            if 0 <= g < self.n_groups:
                lengths[g] += t.numel()
        self.longest = max(lengths)              # elements of the longest group: what a row has to hold
        _need(len(groups) == n and all(t.is_cuda and t.device == dev and t.is_contiguous() for t in self.tensors), "mv_clip_create")
        ptrs = (ctypes.c_void_p * n)(*[t.data_ptr() for t in self.tensors])
        types = (ctypes.c_int * n)(*[_TYPES.get(t.dtype, -1) for t in self.tensors])
        numel = (ctypes.c_int64 * n)(*[t.numel() for t in self.tensors])
        group = (ctypes.c_int * n)(*groups)
        nbytes = int(self.lib.mv_clip_workspace_bytes(numel, n, self.n_groups))
        _need(nbytes > 0, "mv_clip_workspace_bytes")
        # memory of the stream that fills it: other memory may still be in use by what the current stream has yet to run
        with torch.cuda.stream(stream):          # (None: the current one)
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        handle = ctypes.c_void_p()
        self.dev = self.workspace.get_device()
        self.streams = {_raw_stream(self.dev, None)}      # that the allocator knows of
        _check(self.lib.mv_clip_create(ctypes.byref(handle), self._stream(stream), ptrs, types, numel, group, n, self.n_groups,
                                       self.workspace.data_ptr(), nbytes), "mv_clip_create")
        self.handle = handle

    def close(self):
        if getattr(self, "handle", None):
            self.lib.mv_clip_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self, stream: Optional[torch.cuda.Stream]):
        """The stream of a call, of which the allocator is told once: the memory is not given away before that stream is through."""
        raw = _raw_stream(self.dev, stream)
        if raw not in self.streams:
            used = stream if stream is not None else torch.cuda.current_stream(self.dev)
            for t in (self.workspace, *self.tensors):
                t.record_stream(used)
            self.streams.add(raw)
        return raw

    def mv_clip_status(self, stream: Optional[torch.cuda.Stream] = None):
        """Waits for the stream; MvError(MV_ERR_TIMEOUT) if a wait inside a call has run out since the last time it was asked."""
        _check(self.lib.mv_clip_status(self.handle, self._stream(stream)), "mv_clip_status")

    def mv_clip_set_polls(self, polls: int):
        _check(self.lib.mv_clip_set_polls(self.handle, int(polls)), "mv_clip_set_polls")

    def mv_clip_norm(self, norms, stream: Optional[torch.cuda.Stream] = None):
        n, _ = _vector(norms, self.n_groups, _FLOAT, self.dev, "mv_clip_norm")
        _check(self.lib.mv_clip_norm(self.handle, self._stream(stream), n), "mv_clip_norm")

    def mv_clip_scale(self, max_norm: float, norms=None, stream: Optional[torch.cuda.Stream] = None):
        n, _ = _vector(norms, self.n_groups, _FLOAT, self.dev, "mv_clip_scale")
        _check(self.lib.mv_clip_scale(self.handle, self._stream(stream), float(max_norm), n), "mv_clip_scale")

    def mv_clip_pack(self, max_norm: float, rows, norms=None, stream: Optional[torch.cuda.Stream] = None):
        n, _ = _vector(norms, self.n_groups, _FLOAT, self.dev, "mv_clip_pack")
        r, _, G, d, ld, dev = _matrix(rows, _FLOAT, "mv_clip_pack")
        _need(G == self.n_groups and d >= self.longest and dev == self.dev, "mv_clip_pack")
        _check(self.lib.mv_clip_pack(self.handle, self._stream(stream), float(max_norm), r, ld, n), "mv_clip_pack")


class MvContext:
    """A context bound to the current CUDA stream and to a workspace tensor it keeps alive."""

    def __init__(self, N: int, d: int, K: int, device="cuda", stream: Optional[torch.cuda.Stream] = None,
                 mode: int = MV_MODE_AUTO, debug: bool = False):
        self.lib = load_debug() if debug else load()
        self.N, self.d, self.K = int(N), int(d), int(K)
        nbytes = workspace_bytes(N, d, K)
        if nbytes == 0:
            raise MvError(MV_ERR_INVALID_ARG, "mv_workspace_bytes")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.workspace.device)
        handle = ctypes.c_void_p()
        _check(self.lib.mv_create(ctypes.byref(handle), ctypes.c_void_p(self.stream.cuda_stream),
                                  _ptr(self.workspace), nbytes), "mv_create")
        self.handle = handle
        self.set_mode(mode)

    def close(self):
        if getattr(self, "handle", None):
            self.lib.mv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_tail_kernel(self, enable: int):
        """Whole steps as two kernels (streaming pass + one persistent tail kernel): 0 never, 1 where it pays
        (the default), 2 wherever it can run."""
        _check(self.lib.mv_set_tail_kernel(self.handle, int(enable)), "mv_set_tail_kernel")

    def set_mode(self, mode: int):
        _check(self.lib.mv_set_mode(self.handle, int(mode)), "mv_set_mode")

    # the calls below mirror include/mv_sparse.h one to one
    def mv_sparse_step(self, grads, err, out_idx, out_val, K: Optional[int] = None):
        N, d = grads.shape
        _check(self.lib.mv_sparse_step(self.handle, _ptr(grads), _ptr(err), N, d, K or self.K,
                                       _ptr(out_idx), _ptr(out_val)), "mv_sparse_step")

    def mv_vote(self, grads, err, worker_idx=None, worker_bits=None, votes=None, thresh=None, K: Optional[int] = None):
        N, d = grads.shape
        _check(self.lib.mv_vote(self.handle, _ptr(grads), _ptr(err), N, d, K or self.K, _ptr(worker_idx),
                                _ptr(worker_bits), _ptr(votes), _ptr(thresh)), "mv_vote")

    def mv_select(self, votes, N: int, out_idx, mask_bits=None, K: Optional[int] = None):
        _check(self.lib.mv_select(self.handle, _ptr(votes), N, votes.numel(), K or self.K, _ptr(out_idx),
                                  _ptr(mask_bits)), "mv_select")

    def mv_aggregate(self, acc, idx, out_val):
        N, d = acc.shape
        _check(self.lib.mv_aggregate(self.handle, _ptr(acc), N, d, idx.numel(), _ptr(idx), _ptr(out_val)),
               "mv_aggregate")

    def mv_ad_step(self, grads, err, prev_bits, K_ad: int, out_idx, out_val, add_bits=None, drop_bits=None,
                   msum=None, K: Optional[int] = None):
        N, d = grads.shape
        _check(self.lib.mv_ad_step(self.handle, _ptr(grads), _ptr(err), _ptr(prev_bits), N, d, K or self.K, int(K_ad),
                                   _ptr(out_idx), _ptr(out_val), _ptr(add_bits), _ptr(drop_bits), _ptr(msum)),
               "mv_ad_step")

    def mv_topk_union_step(self, grads, err, out_idx, out_val, count, K: Optional[int] = None):
        """SSGD-top-K: out_idx / out_val [capacity >= min(d, N K)], count: int32 [1] on the device."""
        N, d = grads.shape
        _check(self.lib.mv_topk_union_step(self.handle, _ptr(grads), _ptr(err), N, d, K or self.K, _ptr(out_idx),
                                           _ptr(out_val), out_idx.numel(), _ptr(count)), "mv_topk_union_step")

    def mv_select_rs(self, votes, N: int, seed: int, draw: int, out_idx, mask_bits=None, K: Optional[int] = None):
        _check(self.lib.mv_select_rs(self.handle, _ptr(votes), int(N), votes.numel(), int(K or self.K), int(seed), int(draw),
                                     _ptr(out_idx), _ptr(mask_bits)), "mv_select_rs")

    def mv_rs_step(self, grads, err, seed: int, draw: int, out_idx, out_val, K: Optional[int] = None):
        N, d = grads.shape
        _check(self.lib.mv_rs_step(self.handle, _ptr(grads), _ptr(err), int(N), int(d), int(K or self.K), int(seed), int(draw),
                                   _ptr(out_idx), _ptr(out_val)), "mv_rs_step")

    def mv_aggregate_partial(self, acc, idx, out_sum):
        N, d = acc.shape
        _check(self.lib.mv_aggregate_partial(self.handle, _ptr(acc), N, d, idx.numel(), _ptr(idx), _ptr(out_sum)),
               "mv_aggregate_partial")

    def mv_finish_mean(self, total, N_total: int, out_val):
        _check(self.lib.mv_finish_mean(ctypes.c_void_p(self.stream.cuda_stream), _ptr(total), total.numel(), int(N_total),
                                       _ptr(out_val)), "mv_finish_mean")

    def mv_sparse_step_host(self, h_grads, h_out_idx, h_out_val, d_grads, d_err, d_out_idx, d_out_val,
                            K: Optional[int] = None):
        N, d = h_grads.shape
        _check(self.lib.mv_sparse_step_host(self.handle, _ptr(h_grads), N, d, K or self.K, _ptr(h_out_idx),
                                            _ptr(h_out_val), _ptr(d_grads), _ptr(d_err), _ptr(d_out_idx),
                                            _ptr(d_out_val)), "mv_sparse_step_host")

    def read_diag(self, N: Optional[int] = None) -> torch.Tensor:
        N = N or self.N
        out = torch.zeros((N, 4), dtype=torch.int64)
        buf = (ctypes.c_uint32 * (4 * N))()
        _check(self.lib.mv_read_diag(self.handle, N, buf), "mv_read_diag")
        out.copy_(torch.tensor(list(buf), dtype=torch.int64).view(N, 4))
        return out

    def set_kernel_timing(self, every: int):
        """0: off; n >= 1: time the streaming pass on every n-th step."""
        _check(self.lib.mv_set_kernel_timing(self.handle, int(every)), "mv_set_kernel_timing")

    def read_kernel_timing(self):
        """(total milliseconds, launches covered) of the streaming pass since the last read."""
        ms, cnt = ctypes.c_float(), ctypes.c_int()
        _check(self.lib.mv_read_kernel_timing(self.handle, ctypes.byref(ms), ctypes.byref(cnt)),
               "mv_read_kernel_timing")
        return float(ms.value), int(cnt.value)

    def set_phase_timing(self, enable: int):
        """0: off; 1: an event after every launch; 100 + i: only the start and the end of launch i."""
        _check(self.lib.mv_set_phase_timing(self.handle, int(enable)), "mv_set_phase_timing")

    def read_phase_times(self):
        """Milliseconds per kernel launch of the last call, in launch order."""
        buf = (ctypes.c_float * 47)()
        cnt = ctypes.c_int()
        _check(self.lib.mv_read_phase_times(self.handle, buf, 47, ctypes.byref(cnt)), "mv_read_phase_times")
        return [float(buf[i]) for i in range(cnt.value)]

    def last_launches(self) -> int:
        return int(self.lib.mv_last_launches(self.handle))

    def fallback_count(self) -> int:
        """Worker selections that took the full-row route since the context's first call."""
        total = ctypes.c_uint32()
        _check(self.lib.mv_fallback_count(self.handle, ctypes.byref(total)), "mv_fallback_count")
        return int(total.value)

    def debug_status(self) -> int:
        """MV_DBG_* bits collected by a checked build since the last read (always 0 in a normal build)."""
        word = ctypes.c_int()
        _check(self.lib.mv_debug_status(self.handle, ctypes.byref(word)), "mv_debug_status")
        return int(word.value)
