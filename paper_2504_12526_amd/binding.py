"""ctypes binding of libmom.so: same names as the C ABI, argument marshalling only.

Tensors are torch tensors used purely as device (or pinned host) buffers; every step of the
path runs in the library's HIP kernels.  There is no fallback: if the library has not been
built (`python -m paper_2504_12526_amd.build` or `__graft_entry__.build()`), importing the
symbols raises.
"""
import ctypes
import math
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmom.so")

SYMBOLS = ("mom_status_string", "mom_mlp_workspace_bytes", "mom_mlp_prefill", "mom_mlp_prefill_events",
           "mom_mlp_pipelined_workspace_bytes", "mom_mlp_prefill_pipelined",
           "mom_lmhead_last", "mom_mlp_last", "mom_kv_offload", "mom_kv_reload",
           "mom_init", "mom_debug_force_gemm_form", "mom_debug_force_short_form", "mom_debug_force_rect_form", "mom_debug_force_block",
           "mom_mlp_prefill_static",
           "mom_debug_mfma_probe",
           "mom_mx_block_bytes", "mom_mx_kv_append", "mom_mx_kv_read", "mom_mx_attention_workspace_bytes", "mom_mx_attention",
           "mom_mx_quantize", "mom_mx_matvec", "mom_mx_gateup")

MOM_STATIC_WORKSPACE_BYTES = 64 << 20
MOM_MX_MAX_ROWS = 16

(MOM_OK, MOM_ERR_NULL, MOM_ERR_SHAPE, MOM_ERR_ALIGN, MOM_ERR_ALIAS, MOM_ERR_WORKSPACE, MOM_ERR_HIP,
 MOM_ERR_HOST) = range(8)

_lib = None


class MomError(RuntimeError):
    def __init__(self, status, what):
        self.status = int(status)
        super().__init__(f"{what}: status {status} ({status_string(status)})")


def lib():
    """The loaded C-ABI library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build the HIP library first (python -m paper_2504_12526_amd.build)")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
        L.mom_status_string.restype = ctypes.c_char_p
        L.mom_status_string.argtypes = [ctypes.c_int]
        L.mom_mlp_workspace_bytes.restype = sz
        L.mom_mlp_workspace_bytes.argtypes = [i64, i64, i64, i64]
        L.mom_mlp_prefill.restype = ctypes.c_int
        L.mom_mlp_prefill.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, vp, vp, sz, vp]
        L.mom_mlp_prefill_events.restype = ctypes.c_int
        L.mom_mlp_prefill_events.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, vp, vp, sz, vp,
                                             ctypes.POINTER(vp), i64]
        L.mom_mlp_pipelined_workspace_bytes.restype = sz
        L.mom_mlp_pipelined_workspace_bytes.argtypes = [i64, i64, i64, i64]
        L.mom_mlp_prefill_pipelined.restype = ctypes.c_int
        L.mom_mlp_prefill_pipelined.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, vp, vp, sz, vp, vp,
                                                ctypes.POINTER(vp), i64]
        L.mom_lmhead_last.restype = ctypes.c_int
        L.mom_lmhead_last.argtypes = [vp, vp, i64, vp, i64, vp]
        L.mom_kv_offload.restype = ctypes.c_int
        L.mom_kv_offload.argtypes = [vp, vp, vp, vp, sz, vp, vp, vp]
        L.mom_mlp_last.restype = ctypes.c_int
        L.mom_mlp_last.argtypes = [vp, vp, vp, vp, i64, i64, vp, vp, sz, vp]
        L.mom_kv_reload.restype = ctypes.c_int
        L.mom_kv_reload.argtypes = [vp, vp, vp, vp, sz, vp]
        L.mom_mlp_prefill_static.restype = ctypes.c_int
        L.mom_mlp_prefill_static.argtypes = [vp, vp, vp, vp, i64, i64, i64, i64, vp, vp]
        L.mom_init.restype = ctypes.c_int
        L.mom_init.argtypes = []
        L.mom_debug_force_gemm_form.restype = ctypes.c_int
        L.mom_debug_force_gemm_form.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_int]
        L.mom_debug_force_short_form.restype = ctypes.c_int
        L.mom_debug_force_short_form.argtypes = [ctypes.c_int, ctypes.c_int]
        L.mom_debug_force_rect_form.restype = ctypes.c_int
        L.mom_debug_force_rect_form.argtypes = [ctypes.c_int, ctypes.c_int]
        L.mom_debug_force_block.restype = ctypes.c_int
        L.mom_debug_force_block.argtypes = [ctypes.c_int]
        L.mom_debug_mfma_probe.restype = ctypes.c_int
        L.mom_debug_mfma_probe.argtypes = [vp, sz, vp, sz, i64, ctypes.c_int, ctypes.c_int, vp, vp]
        L.mom_mx_block_bytes.restype = sz
        L.mom_mx_block_bytes.argtypes = [i64, i64]
        L.mom_mx_kv_append.restype = ctypes.c_int
        L.mom_mx_kv_append.argtypes = [vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, ctypes.c_int, i64, i64, i64, i64, vp, vp, i64, i64, vp]
        L.mom_mx_kv_read.restype = ctypes.c_int
        L.mom_mx_kv_read.argtypes = [vp, i64, i64, vp, i64, i64, i64, vp, vp, vp]
        L.mom_mx_attention_workspace_bytes.restype = sz
        L.mom_mx_attention_workspace_bytes.argtypes = [i64] * 6
        L.mom_mx_attention.restype = ctypes.c_int
        L.mom_mx_attention.argtypes = [vp, i64, vp, i64, i64, i64, i64, i64, vp, i64, i64, vp, i64, vp, i64, ctypes.c_float, i64,
                                       vp, vp, vp, sz, vp]
        L.mom_mx_quantize.restype = ctypes.c_int
        L.mom_mx_quantize.argtypes = [vp, i64, i64, vp, vp, vp]
        L.mom_mx_matvec.restype = ctypes.c_int
        L.mom_mx_matvec.argtypes = [vp, i64, vp, vp, i64, i64, vp, ctypes.c_int, vp, vp]
        L.mom_mx_gateup.restype = ctypes.c_int
        L.mom_mx_gateup.argtypes = [vp, i64, vp, vp, vp, vp, i64, i64, vp, vp]
        _lib = L
    return _lib


def status_string(status):
    return lib().mom_status_string(int(status)).decode()


def _ptr(t):
    return None if t is None else t.data_ptr()


# torch's own questions for the current device and its current stream's handle, which have no public names; None where torch has no such function.
_current_device, _current_handle = (getattr(torch._C, name, None) for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"))


def _stream(stream):
    """Handle of a stream, None: the current one of the current device (asked by its number where torch answers that: a torch Stream object
    takes 4 us to make, which is more than a small kernel)."""
    if stream is None:
        if _current_device is not None and _current_handle is not None:
            return _current_handle(_current_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream


def _nbytes(t):
    return t.numel() * t.element_size()


def mom_mlp_workspace_bytes(S, H, I, mini_seq):
    return int(lib().mom_mlp_workspace_bytes(S, H, I, mini_seq))


def mom_mlp_prefill(x, W_gate, W_up, W_down, mini_seq, out, workspace, stream=None, check=True):
    """x [S,H], W_gate/W_up [I,H], W_down [H,I], out [S,H] bf16 device tensors; workspace any
    device tensor of at least mom_mlp_workspace_bytes bytes.  Enqueues on `stream`."""
    S, H = x.shape
    I = W_gate.shape[0]
    rc = lib().mom_mlp_prefill(_ptr(x), _ptr(W_gate), _ptr(W_up), _ptr(W_down), S, H, I, int(mini_seq),
                               _ptr(out), _ptr(workspace), _nbytes(workspace), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mlp_prefill")
    return rc


def mom_mlp_prefill_static(x, W_gate, W_up, W_down, mini_seq, out, stream=None, check=True):
    """mom_mlp_prefill with the library's own static workspace (at most MOM_STATIC_WORKSPACE_BYTES)."""
    S, H = x.shape
    I = W_gate.shape[0]
    rc = lib().mom_mlp_prefill_static(_ptr(x), _ptr(W_gate), _ptr(W_up), _ptr(W_down), S, H, I, int(mini_seq),
                                      _ptr(out), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mlp_prefill_static")
    return rc


def mom_mlp_prefill_events(x, W_gate, W_up, W_down, mini_seq, out, workspace, events, stream=None):
    """As mom_mlp_prefill, recording `events` (list of torch.cuda.Event(enable_timing=True),
    already recorded once so that their handles exist) around every kernel."""
    S, H = x.shape
    I = W_gate.shape[0]
    arr = (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    rc = lib().mom_mlp_prefill_events(_ptr(x), _ptr(W_gate), _ptr(W_up), _ptr(W_down), S, H, I, int(mini_seq),
                                      _ptr(out), _ptr(workspace), _nbytes(workspace), _stream(stream),
                                      arr, len(events))
    if rc != MOM_OK:
        raise MomError(rc, "mom_mlp_prefill_events")
    return rc


def mom_mlp_pipelined_workspace_bytes(S, H, I, mini_seq):
    return int(lib().mom_mlp_pipelined_workspace_bytes(int(S), int(H), int(I), int(mini_seq)))


def mom_mlp_prefill_pipelined(x, W_gate, W_up, W_down, mini_seq, out, workspace, stream, stream2, events,
                              check=True):
    """As mom_mlp_prefill with a workspace of mom_mlp_pipelined_workspace_bytes, two mini-sequences at a time; enqueues on `stream`.
    stream2 is not used; events: at least 5 torch.cuda.Event whose handles exist, checked and not used."""
    S, H = x.shape
    I = W_gate.shape[0]
    arr = None if events is None else (ctypes.c_void_p * len(events))(*[e.cuda_event for e in events])
    rc = lib().mom_mlp_prefill_pipelined(_ptr(x), _ptr(W_gate), _ptr(W_up), _ptr(W_down), S, H, I, int(mini_seq),
                                         _ptr(out), _ptr(workspace), _nbytes(workspace), _stream(stream),
                                         _stream(stream2), arr, 0 if events is None else len(events))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mlp_prefill_pipelined")
    return rc


def mom_lmhead_last(x_last, W_lm, logits, stream=None, check=True):
    """x_last [H] bf16, W_lm [V,H] bf16, logits [V] fp32 device tensors."""
    V, H = W_lm.shape
    rc = lib().mom_lmhead_last(_ptr(x_last), _ptr(W_lm), V, _ptr(logits), H, _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_lmhead_last")
    return rc


def mom_init():
    rc = lib().mom_init()
    if rc != MOM_OK:
        raise MomError(rc, "mom_init")
    return rc


def mom_debug_force_gemm_form(tile_edge=0, ring_slots=0, tile_width=0):
    """Testing aid: force the tile form of the matrix-core kernels; (0, 0, 0) = the library's choice."""
    rc = lib().mom_debug_force_gemm_form(int(tile_edge), int(ring_slots), int(tile_width))
    if rc != MOM_OK:
        raise MomError(rc, "mom_debug_force_gemm_form")
    return rc


def mom_debug_force_short_form(token_rows=0, weight_rows=0):
    """Testing aid: force a tile form for few token rows; (0, 0) = the library's choice."""
    rc = lib().mom_debug_force_short_form(int(token_rows), int(weight_rows))
    if rc != MOM_OK:
        raise MomError(rc, "mom_debug_force_short_form")
    return rc


def mom_debug_force_rect_form(token_rows=0, weight_rows=0):
    """Testing aid: force a form of the rectangular tiles; (0, 0) = the library's choice."""
    rc = lib().mom_debug_force_rect_form(int(token_rows), int(weight_rows))
    if rc != MOM_OK:
        raise MomError(rc, "mom_debug_force_rect_form")
    return rc


def mom_debug_force_block(token_rows=0):
    """Testing aid: whole blocks of 16 or 32 token rows in one launch, where the layer fits; 0 = the library's choice."""
    rc = lib().mom_debug_force_block(int(token_rows))
    if rc != MOM_OK:
        raise MomError(rc, "mom_debug_force_block")
    return rc


def mom_debug_mfma_probe(a, b, iters, workgroups, sink, stream=None, order=0):
    """Measurement aid: register-only MFMA loop on operand fragments taken from bf16 tensors a and b
    (order 0: the kernels' back-to-back pairs, 1: K-half by K-half); returns the flop of the launch
    (time it with events on the stream)."""
    if sink.numel() < workgroups * 256 or sink.dtype != torch.float32:
        raise ValueError("sink must hold workgroups*256 float32")
    rc = lib().mom_debug_mfma_probe(_ptr(a), _nbytes(a), _ptr(b), _nbytes(b), int(iters), int(workgroups),
                                    int(order), _ptr(sink), _stream(stream))
    if rc != MOM_OK:
        raise MomError(rc, "mom_debug_mfma_probe")
    return float(workgroups) * 4 * int(iters) * 128 * 16384


def mom_kv_offload(k, v, pinned_host, stream, producer_stream=None, order_event=None, done_event=None,
                   check=True):
    """Copy device k, v (same byte size) to the pinned host tensor (k then v) on `stream`.
    With order_event the copy is ordered after the work already enqueued on producer_stream
    (None = the default stream); done_event is recorded after both copies."""
    nb = _nbytes(k)
    if _nbytes(v) != nb or _nbytes(pinned_host) < 2 * nb:
        raise ValueError("k and v must have equal byte size and pinned_host must hold both")
    rc = lib().mom_kv_offload(_ptr(k), _ptr(v), _ptr(pinned_host), _stream(stream), nb,
                              None if producer_stream is None else _stream(producer_stream),
                              None if order_event is None else ctypes.c_void_p(order_event.cuda_event),
                              None if done_event is None else ctypes.c_void_p(done_event.cuda_event))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_kv_offload")
    return rc


def mom_mlp_last(x_last, W_gate, W_up, W_down, out_last, workspace, stream=None, check=True):
    """x_last [H], W_gate/W_up [I,H], W_down [H,I], out_last [H] bf16 device tensors; workspace >= I*2 bytes."""
    I, H = W_gate.shape
    rc = lib().mom_mlp_last(_ptr(x_last), _ptr(W_gate), _ptr(W_up), _ptr(W_down), H, I, _ptr(out_last),
                            _ptr(workspace), _nbytes(workspace), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mlp_last")
    return rc


def mom_kv_reload(pinned_host, k, v, stream, done_event=None, check=True):
    """Copy k then v back from the pinned host tensor into the device tensors on `stream`."""
    nb = _nbytes(k)
    if _nbytes(v) != nb or _nbytes(pinned_host) < 2 * nb:
        raise ValueError("k and v must have equal byte size and pinned_host must hold both")
    rc = lib().mom_kv_reload(_ptr(pinned_host), _ptr(k), _ptr(v), _stream(stream), nb,
                             None if done_event is None else ctypes.c_void_p(done_event.cuda_event))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_kv_reload")
    return rc


def _dense(name, t, dtype, shape=None):
    if t.dtype != dtype or (shape is not None and t.shape != shape) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {dtype} tensor" + ("" if shape is None else f" of shape {tuple(shape)}"))
    return t


def _tokens(name, t, width=None):
    """[T, heads, head_dim] bf16 whose tokens may lie apart; the elements between two of them."""
    T, heads, d = t.shape
    apart, between, within = t.stride()
    if t.dtype != torch.bfloat16 or (heads > 1 and between != d) or within != 1 or (width is not None and (T, d) != width):
        raise ValueError(f"{name} must be a bfloat16 tensor [tokens, heads, head_dim] whose heads are contiguous")
    return apart if T > 1 else heads * d


_block_bytes = {}


def mom_mx_block_bytes(head_dim, page_tokens):
    n = _block_bytes.get((head_dim, page_tokens))
    if n is None:
        n = _block_bytes[head_dim, page_tokens] = int(lib().mom_mx_block_bytes(int(head_dim), int(page_tokens)))
    return n


def _cache(cache, page_tokens, head_dim):
    block = mom_mx_block_bytes(head_dim, page_tokens)
    if cache.dtype != torch.uint8 or cache.dim() != 3 or block == 0 or cache.shape[2] != block or not cache.is_contiguous():
        raise ValueError("cache must be a contiguous uint8 tensor [pages, kv_heads, mom_mx_block_bytes(head_dim, page_tokens)]")
    return cache.shape[0], cache.shape[1]


def mom_mx_kv_append(k, v, slots, cache, page_tokens, positions=None, inv_freq=None, interleaved=False, q=None, q_out=None,
                     stream=None, check=True):
    """k, v [T, kv_heads, head_dim] bf16 (tokens may lie apart, as slices of one projection do) into the uint8 cache
    [pages, kv_heads, mom_mx_block_bytes] at slots [T] int64.  positions [T] int32 and inv_freq [rot_dim / 2] fp32 rotate the keys
    and, where given, the queries q [T, q_heads, head_dim] into q_out."""
    T, kv_heads, d = k.shape
    pages, heads = _cache(cache, page_tokens, d)
    if v.shape != k.shape or heads != kv_heads:
        raise ValueError("k and v must have the same shape and the cache their heads")
    if (positions is None) != (inv_freq is None) or (q is None) != (q_out is None):
        raise ValueError("positions and inv_freq, q and q_out come together")
    strides = _tokens("k", k), _tokens("v", v)
    _dense("slots", slots, torch.int64, (T,))
    rot = 0
    if inv_freq is not None:
        _dense("positions", positions, torch.int32, (T,))
        rot = 2 * _dense("inv_freq", inv_freq, torch.float32).numel()
    q_stride = q_heads = 0
    if q is not None:
        q_stride, q_heads = _tokens("q", q, (T, d)), q.shape[1]
        _dense("q_out", q_out, torch.bfloat16, q.shape)
    rc = lib().mom_mx_kv_append(_ptr(q), q_stride, _ptr(k), strides[0], _ptr(v), strides[1], _ptr(slots), _ptr(positions if rot else None),
                                _ptr(inv_freq if rot else None), rot, int(bool(interleaved)), T, q_heads, kv_heads, d, _ptr(q_out), _ptr(cache), pages,
                                int(page_tokens), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mx_kv_append")
    return rc


def mom_mx_kv_read(cache, page_tokens, slots, k, v, stream=None, check=True):
    """The tokens at slots [T] int64 as k, v [T, kv_heads, head_dim] bf16."""
    T, kv_heads, d = k.shape
    pages, heads = _cache(cache, page_tokens, d)
    _dense("slots", slots, torch.int64, (T,))
    _dense("k", k, torch.bfloat16, (T, heads, d))
    _dense("v", v, torch.bfloat16, (T, heads, d))
    rc = lib().mom_mx_kv_read(_ptr(cache), pages, int(page_tokens), _ptr(slots), T, kv_heads, d, _ptr(k), _ptr(v), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mx_kv_read")
    return rc


def mom_mx_attention_workspace_bytes(T, B, q_heads, kv_heads, head_dim, max_kv):
    return int(lib().mom_mx_attention_workspace_bytes(int(T), int(B), int(q_heads), int(kv_heads), int(head_dim), int(max_kv)))


def mom_mx_attention(q, cache, page_tokens, page_table, kv_lens, max_kv, out, workspace, q_starts=None, scale=None, window=0, lse=None,
                     stream=None, check=True):
    """q [T, q_heads, head_dim] bf16 (tokens may lie apart) of B sequences over the cache: page_table [B, n] int32 (rows may lie
    apart), kv_lens [B] int32, q_starts [B + 1] int32 or None (T / B tokens each), scale None: 1 / sqrt(head_dim).  out like q, dense;
    lse [T, q_heads] fp32 or None; workspace any device tensor of at least mom_mx_attention_workspace_bytes bytes, or None where that is 0."""
    T, q_heads, d = q.shape
    pages, kv_heads = _cache(cache, page_tokens, d)
    B, each = page_table.shape
    if page_table.dtype != torch.int32 or (each > 1 and page_table.stride(1) != 1) or (B > 1 and page_table.stride(0) < each):
        raise ValueError("page_table must be an int32 tensor [B, n] with contiguous rows")
    # rows that lie apart are passed as one that is as long as their distance, and what lies between them stays out of reach through max_kv
    table_stride = page_table.stride(0) if B > 1 else each
    _dense("kv_lens", kv_lens, torch.int32, (B,))
    if q_starts is not None:
        _dense("q_starts", q_starts, torch.int32, (B + 1,))
    _dense("out", out, torch.bfloat16, q.shape)
    if lse is not None:
        _dense("lse", lse, torch.float32, (T, q_heads))
    rc = lib().mom_mx_attention(_ptr(q), _tokens("q", q), _ptr(q_starts), T, B, q_heads, kv_heads, d, _ptr(cache), pages, int(page_tokens),
                                _ptr(page_table), table_stride, _ptr(kv_lens), min(int(max_kv), each * int(page_tokens)),
                                1.0 / math.sqrt(d) if scale is None else float(scale), int(window), _ptr(out), _ptr(lse),
                                _ptr(workspace), 0 if workspace is None else _nbytes(workspace), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mx_attention")
    return rc


def mom_mx_quantize(w, codes, scales, stream=None, check=True):
    """w [N, K] bf16 into codes [N, K / 2] and scales [N, K / 32] (uint8)."""
    N, K = w.shape
    _dense("w", w, torch.bfloat16)
    _dense("codes", codes, torch.uint8, (N, K // 2))
    _dense("scales", scales, torch.uint8, (N, K // 32))
    rc = lib().mom_mx_quantize(_ptr(w), N, K, _ptr(codes), _ptr(scales), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mx_quantize")
    return rc


def mom_mx_matvec(x, codes, scales, out, residual=None, stream=None, check=True):
    """x [M, K] bf16 times the weight in four bits, codes [N, K / 2] and scales [N, K / 32]: out [M, N] fp32, or bf16 with
    residual [M, N] bf16 added where given."""
    M, K = x.shape
    N = codes.shape[0]
    _dense("x", x, torch.bfloat16)
    _dense("codes", codes, torch.uint8, (N, K // 2))
    _dense("scales", scales, torch.uint8, (N, K // 32))
    _dense("out", out, torch.float32 if out.dtype == torch.float32 else torch.bfloat16, (M, N))
    if residual is not None:
        _dense("residual", residual, torch.bfloat16, (M, N))
    rc = lib().mom_mx_matvec(_ptr(x), M, _ptr(codes), _ptr(scales), N, K, _ptr(out), int(out.dtype == torch.float32), _ptr(residual), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mx_matvec")
    return rc


def mom_mx_gateup(x, gate_codes, gate_scales, up_codes, up_scales, out, stream=None, check=True):
    """silu(x W_gate^T) * (x W_up^T) for x [M, K] bf16 and two weights [N, K] in four bits: out [M, N] bf16."""
    M, K = x.shape
    N = gate_codes.shape[0]
    _dense("x", x, torch.bfloat16)
    for name, c, s in (("gate", gate_codes, gate_scales), ("up", up_codes, up_scales)):
        _dense(name + "_codes", c, torch.uint8, (N, K // 2))
        _dense(name + "_scales", s, torch.uint8, (N, K // 32))
    _dense("out", out, torch.bfloat16, (M, N))
    rc = lib().mom_mx_gateup(_ptr(x), M, _ptr(gate_codes), _ptr(gate_scales), _ptr(up_codes), _ptr(up_scales), N, K, _ptr(out), _stream(stream))
    if check and rc != MOM_OK:
        raise MomError(rc, "mom_mx_gateup")
    return rc
