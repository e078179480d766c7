"""The operators around the decision step, over torch tensors.

Thin marshalling for ``include/asymspec_step.h``: arguments are checked here,
the work is done by the HIP kernels of ``csrc/step/`` on the tensors' device
and its current stream.  Every tensor is on that device; index tensors are
int32.  The calls may be captured into a HIP graph.
"""

from __future__ import annotations

import contextlib
import ctypes

import paper_2608_26004_amd as _asp

__all__ = ["shape_logits", "draw_tokens", "commit_tokens", "plan_slots"]


class _Shape(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("logits", "out")]
                + [(n, ctypes.c_int64) for n in ("request_stride", "row_stride", "out_request_stride",
                                                 "out_row_stride")]
                + [(n, ctypes.c_void_p) for n in ("history", "lengths", "prompt_lengths", "draft_tokens")]
                + [("draft_stride", ctypes.c_int64)]
                + [(n, ctypes.c_void_p) for n in ("id_map", "repetition", "frequency", "presence", "bias_ids",
                                                  "bias_values", "mask", "mask_index")]
                + [(n, ctypes.c_int32) for n in ("dtype", "B", "R", "V", "max_history", "D", "n_ids", "n_bias",
                                                 "n_masks")])


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = _asp.load_library()
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t
        lib.asymspec_shape_logits.argtypes = [ctypes.POINTER(_Shape), vp]
        lib.asymspec_shape_logits.restype = i32
        lib.asymspec_draw_workspace_size.argtypes = [i32, i32, i32]
        lib.asymspec_draw_workspace_size.restype = sz
        lib.asymspec_draw_tokens.argtypes = [vp, i32, i32, i32, i64, vp, vp, i64, vp, i64, vp, i64, vp, sz, vp]
        lib.asymspec_draw_tokens.restype = i32
        lib.asymspec_commit_tokens.argtypes = [vp, vp, vp, i64, vp, i32, vp, vp, vp, i32, vp, i32, i32,
                                               vp, vp, vp, vp, vp]
        lib.asymspec_commit_tokens.restype = i32
        lib.asymspec_plan_slots.argtypes = [vp, vp, vp, vp, i32, vp, vp, i32, vp, i32, i32, i32, i32,
                                            vp, vp, vp, vp, vp, vp]
        lib.asymspec_plan_slots.restype = i32
        _lib = lib
    return _lib


def _on(dev):
    """The tensors' device current, and its stream."""
    import torch
    if dev.type != "cuda":
        raise ValueError(f"tensors must be on the GPU, got {dev}")
    guard = contextlib.nullcontext() if dev.index == torch.cuda.current_device() else torch.cuda.device(dev)
    return guard, torch.cuda.current_stream(dev).cuda_stream


def _need(name, x, dtype, shape, dev, contiguous=True):
    """Address of tensor x (0 for None), which has to be as said."""
    if x is None:
        return None
    if x.dtype != dtype or x.shape != shape or x.device != dev:
        raise ValueError(f"{name} must be {str(dtype).replace('torch.', '')} {list(shape)} on {dev}, got "
                         f"{str(x.dtype).replace('torch.', '')} {list(x.shape)} on {x.device}")
    if contiguous and not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return x.data_ptr()


def _logit_type(x):
    import torch
    if x.dtype == torch.bfloat16:
        return _asp.BF16
    if x.dtype == torch.float32:
        return _asp.FP32
    raise TypeError(f"logits must be bfloat16 or float32, got {x.dtype}")


def _check(st):
    if st != _asp.OK:
        raise _asp.AsymSpecError(st, _asp.status_string(st))


def shape_logits(logits, history=None, lengths=None, prompt_lengths=None, draft_tokens=None,
                 repetition=None, frequency=None, presence=None, bias_ids=None, bias_values=None,
                 mask=None, mask_index=None, id_map=None, out=None):
    """Penalties for repeated tokens, biases and grammar masks on logit rows.

    logits: [B, R, V] bfloat16 or float32, the last dimension contiguous (rows
    may be strided views, such as one position of a [B, K+1, V] buffer);
    history: [B, L] tokens of each request, lengths: [B] how many of them,
    prompt_lengths: [B] how many of those are its prompt (seen, but not counted);
    draft_tokens: [B, D]: row r follows the history and the first D - (R - 1) + r
    drafts (with R = K + 1 and D = K: row r the first r, as fuse_verify's rows;
    with R = 1: all of them), requests may be strided;
    repetition, frequency, presence: [B] float32 or None;
    bias_ids, bias_values: [B, n] (an id out of range is an unused entry; of
    several entries with one id the last counts);
    mask: [M, ceil(V / 32)] int32, bit x % 32 of word x // 32 set where token x is
    allowed, mask_index: [B, R] its row for each logit row (out of range: none);
    id_map: [n_ids]: history and drafts are ids of another vocabulary, whose id x
    is id_map[x] here (out of range: none);
    out: None shapes `logits` in place, else a tensor of the same shape and dtype.
    With c occurrences among the output tokens and drafts ahead of the row, a
    logit v becomes, in fp32: v / repetition (v > 0) or v * repetition if the
    token occurs there or in the prompt; minus frequency * c and minus presence
    if c > 0; plus its bias; -inf if masked.  Returns the shaped tensor."""
    import torch
    i32, f32 = torch.int32, torch.float32
    dt = _logit_type(logits)
    if logits.dim() != 3:
        raise ValueError("logits must be [B, R, V]")
    B, R, V = logits.shape
    dev = logits.device
    if out is None:
        out = logits
    elif out.dtype != logits.dtype or out.shape != logits.shape or out.device != dev:
        raise ValueError("out must have the logits' shape, dtype and device")
    sb, sr, sv = logits.stride()
    ob, orow, ov = out.stride()
    if V > 1 and (sv != 1 or ov != 1):
        raise ValueError("rows of logits must be contiguous")
    L = D = n_bias = n_masks = n_ids = dstride = 0
    if history is not None:
        if history.dim() != 2 or lengths is None:
            raise ValueError("history must be [B, L] with lengths [B]")
        L = history.shape[1]
    elif lengths is not None or prompt_lengths is not None:
        raise ValueError("lengths belong to a history")
    if draft_tokens is not None:
        if draft_tokens.dim() != 2 or (draft_tokens.shape[1] > 1 and draft_tokens.stride(1) != 1):
            raise ValueError("draft_tokens must be [B, D], its rows contiguous")
        D, dstride = draft_tokens.shape[1], draft_tokens.stride(0)
        if D < R - 1:
            raise ValueError("rows behind R - 1 drafts need as many draft_tokens")
    if (bias_ids is None) != (bias_values is None):
        raise ValueError("bias_ids and bias_values belong together")
    if bias_ids is not None:
        if bias_ids.dim() != 2:
            raise ValueError("bias_ids must be [B, n]")
        n_bias = bias_ids.shape[1]
    if (mask is None) != (mask_index is None):
        raise ValueError("mask and mask_index belong together")
    if mask is not None:
        if mask.dim() != 2:
            raise ValueError("mask must be [M, ceil(V / 32)]")
        n_masks = mask.shape[0]
    if id_map is not None:
        n_ids = id_map.numel()
    per = (B,)
    s = _Shape(logits.data_ptr(), out.data_ptr(), sb, sr, ob, orow,
               _need("history", history, i32, (B, L), dev),
               _need("lengths", lengths, i32, per, dev),
               _need("prompt_lengths", prompt_lengths, i32, per, dev),
               _need("draft_tokens", draft_tokens, i32, (B, D), dev, False) if D else None, dstride,
               _need("id_map", id_map, i32, (n_ids,), dev),
               _need("repetition", repetition, f32, per, dev),
               _need("frequency", frequency, f32, per, dev),
               _need("presence", presence, f32, per, dev),
               _need("bias_ids", bias_ids, i32, (B, n_bias), dev) if n_bias else None,
               _need("bias_values", bias_values, f32, (B, n_bias), dev) if n_bias else None,
               _need("mask", mask, i32, (n_masks, (V + 31) // 32), dev) if n_masks else None,
               _need("mask_index", mask_index, i32, (B, R), dev) if n_masks else None,
               dt, B, R, V, L, D, n_ids, n_bias, n_masks)
    if L == 0:
        s.history = s.lengths = s.prompt_lengths = None
    guard, stream = _on(dev)
    with guard:
        _check(_library().asymspec_shape_logits(ctypes.byref(s), stream))
    return out


def draw_tokens(logits, temperature, uniforms, out=None, workspace=None):
    """The drafter's own choice from each row: (token [N] int32, q(token) [N]
    float32).

    logits: [N, V] bfloat16 or float32, rows contiguous (strided views such as
    one position of a [B, K+1, V] buffer are fine); temperature: [N] float32
    (<= 0: the lowest index of the largest logit, q = 1); uniforms: [N] float32 in
    [0, 1), for an inverse-CDF draw from softmax(logits / temperature), summed in
    fp64; out: (token, q) tensors to write, views such as draft_tokens[:, i]
    among them; workspace: a Workspace (by default memory of the call's own).
    Logits of -inf or not a number have no weight; a row without any gives
    token 0 with q = 0."""
    import torch
    i32, f32 = torch.int32, torch.float32
    dt = _logit_type(logits)
    if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be [N, V], its rows contiguous")
    N, V = logits.shape
    dev = logits.device
    guard, stream = _on(dev)
    if out is None:
        out = torch.empty(N, dtype=i32, device=dev), torch.empty(N, dtype=f32, device=dev)
    token, prob = out
    t = _need("temperature", temperature, f32, (N,), dev)
    u = _need("uniforms", uniforms, f32, (N,), dev, False)
    tp = _need("token", token, i32, (N,), dev, False)
    pp = _need("q", prob, f32, (N,), dev, False)
    with guard:
        lib = _library()
        nbytes = lib.asymspec_draw_workspace_size(N, V, dt)
        if nbytes == 0:
            raise _asp.AsymSpecError(_asp.E_ARG, "invalid shape")
        ws = (torch.empty(nbytes, dtype=torch.uint8, device=dev) if workspace is None
              else workspace.get(nbytes, dev))
        _check(lib.asymspec_draw_tokens(logits.data_ptr(), dt, N, V, logits.stride(0), t, u, uniforms.stride(0),
                                        tp, token.stride(0), pp, prob.stride(0), ws.data_ptr(), ws.numel(),
                                        stream))
    return out


def commit_tokens(accept_len, next_token, draft_tokens, history, lengths, finished=None, stop_tokens=None,
                  max_lengths=None, out=None):
    """Joins a step's accepted drafts and emitted tokens to the histories.

    accept_len, next_token: [B], as fuse_verify returns them (-1: the request's
    decision did not complete; it commits nothing); draft_tokens: [B, K], requests
    may be strided; history: [B, L], written in place at lengths [B]; finished: [B]
    int32 (nonzero commits nothing) or None; stop_tokens: [n] or None (a request
    ends with the first of them); max_lengths: [B] or None (L).
    Returns (lengths [B], finished [B], tokens [B, K+1] committed, then -1,
    counts [B]), all int32 and new unless given as `out`; out's lengths and
    finished may be the inputs."""
    import torch
    i32 = torch.int32
    if draft_tokens.dim() != 2 or (draft_tokens.shape[1] > 1 and draft_tokens.stride(1) != 1):
        raise ValueError("draft_tokens must be [B, K], its rows contiguous")
    if history.dim() != 2:
        raise ValueError("history must be [B, L]")
    B, K = draft_tokens.shape
    L = history.shape[1]
    dev = history.device
    n_stop = 0 if stop_tokens is None else stop_tokens.numel()
    per = (B,)
    guard, stream = _on(dev)
    if out is None:
        out = (torch.empty(B, dtype=i32, device=dev), torch.empty(B, dtype=i32, device=dev),
               torch.empty(B, K + 1, dtype=i32, device=dev), torch.empty(B, dtype=i32, device=dev))
    args = (_need("accept_len", accept_len, i32, per, dev), _need("next_token", next_token, i32, per, dev),
            _need("draft_tokens", draft_tokens, i32, (B, K), dev, False) if K else None, draft_tokens.stride(0),
            _need("history", history, i32, (B, L), dev), L, _need("lengths", lengths, i32, per, dev),
            _need("finished", finished, i32, per, dev),
            _need("stop_tokens", stop_tokens, i32, (n_stop,), dev) if n_stop else None, n_stop,
            _need("max_lengths", max_lengths, i32, per, dev), B, K,
            _need("out[0]", out[0], i32, per, dev), _need("out[1]", out[1], i32, per, dev),
            _need("out[2]", out[2], i32, (B, K + 1), dev), _need("out[3]", out[3], i32, per, dev))
    with guard:
        _check(_library().asymspec_commit_tokens(*args, stream))
    return tuple(out)


def plan_slots(lengths, new_tokens, block_table, n_blocks, free_ring, free_state, block_size,
               width=None, total=None, release=None, out=None):
    """Cache blocks and slots for the requests' next tokens.

    Request b has lengths[b] tokens in its cache and gets new_tokens[b] more
    ([B], or None: `width` each); blocks it lacks are taken from the front of
    free_ring, blocks beyond its need (all with release[b]) go back to the end.
    block_table: [B, max_blocks] and free_ring: [pool] are changed in place;
    n_blocks: [B] blocks held and free_state: [2] (front, count of the ring) are
    not: their new values are returned.  Exactly one of
      width: slots is [B, width], row b the slots of request b's tokens, or
      total: slots is [total], the requests' tokens one behind the other.
    Returns (slots int64, -1 where there is no token; short [B] int32, 1 for a
    request that did not get its blocks, which keeps what it has and has no
    slots; n_blocks [B]; free_state [2]), and with `total` also starts [B + 1].
    out: the tensors to write, in that order."""
    import torch
    i32, i64 = torch.int32, torch.int64
    if (width is None) == (total is None):
        raise ValueError("give either width or total")
    if block_table.dim() != 2 or free_ring.dim() != 1:
        raise ValueError("block_table must be [B, max_blocks] and free_ring [pool]")
    if new_tokens is None and width is None:
        raise ValueError("total needs new_tokens")
    if (width if total is None else total) < 1:
        raise ValueError("width or total must be at least 1")
    B, top = block_table.shape
    N = free_ring.shape[0]
    dev = block_table.device
    per = (B,)
    guard, stream = _on(dev)
    places = (B, width) if width else (total,)
    if out is None:
        out = (torch.empty(places, dtype=i64, device=dev), torch.empty(B, dtype=i32, device=dev),
               torch.empty(B, dtype=i32, device=dev), torch.empty(2, dtype=i32, device=dev))
        if total:
            out += (torch.empty(B + 1, dtype=i32, device=dev),)
    args = (_need("lengths", lengths, i32, per, dev), _need("new_tokens", new_tokens, i32, per, dev),
            _need("release", release, i32, per, dev), _need("block_table", block_table, i32, (B, top), dev), top,
            _need("n_blocks", n_blocks, i32, per, dev), _need("free_ring", free_ring, i32, (N,), dev), N,
            _need("free_state", free_state, i32, (2,), dev), block_size, B, width or 0, total or 0,
            _need("out[0]", out[0], i64, places, dev),
            _need("out[4]", out[4], i32, (B + 1,), dev) if total else None,
            _need("out[1]", out[1], i32, per, dev), _need("out[2]", out[2], i32, per, dev),
            _need("out[3]", out[3], i32, (2,), dev))
    with guard:
        _check(_library().asymspec_plan_slots(*args, stream))
    return tuple(out)
