"""The operators around the decision step, over torch tensors.

``_step.so`` checks the arguments and calls the C ABI of
``include/asymspec_step.h``; the work is done by the HIP kernels of
``csrc/step/`` on the tensors' device and its current stream.  Every tensor is
on that device; index tensors are int32.  The calls may be captured into a HIP
graph.  No gradient passes through them: a tensor that a call writes to must not
require one (under torch.no_grad() it may), and has a new version afterwards.
The new outputs of a call share one allocation, which the last of them that is
kept frees (clone() one that is to be kept without the others, or give `out`).
There is no fallback: if a library is missing, every call raises.
"""

from __future__ import annotations

import os

import torch

import paper_2608_26004_amd as _asp

__all__ = ["shape_logits", "draw_tokens", "commit_tokens", "plan_slots"]

BIND_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "_step.so")
_step = None
# the handle of a device's current stream
_raw_stream = torch._C._cuda_getCurrentRawStream


def _bind():
    """Load (once) the binding, behind libasymspec.so."""
    global _step
    if _step is None:
        import importlib.util
        _asp.load_library()
        if not os.path.exists(BIND_PATH):
            raise ImportError(f"{BIND_PATH} is missing: build it with `python -m paper_2608_26004_amd.build`")
        spec = importlib.util.spec_from_file_location("paper_2608_26004_amd._step", BIND_PATH)
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
        mod.set_error(_asp.AsymSpecError)
        _step = mod
    return _step


def _stream(x):
    i = x.get_device() if isinstance(x, torch.Tensor) else -1      # (the binding refuses what is none)
    return _raw_stream(i) if i >= 0 else 0


def shape_logits(logits, history=None, lengths=None, prompt_lengths=None, draft_tokens=None,
                 repetition=None, frequency=None, presence=None, bias_ids=None, bias_values=None,
                 mask=None, mask_index=None, id_map=None, out=None):
    """Penalties for repeated tokens, biases and grammar masks on logit rows.

    logits: [B, R, V] bfloat16 or float32, the last dimension contiguous (rows
    may be strided views, such as one position of a [B, K+1, V] buffer);
    history: [B, L] tokens of each request (L below 2^20), lengths: [B] how many of them,
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
    out: None shapes `logits` in place, else a tensor of the same shape and dtype
    in other memory.
    With c occurrences among the output tokens and drafts ahead of the row, a
    logit v becomes, in fp32: v / repetition (v > 0) or v * repetition if the
    token occurs there or in the prompt; minus frequency * c and minus presence
    if c > 0; plus its bias; -inf if masked.  Returns the shaped tensor."""
    return (_step or _bind()).shape_logits(logits, history, lengths, prompt_lengths, draft_tokens, repetition,
                                           frequency, presence, bias_ids, bias_values, mask, mask_index, id_map,
                                           out, _stream(logits))


def draw_tokens(logits, temperature, uniforms, out=None):
    """The drafter's own choice from each row: (token [N] int32, q(token) [N]
    float32).

    logits: [N, V] bfloat16 or float32, rows contiguous (strided views such as
    one position of a [B, K+1, V] buffer are fine); temperature: [N] float32
    (<= 0: the lowest index of the largest logit, q = 1); uniforms: [N] float32 in
    [0, 1), for an inverse-CDF draw from softmax(logits / temperature), summed in
    fp64; out: (token, q) tensors to write, views such as draft_tokens[:, i]
    among them, which must overlap no other tensor of the call.  Logits of -inf or
    not a number have no weight, as those whose weight beside the row's largest is
    below fp64's smallest number; uniforms of 1 and more give the last token with
    weight, those below 0 or not a number count as 0; a row without any weight gives
    token 0 with q = 0.  The workspace is memory of the call's own, from
    torch's allocator: a Workspace holds what fuse_verify knows again, and a
    captured call must not work in memory that a later one replaces."""
    return (_step or _bind()).draw_tokens(logits, temperature, uniforms, out, _stream(logits))


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
    finished may be the inputs, and otherwise what is written (history among it) must
    overlap no other tensor of the call."""
    return (_step or _bind()).commit_tokens(accept_len, next_token, draft_tokens, history, lengths, finished,
                                            stop_tokens, max_lengths, out, _stream(history))


def plan_slots(lengths, new_tokens, block_table, n_blocks, free_ring, free_state, block_size,
               width=None, total=None, release=None, out=None):
    """Cache blocks and slots for the requests' next tokens.

    Request b of at most 4096 has lengths[b] tokens in its cache and gets new_tokens[b] more
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
    out: the tensors to write, in that order.  What is written (block_table and
    free_ring among it) must overlap no other tensor of the call."""
    return (_step or _bind()).plan_slots(lengths, new_tokens, block_table, n_blocks, free_ring, free_state,
                                         block_size, width or 0, total or 0, release, out, _stream(block_table))
