"""The operators of a paged cache of keys and values in 8 or 4 bits, over torch
tensors.

``plan_slots`` says where a step's tokens go; ``rotate_heads`` turns their queries
and keys by their positions, ``write_cache`` puts the keys and values into the
slots, ``attend_cache`` answers a step's rows from the cache, and ``read_cache``
gives positions back as dense tensors.

A cache is a tuple (keys, key_scales, values, value_scales) of contiguous uint8
tensors: codes [blocks, heads, block_size, dim * bits / 8], and for each 32
channels a scale byte s that stands for 2^(s - 127), [blocks, heads, block_size,
dim / 32].  With 8 bits a code is an e4m3 number, with 4 an e2m1 number, the even
channel in the low half of a byte.  Slot s of ``plan_slots`` is place s %
block_size of block s // block_size, of every head.

``_step.so`` checks the arguments and calls the C ABI of
``include/asymspec_cache.h``; what ``step.py`` says about streams, graphs, new
outputs, gradients and missing libraries holds here too.
"""

from __future__ import annotations

import math

import torch

from . import step as _s

__all__ = ["new_cache", "rotary_frequencies", "rotate_heads", "write_cache", "read_cache", "attend_cache"]


def new_cache(blocks: int, heads: int, block_size: int, dim: int, bits: int = 4, device=None):
    """An empty cache: its four tensors, all zero.

    dim: a multiple of 32, at most 256 (attend_cache: 64, 96, 128, 192 or 256); bits: 8 or 4.
    blocks * heads * block_size must be below 2^31."""
    if bits not in (4, 8):
        raise ValueError(f"bits must be 8 or 4, got {bits}")
    if dim % 32 or not 32 <= dim <= 256:
        raise ValueError(f"dim must be a multiple of 32 up to 256, got {dim}")
    if min(blocks, heads, block_size) < 1 or blocks * heads * block_size >= 1 << 31:
        raise ValueError(f"blocks * heads * block_size must be in [1, 2^31), got {blocks} * {heads} * {block_size}")
    device = torch.device("cuda") if device is None else device
    return tuple(torch.zeros(blocks, heads, block_size, n, dtype=torch.uint8, device=device)
                 for n in (dim * bits // 8, dim // 32) * 2)


def rotary_frequencies(channels: int, base: float = 10000.0, stretch: float = 1.0, kind: str = "linear",
                       context: int = 4096, fast: float = 32.0, slow: float = 1.0, device=None):
    """Radians a position of each of channels / 2 pairs, [channels / 2] float64:
    base^(-2i / channels), stretched for contexts `stretch` times as long as trained:

      "linear"  every frequency over `stretch`
      "base"    a larger base, base * stretch^(channels / (channels - 2)): the
                slowest pair is over `stretch`, the fastest stays
      "ramp"    pairs that turn `fast` times and more in `context` positions stay,
                those that turn `slow` times and less are over `stretch`, and between
                them the share that stays falls evenly with the pair's index (from
                index 0 on at least, and to index channels - 1 at most)
    A ramp goes with rotate_heads' magnitude = 0.1 * log(stretch) + 1."""
    if channels < 2 or channels % 2:
        raise ValueError(f"channels must be even and at least 2, got {channels}")
    if not (base > 1 and stretch > 0):
        raise ValueError("base must be above 1 and stretch above 0")
    i = torch.arange(channels // 2, dtype=torch.float64)
    if kind == "base":
        if channels < 4:
            raise ValueError("a stretched base needs at least 4 channels")
        f = (base * stretch ** (channels / (channels - 2))) ** (-2 * i / channels)
    elif kind == "linear":
        f = base ** (-2 * i / channels) / stretch
    elif kind == "ramp":
        if not (fast > slow > 0 and context > 0):
            raise ValueError("fast must be above slow, and slow and context above 0")
        f = base ** (-2 * i / channels)
        # the index of a pair that turns so often in the context, also where there is none
        at = [channels * math.log(context / (2 * math.pi * turns)) / (2 * math.log(base)) for turns in (fast, slow)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), channels - 1)
        stay = (1 - ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)) * (i < at[1])
        f = f * stay + f / stretch * (1 - stay)
    else:
        raise ValueError(f'kind must be "linear", "base" or "ramp", got {kind!r}')
    return f.to(torch.device("cuda") if device is None else device)


def rotate_heads(q, k, positions, frequencies, interleaved: bool = False, magnitude: float = 1.0, out=None):
    """Rotary positions on the queries and keys of a step's tokens.

    q: [B, R, heads, dim], k: [B, R, its heads, dim] or None, bfloat16 or float32;
    the channels of a head are contiguous, the rest may be strided (parts of one
    projection); positions: [B] int32, token r of request b then stands at
    positions[b] + r (the lengths that plan_slots takes), or [B, R]; negative ones turn
    back; frequencies: [n] float64, radians a position (rotary_frequencies).
    Pair i is channels (i, i + n), or (2i, 2i + 1) where interleaved, and (x, y)
    becomes magnitude * (x cos - y sin, x sin + y cos) of position * frequencies[i]:
    angles in 64 bits, the rest in fp32, rounded once.  Channels from 2n on stay.
    out: (q, k) tensors to write, which may be the inputs themselves (in place) and
    overlap no other tensor of the call.  Returns (q, k), or q where k is None."""
    r = (_s._step or _s._bind()).rotate_heads(q, k, positions, frequencies, interleaved, magnitude,
                                              (out,) if k is None and isinstance(out, torch.Tensor) else out,
                                              _s._stream(q))
    return r if k is not None else r[0]


def write_cache(k, v, slots, cache):
    """Keys and values of new tokens into their slots of a cache, quantised.

    k, v: [B, R, heads, dim] with slots [B, R], or [tokens, heads, dim] with slots
    [tokens], bfloat16 or float32, the channels of a head contiguous; slots: int64, as
    plan_slots returns them (out of range, such as -1: the token is left out; each slot
    at most once).  For each 32 channels the scale is the smallest power of two (2^-100 at
    least) with which the largest magnitude is at most 448 (8 bits) or 6 (4 bits); each
    code is the nearest, ties to even.  Where one of the 32 is not finite (or beyond
    1.75 * 2^127 with 8 bits, 1.5 * 2^127 with 4), all of them read as not a number.  Returns
    the cache, changed in place."""
    return (_s._step or _s._bind()).write_cache(k, v, slots, cache, _s._stream(k))


_TYPES = {torch.bfloat16: 0, torch.float32: 1}


def read_cache(cache, block_table, lengths, width: int, first=None, dtype=torch.bfloat16, out=None):
    """Positions first[b] .. first[b] + width (first: [B] int32, or None: 0) of every
    request as dense tensors (keys, values), [B, width, heads, dim] in bfloat16 or
    float32; both hold a code times its scale exactly.

    block_table: [B, max_blocks] int32, as plan_slots keeps it; lengths: [B] int32, the
    positions that each request has.  A position outside [0, lengths[b]), or without a
    block, is zero.  out: (keys, values) to write, which overlap no other tensor of the
    call."""
    if dtype not in _TYPES:
        raise TypeError(f"dtype must be torch.bfloat16 or torch.float32, got {dtype}")
    return (_s._step or _s._bind()).read_cache(cache, block_table, lengths, width, first, _TYPES[dtype], out,
                                               _s._stream(block_table))


def attend_cache(q, cache, block_table, lengths, new_tokens=None, scale=None, window: int = 0, return_lse: bool = False,
                 out=None):
    """Attention of a step's rows over the cache.

    q: [B, R, heads, dim] bfloat16 or float32 (R at most 64, B at most 4096), the channels
    of a head contiguous; heads a multiple of the cache's, of which head h reads head
    h // (heads / the cache's); block_table: [B, max_blocks], lengths and new_tokens: [B]
    int32, as plan_slots takes them: row r of request b stands at position
    lengths[b] + r and sees the positions up to its own (with a window > 0 the last
    `window` of those), as far as they have a block.  scale: of the products (None:
    dim^-0.5).
    Returns softmax(scale * q . keys) . values, [B, R, heads, dim] in q's type, and with
    return_lse also the logarithm of the softmax's sum, [B, R, heads] float32, with which
    answers from several caches can be joined.  Rows that see nothing and rows from
    new_tokens[b] on are 0, their lse -inf.  What a row does not see has no effect on it,
    whatever is there.  out: the tensor, or with return_lse the two, to write, which
    overlap no other tensor of the call.  The workspace is memory kept for the calls of
    each stream, and on hipStreamPerThread of each thread; a captured call has its own, in
    its graph's memory.  A stream of other making (torch.cuda.ExternalStream) is not to be
    destroyed before its calls have ended: its handle may come back as another stream's."""
    return (_s._step or _s._bind()).attend_cache(q, cache, block_table, lengths, new_tokens, scale, window, return_lse,
                                                 out, _s._stream(q))
