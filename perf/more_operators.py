"""The operators of a paged cache of keys and values held in 8 or 4 bits.

``plan_slots`` places the next tokens of every request in the blocks of a paged
cache; these calls fill the slots and answer from them:

  rotate   ``rotate_heads``   rotary positions on the queries and keys of new tokens
  write    ``write_cache``    keys and values into their slots, 8 or 4 bits each
  read     ``read_cache``     positions of every request back as dense tensors
  attend   ``attend_cache``   attention of a step's rows over the cache

A cache is (keys, key_scales, values, value_scales), uint8: data [blocks, heads,
block_size, dim * bits / 8] and a scale for each 32 channels, [blocks, heads,
block_size, dim / 32].  A scale byte s stands for 2^(s - 127): the smallest power
of two, 2^-100 at least, with which the 32 values' largest magnitude is at most
448 (8 bits: e4m3) or 6 (4 bits: e2m1, the even channel in the low half of a
byte); values are rounded to the nearest, ties to even.

``run`` computes them in plain torch, or, with ``own``, through the package.
"""

import math

import torch

own = False

_ROTATE = dict(op="rotate", B=8, R=3, H=32, Hkv=8, D=128, rot=128, dtype="bf16", pairs="half", far=8192, stretch=1.0)
_WRITE = dict(op="write", B=8, R=3, Hkv=8, D=128, bits=4, bs=16, dtype="bf16", skip=0.1)
_READ = dict(op="read", B=8, L=2048, Hkv=8, D=128, bits=4, bs=16, dtype="bf16")
_ATTEND = dict(op="attend", B=8, R=3, H=32, Hkv=8, D=128, L=8192, bits=4, bs=16, dtype="bf16", window=0, fewer=False)


def _case(base, **kw):
    c = dict(base)
    c.update(kw)
    return c


def listed():
    return [
        # a few agents' rows of a step, far into their contexts: pure latency
        _case(_ROTATE, name="rotate_b8", far=131072),
        # prompts of many requests, one behind the other
        _case(_ROTATE, name="rotate_prompts", B=16384, R=1, far=32768),
        # half of each head, neighbouring channels paired, frequencies stretched
        # for a long context, in fp32
        _case(_ROTATE, name="rotate_part_fp32", B=96, R=6, H=16, Hkv=16, D=96, rot=48, dtype="fp32",
              pairs="neighbours", far=131072, stretch=8.0),
        # the throughput batch's rows of a step, some requests without a slot
        _case(_WRITE, name="write8_b128", B=128, R=7, bits=8),
        # prompts written, and read back for an attention that takes dense tensors
        _case(_WRITE, name="write4_prompts", B=16, R=4096, skip=0.0),
        # the context of a few requests as dense tensors; a ragged one in fp32
        _case(_READ, name="read4_b16", B=16, L=8192),
        _case(_READ, name="read8_ragged_fp32", B=3, L=700, Hkv=5, D=96, bits=8, bs=24, dtype="fp32"),
        # one interactive request's next token: pure latency
        _case(_ATTEND, name="attend_one", B=1, R=1, L=2048),
        # the paper's operating point over an agent's context
        _case(_ATTEND, name="attend4_b8", B=8, R=3, L=16384),
        # a drafter's single tokens over full contexts
        _case(_ATTEND, name="attend4_long", B=2, R=1, L=262144, bs=64),
        # the throughput batch's verification, some requests with fewer rows
        _case(_ATTEND, name="attend8_b128", B=128, R=7, L=8192, bits=8, fewer=True),
        # a window in fp32, a head of keys for each of queries
        _case(_ATTEND, name="attend4_window_fp32", B=32, R=5, H=16, Hkv=16, D=64, L=5000, bs=24, dtype="fp32",
              window=1024),
    ]


_DIMS = (64, 96, 128, 192, 256)
_MOST_TOKENS = 16384 * 40 * 128          # values of the largest listed rotation
_MOST_WRITE = 16 * 4096 * 8 * 128        # of keys written
_MOST_READ = 16 * 8192 * 8 * 128         # of keys read
_MOST_ATTEND = 128 * 8192 * 8 * 128      # of keys attended to
_MOST_ROWS = 128 * 7 * 32 * 8192         # of probabilities


def _logint(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rotate", "write", "read", "attend", "attend", "attend"])
    Hkv, group = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
    D, dtype = rng.choice(_DIMS), rng.choice(["bf16", "bf16", "fp32"])
    bits, bs = rng.choice([4, 4, 8]), rng.choice([1, 16, 16, 24, 32, 64, 128])
    if op == "rotate":
        c = _case(_ROTATE, B=_logint(rng, 1, 16384), R=rng.choice([1, rng.randint(1, 9)]), H=Hkv * group, Hkv=Hkv, D=D,
                  rot=rng.choice([D, D, D // 2, D // 4]), dtype=dtype, pairs=rng.choice(["half", "neighbours"]),
                  far=_logint(rng, 1024, 1 << 20), stretch=rng.choice([1.0, 4.0]))
        most = _MOST_TOKENS // (c["R"] * (c["H"] + Hkv) * D) // (1 if dtype == "bf16" else 2)
    elif op == "write":
        c = _case(_WRITE, B=_logint(rng, 1, 512), R=rng.choice([rng.randint(1, 9), _logint(rng, 10, 4096)]), Hkv=Hkv,
                  D=D, bits=bits, bs=bs, dtype=dtype, skip=rng.choice([0.0, 0.1, 0.5]))
        most = _MOST_WRITE // (c["R"] * Hkv * D) // (1 if dtype == "bf16" else 2)
    elif op == "read":
        c = _case(_READ, B=_logint(rng, 1, 128), L=_logint(rng, 1, 32768), Hkv=Hkv, D=D, bits=bits, bs=bs, dtype=dtype)
        most = _MOST_READ // (c["L"] * Hkv * D) // (1 if dtype == "bf16" else 2)
    else:
        c = _case(_ATTEND, B=_logint(rng, 1, 256), R=rng.choice([1, 3, rng.randint(1, 9)]), H=Hkv * group, Hkv=Hkv, D=D,
                  L=_logint(rng, 1, 131072), bits=bits, bs=bs, dtype=dtype, fewer=rng.random() < 0.3,
                  window=rng.choice([0, 0, 0, _logint(rng, 1, 8192)]))
        most = min(_MOST_ATTEND // (2 * c["L"] * Hkv * D), _MOST_ROWS // (2 * c["R"] * c["H"] * c["L"]))
    if most < 1:
        c["L" if "L" in c else "R"] //= 64
        most = 1
    for k in ("L", "R"):
        if k in c:
            c[k] = max(1, c[k])
    c["B"] = max(1, min(c["B"], most))
    return c


# ------------------------------------------------------------------ inputs --
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _dt(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _frequencies(rot, stretch):
    """Radians a position of each pair of channels; the slow half stretched."""
    f = 10000.0 ** (-torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / rot)
    return torch.where(f < 0.05, f / stretch, f)


def _heads(shape, g, dt):
    """Keys or queries: some channels of a head are several times the others."""
    x = torch.randn(shape, device="cuda", generator=g)
    x *= torch.exp(0.7 * torch.randn(shape[-2:], device="cuda", generator=g))
    return x.to(dt)


def _empty_cache(blocks, c):
    shape = (blocks, c["Hkv"], c["bs"])
    return tuple(torch.zeros(shape + (n,), dtype=torch.uint8, device="cuda")
                 for n in (c["D"] * c["bits"] // 8, c["D"] // 32) * 2)


def _filled_cache(blocks, c, g):
    cache = _empty_cache(blocks, c)
    spread = torch.exp(0.7 * torch.randn(c["Hkv"], 1, c["D"], device="cuda", generator=g))
    n = max(1, (1 << 26) // (c["Hkv"] * c["bs"] * c["D"]))
    for lo in range(0, blocks, n):
        for part, wide in ((0, spread), (2, 1.0)):
            x = torch.randn((min(n, blocks - lo), c["Hkv"], c["bs"], c["D"]), device="cuda", generator=g)
            data, scales = _quantise(x * wide, c["bits"])
            cache[part][lo:lo + n] = data
            cache[part + 1][lo:lo + n] = scales
    return cache


def _pages(lengths, blocks, c, g):
    """Block tables of requests that hold `lengths` positions, blocks in no order."""
    need = (lengths + c["bs"] - 1) // c["bs"]
    top = int(need.max())
    ids = torch.randperm(blocks, device="cuda", generator=g)[:int(need.sum())]
    j = torch.arange(top, device="cuda")
    at = (need.cumsum(0) - need)[:, None] + j
    return torch.where(j < need[:, None], ids[at.clamp_max(len(ids) - 1)], -1).int()


def _lengths(c, g):
    """Between half of the longest and the longest, one request with the longest."""
    n = (c["L"] * (0.5 + 0.5 * torch.rand(c["B"], device="cuda", generator=g))).ceil().long()
    n[0] = c["L"]
    return n


def _prepare_rotate(c, seed):
    g, B, R, H, Hkv, D = _gen(seed), c["B"], c["R"], c["H"], c["Hkv"], c["D"]
    qkv = _heads((B, R, H + 2 * Hkv, D), g, _dt(c))       # one projection's output, as a model has it
    return dict(op="rotate", q=qkv[:, :, :H], k=qkv[:, :, H:H + Hkv],
                positions=torch.randint(0, c["far"], (B,), device="cuda", generator=g).int(),
                frequencies=_frequencies(c["rot"], c["stretch"]), interleaved=c["pairs"] == "neighbours",
                magnitude=1.0 if c["stretch"] == 1.0 else 0.1 * math.log(c["stretch"]) + 1.0)


def _prepare_write(c, seed):
    g, B, R, Hkv, D = _gen(seed), c["B"], c["R"], c["Hkv"], c["D"]
    kv = _heads((B, R, 2 * Hkv, D), g, _dt(c))
    # a step's rows stand anywhere in their requests, a prompt's at the start
    ahead = 0 if R > 9 else 2 * c["bs"] + R
    lengths = (ahead * torch.rand(B, device="cuda", generator=g)).long()
    blocks = B * ((ahead + R + c["bs"] - 1) // c["bs"]) + 1
    table = _pages(lengths + R, blocks, c, g)
    p = lengths[:, None] + torch.arange(R, device="cuda")
    slots = table.gather(1, p // c["bs"]).long() * c["bs"] + p % c["bs"]
    slots[1:][torch.rand(B - 1, device="cuda", generator=g) < c["skip"]] = -1
    return dict(op="write", k=kv[:, :, :Hkv], v=kv[:, :, Hkv:], slots=slots, cache=_empty_cache(blocks, c), table=table,
                lengths=(lengths + R).int(), first=lengths.int(), width=R, dtype=_dt(c), bits=c["bits"])


def _prepare_read(c, seed):
    g = _gen(seed)
    lengths = _lengths(c, g)
    blocks = int(((lengths + c["bs"] - 1) // c["bs"]).sum()) + 1
    return dict(op="read", cache=_filled_cache(blocks, c, g), table=_pages(lengths, blocks, c, g), lengths=lengths.int(),
                first=None, width=c["L"], dtype=_dt(c))


def _prepare_attend(c, seed):
    g, B, R, H, Hkv, D = _gen(seed), c["B"], c["R"], c["H"], c["Hkv"], c["D"]
    n = _lengths(c, g)
    blocks = int(((n + R + c["bs"] - 1) // c["bs"]).sum()) + 1
    new = torch.full((B,), R, device="cuda")
    if c["fewer"]:
        new = torch.where(torch.rand(B, device="cuda", generator=g) < 0.2,
                          (R * torch.rand(B, device="cuda", generator=g)).long(), new)
        new[0] = R
    q = (1.5 * torch.randn((B, R, H + 2 * Hkv, D), device="cuda", generator=g)).to(_dt(c))[:, :, :H]
    return dict(op="attend", q=q, cache=_filled_cache(blocks, c, g), table=_pages(n + R, blocks, c, g),
                lengths=n.int(), new_tokens=new.int() if c["fewer"] else None, scale=1.0 / math.sqrt(D),
                window=c["window"])


def prepare(case, seed):
    return {"rotate": _prepare_rotate, "write": _prepare_write, "read": _prepare_read,
            "attend": _prepare_attend}[case["op"]](case, seed)


# ------------------------------------------------------------- plain forms --
def _power(e):
    """2^e of whole numbers in fp32's normal range, exactly."""
    return ((e + 127) << 23).int().view(torch.float32)


def _quantise(x, bits):
    """(data, scales) of values [..., D] in fp32."""
    x = x.unflatten(-1, (-1, 32))
    m, e = torch.frexp(x.abs().amax(-1))                 # m in [0.5, 1)
    e = (e - (9 if bits == 8 else 3) + (m > (0.875 if bits == 8 else 0.75))).clamp_min(-100)
    x = x * _power(-e)[..., None]
    scales = (e + 127).to(torch.uint8)
    if bits == 8:
        return x.to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2), scales
    a = x.abs()
    # 0 0.5 1 1.5 2 3 4 6; halfway goes to the even code
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = (code + 8 * (x < 0)).to(torch.uint8).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], scales


def _values(data, scales):
    """Their values in fp32."""
    if data.shape[-1] == 32 * scales.shape[-1]:
        x = data.view(torch.float8_e4m3fn).float()
    else:
        code = torch.stack((data & 15, data >> 4), -1).flatten(-2).int()
        low, high = code & 1, (code >> 1) & 3
        x = torch.where(high == 0, 0.5 * low, (1.0 + 0.5 * low) * _power(high - 1))
        x = torch.where(code >= 8, -x, x)
    return (x.unflatten(-1, (-1, 32)) * _power(scales.int() - 127)[..., None]).flatten(-2)


def _of_positions(part, s):
    """Keys (0) or values (2) of every request's positions, [B, Hkv, positions, D]."""
    at = s["table"].long().clamp_min(0)
    x = _values(s["cache"][part][at], s["cache"][part + 1][at])
    return x.transpose(1, 2).flatten(2, 3)


def _plain_rotate(s):
    q, k, f = s["q"], s["k"], s["frequencies"]
    n = len(f)
    p = s["positions"].double()[:, None] + torch.arange(q.shape[1], device=q.device)
    angle = (p[..., None] * f)[:, :, None]
    cos, sin = (s["magnitude"] * angle.cos()).float(), (s["magnitude"] * angle.sin()).float()

    def turned(x):
        y = x.float()
        r = y[..., :2 * n]
        a, b = (r[..., 0::2], r[..., 1::2]) if s["interleaved"] else (r[..., :n], r[..., n:])
        a, b = a * cos - b * sin, a * sin + b * cos
        r = torch.stack((a, b), -1).flatten(-2) if s["interleaved"] else torch.cat((a, b), -1)
        return torch.cat((r, y[..., 2 * n:]), -1).to(x.dtype)

    return turned(q), turned(k)


def _plain_read(s):
    p = torch.arange(s["width"], device=s["table"].device)[None]
    if s["first"] is not None:
        p = p + s["first"].long()[:, None]
    ok = (p < s["lengths"][:, None])[:, :, None, None]
    got = []
    for part in (0, 2):
        x = _of_positions(part, s).transpose(1, 2)
        x = x.gather(1, p.expand(len(x), -1).clamp_max(x.shape[1] - 1)[..., None, None].expand(-1, -1, *x.shape[2:]))
        got.append(torch.where(ok, x, 0.0).to(s["dtype"]))
    return tuple(got)


def _plain_write(s):
    bs, slots = s["cache"][0].shape[2], s["slots"].flatten()
    ok = slots >= 0
    to = slots[ok]
    for part, x in ((0, s["k"]), (2, s["v"])):
        for t, y in zip(s["cache"][part:part + 2], _quantise(x.flatten(0, 1)[ok].float(), s["bits"])):
            t[to // bs, :, to % bs] = y


def _plain_attend(s):
    q, window = s["q"].float(), s["window"]
    B, R, H, D = q.shape
    k = _of_positions(0, s)
    Hkv, n = k.shape[1], k.shape[2]
    q = q.view(B, R, Hkv, -1, D).permute(0, 2, 3, 1, 4).flatten(2, 3)        # [B, Hkv, group * R, D]
    x = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    del k
    x = x.view(B, Hkv, -1, R, n)
    at = s["lengths"].long()[:, None] + torch.arange(R, device=q.device)
    p = torch.arange(n, device=q.device)
    seen = p <= at[..., None]
    if window:
        seen = seen & (p > at[..., None] - window)
    if s["new_tokens"] is not None:
        seen = seen & (torch.arange(R, device=q.device) < s["new_tokens"][:, None])[..., None]
    x = torch.where(seen[:, None, None], x, -math.inf)
    m = x.amax(-1, keepdim=True)
    w = torch.exp(x - torch.where(m > -math.inf, m, 0.0))
    total = w.sum(-1, keepdim=True)
    y = torch.matmul(w.view(B, Hkv, -1, n), _of_positions(2, s)).view(B, Hkv, -1, R, D)
    y = torch.where(total > 0, y / total, 0.0)
    lse = (m + total.log())[..., 0]
    return y.permute(0, 3, 1, 2, 4).reshape(B, R, H, D).to(s["q"].dtype), lse.permute(0, 3, 1, 2).reshape(B, R, H)


def _written(s, read):
    """What a write gives: the cache as the numbers that it holds, or, where no type
    has them, the positions that were written, read back."""
    if s["bits"] == 4:
        return read(s)
    return tuple(x.view(t) for x, t in zip(s["cache"], (torch.float8_e4m3fn, torch.float8_e8m0fnu) * 2))


def _own(s):
    import paper_2608_26004_amd as asp

    def read(s):
        return asp.read_cache(s["cache"], s["table"], s["lengths"], s["width"], first=s["first"], dtype=s["dtype"])

    if s["op"] == "rotate":
        return asp.rotate_heads(s["q"], s["k"], s["positions"], s["frequencies"], interleaved=s["interleaved"],
                                magnitude=s["magnitude"])
    if s["op"] == "write":
        asp.write_cache(s["k"], s["v"], s["slots"], s["cache"])
        return _written(s, read)
    if s["op"] == "read":
        return read(s)
    return asp.attend_cache(s["q"], s["cache"], s["table"], s["lengths"], new_tokens=s["new_tokens"], scale=s["scale"],
                            window=s["window"], return_lse=True)


def run(state):
    if own:
        return _own(state)
    if state["op"] == "write":
        _plain_write(state)
        return _written(state, _plain_read)
    return {"rotate": _plain_rotate, "read": _plain_read, "attend": _plain_attend}[state["op"]](state)


# -------------------------------------------------------------------- work --
def work(case):
    """Queries, keys and values once each way; of a cache, the positions that the
    call writes, or that a row sees (requests have three quarters of the longest
    length on average)."""
    c = case
    el = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rotate":
        n = c["B"] * c["R"] * (c["H"] + c["Hkv"])
        return {"bytes": 2.0 * n * c["D"] * el + 4.0 * c["B"], "flops": 3.0 * n * c["rot"]}
    held = c["D"] * c["bits"] / 8 + c["D"] / 32
    if c["op"] == "write":
        n = 2.0 * c["B"] * c["R"] * c["Hkv"]
        back = n * (c["D"] * el + (1 - c["skip"]) * held) if c["bits"] == 4 else 0.0
        return {"bytes": n * (1 - c["skip"]) * (c["D"] * el + held) + back, "flops": 4.0 * n * c["D"]}
    if c["op"] == "read":
        n = 2.0 * c["B"] * c["L"] * c["Hkv"]
        return {"bytes": n * (c["D"] * el + 0.75 * held), "flops": n * c["D"]}
    rows = c["B"] * c["R"] * c["H"] * (0.9 if c["fewer"] else 1.0)
    seen = 0.75 * c["L"] + c["R"]
    if c["window"]:
        seen = min(seen, c["window"] + c["R"])
    return {"bytes": 2.0 * c["B"] * seen * c["Hkv"] * held + rows * (2.0 * c["D"] * el + 4.0),
            "flops": 4.0 * rows * c["D"] * seen}


# ------------------------------------------------------------- 64-bit check --
def _levels(bits):
    """What a code without its sign stands for, by the formats' definitions."""
    most, bias, low = (127, 7, 3) if bits == 8 else (8, 1, 1)
    got = []
    for code in range(most):
        e, f = code >> low, code & ((1 << low) - 1)
        got.append(math.ldexp(f, 1 - bias - low) if e == 0 else math.ldexp((1 << low) + f, e - bias - low))
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def _exact_stored(x, bits):
    """(values over the scale, scale) of fp64 values [..., D], by a search of the levels."""
    levels = _levels(bits)
    x = x.unflatten(-1, (-1, 32))
    amax, top = x.abs().amax(-1, keepdim=True), float(levels[-1])
    scale = torch.full_like(amax, 2.0 ** -100)
    for e in range(-99, 128):
        scale = torch.where(amax > scale * top, 2.0 ** e, scale)
    y = (x / scale).abs()
    hi = torch.searchsorted(levels, y.contiguous()).clamp_max(len(levels) - 1)
    lo = (hi - 1).clamp_min(0)
    up, down = levels[hi] - y, y - levels[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(levels[code], x).flatten(-2), scale[..., 0]


def _exact_values(cache, part, request, table, first, n):
    """Values in fp64 of a request's n positions from `first` on, [n, Hkv, D]."""
    data, scales = cache[part], cache[part + 1]
    bs, bits = data.shape[2], 8 * data.shape[3] // (32 * scales.shape[3])
    p = torch.arange(first, first + n, device=data.device)
    page = table[request, p // bs].long()
    d = data[page, :, p % bs]
    if bits == 4:
        d = torch.stack([(d >> sh) & 15 for sh in (0, 4)], -1).flatten(-2)
    signs = d >= (128 if bits == 8 else 8)
    v = _levels(bits)[(d.long() & (127 if bits == 8 else 7))]
    scale = torch.exp2(scales[page, :, p % bs].double() - 127)
    return torch.where(signs, -v, v) * scale.repeat_interleave(32, -1)


def exact(case, seed):
    """Rotations as complex products; quantised values by a search of all levels;
    attention request by request; all in fp64."""
    s = prepare(case, seed)
    if case["op"] == "rotate":
        n, got = len(s["frequencies"]), []
        t = s["positions"][:, None] + torch.arange(case["R"], device="cuda", dtype=torch.int32)
        turn = torch.polar(torch.full((), float(s["magnitude"]), device="cuda", dtype=torch.float64),
                           torch.einsum("br,f->brf", t.double(), s["frequencies"]))[:, :, None]
        for x in (s["q"], s["k"]):
            y = x.double()
            z = y[..., :2 * n]
            z = z.unflatten(-1, (n, 2)) if s["interleaved"] else z.unflatten(-1, (2, n)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
            y[..., :2 * n] = z.flatten(-2) if s["interleaved"] else z.transpose(-1, -2).flatten(-2)
            got.append(y)
        return tuple(got)
    if case["op"] == "write" and case["bits"] == 8:
        got = []
        for name in ("k", "v"):
            bs, blocks = case["bs"], s["cache"][0].shape[0]
            y, scale = _exact_stored(s[name].double(), 8)
            data = torch.zeros(blocks * bs, case["Hkv"], case["D"], dtype=torch.float64, device="cuda")
            # (what no call wrote is a scale byte of 0)
            scales = torch.full((blocks * bs, case["Hkv"], case["D"] // 32), 2.0 ** -127, dtype=torch.float64, device="cuda")
            keep = s["slots"] >= 0
            data[s["slots"][keep]], scales[s["slots"][keep]] = y[keep], scale[keep]
            got += [x.unflatten(0, (blocks, bs)).transpose(1, 2) for x in (data, scales)]
        return tuple(got)
    if case["op"] == "write":
        got = []
        for name in ("k", "v"):
            y, scale = _exact_stored(s[name].double(), 4)
            y = y * scale.repeat_interleave(32, -1)
            got.append(torch.where((s["slots"] >= 0)[..., None, None], y, 0.0))
        return tuple(got)
    if case["op"] == "read":
        got = []
        for part in (0, 2):
            y = torch.zeros(case["B"], case["L"], case["Hkv"], case["D"], dtype=torch.float64, device="cuda")
            for b, n in enumerate(s["lengths"].tolist()):
                y[b, :n] = _exact_values(s["cache"], part, b, s["table"], 0, n)
            got.append(y)
        return tuple(got)
    B, R, H, D = s["q"].shape
    y = torch.zeros(B, R, H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((B, R, H), -math.inf, dtype=torch.float64, device="cuda")
    fresh = s["new_tokens"].tolist() if s["new_tokens"] is not None else [R] * B
    for b, n in enumerate(s["lengths"].tolist()):
        if fresh[b] == 0:
            continue
        first = max(0, n - case["window"] + 1) if case["window"] else 0
        k, v = (_exact_values(s["cache"], part, b, s["table"], first, n + fresh[b] - first) for part in (0, 2))
        each = H // case["Hkv"]
        for h in range(case["Hkv"]):
            kh, vh, heads = k[:, h].contiguous(), v[:, h].contiguous(), slice(h * each, (h + 1) * each)
            for r in range(fresh[b]):
                lo = max(0, n + r - case["window"] + 1 - first) if case["window"] else 0
                hi = n + r + 1 - first
                logit = s["q"][b, r, heads].double() @ kh[lo:hi].T * s["scale"]
                y[b, r, heads] = torch.softmax(logit, -1) @ vh[lo:hi]
                lse[b, r, heads] = torch.logsumexp(logit, -1)
    return y, lse
