"""The operators of a quantised paged cache on the GPU, against the plain references
of cache_ref.py (64 bits)."""

import math

import numpy as np
import pytest

import paper_2608_26004_amd as asp

import cache_ref as ref

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}     # half a step, relative
TINY = {"bf16": 2.0 ** -133, "fp32": 2.0 ** -149}


def gpu(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def i32(x):
    return np.asarray(x, np.int32)


def f64(t):
    return t.double().cpu().numpy()


def stored(rng, shape, dtype, scale=1.0):
    return torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32)).cuda().to(DT[dtype])


# ------------------------------------------------------------------- rotate --
def rotated(x, positions, f, interleaved, magnitude):
    """(fp64 rotation, bound on an fp32 evaluation's error) of x [B, R, H, D]."""
    n = len(f)
    a = positions.astype(np.float64)[..., None] * f
    cos, sin = (g(a)[:, :, None] * magnitude for g in (np.cos, np.sin))
    y = x.copy()
    p, q = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if interleaved else (x[..., :n], x[..., n:2 * n])
    c, d = p * cos - q * sin, p * sin + q * cos
    # the angle: three roundings in 64 bits here and there, one to fp32 of at most half
    # a turn; sine and cosine within 2 units; magnitude, two products and a sum
    e = np.abs(a)[:, :, None] * 6 * 2.0 ** -53 + 2 * math.pi * 2.0 ** -26 + 4 * 2.0 ** -24
    err = np.zeros_like(x)
    size = (np.abs(p) + np.abs(q)) * abs(magnitude) * (e + 4 * 2.0 ** -24)
    for out, val in ((y, (c, d)), (err, (size, size))):
        if interleaved:
            out[..., 0:2 * n:2], out[..., 1:2 * n:2] = val
        else:
            out[..., :n], out[..., n:2 * n] = val
    return y, err


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B,R,H,Hk,D,n,interleaved", [
    (1, 1, 1, 1, 64, 32, False), (3, 5, 8, 2, 128, 64, False), (2, 3, 4, 4, 96, 24, True), (5, 1, 3, 1, 80, 13, False),
    (2, 7, 6, 3, 34, 17, True), (1, 2, 2, 1, 2, 1, False), (300, 4, 4, 2, 128, 16, False), (1200, 1, 2, 2, 256, 128, True),
    (4, 2, 5, 1, 1024, 512, False), (2, 2, 3, 1, 100, 8, True)])
def test_rotate(dtype, B, R, H, Hk, D, n, interleaved):
    rng = np.random.default_rng(B * 1000 + D + n)
    qkv = stored(rng, (B, R, H + 2 * Hk, D), dtype, 2.0)
    q, k = qkv[:, :, :H], qkv[:, :, H:H + Hk]
    pos = i32(rng.integers(-50, 200000, B))
    pos[0] = 2 ** 31 - 1 if B > 1 else 77
    f = 10000.0 ** (-np.arange(n) / n)
    for every in (False, True):
        p = pos[:, None].astype(np.int64) + np.arange(R)
        given = pos
        if every:
            p = rng.integers(-2 ** 31, 2 ** 31, (B, R))
            given = i32(p)
        got = asp.rotate_heads(q, k, gpu(given), gpu(f), interleaved=interleaved, magnitude=1.25)
        for x, y in zip((q, k), got):
            want, err = rotated(f64(x), p, f, interleaved, 1.25)
            assert y.is_contiguous() and y.dtype == x.dtype
            off = np.abs(f64(y) - want)
            assert (off <= err + HALF[dtype] * np.abs(want) + TINY[dtype]).all(), (every, off.max())
            assert torch.equal(y[..., 2 * n:], x[..., 2 * n:])
    # in place, within the projection: the values' heads stay
    whole = qkv.clone()
    a, b = whole[:, :, :H], whole[:, :, H:H + Hk]
    ra, rb = asp.rotate_heads(a, b, gpu(given), gpu(f), interleaved=interleaved, magnitude=1.25, out=(a, b))
    assert ra is a and rb is b
    assert torch.equal(a, got[0]) and torch.equal(b, got[1]) and torch.equal(whole[:, :, H + Hk:], qkv[:, :, H + Hk:])
    alone = asp.rotate_heads(q, None, gpu(given), gpu(f), interleaved=interleaved, magnitude=1.25)
    assert torch.equal(alone, got[0])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotate_sines_and_cosines(interleaved):
    """The sine and cosine of an angle, as pairs (1, 0) show them in fp32: within 2 units each,
    also where they are small, half a turn away from none and a quarter."""
    rng = np.random.default_rng(20)
    n, pos = 64, i32(rng.integers(0, 200000, 3000))
    # any angles; and those p turns and a half or a quarter on, and a little, of which 64 bits
    # hold all that counts
    f = np.concatenate([10000.0 ** (-np.arange(n // 2) / (n // 2)),
                        2 * math.pi * (np.array([0.5, 0.25] * (n // 4)) + 10.0 ** -rng.uniform(7, 12, n // 2))])
    q = torch.zeros(len(pos), 1, 1, 2 * n, device="cuda")
    if interleaved:
        q[..., 0::2] = 1
    else:
        q[..., :n] = 1
    y = f64(asp.rotate_heads(q, None, gpu(pos), gpu(f), interleaved=interleaved))[:, 0, 0]
    got = (y[:, 0::2], y[:, 1::2]) if interleaved else (y[:, :n], y[:, n:])
    a = pos[:, None].astype(np.longdouble) * f
    for x, want in zip(got, (np.cos(a), np.sin(a))):
        # a unit is at most 2^-23 of a number; angles are products of three roundings of 2^-53
        assert (np.abs(x - want) <= 2 * 2.0 ** -23 * np.abs(want) + 4 * 2.0 ** -53 * np.abs(a)).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,R,H,Hk,D,n", [
    (10003, 1, 32, 8, 128, 64),             # more than the caches hold, one token a workgroup
    (3335, 3, 31, 9, 128, 16),              # the same, four tokens, and one left over
    (10003, 1, 5, 3, 64, 8),                # eight tokens a workgroup, three left over
    (5001, 1, 3, 1, 32, 2),                 # eight, a pair at a time
    (2051, 1, 6, 2, 128, 32)])              # two, one left over
def test_rotate_many_tokens(dtype, interleaved, B, R, H, Hk, D, n):
    """Calls of many tokens are those of few: against the same call in parts of 500 requests,
    bit for bit, and some tokens against 64 bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(B + n)
    qkv = (2 * torch.randn((B, R, H + 2 * Hk, D), device="cuda", generator=g)).to(DT[dtype])
    q, k = qkv[:, :, :H], qkv[:, :, H:H + Hk]
    pos = torch.randint(-100, 100000, (B,), device="cuda", generator=g).int()
    f = gpu(10000.0 ** (-np.arange(n) / n))
    kw = dict(interleaved=interleaved, magnitude=0.75)
    got = asp.rotate_heads(q, k, pos, f, **kw)
    for lo in range(0, B, 500):
        part = asp.rotate_heads(q[lo:lo + 500], k[lo:lo + 500], pos[lo:lo + 500], f, **kw)
        assert all(torch.equal(a[lo:lo + 500], b) for a, b in zip(got, part)), lo
    some = torch.tensor([0, 1, 2, 3, 4, 5, 6, 7, B // 2, B - 4, B - 3, B - 2, B - 1], device="cuda")
    p = pos[some].cpu().numpy()[:, None].astype(np.int64) + np.arange(R)
    for x, y in zip((q, k), got):
        want, err = rotated(f64(x[some]), p, f.cpu().numpy(), interleaved, 0.75)
        assert (np.abs(f64(y[some]) - want) <= err + HALF[dtype] * np.abs(want) + TINY[dtype]).all()
    rest = qkv[:, :, H + Hk:].clone()
    asp.rotate_heads(q, k, pos, f, out=(q, k), **kw)       # in place
    assert torch.equal(q, got[0]) and torch.equal(k, got[1]) and torch.equal(qkv[:, :, H + Hk:], rest)


def test_rotate_heads_major_and_other_outputs():
    """Heads outside rows, requests in no order of memory, and outputs of other strides."""
    rng = np.random.default_rng(5)
    x = stored(rng, (4, 6, 3, 64), "bf16")                 # [B][heads][R][D]
    q, k = x[:, :4].transpose(1, 2), x[:, 4:].transpose(1, 2)
    pos, f = gpu(i32([3, 9, 0, 100])), gpu(10000.0 ** (-np.arange(32) / 32))
    want = asp.rotate_heads(q.contiguous(), k.contiguous(), pos, f)
    got = asp.rotate_heads(q, k, pos, f)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    out = torch.full((3, 4, 9, 70), 7.0, dtype=torch.bfloat16, device="cuda")      # [R][B][heads][..]
    o = out.transpose(0, 1)
    got = asp.rotate_heads(q, k, pos, f, out=(o[:, :, :4, 3:67], o[:, :, 5:7, :64]))
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert (out[..., 4, :] == 7).all() and (out[..., 7:, :] == 7).all() and (out[..., 67:] == 7).all()
    # in place in the tensor that holds both
    y = x.clone()
    a, b = y[:, :4].transpose(1, 2), y[:, 4:].transpose(1, 2)
    asp.rotate_heads(a, b, pos, f, out=(a, b))
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_rotate_back():
    """Positions below zero turn back what those above turned, but for the roundings."""
    rng = np.random.default_rng(6)
    q = stored(rng, (3, 2, 2, 128), "fp32")
    f = asp.rotary_frequencies(128)
    pos = i32([[5, 100000], [7, 8], [1 << 20, 3]])
    there = asp.rotate_heads(q, None, gpu(pos), f)
    back = asp.rotate_heads(there, None, gpu(-pos), f)
    # two rotations, each within (|x| + |y|) (2 pi 2^-26 + 8 * 2^-24) and half a step
    size = f64(q).reshape(3, 2, 2, 2, 64)
    size = np.abs(size).sum(3, keepdims=True).repeat(2, 3).reshape(q.shape)
    assert (np.abs(f64(back) - f64(q)) <= 2 * 2 * size * (2 * math.pi * 2.0 ** -26 + 9 * 2.0 ** -24)).all()


# -------------------------------------------------------------------- write --
def empty(blocks, heads, S, D, bits, fill=None, rng=None):
    shapes = [(blocks, heads, S, D * bits // 8), (blocks, heads, S, D // 32)] * 2
    if rng is not None:
        return [rng.integers(0, 256, s, dtype=np.uint8) for s in shapes]
    return [np.full(s, fill or 0, np.uint8) for s in shapes]


def on_gpu(cache):
    return tuple(gpu(x) for x in cache)


def assert_cache(got, want):
    for name, a, b in zip(("keys", "key_scales", "values", "value_scales"), got, want):
        a = a.cpu().numpy()
        assert np.array_equal(a, b), (name, np.argwhere(a != b)[:5], a[a != b][:5], b[a != b][:5])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens,heads,D,S", [(1, 1, 32, 1), (5, 3, 64, 16), (17, 2, 96, 7), (33, 5, 128, 32),
                                              (16, 8, 256, 16), (50, 1, 192, 24), (300, 4, 160, 16)])
def test_write(dtype, bits, tokens, heads, D, S):
    rng = np.random.default_rng(tokens * 7 + D)
    N = 2 * tokens // S + 3
    want = empty(N, heads, S, D, bits, rng=rng)           # what is not written stays
    cache = on_gpu(want)
    slots = rng.permutation(N * S)[:tokens].astype(np.int64)
    for i, s in ((0, -1), (2, N * S), (3, -2 ** 40), (4, 2 ** 40)):
        if tokens > 4:
            slots[i] = s
    kv = rng.standard_normal((tokens, 2 * heads, D)) * 10.0 ** rng.integers(-6, 6, (tokens, 2 * heads, 1))
    kv = torch.from_numpy(kv.astype(np.float32)).cuda().to(DT[dtype])
    k, v = kv[:, :heads], kv[:, heads:]
    assert asp.write_cache(k, v, gpu(slots), cache) is cache
    ref.write(want, f64(k), f64(v), slots, bits)
    assert_cache(cache, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("tokens,R,heads,D", [(8200, 1, 5, 128), (2750, 3, 3, 256), (12000, 1, 7, 96)])
def test_write_two_heads_a_lane(dtype, bits, tokens, R, heads, D):
    """As many tokens as let a lane have two heads, the last one of an odd number alone."""
    rng = np.random.default_rng(tokens)
    S = 16
    N = tokens * R // S + 5
    want = empty(N, heads, S, D, bits, rng=rng)
    cache = on_gpu(want)
    slots = rng.permutation(N * S)[:tokens * R].astype(np.int64)
    slots[rng.random(tokens * R) < 0.1] = -1
    kv = stored(rng, (tokens, R, 2 * heads, D), dtype, 3.0)
    k, v = kv[:, :, :heads], kv[:, :, heads:]
    asp.write_cache(k, v, gpu(slots.reshape(tokens, R)), cache)
    ref.write(want, f64(k).reshape(-1, heads, D), f64(v).reshape(-1, heads, D), slots, bits)
    assert_cache(cache, want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("heads,D", [(5, 128), (1, 256), (3, 160)])
def test_write_more_than_the_caches_hold(dtype, bits, heads, D):
    """Inputs above 96 MiB: against the same tokens in calls of 1000, bit for bit."""
    g = torch.Generator(device="cuda")
    g.manual_seed(heads + D)
    tokens, S = (100 << 20) // (2 * heads * D * (2 if dtype == "bf16" else 4)), 32
    N = tokens // S + 3
    kv = (torch.randn((tokens, 2 * heads, D), device="cuda", generator=g) * 3).to(DT[dtype])
    k, v = kv[:, :heads], kv[:, heads:]
    slots = torch.randperm(N * S, device="cuda", generator=g)[:tokens]
    slots[torch.rand(tokens, device="cuda", generator=g) < 0.1] = N * S
    start = [torch.randint(0, 256, x.shape, device="cuda", generator=g, dtype=torch.uint8)
             for x in asp.new_cache(N, heads, S, D, bits)]
    got, want = (tuple(x.clone() for x in start) for _ in range(2))
    asp.write_cache(k, v, slots, got)
    for lo in range(0, tokens, 1000):
        asp.write_cache(k[lo:lo + 1000], v[lo:lo + 1000], slots[lo:lo + 1000], want)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("bits", [4, 8])
def test_write_every_code_and_halfway(bits):
    """Values on, beside and halfway between the codes, at scales from the smallest on."""
    lv = ref.levels(bits)
    mid = (lv[1:] + lv[:-1]) / 2
    vals = np.concatenate([lv, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    vals = np.concatenate([vals, -vals])
    rows = []
    for e in (-100, -99, -20, 0, 13, 119 if bits == 8 else 124):
        for lo in range(0, len(vals), 31):
            x = np.full(32, lv[-1])                        # keeps the scale
            x[1:1 + len(vals[lo:lo + 31])] = vals[lo:lo + 31]
            rows.append(x * 2.0 ** e)
    x = np.zeros((len(rows), 1, 32), np.float32)
    x[:, 0] = np.array(rows, np.float32)
    for dtype in ("fp32", "bf16"):
        t = torch.from_numpy(x).cuda().to(DT[dtype])
        want = empty(len(rows), 1, 1, 32, bits)
        cache = on_gpu(want)
        slots = np.arange(len(rows), dtype=np.int64)
        asp.write_cache(t, -t, gpu(slots), cache)
        ref.write(want, f64(t), -f64(t), slots, bits)
        assert_cache(cache, want)


@pytest.mark.parametrize("bits", [4, 8])
def test_write_all_bf16_values(bits):
    """Each bf16 number as the largest of a block of its fractions, among them the
    infinities, those that are not a number, zeros and what is below the smallest scale."""
    b = np.arange(1 << 16, dtype=np.int64)
    x = torch.from_numpy(b.astype(np.uint16).view(np.int16)).cuda().view(torch.bfloat16)
    frac = torch.linspace(-1, 1, 32, device="cuda")
    frac[31] = 1.0
    t = (x.float()[:, None] * frac).to(torch.bfloat16)
    t[:, 31] = x
    t = t[:, None]
    want = empty(1 << 12, 1, 16, 32, bits)
    cache = on_gpu(want)
    asp.write_cache(t, t.float().flip(0).to(torch.bfloat16), gpu(b), cache)
    with np.errstate(all="ignore"):
        k = f64(t)
        for part, y in ((0, k), (2, k[::-1])):
            codes, scales = ref.encode(y, bits)
            want[part][:] = ref.packed(codes, bits).reshape(want[part].shape[:1] + (16, 1, -1)).transpose(0, 2, 1, 3)
            want[part + 1][:] = scales.reshape(1 << 12, 16, 1, 1).transpose(0, 2, 1, 3)
    assert_cache(cache, want)


# --------------------------------------------------------------------- read --
def tables(rng, lengths, S, N, extra=2):
    """Block tables of distinct blocks in no order, and how many blocks are taken."""
    need = [-(-max(0, int(n)) // S) for n in lengths]
    ids = rng.permutation(N)[:sum(need)]
    t = np.full((len(lengths), max(need) + extra), -1)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = ids[at:at + n]
        at += n
    return i32(t)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("B,heads,D,S,L", [(1, 1, 32, 1, 1), (3, 2, 64, 16, 40), (4, 3, 96, 7, 33), (2, 8, 128, 32, 100),
                                           (3, 1, 256, 24, 50)])
def test_read(dtype, bits, B, heads, D, S, L):
    rng = np.random.default_rng(B + D)
    N = B * (L // S + 2) + 4
    cache = empty(N, heads, S, D, bits, rng=rng)
    for p in (1, 3):                                       # bytes that are written, and 255
        cache[p] = np.where(rng.random(cache[p].shape) < 0.02, 255, rng.integers(100, 150, cache[p].shape)).astype(np.uint8)
    lengths = i32(rng.integers(0, L + 1, B))
    lengths[-1] = L
    table = tables(rng, lengths, S, N)
    if B > 2:
        table[1, 0] = N + 5                                # blocks that are not there
        lengths[0] = -3
    first = i32(rng.integers(-3, L // 2 + 1, B))
    got_cache = on_gpu(cache)
    for f in (None, first):
        k, v = asp.read_cache(got_cache, gpu(table), gpu(lengths), L + 3, first=gpu(f), dtype=DT[dtype])
        for got, want in zip((k, v), ref.read(cache, table, lengths, L + 3, f, bits)):
            assert got.shape == (B, L + 3, heads, D) and got.dtype == DT[dtype]
            assert np.array_equal(f64(got), want, equal_nan=True)
    o = (torch.empty_like(k), torch.empty_like(v))
    assert asp.read_cache(got_cache, gpu(table), gpu(lengths), L + 3, first=gpu(first), dtype=DT[dtype], out=o)[0] is o[0]
    assert all(torch.equal(a.nan_to_num(7), b.nan_to_num(7)) for a, b in zip(o, (k, v)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("B,heads,D,S,L", [(2, 5, 128, 16, 4200), (3, 3, 256, 24, 1900), (1, 7, 96, 7, 6300)])
def test_read_two_heads_a_lane(dtype, bits, B, heads, D, S, L):
    """As many positions as let a lane have two heads, the last one of an odd number alone."""
    rng = np.random.default_rng(B + D)
    N = B * (L // S + 2) + 4
    cache = empty(N, heads, S, D, bits, rng=rng)
    for p in (1, 3):
        cache[p] = np.where(rng.random(cache[p].shape) < 0.02, 255, rng.integers(100, 150, cache[p].shape)).astype(np.uint8)
    lengths = i32([L] + [L - 700] * (B - 1))
    table = tables(rng, lengths, S, N)
    table[0, 2] = -1
    first = i32([17] * B)
    for f in (None, first):
        got = asp.read_cache(on_gpu(cache), gpu(table), gpu(lengths), L, first=gpu(f), dtype=DT[dtype])
        for a, want in zip(got, ref.read(cache, table, lengths, L, f, bits)):
            assert np.array_equal(f64(a), want, equal_nan=True)


# ------------------------------------------------------------------- attend --
def attend_inputs(rng, B, R, H, Hk, D, bits, S, dtype, lengths, garbage=True):
    """Queries, a cache (as arrays) that holds the requests' positions and garbage
    everywhere else, the tables, and spare blocks that nobody has."""
    need = [max(0, int(n)) + R for n in lengths]
    N = sum(-(-n // S) for n in need) + 3
    cache = empty(N, Hk, S, D, bits, rng=rng) if garbage else empty(N, Hk, S, D, bits)
    table = tables(rng, need, S, N, extra=1)
    for b, n in enumerate(need):
        p = np.arange(n)
        slots = table[b, p // S].astype(np.int64) * S + p % S
        k = rng.standard_normal((n, Hk, D)) * np.exp(0.5 * rng.standard_normal((Hk, D)))
        ref.write(cache, k, rng.standard_normal((n, Hk, D)), slots, bits)
    q = stored(rng, (B, R, H + 2, D), dtype, 1.5)[:, :, 1:H + 1]
    return q, cache, table


def check_attend(q, cache, table, lengths, bits, new_tokens=None, scale=None, window=0):
    dtype = "bf16" if q.dtype == torch.bfloat16 else "fp32"
    out, lse = asp.attend_cache(q, on_gpu(cache), gpu(table), gpu(i32(lengths)),
                                new_tokens=None if new_tokens is None else gpu(i32(new_tokens)), scale=scale,
                                window=window, return_lse=True)
    # the formula's scale as the kernel has it, in fp32
    at = float(np.float32(scale if scale is not None else q.shape[-1] ** -0.5))
    x = f64(q)
    if dtype == "bf16":
        x = x.astype(np.float32)                           # (exact; its type says how a probability is split)
    want, wlse, err, lerr = ref.attend(x, cache, table, lengths, new_tokens, at, window, bits)
    got, glse = f64(out), f64(lse)
    for a, e in ((got, err), (glse, lerr), (want, err), (wlse, lerr)):
        a[np.isinf(e)] = 0.0                               # (beyond fp32: anything)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), (np.argwhere(np.isnan(got) != nan)[:5])
    assert np.array_equal(np.isnan(glse), np.isnan(wlse)) and np.array_equal(np.isinf(glse), np.isinf(wlse))
    # (c = scale * log2 e is rounded once more: a relative 2^-24 of the scores, as their bound has)
    ok = np.abs(got - want) <= err + HALF[dtype] * (np.abs(want) + err) + TINY[dtype]
    assert (ok | nan).all(), (np.abs(got - want)[~(ok | nan)][:5], err[~(ok | nan)][:5], np.argwhere(~(ok | nan))[:5])
    fin = np.isfinite(wlse)
    assert (np.abs(glse[fin] - wlse[fin]) <= lerr[fin]).all(), (np.abs(glse[fin] - wlse[fin]).max(), lerr[fin].max())
    alone = asp.attend_cache(q, on_gpu(cache), gpu(table), gpu(i32(lengths)),
                             new_tokens=None if new_tokens is None else gpu(i32(new_tokens)), scale=scale, window=window)
    assert torch.equal(alone.nan_to_num(7), out.nan_to_num(7))
    return out, lse


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("S", [16, 7])
def test_attend_dims(dtype, bits, D, S):
    """Every instance's one row tile, then several, then several groups of them."""
    rng = np.random.default_rng(D + S)
    for B, R, H, Hk in ((2, 1, 2, 1), (2, 3, 8, 1), (1, 5, 24, 2), (1, 9, 8, 1)):
        lengths = rng.integers(0, 300, B)
        q, cache, table = attend_inputs(rng, B, R, H, Hk, D, bits, S, dtype, lengths)
        check_attend(q, cache, table, lengths, bits)


@pytest.mark.parametrize("bits,S,dtype", [(4, 16, "bf16"), (8, 32, "bf16"), (4, 1, "fp32"), (8, 24, "fp32"), (4, 128, "bf16")])
@pytest.mark.parametrize("window", [0, 1, 37, 200])
def test_attend_lengths(bits, S, dtype, window):
    """Lengths of none, one and those around the sizes of units, waves and blocks, with
    fewer rows for some requests, all in one call; negative and far too large ones."""
    rng = np.random.default_rng(window + S)
    lengths = np.array([0, 1, 15, 16, 31, 32, 33, 127, 128, 129, 255, 300, 2, 511, 640])
    R = 3
    new = rng.integers(-1, R + 2, len(lengths))
    new[:3], new[12] = R, 0
    q, cache, table = attend_inputs(rng, len(lengths), R, 4, 2, 64, bits, S, dtype, lengths)
    check_attend(q, cache, table, lengths, bits, new_tokens=new, window=window)
    table[3, 0] = -1                                       # blocks that are not there
    table[6, -2:] = cache[0].shape[0]
    table[11] = -7
    far = lengths.copy()
    far[4], far[5], far[8] = -9, 700, 2 ** 31 - 1
    check_attend(q, cache, table, far, bits, new_tokens=new, window=window)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("R,H,Hk", [(64, 2, 2), (17, 5, 1), (1, 64, 1), (9, 14, 2), (33, 1, 1)])
def test_attend_rows(bits, R, H, Hk):
    rng = np.random.default_rng(R)
    lengths = [0, 100]
    q, cache, table = attend_inputs(rng, 2, R, H, Hk, 64, bits, 16, "bf16", lengths)
    check_attend(q, cache, table, lengths, bits)
    q, cache, table = attend_inputs(rng, 2, R, H, Hk, 128, bits, 16, "bf16", lengths)
    check_attend(q, cache, table, lengths, bits, window=50)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("S", [16, 5])
def test_attend_not_finite(bits, dtype, S):
    """A key that is not finite is felt by the rows that see it, in all channels; a value
    in the 32 channels of its scale; and neither by rows that do not see it."""
    rng = np.random.default_rng(S)
    lengths, R = [40, 130, 7, 260], 4
    q, cache, table = attend_inputs(rng, 4, R, 4, 2, 128, bits, S, dtype, lengths)

    def at(b, p):
        return table[b, p // S], p % S
    a = at(0, 42)                                          # rows 2 and 3
    cache[1][a[0], 1, a[1], 2] = 255
    a = at(1, 132)                                         # a value, rows 2 and 3
    cache[3][a[0], 0, a[1], 1] = 255
    a = at(2, 10)                                          # the last row alone
    cache[3][a[0], 1, a[1], 3] = 255
    a = at(3, 11)                                          # seen by all without a window
    cache[3][a[0], 1, a[1], 0] = 255
    if bits == 8:                                          # a code that is not a number
        a = at(1, 131)
        cache[2][a[0], 1, a[1], 77] = 0x7F
        a = at(2, 3)
        cache[0][a[0], 0, a[1], 5] = 0xFF
    for window in (0, 2, 250):
        out, _ = check_attend(q, cache, table, lengths, bits, window=window)
        assert bool(out.isnan().any())


def test_attend_extremes():
    """Scores far from zero, equal ones, a scale of zero, and a negative one."""
    rng = np.random.default_rng(3)
    lengths = [200, 3]
    q, cache, table = attend_inputs(rng, 2, 2, 4, 2, 64, 4, 16, "fp32", lengths)
    for scale in (0.0, -0.3, 20.0, 1e-6):
        check_attend(q, cache, table, lengths, 4, scale=scale)
    check_attend(q * 0, cache, table, lengths, 4)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-33, -3e-34, 2e-36])
def test_attend_tiny_scales(dtype, scale):
    """Scales far below 1, zero among them, of products far above it."""
    rng = np.random.default_rng(18)
    lengths = [200, 3]
    q, cache, table = attend_inputs(rng, 2, 2, 4, 2, 64, 8, 16, dtype, lengths)
    for part in (1, 3):
        cache[part] = np.clip(cache[part], 120, 130)       # (garbage that is not seen, within fp32)
    cache[1] += 53                                         # 2^53: products of some 1e34
    check_attend((q.float() * 2.0 ** 58).to(q.dtype), cache, table, lengths, 8, scale=scale)
    check_attend(q, cache, table, lengths, 8, scale=scale)


@pytest.mark.parametrize("bits,S", [(4, 16), (8, 64), (4, 24)])
def test_attend_long(bits, S):
    """Requests of very different lengths, cut over many workgroups."""
    rng = np.random.default_rng(bits)
    lengths = [9000, 0, 1, 5000, 130]
    q, cache, table = attend_inputs(rng, 5, 2, 4, 2, 64, bits, S, "bf16", lengths, garbage=False)
    check_attend(q, cache, table, lengths, bits)
    check_attend(q, cache, table, lengths, bits, window=3000, new_tokens=[2, 1, 2, 0, 1])


@pytest.mark.parametrize("bits,dtype", [(4, "bf16"), (8, "fp32")])
@pytest.mark.parametrize("units,window", [
    ([11] * 8, 0),                          # as many units each: pieces of runs, and whole ones
    ([4] * 8 + [8] * 8, 500),
    ([17, 15] * 4, 0),                      # no even pieces: those of one more unit
    ([2, 3] * 40, 0),                       # more runs than workgroups
    ([64] + [1] * 30 + [0, 2], 0)])         # one long request among short ones
def test_attend_shares(bits, dtype, units, window):
    """How units are shared among 512 workgroups, for lengths at and around whole units."""
    rng = np.random.default_rng(sum(units))
    lengths = np.array([max(0, 128 * n - int(rng.choice([2, 3, 65]))) for n in units])
    q, cache, table = attend_inputs(rng, len(units), 2, 8, 8, 128, bits, 32, dtype, lengths)
    check_attend(q, cache, table, lengths, bits, window=window)


@pytest.mark.parametrize("bits,dtype", [(4, "bf16"), (8, "bf16"), (4, "fp32"), (8, "fp32")])
@pytest.mark.parametrize("shares", ["pieces", "larger pieces", "even"])
def test_attend_shares_of_an_instance(bits, dtype, shares):
    """The ways in which units are shared, for lengths that follow from the number of
    workgroups of the instance (which its workspace's size shows)."""
    import ctypes

    import test_cache_abi as abi
    heads, D, S, R = 8, 128, 32, 2
    c = abi.Cache(None, None, None, None, 1 << 20, heads, S, D, bits)
    a = abi.Attend(cache=c, q=abi.Heads(), scale=1.0, dtype=0 if dtype == "bf16" else 1, B=4096, R=R, q_heads=heads, max_blocks=100)
    size = abi.library().asymspec_attend_workspace_size(ctypes.byref(a))
    W, left = divmod(size - 524288 - 112, 2 * 16 * (8 + 4 * D))
    assert left == 0 and W in (512, 768)
    n = W // 32
    units = {"pieces": [n] * 8, "larger pieces": [n - 1, n + 1] * 4, "even": [2, 3] * (W // 16 + 2)}[shares]
    # what the kernel then finds: pieces of the even share's size, or one more, that are enough
    # for all runs, or neither
    everything = heads * sum(units)
    even = -(-everything // W)
    assert everything > W
    taken = [heads * sum(-(-u // m) for u in units) <= W for m in (even, even + 1 + even // 16)]
    assert taken == {"pieces": [True, True], "larger pieces": [False, True], "even": [False, False]}[shares]
    rng = np.random.default_rng(n)
    lengths = np.array([128 * u - int(rng.choice([2, 3, 65])) for u in units])
    q, cache, table = attend_inputs(rng, len(units), R, heads, heads, D, bits, S, dtype, lengths)
    check_attend(q, cache, table, lengths, bits)


@pytest.mark.parametrize("bits,dtype,D,R,H,Hk,lengths", [
    (4, "bf16", 128, 3, 4, 1, [4200]),              # 33 parts, 34 and 65 of 12 rows
    (4, "bf16", 128, 3, 4, 1, [4300, 8200]),
    (8, "bf16", 128, 3, 8, 1, [128 * 90 - 1]),      # two row tiles
    (4, "fp32", 256, 1, 2, 2, [11000]),
    (8, "bf16", 64, 5, 1, 1, [40000]),              # more units than workgroups
    (4, "bf16", 96, 4, 2, 1, [36000, 0, 500])])
def test_attend_joined_in_groups(bits, dtype, D, R, H, Hk, lengths):
    """Few requests with so many parts that groups of them are joined first, with values
    that are not numbers in some parts."""
    rng = np.random.default_rng(D + R)
    q, cache, table = attend_inputs(rng, len(lengths), R, H, Hk, D, bits, 32, dtype, lengths)
    first, _ = check_attend(q, cache, table, lengths, bits)
    for _ in range(3):
        again = asp.attend_cache(q, on_gpu(cache), gpu(table), gpu(i32(lengths)))
        assert torch.equal(again, first)
    cache[3][table[0, 20], 0, 5, 1] = 255
    check_attend(q, cache, table, lengths, bits)
    cache[1][table[0, 40], 0, 7, 0] = 255
    check_attend(q, cache, table, lengths, bits)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("D,H,window", [(64, 8, 0), (96, 8, 70), (128, 48, 0), (192, 8, 33), (256, 8, 0)])
def test_attend_many_short_requests(dtype, bits, D, H, window):
    """More requests of a unit at most than there are workgroups, some without positions,
    rows or blocks; with heads of 128 channels also twice as long."""
    rng = np.random.default_rng(D + H)
    B, R = 110, 3
    lengths = rng.integers(0, 126, B)
    lengths[:4] = 0, 1, 125, 31
    new = rng.integers(0, R + 1, B)
    new[:4] = R, R, R, 0
    for at in (lengths, lengths + 90)[:1 if D != 128 else 2]:
        q, cache, table = attend_inputs(rng, B, R, H, 8, D, bits, 24, dtype, at)
        table[5, 0], table[6], table[7, -1] = -1, cache[0].shape[0], 2 ** 31 - 1
        check_attend(q, cache, table, at, bits, new_tokens=new, window=window)


def test_attend_many_requests():
    rng = np.random.default_rng(9)
    B = 700
    lengths = rng.integers(0, 40, B)
    q, cache, table = attend_inputs(rng, B, 1, 2, 1, 64, 4, 16, "bf16", lengths)
    check_attend(q, cache, table, lengths, 4)


def test_attend_offsets_beyond_32_bits():
    """Blocks whose codes begin beyond 2^32 bytes."""
    S, D, bits = 64, 256, 8
    N = (1 << 32) // (S * D) + 40
    rng = np.random.default_rng(4)
    small = attend_inputs(rng, 1, 2, 4, 1, D, bits, S, "bf16", [600])
    q, cache, table = small
    big = asp.new_cache(N, 1, S, D, bits)
    n = cache[0].shape[0]
    for x, y in zip(big, cache):
        x[N - n:] = gpu(y)
    want = asp.attend_cache(q, on_gpu(cache), gpu(table), gpu(i32([600])))
    moved = np.where(table >= 0, table + N - n, -1).astype(np.int32)
    got = asp.attend_cache(q, big, gpu(moved), gpu(i32([600])))
    assert torch.equal(got, want)
    k, v = asp.read_cache(big, gpu(moved), gpu(i32([602])), 602)
    k2, v2 = asp.read_cache(on_gpu(cache), gpu(table), gpu(i32([602])), 602)
    assert torch.equal(k, k2) and torch.equal(v, v2)
    slots = torch.tensor([[N * S - 1]], device="cuda")
    x = stored(rng, (1, 1, 1, D), "bf16")
    asp.write_cache(x, x, slots, big)
    one = asp.new_cache(1, 1, 1, D, bits)
    asp.write_cache(x, x, slots * 0, one)
    assert all(torch.equal(a[-1, 0, -1], b[0, 0, 0]) for a, b in zip(big, one))


# ----------------------------------------------------------------- together --
def step_state(rng, B, R, H, Hk, D, bits, S, pool):
    dev = "cuda"
    s = dict(cache=asp.new_cache(pool, Hk, S, D, bits), table=torch.full((B, pool // 2), -1, dtype=torch.int32, device=dev),
             held=torch.zeros(B, dtype=torch.int32, device=dev), ring=torch.arange(pool, dtype=torch.int32, device=dev),
             free=torch.tensor([0, pool], dtype=torch.int32, device=dev), lengths=torch.zeros(B, dtype=torch.int32, device=dev))
    return s


def run_step(s, qkv, H, Hk, f, S):
    """One layer's step: slots, rotation, write and answer, all on the device."""
    R = qkv.shape[1]
    slots, short, s["held"], s["free"] = asp.plan_slots(s["lengths"], None, s["table"], s["held"], s["ring"], s["free"], S,
                                                        width=R)
    q, k = asp.rotate_heads(qkv[:, :, :H], qkv[:, :, H:H + Hk], s["lengths"], f)
    asp.write_cache(k, qkv[:, :, H + Hk:], slots, s["cache"])
    return asp.attend_cache(q, s["cache"], s["table"], s["lengths"], return_lse=True) + (short,)


def test_steps_together():
    """Steps of drafts of which some are rejected, over plan_slots' tables, against dense
    attention in 64 bits over the keys and values that were kept."""
    rng = np.random.default_rng(1)
    B, R, H, Hk, D, bits, S = 3, 3, 4, 2, 64, 8, 4
    s = step_state(rng, B, R, H, Hk, D, bits, S, 64)
    f = asp.rotary_frequencies(D)
    fn = f.cpu().numpy()
    kept = [[] for _ in range(B)]
    for step in range(12):
        qkv = stored(rng, (B, R, H + 2 * Hk, D), "bf16")
        out, lse, short = run_step(s, qkv, H, Hk, f, S)
        assert not short.any()
        n = s["lengths"].cpu().numpy()
        pos = n[:, None] + np.arange(R)
        q, k = asp.rotate_heads(qkv[:, :, :H], qkv[:, :, H:H + Hk], gpu(i32(pos)), f)
        want_q, err = rotated(f64(qkv[:, :, :H]), pos, fn, False, 1.0)
        assert (np.abs(f64(q) - want_q) <= err + HALF["bf16"] * np.abs(want_q)).all()
        for b in range(B):
            codes = [ref.decode(*(lambda c: (ref.packed(c[0], bits), c[1]))(ref.encode(f64(x)[b], bits)), bits)
                     for x in (k, qkv[:, :, H + Hk:])]
            for r in range(R):
                keys = np.array([x[0] for x in kept[b]] + list(codes[0][:r + 1]))
                vals = np.array([x[1] for x in kept[b]] + list(codes[1][:r + 1]))
                for h in range(H):
                    t = keys[:, h // 2] @ f64(q)[b, r, h] * D ** -0.5
                    w = np.exp(t - t.max())
                    want = w @ vals[:, h // 2] / w.sum()
                    # scores within 2 (64 + 8) 2^-24 sum |q k| < 0.001; probabilities within 2^-17 more
                    far = (np.abs(keys[:, h // 2]) @ np.abs(f64(q)[b, r, h])).max() * D ** -0.5
                    e = (2 * 2 * 72 * 2.0 ** -24 * far + 2 * 2.0 ** -17 + 100 * 2.0 ** -24) * np.abs(vals[:, h // 2]).max()
                    assert (np.abs(f64(out)[b, r, h] - want) <= e + HALF["bf16"] * (np.abs(want) + e)).all()
                    assert abs(float(lse[b, r, h]) - (t.max() + math.log(w.sum()))) <= 2 * 72 * 2.0 ** -24 * far + 2.0 ** -17 + 40 * 2.0 ** -24
            n_acc = int(rng.integers(0, R)) + 1
            kept[b] += [(codes[0][r], codes[1][r]) for r in range(n_acc)]
        s["lengths"] = gpu(i32([len(x) for x in kept]))


def test_captured_steps_replay():
    """A captured step replayed on new inputs between eager work, each replay against
    eager calls on a copy; and two graphs whose memory is reused in between."""
    rng = np.random.default_rng(2)
    B, R, H, Hk, D, bits, S = 4, 2, 8, 2, 128, 4, 16
    f = asp.rotary_frequencies(D)
    s = step_state(rng, B, R, H, Hk, D, bits, S, 256)
    # some context first
    ctx = stored(rng, (B, 500, 2 * Hk, D), "bf16")
    slots, _, s["held"], s["free"] = asp.plan_slots(s["lengths"], torch.full((B,), 500, dtype=torch.int32, device="cuda"),
                                                    s["table"], s["held"], s["ring"], s["free"], S, width=500)
    asp.write_cache(ctx[:, :, :Hk], ctx[:, :, Hk:], slots, s["cache"])
    s["lengths"] = torch.full((B,), 500, dtype=torch.int32, device="cuda")
    slots, _, s["held"], s["free"] = asp.plan_slots(s["lengths"], None, s["table"], s["held"], s["ring"], s["free"], S,
                                                    width=4 * R)
    x = stored(rng, (B, R, H + 2 * Hk, D), "bf16")
    at = slots[:, :R].clone()
    lengths = s["lengths"].clone()

    def body(cache):
        q, k = asp.rotate_heads(x[:, :, :H], x[:, :, H:H + Hk], lengths, f)
        asp.write_cache(k, x[:, :, H + Hk:], at, cache)
        k, v = asp.read_cache(cache, s["table"], lengths, 64, first=lengths - 60)
        return asp.attend_cache(q, cache, s["table"], lengths, return_lse=True) + (k, v)
    body(s["cache"])
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = body(s["cache"])
        graphs.append((g, out))
    mine = tuple(t.clone() for t in s["cache"])
    for i in range(4):
        x.copy_(stored(rng, x.shape, "bf16"))
        at.copy_(slots[:, i * R:(i + 1) * R])
        lengths.copy_(s["lengths"] + i * R)
        want = [t.clone() for t in body(mine)]
        _ = [torch.empty(1 << 20, device="cuda").fill_(float("nan")) for _ in range(4)]
        g, out = graphs[i % 2]
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
        assert all(torch.equal(a, b) for a, b in zip(s["cache"], mine)), i


def test_captured_attend_replays_over_other_lengths():
    """How a captured call shares its work is decided from the lengths of each replay; eager
    calls with another workspace run in between."""
    rng = np.random.default_rng(9)
    B, most = 96, 8300
    q, cache, table = attend_inputs(rng, B, 3, 32, 8, 128, 4, 32, "bf16", [most] + [300] * (B - 1))
    q, c, t = q[:, :, :32], on_gpu(cache), gpu(table)
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    one = torch.tensor([most], dtype=torch.int32, device="cuda")

    def body():
        return (asp.attend_cache(q, c, t, lengths),
                asp.attend_cache(q[:1, :, :4], tuple(x[:, :1].contiguous() for x in small), t[:1], one))
    small = tuple(x[:, :1] for x in c)
    body()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = body()
    for n in ([300] * B, [most] + [0] * (B - 1), [most] + [300] * (B - 1), [20] * B, [0] * B, [most] + [1] * (B - 1)):
        lengths.copy_(torch.tensor(n))
        want = [x.clone() for x in body()]
        g.replay()
        asp.attend_cache(q[:2], c, t[:2], lengths[:2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), n[:2]


def test_two_streams():
    """Calls on two streams at once, each with a workspace of its own."""
    rng = np.random.default_rng(8)
    lengths = [3000, 100, 2000]
    q, cache, table = attend_inputs(rng, 3, 2, 8, 2, 128, 4, 16, "bf16", lengths, garbage=False)
    c, t, n = on_gpu(cache), gpu(table), gpu(i32(lengths))
    p = torch.randn_like(q)
    want = [asp.attend_cache(x, c, t, n, return_lse=True) for x in (q, p)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for i, x in enumerate((q, p)):
            with torch.cuda.stream(streams[i]):
                got[i].append(asp.attend_cache(x, c, t, n, return_lse=True))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))


def test_one_workspace_for_calls_of_any_shape():
    """The C entry point leaves a workspace's counters zero, so that calls of other shapes
    follow in it; what else is in it does not matter."""
    import ctypes

    import test_cache_abi as abi
    lib = abi.library()
    rng = np.random.default_rng(12)
    ws = torch.full((40 << 20,), 0x5A, dtype=torch.uint8, device="cuda")
    counters = 524288
    ws[:counters] = 0
    calls = []
    for B, R, H, Hk, D, bits, S, lengths in ((3, 2, 8, 2, 128, 4, 16, [4000, 0, 900]), (1, 5, 4, 4, 64, 8, 24, [2000]),
                                             (40, 1, 4, 1, 64, 4, 16, rng.integers(0, 300, 40)), (2, 9, 16, 1, 96, 8, 32, [700, 650])):
        q, cache, table = attend_inputs(rng, B, R, H, Hk, D, bits, S, "bf16", lengths, garbage=False)
        q = q.contiguous()
        c, t, n = on_gpu(cache), gpu(table), gpu(i32(lengths))
        want = asp.attend_cache(q, c, t, n, return_lse=True)
        calls.append((q, c, t, n, want, Hk, D, bits, S))
    for _ in range(3):
        for q, c, t, n, want, Hk, D, bits, S in calls:
            out, lse = (torch.full_like(x, 7) for x in want)
            a = abi.Attend(cache=abi.Cache(*(x.data_ptr() for x in c), c[0].shape[0], Hk, S, D, bits),
                           q=abi.Heads(q.data_ptr(), *q.stride()[:3]), out=out.data_ptr(), lse=lse.data_ptr(),
                           block_table=t.data_ptr(), lengths=n.data_ptr(), new_tokens=None, scale=D ** -0.5, window=0, dtype=0,
                           B=q.shape[0], R=q.shape[1], q_heads=q.shape[2], max_blocks=t.shape[1])
            assert lib.asymspec_attend_workspace_size(ctypes.byref(a)) <= ws.numel()
            st = torch.cuda.current_stream().cuda_stream
            assert lib.asymspec_attend_cache(ctypes.byref(a), ws.data_ptr(), ws.numel(), st) == 0
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            assert not ws[:counters].any()


@pytest.mark.parametrize("offset", [16, 64, 112])
def test_a_workspace_that_begins_within_a_line(offset):
    """A workspace of exactly the size asked for, at any multiple of 16 bytes: the same answers,
    counters left zero, and nothing written beside it."""
    import ctypes

    import test_cache_abi as abi
    lib = abi.library()
    rng = np.random.default_rng(17)
    counters = 524288
    # even shares that cross runs, pieces of runs, joins in groups
    for B, R, H, Hk, D, bits, S, lengths in ((40, 2, 8, 8, 128, 8, 32, [383, 254] * 20), (3, 3, 8, 2, 64, 4, 16, [4000, 0, 900]),
                                             (1, 3, 4, 1, 128, 4, 32, [8200])):
        q, cache, table = attend_inputs(rng, B, R, H, Hk, D, bits, S, "fp32", lengths, garbage=False)
        q = q.contiguous()
        c, t, n = on_gpu(cache), gpu(table), gpu(i32(lengths))
        want = asp.attend_cache(q, c, t, n, return_lse=True)
        out, lse = (torch.full_like(x, 7) for x in want)
        a = abi.Attend(cache=abi.Cache(*(x.data_ptr() for x in c), c[0].shape[0], Hk, S, D, bits),
                       q=abi.Heads(q.data_ptr(), *q.stride()[:3]), out=out.data_ptr(), lse=lse.data_ptr(),
                       block_table=t.data_ptr(), lengths=n.data_ptr(), new_tokens=None, scale=D ** -0.5, window=0, dtype=1,
                       B=B, R=R, q_heads=H, max_blocks=t.shape[1])
        size = lib.asymspec_attend_workspace_size(ctypes.byref(a))
        memory = torch.full((size + 512,), 0x5A, dtype=torch.uint8, device="cuda")
        assert memory.data_ptr() % 512 == 0
        memory[offset:offset + counters] = 0
        for _ in range(3):
            out.fill_(7)
            st = torch.cuda.current_stream().cuda_stream
            assert lib.asymspec_attend_cache(ctypes.byref(a), memory.data_ptr() + offset, size, st) == 0
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
            assert not memory[offset:offset + counters].any()
            assert (memory[:offset] == 0x5A).all() and (memory[offset + size:] == 0x5A).all()


def test_a_growing_workspace():
    """A call that needs a larger workspace while calls in the smaller one are still on
    their way, on a stream of its own."""
    rng = np.random.default_rng(13)
    small = attend_inputs(rng, 2, 1, 2, 1, 64, 4, 16, "bf16", [900, 300], garbage=False)
    large = attend_inputs(rng, 4, 4, 16, 2, 256, 4, 16, "bf16", [3000, 900, 2000, 5], garbage=False)
    args = [(q, on_gpu(c), gpu(t), gpu(i32(n))) for (q, c, t), n in ((small, [900, 300]), (large, [3000, 900, 2000, 5]))]
    want = [asp.attend_cache(*a) for a in args]
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = [asp.attend_cache(*args[0]) for _ in range(30)] + [asp.attend_cache(*args[1])] + \
              [asp.attend_cache(*args[0]) for _ in range(5)]
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert torch.equal(g, want[i == 30]), i


def test_threads_on_the_per_thread_stream():
    """hipStreamPerThread is one handle, and another stream in each thread: each thread's calls
    have a workspace of their own, the same one again, and keep it when they need a larger."""
    import threading
    rng = np.random.default_rng(19)
    lengths = [3000, 100, 2000]
    q, cache, table = attend_inputs(rng, 3, 2, 8, 2, 128, 4, 16, "bf16", lengths, garbage=False)
    c, t, n = on_gpu(cache), gpu(table), gpu(i32(lengths))
    want = asp.attend_cache(q, c, t, n, return_lse=True)
    # (each thread's outputs are its own from the start: torch's allocator knows the handle alone)
    outs = [[tuple(torch.full_like(x, 7) for x in want) for _ in range(8)] for _ in range(2)]
    small = asp.attend_cache(q[:, :, ::4, :64].contiguous(), *(few := (asp.new_cache(1, 2, 16, 64), t[:, :1].contiguous(), n)))
    small_outs = [torch.full_like(small, 7) for _ in range(2)]
    qs = q[:, :, ::4, :64].contiguous()
    torch.cuda.synchronize()
    grown, ready = [], threading.Barrier(2)
    taken = []

    def work(me):
        with torch.cuda.stream(torch.cuda.ExternalStream(2)):
            for turn in range(2):                          # one thread after the other
                if turn == me:
                    before = torch.cuda.memory_allocated()
                    asp.attend_cache(qs, *few, out=small_outs[me])
                    taken.append(torch.cuda.memory_allocated() - before)
                    asp.attend_cache(q, c, t, n, return_lse=True, out=outs[me][0])
                    grown.append(torch.cuda.memory_allocated() - before)
                    asp.attend_cache(q, c, t, n, return_lse=True, out=outs[me][1])
                    grown.append(torch.cuda.memory_allocated() - before)
                    torch.cuda.synchronize()
                ready.wait(60)
            for o in outs[me][2:]:                         # both at once
                asp.attend_cache(q, c, t, n, return_lse=True, out=o)
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    torch.cuda.synchronize()
    assert len(grown) == 4 and taken[0] > 524288 and taken[1] == taken[0]
    assert grown[0] > taken[0] and grown == grown[:1] * 4
    assert all(torch.equal(a, b) for each in outs for o in each for a, b in zip(o, want))
    assert all(torch.equal(x, small) for x in small_outs)


def test_attend_most_requests():
    """4096 requests of one position, some of none, and rows of all of them."""
    rng = np.random.default_rng(14)
    B, S = 4096, 16
    lengths = rng.integers(0, 2, B)
    new = rng.integers(0, 2, B)
    q, cache, table = attend_inputs(rng, B, 1, 1, 1, 64, 8, S, "bf16", lengths, garbage=False)
    check_attend(q, cache, table, lengths, 8, new_tokens=new)


@pytest.mark.parametrize("bits,dtype", [(4, "bf16"), (8, "fp32")])
def test_attend_blocks_that_requests_share(bits, dtype):
    """A prefix that is in the cache once, in several requests' tables."""
    rng = np.random.default_rng(15)
    S, lengths = 16, [200, 200, 200]
    q, cache, table = attend_inputs(rng, 3, 2, 4, 2, 64, bits, S, dtype, lengths)
    table[1, :8] = table[0, :8]
    table[2, :11] = table[0, :11]
    check_attend(q, cache, table, lengths, bits)


def test_lse_joins_two_caches():
    """Answers over the two halves of a context, joined by their lse, are the answer over it
    all, within the roundings of bf16 answers."""
    rng = np.random.default_rng(16)
    q, cache, table = attend_inputs(rng, 2, 1, 4, 2, 64, 8, 16, "fp32", [255, 255])
    c = on_gpu(cache)
    whole, lse = asp.attend_cache(q, c, gpu(table), gpu(i32([255, 255])), return_lse=True)
    parts = [asp.attend_cache(q, c, gpu(t), gpu(i32([127, 127])), return_lse=True) for t in (table[:, :8], table[:, 8:])]
    l = torch.stack([p[1] for p in parts]).double()
    w = torch.softmax(l, 0)[..., None]
    got = (w * torch.stack([p[0] for p in parts]).double()).sum(0)
    # fp32 answers within about 100 u of sums of values below 8; lse within 100 u
    assert (got - whole.double()).abs().max() < 2 * 100 * 2.0 ** -24 * 8
    assert (torch.logsumexp(l, 0) - lse.double()).abs().max() < 100 * 2.0 ** -24 * 16


def test_writes_count_as_versions():
    x = torch.randn(2, 1, 1, 32, device="cuda")
    cache = asp.new_cache(2, 1, 2, 32, 8)
    before = [t._version for t in cache]
    asp.write_cache(x, x, torch.zeros(2, 1, dtype=torch.int64, device="cuda") - 1, cache)
    assert all(t._version > v for t, v in zip(cache, before))
    w = x.clone().requires_grad_()
    with pytest.raises(ValueError, match="requires a gradient"):
        asp.rotate_heads(w, None, torch.zeros(2, dtype=torch.int32, device="cuda"), asp.rotary_frequencies(32), out=(w,))
