"""The operators around the decision step on the GPU, against the plain
references of step_ref.py (64 bits)."""

import math

import numpy as np
import pytest

import paper_2608_26004_amd as asp

import step_ref as ref

torch = pytest.importorskip("torch")
pytestmark = [pytest.mark.gpu, pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}     # half a step, relative
TINY = {"bf16": 2.0 ** -133, "fp32": 2.0 ** -149}  # the smallest subnormals: half a step there is below


def gpu(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()


def stored(rng, shape, dtype, scale=3.0):
    """(device tensor, its values in fp64)."""
    x = torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32)).cuda().to(DT[dtype])
    return x, x.double().cpu().numpy()


def i32(x):
    return np.asarray(x, np.int32)


# --------------------------------------------------------------------- shape --
def shape_inputs(rng, B, R, V, L, D, n_bias, masks, Vh=0):
    ids = lambda *s: i32(rng.integers(-2, (Vh or V) + 2, s))     # noqa: E731  (some out of range)
    lengths = i32(rng.integers(0, L + 1, B)) if L else None
    if L and B > 2:
        lengths[0], lengths[1], lengths[2] = 0, L + 5, -3        # clamped
    kw = dict(history=ids(B, L) if L else None, lengths=lengths,
              prompt_lengths=i32(rng.integers(-1, L + 2, B)) if L and B % 2 else None,
              draft_tokens=ids(B, D) if D else None,
              repetition=(0.5 + rng.random(B)).astype(np.float32), frequency=rng.random(B).astype(np.float32),
              presence=rng.standard_normal(B).astype(np.float32),
              bias_ids=ids(B, n_bias) if n_bias else None,
              bias_values=(3 * rng.standard_normal((B, n_bias))).astype(np.float32) if n_bias else None)
    if L and B > 3:
        kw["repetition"][3], kw["frequency"][3], kw["presence"][3] = 1.0, 0.0, 0.0
    if masks:
        W = (V + 31) // 32
        m = rng.integers(0, 1 << 32, (masks, W), dtype=np.uint64)
        m[0] = 0                                       # nothing allowed
        m[masks // 2] = 0xFFFFFFFF                     # everything
        m[-1, 0], m[-1, 1:] = 1, 0                     # token 0 alone
        kw["mask"] = m.astype(np.uint32).view(np.int32)
        kw["mask_index"] = i32(rng.integers(-1, masks + 1, (B, R)))
    if Vh:
        kw["id_map"] = i32(rng.integers(-1, V + 1, Vh))
    return kw


def ref_shape(x64, kw):
    kw = dict(kw)
    kw["drafts"] = kw.pop("draft_tokens")
    if kw.get("mask") is not None:
        kw["mask"] = kw["mask"].view(np.uint32)
    return ref.shape_logits(x64, **kw)


def assert_shaped(got, want, bound, dtype):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin & ~np.isnan(want)], want[~fin & ~np.isnan(want)])
    # the fp32 steps, then one rounding to the storage type
    with np.errstate(invalid="ignore"):
        lim = bound + HALF[dtype] * (np.abs(want) + bound) + TINY[dtype]
    bad = np.abs(got[fin] - want[fin]) > lim[fin]
    assert not bad.any(), (got[fin][bad][:3], want[fin][bad][:3])


SHAPES = [
    # B, R, V, L, D, n_bias, masks, Vh
    (1, 1, 1, 1, 0, 1, 0, 0), (1, 1, 7, 0, 0, 0, 3, 0), (3, 2, 8, 5, 1, 4, 3, 0), (4, 3, 31, 9, 2, 0, 0, 0),
    (5, 2, 33, 40, 1, 33, 4, 0), (2, 1, 1023, 700, 0, 64, 0, 0), (2, 4, 1025, 513, 5, 100, 3, 0),
    (5, 7, 8200, 3000, 6, 40, 5, 0), (1, 64, 2049, 100, 63, 10, 3, 0), (2, 3, 50257, 6001, 2, 1023, 4, 0),
    (2, 1, 4100, 64, 64, 3, 0, 0), (4, 3, 5003, 800, 2, 30, 3, 777), (3, 2, 600, 300, 1, 0, 0, 9000),
    (40, 2, 40000, 50, 1, 5, 3, 0),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("dims", SHAPES)
def test_shape_matches_reference(dims, dtype):
    B, R, V, L, D, n_bias, masks, Vh = dims
    rng = np.random.default_rng(hash(dims) & 0xFFFF)
    x, x64 = stored(rng, (B, R, V), dtype)
    kw = shape_inputs(rng, B, R, V, L, D, n_bias, masks, Vh)
    want, bound = ref_shape(x64, kw)
    dev = {k: gpu(v) for k, v in kw.items()}
    keep = x.clone()
    out = torch.full_like(x, 77.0)
    res = asp.shape_logits(x, **dev, out=out)
    assert res is out and torch.equal(x, keep)
    assert_shaped(out, want, bound, dtype)
    assert asp.shape_logits(x, **dev) is x             # in place: the same bits
    assert torch.equal(x.view(torch.uint8), out.view(torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_shape_strided_views_and_what_lies_around(dtype):
    """One position of a [B][K+1][V] buffer, an odd offset, a [R][B][V] layout:
    the view is shaped and everything around it keeps its bits."""
    rng = np.random.default_rng(5)
    B, R, V = 3, 2, 1501
    kw = shape_inputs(rng, B, R, V, 200, 1, 20, 3)
    dev = {k: gpu(v) for k, v in kw.items()}
    for view in (lambda b: b[:3, 1:3, 3:3 + V], lambda b: b[:3, :2, :V], lambda b: b.transpose(0, 1)[1:4, :2, 7:7 + V]):
        buf, _ = stored(rng, (4, 4, V + 11), dtype)
        x = view(buf)
        want, bound = ref_shape(x.double().cpu().numpy(), kw)
        before = buf.clone()
        asp.shape_logits(x, **dev)
        assert_shaped(x, want, bound, dtype)
        view(before).copy_(x)
        assert torch.equal(before.view(torch.uint8), buf.view(torch.uint8))


def test_shape_untouched_logits_keep_their_bits():
    """Not-a-number payloads, negative zeros and infinities without a list entry
    stay as they are, in the vectors of changed neighbours too."""
    V = 4099
    bits = np.random.default_rng(6).integers(0, 1 << 16, (1, 1, V), dtype=np.uint16)
    x = gpu(bits.view(np.int16)).view(torch.bfloat16)
    hist = gpu(i32([[5, 4098, 2000]]))
    one = torch.ones(1, device="cuda")
    asp.shape_logits(x, history=hist, lengths=gpu(i32([3])), frequency=one, repetition=one)
    got = x.view(torch.int16).cpu().numpy().view(np.uint16)
    same = np.ones(V, bool)
    same[[5, 4098, 2000]] = False
    assert np.array_equal(got[0, 0, same], bits[0, 0, same])


def test_shape_rows_ahead_of_a_draft_keep_their_bits():
    """A token that only stands among the drafts is untouched in the rows ahead of
    it, whatever its bits, in whole vectors and behind the last one."""
    V, R = 1029, 3
    bits = np.full((1, R, V), 0x7F81, np.uint16)               # signalling not-a-numbers
    x = gpu(bits.view(np.int16)).view(torch.bfloat16)
    one = torch.ones(1, device="cuda")
    asp.shape_logits(x, draft_tokens=gpu(i32([[7, V - 1]])), repetition=2 * one, presence=one)
    got = x.view(torch.int16).cpu().numpy().view(np.uint16)
    changed = got != bits
    assert not changed[0, 0].any()
    assert changed[0, 1].nonzero()[0].tolist() == [7] and changed[0, 2].nonzero()[0].tolist() == [7, V - 1]
    assert torch.isnan(x).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_shape_special_values(dtype):
    """Infinities and not-a-numbers under penalties and masks; biases of
    -inf; a row that the mask empties; the lowest finite value masked."""
    low = float(torch.finfo(DT[dtype]).min)
    x = torch.tensor([[[math.inf, -math.inf, math.nan, low, 0.0, -0.0, 1.0, 2.0, math.nan]] * 2], device="cuda").to(DT[dtype])
    x64 = x.double().cpu().numpy()
    kw = dict(history=i32([[0, 1, 2, 3, 4, 5, 3]]), lengths=i32([7]), prompt_lengths=None, draft_tokens=None,
              repetition=np.float32([2.0]), frequency=np.float32([0.5]), presence=np.float32([1.0]),
              bias_ids=i32([[7, 6, 6]]), bias_values=np.float32([[-math.inf, 5.0, 0.25]]),
              mask=i32([[0], [0b011111111]]), mask_index=i32([[1, 0]]))
    want, bound = ref_shape(x64, kw)
    if dtype == "bf16":
        # the lowest bf16 value times 2 is beyond fp32 too
        assert want[0, 0, 3] < -3.4e38
    with np.errstate(all="ignore"):
        want[want < -3.4028235e38] = -np.inf
    asp.shape_logits(x, **{k: gpu(v) for k, v in kw.items()})
    assert_shaped(x, want, np.nan_to_num(bound, nan=0.0, posinf=0.0), dtype)
    assert torch.isneginf(x[0, 1]).all() and torch.isneginf(x[0, 0, 8])


def test_shape_nothing_to_do():
    x, _ = stored(np.random.default_rng(1), (2, 2, 500), "fp32")
    keep = x.clone()
    assert torch.equal(asp.shape_logits(x), keep)
    out = torch.empty_like(x)
    assert torch.equal(asp.shape_logits(x, out=out), keep)
    h = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    z = torch.zeros(2, dtype=torch.int32, device="cuda")
    assert torch.equal(asp.shape_logits(x, history=h, lengths=z, presence=torch.ones(2, device="cuda")), keep)


def test_shape_long_history_counts():
    """2^20 - 1 tokens, most of them the same one: the count's field holds it."""
    L = (1 << 20) - 1
    h = torch.full((1, L), 3, dtype=torch.int32, device="cuda")
    h[0, ::1000] = 5
    n5 = len(range(0, L, 1000))
    x = torch.zeros(1, 1, 64, device="cuda")
    asp.shape_logits(x, history=h, lengths=torch.tensor([L], dtype=torch.int32, device="cuda"),
                     frequency=torch.full((1,), 2.0 ** -10, device="cuda"),
                     bias_ids=gpu(i32([[3] * 1022 + [5]])), bias_values=gpu(np.float32([[1.0] * 1021 + [4.0, 8.0]])))
    assert x[0, 0, 3].item() == -(L - n5) * 2.0 ** -10 + 4.0      # exact in fp32
    assert x[0, 0, 5].item() == -n5 * 2.0 ** -10 + 8.0
    assert int((x != 0).sum()) == 2


# ---------------------------------------------------------------------- draw --
def check_draw(x, tau, u, **kw):
    tok, q = asp.draw_tokens(x, gpu(tau), gpu(u), **kw)
    t, p, near = ref.draw_tokens(x.double().cpu().numpy(), tau.astype(np.float64), u.astype(np.float64))
    got, gq = tok.cpu().numpy(), q.double().cpu().numpy()
    # fp64 sums of up to 2^20 terms: a step is uncertain by far less than 1e-11
    sure = near > 1e-11
    assert sure.mean() > 0.9 and np.array_equal(got[sure], t[sure])
    # one rounding to fp32, and 1e-11 for the sums
    assert np.all(np.abs(gq - p)[sure] <= p[sure] * (2.0 ** -24 + 1e-11) + 2.0 ** -150)
    return tok, q


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [1, 2, 15, 16, 17, 255, 4095, 4096, 4097, 8191, 50257, 151936, 1100003])
def test_draw_matches_reference(V, dtype):
    rng = np.random.default_rng(V)
    N = 12 if V < 1e6 else 3
    x, _ = stored(rng, (N, V), dtype)
    tau = rng.choice([0.0, -1.0, 0.05, 0.7, 1.0, 3.0, np.nan], N).astype(np.float32)
    u = rng.random(N, dtype=np.float32)
    u[0] = 0.0
    u[1:2] = 1.0 - 2.0 ** -24
    check_draw(x, tau, u)


def test_draw_special_rows():
    """Masked rows, rows without weight, infinities, not-a-numbers, ties,
    temperatures at both ends, uniforms out of range."""
    V, N = 9001, 20
    rng = np.random.default_rng(2)
    x, _ = stored(rng, (N, V), "fp32")
    tau = np.full(N, 0.8, np.float32)
    u = rng.random(N, dtype=np.float32)
    x[0, :-1] = -math.inf                      # the last token alone
    x[1] = -math.inf
    x[2] = math.nan
    x[3, ::2] = math.nan
    x[4, [7, 5000, 9000]] = math.inf           # share all weight
    x[5, [7, 5000]] = math.inf
    x[6] = 0.25                                # ties: the lowest index
    x[7, [4095, 4096]] = 99.0
    tau[1], tau[5], tau[6], tau[7] = 0.0, 0.0, 0.0, 0.0
    tau[8], tau[9], tau[10] = 1e-38, math.inf, 1e30
    x[9, 100:200] = -math.inf
    tau[11], x[11, 50] = math.inf, math.inf
    u[12], u[13], u[14], u[15] = 1.0, 7.0, -1.0, math.nan
    x[12, 8000:] = -math.inf
    x[14, :3] = -math.inf
    x[16] = torch.finfo(torch.float32).min     # the lowest value everywhere: a uniform row
    x[17, 1:] = torch.finfo(torch.float32).min
    tok, q = check_draw(x, tau, u)
    tok, q = tok.cpu(), q.cpu()
    assert tok[0] == V - 1 and q[0] == 1.0
    assert tok[1] == 0 and q[1] == 0.0 and tok[2] == 0 and q[2] == 0.0
    assert tok[3] % 2 == 1 and tok[4] in (7, 5000, 9000) and abs(q[4] - 1 / 3) < 1e-7
    assert tok[5] == 7 and tok[6] == 0 and tok[7] == 4095 and q[7] == 1.0
    assert tok[12] == 7999 and tok[13] == V - 1 and tok[14] == 3 and tok[15] == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offset", [0.0, 1e4, -1e4, 1e30, -1e30])
def test_draw_kinds_of_chunks(offset, dtype):
    """1024 tokens each: all negative, mixed, with -inf, spread wide, with a
    not-a-number, all positive, negative zeros, a part; at temperatures from those
    that leave one token to those that leave all."""
    rng = np.random.default_rng(7)
    N, V = 24, 7 * 1024 + 300
    l = rng.normal(0, 3, (N, V))
    l[:, :1024] = -np.abs(l[:, :1024]) - 0.5
    l[:, 2048 + 5:3072:7] = -np.inf
    l[:, 3072:4096] *= 300.0
    l[:, 4096 + 9] = np.nan
    l[:, 5120:6144] = np.abs(l[:, 5120:6144]) + 0.5
    l[:, 6144:7168] = -0.0
    l[1::3, 3072:4096] = -900.0                 # the wide chunk without the largest one
    x = gpu((l + offset).astype(np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    tau = np.tile(np.float32([0.0, 0.01, 0.4, 1.0, 20.0, 1e4, 1e32, math.inf]), 3)
    check_draw(x, tau, rng.random(N, dtype=np.float32))


@pytest.mark.parametrize("N,V", [(300, 40000), (1500, 17000), (70, 151936), (3, 5000000)])
def test_draw_of_many_tokens(N, V):
    """Large bf16 draws, and a few rows among them with chunks of every kind: each
    row as alone (a row's result does not depend on how many there are), and the
    first ones as the reference has them."""
    rng = np.random.default_rng(N)
    g = torch.Generator(device="cuda").manual_seed(N)
    x = (torch.randn(N, V, generator=g, device="cuda") * 3).to(torch.bfloat16)
    x[0] = 0.0
    x[1, 1024 * 3 + 7] = 0.0
    x[2, 5000 - 900:5000] = -math.inf
    x[3 % N, ::3] = -math.inf
    x[4 % N, 77], x[5 % N, 4900] = math.nan, 200.0
    x[6 % N] *= 100.0
    x[7 % N, 1024:2048] = -150.0
    if N > 8:
        x[7, 2048:4096], x[8] = -math.inf, -math.inf
    tau = rng.choice(np.float32([0.0, 0.1, 0.5, 1.0, 2.0, math.inf]), N).astype(np.float32)
    tau[:9] = np.float32([1.0, 0.8, 0.3, 1.0, 0.19, 2.0, 1.0, 0.6, 3e9])[:min(N, 9)]
    u = rng.random(N, dtype=np.float32)
    tok, q = asp.draw_tokens(x, gpu(tau), gpu(u))
    for n in list(range(min(N, 9))) + [N - 1]:
        check_draw(x[n:n + 1], tau[n:n + 1], u[n:n + 1])
        t1, q1 = asp.draw_tokens(x[n:n + 1], gpu(tau[n:n + 1]), gpu(u[n:n + 1]))
        assert tok[n] == t1[0] and abs(q[n] - q1[0]) <= 2.0 ** -23 * q1[0]


def test_draw_of_the_longest_rows():
    """2^26 tokens of equal logits whose weights are near the largest that a table
    holds: their sum is not beyond fp64."""
    V, u = (1 << 26) + 12345, np.float32(0.3)
    x = torch.full((1, V), 21.625, dtype=torch.bfloat16, device="cuda")
    tok, q = asp.draw_tokens(x, gpu(np.float32([2.0 ** -5])), gpu(u[None]))
    # the first i with i + 1 > u V, which lies half a token from a step
    assert tok[0] == math.floor(float(u) * V) and q[0].item() == np.float32(1.0 / V)


def test_draw_ends_of_the_distribution():
    """Uniforms of 0 and 1 give the first and the last token with weight: one as far
    below the row's largest as fp64's exp gives it, whatever its chunk or the row's
    level; bf16 rows of many tokens."""
    N, V, tau = 300, 40000, 2.0 ** -5
    rng = np.random.default_rng(5)
    x, _ = stored(rng, (N, V), "bf16", 0.5)
    x[:4, :] = 0.5                          # far below 15: weight of 1e-201; at -15: none
    x[:4, 20000] = 15.0
    x[:2, :3000], x[:2, 39000:] = -15.0, -15.0
    x[2:4, 0:5], x[2:4, V - 7:] = -15.0, -15.0
    x[4:8, :5000], x[4:8, 35000:] = -40.0, -40.0      # 1e-264 of what -21 weighs
    x[4:8, 5000:35000] = -21.0
    x[6:8, 30:2000], x[6:8, V - 100:] = -math.inf, -60.0
    t = np.full(N, tau, np.float32)
    u = rng.random(N, dtype=np.float32)
    u[:8] = [0, 1] * 4
    tok, _ = check_draw(x, t, u)
    assert tok[:8].tolist() == [3000, 38999, 5, V - 8, 0, V - 1, 0, V - 101]


@pytest.mark.parametrize("dtype,N,low,top,tau", [
    # one token of 2^-1075.2, rounded to nothing, but its chunk's sum is not when it is
    # multiplied out: 2^-1074.7 for the chunk's scale, times 1024 tokens
    ("fp32", 3, -745.475, -0.20794415, 1.0),
    # the same through the table: tokens of 2^-1079.1, 2^-1069.1 for the chunk
    ("bf16", 300, -8.375, 15.0, 2.0 ** -5)])
def test_draw_of_a_chunk_whose_tokens_have_no_weight(dtype, N, low, top, tau):
    """Whatever their sum would be, the draw does not fall there."""
    V = 40000
    x = torch.full((N, V), low, device="cuda", dtype=DT[dtype])
    x[:, 3000:3010] = top
    u = np.float32([0.0, 1.0, 0.55] * (N // 3))
    tok, q = check_draw(x, np.full(N, tau, np.float32), u)
    assert tok[:3].tolist() == [3000, 3009, 3005] and (q == np.float32(0.1)).all()


@pytest.mark.parametrize("N,V,dtype", [(700, 30000, "bf16"), (200, 70001, "bf16"), (300, 9000, "fp32"), (64, 300000, "fp32")])
def test_draw_with_uniforms_of_one_and_more(N, V, dtype):
    """The last token with weight, also where sums over fewer tokens are rounded to
    more than the row's."""
    x, _ = stored(np.random.default_rng(N), (N, V), dtype)
    x[:, V - 4000:] -= 45.0                  # so little weight that it adds nothing to a sum
    x[::2, V - 1 - N:] = -math.inf
    u = np.resize(np.float32([1.0, 1.0, 1.5, math.inf]), N)
    tok, _ = asp.draw_tokens(x, torch.full((N,), 1.0, device="cuda"), gpu(u))
    want = np.where(np.arange(N) % 2 == 0, V - 2 - N, V - 1)
    assert np.array_equal(tok.cpu().numpy(), want)


def test_draw_of_chunks_far_below_the_largest():
    """Weights of 2^-862 in chunks that a table sums at the level 2^833, beside a
    largest logit beyond the table: counted, though 2^-1695, what is between the two
    levels, is below fp64's range."""
    N, V = 300, 40000
    x = torch.full((N, V), -math.inf, dtype=torch.bfloat16, device="cuda")
    x[:, 3000:3010], x[:, 20000], x[:, 39000:39005] = 57.75, 117.5, 57.75
    u = np.resize(np.float32([0.0, 1.0, 0.5]), N)
    tok, _ = check_draw(x, np.full(N, 0.1, np.float32), u)
    assert tok[:3].tolist() == [3000, 39004, 20000]


def test_draw_every_kind_of_not_a_number():
    """Quiet and signalling ones of either sign, as bf16 bit patterns."""
    V = 5000
    bits = np.full((2, V), 0x3F80, np.uint16)                  # 1.0
    bits[:, 0::4], bits[:, 1::4], bits[:, 2::4] = 0x7F81, 0x7FC0, 0xFF81
    x = gpu(bits.view(np.int16)).view(torch.bfloat16)
    tok, q = asp.draw_tokens(x, gpu(np.float32([0, 1])), gpu(np.float32([0.5, 0.5])))
    assert tok[0] == 3 and q[0] == 1.0
    assert tok[1] == 4 * 625 + 3 and q[1].item() == np.float32(1 / 1250)


def test_draw_strided_views_and_out():
    """One position of the rows' buffer in, columns of [B][K] buffers out; the
    other columns stay; the same bits as from rows on their own."""
    rng = np.random.default_rng(3)
    B, K, V = 9, 4, 5001
    buf, _ = stored(rng, (B, K + 1, V), "bf16")
    tau = rng.choice([0.0, 1.0], B).astype(np.float32)
    uni = torch.from_numpy(rng.random((B, K), dtype=np.float32)).cuda()
    d = torch.full((B, K), -7, dtype=torch.int32, device="cuda")
    q = torch.full((B, K), -7.0, device="cuda")
    for i in range(K):
        want = asp.draw_tokens(buf[:, i].contiguous(), gpu(tau), uni[:, i].contiguous())
        asp.draw_tokens(buf[:, i], gpu(tau), uni[:, i], out=(d[:, i], q[:, i]))
        assert torch.equal(d[:, i], want[0]) and torch.equal(q[:, i], want[1])
        assert (d[:, i + 1:] == -7).all() and (q[:, i + 1:] == -7).all()


def test_draw_outputs_keep_no_large_memory():
    """Tokens that a program keeps do not keep the call's workspace."""
    x = torch.zeros(64, 40000, dtype=torch.bfloat16, device="cuda")
    one = torch.ones(64, device="cuda")
    tok, q = asp.draw_tokens(x, one, one)
    assert max(tok.untyped_storage().nbytes(), q.untyped_storage().nbytes()) <= 1 << 15


def test_draw_follows_the_distribution():
    """2^18 rows of one 5-token distribution: counts within 5 standard deviations."""
    N = 1 << 18
    l = np.float32([0.3, -1.0, 2.0, -np.inf, 1.1])
    x = torch.from_numpy(np.tile(l, (N, 1))).cuda()
    u = np.random.default_rng(4).random(N, dtype=np.float32)
    tok, _ = asp.draw_tokens(x, torch.full((N,), 0.7, device="cuda"), gpu(u))
    p = np.exp(l / np.float64(np.float32(0.7)))
    p /= p.sum()
    n = np.bincount(tok.cpu().numpy(), minlength=5)
    assert np.all(np.abs(n - N * p) <= 5 * np.sqrt(N * p * (1 - p)) + 1e-9)


# -------------------------------------------------------------------- commit --
@pytest.mark.parametrize("B,K,L,n_stop", [(1, 0, 1, 0), (1, 2, 9, 1), (7, 1, 3, 0), (37, 8, 40, 3), (300, 63, 128, 2),
                                          (1000, 4, 500, 70)])
def test_commit_matches_reference(B, K, L, n_stop):
    rng = np.random.default_rng(B + K)
    ids = lambda *s: i32(rng.integers(0, 50, s))     # noqa: E731
    acc, nxt, hist = i32(rng.integers(-2, K + 3, B)), ids(B), ids(B, L)
    wide = ids(B, K + 3)
    lens = i32(rng.integers(-1, L + 2, B))
    fin = i32(rng.random(B) < 0.2) * 3
    stops = i32(rng.integers(0, 200, n_stop))
    maxl = i32(rng.integers(-1, L + 4, B))
    for use_fin, use_max in ((True, True), (False, False)):
        want = ref.commit_tokens(acc, nxt, wide[:, 2:2 + K], hist, lens, fin if use_fin else None, set(stops.tolist()),
                                 maxl if use_max else None)
        h = gpu(hist)
        got = asp.commit_tokens(gpu(acc), gpu(nxt), gpu(wide)[:, 2:2 + K], h, gpu(lens), gpu(fin) if use_fin else None,
                                gpu(stops) if n_stop else None, gpu(maxl) if use_max else None)
        for g, w in zip(got + (h,), want):
            assert np.array_equal(g.cpu().numpy(), w)


def test_commit_in_place_over_steps():
    """Lengths and finished flags written over themselves, step after step."""
    rng = np.random.default_rng(9)
    B, K, L = 50, 3, 60
    hist, lens, fin = i32(rng.integers(0, 99, (B, L))), i32(rng.integers(0, 20, B)), np.zeros(B, np.int32)
    h, ln, f = gpu(hist), gpu(lens), gpu(fin)
    toks, cnt = torch.empty(B, K + 1, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    stops = i32([7])
    for _ in range(25):
        acc, nxt, d = i32(rng.integers(-1, K + 1, B)), i32(rng.integers(0, 99, B)), i32(rng.integers(0, 99, (B, K)))
        lens, fin, t, c, hist = ref.commit_tokens(acc, nxt, d, hist, lens, fin, {7})
        asp.commit_tokens(gpu(acc), gpu(nxt), gpu(d), h, ln, f, gpu(stops), out=(ln, f, toks, cnt))
        for g, w in ((ln, lens), (f, fin), (toks, t), (cnt, c), (h, hist)):
            assert np.array_equal(g.cpu().numpy(), w)
    assert fin.any() and not fin.all()       # both kinds were met


# --------------------------------------------------------------------- slots --
def slot_inputs(rng, B, L, bs, top, N, count, new):
    lens = i32(rng.integers(0, L + 1, B))
    held = i32(np.minimum((lens + bs - 1) // bs + rng.integers(-1, 2, B), top))
    table = i32(rng.integers(0, 10 ** 6, (B, top)))
    return dict(lengths=lens, new_tokens=new, block_table=table, n_blocks=np.maximum(held, 0),
                free_ring=i32(rng.integers(0, 10 ** 6, N)), free_state=i32([int(rng.integers(0, N)), count]),
                release=i32(rng.random(B) < 0.2))


def check_slots(kw, bs, **where):
    want = ref.plan_slots(kw["lengths"], kw["new_tokens"], kw["block_table"], kw["n_blocks"], kw["free_ring"],
                          kw["free_state"], bs, release=kw["release"], **where)
    dev = {k: gpu(v) for k, v in kw.items()}
    got = asp.plan_slots(**dev, block_size=bs, **where)
    slots, short, held, state, starts, table, ring = want
    for g, w in zip(got + (dev["block_table"], dev["free_ring"]),
                    (slots, short, held, state) + ((starts,) if "total" in where else ()) + (table, ring)):
        assert np.array_equal(g.cpu().numpy(), w)
    for k in ("lengths", "n_blocks", "free_state"):
        assert np.array_equal(dev[k].cpu().numpy(), kw[k])
    return want


@pytest.mark.parametrize("B,bs,width", [(1, 1, 1), (1, 16, 3), (5, 16, 9), (64, 4, 2), (255, 16, 7), (257, 1, 3),
                                        (1000, 128, 5), (4096, 16, 4)])
def test_slots_padded(B, bs, width):
    rng = np.random.default_rng(B + bs)
    top = 60 // bs + 3
    for count in (0, B // 3, 4 * B * width):
        N = max(4 * B * width, 1)
        new = i32(rng.integers(-1, width + 2, B))
        for n in (new, None):
            check_slots(slot_inputs(rng, B, 60, bs, top, N, count, n), bs, width=width)


@pytest.mark.parametrize("B,bs,most", [(1, 16, 1), (1, 1, 5000), (7, 32, 900), (64, 16, 700), (300, 8, 40), (4096, 16, 6)])
def test_slots_one_behind_the_other(B, bs, most):
    rng = np.random.default_rng(B + most)
    top = (most + 50) // bs + 3
    new = i32(rng.integers(0, most + 1, B))
    room = int(new.sum())
    for count, total in ((B * top, room + 70), (B, max(1, room)), (B * top // 2, max(1, room // 2))):
        check_slots(slot_inputs(rng, B, 50, bs, top, B * top, count, new), bs, total=total)


def test_slots_state_out_of_range():
    """Counts, fronts, lengths and block ids beyond their range: nothing is read
    or written out of bounds, and the sequential statement still holds."""
    rng = np.random.default_rng(8)
    B, bs, top, N = 40, 16, 6, 50
    for front, count in ((10 ** 9, 30), (-7, 10 ** 9), (49, -5), (-10 ** 9, 50)):
        kw = slot_inputs(rng, B, 80, bs, top, N, 0, i32(rng.integers(-9, 12, B)))
        kw["free_state"] = i32([front, count])
        kw["n_blocks"] = i32(rng.integers(-4, top + 5, B))
        kw["lengths"] = i32(rng.integers(-9, 120, B))
        kw["lengths"][3] = 2 ** 31 - 1
        kw["block_table"][5] = -1
        kw["block_table"][6] = 2 ** 31 - 1
        check_slots(kw, bs, width=9)


def test_slots_pool_is_conserved_over_steps():
    """Many steps of requests that grow, are cut back, end and start anew: every
    block is in exactly one table or in the ring, and live slots are distinct."""
    rng = np.random.default_rng(12)
    B, bs, K1 = 60, 8, 5
    N, top = 150, 12
    lens = np.zeros(B, np.int32)
    table = torch.full((B, top), -1, dtype=torch.int32, device="cuda")
    held = torch.zeros(B, dtype=torch.int32, device="cuda")
    ring = torch.randperm(N).int().cuda()
    state = torch.tensor([17, N], dtype=torch.int32, device="cuda")
    for _ in range(80):
        release = i32(rng.random(B) < 0.1)
        lens[release != 0] = 0
        slots, short, held, state = asp.plan_slots(gpu(lens), None, table, held, ring, state, bs, width=K1,
                                                   release=gpu(release))
        s, sh = slots.cpu().numpy(), short.cpu().numpy()
        live = s[s >= 0]
        assert len(np.unique(live)) == len(live)
        assert np.array_equal((s >= 0).all(1), (sh == 0) & (release == 0))
        t, n, st, rg = (v.cpu().numpy() for v in (table, held, state, ring))
        out = [int(t[b, j]) for b in range(B) for j in range(n[b])]
        free = [int(rg[(st[0] + i) % N]) for i in range(st[1])]
        assert sorted(out + free) == list(range(N))
        grow = rng.integers(0, K1 + 1, B) * ((sh == 0) & (release == 0))
        lens = i32(np.where(rng.random(B) < 0.05, lens // 2, np.minimum(lens + grow, top * bs - K1)))


# ------------------------------------------------------------- used together --
def _step(t, hist, lens, fin, drafts, acc, nxt, table, held, ring, state, tau, u, rep):
    asp.shape_logits(t, history=hist, lengths=lens, draft_tokens=drafts, repetition=rep)
    tok, q = asp.draw_tokens(t[:, 1], tau, u)
    ln, fn, toks, cnt = asp.commit_tokens(acc, nxt, drafts, hist, lens, fin)
    slots, short, held2, state2 = asp.plan_slots(ln, None, table, held, ring, state, 16, width=3, release=fn)
    return tok, q, ln, fn, toks, cnt, slots, short, held2, state2, t, hist, table, ring


def _state(seed):
    rng = np.random.default_rng(seed)
    B, K, V, L, N = 6, 2, 9000, 64, 80
    x, _ = stored(rng, (B, K + 1, V), "bf16")
    return [x, gpu(i32(rng.integers(0, V, (B, L)))), gpu(i32(rng.integers(0, 30, B))), gpu(np.zeros(B, np.int32)),
            gpu(i32(rng.integers(0, V, (B, K)))), gpu(i32(rng.integers(-1, K + 1, B))), gpu(i32(rng.integers(0, V, B))),
            gpu(i32(np.full((B, 8), -1))), gpu(np.zeros(B, np.int32)), gpu(i32(rng.permutation(N))), gpu(i32([0, N])),
            gpu(np.float32([0, 1, 0.7, 0, 1, 1])), gpu(rng.random(B, dtype=np.float32)),
            gpu((1 + rng.random(B)).astype(np.float32))]


def test_captured_steps_replay():
    """A captured step, replayed on new inputs with the program's own eager work
    and synchronisations between the replays, gives the eager results."""
    static = _state(0)
    warm = [v.clone() for v in static]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _step(*warm)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = _step(*static)
    for seed in range(1, 6):
        fresh = _state(seed)
        for a, b in zip(static, fresh):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        want = _step(*fresh)
        for a, b in zip(outs, want):
            assert torch.equal(a, b)


def test_captured_large_draw_and_masked_copy_replay():
    """The draw through a table and a masked copy, captured; replayed on new inputs
    with eager calls of the same between the replays."""
    B, R, V, N = 40, 3, 20011, 300

    def state(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        x = (torch.randn(N, V, generator=g, device="cuda") * 3).to(torch.bfloat16)
        mask = torch.randint(-2 ** 31, 2 ** 31 - 1, (4, (V + 31) // 32), generator=g, device="cuda", dtype=torch.int64)
        return [x, gpu(rng.choice(np.float32([0, 0.7, 1]), N)), gpu(rng.random(N, dtype=np.float32)), mask.int(),
                gpu(i32(rng.integers(-1, 4, (B, R)))), gpu(i32(rng.integers(0, V, (B, 50)))),
                gpu(i32(rng.integers(0, 51, B))), gpu((1 + rng.random(B)).astype(np.float32))]

    def call(x, tau, u, mask, index, hist, lens, rep):
        rows = x[:B * R].view(B, R, V)
        out = torch.empty_like(rows)
        asp.shape_logits(rows, history=hist, lengths=lens, repetition=rep, mask=mask, mask_index=index, out=out)
        return (out.view(torch.int16), *asp.draw_tokens(x, tau, u))

    static = state(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(*static)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = call(*static)
    for seed in range(1, 5):
        fresh = state(seed)
        for a, b in zip(static, fresh):
            a.copy_(b)
        g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, call(*fresh)):
            assert torch.equal(a, b)


def test_calls_on_two_streams_at_once():
    """Two streams, each with its own state, a dozen steps each enqueued in turn."""
    torch.cuda.synchronize()
    states = [[_state(20 + i) for i in range(12)] for _ in range(2)]
    want = [[_step(*[v.clone() for v in st]) for st in row] for row in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for i in range(12):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k].append(_step(*states[k][i]))
    torch.cuda.synchronize()
    for k in range(2):
        for a, b in zip(got[k], want[k]):
            for x, y in zip(a, b):
                assert torch.equal(x, y)


# ------------------------------------------------------------ beside autograd --
def test_calls_that_write_count_as_in_place():
    """Every tensor that a call writes has a new version, so that a backward pass
    that saved it says so; one that is only read, or new, has not."""
    B, K, V, L = 3, 2, 500, 20
    i = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")     # noqa: E731
    x, out, one = torch.randn(B, K + 1, V, device="cuda"), torch.empty(B, K + 1, V, device="cuda"), torch.ones(B, device="cuda")
    hist, lens, d, tok, q = i(B, L), i(B), i(B, K), i(B), torch.empty(B, device="cuda")
    table, held, ring, state = i(B, 4), i(B), torch.arange(12, dtype=torch.int32, device="cuda"), i(2)
    commit_out, slots_out = (i(B), i(B), i(B, K + 1), i(B)), (i(B, 1).long(), i(B), i(B), i(2))
    everything = [x, out, one, hist, lens, d, tok, q, table, held, ring, state, *commit_out, *slots_out]

    def changed(call, want):
        before = [t._version for t in everything]
        new = call()
        assert {id(t) for t, v in zip(everything, before) if t._version > v} == {id(t) for t in want}
        assert all(t._version == 0 for t in new if not any(t is e for e in everything))

    changed(lambda: [asp.shape_logits(x, presence=one)], [x])
    changed(lambda: [asp.shape_logits(x, out=out)], [out])
    changed(lambda: asp.draw_tokens(x[:, 0], one, one), [])
    changed(lambda: asp.draw_tokens(x[:, 0], one, one, out=(tok, q)), [tok, q])
    changed(lambda: asp.commit_tokens(lens, tok, d, hist, lens), [hist])
    changed(lambda: asp.commit_tokens(lens, tok, d, hist, lens, out=commit_out), [hist, *commit_out])
    changed(lambda: asp.plan_slots(lens, None, table, held, ring, state, 16, width=1), [table, ring])
    changed(lambda: asp.plan_slots(lens, None, table, held, ring, state, 16, width=1, out=slots_out),
            [table, ring, *slots_out])
    w = torch.ones(1, device="cuda", requires_grad=True)
    y = (w * x).sum()
    asp.shape_logits(x[:, 1:], presence=one)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
    with torch.inference_mode():
        z = torch.zeros(B, 1, V, device="cuda")
    assert asp.shape_logits(z, presence=one) is z      # a tensor without versions


def test_an_empty_id_map_maps_nothing():
    x, _ = stored(np.random.default_rng(2), (2, 3, 80), "bf16")
    v = x[..., 3:67]
    keep = x.clone()
    ids = torch.zeros(0, dtype=torch.int32, device="cuda")
    h = torch.ones(2, 9, dtype=torch.int32, device="cuda")
    asp.shape_logits(v, history=h, lengths=h[:, 0].contiguous() * 9, presence=torch.ones(2, device="cuda"), id_map=ids)
    assert torch.equal(x, keep)


def test_slots_overlaps_are_refused_by_the_c_entry():
    """(enqueues nothing: the ring, the table and the outputs keep their values)"""
    from test_step_abi import library
    B, top, N = 4, 4, 20
    room = torch.arange(400, dtype=torch.int32, device="cuda")
    keep, p0 = room.clone(), room.data_ptr()
    place = dict(lens=0, new=4, rel=8, table=16, held=32, ring=40, state=60, slots=64, starts=80, short=88, held_out=92,
                 state_out=96)

    def call(**over):
        p = {k: p0 + 4 * v for k, v in {**place, **over}.items()}
        return library().asymspec_plan_slots(p["lens"], p["new"], p["rel"], p["table"], top, p["held"], p["ring"], N,
                                             p["state"], 16, B, 2, 0, p["slots"], p["starts"], p["short"], p["held_out"],
                                             p["state_out"], None)

    for over in (dict(short=8), dict(short=3), dict(held_out=1), dict(held_out=29), dict(state_out=59), dict(starts=0),
                 dict(slots=14), dict(slots=86), dict(ring=31), dict(table=50), dict(state=59), dict(short=90)):
        assert call(**over) == asp.E_ARG, over
    torch.cuda.synchronize()
    assert torch.equal(room, keep)
