"""The operators around the decision step, run together: the loop that stays on
the GPU against the loop that drafts and commits on the host."""

import numpy as np
import pytest

import oracle as O
from paper_2608_26004_amd import driver as drv
from paper_2608_26004_amd import synth

torch = pytest.importorskip("torch")


class HalfRng:
    """The host loop's generator, its drafting uniforms as the GPU gets them."""

    def __init__(self, seed):
        self.rng = np.random.default_rng(seed)

    def random(self, shape, dtype=np.float64):
        if dtype == np.float64:
            return self.rng.random(shape).astype(np.float32).astype(np.float64)
        return self.rng.random(shape, dtype=dtype)


def test_penalties_need_the_resident_loop():
    with pytest.raises(SystemExit):
        drv.main(["--presence", "1.0"])


def test_resident_loop_needs_device_tables():
    with pytest.raises(ValueError):
        drv.ResidentDecoder(drv.TableModels(50, R=8), 2, 1, 0.0)


@pytest.mark.parametrize("K", [1, 3])
@pytest.mark.parametrize("dtype", [synth.BF16, synth.FP32])
@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
def test_resident_loop_is_the_host_loop(dtype, K):
    """Drafting, committing and the paged store on the GPU: the tokens of the
    loop that does them on the host, and its AR and MAL."""
    dev = torch.device("cuda")
    m = drv.TableModels(3000, R=128, rho=1.5, dtype=dtype, seed=11, device=dev)
    tau = np.array([0.0, 1.0, 0.7, 0.0, 1.0, 0.0], np.float32)
    host = drv.SpecDecoder(m, 6, K, tau, seed=12, device=dev)
    host.rng = HalfRng(12)
    res = drv.ResidentDecoder(m, 6, K, tau, seed=12, max_tokens=100, block_size=4)
    for _ in range(15):
        host.step()
        res.step()
    assert res.tokens() == host.tokens
    a, b = res.report(), host.report()
    for k in ("AR", "MAL", "tokens", "steps"):
        assert a[k] == b[k]
    # the store's blocks are those that the lengths need (a position is one behind its tokens)
    need = [-(-(len(t) + 1) // 4) for t in host.tokens]
    held = res.n_blocks.tolist()
    assert all(n <= h <= n + (K + 4) // 4 for n, h in zip(need, held))
    assert sum(held) + int(res.free[1]) == len(res.ring)


def shape32(x, history, drafts, rep, freq, pres):
    """One row's penalties in fp32, token by token."""
    x = x.astype(np.float32).copy()
    out = list(history) + list(drafts)
    for t in set(out):
        c = np.float32(out.count(t))
        x[t] = x[t] / rep if x[t] > 0 else x[t] * rep
        x[t] = (x[t] - freq * c) - pres
    return x


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
def test_resident_loop_with_penalties_matches_a_host_loop():
    """Penalties on all three views with drafts counted, stop tokens and a length
    limit, against a host loop in NumPy with the oracle's decision."""
    V, R, B, K, L = 400, 64, 4, 2, 14
    rep, freq, pres = np.float32(1.3), np.float32(0.4), np.float32(0.25)
    dev = torch.device("cuda")
    m = drv.TableModels(V, R=R, rho=1.0, dtype=synth.FP32, seed=5, device=dev)
    tau = np.array([0.0, 1.0, 0.8, 0.0], np.float32)
    res = drv.ResidentDecoder(m, B, K, tau, seed=6, max_tokens=L, block_size=2, repetition=rep, frequency=freq,
                              presence=pres, stop_tokens=[7, 11, 13])
    rng = HalfRng(6)
    h = drv.roll(np.zeros(B, np.int64), np.arange(B))
    toks, done = [[] for _ in range(B)], [False] * B
    near = np.zeros(B, bool)
    for _ in range(9):
        res.step()
        ud, u = rng.random((B, K)), rng.random((B, K + 1), dtype=np.float32)
        t, a, b = (np.empty((B, K + 1, V), np.float32) for _ in range(3))
        d, q, hs = np.zeros((B, K), np.int32), np.zeros((B, K), np.float32), np.zeros((B, K + 1), np.int64)
        for r in range(B):
            c = h[r]
            for i in range(K + 1):
                hs[r, i] = c
                for x, view in ((t, 0), (a, 1), (b, 2)):
                    x[r, i] = shape32(m.host[view][int(m.row_index(c))], toks[r], d[r, :i], rep, freq, pres)
                if i < K:
                    d[r, i], p = drv._draft_token(a[r, i].astype(np.float64), float(tau[r]), float(ud[r, i]))
                    q[r, i] = np.float32(p)
                    c = drv.roll(c, d[r, i])
        acc, nxt, _, _, out = O.fuse_verify(t, a, b, d, q, u, tau)
        for r in range(B):
            near[r] |= not done[r] and out[r].near_tie(1e-6)
            if done[r]:
                continue
            for x in [int(v) for v in d[r, :acc[r]]] + [int(nxt[r])]:
                if len(toks[r]) == L:
                    break
                toks[r].append(x)
                if x in (7, 11, 13):
                    done[r] = True
                    break
            done[r] = done[r] or len(toks[r]) == L
            h[r] = drv.roll(hs[r, acc[r]], int(nxt[r]))
    got, fin = res.tokens(), res.finished.tolist()
    assert near.sum() <= 1
    for r in range(B):
        if not near[r]:
            assert got[r] == toks[r] and bool(fin[r]) == done[r]
    # requests that ended gave their blocks back at the next step
    res.step()
    assert all(n == 0 for n, f in zip(res.n_blocks.tolist(), fin) if f)


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
def test_resident_loop_with_masks_and_a_small_pool():
    """A grammar that allows even tokens at even positions of a step and odd ones
    at odd positions holds for every draft; requests that find no blocks wait, and
    all of them get to their limit in turn."""
    V, B, K, L = 200, 5, 2, 40
    dev = torch.device("cuda")
    m = drv.TableModels(V, R=32, rho=0.5, seed=9, device=dev)
    words = np.array([0x55555555, 0xAAAAAAAA], np.uint32).view(np.int32)
    mask = torch.from_numpy(np.repeat(words[:, None], (V + 31) // 32, 1)).to(dev)
    index = (torch.arange(K + 1, device=dev) % 2).int().expand(B, K + 1).contiguous()
    res = drv.ResidentDecoder(m, B, K, [0.0, 1.0, 0.7, 1.0, 0.0], seed=3, max_tokens=L, block_size=4, pool=51,
                              mask=mask, mask_index=index)
    waited = 0
    for _ in range(150):
        acc, nxt, tokens = res.step()
        acc, tokens = acc.tolist(), tokens.tolist()
        waited += acc.count(-1)
        for r in range(B):
            got = [x for x in tokens[r] if x >= 0]
            assert [x % 2 for x in got] == [i % 2 for i in range(len(got))]
        if bool((res.finished != 0).all()):
            break
    assert res.lengths.tolist() == [L] * B and waited > 0
    assert res.report()["finished"] == B


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("tau", [0.0, 0.8])
def test_resident_step_does_not_wait_for_the_gpu(tau):
    """Behind work that takes the GPU tens of milliseconds, a step (about one) returns
    while that still runs."""
    m = drv.TableModels(500, R=16, seed=2, device=torch.device("cuda"))
    res = drv.ResidentDecoder(m, 4, 2, tau, seed=3, max_tokens=200, presence=0.5)
    for _ in range(8):
        res.step()
    torch.cuda.synchronize()
    behind = torch.cuda.Event()
    torch.cuda._sleep(50_000_000)       # cycles of a clock between 100 MHz and 2.4 GHz
    behind.record()
    res.step()
    running = not behind.query()
    torch.cuda.synchronize()
    assert running


def test_resident_loop_runs_on_its_models_device():
    """`device` may name it; another one is refused, not ignored."""
    m = drv.TableModels(50, R=8, device="cpu")
    for other in ("cuda", "cuda:1", torch.device("cuda", 0)):
        with pytest.raises(ValueError, match="device"):
            drv.ResidentDecoder(m, 2, 1, 0.0, device=other)
