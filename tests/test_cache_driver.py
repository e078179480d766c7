"""The operators of the quantised cache, run together in the driver's loop: rows, drafts
and commits against a plain recomputation from the tokens."""

import numpy as np
import pytest

import paper_2608_26004_amd as asp
from paper_2608_26004_amd import driver as drv
from paper_2608_26004_amd import synth

import cache_ref as ref

torch = pytest.importorskip("torch")
gpu = pytest.mark.gpu
needs_gpu = pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")


def test_options_belong_together():
    for argv in (["--cache", "4"], ["--window", "5"], ["--resident", "--window", "5"]):
        with pytest.raises(SystemExit):
            drv.main(argv)


def test_tables_need_a_device():
    with pytest.raises(ValueError):
        drv.AttentionModels(50, R=8)


def held(x, bits):
    """fp64 values that a cache holds for x."""
    codes, scales = ref.encode(x, bits)
    return ref.decode(ref.packed(codes, bits), scales, bits)


def turned(x, p, f):
    n = len(f)
    a = p[:, None] * f
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    x = x.astype(np.float64)
    return np.concatenate([x[..., :n] * c - x[..., n:] * s, x[..., :n] * s + x[..., n:] * c], -1)


@gpu
@needs_gpu
@pytest.mark.parametrize("bits,verifier_bits,window,K", [(4, 8, 0, 2), (8, 4, 9, 3), (4, 4, 30, 1)])
def test_rows_follow_from_the_tokens(bits, verifier_bits, window, K):
    """Each view's table row, of every position of every step, is the one that attention in
    64 bits over the tokens' keys and values chooses, wherever the choice is clear."""
    dev = torch.device("cuda")
    B, V, R = 4, 300, 16
    m = drv.AttentionModels(V, R=R, heads=4, kv_heads=2, dim=64, rho=1.0, dtype=synth.FP32, seed=3, device=dev)
    dec = drv.CachedDecoder(m, B, K, [0.0, 1.0, 0.0, 0.8], bits=bits, verifier_bits=verifier_bits, window=window, seed=4,
                            max_tokens=60, block_size=8)
    qkv, anchors = m.qkv.cpu().numpy(), m.anchors.double().cpu().numpy()
    f = m.frequencies.cpu().numpy()
    clear = total = 0
    keys = [np.zeros((0, 2, 64)) for _ in range(B)]        # as the loop turned them
    for _ in range(12):
        before = dec.tokens()
        acc, nxt, _ = dec.step()
        rows = [torch.stack(dec.a_rows, 1), dec.t_rows, dec.b_rows]
        rows = [x.cpu().numpy() for x in rows]
        turned_now = dec.turned.double().cpu().numpy()
        for b in range(B):
            n = len(before[b])
            # the step's inputs: the last committed token and the drafts, of which the commit
            # shows the accepted ones, ahead of the emitted token
            toks = [b % V] + before[b]
            after = dec.tokens()[b][n:]
            seen = len(after) - 1
            inputs = np.array(toks + after[:seen])
            x = qkv[inputs]
            now = turned_now[b, :seen + 1]
            want = turned(x[n:, :6], np.arange(n, len(inputs)), f)
            # angles below 60 in 64 bits, to fp32 within 2 pi 2^-26, sines within 2 units
            assert (np.abs(now - want) <= 2 * np.abs(x[n:, :6]).max() * (2 * np.pi * 2.0 ** -26 + 9 * 2.0 ** -24)).all()
            keys[b] = np.concatenate([keys[b][:n], now[:, 4:]])
            for view, (width, w) in enumerate(((bits, 0), (verifier_bits, window), (bits, window))):
                kk = held(keys[b], width)
                vv = held(x[:, 6:].astype(np.float64), width)
                for r in range(seen + 1):
                    lo = max(0, n + r - w + 1) if w else 0
                    answer = np.empty((4, 64))
                    for h in range(4):
                        t = kk[lo:n + r + 1, h // 2] @ now[r, h] / 8
                        p = np.exp(t - t.max())
                        answer[h] = p @ vv[lo:n + r + 1, h // 2] / p.sum()
                    score = anchors @ answer.ravel()
                    top = np.sort(score)
                    total += 1
                    # an answer's 256 fp32 numbers, below 8, are within 200 u of the formula's, as their
                    # products with anchors below 5 and these products' sum are
                    if top[-1] - top[-2] > 2 * 256 * 8 * 5 * 456 * 2.0 ** -24:
                        clear += 1
                        assert rows[view][b, r] == score.argmax(), (b, r, view, top[-2:])
    assert clear > total * 3 // 4


@gpu
@needs_gpu
def test_equal_views_accept_everything():
    """One table for all views, one width of codes and no window: every draft is accepted."""
    dev = torch.device("cuda")
    m = drv.AttentionModels(2000, R=64, identical=True, dtype=synth.FP32, seed=5, device=dev)
    for x in m.dev[1:]:
        x.copy_(m.dev[0])
    dec = drv.CachedDecoder(m, 5, 2, 0.0, bits=8, verifier_bits=8, seed=6, max_tokens=100)
    for _ in range(20):
        dec.step()
    rep = dec.report()
    assert rep["AR"] == 1.0 and rep["MAL"] == 3.0 and rep["tokens"] == 300


@gpu
@needs_gpu
@pytest.mark.parametrize("pool,all_end", [(20, False), (32, True)])
def test_a_pool_too_small_for_all(pool, all_end):
    """Requests that wait for blocks, end at their limit and give them back.  A request needs
    6 blocks at its end: with 32, six of them that hold 5 leave two, so that one can always
    go on; 20 leave all of them short at some point, which stops them."""
    dev = torch.device("cuda")
    m = drv.AttentionModels(500, R=32, seed=7, device=dev)
    dec = drv.CachedDecoder(m, 6, 2, 0.0, bits=4, window=12, seed=8, max_tokens=20, block_size=4, pool=pool)
    for _ in range(60):
        dec.step()
    assert (dec.report()["finished"] == 6) == all_end
    assert all(len(t) == 20 for t in dec.tokens()) == all_end
    assert int(dec.n_blocks.sum()) + int(dec.free[1]) == pool


@gpu
@needs_gpu
def test_command(capsys):
    drv.main(["--resident", "--cache", "4", "--window", "16", "--B", "4", "--V", "3000", "--R", "64", "--steps", "10",
              "--repetition", "1.2"])
    out = capsys.readouterr().out
    assert '"cache_bits": 4' in out and '"window": 16' in out
