"""Multi-step speculative decoding over table-driven stand-in models.

The loop of Alg. 1 around the decision step: per step the drafter proposes
K tokens autoregressively from its full-context view, the three logit rows of
every position are produced (drafter full view a, drafter compressed view b,
verifier t; Alg. 1 runs the three forwards), ``fuse_verify`` decides, and the
accepted drafts plus the emitted token are committed.  It reports the two
acceptance diagnostics of the paper's acceptance table (App. F):

  AR   accepted drafts / drafts evaluated, where the drafts evaluated in a
       step are the accepted ones plus the first rejected one (Alg. 1 stops
       there; K when all are accepted);
  MAL  mean number of tokens committed per step, accept_len + 1, out of the
       K + 1 positions.

The "models" are stand-ins (no weights are available): three tables of R
logit rows each, indexed by a rolling hash of the context.  A shared prior z
per table row gives the views their agreement; t = z + N(0,1),
a = z + N(0,1), b = a + rho N(0,1) (b is a copy of a when rho = 0), stored in
the logit dtype.  Drafting happens on the host from the stored a rows (it
stands in for the drafter's own sampler, upstream of the decision step); the
rows of the K+1 positions are gathered from device copies of the tables, and
only hashes, drafts and uniforms cross PCIe.

``ResidentDecoder`` runs the same loop with nothing copied to the host between
steps: penalties, biases and masks shape the rows (``shape_logits``), the drafter
draws on the GPU (``draw_tokens``), what a step commits joins the histories there
(``commit_tokens``), and the stand-in models keep their context per position in a
paged store, as a model keeps its keys and values (``plan_slots``).

``CachedDecoder`` is that loop with keys and values: each token has a query, a key
and a value (random tables), and what a row's attention over a paged cache in 8 or 4
bits answers chooses the logit row (``rotate_heads``, ``write_cache``,
``attend_cache``).  The drafter attends to its full context token by token, its
compressed view and the verifier to the last ``window`` positions, K + 1 rows at once.
"""

from __future__ import annotations

import argparse
import json
import time

import numpy as np

from . import synth

_MUL = 1000003
_MASK = 0x7FFFFFFF


def roll(h, tok):
    """Context hash after appending token(s) `tok` (int64 arrays or ints)."""
    return (np.asarray(h, dtype=np.int64) * _MUL + np.asarray(tok, dtype=np.int64) + 1) & _MASK


class TableModels:
    """Verifier / drafter stand-ins: R rows of V logits per view."""

    def __init__(self, V: int, R: int = 512, rho: float = 1.0, prior_scale: float = 3.0,
                 dtype: str = synth.BF16, seed: int = 0, device=None, identical: bool = False):
        rng = np.random.default_rng(seed)
        z = prior_scale * rng.standard_normal((R, V))
        t = z + rng.standard_normal((R, V))
        a = t.copy() if identical else z + rng.standard_normal((R, V))
        b = a.copy() if (identical or rho == 0.0) else a + rho * rng.standard_normal((R, V))
        if dtype == synth.BF16:
            self.host = [synth.f64_to_bf16_bits(x) for x in (t, a, b)]
        else:
            self.host = [x.astype(np.float32) for x in (t, a, b)]
        self.V, self.R, self.dtype = V, R, dtype
        self.dev = None
        if device is not None:
            import torch
            if dtype == synth.BF16:
                self.dev = [torch.from_numpy(x.view(np.int16)).to(device).view(torch.bfloat16)
                            for x in self.host]
            else:
                self.dev = [torch.from_numpy(x).to(device) for x in self.host]

    def row_index(self, h):
        return np.asarray(h, dtype=np.int64) % self.R

    def drafter_row_f64(self, h):
        return synth.stored_to_f64(self.host[1][int(self.row_index(h))])


def _draft_token(a_row: np.ndarray, tau: float, u: float):
    """The drafter's own choice from its full-view row: argmax (tau <= 0) or
    an inverse-CDF draw from softmax(a / tau) with uniform u; returns the
    token and its proposal probability."""
    if not tau > 0:
        return int(np.argmax(a_row)), 1.0
    z = (a_row - np.max(a_row)) / tau
    w = np.exp(z)
    c = np.cumsum(w)
    d = min(int(np.searchsorted(c, u * c[-1], side="right")), len(w) - 1)
    while w[d] == 0.0 and d > 0:
        d -= 1
    return d, float(w[d] / c[-1])


class SpecDecoder:
    """B independent requests decoded with K drafts per step.

    backend "hip": rows gathered on the GPU and the step runs through
    ``fuse_verify``.  backend "host": rows gathered as NumPy arrays and passed
    to ``step_fn(t, a, b, d, q, u, tau) -> (accept_len, next_token)`` (a
    checker; the product path is "hip")."""

    def __init__(self, models: TableModels, B: int, K: int, temperature, beta: float = 1.0,
                 gamma: float = 0.5, gate_mode: int = 0, seed: int = 0, backend: str = "hip",
                 step_fn=None, device=None, early_exit: int = 0, fuse_bonus: bool = False):
        self.m, self.B, self.K = models, B, K
        self.tau = np.broadcast_to(np.asarray(temperature, np.float32), (B,)).copy()
        self.beta, self.gamma, self.gate_mode = beta, gamma, gate_mode
        self.early_exit, self.fuse_bonus = early_exit, fuse_bonus
        self.call_seconds = []
        self.rng = np.random.default_rng(seed)
        self.h = roll(np.zeros(B, np.int64), np.arange(B))     # distinct start contexts
        self.tokens = [[] for _ in range(B)]
        self.backend, self.step_fn, self.device = backend, step_fn, device
        self.accepted = 0
        self.evaluated = 0
        self.committed = 0
        self.steps = 0
        self.log = []
        if backend == "hip":
            import torch
            import paper_2608_26004_amd as asp
            if models.dev is None:
                raise ValueError("the hip backend needs TableModels(device=...)")
            self._torch, self._asp = torch, asp
            self._ws = asp.Workspace(device)
            self._tau_dev = torch.from_numpy(self.tau).to(device)
        elif step_fn is None:
            raise ValueError("the host backend needs step_fn")

    def _draft(self):
        B, K = self.B, self.K
        d = np.zeros((B, K), np.int32)
        q = np.zeros((B, K), np.float32)
        hs = np.zeros((B, K + 1), np.int64)
        ud = self.rng.random((B, K))
        for b in range(B):
            h = self.h[b]
            for i in range(K):
                hs[b, i] = h
                tok, p = _draft_token(self.m.drafter_row_f64(h), float(self.tau[b]), float(ud[b, i]))
                d[b, i], q[b, i] = tok, np.float32(p)
                h = roll(h, tok)
            hs[b, K] = h
        return d, q, hs

    def step(self):
        B, K = self.B, self.K
        d, q, hs = self._draft()
        u = self.rng.random((B, K + 1), dtype=np.float32)
        idx = self.m.row_index(hs).reshape(-1)
        if self.backend == "hip":
            torch = self._torch
            ii = torch.from_numpy(idx).to(self.device)
            t, a, b = (x.index_select(0, ii).view(B, K + 1, self.m.V) for x in self.m.dev)
            dd, qq, uu = (torch.from_numpy(v).to(self.device) for v in (d, q, u))
            torch.cuda.synchronize(self.device)
            t0 = time.perf_counter()
            acc, nxt, _ = self._asp.fuse_verify(
                t, a, b, dd, qq, uu, self._tau_dev, beta=self.beta, gamma=self.gamma,
                gate_mode=self.gate_mode, workspace=self._ws, early_exit=self.early_exit,
                fuse_bonus=self.fuse_bonus)
            acc, nxt = acc.cpu().numpy(), nxt.cpu().numpy()
            self.call_seconds.append(time.perf_counter() - t0)
        else:
            t, a, b = (x[idx].reshape(B, K + 1, self.m.V) for x in self.m.host)
            acc, nxt = self.step_fn(t, a, b, d, q, u, self.tau)
            acc, nxt = np.asarray(acc), np.asarray(nxt)
        for r in range(B):
            j = int(acc[r])
            new = [int(x) for x in d[r, :j]] + [int(nxt[r])]
            self.tokens[r].extend(new)
            h = hs[r, j]
            self.h[r] = roll(h, int(nxt[r]))
            self.accepted += j
            self.evaluated += j + (1 if j < K else 0)
            self.committed += len(new)
        self.steps += 1
        self.log.append((acc.copy(), nxt.copy()))
        return acc, nxt

    def report(self):
        n = self.steps * self.B
        rep = {"steps": self.steps, "requests": self.B, "K": self.K,
               "AR": self.accepted / self.evaluated if self.evaluated else float("nan"),
               "MAL": self.committed / n if n else float("nan"),
               "tokens": self.committed}
        if self.backend == "hip" and len(self.call_seconds) > 1:
            # host-observed latency of the decision call (median, first call
            # excluded): argument checks, launch, the kernel, and the copy of
            # accept_len and next_token back
            rep["decision_call_us"] = 1e6 * float(np.median(self.call_seconds[1:]))
        return rep


class ResidentDecoder:
    """B independent requests decoded with K drafts per step, all of it enqueued
    on the current stream: ``step()`` returns without waiting for the GPU.

    A request's position p (p tokens behind its start) has one entry in a paged
    store, the hash of its context there; a step places K + 1 more, the drafts'
    among them, and what is rejected is written over by the next one.  A request
    ends with a stop token or at max_tokens and gives its blocks back; one that
    gets no blocks waits for a step in which others have given some back (a pool
    that leaves all of them short stops all of them).

    repetition, frequency, presence: penalties, a number or one per request;
    bias_ids, bias_values [B, n], mask [M, ceil(V / 32)] with mask_index [B, K+1]: as
    ``shape_logits`` takes them, applied to all three views; pool: blocks of the
    store (default: enough for every request); device: that of the models (the
    default), on which all of it runs."""

    def __init__(self, models: TableModels, B: int, K: int, temperature, beta: float = 1.0,
                 gamma: float = 0.5, gate_mode: int = 0, seed: int = 0, device=None, early_exit: int = 0,
                 fuse_bonus: bool = False, max_tokens: int = 1024, block_size: int = 16, pool: int | None = None,
                 repetition=None, frequency=None, presence=None, bias_ids=None, bias_values=None, mask=None,
                 mask_index=None, stop_tokens=None):
        import torch
        import paper_2608_26004_amd as asp
        if models.dev is None:
            raise ValueError("the decoder needs TableModels(device=...)")
        self._torch, self._asp = torch, asp
        self.m, self.B, self.K, self.device = models, B, K, models.dev[0].device
        want = self.device if device is None else torch.device(device)
        if want.type != self.device.type or want.index not in (None, self.device.index):
            raise ValueError(f"the models are on device {self.device}, not on {want}")
        self.rng = np.random.default_rng(seed)
        self.kw = dict(beta=beta, gamma=gamma, gate_mode=gate_mode, early_exit=early_exit, fuse_bonus=fuse_bonus,
                       workspace=asp.Workspace(self.device))
        dev, i32 = self.device, torch.int32

        def per_request(x):
            return None if x is None else torch.as_tensor(x, dtype=torch.float32, device=dev).expand(B).contiguous()

        self.tau = per_request(temperature)
        self.shape = dict(repetition=per_request(repetition), frequency=per_request(frequency),
                          presence=per_request(presence), bias_ids=bias_ids, bias_values=bias_values)
        self.mask, self.mask_index = mask, mask_index
        self.shaped = mask is not None or any(v is not None for v in self.shape.values())
        self.stop = None if stop_tokens is None else torch.as_tensor(stop_tokens, dtype=i32, device=dev)
        self.history = torch.zeros(B, max_tokens, dtype=i32, device=dev)
        self.lengths = torch.zeros(B, dtype=i32, device=dev)
        self.finished = torch.zeros(B, dtype=i32, device=dev)
        # the paged store, one entry a position, and one that nobody reads
        self.block_size = block_size
        blocks = -(-(max_tokens + K + 2) // block_size)
        pool = B * blocks if pool is None else pool
        self.store = torch.zeros(pool * block_size + 1, dtype=torch.int64, device=dev)
        self.table = torch.full((B, blocks), -1, dtype=i32, device=dev)
        self.n_blocks = torch.zeros(B, dtype=i32, device=dev)
        self.ring = torch.arange(pool, dtype=i32, device=dev)
        self.free = torch.tensor([0, pool], dtype=i32, device=dev)
        slots = self._place(torch.zeros_like(self.lengths), 1)[0]
        if int(slots.min()) < 0:
            raise ValueError("the pool must hold a block for each request")
        self.at = slots[:, 0]                                  # slot of each request's last position
        self.store[self.at] = torch.from_numpy(roll(np.zeros(B, np.int64), np.arange(B))).to(dev)
        self.counts = torch.zeros(3, dtype=torch.int64, device=dev)    # accepted, evaluated, committed
        self.request_steps = torch.zeros((), dtype=torch.int64, device=dev)
        self.steps = 0

    def _place(self, lengths, width):
        slots, short, self.n_blocks, self.free = self._asp.plan_slots(
            lengths, None, self.table, self.n_blocks, self.ring, self.free, self.block_size, width=width,
            release=self.finished)
        return slots, short

    def _shape(self, rows, drafts, first):
        """Rows first, first + 1, ... of the step behind the history and drafts."""
        if not self.shaped:
            return
        n = rows.shape[1]
        index = None if self.mask is None else self.mask_index[:, first:first + n].contiguous()
        self._asp.shape_logits(rows, history=self.history, lengths=self.lengths,
                               draft_tokens=drafts if drafts.shape[1] else None, mask=self.mask, mask_index=index,
                               **self.shape)

    # What a subclass keeps for a position, other than its context's hash: the table rows
    # that the views' logits are, and what a step leaves behind.
    def _begin(self):
        """(slots of the step's K + 1 positions, short) and the state of the step."""
        slots, short = self._place(self.lengths + 1, self.K + 1)
        self.slots = self._torch.where(slots < 0, len(self.store) - 1, slots)
        self.hs = self._torch.empty(self.B, self.K + 1, dtype=self._torch.int64, device=self.device)
        return short

    def _drafter_rows(self, i, token):
        """Table rows of the drafter's full view of position i, behind `token` (None: i = 0)."""
        h = self.store[self.at] if i == 0 else (self.hs[:, i - 1] * _MUL + token + 1) & _MASK
        if i > 0:
            self.store[self.slots[:, i - 1]] = h
        self.hs[:, i] = h
        return h % self.m.R

    def _view_rows(self):
        """Table rows of the verifier and of the drafter's compressed view, [B, K + 1] each."""
        rows = self.hs % self.m.R
        return rows, rows

    def _end(self, live, j, nxt, tokens, n):
        torch, slots = self._torch, self.slots
        emitted = (self.hs.gather(1, j)[:, 0] * _MUL + nxt + 1) & _MASK
        self.store[torch.where(live, slots.gather(1, j)[:, 0], len(self.store) - 1)] = emitted
        last = slots.gather(1, (n.long() - 1).clamp_min(0)[:, None])[:, 0]
        self.at = torch.where(n > 0, last, self.at)

    def step(self):
        torch, asp, B, K, m = self._torch, self._asp, self.B, self.K, self.m
        dev = self.device
        ud = torch.from_numpy(self.rng.random((B, K)).astype(np.float32)).to(dev, non_blocking=True)
        u = torch.from_numpy(self.rng.random((B, K + 1), dtype=np.float32)).to(dev, non_blocking=True)
        short = self._begin()
        a = torch.empty(B, K + 1, m.V, dtype=m.dev[1].dtype, device=dev)
        d = torch.empty(B, K, dtype=torch.int32, device=dev)
        q = torch.empty(B, K, dtype=torch.float32, device=dev)
        for i in range(K + 1):
            a[:, i] = m.dev[1].index_select(0, self._drafter_rows(i, d[:, i - 1] if i > 0 else None))
            self._shape(a[:, i:i + 1], d[:, :i], i)
            if i < K:
                asp.draw_tokens(a[:, i], self.tau, ud[:, i], out=(d[:, i], q[:, i]))
        t, b = (m.dev[k].index_select(0, rows.reshape(-1)).view(B, K + 1, m.V)
                for k, rows in zip((0, 2), self._view_rows()))
        for x in (t, b):
            self._shape(x, d, 0)
        acc, nxt, _ = asp.fuse_verify(t, a, b, d, q, u, self.tau, **self.kw)
        acc = torch.where(short != 0, -1, acc)                 # no room: the step does not count
        live = (acc >= 0) & (self.finished == 0)
        _, _, tokens, n = asp.commit_tokens(acc, nxt, d, self.history, self.lengths, self.finished, self.stop,
                                            out=(self.lengths, self.finished,
                                                 torch.empty(B, K + 1, dtype=torch.int32, device=dev),
                                                 torch.empty_like(acc)))
        j = acc.clamp_min(0).long()[:, None]
        self._end(live, j, nxt, tokens, n)
        ok = live.long()
        self.counts += torch.stack([(ok * j[:, 0]).sum(), (ok * (j[:, 0] + (acc < K))).sum(), n.sum()])
        self.request_steps += ok.sum()
        self.steps += 1
        return acc, nxt, tokens

    def tokens(self):
        """The committed tokens of every request (copies to the host)."""
        n = self.lengths.tolist()
        return [row[:k] for row, k in zip(self.history.tolist(), n)]

    def report(self):
        accepted, evaluated, committed = self.counts.tolist()
        n = int(self.request_steps)
        return {"steps": self.steps, "requests": self.B, "K": self.K,
                "AR": accepted / evaluated if evaluated else float("nan"),
                "MAL": committed / n if n else float("nan"),
                "tokens": committed, "finished": int((self.finished != 0).sum())}


class AttentionModels(TableModels):
    """Stand-ins whose logit rows are chosen by attention: a token has a query of `heads`
    and a key and value of `kv_heads` heads (random tables, float32), and the row behind a
    position is that of the anchor nearest to the position's answer (the largest
    product)."""

    def __init__(self, V: int, R: int = 512, heads: int = 8, kv_heads: int = 2, dim: int = 64, device=None, seed: int = 0,
                 **kw):
        import torch
        import paper_2608_26004_amd as asp
        super().__init__(V, R=R, device=device, seed=seed, **kw)
        if device is None:
            raise ValueError("the attention's tables need a device")
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.qkv = torch.randn(V, heads + 2 * kv_heads, dim, device=device, generator=g)
        self.anchors = torch.randn(R, heads * dim, device=device, generator=g)
        self.frequencies = asp.rotary_frequencies(dim, device=device)

    def rows(self, answers):
        """Table rows of answers [B, n, heads, dim]."""
        return (answers.flatten(2) @ self.anchors.T).argmax(-1)


class CachedDecoder(ResidentDecoder):
    """ResidentDecoder over AttentionModels: the drafter's keys and values in `bits` bits,
    the verifier's in `verifier_bits`, in the same blocks.  The tokens of a request stand
    at the positions of its history, behind its start token; a step writes the last
    committed token and its drafts, and what is rejected is written over by the next one.

    window: positions that the verifier and the drafter's compressed view see (0: all)."""

    def __init__(self, models: AttentionModels, B: int, K: int, temperature, bits: int = 4, verifier_bits: int = 8,
                 window: int = 0, **kw):
        super().__init__(models, B, K, temperature, **kw)
        torch, asp, m = self._torch, self._asp, models
        blocks = len(self.ring)
        self.caches = [asp.new_cache(blocks, m.kv_heads, self.block_size, m.dim, n, device=self.device)
                       for n in (bits, verifier_bits)]
        self.window = window
        self.last = (torch.arange(B, device=self.device) % m.V).int()       # the start tokens

    def _begin(self):
        m = self.m
        self.slots, short = self._place(self.lengths, self.K + 1)
        self.turned = self._torch.empty(self.B, self.K + 1, m.heads + m.kv_heads, m.dim, device=self.device)
        self.values = self._torch.empty(self.B, self.K + 1, m.kv_heads, m.dim, device=self.device)
        self.a_rows = []
        return short

    def _drafter_rows(self, i, token):
        asp, m = self._asp, self.m
        x = m.qkv[(self.last if i == 0 else token).long()][:, None]
        at = self.lengths + i
        q, k = self.turned[:, i:i + 1].split([m.heads, m.kv_heads], 2)
        asp.rotate_heads(x[:, :, :m.heads], x[:, :, m.heads:m.heads + m.kv_heads], at, m.frequencies, out=(q, k))
        self.values[:, i] = x[:, 0, m.heads + m.kv_heads:]
        asp.write_cache(k, self.values[:, i:i + 1], self.slots[:, i:i + 1].contiguous(), self.caches[0])
        self.a_rows.append(m.rows(asp.attend_cache(q, self.caches[0], self.table, at))[:, 0])
        return self.a_rows[-1]

    def _view_rows(self):
        asp, m = self._asp, self.m
        q, k = self.turned.split([m.heads, m.kv_heads], 2)
        asp.write_cache(k, self.values, self.slots, self.caches[1])
        t, b = (m.rows(asp.attend_cache(q, c, self.table, self.lengths, window=self.window)) for c in reversed(self.caches))
        self.t_rows, self.b_rows = t, b
        return t, b

    def _end(self, live, j, nxt, tokens, n):
        last = tokens.gather(1, (n.long() - 1).clamp_min(0)[:, None])[:, 0]
        self.last = self._torch.where(n > 0, last, self.last)


def main(argv=None):
    ap = argparse.ArgumentParser(description="multi-step speculative decoding over stand-in models")
    ap.add_argument("--B", type=int, default=8)
    ap.add_argument("--K", type=int, default=2)
    ap.add_argument("--V", type=int, default=32000)
    ap.add_argument("--R", type=int, default=512)
    ap.add_argument("--rho", type=float, default=1.0)
    ap.add_argument("--tau", type=float, default=0.0)
    ap.add_argument("--beta", type=float, default=1.0)
    ap.add_argument("--gamma", type=float, default=0.5)
    ap.add_argument("--steps", type=int, default=50)
    ap.add_argument("--dtype", choices=[synth.BF16, synth.FP32], default=synth.BF16)
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--gate", choices=["cda", "fixed", "kl", "lambda"], default="cda")
    ap.add_argument("--early-exit", type=int, default=0)
    ap.add_argument("--resident", action="store_true", help="draft, commit and place on the GPU")
    for name in ("repetition", "frequency", "presence"):
        ap.add_argument("--" + name, type=float, default=None, help="penalty (with --resident)")
    ap.add_argument("--cache", type=int, choices=[4, 8], default=None,
                    help="keys and values of the drafter in so many bits (with --resident)")
    ap.add_argument("--window", type=int, default=0, help="positions that the compressed views see (with --cache)")
    args = ap.parse_args(argv)
    penalties = {n: getattr(args, n) for n in ("repetition", "frequency", "presence")}
    if not args.resident and any(v is not None for v in penalties.values()):
        ap.error("penalties need --resident")
    if args.cache is not None and not args.resident:
        ap.error("--cache needs --resident")
    if args.window and args.cache is None:
        ap.error("--window needs --cache")
    import torch
    dev = torch.device("cuda")
    kind = TableModels if args.cache is None else AttentionModels
    models = kind(args.V, R=args.R, rho=args.rho, dtype=args.dtype, seed=args.seed, device=dev)
    gm = {"cda": 0, "fixed": 1, "kl": 2, "lambda": 3}[args.gate]
    if args.resident:
        kw = dict(beta=args.beta, gamma=args.gamma, gate_mode=gm, seed=args.seed + 1, early_exit=args.early_exit,
                  max_tokens=args.steps * (args.K + 1) + 1, **penalties)
        if args.cache is None:
            dec = ResidentDecoder(models, args.B, args.K, args.tau, **kw)
        else:
            dec = CachedDecoder(models, args.B, args.K, args.tau, bits=args.cache, window=args.window, **kw)
    else:
        dec = SpecDecoder(models, args.B, args.K, args.tau, beta=args.beta, gamma=args.gamma,
                          gate_mode=gm, seed=args.seed + 1, device=dev, early_exit=args.early_exit)
    t0 = time.perf_counter()
    for _ in range(args.steps):
        dec.step()
    torch.cuda.synchronize()
    wall = time.perf_counter() - t0
    rep = dec.report()
    rep.update({"V": args.V, "tau": args.tau, "beta": args.beta, "gamma": args.gamma,
                "rho": args.rho, "gate": args.gate, "early_exit": args.early_exit, "wall_s": wall})
    if args.resident:
        rep.update({"resident": True, **{k: v for k, v in penalties.items() if v is not None}})
    if args.cache is not None:
        rep.update({"cache_bits": args.cache, "window": args.window})
    print(json.dumps(rep))


if __name__ == "__main__":
    main()
