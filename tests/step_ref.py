"""Plain references of the operators around the decision step: loops over
requests and tokens in NumPy, in 64 bits, from the definitions in
include/asymspec_step.h."""

import numpy as np


def shape_logits(x, history=None, lengths=None, prompt_lengths=None, drafts=None, repetition=None,
                 frequency=None, presence=None, bias_ids=None, bias_values=None, mask=None, mask_index=None,
                 id_map=None):
    """(shaped logits in fp64, bound on the rounding of an fp32 evaluation).

    The bound: each of the at most five fp32 operations is off by half a step of
    its result, u = 2^-24 relative; a step's error passes to the result at most
    unchanged (the later steps add), so u times the sum of the intermediates'
    magnitudes, doubled for terms of second order."""
    B, R, V = x.shape
    v = x.astype(np.float64).copy()
    err = np.zeros_like(v)
    D = 0 if drafts is None else drafts.shape[1]

    def ids(t):
        t = np.asarray(t, np.int64)
        if id_map is not None:
            ok = (t >= 0) & (t < len(id_map))
            t = np.where(ok, id_map[np.where(ok, t, 0)] if len(id_map) else -1, -1)
        return t[(t >= 0) & (t < V)]

    for b in range(B):
        n = 0 if history is None else int(np.clip(lengths[b], 0, history.shape[1]))
        p = 0 if prompt_lengths is None else int(np.clip(prompt_lengths[b], 0, n))
        rep, freq, pres = (float(d if a is None else a[b]) for a, d in
                           ((repetition, 1.0), (frequency, 0.0), (presence, 0.0)))
        bias = {}
        if bias_ids is not None:
            for k, t in enumerate(bias_ids[b]):
                if 0 <= t < V:
                    bias[int(t)] = float(bias_values[b][k])
        for r in range(R):
            out = [] if history is None else list(ids(history[b, p:n]))
            if D:
                out += list(ids(drafts[b, :D - (R - 1) + r]))
            count = np.zeros(V, np.int64)
            np.add.at(count, np.asarray(out, np.int64), 1)
            seen = count > 0
            if history is not None:
                seen[ids(history[b, :p])] = True
            w, e = v[b, r], err[b, r]
            with np.errstate(all="ignore"):
                w[seen] = np.where(w[seen] > 0, w[seen] / rep, w[seen] * rep)
                e[seen] += np.abs(w[seen])
                c = count > 0
                sub = freq * count[c]
                w[c] = w[c] - sub
                e[c] += np.abs(sub) + np.abs(w[c])
                w[c] = w[c] - pres
                e[c] += np.abs(w[c])
                for t, val in bias.items():
                    w[t] += val
                    e[t] += np.abs(w[t])
            if mask is not None and 0 <= mask_index[b, r] < len(mask):
                bits = np.unpackbits(mask[mask_index[b, r]].astype("<u4").view(np.uint8), bitorder="little")[:V]
                w[bits == 0] = -np.inf
    return v, 2.0 * 2.0 ** -24 * err


def draw_tokens(x, tau, u):
    """(token, q in fp64, distance of u from the nearest step of the token's
    interval) of each row."""
    N, V = x.shape
    tok, q, near = np.zeros(N, np.int64), np.zeros(N), np.full(N, np.inf)
    for n in range(N):
        l = x[n].astype(np.float64)
        l[np.isnan(l)] = -np.inf
        m = l.max()
        if m == -np.inf:
            continue
        if not tau[n] > 0:
            tok[n], q[n] = int(np.argmax(l)), 1.0
            continue
        w = np.zeros(V)
        live = l > -np.inf
        with np.errstate(all="ignore"):
            far = np.isneginf(l[live] - m)        # below +inf: no weight at any temperature
            w[live] = np.where(l[live] == m, 1.0, np.where(far, 0.0, np.exp((l[live] - m) / np.float64(tau[n]))))
        c = np.cumsum(w)
        uu = float(u[n]) if u[n] > 0 else 0.0
        over = np.nonzero((c > uu * c[-1]) & (w > 0))[0]
        k = int(over[0]) if len(over) else int(np.nonzero(w > 0)[0][-1])
        tok[n], q[n] = k, w[k] / c[-1]
        if 0.0 < uu < 1.0:
            near[n] = min(abs(c[k] / c[-1] - uu), abs((c[k] - w[k]) / c[-1] - uu))
    return tok, q, near


def commit_tokens(accept_len, next_token, drafts, history, lengths, finished=None, stops=(), max_lengths=None):
    B, K = drafts.shape
    L = history.shape[1]
    hist = history.copy()
    new, fin, toks, counts = lengths.copy(), np.zeros(B, np.int32), np.full((B, K + 1), -1, np.int32), np.zeros(B, np.int32)
    for b in range(B):
        done = finished is not None and finished[b] != 0
        valid = 0 <= accept_len[b] <= K
        limit = L if max_lengths is None else min(max(int(max_lengths[b]), 0), L)
        n, stopped = 0, False
        if valid and not done and lengths[b] >= 0:
            for t in list(drafts[b, :accept_len[b]]) + [next_token[b]]:
                if lengths[b] + n >= limit:
                    break
                hist[b, lengths[b] + n] = t
                toks[b, n] = t
                n += 1
                if t in stops:
                    stopped = True
                    break
        new[b] = lengths[b] + n
        counts[b] = n
        fin[b] = done or stopped or (valid and new[b] >= limit)
    return new, fin, toks, counts, hist


def plan_slots(lengths, new_tokens, table, n_blocks, ring, state, bs, width=0, total=0, release=None):
    """The sequential statement: request after request takes from the ring's
    front; what is given back is collected and joins its end afterwards."""
    B, top = table.shape
    N = len(ring)
    table, ring = table.copy(), ring.copy()
    head, count = int(state[0]) % N, int(np.clip(state[1], 0, N))
    front = [int(ring[(head + i) % N]) for i in range(count)]
    took, back = 0, []
    short, after = np.zeros(B, np.int32), np.zeros(B, np.int32)
    rows = []
    asked = 0
    for b in range(B):
        gone = release is not None and release[b] != 0
        n = width if new_tokens is None else max(int(new_tokens[b]), 0)
        if width:
            n = min(n, width)
        n = 0 if gone else n
        ln = max(int(lengths[b]), 0)
        need = 0 if gone else -(-(ln + n) // bs)
        held = int(np.clip(n_blocks[b], 0, top))
        after[b] = held
        if need > top:
            short[b] = 1
        elif need > held:
            asked += need - held
            if asked > count:
                short[b] = 1
            else:
                table[b, held:need] = front[took:took + need - held]
                took += need - held
                after[b] = need
        else:
            back += list(table[b, need:held])
            table[b, need:held] = -1
            after[b] = need
        rows.append([-1 if short[b] else int(table[b, (ln + j) // bs]) * bs + (ln + j) % bs for j in range(n)])
    for i, x in enumerate(back[:N - count]):
        ring[(head + count + i) % N] = x
    new_state = np.array([(head + took) % N, count - took + len(back[:N - count])], np.int32)
    starts = np.concatenate([[0], np.cumsum([len(r) for r in rows])]).astype(np.int32)
    if width:
        slots = np.full((B, width), -1, np.int64)
        for b, r in enumerate(rows):
            slots[b, :len(r)] = r
    else:
        flat = [s for r in rows for s in r][:total]
        slots = np.array(flat + [-1] * (total - len(flat)), np.int64)
    return slots, short, after, new_state, starts, table, ring
