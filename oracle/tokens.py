"""Plain 64-bit statement of the calls for token-generating experts (include/coe.h, "paged key/value cache").  numpy only."""
import numpy as np


def bf16_to_f64(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def plan(block, n_blocks, max_blocks, token_cap, have, add, ring, state, table):
    """One step, request by request.  Returns dict of the outputs; table and ring as they are afterwards."""
    ring, table = ring.copy(), table.copy()
    head, count = int(state[0]), int(state[1])
    limit = max_blocks * block
    seq_len, q_off, slot, position = [], [0], [], []
    taken = back = 0
    closed = None
    for r, (h, a) in enumerate(zip(have, add)):
        h, a = min(max(int(h), 0), limit), int(a)
        owned = -(-h // block)
        if a < 0:
            for j in range(owned):
                ring[(head + count + back + j) % n_blocks] = table[r, j]
            back += owned
            seq_len.append(0)
        else:
            need = -(-(h + a) // block) - owned
            if closed is None and (taken + need > count or len(slot) + a > token_cap or h + a > limit):
                closed = r
            if closed is not None:
                a = need = 0
            for j in range(need):
                table[r, owned + j] = ring[(head + taken + j) % n_blocks]
            taken += need
            for p in range(h, h + a):
                position.append(p)
                b = int(table[r, p // block])
                slot.append(b * block + p % block if 0 <= b < n_blocks else -1)
            seq_len.append(h + a)
        q_off.append(len(slot))
    n = len(slot)
    pad = [-1] * (token_cap - n)
    out = dict(seq_len=seq_len, q_off=q_off, slot=slot + pad, position=position + pad,
               next_state=[(head + taken) % n_blocks, count - taken + back, len(have) if closed is None else closed, n])
    out = {k: np.asarray(v, np.int64).astype(np.int32) for k, v in out.items()}
    out.update(table=table, ring=ring)
    return out


def attention(q, k, v, seq_len, q_off, table, block, window, scale):
    """q [tokens][heads][dim]; k, v [blocks][block][kv_heads][dim]: float64.  Returns out, lse and A = sum of p |v| (for error bounds)."""
    tokens, heads, dim = q.shape
    kv = k.shape[2]
    out = np.zeros((tokens, heads, dim)); size = np.zeros((tokens, heads, dim)); lse = np.full((tokens, heads), -np.inf)
    for r in range(len(seq_len)):
        m = q_off[r + 1] - q_off[r]
        for i in range(m):
            t, pos = q_off[r] + i, seq_len[r] - m + i
            first = max(0, int(pos) - window + 1) if window > 0 else 0
            if pos < 0:
                continue
            j = np.arange(first, pos + 1)
            ids, rows = table[r, j // block], j % block
            known = (ids >= 0) & (ids < k.shape[0])
            ids = np.where(known, ids, 0)
            kk = np.where(known[:, None, None], k[ids, rows], 0.0)
            vv = np.where(known[:, None, None], v[ids, rows], 0.0)
            for h in range(heads):
                g = h // (heads // kv)
                s = scale * (kk[:, g] @ q[t, h])
                top = s.max()
                e = np.exp(s - top)
                lse[t, h] = top + np.log(e.sum())
                out[t, h] = e @ vv[:, g] / e.sum()
                size[t, h] = e @ np.abs(vv[:, g]) / e.sum()
    return out, lse, size


def sample(x, temperature, top_k, top_p, min_p, noise, slack=0.0):
    """One row of float64 logits.  Returns (admissible tokens, ln probabilities of all tokens).  slack: scores that far from the best
    and weights that near a cut (relative) count as admissible; 0 gives the one token of the definition."""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    if top == -np.inf:
        return {-1}, None
    greedy = not temperature > 0 or noise is None
    t = temperature if temperature > 0 else 1.0
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        z = np.where(x == top, 0.0, np.where(np.isinf(x - top), -np.inf, (x - top) / t))
        w = np.exp(z)
        ln = z - np.log(w.sum())
        order = np.argsort(-x, kind="stable")
        order = order[x[order] > -np.inf]
        first = int(order[0])
        if greedy:
            return {first}, ln
        kept = order[:top_k] if 0 < top_k < len(x) else order
        mass = w[kept].sum()
        before = np.cumsum(w[kept]) - w[kept]

        def race(grace):
            ok = np.ones(len(kept), bool)
            if top_p < 1:
                ok &= before < top_p * mass * (1 + grace)
            if min_p > 0:
                ok &= w[kept] >= min_p * (1 - grace)
            ok[0] = True
            ids = kept[ok]
            e = noise[ids].astype(np.float64)
            score = z[ids] - np.log(e)
            score[np.isnan(score) | (e < 0)] = -np.inf
            return ids, score
        ids, score = race(slack)
        strict, strict_score = race(-slack)
        if strict_score.max() == -np.inf:
            return {first} | set(int(i) for i in ids[score > -np.inf]), ln
        best = strict_score.max()
        if slack == 0:
            return {int(ids[score == best].min())}, ln
        near = {int(i) for i in ids[score >= best - slack]} if np.isfinite(best) else {int(ids[score == best].min())}
    return near, ln
