"""Plain 64-bit statement of the calls for token-generating experts (include/coe.h, "paged key/value cache" and "decoders that look at an
encoder's states, and search with beams").  numpy only."""
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


def rotate(x, position, frequency, rotated, neighbours):
    """x [tokens][heads][dim] float64.  Returns the rotated rows and |a| + |b| of every channel's pair (0 where it is not rotated)."""
    out, size, half = np.array(x), np.zeros_like(x), rotated // 2
    angle = position.astype(np.float64)[:, None] * frequency.astype(np.float64)[None, :]
    cos, sin = np.cos(angle)[:, None], np.sin(angle)[:, None]
    first = slice(0, rotated, 2) if neighbours else slice(0, half)
    second = slice(1, rotated, 2) if neighbours else slice(half, rotated)
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * cos - b * sin, b * cos + a * sin
    size[..., first] = size[..., second] = np.abs(a) + np.abs(b)
    return out, size


def cross(q, k, v, q_off, first, length, beams, scale, seen=None, max_new=None, max_rows=None):
    """q [tokens][heads][dim]; k, v [rows][kv_heads][dim]: float64.  Returns out, lse, A = sum of p |v| (for error bounds) and which tokens are
    served."""
    tokens, heads, dim = q.shape
    group = heads // k.shape[1]
    out = np.zeros((tokens, heads, dim)); size = np.zeros((tokens, heads, dim)); lse = np.full((tokens, heads), -np.inf)
    served = np.zeros(tokens, bool)
    for s in range(len(first)):
        begin, end = int(q_off[s * beams]), int(q_off[(s + 1) * beams])
        end = end if max_new is None else min(end, begin + max_new)
        served[begin:end] = True
        f, n = int(first[s]), int(length[s])
        n = 0 if f < 0 else max(0, min(n, len(k) - f, n if max_rows is None else max_rows))
        rows = np.arange(f, f + n)
        if seen is not None:
            rows = rows[seen[rows] != 0]
        if len(rows) == 0:
            continue
        for h in range(heads):
            kk, vv = k[rows, h // group], v[rows, h // group]
            x = scale * (q[begin:end, h] @ kk.T)
            top = x.max(1, keepdims=True)
            e = np.exp(x - top)
            lse[begin:end, h] = (top + np.log(e.sum(1, keepdims=True)))[:, 0]
            out[begin:end, h] = e @ vv / e.sum(1, keepdims=True)
            size[begin:end, h] = e @ np.abs(vv) / e.sum(1, keepdims=True)
    return out, lse, size, served


def beam(x, score, ended, beams, picks, end_token):
    """x [rows][vocab] float64 logits.  Returns (scores, rows, tokens, ended), each [requests][picks], scores float64."""
    requests = len(x) // beams
    out = []
    for r in range(requests):
        found = []
        for row in range(r * beams, (r + 1) * beams):
            s = float(score[row])
            if not s > -np.inf:
                continue
            if ended is not None and ended[row]:
                found.append((-s, row, 0, int(end_token), 1))
                continue
            z = np.where(np.isnan(x[row]), -np.inf, x[row])
            top = z.max()
            if top == -np.inf:
                continue
            with np.errstate(invalid="ignore"):
                z = np.where(z == top, 0.0, np.where(np.isinf(z - top), -np.inf, z - top))
            z = z - np.log(np.exp(z).sum())
            likely = np.argsort(-z, kind="stable")[:picks]
            found += [(-(s + z[t]), row, place, int(t), int(t == end_token)) for place, t in enumerate(likely) if z[t] > -np.inf]
        found = sorted(found)[:picks]
        out.append([(-c[0], c[1], c[3], c[4]) for c in found] + [(-np.inf, -1, -1, 0)] * (picks - len(found)))
    out = np.array(out, np.float64).reshape(requests, picks, 4)
    return out[..., 0], *(out[..., i].astype(np.int32) for i in (1, 2, 3))


def fork(block, n_blocks, beams, parent, seq_len, ring, state, table, next_table):
    """Rows that continue others, request by request.  Returns dict of the outputs; next_table and ring as they are afterwards."""
    ring, next_table = ring.copy(), next_table.copy()
    n, width = table.shape
    head, count = int(state[0]) % n_blocks, min(max(int(state[1]), 0), n_blocks)
    length = np.clip(seq_len, 0, width * block).astype(np.int32)
    copy, next_len = np.full((n, 2), -1, np.int32), np.zeros(n, np.int32)
    taken, given, forked = 0, [], None
    for r in range(n // beams):
        rows = list(range(r * beams, (r + 1) * beams))
        child_of = {i: int(parent[i]) if int(parent[i]) in rows else None for i in rows}
        continued = [p for p in rows if p in child_of.values()]
        owned = {p: -(-int(length[p]) // block) for p in rows}
        inside = lambda b: 0 <= b < n_blocks
        free, seen_parents, copies = [], set(), []
        for j in range(width):
            held = {int(table[p, j]) for p in continued if j < owned[p]}
            for p in rows:
                b = int(table[p, j])
                if p not in continued and j < owned[p] and b not in held and inside(b):
                    held.add(b)
                    free.append(b)
        for i in rows:
            p = child_of[i]
            if p in seen_parents and length[p] % block and inside(int(table[p, owned[p] - 1])):
                copies.append(i)
            seen_parents.add(p if p is not None else -1)
        if forked is None and taken + max(0, len(copies) - len(free)) > count:
            forked = r
        for i in rows:
            p = child_of[i] if forked is None else i
            if p is None:
                continue
            next_len[i] = length[p]
            next_table[i, :owned[p]] = table[p, :owned[p]]
            if forked is None and i in copies:
                if free:
                    to = free.pop(0)
                else:
                    to = ring[(head + taken) % n_blocks]
                    taken += 1
                copy[i] = table[p, owned[p] - 1], to
                next_table[i, owned[p] - 1] = to
        given += free if forked is None else []
    for i, b in enumerate(given):
        ring[(head + count + i) % n_blocks] = b
    state = [(head + taken) % n_blocks, count - taken + len(given), n // beams if forked is None else forked, int((copy[:, 0] >= 0).sum())]
    return dict(next_table=next_table, next_len=next_len, copy=copy, ring=ring, next_state=np.array(state, np.int32))
