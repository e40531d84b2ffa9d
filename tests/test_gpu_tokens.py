"""The calls for token-generating experts against their 64-bit statement: lengths, masks, layouts and values where they can go wrong."""
import math

import numpy as np
import pytest

from oracle import tokens as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_02354_amd import binding
    return binding


def _dev(a):
    import torch
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view(np.int16) if a.dtype == np.uint16 else a).cuda()


def _bf16(a):
    """Round float64 to bf16 bits (to nearest even)."""
    b = np.asarray(a, np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def _stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


# ---- plan -------------------------------------------------------------------------------------------------------
def _plan_gpu(B, block, n_blocks, max_blocks, cap, have, add, ring, state, table):
    import torch
    n = len(have)
    d = dict(have=_dev(np.asarray(have, np.int32)), add=_dev(np.asarray(add, np.int32)), ring=_dev(ring), state=_dev(np.asarray(state, np.int32)),
             table=_dev(table))
    out = {k: torch.full((size,), -77, dtype=torch.int32, device="cuda") for k, size in
           (("seq_len", max(n, 1)), ("q_off", n + 1), ("slot", max(cap, 1)), ("position", max(cap, 1)), ("next_state", 4))}
    B.coe_kv_plan(n, block, n_blocks, max_blocks, cap, *(d[k].data_ptr() for k in ("have", "add", "ring", "state", "table")),
                  *(out[k].data_ptr() for k in ("seq_len", "q_off", "slot", "position", "next_state")), _stream())
    got = {k: v.cpu().numpy() for k, v in out.items()}
    got["seq_len"], got["slot"], got["position"] = got["seq_len"][:n], got["slot"][:cap], got["position"][:cap]
    got["table"], got["ring"] = d["table"].cpu().numpy(), d["ring"].cpu().numpy()
    return got


def _pool(rng, have, block, n_blocks, max_blocks):
    """Random tables for `have` cached tokens, the rest of the ids in a ring that starts anywhere."""
    order = rng.permutation(n_blocks).astype(np.int32)
    table = np.full((len(have), max_blocks), -9, np.int32)
    at = 0
    for r, h in enumerate(have):
        b = -(-int(h) // block)
        table[r, :b] = order[at:at + b]
        at += b
    assert at <= n_blocks
    head = int(rng.integers(n_blocks))
    ring = np.full(n_blocks, -5, np.int32)
    ring[(head + np.arange(n_blocks - at)) % n_blocks] = order[at:]
    return table, ring, [head, n_blocks - at]


@pytest.mark.parametrize("n,block,most,new,done,spare,cap", [
    (0, 16, 1, 1, 0.0, 3, 4),            # no requests: offsets and state all the same
    (1, 8, 40, 1, 0.0, 3, 1),
    (1, 8, 0, 9000, 0.0, 2000, 9000),    # one long prompt, many workgroups
    (7, 16, 100, 40, 0.3, 200, 500),
    (255, 16, 300, 1, 0.1, 300, 256), (256, 32, 300, 2, 0.1, 600, 600), (257, 64, 300, 70, 0.1, 600, 20000),
    (300, 16, 64, 33, 0.0, 100, 20000),  # the pool runs out part of the way
    (300, 16, 64, 33, 0.2, 4000, 1000),  # the token room runs out
    (1000, 16, 64, 0, 0.0, 0, 10),       # nothing grows
    (16384, 8, 30, 3, 0.05, 16384, 60000),
])
def test_plan(B, n, block, most, new, done, spare, cap):
    rng = np.random.default_rng(n + block + most)
    have = rng.integers(0, most + 1, n).astype(np.int32)
    add = rng.integers(0, new + 1, n).astype(np.int32) if new > 1 else np.full(n, new, np.int32)
    add[rng.random(n) < done] = -1
    if new == 9000:
        add[:] = 9000
    max_blocks = -(-(most + new) // block) + 1
    n_blocks = int(sum(-(-have // block))) + spare + 1 if n else spare
    n_blocks = int((-(-have // block)).sum()) + spare + 1
    table, ring, state = _pool(rng, have, block, n_blocks, max_blocks)
    want = T.plan(block, n_blocks, max_blocks, cap, have, add, ring, state, table)
    got = _plan_gpu(B, block, n_blocks, max_blocks, cap, have, add, ring, state, table)
    for k in want:
        assert np.array_equal(got[k], want[k]), k


def test_plan_values_out_of_range(B):
    """Negative and overlong lengths, a request too long for its row, sums beyond 32 bits: clamped or refused, never followed."""
    block, n_blocks, max_blocks = 16, 50, 4
    have = np.array([-5, 30, 1000, 10, 3, 20], np.int32)
    add = np.array([3, 2, -1, 55, 1, -7], np.int32)
    rng = np.random.default_rng(0)
    table = rng.permutation(n_blocks)[:24].reshape(6, 4).astype(np.int32)
    ring = rng.permutation(n_blocks).astype(np.int32)
    for state in ([48, 20], [0, 0]):
        want = T.plan(block, n_blocks, max_blocks, 9, have, add, ring, state, table)
        assert want["next_state"][2] == (3 if state[1] else 0)
        got = _plan_gpu(B, block, n_blocks, max_blocks, 9, have, add, ring, state, table)
        for k in want:
            assert np.array_equal(got[k], want[k]), k
    add = np.full(6, 2 ** 31 - 1, np.int32)
    want = T.plan(block, n_blocks, max_blocks, 9, have, add, ring, [3, 20], table)
    got = _plan_gpu(B, block, n_blocks, max_blocks, 9, have, add, ring, [3, 20], table)
    for k in want:
        assert np.array_equal(got[k], want[k]), k


def test_plan_many_steps_conserve_blocks(B):
    """A service that runs for a while: outputs of a step are the inputs of the next; no block is lost or owned twice."""
    rng = np.random.default_rng(5)
    n, block, n_blocks, max_blocks, cap = 40, 8, 300, 32, 400
    have = np.zeros(n, np.int32)
    table, ring, state = _pool(rng, have, block, n_blocks, max_blocks)
    refused = 0
    for _ in range(60):
        add = np.where(have == 0, rng.integers(0, 60, n), 1).astype(np.int32)
        add[(have > 0) & (rng.random(n) < 0.08)] = -1
        add[have + np.maximum(add, 0) > max_blocks * block] = -1
        want = T.plan(block, n_blocks, max_blocks, cap, have, add, ring, state, table)
        got = _plan_gpu(B, block, n_blocks, max_blocks, cap, have, add, ring, state, table)
        for k in want:
            assert np.array_equal(got[k], want[k]), k
        refused += got["next_state"][2] < n
        have, table, ring, state = got["seq_len"], got["table"], got["ring"], got["next_state"][:2]
        owned = np.concatenate([table[r, :-(-int(h) // block)] for r, h in enumerate(have)])
        free = ring[(state[0] + np.arange(state[1])) % n_blocks]
        assert sorted(np.concatenate([owned, free]).tolist()) == list(range(n_blocks))
    assert refused > 0


# ---- append -----------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("tokens,kv,dim,block,layout", [(1, 1, 8, 8, "token"), (3, 12, 64, 16, "head"), (100, 5, 80, 32, "pair"), (257, 8, 128, 64, "token"),
                                                        (33, 40, 128, 16, "head"), (2000, 2, 24, 1024, "token")])
def test_append(B, tokens, kv, dim, block, layout):
    """Every row lands in its slot, bit for bit (NaN bits too); padding and slots outside the cache are skipped; nothing else changes."""
    import torch
    rng = np.random.default_rng(tokens)
    n_blocks = -(-tokens // block) + 2
    new = rng.integers(0, 65536, (tokens, 3 * kv, dim)).astype(np.uint16)
    slots = rng.permutation(n_blocks * block)[:tokens].astype(np.int32)
    skip = rng.random(tokens) < 0.2
    slot = np.where(skip, rng.choice([-1, -2 ** 31, n_blocks * block, 2 ** 31 - 1], tokens), slots).astype(np.int32)
    k, v, cache = _make_cache(B, rng.integers(0, 65536, (2, n_blocks, block, kv, dim)).astype(np.uint16), layout)
    want = [k.cpu().numpy().view(np.uint16).copy(), v.cpu().numpy().view(np.uint16).copy()]
    for i, w in enumerate(want):
        for t in np.nonzero(~skip)[0]:
            w[slots[t] // block, slots[t] % block] = new[t, (1 + i) * kv:(2 + i) * kv]
    d, s = _dev(new), _dev(slot)
    B.coe_kv_append(cache, tokens, d.data_ptr() + 2 * kv * dim, 3 * kv * dim, dim, d.data_ptr() + 4 * kv * dim, 3 * kv * dim, dim, s.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert np.array_equal(k.cpu().numpy().view(np.uint16), want[0]) and np.array_equal(v.cpu().numpy().view(np.uint16), want[1])


def _make_cache(B, bits, layout):
    """bits [2][blocks][block][kv][dim] -> (k, v as [block][token][head][channel] views, the struct)."""
    import torch
    _, n_blocks, block, kv, dim = bits.shape
    if layout == "token":
        k, v = _dev(bits[0]), _dev(bits[1])
    elif layout == "head":
        k, v = (_dev(b.transpose(0, 2, 1, 3)).permute(0, 2, 1, 3) for b in bits)
    elif layout == "pair":                      # key and value of a token side by side
        both = _dev(bits.transpose(1, 2, 0, 3, 4))
        k, v = both[:, :, 0], both[:, :, 1]
    else:                                       # blocks innermost but for the channels
        k, v = (_dev(b.transpose(2, 1, 0, 3)).permute(2, 1, 0, 3) for b in bits)
    s = k.stride()
    assert s == v.stride()
    return k, v, B.coe_kv_cache(B.COE_DT_BF16, n_blocks, block, kv, dim, k.data_ptr(), v.data_ptr(), s[0], s[1], s[2])


# ---- attention --------------------------------------------------------------------------------------------------
class Attend:
    """Inputs of a call from a list of (cached tokens, new tokens) and a device run of it."""

    def __init__(self, B, lengths, heads, kv, dim, block=16, window=0, layout="token", seed=0, scale=None, sharp=1.0, gaps=False):
        self.B, self.heads, self.kv, self.dim, self.block, self.window, self.layout = B, heads, kv, dim, block, window, layout
        rng = np.random.default_rng(seed)
        self.scale = scale if scale is not None else 1 / math.sqrt(dim)
        self.total = np.array([h + m for h, m in lengths], np.int32)
        self.new = np.array([m for _, m in lengths], np.int32)
        self.off = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        owned = [-(-max(int(t), 0) // block) for t in self.total]
        self.n_blocks = sum(owned) + 3
        order = rng.permutation(self.n_blocks).astype(np.int32)
        self.max_blocks = max(owned) + 2
        self.table = rng.integers(-3, self.n_blocks + 3, (len(lengths), self.max_blocks)).astype(np.int32)     # unused entries: anything
        at = 0
        for r, b in enumerate(owned):
            self.table[r, :b] = order[at:at + b]
            at += b
        tokens = int(self.off[-1])
        self.q = _bf16(sharp * rng.standard_normal((tokens, heads, dim)))
        self.bits = np.full((2, self.n_blocks, block, kv, dim), 0x7FC0, np.uint16)      # rows nobody has written: NaN
        for r, t in enumerate(self.total):
            for j in range(max(int(t), 0)):
                self.bits[:, self.table[r, j // block], j % block] = _bf16(rng.standard_normal((2, kv, dim)))

    def at(self, r, j):
        return self.table[r, j // self.block], j % self.block

    def run(self, max_new=None, lse=True, extra=0, poison=0xFFC0):
        import torch
        B, tokens = self.B, int(self.off[-1])
        k, v, cache = _make_cache(B, self.bits, self.layout)
        q = _dev(np.concatenate([self.q, self.q[:, :2]], 1))         # rows farther apart than they are long
        out = _dev(np.full((tokens + extra, self.heads + 1, self.dim), poison, np.uint16))
        logs = torch.full((tokens + extra, self.heads), 7.5, device="cuda")
        most = int(self.new.max()) if max_new is None else max_new
        need = B.coe_kv_attention_workspace(len(self.new), tokens + extra, most, self.heads, self.kv, self.dim)
        work = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        off, total, table = _dev(self.off), _dev(self.total), _dev(self.table)
        if extra:
            q = torch.cat([q, q[:1].expand(extra, -1, -1)])
        B.coe_kv_attention(cache, len(self.new), tokens + extra, most, self.heads, self.window, self.scale, q.data_ptr(), q.stride(0), q.stride(1),
                           off.data_ptr(), total.data_ptr(), table.data_ptr(), self.max_blocks, out.data_ptr(), out.stride(0), out.stride(1),
                           logs.data_ptr() if lse else 0, work.data_ptr(), need, _stream())
        torch.cuda.synchronize()
        got = out.cpu().numpy().view(np.uint16)
        assert (got[:, -1] == poison).all() and (got[tokens:] == poison).all(), "wrote outside its rows"
        return got[:tokens, :-1], logs.cpu().numpy()[:tokens] if lse else None

    def check(self, got, logs=None, clean=None):
        bits = self.bits if clean is None else clean
        with np.errstate(invalid="ignore"):
            out, lse, size = T.attention(T.bf16_to_f64(self.q), T.bf16_to_f64(bits[0]), T.bf16_to_f64(bits[1]), self.total, self.off, self.table,
                                         self.block, self.window, self.scale)
        g = T.bf16_to_f64(got)
        # bf16 holds 8 bits: a probability is rounded to it (2^-8 of itself at most), as is the result (2^-8); the scores carry fp32 errors: at most
        # (dim + 2) 2^-24 sum|q k| * scale, under 1e-4 for these inputs' scores (sharp rows have larger ones: checked as given),
        # and so do sums over the keys.  Per element |error| <= 2^-8 |out| + (2^-8 + 1e-3) sum p |v|; over all of them the
        # roundings are independent: about 1.7e-3 of the norm, where 4e-3 is allowed.
        bound = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 1e-3) * size + 1e-30
        assert np.isfinite(g).all()
        assert (np.abs(g - out) <= bound).all(), float((np.abs(g - out) / bound).max())
        if out.size >= 4096:
            assert np.linalg.norm(g - out) <= 4e-3 * np.linalg.norm(out)
        if logs is not None:
            assert np.array_equal(np.isinf(logs), np.isinf(lse))
            ok = np.isfinite(lse)
            assert (np.abs(logs[ok] - lse[ok]) <= 2e-4 + 2e-6 * np.abs(lse[ok])).all()


SHAPES = [(12, 12, 64), (32, 8, 128), (8, 1, 64), (6, 2, 80), (24, 8, 96), (7, 7, 8), (5, 5, 40), (14, 2, 128), (16, 1, 128), (33, 1, 64), (80, 2, 128)]


@pytest.mark.parametrize("heads,kv,dim", SHAPES)
def test_attention_single_tokens(B, heads, kv, dim):
    """One new token per request, histories of every remainder of a tile and of a block."""
    lengths = [(h, 1) for h in (0, 1, 7, 8, 15, 16, 17, 30, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 300)]
    a = Attend(B, lengths, heads, kv, dim, seed=heads + dim)
    a.check(*a.run())


@pytest.mark.parametrize("block,layout", [(8, "token"), (16, "head"), (32, "pair"), (64, "inner"), (128, "token"), (1024, "head")])
def test_attention_blocks_and_layouts(B, block, layout):
    for lengths in ([(500, 1), (0, 1), (77, 1), (1024, 1)], [(300, 40), (0, 90), (129, 1), (5, 130)]):
        for heads, kv, dim in ((8, 2, 128), (6, 6, 64)):
            a = Attend(B, lengths, heads, kv, dim, block=block, layout=layout, seed=block)
            a.check(*a.run())


@pytest.mark.parametrize("lengths", [
    [(0, 1)], [(0, 2)], [(0, 31)], [(0, 33)], [(0, 64), (0, 65)], [(0, 127), (0, 128), (0, 129)], [(100, 257)], [(64, 3), (200, 5), (3, 8), (0, 9)],
    [(0, 0), (50, 1), (0, 0), (33, 40), (0, 0)],                    # requests with no new tokens between others
    [(-3, 5), (-5, 5), (-40, 60), (10, 2)],                         # rows before the first cached token see nothing
    [(0, 300), (700, 1), (700, 20), (31, 1), (1000, 64)],
])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 64), (8, 2, 128), (12, 4, 96), (5, 1, 80)])
def test_attention_chunks(B, lengths, heads, kv, dim):
    a = Attend(B, lengths, heads, kv, dim, seed=len(lengths) + dim)
    a.check(*a.run())


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 100, 129, 5000])
def test_attention_window(B, window):
    for lengths in ([(0, 1), (31, 1), (32, 1), (500, 1), (1000, 1)], [(0, 200), (300, 150), (64, 1), (1000, 30)]):
        for heads, kv, dim in ((8, 2, 128), (12, 12, 64)):
            a = Attend(B, lengths, heads, kv, dim, window=window, seed=window)
            a.check(*a.run())


def test_attention_long_histories_are_split(B):
    """Few requests with long histories beside short ones: parts of a history are joined again."""
    for lengths in ([(9000, 1)], [(5000, 1), (3, 1), (7777, 1)], [(6000, 2), (6001, 3)], [(5000, 40), (10, 1)]):
        for heads, kv, dim in ((8, 1, 128), (4, 4, 64)):
            a = Attend(B, lengths, heads, kv, dim, block=64, seed=3)
            a.check(*a.run())


def test_attention_sharp_and_flat_scores(B):
    """Scores of some hundreds (one key takes all), all equal (a plain mean), and a running maximum that rises with every key."""
    a = Attend(B, [(400, 1), (300, 70)], 4, 2, 128, seed=1, sharp=40.0, scale=0.5)
    got, logs = a.run()
    out, lse, size = T.attention(T.bf16_to_f64(a.q), T.bf16_to_f64(a.bits[0]), T.bf16_to_f64(a.bits[1]), a.total, a.off, a.table, 16, 0, a.scale)
    # sum|q k| * scale reaches 40 * 128 * 0.64 * 0.5 = 1640, so a score may be off by 130 * 2^-24 * 1640 = 0.013 at most
    g = T.bf16_to_f64(got)
    assert (np.abs(g - out) <= 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 0.026) * size + 1e-30).all()
    assert (np.abs(logs - lse) <= 0.013 + 1e-6 * np.abs(lse)).all()
    a = Attend(B, [(400, 1), (300, 70)], 4, 2, 64, seed=2, scale=0.0)
    a.check(*a.run())
    for sign in (1.0, -1.0):
        a = Attend(B, [(700, 1), (200, 80)], 4, 2, 64, seed=3)
        a.q[:] = _bf16(np.ones_like(a.q, np.float64))
        for r, t in enumerate(a.total):
            for j in range(t):
                b, row = a.at(r, j)
                a.bits[0, b, row] = _bf16(np.full((2, 64), sign * j / 64.0))
        a.check(*a.run())


@pytest.mark.parametrize("value", [0x7F80, 0xFF80, 0x7FC0, 0x7F7F, 0xFF7F])     # inf, -inf, NaN, the largest, the lowest
@pytest.mark.parametrize("window", [0, 50])
def test_attention_keeps_what_is_masked_out(B, value, window):
    """Keys and values that a row does not see leave its bits alone, whatever they hold."""
    for lengths, bad in ([[(300, 1), (40, 1), (63, 1)], []], [[(60, 150), (0, 70), (90, 1)], [(0, 130), (0, 209), (1, 33), (1, 69)]]):
        for heads, kv, dim in ((8, 2, 128), (4, 4, 64)):
            a = Attend(B, lengths, heads, kv, dim, window=window, seed=9)
            if window:
                bad = bad + [(0, 5)]
            base, base_lse = a.run()
            clean = a.bits.copy()
            for r, j in bad:
                a.bits[(slice(None),) + a.at(r, j)] = value
            a.bits[clean == 0x7FC0] = value                            # rows nobody has written
            got, lse = a.run()
            seen = np.zeros(len(got), bool)                            # rows that do see a bad token
            for r, j in bad:
                for i in range(a.new[r]):
                    pos = a.total[r] - a.new[r] + i
                    seen[a.off[r] + i] |= j <= pos and (window == 0 or j > pos - window)
            assert np.array_equal(got[~seen], base[~seen]) and np.array_equal(lse[~seen], base_lse[~seen])
            if value in (0x7F80, 0xFF80, 0x7FC0) and seen.any():
                assert not np.isfinite(T.bf16_to_f64(got[seen])).all()


def test_attention_unknown_blocks_read_as_zeros(B):
    a = Attend(B, [(200, 1), (90, 64)], 8, 2, 64, seed=4)
    a.table[0, 3], a.table[0, 5], a.table[1, 0] = -1, a.n_blocks, 2 ** 31 - 1
    a.check(*a.run())


def test_attention_length_beyond_the_table(B):
    """seq_len is limited to what the table holds."""
    a = Attend(B, [(100, 1), (63, 1)], 4, 2, 64, seed=4)              # full blocks: every row that comes into reach is written
    a.max_blocks = 7
    a.table = a.table[:, :7].copy()
    a.table[1, 4:] = a.table[0, :3]
    a.total[1] = 10 ** 6
    got, lse = a.run()
    a.total[1] = 112
    a.total[0] = 101
    a.check(got, lse)


def test_attention_fewer_new_tokens_than_announced_and_padding_rows(B):
    a = Attend(B, [(100, 3), (50, 1), (7, 0)], 8, 2, 128, seed=4)
    base = a.run()
    for most, extra in ((3, 5), (200, 0), (300, 9)):
        got, lse = a.run(max_new=most, extra=extra)
        a.check(got, lse)
    assert np.array_equal(a.run(lse=False)[0], base[0])


class Wide(Attend):
    """The same with block tables that could hold 8192 tokens a request, as a server's would."""

    def __init__(self, *args, **kwargs):
        super().__init__(*args, **kwargs)
        wide = np.random.default_rng(1).integers(-3, self.n_blocks + 3, (len(self.table), 8192 // self.block)).astype(np.int32)
        wide[:, :self.max_blocks] = self.table
        self.table, self.max_blocks = wide, wide.shape[1]


@pytest.mark.parametrize("heads,kv,dim", SHAPES)
def test_attention_single_tokens_wide_tables(B, heads, kv, dim):
    lengths = [(h, 1) for h in (0, 1, 7, 8, 15, 16, 17, 30, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 300)]
    a = Wide(B, lengths, heads, kv, dim, seed=heads + dim)
    a.check(*a.run())
    a = Wide(B, [(0, 0), (50, 1), (0, 0), (33, 1), (-3, 2), (0, 0), (-1, 1)], heads, kv, dim, block=64, layout="pair", seed=dim)
    a.check(*a.run())


def test_attention_wide_tables_masks_and_counts(B):
    """Windows, values that are no numbers behind the mask, blocks outside the cache, and 700 requests, with stretches that cross requests."""
    rng = np.random.default_rng(12)
    a = Wide(B, [(int(h), int(rng.random() < 0.9)) for h in rng.integers(0, 60, 700)], 4, 2, 64, seed=1)
    a.check(*a.run())
    for window in (1, 31, 33, 100, 2 ** 31 - 1):
        a = Wide(B, [(0, 1), (31, 2), (32, 1), (500, 3), (1000, 1), (-3, 5)], 8, 2, 128, window=window, seed=window & 0xFFFF)
        a.check(*a.run())
    for value in (0x7F80, 0xFF80, 0x7FC0, 0x7F7F, 0xFF7F):
        a = Wide(B, [(300, 4), (40, 1), (63, 8)], 8, 2, 128, seed=9)
        base, base_lse = a.run()
        clean = a.bits.copy()
        a.bits[(slice(None),) + a.at(0, 302)] = value                 # seen by the last two of the first request's rows
        a.bits[clean == 0x7FC0] = value
        got, lse = a.run()
        seen = np.arange(len(got)) // 2 == 1
        assert np.array_equal(got[~seen], base[~seen]) and np.array_equal(lse[~seen], base_lse[~seen])
    a = Wide(B, [(200, 1), (90, 5)], 8, 2, 64, seed=4)
    a.table[0, 3], a.table[0, 5], a.table[1, 0] = -1, a.n_blocks, 2 ** 31 - 1
    a.check(*a.run())


def test_attention_short_tables_many_histories(B):
    """More histories than compute units, each of them short: a workgroup of its own for each."""
    rng = np.random.default_rng(5)
    for heads, kv, dim, window in ((8, 8, 64, 0), (16, 4, 128, 0), (16, 4, 128, 40), (12, 4, 24, 0)):
        a = Attend(B, [(int(h), int(m)) for h, m in zip(rng.integers(0, 200, 90), rng.integers(0, 4, 90))], heads, kv, dim, window=window, seed=kv)
        a.check(*a.run())


def test_attention_of_many_requests(B):
    """More requests than a workgroup has threads, single tokens only and in a mixed step; most histories are short."""
    rng = np.random.default_rng(12)
    ones = [(int(h), int(rng.random() < 0.9)) for h in rng.integers(0, 60, 700)]
    a = Attend(B, ones, 4, 2, 64, seed=1)
    a.check(*a.run())
    mixed = [(int(h), int(m)) for h, m in zip(rng.integers(0, 40, 1500), rng.integers(0, 4, 1500))]
    mixed[3], mixed[1400] = (200, 70), (0, 129)
    a = Attend(B, mixed, 4, 2, 64, seed=2)
    a.check(*a.run())


@pytest.mark.parametrize("dim", [16, 24, 32, 56, 72, 112, 120])
def test_attention_head_widths(B, dim):
    for lengths in ([(100, 1), (0, 1), (37, 2)], [(60, 100), (33, 1)]):
        a = Attend(B, lengths, 6, 2, dim, seed=dim)
        a.check(*a.run())


def test_attention_largest_window(B):
    """A window beyond every history is none, also for rows that stand before the first cached token."""
    for lengths in ([(-3, 5), (40, 1), (-1, 2)], [(-3, 70), (50, 90), (-40, 60)]):
        base = Attend(B, lengths, 8, 2, 64, seed=1).run()
        for window in (2 ** 31 - 1, 2 ** 31 - 40, 10 ** 6):
            got = Attend(B, lengths, 8, 2, 64, seed=1, window=window).run()
            assert np.array_equal(got[0], base[0]) and np.array_equal(got[1], base[1])


def test_attention_window_past_freed_blocks(B):
    """Blocks that lie wholly before every row's window may be given back: their table entries are not followed."""
    for lengths in ([(500, 1), (300, 2)], [(500, 70), (300, 1)]):
        a = Attend(B, lengths, 8, 2, 64, window=100, seed=3)
        base = a.run()
        for r, (have, _) in enumerate(lengths):
            a.table[r, :(have - 100) // 16] = -1
        got = a.run()
        assert np.array_equal(got[0], base[0]) and np.array_equal(got[1], base[1])


def test_attention_offsets_that_are_no_offsets(B):
    """Row ranges that run backwards or past the tokens take what lies inside; no other row is written, and sound requests are served."""
    for new in (1, 40):
        a = Attend(B, [(60, new), (40, new), (80, new)], 4, 2, 64, seed=4)
        base = a.run()[0]
        import torch
        k, v, cache = _make_cache(B, a.bits, "token")
        q, out = _dev(a.q), _dev(np.full(a.q.shape, 0xFFC0, np.uint16))
        need = B.coe_kv_attention_workspace(3, 3 * new, new, 4, 2, 64)
        work = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        off, total, table = _dev(np.array([0, new, new, 10 ** 9], np.int32)), _dev(a.total), _dev(a.table)
        B.coe_kv_attention(cache, 3, 3 * new, new, 4, 0, a.scale, q.data_ptr(), q.stride(0), q.stride(1), off.data_ptr(), total.data_ptr(), table.data_ptr(),
                           a.max_blocks, out.data_ptr(), out.stride(0), out.stride(1), 0, work.data_ptr(), need, _stream())
        got = out.cpu().numpy().view(np.uint16)
        assert np.array_equal(got[:new], base[:new]) and (got[2 * new:] == 0xFFC0).all()     # the third has more rows than were announced
        off = _dev(np.array([0, new, -7, -9], np.int32))
        out.copy_(_dev(np.full(a.q.shape, 0xFFC0, np.uint16)))
        B.coe_kv_attention(cache, 3, 3 * new, new, 4, 0, a.scale, q.data_ptr(), q.stride(0), q.stride(1), off.data_ptr(), total.data_ptr(), table.data_ptr(),
                           a.max_blocks, out.data_ptr(), out.stride(0), out.stride(1), 0, work.data_ptr(), need, _stream())
        got = out.cpu().numpy().view(np.uint16)
        assert np.array_equal(got[:new], base[:new]) and (got[new:] == 0xFFC0).all()


def test_attention_cache_beyond_4_gib(B):
    """Blocks whose bytes begin past 2^32: the same bits as in a small cache."""
    import torch
    a = Attend(B, [(500, 1), (130, 1), (200, 60)], 8, 2, 128, block=64, seed=5)
    base, base_lse = a.run()
    # the same blocks, 2^20 * 300 elements (600 MiB) apart: the last one begins beyond 2^32 bytes and 2^32 elements
    apart = (1 << 20) * 300
    row = 64 * 2 * 128
    assert a.n_blocks * apart > 2 ** 32
    room = torch.empty(2 * (a.n_blocks - 1) * apart + 4 * row, dtype=torch.int16, device="cuda")
    k = room[:].as_strided((a.n_blocks, row), (apart, 1), 0)
    v = room[:].as_strided((a.n_blocks, row), (apart, 1), (a.n_blocks - 1) * apart + row)
    k.copy_(_dev(a.bits[0].reshape(a.n_blocks, row)))
    v.copy_(_dev(a.bits[1].reshape(a.n_blocks, row)))
    cache = B.coe_kv_cache(B.COE_DT_BF16, a.n_blocks, 64, 2, 128, k.data_ptr(), v.data_ptr(), apart, 256, 128)
    tokens = int(a.off[-1])
    q, out, lse = _dev(a.q), _dev(np.zeros_like(a.q)), torch.zeros(tokens, 8, device="cuda")
    need = B.coe_kv_attention_workspace(3, tokens, 60, 8, 2, 128)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    off, total, table = _dev(a.off), _dev(a.total), _dev(a.table)
    B.coe_kv_attention(cache, 3, tokens, 60, 8, 0, a.scale, q.data_ptr(), q.stride(0), q.stride(1), off.data_ptr(), total.data_ptr(), table.data_ptr(),
                       a.max_blocks, out.data_ptr(), out.stride(0), out.stride(1), lse.data_ptr(), work.data_ptr(), need, _stream())
    assert np.array_equal(out.cpu().numpy().view(np.uint16), base) and np.array_equal(lse.cpu().numpy(), base_lse)
    # and an append there
    slot = _dev(np.array([(a.n_blocks - 1) * 64 + 63], np.int32))
    new = _dev(np.full((1, 2, 128), 0x4040, np.uint16))
    B.coe_kv_append(cache, 1, new.data_ptr(), 256, 128, new.data_ptr(), 256, 128, slot.data_ptr(), _stream())
    assert (k[-1, -256:] == 0x4040).all() and (v[-1, -256:] == 0x4040).all()


def test_attention_repeats_its_bits(B):
    a = Attend(B, [(3000, 1), (100, 1), (900, 90), (0, 300)], 8, 2, 128, seed=6)
    base = a.run()
    for _ in range(3):
        got = a.run()
        assert np.array_equal(got[0], base[0]) and np.array_equal(got[1], base[1])


# ---- sampling ---------------------------------------------------------------------------------------------------
def _sample_gpu(B, x, temperature=None, top_k=None, top_p=None, min_p=None, noise=None, pad=3, logprob=True):
    """x float32 or uint16 (bf16 bits) [rows][vocab]; garbage between the rows."""
    import torch
    rows, vocab = x.shape
    wide = np.full((rows, vocab + pad), 0x7F80 if x.dtype == np.uint16 else np.inf, x.dtype)
    wide[:, :vocab] = x
    d = _dev(wide)
    nz = None
    if noise is not None:
        nz = np.zeros((rows, vocab + 1), np.float32)
        nz[:, :vocab] = noise
        nz = _dev(nz)
    args = [None if a is None else _dev(np.broadcast_to(np.asarray(a, t), (rows,)).copy()) for a, t in
            ((temperature, np.float32), (top_k, np.int32), (top_p, np.float32), (min_p, np.float32))]
    token = torch.full((rows,), -99, dtype=torch.int32, device="cuda")
    lp = torch.full((rows,), 7.0, device="cuda")
    need = B.coe_sample_workspace(rows, vocab)
    work = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    B.coe_sample_tokens(rows, vocab, B.COE_DT_BF16 if x.dtype == np.uint16 else B.COE_DT_F32, d.data_ptr(), vocab + pad,
                        *(0 if a is None else a.data_ptr() for a in args), 0 if nz is None else nz.data_ptr(), vocab + 1, token.data_ptr(),
                        lp.data_ptr() if logprob else 0, work.data_ptr(), need, _stream())
    return token.cpu().numpy(), lp.cpu().numpy()


def _at(a, r, off):
    return off if a is None else float(np.broadcast_to(np.asarray(a), (r + 1,) if np.ndim(a) == 0 else np.shape(a))[r])


def _check_sample(B, x, temperature=None, top_k=None, top_p=None, min_p=None, noise=None):
    token, lp = _sample_gpu(B, x, temperature, top_k, top_p, min_p, noise)
    x64 = T.bf16_to_f64(x) if x.dtype == np.uint16 else x.astype(np.float64)
    f = lambda a: None if a is None else np.asarray(a, np.float32).astype(np.float64)
    temperature, top_p, min_p = f(temperature), f(top_p), f(min_p)
    for r in range(len(x)):
        # scores: (x - max) / T and ln E in fp32, at most 2^-22 of values up to 100: 5e-5 together; masses: sums of up to 10^5 fp32
        # terms by 1024 lanes, 1e-5 of them at most
        near, ln = T.sample(x64[r], _at(temperature, r, 1.0), int(_at(top_k, r, 0)), _at(top_p, r, 1.0), _at(min_p, r, 0.0),
                            None if noise is None else noise[r], slack=1e-4)
        assert int(token[r]) in near, (r, int(token[r]), near)
        if ln is None:
            assert lp[r] == -np.inf
        else:
            assert abs(lp[r] - ln[token[r]]) <= 1e-5 * (1 + abs(ln[token[r]])), r
    return token


def _noise(rng, shape):
    return rng.standard_exponential(shape).astype(np.float32)


@pytest.mark.parametrize("vocab", [1, 2, 63, 64, 65, 1000, 1023, 1024, 1025, 4097, 32003, 50001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sample_sizes(B, vocab, dtype):
    """Every filter and several at once, at vocabularies around the workgroup's stride."""
    rng = np.random.default_rng(vocab)
    settings = [(0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (0.7, 1, 1.0, 0.0), (1.3, 5, 1.0, 0.0), (1.0, 40, 0.9, 0.0), (1.0, vocab - 1, 0.95, 0.0),
                (1.0, vocab, 0.5, 0.0), (1.0, vocab + 7, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (2.0, 0, 0.3, 0.0), (1.0, 0, 1e-6, 0.0), (1.0, 0, 0.0, 0.0),
                (1.0, 0, 1.0, 0.05), (1.0, 0, 1.0, 1.0), (1.0, 50, 0.99, 0.1), (0.05, 700, 0.999, 0.0), (1.0, 1000, 0.8, 0.001), (1.0, -3, 1.5, -1.0)]
    rows = len(settings)
    x = (3 * rng.standard_normal((rows, vocab))).astype(np.float32)
    if dtype == "bf16":
        x = _bf16(x)
    t, k, p, m = (np.array(c) for c in zip(*settings))
    _check_sample(B, x, t, k, p, m, _noise(rng, (rows, vocab)))


@pytest.mark.parametrize("case", ["equal", "two values", "ascending", "descending", "steps", "one large", "lowest", "far below", "zeros"])
@pytest.mark.parametrize("vocab", [70, 3000, 20001])
def test_sample_ties_and_masks(B, case, vocab):
    """Ties go by index, also across the cut of a filter; masks of -inf, of the type's lowest value, and far-off values."""
    rng = np.random.default_rng(vocab)
    one = {"equal": np.full(vocab, 2.5), "two values": rng.integers(0, 2, vocab) * 1.0, "ascending": np.arange(vocab) * 0.01,
           "descending": -np.arange(vocab) * 0.01, "steps": np.floor(rng.standard_normal(vocab) * 4), "one large": np.where(np.arange(vocab) == 11, 50.0, 0.0),
           "lowest": np.where(rng.random(vocab) < 0.9, -3.4028235e38, rng.standard_normal(vocab)),
           "far below": np.where(rng.random(vocab) < 0.99, -1e30, rng.standard_normal(vocab)),
           "zeros": np.where(rng.random(vocab) < 0.5, 0.0, -0.0)}[case].astype(np.float32)
    settings = [(0.0, 0, 1.0, 0.0), (1.0, 0, 1.0, 0.0), (1.0, 3, 1.0, 0.0), (1.0, 33, 0.7, 0.0), (1.0, 0, 0.5, 0.0), (0.3, 0, 0.9, 0.2), (1.0, vocab - 2, 0.99, 0.0),
                (1.0, 2000, 1.0, 0.0)]
    x = np.repeat(one[None], len(settings), 0)
    masked = x.copy()
    masked[:, rng.random(vocab) < 0.6] = -np.inf
    masked[:, 7] = 1.0
    t, k, p, m = (np.array(c) for c in zip(*settings))
    for v in (x, masked, _bf16(x), _bf16(masked)):
        _check_sample(B, v, t, k, p, m, _noise(rng, x.shape))


def test_sample_exact_cuts(B):
    """Weights and masses that fp32 holds exactly: the cut falls where the definition says, not one further."""
    vocab = 64
    x = np.full((vocab, vocab), -np.inf, np.float32)
    x[:, ::8] = 0.0                                   # eight equal tokens at 0, 8, ..., 56
    noise = np.full((vocab, vocab), 1.0, np.float32)
    for r in range(vocab):
        noise[r, 8 * (r % 8)] = 1e-6                  # token r % 8 of them wins if it is kept, else the first
    for p, kept in ((0.5, 4), (0.51, 5), (0.125, 1), (0.126, 2), (0.875, 7), (0.99, 8)):
        token, _ = _sample_gpu(B, x, 1.0, None, p, None, noise)
        assert [int(v) for v in token] == [8 * (r % 8) if r % 8 < kept else 0 for r in range(vocab)], p
    for k in range(1, 9):
        token, _ = _sample_gpu(B, x, 1.0, k, None, None, noise)
        assert [int(v) for v in token] == [8 * (r % 8) if r % 8 < k else 0 for r in range(vocab)], k
    for k, p, kept in ((4, 0.5, 2), (4, 0.51, 3), (6, 0.5, 3), (2, 0.4, 1)):        # the nucleus of what top_k left
        token, _ = _sample_gpu(B, x, 1.0, k, p, None, noise)
        assert [int(v) for v in token] == [8 * (r % 8) if r % 8 < kept else 0 for r in range(vocab)], (k, p)
    x[:, 8] = 0.75                                    # orders that differ in the last bits only
    x[:, 16] = np.nextafter(np.float32(0.75), np.float32(1))
    token, _ = _sample_gpu(B, x, 1.0, 1, None, None, noise)
    assert (token == 16).all()
    tiny = np.zeros((1, 3000), np.float32)
    tiny[0, 0], tiny[0, 100], tiny[0, 200] = 10.0, 1e-9, 2e-9
    n = np.full((1, 3000), 1.0, np.float32)
    n[0, 100], n[0, 200] = 1e-12, 1e-10
    assert _sample_gpu(B, tiny, 1.0, 2, None, None, n)[0][0] == 200 and _sample_gpu(B, tiny, 1.0, 3, None, None, n)[0][0] == 100


@pytest.mark.parametrize("vocab", [5, 300, 5000])
@pytest.mark.parametrize("level", [-3000.0, -200.0, 0.0, 200.0, 3000.0])
def test_sample_far_from_zero(B, vocab, level):
    """Logits that all lie far on one side of 0: threads, wavefronts and masked stretches without a token do not set what weights are
    relative to."""
    rng = np.random.default_rng(vocab)
    x = (level + np.round(64 * rng.standard_normal((6, vocab))) / 16).astype(np.float32)      # exact in fp32
    x[1, vocab // 2:] = -np.inf
    x[2, :vocab // 2] = -np.inf
    for t, k, p in ((1.0, 0, 1.0), (0.5, 0, 0.8), (1.0, 20, 0.9), (3.0, 0, 0.5)):
        _check_sample(B, x, t, k, p, 0.0, _noise(rng, x.shape))


@pytest.mark.parametrize("rows,vocab,dtype", [(300, 17003, "f32"), (300, 17003, "bf16"), (200, 20011, "bf16"), (3, 140001, "f32"), (3, 140001, "bf16"), (60, 70007, "bf16")])
def test_sample_rows_by_number(B, rows, vocab, dtype):
    """One row's tokens do not depend on how many others there are: every filter in turn, checked on some of the rows."""
    rng = np.random.default_rng(rows)
    settings = [(1.0, 0, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (1.0, 0, 0.4, 0.0), (1.0, 60, 0.95, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 900, 1.0, 0.001), (1.0, 5000, 0.9, 0.0),
                (1.5, 0, 0.7, 0.01), (1.0, 0, 0.01, 0.0)]
    x = (3 * rng.standard_normal((rows, vocab), dtype=np.float32)).astype(np.float32)
    x[0, rng.random(vocab) < 0.99] = -np.inf
    if dtype == "bf16":
        x = _bf16(x)
    t, k, p, m = (np.array([c[r % len(settings)] for r in range(rows)]) for c in zip(*settings))
    noise = rng.standard_exponential((rows, vocab), dtype=np.float32)
    some = sorted({0, 1, 2, rows - 1} | set(rng.integers(0, rows, 12).tolist()))
    token, lp = _sample_gpu(B, x, t, k, p, m, noise)
    wide = x if dtype == "f32" else None
    for r in some:
        x64 = (T.bf16_to_f64(x[r]) if wide is None else x[r].astype(np.float64))
        near, ln = T.sample(x64, float(np.float32(t[r])), int(k[r]), float(np.float32(p[r])), float(np.float32(m[r])), noise[r], slack=1e-4)
        assert int(token[r]) in near, (r, int(token[r]), near)
        assert abs(lp[r] - ln[token[r]]) <= 1e-5 * (1 + abs(ln[token[r]])), r


@pytest.mark.parametrize("vocab", [66000])
def test_sample_hidden_winners(B, vocab):
    """The best of the race fall to the nucleus one after the other, and the token that is drawn shares a thread's stretch with them."""
    rng = np.random.default_rng(8)
    rows = 24
    x = np.full((rows, vocab), -4.0, np.float32) + rng.random((rows, vocab), dtype=np.float32)
    noise = np.full((rows, vocab), 1.0, np.float32) + rng.random((rows, vocab), dtype=np.float32)
    for r in range(rows):
        at = rng.integers(0, vocab - 40)
        x[r, at:at + 3] = 9.0, 8.9, 8.8               # the nucleus
        x[r, rng.integers(0, vocab)] += 0.5
        noise[r, at], noise[r, at + 1], noise[r, at + 2] = 3.0, 2.0, 1.5
        for j in range(1, 1 + r % 7):                 # numbers so small that they win, of tokens that are not kept, next to it and far off
            noise[r, (at + 3 + j) if j % 2 else rng.integers(0, vocab)] = 1e-12 * j
    for p in (0.3, 0.6, 0.9):
        _check_sample(B, x, 1.0, 0, p, 0.0, noise)
        _check_sample(B, x[:, :9000], 1.0, 0, p, 0.0, noise[:, :9000])


def test_sample_values_that_are_no_numbers(B):
    rng = np.random.default_rng(3)
    vocab = 2500
    x = rng.standard_normal((12, vocab)).astype(np.float32)
    x[0] = -np.inf                                    # nothing to draw
    x[1] = np.nan
    x[2, :] = -np.inf
    x[2, 1777] = -5.0                                 # a single token
    x[3, rng.random(vocab) < 0.5] = np.nan
    x[4, [100, 7, 2000]] = np.inf                     # shares everything among three
    x[5, 3] = np.inf
    x[6] = 3.4028235e38
    x[7, 5] = 3.4028235e38
    noise = _noise(rng, x.shape)
    noise[8] = np.nan                                 # no usable number: the first token
    noise[9] = -1.0
    noise[10] = np.inf
    noise[11, [40, 50]] = 0.0                         # certain winners, the lower index of the two
    for t, k, p, m in ((1.0, 0, 1.0, 0.0), (0.7, 10, 1.0, 0.0), (1.0, 0, 0.8, 0.0), (1.0, 600, 0.9, 0.01), (0.0, 0, 1.0, 0.0), (np.nan, 0, 1.0, 0.0)):
        token = _check_sample(B, x, t, k, p, m, noise)
        assert token[0] == -1 and token[1] == -1 and token[2] == 1777
        if t == 1.0 and k == 0 and p == 1.0:
            assert token[11] == 40 and token[8] == np.argmax(x[8])
    _check_sample(B, x, np.inf, 0, 1.0, 0.0, noise)
    _check_sample(B, x, 0.0, None, None, None, None)  # greedy needs no numbers
    token, _ = _sample_gpu(B, x, None, None, None, None, noise, logprob=False)
    assert token[2] == 1777


def test_sample_many_rows_have_their_probabilities(B):
    """20,000 draws from one row: counts within five standard deviations of the renormalised probabilities."""
    rng = np.random.default_rng(11)
    rows, vocab = 20000, 300
    one = (2 * rng.standard_normal(vocab)).astype(np.float32)
    x = np.repeat(one[None], rows, 0)
    token, _ = _sample_gpu(B, x, 0.9, 50, 0.9, 0.01, _noise(rng, x.shape))
    z = one.astype(np.float64) / np.float64(np.float32(0.9))
    w = np.exp(z - z.max())
    order = np.argsort(-one, kind="stable")[:50]
    before = np.cumsum(w[order]) - w[order]
    order = order[(before < 0.9 * w[order].sum()) & (w[order] >= 0.01)]
    p = w[order] / w[order].sum()
    count = np.bincount(token, minlength=vocab)
    assert count.sum() == count[order].sum() == rows
    assert (np.abs(count[order] - rows * p) <= 5 * np.sqrt(rows * p * (1 - p)) + 1).all()


# ---- streams and graphs ------------------------------------------------------------------------------------------
def test_a_step_on_another_stream_and_in_a_graph(B):
    """Plan, append, attention and sampling of a step on a stream of their own, then captured: every replay equals the eager run."""
    import torch
    rng = np.random.default_rng(2)
    n, block, n_blocks, max_blocks, cap, heads, kv, dim, vocab = 9, 16, 300, 40, 64, 8, 2, 64, 3000
    have = rng.integers(0, 500, n).astype(np.int32)
    add = np.array([1, 1, 5, 1, 0, -1, 20, 1, 3], np.int32)
    table, ring, state = _pool(rng, have, block, n_blocks, max_blocks)
    d = {k: _dev(np.asarray(v, np.int32)) for k, v in dict(have=have, add=add, ring=ring, state=state, table=table).items()}
    i32 = dict(dtype=torch.int32, device="cuda")
    o = dict(seq_len=torch.zeros(n, **i32), q_off=torch.zeros(n + 1, **i32), slot=torch.zeros(cap, **i32), position=torch.zeros(cap, **i32),
             next=torch.zeros(4, **i32), token=torch.zeros(n, **i32))
    k, v, cache = _make_cache(B, _bf16(rng.standard_normal((2, n_blocks, block, kv, dim))), "token")
    qkv = _dev(_bf16(rng.standard_normal((cap, heads + 2 * kv, dim))))
    out, lse = torch.zeros(cap, heads, dim, dtype=torch.int16, device="cuda"), torch.zeros(cap, heads, device="cuda")
    logits, noise = torch.randn(n, vocab, device="cuda"), torch.empty(n, vocab, device="cuda").exponential_()
    w1, w2 = B.coe_kv_attention_workspace(n, cap, 20, heads, kv, dim), B.coe_sample_workspace(n, vocab)
    work, work2 = torch.empty(max(w1, 16), dtype=torch.uint8, device="cuda"), torch.empty(max(w2, 16), dtype=torch.uint8, device="cuda")
    top_k = torch.full((n,), 30, **i32)
    p = lambda t: t.data_ptr()

    def step(stream):
        B.coe_kv_plan(n, block, n_blocks, max_blocks, cap, p(d["have"]), p(d["add"]), p(d["ring"]), p(d["state"]), p(d["table"]), p(o["seq_len"]), p(o["q_off"]),
                      p(o["slot"]), p(o["position"]), p(o["next"]), stream)
        row = (heads + 2 * kv) * dim
        B.coe_kv_append(cache, cap, p(qkv) + 2 * heads * dim, row, dim, p(qkv) + 2 * (heads + kv) * dim, row, dim, p(o["slot"]), stream)
        B.coe_kv_attention(cache, n, cap, 20, heads, 0, 0.125, p(qkv), row, dim, p(o["q_off"]), p(o["seq_len"]), p(d["table"]), max_blocks, p(out), heads * dim, dim,
                           p(lse), p(work), w1, stream)
        B.coe_sample_tokens(n, vocab, B.COE_DT_F32, p(logits), vocab, 0, p(top_k), 0, 0, p(noise), vocab, p(o["token"]), 0, p(work2), w2, stream)

    outputs = [out, lse, k, v, d["table"], d["ring"], *o.values()]
    torch.cuda.synchronize()
    step(_stream())
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]
    for t in (out, lse, *o.values()):
        t.zero_()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outputs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(torch.cuda.current_stream().cuda_stream)
    for i in range(4):
        for t in (out, lse, *o.values()):
            t.fill_(i)
        work.fill_(i)
        graph.replay()
        torch.cuda.synchronize()
        used = int(o["q_off"][-1])               # rows of no request are not written
        for a, b in zip(outputs, want):
            if a is out or a is lse:
                a, b = a[:used], b[:used]
            assert torch.equal(a, b)


# ---- the example that serves them together ------------------------------------------------------------------------
def _dense_logits(e, expert, ids):
    """The expert's logits at every place of ids: whole rows of scores, fp32 on the CPU, nothing cached."""
    import torch
    f = lambda w: w[expert].float().cpu()
    norm = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)
    n = len(ids)
    x = f(e.embedding)[ids] + f(e.position)[:n]
    mask = torch.full((n, n), -np.inf).triu(1)
    for layer in range(e.layers):
        q, k, v = (norm(x) @ f(e.qkv[layer])).view(n, -1, e.head_dim).split([e.heads, e.kv_heads, e.kv_heads], 1)
        k, v = (a.repeat_interleave(e.heads // e.kv_heads, 1) for a in (k, v))
        s = torch.einsum("qhd,khd->hqk", q, k) * e.head_dim ** -0.5 + mask
        x = x + torch.einsum("hqk,khd->qhd", s.softmax(-1), v).reshape(n, -1) @ f(e.o[layer])
        x = x + torch.nn.functional.gelu(norm(x) @ f(e.up[layer])) @ f(e.down[layer])
    return norm(x) @ f(e.head)


def test_example_generates_what_the_dense_model_says(B):
    """Greedy tokens and log-probabilities of several experts in shared steps, prompts cut into chunks and a cache so small that
    requests wait for blocks, against whole forwards without a cache."""
    import importlib.util
    import pathlib
    spec = importlib.util.spec_from_file_location("generate", pathlib.Path(__file__).parent.parent / "examples" / "generate.py")
    generate = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(generate)
    experts = generate.Experts(3, max_len=200)
    rng = np.random.default_rng(0)
    prompts = [rng.integers(0, experts.vocab, m).tolist() for m in (1, 130, 17, 64, 3, 90, 33)]
    route = [2, 0, 1, 0, 2, 0, 2]
    server = generate.Server(experts, n_blocks=24, block_size=16, token_cap=96)
    tokens, logprobs, steps = server.generate(prompts, route, 6)
    assert steps > 10
    # a bf16 rounding is at most 2^-9 of a value; some ten of them on the way through each of two layers add up to 2^-9 sqrt(20) = 0.9 % of
    # the state, the logits are of deviation 1 (weights: variance 1 / fan-in): 0.01 each, and 0.06 is six deviations
    for prompt, e, drawn, lp in zip(prompts, route, tokens, logprobs):
        assert len(drawn) == 6
        logits = _dense_logits(experts, e, prompt + drawn)[len(prompt) - 1:-1]
        for row, token, value in zip(logits, drawn, lp):
            assert row[token] >= row.max() - 0.12
            assert abs(float(row.log_softmax(-1)[token]) - value) <= 0.12
    # the same with room for everything at once draws the same way at any temperature
    wide = generate.Server(experts, n_blocks=200, block_size=8, token_cap=512)
    again = wide.generate(prompts, route, 6, temperature=0.9, top_p=0.8, seed=3)
    assert wide.generate(prompts, route, 6, temperature=0.9, top_p=0.8, seed=3) == again and all(np.isfinite(v).all() for v in again[1])


@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 64), (8, 2, 128), (12, 4, 96), (16, 1, 80), (7, 1, 8)])
@pytest.mark.parametrize("wide", [False, True])
def test_attention_chunks_by_table_width(B, heads, kv, dim, wide):
    """Chunks of every length around 32 query rows, with histories, windows and empty requests, where tables are narrow (a workgroup
    for 32 rows) and wide."""
    kind = Wide if wide else Attend
    for lengths, window in (([(0, 9), (5, 33), (0, 0), (100, 20), (-4, 11), (31, 1)], 0), ([(0, 40), (64, 17), (90, 50)], 21), ([(200, 64)], 0), ([(0, 65), (0, 1)], 32)):
        a = kind(B, lengths, heads, kv, dim, window=window, seed=dim)
        a.check(*a.run())


def test_attention_chunks_of_narrow_tables_mask(B):
    """Values behind the mask do not reach a row, row by row, in chunks that narrow tables serve."""
    for value in (0x7F80, 0x7FC0, 0x7F7F, 0xFF7F):
        a = Attend(B, [(10, 70), (40, 3)], 8, 2, 64, seed=9)
        base, base_lse = a.run()
        clean = a.bits.copy()
        a.bits[(slice(None),) + a.at(0, 50)] = value                  # seen by the last thirty of the first request's rows
        a.bits[clean == 0x7FC0] = value
        got, lse = a.run()
        seen = np.arange(len(got)) - 40
        seen = (seen >= 0) & (seen < 30)
        assert np.array_equal(got[~seen], base[~seen]) and np.array_equal(lse[~seen], base_lse[~seen])
        assert len(got) == 73


CHUNKS = [
    [(0, 33)], [(0, 64), (0, 65)], [(0, 127), (0, 128), (0, 129)], [(100, 257)], [(64, 3), (200, 35), (3, 8), (0, 9)],
    [(0, 0), (50, 1), (0, 0), (33, 40), (0, 0)], [(-3, 5), (-5, 5), (-40, 60), (10, 2)], [(0, 300), (700, 1), (700, 20), (31, 1), (1000, 64)],
]


@pytest.mark.parametrize("lengths", CHUNKS)
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 64), (8, 2, 128), (12, 4, 96), (5, 1, 80), (2, 2, 8)])
def test_attention_chunks_wide_tables(B, lengths, heads, kv, dim):
    a = Wide(B, lengths, heads, kv, dim, seed=len(lengths) + dim)
    a.check(*a.run())


@pytest.mark.parametrize("block,layout", [(8, "token"), (16, "head"), (32, "pair"), (64, "inner"), (128, "token"), (1024, "head")])
def test_attention_chunks_wide_tables_blocks_and_windows(B, block, layout):
    for window in (0, 1, 31, 33, 64, 129):
        for heads, kv, dim in ((8, 2, 128), (6, 6, 64)):
            a = Wide(B, [(300, 40), (0, 90), (129, 1), (5, 130)], heads, kv, dim, block=block, layout=layout, window=window, seed=block)
            a.check(*a.run())


@pytest.mark.parametrize("value", [0x7F80, 0xFF80, 0x7FC0, 0x7F7F, 0xFF7F])
@pytest.mark.parametrize("window", [0, 50])
def test_attention_chunks_wide_tables_keep_what_is_masked_out(B, value, window):
    for heads, kv, dim in ((8, 2, 128), (4, 4, 64), (6, 2, 96)):
        a = Wide(B, [(60, 150), (0, 70), (90, 1)], heads, kv, dim, window=window, seed=9)
        base, base_lse = a.run()
        clean = a.bits.copy()
        bad = [(0, 130), (0, 209), (1, 33), (1, 69)] + [(0, 5)] * (window > 0)
        for r, j in bad:
            a.bits[(slice(None),) + a.at(r, j)] = value
        a.bits[clean == 0x7FC0] = value
        got, lse = a.run()
        seen = np.zeros(len(got), bool)
        for r, j in bad:
            for i in range(a.new[r]):
                pos = a.total[r] - a.new[r] + i
                seen[a.off[r] + i] |= j <= pos and (window == 0 or j > pos - window)
        assert np.array_equal(got[~seen], base[~seen]) and np.array_equal(lse[~seen], base_lse[~seen])


def test_attention_chunks_wide_tables_odd_inputs(B):
    """Unknown blocks, flat, negative and steep scales, a reference that has to move often, and bits that repeat."""
    a = Wide(B, [(200, 40), (90, 64)], 8, 2, 64, seed=4)
    a.table[0, 3], a.table[0, 5], a.table[1, 0] = -1, a.n_blocks, 2 ** 31 - 1
    a.check(*a.run())
    for scale in (0.0, -0.1, 1e-30):
        a = Wide(B, [(300, 70), (40, 1)], 4, 2, 64, seed=2, scale=scale)
        a.check(*a.run())
    for sign in (1.0, -1.0):                          # scores that rise (fall) by 2 with every key, from -500 on
        a = Wide(B, [(700, 40), (200, 80)], 4, 2, 64, seed=3)
        a.q[:] = _bf16(np.ones_like(a.q, np.float64))
        for r, t in enumerate(a.total):
            for j in range(t):
                a.bits[0][a.at(r, j)] = _bf16(np.full((2, 64), sign * (j - 250) / 4.0))
        got, logs = a.run()
        out, lse, size = T.attention(T.bf16_to_f64(a.q), T.bf16_to_f64(a.bits[0]), T.bf16_to_f64(a.bits[1]), a.total, a.off, a.table, 16, 0, a.scale)
        # keys beyond 64 are rounded alike on both sides; scores are sums of 64 equal numbers, exact but for the scale's rounding and the product's,
        # 2^-23 of at most 1500 together: 2e-4, on a probability twice that
        assert (np.abs(T.bf16_to_f64(got) - out) <= 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2e-3) * size + 1e-30).all()
        assert (np.abs(logs - lse) <= 1e-3 + 1e-6 * np.abs(lse)).all()
    a = Wide(B, [(3000, 1), (100, 1), (900, 90), (0, 300)], 8, 2, 128, seed=6)
    base = a.run()
    for _ in range(3):
        got = a.run()
        assert np.array_equal(got[0], base[0]) and np.array_equal(got[1], base[1])


# ---- scores that are no numbers -----------------------------------------------------------------------------------
# lengths that each kernel serves: (kind of tables, requests, the tokens of request 0 whose keys become NaN)
NAN_PATHS = {
    "narrow tables, single tokens": (Attend, [(100, 1), (40, 1), (0, 1)], range(32, 64)),
    "narrow tables, chunks": (Attend, [(100, 20), (10, 30)], range(32, 64)),
    "wide tables, single tokens": (Wide, [(100, 1), (40, 1), (0, 1)], range(32, 64)),
    "stretches that are joined": (Attend, [(9000, 1), (40, 1), (0, 2)], range(256, 384)),
    "units": (Wide, [(100, 60), (0, 90), (3, 1)], range(64, 128)),
    "units that are cut": (Wide, [(5000, 40), (0, 33), (7, 1)], range(512, 1024)),
}


@pytest.mark.parametrize("path", NAN_PATHS)
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 64), (4, 4, 80)])
def test_attention_scores_that_are_no_numbers(B, path, heads, kv, dim):
    """A NaN score makes its row NaN, output and logarithm, whichever wavefront, part or unit meets it; no other row's bits change."""
    kind, lengths, keys = NAN_PATHS[path]
    a = kind(B, lengths, heads, kv, dim, seed=dim)
    base, base_lse = a.run()
    q, bits = a.q.copy(), a.bits.copy()

    def expect(bad):                                  # [token][head]
        got, lse = a.run()
        numbers = int(np.count_nonzero(~np.isnan(T.bf16_to_f64(got[bad])))), int(np.count_nonzero(~np.isnan(lse[bad])))
        changed = int(np.count_nonzero(got[~bad] != base[~bad])), int(np.count_nonzero(lse[~bad] != base_lse[~bad]))
        assert numbers == (0, 0) and changed == (0, 0)
        a.q[:], a.bits[:] = q, bits
    for place in (0, len(base) - 1, int(a.off[1])):   # a query with a NaN: all of a row's scores
        bad = np.zeros(base.shape[:2], bool)
        bad[place, 1] = True
        a.q[place, 1, 3] = 0x7FC0
        expect(bad)
    for some in (list(keys), [keys[5]], list(range(int(a.total[0])))):              # keys: of a stretch, one, of all a row's tokens
        bad = np.zeros(base.shape[:2], bool)
        for j in some:
            a.bits[(0,) + a.at(0, j)] = 0x7FC0
        for i in range(a.new[0]):
            bad[i] = min(some) <= a.total[0] - a.new[0] + i
        expect(bad)


@pytest.mark.parametrize("path", NAN_PATHS)
def test_attention_scores_that_are_all_minus_infinity(B, path):
    """A row whose scores are all -inf gets zeros and -inf, whatever its values hold."""
    kind, lengths, _ = NAN_PATHS[path]
    a = kind(B, lengths, 8, 2, 64, seed=1)
    base, base_lse = a.run()
    a.q[:a.off[1]] = _bf16(np.ones_like(a.q[:a.off[1]], np.float64))
    base[:a.off[1]], base_lse[:a.off[1]] = 0, -np.inf
    for value in (0x3F80, 0x7F80, 0x7FC0):
        for j in range(int(a.total[0])):
            a.bits[(0,) + a.at(0, j)] = 0xFF80
            a.bits[(1,) + a.at(0, j)] = value
        got, lse = a.run()
        assert not np.count_nonzero(got != base) and not np.count_nonzero(lse != base_lse)


# ---- large values -------------------------------------------------------------------------------------------------
def _steps_of_scores(a, high):
    """Scores of 0, and of 7.5 for the 32 keys of every half tile that high(number of the half) names; values of 2^110, every third negative."""
    a.q[:] = _bf16(np.ones_like(a.q, np.float64))
    a.scale = 1 / a.dim
    for r, t in enumerate(a.total):
        j = np.arange(int(t))
        at = a.table[r, j // a.block], j % a.block
        a.bits[(0,) + at] = _bf16(np.where(high(j // 32), 7.5, 0.0))[:, None, None]
        a.bits[(1,) + at] = np.where(j % 3 == 2, 0xF680, 0x7680).astype(np.uint16)[:, None, None]
    return a


@pytest.mark.parametrize("kind", [Attend, Wide])
@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 64), (4, 4, 128)])
def test_attention_large_values_behind_a_low_start(B, kind, heads, kv, dim):
    """A row's first keys weigh 2^-11 of the others: sums relative to the first maximum must not grow until values of 2^110 overflow."""
    for lengths in ([(400, 40), (440, 9)], [(4056, 40), (10, 1)], [(400, 1), (4000, 1)]):
        for high in (lambda h: h > 0, lambda h: h % 16 >= 8, lambda h: (h % 16 == 1) | (h % 16 == 3)):
            a = _steps_of_scores(kind(B, lengths, heads, kv, dim, seed=1), high)
            a.check(*a.run())


@pytest.mark.parametrize("new", [1, 40])
def test_attention_large_values_of_a_long_history(B, new):
    """More than 2^18 keys of the same weight, values of 2^110: their sum has no room in fp32, their mean has."""
    a = _steps_of_scores(Attend(B, [(270000, new)], 2, 1, 8, block=64), lambda h: h < 0)
    a.bits[1][a.bits[1] == 0xF680] = 0x7680
    a.check(*a.run())


def test_attention_large_values_of_slowly_growing_sums(B):
    """Weights that are each too small to move a row's reference, and whose sum is not: two parts of seventeen tiles that begin with a low half."""
    a = _steps_of_scores(Wide(B, [(2060, 33)] * 40, 8, 8, 8, seed=1), lambda h: (h != 0) & (h != 34))
    a.bits[0][a.bits[0] == 0x40F0] = _bf16(5.3125)
    a.bits[1][a.bits[1] == 0xF680] = 0x7680
    a.check(*a.run())


# ---- block ids outside the cache ----------------------------------------------------------------------------------
@pytest.mark.parametrize("block", [8, 16, 1024])
def test_plan_ids_outside_the_cache(B, block):
    """Ids whose product with the block size would wrap round to a slot of another block give no slot, in the table and in the ring."""
    n_blocks, width, wrap = 50, 8, 2 ** 32 // block
    bad = [v - 2 ** 32 if v >= 2 ** 31 else v for v in (wrap + 1, 2 * wrap, 2 ** 32 - wrap, wrap * 3 + 7, n_blocks, 2 ** 31 - 1, 2 ** 32 - 1, 2 ** 31)]
    bad = [v for v in bad if not 0 <= v < n_blocks and -2 ** 31 <= v < 2 ** 31]
    n = len(bad)
    table = np.zeros((n + 2, width), np.int32)
    table[:n, 0] = bad
    table[n:, 0] = 11, 12
    ring = np.full(n_blocks, 13, np.int32)
    ring[5:5 + n] = bad
    have, add = [block - 3] * (n + 2), [4] * n + [2, 1]             # three tokens in the table's block, one in a block of the ring
    args = (block, n_blocks, width, 4 * n + 5, have, add, ring, [5, 40], table)
    want, got = T.plan(*args), _plan_gpu(B, *args)
    assert (want["slot"][:4 * n] == -1).all() and want["slot"][4 * n:].tolist() == [11 * block + block - 3, 11 * block + block - 2, 12 * block + block - 3, -1, -1]
    for k in want:
        assert np.array_equal(got[k], want[k]), k


# ---- sizes at the end of 32 bits ----------------------------------------------------------------------------------
def test_plan_of_the_largest_token_cap(B):
    """Room for 2^31 - 1 tokens: the padding fills it, and nothing is written outside."""
    import torch
    cap = 2 ** 31 - 1
    room = torch.full((2, cap + 1), 5, dtype=torch.int32, device="cuda")     # 17 GB
    have, add, ring, state, table = (_dev(np.array(v, np.int32)) for v in ([3, 0], [2, 9], np.arange(8), [0, 8], [[7, 0], [0, 0]]))
    out = [torch.zeros(size, dtype=torch.int32, device="cuda") for size in (2, 3, 4)]
    B.coe_kv_plan(2, 16, 8, 2, cap, *(t.data_ptr() for t in (have, add, ring, state, table, *out[:2])), room[0].data_ptr(), room[1].data_ptr(), out[2].data_ptr(),
                  _stream())
    assert [t.tolist() for t in out] == [[5, 9], [0, 2, 11], [1, 7, 2, 11]]
    assert room[:, :11].tolist() == [[7 * 16 + 3, 7 * 16 + 4, *range(9)], [3, 4, *range(9)]]
    assert (room[:, 11:cap] == -1).all().item() and room[:, cap].tolist() == [5, 5]


def test_sample_of_the_largest_vocabulary(B):
    """2^31 - 1 logits: the race's winner falls to the nucleus, and the share of its thread is looked through up to the row's end."""
    import torch
    vocab = 2 ** 31 - 1
    x = torch.full((vocab,), -9.0, dtype=torch.bfloat16, device="cuda")
    noise = torch.ones(vocab, device="cuda")
    first, drawn, lost = 77, vocab - 3000, vocab - 5000                      # the first two make the nucleus of 0.9; all but these three weigh 2^31 e^-69
    x[first], x[drawn], x[lost] = 60.0, 59.0, 55.0
    noise[drawn], noise[lost] = 0.01, 1e-6
    one = lambda v, t: torch.full((1,), v, dtype=t, device="cuda")
    temperature, top_p, token, logprob = one(1.0, torch.float32), one(0.9, torch.float32), one(-9, torch.int32), one(0.0, torch.float32)
    B.coe_sample_tokens(1, vocab, B.COE_DT_BF16, x.data_ptr(), vocab, temperature.data_ptr(), 0, top_p.data_ptr(), 0, noise.data_ptr(), vocab, token.data_ptr(),
                        logprob.data_ptr(), 0, 0, _stream())
    want = -1 - math.log(1 + math.exp(-1) + math.exp(-5))
    assert token.item() == drawn and abs(logprob.item() - want) <= 1e-5 * (1 - want)


# ---- many requests, and requests longer than announced ------------------------------------------------------------
def _check_some(a, got, lse, some):
    """Compare the rows of some requests with the 64-bit statement; `a` is left as it is."""
    import copy
    rows = np.concatenate([np.arange(a.off[r], a.off[r + 1]) for r in some]).astype(int)
    part = copy.copy(a)
    part.q, part.total, part.new, part.table = a.q[rows], a.total[some], a.new[some], a.table[some]
    part.off = np.concatenate([[0], np.cumsum(part.new)]).astype(np.int32)
    part.check(got[rows], lse[rows])


@pytest.mark.parametrize("n", [4097, 5000, 16384])
@pytest.mark.parametrize("chunks", [False, True])
def test_attention_of_thousands_of_requests(B, n, chunks):
    """More requests than the schedule keeps lengths of, and prefix sums beyond the LDS that tiles take, up to the largest number there may be."""
    rng = np.random.default_rng(n)
    lengths = [(int(h), int(m)) for h, m in zip(rng.integers(0, 12, n), rng.integers(0, 3, n))]
    odd = {0: (700, 1), 3: (40, 2), n // 2: (300, 2), n - 2: (0, 0), n - 1: (100, 1)}
    if chunks:
        odd.update({7: (20, 70), n // 3: (0, 129), n - 1: (3, 40)})
    for r, v in odd.items():
        lengths[r] = v
    a = Wide(B, lengths, 2, 1, 32, block=32, seed=n)
    got, lse = a.run()
    _check_some(a, got, lse, sorted(set(odd) | set(range(0, n, 37)) | set(range(n - 40, n))))


@pytest.mark.parametrize("kind,have,new,most", [(Attend, 100, 9, 5), (Attend, 60, 70, 40), (Wide, 100, 9, 5), (Attend, 5000, 7, 3), (Wide, 100, 150, 140), (Wide, 5000, 60, 35)])
@pytest.mark.parametrize("window", [0, 45])
def test_attention_of_requests_longer_than_announced(B, kind, have, new, most, window):
    """The first max_new rows of a request with more new tokens stand where they stand without that limit; the others are not written."""
    a = kind(B, [(30, 2), (have, new), (17, 1), (40, new)], 8, 2, 64, window=window, seed=have)
    got, lse = a.run(max_new=most)
    served = np.concatenate([np.arange(m) < most for m in a.new])
    assert (got[~served] == 0xFFC0).all() and (lse[~served] == 7.5).all() and (~served).sum() == 2 * (new - most)
    out, logs, size = T.attention(T.bf16_to_f64(a.q), T.bf16_to_f64(a.bits[0]), T.bf16_to_f64(a.bits[1]), a.total, a.off, a.table, a.block, window, a.scale)
    # the bounds of Attend.check
    assert (np.abs(T.bf16_to_f64(got) - out)[served] <= (2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 1e-3) * size + 1e-30)[served]).all()
    assert (np.abs(lse - logs)[served] <= (2e-4 + 2e-6 * np.abs(logs))[served]).all()


def test_sample_rows_alone_and_among_others(B):
    """A row's token and logarithm are the same bits alone and among up to 255 others, and within the bounds of the statement among more."""
    rng = np.random.default_rng(4)
    vocab = 9001
    settings = [(1.0, 0, 1.0, 0.0), (0.8, 0, 0.9, 0.0), (1.0, 60, 0.95, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 900, 1.0, 0.001), (1.0, 5000, 0.9, 0.0), (1.5, 0, 0.7, 0.01)]
    x, noise = (3 * rng.standard_normal((300, vocab))).astype(np.float32), _noise(rng, (300, vocab))
    t, k, p, m = (np.array([c[r % len(settings)] for r in range(300)]) for c in zip(*settings))
    token, lp = _sample_gpu(B, x[:256], t[:256], k[:256], p[:256], m[:256], noise[:256])
    for r in range(0, 256, 25):
        one = slice(r, r + 1)
        alone = _sample_gpu(B, x[one], t[one], k[one], p[one], m[one], noise[one])
        assert alone[0][0] == token[r] and alone[1][0] == lp[r]
    _check_sample(B, x, t, k, p, m, noise)
