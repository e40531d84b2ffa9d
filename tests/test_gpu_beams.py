"""The calls for decoders with rotated positions, an encoder to look at and beams against their 64-bit statement: lengths, masks, layouts and
values where they can go wrong."""
import math

import numpy as np
import pytest

from oracle import tokens as T
from tests.test_gpu_tokens import _bf16, _dev, _make_cache, _stream

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2503_02354_amd import binding
    return binding


def _bits(t):
    return t.cpu().numpy().view(np.uint16)


# ---- append with rotation ----------------------------------------------------------------------------------------------
class Rotate:
    """Random rows, positions and slots, with padding and slots outside the cache; a device run and a check of everything it may write."""

    def __init__(self, tokens, heads, kv, dim, rotated, neighbours, block=16, layout="token", far=1000, base=10000.0, seed=0):
        rng = np.random.default_rng(seed)
        self.tokens, self.heads, self.kv, self.dim, self.rotated, self.neighbours, self.block, self.layout = tokens, heads, kv, dim, rotated, neighbours, block, layout
        self.n_blocks = -(-tokens // block) + 2
        self.x = _bf16(rng.standard_normal((tokens, heads + 2 * kv, dim)))
        self.old = rng.integers(0, 65536, (2, self.n_blocks, block, kv, dim)).astype(np.uint16)
        self.position = rng.integers(0, far, tokens).astype(np.int32)
        self.position[rng.random(tokens) < 0.15] = -1
        self.slot = rng.permutation(self.n_blocks * block)[:tokens].astype(np.int32)
        out = rng.random(tokens) < 0.15
        self.slot = np.where(out, rng.choice([-1, -2 ** 31, self.n_blocks * block, 2 ** 31 - 1], tokens), self.slot).astype(np.int32)
        self.frequency = (base ** -(np.arange(rotated // 2) / (rotated / 2))).astype(np.float32)

    def call(self, B, x, q_out, cache, stream=None):
        """x [tokens][heads + 2 kv][dim] on the device; its queries, keys and values are rotated out of it."""
        self.device = getattr(self, "device", None) or [_dev(self.slot), _dev(self.position), _dev(self.frequency)]
        st, h = x.stride(), x.element_size()
        B.coe_kv_append_rotated(cache, self.tokens, self.heads, x.data_ptr(), st[0], st[1], q_out.data_ptr(), q_out.stride(0), q_out.stride(1),
                                x.data_ptr() + h * st[1] * self.heads, st[0], st[1], x.data_ptr() + h * st[1] * (self.heads + self.kv), st[0], st[1],
                                *(d.data_ptr() for d in self.device), self.rotated, B.COE_PAIR_NEIGHBOURS if self.neighbours else B.COE_PAIR_HALVES,
                                _stream() if stream is None else stream)

    def check(self, q_out, k, v, q_before):
        """Bits of what a call left in q_out [tokens][heads][dim] and the caches [blocks][block][kv][dim]."""
        x, h = self.x, self.heads
        live = self.position >= 0
        kept = live & (self.slot >= 0) & (self.slot < self.n_blocks * self.block)
        slot = self.slot[kept]
        want_v = self.old[1].copy()
        want_v[slot // self.block, slot % self.block] = x[kept, h + self.kv:]
        assert np.array_equal(v, want_v)
        untouched = np.ones((self.n_blocks, self.block), bool)
        untouched[slot // self.block, slot % self.block] = False
        assert np.array_equal(k[untouched], self.old[0][untouched]) and np.array_equal(q_out[~live], q_before[~live])
        for got, rows, pos in ((q_out[live], x[live, :h], self.position[live]), (k[slot // self.block, slot % self.block], x[kept, h:h + self.kv], self.position[kept])):
            assert np.array_equal(got[..., self.rotated:], rows[..., self.rotated:])
            want, size = T.rotate(T.bf16_to_f64(rows), pos, self.frequency, self.rotated, self.neighbours)
            # one rounding to bf16 (2^-8 of the value); the angle in turns carries two fp64 roundings of the product (2^-52 of at most 2^31 / 2 pi
            # turns) and one fp32 rounding of at most half a turn (2^-25), so at most 2 pi (2^-23.6 + 2^-25) = 7e-7 off; sine and
            # cosine two fp32 steps (1.2e-7 each), the products and the sum three more roundings (1.8e-7): 2e-6 of |a| + |b| covers them
            assert (np.abs(T.bf16_to_f64(got) - want) <= 2.0 ** -8 * np.abs(want) + 2e-6 * size + 1e-38).all()

    def run(self, B, in_place=False):
        import torch
        k, v, cache = _make_cache(B, self.old, self.layout)
        x = _dev(self.x)
        q_before = self.x[:, :self.heads].copy() if in_place else np.full((self.tokens, self.heads, self.dim), 0x1234, np.uint16)
        q_out = x[:, :self.heads] if in_place else torch.full((self.tokens, self.heads + 1, self.dim + 8), 0x1234, dtype=torch.int16, device="cuda")
        self.call(B, x, q_out, cache)
        torch.cuda.synchronize()
        got = _bits(q_out)
        if not in_place:
            assert (got[:, self.heads:] == 0x1234).all() and (got[..., self.dim:] == 0x1234).all()
        self.check(got[:, :self.heads, :self.dim], _bits(k), _bits(v), q_before)
        return got


@pytest.mark.parametrize("tokens,heads,kv,dim,rotated,block,layout", [
    (1, 1, 1, 8, 8, 8, "token"), (1, 32, 8, 128, 128, 16, "token"), (3, 12, 12, 64, 64, 16, "head"), (5, 5, 5, 40, 40, 32, "pair"), (130, 14, 2, 80, 80, 64, "token"),
    (257, 8, 8, 128, 64, 16, "head"), (33, 40, 40, 128, 128, 16, "inner"), (64, 24, 8, 96, 24, 16, "token"), (9, 4, 2, 64, 20, 16, "token"), (31, 3, 1, 24, 2, 8, "head"),
    (2001, 2, 2, 24, 22, 1024, "token"), (1000, 16, 1, 72, 72, 128, "pair"), (4, 6, 3, 104, 102, 16, "token")])
@pytest.mark.parametrize("neighbours", [False, True])
def test_append_rotated(B, tokens, heads, kv, dim, rotated, block, layout, neighbours):
    Rotate(tokens, heads, kv, dim, rotated, neighbours, block, layout, seed=tokens + dim).run(B)
    Rotate(tokens, heads, kv, dim, rotated, neighbours, block, layout, seed=tokens).run(B, in_place=True)


@pytest.mark.parametrize("far", [1, 2, 100000, 2 ** 31 - 1])
def test_append_rotated_far_positions(B, far):
    """Positions up to the largest, where an angle in 32 bits would be noise."""
    for neighbours in (False, True):
        r = Rotate(300, 4, 2, 64, 64, neighbours, far=far, base=500000.0, seed=3)
        r.position[::7] = far - 1
        r.run(B)


def test_append_rotated_keys_only_and_odd_values(B):
    """heads = 0 appends alone; infinities and NaN stay in their own pairs, and a NaN frequency gives NaN for its pair only."""
    import torch
    r = Rotate(40, 0, 3, 64, 32, False, seed=5)
    k, v, cache = _make_cache(B, r.old, "token")
    x, d = _dev(r.x), [_dev(r.slot), _dev(r.position), _dev(r.frequency)]
    B.coe_kv_append_rotated(cache, 40, 0, 0, 0, 0, 0, 0, 0, x.data_ptr(), 6 * 64, 64, x.data_ptr() + 3 * 64 * 2, 6 * 64, 64, *(t.data_ptr() for t in d), 32, 0, _stream())
    torch.cuda.synchronize()
    r.check(np.zeros((40, 0, 64), np.uint16), _bits(k), _bits(v), np.zeros((40, 0, 64), np.uint16))
    r = Rotate(20, 2, 2, 64, 64, True, seed=6)
    r.position[:] = np.arange(20)
    r.slot[:] = np.arange(20)
    clean = r.run(B)
    r.x[:, :, 5] = 0x7F80                                                 # channels 4 and 5 are a pair
    r.x[:, :, 9] = 0x7FC1
    r.frequency[10] = np.nan                                              # channels 20 and 21
    k, v, cache = _make_cache(B, r.old, "token")
    out = torch.zeros(20, 2, 64, dtype=torch.int16, device="cuda")
    r.device = None
    r.call(B, _dev(r.x), out, cache)
    torch.cuda.synchronize()
    got = _bits(out)
    odd = [4, 5, 8, 9, 20, 21]
    rest = [c for c in range(64) if c not in odd]
    assert np.array_equal(got[..., rest], clean[:, :2, :64][..., rest])
    assert not np.isfinite(T.bf16_to_f64(got[1:][..., odd])).any()


# ---- cross attention ------------------------------------------------------------------------------------------------------
class Cross:
    """Inputs of a call from (rows of the source, new tokens of each of its beams) and a device run of it."""

    def __init__(self, sources, heads, kv, dim, beams=1, layout="pair", hidden=0.0, seed=0, scale=None, sharp=1.0, gap=5):
        rng = np.random.default_rng(seed)
        self.heads, self.kv, self.dim, self.beams, self.layout = heads, kv, dim, beams, layout
        self.scale = scale if scale is not None else 1 / math.sqrt(dim)
        self.length = np.array([n for n, _ in sources], np.int32)
        new = np.array([m if isinstance(m, tuple) else (m,) * beams for _, m in sources], np.int32).reshape(-1, beams)
        self.off = np.concatenate([[0], np.cumsum(new.reshape(-1))]).astype(np.int32)
        self.most = int(new.sum(1).max())
        order = rng.permutation(len(sources))                            # sources lie in any order, rows of nobody between them
        self.first, at = np.zeros(len(sources), np.int32), gap
        for s in order:
            self.first[s] = at
            at += max(int(self.length[s]), 0) + gap
        self.rows = at
        self.q = _bf16(sharp * rng.standard_normal((int(self.off[-1]), heads, dim)))
        self.kv_bits = np.full((2, at, kv, dim), 0x7FC0, np.uint16)      # rows of nobody: NaN
        for f, n in zip(self.first, self.length):
            self.kv_bits[:, f:f + max(int(n), 0)] = _bf16(rng.standard_normal((2, max(int(n), 0), kv, dim)))
        self.seen = None
        if hidden:
            self.seen = (rng.random(at) >= hidden).astype(np.uint8) * rng.integers(1, 256, at).astype(np.uint8)

    def run(self, B, max_new=None, max_rows=None, lse=True, extra=0, poison=0xFFC0, offset=0):
        import torch
        tokens = int(self.off[-1])
        if self.layout == "pair":                                        # keys and values of a row side by side
            both = _dev(self.kv_bits.transpose(1, 0, 2, 3))
            k, v = both[:, 0], both[:, 1]
        elif self.layout == "row":
            k, v = _dev(self.kv_bits[0]), _dev(self.kv_bits[1])
        else:                                                            # heads outermost for keys, rows outermost for values
            k, v = _dev(self.kv_bits[0].transpose(1, 0, 2)).permute(1, 0, 2), _dev(self.kv_bits[1])
        seen = _dev(self.seen) if self.seen is not None else None
        states = B.coe_states(B.COE_DT_BF16, self.rows, self.kv, self.dim, k.data_ptr(), v.data_ptr(), *k.stride()[:2], *v.stride()[:2], seen.data_ptr() if seen is not None else 0)
        q = _dev(np.concatenate([self.q, self.q[:, :2]], 1))             # rows farther apart than they are long
        out = _dev(np.full((tokens + extra, self.heads + 1, self.dim), poison, np.uint16))
        logs = torch.full((tokens + extra, self.heads), 7.5, device="cuda")
        most, longest = self.most if max_new is None else max_new, max(int(self.length.max()), 0) if max_rows is None else max_rows
        need = B.coe_cross_attention_workspace(len(self.length), tokens + extra, most, longest, self.heads, self.kv, self.dim)
        work = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
        d = [_dev(a) for a in (self.off, self.first, self.length)]
        if extra:
            q = torch.cat([q, q[:1].expand(extra, -1, -1)])
        B.coe_cross_attention(states, len(self.length), tokens + extra, self.beams, most, longest, self.heads, self.scale, q.data_ptr(), q.stride(0), q.stride(1),
                              *(t.data_ptr() for t in d), out.data_ptr(), out.stride(0), out.stride(1), logs.data_ptr() if lse else 0, work.data_ptr(), need, _stream())
        torch.cuda.synchronize()
        got = _bits(out)
        assert (got[:, -1] == poison).all() and (got[tokens:] == poison).all(), "wrote outside its rows"
        return got[:tokens, :-1], logs.cpu().numpy()[:tokens] if lse else None

    def check(self, got, logs=None, max_new=None, max_rows=None, poison=0xFFC0):
        out, lse, size, served = T.cross(T.bf16_to_f64(self.q), *T.bf16_to_f64(self.kv_bits), self.off, self.first, self.length, self.beams, self.scale, self.seen, max_new, max_rows)
        assert (got[~served] == poison).all()
        got, out, size, lse = got[served], out[served], size[served], lse[served]
        g = T.bf16_to_f64(got)
        # bf16 holds 8 bits: a probability is rounded to it (2^-8 of itself at most), as is the result (2^-8); the scores carry fp32 errors: at most
        # (dim + 2) 2^-24 sum|q k| * scale, under 1e-4 for these inputs' scores, and so do sums over the rows.  Per element
        # |error| <= 2^-8 |out| + (2^-8 + 1e-3) sum p |v|; over all of them the roundings are independent: about 1.7e-3 of the norm, where
        # 4e-3 is allowed.
        bound = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 1e-3) * size + 1e-30
        assert np.isfinite(g).all()
        assert (np.abs(g - out) <= bound).all(), float((np.abs(g - out) / bound).max())
        if out.size >= 4096:
            assert np.linalg.norm(g - out) <= 4e-3 * np.linalg.norm(out)
        if logs is not None:
            logs = logs[served]
            assert np.array_equal(np.isinf(logs), np.isinf(lse)) and (logs[np.isinf(logs)] < 0).all()
            ok = np.isfinite(lse)
            assert (np.abs(logs[ok] - lse[ok]) <= 2e-4 + 2e-6 * np.abs(lse[ok])).all()


CROSS_SHAPES = [(12, 12, 64), (32, 8, 128), (8, 1, 64), (6, 2, 80), (24, 8, 96), (7, 7, 8), (5, 5, 40), (14, 2, 128), (33, 1, 64), (80, 2, 128), (4, 4, 24)]
EDGES = (1, 2, 7, 15, 16, 17, 31, 32, 33, 63, 64, 65, 96, 127, 128, 129, 200, 255, 257, 0, 300)


@pytest.mark.parametrize("heads,kv,dim", CROSS_SHAPES)
def test_cross_single_tokens(B, heads, kv, dim):
    """One token per source, rows of every remainder of a tile; then three beams to a source."""
    c = Cross([(n, 1) for n in EDGES], heads, kv, dim, seed=heads + dim)
    c.check(*c.run(B))
    c = Cross([(n, 1) for n in EDGES[::2]], heads, kv, dim, beams=3, seed=dim, hidden=0.3)
    c.check(*c.run(B))


@pytest.mark.parametrize("layout", ["pair", "row", "split"])
def test_cross_layouts(B, layout):
    for sources in ([(500, 1), (0, 1), (77, 1), (1024, 1)], [(300, 40), (1, 90), (129, 1), (135, 130)]):
        for heads, kv, dim in ((8, 2, 128), (6, 6, 64), (5, 5, 40)):
            c = Cross(sources, heads, kv, dim, layout=layout, seed=len(layout))
            c.check(*c.run(B))


@pytest.mark.parametrize("sources", [
    [(1, 2)], [(40, 31)], [(64, 33)], [(65, 64), (63, 65)], [(200, 127), (100, 128), (300, 129)], [(64, 257)],
    [(70, 0), (51, 1), (0, 0), (73, 40), (128, 0)],                 # sources without queries between others
    [(0, 5), (0, 70), (33, 3)],                                     # and some without rows
    [(300, 300), (701, 1), (720, 20), (31, 1), (1064, 64)], [(-4, 3), (10, 3)]])
@pytest.mark.parametrize("heads,kv,dim", [(4, 4, 64), (8, 2, 128), (12, 4, 96), (5, 1, 80), (2, 2, 32)])
def test_cross_chunks(B, sources, heads, kv, dim):
    for hidden in (0.0, 0.2):
        c = Cross(sources, heads, kv, dim, seed=len(sources) + dim, hidden=hidden)
        c.check(*c.run(B))


def test_cross_beams_of_different_lengths(B):
    for heads, kv, dim in ((8, 2, 128), (12, 12, 64)):
        c = Cross([(100, (1, 0, 5, 2)), (333, (0, 0, 0, 0)), (64, (40, 1, 1, 0)), (1000, (0, 3, 0, 90))], heads, kv, dim, beams=4, seed=2)
        c.check(*c.run(B))


def test_cross_long_sources_are_split(B):
    """Few sources with many rows beside short ones: parts of a source are joined again."""
    for sources in ([(9000, 1)], [(5000, 1), (3, 1), (7777, 1)], [(6000, 2), (6001, 3)], [(5000, 40), (10, 1)], [(20000, 200)], [(3000, 150), (1, 150)]):
        for heads, kv, dim in ((8, 1, 128), (4, 4, 64), (2, 1, 96)):
            for hidden in (0.0, 0.5):
                c = Cross(sources, heads, kv, dim, seed=3, hidden=hidden)
                c.check(*c.run(B))


def test_cross_many_sources(B):
    """Thousands of sources, most with a row or two."""
    rng = np.random.default_rng(1)
    c = Cross([(int(n), int(m)) for n, m in zip(rng.integers(0, 4, 6000), rng.integers(0, 3, 6000))], 2, 1, 32, seed=4)
    c.check(*c.run(B))
    c = Cross([(int(n), int(m)) for n, m in zip(rng.integers(0, 90, 700), rng.integers(0, 60, 700))], 2, 1, 64, seed=5, hidden=0.1)
    c.check(*c.run(B))


def test_cross_hidden_rows(B):
    """All rows hidden, all but one, whole tiles; and what is hidden may hold anything."""
    for heads, kv, dim in ((8, 2, 128), (4, 4, 64)):
        for m in (1, 5, 150):
            c = Cross([(300, m), (200, m), (64, m), (1, m)], heads, kv, dim, seed=m, hidden=0.1)
            c.seen[c.first[0]:c.first[0] + 300] = 0
            c.seen[c.first[0] + 217] = 9
            c.seen[c.first[1]:c.first[1] + 200] = 0
            c.seen[c.first[2]:c.first[2] + 32] = 0
            got, logs = c.run(B)
            c.check(got, logs)
            for value in (0x7F80, 0xFF80, 0x7FC0, 0x7F7F, 0xFF7F):
                c.kv_bits[:, np.flatnonzero(c.seen == 0)] = value
                again, logs_again = c.run(B)
                assert np.array_equal(got, again) and np.array_equal(logs, logs_again)


def test_cross_sharp_and_flat_scores(B):
    """Scores of some hundreds (one row takes all), all equal (a plain mean), a maximum that rises with every row, a negative scale."""
    for m in (1, 70, 200):
        c = Cross([(400, m), (300, m)], 4, 2, 128, seed=1, sharp=40.0, scale=0.5)
        got, logs = c.run(B)
        out, lse, size, _ = T.cross(T.bf16_to_f64(c.q), *T.bf16_to_f64(c.kv_bits), c.off, c.first, c.length, 1, c.scale)
        # sum|q k| * scale reaches 40 * 128 * 0.64 * 0.5 = 1640, so a score may be off by 130 * 2^-24 * 1640 = 0.013 at most
        assert (np.abs(T.bf16_to_f64(got) - out) <= 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 0.026) * size + 1e-30).all()
        assert (np.abs(logs - lse) <= 0.013 + 1e-6 * np.abs(lse)).all()
        for scale in (0.0, -0.2):
            c = Cross([(400, m), (300, m)], 4, 2, 64, seed=2, scale=scale)
            c.check(*c.run(B))
        for sign in (1.0, -1.0):
            c = Cross([(700, m), (280, m)], 4, 2, 64, seed=3)
            c.q[:] = _bf16(np.ones_like(c.q, np.float64))
            for f, n in zip(c.first, c.length):
                c.kv_bits[0, f:f + n] = _bf16(sign * np.arange(n)[:, None, None] / 64.0 * np.ones((n, 2, 64)))
            c.check(*c.run(B))


@pytest.mark.parametrize("m", [1, 6, 150])
def test_cross_infinite_scores(B, m):
    """Scores of -inf weigh nothing, rows of nothing else are empty; a NaN score makes its queries NaN, and only those of its head."""
    for heads, kv, dim, n in ((4, 2, 64, 300), (8, 2, 128, 3000)):
        c = Cross([(n, m), (50, m)], heads, kv, dim, seed=m)
        c.q[:] = _bf16(np.abs(T.bf16_to_f64(c.q)) + 0.01)
        f = int(c.first[0])
        c.kv_bits[0, f + 3, 0] = 0xFF80
        c.kv_bits[0, f + n - 7, 0] = 0xFF80
        got, logs = c.run(B)
        keep = c.kv_bits.copy()
        seen = np.ones(c.rows, np.uint8)
        seen[[f + 3, f + n - 7]] = 0
        group = heads // kv
        out, lse, _, _ = T.cross(T.bf16_to_f64(c.q[:, :group]), *T.bf16_to_f64(keep[:, :, :1]), c.off, c.first, c.length, 1, c.scale, seen)
        assert (np.abs(T.bf16_to_f64(got[:, :group]) - out) <= 0.02).all() and np.allclose(logs[:, :group], lse, atol=2e-4)
        c.kv_bits[0, int(c.first[1]):int(c.first[1]) + 50, 1] = 0xFF80
        got, logs = c.run(B)
        assert (got[m:, group:] == 0).all() and (logs[m:, group:] == -np.inf).all() and (T.bf16_to_f64(got[m:, :group]) != 0).any()
        c.kv_bits[:] = keep
        c.kv_bits[0, f + n - 1, 0] = 0x7FC0
        got, logs = c.run(B)
        assert np.isnan(T.bf16_to_f64(got[:m, :group])).all() and np.isnan(logs[:m, :group]).all()
        assert np.isfinite(T.bf16_to_f64(got[:m, group:])).all() and np.isfinite(T.bf16_to_f64(got[m:])).all()


def test_cross_large_values_find_room(B):
    """Values of 2^110 and many rows of equal weight stay finite."""
    for m in (1, 40, 150):
        c = Cross([(5000, m), (9, m)], 2, 1, 64, seed=m, scale=0.0)
        c.kv_bits[1] = _bf16(np.full(c.kv_bits[1].shape, 2.0 ** 110))
        got, _ = c.run(B)
        assert (T.bf16_to_f64(got) == 2.0 ** 110).all()


def test_cross_limits_of_sizes(B):
    """max_new and max_rows cut; rows behind the states' end and a negative first are not there; lse may be NULL; rows of no source stay as they are."""
    for heads, kv, dim in ((4, 2, 64), (8, 2, 128)):
        for sources, new, rows in (([(300, 5), (20, 2), (100, 1)], 2, 64), ([(300, 150), (200, 70), (10, 3)], 100, 250), ([(50, 9), (30, 9)], 100, 5000)):
            c = Cross(sources, heads, kv, dim, seed=new)
            got, logs = c.run(B, max_new=new, max_rows=rows, extra=3)
            c.check(got, logs, max_new=new, max_rows=rows)
            assert np.array_equal(got, c.run(B, max_new=new, max_rows=rows, lse=False)[0])
        c = Cross([(300, 3), (200, 40), (100, 1)], heads, kv, dim, seed=8)
        last = int(np.argmax(c.first))
        c.kv_bits[:, c.rows - 5:] = c.kv_bits[:, c.first[last]:c.first[last] + 5]
        c.length[last] += 100000
        c.first[(last + 1) % 3] = -1
        c.check(*c.run(B, max_rows=200000))
        c.length[last] = 2 ** 31 - 1
        c.check(*c.run(B, max_rows=200000))
        c.first[last] = 2 ** 31 - 1
        got, logs = c.run(B, max_rows=200000)
        assert (got[c.off[last]:c.off[last + 1]] == 0).all()


# Sizes at which units of 128 query rows are taken: more than 256 workgroups of 32 rows.  A limit of 50000 rows has them scheduled and cut, and single tokens
# split into stretches; without it short sources' units are found by their workgroups.
LIMITS = [None, 50000]


@pytest.mark.parametrize("max_rows", LIMITS)
@pytest.mark.parametrize("heads,kv,dim", [(16, 8, 64), (32, 8, 128), (24, 12, 96), (10, 10, 80), (16, 8, 24), (9, 9, 40), (8, 8, 8), (32, 32, 32)])
def test_cross_units(B, heads, kv, dim, max_rows):
    for sources in ([(300, 150), (1, 90), (129, 1), (64, 257), (0, 70), (65, 0), (1064, 130), (63, 33)], [(127, 500), (128, 300), (640, 129)]):
        for hidden in (0.0, 0.2):
            c = Cross(sources, heads, kv, dim, seed=len(sources) + dim, hidden=hidden)
            c.check(*c.run(B, max_rows=max_rows))


@pytest.mark.parametrize("n,beams", [(1, 1), (2, 3), (64, 1), (65, 1), (64, 2), (130, 2)])
def test_cross_units_of_many_sources(B, n, beams):
    """On both sides of the number of sources whose units their workgroups find; sources and beams without rows or tokens among them."""
    rng = np.random.default_rng(n + beams)
    sources = [(int(r), tuple(int(m) for m in rng.choice([0, 1, 17, 40, 70], beams))) for r in rng.choice([0, 1, 63, 64, 65, 200], n)]
    sources[n // 2] = (1100, (300,) * beams)
    for heads, kv, dim in ((16, 16, 64), (16, 4, 128)):
        c = Cross(sources, heads, kv, dim, beams=beams, seed=n, hidden=0.1)
        for max_rows in (1200, 6000):
            c.check(*c.run(B, max_rows=max_rows))


@pytest.mark.parametrize("max_rows", LIMITS)
@pytest.mark.parametrize("heads,kv,dim,m", [(32, 8, 128, 150), (16, 16, 64, 150), (8, 2, 128, 1), (4, 4, 64, 5)])
def test_cross_hidden_rows_by_form(B, heads, kv, dim, m, max_rows):
    """As test_cross_hidden_rows, in the forms that its sizes do not take."""
    c = Cross([(300, m), (200, m), (64, m), (1, m)], heads, kv, dim, seed=m, hidden=0.1)
    c.seen[c.first[0]:c.first[0] + 300] = 0
    c.seen[c.first[0] + 217] = 9
    c.seen[c.first[1]:c.first[1] + 200] = 0
    c.seen[c.first[2]:c.first[2] + 32] = 0
    got, logs = c.run(B, max_rows=max_rows)
    c.check(got, logs)
    for value in (0x7F80, 0xFF80, 0x7FC0, 0x7F7F, 0xFF7F):
        c.kv_bits[:, np.flatnonzero(c.seen == 0)] = value
        again, logs_again = c.run(B, max_rows=max_rows)
        assert np.array_equal(got, again) and np.array_equal(logs, logs_again)


@pytest.mark.parametrize("max_rows", LIMITS)
@pytest.mark.parametrize("heads,kv,dim,n,m", [(16, 8, 64, 300, 400), (32, 8, 128, 1500, 400), (8, 2, 128, 300, 1), (6, 6, 64, 300, 4)])
def test_cross_infinite_scores_by_form(B, heads, kv, dim, n, m, max_rows):
    """Scores of -inf and NaN, as test_cross_infinite_scores, in the forms that its sizes do not take; and scores of some hundreds."""
    c = Cross([(n, m), (50, m)], heads, kv, dim, seed=m)
    c.q[:] = _bf16(np.abs(T.bf16_to_f64(c.q)) + 0.01)
    f, group = int(c.first[0]), heads // kv
    c.kv_bits[0, [f + 3, f + n - 7], 0] = 0xFF80
    got, logs = c.run(B, max_rows=max_rows)
    seen = np.ones(c.rows, np.uint8)
    seen[[f + 3, f + n - 7]] = 0
    out, lse, _, _ = T.cross(T.bf16_to_f64(c.q[:, :group]), *T.bf16_to_f64(c.kv_bits[:, :, :1]), c.off, c.first, c.length, 1, c.scale, seen)
    # probabilities of at most 1 rounded to bf16 and values of a few units: 2^-8 of each, 0.02 at most
    assert (np.abs(T.bf16_to_f64(got[:, :group]) - out) <= 0.02).all() and np.allclose(logs[:, :group], lse, atol=2e-4)
    keep = c.kv_bits.copy()
    c.kv_bits[0, int(c.first[1]):int(c.first[1]) + 50, 1] = 0xFF80
    got, logs = c.run(B, max_rows=max_rows)
    rows = slice(group, 2 * group)
    assert (got[m:, rows] == 0).all() and (logs[m:, rows] == -np.inf).all() and (T.bf16_to_f64(got[m:, :group]) != 0).any()
    c.kv_bits[:] = keep
    c.kv_bits[0, f + n - 1, 0] = 0x7FC0
    got, logs = c.run(B, max_rows=max_rows)
    assert np.isnan(T.bf16_to_f64(got[:m, :group])).all() and np.isnan(logs[:m, :group]).all()
    assert np.isfinite(T.bf16_to_f64(got[:m, group:])).all() and np.isfinite(T.bf16_to_f64(got[m:])).all()
    c = Cross([(n, m), (200, m)], heads, kv, dim, seed=1, sharp=40.0, scale=0.5)
    got, logs = c.run(B, max_rows=max_rows)
    out, lse, size, _ = T.cross(T.bf16_to_f64(c.q), *T.bf16_to_f64(c.kv_bits), c.off, c.first, c.length, 1, c.scale)
    # as in test_cross_sharp_and_flat_scores
    assert (np.abs(T.bf16_to_f64(got) - out) <= 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 0.026) * size + 1e-30).all()
    assert (np.abs(logs - lse) <= 0.013 + 1e-6 * np.abs(lse)).all()


@pytest.mark.parametrize("max_rows", LIMITS)
def test_cross_large_values_and_limits_by_form(B, max_rows):
    """Values of 2^110; a maximum that rises with every row; scales of zero and below; max_new; rows of no source; no lse."""
    for heads, kv, m in ((16, 8, 300), (3, 3, 1)):
        c = Cross([(1200, m), (9, m)], heads, kv, 64, seed=m, scale=0.0)
        c.kv_bits[1] = _bf16(np.full(c.kv_bits[1].shape, 2.0 ** 110))
        assert (T.bf16_to_f64(c.run(B, max_rows=max_rows)[0]) == 2.0 ** 110).all()
        for scale in (0.0, -0.2):
            c = Cross([(400, m), (300, m)], heads, kv, 64, seed=2, scale=scale)
            c.check(*c.run(B, max_rows=max_rows))
        for sign in (1.0, -1.0):
            c = Cross([(700, m), (280, m)], heads, kv, 64, seed=3)
            c.q[:] = _bf16(np.ones_like(c.q, np.float64))
            for f, n in zip(c.first, c.length):
                c.kv_bits[0, f:f + n] = _bf16(sign * np.arange(n)[:, None, None] / 64.0 * np.ones((n, kv, 64)))
            c.check(*c.run(B, max_rows=max_rows))
        c = Cross([(300, m), (200, m + 9), (10, 3)], heads, kv, 64, seed=4)
        got, logs = c.run(B, max_new=m, max_rows=max_rows, extra=3)
        c.check(got, logs, max_new=m, max_rows=max_rows)
        assert np.array_equal(got, c.run(B, max_new=m, max_rows=max_rows, lse=False)[0])


@pytest.mark.parametrize("max_rows", [1200, 50000])
def test_cross_units_in_graphs(B, max_rows):
    """Captured and replayed over changed lengths, eager work between: every replay gives what an eager call gives."""
    import torch
    c = Cross([(700, 200), (300, 300), (1200, 90)], 16, 8, 64, seed=11)
    both, q = _dev(c.kv_bits.transpose(1, 0, 2, 3)), _dev(c.q)
    st = B.coe_states(1, c.rows, 8, 64, both.data_ptr(), both[:, 1].data_ptr(), 1024, 64, 1024, 64, 0)
    need = B.coe_cross_attention_workspace(3, len(c.q), c.most, max_rows, 16, 8, 64)
    work, other = (torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(2))
    d = [_dev(a) for a in (c.off, c.first, c.length)]
    out, want = (torch.zeros(c.q.shape, dtype=torch.int16, device="cuda") for _ in range(2))

    def call(to, room):
        B.coe_cross_attention(st, 3, len(c.q), 1, c.most, max_rows, 16, c.scale, q.data_ptr(), 1024, 64, *(t.data_ptr() for t in d), to.data_ptr(), 1024, 64, 0, room.data_ptr(), need,
                              _stream())
    call(out, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, work)
    for lengths in ([700, 300, 1200], [1, 0, 40], [699, 300, 1130], [700, 300, 1200]):
        d[2].copy_(torch.tensor(lengths, dtype=torch.int32))
        out.zero_()
        graph.replay()
        call(want, other)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        torch.randn(1000, device="cuda").sum().item()


def test_cross_longest_sources_first(B):
    """Between one and a few workgroups to a place on the chip sources are ranked by length: equal ones, empty ones, ones without queries among them."""
    rng = np.random.default_rng(12)
    for n, heads, kv, dim, beams in ((100, 16, 8, 64, 2), (256, 4, 4, 32, 1), (70, 8, 8, 128, 3), (129, 10, 5, 40, 1)):
        sources = [(int(a), tuple(int(m) for m in rng.integers(0, 3, beams))) for a in rng.choice([0, 1, 31, 64, 64, 65, 200, 333], n)]
        for hidden in (0.0, 0.4):
            c = Cross(sources, heads, kv, dim, beams=beams, seed=n, hidden=hidden)
            c.check(*c.run(B))


def test_cross_most_sources(B):
    """As many sources as a call takes, single tokens and chunks, a long one among them: the lists of tiles and units at their longest."""
    rng = np.random.default_rng(13)
    rows = rng.integers(0, 3, 16384)
    rows[[0, 7000, 16383]] = 9000, 40, 5000
    c = Cross([(int(n), 1) for n in rows], 2, 2, 32, seed=6, gap=0)
    c.check(*c.run(B))
    new = rng.integers(0, 2, 16384)
    new[[5, 16380]] = 400, 90
    rows[5] = 2000
    c = Cross([(int(n), int(m)) for n, m in zip(rows, new)], 2, 1, 32, seed=7, gap=0)
    c.check(*c.run(B))
    c = Cross([(5, 1)] * 8192, 2, 2, 32, beams=2, seed=8, gap=0)
    c.check(*c.run(B))


@pytest.mark.parametrize("heads,sources,max_rows", [
    (4, [(9000, 2), (30, 3), (500, 1)], 9000), (4, [(90, 2), (30, 3), (50, 1)], 90), (4, [(2000, 200), (3000, 90), (64, 300)], 3000), (4, [(60, 60), (33, 40), (9, 50)], 60),
    (16, [(600, 200), (700, 90), (64, 300)], 700), (16, [(2000, 200), (3000, 90), (64, 300)], 50000), (2, [(2000, 200), (3000, 90), (64, 300)], 50000)])
def test_cross_offsets_that_are_no_offsets(B, heads, sources, max_rows):
    """q_off that runs backwards, outside q or over itself: nothing beside q's rows is touched, and the call ends."""
    c = Cross(sources, heads, heads // 2, 64, seed=1)
    tokens, good = int(c.off[-1]), c.off.copy()
    for off in ([tokens, tokens // 2, 0, -5], [0, tokens, 0, tokens], [-7, 2 ** 31 - 1, -2 ** 31, tokens], [0, 1, 2 ** 31 - 1, 3], [tokens, tokens, tokens, 0]):
        c.off = np.asarray(off, np.int32)
        got = _cross_with_offsets(B, c, good, max_rows)
        assert (got[tokens:] == 0xFFC0).all()


def _cross_with_offsets(B, c, good, max_rows):
    """A run whose arrays have the sizes of the good offsets; returns out with rows behind the tokens."""
    import torch
    tokens = int(good[-1])
    both = _dev(c.kv_bits.transpose(1, 0, 2, 3))
    st = B.coe_states(1, c.rows, c.kv, c.dim, both.data_ptr(), both[:, 1].data_ptr(), *both.stride()[0:1], both.stride(2), both.stride(0), both.stride(2), 0)
    q, out = _dev(c.q), _dev(np.full((tokens + 8, c.heads, c.dim), 0xFFC0, np.uint16))
    need = B.coe_cross_attention_workspace(len(c.length), tokens, c.most, max_rows, c.heads, c.kv, c.dim)
    work = torch.full((need + 256,), 0xAB, dtype=torch.uint8, device="cuda")
    d = [_dev(a) for a in (c.off, c.first, c.length)]
    B.coe_cross_attention(st, len(c.length), tokens, 1, c.most, max_rows, c.heads, c.scale, q.data_ptr(), *q.stride()[:2], *(t.data_ptr() for t in d), out.data_ptr(), *out.stride()[:2], 0,
                          work.data_ptr(), need, _stream())
    torch.cuda.synchronize()
    assert (work[need:] == 0xAB).all()
    return _bits(out)


def test_cross_far_rows(B):
    """States of more than 2^32 bytes."""
    import torch
    n, stride = 70000, 40000                                             # elements; 5.6 GB
    big = torch.zeros(n * stride, dtype=torch.bfloat16, device="cuda")
    rows = big.view(n, stride)
    gen = torch.Generator(device="cuda").manual_seed(0)
    rows[:, :256] = torch.randn(n, 256, generator=gen, device="cuda").bfloat16()
    k, v = rows[:, :128].view(n, 2, 64), rows[:, 128:256].view(n, 2, 64)
    for sources in ([(69990, 100, 1), (69000, 990, 2)], [(0, 70000, 1)], [(40000, 30000, 140), (69900, 100, 140)]):
        first, length, new = ([s[i] for s in sources] for i in range(3))
        off = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        q = torch.randn(int(off[-1]), 4, 64, generator=gen, device="cuda").bfloat16()
        out, lse = torch.empty_like(q), torch.empty(len(q), 4, device="cuda")
        need = B.coe_cross_attention_workspace(len(first), len(q), max(new), max(length), 4, 2, 64)
        work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        d = [_dev(np.asarray(a, np.int32)) for a in (off, first, length)]
        B.coe_cross_attention(B.coe_states(1, n, 2, 64, k.data_ptr(), v.data_ptr(), stride, 64, stride, 64, 0), len(first), len(q), 1, max(new), max(length), 4, 0.125,
                              q.data_ptr(), 256, 64, *(t.data_ptr() for t in d), out.data_ptr(), 256, 64, lse.data_ptr(), work.data_ptr(), need, _stream())
        torch.cuda.synchronize()
        for s, (f, m, _) in enumerate(sources):
            for h in range(4):
                kk, vv = k[f:f + m, h // 2].double(), v[f:f + m, h // 2].double()
                x = q[off[s]:off[s + 1], h].double() @ kk.t().contiguous() * 0.125
                p = torch.softmax(x, 1)
                # as in Cross.check
                bound = 2.0 ** -8 * (p @ vv).abs() + (2.0 ** -8 + 1e-3) * (p @ vv.abs())
                assert ((out[off[s]:off[s + 1], h].double() - p @ vv).abs() <= bound).all()
                assert ((lse[off[s]:off[s + 1], h].double() - torch.logsumexp(x, 1)).abs() <= 2e-4).all()
    del big, rows, k, v


def test_cross_bits_do_not_depend_on_company(B):
    """The same inputs give the same bits, call after call; a source gives the same among others that change nothing about the sizes."""
    for m in (1, 40, 200):
        c = Cross([(700, m), (300, m), (1200, m)], 8, 2, 128, seed=7)
        a, la = c.run(B)
        for _ in range(3):
            b, lb = c.run(B)
            assert np.array_equal(a, b) and np.array_equal(la, lb)


# ---- beams ----------------------------------------------------------------------------------------------------------------------
def _select(B, x, score, ended, beams, picks, end, dtype="f32", extra=3, repeat=1):
    """x [rows][vocab]: float32, or bf16 bits.  Returns what the call wrote."""
    import torch
    rows, vocab = x.shape
    n = rows // beams
    d = _dev(np.concatenate([x, x[:, :1].repeat(extra, 1)], 1))           # rows farther apart than they are long
    s, e = _dev(np.asarray(score, np.float32)), None if ended is None else _dev(np.asarray(ended, np.int32))
    out = [torch.full((n + 1, picks), 77, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32, torch.int32)]
    need = B.coe_beam_workspace(n, beams, picks, vocab)
    work = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    for _ in range(repeat):
        B.coe_beam_select(n, beams, picks, vocab, B.COE_DT_F32 if dtype == "f32" else B.COE_DT_BF16, d.data_ptr(), vocab + extra, s.data_ptr(), 0 if e is None else e.data_ptr(), end,
                          *(o.data_ptr() for o in out), work.data_ptr(), need, _stream())
    torch.cuda.synchronize()
    out = [o.cpu().numpy() for o in out]
    assert all((o[n:] == 77).all() for o in out)
    return [o[:n] for o in out]


def _check_select(B, x, score, ended, beams, picks, end, dtype="f32"):
    got = _select(B, x, score, ended, beams, picks, end, dtype)
    want = T.beam(T.bf16_to_f64(x) if dtype == "bf16" else x.astype(np.float64), score, ended, beams, picks, end)
    for g, w in zip(got[1:], want[1:]):
        assert np.array_equal(g, w)
    # one rounding to fp32; weights and short sums in fp32 put at most 2^-20 on the logarithm of the sum
    finite = np.isfinite(want[0])
    assert np.array_equal(got[0][~finite], want[0][~finite].astype(np.float32))
    assert (np.abs(got[0][finite] - want[0][finite]) <= 2.0 ** -24 * np.abs(want[0][finite]) + 2.0 ** -20).all()
    return got


@pytest.mark.parametrize("beams,picks", [(1, 1), (1, 2), (2, 4), (4, 8), (5, 11), (8, 16), (3, 64), (16, 33), (32, 64), (32, 1)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select(B, beams, picks, dtype):
    """Vocabularies from one token to many, odd ones among them; some beams ended, some not there.  Equal bf16 logits are common: ties go by index."""
    for n, vocab in ((1, 1), (3, 2), (2, 7), (1, 63), (5, 65), (2, 255), (1, 1000), (3, 1025), (2, 4099), (1, 20001), (1, 70000), (40, 300)):
        rng = np.random.default_rng(vocab + beams)
        x = 3 * rng.standard_normal((n * beams, vocab))
        x = _bf16(x) if dtype == "bf16" else x.astype(np.float32)
        score = -rng.uniform(1, 9, n * beams)
        score[rng.random(n * beams) < 0.15] = -np.inf
        score[rng.random(n * beams) < 0.05] = np.nan
        ended = rng.random(n * beams) < 0.2
        score = score.astype(np.float32)
        _check_select(B, x, score, ended * rng.integers(1, 9, n * beams), beams, picks, min(2, vocab - 1), dtype)
        _check_select(B, x, score, None, beams, picks, 1 << 30, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_ties_and_orders(B, dtype):
    """Rows of one value, rising, falling, a few values only; equal beams; the best at the ends of a row."""
    to = (lambda a: _bf16(a)) if dtype == "bf16" else (lambda a: np.asarray(a, np.float32))
    for vocab in (50, 1000, 9001, 40000):
        i = np.arange(vocab)
        for row in (np.zeros(vocab), i / 64.0, -i / 64.0, (i * 7919 % 5).astype(float), np.where(i == vocab - 1, 5.0, 0.0), np.where(i == 0, 5.0, 0.0), -1e30 * (i % 3), 1e30 * (i % 3)):
            x = to(np.tile(row, (4, 1)))
            for score in (np.zeros(4), np.array([-1.0, -1, -2, -1]), np.array([0, -np.inf, -np.inf, -np.inf])):
                for picks in (1, 5, 64):
                    _check_select(B, x, score.astype(np.float32), None, 4, picks, 2, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_odd_values(B, dtype):
    """-inf and NaN are no candidates and weigh nothing; +inf takes all; rows without a candidate bring none; scores of any size."""
    to = (lambda a: _bf16(a)) if dtype == "bf16" else (lambda a: np.asarray(a, np.float32))
    rng = np.random.default_rng(0)
    for vocab in (5, 600, 30000):
        x = 2 * rng.standard_normal((12, vocab))
        x[0] = -np.inf
        x[1, 1:] = -np.inf
        x[2, ::2] = -np.inf
        x[5, :] = -np.inf
        x[6, 3] = np.inf
        x[7, [1, 4]] = np.inf
        x[8, 2:] = -3e38
        bits = to(x)
        if dtype == "bf16":
            bits[3, ::3], bits[4], bits[9, 1:] = 0x7FC0, 0xFFC1, 0x7FA0
        else:
            bits[3, ::3], bits[4], bits[9, 1:] = np.nan, -np.nan, np.nan
        for score in (np.linspace(-9, -1, 12), np.full(12, -1e30), np.zeros(12), np.where(np.arange(12) % 3 == 0, np.inf, 3e38)):
            _check_select(B, bits, score.astype(np.float32), None, 4, 9, 2, dtype)
            _check_select(B, bits, score.astype(np.float32), np.ones(12), 4, 9, -7, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_large_logits(B, dtype):
    """Maxima on both sides of 2^16, up to the largest, apart in a row's parts and among a request's rows: sums change their reference there."""
    rng = np.random.default_rng(8)
    to = (lambda a: _bf16(a)) if dtype == "bf16" else (lambda a: np.asarray(a, np.float32))
    for vocab in (700, 5000, 50000):
        x = 3 * rng.standard_normal((12, vocab))
        x[1] += 65530
        x[2] += 65545
        x[3] -= 65540
        x[4] += 1e6
        x[5, ::2] += 1e6
        x[6, vocab // 2:] += 65540
        x[7, vocab // 2:] -= 65540
        x[8] *= 1e30
        x[9, 5] = 3e38
        x[10] = -3e38
        x[11, :vocab // 3] = -1e5
        _check_select(B, to(x), np.linspace(-4, -1, 12).astype(np.float32), None, 4, 9, 2, dtype)
        _check_select(B, to(x), np.zeros(12, np.float32), None, 12, 40, 2, dtype)


@pytest.mark.parametrize("beams,picks", [(1, 64), (2, 64), (3, 64), (1, 40), (7, 50), (32, 64)])
def test_select_best_in_few_places(B, beams, picks):
    """Many picks of few rows: random ones, all in one part of a row, all in one row, a part's best spread over the others'."""
    rng = np.random.default_rng(beams + picks)
    for vocab in (3000, 130000 if beams < 8 else 20000):
        x = 3 * rng.standard_normal((2 * beams, vocab))
        score = -rng.uniform(0, 1, 2 * beams).astype(np.float32)
        for bits, dtype in ((_bf16(x), "bf16"), (x.astype(np.float32), "f32")):
            _check_select(B, bits, score, None, beams, picks, 2, dtype)
            _check_select(B, bits, score - 50 * (np.arange(2 * beams) % beams != 0).astype(np.float32), None, beams, picks, 2, dtype)
        rising = (np.arange(vocab) / 1000.0 + np.arange(2 * beams)[:, None] % beams).astype(np.float32)
        _check_select(B, rising, score, None, beams, picks, 2)
        _check_select(B, rising[:, ::-1].copy(), score, None, beams, picks, 2)
        one = x.astype(np.float32)
        one[:, vocab // 2:vocab // 2 + 100] += 20
        _check_select(B, one, score, None, beams, picks, 2)


def test_select_misaligned_rows(B):
    """Rows that begin anywhere: odd strides and bases."""
    import torch
    rng = np.random.default_rng(3)
    for dtype, t in (("f32", np.float32), ("bf16", np.uint16)):
        for vocab, shift in ((1001, 1), (2051, 3), (333, 5), (10007, 7)):
            x = 2 * rng.standard_normal((6, vocab))
            x = _bf16(x) if dtype == "bf16" else x.astype(np.float32)
            room = np.zeros(6 * (vocab + 2) + 16, t)
            room[shift:shift + 6 * (vocab + 2)].reshape(6, -1)[:, :vocab] = x
            room[shift:shift + 6 * (vocab + 2)].reshape(6, -1)[:, vocab:] = 0x7F7F if dtype == "bf16" else 3e38
            d, s = _dev(room), _dev(np.zeros(6, np.float32))
            out = [torch.zeros(2, 4, dtype=q, device="cuda") for q in (torch.float32, torch.int32, torch.int32)]
            need = B.coe_beam_workspace(2, 3, 4, vocab)
            work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
            B.coe_beam_select(2, 3, 4, vocab, B.COE_DT_F32 if dtype == "f32" else B.COE_DT_BF16, d.data_ptr() + shift * room.itemsize, vocab + 2, s.data_ptr(), 0, 2,
                              *(o.data_ptr() for o in out), 0, work.data_ptr(), need, _stream())
            want = T.beam(T.bf16_to_f64(x) if dtype == "bf16" else x.astype(np.float64), np.zeros(6), None, 3, 4, 2)
            assert np.array_equal(out[1].cpu().numpy(), want[1]) and np.array_equal(out[2].cpu().numpy(), want[2])


def test_select_many_requests(B):
    rng = np.random.default_rng(4)
    for n, beams, vocab in ((3000, 2, 40), (700, 8, 1500), (200, 4, 9000)):
        x = (2 * rng.standard_normal((n * beams, vocab))).astype(np.float32)
        _check_select(B, x, -rng.uniform(0, 5, n * beams).astype(np.float32), rng.random(n * beams) < 0.1, beams, 2 * beams, 1)


def test_select_the_same_again(B):
    rng = np.random.default_rng(5)
    x = _bf16(rng.standard_normal((8, 30000)))
    a = _select(B, x, np.zeros(8), None, 4, 16, 2, "bf16")
    b = _select(B, x, np.zeros(8), None, 4, 16, 2, "bf16", repeat=5)
    assert all(np.array_equal(p, q) for p, q in zip(a, b))
    one = _select(B, x[:4], np.zeros(4), None, 4, 16, 2, "bf16")
    assert all(np.array_equal(p[:1], q) for p, q in zip(a, one))


# ---- fork and copy --------------------------------------------------------------------------------------------------------------
def _fork(B, block, n_blocks, beams, parent, seq_len, ring, state, table, extra=1):
    import torch
    n, width = table.shape
    d = [_dev(np.asarray(a, np.int32)) for a in (parent, seq_len, table, ring, state)]
    out = [torch.full(s, -77, dtype=torch.int32, device="cuda") for s in ((n + extra, width), (n + extra,), (n + extra, 2), (4,))]
    need = B.coe_kv_fork_workspace(n // beams, beams)
    work = torch.full((max(need, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    B.coe_kv_fork(n // beams, beams, block, n_blocks, width, *(t.data_ptr() for t in d), *(t.data_ptr() for t in out), work.data_ptr(), need, _stream())
    torch.cuda.synchronize()
    got = [o.cpu().numpy() for o in out]
    assert all((o[n:] == -77).all() for o in got[:3])
    assert all(np.array_equal(t.cpu().numpy(), np.asarray(a, np.int32)) for t, a in zip((d[0], d[1], d[2], d[4]), (parent, seq_len, table, state)))
    return dict(next_table=got[0][:n], next_len=got[1][:n], copy=got[2][:n], next_state=got[3], ring=d[3].cpu().numpy())


def _check_fork(B, block, n_blocks, beams, parent, seq_len, ring, state, table):
    got = _fork(B, block, n_blocks, beams, parent, seq_len, ring, state, table)
    want = T.fork(block, n_blocks, beams, parent, seq_len, ring, state, table, np.full(table.shape, -77, np.int32))
    for name in want:
        assert np.array_equal(got[name], want[name]), name
    return got


def _families(rng, requests, beams, block, most, width=None):
    """Tables as forks leave them: per request a common beginning, own ends, all of one length; some requests with a prompt in a random row."""
    lens = rng.integers(0, most + 1, requests)
    width = width or -(-most // block) + 1
    table, length = np.full((requests * beams, width), -9, np.int32), np.zeros(requests * beams, np.int32)
    pieces, total = [], 0
    for r, m in enumerate(lens):
        b = -(-int(m) // block)
        if rng.random() < 0.25:
            row = r * beams + int(rng.integers(beams))
            length[row] = m
            pieces.append((row, row + 1, 0, b))
        else:
            shared = int(rng.integers(0, m // block + 1))
            length[r * beams:(r + 1) * beams] = m
            pieces.append((r * beams, (r + 1) * beams, 0, shared))
            pieces += [(row, row + 1, shared, b) for row in range(r * beams, (r + 1) * beams)]
    total = sum(hi - lo for *_, lo, hi in pieces)
    return table, length, pieces, total


def _fill(rng, table, pieces, n_blocks):
    order = rng.permutation(n_blocks).astype(np.int32)
    at = 0
    for r0, r1, lo, hi in pieces:
        table[r0:r1, lo:hi] = order[at:at + hi - lo]
        at += hi - lo
    head = int(rng.integers(n_blocks))
    ring = np.full(n_blocks, -5, np.int32)
    ring[(head + np.arange(n_blocks - at)) % n_blocks] = order[at:]
    return ring, [head, n_blocks - at]


@pytest.mark.parametrize("requests,beams,block,most", [(0, 4, 16, 10), (1, 1, 8, 0), (1, 1, 16, 100), (1, 4, 16, 700), (3, 2, 8, 9), (7, 5, 32, 500), (40, 8, 16, 300), (5, 32, 16, 3000),
                                                       (1, 32, 8, 6000), (257, 4, 64, 900), (500, 32, 8, 30), (16384, 1, 8, 20), (5000, 3, 16, 40)])
@pytest.mark.parametrize("spare", [0, 3, 10000])
def test_fork(B, requests, beams, block, most, spare):
    rng = np.random.default_rng(requests + beams + spare)
    table, length, pieces, total = _families(rng, requests, beams, block, most)
    n_blocks = max(total + spare, 1)
    ring, state = _fill(rng, table, pieces, n_blocks)
    n = requests * beams
    row0 = np.arange(n) // max(beams, 1) * beams
    parent = (row0 + rng.integers(0, beams, n)).astype(np.int32)
    parent[rng.random(n) < 0.1] = -1
    parent = np.where(np.repeat(rng.random(requests) < 0.1, beams), -1, parent).astype(np.int32)
    _check_fork(B, block, n_blocks, beams, parent, length, ring, state, table)
    _check_fork(B, block, n_blocks, beams, np.arange(n, dtype=np.int32), length, ring, state, table)


def test_fork_values_out_of_range(B):
    """Parents of other requests, lengths beyond the table, ids outside the cache in table and ring, a state that is no state: nothing is followed."""
    rng = np.random.default_rng(1)
    block, n_blocks, beams, width = 16, 60, 4, 5
    for trial in range(20):
        table = rng.permutation(n_blocks)[:40].reshape(8, 5).astype(np.int32)
        ring = np.full(n_blocks, -5, np.int32)
        ring[:20] = [b for b in range(n_blocks) if b not in table]
        length = rng.choice([-3, 0, 5, 16, 33, 70, 80, 1000], 8).astype(np.int32)
        parent = rng.integers(-2, 11, 8).astype(np.int32)
        table[rng.random((8, 5)) < 0.1] = rng.choice([-1, 60, 2 ** 31 - 1, -2 ** 31])
        if trial % 2:
            ring[rng.random(n_blocks) < 0.3] = 1000
        _check_fork(B, block, n_blocks, beams, parent, length, ring, [0, 20], table)
        _check_fork(B, block, n_blocks, beams, parent, length, ring, [0, -4], table)
    # no state of a ring: what is in the ring afterwards is anybody's, but the call stays inside its arrays
    for state in ([2 ** 31 - 1, 2 ** 31 - 1], [-2 ** 31, 60]):
        _fork(B, block, n_blocks, beams, parent, length, ring, state, table)


def test_fork_many_steps_conserve_blocks(B):
    """A search that runs for a while, plan and fork in turn: every block has an owner or lies in the ring, never both, and histories follow."""
    import torch
    rng = np.random.default_rng(6)
    requests, beams, block, n_blocks, width = 6, 4, 8, 160, 24
    n = requests * beams
    table, ring, state = np.zeros((n, width), np.int32), rng.permutation(n_blocks).astype(np.int32), np.array([0, n_blocks], np.int32)
    length = np.zeros(n, np.int32)
    cache = torch.full((n_blocks, block, 1, 8), -1, dtype=torch.bfloat16, device="cuda")
    struct = B.coe_kv_cache(B.COE_DT_BF16, n_blocks, block, 1, 8, cache.data_ptr(), cache.data_ptr(), *cache.stride()[:3])
    history = [[] for _ in range(n)]
    stamp = 0
    for step in range(60):
        fresh = (length.reshape(requests, beams) == 0).all(1)
        add = np.zeros(n, np.int32)
        for r in range(requests):
            if fresh[r]:
                add[r * beams] = rng.integers(1, 30)
            else:
                add[r * beams:(r + 1) * beams] = (length[r * beams:(r + 1) * beams] > 0)
        plan = T.plan(block, n_blocks, width, 400, length, add, ring, state, table)
        d = {k: _dev(v) for k, v in dict(have=length, add=add, ring=ring, state=np.asarray(state, np.int32), table=table).items()}
        out = {k: torch.zeros(s, dtype=torch.int32, device="cuda") for k, s in (("seq_len", n), ("q_off", n + 1), ("slot", 400), ("position", 400), ("next_state", 4))}
        B.coe_kv_plan(n, block, n_blocks, width, 400, *(t.data_ptr() for t in d.values()), *(t.data_ptr() for t in out.values()), _stream())
        table, ring, length, state = d["table"].cpu().numpy(), d["ring"].cpu().numpy(), out["seq_len"].cpu().numpy(), out["next_state"].cpu().numpy()[:2]
        assert np.array_equal(table, plan["table"]) and np.array_equal(length, plan["seq_len"])
        off, slot = plan["q_off"], plan["slot"]
        flat = cache.view(-1, 8)
        for row in range(n):
            for t in range(off[row], off[row + 1]):
                stamp = (stamp + 1) % 251
                flat[int(slot[t])] = float(stamp)
                history[row].append(stamp)
        parent = np.full(n, -1, np.int32)
        for r in range(requests):
            rows = [i for i in range(r * beams, (r + 1) * beams) if length[i] > 0]
            if rows and max(length[rows]) < 100 and rng.random() > 0.06:
                parent[r * beams:(r + 1) * beams] = rng.choice(rows, beams)
        got = _check_fork(B, block, n_blocks, beams, parent, length, ring, state, table)
        c, l = _dev(got["copy"]), _dev(got["next_len"])
        B.coe_kv_copy([struct], n, c.data_ptr(), l.data_ptr(), _stream())
        forked = got["next_state"][2] * beams
        history = [list(history[parent[i]]) if i < forked and parent[i] >= 0 else list(history[i]) if i >= forked else [] for i in range(n)]
        table, ring, length, state = got["next_table"], got["ring"], got["next_len"], got["next_state"][:2]
        held = {int(b) for i in range(n) for b in table[i, :-(-int(length[i]) // block)]}
        free = ring[(state[0] + np.arange(state[1])) % n_blocks].tolist()
        assert sorted(list(held) + free) == list(range(n_blocks))
        now = cache[:, :, 0, 0].float().cpu().numpy()
        for i in range(n):
            assert length[i] == len(history[i])
            assert now[table[i, np.arange(length[i]) // block], np.arange(length[i]) % block].tolist() == history[i]


@pytest.mark.parametrize("layers,kv,dim,block,layout", [(1, 1, 8, 8, "token"), (3, 5, 40, 16, "head"), (33, 2, 64, 16, "pair"), (70, 1, 24, 32, "inner"), (2, 40, 128, 64, "token"),
                                                        (2, 3, 72, 1024, "token")])
def test_copy(B, layers, kv, dim, block, layout):
    """The first rows of a block, in every layer, bit for bit; whole blocks where the length is a multiple; nothing for entries outside the cache."""
    import torch
    rng = np.random.default_rng(layers)
    n_blocks, n = 24, 9
    bits = [rng.integers(0, 65536, (2, n_blocks, block, kv, dim)).astype(np.uint16) for _ in range(layers)]
    made = [_make_cache(B, b, layout) for b in bits]
    order = rng.permutation(n_blocks)
    copy = np.stack([order[:n], order[n:2 * n]], 1).astype(np.int32)
    copy[1], copy[3], copy[5] = (-1, -1), (n_blocks, 3), (4, 2 ** 31 - 1)
    copy[7, 0] = copy[8, 0]                                              # one block to two others
    seq_len = rng.integers(1, 1000 * block, n).astype(np.int32) | 1
    seq_len[2], seq_len[4] = 5 * block, block - 1
    c, l = _dev(copy), _dev(seq_len)
    B.coe_kv_copy([m[2] for m in made], n, c.data_ptr(), l.data_ptr(), _stream())
    torch.cuda.synchronize()
    for (k, v, _), b in zip(made, bits):
        for i in range(n):
            if 0 <= copy[i, 0] < n_blocks and 0 <= copy[i, 1] < n_blocks:
                rows = seq_len[i] % block or block
                b[:, copy[i, 1], :rows] = b[:, copy[i, 0], :rows]
        assert np.array_equal(_bits(k), b[0]) and np.array_equal(_bits(v), b[1])


def test_rows_beyond_32_bits(B):
    """Caches, tokens and logits whose offsets pass 2^32 bytes."""
    import torch
    big = torch.zeros(3 * 2 ** 30 + 64, dtype=torch.bfloat16, device="cuda")         # 6 GiB
    # a cache of 3000 blocks, 2^21 bytes apart; the tokens' rows lie in a tensor of their own, 2^23 bytes apart
    n, stride, block = 3000, 2 ** 20, 8
    kv = big[:n * stride].view(n, stride)
    cache = B.coe_kv_cache(B.COE_DT_BF16, n, block, 2, 64, kv.data_ptr(), kv[:, 4096:].data_ptr(), stride, 128, 64)
    rot = Rotate(600, 4, 2, 64, 64, False, seed=4)
    x, q_out = _dev(rot.x), torch.zeros(600, 4, 64, dtype=torch.int16, device="cuda")
    rot.slot = (n * block - 1 - 39 * np.arange(600)).astype(np.int32)     # the last rows of the cache, one in 39
    rot.position = np.arange(600).astype(np.int32)
    rot.device = [_dev(rot.slot), _dev(rot.position), _dev(rot.frequency)]
    rot.call(B, x, q_out, cache)
    torch.cuda.synchronize()
    at = _dev((rot.slot // block).astype(np.int64)) * stride + _dev((rot.slot % block).astype(np.int64)) * 128
    take = lambda off: big[(at + off)[:, None] + torch.arange(128, device="cuda")].view(600, 2, 64)
    want, size = T.rotate(T.bf16_to_f64(rot.x[:, 4:6]), rot.position, rot.frequency, 64, False)
    assert (np.abs(take(0).double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2e-6 * size + 1e-38).all()          # as in Rotate.check
    assert np.array_equal(_bits(take(4096).view(torch.int16)), rot.x[:, 6:])
    # blocks to others on both sides of 2^32 bytes
    copy, length = _dev(np.array([[n - 1, 0], [n - 6, 1], [10, n - 2]], np.int32)), _dev(np.array([8, 3, 5], np.int32))
    kv[10, :1024], kv[10, 4096:5120] = 3.0, 5.0
    before = kv[[n - 1, n - 6], :5120].clone()
    B.coe_kv_copy([cache], 3, copy.data_ptr(), length.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert torch.equal(kv[0, :1024], before[0, :1024]) and torch.equal(kv[0, 4096:5120], before[0, 4096:])
    assert torch.equal(kv[1, :384], before[1, :384]) and (kv[1, 384:1024] == 0).all()
    assert (kv[n - 2, :640] == 3).all() and (kv[n - 2, 4096:4736] == 5).all() and (kv[n - 2, 640:1024] == 0).all()
    # tokens far apart, in and out
    rows = big[:700 * 2 ** 22].view(700, 2 ** 22)
    rows[:600, :512] = x.view(torch.bfloat16).reshape(600, 512)
    rows[:, 1024:1280] = 7.0
    small_k, small_v, small = _make_cache(B, rot.old, "token")
    rot.slot = np.arange(600).astype(np.int32)
    rot.device = [_dev(rot.slot), _dev(rot.position), _dev(rot.frequency)]
    d = rot.device
    B.coe_kv_append_rotated(small, 600, 4, rows.data_ptr(), 2 ** 22, 64, rows[:, 1024:].data_ptr(), 2 ** 22, 64, rows[:, 256:].data_ptr(), 2 ** 22, 64, rows[:, 384:].data_ptr(), 2 ** 22, 64,
                            *(t.data_ptr() for t in d), 64, 0, _stream())
    torch.cuda.synchronize()
    rot.check(_bits(rows[:600, 1024:1280].contiguous().view(torch.int16)).reshape(600, 4, 64), _bits(small_k), _bits(small_v), np.zeros((600, 4, 64), np.uint16))
    assert (rows[600:, 1024:1280] == 7).all()
    # and logits
    logits = big[:16 * 190000000].view(16, 190000000)
    bits = _bf16(2 * np.random.default_rng(0).standard_normal((16, 5003)))
    logits[:, 1:5004] = _dev(bits).view(torch.bfloat16)
    out = [torch.zeros(4, 8, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32, torch.int32)]
    need = B.coe_beam_workspace(4, 4, 8, 5003)
    work, score = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), torch.zeros(16, device="cuda")
    B.coe_beam_select(4, 4, 8, 5003, B.COE_DT_BF16, logits[:, 1:].data_ptr(), 190000000, score.data_ptr(), 0, 2, *(t.data_ptr() for t in out), work.data_ptr(), need, _stream())
    torch.cuda.synchronize()
    want = T.beam(T.bf16_to_f64(bits), np.zeros(16), None, 4, 8, 2)
    assert all(np.array_equal(o.cpu().numpy(), w) for o, w in zip(out[1:], want[1:]))


def test_select_long_rows(B):
    """Millions of tokens in a row; the best at its ends and where parts meet."""
    rng = np.random.default_rng(14)
    for dtype in ("f32", "bf16"):
        x = rng.standard_normal((2, 5000001))
        x[0, [0, -1, 2500000]], x[1, 1234567] = 9.0, 8.0
        _check_select(B, _bf16(x) if dtype == "bf16" else x.astype(np.float32), np.array([-1, -1.5], np.float32), None, 2, 32, 2, dtype)


def test_calls_at_once(B):
    """Calls on two streams together, each with a workspace of its own, give what they give alone."""
    import torch
    rng = np.random.default_rng(15)
    x = [_dev((2 * rng.standard_normal((16, 50000))).astype(np.float32)) for _ in range(2)]
    score = torch.zeros(16, device="cuda")
    c = Cross([(900, 90), (3000, 1), (500, 200)], 8, 2, 64, seed=3)
    both = _dev(c.kv_bits.transpose(1, 0, 2, 3))
    st = B.coe_states(1, c.rows, 2, 64, both.data_ptr(), both[:, 1].data_ptr(), 256, 64, 256, 64, 0)
    qs = [_dev(c.q), _dev(c.q[::-1].copy())]
    d = [_dev(a) for a in (c.off, c.first, c.length)]
    needs = B.coe_beam_workspace(4, 4, 8, 50000), B.coe_cross_attention_workspace(3, len(c.q), c.most, 3000, 8, 2, 64)

    def room():
        return [torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda") for n in needs]

    def outputs():
        return [torch.zeros(4, 8, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32)] + [torch.zeros(len(c.q), 8, 64, dtype=torch.int16, device="cuda")]

    def go(i, work, out, stream):
        B.coe_cross_attention(st, 3, len(c.q), 1, c.most, 3000, 8, 0.125, qs[i].data_ptr(), 512, 64, *(t.data_ptr() for t in d), out[3].data_ptr(), 512, 64, 0, work[1].data_ptr(), needs[1], stream)
        B.coe_beam_select(4, 4, 8, 50000, 0, x[i].data_ptr(), 50000, score.data_ptr(), 0, 2, *(t.data_ptr() for t in out[:3]), 0, work[0].data_ptr(), needs[0], stream)
    alone, work = [], room()
    for i in range(2):
        out = outputs()
        go(i, work, out, _stream())
        alone.append(out)
    torch.cuda.synchronize()
    streams, works, outs = [torch.cuda.Stream() for _ in range(2)], [room() for _ in range(2)], [outputs() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            go(i, works[i], outs[i], streams[i].cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i in range(2) for a, b in zip(alone[i], outs[i]))


# ---- streams, graphs ------------------------------------------------------------------------------------------------------------
def test_calls_on_another_stream_and_in_graphs(B):
    """One step captured and replayed several times, eager work between the replays, against the eager result; on a stream of its own."""
    import torch
    rng = np.random.default_rng(9)
    block, n_blocks, beams, requests, width = 16, 200, 4, 3, 20
    n = requests * beams
    table, length, pieces, _ = _families(rng, requests, beams, block, 200, width)
    ring, state = _fill(rng, table, pieces, n_blocks)
    parent = (np.arange(n) // beams * beams + rng.integers(0, beams, n)).astype(np.int32)
    crosses = [Cross([(700, m), (300, m), (1200, m)], 8, 2, 128, seed=7) for m in (4, 60)]
    logits, score = _dev(rng.standard_normal((n, 30000)).astype(np.float32)), _dev(np.zeros(n, np.float32))
    rot = Rotate(50, 4, 2, 64, 64, False, seed=2)
    k, v, cache = _make_cache(B, rot.old, "token")
    x, q_out = _dev(rot.x), torch.zeros(50, 4, 64, dtype=torch.int16, device="cuda")
    rot.device = [_dev(rot.slot), _dev(rot.position), _dev(rot.frequency)]
    ints = [_dev(np.asarray(a, np.int32)) for a in (parent, length, table, ring, state)]
    fork_out = [torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((n, width), (n,), (n, 2), (4,))]
    picks = [torch.zeros(requests, 8, dtype=t, device="cuda") for t in (torch.float32, torch.int32, torch.int32, torch.int32)]
    bufs = []
    for c in crosses:
        both, q = _dev(c.kv_bits.transpose(1, 0, 2, 3)), _dev(c.q)
        need = B.coe_cross_attention_workspace(3, len(c.q), c.most, 1200, 8, 2, 128)
        bufs.append((c, both, q, torch.zeros(c.q.shape, dtype=torch.int16, device="cuda"), torch.zeros(len(c.q), 8, device="cuda"),
                     torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), need, [_dev(a) for a in (c.off, c.first, c.length)]))
    needs = B.coe_beam_workspace(requests, beams, 8, 30000), B.coe_kv_fork_workspace(requests, beams)
    works = [torch.empty(max(m, 16), dtype=torch.uint8, device="cuda") for m in needs]
    outputs = [k, v, q_out, *fork_out, ints[3], *picks, *(b[3] for b in bufs), *(b[4] for b in bufs)]

    def step(stream):
        rot.call(B, x, q_out, cache, stream)
        for c, both, q, out, lse, work, need, d in bufs:
            st = B.coe_states(1, c.rows, 2, 128, both.data_ptr(), both.data_ptr() + 2 * 256, 512, 128, 512, 128, 0)
            B.coe_cross_attention(st, 3, len(c.q), 1, c.most, 1200, 8, c.scale, q.data_ptr(), 1024, 128, *(t.data_ptr() for t in d), out.data_ptr(), 1024, 128, lse.data_ptr(),
                                  work.data_ptr(), need, stream)
        B.coe_beam_select(requests, beams, 8, 30000, 0, logits.data_ptr(), 30000, score.data_ptr(), 0, 2, *(t.data_ptr() for t in picks), works[0].data_ptr(), needs[0], stream)
        B.coe_kv_fork(requests, beams, block, n_blocks, width, *(t.data_ptr() for t in ints), *(t.data_ptr() for t in fork_out), works[1].data_ptr(), needs[1], stream)
        B.coe_kv_copy([cache], n, fork_out[2].data_ptr(), fork_out[1].data_ptr(), stream)
    before = [t.clone() for t in outputs]
    step(_stream())
    torch.cuda.synchronize()
    want = [t.clone() for t in outputs]

    def reset():
        for t, b in zip(outputs, before):
            t.copy_(b)
        torch.cuda.synchronize()
    side = torch.cuda.Stream()
    reset()
    step(side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(t, w) for t, w in zip(outputs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(_stream())
    for _ in range(4):
        reset()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(outputs, want))
        torch.randn(1000, device="cuda").sum().item()


# ---- the example that puts them together ------------------------------------------------------------------------------------------
def _dense_decoder(d, states, ids):
    """The decoder's logits at every place of ids: whole rows of scores, fp32 on the CPU, nothing cached, positions turned in fp64."""
    import torch
    f = lambda w: w.float().cpu()
    norm = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-5)
    n, group = len(ids), d.heads // d.kv_heads
    x, seen = f(d.embedding)[ids], f(states)
    mask = torch.full((n, n), -np.inf).triu(1)

    def turn(a):
        out, _ = T.rotate(a.double().numpy(), np.arange(n), d.frequency.cpu().numpy(), d.rotated, False)
        return torch.from_numpy(out).float()

    def attend(q, k, v, mask):
        k, v = (a.repeat_interleave(group, 1) for a in (k, v))
        s = torch.einsum("qhd,khd->hqk", q, k) * d.head_dim ** -0.5 + mask
        return torch.einsum("hqk,khd->qhd", s.softmax(-1), v).reshape(n, -1)
    for layer in range(d.layers):
        q, k, v = (norm(x) @ f(d.qkv[layer])).view(n, -1, d.head_dim).split([d.heads, d.kv_heads, d.kv_heads], 1)
        x = x + attend(turn(q), turn(k), v, mask) @ f(d.o[layer])
        k, v = (seen @ f(d.cross_kv[layer])).view(len(seen), -1, d.head_dim).split([d.kv_heads, d.kv_heads], 1)
        x = x + attend((norm(x) @ f(d.cross_q[layer])).view(n, d.heads, d.head_dim), k, v, 0.0) @ f(d.cross_o[layer])
        x = x + torch.nn.functional.gelu(norm(x) @ f(d.up[layer])) @ f(d.down[layer])
    return norm(x) @ f(d.head)


def test_example_writes_what_the_dense_model_scores(B):
    """Beams over states and prompts of different lengths, blocks shared and copied: every beam's score is what whole forwards without a cache give its
    tokens, the search with one beam takes the best token at every place, and all blocks come back."""
    import importlib.util
    import pathlib
    import torch
    spec = importlib.util.spec_from_file_location("describe", pathlib.Path(__file__).parent.parent / "examples" / "describe.py")
    describe = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(describe)
    d = describe.Decoder(rotated=16)
    rng = np.random.default_rng(0)
    g = torch.Generator().manual_seed(2)
    states = [torch.randn(m, d.width, generator=g).bfloat16().cuda() for m in (1, 197, 30, 64, 300)]
    prompts = [rng.integers(2, d.vocab, m).tolist() for m in (1, 20, 7, 16, 33)]
    writer = describe.Writer(d, n_blocks=80, block_size=8, max_len=48)
    for beams, new in ((4, 10), (1, 6), (7, 3)):
        found = writer.write(states, prompts, beams, new)
        assert sorted(writer.ring[(int(writer.state[0]) + torch.arange(80, device="cuda")) % 80].tolist()) == list(range(80)) and int(writer.state[1]) == 80
        for s, prompt, list_ in zip(states, prompts, found):
            assert len(list_) == beams and len({tuple(t) for t, _ in list_}) == beams
            scores = [v for _, v in list_]
            assert scores == sorted(scores, reverse=True)
            for tokens, score in list_:
                logits = _dense_decoder(d, s, prompt + tokens)[len(prompt) - 1:-1]
                lp = logits.log_softmax(-1)[torch.arange(len(tokens)), tokens]
                # a bf16 rounding is at most 2^-8 of a value, uniform inside that: 2^-8 / sqrt(3) in the root mean square.  Some fifteen of them on
                # the way through each of two layers add up to 2^-8 sqrt(30 / 3) = 1.2 % of the state, the logits are of deviation 1 (weights:
                # variance 1 / fan-in): 0.012 each, 0.12 is ten deviations of a token
                assert abs(float(lp.sum()) - score) <= 0.12 * len(tokens)
                if beams == 1:
                    assert (logits[torch.arange(len(tokens)), tokens] >= logits.max(-1).values - 0.12).all()
    small = describe.Writer(d, n_blocks=20, block_size=8, max_len=48)
    with pytest.raises(RuntimeError, match="too small"):
        small.write(states, prompts, 4, 10)


@pytest.mark.parametrize("heads,dim", [(1, 32), (2, 64), (4, 128), (1, 24)])
def test_cross_large_values_in_the_most_parts(B, heads, dim):
    """Just below 2^26 rows, all in one place, of equal weight and with values of 2^110: as many parts as there are stretches, each with as many
    weights as a call within its limits can give it.  Sums of equal powers of two are exact up to 2^24 weights and 2^-24 of them off beyond, far below the
    half step of 2^-9 that a result of 2^110 has room for."""
    import torch
    n = 2 ** 26 - 1
    k, v = torch.ones(dim, dtype=torch.bfloat16, device="cuda"), torch.full((dim,), 2.0 ** 110, dtype=torch.bfloat16, device="cuda")
    q = torch.randn(heads, dim, generator=torch.Generator().manual_seed(dim)).bfloat16().cuda()
    out, lse = torch.zeros(heads, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(heads, device="cuda")
    need = B.coe_cross_attention_workspace(1, 1, 1, n, heads, 1, dim)
    assert need > 0
    work, d = torch.empty(need, dtype=torch.uint8, device="cuda"), [_dev(np.array(a, np.int32)) for a in ([0, 1], [0], [n])]
    B.coe_cross_attention(B.coe_states(1, n, 1, dim, k.data_ptr(), v.data_ptr(), 0, 0, 0, 0, 0), 1, 1, 1, 1, n, heads, 0.0, q.data_ptr(), heads * dim, dim, *(t.data_ptr() for t in d),
                          out.data_ptr(), heads * dim, dim, lse.data_ptr(), work.data_ptr(), need, _stream())
    torch.cuda.synchronize()
    assert (out.float() == 2.0 ** 110).all()
    # log2 of the sum within a step of its 26 (2^-19), times ln 2 1.3e-6; ln 2 itself 5e-7 of 18, the product's rounding 2^-20: 2.8e-6 in all
    assert (lse.double() - math.log(n)).abs().max() <= 4 * 18 * 2.0 ** -24


# ---- forms that the sizes above do not choose --------------------------------------------------------------------------------
def _is_whole(B, c, max_rows):
    """Above 64 sources only the form with a workgroup for every 32 query rows needs no workspace; returns its workgroups."""
    rows = c.most * (c.heads // c.kv)
    assert len(c.length) > 64 and B.coe_cross_attention_workspace(len(c.length), int(c.off[-1]), c.most, max_rows, c.heads, c.kv, c.dim) == 0
    return len(c.length) * c.kv * -(-rows // 32)


@pytest.mark.parametrize("n,beams,heads,kv,dim,tokens,rows", [
    (65, 1, 2, 2, 64, 100, 200), (100, 2, 2, 2, 64, 50, 200), (65, 1, 2, 2, 96, 100, 200), (81, 1, 2, 2, 128, 90, 120), (65, 4, 8, 2, 64, 10, 200), (70, 1, 8, 2, 128, 33, 180),
    (65, 1, 8, 2, 96, 33, 200), (72, 1, 6, 3, 40, 40, 200)])
def test_cross_ranked_sources_with_several_row_blocks(B, n, beams, heads, kv, dim, tokens, rows):
    """More than 64 short sources with more than 32 query rows: ranked by length, a source's row blocks and heads on one die; sources without rows,
    without tokens, with full and short last blocks among them."""
    rng = np.random.default_rng(n + dim)
    sources = [(int(a), tuple(int(m) for m in rng.choice([0, 1, tokens // 3, tokens - 1, tokens], beams))) for a in rng.choice([0, 1, 31, 32, 33, 100, rows - 1, rows], n)]
    sources[n // 3], sources[n - 1], sources[0] = (rows, (tokens,) * beams), (rows, (tokens,) * beams), (0, (tokens,) * beams)
    for hidden in (0.0, 0.3):
        c = Cross(sources, heads, kv, dim, beams=beams, seed=n, hidden=hidden)
        assert 256 < _is_whole(B, c, rows) <= 1024 and c.most * (heads // kv) > 32
        got, logs = c.run(B)
        c.check(got, logs)
        for value in (0x7FC0, 0xFF80) if hidden else ():
            c.kv_bits[:, np.flatnonzero(c.seen == 0)] = value
            again, logs_again = c.run(B)
            assert np.array_equal(got, again) and np.array_equal(logs, logs_again)


@pytest.mark.parametrize("dim", [64, 128])
def test_cross_unranked_sources_with_several_row_blocks(B, dim):
    """More sources than are ranked, two row blocks each."""
    rng = np.random.default_rng(dim)
    sources = [(int(a), int(m)) for a, m in zip(rng.choice([0, 1, 33, 64, 100], 300), rng.choice([0, 1, 32, 33, 40], 300))]
    sources[7] = (100, 40)
    for hidden in (0.0, 0.3):
        c = Cross(sources, 2, 1, dim, seed=dim, hidden=hidden) if dim == 64 else Cross(sources, 1, 1, dim, seed=dim, hidden=hidden)
        assert 256 < _is_whole(B, c, 100) <= 1536
        c.check(*c.run(B))


@pytest.mark.parametrize("n,heads,kv,dim,rows,beams", [(200, 16, 8, 64, 800, 2), (200, 8, 8, 96, 550, 1), (129, 12, 12, 128, 400, 2), (256, 8, 8, 64, 780, 1)])
def test_cross_ranked_sources_beyond_a_thousand_workgroups(B, n, heads, kv, dim, rows, beams):
    """Longer sources are ranked up to 2048 workgroups: several rounds of the chip's compute units, every second the other way round."""
    rng = np.random.default_rng(n)
    sources = [(int(a), tuple(int(m) for m in rng.integers(0, 3, beams))) for a in rng.choice([0, 1, 64, 64, 65, 300, rows], n)]
    sources[n // 2] = (rows, (2,) * beams)
    for hidden in (0.0, 0.4):
        c = Cross(sources, heads, kv, dim, beams=beams, seed=n, hidden=hidden)
        assert 1024 < _is_whole(B, c, rows) <= 2048 and rows * dim >= 49152
        c.check(*c.run(B))


@pytest.mark.parametrize("heads,kv,dim,m,max_rows", [
    (8, 2, 128, 1, 640), (8, 2, 128, 1, 50000), (4, 4, 64, 40, 1200), (4, 1, 32, 8, 50000),          # a workgroup each; stretches
    (16, 8, 64, 400, 1200), (32, 8, 128, 400, 1200), (32, 8, 128, 400, 50000), (2, 1, 64, 300, 50000)])       # units, listed; scheduled and cut
def test_cross_bits_do_not_depend_on_the_others(B, heads, kv, dim, m, max_rows):
    """At equal sizes a source's bits are the same whatever the other sources and their queries hold, and a query's whatever the queries beside it do: where
    some need another reference than others, or are NaN, the rest keep theirs."""
    rng = np.random.default_rng(dim + m)
    rows = [min(n, max_rows) for n in (600, 333, 1200)]
    for hidden in (0.0, 0.2):
        c = Cross([(n, m) for n in rows], heads, kv, dim, seed=m, hidden=hidden)
        want, logs = c.run(B, max_rows=max_rows)
        c.check(want, logs)
        q, states = c.q.copy(), c.kv_bits.copy()
        own, mine = slice(int(c.off[1]), int(c.off[2])), slice(int(c.first[1]), int(c.first[1]) + rows[1])
        for sharp, odd in ((30.0, None), (0.0, None), (1.0, 0x7FC0), (1.0, 0x7F80)):
            c.q[:], c.kv_bits[:] = _bf16(sharp * rng.standard_normal(q.shape)), _bf16(sharp * rng.standard_normal(states.shape))
            if odd is not None:
                c.q[::3], c.kv_bits[:, ::5] = odd, odd
            c.q[own], c.kv_bits[:, mine] = q[own], states[:, mine]
            got, again = c.run(B, max_rows=max_rows)
            assert np.array_equal(got[own], want[own]) and np.array_equal(again[own], logs[own])
        c.kv_bits[:] = states
        for sharp, odd in ((30.0, None), (0.0, None), (1.0, 0x7FC0)):
            for kept in (0, 1):                                          # every second token, so that a tile of rows holds both sorts
                other = np.arange(len(q)) % 2 != kept
                c.q[:] = q
                c.q[other] = _bf16(sharp * rng.standard_normal(q[other].shape)) if odd is None else odd
                got, again = c.run(B, max_rows=max_rows)
                assert np.array_equal(got[~other], want[~other]) and np.array_equal(again[~other], logs[~other])


@pytest.mark.parametrize("dtype,vocab", [("bf16", 130001), ("f32", 60001)])
def test_select_odd_values_in_large_batches(B, dtype, vocab):
    """More than 12 MB of logits, which are loaded past the caches: what test_select_odd_values and test_select_large_logits hold, late in a row too,
    masks of finite values over most of a vocabulary, ended and absent beams, rows at odd places."""
    to = (lambda a: _bf16(a)) if dtype == "bf16" else (lambda a: np.asarray(a, np.float32))
    rng = np.random.default_rng(vocab)
    x = 3 * rng.standard_normal((64, vocab))
    assert to(x[:1]).nbytes * 64 >= 12 << 20
    hide = rng.random((64, vocab)) < 0.9
    for row, value in ((8, -1e4), (9, -1e9), (10, -3.38e38), (11, -np.inf), (12, -100.0), (13, -65540.0)):
        x[row, hide[row]] = value
    x[16], x[17, 1:], x[18, :-1] = -np.inf, -np.inf, -np.inf
    x[19, -2], x[20, [5, -1]] = np.inf, np.inf
    x[21, -3] += 1e6
    x[22] += 65545
    x[23] -= 65540
    x[24, vocab // 2:] += 65540
    x[25, vocab // 2:] -= 1e6
    x[26] *= 1e30
    x[27] = -3e38
    x[28, :vocab // 3] = -1e5
    bits = to(x)
    nan = (0x7FC0, 0xFFC1) if dtype == "bf16" else (np.float32(np.nan), -np.float32(np.nan))
    bits[32, -1], bits[33, 7], bits[34, ::3], bits[35], bits[36, 1:] = nan[0], nan[1], nan[0], nan[1], nan[0]
    bits[37, hide[37]] = nan[0]
    score = -rng.uniform(0, 9, 64).astype(np.float32)
    score[[3, 40]], score[[5, 50]] = -np.inf, np.nan
    ended = np.zeros(64)
    ended[[1, 14, 33, 41, 42, 63]] = 1
    for picks in (9, 32):
        _check_select(B, bits, score, ended, 8, picks, 2, dtype)
    _check_select(B, bits, -rng.uniform(0, 9, 64).astype(np.float32), None, 16, 16, 2, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_select_the_longest_row(B, dtype):
    """A row of 2^31 - 1 tokens of one logit, and a few better ones: at its ends and next to 2^30.  Equal ones come by token."""
    import torch
    vocab, t = 2 ** 31 - 1, torch.float32 if dtype == "f32" else torch.bfloat16
    x = torch.full((vocab,), -8.0, dtype=t, device="cuda")
    best = {vocab - 1: 9.0, 2 ** 30: 8.5, 0: 8.0, 2 ** 30 - 1: 7.5, vocab - 8: 7.0, 123456789: 7.0}
    for i, value in best.items():
        x[i] = value
    out, score = [torch.zeros(8, dtype=q, device="cuda") for q in (torch.float32, torch.int32, torch.int32)], torch.full((1,), -2.0, device="cuda")
    need = B.coe_beam_workspace(1, 1, 8, vocab)
    work = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    B.coe_beam_select(1, 1, 8, vocab, B.COE_DT_F32 if dtype == "f32" else B.COE_DT_BF16, x.data_ptr(), vocab, score.data_ptr(), 0, 2, *(o.data_ptr() for o in out), 0, work.data_ptr(), need,
                      _stream())
    torch.cuda.synchronize()
    del x
    tokens = [vocab - 1, 2 ** 30, 0, 2 ** 30 - 1, 123456789, vocab - 8, 1, 2]
    logits = np.array([9.0, 8.5, 8.0, 7.5, 7.0, 7.0, -8.0, -8.0])
    lse = math.log(sum(math.exp(v) for v in best.values()) + (vocab - len(best)) * math.exp(-8.0))
    assert out[2].tolist() == tokens and out[1].tolist() == [0] * 8
    # as in _check_select: a lane's sum of 2^15 terms of one value is exact, or has one larger term, beside which each rounds by 2^-24 of the sum: 2^-9
    # of that lane's sum at most, which is a term of 2^16 such sums
    assert (np.abs(out[0].double().cpu().numpy() - (-2.0 + logits - lse)) <= 2.0 ** -24 * 32 + 2.0 ** -20).all()
