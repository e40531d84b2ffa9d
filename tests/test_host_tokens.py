"""Refusals of the calls for token-generating experts: arguments are checked before anything touches a device (no GPU needed; the
pointers are never followed), and the 64-bit statement against cases worked by hand."""
import numpy as np
import pytest

from oracle import tokens as T


@pytest.fixture(scope="module")
def B():
    from paper_2503_02354_amd import build
    if build.needs_build():
        build.build()
    from paper_2503_02354_amd import binding
    return binding


_ROOM = np.zeros(64, np.int64)
P = (_ROOM.ctypes.data + 63) // 64 * 64       # aligned host memory: an address that is not null


def _refused(B, code, text, call, *args):
    with pytest.raises(B.CoEError) as e:
        call(*args)
    assert e.value.code == code and text in str(e.value), str(e.value)


def test_plan_refuses(B):
    ok = dict(n=4, block=16, blocks=100, width=8, cap=10, have=P, add=P, ring=P, state=P, table=P, seq_len=P + 16, q_off=P, slot=P, position=P, next=P + 32)

    def call(**kw):
        B.coe_kv_plan(*{**ok, **kw}.values())
    for kw, text in ((dict(n=-1), "n_requests"), (dict(n=B.COE_KV_MAX_REQUESTS + 1), "n_requests"), (dict(block=12), "block_size"), (dict(block=4), "block_size"),
                     (dict(block=2048), "block_size"), (dict(block=0), "block_size"), (dict(blocks=0), "n_blocks"), (dict(blocks=2 ** 28), "n_blocks"),
                     (dict(width=0), "max_blocks"), (dict(width=2 ** 28), "max_blocks"), (dict(cap=-1), "token_cap"), (dict(have=0), "null"), (dict(add=0), "null"),
                     (dict(ring=0), "null"), (dict(state=0), "null"), (dict(table=0), "null"), (dict(seq_len=0), "null"), (dict(q_off=0), "null"),
                     (dict(slot=0), "null"), (dict(position=0), "null"), (dict(next=0), "null"), (dict(seq_len=P), "alias"), (dict(next=P), "alias")):
        with pytest.raises(B.CoEError) as e:
            call(**kw)
        assert e.value.code == B.COE_EINVAL and text in str(e.value) and "coe_kv_plan" in str(e.value), (kw, str(e.value))


def _cache(B, **kw):
    ok = dict(dtype=1, n_blocks=10, block_size=16, kv_heads=2, head_dim=64, k=P, v=P, block_stride=2048, token_stride=128, head_stride=64)
    return B.coe_kv_cache(*{**ok, **kw}.values())


BAD_CACHES = [(dict(k=0), "null"), (dict(v=0), "null"), (dict(dtype=0), "dtype"), (dict(block_size=20), "block_size"), (dict(head_dim=0), "head_dim"),
              (dict(head_dim=60), "head_dim"), (dict(head_dim=136), "head_dim"), (dict(kv_heads=0), "kv_heads"), (dict(n_blocks=0), "n_blocks"),
              (dict(n_blocks=2 ** 27), "n_blocks"), (dict(k=P + 8), "aligned"), (dict(v=P + 2), "aligned"), (dict(block_stride=2044), "strides"),
              (dict(token_stride=-128), "strides"), (dict(head_stride=12), "strides"), (dict(token_stride=2 ** 27), "2^31 bytes"),
              (dict(token_stride=56), "smaller than head_dim"), (dict(head_stride=8), "smaller than head_dim"), (dict(block_stride=0), "smaller than head_dim")]


@pytest.mark.parametrize("kw,text", BAD_CACHES)
def test_cache_refused_by_append_and_attention(B, kw, text):
    _refused(B, B.COE_EINVAL, text, B.coe_kv_append, _cache(B, **kw), 1, P, 128, 64, P, 128, 64, P, 0)
    _refused(B, B.COE_EINVAL, text, B.coe_kv_attention, _cache(B, **kw), 1, 1, 1, 4, 0, 1.0, P, 256, 64, P, P, P, 4, P, 256, 64, P, P, 1 << 40, 0)


def test_append_refuses(B):
    c = _cache(B)
    _refused(B, B.COE_EINVAL, "n_tokens", B.coe_kv_append, c, -1, P, 128, 64, P, 128, 64, P, 0)
    for i in (2, 5, 8):
        args = [c, 1, P, 128, 64, P, 128, 64, P, 0]
        args[i] = 0
        _refused(B, B.COE_EINVAL, "null", B.coe_kv_append, *args)
    for i, bad in ((2, P + 4), (3, 100), (4, -64), (5, P + 8), (6, 4), (7, 63)):
        args = [c, 1, P, 128, 64, P, 128, 64, P, 0]
        args[i] = bad
        _refused(B, B.COE_EINVAL, "aligned", B.coe_kv_append, *args)
    B.coe_kv_append(c, 0, 0, 0, 0, 0, 0, 0, 0, 0)                        # nothing to do


def test_attention_refuses(B):
    names = ("cache", "n", "tokens", "new", "heads", "window", "scale", "q", "qt", "qh", "off", "len", "table", "width", "out", "ot", "oh", "lse", "work",
             "bytes", "stream")
    ok = dict(zip(names, (_cache(B), 2, 3, 2, 4, 0, 0.125, P, 256, 64, P, P, P, 4, P, 256, 64, P, P, 1 << 40, 0)))

    def bad(text, code=B.COE_EINVAL, **kw):
        _refused(B, code, text, B.coe_kv_attention, *{**ok, **kw}.values())
    for kw in (dict(n=-1), dict(n=B.COE_KV_MAX_REQUESTS + 1), dict(tokens=-1), dict(new=-1), dict(window=-1)):
        bad("size", **kw)
    bad("heads", heads=0), bad("heads", heads=3), bad("max_blocks", width=0), bad("max_blocks", width=2 ** 27), bad("2^31", tokens=2 ** 30)
    bad("scale", scale=float("nan")), bad("scale", scale=float("inf"))
    for name in ("q", "off", "len", "table", "out"):
        bad("null", **{name: 0})
    for kw in (dict(q=P + 8), dict(qt=100), dict(qh=-8), dict(out=P + 2), dict(ot=4), dict(oh=63)):
        bad("aligned", **kw)
    bad("smaller than head_dim", ot=0), bad("smaller than head_dim", oh=8)
    for kw in (dict(n=0), dict(tokens=0), dict(new=0)):
        B.coe_kv_attention(*{**ok, **kw}.values())                       # nothing to do
    need = B.coe_kv_attention_workspace(2, 3, 2, 4, 2, 64)
    assert need >= 0
    if need:
        bad("workspace", B.COE_ERANGE, bytes=need - 1), bad("workspace", work=0), bad("workspace", work=P + 8)
    for args in ((-1, 1, 1, 4, 2, 64), (1, -1, 1, 4, 2, 64), (1, 1, -1, 4, 2, 64), (1, 1, 1, 3, 2, 64), (1, 1, 1, 0, 2, 64), (1, 1, 1, 4, 0, 64), (1, 1, 1, 4, 2, 65),
                 (1, 1, 1, 4, 2, 256)):
        _refused(B, B.COE_EINVAL, "bad size", B.coe_kv_attention_workspace, *args)


def test_sample_refuses(B):
    names = ("rows", "vocab", "dtype", "logits", "stride", "t", "k", "p", "m", "noise", "noise_stride", "token", "logprob", "work", "bytes", "stream")
    ok = dict(zip(names, (2, 100, 0, P, 100, P, P, P, P, P, 100, P, P, P, 1 << 40, 0)))

    def bad(text, code=B.COE_EINVAL, **kw):
        _refused(B, code, text, B.coe_sample_tokens, *{**ok, **kw}.values())
    bad("n_rows", rows=-1), bad("vocab", vocab=0), bad("dtype", dtype=2), bad("null", logits=0), bad("null", token=0), bad("greedy", noise=0, t=0)
    bad("misaligned", logits=P + 2), bad("misaligned", noise=P + 1), bad("misaligned", logits=P + 1, dtype=1), bad("stride", stride=99), bad("stride", noise_stride=99)
    B.coe_sample_tokens(*{**ok, "rows": 0}.values())
    need = B.coe_sample_workspace(2, 100)
    assert need >= 0
    if need:
        bad("workspace", B.COE_ERANGE, bytes=need - 1), bad("workspace", work=0)
    _refused(B, B.COE_EINVAL, "bad size", B.coe_sample_workspace, -1, 5)
    _refused(B, B.COE_EINVAL, "bad size", B.coe_sample_workspace, 5, 0)


def test_statement_of_plan_by_hand():
    """Blocks of 8; request 0 has 7 tokens and takes none for one more, request 1 has 8 and takes one, 2 is finished, 3 does not fit."""
    table = np.array([[5, 0], [6, 0], [1, 3], [0, 0]], np.int32)
    ring = np.array([9, 9, 9, 9, 9, 9, 9, 4], np.int32)
    out = T.plan(8, 8, 2, 9, [7, 8, 12, 0], [1, 1, -1, 3], ring, [7, 1], table)
    assert out["seq_len"].tolist() == [8, 9, 0, 0] and out["q_off"].tolist() == [0, 1, 2, 2, 2]
    assert out["slot"].tolist() == [5 * 8 + 7, 4 * 8] + [-1] * 7 and out["position"].tolist() == [7, 8] + [-1] * 7
    assert out["table"].tolist() == [[5, 0], [6, 4], [1, 3], [0, 0]] and out["ring"].tolist() == [1, 3, 9, 9, 9, 9, 9, 4]
    assert out["next_state"].tolist() == [0, 2, 3, 2]


def test_statement_of_attention_by_hand():
    k = np.zeros((2, 8, 1, 2)); v = np.zeros((2, 8, 1, 2))
    k[1, 0, 0], k[1, 1, 0] = (1, 0), (0, 1)
    v[1, 0, 0], v[1, 1, 0] = (2, -2), (4, 0)
    q = np.array([[[np.log(3.0), 0.0]], [[np.log(3.0), 0.0]]])
    out, lse, _ = T.attention(q, k, v, [2], [0, 2], np.array([[1]]), 8, 0, 1.0)
    assert np.allclose(out[0, 0], [2, -2]) and np.allclose(lse[0, 0], np.log(3))
    assert np.allclose(out[1, 0], [(3 * 2 + 4) / 4, -6 / 4]) and np.allclose(lse[1, 0], np.log(4))
    out, lse, _ = T.attention(q, k, v, [1], [0, 2], np.array([[1]]), 8, 0, 1.0)
    assert np.all(out[0] == 0) and lse[0, 0] == -np.inf and np.allclose(out[1, 0], [2, -2])


def test_statement_of_sampling_by_hand():
    x = np.log(np.array([1.0, 4.0, 2.0, 1.0]))
    e = np.array([1e-3, 1.0, 0.1, 1e-4])
    assert T.sample(x, 1.0, 0, 1.0, 0.0, e)[0] == {3} and T.sample(x, 1.0, 3, 1.0, 0.0, e)[0] == {0} and T.sample(x, 1.0, 2, 1.0, 0.0, e)[0] == {2}
    assert T.sample(x, 1.0, 0, 0.5, 0.0, e)[0] == {1} and T.sample(x, 1.0, 0, 0.51, 0.0, e)[0] == {2} and T.sample(x, 1.0, 0, 1.0, 0.3, e)[0] == {2}
    assert T.sample(x, 0.0, 0, 1.0, 0.0, e)[0] == {1} and T.sample(np.full(4, -np.inf), 1.0, 0, 1.0, 0.0, e)[0] == {-1}
    assert np.allclose(T.sample(x, 1.0, 0, 1.0, 0.0, e)[1], np.log(np.array([1, 4, 2, 1]) / 8))


def test_statement_of_plan_ids_outside_the_cache():
    """Blocks of 16 of a cache of 8: an id from the table and one from the ring that would wrap round to other blocks' slots in 32 bits."""
    table = np.array([[0x10000001, 0], [3, 0]], np.int32)
    out = T.plan(16, 8, 2, 4, [15, 2], [2, 1], np.full(8, -2 ** 28, np.int32), [0, 8], table)
    assert out["slot"].tolist() == [-1, -1, 3 * 16 + 2, -1] and out["position"].tolist() == [15, 16, 2, -1]
    assert out["table"].tolist() == [[0x10000001, -2 ** 28], [3, 0]] and out["next_state"].tolist() == [1, 7, 2, 3]


def test_attention_refuses_sizes_that_leave_no_room_for_whole_tiles(B):
    """Lengths and query rows so near 2^31 that rounding them up to a tile of 32, 64 or 128 does not fit 32 bits."""
    def call(heads, tokens, block, width):
        B.coe_kv_attention(_cache(B, kv_heads=1, n_blocks=1, block_size=block, block_stride=64 * 1024), 1, tokens, tokens, heads, 0, 1.0, P, 64, 64, P, P, P, width,
                           P, 64, 64, P, P, 0, 0)
    for heads, tokens, block, width, text in ((1, 2 ** 31 - 1, 16, 4, "n_tokens * heads"), (3, (2 ** 31 - 1) // 3, 16, 4, "n_tokens * heads"), (1, 2 ** 31 - 4095, 16, 4, "n_tokens * heads"),
                                              (1, 1, 8, 2 ** 28 - 1, "max_blocks"), (1, 1, 16, 2 ** 27 - 1, "max_blocks"), (1, 1, 1024, 2 ** 21 - 3, "max_blocks")):
        _refused(B, B.COE_EINVAL, text, call, heads, tokens, block, width)
    for sizes in ((1, 2 ** 31 - 4096, 16, 4), (1, 1, 8, 2 ** 28 - 512), (1, 1, 1024, 2 ** 21 - 4)):       # the largest get as far as the workspace
        _refused(B, B.COE_ERANGE, "workspace", call, *sizes)
