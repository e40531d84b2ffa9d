"""Refusals of the calls for decoders with rotated positions, an encoder to look at and beams (arguments are checked before anything touches a
device; the pointers are never followed), and their 64-bit statement against cases worked by hand.  No GPU needed."""
import ctypes

import numpy as np
import pytest

from oracle import tokens as T
from tests.test_host_tokens import BAD_CACHES, P, _cache, _refused


@pytest.fixture(scope="module")
def B():
    from paper_2503_02354_amd import build
    if build.needs_build():
        build.build()
    from paper_2503_02354_amd import binding
    return binding


def _rotated(B, **kw):
    ok = dict(cache=_cache(B), tokens=2, heads=4, q=P, qt=256, qh=64, out=P + 16, ot=256, oh=64, k=P, kt=128, kh=64, v=P, vt=128, vh=64, slot=P, position=P,
              frequency=P, rotated=64, pairing=0, stream=0)
    B.coe_kv_append_rotated(*{**ok, **kw}.values())


@pytest.mark.parametrize("kw,text", BAD_CACHES)
def test_caches_are_refused(B, kw, text):
    _refused(B, B.COE_EINVAL, text, lambda: _rotated(B, cache=_cache(B, **kw)))
    _refused(B, B.COE_EINVAL, text, B.coe_kv_copy, [_cache(B), _cache(B, **kw)], 1, P, P, 0)


def test_append_rotated_refuses(B):
    for kw, text in ((dict(tokens=-1), "n_tokens"), (dict(heads=-1), "heads"), (dict(heads=65536), "heads"), (dict(rotated=0), "rotated"), (dict(rotated=66), "rotated"),
                     (dict(rotated=7), "rotated"), (dict(rotated=-2), "rotated"), (dict(pairing=2), "pairing"), (dict(pairing=-1), "pairing"), (dict(ot=56), "smaller"), (dict(oh=8), "smaller"),
                     (dict(out=P, ot=512), "in place"), (dict(out=P, oh=72), "in place")):
        _refused(B, B.COE_EINVAL, text, lambda: _rotated(B, **kw))
    for name in ("q", "out", "k", "v", "slot", "position", "frequency"):
        _refused(B, B.COE_EINVAL, "null", lambda: _rotated(B, **{name: 0}))
    for kw in (dict(q=P + 8), dict(out=P + 2), dict(k=P + 4), dict(v=P + 8), dict(qt=100), dict(qh=-64), dict(ot=260), dict(oh=65), dict(kt=4), dict(kh=-8), dict(vt=9), dict(vh=12)):
        _refused(B, B.COE_EINVAL, "aligned", lambda: _rotated(B, **kw))
    _rotated(B, tokens=0, q=0, k=0, v=0)                                  # nothing to do


def _states(B, **kw):
    ok = dict(dtype=1, n_rows=100, kv_heads=2, head_dim=64, k=P, v=P, kr=128, kh=64, vr=128, vh=64, seen=0)
    return B.coe_states(*{**ok, **kw}.values())


def _cross(B, **kw):
    ok = dict(states=_states(B), sources=2, tokens=4, beams=2, new=2, rows=50, heads=4, scale=0.125, q=P, qt=256, qh=64, off=P, first=P, length=P, out=P, ot=256,
              oh=64, lse=P, work=P, bytes=1 << 40, stream=0)
    B.coe_cross_attention(*{**ok, **kw}.values())


def test_cross_attention_refuses(B):
    def bad(text, code=B.COE_EINVAL, **kw):
        _refused(B, code, text, lambda: _cross(B, **kw))
    for kw, text in ((dict(dtype=0), "dtype"), (dict(n_rows=-1), "n_rows"), (dict(head_dim=0), "head_dim"), (dict(head_dim=60), "head_dim"), (dict(head_dim=136), "head_dim"),
                     (dict(kv_heads=0), "kv_heads"), (dict(k=0), "null"), (dict(v=0), "null"), (dict(k=P + 8), "aligned"), (dict(v=P + 2), "aligned"), (dict(kr=100), "strides"),
                     (dict(kh=-64), "strides"), (dict(vr=4), "strides"), (dict(vh=9), "strides"), (dict(kr=2 ** 24), "2^31 bytes"), (dict(vr=2 ** 24), "2^31 bytes")):
        bad(text, states=_states(B, **kw))
    for kw in (dict(sources=-1), dict(beams=0), dict(beams=-2), dict(tokens=-1), dict(new=-1), dict(rows=-1), dict(rows=2 ** 31 - 4095),
               dict(sources=B.COE_KV_MAX_REQUESTS, beams=2), dict(sources=2 ** 20, beams=2 ** 20)):
        bad("size", **kw)
    bad("heads", heads=0), bad("heads", heads=3), bad("2^30", tokens=2 ** 28 + 1), bad("scale", scale=float("nan")), bad("scale", scale=float("-inf"))
    bad("2^22", states=_states(B, kv_heads=300), heads=300, sources=14000, beams=1)
    for name in ("q", "off", "first", "length", "out"):
        bad("null", **{name: 0})
    for kw in (dict(q=P + 8), dict(qt=100), dict(qh=-8), dict(out=P + 2), dict(ot=4), dict(oh=63)):
        bad("aligned", **kw)
    bad("smaller than head_dim", ot=0), bad("smaller than head_dim", oh=8)
    for kw in (dict(sources=0), dict(tokens=0), dict(new=0)):
        _cross(B, **kw)                                                   # nothing to do
    for sizes in ((2, 4, 2, 50), (1, 1, 1, 100000), (3, 9000, 3000, 9000)):
        need = B.coe_cross_attention_workspace(*sizes, 4, 2, 64)
        assert need >= 0
        if need:
            kw = dict(zip(("sources", "tokens", "new", "rows"), sizes), beams=1)
            bad("workspace", B.COE_ERANGE, bytes=need - 1, **kw), bad("workspace", work=0, **kw), bad("workspace", work=P + 8, **kw)
    for args in ((-1, 1, 1, 9, 4, 2, 64), (1, -1, 1, 9, 4, 2, 64), (1, 1, -1, 9, 4, 2, 64), (1, 1, 1, -1, 4, 2, 64), (1, 1, 1, 9, 3, 2, 64), (1, 1, 1, 9, 4, 0, 64),
                 (1, 1, 1, 9, 4, 2, 65), (1, 1, 1, 2 ** 31 - 1, 4, 2, 64), (1, 2 ** 28 + 1, 1, 9, 4, 2, 64), (14000, 1, 1, 9, 300, 300, 64), (B.COE_KV_MAX_REQUESTS + 1, 1, 1, 9, 4, 2, 64)):
        _refused(B, B.COE_EINVAL, "bad size", B.coe_cross_attention_workspace, *args)


def test_beam_select_refuses(B):
    names = ("requests", "beams", "picks", "vocab", "dtype", "logits", "stride", "score", "ended", "end", "next_score", "row", "token", "next_ended", "work", "bytes", "stream")
    ok = dict(zip(names, (2, 4, 8, 100, 0, P, 100, P, P, 2, P + 16, P, P, P + 32, P, 1 << 40, 0)))

    def bad(text, code=B.COE_EINVAL, **kw):
        _refused(B, code, text, B.coe_beam_select, *{**ok, **kw}.values())
    bad("n_requests", requests=-1), bad("vocab", vocab=0), bad("beams", beams=0), bad("beams", beams=B.COE_BEAM_MAX + 1), bad("picks", picks=0)
    bad("picks", picks=B.COE_BEAM_PICKS_MAX + 1), bad("dtype", dtype=2), bad("2^23", requests=2 ** 30), bad("2^23", requests=2 ** 21)
    for name in ("logits", "score", "next_score", "row", "token"):
        bad("null", **{name: 0})
    bad("misaligned", logits=P + 2), bad("misaligned", logits=P + 1, dtype=1), bad("stride", stride=99), bad("alias", next_score=P), bad("alias", next_ended=P)
    B.coe_beam_select(*{**ok, "requests": 0}.values())
    for sizes in ((2, 4, 8, 100), (1, 4, 8, 50000), (300, 8, 16, 128000)):
        need = B.coe_beam_workspace(*sizes)
        assert need >= 0
        if need:
            kw = dict(zip(("requests", "beams", "picks", "vocab"), sizes), stride=sizes[3])
            bad("workspace", B.COE_ERANGE, bytes=need - 1, **kw), bad("workspace", work=0, **kw), bad("workspace", work=P + 8, **kw)
    for args in ((-1, 4, 8, 100), (1, 0, 8, 100), (1, 33, 8, 100), (1, 4, 0, 100), (1, 4, 65, 100), (1, 4, 8, 0), (2 ** 30, 4, 8, 10), (2 ** 21, 4, 8, 10)):
        _refused(B, B.COE_EINVAL, "bad size", B.coe_beam_workspace, *args)


def test_fork_refuses(B):
    names = ("requests", "beams", "block", "blocks", "width", "parent", "len", "table", "ring", "state", "next_table", "next_len", "copy", "next", "work", "bytes", "stream")
    ok = dict(zip(names, (2, 4, 16, 100, 8, P, P, P, P, P, P + 16, P + 32, P, P + 48, P, 1 << 40, 0)))

    def bad(text, code=B.COE_EINVAL, **kw):
        _refused(B, code, text, B.coe_kv_fork, *{**ok, **kw}.values())
    bad("n_requests", requests=-1), bad("n_requests", requests=B.COE_KV_MAX_REQUESTS), bad("beams", beams=0), bad("beams", beams=B.COE_BEAM_MAX + 1)
    bad("block_size", block=12), bad("block_size", block=4), bad("block_size", block=2048), bad("n_blocks", blocks=0), bad("n_blocks", blocks=2 ** 28)
    bad("max_blocks", width=0), bad("max_blocks", width=2 ** 28), bad("max_blocks * beams", block=8, width=2 ** 27, beams=32)
    for name in ("parent", "len", "table", "ring", "state", "next_table", "next_len", "copy", "next"):
        bad("null", **{name: 0})
    bad("alias", next_table=P), bad("alias", next_len=P), bad("alias", next=P), bad("aligned", copy=P + 4)
    need = B.coe_kv_fork_workspace(2, 4)
    assert need >= 0
    if need:
        bad("workspace", B.COE_ERANGE, bytes=need - 1), bad("workspace", work=0), bad("workspace", work=P + 8)
    for args in ((-1, 4), (1, 0), (1, 33), (B.COE_KV_MAX_REQUESTS, 2)):
        _refused(B, B.COE_EINVAL, "bad size", B.coe_kv_fork_workspace, *args)


def test_copy_refuses(B):
    c = _cache(B)
    _refused(B, B.COE_EINVAL, "n -1", B.coe_kv_copy, [c], -1, P, P, 0)
    _refused(B, B.COE_EINVAL, "exceeds", B.coe_kv_copy, [c], B.COE_KV_MAX_REQUESTS + 1, P, P, 0)
    _refused(B, B.COE_EINVAL, "null", B.coe_kv_copy, [c], 1, 0, P, 0)
    _refused(B, B.COE_EINVAL, "null", B.coe_kv_copy, [c], 1, P, 0, 0)
    _refused(B, B.COE_EINVAL, "aligned", B.coe_kv_copy, [c], 1, P + 4, P, 0)
    _refused(B, B.COE_EINVAL, "block_size", B.coe_kv_copy, [c, _cache(B, block_size=8)], 1, P, P, 0)
    assert B.lib.coe_kv_copy(1, None, 1, P, P, None) == B.COE_EINVAL and B.lib.coe_kv_copy(-1, None, 1, P, P, None) == B.COE_EINVAL
    B.coe_kv_copy([], 1, P, P, 0)
    B.coe_kv_copy([c] * 3, 0, 0, 0, 0)                                    # nothing to do
    B.coe_kv_copy((B.coe_kv_cache * 2)(c, c), 0, 0, 0, 0)
    assert ctypes.sizeof(B.coe_states) == 72


# ---- the statement --------------------------------------------------------------------------------------------------
def test_statement_of_rotation_by_hand():
    """A quarter turn at position 1, half a turn at 2; the last channel pair stays."""
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0, 6.0]]] * 2)
    f = np.array([np.pi / 2, 0.0])
    out, size = T.rotate(x, np.array([1, 2]), f, 4, False)
    assert np.allclose(out, [[[-3, 2, 1, 4, 5, 6]], [[-1, 2, -3, 4, 5, 6]]]) and np.allclose(size[0, 0], [4, 6, 4, 6, 0, 0])
    out, size = T.rotate(x, np.array([1, 2]), f, 4, True)
    assert np.allclose(out, [[[-2, 1, 3, 4, 5, 6]], [[-1, -2, 3, 4, 5, 6]]]) and np.allclose(size[0, 0], [3, 3, 7, 7, 0, 0])


def test_statement_of_cross_attention_by_hand():
    k, v = np.array([[[1.0, 0]], [[0, 1.0]], [[9.0, 9.0]]]), np.array([[[2.0, -2]], [[4.0, 0]], [[7.0, 7]]])
    q = np.array([[[np.log(3.0), 0.0]]] * 3)
    out, lse, _, served = T.cross(q, k, v, [0, 1, 2, 3, 3], [0, 1], [2, 9], 2, 1.0, seen=np.array([1, 1, 0]))
    assert served.all() and np.allclose(out[:2, 0], [(3 * 2 + 4) / 4, -6 / 4]) and np.allclose(lse[:2], np.log(4)) and np.allclose(out[2, 0], [4, 0]) and lse[2, 0] == 0
    out, lse, _, served = T.cross(q, k, v, [0, 3], [-1], [2], 1, 1.0, max_new=2)
    assert served.tolist() == [True, True, False] and (out == 0).all() and np.isinf(lse).all()


def test_statement_of_beams_by_hand():
    x = np.log(np.array([[1.0, 4, 2, 1], [1, 1, 1, 5], [2, 2, 2, 2], [9, 9, 9, 9]]))
    s, row, token, ended = T.beam(x, list(np.log([0.5, 0.4, 0.06])) + [-np.inf], [0, 0, 0, 0], 4, 5, 1)
    assert row[0].tolist() == [0, 1, 0, 0, 0] and token[0].tolist() == [1, 3, 2, 0, 3] and ended[0].tolist() == [1, 0, 0, 0, 0]
    assert np.allclose(np.exp(s[0]), [0.25, 0.25, 0.125, 0.0625, 0.0625])
    s, row, token, ended = T.beam(x, list(np.log([0.5, 0.4, 0.3])) + [-np.inf], [0, 1, 1, 1], 4, 4, 1)
    assert row[0].tolist() == [1, 2, 0, 0] and token[0].tolist() == [1, 1, 1, 2] and ended[0].tolist() == [1, 1, 1, 0]
    s, row, token, ended = T.beam(np.array([[-np.inf, np.nan], [np.inf, 1.0]]), [0.0, -1.0], None, 2, 3, 0)
    assert row[0].tolist() == [1, -1, -1] and token[0].tolist() == [0, -1, -1] and s[0].tolist() == [-1, -np.inf, -np.inf] and ended[0].tolist() == [1, 0, 0]


def test_statement_of_fork_by_hand():
    """Blocks of 8.  Request 0: 10 tokens, first blocks shared; row 0 has two children, row 1 none: its last block is taken for the copy.  Request
    1: 16 tokens, nothing to copy; rows swap.  Request 2 is finished and gives three blocks back.  Request 3: a prompt in its first row, continued by both, needs
    a block of the ring."""
    table = np.array([[5, 6, 0], [5, 7, 0], [1, 2, 0], [1, 3, 0], [8, 9, 0], [8, 10, 0], [11, 0, 0], [0, 0, 0]], np.int32)
    ring = np.array([12, 13, 14] + [99] * 12, np.int32)
    out = T.fork(8, 15, 2, [0, 0, 3, 2, -1, -1, 6, 6], [10, 10, 16, 16, 12, 12, 5, 0], ring, [0, 3], table, np.full((8, 3), -4, np.int32))
    assert out["next_table"].tolist() == [[5, 6, -4], [5, 7, -4], [1, 3, -4], [1, 2, -4], [-4] * 3, [-4] * 3, [11, -4, -4], [12, -4, -4]]
    assert out["next_len"].tolist() == [10, 10, 16, 16, 0, 0, 5, 5] and out["copy"].tolist() == [[-1, -1], [6, 7]] + [[-1, -1]] * 5 + [[11, 12]]
    assert out["ring"].tolist() == [12, 13, 14, 8, 9, 10] + [99] * 9 and out["next_state"].tolist() == [1, 5, 4, 2]
    out = T.fork(8, 15, 2, [0, 0, 3, 2, -1, -1, 6, 6], [10, 10, 16, 16, 12, 12, 5, 0], ring, [0, 0], table, np.full((8, 3), -4, np.int32))
    assert out["next_len"].tolist() == [10, 10, 16, 16, 0, 0, 5, 0] and out["next_state"].tolist() == [0, 3, 3, 1] and out["next_table"][6:].tolist() == [[11, -4, -4], [-4] * 3]
