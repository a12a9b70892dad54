"""KV cache operators on the CPU: the oracle pinned to hand-worked cases, and
the refusals of the entry points (made-up addresses: every check runs before
the first HIP call)."""
import ctypes as C
import math

import numpy as np
import pytest

from oracle import kvstep
from paper_2511_11617_amd import atp

# ---- the oracle ----------------------------------------------------------------


def test_extend_by_hand():
    # 4-token blocks; sequence 0 fills its block and takes one more, 1 starts, 2 has nothing new
    table = [[5, -1, -1], [-1, -1, -1], [0, 2, -1]]
    new, starts, slots, pos, status = kvstep.extend(table, [3, 0, 7], [2, 5, 0], 4, 7, 9)
    assert new.tolist() == [[5, 1, -1], [3, 4, -1], [0, 2, -1]]
    assert starts == [0, 2, 7, 7]
    assert slots == [23, 4, 12, 13, 14, 15, 16, -1, -1] and pos == [3, 4, 0, 1, 2, 3, 4, 0, 0]
    assert status == [0, 7, 3, 1]


def test_extend_refusals():
    assert kvstep.extend([[0, -1]], [4], [1], 4, 1, 1)[4] == [kvstep.ECAPACITY, 0, 1, 0]
    assert kvstep.extend([[0, 7]], [4], [0], 4, 7, 1)[4][0] == kvstep.EINVAL   # id 7 of 7
    assert kvstep.extend([[0], [0]], [3, 3], [1, 0], 4, 2, 1)[4][0] == kvstep.EINVAL  # a shared block would be written
    assert kvstep.extend([[0], [0]], [3, 3], [0, 0], 4, 2, 1)[4][0] == kvstep.OK
    assert kvstep.extend([[0]], [4], [1], 4, 2, 1)[4][0] == kvstep.EINVAL      # past max_blocks


def test_rotation_by_hand():
    x = np.zeros((1, 1, 4))
    x[0, 0] = [1, 0, 0, 2]
    f = kvstep.frequencies(4, 100.0)
    assert f == [1.0, pytest.approx(0.1)]
    y = kvstep.rotate(x, [2], f)[0, 0]  # pairs (0, 2) by 2, (1, 3) by 0.2
    assert y == pytest.approx([math.cos(2), -2 * math.sin(.2), math.sin(2), 2 * math.cos(.2)])
    y = kvstep.rotate(x, [2], f, interleaved=True, amplitude=3.0)[0, 0]
    assert y == pytest.approx([3 * math.cos(2), 3 * math.sin(2), -6 * math.sin(.2), 6 * math.cos(.2)])


def test_scaled_frequencies():
    assert kvstep.frequencies(4, 100.0, "linear", 4.0) == pytest.approx([0.25, 0.025])
    # turns over 1000 positions: 159.2 (kept), 15.92 (between 10 and 20: keep 0.5915)
    k = (1000 * 0.1 / (2 * math.pi) - 10) / 10
    assert kvstep.frequencies(4, 100.0, "parts", 4.0, 10, 20, 1000) == pytest.approx([1.0, 0.1 * k + 0.025 * (1 - k)])


def test_attention_by_hand():
    q = np.array([[[1.0, 0.0]], [[0.0, 1.0]]])
    K, V = np.array([[[0.0, 0.0]], [[math.log(3), 5.0]], [[9.0, 0.0]]]), np.array([[[1.0, 2.0]], [[5.0, 6.0]], [[8.0, 9.0]]])
    out, lse, *_ = kvstep.attend(q, [K], [V], [0, 2], [1], (0, 1), (0, 1), 1, 1.0)
    assert out[0, 0] == pytest.approx([4, 5]) and lse[0, 0] == pytest.approx(math.log(4))  # weights 1/4, 3/4
    out, lse, *_ = kvstep.attend(q, [K], [V], [0, 2], [1], (0, 1), (0, 1), 1, 1.0, window=1)
    assert out[:, 0] == pytest.approx(V[1:, 0])
    out, lse, *_ = kvstep.attend(q, [K], [V], [0, 2], [1], (0, 1), (0, 1), 1, 1.0, seen=[[False] * 3])
    assert not out.any() and np.all(np.isneginf(lse))


# ---- refusals ---------------------------------------------------------------------
A = 1 << 40  # made-up device addresses, 1 GiB apart


def _addr(i):
    return A + (i << 30)


def _cache(**kw):
    d = dict(arena=_addr(0), arena_bytes=1 << 29, num_layers=2, block_tokens=16, head_dim=64, num_blocks=64,
             q_heads=(3, 8), kv_heads=(0, 2), group=4)
    d.update(kw)
    return atp.KVCache(**d)


def _step(**kw):
    d = dict(block_table=_addr(1), n_seq=4, max_blocks=8, cached=_addr(2), fresh=_addr(3), starts=_addr(4), slots=_addr(5),
             positions=_addr(6), max_tokens=8, max_fresh=2, max_ctx=128, status=_addr(7))
    d.update(kw)
    return atp.KVStep(**d)


def _extend(c=None, s=None, table=_addr(8), ws=_addr(9), ws_bytes=1 << 20):
    atp.kv_extend(c or _cache(), s or _step(), table, ws, ws_bytes, 0)


def _append(c=None, s=None, layer=1, rope=atp.Rope(64), q=_addr(10), qs=320, k=_addr(11), ks=128, v=_addr(12), vs=128,
            o=_addr(13), os=320):
    atp.kv_append(c or _cache(), s or _step(), layer, rope, q, qs, k, ks, v, vs, o, os, 0)


def _attend(c=None, s=None, layer=1, mask=atp.Mask(0.125), q=_addr(10), qs=320, o=_addr(13), os=320, lse=_addr(14),
            ws=_addr(9), ws_bytes=1 << 29):
    atp.kv_attend(c or _cache(), s or _step(), layer, mask, q, qs, o, os, lse, ws, ws_bytes, 0)


def _refused(code, text, f, *args, **kw):
    with pytest.raises(atp.AtpError) as e:
        f(*args, **kw)
    assert e.value.code == code and text in str(e.value), str(e.value)


BAD_CACHES = [
    (dict(block_tokens=0), "block_tokens"), (dict(num_blocks=0), "num_blocks"), (dict(num_blocks=1 << 31), "num_blocks")]
BAD_SHAPES = BAD_CACHES + [
    (dict(head_dim=0), "head_dim"), (dict(head_dim=60), "head_dim"), (dict(head_dim=264), "head_dim"),
    (dict(num_layers=0), "num_layers"), (dict(layout=2), "layout"), (dict(dtype=atp.E4M3), "dtype"),
    (dict(dtype=atp.BF16, cache_dtype=atp.FP16), "cache_dtype"), (dict(cache_dtype=atp.E4M3), "scales"),
    (dict(scales=_addr(15)), "scales"), (dict(q_heads=(5, 4)), "head range"), (dict(q_heads=(-1, 4)), "head range"),
    (dict(group=0), "group"), (dict(kv_heads=(1, 2)), "kv_heads"), (dict(kv_heads=(0, 1)), "kv_heads"),
    (dict(block_tokens=1 << 27), "2 GiB")]


@pytest.mark.parametrize("kw,text", BAD_CACHES)
def test_extend_refuses_a_bad_cache(kw, text):
    _refused(atp.EINVAL, text, _extend, _cache(**kw))


@pytest.mark.parametrize("kw,text", BAD_SHAPES)
def test_append_and_attend_refuse_a_bad_cache(kw, text):
    _refused(atp.EINVAL, text, _append, _cache(**kw))
    _refused(atp.EINVAL, text, _attend, _cache(**kw))
    _refused(atp.EINVAL, text, atp.kv_attend_workspace, _cache(**kw), _step())


def test_a_rank_whose_kv_widths_do_not_cover_its_query_heads_is_refused():
    # 40 / 8 heads, widths 14/13/13 and 3/3/2 as the dense 4 -> 3 workload states them: rank 1 lacks KV head 2
    _refused(atp.EINVAL, "KV head", _attend, _cache(q_heads=(14, 27), kv_heads=(3, 6), group=5))


def test_arena_refusals():
    need = 2 * 2 * 64 * 2 * 16 * 64 * 2
    for f in (_append, _attend):
        _refused(atp.ECAPACITY, "arena_bytes", f, _cache(arena_bytes=need - 1))
        _refused(atp.EINVAL, "arena is NULL", f, _cache(arena=0))
        _refused(atp.EALIGN, "arena", f, _cache(arena=_addr(0) + 128))
        _refused(atp.EINVAL, "layer", f, layer=2)
        _refused(atp.EINVAL, "layer", f, layer=-1)


@pytest.mark.parametrize("kw", [dict(n_seq=-1), dict(max_tokens=-1), dict(max_blocks=-1), dict(max_blocks=0)])
def test_step_size_refusals(kw):
    _refused(atp.EINVAL, "step", _extend, s=_step(**kw))
    _refused(atp.EINVAL, "step", _attend, s=_step(**kw))


@pytest.mark.parametrize("field", ["block_table", "cached", "fresh", "starts", "slots", "positions", "status"])
def test_extend_refuses_missing_misaligned_and_overlapping_buffers(field):
    _refused(atp.EINVAL, field, _extend, s=_step(**{field: 0}))
    _refused(atp.EALIGN, field, _extend, s=_step(**{field: _addr(1) + 2}))
    if field in ("cached", "fresh"):
        _refused(atp.EINVAL, "overlaps an input", _extend, s=_step(**{field: _addr(1) + 4}))
    elif field != "block_table":
        _refused(atp.EINVAL, "overlap", _extend, s=_step(**{field: _addr(1) + 8}))
    else:
        _refused(atp.EINVAL, "overlaps an input", _extend, s=_step(block_table=_addr(8) + 4))


def test_extend_workspace_refusals():
    n = atp.kv_extend_workspace(_cache(), _step())
    _refused(atp.ECAPACITY, "workspace", _extend, ws_bytes=n - 1)
    _refused(atp.EINVAL, "workspace", _extend, ws=0)
    _refused(atp.EALIGN, "workspace", _extend, ws=_addr(9) + 64)
    _refused(atp.EINVAL, "overlap", _extend, ws=_addr(1))


@pytest.mark.parametrize("rope", [
    dict(rot_dim=63), dict(rot_dim=-2), dict(rot_dim=66), dict(rot_dim=64, base=0.0), dict(rot_dim=64, base=math.inf),
    dict(rot_dim=64, scaling=3), dict(rot_dim=64, scaling=atp.ROPE_LINEAR, factor=0.0),
    dict(rot_dim=64, scaling=atp.ROPE_PARTS, factor=4.0, low=8.0, high=8.0, original=100.0),
    dict(rot_dim=64, scaling=atp.ROPE_PARTS, factor=4.0, low=1.0, high=8.0, original=0.0),
    dict(rot_dim=64, amplitude=math.nan)])
def test_rope_refusals(rope):
    _refused(atp.EINVAL, "rope", _append, rope=atp.Rope(**rope))


def test_row_refusals():
    for f, names in ((_append, "qkvo"), (_attend, "qo")):
        for n in names:
            _refused(atp.EINVAL, "NULL", f, **{n: 0})
            _refused(atp.EALIGN, "16-byte", f, **{n: _addr(10) + 8})
            _refused(atp.EINVAL, "stride", f, **{n + "s": 64})
            _refused(atp.EALIGN, "16-byte", f, **{n + "s": 324})
    _refused(atp.EINVAL, "overlaps an input", _append, o=_addr(10), os=328)       # q_out in q's place at another stride
    _refused(atp.EINVAL, "overlaps an input", _append, o=_addr(11))
    _refused(atp.EINVAL, "arena overlaps", _append, k=_addr(0) + 256)
    _refused(atp.EINVAL, "overlaps the arena", _append, o=_addr(0) + 256)
    _refused(atp.EINVAL, "out overlaps q", _attend, o=_addr(10))
    _refused(atp.EINVAL, "out overlaps q", _attend, o=_addr(10) + 16 * 39, os=640, qs=640)
    _refused(atp.EINVAL, "arena", _attend, o=_addr(0))
    _refused(atp.EINVAL, "lse overlaps", _attend, lse=_addr(10))
    _refused(atp.EALIGN, "lse", _attend, lse=_addr(14) + 2)


def test_append_refuses_more_rows_than_a_launch_takes():
    _refused(atp.EINVAL, "2^26", _append, s=_step(max_tokens=1 << 26))


def test_attend_mask_and_bound_refusals():
    _refused(atp.EINVAL, "scale", _attend, mask=atp.Mask(math.nan))
    for cap in (-1.0, 1e-7, math.inf, math.nan):
        _refused(atp.EINVAL, "softcap", _attend, mask=atp.Mask(1.0, softcap=cap))
    _refused(atp.EINVAL, "window", _attend, mask=atp.Mask(1.0, window=-1))
    _refused(atp.EINVAL, "max_ctx", _attend, s=_step(max_ctx=1))
    _refused(atp.EINVAL, "negative bound", _attend, s=_step(max_fresh=-1))
    _refused(atp.EINVAL, "2^30", _attend, s=_step(max_ctx=(1 << 30) + 1))
    _refused(atp.EINVAL, "int32", _attend, s=_step(max_tokens=1 << 29))
    # HIP counts a launch's threads in 32 bits
    _refused(atp.EINVAL, "one launch", _attend, s=_step(n_seq=1 << 23, max_blocks=1, max_fresh=1, max_ctx=16, max_tokens=8))


def test_attend_workspace_refusals():
    # one long session: its length is split, so a workspace is needed
    s = _step(n_seq=1, max_blocks=8192, max_tokens=1, max_fresh=1, max_ctx=131072)
    n = atp.kv_attend_workspace(_cache(), s)
    assert n > 0
    _refused(atp.ECAPACITY, "workspace", _attend, s=s, ws_bytes=n - 1)
    _refused(atp.EINVAL, "workspace", _attend, s=s, ws=0)
    _refused(atp.EALIGN, "workspace", _attend, s=s, ws=_addr(9) + 64)
    for other in (_addr(10), _addr(13), _addr(14), _addr(0)):
        _refused(atp.EINVAL, "workspace overlaps", _attend, s=s, ws=other)


def test_null_descriptions_are_refused():
    L, n, cache, step = atp.lib, C.c_uint64(), _cache(), _step()
    for c, s in ((None, step.ref), (cache.ref, None)):
        assert L.atp_kv_extend(c, s, None, None, 0, None) == atp.EINVAL
        assert L.atp_kv_append(c, s, 0, None, *[None, 0] * 4, None) == atp.EINVAL
        assert L.atp_kv_attend(c, s, 0, None, *[None, 0] * 2, None, None, 0, None) == atp.EINVAL
        assert L.atp_kv_extend_workspace(c, s, C.byref(n)) == atp.EINVAL
        assert L.atp_kv_attend_workspace(c, s, C.byref(n)) == atp.EINVAL
    assert L.atp_kv_extend_workspace(cache.ref, step.ref, None) == atp.EINVAL
    assert L.atp_kv_attend_workspace(cache.ref, step.ref, None) == atp.EINVAL
    _refused(atp.EINVAL, "mask is NULL", lambda: atp._check(
        L.atp_kv_attend(cache.ref, step.ref, 0, None, _addr(10), 320, _addr(13), 320, None, None, 0, None)))


def test_nothing_to_do_is_ok_without_a_gpu():
    _append(s=_step(max_tokens=0))
    _append(_cache(q_heads=(0, 0), kv_heads=(0, 0), arena=0))
    for kw in (dict(n_seq=0), dict(max_tokens=0), dict(max_fresh=0)):
        _attend(s=_step(**kw))
    _attend(_cache(q_heads=(4, 4), kv_heads=(0, 2)))


# ---- buffers that a kernel reads while another argument writes them ------------------


@pytest.mark.parametrize("read", ["block_table", "cached", "starts", "slopes", "scales"])
def test_attend_refuses_outputs_over_what_it_reads(read):
    at = _addr(20)
    s = dict(n_seq=1, max_blocks=8192, max_tokens=1, max_fresh=1, max_ctx=131072)  # a workspace is needed
    s, c, m = _step(**s, **({read: at} if read in ("block_table", "cached", "starts") else {})), _cache(), atp.Mask(0.125)
    if read == "slopes":
        m = atp.Mask(0.125, slopes=at)
    elif read == "scales":
        c = _cache(cache_dtype=atp.E4M3, scales=at)
    for kw in (dict(o=at), dict(lse=at), dict(ws=at)):
        _refused(atp.EINVAL, "overlaps", _attend, c, s, mask=m, **kw)
    # the last word that the call reads and the first behind it
    words = {"block_table": 8192, "cached": 1, "starts": 2, "slopes": 5, "scales": 8}[read]
    s.d.status = at + 4 * (words - 1)
    _refused(atp.EINVAL, "status overlaps", _attend, c, s, mask=m)
    s.d.status = at + 4 * words
    _refused(atp.EINVAL, "workspace overlaps", _attend, c, s, mask=m, ws=_addr(0))  # gets past the status


@pytest.mark.parametrize("read", ["slots", "positions", "scales"])
def test_append_refuses_outputs_over_what_it_reads(read):
    at = _addr(20)
    c = _cache(cache_dtype=atp.E4M3, scales=at) if read == "scales" else _cache()
    s = _step(**({} if read == "scales" else {read: at}))
    _refused(atp.EINVAL, "overlaps", _append, c, s, o=at)
    c.d.arena = at  # the cache is written too
    _refused(atp.EINVAL, "overlaps", _append, c, s)
    c.d.arena = _addr(0)
    words = {"slots": 16, "positions": 8, "scales": 8}[read]
    s.d.status = at + 4 * (words - 1)
    _refused(atp.EINVAL, "status overlaps", _append, c, s)
    s.d.status = at + 4 * words
    _refused(atp.EINVAL, "q_out overlaps the arena", _append, c, s, o=_addr(0) + 256)


def test_status_apart_from_the_rows_and_the_cache():
    for f, kw in ((_append, dict(o=_addr(13))), (_attend, dict(o=_addr(13)))):
        for at in (_addr(13) + 4, _addr(10) + 4, _addr(0) + 4):
            _refused(atp.EINVAL, "status overlaps", f, s=_step(status=at), **kw)
    for at in (_addr(14), _addr(9)):
        s = _step(n_seq=1, max_blocks=8192, max_tokens=1, max_fresh=1, max_ctx=131072, status=at)
        _refused(atp.EINVAL, "status overlaps", _attend, s=s)


def test_append_takes_rows_up_to_a_launch_of_32_bits_of_threads():
    """4 rows a workgroup of 256 threads: 2^24 - 1 workgroups are the most."""
    for rows in ((1 << 26) - 3, (1 << 26) - 1):
        _refused(atp.EINVAL, "2^26", _append, s=_step(max_tokens=rows))
    _refused(atp.EINVAL, "q is NULL", _append, s=_step(max_tokens=(1 << 26) - 4), q=0)  # gets past that check
