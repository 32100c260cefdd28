"""The cache operators without a GPU: frequencies, shapes and refusals.  Every
call here fails its host checks or is host code: nothing is enqueued."""
import ctypes as C
import math

import pytest

from paper_2608_14376_amd import corun
from tests import cache_reference as ref

P = 1 << 20   # a pointer on a 16-byte boundary that no refused call looks at


def _kv(layout=corun.KV_CONTIGUOUS, n_slots=4, max_seq_len=256, page_size=32, num_pages=64, mpp=8, dtype=corun.KV_E4M3,
        blk=32, ptr=P, scales=P, table=P):
    one = lambda p: C.cast((C.c_void_p * 1)(p), corun._PP)
    kv = corun.KV(layout, n_slots, max_seq_len, page_size, num_pages, mpp, one(ptr), one(ptr), table, dtype, blk,
                  one(scales), one(scales))
    return kv


def _rope(**kw):
    return corun.rope(**{"head_dim": 128, **kw})


def _i32(*v):
    return (C.c_int32 * len(v))(*v)


def decode_append(kv, rope, layer=0, nq=8, nkv=2, rows=2, qkv=P, ld=1536, valid=None, pos=P, q=P, ldq=1024):
    return corun.load().corun_decode_append(C.addressof(kv) if kv else None, layer, nq, nkv,
                                            C.addressof(rope) if rope else None, rows, qkv, ld, valid, pos, q, ldq, None)


def prefill_append(kv, rope, n=2, lens=(3, 4), starts=(0, 5), slots=(0, 1), nq=8, nkv=2, qkv=P, ld=1536, q=P, ldq=1024):
    return corun.load().corun_prefill_append(C.addressof(kv), 0, nq, nkv, C.addressof(rope), n,
                                             _i32(*lens) if lens else None, _i32(*starts) if starts else None,
                                             _i32(*slots) if slots else None, qkv, ld, q, ldq, None)


def decode_attention(kv, nq=8, nkv=2, d=128, rows=2, q=P, ldq=1024, lens=P, max_len=0, out=P, ldo=1024, ws=P, ws_bytes=1 << 40,
                     layer=0):
    return corun.load().corun_decode_attention(C.addressof(kv), layer, nq, nkv, d, rows, q, ldq, None, lens, max_len, out,
                                               ldo, ws, ws_bytes, None)


def prefill_attention(kv, n=2, lens=(3, 4), starts=(0, 5), slots=(0, 1), nq=8, nkv=2, d=128, q=P, ldq=1024, out=P, ldo=1024,
                      ws=P, ws_bytes=1 << 40):
    return corun.load().corun_prefill_attention(C.addressof(kv), 0, nq, nkv, d, n, _i32(*lens), _i32(*starts),
                                                _i32(*slots), q, ldq, out, ldo, ws, ws_bytes, None)


@pytest.mark.parametrize("kw", [
    dict(theta=1e6),
    dict(theta=1e4, rot_dim=64, layout=corun.ROPE_INTERLEAVED),
    dict(theta=1e4, rot_dim=6),
    dict(theta=1e6, scaling=corun.ROPE_LINEAR, factor=4.0),
    dict(theta=5e5, scaling=corun.ROPE_BANDS, factor=8.0, low=1.0, high=4.0, trained_len=8192),
    dict(theta=1e4, scaling=corun.ROPE_BANDS, factor=16.0, low=1.0, high=32.0, trained_len=4096, magnitude=1.2),
])
def test_rope_frequencies(kw):
    r = _rope(**kw)
    rot = kw.get("rot_dim", 128)
    name = {0: "none", 1: "linear", 2: "bands"}[kw.get("scaling", 0)]
    want = ref.freqs(kw["theta"], rot, name, kw.get("factor", 1.0), kw.get("low", 0.0), kw.get("high", 0.0),
                     kw.get("trained_len", 0))
    assert r.rot_dim == rot and r.head_dim == 128
    assert math.isclose(r.magnitude, kw.get("magnitude", 1.0), rel_tol=1e-7)
    for i, f in enumerate(want):
        assert math.isclose(r.freq[i], f, rel_tol=1e-13), i
    assert all(f == 0.0 for f in list(r.freq)[rot // 2:])


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), corun.E_SHAPE), (dict(rot_dim=7), corun.E_SHAPE), (dict(rot_dim=130), corun.E_SHAPE),
    (dict(rot_dim=-2), corun.E_SHAPE), (dict(layout=2), corun.E_INVAL), (dict(scaling=3), corun.E_INVAL),
    (dict(theta=1.0), corun.E_INVAL), (dict(theta=math.nan), corun.E_INVAL), (dict(theta=math.inf), corun.E_INVAL),
    (dict(scaling=1, factor=0.5), corun.E_INVAL), (dict(scaling=1, factor=math.nan), corun.E_INVAL),
    (dict(scaling=2, factor=2.0, low=1.0, high=1.0, trained_len=10), corun.E_INVAL),
    (dict(scaling=2, factor=2.0, low=-1.0, high=1.0, trained_len=10), corun.E_INVAL),
    (dict(scaling=2, factor=2.0, low=1.0, high=4.0, trained_len=0), corun.E_INVAL),
    (dict(magnitude=-1.0), corun.E_INVAL), (dict(magnitude=math.nan), corun.E_INVAL),
])
def test_rope_refusals(kw, status):
    with pytest.raises(corun.CorunError) as e:
        _rope(**kw)
    assert e.value.status == status and corun.last_error()


CACHES = [
    (dict(layout=3), corun.E_INVAL), (dict(max_seq_len=0), corun.E_CAPACITY), (dict(max_seq_len=40), corun.E_CAPACITY),
    (dict(dtype=2), corun.E_INVAL), (dict(blk=8), corun.E_SHAPE), (dict(blk=48), corun.E_SHAPE),
    (dict(blk=128), corun.E_SHAPE), (dict(blk=64, max_seq_len=96), corun.E_SHAPE), (dict(n_slots=0), corun.E_CAPACITY),
    (dict(layout=corun.KV_PAGED, page_size=24), corun.E_CAPACITY), (dict(layout=corun.KV_PAGED, page_size=48), corun.E_SHAPE),
    (dict(layout=corun.KV_PAGED, num_pages=0), corun.E_CAPACITY), (dict(layout=corun.KV_PAGED, mpp=0), corun.E_CAPACITY),
    (dict(layout=corun.KV_PAGED, page_size=1 << 21), corun.E_SHAPE), (dict(layout=corun.KV_PAGED, table=None), corun.E_INVAL),
    (dict(ptr=None), corun.E_INVAL), (dict(ptr=P + 8), corun.E_INVAL), (dict(scales=None), corun.E_INVAL),
]


@pytest.mark.parametrize("kw,status", CACHES)
def test_cache_refusals(kw, status):
    kv, rope = _kv(**kw), _rope()
    for st in (decode_append(kv, rope), prefill_append(kv, rope), decode_attention(kv), prefill_attention(kv)):
        assert st == status, corun.last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(rope=None), corun.E_INVAL), (dict(kv=None), corun.E_INVAL), (dict(layer=-1), corun.E_INVAL),
    (dict(nq=7), corun.E_SHAPE), (dict(nq=34, ld=38 * 128, ldq=34 * 128), corun.E_SHAPE), (dict(nkv=0), corun.E_SHAPE),
    (dict(rows=0), corun.E_SHAPE), (dict(rows=5), corun.E_CAPACITY), (dict(qkv=None), corun.E_INVAL),
    (dict(qkv=P + 2), corun.E_INVAL), (dict(ld=1528), corun.E_SHAPE), (dict(ld=1540), corun.E_INVAL),
    (dict(q=None), corun.E_INVAL), (dict(q=P + 4), corun.E_INVAL), (dict(ldq=1016), corun.E_SHAPE), (dict(pos=None), corun.E_INVAL),
])
def test_decode_append_refusals(kw, status):
    kw = dict(kw)
    kv = kw.pop("kv") if "kv" in kw else _kv()
    rope = kw.pop("rope") if "rope" in kw else _rope()
    assert decode_append(kv, rope, **kw) == status, corun.last_error()


def test_a_filled_in_rope_is_checked():
    for change, status in (("rot_dim", corun.E_SHAPE), ("layout", corun.E_INVAL), ("head_dim", corun.E_SHAPE)):
        r = _rope()
        setattr(r, change, 999)
        assert decode_append(_kv(), r) == status
    r = _rope()
    r.freq[3] = math.nan
    assert decode_append(_kv(), r) == corun.E_INVAL
    r = _rope()
    r.magnitude = math.inf
    assert prefill_append(_kv(), r) == corun.E_INVAL


SEQS = [
    (dict(n=0), corun.E_INVAL), (dict(n=65, lens=[1] * 65, starts=[0] * 65, slots=list(range(65))), corun.E_INVAL),
    (dict(lens=(3, 0)), corun.E_INVAL), (dict(starts=(0, -1)), corun.E_INVAL), (dict(slots=(0, 4)), corun.E_INVAL),
    (dict(slots=(-1, 0)), corun.E_INVAL), (dict(slots=(1, 1)), corun.E_INVAL), (dict(lens=(3, 252)), corun.E_CAPACITY),
    (dict(starts=(2**31 - 1, 0)), corun.E_CAPACITY),
]


@pytest.mark.parametrize("kw,status", SEQS)
def test_sequence_refusals(kw, status):
    assert prefill_append(_kv(), _rope(), **kw) == status, corun.last_error()
    assert prefill_attention(_kv(), **kw) == status, corun.last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(d=96), corun.E_SHAPE), (dict(nq=9), corun.E_SHAPE), (dict(rows=5), corun.E_CAPACITY), (dict(lens=None), corun.E_INVAL),
    (dict(max_len=-1), corun.E_CAPACITY), (dict(max_len=257), corun.E_CAPACITY), (dict(q=P + 8), corun.E_INVAL),
    (dict(out=None), corun.E_INVAL), (dict(ldo=1000), corun.E_SHAPE), (dict(layer=-2), corun.E_INVAL),
])
def test_decode_attention_refusals(kw, status):
    assert decode_attention(_kv(), **kw) == status, corun.last_error()


def test_attention_reads_8_bit_caches_only():
    kv = _kv(dtype=corun.KV_BF16)
    assert decode_attention(kv) == corun.E_INVAL and prefill_attention(kv) == corun.E_INVAL


def test_workspace_is_checked():
    kv = _kv(max_seq_len=4096, n_slots=64)
    L = corun.load()
    need = L.corun_decode_attention_workspace(C.addressof(kv), 8, 2, 128, 64, 0)
    assert need >= 0
    assert L.corun_decode_attention_workspace(C.addressof(kv), 8, 2, 128, 65, 0) == corun.E_CAPACITY
    if need:
        assert decode_attention(kv, rows=64, ws_bytes=need - 1) == corun.E_CAPACITY
        assert decode_attention(kv, rows=64, ws=None) == corun.E_INVAL
        assert decode_attention(kv, rows=64, ws=P + 8) == corun.E_INVAL


def test_launch_limits_refused():
    kv = _kv(n_slots=65535)
    assert decode_append(kv, _rope(), nq=4096, nkv=4096, rows=65535, ld=3 * 4096 * 128, ldq=4096 * 128) == corun.E_SHAPE
    kv = _kv(n_slots=16, max_seq_len=1 << 20)
    args = dict(n=16, lens=[1 << 20] * 16, starts=[0] * 16, slots=range(16))
    assert prefill_attention(kv, nq=128, nkv=8, ldq=128 * 128, ldo=128 * 128, **args) == corun.E_SHAPE
    args["lens"][0] += 16
    assert prefill_attention(_kv(n_slots=16, max_seq_len=1 << 21), **args) == corun.E_SHAPE      # over 2^24 rows


def prefill_workspace(kv, lens, starts=None, nq=8, nkv=2, d=128):
    return corun.load().corun_prefill_attention_workspace(C.addressof(kv), nq, nkv, d, len(lens), _i32(*lens),
                                                          _i32(*starts) if starts else None)


def test_prefill_workspace_and_its_refusals():
    kv = _kv(max_seq_len=1 << 14)
    unit = 4 * (32 * 128 + 64)                        # a split's rows of a head, their maxima and sums
    # 33 rows behind 4000 tokens: two blocks of rows, four workgroups, 64 tiles: eight splits of eight
    assert prefill_workspace(kv, [33], [4000]) == 8 * 2 * 8 * unit
    assert prefill_workspace(kv, [33], [4000], d=64) == 8 * 2 * 8 * 4 * (32 * 64 + 64)
    assert prefill_workspace(kv, [33, 5, 33], [4000, 0, 4000]) == 16 * 2 * 8 * unit
    assert prefill_workspace(kv, [900]) == 0          # 15 tiles
    assert prefill_workspace(kv, [2049], [8000]) == 3 * 65 * 8 * unit   # 130 workgroups, 158 tiles
    assert prefill_workspace(kv, [2049], [1900]) == 0
    assert prefill_workspace(kv, [4100], [8000]) == 0  # 129 blocks of rows: 258 workgroups
    assert prefill_workspace(kv, [0]) == corun.E_INVAL
    assert prefill_workspace(kv, [1], [1 << 14]) == corun.E_CAPACITY
    assert prefill_workspace(kv, [1], nq=9) == corun.E_SHAPE
    args = dict(n=1, lens=[33], starts=[4000], slots=[1])
    need = prefill_workspace(kv, [33], [4000])
    assert prefill_attention(kv, ws=None, **args) == corun.E_INVAL
    assert prefill_attention(kv, ws=P + 8, **args) == corun.E_INVAL
    assert prefill_attention(kv, ws_bytes=need - 1, **args) == corun.E_CAPACITY
    assert prefill_attention(kv, ws=None, ws_bytes=0, **args) == corun.E_INVAL
    assert prefill_attention(kv, ws=None, ws_bytes=-1, n=1, lens=[3], starts=[0], slots=[0]) == corun.E_CAPACITY


def test_engine_chunks_that_make_too_many_splits():
    cfg = corun.model_cfg(dict(n_layers=1, hidden=256, n_heads=4, n_kv_heads=2, head_dim=64, ffn=688, vocab=1024, n_experts=0,
                               top_k=0, expert_ffn=0, rms_eps=1e-6, rope_theta=10000.0))
    out = (C.c_int32 * 64)()
    for chunk, ok in ((64, False), (128, True), (0, True)):
        kv, opt = _kv(max_seq_len=2048 * 64), corun.options(attn_chunk=chunk)
        n = corun.load().corun_describe_plan(C.byref(cfg), C.byref(kv), 2, C.byref(opt), C.addressof(out), 64)
        assert n > 0 if ok else n == corun.E_INVAL
    kv, opt = _kv(max_seq_len=2048 * 64, dtype=corun.KV_BF16), corun.options(attn_chunk=64)
    assert corun.load().corun_describe_plan(C.byref(cfg), C.byref(kv), 2, C.byref(opt), C.addressof(out), 64) > 0


def test_engine_chunks_count_a_capacity_s_last_split():
    """A capacity that is no multiple of the chunk has a further, shorter split."""
    cfg = corun.model_cfg(dict(n_layers=1, hidden=256, n_heads=4, n_kv_heads=2, head_dim=64, ffn=688, vocab=1024, n_experts=0,
                               top_k=0, expert_ffn=0, rms_eps=1e-6, rope_theta=10000.0))
    out, opt = (C.c_int32 * 64)(), corun.options(attn_chunk=64)
    for cap, ok in ((2047 * 64, True), (2047 * 64 + 16, False), (2046 * 64 + 16, True)):
        for kv in (_kv(max_seq_len=cap, blk=16), _kv(layout=corun.KV_PAGED, page_size=16, mpp=cap // 16, blk=16)):
            n = corun.load().corun_describe_plan(C.byref(cfg), C.byref(kv), 2, C.byref(opt), C.addressof(out), 64)
            assert n > 0 if ok else n == corun.E_INVAL, (cap, n)
