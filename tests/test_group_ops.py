"""The operators for sequences that share a beginning without a GPU: sizes and
refusals.  Every call here fails its host checks or is host code: nothing is
enqueued."""
import ctypes as C

import pytest

from paper_2608_14376_amd import corun
from tests.test_cache_ops import P, _i32, _kv


def beam(logits=P, ld=1024, vocab=1000, groups=2, beams=4, scores=P, valid=None, finished=None, weights=None, end=-1,
         keep=8, tokens=P, parents=P, out=P, fin=None, ws=P, ws_bytes=1 << 40):
    return corun.load().corun_beam_select(logits, ld, vocab, groups, beams, scores, valid, finished, weights, end, keep,
                                          tokens, parents, out, fin, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(logits=None), corun.E_INVAL), (dict(scores=None), corun.E_INVAL), (dict(tokens=None), corun.E_INVAL),
    (dict(parents=None), corun.E_INVAL), (dict(out=None), corun.E_INVAL), (dict(logits=P + 2), corun.E_INVAL),
    (dict(ld=999), corun.E_SHAPE), (dict(vocab=0), corun.E_SHAPE), (dict(vocab=(1 << 19) + 1, ld=1 << 20), corun.E_SHAPE),
    (dict(groups=0), corun.E_SHAPE), (dict(groups=16384), corun.E_SHAPE), (dict(beams=0), corun.E_SHAPE),
    (dict(beams=65), corun.E_SHAPE), (dict(keep=0), corun.E_SHAPE), (dict(keep=65), corun.E_SHAPE),
    (dict(end=-2), corun.E_INVAL), (dict(end=1000), corun.E_INVAL), (dict(finished=P), corun.E_INVAL),
    (dict(ws=None), corun.E_INVAL), (dict(ws=P + 4), corun.E_INVAL), (dict(ws_bytes=3), corun.E_CAPACITY),
])
def test_beam_refusals(kw, status):
    assert beam(**kw) == status
    assert corun.last_error()


def test_beam_workspace():
    size = corun.beam_select_workspace
    assert 0 < size(1, 1, 1, 1) <= size(151936, 1, 4, 8) <= size(151936, 64, 4, 8)
    for bad in ((0, 1, 1, 1), (10, 0, 1, 1), (10, 1, 0, 1), (10, 1, 1, 0), (10, 1, 65, 1), (10, 65536, 1, 1)):
        with pytest.raises(corun.CorunError):
            size(*bad)


PAGED = dict(layout=corun.KV_PAGED)


def assign(kv, layers=1, nkv=2, d=128, table=P, held=P, src=P, keep=P, hold=None, status=P, ws=P, ws_bytes=1 << 40):
    return corun.load().corun_pages_assign(C.addressof(kv) if kv else None, layers, nkv, d, table, held, src, keep, hold,
                                           status, ws, ws_bytes, None)


def compact(kv, layers=1, nkv=2, d=128, table=P, held=P, status=P, ws=P, ws_bytes=1 << 40):
    return corun.load().corun_pages_compact(C.addressof(kv) if kv else None, layers, nkv, d, table, held, status, ws,
                                            ws_bytes, None)


@pytest.mark.parametrize("kv,kw,status", [
    (dict(layout=corun.KV_CONTIGUOUS), {}, corun.E_INVAL), (dict(page_size=24), {}, corun.E_CAPACITY),
    (dict(blk=64), {}, corun.E_SHAPE), (dict(n_slots=0), {}, corun.E_CAPACITY), (dict(dtype=2), {}, corun.E_INVAL),
    (dict(num_pages=(1 << 20) + 1), {}, corun.E_SHAPE), (dict(n_slots=1 << 19, mpp=1 << 10), {}, corun.E_SHAPE),
    (dict(page_size=1 << 21), {}, corun.E_SHAPE), (dict(ptr=None), {}, corun.E_INVAL), (dict(ptr=P + 8), {}, corun.E_INVAL),
    (dict(scales=None), {}, corun.E_INVAL), (dict(table=None), dict(table=None), corun.E_INVAL),
    ({}, dict(table=P + 64), corun.E_INVAL), ({}, dict(table=None), corun.E_INVAL), ({}, dict(held=None), corun.E_INVAL),
    ({}, dict(status=None), corun.E_INVAL), ({}, dict(layers=0), corun.E_INVAL), ({}, dict(d=96), corun.E_SHAPE),
    ({}, dict(nkv=0), corun.E_SHAPE), (dict(page_size=1 << 20), dict(nkv=512), corun.E_SHAPE), ({}, dict(ws=None), corun.E_INVAL), ({}, dict(ws=P + 8), corun.E_INVAL),
    ({}, dict(ws_bytes=16), corun.E_CAPACITY),
])
def test_pages_refusals(kv, kw, status):
    kv = _kv(**{**PAGED, **kv})
    assert assign(kv, **kw) == status and corun.last_error()
    assert compact(kv, **kw) == status


def test_pages_null_arguments():
    assert assign(None) == compact(None) == corun.E_INVAL
    assert assign(_kv(**PAGED), src=None) == assign(_kv(**PAGED), keep=None) == corun.E_INVAL
    assert corun.load().corun_pages_workspace(None) == corun.E_INVAL
    assert corun.load().corun_pages_workspace(C.addressof(_kv(**PAGED))) > 0


def shared(kv, layer=0, nq=8, nkv=2, d=128, groups=(2, 1), n=None, q=P, ldq=1024, lens=P, slots=None, prefix=P, most=(0, 0),
           out=P, ldo=1024, ws=P, ws_bytes=1 << 40):
    return corun.load().corun_shared_attention(C.addressof(kv) if kv else None, layer, nq, nkv, d,
                                               len(groups) if n is None else n, _i32(*groups) if groups else None, q, ldq,
                                               None, lens, slots, prefix, *most, out, ldo, ws, ws_bytes, None)


@pytest.mark.parametrize("dtype", [corun.KV_BF16, corun.KV_E4M3])
@pytest.mark.parametrize("kw,status", [
    (dict(nq=9), corun.E_SHAPE), (dict(nq=34), corun.E_SHAPE), (dict(nq=0), corun.E_SHAPE), (dict(d=96), corun.E_SHAPE),
    (dict(groups=(2, 0)), corun.E_INVAL), (dict(groups=(2, -1)), corun.E_INVAL), (dict(groups=()), corun.E_INVAL),
    (dict(n=0), corun.E_INVAL), (dict(groups=(1,) * 257), corun.E_INVAL), (dict(groups=(3, 2)), corun.E_CAPACITY),
    (dict(groups=(2**31 - 1, 2**31 - 1)), corun.E_SHAPE), (dict(layer=-1), corun.E_INVAL),
    (dict(most=(257, 0)), corun.E_CAPACITY), (dict(most=(0, 257)), corun.E_CAPACITY), (dict(most=(-1, 0)), corun.E_CAPACITY),
    (dict(q=None), corun.E_INVAL), (dict(q=P + 8), corun.E_INVAL), (dict(ldq=1020), corun.E_INVAL),
    (dict(ldq=1016), corun.E_SHAPE), (dict(out=None), corun.E_INVAL), (dict(ldo=1016), corun.E_SHAPE),
    (dict(lens=None), corun.E_INVAL), (dict(prefix=None), corun.E_INVAL),
])
def test_shared_attention_refusals(dtype, kw, status):
    assert shared(_kv(dtype=dtype), **kw) == status and corun.last_error()


def test_shared_attention_refuses_too_many_workgroups():
    kv = _kv(n_slots=60000, max_seq_len=1024)
    rows = (60000,)
    assert shared(kv, nq=4096, nkv=4096, d=64, groups=rows, ldq=1 << 18, ldo=1 << 18) == corun.E_SHAPE
    assert corun.load().corun_shared_attention_workspace(C.addressof(kv), 4096, 4096, 64, 1, _i32(*rows), 0, 0) == corun.E_SHAPE


def test_shared_attention_refuses_caches():
    assert shared(None) == corun.E_INVAL
    assert shared(_kv(ptr=None)) == shared(_kv(scales=None)) == shared(_kv(layout=3)) == corun.E_INVAL
    assert shared(_kv(**PAGED, table=None)) == corun.E_INVAL


@pytest.mark.parametrize("dtype", [corun.KV_BF16, corun.KV_E4M3])
def test_shared_attention_workspace(dtype):
    L, rows = corun.load(), _i32(3, 1)
    kv = _kv(dtype=dtype, max_seq_len=65536, n_slots=4)
    size = lambda a, b, g=rows, n=2: L.corun_shared_attention_workspace(C.addressof(kv), 8, 2, 128, n, g, a, b)
    assert 0 <= size(64, 64) <= size(65536, 64) <= size(0, 0)
    assert size(0, 0, None) == corun.E_INVAL and size(0, 0, rows, 0) == corun.E_INVAL
    need = size(0, 0)
    if need:
        assert shared(kv, groups=(3, 1), ws_bytes=need - 1) == corun.E_CAPACITY
        assert shared(kv, groups=(3, 1), ws=P + 4) == shared(kv, groups=(3, 1), ws=None) == corun.E_INVAL
