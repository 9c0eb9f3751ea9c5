"""The cache's and the rotation's C entry points refuse what they cannot do before they touch a device (no GPU needed)."""
import ctypes as C

import pytest

from paper_2503_14153_b200 import cache as pc


@pytest.fixture(scope="module")
def lib():
    from paper_2503_14153_b200 import build
    build.build()
    return pc._library()[0]


def _cache(**kw):
    v = dict(n_layers=2, n_kv_heads=4, head_dim=64, n_pages=8, max_seqs=2, pages_per_seq=4, format=0, codes=4096, scales=4096, page_table=4096, refs=4096, lens=4096, status=4096)
    v.update(kw)
    return pc._Cache(**v)


def _call(f, c, a, *rest):
    return f(C.addressof(c) if c is not None else None, C.addressof(a) if a is not None else None, *rest)


@pytest.mark.parametrize("kw", [dict(head_dim=96), dict(head_dim=0), dict(format=2), dict(n_pages=0), dict(n_layers=-1), dict(codes=None), dict(codes=4100), dict(lens=None), dict(status=None),
                                dict(n_pages=1 << 28), dict(pages_per_seq=1 << 27)])
def test_bad_caches(lib, kw):
    c = _cache(**kw)
    assert lib.spec_cache_scratch_bytes(C.addressof(c)) == 0
    assert lib.spec_cache_attention_scratch(C.addressof(c), 4, 1, 1) == 0
    a = pc._AttentionArgs(q=16, k=16, v=16, out=16, type=1, rows=1, batch=1, n_heads=4, max_rows=1)
    assert _call(lib.spec_cache_attention, c, a, 16, 1 << 30, None) == -1
    assert lib.spec_cache_fork(C.addressof(c), 1, 16, 16, None) == -1
    assert lib.spec_cache_truncate(C.addressof(c), 1, None, None, None) == -1
    assert lib.spec_last_error(None)


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(type=3), dict(rows=-1), dict(batch=3), dict(batch=-1), dict(n_heads=6), dict(n_heads=0), dict(layer=2), dict(layer=-1),
                                dict(max_rows=0), dict(max_rows=1), dict(mask=16, mask_words=0), dict(batch=70000, rows=70000), dict(q=4104), dict(q_row_stride=4), dict(k_head_stride=3), dict(v=8),
                                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_bad_attention(lib, kw):
    ren = {"q_row_stride": "q_row", "k_head_stride": "k_head"}
    v = dict(q=4096, k=4096, v=4096, out=4096, type=1, rows=4, batch=2, n_heads=8, layer=0, max_rows=2, q_row=512, q_head=64, k_row=256, k_head=64, v_row=256, v_head=64, scale=0.1)
    v.update({ren.get(k, k): x for k, x in kw.items()})
    c = _cache()
    assert _call(lib.spec_cache_attention, c, pc._AttentionArgs(**v), 4096, 1 << 40, None) == -1, kw
    assert b"spec_cache_attention" in lib.spec_last_error(None)


def test_scratch_that_is_too_small(lib):
    c = _cache()
    a = pc._AttentionArgs(q=4096, k=4096, v=4096, out=4096, type=1, rows=4, batch=2, n_heads=8, max_rows=2, q_row=512, q_head=64, k_row=256, k_head=64, v_row=256, v_head=64, scale=0.1)
    need = lib.spec_cache_attention_scratch(C.addressof(c), 8, 2, 2)
    assert need > 0 and _call(lib.spec_cache_attention, c, a, 4096, need - 1, None) == -3
    assert _call(lib.spec_cache_attention, c, a, None, need, None) == -3
    assert _call(lib.spec_cache_attention, c, a, 4100, need, None) == -3
    n = lib.spec_cache_scratch_bytes(C.addressof(c))
    assert lib.spec_cache_reserve(C.addressof(c), 1, None, 4096, 4096, 4096, n - 1, None) == -3
    assert lib.spec_cache_compact(C.addressof(c), 4096, None, n, None) == -3


@pytest.mark.parametrize("kw", [dict(k=None), dict(counts=None), dict(type=7), dict(rows=5), dict(layers=3), dict(layer0=1), dict(layer0=-1), dict(max_count=-1), dict(k=4100), dict(k_row=4), dict(v_layer=3)])
def test_bad_store(lib, kw):
    v = dict(k=4096, v=4096, counts=4096, type=1, rows=4, batch=2, layer0=0, layers=2, max_count=2, k_layer=1024, k_row=256, k_head=64, v_layer=1024, v_row=256, v_head=64)
    v.update(kw)
    assert _call(lib.spec_cache_store, _cache(), pc._StoreArgs(**v), None) == -1, kw


@pytest.mark.parametrize("kw", [dict(k=None), dict(type=-1), dict(layers=3), dict(window=-1), dict(batch=-2), dict(v=4104)])
def test_bad_read(lib, kw):
    v = dict(k=4096, v=4096, type=1, batch=2, window=16, layer0=0, layers=2)
    v.update(kw)
    assert _call(lib.spec_cache_read, _cache(), pc._ReadArgs(**v), None) == -1, kw


@pytest.mark.parametrize("kw", [dict(q=None), dict(v_out=None), dict(table=None), dict(rot_dim=7), dict(rot_dim=66), dict(rot_dim=0), dict(head_dim=63), dict(in_type=3), dict(out_type=-1), dict(rows=-1), dict(span=0)])
def test_bad_rotary(lib, kw):
    v = dict(q=4096, k=4096, v=4096, q_out=4096, k_out=4096, v_out=4096, positions=4096, table=4096, in_type=0, out_type=1, rows=2, n_heads=4, n_kv_heads=2, n_v_heads=2, head_dim=64, rot_dim=64, span=10)
    v.update(kw)
    assert lib.spec_rotary(C.addressof(pc._RotaryArgs(**v)), None) == -1, kw
    assert lib.spec_rotary_table(4096, None, 4, 4, 1.0, None) == -1 and lib.spec_rotary_table(4096, 4096, 0, 4, 1.0, None) == -1


def test_null_arguments_and_empty_calls(lib):
    c = _cache()
    for f, rest in ((lib.spec_cache_attention, (4096, 1 << 30, None)), (lib.spec_cache_store, (None,)), (lib.spec_cache_read, (None,))):
        assert _call(f, c, None, *rest) == -1 and _call(f, None, pc._AttentionArgs(), *rest) == -1
    assert lib.spec_rotary(None, None) == -1
    assert lib.spec_cache_fork(C.addressof(c), 1, None, 4096, None) == -1 and lib.spec_cache_fork(C.addressof(c), -1, 4096, 4096, None) == -1
    assert lib.spec_cache_reserve(C.addressof(c), 1025, None, 4096, 4096, 4096, 1 << 30, None) == -1
    # nothing to do is no error
    assert _call(lib.spec_cache_attention, c, pc._AttentionArgs(), 4096, 0, None) == 0
    assert _call(lib.spec_cache_store, c, pc._StoreArgs(), None) == 0 and _call(lib.spec_cache_read, c, pc._ReadArgs(), None) == 0
    assert lib.spec_rotary(C.addressof(pc._RotaryArgs()), None) == 0
    for call in (lib.spec_cache_fork(C.addressof(c), 0, None, None, None), lib.spec_cache_truncate(C.addressof(c), 0, None, None, None), lib.spec_cache_reserve(C.addressof(c), 0, None, None, None, None, 0, None)):
        assert call == 0
