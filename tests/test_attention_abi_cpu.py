"""Argument checks of the attention and paged-cache calls on the host: every one returns before a
launch, so none needs a GPU."""
import ctypes as C

import numpy as np
import pytest

import paper_2508_02401_gb300 as ckv
from tests.test_abi_cpu import FakeBatch, _cfg

_P = 0x40000  # a 256-byte-aligned fake device address
_WS = 1 << 40
_NO_GPU = not __import__("torch").cuda.is_available()


@pytest.fixture(scope="module")
def lib():
    from paper_2508_02401_gb300 import build
    build.build()
    return ckv.load()


def _cache(k=_P, v=_P, stride=0, pages=10, page=16):
    return C.byref(ckv._PagedCache(k, v, stride, pages, page))


def _prefill(lib, cfg=None, cu=(0, 100, 300), q=_P, q_tok=0, q_head=0, k=_P, v=_P, tok=0, head=0, out=_P, lse=None,
             lse_st=0, win=None, win_st=0, ws=_P, ws_bytes=_WS):
    cfg = cfg or _cfg()
    return lib.ckv_prefill_attention(cfg.ref, FakeBatch(cu).ref, q, q_tok, q_head, k, v, tok, head, out, lse, lse_st,
                                     win, win_st, ws, ws_bytes, None)


def _paged(lib, cfg=None, cache=None, S=2, T=2, table=_P, blocks=4, lens=_P, cu=_P, q=_P, q_tok=0, q_head=0, out=_P,
           lse=None, lse_st=0, ws=_P, ws_bytes=_WS):
    cfg = cfg or _cfg()
    return lib.ckv_paged_attention(cfg.ref, cache or _cache(), S, T, table, blocks, lens, cu, q, q_tok, q_head, out,
                                   lse, lse_st, ws, ws_bytes, None)


def _tables(lib, page=16, rows=2, lens=_P, new=_P + 64, ring=_P + 128, pages=10, pool=_P + 192, table=_P + 256, blocks=4,
            slots=_P + 320, cap=5, cu=_P + 384, lens_out=_P, pool_out=_P + 192, ws=_P + 1024, ws_bytes=_WS):
    return lib.ckv_block_tables(page, rows, lens, new, ring, pages, pool, table, blocks, slots, cap, cu, lens_out,
                                pool_out, ws, ws_bytes, None)


def _write(lib, cfg=None, cache=None, n=3, k=_P, v=_P, tok=0, head=0, slots=_P, ws=_P, ws_bytes=_WS):
    cfg = cfg or _cfg()
    return lib.ckv_cache_write(cfg.ref, cache or _cache(), n, k, v, tok, head, slots, ws, ws_bytes, None)


def test_workspace_size(lib):
    n = ckv.ckv_attention_workspace_size(_cfg())
    assert n % 4 == 0 and n > 256
    with pytest.raises(ckv.CkvError, match="window"):
        ckv.ckv_attention_workspace_size(_cfg(window=0))
    assert lib.ckv_attention_workspace_size(_cfg().ref, None) == 1
    need = [(_prefill, {}), (_paged, {}), (_tables, {}), (_write, {})]
    for call, kw in need:
        assert call(lib, ws_bytes=n - 1, **kw) == 3
        assert call(lib, ws=_P + 128, **kw) == 3
        assert call(lib, ws=None, **kw) == 3


@pytest.mark.parametrize("kw,expect", [
    (dict(q=None), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(out=None), 1), (dict(q=_P + 8), 1),
    (dict(k=_P + 2), 1), (dict(out=_P + 4), 1), (dict(q_tok=12), 1), (dict(q_head=-8), 1), (dict(tok=-1024), 1),
    (dict(head=4), 1), (dict(tok=1 << 38), 2), (dict(lse=_P + 2), 1), (dict(lse=_P, lse_st=299), 1),
    (dict(win=_P, win_st=63), 1), (dict(lse=_P, lse_st=-5), 1), (dict(cu=(0, 5, 3)), 1), (dict(cu=(1, 5)), 1),
    (dict(cu=(0, 0, 0)), 0),  # nothing to do
])
def test_prefill_attention_arguments(lib, kw, expect):
    assert _prefill(lib, **kw) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(S=0), 1), (dict(T=-1), 1), (dict(blocks=0), 1), (dict(table=None), 1), (dict(lens=None), 1), (dict(cu=None), 1),
    (dict(table=_P + 2), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(q=_P + 8), 1), (dict(q_tok=4), 1),
    (dict(lse=_P, lse_st=1), 1), (dict(blocks=1 << 28), 2), (dict(T=0), 0),
])
def test_paged_attention_arguments(lib, kw, expect):
    assert _paged(lib, **kw) == expect


@pytest.mark.parametrize("cache,expect", [
    (dict(k=None), 1), (dict(v=None), 1), (dict(k=_P + 8), 1), (dict(page=0), 1), (dict(page=24), 2), (dict(page=256), 2),
    (dict(pages=0), 1), (dict(pages=1 << 27), 2), (dict(stride=4), 1), (dict(stride=16 * 8 * 128 - 8), 1),
    (dict(stride=16 * 8 * 128 + 4), 1), (dict(stride=1 << 38), 2),
])
def test_cache_arguments(lib, cache, expect):
    assert _paged(lib, cache=_cache(**cache)) == expect
    assert _write(lib, cache=_cache(**cache)) == expect
    cfg = _cfg()
    assert lib.ckv_paged_attention(cfg.ref, None, 2, 2, _P, 4, _P, _P, _P, 0, 0, _P, None, 0, _P, _WS, None) == 1


@pytest.mark.parametrize("kw,expect", [
    (dict(page=0), 1), (dict(page=48), 2), (dict(rows=0), 1), (dict(pages=0), 1), (dict(blocks=0), 1), (dict(cap=-1), 1),
    (dict(lens=None), 1), (dict(new=None), 1), (dict(ring=None), 1), (dict(pool=None), 1), (dict(table=None), 1),
    (dict(slots=None), 1), (dict(cu=None), 1), (dict(lens_out=None), 1), (dict(pool_out=None), 1),
    (dict(lens=_P + 1), 1), (dict(pool=_P + 4), 1), (dict(slots=_P + 2), 1), (dict(pages=1 << 27), 2),
    (dict(blocks=1 << 27), 2),
])
def test_block_tables_arguments(lib, kw, expect):
    assert _tables(lib, **kw) == expect


@pytest.mark.parametrize("kw", [
    dict(new=_P), dict(cu=_P), dict(cu=_P + 68), dict(slots=_P + 124), dict(table=_P + 204), dict(ring=_P + 256),
    dict(lens_out=_P + 64), dict(lens_out=_P + 4), dict(pool_out=_P + 200), dict(pool_out=_P), dict(cu=_P + 320),
    dict(lens_out=_P + 60), dict(table=_P + 300),
])
def test_block_tables_arrays_do_not_overlap(lib, kw):
    assert _tables(lib, **kw) == 1


@pytest.mark.parametrize("kw,expect", [
    (dict(n=-1), 1), (dict(k=None), 1), (dict(v=_P + 8), 1), (dict(slots=None), 1), (dict(slots=_P + 1), 1),
    (dict(tok=4), 1), (dict(head=-8), 1), (dict(n=0), 0),
])
def test_cache_write_arguments(lib, kw, expect):
    assert _write(lib, **kw) == expect


def test_config_is_checked(lib):
    for cfg, expect in ((_cfg(head_dim=64), 2), (_cfg(num_kv_heads=5), 1), (_cfg(softmax_scale=-1.0), 1),
                        (_cfg(num_q_heads=512, num_kv_heads=8, head_mask=np.ones((2, 512), np.uint8)), 2)):
        assert _prefill(lib, cfg=cfg) == expect
        assert _paged(lib, cfg=cfg) == expect
        assert _write(lib, cfg=cfg) == expect


@pytest.mark.skipif(not _NO_GPU, reason="CPU-only behaviour")
def test_valid_calls_without_a_gpu_report_a_cuda_error(lib):
    for call in (_prefill, _paged, _tables, _write):
        assert call(lib) == 4
