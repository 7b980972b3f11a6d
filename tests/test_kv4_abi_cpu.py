"""Argument checks of the appends and of the attention over 4 bits on the host: every one returns before a launch, so
none needs a GPU."""
import ctypes as C

import pytest

import paper_2508_02401_gb300 as ckv
from tests.test_abi_cpu import _cfg
from tests.test_attention_abi_cpu import _cache

_P = 0x4000000  # 256-byte-aligned fake device addresses, far apart
_STEP = 0x1000000
_K, _V, _SLOTS, _Q, _QO, _KO, _VO, _POS, _TAB, _PAGES, _VP, _W = (_P + i * _STEP for i in range(12))
_WS = 1 << 40
_NO_GPU = not __import__("torch").cuda.is_available()


@pytest.fixture(scope="module")
def lib():
    from paper_2508_02401_gb300 import build
    build.build()
    return ckv.load()


def _cache4(pages_at=_PAGES, stride=0, pages=10, page=16):
    return C.byref(ckv._PagedCacheQ4(pages_at, stride, pages, page))


def _rot(cs=_TAB, n=100, rd=128, inter=0):
    return C.byref(ckv._Rotation(cs, n, rd, inter))


_NONE = object()


def _append(lib, q4, cfg=None, cache=None, n=3, q=None, q_tok=0, q_head=0, q_out=None, k=_K, v=_V, tok=0, head=0, k_out=None,
            v_out=None, rot=_NONE, pos=_POS, slots=_SLOTS, ws=_W, ws_bytes=_WS):
    cfg = cfg or _cfg()
    rot = _rot() if rot is _NONE else rot
    if q4:
        return lib.ckv_cache_append_q4(cfg.ref, cache or _cache4(), n, q, q_tok, q_head, q_out, k, v, tok, head, k_out, v_out, rot,
                                       pos, slots, ws, ws_bytes, None)
    return lib.ckv_cache_append(cfg.ref, cache or _cache(_PAGES, _VP), n, q, q_tok, q_head, q_out, k, v, tok, head, k_out, rot, pos,
                                slots, ws, ws_bytes, None)


def _paged4(lib, cfg=None, cache=None, S=2, T=2, table=_P, blocks=4, lens=_P, cu=_P, q=_P, q_tok=0, q_head=0, out=_P,
            lse=None, lse_st=0, ws=_P, ws_bytes=_WS):
    cfg = cfg or _cfg()
    return lib.ckv_paged_attention_q4(cfg.ref, cache or _cache4(), S, T, table, blocks, lens, cu, q, q_tok, q_head, out,
                                      lse, lse_st, ws, ws_bytes, None)


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("kw,expect", [
    (dict(n=-1), 1), (dict(k=None), 1), (dict(v=None), 1), (dict(k=_K + 8), 1), (dict(v=_V + 2), 1), (dict(slots=None), 1),
    (dict(slots=_SLOTS + 1), 1), (dict(pos=None), 1), (dict(pos=_POS + 2), 1), (dict(tok=4), 1), (dict(head=-8), 1),
    (dict(tok=1 << 38), 2), (dict(q=_Q), 1), (dict(q_out=_QO), 1), (dict(q=_Q + 8, q_out=_QO), 1), (dict(q=_Q, q_out=_QO + 4), 1),
    (dict(q=_Q, q_out=_QO, q_tok=12), 1), (dict(k_out=_KO + 2), 1), (dict(rot=_rot(cs=None)), 1), (dict(rot=_rot(cs=_TAB + 4)), 1),
    (dict(rot=_rot(n=0)), 1), (dict(rot=_rot(rd=0)), 1), (dict(rot=_rot(rd=8)), 1), (dict(rot=_rot(rd=24)), 1),
    (dict(rot=_rot(rd=144)), 1), (dict(rot=_rot(rd=-16)), 1), (dict(rot=_rot(inter=2)), 1), (dict(ws=None), 3),
    (dict(ws=_W + 128), 3), (dict(ws_bytes=100), 3), (dict(n=0), 0), (dict(n=0, k=None, v=None, slots=None, pos=None), 0),
])
def test_append_arguments(lib, q4, kw, expect):
    assert _append(lib, q4, **kw) == expect


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("kw", [
    dict(k_out=_V), dict(k_out=_K + 16), dict(k_out=_K, tok=2048), dict(k_out=_SLOTS - 16), dict(k_out=_POS), dict(k_out=_TAB + 128),
    dict(k_out=_PAGES), dict(k_out=_PAGES + 160), dict(q=_Q, q_out=_K), dict(q=_Q, q_out=_Q + 256), dict(q=_Q, q_out=_Q, q_tok=6144),
    dict(q=_Q, q_out=_PAGES - 128), dict(q=_Q, q_out=_KO, k_out=_KO + 16), dict(k=_PAGES + 64), dict(v=_PAGES), dict(slots=_PAGES),
    dict(q=_PAGES, q_out=_QO), dict(pos=_PAGES + 4), dict(rot=_rot(cs=_PAGES)),
])
def test_append_writes_over_nothing(lib, q4, kw):
    assert _append(lib, q4, **kw) == 1


_PAGE = 16 * 8 * 256  # bytes of a bf16 page of K


@pytest.mark.parametrize("v_at,stride,pages", [
    (_PAGES, 0, 10), (_PAGES + 16, 0, 10), (_PAGES + _PAGE - 16, 0, 1), (_PAGES - _PAGE + 16, 0, 1), (_PAGES + 3 * _PAGE, 0, 10),
    (_PAGES + 9 * _PAGE, 0, 10), (_PAGES - 9 * _PAGE - 16, 0, 10), (_PAGES + _PAGE - 16, _PAGE, 10), (_PAGES + _PAGE + 16, _PAGE, 10),
    (_PAGES + 2 * _PAGE, _PAGE, 10), (_PAGES + 3 * _PAGE - 16, _PAGE, 2), (_PAGES - 3 * _PAGE + 16, _PAGE, 2),
])
def test_append_refuses_pages_of_k_over_pages_of_v(lib, v_at, stride, pages):
    assert _append(lib, False, cache=_cache(_PAGES, v_at, stride, pages)) == 1


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("kw", [
    dict(k_out=_W), dict(q=_Q, q_out=_W - 16), dict(slots=_W), dict(pos=_W + 256), dict(k=_W + 1024), dict(v=_W - 256),
    dict(q=_W, q_out=_QO), dict(rot=_rot(cs=_W - 64)),
])
def test_append_refuses_a_workspace_over_the_rest(lib, q4, kw):
    assert _append(lib, q4, **kw) == 1
    assert _append(lib, q4, cache=_cache4(_W - 16) if q4 else _cache(_W + 512, _VP)) == 1
    if not q4:
        assert _append(lib, q4, cache=_cache(_VP, _W)) == 1


def test_append_q4_outputs(lib):
    for kw in (dict(v_out=_VO + 8), dict(v_out=_K), dict(k_out=_KO, v_out=_KO), dict(v_out=_V, tok=2048), dict(k_out=_V, v_out=_K)):
        assert _append(lib, True, **kw) == 1
    # rows that are rotated already: no positions, no queries
    assert _append(lib, True, rot=None) == 1
    assert _append(lib, True, rot=None, pos=None, q=_Q, q_out=_QO) == 1
    assert _append(lib, False, rot=None, pos=None) == 1


@pytest.mark.parametrize("cache,expect", [
    (dict(pages_at=None), 1), (dict(pages_at=_PAGES + 8), 1), (dict(page=0), 1), (dict(page=24), 2), (dict(page=256), 2),
    (dict(pages=0), 1), (dict(pages=1 << 27), 2), (dict(stride=8), 1), (dict(stride=16 * 8 * 144 - 16), 1),
    (dict(stride=16 * 8 * 144 + 8), 1), (dict(stride=1 << 38), 2),
])
def test_cache_arguments(lib, cache, expect):
    assert _append(lib, True, cache=_cache4(**cache)) == expect
    assert _paged4(lib, cache=_cache4(**cache)) == expect
    cfg = _cfg()
    assert lib.ckv_paged_attention_q4(cfg.ref, None, 2, 2, _P, 4, _P, _P, _P, 0, 0, _P, None, 0, _P, _WS, None) == 1
    assert lib.ckv_cache_append_q4(cfg.ref, None, 2, None, 0, 0, None, _K, _V, 0, 0, None, None, _rot(), _POS, _SLOTS, _W, _WS, None) == 1


@pytest.mark.parametrize("kw,expect", [
    (dict(S=0), 1), (dict(T=-1), 1), (dict(blocks=0), 1), (dict(table=None), 1), (dict(lens=None), 1), (dict(cu=None), 1),
    (dict(table=_P + 2), 1), (dict(q=None), 1), (dict(out=None), 1), (dict(q=_P + 8), 1), (dict(q_tok=4), 1),
    (dict(lse=_P, lse_st=1), 1), (dict(blocks=1 << 28), 2), (dict(T=0), 0), (dict(ws=None), 3), (dict(ws_bytes=5), 3),
])
def test_paged_attention_arguments(lib, kw, expect):
    assert _paged4(lib, **kw) == expect


def test_config_is_checked(lib):
    for cfg, expect in ((_cfg(head_dim=64), 2), (_cfg(num_kv_heads=5), 1), (_cfg(softmax_scale=-1.0), 1)):
        assert _append(lib, False, cfg=cfg) == expect
        assert _append(lib, True, cfg=cfg) == expect
        assert _paged4(lib, cfg=cfg) == expect


@pytest.mark.skipif(not _NO_GPU, reason="CPU-only behaviour")
def test_valid_calls_without_a_gpu_report_a_cuda_error(lib):
    for q4 in (False, True):
        assert _append(lib, q4, q=_Q, q_out=_QO, k_out=_KO) == 4
        assert _append(lib, q4, q=_Q, q_out=_Q, k_out=_K) == 4  # in place
    assert _append(lib, True, rot=None, pos=None, k_out=_K, v_out=_V) == 4
    assert _paged4(lib) == 4
    # K's and V's pages side by side, alternating, or V's before K's
    for v_at, stride, pages in ((_PAGES + 10 * _PAGE, 0, 10), (_PAGES - 10 * _PAGE, 0, 10), (_PAGES + _PAGE, _PAGE, 10),
                                (_PAGES - _PAGE, _PAGE, 10), (_PAGES + 2 * _PAGE, 3 * _PAGE // 2, 10), (_PAGES + 4 * _PAGE, _PAGE, 2),
                                (_PAGES + _PAGE, 0, 1)):
        assert _append(lib, False, cache=_cache(_PAGES, v_at, stride, pages)) == 4


def test_an_older_library_is_named(lib, monkeypatch):
    """A library without one of the calls, though its version is the same: said when it is loaded, and nothing of it is kept."""

    class Older:
        def __getattr__(self, name):
            if name == "ckv_cache_append_q4":
                raise AttributeError(name)
            return getattr(lib, name)

    monkeypatch.setattr(ckv, "_lib", None)
    monkeypatch.setattr(ckv.C, "CDLL", lambda path: Older())
    with pytest.raises(ImportError, match="ckv_cache_append_q4.*version 7.*build"):
        ckv.load()
    assert ckv._lib is None
