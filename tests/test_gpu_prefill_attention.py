"""ckv_prefill_attention against a plain 64-bit attention: lengths around the tiles, ragged and empty
sequences, head layouts, strides, logits that grow, fall, tie and overflow a naive exponential, values
that must not leak, streams, captured graphs, and its way into the compression."""
import math

import numpy as np
import pytest
import torch

import paper_2508_02401_gb300 as ckv
from tests import attention_ref as ref
from tests.gpu_util import Guarded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    ckv.load()


def config(hq=8, hkv=2, window=32, **kw):
    return ckv.Config(num_layers=1, num_q_heads=hq, num_kv_heads=hkv, window=window, pool_kernel=7,
                      pool_type=ckv.POOL_MAX, head_order=ckv.POOL_THEN_SUM,
                      head_mask=np.ones((1, hq), np.uint8), budgets=np.array([64], np.int32), **kw)


def normal(*shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 17 * sum(shape))
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def run(cfg, lens, q, k, v, stream=None, pad=0, **strides):
    """The call with canaries around every output; (out, lse, lse_win) with NaN where nothing was written."""
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    batch = ckv.Batch(cu)
    T, S, hq, w = int(cu[-1]), len(lens), cfg.num_q_heads, cfg.window
    ws = ckv.new_attention_workspace(cfg)
    out = Guarded((T, hq, 128), torch.bfloat16, math.nan)
    lse = Guarded((hq, T + pad), torch.float32, math.nan)
    win = Guarded((hq, S * w + pad), torch.float32, math.nan)
    ckv.ckv_prefill_attention(cfg, batch, q, k, v, out.view, ws, lse=lse.view, lse_win=win.view,
                              lse_head_stride=T + pad if pad else 0, lse_win_head_stride=S * w + pad if pad else 0,
                              stream=stream, **strides)
    assert ckv.ckv_read_device_status(ws, stream=stream) == (0, 0)
    for g in (out, lse, win):
        g.check()
    if pad:
        assert bool(lse.view[:, T:].isnan().all()) and bool(win.view[:, S * w:].isnan().all())
    # the counters of split units are left zero for the next call
    assert not bool(ws[:1536].any())
    return out.view, lse.view[:, :T], win.view[:, :S * w]


def check(cfg, lens, q, k, v, scale=None, **kw):
    out, lse, win = run(cfg, lens, q, k, v, **kw)
    a, w = 0, cfg.window
    for s, n in enumerate(lens):
        o, l, tol, tol_l = ref.rows(q[a:a + n], k[a:a + n], v[a:a + n], torch.arange(n), scale)
        ref.assert_close(out[a:a + n], o, tol, f"out of sequence {s} ({n} tokens)")
        ref.assert_close(lse[:, a:a + n], l, tol_l, f"lse of sequence {s} ({n} tokens)")
        t = min(w, n)
        assert torch.equal(win[:, s * w + w - t:s * w + w], lse[:, a + n - t:a + n])
        assert bool(win[:, s * w:s * w + w - t].isnan().all())
        a += n
    return out, lse, win


LENS = [(1,), (2, 5), (31, 32, 33, 34), (63, 64, 65), (127, 128, 129), (255, 256, 257), (0, 300, 0, 1, 77, 0),
        (1000, 513), (2049,), (17,) * 40]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("hq,hkv", [(8, 2), (4, 4), (28, 4)])
def test_lengths_and_heads(lens, hq, hkv):
    T = sum(lens)
    check(config(hq, hkv), lens, normal(T, hq, 128, seed=1), normal(T, hkv, 128, seed=2), normal(T, hkv, 128, seed=3))


@pytest.mark.parametrize("hq,hkv", [(1, 1), (6, 1), (96, 1), (256, 1), (256, 2), (15, 5), (256, 256)])
def test_unusual_groups(hq, hkv):
    lens = (70, 1, 150)
    T = sum(lens)
    check(config(hq, hkv, window=8), lens, normal(T, hq, 128, seed=1), normal(T, hkv, 128, seed=2),
          normal(T, hkv, 128, seed=3), pad=3)


@pytest.mark.parametrize("max_ctas", [1, 7])
def test_capped_grid(max_ctas):
    lens = (500, 3, 900)
    T = sum(lens)
    check(config(max_ctas=max_ctas), lens, normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2),
          normal(T, 2, 128, seed=3))


@pytest.mark.parametrize("max_ctas", [0, 3, 64])
@pytest.mark.parametrize("lens", [(1000,), (1024, 1025, 1000), (900, 40, 1300, 2, 1151, 1153, 640, 1)])
def test_prompts_about_the_length_of_uncut_units(lens, max_ctas):
    """Row tiles of up to eight key tiles are whole, those above are cut, in runs that begin and end inside them."""
    T = sum(lens)
    check(config(8, 2, max_ctas=max_ctas), lens, normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2), normal(T, 2, 128, seed=3))


def test_many_prompts():
    """More sequences than the plan has threads, empty ones among them."""
    lens = tuple(int(x) for x in np.random.default_rng(3).integers(0, 9, 900))
    T = sum(lens)
    check(config(2, 1, window=8), lens, normal(T, 2, 128, seed=1), normal(T, 1, 128, seed=2), normal(T, 1, 128, seed=3))


def test_one_long_prompt_per_cta_split():
    """Few row tiles and many keys: units are cut over CTAs and joined."""
    lens = (6001,)
    check(config(2, 1, window=64), lens, normal(6001, 2, 128, seed=1), normal(6001, 1, 128, seed=2),
          normal(6001, 1, 128, seed=3))


@pytest.mark.parametrize("hq,hkv", [(2, 2), (8, 2), (28, 4)])
@pytest.mark.parametrize("max_ctas", [0, 1, 5])
def test_key_tiles_of_one_row_tile(hq, hkv, max_ctas):
    """A unit's first row tile does not see its last keys, short units have no second one, and parts of cut units
    may have no tile for either: every tile of the ring is released once by both, call after call."""
    lens = (100, 257, 1500, 128, 40, 2700, 129, 1, 1900)
    T = sum(lens)
    cfg = config(hq, hkv, max_ctas=max_ctas)
    q, k, v = normal(T, hq, 128, seed=1), normal(T, hkv, 128, seed=2), normal(T, hkv, 128, seed=3)
    out, lse, _ = check(cfg, lens, q, k, v)
    for _ in range(10):
        again = run(cfg, lens, q, k, v)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_strided_tensors():
    """q, k and v as slices of one fused projection [T, H_q + 2 H_kv, 128], and k, v interleaved."""
    hq, hkv, lens = 8, 2, (300, 77)
    T = sum(lens)
    fused = normal(T, hq + 2 * hkv, 128, seed=4)
    q, k, v = fused[:, :hq], fused[:, hq:hq + hkv], fused[:, hq + hkv:]
    st = (hq + 2 * hkv) * 128
    check(config(hq, hkv), lens, q, k, v, q_tok_stride=st, tok_stride=st)
    # heads outermost: [H, T, 128]
    qh, kh, vh = (normal(h, T, 128, seed=5 + h).transpose(0, 1) for h in (hq, hkv, hkv))
    check(config(hq, hkv), lens, qh, kh, vh, q_tok_stride=128, q_head_stride=T * 128, tok_stride=128,
          head_stride=T * 128)


@pytest.mark.parametrize("scale", [0.02, 1.0])
def test_given_scale(scale):
    T = 400
    check(config(softmax_scale=scale), (T,), normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2),
          normal(T, 2, 128, seed=3), scale=np.float32(scale).item())


@pytest.mark.parametrize("kind", ["rising", "falling", "spikes", "equal", "zero_q", "huge", "lowest"])
def test_logits_of_every_kind(kind):
    """Running maxima that move at every key tile, that never move, far logits, equal ones."""
    T, hq, hkv = 1500, 4, 2
    q, k, v = normal(T, hq, 128, seed=1), normal(T, hkv, 128, seed=2), normal(T, hkv, 128, seed=3)
    if kind in ("rising", "falling"):
        q = torch.ones_like(q)
        ramp = torch.arange(T, device="cuda", dtype=torch.float32) / 64
        k = (ramp if kind == "rising" else ramp.flip(0))[:, None, None].expand(T, hkv, 128).to(torch.bfloat16).contiguous()
    elif kind == "spikes":
        k[::97] *= 20
        q *= 4
    elif kind == "equal":
        k = k[:1].expand(T, hkv, 128).contiguous()
    elif kind == "zero_q":
        q = torch.zeros_like(q)
    elif kind == "huge":
        q, k = q * 60, k * 60
    else:  # logits of about -1e7, then +1e7: equal, so every row is the mean of its largest
        q, k = torch.full_like(q, 1000.0), torch.full_like(k, -1000.0)
        k[700:] = 1000.0
        out, _, _ = check(config(hq, hkv), (T,), q, k, v)
        for i in (0, 5, 699, 700, 701, 1499):
            seen = v[700:i + 1] if i >= 700 else v[:i + 1]
            seen = seen.double().repeat_interleave(hq // hkv, 1)
            ref.assert_close(out[i], seen.mean(0), 2.0 ** -7 * seen.abs().mean(0), f"row {i}")
        return
    check(config(hq, hkv), (T,), q, k, v)


def test_nothing_leaks_between_sequences():
    """NaN and infinities in one sequence of a packed batch leave the others' rows as they are, and
    those behind the last token of the buffers too."""
    lens = (130, 70, 257)
    T = sum(lens)
    q, k, v = normal(T + 40, 8, 128, seed=1), normal(T + 40, 2, 128, seed=2), normal(T + 40, 2, 128, seed=3)
    want = run(config(), lens, q[:T], k[:T], v[:T])
    k[130:200], v[130:200] = math.nan, math.inf
    q[130:200] = -math.inf
    for x in (q, k, v):
        x[T:] = math.nan
    got = run(config(), lens, q, k, v)
    for a, b in ((0, 130), (200, T)):
        assert torch.equal(got[0][a:b], want[0][a:b])
        assert torch.equal(got[1][:, a:b], want[1][:, a:b])


def test_masked_keys_of_any_value():
    """Keys that a row does not see may be anything: NaN and infinities in k[j] reach rows >= j only."""
    T = 700
    q, k, v = normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2), normal(T, 2, 128, seed=3)
    want = run(config(), (T,), q, k, v)
    for bad in (math.nan, math.inf, -math.inf, torch.finfo(torch.bfloat16).min):
        kk = k.clone()
        kk[333:] = bad
        got = run(config(), (T,), q, kk, v)
        assert torch.equal(got[0][:333], want[0][:333]) and torch.equal(got[1][:, :333], want[1][:, :333])


@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2), (28, 4), (6, 2)])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_values_that_are_not_finite_reach_no_row_far_before_them(hq, hkv, bad):
    """A row at least 256 tokens before such a value is as if it were not there; every row that sees it is not finite."""
    T = 1300
    cfg, q, k, v = config(hq, hkv), normal(T, hq, 128, seed=1), normal(T, hkv, 128, seed=2), normal(T, hkv, 128, seed=3)
    want = run(cfg, (T,), q, k, v)
    for j in (256, 511, 700, 1023, 1299):
        vv = v.clone()
        vv[j] = bad
        got = run(cfg, (T,), q, k, vv)
        assert torch.equal(got[0][:j - 255], want[0][:j - 255]) and torch.equal(got[1], want[1])
        assert not bool(got[0][j:].isfinite().any())


@pytest.mark.parametrize("span", [(0, 1), (256, 640), (0, 4096), (4000, 4096)])
def test_nan_keys_that_rows_see(span):
    """NaN keys, a tile's or a part's worth of them: every row that sees one is NaN, in out and lse."""
    T, hq = 4500, 2  # few row tiles: their keys are cut over CTAs
    cfg, q, k, v = config(hq, 1), normal(T, hq, 128, seed=1), normal(T, 1, 128, seed=2), normal(T, 1, 128, seed=3)
    k[span[0]:span[1]] = math.nan
    out, lse, _ = run(cfg, (T,), q, k, v)
    assert bool(out[span[0]:].isnan().all()) and bool(lse[:, span[0]:].isnan().all())
    assert not bool(out[:span[0]].isnan().any()) and not bool(lse[:, :span[0]].isnan().any())


def test_every_output_is_optional_and_repeatable():
    T = 1000
    cfg, q, k, v = config(), normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2), normal(T, 2, 128, seed=3)
    want = run(cfg, (T,), q, k, v)
    batch, ws = ckv.Batch([0, T]), ckv.new_attention_workspace(cfg)
    for _ in range(2):  # the same workspace again
        out = torch.empty_like(q)
        ckv.ckv_prefill_attention(cfg, batch, q, k, v, out, ws)
        assert torch.equal(out, want[0])


def test_other_stream_and_graph():
    T = 900
    cfg, q, k, v = config(), normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2), normal(T, 2, 128, seed=3)
    want = run(cfg, (T,), q, k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(cfg, (T,), q, k, v, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0])
    batch, ws, out = ckv.Batch([0, T]), ckv.new_attention_workspace(cfg), torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ckv.ckv_prefill_attention(cfg, batch, q, k, v, out, ws)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert torch.equal(out, want[0])
    q2 = normal(T, 8, 128, seed=9)
    q.copy_(q2)
    graph.replay()
    assert torch.equal(out, run(cfg, (T,), q2, k, v)[0])


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    T = 3000
    cfg = config(max_ctas=70)
    sides = [torch.cuda.Stream() for _ in range(2)]
    ins = [[normal(T, h, 128, seed=s) for s, h in ((10 * i, 8), (10 * i + 1, 2), (10 * i + 2, 2))] for i in range(2)]
    wants = [run(cfg, (T,), *x)[0].clone() for x in ins]
    batch = ckv.Batch([0, T])
    wss, outs = [ckv.new_attention_workspace(cfg) for _ in range(2)], [torch.zeros_like(x[0]) for x in ins]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            ckv.ckv_prefill_attention(cfg, batch, *ins[i], outs[i], wss[i], stream=sides[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], wants[i])


def test_lengths_on_the_device_that_disagree_are_reported():
    cfg, T = config(), 200
    q, k, v = normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2), normal(T, 2, 128, seed=3)
    ws, out = ckv.new_attention_workspace(cfg), Guarded((T, 8, 128), torch.bfloat16)
    batch = ckv.Batch([0, 100, T], cu_seqlens_dev=torch.tensor([0, 120, T], dtype=torch.int32, device="cuda"))
    ckv.ckv_prefill_attention(cfg, batch, q, k, v, out.view, ws)
    assert ckv.ckv_read_device_status(ws)[0] == 1
    # lengths past the end of the buffers are not followed
    batch = ckv.Batch([0, 100, T], cu_seqlens_dev=torch.tensor([0, 100, T + 5000], dtype=torch.int32, device="cuda"))
    ckv.ckv_prefill_attention(cfg, batch, q, k, v, out.view, ws)
    assert ckv.ckv_read_device_status(ws)[0] != 0
    out.check()


@pytest.mark.parametrize("dev", [(0, 0, 0, 0), (7, 7, 7, 7), (0, 150, 100, 200), (0, 100, 100, 5000), (-3, 100, 150, 200),
                                 (0, 200, 100, 200)])
def test_device_lengths_without_tokens_or_out_of_order_are_reported(dev):
    """A copy that is not there yet (no token at all) or that makes no sense: code 1 and nothing written."""
    cfg, T = config(), 200
    q, k, v = normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2), normal(T, 2, 128, seed=3)
    ws, out = ckv.new_attention_workspace(cfg), Guarded((T, 8, 128), torch.bfloat16, 7.0)
    batch = ckv.Batch([0, 100, 150, T], cu_seqlens_dev=torch.tensor(dev, dtype=torch.int32, device="cuda"))
    ckv.ckv_prefill_attention(cfg, batch, q, k, v, out.view, ws)
    assert ckv.ckv_read_device_status(ws)[0] == 1
    out.check()
    assert bool((out.view == 7).all())


def test_refusals():
    cfg, T = config(), 64
    q, k, v = normal(T, 8, 128), normal(T, 2, 128), normal(T, 2, 128)
    out, ws, batch = torch.empty_like(q), ckv.new_attention_workspace(cfg), ckv.Batch([0, T])

    def call(q=q, k=k, v=v, out=out, batch=batch, **kw):
        ckv.ckv_prefill_attention(cfg, batch, q, k, v, out, ws, **kw)

    call()
    for bad in (dict(q=q.float()), dict(k=k.cpu()), dict(v=v[:, :1]), dict(out=out[:-1]), dict(q=q[::2]),
                dict(q=q[:-1]), dict(lse=torch.empty(8, T - 1, device="cuda")),
                dict(lse_win=torch.empty(8, 32, dtype=torch.float64, device="cuda")), dict(k=k[:, :, :64]),
                dict(tok_stride=512), dict(out=out.transpose(0, 1)), dict(batch=ckv.Batch([0, T], device="cpu")),
                dict(batch=ckv.Batch([0, T], cu_seqlens_dev=batch.cu_dev.long())),
                dict(batch=ckv.Batch([0, T], cu_seqlens_dev=batch.cu_dev[:1]))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ckv.CkvError):
        call(lse=torch.empty(8 * T, device="cuda"), lse_head_stride=T - 1)
