"""ckv_paged_attention against a plain 64-bit attention: single tokens, chunks and mixtures of them over
pages of every size in any order, unused page rows of any value, long caches cut over CTAs, padding
rows, lengths that grow under a captured graph, bad pages and lengths."""
import math

import numpy as np
import pytest
import torch

import paper_2508_02401_gb300 as ckv
from tests import attention_ref as ref
from tests.gpu_util import Guarded
from tests.test_gpu_prefill_attention import config, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    ckv.load()


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


class Paged:
    """A batch over a paged cache: pages in random order, everything that is not a cached row NaN."""

    def __init__(self, cfg, lens, new, page, seed=0, pad=0, spare=2, interleaved=False, extra_blocks=0):
        self.cfg, self.lens, self.new, self.page = cfg, list(lens), list(new), page
        hq, hkv = cfg.num_q_heads, cfg.num_kv_heads
        g = np.random.default_rng(seed)
        blocks = [-(-n // page) for n in lens]
        pages = sum(blocks) + spare
        order = g.permutation(pages)
        self.table = np.full((len(lens), max(1, max(blocks)) + extra_blocks), -1, np.int32)
        if interleaved:
            both = torch.full((pages, 2, page, hkv, 128), math.nan, dtype=torch.bfloat16, device="cuda")
            self.k_pages, self.v_pages = both[:, 0], both[:, 1]
        else:
            self.k_pages = torch.full((pages, page, hkv, 128), math.nan, dtype=torch.bfloat16, device="cuda")
            self.v_pages = torch.full_like(self.k_pages, math.nan)
        self.k, self.v, at = [], [], 0
        for s, n in enumerate(lens):
            self.table[s, :blocks[s]] = order[at:at + blocks[s]]
            at += blocks[s]
            k, v = normal(n, hkv, 128, seed=seed + 3 * s + 1), normal(n, hkv, 128, seed=seed + 3 * s + 2)
            self.k.append(k)
            self.v.append(v)
            j = torch.arange(n, device="cuda")
            p = dev(self.table[s], torch.int64)[j // page]
            self.k_pages[p, j % page], self.v_pages[p, j % page] = k, v
        self.cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.T = int(self.cu[-1]) + pad
        self.q = normal(self.T, hq, 128, seed=seed + 1000)

    def run(self, base=0, pad=0, status=(0, 0), max_blocks=None, q=None, ws=None, stream=None, **strides):
        cfg, hq = self.cfg, self.cfg.num_q_heads
        q = self.q if q is None else q
        out = Guarded((self.T, hq, 128), torch.bfloat16, 7.0)
        lse = Guarded((hq, self.T + pad), torch.float32, 7.0)
        ws = ckv.new_attention_workspace(cfg) if ws is None else ws
        ckv.ckv_paged_attention(cfg, ckv.PagedCache(self.k_pages, self.v_pages), dev(self.table), dev(self.lens),
                                dev(self.cu + base), q, out.view, ws, lse=lse.view,
                                lse_head_stride=self.T + pad if pad else 0, stream=stream, **strides)
        assert ckv.ckv_read_device_status(ws, stream=stream)[0] == status[0]
        out.check()
        lse.check()
        assert not bool(ws[256:1536].any())
        return out.view, lse.view

    def check(self, **kw):
        out, lse = self.run(**kw)
        for s, (L, n) in enumerate(zip(self.lens, self.new)):
            a = int(self.cu[s])
            o, l, tol, tol_l = ref.rows(self.q[a:a + n], self.k[s], self.v[s], torch.arange(L - n, L))
            ref.assert_close(out[a:a + n], o, tol, f"out of sequence {s} ({n} of {L})")
            ref.assert_close(lse[:, a:a + n], l, tol_l, f"lse of sequence {s} ({n} of {L})")
        end = int(self.cu[-1])  # rows behind the last sequence are left as they were
        assert bool((out[end:] == 7).all()) and bool((lse[:, end:] == 7).all())
        return out, lse


CASES = [
    ((1,), (1,)), ((2, 1, 3), (1, 1, 1)), ((127, 128, 129, 130), (1, 1, 1, 1)),
    ((16, 17, 33, 64, 65), (1, 1, 1, 1, 1)), ((500, 0, 300, 0), (1, 0, 1, 0)),
    ((300, 400, 77), (4, 0, 5)), ((200, 900), (200, 1)), ((1000, 513, 700), (130, 257, 64)),
    ((129,) * 50, (1,) * 50), ((4000, 10, 2500), (1, 10, 1)),
]


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_lengths_and_pages(case, page):
    lens, new = CASES[case]
    hq, hkv = [(8, 2), (28, 4), (4, 4)][case % 3]
    Paged(config(hq, hkv), lens, new, page, seed=case, pad=case % 3, extra_blocks=case % 2).check()


@pytest.mark.parametrize("hq,hkv,new", [(1, 1, 1), (6, 1, 3), (96, 1, 2), (256, 1, 1), (256, 2, 2), (15, 5, 9)])
def test_unusual_groups(hq, hkv, new):
    Paged(config(hq, hkv), (700, 131, 40), (new, new, new), 16, seed=5).check(pad=3)


@pytest.mark.parametrize("new", [1, 2, 3, 4, 5, 70])
@pytest.mark.parametrize("max_ctas", [0, 5])
def test_long_caches_are_cut_and_joined(new, max_ctas):
    Paged(config(8, 2, max_ctas=max_ctas), (20011, 77, 9000), (new, new, 1), 64, seed=6).check()


@pytest.mark.parametrize("new", [1, 70])
def test_nan_keys_in_one_part(new):
    """A stretch of NaN keys as long as a part of a cut unit makes the rows that see it NaN."""
    c = Paged(config(8, 2), (9001, 500), (new, 1), 32, seed=17)
    pages = dev(c.table[0], torch.int64)[64:160]
    c.k_pages[pages] = math.nan
    out, lse = c.run()
    assert bool(out[:new].isnan().all()) and bool(lse[:, :new].isnan().all())
    assert not bool(out[new:].isnan().any()) and not bool(lse[:, new:].isnan().any())


@pytest.mark.parametrize("singles", [0, 1])
@pytest.mark.parametrize("chunk", [1, 17, 40, 41, 42, 130, 300])
def test_a_chunk_among_single_tokens(chunk, singles):
    """Either kernel takes single tokens (or idle sequences) and a chunk in one call."""
    lens, new = [33 + 7 * i for i in range(40)] + [900], [singles] * 40 + [chunk]
    Paged(config(8, 2), lens, new, 32, seed=19).check()


@pytest.mark.parametrize("hq,hkv", [(2, 2), (28, 4)])
@pytest.mark.parametrize("max_ctas", [0, 1, 5])
def test_key_tiles_of_one_row_tile(hq, hkv, max_ctas):
    """Chunks whose units' first row tile sees fewer key tiles than the second, and units that have one row tile."""
    c = Paged(config(hq, hkv, max_ctas=max_ctas), (1500, 300, 2700, 129, 640), (257, 3, 300, 129, 100), 16, seed=23)
    out, lse = c.check()
    for _ in range(10):
        again = c.run()
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_many_sequences():
    """More sequences than the plan has threads, empty ones among them."""
    g = np.random.default_rng(3)
    lens = [int(x) for x in g.integers(0, 40, 1500)]
    new = [min(n, int(x)) for n, x in zip(lens, g.integers(0, 3, 1500))]
    Paged(config(4, 1), lens, new, 16, seed=18, pad=3).check()


def test_growing_maxima_over_the_cut():
    """Each key tile's logits above the last one's: every part of a cut unit has another reference."""
    c = Paged(config(8, 2), (9001,), (2,), 32, seed=7)
    ramp = (torch.arange(9001, device="cuda", dtype=torch.float32) / 256)[:, None, None]
    c.q = torch.ones_like(c.q)
    k = ramp.expand(9001, 2, 128).to(torch.bfloat16)
    c.k[0] = k
    j = torch.arange(9001, device="cuda")
    c.k_pages[dev(c.table[0], torch.int64)[j // 32], j % 32] = k
    c.check()


def test_offset_cu_and_strided_q():
    """cu_new as a slice of a longer array (it need not begin at 0), q inside a fused projection."""
    c = Paged(config(8, 2), (300, 40, 513), (1, 7, 33), 32, seed=8)
    fused = torch.zeros((c.T, 12, 128), dtype=torch.bfloat16, device="cuda")
    fused[:, :8] = c.q
    c.check(base=1000)
    want = c.run()
    got = c.run(q=fused[:, :8], q_tok_stride=12 * 128)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_one_buffer_for_k_and_v():
    Paged(config(8, 2), (300, 40, 513), (1, 7, 33), 32, seed=9, interleaved=True).check()


def test_pages_shared_by_two_sequences():
    """A common prefix: the same pages in both rows of the table."""
    c = Paged(config(8, 2), (256, 300), (1, 1), 64, seed=10)
    c.table[0, :4] = c.table[1, :4]
    c.k[0], c.v[0] = c.k[1][:256], c.v[1][:256]
    c.check()


def test_offsets_beyond_32_bits():
    """Pages whose elements lie beyond 2^32 of the buffer (8 heads, 4.3M slots), first and last ones."""
    hkv, page = 8, 128
    pages = (1 << 32) // (page * hkv * 128) + 9
    c = Paged(config(32, hkv), (500, 900), (1, 20), page, seed=11)
    big = torch.zeros((pages, page, hkv, 128), dtype=torch.bfloat16, device="cuda")
    where = torch.tensor([pages - 1 - i if i % 2 else i for i in range(c.k_pages.shape[0])], device="cuda")
    big[where] = c.k_pages
    c.k_pages = big
    big_v = torch.zeros_like(big)
    big_v[where] = c.v_pages
    c.v_pages = big_v
    live = c.table >= 0
    c.table[live] = where.cpu().numpy()[c.table[live]]
    c.check()


def test_replayed_while_lengths_grow():
    """One captured call over device lengths: each replay sees the lengths of its time."""
    cfg = config(8, 2)
    c = Paged(cfg, (520, 200), (1, 1), 16, seed=12)
    ws, cache = ckv.new_attention_workspace(cfg), ckv.PagedCache(c.k_pages, c.v_pages)
    lens, cu, table, out = dev([1, 1]), dev(c.cu), dev(c.table), torch.zeros_like(c.q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ckv.ckv_paged_attention(cfg, cache, table, lens, cu, c.q, out, ws)
    for now in ([1, 2], [17, 129], [128, 200], [520, 16], [400, 199]):
        lens.copy_(dev(now))
        graph.replay()
        for s in range(2):
            o, _, tol, _ = ref.rows(c.q[s:s + 1], c.k[s][:now[s]], c.v[s][:now[s]], torch.tensor([now[s] - 1]))
            ref.assert_close(out[s:s + 1], o, tol, f"lengths {now}, sequence {s}")
    assert ckv.ckv_read_device_status(ws)[0] == 0


def test_same_results_on_another_stream_and_again():
    c = Paged(config(8, 2), (5000, 77, 300), (1, 1, 40), 32, seed=13)
    want = [x.clone() for x in c.run()]
    side, ws = torch.cuda.Stream(), ckv.new_attention_workspace(c.cfg)
    torch.cuda.synchronize()
    for _ in range(3):
        got = c.run(stream=side, ws=ws)
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("hq,hkv", [(4, 4), (8, 2)])
@pytest.mark.parametrize("new", [3, 600])
def test_values_that_are_not_finite_reach_no_row_far_before_them(hq, hkv, new):
    """As in a prompt, from chunks that begin inside a tile."""
    L = 1171
    c = Paged(config(hq, hkv), (L, 300), (new, 1), 32, seed=24)
    want = [x.clone() for x in c.run()]
    for j in (L - 1, L - 300, L - 599):
        at = int(c.table[0, j // 32]), j % 32
        was = c.v_pages[at].clone()
        c.v_pages[at] = math.nan
        out, lse = c.run()
        c.v_pages[at] = was
        first = j - (L - new)  # the first query row that sees it
        far = max(0, first - 255)
        assert torch.equal(out[:far], want[0][:far]) and torch.equal(lse, want[1])
        assert bool(out[max(0, first):new].isnan().all()) and torch.equal(out[new:], want[0][new:])


def test_calls_of_both_kernels_at_once():
    """Three streams, a workspace each: single tokens, chunks, and the next step's tables beside them."""
    one, chunk = Paged(config(8, 2), (5000, 77, 300), (1, 1, 1), 32, seed=25), Paged(config(8, 2), (3000, 900), (300, 70), 32, seed=26)
    calls = []
    for c in (one, chunk):
        out = torch.zeros_like(c.q)
        calls.append((c, ckv.PagedCache(c.k_pages, c.v_pages), dev(c.table), dev(c.lens), dev(c.cu), out,
                      ckv.new_attention_workspace(c.cfg), torch.cuda.Stream(), c.run()[0].clone()))
    rows, pages = 500, 2000
    lens, ring, pool = dev(np.zeros(rows)), dev(np.arange(pages)), dev([0, pages], torch.int64)
    table, slots, cu = dev(np.zeros((rows, 4))), dev(np.zeros(rows)), dev(np.zeros(rows + 1))
    new, ws, side = dev(np.ones(rows)), ckv.new_attention_workspace(one.cfg), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(60):
        for c, cache, t, n, cn, out, w, stream, _ in calls:
            ckv.ckv_paged_attention(c.cfg, cache, t, n, cn, c.q, out, w, stream=stream)
        ckv.ckv_block_tables(16, lens, new, ring, pool, table, slots, cu, lens, pool, ws, stream=side)
    torch.cuda.synchronize()
    for c, _, _, _, _, out, w, _, want in calls:
        assert torch.equal(out, want) and ckv.ckv_read_device_status(w) == (0, 0)
    assert ckv.ckv_read_device_status(ws) == (0, 0)
    assert bool((lens == 60).all()) and pool.tolist() == [2000, 2000]
    assert sorted(table.reshape(-1).tolist()) == list(range(pages))


@pytest.mark.parametrize("what", ["page", "negative", "short", "long", "decreasing", "past_the_end", "negative_cu"])
def test_bad_lengths_and_pages_are_reported(what):
    """Other sequences' rows are right all the same; nothing outside the outputs is touched."""
    c = Paged(config(8, 2), (300, 200, 400), (1, 3, 2), 32, seed=14)
    lens = list(c.lens)
    good = [0, 2]
    if what == "page":
        c.table[1, 3] = c.k_pages.shape[0]
    elif what == "negative":
        c.table[1, 0] = -5
    elif what == "short":
        c.lens[1] = 2
    elif what == "long":
        c.lens[1] = 13 * 32 + 1
    else:  # rows that cannot be told apart: nothing is written
        i, x = dict(decreasing=(2, 0), past_the_end=(3, 5000), negative_cu=(1, -70))[what]
        c.cu[i] = x
        good = []
    rows = [(0, 1), (1, 4), (4, 6)]
    out, lse = c.run(status=(3, 0))
    if not good:
        assert bool((out == 7).all()) and bool((lse == 7).all())
    for s in good:  # (how a sequence is cut over CTAs, and so its last bits, depends on the others)
        a, b = rows[s]
        o, l, tol, tol_l = ref.rows(c.q[a:b], c.k[s], c.v[s], torch.arange(lens[s] - (b - a), lens[s]))
        ref.assert_close(out[a:b], o, tol, f"out of sequence {s}")
        ref.assert_close(lse[:, a:b], l, tol_l, f"lse of sequence {s}")


def test_refusals():
    c = Paged(config(8, 2), (300, 200), (1, 1), 32, seed=15)
    cfg, cache, ws = c.cfg, ckv.PagedCache(c.k_pages, c.v_pages), ckv.new_attention_workspace(c.cfg)
    base = dict(table=dev(c.table), lens=dev(c.lens), cu=dev(c.cu), q=c.q, out=torch.empty_like(c.q))

    def call(cache=cache, cfg=cfg, lse=None, **kw):
        a = {**base, **kw}
        ckv.ckv_paged_attention(cfg, cache, a["table"], a["lens"], a["cu"], a["q"], a["out"], ws, lse=lse)

    call()
    for bad in (dict(table=base["table"].long()), dict(lens=dev([300])), dict(cu=dev([0, 1])),
                dict(q=c.q.float()), dict(out=torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda")),
                dict(cfg=config(8, 4)), dict(table=base["table"].reshape(-1)), dict(q=c.q.cpu()),
                dict(lse=torch.empty(8, 1, device="cuda"))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):
        ckv.PagedCache(c.k_pages, c.v_pages.float())
    with pytest.raises(ValueError):
        ckv.PagedCache(c.k_pages.transpose(1, 2), c.v_pages.transpose(1, 2))
    odd = torch.zeros((4, 24, 2, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ckv.CkvError, match="page_size"):
        call(cache=ckv.PagedCache(odd, odd))
