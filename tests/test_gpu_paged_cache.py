"""ckv_block_tables and ckv_cache_write against plain Python, and a decode loop that runs the whole way:
prefill attention, compression with its lse, tables, rows into the cache, attention of new tokens."""
import math

import numpy as np
import pytest
import torch

import oracle
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
    oracle.build()


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


class Tables:
    """The tables on the GPU beside a plain allocator that does the same."""

    def __init__(self, rows, pages, blocks, page, seed=0, start=0):
        g = np.random.default_rng(seed)
        self.page, self.lens = page, np.zeros(rows, np.int64)
        self.ring = np.roll(g.permutation(pages), start % pages).astype(np.int64)
        self.pool = np.array([start, start + pages], np.int64)
        self.table = np.full((rows, blocks), -9, np.int64)
        self.d = dict(lens=dev(self.lens), ring=dev(self.ring), pool=dev(self.pool, torch.int64),
                      table=dev(self.table))
        self.ws = ckv.new_attention_workspace(config())

    def plain(self, new, cap):
        page, n_pages = self.page, len(self.ring)
        have, add = -(-self.lens // page), np.maximum(new, 0)
        want = -(-(self.lens + add) // page)
        slots, cu = np.full(cap, -1), np.concatenate([[0], np.cumsum(add)])
        if (self.lens + add > self.table.shape[1] * page).any() or (new < -1).any():
            why = 1
        elif cu[-1] > cap:
            why = 2
        elif (want - have).sum() > self.pool[1] - self.pool[0]:
            why = 4
        else:
            why = 0
            taken, back = self.pool
            for r, n in enumerate(new):
                if n < 0:
                    for b in range(have[r]):
                        self.ring[back % n_pages] = self.table[r, b]
                        back += 1
                    self.lens[r] = 0
                    continue
                for b in range(have[r], want[r]):
                    self.table[r, b] = self.ring[taken % n_pages]
                    taken += 1
                for i in range(n):
                    pos = self.lens[r] + i
                    slots[cu[r] + i] = self.table[r, pos // page] * page + pos % page
                self.lens[r] += n
            self.pool = np.array([taken, back])
        return slots, cu if not why else np.zeros_like(cu), why

    def step(self, new, cap=None, in_place=True):
        new = np.asarray(new)
        cap = int(np.maximum(new, 0).sum()) + 3 if cap is None else cap
        slots, cu, why = self.plain(new, cap)
        g_slots, g_cu = Guarded((cap,), torch.int32, -77), Guarded((len(new) + 1,), torch.int32, -77)
        d = self.d
        lens_out, pool_out = (d["lens"], d["pool"]) if in_place else (torch.zeros_like(d["lens"]), torch.zeros_like(d["pool"]))
        before = d["lens"].clone()
        ckv.ckv_block_tables(self.page, d["lens"], dev(new), d["ring"], d["pool"], d["table"], g_slots.view,
                             g_cu.view, lens_out, pool_out, self.ws)
        code, detail = ckv.ckv_read_device_status(self.ws)
        assert (code, detail) == ((5, why) if why else (0, 0))
        g_slots.check()
        g_cu.check()
        if not in_place:
            assert torch.equal(d["lens"], before)
            d["lens"], d["pool"] = lens_out, pool_out
        for name, got, want in (("slots", g_slots.view, slots), ("cu", g_cu.view, cu), ("lens", d["lens"], self.lens),
                                ("pool", d["pool"], self.pool), ("table", d["table"], self.table),
                                ("ring", d["ring"], self.ring)):
            np.testing.assert_array_equal(got.cpu().numpy(), want, err_msg=name)
        assert not bool(self.ws.any())
        return g_slots.view, g_cu.view


@pytest.mark.parametrize("rows,page", [(1, 16), (3, 32), (40, 64), (1500, 16), (5000, 128)])
@pytest.mark.parametrize("in_place", [True, False])
def test_steps_of_a_serving_loop(rows, page, in_place):
    """Admission, single tokens, chunks, rows given back and admitted anew, over and over."""
    g = np.random.default_rng(rows)
    t = Tables(rows, rows * (600 // page + 2), 600 // page + 1, page, seed=rows, start=(1 << 33) + 5)
    t.step(g.integers(0, 200, rows), in_place=in_place)
    for i in range(8):
        new = np.ones(rows, int) if i % 3 else g.integers(0, 40, rows)
        if i % 2:
            new[g.random(rows) < 0.2] = -1
        t.step(new, in_place=in_place)
    t.step(np.full(rows, -1), in_place=in_place)
    t.step(np.zeros(rows, int), cap=0, in_place=in_place)
    t.step(np.full(rows, 5), in_place=in_place)


def test_long_rows_over_many_ctas():
    t = Tables(3, 20000, 16000, 16, seed=1)
    t.step([200001, 0, 17])
    t.step([1, 40000, 50000])
    t.step([-1, 1, -1])
    t.step([0, 1, 100000])


def test_what_does_not_fit_changes_nothing():
    t = Tables(4, 10, 8, 16, seed=2)
    t.step([16, 20, 0, 1])
    t.step([1, 200, 1, 1])            # a row longer than its table
    t.step([1, 1, 1, 1], cap=3)       # more tokens than the slot map
    t.step([60, 60, 60, 60])          # more pages than are free
    t.step([1, -2, 1, 1])             # no such command
    t.step([40, 1, 1, 1])
    # pages given back in a call are not handed out in it
    t.step([128 - 56, -1, 1, 1])
    t.step([1, 1, 1, 1])


def test_bad_lengths_counters_and_pages():
    t = Tables(2, 10, 8, 16, seed=3)
    d, ws = t.d, t.ws
    slots, cu = torch.zeros(8, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")

    def call(lens, new, pool, ring=d["ring"]):
        lens, pool = dev(lens), dev(pool, torch.int64)
        was = lens.clone(), pool.clone()
        ckv.ckv_block_tables(16, lens, dev(new), ring, pool, d["table"], slots, cu, lens, pool, ws)
        return ckv.ckv_read_device_status(ws), bool((lens == was[0]).all()) and bool((pool == was[1]).all())

    assert call([-1, 5], [1, 1], [0, 10]) == ((5, 1), True)
    assert call([0, 5], [1, 2 ** 31 - 1], [0, 10]) == ((5, 1), True)
    assert call([0, 0], [1, 1], [5, 3]) == ((5, 3), True)
    assert call([0, 0], [1, 1], [0, 11]) == ((5, 3), True)
    assert call([0, 40], [1, -1], [0, 10]) == ((5, 3), True)   # more pages given back than there are
    assert call([0, 0], [1, 1], [10, 10]) == ((5, 4), True)
    assert bool((slots == -1).all()) and not bool(cu.any())
    (code, _), same = call([0, 0], [1, 1], [0, 10], ring=dev([10, 3, -1, 4, 5, 6, 7, 8, 9, 0]))
    assert code == 3 and not same and slots[:3].tolist() == [-1, 48, -1]


def test_bad_pages_given_back():
    """Table entries outside the cache are reported with their row when the row is given back, and -1 is in the ring in
    their place."""
    t = Tables(3, 10, 8, 16, seed=5)
    d, ws = t.d, t.ws
    slots, cu = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    ring, pool, lens = dev([0, 0, 0, 0, 7, 8, 0, 0, 0, 0]), dev([4, 6], torch.int64), dev([16, 40, 0])
    d["table"][0, 0] = 5
    d["table"][1, :3] = dev([2, -1, 10])

    def call(new):
        ckv.ckv_block_tables(16, lens, dev(new), ring, pool, d["table"], slots, cu, lens, pool, ws)
        return ckv.ckv_read_device_status(ws)

    assert call([-1, -1, 1]) == (3, 1)
    assert ring[4:].tolist() == [7, 8, 5, 2, -1, -1] and pool.tolist() == [5, 10] and lens.tolist() == [0, 0, 1]
    assert slots[:2].tolist() == [7 * 16, -1]
    assert call([48, 0, 15]) == (0, 0)  # pages 8, 5 and 2
    assert call([0, 1, 0]) == (3, 1) and slots[:2].tolist() == [-1, -1]  # the first of the bad ones


def test_tables_replayed_in_a_graph():
    """The step of a decode loop, captured once: lengths, counters and tables move on the device."""
    t = Tables(6, 200, 20, 16, seed=4)
    t.step([5, 16, 31, 0, 100, 64])
    d = t.d
    ones, slots, cu = dev([1] * 6), torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(7, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ckv.ckv_block_tables(16, d["lens"], ones, d["ring"], d["pool"], d["table"], slots, cu, d["lens"], d["pool"], t.ws)
    for _ in range(40):
        graph.replay()
        want, _, _ = t.plain(np.ones(6, int), 6)
        np.testing.assert_array_equal(slots.cpu().numpy(), want)
        np.testing.assert_array_equal(d["table"].cpu().numpy(), t.table)


@pytest.mark.parametrize("tokens,hkv,page", [(1, 1, 16), (3, 2, 16), (65, 8, 64), (1000, 4, 32), (257, 5, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_cache_write(tokens, hkv, page, interleaved):
    g = np.random.default_rng(tokens)
    pages = tokens // page + 3
    slots = g.permutation(pages * page)[:tokens]
    slots[::5] = -1
    src = normal(tokens, 2, hkv, 128, seed=1)
    k, v = (src[:, 0], src[:, 1]) if interleaved else (src[:, 0].contiguous(), src[:, 1].contiguous())
    shape = (pages, 2, page, hkv, 128)
    if interleaved:
        g_kv = [Guarded(shape, torch.bfloat16, 3.0)]
        kp, vp = g_kv[0].view[:, 0], g_kv[0].view[:, 1]
    else:
        g_kv = [Guarded((pages, page, hkv, 128), torch.bfloat16, 3.0) for _ in range(2)]
        kp, vp = g_kv[0].view, g_kv[1].view
    cfg = config(hkv, hkv)
    ws = ckv.new_attention_workspace(cfg)
    ckv.ckv_cache_write(cfg, ckv.PagedCache(kp, vp), k, v, dev(slots), ws, tok_stride=2 * hkv * 128 if interleaved else 0)
    assert ckv.ckv_read_device_status(ws) == (0, 0)
    for guard in g_kv:
        guard.check()
    for got, x in ((kp, k), (vp, v)):
        want = torch.full((pages * page, hkv, 128), 3.0, dtype=torch.bfloat16, device="cuda")
        live = dev(slots, torch.int64) >= 0
        want[dev(slots, torch.int64)[live]] = x[live]
        assert torch.equal(got.reshape(-1, hkv, 128), want)


def test_cache_write_skips_slots_outside_the_cache():
    cfg = config(2, 2)
    k, v = normal(4, 2, 128, seed=1), normal(4, 2, 128, seed=2)
    kp, vp = Guarded((2, 16, 2, 128), torch.bfloat16, 3.0), Guarded((2, 16, 2, 128), torch.bfloat16, 3.0)
    ws = ckv.new_attention_workspace(cfg)
    ckv.ckv_cache_write(cfg, ckv.PagedCache(kp.view, vp.view), k, v, dev([32, 5, -7, 2 ** 31 - 1]), ws)
    assert ckv.ckv_read_device_status(ws)[0] == 3
    kp.check()
    vp.check()
    assert torch.equal(kp.view.reshape(32, 2, 128)[5], k[1])
    assert int((kp.view.reshape(32, -1) != 3).any(1).sum()) == 1


def test_refusals():
    cfg, ws = config(2, 2), ckv.new_attention_workspace(config(2, 2))
    k = normal(4, 2, 128)
    pages = torch.zeros((2, 16, 2, 128), dtype=torch.bfloat16, device="cuda")
    cache = ckv.PagedCache(pages, pages.clone())
    for bad in (dict(k=k[:3]), dict(k=k.float()), dict(slots=dev([1, 2, 3, 4], torch.int64)), dict(cfg=config(4, 4)),
                dict(v=k[:, :1])):
        a = dict(k=k, v=k, slots=dev([1, 2, 3, 4]), cfg=cfg)
        a.update(bad)
        with pytest.raises(ValueError):
            ckv.ckv_cache_write(a["cfg"], cache, a["k"], a["v"], a["slots"], ws)
    t = Tables(2, 10, 8, 16)
    d, i = t.d, torch.int32
    good = dict(lens=d["lens"], new=dev([1, 1]), ring=d["ring"], pool=d["pool"], table=d["table"],
                slots=torch.zeros(2, dtype=i, device="cuda"), cu=torch.zeros(3, dtype=i, device="cuda"))
    for bad in (dict(new=dev([1])), dict(new=dev([1, 1], torch.int64)), dict(pool=dev([0, 10])), dict(cu=dev([0, 0])),
                dict(table=d["table"][:1]), dict(ring=d["ring"].cpu()), dict(table=d["table"][:, ::2])):
        a = {**good, **bad}
        with pytest.raises(ValueError):
            ckv.ckv_block_tables(16, a["lens"], a["new"], a["ring"], a["pool"], a["table"], a["slots"], a["cu"],
                                 a["lens"], a["pool"], ws)


def test_pages_that_overlap_are_refused():
    """Pages expanded over the first dimension, or less than a page apart: the rows that a call of such strides would
    reach are not there."""
    one = torch.zeros((1, 16, 2, 128), dtype=torch.bfloat16, device="cuda")
    assert ckv.PagedCache(one, one.clone()).num_pages == 1
    for pages in (one.expand(4, 16, 2, 128), one.as_strided((2, 8, 2, 128), (2048 - 256, 256, 128, 1)),
                  one.as_strided((2, 8, 2, 128), (256, 256, 128, 1))):
        with pytest.raises(ValueError, match="page"):
            ckv.PagedCache(pages, pages)


@pytest.mark.parametrize("hq,hkv,page,lens", [(8, 2, 16, (300, 40, 700)), (28, 4, 32, (513, 1000))])
def test_prefill_compress_cache_decode(hq, hkv, page, lens):
    """Two layers of different budgets over one pool of pages: the prefill attention's window lse feeds
    the compression, the kept rows go to the pages, and captured decode steps answer over them."""
    layers, w, steps = 2, 32, 20
    budgets = np.array([48, 130], np.int32)
    mask = np.zeros((layers, hq), np.uint8)
    mask[:, ::hq // hkv] = 1
    cfg = ckv.Config(num_layers=layers, num_q_heads=hq, num_kv_heads=hkv, window=w, pool_kernel=7,
                     pool_type=ckv.POOL_MAX, head_order=ckv.POOL_THEN_SUM, head_mask=mask, budgets=budgets)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    S, T = len(lens), int(cu[-1])
    batch, ws = ckv.Batch(cu), ckv.new_attention_workspace(cfg)
    kept, keeps = [], []
    for l in range(layers):
        q, k, v = (normal(T, h, 128, seed=10 * l + i) for i, h in enumerate((hq, hkv, hkv)))
        out, lse_win = torch.zeros_like(q), torch.zeros((hq, S * w), device="cuda")
        ckv.ckv_prefill_attention(cfg, batch, q, k, v, out, ws, lse_win=lse_win)
        for s in range(S):
            a, b = int(cu[s]), int(cu[s + 1])
            o, _, tol, _ = ref.rows(q[a:b], k[a:b], v[a:b], torch.arange(b - a))
            ref.assert_close(out[a:b], o, tol, f"prefill, layer {l}, sequence {s}")
        q_win = torch.stack([q[int(e) - w:int(e)] for e in cu[1:]])
        cws = ckv.new_workspace(cfg, l, batch)
        got = []
        for given in (True, False):
            idx, ck, ko, vo, cu_keep = ckv.new_outputs(cfg, l, batch)
            pooled = torch.zeros((hkv, T), device="cuda")
            if given:
                ckv.ckv_compress_layer_lse(cfg, l, batch, q_win, k, v, lse_win, idx, ck, ko, vo, cws, pooled_out=pooled)
            else:
                ckv.ckv_compress_layer(cfg, l, batch, q_win, k, v, idx, ck, ko, vo, cws, pooled_out=pooled)
            assert ckv.ckv_read_device_status(cws)[0] == 0
            got.append((idx, ko, vo, pooled))
        # the same pooled scores with the attention's lse as with the scoring's own: |lse error| <= 1e-3
        # would change a probability by 1e-3 of it
        assert torch.allclose(got[0][3], got[1][3], rtol=2e-3, atol=1e-9)
        kept.append(got[0][1:3])
        keeps.append(np.diff(cu_keep))
    # pages for every layer's rows, and the kept rows in them
    rows, pages = layers * S, 200
    blocks = 16
    d = dict(lens=dev(np.zeros(rows)), ring=dev(np.random.default_rng(1).permutation(pages)),
             pool=dev([0, pages], torch.int64), table=dev(np.zeros((rows, blocks))))
    cache = ckv.new_paged_cache(cfg, pages, page)
    cache.k_pages.fill_(math.nan)
    cache.v_pages.fill_(math.nan)
    admit, total = np.concatenate(keeps), int(np.concatenate(keeps).sum())
    slots, cu_new = torch.zeros(total, dtype=torch.int32, device="cuda"), torch.zeros(rows + 1, dtype=torch.int32, device="cuda")
    ckv.ckv_block_tables(page, d["lens"], dev(admit), d["ring"], d["pool"], d["table"], slots, cu_new, d["lens"],
                         d["pool"], ws)
    at = 0
    for l in range(layers):
        n = int(keeps[l].sum())
        ckv.ckv_cache_write(cfg, cache, kept[l][0], kept[l][1], slots[at:at + n], ws)
        at += n
    # a decode step of both layers, captured once
    nq, nk, nv = (torch.zeros((layers, S, h, 128), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    out, ones = torch.zeros((layers, S, hq, 128), dtype=torch.bfloat16, device="cuda"), dev(np.ones(rows))
    step_slots, step_cu = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows + 1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ckv.ckv_block_tables(page, d["lens"], ones, d["ring"], d["pool"], d["table"], step_slots, step_cu, d["lens"],
                             d["pool"], ws)
        for l in range(layers):
            sl = slice(l * S, (l + 1) * S)
            ckv.ckv_cache_write(cfg, cache, nk[l], nv[l], step_slots[sl], ws)
            ckv.ckv_paged_attention(cfg, cache, d["table"][sl], d["lens"][sl], step_cu[l * S:(l + 1) * S + 1], nq[l],
                                    out[l], ws)
    keys = [[(k[int(a):int(b)], v[int(a):int(b)]) for a, b in zip(c, c[1:])]
            for (k, v), c in ((kept[l], np.concatenate([[0], np.cumsum(keeps[l])])) for l in range(layers))]
    for step in range(steps):
        for x, h in ((nq, hq), (nk, hkv), (nv, hkv)):
            x.copy_(normal(layers, S, h, 128, seed=100 * step + h))
        graph.replay()
        for l in range(layers):
            for s in range(S):
                keys[l][s] = (torch.cat([keys[l][s][0], nk[l, s:s + 1]]), torch.cat([keys[l][s][1], nv[l, s:s + 1]]))
                kk, vv = keys[l][s]
                o, _, tol, _ = ref.rows(nq[l, s:s + 1], kk, vv, torch.tensor([len(kk) - 1]))
                ref.assert_close(out[l, s:s + 1], o, tol, f"step {step}, layer {l}, sequence {s}")
    assert ckv.ckv_read_device_status(ws) == (0, 0)
    assert d["lens"].tolist() == [int(n) + steps for n in admit]
