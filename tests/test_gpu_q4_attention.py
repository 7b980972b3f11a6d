"""ckv_paged_attention_q4 against a plain 64-bit attention over the values that the cache holds: the calls that
test_gpu_paged_attention.py makes of a bf16 cache, everything that is not a cached row NaN, and the whole way of a
prompt and its next tokens through the 4-bit cache."""
import math

import numpy as np
import pytest
import torch

import paper_2508_02401_gb300 as ckv
from tests import attention_ref as ref
from tests import kv4_ref
from tests.gpu_util import Guarded
from tests.test_gpu_paged_attention import CASES, Paged, dev
from tests.test_gpu_prefill_attention import config, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    ckv.load()


class Paged4(Paged):
    """The batch of Paged in 4 bits; k and v become what the cache holds."""

    def __init__(self, cfg, lens, new, page, seed=0, spread=0.0, **kw):
        super().__init__(cfg, lens, new, page, seed=seed, **kw)
        if spread:  # a few channels are far larger than the others, and rows differ in size
            g = torch.Generator(device="cuda").manual_seed(seed)
            f = torch.exp2(spread * torch.randn(128, generator=g, device="cuda"))
            for x in (self.k, self.v):
                for s in range(len(x)):
                    x[s] = (x[s] * f * torch.exp2(spread * torch.randn(x[s].shape[:2], generator=g, device="cuda"))[..., None]).to(torch.bfloat16)
            self.fill()
        self.hold()

    def fill(self):
        for s, n in enumerate(self.lens):
            j = torch.arange(n, device="cuda")
            p = dev(self.table[s], torch.int64)[j // self.page]
            self.k_pages[p, j % self.page], self.v_pages[p, j % self.page] = self.k[s], self.v[s]

    def hold(self):
        n, page, h, _ = self.k_pages.shape
        self.pages = torch.zeros((n, h, 2, page * 72), dtype=torch.uint8, device="cuda")
        slots = torch.arange(n * page, device="cuda")
        for i, x in enumerate((self.k_pages, self.v_pages)):
            kv4_ref.put(self.pages, page, slots, x.reshape(n * page, h, 128), i)
        for x in (self.k, self.v):
            if len(x):
                x[:] = kv4_ref.held(torch.cat(x)).split([len(y) for y in x])
        self.k_pages = self.v_pages = None

    def run(self, base=0, pad=0, status=(0, 0), q=None, ws=None, stream=None, **strides):
        cfg, hq = self.cfg, self.cfg.num_q_heads
        q = self.q if q is None else q
        out = Guarded((self.T, hq, 128), torch.bfloat16, 7.0)
        lse = Guarded((hq, self.T + pad), torch.float32, 7.0)
        ws = ckv.new_attention_workspace(cfg) if ws is None else ws
        ckv.ckv_paged_attention_q4(cfg, ckv.PagedCacheQ4(self.pages, self.page), dev(self.table), dev(self.lens),
                                   dev(self.cu + base), q, out.view, ws, lse=lse.view,
                                   lse_head_stride=self.T + pad if pad else 0, stream=stream, **strides)
        assert ckv.ckv_read_device_status(ws, stream=stream)[0] == status[0]
        out.check()
        lse.check()
        assert not bool(ws[256:1536].any())
        return out.view, lse.view

    def set_group(self, s, j, which, group, scale):
        """The scale word of a cached row's group, as it stands in the page."""
        page, row, P = int(self.table[s, j // self.page]), j % self.page, self.page
        at = 64 * P + row * 8 + group * 2
        self.pages[page, :, which, at:at + 2] = torch.tensor([scale & 255, scale >> 8], dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("case", range(len(CASES)))
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_lengths_and_pages(case, page):
    lens, new = CASES[case]
    hq, hkv = [(8, 2), (28, 4), (4, 4)][case % 3]
    Paged4(config(hq, hkv), lens, new, page, seed=case, pad=case % 3, extra_blocks=case % 2).check()


@pytest.mark.parametrize("hq,hkv,new", [(1, 1, 1), (6, 1, 3), (96, 1, 2), (256, 1, 1), (256, 2, 2), (15, 5, 9), (24, 2, 1),
                                        (9, 1, 1), (16, 1, 1), (16, 2, 2), (34, 2, 1)])
def test_unusual_groups(hq, hkv, new):
    Paged4(config(hq, hkv), (700, 131, 40), (new, new, new), 16, seed=5).check(pad=3)


@pytest.mark.parametrize("new", [1, 2, 3, 4, 5, 8, 9, 70])
@pytest.mark.parametrize("max_ctas", [0, 5])
def test_long_caches_are_cut_and_joined(new, max_ctas):
    Paged4(config(8, 2, max_ctas=max_ctas), (20011, 77, 9000), (new, new, 1), 64, seed=6).check()


@pytest.mark.parametrize("new", [1, 3, 200])
@pytest.mark.parametrize("spread", [1.5, 4.0])
def test_channels_and_rows_of_very_different_sizes(new, spread):
    """Scales over many powers of two, in a row, between rows and between K's and V's groups."""
    c = Paged4(config(8, 2), (1500, 300), (new, new), 32, seed=31, spread=spread)
    c.q = (c.q.float() * 2.0 ** (-2 * spread)).to(torch.bfloat16)  # (logits stay of a softmax's size)
    c.check()


@pytest.mark.parametrize("new", [1, 40])
def test_zero_points_at_the_ends(new):
    """Groups that are all positive or all negative: zero points of 0 and 15, codes at both ends."""
    c = Paged(config(8, 2), (900, 130), (new, 1), 64, seed=32)
    for i, x in enumerate((c.k, c.v)):
        for s in range(2):
            sign = torch.where(torch.arange(x[s].shape[0], device="cuda") % 2 == i, 1.0, -1.0)[:, None, None]
            x[s] = (x[s].abs() * sign * 0.5).to(torch.bfloat16)
    c.__class__ = Paged4
    c.fill()
    c.hold()
    c.check()


@pytest.mark.parametrize("new", [1, 70])
def test_nan_keys_in_one_part(new):
    """A stretch of NaN keys as long as a part of a cut unit makes the rows that see it NaN."""
    c = Paged4(config(8, 2), (9001, 500), (new, 1), 32, seed=17)
    block = c.pages[dev(c.table[0], torch.int64)[64:160], :, 0]
    block[..., 64 * 32:] = torch.tensor([0xC0, 0x7F], dtype=torch.uint8, device="cuda").repeat(32 * 4)
    c.pages[dev(c.table[0], torch.int64)[64:160], :, 0] = block
    out, lse = c.run()
    assert bool(out[:new].isnan().all()) and bool(lse[:, :new].isnan().all())
    assert not bool(out[new:].isnan().any()) and not bool(lse[:, new:].isnan().any())


@pytest.mark.parametrize("group", [0, 3])
def test_one_nan_group(group):
    """Of a key: every logit of it.  Of a value: the group's channels, in rows that see it."""
    c = Paged4(config(8, 2), (700, 300), (1, 1), 16, seed=33)
    want = [x.clone() for x in c.run()]
    c.set_group(0, 321, 1, group, 0x7FC0)
    out, lse = c.run()
    mine = torch.zeros(128, dtype=torch.bool, device="cuda")
    mine[32 * group:32 * group + 32] = True
    assert bool(out[0][:, mine].isnan().all()) and torch.equal(out[0][:, ~mine], want[0][0][:, ~mine])
    assert torch.equal(out[1], want[0][1]) and torch.equal(lse, want[1])
    c.set_group(0, 321, 0, group, 0x7FC0)
    out, lse = c.run()
    assert bool(out[0].isnan().all()) and bool(lse[:, 0].isnan().all())
    assert torch.equal(out[1], want[0][1]) and torch.equal(lse[:, 1], want[1][:, 1])


@pytest.mark.parametrize("singles", [0, 1])
@pytest.mark.parametrize("chunk", [1, 17, 40, 41, 42, 130, 300])
def test_a_chunk_among_single_tokens(chunk, singles):
    """Single tokens (or idle sequences) and a chunk in one call."""
    lens, new = [33 + 7 * i for i in range(40)] + [900], [singles] * 40 + [chunk]
    Paged4(config(8, 2), lens, new, 32, seed=19).check()


@pytest.mark.parametrize("hq,hkv", [(2, 2), (28, 4)])
@pytest.mark.parametrize("max_ctas", [0, 1, 5])
def test_key_tiles_of_one_row_tile(hq, hkv, max_ctas):
    """Chunks whose units' first row tile sees fewer key tiles than the second, and units that have one row tile."""
    c = Paged4(config(hq, hkv, max_ctas=max_ctas), (1500, 300, 2700, 129, 640), (257, 3, 300, 129, 100), 16, seed=23)
    out, lse = c.check()
    for _ in range(10):
        again = c.run()
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


@pytest.mark.parametrize("hq,hkv,new", [(8, 2, 1), (16, 2, 1), (8, 2, 2), (32, 2, 1)])
def test_units_end_to_end(hq, hkv, new):
    """Many short sequences a CTA, and the same bits each time."""
    g = np.random.default_rng(4)
    lens = [int(x) for x in g.integers(new, 900, 300)]
    c = Paged4(config(hq, hkv, max_ctas=9), lens, [new] * 300, 16, seed=34)
    out, lse = c.check()
    for _ in range(5):
        again = c.run()
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)


def test_many_sequences():
    """More sequences than the plan has threads, empty ones among them."""
    g = np.random.default_rng(3)
    lens = [int(x) for x in g.integers(0, 40, 1500)]
    new = [min(n, int(x)) for n, x in zip(lens, g.integers(0, 3, 1500))]
    Paged4(config(4, 1), lens, new, 16, seed=18, pad=3).check()


@pytest.mark.parametrize("new", [1, 2, 60])
def test_growing_maxima_over_the_cut(new):
    """Each key tile's logits above the last one's: every part of a cut unit has another reference."""
    c = Paged(config(8, 2), (9001,), (new,), 32, seed=7)
    c.__class__ = Paged4
    c.q = torch.ones_like(c.q)
    c.k[0] = (torch.arange(9001, device="cuda", dtype=torch.float32) / 256)[:, None, None].expand(9001, 2, 128).to(torch.bfloat16)
    c.fill()
    c.hold()
    c.check()


@pytest.mark.parametrize("new", [1, 40])
def test_logits_of_any_size(new):
    """Sharp softmaxes: a few keys carry all, the others' numerators vanish."""
    c = Paged4(config(8, 2), (3000, 260), (new, 1), 64, seed=35)
    c.q = (c.q.float() * 20).to(torch.bfloat16)
    c.check()
    c.q = torch.zeros_like(c.q)  # all keys alike
    c.check()


@pytest.mark.parametrize("scale", [0.01, 0.4])
@pytest.mark.parametrize("new", [1, 3, 40])
def test_a_given_scale(new, scale):
    c = Paged4(config(12, 2, softmax_scale=scale), (3000, 260), (new, 1), 32, seed=36)
    out, lse = c.run()
    for s, (L, n) in enumerate(zip(c.lens, c.new)):
        a = int(c.cu[s])
        o, l, tol, tol_l = ref.rows(c.q[a:a + n], c.k[s], c.v[s], torch.arange(L - n, L), scale)
        ref.assert_close(out[a:a + n], o, tol, f"out of sequence {s}")
        ref.assert_close(lse[:, a:a + n], l, tol_l, f"lse of sequence {s}")


def test_no_tokens():
    """Sequences without query rows: nothing is written, whatever their lengths."""
    c = Paged4(config(8, 2), (300, 0, 40), (0, 0, 0), 16, seed=37, pad=2)
    out, lse = c.run()
    assert bool((out == 7).all()) and bool((lse == 7).all())
    none = torch.zeros((0, 8, 128), dtype=torch.bfloat16, device="cuda")
    ws = ckv.new_attention_workspace(c.cfg)
    ckv.ckv_paged_attention_q4(c.cfg, ckv.PagedCacheQ4(c.pages, 16), dev(c.table), dev(c.lens), dev(c.cu), none, torch.empty_like(none), ws)
    assert ckv.ckv_read_device_status(ws) == (0, 0)


def test_offset_cu_and_strided_q():
    """cu_new as a slice of a longer array (it need not begin at 0), q inside a fused projection."""
    c = Paged4(config(8, 2), (300, 40, 513), (1, 7, 33), 32, seed=8)
    fused = torch.zeros((c.T, 12, 128), dtype=torch.bfloat16, device="cuda")
    fused[:, :8] = c.q
    c.check(base=1000)
    want = c.run()
    got = c.run(q=fused[:, :8], q_tok_stride=12 * 128)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    one = Paged4(config(8, 2), (300, 40, 513), (1, 1, 1), 32, seed=8)
    heads_first = one.q.transpose(0, 1).contiguous()  # [8, T, 128]
    got = one.run(q=heads_first.transpose(0, 1), q_tok_stride=128, q_head_stride=3 * 128)
    assert torch.equal(got[0], one.run()[0])


@pytest.mark.parametrize("new", [1, 50])
def test_strided_pages(new):
    """Pages with room behind each of them (layers side by side in one buffer)."""
    c = Paged4(config(8, 2), (300, 77), (new, 1), 32, seed=36)
    want = c.run()
    wide = torch.full((c.pages.shape[0], 3, *c.pages.shape[1:]), 0x7F, dtype=torch.uint8, device="cuda")
    wide[:, 1] = c.pages
    c.pages = wide[:, 1]
    got = c.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_pages_shared_by_two_sequences():
    """A common prefix: the same pages in both rows of the table."""
    c = Paged4(config(8, 2), (256, 300), (1, 1), 64, seed=10)
    c.table[0, :4] = c.table[1, :4]
    c.k[0], c.v[0] = c.k[1][:256], c.v[1][:256]
    c.check()


@pytest.mark.parametrize("new", [(1, 1), (1, 20)])
def test_offsets_beyond_32_bits(new):
    """Pages that lie beyond 2^32 bytes of the buffer, first and last ones."""
    page, hkv = 128, 8
    c = Paged4(config(32, hkv), (500, 900), new, page, seed=11)
    pages = (1 << 32) // (page * hkv * 144) + 9
    big = torch.zeros((pages, *c.pages.shape[1:]), dtype=torch.uint8, device="cuda")
    where = torch.tensor([pages - 1 - i if i % 2 else i for i in range(c.pages.shape[0])], device="cuda")
    big[where] = c.pages
    c.pages = big
    live = c.table >= 0
    c.table[live] = where.cpu().numpy()[c.table[live]]
    c.check()


@pytest.mark.parametrize("new", [1, 9])
def test_replayed_while_lengths_grow(new):
    """One captured call over device lengths: each replay sees the lengths of its time."""
    cfg = config(8, 2)
    c = Paged4(cfg, (520, 200), (new, new), 16, seed=12)
    ws, cache = ckv.new_attention_workspace(cfg), ckv.PagedCacheQ4(c.pages, 16)
    lens, cu, table, out = dev([new, new]), dev(c.cu), dev(c.table), torch.zeros_like(c.q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ckv.ckv_paged_attention_q4(cfg, cache, table, lens, cu, c.q, out, ws)
    for now in ([9, 10], [17, 129], [128, 200], [520, 16], [400, 199]):
        lens.copy_(dev(now))
        graph.replay()
        for s in range(2):
            o, _, tol, _ = ref.rows(c.q[new * s:new * (s + 1)], c.k[s][:now[s]], c.v[s][:now[s]], torch.arange(now[s] - new, now[s]))
            ref.assert_close(out[new * s:new * (s + 1)], o, tol, f"lengths {now}, sequence {s}")
    assert ckv.ckv_read_device_status(ws)[0] == 0


def test_same_results_on_another_stream_and_again():
    c = Paged4(config(8, 2), (5000, 77, 300), (1, 1, 40), 32, seed=13)
    d = Paged4(config(8, 2), (5000, 77, 300), (1, 1, 1), 32, seed=13)
    for x in (c, d):
        want = [y.clone() for y in x.run()]
        side, ws = torch.cuda.Stream(), ckv.new_attention_workspace(x.cfg)
        torch.cuda.synchronize()
        for _ in range(3):
            got = x.run(stream=side, ws=ws)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_calls_at_once():
    """Three streams, a workspace each: single tokens and chunks over 4 bits, an append into other pages beside them."""
    one, chunk = Paged4(config(8, 2), (5000, 77, 300), (1, 1, 1), 32, seed=25), Paged4(config(8, 2), (3000, 900), (300, 70), 32, seed=26)
    calls = []
    for c in (one, chunk):
        out = torch.zeros_like(c.q)
        calls.append((c, ckv.PagedCacheQ4(c.pages, 32), dev(c.table), dev(c.lens), dev(c.cu), out, ckv.new_attention_workspace(c.cfg),
                      torch.cuda.Stream(), c.run()[0].clone()))
    k, v, slots = normal(900, 2, 128, seed=1), normal(900, 2, 128, seed=2), dev(np.random.default_rng(1).permutation(960)[:900])
    rot, pos, ws, side = ckv.new_rotation(900), dev(np.arange(900)), ckv.new_attention_workspace(one.cfg), torch.cuda.Stream()
    cache = ckv.PagedCacheQ4(torch.zeros((30, 2, 2, 32 * 72), dtype=torch.uint8, device="cuda"), 32)
    torch.cuda.synchronize()
    for _ in range(60):
        for c, pages, t, n, cn, out, w, stream, _ in calls:
            ckv.ckv_paged_attention_q4(c.cfg, pages, t, n, cn, c.q, out, w, stream=stream)
        ckv.ckv_cache_append_q4(one.cfg, cache, k, v, slots, ws, rotation=rot, positions=pos, stream=side)
    torch.cuda.synchronize()
    for c, _, _, _, _, out, w, _, want in calls:
        assert torch.equal(out, want) and ckv.ckv_read_device_status(w) == (0, 0)
    assert ckv.ckv_read_device_status(ws) == (0, 0)
    want = torch.zeros_like(cache.pages)
    kv4_ref.put(want, 32, slots, kv4_ref.rotate(k, rot.cos_sin, pos), 0)
    kv4_ref.put(want, 32, slots, v, 1)
    assert torch.equal(cache.pages, want)


@pytest.mark.parametrize("new", [(1, 3, 2), (1, 1, 1), (1, 60, 70)])
@pytest.mark.parametrize("what", ["page", "negative", "short", "long", "decreasing", "past_the_end", "negative_cu"])
def test_bad_lengths_and_pages_are_reported(what, new):
    """Other sequences' rows are right all the same; nothing outside the outputs is touched."""
    c = Paged4(config(8, 2), (300, 200, 400), new, 32, seed=14)
    lens = list(c.lens)
    good = [0, 2]
    if what == "page":
        c.table[1, 3] = c.pages.shape[0]
    elif what == "negative":
        c.table[1, 0] = -5
    elif what == "short":
        c.lens[1] = new[1] - 1
    elif what == "long":
        c.lens[1] = 13 * 32 + 1
    else:  # rows that cannot be told apart: nothing is written
        i, x = dict(decreasing=(2, 0), past_the_end=(3, 5000), negative_cu=(1, -70))[what]
        c.cu[i] = x
        good = []
    rows = [(0, new[0]), (new[0], new[0] + new[1]), (new[0] + new[1], sum(new))]
    out, lse = c.run(status=(3, 0))
    if not good:
        assert bool((out == 7).all()) and bool((lse == 7).all())
    for s in good:  # (how a sequence is cut over CTAs, and so its last bits, depends on the others)
        a, b = rows[s]
        o, l, tol, tol_l = ref.rows(c.q[a:b], c.k[s], c.v[s], torch.arange(lens[s] - (b - a), lens[s]))
        ref.assert_close(out[a:b], o, tol, f"out of sequence {s}")
        ref.assert_close(lse[:, a:b], l, tol_l, f"lse of sequence {s}")


@pytest.mark.parametrize("hq,hkv,new", [(8, 2, 1), (8, 2, 3), (8, 2, 60), (28, 4, 300)])
@pytest.mark.parametrize("max_ctas", [0, 1])
@pytest.mark.parametrize("page", [16, 128])
def test_a_bad_page_reads_as_zeros(hq, hkv, new, max_ctas, page):
    """Bit for bit what a page of zero bytes gives, whatever was loaded before: the first and other sequences' rows are none of it."""
    c = Paged4(config(hq, hkv, max_ctas=max_ctas), (2900, 1300, 700), (new, new, 1), page, seed=38)
    c.pages = torch.cat([c.pages, torch.zeros_like(c.pages[:1])])
    last = c.pages.shape[0] - 1
    blocks = [0, 2, 5, 1300 // page] if page == 16 else [1, 4, 1300 // page]
    c.table[1, blocks] = last
    want = c.run()
    for bad in (last + 1, -1, 2 ** 31 - 1):
        c.table[1, blocks] = bad
        got = c.run(status=(3, 0))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    c = Paged4(config(8, 2), (300, 200), (1, 1), 32, seed=15)
    cfg, cache, ws = c.cfg, ckv.PagedCacheQ4(c.pages, 32), ckv.new_attention_workspace(c.cfg)
    base = dict(table=dev(c.table), lens=dev(c.lens), cu=dev(c.cu), q=c.q, out=torch.empty_like(c.q))

    def call(cache=cache, cfg=cfg, lse=None, **kw):
        a = {**base, **kw}
        ckv.ckv_paged_attention_q4(cfg, cache, a["table"], a["lens"], a["cu"], a["q"], a["out"], ws, lse=lse)

    call()
    bf = ckv.new_paged_cache(cfg, 30, 32)
    for bad in (dict(table=base["table"].long()), dict(lens=dev([300])), dict(cu=dev([0, 1])),
                dict(q=c.q.float()), dict(out=torch.empty(1, 8, 128, dtype=torch.bfloat16, device="cuda")),
                dict(cfg=config(8, 4)), dict(table=base["table"].reshape(-1)), dict(q=c.q.cpu()),
                dict(lse=torch.empty(8, 1, device="cuda")), dict(cache=bf)):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):  # a 4-bit cache in the bf16 call
        ckv.ckv_paged_attention(cfg, cache, base["table"], base["lens"], base["cu"], c.q, base["out"], ws)
    with pytest.raises(ckv.CkvError, match="page_size"):
        call(cache=ckv.PagedCacheQ4(torch.zeros((4, 2, 2, 24 * 72), dtype=torch.uint8, device="cuda"), 24))


@pytest.mark.parametrize("hq,hkv,interleaved", [(8, 2, False), (28, 4, True)])
def test_a_prompt_and_its_next_tokens(hq, hkv, interleaved):
    """Unrotated projections of two prompts -> rotation (into a bf16 cache beside) -> prefill attention -> compression with
    its lse -> the kept rows into 4 bits -> three decode steps: tables, append, attention."""
    lens, w, budget, page = (700, 260), 32, 150, 16
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T, S = int(cu[-1]), len(lens)
    cfg = ckv.Config(num_layers=1, num_q_heads=hq, num_kv_heads=hkv, window=w, pool_kernel=5, pool_type=ckv.POOL_MAX,
                     head_order=ckv.POOL_THEN_SUM, head_mask=np.ones((1, hq), np.uint8), budgets=np.array([budget], np.int32))
    rot = ckv.new_rotation(2000, 500000.0, interleaved=interleaved)
    qkv = normal(T, hq + 2 * hkv, 128, seed=40)
    q0, k0, v0 = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    pos = dev(np.concatenate([np.arange(n) for n in lens]))
    ws = ckv.new_attention_workspace(cfg)
    q, k = torch.zeros(T, hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, hkv, 128, dtype=torch.bfloat16, device="cuda")
    full = ckv.new_paged_cache(cfg, -(-T // page), page)
    ckv.ckv_cache_append(cfg, full, k0, v0, dev(np.arange(T)), rot, pos, ws, q=q0, q_out=q, k_out=k,
                         tok_stride=(hq + 2 * hkv) * 128, q_tok_stride=(hq + 2 * hkv) * 128)
    assert torch.equal(k, kv4_ref.rotate(k0, rot.cos_sin, pos, interleaved)) and torch.equal(full.k_pages.view(-1, hkv, 128)[:T], k)
    v = v0.contiguous()
    att, lse_win = torch.zeros_like(q), torch.zeros((hq, S * w), device="cuda")
    batch = ckv.Batch(cu)
    ckv.ckv_prefill_attention(cfg, batch, q, k, v, att, ws, lse_win=lse_win)
    q_win = torch.stack([q[int(cu[s + 1]) - w:int(cu[s + 1])] for s in range(S)])
    idx, cu_keep_dev, k_kept, v_kept, cu_keep = ckv.new_outputs(cfg, 0, batch)
    cws = ckv.new_workspace(cfg, 0, batch)
    ckv.ckv_compress_layer_lse(cfg, 0, batch, q_win, k, v, lse_win, idx, cu_keep_dev, k_kept, v_kept, cws)
    pages, i32 = 60, dict(dtype=torch.int32, device="cuda")
    cache = ckv.new_paged_cache_q4(cfg, pages, page)
    held, ring = torch.zeros(S, **i32), torch.randperm(pages, device="cuda").to(torch.int32)
    pool, table = torch.tensor([0, pages], dtype=torch.int64, device="cuda"), torch.zeros((S, 20), **i32)
    keep = torch.diff(cu_keep_dev)
    slots, cu_new = torch.zeros(int(cu_keep[-1]), **i32), torch.zeros(S + 1, **i32)
    ckv.ckv_block_tables(page, held, keep, ring, pool, table, slots, cu_new, held, pool, ws)
    ckv.ckv_cache_append_q4(cfg, cache, k_kept, v_kept, slots, ws)
    rows_k = [kv4_ref.held(k_kept[int(cu_keep[s]):int(cu_keep[s + 1])]) for s in range(S)]
    rows_v = [kv4_ref.held(v_kept[int(cu_keep[s]):int(cu_keep[s + 1])]) for s in range(S)]
    for step, n in enumerate((1, 1, 3)):
        new = normal(S * n, hq + 2 * hkv, 128, seed=50 + step)
        qn, kn, vn = new[:, :hq], new[:, hq:hq + hkv], new[:, hq + hkv:]
        at = dev(np.concatenate([m + step + np.arange(n) for m in lens]))  # the tokens' own positions, not the cache's
        slots, cu_new = torch.zeros(S * n, **i32), torch.zeros(S + 1, **i32)
        ckv.ckv_block_tables(page, held, torch.full((S,), n, **i32), ring, pool, table, slots, cu_new, held, pool, ws)
        q_rot, out = torch.zeros(S * n, hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(S * n, hq, 128, dtype=torch.bfloat16, device="cuda")
        ckv.ckv_cache_append_q4(cfg, cache, kn, vn, slots, ws, rotation=rot, positions=at, q=qn, q_out=q_rot,
                                tok_stride=(hq + 2 * hkv) * 128, q_tok_stride=(hq + 2 * hkv) * 128)
        ckv.ckv_paged_attention_q4(cfg, cache, table, held, cu_new, q_rot, out, ws)
        assert ckv.ckv_read_device_status(ws) == (0, 0)
        assert torch.equal(q_rot, kv4_ref.rotate(qn, rot.cos_sin, at, interleaved))
        hk, hv = kv4_ref.held(kv4_ref.rotate(kn, rot.cos_sin, at, interleaved)), kv4_ref.held(vn)
        for s in range(S):
            rows_k[s], rows_v[s] = torch.cat([rows_k[s], hk[s * n:s * n + n]]), torch.cat([rows_v[s], hv[s * n:s * n + n]])
            L = len(rows_k[s])
            assert int(held[s]) == L
            o, _, tol, _ = ref.rows(q_rot[s * n:s * n + n], rows_k[s], rows_v[s], torch.arange(L - n, L))
            ref.assert_close(out[s * n:s * n + n], o, tol, f"step {step}, sequence {s}")
