"""ckv_cache_append and ckv_cache_append_q4, bit for bit against the rotation in 64 bits and the rows in 4 bits by their
definition: every pairing and width, head counts, strided and in-place rows, tokens without a slot or a position, groups of
every kind, bad slots and positions, captured calls, offsets beyond 32 bits."""
import math

import numpy as np
import pytest
import torch

import paper_2508_02401_gb300 as ckv
from tests import kv4_ref
from tests.gpu_util import Guarded
from tests.test_gpu_prefill_attention import config, normal
from tests.test_kv4_ref_cpu import far_apart

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    ckv.load()


def dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


def same(got, want, what=""):
    """Bit for bit (any NaN for a NaN)."""
    eq = (got == want) | (got.isnan() & want.isnan()) if got.is_floating_point() else got == want
    assert bool(eq.all()), f"{what}: {int((~eq).sum())} of {eq.numel()} differ, first at {(~eq).nonzero()[0].tolist()}"


class Append:
    """A call's inputs; q4 or bf16 cache."""

    def __init__(self, T, hq=8, hkv=2, page=16, q4=False, rd=128, interleaved=False, fused=False, skip=0, span=5000, seed=0,
                 queries=True, base=10000.0):
        self.T, self.hq, self.hkv, self.page, self.q4, self.rd = T, hq, hkv, page, q4, rd
        self.cfg, self.interleaved, self.fused = config(hq, hkv), interleaved, fused
        g = np.random.default_rng(seed)
        if fused:
            both = normal(T, hq + 2 * hkv, 128, seed=seed + 1)
            self.q, self.k, self.v = both[:, :hq], both[:, hq:hq + hkv], both[:, hq + hkv:]
            self.strides = dict(tok_stride=(hq + 2 * hkv) * 128)
        else:
            self.q, self.k, self.v = normal(T, hq, 128, seed=seed + 1), normal(T, hkv, 128, seed=seed + 2), normal(T, hkv, 128, seed=seed + 3)
            self.strides = {}
        if not queries:
            self.q = None
        elif fused:
            self.strides["q_tok_stride"] = self.strides["tok_stride"]
        self.num_pages = -(-max(T, 1) // page) + 3
        slots = g.permutation(self.num_pages * page)[:T]
        if skip:
            slots[::skip] = -1
        self.slots = dev(slots)
        self.rot = ckv.new_rotation(span, base, rd, interleaved) if rd else None
        self.positions = dev(g.integers(0, span, T)) if rd else None
        self.ws = ckv.new_attention_workspace(self.cfg)

    def empty_cache(self):
        n, p, h = self.num_pages, self.page, self.hkv
        if self.q4:
            return Guarded((n, h, 2, p * 72), torch.uint8, 0xA5)
        return Guarded((n, 2, p, h, 128), BF, 7.0)

    def run(self, outs=True, status=(0, 0), inplace=False, stream=None, **kw):
        pages = self.empty_cache()
        cache = ckv.PagedCacheQ4(pages.view, self.page) if self.q4 else ckv.PagedCache(pages.view[:, 0], pages.view[:, 1])
        args = dict(self.strides, **kw)
        buf = {}
        if outs:
            buf["k_out"] = Guarded((self.T, self.hkv, 128), BF, 9.0)
            if self.q4:
                buf["v_out"] = Guarded((self.T, self.hkv, 128), BF, 9.0)
        k, v, q = self.k, self.v, self.q
        if self.q is not None:
            buf["q_out"] = Guarded((self.T, self.hq, 128), BF, 9.0)
        if inplace:
            for name, x in (("k_out", k), ("v_out", v), ("q_out", q)):
                if name in buf:
                    buf[name].view.copy_(x)
            k, q = buf["k_out"].view, buf["q_out"].view
            v = buf["v_out"].view if self.q4 else v
        args.update({n: b.view for n, b in buf.items()})
        if self.q is not None:
            args["q"] = q
        if self.q4:
            ckv.ckv_cache_append_q4(self.cfg, cache, k, v, self.slots, self.ws, rotation=self.rot, positions=self.positions,
                                    stream=stream, **args)
        else:
            ckv.ckv_cache_append(self.cfg, cache, k, v, self.slots, self.rot, self.positions, self.ws, stream=stream, **args)
        assert ckv.ckv_read_device_status(self.ws, stream=stream) == status
        pages.check()
        for b in buf.values():
            b.check()
        return pages.view, {n: b.view for n, b in buf.items()}

    def check(self, done=None, **kw):
        """`done`: the tokens that the call does something for (all)."""
        pages, out = self.run(**kw)
        want = self.empty_cache().view
        done = torch.ones(self.T, dtype=torch.bool, device="cuda") if done is None else done
        pos = torch.where(done, self.positions, 0) if self.rd else None
        turn = (lambda x: kv4_ref.rotate(x, self.rot.cos_sin, pos, self.interleaved)) if self.rd else (lambda x: x)
        k, v = turn(self.k), self.v.contiguous()
        n = self.num_pages * self.page
        slots = torch.where(done & (self.slots >= 0) & (self.slots < n), self.slots, -1)
        if self.q4:
            kv4_ref.put(want, self.page, slots, k, 0)
            kv4_ref.put(want, self.page, slots, v, 1)
            k, v = kv4_ref.held(k), kv4_ref.held(v)
        else:
            t = (slots >= 0).nonzero()[:, 0]
            for i, x in enumerate((k, v)):
                want[slots[t].long() // self.page, i, slots[t].long() % self.page] = x[t]
        same(pages, want, "pages")
        if self.q is not None:
            same(out["q_out"][done], turn(self.q)[done], "q_out")
        for name, x in (("k_out", k), ("v_out", v)):
            if name in out:
                same(out[name][done], x[done], name)
                assert bool((out[name][~done] == 9).all())
        return pages, out


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 33, 1000])
@pytest.mark.parametrize("page", [16, 128])
def test_lengths(T, page, q4):
    Append(T, page=page, q4=q4, seed=T, fused=T % 2 == 1, skip=3 if T == 33 else 0).check()


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("rd", [16, 32, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(rd, interleaved, q4):
    Append(60, hq=12, hkv=3, rd=rd, interleaved=interleaved, q4=q4, page=32, seed=rd).check()


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("hq,hkv", [(32, 8), (28, 4), (1, 1), (5, 5), (256, 2), (6, 3), (7, 1)])
def test_heads(hq, hkv, q4):
    Append(40, hq=hq, hkv=hkv, q4=q4, page=64, seed=hq, fused=True, skip=7).check()


@pytest.mark.parametrize("q4", [False, True])
def test_without_queries_or_outputs(q4):
    Append(100, q4=q4, queries=False, seed=4).check()
    Append(100, q4=q4, queries=False, seed=5).check(outs=False)


@pytest.mark.parametrize("skip", [0, 2])
def test_rows_that_are_rotated_already(skip):
    Append(300, q4=True, rd=0, queries=False, skip=skip, seed=6).check()


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_in_place(q4, interleaved):
    a = Append(77, hq=9, hkv=3, q4=q4, interleaved=interleaved, rd=96, seed=7)
    a.check(inplace=True)


@pytest.mark.parametrize("q4", [False, True])
def test_far_positions_and_many_rows(q4):
    """A sum that fp32 would round to another bf16 number is found among so many."""
    Append(20000, hq=8, hkv=4, q4=q4, seed=8, span=131072, base=500000.0).check()


@pytest.mark.parametrize("q4", [False, True])
def test_sums_that_cancel(q4):
    """a cos - b sin near zero, and near ties of bf16: b is a cos / sin rounded, so the difference is all rounding."""
    a = Append(4000, hq=2, hkv=2, q4=q4, seed=9)
    c, s = (x[:, None] for x in a.rot.cos_sin.double()[a.positions.long()].split(64, 1))
    for x in (a.q, a.k):
        x[..., 64:] = (x[..., :64].double() * c / s).clamp(-1e4, 1e4).to(BF)
    a.check()


@pytest.mark.parametrize("q4", [False, True])
def test_sums_next_to_a_tie(q4):
    """c - b s with c a tie of bf16 and b s = +-2^-24 (1 + 127 / 2^31): by 2^-48 past what would still round to the tie in 32 bits.
    From 1 + 2^-8 the sum above goes up, from 1 + 3 2^-8 (whose even neighbour is the upper one) the sum below goes down."""
    a = Append(64, hq=4, hkv=2, q4=q4, seed=20)
    a.rot.cos_sin[:, :64] = 1 + 2.0 ** -8 * torch.where(torch.arange(64, device="cuda") % 4 < 2, 1.0, 3.0)
    a.rot.cos_sin[:, 64:] = 8421505 * 2.0 ** -48  # 255 * 8421505 = 2^31 + 127
    b = 255 / 128 * torch.where(torch.arange(64, device="cuda") % 2 == 0, 1.0, -1.0)
    for x in (a.q, a.k):
        x[..., :64], x[..., 64:] = 1.0, b
        x[::2] = x[::2].roll(64, -1)
    a.check()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("low,high", [(-110, -90), (-130, -110), (-140, -125)])
def test_tiny_rows(low, high, interleaved):
    """Products and sums that fp32 has as subnormal numbers, results that bf16 has as such."""
    a = Append(6000, hq=8, hkv=4, seed=21, interleaved=interleaved)
    g = torch.Generator(device="cuda").manual_seed(22)
    for x in (a.q, a.k):
        x.copy_((x.double() * torch.exp2(torch.randint(low, high, (*x.shape[:2], 1), generator=g, device="cuda").double())).to(BF))
    a.check()


def test_rows_with_zeros():
    """Rows, words and single pairs of zeros."""
    a = Append(200, hq=4, hkv=2, seed=24)
    for x in (a.q, a.k):
        x[::4] = 0
        x[1::4, :, 6:60:2] = 0
        x[1::4, :, 70:124:2] = 0
        x[2::4, :, :64] = 0
    a.check()


def test_sums_beyond_the_products():
    """Products that fp32 does not have, their sum within it, and sums beyond it."""
    a = Append(40, hq=4, hkv=2, seed=23)
    a.rot.cos_sin[:, :64], a.rot.cos_sin[:, 64:] = 1.75, 1.5
    for x in (a.q, a.k):
        x[..., :64], x[..., 64:] = 3e38, 3.2e38
        x[::3, :, 64:] = 1.0
        x[1::3] = -x[1::3]
    a.check()


@pytest.mark.parametrize("kind", ["constant", "zero", "positive", "negative", "outlier", "ties", "tiny", "huge", "signs", "edge"])
def test_groups(kind):
    a = Append(500, q4=True, rd=0, queries=False, seed=10)
    g = torch.Generator(device="cuda").manual_seed(11)
    for i, name in enumerate(("k", "v")):
        x = getattr(a, name).float()
        if kind == "constant":
            x = x[..., :1].expand(x.shape)
        elif kind == "zero":
            x = x * (torch.arange(128, device="cuda") // 32 != 1 + i)
        elif kind == "positive":
            x = x.abs() + 100
        elif kind == "negative":
            x = -x.abs() * 1e-3
        elif kind == "outlier":
            x[..., 17 + i::40] *= 1000
        elif kind == "ties":  # multiples of half of a step
            x = torch.randint(-15, 16, x.shape, generator=g, device="cuda") * 0.5 * (1 + torch.randint(0, 8, x.shape[:2], generator=g, device="cuda")[..., None] / 8)
        elif kind == "tiny":  # around the least scale, and below what bf16 has as normal numbers
            x = x * torch.exp2(torch.randint(-132, -94, x.shape[:2], generator=g, device="cuda")[..., None].double()).float()
        elif kind == "huge":
            x = x * 1e37
        elif kind == "signs":
            x = torch.where(x > 0, 1.0, -1.0) * 0.0
        else:  # ranges of 15 scales, or a step of bf16 beside
            x = torch.randint(0, 2, x.shape, generator=g, device="cuda") * 15.0 * (1 + torch.randint(0, 8, x.shape[:2], generator=g, device="cuda")[..., None] / 8)
            x[::3] = x[::3] * 1.0079
        setattr(a, name, x.to(BF).contiguous())
    _, out = a.check()
    x, h = a.k.double(), out["k_out"].double()
    _, s, _ = kv4_ref.quantise(a.k)
    assert bool(((h - x).abs() <= s.repeat_interleave(32, -1) / 2).all())


def test_groups_whose_range_is_rounded():
    a = Append(64, hkv=1, hq=1, q4=True, rd=0, queries=False, seed=25)
    a.k, a.v = far_apart().cuda()[:, None], -far_apart().cuda()[:, None]
    a.check()


def test_values_that_are_not_finite():
    """Their group reads as NaN, the others as they are."""
    a = Append(40, q4=True, rd=0, queries=False, seed=12)
    a.k[3, 0, 5], a.k[4, 1, 127], a.v[5, 0, 64], a.v[39, 1, 0] = math.nan, math.inf, -math.inf, math.nan
    a.k[7, 0, :64], a.k[7, 0, 3] = 3e38, -3e38  # (a range beyond fp32)
    _, out = a.check()
    assert int(out["k_out"].isnan().sum()) == 96 and int(out["v_out"].isnan().sum()) == 64
    b = Append(40, rd=64, seed=12)  # a rotated pair: both of its channels, no other
    b.k[3, 0, 5] = math.nan
    _, out = b.check()
    assert out["k_out"][3, 0].isnan().nonzero()[:, 0].tolist() == [5, 37]
    b.q[2, 1, 100] = math.inf  # (passes through)
    _, out = b.check()
    assert bool(out["q_out"][2, 1, 100].isinf()) and int((~out["q_out"].isfinite()).sum()) == 1


@pytest.mark.parametrize("q4", [False, True])
def test_padding_and_bad_positions(q4):
    a = Append(50, q4=q4, seed=13)
    done = torch.ones(50, dtype=torch.bool, device="cuda")
    done[[0, 17, 49]] = False
    a.positions[~done] = -1
    a.check(done=done)
    a.positions[17] = 5000  # the table has 5000
    done[17] = False
    a.check(done=done, status=(3, 17))
    a.positions[17] = -2
    a.check(done=done, status=(3, 17))
    a.positions[17], done[17] = 4999, True
    a.check(done=done)


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("bad", [-2, 7 * 16, 2 ** 31 - 1, -2 ** 31])
def test_bad_slots(q4, bad):
    """Skipped and reported; the rotated rows are written all the same."""
    a = Append(50, q4=q4, seed=14)
    assert a.num_pages == 7
    a.slots[31] = bad
    a.check(status=(3, 31))


@pytest.mark.parametrize("q4", [False, True])
def test_offsets_beyond_32_bits(q4):
    """First and last pages of a cache of more than 2^32 elements (bytes)."""
    hkv, page, T = 8, 128, 600
    a = Append(T, hq=8, hkv=hkv, page=page, q4=q4, seed=15, queries=False)
    pages = (1 << 32) // (page * hkv * (144 if q4 else 128)) + 9
    slots = np.arange(T)
    slots[::2] = pages * page - 1 - slots[::2]
    a.slots = dev(slots)
    if q4:
        big = torch.zeros((pages, hkv, 2, page * 72), dtype=torch.uint8, device="cuda")
        ckv.ckv_cache_append_q4(a.cfg, ckv.PagedCacheQ4(big, page), a.k, a.v, a.slots, a.ws, rotation=a.rot, positions=a.positions)
    else:
        big, big_v = (torch.zeros((pages, page, hkv, 128), dtype=BF, device="cuda") for _ in range(2))
        ckv.ckv_cache_append(a.cfg, ckv.PagedCache(big, big_v), a.k, a.v, a.slots, a.rot, a.positions, a.ws)
    assert ckv.ckv_read_device_status(a.ws) == (0, 0)
    k, near = kv4_ref.rotate(a.k, a.rot.cos_sin, a.positions), list(range(5)) + list(range(pages - 5, pages))
    if q4:
        want = torch.zeros((10, hkv, 2, page * 72), dtype=torch.uint8, device="cuda")
        s = torch.where(a.slots >= 5 * page, a.slots - (pages - 10) * page, a.slots)
        kv4_ref.put(want, page, s, k, 0)
        kv4_ref.put(want, page, s, a.v, 1)
        same(big[near], want)
        assert not bool(big[5:pages - 5].any())
    else:
        same(big.view(-1, hkv, 128)[a.slots.long()], k)
        same(big_v.view(-1, hkv, 128)[a.slots.long()], a.v)
        assert int((big != 0).any(-1).any(-1).sum()) == T


@pytest.mark.parametrize("q4", [False, True])
@pytest.mark.parametrize("layer", [0, 2])
def test_pages_of_layers_side_by_side(q4, layer):
    """One buffer with three layers' pages between each other: the others' bytes stay."""
    a = Append(70, page=32, q4=q4, seed=18, queries=False)
    shape = (a.num_pages, 3, a.hkv, 2, 32 * 72) if q4 else (a.num_pages, 3, 2, 32, a.hkv, 128)
    both = torch.full(shape, 7, dtype=torch.uint8 if q4 else BF, device="cuda")
    mine = both[:, layer]
    if q4:
        ckv.ckv_cache_append_q4(a.cfg, ckv.PagedCacheQ4(mine, 32), a.k, a.v, a.slots, a.ws, rotation=a.rot, positions=a.positions)
    else:
        ckv.ckv_cache_append(a.cfg, ckv.PagedCache(mine[:, 0], mine[:, 1]), a.k, a.v, a.slots, a.rot, a.positions, a.ws)
    assert ckv.ckv_read_device_status(a.ws) == (0, 0)
    want, k = torch.full_like(both, 7), kv4_ref.rotate(a.k, a.rot.cos_sin, a.positions)
    for i, x in enumerate((k, a.v)):
        if q4:
            kv4_ref.put(want[:, layer], 32, a.slots, x, i)
        else:
            want[a.slots.long() // 32, layer, i, a.slots.long() % 32] = x
    same(both, want)


@pytest.mark.parametrize("q4", [False, True])
def test_no_tokens(q4):
    a = Append(0, q4=q4, seed=19)
    pages, _ = a.run(outs=False)
    assert bool((pages == (0xA5 if q4 else 7)).all())


@pytest.mark.parametrize("q4", [False, True])
def test_captured_and_replayed(q4):
    """One captured call over device positions and slots: each replay sees those of its time; on another stream too."""
    a = Append(33, q4=q4, seed=16)
    pages = a.empty_cache().view
    cache = ckv.PagedCacheQ4(pages, a.page) if q4 else ckv.PagedCache(pages[:, 0], pages[:, 1])
    q_out, k_out = torch.zeros_like(a.q), torch.zeros_like(a.k)
    kw = dict(q=a.q, q_out=q_out, k_out=k_out)

    def call(stream=None):
        if q4:
            ckv.ckv_cache_append_q4(a.cfg, cache, a.k, a.v, a.slots, a.ws, rotation=a.rot, positions=a.positions, stream=stream, **kw)
        else:
            ckv.ckv_cache_append(a.cfg, cache, a.k, a.v, a.slots, a.rot, a.positions, a.ws, stream=stream, **kw)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    call(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for step in range(3):
        a.positions.copy_((a.positions * 3 + 1) % 5000)
        a.slots.copy_(a.slots.roll(1))
        a.k.copy_(a.k.roll(1, 0))
        pages.fill_(7)
        graph.replay()
        k = kv4_ref.rotate(a.k, a.rot.cos_sin, a.positions)
        same(q_out, kv4_ref.rotate(a.q, a.rot.cos_sin, a.positions))
        same(k_out, kv4_ref.held(k) if q4 else k)
        want = torch.full_like(pages, 7)
        if q4:
            kv4_ref.put(want, a.page, a.slots, k, 0)
            kv4_ref.put(want, a.page, a.slots, a.v, 1)
        else:
            for i, x in enumerate((k, a.v)):
                want[a.slots.long() // a.page, i, a.slots.long() % a.page] = x
        same(pages, want)
    assert ckv.ckv_read_device_status(a.ws) == (0, 0)


def test_refusals():
    for q4 in (False, True):
        a = Append(20, q4=q4, seed=17)
        pages = a.empty_cache().view
        cache = ckv.PagedCacheQ4(pages, a.page) if q4 else ckv.PagedCache(pages[:, 0], pages[:, 1])
        other = ckv.PagedCache(*(torch.zeros((4, 16, 2, 128), dtype=BF, device="cuda") for _ in range(2))) if q4 else \
            ckv.PagedCacheQ4(torch.zeros((4, 2, 2, 16 * 72), dtype=torch.uint8, device="cuda"), 16)
        base = dict(cache=cache, k=a.k, v=a.v, slots=a.slots, rotation=a.rot, positions=a.positions, q=a.q, q_out=torch.empty_like(a.q),
                    k_out=torch.empty_like(a.k))

        def call(cfg=a.cfg, **kw):
            b = {**base, **kw}
            more = {x: b[x] for x in ("q", "q_out", "k_out", "v_out", "tok_stride") if x in b}
            if q4:
                ckv.ckv_cache_append_q4(cfg, b["cache"], b["k"], b["v"], b["slots"], a.ws, rotation=b["rotation"], positions=b["positions"], **more)
            else:
                ckv.ckv_cache_append(cfg, b["cache"], b["k"], b["v"], b["slots"], b["rotation"], b["positions"], a.ws, **more)

        call()
        for bad in (dict(k=a.k.float()), dict(k=a.k[:10]), dict(v=a.v.cpu()), dict(slots=a.slots.long()), dict(positions=a.positions[:5]),
                    dict(positions=a.positions.float()), dict(q_out=None), dict(q=None), dict(q=a.q[:, :4]), dict(k_out=torch.empty(3, device="cuda")),
                    dict(cfg=config(8, 4)), dict(cache=other), dict(tok_stride=999), dict(k_out=a.k.transpose(0, 1))):
            with pytest.raises(ValueError):
                call(**bad)
        with pytest.raises(ckv.CkvError):  # the outputs over one another, over another row
            call(k_out=base["q_out"].view(-1)[:a.k.numel()].view(a.k.shape))
        both = torch.zeros(41 * 2 * 128, dtype=BF, device="cuda")
        with pytest.raises(ckv.CkvError):
            call(k=both[:20 * 256].view(20, 2, 128), k_out=both[256:21 * 256].view(20, 2, 128))
        with pytest.raises(ckv.CkvError, match="over one of its inputs"):
            call(k_out=a.v)
        with pytest.raises(ckv.CkvError, match="rotary_dim"):
            call(rotation=ckv.new_rotation(5000, rotary_dim=24))
    for bad in (torch.zeros((4, 2, 2, 16 * 72), dtype=torch.int8, device="cuda"), torch.zeros((4, 2, 2, 16 * 71), dtype=torch.uint8, device="cuda"),
                torch.zeros((4, 2, 2, 16 * 72), dtype=torch.uint8), torch.zeros((4, 4, 2, 16 * 72), dtype=torch.uint8, device="cuda")[:, ::2],
                torch.zeros((2, 2, 2, 16 * 72), dtype=torch.uint8, device="cuda")[:1].expand(4, 2, 2, 16 * 72)):
        with pytest.raises(ValueError):
            ckv.PagedCacheQ4(bad, 16)
    for bad in (torch.zeros(10, 128), torch.zeros(10, 128, device="cuda").half(), torch.zeros(10, 256, device="cuda")[:, :128]):
        with pytest.raises(ValueError):
            ckv.Rotation(bad)
