"""The paged cache where rows arrive unrotated and where it holds 4 bits a value, as cases that can be timed and
compared: new tokens' queries and keys rotated by their positions on the way into the cache, the same into a cache of
4 bits, and the attention of new tokens over such a cache.

Head counts and lengths are those of the library's workloads (32 query / 8 KV heads, 28 / 4 heads, head_dim 128,
131072 tokens in a cache) and of a serving batch.

A row of 128 values in 4 bits, in four groups of 32 (all of it exact in bf16, so that a cached value is a bf16 number):
  range = max(x, 0) - min(x, 0) over the group; the scale s is the least number of 4 significant bits (2^-100 at least)
  with 15 s >= range; the zero point z = round(-min(x, 0) / s), the codes n = clamp(round(x / s) + z, 0, 15) (ties to
  even); a value is s (n - z).
  A group is 16 bytes: 32-bit words of 8 channels, channel c of a word in nibble c / 2 + 4 (c % 2); its scale and zero point
  are 16 bits, the scale's bf16 pattern (whose low nibble is 0) with z in the low nibble.
  A page of one head: K codes [4 groups][page][16 bytes], K scales [page][4] 16 bits, then V's.

A case: `op` and its sizes; lists are comma-separated texts.
  append   lens (new tokens of each sequence, at consecutive positions), q_heads, kv_heads, page, rotary (rotated
           channels), interleaved (pairs of neighbours instead of halves), fused (q, k and v lie in one buffer), skip (every
           skip-th token has no slot; 0 = none), span (positions of the rotation's table)
  append4  the same into a cache of 4 bits; rotary 0: the rows are rotated already, and there are no queries
  paged4   lens (cached tokens, the new ones included), new (new tokens per sequence), q_heads, kv_heads, page, pad
           (query rows behind the last sequence)
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
D = 128
SCALE = 1.0 / math.sqrt(D)


def _ints(text):
    return [int(x) for x in text.split(",")]


def _text(values):
    return ",".join(str(int(v)) for v in values)


def listed():
    gen = np.random.default_rng(17)
    batch64 = np.exp(gen.uniform(math.log(128), math.log(8192), 64)).astype(int)
    drafts = np.exp(gen.uniform(math.log(512), math.log(16384), 40)).astype(int)
    return [
        # one decode step's q, k and v of 64 requests, out of a fused projection: latency
        dict(name="append_64", op="append", lens=_text([1] * 64), q_heads=32, kv_heads=8, page=64, rotary=128,
             interleaved=False, fused=True, skip=0, span=131072),
        # a batch of prompts on the 28 / 4 head model: every query and key, a few tokens without a slot
        dict(name="append_prompts_28_4", op="append", lens="4981,8209,1,333,7001", q_heads=28, kv_heads=4, page=16,
             rotary=128, interleaved=False, fused=True, skip=13, span=32768),
        # a long chunk on a model that rotates half of the channels, neighbours in pairs
        dict(name="append_chunk_half", op="append", lens="8192", q_heads=32, kv_heads=8, page=32, rotary=64,
             interleaved=True, fused=False, skip=0, span=32768),
        # one decode step of 64 requests into 4 bits
        dict(name="append4_64", op="append4", lens=_text([1] * 64), q_heads=32, kv_heads=8, page=64, rotary=128,
             interleaved=False, fused=True, skip=0, span=131072),
        # kept rows of a compressed prompt batch (rotated before they were scored) into 4 bits, some rows of it padding
        dict(name="append4_kept_40001", op="append4", lens="40001", q_heads=8, kv_heads=8, page=16, rotary=0,
             interleaved=False, fused=False, skip=11, span=0),
        # a chunk of two prompts into 4 bits, rotated on the way
        dict(name="append4_chunk_28_4", op="append4", lens="4096,3001", q_heads=28, kv_heads=4, page=32, rotary=128,
             interleaved=False, fused=True, skip=0, span=32768),
        # one request's next token over a compressed cache: the smallest call, latency
        dict(name="decode4_1x1056", op="paged4", lens="1056", new="1", q_heads=32, kv_heads=8, page=16, pad=0),
        # a serving batch's next tokens, ragged caches, padded to a captured batch size
        dict(name="decode4_64", op="paged4", lens=_text(batch64), new=_text([1] * 64), q_heads=32, kv_heads=8,
             page=64, pad=8),
        # next tokens over uncompressed long caches: the bytes of the cache
        dict(name="decode4_8x131072", op="paged4", lens=_text([131072 - 17 * i for i in range(8)]),
             new=_text([1] * 8), q_heads=32, kv_heads=8, page=32, pad=0),
        # short drafts to be verified on the 28 / 4 head model
        dict(name="draft4_40x2", op="paged4", lens=_text(drafts), new=_text([2] * 40), q_heads=28, kv_heads=4, page=16,
             pad=0),
        # chunked prefill beside single tokens: ragged chunks over ragged caches
        dict(name="chunk4_ragged_28_4", op="paged4", lens="24001,1029,8192,32768,513", new="1024,77,1,512,513",
             q_heads=28, kv_heads=4, page=16, pad=0),
        # one long chunk over a long cache
        dict(name="chunk4_2048", op="paged4", lens="34816", new="2048", q_heads=32, kv_heads=8, page=128, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hq, hkv = rng.choice([(32, 8), (28, 4), (8, 2), (4, 4)])
    op, page = rng.choice(["append", "append4", "paged4", "paged4"]), rng.choice([16, 32, 64, 128])
    if op != "paged4":
        total = _log(rng, 1, 20000)
        seqs = rng.choice([1, 1, total, rng.randint(1, 9)]) if total <= 300 else rng.randint(1, 9)
        cuts = sorted(rng.randint(0, total) for _ in range(seqs - 1))
        lens = [b - a for a, b in zip([0] + cuts, cuts + [total])]
        return dict(op=op, lens=_text(lens), q_heads=hq, kv_heads=hkv, page=page,
                    rotary=rng.choice([128, 128, 64, 48, 0 if op == "append4" else 96]), interleaved=rng.random() < 0.3,
                    fused=rng.random() < 0.6, skip=rng.choice([0, 0, 2, 13]), span=rng.choice([32768, 131072]))
    seqs = _log(rng, 1, 96)
    longest = _log(rng, 64, 400000 // seqs if seqs > 3 else 131072)
    most = rng.choice([1, 1, 8, 700])
    lens = [max(1, int(longest * rng.random())) for _ in range(seqs - 1)] + [longest]
    new = [min(n, 1 if most == 1 else rng.randint(1, max(1, most // (1 + seqs // 8)))) for n in lens]
    while sum(n * L for n, L in zip(new, lens)) * hq > 2048 * 32768 * 32:
        new = [(n + 1) // 2 for n in new]
    return dict(op=op, lens=_text(lens), new=_text(new), q_heads=hq, kv_heads=hkv, page=page, pad=rng.choice([0, 0, 5]))


def _normal(shape, seed, k, heavy=False):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + k)
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if heavy:  # a few channels of the keys are ten times the others, as in trained models
        c = torch.randperm(D, generator=g, device="cuda")[:4]
        x[..., c] *= 10
    return x.to(torch.bfloat16)


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


def _config(q_heads, kv_heads):
    import paper_2508_02401_gb300 as ckv
    return ckv.Config(num_layers=1, num_q_heads=q_heads, num_kv_heads=kv_heads, window=32, pool_kernel=7,
                      pool_type=ckv.POOL_MAX, head_order=ckv.POOL_THEN_SUM,
                      head_mask=np.ones((1, q_heads), np.uint8), budgets=np.array([256], np.int32))


def prepare(case, seed):
    st = dict(case=case)
    hq, hkv, P = case["q_heads"], case["kv_heads"], case["page"]
    g = np.random.default_rng(seed * 7919 + 5)
    if case["op"] == "paged4":
        lens, new = np.array(_ints(case["lens"])), np.array(_ints(case["new"]))
        blocks = -(-lens // P)
        n_pages = int(blocks.sum()) + 3
        table = np.zeros((len(lens), int(blocks.max())), np.int32)
        table[np.arange(table.shape[1]) < blocks[:, None]] = g.permutation(n_pages)[:int(blocks.sum())]
        cu = np.concatenate([[0], np.cumsum(new)])
        T = int(cu[-1]) + case["pad"]
        pages = torch.empty((n_pages, hkv, 2, P * 72), dtype=torch.uint8, device="cuda")
        for i in range(2):
            codes, scales = _quantise(_normal((n_pages, hkv, P, D), seed, 2 + i, i == 0).float())
            pages[:, :, i, :P * 64] = _words(codes).view(n_pages, hkv, P, 4, 16).transpose(2, 3).reshape(n_pages, hkv, -1)
            pages[:, :, i, P * 64:] = scales.reshape(n_pages, hkv, -1)
        st.update(table=_dev(table), lens=_dev(lens), cu=_dev(cu), n_max=int(new.max()), l_max=int(lens.max()),
                  q=_normal((T, hq, D), seed, 1), pages=pages,
                  out=torch.zeros((T, hq, D), dtype=torch.bfloat16, device="cuda"),
                  lse=torch.zeros((hq, T), dtype=torch.float32, device="cuda"))
        if own:
            import paper_2508_02401_gb300 as ckv
            st["cfg"] = _config(hq, hkv)
            st["cache"] = ckv.PagedCacheQ4(pages, P)
            st["ws"] = ckv.new_attention_workspace(st["cfg"])
        return st
    lens, rd = _ints(case["lens"]), case["rotary"]
    T = sum(lens)
    n_pages = -(-T // P) + 2
    slots = (g.permutation(n_pages)[:-(-T // P), None] * P + np.arange(P)).reshape(-1)[:T]
    if case["skip"]:
        slots[::case["skip"]] = -1
    heads = hq + 2 * hkv
    if case["fused"]:
        both = torch.cat([_normal((T, hq, D), seed, 1), _normal((T, hkv, D), seed, 2, True),
                          _normal((T, hkv, D), seed, 3)], 1)
        q, k, v = both[:, :hq], both[:, hq:hq + hkv], both[:, hq + hkv:]
        st.update(q=q, k=k, v=v, tok_stride=heads * D)
    else:
        st.update(q=_normal((T, hq, D), seed, 1), k=_normal((T, hkv, D), seed, 2, True), v=_normal((T, hkv, D), seed, 3),
                  tok_stride=0)
    st.update(slots=_dev(slots), k_out=torch.zeros((T, hkv, D), dtype=torch.bfloat16, device="cuda"))
    if rd:
        first = g.integers(0, case["span"] - np.array(lens) + 1)
        positions = np.concatenate([a + np.arange(n) for a, n in zip(first, lens)])
        # the angles in 64 bits: the far positions' would lose their digits in 32
        angle = torch.arange(case["span"], device="cuda", dtype=torch.float64)[:, None] * \
            500000.0 ** (-torch.arange(rd // 2, device="cuda", dtype=torch.float64) * 2 / rd)
        st.update(positions=_dev(positions), cos_sin=torch.cat([angle.cos(), angle.sin()], 1).float(),
                  q_out=torch.zeros((T, hq, D), dtype=torch.bfloat16, device="cuda"))
    if case["op"] == "append":
        st.update(k_pages=torch.zeros((n_pages, P, hkv, D), dtype=torch.bfloat16, device="cuda"),
                  v_pages=torch.zeros((n_pages, P, hkv, D), dtype=torch.bfloat16, device="cuda"))
    else:
        st.update(pages=torch.zeros((n_pages, hkv, 2, P * 72), dtype=torch.uint8, device="cuda"),
                  v_out=torch.zeros((T, hkv, D), dtype=torch.bfloat16, device="cuda"))
    if own:
        import paper_2508_02401_gb300 as ckv
        st["cfg"] = _config(hq, hkv)
        st["cache"] = ckv.PagedCache(st["k_pages"], st["v_pages"]) if case["op"] == "append" else \
            ckv.PagedCacheQ4(st["pages"], P)
        st["ws"] = ckv.new_attention_workspace(st["cfg"])
        st["rotation"] = ckv.Rotation(st["cos_sin"], interleaved=case["interleaved"]) if rd else None
    return st


# ------------------------------------------------------------------------------- plain forms
def _rotate(x, st):
    """x [T, H, 128] bf16 by the positions' angles, in 64 bits, rounded to 32 and then to bf16."""
    rd = st["case"]["rotary"]
    if not rd:
        return x.contiguous()
    cos, sin = (t[:, None] for t in st["cos_sin"][st["positions"].long()].double().split(rd // 2, 1))
    y = x.double()
    a, b = (y[..., 0:rd:2], y[..., 1:rd:2]) if st["case"]["interleaved"] else (y[..., :rd // 2], y[..., rd // 2:rd])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if st["case"]["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., rd:]], -1).float().to(torch.bfloat16)


def _quantise(x):
    """x [..., 128] in 32 bits -> codes [..., 128], scales and zero points [..., 8] bytes."""
    x = x.unflatten(-1, (4, 32))
    low, high = x.amin(-1, keepdim=True).clamp_max(0), x.amax(-1, keepdim=True).clamp_min(0)
    wide = high - low
    bits = (wide / 15).view(torch.int32) & -(1 << 20)  # the sign, the exponent and 3 bits of the fraction
    s = torch.where(bits.view(torch.float32) * 15 < wide, bits + (1 << 20), bits).view(torch.float32).clamp_min(2.0 ** -100)
    z = (-low / s).round()
    n = ((x / s).round() + z).clamp(0, 15)
    word = (s.view(torch.int32) >> 16) | z.int()
    return n.int().flatten(-2), word[..., 0].to(torch.int16).view(torch.uint8)


def _words(codes):
    """codes [..., 128] -> bytes [..., 64]: words of 8 channels, the even ones in the low half."""
    n = codes.unflatten(-1, (16, 4, 2)).long()
    shift = torch.tensor([[0, 16], [4, 20], [8, 24], [12, 28]], device=codes.device)
    return (n << shift).sum((-1, -2)).to(torch.int32).view(torch.uint8)


def _values(codes, scales):
    """The values in 32 bits of codes [..., 128] and scales [..., 8] bytes."""
    word = scales.contiguous().view(torch.int16).int()
    s, z = ((word & 0xFFF0) << 16).view(torch.float32), (word & 15).float()
    return ((codes.unflatten(-1, (4, 32)).float() - z[..., None]) * s[..., None]).flatten(-2)


def _plain_append(st):
    slots, P = st["slots"].long(), st["case"]["page"]
    k, v = _rotate(st["k"], st), st["v"]
    n = st["k_pages"].shape[0] * P
    to = torch.where(slots < 0, n, slots)
    kp, vp = (torch.cat([st[x].view(n, -1, D), st[x].new_zeros(1, v.shape[1], D)]) for x in ("k_pages", "v_pages"))
    kp[to], vp[to] = k, v
    return dict(q=_rotate(st["q"], st), k=k, k_pages=kp[:n].view(st["k_pages"].shape), v_pages=vp[:n].view(st["v_pages"].shape))


def _plain_append4(st):
    slots, P = st["slots"].long(), st["case"]["page"]
    rows = torch.stack([_rotate(st["k"], st), st["v"]], 2).float()  # [T, H, 2, 128]
    codes, scales = _quantise(rows)
    kv = _values(codes, scales).to(torch.bfloat16)
    n = st["pages"].shape[0]
    pages = torch.cat([st["pages"], st["pages"].new_zeros(1, *st["pages"].shape[1:])])
    page, row = torch.where(slots < 0, n, slots // P), slots.clamp_min(0) % P
    pages[..., :P * 64].unflatten(-1, (4, P, 16))[page, :, :, :, row] = _words(codes).unflatten(-1, (4, 16))
    pages[..., P * 64:].unflatten(-1, (P, 8))[page, :, :, row] = scales
    found = dict(k=kv[:, :, 0].contiguous(), v=kv[:, :, 1].contiguous(), pages=pages[:n])
    return {**found, "q": _rotate(st["q"], st)} if st["case"]["rotary"] else found


def _softmax_rows(q, k, v, visible):
    """q [B, H, G, n, D], k, v [B, H, L, D] in 32 bits, visible [B, n, L] -> out like q, lse."""
    B, H, G, n, _ = q.shape
    s = torch.matmul(q.reshape(B, H, G * n, D), k.transpose(-1, -2)).reshape(B, H, G, n, -1) * SCALE
    s.masked_fill_(~visible[:, None, None], -math.inf)
    m = s.amax(-1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    e = s.sub_(m).exp_()
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e.reshape(B, H, G * n, -1), v).reshape(q.shape) / total
    return o, (m + total.log())[..., 0]


def _cached(st, which):
    """Every page's rows of K (0) or V (1) in 32 bits: [pages, H, page, 128]."""
    P, pages = st["case"]["page"], st["pages"][:, :, which]
    words = pages[..., :P * 64].unflatten(-1, (4, P, 16)).transpose(2, 3).reshape(*pages.shape[:2], P, 64).view(torch.int32)
    shift = torch.tensor([0, 16, 4, 20, 8, 24, 12, 28], device="cuda", dtype=torch.int32)
    codes = ((words[..., None] >> shift) & 15).flatten(-2)
    return _values(codes, pages[..., P * 64:].unflatten(-1, (P, 8)))


def _plain_paged4(st):
    c, P = st["case"], st["case"]["page"]
    hq, hkv = c["q_heads"], c["kv_heads"]
    G, T, n, L = hq // hkv, st["q"].shape[0], st["n_max"], st["l_max"]
    S = st["lens"].shape[0]
    j = torch.arange(L, device="cuda")
    cached = (st["lens"][:, None] > j)[:, None, :, None]
    table = st["table"].long()
    # [S, blocks, H, page, 128] -> [S, H, L, 128]
    k, v = (torch.where(cached, _cached(st, i)[table].transpose(1, 2).reshape(S, hkv, -1, D)[:, :, :L], 0) for i in range(2))
    start, count = st["cu"][:-1].long(), (st["cu"][1:] - st["cu"][:-1]).long()
    i = torch.arange(n, device="cuda")
    row = torch.where(i < count[:, None], start[:, None] + i, T)  # row T: none
    q = torch.cat([st["q"], st["q"].new_zeros(1, hq, D)])[row].float().reshape(S, n, hkv, G, D).permute(0, 2, 3, 1, 4)
    pos = (st["lens"].long() - count)[:, None] + i
    o, ls = _softmax_rows(q, k, v, j <= torch.minimum(pos, st["lens"].long()[:, None] - 1)[:, :, None])
    out = torch.zeros((T + 1, hq, D), dtype=torch.bfloat16, device="cuda")
    out[row.reshape(-1)] = o.permute(0, 3, 1, 2, 4).reshape(S * n, hq, D).to(torch.bfloat16)
    lse = torch.zeros((T + 1, hq), dtype=torch.float32, device="cuda")
    lse[row.reshape(-1)] = ls.permute(0, 3, 1, 2).reshape(S * n, hq)
    return dict(out=out[:T], lse=lse[:T].t().contiguous())


def run(state):
    st, op = state, state["case"]["op"]
    if not own:
        return {"append": _plain_append, "append4": _plain_append4, "paged4": _plain_paged4}[op](st)
    import paper_2508_02401_gb300 as ckv
    if op == "paged4":
        ckv.ckv_paged_attention_q4(st["cfg"], st["cache"], st["table"], st["lens"], st["cu"], st["q"], st["out"],
                                   st["ws"], lse=st["lse"])
        return dict(out=st["out"], lse=st["lse"])
    strides = dict(tok_stride=st["tok_stride"], q_tok_stride=st["tok_stride"])
    if op == "append":
        ckv.ckv_cache_append(st["cfg"], st["cache"], st["k"], st["v"], st["slots"], st["rotation"], st["positions"],
                             st["ws"], q=st["q"], q_out=st["q_out"], k_out=st["k_out"], **strides)
        return dict(q=st["q_out"], k=st["k_out"], k_pages=st["k_pages"], v_pages=st["v_pages"])
    if st["case"]["rotary"]:
        ckv.ckv_cache_append_q4(st["cfg"], st["cache"], st["k"], st["v"], st["slots"], st["ws"],
                                rotation=st["rotation"], positions=st["positions"], q=st["q"], q_out=st["q_out"],
                                k_out=st["k_out"], v_out=st["v_out"], **strides)
        return dict(k=st["k_out"], v=st["v_out"], pages=st["pages"], q=st["q_out"])
    ckv.ckv_cache_append_q4(st["cfg"], st["cache"], st["k"], st["v"], st["slots"], st["ws"], k_out=st["k_out"],
                            v_out=st["v_out"], tok_stride=st["tok_stride"])
    return dict(k=st["k_out"], v=st["v_out"], pages=st["pages"])


# ------------------------------------------------------------------------------- 64 bits
def _exact_turn(x, st):
    """The rotation as a complex product, in 64 bits."""
    rd, x = st["case"]["rotary"], x.double()
    if not rd:
        return x
    t = st["cos_sin"].double().index_select(0, st["positions"].long())
    w = torch.complex(t[:, :rd // 2], t[:, rd // 2:]).unsqueeze(1)
    lead = torch.arange(rd // 2, device="cuda")
    re, im = (2 * lead, 2 * lead + 1) if st["case"]["interleaved"] else (lead, lead + rd // 2)
    c = torch.complex(x[..., re], x[..., im]) * w
    y = x.clone()
    y[..., re], y[..., im] = c.real, c.imag
    return y


def _power(e):
    """2^e in 64 bits, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_held(x):
    """What 4 bits hold of x [T, H, 128] (bf16 numbers in 64 bits), group by group from the definition."""
    found = torch.empty_like(x)
    for g in range(0, D, 32):
        y = x[..., g:g + 32]
        low = torch.minimum(y.min(-1, keepdim=True).values, torch.zeros((), dtype=y.dtype, device=y.device))
        wide = torch.maximum(y.max(-1, keepdim=True).values, torch.zeros((), dtype=y.dtype, device=y.device)) - low
        e = torch.frexp(wide / 15).exponent
        unit = _power(e.clamp_min(-200) - 4)
        s = torch.ceil(wide / 15 / unit) * unit
        s = torch.clamp_min(torch.where((s - unit) * 15 >= wide, s - unit, s), 2.0 ** -100)  # (the quotient is rounded)
        z = torch.round(-low / s)
        found[..., g:g + 32] = s * (torch.minimum(torch.maximum(torch.round(y / s), -z), 15 - z))
    return found


def _exact_append(case, seed):
    st = prepare(case, seed)
    k, v = _exact_turn(st["k"], st), st["v"].double()
    found = dict(q=_exact_turn(st["q"], st)) if case["rotary"] else {}
    slots = st["slots"].long()
    there = slots >= 0
    if case["op"] == "append":
        kp, vp = torch.zeros_like(st["k_pages"], dtype=torch.float64), torch.zeros_like(st["v_pages"], dtype=torch.float64)
        kp.view(-1, *k.shape[1:])[slots[there]], vp.view(-1, *v.shape[1:])[slots[there]] = k[there], v[there]
        return dict(found, k=k, k_pages=kp, v_pages=vp)
    # (the rows that are held are bf16)
    return dict(found, k=_exact_held(k.float().to(torch.bfloat16).double()), v=_exact_held(v), pages=None)


def exact(case, seed):
    """Attention row by row of heads, in 64 bits."""
    if case["op"] != "paged4":
        return _exact_append(case, seed)
    if work(case)["flops"] > 4e12:
        return None
    st = prepare(case, seed)
    hq, hkv, P = case["q_heads"], case["kv_heads"], case["page"]
    G, T = hq // hkv, st["q"].shape[0]
    out = torch.zeros((T, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((hq, T), dtype=torch.float64, device="cuda")

    def rows(head, which, page, row):
        """[L, 128] out of the pages' bytes."""
        block = st["pages"][page, head, which]
        i = torch.arange(len(page), device="cuda")
        found = []
        for g in range(4):
            at = g * 16 * P + 16 * row[:, None] + torch.arange(16, device="cuda")
            code = block[i[:, None], at].long().reshape(-1, 4, 4)  # [L, word, byte]: channels 0 2, 4 6, 1 3, 5 7
            code = torch.stack([code & 15, code >> 4], -1).reshape(-1, 4, 8)[:, :, [0, 4, 1, 5, 2, 6, 3, 7]].reshape(-1, 32)
            lo, hi = (block[i, 64 * P + 8 * row + 2 * g + b].long() for b in range(2))
            # a bf16 pattern: the exponent from its high bits, then 3 bits of the fraction
            s = (8 + ((lo >> 4) & 7)).double() * _power((hi & 127) * 2 + (lo >> 7) - 130)
            found.append(s[:, None] * (code - (lo & 15)[:, None]))
        return torch.cat(found, 1)

    at = 0
    for s, (L, n) in enumerate(zip(_ints(case["lens"]), _ints(case["new"]))):
        j = torch.arange(L, device="cuda")
        page, row = st["table"][s, j // P].long(), j % P
        for g in range(hkv):
            k, v = rows(g, 0, page, row), rows(g, 1, page, row)
            for h in range(g * G, (g + 1) * G):
                for i in range(0, n, 4096):
                    q = st["q"][at + i:at + min(n, i + 4096), h].double()
                    seen = L - n + i + len(q)
                    x = torch.einsum("id,jd->ij", q, k[:seen]) / math.sqrt(D)
                    x[torch.arange(seen, device="cuda") > (torch.arange(len(q), device="cuda") + seen - len(q))[:, None]] = -math.inf
                    l = torch.logsumexp(x, 1)
                    out[at + i:at + i + len(q), h] = torch.einsum("ij,jd->id", torch.exp(x - l[:, None]), v[:seen])
                    lse[h, at + i:at + i + len(q)] = l
        at += n
    return dict(out=out, lse=lse)


def work(case):
    hq, hkv = case["q_heads"], case["kv_heads"]
    if case["op"] == "paged4":
        lens, new = _ints(case["lens"]), _ints(case["new"])
        T, pages = sum(new), sum(-(-L // case["page"]) for L in lens)
        pairs = sum(n * (L - n) + n * (n + 1) // 2 for L, n in zip(lens, new))
        return dict(bytes=sum(lens) * hkv * 144 + T * hq * (2 * 256 + 4) + 4 * pages, flops=pairs * hq * D * 4)
    T = sum(_ints(case["lens"]))
    kept = T - (-(-T // case["skip"]) if case["skip"] else 0)
    rd = case["rotary"]
    turned = T * (2 * hq * 256 + 4 * rd + 4) if rd else 0  # queries in and out, the angles, the positions
    held = kept * hkv * (512 if case["op"] == "append" else 144)
    outs = T * hkv * (256 if case["op"] == "append" else 512)
    return dict(bytes=turned + T * (hkv * 512 + 4) + held + outs,
                flops=T * (3 * rd * (hq + hkv) + (0 if case["op"] == "append" else 10 * 2 * D * hkv)))
