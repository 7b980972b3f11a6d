"""Attention around the compressed cache, as cases that can be timed and compared: the prefill
attention of packed prompts (with the lse that the compression takes), the block tables and slot
maps of a paged cache, the rows' way into its pages, and the attention of new tokens over it.

Head counts and lengths are those of the library's workloads (32 query / 8 KV heads, 28 / 4 heads,
head_dim 128, prompts up to 32768 packed, 131072 in a cache) and of a serving batch.

A case: `op` and its sizes; lists are comma-separated texts.
  prompt   lens, q_heads, kv_heads, window, interleaved (k and v share one buffer)
  paged    lens (cached tokens, the new ones included), new (new tokens per sequence), page, pad
           (query rows behind the last sequence)
  tables   rows, lo, hi (cached tokens per row), new_lo, new_hi, page, drop (every drop-th row is
           given back instead; 0 = none)
  write    tokens, kv_heads, page, skip (every skip-th token has no slot; 0 = none)
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
    gen = np.random.default_rng(11)
    batch64 = np.exp(gen.uniform(math.log(128), math.log(8192), 64)).astype(int)
    return [
        # one short prompt, one token past a key tile: the time to its first token is all latency
        dict(name="prompt_129", op="prompt", lens="129", q_heads=32, kv_heads=8, window=32, interleaved=False),
        # one prompt of the 8192-token workload
        dict(name="prompt_8192", op="prompt", lens="8192", q_heads=32, kv_heads=8, window=32, interleaved=False),
        # a packed batch of very different prompts on the 28 / 4 head model, k and v in one buffer
        dict(name="prompt_ragged_28_4", op="prompt", lens="4981,12873,1,8209,333,16301", q_heads=28, kv_heads=4,
             window=32, interleaved=True),
        # one long prompt of the 32768-token workload
        dict(name="prompt_32768", op="prompt", lens="32768", q_heads=32, kv_heads=8, window=32, interleaved=False),
        # one request's next token over a compressed cache: the smallest call, latency
        dict(name="decode_1x1056", op="paged", lens="1056", new="1", q_heads=32, kv_heads=8, page=16, pad=0),
        # a serving batch's next tokens, ragged caches, padded to a captured batch size
        dict(name="decode_64", op="paged", lens=_text(batch64), new=_text([1] * 64), q_heads=32, kv_heads=8,
             page=64, pad=8),
        # next tokens over uncompressed long caches: the bytes of the cache
        dict(name="decode_8x131072", op="paged", lens=_text([131072 - 17 * i for i in range(8)]),
             new=_text([1] * 8), q_heads=32, kv_heads=8, page=32, pad=0),
        # chunked prefill beside single tokens: ragged chunks over ragged caches
        dict(name="chunk_ragged_28_4", op="paged", lens="24001,1029,8192,32768,513", new="1024,77,1,512,513",
             q_heads=28, kv_heads=4, page=16, pad=0),
        # one decode step's tables for 32 layers of 64 requests (every layer has lengths of its own)
        dict(name="tables_2048x1", op="tables", rows=2048, lo=0, hi=2048, new_lo=1, new_hi=1, page=16, drop=0),
        # requests admitted: kept prompts of 32 layers of 8 requests, others given back
        dict(name="tables_admit_256", op="tables", rows=256, lo=0, hi=4096, new_lo=0, new_hi=1023, page=32, drop=7),
        # one decode step's rows of 64 requests
        dict(name="write_64", op="write", tokens=64, kv_heads=8, page=64, skip=0),
        # kept rows of a prompt batch into the pages, some rows of it padding
        dict(name="write_40001", op="write", tokens=40001, kv_heads=8, page=16, skip=11),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hq, hkv = rng.choice([(32, 8), (28, 4), (8, 2), (4, 4)])
    op = rng.choice(["prompt", "paged", "tables", "write"])
    if op == "prompt":
        top = _log(rng, 32, 24000)
        lens = [max(1, int(top * rng.random())) for _ in range(rng.randint(0, 7))]
        lens.insert(rng.randint(0, len(lens)), top)
        while sum(n * n for n in lens) * hq > 32768 * 32768 * 24:
            lens.pop()
        return dict(op=op, lens=_text(lens), q_heads=hq, kv_heads=hkv, window=rng.choice([8, 32, 64]),
                    interleaved=rng.random() < 0.3)
    if op == "paged":
        seqs = _log(rng, 1, 96)
        longest = _log(rng, 64, 400000 // seqs if seqs > 3 else 131072)
        most = rng.choice([1, 1, 8, 700])
        lens = [max(1, int(longest * rng.random())) for _ in range(seqs - 1)] + [longest]
        new = [min(n, 1 if most == 1 else rng.randint(1, max(1, most // (1 + seqs // 8)))) for n in lens]
        return dict(op=op, lens=_text(lens), new=_text(new), q_heads=hq, kv_heads=hkv,
                    page=rng.choice([16, 32, 64, 128]), pad=rng.choice([0, 0, 5]))
    if op == "tables":
        rows = _log(rng, 1, 6000)
        hi = rng.choice([0, 100, 4000])
        new_hi = rng.choice([1, 1, _log(rng, 2, 1 + 200000 // rows)])
        return dict(op=op, rows=rows, lo=0, hi=hi, new_lo=0 if new_hi > 1 else 1, new_hi=new_hi,
                    page=rng.choice([16, 32, 64, 128]), drop=rng.choice([0, 3, 10]))
    return dict(op=op, tokens=_log(rng, 1, 60000), kv_heads=hkv, page=rng.choice([16, 32, 64, 128]),
                skip=rng.choice([0, 2, 13]))


def _normal(shape, seed, k, heavy=False):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + k)
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if heavy:  # a few channels of the keys are ten times the others, as in trained models
        c = torch.randperm(D, generator=g, device="cuda")[:4]
        x[..., c] *= 10
    return x.to(torch.bfloat16)


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.asarray(a), dtype=dtype, device="cuda")


def _config(q_heads, kv_heads, window=32):
    import paper_2508_02401_gb300 as ckv
    return ckv.Config(num_layers=1, num_q_heads=q_heads, num_kv_heads=kv_heads, window=window, pool_kernel=7,
                      pool_type=ckv.POOL_MAX, head_order=ckv.POOL_THEN_SUM,
                      head_mask=np.ones((1, q_heads), np.uint8), budgets=np.array([256], np.int32))


def prepare(case, seed):
    st = dict(case=case)
    op = case["op"]
    if op == "prompt":
        hq, hkv = case["q_heads"], case["kv_heads"]
        cu = np.concatenate([[0], np.cumsum(_ints(case["lens"]))]).astype(np.int32)
        T = int(cu[-1])
        st.update(cu=cu, q=_normal((T, hq, D), seed, 1))
        if case["interleaved"]:
            kv = torch.stack([_normal((T, hkv, D), seed, 2, True), _normal((T, hkv, D), seed, 3)], 1)
            st.update(k=kv[:, 0], v=kv[:, 1], tok_stride=2 * hkv * D)
        else:
            st.update(k=_normal((T, hkv, D), seed, 2, True), v=_normal((T, hkv, D), seed, 3), tok_stride=0)
        S, w = len(cu) - 1, case["window"]
        st.update(out=torch.zeros((T, hq, D), dtype=torch.bfloat16, device="cuda"),
                  lse=torch.zeros((hq, T), dtype=torch.float32, device="cuda"),
                  lse_win=torch.zeros((hq, S * w), dtype=torch.float32, device="cuda"))
        if own:
            import paper_2508_02401_gb300 as ckv
            st["cfg"] = _config(hq, hkv, w)
            st["batch"] = ckv.Batch(cu)
            st["ws"] = ckv.new_attention_workspace(st["cfg"])
        return st
    if op == "paged":
        hq, hkv, P = case["q_heads"], case["kv_heads"], case["page"]
        lens, new = np.array(_ints(case["lens"])), np.array(_ints(case["new"]))
        blocks = -(-lens // P)
        g = np.random.default_rng(seed * 7919 + 5)
        n_pages = int(blocks.sum()) + 3
        pages = g.permutation(n_pages)[:int(blocks.sum())]
        table = np.zeros((len(lens), int(blocks.max())), np.int32)
        at = 0
        for s, b in enumerate(blocks):
            table[s, :b] = pages[at:at + b]
            at += int(b)
        cu = np.concatenate([[0], np.cumsum(new)])
        T = int(cu[-1]) + case["pad"]
        st.update(table=_dev(table), lens=_dev(lens), cu=_dev(cu), n_max=int(new.max()), l_max=int(lens.max()),
                  q=_normal((T, hq, D), seed, 1), k=_normal((n_pages, P, hkv, D), seed, 2, True),
                  v=_normal((n_pages, P, hkv, D), seed, 3),
                  out=torch.zeros((T, hq, D), dtype=torch.bfloat16, device="cuda"),
                  lse=torch.zeros((hq, T), dtype=torch.float32, device="cuda"))
        if own:
            import paper_2508_02401_gb300 as ckv
            st["cfg"] = _config(hq, hkv)
            st["cache"] = ckv.PagedCache(st["k"], st["v"])
            st["ws"] = ckv.new_attention_workspace(st["cfg"])
        return st
    if op == "tables":
        n, P = case["rows"], case["page"]
        g = np.random.default_rng(seed * 7919 + 5)
        lens = g.integers(case["lo"], case["hi"] + 1, n)
        new = g.integers(case["new_lo"], case["new_hi"] + 1, n)
        if case["drop"]:
            new[::case["drop"]] = -1
        have = -(-lens // P)
        widest = max(1, -(-(case["hi"] + case["new_hi"]) // P))  # sizes follow from the case, not from the seed
        n_pages = n * widest + 7
        perm = g.permutation(n_pages)
        table = np.full((n, widest), -1, np.int32)
        at = 0
        for r in range(n):
            table[r, :have[r]] = perm[at:at + have[r]]
            at += int(have[r])
        # the ring of free pages, somewhere in its life: `taken` counts the pages ever handed out
        taken = int(g.integers(0, 5)) * n_pages + int(g.integers(0, n_pages))
        ring = np.full(n_pages, -1, np.int32)
        free = perm[at:]
        ring[(taken + np.arange(len(free))) % n_pages] = free
        cap = n * case["new_hi"] + 5  # the tokens that a step may bring; those that it does not have no slot
        st.update(lens=_dev(lens), new=_dev(new), table=_dev(table), free=_dev(ring),
                  pool=_dev([taken, taken + len(free)], torch.int64), cap=cap,
                  slots=torch.zeros(cap, dtype=torch.int32, device="cuda"),
                  cu=torch.zeros(n + 1, dtype=torch.int32, device="cuda"),
                  lens_out=torch.zeros(n, dtype=torch.int32, device="cuda"),
                  pool_out=torch.zeros(2, dtype=torch.int64, device="cuda"))
        if own:
            import paper_2508_02401_gb300 as ckv
            st["ws"] = ckv.new_attention_workspace(_config(32, 8))
        return st
    T, hkv, P = case["tokens"], case["kv_heads"], case["page"]
    g = np.random.default_rng(seed * 7919 + 5)
    n_pages = -(-T // P) + 2
    slots = (g.permutation(n_pages)[:-(-T // P), None] * P + np.arange(P)).reshape(-1)[:T]
    if case["skip"]:
        slots[::case["skip"]] = -1
    st.update(slots=_dev(slots), k=_normal((T, hkv, D), seed, 2), v=_normal((T, hkv, D), seed, 3),
              k_pages=torch.zeros((n_pages, P, hkv, D), dtype=torch.bfloat16, device="cuda"),
              v_pages=torch.zeros((n_pages, P, hkv, D), dtype=torch.bfloat16, device="cuda"))
    if own:
        import paper_2508_02401_gb300 as ckv
        st["cfg"] = _config(hkv, hkv)
        st["cache"] = ckv.PagedCache(st["k_pages"], st["v_pages"])
        st["ws"] = ckv.new_attention_workspace(st["cfg"])
    return st


# ------------------------------------------------------------------------------- plain forms
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


def _plain_prompt(st):
    c, cu = st["case"], st["cu"]
    hq, hkv, w = c["q_heads"], c["kv_heads"], c["window"]
    G = hq // hkv
    out, lse, lse_win = torch.zeros_like(st["out"]), torch.zeros_like(st["lse"]), torch.zeros_like(st["lse_win"])
    for s in range(len(cu) - 1):
        a, b = int(cu[s]), int(cu[s + 1])
        n = b - a
        k, v = (st[x][a:b].float().transpose(0, 1).contiguous() for x in ("k", "v"))
        q = st["q"][a:b].float().reshape(n, hkv, G, D).permute(1, 2, 0, 3)
        step = max(1, min(n, (1 << 29) // (hq * max(n, 1))))  # rows whose logits take 2 GB
        for i in range(0, n, step):
            j = min(n, i + step)
            pos = torch.arange(i, j, device="cuda")
            o, ls = _softmax_rows(q[None, :, :, i:j], k[None, :, :j], v[None, :, :j],
                                  (torch.arange(j, device="cuda") <= pos[:, None])[None])
            out[a + i:a + j] = o[0].permute(2, 0, 1, 3).reshape(j - i, hq, D).to(torch.bfloat16)
            lse[:, a + i:a + j] = ls[0].reshape(hq, j - i)
        t = min(w, n)
        lse_win[:, s * w + w - t:s * w + w] = lse[:, b - t:b]
    return dict(out=out, lse=lse, lse_win=lse_win)


def _plain_paged(st):
    c, P = st["case"], st["case"]["page"]
    hq, hkv = c["q_heads"], c["kv_heads"]
    G, T, n, L = hq // hkv, st["q"].shape[0], st["n_max"], st["l_max"]
    S = st["lens"].shape[0]
    j = torch.arange(L, device="cuda")
    cached = st["lens"][:, None] > j
    slot = st["table"].long()[:, j // P] * P + j % P
    k, v = (torch.where(cached[:, None, :, None], st[x].view(-1, hkv, D)[slot].permute(0, 2, 1, 3), 0).float()
            for x in ("k", "v"))
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


def _plain_tables(st):
    P, cap = st["case"]["page"], st["cap"]
    lens, new, table, free, pool = st["lens"].long(), st["new"].long(), st["table"], st["free"], st["pool"]
    n, n_pages = lens.shape[0], free.shape[0]
    add, have = new.clamp_min(0), (lens + P - 1) // P
    want = (lens + add + P - 1) // P
    take, give = want - have, torch.where(new < 0, have, 0)
    cu = torch.cat([add.new_zeros(1), add.cumsum(0)])
    first, back = take.cumsum(0) - take, give.cumsum(0) - give
    # the new blocks' pages, in the table
    b = torch.arange(table.shape[1], device="cuda")
    fresh = (b >= have[:, None]) & (b < want[:, None])
    table = torch.where(fresh, free[(pool[0] + first[:, None] + b - have[:, None]) % n_pages], table)
    # the new tokens' slots
    t = torch.arange(cap, device="cuda")
    row = (torch.searchsorted(cu, t, right=True) - 1).clamp(0, n - 1)
    pos = lens[row] + t - cu[row]
    slots = torch.where(t < cu[-1], table[row, (pos // P).clamp(0, table.shape[1] - 1)] * P + pos % P, -1)
    # pages given back, behind the ring's last free page
    gone = (new < 0)[:, None] & (b < have[:, None])
    to = torch.where(gone, (pool[1] + back[:, None] + b) % n_pages, n_pages)
    free = torch.cat([free, free.new_zeros(1)])
    free[to.reshape(-1)] = table.reshape(-1)
    lens_out = torch.where(new < 0, 0, lens + add)
    return dict(table=table, slots=slots.int(), cu=cu.int(), lens=lens_out.int(), free=free[:n_pages],
                pool=pool + torch.stack([take.sum(), give.sum()]))


def _plain_write(st):
    slots = st["slots"].long()
    n = st["k_pages"].shape[0] * st["k_pages"].shape[1]
    found = []
    for x in ("k", "v"):
        pages = st[x + "_pages"]
        flat = torch.cat([pages.view(n, *pages.shape[2:]), pages.new_zeros(1, *pages.shape[2:])])
        flat[torch.where(slots < 0, n, slots)] = st[x]
        found.append(flat[:n].view(pages.shape))
    return dict(k_pages=found[0], v_pages=found[1])


def run(state):
    st, op = state, state["case"]["op"]
    if not own:
        return {"prompt": _plain_prompt, "paged": _plain_paged, "tables": _plain_tables, "write": _plain_write}[op](st)
    import paper_2508_02401_gb300 as ckv
    if op == "prompt":
        ckv.ckv_prefill_attention(st["cfg"], st["batch"], st["q"], st["k"], st["v"], st["out"], st["ws"],
                                  lse=st["lse"], lse_win=st["lse_win"], tok_stride=st["tok_stride"])
        return dict(out=st["out"], lse=st["lse"], lse_win=st["lse_win"])
    if op == "paged":
        ckv.ckv_paged_attention(st["cfg"], st["cache"], st["table"], st["lens"], st["cu"], st["q"], st["out"],
                                st["ws"], lse=st["lse"])
        return dict(out=st["out"], lse=st["lse"])
    if op == "tables":
        ckv.ckv_block_tables(st["case"]["page"], st["lens"], st["new"], st["free"], st["pool"], st["table"],
                             st["slots"], st["cu"], st["lens_out"], st["pool_out"], st["ws"])
        return dict(table=st["table"], slots=st["slots"], cu=st["cu"], lens=st["lens_out"], free=st["free"],
                    pool=st["pool_out"])
    ckv.ckv_cache_write(st["cfg"], st["cache"], st["k"], st["v"], st["slots"], st["ws"])
    return dict(k_pages=st["k_pages"], v_pages=st["v_pages"])


# ------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """Attention row by row of heads, in 64 bits; the other operators move bits."""
    op = case["op"]
    if op not in ("prompt", "paged") or work(case)["flops"] > 4e12:
        return None
    st = prepare(case, seed)
    hq, hkv = case["q_heads"], case["kv_heads"]
    G, T = hq // hkv, st["q"].shape[0]
    out = torch.zeros((T, hq, D), dtype=torch.float64, device="cuda")
    lse = torch.zeros((hq, T), dtype=torch.float64, device="cuda")
    if op == "prompt":
        cu = [int(x) for x in st["cu"]]
        spans = [(a, b - a, torch.arange(a, b, device="cuda"), b - a) for a, b in zip(cu, cu[1:])]
        kk, vv = st["k"], st["v"]
    else:
        P, cu, spans = case["page"], [0], []
        for s, (L, n) in enumerate(zip(_ints(case["lens"]), _ints(case["new"]))):
            j = torch.arange(L, device="cuda")
            spans.append((cu[-1], n, st["table"][s, j // P].long() * P + j % P, L))
            cu.append(cu[-1] + n)
        kk, vv = st["k"].view(-1, hkv, D), st["v"].view(-1, hkv, D)
    for a, n, rows, L in spans:
        for g in range(hkv):
            k, v = kk[rows, g].double(), vv[rows, g].double()
            for h in range(g * G, (g + 1) * G):
                for i in range(0, n, 4096):
                    q = st["q"][a + i:a + min(n, i + 4096), h].double()
                    seen = L - n + i + len(q)
                    s = torch.einsum("id,jd->ij", q, k[:seen]) / math.sqrt(D)
                    over = torch.arange(seen, device="cuda") > (torch.arange(len(q), device="cuda") + seen - len(q))[:, None]
                    s[over] = -math.inf
                    l = torch.logsumexp(s, 1)
                    out[a + i:a + i + len(q), h] = torch.einsum("ij,jd->id", torch.exp(s - l[:, None]), v[:seen])
                    lse[h, a + i:a + i + len(q)] = l
    if op == "paged":
        return dict(out=out, lse=lse)
    w = case["window"]
    lse_win = torch.zeros((hq, len(spans) * w), dtype=torch.float64, device="cuda")
    for s, (a, n, _, _) in enumerate(spans):
        for r in range(w):
            if n - w + r >= 0:
                lse_win[:, s * w + r] = lse[:, a + n - w + r]
    return dict(out=out, lse=lse, lse_win=lse_win)


def work(case):
    op = case["op"]
    if op == "prompt":
        lens = _ints(case["lens"])
        hq, hkv, T = case["q_heads"], case["kv_heads"], sum(lens)
        pairs = sum(n * (n + 1) // 2 for n in lens)
        return dict(bytes=T * (hq * (2 * 256 + 4) + hkv * 2 * 256) + len(lens) * case["window"] * hq * 4,
                    flops=pairs * hq * D * 4)
    if op == "paged":
        lens, new = _ints(case["lens"]), _ints(case["new"])
        hq, hkv, T = case["q_heads"], case["kv_heads"], sum(new)
        pairs = sum(n * (L - n) + n * (n + 1) // 2 for L, n in zip(lens, new))
        pages = sum(-(-L // case["page"]) for L in lens)
        return dict(bytes=sum(lens) * hkv * 2 * 256 + T * hq * (2 * 256 + 4) + 4 * pages, flops=pairs * hq * D * 4)
    if op == "tables":
        n = case["rows"]
        new = (case["new_lo"] + case["new_hi"]) / 2 * n
        return dict(bytes=int(n * 16 + (n * case["new_hi"] + 5) * 4 + 8 * new / case["page"]), flops=0)
    kept = case["tokens"] - (-(-case["tokens"] // case["skip"]) if case["skip"] else 0)
    return dict(bytes=kept * case["kv_heads"] * 2 * 2 * 256 + case["tokens"] * 4, flops=0)
