// What the two attention kernels share (attention_tiles.cu: 256 query rows a CTA; attention_few.cu: a few query rows):
// the plan that cuts the units' key tiles over the CTAs, the loads of K and V tiles, and instructions.
//
// Query row i of a sequence with n query rows and L keys stands at position L - n + i and sees keys
// j <= L - n + i:  o = sum_j exp(c q.k_j - lse) v_j,  lse = log sum_j exp(c q.k_j).
//
// One pass over the keys in tiles of 128 (the online softmax): with a reference m of the row's logits,
// l = sum 2^(x_j - m) and o = sum 2^(x_j - m) v_j; when a tile's maximum passes m by more than 2^8, m
// moves there and l and o are multiplied by 2^(m_old - m_new).  A smaller excess is left (a published refinement of
// the online softmax): numerators up to 2^8 cost no precision, and the reference then hardly ever moves after a row's
// first tile.  The numerators are rounded to bf16 for the product with v (2^-8 of each at most): the tensor core takes two
// operands of one type, and v is bf16.  Their sum l takes them as they were, in 32 bits.
//
// A unit is (sequence, row tile, block of a KV head's query heads); its rows are (token, head) pairs,
// token major, so that the heads that share keys share the tile.  The units stand in order on a line, each
// with a fixed cost (in key tiles) and then its key tiles, and the line is cut into one run of equal length per
// CTA.  A unit that several CTAs share is joined by the last of them to finish, from partial results in the
// workspace, in order of its parts: the result does not depend on which CTA that is.  Every CTA finds its
// run from the lengths on the device.
#pragma once

#include <limits.h>

#include "ckv_device.cuh"
#include "ckv_internal.h"
#include "score_common.cuh"

namespace ckv {
namespace {

// A row's reference moves when a tile's maximum passes it by 2^8.
constexpr float kAttnTau = 8.0f;
constexpr int kAttnItemRing = 4;

struct alignas(128) AttnParams {
    CUtensorMap tmap_q;  // {128, H_q, T}, box {64, hp, tp}   (attention_tiles.cu)
    CUtensorMap tmap_k;  // {128, H_kv, T}, box {64, 1, 128}, or pages {128, H_kv, page_size, num_pages}, box
    CUtensorMap tmap_v;  //   {64, 1, page_size, 1}
    AttnLaunch a;
    int G, hp, tp, nhb;  // heads of a KV group; heads and tokens of a row tile; head blocks of a group
    int unit_cost;       // what a unit costs beside its key tiles, in key tiles
    int min_run;         // length of a CTA's run, at least
    int whole_tiles;     // units of up to so many key tiles are not cut
    float join_cost;     // what the join of a unit's part costs, in key tiles (0: nothing to speak of)
    int page_shift;
    float c;             // scale * log2(e)
    long long wait_cycles;
};

// One unit's part in this CTA.  `part` is -1 for a whole unit.
struct Item {
    int q_row, ntok, pos0, len;    // first query row (of q), tokens, position of the first, keys
    int kv0, head0, g, nheads;     // first key row (packed), first query head, KV head, heads
    int t0, n[2];                  // first key tile; tiles of either warpgroup (attention_tiles.cu)
    int n_tiles;                   // key tiles
    int seq, part, n_parts, cta0;  // part of n_parts, the first of them in CTA cta0
};
static_assert(sizeof(Item) == 64, "Item");
constexpr int kEndItem = -2;  // Item::part

// ---------------------------------------------------------------------------- instructions
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2,
                                            int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}

// Shared-memory matrix descriptors with the 128-byte swizzle as two words: the high one is constant (8-row
// groups 1024 bytes apart), the low one the address in 16-byte units and the leading offset.
//   K-major (Q, K): rows of 64 dims, the other 64 dims 16 KB further on (a separate descriptor).
//   N (or M) contiguous (V as [key][dim]): 64-dim halves 16 KB apart (the leading offset), 8-key groups 1024 bytes.
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
constexpr uint32_t kDescLoK = 1u << 16, kDescLoV = static_cast<uint32_t>(kHalfBytes >> 4) << 16;
__device__ __forceinline__ uint32_t desc_addr(const void* p) { return (smem_u32(p) & 0x3FFFFu) >> 4; }

// D[tmem] (+)= A[smem] * B[smem], one elected thread; A's descriptor with kDescHi, B's with B_HI.
template <uint32_t B_HI>
__device__ __forceinline__ void umma_ss(uint32_t d_tmem, uint32_t a_lo, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %6};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_lo), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(kDescHi), "n"(B_HI)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem].  A: 128 rows (lanes), 16 bf16 in 8 columns.
__device__ __forceinline__ void umma_ts(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 b;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "mov.b64 b, {%2, %5};\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "r"(b_lo), "r"(idesc), "r"(accumulate), "n"(kDescHi)
        : "memory");
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// Waits that a warp agrees on (false: give up).
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort, long long lim) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort, lim));
}

// The waits for a tile, several in a row on the path from one product to the next, where a vote costs 1% and more.
// One that gives up (or finds that another has) returns like the others: what follows works on whatever the
// buffers hold, at addresses that are valid all the same, and the roles leave at their next item, whose waits
// are agreed on.  The result is for the MMA issuers: after a wait that gave up, a later one on the same barrier can take
// the phase before for its own, so from then on they release no tile, and the loader never loads over one that is still on its
// way.
__device__ __forceinline__ bool tile_wait(uint64_t* bar, uint32_t parity, volatile int* abort, long long lim, int* status) {
    if (mbar_wait(bar, parity, abort, lim)) return true;
    *abort = 1;
    record_error(status, kDevTimeout, 45);
    return false;
}

// A value that all lanes hold, in a uniform register.
__device__ __forceinline__ int uniform(int v) { return __reduce_max_sync(0xffffffffu, v); }

// Rows [valid, 128) of a V tile (MMA issuers, a whole warp): behind the sequence's end they hold anything, and
// while their numerators are 0, 0 * NaN is not.
__device__ __forceinline__ void clear_rows(uint8_t* tile, int valid, int lane) {
    for (int x = valid * 8 + lane; x < kTileKeys * 8; x += 32) {
        *reinterpret_cast<uint4*>(tile + x * 16) = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(tile + kHalfBytes + x * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    fence_proxy_async_smem();
}

// ---------------------------------------------------------------------------- the plan
// Sum over i < n of floor((a i + b) / m), by the steps of Euclid's algorithm on (a, m): the known recursion for sums
// of floors, which swaps the two after each division.
__device__ inline unsigned long long floor_sum(unsigned long long n, unsigned long long m, unsigned long long a,
                                               unsigned long long b) {
    unsigned long long s = 0;
    while (n > 0) {
        s += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m;
        b %= m;
        const unsigned long long y = a * n + b;
        if (y < m) break;
        n = y / m;
        b = y % m;
        const unsigned long long t = m;
        m = a;
        a = t;
    }
    return s;
}

struct Seq {
    int row0, n, len;  // first query row, query rows (0: nothing to do), keys
};

// Sequence s; `bad` if cu is out of order (then nothing of the call is done), n = 0 and a status if only
// its length makes no sense.
__device__ __forceinline__ Seq get_seq(const AttnLaunch& a, int s, int cu0, bool& bad, bool report) {
    const int c0 = a.cu[s], c1 = a.cu[s + 1];
    bad |= c1 < c0 || c0 < cu0 || static_cast<long long>(c1) - cu0 > a.T;
    Seq q{c0 - cu0, c1 - c0, c1 - c0};
    if (a.lens) {
        q.len = a.lens[s];
        if (q.len < q.n || q.len > static_cast<long long>(a.max_blocks) * a.page_size) {
            if (report) record_error(a.status, kDevBadIndex, s);
            q.n = 0;
        }
    }
    return q;
}

// Key tiles of row tile j (of tq tokens) of a sequence, and the cost of the row tiles before it (j = nj: of all).
__device__ __forceinline__ int unit_tiles(const Seq& q, int tq, int j) {
    return (q.len - q.n + min((j + 1) * static_cast<long long>(tq), static_cast<long long>(q.n)) - 1) / kTileKeys + 1;
}
__device__ __forceinline__ long long cost_before(const AttnParams& p, const Seq& q, int tq, int j, int nj) {
    const int full = j == nj ? nj - 1 : j;
    long long s = static_cast<long long>(j) * p.unit_cost;
    if (full > 0) s += static_cast<long long>(floor_sum(full, kTileKeys, tq, q.len - q.n + tq - 1)) + full;
    return j == nj && nj > 0 ? s + unit_tiles(q, tq, nj - 1) : s;
}

// This CTA's run: positions [w0, w1) of the line, of W over `ctas` CTAs; CTA b's begins at floor(b W / ctas).
struct Run {
    long long w0, w1, W;
    int ctas;
    // the CTA of position x
    __device__ int cta_of(long long x) const { return static_cast<int>(((x + 1) * ctas - 1) / W); }
};
// Where it begins: sequence s, and w0's offset in it.
struct RunStart {
    long long offset;
    Seq q;
    int s;
};
constexpr int kScanBytes = 14 * 8 + static_cast<int>(sizeof(RunStart)) + 14 * 4;

// Whole block; false (for all of it): nothing to do.  `scan`: kScanBytes of shared memory, the RunStart in it
// to be read after the next barrier.
__device__ __forceinline__ RunStart* run_start(long long* scan) { return reinterpret_cast<RunStart*>(scan + 14); }
template <int THREADS>
__device__ __forceinline__ bool find_run(const AttnParams& p, int tq, int heads, long long* scan, Run& r) {
    static_assert(THREADS / 32 <= 14, "scan");
    const AttnLaunch& a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cu0 = a.cu[0];
    const int per = (a.S - 1) / THREADS + 1;
    const int s_lo = min(static_cast<long long>(threadIdx.x) * per, static_cast<long long>(a.S));
    const int s_hi = s_lo + min(per, a.S - s_lo);
    auto cost = [&](const Seq& q) {
        const int nj = (q.n + tq - 1) / tq;
        return q.n > 0 ? heads * cost_before(p, q, tq, nj, nj) : 0ll;
    };
    int* scan_units = reinterpret_cast<int*>(run_start(scan) + 1);
    long long own = 0;
    int units = 0;
    bool bad = false;
    Seq q{0, 0, 0};
    for (int s = s_lo; s < s_hi; ++s) {
        q = get_seq(a, s, cu0, bad, blockIdx.x == 0);
        own += cost(q);
        units += (q.n + tq - 1) / tq;
    }
    units = __reduce_add_sync(0xffffffffu, units);
    long long incl = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) {
        scan[warp] = incl;
        scan_units[warp] = units;
    }
    bad = __syncthreads_or(bad);
    long long before = incl - own;
    r.W = 0;
    units = 0;
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) {
        if (i < warp) before += scan[i];
        r.W += scan[i];
        units += scan_units[i];
    }
    // The host's copy of a batch is in order and has tokens (a call without any is not launched): no need of its hash.
    if ((bad || (r.W == 0 && a.check_hash)) && blockIdx.x == 0 && threadIdx.x == 0)
        record_error(a.status, a.check_hash ? kDevBadSeqlens : kDevBadIndex, -1);
    if (bad || r.W == 0) return false;
    // A unit of k tiles in runs of r of them takes r and its k / r parts' joins: least at r = sqrt(k join_cost).
    int least = p.min_run;
    if (p.join_cost > 0.f)
        least = max(least, static_cast<int>(sqrtf(p.join_cost * static_cast<float>(r.W) / (static_cast<float>(units) * heads))));
    const long long most = (r.W + least - 1) / least;
    r.ctas = most < gridDim.x ? static_cast<int>(most) : static_cast<int>(gridDim.x);
    const int b = blockIdx.x;
    if (b >= r.ctas) return false;
    const long long each = r.W / r.ctas;
    const int left = static_cast<int>(r.W - each * r.ctas);
    r.w0 = each * b + b * left / r.ctas;
    r.w1 = each * (b + 1) + (b + 1) * left / r.ctas;
    if (r.w0 >= before && r.w0 < before + own) {  // the thread whose sequences hold w0
        RunStart* st = run_start(scan);
        int s = s_lo;
        if (per > 1) {
            for (;; ++s) {
                bool ignore = false;
                q = get_seq(a, s, cu0, ignore, false);
                const long long w = cost(q);
                if (r.w0 < before + w) break;
                before += w;
            }
        }
        st->offset = r.w0 - before;
        st->q = q;
        st->s = s;
    }
    return true;
}

// Whether cu on the device is the host's copy (seqlens_hash, by a whole warp: some 30 cycles an entry, which is why
// a warp without another job does it; not inlined: beside the tiles kernel's loops it cost them 5%).
__device__ __noinline__ void check_seqlens(const AttnLaunch& a) {
    const int lane = threadIdx.x & 31;
    uint32_t h = 2166136261u;
    for (int i0 = 0; i0 <= a.S; i0 += 32) {
        const uint32_t v = i0 + lane <= a.S ? static_cast<uint32_t>(a.cu[i0 + lane]) : 0u;
        for (int i = 0; i < 32 && i0 + i <= a.S; ++i) h = (h ^ __shfl_sync(0xffffffffu, v, i)) * 16777619u;
    }
    if (lane == 0 && h != a.cu_hash) record_error(a.status, kDevBadSeqlens, 120);
}

// The items of a run, one after the other (a whole warp).
struct Walk {
    const AttnParams& p;
    const Run& r;
    const int tq, heads;
    Seq q;
    int s, nj, j, hb, t0, kt;  // kt: key tiles of row tile j
    long long at;              // the position of tile t0

    __device__ Walk(const AttnParams& p_, const Run& r_, int tq_, int heads_, long long* scan)
        : p(p_), r(r_), tq(tq_), heads(heads_) {
        const RunStart* st = run_start(scan);
        s = st->s;
        q = st->q;
        nj = (q.n + tq - 1) / tq;
        long long off = st->offset;
        int lo = 0, hi = nj;  // the row tile that holds the offset: 32 candidates at a time
        while (hi - lo > 1) {
            const int step = (hi - lo + 31) / 32, cand = lo + (threadIdx.x & 31) * step;
            const bool le = cand < hi && heads * cost_before(p, q, tq, cand, nj) <= off;
            lo += (31 - __clz(__ballot_sync(0xffffffffu, le))) * step;
            hi = min(hi, lo + step);
        }
        j = lo;
        if (j > 0) off -= heads * cost_before(p, q, tq, j, nj);
        kt = unit_tiles(q, tq, j);
        const int cost = kt + p.unit_cost;
        hb = static_cast<int>(off / cost);
        t0 = static_cast<int>(off - static_cast<long long>(hb) * cost);
        at = r.w0 + max(0, p.unit_cost - t0);
        t0 = max(0, t0 - p.unit_cost);
        if (t0 > 0 && kt <= p.whole_tiles) {  // another CTA's
            at += kt - t0 + p.unit_cost;
            t0 = kt;
        }
    }

    // Item::n is left to the kernel.
    __device__ bool next(Item& I) {
        if (t0 == kt) {  // the next unit
            t0 = 0;
            if (++hb == heads) {
                hb = 0;
                if (++j == nj && at < r.w1) {
                    j = 0;
                    bool ignore = false;
                    const int cu0 = p.a.cu[0];
                    do {
                        if (++s >= p.a.S) break;
                        q = get_seq(p.a, s, cu0, ignore, false);
                    } while (q.n <= 0);
                    nj = (q.n + tq - 1) / tq;
                }
                if (at < r.w1) kt = unit_tiles(q, tq, j);
            }
        }
        if (at >= r.w1) {
            I.part = kEndItem;
            return false;
        }
        const int t1 = kt <= p.whole_tiles ? kt : static_cast<int>(min(static_cast<long long>(kt), t0 + (r.w1 - at)));
        const int g = p.nhb == 1 ? hb : hb / p.nhb, b = hb - g * p.nhb;
        I.ntok = min(tq, q.n - j * tq);
        I.q_row = q.row0 + j * tq;
        I.pos0 = q.len - q.n + j * tq;
        I.len = q.len;
        I.kv0 = q.row0;
        I.g = g;
        I.head0 = g * p.G + b * p.hp;
        I.nheads = min(p.hp, p.G - b * p.hp);
        I.t0 = t0;
        I.n_tiles = t1 - t0;
        I.seq = s;
        I.part = -1;
        I.n_parts = 1;
        I.cta0 = 0;
        if (t0 > 0 || t1 < kt) {
            const long long u0 = at - t0;
            I.cta0 = r.cta_of(u0);
            I.n_parts = r.cta_of(u0 + kt - 1) - I.cta0 + 1;
            I.part = static_cast<int>(blockIdx.x) - I.cta0;
        }
        at += I.n_tiles + p.unit_cost;
        t0 = kt;
        return true;
    }
};

// A CTA's partial results of ROWS unit rows (an unnormalised output row of 128, its reference, its sum): slot 1
// for the unit that begins in its run, 0 for one that an earlier CTA began.
template <int ROWS>
__device__ __forceinline__ float* partial_of(const AttnLaunch& a, int cta, bool begins) {
    return a.partials + (static_cast<size_t>(cta) * 2 + (begins ? 1 : 0)) * (ROWS * (kHeadDim + 2));
}

// Whether this CTA is the last of the unit's parts to arrive: one thread, after a barrier with those that wrote the
// part and before one with those that join them (a release covers what came before it by barriers, too).
__device__ __forceinline__ bool last_part(const AttnLaunch& a, const Item& I) {
    int* cnt = a.counters + I.cta0;
    int n;
    asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;" : "=r"(n) : "l"(cnt) : "memory");
    const bool last = n == I.n_parts - 1;
    if (last) *cnt = 0;  // left zero for the next call
    return last;
}

// WINDOW: the call has the window rows' lse as an output (prompts).
template <bool WINDOW>
__device__ __forceinline__ void write_lse(const AttnLaunch& a, const Item& I, int tok, int head, float mc, float l) {
    if (!a.lse && !(WINDOW && a.lse_win)) return;
    const float lse = (mc + lg2_approx(l)) * 0.6931471805599453f;  // (2^-22 of absolute error in the logarithm)
    const int t = I.q_row + tok, h = I.head0 + head;
    if (a.lse) a.lse[h * a.lse_stride + t] = lse;
    if (WINDOW && a.lse_win) {
        const int rw = I.pos0 + tok - (I.len - a.w);
        if (rw >= 0) a.lse_win[h * a.lse_win_stride + static_cast<long long>(I.seq) * a.w + rw] = lse;
    }
}

// ---------------------------------------------------------------------------- K and V tiles
// One warp loads an item's tiles into the ring: K0 V0 K1 V1 ...
template <bool PAGED, int RING>
struct TileLoader {
    const AttnParams& p;
    uint8_t* ring;
    uint64_t* full;
    uint64_t* freed;
    volatile int* abort;
    long long lim;
    uint32_t slot = 0, phase = 1, use = 0;

    __device__ bool load(const CUtensorMap* map, const Item& I, int u, int page, int first) {
        if (!warp_wait(&freed[slot], phase, abort, lim)) return false;
        const int lane = threadIdx.x & 31;
        uint8_t* d = ring + slot * kTileBytes;
        if (lane == 0) mbar_arrive_expect_tx(&full[slot], kTileBytes);
        __syncwarp();
        if (PAGED) {  // a lane a page
            const int ppt = kTileKeys >> p.page_shift;
            if (lane >= first && lane < first + ppt) {
                d += (lane - first) << (p.page_shift + 7);
                tma_load_4d(d, map, &full[slot], 0, I.g, 0, page);
                tma_load_4d(d + kHalfBytes, map, &full[slot], 64, I.g, 0, page);
            }
        } else if (lane == 0) {
            const int tok = I.kv0 + (I.t0 + u) * kTileKeys;
            tma_load_3d(d, map, &full[slot], 0, I.g, tok);
            tma_load_3d(d + kHalfBytes, map, &full[slot], 64, I.g, tok);
        }
        __syncwarp();
        ++use;
        if (++slot == RING) {
            slot = 0;
            phase ^= 1;
        }
        return true;
    }

    __device__ bool item(const Item& I) {
        // Page indices: lane l holds block l of a window of 32 blocks, the next window's at hand.
        const AttnLaunch& a = p.a;
        const int ppt_shift = PAGED ? 7 - p.page_shift : 0, win_shift = 5 - ppt_shift;  // pages a tile, tiles a window
        const int blocks = PAGED ? (I.len + a.page_size - 1) >> p.page_shift : 0;
        const int* row = PAGED ? a.table + static_cast<size_t>(I.seq) * a.max_blocks : nullptr;
        auto window = [&](int u) {
            const int b = ((I.t0 + u) << ppt_shift) + static_cast<int>(threadIdx.x & 31);
            int pg = a.num_pages;  // beyond the last page: the load fills with zeros
            if (PAGED && b < blocks && u < I.n_tiles) {
                pg = row[b];
                if (pg < 0 || pg >= a.num_pages) {
                    record_error(a.status, kDevBadIndex, I.seq);
                    pg = a.num_pages;
                }
            }
            return pg;
        };
        const int per = 1 << win_shift;
        int now = PAGED ? window(0) : 0, ahead = PAGED ? window(per) : 0;
        for (int u = 0; u < I.n_tiles; ++u) {
            if (PAGED && u > 0 && (u & (per - 1)) == 0) {
                now = ahead;
                ahead = window(u + per);
            }
            const int first = (u & (per - 1)) << ppt_shift;
            if (!load(&p.tmap_k, I, u, now, first) || !load(&p.tmap_v, I, u, now, first)) return false;
        }
        return true;
    }

    // Lets every issued copy land, before the block may exit: others' waits for them may have given up.
    __device__ void drain() {
        volatile int never = 0;
        for (uint32_t k = use > RING ? use - RING : 0; k < use; ++k) mbar_wait(&full[k % RING], (k / RING) & 1, &never);
    }
};

// Host: lets a kernel have its shared memory, once a device (a benign race: the call is idempotent).
constexpr int kAttnMaxDevices = 64;
template <class Kernel>
cudaError_t attn_configure(Kernel kern, int bytes, bool (&configured)[kAttnMaxDevices]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < kAttnMaxDevices && configured[dev]) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < kAttnMaxDevices) configured[dev] = true;
    return e;
}

}  // namespace
}  // namespace ckv
