// Causal attention of packed prompts and of new tokens over a paged cache.
//
// Query row i of a sequence with n query rows and L keys stands at position L - n + i and sees keys
// j <= L - n + i:  o = sum_j exp(c q.k_j - lse) v_j,  lse = log sum_j exp(c q.k_j).
//
// One pass over the keys in tiles of 128 (the online softmax): with a reference m of the row's logits,
// l = sum 2^(x_j - m) and o = sum 2^(x_j - m) v_j; when a tile's maximum passes m by more than 2^8, m
// moves there and l and o are multiplied by 2^(m_old - m_new).  A smaller excess is left: numerators up
// to 2^8 cost no precision, and the reference then hardly ever moves after a row's first tile.
//
// Work.  A unit is (sequence, row tile, block of a KV head's query heads).  The rows of a tile are
// (token, head) pairs, token major, so that the heads that share keys share the tile: hp heads of
// 128 / hp tokens fill the MMA's 128 rows.  With TILES = 2 a unit has two such tiles, which a CTA's two
// softmax warpgroups take one each against the same keys; with TILES = 1 it has one, and the warpgroups
// take its even and odd key tiles and join at the end.  The key tiles of all units, in order, are cut
// into one run of equal length per CTA.  A unit that several CTAs share is joined by the last of them
// to finish, from partial results in the workspace, in order of its parts: the result does not depend
// on which CTA that is.  Every CTA finds its run from the lengths on the device.
#include "ckv_device.cuh"
#include "ckv_internal.h"
#include "score_common.cuh"

namespace ckv {
namespace {

constexpr int kAttnThreads = 384;
constexpr int kAttnRing = 5;       // 32 KB tiles of K and V, in the order of their use
constexpr int kAttnItemRing = 4;
constexpr int kMmaWarp = 8, kLoadWarp = 9, kQWarp = 10;  // warps 0-3, 4-7: softmax; 10, 11: query rows
// A row's reference moves when a tile's maximum passes it by 2^8.
constexpr float kAttnTau = 8.0f;
// What a unit costs beside its key tiles, in key tiles: its first ones stand before its tiles in a run.
constexpr int kUnitCost = 3;

struct alignas(128) AttnParams {
    CUtensorMap tmap_q;  // {128, H_q, T}, box {64, hp, tp}   (TILES = 2)
    CUtensorMap tmap_k;  // {128, H_kv, T}, box {64, 1, 128}, or pages {128, H_kv, page_size, num_pages}, box
    CUtensorMap tmap_v;  //   {64, 1, page_size, 1}
    AttnLaunch a;
    int G, hp, tp, nhb;  // heads of a KV group; heads and tokens of a tile; head blocks of a group
    int min_run;         // key tiles of a CTA's run, at least
    int page_shift;
    float c;             // scale * log2(e)
    long long wait_cycles;
};

// One unit's part in this CTA.  `part` is -1 for a whole unit.
struct Item {
    int q_row, ntok, pos0, len;    // first query row (of q), tokens, position of the first, keys
    int kv0, head0, g, nheads;     // first key row (packed), first query head, KV head, heads
    int t0, n[2];                  // first key tile; tiles of either warpgroup
    int n_tiles;                   // key tiles loaded
    int seq, part, n_parts, cta0;  // part of n_parts, the first of them in CTA cta0
};
constexpr int kEndItem = -2;  // Item::part

struct AttnSmem {
    static constexpr int kRingOff = 0;
    static constexpr int kQ = kAttnRing * kTileBytes;
    static constexpr int kStats = kQ + 2 * kTileBytes;  // float2 [2][128]
    static constexpr int kItems = kStats + 2048;
    static constexpr int kBars = kItems + kAttnItemRing * static_cast<int>(sizeof(Item));
    static constexpr int kFull = 0, kFree = kFull + kAttnRing, kQFull = kFree + kAttnRing, kQFree = kQFull + 2,
                         kSFull = kQFree + 2, kPFull = kSFull + 2, kPvDone = kPFull + 2, kItemFull = kPvDone + 2,
                         kItemFree = kItemFull + kAttnItemRing, kPair = kItemFree + kAttnItemRing,
                         kDone = kPair + 1, kNumBars = kDone + 1;
    static constexpr int kScan = kBars + 8 * kNumBars;  // long long [16]
    static constexpr int kMisc = kScan + 8 * 16;        // TMEM base, abort, verdict, bad
    static constexpr int kBytes = kMisc + 16;
};
static_assert(AttnSmem::kBytes <= 232448, "shared memory");
static_assert(sizeof(Item) == 64, "Item");

// ---------------------------------------------------------------------------- instructions
__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2,
                                            int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(smem_u32(dst)),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(smem_u32(bar))
        : "memory");
}

// D[tmem] (+)= A[tmem] * B[smem], one elected thread.  A: 128 rows (lanes), 16 bf16 in 8 columns.
__device__ __forceinline__ void umma_bf16_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                             uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// An operand with its M or N dimension contiguous (V as [key][dim]): 128-byte rows of 64 dims, 8-key
// groups 1024 bytes apart, the two halves of the dims 16 KB apart.
__device__ __forceinline__ uint64_t sdesc_mn_major_sw128(uint32_t saddr) {
    uint64_t d = 0;
    d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
    d |= static_cast<uint64_t>(kHalfBytes >> 4) << 16;  // leading: between 64-dim halves
    d |= static_cast<uint64_t>(1024 >> 4) << 32;        // stride: between 8-key groups
    d |= static_cast<uint64_t>(1) << 46;
    d |= static_cast<uint64_t>(2) << 61;
    return d;
}
constexpr uint32_t kIdescQk = idesc_bf16_f32(128, 128);
constexpr uint32_t kIdescPv = idesc_bf16_f32(128, 128) | (1u << 16);  // B with N contiguous

__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
          "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
          "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
          "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void reg_fence32(float* v) {
#pragma unroll
    for (int i = 0; i < 32; ++i) asm volatile("" : "+f"(v[i]));
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
        "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]),
        "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]),
        "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
        : "memory");
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ---------------------------------------------------------------------------- the plan
// Sum over i < n of floor((a i + b) / m), by the steps of Euclid's algorithm on (a, m).
__device__ unsigned long long floor_sum(unsigned long long n, unsigned long long m, unsigned long long a,
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

// Key tiles of row tile j of a sequence, and the cost of the row tiles before it (j = nj: of all nj), in key
// tiles and kUnitCost for each.
__device__ __forceinline__ int unit_tiles(const Seq& q, int tq, int j) {
    return (q.len - q.n + min((j + 1) * static_cast<long long>(tq), static_cast<long long>(q.n)) - 1) / kTileKeys + 1;
}
__device__ __forceinline__ long long cost_before(const Seq& q, int tq, int j, int nj) {
    const int full = j == nj ? nj - 1 : j;
    long long s = static_cast<long long>(j) * kUnitCost;
    if (full > 0) s += static_cast<long long>(floor_sum(full, kTileKeys, tq, q.len - q.n + tq - 1)) + full;
    return j == nj && nj > 0 ? s + unit_tiles(q, tq, nj - 1) : s;
}

// ---------------------------------------------------------------------------- the kernel
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity, volatile int* abort, long long lim) {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort, lim));
}

// Barrier of the 256 softmax threads (8 arrivals).
__device__ __forceinline__ bool pair_sync(uint64_t* bar, uint32_t& phase, volatile int* abort, long long lim) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
    const bool ok = warp_wait(bar, phase, abort, lim);
    phase ^= 1;
    return ok;
}

template <bool PAGED, int TILES>
__global__ void __launch_bounds__(kAttnThreads, 1) attention_kernel(const __grid_constant__ AttnParams p) {
    using SM = AttnSmem;
    constexpr int kRows = 128 * TILES;  // rows of a unit
    extern __shared__ __align__(1024) uint8_t sm[];
    uint8_t* ring = sm + SM::kRingOff;
    uint8_t* qbuf = sm + SM::kQ;
    float2* stats = reinterpret_cast<float2*>(sm + SM::kStats);
    Item* items = reinterpret_cast<Item*>(sm + SM::kItems);
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + SM::kBars);
    uint64_t* full = bars + SM::kFull;
    uint64_t* freed = bars + SM::kFree;
    uint64_t* q_full = bars + SM::kQFull;
    uint64_t* q_free = bars + SM::kQFree;
    uint64_t* s_full = bars + SM::kSFull;
    uint64_t* p_full = bars + SM::kPFull;
    uint64_t* pv_done = bars + SM::kPvDone;
    uint64_t* item_full = bars + SM::kItemFull;
    uint64_t* item_free = bars + SM::kItemFree;
    uint64_t* pair = bars + SM::kPair;
    uint64_t* done = bars + SM::kDone;
    long long* scan = reinterpret_cast<long long*>(sm + SM::kScan);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + SM::kMisc);
    volatile int* abort = reinterpret_cast<volatile int*>(sm + SM::kMisc + 4);
    volatile int* verdict = reinterpret_cast<volatile int*>(sm + SM::kMisc + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const AttnLaunch& a = p.a;
    const int tq = TILES * p.tp;         // tokens of a unit
    const int heads = a.Hkv * p.nhb;     // units of a row tile
    if ((smem_u32(sm) & 1023u) != 0) {  // the swizzled tiles need an aligned base
        if (threadIdx.x == 0) record_error(a.status, kDevBadIndex, -2);
        return;
    }

    // ---- this CTA's run: positions [w0, w1) of all units' in order, a unit's being kUnitCost and its tiles
    const int cu0 = a.cu[0];
    const int per = (a.S + kAttnThreads - 1) / kAttnThreads;
    const int s_lo = min(static_cast<long long>(threadIdx.x) * per, static_cast<long long>(a.S));
    const int s_hi = min(s_lo + per, a.S);
    long long own = 0;
    bool bad = false;
    for (int s = s_lo; s < s_hi; ++s) {
        const Seq q = get_seq(a, s, cu0, bad, blockIdx.x == 0);
        const int nj = (q.n + tq - 1) / tq;
        if (q.n > 0) own += cost_before(q, tq, nj, nj);
    }
    own *= heads;
    long long incl = own;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) scan[warp] = incl;
    if (threadIdx.x == 0) *abort = 0;
    bad = __syncthreads_or(bad);
    long long before = incl - own, W = 0;
#pragma unroll
    for (int i = 0; i < kAttnThreads / 32; ++i) {
        if (i < warp) before += scan[i];
        W += scan[i];
    }
    if (blockIdx.x == 0 && threadIdx.x == kAttnThreads - 1) {
        if (a.check_hash && seqlens_hash(a.cu, a.S) != a.cu_hash) record_error(a.status, kDevBadSeqlens, 120);
        else if (bad) record_error(a.status, kDevBadIndex, -1);
    }
    if (bad || W == 0) return;
    long long ctas = (W + p.min_run - 1) / p.min_run;
    if (ctas > gridDim.x) ctas = gridDim.x;
    if (blockIdx.x >= ctas) return;
    const long long w0 = blockIdx.x * W / ctas, w1 = (blockIdx.x + 1) * W / ctas;
    if (w0 >= before && w0 < before + own) {  // the thread whose sequences hold w0
        long long at = before;
        for (int s = s_lo; s < s_hi; ++s) {
            bool b = false;
            const Seq q = get_seq(a, s, cu0, b, false);
            const int nj = (q.n + tq - 1) / tq;
            const long long w = q.n > 0 ? heads * cost_before(q, tq, nj, nj) : 0;
            if (w0 < at + w) {
                scan[13] = s;
                scan[14] = w0 - at;
                break;
            }
            at += w;
        }
    }

    if (threadIdx.x == 0) {
        for (int i = 0; i < kAttnRing; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&freed[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], TILES == 2 ? 1 : 2);
            mbar_init(&q_free[i], TILES == 2 ? 1 : 2);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 4);
            mbar_init(&pv_done[i], 1);
        }
        for (int i = 0; i < kAttnItemRing; ++i) {
            mbar_init(&item_full[i], 1);
            mbar_init(&item_free[i], TILES == 2 ? 9 : 11);  // softmax warps, the MMA issuer, the query loaders
        }
        mbar_init(pair, 8);
        mbar_init(done, 1);
        fence_mbar_init();
    }
    if (warp == kLoadWarp && lane == 0) {
        if (TILES == 2) tma_prefetch_desc(&p.tmap_q);
        tma_prefetch_desc(&p.tmap_k);
        tma_prefetch_desc(&p.tmap_v);
    }
    if (warp == kMmaWarp) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = *tmem_slot;
    // TMEM columns: S of either warpgroup at 0 and 128 (its P, in bf16, over the first 64), O at 256 and 384.
    const long long lim = p.wait_cycles;

    if (warp >= kMmaWarp) {
        // 384 threads * 168 = 128 * 72 + 256 * 216 registers
        setmaxnreg_dec<72>();
        if (warp == kLoadWarp) {
            // ------------------------------------------------------------ items, K and V tiles
            int s = static_cast<int>(scan[13]);
            long long off = scan[14], at = w0;
            bool ignore = false, ok = true;
            Seq q = get_seq(a, s, cu0, ignore, false);
            int nj = (q.n + tq - 1) / tq, j = 0, hb = 0, t0 = 0;
            {  // the row tile that holds `off`
                int lo = 0, hi = nj;
                while (hi - lo > 1) {
                    const int step = (hi - lo + 31) / 32, cand = lo + lane * step;
                    const bool le = cand < hi && heads * cost_before(q, tq, cand, nj) <= off;
                    const int top = 31 - __clz(__ballot_sync(0xffffffffu, le));
                    lo += top * step;
                    hi = min(hi, lo + step);
                }
                j = lo;
                off -= heads * cost_before(q, tq, j, nj);
                const int cost = unit_tiles(q, tq, j) + kUnitCost;
                hb = static_cast<int>(off / cost);
                t0 = static_cast<int>(off - static_cast<long long>(hb) * cost);
                at += max(0, kUnitCost - t0);  // the position of tile t0
                t0 = max(0, t0 - kUnitCost);
            }
            uint32_t use = 0, qn[2] = {0, 0};
            int it = 0;
            for (; ok; ++it) {
                const int slot = it % kAttnItemRing;
                if (!(ok = warp_wait(&item_free[slot], ((it / kAttnItemRing) & 1) ^ 1, abort, lim))) break;
                const bool end = at >= w1;
                Item I;
                if (!end) {
                    const int kt = unit_tiles(q, tq, j);
                    const int t1 = static_cast<int>(min(static_cast<long long>(kt), t0 + (w1 - at)));
                    const int g = hb / p.nhb, b = hb - g * p.nhb;
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
                    if (TILES == 2) {
                        const int ka = (I.pos0 + min(p.tp, I.ntok) - 1) / kTileKeys + 1;
                        I.n[0] = max(0, min(t1, ka) - t0);
                        I.n[1] = I.ntok > p.tp ? I.n_tiles : 0;
                    } else {
                        I.n[0] = (I.n_tiles + 1) >> 1;
                        I.n[1] = I.n_tiles >> 1;
                    }
                    I.seq = s;
                    I.part = -1;
                    I.n_parts = 1;
                    I.cta0 = 0;
                    if (t0 > 0 || t1 < kt) {  // the CTA of position x is floor(((x + 1) ctas - 1) / W)
                        const long long u0 = at - t0;
                        I.cta0 = static_cast<int>(((u0 + 1) * ctas - 1) / W);
                        I.n_parts = static_cast<int>(((u0 + kt) * ctas - 1) / W) - I.cta0 + 1;
                        I.part = static_cast<int>(blockIdx.x) - I.cta0;
                    }
                } else {
                    I.part = kEndItem;
                }
                if (lane == 0) {
                    items[slot] = I;
                    mbar_arrive(&item_full[slot]);
                }
                __syncwarp();
                if (end) break;
                if (TILES == 2) {  // the query rows, tile by tile
                    for (int X = 0; X < 2; ++X) {
                        if (I.n[X] == 0) continue;
                        if (!(ok = warp_wait(&q_free[X], (qn[X] & 1) ^ 1, abort, lim))) break;
                        ++qn[X];
                        if (lane == 0) {
                            mbar_arrive_expect_tx(&q_full[X], static_cast<uint32_t>(p.hp * p.tp * 256));
                            uint8_t* d = qbuf + X * kTileBytes;
                            tma_load_3d(d, &p.tmap_q, &q_full[X], 0, I.head0, I.q_row + X * p.tp);
                            tma_load_3d(d + kHalfBytes, &p.tmap_q, &q_full[X], 64, I.head0, I.q_row + X * p.tp);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                }
                // Page indices: lane l holds block l of a window of 32 blocks; two windows at hand.
                const int ppt_shift = PAGED ? 7 - p.page_shift : 0;  // pages per tile
                const int win_shift = 5 - ppt_shift;                 // tiles per window
                const int blocks = PAGED ? (I.len + a.page_size - 1) >> p.page_shift : 0;
                const int* row = PAGED ? a.table + static_cast<size_t>(s) * a.max_blocks : nullptr;
                int win = 0, page[2] = {0, 0};
                auto window = [&](int w) {
                    const int b = ((I.t0 + (w << win_shift)) << ppt_shift) + lane;
                    int pg = a.num_pages;  // beyond the last page: the load fills with zeros
                    if (b < blocks && (w << win_shift) < I.n_tiles) {
                        pg = row[b];
                        if (pg < 0 || pg >= a.num_pages) {
                            record_error(a.status, kDevBadIndex, s);
                            pg = a.num_pages;
                        }
                    }
                    return pg;
                };
                if (PAGED) {
                    page[0] = window(0);
                    page[1] = window(1);
                }
                auto load = [&](const CUtensorMap* map, int u) {
                    const uint32_t sl = use % kAttnRing;
                    if (!warp_wait(&freed[sl], ((use / kAttnRing) & 1) ^ 1, abort, lim)) return false;
                    uint8_t* d = ring + sl * kTileBytes;
                    if (lane == 0) mbar_arrive_expect_tx(&full[sl], kTileBytes);
                    __syncwarp();
                    if (PAGED) {
                        const int pg = (u >> win_shift) == win ? page[0] : page[1];
                        const int first = (u & ((1 << win_shift) - 1)) << ppt_shift;
                        if (lane >= first && lane < first + (1 << ppt_shift)) {
                            d += (lane - first) << (p.page_shift + 7);
                            tma_load_4d(d, map, &full[sl], 0, I.g, 0, pg);
                            tma_load_4d(d + kHalfBytes, map, &full[sl], 64, I.g, 0, pg);
                        }
                    } else if (lane == 0) {
                        const int tok = I.kv0 + (I.t0 + u) * kTileKeys;
                        tma_load_3d(d, map, &full[sl], 0, I.g, tok);
                        tma_load_3d(d + kHalfBytes, map, &full[sl], 64, I.g, tok);
                    }
                    __syncwarp();
                    ++use;
                    return true;
                };
                // The order in which the MMAs use them: K0 V0 K1 V1 ... or, with two key tiles at a time,
                // K0 K1 V0 K2 V1 K3 ... V(n-2) V(n-1).
                const int ahead = TILES == 2 ? 0 : 1;
                for (int u = -ahead; u < I.n_tiles && ok; ++u) {
                    if (u == -1) {
                        ok = load(&p.tmap_k, 0);
                        continue;
                    }
                    if (u + ahead < I.n_tiles) ok = load(&p.tmap_k, u + ahead);
                    if (PAGED && (u >> win_shift) != win) {
                        ++win;
                        page[0] = page[1];
                        page[1] = window(win + 1);
                    }
                    ok = ok && load(&p.tmap_v, u);
                }
                // the next unit
                at += I.n_tiles + kUnitCost;
                t0 = 0;
                if (++hb == heads) {
                    hb = 0;
                    if (++j == nj) {
                        j = 0;
                        do {
                            if (++s >= a.S) break;
                            q = get_seq(a, s, cu0, ignore, false);
                        } while (q.n <= 0);
                        nj = (q.n + tq - 1) / tq;
                    }
                }
            }
            if (!ok) {
                *abort = 1;
                if (lane == 0) record_error(a.status, kDevTimeout, 41);
                // let every issued copy land before the block may exit
                volatile int never = 0;
                for (uint32_t k = use > kAttnRing ? use - kAttnRing : 0; k < use; ++k)
                    mbar_wait(&full[k % kAttnRing], (k / kAttnRing) & 1, &never);
                for (int X = 0; X < 2; ++X)
                    if (TILES == 2 && qn[X] > 0) mbar_wait(&q_full[X], (qn[X] - 1) & 1, &never);
            }
            __syncwarp();
        } else if (warp == kMmaWarp) {
            // ------------------------------------------------------------ MMA issuer
            const bool leader = elect_one();
            const uint64_t k_desc = sdesc_k_major_sw128(smem_u32(ring));
            const uint64_t v_desc = sdesc_mn_major_sw128(smem_u32(ring));
            const uint64_t q_desc = sdesc_k_major_sw128(smem_u32(qbuf));
            uint32_t base = 0, qn[2] = {0, 0}, pn[2] = {0, 0};
            bool ok = true;
            Item I;
            int it = 0;
            auto fetch = [&]() {
                const int slot = it % kAttnItemRing;
                if (!warp_wait(&item_full[slot], (it / kAttnItemRing) & 1, abort, lim)) return false;
                I = items[slot];
                __syncwarp();
                if (leader) mbar_arrive(&item_free[slot]);
                __syncwarp();
                ++it;
                return true;
            };
            // the ring position of K and V tile i of warpgroup X
            auto k_pos = [&](int X, int i) {
                if (TILES == 2) return base + 2 * i;
                const int u = 2 * i + X;
                return base + (u < 2 ? u : 2 * u - 1);
            };
            auto v_pos = [&](int X, int i) {
                if (TILES == 2) return base + 2 * i + 1;
                const int u = 2 * i + X;
                return base + (u < I.n_tiles - 1 ? 2 * u + 2 : 2 * I.n_tiles - 1);
            };
            auto qk = [&](int X, int i) {
                int qs = X;
                if (i == 0) {  // the item's query rows
                    const uint32_t ph = TILES == 2 ? qn[X] & 1 : ((it - 1) >> 1) & 1;
                    qs = TILES == 2 ? X : (it - 1) & 1;
                    if (!warp_wait(&q_full[qs], ph, abort, lim)) return false;
                    if (TILES == 2) ++qn[X];
                } else if (TILES == 1) {
                    qs = (it - 1) & 1;
                }
                const uint32_t pos = k_pos(X, i), sl = pos % kAttnRing;
                if (!warp_wait(&full[sl], (pos / kAttnRing) & 1, abort, lim)) return false;
                tc_fence_after_sync();
                if (leader) {
                    const uint64_t ad = q_desc + static_cast<uint64_t>(qs * (kTileBytes >> 4));
                    const uint64_t bd = k_desc + static_cast<uint64_t>(sl * (kTileBytes >> 4));
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk) {
                        const uint64_t o = ((kk >> 2) * kHalfBytes + (kk & 3) * 32) >> 4;
                        umma_bf16(tmem_base + X * 128, ad + o, bd + o, kIdescQk, kk > 0 ? 1u : 0u);
                    }
                    umma_commit(&s_full[X]);
                    if (TILES == 1 || X == 1 || i >= I.n[1]) umma_commit(&freed[sl]);
                    if (i == I.n[X] - 1) umma_commit(&q_free[qs]);
                }
                __syncwarp();
                return true;
            };
            auto pv = [&](int X, int i) {
                const uint32_t pos = v_pos(X, i), sl = pos % kAttnRing;
                if (!warp_wait(&full[sl], (pos / kAttnRing) & 1, abort, lim)) return false;
                const int kt = I.t0 + (TILES == 2 ? i : 2 * i + X);
                const int valid = I.len - kt * kTileKeys;
                if (valid < kTileKeys && (TILES == 1 || X == 0 || i >= I.n[0])) {
                    // Rows behind the sequence's end hold anything; their numerators are 0, and 0 * NaN is not.
                    uint8_t* d = ring + sl * kTileBytes;
                    for (int x = valid * 8 + lane; x < kTileKeys * 8; x += 32) {
                        *reinterpret_cast<uint4*>(d + x * 16) = make_uint4(0u, 0u, 0u, 0u);
                        *reinterpret_cast<uint4*>(d + kHalfBytes + x * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                if (!warp_wait(&p_full[X], pn[X] & 1, abort, lim)) return false;
                ++pn[X];
                tc_fence_after_sync();
                if (leader) {
                    const uint64_t bd = v_desc + static_cast<uint64_t>(sl * (kTileBytes >> 4));
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_bf16_ta(tmem_base + 256 + X * 128, tmem_base + X * 128 + kk * 8,
                                     bd + static_cast<uint64_t>(kk * (2048 >> 4)), kIdescPv, i > 0 || kk > 0 ? 1u : 0u);
                    if (i == I.n[X] - 1) umma_commit(&pv_done[X]);
                    if (TILES == 1 || X == 1 || i >= I.n[1]) umma_commit(&freed[sl]);
                }
                __syncwarp();
                return true;
            };
            ok = fetch();
            while (ok && I.part != kEndItem) {
                if (TILES == 1 && I.n[1] == 0 && leader) mbar_arrive(&q_free[(it - 1) & 1]);  // no odd key tile
#pragma unroll
                for (int X = 0; X < 2; ++X)
                    if (ok && I.n[X] > 0) ok = qk(X, 0);
                const int n = max(I.n[0], I.n[1]);
                for (int i = 0; i < n && ok; ++i) {
#pragma unroll
                    for (int X = 0; X < 2; ++X) {
                        if (ok && i < I.n[X]) ok = pv(X, i);
                        if (ok && i + 1 < I.n[X]) ok = qk(X, i + 1);
                    }
                }
                base += 2 * I.n_tiles;
                ok = ok && fetch();
            }
            if (leader) {
                if (!ok) {
                    *abort = 1;
                    record_error(a.status, kDevTimeout, 42);
                }
                umma_commit(done);
            }
            __syncwarp();
            volatile int never = 0;
            mbar_wait(done, 0, &never);
            __syncwarp();
        } else if (TILES == 1) {
            // ------------------------------------------------------------ query rows (two warps)
            // Plain loads: a unit of single tokens has few rows, and TMA would fetch a whole tile.
            const int tid = threadIdx.x - kQWarp * 32;
            bool ok = true;
            for (int it = 0; ok; ++it) {
                const int slot = it % kAttnItemRing, qs = it & 1;
                if (!(ok = warp_wait(&item_full[slot], (it / kAttnItemRing) & 1, abort, lim))) break;
                const Item I = items[slot];
                __syncwarp();
                if (lane == 0) mbar_arrive(&item_free[slot]);
                if (I.part == kEndItem) break;
                if (!(ok = warp_wait(&q_free[qs], ((it >> 1) & 1) ^ 1, abort, lim))) break;
                const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q);
                uint8_t* dst = qbuf + qs * kTileBytes;
                const int chunks = I.ntok * p.hp * 16;
#pragma unroll 4
                for (int x = tid; x < chunks; x += 64) {
                    const int r = x >> 4, ch = x & 15;
                    const int t = r / p.hp, h = r - t * p.hp;
                    if (h >= I.nheads) continue;
                    const uint4 val = *reinterpret_cast<const uint4*>(
                        src + (I.q_row + t) * a.q_tok + (I.head0 + h) * a.q_head + ch * 8);
                    *reinterpret_cast<uint4*>(dst + (ch >> 3) * kHalfBytes + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = val;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&q_full[qs]);
                __syncwarp();
            }
            if (!ok) {
                *abort = 1;
                if (lane == 0) record_error(a.status, kDevTimeout, 43);
            }
        }
    } else {
        // ---------------------------------------------------------------- softmax, a row a thread
        setmaxnreg_inc<216>();
        const int X = warp >> 2, r = threadIdx.x & 127;
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_tmem = tmem_base + X * 128 + lane_base, o_tmem = tmem_base + 256 + X * 128 + lane_base;
        const int t_r = r / p.hp, h_r = r - t_r * p.hp;  // the row's token and head in its tile
        const int tok = t_r + (TILES == 2 ? X * p.tp : 0);
        const float c = p.c, tau = kAttnTau / p.c;
        uint32_t sn = 0, items_done = 0, pair_phase = 0;  // tiles and items with tiles, so far
        bool ok = true;
        for (int it = 0; ok; ++it) {
            const int slot = it % kAttnItemRing;
            if (!(ok = warp_wait(&item_full[slot], (it / kAttnItemRing) & 1, abort, lim))) break;
            const Item I = items[slot];
            __syncwarp();
            if (lane == 0) mbar_arrive(&item_free[slot]);
            if (I.part == kEndItem) break;
            const bool valid = t_r < p.tp && tok < I.ntok && h_r < I.nheads;
            const bool any = __any_sync(0xffffffffu, valid);
            const int pos = I.pos0 + tok;
            const int n = I.n[X];
            float m = -INFINITY, mc = 0.f, l = 0.f;  // reference (raw), times c, sum
            for (int i = 0; i < n; ++i, ++sn) {
                if (!(ok = warp_wait(&s_full[X], sn & 1, abort, lim))) break;
                if (any) {
                    tc_fence_after_sync();
                    float s[128];
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) tmem_ld32(s_tmem + q4 * 32, s + q4 * 32);
                    tmem_ld_wait();
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) reg_fence32(s + q4 * 32);
                    const int kt = I.t0 + (TILES == 2 ? i : 2 * i + X);
                    const int nv = valid ? pos + 1 - kt * kTileKeys : kTileKeys;  // keys of the tile the row sees
                    if (__any_sync(0xffffffffu, nv < kTileKeys)) {
#pragma unroll
                        for (int x = 0; x < 128; ++x) s[x] = x < nv ? s[x] : -INFINITY;
                    }
                    float mx[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) mx[x] = fmaxf(s[x], s[x + 8]);
#pragma unroll
                    for (int x = 16; x < 128; x += 16)
#pragma unroll
                        for (int y = 0; y < 8; ++y) mx[y] = max3(mx[y], s[x + y], s[x + y + 8]);
                    const float mt = max3(max3(mx[0], mx[1], mx[2]), max3(mx[3], mx[4], mx[5]), fmaxf(mx[6], mx[7]));
                    if (i == 0) {
                        m = mt;
                        mc = m == -INFINITY ? 0.f : m * c;
                    } else if (__any_sync(0xffffffffu, mt > m + tau)) {
                        // Move the reference of the rows that need it.  The last tile's product is in O: it was
                        // issued before this tile's logits, whose commit waits for all before it.
                        const float mn = mt > m + tau ? mt : m;
                        const float f = mn == m ? 1.f : ex2_approx((m - mn) * c);
#pragma unroll 1
                        for (int q4 = 0; q4 < 8; ++q4) {
                            float o[16];
                            tmem_ld16_nowait(o_tmem + q4 * 16, o);
                            tmem_ld_wait();
                            reg_fence(o);
#pragma unroll
                            for (int x = 0; x < 16; ++x) o[x] *= f;
                            tmem_st16(o_tmem + q4 * 16, o);
                        }
                        l *= f;
                        m = mn;
                        mc = m == -INFINITY ? 0.f : m * c;
                    }
                    float sum[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) sum[x] = 0.f;
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        uint32_t pk[32];
#pragma unroll
                        for (int x = 0; x < 64; x += 2) {
                            float* e = s + hf * 64 + x;
                            fma2(e[0], e[1], e[0], e[1], c, c, -mc, -mc);
                            e[0] = ex2_approx(e[0]);
                            e[1] = ex2_approx(e[1]);
                            float* t = sum + (x & 6);
                            add2(t[0], t[1], t[0], t[1], e[0], e[1]);
                            pk[x >> 1] = pack_bf16(e[0], e[1]);
                        }
                        tmem_st32(s_tmem + hf * 32, pk);
                    }
                    l += ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
                    tmem_st_wait();
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[X]);
                __syncwarp();
            }
            if (!ok) break;
            if (n > 0) {
                if (!(ok = warp_wait(&pv_done[X], items_done & 1, abort, lim))) break;
                ++items_done;
            }
            tc_fence_after_sync();
            if (m == -INFINITY) mc = -INFINITY;  // the row saw no key here
            // ---- the unit's (or this part's) result: columns [col0, col0 + cols) of the row
            constexpr int kCols = TILES == 2 ? 128 : 64;
            const int col0 = TILES == 2 ? 0 : X * 64;
            float fa = 1.f, fb = 0.f;  // weights of the warpgroups' results (TILES = 1)
            if (TILES == 1) {
                stats[X * 128 + r] = make_float2(mc, l);
                tc_fence_before_sync();
                if (!(ok = pair_sync(pair, pair_phase, abort, lim))) break;
                tc_fence_after_sync();
                const float2 sa = stats[r], sb = stats[128 + r];
                const float M = fmaxf(sa.x, sb.x);
                fa = sa.x == -INFINITY ? 0.f : ex2_approx(sa.x - M);
                fb = sb.x == -INFINITY ? 0.f : ex2_approx(sb.x - M);
                mc = M;
                l = sa.y * fa + sb.y * fb;
            }
            const bool whole = I.part < 0;
            float* part = nullptr;
            if (!whole)
                part = a.partials + (static_cast<size_t>(blockIdx.x) * 2 + (I.part == 0 ? 1 : 0)) * attn_partial_floats();
            const int row = TILES == 2 ? X * 128 + r : r;
            if (any && (TILES == 1 || n > 0)) {
                const float inv = whole ? 1.f / l : 1.f;
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) +
                                     (static_cast<long long>(I.q_row + tok) * a.Hq + I.head0 + h_r) * kHeadDim + col0;
#pragma unroll
                for (int q4 = 0; q4 < kCols / 32; ++q4) {
                    float o[32];
                    tmem_ld32((TILES == 2 ? o_tmem : tmem_base + 256 + lane_base) + col0 + q4 * 32, o);
                    if (TILES == 1 && I.n[1] > 0) {
                        float o2[32];
                        tmem_ld32(tmem_base + 384 + lane_base + col0 + q4 * 32, o2);
                        tmem_ld_wait();
                        reg_fence32(o);
                        reg_fence32(o2);
#pragma unroll
                        for (int x = 0; x < 32; ++x) o[x] = o[x] * fa + o2[x] * fb;
                    } else {
                        tmem_ld_wait();
                        reg_fence32(o);
                    }
                    if (!valid) continue;
                    if (whole) {
#pragma unroll
                        for (int x = 0; x < 32; x += 8)
                            *reinterpret_cast<uint4*>(out + q4 * 32 + x) =
                                make_uint4(pack_bf16(o[x] * inv, o[x + 1] * inv), pack_bf16(o[x + 2] * inv, o[x + 3] * inv),
                                           pack_bf16(o[x + 4] * inv, o[x + 5] * inv), pack_bf16(o[x + 6] * inv, o[x + 7] * inv));
                    } else {  // [column / 4][row] in fours
                        float4* d = reinterpret_cast<float4*>(part);
#pragma unroll
                        for (int x = 0; x < 32; x += 4)
                            d[((col0 + q4 * 32 + x) >> 2) * kRows + row] = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
                    }
                }
            }
            auto write_lse = [&](int tk, int hd, float mcv, float lv) {
                const float lse = (mcv + log2f(lv)) * 0.6931471805599453f;
                const int t = I.q_row + tk, h = I.head0 + hd;
                if (a.lse) a.lse[h * a.lse_stride + t] = lse;
                if (a.lse_win) {
                    const int rw = I.pos0 + tk - (I.len - a.w);
                    if (rw >= 0) a.lse_win[h * a.lse_win_stride + static_cast<long long>(I.seq) * a.w + rw] = lse;
                }
            };
            if (valid && (TILES == 2 || X == 0)) {
                if (whole) {
                    write_lse(tok, h_r, mc, l);
                } else {
                    part[kRows * 128 + row] = mc;
                    part[kRows * 129 + row] = l;
                }
            }
            if (TILES == 1 || !whole) {  // the other warpgroup has read O; the part is written
                if (!whole) __threadfence();
                tc_fence_before_sync();
                if (!(ok = pair_sync(pair, pair_phase, abort, lim))) break;
                tc_fence_after_sync();
            }
            if (!whole) {
                if (threadIdx.x == 0) {
                    int* cnt = a.counters + I.cta0;
                    const int before_me = atomicAdd(cnt, 1);
                    const bool last = before_me == I.n_parts - 1;
                    if (last) *cnt = 0;
                    *verdict = last;
                    __threadfence();
                }
                if (!(ok = pair_sync(pair, pair_phase, abort, lim))) break;
                if (*verdict) {
                    // this CTA finished last: join the parts
                    __threadfence();
                    auto part_of = [&](int k) {
                        return a.partials + (static_cast<size_t>(I.cta0 + k) * 2 + (k == 0 ? 1 : 0)) * attn_partial_floats();
                    };
                    if (TILES == 1 && I.ntok * p.hp <= 16) {
                        // few rows, perhaps many parts: four columns of a row a thread, four parts at a time
                        for (int e = threadIdx.x; e < 32 * 16; e += 256) {
                            const int rr = e & 15, c4 = e >> 4;
                            const int ti = rr / p.hp, hi = rr - ti * p.hp;
                            if (ti >= I.ntok || hi >= I.nheads) continue;
                            float M = -INFINITY, L = 0.f;
                            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                            for (int k0 = 0; k0 < I.n_parts; k0 += 4) {
                                float pm[4], pl[4];
                                float4 po[4];
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    pm[k] = -INFINITY;
                                    if (k0 + k >= I.n_parts) continue;
                                    const float* src = part_of(k0 + k);
                                    pm[k] = __ldcg(src + kRows * 128 + rr);
                                    pl[k] = __ldcg(src + kRows * 129 + rr);
                                    po[k] = __ldcg(reinterpret_cast<const float4*>(src) + c4 * kRows + rr);
                                }
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    if (pm[k] == -INFINITY) continue;  // no key seen: its values are not to be used
                                    const float Mn = fmaxf(M, pm[k]);
                                    const float f0 = M == -INFINITY ? 0.f : ex2_approx(M - Mn), f1 = ex2_approx(pm[k] - Mn);
                                    M = Mn;
                                    L = L * f0 + pl[k] * f1;
                                    acc.x = acc.x * f0 + po[k].x * f1;
                                    acc.y = acc.y * f0 + po[k].y * f1;
                                    acc.z = acc.z * f0 + po[k].z * f1;
                                    acc.w = acc.w * f0 + po[k].w * f1;
                                }
                            }
                            const float inv = 1.f / L;
                            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) +
                                                 (static_cast<long long>(I.q_row + ti) * a.Hq + I.head0 + hi) * kHeadDim + c4 * 4;
                            *reinterpret_cast<uint2*>(out) =
                                make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                            if (c4 == 0) write_lse(ti, hi, M, L);
                        }
                    } else if (valid) {  // a thread its row (half of it), part after part
                        float acc[kCols], M = -INFINITY, L = 0.f;
#pragma unroll
                        for (int x = 0; x < kCols; ++x) acc[x] = 0.f;
#pragma unroll 1
                        for (int k = 0; k < I.n_parts; ++k) {
                            const float* src = part_of(k);
                            const float pm = __ldcg(src + kRows * 128 + row), pl = __ldcg(src + kRows * 129 + row);
                            float4 po[kCols / 4];
#pragma unroll
                            for (int x = 0; x < kCols / 4; ++x)
                                po[x] = __ldcg(reinterpret_cast<const float4*>(src) + ((col0 >> 2) + x) * kRows + row);
                            if (pm == -INFINITY) continue;  // no key seen: its values are not to be used
                            const float Mn = fmaxf(M, pm);
                            const float f0 = M == -INFINITY ? 0.f : ex2_approx(M - Mn), f1 = ex2_approx(pm - Mn);
                            M = Mn;
                            L = L * f0 + pl * f1;
#pragma unroll
                            for (int x = 0; x < kCols / 4; ++x) {
                                acc[4 * x] = acc[4 * x] * f0 + po[x].x * f1;
                                acc[4 * x + 1] = acc[4 * x + 1] * f0 + po[x].y * f1;
                                acc[4 * x + 2] = acc[4 * x + 2] * f0 + po[x].z * f1;
                                acc[4 * x + 3] = acc[4 * x + 3] * f0 + po[x].w * f1;
                            }
                        }
                        const float inv = 1.f / L;
                        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) +
                                             (static_cast<long long>(I.q_row + tok) * a.Hq + I.head0 + h_r) * kHeadDim + col0;
#pragma unroll
                        for (int x = 0; x < kCols; x += 8)
                            *reinterpret_cast<uint4*>(out + x) =
                                make_uint4(pack_bf16(acc[x] * inv, acc[x + 1] * inv), pack_bf16(acc[x + 2] * inv, acc[x + 3] * inv),
                                           pack_bf16(acc[x + 4] * inv, acc[x + 5] * inv), pack_bf16(acc[x + 6] * inv, acc[x + 7] * inv));
                        if (col0 == 0) write_lse(tok, h_r, M, L);
                    }
                }
            }
        }
        if (!ok) {
            *abort = 1;
            if (lane == 0) record_error(a.status, kDevTimeout, 44);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == kMmaWarp) tmem_dealloc(tmem_base, 512);
}

template <bool PAGED, int TILES>
cudaError_t launch_variant(const AttnParams& p, int grid, cudaStream_t stream) {
    auto kern = attention_kernel<PAGED, TILES>;
    static bool configured = false;  // benign race: the attribute call is idempotent
    if (!configured) {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, AttnSmem::kBytes);
        if (e != cudaSuccess) return e;
        configured = true;
    }
    NvtxRange range("attention_kernel");
    kern<<<grid, kAttnThreads, AttnSmem::kBytes, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention(const AttnLaunch& L, const CUtensorMap& map_q, const CUtensorMap& map_k,
                             const CUtensorMap& map_v, int tiles, cudaStream_t stream) {
    AttnParams p;
    p.tmap_q = map_q;
    p.tmap_k = map_k;
    p.tmap_v = map_v;
    p.a = L;
    p.G = L.Hq / L.Hkv;
    p.hp = attn_heads_per_tile(L.Hq, L.Hkv);
    p.tp = kTileKeys / p.hp;
    p.nhb = (p.G + p.hp - 1) / p.hp;
    p.min_run = 4;
    p.page_shift = 0;
    while ((1 << p.page_shift) < L.page_size) ++p.page_shift;
    p.c = L.scale * 1.4426950408889634f;
    p.wait_cycles = wait_limit_cycles();
    int grid = device_sm_count();
    if (grid <= 0) return cudaErrorNoDevice;
    if (grid > kAttnMaxCtas) grid = kAttnMaxCtas;
    if (L.max_ctas > 0 && L.max_ctas < grid) grid = L.max_ctas;
    if (L.paged) return tiles == 2 ? launch_variant<true, 2>(p, grid, stream) : launch_variant<true, 1>(p, grid, stream);
    return tiles == 2 ? launch_variant<false, 2>(p, grid, stream) : launch_variant<false, 1>(p, grid, stream);
}

}  // namespace ckv
