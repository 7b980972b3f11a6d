// Attention with two row tiles of 128 (token, head) rows a CTA (attention_common.cuh): prompts, and chunks of new
// tokens over a paged cache.
//
// hp heads of 128 / hp tokens fill the MMA's 128 rows.  A CTA's two softmax warpgroups take a row tile each, a
// row a thread, against the same K and V tiles; S = Q K^T comes from the tensor core into TMEM, the numerators go
// back in bf16 over it, and O += P V takes them from there.
//
// Bound by the power limit and, before it, by the path from one product to the next.  A key tile takes
// the tensor core 2048 cycles (four products of 128 x 128 x 128, 512 each, the rate that MMAs issued back to back
// reach).  One prompt of 32768 tokens (32 / 8 heads): 1475 TFLOP/s at 1375 W and 1670 MHz, where the tensor core is at
// work 72% of the time; without its loads (a copy that skipped them) 1820.
#include <type_traits>

#include "attention_common.cuh"

namespace ckv {
namespace {

constexpr int kThreadsT = 384;
constexpr int kRingT = 5;  // K and V tiles of 32 KB
constexpr int kMmaWarp = 8, kLoadWarp = 10;  // warps 0-3, 4-7: softmax; 8, 9: the MMAs of either
constexpr int kRowsT = 256;
static_assert(static_cast<size_t>(kAttnTilesCtas) * 2 * kRowsT * 130 <= kAttnPartialFloats, "workspace");

struct TilesSmem {
    static constexpr int kQ = kRingT * kTileBytes;
    static constexpr int kItems = kQ + 2 * kTileBytes;
    static constexpr int kBars = kItems + kAttnItemRing * static_cast<int>(sizeof(Item));
    static constexpr int kFull = 0, kFree = kFull + kRingT, kQFull = kFree + kRingT, kQFree = kQFull + 2,
                         kSFull = kQFree + 2, kPFull = kSFull + 2, kPvDone = kPFull + 2, kTurn = kPvDone + 2,
                         kItemFull = kTurn + 2, kItemFree = kItemFull + kAttnItemRing,
                         kPair = kItemFree + kAttnItemRing, kDone = kPair + 1, kNumBars = kDone + 1;
    static constexpr int kScan = kBars + 8 * kNumBars;
    static constexpr int kMisc = kScan + kScanBytes;  // TMEM base, abort, verdict
    static constexpr int kBytes = kMisc + 16;
};
static_assert(TilesSmem::kBytes <= 232448, "shared memory");

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
__device__ __forceinline__ void tmem_st16u(uint32_t taddr, const uint32_t* v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
        "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}

// 16 bf16 of a row; a thread's rows lie apart, so whole 32-byte sectors where the alignment allows.
__device__ __forceinline__ void store_bf16(__nv_bfloat16* out, const uint32_t* v, bool wide) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                     "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                     : "memory");
    } else {
        reinterpret_cast<uint4*>(out)[0] = make_uint4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<uint4*>(out)[1] = make_uint4(v[4], v[5], v[6], v[7]);
    }
}

// Barrier of the 256 softmax threads (8 arrivals).
__device__ __forceinline__ bool pair_sync(uint64_t* bar, uint32_t& phase, volatile int* abort, long long lim) {
    __syncwarp();
    if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
    const bool ok = warp_wait(bar, phase, abort, lim);
    phase ^= 1;
    return ok;
}

template <bool PAGED>
__global__ void __launch_bounds__(kThreadsT, 1) attention_tiles_kernel(const __grid_constant__ AttnParams p) {
    using SM = TilesSmem;
    extern __shared__ __align__(1024) uint8_t sm[];
    uint8_t* ring = sm;
    uint8_t* qbuf = sm + SM::kQ;
    Item* items = reinterpret_cast<Item*>(sm + SM::kItems);
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + SM::kBars);
    uint64_t* full = bars + SM::kFull;
    uint64_t* freed = bars + SM::kFree;
    uint64_t* q_full = bars + SM::kQFull;
    uint64_t* q_free = bars + SM::kQFree;
    uint64_t* s_full = bars + SM::kSFull;
    uint64_t* p_full = bars + SM::kPFull;
    uint64_t* pv_done = bars + SM::kPvDone;
    uint64_t* turn = bars + SM::kTurn;
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
    const int tq = 2 * p.tp, heads = a.Hkv * p.nhb;  // tokens of a unit; units of a row tile
    if ((smem_u32(sm) & 1023u) != 0) {               // the swizzled tiles need an aligned base
        if (threadIdx.x == 0) record_error(a.status, kDevBadIndex, -2);
        return;
    }
    if (threadIdx.x == 0) {
        *abort = 0;
        for (int i = 0; i < kRingT; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&freed[i], 2);  // the MMA issuers
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_free[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 4);
            mbar_init(&pv_done[i], 1);
            mbar_init(&turn[i], 1);
        }
        for (int i = 0; i < kAttnItemRing; ++i) {
            mbar_init(&item_full[i], 1);
            mbar_init(&item_free[i], 10);  // softmax warps, MMA issuers
        }
        mbar_init(pair, 8);
        mbar_init(done, 2);
        fence_mbar_init();
    }
    if (warp == kLoadWarp && lane == 0) {
        tma_prefetch_desc(&p.tmap_q);
        tma_prefetch_desc(&p.tmap_k);
        tma_prefetch_desc(&p.tmap_v);
    }
    if (warp == kMmaWarp) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    Run run;
    const bool busy = find_run<kThreadsT>(p, tq, heads, scan, run);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (!busy) {
        if (warp == kMmaWarp) tmem_dealloc(*tmem_slot, 512);
        return;
    }
    // TMEM columns (all are allocated, so they start at 0), + 128 X: the logits S of warpgroup X and, over their
    // first 64, its numerators P in bf16; its output O.
    constexpr uint32_t kTmS = 0, kTmO = 256;
    const long long lim = p.wait_cycles;

    // -------------------------------------------------------------------- MMA issuers, one a softmax warpgroup
    // S = Q K^T and O += P V of warpgroup X.  The two take turns: the tensor core holds up an issue of eight MMAs until
    // some 200 cycles before it is done with them, and with one issuer for both, its waits between the products
    // (about 560 cycles for each) left the tensor core idle; without turns the warpgroups' products interleave and finish
    // together, with nothing to overlap the softmaxes (one prompt of 8192 tokens, on one box: 374 us with one issuer, 436
    // without turns, 367 so; 370 to 400 by box).  An issuer waits for its tiles while the other issues.
    // The next logits go over the numerators of the tile before: their MMAs follow, from the same thread, those of the
    // product that reads them, and the tensor core takes one thread's MMAs in the order of their issue.
    // A turn is the product of a tile and then the logits of the warpgroup's next (or of its next unit's first):
    // its softmax runs in the other's turn.
    auto mma_role = [&](auto xc) {
        constexpr int X = decltype(xc)::value;
        constexpr uint32_t kTileUnits = kTileBytes >> 4;
        const uint32_t ring_addr = desc_addr(ring), q_addr = desc_addr(qbuf);
        int n0_ = 0, n1_ = 0, keys_ = 0, end_ = 0;  // the next item: tiles of either warpgroup, keys from its first tile on
        uint32_t qn = 0, pn = 0, turns = 0;         // items, tiles and turns of this one
        uint32_t cs = 0, cph = 0;                   // ring slot and phase of the current tile's K
        int it = 0;
        bool ok = true, live = true;  // live (a lane's own): none of its waits for a tile gave up
        auto fetch = [&]() {
            const int slot = it % kAttnItemRing;
            if (!warp_wait(&item_full[slot], (it / kAttnItemRing) & 1, abort, lim)) return false;
            end_ = uniform(items[slot].part == kEndItem);
            n0_ = uniform(items[slot].n[0]);
            n1_ = uniform(items[slot].n[1]);
            keys_ = uniform(items[slot].len - items[slot].t0 * kTileKeys);
            __syncwarp();
            if (elect_one()) mbar_arrive(&item_free[slot]);
            __syncwarp();
            ++it;
            return true;
        };
        auto slot_of = [&](uint32_t d) { return cs + d >= kRingT ? cs + d - kRingT : cs + d; };  // d after the current K
        auto phase_of = [&](uint32_t d) { return cs + d >= kRingT ? cph ^ 1 : cph; };
        // One turn: the product of the current tile (`do_pv`; of its V, `valid` rows are the sequence's) and the logits
        // of one (`do_qk`; K at ring position kd, with an item's first tile also its query rows).  `has_v`, `has_k`: there are
        // such tiles, whether or not this warpgroup has a part in them.  Both issuers release every tile: a commit
        // covers only the MMAs of its own thread.  One without a part in a tile arrives plainly, after it has seen the tile
        // in the ring too: the slot's release before that load is then complete, so it never arrives twice in one.
        auto play = [&](bool do_pv, bool first_v, bool last_v, bool has_v, int valid, bool clear, bool do_qk, uint32_t kd,
                        bool first_q, bool last_q, bool has_k) {
            const uint32_t ks = slot_of(kd), vs = slot_of(1);
            // (uniform registers)
            const uint32_t q_lo = uniform((q_addr + X * kTileUnits) | kDescLoK);
            const uint32_t k_lo = uniform((ring_addr + ks * kTileUnits) | kDescLoK);
            const uint32_t v_lo = uniform((ring_addr + vs * kTileUnits) | kDescLoV);
            const uint32_t accumulate = uniform(first_v ? 0 : 1);
            if (do_qk && first_q) {
                if (!warp_wait(&q_full[X], qn & 1, abort, lim)) return false;
                ++qn;
            }
            if (has_k) live &= tile_wait(&full[ks], phase_of(kd), abort, lim, a.status);
            if (has_v) live &= tile_wait(&full[vs], phase_of(1), abort, lim, a.status);
            if (do_pv) {
                if (valid < kTileKeys && clear) clear_rows(ring + vs * kTileBytes, valid, lane);
                tile_wait(&p_full[X], pn & 1, abort, lim, a.status);
                ++pn;
            }
            // this one's k-th turn comes after the other's k-th (X = 1) or (k - 1)-th (X = 0)
            tile_wait(&turn[X], (turns & 1) ^ (X == 0 ? 1 : 0), abort, lim, a.status);
            ++turns;
            __syncwarp();
            tc_fence_after_sync();
            if (elect_one()) {
                if (do_pv) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_ts(kTmO + X * 128, kTmS + X * 128 + kk * 8, v_lo + kk * (2048 >> 4), kIdescPv,
                                kk > 0 ? 1u : accumulate);
                    if (last_v) umma_commit(&pv_done[X]);
                }
                if (do_qk) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk) {
                        constexpr uint32_t half = kHalfBytes >> 4;
                        umma_ss<kDescHi>(kTmS + X * 128, q_lo + (kk >> 2) * half + (kk & 3) * 2,
                                         k_lo + (kk >> 2) * half + (kk & 3) * 2, kIdescQk, kk > 0 ? 1u : 0u);
                    }
                    umma_commit(&s_full[X]);
                }
                tc_fence_before_sync();
                mbar_arrive(&turn[X ^ 1]);
                if (live) {
                    if (do_pv) umma_commit(&freed[vs]);
                    else if (has_v) mbar_arrive(&freed[vs]);
                    if (do_qk) umma_commit(&freed[ks]);
                    else if (has_k) mbar_arrive(&freed[ks]);
                }
                if (do_qk && last_q) umma_commit(&q_free[X]);
            }
            __syncwarp();
            return true;
        };
        ok = fetch();
        if (ok && !end_) {  // the first item's first logits
            const int n = X ? n1_ : n0_;
            ok = play(false, false, false, false, 0, false, n > 0, 0, true, n == 1, true);
        }
        while (ok && !end_) {
            const int n0 = n0_, n1 = n1_, keys = keys_, n = X ? n1 : n0, rounds = max(n0, n1);
            for (int i = 0; i < rounds && ok; ++i) {
                const bool last = i == rounds - 1;
                if (last && !(ok = fetch())) break;
                const int n_ = X ? n1_ : n0_;
                const bool more = i + 1 < n, begin = last && !end_ && n_ > 0;
                ok = play(i < n, i == 0, i == n - 1, true, keys - i * kTileKeys, X == 0 || i >= n0, more || begin, 2, begin,
                          begin ? n_ == 1 : i + 2 == n, !last || !end_);
                cph = phase_of(2);
                cs = slot_of(2);
            }
        }
        if (elect_one()) {
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
    };

    if (warp >= kMmaWarp) {
        // 384 threads * 168 = 128 * 72 + 256 * 216 registers
        setmaxnreg_dec<72>();
        if (warp == kLoadWarp) {
            // ------------------------------------------------------------ items, query rows, K and V tiles
            Walk walk(p, run, tq, heads, scan);
            TileLoader<PAGED, kRingT> tiles{p, ring, full, freed, abort, lim};
            uint32_t qn0 = 0, qn1 = 0;
            bool ok = true;
            for (int it = 0; ok; ++it) {
                const int slot = it % kAttnItemRing;
                if (!(ok = warp_wait(&item_free[slot], ((it / kAttnItemRing) & 1) ^ 1, abort, lim))) break;
                Item I;
                const bool more = walk.next(I);
                if (more) {
                    const int ka = (I.pos0 + min(p.tp, I.ntok) - 1) / kTileKeys + 1;  // key tiles of the first row tile
                    I.n[0] = max(0, min(I.t0 + I.n_tiles, ka) - I.t0);
                    I.n[1] = I.ntok > p.tp ? I.n_tiles : 0;
                }
                if (lane == 0) {
                    items[slot] = I;
                    mbar_arrive(&item_full[slot]);
                }
                __syncwarp();
                if (!more) break;
#pragma unroll
                for (int X = 0; X < 2; ++X) {
                    uint32_t& qn = X ? qn1 : qn0;
                    if (!ok || I.n[X] == 0) continue;
                    if (!(ok = warp_wait(&q_free[X], (qn & 1) ^ 1, abort, lim))) break;
                    ++qn;
                    if (lane == 0) {
                        mbar_arrive_expect_tx(&q_full[X], static_cast<uint32_t>(p.hp * p.tp * 256));
                        uint8_t* d = qbuf + X * kTileBytes;
                        tma_load_3d(d, &p.tmap_q, &q_full[X], 0, I.head0, I.q_row + X * p.tp);
                        tma_load_3d(d + kHalfBytes, &p.tmap_q, &q_full[X], 64, I.head0, I.q_row + X * p.tp);
                    }
                    __syncwarp();
                }
                ok = ok && tiles.item(I);
            }
            if (!ok) {
                *abort = 1;
                if (lane == 0) record_error(a.status, kDevTimeout, 41);
            }
            volatile int never = 0;
            tiles.drain();
            if (qn0 > 0) mbar_wait(&q_full[0], (qn0 - 1) & 1, &never);
            if (qn1 > 0) mbar_wait(&q_full[1], (qn1 - 1) & 1, &never);
            __syncwarp();
        } else if (warp < kLoadWarp) {
            if (warp == kMmaWarp) mma_role(std::integral_constant<int, 0>{});
            else mma_role(std::integral_constant<int, 1>{});
        } else if (a.check_hash && blockIdx.x == 0) {
            check_seqlens(a);
        }
    } else {
        // ---------------------------------------------------------------- softmax, a row a thread
        setmaxnreg_inc<216>();
        const int X = warp >> 2, r = threadIdx.x & 127, row = threadIdx.x;
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t s_tmem = kTmS + X * 128 + lane_base, o_tmem = kTmO + X * 128 + lane_base;
        const int t_r = r / p.hp, h_r = r - t_r * p.hp, tok = t_r + X * p.tp;  // the row's token and head
        const float c = p.c, tau = kAttnTau / p.c;
        const bool wide = (reinterpret_cast<uintptr_t>(a.out) & 31) == 0;
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
            // Keys that the row sees from the item's first tile on (a row of no use: all), and the tiles of which
            // every row of the warp sees all.
            const int sees = valid ? I.pos0 + tok + 1 - I.t0 * kTileKeys : INT_MAX;
            const int unmasked = __reduce_min_sync(0xffffffffu, sees) >> 7;
            const int n = I.n[X];
            float m = -INFINITY, mc = 0.f, l = 0.f;  // reference (raw), times c, sum
            for (int i = 0; i < n; ++i, ++sn) {
                tile_wait(&s_full[X], sn & 1, abort, lim, a.status);
                __syncwarp();
                if (any) {
                    tc_fence_after_sync();
                    float s[128];
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) tmem_ld32(s_tmem + q4 * 32, s + q4 * 32);
                    tmem_ld_wait();
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) reg_fence32(s + q4 * 32);
                    if (i >= unmasked) {
                        const int nv = sees - i * kTileKeys;  // keys of the tile that the row sees
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
                    // 32 columns at a time, each step over all of them: 911 cycles a tile for one warp and 1425 for
                    // the two of a scheduler, against 1213 and 1722 taken pair by pair.
                    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int q4 = 0; q4 < 4; ++q4) {
                        float* e = s + q4 * 32;
                        uint32_t pk[16];
#pragma unroll
                        for (int x = 0; x < 32; ++x) e[x] = fmaf(e[x], c, -mc);
#pragma unroll
                        for (int x = 0; x < 32; ++x) e[x] = ex2_approx(e[x]);
#pragma unroll
                        for (int x = 0; x < 32; x += 2) pk[x >> 1] = pack_bf16(e[x], e[x + 1]);
#pragma unroll
                        for (int x = 0; x < 32; x += 4) {
                            add2(sum[0], sum[1], sum[0], sum[1], e[x], e[x + 1]);
                            add2(sum[2], sum[3], sum[2], sum[3], e[x + 2], e[x + 3]);
                        }
                        tmem_st16u(s_tmem + q4 * 16, pk);
                    }
                    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    tmem_st_wait();
                }
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[X]);
                __syncwarp();
            }
            if (n > 0) {
                if (!(ok = warp_wait(&pv_done[X], items_done & 1, abort, lim))) break;
                ++items_done;
            }
            tc_fence_after_sync();
            if (m == -INFINITY && l == 0.f) mc = -INFINITY;  // the row saw no key here (or, with a NaN in l, only NaN)
            // ---- the unit's (or this part's) result
            const bool whole = I.part < 0;
            float* part = whole ? nullptr : partial_of<kRowsT>(a, blockIdx.x, I.part == 0);
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) +
                                 (static_cast<long long>(I.q_row + tok) * a.Hq + I.head0 + h_r) * kHeadDim;
            if (any && n > 0) {
                const float inv = 1.f / l;
#pragma unroll
                for (int q4 = 0; q4 < 4; ++q4) {
                    float o[32];
                    tmem_ld32(o_tmem + q4 * 32, o);
                    tmem_ld_wait();
                    reg_fence32(o);
                    if (!valid) continue;
                    if (whole) {
                        uint32_t pk[16];
#pragma unroll
                        for (int x = 0; x < 16; ++x) pk[x] = pack_bf16(o[2 * x] * inv, o[2 * x + 1] * inv);
                        store_bf16(out + q4 * 32, pk, wide);
                        store_bf16(out + q4 * 32 + 16, pk + 8, wide);
                    } else {  // [column / 4][row] in fours
                        float4* d = reinterpret_cast<float4*>(part);
#pragma unroll
                        for (int x = 0; x < 32; x += 4)
                            d[((q4 * 32 + x) >> 2) * kRowsT + row] = make_float4(o[x], o[x + 1], o[x + 2], o[x + 3]);
                    }
                }
            }
            if (whole) {
                if (valid) write_lse<!PAGED>(a, I, tok, h_r, mc, l);
                continue;
            }
            if (valid) {
                part[kRowsT * 128 + row] = mc;
                part[kRowsT * 129 + row] = l;
            }
            if (!(ok = pair_sync(pair, pair_phase, abort, lim))) break;
            if (threadIdx.x == 0) *verdict = last_part(a, I);
            if (!(ok = pair_sync(pair, pair_phase, abort, lim))) break;
            if (!*verdict || !valid) continue;
            // This CTA finished last: it joins the parts, a thread its row, part after part.
            float M = 0.f, L = 0.f;
#pragma unroll 1
            for (int q4 = 0; q4 < 128; q4 += 64) {
                float acc[64];
                M = -INFINITY;
                L = 0.f;
#pragma unroll
                for (int x = 0; x < 64; ++x) acc[x] = 0.f;
#pragma unroll 1
                for (int k = 0; k < I.n_parts; ++k) {
                    const float* src = partial_of<kRowsT>(a, I.cta0 + k, k == 0);
                    const float pm = __ldcg(src + kRowsT * 128 + row), pl = __ldcg(src + kRowsT * 129 + row);
                    float4 po[16];
#pragma unroll
                    for (int x = 0; x < 16; ++x) po[x] = __ldcg(reinterpret_cast<const float4*>(src) + ((q4 >> 2) + x) * kRowsT + row);
                    if (pm == -INFINITY) continue;  // no key seen: its values are not to be used
                    const float Mn = fmaxf(M, pm);
                    const float f0 = M == -INFINITY ? 0.f : ex2_approx(M - Mn), f1 = ex2_approx(pm - Mn);
                    M = Mn;
                    L = L * f0 + pl * f1;
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        acc[4 * x] = acc[4 * x] * f0 + po[x].x * f1;
                        acc[4 * x + 1] = acc[4 * x + 1] * f0 + po[x].y * f1;
                        acc[4 * x + 2] = acc[4 * x + 2] * f0 + po[x].z * f1;
                        acc[4 * x + 3] = acc[4 * x + 3] * f0 + po[x].w * f1;
                    }
                }
                const float inv = 1.f / L;
#pragma unroll
                for (int x = 0; x < 64; x += 16) {
                    uint32_t pk[8];
#pragma unroll
                    for (int y = 0; y < 8; ++y) pk[y] = pack_bf16(acc[x + 2 * y] * inv, acc[x + 2 * y + 1] * inv);
                    store_bf16(out + q4 + x, pk, wide);
                }
            }
            write_lse<!PAGED>(a, I, tok, h_r, M, L);
        }
        if (!ok) {
            *abort = 1;
            if (lane == 0) record_error(a.status, kDevTimeout, 44);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == kMmaWarp) tmem_dealloc(*tmem_slot, 512);
}

template <bool PAGED>
cudaError_t launch_variant(const AttnParams& p, int grid, cudaStream_t stream) {
    auto kern = attention_tiles_kernel<PAGED>;
    static bool configured[kAttnMaxDevices] = {};
    const cudaError_t e = attn_configure(kern, TilesSmem::kBytes, configured);
    if (e != cudaSuccess) return e;
    NvtxRange range("attention_tiles_kernel");
    kern<<<grid, kThreadsT, TilesSmem::kBytes, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_tiles(const AttnLaunch& L, const CUtensorMap& map_q, const CUtensorMap& map_k,
                                   const CUtensorMap& map_v, cudaStream_t stream) {
    AttnParams p;
    p.tmap_q = map_q;
    p.tmap_k = map_k;
    p.tmap_v = map_v;
    p.a = L;
    p.G = L.Hq / L.Hkv;
    p.hp = attn_heads_per_tile(L.Hq, L.Hkv);
    p.tp = kTileKeys / p.hp;
    p.nhb = (p.G + p.hp - 1) / p.hp;
    p.unit_cost = 3;
    p.min_run = 4;
    // 1000 tokens (32/8 heads) 31.9 us with 4, 23.9 with 8; 8 x 1000 98.7 and 89.4 (92 on other boxes); 2048 tokens 48.7
    // with 4 and 8, 57.7 with 16.
    p.whole_tiles = 8;
    p.join_cost = 1.f;
    p.page_shift = 0;
    while ((1 << p.page_shift) < L.page_size) ++p.page_shift;
    p.c = L.scale * 1.4426950408889634f;
    p.wait_cycles = wait_limit_cycles();
    int grid = device_sm_count();
    if (grid <= 0) return cudaErrorNoDevice;
    if (L.max_ctas > 0 && L.max_ctas < grid) grid = L.max_ctas;
    if (grid > kAttnTilesCtas) grid = kAttnTilesCtas;
    return L.paged ? launch_variant<true>(p, grid, stream) : launch_variant<false>(p, grid, stream);
}

}  // namespace ckv
