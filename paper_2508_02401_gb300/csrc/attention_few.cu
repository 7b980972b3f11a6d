// Attention of a few query rows a sequence over a paged cache (attention_common.cuh): single tokens, short drafts.
//
// With G heads of one token on a KV head, 128 rows of the MMA would hold G; so the keys take the MMA's M and up to
// 16 (token, head) rows its N: S^T [128 keys][16] = K Q^T, a key a thread, and O^T [128 dims][16] += V^T P with the
// numerators P [128 keys][16] in shared memory.  The rows' sums stay in the threads until a unit's end, and the
// references are moved by the warps together when a vote says so.
//
// Bound by the loads of K and V: 64 KB a key tile, 1.5 us of an SM's share of the bandwidth (8 caches of 131072
// tokens, 4.3 GB: 620 us, 6.9 TB/s).  Two CTAs run on an SM, so that one's start and end of a unit lie beside the
// other's loads; what they do not hide shows on short caches (256 of 300 tokens, 319 MB: 61 us).
#include "attention_common.cuh"

namespace ckv {
namespace {

constexpr int kThreadsF = 256;
constexpr int kMmaWarpF = 4, kLoadWarpF = 5, kQWarpF = 6;  // warps 0-3: softmax; 7: idle

constexpr int kN = 16;        // (token, head) columns of the MMAs
constexpr int kCtasF = 2;     // on an SM
constexpr int kRingF = 3;     // K and V tiles of 32 KB
constexpr int kQBytesF = kN * 256, kPBytesF = kN * 256;
constexpr int kTmemF = 64;    // columns: two S, one O (48)
// P as the second MMA's B: rows of 32 bytes a key, swizzled over as many; 8-key groups of 256 bytes.
constexpr uint32_t kPGroup = 256, kPHi = (kPGroup >> 4) | (1u << 14) | (6u << 29);

struct FewSmem {
    static constexpr int kQ = kRingF * kTileBytes;
    static constexpr int kP = kQ + 2 * kQBytesF;
    static constexpr int kRed = kP + kPBytesF;   // float [4][kN]
    static constexpr int kRef = kRed + 16 * kN;  // float [kN]: the rows' references, times c
    static constexpr int kItems = kRef + 4 * kN;
    static constexpr int kBars = kItems + kAttnItemRing * static_cast<int>(sizeof(Item));
    static constexpr int kFull = 0, kFree = kFull + kRingF, kQFull = kFree + kRingF, kQFree = kQFull + 2,
                         kSFull = kQFree + 2, kPFull = kSFull + 2, kPvDone = kPFull + 1, kItemFull = kPvDone + 1,
                         kItemFree = kItemFull + kAttnItemRing, kDone = kItemFree + kAttnItemRing, kNumBars = kDone + 1;
    static constexpr int kScan = kBars + 8 * kNumBars;
    static constexpr int kMisc = kScan + kScanBytes;
    static constexpr int kBytes = kMisc + 16;
};
static_assert(FewSmem::kBytes <= 115712, "shared memory of two CTAs");
static_assert(static_cast<size_t>(kAttnMaxCtas) * 2 * kN * 130 <= kAttnPartialFloats, "workspace");

// Barriers of the softmax warps.  None leaves without the others: they agree on every item, and no wait for a
// tile makes one leave.
__device__ __forceinline__ void group_bar() { asm volatile("barrier.cta.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool group_or(bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"(x ? 1u : 0u)
        : "memory");
    return r != 0;
}

// COLS (4, 8 or 16) columns of a thread's lane; complete on return.
template <int COLS>
__device__ __forceinline__ void tmem_load(uint32_t taddr, float* v) {
    if constexpr (COLS == 4) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(taddr) : "memory");
    } else if constexpr (COLS == 8) {
        asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                     : "r"(taddr) : "memory");
    } else {
        tmem_ld16_nowait(taddr, reinterpret_cast<float(&)[16]>(*v));
    }
    tmem_ld_wait();
#pragma unroll
    for (int i = 0; i < COLS; ++i) asm volatile("" : "+f"(v[i]));
}
template <int COLS>
__device__ __forceinline__ void tmem_store(uint32_t taddr, const float* v) {
    if constexpr (COLS == 4) {
        asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1,%2,%3,%4};" ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]),
                     "f"(v[3]) : "memory");
    } else if constexpr (COLS == 8) {
        asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(taddr), "f"(v[0]), "f"(v[1]),
                     "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
    } else {
        tmem_st16(taddr, reinterpret_cast<const float(&)[16]>(*v));
    }
}

// COLS of the 16 columns hold rows (4, 8 or 16): the others' numerators stay zero.
template <int COLS>
__global__ void __launch_bounds__(kThreadsF, kCtasF) attention_few_kernel(const __grid_constant__ AttnParams p) {
    using C = FewSmem;
    constexpr uint32_t kIdescS = idesc_bf16_f32(128, kN);
    constexpr uint32_t kIdescO = idesc_bf16_f32(128, kN) | (1u << 15) | (1u << 16);  // A and B with M, N contiguous
    extern __shared__ __align__(1024) uint8_t sm[];
    uint8_t* ring = sm;
    uint8_t* qbuf = sm + C::kQ;
    uint8_t* pbuf = sm + C::kP;
    float* red = reinterpret_cast<float*>(sm + C::kRed);
    float* ref = reinterpret_cast<float*>(sm + C::kRef);
    Item* items = reinterpret_cast<Item*>(sm + C::kItems);
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + C::kBars);
    uint64_t* full = bars + C::kFull;
    uint64_t* freed = bars + C::kFree;
    uint64_t* q_full = bars + C::kQFull;
    uint64_t* q_free = bars + C::kQFree;
    uint64_t* s_full = bars + C::kSFull;
    uint64_t* p_full = bars + C::kPFull;
    uint64_t* pv_done = bars + C::kPvDone;
    uint64_t* item_full = bars + C::kItemFull;
    uint64_t* item_free = bars + C::kItemFree;
    uint64_t* done = bars + C::kDone;
    long long* scan = reinterpret_cast<long long*>(sm + C::kScan);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + C::kMisc);
    volatile int* abort = reinterpret_cast<volatile int*>(sm + C::kMisc + 4);
    volatile int* verdict = reinterpret_cast<volatile int*>(sm + C::kMisc + 8);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const AttnLaunch& a = p.a;
    const int heads = a.Hkv;            // units of a row tile (a unit has whole KV groups of G = p.hp heads)
    if ((smem_u32(sm) & 1023u) != 0) {  // the swizzled tiles need an aligned base
        if (threadIdx.x == 0) record_error(a.status, kDevBadIndex, -2);
        return;
    }
    if (threadIdx.x == 0) {
        *abort = 0;
        for (int i = 0; i < kRingF; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&freed[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_free[i], 1);
            mbar_init(&s_full[i], 1);
        }
        mbar_init(p_full, 4);
        mbar_init(pv_done, 1);
        for (int i = 0; i < kAttnItemRing; ++i) {
            mbar_init(&item_full[i], 1);
            mbar_init(&item_free[i], 6);  // softmax warps, the MMA issuer, the query loader
        }
        mbar_init(done, 1);
        fence_mbar_init();
    }
    if (warp == kLoadWarpF && lane == 0) {
        tma_prefetch_desc(&p.tmap_k);
        tma_prefetch_desc(&p.tmap_v);
    }
    if (warp == kMmaWarpF) {
        tmem_alloc(tmem_slot, kTmemF);
        tmem_relinquish();
    }
    // Query rows that a unit does not have are never loaded: zeros (or another unit's rows) in their place.
    static_assert(C::kP == C::kQ + 2 * kQBytesF, "P follows the query buffers");
    for (int i = threadIdx.x; i < (2 * kQBytesF + kPBytesF) / 16; i += kThreadsF)
        reinterpret_cast<uint4*>(qbuf)[i] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    Run run;
    const bool busy = find_run<kThreadsF>(p, p.tp, heads, scan, run);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (!busy) {
        if (warp == kMmaWarpF) tmem_dealloc(*tmem_slot, kTmemF);
        return;
    }
    const uint32_t tm_s = *tmem_slot, tm_o = tm_s + 2 * kN;  // S of even and odd tiles, O
    const long long lim = p.wait_cycles;

    if (warp == kLoadWarpF) {
        // ---------------------------------------------------------------- items, K and V tiles
        Walk walk(p, run, p.tp, heads, scan);
        TileLoader<true, kRingF> tiles{p, ring, full, freed, abort, lim};
        bool ok = true;
        for (int it = 0; ok; ++it) {
            const int slot = it % kAttnItemRing;
            if (!(ok = warp_wait(&item_free[slot], ((it / kAttnItemRing) & 1) ^ 1, abort, lim))) break;
            Item I;
            const bool more = walk.next(I);
            if (lane == 0) {
                items[slot] = I;
                mbar_arrive(&item_full[slot]);
            }
            __syncwarp();
            if (!more) break;
            ok = tiles.item(I);
        }
        if (!ok) {
            *abort = 1;
            if (lane == 0) record_error(a.status, kDevTimeout, 51);
        }
        tiles.drain();
        __syncwarp();
    } else if (warp == kQWarpF) {
        // ---------------------------------------------------------------- query rows
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
            uint8_t* dst = qbuf + qs * kQBytesF;
            const int chunks = p.tp * p.hp * 16;
#pragma unroll 4
            for (int x = lane; x < chunks; x += 32) {
                const int r = x >> 4, ch = x & 15;
                const int t = r / p.hp, h = r - t * p.hp;
                if (t >= I.ntok) continue;
                const uint4 val = *reinterpret_cast<const uint4*>(
                    src + (I.q_row + t) * a.q_tok + (I.head0 + h) * a.q_head + ch * 8);
                *reinterpret_cast<uint4*>(dst + (ch >> 3) * (kN * 128) + r * 128 + (((ch & 7) ^ (r & 7)) << 4)) = val;
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_full[qs]);
            __syncwarp();
        }
        if (!ok) {
            *abort = 1;
            if (lane == 0) record_error(a.status, kDevTimeout, 53);
        }
    } else if (warp == kMmaWarpF) {
        // ---------------------------------------------------------------- MMA issuer
        // The logits of a tile before the product of the one before it: S has two buffers, and the numerators of a
        // tile are there only when its S has been read.  An item's first logits come after the last product of the
        // one before it, whose result would otherwise wait for a K still on its way (256 caches of 300 tokens: 72 -> 67
        // us).
        constexpr uint32_t kTileUnits = kTileBytes >> 4;
        const uint32_t ring_addr = desc_addr(ring), q_addr = desc_addr(qbuf), p_lo = desc_addr(pbuf) | (1u << 16);
        uint32_t sn = 0, pn = 0, cs = 0, cph = 0;  // logits and products issued; ring slot and phase of the next K
        int it = 0, end_ = 0, n_ = 0, keys_ = 0;
        bool ok = true, live = true;  // live (a lane's own): none of its waits for a tile gave up
        auto fetch = [&]() {
            const int slot = it % kAttnItemRing;
            if (!warp_wait(&item_full[slot], (it / kAttnItemRing) & 1, abort, lim)) return false;
            end_ = uniform(items[slot].part == kEndItem);
            n_ = uniform(items[slot].n_tiles);
            keys_ = uniform(items[slot].len - items[slot].t0 * kTileKeys);
            __syncwarp();
            if (elect_one()) mbar_arrive(&item_free[slot]);
            __syncwarp();
            ++it;
            return true;
        };
        auto slot_of = [&](uint32_t d) { return cs + d >= kRingF ? cs + d - kRingF : cs + d; };
        auto phase_of = [&](uint32_t d) { return cs + d >= kRingF ? cph ^ 1 : cph; };
        auto qk = [&](uint32_t d, bool first, bool last) {  // K at ring position d; item it - 1
            const uint32_t ks = slot_of(d), qs = (it - 1) & 1;
            if (first && !warp_wait(&q_full[qs], ((it - 1) >> 1) & 1, abort, lim)) return false;
            const uint32_t k_lo = uniform((ring_addr + ks * kTileUnits) | kDescLoK);
            const uint32_t q_lo = uniform((q_addr + qs * (kQBytesF >> 4)) | kDescLoK);
            const uint32_t d_tmem = uniform(tm_s + (sn & 1) * kN);
            live &= tile_wait(&full[ks], phase_of(d), abort, lim, a.status);
            __syncwarp();
            tc_fence_after_sync();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    umma_ss<kDescHi>(d_tmem, k_lo + (kk >> 2) * (kHalfBytes >> 4) + (kk & 3) * 2,
                                     q_lo + (kk >> 2) * (kN * 128 >> 4) + (kk & 3) * 2, kIdescS, kk > 0 ? 1u : 0u);
                umma_commit(&s_full[sn & 1]);
                if (live) umma_commit(&freed[ks]);
                if (last) umma_commit(&q_free[qs]);
            }
            __syncwarp();
            ++sn;
            return true;
        };
        ok = fetch();
        if (ok && !end_) ok = qk(0, true, n_ == 1);
        while (ok && !end_) {
            const int n = n_, keys = keys_;
            for (int i = 0; i < n && ok; ++i) {
                const bool last = i == n - 1;
                if (last && !(ok = fetch())) break;
                // ring: K(i) V(i) K(i + 1)
                if (!last && !(ok = qk(2, false, i + 2 == n))) break;
                const uint32_t vs = slot_of(1);
                const uint32_t v_lo = uniform((ring_addr + vs * kTileUnits) | kDescLoV), d_tmem = uniform(tm_o);
                const uint32_t accumulate = uniform(i > 0);
                live &= tile_wait(&full[vs], phase_of(1), abort, lim, a.status);
                if (keys - i * kTileKeys < kTileKeys) clear_rows(ring + vs * kTileBytes, keys - i * kTileKeys, lane);
                tile_wait(p_full, pn & 1, abort, lim, a.status);
                ++pn;
                __syncwarp();
                tc_fence_after_sync();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_ss<kPHi>(d_tmem, v_lo + kk * (2048 >> 4), p_lo + kk * (2 * kPGroup >> 4), kIdescO,
                                         kk > 0 ? 1u : accumulate);
                    umma_commit(pv_done);
                    if (live) umma_commit(&freed[vs]);
                }
                __syncwarp();
                if (last && !end_) ok = qk(2, true, n_ == 1);
                cph = phase_of(2);
                cs = slot_of(2);
            }
        }
        if (elect_one()) {
            if (!ok) {
                *abort = 1;
                record_error(a.status, kDevTimeout, 52);
            }
            umma_commit(done);
        }
        __syncwarp();
        volatile int never = 0;
        mbar_wait(done, 0, &never);
        __syncwarp();
    } else if (warp < 4) {
        // ---------------------------------------------------------------- softmax, a key a thread
        const int key = threadIdx.x;
        const uint32_t lane_base = static_cast<uint32_t>(warp * 32) << 16;
        const float c = p.c;
        uint32_t sn = 0;
        bool ok = true;
        float l[COLS];  // this thread's keys' sums
        // The product of the tile before the current one is in O, and its numerators have been read.
        auto wait_pv = [&](uint32_t tile) {
            if (tile == 0) return;
            tile_wait(pv_done, (tile - 1) & 1, abort, lim, a.status);
            __syncwarp();
            tc_fence_after_sync();
        };
        for (int it = 0; ok; ++it) {
            const int slot = it % kAttnItemRing;
            ok = !group_or(!warp_wait(&item_full[slot], (it / kAttnItemRing) & 1, abort, lim));
            if (!ok) break;
            const Item I = items[slot];
            __syncwarp();
            if (lane == 0) mbar_arrive(&item_free[slot]);
            if (I.part == kEndItem) break;
#pragma unroll
            for (int x = 0; x < COLS; ++x) l[x] = 0.f;
            if (key < COLS) ref[key] = -INFINITY;
            group_bar();
            const int rows = I.ntok * p.hp;
            // The first key that some row does not see.
            const int first_end = I.pos0 + 1;
            for (int i = 0; i < I.n_tiles; ++i, ++sn) {
                const int k0 = (I.t0 + i) * kTileKeys;
                tile_wait(&s_full[sn & 1], (sn >> 1) & 1, abort, lim, a.status);
                __syncwarp();
                tc_fence_after_sync();
                float s[COLS];
                tmem_load<COLS>(tm_s + (sn & 1) * kN + lane_base, s);
                tc_fence_before_sync();
                if (k0 + kTileKeys > first_end) {
                    int ends = first_end - (k0 + key), h = 0;  // positive: the row of column x sees the key
#pragma unroll
                    for (int x = 0; x < COLS; ++x) {
                        s[x] = ends > 0 ? s[x] : -INFINITY;
                        if (++h == p.hp) {
                            h = 0;
                            ++ends;
                        }
                    }
                }
                float over = -INFINITY;
#pragma unroll
                for (int x = 0; x < COLS; ++x) {
                    s[x] *= c;
                    over = fmaxf(over, x < rows ? s[x] - ref[x] : -INFINITY);
                }
                if (group_or(over > kAttnTau)) {
                    wait_pv(sn);
                    // Move the references that a key passes by more than 2^8 (or that have none yet).
#pragma unroll
                    for (int x = 0; x < COLS; ++x) {
                        const float w = redux_max(s[x]);
                        if (lane == 0) red[warp * COLS + x] = w;
                    }
                    group_bar();
                    float o[COLS];
                    if (i > 0) tmem_load<COLS>(tm_o + lane_base, o);
#pragma unroll
                    for (int x = 0; x < COLS; ++x) {
                        const float mx = fmaxf(fmaxf(red[x], red[COLS + x]), fmaxf(red[2 * COLS + x], red[3 * COLS + x]));
                        const float f = mx - ref[x] > kAttnTau ? ex2_approx(ref[x] - mx) : 1.f;  // (no: -inf - -inf)
                        l[x] *= f;
                        o[x] *= f;
                    }
                    if (i > 0) tmem_store<COLS>(tm_o + lane_base, o);
                    tmem_st_wait();
                    tc_fence_before_sync();
                    group_bar();  // ref is read
                    if (key < COLS) {
                        const float mx = fmaxf(fmaxf(red[key], red[COLS + key]), fmaxf(red[2 * COLS + key], red[3 * COLS + key]));
                        if (mx - ref[key] > kAttnTau) ref[key] = mx;
                    }
                    group_bar();
                }
                uint32_t pk[COLS / 2];
#pragma unroll
                for (int x = 0; x < COLS; ++x) {
                    s[x] = ex2_approx(s[x] - fmaxf(ref[x], -3e38f));  // (-inf: a row that has seen no key yet)
                    l[x] += s[x];
                }
#pragma unroll
                for (int x = 0; x < COLS; x += 2) pk[x >> 1] = pack_bf16(s[x], s[x + 1]);
                wait_pv(sn);  // the last tile's numerators are read
                // The key's row of P, its 16-byte pieces swizzled by the address bits above the row's.
                uint8_t* prow = pbuf + key * (2 * kN);
                const int sw = (key >> 2) & 1;
                if constexpr (COLS == 4) {
                    *reinterpret_cast<uint2*>(prow + (sw << 4)) = make_uint2(pk[0], pk[1]);
                } else {
#pragma unroll
                    for (int x = 0; x < COLS / 8; ++x)
                        *reinterpret_cast<uint4*>(prow + ((x ^ sw) << 4)) =
                            make_uint4(pk[4 * x], pk[4 * x + 1], pk[4 * x + 2], pk[4 * x + 3]);
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full);
                __syncwarp();
            }
            // ---- the unit's (or this part's) result: the rows' sums over the threads, then a dim a thread
            if constexpr (COLS >= 8) {
                float none[COLS];
#pragma unroll
                for (int x = 0; x < COLS; ++x) none[x] = 0.f;
                transpose_reduce<COLS>(l, none, lane);  // lane: column lane / (32 / COLS)
                if (lane % (32 / COLS) == 0) red[warp * COLS + lane / (32 / COLS)] = l[0];
            } else {
#pragma unroll
                for (int x = 0; x < COLS; ++x) l[x] = warp_sum(l[x]);
                if (lane == 0) {
#pragma unroll
                    for (int x = 0; x < COLS; ++x) red[warp * COLS + x] = l[x];
                }
            }
            wait_pv(sn);
            group_bar();
            float o[COLS];
            tmem_load<COLS>(tm_o + lane_base, o);
            tc_fence_before_sync();
            const bool whole = I.part < 0;
            float* part = whole ? nullptr : partial_of<kN>(a, blockIdx.x, I.part == 0);
            const int dim = threadIdx.x;
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) + (static_cast<long long>(I.q_row) * a.Hq + I.head0) * kHeadDim + dim;
            int t = 0, h = -1;
#pragma unroll
            for (int x = 0; x < COLS; ++x) {
                if (x >= rows) break;
                if (++h == p.hp) {
                    h = 0;
                    ++t;
                }
                const float L = (red[x] + red[COLS + x]) + (red[2 * COLS + x] + red[3 * COLS + x]);
                if (whole) {
                    out[(t * a.Hq + h) * kHeadDim] = __float2bfloat16(o[x] * (1.f / L));
                    if (dim == 0) write_lse<false>(a, I, t, h, ref[x], L);
                } else {
                    part[x * 128 + dim] = o[x];
                    if (dim == 0) {
                        part[kN * 128 + x] = L == 0.f ? ref[x] : fmaxf(ref[x], -3e38f);  // (only NaN seen: joined)
                        part[kN * 129 + x] = L;
                    }
                }
            }
            if (whole) {
                group_bar();  // red is read
                continue;
            }
            group_bar();
            if (threadIdx.x == 0) *verdict = last_part(a, I);
            group_bar();
            if (!*verdict) continue;
            // This CTA finished last: it joins the parts, a warp a row; a lane holds a part's weight and, of
            // the row, four dims.
            for (int x = warp; x < rows; x += 4) {
                const int tx = x / p.hp, hx = x - tx * p.hp;
                float M = -INFINITY, L = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int k0 = 0; k0 < I.n_parts; k0 += 32) {
                    const int n = min(32, I.n_parts - k0);
                    float pm = -INFINITY, pl = 0.f;
                    if (lane < n) {
                        const float* src = partial_of<kN>(a, I.cta0 + k0 + lane, k0 + lane == 0);
                        pm = __ldcg(src + kN * 128 + x);
                        pl = __ldcg(src + kN * 129 + x);
                    }
                    const float Mn = fmaxf(M, redux_max(pm));
                    const float f0 = M == -INFINITY ? 0.f : ex2_approx(M - Mn);
                    const float w = pm == -INFINITY ? 0.f : ex2_approx(pm - Mn);  // (0: no key seen)
                    M = Mn;
                    L = L * f0 + warp_sum(pl * w);
                    acc = make_float4(acc.x * f0, acc.y * f0, acc.z * f0, acc.w * f0);
#pragma unroll 1
                    for (int k = 0; k < n; k += 8) {
                        float4 o[8];
#pragma unroll
                        for (int y = 0; y < 8; ++y)
                            o[y] = k + y < n ? __ldcg(reinterpret_cast<const float4*>(
                                                   partial_of<kN>(a, I.cta0 + k0 + k + y, k0 + k + y == 0) + x * 128) + lane)
                                             : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                        for (int y = 0; y < 8; ++y) {
                            const float wy = __shfl_sync(0xffffffffu, w, (k + y) & 31);
                            if (k + y >= n) continue;
                            acc.x += o[y].x * wy;
                            acc.y += o[y].y * wy;
                            acc.z += o[y].z * wy;
                            acc.w += o[y].w * wy;
                        }
                    }
                }
                const float inv = 1.f / L;
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) +
                                     (static_cast<long long>(I.q_row + tx) * a.Hq + I.head0 + hx) * kHeadDim + lane * 4;
                *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                if (lane == 0) write_lse<false>(a, I, tx, hx, M, L);
            }
        }
        if (!ok) {
            *abort = 1;
            if (lane == 0) record_error(a.status, kDevTimeout, 54);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == kMmaWarpF) tmem_dealloc(*tmem_slot, kTmemF);
}

template <int COLS>
cudaError_t launch_few(const AttnLaunch& L, AttnParams& p, cudaStream_t stream) {
    auto kern = attention_few_kernel<COLS>;
    static bool configured[kAttnMaxDevices] = {};
    const cudaError_t e = attn_configure(kern, FewSmem::kBytes, configured);
    if (e != cudaSuccess) return e;
    p.hp = p.G;
    p.tp = COLS / p.G;
    p.nhb = 1;
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorNoDevice;
    int grid = sms * kCtasF;
    if (L.max_ctas > 0 && L.max_ctas < sms) grid = L.max_ctas;  // (two could go to an SM each)
    if (grid > kAttnMaxCtas) grid = kAttnMaxCtas;
    NvtxRange range("attention_few_kernel");
    kern<<<grid, kThreadsF, FewSmem::kBytes, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_few(const AttnLaunch& L, const CUtensorMap& map_k, const CUtensorMap& map_v, int rows,
                                 cudaStream_t stream) {
    AttnParams p;
    p.tmap_k = map_k;
    p.tmap_v = map_v;
    p.a = L;
    p.G = L.Hq / L.Hkv;
    p.unit_cost = 2;
    p.min_run = 1;
    p.whole_tiles = 0;  // (a part costs little here: 4 x 700 keys 10.8 us, 11.8 with 3)
    p.join_cost = 0.f;
    p.page_shift = 0;
    while ((1 << p.page_shift) < L.page_size) ++p.page_shift;
    p.c = L.scale * 1.4426950408889634f;
    p.wait_cycles = wait_limit_cycles();
    // Only the columns in use are worked on: 256 caches of 300 tokens, 4 rows each, 61.9 us with 4 columns, 67.1 with 16
    // (when it was measured; 61 now).
    return rows <= 4 ? launch_few<4>(L, p, stream) : rows <= 8 ? launch_few<8>(L, p, stream) : launch_few<16>(L, p, stream);
}

}  // namespace ckv
