// Attention of a few query rows a sequence over a paged cache of 4 bits (attention_few.cuh, kv4.cuh).
//
// The cached values are bf16 numbers, so the products are those of the bf16 cache; between the loads and the MMAs, four
// warps turn the tile's codes into K, a key a lane, in tensor memory (the first operand of S^T = K Q^T), and four into V, a key
// a row, in shared memory (the first operand of O^T += V^T P, which has the dims on its rows and so cannot come from the
// lanes of keys).
#include "attention_few.cuh"
#include <string.h>

#include "kv4_loader.cuh"

namespace ckv {
namespace {

constexpr int kThreadsF4 = 512;
constexpr int kWarpV = 8, kLoadWarp4 = 12, kMmaWarp4 = 13, kQWarp4 = 14;  // warps 0-3: softmax; 4-7: K; 8-11: V; 15: idle
constexpr int kRing4 = 6;  // packed tiles of 18 KB
constexpr int kBuf4 = 3;   // K tiles in tensor memory, V tiles in shared memory
constexpr int kTmemK4 = 64;   // columns of a K tile, from the first
constexpr int kTmem4 = 256;   // three K, two S, one O

struct FewSmem4 {
    static constexpr int kV = 0;
    static constexpr int kQ = kBuf4 * kTileBytes;
    static constexpr int kP = kQ + 2 * kQBytesF;
    static constexpr int kRing = kP + kPBytesF;
    static constexpr int kRed = kRing + kRing4 * kPackedTile;
    static constexpr int kRef = kRed + kRedBytesF;
    static constexpr int kItems = kRef + kRefBytesF;
    static constexpr int kBars = kItems + kAttnItemRing * static_cast<int>(sizeof(Item));
    static constexpr int kFull = 0, kFree = kFull + kRing4, kKReady = kFree + kRing4, kKFree = kKReady + kBuf4,
                         kVReady = kKFree + kBuf4, kVFree = kVReady + kBuf4, kQFull = kVFree + kBuf4, kQFree = kQFull + 2,
                         kSFull = kQFree + 2, kPFull = kSFull + 2, kPvDone = kPFull + 1, kItemFull = kPvDone + 1,
                         kItemFree = kItemFull + kAttnItemRing, kDone = kItemFree + kAttnItemRing, kNumBars = kDone + 1;
    static constexpr int kScan = kBars + 8 * kNumBars;
    static constexpr int kMisc = kScan + kScanBytes;
    static constexpr int kBytes = kMisc + 16;
};
static_assert(FewSmem4::kBytes <= 232448, "shared memory");
static_assert(FewSmem4::kRing % 16 == 0 && FewSmem4::kRed % 16 == 0 && kPackedTile % 16 == 0, "alignment");

// A ring of buffers that one side fills and another empties: the current one, and the phase of its barrier.
template <int N>
struct Turn {
    uint32_t at = 0, phase = 0;
    __device__ void next() {
        if (++at == N) {
            at = 0;
            phase ^= 1;
        }
    }
};

template <int COLS>
__global__ void __launch_bounds__(kThreadsF4, 1) attention_few_q4_kernel(const __grid_constant__ AttnParams p) {
    using C = FewSmem4;
    extern __shared__ __align__(1024) uint8_t sm[];
    uint8_t* vbuf = sm + C::kV;
    uint8_t* qbuf = sm + C::kQ;
    uint8_t* pbuf = sm + C::kP;
    uint8_t* ring = sm + C::kRing;
    float* red = reinterpret_cast<float*>(sm + C::kRed);
    float* ref = reinterpret_cast<float*>(sm + C::kRef);
    Item* items = reinterpret_cast<Item*>(sm + C::kItems);
    uint64_t* bars = reinterpret_cast<uint64_t*>(sm + C::kBars);
    uint64_t* full = bars + C::kFull;
    uint64_t* freed = bars + C::kFree;
    uint64_t* k_ready = bars + C::kKReady;
    uint64_t* k_free = bars + C::kKFree;
    uint64_t* v_ready = bars + C::kVReady;
    uint64_t* v_free = bars + C::kVFree;
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
        for (int i = 0; i < kRing4; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&freed[i], 8);  // the warps of K and V
        }
        for (int i = 0; i < kBuf4; ++i) {
            mbar_init(&k_ready[i], 4);
            mbar_init(&k_free[i], 1);
            mbar_init(&v_ready[i], 4);
            mbar_init(&v_free[i], 1);
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
            mbar_init(&item_free[i], 14);  // the warps of the softmax, of K and V, the MMA issuer, the query loader
        }
        mbar_init(done, 1);
        fence_mbar_init();
    }
    if (warp == kMmaWarp4) {
        tmem_alloc(tmem_slot, kTmem4);
        tmem_relinquish();
    }
    // Query rows that a unit does not have are never loaded: zeros (or another unit's rows) in their place.
    static_assert(C::kP == C::kQ + 2 * kQBytesF, "P follows the query buffers");
    for (int i = threadIdx.x; i < (2 * kQBytesF + kPBytesF) / 16; i += kThreadsF4)
        reinterpret_cast<uint4*>(qbuf)[i] = make_uint4(0u, 0u, 0u, 0u);
    fence_proxy_async_smem();
    Run run;
    const bool busy = find_run<kThreadsF4>(p, p.tp, heads, scan, run);
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (!busy) {
        if (warp == kMmaWarp4) tmem_dealloc(*tmem_slot, kTmem4);
        return;
    }
    const uint32_t tm_k = *tmem_slot, tm_s = tm_k + kBuf4 * kTmemK4, tm_o = tm_s + 2 * kN;
    const long long lim = p.wait_cycles;
    const FewRoles R{qbuf, pbuf, red, ref, items, item_full, item_free, q_full, q_free, s_full, p_full, pv_done, abort, verdict, tm_s, tm_o};
    // The next item of a role (a whole warp): false when there is none, or at a wait that gave up (then `ok` is false).
    auto next_item = [&](int it, Item& I, bool& ok) {
        const int slot = it % kAttnItemRing;
        if (!(ok = warp_wait(&item_full[slot], (it / kAttnItemRing) & 1, abort, lim))) return false;
        I = items[slot];
        __syncwarp();
        if (lane == 0) mbar_arrive(&item_free[slot]);
        __syncwarp();
        return I.part != kEndItem;
    };

    if (warp == kLoadWarp4) {
        // ---------------------------------------------------------------- items, packed tiles
        Walk walk(p, run, p.tp, heads, scan);
        PackedLoader<kRing4> tiles{p, ring, full, freed, abort, lim};
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
            if (lane == 0) record_error(a.status, kDevTimeout, 61);
        }
        tiles.drain();
        __syncwarp();
    } else if (warp == kQWarp4) {
        few_query_role(p, R, lim);
    } else if (warp == kMmaWarp4) {
        // ---------------------------------------------------------------- MMA issuer
        // The logits of a tile before the product of the one before it, as over a bf16 cache.
        const uint32_t q_addr = desc_addr(qbuf), v_addr = desc_addr(vbuf), p_lo = desc_addr(pbuf) | (1u << 16);
        Turn<kBuf4> kt, vt;
        uint32_t sn = 0, pn = 0;  // logits and products issued
        int it = 0;
        Item I;
        bool ok = true, more = next_item(it++, I, ok);
        auto qk = [&](bool first, bool last) {  // item it - 1
            const uint32_t qs = (it - 1) & 1;
            if (first && !warp_wait(&q_full[qs], ((it - 1) >> 1) & 1, abort, lim)) return false;
            const uint32_t q_lo = uniform((q_addr + qs * (kQBytesF >> 4)) | kDescLoK);
            const uint32_t d_tmem = uniform(tm_s + (sn & 1) * kN), k_tmem = uniform(tm_k + kt.at * kTmemK4);
            tile_wait(&k_ready[kt.at], kt.phase, abort, lim, a.status);
            __syncwarp();
            tc_fence_after_sync();
            if (elect_one()) {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk)
                    umma_ts(d_tmem, k_tmem + kk * 8, q_lo + (kk >> 2) * (kN * 128 >> 4) + (kk & 3) * 2, kIdescFewS, kk > 0 ? 1u : 0u);
                umma_commit(&s_full[sn & 1]);
                umma_commit(&k_free[kt.at]);
                if (last) umma_commit(&q_free[qs]);
            }
            __syncwarp();
            kt.next();
            ++sn;
            return true;
        };
        if (more) ok = qk(true, I.n_tiles == 1);
        while (ok && more) {
            const int n = I.n_tiles;
            for (int i = 0; i < n && ok; ++i) {
                const bool last = i == n - 1;
                if (last) {
                    more = next_item(it++, I, ok);
                    if (!ok) break;
                }
                if (!last && !(ok = qk(false, i + 2 == n))) break;
                const uint32_t v_lo = uniform((v_addr + vt.at * (kTileBytes >> 4)) | kDescLoV), d_tmem = uniform(tm_o);
                const uint32_t accumulate = uniform(i > 0);
                tile_wait(&v_ready[vt.at], vt.phase, abort, lim, a.status);
                tile_wait(p_full, pn & 1, abort, lim, a.status);
                ++pn;
                __syncwarp();
                tc_fence_after_sync();
                if (elect_one()) {
#pragma unroll
                    for (int kk = 0; kk < 8; ++kk)
                        umma_ss<kPHi>(d_tmem, v_lo + kk * (2048 >> 4), p_lo + kk * (2 * kPGroup >> 4), kIdescFewO, kk > 0 ? 1u : accumulate);
                    umma_commit(pv_done);
                    umma_commit(&v_free[vt.at]);
                }
                __syncwarp();
                vt.next();
                if (last && more) ok = qk(true, I.n_tiles == 1);
            }
        }
        if (elect_one()) {
            if (!ok) {
                *abort = 1;
                record_error(a.status, kDevTimeout, 62);
            }
            umma_commit(done);
        }
        __syncwarp();
        volatile int never = 0;
        mbar_wait(done, 0, &never);
        __syncwarp();
    } else if (warp < 4) {
        few_softmax_role<COLS>(p, R, lim);
    } else if (warp < kLoadWarp4) {
        // ---------------------------------------------------------------- codes into K and V, a key a thread
        const bool is_v = warp >= kWarpV;
        const int key = threadIdx.x & 127;
        const uint32_t lane_base = static_cast<uint32_t>((warp & 3) * 32) << 16;
        Turn<kRing4> in;
        Turn<kBuf4> to;
        bool ok = true, live = true;  // live (a lane's own): none of its waits for a tile gave up
        Item I;
        for (int it = 0; next_item(it, I, ok); ++it) {
            for (int i = 0; i < I.n_tiles; ++i) {
                live &= tile_wait(&full[in.at], in.phase, abort, lim, a.status);
                __syncwarp();
                Kv4Row r = packed_row(ring + in.at * kPackedTile, p.page_shift, key, is_v);
                __syncwarp();
                if (lane == 0 && live) mbar_arrive(&freed[in.at]);
                in.next();
                tile_wait(is_v ? &v_free[to.at] : &k_free[to.at], to.phase ^ 1, abort, lim, a.status);
                __syncwarp();
                if (is_v) {
                    // Rows behind the sequence's end hold anything, and while their numerators are 0, 0 * NaN is not.
                    if (key >= I.len - (I.t0 + i) * kTileKeys) {
                        r.scales = make_uint2(0u, 0u);
#pragma unroll
                        for (int g = 0; g < 4; ++g) r.codes[g] = make_uint4(0u, 0u, 0u, 0u);
                    }
                    uint8_t* row = vbuf + to.at * kTileBytes + key * 128;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        uint32_t v[16];
                        kv4_group(r, g, v);
#pragma unroll
                        for (int x = 0; x < 4; ++x)
                            *reinterpret_cast<uint4*>(row + (g >> 1) * kHalfBytes + ((((g & 1) * 4 + x) ^ (key & 7)) << 4)) =
                                make_uint4(v[4 * x], v[4 * x + 1], v[4 * x + 2], v[4 * x + 3]);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&v_ready[to.at]);
                } else {
                    tc_fence_after_sync();
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        uint32_t v[16];
                        kv4_group(r, g, v);
                        tmem_st16u(tm_k + to.at * kTmemK4 + g * 16 + lane_base, v);
                    }
                    tmem_st_wait();
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&k_ready[to.at]);
                }
                __syncwarp();
                to.next();
            }
        }
        if (!ok) {
            *abort = 1;
            if (lane == 0) record_error(a.status, kDevTimeout, is_v ? 64 : 63);
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    if (warp == kMmaWarp4) tmem_dealloc(*tmem_slot, kTmem4);
}

template <int COLS>
cudaError_t launch_few_q4(const AttnLaunch& L, AttnParams& p, cudaStream_t stream) {
    auto kern = attention_few_q4_kernel<COLS>;
    static bool configured[kAttnMaxDevices] = {};
    const cudaError_t e = attn_configure(kern, FewSmem4::kBytes, configured);
    if (e != cudaSuccess) return e;
    p.hp = p.G;
    p.tp = COLS / p.G;
    p.nhb = 1;
    int grid = device_sm_count();
    if (grid <= 0) return cudaErrorNoDevice;
    if (L.max_ctas > 0 && L.max_ctas < grid) grid = L.max_ctas;
    if (grid > kAttnMaxCtas) grid = kAttnMaxCtas;
    NvtxRange range("attention_few_q4_kernel");
    kern<<<grid, kThreadsF4, FewSmem4::kBytes, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_few_q4(const AttnLaunch& L, int rows, cudaStream_t stream) {
    AttnParams p;
    memset(&p, 0, sizeof p);
    p.a = L;
    p.G = L.Hq / L.Hkv;
    p.unit_cost = 2;
    p.min_run = 1;
    p.page_shift = 0;
    while ((1 << p.page_shift) < L.page_size) ++p.page_shift;
    p.c = L.scale * 1.4426950408889634f;
    p.wait_cycles = wait_limit_cycles();
    return rows <= 4 ? launch_few_q4<4>(L, p, stream) : rows <= 8 ? launch_few_q4<8>(L, p, stream) : launch_few_q4<16>(L, p, stream);
}

}  // namespace ckv
