// What the kernels for a few query rows a sequence share (attention_few.cu: a bf16 cache; attention_few_q4.cu: one in 4
// bits): the roles that load the query rows and that turn logits into numerators and results.
//
// The keys take the MMA's M and up to 16 (token, head) rows its N: S^T [128 keys][16] = K Q^T, a key a thread, and
// O^T [128 dims][16] += V^T P with the numerators P [128 keys][16] in shared memory.  The rows' sums stay in the threads
// until a unit's end, and the references are moved by the warps together when a vote says so.
#pragma once

#include "attention_common.cuh"

namespace ckv {
namespace {

constexpr int kN = 16;  // (token, head) columns of the MMAs
constexpr int kQBytesF = kN * 256, kPBytesF = kN * 256;
// P as the second MMA's B: rows of 32 bytes a key, swizzled over as many; 8-key groups of 256 bytes.
constexpr uint32_t kPGroup = 256, kPHi = (kPGroup >> 4) | (1u << 14) | (6u << 29);
constexpr uint32_t kIdescFewS = idesc_bf16_f32(128, kN);
constexpr uint32_t kIdescFewO = idesc_bf16_f32(128, kN) | (1u << 15) | (1u << 16);  // A and B with M, N contiguous
constexpr int kRedBytesF = 16 * kN, kRefBytesF = 4 * kN;

// The roles' shared memory.
struct FewRoles {
    uint8_t* qbuf;     // two buffers of query rows
    uint8_t* pbuf;     // numerators
    float* red;        // [4][kN]
    float* ref;        // [kN]: the rows' references, times c
    const Item* items;
    uint64_t *item_full, *item_free, *q_full, *q_free, *s_full, *p_full, *pv_done;
    volatile int *abort, *verdict;
    uint32_t tm_s, tm_o;  // S of even and odd tiles, O
};

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

// The query rows of the items (a warp).
__device__ __forceinline__ void few_query_role(const AttnParams& p, const FewRoles& R, long long lim) {
    const AttnLaunch& a = p.a;
    const int lane = threadIdx.x & 31;
    uint8_t* qbuf = R.qbuf;
    uint64_t *item_full = R.item_full, *item_free = R.item_free, *q_full = R.q_full, *q_free = R.q_free;
    const Item* items = R.items;
    volatile int* abort = R.abort;
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
}

// Numerators and results (four warps, a key a thread).  COLS of the 16 columns hold rows (4, 8 or 16).
template <int COLS>
__device__ __forceinline__ void few_softmax_role(const AttnParams& p, const FewRoles& R, long long lim) {
    const AttnLaunch& a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t* pbuf = R.pbuf;
    float *red = R.red, *ref = R.ref;
    const Item* items = R.items;
    uint64_t *item_full = R.item_full, *item_free = R.item_free, *s_full = R.s_full, *p_full = R.p_full, *pv_done = R.pv_done;
    volatile int *abort = R.abort, *verdict = R.verdict;
    const uint32_t tm_s = R.tm_s, tm_o = R.tm_o;
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

}  // namespace
}  // namespace ckv
