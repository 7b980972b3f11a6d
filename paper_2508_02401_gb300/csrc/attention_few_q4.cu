// Attention of a few query rows a sequence over a paged cache of 4 bits (attention_common.cuh, kv4.cuh).
//
// A warp takes 16 keys of a tile at a time, straight from the pages into registers, and turns the codes into
// operands there: S^T [16 keys][8 rows] = K Q^T and O^T [128 dims][8 rows] += V^T P by m16n8k16 MMAs.  The keys of K's
// fragments and the channels of all of them are taken in the order that makes a thread's share of a row lie together:
//   K  (rows: keys)      thread (r, c) = (lane / 4, lane % 4): group c of keys 4 (r / 2) + r % 2 and 2 on, 16 bytes of each
//   Q  (columns: rows)   row r, channels 32 c to 32 c + 31: 64 bytes
//   V  (rows: channels)  channels 16 r to 16 r + 15 of keys 4 c to 4 c + 3, 8 bytes of each
// A warp has a softmax of its own (reference, sums, output); the warps of a CTA are joined at a unit's end, the parts of a
// unit by the CTA that finishes last.  No warp waits for another within a unit, and no thread for a copy.
//
// Bound by the instructions that make bf16 numbers of codes, not by memory (0.28 of a bf16 cache's bytes): a step of 16 keys
// is some 415 instructions, 112 of them shifts and masks and 128 differences and products of two bf16 numbers, all of which issue
// at half rate.  8 caches of 131072 tokens, one new token (4 rows a KV head, 1.21 GB): 269 us, 4.5 TB/s (a bf16 cache, 4.29 GB,
// 623 us); the schedulers issue in 58 to 63% of the cycles, the rest is four warps' latencies.  With the differences, products
// and masks left out (wrong results) a form of the loop took 241 us.  Legacy MMAs, since their operands come from registers, where the
// codes are unpacked; of the tensor core's time 18% is used.  What else was built, us on those caches, when the kernel took 286 (before
// the loads in place of this step's and the joins' loads side by side; the prefetches when it took 274):
//   tcgen05, keys on M: K unpacked into tensor memory, V into shared memory            425
//   tcgen05 on the codes as 8-bit floats, numerators as pairs of those (too coarse)      339
//   packed blocks by bulk copies into a ring of the CTA, scales behind the MMAs        305
//   a ring of asynchronous copies for each warp                                        312
//   8-bit-float MMAs for the logits                                                    334
//   9 or 10 warps a CTA 327; one CTA of 16 warps 282, but 64 caches of 128 to 8192 74 against 50 then
//   two steps a trip of the loop 288; a later step asked into L2, its rows 306, its pages by bulk prefetches 290
//   s n in one fused operation, the zero points' part by MMAs of their own (fewer instructions, longer chains, and
//   the small channels of a group with a large one cancel) 295
#include <new>
#include <string.h>

#include "attention_common.cuh"
#include "kv4.cuh"

namespace ckv {
namespace {

constexpr int kCtas4 = 2;  // on an SM
constexpr int kRows4 = 16;
constexpr int kPitch4 = 132;  // floats between the warps' output rows in shared memory
constexpr float kNoRef = -3e38f;
static_assert(static_cast<size_t>(kAttnMaxCtas) * 2 * kRows4 * 130 <= kAttnPartialFloats, "workspace");

// One step's bytes of a thread.
struct Step {
    uint4 k[2];
    uint2 v[4];
    uint32_t ks[2], vs[4];  // scale words
};

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit values, a row's pair a thread.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// N8: blocks of 8 rows (1 or 2).
template <int N8>
struct FewSmem4 {
    // 16 rows: 168 registers a thread (and 40 bytes of spills), so six warps a CTA (40 sequences, 14 rows each, 49.5 us; one CTA of
    // 12 warps 57).
    static constexpr int kWarps4 = N8 == 1 ? 8 : 6;
    static constexpr int kBufs = N8 == 1 ? 2 : 1;  // of the warps' outputs (two: no barrier after they are read)
    float o[kBufs][kWarps4][8 * N8][kPitch4];
    float m[kBufs][kWarps4][8 * N8], l[kBufs][kWarps4][8 * N8];
    Item items[4];
    Run run;
    long long scan[(kScanBytes + 7) / 8];
    alignas(16) unsigned char walk[sizeof(Walk)];
    int verdict;
};

template <int N8>
__global__ void __launch_bounds__(32 * FewSmem4<N8>::kWarps4, kCtas4) attention_few_q4_kernel(const __grid_constant__ AttnParams p) {
    constexpr int kWarps4 = FewSmem4<N8>::kWarps4, kThreads4 = 32 * kWarps4;
    extern __shared__ __align__(16) unsigned char sm[];
    FewSmem4<N8>& S = *reinterpret_cast<FewSmem4<N8>*>(sm);
    const int warp = uniform(threadIdx.x >> 5), lane = threadIdx.x & 31, r = lane >> 2, c = lane & 3;
    const AttnLaunch& a = p.a;
    const int shift = p.page_shift, heads = a.Hkv;
    Run run;
    if (!find_run<kThreads4>(p, p.tp, heads, S.scan, run)) return;
    if (threadIdx.x == 0) S.run = run;
    __syncthreads();
    Walk* walk = reinterpret_cast<Walk*>(S.walk);
    if (warp == kWarps4 - 1) {  // items, three ahead (a slot is written when every warp is past the item four before)
        Walk w(p, S.run, p.tp, heads, S.scan);
        if (lane == 0) {
            new (walk) Walk(w);
            walk->next(S.items[0]);
        }
    }
    __syncthreads();

    // A thread's place in a block of a page: K's and V's codes and scales.
    const int key = 4 * (r >> 1) + (r & 1);
    const uint32_t at_k = (((c << shift) + key) << 4), at_ks = (64u << shift) + key * 8 + c * 2;
    const uint32_t at_v = (72u << shift) + ((((r >> 1) << shift) + 4 * c) << 4) + (r & 1) * 8;
    const uint32_t at_vs = (136u << shift) + 4 * c * 8 + (r >> 1) * 2;

    auto steps_of = [&](const Item& I) {  // of this warp
        const int keys = min(I.n_tiles * kTileKeys, I.len - I.t0 * kTileKeys);
        return (((keys + 15) >> 4) - warp + kWarps4 - 1) / kWarps4;
    };
    // The pages of the warp's steps i0 to i0 + 31, a step a lane.
    auto window = [&](const Item& I, int i0) {
        const int i = i0 + lane;
        int page = a.num_pages;
        if (i < steps_of(I))
            page = table_page(a, I.seq, a.table + static_cast<size_t>(I.seq) * a.max_blocks,
                              (I.t0 * kTileKeys + (warp + i * kWarps4) * 16) >> shift);
        return page;
    };
    // Where a step's 16 rows begin in K's codes of a page, and in its scales (16 and 8 bytes a row before them); null for a
    // page that is out of range (reported; the sequence's rows are undefined).
    struct Place {
        const uint8_t* codes;
        const uint8_t* scales;
    };
    auto place = [&](const Item& I, int i, int page) {
        if (page >= a.num_pages) return Place{nullptr, nullptr};
        const int row = (warp + i * kWarps4) * 16 & ((1 << shift) - 1);
        const uint8_t* b = static_cast<const uint8_t*>(a.k) + page * a.page_stride +
                           static_cast<long long>(I.g) * (2 * kKv4RowBytes << shift) + row * 8;
        return Place{b + row * 8, b};
    };
    auto load_k = [&](Step& x, const Place& b) {
        if (b.codes) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                x.k[y] = __ldg(reinterpret_cast<const uint4*>(b.codes + at_k + y * 32));
                x.ks[y] = __ldg(reinterpret_cast<const unsigned short*>(b.scales + at_ks + y * 16));
            }
        } else {
            x.k[0] = x.k[1] = make_uint4(0u, 0u, 0u, 0u);
            x.ks[0] = x.ks[1] = 0u;
        }
    };
    auto load_v = [&](Step& x, const Place& b) {
        if (b.codes) {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                x.v[y] = __ldg(reinterpret_cast<const uint2*>(b.codes + at_v + y * 16));
                x.vs[y] = __ldg(reinterpret_cast<const unsigned short*>(b.scales + at_vs + y * 8));
            }
        } else {
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                x.v[y] = make_uint2(0u, 0u);
                x.vs[y] = 0u;
            }
        }
    };
    auto load = [&](Step& x, const Place& b) {
        load_k(x, b);
        load_v(x, b);
    };

    int now = 0;
    Step x;
    {
        const Item& I = S.items[0];
        if (I.part == kEndItem) return;
        now = window(I, 0);
        if (steps_of(I) > 0) load(x, place(I, 0, uniform(__shfl_sync(0xffffffffu, now, 0))));
        if (threadIdx.x == kThreads4 - 32) {  // beside the loads
            walk->next(S.items[1]);
            walk->next(S.items[2]);
        }
        __syncthreads();
    }
    for (int it = 0;; ++it) {
        const Item& I = S.items[it & 3];
        if (I.part == kEndItem) break;
        const Item& J = S.items[(it + 1) & 3];
        const int n = steps_of(I), nj = J.part == kEndItem ? 0 : steps_of(J);
        int ahead = n > 32 ? window(I, 32) : nj > 0 ? window(J, 0) : 0;
        const int rows = I.ntok * p.hp;
        // the query rows, as the second operand
        uint32_t q[N8][16];
#pragma unroll
        for (int b = 0; b < N8; ++b) {
            const int row = b * 8 + r, t = row / p.hp;
            const uint4* src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.q) + (I.q_row + t) * a.q_tok +
                                                              (I.head0 + row - t * p.hp) * a.q_head + c * 32);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const uint4 w = row < rows ? __ldg(src + y) : make_uint4(0u, 0u, 0u, 0u);
                q[b][4 * y] = w.x, q[b][4 * y + 1] = w.y, q[b][4 * y + 2] = w.z, q[b][4 * y + 3] = w.w;
            }
            if (J.part != kEndItem && t < J.ntok)  // the next item's, so that they are near then
                asm volatile("prefetch.global.L1 [%0];" ::"l"(static_cast<const __nv_bfloat16*>(a.q) + (J.q_row + t) * a.q_tok +
                                                              (J.head0 + row - t * p.hp) * a.q_head + c * 32));
        }
        float ref[N8][2], l[N8][2], o[N8][8][4];
        int end[N8][2];  // of the columns: the first key that the row does not see
#pragma unroll
        for (int b = 0; b < N8; ++b) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                ref[b][e] = kNoRef;
                l[b][e] = 0.f;
                end[b][e] = I.pos0 + 1 + (b * 8 + 2 * c + e) / p.hp;
            }
#pragma unroll
            for (int y = 0; y < 8; ++y)
#pragma unroll
                for (int z = 0; z < 4; ++z) o[b][y][z] = 0.f;
        }
        if (n == 0 && nj > 0) {
            now = ahead;
            load(x, place(J, 0, uniform(__shfl_sync(0xffffffffu, now, 0))));
        }
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            // The next step's rows are loaded as soon as this one's are used, K's behind the logits and V's behind the output; with 16
            // rows, where fewer warps hide a load, now.  (8 caches of 131072 tokens, 4 rows, 275 us, 293 with all of them now; 40 of
            // 512 to 16384, 14 rows, 54 and 51: both when the present 269 and 49.5 were 275 and 51.)
            Step here;
            if constexpr (N8 == 2) here = x;
            Step& cur = N8 == 2 ? here : x;
            Place next{nullptr, nullptr};
            if (i + 1 < n) {
                if (((i + 1) & 31) == 0) {
                    now = ahead;
                    ahead = n > i + 33 ? window(I, i + 33) : nj > 0 ? window(J, 0) : 0;
                }
                next = place(I, i + 1, uniform(__shfl_sync(0xffffffffu, now, (i + 1) & 31)));
                if constexpr (N8 == 2) load(x, next);
            } else if (nj > 0) {
                now = ahead;
                next = place(J, 0, uniform(__shfl_sync(0xffffffffu, now, 0)));
                if constexpr (N8 == 2) load(x, next);
            }
            const int k0 = I.t0 * kTileKeys + (warp + i * kWarps4) * 16;
            // ---- logits
            float s[N8][4];
#pragma unroll
            for (int b = 0; b < N8; ++b)
#pragma unroll
                for (int y = 0; y < 4; ++y) s[b][y] = 0.f;
            {
                uint32_t s0, z0, s1, z1;
                kv4_scale(cur.ks[0], s0, z0);
                kv4_scale(cur.ks[1], s1, z1);
                const uint32_t wa[4] = {cur.k[0].x, cur.k[0].y, cur.k[0].z, cur.k[0].w};
                const uint32_t wb[4] = {cur.k[1].x, cur.k[1].y, cur.k[1].z, cur.k[1].w};
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const uint4 ka = kv4_word(wa[w], s0, z0), kb = kv4_word(wb[w], s1, z1);
#pragma unroll
                    for (int b = 0; b < N8; ++b) {
                        mma16816(s[b], ka.x, kb.x, ka.y, kb.y, q[b][4 * w], q[b][4 * w + 1]);
                        mma16816(s[b], ka.z, kb.z, ka.w, kb.w, q[b][4 * w + 2], q[b][4 * w + 3]);
                    }
                }
            }
            if constexpr (N8 == 1) load_k(x, next);
            // ---- numerators
            if (k0 + 16 > I.pos0 + 1) {  // some row does not see some key
                const int j = k0 + key;
#pragma unroll
                for (int b = 0; b < N8; ++b)
#pragma unroll
                    for (int y = 0; y < 4; ++y)
                        if (j + (y >> 1) * 2 >= end[b][y & 1]) s[b][y] = -INFINITY;
                // Rows behind the sequence's end hold anything, and while their numerators are 0, 0 * NaN is not.
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    if (k0 + 4 * c + y >= I.len) cur.vs[y] = 0u;
            }
            float x2[N8][4], over = -INFINITY;  // the logits over their references
#pragma unroll
            for (int b = 0; b < N8; ++b)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    x2[b][y] = fmaf(s[b][y], p.c, -ref[b][y & 1]);
                    over = fmaxf(over, x2[b][y]);
                }
            if (__any_sync(0xffffffffu, over > kAttnTau)) {
                // Move the references that a key passes by more than 2^8 (or that have none yet).
#pragma unroll
                for (int b = 0; b < N8; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float mx = fmaxf(s[b][e], s[b][e + 2]) * p.c;
#pragma unroll
                        for (int y = 4; y < 32; y <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, y));
                        const bool move = mx - ref[b][e] > kAttnTau;
                        const float f = move ? ex2_approx(ref[b][e] - mx) : 1.f;
                        if (move) ref[b][e] = mx;
                        x2[b][e] = fmaf(s[b][e], p.c, -ref[b][e]);
                        x2[b][e + 2] = fmaf(s[b][e + 2], p.c, -ref[b][e]);
                        l[b][e] *= f;
#pragma unroll
                        for (int y = 0; y < 8; ++y) {
                            o[b][y][e] *= f;
                            o[b][y][e + 2] *= f;
                        }
                    }
            }
            uint32_t pb[N8][2];
#pragma unroll
            for (int b = 0; b < N8; ++b) {
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    x2[b][y] = ex2_approx(x2[b][y]);
                    l[b][y & 1] += x2[b][y];
                }
                pb[b][0] = transpose8(pack_bf16(x2[b][0], x2[b][1]));
                pb[b][1] = transpose8(pack_bf16(x2[b][2], x2[b][3]));
            }
            // ---- output
            {
                const uint32_t c01 = __byte_perm(cur.vs[0], cur.vs[1], 0x5410), c23 = __byte_perm(cur.vs[2], cur.vs[3], 0x5410);
                const uint32_t s01 = c01 & 0xfff0fff0u, s23 = c23 & 0xfff0fff0u;
                const uint32_t z01 = kv4_pair(c01), z23 = kv4_pair(c23);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t v0 = w ? cur.v[0].y : cur.v[0].x, v1 = w ? cur.v[1].y : cur.v[1].x;
                    const uint32_t v2 = w ? cur.v[2].y : cur.v[2].x, v3 = w ? cur.v[3].y : cur.v[3].x;
                    // even channels of two keys, odd channels
                    const uint4 e01 = kv4_word(__byte_perm(v0, v1, 0x5410), s01, z01);
                    const uint4 d01 = kv4_word(__byte_perm(v0, v1, 0x7632), s01, z01);
                    const uint4 e23 = kv4_word(__byte_perm(v2, v3, 0x5410), s23, z23);
                    const uint4 d23 = kv4_word(__byte_perm(v2, v3, 0x7632), s23, z23);
#pragma unroll
                    for (int b = 0; b < N8; ++b) {
                        mma16816(o[b][4 * w], e01.x, d01.x, e23.x, d23.x, pb[b][0], pb[b][1]);
                        mma16816(o[b][4 * w + 1], e01.y, d01.y, e23.y, d23.y, pb[b][0], pb[b][1]);
                        mma16816(o[b][4 * w + 2], e01.z, d01.z, e23.z, d23.z, pb[b][0], pb[b][1]);
                        mma16816(o[b][4 * w + 3], e01.w, d01.w, e23.w, d23.w, pb[b][0], pb[b][1]);
                    }
                }
            }
            if constexpr (N8 == 1) load_v(x, next);
        }
        const int buf = it & (FewSmem4<N8>::kBufs - 1);
        // ---- the unit's (or this part's) result: the warps' outputs side by side, then a warp a row
#pragma unroll
        for (int b = 0; b < N8; ++b)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[b][e];
#pragma unroll
                for (int y = 4; y < 32; y <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, y);
                const int row = b * 8 + 2 * c + e;
                if (row >= rows) continue;
                if (r == 0) {
                    S.m[buf][warp][row] = ref[b][e];
                    S.l[buf][warp][row] = sum;
                }
                float4* d = reinterpret_cast<float4*>(&S.o[buf][warp][row][16 * r]);
#pragma unroll
                for (int y = 0; y < 4; ++y)
                    d[y] = make_float4(o[b][2 * y][e], o[b][2 * y][e + 2], o[b][2 * y + 1][e], o[b][2 * y + 1][e + 2]);
            }
        __syncthreads();
        if (threadIdx.x == kThreads4 - 32) walk->next(S.items[(it + 3) & 3]);
        const bool whole = I.part < 0;
        float* part = whole ? nullptr : partial_of<kRows4>(a, blockIdx.x, I.part == 0);
        for (int row = warp; row < rows; row += kWarps4) {
            float wm = lane < kWarps4 ? S.m[buf][lane][row] : kNoRef;
            const float wl = lane < kWarps4 ? S.l[buf][lane][row] : 0.f;
            const float M = redux_max(wm);
            wm = ex2_approx(wm - M);  // (of a warp that saw no key: 0, or 1 for 0 keys)
            const float L = warp_sum(wm * wl);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int y = 0; y < kWarps4; ++y) {
                const float f = __shfl_sync(0xffffffffu, wm, y);
                const float4 v = *reinterpret_cast<const float4*>(&S.o[buf][y][row][4 * lane]);
                acc.x += v.x * f;
                acc.y += v.y * f;
                acc.z += v.z * f;
                acc.w += v.w * f;
            }
            const int t = row / p.hp, h = row - t * p.hp;
            if (whole) {
                const float inv = 1.f / L;
                __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.out) +
                                     (static_cast<long long>(I.q_row + t) * a.Hq + I.head0 + h) * kHeadDim + lane * 4;
                *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                if (lane == 0) write_lse<false>(a, I, t, h, M, L);
            } else {
                reinterpret_cast<float4*>(part + row * 128)[lane] = acc;
                if (lane == 0) {
                    part[kRows4 * 128 + row] = M;
                    part[kRows4 * 129 + row] = L;
                }
            }
        }
        if (FewSmem4<N8>::kBufs == 1 || !whole) __syncthreads();
        if (whole) continue;
        if (threadIdx.x == 0) S.verdict = last_part(a, I);
        __syncthreads();
        if (!S.verdict) continue;
        for (int row = warp; row < rows; row += kWarps4) join_row<kRows4>(a, I, row, row / p.hp, row % p.hp);
    }
}

template <int N8>
cudaError_t launch_few_q4(const AttnLaunch& L, AttnParams& p, cudaStream_t stream) {
    auto kern = attention_few_q4_kernel<N8>;
    static bool configured[kAttnMaxDevices] = {};
    using SM = FewSmem4<N8>;
    constexpr int bytes = static_cast<int>(sizeof(SM));
    static_assert(bytes <= 115712, "shared memory of two CTAs");
    const cudaError_t e = attn_configure(kern, bytes, configured);
    if (e != cudaSuccess) return e;
    const int sms = device_sm_count();
    if (sms <= 0) return cudaErrorNoDevice;
    int grid = sms * kCtas4;
    if (L.max_ctas > 0 && L.max_ctas < sms) grid = L.max_ctas;  // (two could go to an SM each)
    if (grid > kAttnMaxCtas) grid = kAttnMaxCtas;
    NvtxRange range("attention_few_q4_kernel");
    kern<<<grid, 32 * SM::kWarps4, bytes, stream>>>(p);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_few_q4(const AttnLaunch& L, int rows, cudaStream_t stream) {
    AttnParams p;
    memset(&p, 0, sizeof p);
    p.a = L;
    p.G = L.Hq / L.Hkv;
    p.hp = p.G;
    p.tp = (rows <= 8 ? 8 : 16) / p.G;
    p.nhb = 1;
    p.unit_cost = 2;  // key tiles (64 caches of 128 to 8192, now 42.2 us, when they took 45.7: 1 51.4, 3 47.2, 6 52.4)
    p.min_run = 1;
    while ((1 << p.page_shift) < L.page_size) ++p.page_shift;
    p.c = L.scale * 1.4426950408889634f;
    return rows <= 8 ? launch_few_q4<1>(L, p, stream) : launch_few_q4<2>(L, p, stream);
}

}  // namespace ckv
