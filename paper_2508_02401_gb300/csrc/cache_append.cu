// New tokens' way into the paged cache: queries and keys are rotated by their tokens' positions, keys and values go into
// their slots, as bf16 or in 4 bits (kv4.cuh).
//
// Rotation of a pair (a, b) by the angle t: (a cos t - b sin t, b cos t + a sin t), with cos and sin from the
// caller's table.  The result is the exact one rounded to 32 bits and then to bf16, so that a key's codes in 4 bits do
// not depend on how an fp32 sum happened to be rounded (rotate8).
//
// Bound by memory: every row is read once and written once or twice.  A half-warp takes four rows of one token, 16 bytes a
// lane and row, with the token's angles in registers: loaded once for four rows they cost half of what a row does.
// 40001 kept rows into 4 bits, no rotation (370 MB): 67 us, 5.5 TB/s.  20525 tokens with queries (28 / 4 heads, keys kept too,
// 407 MB): 74.5 us, 5.5 TB/s; 8192 of 32 / 8 heads 42.5 us, 5.2; 7097 into 4 bits 32 us, 4.3, where the rotation and the
// codes keep the schedulers at work.  36 warps an SM (56 registers, some spilled).  That, the rows and their order were measured with the
// rare sums still inlined (the present form was 77.0, 43.1 and 32.8 us then): with 24 / 28 / 32 / 40 warps the second
// took 90.8 / 83.6 / 79.5 / 80.0 us, the third 49.9 / 46.7 / 45.0 / 42.3, the fourth 35.9 / 34.2 / 33.1 /
// 33.8; two rows a half-warp 97, 48 and 39, eight 79, 43 and 37; the warps of a token side by side, for its angles, 78, 42 and 33.
// A decode step's append is a launch and one chain of loads (64 tokens: 2.9 us on the GPU, 3.8 into 4 bits).
#include <float.h>

#include "ckv_device.cuh"
#include "ckv_internal.h"
#include "kv4.cuh"

namespace ckv {
namespace {

constexpr int kAppThreads = 128, kAppCtas = 9;
constexpr int kAppToks = kAppThreads / 16;  // tokens of a CTA
constexpr int kAppQ = 4, kAppKv = 2;        // query heads, KV heads (a row of K and one of V each) of a half-warp
constexpr int kAppRows = 4;
static_assert(kAppQ == kAppRows && 2 * kAppKv == kAppRows, "rows of a half-warp");

enum { kRotNone = 0, kRotHalves = 1, kRotPairs = 2 };

// The angles of a lane's 8 channels: out_i = x_i c_i + y_i s_i with y_i the other value of the pair.
struct Angles {
    float c[8], s[8];
    int src;      // lane (of 16) that holds the other values (halves)
    bool active;  // the channels are rotated
};

template <int ROT>
__device__ __forceinline__ void load_angles(const AppendLaunch& p, int pos, int c, bool live, Angles& A) {
    const int half = p.rotary >> 1;
    A.src = c;
    A.active = live && c * 8 < p.rotary;
    const bool upper = ROT == kRotHalves && c * 8 >= half;
    if (c * 8 < p.rotary && ROT == kRotHalves) A.src = upper ? c - (half >> 3) : c + (half >> 3);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        A.c[i] = 1.f;
        A.s[i] = 0.f;
    }
    if (!A.active) return;
    const float* row = p.cos_sin + static_cast<size_t>(pos) * p.rotary;
    if constexpr (ROT == kRotHalves) {
        const int a = upper ? c * 8 - half : c * 8;
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 co = *reinterpret_cast<const float4*>(row + a + i), si = *reinterpret_cast<const float4*>(row + half + a + i);
            A.c[i] = co.x, A.c[i + 1] = co.y, A.c[i + 2] = co.z, A.c[i + 3] = co.w;
            A.s[i] = si.x, A.s[i + 1] = si.y, A.s[i + 2] = si.z, A.s[i + 3] = si.w;
        }
        if (!upper) {
#pragma unroll
            for (int i = 0; i < 8; ++i) A.s[i] = -A.s[i];
        }
    } else {
        const float4 co = *reinterpret_cast<const float4*>(row + c * 4), si = *reinterpret_cast<const float4*>(row + half + c * 4);
        A.c[0] = A.c[1] = co.x, A.c[2] = A.c[3] = co.y, A.c[4] = A.c[5] = co.z, A.c[6] = A.c[7] = co.w;
        A.s[1] = si.x, A.s[3] = si.y, A.s[5] = si.z, A.s[7] = si.w;
        A.s[0] = -si.x, A.s[2] = -si.y, A.s[4] = -si.z, A.s[6] = -si.w;
    }
}

// a c + b s, rounded to 32 bits.  In 64 bits the products are exact, and a sum rounded to odd (where bits are lost, the neighbour
// whose last bit is 1) rounds to 32 bits as the exact one does.
__device__ __forceinline__ float turn_wide(float a, float c, float b, float s) {
    const double p = static_cast<double>(a) * c, q = static_cast<double>(b) * s, r = p + q, t = r - p, e = (p - (r - t)) + (q - t);
    long long bits = __double_as_longlong(r);
    if ((e > 0.0 || e < 0.0) && !(bits & 1)) bits += (e > 0.0) == (r > 0.0) ? 1 : -1;
    return __double2float_rn(__longlong_as_double(bits));
}

// Bounds of the same: the products' and the sum's rounding errors (exact by fused operations and the known error of a sum
// of two, but for 2^-149 where a product is below what fp32 holds to 24 bits) go to the sum, with their own roundings to either side.
__device__ __forceinline__ void turn_bounds(float a, float c, float b, float s, float& lo, float& hi) {
    // (intrinsics: the compiler would fuse a product with a sum)
    const float p = __fmul_rn(a, c), q = __fmul_rn(b, s), u = __fadd_rn(fmaf(a, c, -p), fmaf(b, s, -q));
    const float r = __fadd_rn(p, q), t = __fadd_rn(r, -p), e = __fadd_rn(__fadd_rn(p, -__fadd_rn(r, -t)), __fadd_rn(q, -t));
    const float v = __fadd_rn(e, u), d = fmaf(__fadd_rn(fabsf(u), fabsf(v)), 0x1p-22f, 0x1p-140f);
    lo = __fadd_rn(r, __fadd_rn(v, -d));
    hi = __fadd_rn(r, __fadd_rn(v, d));
    if (!(hi - lo <= FLT_MAX)) lo = 1.f, hi = 0.f;  // (beyond fp32 on the way: bounds that differ)
    if (a == 0.f && b == 0.f) lo = hi = r;          // (the bounds are -0 and 0)
}

// Two channels (x: their own values, y: the others of their pairs), where the fp32 results do not decide.  A function of its own:
// inlined, with the sum in 64 bits or without, it costs the loops around it registers (20525 tokens 89 and 105 us, 74.6 so).
__device__ __noinline__ uint32_t turn_pair(uint32_t x, uint32_t y, float c0, float s0, float c1, float s1) {
    const float x0 = bf16_lo(x), x1 = bf16_hi(x), y0 = bf16_lo(y), y1 = bf16_hi(y);
    float l[2], h[2];
    turn_bounds(x0, c0, y0, s0, l[0], h[0]);
    turn_bounds(x1, c1, y1, s1, l[1], h[1]);
    const uint32_t lo = pack_bf16x2(l[0], l[1]);
    if (lo == pack_bf16x2(h[0], h[1])) return lo;
    return pack_bf16x2(turn_wide(x0, c0, y0, s0), turn_wide(x1, c1, y1, s1));
}

// A lane's 8 channels of a row, rotated (a whole half-warp).  The fp32 result r = a c + q, q = b s, is off by 2^-24 (|q| + |r|)
// at most, or by 2^-149 among the smallest numbers; where all numbers so near round to one bf16 number, that is the result (roundings
// keep the order of numbers).  Otherwise (one pair in 2000) closer bounds decide, and where those differ too the sum in 64 bits.
template <int ROT>
__device__ __forceinline__ uint4 rotate8(const uint4& x4, const Angles& A) {
    const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
    uint32_t y[4];
    if constexpr (ROT == kRotHalves) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __shfl_sync(0xffffffffu, x[i], A.src, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __byte_perm(x[i], x[i], 0x1032);
    }
    if (!A.active) return x4;
    uint32_t lo[4], hi[4], differ = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float l[2], h[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float xf = e ? bf16_hi(x[i]) : bf16_lo(x[i]), yf = e ? bf16_hi(y[i]) : bf16_lo(y[i]);
            const float q = yf * A.s[2 * i + e], r = fmaf(xf, A.c[2 * i + e], q);
            const float w = fabsf(q) + (fabsf(r) + 0x1p-124f);
            l[e] = fmaf(w, -0x1.00001p-24f, r);
            h[e] = fmaf(w, 0x1.00001p-24f, r);
        }
        lo[i] = pack_bf16x2(l[0], l[1]);
        hi[i] = pack_bf16x2(h[0], h[1]);
        differ |= lo[i] ^ hi[i];
    }
    if (differ) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lo[i] != hi[i]) lo[i] = turn_pair(x[i], y[i], A.c[2 * i], A.s[2 * i], A.c[2 * i + 1], A.s[2 * i + 1]);
    }
    return make_uint4(lo[0], lo[1], lo[2], lo[3]);
}

template <bool Q4, int ROT>
__global__ void __launch_bounds__(kAppThreads, kAppCtas) cache_append_kernel(const __grid_constant__ AppendLaunch p) {
    const int c = threadIdx.x & 15;
    const int nq = p.q ? (p.Hq + kAppQ - 1) / kAppQ : 0, chunks = nq + (p.Hkv + kAppKv - 1) / kAppKv;
    const int block = blockIdx.x / chunks, ch = blockIdx.x - block * chunks;
    const int t = block * kAppToks + static_cast<int>(threadIdx.x >> 4);
    bool live = t < p.T;
    // Every load that does not wait for another goes first: the rows, the position, the slot.
    const bool query = ROT != kRotNone && ch < nq;
    const int h0 = query ? ch * kAppQ : (ch - nq) * kAppKv;
    uint4 x[kAppRows];  // queries, or K and V of each head
#pragma unroll
    for (int u = 0; u < kAppRows; ++u) {
        const int h = query ? h0 + u : h0 + (u >> 1);
        const bool v = u & 1;
        x[u] = make_uint4(0u, 0u, 0u, 0u);
        if (live && h < (query ? p.Hq : p.Hkv)) {
            const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(query ? p.q : v ? p.v : p.k);
            x[u] = *reinterpret_cast<const uint4*>(src + (query ? t * p.q_tok + h * p.q_head : t * p.tok_stride + h * p.head_stride) + c * 8);
        }
    }
    int slot = live && !query ? p.slots[t] : -1;
    Angles A;
    if constexpr (ROT != kRotNone) {
        const int pos = live ? p.positions[t] : -1;
        if (pos < 0 || pos >= p.num_positions) {
            if (pos != -1 && c == 0) record_error(p.status, kDevBadIndex, t);
            live = false;
        }
        load_angles<ROT>(p, pos, c, live, A);
    }
    if (query) {
#pragma unroll
        for (int u = 0; u < kAppQ; ++u) {
            if constexpr (ROT != kRotNone) x[u] = rotate8<ROT>(x[u], A);
            if (live && h0 + u < p.Hq)
                *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.q_out) +
                                          (static_cast<long long>(t) * p.Hq + h0 + u) * kHeadDim + c * 8) = x[u];
        }
        return;
    }
    if (!live) slot = -1;
    if (slot < -1 || slot >= p.num_slots) {
        if (c == 0 && h0 == 0) record_error(p.status, kDevBadIndex, t);
        slot = -1;
    }
    const long long page = slot >> p.shift;
    const int row = slot & ((1 << p.shift) - 1);
#pragma unroll
    for (int u = 0; u < kAppKv; ++u) {
        uint4 k = x[2 * u];
        const uint4 v = x[2 * u + 1];
        if constexpr (ROT != kRotNone) k = rotate8<ROT>(k, A);
        const bool has = live && h0 + u < p.Hkv;
        const long long to = (static_cast<long long>(t) * p.Hkv + h0 + u) * kHeadDim + c * 8;
        if constexpr (Q4) {
            const Kv4Lane kq = kv4_quantise(k), vq = kv4_quantise(v);
            if (has && slot >= 0) {
                uint8_t* d = static_cast<uint8_t*>(p.k_pages) + page * p.page_stride +
                             (static_cast<long long>(h0 + u) << p.shift) * (2 * kKv4RowBytes);
                kv4_store(d, p.shift, row, c, kq);
                kv4_store(d + (kKv4RowBytes << p.shift), p.shift, row, c, vq);
            }
            if (has && p.k_out) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.k_out) + to) = kv4_values(kq);
            if (has && p.v_out) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.v_out) + to) = kv4_values(vq);
        } else {
            if (has && slot >= 0) {
                const long long d = page * p.page_stride + (static_cast<long long>(row) * p.Hkv + h0 + u) * kHeadDim + c * 8;
                *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.k_pages) + d) = k;
                *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.v_pages) + d) = v;
            }
            if (has && p.k_out) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.k_out) + to) = k;
        }
    }
}

template <bool Q4, int ROT>
cudaError_t launch(const AppendLaunch& L, unsigned grid, cudaStream_t stream) {
    cache_append_kernel<Q4, ROT><<<grid, kAppThreads, 0, stream>>>(L);
    return cudaGetLastError();
}

}  // namespace

long long append_blocks(int T, int Hq, int Hkv) {
    return static_cast<long long>((T - 1) / kAppToks + 1) * ((Hq + kAppQ - 1) / kAppQ + (Hkv + kAppKv - 1) / kAppKv);
}

cudaError_t launch_cache_append(const AppendLaunch& L, cudaStream_t stream) {
    const unsigned grid = static_cast<unsigned>(append_blocks(L.T, L.q ? L.Hq : 0, L.Hkv));
    NvtxRange range("cache_append_kernel");
    const int rot = !L.cos_sin ? kRotNone : L.interleaved ? kRotPairs : kRotHalves;
    if (L.q4)
        return rot == kRotNone ? launch<true, kRotNone>(L, grid, stream)
               : rot == kRotPairs ? launch<true, kRotPairs>(L, grid, stream) : launch<true, kRotHalves>(L, grid, stream);
    return rot == kRotPairs ? launch<false, kRotPairs>(L, grid, stream) : launch<false, kRotHalves>(L, grid, stream);
}

}  // namespace ckv
