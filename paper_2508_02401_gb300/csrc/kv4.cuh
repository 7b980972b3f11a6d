// A row of 128 values in 4 bits: four groups of 32 channels, each with a scale s of 4 significant bits and a zero point z.
//   wide = max(x, 0) - min(x, 0), rounded to fp32;  s = the least such number, 2^-100 at least, with 15 s >= wide
//   z = round(-min(x, 0) / s),  n = clamp(round(x / s) + z, 0, 15)  (ties to even);  the value is s (n - z)
// |value - x| <= s / 2: max / s - min / s <= 15, so a code is clamped only where two ties were both rounded up.  (The
// rounding of the range changes nothing of it: where it does round, the smaller of max and -min is below 2^-15 of the range, its
// codes are those of 0, and the larger is 15 s at most.)  n - z
// has 4 bits and a sign, s 4 significant bits, so the value is a bf16 number: nothing that reads the cache rounds it.
// A group with a NaN, an infinity or a range beyond fp32 has s = NaN: every value of it is NaN.
//
// In a page of P tokens, per head: K's codes [4 groups][P][16 bytes], K's scales [P][4 groups][2 bytes], then V's.  A
// group's 16 bytes are four words of 8 channels, channel c of a word in nibble c / 2 + 4 (c % 2), so that a mask of
// two nibbles gives a pair of neighbours (a mask and a magic exponent: a published technique of 4-bit kernels).  A scale is its bf16 pattern, whose low nibble is free: z.
#pragma once

#include <float.h>

#include "ckv_device.cuh"

namespace ckv {

constexpr int kKv4RowBytes = 72;  // 64 of codes, 8 of scales

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }
__device__ __forceinline__ uint32_t bf16x2_sub(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_mul(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_min_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_max_nan(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// (w & 0x000f000f) | 0x43004300 in one instruction (the compiler makes two of it).
__device__ __forceinline__ uint32_t kv4_pair(uint32_t w) {
    uint32_t r;
    asm("lop3.b32 %0, %1, 0x000f000f, 0x43004300, 0xea;" : "=r"(r) : "r"(w));
    return r;
}

// A scale word's pair (s, s) and pair (128 + z, 128 + z) in bf16.
__device__ __forceinline__ void kv4_scale(uint32_t word, uint32_t& s2, uint32_t& z2) {
    const uint32_t both = __byte_perm(word, 0u, 0x1010);
    s2 = both & 0xfff0fff0u;
    z2 = kv4_pair(both);
}

// The 8 values of a word as four bf16 pairs.  0x4300 | n is 128 + n (bf16 has steps of 1 there); the difference of two
// such numbers and its product with s are exact.
__device__ __forceinline__ uint4 kv4_word(uint32_t w, uint32_t s2, uint32_t z2) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = bf16x2_mul(bf16x2_sub(kv4_pair(w >> (4 * i)), z2), s2);
    return make_uint4(x[0], x[1], x[2], x[3]);
}

// A lane's share of a row (16 lanes of a half-warp, 8 channels each, a group in 4 of them).
struct Kv4Lane {
    uint32_t word;   // codes
    uint32_t scale;  // the group's
};

__device__ __forceinline__ uint4 kv4_values(const Kv4Lane& q) {
    uint32_t s2, z2;
    kv4_scale(q.scale, s2, z2);
    return kv4_word(q.word, s2, z2);
}

// A whole warp, two rows.
__device__ __forceinline__ Kv4Lane kv4_quantise(const uint4& x4) {
    const uint32_t x[4] = {x4.x, x4.y, x4.z, x4.w};
    uint32_t mn = bf16x2_min_nan(bf16x2_min_nan(x[0], x[1]), bf16x2_min_nan(x[2], x[3]));
    uint32_t mx = bf16x2_max_nan(bf16x2_max_nan(x[0], x[1]), bf16x2_max_nan(x[2], x[3]));
    mn = bf16x2_min_nan(mn, 0u);
    mx = bf16x2_max_nan(mx, 0u);
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        mn = bf16x2_min_nan(mn, __shfl_xor_sync(0xffffffffu, mn, o));
        mx = bf16x2_max_nan(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    }
    mn = bf16x2_min_nan(mn, __byte_perm(mn, mn, 0x1032));
    mx = bf16x2_max_nan(mx, __byte_perm(mx, mx, 0x1032));
    const float low = bf16_lo(mn), wide = bf16_lo(mx) - low;
    Kv4Lane q;
    if (!(wide <= FLT_MAX)) {
        q.word = 0u;
        q.scale = 0x7fc0u;
        return q;
    }
    // The quotient is off by a rounding or two, its first 4 bits by one step down at most where it matters: where wide is
    // 15 s exactly, which the product tells (exact in 32 bits).
    uint32_t sb = __float_as_uint(wide * (1.f / 15.f)) & 0xfff00000u;
    if (__uint_as_float(sb) * 15.f < wide) sb += 1u << 20;
    const float s = fmaxf(__uint_as_float(sb), 0x1p-100f), inv = __frcp_rn(s);
    // x / s to an integer.  x / s is a tie, or 2^-9 and more away from one (x has 8 significant bits, s 4); x * inv is 2^-19
    // off at most.  Rounded to steps of 2^-11 (the sum with 6144) a tie is a tie again, and the second sum rounds
    // it to even.
    auto whole = [&](float v) { return static_cast<int>(__float_as_uint(fmaf(v, inv, 6144.f) + (12582912.f - 6144.f))) - 0x4B400000; };
    const int z = whole(-low);
    uint32_t w = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int a = min(max(whole(bf16_lo(x[i])) + z, 0), 15), b = min(max(whole(bf16_hi(x[i])) + z, 0), 15);
        w |= static_cast<uint32_t>(a) << (4 * i) | static_cast<uint32_t>(b) << (4 * i + 16);
    }
    q.word = w;
    q.scale = (__float_as_uint(s) >> 16) | static_cast<uint32_t>(z);
    return q;
}

// A row's 64 bytes of codes and its four scale words, from a block of a page of 1 << shift tokens in shared memory.
struct Kv4Row {
    uint4 codes[4];
    uint2 scales;
};
__device__ __forceinline__ Kv4Row kv4_row(const uint8_t* block, int shift, int row) {
    Kv4Row r;
#pragma unroll
    for (int g = 0; g < 4; ++g) r.codes[g] = *reinterpret_cast<const uint4*>(block + (((g << shift) + row) << 4));
    r.scales = *reinterpret_cast<const uint2*>(block + (64 << shift) + row * 8);
    return r;
}
// Group g's 32 values as 16 bf16 pairs.
__device__ __forceinline__ void kv4_group(const Kv4Row& r, int g, uint32_t (&v)[16]) {
    uint32_t s2, z2;
    const uint32_t pair = g < 2 ? r.scales.x : r.scales.y;
    kv4_scale(g & 1 ? pair >> 16 : pair & 0xffffu, s2, z2);
    const uint32_t w[4] = {r.codes[g].x, r.codes[g].y, r.codes[g].z, r.codes[g].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4 x = kv4_word(w[i], s2, z2);
        v[4 * i] = x.x;
        v[4 * i + 1] = x.y;
        v[4 * i + 2] = x.z;
        v[4 * i + 3] = x.w;
    }
}

// The lane's share into `row` of a page's K or V block of one head.
__device__ __forceinline__ void kv4_store(uint8_t* block, int shift, int row, int c, const Kv4Lane& q) {
    *reinterpret_cast<uint32_t*>(block + ((((c >> 2) << shift) + row) << 4) + ((c & 3) << 2)) = q.word;
    if ((c & 3) == 0) *reinterpret_cast<uint16_t*>(block + (64 << shift) + row * 8 + (c >> 2) * 2) = static_cast<uint16_t>(q.scale);
}

}  // namespace ckv
