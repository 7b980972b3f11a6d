// Attention of new tokens over a paged cache of 4 bits (kv4.cuh): a CTA a (token, query head), a key a thread for the
// logits and a channel a thread for the output, one pass over the keys with a running maximum and sum.
#include "attention_common.cuh"
#include "kv4.cuh"

namespace ckv {
namespace {

__global__ void __launch_bounds__(128) attention_q4_kernel(const __grid_constant__ AttnLaunch a, int shift) {
    __shared__ float q[128], p[128];
    __shared__ int where[128];
    __shared__ float red[4];
    const int t = blockIdx.x, h = blockIdx.y, g = h / (a.Hq / a.Hkv), tid = threadIdx.x;
    const int cu0 = a.cu[0];
    bool bad = false;
    int found = -1;
    for (int s = tid; s < a.S; s += 128) {
        const Seq x = get_seq(a, s, cu0, bad, blockIdx.x == 0 && blockIdx.y == 0);
        if (t >= x.row0 && t < x.row0 + x.n) found = s;
    }
    if (__syncthreads_or(bad)) {
        if (t == 0 && h == 0 && tid == 0) record_error(a.status, kDevBadIndex, -1);
        return;
    }
    if (tid == 0) where[0] = -1;
    __syncthreads();
    if (found >= 0) where[0] = found;
    __syncthreads();
    const int seq = where[0];
    if (seq < 0) return;
    bool ignore = false;
    const Seq x = get_seq(a, seq, cu0, ignore, false);
    const int sees = x.len - x.n + t - x.row0 + 1;
    q[tid] = __bfloat162float(static_cast<const __nv_bfloat16*>(a.q)[t * a.q_tok + h * a.q_head + tid]) * a.scale;
    __syncthreads();
    float m = -INFINITY, l = 0.f, o = 0.f;
    const int* row = a.table + static_cast<size_t>(seq) * a.max_blocks;
    for (int j0 = 0; j0 < sees; j0 += 128) {
        const int j = j0 + tid;
        int page = j < sees ? row[j >> shift] : 0;
        if (page < 0 || page >= a.num_pages) {
            record_error(a.status, kDevBadIndex, seq);
            page = 0;
        }
        where[tid] = page;
        const uint8_t* block = static_cast<const uint8_t*>(a.k) + page * a.page_stride + (static_cast<long long>(g) << shift) * (2 * kKv4RowBytes);
        const int r = j & ((1 << shift) - 1);
        float s = 0.f;
        for (int w = 0; w < 16; ++w) {
            uint32_t s2, z2;
            kv4_scale(reinterpret_cast<const uint16_t*>(block + (64 << shift))[r * 4 + (w >> 2)], s2, z2);
            const uint4 v = kv4_word(reinterpret_cast<const uint32_t*>(block)[((((w >> 2) << shift) + r) << 2) + (w & 3)], s2, z2);
            s += bf16_lo(v.x) * q[w * 8] + bf16_hi(v.x) * q[w * 8 + 1] + bf16_lo(v.y) * q[w * 8 + 2] + bf16_hi(v.y) * q[w * 8 + 3] +
                 bf16_lo(v.z) * q[w * 8 + 4] + bf16_hi(v.z) * q[w * 8 + 5] + bf16_lo(v.w) * q[w * 8 + 6] + bf16_hi(v.w) * q[w * 8 + 7];
        }
        if (j >= sees) s = -INFINITY;
        const float wm = redux_max(s);
        if ((tid & 31) == 0) red[tid >> 5] = wm;
        __syncthreads();
        const float mn = fmaxf(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])), m), f = m == -INFINITY ? 0.f : expf(m - mn);
        m = mn;
        p[tid] = s == -INFINITY ? 0.f : expf(s - mn);
        __syncthreads();
        l *= f;
        o *= f;
        for (int k = 0; k < min(128, sees - j0); ++k) {
            const uint8_t* vb = static_cast<const uint8_t*>(a.k) + where[k] * a.page_stride +
                                ((static_cast<long long>(g) << shift) * 2 + (1 << shift)) * kKv4RowBytes;
            const int rk = (j0 + k) & ((1 << shift) - 1), w = tid >> 3, c = tid & 7;
            const uint32_t word = reinterpret_cast<const uint32_t*>(vb)[((((w >> 2) << shift) + rk) << 2) + (w & 3)];
            const uint32_t sc = reinterpret_cast<const uint16_t*>(vb + (64 << shift))[rk * 4 + (w >> 2)];
            const int n = static_cast<int>(word >> (4 * (c >> 1) + 16 * (c & 1))) & 15;
            o += p[k] * __uint_as_float((sc & 0xfff0u) << 16) * static_cast<float>(n - static_cast<int>(sc & 15u));
            l += p[k];
        }
        __syncthreads();
    }
    static_cast<__nv_bfloat16*>(a.out)[(static_cast<long long>(t) * a.Hq + h) * kHeadDim + tid] = __float2bfloat16(o / l);
    if (a.lse && tid == 0) a.lse[h * a.lse_stride + t] = m + logf(l);
}

}  // namespace

cudaError_t launch_attention_q4(const AttnLaunch& L, cudaStream_t stream) {
    int shift = 0;
    while ((1 << shift) < L.page_size) ++shift;
    NvtxRange range("attention_q4_kernel");
    attention_q4_kernel<<<dim3(static_cast<unsigned>(L.T), static_cast<unsigned>(L.Hq)), 128, 0, stream>>>(L, shift);
    return cudaGetLastError();
}

}  // namespace ckv
