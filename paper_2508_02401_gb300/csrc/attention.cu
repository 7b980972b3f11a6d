// Causal attention of packed prompts and of new tokens over a paged cache.
//
// Query row i of a sequence with n query rows and L keys stands at position L - n + i and sees keys
// j <= L - n + i:  o = sum_j exp(c q.k_j - lse) v_j,  lse = log sum_j exp(c q.k_j).
#include "ckv_device.cuh"
#include "ckv_internal.h"

namespace ckv {
namespace {

constexpr int kWarps = 8;

// One warp per (query row, head), four dims a lane, one key at a time with a running maximum.
__global__ void __launch_bounds__(kWarps * 32) attention_rows_kernel(const __grid_constant__ AttnLaunch p) {
    const int lane = threadIdx.x & 31;
    const long long unit = static_cast<long long>(blockIdx.x) * kWarps + (threadIdx.x >> 5);
    const long long t = unit / p.Hq;
    const int h = static_cast<int>(unit - t * p.Hq);
    bool bad = false;  // cu has to rise from row 0 to at most T
    for (int s = lane; s < p.S; s += 32)
        bad |= p.cu[s + 1] < p.cu[s] || p.cu[s] < p.cu[0] || p.cu[s + 1] - p.cu[0] > p.T;
    if (__any_sync(0xffffffffu, bad)) {
        if (lane == 0) record_error(p.status, kDevBadIndex, -1);
        return;
    }
    if (p.check_hash && unit == 0 && lane == 0 && seqlens_hash(p.cu, p.S) != p.cu_hash)
        record_error(p.status, kDevBadSeqlens, 120);
    if (t >= p.T) return;
    int lo = 0, hi = p.S;  // the sequence of row t: cu[lo] <= t < cu[lo + 1]
    const int base = p.cu[0];
    if (t >= p.cu[p.S] - base || base < 0) return;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (p.cu[mid] - base <= t) lo = mid;
        else hi = mid;
    }
    const int s = lo, row0 = p.cu[s] - base, n = p.cu[s + 1] - p.cu[s];
    const int len = p.lens ? p.lens[s] : n;
    if (len < n || (p.paged && len > static_cast<long long>(p.max_blocks) * p.page_size)) {
        if (lane == 0) record_error(p.status, kDevBadIndex, s);
        return;
    }
    const int i = static_cast<int>(t) - row0, seen = len - n + i + 1, g = h / (p.Hq / p.Hkv);
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    const __nv_bfloat16* qp = static_cast<const __nv_bfloat16*>(p.q) + t * p.q_tok + h * p.q_head + lane * 4;
    for (int c = 0; c < 4; ++c) q[c] = __bfloat162float(qp[c]) * p.scale;
    for (int j = 0; j < seen; ++j) {
        long long at;
        if (p.paged) {
            const int page = p.table[static_cast<size_t>(s) * p.max_blocks + j / p.page_size];
            if (page < 0 || page >= p.num_pages) {
                if (lane == 0) record_error(p.status, kDevBadIndex, s);
                return;
            }
            at = page * p.page_stride + static_cast<long long>(j % p.page_size) * p.Hkv * kHeadDim + g * kHeadDim;
        } else {
            at = (row0 + j) * p.tok_stride + g * p.head_stride;
        }
        const __nv_bfloat16* kp = static_cast<const __nv_bfloat16*>(p.k) + at + lane * 4;
        const __nv_bfloat16* vp = static_cast<const __nv_bfloat16*>(p.v) + at + lane * 4;
        float x = 0.f;
        for (int c = 0; c < 4; ++c) x += q[c] * __bfloat162float(kp[c]);
        x = warp_sum(x);
        const float mn = fmaxf(m, x), ms = mn == -INFINITY ? 0.f : mn;
        const float f = expf(m - ms), e = expf(x - ms);
        l = l * f + e;
        m = mn;
        for (int c = 0; c < 4; ++c) o[c] = o[c] * f + e * __bfloat162float(vp[c]);
    }
    __nv_bfloat16* op = static_cast<__nv_bfloat16*>(p.out) + (t * p.Hq + h) * kHeadDim + lane * 4;
    for (int c = 0; c < 4; ++c) op[c] = __float2bfloat16(o[c] / l);
    if (lane == 0) {
        const float lse = m + logf(l);
        if (p.lse) p.lse[h * p.lse_stride + t] = lse;
        if (p.lse_win && i >= n - p.w) p.lse_win[h * p.lse_win_stride + static_cast<long long>(s) * p.w + (i - (n - p.w))] = lse;
    }
}

}  // namespace

cudaError_t launch_attention(const AttnLaunch& L, cudaStream_t stream) {
    if (L.T == 0) return cudaSuccess;
    const long long units = static_cast<long long>(L.T) * L.Hq;
    NvtxRange range("attention_rows_kernel");
    attention_rows_kernel<<<static_cast<unsigned>((units + kWarps - 1) / kWarps), kWarps * 32, 0, stream>>>(L);
    return cudaGetLastError();
}

}  // namespace ckv
