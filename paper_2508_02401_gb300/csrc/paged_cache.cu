// The paged cache that the kept rows and the new tokens live in: block tables and slot maps built
// on the GPU from the rows' lengths (block_tables_kernel) and the copy of packed K/V rows into
// their slots (cache_write_kernel).
#include "ckv_device.cuh"
#include "ckv_internal.h"

namespace ckv {
namespace {

constexpr int kTabThreads = 1024;

struct TablesParams {
    TablesLaunch a;
    int shift;         // log2(page_size)
    long long seg;     // entries of the slot map of one CTA's share
};

struct RowCounts {
    long long add, take, give;
};

// Row r: tokens it gains, pages it takes, pages it gives back; false if its lengths make no sense.
__device__ __forceinline__ bool row_counts(const TablesParams& p, int r, int& len, RowCounts& c) {
    len = p.a.lens[r];
    const int nw = p.a.new_lens[r];
    const long long P1 = (1ll << p.shift) - 1;
    const long long have = (static_cast<long long>(len) + P1) >> p.shift;
    const long long add = nw > 0 ? nw : 0;
    c.add = add;
    c.take = ((len + add + P1) >> p.shift) - have;
    c.give = nw < 0 ? have : 0;
    return len >= 0 && nw >= -1 && len + add <= static_cast<long long>(p.a.max_blocks) << p.shift;
}

// Exclusive prefix sums over the block's threads of three values; `total` are the sums.
__device__ __forceinline__ RowCounts block_scan(const RowCounts& v, RowCounts* warp_sums, RowCounts* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    auto warp_scan = [&](RowCounts x) {
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long a = __shfl_up_sync(0xffffffffu, x.add, o), t = __shfl_up_sync(0xffffffffu, x.take, o),
                            g = __shfl_up_sync(0xffffffffu, x.give, o);
            if (lane >= o) {
                x.add += a;
                x.take += t;
                x.give += g;
            }
        }
        return x;
    };
    const RowCounts x = warp_scan(v);
    if (lane == 31) warp_sums[warp] = x;
    __syncthreads();
    if (warp == 0) warp_sums[lane] = warp_scan(warp_sums[lane]);
    __syncthreads();
    *total = warp_sums[31];
    const RowCounts b = warp ? warp_sums[warp - 1] : RowCounts{0, 0, 0};
    return {x.add - v.add + b.add, x.take - v.take + b.take, x.give - v.give + b.give};
}

// The thread whose share [first[i], first[i + 1]) holds x (shares may be empty; x < first[1024]).
__device__ __forceinline__ int find_share(const long long* first, long long x) {
    int lo = 0, hi = kTabThreads;  // first[lo] <= x < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

// One launch, no CTA waits for another: every CTA computes the prefix sums over all rows itself
// (n * 8 bytes from L2) and then writes its share of the slot map, the table entries of the pages
// whose first token lies in that share, and every grid-th page given back.  A token's row is found
// by bisection over the 1024 threads' shares of rows and a walk of at most n / 1024 rows.  Lengths and
// the pool counters are written by the CTA that finishes last, when all have read them, so they may be
// updated in place; the new blocks' entries and the ring's free part are disjoint from what is read.
__global__ void __launch_bounds__(kTabThreads) block_tables_kernel(const __grid_constant__ TablesParams p) {
    __shared__ long long first_tok[kTabThreads + 1], first_page[kTabThreads + 1], first_back[kTabThreads + 1];
    __shared__ RowCounts warp_sums[32];
    __shared__ int last_s;
    const int n = p.a.n_rows, tid = threadIdx.x;
    const int per = (n - 1) / kTabThreads + 1;
    const int r0 = min(static_cast<long long>(tid) * per, static_cast<long long>(n)), r1 = r0 + min(per, n - r0);
    bool bad = false;
    RowCounts sum{0, 0, 0};
    for (int r = r0; r < r1; ++r) {
        int len;
        RowCounts c;
        if (!row_counts(p, r, len, c)) {
            bad = true;
            continue;
        }
        sum.add += c.add;
        sum.take += c.take;
        sum.give += c.give;
    }
    const long long taken = p.a.pool[0], returned = p.a.pool[1], cap_pages = p.a.num_pages;
    RowCounts total;
    const RowCounts before = block_scan(sum, warp_sums, &total);
    const long long toks = total.add, pages = total.take, back = total.give;
    first_tok[tid] = before.add;
    first_page[tid] = before.take;
    first_back[tid] = before.give;
    if (tid == 0) {
        first_tok[kTabThreads] = toks;
        first_page[kTabThreads] = pages;
        first_back[kTabThreads] = back;
    }
    const bool bad_rows = __syncthreads_or(bad);
    int why = 0;  // the status detail
    if (bad_rows) why = 1;
    else if (toks > p.a.cap) why = 2;
    else if (taken < 0 || returned < taken || returned - taken > cap_pages ||
             returned - taken + back > cap_pages)
        why = 3;
    else if (pages > returned - taken) why = 4;
    const bool ok = why == 0;
    if (!ok && blockIdx.x == 0 && tid == 0) record_error(p.a.status, kDevPool, why);

    // ring positions of the first page taken and given back; from there on less than one round
    const long long take0 = ok ? taken % cap_pages : 0, give0 = ok ? returned % cap_pages : 0;
    const int P1 = (1 << p.shift) - 1;
    const long long a = blockIdx.x * p.seg;
    const long long b = min(a + p.seg, static_cast<long long>(p.a.cap));
    for (long long t = a + tid; t < b; t += kTabThreads) {
        int slot = -1;
        if (ok && t < toks) {
            const int share = find_share(first_tok, t);
            long long at = first_tok[share], page0 = first_page[share];
            int r = share * per, len;
            RowCounts c;
            for (;; ++r) {
                row_counts(p, r, len, c);
                if (t < at + c.add) break;
                at += c.add;
                page0 += c.take;
            }
            const int pos = len + static_cast<int>(t - at);
            const int block = pos >> p.shift, have = (len + P1) >> p.shift;
            int* entry = p.a.table + static_cast<size_t>(r) * p.a.max_blocks + block;
            int page;
            if (block < have) {
                page = *entry;
            } else {
                const long long x = take0 + page0 + (block - have);
                page = p.a.free_pages[x < cap_pages ? x : x - cap_pages];
                if ((pos & P1) == 0) *entry = page;
            }
            if (page < 0 || page >= p.a.num_pages) record_error(p.a.status, kDevBadIndex, r);
            else slot = (page << p.shift) + (pos & P1);
        }
        p.a.slots[t] = slot;
    }
    if (ok) {
        for (long long x = static_cast<long long>(blockIdx.x) * kTabThreads + tid; x < back;
             x += static_cast<long long>(gridDim.x) * kTabThreads) {
            const int share = find_share(first_back, x);
            long long at = first_back[share];
            int r = share * per, len;
            RowCounts c;
            for (;; ++r) {
                row_counts(p, r, len, c);
                if (x < at + c.give) break;
                at += c.give;
            }
            const long long to = give0 + x;
            int page = p.a.table[static_cast<size_t>(r) * p.a.max_blocks + (x - at)];
            if (page < 0 || page >= p.a.num_pages) {  // (its place in the ring is counted already)
                record_error(p.a.status, kDevBadIndex, r);
                page = -1;
            }
            p.a.free_pages[to < cap_pages ? to : to - cap_pages] = page;
        }
    }
    if (blockIdx.x == 0) {
        long long at = first_tok[tid];
        for (int r = r0; r < r1; ++r) {
            p.a.cu[r] = ok ? static_cast<int>(at) : 0;
            int len;
            RowCounts c;
            row_counts(p, r, len, c);
            at += c.add;
        }
        if (tid == 0) p.a.cu[n] = ok ? static_cast<int>(toks) : 0;
    }
    // the last CTA updates what the others read
    __syncthreads();
    if (tid == 0) {
        __threadfence();
        const int k = gridDim.x > 1 ? atomicAdd(p.a.ticket, 1) : 0;
        last_s = k == static_cast<int>(gridDim.x) - 1;
        if (last_s && gridDim.x > 1) *p.a.ticket = 0;
        __threadfence();
    }
    __syncthreads();
    if (!last_s) return;
    for (int r = r0; r < r1; ++r) {
        int len;
        RowCounts c;
        row_counts(p, r, len, c);
        p.a.lens_out[r] = !ok ? len : p.a.new_lens[r] < 0 ? 0 : len + static_cast<int>(c.add);
    }
    if (tid == 0) {
        p.a.pool_out[0] = taken + (ok ? pages : 0);
        p.a.pool_out[1] = returned + (ok ? back : 0);
    }
}

constexpr int kWriteUnroll = 4;   // rows in flight per half-warp
constexpr int kWriteThreads = 256;
constexpr int kWriteRows = kWriteThreads / 16 * kWriteUnroll;

// A row is one (token, head): 256 bytes of K and of V, 16 bytes a lane of a half-warp.
__global__ void __launch_bounds__(kWriteThreads) cache_write_kernel(const __grid_constant__ CacheWriteLaunch p) {
    const int c = threadIdx.x & 15;
    const long long row0 = static_cast<long long>(blockIdx.x) * kWriteRows + (threadIdx.x >> 4);
    const long long rows = static_cast<long long>(p.T) * p.Hkv;
    uint4 k[kWriteUnroll], v[kWriteUnroll];
    long long dst[kWriteUnroll];
#pragma unroll
    for (int u = 0; u < kWriteUnroll; ++u) {
        const long long row = row0 + u * (kWriteThreads / 16);
        dst[u] = -1;
        if (row >= rows) continue;
        const int t = static_cast<int>(row / p.Hkv), g = static_cast<int>(row - static_cast<long long>(t) * p.Hkv);
        const int slot = p.slots[t];
        if (slot < 0 || slot >= p.num_slots) {
            if (slot != -1 && c == 0) record_error(p.status, kDevBadIndex, t);
            continue;
        }
        dst[u] = static_cast<long long>(slot >> p.shift) * p.page_stride +
                 (static_cast<long long>(slot & ((1 << p.shift) - 1)) * p.Hkv + g) * kHeadDim + c * 8;
        const long long src = t * p.tok_stride + g * p.head_stride + c * 8;
        k[u] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.k) + src);
        v[u] = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.v) + src);
    }
#pragma unroll
    for (int u = 0; u < kWriteUnroll; ++u) {
        if (dst[u] < 0) continue;
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.k_pages) + dst[u]) = k[u];
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.v_pages) + dst[u]) = v[u];
    }
}

}  // namespace

cudaError_t launch_block_tables(const TablesLaunch& L, cudaStream_t stream) {
    TablesParams p;
    p.a = L;
    p.shift = 0;
    while ((1 << p.shift) < L.page_size) ++p.shift;
    // One wave of CTAs (each repeats the prefix sums over the rows), of 256 tokens or more: 256 rows of 1000 tokens
    // 7.2 us, 10.8 with two waves, 19.0 with four; 2048 rows of 4 tokens 6.7 us, 7.2 with 512 and more a CTA,
    // 11.3 with 4096.
    // A CTA for every 64 rows, too, whose pages may go back: 5000 rows of up to 4000 tokens, a third of them given back, 13.3 us,
    // with the tokens' CTAs alone 22.5 (64 rows in two CTAs instead of one: 6.2 us, 5.2).
    const int sms = device_sm_count() > 0 ? device_sm_count() : 1;
    const long long work = max(static_cast<long long>(L.cap), 256ll * ((L.n_rows - 1) / 64 + 1));
    p.seg = max(256ll, (work + sms - 1) / sms);
    const long long grid = (work + p.seg - 1) / p.seg;
    NvtxRange range("block_tables_kernel");
    block_tables_kernel<<<static_cast<unsigned>(grid), kTabThreads, 0, stream>>>(p);
    return cudaGetLastError();
}

cudaError_t launch_cache_write(const CacheWriteLaunch& L, cudaStream_t stream) {
    const long long rows = static_cast<long long>(L.T) * L.Hkv;
    if (rows == 0) return cudaSuccess;
    NvtxRange range("cache_write_kernel");
    cache_write_kernel<<<static_cast<unsigned>((rows + kWriteRows - 1) / kWriteRows), kWriteThreads, 0, stream>>>(L);
    return cudaGetLastError();
}

}  // namespace ckv
