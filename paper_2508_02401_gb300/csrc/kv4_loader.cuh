// Tiles of 128 cached rows in 4 bits, from the pages into a ring of shared memory and from there, as bf16, into the tiles
// that the MMAs read.
#pragma once

#include "attention_common.cuh"
#include "kv4.cuh"

namespace ckv {
namespace {

constexpr int kPackedTile = kKv4RowBytes * kTileKeys;  // K or V of 128 tokens of a head: 9 KB
static_assert(kPackedTile % 16 == 0, "alignment");

__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_u32(dst)),
                 "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// One warp loads an item's packed tiles into the ring: K0 V0 K1 V1 ..., a page a lane (its block of K or V is one copy:
// a multiple of 1152 bytes at such an offset, so the 16-byte rule of copies holds for any page size).  A page that is out of
// range is not loaded: `loaded` has a bit a page of each slot's tile, for the unpacking warps, to which the others' rows are zeros.
template <int RING>
struct PackedLoader {
    const AttnParams& p;
    uint8_t* ring;
    uint64_t* full;
    uint64_t* freed;
    uint32_t* loaded;
    volatile int* abort;
    long long lim;
    uint32_t slot = 0, phase = 1, use = 0;

    __device__ bool load(const Item& I, int page, int first, int v) {
        if (!warp_wait(&freed[slot], phase, abort, lim)) return false;
        const AttnLaunch& a = p.a;
        const int lane = threadIdx.x & 31;
        const uint32_t bytes = kKv4RowBytes << p.page_shift;
        const bool mine = lane >= first && lane < first + (kTileKeys >> p.page_shift) && page < a.num_pages;
        const uint32_t pages = __ballot_sync(0xffffffffu, mine);
        if (lane == 0) {
            loaded[slot] = pages >> first;  // (published by the arrival)
            mbar_arrive_expect_tx(&full[slot], __popc(pages) * bytes);
        }
        __syncwarp();
        if (mine)
            bulk_load(ring + slot * kPackedTile + (lane - first) * bytes,
                      static_cast<const uint8_t*>(a.k) + page * a.page_stride + (2ll * I.g + v) * bytes, bytes, &full[slot]);
        __syncwarp();
        ++use;
        if (++slot == RING) {
            slot = 0;
            phase ^= 1;
        }
        return true;
    }

    __device__ bool item(const Item& I) {
        // Page indices: lane l holds block l of a window of 32 blocks, the next window's at hand.
        const AttnLaunch& a = p.a;
        const int ppt_shift = 7 - p.page_shift, win_shift = 5 - ppt_shift;  // pages a tile, tiles a window
        const int blocks = (I.len + a.page_size - 1) >> p.page_shift;
        const int* row = a.table + static_cast<size_t>(I.seq) * a.max_blocks;
        auto window = [&](int u) {
            const int b = ((I.t0 + u) << ppt_shift) + static_cast<int>(threadIdx.x & 31);
            return b < blocks && u < I.n_tiles ? table_page(a, I.seq, row, b) : a.num_pages;
        };
        const int per = 1 << win_shift;
        int now = window(0), ahead = window(per);
        for (int u = 0; u < I.n_tiles; ++u) {
            if (u > 0 && (u & (per - 1)) == 0) {
                now = ahead;
                ahead = window(u + per);
            }
            const int first = (u & (per - 1)) << ppt_shift;
            if (!load(I, now, first, 0) || !load(I, now, first, 1)) return false;
        }
        return true;
    }

    // Lets every issued copy land, before the block may exit: others' waits for them may have given up.
    __device__ void drain() {
        volatile int never = 0;
        for (uint32_t k = use > RING ? use - RING : 0; k < use; ++k) mbar_wait(&full[k % RING], (k / RING) & 1, &never);
    }
};

// Row `key` of a packed tile into a tile of 64-dim halves, 128 keys of 128 bytes with the 128-byte swizzle.
__device__ __forceinline__ void unpack_row(const Kv4Row& r, uint8_t* tile, int key) {
    uint8_t* row = tile + key * 128;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        uint32_t v[16];
        kv4_group(r, g, v);
#pragma unroll
        for (int x = 0; x < 4; ++x)
            *reinterpret_cast<uint4*>(row + (g >> 1) * kHalfBytes + ((((g & 1) * 4 + x) ^ (key & 7)) << 4)) =
                make_uint4(v[4 * x], v[4 * x + 1], v[4 * x + 2], v[4 * x + 3]);
    }
}

}  // namespace
}  // namespace ckv
