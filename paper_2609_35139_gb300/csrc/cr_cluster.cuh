// What the selecting kernels (sampling, eviction) share: values exchanged between the
// CTAs of a cluster, sums over a CTA, and the search for the place in descending order
// where a running sum passes a target.  A CTA's shared memory is gone when it returns: it does so only
// behind a cluster_sync that follows the last access of the others to it.
#pragma once
#include "cr_ptx.cuh"

namespace cr {

constexpr int kSelThreads = 512;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelBins = 2048;
constexpr int kSelPerThread = kSelBins / kSelThreads;
constexpr int kMaxCluster = 8;

__device__ __forceinline__ uint32_t cluster_nctas() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void st_cluster_u64(uint32_t addr, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_f32(uint32_t addr, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ uint4 ld_cluster_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(addr)
                 : "memory");
    return v;
}

// Order-preserving map of fp32 to unsigned (-0 as +0; NaN is for the caller).
__device__ __forceinline__ uint32_t float_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_float(uint32_t k) {
    return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k);
}
constexpr uint32_t kKeyNegInf = 0x007fffffu, kKeyPosInf = 0xff800000u;

// Shared memory of one search: histograms of 64-bit sums in two halves, two of them in
// turn, and what a CTA's threads tell one another.
struct SelShared {
    uint32_t hist[2][2][kSelBins];
    uint64_t xch[6][kMaxCluster];       // values of every CTA of the cluster
    uint64_t warp[kSelWarps];
    uint64_t warp2[kSelWarps];
    uint64_t found[3];                  // bin, sum before it, sum of it
};

// Sum of v over the CTA's threads before this one, and of all (by all threads; the
// caller keeps uses of `warp` apart by barriers).
__device__ __forceinline__ uint64_t block_scan(uint64_t v, uint64_t* warp, uint64_t* total) {
    const uint32_t lane = lane_id(), w = warp_id();
    uint64_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= static_cast<uint32_t>(o)) x += y;
    }
    if (lane == 31) warp[w] = x;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kSelWarps; ++i) {
        const uint64_t y = warp[i];
        if (i < static_cast<int>(w)) before += y;
        all += y;
    }
    *total = all;
    return before + x - v;
}

// Tell v to slot `which` of every CTA of the cluster (by thread 0 .. n - 1, visible after
// the next cluster_sync).
__device__ __forceinline__ void tell(SelShared& sh, int which, uint64_t v, uint32_t n, uint32_t rank) {
    if (threadIdx.x < n) st_cluster_u64(mapa_shared(smem_u32(&sh.xch[which][rank]), threadIdx.x), v);
}

// Add v to a bin of the CTA's histogram.
template <bool kWide>
__device__ __forceinline__ void hist_add(uint32_t (*h)[kSelBins], int bin, uint64_t v) {
    if (!kWide) {
        atomicAdd(&h[0][bin], static_cast<uint32_t>(v));
        return;
    }
    const uint32_t lo = static_cast<uint32_t>(v);
    const uint32_t was = atomicAdd(&h[0][bin], lo);
    const uint32_t up = static_cast<uint32_t>(v >> 32) + (was + lo < was ? 1u : 0u);
    if (up) atomicAdd(&h[1][bin], up);
}

// After a cluster_sync (a barrier, for one CTA alone) behind hist_add: the sums of this thread's
// bins (the kSelPerThread from threadIdx.x * kSelPerThread on) over CTAs [r0, r0 + n) of the
// cluster.  Clears the other histogram.
template <bool kWide>
__device__ __forceinline__ void hist_merge(SelShared& sh, int turn, uint32_t r0, uint32_t n, uint64_t (&v)[kSelPerThread]) {
    const int b0 = static_cast<int>(threadIdx.x) * kSelPerThread;
#pragma unroll
    for (int i = 0; i < kSelPerThread; ++i) v[i] = 0;
    auto add = [&](uint4 x, int by) {
        v[0] += static_cast<uint64_t>(x.x) << by, v[1] += static_cast<uint64_t>(x.y) << by;
        v[2] += static_cast<uint64_t>(x.z) << by, v[3] += static_cast<uint64_t>(x.w) << by;
    };
#pragma unroll
    for (int half = 0; half < (kWide ? 2 : 1); ++half) {
        if (n == 1) {
            add(*reinterpret_cast<const uint4*>(&sh.hist[turn][half][b0]), 32 * half);
            continue;
        }
        const uint32_t mine = smem_u32(&sh.hist[turn][half][b0]);
        uint4 x[kMaxCluster];             // all on their way at once
#pragma unroll
        for (uint32_t r = 0; r < kMaxCluster; ++r) x[r] = r < n ? ld_cluster_v4(mapa_shared(mine, r0 + r)) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (uint32_t r = 0; r < kMaxCluster; ++r) add(x[r], 32 * half);
    }
    *reinterpret_cast<uint4*>(&sh.hist[turn ^ 1][0][b0]) = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(&sh.hist[turn ^ 1][1][b0]) = make_uint4(0, 0, 0, 0);
}
static_assert(kSelPerThread == 4, "a thread's bins are one 16-byte load");

// The first bin whose running sum (bin 0 first) reaches the target, told to all threads
// through sh.found: bin, sum before it, its own; false if the whole does not reach it.
template <typename F>
__device__ __forceinline__ bool bins_find(SelShared& sh, const uint64_t (&v)[kSelPerThread], F target_of, uint64_t* total) {
    uint64_t before = block_scan(v[0] + v[1] + v[2] + v[3], sh.warp, total);
    const uint64_t target = target_of(*total);
#pragma unroll
    for (int i = 0; i < kSelPerThread; ++i) {
        if (before < target && target <= before + v[i]) {
            sh.found[0] = threadIdx.x * kSelPerThread + i;
            sh.found[1] = before;
            sh.found[2] = v[i];
        }
        before += v[i];
    }
    __syncthreads();
    return target <= *total;
}
template <bool kWide, typename F>
__device__ __forceinline__ bool hist_find(SelShared& sh, int turn, uint32_t r0, uint32_t n, F target_of, uint64_t* total) {
    uint64_t v[kSelPerThread];
    hist_merge<kWide>(sh, turn, r0, n, v);
    return bins_find(sh, v, target_of, total);
}

}  // namespace cr
