// Cutting a request's paged cache to a budget, KV head by KV head.  Of a head's L tokens
// the first, the last and, of the others, the heaviest stay, `keep` in all, in their order:
//   kept = sort({first ones} + {last ones} + top_{rest}(w)),  K', V', w'[i] = K, V, w[kept[i]].
//
// Two kernels.  select_kernel: a cluster a (request, head) finds the weight of the last
// token that stays, by histograms over the bits of an order-preserving key (2048 bins a
// level, three levels at most: 11 + 11 + 10 bits, fewer when a bin ends where the budget
// does), and writes the list kept[].  move_kernel: 64 tokens of a head a CTA.  The list
// is increasing, so token i's new place is at or before its old one: rows that a chunk
// overwrites are read by itself and by chunks before it alone.  A CTA therefore loads its
// rows, says so, waits until those chunks have said so too, and stores; chunks are given
// out in order, so that what a CTA waits for has always been started.
#include "cr_cluster.cuh"
#include "cr_internal.h"

namespace cr {
namespace {

constexpr int kMoveRows = 64;       // tokens of a chunk
constexpr int kMoveThreads = 256;

struct Chain {
    int r, head, len, keep;
    const int32_t* table;
};
__device__ __forceinline__ Chain chain_of(const EvictParams& p, int chain, bool tell_errors) {
    Chain c;
    c.r = chain / p.n_kv_heads;
    c.head = chain - c.r * p.n_kv_heads;
    c.table = p.table + c.r * p.blocks;
    const int64_t most = p.blocks << p.block_shift;
    c.len = p.kv_len[c.r];
    c.keep = p.keep[c.r];
    if (tell_errors && (c.len < 0 || c.len > most || c.keep < 0)) report(p.status, CR_DEV_INDEX, 943);
    if (c.len < 0) c.len = 0;
    if (c.len > most) c.len = static_cast<int>(most);
    c.keep = max(0, min(c.keep, p.max_keep));
    return c;
}
// Slot of token j, or -1 for a block outside the cache.
__device__ __forceinline__ int64_t slot_of(const EvictParams& p, const int32_t* table, int j) {
    const int block = table[j >> p.block_shift];
    if (block < 0 || block >= p.n_blocks) {
        report(p.status, CR_DEV_INDEX, 944);
        return -1;
    }
    return (static_cast<int64_t>(block) << p.block_shift) + (j & ((1 << p.block_shift) - 1));
}

template <bool kCached>
__global__ void __launch_bounds__(kSelThreads) select_kernel(const __grid_constant__ EvictParams p) {
    extern __shared__ uint32_t keys[];          // (kCached) the CTA's tokens
    __shared__ __align__(16) SelShared sh;
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t rank = cluster_ctarank(), n_ranks = cluster_nctas();
    const int chain = static_cast<int>(blockIdx.x / n_ranks), tid = static_cast<int>(threadIdx.x);
    const int warp = static_cast<int>(warp_id()), lane = static_cast<int>(lane_id());
    const Chain ch = chain_of(p, chain, rank == 0 && tid == 0);
    const int len = ch.len, fresh = min(len, ch.keep);
    int32_t* kept = p.kept + static_cast<int64_t>(chain) * p.max_keep;
    if (rank == 0) {
        if (tid == 0) {
            if (ch.head == 0) p.new_len[ch.r] = fresh;
            if (chain == 0) *p.ticket = 0;
        }
        for (int i = tid; i < p.chunks; i += kSelThreads) p.flags[static_cast<int64_t>(chain) * p.chunks + i] = 0;
    }
    if (len <= ch.keep) {
        for (int i = static_cast<int>(rank) * kSelThreads + tid; i < len; i += static_cast<int>(n_ranks) * kSelThreads) kept[i] = i;
        return;
    }
    cluster_sync();
    const int last = min(p.last, fresh), first = min(p.first, fresh - last);
    const int mid0 = first, mid1 = len - last;
    // this CTA's tokens, and each warp's of them, lie together: order is that of (rank, warp, step, lane)
    const int per_warp = ((len + static_cast<int>(n_ranks) * kSelWarps - 1) / (static_cast<int>(n_ranks) * kSelWarps) + 31) & ~31;
    const int j0 = (static_cast<int>(rank) * kSelWarps + warp) * per_warp, j1 = min(len, j0 + per_warp);
    const float* weights = p.weights + static_cast<int64_t>(ch.head) * p.num_slots;
    auto weight_key = [&](int j) -> uint32_t {
        const int64_t slot = slot_of(p, ch.table, j);
        const float x = slot < 0 ? key_float(kKeyNegInf) : weights[slot];
        return x != x ? 0xffffffffu : float_key(x);
    };
    if (kCached)
        for (int j = j0 + lane; j < j1; j += 32) keys[warp * per_warp + j - j0] = weight_key(j);
    auto key_at = [&](int j) -> uint32_t { return kCached ? keys[warp * per_warp + j - j0] : weight_key(j); };
    *reinterpret_cast<uint4*>(&sh.hist[0][0][tid * kSelPerThread]) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    // the cut: tokens with a larger key stay, and `ties` of those with this one
    uint32_t lo = 0, hi = 0xffffffffu, cut = 0xffffffffu;
    uint64_t rest = static_cast<uint64_t>(fresh - first - last), ties = 0;
    int shift = 21;
    for (int level = 0; rest != 0; ++level) {
        for (int j = j0 + lane; j < j1; j += 32) {
            if (j < mid0 || j >= mid1) continue;
            const uint32_t key = key_at(j);
            if (key >= lo && key <= hi) hist_add<false>(sh.hist[level & 1], static_cast<int>((hi - key) >> shift), 1);
        }
        cluster_sync();
        uint64_t total;
        hist_find<false>(sh, level & 1, 0, n_ranks, [&](uint64_t) { return rest; }, &total);
        rest -= sh.found[1];
        hi -= static_cast<uint32_t>(sh.found[0]) << shift;
        lo = hi - ((1u << shift) - 1);
        cut = lo;
        ties = rest;
        if (sh.found[2] == rest) ties = ~0ull >> 1;      // the bin whole
        if (sh.found[2] == rest || shift == 0) break;
        shift = shift == 21 ? 10 : 0;
    }
    // places: what stays before this CTA, before this warp, before this token
    uint64_t mine = 0;                       // ties in the upper half
    for (int j = j0 + lane; j < j1; j += 32) {
        const bool mid = j >= mid0 && j < mid1;
        const uint32_t key = mid ? key_at(j) : 0;
        mine += !mid || key > cut ? 1ull : key == cut ? 1ull << 32 : 0ull;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    if (lane == 0) sh.warp2[warp] = mine;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kSelWarps; ++i) {
        if (i < warp) before += sh.warp2[i];
        all += sh.warp2[i];
    }
    tell(sh, 0, all, n_ranks, rank);
    cluster_sync();
    for (uint32_t i = 0; i < rank; ++i) before += sh.xch[0][i];
    uint64_t sure_before = before & 0xffffffffull, ties_before = before >> 32;
    for (int j = j0 + lane; j - lane < j1; j += 32) {
        const bool in = j < j1, mid = j >= mid0 && j < mid1;
        const uint32_t key = in && mid ? key_at(j) : 0;
        const bool sure = in && (!mid || key > cut), tie = in && mid && key == cut;
        const uint32_t s = __ballot_sync(0xffffffffu, sure), e = __ballot_sync(0xffffffffu, tie);
        const uint32_t below = (1u << lane) - 1;
        const uint64_t tie_rank = ties_before + __popc(e & below);
        const uint64_t place = sure_before + __popc(s & below) + (tie_rank < ties ? tie_rank : ties);
        if ((sure || (tie && tie_rank < ties)) && place < static_cast<uint64_t>(fresh)) kept[place] = j;
        sure_before += __popc(s);
        ties_before += __popc(e);
    }
}

// Poll a flag until it is set; false if that takes longer than any wait may.
__device__ __forceinline__ bool wait_flag(const uint32_t* flag, unsigned* status) {
    const uint64_t t0 = globaltimer();
    for (uint32_t i = 1;; ++i) {
        uint32_t v;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(flag) : "memory");
        if (v) return true;
        if ((i & 31u) == 0u) {
            if (*reinterpret_cast<volatile unsigned*>(status) == CR_DEV_TIMEOUT) return false;
            if (globaltimer() - t0 > CR_WAIT_TIMEOUT_NS) {
                report(status, CR_DEV_TIMEOUT, 945);
                return false;
            }
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const __grid_constant__ EvictParams p) {
    constexpr int kPieces = D / 8;                                           // 16-byte pieces of a row
    constexpr int kMine = 2 * kMoveRows * kPieces / kMoveThreads;            // of K and V, a thread
    __shared__ int64_t from[kMoveRows], to[kMoveRows];
    __shared__ uint32_t ticket;
    __shared__ int ok;
    pdl_launch_dependents();
    pdl_wait();
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31;
    if (tid == 0) ticket = atomicAdd(p.ticket, 1u);
    __syncthreads();
    const int chain = static_cast<int>(ticket / static_cast<uint32_t>(p.chunks));
    const int c = static_cast<int>(ticket % static_cast<uint32_t>(p.chunks));
    if (chain >= p.n_req * p.n_kv_heads) return;
    const int r = chain / p.n_kv_heads, head = chain - r * p.n_kv_heads;
    const int32_t* table = p.table + r * p.blocks;
    // (the length that the list was made for, whatever kv_len says by now)
    const int fresh = p.new_len[r], i0 = c * kMoveRows, n = min(kMoveRows, fresh - i0);
    if (n <= 0) return;
    const int64_t most = p.blocks << p.block_shift;
    const int32_t* kept = p.kept + static_cast<int64_t>(chain) * p.max_keep;
    if (kept[i0 + n - 1] == i0 + n - 1) return;          // (increasing, so all of the chunk stay where they are)
    if (tid < kMoveRows) {
        from[tid] = to[tid] = -1;
        if (tid < n) {
            const int j = kept[i0 + tid];
            if (j > i0 + tid && j < most) {
                const int64_t a = slot_of(p, table, j), b = slot_of(p, table, i0 + tid);
                if (a >= 0 && b >= 0) from[tid] = a, to[tid] = b;
            }
        }
    }
    __syncthreads();
    const int64_t width = static_cast<int64_t>(p.n_kv_heads) * D;
    uint4 x[kMine];
    float w = 0.0f;
    float* weights = p.weights + static_cast<int64_t>(head) * p.num_slots;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int q = i * kMoveThreads + tid, row = q / kPieces % kMoveRows;
        const uint16_t* plane = q / kPieces < kMoveRows ? p.k : p.v;
        if (from[row] >= 0) x[i] = *reinterpret_cast<const uint4*>(plane + from[row] * width + head * D + q % kPieces * 8);
    }
    if (tid < kMoveRows && from[tid] >= 0) w = weights[from[tid]];
    __syncthreads();                                      // every load of the chunk is done
    uint32_t* flags = p.flags + static_cast<int64_t>(chain) * p.chunks;
    if (tid == 0) {
        ok = 1;
        __threadfence();
        asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(flags + c), "r"(1u) : "memory");
    }
    __syncthreads();
    if (tid < 32) {
        // the chunks before this one that read rows at or behind its first
        bool fine = true;
        for (int b = c - 1; b >= 0; b -= 32) {
            const int mine = b - lane;
            const bool need = mine >= 0 && kept[mine * kMoveRows + kMoveRows - 1] >= i0;
            if (need) fine = wait_flag(flags + mine, p.status) && fine;
            if (!__any_sync(0xffffffffu, need)) break;
        }
        if (!__all_sync(0xffffffffu, fine) && lane == 0) ok = 0;
    }
    __syncthreads();
    if (!ok) return;
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
        const int q = i * kMoveThreads + tid, row = q / kPieces % kMoveRows;
        uint16_t* plane = q / kPieces < kMoveRows ? p.k : p.v;
        if (to[row] >= 0) *reinterpret_cast<uint4*>(plane + to[row] * width + head * D + q % kPieces * 8) = x[i];
    }
    if (tid < kMoveRows && to[tid] >= 0) weights[to[tid]] = w;
}

constexpr int kCachedKeys = 48 * 1024;      // most tokens of a CTA whose keys it keeps in shared memory

}  // namespace

int64_t evict_chunks(int64_t max_keep) { return (max_keep + kMoveRows - 1) / kMoveRows; }

cr_status launch_evict(const EvictParams& p, int head_dim, cudaStream_t st) {
    const int64_t chains = static_cast<int64_t>(p.n_req) * p.n_kv_heads;
    const int64_t most = p.blocks << p.block_shift;
    int ranks = kMaxCluster;
    while (ranks > 1 && chains * ranks > 2 * num_sms()) ranks /= 2;
    while (ranks < kMaxCluster && most > static_cast<int64_t>(ranks) * (kCachedKeys - 32 * kSelWarps)) ranks *= 2;
    const int64_t per_warp = (most + ranks * kSelWarps - 1) / (ranks * kSelWarps) + 31;
    const bool cached = per_warp * kSelWarps <= kCachedKeys;
    const int smem = cached ? static_cast<int>(per_warp * kSelWarps * 4) : 0;
    static unsigned long long attr_done = 0;
    cr_status s = ensure_smem_attr(select_kernel<true>, kCachedKeys * 4, &attr_done);
    if (s != CR_OK) return s;
    s = launch_cluster(cached ? select_kernel<true> : select_kernel<false>, dim3(static_cast<unsigned>(chains * ranks)),
                       dim3(kSelThreads), ranks, smem, st, p);
    if (s != CR_OK) return s;
    return launch_pdl(head_dim == 128 ? move_kernel<128> : move_kernel<64>, dim3(static_cast<unsigned>(chains * p.chunks)),
                      dim3(kMoveThreads), 0, st, p);
}

}  // namespace cr
