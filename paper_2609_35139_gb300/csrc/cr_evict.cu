// Cutting a request's paged cache to a budget, KV head by KV head.  Of a head's L tokens
// the first, the last and, of the others, the heaviest stay, `keep` in all, in their order:
//   kept = sort({first ones} + {last ones} + top_{rest}(w)),  K', V', w'[i] = K, V, w[kept[i]].
//
// Two kernels.  select_kernel: a CTA a (request, head), or a cluster for long ones, finds the weight
// of the last token that stays, by histograms over the bits of an order-preserving key (2048 bins a
// level, three levels at most: 11 + 11 + 10 bits; fewer when a bin ends where the budget does, or
// holds so few that they are compared each with each), and writes the list kept[].  move_kernel: 64
// tokens of a head a CTA, K and V rows by asynchronous copies through shared memory (rows of 256
// bytes by bulk copies were no faster: too many for the copy engine).  The list is
// increasing, so token i's new place is at or before its old one: rows that a chunk overwrites are
// read by itself and by chunks before it alone.  A CTA therefore loads its rows, says so, waits
// until those chunks have said so too, and stores; chunks are given out in order, so that what a
// CTA waits for has always been started.
//
// 16 requests of 6144 to 10240 tokens, 8 heads of 128, cut to 4096: 122 us, of which the list takes 19
// (one CTA a chain: its passes over 10240 keys in shared memory) and the moves 104, 547 MB at 5.3 TB/s
// (0.78 of the copy rate; every chunk waits for a look-up of list and table, and rows are pieces of 256
// bytes).  One request of 5120 cut to 2048: 21 us, list and moves in turn.
#include "cr_cluster.cuh"
#include "cr_internal.h"

namespace cr {
namespace {

constexpr int kMoveRows = 64;       // tokens of a chunk
constexpr int kMoveThreads = 4 * kMoveRows;
constexpr int kPairs = 256;         // so many tokens of a bin are compared each with each (611 tokens: 10.6 us for 11.8)

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
    __shared__ uint32_t pair[kPairs];
    __shared__ int pairs;
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t rank = cluster_ctarank(), n_ranks = cluster_nctas();
    const int chain = static_cast<int>(blockIdx.x / n_ranks), tid = static_cast<int>(threadIdx.x);
    const int warp = static_cast<int>(warp_id()), lane = static_cast<int>(lane_id());
    Chain ch = chain_of(p, chain, rank == 0 && tid == 0);
    // (one thread's reading, and then the first CTA's, for all: what is written meanwhile divides no one)
    if (n_ranks > 1) cluster_sync();
    if (rank == 0 && tid == 0)
        for (uint32_t i = 0; i < n_ranks; ++i)
            st_cluster_u64(mapa_shared(smem_u32(&sh.xch[1][0]), i), static_cast<uint64_t>(ch.len) << 32 | static_cast<uint32_t>(ch.keep));
    if (n_ranks > 1) cluster_sync();
    else __syncthreads();
    ch.len = static_cast<int>(sh.xch[1][0] >> 32);
    ch.keep = static_cast<int>(sh.xch[1][0]);
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
    if (tid == 0) pairs = 0;
    if (kCached) {
        // blocks, then weights, of sixteen steps on their way at once
        constexpr int kDeep = 16;
        for (int j = j0 + lane; j < j1; j += 32 * kDeep) {
            int block[kDeep];
            float x[kDeep];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) block[k] = j + 32 * k < j1 ? ch.table[(j + 32 * k) >> p.block_shift] : 0;
#pragma unroll
            for (int k = 0; k < kDeep; ++k) {
                const bool there = block[k] >= 0 && block[k] < p.n_blocks;
                if (!there) report(p.status, CR_DEV_INDEX, 944);
                x[k] = there && j + 32 * k < j1
                           ? weights[(static_cast<int64_t>(block[k]) << p.block_shift) + ((j + 32 * k) & ((1 << p.block_shift) - 1))]
                           : key_float(kKeyNegInf);
            }
#pragma unroll
            for (int k = 0; k < kDeep; ++k)
                if (j + 32 * k < j1) keys[warp * per_warp + j + 32 * k - j0] = x[k] != x[k] ? 0xffffffffu : float_key(x[k]);
        }
    }
    auto key_at = [&](int j) -> uint32_t { return kCached ? keys[warp * per_warp + j - j0] : weight_key(j); };
    // This warp's tokens, four steps of 32 at a time: f(first of this lane's four, keys, which are in the middle).
    constexpr int kSteps = 4;
    auto steps = [&](auto f) {
#pragma unroll 1
        for (int j = j0 + lane; j - lane < j1; j += 32 * kSteps) {
            uint32_t key[kSteps];
            bool mid[kSteps];
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int i = j + 32 * k;
                mid[k] = i < j1 && i >= mid0 && i < mid1;
                key[k] = mid[k] ? key_at(i) : 0u;
            }
            f(j, key, mid);
        }
    };
    *reinterpret_cast<uint4*>(&sh.hist[0][0][tid * kSelPerThread]) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    // the cut: tokens with a larger key stay, and `ties` of those with this one
    uint32_t lo = 0, hi = 0xffffffffu, cut = 0xffffffffu;
    uint64_t rest = static_cast<uint64_t>(fresh - first - last), ties = 0;
    int shift = 21;
    for (int level = 0; rest != 0; ++level) {
        uint32_t* h = sh.hist[level & 1][0];
        steps([&](int, const uint32_t (&key)[kSteps], const bool (&mid)[kSteps]) {
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
                if (mid[k] && key[k] >= lo && key[k] <= hi) atomicAdd(h + ((hi - key[k]) >> shift), 1u);
        });
        if (n_ranks == 1) __syncthreads();
        else cluster_sync();
        uint64_t total;
        hist_find<false>(sh, level & 1, 0, n_ranks, [&](uint64_t) { return rest; }, &total);
        rest -= sh.found[1];
        hi -= static_cast<uint32_t>(sh.found[0]) << shift;
        lo = hi - ((1u << shift) - 1);
        cut = lo;
        ties = rest;
        if (sh.found[2] == rest) ties = ~0ull >> 1;      // the bin whole
        if (sh.found[2] == rest || shift == 0) break;
        if (n_ranks == 1 && sh.found[2] <= kPairs) {
            steps([&](int, const uint32_t (&key)[kSteps], const bool (&mid)[kSteps]) {
#pragma unroll
                for (int k = 0; k < kSteps; ++k)
                    if (mid[k] && key[k] >= lo && key[k] <= hi) pair[atomicAdd(&pairs, 1)] = key[k];
            });
            __syncthreads();
            const int m = pairs;
            // q threads a token, neighbours in a warp
            const int q = m <= 64 ? 8 : m <= 128 ? 4 : 2, e = tid / q;
            const uint32_t key = e < m ? pair[e] : 0u;
            uint32_t more = 0, same = 0;
#pragma unroll 8
            for (int i = tid % q; i < m; i += q) {
                const uint32_t other = pair[i];
                more += other > key ? 1u : 0u;
                same += other == key ? 1u : 0u;
            }
            for (int o = 1; o < q; o <<= 1) {
                more += __shfl_xor_sync(0xffffffffu, more, o);
                same += __shfl_xor_sync(0xffffffffu, same, o);
            }
            if (e < m && more < rest && rest <= static_cast<uint64_t>(more) + same) {
                sh.found[0] = key;
                sh.found[1] = more;
            }
            __syncthreads();
            cut = static_cast<uint32_t>(sh.found[0]);
            ties = rest - sh.found[1];
            break;
        }
        shift = shift == 21 ? 10 : 0;
    }
    // places: what stays before this CTA, before this warp, before this token
    uint32_t sure = 0, tied = 0;
    steps([&](int j, const uint32_t (&key)[kSteps], const bool (&mid)[kSteps]) {
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            sure += j + 32 * k < j1 && (!mid[k] || key[k] > cut) ? 1u : 0u;
            tied += mid[k] && key[k] == cut ? 1u : 0u;
        }
    });
    const uint64_t mine = static_cast<uint64_t>(__reduce_add_sync(0xffffffffu, tied)) << 32 | __reduce_add_sync(0xffffffffu, sure);
    if (lane == 0) sh.warp2[warp] = mine;
    __syncthreads();
    uint64_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kSelWarps; ++i) {
        if (i < warp) before += sh.warp2[i];
        all += sh.warp2[i];
    }
    if (n_ranks > 1) {
        tell(sh, 0, all, n_ranks, rank);
        cluster_sync();
        for (uint32_t i = 0; i < rank; ++i) before += sh.xch[0][i];
    }
    const uint32_t most_ties = static_cast<uint32_t>(min(ties, static_cast<uint64_t>(INT32_MAX)));
    uint32_t sure_before = static_cast<uint32_t>(before), ties_before = static_cast<uint32_t>(before >> 32);
    steps([&](int j, const uint32_t (&key)[kSteps], const bool (&mid)[kSteps]) {
        uint32_t s[kSteps], e[kSteps];
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            s[k] = __ballot_sync(0xffffffffu, j + 32 * k < j1 && (!mid[k] || key[k] > cut));
            e[k] = __ballot_sync(0xffffffffu, mid[k] && key[k] == cut);
        }
        const uint32_t below = (1u << lane) - 1;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const uint32_t tie_rank = ties_before + __popc(e[k] & below);
            const uint32_t place = sure_before + __popc(s[k] & below) + min(tie_rank, most_ties);
            const bool stays = (s[k] >> lane & 1u) || ((e[k] >> lane & 1u) && tie_rank < most_ties);
            if (stays && place < static_cast<uint32_t>(fresh)) kept[place] = j + 32 * k;
            sure_before += __popc(s[k]);
            ties_before += __popc(e[k]);
        }
    });
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

// A CTA looks a chunk up and starts its loads while those of the chunk before are on their way,
// and then finishes that one, so that its chain of waits (ticket, list, block, rows) is hidden.
template <int D>
__global__ void __launch_bounds__(kMoveThreads) move_kernel(const __grid_constant__ EvictParams p) {
    constexpr int kPieces = D / 8;                             // 16-byte pieces of a row
    constexpr int kMine = 2 * kMoveRows * kPieces / kMoveThreads;
    extern __shared__ __align__(128) uint8_t rows[];           // [2][rows of K, then of V][2 D]
    __shared__ int64_t from[2][kMoveRows], to[2][kMoveRows];   // slots, or -1
    __shared__ uint32_t tickets[2];
    __shared__ int ok;
    const int tid = static_cast<int>(threadIdx.x);
    pdl_launch_dependents();
    pdl_wait();
    const int64_t most = p.blocks << p.block_shift, width = static_cast<int64_t>(p.n_kv_heads) * D;
    const uint32_t total = static_cast<uint32_t>(p.n_req) * p.chunks * p.n_kv_heads;
    struct Chunk {
        bool there, live;       // is one; has rows to move
        int chain, head, c;
        int need;               // first chunk that may read this one's places
        float w;                // the weight of this thread's row
    };
    // Look up a chunk and start its loads.
    auto start = [&](uint32_t ticket, int buf) {
        Chunk x;
        x.there = x.live = false;
        x.w = 0.0f;
        if (ticket < total) {
            // All requests' first chunks, then their second ones, and so on: a chunk waits for the one
            // before it, which has then long been started.  (Request by request: 197 us for 138.)  The
            // heads of a chunk lie next to one another: their rows are neighbours in memory.
            const int line = static_cast<int>(ticket) / p.n_kv_heads;
            x.head = static_cast<int>(ticket) - line * p.n_kv_heads;
            x.c = line / p.n_req;
            const int r = line - x.c * p.n_req;
            x.chain = r * p.n_kv_heads + x.head;
            const int32_t* table = p.table + r * p.blocks;
            const int32_t* kept = p.kept + static_cast<int64_t>(x.chain) * p.max_keep;
            // (the length that the list was made for, whatever kv_len says by now)
            const int fresh = p.new_len[r], len = p.kv_len[r], i0 = x.c * kMoveRows, n = min(kMoveRows, fresh - i0);
            if (n > 0) {
                x.there = true;
                // token i comes from i + (len - fresh) at most
                x.need = max(0, x.c - 1 - max(0, len - fresh) / kMoveRows);
                x.live = kept[i0 + n - 1] != i0 + n - 1;       // (increasing: where the last stays in its place, all do)
                if (tid < kMoveRows) {
                    int64_t a = -1, b = -1;
                    if (tid < n) {
                        const int i = i0 + tid, j = kept[i], to_block = table[i >> p.block_shift];
                        if (j > i && j < most) {
                            a = slot_of(p, table, j);
                            if (to_block >= 0 && to_block < p.n_blocks)
                                b = (static_cast<int64_t>(to_block) << p.block_shift) + (i & ((1 << p.block_shift) - 1));
                            else report(p.status, CR_DEV_INDEX, 944);
                            if (a < 0 || b < 0) a = b = -1;
                        }
                    }
                    from[buf][tid] = a;
                    to[buf][tid] = b;
                    if (a >= 0) x.w = p.weights[static_cast<int64_t>(x.head) * p.num_slots + a];
                }
            }
        }
        __syncthreads();
        if (x.live) {
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int q = k * kMoveThreads + tid, row = q / kPieces % kMoveRows;
                const uint16_t* plane = q < kMoveRows * kPieces ? p.k : p.v;
                const int64_t a = from[buf][row];
                if (a >= 0)
                    cp_async16(rows + buf * (2 * kMoveRows * 2 * D) + q * 16, plane + a * width + x.head * D + q % kPieces * 8, 16);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        return x;
    };
    // The chunk before the one started last.  False: a wait gave up.
    auto finish = [&](const Chunk& x, int buf) -> bool {
        asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncthreads();                   // every load of the chunk is done
        if (!x.there) return true;
        uint32_t* flags = p.flags + static_cast<int64_t>(x.chain) * p.chunks;
        if (tid == 0) {
            ok = 1;
            asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(flags + x.c), "r"(1u) : "memory");
        }
        if (!x.live) return true;
        __syncthreads();
        if (tid < 32) {
            bool fine = true;
            for (int b = x.need + tid; b < x.c; b += 32) fine = wait_flag(flags + b, p.status) && fine;
            if (!fine) ok = 0;
        }
        __syncthreads();
        if (!ok) return false;
#pragma unroll
        for (int k = 0; k < kMine; ++k) {
            const int q = k * kMoveThreads + tid, row = q / kPieces % kMoveRows;
            uint16_t* plane = q < kMoveRows * kPieces ? p.k : p.v;
            const int64_t b = to[buf][row];
            if (b >= 0)
                *reinterpret_cast<uint4*>(plane + b * width + x.head * D + q % kPieces * 8) =
                    *reinterpret_cast<const uint4*>(rows + buf * (2 * kMoveRows * 2 * D) + q * 16);
        }
        if (tid < kMoveRows && to[buf][tid] >= 0) p.weights[static_cast<int64_t>(x.head) * p.num_slots + to[buf][tid]] = x.w;
        return true;
    };
    // a chunk's ticket is drawn while the one before it is started (none, where there is a CTA a chunk)
    const bool alone = gridDim.x >= total;
    if (tid == 0) {
        tickets[0] = atomicAdd(p.ticket, 1u);
        tickets[1] = alone ? total : atomicAdd(p.ticket, 1u);
    }
    __syncthreads();
    uint32_t ticket = tickets[0];
    Chunk now = start(ticket, 0);
    for (int buf = 0; ticket < total; buf ^= 1) {
        ticket = tickets[buf ^ 1];
        uint32_t drawn = total;
        if (tid == 0 && !alone) drawn = atomicAdd(p.ticket, 1u);
        const Chunk next = start(ticket, buf ^ 1);
        if (!finish(now, buf)) break;
        if (tid == 0) tickets[buf] = drawn;
        __syncthreads();
        now = next;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Tokens that a CTA selects among faster than a cluster of more would (a request of 5120 cut to 2048:
// 20.9 us, with clusters of four 26.6; 16 of up to 10240: 122, with clusters of two 132).
constexpr int kAlone = 16 * 1024;
constexpr int kCachedKeys = 48 * 1024;      // most tokens of a CTA whose keys it keeps in shared memory

}  // namespace

int64_t evict_chunks(int64_t max_keep) { return (max_keep + kMoveRows - 1) / kMoveRows; }

cr_status launch_evict(const EvictParams& p, int head_dim, cudaStream_t st) {
    const int64_t chains = static_cast<int64_t>(p.n_req) * p.n_kv_heads;
    const int64_t most = p.blocks << p.block_shift;
    int ranks = kMaxCluster;
    while (ranks > 1 && (chains * ranks > 2 * num_sms() || most <= kAlone * (ranks / 2))) ranks /= 2;
    while (ranks < kMaxCluster && most > static_cast<int64_t>(ranks) * (kCachedKeys - 32 * kSelWarps)) ranks *= 2;
    const int64_t per_warp = (most + ranks * kSelWarps - 1) / (ranks * kSelWarps) + 31;
    const bool cached = per_warp * kSelWarps <= kCachedKeys;
    const int smem = cached ? static_cast<int>(per_warp * kSelWarps * 4) : 0;
    static unsigned long long attr_done = 0;
    cr_status s = ensure_smem_attr(select_kernel<true>, kCachedKeys * 4, &attr_done);
    if (s != CR_OK) return s;
    const auto select = cached ? select_kernel<true> : select_kernel<false>;
    const dim3 grid(static_cast<unsigned>(chains * ranks));
    s = ranks == 1 ? launch_pdl(select, grid, dim3(kSelThreads), smem, st, p)
                   : launch_cluster(select, grid, dim3(kSelThreads), ranks, smem, st, p);
    if (s != CR_OK) return s;
    const int move_smem = 4 * kMoveRows * 2 * head_dim;
    static unsigned long long move_done = 0;
    if ((s = ensure_smem_attr(move_kernel<128>, 4 * kMoveRows * 256, &move_done)) != CR_OK) return s;
    // (what fits: 64 KB of shared memory a CTA for heads of 128; two an SM: 146 us for 122)
    const int64_t ctas = static_cast<int64_t>(num_sms()) * (head_dim == 128 ? 3 : 6), chunks = chains * p.chunks;
    return launch_pdl(head_dim == 128 ? move_kernel<128> : move_kernel<64>, dim3(static_cast<unsigned>(chunks < ctas ? chunks : ctas)),
                      dim3(kMoveThreads), move_smem, st, p);
}

}  // namespace cr
