// Attention weight gathered by the tokens of a paged cache:
//   w[h][slot(j)] (+)= sum over the rows i that see j, and the query heads of KV head h,
//                      exp(scale q_i . k_j - lse_i),
// the sum over a call's rows of the weights that attention gave token j (lse_i is the
// row's log-sum-exp there).  Segments, rows and what they see are those of the attention
// calls: a request's rows over its own tokens, causal among the new ones, and a group's
// rows over its prefix.  As there, segments of few rows (PAGED_ROWS) and of many
// (PAGED_TILES) go different ways, each kind's work laid out as one line on the device and
// cut evenly, whatever the lengths are:
//   few    bound by HBM (each byte of K is used for 2 x rows flops): K from memory straight
//          into the registers of m16n8k16 MMAs, 16 keys a warp at a time;
//   many   bound by the tensor cores and the exponentials: tcgen05 with the keys as M, so that
//          a thread holds one key's scores of a tile of rows and its sum takes no exchange.
// In units of log2 a weight is 2^(s x - c), x = q . k, s = scale log2(e), c = lse s / scale:
// the rounding of s then scales score and lse alike, and what counts is their difference.
#include <cuda_bf16.h>

#include "cr_internal.h"
#include "cr_ptx.cuh"

namespace cr {
namespace {

constexpr int kMaxSegments = 2 * kMaxReq;
constexpr int kAll = INT32_MAX;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

// ------------------------------------------------------------------ segments
struct Segment {
    int t0, nt;            // query tokens
    int kind;
    int len;               // keys
    int past;              // row token i sees keys j <= past + i (kAll: every key)
    const int32_t* table;
    bool own;
};
// A length that is changed during a call leaves its results undefined, but every loop and
// index below stays bounded whatever it becomes, and a warp takes one lane's reading (kWarp).
template <bool kWarp>
__device__ __forceinline__ Segment segment(const WeighParams& p, int s) {
    Segment g;
    g.own = s >= p.n_groups;
    const int r = s - p.n_groups;
    const int4 d = p.seg[s];
    const int64_t blocks = g.own ? p.own_blocks : p.prefix_blocks;
    const int64_t most = blocks << p.block_shift;
    int len = g.own ? p.own_len[r] : p.prefix_len[s];
    if (kWarp) len = __shfl_sync(0xffffffffu, len, 0);
    if (len < 0 || len > most) {
        report(p.status, CR_DEV_INDEX, 941);
        len = len < 0 ? 0 : static_cast<int>(most);
    }
    g.t0 = d.x;
    g.nt = d.y;
    g.kind = d.w;
    g.len = len;
    g.past = g.own ? len - d.y : kAll;
    g.table = g.own ? p.own_table + r * p.own_blocks : p.prefix_table + s * p.prefix_blocks;
    return g;
}
// Block of a key, or -1 for one outside the cache.
__device__ __forceinline__ int block_of(const WeighParams& p, const int32_t* table, int key) {
    const int block = table[key >> p.block_shift];
    if (block >= 0 && block < p.n_blocks) return block;
    report(p.status, CR_DEV_INDEX, 942);
    return -1;
}
__device__ __forceinline__ int64_t slot_in(const WeighParams& p, int block, int key) {
    return (static_cast<int64_t>(block) << p.block_shift) + (key & ((1 << p.block_shift) - 1));
}
// Give a key's sum to its slot: a new token's is written, others' are added to.
__device__ __forceinline__ void give(const WeighParams& p, int head, int64_t slot, bool fresh, float sum) {
    float* w = p.weights + static_cast<int64_t>(head) * p.num_slots + slot;
    if (fresh) *w = sum;
    else atomicAdd(w, sum);
}
__device__ __forceinline__ float log2_lse(const WeighParams& p, float lse) { return fmaf(lse, p.lse_hi, lse * p.lse_lo); }

// The line of one kind of work, by all threads of the CTA: cum[s] = work of the segments
// before s, cum[n] = all of it.  cost(segment) is a segment's.
template <int kThreads, typename F>
__device__ __forceinline__ void make_line(const WeighParams& p, int64_t* cum, int64_t* warp_sum, F cost) {
    const int n = p.n_groups + p.n_req, tid = static_cast<int>(threadIdx.x);
    const uint32_t lane = lane_id(), warp = warp_id();
    if (n == 1) {
        if (tid == 0) {
            cum[0] = 0;
            cum[1] = cost(segment<false>(p, 0));
        }
        __syncthreads();
        return;
    }
    constexpr int kEach = (kMaxSegments + kThreads) / kThreads;          // (the line's end has a place too)
    int64_t c[kEach], mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int s = tid * kEach + i;
        c[i] = s < n ? cost(segment<false>(p, s)) : 0;
        mine += c[i];
    }
    int64_t x = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= static_cast<uint32_t>(o)) x += y;
    }
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    x -= mine;
    for (uint32_t w = 0; w < warp; ++w) x += warp_sum[w];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int s = tid * kEach + i;
        if (s <= n) cum[s] = x;
        x += c[i];
    }
    __syncthreads();
}
// The segment that holds place `at` of the line.
__device__ __forceinline__ int find_segment(const int64_t* cum, int n, int64_t at) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cum[mid] <= at) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// ------------------------------------------------------------------ few rows
constexpr int kFewThreads = 128;
constexpr int kFewWarps = kFewThreads / 32;
constexpr int kFewCtas = 3;         // an SM
constexpr int kChunk = 16;          // keys of a chunk
constexpr int kFewRows = 16;        // most rows (as the plan's)

__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, const uint32_t* b) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
__device__ __forceinline__ uint4 load_once(const uint16_t* src) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(src));
    return v;
}

// A warp takes its part of the line of (segment, KV head, 16 keys).  Bound by HBM: 16 requests of
// 6144 to 10240 tokens, 8 KV heads of 128, take 48 us for 273 MB (0.84 of the copy rate); one
// request of 5120 takes 5.0 us: launch, schedule and first keys.  Three CTAs an SM, so that 12 chunks
// of 4 KB an SM and their successors are on their way (two: 62 and 5.9 us, four: 48 and 5.5).
// The order of the products' k is free as long as both operands share it, so a thread loads whole
// 16-byte pieces and feeds each to two MMAs.  While a chunk is worked on, the next one's K and the
// blocks of the one after that are on their way.
template <int D>
__global__ void __launch_bounds__(kFewThreads, kFewCtas) weigh_few_kernel(const __grid_constant__ WeighParams p) {
    constexpr int kPieces = D / 32;            // 16-byte pieces of a row in each of a quad's threads
    __shared__ int64_t cum[kMaxSegments + 1];
    __shared__ int64_t warp_sum[kFewWarps];
    pdl_launch_dependents();
    pdl_wait();
    make_line<kFewThreads>(p, cum, warp_sum, [&](const Segment& g) -> int64_t {
        return g.kind == PAGED_ROWS ? static_cast<int64_t>((g.len + kChunk - 1) / kChunk) * p.n_kv_heads : 0;
    });
    const int n_seg = p.n_groups + p.n_req;
    const int64_t total = cum[n_seg], workers = static_cast<int64_t>(gridDim.x) * kFewWarps;
    const int64_t per = (total + workers - 1) / workers;
    // (the CTAs' first warps come first, so that a short line spreads over all SMs)
    int64_t at = (static_cast<int64_t>(warp_id()) * gridDim.x + blockIdx.x) * per;
    const int64_t end = min(total, at + per);
    if (at >= end) return;
    const uint32_t lane = lane_id();
    const int g = static_cast<int>(lane >> 2), t = static_cast<int>(lane & 3u);
    const int64_t width = static_cast<int64_t>(p.n_kv_heads) * D;

    int seg = find_segment(cum, n_seg, at);
    Segment sg = segment<true>(p, seg);
    int chunks = max(1, (sg.len + kChunk - 1) / kChunk);
    int head = static_cast<int>((at - cum[seg]) / chunks), chunk = static_cast<int>((at - cum[seg]) % chunks);
    head = min(head, p.n_kv_heads - 1);

    struct Place {              // a chunk on its way
        int seg, head, key0;
        int block[2];           // of this thread's keys, -1 past the end or outside the cache
    };
    // the next chunk of the line and its blocks
    auto next = [&]() {
        Place x;
        x.seg = seg;
        x.head = head;
        x.key0 = chunk * kChunk;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int key = x.key0 + g + 8 * i;
            x.block[i] = key < sg.len ? block_of(p, sg.table, key) : -1;
        }
        if (++chunk >= chunks) {
            chunk = 0;
            if (++head >= p.n_kv_heads) {
                head = 0;
                do ++seg;
                while (seg < n_seg - 1 && cum[seg + 1] == cum[seg]);
                if (seg < n_seg) {
                    sg = segment<true>(p, seg);
                    chunks = max(1, (sg.len + kChunk - 1) / kChunk);
                } else {
                    seg = n_seg - 1;
                }
            }
        }
        return x;
    };
    uint32_t k[2][kPieces][4];
    auto load = [&](const Place& x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint16_t* src = p.k + slot_in(p, max(0, x.block[i]), x.key0 + g + 8 * i) * width + x.head * D + t * 8;
#pragma unroll
            for (int c = 0; c < kPieces; ++c) {
                const uint4 v = x.block[i] < 0 ? make_uint4(0, 0, 0, 0) : load_once(src + c * 32);
                k[i][c][0] = v.x, k[i][c][1] = v.y, k[i][c][2] = v.z, k[i][c][3] = v.w;
            }
        }
    };
    // the rows of a (segment, head): Q in MMA layout, c of rows 2 t, 2 t + 1 of each eight and
    // the last key that they see
    uint32_t q[2][kPieces][4];
    float c_lse[2][2];
    int see[2][2];
    int rows = 0, past = 0;
    auto enter = [&](const Place& x) {
        const Segment s = segment<true>(p, x.seg);
        rows = min(kFewRows, s.nt * p.group);
        past = s.past;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = min(8 * h + g, rows - 1), tok = row / p.group;
            const uint16_t* src = p.q + static_cast<int64_t>(s.t0 + tok) * p.ldq +
                                  static_cast<int64_t>(x.head * p.group + row - tok * p.group) * D + t * 8;
#pragma unroll
            for (int c = 0; c < kPieces; ++c) {
                const uint4 v = *reinterpret_cast<const uint4*>(src + c * 32);
                q[h][c][0] = v.x, q[h][c][1] = v.y, q[h][c][2] = v.z, q[h][c][3] = v.w;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int n = 8 * h + 2 * t + e, nt = n / p.group;
                see[h][e] = -1;
                c_lse[h][e] = 0.0f;
                if (n < rows) {
                    const float lse = p.lse[static_cast<int64_t>(s.t0 + nt) * p.n_q_heads + x.head * p.group + n - nt * p.group];
                    c_lse[h][e] = -log2_lse(p, lse);
                    if (lse != neg_inf()) see[h][e] = s.own ? min(s.len - 1, s.past + nt) : s.len - 1;
                }
            }
        }
    };
    Place now = next();
    enter(now);
    load(now);
    Place then = now;
    const int n = static_cast<int>(min(end - at, static_cast<int64_t>(INT32_MAX)));
    if (n > 1) then = next();
    for (int step = 0; step < n; ++step) {
        // An MMA cuts what it adds off below its accumulator's last bit, 1e-7 to 2e-7 of a score by the
        // eighth: each starts from zero, and their results are added with rounding.
        float c[2][4] = {};
        auto add = [&](float (&sum)[4], const uint32_t* a, const uint32_t* b) {
            float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            mma16816(x, a, b);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += x[e];
        };
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint32_t a0[4] = {k[0][i][0], k[1][i][0], k[0][i][1], k[1][i][1]};
            const uint32_t a1[4] = {k[0][i][2], k[1][i][2], k[0][i][3], k[1][i][3]};
            add(c[0], a0, &q[0][i][0]);
            add(c[0], a1, &q[0][i][2]);
            if (rows > 8) {
                add(c[1], a0, &q[1][i][0]);
                add(c[1], a1, &q[1][i][2]);
            }
        }
        const Place done = now;
        const float cl[2][2] = {{c_lse[0][0], c_lse[0][1]}, {c_lse[1][0], c_lse[1][1]}};
        const int sl[2][2] = {{see[0][0], see[0][1]}, {see[1][0], see[1][1]}};
        const int two = rows > 8, past_done = past;
        if (step + 1 < n) {
            now = then;
            load(now);
            if (step + 2 < n) then = next();
            if (now.seg != done.seg || now.head != done.head) enter(now);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int key = done.key0 + g + 8 * i;
            float sum = 0.0f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (h && !two) break;
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (key <= sl[h][e]) sum += ex2(fmaf(c[h][2 * i + e], p.scale_log2, cl[h][e]));
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            if (t == 0 && done.block[i] >= 0) give(p, done.head, slot_in(p, done.block[i], key), key >= past_done, sum);
        }
    }
}

// ------------------------------------------------------------------ many rows
// One CTA per SM takes its part of the line.  A unit is a segment's KV head and 256 of its
// keys, which stay in shared memory while the rows that see them pass in tiles of up to 128
// (whole tokens: a token's rows are the heads of the KV head's group), a step each:
//   warp 0       walks the line unit by unit, for all others, and brings the units' K by TMA
//   warp 1       MMA issue: S_h = K_h Q^T for the unit's two halves of 128 keys
//   warps 2, 3   tiles of Q by TMA and their rows' c, asked for two tiles ahead, in turn: one warp
//                takes longer over a tile than its MMAs do
//   warps 4..19  sums, one key a thread: two warpgroups a half, which take turns at the tiles and
//                add up at the unit's end
// 2048 new tokens over 8192, 32 heads on 8 of 128: 131 us (156 GFLOP at 0.63 of the tensor peak; the
// prompt over 8192 new ones 608).  What bounds it is both sides of the hand-over of S: with the sums
// left out it takes 118 us, with an eighth of the MMAs as well 75.  An MMA of 128 keys and 128 rows
// with both operands in shared memory takes more than its 64 clocks beside Q's arrival; K in TMEM in
// its place leaves three buffers of S for four, and took 141 (184 before the warpgroups took turns).
// Eight summing warps with 128 scores each in registers: 155.  Turns of 16
// rows instead of a tile: 132.
// A unit cut between CTAs leaves its parts in the workspace, joined by a second kernel in the
// order of the line.
constexpr int kKeys = 256;
constexpr int kTileRows = 128;
constexpr int kTileThreads = 640;
constexpr int kSumWarps = 16;
constexpr int kQStages = 3;      // tiles of Q
constexpr int kCStages = 4;      // the rows' c
constexpr int kUnitSlots = 4;    // units told of
// what starting a unit costs, in steps: the line counts it before the unit's own (K's way to shared
// memory and the exchange at the end; 2: the prompt 140 us for 131, 8: 64 answers over a prefix of 5120
// 20.7 us for 18.2)
constexpr int kUnitCost = 4;
// The MMAs of a score cut what they add off below the accumulator's last bit, d / 16 times: it comes
// out smaller by 0.8e-7 to 2.2e-7 of itself (the slope of its error over scores of 3 to 13; caches
// with outlier channels lose most).  The scale makes up for the middle of that: right on average, and
// at most these 1.5e-7 of the score too much where nothing was cut off or where its parts cancelled, which
// is less than d / 16 MMAs may lose of those parts.
template <int D>
constexpr float kCutOff = D == 128 ? 1.5e-7f : 1.1e-7f;

// Tiles [tile_a, tile_b) of a unit (none: the line is done).
struct Unit {
    int head, key0, len, past;
    int t0, nt;                 // the segment's query tokens
    int tile_a, tile_b;
    int part;                   // -1: the unit whole; 0 and 1: a part of one that ends (starts) here
    int pad;
    const int32_t* table;
};

template <int D>
struct TileCfg {
    static constexpr int kHalves = D / 64;                          // 128-byte column halves of a row
    static constexpr uint32_t kGroup = kHalves * 1024;              // eight rows of K: [halves][8][128 bytes]
    static constexpr uint32_t kK = kKeys / 8 * kGroup;              // a unit's keys
    static constexpr uint32_t kQHalf = kTileRows * 128;
    static constexpr uint32_t kQ = kHalves * kQHalf;
    static constexpr uint32_t kRing = 2 * kK;
    static constexpr uint32_t kC = kRing + kQStages * kQ;           // [stages][rows] c
    static constexpr uint32_t kBlind = kC + kCStages * kTileRows * 4;   // [stages][rows / 32] rows that count for nothing
    static constexpr uint32_t kUnits = kBlind + kCStages * kTileRows / 8;
    static constexpr uint32_t kBars = kUnits + kUnitSlots * sizeof(Unit);
    static constexpr int kNumBars = 2 * 2 + 2 * kQStages + 2 * kCStages + 2 * kUnitSlots + 2 * 2 + 4 + 2;
    static constexpr uint32_t kSmem = kBars + kNumBars * 8 + 16;
    static_assert(kSmem <= 232448, "shared memory of an SM");
};
static_assert(sizeof(Unit) % 16 == 0, "slots");

// Rows of a tile: whole tokens, `tokens` of them, or (more than 128 heads in a group)
// pieces of one token's heads.
struct Tiling {
    int tokens;                 // of a tile (1 if pieces > 1)
    int pieces;                 // tiles a token
};
__host__ __device__ __forceinline__ Tiling tiling(int group) {
    if (group > kTileRows) return {1, (group + kTileRows - 1) / kTileRows};
    const int most = kTileRows / group;
    // a multiple of 16 rows has no ragged step; worth up to a quarter of the tile
    for (int t = most; t > 0 && t * group >= kTileRows * 3 / 4; --t)
        if (t * group % 16 == 0) return {t, 1};
    return {most, 1};
}
__device__ __forceinline__ int tiles_of(const Tiling& ti, int nt) {
    return ti.pieces > 1 ? nt * ti.pieces : (nt + ti.tokens - 1) / ti.tokens;
}
// First tile whose rows see key0 of the segment.
__device__ __forceinline__ int first_tile(const Tiling& ti, const Segment& g, int key0) {
    const int i = max(0, key0 - g.past);
    return ti.pieces > 1 ? i * ti.pieces : i / ti.tokens;
}
// Steps of a KV head, with what its units cost; units before `even` all have every tile.
__device__ __forceinline__ int64_t head_cost(const Tiling& ti, const Segment& g, int* even) {
    const int units = (g.len + kKeys - 1) / kKeys, tiles = tiles_of(ti, g.nt);
    int64_t c = static_cast<int64_t>(units) * (tiles + kUnitCost);
    int k = units;
    if (g.own) {
        const int64_t reach = static_cast<int64_t>(g.past) + ti.tokens;       // first_tile(key0) == 0 for key0 < reach
        k = static_cast<int>(min(static_cast<int64_t>(units), max(static_cast<int64_t>(0), (reach + kKeys - 1) / kKeys)));
        for (int u = k; u < units; ++u) c -= first_tile(ti, g, u * kKeys);
    }
    *even = k;
    return c;
}

template <int D>
__global__ void __launch_bounds__(kTileThreads, 1)
    weigh_tiles_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_q,
                       const __grid_constant__ CUtensorMap tm_q_small, const __grid_constant__ WeighParams p) {
    using Cfg = TileCfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t* k_full = reinterpret_cast<uint64_t*>(smem + Cfg::kBars);
    uint64_t* k_empty = k_full + 2;
    uint64_t* q_full = k_empty + 2;
    uint64_t* q_empty = q_full + kQStages;
    uint64_t* c_full = q_empty + kQStages;
    uint64_t* c_empty = c_full + kCStages;
    uint64_t* u_full = c_empty + kCStages;
    uint64_t* u_empty = u_full + kUnitSlots;
    uint64_t* s_full = u_empty + kUnitSlots;
    uint64_t* s_empty = s_full + 2;
    uint64_t* x_full = s_empty + 2;              // [units][halves] the second warpgroup's sums
    uint64_t* k_done = x_full + 4;               // the unit's MMAs are complete
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(k_done + 2);
    int* abort_flag = reinterpret_cast<int*>(tmem_slot + 1);
    Unit* unit_of = reinterpret_cast<Unit*>(smem + Cfg::kUnits);
    float* c_of = reinterpret_cast<float*>(smem + Cfg::kC);
    uint32_t* blind_of = reinterpret_cast<uint32_t*>(smem + Cfg::kBlind);
    const uint32_t warp = warp_id(), lane = lane_id();
    if (smem_u32(smem) & 1023u) {               // (the tiles' swizzle and TMA need it)
        if (threadIdx.x == 0) report(p.status, CR_DEV_TIMEOUT, 959);
        return;
    }
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(&k_full[i], 1);
            mbar_init(&k_empty[i], 1 + kSumWarps / 2);      // the MMAs, and the first warpgroups
            mbar_init(&k_done[i], 1);
            mbar_init(&s_full[i], 1);
            mbar_init(&s_empty[i], kSumWarps / 2);          // tile t's sums are those of warpgroups t mod 2
        }
        for (int i = 0; i < 4; ++i) mbar_init(&x_full[i], 4);
        for (int i = 0; i < kQStages; ++i) {
            mbar_init(&q_full[i], 1);
            mbar_init(&q_empty[i], 1);
        }
        for (int i = 0; i < kCStages; ++i) {
            mbar_init(&c_full[i], 1);
            mbar_init(&c_empty[i], kSumWarps / 2);
        }
        for (int i = 0; i < kUnitSlots; ++i) {
            mbar_init(&u_full[i], 1);
            mbar_init(&u_empty[i], 3 + kSumWarps);          // every warp but the walker
        }
        fence_barrier_init();
    }
    if (warp == 1) tmem_alloc(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    pdl_launch_dependents();
    const Tiling ti = tiling(p.group);
    // the line, where K comes later
    int64_t* cum = reinterpret_cast<int64_t*>(smem);
    make_line<kTileThreads>(p, cum, cum + kMaxSegments + 2, [&](const Segment& g) -> int64_t {
        int even;
        return g.kind >= 0 ? head_cost(ti, g, &even) * p.n_kv_heads : 0;
    });
    const int n_seg = p.n_groups + p.n_req;
    const int64_t total = cum[n_seg], per = (total + gridDim.x - 1) / gridDim.x;
    int64_t at = min(total, per * blockIdx.x);
    const int64_t end = min(total, at + per);
    int seg = find_segment(cum, n_seg, at);
    int64_t off = at - cum[seg];
    fence_async_smem();
    __syncthreads();                            // cum is read
    const uint32_t tmem = *tmem_slot;
    const WaitCtx wc{abort_flag, p.status};

    // The i-th unit, for every warp but the walker.
    auto unit_at = [&](uint32_t i, Unit* u) -> bool {
        if (!mbar_wait_warp(&u_full[i % kUnitSlots], i / kUnitSlots & 1u, wc, 950)) return false;
        *u = unit_of[i % kUnitSlots];
        __syncwarp();
        if (lane == 0) mbar_arrive(&u_empty[i % kUnitSlots]);
        return u->tile_b > u->tile_a;
    };
    // A tile's rows: how many, the first's token (of the segment) and head of the group.
    auto tile_at = [&](const Unit& u, int tile, int* tok0, int* g0) -> int {
        if (ti.pieces == 1) {
            *tok0 = tile * ti.tokens;
            *g0 = 0;
            return min(ti.tokens, u.nt - *tok0) * p.group;
        }
        *tok0 = tile / ti.pieces;
        *g0 = (tile - *tok0 * ti.pieces) * kTileRows;
        return min(kTileRows, p.group - *g0);
    };
    const int small = max(1, 32 / p.group);     // tokens of the smaller box of Q

    if (warp == 0) {
        // ---------------------------------------------------- units and K
        Segment g = segment<true>(p, seg);
        int units = (g.len + kKeys - 1) / kKeys, tiles = tiles_of(ti, g.nt), head = 0, unit = 0;
        if (at < end) {
            int even;
            const int64_t a_head = max(static_cast<int64_t>(1), head_cost(ti, g, &even));
            head = static_cast<int>(min(off / a_head, static_cast<int64_t>(p.n_kv_heads - 1)));
            off -= head * a_head;
            unit = static_cast<int>(min(off / (tiles + kUnitCost), static_cast<int64_t>(even)));
            off -= static_cast<int64_t>(unit) * (tiles + kUnitCost);
            while (unit < units - 1) {
                const int c = tiles - first_tile(ti, g, unit * kKeys) + kUnitCost;
                if (off < c) break;
                off -= c;
                ++unit;
            }
        }
        bool tail = false, headed = false, tail_last = false, started = false;
        int4 head_part = make_int4(0, 0, 0, 0);
        auto next_unit = [&](Unit* u) -> bool {
            u->tile_a = u->tile_b = 0;
            for (;;) {
                if (at >= end) return false;
                if (started && ++unit >= units) {
                    unit = 0;
                    if (++head >= p.n_kv_heads) {
                        head = 0;
                        do {
                            if (++seg >= n_seg) {
                                at = end;
                                return false;
                            }
                            g = segment<true>(p, seg);
                        } while (g.kind < 0 || g.len == 0);
                        units = (g.len + kKeys - 1) / kKeys;
                        tiles = tiles_of(ti, g.nt);
                    }
                }
                started = true;
                // the unit's steps here: tiles [a, b) of [f, tiles)
                const int f = first_tile(ti, g, unit * kKeys);
                const int64_t cost = tiles - f + kUnitCost, take = max(static_cast<int64_t>(1), min(cost - off, end - at));
                const int a = f + static_cast<int>(max(static_cast<int64_t>(0), off - kUnitCost));
                const int b = min(tiles, f + static_cast<int>(max(static_cast<int64_t>(0), off + take - kUnitCost)));
                at += take;
                off = 0;
                if (a >= b) continue;
                const int part = a == f ? (b == tiles ? -1 : 1) : 0;
                if (part == 1) {
                    headed = true;
                    head_part = make_int4(1, seg, head, unit);
                } else if (part == 0) {
                    tail = true;
                    tail_last = b == tiles;
                }
                *u = {head, unit * kKeys, g.len, g.past, g.t0, g.nt, a, b, part, 0, g.table};
                return true;
            }
        };
        const int box_shift = min(p.block_shift, 7);            // K comes in boxes of min(block, 128) rows
        const int box_key = static_cast<int>(lane) << box_shift;
        const uint32_t box_at = static_cast<uint32_t>(box_key) * (Cfg::kHalves * 128);
        const bool mine = box_key < kKeys;
        auto block_at = [&](const Unit& u) -> int {             // of this lane's box; past the end: past the cache,
            const int key = u.key0 + box_key;                   // where a box reads zeros
            return mine && u.tile_b > u.tile_a && key < u.len ? u.table[key >> p.block_shift] : p.n_blocks;
        };
        uint32_t kb = 0, kph = 1;
        Unit u, then;
        next_unit(&u);
        int block = block_at(u);
        bool ok = true;
        for (uint32_t i = 0; ok; ++i) {
            if (!(ok = mbar_wait_warp(&u_empty[i % kUnitSlots], (i / kUnitSlots & 1u) ^ 1u, wc, 951))) break;
            if (lane == 0) {
                unit_of[i % kUnitSlots] = u;
                mbar_arrive(&u_full[i % kUnitSlots]);
            }
            __syncwarp();
            if (u.tile_b <= u.tile_a) break;
            next_unit(&then);
            const int next_block = block_at(then);              // in flight while this unit waits
            if (block < 0 || block > p.n_blocks || (block == p.n_blocks && mine && u.key0 + box_key < u.len)) {
                report(p.status, CR_DEV_INDEX, 942);
                block = p.n_blocks;
            }
            const int row = (block << p.block_shift) +
                            (block == p.n_blocks ? 0 : (u.key0 + box_key) & ((1 << p.block_shift) - 1));
            if (!(ok = mbar_wait_warp(&k_empty[kb], kph, wc, 952))) break;
            if (lane == 0) mbar_expect_tx(&k_full[kb], Cfg::kK);
            __syncwarp();
            if (mine) tma_load_4d(smem + kb * Cfg::kK + box_at, &tm_k, &k_full[kb], 0, 0, u.head * Cfg::kHalves, row >> 3);
            __syncwarp();
            kb ^= 1u;
            kph ^= kb == 0 ? 1u : 0u;
            u = then;
            block = next_block;
        }
        if (lane == 0) {
            p.part_head[blockIdx.x] = headed ? head_part : make_int4(0, 0, 0, 0);
            p.part_tail[blockIdx.x] = tail ? (tail_last ? 2 : 1) : 0;
        }
    } else if (warp == 1) {
        // ---------------------------------------------------- MMA issue
        const uint64_t dk0 = smem_desc(smem_u32(smem), 16, Cfg::kGroup, SWZ_128B);
        const uint64_t dq0 = smem_desc(smem_u32(smem + Cfg::kRing), 16, 1024, SWZ_128B);
        uint32_t kb = 0, kph = 0, qs = 0, qph = 0, ts = 0, tph = 1;
        Unit u;
        bool ok = true;
        for (uint32_t i = 0; ok && unit_at(i, &u); ++i) {
            if (!mbar_wait_warp(&k_full[kb], kph, wc, 953)) break;
            const uint64_t dk = dk0 + static_cast<uint64_t>(kb) * (Cfg::kK >> 4);
            for (int tile = u.tile_a; tile < u.tile_b; ++tile) {
                int tok0, g0;
                const int n = tile_at(u, tile, &tok0, &g0);
                if (!(ok = mbar_wait_warp(&q_full[qs], qph, wc, 954))) break;
                if (!(ok = mbar_wait_warp(&s_empty[ts], tph, wc, 955))) break;
                tc_fence_after();
                const uint32_t idesc = idesc_bf16(128, (n + 15) & ~15, false, false);
                const uint64_t dq = dq0 + static_cast<uint64_t>(qs) * (Cfg::kQ >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
                            mma_bf16_ss(tmem + (ts * 2 + h) * 128,
                                        dk + h * (16 * Cfg::kGroup >> 4) + (k >> 2) * (1024 >> 4) + (k & 3) * 2,
                                        dq + (k >> 2) * (Cfg::kQHalf >> 4) + (k & 3) * 2, idesc, k != 0 ? 1u : 0u);
                    }
                    mma_commit(&s_full[ts]);
                    mma_commit(&q_empty[qs]);
                    if (tile + 1 == u.tile_b) {
                        mma_commit(&k_empty[kb]);
                        mma_commit(&k_done[kb]);
                    }
                }
                __syncwarp();
                if (++qs == kQStages) {
                    qs = 0;
                    qph ^= 1u;
                }
                ts ^= 1u;
                tph ^= ts == 0 ? 1u : 0u;
            }
            kb ^= 1u;
            kph ^= kb == 0 ? 1u : 0u;
        }
    } else if (warp < 4) {
        // ---------------------------------------------------- tiles of Q, and c of their rows
        const int turn = static_cast<int>(warp) - 2;
        // rows lane, lane + 32, ... of a tile: where their lse lies
        int lse_at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = static_cast<int>(lane) + 32 * i, tok = ti.pieces > 1 ? 0 : r / p.group;
            lse_at[i] = tok * p.n_q_heads + r - tok * p.group;
        }
        uint32_t step = 0;                  // tiles before, by both warps
        Unit u;
        bool ok = true;
        for (uint32_t i = 0; ok && unit_at(i, &u); ++i) {
            const bool few = ti.pieces == 1 && u.nt <= small;
            const CUtensorMap* map = few ? &tm_q_small : &tm_q;
            const uint32_t box = static_cast<uint32_t>((few ? small : ti.tokens) * min(p.group, kTileRows)) * 128u;
            auto ask = [&](int tile, float (&lse)[4]) {
                if (tile >= u.tile_b) return;
                int tok0, g0;
                const int n = tile_at(u, tile, &tok0, &g0);
                const float* src = p.lse + static_cast<int64_t>(u.t0 + tok0) * p.n_q_heads + (u.head * p.group + g0);
#pragma unroll
                for (int k = 0; k < 4; ++k) lse[k] = static_cast<int>(lane) + 32 * k < n ? src[lse_at[k]] : 0.0f;
            };
            const int first = u.tile_a + ((static_cast<int>(step) + turn) & 1);
            float lse[4];
            ask(first, lse);
            for (int tile = first; tile < u.tile_b; tile += 2) {
                const uint32_t st = step + static_cast<uint32_t>(tile - u.tile_a), qs = st % kQStages, cs = st % kCStages;
                int tok0, g0;
                tile_at(u, tile, &tok0, &g0);
                if (!(ok = mbar_wait_warp(&q_empty[qs], (st / kQStages & 1u) ^ 1u, wc, 956))) break;
                if (elect_one()) {
                    mbar_expect_tx(&q_full[qs], box * Cfg::kHalves);
#pragma unroll
                    for (int h = 0; h < Cfg::kHalves; ++h)
                        tma_load_3d(smem + Cfg::kRing + qs * Cfg::kQ + h * Cfg::kQHalf, map, &q_full[qs], h * 64,
                                    u.head * p.group + g0, u.t0 + tok0);
                }
                __syncwarp();
                float c[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) c[k] = -log2_lse(p, lse[k]);
                const bool none = fminf(fminf(lse[0], lse[1]), fminf(lse[2], lse[3])) == neg_inf();
                uint32_t blind = 0;             // (lanes 0 .. 3: of rows 32 lane .. 32 lane + 31)
                if (__any_sync(0xffffffffu, none)) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t b = __ballot_sync(0xffffffffu, lse[k] == neg_inf());
                        if (lane == static_cast<uint32_t>(k)) blind = b;
                    }
                }
                ask(tile + 2, lse);
                if (!(ok = mbar_wait_warp(&c_empty[cs], (st / kCStages & 1u) ^ 1u, wc, 957))) break;
#pragma unroll
                for (int k = 0; k < 4; ++k) c_of[cs * kTileRows + lane + 32 * k] = c[k];
                if (lane < 4) blind_of[cs * 4 + lane] = blind;
                __syncwarp();
                if (lane == 0) mbar_arrive(&c_full[cs]);
            }
            step += static_cast<uint32_t>(u.tile_b - u.tile_a);
        }
    } else {
        // ---------------------------------------------------- sums
        const int group = (static_cast<int>(warp) - 4) >> 2, h = group & 1, turn = group >> 1;
        const int lane_key = static_cast<int>((warp & 3u) * 32 + lane), key = h * 128 + lane_key;     // of the half, of the unit
        const uint32_t lane_off = ((warp & 3u) * 32u) << 16;
        const float sc = p.scale_log2, sc_lo = sc * kCutOff<D>;
        uint32_t step = 0, kb = 0, kph = 0;         // tiles before, by all warpgroups; the unit's buffer of K
        Unit u;
        bool ok = true;
        for (uint32_t i = 0; ok && unit_at(i, &u); ++i) {
            float sum = 0.0f, lost = 0.0f;          // of the unit, and what its roundings lost
            const int block = turn == 0 && u.key0 + key < u.len ? block_of(p, u.table, u.key0 + key) : -1;
            const int skip = (static_cast<int>(step) + turn) & 1;
            for (int tile = u.tile_a + skip; tile < u.tile_b; tile += 2) {
                const uint32_t st = step + static_cast<uint32_t>(tile - u.tile_a), cs = st % kCStages, ts = st & 1u;
                int tok0, g0;
                const int n = tile_at(u, tile, &tok0, &g0);
                if (!(ok = mbar_wait_warp(&c_full[cs], st / kCStages & 1u, wc, 958))) break;
                if (!(ok = mbar_wait_warp(&s_full[ts], st >> 1 & 1u, wc, 960))) break;
                tc_fence_after();
                // 16 rows at a time; the next ones come while these are summed
                const uint32_t d = tmem + lane_off + (ts * 2 + h) * 128;
                const float* c_tile = c_of + cs * kTileRows;
                const uint4 blind4 = *reinterpret_cast<const uint4*>(blind_of + cs * 4);
                const bool any_blind = (blind4.x | blind4.y | blind4.z | blind4.w) != 0;
                float x[2][16], acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                auto add_full = [&](const float* v, const float* cv) {
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const float4 c = *reinterpret_cast<const float4*>(cv + j);
                        float y[4];
                        ffma2(y[0], y[1], v[j], v[j + 1], sc, sc, c.x, c.y);
                        ffma2(y[2], y[3], v[j + 2], v[j + 3], sc, sc, c.z, c.w);
                        ffma2(y[0], y[1], v[j], v[j + 1], sc_lo, sc_lo, y[0], y[1]);
                        ffma2(y[2], y[3], v[j + 2], v[j + 3], sc_lo, sc_lo, y[2], y[3]);
                        fadd2(acc[0], acc[1], acc[0], acc[1], ex2(y[0]), ex2(y[1]));
                        fadd2(acc[2], acc[3], acc[2], acc[3], ex2(y[2]), ex2(y[3]));
                    }
                };
                const int sees = u.past == kAll ? kKeys : u.past + tok0 + 1 - u.key0;   // keys of the unit that the first token sees
                if (n == kTileRows && sees >= kKeys && !any_blind) {
                    tmem_ld16(d, x[0]);
#pragma unroll
                    for (int k = 0; k < kTileRows / 16; ++k) {
                        tmem_landed16(x[k & 1]);
                        if (k + 1 < kTileRows / 16) {
                            tmem_ld16(d + 16 * (k + 1), x[(k + 1) & 1]);
                        } else {
                            tc_fence_before();
                            if (elect_one()) mbar_arrive(&s_empty[ts]);
                        }
                        add_full(x[k & 1], c_tile + 16 * k);
                    }
                } else {
                    // rows are in the order of their tokens, so a key is seen by those from one on: by the
                    // first of the warp's keys from lo0 on, by the last from lo31 on
                    const int lo = max(0, key + 1 - sees) * p.group;
                    const int lo0 = __shfl_sync(0xffffffffu, lo, 0), lo31 = __shfl_sync(0xffffffffu, lo, 31);
                    int col = lo0 & ~15;
                    if (col < n) tmem_ld16(d + col, x[0]);
#pragma unroll 1
                    for (; col < n; col += 32) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int at = col + 16 * k;
                            if (at >= n) break;
                            tmem_landed16(x[k]);
                            if (at + 16 < n) tmem_ld16(d + at + 16, x[k ^ 1]);
                            const uint32_t blind = any_blind ? blind_of[cs * 4 + (at >> 5)] >> (at & 16) & 0xffffu : 0u;
                            if (at >= lo31 && at + 16 <= n && blind == 0) {
                                add_full(x[k], c_tile + at);
                                continue;
                            }
                            // (selected before the sum, so that a row that does not count brings no NaN in)
                            const uint32_t in = ~blind & (at + 16 <= n ? 0xffffu : (1u << (n - at)) - 1u) &
                                                (lo <= at ? 0xffffu : lo >= at + 16 ? 0u : 0xffffu << (lo - at));
#pragma unroll
                            for (int j = 0; j < 16; ++j) {
                                const float e = ex2(fmaf(x[k][j], sc_lo, fmaf(x[k][j], sc, c_tile[at + j])));
                                acc[j & 3] += in >> j & 1u ? e : 0.0f;
                            }
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&s_empty[ts]);
                }
                const float add = (acc[0] + acc[1]) + (acc[2] + acc[3]), now = sum + add;
                lost += add - (now - sum);
                sum = now;
                __syncwarp();
                if (lane == 0) mbar_arrive(&c_empty[cs]);
            }
            step += static_cast<uint32_t>(u.tile_b - u.tile_a);
            if (!ok) break;
            // the two warpgroups of a half add up where the unit's K was, once the MMAs are done with it
            float* other = reinterpret_cast<float*>(smem + kb * Cfg::kK) + h * 128;
            if (turn) {
                if (!(ok = mbar_wait_warp(&k_done[kb], kph, wc, 964))) break;
                other[lane_key] = sum + lost;
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(&x_full[2 * kb + h]);
            } else {
                if (!(ok = mbar_wait_warp(&x_full[2 * kb + h], kph, wc, 961))) break;
                const float all = (sum + lost) + other[lane_key];
                __syncwarp();
                if (lane == 0) mbar_arrive(&k_empty[kb]);
                if (u.part >= 0) p.part_sum[(static_cast<int64_t>(blockIdx.x) * 2 + u.part) * kKeys + key] = all;
                else if (block >= 0) give(p, u.head, slot_in(p, block, u.key0 + key), u.key0 + key >= u.past, all);
            }
            kb ^= 1u;
            kph ^= kb == 0 ? 1u : 0u;
        }
    }
    // (a role that gave a wait up leaves its copies time to land)
    __syncwarp();
    if (*reinterpret_cast<volatile int*>(abort_flag)) {
        const uint64_t t0 = globaltimer();
        while (globaltimer() - t0 < 50000ull) {
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, 512);
}

// The parts of the units that the line's cuts went through: CTA c's unit starts there and goes
// on in the CTAs behind it.
__global__ void __launch_bounds__(kKeys) weigh_join_kernel(const __grid_constant__ WeighParams p, int n_ctas) {
    pdl_launch_dependents();
    pdl_wait();
    const int c = static_cast<int>(blockIdx.x), key = static_cast<int>(threadIdx.x);
    const int4 part = p.part_head[c];
    if (!part.x) return;
    float sum = p.part_sum[(static_cast<int64_t>(c) * 2 + 1) * kKeys + key];
    for (int i = c + 1; i < n_ctas; ++i) {
        const int t = p.part_tail[i];
        if (t == 0) break;
        sum += p.part_sum[static_cast<int64_t>(i) * 2 * kKeys + key];
        if (t == 2) break;
    }
    const Segment g = segment<false>(p, part.y);
    const int j = part.w * kKeys + key;
    if (j >= g.len) return;
    const int block = block_of(p, g.table, j);
    if (block >= 0) give(p, part.z, slot_in(p, block, j), j >= g.past, sum);
}

// ------------------------------------------------------------------ host
template <int D>
cr_status launch_tiles(const WeighParams& p, const cr_paged_layer& c, int n_tokens, int n_ctas, cudaStream_t st) {
    using Cfg = TileCfg<D>;
    const Tiling ti = tiling(p.group);
    const int heads = p.group < kTileRows ? p.group : kTileRows;
    const int small = 32 / p.group < 1 ? 1 : 32 / p.group;
    const int box = c.block_size < 128 ? c.block_size : 128;
    CUtensorMap tk, tq, tqs;
    if (!make_tmap_groups(&tk, c.k, static_cast<uint64_t>(c.n_kv_heads) * D, static_cast<uint64_t>(p.n_blocks) << p.block_shift,
                          Cfg::kHalves, box / 8) ||
        !make_tmap_3d(&tq, p.q, D, p.n_q_heads, n_tokens, D * 2, p.ldq * 2, 64, heads, ti.tokens) ||
        !make_tmap_3d(&tqs, p.q, D, p.n_q_heads, n_tokens, D * 2, p.ldq * 2, 64, heads, small))
        return CR_ERR_INVALID_ARG;
    static unsigned long long attr_done = 0;
    cr_status s = ensure_smem_attr(weigh_tiles_kernel<D>, static_cast<int>(Cfg::kSmem), &attr_done);
    if (s != CR_OK) return s;
    s = launch_pdl(weigh_tiles_kernel<D>, dim3(n_ctas), dim3(kTileThreads), Cfg::kSmem, st, tk, tq, tqs, p);
    if (s != CR_OK) return s;
    return launch_pdl(weigh_join_kernel, dim3(n_ctas), dim3(kKeys), 0, st, p, n_ctas);
}

}  // namespace

size_t weigh_part_bytes(int n_ctas) { return static_cast<size_t>(n_ctas) * (2 * kKeys * sizeof(float) + sizeof(int4) + sizeof(int32_t)); }

cr_status launch_weigh(WeighParams& p, const cr_paged_layer& c, const cr_attention_batch& b, cudaStream_t st) {
    uint8_t* parts = paged_weigh_parts(b);
    p.part_sum = reinterpret_cast<float*>(parts);
    p.part_head = reinterpret_cast<int4*>(parts + static_cast<size_t>(b.n_ctas) * 2 * kKeys * sizeof(float));
    p.part_tail = reinterpret_cast<int32_t*>(p.part_head + b.n_ctas);
    // Segments of few rows beside others go the others' way: one kernel, where two after one another
    // took 25.5 us instead of 17.8 (64 answers of one token over 30 to 250 and a prefix of 5120).
    if (b.n_units[PAGED_TILES])
        return c.head_dim == 128 ? launch_tiles<128>(p, c, b.n_tokens, b.n_ctas, st) : launch_tiles<64>(p, c, b.n_tokens, b.n_ctas, st);
    return launch_pdl(c.head_dim == 128 ? weigh_few_kernel<128> : weigh_few_kernel<64>, dim3(kFewCtas * num_sms()), dim3(kFewThreads), 0, st, p);
}

}  // namespace cr
