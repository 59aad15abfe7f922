// Attention over a paged cache, with or without prefixes shared by groups of
// requests:
//   o_i = sum_j softmax_j(scale q_i . k_j) v_j
// over the keys that row i sees: its group's whole prefix and the tokens of its
// own request up to itself.  The keys form segments (PagedParams), each walked
// in chunks with a running maximum m and sum l per row, in units of log2:
//   x_j = scale log2(e) q.k_j,  m' = max(m, max x),  l' = l 2^(m - m') + sum 2^(x - m'),
//   O' = O 2^(m - m') + sum 2^(x - m') v,
// and the parts of a row are joined by
//   M = max_p m_p,  o = sum_p 2^(m_p - M) O_p / sum_p 2^(m_p - M) l_p.
//
// A segment's rows are the query tokens' heads of one KV head, which read the same
// keys: a decode step has a few of them, a prompt or a prefix shared by many
// requests hundreds.  Few rows are bound by HBM (each K and V byte is used for
// 2 x rows flops) and go through mma.sync with the keys as M; many are bound by
// the tensor cores or shared memory and go through tcgen05 in tiles of 128 rows.
// Both kinds run in one launch, in different CTAs (a call of one kind alone in a
// kernel without the other's code).  The work of each kind is one
// line of chunks, segment by segment and unit by unit, which its workers cut into
// equal parts whatever the sequences' lengths are; lengths and blocks are read on
// the device, so nothing is planned on the host but the batch's shape.
//
// Measured in a CUDA graph, alternating between two inputs (bf16, 32 heads over 8
// of 128 unless said, SM clock 2.07 GHz): a 2048-token prompt over 8192 cached tokens 213 us (1.45
// PFLOP/s, 0.77 of the measured burst bf16 rate); 256 answers over a shared
// 32768-token prefix and 100-500 tokens of their own 130 us; a decode step of 16
// requests of 6-10k tokens 92 us (5.9 TB/s, 0.87 of the measured copy rate; the
// kernel alone 84, 6.4 TB/s); one of 5120 tokens 9.9 us.
#include <cuda_bf16.h>
#include <string.h>

#include "cr_internal.h"
#include "cr_ptx.cuh"

namespace cr {
namespace {

constexpr int kMaxSegments = 2 * kMaxReq;
// Segments of few rows (PAGED_ROWS): a unit is a KV head, all of its rows.
constexpr int kRowsTile = 16;       // most rows: two N = 8 tiles of m16n8k16
constexpr int kChunk = 16;          // keys of a chunk
constexpr int kRowsWarps = 12;      // workers in a CTA
constexpr int kMinChunks = 2;       // fewest chunks a worker takes
// Segments of many rows (PAGED_TILES): a unit is a KV head and 256 rows.
constexpr int kPair = 256;          // rows of a unit: two 128-row tiles
constexpr int kKeys = 128;          // keys of a chunk
// What starting a unit costs a tile CTA (its rows of Q in, results out), in
// chunks: the line of tiles counts them before a unit's own.  (40 questions of 60
// to 120 tokens over 100 to 900: 119 us without, 96, 87 and 85 with 1, 2 and 3.)
constexpr int kUnitCost = 3;
constexpr int kBlockRows = 4;       // rows that a warp of the join takes together
constexpr float kRescaleLog2 = 8.0f;   // a running maximum moves when a chunk exceeds it by more than 2^8

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

// ------------------------------------------------------------------ segments
struct Segment {
    int t0, nt;            // query tokens
    int unit_base, kind;
    int len;               // keys
    int blocks;            // entries of `table` that hold them
    const int32_t* table;
    bool own;              // causal among the last nt keys
};

__device__ __forceinline__ int clamp_len(const PagedParams& p, int len, int64_t max_blocks) {
    const int64_t most = max_blocks << p.block_shift;
    if (len >= 0 && len <= most) return len;
    report(p.status, CR_DEV_INDEX, 911);
    return len < 0 ? 0 : static_cast<int>(most);
}

// A CTA reads a length when it makes the line and again when it comes to the
// segment.  Lengths that are changed during a call leave its results undefined, but
// every loop and index below stays bounded by what the plan says, and a warp takes
// one lane's reading (kWarp), so that nothing waits or writes elsewhere for it.
template <bool kWarp>
__device__ __forceinline__ Segment segment(const PagedParams& p, int s) {
    Segment g;
    g.own = s >= p.n_groups;
    const int r = s - p.n_groups;
    const int4 d = p.seg[s];
    int len = g.own ? p.own_len[r] : p.prefix_len[s];
    if (kWarp) len = __shfl_sync(0xffffffffu, len, 0);      // behind both loads
    g.t0 = d.x;
    g.nt = d.y;
    g.unit_base = d.z;
    g.kind = d.w;
    g.table = g.own ? p.own_table + r * p.own_blocks : p.prefix_table + s * p.prefix_blocks;
    g.len = clamp_len(p, len, g.own ? p.own_blocks : p.prefix_blocks);
    g.blocks = (g.len + (1 << p.block_shift) - 1) >> p.block_shift;
    return g;
}

// Query token of row n of a segment.
__device__ __forceinline__ int token_of(const PagedParams& p, int n) {
    return static_cast<int>((__umulhi(p.group_mul, static_cast<uint32_t>(n)) + static_cast<uint32_t>(n)) >> p.group_shift);
}

// Keys that a row of the segment sees: all of a prefix, one's own tokens up to
// the row's own (never negative).
__device__ __forceinline__ int row_limit(const PagedParams& p, const Segment& g, int row) {
    if (!g.own) return g.len;
    const int lim = g.len - g.nt + token_of(p, row) + 1;
    return lim < 0 ? 0 : lim;
}
// Chunks that rows [row0, row0 + n) of the segment need (row0 must be one of its rows).
__device__ __forceinline__ int chunks_of(const PagedParams& p, const Segment& g, int row0, int n, int chunk) {
    const int last = min(row0 + n, g.nt * p.group) - 1;
    return (row_limit(p, g, last) + chunk - 1) / chunk;
}

// Chunks of all units of a segment of kind `which`; publish: leave the line
// of an own segment's units for the join.
template <int which>
__device__ __forceinline__ int segment_cost(const PagedParams& p, const Segment& g, bool publish = false) {
    const int rows = g.nt * p.group;
    int c = 0;
    if (which == PAGED_ROWS) {
        c = (g.len + kChunk - 1) / kChunk;          // (one row tile)
    } else if (!g.own) {
        c = g.len ? (rows + kPair - 1) / kPair * ((g.len + kKeys - 1) / kKeys + kUnitCost) : 0;
    } else {
        int2* unit = publish ? p.part[PAGED_TILES].unit + g.unit_base : nullptr;
        for (int r = 0; r < rows; r += kPair) {
            const int n = chunks_of(p, g, r, kPair, kKeys);
            if (publish) unit[r / kPair] = make_int2(c, n);
            c += n ? n + kUnitCost : 0;
        }
    }
    return c * p.n_kv_heads;
}
template <int which>
__device__ __forceinline__ int segment_cost(const PagedParams& p, int s) {        // (by a whole warp)
    if (s >= p.n_groups + p.n_req) return 0;
    const Segment g = segment<true>(p, s);
    return g.kind == which ? segment_cost<which>(p, g) : 0;
}

// Chunks of the line that one worker takes.
template <int which>
__device__ __forceinline__ int per_worker(int total, int n_workers) {
    const int c = (total - 1) / n_workers + 1;
    const int least = which == PAGED_ROWS ? kMinChunks : 1;
    return c < least ? least : c;
}

// How many of the CTAs do tiles when a call has chunks of both kinds: by the
// time that the chunks take a CTA, about 1.5 us for two row tiles on 128 keys
// and 0.09 us for 16 keys among twelve warps.  (256 answers over a shared prefix:
// 142, 138, 133, 133 and 135.5 us with 0.075, 0.08, 0.085, 0.09 and 0.1; four groups of 13
// over 2.5 to 10 thousand: 54, 54, 42.4, 42.4 and 42.4.)
constexpr float kTileCost = 1.5f, kRowsCost = 0.09f;
__device__ __forceinline__ int tile_ctas(int tiles, int rows, int n) {
    if (rows == 0) return n;
    if (tiles == 0) return 0;
    const float t = kTileCost * static_cast<float>(tiles), r = kRowsCost * static_cast<float>(rows);
    const int x = static_cast<int>(static_cast<float>(n) * t / (t + r) + 0.5f);
    return max(1, min(min(x, n - 1), tiles));
}

// What the join reads of a line: two segments an entry, each's first chunk and length,
// then the chunks per worker with the multiplier and shift that divide by it
// (as the host's for the group: n / per = (umulhi(n, mul) + n) >> shift, n < 2^31).
constexpr int kSchedPer = 2 * kMaxSegments, kSchedInts = kSchedPer + 3;
__device__ __forceinline__ void publish_per(int* sched, int per) {
    const int shift = 32 - __clz(per - 1);               // the smallest with 2^shift >= per
    sched[kSchedPer] = per;
    sched[kSchedPer + 1] =
        static_cast<int>(static_cast<uint32_t>((((1ull << shift) - per) << 32) / per + 1));
    sched[kSchedPer + 2] = shift;
}

// The lines of both kinds of chunks (their lengths fit 31 bits: the host
// checks), by all threads of the CTA (256 or more).  This CTA's kind and place
// among the CTAs of its kind, and its line: cum[i] = chunks of its kind before
// segment 2 i, two segments an entry to save shared memory.
constexpr int kCumEntries = kMaxSegments / 2 + 1;
struct Share {
    bool tiles;
    int index, count;          // CTA of this kind, and how many there are
    int total, per;            // chunks of the line, and a worker's
};
template <bool kRows, bool kTiles>
__device__ __forceinline__ Share schedule(const PagedParams& p, int* cum, int64_t* warp_sum) {
    const int i = static_cast<int>(threadIdx.x);
    const bool publish = blockIdx.x == 0;           // for the join
    int64_t c[2] = {0, 0};                          // tiles in the upper half, rows in the lower
    int len[2] = {0, 0};
    if (i < kMaxSegments / 2) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (2 * i + k >= p.n_groups + p.n_req) continue;
            const Segment g = segment<false>(p, 2 * i + k);
            len[k] = g.len;
            if (kTiles && g.kind == PAGED_TILES) c[k] = static_cast<int64_t>(segment_cost<PAGED_TILES>(p, g, publish)) << 32;
            else if (kRows && g.kind == PAGED_ROWS) c[k] = segment_cost<PAGED_ROWS>(p, g);
        }
    }
    int64_t x = c[0] + c[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (static_cast<int>(lane_id()) >= o) x += y;
    }
    if (lane_id() == 31) warp_sum[warp_id()] = x;
    __syncthreads();
    int64_t total = 0;
    const uint32_t used = static_cast<uint32_t>(p.n_groups + p.n_req + 63) >> 6;   // warps that hold segments
    for (uint32_t w = 0; w < used; ++w) {
        if (w < warp_id()) x += warp_sum[w];
        total += warp_sum[w];
    }
    const int tiles = static_cast<int>(total >> 32), rows = static_cast<int>(total);
    const int n = static_cast<int>(gridDim.x), nt = tile_ctas(tiles, rows, n);
    const int per_t = per_worker<PAGED_TILES>(tiles, max(nt, 1));
    const int per_r = per_worker<PAGED_ROWS>(rows, max(n - nt, 1) * kRowsWarps);
    Share sh;
    sh.tiles = static_cast<int>(blockIdx.x) < nt;
    sh.index = static_cast<int>(blockIdx.x) - (sh.tiles ? 0 : nt);
    sh.count = sh.tiles ? nt : n - nt;
    sh.total = sh.tiles ? tiles : rows;
    sh.per = sh.tiles ? per_t : per_r;
    if (i < kMaxSegments / 2) {
        cum[i + 1] = sh.tiles ? static_cast<int>(x >> 32) : static_cast<int>(x);
        if (publish) {
            const int64_t a = x - c[0] - c[1], b = x - c[1];
            if (p.part[PAGED_TILES].sched)
                reinterpret_cast<int4*>(p.part[PAGED_TILES].sched)[i] =
                    make_int4(static_cast<int>(a >> 32), len[0], static_cast<int>(b >> 32), len[1]);
            if (p.part[PAGED_ROWS].sched)
                reinterpret_cast<int4*>(p.part[PAGED_ROWS].sched)[i] =
                    make_int4(static_cast<int>(a), len[0], static_cast<int>(b), len[1]);
        }
    }
    if (i == 0) {
        cum[0] = 0;
        if (publish) {
            if (p.part[PAGED_TILES].sched) publish_per(p.part[PAGED_TILES].sched, per_t);
            if (p.part[PAGED_ROWS].sched) publish_per(p.part[PAGED_ROWS].sched, per_r);
        }
    }
    __syncthreads();
    return sh;
}

// The segment that holds place `at` of the line, its number and its own first place.
template <int which>
__device__ __forceinline__ Segment segment_at(const PagedParams& p, const int* cum, int at, int* number, int* start) {
    int lo = 0, hi = (p.n_groups + p.n_req - 1) >> 1;      // the last pair that starts at or before it
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cum[mid] <= at) lo = mid;
        else hi = mid - 1;
    }
    const int c0 = segment_cost<which>(p, 2 * lo);
    const bool second = at >= cum[lo] + c0 && 2 * lo + 1 < p.n_groups + p.n_req;
    *start = cum[lo] + (second ? c0 : 0);
    *number = 2 * lo + (second ? 1 : 0);
    Segment g = segment<true>(p, *number);
    if (g.kind != which) {        // (a changed length; the pair has a segment of this kind, or it would not be on the line)
        *number ^= 1;
        *start = cum[lo];
        g = segment<true>(p, *number);
    }
    return g;
}

// Where the partial of a worker's piece of a unit lies.  Unit and worker both
// grow along the line, so their sum is a place of its own.  Tiles without
// prefixes: units that lie in one piece are finished there, which leaves each
// worker its first and last piece.
template <int which>
__device__ __forceinline__ int64_t part_slot(const PagedParams& p, int unit, int worker, bool first) {
    if (which == PAGED_TILES && p.n_groups == 0) return 2ll * worker + (first ? 0 : 1);
    return static_cast<int64_t>(unit) + worker;
}

// Column c (of eight that start at a multiple of 8) of O of the partials' row
// `row`.  Of few rows: row by row.  Of tiles, where a thread holds a row: rows lie
// next to one another, 32 bytes of each, and a warp writes whole lines.
template <int which, int D>
__device__ __forceinline__ int64_t part_at(int64_t row, int c) {
    if (which == PAGED_ROWS) return row * D + c;
    return (row >> 7) * (128 * D) + (row & 127) * 8 + (c >> 3) * 1024 + (c & 7);
}

// ------------------------------------------------------------------ few rows
template <int D>
struct RowsCfg {
    static constexpr int kHalves = D / 64;                       // 128-byte column halves of a row
    static constexpr uint32_t kTile = kHalves * kChunk * 128;    // K (or V) of a chunk
    static constexpr uint32_t kStage = 2 * kTile;
    static constexpr int kStages = D == 128 ? 2 : 4;
    static constexpr uint32_t kBars = kRowsWarps * kStages * kStage;
    static constexpr uint32_t kEnd = kBars + kRowsWarps * kStages * 8;
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, const uint32_t* b) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// The transpose of an 8x8 matrix of 16-bit values, two of a row in each thread.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// After a wait that gave up: leave the copies in flight time to land before the
// CTA's shared memory is given back.
__device__ __forceinline__ void drain_pause() {
    const uint64_t t0 = globaltimer();
    while (globaltimer() - t0 < 50000ull) {
    }
}

// Where a warp stands on the line of chunks.
struct Cursor {
    int seg, head, chunk;       // a unit is a KV head of a segment
    int n_chunks;
    Segment g;
};

__device__ __forceinline__ void enter(Cursor& c, int seg, const Segment& g) {
    c.seg = seg;
    c.g = g;
    c.n_chunks = max(1, (g.len + kChunk - 1) / kChunk);
}
__device__ __forceinline__ void seek(const PagedParams& p, Cursor& c, const int* cum, int at) {
    int seg, start;
    const Segment g = segment_at<PAGED_ROWS>(p, cum, at, &seg, &start);
    enter(c, seg, g);
    c.head = min((at - start) / c.n_chunks, p.n_kv_heads - 1);
    c.chunk = min(at - start - c.head * c.n_chunks, c.n_chunks - 1);
}
// One chunk on; the caller knows that the line goes on.
__device__ __forceinline__ void advance(const PagedParams& p, Cursor& c) {
    if (++c.chunk < c.n_chunks) return;
    c.chunk = 0;
    if (++c.head < p.n_kv_heads) return;
    c.head = 0;
    const int end = p.n_groups + p.n_req;
    for (int s = c.seg + 1; s < end; ++s) {
        const Segment g = segment<true>(p, s);
        if (g.kind == PAGED_ROWS && g.len > 0) return enter(c, s, g);    // (others have no work here)
    }
}

// T sets of eight rows of a unit as a warp holds them, and one chunk of 16 keys
// for them.  Keys are the M dimension of both products, rows the N: S^T = K Q^T
// and O^T = V^T P^T, which wastes fewer of the m16n8k16 products on missing rows
// than rows as M would (a decode step has 4 to 8); at about 32 clocks each, they
// are what a chunk's time is made of.  A thread holds keys kq, kq + 8 of S, rows
// rq, rq + 1 of each eight, and d kq, kq + 8 of each sixteen of O.
template <int D, int T>
struct RowsState {
    uint32_t qf[T][D / 16][2];
    float o[T][D / 16][4];
    float m[T][2], l[T][2];
    int lim[T][2];             // keys that the row sees
};
template <int D, int T, int TMAX>
__device__ __forceinline__ void rows_chunk(RowsState<D, TMAX>& w, uint32_t kb, uint32_t vb, int key0, float scale) {
    constexpr uint32_t kGroup = D / 64 * 1024;           // eight keys
    const uint32_t lane = lane_id();
    // ldmatrix rows of this lane: K (keys by 8, then d by 8), V transposed (d by 8, then keys by 8)
    const uint32_t r8 = lane & 7;
    const uint32_t k_at = kb + ((lane >> 3) & 1) * kGroup + r8 * 128, k_odd = lane >> 4;
    const uint32_t v_at = vb + (lane >> 4) * kGroup + r8 * 128, v_odd = (lane >> 3) & 1;
    float s[T][2][4] = {};       // two chains over d
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        const uint32_t c = 2 * k + k_odd;
        uint32_t a[4];
        ldsm4(k_at + (c >> 3) * 1024 + (((c & 7) ^ r8) << 4), a);
#pragma unroll
        for (int t = 0; t < T; ++t) mma16816(s[t][k & 1], a, w.qf[t][k]);
    }
    const int key = key0 + static_cast<int>(lane >> 2);
    uint32_t pk[T][2];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        // elements 0, 1: key, rows rq, rq + 1; 2, 3: key + 8
        float x[4], mx[2];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = (s[t][0][e] + s[t][1][e]) * scale;
            if (key + 4 * (e & 2) >= w.lim[t][e & 1]) x[e] = neg_inf();
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) mx[h] = fmaxf(x[h], x[2 + h]);
#pragma unroll
        for (int d = 4; d < 32; d <<= 1)
#pragma unroll
            for (int h = 0; h < 2; ++h) mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], d));
        // move the reference when this chunk would push P past 2^8 (any reference
        // gives the same quotient O / l)
        if (__any_sync(0xffffffffu, mx[0] > w.m[t][0] + kRescaleLog2 || mx[1] > w.m[t][1] + kRescaleLog2)) {
            float alpha[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float nm = fmaxf(w.m[t][h], mx[h]);
                alpha[h] = nm == w.m[t][h] ? 1.0f : ex2(w.m[t][h] - nm);
                w.l[t][h] *= alpha[h];
                w.m[t][h] = nm;
            }
#pragma unroll
            for (int n = 0; n < D / 16; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) w.o[t][n][e] *= alpha[e & 1];
        }
        const float r0 = w.m[t][0] == neg_inf() ? 0.0f : w.m[t][0];   // a row that has seen nothing keeps P = 0
        const float r1 = w.m[t][1] == neg_inf() ? 0.0f : w.m[t][1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float e0 = ex2(x[2 * h] - r0), e1 = ex2(x[2 * h + 1] - r1);
            w.l[t][0] += e0;
            w.l[t][1] += e1;
            pk[t][h] = transpose8x8(pack_bf16x2(e0, e1));    // from keys by row pairs to rows by key pairs
        }
    }
#pragma unroll
    for (int n = 0; n < D / 16; ++n) {
        const uint32_t c = 2 * n + v_odd;
        uint32_t a[4];
        ldsm4_t(v_at + (c >> 3) * 1024 + (((c & 7) ^ r8) << 4), a);
#pragma unroll
        for (int t = 0; t < T; ++t) mma16816(w.o[t][n], a, pk[t]);
    }
}

// Warp `warp` of a CTA for segments of few rows.  Every warp is a worker of its
// own: it loads its chunks by TMA into its own ring, multiplies them with the
// unit's rows (one or two sets of eight) and writes one partial (m, l, O) per unit that its
// piece of the line touches.
template <int D>
__device__ __forceinline__ void rows_warp(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const PagedParams& p,
                                          uint8_t* smem, const int* cum, const Share& sh, const WaitCtx& wc,
                                          uint32_t warp) {
    using Cfg = RowsCfg<D>;
    constexpr int NS = Cfg::kStages;
    const uint32_t lane = lane_id();
    uint8_t* ring = smem + warp * NS * Cfg::kStage;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Cfg::kBars) + warp * NS;
    const int worker = static_cast<int>(warp) * sh.count + sh.index;
    const int64_t from = static_cast<int64_t>(worker) * sh.per;
    if (from >= sh.total) return;
    const int begin = static_cast<int>(from);
    const int end = static_cast<int>(min(static_cast<int64_t>(sh.total), from + sh.per));

    // ---- loads, up to NS chunks ahead of the products
    Cursor ld;
    seek(p, ld, cum, begin);
    int ld_at = begin;
    int page_base = 0, page_seg = -1, page_id = 0;    // 32 entries of the table, one a lane
    auto load = [&](int stage) {
        const int first = (ld.chunk * kChunk) >> p.block_shift;
        const int in_block = (ld.chunk * kChunk) & ((1 << p.block_shift) - 1);
        const int last = p.block_shift < 4 ? first + 1 : first;
        if (page_seg != ld.seg || first < page_base || last - page_base > 31) {
            page_seg = ld.seg;
            page_base = first;
            const int e = first + static_cast<int>(lane);
            page_id = e < ld.g.blocks ? ld.g.table[e] : p.n_blocks;   // past the end: past the cache, read as zeros
            if (page_id < 0 || (page_id >= p.n_blocks && e < ld.g.blocks)) {
                report(p.status, CR_DEV_INDEX, 912);
                page_id = p.n_blocks;
            }
        }
        const int g0 = ((__shfl_sync(0xffffffffu, page_id, first - page_base) << p.block_shift) + in_block) >> 3;
        const int g1 = (__shfl_sync(0xffffffffu, page_id, last - page_base) << p.block_shift) >> 3;
        uint8_t* dst = ring + stage * Cfg::kStage;
        if (elect_one()) {
            mbar_expect_tx(&full[stage], Cfg::kStage);
            tma_load_4d(dst, &tm_k, &full[stage], 0, 0, ld.head * Cfg::kHalves, g0);
            tma_load_4d(dst + Cfg::kTile, &tm_v, &full[stage], 0, 0, ld.head * Cfg::kHalves, g0);
            if (p.block_shift < 4) {     // blocks of 8: two boxes of 8 rows
                tma_load_4d(dst + Cfg::kTile / 2, &tm_k, &full[stage], 0, 0, ld.head * Cfg::kHalves, g1);
                tma_load_4d(dst + Cfg::kTile + Cfg::kTile / 2, &tm_v, &full[stage], 0, 0, ld.head * Cfg::kHalves, g1);
            }
        }
        __syncwarp();
        if (++ld_at < end) advance(p, ld);
    };
    for (int s = 0; s < NS && ld_at < end; ++s) load(s);

    // ---- products
    Cursor cur;
    seek(p, cur, cum, begin);
    const int kq = static_cast<int>(lane >> 2);
    const int rq = static_cast<int>(lane & 3) * 2;
    RowsState<D, 2> st;
    bool fresh = true;
    int stage = 0, rows = 0;
    uint32_t phase = 0;
    for (int at = begin; at < end; ++at) {
        if (fresh) {
            fresh = false;
            rows = cur.g.nt * p.group;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const int row = 8 * t + kq;
                const bool ok = row < rows;
                const int tok = token_of(p, row);
                const uint16_t* src = p.q + (cur.g.t0 + tok) * p.ldq +
                                      static_cast<int64_t>(cur.head * p.group + row - tok * p.group) * D + rq;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    st.qf[t][k][0] = ok ? *reinterpret_cast<const uint32_t*>(src + 16 * k) : 0u;
                    st.qf[t][k][1] = ok ? *reinterpret_cast<const uint32_t*>(src + 16 * k + 8) : 0u;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // (missing rows compute on zeros and are not written)
                    st.lim[t][h] = 8 * t + rq + h < rows ? row_limit(p, cur.g, 8 * t + rq + h) : cur.g.len;
                    st.m[t][h] = neg_inf();
                    st.l[t][h] = 0.0f;
                }
#pragma unroll
                for (int n = 0; n < D / 16; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) st.o[t][n][e] = 0.0f;
            }
        }
        if (!mbar_wait_warp(&full[stage], phase, wc, 913)) {
            drain_pause();
            return;
        }
        uint8_t* kv = ring + stage * Cfg::kStage;
        const int k0 = cur.chunk * kChunk;
        if (k0 + kChunk > cur.g.len) {
            // the rows of V past the segment's end meet P = 0: they must not hold NaN
            const int from = cur.g.len - k0;
            for (int i = static_cast<int>(lane); i < (kChunk - from) * 8 * Cfg::kHalves; i += 32) {
                const int row = from + i / (8 * Cfg::kHalves);
                const int c = i % (8 * Cfg::kHalves);
                *reinterpret_cast<uint4*>(kv + Cfg::kTile + (row >> 3) * (Cfg::kTile / 2) + (c >> 3) * 1024 +
                                          (row & 7) * 128 + (c & 7) * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async_smem();      // before the stage's next TMA load
            __syncwarp();
        }
        if (rows > 8) rows_chunk<D, 2>(st, smem_u32(kv), smem_u32(kv) + Cfg::kTile, k0, p.scale_log2);
        else rows_chunk<D, 1>(st, smem_u32(kv), smem_u32(kv) + Cfg::kTile, k0, p.scale_log2);
        __syncwarp();                                  // every lane has read the stage
        if (ld_at < end) load(stage);
        if (++stage == NS) {
            stage = 0;
            phase ^= 1u;
        }
        if (at + 1 == end || cur.chunk + 1 == cur.n_chunks) {
            // the piece of this unit ends: its partial
            const int unit = cur.g.unit_base + cur.head;
            const int64_t slot = part_slot<PAGED_ROWS>(p, unit, worker, false);
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                if (8 * t >= rows) break;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) st.l[t][h] += __shfl_xor_sync(0xffffffffu, st.l[t][h], d);
                    const int r = 8 * t + rq + h;
                    if (r < rows) {
                        float* dst = p.part[PAGED_ROWS].o + part_at<PAGED_ROWS, D>(slot * kRowsTile + r, kq);
#pragma unroll
                        for (int n = 0; n < D / 16; ++n) {
                            dst[16 * n] = st.o[t][n][h];
                            dst[16 * n + 8] = st.o[t][n][2 + h];
                        }
                        if (kq == 0) p.part[PAGED_ROWS].ml[slot * kRowsTile + r] = make_float2(st.m[t][h], st.l[t][h]);
                    }
                }
            }
            fresh = true;
        }
        if (at + 1 < end) advance(p, cur);
    }
}

// Log-sum-exp in natural units from a running maximum (log2 units) and sum.  A row
// that has seen nothing, or scores of -inf alone, has m = -inf and l = 0; one whose
// scores are all NaN has m = -inf too, and l = NaN.
__device__ __forceinline__ float finish_lse(float m, float l) { return (m + log2f(l)) * 0.6931471805599453f; }
// What a row's sum of 2^(x - m) v is multiplied by.  Whether the row sees anything is
// told by its keys, not by m or l: 0 / 0 of scores of -inf, and NaN, stay NaN.
__device__ __forceinline__ float finish_scale(bool sees, float l) { return sees ? 1.0f / l : 0.0f; }

// ------------------------------------------------------------------ the kernel
// One CTA per SM.  A call's CTAs are shared out between segments of few rows
// (rows_warp, in every warp) and of many (tiles); both run side by side, as the
// first are bound by memory and the second, often, are not.
//
// A tile CTA takes its part of the line of (unit, 128-key chunk).  A unit's two
// 128-row tiles w = 0, 1 share every K and V tile that is loaded:
//   warp 0       TMA: K_j, V_j of the chunks into a ring, a block of the cache a box
//   warps 1, 2   MMA issue for row tile 0, 1: S_w = Q_w K_j^T, O_w += P_w V_j
//   warp 3       finds the pieces (chunks of one unit), ahead of the others
//   warps 4..7   softmax of row tile 0, one row per thread; they also bring the
//                rows of Q into shared memory and write the results out
//   warps 8..11  the same for row tile 1
// With head_dim 128, O of two row tiles takes half of the 512 TMEM columns and S
// the other half, so that P (bf16) can only take the place of S.  A chunk goes in
// two halves of 64 keys: while the softmax works on one half of S, PV of the half
// before it and then S of that half's successor run.  One thread issues a row
// tile's MMAs, and MMAs of one thread run in order: S_h of chunk j + 1 does not
// overwrite P_h before PV_h of chunk j has read it.
// What bounds it is shared memory: per chunk and row tile, S reads Q twice and K
// (96 KB; MMAs of N = 64 take 386 clocks instead of 256), PV reads V (32 KB), and
// half of the chunk's 64 KB is written by TMA: 2570 clocks of its 128 bytes a
// clock for two row tiles, against 2048 of MMAs; 3150 are measured.  Built and
// timed as well: S in one buffer beside two of P, which takes S off the softmax's
// path but not off shared memory (3540); and, while a block still came in two
// boxes (3530 as it is), S whole with N = 128, softmax and MMAs of a row tile in
// turn (3560), and that with two threads a row (a third slower).
template <int D>
struct TileCfg {
    static constexpr int kHalves = D / 64;                    // 128-byte column halves of a row
    static constexpr uint32_t kHalfBytes = 128 * 128;
    static constexpr uint32_t kTile = kHalves * kHalfBytes;   // one Q, K or V tile
    static constexpr uint32_t kGroup = kHalves * 1024;        // eight rows of a K or V tile: [halves][8][128 bytes]
    static constexpr int kStages = D == 128 ? 5 : 11;
    static constexpr uint32_t kRing = 2 * kTile;
    static constexpr uint32_t kBars = kRing + kStages * kTile;
    static constexpr int kNumBars = 2 * kStages + 2 + 4 + 4 + 2 + 2 + 2 * 2;
    static constexpr uint32_t kPieces = kBars + kNumBars * 8 + 8;
    static constexpr uint32_t kCum = kPieces + 2 * 80;        // (shared by both kinds of CTA)
    static constexpr uint32_t kSums = kCum + ((kCumEntries * 4 + 7) & ~7);
    static constexpr uint32_t kSmem = 1024 + kSums + 12 * 8;
    static constexpr uint32_t kTmemS = 0;                     // S_w at w * 128, half h at + 64 h; P over each half's S
    static constexpr uint32_t kTmemO = 256;                   // O_w at 256 + w * D
};
static_assert(TileCfg<128>::kSmem <= 232448 && TileCfg<64>::kSmem <= 232448, "shared memory of an SM");
static_assert(RowsCfg<128>::kEnd <= TileCfg<128>::kBars && RowsCfg<64>::kEnd <= TileCfg<64>::kBars, "rings over each other");

constexpr int kTileThreads = 384;
constexpr uint32_t kRegsLaunch = 168;     // 65536 / 384
constexpr uint32_t kRegsCtl = 72;
constexpr uint32_t kRegsSoftmax = 216;
static_assert(kRegsCtl * 128 + 2 * kRegsSoftmax * 128 <= kRegsLaunch * kTileThreads,
              "register split exceeds the launch allocation");

// Chunks [j0, j1) of a unit: rows [row0, row0 + kPair) of a segment and one KV head.
struct Piece {
    const int32_t* table;      // the segment's blocks
    int blocks, len;           // the segment's keys
    int t0, rows;              // its query tokens' first, and rows
    int shift;                 // row n sees keys j < min(len, shift + token_of(n)), a prefix's all len
    int head, row0;
    int slot;                  // of the partial, or -1: the unit lies whole in the piece and is finished here
    int j0, j1;
    int turn;                  // chunks are taken in the order j0 + turn .. j1 - 1, j0 .. j0 + turn - 1
    int n_0, n_1;              // chunks of the unit that row tile 0, 1 needs
    int more;                  // 0: no piece, the line is done
    __device__ __forceinline__ int chunks(int w) const { return min(j1, w ? n_1 : n_0) - j0; }
    __device__ __forceinline__ int at(int i) const {      // the i-th chunk taken
        const int j = j0 + turn + i;
        return j < j1 ? j : j - (j1 - j0);
    }
};
static_assert(sizeof(Piece) <= 80, "piece slots");

// The piece that starts at place *line of a CTA's part [begin, end) of the line.
// *line moves past it; it may be empty (the part ends before the unit's chunks).
__device__ __forceinline__ Piece piece_at(const PagedParams& p, const int* cum, const Share& sh, int* line, int begin,
                                          int end) {
    const int at = *line;
    Piece q;
    int seg, start;
    const Segment g = segment_at<PAGED_TILES>(p, cum, at, &seg, &start);
    q.table = g.table;
    q.blocks = g.blocks;
    q.len = g.len;
    q.t0 = g.t0;
    q.rows = g.nt * p.group;
    q.shift = g.own ? g.len - g.nt + 1 : INT32_MAX / 2;
    const int pairs = (q.rows + kPair - 1) / kPair;
    int off = at - start;
    const int per_head = max(1, segment_cost<PAGED_TILES>(p, g) / p.n_kv_heads);
    q.head = min(off / per_head, p.n_kv_heads - 1);
    off -= q.head * per_head;
    int t, n_unit;
    if (!g.own) {
        n_unit = (g.len + kKeys - 1) / kKeys;
        t = min(off / (n_unit + kUnitCost), pairs - 1);
        off -= t * (n_unit + kUnitCost);
    } else {
        for (t = 0;; ++t) {
            n_unit = chunks_of(p, g, t * kPair, kPair, kKeys);
            const int n = n_unit ? n_unit + kUnitCost : 0;
            if (off < n || t + 1 == pairs) break;
            off -= n;
        }
    }
    const int take = max(1, min(n_unit + kUnitCost - off, end - at));
    *line = at + take;
    q.row0 = t * kPair;
    q.j0 = min(max(0, off - kUnitCost), n_unit);
    q.j1 = min(max(0, off + take - kUnitCost), n_unit);
    q.n_0 = chunks_of(p, g, q.row0, 128, kKeys);
    q.n_1 = q.row0 + 128 < q.rows ? chunks_of(p, g, q.row0 + 128, 128, kKeys) : 0;
    const bool whole = q.j0 == 0 && q.j1 == n_unit && p.n_groups == 0;
    q.slot = whole ? -1
                   : static_cast<int>(part_slot<PAGED_TILES>(p, g.unit_base + q.head * pairs + t, sh.index, at == begin));
    // The row tiles of a prefix read the same keys, in different CTAs and cut in
    // different places.  Each takes chunk j at step j mod per of its work, so that
    // they read it at the same time, once from memory.
    q.turn = 0;
    if (!g.own && pairs > 1) {
        const int turn = (sh.per - q.j0 % sh.per) % sh.per;
        if (turn < q.j1 - q.j0) q.turn = turn;
    }
    q.more = 1;
    return q;
}

// 32 bytes from eight registers.
__device__ __forceinline__ void store_f8(float* dst, const float* v) {
    asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "f"(v[0]), "f"(v[1]), "f"(v[2]),
                 "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7])
                 : "memory");
}

// kRows, kTiles: the kinds of segment that the call has.  One kernel for both would
// do (a CTA finds its kind in the schedule), but with code of one kind alone it
// is faster: 4 rows of 16 requests over 3 to 9k tokens 47.5 us -> 44.0, a decode step
// of 5120 tokens 10.6 -> 9.9, 40 questions 82.9 -> 80.1, a prompt 224.5 -> 221.6.
template <int D, bool kRows, bool kTiles>
__global__ void __launch_bounds__(kTileThreads, 1)
    paged_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                 const __grid_constant__ CUtensorMap tm_k16, const __grid_constant__ CUtensorMap tm_v16,
                 const __grid_constant__ PagedParams p) {
    using Cfg = TileCfg<D>;
    constexpr int NS = Cfg::kStages;
    constexpr uint32_t IDESC_S = idesc_bf16(128, 64, false, false);
    constexpr uint32_t IDESC_PV = idesc_bf16(128, D, false, true);
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                               ~static_cast<uintptr_t>(1023));
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Cfg::kBars);   // ring stage loaded
    uint64_t* empty = full + NS;      // both issuers are done with it
    uint64_t* q_full = empty + NS;    // [2] rows of Q in shared memory
    uint64_t* s_full = q_full + 2;    // [2][2] half h of S_w in TMEM
    uint64_t* p_full = s_full + 4;    // [2][2] half h of P_w in TMEM
    uint64_t* o_step = p_full + 4;    // [2] O_w holds one more half
    uint64_t* o_full = o_step + 2;    // [2] O_w complete for the piece
    uint64_t* piece_full = o_full + 2;        // [2]
    uint64_t* piece_empty = piece_full + 2;   // [2]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(piece_empty + 2);
    int* abort_flag = reinterpret_cast<int*>(tmem_slot + 1);
    Piece* pieces = reinterpret_cast<Piece*>(smem + Cfg::kPieces);
    int* cum = reinterpret_cast<int*>(smem + Cfg::kCum);
    int64_t* warp_sum = reinterpret_cast<int64_t*>(smem + Cfg::kSums);

    const uint32_t warp = warp_id(), lane = lane_id();
    if (kRows && lane == 0) {
        uint64_t* bars = reinterpret_cast<uint64_t*>(smem + RowsCfg<D>::kBars) + warp * RowsCfg<D>::kStages;
        for (int s = 0; s < RowsCfg<D>::kStages; ++s) mbar_init(&bars[s], 1);
        fence_barrier_init();
    }
    if (threadIdx.x == 0) *abort_flag = 0;
    if (kTiles && threadIdx.x == 0) {
        for (int s = 0; s < NS; ++s) {
            mbar_init(&full[s], 1);
            mbar_init(&empty[s], 2);
        }
        for (int w = 0; w < 2; ++w) {
            mbar_init(&q_full[w], 4);
            mbar_init(&o_step[w], 1);
            mbar_init(&o_full[w], 1);
            mbar_init(&piece_full[w], 1);
            mbar_init(&piece_empty[w], 11);      // every warp but warp 3
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&s_full[i], 1);
            mbar_init(&p_full[i], 4);
        }
        fence_barrier_init();
    }
    if (kTiles && warp == 1) tmem_alloc(tmem_slot, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    pdl_wait();
    // The join's blocks start as SMs fall idle and read what earlier kernels have left:
    // not before those are complete.
    pdl_launch_dependents();
    const Share sh = schedule<kRows, kTiles>(p, cum, warp_sum);
    const uint32_t tmem = *tmem_slot;
    const WaitCtx wc{abort_flag, p.status};
    // The i-th piece, for every warp but warp 3; a warp gives it back once read.
    auto next_piece = [&](uint32_t i, Piece* q) -> bool {
        if (!mbar_wait_warp(&piece_full[i & 1u], (i >> 1) & 1u, wc, 930)) return false;
        *q = pieces[i & 1u];
        __syncwarp();
        if (lane == 0) mbar_arrive(&piece_empty[i & 1u]);
        return q->more != 0;
    };

    if (kRows && !(kTiles && sh.tiles)) {
        rows_warp<D>(tm_k16, tm_v16, p, smem, cum, sh, wc, warp);
    } else if constexpr (!kTiles) {
    } else if (warp < 4) {
        setmaxnreg_dec<kRegsCtl>();
        if (warp == 3) {
            // ------------------------------------------------ pieces
            const int64_t from = static_cast<int64_t>(sh.index) * sh.per;
            const int begin = static_cast<int>(min(static_cast<int64_t>(sh.total), from));
            const int end = static_cast<int>(min(static_cast<int64_t>(sh.total), from + sh.per));
            int at = begin;
            for (uint32_t i = 0;; ++i) {
                Piece q;
                q.more = 0;
                while (at < end) {
                    q = piece_at(p, cum, sh, &at, begin, end);
                    if (q.j1 > q.j0) break;
                    q.more = 0;
                }
                if (!mbar_wait_warp(&piece_empty[i & 1u], ((i >> 1) & 1u) ^ 1u, wc, 931)) break;
                if (lane == 0) {
                    pieces[i & 1u] = q;
                    mbar_arrive(&piece_full[i & 1u]);
                }
                __syncwarp();
                if (!q.more) break;
            }
        } else if (warp == 0) {
            // ------------------------------------------------ loads
            // A tile of 128 keys is boxes of min(block, 128) rows; each lane issues one
            // box of K, later of V, from the block that its table entry names.  Entries
            // past the sequence point past the cache, where a box reads zeros.
            const int box_shift = min(p.block_shift, 7);
            const int sub = static_cast<int>(lane);                      // box of the tile
            const uint32_t box_at = (static_cast<uint32_t>(sub) << box_shift) * (Cfg::kHalves * 128);
            const bool mine = sub < (kKeys >> box_shift);
            auto row_of = [&](const Piece& q, int j) -> int {
                const int key = j * kKeys + (sub << box_shift);
                const int e = key >> p.block_shift;
                int id = mine && e < q.blocks ? q.table[e] : p.n_blocks;
                if (id < 0 || (id >= p.n_blocks && mine && e < q.blocks)) {
                    report(p.status, CR_DEV_INDEX, 914);
                    id = p.n_blocks;
                }
                return (id << p.block_shift) + (id == p.n_blocks ? 0 : key & ((1 << p.block_shift) - 1));
            };
            uint32_t st = 0, ph = 1;  // next ring stage, and the parity of its last release
            bool ok = true;
            Piece q;
            for (uint32_t i = 0; ok && next_piece(i, &q); ++i) {
                int row = row_of(q, q.at(0));
                const int steps = q.j1 - q.j0;
                for (int k = 0; k < steps && ok; ++k) {
                    const int row_now = row;
                    if (k + 1 < steps) row = row_of(q, q.at(k + 1));      // in flight while this tile waits
#pragma unroll 1
                    for (int kv = 0; kv < 2; ++kv) {
                        if (!(ok = mbar_wait_warp(&empty[st], ph, wc, 921))) break;
                        uint8_t* dst = smem + Cfg::kRing + st * Cfg::kTile;
                        if (lane == 0) mbar_expect_tx(&full[st], Cfg::kTile);
                        __syncwarp();
                        if (mine) tma_load_4d(dst + box_at, kv ? &tm_v : &tm_k, &full[st], 0, 0, q.head * Cfg::kHalves, row_now >> 3);
                        __syncwarp();
                        if (++st == NS) {
                            st = 0;
                            ph ^= 1u;
                        }
                    }
                }
            }
            if (!ok) drain_pause();
        } else {
            // ------------------------------------------------ MMA issue
            const int w = static_cast<int>(warp) - 1;
            const uint64_t dq = smem_desc(smem_u32(smem + w * Cfg::kTile), 16, 1024, SWZ_128B);
            const uint64_t dk0 = smem_desc(smem_u32(smem + Cfg::kRing), 16, Cfg::kGroup, SWZ_128B);
            const uint64_t dv0 = smem_desc(smem_u32(smem + Cfg::kRing), 1024, Cfg::kGroup, SWZ_128B);
            const uint32_t ds = tmem + Cfg::kTmemS + w * 128;
            const uint32_t dout = tmem + Cfg::kTmemO + w * D;
            uint32_t st = 0, ph = 0;  // ring stage that comes next, and its parity
            auto step = [&]() {
                if (++st == NS) {
                    st = 0;
                    ph ^= 1u;
                }
            };
            uint32_t nq = 0, np = 0;  // pieces and chunks done
            bool ok = true;
            // keys 64 h .. 64 h + 63 of the K tile in stage `sk`
            auto issue_s = [&](uint32_t sk, int h) {
                const uint64_t dk = dk0 + static_cast<uint64_t>(sk) * (Cfg::kTile >> 4) + h * (8 * Cfg::kGroup >> 4);
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        mma_bf16_ss(ds + 64 * h, dq + (k >> 2) * (Cfg::kHalfBytes >> 4) + (k & 3) * 2,
                                    dk + (k >> 2) * (1024 >> 4) + (k & 3) * 2, IDESC_S, k != 0 ? 1u : 0u);
                    }
                    mma_commit(&s_full[2 * w + h]);
                    if (h == 1) mma_commit(&empty[sk]);
                }
                __syncwarp();
            };
            auto wait_full = [&](unsigned site) -> bool {
                if (!mbar_wait_warp(&full[st], ph, wc, site)) return false;
                tc_fence_after();
                return true;
            };
            Piece q;
            for (uint32_t i = 0; ok && next_piece(i, &q); ++i) {
                const int n = q.chunks(w);                // this row tile's chunks of the piece
                if (n > 0) {
                    ok = mbar_wait_warp(&q_full[w], nq & 1u, wc, 923) && wait_full(922);
                    ++nq;
                    if (ok) {
                        tc_fence_after();
                        issue_s(st, 0);
                        issue_s(st, 1);
                        step();
                    }
                    for (int j = 0; j < n && ok; ++j, ++np) {
                        if (!(ok = wait_full(924))) break;
                        const uint32_t sv = st;
                        step();
                        const int past = (q.at(j) + 1) * kKeys - q.len;
                        if (past > 0) {
                            // keys past the segment's end meet P = 0: their V must not be NaN.
                            // (Both issuers may write these zeros; neither reads anything else.)
                            uint8_t* v = smem + Cfg::kRing + sv * Cfg::kTile;
                            for (int k = static_cast<int>(lane); k < past * 8 * Cfg::kHalves; k += 32) {
                                const int row = kKeys - 1 - k / (8 * Cfg::kHalves);
                                const int c = k % (8 * Cfg::kHalves);
                                *reinterpret_cast<uint4*>(v + (row >> 3) * Cfg::kGroup + (c >> 3) * 1024 + (row & 7) * 128 +
                                                          (c & 7) * 16) = make_uint4(0, 0, 0, 0);
                            }
                            fence_async_smem();
                            __syncwarp();
                        }
                        const uint64_t dv = dv0 + static_cast<uint64_t>(sv) * (Cfg::kTile >> 4);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if (!(ok = mbar_wait_warp(&p_full[2 * w + h], np & 1u, wc, 925))) break;
                            tc_fence_after();
                            if (elect_one()) {
#pragma unroll
                                for (int k = 0; k < 4; ++k)      // 16 keys: 8 columns of P, two groups of V
                                    mma_bf16_ts(dout, ds + 64 * h + 8 * k, dv + (4 * h + k) * (2 * Cfg::kGroup >> 4), IDESC_PV,
                                                (j > 0 || h != 0 || k != 0) ? 1u : 0u);
                                mma_commit(&o_step[w]);
                                if (h == 1) {
                                    mma_commit(&empty[sv]);
                                    if (j + 1 == n) mma_commit(&o_full[w]);
                                }
                            }
                            __syncwarp();
                            if (j + 1 < n) {
                                if (h == 0 && !(ok = wait_full(922))) break;
                                issue_s(st, h);
                                if (h == 1) step();
                            }
                        }
                    }
                }
                // Chunks that only the other row tile needs: wait for them all the same, so
                // that every wait stays within one phase of its barrier.
                for (int k = 2 * max(n, 0); k < 2 * (q.j1 - q.j0) && ok; ++k) {
                    ok = wait_full(928);
                    if (ok && elect_one()) mbar_arrive(&empty[st]);
                    __syncwarp();
                    step();
                }
            }
            if (!ok) drain_pause();
        }
    } else {
        setmaxnreg_inc<kRegsSoftmax>();
        // ---------------------------------------------------- softmax
        const int w = warp >= 8 ? 1 : 0;
        const int r = static_cast<int>((warp & 3u) * 32 + lane);     // row of the tile
        const uint32_t lane_off = ((warp & 3u) * 32u) << 16;
        const uint32_t ts = tmem + lane_off + Cfg::kTmemS + w * 128;
        const uint32_t to = tmem + lane_off + Cfg::kTmemO + w * D;
        const float sc = p.scale_log2;
        uint32_t ns = 0, no = 0;        // chunks and pieces done
        bool ok = true;
        // This warp's rows of a piece's Q into shared memory, swizzled as the MMA reads
        // them (kLanes lanes read a row together), once the MMAs of the piece before
        // on this tile are complete: this group has seen their S.
        auto load_q = [&](const Piece& q) {
            if (q.chunks(w) <= 0) return;
            constexpr int kLanes = 8 * Cfg::kHalves;
            const int row = q.row0 + 128 * w + r, tok = token_of(p, row);
            // (a row past the unit's last takes the first's values: it is not written)
            const int64_t mine = row < q.rows ? static_cast<int64_t>(q.t0 + tok) * p.ldq +
                                                    static_cast<int64_t>(q.head * p.group + row - tok * p.group) * D
                                              : static_cast<int64_t>(q.t0) * p.ldq;
            uint8_t* dst = smem + w * Cfg::kTile;
            const int c = static_cast<int>(lane) % kLanes;
            uint4 v[kLanes];
#pragma unroll
            for (int k = 0; k < kLanes; ++k) {
                const int64_t at = __shfl_sync(0xffffffffu, mine, k * (32 / kLanes) + static_cast<int>(lane) / kLanes);
                v[k] = *reinterpret_cast<const uint4*>(p.q + at + c * 8);
            }
#pragma unroll
            for (int k = 0; k < kLanes; ++k) {
                const int rr = static_cast<int>((warp & 3u) * 32) + k * (32 / kLanes) + static_cast<int>(lane) / kLanes;
                *reinterpret_cast<uint4*>(dst + (c >> 3) * Cfg::kHalfBytes + rr * 128 + (((c & 7) ^ (rr & 7)) << 4)) = v[k];
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_full[w]);
        };
        Piece q;
        bool more = next_piece(0, &q);
        if (more) load_q(q);
        for (uint32_t i = 0; ok && more; ++i) {
            const int row = q.row0 + 128 * w + r;
            const bool valid = row < q.rows;
            const bool live = __any_sync(0xffffffffu, valid);
            // (rows past the unit's last compute on the first row's Q and are not written)
            const int lim = valid ? max(0, min(q.len, q.shift + token_of(p, row))) : INT32_MAX;
            const int n = q.chunks(w);
            float m = neg_inf(), l = 0.0f;
            for (int k = 0; k < 2 * n; ++k) {
                const int h = k & 1;
                ok = mbar_wait(&s_full[2 * w + h], ns & 1u, wc, 926);
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                if (live) {                 // (a warp without rows: its lanes of P are never read out)
                    tc_fence_after();
                    float s[64];
                    tmem_ld32(ts + 64 * h, s);
                    tmem_ld32(ts + 64 * h + 32, s + 32);
                    tmem_wait_ld();
                    const int hi = lim - (q.at(k >> 1) * kKeys + 64 * h);       // keys of this half that the row sees
                    if (__any_sync(0xffffffffu, hi < 64)) {
#pragma unroll
                        for (int e = 0; e < 64; ++e) s[e] = e < hi ? s[e] : neg_inf();
                    }
                    float mxv[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) mxv[e] = fmaxf(s[2 * e], s[2 * e + 1]);
#pragma unroll
                    for (int e = 16; e < 64; e += 2) mxv[(e >> 1) & 7] = fmax3(mxv[(e >> 1) & 7], s[e], s[e + 1]);
                    const float mx = sc * fmaxf(fmax3(mxv[0], mxv[1], mxv[2]),
                                                fmax3(fmax3(mxv[3], mxv[4], mxv[5]), mxv[6], mxv[7]));
                    // move the reference on the first half, or when this one would push P
                    // past 2^8 (any reference gives the same quotient O / l)
                    if (__any_sync(0xffffffffu, k == 0 || mx > m + kRescaleLog2)) {
                        const float nm = fmaxf(m, mx);
                        if (k > 0) {
                            // O up to the half before this one (S of this half was issued
                            // behind the PV before that, so the wait is within a phase)
                            ok = mbar_wait(&o_step[w], (2 * ns + h + 1) & 1u, wc, 927);
                            if (!(ok = __all_sync(0xffffffffu, ok))) break;
                            tc_fence_after();
                            const float alpha = m == nm ? 1.0f : ex2(m - nm);
#pragma unroll 1
                            for (int c = 0; c < D; c += 16) {
                                float o[16];
                                tmem_ld16(to + c, o);
                                tmem_wait_ld();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] *= alpha;
                                tmem_st16(to + c, o);
                            }
                            l *= alpha;
                        }
                        m = nm;
                    }
                    const float ref = m == neg_inf() ? 0.0f : m;    // a row that has seen nothing keeps P = 0
                    float sum[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
                    uint32_t pk[32];
#pragma unroll
                    for (int e = 0; e < 64; e += 2) {
                        float t0, t1;
                        ffma2(t0, t1, s[e], s[e + 1], sc, sc, -ref, -ref);
                        const float e0 = ex2(t0), e1 = ex2(t1);
                        const int b = (e >> 1) & 3;
                        fadd2(sum[2 * b], sum[2 * b + 1], sum[2 * b], sum[2 * b + 1], e0, e1);
                        pk[e >> 1] = pack_bf16x2(e0, e1);
                    }
                    tmem_st32u(ts + 64 * h, pk);
                    l += ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                }
                if (lane == 0) mbar_arrive(&p_full[2 * w + h]);
                if (h == 1) ++ns;
            }
            if (!ok) break;
            // the next piece's S can run beside what is left of this one
            Piece after;
            more = next_piece(i + 1, &after);
            if (more) load_q(after);
            if (n > 0) {
                ok = mbar_wait(&o_full[w], no & 1u, wc, 929);
                ++no;
                if (!(ok = __all_sync(0xffffffffu, ok))) break;
                tc_fence_after();
            }
            if (q.slot < 0) {
                const int tok = token_of(p, row);
                const int64_t t = q.t0 + tok;
                const int qh = q.head * p.group + row - tok * p.group;
                const float inv = finish_scale(lim > 0, l);
                if (valid && p.lse) p.lse[t * p.n_q_heads + qh] = finish_lse(m, l);
                uint16_t* dst = p.out + t * p.ldo + static_cast<int64_t>(qh) * D;
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    if (n > 0) {
                        tmem_ld32(to + c, o);
                        tmem_wait_ld();
                    }
                    if (valid) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t u[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                u[k] = lim <= 0 ? 0u : pack_bf16x2(o[8 * e + 2 * k] * inv, o[8 * e + 2 * k + 1] * inv);
                            *reinterpret_cast<uint4*>(dst + c + 8 * e) = make_uint4(u[0], u[1], u[2], u[3]);
                        }
                    }
                }
            } else {
                const int64_t slot = static_cast<int64_t>(q.slot) * kPair + 128 * w + r;
                if (valid) p.part[PAGED_TILES].ml[slot] = make_float2(m, l);
                if (n > 0 && live) {
                    float* dst = p.part[PAGED_TILES].o + part_at<PAGED_TILES, D>(slot, 0);
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        tmem_ld32(to + c, o);
                        tmem_wait_ld();
                        if (valid) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) store_f8(dst + (c + 8 * e) * 128, o + 8 * e);
                        }
                    }
                }
            }
            tc_fence_before();      // O_w read before this group's next P is seen
            q = after;
        }
    }
    __syncthreads();
    if (kTiles && warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ------------------------------------------------------------------ join
// Where the rows of one KV head of one segment have their partials: those of a
// unit's row r are part_entry(.., i, r), i < n.
struct UnitParts {
    int n, w0, per, a, number, size;
    bool tiles, finished;
};
struct SegmentLine {
    const PagedPart* part;
    int t0, nt, len, unit_base;
    int first, per, per_mul, per_shift, size, units;       // units of one head
    bool tiles, own;
    // whether query token t of the segment sees any of its keys
    __device__ __forceinline__ bool sees(int t) const { return own ? len - nt + (t - t0) + 1 > 0 : len > 0; }
};
// What the join needs of a segment: first what was there before the main kernel,
// then the line that it has published, with the lengths that it was made from; each
// with its loads side by side.
__device__ __forceinline__ SegmentLine segment_shape(const PagedParams& p, int s) {
    SegmentLine x;
    x.own = s >= p.n_groups;
    const int4 d = p.seg[s];
    x.t0 = d.x;
    x.nt = d.y;
    x.unit_base = d.z;
    x.tiles = d.w == PAGED_TILES;
    x.part = &p.part[x.tiles ? PAGED_TILES : PAGED_ROWS];
    x.size = x.tiles ? kPair : kRowsTile;
    x.units = (x.nt * p.group + x.size - 1) / x.size;
    return x;
}
__device__ __forceinline__ void segment_line(SegmentLine& x, int s) {
    const int* sched = x.part->sched;
    const int2 mine = reinterpret_cast<const int2*>(sched)[s];
    x.first = mine.x;
    x.len = mine.y;
    x.per = sched[kSchedPer];
    x.per_mul = sched[kSchedPer + 1];
    x.per_shift = sched[kSchedPer + 2];
}
__device__ __forceinline__ int div_per(const SegmentLine& x, int n) {
    return static_cast<int>((__umulhi(static_cast<uint32_t>(x.per_mul), static_cast<uint32_t>(n)) +
                             static_cast<uint32_t>(n)) >> x.per_shift);
}
__device__ __forceinline__ UnitParts unit_parts(const PagedParams& p, const SegmentLine& x, int head, int unit) {
    UnitParts u;
    u.tiles = x.tiles;
    u.size = x.size;
    u.per = x.per;
    // the unit's chunks [a + c, a + c + n) of the line, behind the c of its start
    const int c = x.tiles ? kUnitCost : 0;
    int n;
    if (!x.tiles || !x.own) {
        n = x.tiles ? (x.len + kKeys - 1) / kKeys : (x.len + kChunk - 1) / kChunk;
        u.a = (head * x.units + unit) * (n + c);
    } else {
        const int2* line = x.part->unit + x.unit_base;
        const int2 mine = line[unit], last = line[x.units - 1];
        n = mine.y;
        u.a = head * (last.x + (last.y ? last.y + c : 0)) + mine.x;
    }
    u.a += x.first;
    u.number = x.unit_base + head * x.units + unit;
    u.w0 = div_per(x, u.a + c);
    u.n = n ? div_per(x, u.a + c + n - 1) - u.w0 + 1 : 0;
    u.finished = x.tiles && u.n == 1 && p.n_groups == 0;           // by the main kernel
    return u;
}
__device__ __forceinline__ int64_t part_entry(const PagedParams& p, const UnitParts& u, int i, int r) {
    const int w = u.w0 + i;
    const int64_t slot = u.tiles ? part_slot<PAGED_TILES>(p, u.number, w, w * u.per >= u.a)
                                 : part_slot<PAGED_ROWS>(p, u.number, w, false);
    return slot * u.size + r;
}

// Few rows, each perhaps of many partials: a CTA of W warps per (token, query
// head).  The warps share the row's partials; W * 32 at a time their maxima are
// gathered first, so that the loads of O do not wait for one another: twelve a warp
// are in flight (with four a decode step of 5120 tokens takes 1.8 us longer).
template <int D, int W, bool kPrefix>
__global__ void __launch_bounds__(W * 32) join_few_kernel(const __grid_constant__ PagedParams p) {
    constexpr int V = D / 32;
    constexpr int NT = W * 32;
    constexpr int kDeep = 12;
    __shared__ float weight[NT];
    __shared__ const float* base[NT];
    __shared__ bool tiles[NT];
    __shared__ float red[2][W];
    __shared__ float sums[W][D];
    pdl_launch_dependents();
    const int t = static_cast<int>(blockIdx.x / p.n_q_heads);
    const int qh = static_cast<int>(blockIdx.x - t * p.n_q_heads);
    const int head = token_of(p, qh);                    // qh / group
    const int lane = static_cast<int>(lane_id()), warp = static_cast<int>(warp_id());
    const int2 seg = p.token[t];
    SegmentLine x[2];
    x[0] = segment_shape(p, seg.x);
    x[1] = kPrefix ? segment_shape(p, seg.y) : x[0];
    pdl_wait();
    segment_line(x[0], seg.x);
    if (kPrefix) segment_line(x[1], seg.y);
    else x[1] = x[0];
    UnitParts u[2];
    int r[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int row = (t - x[k].t0) * p.group + qh - head * p.group;
        const int unit = x[k].tiles ? row / kPair : row / kRowsTile;
        u[k] = unit_parts(p, x[k], head, unit);
        r[k] = row - unit * x[k].size;
    }
    if (!kPrefix) u[1].n = 0;
    if (u[0].finished) return;
    const bool sees = x[0].sees(t) || (kPrefix && x[1].sees(t));
    const int n = u[0].n + u[1].n;
    float acc[V] = {};
    float m = neg_inf(), l = 0.0f;
    for (int i0 = 0; i0 < n; i0 += NT) {
        const int i = i0 + static_cast<int>(threadIdx.x);
        float2 ml = make_float2(neg_inf(), 0.0f);
        if (i < n) {
            const bool own = !kPrefix || i < u[0].n;
            const int64_t e = own ? part_entry(p, u[0], i, r[0]) : part_entry(p, u[1], i - u[0].n, r[1]);
            const PagedPart& part = own ? *x[0].part : *x[1].part;
            const bool tile = own ? u[0].tiles : u[1].tiles;
            ml = part.ml[e];
            base[threadIdx.x] = part.o + (tile ? part_at<PAGED_TILES, D>(e, 0) : part_at<PAGED_ROWS, D>(e, 0));
            tiles[threadIdx.x] = tile;
        }
        float mx = ml.x;
#pragma unroll
        for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        if (lane == 0) red[0][warp] = mx;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < W; ++k) mx = fmaxf(mx, red[0][k]);
        const float nm = fmaxf(m, mx);
        const float ref = nm == neg_inf() ? 0.0f : nm;
        const float w = ex2(ml.x - ref);                 // 0 for what a row has not seen
        weight[threadIdx.x] = w;
        float sum = w * ml.y;
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) red[1][warp] = sum;
        __syncthreads();
        const float f = ex2(m - ref);
        l *= f;
#pragma unroll
        for (int k = 0; k < W; ++k) l += red[1][k];
        m = nm;
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] *= f;
        const int most = min(NT, n - i0);
        for (int k0 = warp; k0 < most; k0 += W * kDeep) {
            float o[kDeep][V], g[kDeep];
#pragma unroll
            for (int j = 0; j < kDeep; ++j) {
                const int k = k0 + j * W;
                g[j] = k < most ? weight[k] : 0.0f;
                // (an unseen part's O may never have been written)
                const float* src = g[j] != 0.0f ? base[k] + (tiles[k] ? part_at<PAGED_TILES, D>(0, lane * V) : lane * V) : nullptr;
                if (V == 4) *reinterpret_cast<float4*>(o[j]) = src ? *reinterpret_cast<const float4*>(src) : float4{};
                else *reinterpret_cast<float2*>(o[j]) = src ? *reinterpret_cast<const float2*>(src) : float2{};
            }
#pragma unroll
            for (int j = 0; j < kDeep; ++j)
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] += g[j] * o[j][v];
        }
        __syncthreads();
    }
#pragma unroll
    for (int v = 0; v < V; ++v) sums[warp][lane * V + v] = acc[v];
    __syncthreads();
    if (static_cast<int>(threadIdx.x) < D / 2) {
        const float inv = finish_scale(sees, l);
        const int c = threadIdx.x * 2;
        float o[2] = {0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < W; ++k) {
            o[0] += sums[k][c];
            o[1] += sums[k][c + 1];
        }
        *reinterpret_cast<uint32_t*>(p.out + t * p.ldo + static_cast<int64_t>(qh) * D + c) =
            pack_bf16x2(o[0] * inv, o[1] * inv);
    }
    if (p.lse && threadIdx.x == 0) p.lse[blockIdx.x] = finish_lse(m, l);
}

// A warp per (token, query head): each lane takes one partial's maximum and sum,
// and sixteen partials' O are in flight together.
template <int D, bool kPrefix>
__global__ void __launch_bounds__(128) join_kernel(const __grid_constant__ PagedParams p) {
    constexpr int V = D / 32;
    constexpr int kDeep = 16;
    pdl_launch_dependents();
    const int64_t w = blockIdx.x * 4ll + warp_id();
    if (w >= static_cast<int64_t>(p.n_tokens) * p.n_q_heads) {
        pdl_wait();
        return;
    }
    const int lane = static_cast<int>(lane_id());
    const int t = static_cast<int>(w / p.n_q_heads);
    const int qh = static_cast<int>(w - static_cast<int64_t>(t) * p.n_q_heads);
    const int head = token_of(p, qh);                    // qh / group
    const int2 seg = p.token[t];
    SegmentLine x[2];
    x[0] = segment_shape(p, seg.x);
    x[1] = kPrefix ? segment_shape(p, seg.y) : x[0];
    pdl_wait();
    segment_line(x[0], seg.x);
    if (kPrefix) segment_line(x[1], seg.y);
    else x[1] = x[0];
    UnitParts u[2];
    const PagedPart* part[2];
    int r[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int row = (t - x[k].t0) * p.group + qh - head * p.group;
        const int unit = x[k].tiles ? row / kPair : row / kRowsTile;
        u[k] = unit_parts(p, x[k], head, unit);
        r[k] = row - unit * x[k].size;
        part[k] = x[k].part;
    }
    if (!kPrefix) u[1].n = 0;
    if (u[0].finished) return;
    const bool sees = x[0].sees(t) || (kPrefix && x[1].sees(t));
    const int n = u[0].n + u[1].n;
    float acc[V] = {};
    float m = neg_inf(), l = 0.0f;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int i = i0 + lane;
        float2 ml = make_float2(neg_inf(), 0.0f);
        const float* base = nullptr;
        if (i < n) {
            const int k = !kPrefix || i < u[0].n ? 0 : 1;
            const int64_t e = k ? part_entry(p, u[1], i - u[0].n, r[1]) : part_entry(p, u[0], i, r[0]);
            const PagedPart& x = k ? *part[1] : *part[0];
            ml = x.ml[e];
            base = x.o + ((k ? u[1].tiles : u[0].tiles) ? part_at<PAGED_TILES, D>(e, 0) : part_at<PAGED_ROWS, D>(e, 0));
        }
        float mx = ml.x;
#pragma unroll
        for (int o = 16; o; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        const float nm = fmaxf(m, mx);
        const float ref = nm == neg_inf() ? 0.0f : nm;
        const float g = ex2(ml.x - ref);                 // 0 for what a row has not seen
        float sum = g * ml.y;
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const float f = ex2(m - ref);
        l = l * f + sum;
        m = nm;
#pragma unroll
        for (int v = 0; v < V; ++v) acc[v] *= f;
        const int most = min(32, n - i0);
        for (int k0 = 0; k0 < most; k0 += kDeep) {
            float o[kDeep][V];
            float gk[kDeep];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) {
                gk[k] = __shfl_sync(0xffffffffu, g, k0 + k);
                const float* src = reinterpret_cast<const float*>(
                    __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(base), k0 + k));
                // (an unseen part's O may never have been written)
                const bool seen = k0 + k < most && gk[k] != 0.0f;
                src += (!kPrefix || i0 + k0 + k < u[0].n ? u[0].tiles : u[1].tiles) ? part_at<PAGED_TILES, D>(0, lane * V) : lane * V;
                if (V == 4) *reinterpret_cast<float4*>(o[k]) = seen ? *reinterpret_cast<const float4*>(src) : float4{};
                else *reinterpret_cast<float2*>(o[k]) = seen ? *reinterpret_cast<const float2*>(src) : float2{};
            }
#pragma unroll
            for (int k = 0; k < kDeep; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v] += gk[k] * o[k][v];
        }
    }
    const float inv = finish_scale(sees, l);
    uint16_t* dst = p.out + t * p.ldo + static_cast<int64_t>(qh) * D + lane * V;
    if (V == 4)
        *reinterpret_cast<uint2*>(dst) =
            make_uint2(pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[V - 2] * inv, acc[V - 1] * inv));
    else
        *reinterpret_cast<uint32_t*>(dst) = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    if (p.lse && lane == 0) p.lse[w] = finish_lse(m, l);
}

// Many rows, each of a few partials: a warp per four rows of a request and KV
// head, eight lanes a row, which find its partials and bring their maxima and sums;
// then each lane adds up a quarter of a row's O, so that a load takes whole lines of
// four neighbouring rows in the tiles' layout.  Rows that the main kernel has
// finished are left alone.  The loads wait for one another three or four deep, so many
// warps have to be resident: 8 CTAs of 64 registers an SM, 6 of 80 with prefixes; or,
// of fewer rows, kDeep partials' O in flight.
// (160 requests of 20 to 40 tokens over four prefixes, 3 partials a row: 268 us, 277 with
// all lanes on one row at a time and 4 CTAs, 264 with 8, where 8192 rows of 7 lose 2.)
template <int D, bool kPrefix, int kDeep>
__global__ void __launch_bounds__(128, kDeep > 1 ? 2 : kPrefix ? 6 : 8)
    join_blocks_kernel(const __grid_constant__ PagedParams p) {
    constexpr int R = kBlockRows, K = D / 32;
    static_assert(8 % kDeep == 0, "eight partials at a time");
    pdl_launch_dependents();
    const int b = static_cast<int>(blockIdx.x * 4 + warp_id());
    if (b >= p.n_row_blocks) {
        pdl_wait();
        return;
    }
    const int lane = static_cast<int>(lane_id());
    // columns 4 c .. 4 c + 3 of O's row `q`, c = col + 8 k: a load of a warp takes whole lines
    const int q = (lane >> 1) & 3, col = (lane >> 3) * 2 + (lane & 1);
    const int4 at = p.row_block[b];                      // own segment, prefix segment or -1, KV head, first row
    SegmentLine x0 = segment_shape(p, at.x), x1 = kPrefix ? segment_shape(p, at.y) : x0;
    const int rows = min(R, x0.nt * p.group - at.w), t0 = x0.t0;
    const int mine = min(lane >> 3, rows - 1);           // this lane's row
    pdl_wait();
    segment_line(x0, at.x);
    if (kPrefix) segment_line(x1, at.y);
    int row0 = at.w + mine, row1 = row0 + (kPrefix ? (t0 - x1.t0) * p.group : 0);
    const int unit0 = x0.tiles ? row0 / kPair : row0 / kRowsTile, unit1 = x1.tiles ? row1 / kPair : row1 / kRowsTile;
    const UnitParts u0 = unit_parts(p, x0, at.z, unit0);
    if (u0.finished) return;                             // (the rows lie in one unit)
    const int t = t0 + token_of(p, row0);
    const bool sees = x0.sees(t) || (kPrefix && x1.sees(t));
    UnitParts u1 = u0;
    if (kPrefix) u1 = unit_parts(p, x1, at.z, unit1);
    row0 -= unit0 * u0.size;
    row1 -= unit1 * u1.size;
    const int n = u0.n + (kPrefix ? u1.n : 0);
    const int most = __reduce_max_sync(0xffffffffu, n);
    float acc[K][4] = {};
    float m = neg_inf(), l = 0.0f;
#pragma unroll 1
    for (int i0 = 0; i0 < most; i0 += 8) {
        const int i = i0 + (lane & 7);
        float2 ml = make_float2(neg_inf(), 0.0f);
        const float* base = nullptr;                     // of the row; its columns lie part_at(0, c) further
        int step = 0;
        if (i < n) {
            const bool pre = kPrefix && i >= u0.n;
            const int64_t e = pre ? part_entry(p, u1, i - u0.n, row1) : part_entry(p, u0, i, row0);
            const PagedPart& part = pre ? *x1.part : *x0.part;
            const bool tiles = pre ? u1.tiles : u0.tiles;
            ml = part.ml[e];
            base = part.o + (tiles ? part_at<PAGED_TILES, D>(e, 0) : part_at<PAGED_ROWS, D>(e, 0));
            step = tiles;
        }
        const int here = min(8, most - i0);
        float o[kDeep][K][4];
        auto load = [&](int j, float (*to)[4]) {
            const float* src = reinterpret_cast<const float*>(
                __shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(base), 8 * q + j));
            const bool tiles = __shfl_sync(0xffffffffu, step, 8 * q + j) != 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = 4 * (col + 8 * k);
                const float* from = src + (tiles ? part_at<PAGED_TILES, D>(0, c) : c);
                *reinterpret_cast<float4*>(to[k]) = src && j < here ? *reinterpret_cast<const float4*>(from) : float4{};
            }
        };
#pragma unroll
        for (int d = 0; d < kDeep; ++d) load(d, o[d]);   // beside the maxima
        float mx = ml.x;
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
        const float nm = fmaxf(m, mx);
        const float ref = nm == neg_inf() ? 0.0f : nm;
        const float g = ex2(ml.x - ref);                 // 0 for what a row has not seen
        float sum = g * ml.y;
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const float f = ex2(m - ref);
        l = l * f + sum;
        m = nm;
        if (i0) {
            const float fq = __shfl_sync(0xffffffffu, f, 8 * q);
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[k][v] *= fq;
        }
#pragma unroll 1
        for (int j0 = 0; j0 < here; j0 += kDeep) {
            if (j0) {
#pragma unroll
                for (int d = 0; d < kDeep; ++d) load(j0 + d, o[d]);
            }
#pragma unroll
            for (int d = 0; d < kDeep; ++d) {
                // (an unseen part's O may never have been written)
                const float gq = __shfl_sync(0xffffffffu, g, 8 * q + j0 + d);
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int v = 0; v < 4; ++v) acc[k][v] += gq == 0.0f ? 0.0f : gq * o[d][k][v];
            }
        }
    }
    const float inv = finish_scale(sees, l);
    const float iq = __shfl_sync(0xffffffffu, inv, 8 * q);
    if (q < rows) {
        const int tok = token_of(p, at.w + q);
        const int qh = at.z * p.group + at.w + q - tok * p.group;
        uint16_t* dst = p.out + (t0 + tok) * p.ldo + static_cast<int64_t>(qh) * D + 4 * col;
#pragma unroll
        for (int k = 0; k < K; ++k)
            *reinterpret_cast<uint2*>(dst + 32 * k) =
                make_uint2(pack_bf16x2(acc[k][0] * iq, acc[k][1] * iq), pack_bf16x2(acc[k][2] * iq, acc[k][3] * iq));
    }
    if (p.lse && (lane & 7) == 0 && lane >> 3 < rows) {
        const int tok = token_of(p, at.w + mine);
        const int qh = at.z * p.group + at.w + mine - tok * p.group;
        p.lse[static_cast<int64_t>(t0 + tok) * p.n_q_heads + qh] = finish_lse(m, l);
    }
}

// ------------------------------------------------------------------ plan
// The batch's shape to the device, once for all calls of the batch.
__global__ void __launch_bounds__(256) plan_kernel(const __grid_constant__ PagedPlan p) {
    pdl_launch_dependents();
    pdl_wait();
    const int i = static_cast<int>(blockIdx.x * blockDim.x + threadIdx.x);
    if (i < 2 * kMaxReq) p.seg[i] = make_int4(p.segs[i].t0, p.segs[i].nt, p.segs[i].unit_base, p.segs[i].kind);
    if (i < p.n_row_blocks) {
        // the request of row block i: the last whose blocks start at or before it
        // (starts do not decrease; requests without rows have their successor's)
        int lo = 0, hi = p.n_req - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.segs[p.n_groups + mid].block_base <= i) lo = mid;
            else hi = mid - 1;
        }
        const PagedSegment& g = p.segs[p.n_groups + lo];
        const int per_head = (g.nt * p.group + kBlockRows - 1) / kBlockRows, u = i - g.block_base;
        int prefix = -1;
        if (p.n_groups) {
            int a = 0, z = p.n_groups - 1;
            while (a < z) {
                const int mid = (a + z + 1) >> 1;
                if (p.cu_group[mid] <= lo) a = mid;
                else z = mid - 1;
            }
            prefix = a;
        }
        p.row_block[i] = make_int4(p.n_groups + lo, prefix, u / per_head, u % per_head * kBlockRows);
    }
    if (i >= p.n_tokens) return;
    int lo = 0, hi = p.n_req - 1;                 // the request of token i
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.cu_q[mid] <= i) lo = mid;
        else hi = mid - 1;
    }
    const int req = lo;
    if (p.n_groups) {
        lo = 0;
        hi = p.n_groups - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.cu_group[mid] <= req) lo = mid;
            else hi = mid - 1;
        }
    }
    p.token[i] = make_int2(p.n_groups + req, p.n_groups ? lo : -1);
}

// ------------------------------------------------------------------ host
size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// A segment of more rows than this goes to tiles.  (16 requests of 28 rows over 3 to
// 9k tokens: 64 us as two units of few rows, which read the keys twice, 48 as tiles.)
constexpr int kRowsMost = kRowsTile;
// A call of more rows (tokens times query heads) than this joins them in blocks, up
// to the second number with eight partials in flight.  (Whole calls, row by row, in
// blocks eight and one deep: 2156 rows of 11 partials 22.3, 22.5 and 36.8 us; 3500 of 6 42.5,
// 39.3 and 48.3; 8192 of 7 139.5, 130.5 and 129; 134000 of 3 433, 309.5 and 267.)  One of
// at most two rows an SM, whose keys are cut into some hundred parts, joins each in
// a CTA (32 rows of 160: 9.9 us instead of 26.6 by a warp a row).
constexpr int kJoinRows = 2500, kJoinDeepRows = 6000;

// Where the plan and the partials of both kernels lie in a workspace; its size.
size_t paged_layout(const cr_attention_batch& b, uint8_t* ws, int4** seg, int2** token, int4** row_block, PagedPart* part,
                    uint8_t** weigh) {
    size_t at = 0;
    *seg = reinterpret_cast<int4*>(ws);
    at += align256(2 * kMaxReq * sizeof(int4));
    *token = reinterpret_cast<int2*>(ws + at);
    at += align256(static_cast<size_t>(b.n_tokens) * sizeof(int2));
    *row_block = reinterpret_cast<int4*>(ws + at);
    at += align256(static_cast<size_t>(b.n_row_blocks) * sizeof(int4));
    for (int k = 0; k < 2; ++k) {
        PagedPart& q = part[k];
        q.n_units = b.n_units[k];
        q.sched = nullptr;
        if (q.n_units == 0) continue;
        const size_t workers = static_cast<size_t>(b.n_ctas) * (k == PAGED_TILES ? 1 : kRowsWarps);
        const size_t slots = k == PAGED_TILES && b.n_groups == 0 ? 2 * workers : static_cast<size_t>(q.n_units) + workers;
        const size_t rows = slots * (k == PAGED_TILES ? kPair : kRowsTile);
        q.sched = reinterpret_cast<int32_t*>(ws + at);
        at += align256(kSchedInts * sizeof(int32_t));
        q.unit = reinterpret_cast<int2*>(ws + at);
        at += align256(k == PAGED_TILES ? static_cast<size_t>(q.n_units) * sizeof(int2) : 0);
        q.ml = reinterpret_cast<float2*>(ws + at);
        at += align256(rows * sizeof(float2));
        q.o = reinterpret_cast<float*>(ws + at);
        at += align256(rows * b.head_dim * sizeof(float));
    }
    *weigh = ws + at;
    at += align256(weigh_part_bytes(b.n_ctas));
    return at;
}

bool cache_maps(const cr_paged_layer& c, const PagedParams& p, int box_rows, CUtensorMap* tk, CUtensorMap* tv) {
    const uint64_t width = static_cast<uint64_t>(c.n_kv_heads) * c.head_dim;
    const uint64_t whole = static_cast<uint64_t>(p.n_blocks) << p.block_shift;   // rows past it read as zeros
    const uint32_t groups = (c.block_size < box_rows ? c.block_size : box_rows) / 8;
    const uint32_t halves = static_cast<uint32_t>(c.head_dim) / 64;
    return make_tmap_groups(tk, c.k, width, whole, halves, groups) &&
           make_tmap_groups(tv, c.v, width, whole, halves, groups);
}

template <int D, bool kRows, bool kTiles>
cr_status launch_main(const PagedParams& p, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tk16,
                      const CUtensorMap& tv16, cudaStream_t st) {
    using Cfg = TileCfg<D>;
    static unsigned long long attr_done = 0;
    static int regs_ok = -1;
    cr_status s = ensure_smem_attr(paged_kernel<D, kRows, kTiles>, static_cast<int>(Cfg::kSmem), &attr_done);
    if (s != CR_OK) return s;
    // raising the softmax warps' registers only completes if the launch reserved what the split assumes
    int ok = kTiles ? __atomic_load_n(&regs_ok, __ATOMIC_ACQUIRE) : 1;
    if (ok < 0) {
        cudaFuncAttributes fa;
        if ((s = cuda_check(cudaFuncGetAttributes(&fa, paged_kernel<D, kRows, kTiles>))) != CR_OK) return s;
        ok = fa.numRegs >= static_cast<int>(kRegsLaunch) && fa.maxThreadsPerBlock >= kTileThreads;
        __atomic_store_n(&regs_ok, ok, __ATOMIC_RELEASE);
    }
    if (!ok) return CR_ERR_UNSUPPORTED;
    return launch_pdl(paged_kernel<D, kRows, kTiles>, dim3(p.n_ctas), dim3(kTileThreads), Cfg::kSmem, st, tk, tv, tk16,
                      tv16, p);
}

template <int D>
cr_status launch_d(const cr_paged_layer& c, PagedParams& p, cudaStream_t st) {
    CUtensorMap tk, tv, tk16, tv16;
    if (!cache_maps(c, p, kChunk, &tk16, &tv16)) return CR_ERR_INVALID_ARG;
    // (without a segment of many rows the tiles' maps are not used)
    if (p.part[PAGED_TILES].n_units == 0) tk = tk16, tv = tv16;
    else if (!cache_maps(c, p, kKeys, &tk, &tv)) return CR_ERR_INVALID_ARG;
    const bool tiles = p.part[PAGED_TILES].n_units != 0, few = p.part[PAGED_ROWS].n_units != 0;
    cr_status s = tiles && few ? launch_main<D, true, true>(p, tk, tv, tk16, tv16, st)
                  : tiles      ? launch_main<D, false, true>(p, tk, tv, tk16, tv16, st)
                               : launch_main<D, true, false>(p, tk, tv, tk16, tv16, st);
    if (s != CR_OK) return s;
    const int64_t rows = static_cast<int64_t>(p.n_tokens) * p.n_q_heads;
    if (rows <= 2 * num_sms())
        return launch_pdl(p.n_groups ? join_few_kernel<D, 16, true> : join_few_kernel<D, 16, false>,
                          dim3(static_cast<unsigned>(rows)), dim3(512), 0, st, p);
    const dim3 blocks(static_cast<unsigned>((p.n_row_blocks + 3) / 4));
    if (rows > kJoinDeepRows)
        return launch_pdl(p.n_groups ? join_blocks_kernel<D, true, 1> : join_blocks_kernel<D, false, 1>, blocks, dim3(128),
                          0, st, p);
    if (rows > kJoinRows)
        return launch_pdl(p.n_groups ? join_blocks_kernel<D, true, 8> : join_blocks_kernel<D, false, 8>, blocks, dim3(128),
                          0, st, p);
    return launch_pdl(p.n_groups ? join_kernel<D, true> : join_kernel<D, false>,
                      dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(128), 0, st, p);
}

}  // namespace

size_t paged_plan(PagedPlan& p, cr_attention_batch& b) {
    int64_t u[2] = {0, 0}, blocks = 0;
    memset(p.segs, 0, sizeof(p.segs));
    for (int s = 0; s < p.n_groups + p.n_req; ++s) {
        const int t0 = s < p.n_groups ? p.cu_q[p.cu_group[s]] : p.cu_q[s - p.n_groups];
        const int t1 = s < p.n_groups ? p.cu_q[p.cu_group[s + 1]] : p.cu_q[s - p.n_groups + 1];
        const int64_t rows = static_cast<int64_t>(t1 - t0) * (b.n_q_heads / b.n_kv_heads);
        const int k = rows > kRowsMost ? PAGED_TILES : PAGED_ROWS;
        const int64_t size = k == PAGED_TILES ? kPair : kRowsTile;
        p.segs[s] = {t0, t1 - t0, static_cast<int32_t>(u[k]), rows ? k : -1, static_cast<int32_t>(blocks)};
        if (s >= p.n_groups) blocks += (rows + kBlockRows - 1) / kBlockRows * b.n_kv_heads;
        u[k] += (rows + size - 1) / size * b.n_kv_heads;
        if (u[k] > INT32_MAX / 4) return 0;
    }
    for (int k = 0; k < 2; ++k) b.n_units[k] = static_cast<int32_t>(u[k]);
    b.n_ctas = num_sms();
    if (blocks > INT32_MAX / 4) return 0;
    p.group = b.n_q_heads / b.n_kv_heads;
    p.n_row_blocks = b.n_row_blocks = static_cast<int32_t>(blocks);
    int4 *seg, *row_block;
    int2* token;
    PagedPart part[2];
    uint8_t* weigh;
    return paged_layout(b, nullptr, &seg, &token, &row_block, part, &weigh);
}

cr_status launch_paged_plan(PagedPlan& p, const cr_attention_batch& b, cudaStream_t st) {
    PagedPart part[2];
    uint8_t* weigh;
    paged_layout(b, static_cast<uint8_t*>(b.workspace), &p.seg, &p.token, &p.row_block, part, &weigh);
    int n = p.n_tokens > 2 * kMaxReq ? p.n_tokens : 2 * kMaxReq;
    if (n < p.n_row_blocks) n = p.n_row_blocks;
    return launch_pdl(plan_kernel, dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, st, p);
}

const int4* paged_segments(const cr_attention_batch& b) {
    int4 *seg, *row_block;
    int2* token;
    PagedPart part[2];
    uint8_t* weigh;
    paged_layout(b, static_cast<uint8_t*>(b.workspace), &seg, &token, &row_block, part, &weigh);
    return seg;
}

uint8_t* paged_weigh_parts(const cr_attention_batch& b) {
    int4 *seg, *row_block;
    int2* token;
    PagedPart part[2];
    uint8_t* weigh;
    paged_layout(b, static_cast<uint8_t*>(b.workspace), &seg, &token, &row_block, part, &weigh);
    return weigh;
}

cr_status launch_paged_attention(PagedParams& p, const cr_paged_layer& cache, const cr_attention_batch& b,
                                 cudaStream_t st) {
    // the lines of chunks are counted in 32 bits
    const int64_t most = p.prefix_table && p.prefix_blocks > p.own_blocks ? p.prefix_blocks : p.own_blocks;
    for (int k = 0; k < 2; ++k) {
        const int64_t chunk = k == PAGED_TILES ? kKeys : kChunk;
        if (b.n_units[k] * (((most << p.block_shift) + chunk - 1) / chunk + kUnitCost) > INT32_MAX / 2)
            return CR_ERR_UNSUPPORTED;
    }
    int4 *seg, *row_block;
    int2* token;
    uint8_t* weigh;
    paged_layout(b, static_cast<uint8_t*>(b.workspace), &seg, &token, &row_block, p.part, &weigh);
    p.n_ctas = b.n_ctas;
    p.seg = seg;
    p.token = token;
    p.row_block = row_block;
    p.n_row_blocks = b.n_row_blocks;
    return cache.head_dim == 128 ? launch_d<128>(cache, p, st) : launch_d<64>(cache, p, st);
}

}  // namespace cr
