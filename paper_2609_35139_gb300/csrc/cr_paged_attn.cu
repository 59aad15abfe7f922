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
// The work of a call is one line of chunks, segment by segment and unit by
// unit, which the workers cut into equal pieces whatever the sequences' lengths
// are; the lengths are read on the device, so nothing is planned on the host.
#include <cuda_bf16.h>

#include "cr_internal.h"
#include "cr_ptx.cuh"

namespace cr {
namespace {

constexpr int kMaxSegments = 2 * kMaxReq;
constexpr int kRowsTile = 16;       // rows of a unit: one m16 tile
constexpr int kChunk = 16;          // keys of a chunk
constexpr int kRowsWarps = 8;
constexpr int kMinChunks = 4;       // fewest chunks a worker takes

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

// ------------------------------------------------------------------ segments
struct Segment {
    int t0, nt;            // query tokens
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

__device__ __forceinline__ Segment segment(const PagedParams& p, int s) {
    Segment g;
    g.own = s >= p.n_groups;
    if (g.own) {
        const int r = s - p.n_groups;
        g.t0 = p.cu_q[r];
        g.nt = p.cu_q[r + 1] - g.t0;
        g.table = p.own_table + r * p.own_blocks;
        g.len = clamp_len(p, p.own_len[r], p.own_blocks);
    } else {
        g.t0 = p.cu_q[p.cu_group[s]];
        g.nt = p.cu_q[p.cu_group[s + 1]] - g.t0;
        g.table = p.prefix_table + s * p.prefix_blocks;
        g.len = clamp_len(p, p.prefix_len[s], p.prefix_blocks);
    }
    g.blocks = (g.len + (1 << p.block_shift) - 1) >> p.block_shift;
    return g;
}

// Keys that a row of the segment sees: all of a prefix, one's own tokens up to
// the row's own (never negative).
__device__ __forceinline__ int row_limit(const PagedParams& p, const Segment& g, int row) {
    if (!g.own) return g.len;
    const int lim = g.len - g.nt + row / p.group + 1;
    return lim < 0 ? 0 : lim;
}

// cum[s] = chunks before segment s, for s = 0 .. n_seg; by all of the CTA's
// kRowsWarps * 32 threads, two segments a thread.
__device__ void schedule(const PagedParams& p, int64_t* cum, int64_t* warp_sum) {
    const int n_seg = p.n_groups + p.n_req;
    int64_t c[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int s = 2 * static_cast<int>(threadIdx.x) + k;
        c[k] = 0;
        if (s < n_seg) {
            const int64_t units = p.unit_base[s + 1] - p.unit_base[s];
            if (units) c[k] = units * ((segment(p, s).len + kChunk - 1) / kChunk);
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
    int64_t before = 0;
    for (uint32_t w = 0; w < warp_id(); ++w) before += warp_sum[w];
    x += before;
    const int s = 2 * static_cast<int>(threadIdx.x);
    if (s < n_seg) cum[s + 1] = x - c[1];
    if (s + 1 < n_seg) cum[s + 2] = x;
    if (threadIdx.x == 0) cum[0] = 0;
    __syncthreads();
}

// Chunks of the line that one worker takes.
__device__ __forceinline__ int64_t chunks_per_worker(int64_t total, int n_workers) {
    const int64_t c = (total + n_workers - 1) / n_workers;
    return c < kMinChunks ? kMinChunks : c;
}

// ------------------------------------------------------------------ rows kernel
template <int D>
struct RowsCfg {
    static constexpr int kHalves = D / 64;                       // 128-byte column halves of a row
    static constexpr uint32_t kTile = kHalves * kChunk * 128;    // K (or V) of a chunk
    static constexpr uint32_t kStage = 2 * kTile;
    static constexpr int kStages = D == 128 ? 3 : 6;
    static constexpr uint32_t kBars = kRowsWarps * kStages * kStage;
    static constexpr uint32_t kCum = kBars + kRowsWarps * kStages * 8;
    static constexpr uint32_t kSmem = 1024 + kCum + (kMaxSegments + 1) * 8 + kRowsWarps * 8 + 16;
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

// After a wait that gave up: leave the copies in flight time to land before the
// CTA's shared memory is given back.
__device__ __forceinline__ void drain_pause() {
    const uint64_t t0 = globaltimer();
    while (globaltimer() - t0 < 50000ull) {
    }
}

// Where a warp stands on the line of chunks.
struct Cursor {
    int seg, unit, chunk;       // unit within the segment
    int units, n_chunks;
    Segment g;
};

__device__ __forceinline__ void enter(const PagedParams& p, Cursor& c, int seg) {
    c.seg = seg;
    c.units = p.unit_base[seg + 1] - p.unit_base[seg];
    c.g = segment(p, seg);
    c.n_chunks = (c.g.len + kChunk - 1) / kChunk;
}
__device__ __forceinline__ void seek(const PagedParams& p, Cursor& c, const int64_t* cum, int64_t at) {
    int lo = 0, hi = p.n_groups + p.n_req - 1;      // the last segment that starts at or before `at`
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (cum[mid] <= at) lo = mid;
        else hi = mid - 1;
    }
    enter(p, c, lo);
    const int64_t off = at - cum[lo];
    c.unit = static_cast<int>(off / c.n_chunks);
    c.chunk = static_cast<int>(off - static_cast<int64_t>(c.unit) * c.n_chunks);
}
// One chunk on; the caller knows that the line goes on.
__device__ __forceinline__ void advance(const PagedParams& p, Cursor& c, const int64_t* cum) {
    if (++c.chunk < c.n_chunks) return;
    c.chunk = 0;
    if (++c.unit < c.units) return;
    c.unit = 0;
    int s = c.seg + 1;
    while (cum[s + 1] == cum[s]) ++s;               // segments without work
    enter(p, c, s);
}

// Every warp is a worker of its own: it loads its chunks by TMA into its own
// ring, multiplies them with the unit's rows (one m16 tile) and writes one
// partial (m, l, O) per unit that its piece of the line touches.
template <int D>
__global__ void __launch_bounds__(kRowsWarps * 32, 1)
    rows_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                const __grid_constant__ PagedParams p) {
    using Cfg = RowsCfg<D>;
    constexpr int NS = Cfg::kStages;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                               ~static_cast<uintptr_t>(1023));
    const uint32_t warp = warp_id(), lane = lane_id();
    uint8_t* ring = smem + warp * NS * Cfg::kStage;
    uint64_t* full = reinterpret_cast<uint64_t*>(smem + Cfg::kBars) + warp * NS;
    int64_t* cum = reinterpret_cast<int64_t*>(smem + Cfg::kCum);
    int64_t* warp_sum = cum + kMaxSegments + 1;
    int* abort_flag = reinterpret_cast<int*>(warp_sum + kRowsWarps);
    pdl_launch_dependents();
    if (lane == 0)
        for (int s = 0; s < NS; ++s) mbar_init(&full[s], 1);
    if (threadIdx.x == 0) *abort_flag = 0;
    fence_barrier_init();
    pdl_wait();
    schedule(p, cum, warp_sum);      // (its barriers also order the initialisation)

    const int n_seg = p.n_groups + p.n_req;
    const int64_t total = cum[n_seg];
    const int64_t per = chunks_per_worker(total, p.n_workers);
    if (blockIdx.x == 0) {
        for (int s = threadIdx.x; s <= n_seg; s += blockDim.x) p.sched[s] = cum[s];
        if (threadIdx.x == 0) p.sched[n_seg + 1] = per;
    }
    const int worker = static_cast<int>(warp * gridDim.x + blockIdx.x);
    const int64_t begin = worker * per;
    const int64_t end = min(total, begin + per);
    if (begin >= end) return;
    const WaitCtx wc{abort_flag, p.status};

    // ---- loads, up to NS chunks ahead of the products
    Cursor ld;
    seek(p, ld, cum, begin);
    int64_t ld_at = begin;
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
        const int head = ld.unit / (ld.units / p.n_kv_heads);
        const int x = head * D;
        const int y0 = (__shfl_sync(0xffffffffu, page_id, first - page_base) << p.block_shift) + in_block;
        const int y1 = __shfl_sync(0xffffffffu, page_id, last - page_base) << p.block_shift;
        uint8_t* dst = ring + stage * Cfg::kStage;
        if (elect_one()) {
            mbar_expect_tx(&full[stage], Cfg::kStage);
#pragma unroll
            for (int h = 0; h < Cfg::kHalves; ++h) {
                uint8_t* k = dst + h * (kChunk * 128);
                uint8_t* v = k + Cfg::kTile;
                tma_load_2d(k, &tm_k, &full[stage], x + 64 * h, y0);
                tma_load_2d(v, &tm_v, &full[stage], x + 64 * h, y0);
                if (p.block_shift < 4) {     // blocks of 8: two boxes of 8 rows
                    tma_load_2d(k + 1024, &tm_k, &full[stage], x + 64 * h, y1);
                    tma_load_2d(v + 1024, &tm_v, &full[stage], x + 64 * h, y1);
                }
            }
        }
        __syncwarp();
        if (++ld_at < end) advance(p, ld, cum);
    };
    for (int s = 0; s < NS && ld_at < end; ++s) load(s);

    // ---- products
    Cursor cur;
    seek(p, cur, cum, begin);
    const int rq = static_cast<int>(lane >> 2);      // this thread's rows of the tile: rq, rq + 8
    const int cq = static_cast<int>(lane & 3) * 2;
    uint32_t qf[D / 16][4];
    float o[D / 8][4];
    float m[2], l[2];
    int lim[2];
    bool fresh = true;
    int stage = 0;
    uint32_t phase = 0;
    for (int64_t at = begin; at < end; ++at) {
        const int tiles = cur.units / p.n_kv_heads;
        const int head = cur.unit / tiles;
        const int row0 = (cur.unit - head * tiles) * kRowsTile;
        const int rows = cur.g.nt * p.group - row0;      // valid rows of the tile
        if (fresh) {
            fresh = false;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = row0 + rq + 8 * h;
                const bool ok = rq + 8 * h < rows;
                const int tok = row / p.group;
                const uint16_t* src = p.q + (cur.g.t0 + tok) * p.ldq +
                                      static_cast<int64_t>(head * p.group + row - tok * p.group) * D + cq;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    qf[k][h] = ok ? *reinterpret_cast<const uint32_t*>(src + 16 * k) : 0u;
                    qf[k][2 + h] = ok ? *reinterpret_cast<const uint32_t*>(src + 16 * k + 8) : 0u;
                }
                lim[h] = ok ? row_limit(p, cur.g, row) : 0;
                m[h] = neg_inf();
                l[h] = 0.0f;
            }
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = 0.0f;
        }
        if (!mbar_wait_warp(&full[stage], phase, wc, 913)) {
            drain_pause();
            return;
        }
        const uint32_t kb = smem_u32(ring + stage * Cfg::kStage);
        const uint32_t vb = kb + Cfg::kTile;
        const int k0 = cur.chunk * kChunk;
        if (k0 + kChunk > cur.g.len) {
            // the rows of V past the segment's end meet P = 0: they must not hold NaN
            const int from = cur.g.len - k0;
            uint8_t* v = ring + stage * Cfg::kStage + Cfg::kTile;
            for (int i = static_cast<int>(lane); i < (kChunk - from) * 8 * Cfg::kHalves; i += 32) {
                const int row = from + i / (8 * Cfg::kHalves);
                const int c = i % (8 * Cfg::kHalves);
                *reinterpret_cast<uint4*>(v + (c >> 3) * (kChunk * 128) + row * 128 + (c & 7) * 16) =
                    make_uint4(0, 0, 0, 0);
            }
            fence_async_smem();      // before the stage's next TMA load
            __syncwarp();
        }
        float s[2][4] = {};
        {
            const int key = static_cast<int>((lane >> 4) * 8 + (lane & 7));
            const int odd = static_cast<int>((lane >> 3) & 1);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const int c = 2 * k + odd;
                uint32_t b[4];
                ldsm4(kb + (c >> 3) * (kChunk * 128) + key * 128 + (((c & 7) ^ (key & 7)) << 4), b);
                mma16816(s[0], qf[k], b);
                mma16816(s[1], qf[k], b + 2);
            }
        }
        // scores of row rq (elements 0, 1) and rq + 8 (2, 3), keys k0 + 8 n + cq + {0, 1}
        const bool mask = k0 + kChunk > cur.g.len || cur.g.own;
        float mx[2] = {neg_inf(), neg_inf()};
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = s[n][e] * p.scale_log2;
                if (mask && k0 + 8 * n + cq + (e & 1) >= lim[e >> 1]) x = neg_inf();
                s[n][e] = x;
                mx[e >> 1] = fmaxf(mx[e >> 1], x);
            }
        float ref[2];
        bool moved = false;
        float alpha[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
            mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
            const float nm = fmaxf(m[h], mx[h]);
            alpha[h] = nm == m[h] ? 1.0f : ex2(m[h] - nm);
            moved |= nm != m[h];
            m[h] = nm;
            ref[h] = nm == neg_inf() ? 0.0f : nm;     // a row that has seen nothing keeps P = 0
        }
        if (__any_sync(0xffffffffu, moved)) {
            l[0] *= alpha[0];
            l[1] *= alpha[1];
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] *= alpha[e >> 1];
        }
        // P as two bf16 terms (the products are far from being the bound here),
        // so that its rounding does not add to that of the output
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float e0 = ex2(s[n][2 * h] - ref[h]), e1 = ex2(s[n][2 * h + 1] - ref[h]);
                l[h] += e0 + e1;
                split_bf16x2(e0, e1, &hi[2 * n + h], &lo[2 * n + h]);
            }
        {
            const int key = static_cast<int>(((lane >> 3) & 1) * 8 + (lane & 7));
            const int odd = static_cast<int>(lane >> 4);
#pragma unroll
            for (int n = 0; n < D / 16; ++n) {
                const int c = 2 * n + odd;
                uint32_t b[4];
                ldsm4_t(vb + (c >> 3) * (kChunk * 128) + key * 128 + (((c & 7) ^ (key & 7)) << 4), b);
                mma16816(o[2 * n], hi, b);
                mma16816(o[2 * n + 1], hi, b + 2);
                mma16816(o[2 * n], lo, b);
                mma16816(o[2 * n + 1], lo, b + 2);
            }
        }
        __syncwarp();                                  // every lane has read the stage
        if (ld_at < end) load(stage);
        if (++stage == NS) {
            stage = 0;
            phase ^= 1u;
        }
        if (at + 1 == end || cur.chunk + 1 == cur.n_chunks) {
            // the piece of this unit ends: its partial
            const int64_t slot = p.unit_base[cur.seg] + cur.unit + worker;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], 1);
                l[h] += __shfl_xor_sync(0xffffffffu, l[h], 2);
                const int r = rq + 8 * h;
                if (r < rows) {
                    float* dst = p.part_o + (slot * kRowsTile + r) * D + cq;
#pragma unroll
                    for (int n = 0; n < D / 8; ++n)
                        *reinterpret_cast<float2*>(dst + 8 * n) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
                    if (cq == 0) p.part_ml[slot * kRowsTile + r] = make_float2(m[h], l[h]);
                }
            }
            fresh = true;
        }
        if (at + 1 < end) advance(p, cur, cum);
    }
}

// ------------------------------------------------------------------ join
// One warp per (token, query head): the row's partials joined, its output and
// log-sum-exp written.
template <int D>
__global__ void __launch_bounds__(128) join_kernel(const __grid_constant__ PagedParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const int64_t w = blockIdx.x * 4ll + warp_id();
    if (w >= static_cast<int64_t>(p.n_tokens) * p.n_q_heads) return;
    const int lane = static_cast<int>(lane_id());
    const int t = static_cast<int>(w / p.n_q_heads);
    const int qh = static_cast<int>(w - static_cast<int64_t>(t) * p.n_q_heads);
    const int head = qh / p.group;
    const int n_seg = p.n_groups + p.n_req;
    const int64_t per = p.sched[n_seg + 1];
    int lo = 0, hi = p.n_req - 1;                 // the request of token t
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.cu_q[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    const int req = lo;
    int seg[2] = {p.n_groups + req, -1};
    if (p.n_groups) {
        lo = 0;
        hi = p.n_groups - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (p.cu_group[mid] <= req) lo = mid;
            else hi = mid - 1;
        }
        seg[1] = lo;
    }
    constexpr int V = D / 32;
    float acc[V] = {};
    float m = neg_inf(), l = 0.0f;
    for (int k = 0; k < 2; ++k) {
        const int s = seg[k];
        if (s < 0) continue;
        const int units = p.unit_base[s + 1] - p.unit_base[s];
        const int64_t c0 = p.sched[s];
        const int64_t n_chunks = (p.sched[s + 1] - c0) / units;
        if (n_chunks == 0) continue;
        const int t0 = k == 0 ? p.cu_q[req] : p.cu_q[p.cu_group[s]];
        const int row = (t - t0) * p.group + qh - head * p.group;
        const int unit = head * (units / p.n_kv_heads) + row / kRowsTile;
        const int64_t a = c0 + unit * n_chunks;
        const int64_t w0 = a / per, w1 = (a + n_chunks - 1) / per;
        const int64_t base = p.unit_base[s] + unit;
        const int r = row % kRowsTile;
        for (int64_t i = w0; i <= w1; ++i) {
            const int64_t at = (base + i) * kRowsTile + r;
            const float2 ml = p.part_ml[at];
            if (ml.x == neg_inf()) continue;
            const float nm = fmaxf(m, ml.x);
            const float f0 = ex2(m - nm), f1 = ex2(ml.x - nm);
            const float* src = p.part_o + at * D + lane * V;
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v] = acc[v] * f0 + src[v] * f1;
            l = l * f0 + ml.y * f1;
            m = nm;
        }
    }
    const float inv = m == neg_inf() ? 0.0f : 1.0f / l;
    uint16_t* dst = p.out + t * p.ldo + static_cast<int64_t>(qh) * D + lane * V;
#pragma unroll
    for (int v = 0; v < V; v += 2)
        *reinterpret_cast<uint32_t*>(dst + v) = pack_bf16x2(acc[v] * inv, acc[v + 1] * inv);
    if (p.lse && lane == 0)
        p.lse[w] = m == neg_inf() ? neg_inf() : (m + log2f(l)) * 0.6931471805599453f;
}

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

struct PagedLayout {
    size_t sched, ml, o, total;
};
PagedLayout paged_layout(const PagedParams& p, int head_dim) {
    const size_t slots = static_cast<size_t>(p.unit_base[p.n_groups + p.n_req]) + p.n_workers;
    PagedLayout w{};
    w.sched = 0;
    w.ml = align256((kMaxSegments + 2) * sizeof(int64_t));
    w.o = w.ml + align256(slots * kRowsTile * sizeof(float2));
    w.total = w.o + align256(slots * kRowsTile * head_dim * sizeof(float));
    return w;
}

template <int D>
cr_status launch_d(const CUtensorMap& tk, const CUtensorMap& tv, const PagedParams& p, cudaStream_t st) {
    using Cfg = RowsCfg<D>;
    static unsigned long long attr_done = 0;
    cr_status s = ensure_smem_attr(rows_kernel<D>, static_cast<int>(Cfg::kSmem), &attr_done);
    if (s != CR_OK) return s;
    s = launch_pdl(rows_kernel<D>, dim3(p.n_workers / kRowsWarps), dim3(kRowsWarps * 32), Cfg::kSmem, st, tk, tv, p);
    if (s != CR_OK) return s;
    const int64_t rows = static_cast<int64_t>(p.n_tokens) * p.n_q_heads;
    return launch_pdl(join_kernel<D>, dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(128), 0, st, p);
}

// Units of the segments and workers, from the batch in p.
bool paged_plan(PagedParams& p) {
    int64_t u = 0;
    for (int s = 0; s < p.n_groups + p.n_req; ++s) {
        p.unit_base[s] = static_cast<int32_t>(u);
        const int64_t nt = s < p.n_groups ? p.cu_q[p.cu_group[s + 1]] - p.cu_q[p.cu_group[s]]
                                          : p.cu_q[s - p.n_groups + 1] - p.cu_q[s - p.n_groups];
        u += (nt * p.group + kRowsTile - 1) / kRowsTile * p.n_kv_heads;
        if (u > INT32_MAX / 2) return false;
    }
    p.unit_base[p.n_groups + p.n_req] = static_cast<int32_t>(u);
    p.n_workers = num_sms() * kRowsWarps;
    return true;
}

}  // namespace

size_t paged_workspace_bytes(const PagedParams& q, int head_dim) {
    PagedParams p = q;
    return paged_plan(p) ? paged_layout(p, head_dim).total : 0;
}

cr_status launch_paged_attention(PagedParams& p, const cr_paged_layer& cache, void* workspace, cudaStream_t st) {
    if (!paged_plan(p)) return CR_ERR_UNSUPPORTED;
    const PagedLayout w = paged_layout(p, cache.head_dim);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    p.sched = reinterpret_cast<int64_t*>(ws + w.sched);
    p.part_ml = reinterpret_cast<float2*>(ws + w.ml);
    p.part_o = reinterpret_cast<float*>(ws + w.o);
    const uint64_t width = static_cast<uint64_t>(cache.n_kv_heads) * cache.head_dim;
    const uint64_t whole = static_cast<uint64_t>(p.n_blocks) << p.block_shift;   // rows past it read as zeros
    const uint32_t rows = cache.block_size < kChunk ? cache.block_size : kChunk;
    CUtensorMap tk, tv;
    if (!make_tmap_2d(&tk, cache.k, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, width, whole, width * 2, 64, rows,
                      CU_TENSOR_MAP_SWIZZLE_128B) ||
        !make_tmap_2d(&tv, cache.v, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, width, whole, width * 2, 64, rows,
                      CU_TENSOR_MAP_SWIZZLE_128B))
        return CR_ERR_INVALID_ARG;
    return cache.head_dim == 128 ? launch_d<128>(tk, tv, p, st) : launch_d<64>(tk, tv, p, st);
}

}  // namespace cr
