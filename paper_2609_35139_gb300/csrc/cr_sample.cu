// Drawing the next token of every row of logits with a given uniform number:
//   w_i = exp((x_i - max x) / T),
//   kept = the top_k largest, of these the shortest run in descending order whose
//          predecessors' share of the sum stays below top_p, of these w_i >= min_p,
//   token = the first kept i, in the order of the vocabulary, with sum_{j <= i} w_j > u sum w.
// Equal logits are ranked by index.
//
// A row is one cluster's, from a CTA a row where there are many rows to eight where there are few.
// It is passed over two to four times: read from memory once and then from L2, or, where the rows on
// their way are more than L2 holds, from memory twice.  Both cuts are places in
// descending order where a running sum (of ones, or of w) passes a target; nothing is sorted.
// Values are told apart by the step of 2^(1/64) that their w falls into.  top_k: if every CTA's
// share of k is reached by its threads' largest values alone down to some value, k values are
// reached there, and the cut lies among the values down to it, little more than k, which are
// brought to every CTA.  top_p alone: a count of the values by step says nearly where the cut is; the
// values of the steps around it, mostly some hundred, are brought to every CTA,
// and with the exact sum of what is above them give the exact place (or tell that the cut is
// elsewhere, and it is searched among all values).  What a cut keeps is then in that list, or above it
// and summed by warps already, so no other pass is made; a short list alone gives the token, without
// another word between the CTAs (one row with top-k and top-p: 14 us for 17, 512 with top-k: 93 for 111).
//
// The answer turns on where u times a sum falls among up to 2^20 partial sums, so the weights
// are integers in units of 2^-44 (up to 2^-43.9 of the largest), off by less than a unit and 2^-26.9 of
// themselves, and their sums are exact and the same in any order.
//
// One row of 131072 fp32 with top-k and top-p takes 14.2 us, 16 of 32003 bf16 with none 10.3, 64 of 100003
// fp32 with filters of their own 44: cluster barriers and searches one after the other.  512 of 131072
// fp32 with top-p take 230 (268 MB in 0.17 of the copy rate): 25 us to bring a row's values from L2 for
// the largest, 44 to count them, some 100 to weigh them, 45 for the rest, and the 304 rows on their
// way are more than L2 holds.
#include <type_traits>

#include "cr_cluster.cuh"
#include "cr_internal.h"

namespace cr {
namespace {

constexpr int kOne = 44;               // no weight is above 2^44
constexpr int kStep = 128;             // a warp's values are a multiple of this, in steps of four a thread
// fewest values worth a CTA: 16 rows of 32003 take 10.9 us with eight CTAs a row, 11.6 with four, 14.6
// with two
constexpr int kLeast = 4 * 1024;
constexpr int kListSize = 2048;        // values of a row that a cut is searched among, an equal part for each CTA
constexpr int kPairs = 256;            // so many of them are compared each with each
// so many are looked through without narrowing the steps further (512 rows of 131072: 237 us, with 256
// and 1280 in its place 236 and 240, without narrowing, when the list overflows, 1139)
constexpr uint64_t kFewEnough = 640;
constexpr int kLastBin = kSelBins - 2;             // steps are counted up to this one
constexpr float kRound64 = 196608.0f;              // 1.5 2^17: adding it rounds to a multiple of 1/64
constexpr uint32_t kRound64Bits = 0x48400000u;     // as an integer
constexpr float kRound16 = 786432.0f;              // the same for 1/16
constexpr int kRound16Bits = 0x49400000;

// 2^(j / 16), j = 0 .. 15, in units of 2^-28.
__constant__ uint32_t kExpTable[16] = {268435456, 280320109, 292730940, 305691246, 319225354, 333358668, 348117717, 363530205,
                                       379625062, 396432500, 413984066, 432312707, 451452825, 471440350, 492312797, 514109347};

// What the threads of a CTA share.
struct alignas(16) Shared {
    SelShared sel;
    uint2 table[16];           // kExpTable, and as floats
    float list[kListSize];
    int token_of[kListSize];
    uint8_t warp_of[kListSize];                     // of this CTA's part of the list
    uint32_t counts[kMaxCluster];
    ulonglong2 pair[kPairs];   // of a listed value: key and, below it, what falls as the token rises; weight
    uint64_t how[3];           // temperature and top_k, top_p and min_p, u
    uint64_t place[4];         // of a cut: key, what is missing there, what lies above, whether found
    uint64_t warp_before[kSelWarps];
    float top;                 // the row's largest value
    float lowest;              // of the threads' largest values in this CTA
    float c_hi, c_lo;          // c = log2(e) / T in two parts
    float shift, zero;         // weights are 2^44 2^((x - shift) c - R): zero is kRound16 - R
    float ahead;               // (max x - shift) c - R
    double least;              // T log(min_p): the smallest x - max that min_p keeps
    int listed;
    const void* row;           // this CTA's places, of which every fourth starts a load of four
    int begin, end;            // those that hold values
    int base;                  // token of the first place
    int per_warp;              // places of a warp
    bool bf16;
    int turn;                  // histogram in use
    uint32_t rank, n;
    uint32_t full;             // CTAs whose every place holds a value (one at least)
};
extern __shared__ __align__(16) uint8_t smem[];
__device__ __forceinline__ Shared& shared() { return *reinterpret_cast<Shared*>(smem); }
static_assert(sizeof(Shared) <= 100 * 1024, "two CTAs an SM");

__device__ __forceinline__ float value_at(int i) {
    const Shared& g = shared();
    if (g.bf16) return __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const uint16_t*>(g.row) + i)) << 16);
    return __ldg(static_cast<const float*>(g.row) + i);
}

// How far below the largest x lies, in steps of 2^(1/64) of the weight: does not fall as x falls,
// and is more than any step that counts for an x too far down to be told (-inf among them).
__device__ __forceinline__ uint32_t step_of(float x, float top, float c_hi) {
    return kRound64Bits - __float_as_uint(fmaf(x - top, c_hi, kRound64));
}
// Integer weight of the middle of a step, nearly.
__device__ __forceinline__ uint64_t step_weight(int step, float ahead) {
    return static_cast<uint64_t>(__float2uint_rn(ex2(fmaf(static_cast<float>(step & 63), -1.0f / 64.0f, ahead)) * (1 << 28))) << (kOne - 28) >> (step >> 6);
}
__device__ __forceinline__ uint32_t shift_right(uint32_t v, uint32_t by) {           // (0 for 32 and more)
    uint32_t r;
    asm("shr.u32 %0, %1, %2;" : "=r"(r) : "r"(v), "r"(by));
    return r;
}
// Integer weight of x, as a product: 2^44 2^t, t = (x - shift) c - R, with R a multiple of 1/16 just
// above (max x - shift) c (the largest weight is 2^-1/8 to 1 of 2^44; every sum is compared with sums
// alone).  x - shift is exact: shift is 0, or, where |max x c| is 2^17 or more, max x, from which
// any x that weighs something is no further than 2^-11 of itself.  (x - max x in its place would be off by
// 2^-25 of itself, up to 2^-19 of a weight, and the same for all equal logits.)  t = k / 16 + f, k a
// (negative) integer, |f| <= 1/32, by FMA and c in two parts:
// 2^t = 2^floor(k / 16) T[k mod 16] (1 + y), y = 2^f - 1 by its series (y < 2^-5.5, so its fp32
// rounding is 2^-30 of the weight).  Off by 2^-26.9 of the weight at most (2^-29 for the table and as much for
// the product, 2^-30.5 for each of two roundings of f and four of the rest), and cut off to whole units.
// (A table of 16 is one row of the banks: no conflicts.)
struct Product {
    uint32_t a, b;
};
struct Scale {
    float c_hi, c_lo, shift, zero;
};
__device__ __forceinline__ Scale scale_of() {
    const Shared& g = shared();
    return {g.c_hi, g.c_lo, g.shift, g.zero};
}
__device__ __forceinline__ Product weight_parts(float x, const Scale& c) {
    const float d = x - c.shift, r = fmaf(d, c.c_hi, c.zero);
    const int bits = __float_as_int(r);
    const float f = fmaf(d, c.c_lo, fmaf(d, c.c_hi, c.zero - r));
    // 2^f - 1 = f ln 2 + (f ln 2)^2 / 2 + ...
    const float y = f * fmaf(f, fmaf(f, fmaf(f, 9.61812911e-3f, 5.55041087e-2f), 2.40226507e-1f), 6.93147181e-1f);
    const uint2 t = shared().table[bits & 15];
    const uint32_t w = t.x + static_cast<uint32_t>(__float2int_rn(__uint_as_float(t.y) * y));
    // w 2^(16 - down) (of a value far down, -inf too, the sign of r makes `down` large and a 0)
    const int down = (kRound16Bits >> 4) - (bits >> 4);
    return {shift_right(w, static_cast<uint32_t>(max(down - (kOne - 28), 0))),
            max(shift_right(1u << (kOne - 28), static_cast<uint32_t>(down)), 1u)};
}
__device__ __forceinline__ uint64_t weight(float x, const Scale& c) {
    const Product w = weight_parts(x, c);
    return static_cast<uint64_t>(w.a) * w.b;
}
__device__ __noinline__ uint64_t weight_of(float x) { return weight(x, scale_of()); }

// 2^64 v for v in [0, 1), exact down to 2^-40.
__device__ __forceinline__ uint64_t fraction64(float v) {
    const uint32_t b = __float_as_uint(v);
    const int s = static_cast<int>(b >> 23) - 86;
    const uint64_t m = (b & 0x7fffffu) | 0x800000u;
    return s >= 0 ? m << s : s > -24 ? m >> -s : 0;
}

// The parts below run once or a few times a row, one after the other: each is one copy of
// code (inlined where they are called they made 250 KB, and fetching it was most of the time).

// Batches of this thread's values, a warp's values lying together: f(v, place), v of eight values,
// place(k) where v[k] lies.  A
// batch is asked for before the one ahead of it is used (four batches ahead: 272 us for 260, the
// registers spill).  kDown: the last first, so that a pass begins with what the one before it read
// last (512 rows of 131072 with top-k: 111 us for 123).  (-inf in the place of what is not there.)
constexpr int kBatch = 8, kBatchStep = 32 * kBatch;
template <bool kBf16, bool kDown, typename F>
__device__ __forceinline__ void batches(F f) {
    const Shared& g = shared();
    const int lane = static_cast<int>(lane_id()), from = static_cast<int>(warp_id()) * g.per_warp;
    const int to = min(g.end, from + g.per_warp), begin = g.begin;
    // whole batches in loads of four: from 4 lane on and 128 further on
    const int skip = from < begin ? kBatchStep : 0, whole = max(0, to - from) / kBatchStep * kBatchStep;
    const int n = max(0, whole - skip) / kBatchStep;
    using Raw = typename std::conditional<kBf16, uint2, uint4>::type;
    const Raw* src = reinterpret_cast<const Raw*>(static_cast<const uint8_t*>(g.row) + static_cast<int64_t>(from + skip) * (kBf16 ? 2 : 4)) + lane +
                     (kDown ? (n - 1) * 64 : 0);
    Raw a, b;
    if (n) a = __ldg(src), b = __ldg(src + 32);
#pragma unroll 1
    for (int i = n; i > 0; --i) {
        float v[kBatch];
        if constexpr (kBf16) {
            const uint32_t w[4] = {a.x, a.y, b.x, b.y};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                v[2 * k] = __uint_as_float(w[k] << 16);
                v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
            }
        } else {
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(w[k]);
        }
        src += kDown ? -64 : 64;
        if (i > 1) a = __ldg(src), b = __ldg(src + 32);
        f(v, [&](int k) { return from + skip + (kDown ? i - 1 : n - i) * kBatchStep + 128 * (k >> 2) + 4 * lane + (k & 3); });
    }
    // the first (where the row starts inside it) and the last
#pragma unroll 1
    for (int at = skip ? from : from + whole; at < to; at = max(at + kBatchStep, from + whole)) {
        float v[kBatch];
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = at + lane + 32 * k;
            v[k] = __int_as_float(0xff800000);
            if (i < begin || i >= to) continue;
            if (kBf16) v[k] = __uint_as_float(static_cast<uint32_t>(__ldg(static_cast<const uint16_t*>(g.row) + i)) << 16);
            else v[k] = __ldg(static_cast<const float*>(g.row) + i);
        }
        f(v, [&](int k) { return at + lane + 32 * k; });
    }
}
// The same for either type.
template <bool kDown, typename F>
__device__ __forceinline__ void all_batches(F f) {
    if (shared().bf16) batches<true, kDown>(f);
    else batches<false, kDown>(f);
}

// Sum of the weights of this thread's values above `floor`; *ties: how many equal it.
__device__ __noinline__ uint64_t sum_weights(float floor, uint32_t* ties) {
    const Scale scale = scale_of();
    uint64_t sum = 0;
    uint32_t same = 0;
    all_batches<true>([&](const float (&v)[kBatch], auto) {
        float most = v[0];
#pragma unroll
        for (int k = 1; k < kBatch; ++k) most = fmaxf(most, v[k]);
        if (!__any_sync(0xffffffffu, most >= floor)) return;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            same += v[k] == floor ? 1u : 0u;
            const Product w = weight_parts(v[k], scale);
            sum += static_cast<uint64_t>(v[k] > floor ? w.a : 0u) * w.b;
        }
    });
    *ties = same;
    return sum;
}
// The same of the values that this CTA brought to the list, those of a warp by the warp.
__device__ __noinline__ uint64_t sum_listed(float floor, uint32_t* ties) {
    const Shared& g = shared();
    const int n = static_cast<int>(g.counts[g.rank]), at = static_cast<int>(g.rank) * (kListSize / static_cast<int>(g.n));
    uint64_t sum = 0;
    uint32_t same = 0;
#pragma unroll 1
    for (int i = static_cast<int>(lane_id()); i < n; i += 32) {
        const float x = g.list[at + i];
        if (g.warp_of[i] != warp_id() || !(x >= floor)) continue;
        if (x > floor) sum += weight(x, scale_of());
        else ++same;
    }
    *ties = same;
    return sum;
}

// The number of this thread's values by step, up to `last`, into the histogram.
__device__ __noinline__ void count_steps(int last) {
    Shared& g = shared();
    const float top = g.top, c_hi = g.c_hi;
    uint32_t* h = g.sel.hist[g.turn][0];
    all_batches<true>([&](const float (&v)[kBatch], auto) {
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const uint32_t s = step_of(v[k], top, c_hi);
            if (s <= static_cast<uint32_t>(last)) atomicAdd(h + s, 1u);
        }
    });
}

// Sum over the cluster of what all threads have, told in slot `slot`: the first half before a
// cluster_sync, the second behind it.
__device__ __noinline__ void tell_sum(int slot, uint64_t mine) {
    Shared& g = shared();
    uint64_t all;
    __syncthreads();
    block_scan(mine, g.sel.warp, &all);
    tell(g.sel, slot, all, g.n, g.rank);
}
__device__ __forceinline__ uint64_t told_sum(int slot) {
    const Shared& g = shared();
    uint64_t all = 0;
    for (uint32_t i = 0; i < g.n; ++i) all += g.sel.xch[slot][i];
    return all;
}

// The cluster's sums of this thread's bins of the histogram in use, which is then the other one.
struct Bins {
    uint64_t v[kSelPerThread];
};
__device__ __noinline__ Bins merge_bins(bool wide, bool local) {
    Shared& g = shared();
    Bins b;
    const int turn = g.turn;
    if (wide) hist_merge<true>(g.sel, turn, local ? g.rank : 0, local ? 1 : g.n, b.v);
    else hist_merge<false>(g.sel, turn, local ? g.rank : 0, local ? 1 : g.n, b.v);
    return b;
}
// The first bin whose running sum reaches the target (bins_find); the histograms change places.
struct Found {
    uint64_t before, total, own;
    int bin;                   // -1: the whole does not reach it
};
__device__ __noinline__ Found find_bin(const Bins& b, uint64_t target) {
    Shared& g = shared();
    Found f;
    const bool in = bins_find(g.sel, b.v, [&](uint64_t) { return target; }, &f.total);
    f.bin = in ? static_cast<int>(g.sel.found[0]) : -1;
    f.before = g.sel.found[1];
    f.own = g.sel.found[2];
    __syncthreads();
    return f;
}
__device__ __forceinline__ Bins next_bins(bool wide, bool local) {
    if (local) __syncthreads();
    else cluster_sync();
    const Bins b = merge_bins(wide, local);
    __syncthreads();
    if (threadIdx.x == 0) shared().turn ^= 1;
    __syncthreads();
    return b;
}

// Bring the values in [low, high] to every CTA; false if they are too many.  kSums: the weights of
// all values summed into *total, of those above high into *before (each warp's left in
// warp_before).
template <bool kSums>
__device__ __noinline__ bool gather(float low, float high, uint64_t* before, uint64_t* total) {
    Shared& g = shared();
    const Scale scale = scale_of();
    const int per_rank = kListSize / static_cast<int>(g.n);
    uint64_t sum = 0, sum_before = 0;
    all_batches<!kSums>([&](const float (&v)[kBatch], auto place) {
        float most = __int_as_float(0xff800000);          // of those that are not above high
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const bool above = v[k] > high;
            most = fmaxf(most, above ? most : v[k]);
            if (kSums) {
                const uint64_t w = weight(v[k], scale);
                sum += w;
                if (above) sum_before += w;
            }
        }
        if (!__any_sync(0xffffffffu, most >= low)) return;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            if (!(v[k] >= low && v[k] <= high)) continue;
            const int at = atomicAdd(&g.listed, 1);
            if (at >= per_rank) continue;
            g.list[g.rank * per_rank + at] = v[k];
            g.token_of[g.rank * per_rank + at] = g.base + place(k);
            g.warp_of[at] = static_cast<uint8_t>(warp_id());
        }
    });
    if (kSums) {
        tell_sum(1, sum);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum_before += __shfl_xor_sync(0xffffffffu, sum_before, o);
        if (lane_id() == 0) g.warp_before[warp_id()] = sum_before;
    }
    __syncthreads();
    const int mine = min(g.listed, per_rank), at = static_cast<int>(g.rank) * per_rank;
    for (uint32_t r = 0; r < g.n; ++r) {
        if (r == g.rank) continue;
        for (int i = static_cast<int>(threadIdx.x); i < mine; i += kSelThreads) {
            st_cluster_f32(mapa_shared(smem_u32(&g.list[at + i]), r), g.list[at + i]);
            if (!kSums) st_cluster_f32(mapa_shared(smem_u32(&g.token_of[at + i]), r), __int_as_float(g.token_of[at + i]));
        }
    }
    if (kSums) {
        uint64_t all = 0;
        for (int w = 0; w < kSelWarps; ++w) all += g.warp_before[w];
        tell(g.sel, 3, all, g.n, g.rank);
    }
    tell(g.sel, 2, static_cast<uint64_t>(g.listed), g.n, g.rank);
    cluster_sync();
    bool fits = true;
    for (uint32_t r = 0; r < g.n; ++r) fits = fits && g.sel.xch[2][r] <= static_cast<uint64_t>(per_rank);
    if (kSums) *before = told_sum(3), *total = told_sum(1);
    if (threadIdx.x == 0) g.listed = 0;
    if (threadIdx.x < g.n) g.counts[threadIdx.x] = static_cast<uint32_t>(g.sel.xch[2][threadIdx.x]);
    __syncthreads();
    return fits;
}

// The place in descending order of the values above `floor` where the running sum of their
// weights (mass; else their number) reaches the target.  list: among the gathered values, which
// every CTA has; else among the row's.  [lo, hi]: keys that the place may have, with nothing in
// them that comes after the whole set and before its end.
struct Place {
    uint32_t key;              // of the place
    uint64_t rest, own;        // what is missing after everything above the key; the sum of those that equal it
    uint64_t total;            // of all
    bool in;                   // the whole reaches the target (else key, rest and own are nothing's)
};
__device__ __noinline__ Place find_key(bool mass, bool list, uint32_t lo, uint32_t hi, float floor, uint64_t target) {
    Shared& g = shared();
    const Scale scale = scale_of();
    const int stride = kListSize / static_cast<int>(g.n);
    auto each_listed = [&](auto f) {
        for (int r = 0; r < static_cast<int>(g.n); ++r)
#pragma unroll 1
            for (int i = static_cast<int>(threadIdx.x); i < static_cast<int>(g.counts[r]); i += kSelThreads) f(g.list[r * stride + i]);
    };
    constexpr int kFew = 32;
    Place p = {};
    p.rest = target;
    for (bool first = true;; first = false) {
        const int shift = max(0, 21 - __clz(hi - lo));
        uint32_t(*h)[kSelBins] = g.sel.hist[g.turn];
        auto add = [&](float x) {
            const uint32_t key = float_key(x);
            if (key < lo || key > hi || !(x > floor)) return;
            const int bin = static_cast<int>((hi - key) >> shift);
            if (!mass) {
                hist_add<false>(h, bin, 1);
            } else {
                const uint64_t w = weight(x, scale);
                if (w) hist_add<true>(h, bin, w);
            }
        };
        if (list) {
            each_listed(add);
        } else {
#pragma unroll 1
            for (int i = g.begin + static_cast<int>(threadIdx.x); i < g.end; i += kSelThreads) add(value_at(i));
        }
        const Found f = find_bin(next_bins(mass, list), p.rest);
        if (first) p.total = f.total;
        p.in = f.bin >= 0;
        if (!p.in) return p;
        p.rest -= f.before;
        hi -= static_cast<uint32_t>(f.bin) << shift;
        if (shift == 0) {
            p.key = hi;
            p.own = f.own;
            return p;
        }
        lo = max(lo, hi - ((1u << shift) - 1));
        if (!list) continue;
        // few values of the list are left, mostly: compared each with each (64 rows of 100003: 44 us for 50)
        each_listed([&](float x) {
            const uint32_t key = float_key(x);
            if (key < lo || key > hi || !(x > floor)) return;
            const uint64_t w = mass ? weight(x, scale) : 1;
            const int at = w ? atomicAdd(&g.listed, 1) : kFew;
            if (at < kFew) g.pair[at] = make_ulonglong2(key, w);
        });
        __syncthreads();
        const int m = g.listed;
        if (static_cast<int>(threadIdx.x) < min(m, kFew)) {
            const ulonglong2 mine = g.pair[threadIdx.x];
            uint64_t above = 0, own = 0;
#pragma unroll 1
            for (int j = 0; j < min(m, kFew); ++j) {
                if (g.pair[j].x > mine.x) above += g.pair[j].y;
                if (g.pair[j].x == mine.x) own += mine.y;
            }
            if (above < p.rest && p.rest <= above + own) {
                g.place[0] = mine.x;
                g.place[1] = p.rest - above;
                g.place[2] = own;
            }
        }
        __syncthreads();
        p.key = static_cast<uint32_t>(g.place[0]);
        if (m <= kFew) p.rest = g.place[1], p.own = g.place[2];
        __syncthreads();
        if (threadIdx.x == 0) g.listed = 0;
        if (m <= kFew) return p;
    }
}

// The value where step `last` ends or, with a step more for the roundings, is certainly over; the
// smallest that is finite if that is further down.
__device__ __forceinline__ float step_end(float last) {
    const Shared& g = shared();
    return fmaxf(g.top - (last + 0.5f) * ((1.0f / 64.0f) / g.c_hi), -3.4028235e38f);
}
__device__ __forceinline__ float step_over(int last) { return step_end(static_cast<float>(last) + 1.5f); }

// What stays of a row: values above the key, and of those equal to it the first `ties`.
struct Cut {
    uint32_t key;
    uint64_t ties;
};
__device__ __forceinline__ float cut_value(const Cut& c) { return key_float(c.key); }
// Everything from the key on: above what comes before it (before +0 that is not -0).
__device__ __forceinline__ Cut cut_from(uint32_t key) { return {key == 0x80000000u ? key - 2 : key - 1, 0}; }

// top_p's target: the share of z, rounded up.
__device__ __forceinline__ uint64_t share_of(uint64_t z, float top_p) {
    const uint64_t part = top_p > 0.0f ? fraction64(top_p) : 0;
    return max(1ull, static_cast<unsigned long long>(__umul64hi(z, part) + (z * part != 0)));
}
// top_p's cut within top_k's: at the place found among what lies above it, or among its equals, of
// which `missing` is still needed.
__device__ __noinline__ Cut mass_cut(Cut cut, const Place& p, uint64_t missing) {
    const uint64_t w = weight_of(key_float(p.in ? p.key : cut.key));
    if (p.in) cut.key = p.key;
    if (w) cut.ties = p.in ? (p.rest + w - 1) / w : min(cut.ties, (missing + w - 1) / w);
    return p.in && w && cut.ties * w >= p.own ? cut_from(p.key) : cut;
}

// The listed values, m <= kPairs of them, each with its weight, to be compared each with each: thread
// tid looks at value tid / q, with q - 1 neighbours in its warp.
__device__ __forceinline__ int pairs_of(int m) {
    Shared& g = shared();
    const int tid = static_cast<int>(threadIdx.x), stride = kListSize / static_cast<int>(g.n);
    if (tid < m) {
        int r = 0, i = tid;
        while (i >= static_cast<int>(g.counts[r])) i -= static_cast<int>(g.counts[r++]);
        const float x = g.list[r * stride + i];
        g.pair[tid] = make_ulonglong2(static_cast<uint64_t>(float_key(x)) << 32 | ~static_cast<uint32_t>(g.token_of[r * stride + i]),
                                      weight(x, scale_of()));
    }
    return m <= 64 ? 3 : m <= 128 ? 2 : 1;           // log2(q)
}
// Sum over the q neighbours.
__device__ __forceinline__ uint64_t sum_pairs(uint64_t v, int log_q) {
    for (int o = 1; o < 1 << log_q; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The place among the m listed values where the weights reach `target`; false if they do not.
__device__ __noinline__ bool cut_pairs(int m, uint64_t target, Cut* cut) {
    Shared& g = shared();
    const int log_q = pairs_of(m), tid = static_cast<int>(threadIdx.x), e = tid >> log_q;
    if (tid == 0) g.place[3] = 0;
    __syncthreads();
    const uint32_t key = e < m ? static_cast<uint32_t>(g.pair[e].x >> 32) : 0xffffffffu;
    uint64_t above = 0, same = 0;
#pragma unroll 2
    for (int j = tid & ((1 << log_q) - 1); j < m; j += 1 << log_q) {
        const ulonglong2 other = g.pair[j];
        const uint32_t k = static_cast<uint32_t>(other.x >> 32);
        if (k > key) above += other.y;
        if (k == key) same += 1;
    }
    above = sum_pairs(above, log_q), same = sum_pairs(same, log_q);
    const uint64_t w = e < m ? g.pair[e].y : 0;
    // (of equal values every thread writes the same)
    if (w && above < target && target <= above + same * w) {
        const uint64_t ties = (target - above + w - 1) / w;
        const Cut c = ties >= same ? cut_from(key) : Cut{key, ties};
        g.place[0] = c.key;
        g.place[1] = c.ties;
        g.place[3] = 1;
    }
    __syncthreads();
    if (!g.place[3]) return false;
    *cut = {static_cast<uint32_t>(g.place[0]), g.place[1]};
    return true;
}

__device__ __forceinline__ int listed_values() {
    const Shared& g = shared();
    int m = 0;
    for (uint32_t r = 0; r < g.n; ++r) m += static_cast<int>(g.counts[r]);
    return m;
}

// A row's token, x its logit of weight w among kept ones of weight `all`.
__device__ __forceinline__ void give(const SampleParams& p, int64_t r, int token, float x, uint64_t w, uint64_t all) {
    const Shared& g = shared();
    p.token[r] = token;
    if (!p.logp) return;
    // of a share above a half from what is left beside it; else from its logit
    const float rest = static_cast<float>(all - w), whole = static_cast<float>(all);
    const float z = g.ahead + ((x - g.top) * g.c_hi + (x - g.top) * g.c_lo);
    p.logp[r] = w > all / 2 ? log1pf(-rest / whole) : z * 0.693147180559945f - logf(whole * (1.0f / (1ull << kOne)));
}
// The place of u in the sum `all`.
__device__ __forceinline__ uint64_t place_of(float u, uint64_t all) {
    return u >= 1.0f ? all - 1 : u > 0.0f ? __umul64hi(all, fraction64(u)) : 0;
}

// The token among the m <= kPairs listed values that top_k, top_p and a least key leave.  Which come
// before one in descending order, and which of those that stay come before it by index, is told by
// comparing each with each.
__device__ __noinline__ void draw_pairs(const SampleParams& p, int64_t r, float u, int m, uint64_t k, float top_p, uint32_t least) {
    Shared& g = shared();
    const int log_q = pairs_of(m), tid = static_cast<int>(threadIdx.x), e = tid >> log_q, j0 = tid & ((1 << log_q) - 1);
    __syncthreads();
    const ulonglong2 mine = e < m ? g.pair[e] : make_ulonglong2(0, 0);
    uint64_t above = 0, rank = 0;
#pragma unroll 2
    for (int j = j0; j < m; j += 1 << log_q) {
        const ulonglong2 other = g.pair[j];
        if (other.x > mine.x) above += other.y, rank += 1;
    }
    above = sum_pairs(above, log_q), rank = sum_pairs(rank, log_q);
    // what top_k leaves: the sum down to the k-th, or to the last where a mask leaves fewer than k
    if (rank == min(k, static_cast<uint64_t>(m)) - 1 && e < m) g.place[0] = above + mine.y;
    __syncthreads();
    const bool stays = rank < k && (!(top_p < 1.0f) || above < share_of(g.place[0], top_p)) && static_cast<uint32_t>(mine.x >> 32) >= least;
    const uint64_t w = stays ? mine.y : 0;
    if (j0 == 0 && e < m) g.pair[e].y = w;
    __syncthreads();
    uint64_t run = 0, all = 0;
#pragma unroll 2
    for (int j = j0; j < m; j += 1 << log_q) {
        const ulonglong2 other = g.pair[j];
        all += other.y;
        if (static_cast<uint32_t>(other.x) > static_cast<uint32_t>(mine.x)) run += other.y;
    }
    all = sum_pairs(all, log_q), run = sum_pairs(run, log_q);
    const uint64_t at = place_of(u, all);
    if (j0 == 0 && e < m && at >= run && at < run + w)
        give(p, r, static_cast<int>(~static_cast<uint32_t>(mine.x)), key_float(static_cast<uint32_t>(mine.x >> 32)), w, all);
}

// top_k's cut, and top_p's within it, the long way: searched among all values.
__device__ __noinline__ Cut cut_of_all(uint64_t k, float top_p, uint32_t kmax) {
    Cut cut = {kKeyNegInf, ~0ull >> 1};
    if (k) {
        const Place p = find_key(false, false, kKeyNegInf + 1, kmax, key_float(kKeyNegInf), k);
        if (p.in) cut = {p.key, p.rest};
    }
    if (!(top_p < 1.0f)) return cut;
    const float floor = cut_value(cut);
    uint32_t none;
    tell_sum(0, sum_weights(floor, &none));
    cluster_sync();
    const uint64_t above = told_sum(0);
    const uint64_t target = share_of(above + (cut.key > kKeyNegInf ? cut.ties * weight_of(floor) : 0), top_p);
    const Place p = find_key(true, false, cut.key + 1, kmax, floor, target);
    return mass_cut(cut, p, target - p.total);
}

// The cut of top_k (k > 0) and of top_p within it.  *listed: what stays is in the list; none is looked
// for where that is short enough for draw_pairs.
__device__ __noinline__ Cut cut_by_count(uint64_t k, float top_p, float mine_top, uint32_t kmax, bool* listed) {
    Shared& g = shared();
    const uint64_t each = (k + g.full - 1) / g.full;
    float low;
    if (each <= kSelThreads / 4) {
        // down to which value a full CTA's share of k is reached by its threads' largest, by bins from the
        // top to the lowest of them (the steps of the weights would end too soon at low temperatures: 104 us
        // for 14 at 0.3); the smallest of those in the bins down to there
        const float scale = static_cast<float>(kLastBin) / (g.top - g.lowest);
        const bool any = mine_top > __int_as_float(0xff800000);
        const int bin = __float2int_rz(fminf((g.top - mine_top) * scale, static_cast<float>(kLastBin)));
        if (any) atomicAdd(&g.sel.hist[g.turn][0][bin], 1u);
        const Found f = find_bin(next_bins(false, true), each);
        const bool counts = g.rank < g.full;
        const uint32_t mine = __reduce_min_sync(0xffffffffu, counts && any && bin <= f.bin ? float_key(mine_top) : 0xffffffffu);
        if (lane_id() == 0) g.sel.warp2[warp_id()] = mine;
        __syncthreads();
        // (too few threads with a value: everything)
        uint64_t least = counts && f.bin < 0 ? kKeyNegInf + 1 : 0xffffffffu;
        for (int i = 0; i < kSelWarps; ++i) least = min(least, g.sel.warp2[i]);
        tell(g.sel, 1, least, g.n, g.rank);
        cluster_sync();
        for (uint32_t r = 0; r < g.n; ++r) least = min(least, g.sel.xch[1][r]);
        low = key_float(static_cast<uint32_t>(least));
    } else {
        // (so many that all values are counted)
        count_steps(kLastBin);
        const Found f = find_bin(next_bins(false, false), k);
        if (f.bin < 0) return cut_of_all(k, top_p, kmax);
        low = step_over(f.bin);
    }
    if (!gather<false>(low, g.top, nullptr, nullptr)) return cut_of_all(k, top_p, kmax);
    *listed = true;
    const int m = listed_values();
    Cut cut = {kKeyNegInf, 0};
    if (m <= kPairs) return cut;
    const uint32_t lo = float_key(low);
    // (fewer than k above -inf, where a mask leaves no more: all of them stay)
    const Place p = find_key(false, true, lo, kmax, key_float(kKeyNegInf), k);
    if (p.in) cut = p.rest >= p.own ? cut_from(p.key) : Cut{p.key, p.rest};
    if (!(top_p < 1.0f)) return cut;
    const float floor = cut_value(cut);
    // (the sum of what is above the cut: no target reached)
    const uint64_t above = find_key(true, true, lo, kmax, floor, ~0ull).total;
    const uint64_t target = share_of(above + cut.ties * weight_of(floor), top_p);
    return mass_cut(cut, find_key(true, true, lo, kmax, floor, target), target - above);
}

// The cut of top_p alone.  *listed: what stays is in the list or above it, and the weights of
// what is above it are in warp_before.
__device__ __noinline__ Cut cut_by_mass(float top_p, int vocab, uint32_t kmax, bool* listed) {
    Shared& g = shared();
    // A value so light that all values of the row together, if they were like it, would not make up
    // what the share leaves out of the largest one alone is cut: below (1 - top_p) / vocab.  Values
    // of 2^-8 of that are counted too, for the estimate of the sum.
    const float light = (1.0f - fmaxf(top_p, 0.0f)) / static_cast<float>(vocab) * 0.5f;
    const int last_step = min(kLastBin, 64 * (9 - ilogbf(light)));
    count_steps(last_step);
    const Bins count = next_bins(false, false);
    Bins mass;
#pragma unroll
    for (int i = 0; i < kSelPerThread; ++i) mass.v[i] = count.v[i] * step_weight(static_cast<int>(threadIdx.x) * kSelPerThread + i, g.ahead);
    // The counts times the weights of the steps' middles are off by 2^(1/128), less than 2^-7, from the
    // steps' sums: the cut lies in steps [first, last].  Where those hold too many values, single ones
    // weigh little and the counts are much closer than that: a step to each side is enough.
    if (threadIdx.x < 3) g.sel.found[threadIdx.x] = static_cast<uint64_t>(last_step);
    if (threadIdx.x == 3) g.place[0] = 0, g.place[1] = static_cast<uint64_t>(vocab);
    uint64_t all, none;
    uint64_t run = block_scan(mass.v[0] + mass.v[1] + mass.v[2] + mass.v[3], g.sel.warp, &all);
    uint64_t run_count = block_scan(count.v[0] + count.v[1] + count.v[2] + count.v[3], g.sel.warp2, &none);
    uint64_t aim = share_of(all, top_p);
    const uint64_t least = max(1ull, static_cast<unsigned long long>(aim - (aim >> 7) - 1)), most = aim + (aim >> 7) + 1;
#pragma unroll
    for (int i = 0; i < kSelPerThread; ++i) {
        const uint64_t next = run + mass.v[i];
        const uint64_t step = threadIdx.x * kSelPerThread + i;
        if (run < least && least <= next) g.sel.found[0] = step, g.place[0] = run_count;
        run_count += count.v[i];
        if (run < aim && aim <= next) g.sel.found[1] = step;
        if (run < most && most <= next) g.sel.found[2] = step, g.place[1] = run_count;
        run = next;
    }
    __syncthreads();
    int first = static_cast<int>(g.sel.found[0]), mid = static_cast<int>(g.sel.found[1]), last = static_cast<int>(g.sel.found[2]);
    const bool narrow = g.place[1] - g.place[0] > kFewEnough;
    __syncthreads();
    for (int tries = 0; tries < 3; ++tries) {
        if (narrow) {
            if (tries) {
                const Found f = find_bin(mass, aim);
                mid = f.bin < 0 ? last_step : f.bin;
            }
            first = max(0, mid - 1);
            last = min(kLastBin, mid + 1);
        }
        const float low = step_end(static_cast<float>(last)), high = fminf(step_end(static_cast<float>(first - 1)), g.top);
        uint64_t before, total;
        if (!gather<true>(low, high, &before, &total)) break;
        const uint64_t target = share_of(total, top_p);
        if (before < target) {
            const int m = listed_values();
            Cut cut = {kKeyNegInf, ~0ull >> 1};
            bool found;
            if (m <= kPairs) {
                found = cut_pairs(m, target - before, &cut);
            } else {
                const Place p = find_key(true, true, float_key(low), float_key(high), key_float(kKeyNegInf), target - before);
                found = p.in;
                if (found) cut = mass_cut(cut, p, 0);
            }
            if (found) {
                *listed = true;
                return cut;
            }
        }
        if (!narrow) break;
        // what the counts were off by down to there is known now
        uint64_t above = 0;
#pragma unroll
        for (int i = 0; i < kSelPerThread; ++i)
            above += static_cast<int>(threadIdx.x) * kSelPerThread + i < first ? mass.v[i] : 0;
        block_scan(above, g.sel.warp, &all);
        __syncthreads();
        aim = target + all - before;
        if (static_cast<int64_t>(aim) < 1) aim = 1;
        cluster_sync();                      // what was told is read
    }
    return cut_of_all(0, top_p, kmax);
}

// This thread's largest value, NaN if it met one, by the first read of the row, with many loads on
// their way.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __noinline__ float largest() {
    const Shared& g = shared();
    float top[2] = {__int_as_float(0xff800000), __int_as_float(0xff800000)};
    auto see = [&](float a, float b, int k) { top[k] = max3(top[k], a, b); };
    auto see2 = [&](uint32_t w, int k) { see(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u), k); };
    const int lane = static_cast<int>(lane_id()), from = static_cast<int>(warp_id()) * g.per_warp;
    const int to = min(g.end, from + g.per_warp), begin = g.begin;
    constexpr int kDeep = 8;               // steps on their way at once
    const int skip = from < begin ? kStep : 0, whole = max(0, to - from) / kStep * kStep;
    int at = skip;
    if (g.bf16) {
        const uint2* x = reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(g.row) + from) + lane;
#pragma unroll 1
        for (; at + kDeep * kStep <= whole; at += kDeep * kStep) {
            uint2 v[kDeep];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) v[k] = __ldg(x + at / 4 + 32 * k);
#pragma unroll
            for (int k = 0; k < kDeep; ++k) see2(v[k].x, 0), see2(v[k].y, 1);
        }
#pragma unroll 4
        for (; at < whole; at += kStep) {
            const uint2 v = __ldg(x + at / 4);
            see2(v.x, 0), see2(v.y, 1);
        }
    } else {
        const float4* x = reinterpret_cast<const float4*>(static_cast<const float*>(g.row) + from) + lane;
#pragma unroll 1
        for (; at + kDeep * kStep <= whole; at += kDeep * kStep) {
            float4 v[kDeep];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) v[k] = __ldg(x + at / 4 + 32 * k);
#pragma unroll
            for (int k = 0; k < kDeep; ++k) see(v[k].x, v[k].y, 0), see(v[k].z, v[k].w, 1);
        }
#pragma unroll 4
        for (; at < whole; at += kStep) {
            const float4 v = __ldg(x + at / 4);
            see(v.x, v.y, 0), see(v.z, v.w, 1);
        }
    }
    // the first (where the row starts inside it) and the last, one by one
#pragma unroll 4
    for (int i = max(from + whole, begin) + lane; i < to; i += 32) see(value_at(i), top[1], 0);
    if (skip)
        for (int i = begin + lane; i < min(from + kStep, to); i += 32) see(value_at(i), top[1], 0);
    return max3(top[0], top[1], top[1]);
}

__global__ void __launch_bounds__(kSelThreads, 2) sample_kernel(const __grid_constant__ SampleParams p) {
    Shared& g = shared();
    SelShared& sh = g.sel;
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t rank = cluster_ctarank(), n = cluster_nctas();
    const int64_t r = blockIdx.x / n;
    const int tid = static_cast<int>(threadIdx.x), warp = static_cast<int>(warp_id()), lane = static_cast<int>(lane_id());
    float temperature = p.temperature ? p.temperature[r] : p.one.temperature;
    int top_k = p.top_k ? p.top_k[r] : p.one.top_k;
    float top_p = p.top_p ? p.top_p[r] : p.one.top_p;
    float min_p = p.min_p ? p.min_p[r] : p.one.min_p;
    float u = p.uniform[r];
    // a row starts up to three places after one that a load of four may start at; places are shared out
    // in whole steps
    const int64_t row0 = r * p.ld;
    const int lead = static_cast<int>(((reinterpret_cast<uintptr_t>(p.logits) / (p.bf16 ? 2 : 4)) + static_cast<uint64_t>(row0)) & 3u);
    const int per_warp = ((lead + p.vocab + static_cast<int>(n) * kSelWarps - 1) / (static_cast<int>(n) * kSelWarps) + kStep - 1) / kStep * kStep;
    const int base = static_cast<int>(rank) * kSelWarps * per_warp - lead;        // token of the CTA's first place
    if (tid == 0) {
        g.row = static_cast<const uint8_t*>(p.logits) + (row0 + base) * (p.bf16 ? 2 : 4);
        g.bf16 = p.bf16;
        g.per_warp = per_warp;
        g.begin = max(0, -base);
        g.end = max(0, min(p.vocab - base, kSelWarps * per_warp));
        g.base = base;
        // (one thread's reading, and then the first CTA's, for all: what is written meanwhile divides no one)
        g.how[0] = static_cast<uint64_t>(__float_as_uint(temperature)) << 32 | static_cast<uint32_t>(top_k);
        g.how[1] = static_cast<uint64_t>(__float_as_uint(top_p)) << 32 | __float_as_uint(min_p);
        g.how[2] = __float_as_uint(u);
        g.listed = 0;
        g.turn = 0;
        g.rank = rank;
        g.n = n;
        g.full = static_cast<uint32_t>(max(1, (lead + p.vocab) / (kSelWarps * per_warp)));
    }
    __syncthreads();
    const float mine_top = largest();
    if (tid < 16) g.table[tid] = make_uint2(kExpTable[tid], __float_as_uint(__uint2float_rn(kExpTable[tid])));
    if (tid == 64) {
        const double c = 1.4426950408889634 / static_cast<double>(fmaxf(temperature, 0x1p-127f));     // (finite in fp32)
        g.c_hi = static_cast<float>(c);
        g.c_lo = static_cast<float>(c - static_cast<double>(g.c_hi));
        g.least = min_p > 0.0f ? static_cast<double>(temperature) * log(fmin(static_cast<double>(min_p), 1.0)) : 0.0;
    }
    *reinterpret_cast<uint4*>(&sh.hist[0][0][tid * kSelPerThread]) = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(&sh.hist[0][1][tid * kSelPerThread]) = make_uint4(0, 0, 0, 0);
    const uint32_t most = __reduce_max_sync(0xffffffffu, mine_top != mine_top ? 0xffffffffu : float_key(mine_top));
    const uint32_t fewest = __reduce_min_sync(0xffffffffu, mine_top > __int_as_float(0xff800000) ? float_key(mine_top) : 0xffffffffu);
    if (lane == 0) sh.warp[warp] = most, sh.warp2[warp] = fewest;
    cluster_sync();                             // (every CTA has started, and this one's are in sh.warp)
    uint64_t told = 0;
#pragma unroll
    for (int i = 0; i < kSelWarps; ++i) told = max(told, sh.warp[i]);
    if (n > 1) {
        tell(sh, 0, told, n, rank);
        if (rank == 0 && tid >= 1 && tid < static_cast<int>(n))
            for (int i = 0; i < 3; ++i) st_cluster_u64(mapa_shared(smem_u32(&g.how[i]), static_cast<uint32_t>(tid)), g.how[i]);
        cluster_sync();
        for (uint32_t i = 0; i < n; ++i) told = max(told, sh.xch[0][i]);
    }
    temperature = __uint_as_float(static_cast<uint32_t>(g.how[0] >> 32)), top_k = static_cast<int>(g.how[0]);
    top_p = __uint_as_float(static_cast<uint32_t>(g.how[1] >> 32)), min_p = __uint_as_float(static_cast<uint32_t>(g.how[1]));
    u = __uint_as_float(static_cast<uint32_t>(g.how[2]));
    const uint32_t kmax = static_cast<uint32_t>(told);
    // no largest logit, or no temperature: no token
    if (kmax >= kKeyPosInf || kmax <= kKeyNegInf || !(temperature >= 0.0f && temperature <= 3.4028235e38f)) {
        if (rank == 0 && tid == 0) {
            p.token[r] = -1;
            if (p.logp) p.logp[r] = __int_as_float(0x7fc00000);
        }
        return;
    }
    const float top = key_float(kmax);
    if (tid == 0) {
        uint64_t least = kmax;
#pragma unroll
        for (int i = 0; i < kSelWarps; ++i) least = min(least, sh.warp2[i]);
        g.top = top;
        g.lowest = key_float(static_cast<uint32_t>(least));
        // R: from 1/16 to 1/8 above the product, whose roundings are less than the 1/16
        const float p = top * g.c_hi, up = fabsf(p) < 131072.0f ? ceilf(p * 16.0f) * 0.0625f + 0.0625f : 0.0f;
        g.shift = fabsf(p) < 131072.0f ? 0.0f : top;
        g.zero = kRound16 - up;
        g.ahead = g.shift == 0.0f ? fmaf(top, g.c_hi, -up) + top * g.c_lo : 0.0f;
    }
    __syncthreads();
    Cut cut = {kKeyNegInf, ~0ull >> 1};
    bool listed = false, above_list = false;    // what stays is in the list, or above it
    if (temperature == 0.0f) {
        cut = {kmax, 1};
    } else {
        if (top_k > 0 && top_k < p.vocab) cut = cut_by_count(static_cast<uint64_t>(top_k), top_p, mine_top, kmax, &listed);
        else if (top_p < 1.0f) cut = cut_by_mass(top_p, p.vocab, kmax, &listed), above_list = listed;
        const uint32_t least = min_p > 0.0f ? min(kmax, float_key(__double2float_ru(static_cast<double>(top) + g.least))) : 0;
        if (listed && !above_list) {
            const int m = listed_values();
            if (m <= kPairs) {
                if (rank == 0) draw_pairs(p, r, u, m, static_cast<uint64_t>(top_k), top_p, least);
                return;
            }
        }
        if (least > cut.key) {
            cut = cut_from(least);
            listed = listed && !above_list;
        }
    }

    // sums over what stays: of this CTA's warps, then of the cluster's CTAs
    const float floor = cut_value(cut);
    uint32_t ties;
    uint64_t sum = listed ? sum_listed(floor, &ties) : sum_weights(floor, &ties);
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    ties = __reduce_add_sync(0xffffffffu, ties);
    __syncthreads();
    if (lane == 0) {
        sh.warp[warp] = sum + (listed && above_list ? g.warp_before[warp] : 0);
        sh.warp2[warp] = ties;
    }
    __syncthreads();
    uint64_t cta_sum = 0, cta_ties = 0;
#pragma unroll
    for (int i = 0; i < kSelWarps; ++i) {
        cta_sum += sh.warp[i];
        cta_ties += sh.warp2[i];
    }
    tell(sh, 4, cta_sum, n, rank);
    tell(sh, 5, cta_ties, n, rank);
    cluster_sync();
    const uint64_t w_tie = cut.key > kKeyNegInf && cut.ties ? weight_of(floor) : 0;
    // weight of the first of the ties that come after `before` of them
    auto tie_part = [&](uint64_t before, uint64_t count) -> uint64_t {
        return before >= cut.ties ? 0 : min(count, cut.ties - before) * w_tie;
    };
    // the place that u names among them: first of the cluster's CTAs, then of this one's warps, in lanes
    // 0 .. 15 side by side
    auto scan16 = [&](uint64_t v) {              // sum of lanes before this one
        uint64_t x = v;
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
            const uint64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        return x - v;
    };
    const bool there = lane < static_cast<int>(n);
    uint64_t part = there ? sh.xch[4][lane] : 0, same = there ? sh.xch[5][lane] : 0;
    uint64_t same_before = w_tie ? scan16(same) : 0;
    part += tie_part(same_before, same);
    uint64_t start = scan16(part);
    const uint64_t all = __shfl_sync(0xffffffffu, start + part, static_cast<int>(n) - 1);
    const uint64_t at = place_of(u, all);
    start = __shfl_sync(0xffffffffu, start, static_cast<int>(rank));
    uint64_t ties_before = __shfl_sync(0xffffffffu, same_before, static_cast<int>(rank));
    part = lane < kSelWarps ? sh.warp[lane] : 0;
    same = lane < kSelWarps ? sh.warp2[lane] : 0;
    same_before = w_tie ? ties_before + scan16(same) : 0;
    part += tie_part(same_before, same);
    const uint64_t run0 = start + scan16(part);
    // the warp whose values hold it; the CTA takes those up again, some next to one another a thread
    const int owner = __ffs(__ballot_sync(0xffffffffu, lane < kSelWarps && at >= run0 && at < run0 + part)) - 1;
    if (owner < 0) return;
    start = __shfl_sync(0xffffffffu, run0, owner);
    ties_before = __shfl_sync(0xffffffffu, same_before, owner);
    const int each = (per_warp + kSelThreads - 1) / kSelThreads;
    const int place = owner * per_warp + tid * each, from = max(g.begin, place);
    const int to = min(g.end, min((owner + 1) * per_warp, place + each));
    const Scale scale = scale_of();
    uint64_t mine = 0, total;
    uint32_t tied = 0;
    for (int i = from; i < to; ++i) {
        const float v = value_at(i);
        if (v > floor) mine += weight(v, scale);
        tied += v == floor ? 1u : 0u;
    }
    __syncthreads();                            // sh.warp is read
    uint64_t run_ties = ties_before;
    if (w_tie) {
        run_ties += block_scan(tied, sh.warp, &total);
        __syncthreads();
        mine += tie_part(run_ties, tied);
    }
    uint64_t run = start + block_scan(mine, sh.warp, &total);
    if (at < run || at >= run + mine) return;
    for (int i = from; i < to; ++i) {
        const float v = value_at(i);
        uint64_t w = v > floor ? weight(v, scale) : 0;
        if (v == floor) w = tie_part(run_ties++, 1);
        run += w;
        if (at >= run) continue;
        give(p, r, base + i, v, w, all);
        return;
    }
}

}  // namespace

// (so that the sum of a row's weights fits 64 bits)
int64_t sample_max_vocab() { return (1 << (64 - kOne)) - 1; }

cr_status launch_sample(const SampleParams& p, cudaStream_t st) {
    // (one wave of CTAs: 64 rows of 100003 took 49 us with four CTAs each, 52 with two, 170 with eight)
    int ranks = kMaxCluster;
    while (ranks > 1 && (static_cast<int64_t>(p.n_rows) * ranks > 2 * num_sms() || p.vocab < ranks * kLeast)) ranks /= 2;
    static unsigned long long attr_done = 0;
    const cr_status s = ensure_smem_attr(sample_kernel, sizeof(Shared), &attr_done);
    if (s != CR_OK) return s;
    return launch_cluster(sample_kernel, dim3(static_cast<unsigned>(p.n_rows * ranks)), dim3(kSelThreads), ranks, sizeof(Shared), st, p);
}

}  // namespace cr
