// Drawing the next token of every row of logits with a given uniform number:
//   w_i = exp((x_i - max x) / T),
//   kept = the top_k largest, of these the shortest run in descending order whose
//          predecessors' share of the sum stays below top_p, of these w_i >= min_p,
//   token = the first kept i, in the order of the vocabulary, with sum_{j <= i} w_j > u sum w.
// Equal logits are ranked by index.
//
// A row lies in the shared memory of a cluster of CTAs, read once.  Both cuts are places in
// descending order where a running sum (of ones, or of w) passes a target; nothing is sorted.
// Values are told apart by the step of 2^(1/64) that their w falls into.  The threads' largest
// values alone bound a cut from below (k of them reach the k-th value), so that a top_k cut is
// found among little more than k values, told to every CTA of the cluster; for top_p alone a
// histogram of the steps brackets the cut to within 2^-7 of the sum, and the values of those
// steps, mostly a few hundred, give the exact place.
//
// The answer turns on where u times a sum falls among up to 2^18 partial sums, so the weights
// are integers in units of 2^-44 of the largest, good to about 2^-28 of themselves, and their
// sums are exact and the same in any order.
#include "cr_cluster.cuh"
#include "cr_internal.h"

namespace cr {
namespace {

constexpr int kOne = 44;               // the largest weight is 2^44
constexpr int kVec = 4;                // values a thread takes together
constexpr int kStep = 32 * kVec;       // values a warp takes together
constexpr int kMaxChunk = 44 * 1024;   // values of a row in one CTA
constexpr int kChunk = 16 * 1024;      // of those, so that two CTAs share an SM
constexpr int kListSize = 2048;        // values of a row that a cut is searched among, an equal part for each CTA

// 2^(j / 64), j = 0 .. 63, in units of 2^-28.
__constant__ uint32_t kExpTable[64] = {
    268435456, 271358526, 274313427, 277300504, 280320109, 283372595, 286458320, 289577647, 292730940, 295918571, 299140913,
    302398344, 305691246, 309020006, 312385013, 315786663, 319225354, 322701490, 326215479, 329767733, 333358668, 336988706,
    340658272, 344367798, 348117717, 351908471, 355740503, 359614263, 363530205, 367488790, 371490480, 375535746, 379625062,
    383758908, 387937769, 392162134, 396432500, 400749367, 405113241, 409524635, 413984066, 418492057, 423049137, 427655840,
    432312707, 437020283, 441779122, 446589781, 451452825, 456368824, 461338355, 466362000, 471440350, 476573998, 481763549,
    487009610, 492312797, 497673732, 503093043, 508571368, 514109347, 519707630, 525366875, 531087746};

struct RowScale {
    float hi, lo;          // c = log2(e) / T in two parts
    double least;          // T log(min_p): the smallest x - max that min_p keeps
};
constexpr float kRound = 12582912.0f;              // 1.5 2^23: adding it rounds to an integer
constexpr int kRoundBits = 0x4b400000;             // as an integer
constexpr int kFarStep = 64 * (kOne + 1);          // from this step on a value weighs nothing

// How far below the largest x lies, in steps of 2^(1/64) of the weight: does not fall as x falls.
__device__ __forceinline__ float steps_rounded(float d, const RowScale& sc) {
    return fmaf(fmaxf(d * sc.hi, -1e4f), 64.0f, kRound);
}
__device__ __forceinline__ int step_of(float x, float top, const RowScale& sc) {
    return kRoundBits - __float_as_int(steps_rounded(x - top, sc));
}
// Integer weight of the middle of a step.
__device__ __forceinline__ uint64_t step_weight(int step, const uint2* table) {
    return static_cast<uint64_t>(table[-step & 63].x + kRoundBits) << (kOne - 28) >> ((step + 63) >> 6);
}
// Integer weight of x.  With t = (x - max) log2(e) / T = k / 64 + f, k the (negative) step,
// |f| <= 1/128, the difference formed exactly by FMA and c in two parts:
// 2^t = 2^floor(k / 64) T[k mod 64] (1 + y), y = 2^f - 1 by its series (y < 2^-7.5, so its fp32
// rounding is 2^-31 of the weight).  table: T in units of 2^-28 less kRoundBits, and as a float.
__device__ __forceinline__ uint64_t weight(float x, float top, const RowScale& sc, const uint2* table) {
    const float d = x - top;
    const float r = steps_rounded(d, sc);
    const int step = kRoundBits - __float_as_int(r);
    if (step >= kFarStep) return 0;
    const float f = fmaf(d, sc.lo, fmaf(d, sc.hi, (r - kRound) * (-1.0f / 64.0f)));
    // 2^f - 1 = f ln 2 + (f ln 2)^2 / 2 + ...
    const float y = f * fmaf(f, fmaf(f, fmaf(f, 9.61812911e-3f, 5.55041087e-2f), 2.40226507e-1f), 6.93147181e-1f);
    const uint2 t = table[-step & 63];
    const uint32_t w = t.x + static_cast<uint32_t>(__float_as_int(fmaf(__uint_as_float(t.y), y, kRound)));
    return (static_cast<uint64_t>(w) << (kOne - 28)) >> ((step + 63) >> 6);
}

// 2^64 v for v in [0, 1), exact down to 2^-40.
__device__ __forceinline__ uint64_t fraction64(float v) {
    const uint32_t b = __float_as_uint(v);
    const int s = static_cast<int>(b >> 23) - 86;
    const uint64_t m = (b & 0x7fffffu) | 0x800000u;
    return s >= 0 ? m << s : s > -24 ? m >> -s : 0;
}

struct Row {
    const float* x;            // this CTA's values, a warp's together
    int base, per_warp;        // index in the row of this warp's first value, and how many it has
    int vocab;
};
// All of this thread's values, four at a time: f(value, index in the row).
template <typename F>
__device__ __forceinline__ void each(const Row& r, F f) {
    const int lane = static_cast<int>(lane_id());
    const float* x = r.x + static_cast<int>(warp_id()) * r.per_warp;
    for (int i = lane * kVec; i < r.per_warp; i += kStep) {
        if (r.base + i >= r.vocab) break;
        const float4 v = *reinterpret_cast<const float4*>(x + i);
        f(v.x, r.base + i);
        f(v.y, r.base + i + 1);
        f(v.z, r.base + i + 2);
        f(v.w, r.base + i + 3);
    }
}

// What stays of a row: values above the key, and of those equal to it the first `ties`.
struct Cut {
    uint32_t key;
    uint64_t ties;
};

// The place in descending order of a set of values with keys in [lo, hi] where the running sum
// of value(x) reaches the target; false if the whole does not.  cut->ties is what is still
// missing after everything above cut->key.  all(f) calls f(x) for this CTA's values: all of the
// set (kLocal), or its part of the cluster's.
template <bool kWide, bool kLocal, typename A, typename V, typename T>
__device__ __forceinline__ bool find_key(SelShared& sh, int& turn, uint32_t rank, uint32_t n, uint32_t lo, uint32_t hi, A all,
                                         V value, T target_of, Cut* cut, uint64_t* total) {
    uint64_t rest = 0;
    for (bool first = true;; first = false) {
        const int shift = max(0, 21 - __clz(hi - lo));
        all([&](float x) {
            const uint32_t key = float_key(x);
            if (key < lo || key > hi) return;
            const uint64_t v = value(x);
            if (v) hist_add<kWide>(sh.hist[turn], static_cast<int>((hi - key) >> shift), v);
        });
        if (kLocal) __syncthreads();
        else cluster_sync();
        uint64_t sum;
        const bool reached = hist_find<kWide>(sh, turn, kLocal ? rank : 0, kLocal ? 1 : n,
                                              [&](uint64_t s) { return first ? rest = target_of(s) : rest; }, &sum);
        turn ^= 1;
        if (first) *total = sum;
        if (!reached) return false;
        rest -= sh.found[1];
        hi -= static_cast<uint32_t>(sh.found[0]) << shift;
        if (kLocal) __syncthreads();            // sh.found is read
        if (shift == 0) break;
        lo = max(lo, hi - ((1u << shift) - 1));
    }
    cut->key = hi;
    cut->ties = rest;
    return true;
}

// The same for all values above `floor`, which may lie anywhere: first by equal steps of x.
template <bool kWide, typename V, typename T>
__device__ __forceinline__ bool find_cut(SelShared& sh, int& turn, uint32_t rank, uint32_t n, const Row& row, float top, float least,
                                         uint32_t floor, V value, T target_of, Cut* cut, uint64_t* total) {
    const float range = top - least;
    const float s = range > 1e-30f && range < 3e38f ? (kSelBins - 1) / range : 0.0f;   // (0: one step holds all)
    auto bin_of = [&](float x) { return min(kSelBins - 1, static_cast<int>((top - x) * s)); };
    each(row, [&](float x, int) {
        if (float_key(x) <= floor) return;
        const uint64_t v = value(x);
        if (v) hist_add<kWide>(sh.hist[turn], bin_of(x), v);
    });
    cluster_sync();
    uint64_t target = 0;
    const bool reached = hist_find<kWide>(sh, turn, 0, n, [&](uint64_t all) { return target = target_of(all); }, total);
    turn ^= 1;
    if (!reached) return false;
    const int bin0 = static_cast<int>(sh.found[0]);
    const uint64_t rest = target - sh.found[1];
    // keys that the step's values may have: a step more on both sides, for the roundings
    uint32_t lo = float_key(least), hi = float_key(top);
    if (s > 0.0f) {
        const float w = range / (kSelBins - 1);
        hi = min(hi, float_key(top - static_cast<float>(bin0 - 1) * w));
        if (bin0 < kSelBins - 1) lo = max(lo, float_key(top - static_cast<float>(bin0 + 2) * w));
    }
    uint64_t in_step;
    return find_key<kWide, false>(
        sh, turn, rank, n, lo, hi, [&](auto f) { each(row, [&](float x, int) { f(x); }); },
        [&](float x) -> uint64_t { return float_key(x) > floor && bin_of(x) == bin0 ? value(x) : 0; },
        [&](uint64_t) { return rest; }, cut, &in_step);
}

// Keys that values of the steps (above, last] may have: a step more on both sides, for the
// roundings.
__device__ __forceinline__ uint32_t step_key_hi(int above, float top, uint32_t kmax, const RowScale& sc) {
    return min(kmax, float_key(top - static_cast<float>(above - 1) * ((1.0f / 64.0f) / sc.hi)));
}
__device__ __forceinline__ uint32_t step_key_lo(int last, float top, const RowScale& sc) {
    return float_key(top - static_cast<float>(last + 2) * ((1.0f / 64.0f) / sc.hi));
}

template <bool kBf16, bool kAligned>
__global__ void __launch_bounds__(kSelThreads, 2) sample_kernel(const __grid_constant__ SampleParams p) {
    extern __shared__ float4 values[];
    __shared__ __align__(16) SelShared sh;
    __shared__ uint2 table[64];
    __shared__ RowScale scale;
    __shared__ float list[kListSize];
    __shared__ int listed;
    float* x = reinterpret_cast<float*>(values);
    pdl_launch_dependents();
    pdl_wait();
    const uint32_t rank = cluster_ctarank(), n = cluster_nctas();
    const int64_t r = blockIdx.x / n;
    const int tid = static_cast<int>(threadIdx.x), warp = static_cast<int>(warp_id()), lane = static_cast<int>(lane_id());
    const float temperature = p.temperature ? p.temperature[r] : p.one.temperature;
    const int top_k = p.top_k ? p.top_k[r] : p.one.top_k;
    const float top_p = p.top_p ? p.top_p[r] : p.one.top_p;
    const float min_p = p.min_p ? p.min_p[r] : p.one.min_p;
    const float u = p.uniform[r];
    Row row;
    row.x = x;
    row.vocab = p.vocab;
    row.per_warp = ((p.vocab + static_cast<int>(n) * kSelWarps - 1) / (static_cast<int>(n) * kSelWarps) + kStep - 1) / kStep * kStep;
    row.base = (static_cast<int>(rank) * kSelWarps + warp) * row.per_warp;
    const float ninf = __int_as_float(0xff800000);

    // the row into shared memory; its largest value and its smallest above -inf
    float top = ninf, least = -ninf;
    bool nan = false;
    {
        float* dst = x + warp * row.per_warp;
        auto put = [&](int i, const float (&v)[kVec]) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                nan = nan || v[e] != v[e];
                top = fmaxf(top, v[e]);
                least = fminf(least, v[e] == ninf ? -ninf : v[e]);
            }
            *reinterpret_cast<float4*>(dst + i) = make_float4(v[0], v[1], v[2], v[3]);
        };
        int i = lane * kVec;
        if (kAligned) {
            // several steps on their way at once
            constexpr int kDeep = 8;
            const int whole = min(row.per_warp, (p.vocab - row.base) / kStep * kStep);
            for (; i + (kDeep - 1) * kStep < whole; i += kDeep * kStep) {
                uint4 w[kDeep];
#pragma unroll
                for (int k = 0; k < kDeep; ++k) {
                    const int64_t src = r * p.ld + row.base + i + k * kStep;
                    if (kBf16) {
                        const uint2 h = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p.logits) + src);
                        w[k] = make_uint4(h.x << 16, h.x & 0xffff0000u, h.y << 16, h.y & 0xffff0000u);
                    } else {
                        w[k] = *reinterpret_cast<const uint4*>(static_cast<const float*>(p.logits) + src);
                    }
                }
#pragma unroll
                for (int k = 0; k < kDeep; ++k)
                    put(i + k * kStep, {__uint_as_float(w[k].x), __uint_as_float(w[k].y), __uint_as_float(w[k].z),
                                        __uint_as_float(w[k].w)});
            }
        }
        for (; i < row.per_warp && row.base + i < p.vocab; i += kStep) {
            const int64_t src = r * p.ld + row.base + i;
            float v[kVec];
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                v[e] = ninf;
                if (row.base + i + e >= p.vocab) continue;
                v[e] = kBf16 ? __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(p.logits)[src + e]) << 16)
                             : static_cast<const float*>(p.logits)[src + e];
            }
            put(i, v);
        }
    }
    const float mine_top = top;                 // of this thread's values
    if (tid < 64) table[tid] = make_uint2(kExpTable[tid] - kRoundBits, __float_as_uint(__uint2float_rn(kExpTable[tid])));
    if (tid == 0) listed = 0;
    if (tid == 64) {
        const double c = 1.4426950408889634 / static_cast<double>(fmaxf(temperature, 0x1p-127f));     // (finite in fp32)
        scale.hi = static_cast<float>(c);
        scale.lo = static_cast<float>(c - static_cast<double>(scale.hi));
        scale.least = min_p > 0.0f ? static_cast<double>(temperature) * log(fmin(static_cast<double>(min_p), 1.0)) : 0.0;
    }
    *reinterpret_cast<uint4*>(&sh.hist[0][0][tid * kSelPerThread]) = make_uint4(0, 0, 0, 0);
    *reinterpret_cast<uint4*>(&sh.hist[0][1][tid * kSelPerThread]) = make_uint4(0, 0, 0, 0);
    const uint32_t most = __reduce_max_sync(0xffffffffu, nan ? 0xffffffffu : float_key(top));
    const uint32_t fewest = __reduce_min_sync(0xffffffffu, float_key(least));
    if (lane == 0) sh.warp[warp] = static_cast<uint64_t>(most) << 32 | fewest;
    cluster_sync();                             // (every CTA has started, and this one's are in sh.warp)
    uint32_t kmax = 0, kmin = 0xffffffffu;
    auto merge = [&](uint64_t v) {
        kmax = max(kmax, static_cast<uint32_t>(v >> 32));
        kmin = min(kmin, static_cast<uint32_t>(v));
    };
#pragma unroll
    for (int i = 0; i < kSelWarps; ++i) merge(sh.warp[i]);
    tell(sh, 0, static_cast<uint64_t>(kmax) << 32 | kmin, n, rank);
    cluster_sync();
    for (uint32_t i = 0; i < n; ++i) merge(sh.xch[0][i]);
    // no largest logit, or no temperature: no token
    if (kmax >= kKeyPosInf || kmax <= kKeyNegInf || !(temperature >= 0.0f && temperature <= 3.4028235e38f)) {
        if (rank == 0 && tid == 0) {
            p.token[r] = -1;
            if (p.logp) p.logp[r] = __int_as_float(0x7fc00000);
        }
        return;
    }
    top = key_float(kmax);
    const RowScale sc = scale;
    Cut cut = {kKeyNegInf, ~0ull >> 1};
    int turn = 0;
    if (temperature == 0.0f) {
        cut.key = kmax;
        cut.ties = 1;
    } else if ((top_k > 0 && top_k < p.vocab) || top_p < 1.0f) {
        const bool by_count = top_k > 0 && top_k < p.vocab, by_mass = top_p < 1.0f;
        const float range0 = key_float(kmin);
        const int per_rank = kListSize / static_cast<int>(n);
        uint64_t count[kSelPerThread], total, z = 0;     // values of this thread's steps; what top_p takes a share of
        auto w_of = [&](float v) { return weight(v, top, sc, table); };
        auto one = [](float) { return 1ull; };
        // f of every value that was gathered
        auto gathered = [&](auto f) {
#pragma unroll
            for (int i = tid; i < kListSize; i += kSelThreads)
                if (static_cast<uint64_t>(i & (per_rank - 1)) < sh.xch[2][i / per_rank]) f(list[i]);
        };
        // Sum over the cluster of what the threads of its CTAs have (told in slot 3, seen after a cluster_sync).
        auto tell_sum = [&](uint64_t mine) {
            uint64_t all;
            __syncthreads();
            block_scan(mine, sh.warp, &all);
            tell(sh, 3, all, n, rank);
        };
        auto told_sum = [&]() {
            uint64_t all = 0;
            for (uint32_t i = 0; i < n; ++i) all += sh.xch[3][i];
            return all;
        };
        // Bring the values of steps (above, last] to every CTA, and sum the weights of what top_k
        // leaves of those before.  False if they are too many.
        auto gather = [&](int above, int last, uint64_t* sum) -> bool {
            uint64_t mine = 0;
            each(row, [&](float v, int) {
                const int s = step_of(v, top, sc);
                if (s > last) return;
                if (s > above) {
                    const int at = atomicAdd(&listed, 1);
                    if (at >= per_rank) return;
                    const uint32_t to = smem_u32(&list[rank * per_rank + at]);
                    for (uint32_t i = 0; i < n; ++i) st_cluster_f32(mapa_shared(to, i), v);
                } else if (sum && float_key(v) > cut.key) {
                    mine += w_of(v);
                }
            });
            if (sum) tell_sum(mine);
            __syncthreads();
            tell(sh, 2, static_cast<uint64_t>(listed), n, rank);
            cluster_sync();
            if (tid == 0) listed = 0;
            bool fits = true;
            for (uint32_t i = 0; i < n; ++i) fits = fits && sh.xch[2][i] <= per_rank;
            if (sum) *sum = told_sum();
            return fits;
        };
        // Count the steps' values up to `last`.
        auto count_steps = [&](int last) {
            each(row, [&](float v, int) {
                const int s = step_of(v, top, sc);
                if (s <= last) atomicAdd(&sh.hist[turn][0][s], 1u);
            });
            cluster_sync();
            hist_merge<false>(sh, turn, 0, n, count);
            turn ^= 1;
        };
        auto share = [&]() {                 // of z
            const uint64_t part = top_p > 0.0f ? fraction64(top_p) : 0;
            return max(1ull, static_cast<unsigned long long>(__umul64hi(z, part) + (z * part != 0)));
        };
        // top_p's cut below top_k's: c found among the values above it, or (not in) among its equals, of
        // which `missing` is still needed
        auto cut_mass = [&](bool in, const Cut& c, uint64_t missing) {
            const uint64_t w = w_of(key_float(in ? c.key : cut.key));
            if (in) cut.key = c.key;
            if (w) cut.ties = in ? (c.ties + w - 1) / w : min(cut.ties, (missing + w - 1) / w);
        };

        // the threads' largest values by step, and (top_p alone) the sum of all weights
        {
            const int s = step_of(mine_top, top, sc);
            if (s < kSelBins - 1) atomicAdd(&sh.hist[turn][0][s], 1u);
            if (!by_count) {
                uint64_t mine = 0;
                each(row, [&](float v, int) { mine += w_of(v); });
                tell_sum(mine);
            }
            cluster_sync();
            hist_merge<false>(sh, turn, 0, n, count);
            turn ^= 1;
            if (!by_count) z = told_sum();
        }
        int last_step = kSelBins - 2;        // no cut lies in steps behind it
        bool mass_done = !by_mass;
        if (by_count) {
            const uint64_t k = static_cast<uint64_t>(top_k);
            bool found = false;
            Cut c;
            if (bins_find(sh, count, [&](uint64_t) { return k; }, &total)) {
                last_step = static_cast<int>(sh.found[0]);
                if (gather(-1, last_step, nullptr)) {
                    // all that can stay is in every CTA
                    const uint32_t lo = step_key_lo(last_step, top, sc);
                    found = find_key<false, true>(sh, turn, rank, n, lo, kmax, gathered, one, [&](uint64_t) { return k; }, &c, &total);
                    cut = c;
                    if (by_mass) {
                        uint64_t mine = 0;
                        gathered([&](float v) {
                            if (float_key(v) > cut.key) mine += w_of(v);
                        });
                        block_scan(mine, sh.warp, &z);
                        const uint64_t above_cut = z;
                        z += cut.ties * w_of(key_float(cut.key));
                        __syncthreads();
                        const uint64_t target = share();
                        const bool in = find_key<true, true>(
                            sh, turn, rank, n, lo, kmax, gathered, [&](float v) { return float_key(v) > cut.key ? w_of(v) : 0; },
                            [&](uint64_t) { return target; }, &c, &total);
                        cut_mass(in, c, target - above_cut);
                        mass_done = true;
                    }
                }
            }
            if (!found) {
                // many values: the step first
                count_steps(last_step);
                if (bins_find(sh, count, [&](uint64_t) { return k; }, &total)) {
                    const int step = static_cast<int>(sh.found[0]);
                    const uint64_t rest = k - sh.found[1];
                    last_step = step;
                    if (gather(step - 1, step, nullptr))
                        found = find_key<false, true>(sh, turn, rank, n, step_key_lo(step, top, sc), step_key_hi(step - 1, top, kmax, sc),
                                                      gathered, one, [&](uint64_t) { return rest; }, &c, &total);
                }
                // (a cut farther down than the steps go, or among too many values)
                if (!found)
                    found = find_cut<false>(sh, turn, rank, n, row, top, range0, kKeyNegInf, one, [&](uint64_t) { return k; }, &c, &total);
                if (found) cut = c;
            }
        }
        if (!mass_done) {
            uint64_t target, before = 0;
            uint64_t v[kSelPerThread];
            auto masses = [&]() {
#pragma unroll
                for (int i = 0; i < kSelPerThread; ++i) {
                    const int s = tid * kSelPerThread + i;
                    v[i] = s <= last_step ? count[i] * step_weight(s, table) : 0;
                }
            };
            if (by_count) {
                uint64_t mine = 0;
                each(row, [&](float x1, int) {
                    if (float_key(x1) > cut.key) mine += w_of(x1);
                });
                tell_sum(mine);
                cluster_sync();
                z = told_sum() + (cut.key > kKeyNegInf ? cut.ties * w_of(key_float(cut.key)) : 0);
                target = share();
            } else {
                // The cut lies no farther than where the threads' largest values alone reach the target, or
                // than where all values of the row together would not make up what is left beside it.
                target = share();
                masses();
                if (bins_find(sh, v, [&](uint64_t) { return target + (target >> 7) + 1; }, &total)) last_step = static_cast<int>(sh.found[0]);
                const uint64_t light = (z - target) / static_cast<uint64_t>(p.vocab) >> 1;
                const int far_step = light ? (kOne - 63 + __clzll(static_cast<long long>(light)) + 1) * 64 : kSelBins - 2;
                last_step = min(last_step, min(far_step, kSelBins - 2));
                __syncthreads();
            }
            count_steps(last_step);
            // The counts times the weights of the steps' middles are off by 2^(1/128), less than 2^-7, from
            // the steps' sums: the cut lies in the steps behind `above`, up to `last`.
            masses();
            const bool at_least = bins_find(sh, v, [&](uint64_t) { return max(1ull, target - (target >> 7) - 1ull); }, &total);
            const int above = at_least ? static_cast<int>(sh.found[0]) - 1 : last_step;
            __syncthreads();
            const bool at_most = bins_find(sh, v, [&](uint64_t) { return target + (target >> 7) + 1; }, &total);
            const int last = at_most ? static_cast<int>(sh.found[0]) : last_step;
            Cut c;
            bool in = false, found = false;
            if (at_most || last_step < kSelBins - 2) {       // (else it may lie farther down than the steps go)
                if (gather(above, last, &before)) {
                    in = find_key<true, true>(
                        sh, turn, rank, n, step_key_lo(last, top, sc), step_key_hi(above, top, kmax, sc), gathered,
                        [&](float x1) { return float_key(x1) > cut.key ? w_of(x1) : 0; }, [&](uint64_t) { return target - before; }, &c,
                        &total);
                    total += before;
                    found = true;
                }
            }
            if (!found) {
                const float far = fmaxf(range0, top - static_cast<float>(kOne + 2) / sc.hi);
                in = find_cut<true>(sh, turn, rank, n, row, top, far, cut.key, w_of, [&](uint64_t) { return target; }, &c, &total);
            }
            cut_mass(in, c, target - total);
        }
    }
    if (temperature != 0.0f) {
        if (min_p > 0.0f) {
            const uint32_t k = min(kmax, float_key(__double2float_ru(static_cast<double>(top) + sc.least)));
            if (k > cut.key) {                // everything from k on: above k - 1
                cut.key = k - 1;
                cut.ties = 0;
            }
        }
    }

    // sums over what stays: of this CTA's warps, then of the cluster's CTAs
    uint64_t sum = 0;
    uint32_t ties = 0;
    each(row, [&](float v, int) {
        const uint32_t key = float_key(v);
        if (key > cut.key) sum += weight(v, top, sc, table);
        ties += key == cut.key ? 1u : 0u;
    });
#pragma unroll
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    ties = __reduce_add_sync(0xffffffffu, ties);
    __syncthreads();
    if (lane == 0) {
        sh.warp[warp] = sum;
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
    const uint64_t w_tie = cut.key > kKeyNegInf ? weight(key_float(cut.key), top, sc, table) : 0;
    // weight of the first of the ties that come after `before` of them
    auto tie_part = [&](uint64_t before, uint64_t count) -> uint64_t {
        return before >= cut.ties ? 0 : min(count, cut.ties - before) * w_tie;
    };
    uint64_t all = 0, start = 0, ties_before = 0, seen_ties = 0;
    for (uint32_t i = 0; i < n; ++i) {
        if (i == rank) {
            start = all;
            ties_before = seen_ties;
        }
        all += sh.xch[4][i] + tie_part(seen_ties, sh.xch[5][i]);
        seen_ties += sh.xch[5][i];
    }
    const uint64_t at = u >= 1.0f ? all - 1 : u > 0.0f ? __umul64hi(all, fraction64(u)) : 0;
    for (int i = 0; i < warp; ++i) {
        start += sh.warp[i] + tie_part(ties_before, sh.warp2[i]);
        ties_before += sh.warp2[i];
    }
    if (at < start || at >= start + sh.warp[warp] + tie_part(ties_before, sh.warp2[warp])) return;
    // this warp holds it: step by step through its values
    for (int i = 0; i < row.per_warp; i += kStep) {
        const float4 v4 = *reinterpret_cast<const float4*>(x + warp * row.per_warp + i + lane * kVec);
        float v[kVec] = {v4.x, v4.y, v4.z, v4.w};
        uint64_t w[kVec];
        uint32_t t[kVec], mine = 0;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            const bool in = row.base + i + lane * kVec + e < p.vocab;
            const uint32_t key = in ? float_key(v[e]) : 0u;
            w[e] = in && key > cut.key ? weight(v[e], top, sc, table) : 0;
            t[e] = in && key == cut.key ? 1u : 0u;
            mine += t[e];
        }
        uint32_t incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        uint64_t rank_of = ties_before + incl - mine, lane_sum = 0;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
            if (t[e]) w[e] = rank_of < cut.ties ? w_tie : 0;
            rank_of += t[e];
            lane_sum += w[e];
        }
        uint64_t scan = lane_sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t y = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += y;
        }
        const uint64_t step_sum = __shfl_sync(0xffffffffu, scan, 31);
        ties_before += __shfl_sync(0xffffffffu, incl, 31);
        if (at >= start + step_sum) {
            start += step_sum;
            continue;
        }
        uint64_t run = start + scan - lane_sum;
        if (at >= run && at < run + lane_sum) {
#pragma unroll
            for (int e = 0; e < kVec; ++e) {
                if (at >= run && at < run + w[e]) {
                    p.token[r] = row.base + i + lane * kVec + e;
                    if (p.logp) {
                        // of a share above a half from what is left beside it; else from its logit
                        const float rest = static_cast<float>(all - w[e]), whole = static_cast<float>(all);
                        const float z = (v[e] - top) * sc.hi + (v[e] - top) * sc.lo;
                        p.logp[r] = w[e] > all / 2 ? log1pf(-rest / whole)
                                                   : z * 0.693147180559945f - logf(whole * (1.0f / (1ull << kOne)));
                    }
                }
                run += w[e];
            }
        }
        return;
    }
}

template <bool kBf16, bool kAligned>
cr_status launch(const SampleParams& p, cudaStream_t st) {
    int ranks = kMaxCluster;
    while (ranks > 1 && static_cast<int64_t>(p.n_rows) * ranks > num_sms()) ranks /= 2;
    while (ranks < kMaxCluster && p.vocab > ranks * kChunk) ranks *= 2;
    const int per_warp = ((p.vocab + ranks * kSelWarps - 1) / (ranks * kSelWarps) + kStep - 1) / kStep * kStep;
    static unsigned long long attr_done = 0;
    const cr_status s = ensure_smem_attr(sample_kernel<kBf16, kAligned>, kMaxChunk * 4, &attr_done);
    if (s != CR_OK) return s;
    return launch_cluster(sample_kernel<kBf16, kAligned>, dim3(static_cast<unsigned>(p.n_rows * ranks)), dim3(kSelThreads), ranks,
                          static_cast<size_t>(per_warp) * kSelWarps * 4, st, p);
}

}  // namespace

int64_t sample_max_vocab() { return static_cast<int64_t>(kMaxCluster) * (kMaxChunk - kSelWarps * kStep); }

cr_status launch_sample(const SampleParams& p, bool bf16, cudaStream_t st) {
    const int64_t size = bf16 ? 2 : 4, unit = kVec * size;        // a thread's values in one load
    const bool aligned = (reinterpret_cast<uintptr_t>(p.logits) % unit) == 0 && (p.ld * size) % unit == 0;
    return bf16 ? (aligned ? launch<true, true>(p, st) : launch<true, false>(p, st))
                : (aligned ? launch<false, true>(p, st) : launch<false, false>(p, st));
}

}  // namespace cr
