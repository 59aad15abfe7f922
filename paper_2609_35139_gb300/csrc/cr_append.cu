// Appending new tokens to one layer of a paged cache: K rotated by R_M(pos)
// and V written at the tokens' slots, Q rotated for the attention that follows.
//   x'[i] = x[i] cos a - x[i + d/2] sin a,  x'[i + d/2] = x[i + d/2] cos a + x[i] sin a,
//   a = pos * f_i
// in fp32 with one rounding to bf16.  Bound by HBM bandwidth (about three
// flops per value): 16384 tokens of 32 query and 8 KV heads of 128 take 65 us,
// 6.2 TB/s or 0.91 of the measured copy rate; for a few tokens by latency, 2.3 us
// in a graph.
#include <cuda_bf16.h>

#include "cr_internal.h"
#include "cr_ptx.cuh"

namespace cr {
namespace {

constexpr int kThreads = 256;

// Eight consecutive values as fp32, from bf16 (one 16-byte load) or fp32 (two).
template <bool kF32>
struct Vec8 {
    uint4 a, b;
    __device__ __forceinline__ void load(const void* base, int64_t elem) {
        if (kF32) {
            const uint4* p = reinterpret_cast<const uint4*>(static_cast<const float*>(base) + elem);
            a = p[0];
            b = p[1];
        } else {
            a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(base) + elem);
        }
    }
    __device__ __forceinline__ void get(float* x) const {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
        if (kF32) {
            const uint32_t u[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = __uint_as_float(w[i]);
                x[4 + i] = __uint_as_float(u[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[2 * i] = __uint_as_float(w[i] << 16);
                x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            }
        }
    }
};

__device__ __forceinline__ void store8(uint16_t* dst, const float* x) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]),
                                                pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// cos and sin of pos * f: a = fl(pos f) and its exact remainder e = pos f - a
// (FMA), then (cos a, sin a) turned by e.  At a long cache's positions a reaches
// 2^17, so e reaches 2^-8 and its square counts: the turn goes to e^4 (error
// e^5 / 120, below 2^-26 up to positions of 2^20).  Past those the position is
// taken in two parts, its low 8 bits and the rest, both exact in fp32: a is the
// rest's product, and the low bits' product with a's remainder, up to some
// hundreds, is a second angle r to turn by; what is left after both is tiny.
constexpr int kNearPos = 1 << 20;
__device__ __forceinline__ void angle(int pos, float f, float* s, float* c) {
    const bool far = pos > kNearPos || pos < -kNearPos;
    const float hi = static_cast<float>(far ? pos & ~0xff : pos);
    const float a = hi * f;
    float e = fmaf(hi, f, -a);
    float sa, ca;
    sincosf(a, &sa, &ca);
    if (far) {
        const float lo = static_cast<float>(pos & 0xff), b = lo * f;
        const float r = b + e, back = r - b;               // r and what its rounding lost (two-sum)
        const float lost = (b - (r - back)) + (e - back);
        float sr, cr;
        sincosf(r, &sr, &cr);
        const float x = ca * cr - sa * sr;
        sa = sa * cr + ca * sr;
        ca = x;
        e = lost + fmaf(lo, f, -b);
    }
    const float e2 = e * e;
    const float se = e - e * e2 * (1.0f / 6.0f);
    const float ce1 = e2 * (e2 * (1.0f / 24.0f) - 0.5f);   // cos e - 1
    *c = ca + (ca * ce1 - sa * se);
    *s = sa + (sa * ce1 + ca * se);
}

// One token per CTA.  Its d/2 angles are evaluated once into shared memory; an
// item is then one 8-value piece of a head with its partner d/2 further on (Q
// and K heads), or two 8-value pieces that are rounded alone (V, and all of them
// without a rotation).
// Eight CTAs an SM (32 registers): 16384 tokens take 64.7 us, 72.3 with six.
template <bool kF32>
__global__ void __launch_bounds__(kThreads, 8) append_kernel(const __grid_constant__ AppendParams p) {
    __shared__ float cs[64], sn[64];
    pdl_launch_dependents();
    pdl_wait();
    const int64_t t = blockIdx.x;
    const int half = p.head_dim >> 1;
    const int64_t slot = p.slot[t];
    if (threadIdx.x == 0 && slot >= p.num_slots) report(p.status, CR_DEV_INDEX, 910);
    const bool write = slot >= 0 && slot < p.num_slots;
    if (p.rotate && static_cast<int>(threadIdx.x) < half) {
        float s, c;
        angle(p.pos[t], p.inv_freq[threadIdx.x], &s, &c);
        cs[threadIdx.x] = c;
        sn[threadIdx.x] = s;
    }
    __syncthreads();
    const int per_head = half >> 3;                       // pairs of 8-value pieces in a head
    const int n_items = (p.n_q_heads + 2 * p.n_kv_heads) * per_head;
    const int64_t width = static_cast<int64_t>(p.n_kv_heads) * p.head_dim;
    for (int item = threadIdx.x; item < n_items; item += kThreads) {
        const int head = item / per_head;
        const int i = (item - head * per_head) * 8;
        const bool is_q = head < p.n_q_heads;
        const bool is_v = head >= p.n_q_heads + p.n_kv_heads;
        if (!is_q && !write) continue;
        const void* src;
        int64_t at;
        uint16_t* dst;
        if (is_q) {
            src = p.q;
            at = t * p.ldq + static_cast<int64_t>(head) * p.head_dim + i;
            dst = p.q_out + t * p.ldq_out + static_cast<int64_t>(head) * p.head_dim + i;
        } else {
            const int64_t h = static_cast<int64_t>(head - p.n_q_heads - (is_v ? p.n_kv_heads : 0)) * p.head_dim + i;
            src = is_v ? p.v_in : p.k_in;
            at = t * (is_v ? p.ldv : p.ldk) + h;
            dst = (is_v ? p.v : p.k) + slot * width + h;
        }
        Vec8<kF32> va, vb;
        va.load(src, at);
        vb.load(src, at + half);
        float a[8], b[8];
        va.get(a);
        vb.get(b);
        if (!is_v && p.rotate) {         // (without, an infinity must not meet its pair's sine of 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float c = cs[i + j], s = sn[i + j];
                const float x = a[j] * c - b[j] * s;
                b[j] = b[j] * c + a[j] * s;
                a[j] = x;
            }
        }
        store8(dst, a);
        store8(dst + half, b);
    }
}

}  // namespace

cr_status launch_append(const AppendParams& p, bool f32, int64_t n_tokens, cudaStream_t st) {
    const dim3 grid(static_cast<unsigned>(n_tokens));
    return f32 ? launch_pdl(append_kernel<true>, grid, dim3(kThreads), 0, st, p)
               : launch_pdl(append_kernel<false>, grid, dim3(kThreads), 0, st, p);
}

}  // namespace cr
