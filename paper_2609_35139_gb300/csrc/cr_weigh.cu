// Attention weight gathered by the tokens of a paged cache:
//   w[h][slot(j)] (+)= sum over the rows i that see j, and the query heads of KV head h,
//                      exp(scale q_i . k_j - lse_i),
// the sum over a call's rows of the weights that attention gave token j (lse_i is the
// row's log-sum-exp there).  Segments, rows and what they see are those of the attention
// calls: a request's rows over its own tokens, causal among the new ones, and a group's
// rows over its prefix.  Products take bf16 with fp32 accumulation, the sum is fp32.
#include <cuda_bf16.h>

#include "cr_internal.h"
#include "cr_ptx.cuh"

namespace cr {
namespace {

constexpr int kWarps = 4;
constexpr int kWarpKeys = 16;
constexpr int kBlockKeys = kWarps * kWarpKeys;

__device__ __forceinline__ float neg_inf() { return __int_as_float(0xff800000); }

__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, const uint32_t* b) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

// A warp takes 16 keys of one KV head, as the M of m16n8k16, and all rows of the segment
// that see them, eight at a time.  The order of the products' k is free as long as both
// operands share it: a thread loads whole 16-byte pieces and feeds each to two MMAs.
template <int D>
__global__ void __launch_bounds__(kWarps * 32) weigh_kernel(const __grid_constant__ WeighParams p) {
    pdl_launch_dependents();
    pdl_wait();
    constexpr int kPieces = D / 32;            // 16-byte pieces of a row in each of a quad's threads
    const int s = static_cast<int>(blockIdx.z), head = static_cast<int>(blockIdx.y);
    const bool own = s >= p.n_groups;
    const int r = s - p.n_groups;
    const int4 shape = p.seg[s];
    const int nt = shape.y;
    const int64_t blocks = own ? p.own_blocks : p.prefix_blocks;
    int len = own ? p.own_len[r] : p.prefix_len[s];
    const int64_t most = blocks << p.block_shift;
    if (len < 0 || len > most) {
        report(p.status, CR_DEV_INDEX, 941);
        len = len < 0 ? 0 : static_cast<int>(most);
    }
    if (nt == 0) return;
    const int32_t* table = own ? p.own_table + r * p.own_blocks : p.prefix_table + s * p.prefix_blocks;
    const uint32_t warp = warp_id(), lane = lane_id();
    const int g = static_cast<int>(lane >> 2), t = static_cast<int>(lane & 3u);
    const int key0 = static_cast<int>(blockIdx.x) * kBlockKeys + static_cast<int>(warp) * kWarpKeys;
    if (key0 >= len) return;
    const int64_t width = static_cast<int64_t>(p.n_kv_heads) * D;
    int64_t slot[2];
    uint32_t k[2][kPieces][4];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int key = key0 + g + 8 * i;
        slot[i] = -1;
        if (key < len) {
            const int block = table[key >> p.block_shift];
            if (block < 0 || block >= p.n_blocks) report(p.status, CR_DEV_INDEX, 942);
            else slot[i] = (static_cast<int64_t>(block) << p.block_shift) + (key & ((1 << p.block_shift) - 1));
        }
#pragma unroll
        for (int c = 0; c < kPieces; ++c) {
            const uint4 x = slot[i] < 0 ? make_uint4(0, 0, 0, 0)
                                        : *reinterpret_cast<const uint4*>(p.k + slot[i] * width + head * D + (c * 4 + t) * 8);
            k[i][c][0] = x.x, k[i][c][1] = x.y, k[i][c][2] = x.z, k[i][c][3] = x.w;
        }
    }
    const int rows = nt * p.group;
    const int past = own ? len - nt : INT32_MAX / 2;           // row n sees keys j < past + token_of(n) + 1
    const int row_first = own ? max(0, key0 - past) * p.group / 8 * 8 : 0;
    float sum[2] = {0.0f, 0.0f};
    for (int row0 = row_first; row0 < rows; row0 += 8) {
        float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const int row = min(row0 + g, rows - 1), tok = row / p.group;
        const uint16_t* q = p.q + static_cast<int64_t>(shape.x + tok) * p.ldq +
                            static_cast<int64_t>(head * p.group + row - tok * p.group) * D;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint4 x = *reinterpret_cast<const uint4*>(q + (i * 4 + t) * 8);
            const uint32_t b0[2] = {x.x, x.y}, b1[2] = {x.z, x.w};
            const uint32_t a0[4] = {k[0][i][0], k[1][i][0], k[0][i][1], k[1][i][1]};
            const uint32_t a1[4] = {k[0][i][2], k[1][i][2], k[0][i][3], k[1][i][3]};
            mma16816(c, a0, b0);
            mma16816(c, a1, b1);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int n = row0 + 2 * t + e;
            if (n >= rows) continue;
            const int nk = n / p.group;
            const float lse = p.lse[static_cast<int64_t>(shape.x + nk) * p.n_q_heads + head * p.group + n - nk * p.group];
            if (lse == neg_inf()) continue;
            const int limit = own ? past + nk + 1 : len;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (key0 + g + 8 * i < limit) sum[i] += ex2(fmaf(c[2 * i + e], p.scale_log2, -lse * 1.4426950408889634f));
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
        sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
        if (t == 0 && slot[i] >= 0) {
            float* w = p.weights + static_cast<int64_t>(head) * p.num_slots + slot[i];
            if (key0 + g + 8 * i >= past) *w = sum[i];
            else atomicAdd(w, sum[i]);
        }
    }
}

}  // namespace

cr_status launch_weigh(const WeighParams& p, int head_dim, cudaStream_t st) {
    const int64_t most = (p.own_blocks > p.prefix_blocks || p.n_groups == 0 ? p.own_blocks : p.prefix_blocks) << p.block_shift;
    const dim3 grid(static_cast<unsigned>((most + kBlockKeys - 1) / kBlockKeys), p.n_kv_heads, p.n_groups + p.n_req);
    return launch_pdl(head_dim == 128 ? weigh_kernel<128> : weigh_kernel<64>, grid, dim3(kWarps * 32), 0, st, p);
}

}  // namespace cr
