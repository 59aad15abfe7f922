// C ABI of the answering calls (include/cr.h): host-side validation and the
// launches of appending to, and attending over, a paged cache.
#include <math.h>
#include <string.h>

#include "cr_internal.h"

using namespace cr;

namespace {

cr_status check_layer(const cr_paged_layer* c) {
    if (!c || !c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) return CR_ERR_INVALID_ARG;
    if (c->n_kv_heads < 1 || c->block_size < 1 || c->num_slots < c->block_size || c->num_slots > INT32_MAX / 2)
        return CR_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return CR_ERR_UNSUPPORTED;
    if (c->block_size < 8 || (c->block_size & (c->block_size - 1)) != 0) return CR_ERR_UNSUPPORTED;
    if (c->n_kv_heads > 4096) return CR_ERR_UNSUPPORTED;
    return CR_OK;
}

// A batch's shape: request offsets and groups, checked.
cr_status set_batch(PagedPlan& p, cr_attention_batch& b, int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                    const int32_t* cu_q, int32_t n_req, const int32_t* cu_group, int32_t n_groups) {
    if (!cu_q || n_req < 1 || n_req > kMaxReq || n_q_heads < 1 || n_kv_heads < 1 || n_q_heads % n_kv_heads != 0)
        return CR_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return CR_ERR_UNSUPPORTED;
    if (n_kv_heads > 4096 || n_q_heads > 65536) return CR_ERR_UNSUPPORTED;
    if (cu_q[0] != 0) return CR_ERR_INVALID_ARG;
    for (int r = 0; r < n_req; ++r)
        if (cu_q[r + 1] < cu_q[r]) return CR_ERR_INVALID_ARG;
    if (cu_q[n_req] < 1) return CR_ERR_INVALID_ARG;
    if (static_cast<int64_t>(cu_q[n_req]) * n_q_heads > INT32_MAX / 2) return CR_ERR_UNSUPPORTED;
    if (cu_group) {
        if (n_groups < 1 || n_groups > kMaxReq || cu_group[0] != 0 || cu_group[n_groups] != n_req)
            return CR_ERR_INVALID_ARG;
        for (int g = 0; g < n_groups; ++g)
            if (cu_group[g + 1] < cu_group[g]) return CR_ERR_INVALID_ARG;
        memcpy(p.cu_group, cu_group, sizeof(int32_t) * (n_groups + 1));
    }
    memcpy(p.cu_q, cu_q, sizeof(int32_t) * (n_req + 1));
    p.n_req = n_req;
    p.n_groups = cu_group ? n_groups : 0;
    p.n_tokens = cu_q[n_req];
    b.n_q_heads = n_q_heads;
    b.n_kv_heads = n_kv_heads;
    b.head_dim = head_dim;
    b.n_req = n_req;
    b.n_groups = p.n_groups;
    b.n_tokens = p.n_tokens;
    return CR_OK;
}

cr_status attend(const cr_paged_layer* cache, const cr_attention_batch* b, const uint16_t* q, int64_t ldq,
                 const int32_t* block_table, int64_t max_blocks, const int32_t* kv_len, bool prefix,
                 const int32_t* prefix_table, int64_t max_prefix_blocks, const int32_t* prefix_len, float scale,
                 uint16_t* out, int64_t ldo, float* lse, void* stream) {
    cr_status s = check_layer(cache);
    if (s != CR_OK) return s;
    if (!b || b->n_tokens < 1 || b->n_req < 1 || b->n_req > kMaxReq || b->n_groups < 0 || b->n_groups > kMaxReq ||
        b->n_kv_heads != cache->n_kv_heads || b->head_dim != cache->head_dim || b->n_q_heads < b->n_kv_heads ||
        b->n_q_heads % b->n_kv_heads != 0 || (b->n_groups > 0) != prefix || !b->workspace)
        return CR_ERR_INVALID_ARG;
    const int64_t width = static_cast<int64_t>(b->n_q_heads) * cache->head_dim;
    if (!q || !out || !block_table || !kv_len || !aligned16(q) || !aligned16(out) || !aligned16(block_table) ||
        !aligned16(kv_len) || (lse && !aligned16(lse)))
        return CR_ERR_INVALID_ARG;
    if (prefix && (!prefix_table || !prefix_len || !aligned16(prefix_table) || !aligned16(prefix_len) ||
                   max_prefix_blocks < 1))
        return CR_ERR_INVALID_ARG;
    if (ldq < width || ldo < width || (ldq % 8) != 0 || (ldo % 8) != 0 || max_blocks < 1) return CR_ERR_INVALID_ARG;
    // a sequence's length is counted in 32 bits
    if (max_blocks > (INT32_MAX / 2) / cache->block_size ||
        (prefix && max_prefix_blocks > (INT32_MAX / 2) / cache->block_size))
        return CR_ERR_UNSUPPORTED;
    if (!(scale > 0.0f) || !isfinite(scale)) return CR_ERR_INVALID_ARG;
    PagedParams p;
    p.q = q;
    p.out = out;
    p.lse = lse;
    p.ldq = ldq;
    p.ldo = ldo;
    p.own_table = block_table;
    p.own_len = kv_len;
    p.own_blocks = max_blocks;
    p.prefix_table = prefix_table;
    p.prefix_len = prefix_len;
    p.prefix_blocks = max_prefix_blocks;
    p.scale_log2 = scale * 1.4426950408889634f;
    p.n_blocks = static_cast<int32_t>(cache->num_slots / cache->block_size);
    p.block_shift = __builtin_ctz(static_cast<unsigned>(cache->block_size));
    p.n_req = b->n_req;
    p.n_groups = b->n_groups;
    p.n_q_heads = b->n_q_heads;
    p.n_kv_heads = b->n_kv_heads;
    p.group = b->n_q_heads / b->n_kv_heads;
    p.n_tokens = b->n_tokens;
    // division by an invariant integer by multiplication (Granlund and Montgomery 1994)
    p.group_shift = 0;
    while ((1u << p.group_shift) < static_cast<uint32_t>(p.group)) ++p.group_shift;
    p.group_mul = static_cast<uint32_t>(((1ull << 32) * ((1ull << p.group_shift) - p.group)) / p.group + 1);
    p.status = device_status_ptr();
    if (!p.status) return CR_ERR_CUDA;
    return launch_paged_attention(p, *cache, *b, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" {

cr_status cr_paged_append(const cr_paged_layer* cache, const void* k, int64_t ldk, const void* v,
                          int64_t ldv, const void* q, int64_t ldq, int32_t n_q_heads,
                          int32_t in_dtype, int64_t n_tokens, const int32_t* pos,
                          const float* inv_freq_host, int32_t rope_mode,
                          const int64_t* slot_mapping, uint16_t* q_out, int64_t ldq_out,
                          void* stream) {
    const cr_status s = check_layer(cache);
    if (s != CR_OK) return s;
    if (in_dtype != CR_F32 && in_dtype != CR_BF16) return CR_ERR_INVALID_ARG;
    if (rope_mode != CR_ROPE_NONE && rope_mode != CR_ROPE_GLOBAL) return CR_ERR_INVALID_ARG;
    if (rope_mode == CR_ROPE_GLOBAL && (!inv_freq_host || !pos)) return CR_ERR_INVALID_ARG;
    if (n_tokens < 1 || n_tokens > INT32_MAX / 2) return CR_ERR_INVALID_ARG;
    const int64_t unit = in_dtype == CR_F32 ? 4 : 8;      // elements of 16 bytes
    const int64_t width = static_cast<int64_t>(cache->n_kv_heads) * cache->head_dim;
    if (!k || !v || !slot_mapping || !aligned16(k) || !aligned16(v) || !aligned16(slot_mapping) ||
        (pos && !aligned16(pos)))
        return CR_ERR_INVALID_ARG;
    if (ldk < width || ldv < width || ldk % unit != 0 || ldv % unit != 0) return CR_ERR_INVALID_ARG;
    if (q) {
        if (n_q_heads < 1) return CR_ERR_INVALID_ARG;
        if (n_q_heads > 65536) return CR_ERR_UNSUPPORTED;
        const int64_t qw = static_cast<int64_t>(n_q_heads) * cache->head_dim;
        if (!q_out || !aligned16(q) || !aligned16(q_out) || ldq < qw || ldq % unit != 0 || ldq_out < qw ||
            ldq_out % 8 != 0)
            return CR_ERR_INVALID_ARG;
        // in place only where a row's new values take the places of its old ones
        if (static_cast<const void*>(q_out) == q && (in_dtype == CR_F32 || ldq_out != ldq)) return CR_ERR_INVALID_ARG;
    }
    AppendParams p{};
    p.status = device_status_ptr();
    if (!p.status) return CR_ERR_CUDA;
    p.q = q;
    p.k_in = k;
    p.v_in = v;
    p.ldq = ldq;
    p.ldk = ldk;
    p.ldv = ldv;
    p.q_out = q_out;
    p.ldq_out = ldq_out;
    p.k = static_cast<uint16_t*>(cache->k);
    p.v = static_cast<uint16_t*>(cache->v);
    p.pos = pos;
    p.slot = slot_mapping;
    p.num_slots = cache->num_slots;
    p.n_q_heads = q ? n_q_heads : 0;
    p.n_kv_heads = cache->n_kv_heads;
    p.head_dim = cache->head_dim;
    p.rotate = rope_mode == CR_ROPE_GLOBAL;
    if (p.rotate) memcpy(p.inv_freq, inv_freq_host, sizeof(float) * (cache->head_dim / 2));
    return launch_append(p, in_dtype == CR_F32, n_tokens, static_cast<cudaStream_t>(stream));
}

size_t cr_attention_workspace_bytes(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                                    const int32_t* cu_q_host, int32_t n_req,
                                    const int32_t* cu_group_host, int32_t n_groups) {
    PagedPlan plan;
    cr_attention_batch b;
    if (set_batch(plan, b, n_q_heads, n_kv_heads, head_dim, cu_q_host, n_req, cu_group_host, n_groups) != CR_OK) return 0;
    return paged_plan(plan, b);
}

cr_status cr_attention_plan(int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim,
                            const int32_t* cu_q_host, int32_t n_req, const int32_t* cu_group_host,
                            int32_t n_groups, void* workspace, size_t workspace_bytes,
                            cr_attention_batch* batch, void* stream) {
    PagedPlan plan;
    cr_attention_batch b;
    if (!batch || !workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return CR_ERR_INVALID_ARG;
    cr_status s = set_batch(plan, b, n_q_heads, n_kv_heads, head_dim, cu_q_host, n_req, cu_group_host, n_groups);
    if (s != CR_OK) return s;
    const size_t need = paged_plan(plan, b);
    if (need == 0) return CR_ERR_UNSUPPORTED;
    if (workspace_bytes < need) return CR_ERR_INVALID_ARG;
    b.workspace = workspace;
    b.workspace_bytes = workspace_bytes;
    if ((s = launch_paged_plan(plan, b, static_cast<cudaStream_t>(stream))) == CR_OK) *batch = b;
    return s;
}

cr_status cr_paged_attention(const cr_paged_layer* cache, const cr_attention_batch* batch,
                             const uint16_t* q, int64_t ldq, const int32_t* block_table,
                             int64_t max_blocks, const int32_t* kv_len, float scale, uint16_t* out,
                             int64_t ldo, float* lse, void* stream) {
    return attend(cache, batch, q, ldq, block_table, max_blocks, kv_len, false, nullptr, 0, nullptr, scale, out, ldo,
                  lse, stream);
}

cr_status cr_prefix_attention(const cr_paged_layer* cache, const cr_attention_batch* batch,
                              const uint16_t* q, int64_t ldq, const int32_t* block_table,
                              int64_t max_blocks, const int32_t* kv_len,
                              const int32_t* prefix_table, int64_t max_prefix_blocks,
                              const int32_t* prefix_len, float scale, uint16_t* out, int64_t ldo,
                              float* lse, void* stream) {
    return attend(cache, batch, q, ldq, block_table, max_blocks, kv_len, true, prefix_table, max_prefix_blocks,
                  prefix_len, scale, out, ldo, lse, stream);
}

}  // extern "C"
