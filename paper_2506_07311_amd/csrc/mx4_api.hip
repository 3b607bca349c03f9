// C ABI of normalised heads, positions of several numbers and the 4-bit cache: argument validation and dispatch.  Every check is a host
// check made before the first launch; nothing here touches device memory.
#include <algorithm>

#include "mx4.h"

using namespace pa;

namespace pa {

pa_status check_mx4_cache(const pa_mx4_cache_desc* c)
{
    if (!c || !c->records) return PA_ERR_INVALID_ARG;
    if (c->num_pages <= 0 || c->num_kv_heads <= 0 || c->head_dim <= 0 || c->page_size <= 0 || (c->page_size & (c->page_size - 1)))
        return PA_ERR_INVALID_ARG;
    const size_t record = pa_mx4_record_bytes(c->page_size, c->head_dim);
    if (record == 0) return PA_ERR_UNSUPPORTED;
    if (c->head_stride < 0 || (c->num_kv_heads > 1 && c->head_stride < (int64_t)record) || c->page_stride < (int64_t)record)
        return PA_ERR_INVALID_ARG;
    if (c->page_stride % 16 || c->head_stride % 16 || ((uintptr_t)c->records & 15)) return PA_ERR_UNSUPPORTED;
    return PA_OK;
}

}  // namespace pa

namespace {

inline hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }

bool known(pa_dtype t) { return t == PA_DTYPE_F32 || t == PA_DTYPE_BF16 || t == PA_DTYPE_F16; }

pa_status check_mx4(const pa_mx4_cache_desc* c, pa_dtype dtype)
{
    const pa_status st = check_mx4_cache(c);
    return st != PA_OK || known(dtype) ? st : PA_ERR_UNSUPPORTED;
}

// What paged_norm_rope_append asks of its tokens; strides of 0 become those of contiguous ones.
pa_status check_tokens(pa_norm_rope& r, pa_dtype dtype, int32_t kv_heads, int32_t d, bool& nothing)
{
    nothing = false;
    if (r.T < 0 || r.batch < 0 || r.max_blocks < 0 || r.rotary_dim < 0 || r.rotary_dim % 2 || r.rotary_dim > d) return PA_ERR_INVALID_ARG;
    if (r.q_stride < 0 || r.q_out_stride < 0 || r.k_stride < 0 || r.v_stride < 0 || !(r.mscale == r.mscale)) return PA_ERR_INVALID_ARG;
    if (!(r.eps >= 0.f) || r.eps > 3.4e38f || !(r.weight_offset == r.weight_offset)) return PA_ERR_INVALID_ARG;
    if (!r.q != !r.q_out || !r.k_new != !r.v_new) return PA_ERR_INVALID_ARG;
    nothing = r.T == 0 || (!r.q && !r.k_new);
    if (nothing) return PA_OK;
    if (r.q && r.num_q_heads <= 0) return PA_ERR_INVALID_ARG;
    if (r.rotary_dim > 0 && (!r.rope_positions || !r.inv_freq || ((uintptr_t)r.inv_freq & 7) || r.axes <= 0)) return PA_ERR_INVALID_ARG;
    if (r.rotary_dim > 0 && r.axes > 1 && !r.pair_axes) return PA_ERR_INVALID_ARG;
    if (r.k_new && (!r.seq_ids || !r.positions || !r.block_table || r.batch == 0 || r.max_blocks == 0)) return PA_ERR_INVALID_ARG;
    if ((r.q_weight || r.k_weight) && r.weight_dtype != dtype && r.weight_dtype != PA_DTYPE_F32) return PA_ERR_UNSUPPORTED;
    const int64_t epv = dtype == PA_DTYPE_F32 ? 4 : 8;
    const int64_t q_row = (int64_t)r.num_q_heads * d, kv_row = (int64_t)kv_heads * d;
    if (r.q_stride == 0) r.q_stride = q_row;
    if (r.q_out_stride == 0) r.q_out_stride = q_row;
    if (r.k_stride == 0) r.k_stride = kv_row;
    if (r.v_stride == 0) r.v_stride = kv_row;
    if (r.q && (r.q_stride < q_row || r.q_out_stride < q_row || (r.q == r.q_out && r.q_stride != r.q_out_stride))) return PA_ERR_INVALID_ARG;
    if (r.k_new && (r.k_stride < kv_row || r.v_stride < kv_row)) return PA_ERR_INVALID_ARG;
    if (r.T >= 1 << 25) return PA_ERR_UNSUPPORTED;           // (128 threads a token: those of a launch stay below 2^32)
    if (r.q_stride % epv || r.q_out_stride % epv || r.k_stride % epv || r.v_stride % epv) return PA_ERR_UNSUPPORTED;
    if (((uintptr_t)r.q | (uintptr_t)r.q_out | (uintptr_t)r.k_new | (uintptr_t)r.v_new | (uintptr_t)r.q_weight | (uintptr_t)r.k_weight) & 15)
        return PA_ERR_UNSUPPORTED;
    return PA_OK;
}

}  // namespace

extern "C" {

pa_status paged_norm_rope_append(const pa_kv_cache_desc* cache, const pa_norm_rope* tokens, void* stream)
{
    const pa_status st = check_cache(cache);
    if (st != PA_OK) return st;
    if (!tokens) return PA_ERR_INVALID_ARG;
    pa_norm_rope r = *tokens;
    bool nothing;
    const pa_status ts = check_tokens(r, cache->dtype, cache->num_kv_heads, cache->head_dim, nothing);
    if (ts != PA_OK || nothing) return ts;
    return launch_norm_rope_append(cache, nullptr, cache->dtype, r, stream_of(stream));
}

size_t pa_mx4_record_bytes(int32_t page_size, int32_t head_dim)
{
    if (page_size < 16 || (page_size & (page_size - 1)) || page_size > (1 << 20)) return 0;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return 0;
    return (size_t)page_size * head_dim / 16 * 17;
}

pa_status paged_norm_rope_append_mx4(const pa_mx4_cache_desc* cache, pa_dtype dtype, const pa_norm_rope* tokens, void* stream)
{
    const pa_status st = check_mx4(cache, dtype);
    if (st != PA_OK) return st;
    if (!tokens) return PA_ERR_INVALID_ARG;
    pa_norm_rope r = *tokens;
    bool nothing;
    const pa_status ts = check_tokens(r, dtype, cache->num_kv_heads, cache->head_dim, nothing);
    if (ts != PA_OK || nothing) return ts;
    return launch_norm_rope_append(nullptr, cache, dtype, r, stream_of(stream));
}

pa_status paged_kv_append_mx4(const pa_mx4_cache_desc* cache, pa_dtype dtype, const void* k_new, const void* v_new,
                              const int32_t* seq_ids, const int32_t* positions, int32_t T, const int32_t* block_table,
                              int32_t batch, int32_t max_blocks, void* stream)
{
    const pa_status st = check_mx4(cache, dtype);
    if (st != PA_OK) return st;
    if (T < 0 || batch < 0 || max_blocks < 0) return PA_ERR_INVALID_ARG;
    if (T == 0) return PA_OK;
    if (!k_new || !v_new) return PA_ERR_INVALID_ARG;
    pa_norm_rope r = {};
    r.k_new = k_new;
    r.v_new = v_new;
    r.seq_ids = seq_ids;
    r.positions = positions;
    r.block_table = block_table;
    r.T = T;
    r.batch = batch;
    r.max_blocks = max_blocks;
    r.mscale = 1.f;
    bool nothing;
    const pa_status ts = check_tokens(r, dtype, cache->num_kv_heads, cache->head_dim, nothing);
    if (ts != PA_OK || nothing) return ts;
    return launch_norm_rope_append(nullptr, cache, dtype, r, stream_of(stream));
}

pa_status paged_kv_gather_mx4(const pa_mx4_cache_desc* cache, pa_dtype dtype, void* out_k, void* out_v, int32_t total_rows,
                              const int32_t* block_table, const int32_t* first_lens, const int32_t* seq_lens, const int32_t* cu_lens,
                              int32_t batch, int32_t max_blocks, int32_t max_seq_len, void* stream)
{
    const pa_status st = check_mx4(cache, dtype);
    if (st != PA_OK) return st;
    if (total_rows < 0 || batch < 0 || max_blocks < 0 || max_seq_len < 0) return PA_ERR_INVALID_ARG;
    if (total_rows == 0 || batch == 0 || max_seq_len == 0) return PA_OK;
    if (!out_k || !out_v || !block_table || !seq_lens || !cu_lens || max_blocks == 0) return PA_ERR_INVALID_ARG;
    if ((((uintptr_t)out_k | (uintptr_t)out_v) & 15) || cache->num_kv_heads > 8192) return PA_ERR_UNSUPPORTED;
    // (256 threads for 8 rows that may have a token: those of a launch stay below 2^32)
    if (std::min((int64_t)total_rows, (int64_t)batch * max_seq_len) > (1 << 27) - 8) return PA_ERR_UNSUPPORTED;
    return launch_kv_gather_mx4(cache, dtype, out_k, out_v, total_rows, block_table, first_lens, seq_lens, cu_lens, batch, max_blocks,
                                max_seq_len, stream_of(stream));
}

size_t paged_attention_mx4_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                           int32_t total_q, int32_t max_q_len, int32_t max_seq_len)
{
    if (batch <= 0 || num_kv_heads <= 0 || num_q_heads < num_kv_heads || head_dim <= 0 || total_q <= 0 || max_q_len <= 0 || max_seq_len < 0)
        return 256;
    return mx4_workspace_bytes(batch, num_q_heads, num_kv_heads, head_dim, total_q, max_q_len, max_seq_len);
}

pa_status paged_attention_mx4(const pa_mx4_cache_desc* cache, pa_dtype dtype, const void* q, void* out, float* lse,
                              const int32_t* cu_q_lens, int32_t total_q, int32_t max_q_len, const int32_t* block_table,
                              const int32_t* seq_lens, int32_t batch, int32_t num_q_heads, int32_t max_blocks,
                              int32_t max_seq_len, float scale, void* workspace, size_t workspace_bytes, void* stream)
{
    const pa_status st = check_mx4(cache, dtype);
    if (st != PA_OK) return st;
    if (batch < 0 || total_q < 0 || max_q_len < 0 || max_blocks < 0 || max_seq_len < 0) return PA_ERR_INVALID_ARG;
    if (num_q_heads <= 0 || num_q_heads % cache->num_kv_heads != 0 || !(scale == scale)) return PA_ERR_INVALID_ARG;
    if (batch == 0 || total_q == 0 || max_q_len == 0) return PA_OK;
    if (!q || !out || !cu_q_lens || !block_table || !seq_lens) return PA_ERR_INVALID_ARG;
    if (((uintptr_t)q | (uintptr_t)out) & 15) return PA_ERR_UNSUPPORTED;
    if ((int64_t)max_blocks * cache->page_size < max_seq_len) return PA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < paged_attention_mx4_workspace_bytes(batch, num_q_heads, cache->num_kv_heads, cache->head_dim,
                                                                            total_q, max_q_len, max_seq_len))
        return PA_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace & 255) return PA_ERR_INVALID_ARG;
    const Mx4Args a = {cache, dtype, q, out, lse, cu_q_lens, seq_lens, block_table, batch, total_q, max_q_len, num_q_heads, max_blocks,
                       max_seq_len, scale};
    return launch_attention_mx4(a, workspace, stream_of(stream));
}

}  // extern "C"
