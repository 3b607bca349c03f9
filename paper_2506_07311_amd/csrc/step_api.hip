// C ABI of a step of drafted tokens: argument validation and dispatch.  Every check is a host check made before the first
// launch; nothing here touches device memory.
#include <math.h>

#include "common.h"

using namespace pa;

namespace {

bool is_pow2(int32_t x) { return x > 0 && (x & (x - 1)) == 0; }

inline hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }

constexpr int32_t kMaxPath = 8192;     // tokens of a path that the acceptance kernel keeps in LDS

}  // namespace

extern "C" {

pa_status paged_plan_step(const int32_t* ctx_lens, const int32_t* new_lens, int32_t batch, const int32_t* parents,
                          int32_t page_size, int32_t* block_table, int32_t max_blocks, int32_t* num_blocks,
                          const int32_t* free_pages, int32_t* free_count, int32_t max_rows, int32_t* seq_lens,
                          int32_t* cu_q_lens, int32_t* seq_ids, int32_t* positions, int32_t* rope_positions,
                          uint64_t* tree_mask, int32_t mask_words, int32_t* shortage, void* stream)
{
    if (batch < 0 || max_blocks < 0 || max_rows < 0 || mask_words < 0 || !is_pow2(page_size)) return PA_ERR_INVALID_ARG;
    if (batch == 0) return PA_OK;
    if (!ctx_lens || !new_lens || !block_table || !num_blocks || !free_pages || !free_count || !seq_lens || !cu_q_lens ||
        !shortage || max_blocks == 0)
        return PA_ERR_INVALID_ARG;
    if (max_rows > 0 && (!seq_ids || !positions)) return PA_ERR_INVALID_ARG;
    if (tree_mask && (mask_words == 0 || ((uintptr_t)tree_mask & 7))) return PA_ERR_INVALID_ARG;
    if (seq_lens == ctx_lens || seq_lens == new_lens) return PA_ERR_INVALID_ARG;   // (read while they are written)
    StepPlanArgs p = {ctx_lens, new_lens, parents, free_pages, batch, page_size, max_blocks, max_rows, mask_words, block_table,
                      num_blocks, free_count, seq_lens, cu_q_lens, seq_ids, positions, rope_positions, tree_mask, shortage};
    return launch_plan_step(p, stream_of(stream));
}

pa_status paged_release_blocks(const int32_t* keep_lens, int32_t batch, int32_t page_size, int32_t* block_table,
                               int32_t max_blocks, int32_t* num_blocks, int32_t* free_pages, int32_t* free_count,
                               int32_t max_free, void* stream)
{
    if (batch < 0 || max_blocks < 0 || max_free < 0 || !is_pow2(page_size)) return PA_ERR_INVALID_ARG;
    if (batch == 0) return PA_OK;
    if (!keep_lens || !block_table || !num_blocks || !free_pages || !free_count || max_blocks == 0) return PA_ERR_INVALID_ARG;
    return launch_release_blocks(keep_lens, batch, page_size, block_table, max_blocks, num_blocks, free_pages, free_count,
                                 max_free, stream_of(stream));
}

pa_status pa_rope_frequencies(double* inv_freq, float* mscale, int32_t rotary_dim, double base, pa_rope_scaling scaling,
                              double factor, double context, double slow, double fast)
{
    if (!inv_freq || !mscale || rotary_dim < 2 || rotary_dim % 2 || !(base > 1.0) || !(factor >= 1.0) || isinf(base) || isinf(factor))
        return PA_ERR_INVALID_ARG;
    const double r = rotary_dim, two_pi = 6.283185307179586;
    const bool between = scaling == PA_ROPE_PARTS || scaling == PA_ROPE_RAMP;
    if (between && (!(context > 0.0) || !(slow > 0.0) || !(fast > slow) || isinf(context) || isinf(fast))) return PA_ERR_INVALID_ARG;
    if ((int)scaling < PA_ROPE_NONE || (int)scaling > PA_ROPE_RAMP) return PA_ERR_INVALID_ARG;
    if (scaling == PA_ROPE_BASE && rotary_dim > 2) base *= pow(factor, r / (r - 2.0));
    // the number at which a pair would turn so many times in `context` tokens: base^(-2 i / r) context = 2 pi turns
    double from = 0.0, to = 0.0;
    if (scaling == PA_ROPE_RAMP) {
        from = floor(r * log(context / (two_pi * fast)) / (2.0 * log(base)));
        to = ceil(r * log(context / (two_pi * slow)) / (2.0 * log(base)));
        from = from < 0.0 ? 0.0 : from;
        to = to > r - 1.0 ? r - 1.0 : to;
    }
    for (int32_t i = 0; i < rotary_dim / 2; ++i) {
        const double f = pow(base, -2.0 * i / r);
        double keep = 1.0;                                   // how much of f stays unscaled
        if (scaling == PA_ROPE_LINEAR) keep = 0.0;
        if (scaling == PA_ROPE_PARTS) keep = (context * f / two_pi - slow) / (fast - slow);
        if (scaling == PA_ROPE_RAMP) keep = 1.0 - (i - from) / (to - from > 1e-3 ? to - from : 1e-3);
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        inv_freq[i] = f * keep + f / factor * (1.0 - keep);
    }
    *mscale = scaling == PA_ROPE_RAMP ? (float)(0.1 * log(factor) + 1.0) : 1.f;
    return PA_OK;
}

pa_status paged_rope_append(const pa_kv_cache_desc* cache, const void* q, int64_t q_stride, void* q_out,
                            int64_t q_out_stride, int32_t num_q_heads, const void* k_new, int64_t k_stride,
                            const void* v_new, int64_t v_stride, const int32_t* rope_positions, const int32_t* seq_ids,
                            const int32_t* positions, int32_t T, const int32_t* block_table, int32_t batch,
                            int32_t max_blocks, const double* inv_freq, int32_t rotary_dim, int32_t interleaved,
                            float mscale, void* stream)
{
    const pa_status st = check_cache(cache);
    if (st != PA_OK) return st;
    if (T < 0 || batch < 0 || max_blocks < 0 || rotary_dim < 0 || rotary_dim % 2 || rotary_dim > cache->head_dim)
        return PA_ERR_INVALID_ARG;
    if (q_stride < 0 || q_out_stride < 0 || k_stride < 0 || v_stride < 0 || !(mscale == mscale)) return PA_ERR_INVALID_ARG;
    if (!q != !q_out || !k_new != !v_new) return PA_ERR_INVALID_ARG;
    if (T == 0 || (!q && !k_new)) return PA_OK;
    if (q && num_q_heads <= 0) return PA_ERR_INVALID_ARG;
    if (rotary_dim > 0 && (!rope_positions || !inv_freq || ((uintptr_t)inv_freq & 7))) return PA_ERR_INVALID_ARG;
    if (k_new && (!seq_ids || !positions || !block_table || batch == 0 || max_blocks == 0)) return PA_ERR_INVALID_ARG;
    const int64_t epv = cache->dtype == PA_DTYPE_F32 ? 4 : 8;
    const int64_t q_row = (int64_t)num_q_heads * cache->head_dim, kv_row = (int64_t)cache->num_kv_heads * cache->head_dim;
    if (q_stride == 0) q_stride = q_row;
    if (q_out_stride == 0) q_out_stride = q_row;
    if (k_stride == 0) k_stride = kv_row;
    if (v_stride == 0) v_stride = kv_row;
    if (q && (q_stride < q_row || q_out_stride < q_row || (q == q_out && q_stride != q_out_stride))) return PA_ERR_INVALID_ARG;
    if (k_new && (k_stride < kv_row || v_stride < kv_row)) return PA_ERR_INVALID_ARG;
    if (q_stride % epv || q_out_stride % epv || k_stride % epv || v_stride % epv) return PA_ERR_UNSUPPORTED;
    if (((uintptr_t)q | (uintptr_t)q_out | (uintptr_t)k_new | (uintptr_t)v_new) & 15) return PA_ERR_UNSUPPORTED;
    RopeArgs r = {q, q_out, k_new, v_new, q_stride, q_out_stride, k_stride, v_stride, inv_freq, rope_positions, seq_ids, positions,
                  block_table, T, num_q_heads, batch, max_blocks, rotary_dim, interleaved != 0, mscale};
    return launch_rope_append(cache, r, stream_of(stream));
}

size_t paged_attention_tree_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim,
                                            int32_t total_q, int32_t max_q_len, int32_t max_seq_len)
{
    if (batch <= 0 || num_kv_heads <= 0 || num_q_heads < num_kv_heads || head_dim <= 0 || total_q <= 0 || max_q_len < 0 ||
        max_seq_len < 0)
        return 256;
    size_t most = 256;                                       // (the type is not known here)
    for (const bool f32 : {false, true}) {
        const TreePlan p = plan_tree(batch, num_q_heads, num_kv_heads, head_dim, max_q_len, max_seq_len, f32);
        const size_t bytes = p.part_o_bytes + p.part_lse_bytes + p.cuts_bytes;
        if (bytes > most) most = bytes;
    }
    return most;
}

pa_status paged_attention_tree(const pa_kv_cache_desc* cache, const void* q, void* out, float* lse,
                               const int32_t* cu_q_lens, int32_t total_q, int32_t max_q_len, const uint64_t* tree_mask,
                               int32_t mask_words, const int32_t* block_table, const int32_t* seq_lens, int32_t batch,
                               int32_t num_q_heads, int32_t max_blocks, int32_t max_seq_len, float scale, void* workspace,
                               size_t workspace_bytes, void* stream)
{
    const pa_status st = check_cache(cache);
    if (st != PA_OK) return st;
    if (batch < 0 || total_q < 0 || max_q_len < 0 || mask_words < 0 || max_blocks < 0 || max_seq_len < 0)
        return PA_ERR_INVALID_ARG;
    if (num_q_heads <= 0 || num_q_heads % cache->num_kv_heads != 0 || !(scale == scale)) return PA_ERR_INVALID_ARG;
    if (batch == 0 || total_q == 0 || max_q_len == 0) return PA_OK;
    if (!q || !out || !cu_q_lens || !tree_mask || !block_table || !seq_lens) return PA_ERR_INVALID_ARG;
    if ((int64_t)mask_words * 64 < max_q_len || ((uintptr_t)tree_mask & 7)) return PA_ERR_INVALID_ARG;
    if (((uintptr_t)q | (uintptr_t)out) & 15) return PA_ERR_UNSUPPORTED;
    if ((int64_t)max_blocks * cache->page_size < max_seq_len) return PA_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < paged_attention_tree_workspace_bytes(batch, num_q_heads, cache->num_kv_heads, cache->head_dim,
                                                                             total_q, max_q_len, max_seq_len))
        return PA_ERR_WORKSPACE_TOO_SMALL;
    if ((uintptr_t)workspace & 255) return PA_ERR_INVALID_ARG;
    TreeArgs a = {make_view(cache), cache->dtype, q, out, lse, cu_q_lens, seq_lens, tree_mask, block_table, mask_words, batch, total_q,
                  max_q_len, num_q_heads, max_blocks, max_seq_len, scale};
    if (!portable_kernels_only() && tree_mfma_supported(a)) return launch_tree_mfma(a, workspace, stream_of(stream));
    return launch_tree_generic(a, stream_of(stream));
}

pa_status paged_tree_accept(const pa_kv_cache_desc* cache, const int32_t* cu_q_lens, const int32_t* seq_lens, int32_t batch,
                            int32_t max_q_len, const int32_t* parents, const int32_t* tokens, const int32_t* targets,
                            int32_t* path, int32_t max_path, int32_t* path_lens, int32_t* next_tokens, int32_t* kept_lens,
                            const int32_t* block_table, int32_t max_blocks, void* stream)
{
    const pa_status st = check_cache(cache);
    if (st != PA_OK) return st;
    if (batch < 0 || max_q_len < 0 || max_path <= 0 || max_blocks < 0) return PA_ERR_INVALID_ARG;
    if (!tokens != !targets || !tokens != !parents || (!tokens && next_tokens)) return PA_ERR_INVALID_ARG;
    if (batch == 0) return PA_OK;
    if (!cu_q_lens || !seq_lens || !path || !path_lens || !block_table || max_blocks == 0) return PA_ERR_INVALID_ARG;
    if (kept_lens == seq_lens) return PA_ERR_INVALID_ARG;     // (read while they are written)
    const int32_t cap = max_path < max_q_len ? max_path : max_q_len > 0 ? max_q_len : 1;
    if (cap > kMaxPath) return PA_ERR_UNSUPPORTED;
    TreeAcceptArgs t = {cu_q_lens, seq_lens, parents, tokens, targets, block_table, path, path_lens, next_tokens, kept_lens, batch,
                        max_path, cap, max_blocks};
    return launch_tree_accept(cache, t, stream_of(stream));
}

}  // extern "C"
