// The 4-bit cache (internal header): where a record holds what, and a block's rounding.  The layout is the header's.
#pragma once

#include "common.h"

namespace pa {

struct Mx4View {
    char* records;
    int64_t page_stride, head_stride;   // bytes
    int32_t log2_page, head_dim, num_kv_heads, num_pages;
};

inline Mx4View make_view(const pa_mx4_cache_desc* c)
{
    Mx4View v = {(char*)c->records, c->page_stride, c->head_stride, 0, c->head_dim, c->num_kv_heads, c->num_pages};
    while ((1 << v.log2_page) < c->page_size) ++v.log2_page;
    return v;
}

#if defined(__HIPCC__)

// 16 bytes of cache lines that the wave fills whole, by one store or two behind each other, and that this kernel's L2 has no further use for (us on
// data from memory, with plain stores / so: 17000 tokens of 8 KV heads of 256 taken out, 140 MB, behind 3000 stored 61 / 40).
__device__ __forceinline__ void store_past_cache(void* dst, uint4 x)
{
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    const u32x4 y = {x.x, x.y, x.z, x.w};
    __builtin_nontemporal_store(y, reinterpret_cast<u32x4*>(dst));
}

// Bytes from a record's start.  K codes of a slot.
__device__ __forceinline__ int32_t mx4_k_codes(int32_t d, int32_t slot) { return slot * (d / 2); }
// V codes of elements 4 u .. 4 u + 3 of a head.
__device__ __forceinline__ int32_t mx4_v_codes(int32_t log2_page, int32_t d, int32_t slot, int32_t u)
{
    const int32_t w = d / 32;                                // bytes of a cell's row: 2, 4 or 8
    return ((d / 2) << log2_page) + ((slot >> 3) * 16 + 2 * u / w) * 8 * w + (slot & 7) * w + 2 * u % w;
}
// Scale of block b of K (what = 0) or V (1).
__device__ __forceinline__ int32_t mx4_scale(int32_t log2_page, int32_t d, int32_t slot, int32_t b, int32_t what)
{
    return ((d + what * (d / 32) + b) << log2_page) + slot;
}

// Scale byte of a block from the bits of its largest magnitude (an infinity's or a NaN's are larger than any finite number's).
__device__ __forceinline__ uint32_t mx4_scale_of(uint32_t top)
{
    const int32_t e = (int32_t)(top >> 23) - 2;
    return top >= 0x7f800000u ? 255u : (uint32_t)max(e, 0);
}

// Codes of eight elements under a scale byte other than 255: the hardware's conversion divides by the power of two, rounds to nearest even
// and ends at 6, as defined.
__device__ __forceinline__ uint32_t mx4_codes(const float (&x)[8], uint32_t scale)
{
    const float unit = __uint_as_float(scale << 23);         // (its exponent alone is read: 0 is 2^-127)
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], unit, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], unit, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], unit, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], unit, 3);
}
__device__ __forceinline__ uint32_t mx4_codes(const float (&x)[4], uint32_t scale)
{
    const float unit = __uint_as_float(scale << 23);
    const uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0], x[1], unit, 0);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], unit, 1);
}

#endif

pa_status check_mx4_cache(const pa_mx4_cache_desc* c);
pa_status launch_mx4_copy_page(const pa_mx4_cache_desc* c, int32_t src_page, int32_t dst_page, hipStream_t stream);
pa_status launch_kv_gather_mx4(const pa_mx4_cache_desc* c, pa_dtype dtype, void* out_k, void* out_v, int32_t rows,
                               const int32_t* block_table, const int32_t* first_lens, const int32_t* seq_lens, const int32_t* cu_lens,
                               int32_t batch, int32_t max_blocks, int32_t max_seq_len, hipStream_t stream);
// Into a 4-bit cache (to4), or one of the tokens' own type (cache).
pa_status launch_norm_rope_append(const pa_kv_cache_desc* cache, const pa_mx4_cache_desc* to4, pa_dtype dtype, const pa_norm_rope& r,
                                  hipStream_t stream);

struct Mx4Args {
    const pa_mx4_cache_desc* cache;
    pa_dtype dtype;
    const void* q;
    void* out;
    float* lse;
    const int32_t* cu_q_lens;
    const int32_t* seq_lens;
    const int32_t* block_table;
    int32_t batch, total_q, max_q_len, num_q_heads, max_blocks, max_seq_len;
    float scale;
};
size_t mx4_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t total_q, int32_t max_q_len,
                           int32_t max_seq_len);
pa_status launch_attention_mx4(const Mx4Args& a, void* workspace, hipStream_t stream);

}  // namespace pa
