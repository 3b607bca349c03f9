// Algorithm 1's Gather from a cache of 4-bit elements: the values that codes and scales stand for, in the wanted type; and the copy of a page.
#include <algorithm>

#include "mx4.h"

namespace pa {

namespace {

constexpr int kThreads = 256;

// ROWS rows a workgroup at a time, a thread 8 elements of a row's head at a time: 4 bytes of codes and a scale in, 16 or 32 bytes out.  Bound by
// the bytes that it writes: 4096 tokens of 8 heads of 256, 43 MB in 16 bits, 14.0 us, 76 MB in 32 19.2 (there a lane's two stores fill a line's two halves in
// turn).  MORE: the grid does not reach all rows, and a workgroup goes on (without that loop 320000 tokens of 8 heads of 128 take
// 399 us, with it 411).
template <pa_dtype DT, int ROWS, bool MORE>
__global__ __launch_bounds__(kThreads) void paged_kv_gather_mx4_kernel(Mx4View c, void* out_k, void* out_v, int32_t rows,
                                                                       const int32_t* __restrict__ block_table,
                                                                       const int32_t* __restrict__ first_lens,
                                                                       const int32_t* __restrict__ seq_lens,
                                                                       const int32_t* __restrict__ cu_lens, int32_t batch, int32_t max_blocks,
                                                                       uint32_t by_heads)
{
    __shared__ int64_t sm_page[ROWS];                        // bytes from the first record on; -1: no such token
    __shared__ int32_t sm_slot[ROWS];
    const int32_t d = c.head_dim, lp = c.log2_page;
    const int lane = threadIdx.x & 63;
    const int32_t log2_pieces = d == 64 ? 3 : d == 128 ? 4 : 5, pieces = 1 << log2_pieces, each = ROWS * c.num_kv_heads * pieces;
    for (int32_t row0 = (int32_t)blockIdx.x * ROWS;;) {
        // a wave finds its rows' sequences: the first whose end lies behind the row
        for (int32_t k = threadIdx.x >> 6; k < ROWS; k += kThreads / 64) {
            const int32_t r = row0 + min(k, rows - 1 - row0);    // (the last row's again)
            int32_t s = -1;
            for (int32_t i0 = 0; i0 < batch && s < 0; i0 += 64) {
                const uint64_t hit = __ballot(i0 + lane < batch && cu_lens[min(i0 + lane, batch - 1) + 1] > r);
                if (hit) s = i0 + __ffsll((unsigned long long)hit) - 1;
            }
            int64_t at = -1;
            int32_t slot = 0;
            if (s >= 0 && k < rows - row0 && r >= cu_lens[s]) {
                const int64_t t = (int64_t)r - cu_lens[s] + (first_lens ? max(first_lens[s], 0) : 0);
                if (t < seq_lens[s] && t >> lp < max_blocks) {
                    const int32_t page = block_table[(int64_t)s * max_blocks + (t >> lp)];
                    if (page >= 0 && page < c.num_pages) at = (int64_t)page * c.page_stride;
                    slot = (int32_t)t & ((1 << lp) - 1);
                }
            }
            if (lane == 0) {
                sm_page[k] = at;
                sm_slot[k] = slot;
            }
        }
        __syncthreads();
        for (int32_t i = threadIdx.x; i < 2 * each; i += kThreads) {
            const int32_t what = i >= each, j = what ? i - each : i;
            const uint32_t u = j & (pieces - 1), hk = (uint32_t)j >> log2_pieces;
            const uint32_t k = c.num_kv_heads == 1 ? hk : __umulhi(hk, by_heads), h = hk - k * c.num_kv_heads;
            if (sm_page[k] < 0) continue;
            const int32_t slot = sm_slot[k];
            const char* const base = c.records + sm_page[k];
            const char* const rec = base + h * c.head_stride;
            uint32_t codes;
            if (what == 0) {
                codes = *reinterpret_cast<const uint32_t*>(rec + mx4_k_codes(d, slot) + 4 * u);
            } else if (d == 64) {
                codes = *reinterpret_cast<const uint16_t*>(rec + mx4_v_codes(lp, d, slot, 2 * u)) |
                        (uint32_t)*reinterpret_cast<const uint16_t*>(rec + mx4_v_codes(lp, d, slot, 2 * u + 1)) << 16;
            } else {
                codes = *reinterpret_cast<const uint32_t*>(rec + mx4_v_codes(lp, d, slot, 2 * u));
            }
            const uint32_t scale = *reinterpret_cast<const uint8_t*>(rec + mx4_scale(lp, d, slot, u / 4, what));
            const float unit = __uint_as_float(scale << 23); // (the conversion reads its exponent alone: 0 is 2^-127, 255 NaN)
            const int64_t at = (((int64_t)row0 + k) * c.num_kv_heads + h) * d + 8 * u;
            typedef __attribute__((ext_vector_type(2))) float f32x2;
            float x[8];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x2 v = b == 0 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0)
                                : b == 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1)
                                : b == 2 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2)
                                         : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3);
                x[2 * b] = v[0];
                x[2 * b + 1] = v[1];
            }
            if (DT == PA_DTYPE_F32) {
                float* const dst = (float*)(what ? out_v : out_k) + at;
                store_past_cache(dst, __builtin_bit_cast(uint4, float4{x[0], x[1], x[2], x[3]}));
                store_past_cache(dst + 4, __builtin_bit_cast(uint4, float4{x[4], x[5], x[6], x[7]}));
            } else {
                typedef typename std::conditional<DT == PA_DTYPE_F16, ElemF16, ElemBf16>::type E;
                store_past_cache((uint16_t*)(what ? out_v : out_k) + at,
                                 uint4{E::pack(x[0], x[1]), E::pack(x[2], x[3]), E::pack(x[4], x[5]), E::pack(x[6], x[7])});
            }
        }
        if (!MORE) return;
        if (rows - row0 <= (int32_t)gridDim.x * ROWS) return;
        row0 += (int32_t)gridDim.x * ROWS;
        if (row0 >= cu_lens[batch]) return;
        __syncthreads();                                     // (before the next rows' pages)
    }
}

// A KV head's record a blockIdx.y.
__global__ __launch_bounds__(kThreads) void paged_mx4_copy_page_kernel(const char* src, char* dst, int64_t head_stride, int32_t record)
{
    const int32_t at = ((int32_t)blockIdx.x * kThreads + (int32_t)threadIdx.x) * 16;
    const int64_t head = (int64_t)blockIdx.y * head_stride;
    if (at < record) *reinterpret_cast<uint4*>(dst + head + at) = *reinterpret_cast<const uint4*>(src + head + at);
}

}  // namespace

pa_status launch_mx4_copy_page(const pa_mx4_cache_desc* c, int32_t src_page, int32_t dst_page, hipStream_t stream)
{
    if (src_page < 0 || dst_page < 0 || src_page >= c->num_pages || dst_page >= c->num_pages) return PA_ERR_INVALID_ARG;
    if (c->num_kv_heads > 65535) return PA_ERR_UNSUPPORTED;
    const int32_t record = (int32_t)pa_mx4_record_bytes(c->page_size, c->head_dim);   // a multiple of 16, at most 2^28 17 / 16
    const dim3 grid((uint32_t)((record + 16 * kThreads - 1) / (16 * kThreads)), (uint32_t)c->num_kv_heads);
    ProfileScope prof("paged_mx4_copy_page_kernel", stream);
    hipLaunchKernelGGL(paged_mx4_copy_page_kernel, grid, dim3(kThreads), 0, stream, (const char*)c->records + src_page * c->page_stride,
                       (char*)c->records + dst_page * c->page_stride, c->head_stride, record);
    return launch_status();
}

pa_status launch_kv_gather_mx4(const pa_mx4_cache_desc* c, pa_dtype dtype, void* out_k, void* out_v, int32_t rows,
                               const int32_t* block_table, const int32_t* first_lens, const int32_t* seq_lens, const int32_t* cu_lens,
                               int32_t batch, int32_t max_blocks, int32_t max_seq_len, hipStream_t stream)
{
    const Mx4View v = make_view(c);
    // x / heads = high word of x ceil(2^32 / heads) while x heads < 2^32; x is below 8 heads
    const uint32_t by_heads = (uint32_t)((((int64_t)1 << 32) + c->num_kv_heads - 1) / c->num_kv_heads);
    // Rows of a workgroup (us with 8 / 1, 8 KV heads of 128, append and gather: 80 rows 9.7 / 6.3, 600 11.1 / 7.8, 1400 13.4 / 11.3, 3000 16.7 / 16.8,
    // 6000 23.4 / 25.7).
    const int32_t each = rows <= 2048 ? 1 : 8;
    // Workgroups for as many rows as there can be tokens, and to fill the machine: what `rows` has room for beyond them they pass over in turn (3000 tokens
    // into 2^20 rows 6.6 us, with workgroups for all rows 140).
    const int64_t pieces = ((int64_t)rows + each - 1) / each, tokens = (int64_t)batch * max_seq_len;
    const uint32_t grid = (uint32_t)std::min(pieces, std::max(tokens / each + 1, (int64_t)2048));
    const bool more = grid < pieces;                         // (pieces of 8 rows, then)
    ProfileScope prof("paged_kv_gather_mx4_kernel", stream);
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, stream, v, out_k, out_v, rows, block_table, first_lens, seq_lens, cu_lens, batch,
                           max_blocks, by_heads);
    };
    auto of = [&](auto type) {
        constexpr pa_dtype DT = decltype(type)::value;
        if (each == 1) launch(paged_kv_gather_mx4_kernel<DT, 1, false>);
        else more ? launch(paged_kv_gather_mx4_kernel<DT, 8, true>) : launch(paged_kv_gather_mx4_kernel<DT, 8, false>);
    };
    if (dtype == PA_DTYPE_F32) of(std::integral_constant<pa_dtype, PA_DTYPE_F32>());
    else if (dtype == PA_DTYPE_BF16) of(std::integral_constant<pa_dtype, PA_DTYPE_BF16>());
    else of(std::integral_constant<pa_dtype, PA_DTYPE_F16>());
    return launch_status();
}

}  // namespace pa
