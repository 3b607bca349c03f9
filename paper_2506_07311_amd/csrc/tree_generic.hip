// Attention of trees of drafted tokens, portable kernel: any dtype, head_dim, page size and group.
//
// Query i of a sequence with n drafted tokens and len keys sees the context, keys j < len - n, and of the drafted tokens those
// its mask names: key len - n + t if bit t of its words is set.  One workgroup a (query, head); its four waves take 64 keys in
// turn: a lane computes the score of one key from its row, the wave the block's maximum and sum (online softmax in 32 bits),
// then lanes stand for columns and walk the block's keys.  K and V are read once per query and head.
#include "common.h"

namespace pa {

namespace {

constexpr int kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kShift = 24.f, kLargest = 0x1p-24f;   // weight of the largest score: of up to 2^24 keys no sum of finite values overflows

template <pa_dtype DT>
__device__ __forceinline__ float load_elem(const void* p, int64_t i)
{
    if (DT == PA_DTYPE_F32) return static_cast<const float*>(p)[i];
    const uint32_t b = static_cast<const uint16_t*>(p)[i];
    return DT == PA_DTYPE_BF16 ? bf16_bits_to_float(b) : f16_bits_to_float(b);
}

template <pa_dtype DT>
__device__ __forceinline__ void store_elem(void* p, int64_t i, float x)
{
    if (DT == PA_DTYPE_F32) static_cast<float*>(p)[i] = x;
    else static_cast<uint16_t*>(p)[i] = (uint16_t)(DT == PA_DTYPE_BF16 ? float_to_bf16_bits(x) : float_to_f16_bits(x));
}

template <pa_dtype DT>
__global__ __launch_bounds__(kWaves * 64) void paged_attention_tree_generic_kernel(
    CacheView cache, const void* __restrict__ q, void* __restrict__ out, float* __restrict__ lse,
    const int32_t* __restrict__ cu_q_lens, const int32_t* __restrict__ seq_lens, const uint64_t* __restrict__ tree_mask,
    int32_t mask_words, const int32_t* __restrict__ block_table, int32_t batch, int32_t num_q_heads, int32_t max_blocks,
    float scale)
{
    __shared__ float sm_q[256];
    __shared__ float sm_p[kWaves][64];
    __shared__ float sm_o[kWaves][256];
    __shared__ float sm_m[kWaves], sm_l[kWaves];
    const int32_t row = blockIdx.x, h = blockIdx.y;
    if (row >= cu_q_lens[batch]) return;                     // behind the last sequence: left as it was
    const RowInfo r = locate_row(cu_q_lens, seq_lens, batch, row, 0);
    const int32_t d = cache.head_dim;
    const int32_t kvh = h / (num_q_heads / cache.num_kv_heads);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t at = ((int64_t)row * num_q_heads + h) * d;
    const uint64_t* const mask = tree_mask + (int64_t)row * mask_words;
    const int32_t* const table = block_table + (int64_t)r.seq * max_blocks;
    for (int32_t c = threadIdx.x; c < d; c += kWaves * 64) sm_q[c] = load_elem<DT>(q, at + c);
    __syncthreads();
    const int32_t ctx = r.len - r.q_len;
    auto slot = [&](int32_t j) {
        return (int64_t)table[j >> cache.log2_page] * cache.page_stride + (int64_t)(j & (cache.page_size - 1)) * cache.token_stride +
               (int64_t)kvh * cache.head_stride;
    };
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int32_t j0 = 64 * wave; j0 < r.len; j0 += 64 * kWaves) {
        const int32_t j = j0 + lane, node = j - ctx;
        const bool seen = j < r.len && (node < 0 || ((node >> 6) < mask_words && (mask[node >> 6] >> (node & 63)) & 1));
        float x = -INFINITY;
        if (seen) {
            const int64_t k = slot(j);
            x = 0.f;
            for (int32_t c = 0; c < d; ++c) x = __builtin_fmaf(sm_q[c], load_elem<DT>(cache.k, k + c), x);
            x *= scale;
        }
        const float top = fmaxf(m, wave_max(x));
        const float use = top == -INFINITY ? 0.f : top;      // (no key so far)
        const float alpha = __builtin_amdgcn_exp2f((m - use) * kLog2e);
        const float p = seen ? kLargest * __builtin_amdgcn_exp2f((x - use) * kLog2e) : 0.f;
        l = l * alpha + wave_sum(p);
        m = top;
        sm_p[wave][lane] = p;
        const uint64_t any = __ballot(seen);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] *= alpha;
        for (int32_t u = 0; u < 64; ++u) {
            if (!((any >> u) & 1)) continue;                 // a key that is not seen is not read
            const float w = sm_p[wave][u];
            const int64_t v = slot(j0 + u);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane + 64 * i < d) o[i] = __builtin_fmaf(w, load_elem<DT>(cache.v, v + lane + 64 * i), o[i]);
        }
    }
    if (lane == 0) {
        sm_m[wave] = m;
        sm_l[wave] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) sm_o[wave][lane + 64 * i] = o[i];
    __syncthreads();
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sm_m[w]);
    float weight[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        // (a wave without a maximum has no keys, its sum is 0, or nothing but NaN among its scores, which it hands on)
        weight[w] = sm_m[w] == -INFINITY ? 0.f * sm_l[w] : __builtin_amdgcn_exp2f((sm_m[w] - top) * kLog2e);
        sum += weight[w] * sm_l[w];
    }
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
    for (int32_t c = threadIdx.x; c < d; c += kWaves * 64) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) x = __builtin_fmaf(weight[w], sm_o[w][c], x);
        store_elem<DT>(out, at + c, x * inv);
    }
    if (lse && threadIdx.x == 0)
        lse[(int64_t)row * num_q_heads + h] = sum == 0.f ? -INFINITY : top + (__builtin_amdgcn_logf(sum) + kShift) * kLn2;
}

template <pa_dtype DT>
void launch_dtype(const TreeArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL((paged_attention_tree_generic_kernel<DT>), dim3(a.total_q, a.num_q_heads), dim3(kWaves * 64), 0, stream,
                       a.cache, a.q, a.out, a.lse, a.cu_q_lens, a.seq_lens, a.tree_mask, a.mask_words, a.block_table, a.batch,
                       a.num_q_heads, a.max_blocks, a.scale);
}

}  // namespace

pa_status launch_tree_generic(const TreeArgs& a, hipStream_t stream)
{
    if (a.num_q_heads > 65535) return PA_ERR_UNSUPPORTED;
    ProfileScope prof("paged_attention_tree_generic_kernel", stream);
    if (a.dtype == PA_DTYPE_F32) launch_dtype<PA_DTYPE_F32>(a, stream);
    else if (a.dtype == PA_DTYPE_BF16) launch_dtype<PA_DTYPE_BF16>(a, stream);
    else launch_dtype<PA_DTYPE_F16>(a, stream);
    return launch_status();
}

}  // namespace pa
