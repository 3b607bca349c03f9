// Rotary positions of a step's queries and keys, and Algorithm 1's Assign of the turned K rows and the V rows, as one pass.
//
// A head's leading rotary_dim elements are pairs (x, y); pair i of a token at position p is turned by theta = p f_i:
//     (x, y) -> m (x cos theta - y sin theta, x sin theta + y cos theta)
// with f_i = inv_freq[i] radians a position and m = mscale; the rest of the head is copied.  A pair is (i, i + r/2) or
// (2i, 2i + 1).  At position 131072 a 32-bit product p f_i is off by up to 0.008 radians, so the angle is formed in 64 bits, as
// turns, and only what is left of a whole turn goes to the 32-bit sine and cosine; their products with x and y are
// 32-bit, the result is rounded once.
#include "common.h"

namespace pa {

namespace {

constexpr int kThreads = 256;

struct RopeKernelArgs {
    const void* q;
    void* q_out;
    const void* k_new;
    const void* v_new;
    void* k_cache;
    void* v_cache;
    const double* inv_freq;
    const int32_t* rope_positions;
    const int32_t* seq_ids;
    const int32_t* positions;
    const int32_t* block_table;
    int64_t q_stride, q_out_stride, k_stride, v_stride;      // elements between tokens
    int64_t page_stride, token_stride, head_stride;          // elements
    int32_t T, q_heads, kv_heads;                            // (0 heads: that part is absent)
    int32_t head_dim, half, batch, max_blocks, log2_page, num_pages;
    float mscale;
};

template <pa_dtype DT>
struct Elem;
template <>
struct Elem<PA_DTYPE_F32> {
    typedef float T;
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ float put(float x) { return x; }
};
template <>
struct Elem<PA_DTYPE_BF16> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(uint16_t x) { return bf16_bits_to_float(x); }
    static __device__ __forceinline__ uint16_t put(float x) { return (uint16_t)float_to_bf16_bits(x); }
};
template <>
struct Elem<PA_DTYPE_F16> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(uint16_t x) { return f16_bits_to_float(x); }
    static __device__ __forceinline__ uint16_t put(float x) { return (uint16_t)float_to_f16_bits(x); }
};

// One workgroup a token: cosines and sines of its pairs into LDS, then element by element over the heads.
template <pa_dtype DT, bool INTER>
__global__ __launch_bounds__(kThreads) void paged_rope_append_kernel(RopeKernelArgs a)
{
    typedef Elem<DT> E;
    typedef typename E::T T;
    __shared__ float2 sm_cs[128];                            // head_dim is at most 256
    const int32_t t = blockIdx.x;
    const int32_t d = a.head_dim, half = a.half;
    if ((int)threadIdx.x < half) {
        const double turns = (double)a.rope_positions[t] * (a.inv_freq[threadIdx.x] * 0.15915494309189535);
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        sm_cs[threadIdx.x] = float2{cs * a.mscale, sn * a.mscale};
    }
    // where the token goes: nowhere without a position or a page
    int64_t slot = -1;
    if (a.kv_heads > 0) {
        const int32_t pos = a.positions[t], s = a.seq_ids[t];
        if (pos >= 0 && s >= 0 && s < a.batch && (pos >> a.log2_page) < a.max_blocks) {
            const int32_t page = a.block_table[(int64_t)s * a.max_blocks + (pos >> a.log2_page)];
            if (page >= 0 && page < a.num_pages)
                slot = (int64_t)page * a.page_stride + (int64_t)(pos & ((1 << a.log2_page) - 1)) * a.token_stride;
        }
    }
    __syncthreads();
    const int32_t units = half + (d - 2 * half);             // pairs, then single elements
    auto turn = [&](const T* src, T* dst, int32_t u) {
        if (u >= half) {
            dst[u + half] = src[u + half];
            return;
        }
        const int32_t ix = INTER ? 2 * u : u, iy = INTER ? 2 * u + 1 : u + half;
        const float2 cs = sm_cs[u];
        const float x = E::get(src[ix]), y = E::get(src[iy]);
        dst[ix] = E::put(x * cs.x - y * cs.y);
        dst[iy] = E::put(x * cs.y + y * cs.x);
    };
    for (int32_t i = threadIdx.x; i < a.q_heads * units; i += kThreads) {
        const int32_t h = i / units, u = i % units;
        turn((const T*)a.q + t * a.q_stride + (int64_t)h * d, (T*)a.q_out + t * a.q_out_stride + (int64_t)h * d, u);
    }
    if (slot < 0) return;
    for (int32_t i = threadIdx.x; i < a.kv_heads * units; i += kThreads) {
        const int32_t h = i / units, u = i % units;
        turn((const T*)a.k_new + t * a.k_stride + (int64_t)h * d, (T*)a.k_cache + slot + h * a.head_stride, u);
    }
    for (int32_t i = threadIdx.x; i < a.kv_heads * d; i += kThreads) {
        const int32_t h = i / d, u = i % d;
        ((T*)a.v_cache)[slot + h * a.head_stride + u] = ((const T*)a.v_new)[t * a.v_stride + i];
    }
}

template <pa_dtype DT>
void launch_dtype(const RopeKernelArgs& a, bool inter, hipStream_t stream)
{
    if (inter)
        hipLaunchKernelGGL((paged_rope_append_kernel<DT, true>), dim3(a.T), dim3(kThreads), 0, stream, a);
    else
        hipLaunchKernelGGL((paged_rope_append_kernel<DT, false>), dim3(a.T), dim3(kThreads), 0, stream, a);
}

}  // namespace

pa_status launch_rope_append(const pa_kv_cache_desc* c, const RopeArgs& r, hipStream_t stream)
{
    const CacheView v = make_view(c);
    RopeKernelArgs a;
    a.q = r.q;
    a.q_out = r.q_out;
    a.k_new = r.k_new;
    a.v_new = r.v_new;
    a.k_cache = c->k_cache;
    a.v_cache = c->v_cache;
    a.inv_freq = r.inv_freq;
    a.rope_positions = r.rope_positions;
    a.seq_ids = r.seq_ids;
    a.positions = r.positions;
    a.block_table = r.block_table;
    a.q_stride = r.q_stride;
    a.q_out_stride = r.q_out_stride;
    a.k_stride = r.k_stride;
    a.v_stride = r.v_stride;
    a.page_stride = c->page_stride;
    a.token_stride = c->token_stride;
    a.head_stride = c->head_stride;
    a.T = r.T;
    a.q_heads = r.q ? r.num_q_heads : 0;
    a.kv_heads = r.k_new ? c->num_kv_heads : 0;
    a.head_dim = c->head_dim;
    a.half = r.rotary_dim / 2;
    a.batch = r.batch;
    a.max_blocks = r.max_blocks;
    a.log2_page = v.log2_page;
    a.num_pages = c->num_pages;
    a.mscale = r.mscale;
    ProfileScope prof("paged_rope_append_kernel", stream);
    if (c->dtype == PA_DTYPE_F32) launch_dtype<PA_DTYPE_F32>(a, r.interleaved, stream);
    else if (c->dtype == PA_DTYPE_BF16) launch_dtype<PA_DTYPE_BF16>(a, r.interleaved, stream);
    else launch_dtype<PA_DTYPE_F16>(a, r.interleaved, stream);
    return launch_status();
}

}  // namespace pa
