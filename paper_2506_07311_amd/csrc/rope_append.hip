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

// Where token t goes in the pools: nowhere (-1) without a position or a page.
__device__ __forceinline__ int64_t slot_of(const RopeKernelArgs& a, int32_t t)
{
    const int32_t pos = a.positions[t], s = a.seq_ids[t];
    if (pos < 0 || s < 0 || s >= a.batch || (pos >> a.log2_page) >= a.max_blocks) return -1;
    const int32_t page = a.block_table[(int64_t)s * a.max_blocks + (pos >> a.log2_page)];
    if (page < 0 || page >= a.num_pages) return -1;
    return (int64_t)page * a.page_stride + (int64_t)(pos & ((1 << a.log2_page) - 1)) * a.token_stride;
}

// mscale times cosine and sine of pair i of a token.
__device__ __forceinline__ float2 turn_of(const RopeKernelArgs& a, int32_t t, int32_t i)
{
    const double turns = (double)a.rope_positions[t] * (a.inv_freq[i] * 0.15915494309189535);
    float sn, cs;
    sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
    return float2{cs * a.mscale, sn * a.mscale};
}

// 16 bytes at a time, where the turned part divides into such pieces.  A workgroup takes a token, or a part of one's heads where
// there are few: cosines and sines once for all heads into LDS, then a thread's pieces: two of a pair of halves, one of neighbours, one to
// copy.  Bound by reading and writing q, K and V once; a thread's first piece is on its way while the angles are formed.  8192 tokens of 32 / 8
// heads of 128, 201 MB read and written: 34 us (5.9 TB/s) on the same data again, 43 (4.7, as a copy of 4 GiB) on data from memory.  Four
// tokens a workgroup instead of one: 33.8 / 33.3, 5000 tokens 23.6 / 23.7, 2048 14.7 / 11.1.
template <pa_dtype DT, bool INTER>
__global__ __launch_bounds__(kThreads) void paged_rope_append_wide_kernel(RopeKernelArgs a)
{
    typedef Elem<DT> E;
    typedef typename E::T T;
    constexpr int V = 16 / sizeof(T);
    __shared__ __attribute__((aligned(16))) float sm_c[128], sm_s[128];   // head_dim is at most 256
    __shared__ int64_t sm_slot;
    const int32_t d = a.head_dim, half = a.half;
    const int64_t t = blockIdx.x;
    const int32_t turned = INTER ? 2 * half / V : half / V;  // pieces of a head that turn, then those to copy
    const int32_t pieces = turned + (d - 2 * half) / V, copies = d / V;
    const int32_t q_tasks = a.q_heads * pieces, k_tasks = a.kv_heads * pieces, all = q_tasks + k_tasks + a.kv_heads * copies;
    const int32_t mine = (all + (int32_t)gridDim.y - 1) / (int32_t)gridDim.y, begin = mine * (int32_t)blockIdx.y;
    const int32_t end = min(begin + mine, all);

    struct Piece {
        const T* src;            // of the piece's first element
        int32_t u;               // number of the piece in its head; -1: to copy
        int32_t what;            // 0: q, 1: K, 2: V
        int64_t at;              // where it goes within its token
    };
    auto locate = [&](int32_t j) {
        Piece p;
        p.what = j < q_tasks ? 0 : j < q_tasks + k_tasks ? 1 : 2;
        j -= p.what == 0 ? 0 : p.what == 1 ? q_tasks : q_tasks + k_tasks;
        const int32_t n = p.what == 2 ? copies : pieces, h = j / n;
        p.u = j - h * n;
        int32_t first = p.u * V;                             // element of the head
        if (p.what == 2 || p.u >= turned) {
            if (p.what != 2) first = 2 * half + (p.u - turned) * V;
            p.u = -1;
        }
        const T* const base = p.what == 0 ? (const T*)a.q + t * a.q_stride : p.what == 1 ? (const T*)a.k_new + t * a.k_stride
                                                                                           : (const T*)a.v_new + t * a.v_stride;
        p.src = base + (int64_t)h * d + first;
        p.at = (p.what == 0 ? (int64_t)h * d : h * a.head_stride) + first;
        return p;
    };
    struct Pair {
        uint4 x, y;
    };
    auto load = [&](const Piece& p) {
        Pair v;
        v.x = *reinterpret_cast<const uint4*>(p.src);
        v.y = v.x;
        if (!INTER && p.u >= 0) v.y = *reinterpret_cast<const uint4*>(p.src + half);
        return v;
    };
    Piece p;
    Pair v;
    int32_t i = begin + threadIdx.x;
    if (i < end) {
        p = locate(i);
        v = load(p);
    }
    if (a.kv_heads > 0 && threadIdx.x == 0) sm_slot = slot_of(a, (int32_t)t);
    if ((int)threadIdx.x < half) {
        const float2 cs = turn_of(a, (int32_t)t, threadIdx.x);
        sm_c[threadIdx.x] = cs.x;
        sm_s[threadIdx.x] = cs.y;
    }
    __syncthreads();
    while (i < end) {
        T* dst = nullptr;
        if (p.what == 0) dst = (T*)a.q_out + t * a.q_out_stride + p.at;
        else if (sm_slot >= 0) dst = (T*)(p.what == 1 ? a.k_cache : a.v_cache) + sm_slot + p.at;
        if (dst) {
            if (p.u >= 0) {
                T x[V], y[V];
                __builtin_memcpy(x, &v.x, 16);
                __builtin_memcpy(y, &v.y, 16);
                if (INTER) {
                    const int32_t at = p.u * (V / 2);
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const float c = sm_c[at + e / 2], s = sm_s[at + e / 2];
                        const float fx = E::get(x[e]), fy = E::get(x[e + 1]);
                        x[e] = E::put(fx * c - fy * s);
                        x[e + 1] = E::put(fx * s + fy * c);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float c = sm_c[p.u * V + e], s = sm_s[p.u * V + e];
                        const float fx = E::get(x[e]), fy = E::get(y[e]);
                        x[e] = E::put(fx * c - fy * s);
                        y[e] = E::put(fx * s + fy * c);
                    }
                    __builtin_memcpy(&v.y, y, 16);
                    *reinterpret_cast<uint4*>(dst + half) = v.y;
                }
                __builtin_memcpy(&v.x, x, 16);
            }
            *reinterpret_cast<uint4*>(dst) = v.x;
        }
        i += kThreads;
        if (i < end) {
            p = locate(i);
            v = load(p);
        }
    }
}

// Pair by pair, whatever the turned part: a workgroup a token.
template <pa_dtype DT, bool INTER>
__global__ __launch_bounds__(kThreads) void paged_rope_append_kernel(RopeKernelArgs a)
{
    typedef Elem<DT> E;
    typedef typename E::T T;
    __shared__ float2 sm_cs[128];                            // head_dim is at most 256
    const int32_t t = blockIdx.x;
    const int32_t d = a.head_dim, half = a.half;
    if ((int)threadIdx.x < half) sm_cs[threadIdx.x] = turn_of(a, t, threadIdx.x);
    const int64_t slot = a.kv_heads > 0 ? slot_of(a, t) : -1;
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

template <pa_dtype DT, bool INTER>
void launch_layout(const RopeKernelArgs& a, hipStream_t stream)
{
    constexpr int V = DT == PA_DTYPE_F32 ? 4 : 8;
    if ((INTER ? 2 * a.half : a.half) % V != 0) {
        hipLaunchKernelGGL((paged_rope_append_kernel<DT, INTER>), dim3(a.T), dim3(kThreads), 0, stream, a);
        return;
    }
    // Where tokens are few, a thread takes a piece or two (us with / without, 32 / 8 heads of 128: 40 tokens 3.9 / 4.6, 300 4.4 / 5.2, 700
    // 6.0 / 6.3, 2048 11.4 / 11.1).
    const int32_t pieces = (a.q_heads + a.kv_heads) * ((INTER ? 2 * a.half : a.half) / V + (a.head_dim - 2 * a.half) / V) +
                           a.kv_heads * a.head_dim / V;
    const int32_t parts = a.T >= 1024 ? 1 : (pieces + kThreads - 1) / kThreads;
    hipLaunchKernelGGL((paged_rope_append_wide_kernel<DT, INTER>), dim3(a.T, parts), dim3(kThreads), 0, stream, a);
}

template <pa_dtype DT>
void launch_dtype(const RopeKernelArgs& a, bool inter, hipStream_t stream)
{
    if (inter) launch_layout<DT, true>(a, stream);
    else launch_layout<DT, false>(a, stream);
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
