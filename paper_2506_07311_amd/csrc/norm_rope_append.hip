// Norms of the heads of q and K, their rotary positions of one or several numbers, and Algorithm 1's Assign, as one pass, into pages
// of the tokens' own type or of 4-bit elements.
//
//     y = x rsqrt(mean(x^2) + eps) (offset + w),   (y_i, y_j) -> m (y_i cos t - y_j sin t, y_i sin t + y_j cos t)
// with t = p[axis of the pair] f_pair, the angle in 64 bits as turns (rope_append.hip).  Everything is 32-bit and rounded once.
#include "mx4.h"

namespace pa {

namespace {

constexpr int kThreads = 256;

// Who a pair's elements are: neighbours; halves, a lane's 16 bytes with another lane's; halves of a turned part that does not divide so.
constexpr int kNeighbours = 0, kHalves = 1, kOddHalves = 2;

struct NormRopeArgs {
    pa_norm_rope r;
    void* k_cache;
    void* v_cache;
    int64_t page_stride, token_stride, head_stride;          // elements (a 4-bit cache: page and head, bytes)
    int32_t q_heads, kv_heads;                               // (0 heads: that part is absent)
    int32_t d, half, log2_page, num_pages;
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

template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}
// What lanes ^ 1, ^ 2, then of the other half of 8 and of 16 hold, once the lanes nearer by agree; further ones through LDS.
template <int STEP>
__device__ __forceinline__ uint32_t other(uint32_t x)
{
    if (STEP == 1) return moved<0xB1>(x);                    // quad_perm 1, 0, 3, 2
    if (STEP == 2) return moved<0x4E>(x);                    // quad_perm 2, 3, 0, 1
    if (STEP == 4) return moved<0x141>(x);                   // row_half_mirror
    if (STEP == 8) return moved<0x140>(x);                   // row_mirror
    return (uint32_t)__shfl_xor((int)x, STEP);
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
    if (LANES > 1) v += __uint_as_float(other<1>(__float_as_uint(v)));
    if (LANES > 2) v += __uint_as_float(other<2>(__float_as_uint(v)));
    if (LANES > 4) v += __uint_as_float(other<4>(__float_as_uint(v)));
    if (LANES > 8) v += __uint_as_float(other<8>(__float_as_uint(v)));
    if (LANES > 16) v += __uint_as_float(other<16>(__float_as_uint(v)));
    if (LANES > 32) v += __uint_as_float(other<32>(__float_as_uint(v)));
    return v;
}
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
    v = max(v, other<1>(v));
    v = max(v, other<2>(v));
    if (LANES > 4) v = max(v, other<4>(v));
    return v;
}

// Elements at .. at + V - 1 of a head: z inv (offset + w).
template <pa_dtype DT, int V>
__device__ __forceinline__ void weigh(float (&z)[V], const void* weights, int64_t at, bool f32, float offset, float inv)
{
    typedef Elem<DT> E;
    typedef typename E::T T;
#pragma unroll
    for (int e = 0; e < V; ++e) z[e] *= inv;
    if (!weights) return;
    if (f32) {
#pragma unroll
        for (int e = 0; e < V; e += 4) {
            const float4 w = *reinterpret_cast<const float4*>((const float*)weights + at + e);
            z[e] *= offset + w.x;
            z[e + 1] *= offset + w.y;
            z[e + 2] *= offset + w.z;
            z[e + 3] *= offset + w.w;
        }
    } else {
        T raw[V];
        const uint4 w = *reinterpret_cast<const uint4*>((const T*)weights + at);
        __builtin_memcpy(raw, &w, 16);
#pragma unroll
        for (int e = 0; e < V; ++e) z[e] *= offset + E::get(raw[e]);
    }
}

// A head is LANES lanes of a wave (a power of two), 16 bytes each; a workgroup has 256 / LANES heads of one token at a time.  Bound by
// reading and writing q, K and V once.
template <pa_dtype DT, int PAIRS, bool TO4, int LANES>
__global__ __launch_bounds__(kThreads) void paged_norm_rope_append_kernel(NormRopeArgs a)
{
    typedef Elem<DT> E;
    typedef typename E::T T;
    constexpr int V = 16 / sizeof(T), HEADS = kThreads / LANES;
    __shared__ __attribute__((aligned(16))) float sm_c[128], sm_s[128];   // head_dim is at most 256
    const pa_norm_rope& r = a.r;
    const int32_t d = a.d, half = a.half, u = threadIdx.x % LANES, first = u * V;
    const int64_t t = blockIdx.x;
    const bool live = first < d;
    const int32_t heads = a.q_heads + 2 * a.kv_heads;
    const int32_t mine = (heads + (int32_t)gridDim.y - 1) / (int32_t)gridDim.y;
    const int32_t begin = mine * (int32_t)blockIdx.y, end = min(begin + mine, heads);
    constexpr bool INTER = PAIRS == kNeighbours;
    const bool turned = first < 2 * half;
    const int32_t partner = PAIRS != kHalves || !turned ? first : first < half ? first + half : first - half;

    struct Piece {
        const T* src;            // of the head
        int32_t what, h;         // 0: q, 1: K, 2: V
        uint4 x, y;
    };
    auto load = [&](int32_t j) {
        Piece p;
        p.what = j < a.q_heads ? 0 : j < a.q_heads + a.kv_heads ? 1 : 2;
        p.h = j - (p.what == 0 ? 0 : p.what == 1 ? a.q_heads : a.q_heads + a.kv_heads);
        p.src = (p.what == 0 ? (const T*)r.q + t * r.q_stride : p.what == 1 ? (const T*)r.k_new + t * r.k_stride
                                                                            : (const T*)r.v_new + t * r.v_stride) + (int64_t)p.h * d;
        p.x = uint4{0, 0, 0, 0};
        p.y = p.x;
        if (live) {
            p.x = *reinterpret_cast<const uint4*>(p.src + first);
            if (PAIRS == kHalves && p.what != 2) p.y = *reinterpret_cast<const uint4*>(p.src + partner);
        }
        return p;
    };
    int32_t j = begin + (int32_t)threadIdx.x / LANES;
    Piece p;
    if (j < end) p = load(j);
    int64_t slot = -1;           // (elements, or in a 4-bit cache bytes, of the page)
    int32_t place = 0;
    if (a.kv_heads > 0) {
        const int32_t pos = r.positions[t], s = r.seq_ids[t];
        if (pos >= 0 && s >= 0 && s < r.batch && (pos >> a.log2_page) < r.max_blocks) {
            const int32_t page = r.block_table[(int64_t)s * r.max_blocks + (pos >> a.log2_page)];
            place = pos & ((1 << a.log2_page) - 1);
            if (page >= 0 && page < a.num_pages) slot = (int64_t)page * a.page_stride + (TO4 ? 0 : place * a.token_stride);
        }
    }
    if ((int32_t)threadIdx.x < half) {
        const int32_t i = threadIdx.x;
        const int32_t axis = r.pair_axes ? min(max(r.pair_axes[i], 0), r.axes - 1) : 0;   // (no read out of range)
        const double turns = (double)r.rope_positions[(int64_t)axis * r.T + t] * (r.inv_freq[i] * 0.15915494309189535);
        float sn, cs;
        sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
        sm_c[i] = cs * r.mscale;
        sm_s[i] = sn * r.mscale;
    }
    __syncthreads();
    for (; j < end;) {
        const bool q = p.what == 0;
        float x[V];
        {
            T raw[V];
            __builtin_memcpy(raw, &p.x, 16);
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = E::get(raw[e]);
        }
        if (p.what != 2) {
            // the norm's factor, and the weights of element i of the head
            float inv = 1.f;
            const bool norm = q ? r.norm_q : r.norm_k;
            if (norm) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) sum += x[e] * x[e];
                sum = lanes_sum<LANES>(sum);
                const float mean = sum / (float)d + r.eps;
                inv = 1.f / __builtin_sqrtf(mean);
                if (!(sum < 0x1p+120f) || mean < 0x1p-60f) {   // squares that fp32 does not hold
                    double s64 = 0.0;
#pragma unroll
                    for (int e = 0; e < V; ++e) s64 += (double)x[e] * (double)x[e];
#pragma unroll
                    for (int i = 1; i < LANES; i *= 2) s64 += __shfl_xor(s64, i);
                    inv = (float)(1.0 / sqrt(s64 / d + (double)r.eps));
                }
            }
            const void* const weights = q ? r.q_weight : r.k_weight;
            const int64_t at = (q ? r.q_weight_heads : r.k_weight_heads) ? (int64_t)p.h * d : 0;
            const bool f32 = r.weight_dtype == PA_DTYPE_F32;
            if (live && norm) weigh<DT>(x, weights, at + first, f32, r.weight_offset, inv);
            if (live && turned) {
                if (INTER) {
#pragma unroll
                    for (int e = 0; e < V; e += 2) {
                        const int32_t i = (first + e) / 2;
                        if (i >= half) break;
                        const float c = sm_c[i], s = sm_s[i], fx = x[e], fy = x[e + 1];
                        x[e] = fx * c - fy * s;
                        x[e + 1] = fx * s + fy * c;
                    }
                } else if (PAIRS == kHalves) {
                    float y[V];
                    T raw[V];
                    __builtin_memcpy(raw, &p.y, 16);
#pragma unroll
                    for (int e = 0; e < V; ++e) y[e] = E::get(raw[e]);
                    if (norm) weigh<DT>(y, weights, at + partner, f32, r.weight_offset, inv);
                    const int32_t i = min(first, partner);
                    const bool lower = first < half;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const float c = sm_c[i + e], s = sm_s[i + e];
                        x[e] = x[e] * c + y[e] * (lower ? -s : s);
                    }
                } else {
                    // (a wave's lanes have all read before one writes: a head lies within it)
                    float y[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int32_t i = first + e;
                        y[e] = 0.f;
                        if (i >= 2 * half) continue;
                        const int32_t k = i < half ? i + half : i - half;
                        y[e] = E::get(p.src[k]);
                        if (norm) y[e] *= inv;
                        if (norm && weights) y[e] *= r.weight_offset + (f32 ? ((const float*)weights)[at + k] : E::get(((const T*)weights)[at + k]));
                    }
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        const int32_t i = first + e;
                        if (i >= 2 * half) continue;
                        const float c = sm_c[i < half ? i : i - half], s = sm_s[i < half ? i : i - half];
                        x[e] = x[e] * c + y[e] * (i < half ? -s : s);
                    }
                }
            }
        }
        const int32_t what = p.what, h = p.h;
        j += HEADS;
        if (j < end) p = load(j);
        if (TO4 && what != 0) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < V; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
            const uint32_t scale = mx4_scale_of(lanes_max<32 / V>(top));
            uint32_t codes = 0;
#pragma unroll
            for (int e = 0; e < V; ++e) codes |= mx4_code(x[e], scale) << 4 * e;
            if (scale == 255) codes = 0;
            if (slot < 0 || !live) continue;
            char* const rec = (char*)a.k_cache + slot + h * a.head_stride;
            const int32_t lp = a.log2_page;
            if (what == 1) {
                char* const dst = rec + mx4_k_codes(lp, d, place) + u * (V / 2);
                if (V == 8) *reinterpret_cast<uint32_t*>(dst) = codes;
                else *reinterpret_cast<uint16_t*>(dst) = (uint16_t)codes;
            } else {
                char* const dst = rec + mx4_v_codes(lp, d, place, first / 4);
                if (V == 4) {
                    *reinterpret_cast<uint16_t*>(dst) = (uint16_t)codes;
                } else if (d == 64) {
                    *reinterpret_cast<uint16_t*>(dst) = (uint16_t)codes;
                    *reinterpret_cast<uint16_t*>(rec + mx4_v_codes(lp, d, place, first / 4 + 1)) = (uint16_t)(codes >> 16);
                } else {
                    *reinterpret_cast<uint32_t*>(dst) = codes;
                }
            }
            if (first % 32 == 0) *reinterpret_cast<uint8_t*>(rec + mx4_scale(lp, d, place, first / 32, what - 1)) = (uint8_t)scale;
            continue;
        }
        T* dst = nullptr;
        if (what == 0) dst = (T*)r.q_out + t * r.q_out_stride + (int64_t)h * d;
        else if (slot >= 0) dst = (T*)(what == 1 ? a.k_cache : a.v_cache) + slot + h * a.head_stride;
        if (dst && live) {
            T raw[V];
#pragma unroll
            for (int e = 0; e < V; ++e) raw[e] = E::put(x[e]);
            uint4 out;
            __builtin_memcpy(&out, raw, 16);
            *reinterpret_cast<uint4*>(dst + first) = out;
        }
    }
}

template <pa_dtype DT, int PAIRS, bool TO4, int LANES>
void launch_lanes(const NormRopeArgs& a, hipStream_t stream)
{
    const int32_t heads = a.q_heads + 2 * a.kv_heads, once = kThreads / LANES;
    const int32_t parts = a.r.T >= 1024 ? 1 : (heads + once - 1) / once;
    hipLaunchKernelGGL((paged_norm_rope_append_kernel<DT, PAIRS, TO4, LANES>), dim3(a.r.T, parts), dim3(kThreads), 0, stream, a);
}

template <pa_dtype DT, int PAIRS, bool TO4>
void launch_pairs(const NormRopeArgs& a, hipStream_t stream)
{
    constexpr int V = DT == PA_DTYPE_F32 ? 4 : 8;
    const int32_t lanes = (a.d + V - 1) / V;
    if (lanes <= 8) launch_lanes<DT, PAIRS, TO4, 8>(a, stream);
    else if (lanes <= 16) launch_lanes<DT, PAIRS, TO4, 16>(a, stream);
    else if (lanes <= 32) launch_lanes<DT, PAIRS, TO4, 32>(a, stream);
    else if constexpr (V == 4) launch_lanes<DT, PAIRS, TO4, 64>(a, stream);
}

template <pa_dtype DT, bool TO4>
void launch_dtype(const NormRopeArgs& a, hipStream_t stream)
{
    constexpr int V = DT == PA_DTYPE_F32 ? 4 : 8;
    if (a.r.interleaved) launch_pairs<DT, kNeighbours, TO4>(a, stream);
    else if (a.half % V == 0) launch_pairs<DT, kHalves, TO4>(a, stream);
    else launch_pairs<DT, kOddHalves, TO4>(a, stream);
}

}  // namespace

pa_status launch_norm_rope_append(const pa_kv_cache_desc* cache, const pa_mx4_cache_desc* to4, pa_dtype dtype, const pa_norm_rope& r,
                                  hipStream_t stream)
{
    NormRopeArgs a;
    a.r = r;
    a.q_heads = r.q ? r.num_q_heads : 0;
    a.half = r.rotary_dim / 2;
    if (to4) {
        const Mx4View v = make_view(to4);
        a.k_cache = a.v_cache = v.records;
        a.page_stride = v.page_stride;
        a.token_stride = 0;
        a.head_stride = v.head_stride;
        a.kv_heads = r.k_new ? v.num_kv_heads : 0;
        a.d = v.head_dim;
        a.log2_page = v.log2_page;
        a.num_pages = v.num_pages;
    } else {
        const CacheView v = make_view(cache);
        a.k_cache = cache->k_cache;
        a.v_cache = cache->v_cache;
        a.page_stride = v.page_stride;
        a.token_stride = v.token_stride;
        a.head_stride = v.head_stride;
        a.kv_heads = r.k_new ? v.num_kv_heads : 0;
        a.d = v.head_dim;
        a.log2_page = v.log2_page;
        a.num_pages = cache->num_pages;
    }
    ProfileScope prof("paged_norm_rope_append_kernel", stream);
    if (dtype == PA_DTYPE_F32) to4 ? launch_dtype<PA_DTYPE_F32, true>(a, stream) : launch_dtype<PA_DTYPE_F32, false>(a, stream);
    else if (dtype == PA_DTYPE_BF16) to4 ? launch_dtype<PA_DTYPE_BF16, true>(a, stream) : launch_dtype<PA_DTYPE_BF16, false>(a, stream);
    else to4 ? launch_dtype<PA_DTYPE_F16, true>(a, stream) : launch_dtype<PA_DTYPE_F16, false>(a, stream);
    return launch_status();
}

}  // namespace pa
