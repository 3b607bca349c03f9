// Norms of the heads of q and K, their rotary positions of one or several numbers, and Algorithm 1's Assign, as one pass, into pages
// of the tokens' own type or of 4-bit elements.
//
//     y = x rsqrt(mean(x^2) + eps) (offset + w),   (y_i, y_j) -> m (y_i cos t - y_j sin t, y_i sin t + y_j cos t)
// with t = p[axis of the pair] f_pair, the angle in 64 bits as turns (rope_append.hip), and so its sine and cosine.  The rest is 32-bit and
// rounded once.  K on its way to 4 bits takes the steps one by one, each rounded to fp32: squares, their sum in fours and then of neighbours, its product
// with 1 / d, eps, an inverse root (a unit in the last place), the products with it and with the weight, those with cosine and sine (64-bit, mscale
// in them, rounded once), their sum.  A last bit of it can decide between two codes, a third of the value apart; so the header names the steps, and
// a program that takes them gets the same codes but where the two roots differ.  It is not nearer to the definition than fused products are.
// (In 64 bits throughout it costs the registers of three waves of seven, 4096 tokens with their gather 31 -> 36 us, these steps 31.5; 64
// bits where a border is near, 39: the last of those heads ends late.)
#include "mx4.h"

namespace pa {

namespace {

constexpr int kThreads = 128;

// Who a pair's elements are: neighbours; halves, a lane's 16 bytes with another lane's; halves of a turned part that does not divide so.
constexpr int kNeighbours = 0, kHalves = 1, kOddHalves = 2;

struct NormRopeArgs {
    pa_norm_rope r;
    void* k_cache;
    void* v_cache;
    int64_t page_stride, token_stride, head_stride;          // elements (a 4-bit cache: page and head, bytes)
    int32_t q_heads, kv_heads;                               // (0 heads: that part is absent)
    int32_t d, half, log2_page, num_pages;
    float by_d;                                              // 1 / d
    double by_d64;
};

template <pa_dtype DT>
struct Elem;
template <>
struct Elem<PA_DTYPE_F32> {
    typedef float T;
    static __device__ __forceinline__ float get(float x) { return x; }
    static __device__ __forceinline__ uint4 pack(const float (&x)[4])
    {
        return uint4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
    }
};
template <>
struct Elem<PA_DTYPE_BF16> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(uint16_t x) { return bf16_bits_to_float(x); }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8])
    {
        return uint4{ElemBf16::pack(x[0], x[1]), ElemBf16::pack(x[2], x[3]), ElemBf16::pack(x[4], x[5]), ElemBf16::pack(x[6], x[7])};
    }
};
template <>
struct Elem<PA_DTYPE_F16> {
    typedef uint16_t T;
    static __device__ __forceinline__ float get(uint16_t x) { return f16_bits_to_float(x); }
    static __device__ __forceinline__ uint4 pack(const float (&x)[8])
    {
        return uint4{ElemF16::pack(x[0], x[1]), ElemF16::pack(x[2], x[3]), ElemF16::pack(x[4], x[5]), ElemF16::pack(x[6], x[7])};
    }
};

// Of q, K and V, by values: a choice between variables that a lambda has by reference would put them into memory.
template <typename X>
__device__ __forceinline__ X pick(int32_t what, X q, X k, X v)
{
    return what == 0 ? q : what == 1 ? k : v;
}

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
__device__ __forceinline__ double lanes_sum(double v)
{
    auto step = [&](auto move) {
        const uint64_t b = (uint64_t)__double_as_longlong(v);
        v += __longlong_as_double((long long)((uint64_t)move((uint32_t)(b >> 32)) << 32 | move((uint32_t)b)));
    };
    if (LANES > 1) step([](uint32_t x) { return other<1>(x); });
    if (LANES > 2) step([](uint32_t x) { return other<2>(x); });
    if (LANES > 4) step([](uint32_t x) { return other<4>(x); });
    if (LANES > 8) step([](uint32_t x) { return other<8>(x); });
    if (LANES > 16) step([](uint32_t x) { return other<16>(x); });
    if (LANES > 32) step([](uint32_t x) { return other<32>(x); });
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

// 1 / sqrt(x) in 64 bits: the hardware's 32-bit root and a step of Newton's method, or what the library does where 32 bits do not hold x.
__device__ __forceinline__ double root_of_inverse(double x)
{
    if (!(x > 0x1p-100 && x < 0x1p+100)) return 1.0 / sqrt(x);
    double r = (double)__builtin_amdgcn_rsqf((float)x);      // (to 2^-22: after the step to 2^-43, after another to the last bits)
    r = r * fma(-0.5 * x * r, r, 1.5);
    return r * fma(-0.5 * x * r, r, 1.5);
}

// Products and sums that are rounded each by itself.
__device__ __forceinline__ float times(float x, float y)
{
#pragma clang fp contract(off)
    return x * y;
}
__device__ __forceinline__ float plus(float x, float y)
{
#pragma clang fp contract(off)
    return x + y;
}

// Sine and cosine of so many turns, in 64 bits: an eighth of a turn at most is left to the Taylor series, whose next terms are below 2^-45 (sine) and
// 2^-41 (cosine); both are then rounded to 2^-25.
__device__ __forceinline__ void sine_cosine(double turns, double& sn, double& cs)
{
    turns -= rint(turns);
    const double quarter = rint(4.0 * turns);
    const double x = 6.283185307179586 * (turns - 0.25 * quarter), z = x * x;
    double s = 1.0 / 6227020800.0, c = 1.0 / 479001600.0;    // 1 / 13!, 1 / 12!
    s = fma(s, z, -1.0 / 39916800.0);
    c = fma(c, z, -1.0 / 3628800.0);
    s = fma(s, z, 1.0 / 362880.0);
    c = fma(c, z, 1.0 / 40320.0);
    s = fma(s, z, -1.0 / 5040.0);
    c = fma(c, z, -1.0 / 720.0);
    s = fma(s, z, 1.0 / 120.0);
    c = fma(c, z, 1.0 / 24.0);
    s = fma(s, z, -1.0 / 6.0);
    c = fma(c, z, -0.5);
    s = fma(s * z, x, x);
    c = fma(c, z, 1.0);
    const int q = (int)quarter;
    sn = q == 0 ? s : q == 1 ? c : q == -1 ? -c : -s;
    cs = q == 0 ? c : q == 1 ? -s : q == -1 ? s : -c;
}

// A head is LANES lanes of a wave (a power of two), 16 bytes each; a workgroup has 128 / LANES heads of one token at a time.  Of an element x
// with partner y the lane keeps a = m cos t (offset + w) and b = -+ m sin t (offset + w of the partner), the same for all heads where they
// share weights: a head costs it the sum of squares and x inv a + y inv b.  Bound by reading and writing q, K and V once: 8192 tokens of 32 / 8
// heads of 128, 201 MB, 36 us on the same data again (5.6 TB/s), 42.8 on data from memory (4.7, as a copy of 4 GiB).  A token's first wait is for
// its angles; two waves a workgroup lose least there (64 / 128 / 256 / 512 threads: 38.0 / 34.4 / 35.9 / 51.8, before sine and cosine were
// 64-bit, 0.9 more).  Two pieces in flight instead of one cost registers and gain nothing (35.9 / 38.0).
template <pa_dtype DT, int PAIRS, bool TO4, int LANES>
__global__ __launch_bounds__(kThreads, TO4 && PAIRS != kOddHalves ? 6 : 1) void paged_norm_rope_append_kernel(NormRopeArgs a)
{
    typedef Elem<DT> E;
    typedef typename E::T T;
    constexpr int V = 16 / sizeof(T), HEADS = kThreads / LANES;
    // cosines and sines of the pairs (head_dim is at most 256), behind them 1 and 0
    __shared__ __attribute__((aligned(16))) float sm_c[136], sm_s[136];
    const pa_norm_rope& r = a.r;
    const float by_d = a.by_d;
    const int32_t d = a.d, half = a.half, u = threadIdx.x % LANES, first = u * V;
    // Workgroup i runs on chiplet i % 8: 16 tokens in a row on one, since up to 8 tokens share cache lines of a record (us without / with, 6000
    // tokens into 4 bits and out again 23.7 / 20.7, 16000 47.5 / 38.2).
    int64_t t = blockIdx.x;
    if (TO4 && (t | 127) < (int64_t)gridDim.x) t = (t & ~127) | (t & 7) << 4 | (t >> 3 & 15);
    const bool live = first < d;
    const int32_t heads = a.q_heads + 2 * a.kv_heads;
    const int32_t mine = (heads + (int32_t)gridDim.y - 1) / (int32_t)gridDim.y;
    const int32_t begin = mine * (int32_t)blockIdx.y, end = min(begin + mine, heads);
    constexpr bool INTER = PAIRS == kNeighbours;
    const bool turned = first < 2 * half;
    const int32_t partner = PAIRS != kHalves || !turned ? first : first < half ? first + half : first - half;

    const char* const q_weight = (const char*)(r.norm_q ? r.q_weight : nullptr);
    const char* const k_weight = (const char*)(r.norm_k ? r.k_weight : nullptr);
    const bool f32 = r.weight_dtype == PA_DTYPE_F32;
    const T* const q_row = (const T*)r.q + t * r.q_stride;
    const T* const k_row = (const T*)r.k_new + t * r.k_stride;
    const T* const v_row = (const T*)r.v_new + t * r.v_stride;
    struct Piece {
        const T* src;            // of the head
        int32_t what, h;         // 0: q, 1: K, 2: V
        uint4 x;
    };
    auto load = [&](int32_t j) {
        Piece p;
        p.what = j < a.q_heads ? 0 : j < a.q_heads + a.kv_heads ? 1 : 2;
        p.h = j - pick(p.what, 0, a.q_heads, a.q_heads + a.kv_heads);
        p.src = pick(p.what, q_row, k_row, v_row) + (uint32_t)(p.h * d);
        p.x = *reinterpret_cast<const uint4*>(p.src + (live ? first : 0));
        if (!live) p.x = uint4{0, 0, 0, 0};
        return p;
    };
    // w of the lane's elements
    auto weights_at = [&](float (&w)[V], const char* weights, int32_t at) {
        const int32_t i = at + (live ? first : 0);
        if (DT == PA_DTYPE_F32 || f32) {
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const float4 x = *reinterpret_cast<const float4*>((const float*)weights + i + e);
                w[e] = x.x, w[e + 1] = x.y, w[e + 2] = x.z, w[e + 3] = x.w;
            }
        } else {
            T raw[V];
            const uint4 x = *reinterpret_cast<const uint4*>((const T*)weights + i);
            __builtin_memcpy(raw, &x, 16);
#pragma unroll
            for (int e = 0; e < V; ++e) w[e] = E::get(raw[e]);
        }
    };
    const int from = ((int)threadIdx.x & 63) - u + partner / V;   // the partner's lane
    // weights of the lane's elements and of their partners, offset not yet added (1 in all without weights)
    auto both_weights = [&](float (&w)[V], float (&other)[V], const char* weights, int32_t at_head) {
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = 1.f;
        if (weights) weights_at(w, weights, at_head);
#pragma unroll
        for (int e = 0; e < V; ++e) {
            const int32_t i = first + e;
            other[e] = INTER ? w[e ^ 1] : PAIRS == kHalves ? __shfl(w[e], from) : 1.f;
            if (PAIRS == kOddHalves && weights && i < 2 * half) {
                const int32_t k = at_head + (i < half ? i + half : i - half);
                other[e] = f32 ? ((const float*)weights)[k] : E::get(((const T*)weights)[k]);
            }
        }
    };
    // the partners of a piece's elements; 0 where nothing turns
    auto partners = [&](float (&y)[V], const float (&x)[V], const Piece& p) {
        if (INTER) {
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = first + e < 2 * half ? x[e ^ 1] : 0.f;
        } else if (PAIRS == kHalves) {
            T raw[V];
            const uint4 v = uint4{(uint32_t)__shfl((int)p.x.x, from), (uint32_t)__shfl((int)p.x.y, from),
                                  (uint32_t)__shfl((int)p.x.z, from), (uint32_t)__shfl((int)p.x.w, from)};
            __builtin_memcpy(raw, &v, 16);
#pragma unroll
            for (int e = 0; e < V; ++e) y[e] = turned ? E::get(raw[e]) : 0.f;
        } else {
            // (a wave's lanes have all read before one writes: a head lies within it)
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const int32_t i = first + e;
                y[e] = i < 2 * half ? E::get(p.src[i < half ? i + half : i - half]) : 0.f;
            }
        }
    };
    // where element e's cosine and sine stand, and whether it is a pair's first
    const int32_t at_halves = turned ? min(first, partner) : 128, at_pairs = live ? first / 2 : 128;
    auto pair_of = [&](int e) {
        const int32_t i = first + e;
        return INTER ? at_pairs + e / 2 : PAIRS == kHalves ? at_halves + e : i < half ? i : i < 2 * half ? i - half : 128;
    };
    auto is_first = [&](int e) { return INTER ? e % 2 == 0 : first + e < half; };
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
    for (int32_t i = half + (int32_t)threadIdx.x; i < 136; i += kThreads) {
        sm_c[i] = 1.f;
        sm_s[i] = 0.f;
    }
    for (int32_t i = threadIdx.x; i < half; i += kThreads) {
        const int32_t axis = r.pair_axes ? min(max(r.pair_axes[i], 0), r.axes - 1) : 0;   // (no read out of range)
        const double turns = (double)r.rope_positions[(int64_t)axis * r.T + t] * (r.inv_freq[i] * 0.15915494309189535);
        double sn, cs;
        sine_cosine(turns, sn, cs);
        sm_c[i] = (float)(cs * r.mscale);
        sm_s[i] = (float)(sn * r.mscale);
    }
    __syncthreads();
    float fa[V], fb[V];          // a and b; on the way to 4 bits the weights alone
    int32_t have = -1;           // whose factors these are: q (0), K (1), no one's (-1)
    for (; j < end;) {
        const int32_t what = p.what, h = p.h;
        const bool norm = what != 2 && pick(what, r.norm_q, r.norm_k, 0);
        float x[V];
        {
            T raw[V];
            __builtin_memcpy(raw, &p.x, 16);
#pragma unroll
            for (int e = 0; e < V; ++e) x[e] = E::get(raw[e]);
        }
        if (what != 2 && (norm || half > 0)) {
            const char* const weights = pick(what, q_weight, k_weight, q_weight);
            const bool each = weights && pick(what, r.q_weight_heads, r.k_weight_heads, 0);
            const int32_t at_head = each ? h * d : 0;
            float y[V];
            partners(y, x, p);
            auto in_64 = [&] {                               // of squares that fp32 does not hold
                double sum = 0.0;
#pragma unroll
                for (int e = 0; e < V; ++e) sum = fma((double)x[e], (double)x[e], sum);
                const double root = root_of_inverse(lanes_sum<LANES>(sum) * a.by_d64 + (double)r.eps);
                if (!(root > 0x1p+100)) return (float)root;
                // (subnormal heads: the inverse of a root below 2^-128 is none of fp32's numbers; 2^64 of it goes into the factors)
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    fa[e] *= 0x1p+64f;
                    fb[e] *= 0x1p+64f;
                }
                have = -1;
                return (float)(root * 0x1p-64);
            };
            if (have != what || each) {
                both_weights(fa, fb, weights, at_head);
                const float offset = weights ? r.weight_offset : 0.f;
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    fa[e] += offset;
                    fb[e] += offset;
                    if (TO4) continue;
                    const int32_t at = pair_of(e);
                    const float sn = sm_s[at] * fb[e];
                    fa[e] *= sm_c[at];
                    fb[e] = first + e >= 2 * half ? -0.f : is_first(e) ? -sn : sn;   // (with y = 0: a zero keeps its sign)
                }
                have = what;
            }
            float inv = 1.f;
            if (norm) {
                float four[V / 4];
#pragma unroll
                for (int e = 0; e < V; ++e)
                    four[e / 4] = e % 4 == 0 ? times(x[e], x[e]) : TO4 ? plus(four[e / 4], times(x[e], x[e])) : __builtin_fmaf(x[e], x[e], four[e / 4]);
                float sum = four[0];
                if (V == 8) sum = plus(four[0], four[V / 4 - 1]);
                sum = lanes_sum<LANES>(sum);
                const float mean = plus(times(sum, by_d), r.eps);
                inv = __builtin_amdgcn_rsqf(mean);           // (a unit in the last place)
                if (!(sum < 0x1p+120f) || mean < 0x1p-60f) inv = in_64();
            }
            if constexpr (TO4) {
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    const int32_t at = pair_of(e);
                    const float z = times(times(x[e], inv), fa[e]), zc = times(z, sm_c[at]), zs = times(times(times(y[e], inv), fb[e]), sm_s[at]);
                    x[e] = first + e >= 2 * half ? z : plus(zc, is_first(e) ? -zs : zs);
                }
            } else {
#pragma unroll
                for (int e = 0; e < V; ++e) x[e] = __builtin_fmaf(y[e] * inv, fb[e], x[e] * inv * fa[e]);
            }
        }
        uint4 out = p.x;         // (V as it is)
        j += HEADS;
        if (j < end) p = load(j);
        if (TO4 && what != 0) {
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < V; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
            const uint32_t scale = mx4_scale_of(lanes_max<32 / V>(top));
            const uint32_t codes = scale == 255 ? 0u : mx4_codes(x, scale);
            if (slot < 0 || !live) continue;
            char* const rec = (char*)a.k_cache + slot + h * a.head_stride;
            const int32_t lp = a.log2_page;
            if (what == 1) {
                char* const dst = rec + mx4_k_codes(d, place) + u * (V / 2);
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
        else if (slot >= 0) dst = pick(what, (T*)a.k_cache, (T*)a.k_cache, (T*)a.v_cache) + slot + h * a.head_stride;
        if (dst && live) {
            if (what != 2) out = E::pack(x);
            store_past_cache(dst + first, out);
        }
    }
}

template <pa_dtype DT, int PAIRS, bool TO4, int LANES>
void launch_lanes(const NormRopeArgs& a, hipStream_t stream)
{
    const int32_t heads = a.q_heads + 2 * a.kv_heads, once = kThreads / LANES;
    // Few tokens are spread over several workgroups each (us with 2048 / 4096 in the place of 4096: 8 tokens of 32 / 8 heads of 128 4.0 / 4.0, 240
    // 4.6 / 4.8, 600 6.2 / 6.4; 900 of 32 / 32 heads of 80 9.8 / 9.0).
    const int32_t parts = min((heads + once - 1) / once, max(1, 4096 / a.r.T));
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
    a.by_d = 1.f / (float)a.d;
    a.by_d64 = 1.0 / a.d;
    ProfileScope prof("paged_norm_rope_append_kernel", stream);
    if (dtype == PA_DTYPE_F32) to4 ? launch_dtype<PA_DTYPE_F32, true>(a, stream) : launch_dtype<PA_DTYPE_F32, false>(a, stream);
    else if (dtype == PA_DTYPE_BF16) to4 ? launch_dtype<PA_DTYPE_BF16, true>(a, stream) : launch_dtype<PA_DTYPE_BF16, false>(a, stream);
    else to4 ? launch_dtype<PA_DTYPE_F16, true>(a, stream) : launch_dtype<PA_DTYPE_F16, false>(a, stream);
    return launch_status();
}

}  // namespace pa
