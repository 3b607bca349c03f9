// Attention of a sequence's last tokens over a cache of 4-bit elements, on the matrix cores.  Internal header: the kernel templates.
//
// The n new queries and the G query heads of a KV head are n G rows.  Both products are transposed (v_mfma_f32_16x16x32_bf16,
// lane % 16 = row), so softmax statistics are a lane's own:
//     S^T[key, row] = K Q^T,   O^T[column, row] += V^T P^T.
//   * A wave walks keys 32 at a time and takes what it needs of a record straight into registers: a lane's K codes are a
//     quarter of a key's, its V codes 8 keys by head_dim / 16 elements, which the record holds in one piece; 16 KB of 16-bit K
//     and V (head_dim 128) are 4.25 KB in six loads.  No LDS is involved until the end, but where waves share operands (SHARED).
//   * Codes become bf16, exactly, by the hardware's conversion under a block's scale, two elements at a time.  For K those are the operand as
//     it stands; a lane's V pairs are elements of one key and are exchanged with the next key's by two byte permutes.
//   * Queries enter with all their bits: bf16 as they are, fp16 as two bf16 terms (since K is made bf16, whatever its scales), fp32 as three.
//     Weights enter as two terms (2^-17 of a weight, below the half step of a 16-bit output; about one bf16 output in 500 is the neighbour of
//     what fp32 weights give), with fp32 queries as three.  A third term for all costs, us: 4 prompts of 2047 234 -> 269, 1000 tokens
//     behind 31000 689 -> 826, one token on 16 x 8000..9000 36.2 -> 42.8.
//   * Softmax is online in the log2 domain against a reference that trails the maximum; only where a lane's weights sum to more
//     than they may is it raised and O rescaled.
//   * Keys are masked by selection.  A V block of NaN that some rows of a tile do not see would reach them through a product with
//     a weight of zero, and sums of finite values may leave the range of fp32 where their mean does not; both leave their mark on an
//     accumulator, and such a piece of work is done again (CAREFUL): with weights of at most 2^-24 (tree_share.h), and NaN added to the rows
//     that see it only.
//   * Work is shared, and what is cut merged, as for drafted trees (tree_share.h).
#pragma once

#include "mx4.h"
#include "tree_share.h"

namespace pa {

namespace {

// RT tiles of 16 rows a wave; RW waves beside each other in rows, KW along the keys; OCC workgroups on a compute unit; keys in flight: DEEP
// steps of 32.  SHARED: four waves of rows, of which each makes operands of a quarter of a tile's codes, in LDS, for all of them.
template <pa_dtype DT, int D, int RT, int RW, int KW, int OCC, int DEEP, bool SHARED = false>
struct Mx4Shape {
    static constexpr int kRows = 16 * RT * RW, kWaveRows = 16, kColumns = D;
    static constexpr int kWaves = RW * KW, kOcc = OCC, kTile = KW == 1 ? 64 : 32 * KW, kLeastTiles = 1;
    static constexpr bool kCut = true;
    static constexpr int kQT = DT == PA_DTYPE_BF16 ? 1 : DT == PA_DTYPE_F16 ? 2 : 3;   // terms of a query
    static constexpr int kPT = DT == PA_DTYPE_F32 ? 3 : 2;                             // terms of a weight
    static constexpr int kLanes = D / 64;                    // float4s of a lane and row quarter
    static constexpr int kJoin = KW > 1 ? RW * KW * RT * D * 16 * 4 : 0;               // bytes in which the waves' results meet
    static constexpr int kTileB = 2 * 64 * D * 2;            // bytes of a tile's operands
    static constexpr int kLds = SHARED ? 2 * kTileB : kJoin + kWaves * RT * 16 * 8 + 1024;
    static_assert(KW == 1 || KW == 2 || KW == 4 || KW == 8, "their join knows log2 of it");
    static_assert(!SHARED || (KW == 1 && RW == 4 && D <= 128), "a quarter is 16 keys of K, 32 keys and half of the columns of V");
    static constexpr int kSteps = D / 32, kTiles = D / 16;
    static constexpr int kKDwords = D / 32, kVDwords = D / 16;                         // of a lane: per key, and for its 8 keys
    static constexpr int kKScales = D > 128 ? 2 : 1;

    // What a lane takes of 32 keys.  K rows r = lane % 16 of the two products are keys 8 (r / 4) + r % 4 and four further, so that
    // its S^T rows are the keys of its V codes.
    struct Keys {
        uint32_t k[2][kKDwords], v[kVDwords];
        uint2 ks[kKScales], vs;
    };

    // Codes are read once where no other wave has rows beside: past the caches (us from memory without / so: 16 x 131072 tokens 398 / 365, 6.25 TB/s, as a
    // plain read; 64 on 64 to 32768 81 / 76, 16 x 8000..9000 38.9 / 35.1, head_dim 64 27.9 / 25.9; 256 x 1000 that share 512, which the last-level cache still holds, 39.5 / 42.2.
    // At head_dim 256, where a lane's two pieces of a line come by two loads, 66.6 / 84.6).
    typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
    typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
    template <typename T, typename V>
    static __device__ __forceinline__ T read(const char* p)
    {
        if (RW == 1 && D <= 128) return __builtin_bit_cast(T, __builtin_nontemporal_load(reinterpret_cast<const V*>(p)));
        return *reinterpret_cast<const T*>(p);
    }

    static __device__ __forceinline__ uint32_t scale_bits(uint2 s, int i)   // scale of key i of 8, as a float's bits
    {
        const uint32_t w = i < 4 ? s.x : s.y;
        switch (i & 3) {
            case 0: return (w << 23) & 0x7f800000u;
            case 1: return (w << 15) & 0x7f800000u;
            case 2: return (w << 7) & 0x7f800000u;
        }
        return (w >> 1) & 0x7f800000u;
    }
    template <int B>
    static __device__ __forceinline__ uint32_t bf16_pair(uint32_t codes, float unit)   // elements 2 B, 2 B + 1 of 8
    {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, unit, B));
    }
    static __device__ __forceinline__ uint4 bf16_eight(uint32_t codes, float unit)
    {
        return uint4{bf16_pair<0>(codes, unit), bf16_pair<1>(codes, unit), bf16_pair<2>(codes, unit), bf16_pair<3>(codes, unit)};
    }
    // A lane's V codes are d / 32 bytes of each of its 8 keys, in their order.
    template <int B>
    static __device__ __forceinline__ uint32_t v_pair(const uint32_t (&v)[kVDwords], int key, float unit)   // elements 2 B, 2 B + 1
    {
        if constexpr (D == 64) return key & 1 ? bf16_pair<2 + B>(v[key / 2], unit) : bf16_pair<B>(v[key / 2], unit);
        else return bf16_pair<B % 4>(v[key * (D / 128) + B / 4], unit);
    }

    static __device__ __forceinline__ void store(void* out, int64_t at, float4 x)
    {
        if (DT == PA_DTYPE_F32) {
            *reinterpret_cast<float4*>((float*)out + at) = x;
        } else {
            typedef typename std::conditional<DT == PA_DTYPE_F16, ElemF16, ElemBf16>::type E;
            *reinterpret_cast<uint2*>((uint16_t*)out + at) = uint2{E::pack(x.x, x.y), E::pack(x.z, x.w)};
        }
    }

    // Eight elements of a query as kQT bf16 operands.
    static __device__ __forceinline__ void query(uint4 (&q)[kQT], const void* src, int64_t at, uint32_t flip, bool zero)
    {
        float x[8];
        if (DT == PA_DTYPE_BF16) {
            uint4 r = *reinterpret_cast<const uint4*>((const uint16_t*)src + at);
            const uint32_t f = flip | flip >> 16;
            r = uint4{r.x ^ f, r.y ^ f, r.z ^ f, r.w ^ f};
            q[0] = zero ? uint4{0, 0, 0, 0} : r;
            return;
        }
        if (DT == PA_DTYPE_F16) {
            const uint4 r = *reinterpret_cast<const uint4*>((const uint16_t*)src + at);
            x[0] = ElemF16::lo_of(r.x), x[1] = ElemF16::hi_of(r.x), x[2] = ElemF16::lo_of(r.y), x[3] = ElemF16::hi_of(r.y);
            x[4] = ElemF16::lo_of(r.z), x[5] = ElemF16::hi_of(r.z), x[6] = ElemF16::lo_of(r.w), x[7] = ElemF16::hi_of(r.w);
        } else {
            const float4 r = *reinterpret_cast<const float4*>((const float*)src + at), s = *reinterpret_cast<const float4*>((const float*)src + at + 4);
            x[0] = r.x, x[1] = r.y, x[2] = r.z, x[3] = r.w, x[4] = s.x, x[5] = s.y, x[6] = s.z, x[7] = s.w;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = zero ? 0.f : __uint_as_float(__float_as_uint(x[e]) ^ flip);
#pragma unroll
        for (int t = 0; t < kQT; ++t) {
            const uint4 w = uint4{ElemBf16::pack(x[0], x[1]), ElemBf16::pack(x[2], x[3]), ElemBf16::pack(x[4], x[5]), ElemBf16::pack(x[6], x[7])};
            q[t] = w;
            x[0] -= ElemBf16::lo_of(w.x), x[1] -= ElemBf16::hi_of(w.x), x[2] -= ElemBf16::lo_of(w.y), x[3] -= ElemBf16::hi_of(w.y);
            x[4] -= ElemBf16::lo_of(w.z), x[5] -= ElemBf16::hi_of(w.z), x[6] -= ElemBf16::lo_of(w.w), x[7] -= ElemBf16::hi_of(w.w);
        }
    }

    // Weights of 32 keys from their raw scores (-inf: not seen), as operands; sc > 0.
    template <bool CAREFUL>
    static __device__ __forceinline__ void weights(uint4 (&w)[RT][kPT], const mfma_f32x4 (&s)[RT][2], mfma_f32x4 (&o)[RT][kTiles], float (&m)[RT],
                                                   float (&l)[RT], float sc)
    {
        constexpr float kBelow = CAREFUL ? kCarefulBelow : 0.f, kSumMax = CAREFUL ? 0.5f * kCarefulSumMax : kWeightSumMax;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            float p[8], psum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][i / 4][i % 4], sc, -m[rt]));
                psum += p[i];
            }
            if (__any(!(psum <= kSumMax))) {         // also the NaN or infinity of a fresh reference
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, s[rt][i / 4][i % 4]);
                const float m_new = fmaxf(m[rt], row_max<4>(top) * sc - kBelow);
                const float use = m_new == -INFINITY ? 0.f : m_new;   // (no key so far)
                const float alpha = __builtin_amdgcn_exp2f(m[rt] - use);
#pragma unroll
                for (int j = 0; j < kTiles; ++j) o[rt][j] *= alpha;
                l[rt] *= alpha;
                m[rt] = m_new;
                psum = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][i / 4][i % 4], sc, -use));
                    psum += p[i];
                }
            }
            l[rt] += psum;
#pragma unroll
            for (int u = 0; u < kPT; ++u) {
                w[rt][u] = uint4{ElemBf16::pack(p[0], p[1]), ElemBf16::pack(p[2], p[3]), ElemBf16::pack(p[4], p[5]),
                                 ElemBf16::pack(p[6], p[7])};
                if (u + 1 < kPT) {
                    p[0] -= ElemBf16::lo_of(w[rt][u].x), p[1] -= ElemBf16::hi_of(w[rt][u].x);
                    p[2] -= ElemBf16::lo_of(w[rt][u].y), p[3] -= ElemBf16::hi_of(w[rt][u].y);
                    p[4] -= ElemBf16::lo_of(w[rt][u].z), p[5] -= ElemBf16::hi_of(w[rt][u].z);
                    p[6] -= ElemBf16::lo_of(w[rt][u].w), p[7] -= ElemBf16::hi_of(w[rt][u].w);
                }
            }
        }
    }

    template <bool CAREFUL>
    static __device__ __forceinline__ bool work(char* buf, uint32_t* flags, const TreeKernelArgs& a, const TreeItem& item, int32_t kvh)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        const int kw = wave % KW, rw = wave / KW, row16 = lane & 15, g = lane >> 4;
        const int32_t n_rows = item.n * a.group, lp = a.cache.log2_page, P = 1 << lp;
        // where a workgroup has a whole row block, those that see most come first
        const int32_t rb = a.wgs == 0 ? (n_rows + kRows - 1) / kRows - 1 - item.rb : item.rb;
        const int32_t r0 = rb * kRows + 16 * RT * rw;
        const float scale = a.scale;
        const float sc = scale == 0.f ? 1.f : fabsf(scale) * 1.4426950408889634f;
        // queries, the rows' places in the output, and how many keys each sees
        uint4 q[RT][kQT][kSteps];
        int32_t sees[RT];
        int64_t out_row[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const int32_t r = r0 + 16 * rt + row16;
            const bool live = r < n_rows;
            const int32_t qi = live ? r / a.group : 0, h = live ? r - qi * a.group : 0;
            out_row[rt] = live ? (int64_t)(item.row0 + qi) * a.num_q_heads + kvh * a.group + h : -1;
            sees[rt] = live ? min(max(item.len - item.n + qi + 1, 0), item.len) : 0;
            uint4 one[kQT];
#pragma unroll
            for (int t = 0; t < kSteps; ++t) {
                if (live) {
                    query(one, a.q, out_row[rt] * D + g * (D / 4) + 8 * t, scale < 0.f ? 0x80000000u : 0u, scale == 0.f);
                } else {
#pragma unroll
                    for (int i = 0; i < kQT; ++i) one[i] = uint4{0, 0, 0, 0};
                }
#pragma unroll
                for (int i = 0; i < kQT; ++i) q[rt][i][t] = one[i];
            }
        }
        // steps of 32 keys: this wave's are kw, kw + KW, .. of the piece's; none that no row of the wave sees
        const int32_t last_row = min(r0 + 16 * RT, n_rows) - 1;
        const int32_t most = r0 < n_rows ? min(max(item.len - item.n + last_row / a.group + 1, 0), item.len) : 0;
        const int32_t least = r0 < n_rows ? max(item.len - item.n + r0 / a.group + 1, 0) : 0;   // (the first row's; masks from there on)
        const int32_t step0 = item.tile_begin * (kTile / 32) + kw;
        const int32_t steps_end = min(item.tile_end * (kTile / 32), (most + 31) / 32);
        const int32_t steps = steps_end > step0 ? (steps_end - step0 + KW - 1) / KW : 0;

        mfma_f32x4 o[RT][kTiles];
        float m[RT], l[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            m[rt] = -INFINITY;
            l[rt] = 0.f;
#pragma unroll
            for (int j = 0; j < kTiles; ++j) o[rt][j] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
        }
        if constexpr (SHARED && !CAREFUL) {
            // (all waves walk to the end of the workgroup's rows)
            const int32_t far_row = min(rb * kRows + kRows, n_rows) - 1;
            const int32_t wg_most = min(max(item.len - item.n + far_row / a.group + 1, 0), item.len);
            const int32_t tile_end = min(item.tile_end, (wg_most + 63) / 64), tiles = tile_end - item.tile_begin;
            if (tiles > 0) shared(buf, a, item, kvh, tiles, most, least, sees, q, o, m, l, sc);
        } else if (steps > 0) {
            const int32_t* const table = a.block_table + (int64_t)item.s * a.max_blocks;
            const char* const base = (const char*)a.cache.k + (int64_t)kvh * a.cache.head_stride;
            const int32_t last_block = (item.len - 1) >> lp;
            // a lane's offsets within a record (pages of 16 tokens: 32 keys are two pages, octets 0, 1 and 2, 3)
            const int ko = row16 >> 2, vo = g;
            const int32_t kslot = (8 * ko) & (P - 1), vslot = (8 * vo) & (P - 1);
            const int32_t k_at = (kslot + (row16 & 3)) * (D / 2) + g * (D / 8);
            const int32_t v_at = ((D / 2) << lp) + vslot * (D / 2) + row16 * (D / 4);
            const int32_t ks_at = ((D + g * (D / 4) / 32) << lp) + kslot;
            const int32_t vs_at = ((D + D / 32 + row16 * (D / 16) / 32) << lp) + vslot;
            // pages of 32 steps at a time, lane 2 n + h those of keys 16 h .. of the wave's n-th step, and of the next 32
            auto pages_of = [&](int32_t n) {
                const int32_t key = 32 * (step0 + KW * min(n + (lane >> 1), steps - 1)) + 16 * (lane & 1);
                return table[min(key >> lp, last_block)];
            };
            int32_t pages = pages_of(0), more = pages_of(32);
            auto load = [&](Keys& x, int32_t n) {
                if (n > 0 && (n & 31) == 0) {
                    pages = more;
                    more = pages_of(n + 32);
                }
                const int32_t key0 = 32 * (step0 + KW * n);
                const char* const first = base + (int64_t)__builtin_amdgcn_readlane(pages, 2 * (n & 31)) * a.cache.page_stride;
                const char* const second = base + (int64_t)__builtin_amdgcn_readlane(pages, 2 * (n & 31) + 1) * a.cache.page_stride;
                const int32_t slot = key0 & (P - 1);
                const char* const kp = (ko >= 2 ? second : first) + slot * (D / 2) + k_at;
                const char* const vp = (vo >= 2 ? second : first) + slot * (D / 2) + v_at;
                const char* const ksp = (ko >= 2 ? second : first) + slot + ks_at;
                const char* const vsp = (vo >= 2 ? second : first) + slot + vs_at;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if constexpr (D == 64) {
                        const uint2 w = read<uint2, u32x2>(kp + i * (4 * D / 2));
                        x.k[i][0] = w.x, x.k[i][1] = w.y;
                    } else {
#pragma unroll
                        for (int j = 0; j < kKDwords; j += 4) {
                            const uint4 w = read<uint4, u32x4>(kp + i * (4 * D / 2) + 4 * j);
                            x.k[i][j] = w.x, x.k[i][j + 1] = w.y, x.k[i][j + 2] = w.z, x.k[i][j + 3] = w.w;
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < kKScales; ++j) x.ks[j] = *reinterpret_cast<const uint2*>(ksp + (j << lp));
#pragma unroll
                for (int j = 0; j < kVDwords; j += 4) {
                    const uint4 w = read<uint4, u32x4>(vp + 4 * j);
                    x.v[j] = w.x, x.v[j + 1] = w.y, x.v[j + 2] = w.z, x.v[j + 3] = w.w;
                }
                x.vs = *reinterpret_cast<const uint2*>(vsp);
            };
            auto compute = [&](Keys& x, int32_t step) {
                const int32_t key0 = 32 * step;
                mfma_f32x4 s[RT][2];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) s[rt][i] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
                float unit[2][kKScales];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < kKScales; ++j)
                        unit[i][j] = __uint_as_float((((i ? x.ks[j].y : x.ks[j].x) >> (8 * (row16 & 3))) & 0xffu) << 23);
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    const uint4 k0 = bf16_eight(x.k[0][t], unit[0][kKScales == 2 ? t / 4 : 0]);
                    const uint4 k1 = bf16_eight(x.k[1][t], unit[1][kKScales == 2 ? t / 4 : 0]);
#pragma unroll
                    for (int u = 0; u < kQT; ++u)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            s[rt][0] = ElemBf16::mfma16(k0, q[rt][kQT - 1 - u][t], s[rt][0]);
                            s[rt][1] = ElemBf16::mfma16(k1, q[rt][kQT - 1 - u][t], s[rt][1]);
                        }
                }
                const bool masked = key0 + 32 > least;       // (the same for the whole wave)
                if (masked) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (key0 + 8 * g + i >= sees[rt]) s[rt][i / 4][i % 4] = -INFINITY;
                    // slots behind the sequence may hold anything, NaN among it
                    const int32_t left = item.len - key0 - 8 * g;
                    if (left < 8) {
                        const uint64_t keep = left <= 0 ? 0 : ~0ull >> (64 - 8 * left);
                        x.vs.x &= (uint32_t)keep;
                        x.vs.y &= (uint32_t)(keep >> 32);
                    }
                }
                uint4 w[RT][kPT];
                weights<CAREFUL>(w, s, o, m, l, sc);
                if (CAREFUL) {
                    // blocks of NaN count for 0 in the product; rows that see one get NaN in its columns by a product of ones
                    uint4 ones = uint4{0, 0, 0, 0};
                    uint32_t* const one = reinterpret_cast<uint32_t*>(&ones);
                    bool any = false;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint32_t& word = i < 4 ? x.vs.x : x.vs.y;
                        if ((word >> (8 * (i & 3)) & 0xffu) == 255u) {
                            any = true;
                            one[i / 2] |= 0x3f80u << (16 * (i & 1));
                            word &= ~(0xffu << (8 * (i & 3)));
                        }
                    }
                    if (__any(any)) {
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            uint4 see = uint4{0, 0, 0, 0};
                            uint32_t* const bit = reinterpret_cast<uint32_t*>(&see);
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (key0 + 8 * g + i < sees[rt]) bit[i / 2] |= 0x3f80u << (16 * (i & 1));
                            const mfma_f32x4 hit = ElemBf16::mfma16(ones, see, mfma_f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                            for (int j = 0; j < kTiles; ++j)
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    if (hit[i] > 0.f) o[rt][j][i] = NAN;
                        }
                    }
                }
                // O^T += V^T P^T, two columns of a lane at a time
                float vu[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) vu[i] = __uint_as_float(scale_bits(x.vs, i));
                columns<0>(x, vu, w, o);
            };
            Keys ring[DEEP];
#pragma unroll
            for (int i = 0; i < DEEP; ++i) load(ring[i], min(i, steps - 1));
            int32_t n = 0;
            for (; n + 2 * DEEP <= steps; n += DEEP) {
#pragma unroll
                for (int i = 0; i < DEEP; ++i) {
                    compute(ring[i], step0 + KW * (n + i));
                    load(ring[i], n + i + DEEP);
                }
            }
#pragma unroll
            for (int i = 0; i < DEEP; ++i) {                 // (fewer than 2 DEEP are left)
                if (n + i < steps) compute(ring[i], step0 + KW * (n + i));
                if (n + i + DEEP < steps) load(ring[i], n + i + DEEP);
            }
#pragma unroll
            for (int i = 0; i < DEEP; ++i)
                if (n + i + DEEP < steps) compute(ring[i], step0 + KW * (n + i + DEEP));
        }
        // statistics of whole rows, and whether something has to be done again
        bool bad = false;
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            l[rt] = row_sum(l[rt]);
            float z = 0.f * l[rt];
#pragma unroll
            for (int j = 0; j < kTiles; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) z = __builtin_fmaf(0.f, o[rt][j][i], z);
            bad |= z != 0.f;
        }
        if (!CAREFUL) {
            const bool again = __any(bad);
            if (lane == 0) flags[wave] = again;
        }
        float* const stats = reinterpret_cast<float*>(buf + kJoin);   // [row wave][RT][KW][16] of m, then of l
        constexpr int kStats = RW * RT * KW * 16;
        float4* const meet = reinterpret_cast<float4*>(buf);          // [row wave][RT][KW][4][kLanes][64]
        if (KW > 1) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const int at = ((rw * RT + rt) * KW + kw) * 16 + row16;
                if (g == 0) {
                    stats[at] = m[rt];
                    stats[kStats + at] = l[rt];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < kLanes; ++c)
                        meet[((((rw * RT + rt) * KW + kw) * 4 + i) * kLanes + c) * 64 + lane] =
                            float4{o[rt][4 * c][i], o[rt][4 * c + 1][i], o[rt][4 * c + 2][i], o[rt][4 * c + 3][i]};
            }
        }
        if (KW > 1 || !CAREFUL) __syncthreads();
        bool again = false;
        if (!CAREFUL) {
#pragma unroll
            for (int i = 0; i < kWaves; ++i) again |= flags[i] != 0;
        }
        if (!again) {
            // a row tile's KW waves share its columns: unit i kLanes + c is columns (4 g + i) D / 16 + 4 c .. + 3 of each row
            constexpr int kUnits = 4 * kLanes;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                float top = m[rt], sum = l[rt], weight[KW];
                weight[0] = 1.f;
                if (KW > 1) {
                    const int at = (rw * RT + rt) * KW * 16 + row16;
                    top = -INFINITY;
#pragma unroll
                    for (int k = 0; k < KW; ++k) top = fmaxf(top, stats[at + 16 * k]);
                    sum = 0.f;
#pragma unroll
                    for (int k = 0; k < KW; ++k) {
                        // (a mean: no sum of the waves' overflows)
                        weight[k] = top == -INFINITY ? 0.f : (1.f / KW) * __builtin_amdgcn_exp2f(stats[at + 16 * k] - top);
                        sum += stats[kStats + at + 16 * k] * weight[k];
                    }
                    top += KW == 8 ? 3.f : KW == 4 ? 2.f : 1.f;
                }
                const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
                auto leave = [&](int i, int c, float4 x) {
                    x = float4{x.x * inv, x.y * inv, x.z * inv, x.w * inv};
                    const int32_t col = (4 * g + i) * (D / 16) + 4 * c;
                    if (item.slot < 0) {
                        if (out_row[rt] >= 0) store(a.out, out_row[rt] * D + col, x);
                    } else {
                        float4* const part = reinterpret_cast<float4*>(a.part_o) + (item.slot * (kRows / 16) + rw * RT + rt) * (4 * D);
                        part[col / 4 * 16 + row16] = x;
                    }
                };
                if constexpr (KW == 1) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int c = 0; c < kLanes; ++c)
                            leave(i, c, float4{o[rt][4 * c][i], o[rt][4 * c + 1][i], o[rt][4 * c + 2][i], o[rt][4 * c + 3][i]});
                } else {
                    for (int unit = kw; unit < kUnits; unit += KW) {
                        float4 x = float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int k = 0; k < KW; ++k) {
                            const float4 y = meet[(((rw * RT + rt) * KW + k) * kUnits + unit) * 64 + lane];
                            x = float4{x.x + weight[k] * y.x, x.y + weight[k] * y.y, x.z + weight[k] * y.z, x.w + weight[k] * y.w};
                        }
                        leave(unit / kLanes, unit % kLanes, x);
                    }
                }
                if (g == 0 && kw == 0) {
                    const float lse = sum == 0.f ? -INFINITY : top + __builtin_amdgcn_logf(sum);
                    if (item.slot >= 0) a.part_lse[item.slot * kRows + 16 * (rw * RT + rt) + row16] = lse;
                    else if (a.lse && out_row[rt] >= 0) a.lse[out_row[rt]] = lse * kLn2;
                }
            }
        }
        __syncthreads();                                     // (the next piece writes flags and LDS)
        return again;
    }

    // The walk of SHARED: operands of a tile of 64 keys are made while the tile before is computed, from codes that were asked for a tile
    // earlier.  1000 tokens behind 30000, 32 / 8 heads: 667 us where a wave makes its own 742; 1.5 of the 4 rows keys d flops for the weights' second
    // term, 1.12 PFLOP/s (a library product of 8192 x 8192 x 8192 1.21).  A wave at its products goes before one at its weights (without 682).
    static __device__ __forceinline__ void shared(char* buf, const TreeKernelArgs& a, const TreeItem& item, int32_t kvh, int32_t tiles, int32_t most,
                                                  int32_t least, const int32_t (&sees)[RT], const uint4 (&q)[RT][kQT][kSteps],
                                                  mfma_f32x4 (&o)[RT][kTiles], float (&m)[RT], float (&l)[RT], float sc)
    {
        const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        const int row16 = lane & 15, g = lane >> 4, half = wave & 1, sub = wave >> 1;
        const int32_t lp = a.cache.log2_page, P = 1 << lp;
        const int32_t* const table = a.block_table + (int64_t)item.s * a.max_blocks;
        const char* const base = (const char*)a.cache.k + (int64_t)kvh * a.cache.head_stride;
        const int32_t last_block = (item.len - 1) >> lp;
        const int ko = row16 >> 2, vo = g;
        const int32_t kslot = (8 * ko) & (P - 1), vslot = (8 * vo) & (P - 1);
        const int32_t k_at = (kslot + (row16 & 3) + 4 * half) * (D / 2) + g * (D / 8);
        const int32_t v_at = ((D / 2) << lp) + vslot * (D / 2) + row16 * (D / 4);
        const int32_t ks_at = ((D + g * (D / 4) / 32) << lp) + kslot;
        const int32_t vs_at = ((D + D / 32 + row16 * (D / 16) / 32) << lp) + vslot;
        uint32_t k[kKDwords], v[kVDwords];
        uint2 ks, vs;
        auto load = [&](int32_t tile) {
            const int32_t key0 = 64 * (item.tile_begin + tile) + 32 * sub;
            const int32_t b0 = min(key0 >> lp, last_block), b1 = min((key0 + 16) >> lp, last_block);
            const char* const first = base + (int64_t)table[b0] * a.cache.page_stride;
            const char* const second = base + (int64_t)table[b1] * a.cache.page_stride;
            const int32_t slot = key0 & (P - 1);
            const char* const kp = (ko >= 2 ? second : first) + slot * (D / 2) + k_at;
            const char* const vp = (vo >= 2 ? second : first) + slot * (D / 2) + v_at;
            if constexpr (D == 64) {
                const uint2 w = *reinterpret_cast<const uint2*>(kp);
                k[0] = w.x, k[1] = w.y;
            } else {
                const uint4 w = *reinterpret_cast<const uint4*>(kp);
                k[0] = w.x, k[1] = w.y, k[2] = w.z, k[3] = w.w;
            }
            ks = *reinterpret_cast<const uint2*>((ko >= 2 ? second : first) + slot + ks_at);
#pragma unroll
            for (int j = 0; j < kVDwords; j += 4) {
                const uint4 w = *reinterpret_cast<const uint4*>(vp + 4 * j);
                v[j] = w.x, v[j + 1] = w.y, v[j + 2] = w.z, v[j + 3] = w.w;
            }
            vs = *reinterpret_cast<const uint2*>((vo >= 2 ? second : first) + slot + vs_at);
        };
        // [16 keys][step][lane] of K, then [32 keys][column tile][lane] of V
        auto make = [&](int32_t tile, uint4* to) {
            const float unit = __uint_as_float((((half ? ks.y : ks.x) >> (8 * (row16 & 3))) & 0xffu) << 23);
#pragma unroll
            for (int t = 0; t < kSteps; ++t) to[(wave * kSteps + t) * 64 + lane] = bf16_eight(k[t], unit);
            // slots behind the sequence may hold anything, NaN among it
            const int32_t left = item.len - 64 * (item.tile_begin + tile) - 32 * sub - 8 * g;
            if (left < 8) {
                const uint64_t keep = left <= 0 ? 0 : ~0ull >> (64 - 8 * left);
                vs.x &= (uint32_t)keep;
                vs.y &= (uint32_t)(keep >> 32);
            }
            float vu[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) vu[i] = __uint_as_float(scale_bits(vs, i));
            uint32_t mine[kVDwords];                         // the wave's half of the columns in front
#pragma unroll
            for (int j = 0; j < kVDwords; ++j) mine[j] = v[j] >> (half * (D / 8));
            uint4* const vt = to + 4 * kSteps * 64 + (sub * kTiles + half * (kTiles / 2)) * 64 + lane;
            halves<0>(vt, mine, vu);
        };
        load(0);
        make(0, reinterpret_cast<uint4*>(buf));
        if (tiles > 1) load(1);
        __syncthreads();
        for (int32_t i = 0; i < tiles; ++i) {
            if (i + 1 < tiles) make(i + 1, reinterpret_cast<uint4*>(buf + ((i + 1) & 1) * kTileB));
            if (i + 2 < tiles) load(i + 2);
            const uint4* const from = reinterpret_cast<const uint4*>(buf + (i & 1) * kTileB);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int32_t key0 = 64 * (item.tile_begin + i) + 32 * u;
                if (key0 >= most) break;
                __builtin_amdgcn_s_setprio(1);
                mfma_f32x4 s[RT][2];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) s[rt][h] = mfma_f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int t = 0; t < kSteps; ++t) {
                    const uint4 k0 = from[(2 * u * kSteps + t) * 64 + lane], k1 = from[((2 * u + 1) * kSteps + t) * 64 + lane];
#pragma unroll
                    for (int z = 0; z < kQT; ++z)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            s[rt][0] = ElemBf16::mfma16(k0, q[rt][kQT - 1 - z][t], s[rt][0]);
                            s[rt][1] = ElemBf16::mfma16(k1, q[rt][kQT - 1 - z][t], s[rt][1]);
                        }
                }
                if (key0 + 32 > least) {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (key0 + 8 * g + e >= sees[rt]) s[rt][e / 4][e % 4] = -INFINITY;
                }
                uint4 w[RT][kPT];
                __builtin_amdgcn_s_setprio(0);
                weights<false>(w, s, o, m, l, sc);
                __builtin_amdgcn_s_setprio(1);
                const uint4* const vt = from + 4 * kSteps * 64 + u * kTiles * 64 + lane;
#pragma unroll
                for (int j = 0; j < kTiles; j += 2) {
                    const uint4 v0 = vt[j * 64], v1 = vt[(j + 1) * 64];
#pragma unroll
                    for (int z = 0; z < kPT; ++z)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            o[rt][j] = ElemBf16::mfma16(v0, w[rt][kPT - 1 - z], o[rt][j]);
                            o[rt][j + 1] = ElemBf16::mfma16(v1, w[rt][kPT - 1 - z], o[rt][j + 1]);
                        }
                }
            }
            __builtin_amdgcn_s_setprio(0);
            __syncthreads();
        }
    }

    template <int B>
    static __device__ __forceinline__ void halves(uint4* to, const uint32_t (&v)[kVDwords], const float (&vu)[8])
    {
        uint4 even, odd;
        column_pair<B>(even, odd, v, vu);
        to[2 * B * 64] = even;
        to[(2 * B + 1) * 64] = odd;
        if constexpr (B + 1 < D / 64) halves<B + 1>(to, v, vu);
    }

    // Operands of a lane's columns 2 B and 2 B + 1.
    template <int B>
    static __device__ __forceinline__ void column_pair(uint4& ve, uint4& vd, const uint32_t (&v)[kVDwords], const float (&vu)[8])
    {
        uint32_t even[4], odd[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t y0 = v_pair<B>(v, 2 * k, vu[2 * k]), y1 = v_pair<B>(v, 2 * k + 1, vu[2 * k + 1]);
            even[k] = __builtin_amdgcn_perm(y1, y0, 0x05040100u);
            odd[k] = __builtin_amdgcn_perm(y1, y0, 0x07060302u);
        }
        ve = uint4{even[0], even[1], even[2], even[3]};
        vd = uint4{odd[0], odd[1], odd[2], odd[3]};
    }

    template <int B>
    static __device__ __forceinline__ void columns(const Keys& x, const float (&vu)[8], const uint4 (&w)[RT][kPT], mfma_f32x4 (&o)[RT][kTiles])
    {
        uint4 ve, vd;
        column_pair<B>(ve, vd, x.v, vu);
#pragma unroll
        for (int u = 0; u < kPT; ++u)                        // (products that wait for each other lie apart)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                o[rt][2 * B] = ElemBf16::mfma16(ve, w[rt][kPT - 1 - u], o[rt][2 * B]);
                o[rt][2 * B + 1] = ElemBf16::mfma16(vd, w[rt][kPT - 1 - u], o[rt][2 * B + 1]);
            }
        if constexpr (B + 1 < D / 32) columns<B + 1>(x, vu, w, o);
    }

    static __device__ __forceinline__ float row_sum(float x)   // over the four lanes of a row
    {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        const auto u = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return __uint_as_float(u[0]) + __uint_as_float(u[1]);
    }
};

// Up to 16 rows: shape 0 has four waves along the keys, shape 4 eight.  Up to 32: shape 1, four; up to 64: shape 2, two; beyond: shape 3, a wave a
// row tile.
template <pa_dtype DT, int D>
pa_status launch_mx4_shape(const TreeKernelArgs& a, bool merge, int shape, hipStream_t stream)
{
    constexpr bool kWide = D == 256 || DT == PA_DTYPE_F32;   // O and Q of 32 rows do not fit a wave's registers
    constexpr bool kWhole = D == 256 && DT != PA_DTYPE_BF16; // nor those of 16 rows half of a SIMD's
    constexpr int OCC = kWhole ? 1 : 2, DEEP = 2, DEEP1 = DT == PA_DTYPE_F16 && D < 256 ? 1 : DEEP;
    switch (shape) {
        case 0: return launch_tree_of<Mx4Shape<DT, D, 1, 1, 4, OCC, DEEP>>(a, merge, stream);
        case 4: return launch_tree_of<Mx4Shape<DT, D, 1, 1, kWhole ? 4 : 8, 1, DEEP>>(a, merge, stream);
        case 1: return launch_tree_of<Mx4Shape<DT, D, kWide ? 1 : 2, kWide ? 2 : 1, kWide ? 2 : 4, OCC, DEEP1>>(a, merge, stream);
        case 2: return launch_tree_of<Mx4Shape<DT, D, kWide ? 1 : 2, kWide ? 4 : 2, kWide ? 1 : 2, OCC, DEEP1>>(a, merge, stream);
    }
    return launch_tree_of<Mx4Shape<DT, D, kWide ? 1 : 2, 4, 1, OCC, DEEP, (D < 256)>>(a, merge, stream);
}

template <int D>
pa_status launch_mx4_dim(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int shape, hipStream_t stream)
{
    switch (dtype) {
        case PA_DTYPE_F32: return launch_mx4_shape<PA_DTYPE_F32, D>(a, merge, shape, stream);
        case PA_DTYPE_F16: return launch_mx4_shape<PA_DTYPE_F16, D>(a, merge, shape, stream);
        default: return launch_mx4_shape<PA_DTYPE_BF16, D>(a, merge, shape, stream);
    }
}

}  // namespace

}  // namespace pa
