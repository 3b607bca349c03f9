// Attention of trees of drafted tokens for fp32 pools with pages of 16 tokens and more, on the fp32 matrix cores.
//
// As for the 16-bit pools (tree_mfma_impl.h), in v_mfma_f32_16x16x4 tiles, lane % 16 = row:
//     S^T[key, row] = K Q^T,   O^T[column, row] += V^T P^T.
// An fp32 product costs 16 times a 16-bit one, so the call is bound by its 4 * rows * d flops a key from about 16 rows a (sequence,
// KV head) on, and waves of 16 rows waste the fewest of them on rows that are not there.  A workgroup's eight waves, two a matrix
// core, take 128 rows, or 64 or 32 with two or four waves beside each other along a tile's 64 keys; up to 16 rows four waves
// take 16 keys each (more would find no keys), and above 128 columns there are four, since a wave's O and Q fill its registers.
// What a wave takes of a tile it takes at once: all its score products, their softmax, all products with V, so that few gaps
// are left between matrix instructions.  Since any order of a contraction's index serves, a lane reads 16 bytes of a K row for
// four products (product e takes element e of each lane's four), and P^T is the second product's operand as the first one leaves
// it: step r takes keys 4 g + r, of lane group g.  Operands are read ahead of their products.  A tile's K rows are swizzled for
// reads of one 16-byte piece of 16 rows, its V rows for reads of 16 columns of rows 4 apart.
//
// us (TFLOP/s, of the 157 that the matrix cores have) with 32 / 8 heads of 128: 8 x 64 tokens on 2048 174 (99), 8 x 16 65 (66), 8 x 8
// 45; with four waves, 64 rows and operands read when needed 232, 88, 54; eight waves alone 232, 81, 51; operands ahead 193, 69,
// 45; 32 keys at once 181, 65, 45.
#include "tree_share.h"

namespace pa {

namespace {

typedef mfma_f32x4 f32x4;

template <int WR, int DP>
struct Tree32 {
    static constexpr bool kCut = true;
    static constexpr int kWaves = WR > 1 && DP <= 128 ? 8 : 4, kOcc = 1, kRows = 16 * WR, kWaveRows = 16, kColumns = DP;
    static constexpr int kTile = DP > 128 ? 32 : 64;
    static constexpr int kKW = kWaves / WR < kTile / 16 ? kWaves / WR : kTile / 16;        // waves that share 16 rows
    static constexpr int kSubs = kTile / 16 / kKW;                               // times 16 keys of a tile that a wave takes
    static constexpr int kRowB = 4 * DP, kTileB = kTile * kRowB, kBufB = 2 * kTileB;
    static constexpr int kBufs = DP > 64 ? 2 : 4, kLds = kBufs * kBufB;
    static constexpr int kLoads = kTileB / (1024 * kWaves);
    template <bool CAREFUL>
    static __device__ __forceinline__ bool work(char* buf, uint32_t* flags, const TreeKernelArgs& a, const TreeItem& it, int32_t kvh);
    static __device__ __forceinline__ void store(void* out, int64_t at, float4 v)
    {
        *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = v;
    }
};

// Where 16-byte piece L of row r of a tile's K, V part stands in its row.
__device__ __forceinline__ int piece_k(int L, int r) { return (L & ~15) | ((L & 15) ^ swz(r)); }
__device__ __forceinline__ int piece_v(int L, int r) { return (L & ~15) | ((L & 15) ^ ((r & 12) | (r & 3))); }

template <int WR, int DP>
template <bool CAREFUL>
__device__ __forceinline__ bool Tree32<WR, DP>::work(char* buf, uint32_t* flags, const TreeKernelArgs& a, const TreeItem& it, int32_t kvh)
{
    constexpr int RB = kRows, KW = kKW, NW = kWaves, NB = kBufs, ROWB = kRowB, J = DP / 16, N = kSubs;
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                            // (what follows from it is not kept across pieces of work)
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ql = lane & 15, g = lane >> 4;
    const int rw = wave % WR, kw = wave / WR;                // (kw >= KW: loads alone)
    const int32_t d = a.cache.head_dim, G = a.group, len = it.len, ctx = it.len - it.n, n_rows = it.n * G;
    const int32_t r_lane = it.rb * RB + 16 * rw + ql;
    const int32_t r = min(r_lane, n_rows - 1);
    const int32_t qi = r / G, h = kvh * G + r % G;
    const bool live = it.rb * RB + 16 * rw < n_rows && kw < KW;   // this wave has rows (wave-uniform)
    const uint64_t* const mask = a.tree_mask + (int64_t)(it.row0 + qi) * a.mask_words;
    const int32_t* const table = a.block_table + (int64_t)it.s * a.max_blocks;
    const int32_t last_key = len - 1;

    // Q as B operand: lane % 16 = row, elements 16 j + 4 g + e; 0 behind head_dim
    const float* const qrow = static_cast<const float*>(a.q) + ((int64_t)(it.row0 + qi) * a.num_q_heads + h) * d;
    f32x4 qf[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        qf[j] = (f32x4)(0.f);
        if (16 * j + 4 * g < d) qf[j] = *reinterpret_cast<const f32x4*>(qrow + 16 * j + 4 * g);
    }

    // fetch role: instruction i of a wave fills rows RPI * (wave + NW i) .. of the tile, a lane the piece at position lane % PPR of its
    // row (pieces that head_dim does not have repeat others)
    constexpr int RPI = 1024 / ROWB, PPR = ROWB / 16, STEP = NW * RPI;
    const int frow = RPI * wave + lane / PPR;
    const uint32_t lds0 = lds_address(buf) + 1024 * wave;
    int32_t pages[NB - 1][kLoads];
    auto load_pages = [&](int b, int32_t t0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int32_t key = __builtin_amdgcn_readfirstlane(t0 + RPI * wave + STEP * i);
            pages[b][i] = table[min(key, last_key) >> a.cache.log2_page];
        }
    };
    auto fetch = [&](int b, int p, int32_t t0) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int row = frow + STEP * i;
            const int32_t slot = min(t0 + row, last_key) & (a.cache.page_size - 1);
            int64_t page_off = ((int64_t)pages[p][i] * a.cache.page_stride + kvh * a.cache.head_stride) * 4;
            asm volatile("" : "+s"(page_off));               // stays in scalar registers
            const uint32_t off = (uint32_t)slot * (uint32_t)(a.cache.token_stride * 4);
            const uint32_t pk = (uint32_t)piece_k(lane % PPR, row) % (uint32_t)(d / 4), pv = (uint32_t)piece_v(lane % PPR, row) % (uint32_t)(d / 4);
            load_to_lds16(lds0 + b * kBufB, 1024 * NW * i, reinterpret_cast<const char*>(a.cache.k) + page_off, off + 16 * pk);
            load_to_lds16(lds0 + b * kBufB, 1024 * NW * i + kTileB, reinterpret_cast<const char*>(a.cache.v) + page_off, off + 16 * pv);
        }
    };
#pragma unroll
    for (int i = 0; i < NB - 1; ++i) load_pages(i, min(it.tile_begin + i, it.tile_end - 1) * kTile);
    fetch(0, 0, it.tile_begin * kTile);
    // (a positive scale: masking commutes with it; a negative one's sign goes to Q, and for a scale of 0 Q is 0)
    const float sign = a.scale < 0.f ? -1.f : a.scale == 0.f ? 0.f : 1.f;
    const float sc = a.scale == 0.f ? 1.f : __builtin_fabsf(a.scale) * kLog2e;
#pragma unroll
    for (int j = 0; j < J; ++j) qf[j] = sign == 0.f ? (f32x4)(0.f) : qf[j] * sign;
    int32_t ahead = it.tile_begin + 1;                       // the tile to fetch next
#pragma unroll
    for (int i = 1; i < NB - 1; ++i) {
        if (ahead < it.tile_end) fetch(i, i, ahead++ * kTile);
    }
    if (ahead < it.tile_end) load_pages(0, ahead * kTile);

    f32x4 o[J];
#pragma unroll
    for (int c = 0; c < J; ++c) o[c] = (f32x4)(0.f);
    float m = -INFINITY, l = 0.f;
    int b = 0;
#pragma unroll 1
    for (int32_t t = it.tile_begin; t < it.tile_end; ++t) {
        const int32_t after = ahead - t - 1;                 // tiles in flight behind this one
        constexpr int MANY = NB - 2;
        if (after >= MANY) wait_tiles_but<kLoads, MANY>();
        else wait_tiles_but<kLoads, 0>();
        __syncthreads();                                     // tile t is there, and tile t - 1 done with
        if (ahead < it.tile_end) {
            fetch(b == 0 ? NB - 1 : b - 1, 0, ahead * kTile);
            if (++ahead < it.tile_end) load_pages(0, ahead * kTile);
        }
        const char* const kbuf = buf + b * kBufB;
#pragma unroll 1
        for (int sub = kw * N; sub < kTile / 16; sub += KW * N) {
            const int32_t key0 = t * kTile + 16 * sub;
            if (!live || key0 >= len) break;                 // (wave-uniform)
            const char* const kh = kbuf + 16 * sub * ROWB;
            const char* const vh = kh + kTileB;
            constexpr int AHEAD = 4;
            f32x4 kf[AHEAD];
            auto read_k = [&](int i) {                       // 16 keys after 16 keys
                const int j = i % J;
                const f32x4 k = *reinterpret_cast<const f32x4*>(kh + (16 * (i / J) + ql) * ROWB + 16 * piece_k(4 * j + g, ql));
                // (behind head_dim stand other pieces of the row: Q is 0 there, but 0 times an infinity of K is not)
                return CAREFUL && 16 * j + 4 * g >= d ? (f32x4)(0.f) : k;
            };
            float vf[2][J];
            auto read_v = [&](int i) {
                const int key = 4 * g + i % 4;
#pragma unroll
                for (int c = 0; c < J; ++c)
                    vf[i & 1][c] = *reinterpret_cast<const float*>(vh + (16 * (i / 4) + key) * ROWB + 16 * piece_v(4 * c + (ql >> 2), key) + 4 * (ql & 3));
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) kf[i] = read_k(i);
            f32x4 s[N], p[N];
#pragma unroll
            for (int u = 0; u < N; ++u) {
                f32x4 s0 = (f32x4)(0.f), s1 = (f32x4)(0.f);
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    const int i = u * J + j;
                    const f32x4 k = kf[i % AHEAD];
                    s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[0], qf[j][0], s0, 0, 0, 0);
                    s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[1], qf[j][1], s1, 0, 0, 0);
                    s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[2], qf[j][2], s0, 0, 0, 0);
                    s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[3], qf[j][3], s1, 0, 0, 0);
                    if (i + AHEAD < N * J) kf[i % AHEAD] = read_k(i + AHEAD);
                    __builtin_amdgcn_sched_barrier(0);
                }
                s[u] = s0 + s1;
            }
            if (!CAREFUL) read_v(0);
            __builtin_amdgcn_sched_barrier(0);
            uint32_t vis[(N + 1) / 2];                       // 32 keys each
#pragma unroll
            for (int u = 0; u < N; u += 2) vis[u / 2] = ~0u;
            if (key0 + 16 * N > ctx) {                       // (wave-uniform: drafted keys, or the end)
#pragma unroll
                for (int u = 0; u < N; u += 2) vis[u / 2] = visible_keys(mask, a.mask_words, key0 + 16 * u, ctx, len);
#pragma unroll
                for (int u = 0; u < N; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[u][i] = (vis[u / 2] >> (16 * (u & 1) + 4 * g + i)) & 1u ? s[u][i] : -INFINITY;
            }
            // online softmax against a reference that trails the maximum
            float psum = 0.f;
#pragma unroll
            for (int u = 0; u < N; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], sc, -m));
                    psum += p[u][i];
                }
            if (__any(!(psum <= (CAREFUL ? kCarefulSumMax : kWeightSumMax)))) {
                float top = -INFINITY;
#pragma unroll
                for (int u = 0; u < N; ++u) top = fmaxf(top, fmaxf(fmaxf(s[u][0], s[u][1]), fmaxf(s[u][2], s[u][3])));
                const float m_new = fmaxf(m, row_max<4>(top) * sc - (CAREFUL ? kCarefulBelow : 0.f));
                const float use = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = __builtin_amdgcn_exp2f(m - use);
#pragma unroll
                for (int c = 0; c < J; ++c) o[c] *= alpha;
                l *= alpha;
                m = m_new;
                psum = 0.f;
#pragma unroll
                for (int u = 0; u < N; ++u)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], sc, -use));
                        psum += p[u][i];
                    }
            }
            l += psum;
            if (CAREFUL) {
                // key by key on the vector unit, each only to the rows that see it
#pragma unroll
                for (int u = 0; u < N; ++u)
#pragma unroll 1
                    for (int k = 0; k < 16; ++k) {
                        const float own = (k & 2) ? ((k & 1) ? p[u][3] : p[u][2]) : ((k & 1) ? p[u][1] : p[u][0]);
                        const float w = __shfl(own, ql + 16 * (k >> 2), 64);
                        const bool seen = (vis[u / 2] >> (16 * (u & 1) + k)) & 1u;
#pragma unroll
                        for (int c = 0; c < J; ++c) {
                            const f32x4 v = *reinterpret_cast<const f32x4*>(vh + (16 * u + k) * ROWB + 16 * piece_v(4 * c + g, k));
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[c][e] = seen ? __builtin_fmaf(w, v[e], o[c][e]) : o[c][e];
                        }
                    }
                continue;
            }
#pragma unroll
            for (int i = 0; i < 4 * N; ++i) {
                if (i < 4 * N - 1) read_v(i + 1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int c = 0; c < J; ++c) o[c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[i & 1][c], p[i / 4][i % 4], o[c], 0, 0, 0);
            }
        }
        b = b == NB - 1 ? 0 : b + 1;
    }

    bool again = false;
    if (!CAREFUL) {
        bool odd = false;
#pragma unroll
        for (int c = 0; c < J; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= !(__builtin_fabsf(o[c][e]) <= 3.402823466e38f);
        const bool any = __any(odd);
        if (lane == 0) flags[wave] = any ? 1u : 0u;
    }
    __syncthreads();                                         // (the tile buffers are free)
    if (!CAREFUL) {
#pragma unroll
        for (int w = 0; w < NW; ++w) again |= flags[w] != 0;
        if (again) return true;
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (KW > 1) {                                            // the waves of 16 rows meet
        f32x4* const po = reinterpret_cast<f32x4*>(buf);
        auto at = [&](int k) { return ((k - 1) * WR + rw) * (J + 1) * 64 + lane; };
        if (kw > 0 && kw < KW) {
#pragma unroll
            for (int c = 0; c < J; ++c) po[at(kw) + c * 64] = o[c];
            po[at(kw) + J * 64] = f32x4{m, l, 0.f, 0.f};
        }
        __syncthreads();
        if (kw == 0) {
#pragma unroll
            for (int k = 1; k < KW; ++k) {
                const f32x4 ml = po[at(k) + J * 64];
                const float top = fmaxf(m, ml[0]), use = top == -INFINITY ? 0.f : top;
                const float wa = 0.5f * __builtin_amdgcn_exp2f(m - use), wb = 0.5f * __builtin_amdgcn_exp2f(ml[0] - use);
                l = l * wa + ml[1] * wb;
                m = top + 1.f;                               // (a mean: no sum of the two overflows)
#pragma unroll
                for (int c = 0; c < J; ++c) o[c] = o[c] * wa + po[at(k) + c * 64] * wb;
            }
        }
        __syncthreads();                                     // (before the next piece of work loads over them)
    }
    if (!live || kw > 0) return false;
    const float inv = l > 0.f ? 1.f / l : 0.f;               // (a NaN among the scores is in O as well)
    const float lse2 = l <= 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);
    if (it.slot >= 0) {                                      // a partial, lane by lane
        f32x4* const po = reinterpret_cast<f32x4*>(a.part_o) + (it.slot * WR + rw) * (J * 64) + lane;
#pragma unroll
        for (int c = 0; c < J; ++c) po[c * 64] = o[c] * inv;
        if (g == 0) a.part_lse[it.slot * RB + 16 * rw + ql] = lse2;
        return false;
    }
    if (r_lane >= n_rows) return false;
    const int64_t row = (int64_t)(it.row0 + qi) * a.num_q_heads + h;
    float* const orow = static_cast<float*>(a.out) + row * d;
#pragma unroll
    for (int c = 0; c < J; ++c)
        if (16 * c + 4 * g < d) *reinterpret_cast<f32x4*>(orow + 16 * c + 4 * g) = o[c] * inv;
    if (a.lse && g == 0) a.lse[row] = lse2 * kLn2;
    return false;
}

template <int DP>
pa_status launch_rows(const TreeKernelArgs& a, bool merge, int row_waves, hipStream_t stream)
{
    if constexpr (DP <= 128) {
        if (row_waves == 1) return launch_tree_of<Tree32<1, DP>>(a, merge, stream);
        if (row_waves == 8) return launch_tree_of<Tree32<8, DP>>(a, merge, stream);
    }
    if (row_waves == 2) return launch_tree_of<Tree32<2, DP>>(a, merge, stream);
    return launch_tree_of<Tree32<4, DP>>(a, merge, stream);
}

}  // namespace

pa_status launch_tree_f32(const TreeKernelArgs& a, bool merge, int row_waves, hipStream_t stream)
{
    const int32_t d = a.cache.head_dim;
    return d <= 64 ? launch_rows<64>(a, merge, row_waves, stream) : d <= 128 ? launch_rows<128>(a, merge, row_waves, stream) : launch_rows<256>(a, merge, row_waves, stream);
}

}  // namespace pa
