// What the matrix-core kernels for drafted trees share (internal header): how a call's key tiles are divided among workgroups, the
// kernel around a piece of work, and the merge of what the division cuts.
//
// A shape S says what a workgroup does: kRows rows (query, head of the KV head's group) of one sequence at a time, kWaveRows
// of them a wave, in kColumns columns; tiles of kTile keys; kWaves waves, kOcc workgroups on a compute unit, kLds bytes of LDS; kCut: its
// row blocks may be cut; a sequence has kLeastTiles tiles even where it has no key (0: rows of an empty one are left as they are); and
//     work<CAREFUL>(buf, flags, args, item, KV head)   does a piece of work; true: it has to be done again with CAREFUL
//     store(out, element, float4)                     four output columns
#pragma once

#include "prefill_tiles.h"

namespace pa {

struct TreeKernelArgs {
    CacheView cache;
    const void* q;
    void* out;
    float* lse;
    // (kernel arguments of their own: the compiler has to know that nothing else points there, or page ids come by vector loads,
    // and each wait for one is a wait for every tile in flight: 16 x 16 tokens on 131072 2512 us)
    const int32_t* cu_q_lens;
    const int32_t* seq_lens;
    const uint64_t* tree_mask;
    const int32_t* block_table;
    float* part_o;               // [KV head][workgroup][2][wave of rows][rows x columns as the wave holds them], normalised
    float* part_lse;             // [KV head][workgroup][2][row], log2 domain
    int2* cuts;                  // [KV head][sequence][row block]: first workgroup and number of pieces
    int32_t mask_words, batch, num_q_heads, max_blocks, group;
    int32_t wgs;                 // workgroups of a KV head that share the tiles; 0: one a (sequence, row block)
    int32_t row_blocks;          // most row blocks of a sequence
    int32_t together;            // != 0: the KV heads of a share on one chiplet
    float scale;
};

namespace {

using namespace prefill;

// Fewest tiles of a workgroup that shares them.
constexpr int32_t kTreeMinTiles = 2;
// What a piece of work costs besides its tiles, in tiles (us with 0 / 4 / 8: 64 x 8 tokens on 64 to 32768 243 / 231 / 236, 16 x 8 on 300
// to 30000 88.2 / 85.0 / 86.3).
constexpr int32_t kTreePieceTiles = 4;
// Most tiles of a workgroup that has one piece of work (with 0 / 12 / 40: 1 x 8 on 20000 26.2 / 25.3 / 25.3, 2 x 40 on 4000 31.3 / 29.1 / 29.1,
// 16 x 8 on 300 to 30000 86.3 / 85.0 / 89.4, 8 x 64 on 3600 63.5 / 63.9 / 67.6).
constexpr int32_t kTreeMaxChunk = 12;
// Workgroups that share a row block; the merge has 32 weights of each in LDS.
constexpr int32_t kTreeMaxPieces = 256;
// Weights are taken against a reference that trails the maximum, so a sum of finite values times weights can leave the range of fp32
// where their mean does not.  It is then done again (CAREFUL) with the reference 2^24 above the largest score and taken anew
// where a lane's 16 weights sum to more than 2^-20: of up to 2^24 keys all weights sum to at most 1.  (They are fp32 there.)
constexpr float kCarefulBelow = -24.f, kCarefulSumMax = 1.f / (1 << 20);

// This wave's loads to LDS have landed but for the last N tiles' (LOADS of either pool each).  In order, so what the compiler
// has issued in between makes it wait for more, not for less.
template <int LOADS, int N>
__device__ __forceinline__ void wait_tiles_but()
{
    constexpr int V = 2 * LOADS * N;
    static_assert(V < 64, "more loads than the counter holds");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (V & 15) | ((V >> 4) << 14));   // vmcnt: bits 3..0 and 15..14
}

// A row's view of 32 keys from key0 on: bit i = key key0 + i is visible.
__device__ __forceinline__ uint32_t visible_keys(const uint64_t* __restrict__ mask, int32_t words, int32_t key0, int32_t ctx,
                                                 int32_t len)
{
    const int32_t node = key0 - ctx;
    uint32_t bits;
    if (node <= -32) {
        bits = ~0u;
    } else if (node < 0) {
        bits = ((uint32_t)mask[0] << -node) | ((1u << -node) - 1u);
    } else {
        const int32_t w = node >> 6, sh = node & 63;
        const uint64_t lo = w < words ? mask[w] >> sh : 0;
        const uint64_t hi = sh && w + 1 < words ? mask[w + 1] << (64 - sh) : 0;
        bits = (uint32_t)(lo | hi);
    }
    const int32_t left = len - key0;
    return left >= 32 ? bits : left <= 0 ? 0u : bits & ((1u << left) - 1u);
}

// A workgroup's piece of work: key tiles [tile_begin, tile_end) of row block rb of sequence s.
struct TreeItem {
    int32_t s, rb, row0, n, len, tile_begin, tile_end;
    int64_t slot;                // >= 0: a partial
};

// Row blocks and key tiles of sequence i.
struct TreeSeq {
    int32_t row0, n, len, blocks, tiles;
};
template <typename S>
__device__ __forceinline__ TreeSeq tree_seq(const TreeKernelArgs& a, int32_t i)
{
    TreeSeq q = {0, 0, 0, 0, 0};
    if (i < a.batch) {
        q.row0 = a.cu_q_lens[i];
        q.n = a.cu_q_lens[i + 1] - q.row0;
        q.len = a.seq_lens[i];
        q.blocks = q.n > 0 ? min((q.n * a.group + S::kRows - 1) / S::kRows, a.row_blocks) : 0;   // (n keeps to its bound)
        q.tiles = max((q.len + S::kTile - 1) / S::kTile, S::kLeastTiles);
    }
    return q;
}

// How a KV head's workgroups share the call's key tiles.  Where they are few, every row block is cut into chunks of about `chunk`
// tiles, one a workgroup.  Otherwise (chunk == 0) all tiles stand in a row, each row block's behind kTreePieceTiles places for what a
// piece of work costs besides its tiles, and workgroup x of wgs takes places [x all / wgs, (x + 1) all / wgs).
// (32-bit numbers: calls with more places are the portable kernel's, and a 64-bit division takes 0.2 us.)
struct TreeShare {
    int32_t all, wgs, chunk;
    uint32_t each, rest;         // all = wgs each + rest
    __device__ __forceinline__ int32_t begin(int32_t x) const   // floor(x all / wgs)
    {
        return (int32_t)((uint32_t)x * each + (uint32_t)x * rest / (uint32_t)wgs);
    }
};
template <typename S>
__device__ __forceinline__ TreeShare tree_share(const TreeKernelArgs& a, int lane, const TreeSeq& own)   // own: sequence `lane`
{
    int32_t tiles = 0, blocks = 0;
    for (int32_t i0 = 0; i0 < a.batch; i0 += 64) {
        const TreeSeq q = i0 == 0 ? own : tree_seq<S>(a, i0 + lane);
        tiles += wave_total_moves(q.blocks * q.tiles);
        blocks += wave_total_moves(q.blocks);
    }
    TreeShare r = {tiles + kTreePieceTiles * blocks, 1, 0, 0, 0};
    if (blocks < a.wgs) {
        const uint32_t c = (uint32_t)(tiles + a.wgs - blocks - 1) / (uint32_t)(a.wgs - blocks);
        if (c <= kTreeMaxChunk) r.chunk = max((int32_t)c, kTreeMinTiles);
        // A workgroup that has its compute unit to itself is worth up to four tiles (us without / with: 8 x 16 tokens on 128 to 2048
        // 21.2 / 18.4; four tiles in any case: 2 x 8 on 1500 13.9 / 14.6).
        if (S::kOcc > 1 && r.chunk > 0 && r.chunk < 4) {
            const int32_t alone = a.wgs / S::kOcc - blocks;
            r.chunk = max(r.chunk, alone <= 0 ? 4 : min(4, (int32_t)((uint32_t)(tiles + alone - 1) / (uint32_t)alone)));
        }
    }
    if (r.chunk == 0) {
        r.wgs = min(max(r.all / (kTreeMinTiles + kTreePieceTiles), 1), a.wgs);
        r.each = (uint32_t)r.all / (uint32_t)r.wgs;
        r.rest = (uint32_t)r.all % (uint32_t)r.wgs;
    }
    return r;
}
// Places of a row block of the sequence: chunks, or tiles and what comes before them.
__device__ __forceinline__ int32_t tree_places(const TreeShare& r, const TreeSeq& q)
{
    return q.blocks == 0 ? 0 : r.chunk > 0 ? (int32_t)((uint32_t)(q.tiles + r.chunk - 1) / (uint32_t)r.chunk) : q.tiles + kTreePieceTiles;
}

template <typename S>
__global__ __launch_bounds__(64 * S::kWaves, S::kOcc * S::kWaves / 4) void paged_attention_tree_mfma_kernel(
    TreeKernelArgs a, const int32_t* __restrict__ cu_q_lens, const int32_t* __restrict__ seq_lens,
    const int32_t* __restrict__ block_table, const uint64_t* __restrict__ tree_mask)
{
    a.cu_q_lens = cu_q_lens;
    a.seq_lens = seq_lens;
    a.block_table = block_table;
    a.tree_mask = tree_mask;
    __shared__ __attribute__((aligned(1024))) char buf[S::kLds];
    __shared__ uint32_t flags[8];
    const int lane = threadIdx.x & 63;
    const int32_t hkv = a.cache.num_kv_heads;
    // Workgroup i runs on chiplet i % 8.  KV heads in a row spread over the chiplets; where their rows share cache lines (160 or 192
    // bytes a row), the heads of a share stay on one, whose L2 then reads such a line once (us without / with: 8 x 8 tokens on 30000, head_dim
    // 80 146 / 117, 96 150 / 138; where they do not, 128 181 / 188, 64 112 / 117).
    int32_t kvh = (int32_t)(blockIdx.x % (uint32_t)hkv), x = (int32_t)(blockIdx.x / (uint32_t)hkv);
    if (a.together) {
        kvh = (int32_t)(blockIdx.x / 8 % (uint32_t)hkv);
        x = (int32_t)(blockIdx.x % 8 + 8 * (blockIdx.x / 8 / (uint32_t)hkv));
        if (a.wgs > 0 && x >= a.wgs) return;
    }
    // this workgroup's places [t, t_end), the sequence of the first and that one's first place
    int32_t s = 0;
    int32_t t = 0, t_end = 1, first = 0;
    TreeShare share = {0, 0, 0, 0, 0};
    TreeSeq q = {0, 0, 0, 0, 0};
    if (!S::kCut || a.wgs == 0) {                            // one row block
        s = x / a.row_blocks;
        q = tree_seq<S>(a, s);
        if (x % a.row_blocks >= q.blocks || q.tiles <= 0) return;   // (or no sequence's)
    } else {
        const TreeSeq start = tree_seq<S>(a, lane);
        share = tree_share<S>(a, lane, start);
        if (share.chunk > 0) {
            t = x;
            t_end = t + 1;
        } else {
            if (x >= share.wgs) return;
            t = share.begin(x);
            t_end = share.begin(x + 1);
        }
        bool found = false;
        for (int32_t i0 = 0; i0 < a.batch; i0 += 64) {
            const TreeSeq own = i0 == 0 ? start : tree_seq<S>(a, i0 + lane);
            const int32_t mine = own.blocks * tree_places(share, own), inc = wave_scan_moves(mine);
            const uint64_t hit = __ballot(first + inc > t);
            if (hit) {
                const int f = __ffsll((unsigned long long)hit) - 1;
                s = i0 + f;
                first += __builtin_amdgcn_readlane(inc, f) - __builtin_amdgcn_readlane(mine, f);
                q.row0 = __builtin_amdgcn_readlane(own.row0, f);
                q.n = __builtin_amdgcn_readlane(own.n, f);
                q.len = __builtin_amdgcn_readlane(own.len, f);
                q.blocks = __builtin_amdgcn_readlane(own.blocks, f);
                q.tiles = __builtin_amdgcn_readlane(own.tiles, f);
                found = true;
                break;
            }
            first += __builtin_amdgcn_readlane(inc, 63);
        }
        if (!found) return;
    }
    while (t < t_end) {
        TreeItem it;
        it.s = s;
        it.row0 = q.row0;
        it.n = q.n;
        it.len = q.len;
        if (!S::kCut || a.wgs == 0) {
            it.rb = x % a.row_blocks;
            it.tile_begin = 0;
            it.tile_end = q.tiles;
            it.slot = -1;
            t = t_end;
        } else {
            const int32_t places = tree_places(share, q);
            if (t >= first + q.blocks * places) {            // (nothing, or nothing more, of this one)
                first += q.blocks * places;
                if (++s >= a.batch) return;
                q = tree_seq<S>(a, s);
                continue;
            }
            it.rb = (int32_t)((uint32_t)(t - first) / (uint32_t)places);
            const int32_t at = t - first - it.rb * places;
            if (share.chunk > 0) {
                it.tile_begin = (int32_t)((uint32_t)(at * q.tiles) / (uint32_t)places);
                it.tile_end = (int32_t)((uint32_t)((at + 1) * q.tiles) / (uint32_t)places);
                t = t_end;
            } else {
                const int32_t to = min(places, at + (t_end - t));
                it.tile_begin = max(at - kTreePieceTiles, 0);
                it.tile_end = max(to - kTreePieceTiles, 0);
                t += to - at;
            }
            const bool whole = it.tile_begin == 0 && it.tile_end == q.tiles;
            it.slot = whole ? -1 : ((int64_t)kvh * a.wgs + x) * 2 + (it.tile_begin == 0 ? 1 : 0);
            if (it.tile_begin == it.tile_end) continue;      // (places before the tiles alone)
            if (it.tile_begin == 0 && threadIdx.x == 0) {    // what the merge has to know: workgroups up to the last tile's
                int32_t pieces = places;
                if (share.chunk == 0) {
                    // (the workgroup of the block's last place y: floor(((y + 1) wgs - 1) / all))
                    const int64_t end = first + (int64_t)(it.rb + 1) * places;
                    pieces = (int32_t)((end * share.wgs - 1) / share.all) - x + 1;
                }
                a.cuts[((int64_t)kvh * a.batch + s) * a.row_blocks + it.rb] = int2{x, pieces};
            }
        }
        if (S::template work<false>(buf, flags, a, it, kvh)) S::template work<true>(buf, flags, a, it, kvh);
    }
}

// The pieces of a row block that were cut, merged by their log-sum-exps.  Grid (sequences x row blocks x row waves x
// PARTS, KV heads): a wave's rows and a part of their columns each, in the partials' own order, so that a call of few sequences spreads over the
// machine as well.  Statistics first, all at once, and their weights into LDS.
template <typename S, int PARTS, int NW>
__global__ __launch_bounds__(64 * NW) void paged_attention_tree_merge_kernel(
    TreeKernelArgs a, const int32_t* __restrict__ cu_q_lens, const int32_t* __restrict__ seq_lens)
{
    a.cu_q_lens = cu_q_lens;
    a.seq_lens = seq_lens;
    constexpr int RB = S::kRows, RW = S::kWaveRows, WR = RB / RW, VECS = RW * S::kColumns / 4, MINE = VECS / PARTS, LINES = MINE / 64;
    extern __shared__ float weight[];                        // [pieces][RW]
    __shared__ float sm_top[RW], sm_sum[RW], sm_red[64 * NW / RW][RW];
    __shared__ float4 sm_acc[NW][LINES][64];
    const int32_t kvh = blockIdx.y, part = (int32_t)(blockIdx.x % PARTS);
    const int32_t rw = (int32_t)(blockIdx.x / PARTS) % WR;
    const int32_t u = (int32_t)(blockIdx.x / (PARTS * WR)), s = u / a.row_blocks, rb = u % a.row_blocks;
    const int2 cut = a.cuts[((int64_t)kvh * a.batch + s) * a.row_blocks + rb];
    const TreeSeq own = tree_seq<S>(a, s);
    const int32_t n_rows = own.n * a.group, r0 = rb * RB + RW * rw, d = a.cache.head_dim;
    if (rb >= own.blocks || r0 >= n_rows || own.tiles <= 0) return;   // (and then the cut is no one's)
    const int32_t pieces = cut.y;
    if (pieces == 1) return;
    const int64_t slot0 = ((int64_t)kvh * a.wgs + cut.x) * 2;
    auto slot = [&](int32_t k) { return slot0 + 2 * (int64_t)k + (k == 0 ? 1 : 0); };
    // float4 j of a wave's partial: lane j % 64 holds row j % RW, four columns of every 4 * 64 / RW.  Each of the NW waves takes
    // every NW-th piece, several pieces at a time, the first of them ahead of their weights; then they meet in LDS.
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane % RW;
    const float4* const po = reinterpret_cast<const float4*>(a.part_o) + rw * VECS + part * MINE + lane;
    constexpr int DEEP = LINES > 2 ? 2 : 8 / LINES;          // pieces at a time
    float4 v[DEEP][LINES];
    auto read = [&](int32_t k0) {
#pragma unroll
        for (int k = 0; k < DEEP; ++k)
#pragma unroll
            for (int i = 0; i < LINES; ++i) v[k][i] = po[slot(min(k0 + NW * k, pieces - 1)) * (WR * VECS) + 64 * i];
    };
    read(wave);
    constexpr int GROUPS = 64 * NW / RW;                     // threads a row
    const int32_t srow = threadIdx.x % RW, group = threadIdx.x / RW;
    float top = -INFINITY;
    for (int32_t k0 = group; k0 < pieces; k0 += 8 * GROUPS) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = a.part_lse[slot(min(k0 + i * GROUPS, pieces - 1)) * RB + RW * rw + srow];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (k0 + i * GROUPS < pieces) weight[(k0 + i * GROUPS) * RW + srow] = x[i];
            top = fmaxf(top, x[i]);
        }
    }
    sm_red[group][srow] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) top = fmaxf(top, sm_red[i][srow]);
    __syncthreads();
    const float use = top == -INFINITY ? 0.f : top;
    float wsum = 0.f;
    for (int32_t k = group; k < pieces; k += GROUPS) {       // (the thread's own)
        static_assert(kTreeMaxPieces <= 256, "weights of at most 2^-8: no sum of means overflows");
        const float w = 0x1p-8f * __builtin_amdgcn_exp2f(weight[k * RW + srow] - use);
        weight[k * RW + srow] = w;
        wsum += w;
    }
    sm_red[group][srow] = wsum;
    __syncthreads();
    if (group == 0) {
        wsum = 0.f;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) wsum += sm_red[i][srow];
        sm_top[srow] = top + 8.f;
        sm_sum[srow] = wsum;
    }
    __syncthreads();
    float4 acc[LINES];
#pragma unroll
    for (int i = 0; i < LINES; ++i) acc[i] = float4{0.f, 0.f, 0.f, 0.f};
    for (int32_t k0 = wave; k0 < pieces; k0 += NW * DEEP) {
        if (k0 > wave) read(k0);
#pragma unroll
        for (int k = 0; k < DEEP; ++k) {
            if (k0 + NW * k >= pieces) break;
            const float w = weight[(k0 + NW * k) * RW + row];
#pragma unroll
            for (int i = 0; i < LINES; ++i)
                acc[i] = float4{__builtin_fmaf(w, v[k][i].x, acc[i].x), __builtin_fmaf(w, v[k][i].y, acc[i].y),
                                __builtin_fmaf(w, v[k][i].z, acc[i].z), __builtin_fmaf(w, v[k][i].w, acc[i].w)};
        }
    }
#pragma unroll
    for (int i = 0; i < LINES; ++i) sm_acc[wave][i][lane] = acc[i];
    __syncthreads();
    for (int32_t i = wave; i < LINES; i += NW) {
        const int32_t j = part * MINE + 64 * i + lane, c = 4 * (j / RW), r = r0 + row;
        if (r >= n_rows || c >= d) continue;
        float4 x = sm_acc[0][i][lane];
#pragma unroll
        for (int k = 1; k < NW; ++k) {
            const float4 y = sm_acc[k][i][lane];
            x = float4{x.x + y.x, x.y + y.y, x.z + y.z, x.w + y.w};
        }
        const float sum = sm_sum[row], inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
        const int64_t out_row = (int64_t)(own.row0 + r / a.group) * a.num_q_heads + kvh * a.group + r % a.group;
        S::store(a.out, out_row * d + c, float4{x.x * inv, x.y * inv, x.z * inv, x.w * inv});
        if (a.lse && c == 0) a.lse[out_row] = sum == 0.f ? -INFINITY : (sm_top[row] + __builtin_amdgcn_logf(sum)) * kLn2;
    }
}

template <typename S, int PARTS, int NW>
void launch_tree_merge(const TreeKernelArgs& a, hipStream_t stream)
{
    const uint32_t x = (uint32_t)((int64_t)a.batch * a.row_blocks * (S::kRows / S::kWaveRows) * PARTS);
    hipLaunchKernelGGL((paged_attention_tree_merge_kernel<S, PARTS, NW>), dim3(x, (uint32_t)a.cache.num_kv_heads), dim3(64 * NW),
                       (size_t)a.wgs * S::kWaveRows * sizeof(float), stream, a, a.cu_q_lens, a.seq_lens);
}

// The attention kernel, or the merge behind it.
template <typename S>
pa_status launch_tree_of(const TreeKernelArgs& a, bool merge, hipStream_t stream)
{
    const int64_t units = (int64_t)a.batch * a.row_blocks;
    const int64_t shares = a.wgs > 0 ? a.wgs : units, grid = (a.together ? (shares + 7) / 8 * 8 : shares) * a.cache.num_kv_heads;
    // A merging workgroup takes four lines of 64 vectors of a wave's columns, or one and with twice the waves where there are few
    // (us with four / one: 2 x 8 tokens on 1500, 512 workgroups, 16.1 / 15.3; 8 x 16 on 128 to 2048, 2048 workgroups, 22.1 / 24.4;
    // with one, of four / eight / sixteen waves: 1 x 8 on 100000 with 8 / 1 heads, 32 workgroups and 256 pieces, 38.1 / 29.3 / 25.4,
    // 2 x 8 on 1500 14.1 / 13.8 / 16.6; a wave's first pieces ahead of their weights took 1 to 1.4 off the first).
    constexpr int LINES = S::kWaveRows * S::kColumns / 256, PARTS = LINES > 4 ? LINES / 4 : 1;
    const int64_t waves = units * (S::kRows / S::kWaveRows);
    if (grid > 0x7fffffffLL || waves * LINES > 0x7fffffffLL || a.cache.num_kv_heads > 65535) return PA_ERR_UNSUPPORTED;
    if (merge) {
        if constexpr (S::kCut) {
            if (waves * LINES * a.cache.num_kv_heads <= 512) launch_tree_merge<S, LINES, 8>(a, stream);
            else launch_tree_merge<S, PARTS, 4>(a, stream);
        }
    } else {
        hipLaunchKernelGGL((paged_attention_tree_mfma_kernel<S>), dim3((uint32_t)grid), dim3(64 * S::kWaves), 0, stream, a,
                           a.cu_q_lens, a.seq_lens, a.block_table, a.tree_mask);
    }
    return launch_status();
}

}  // namespace

}  // namespace pa
