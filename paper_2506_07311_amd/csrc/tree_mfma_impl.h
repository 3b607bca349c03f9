// Attention of trees of drafted tokens on the matrix cores: bf16 / fp16 pools, pages of 16 tokens and more, any head_dim the
// library takes (computed in DP = 64, 96, 128 or 256 columns).  Internal header: the kernel templates.
//
// A sequence's n drafted queries and the G query heads of a KV head are n * G rows that all see the context and differ
// in the last n keys only.  The context's K and V are read once for all of them, so up to about 200 rows the call is bound by
// that read, not by its 4 * rows * d flops a key; what the kernel is built for is to keep it going.
//   * A workgroup of four or eight waves owns RB = 32 * WR rows of one (sequence, KV head) and walks keys in tiles, whose K and V
//     rows the load unit writes straight into LDS through the block table, one to seven tiles ahead.  Rows are stored in
//     16-byte pieces swizzled so that neither kind of operand read meets a bank conflict.
//   * Beyond 128 rows (64 above 128 columns) a wave takes 32 rows and all 64 keys.  With fewer, two waves share 32 rows and halve the
//     tile, or on short contexts that leave a compute unit to each workgroup four waves with tiles of 128 keys; their results meet in
//     LDS at the end.
//   * Both products are transposed (v_mfma_f32_32x32x16, lane % 32 = row), so softmax statistics are a lane's own:
//         S^T[key, row] = K Q^T,   O^T[column, row] += V^T P^T.
//   * Softmax is online in the log2 domain against a reference that trails the maximum: weights are taken with the
//     reference as it stands, and only where a lane's sum leaves the range that 16-bit operands carry is it raised and O
//     rescaled.  Weights enter as two 16-bit terms (p = hi + lo), whatever the call's sizes and bounds are: a sequence's weights do
//     not become coarser because of the others' rows or of a loose bound.  Up to 64 rows the second term's matrix work hides behind the
//     read; with more it is a third of the matrix work (16 x 16 tokens on 131072, 64 / 8 heads, 1970 us where one term took 1600, 32 x 64 on
//     8000 413 / 320; but one term, 2^-9 of a weight in bf16, left an error against 64 bits 1.41 times that of the output's rounding, and more
//     where weights cancel).
//   * A key is masked by selection: key len - n + t of a tile is seen by a row if bit t of the row's words is set, 32 bits at a
//     time; tiles that end in the context take no mask at all.  An infinity or a NaN in a V row that some rows of a tile
//     do not see would reach them through a product with a weight of zero.  It always leaves its mark on an accumulator, so
//     they are looked at once, at the end, and such a piece of work is done again key by key (CAREFUL).  So is one with an infinity in K
//     that met the zeros of Q behind head_dim, and one whose sums of finite values left the range of fp32 (kCarefulBelow).
//   * Work is the batch's key tiles in a row (sequence, row block, tile), cut evenly over the workgroups of a KV head whatever the
//     lengths are; what a cut leaves unfinished goes to the workspace, and a second launch merges it.  On short contexts
//     a workgroup takes a whole row block and there is no second launch.
#pragma once

#include "tree_share.h"

namespace pa {

namespace {

template <int DP>
struct TreeGeo {
    static constexpr int kRowB = DP > 128 ? 512 : DP > 64 ? 256 : 128;   // bytes of a row in LDS
    static constexpr int kKS = DP / 16;                                  // steps of a score product
    static constexpr int kT = DP / 32;                                   // 32-column blocks of O
};

// A workgroup's waves: WR beside each other in rows, KW along a tile's keys.  Buffers as LDS holds them: what is in flight
// beside the tile being computed has to cover the memory's latency at its full rate, about 100 KB a compute unit.
template <int WR, int DP>
struct TreeShape {
    static constexpr int kKW = WR == 1 ? 4 : WR == 2 || (WR == 4 && DP <= 128) ? 2 : 1;
    static constexpr int kWaves = WR * kKW;
    static constexpr int kTile = WR == 1 ? 128 : 64;                     // keys
    static constexpr int kTileB = kTile * TreeGeo<DP>::kRowB;            // K part of a buffer; V follows
    static constexpr int kBufB = 2 * kTileB;
    static constexpr int kOcc = DP <= 128 && WR == 2 ? 2 : 1;            // workgroups of a compute unit
    static constexpr int kBufs = 131072 / (kOcc * kBufB);
    static constexpr int kLoads = kTileB / (1024 * kWaves);              // load instructions of a wave and pool a tile
};

// Byte offset inside its LDS row r of logical 16-byte piece L (rows of 512 bytes swizzle each half by itself; of rows of
// 128 bytes two share the banks).
template <int DP>
__device__ __forceinline__ int tree_piece(int L, int r)
{
    if (DP <= 64) return 16 * (L ^ (((r & 2) << 1) | ((r >> 2) & 3)));
    return 16 * ((L & 16) | ((L & 15) ^ swz(r)));
}

// V^T operand of 32 columns and 16 keys from row-major V: two transpose loads (keys 0-3 / 4-7 of a lane's contraction slots).
__device__ __forceinline__ uint4 tree_v_frag(const char* lo, const char* hi)
{
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    struct pair {
        s16x4 lo, hi;
    } r;
    r.lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(lo));
    r.hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(hi));
    return __builtin_bit_cast(uint4, r);
}

template <typename E>
__device__ __forceinline__ void tree_pack(uint4& w, uint4& wl, const f32x16& p, int r0)
{
    w.x = E::pack(p[r0 + 0], p[r0 + 1]);
    w.y = E::pack(p[r0 + 2], p[r0 + 3]);
    w.z = E::pack(p[r0 + 4], p[r0 + 5]);
    w.w = E::pack(p[r0 + 6], p[r0 + 7]);
    wl.x = E::pack(p[r0 + 0] - E::lo_of(w.x), p[r0 + 1] - E::hi_of(w.x));
    wl.y = E::pack(p[r0 + 2] - E::lo_of(w.y), p[r0 + 3] - E::hi_of(w.y));
    wl.z = E::pack(p[r0 + 4] - E::lo_of(w.z), p[r0 + 5] - E::hi_of(w.z));
    wl.w = E::pack(p[r0 + 6] - E::lo_of(w.w), p[r0 + 7] - E::hi_of(w.w));
}

// Where the softmax reference stands when it is taken, in powers of two below the largest score, and what a lane's 16 weights may
// sum to before it is taken anew.  fp16 has steps of 2^-24 at its least: with the reference at the largest score a second term of weights
// below 2^-9 of the largest loses bits and weights below 2^-25 are 0, while the sum of the weights has them (131072 keys of which one leads by
// e^18, the others of mean value 1, computed so in numpy: off by nine half steps).  2^11 below, with sums up to the largest fp16 number, a weight is kept
// to 2^-36 of the largest.  bf16 has the exponents of fp32.
// CAREFUL: see kCarefulBelow.
template <typename E, bool CAREFUL>
struct TreeReference {
    static constexpr bool kHalf = E::kDtype == PA_DTYPE_F16;
    static constexpr float kBelow = CAREFUL ? kCarefulBelow : kHalf ? 11.f : 0.f;
    static constexpr float kSumMax = CAREFUL ? kCarefulSumMax : kHalf ? 65504.f : kWeightSumMax;
    static_assert(CAREFUL || !kHalf || 16 * 2048 <= kSumMax, "16 weights of the largest score");
};

// Weights of 32 keys from their raw scores (-inf: not seen); sc > 0.
template <typename R, int T>
__device__ __forceinline__ void tree_softmax(f32x16& p, const f32x16& s, f32x16 (&o)[T], float& m, float& l, float sc)
{
    float psum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, -m));
        psum += p[r];
    }
    if (__any(!(psum <= R::kSumMax))) {                      // also the NaN or infinity of a fresh reference
        float top = -INFINITY;
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[r]);
        const float m_new = fmaxf(m, row_max<2>(top) * sc - R::kBelow);
        const float use = m_new == -INFINITY ? 0.f : m_new;  // (no key so far)
        const float alpha = __builtin_amdgcn_exp2f(m - use);
#pragma unroll
        for (int t = 0; t < T; ++t) o[t] *= alpha;
        l *= alpha;
        m = m_new;
        psum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            p[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], sc, -use));
            psum += p[r];
        }
    }
    l += psum;
}

// O^T += V^T P^T for 32 keys of which V may hold values that are not finite: key by key on the vector unit, each added only to the
// rows that see it.  vh = V's rows of the 32 keys; vis = their bits.
template <typename E, int DP, int T>
__device__ __forceinline__ void tree_pv_by_key(f32x16 (&o)[T], f32x16 p, const char* vh, uint32_t vis, int ql, int hh)
{
#pragma unroll 1
    for (int i = 0; i < 32; ++i) {
        const int key = 8 * (i >> 3) + 4 * (i & 1) + ((i >> 1) & 3);
        const float w = __shfl(p[0], ql + 32 * (i & 1), 64);
        const bool seen = (vis >> key) & 1u;
        const char* const row = vh + key * TreeGeo<DP>::kRowB + 8 * hh;
#pragma unroll
        for (int c = 0; c < 4 * T; ++c) {
            const uint2 v = *reinterpret_cast<const uint2*>(row + tree_piece<DP>(c, key));
            o[c / 4][4 * (c % 4) + 0] = seen ? __builtin_fmaf(w, E::lo_of(v.x), o[c / 4][4 * (c % 4) + 0]) : o[c / 4][4 * (c % 4) + 0];
            o[c / 4][4 * (c % 4) + 1] = seen ? __builtin_fmaf(w, E::hi_of(v.x), o[c / 4][4 * (c % 4) + 1]) : o[c / 4][4 * (c % 4) + 1];
            o[c / 4][4 * (c % 4) + 2] = seen ? __builtin_fmaf(w, E::lo_of(v.y), o[c / 4][4 * (c % 4) + 2]) : o[c / 4][4 * (c % 4) + 2];
            o[c / 4][4 * (c % 4) + 3] = seen ? __builtin_fmaf(w, E::hi_of(v.y), o[c / 4][4 * (c % 4) + 3]) : o[c / 4][4 * (c % 4) + 3];
            __builtin_amdgcn_sched_barrier(0);
        }
        if (i & 1) p = __builtin_shufflevector(p, p, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 0);   // the next pair's weight
    }
}

// Returns whether it has to be done again with CAREFUL (the same on every thread).
template <int WR, bool CAREFUL, typename E, int DP>
__device__ __forceinline__ bool tree_piece_of_work(char* buf, uint32_t* flags, const TreeKernelArgs& a, const TreeItem& it, int32_t kvh)
{
    typedef TreeGeo<DP> Geo;
    typedef TreeShape<WR, DP> Shape;
    constexpr int RB = 32 * WR, KW = Shape::kKW, NW = Shape::kWaves, NB = Shape::kBufs, ROWB = Geo::kRowB, T = Geo::kT, KS = Geo::kKS;
    constexpr int TK = Shape::kTile, HALVES = TK / 32 / KW;   // how often a wave takes 32 keys of a tile
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));                            // (what follows from it is not kept across pieces of work)
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int ql = lane & 31, hh = lane >> 5;
    const int rw = wave % WR, kw = wave / WR;
    const int32_t d = a.cache.head_dim, G = a.group, len = it.len, ctx = it.len - it.n, n_rows = it.n * G;
    const int32_t r_lane = it.rb * RB + 32 * rw + ql;
    const int32_t r = min(r_lane, n_rows - 1);
    const int32_t qi = r / G, h = kvh * G + r % G;
    const bool live = it.rb * RB + 32 * rw < n_rows;         // this wave has rows (wave-uniform)
    const uint64_t* const mask = a.tree_mask + (int64_t)(it.row0 + qi) * a.mask_words;
    const int32_t* const table = a.block_table + (int64_t)it.s * a.max_blocks;
    const int32_t last_key = len - 1;

    // Q as B operand: lane % 32 = row, step ks covers 8 elements of either lane half; 0 behind head_dim
    const uint16_t* const qrow = static_cast<const uint16_t*>(a.q) + ((int64_t)(it.row0 + qi) * a.num_q_heads + h) * d;
    uint4 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        qf[ks] = uint4{0, 0, 0, 0};
        if (16 * ks + 8 * hh < d) qf[ks] = *reinterpret_cast<const uint4*>(qrow + 16 * ks + 8 * hh);
    }

    // fetch role: instruction i of a wave fills rows RPI * (wave + NW i) .. of the tile, a lane the piece at position lane % PPR of
    // row RPI * (wave + NW i) + lane / PPR (pieces that head_dim does not have repeat others).  The swizzle repeats every 16
    // rows: with 8 rows between a wave's instructions, two in a row differ.
    constexpr int RPI = 1024 / ROWB, PPR = ROWB / 16, STEP = NW * RPI;
    const int frow = RPI * wave + lane / PPR;
    uint32_t lane_off[STEP == 8 ? 2 : 1];
#pragma unroll
    for (int v = 0; v < (STEP == 8 ? 2 : 1); ++v) {
        int piece = tree_piece<DP>(lane % PPR, frow + 8 * v) / 16;         // (the swizzle undoes itself)
        piece %= d / 8;
        lane_off[v] = 16 * piece;
    }
    const uint32_t lds0 = lds_address(buf) + 1024 * wave;
    int32_t pages[NB - 1][Shape::kLoads];                    // of the rows of each instruction (16 rows and more lie in one page)
    auto load_pages = [&](int b, int32_t t0) {
#pragma unroll
        for (int i = 0; i < Shape::kLoads; ++i) {
            const int32_t key = __builtin_amdgcn_readfirstlane(t0 + RPI * wave + STEP * i);
            pages[b][i] = table[min(key, last_key) >> a.cache.log2_page];
        }
    };
    auto fetch = [&](int b, int p, int32_t t0) {
#pragma unroll
        for (int i = 0; i < Shape::kLoads; ++i) {
            const int32_t slot = min(t0 + frow + STEP * i, last_key) & (a.cache.page_size - 1);
            int64_t page_off = ((int64_t)pages[p][i] * a.cache.page_stride + kvh * a.cache.head_stride) * 2;
            asm volatile("" : "+s"(page_off));               // stays in scalar registers
            const uint32_t off = (uint32_t)slot * (uint32_t)(a.cache.token_stride * 2) + lane_off[STEP == 8 ? i & 1 : 0];
            load_to_lds16(lds0 + b * Shape::kBufB, 1024 * NW * i, reinterpret_cast<const char*>(a.cache.k) + page_off, off);
            load_to_lds16(lds0 + b * Shape::kBufB, 1024 * NW * i + Shape::kTileB, reinterpret_cast<const char*>(a.cache.v) + page_off, off);
        }
    };

    // The first NB - 1 tiles (a piece of work has a tile at least), the page ids of all of them in one trip.  Q is waited for
    // behind the first of them: what is issued between a load and its wait is waited for as well.
#pragma unroll
    for (int i = 0; i < NB - 1; ++i) load_pages(i, min(it.tile_begin + i, it.tile_end - 1) * TK);
    fetch(0, 0, it.tile_begin * TK);
    // operand offsets: K piece 2 ks + hh of row ql; V pieces of the 32 columns t for the lane's transpose-load row, key 4 hh + j
    // (and 8 on) of a 16-key step, columns 4 qq .. + 3 of the 16-column block dblk
    uint32_t kx[KS], vx[2 * T];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kx[ks] = ql * ROWB + tree_piece<DP>(2 * ks + hh, ql);
    {
        const int j = (lane & 15) >> 2, qq = lane & 3, dblk = (lane >> 4) & 1;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int piece = 4 * t + 2 * dblk + (qq >> 1);
            vx[2 * t] = (4 * hh + j) * ROWB + tree_piece<DP>(piece, 4 * hh + j) + 8 * (qq & 1);
            vx[2 * t + 1] = (4 * hh + j + 8) * ROWB + tree_piece<DP>(piece, 4 * hh + j + 8) + 8 * (qq & 1);
        }
    }
    // The scale that the scores get is positive, so that masking commutes with it: a negative one's sign goes to Q, and for a scale of 0
    // Q is 0.
    const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u, hold = a.scale == 0.f ? 0u : ~0u;
    const float sc = a.scale == 0.f ? 1.f : __builtin_fabsf(a.scale) * kLog2e;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
        qf[ks] = uint4{(qf[ks].x ^ flip) & hold, (qf[ks].y ^ flip) & hold, (qf[ks].z ^ flip) & hold, (qf[ks].w ^ flip) & hold};
    int32_t ahead = it.tile_begin + 1;                       // the tile to fetch next
#pragma unroll
    for (int i = 1; i < NB - 1; ++i) {
        if (ahead < it.tile_end) fetch(i, i, ahead++ * TK);
    }
    if (ahead < it.tile_end) load_pages(0, ahead * TK);

    f32x16 o[T];
#pragma unroll
    for (int t = 0; t < T; ++t) o[t] = (f32x16)(0.f);
    float m = -INFINITY, l = 0.f;

    int b = 0;
#pragma unroll 1
    for (int32_t t = it.tile_begin; t < it.tile_end; ++t) {
        const int32_t after = ahead - t - 1;                 // tiles in flight behind this one
        constexpr int MANY = NB - 2, SOME = MANY > 3 ? 3 : MANY > 1 ? 1 : 0;
        if (after >= MANY) wait_tiles_but<Shape::kLoads, MANY>();
        else if (after >= SOME) wait_tiles_but<Shape::kLoads, SOME>();
        else wait_tiles_but<Shape::kLoads, 0>();
        __syncthreads();                                     // tile t is there, and tile t - 1 done with
        if (ahead < it.tile_end) {
            fetch(b == 0 ? NB - 1 : b - 1, 0, ahead * TK);
            if (++ahead < it.tile_end) load_pages(0, ahead * TK);   // (a tile before they are needed)
        }
        const char* const kbuf = buf + b * Shape::kBufB;
#pragma unroll 1
        for (int i = 0; i < HALVES; ++i) {
            const int half = KW > 1 ? kw : i;
            const int32_t key0 = t * TK + 32 * half;
            if (!live || key0 >= len) continue;              // (wave-uniform)
            f32x16 s = (f32x16)(0.f), p;
            const char* const kh = kbuf + 32 * half * ROWB;
            const char* const vh = kh + Shape::kTileB;
            // The operand reads are kept four ahead of their products and V's first step comes behind K's last: left to itself the
            // compiler waits for each read in front of the product that takes it.
            uint4 va[T], vb[T];
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                uint4 kf = *reinterpret_cast<const uint4*>(kh + kx[ks]);
                // (behind head_dim stand other pieces of the row: Q is 0 there, but 0 times an infinity of K is not)
                if (CAREFUL && 16 * ks + 8 * hh >= d) kf = uint4{0, 0, 0, 0};
                s = E::mfma32(kf, qf[ks], s);
            }
            if (!CAREFUL) {
#pragma unroll
                for (int c = 0; c < T; ++c) va[c] = tree_v_frag(vh + vx[2 * c], vh + vx[2 * c + 1]);
            }
            __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                if (ks + 4 < KS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                else __builtin_amdgcn_sched_group_barrier(0x100, (T + 1) / 2, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            uint32_t vis = ~0u;
            if (key0 + 32 > ctx) {                           // (wave-uniform: drafted keys, or the end)
                vis = visible_keys(mask, a.mask_words, key0, ctx, len);
                const uint32_t own = vis >> (4 * hh);        // score r is key 8 (r / 4) + 4 hh + r % 4
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = (own >> (8 * (r / 4) + r % 4)) & 1u ? s[r] : -INFINITY;
            }
            tree_softmax<TreeReference<E, CAREFUL>>(p, s, o, m, l, sc);
            if (CAREFUL) {
                tree_pv_by_key<E, DP, T>(o, p, vh, vis, ql, hh);
                continue;
            }
            __builtin_amdgcn_sched_barrier(0);
            uint4 w, wl;
            tree_pack<E>(w, wl, p, 0);
#pragma unroll
            for (int c = 0; c < T; ++c) {
                o[c] = E::mfma32(va[c], w, o[c]);
                o[c] = E::mfma32(va[c], wl, o[c]);
            }
#pragma unroll
            for (int c = 0; c < T; ++c) vb[c] = tree_v_frag(vh + 16 * ROWB + vx[2 * c], vh + 16 * ROWB + vx[2 * c + 1]);
            tree_pack<E>(w, wl, p, 8);
#pragma unroll
            for (int c = 0; c < T; ++c) {
                o[c] = E::mfma32(vb[c], w, o[c]);
                o[c] = E::mfma32(vb[c], wl, o[c]);
            }
            __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
#pragma unroll
            for (int c = 0; c < 2 * T; ++c) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
                __builtin_amdgcn_sched_group_barrier(0x002, 32 / T, 1);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        b = b == NB - 1 ? 0 : b + 1;
    }

    // Vector i of a wave's O is four columns of its rows.  Two waves that share rows exchange halves of theirs through a buffer that no
    // tile is in (buffers b on, but for the last tile's), so both join and store.
    l += __shfl_xor(l, 32, 64);
    constexpr int VECS = 4 * T, MINE = VECS / KW;
    auto vec = [&](int i) { return float4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]}; };
    float4* const met = reinterpret_cast<float4*>(buf + (b + rw / 2) % NB * Shape::kBufB) + rw % 2 * (VECS * 64) + lane;
    float2* const ml = reinterpret_cast<float2*>(buf + NB * Shape::kBufB) + rw * (KW * 64) + lane;
    if (!CAREFUL) {
        float odd[4] = {0.f, 0.f, 0.f, 0.f};                 // (0 times what is not finite is NaN)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) odd[i % 4] = __builtin_fmaf(o[t][i], 0.f, odd[i % 4]);
        const bool any = __any(!((odd[0] + odd[1]) + (odd[2] + odd[3]) == 0.f));
        if (lane == 0) flags[wave] = any ? 1u : 0u;
    }
    if (KW == 4) {
        float4* const all = reinterpret_cast<float4*>(buf + b * Shape::kBufB) + kw * (VECS * 64) + lane;
#pragma unroll
        for (int i = 0; i < VECS; ++i)
            if (i / MINE != kw) all[i * 64] = vec(i);
    }
    if (KW == 2) {
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            if (kw == 0) met[(MINE + i) * 64] = vec(VECS - MINE + i);
            else met[i * 64] = vec(i);
        }
    }
    if (KW > 1) ml[kw * 64] = float2{m, l};
    __syncthreads();                                         // (the tile buffers are free)
    if (!CAREFUL) {
        bool again = false;
#pragma unroll
        for (int w = 0; w < NW; ++w) again |= flags[w] != 0;
        if (again) return true;
    }
    float4 mine[MINE];
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        if (KW == 1 || kw == 0) mine[i] = vec(i);
        else if (KW == 2 || kw == 3) mine[i] = vec(VECS - MINE + i);
        else if (kw == 1) mine[i] = vec(VECS / 4 + i);
        else mine[i] = vec(VECS / 2 + i);
    }
    if (KW == 4) {
        const float4* const all = reinterpret_cast<const float4*>(buf + b * Shape::kBufB) + MINE * kw * 64 + lane;
        float2 s[KW];
#pragma unroll
        for (int k = 0; k < KW; ++k) s[k] = ml[k * 64];
        const float own = m;
        m = fmaxf(fmaxf(s[0].x, s[1].x), fmaxf(s[KW / 2].x, s[KW - 1].x));
        const float use = m == -INFINITY ? 0.f : m, wo = 0.25f * __builtin_amdgcn_exp2f(own - use);   // (a mean: no sum of the four overflows)
        l = 0.f;
#pragma unroll
        for (int i = 0; i < MINE; ++i) mine[i] = float4{mine[i].x * wo, mine[i].y * wo, mine[i].z * wo, mine[i].w * wo};
#pragma unroll
        for (int k = 0; k < KW; ++k) {
            const float w = 0.25f * __builtin_amdgcn_exp2f(s[k].x - use);
            l = __builtin_fmaf(s[k].y, w, l);
            if (k == kw) continue;
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
                const float4 v = all[(k * VECS + i) * 64];
                mine[i] = float4{__builtin_fmaf(v.x, w, mine[i].x), __builtin_fmaf(v.y, w, mine[i].y), __builtin_fmaf(v.z, w, mine[i].z),
                                 __builtin_fmaf(v.w, w, mine[i].w)};
            }
        }
        m += 2.f;
        __syncthreads();                                     // (before the next piece of work loads over them)
    }
    if (KW == 2) {
        const float2 m0 = ml[0], m1 = ml[64];
        m = fmaxf(m0.x, m1.x);
        const float use = m == -INFINITY ? 0.f : m;
        const float w0 = 0.5f * __builtin_amdgcn_exp2f(m0.x - use), w1 = 0.5f * __builtin_amdgcn_exp2f(m1.x - use);   // (a mean)
        l = m0.y * w0 + m1.y * w1;
        m += 1.f;
        const float wa = kw == 0 ? w0 : w1, wb = kw == 0 ? w1 : w0;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const float4 v = met[(i + MINE * kw) * 64];
            mine[i] = float4{mine[i].x * wa + v.x * wb, mine[i].y * wa + v.y * wb, mine[i].z * wa + v.z * wb, mine[i].w * wa + v.w * wb};
        }
        __syncthreads();                                     // (before the next piece of work loads over them)
    }
    if (!live) return false;
    const float inv = l > 0.f ? 1.f / l : 0.f;               // (a NaN among the scores is in O as well)
    const float lse2 = l <= 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l);
    const int first = KW == 1 ? 0 : kw * MINE;
    if (it.slot >= 0) {                                      // a partial, lane by lane: whole lines a store
        float4* const po = reinterpret_cast<float4*>(a.part_o) + (it.slot * WR + rw) * (VECS * 64) + first * 64 + lane;
#pragma unroll
        for (int i = 0; i < MINE; ++i) po[i * 64] = float4{mine[i].x * inv, mine[i].y * inv, mine[i].z * inv, mine[i].w * inv};
        if (hh == 0 && first == 0) a.part_lse[it.slot * RB + 32 * rw + ql] = lse2;
        return false;
    }
    if (r_lane >= n_rows) return false;
    const int64_t row = (int64_t)(it.row0 + qi) * a.num_q_heads + h;
    uint16_t* const orow = static_cast<uint16_t*>(a.out) + row * d + 8 * first + 4 * hh;
#pragma unroll
    for (int i = 0; i < MINE; ++i) {
        if (8 * (first + i) >= d) continue;                  // columns behind head_dim
        *reinterpret_cast<uint2*>(orow + 8 * i) = uint2{E::pack(mine[i].x * inv, mine[i].y * inv), E::pack(mine[i].z * inv, mine[i].w * inv)};
    }
    if (a.lse && hh == 0 && first == 0) a.lse[row] = lse2 * kLn2;
    return false;
}

template <int WR, typename E, int DP>
struct Tree16 {
    typedef TreeShape<WR, DP> Shape;
    static constexpr bool kCut = WR > 1;                                 // (one wave of rows is for calls without a cut)
    static constexpr int kLeastTiles = 0;
    static constexpr int kRows = 32 * WR, kWaveRows = 32, kColumns = DP, kTile = Shape::kTile, kWaves = Shape::kWaves, kOcc = Shape::kOcc;
    static constexpr int kLds = Shape::kBufs * Shape::kBufB + (Shape::kKW - 1) * WR * 1024;   // (maxima and sums of two waves)
    template <bool CAREFUL>
    static __device__ __forceinline__ bool work(char* buf, uint32_t* flags, const TreeKernelArgs& a, const TreeItem& it, int32_t kvh)
    {
        return tree_piece_of_work<WR, CAREFUL, E, DP>(buf, flags, a, it, kvh);
    }
    static __device__ __forceinline__ void store(void* out, int64_t at, float4 v)
    {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = uint2{E::pack(v.x, v.y), E::pack(v.z, v.w)};
    }
};

template <typename E, int DP>
pa_status launch_tree_type(const TreeKernelArgs& a, bool merge, int row_waves, hipStream_t stream)
{
    if constexpr (DP <= 128) {
        if (row_waves == 1) return launch_tree_of<Tree16<1, E, DP>>(a, merge, stream);
        if (row_waves == 8) return launch_tree_of<Tree16<8, E, DP>>(a, merge, stream);
    }
    if (row_waves == 2) return launch_tree_of<Tree16<2, E, DP>>(a, merge, stream);
    return launch_tree_of<Tree16<4, E, DP>>(a, merge, stream);
}

template <int DP>
pa_status launch_tree_dim(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int row_waves, hipStream_t stream)
{
    return dtype == PA_DTYPE_BF16 ? launch_tree_type<ElemBf16, DP>(a, merge, row_waves, stream)
                                  : launch_tree_type<ElemF16, DP>(a, merge, row_waves, stream);
}

}  // namespace

}  // namespace pa
