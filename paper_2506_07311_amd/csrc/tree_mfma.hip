// Matrix-core attention of drafted trees (tree_mfma_impl.h) at up to 128 columns, and its plan.
#include "tree_mfma_impl.h"

namespace pa {

pa_status launch_tree_d256(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int row_waves, hipStream_t stream);
pa_status launch_tree_d128(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int row_waves, hipStream_t stream)
{
    return launch_tree_dim<128>(a, merge, dtype, row_waves, stream);
}
pa_status launch_tree_d96(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int row_waves, hipStream_t stream);
pa_status launch_tree_d64(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int row_waves, hipStream_t stream);

pa_status launch_tree_f32(const TreeKernelArgs& a, bool merge, int row_waves, hipStream_t stream);

namespace {

int32_t columns_of(int32_t d, bool f32) { return d <= 64 ? 64 : d <= 96 && !f32 ? 96 : d <= 128 ? 128 : 256; }

// Keys of a tile that a cut call's workgroups share.
int32_t tile_of(int32_t columns, bool f32) { return f32 && columns > 128 ? 32 : 64; }

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

// 16-bit pools: up to 64 rows a (sequence, KV head) two waves share 32 rows, up to 128 at head_dims up to 128 as well, with eight
// waves; beyond that a workgroup takes 256 rows (128 above head_dim 128, where a wave's O and Q fill its registers).  fp32 pools: 16 rows a
// wave, 16, 32, 64 or 128 a workgroup.  The tiles are shared by as many workgroups as the machine holds at once.
//
// On short contexts a row block (a "unit" with its KV head) is one workgroup's and there is no merge:
//   * up to kPlainTiles tiles (us with 4 / 8 / 16: 16 x 8 tokens on 300 to 400 18.1 / 12.7 / 12.8, 4 x 8 on 800 to 900 15.8 / 15.7 / 20.8);
//     blocks of more than 64 rows are then made smaller until there is one for each compute unit (with / without: bf16 3 x 40 on 400 13.2 /
//     23.9, 16 x 40 on 350 19.1 / 24.5, fp32 3 x 40 on 400 27.7 / 65; until there are two: 32 x 40 on 350 35.7 / 28.7);
//   * 16-bit pools, units for half of the workgroups that the machine holds: up to kFullTiles, and as often as many as there are
//     rounds of them, since the longest one then is a small part of the call (with / without: 32 x 16 on 800 to 900 24.3 / 37.0, 32 x 64
//     55.0 / 81.7, 32 x 32 on 700 to 1400 41.8 / 54.3, 200 x 8 on 64 to 2000 116 / 123; where lengths are far apart 32 x 16 on 64 to 1500
//     29.8 / 26.3, 200 x 8 on 64 to 4000 191 / 184; a quarter of the workgroups, 8 x 64 on 700 to 1400, 62.0 / 36.3); above 128 columns,
//     where a workgroup holds only two tiles, units for all workgroups and up to 2 kPlainTiles (32 x 16 on 800 to 900, 16 / 8 heads,
//     44.9 / 60.1; 24 tiles: 100 x 16 on 64 to 3000 201 / 158; half of them: 16 x 16 on 700 to 1400 53.3 / 42.3);
//   * fp32 pools take kPlainTiles in any case (a matrix core does 1/16 of the work in the time: 8 x 40 on 600 to 900 132 / 89).
// Up to 32 rows whose workgroup has its compute unit to itself are four waves', a quarter of a tile of 128 keys each, of as many keys
// (with / without: 1 x 8 on 500 11.5 / 13.6, 16 x 8 on 350 11.9 / 12.9, 32 x 8 on 850 24.3 / 33.5, 16 x 8 on 850 19.8 / 21.7; 4 x 8 on 850, 32
// workgroups, 17.4 / 15.8, 64 x 8 on 400, 512 workgroups, 29.3 / 22.3).
TreePlan plan_tree(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t max_q_len, int32_t max_seq_len, bool f32)
{
    constexpr int32_t kPlainTiles = 8, kFullTiles = 24;
    TreePlan p;
    const int64_t rows = (int64_t)max_q_len * (num_q_heads / num_kv_heads);
    const int32_t columns = columns_of(head_dim, f32), wave_rows = f32 ? 16 : 32;
    if (f32) p.row_waves = rows <= 16 && columns <= 128 ? 1 : rows <= 32 ? 2 : rows <= 64 || columns > 128 ? 4 : 8;
    else p.row_waves = rows <= 64 ? 2 : rows <= 128 || columns > 128 ? 4 : 8;
    auto blocks_of = [&](int32_t waves) { return (rows + wave_rows * waves - 1) / (wave_rows * waves); };
    const int32_t tile = tile_of(columns, f32);
    const int64_t tiles = ((int64_t)max_seq_len + tile - 1) / tile;
    const int64_t cus = device_cus(), heads = (int64_t)batch * num_kv_heads;
    if (!f32 && rows <= 32 && columns <= 128 && heads <= cus && tiles <= (2 * heads >= cus ? kFullTiles : kPlainTiles)) {
        p.row_waves = 1;
    } else if (tiles <= kPlainTiles) {
        while (p.row_waves > 2 && heads * blocks_of(p.row_waves) < cus) p.row_waves /= 2;
    }
    const int64_t blocks = blocks_of(p.row_waves), units = heads * blocks;
    p.row_blocks = blocks < 1 ? 1 : (int32_t)blocks;
    p.wgs = 0;
    p.part_o_bytes = p.part_lse_bytes = p.cuts_bytes = 0;
    const int64_t slots = cus * (columns <= 128 && p.row_waves == 2 && !f32 ? 2 : 1);
    int64_t plain = kPlainTiles;
    if (!f32 && columns <= 128 && 2 * units >= slots) plain = kFullTiles * (units > slots ? units / slots : 1);
    if (!f32 && columns > 128 && units >= slots) plain = 2 * kPlainTiles;
    if (tiles > plain && (f32 || p.row_waves > 1)) {
        const int64_t most = (batch * blocks * tiles + kTreeMinTiles - 1) / kTreeMinTiles;
        int64_t wgs = slots / num_kv_heads;
        if (wgs > most) wgs = most;
        p.wgs = wgs < 1 ? 1 : wgs > kTreeMaxPieces ? kTreeMaxPieces : (int32_t)wgs;
        const size_t part_rows = (size_t)p.wgs * num_kv_heads * 2 * wave_rows * p.row_waves;
        p.part_o_bytes = align256(part_rows * columns * sizeof(float));
        p.part_lse_bytes = align256(part_rows * sizeof(float));
        p.cuts_bytes = align256((size_t)num_kv_heads * batch * p.row_blocks * sizeof(int2));
    }
    return p;
}

bool tree_mfma_supported(const TreeArgs& a)
{
    // (a lane's offset within a page is one of 32 bits)
    if (a.cache.page_size < 16 || a.cache.token_stride * a.cache.page_size >= ((int64_t)1 << 29)) return false;
    // Bounds so loose that the places of a KV head pass 31 bits, or a launch 2^32 threads, are the portable kernel's, whose grid goes by
    // the rows that there are.
    const bool f32 = a.dtype == PA_DTYPE_F32;
    const TreePlan p = plan_tree(a.batch, a.num_q_heads, a.cache.num_kv_heads, a.cache.head_dim, a.max_q_len, a.max_seq_len, f32);
    const int32_t columns = columns_of(a.cache.head_dim, f32), rows = p.row_waves * (f32 ? 16 : 32);
    const int64_t units = (int64_t)a.batch * p.row_blocks, threads = (int64_t)1 << 32;
    if ((p.wgs > 0 ? p.wgs + 7 : units + 7) * a.cache.num_kv_heads * 512 >= threads) return false;
    return p.wgs == 0 || ((a.max_seq_len + (int64_t)tile_of(columns, f32) - 1) / tile_of(columns, f32) + kTreePieceTiles <= 0x7fffffff / units &&
                          units * rows * columns / 4 < threads);   // (the merge: 256 threads for four lines of 64 vectors)
}

pa_status launch_tree_mfma(const TreeArgs& t, void* workspace, hipStream_t stream)
{
    const TreePlan p = plan_tree(t.batch, t.num_q_heads, t.cache.num_kv_heads, t.cache.head_dim, t.max_q_len, t.max_seq_len,
                                 t.dtype == PA_DTYPE_F32);
    TreeKernelArgs a;
    a.cache = t.cache;
    a.q = t.q;
    a.out = t.out;
    a.lse = t.lse;
    a.cu_q_lens = t.cu_q_lens;
    a.seq_lens = t.seq_lens;
    a.tree_mask = t.tree_mask;
    a.block_table = t.block_table;
    a.part_o = reinterpret_cast<float*>(workspace);
    a.part_lse = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + p.part_o_bytes);
    a.cuts = reinterpret_cast<int2*>(reinterpret_cast<char*>(a.part_lse) + p.part_lse_bytes);
    a.mask_words = t.mask_words;
    a.batch = t.batch;
    a.num_q_heads = t.num_q_heads;
    a.max_blocks = t.max_blocks;
    a.group = t.num_q_heads / t.cache.num_kv_heads;
    a.wgs = p.wgs;
    a.row_blocks = p.row_blocks;
    a.scale = t.scale;
    a.together = t.cache.head_stride * (t.dtype == PA_DTYPE_F32 ? 4 : 2) % 128 != 0;
    auto launch = [&](bool merge) {
        if (t.dtype == PA_DTYPE_F32) return launch_tree_f32(a, merge, p.row_waves, stream);
        switch (columns_of(t.cache.head_dim, false)) {
            case 64: return launch_tree_d64(a, merge, t.dtype, p.row_waves, stream);
            case 96: return launch_tree_d96(a, merge, t.dtype, p.row_waves, stream);
            case 128: return launch_tree_d128(a, merge, t.dtype, p.row_waves, stream);
        }
        return launch_tree_d256(a, merge, t.dtype, p.row_waves, stream);
    };
    {
        ProfileScope prof("paged_attention_tree_mfma_kernel", stream);
        const pa_status st = launch(false);
        if (st != PA_OK || p.wgs == 0) return st;
    }
    ProfileScope prof("paged_attention_tree_merge_kernel", stream);
    return launch(true);
}

}  // namespace pa
