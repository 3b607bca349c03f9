// Attention over a cache of 4-bit elements (mx4_attention_impl.h) at head_dim 128, and its plan.
#include "mx4_attention_impl.h"

namespace pa {

pa_status launch_mx4_d64(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int shape, hipStream_t stream);
pa_status launch_mx4_d256(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int shape, hipStream_t stream);
pa_status launch_mx4_d128(const TreeKernelArgs& a, bool merge, pa_dtype dtype, int shape, hipStream_t stream)
{
    return launch_mx4_dim<128>(a, merge, dtype, shape, stream);
}

namespace {

struct Mx4Plan {
    int shape;                   // launch_mx4_shape's
    int32_t rows;                // of a workgroup
    int32_t row_blocks;          // most row blocks of a sequence
    int32_t wgs;                 // workgroups of a KV head that share all key tiles; 0: one a row block, no partials
    int32_t tile;                // keys
    size_t part_o_bytes, part_lse_bytes, cuts_bytes;
};

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// `wide`: 16 rows a wave where others take 32 (mx4_attention_impl.h).
Mx4Plan plan_mx4(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t d, int32_t total_q, int32_t max_q_len, int32_t max_seq_len,
                 pa_dtype dtype)
{
    const bool f32 = dtype == PA_DTYPE_F32, bf16 = dtype == PA_DTYPE_BF16;
    const bool wide = d == 256 || f32, whole = d == 256 && !bf16;
    Mx4Plan p = {};
    if (max_q_len > total_q) max_q_len = total_q;            // (a loose bound)
    const int64_t rows = (int64_t)max_q_len * (num_q_heads / num_kv_heads), keys = max_seq_len;
    const int64_t cus = device_cus(), heads = (int64_t)batch * num_kv_heads;
    int64_t whole_keys;                                      // longest contexts whose row blocks stay whole
    if (rows <= 16) {
        // A row block (a "unit" with its KV head) is one workgroup's where units fill the machine, or contexts are short; otherwise the keys are
        // shared and merged.  us, 32 / 8 heads of 128, eight waves whole / cut, four waves whole / cut:
        //     8 x 500..1000 9.6 / 13.3 10.2 / 13.3       8 x 128..2048 13.9 / 13.1 15.5 / 12.2      32 x 2000..4000 24.2 / 28.7 26.6 / 26.7
        //     64 x 500..1000 19.3 / 19.3 15.0 / 22.4     64 x 2000..4000 42.1 / 45.2 38.1 / 42.8    100 x 300..3000 42.4 / 41.3 39.0 / 36.2
        //     200 x 500..600 49.2 / 49.2 33.9 / 43.1     400 x 100..2000 110 / 104 76.0 / 81.1      64 x 64..32768 - / 78.1 - / 83.3
        //     1 x 4000 - / 13.7 - / 12.7                 1 x 100000 - / 28.0 - / 28.5               16 x 131072, 64 heads - / 396 - / 402
        if (heads <= cus) {
            p.shape = keys > 128 ? 4 : 0;
            whole_keys = 4 * heads >= 3 * cus ? 4096 : 1536;
        } else {
            p.shape = 0;
            whole_keys = 4096 * (heads / (2 * cus) > 1 ? heads / (2 * cus) : 1);
        }
        if (keys > whole_keys) p.shape = heads * keys >= cus * 2048 ? 4 : 0;
    } else {
        p.shape = rows <= 32 ? 1 : rows <= 64 ? 2 : 3;
    }
    p.rows = p.shape == 0 || p.shape == 4 ? 16 : p.shape == 1 ? 32 : p.shape == 2 || wide ? 64 : 128;
    p.tile = p.shape == 4 && !whole ? 256 : p.shape == 0 || p.shape == 4 || (p.shape == 1 && !wide) ? 128 : 64;
    const int64_t blocks = (rows + p.rows - 1) / p.rows;
    p.row_blocks = blocks < 1 ? 1 : (int32_t)blocks;
    const int64_t slots = cus * (p.shape == 4 || whole ? 1 : 2);
    // More rows, the same way (us whole / cut: 16 x 8 on 500..1000 13.8 / 16.8, 4 x 16 19.8 / 16.4, 16 x 16 20.0 / 26.3, 32 x 8 on 1500..3000 26.6 / 33.9,
    // 32 x 16 44.8 / 49.5, 64 x 16 72.9 / 80.5, on 300..6000 99.4 / 74.4; 16 x 32 on 500..1000 36.5 / 32.7, 32 x 32 39.0 / 48.2, on 1500..3000 96.5 / 76.7,
    // 64 x 32 129 / 133).
    if (p.shape == 1) whole_keys = heads >= cus ? 4096 : 1024;
    if (p.shape == 2) whole_keys = heads >= cus ? 4096 : 2 * heads >= cus ? 1024 : 512;
    if (p.shape == 3) {
        // Whole, too, where the rows that there are fill the machine, once for whole prompts and eight times for chunks behind contexts, whose lengths
        // may be far apart; but shared where sequences do not bring about as many rows each (four chunks of 512 tokens behind 64 to 32768 whole /
        // shared 722 / 417 us).
        const int64_t units = num_kv_heads * ((int64_t)total_q * (num_q_heads / num_kv_heads) / p.rows);
        whole_keys = units >= 2 * cus ? 4096 : units >= cus ? 1536 : 512;
        if (units >= slots * (keys <= 2 * (int64_t)max_q_len ? 1 : 8)) whole_keys = keys;
        if (2 * (int64_t)total_q < (int64_t)batch * max_q_len) whole_keys = 512;
    }
    const bool cut = keys > whole_keys;
    const int64_t tiles = ((int64_t)max_seq_len + p.tile - 1) / p.tile;
    if (cut) {
        const int64_t most = ((int64_t)batch * p.row_blocks * tiles + kTreeMinTiles - 1) / kTreeMinTiles;
        int64_t wgs = slots / num_kv_heads;
        if (wgs > most) wgs = most;
        p.wgs = wgs < 1 ? 1 : wgs > kTreeMaxPieces ? kTreeMaxPieces : (int32_t)wgs;
        const size_t part_rows = (size_t)p.wgs * num_kv_heads * 2 * p.rows;
        p.part_o_bytes = align256(part_rows * d * sizeof(float));
        p.part_lse_bytes = align256(part_rows * sizeof(float));
        p.cuts_bytes = align256((size_t)num_kv_heads * batch * p.row_blocks * sizeof(int2));
    }
    return p;
}

}  // namespace

size_t mx4_workspace_bytes(int32_t batch, int32_t num_q_heads, int32_t num_kv_heads, int32_t head_dim, int32_t total_q, int32_t max_q_len,
                           int32_t max_seq_len)
{
    size_t most = 256;                                       // (the type is not known here)
    for (const pa_dtype dtype : {PA_DTYPE_F32, PA_DTYPE_BF16, PA_DTYPE_F16}) {
        const Mx4Plan p = plan_mx4(batch, num_q_heads, num_kv_heads, head_dim, total_q, max_q_len, max_seq_len, dtype);
        const size_t bytes = p.part_o_bytes + p.part_lse_bytes + p.cuts_bytes;
        if (bytes > most) most = bytes;
    }
    return most;
}

pa_status launch_attention_mx4(const Mx4Args& t, void* workspace, hipStream_t stream)
{
    const pa_mx4_cache_desc* const c = t.cache;
    const Mx4Plan p = plan_mx4(t.batch, t.num_q_heads, c->num_kv_heads, c->head_dim, t.total_q, t.max_q_len, t.max_seq_len, t.dtype);
    // Places of a KV head stay below 2^31, threads of a launch below 2^32.
    const int64_t units = (int64_t)t.batch * p.row_blocks, threads = (int64_t)1 << 32;
    const int64_t tiles = ((int64_t)t.max_seq_len + p.tile - 1) / p.tile;
    if ((p.wgs > 0 ? p.wgs : units) * c->num_kv_heads * 512 >= threads) return PA_ERR_UNSUPPORTED;
    if (p.wgs > 0 && (tiles + kTreePieceTiles > 0x7fffffff / units || units * p.rows * c->head_dim / 4 >= threads)) return PA_ERR_UNSUPPORTED;
    const Mx4View v = make_view(c);
    TreeKernelArgs a = {};
    a.cache.k = a.cache.v = v.records;
    a.cache.page_stride = v.page_stride;
    a.cache.head_stride = v.head_stride;
    a.cache.page_size = c->page_size;
    a.cache.log2_page = v.log2_page;
    a.cache.num_kv_heads = c->num_kv_heads;
    a.cache.head_dim = c->head_dim;
    a.q = t.q;
    a.out = t.out;
    a.lse = t.lse;
    a.cu_q_lens = t.cu_q_lens;
    a.seq_lens = t.seq_lens;
    a.block_table = t.block_table;
    a.part_o = reinterpret_cast<float*>(workspace);
    a.part_lse = reinterpret_cast<float*>(reinterpret_cast<char*>(workspace) + p.part_o_bytes);
    a.cuts = reinterpret_cast<int2*>(reinterpret_cast<char*>(a.part_lse) + p.part_lse_bytes);
    a.batch = t.batch;
    a.num_q_heads = t.num_q_heads;
    a.max_blocks = t.max_blocks;
    a.group = t.num_q_heads / c->num_kv_heads;
    a.wgs = p.wgs;
    a.row_blocks = p.row_blocks;
    a.scale = t.scale;
    auto launch = [&](bool merge) {
        if (c->head_dim == 64) return launch_mx4_d64(a, merge, t.dtype, p.shape, stream);
        if (c->head_dim == 128) return launch_mx4_d128(a, merge, t.dtype, p.shape, stream);
        return launch_mx4_d256(a, merge, t.dtype, p.shape, stream);
    };
    // (A profiler shows both launches under the names of the kernels around a piece of work, paged_attention_tree_*_kernel<Mx4Shape>.)
    {
        ProfileScope prof("paged_attention_mx4_kernel", stream);
        const pa_status st = launch(false);
        if (st != PA_OK || p.wgs == 0) return st;
    }
    ProfileScope prof("paged_attention_mx4_merge_kernel", stream);
    return launch(true);
}

}  // namespace pa
