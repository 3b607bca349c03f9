// Bookkeeping of a step of drafted tokens on the GPU: slots, positions, ancestor masks and pages from request lengths
// (paged_plan_step), pages back to the free list (paged_release_blocks), and the accepted path of a verified tree with
// its K and V rows moved together (paged_tree_accept).  All three move a few kilobytes; what counts is that a step
// needs no round trip to the host, and the launches' own latency.
#include "common.h"

namespace pa {

namespace {

// ---- plan and release ----------------------------------------------------------------------------------------------
constexpr int kReleaseThreads = 1024;

// Inclusive sum over the workgroup (N threads) of one value a thread; `total` gets the whole sum.  sm: N / 64 numbers,
// free for the next call on return.
template <int N, typename T>
__device__ __forceinline__ T group_scan(T v, T* sm, T& total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const T up = __shfl_up(v, o, 64);
        if (lane >= o) v += up;
    }
    if (lane == 63) sm[wave] = v;
    __syncthreads();
    total = 0;
    T before = 0;
#pragma unroll
    for (int w = 0; w < N / 64; ++w) {
        const T x = sm[w];
        if (w < wave) before += x;
        total += x;
    }
    __syncthreads();
    return v + before;
}

// The sequence of a block of them that item m belongs to: the first whose inclusive sum exceeds it (m < the last sum).
template <int N>
__device__ __forceinline__ int32_t find_in(const int32_t* ends, int32_t m)
{
    int32_t lo = 0, hi = N - 1;
    while (lo < hi) {
        const int32_t mid = (lo + hi) >> 1;
        if (ends[mid] > m) hi = mid; else lo = mid + 1;
    }
    return lo;
}

struct PlanArgs {
    const int32_t* ctx_lens;
    const int32_t* new_lens;
    const int32_t* parents;      // or null: every token follows the one before it
    const int32_t* free_pages;
    int32_t* block_table;
    int32_t* num_blocks;
    int32_t* free_count;
    int32_t* seq_lens;
    int32_t* cu_q_lens;
    int32_t* seq_ids;
    int32_t* positions;
    int32_t* rope_positions;     // or null
    uint64_t* tree_mask;         // or null
    int32_t* shortage;
    int32_t batch, max_blocks, log2_page, max_rows, mask_words;
};

__device__ __forceinline__ int64_t blocks_for(int64_t tokens, int32_t log2_page)
{
    return (tokens + (1LL << log2_page) - 1) >> log2_page;
}

__device__ __forceinline__ int32_t at_most_int32(int64_t x) { return (int32_t)min(x, (int64_t)0x7fffffff); }

// Workgroup 0: everything that is one value a sequence, and the pages.  It alone writes what it and the others read
// nothing of but itself (counts, table, free list), so that a call can work in place in one launch; the others derive the
// rows' values from ctx_lens and new_lens, whether the request is granted or not.  Rows and pages are counted in 64 bits: lengths of
// several sequences, each within 31 bits, may add up to more, and what is refused for it must be seen to be.
template <int N>
__device__ __forceinline__ void plan_sequences(const PlanArgs& a)
{
    __shared__ int64_t sm64[N / 64];
    __shared__ int32_t sm_end[N];
    const int tid = threadIdx.x;
    const int32_t count = a.free_count[0];
    int32_t rows = 0, ctx = 0, have = 0;
    int32_t row_end = 0, need_end = 0;                       // (sums of 32 bits: exact where the request is granted)
    int64_t need = 0, rows_here = 0, pages_here = 0;
    bool late = false;
    auto look = [&](int32_t s) {                             // this thread's sequence, and the sums up to it
        need = 0;
        rows = 0;
        late = false;
        if (s < a.batch) {
            rows = max(a.new_lens[s], 0);
            ctx = a.ctx_lens[s];
            have = a.num_blocks[s];
            const int64_t tokens = (int64_t)ctx + rows;
            const int64_t want = blocks_for(tokens, a.log2_page);
            need = max(want - have, (int64_t)0);
            late = want > a.max_blocks || tokens > 0x7fffffff || (a.tree_mask && rows > 64LL * a.mask_words);
        }
        uint32_t r32, p32;
        row_end = (int32_t)group_scan<N>((uint32_t)rows, reinterpret_cast<uint32_t*>(sm64), r32);
        need_end = (int32_t)group_scan<N>((uint32_t)need, reinterpret_cast<uint32_t*>(sm64), p32);
        rows_here = r32;
        pages_here = p32;
        constexpr int32_t kSmall = (int32_t)(0x80000000u / N);   // N of them stay within 32 bits
        if (__syncthreads_or(rows > kSmall || need > kSmall)) {   // (in any case: 512 sequences and a release 12.5 us instead of 11.5)
            group_scan<N>((int64_t)rows, sm64, rows_here);
            group_scan<N>(need, sm64, pages_here);
        }
    };
    int64_t need_all = 0, long_all = 0, rows_all = 0;
    for (int32_t s0 = 0; s0 < a.batch; s0 += N) {
        look(s0 + tid);
        need_all += pages_here;
        rows_all += rows_here;
        long_all += __syncthreads_count(late);
    }
    if (rows_all > a.max_rows) long_all += rows_all - a.max_rows;
    const bool ok = need_all <= count && long_all == 0;
    int64_t rows_before = 0, pages_before = 0;
    for (int32_t s0 = 0; s0 < a.batch; s0 += N) {
        const int32_t s = s0 + tid;
        if (a.batch > N) look(s);                            // (one block of sequences is still at hand)
        sm_end[tid] = need_end;
        if (s < a.batch) {
            a.cu_q_lens[s + 1] = ok ? (int32_t)rows_before + row_end : 0;
            a.seq_lens[s] = ok ? ctx + rows : ctx;
        }
        __syncthreads();
        if (ok) {
            for (int32_t m = tid; m < pages_here; m += N) {   // (granted: 31 bits)
                const int32_t f = find_in<N>(sm_end, m);
                const int32_t at = m - (f ? sm_end[f - 1] : 0);
                a.block_table[(int64_t)(s0 + f) * a.max_blocks + a.num_blocks[s0 + f] + at] =
                    a.free_pages[count - 1 - pages_before - m];
            }
            __syncthreads();                                 // (the counts have been read)
            if (need > 0) a.num_blocks[s] = have + (int32_t)need;
        }
        rows_before += rows_here;
        pages_before += pages_here;
        __syncthreads();
    }
    if (tid == 0) {
        a.cu_q_lens[0] = 0;
        if (ok) a.free_count[0] = count - (int32_t)need_all;
        a.shortage[0] = at_most_int32(max(need_all - count, (int64_t)0));
        a.shortage[1] = at_most_int32(long_all);
    }
    for (int64_t r = min(rows_all, (int64_t)a.max_rows) + tid; r < a.max_rows; r += N) {
        a.seq_ids[r] = -1;
        a.positions[r] = -1;
        if (a.rope_positions) a.rope_positions[r] = 0;
        if (a.tree_mask)
            for (int32_t w = 0; w < a.mask_words; ++w) a.tree_mask[r * a.mask_words + w] = 0;
    }
}

// One wave: the rows of sequence s, 64 at a time.  The mask and the depth of a token come from its chain of parents, among the 64 by
// doubling (after round k a lane holds the union of the 2^k nearest and points 2^k up: 6 rounds of lane moves); a chain that leaves
// them goes on with the row of the token that it leaves to, which this wave has written before.
__device__ __forceinline__ void plan_rows(const PlanArgs& a, int32_t s)
{
    const int lane = threadIdx.x & 63;
    int64_t start = 0;                                       // (64 bits, as for workgroup 0)
    for (int32_t i = lane; i < s; i += 64) start += max(a.new_lens[i], 0);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) start += __shfl_xor(start, o, 64);
    const int32_t ctx = a.ctx_lens[s];
    const int32_t n = (int32_t)max(min((int64_t)a.new_lens[s], a.max_rows - start), (int64_t)0);   // of those that have a row
    for (uint32_t from = 0; from < (uint32_t)n; from += 64) {   // (n may be the largest 31-bit number)
        const int32_t base = (int32_t)from, i = base + lane;
        const int64_t r = start + i;
        const bool live = i >= 0 && i < n;
        int32_t depth = i;
        if (a.parents) {
            int32_t up = live ? a.parents[r] : -1;           // < 0: none, else a number within the sequence
            if (up < 0 || up >= i) up = -1;
            uint64_t bits = 1ull << lane;
            depth = up >= 0 ? 1 : 0;                         // steps to `up`, or to the root
            while (__any(up >= base)) {
                const int from = up >= base ? up - base : lane;
                const uint64_t b = __shfl((unsigned long long)bits, from, 64);
                const int32_t d = __shfl(depth, from, 64), u = __shfl(up, from, 64);
                if (up >= base) {
                    bits |= b;
                    depth += d;
                    up = u;
                }
            }
            if (base > 0) __threadfence_block();             // (the rows before are there)
            const int64_t above = start + up;                // < r
            if (live && up >= 0 && a.rope_positions) depth += a.rope_positions[above] - ctx;
            if (live && a.tree_mask)
                for (int32_t w = 0; w < a.mask_words; ++w)
                    a.tree_mask[r * a.mask_words + w] = w == base >> 6 ? bits : up >= 0 && w < base >> 6 ? a.tree_mask[above * a.mask_words + w] : 0;
        } else if (live && a.tree_mask) {
            for (int32_t w = 0; w < a.mask_words; ++w) {
                const int32_t k = i - 64 * w;                // bits 0 .. k of the word
                a.tree_mask[r * a.mask_words + w] = k < 0 ? 0 : k >= 63 ? ~0ull : (2ull << k) - 1;
            }
        }
        if (live) {
            a.seq_ids[r] = s;
            a.positions[r] = (int32_t)((uint32_t)ctx + (uint32_t)i);   // (past 31 bits: negative, which no append stores)
            if (a.rope_positions) a.rope_positions[r] = (int32_t)((uint32_t)ctx + (uint32_t)depth);
        }
    }
}

// (N threads: as many sequences at a time.  us with 256 / 1024, a release in front: 1 sequence 7.3 / 8.8, 200 7.6 / 9.0, 300 10.7 / 9.1,
// 512 14.0 / 11.0.)  Bound by the launch and three trips to memory: lengths and counts, free list, table.
template <int N>
__global__ __launch_bounds__(N) void paged_plan_step_kernel(PlanArgs a)
{
    if (blockIdx.x == 0) {
        plan_sequences<N>(a);
        return;
    }
    const int32_t s = ((int32_t)blockIdx.x - 1) * (N / 64) + (int32_t)(threadIdx.x >> 6);
    if (s < a.batch) plan_rows(a, s);
}

// Blocks of a sequence beyond ceil(keep_lens / P) go back to the end of the free list, the last one first: a plan that asks
// for the same blocks again gets the same pages.  Where the list has no room for all of them, its free places go to the last ones, and
// the rest, a row's first, stay mapped: no page is in neither.  One workgroup: the list is one.  About 4 us, next to all of it
// the launch and two trips.
__global__ __launch_bounds__(kReleaseThreads) void paged_release_blocks_kernel(
    const int32_t* __restrict__ keep_lens, int32_t* __restrict__ block_table, int32_t* __restrict__ num_blocks,
    int32_t* __restrict__ free_pages, int32_t* __restrict__ free_count, int32_t batch, int32_t max_blocks,
    int32_t log2_page, int32_t max_free)
{
    __shared__ int32_t sm[kReleaseThreads / 64];
    __shared__ int32_t sm_end[kReleaseThreads];
    const int tid = threadIdx.x;
    auto kept = [&](int32_t s) { return (int32_t)blocks_for(max(keep_lens[s], 0), log2_page); };
    auto gone = [&](int32_t s) { return s < batch ? max(min(num_blocks[s], max_blocks) - kept(s), 0) : 0; };
    const int32_t count = free_count[0];
    int32_t all = 0;
    for (int32_t s0 = 0; s0 < batch; s0 += kReleaseThreads) {
        int32_t t;
        group_scan<kReleaseThreads>(gone(s0 + tid), sm, t);
        all += t;
    }
    int32_t before = 0;
    for (int32_t s0 = 0; s0 < batch; s0 += kReleaseThreads) {
        int32_t here;
        const int32_t mine = gone(s0 + tid);
        sm_end[tid] = group_scan<kReleaseThreads>(mine, sm, here);
        __syncthreads();
        for (int32_t m = tid; m < here; m += kReleaseThreads) {
            const int32_t f = find_in<kReleaseThreads>(sm_end, m);
            const int32_t at = m - (f ? sm_end[f - 1] : 0);
            int32_t* const entry = block_table + (int64_t)(s0 + f) * max_blocks + kept(s0 + f) + at;
            const int64_t to = (int64_t)count + all - 1 - before - m;
            if (to >= max_free) continue;
            free_pages[to] = *entry;
            *entry = -1;
        }
        __syncthreads();
        if (mine > 0) {
            const int64_t first = (int64_t)count + all - 1 - before - (sm_end[tid] - mine);   // where this row's first one would go
            num_blocks[s0 + tid] = kept(s0 + tid) + (int32_t)min(max(first + 1 - max_free, (int64_t)0), (int64_t)mine);
        }
        before += here;
        __syncthreads();
    }
    if (tid == 0) free_count[0] = (int32_t)max(min((int64_t)count + all, (int64_t)max_free), (int64_t)count);
}

// ---- acceptance ----------------------------------------------------------------------------------------------------
constexpr int kAcceptThreads = 256;

struct AcceptArgs {
    const int32_t* cu_q_lens;
    const int32_t* seq_lens;
    const int32_t* parents;      // with tokens and targets: the path is found here; all null: it is given
    const int32_t* tokens;
    const int32_t* targets;
    const int32_t* block_table;
    int32_t* path;               // [batch, max_path]
    int32_t* path_lens;
    int32_t* next_tokens;        // or null
    int32_t* kept_lens;          // or null
    uint4* k_cache;
    uint4* v_cache;
    int64_t page_stride_v, token_stride_v, head_stride_v;   // in 16-byte pieces
    int32_t max_path, cap, max_blocks, log2_page, num_kv_heads, vec_per_head, num_pages;   // cap: most tokens of a path
};

// The path through the tree: node 0, then of the last one's children with the token the model chose there the first, while
// there is one.  Wave 0; sm_path and the result are the same on every lane.
__device__ __forceinline__ int32_t walk_tree(const AcceptArgs& a, int32_t row0, int32_t n, int32_t* sm_path, int32_t& next)
{
    const int lane = threadIdx.x & 63;
    int32_t count = 0, cur = 0;
    if (n <= 64) {                                           // the whole tree in one wave's registers
        const bool live = lane < n;
        const int32_t up = live ? a.parents[row0 + lane] : -1;
        const int32_t token = live ? a.tokens[row0 + lane] : -1;
        const int32_t target = live ? a.targets[row0 + lane] : -1;
        for (;;) {
            if (lane == 0) sm_path[count] = cur;
            ++count;
            next = __builtin_amdgcn_readlane(target, cur);
            if (count == a.cap) return count;
            const uint64_t hit = __ballot(live && lane > cur && up == cur && token == next);
            if (!hit) return count;
            cur = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)hit) - 1);
        }
    }
    for (;;) {
        if (lane == 0) sm_path[count] = cur;
        ++count;
        next = a.targets[row0 + cur];
        if (count == a.cap) return count;
        int32_t found = -1;
        for (int32_t base = cur + 1; base < n && found < 0; base += 64) {
            const int32_t c = base + lane;
            const uint64_t hit = __ballot(c < n && a.parents[row0 + min(c, n - 1)] == cur && a.tokens[row0 + min(c, n - 1)] == next);
            if (hit) found = base + __ffsll((unsigned long long)hit) - 1;
        }
        if (found < 0) return count;
        cur = __builtin_amdgcn_readfirstlane(found);
    }
}

// Grid (sequences, pieces of a token's K and V rows / 256).  A thread moves one 16-byte piece of all the path's rows, eight at a
// time and in the path's order: a path climbs (path[i] >= i, and each further than the one before), so no row is
// written before it has been read.  Bound by the launch and five trips (lengths, tree, page ids, rows in, rows out): 8 sequences of 16
// tokens 4.9 us, 256 of up to 64 12.
__global__ __launch_bounds__(kAcceptThreads) void paged_tree_accept_kernel(AcceptArgs a)
{
    extern __shared__ int32_t sm_path[];                     // [cap]
    __shared__ int32_t sm_len;
    const int32_t s = blockIdx.x;
    const int32_t row0 = a.cu_q_lens[s], n = a.cu_q_lens[s + 1] - row0;
    const int32_t ctx = a.seq_lens[s] - n;
    if (n <= 0) {                                            // (nothing drafted: nothing to keep)
        if (blockIdx.y == 0) {
            for (int32_t i = threadIdx.x; a.tokens && i < a.max_path; i += kAcceptThreads) a.path[(int64_t)s * a.max_path + i] = -1;
            if (threadIdx.x == 0) {
                if (a.tokens) a.path_lens[s] = 0;
                if (a.tokens && a.next_tokens) a.next_tokens[s] = -1;
                if (a.kept_lens) a.kept_lens[s] = ctx;
            }
        }
        return;
    }
    if (threadIdx.x < 64) {
        int32_t len, next = -1;
        if (a.tokens) {
            len = walk_tree(a, row0, n, sm_path, next);
        } else {
            len = min(max(a.path_lens[s], 0), min(n, a.cap));
            for (int32_t i = threadIdx.x; i < len; i += 64)
                sm_path[i] = min(max(a.path[(int64_t)s * a.max_path + i], 0), n - 1);
        }
        if (threadIdx.x == 0) {
            sm_len = len;
            if (blockIdx.y == 0) {
                if (a.tokens) a.path_lens[s] = len;
                if (a.tokens && a.next_tokens) a.next_tokens[s] = next;
                if (a.kept_lens) a.kept_lens[s] = ctx + len;
            }
        }
    }
    __syncthreads();
    const int32_t len = sm_len;
    if (a.tokens && blockIdx.y == 0)
        for (int32_t i = threadIdx.x; i < a.max_path; i += kAcceptThreads)
            a.path[(int64_t)s * a.max_path + i] = i < len ? sm_path[i] : -1;
    // 64 rows' places at a time, a thread each, then every thread's piece of them
    __shared__ int64_t sm_from[64], sm_to[64];               // 16-byte pieces into a pool; to < 0: nothing to move
    const int32_t piece = (int32_t)blockIdx.y * kAcceptThreads + threadIdx.x;
    const int32_t per_pool = a.num_kv_heads * a.vec_per_head;
    uint4* const pool = piece < per_pool ? a.k_cache : a.v_cache;
    const int32_t p = piece < per_pool ? piece : piece - per_pool;
    const int64_t in_token = (int64_t)(p / a.vec_per_head) * a.head_stride_v + p % a.vec_per_head;
    const int32_t* const table = a.block_table + (int64_t)s * a.max_blocks;
    auto place = [&](int32_t t) -> int64_t {                 // of token t, -1: it has no page
        if (t < 0 || (t >> a.log2_page) >= a.max_blocks) return -1;
        const int32_t page = table[t >> a.log2_page];
        if (page < 0 || page >= a.num_pages) return -1;
        return (int64_t)page * a.page_stride_v + (int64_t)(t & ((1 << a.log2_page) - 1)) * a.token_stride_v;
    };
    constexpr int kBatch = 8;
    for (int32_t base = 0; base < len; base += 64) {
        const int32_t rows = min(len - base, 64);
        if ((int)threadIdx.x < rows) {
            const int32_t i = base + threadIdx.x;
            const int64_t from = place(ctx + sm_path[i]), to = place(ctx + i);
            sm_from[threadIdx.x] = from;
            sm_to[threadIdx.x] = from < 0 || sm_path[i] == i ? -1 : to;
        }
        __syncthreads();
        if (piece < 2 * per_pool) {
            for (int32_t i0 = 0; i0 < rows; i0 += kBatch) {
                uint4 row[kBatch];
#pragma unroll
                for (int u = 0; u < kBatch; ++u)
                    if (i0 + u < rows && sm_to[i0 + u] >= 0) row[u] = pool[sm_from[i0 + u] + in_token];
#pragma unroll
                for (int u = 0; u < kBatch; ++u)
                    if (i0 + u < rows && sm_to[i0 + u] >= 0) pool[sm_to[i0 + u] + in_token] = row[u];
            }
        }
        __syncthreads();
    }
}

int log2_of(int32_t page_size)
{
    int l = 0;
    while ((1 << l) < page_size) ++l;
    return l;
}

}  // namespace

pa_status launch_plan_step(const StepPlanArgs& p, hipStream_t stream)
{
    PlanArgs a;
    a.ctx_lens = p.ctx_lens;
    a.new_lens = p.new_lens;
    a.parents = p.parents;
    a.free_pages = p.free_pages;
    a.block_table = p.block_table;
    a.num_blocks = p.num_blocks;
    a.free_count = p.free_count;
    a.seq_lens = p.seq_lens;
    a.cu_q_lens = p.cu_q_lens;
    a.seq_ids = p.seq_ids;
    a.positions = p.positions;
    a.rope_positions = p.rope_positions;
    a.tree_mask = p.tree_mask;
    a.shortage = p.shortage;
    a.batch = p.batch;
    a.max_blocks = p.max_blocks;
    a.log2_page = log2_of(p.page_size);
    a.max_rows = p.max_rows;
    a.mask_words = p.mask_words;
    ProfileScope prof("paged_plan_step_kernel", stream);
    if (p.batch <= 256) hipLaunchKernelGGL(paged_plan_step_kernel<256>, dim3(1 + (p.batch + 3) / 4), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(paged_plan_step_kernel<1024>, dim3(1 + (p.batch + 15) / 16), dim3(1024), 0, stream, a);
    return launch_status();
}

pa_status launch_release_blocks(const int32_t* keep_lens, int32_t batch, int32_t page_size, int32_t* block_table,
                                int32_t max_blocks, int32_t* num_blocks, int32_t* free_pages, int32_t* free_count,
                                int32_t max_free, hipStream_t stream)
{
    ProfileScope prof("paged_release_blocks_kernel", stream);
    hipLaunchKernelGGL(paged_release_blocks_kernel, dim3(1), dim3(kReleaseThreads), 0, stream, keep_lens, block_table,
                       num_blocks, free_pages, free_count, batch, max_blocks, log2_of(page_size), max_free);
    return launch_status();
}

pa_status launch_tree_accept(const pa_kv_cache_desc* c, const TreeAcceptArgs& t, hipStream_t stream)
{
    const CacheView v = make_view(c);
    const int32_t epv = c->dtype == PA_DTYPE_F32 ? 4 : 8;     // elements per 16-byte piece
    AcceptArgs a;
    a.cu_q_lens = t.cu_q_lens;
    a.seq_lens = t.seq_lens;
    a.parents = t.parents;
    a.tokens = t.tokens;
    a.targets = t.targets;
    a.block_table = t.block_table;
    a.path = t.path;
    a.path_lens = t.path_lens;
    a.next_tokens = t.next_tokens;
    a.kept_lens = t.kept_lens;
    a.k_cache = (uint4*)c->k_cache;
    a.v_cache = (uint4*)c->v_cache;
    a.page_stride_v = c->page_stride / epv;
    a.token_stride_v = c->token_stride / epv;
    a.head_stride_v = c->head_stride / epv;
    a.max_path = t.max_path;
    a.cap = t.cap;
    a.max_blocks = t.max_blocks;
    a.log2_page = v.log2_page;
    a.num_kv_heads = c->num_kv_heads;
    a.vec_per_head = c->head_dim / epv;
    a.num_pages = c->num_pages;
    const int64_t pieces = 2LL * a.num_kv_heads * a.vec_per_head;
    const int64_t groups = (pieces + kAcceptThreads - 1) / kAcceptThreads;
    if (groups > 65535) return PA_ERR_UNSUPPORTED;
    ProfileScope prof("paged_tree_accept_kernel", stream);
    hipLaunchKernelGGL(paged_tree_accept_kernel, dim3((uint32_t)t.batch, (uint32_t)groups), dim3(kAcceptThreads),
                       (size_t)t.cap * sizeof(int32_t), stream, a);
    return launch_status();
}

}  // namespace pa
