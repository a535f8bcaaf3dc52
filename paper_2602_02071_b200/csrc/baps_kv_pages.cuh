// Pages of the cache: rows of a batch rebuilt from parents (baps_kv_fork), used pages moved to the front (baps_kv_compact).
//
// Both are a prefix sum over the pages' reference counts, whole-number work on tables, and copies of pages.  Every choice
// (which free page, which hole) is by rank in ascending order, so that results are the same from call to call; the only
// atomics add whole numbers.  What bounds them: the copies' memory traffic for large pools, a chain of launches for small ones.
#pragma once
#include "baps_common.cuh"

namespace baps {

struct KvPool {
    uint8_t *codes[2];
    float *scale[2];
    int n_pages, Hkv, page;
    int64_t page_bytes;             // Hkv * page * D, a multiple of 1024
};

// Slice `part` of `parts` of page src, K and V and (part 0) the scales, to page dst.
__device__ __forceinline__ void copy_page(const KvPool &c, int64_t src, int64_t dst, int part, int parts)
{
    const int n16 = (int)(c.page_bytes / 16);
    for (int which = 0; which < 2; ++which) {
        const uint4 *from = reinterpret_cast<const uint4 *>(c.codes[which] + src * c.page_bytes);
        uint4 *to = reinterpret_cast<uint4 *>(c.codes[which] + dst * c.page_bytes);
        const int step = parts * (int)blockDim.x;
        int i = part * (int)blockDim.x + (int)threadIdx.x;
        for (; i + 3 * step < n16; i += 4 * step) {
            const uint4 a = from[i], b = from[i + step], d = from[i + 2 * step], e = from[i + 3 * step];
            to[i] = a; to[i + step] = b; to[i + 2 * step] = d; to[i + 3 * step] = e;
        }
        for (; i < n16; i += step) to[i] = from[i];
        if (part == 0)
            for (int h = threadIdx.x; h < c.Hkv; h += blockDim.x) c.scale[which][dst * c.Hkv + h] = c.scale[which][src * c.Hkv + h];
    }
}

// Sum over the block's threads before this one, and over all (blockDim.x a multiple of 32, up to 1024).
__device__ __forceinline__ int block_scan(int x, int *s_warp, int &total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int y = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int z = __shfl_up_sync(0xffffffffu, y, o);
        if (lane >= o) y += z;
    }
    if (lane == 31) s_warp[warp] = y;
    __syncthreads();
    if (warp == 0) {
        int w = lane < warps ? s_warp[lane] : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int z = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += z;
        }
        s_warp[lane] = w;
    }
    __syncthreads();
    const int before = warp ? s_warp[warp - 1] : 0;
    total = s_warp[warps - 1];
    __syncthreads();                                              // s_warp may be written again
    return before + y - x;
}

// ---- fork -----------------------------------------------------------------------------------------
struct KvForkParams {
    KvPool pool;
    const int32_t *table, *lengths, *refs, *parents;
    int32_t *new_table, *new_lengths, *new_refs;
    int32_t *begin, *first, *free_pages;         // workspace: [new_rows], [new_rows], [most]
    int rows, new_rows, width, reserve, window, sinks;
    int most;                                     // free pages that can be asked for, n_pages at most
};

constexpr int kForkRows = 8192;                   // rows of the old table at most

struct ForkRow {
    bool valid, fits;
    int parent, length, held, total;
};
__device__ __forceinline__ ForkRow fork_row(const KvForkParams &p, int parent)
{
    ForkRow r;
    r.parent = parent;
    r.valid = parent >= 0 && parent < p.rows;
    r.length = r.valid ? max(p.lengths[parent], 0) : 0;
    const int64_t page = p.pool.page, total = ((int64_t)r.length + p.reserve + page - 1) / page;
    r.held = (int)(((int64_t)r.length + page - 1) / page);
    r.fits = r.valid && total <= p.width;
    r.total = (int)min(total, (int64_t)p.width);
    return r;
}
// Page of column c (c < held) of the parent's row that a later query can see, -1 otherwise.
__device__ __forceinline__ int fork_entry(const KvForkParams &p, const ForkRow &r, int c)
{
    const int64_t page = p.pool.page, from = c * page, to = from + page;
    if (!(from < p.sinks || to > (int64_t)r.length - p.window + 1)) return -1;
    const int e = p.table[(int64_t)r.parent * p.width + c];
    return e >= 0 && e < p.pool.n_pages ? e : -1;
}
__device__ __forceinline__ bool fork_copies(const KvForkParams &p, const ForkRow &r, bool first)
{
    return r.fits && !first && r.length % p.pool.page != 0 && fork_entry(p, r, r.held - 1) >= 0;
}

// Block 0: what every row needs and where its share of the free pages begins (first[i]: bit 0 the oldest child of its
// parent), then the lowest free pages, as many as can be asked for.  The other blocks clear new_refs.
__global__ void __launch_bounds__(1024)
kv_fork_plan_kernel(const KvForkParams p)
{
    __shared__ int s_warp[32];
    __shared__ int s_oldest[kForkRows];            // of each parent: its first child
    allow_next_kernel();
    await_previous_kernel();
    if (blockIdx.x > 0) {
        for (int i = ((int)blockIdx.x - 1) * 1024 + (int)threadIdx.x; i < p.pool.n_pages; i += ((int)gridDim.x - 1) * 1024) p.new_refs[i] = 0;
        return;
    }
    for (int i = threadIdx.x; i < p.rows; i += 1024) s_oldest[i] = 0x7fffffff;
    __syncthreads();
    for (int i = threadIdx.x; i < p.new_rows; i += 1024) {
        const int parent = p.parents[i];
        if (parent >= 0 && parent < p.rows) atomicMin(s_oldest + parent, i);
    }
    __syncthreads();
    int base = 0;
    for (int i0 = 0; i0 < p.new_rows; i0 += 1024) {
        const int i = i0 + threadIdx.x;
        int need = 0;
        if (i < p.new_rows) {
            const int parent = p.parents[i];
            const ForkRow r = fork_row(p, parent);
            const bool oldest = r.valid && s_oldest[parent] == i;
            if (r.fits) need = r.total - r.held + (fork_copies(p, r, oldest) ? 1 : 0);
            p.first[i] = oldest ? 1 : 0;
        }
        int sum;
        const int before = block_scan(need, s_warp, sum);
        if (i < p.new_rows) p.begin[i] = base + before;
        base += sum;
    }
    const int need = min(base, p.most);
    int found = 0;
    // (four pages per thread and step, the next step's on their way; the array is aligned for 16-byte loads)
    auto load = [&](int64_t i) {
        int4 v = make_int4(1, 1, 1, 1);
        if (i + 3 < p.pool.n_pages) {
            v = *reinterpret_cast<const int4 *>(p.refs + i);
        } else {
            if (i < p.pool.n_pages) v.x = p.refs[i];
            if (i + 1 < p.pool.n_pages) v.y = p.refs[i + 1];
            if (i + 2 < p.pool.n_pages) v.z = p.refs[i + 2];
        }
        return v;
    };
    int4 now = load(4 * (int)threadIdx.x);
    for (int64_t i0 = 0; i0 < p.pool.n_pages && found < need; i0 += 4096) {
        const int i = (int)i0 + 4 * (int)threadIdx.x;
        const int r[4] = {now.x, now.y, now.z, now.w};
        now = load((int64_t)i + 4096);
        int free_here = 0, sum;
#pragma unroll
        for (int k = 0; k < 4; ++k) free_here += r[k] == 0;
        int at = found + block_scan(free_here, s_warp, sum);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (r[k] == 0) {
                if (at < need) p.free_pages[at] = i + k;
                ++at;
            }
        found += sum;
    }
    // what is missing is marked, so that rows that would take it see it
    for (int i = found + (int)threadIdx.x; i < need; i += 1024) p.free_pages[i] = -1;
}

// Blocks (row, part): part 0 writes the row of the table and counts, all parts copy a slice of the last page.
__global__ void __launch_bounds__(256)
kv_fork_rows_kernel(const KvForkParams p)
{
    allow_next_kernel();
    await_previous_kernel();
    const int i = blockIdx.x;
    const ForkRow r = fork_row(p, p.parents[i]);
    const bool copies = fork_copies(p, r, p.first[i] != 0);
    const int begin = p.begin[i], need = r.fits ? r.total - r.held + (copies ? 1 : 0) : 0;
    // every page that this row and the rows before it take was found
    bool ok = r.fits && (int64_t)begin + need <= p.most;
    if (ok && begin + need > 0) ok = p.free_pages[begin + need - 1] >= 0;
    const int copy_to = ok && copies ? p.free_pages[begin] : -1;
    if (copy_to >= 0) copy_page(p.pool, fork_entry(p, r, r.held - 1), copy_to, blockIdx.y, gridDim.y);
    if (blockIdx.y > 0) return;
    int32_t *row = p.new_table + (int64_t)i * p.width;
    for (int c = threadIdx.x; c < p.width; c += blockDim.x) {
        int e = -1;
        if (ok && c < r.held) e = copies && c == r.held - 1 ? copy_to : fork_entry(p, r, c);
        else if (ok && c < r.total) e = p.free_pages[begin + (copies ? 1 : 0) + c - r.held];
        row[c] = e;
        if (e >= 0) atomicAdd(p.new_refs + e, 1);
    }
    if (threadIdx.x == 0) p.new_lengths[i] = r.valid ? (ok ? r.length : -1) : 0;
}

// ---- compact ----------------------------------------------------------------------------------------
struct KvCompactParams {
    KvPool pool;
    const int32_t *table, *refs;
    int32_t *new_table, *new_refs, *page_map, *n_live;
    int32_t *chunk_live;                    // workspace: [chunks] used pages of a chunk of 1024
    int32_t *holes, *movers;                // workspace: [n_pages] each
    int32_t *n_moves;                       // workspace: [1]
    int rows, width, chunks;
};

__global__ void __launch_bounds__(1024)
kv_compact_count_kernel(const KvCompactParams p)
{
    allow_next_kernel();
    await_previous_kernel();
    const int i = blockIdx.x * 1024 + threadIdx.x;
    const int n = __syncthreads_count(i < p.pool.n_pages && p.refs[i] > 0);
    if (threadIdx.x == 0) p.chunk_live[blockIdx.x] = n;
}

// Every block: used pages before its chunk and in all, then the ranks of its pages.  A used page at or behind n_live is
// mover number (used pages before it) - (used pages before n_live), a free page before n_live is hole number (free pages
// before it); both lists are as long as each other.  kCounted: the chunks' counts are there; otherwise every block
// reads all counts of references (up to kCompactDirect pages, 256 KB from L2), which saves a launch.  Measured, us, direct / counted (97 % of the pages
// used, 1 KB of codes each): 1024 pages 4.9, 6.3; 4096 5.4, 6.4; 16384 7.5, 7.7; 32768 10.8, 8.9; 65536 14.4, 11.8; 131072 32.6, 19.5: the
// line could stand at a quarter of where it does.
// page_map of a mover is for the time being -2 - its number counted from the end.
constexpr int kCompactDirect = 65536;
template <bool kCounted>
__global__ void __launch_bounds__(1024)
kv_compact_lists_kernel(const KvCompactParams p)
{
    __shared__ int s_warp[32];
    allow_next_kernel();
    await_previous_kernel();
    const int chunk = blockIdx.x;
    int before = 0, live = 0, sum;
    if constexpr (kCounted) {
        for (int k = threadIdx.x; k < p.chunks; k += 1024) {
            const int n = p.chunk_live[k];
            live += n;
            if (k < chunk) before += n;
        }
    } else {
#pragma unroll 4
        for (int i = threadIdx.x; i < p.pool.n_pages; i += 1024) {
            const int used = p.refs[i] > 0 ? 1 : 0;
            live += used;
            if (i < chunk * 1024) before += used;
        }
    }
    block_scan(live, s_warp, sum);
    live = sum;
    block_scan(before, s_warp, sum);
    before = sum;
    const int i = chunk * 1024 + threadIdx.x;
    const int refs = i < p.pool.n_pages ? p.refs[i] : 0;
    const int rank = before + block_scan(refs > 0 ? 1 : 0, s_warp, sum);       // used pages before page i
    if (i < p.pool.n_pages) {
        const bool mover = refs > 0 && i >= live;
        if (mover) p.movers[live - 1 - rank] = i;
        if (refs <= 0 && i < live) p.holes[i - rank] = i;
        p.page_map[i] = mover ? -2 - (live - 1 - rank) : refs > 0 ? i : -1;
        p.new_refs[i] = refs > 0 && i < live ? refs : 0;
    }
    // movers = used pages behind the first n_live
    if (i == live - 1) *p.n_moves = live - rank - (refs > 0 ? 1 : 0);
    if (chunk == 0 && threadIdx.x == 0) {
        *p.n_live = live;
        if (live == 0) *p.n_moves = 0;
    }
}

// The first table_blocks blocks rewrite the table (an entry that a block of movers has not settled yet gives the same), the
// others copy, (move, part), striding over the moves.
__global__ void __launch_bounds__(256)
kv_compact_move_kernel(const KvCompactParams p, int table_blocks, int parts)
{
    allow_next_kernel();
    await_previous_kernel();
    const int n = *p.n_moves;
    if ((int)blockIdx.x < table_blocks) {
        const int64_t entries = (int64_t)p.rows * p.width;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < entries; i += (int64_t)table_blocks * 256) {
            const int e = p.table[i];
            int to = e >= 0 && e < p.pool.n_pages ? *const_cast<volatile int32_t *>(p.page_map + e) : -1;
            if (to < -1) to = p.holes[n - 1 - (-2 - to)];
            p.new_table[i] = to;
        }
        return;
    }
    const int first = ((int)blockIdx.x - table_blocks) / parts, part = ((int)blockIdx.x - table_blocks) % parts;
    const int step = ((int)gridDim.x - table_blocks) / parts;
    for (int k = first; k < n; k += step) {
        const int src = p.movers[n - 1 - k], dst = p.holes[k];
        copy_page(p.pool, src, dst, part, parts);
        if (part == 0 && threadIdx.x == 0) {
            p.page_map[src] = dst;
            p.new_refs[dst] = p.refs[src];
        }
    }
}

// Blocks per page copied: about 16 KB of K and as much of V each.
static inline unsigned copy_parts(int64_t page_bytes) { return (unsigned)((page_bytes + 16383) / 16384 < 16 ? (page_bytes + 16383) / 16384 : 16); }

static inline baps_status kv_fork_launch(const KvForkParams &p, cudaStream_t stream)
{
    const unsigned clear = (unsigned)((p.pool.n_pages + 4095) / 4096 < 64 ? (p.pool.n_pages + 4095) / 4096 : 64);
    const baps_status s = launch_kernel(kv_fork_plan_kernel, 1 + clear, 1024, 0, stream, p);
    if (s != BAPS_OK) return s;
    return launch_kernel(kv_fork_rows_kernel, dim3((unsigned)p.new_rows, copy_parts(p.pool.page_bytes)), 256, 0, stream, p);
}

static inline baps_status kv_compact_launch(const KvCompactParams &p, cudaStream_t stream)
{
    baps_status s = BAPS_OK;
    if (p.pool.n_pages <= kCompactDirect) {
        s = launch_kernel(kv_compact_lists_kernel<false>, (unsigned)p.chunks, 1024, 0, stream, p);
    } else {
        s = launch_kernel(kv_compact_count_kernel, (unsigned)p.chunks, 1024, 0, stream, p);
        if (s == BAPS_OK) s = launch_kernel(kv_compact_lists_kernel<true>, (unsigned)p.chunks, 1024, 0, stream, p);
    }
    if (s != BAPS_OK) return s;
    const int64_t parts = copy_parts(p.pool.page_bytes), want = 16LL * num_sms() / parts;
    const int64_t moves = want < p.pool.n_pages ? (want > 0 ? want : 1) : p.pool.n_pages;
    const int64_t wide = ((int64_t)p.rows * p.width + 255) / 256, table_blocks = wide < 512 ? wide : 512;
    return launch_kernel(kv_compact_move_kernel, (unsigned)(table_blocks + moves * parts), 256, 0, stream, p, (int)table_blocks, (int)parts);
}

} // namespace baps
