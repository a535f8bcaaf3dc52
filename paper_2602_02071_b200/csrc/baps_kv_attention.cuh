// Attention of the last T tokens of every sequence over the 8-bit cache.
//
//     s = c * k_scale * (q . k_code),  w = 2^(s - m),  l = sum w,  O~ = sum w * v_scale * v_code;   O = O~ / l
// A part of the keys hands on its (m, l) and O, not O~: a sum of values may be beyond float32 where their mean is not.  Parts are
// joined as  m = max m_i,  l = sum 2^(m_i - m) l_i,  O = sum (2^(m_i - m) l_i / l) O_i.
// with c = log2(e) * scale and a running reference m, six below a maximum that is followed when a score passes it by more
// than 8, so that weights stay below 2^14.  Codes become fp16 in registers (exactly: E4M3 has 4 significant bits), q is scaled
// by a power of two per row so that its 8 or 11 bits fit fp16 (what is lost is below 2^-25 of the row's largest element),
// and both products run on mma.sync m16n8k16 with float32 accumulation; the weights are rounded to fp16 (half a step, 2^-11)
// after they have been summed.  The scales are applied in float32; O~ is kept in units of a value scale that is followed
// where a page's leaves [unit / 64, unit], down to 2^-64 of the largest that there was: O~, below 2^14 * 448 in units of that one
// for each key, then stays below 2^118 for 2^31 keys, and what is smaller does not count.
//
// What bounds it: the bytes of K and V, one per element: 48 sequences of 8192 to 32768 tokens, 32 / 8 heads of 128, pages of 64,
// 298 us for one draw of lengths (2.00 GB) ten times in a graph, 6.7 TB/s, some of it from L2; 316 us with lengths and pages drawn anew for each
// call (2.01 GB on average), 6.4 TB/s.  mma.sync, not tcgen05: the codes have to be widened in registers on the way, and a CTA has 8 to 32 rows of
// queries, where a tcgen05 tile has 128.  K and V are the operand with 16 rows and the queries the one with 8 columns
// (S^T = K Q^T, O^T = V^T P^T), so that eight query rows waste nothing: a product of 16 x 8 x 16 takes 8 cycles of a scheduler's
// tensor core and covers 256 codes.  (Queries as the 16 rows: twice the products, 471 us.  E4M3 operands, q and weights in two
// parts each: mma.sync m16n8k32 is carried out as fp16 products with both operands widened every time, 26 cycles instead
// of 5 once they change, 433 us.)
//
// Work is cut evenly whatever the lengths: the 64-key tiles of all sequences and kv heads, visible ones only, in one row;
// CTA i takes an equal share.  What a CTA does of a sequence and head that is not whole goes to the workspace and a
// second kernel joins it, in the order of the CTAs.  (Short ones, and those that a window cuts to one length, go to clusters:
// kv_shape.)  Each of a CTA's four warps takes every fourth 32 keys of its share for 8 to 32 rows of queries and keeps
// m, l and O~ in registers; they are joined through shared memory where a sequence and head ends.  A warp copies its own
// keys (16 bytes per lane, two to four steps ahead), so that no warp waits for another before that.
// (Before: a producer warp and TMA boxes into a ring of tiles.  The same 6.5 TB/s for pages of 64 tokens, but a box takes
// about 120 cycles of the SM's unit however small it is, 414 us for 309 with pages of 16; and a fifth warp costs a fifth of
// the registers.)
//
// Fragments (g = lane / 4, t = lane % 4).  The order of keys within 16 is free: place i is key key_of(i), chosen so that
// neither the reads of K nor those of V, which ldmatrix transposes byte by byte, meet a bank twice.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "baps_attention_window.cuh"
#include "baps_kv_append.cuh"

namespace baps {

struct KvAttnParams {
    const void *q;
    void *out;
    float *lse;
    int64_t qs_b, qs_h, qs_t, os_b, os_h, os_t;
    const int32_t *table, *lengths;
    const uint8_t *k, *v;
    const float *k_scale, *v_scale;
    int width, B, H, Hkv, T, G, R, groups;      // G = H / Hkv, R = T * G rows per kv head, in `groups` groups of kRows
    int n_pages, page, window, sinks;           // window: up to width * page
    float c;
    // workspace: per CTA two partial results (rows x (D floats), divided by l), (m, l) of their rows, and which item they belong to
    float *part_o;
    float2 *part_ml;
    int2 *desc;                                  // (item, last CTA that has part of it); item -1: none begins here and goes on
};

constexpr int kKvTile = 64, kKvLogTile = 6, kKvStep = 32, kKvMaxB = 4096;
constexpr int kKvMinTiles = 2;                   // tiles that a CTA takes at least
constexpr int kKvMaxCluster = 8;                 // CTAs of a cluster at most

// kTiles: groups of eight rows that a CTA serves.
template <int D, int kTiles>
struct KvLayout {
    static constexpr int kWarps = 4, kThreads = 128, kRows = 8 * kTiles;
    static constexpr int kCtasPerSm = D == 64 && kTiles < 4 ? 3 : 2;
    static constexpr int kSlotBytes = 2 * kKvStep * D;                   // K and V of a step
    static constexpr int kSlots = D == 64 ? (kTiles == 2 ? 3 : 4) : 2;
    // Three slots and more: the slot that the step before was in is filled while this step's products run, else behind them.
    static constexpr bool kCopyFirst = kSlots > 2;
    static constexpr int kSlotOff = 0;                                   // [warp][slot]
    static constexpr int kJoinOff = kWarps * kSlots * kSlotBytes;        // [warp][kTiles][D / 8][lane] float2
    static constexpr int kMlOff = kJoinOff + kWarps * kTiles * 8 * D * 4;    // [warp][8 kTiles] (m, l)
    static constexpr int kQOff = kMlOff + kWarps * kTiles * 8 * 8;       // [kTiles][D / 16][lane] uint2
    static constexpr int kMetaOff = kQOff + kTiles * 8 * D * 2;          // [warp][slot] float4: k_scale, v_scale of both 16-key blocks
    static constexpr int kSeqOff = kMetaOff + kWarps * kSlots * 16;      // int len[B], pre[B + 1]
    static constexpr int dyn_bytes(int B) { return kSeqOff + (2 * B + 1) * 4; }
    static_assert(dyn_bytes(kKvMaxB) <= 227 * 1024, "shared memory of a CTA");
    static_assert(kCtasPerSm * (dyn_bytes(64) + 1024) <= 228 * 1024, "shared memory of an SM");
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// fp16 values of the two lower / upper codes of a word
__device__ __forceinline__ uint32_t widen_lo(uint32_t x)
{
    uint32_t d;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(d) : "r"(x));
    return d;
}
__device__ __forceinline__ uint32_t widen_hi(uint32_t x)
{
    uint32_t d;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n\t}" : "=r"(d) : "r"(x));
    return d;
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Two 16 x 16 matrices of bytes, transposed: r[2 m + h] of thread (g, t) is column 8 h + g, rows 4 t .. 4 t + 3 of matrix m.
__device__ __forceinline__ void ldmatrix_bytes(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const void *from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kMayBeOpen>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kMayBeOpen) : "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address in CTA `rank` of the cluster of what stands at addr in this one
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float4 cluster_f32x4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float2 cluster_f32x2(uint32_t addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}
// 8 x 8 matrix of 16-bit elements, transposed between the threads of a warp
__device__ __forceinline__ uint32_t transpose8(uint32_t x)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(x));
    return d;
}
// Key (0 .. 15) that stands at place i of a product over 16 keys.
__device__ __forceinline__ int key_of(int i)
{
    const int e0 = i & 1, e1 = (i >> 1) & 1, t0 = (i >> 2) & 1, t1 = i >> 3;
    return t1 << 3 | t0 << 2 | e0 << 1 | (t1 ^ e1);
}

// Positions that a sequence's queries see, as 64-key tiles.
__device__ __forceinline__ KeyTiles kv_tiles(int len, int T, int window, int sinks)
{
    const int last = max(len, 1) - 1;
    return key_tiles(min(max(len - T, 0), last), last, window, sinks, kKvLogTile);
}

// Where tile number w of all stands: sequence, kv head and row group, tile of that sequence.
struct KvPlace { int b, hr, i, n; };
__device__ __forceinline__ KvPlace kv_place(const int *pre, int B, int heads, int w)
{
    int lo = 0, hi = B - 1;                              // last b with pre[b] * heads <= w
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((int64_t)pre[mid] * heads <= w) lo = mid; else hi = mid - 1;
    }
    KvPlace a;
    a.b = lo;
    a.n = pre[lo + 1] - pre[lo];
    const int x = w - pre[lo] * heads;
    a.hr = x / a.n;
    a.i = x - a.hr * a.n;
    return a;
}

template <typename T16>
__device__ __forceinline__ T16 from_float(float x)
{
    if constexpr (__is_same(T16, __half)) return __float2half_rn(x); else return __float2bfloat16_rn(x);
}
__device__ __forceinline__ void kv_store_lse(const KvAttnParams &p, int b, int h, int tq, float m, float l)
{
    if (p.lse) p.lse[((int64_t)b * p.H + h) * p.T + tq] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}
__device__ __forceinline__ float kv_inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }     // (0: no key at all)
// Elements d0 .. d0 + 3 of an output row; d0 = 0 brings the lse along.
template <typename T16>
__device__ __forceinline__ void kv_store(const KvAttnParams &p, int b, int h, int tq, int d0, const float (&o)[4], float m, float l)
{
    *reinterpret_cast<uint2 *>(reinterpret_cast<T16 *>(p.out) + b * p.os_b + h * p.os_h + tq * p.os_t + d0) =
        make_uint2(pack16<T16>(o[0], o[1]), pack16<T16>(o[2], o[3]));
    if (d0 == 0) kv_store_lse(p, b, h, tq, m, l);
}

// kClusters: a cluster of CTAs takes one sequence and head and cuts its tiles evenly; its parts are joined through the CTAs'
// shared memory, in one launch and without a workspace.
template <typename T16, int D, int kTiles, bool kClusters>
__global__ void __launch_bounds__(KvLayout<D, kTiles>::kThreads, KvLayout<D, kTiles>::kCtasPerSm)
kv_attention_kernel(const KvAttnParams p)
{
    using namespace sm100;
    using L = KvLayout<D, kTiles>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sbase = smem_u32(smem);
    int *s_len = reinterpret_cast<int *>(smem + L::kSeqOff), *s_pre = s_len + p.B;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    allow_next_kernel();
    await_previous_kernel();
    const int heads = p.Hkv * p.groups;
    const int64_t most = (int64_t)p.width * p.page;
    int w0 = 0, w1 = 0, per = 1;
    int len_here = 0;                                                      // kClusters: of the one sequence
    KvPlace item{0, 0, 0, 0};
    if constexpr (kClusters) {
        const unsigned size = cluster_size(), rank = cluster_rank(), number = blockIdx.x / size;
        item.b = (int)(number / (unsigned)heads);
        item.hr = (int)(number % (unsigned)heads);
        len_here = (int)min((int64_t)max(p.lengths[item.b], 0), most);
        item.n = kv_tiles(len_here, p.T, p.window, p.sinks).count();
        item.i = (int)((int64_t)item.n * rank / size);
        w1 = (int)((int64_t)item.n * (rank + 1) / size) - item.i;
    } else {
        // ---- every CTA's share: tiles of each sequence, their running sum ---------------------------------
        for (int b = tid; b < p.B; b += L::kThreads) {
            const int len = (int)min((int64_t)max(p.lengths[b], 0), most);
            s_len[b] = len;
            s_pre[b + 1] = kv_tiles(len, p.T, p.window, p.sinks).count();
        }
        if (tid == 0) s_pre[0] = 0;
        __syncthreads();
        if (warp == 0) {
            int sum = 0;
            for (int b0 = 0; b0 < p.B; b0 += 32) {
                int x = b0 + lane < p.B ? s_pre[b0 + lane + 1] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, x, o);
                    if (lane >= o) x += y;
                }
                if (b0 + lane < p.B) s_pre[b0 + lane + 1] = sum + x;
                sum += __shfl_sync(0xffffffffu, x, 31);
            }
        }
        __syncthreads();
        const int total = s_pre[p.B] * heads;                              // (fits: checked on the host)
        per = max((total + (int)gridDim.x - 1) / (int)gridDim.x, kKvMinTiles);
        w0 = (int)min((int64_t)blockIdx.x * per, (int64_t)total);
        w1 = (int)min((int64_t)w0 + per, (int64_t)total);
        if (tid == 0) p.desc[blockIdx.x] = make_int2(-1, 0);
        if (w0 >= w1) return;
    }
    auto place_of = [&](int w) -> KvPlace {
        if constexpr (kClusters) return KvPlace{item.b, item.hr, item.i + w, item.n};
        else return kv_place(s_pre, p.B, heads, w);
    };
    auto len_of = [&](int b) { return kClusters ? len_here : s_len[b]; };

    // ---- the warp's steps: number k is half (u & 1) of tile w0 + (u >> 1), u = warp + 4 k ---------------
    // What lane l knows of step k0 + l, 32 steps at a time, the next 32 on their way: rows of the pool's [n_pages * Hkv * page, D]
    // view where its two 16-key blocks begin (-1: no page, or no key that a query sees), their scales.
    struct Ahead { int row_a, row_b; float ka, va, kb, vb; };
    const int steps = w1 - w0 > warp / 2 ? (2 * (w1 - w0) - warp + 3) / 4 : 0;
    auto fetch = [&](int k0) {
        Ahead x{-1, -1, -1.f, 0.f, -1.f, 0.f};
        const int k = k0 + lane;
        if (k < steps) {
            const int u = warp + 4 * k;
            const KvPlace a = place_of(w0 + (u >> 1));
            const int len = len_of(a.b), first = max(len - p.T, 0), hk = a.hr / p.groups;
            const int pos = kv_tiles(len, p.T, p.window, p.sinks).tile(a.i) * kKvTile + (u & 1) * kKvStep;
            auto block = [&](int at, int &row, float &ks, float &vs) {
                if (at >= len || !(at + 15 > first - p.window || at < p.sinks)) return;
                const int id = p.table[(int64_t)a.b * p.width + at / p.page];
                if (id < 0 || id >= p.n_pages) return;
                const int64_t ph = (int64_t)id * p.Hkv + hk;
                row = (int)(ph * p.page + at % p.page);
                ks = p.k_scale[ph];
                vs = p.v_scale[ph];
            };
            block(pos, x.row_a, x.ka, x.va);
            block(pos + 16, x.row_b, x.kb, x.vb);
        }
        return x;
    };
    const uint32_t slots = sbase + L::kSlotOff + (uint32_t)(warp * L::kSlots * L::kSlotBytes);
    const uint32_t metas = sbase + L::kMetaOff + (uint32_t)(warp * L::kSlots * 16);
    // byte offset of 16-byte part `part` of row `row`: parts of neighbouring rows change places, so that eight rows' parts
    // of one number stand in different banks
    auto place = [](int row, int part) { return (uint32_t)(row * D + ((part ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4)); };
    constexpr int kParts = D / 16, kRowsAtOnce = 32 / kParts;
    const int c_row = lane / kParts, c_part = lane % kParts;
    Ahead now = fetch(0), next = steps > 32 ? fetch(32) : now;
    int next_k = 0, next_slot = 0;                                       // the step to be copied next, and where to
    auto copy_step = [&] {
        if (next_k < steps) {
            if (next_k > 0 && (next_k & 31) == 0) { now = next; next = next_k + 32 < steps ? fetch(next_k + 32) : now; }
            const int row_a = __shfl_sync(0xffffffffu, now.row_a, next_k & 31), row_b = __shfl_sync(0xffffffffu, now.row_b, next_k & 31);
            const uint32_t to = slots + (uint32_t)(next_slot * L::kSlotBytes);
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                const int row = blk ? row_b : row_a;
                if (row < 0) continue;
                const int64_t from = (int64_t)(row + c_row) * D + c_part * 16;
                const uint8_t *k = p.k + from, *v = p.v + from;
#pragma unroll
                for (int r0 = 0; r0 < 16; r0 += kRowsAtOnce) {
                    const uint32_t at = to + place(16 * blk + r0 + c_row, c_part);
                    copy16(at, k + r0 * D);
                    copy16(at + kKvStep * D, v + r0 * D);
                }
            }
            float4 scales;                                               // k_scale -1: no such block
            scales.x = __shfl_sync(0xffffffffu, now.ka, next_k & 31); scales.y = __shfl_sync(0xffffffffu, now.va, next_k & 31);
            scales.z = __shfl_sync(0xffffffffu, now.kb, next_k & 31); scales.w = __shfl_sync(0xffffffffu, now.vb, next_k & 31);
            if (lane == 0) sts_f32x4(metas + 16u * (uint32_t)next_slot, scales);
        }
        copies_commit();                                                 // (a group for every step, also behind the last)
        ++next_k;
        next_slot = next_slot + 1 < L::kSlots ? next_slot + 1 : 0;
    };
    for (int i = 0; i < L::kSlots - (L::kCopyFirst ? 1 : 0); ++i) copy_step();

    const int g = lane >> 2, t = lane & 3;
    // What this lane addresses of the first 16 keys of a step (the second 16 and other parts: plus 16 rows, exclusive or, which
    // the order of parts lets through).  K: places of product rows 0 .. 7 and 8 .. 15, parts 0 and 1.  V: place lane % 16 of
    // the first (lanes 0 .. 15) or second 16 keys.
    const uint32_t k_at = place(key_of(4 * ((lane & 7) >> 1) + 2 * (lane >> 3 & 1) + (lane & 1)), lane >> 4);
    const uint32_t v_at = kKvStep * D + place(16 * (lane >> 4) + key_of(lane & 15), 0);
    // the thread's keys of each 16: of the scores (product rows g, g + 8), of V (places 4 t .. 4 t + 3)
    const int s_key[2] = {key_of(4 * (g >> 1) + (g & 1)), key_of(4 * (g >> 1) + 2 + (g & 1))};
    const uint32_t q_at = sbase + L::kQOff + (uint32_t)(lane * 8);

    int step = 0, slot = 0;
    for (int w = w0; kClusters || w < w1;) {
        const KvPlace a = place_of(w);
        const int tiles = min(a.n - a.i, w1 - w);
        const int len = len_of(a.b), hk = a.hr / p.groups, row_base = (a.hr % p.groups) * L::kRows;
        const KeyTiles kt = kv_tiles(len, p.T, p.window, p.sinks);
        const int q_first = len - p.T;                                   // position of query 0, maybe below 0
        const int steps_here = 2 * (w + tiles - w0);                     // u below this: of this sequence and head

        // ---- the rows of q: row r is query r % T of head r / T of the group ------------------------------------
        float cq[kTiles][2], m[kTiles][2], l[kTiles][2];                 // of rows 2 t, 2 t + 1
        int pos[kTiles][2];                                              // their positions; below 0: sees nothing
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt) {
            const int r = row_base + 8 * qt + g;
            const bool there = r < p.R;
            const int tq = r % p.T;
            float x[D / 4], big = 0.f;
            const T16 *src = reinterpret_cast<const T16 *>(p.q) + a.b * p.qs_b + (hk * p.G + r / p.T) * p.qs_h + tq * p.qs_t + 4 * t;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                uint2 u = make_uint2(0, 0);
                if (there) u = *reinterpret_cast<const uint2 *>(src + 16 * i);
                const float2 f0 = values2<T16>(u.x), f1 = values2<T16>(u.y);
                x[4 * i] = f0.x; x[4 * i + 1] = f0.y; x[4 * i + 2] = f1.x; x[4 * i + 3] = f1.y;
#pragma unroll
                for (int k = 0; k < 4; ++k) big = fmaxf(big, fabsf(x[4 * i + k]));
            }
            float scale = 1.f, back = p.c;
            if constexpr (!__is_same(T16, __half)) {                     // largest element of the row to [1, 2)
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                const uint32_t e = min(max(__float_as_uint(big) >> 23, 1u), 253u);
                scale = __uint_as_float((254u - e) << 23);
                back *= __uint_as_float(e << 23);
            }
            // elements 16 i + 4 t .. + 3 of row g (all four warps write the same)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                sts_u32x2(q_at + (uint32_t)((qt * (D / 16) + i) * 256), pack16<__half>(x[4 * i] * scale, x[4 * i + 1] * scale),
                          pack16<__half>(x[4 * i + 2] * scale, x[4 * i + 3] * scale));
            const int here = there ? q_first + tq : -1;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                cq[qt][e] = __shfl_sync(0xffffffffu, back, 4 * (2 * t + e));
                pos[qt][e] = __shfl_sync(0xffffffffu, here, 4 * (2 * t + e));
                m[qt][e] = -INFINITY;
                l[qt][e] = 0.f;
            }
        }
        __syncwarp();
        float o[kTiles][D / 16][4];                                      // elements 16 i + g, + 8 of rows 2 t, 2 t + 1
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) o[qt][i][k] = 0.f;
        float unit = 0.f, inv_unit = 0.f;                                // value scale that O~ is in units of; 0: none yet
        float unit_most = 0.f;                                           // the largest that it has been
        auto times = [&](int qt, float f0, float f1) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) { o[qt][i][0] *= f0; o[qt][i][1] *= f1; o[qt][i][2] *= f0; o[qt][i][3] *= f1; }
        };
        auto to_unit = [&](float next) {
            inv_unit = pow2_inverse(next);
            const float f = unit * inv_unit;
#pragma unroll
            for (int qt = 0; qt < kTiles; ++qt) times(qt, f, f);
            unit = next;
        };

        for (; warp + 4 * step < steps_here; ++step) {
            copies_wait<L::kSlots - (L::kCopyFirst ? 2 : 1)>();
            __syncwarp();                                                // what the other lanes copied is there too
            if constexpr (L::kCopyFirst) copy_step();
            const int u = warp + 4 * step;
            const int c0 = kt.tile(a.i + (w0 + (u >> 1) - w)) * kKvTile + (u & 1) * kKvStep;
            // every query sees every key of the step
            const bool all = c0 + kKvStep - 1 <= q_first && (c0 > len - 1 - p.window || c0 + kKvStep - 1 < p.sinks);
            const uint32_t base = slots + (uint32_t)(slot * L::kSlotBytes);
            const float4 scales = lds_f32x4(metas + 16u * (uint32_t)slot);
            const float2 sa = make_float2(scales.x, scales.y), sb = make_float2(scales.z, scales.w);
            const bool gone_a = sa.x == -1.f, gone_b = sb.x == -1.f;
            if (!(gone_a && gone_b)) {
                // ---- scores: sc[qt][block]: keys s_key[0] (rows 2 t, 2 t + 1), s_key[1] ------------------------
                float sc[kTiles][2][4];
#pragma unroll
                for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
                    for (int k = 0; k < 8; ++k) sc[qt][k >> 2][k & 3] = 0.f;
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    uint2 q[kTiles][2];
#pragma unroll
                    for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) q[qt][e] = lds_u32x2(q_at + (uint32_t)((qt * (D / 16) + 2 * j + e) * 256));
#pragma unroll
                    for (int blk = 0; blk < 2; ++blk) {
                        uint32_t u[4];                                   // parts 2 j (rows g, g + 8), 2 j + 1
                        ldmatrix4(u, base + ((k_at + blk * 16 * D) ^ (uint32_t)(32 * j)));
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t k16[4] = {widen_lo(u[2 * e]), widen_lo(u[2 * e + 1]), widen_hi(u[2 * e]), widen_hi(u[2 * e + 1])};
#pragma unroll
                            for (int qt = 0; qt < kTiles; ++qt) mma_f16(sc[qt][blk], k16, q[qt][e].x, q[qt][e].y);
                        }
                    }
                }
                const bool part = !all || gone_a || gone_b;
                uint32_t keep[2] = {0xffffffffu, 0xffffffffu};           // bytes of V whose keys some query sees
                if (part) {
#pragma unroll
                    for (int blk = 0; blk < 2; ++blk) {
                        const bool gone = blk ? gone_b : gone_a;
#pragma unroll
                        for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const int j = c0 + 16 * blk + s_key[k >> 1], at_pos = pos[qt][k & 1];
                                if (gone || !sees(at_pos, j, p.window, p.sinks)) sc[qt][blk][k] = -INFINITY;
                            }
                        keep[blk] = 0u;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int j = c0 + 16 * blk + key_of(4 * t + k);
                            if (!gone && j < len && (j > max(q_first, 0) - p.window || j < p.sinks)) keep[blk] |= 0xffu << (8 * k);
                        }
                    }
                }
                // ---- running reference; scores in base 2 are sc * f (f above 0, so that a hidden one stays -infinity) --
                float mx[kTiles][2], f[kTiles][2][2];
                bool rises = false;
#pragma unroll
                for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        f[qt][e][0] = fmaxf(cq[qt][e] * sa.x, 1.17549435e-38f);
                        f[qt][e][1] = fmaxf(cq[qt][e] * sb.x, 1.17549435e-38f);
                        mx[qt][e] = fmaxf(fmaxf(sc[qt][0][e], sc[qt][0][2 + e]) * f[qt][e][0], fmaxf(sc[qt][1][e], sc[qt][1][2 + e]) * f[qt][e][1]);
                        rises |= mx[qt][e] > m[qt][e] + 14.f;
                    }
                if (__any_sync(0xffffffffu, rises)) {
#pragma unroll
                    for (int qt = 0; qt < kTiles; ++qt) {
                        float back[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = mx[qt][e];
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
                            const float m_new = fmaxf(m[qt][e], top - 6.f);
                            back[e] = m[qt][e] == -INFINITY ? 1.f : ex2_approx(m[qt][e] - m_new);
                            m[qt][e] = m_new;
                            l[qt][e] *= back[e];
                        }
                        times(qt, back[0], back[1]);
                    }
                }
                // ---- the unit of O~ ----------------------------------------------------------------------------
                const float va = gone_a ? sb.y : sa.y, vb = gone_b ? sa.y : sb.y;
                const float v_most = fmaxf(va, vb), v_least = fminf(va, vb);
                if (!(v_most <= unit && v_least * 64.f >= unit)) {
                    if (unit == 0.f) { unit = v_most; inv_unit = pow2_inverse(unit); }
                    else if (v_most > unit_most * 5.421010862427522e-20f) to_unit(v_most);   // 2^-64; below, it does not count
                    unit_most = fmaxf(unit_most, unit);
                }
                // ---- weights ---------------------------------------------------------------------------------------
#pragma unroll
                for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float mu = m[qt][e] == -INFINITY ? 0.f : m[qt][e];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            float &x = sc[qt][k >> 1][2 * (k & 1) + e];
                            x = ex2_approx(fmaf(x, f[qt][e][k >> 1], -mu));
                            l[qt][e] += x;
                        }
                    }
                // ---- O~ += P V: at once, or one block after the other where their scales are far apart -----------
                const bool apart = v_least * 64.f < unit && va != vb;
#pragma unroll 1
                for (int pass = 0; pass < (apart ? 2 : 1); ++pass) {
                    float fa = va * inv_unit, fb = vb * inv_unit;        // powers of two up to 1
                    if (apart) {
                        const float mine = pass ? vb : va;
                        if (mine > unit_most * 5.421010862427522e-20f && mine != unit) to_unit(mine);
                        fa = pass ? 0.f : mine * inv_unit;
                        fb = pass ? mine * inv_unit : 0.f;
                    }
                    uint32_t pb[kTiles][2][2];                           // per block: places 0 .. 7, 8 .. 15 of row g
#pragma unroll
                    for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
                        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                            for (int k = 0; k < 2; ++k)
                                pb[qt][blk][k] = transpose8(pack16<__half>(sc[qt][blk][2 * k] * (blk ? fb : fa), sc[qt][blk][2 * k + 1] * (blk ? fb : fa)));
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t u[4];                                   // per block: elements 16 c + g, 16 c + 8 + g
                        ldmatrix_bytes(u, base + (v_at ^ (uint32_t)(16 * c)));
                        if (part) { u[0] &= keep[0]; u[1] &= keep[0]; u[2] &= keep[1]; u[3] &= keep[1]; }
#pragma unroll
                        for (int blk = 0; blk < 2; ++blk) {
                            const uint32_t v16[4] = {widen_lo(u[2 * blk]), widen_lo(u[2 * blk + 1]), widen_hi(u[2 * blk]), widen_hi(u[2 * blk + 1])};
#pragma unroll
                            for (int qt = 0; qt < kTiles; ++qt) mma_f16(o[qt][c], v16, pb[qt][blk][0], pb[qt][blk][1]);
                        }
                    }
                }
            }
            __syncwarp();                                                // every lane has read the slot
            if constexpr (!L::kCopyFirst) copy_step();
            slot = slot + 1 < L::kSlots ? slot + 1 : 0;
        }

        // ---- join the warps that share these rows ----------------------------------------------------------
        float2 *join = reinterpret_cast<float2 *>(smem + L::kJoinOff);
        float2 *ml = reinterpret_cast<float2 *>(smem + L::kMlOff);
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l[qt][e] += __shfl_xor_sync(0xffffffffu, l[qt][e], x);
                if (g == 0) ml[warp * 8 * kTiles + 8 * qt + 2 * t + e] = make_float2(m[qt][e], l[qt][e]);
            }
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt) {
            const float inv0 = kv_inverse(l[qt][0]), inv1 = kv_inverse(l[qt][1]);
#pragma unroll
            for (int k = 0; k < D / 8; ++k)                              // element 8 k + g of rows 2 t, 2 t + 1
                join[((warp * kTiles + qt) * (D / 8) + k) * 32 + lane] =
                    make_float2(o[qt][k >> 1][2 * (k & 1)] * inv0 * unit, o[qt][k >> 1][2 * (k & 1) + 1] * inv1 * unit);
        }
        __syncthreads();
        const bool whole = tiles == a.n;
        // Each warp joins every fourth of the (rows, 8 elements) entries, a thread what its own lane wrote: element 8 k + g of
        // rows 2 t, 2 t + 1 (no two lanes in a bank; read by output row, 16 at a time met in one and the join took 3700 cycles)
#pragma unroll
        for (int qt = 0; qt < kTiles; ++qt) {
            float M[2], Lsum[2], f[2][L::kWarps];
            int64_t to[2];                                               // first element of the row, wherever it goes
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int rr = 8 * qt + 2 * t + e, r = row_base + rr;
                M[e] = -INFINITY;
                Lsum[e] = 0.f;
#pragma unroll
                for (int y = 0; y < L::kWarps; ++y) M[e] = fmaxf(M[e], ml[y * 8 * kTiles + rr].x);
                const float Mu = M[e] == -INFINITY ? 0.f : M[e];
#pragma unroll
                for (int y = 0; y < L::kWarps; ++y) {
                    const float2 own = ml[y * 8 * kTiles + rr];
                    f[e][y] = ex2_approx(own.x - Mu) * own.y;
                    Lsum[e] += f[e][y];
                }
                const float inv = kv_inverse(Lsum[e]);
#pragma unroll
                for (int y = 0; y < L::kWarps; ++y) f[e][y] *= inv;
                if (kClusters) {
                    to[e] = rr * D;
                } else if (whole) {
                    to[e] = a.b * p.os_b + (hk * p.G + r / p.T) * p.os_h + r % p.T * p.os_t;
                } else {
                    to[e] = ((int64_t)(2 * blockIdx.x + (a.i == 0 ? 1 : 0)) * L::kRows + rr) * D;
                }
                if (r >= p.R) to[e] = -1;
                if (warp == 0 && g == 0 && r < p.R) {
                    if (kClusters) *reinterpret_cast<float2 *>(smem + L::kRows * D * 4 + rr * 8) = make_float2(M[e], Lsum[e]);
                    else if (whole) kv_store_lse(p, a.b, hk * p.G + r / p.T, r % p.T, M[e], Lsum[e]);
                    else p.part_ml[to[e] / D] = make_float2(M[e], Lsum[e]);
                }
            }
            for (int k = warp; k < D / 8; k += L::kWarps) {
                float acc[2] = {0.f, 0.f};
#pragma unroll
                for (int y = 0; y < L::kWarps; ++y) {
                    const float2 u = join[((y * kTiles + qt) * (D / 8) + k) * 32 + lane];
                    acc[0] += f[0][y] * u.x;
                    acc[1] += f[1][y] * u.y;
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    if (to[e] < 0) continue;
                    const int64_t at = to[e] + 8 * k + g;
                    if (kClusters) reinterpret_cast<float *>(smem)[at] = acc[e];     // over the slots, which every warp is done with
                    else if (whole) reinterpret_cast<T16 *>(p.out)[at] = from_float<T16>(acc[e]);
                    else p.part_o[at] = acc[e];
                }
            }
        }
        if constexpr (kClusters) {
            const int size = (int)cluster_size();
            cluster_sync();
            for (int x = (int)cluster_rank() * L::kThreads + tid; x < 8 * kTiles * (D / 4); x += size * L::kThreads) {
                const int rr = x / (D / 4), d0 = x % (D / 4) * 4, r = row_base + rr;
                if (r >= p.R) continue;
                float M = -INFINITY, Lsum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
                const uint32_t o_at = sbase + (uint32_t)((rr * D + d0) * 4), ml_at = sbase + (uint32_t)(L::kRows * D * 4 + rr * 8);
                float2 own[kKvMaxCluster];
                float4 u[kKvMaxCluster];
#pragma unroll
                for (int y = 0; y < kKvMaxCluster; ++y) {                // (all on their way together)
                    own[y] = make_float2(-INFINITY, 0.f);
                    u[y] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (y < size) { own[y] = cluster_f32x2(cluster_addr(ml_at, y)); u[y] = cluster_f32x4(cluster_addr(o_at, y)); }
                }
#pragma unroll
                for (int y = 0; y < kKvMaxCluster; ++y) M = fmaxf(M, own[y].x);
                const float Mu = M == -INFINITY ? 0.f : M;
#pragma unroll
                for (int y = 0; y < kKvMaxCluster; ++y) Lsum += own[y].y *= ex2_approx(own[y].x - Mu);
                const float inv = kv_inverse(Lsum);
#pragma unroll
                for (int y = 0; y < kKvMaxCluster; ++y) {
                    const float f = own[y].y * inv;
                    acc[0] += f * u[y].x; acc[1] += f * u[y].y; acc[2] += f * u[y].z; acc[3] += f * u[y].w;
                }
                kv_store<T16>(p, a.b, hk * p.G + r / p.T, r % p.T, d0, acc, M, Lsum);
            }
            cluster_sync();                                              // what other CTAs read stays until they have
            return;
        }
        if (tid == 0 && a.i == 0 && !whole) p.desc[blockIdx.x] = make_int2(a.b * heads + a.hr, (w + a.n - 1) / per);
        __syncthreads();                                                 // before the buffers, and q, are written again
        w += tiles;
    }
}

// Joins the parts of the item that begins in CTA blockIdx.x of the kernel above and ends in a later one, in the order of
// the CTAs.  Blocks (CTA, rows); D / 4 threads per row and part, four elements each; 512 / D of those, for as many parts of one
// row (kRows = 8), or two parts and more rows.  The loads of the parts' O~ do not wait for their maxima, so that a block takes
// three round trips to memory, whatever the number of parts up to kEach * kSide.
template <int D, int kRows>
struct JoinShape {
    static constexpr int kLanes = D / 4, kSide = kRows == 8 ? 128 / kLanes : 2, kRowsHere = 128 / kLanes / kSide, kEach = 4;
};
template <typename T16, int D, int kRows>
__global__ void __launch_bounds__(128)
kv_join_kernel(const KvAttnParams p)
{
    using J = JoinShape<D, kRows>;
    constexpr int kLanes = J::kLanes, kSide = J::kSide, kEach = J::kEach;
    __shared__ float s_o[J::kRowsHere][kSide][kLanes][6];
    allow_next_kernel();
    await_previous_kernel();
    const int2 what = p.desc[blockIdx.x];
    if (what.x < 0) return;
    const int x = threadIdx.x % kLanes, side = threadIdx.x / kLanes % kSide, sub = threadIdx.x / (kLanes * kSide);
    const int heads = p.Hkv * p.groups, hr = what.x % heads, rr = blockIdx.y * J::kRowsHere + sub;
    const int r = hr % p.groups * kRows + rr;
    const bool there = r < p.R;
    const int parts = what.y - (int)blockIdx.x + 1;
    auto row = [&](int k) { return (int64_t)(2 * ((int)blockIdx.x + k) + (k == 0 ? 1 : 0)) * kRows + rr; };
    // each side its own parts against their own maximum, then the sides together; acc: O, l
    float m = -INFINITY, acc[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; there && k0 < parts; k0 += kEach * kSide) {
        float4 u[kEach];
        float2 ml[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int k = k0 + i * kSide + side;
            u[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            ml[i] = make_float2(-INFINITY, 0.f);
            if (k < parts) {
                u[i] = *reinterpret_cast<const float4 *>(p.part_o + row(k) * D + 4 * x);
                ml[i] = p.part_ml[row(k)];
            }
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < kEach; ++i) top = fmaxf(top, ml[i].x);
        const float mu = top == -INFINITY ? 0.f : top;
        float back = ex2_approx(m - mu) * acc[4];
        acc[4] = back;
#pragma unroll
        for (int i = 0; i < kEach; ++i) acc[4] += ml[i].y *= ex2_approx(ml[i].x - mu);
        const float inv = kv_inverse(acc[4]);
        back *= inv;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= back;
        m = top;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const float f = ml[i].y * inv;
            acc[0] += f * u[i].x; acc[1] += f * u[i].y; acc[2] += f * u[i].z; acc[3] += f * u[i].w;
        }
    }
#pragma unroll
    for (int e = 0; e < 5; ++e) s_o[sub][side][x][e] = acc[e];
    s_o[sub][side][x][5] = m;
    __syncthreads();
    if (side > 0 || !there) return;
    float all = m;
#pragma unroll
    for (int k = 1; k < kSide; ++k) all = fmaxf(all, s_o[sub][k][x][5]);
    const float mu = all == -INFINITY ? 0.f : all;
    float f[kSide], l = 0.f;
#pragma unroll
    for (int k = 0; k < kSide; ++k) l += f[k] = ex2_approx(s_o[sub][k][x][5] - mu) * s_o[sub][k][x][4];
    const float inv = kv_inverse(l);
    float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kSide; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += f[k] * inv * s_o[sub][k][x][e];
    kv_store<T16>(p, what.x / heads, hr / p.groups * p.G + r / p.T, r % p.T, 4 * x, o, all, l);
}

// Rows of a kv head go to a CTA 8 or 16 (D = 64: up to 32) at a time, as many as its registers hold; more are items of their own,
// which CTAs work on at about the same time, so that most of what they read again comes from L2.
// Sequences and kv heads ("items") that are short, or cut to one length by a window, go to a cluster of up to eight CTAs each,
// as many as still run all at the same time, or to one CTA: one launch, nothing to join through memory, no CTA with two items.
// That is taken where a CTA gets few enough tiles for it (most_tiles: what an item can have, by the table's width and the window):
//   24 for an item to itself, 16 in a cluster, 36 where the window sets the length and the clusters fill four fifths of the machine.
// Measured against the even cut, us (clusters first, 32 / 8 heads of 128, lengths from a quarter of the longest unless said):
//   an item to itself: 30 sequences of up to 1536 tokens (24 tiles) 16.8, 22.2, 75 of them 37.2, 47.1; beyond the line still, 30 of 2048 21.5, 26.0, of
//   3000 29.5, 30.3;
//   clusters of eight: one sequence of 2000 6.5, 10.1, of 4000 8.2, 11.2, of 8192 (16 tiles) 11.2, 10.1; two of 8192 12.5, 14.2, four 13.2, 16.2; beyond,
//   one of 12000 14.3, 13.0, of 16000 17.8, 14.5, four of 12000 17.0, 17.5;
//   where a window of 4096 sets the length, 16 / 4 heads: 32 sequences (clusters of two, 35 tiles) 27.3, 32.3, 37 of them 29.8, 35.5; 20 (of three) 16.7, 21.1; 16 (of
//   four) 14.3, 18.9; four queries each and heads of 64 (of three) 20.2, 25.9; short of the line, 25 sequences (200 of 296 places) 23.3, 25.2; beyond,
//   window 5000 31.5, 36.3.  So the lines are on the even cut's side by up to a fifth, but for one sequence alone, which loses a tenth at 8192.
struct KvShape { int tiles, groups, ctas, cluster; };
static inline KvShape kv_shape(int R, int D, int64_t items, int64_t most_tiles, bool by_window)
{
    KvShape s;
    s.tiles = R <= 8 ? 1 : R <= 16 || D == 128 ? 2 : 4;
    s.groups = (R + 8 * s.tiles - 1) / (8 * s.tiles);
    s.ctas = num_sms() * (D == 64 && s.tiles < 4 ? 3 : 2);
    s.cluster = 0;
    items *= s.groups;
    for (int c = 1; c <= kKvMaxCluster; ++c) {
        const int64_t each = (most_tiles + c - 1) / c;
        const bool fits = items * c <= s.ctas, full = fits && 5 * items * c >= 4 * s.ctas;
        if (c == 1 ? each <= 24 : fits && (each <= 16 || (by_window && full && each <= 36))) s.cluster = c;
    }
    return s;
}
// Tiles that a sequence can have by its row of the table, and by the window.
static inline int64_t kv_held_tiles(int page, int table_width) { return ((int64_t)table_width * page + kKvTile - 1) / kKvTile; }
static inline int64_t kv_seen_tiles(int T, int window, int sinks) { return ((int64_t)window + T) / kKvTile + sinks / kKvTile + 4; }
static inline KvShape kv_shape_of(int B, int Hkv, int R, int D, int page, int table_width, int T, int window, int sinks)
{
    const int64_t held = kv_held_tiles(page, table_width), seen = kv_seen_tiles(T, window, sinks);
    return kv_shape(R, D, (int64_t)B * Hkv, held < seen ? held : seen, seen < held);
}
// Bytes: part_o, part_ml, desc
static inline size_t kv_workspace(const KvShape &s, int D)
{
    if (s.cluster) return 0;
    const size_t rows = (size_t)s.ctas * 2 * 8 * s.tiles;
    return rows * D * 4 + rows * 8 + (size_t)s.ctas * 8;
}

template <typename T16, int D, int kTiles>
static inline baps_status kv_attention_launch(const KvAttnParams &p, const KvShape &shape, cudaStream_t stream)
{
    using L = KvLayout<D, kTiles>;
    if (shape.cluster) {
        const size_t smem = (size_t)L::dyn_bytes(0);
        if (cudaFuncSetAttribute(kv_attention_kernel<T16, D, kTiles, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess)
            return BAPS_ERR_CUDA;
        return launch_clusters(kv_attention_kernel<T16, D, kTiles, true>, (unsigned)(p.B * p.Hkv * p.groups * shape.cluster),
                               (unsigned)shape.cluster, L::kThreads, smem, stream, p);
    }
    if (cudaFuncSetAttribute(kv_attention_kernel<T16, D, kTiles, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             L::dyn_bytes(kKvMaxB)) != cudaSuccess)
        return BAPS_ERR_CUDA;
    const baps_status s = launch_kernel(kv_attention_kernel<T16, D, kTiles, false>, (unsigned)shape.ctas, L::kThreads,
                                        (size_t)L::dyn_bytes(p.B), stream, p);
    if (s != BAPS_OK) return s;
    const int rows = p.R < L::kRows ? p.R : L::kRows, at_once = JoinShape<D, L::kRows>::kRowsHere;
    return launch_kernel(kv_join_kernel<T16, D, L::kRows>, dim3((unsigned)shape.ctas, (unsigned)((rows + at_once - 1) / at_once)), 128, 0, stream, p);
}

template <typename T16>
static inline baps_status kv_attention_shape(const KvAttnParams &p, int D, const KvShape &s, cudaStream_t stream)
{
    if (D == 128) return s.tiles == 1 ? kv_attention_launch<T16, 128, 1>(p, s, stream) : kv_attention_launch<T16, 128, 2>(p, s, stream);
    if (s.tiles == 4) return kv_attention_launch<T16, 64, 4>(p, s, stream);
    return s.tiles == 1 ? kv_attention_launch<T16, 64, 1>(p, s, stream) : kv_attention_launch<T16, 64, 2>(p, s, stream);
}

} // namespace baps
