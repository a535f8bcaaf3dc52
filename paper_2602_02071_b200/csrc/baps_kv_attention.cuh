// Attention of the last T tokens of every sequence over the 8-bit cache.
//
//     s = c * k_scale * (q . k_code),  w = 2^(s - m),  l = sum w,  O~ = sum w * v_scale * v_code;   O = O~ / l
// with c = log2(e) * scale and a running maximum m that moves only when a score passes it by more than 8.  Codes become
// fp16 in registers (exactly: E4M3 has 4 significant bits), q is scaled by a power of two per row so that its 8 or 11 bits
// fit fp16 (what is lost is below 2^-24 of the row's largest element), and both products run on fp16 mma.sync
// with float32 accumulation; the weights are rounded to fp16 (half a step, 2^-12) after they have been summed.  The two
// scales are applied in float32, v_scale by keeping O~ in units of the page's scale.
//
// What bounds it: the bytes of K and V, one per element.  mma.sync, not tcgen05, because the codes have to be widened in
// registers on the way, and because 16 rows of queries (T * H / Hkv) are all there is: the products need a third of what
// mma.sync gives at full memory rate.
//
// Work is cut evenly whatever the lengths: the 64-key tiles of all sequences and kv heads, visible ones only, in one row;
// CTA i takes an equal share.  What a CTA does of a sequence and head that is not whole goes to the workspace and a
// second kernel joins it, in the order of the CTAs.  A tile is loaded by TMA, page by page, into a ring of stages; each
// consumer warp takes 16-key steps of it for 16 rows and keeps m, l and O~ in registers, and the warps are joined
// through shared memory where a sequence and head ends.
//
// Fragments (mma m16n8k16; g = lane / 4, t = lane % 4).  The order of the head's elements within a product and that of keys
// within a step are free, so a thread takes whole 16-byte pieces: of K row(g) elements 16 t .. 16 t + 15 of each 64, of V
// rows row(2 t), row(2 t + 1) elements g D / 8 .. + D / 8 - 1.  row() is chosen so that neither read of the swizzled tile
// meets a bank twice.
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
    const float *k_scale, *v_scale;
    int width, B, H, Hkv, T, G, R, groups;      // G = H / Hkv, R = T * G rows per kv head, in `groups` groups of kRows
    int n_pages, page, window, sinks;
    float c;
    // workspace: per CTA two partial results (rows x (D floats)), (m, l) of their rows, and which item they belong to
    float *part_o;
    float2 *part_ml;
    int2 *desc;                                  // (item, last CTA that has part of it); item -1: none begins here and goes on
};

constexpr int kKvTile = 64, kKvLogTile = 6, kKvMaxB = 4096;
constexpr int kKvMinTiles = 2;                   // tiles that a CTA takes at least

template <int D, int kChunks, int kKeyGroups>
struct KvLayout {
    static constexpr int kWarps = kChunks * kKeyGroups, kRows = 16 * kChunks, kThreads = kWarps * 32 + 32;
    static constexpr int kCtasPerSm = kWarps == 4 ? 2 : 1;
    static constexpr int kTileBytes = kKvTile * D;                       // of K, and of V
    static constexpr int kStages = (kCtasPerSm == 2 ? 64 : 128) * 1024 / (2 * kTileBytes);
    static constexpr int kRingOff = 0;
    static constexpr int kJoinOff = kStages * 2 * kTileBytes;            // [warp][D / 8][lane] float4
    static constexpr int kMlOff = kJoinOff + kWarps * 16 * D * 4;        // [warp][16] (m, l)
    static constexpr int kMetaOff = kMlOff + kWarps * 16 * 8;            // [stage][4] (k_scale, v_scale)
    static constexpr int kBarOff = kMetaOff + kStages * 4 * 8;
    static constexpr int kMiscOff = kBarOff + 2 * kStages * 8;
    static constexpr int kSeqOff = kMiscOff + 16;                        // int len[B], pre[B + 1]
    static int dyn_bytes(int B) { return kSeqOff + (2 * B + 1) * 4 + 1024; }
};

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// fp16 values of the two codes in the lower / upper half of a word
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
__device__ __forceinline__ float to_float(T16 x)
{
    if constexpr (__is_same(T16, __half)) return __half2float(x); else return __bfloat162float(x);
}

// Elements d0 .. d0 + 3 of an output row from O~ and l (against the maximum m); d0 = 0 brings the lse along.
template <typename T16>
__device__ __forceinline__ void kv_store(const KvAttnParams &p, int b, int h, int tq, int d0, float4 o, float m, float l)
{
    const float inv = l == 0.f ? 0.f : 1.f / l;
    *reinterpret_cast<uint2 *>(reinterpret_cast<T16 *>(p.out) + b * p.os_b + h * p.os_h + tq * p.os_t + d0) =
        make_uint2(pack16<T16>(o.x * inv, o.y * inv), pack16<T16>(o.z * inv, o.w * inv));
    if (d0 == 0 && p.lse)
        p.lse[((int64_t)b * p.H + h) * p.T + tq] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
}

template <typename T16, int D, int kChunks, int kKeyGroups>
__global__ void __launch_bounds__(KvLayout<D, kChunks, kKeyGroups>::kThreads, KvLayout<D, kChunks, kKeyGroups>::kCtasPerSm)
kv_attention_kernel(const __grid_constant__ CUtensorMap mk, const __grid_constant__ CUtensorMap mv, const KvAttnParams p)
{
    using namespace sm100;
    using L = KvLayout<D, kChunks, kKeyGroups>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t sbase = smem_u32(smem);
    auto full = [&](int s) { return sbase + L::kBarOff + 8u * (uint32_t)s; };
    auto empty = [&](int s) { return sbase + L::kBarOff + 8u * (uint32_t)(L::kStages + s); };
    volatile int *s_abort = reinterpret_cast<volatile int *>(smem + L::kMiscOff);
    int *s_len = reinterpret_cast<int *>(smem + L::kSeqOff), *s_pre = s_len + p.B;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    allow_next_kernel();
    if (tid == 0) {
        for (int s = 0; s < L::kStages; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), L::kWarps); }
        mbar_fence_init();
        *s_abort = 0;
    }
    await_previous_kernel();
    // ---- every CTA's share: tiles of each sequence, their running sum ---------------------------------
    const int64_t most = (int64_t)p.width * p.page;
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
    const int heads = p.Hkv * p.groups;
    const int total = s_pre[p.B] * heads;                                  // (fits: checked on the host)
    const int per = max((total + (int)gridDim.x - 1) / (int)gridDim.x, kKvMinTiles);
    const int w0 = (int)min((int64_t)blockIdx.x * per, (int64_t)total), w1 = min(w0 + per, total);
    if (tid == 0) p.desc[blockIdx.x] = make_int2(-1, 0);
    if (w0 >= w1) return;
    constexpr int kBoxRowsMax = kKvTile;
    const int box_rows = min(p.page, kBoxRowsMax), boxes = kKvTile / box_rows;

    if (warp == L::kWarps) {
        // ======================= producer: a lane per page box of the next 32 ============================
        const int per_batch = 32 / boxes;
        struct Box { int y; float ks, vs; };
        auto fetch = [&](int w) {
            Box x{-1, -1.f, 0.f};
            const int mine = w + lane / boxes;
            if (mine < w1) {
                const KvPlace a = kv_place(s_pre, p.B, heads, mine);
                const int len = s_len[a.b];
                const int pos = kv_tiles(len, p.T, p.window, p.sinks).tile(a.i) * kKvTile + (lane % boxes) * box_rows;
                if (pos < len) {
                    const int id = p.table[(int64_t)a.b * p.width + pos / p.page];
                    if (id >= 0 && id < p.n_pages) {
                        const int64_t ph = (int64_t)id * p.Hkv + a.hr / p.groups;
                        x.y = (int)(ph * p.page + pos % p.page);
                        x.ks = p.k_scale[ph];
                        x.vs = p.v_scale[ph];
                    }
                }
            }
            return x;
        };
        Box now = fetch(w0);
        int n = 0;                                                       // tiles issued
        bool ok = true;
        for (int w = w0; ok && w < w1; w += per_batch) {
            const Box next = w + per_batch < w1 ? fetch(w + per_batch) : now;
            for (int k = 0; k < per_batch && w + k < w1; ++k, ++n) {
                const int s = n % L::kStages;
                ok = __all_sync(0xffffffffu, mbar_wait(empty(s), (uint32_t)((n / L::kStages) & 1) ^ 1u, s_abort, &g_async_status, 0x500));
                if (!ok) break;
                const bool mine = lane / boxes == k;
                const unsigned there = __ballot_sync(0xffffffffu, mine && now.y >= 0);
                if (mine)
                    *reinterpret_cast<float2 *>(smem + L::kMetaOff + (s * 4 + lane % boxes) * 8) = make_float2(now.ks, now.vs);
                __syncwarp();
                if (lane == 0) mbar_arrive_expect_tx(full(s), (uint32_t)(__popc(there) * 2 * box_rows * D));
                __syncwarp();
                if (mine && now.y >= 0) {
                    const uint32_t at = sbase + L::kRingOff + s * 2 * L::kTileBytes + (lane % boxes) * box_rows * D;
                    tma_load_2d(at, &mk, 0, now.y, full(s));
                    tma_load_2d(at + L::kTileBytes, &mv, 0, now.y, full(s));
                }
            }
            now = next;
        }
        if (*s_abort) {
            // copies in flight land before the CTA's shared memory is released
            for (int l = n > L::kStages ? n - L::kStages : 0; l < n; ++l) {
                const uint64_t t0 = globaltimer_ns();
                while (!mbar_try_wait(full(l % L::kStages), (uint32_t)((l / L::kStages) & 1)) && globaltimer_ns() - t0 < 2000000ull) {}
            }
        }
        return;
    }

    // ======================= consumers =====================================================================
    const int chunk = warp / kKeyGroups, kg = warp % kKeyGroups;
    const int g = lane >> 2, t = lane & 3;
    constexpr int kSegs = D / 64;
    // key row of fragment index i (0 .. 7) within eight rows, see the file comment
    auto row_of = [](int i) {
        const int b0 = i & 1, b1 = (i >> 1) & 1, b2 = i >> 2;
        return D == 128 ? ((b2 ^ b0) << 2) | (b1 << 1) | b0 : (b2 << 2) | (b0 << 1) | (b1 ^ b0);
    };
    const int kr = row_of(g), v0r = row_of(2 * t), v1r = row_of(2 * t + 1);
    // byte offset in a swizzled tile of 16-byte part `part` of row `row`
    auto at = [](int row, int part) { return (uint32_t)(row * D + ((part ^ (D == 128 ? row & 7 : (row >> 1) & 3)) << 4)); };

    int n = 0;                                                           // tiles used
    for (int w = w0; w < w1;) {
        const KvPlace a = kv_place(s_pre, p.B, heads, w);
        const int tiles = min(a.n - a.i, w1 - w);
        const int len = s_len[a.b], hk = a.hr / p.groups, row_base = (a.hr % p.groups) * L::kRows + chunk * 16;
        const KeyTiles kt = kv_tiles(len, p.T, p.window, p.sinks);
        const int q_first = len - p.T;                                   // position of query 0, maybe below 0

        // ---- the warp's 16 rows of q: row r is query r % T of head r / T of the group ---------------------
        uint32_t qa[kSegs * 4][4];
        float cq[2], m[2], l[2];
        int pos[2];                                                      // of the thread's two rows; below 0: sees nothing
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = row_base + g + 8 * half;
            const bool there = r < p.R;
            const int tq = r % p.T, hq = hk * p.G + r / p.T;
            pos[half] = there ? q_first + tq : -1;
            float x[kSegs * 16];
            if (there) {
                const T16 *src = reinterpret_cast<const T16 *>(p.q) + a.b * p.qs_b + hq * p.qs_h + tq * p.qs_t + 16 * t;
#pragma unroll
                for (int s = 0; s < kSegs; ++s)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(src + 64 * s + 8 * e);
                        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float2 f = values2<T16>(u[k]);
                            x[16 * s + 8 * e + 2 * k] = f.x; x[16 * s + 8 * e + 2 * k + 1] = f.y;
                        }
                    }
            } else {
#pragma unroll
                for (int k = 0; k < kSegs * 16; ++k) x[k] = 0.f;
            }
            float scale = 1.f, back = 1.f;
            if constexpr (!__is_same(T16, __half)) {                     // largest element of the row to [1, 2)
                float big = 0.f;
#pragma unroll
                for (int k = 0; k < kSegs * 16; ++k) big = fmaxf(big, fabsf(x[k]));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
                const uint32_t e = min(max(__float_as_uint(big) >> 23, 1u), 253u);
                back = __uint_as_float(e << 23);
                scale = __uint_as_float((254u - e) << 23);
            }
            cq[half] = p.c * back;
            m[half] = -INFINITY;
            l[half] = 0.f;
#pragma unroll
            for (int s = 0; s < kSegs; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k) {                            // product k of the segment: bytes 4 k .. 4 k + 3
                    qa[s * 4 + k][half] = pack16<__half>(x[16 * s + 4 * k] * scale, x[16 * s + 4 * k + 1] * scale);
                    qa[s * 4 + k][half + 2] = pack16<__half>(x[16 * s + 4 * k + 2] * scale, x[16 * s + 4 * k + 3] * scale);
                }
        }
        float o[D / 8][4];
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) o[i][k] = 0.f;
        float unit = 0.f;                                                // scale of the page that O~ is in units of; 0: none yet

        for (int i = 0; i < tiles; ++i, ++n) {
            const int s = n % L::kStages;
            mbar_wait(full(s), (uint32_t)((n / L::kStages) & 1), s_abort, &g_async_status, 0x510);
            const int c0 = kt.tile(a.i + i) * kKvTile;
            // every query sees every key of the tile
            const bool all = c0 + kKvTile - 1 <= q_first && (c0 > len - 1 - p.window || c0 + kKvTile - 1 < p.sinks);
            const uint32_t ktile = sbase + L::kRingOff + s * 2 * L::kTileBytes, vtile = ktile + L::kTileBytes;
#pragma unroll 1
            for (int step = 0; step < 4 / kKeyGroups; ++step) {
                const int key0 = (kg * (4 / kKeyGroups) + step) * 16;    // of the tile
                const float2 meta = *reinterpret_cast<const float2 *>(smem + L::kMetaOff + (s * 4 + key0 / box_rows) * 8);
                if (meta.x < 0.f) continue;                              // no such page
                // ---- scores: two n-tiles of eight keys -------------------------------------------------------
                float sc[2][4];
#pragma unroll
                for (int nt = 0; nt < 2; ++nt) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) sc[nt][k] = 0.f;
#pragma unroll
                    for (int seg = 0; seg < kSegs; ++seg) {
                        const uint4 kv = lds_u32x4(ktile + at(key0 + 8 * nt + kr, 4 * seg + t));
                        const uint32_t u[4] = {kv.x, kv.y, kv.z, kv.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) mma_f16(sc[nt], qa[seg * 4 + k], widen_lo(u[k]), widen_hi(u[k]));
                    }
                }
                // ---- s in base 2, mask ----------------------------------------------------------------------
                bool hide[4] = {false, false, false, false};             // keys that no query sees: V may hold anything
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float f = cq[half] * meta.x;
#pragma unroll
                    for (int k = 0; k < 4; ++k) sc[k >> 1][2 * half + (k & 1)] *= f;
                }
                if (!all) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int j = c0 + key0 + 8 * (k >> 1) + ((k & 1) ? v1r : v0r);
                        hide[k] = j >= len || !(j > max(q_first, 0) - p.window || j < p.sinks);
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            const bool see = j <= pos[half] && (j > pos[half] - p.window || j < p.sinks);
                            if (!see) sc[k >> 1][2 * half + (k & 1)] = -INFINITY;
                        }
                    }
                }
                // ---- running maximum ------------------------------------------------------------------------
                float mx[2];
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    mx[half] = fmaxf(fmaxf(sc[0][2 * half], sc[0][2 * half + 1]), fmaxf(sc[1][2 * half], sc[1][2 * half + 1]));
                if (__any_sync(0xffffffffu, mx[0] > m[0] + 8.f || mx[1] > m[1] + 8.f)) {
                    float f[2];
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        mx[half] = fmaxf(mx[half], __shfl_xor_sync(0xffffffffu, mx[half], 1));
                        mx[half] = fmaxf(mx[half], __shfl_xor_sync(0xffffffffu, mx[half], 2));
                        const float m_new = fmaxf(m[half], mx[half]);
                        f[half] = m[half] == -INFINITY ? 1.f : ex2_approx(m[half] - m_new);
                        m[half] = m_new;
                        l[half] *= f[half];
                    }
#pragma unroll
                    for (int k = 0; k < D / 8; ++k) { o[k][0] *= f[0]; o[k][1] *= f[0]; o[k][2] *= f[1]; o[k][3] *= f[1]; }
                }
                // ---- O~ in units of this page's value scale ---------------------------------------------------
                float in_unit = 1.f;
                if (meta.y != unit) {
                    if (unit == 0.f) unit = meta.y;
                    else if (meta.y < unit * 5.421010862427522e-20f) in_unit = 0.f;          // 2^-64: does not count
                    else {
                        const float f = unit / meta.y;
#pragma unroll
                        for (int k = 0; k < D / 8; ++k)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[k][e] *= f;
                        unit = meta.y;
                    }
                }
                // ---- weights --------------------------------------------------------------------------------
                uint32_t pa[4];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float mu = m[half] == -INFINITY ? 0.f : m[half];
#pragma unroll
                    for (int nt = 0; nt < 2; ++nt) {
                        const float x = ex2_approx(sc[nt][2 * half] - mu), y = ex2_approx(sc[nt][2 * half + 1] - mu);
                        l[half] += x + y;
                        pa[half + 2 * nt] = pack16<__half>(x * in_unit, y * in_unit);
                    }
                }
                // ---- O~ += P V ------------------------------------------------------------------------------
                constexpr int kWords = D / 32;                           // 4-byte words of a thread's part of a V row
                uint32_t v[4][kWords];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int row = key0 + 8 * (k >> 1) + ((k & 1) ? v1r : v0r);
                    if constexpr (D == 128) {
                        const uint4 u = lds_u32x4(vtile + at(row, g));
                        v[k][0] = u.x; v[k][1] = u.y; v[k][2] = u.z; v[k][3] = u.w;
                    } else {
                        const float2 u = lds_f32x2(vtile + at(row, g >> 1) + (g & 1) * 8);
                        v[k][0] = __float_as_uint(u.x); v[k][1] = __float_as_uint(u.y);
                    }
                    if (!all) {
#pragma unroll
                        for (int e = 0; e < kWords; ++e) v[k][e] = hide[k] ? 0u : v[k][e];
                    }
                }
#pragma unroll
                for (int e = 0; e < kWords; ++e) {
                    const uint32_t ab = __byte_perm(v[0][e], v[1][e], 0x5140), ab2 = __byte_perm(v[0][e], v[1][e], 0x7362);
                    const uint32_t cd = __byte_perm(v[2][e], v[3][e], 0x5140), cd2 = __byte_perm(v[2][e], v[3][e], 0x7362);
                    mma_f16(o[4 * e], pa, widen_lo(ab), widen_lo(cd));
                    mma_f16(o[4 * e + 1], pa, widen_hi(ab), widen_hi(cd));
                    mma_f16(o[4 * e + 2], pa, widen_lo(ab2), widen_lo(cd2));
                    mma_f16(o[4 * e + 3], pa, widen_hi(ab2), widen_hi(cd2));
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty(s));
        }

        // ---- join the warps that share these rows ----------------------------------------------------------
        float4 *join = reinterpret_cast<float4 *>(smem + L::kJoinOff);
        float2 *ml = reinterpret_cast<float2 *>(smem + L::kMlOff);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
            l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
            if (t == 0) ml[warp * 16 + g + 8 * half] = make_float2(m[half], l[half]);
        }
        // thread (g, t) holds elements (2 t) D / 8 + i and (2 t + 1) D / 8 + i, i = 0 .. D / 8 - 1, of rows g and g + 8:
        // slot (half, e, quarter) is elements (2 t + e) D / 8 + 4 quarter .. + 3 of row g + 8 half
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int qr = 0; qr < D / 32; ++qr)
                    join[(warp * (D / 8) + (half * 2 + e) * (D / 32) + qr) * 32 + lane] =
                        make_float4(o[4 * qr][2 * half + e] * unit, o[4 * qr + 1][2 * half + e] * unit,
                                    o[4 * qr + 2][2 * half + e] * unit, o[4 * qr + 3][2 * half + e] * unit);
        named_bar_sync(1, L::kWarps * 32);
        const bool whole = tiles == a.n;
        const bool good = *s_abort == 0;
        const int slot = 2 * blockIdx.x + (a.i == 0 ? 1 : 0);
        // the chunk's kKeyGroups warps share its D / 8 slots of 32 lanes
        for (int sl = kg; good && sl < D / 8; sl += kKeyGroups) {
            const int half = sl / (2 * (D / 32)), e = sl / (D / 32) % 2, qr = sl % (D / 32);
            const int rr = g + 8 * half, r = row_base + rr;
            if (r >= p.R) continue;
            float M = -INFINITY, Lsum = 0.f;
            float2 part[kKeyGroups];
#pragma unroll
            for (int x = 0; x < kKeyGroups; ++x) { part[x] = ml[(chunk * kKeyGroups + x) * 16 + rr]; M = fmaxf(M, part[x].x); }
            const float Mu = M == -INFINITY ? 0.f : M;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int x = 0; x < kKeyGroups; ++x) {
                const float f = ex2_approx(part[x].x - Mu);
                const float4 u = join[((chunk * kKeyGroups + x) * (D / 8) + sl) * 32 + lane];
                Lsum += f * part[x].y;
                acc.x += f * u.x; acc.y += f * u.y; acc.z += f * u.z; acc.w += f * u.w;
            }
            const int d0 = (2 * t + e) * (D / 8) + 4 * qr;
            if (whole) {
                kv_store<T16>(p, a.b, hk * p.G + r / p.T, r % p.T, d0, acc, M, Lsum);
            } else {
                *reinterpret_cast<float4 *>(p.part_o + ((int64_t)slot * L::kRows + chunk * 16 + rr) * D + d0) = acc;
                if (d0 == 0) p.part_ml[(int64_t)slot * L::kRows + chunk * 16 + rr] = make_float2(M, Lsum);
            }
        }
        if (tid == 0 && a.i == 0 && !whole) p.desc[blockIdx.x] = make_int2(a.b * heads + a.hr, (w + a.n - 1) / per);
        named_bar_sync(1, L::kWarps * 32);                               // before the buffers are written again
        w += tiles;
    }
}

// Joins the parts of the item that begins in CTA blockIdx.x of the kernel above and ends in a later one, in the CTAs' order.
// Blocks (CTA, rows): 512 / D rows, four elements per thread.
template <typename T16, int D, int kRows>
__global__ void __launch_bounds__(128)
kv_join_kernel(const KvAttnParams p)
{
    allow_next_kernel();
    await_previous_kernel();
    const int2 what = p.desc[blockIdx.x];
    if (what.x < 0) return;
    const int heads = p.Hkv * p.groups, hr = what.x % heads;
    const int rr = blockIdx.y * (512 / D) + threadIdx.x / (D / 4), d0 = threadIdx.x % (D / 4) * 4;
    const int r = hr % p.groups * kRows + rr;
    if (r >= p.R) return;
    const int parts = what.y - (int)blockIdx.x + 1;
    auto row = [&](int k) { return (int64_t)(2 * ((int)blockIdx.x + k) + (k == 0 ? 1 : 0)) * kRows + rr; };
    float m = -INFINITY, l = 0.f;
    for (int k = 0; k < parts; ++k) m = fmaxf(m, p.part_ml[row(k)].x);
    const float mu = m == -INFINITY ? 0.f : m;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int k = 0; k < parts; ++k) {
        const float2 ml = p.part_ml[row(k)];
        const float4 u = *reinterpret_cast<const float4 *>(p.part_o + row(k) * D + d0);
        const float f = ex2_approx(ml.x - mu);
        l += f * ml.y;
        o.x += f * u.x; o.y += f * u.y; o.z += f * u.z; o.w += f * u.w;
    }
    kv_store<T16>(p, what.x / heads, hr / p.groups * p.G + r / p.T, r % p.T, d0, o, m, l);
}

// Rows of a kv head go to a CTA 16, 32 or 64 at a time, so that its K and V are read once wherever that can be: 16 rows take four
// warps (two CTAs per SM), more take eight that read every tile once per 16 rows.
struct KvShape { int chunks, groups, ctas; };
static inline KvShape kv_shape(int R)
{
    KvShape s;
    s.chunks = R <= 16 ? 1 : R <= 32 ? 2 : 4;
    s.groups = (R + 16 * s.chunks - 1) / (16 * s.chunks);
    s.ctas = num_sms() * (s.chunks == 1 ? 2 : 1);
    return s;
}
// Bytes: part_o, part_ml, desc
static inline size_t kv_workspace(const KvShape &s, int D)
{
    const size_t rows = (size_t)s.ctas * 2 * 16 * s.chunks;
    return rows * D * 4 + rows * 8 + (size_t)s.ctas * 8;
}

template <typename T16, int D, int kChunks, int kKeyGroups>
static inline baps_status kv_attention_launch(const CUtensorMap &mk, const CUtensorMap &mv, const KvAttnParams &p, int ctas,
                                              cudaStream_t stream)
{
    using L = KvLayout<D, kChunks, kKeyGroups>;
    if (cudaFuncSetAttribute(kv_attention_kernel<T16, D, kChunks, kKeyGroups>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             L::dyn_bytes(kKvMaxB)) != cudaSuccess)
        return BAPS_ERR_CUDA;
    const baps_status s = launch_kernel(kv_attention_kernel<T16, D, kChunks, kKeyGroups>, (unsigned)ctas, L::kThreads,
                                        (size_t)L::dyn_bytes(p.B), stream, mk, mv, p);
    if (s != BAPS_OK) return s;
    return launch_kernel(kv_join_kernel<T16, D, L::kRows>, dim3((unsigned)ctas, (unsigned)(L::kRows * D / 512)), 128, 0, stream, p);
}

template <typename T16, int D>
static inline baps_status kv_attention_rows(const CUtensorMap &mk, const CUtensorMap &mv, const KvAttnParams &p,
                                            const KvShape &s, cudaStream_t stream)
{
    if (s.chunks == 1) return kv_attention_launch<T16, D, 1, 4>(mk, mv, p, s.ctas, stream);
    if (s.chunks == 2) return kv_attention_launch<T16, D, 2, 4>(mk, mv, p, s.ctas, stream);
    return kv_attention_launch<T16, D, 4, 2>(mk, mv, p, s.ctas, stream);
}

} // namespace baps
