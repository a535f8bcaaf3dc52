// Attention of whole prompts with a sliding window and a few first tokens that stay visible, on tcgen05 (bf16 or fp16).
//
// Row r of a sequence sees key c where c <= r and (c > r - window or c < sinks).  The plain softmax, one pass over the keys:
//     m = running maximum, l = sum 2^(c s - m), O~ = sum 2^(c s - m) v;   O = O~ / l, lse = ln 2 (m + log2 l)
// with s = q . k and c = log2(e) * scale.  m is held back: it moves only when a row's maximum passes it by more than 8
// (weights stay below 2^8, exact in what follows), so that O~, which lives in tensor memory, is hardly ever rescaled.
// S, l and O~ are float32; the weights are rounded to the inputs' type for the P V product (half a step, 2^-8 or 2^-11
// of each weight) and summed before that rounding.
//
// Heads of 128: one CTA owns two consecutive 128-row query tiles (t = 0, 1; small grids: one) of one head, which share the K / V
// stream: the 128-key tiles that hold first tokens, then those from the window's left edge to the diagonal.  A stream takes
// part in the key tiles that some row of its own sees.
//   warps 0-15      softmax: stream t = w / 8; two threads per row, 64 key columns each, in two chunks of 32
//   warp 16         TMA producer: Q tiles, then K_0, V_0, K_1, ... through a ring of key tiles
//   warp 17         MMA issuer, per key tile and stream: P V for the keys of the second chunks as soon as their weights are
//                   there, then for the others, and Q K^T of the stream's next key tile into the same columns; in a sequence's last
//                   V tile it zeroes what stands behind the end first (a weight of 0 does not hide a NaN)
// (warps 18, 19 idle: they complete the warpgroup whose registers go to the softmax warps.)
// Heads of 64: one query tile per CTA, three CTAs per SM, key tiles of 64, one thread per row; the same roles in six warps.
// TMEM: S of each stream, then O; the 16-bit weights of column quarter q overwrite columns [32 q, 32 q + 16) of S_t.
// Tensor memory is taken after the kernel ahead has ended and before the next one may start.  All waits are bounded; after an
// expired one every later wait returns at once and the roles run on to the common teardown without storing.
//
// What bounds it: the chain of a stream, scores to weights to products, as in paired_attention_tc_kernel, and at the longest sizes the
// power limit.  32 / 8 heads of 128, 32768 tokens, window 4096: 1.81 to 1.85 ms (1157 TFLOP/s of visible pairs; 94 % of the pairs in the
// tiles are visible).  With one thread per row and four warps per stream 1.96 ms: 3900 cycles for a pair of key tiles, in which
// the exponentials need 2048 of their pipe and the products 1024 of the tensor core.  Exponentials by a polynomial of degree 4
// on the FMA pipe, for an eighth to a half of the columns: no gain then, 1.85 to 1.91 ms in this form.
// Heads of 64: a padded batch of 8 x 4001 tokens, 16 / 4 heads, window 500, 20 first tokens: 117 us; as two streams per CTA, one CTA per SM 169 (a CTA
// lives for six or seven tiles: its start and end are as long as its work), one stream and 128-key tiles, two per SM 134. Chunks of 32 keys that
// no row of a warp sees are skipped (144 to 134 us).
// 96 registers at launch: the form with two query tiles spills 8 bytes, the one with heads of 64 36.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "baps_common.cuh"
#include "baps_register_split.cuh"
#include "baps_sm100.cuh"
#include "baps_tma_host.cuh"
#include "baps_visible.cuh"

namespace baps {

#ifdef BAPS_TEST_SKIP_LOAD
// Test build only: number of the K / V tile load that window_attention_kernel's producer leaves out.  -1: none.
static __device__ int g_test_skip_window_load = -1;
#endif

struct WindowParams {
    void *out;
    float *lse;
    const int32_t *lengths;
    int64_t os_b, os_h, os_s;      // strides of out, elements
    int B, H, Hkv, S, window, sinks, nitems;          // window: up to S; nitems: work items per head, of one or two query tiles
    float c;
};

// kStreams: query tiles of a CTA; kKeys: keys of a tile, 128 (two threads per row) or 64 (one).
template <int D, int kStreams, int kKeys>
struct WinLayout {
    static constexpr int kHalves = kKeys / 64, kWarpsOfStream = 4 * kHalves, kSoftmaxWarps = kStreams * kWarpsOfStream;
    static constexpr bool kShares = kStreams == 2;                     // of registers: the softmax warps take some of the others' (kTcSplit)
    static constexpr int kThreads = kShares ? kTcSplit.threads : kSoftmaxWarps * 32 + 64;
    static constexpr int kCtasPerSm = kKeys == 64 ? 3 : 1;
    static constexpr int kQBytes = 128 * D * 2, kKvBytes = kKeys * D * 2, kBoxBytes = kKeys * 128;
    static constexpr int kStages = 4;
    static constexpr int kLogKeys = kKeys == 64 ? 6 : 7;
    static constexpr int kQOff = 0;
    static constexpr int kKvOff = kStreams * kQBytes;
    static constexpr int kBarOff = kKvOff + kStages * kKvBytes;
    static constexpr int kOCol = kKeys * kStreams, kTmemCols = kKeys == 64 ? 128 : 256 * kStreams;      // S of each stream, then O
    // q_full, s_full[2], p_full[2][2], o_done[2], kv_full[stages], kv_empty[stages]
    static constexpr int kXchgOff = (kBarOff + (9 + 2 * kStages) * 8 + 15) & ~15;      // float xchg[2 tiles][128][2]
    static constexpr int kMiscOff = kXchgOff + 2 * 128 * 2 * 4;
    static constexpr int kDynBytes = kMiscOff + 16 + 1024;
    static_assert((D == 128 && kKeys == 128) || (D == 64 && kKeys == 64 && kStreams == 1), "forms that are looked after");
};

template <typename T16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi)
{
    if constexpr (sizeof(T16) == 2 && __is_same(T16, __half)) {
        uint32_t d;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
        return d;
    } else {
        return pack_bf16x2(lo, hi);
    }
}

__device__ __forceinline__ float max8w(const uint32_t *x)
{
    return max3(max3(__uint_as_float(x[0]), __uint_as_float(x[1]), __uint_as_float(x[2])),
                max3(__uint_as_float(x[3]), __uint_as_float(x[4]), __uint_as_float(x[5])),
                fmaxf(__uint_as_float(x[6]), __uint_as_float(x[7])));
}

template <typename T16, int D, int kStreams, int kKeys>
__global__ void __launch_bounds__(WinLayout<D, kStreams, kKeys>::kThreads, WinLayout<D, kStreams, kKeys>::kCtasPerSm)
window_attention_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                        const __grid_constant__ CUtensorMap mv, const WindowParams p)
{
    using namespace sm100;
    using L = WinLayout<D, kStreams, kKeys>;
    constexpr int kProducer = L::kSoftmaxWarps, kIssuer = kProducer + 1, kOCol = L::kOCol;
    constexpr bool kHalf = __is_same(T16, __half);
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const uint32_t sbase = smem_u32(smem);
    auto bar = [&](int i) { return sbase + L::kBarOff + 8u * (uint32_t)i; };
    constexpr int BQ = 0, BS = 1, BP = 3, BD = 7, BKF = 9, BKE = 9 + L::kStages;
    uint32_t *s_tmem = reinterpret_cast<uint32_t *>(smem + L::kMiscOff);
    volatile int *s_abort = reinterpret_cast<volatile int *>(smem + L::kMiscOff + 4);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // blocks: query heads of a kv head next to each other, later rows (more keys, while the window fills) first
    const int heads = p.B * p.H;
    const int h = (int)(blockIdx.x % (unsigned)heads) % p.H, b = (int)(blockIdx.x % (unsigned)heads) / p.H;
    const int q0 = kStreams * (p.nitems - 1 - (int)(blockIdx.x / (unsigned)heads));
    const int hk = h / (p.H / p.Hkv);

    await_previous_kernel();
    const int len = p.lengths ? min(max(p.lengths[b], 0), p.S) : p.S;
    if (q0 * 128 >= len) return;
    // last rows of the two query tiles; the second is absent where the sequence ends in the first
    const bool two = kStreams == 2 && (q0 + 1) * 128 < len;
    const int last0 = min(q0 * 128 + 127, len - 1), last1 = min(q0 * 128 + 128 * kStreams - 1, len - 1);
    const KeyTiles kt = key_tiles(q0 * 128, last1, p.window, p.sinks, L::kLogKeys);
    const KeyTiles mine0 = key_tiles(q0 * 128, last0, p.window, p.sinks, L::kLogKeys);
    const KeyTiles mine1 = key_tiles(min(q0 * 128 + 128, last1), last1, p.window, p.sinks, L::kLogKeys);
    const int J = kt.count();
    auto takes = [&](int t, int j) { return t == 0 ? mine0.has(kt.tile(j)) : two && mine1.has(kt.tile(j)); };
    auto stage_of = [&](int l) { return l % L::kStages; };
    auto parity_of = [&](int l) { return (uint32_t)((l / L::kStages) & 1); };
    // the sequence's last V tile holds rows behind its end (rows behind S come as zeros)
    const bool ragged = len < p.S && (len & (kKeys - 1)) != 0 && kt.w1 == (len - 1) >> L::kLogKeys;

    if (tid == 0) {
        mbar_init(bar(BQ), 1);
        for (int t = 0; t < 2; ++t) { mbar_init(bar(BS + t), 1); mbar_init(bar(BD + t), 1); }
        for (int i = 0; i < 4; ++i) mbar_init(bar(BP + i), L::kWarpsOfStream);
        for (int s = 0; s < L::kStages; ++s) { mbar_init(bar(BKF + s), 1); mbar_init(bar(BKE + s), 1); }
        mbar_fence_init();
        *s_abort = 0;
    }
    if (warp == kIssuer) { tmem_alloc(smem_u32(s_tmem), L::kTmemCols); tmem_relinquish(); }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    allow_next_kernel();
    const uint32_t tmem = *s_tmem;

    if (warp >= L::kSoftmaxWarps) {
        if constexpr (L::kShares) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTcSplit.few));
        if (warp == kProducer) {
        // ======================= TMA producer ======================================================
        if (lane == 0) {
            mbar_arrive_expect_tx(bar(BQ), (two ? 2u : 1u) * L::kQBytes);
            for (int t = 0; t < (two ? 2 : 1); ++t)
                for (int hh = 0; hh < D / 64; ++hh)
                    tma_load_4d(sbase + L::kQOff + t * L::kQBytes + hh * 16384, &mq, hh * 64, (q0 + t) * 128, h, b, bar(BQ));
            int issued = 0;
            for (int l = 0; l < 2 * J; ++l) {
                const int s = stage_of(l);
                if (!mbar_wait(bar(BKE + s), parity_of(l) ^ 1u, s_abort, &g_async_status, 0x400 + s)) break;
#ifdef BAPS_TEST_SKIP_LOAD
                if (l == g_test_skip_window_load) { issued = l + 1; continue; }         // this tile never arrives
#endif
                mbar_arrive_expect_tx(bar(BKF + s), L::kKvBytes);
                for (int hh = 0; hh < D / 64; ++hh)
                    tma_load_4d(sbase + L::kKvOff + s * L::kKvBytes + hh * L::kBoxBytes, (l & 1) ? &mv : &mk, hh * 64,
                                kt.tile(l >> 1) * kKeys, hk, b, bar(BKF + s));
                issued = l + 1;
            }
            if (*s_abort) {
                // copies in flight land before the CTA's shared memory is released
                for (int l = issued > L::kStages ? issued - L::kStages : 0; l < issued; ++l) {
                    const uint64_t t0 = globaltimer_ns();
                    while (!mbar_try_wait(bar(BKF + stage_of(l)), parity_of(l)) && globaltimer_ns() - t0 < 2000000ull) {}
                }
            }
        }
        } else if (warp == kIssuer) {
        // ======================= MMA issuer ========================================================
        constexpr uint32_t fmt = kHalf ? 0u : (1u << 7) | (1u << 10);
        constexpr uint32_t idesc_qk = (make_idesc_bf16(128, kKeys, false) & ~((7u << 7) | (7u << 10))) | fmt;
        constexpr uint32_t idesc_pv = (make_idesc_bf16(128, D, true) & ~((7u << 7) | (7u << 10))) | fmt;
        auto wait_all = [&](uint32_t bar_addr, uint32_t parity, int code) -> bool {
            return __all_sync(0xffffffffu, mbar_wait(bar_addr, parity, s_abort, &g_async_status, code));
        };
        const bool leader = elect_one();
        auto mma_qk = [&](int t, int j) {
            const uint32_t qd = sdesc_lo(sbase + L::kQOff + t * L::kQBytes, 16);
            const uint32_t kd = sdesc_lo(sbase + L::kKvOff + stage_of(2 * j) * L::kKvBytes, 16);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                mma_ss_lo(tmem + t * kKeys, qd + (uint32_t)(((ks >> 2) * 16384 + (ks & 3) * 32) >> 4),
                          kd + (uint32_t)(((ks >> 2) * L::kBoxBytes + (ks & 3) * 32) >> 4), idesc_qk, ks > 0);
            mma_commit(bar(BS + t));
        };
        // O_t += P V_j over the keys of one half of the weights: the odd 32-column quarters (first), then the even ones
        auto mma_pv = [&](int t, int j, int half, bool more) {
            const uint32_t vd = sdesc_lo(sbase + L::kKvOff + stage_of(2 * j + 1) * L::kKvBytes, L::kBoxBytes);
#pragma unroll
            for (int i = 0; i < 2 * L::kHalves; ++i) {
                const int quarter = (i >> 1) * 2 + 1 - half, ks = 2 * quarter + (i & 1);
                mma_ts_lo(tmem + kOCol + t * 128, tmem + t * kKeys + quarter * 32 + (i & 1) * 8, vd + ks * 128, idesc_pv, half || i || more);
            }
        };
        // A stream's next Q K^T is issued behind its P V, into the same columns.
        int done[2] = {0, 0};                          // key tiles that the stream has been through
        auto next_of = [&](int t, int j) { while (j < J && !takes(t, j)) ++j; return j; };
        int nj[2] = {next_of(0, 0), kStreams == 2 ? next_of(1, 0) : J};    // the tile whose scores were asked for last (J: no more)
        int k_there = 0, k_freed = 0;                  // K tiles waited for, and given back
        bool ok = wait_all(bar(BQ), 0, 0x410);
        auto need_k = [&](int j) {
            for (; ok && k_there <= j; ++k_there) ok = wait_all(bar(BKF + stage_of(2 * k_there)), parity_of(2 * k_there), 0x411);
        };
        // K_f is free when both streams have asked for their scores of it, or of a later tile
        auto free_k = [&] {
            for (; k_freed < J && k_freed <= min(nj[0], nj[1]); ++k_freed) mma_commit(bar(BKE + stage_of(2 * k_freed)));
        };
        for (int t = 0; t < kStreams; ++t)
            if (nj[t] < J) {
                need_k(nj[t]);
                if (!ok) break;
                tc_fence_after_sync();
                if (leader) mma_qk(t, nj[t]);
                __syncwarp();
            }
        if (ok && leader) free_k();
        k_freed = min(J, min(nj[0], nj[1]) + 1);
        for (int j = 0; ok && j < J; ++j) {
            ok = wait_all(bar(BKF + stage_of(2 * j + 1)), parity_of(2 * j + 1), 0x420);
            if (ok && ragged && j == J - 1) {
                // rows behind the sequence's end: a weight of 0 does not hide a NaN
                const uint32_t stage = sbase + L::kKvOff + stage_of(2 * j + 1) * L::kKvBytes;
                const int first = len & (kKeys - 1);
#pragma unroll 1
                for (int i = lane; i < (kKeys - first) * (D / 8); i += 32) {
                    const int row = first + i / (D / 8), part = i % (D / 8);
                    sts_u32x4(stage + (uint32_t)((part >> 3) * L::kBoxBytes + row * 128 + (part & 7) * 16), make_uint4(0, 0, 0, 0));
                }
                fence_async_shared();
                __syncwarp();
            }
            for (int t = 0; ok && t < kStreams; ++t) {
                if (nj[t] != j) continue;
                const int nx = next_of(t, j + 1);
                if (nx < J) need_k(nx);
                ok = ok && wait_all(bar(BP + 2 * t), (uint32_t)(done[t] & 1), 0x430 + t);
                if (!ok) break;
                tc_fence_after_sync();
                if (leader) mma_pv(t, j, 0, done[t] > 0);
                __syncwarp();
                ok = wait_all(bar(BP + 2 * t + 1), (uint32_t)(done[t] & 1), 0x432 + t);
                if (!ok) break;
                tc_fence_after_sync();
                nj[t] = nx;
                if (leader) {
                    mma_pv(t, j, 1, true);
                    if (nx < J) mma_qk(t, nx);
                    else mma_commit(bar(BD + t));
                    free_k();
                }
                k_freed = min(J, min(nj[0], nj[1]) + 1);
                ++done[t];
                __syncwarp();
            }
            if (ok && leader) mma_commit(bar(BKE + stage_of(2 * j + 1)));
            __syncwarp();
        }
        }
    } else {
        if constexpr (L::kShares) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTcSplit.many));
        // ======================= softmax warps =====================================================
        const int t = warp / L::kWarpsOfStream, q4 = warp & 3, ch = L::kHalves == 2 ? (warp >> 2) & 1 : 0;
        constexpr int kMyCols = D / L::kHalves;                       // columns of O~ that a thread looks after
        if (t == 0 || two) {
        const int row = q4 * 32 + lane;                               // of the query tile
        const int r = (q0 + t) * 128 + row;                           // of the sequence
        const uint32_t lane_sel = (uint32_t)(q4 * 32) << 16;
        const uint32_t s_addr = tmem + lane_sel + t * kKeys + ch * 64, o_addr = tmem + lane_sel + kOCol + t * 128 + ch * kMyCols;
        const uint32_t xrow = sbase + L::kXchgOff + (uint32_t)((t * 128 + row) * 8);
        const uint32_t row_bar = 1 + t * 4 + q4;                      // the two warps that share these rows
        const int r_first = (q0 + t) * 128, r_last = r_first + 127;
        const float c = p.c;
        const uint64_t c2 = pack2(c, c);
        float m = -INFINITY, l = 0.f;
        int n = 0;
        for (int j = 0; j < J; ++j) {
            if (!takes(t, j)) continue;
            const int c0 = kt.tile(j) * kKeys;
            // every row of the stream sees every key of the tile
            const bool all = c0 + kKeys - 1 <= r_first && (c0 > r_last - p.window || c0 + kKeys - 1 < p.sinks);
            mbar_wait(bar(BS + t), (uint32_t)(n & 1), s_abort, &g_async_status, 0x450 + t);
            tc_fence_after_sync();
            uint32_t x[32], y[32];
            tmem_ld32(s_addr, x);
            tmem_ld32(s_addr + 32, y);
            tmem_wait_ld();
            bool no_x = false, no_y = false;              // no row of the warp sees any key of the chunk
            if (!all) {
                const uint32_t sx = visible_columns(r, c0 + ch * 64, p.window, p.sinks);
                const uint32_t sy = visible_columns(r, c0 + ch * 64 + 32, p.window, p.sinks);
                no_x = !__any_sync(0xffffffffu, sx != 0u);
                no_y = !__any_sync(0xffffffffu, sy != 0u);
                if (!no_x && !__all_sync(0xffffffffu, sx == 0xffffffffu)) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[k] = (sx >> k & 1u) ? x[k] : 0xFF800000u;
                }
                if (!no_y && !__all_sync(0xffffffffu, sy == 0xffffffffu)) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) y[k] = (sy >> k & 1u) ? y[k] : 0xFF800000u;
                }
            }
            auto max32 = [&](const uint32_t (&v)[32]) { return fmaxf(max3(max8w(&v[0]), max8w(&v[8]), max8w(&v[16])), max8w(&v[24])); };
            const float mx = fmaxf(no_x ? -INFINITY : max32(x), no_y ? -INFINITY : max32(y)) * c;
            // ---- the maximum moves in some of these rows: both threads of a row go on with the same one -------
            bool rises = mx > m + 8.f;
            if constexpr (L::kHalves == 2) rises = named_bar_or(row_bar, 64, rises);
            else rises = __any_sync(0xffffffffu, rises);
            if (rises) {
                float2 both = make_float2(mx, mx);
                if constexpr (L::kHalves == 2) {
                    sts_f32(xrow + 4u * (uint32_t)ch, mx);
                    named_bar_sync(row_bar, 64);
                    both = lds_f32x2(xrow);
                }
                const float m_new = max3(m, both.x, both.y);
                const float f = m == -INFINITY ? 1.f : ex2_approx(m - m_new);      // (nothing there yet: l = 0, O~ = 0)
                if (n > 0) {
#pragma unroll 1
                    for (int i0 = 0; i0 < kMyCols; i0 += 16) {
                        uint32_t o[16];
                        tmem_ld16(o_addr + i0, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        tmem_st16(o_addr + i0, o);
                    }
                }
                l *= f;
                m = m_new;
            }
            const float mu = m == -INFINITY ? 0.f : -m;
            const uint64_t m2 = pack2(mu, mu);
            uint64_t s01 = 0ull, s23 = 0ull;
            auto weights = [&](int i, const uint32_t (&v)[32], bool none) {
                uint32_t pk[16];
                if (none) {
#pragma unroll
                    for (int k = 0; k < 16; ++k) pk[k] = 0u;
                } else
#pragma unroll
                for (int k = 0; k < 32; k += 4) {
                    float w[4];
                    unpack2(fma2(pack2(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), c2, m2), w[0], w[1]);
                    unpack2(fma2(pack2(__uint_as_float(v[k + 2]), __uint_as_float(v[k + 3])), c2, m2), w[2], w[3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = ex2_approx(w[e]);
                    s01 = add2(s01, pack2(w[0], w[1]));
                    s23 = add2(s23, pack2(w[2], w[3]));
                    pk[k >> 1] = pack16<T16>(w[0], w[1]);
                    pk[(k >> 1) + 1] = pack16<T16>(w[2], w[3]);
                }
                tmem_st16(s_addr + 32 * i, pk);
            };
            auto arrive = [&](int half) {
                tmem_wait_st();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(BP + 2 * t + half));
            };
            weights(1, y, no_y);
            arrive(0);                                    // the tensor core starts on the keys of the second chunks
            weights(0, x, no_x);
            arrive(1);
            float a0, a1, a2, a3;
            unpack2(s01, a0, a1); unpack2(s23, a2, a3);
            l += (a0 + a1) + (a2 + a3);
            ++n;
        }
        // ---- O = O~ / l, through the (now idle) Q tile so that the stores are whole rows --------------------
        const bool good = mbar_wait(bar(BD + t), 0, s_abort, &g_async_status, 0x460 + t) && *s_abort == 0;
        tc_fence_after_sync();
        if constexpr (L::kHalves == 2) {
            named_bar_sync(row_bar, 64);                  // the partner has read the last maxima
            sts_f32(xrow + 4u * (uint32_t)ch, l);
            named_bar_sync(row_bar, 64);
            const float2 both = lds_f32x2(xrow);
            l = both.x + both.y;
        }
        const float inv = 1.f / l;
        constexpr int kChunks = D / 8;                               // 16-byte parts of a row
        const uint32_t stage = sbase + L::kQOff + t * L::kQBytes;
#pragma unroll 1
        for (int i0 = 0; i0 < kMyCols; i0 += 16) {
            uint32_t rr[16];
            tmem_ld16(o_addr + i0, rr);
            tmem_wait_ld();
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = pack16<T16>(__uint_as_float(rr[2 * i]) * inv, __uint_as_float(rr[2 * i + 1]) * inv);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int part = (ch * kMyCols + i0) / 8 + i;
                sts_u32x4(stage + (uint32_t)(row * 2 * D + (part ^ (row & (kChunks - 1))) * 16),
                          make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
            }
        }
        if constexpr (L::kHalves == 2) named_bar_sync(row_bar, 64);
        else __syncwarp();
        T16 *out = reinterpret_cast<T16 *>(p.out) + b * p.os_b + h * p.os_h;
        constexpr int kRowsAtOnce = 32 / kChunks;
#pragma unroll 4
        for (int i = 0; i < kChunks / L::kHalves; ++i) {
            const int rw = q4 * 32 + ch * 16 + i * kRowsAtOnce + lane / kChunks, part = lane % kChunks;
            const uint4 v = lds_u32x4(stage + (uint32_t)(rw * 2 * D + (part ^ (rw & (kChunks - 1))) * 16));
            const int64_t gr = (int64_t)(q0 + t) * 128 + rw;
            if (good && gr < len) *reinterpret_cast<uint4 *>(out + gr * p.os_s + part * 8) = v;
        }
        if (good && ch == 0 && p.lse && r < len) p.lse[((int64_t)b * p.H + h) * p.S + r] = (m + log2f(l)) * 0.69314718055994531f;
        }
    }

    // ---- teardown -------------------------------------------------------------------------------
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kIssuer) { __syncwarp(); tmem_dealloc(tmem, L::kTmemCols); }
}

template <typename T16, int D, int kStreams, int kKeys>
static inline baps_status window_launch(const CUtensorMap *maps, WindowParams &p, cudaStream_t stream)
{
    using L = WinLayout<D, kStreams, kKeys>;
    constexpr auto kernel = window_attention_kernel<T16, D, kStreams, kKeys>;
    p.nitems = (p.S + 128 * kStreams - 1) / (128 * kStreams);
    const long long blocks = (long long)p.B * p.H * p.nitems;
    if (blocks > 0x7fffffffLL) return BAPS_ERR_UNSUPPORTED;
    if ((L::kShares && !has_registers_for<window_attention_kernel<T16, D, kStreams, kKeys>>(kTcSplit)) ||
        cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynBytes) != cudaSuccess)
        return BAPS_ERR_CUDA;
    return launch_kernel(kernel, (unsigned)blocks, L::kThreads, (size_t)L::kDynBytes, stream, maps[0], maps[1], maps[2], p);
}

// Two query tiles per CTA share their K / V stream; one where that leaves SMs without a CTA.
// Measured, us, one / two tiles per CTA (heads x tokens, window).  Fewer pairs of tiles than SMs, where one is taken: 37 x 333, 128: 8.4, 9.5; 28 x 1024,
// all: 18.3, 21.0; 9 x 2048, 512: 13.3, 18.3; 3 x 8192, 4096: 55, 71.  As many and more, two: 37 x 1024, all: 21.7, 21.2; 18 x 2048, 512: 25.4, 18.9; 5 x
// 8192, 4096: 107, 71; but 95 x 333, 128: 14.2, 18.2.  Short of the line, where single tiles of even length come to a second wave, the rule
// is behind: 14 x 2048, 512: 25.0, 18.8; 3 x 8192, 1000: 37, 27.
static inline int window_box_keys(int D) { return D == 64 ? 64 : 128; }
template <typename T16>
static inline baps_status window_shape(const CUtensorMap *maps, WindowParams &p, int D, cudaStream_t stream)
{
    const bool small = (long long)p.B * p.H * ((p.S + 255) / 256) < num_sms();
    if (D == 64) return window_launch<T16, 64, 1, 64>(maps, p, stream);
    return small ? window_launch<T16, 128, 1, 128>(maps, p, stream) : window_launch<T16, 128, 2, 128>(maps, p, stream);
}

} // namespace baps
