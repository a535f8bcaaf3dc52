// New keys and values into the pages of the 8-bit cache.
//
// Per page and head, for K and for V:  a = largest finite |x| of the new elements (at least 2^-100),
//     s = smallest 2^e with a <= 448 s, not below the old scale where older tokens stay;   code = E4M3(x / s),
// and, where s grew, code' = E4M3(value(code) * old / s) for the rest of the page.  Scales are powers of two, so x / s is exact
// and every element is rounded once (again only where a grown scale makes it subnormal).
//
// What bounds it: memory for prompts (two bytes read, one written per element), launch and two dependent loads (table, then
// scale) for single tokens.  A group of warps owns one page and head of K or of V, keeps what it has read in registers
// between the maximum and the conversion, and so reads its tokens once.  A thread holds eight times 16 bytes at most and the
// kernel is held to 64 registers, so that an SM has 1024 threads' loads in flight (128 KB): 12 prompts of up to 8K tokens, 8 heads of
// 128, pages of 64: 84 us (5.9 TB/s), 93 us with 91 registers and 640 threads.  The forms in which a thread holds eight loads, this one among them, spill
// 44 bytes, or 72 where one warp has a page to itself (16 tokens of 128, 32 of 64); the others nothing.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "baps_common.cuh"
#include "baps_sm100.cuh"

namespace baps {

struct KvAppendParams {
    const void *src[2];                 // K, V
    uint8_t *codes[2];
    float *scale[2];
    int64_t token_stride[2], head_stride[2];
    int64_t n_tokens;
    const int32_t *starts, *lengths, *table;
    int table_width, B, Hkv, n_pages, max_new;
};

constexpr int kAppendThreads = 128;    // of a block, at least
constexpr int kAppendFew = 8;           // new tokens of a sequence up to which a call is one of few rows per page

// smallest power of two s with a <= 448 s = 1.75 * 2^8 s, for 2^-100 <= a < infinity
__device__ __forceinline__ float scale_for(float a)
{
    const uint32_t bits = __float_as_uint(fmaxf(a, 7.888609052210118e-31f));
    const uint32_t over = (bits & 0x7fffffu) > 0x600000u ? 1u : 0u;              // mantissa above 1.75
    return __uint_as_float(((bits >> 23) - 8u + over) << 23);
}
__device__ __forceinline__ float pow2_inverse(float s) { return __uint_as_float(0x7f000000u - __float_as_uint(s)); }

// four codes of x[0..3], the first in the lowest byte; to nearest even, saturating, NaN to 0x7f
__device__ __forceinline__ uint32_t e4m3x4(const float *x)
{
    uint16_t lo, hi;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x[1]), "f"(x[0]));
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x[3]), "f"(x[2]));
    return (uint32_t)lo | (uint32_t)hi << 16;
}
__device__ __forceinline__ void e4m3x4_values(uint32_t codes, float *x)
{
    uint32_t h0, h1;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h0) : "h"((uint16_t)codes));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h1) : "h"((uint16_t)(codes >> 16)));
    const float2 a = __half22float2(*reinterpret_cast<__half2 *>(&h0)), b = __half22float2(*reinterpret_cast<__half2 *>(&h1));
    x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
}
template <typename T16>
__device__ __forceinline__ float2 values2(uint32_t pair)
{
    if constexpr (__is_same(T16, __half)) return __half22float2(*reinterpret_cast<__half2 *>(&pair));
    else return make_float2(__uint_as_float(pair << 16), __uint_as_float(pair & 0xffff0000u));
}

// kRowsMost: new tokens that a page can get in a call; kWarps: warps that share a page and head.
template <int D, int kRowsMost>
struct AppendShape {
    // (two warps per page, which share a barrier and hold more each, lost to four: 107 to 93 us with pages of 32, 56 to 49 at D = 64)
    static constexpr int kWarps = kRowsMost * D <= 2048 ? 1 : kRowsMost * D <= 8192 ? 4 : 8;
    static constexpr int kThreads = kWarps > 4 ? 32 * kWarps : kAppendThreads, kItems = kThreads / (32 * kWarps);
};

template <typename T16, int D, int kPage, int kRowsMost>
__global__ void __launch_bounds__(AppendShape<D, kRowsMost>::kThreads, 1024 / AppendShape<D, kRowsMost>::kThreads)
kv_append_kernel(const KvAppendParams p)
{
    using A = AppendShape<D, kRowsMost>;
    constexpr int kWarps = A::kWarps, kItems = A::kItems, kGroup = kWarps * 32;
    constexpr int kParts = D / 8;                                  // 8-element parts of a row, one per thread
    constexpr int kRows = kGroup / kParts;                         // rows in one step of the group
    constexpr int kSteps = (kRowsMost + kRows - 1) / kRows;
    static_assert(kSteps >= 1 && kSteps <= 8, "what a thread keeps of a page");
    __shared__ float s_max[A::kThreads / 32];
    allow_next_kernel();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int group = warp / kWarps, in_group = (int)threadIdx.x % kGroup;
    // item: K or V of one head; blocks: x items, then pages of the sequence, z sequence.  Items first: a token's heads stand
    // beside each other, so neighbouring blocks read one run of memory (the prompts above: 126 us the other way, 92 then).
    const int item_blocks = (2 * p.Hkv + kItems - 1) / kItems;
    const int item = (int)(blockIdx.x % item_blocks) * kItems + group;
    const int *lengths = await_previous_kernel(p.lengths);
    if (item >= 2 * p.Hkv) return;                                 // (here and below: a whole group, which shares no barrier with others)
    const int which = item >= p.Hkv ? 1 : 0, head = item - which * p.Hkv;
    const int64_t held = max(lengths[blockIdx.z], 0);
    const int64_t t0 = min((int64_t)max(p.starts[blockIdx.z], 0), p.n_tokens);
    const int64_t t1 = min(min((int64_t)max(p.starts[blockIdx.z + 1], 0), p.n_tokens), t0 + p.max_new);
    const int64_t page_no = held / kPage + blockIdx.x / item_blocks;
    const int64_t lo = max(held, page_no * kPage), hi = min(held + (t1 - t0), (page_no + 1) * kPage);
    if (lo >= hi || page_no >= p.table_width) return;
    const int page = p.table[(int64_t)blockIdx.z * p.table_width + page_no];
    const int slot0 = (int)(lo - page_no * kPage), n = (int)(hi - lo);          // places slot0 .. slot0 + n - 1
    const int part = in_group % kParts, row0 = in_group / kParts;
    const T16 *src = reinterpret_cast<const T16 *>(p.src[which]) + (t0 + (lo - held)) * p.token_stride[which] +
                     head * p.head_stride[which] + part * 8;
    uint4 x[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int row = i * kRows + row0;
        x[i] = row < n ? *reinterpret_cast<const uint4 *>(src + row * p.token_stride[which]) : make_uint4(0, 0, 0, 0);
    }
    // (the page's number is only now needed: its load and those of the tokens are on their way together)
    if (page < 0 || page >= p.n_pages) return;
    uint8_t *codes = p.codes[which] + ((int64_t)page * p.Hkv + head) * (kPage * D) + part * 8;
    float *scale_at = p.scale[which] + (int64_t)page * p.Hkv + head;
    const float old = slot0 > 0 ? *scale_at : 0.f;

    float a = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 v = values2<T16>(w[k]);
            const float v0 = fabsf(v.x), v1 = fabsf(v.y);
            a = fmaxf(a, v0 < INFINITY ? v0 : 0.f);                // (NaN: the comparison fails too)
            a = fmaxf(a, v1 < INFINITY ? v1 : 0.f);
        }
    }
    a = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(a)));      // a >= 0: ordered like its bits
    if constexpr (kWarps > 1) {
        if (lane == 0) s_max[warp] = a;
        named_bar_sync(1 + group, kGroup);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) a = fmaxf(a, s_max[group * kWarps + w]);
    }
    const float s = fmaxf(scale_for(a), old), inv = pow2_inverse(s);
    __syncwarp();                                                  // every lane has read the old scale
    if (in_group == 0) *scale_at = s;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        const int row = i * kRows + row0;
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float2 u = values2<T16>(w[k]);
            v[2 * k] = u.x * inv; v[2 * k + 1] = u.y * inv;
        }
        if (row < n) *reinterpret_cast<uint2 *>(codes + (slot0 + row) * D) = make_uint2(e4m3x4(v), e4m3x4(v + 4));
    }
    if (slot0 > 0 && s > old) {                                    // the rest of the page against the grown scale
        const float f = old * inv;
#pragma unroll 4
        for (int row = row0; row < kPage; row += kRows) {
            if (row >= slot0 && row < slot0 + n) continue;
            uint2 *at = reinterpret_cast<uint2 *>(codes + row * D);
            const uint2 c = *at;
            float v[8];
            e4m3x4_values(c.x, v); e4m3x4_values(c.y, v + 4);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= f;
            *at = make_uint2(e4m3x4(v), e4m3x4(v + 4));
        }
    }
}

template <typename T16, int D, int kPage, int kRowsMost>
static inline baps_status kv_append_launch(const KvAppendParams &p, cudaStream_t stream)
{
    using A = AppendShape<D, kRowsMost>;
    // pages that max_new tokens can touch, wherever the first one stands
    const int64_t pages = ((int64_t)p.max_new + 2 * kPage - 2) / kPage;
    const int64_t blocks = pages * ((2 * p.Hkv + A::kItems - 1) / A::kItems);
    if (blocks > 0x7fffffffLL) return BAPS_ERR_UNSUPPORTED;
    return launch_kernel(kv_append_kernel<T16, D, kPage, kRowsMost>, dim3((unsigned)blocks, 1, (unsigned)p.B), A::kThreads, 0, stream, p);
}
// Few tokens per sequence: a page gets no more rows than that, and fewer threads read them.  Measured, us, few / whole pages: 96 sequences, 8 heads of
// 128, pages of 64: one token 2.8, 5.7, eight 3.1, 7.0; pages of 16: 2.8, 3.2 and 3.1, 4.4; 8 sequences 1.7, 2.4 and 1.8, 3.0.  (A third form for up
// to 16 tokens would gain too: 16 of them 4.6 for 7.3.)
template <typename T16, int D, int kPage>
static inline baps_status kv_append_rows(const KvAppendParams &p, cudaStream_t stream)
{
    return p.max_new <= kAppendFew ? kv_append_launch<T16, D, kPage, kAppendFew>(p, stream) : kv_append_launch<T16, D, kPage, kPage>(p, stream);
}

template <typename T16, int D>
static inline baps_status kv_append_page(const KvAppendParams &p, int page, cudaStream_t stream)
{
    switch (page) {
    case 16: return kv_append_rows<T16, D, 16>(p, stream);
    case 32: return kv_append_rows<T16, D, 32>(p, stream);
    case 64: return kv_append_rows<T16, D, 64>(p, stream);
    default: return kv_append_rows<T16, D, 128>(p, stream);
    }
}

} // namespace baps
