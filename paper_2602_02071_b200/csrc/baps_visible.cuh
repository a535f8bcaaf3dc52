// Which keys a query of the serving attention sees: the query at position p sees key j where j <= p and (j > p - window or
// j < sinks).
// Integer arithmetic only: compiles for the device, and by itself as plain C++ (the CPU test does so, under a check for overflow).
#pragma once
#include <cstdint>
#ifdef __CUDACC__
#define BAPS_SEE_HD __host__ __device__ __forceinline__
#else
#define BAPS_SEE_HD inline
#endif

namespace baps {

// A window of `places` keys hides nothing from a sequence of that length, however much longer the caller's is.  The kernels get
// this one, so that position - window stays an int for the cache's positions, from -16 (queries before a short sequence's first
// key) up, and position - window - b0 for a prompt's rows and the columns of their tiles.
constexpr int kMostPlaces = 0x7fffff00;               // of a prompt
BAPS_SEE_HD int limited_window(int window, int64_t places) { return window < places ? window : (int)places; }

BAPS_SEE_HD bool sees(int position, int key, int window, int sinks)
{
    return key <= position && (key > position - window || key < sinks);
}

// Keys b0 .. b0 + 31 that the query at `position` >= 0 sees, as bits; b0 at most 2^8 behind it.
BAPS_SEE_HD uint32_t visible_columns(int position, int b0, int window, int sinks)
{
    struct { BAPS_SEE_HD uint32_t operator()(int n) const { return n <= 0 ? 0u : n >= 32 ? 0xffffffffu : (1u << n) - 1u; } } first;
    const uint32_t behind = first(position + 1 - b0);
    return behind & (~first(position - window + 1 - b0) | first(sinks - b0));
}

// Key tiles that rows [r0, r1] see (r0 <= r1): first tokens' tiles 0 .. ns - 1, then w0 .. w1.
struct KeyTiles {
    int ns, w0, w1;
    BAPS_SEE_HD int count() const { return ns + w1 - w0 + 1; }
    BAPS_SEE_HD int tile(int i) const { return i < ns ? i : w0 + i - ns; }
    BAPS_SEE_HD bool has(int tile) const { return tile < ns || (tile >= w0 && tile <= w1); }
};
BAPS_SEE_HD KeyTiles key_tiles(int r0, int r1, int window, int sinks, int log2_tile)
{
    const int lo = r0 - window >= 0 ? r0 - window + 1 : 0;          // (no overflow: r0 >= 0, window >= 1)
    KeyTiles k;
    k.w0 = lo >> log2_tile;
    k.w1 = r1 >> log2_tile;
    const int seen = sinks < lo ? sinks : lo;                       // first tokens left of the window
    k.ns = seen > 0 ? ((seen - 1) >> log2_tile) + 1 : 0;
    if (k.ns > k.w0) k.ns = k.w0;
    return k;
}

} // namespace baps
