// C-ABI entry points of the serving operators (declared in include/baps.h): windowed attention of prompts, the 8-bit
// key-value cache, attention over it, its pages.
#include "baps_common.cuh"
#include "baps_attention_window.cuh"
#include "baps_kv_append.cuh"
#include "baps_kv_attention.cuh"
#include "baps_kv_pages.cuh"

#include <cmath>

using namespace baps;

namespace {

bool strides_ok(const int64_t *s, int n)
{
    for (int i = 0; i < n; ++i)
        if (s[i] < 8 || s[i] % 8 != 0 || s[i] >= (int64_t)1 << 38) return false;      // TMA: below 2^40 bytes
    return true;
}

float base2_scale(float scale, int D) { return (float)(1.4426950408889634074 * (scale > 0.f ? (double)scale : 1.0 / std::sqrt((double)D))); }

// Visibility, scale and type, shared by the two attention calls.
baps_status check_softmax(int window, int sinks, float scale, int dtype)
{
    // (a scale that is infinite in base 2 makes NaN of a score of 0)
    if (window < 1 || sinks < 0 || !(scale >= 0.f) || !std::isfinite(base2_scale(scale, 64))) return BAPS_ERR_INVALID_ARG;
    return dtype == BAPS_DTYPE_BF16 || dtype == BAPS_DTYPE_F16 ? BAPS_OK : BAPS_ERR_UNSUPPORTED;
}

baps_status check_cache(const baps_kv_cache *c)
{
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale) return BAPS_ERR_INVALID_ARG;
    if (c->n_pages <= 0 || c->Hkv <= 0) return BAPS_ERR_INVALID_ARG;
    if ((c->page != 16 && c->page != 32 && c->page != 64 && c->page != 128) || (c->D != 64 && c->D != 128)) return BAPS_ERR_UNSUPPORTED;
    if ((int64_t)c->n_pages * c->Hkv * c->page > 0x7fffffffLL || c->Hkv > 32767) return BAPS_ERR_UNSUPPORTED;   // 32-bit row number
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned4(c->k_scale) || !aligned4(c->v_scale)) return BAPS_ERR_ALIGNMENT;
    return BAPS_OK;
}

KvPool pool_of(const baps_kv_cache *c)
{
    return {{c->k, c->v}, {c->k_scale, c->v_scale}, c->n_pages, c->Hkv, c->page, (int64_t)c->Hkv * c->page * c->D};
}

size_t pages_workspace(int64_t rows, int64_t n_pages) { return (size_t)(2 * rows + 2 * n_pages + n_pages / 1024 + 16) * 4; }

} // namespace

namespace baps {
baps_status take_serving_status() { return take_async_status(); }
}

extern "C" {

#ifdef BAPS_TEST_SKIP_LOAD
// Test build only: as baps_test_skip_kv_load, for the windowed attention.
int baps_test_skip_window_load(int l)
{
    return cudaMemcpyToSymbol(g_test_skip_window_load, &l, sizeof(int)) == cudaSuccess ? 0 : -1;
}
#endif

baps_status baps_attention_window_fwd(const void *q, const void *k, const void *v, void *out, float *lse,
                                      const int32_t *lengths, const int64_t *strides, int B, int H, int Hkv, int S,
                                      int D, int window, int sinks, float scale, int dtype, baps_stream stream)
{
    if (!q || !k || !v || !out) return BAPS_ERR_INVALID_ARG;
    if (B <= 0 || H <= 0 || Hkv <= 0 || S <= 0 || D <= 0 || H % Hkv != 0) return BAPS_ERR_INVALID_ARG;
    const baps_status st = check_softmax(window, sinks, scale, dtype);
    if (st != BAPS_OK) return st;
    if ((D != 64 && D != 128) || B > 65535 || H > 65535 || S > kMostPlaces) return BAPS_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned4(lse) || !aligned4(lengths)) return BAPS_ERR_ALIGNMENT;
    int64_t s[12];
    for (int i = 0; i < 4; ++i) {
        const int heads = i == 1 || i == 2 ? Hkv : H;
        s[3 * i] = (int64_t)heads * S * D; s[3 * i + 1] = (int64_t)S * D; s[3 * i + 2] = D;
        if (strides)
            for (int d = 0; d < 3; ++d) s[3 * i + d] = strides[3 * i + d];
    }
    if (!strides_ok(s, 12)) return strides ? BAPS_ERR_INVALID_ARG : BAPS_ERR_UNSUPPORTED;
    if (!have_device()) return BAPS_ERR_CUDA;
    CUtensorMap maps[3];
    const bool half = dtype == BAPS_DTYPE_F16;
    const uint32_t keys = (uint32_t)window_box_keys(D);
    if (!make_tmap_heads16(maps, q, half, B, H, S, D, s, 128) || !make_tmap_heads16(maps + 1, k, half, B, Hkv, S, D, s + 3, keys) ||
        !make_tmap_heads16(maps + 2, v, half, B, Hkv, S, D, s + 6, keys))
        return BAPS_ERR_CUDA;
    WindowParams p;
    p.out = out; p.lse = lse; p.lengths = lengths;
    p.os_b = s[9]; p.os_h = s[10]; p.os_s = s[11];
    p.B = B; p.H = H; p.Hkv = Hkv; p.S = S; p.window = limited_window(window, S); p.sinks = sinks;
    p.c = base2_scale(scale, D);
    return half ? window_shape<__half>(maps, p, D, as_stream(stream)) : window_shape<__nv_bfloat16>(maps, p, D, as_stream(stream));
}

baps_status baps_kv_append(const baps_kv_cache *cache, const void *k_new, const void *v_new, const int64_t *strides,
                           int64_t n_tokens, const int32_t *starts, const int32_t *lengths, const int32_t *table,
                           int table_width, int B, int max_new, int dtype, baps_stream stream)
{
    const baps_status st = check_cache(cache);
    if (st != BAPS_OK) return st;
    if (n_tokens < 0 || B < 0 || max_new < 0 || table_width <= 0) return BAPS_ERR_INVALID_ARG;
    if (dtype != BAPS_DTYPE_BF16 && dtype != BAPS_DTYPE_F16) return BAPS_ERR_UNSUPPORTED;
    if (n_tokens == 0 || B == 0 || max_new == 0) return BAPS_OK;
    if (!k_new || !v_new || !starts || !lengths || !table) return BAPS_ERR_INVALID_ARG;
    if (B > 65535) return BAPS_ERR_UNSUPPORTED;
    if (!aligned16(k_new) || !aligned16(v_new) || !aligned4(starts) || !aligned4(lengths) || !aligned4(table)) return BAPS_ERR_ALIGNMENT;
    if (strides && !strides_ok(strides, 4)) return BAPS_ERR_INVALID_ARG;
    if (!have_device()) return BAPS_ERR_CUDA;
    KvAppendParams p;
    p.src[0] = k_new; p.src[1] = v_new;
    p.codes[0] = cache->k; p.codes[1] = cache->v;
    p.scale[0] = cache->k_scale; p.scale[1] = cache->v_scale;
    for (int i = 0; i < 2; ++i) {
        p.token_stride[i] = strides ? strides[2 * i] : (int64_t)cache->Hkv * cache->D;
        p.head_stride[i] = strides ? strides[2 * i + 1] : cache->D;
    }
    p.n_tokens = n_tokens;
    p.starts = starts; p.lengths = lengths; p.table = table;
    p.table_width = table_width; p.B = B; p.Hkv = cache->Hkv; p.n_pages = cache->n_pages;
    p.max_new = (int)(max_new < n_tokens ? max_new : n_tokens);
    cudaStream_t s = as_stream(stream);
    if (dtype == BAPS_DTYPE_F16)
        return cache->D == 128 ? kv_append_page<__half, 128>(p, cache->page, s) : kv_append_page<__half, 64>(p, cache->page, s);
    return cache->D == 128 ? kv_append_page<__nv_bfloat16, 128>(p, cache->page, s) : kv_append_page<__nv_bfloat16, 64>(p, cache->page, s);
}

size_t baps_kv_attention_workspace(int B, int H, int Hkv, int T, int D, int page, int table_width, int window, int sinks)
{
    if (B <= 0 || B > kKvMaxB || H <= 0 || Hkv <= 0 || H % Hkv != 0 || T <= 0 || T > 16 || (D != 64 && D != 128)) return 0;
    if ((page != 16 && page != 32 && page != 64 && page != 128) || table_width <= 0 || window < 1 || sinks < 0) return 0;
    if ((int64_t)T * (H / Hkv) > 65536) return 0;
    return kv_workspace(kv_shape_of(B, Hkv, T * (H / Hkv), D, page, table_width, T, window, sinks), D);
}

baps_status baps_kv_attention(const void *q, void *out, float *lse, const baps_kv_cache *cache, const int32_t *table,
                              int table_width, const int32_t *lengths, const int64_t *strides, int B, int H, int T,
                              int window, int sinks, float scale, int dtype, void *workspace, size_t workspace_bytes,
                              baps_stream stream)
{
    baps_status st = check_cache(cache);
    if (st != BAPS_OK) return st;
    if (!q || !out || !table || !lengths) return BAPS_ERR_INVALID_ARG;
    if (B <= 0 || H <= 0 || T <= 0 || table_width <= 0 || H % cache->Hkv != 0) return BAPS_ERR_INVALID_ARG;
    st = check_softmax(window, sinks, scale, dtype);
    if (st != BAPS_OK) return st;
    if (T > 16 || B > kKvMaxB || (int64_t)T * (H / cache->Hkv) > 65536) return BAPS_ERR_UNSUPPORTED;
    const int64_t places = (int64_t)table_width * cache->page;
    if (places > 0x7fffffff - kKvTile) return BAPS_ERR_UNSUPPORTED;
    if (!aligned16(q) || !aligned16(out) || !aligned4(lse) || !aligned4(table) || !aligned4(lengths) || !aligned16(workspace)) return BAPS_ERR_ALIGNMENT;
    const int D = cache->D;
    int64_t s[6] = {(int64_t)H * T * D, (int64_t)T * D, D, (int64_t)H * T * D, (int64_t)T * D, D};
    if (strides) {
        if (!strides_ok(strides, 6)) return BAPS_ERR_INVALID_ARG;
        for (int i = 0; i < 6; ++i) s[i] = strides[i];
    }
    const int64_t held = kv_held_tiles(cache->page, table_width), seen = kv_seen_tiles(T, window, sinks), tiles = held < seen ? held : seen;
    const KvShape shape = kv_shape_of(B, cache->Hkv, T * (H / cache->Hkv), D, cache->page, table_width, T, window, sinks);
    const size_t need = kv_workspace(shape, D);
    if (need > 0 && (!workspace || workspace_bytes < need)) return BAPS_ERR_INVALID_ARG;
    // tiles of the whole call are a 32-bit count
    if (tiles * B * cache->Hkv * shape.groups > 0x7fffffffLL - 4096) return BAPS_ERR_UNSUPPORTED;
    if (!have_device()) return BAPS_ERR_CUDA;
    KvAttnParams p;
    p.q = q; p.out = out; p.lse = lse;
    p.qs_b = s[0]; p.qs_h = s[1]; p.qs_t = s[2]; p.os_b = s[3]; p.os_h = s[4]; p.os_t = s[5];
    p.table = table; p.lengths = lengths; p.k = cache->k; p.v = cache->v; p.k_scale = cache->k_scale; p.v_scale = cache->v_scale;
    p.width = table_width; p.B = B; p.H = H; p.Hkv = cache->Hkv; p.T = T; p.G = H / cache->Hkv; p.R = T * p.G; p.groups = shape.groups;
    p.n_pages = cache->n_pages; p.page = cache->page; p.window = limited_window(window, places); p.sinks = sinks;
    p.c = base2_scale(scale, D);
    const size_t part_rows = (size_t)shape.ctas * 2 * 8 * shape.tiles;
    p.part_o = static_cast<float *>(workspace);
    p.part_ml = reinterpret_cast<float2 *>(p.part_o + part_rows * D);
    p.desc = reinterpret_cast<int2 *>(p.part_ml + part_rows);
    cudaStream_t cs = as_stream(stream);
    return dtype == BAPS_DTYPE_F16 ? kv_attention_shape<__half>(p, D, shape, cs) : kv_attention_shape<__nv_bfloat16>(p, D, shape, cs);
}

size_t baps_kv_pages_workspace(int rows, int n_pages)
{
    return rows < 0 || n_pages <= 0 ? 0 : pages_workspace(rows, n_pages);
}

baps_status baps_kv_fork(const baps_kv_cache *cache, const int32_t *table, const int32_t *lengths, int rows,
                         const int32_t *refs, const int32_t *parents, int new_rows, int table_width, int reserve,
                         int window, int sinks, int32_t *new_table, int32_t *new_lengths, int32_t *new_refs,
                         void *workspace, size_t workspace_bytes, baps_stream stream)
{
    const baps_status st = check_cache(cache);
    if (st != BAPS_OK) return st;
    if (!table || !lengths || !refs || !parents || !new_table || !new_lengths || !new_refs || !workspace) return BAPS_ERR_INVALID_ARG;
    if (rows <= 0 || new_rows <= 0 || table_width <= 0 || reserve < 0 || window < 1 || sinks < 0) return BAPS_ERR_INVALID_ARG;
    if (rows > kForkRows) return BAPS_ERR_UNSUPPORTED;
    if ((int64_t)new_rows * table_width + new_rows > 0x7fffffffLL) return BAPS_ERR_UNSUPPORTED;
    if (!aligned4(table) || !aligned4(lengths) || !aligned16(refs) || !aligned4(parents) || !aligned4(new_table) ||
        !aligned4(new_lengths) || !aligned4(new_refs) || !aligned16(workspace))
        return BAPS_ERR_ALIGNMENT;
    if (workspace_bytes < pages_workspace(new_rows, cache->n_pages)) return BAPS_ERR_INVALID_ARG;
    if (!have_device()) return BAPS_ERR_CUDA;
    KvForkParams p;
    p.pool = pool_of(cache);
    p.table = table; p.lengths = lengths; p.refs = refs; p.parents = parents;
    p.new_table = new_table; p.new_lengths = new_lengths; p.new_refs = new_refs;
    p.begin = static_cast<int32_t *>(workspace);
    p.first = p.begin + new_rows;
    p.free_pages = p.first + new_rows;
    p.rows = rows; p.new_rows = new_rows; p.width = table_width; p.reserve = reserve; p.window = window; p.sinks = sinks;
    const int64_t asked = (int64_t)new_rows * (((int64_t)reserve + cache->page - 1) / cache->page + 1);
    p.most = (int)(asked < cache->n_pages ? asked : cache->n_pages);
    return kv_fork_launch(p, as_stream(stream));
}

baps_status baps_kv_compact(const baps_kv_cache *cache, const int32_t *table, int rows, int table_width, const int32_t *refs,
                            int32_t *new_table, int32_t *new_refs, int32_t *page_map, int32_t *n_live,
                            void *workspace, size_t workspace_bytes, baps_stream stream)
{
    const baps_status st = check_cache(cache);
    if (st != BAPS_OK) return st;
    if (rows < 0 || table_width < 0) return BAPS_ERR_INVALID_ARG;
    const bool entries = rows > 0 && table_width > 0;
    if ((entries && (!table || !new_table)) || !refs || !new_refs || !page_map || !n_live || !workspace) return BAPS_ERR_INVALID_ARG;
    if (!aligned4(table) || !aligned4(refs) || !aligned4(new_table) || !aligned4(new_refs) || !aligned4(page_map) ||
        !aligned4(n_live) || !aligned16(workspace))
        return BAPS_ERR_ALIGNMENT;
    if (workspace_bytes < pages_workspace(0, cache->n_pages)) return BAPS_ERR_INVALID_ARG;
    if (!have_device()) return BAPS_ERR_CUDA;
    KvCompactParams p;
    p.pool = pool_of(cache);
    p.table = table; p.refs = refs; p.new_table = new_table; p.new_refs = new_refs; p.page_map = page_map; p.n_live = n_live;
    p.chunks = (cache->n_pages + 1023) / 1024;
    p.holes = static_cast<int32_t *>(workspace);
    p.movers = p.holes + cache->n_pages;
    p.chunk_live = p.movers + cache->n_pages;
    p.n_moves = p.chunk_live + p.chunks;
    p.rows = rows; p.width = table_width;
    return kv_compact_launch(p, as_stream(stream));
}

} // extern "C"
