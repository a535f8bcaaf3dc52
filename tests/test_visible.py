"""Which keys the serving attention's queries see (``csrc/baps_visible.cuh``, compiled here as plain C++ with every signed
overflow an error) against the definition in 64 bits, up to the longest sequences and windows of any int."""
import os
import re
import subprocess

from paper_2602_02071_b200 import build

PROGRAM = r"""
#include "baps_visible.cuh"
#include <cstdio>
#include <cstdlib>
using namespace baps;
static bool plain(int64_t p, int64_t j, int64_t window, int64_t sinks) { return j <= p && (j > p - window || j < sinks); }
static long long checked = 0;
static void check(bool ok, const char *what, long long S, long long r, long long j, long long window, long long sinks)
{
    ++checked;
    if (ok) return;
    std::printf("%s: S %lld position %lld key %lld window %lld sinks %lld\n", what, S, r, j, window, sinks);
    std::exit(1);
}
int main()
{
    const int top = 0x7fffffff, lengths[] = {1, 2, 33, 200, 4097, 1 << 20, kMostPlaces - 1, kMostPlaces};
    for (int S : lengths) {
        const int windows[] = {1, 2, 31, 100, 128, S - 1 > 0 ? S - 1 : 1, S, top - 1, top}, sink_counts[] = {0, 1, 37, 128, S - 1, S, top};
        for (int given : windows) for (int sinks : sink_counts) {
            const int window = limited_window(given, S);
            const int64_t at[] = {0, 1, 30, 127, 128, S / 2, (int64_t)S - 129, (int64_t)S - 2, (int64_t)S - 1};
            for (int64_t r64 : at) {
                if (r64 < 0 || r64 >= S) continue;
                const int r = (int)r64, tile = r & ~127;
                // every chunk of 32 keys of the row's own 128-key tile, of the first one and of those at the window's edge
                const int64_t edge = (int64_t)r - given + 1 > 0 ? (int64_t)r - given + 1 : 0;
                const int tiles[] = {tile, 0, (int)(edge & ~127)};
                for (int c0 : tiles) for (int b0 = c0; b0 < c0 + 128; b0 += 32) {
                    const uint32_t bits = visible_columns(r, b0, window, sinks);
                    for (int k = 0; k < 32; ++k) check((bits >> k & 1u) == plain(r, (int64_t)b0 + k, given, sinks), "columns", S, r, (int64_t)b0 + k, given, sinks);
                }
                // the tiles of 64 and 128 keys hold every key that a row of [r, r + 127] sees, and no tile is named twice
                for (int log2_tile = 6; log2_tile <= 7; ++log2_tile) {
                    const int r1 = (int)(r64 + 127 < S ? r64 + 127 : S - 1);
                    const KeyTiles t = key_tiles(r, r1, window, sinks, log2_tile);
                    check(t.ns <= t.w0 && t.w0 <= t.w1 && t.count() >= 1 && t.tile(t.count() - 1) == t.w1, "tiles", S, r, 0, given, sinks);
                    const int64_t keys[] = {0, 1, 63, 64, 128, sinks - 1, sinks, edge - 1, edge, edge + 64, r64 - 1, r64, r1};
                    for (int64_t j : keys)
                        if (j >= 0 && j < S && (plain(r, j, given, sinks) || plain(r1, j, given, sinks)))
                            check(t.has((int)(j >> log2_tile)), "tile of a key", S, r, j, given, sinks);
                }
            }
            // queries of the cache: positions from -16 on
            for (int64_t p = -16; p < 40 && p < S; ++p)
                for (int64_t j = 0; j < 64 && j < S; ++j) check(sees((int)p, (int)j, window, sinks) == plain(p, j, given, sinks), "sees", S, p, j, given, sinks);
        }
    }
    const int most = top - 64;                    // places of a cache
    const int positions[] = {-16, -1, 0, 5, most - 2, most - 1}, windows[] = {1, 7, most - 1, most, top};
    for (int p : positions) for (int given : windows) for (int j = most - 40; j < most; ++j)
        check(sees(p, j, limited_window(given, most), 3) == plain(p, j, given, 3), "sees", most, p, j, given, 3);
    std::printf("%lld\n", checked);
}
"""


def test_visibility_without_overflow(tmp_path):
    (tmp_path / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", build.CSRC, "-o", str(tmp_path / "main"),
                    str(tmp_path / "main.cpp")], check=True)
    res = subprocess.run([str(tmp_path / "main")], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
    assert int(res.stdout) > 100000


def test_the_kernels_are_given_the_limited_window():
    code = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "baps_serving.cu")).read())
    assert re.findall(r"p\.window = ([^;]*);", code) == ["limited_window(window, S)", "limited_window(window, places)", "window"]    # (fork: 64 bits)
    pages = open(os.path.join(build.CSRC, "baps_kv_pages.cuh")).read()
    assert re.findall(r"[^\n]*p\.window[^\n]*", pages) == ["    if (!(from < p.sinks || to > (int64_t)r.length - p.window + 1)) return -1;"]
