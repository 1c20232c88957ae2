"""The walks over keys (csrc/key_walk.cuh) on the CPU: the header is compiled for the host with sums that trap when they wrap,
and compared with the definition, for short lengths key by key and for lengths up to 2^31 - 1 around every border."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_02647_b200", "csrc")
FLAGS = ["-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=signed-integer-overflow", "-fsanitize-undefined-trap-on-error",
         "-D__host__=", "-D__device__="]

HEAD = r"""
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <set>
#include <vector>
#include "key_walk.cuh"
using namespace fedattn;
typedef int64_t ll;
constexpr int kMost = 2147483647;
#define CHECK(x) do { if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); } } while (0)
"""

WINDOW = HEAD + r"""
// [lo, hi) and [0, sink) of row i, in 64 bits
struct Seen { ll lo, hi, sink; bool operator()(ll j) const { return (j >= lo && j < hi) || j < sink; } };
static Seen seen_of(ll i, ll len, ll window, ll n_sink, bool causal)
{
    const ll end = causal ? i + 1 : len;
    return {std::max(i - window + 1, (ll)0), std::min(i + window, end), std::min(n_sink, end)};
}
// The tiles of `size` keys that rows first .. last walk over.
static void check(int len, int first, int last, int window, int n_sink, bool causal, int size, bool every_tile)
{
    const Seen a = seen_of(first, len, window, n_sink, causal), b = seen_of(last, len, window, n_sink, causal);
    const WindowRule fa(first, len, window, n_sink, causal), fb(last, len, window, n_sink, causal);
    CHECK(fa.lo == a.lo && fa.hi == a.hi && fa.sink == a.sink && fb.lo == b.lo && fb.hi == b.hi && fb.sink == b.sink);
    const WindowKeys keys(fa, fb, len);
    const ll n = std::max(b.hi - std::max(a.lo, b.sink), (ll)0) + b.sink;       // sinks, and what lies behind them
    CHECK(keys.n == n);
    auto key = [&](ll i) { return i < b.sink ? i : std::max(a.lo, b.sink) + (i - b.sink); };
    const int tiles = tiles_for(keys.n, size);
    CHECK(tiles == (n + size - 1) / size);
    std::set<int> at;
    for (int t : {0, 1, tiles - 2, tiles - 1, keys.n_sinks / size - 1, keys.n_sinks / size, keys.n_sinks / size + 1}) at.insert(t);
    if (every_tile) for (int t = 0; t < tiles; ++t) at.insert(t);
    for (int t : at) {
        if (t < 0 || t >= tiles) continue;
        CHECK(keys.left(t, size) == n - (ll)t * size && keys.at(t * size) == key((ll)t * size));
        for (int x = 0; x < size; ++x) {
            const ll i = (ll)t * size + x;
            CHECK((x < keys.left(t, size)) == (i < n));
            CHECK(keys.in_tile(t, size, x) == key(std::min(i, n - 1)));
        }
    }
    if (every_tile) {                                           // nothing that a row sees is left out, nothing comes twice
        std::vector<int> times(len);
        for (ll i = 0; i < n; ++i) { CHECK(key(i) >= 0 && key(i) < len); ++times[key(i)]; }
        for (int i = first; i <= last; ++i)
            for (int j = 0; j < len; ++j) CHECK(times[j] <= 1 && (times[j] == 1 || !seen_of(i, len, window, n_sink, causal)(j)));
    }
}

int main()
{
    for (int size : {64, 128}) {
        for (int n = 1; n <= 3; ++n) CHECK(tiles_for(n * size, size) == n && tiles_for(n * size + 1, size) == n + 1);
        CHECK(tiles_for(0, size) == 0 && tiles_for(-5, size) == 0 && tiles_for(kMost, size) == (kMost - 1) / size + 1);
        for (int causal = 0; causal < 2; ++causal) {
            for (int len : {1, 2, 63, 64, 65, 128, 200})
                for (int window : {1, 2, 31, 64, 100, 199, 200, 201, kMost})
                    for (int sink : {0, 1, 5, 64, 130, 200, kMost})
                        for (int first = 0; first < len; first += 1 + len / 9) {
                            check(len, first, std::min(first + 31, len - 1), window, sink, causal, size, true);
                            check(len, first, first, window, sink, causal, size, true);
                        }
            for (int len : {kMost, kMost - 1, kMost - 2, kMost - 3, kMost - 4, kMost - 63, kMost - 64, kMost - 127, kMost - 128, kMost - 1000})
                for (int window : {1, 2, 100, len - 1, len, kMost})
                    for (int sink : {0, 1, 5, 100, len - 200, len - 1, kMost})
                        for (int first : {0, 1, len / 2, len - 40, len - 2, len - 1})
                            for (int last : {first, std::min(first, len - 32) + 31})
                                if (last >= first) check(len, first, last, window, sink, causal, size, false);
        }
        const WindowRule none(-1, 0, 5, 3, true);
        CHECK(WindowKeys(none, none, 0).n == 0);
    }
    return 0;
}
"""

CACHE = HEAD + r"""
constexpr int kKeys = 32;
static void check(int rows, int window, int n_sink, bool every_key)
{
    const CacheWalk<kKeys> w(rows, window, n_sink);
    const ll len = std::max(rows, 0);
    auto seen = [&](ll j) { return j >= 0 && j < len && (window == 0 || j >= len - window || j < n_sink); };
    CHECK(w.n_tiles >= 0 && w.n_tiles <= (len + kKeys - 1) / kKeys);
    std::vector<int> times(every_key ? len : 0);
    std::set<int> tiles;
    for (int t : {0, 1, w.n_a - 2, w.n_a - 1, w.n_a, w.n_a + 1, w.n_tiles - 2, w.n_tiles - 1}) tiles.insert(t);
    if (every_key) for (int t = 0; t < w.n_tiles; ++t) tiles.insert(t);
    for (int t : tiles) {
        if (t < 0 || t >= w.n_tiles) continue;
        const int k0 = w.key0(t);
        CHECK(k0 >= 0 && k0 < len && k0 % kKeys == 0 && (t == 0 || w.key0(t - 1) < k0));
        bool all = true;
        for (int x = 0; x < kKeys; ++x) {
            const ll j = (ll)k0 + x;
            if (j <= kMost) CHECK(w.sees((int)j) == seen(j));
            all = all && seen(j);
            if (every_key && j < len) ++times[j];
        }
        CHECK(!w.sees_all(k0) || all);
        CHECK(w.sees_all(k0) || !all || (k0 < w.a && w.a >= w.b));          // (sinks that end where the window begins may be tested)
    }
    for (int j = 0; j < (every_key ? len : 0); ++j) CHECK(times[j] <= 1 && (!seen(j) || times[j] == 1));
    if (!every_key && len > 0) {                                // the ends of both ranges are in the walk's first and last tiles
        CHECK(w.key0(w.n_tiles - 1) == (len - 1) / kKeys * kKeys);
        if (window == 0 || window >= len) CHECK(w.n_tiles == (len - 1) / kKeys + 1);
    }
}

int main()
{
    for (int rows : {-7, 0, 1, 2, 31, 32, 33, 63, 64, 100, 257})
        for (int window : {0, 1, 2, 31, 32, 33, 100, 256, 257, 300, kMost})
            for (int sink : {0, 1, 5, 31, 32, 33, 64, 200, 257, kMost}) check(rows, window, sink, true);
    for (int rows : {kMost - 15, kMost - 16, kMost - 17, kMost - 20, kMost - 30, kMost - 31, kMost - 32, kMost - 33, kMost - 1000})
        for (int window : {0, 1, 33, 1000, rows - 1, rows, kMost})
            for (int sink : {0, 1, 40, rows - 100, rows - 1, kMost}) check(rows, window, sink, false);
    return 0;
}
"""


def run(tmp_path, text):
    if not shutil.which("g++"):
        pytest.skip("needs g++")
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(text)
    subprocess.check_call(["g++", *FLAGS, "-I", CSRC, str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout or "a sum wrapped (signal %d)" % -r.returncode


def test_window_keys(tmp_path):
    run(tmp_path, WINDOW)


def test_cache_walk(tmp_path):
    run(tmp_path, CACHE)
