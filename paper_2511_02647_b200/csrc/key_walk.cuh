// Which keys a row sees, through a window or in a 4-bit cache, and how the tiles of a walk over them are counted.  Plain arithmetic on ints up to 2^31 - 1,
// for host and device: no sum here passes the last key, so none wraps where a segment or a cache is as long as an int counts.
#pragma once

namespace fedattn {

// tiles of `size` keys that n keys take
__host__ __device__ constexpr int tiles_for(int n, int size) { return n > 0 ? (n - 1) / size + 1 : 0; }

// Which keys of its segment (or cache) of `len` rows row i sees through a window: those at a distance below `window`, not behind it
// when causal, and the first n_sink (causal: as far as they are not behind it): [lo, hi) and [0, sink).  A decode row stands at
// len - 1 (the last cached row), causal.
struct WindowRule {
    int lo, hi, sink;
    __host__ __device__ WindowRule(int i, int len, int window, int n_sink, bool causal)
    {
        lo = i >= window ? i - window + 1 : 0;
        hi = causal ? i + 1 : (len - i > window ? i + window : len);
        const int most = causal ? i + 1 : len;
        sink = n_sink < most ? n_sink : most;
    }
};

// The keys that some row of a tile of rows sees, counted through: the sinks, then, right behind them, those from the first row's window on.
// first, last: what the tile's first and last row see.
struct WindowKeys {
    int n_sinks, gap, n;          // sinks, how far the keys behind them are moved, all keys
    __host__ __device__ WindowKeys() : n_sinks(0), gap(0), n(0) {}
    __host__ __device__ WindowKeys(const WindowRule &first, const WindowRule &last, int len) : WindowKeys()
    {
        if (len <= 0) return;
        n_sinks = last.sink;
        gap = first.lo > n_sinks ? first.lo - n_sinks : 0;
        n = last.hi - gap > n_sinks ? last.hi - gap : n_sinks;
    }
    // the i-th of them, 0 <= i < n, from the segment's start
    __host__ __device__ int at(int i) const { return i + (i >= n_sinks ? gap : 0); }
    // of tile t (one of tiles_for(n, size)): how many there are from its first key on
    __host__ __device__ int left(int t, int size) const { return n - t * size; }
    // its key x, or the last of all where x lies behind that
    __host__ __device__ int in_tile(int t, int size, int x) const
    {
        const int most = left(t, size) - 1;
        return at(t * size + (x < most ? x : most));
    }
};

// Which keys a cache of `rows` rows shows to its new token: [0, a) and [b, len).  window 0: all of them.  The walk goes over the tiles of kKeys
// keys 0 .. n_a - 1, then t_b and on.
template <int kKeys> struct CacheWalk {
    int a, b, len, n_a, t_b, n_tiles;
    __host__ __device__ CacheWalk(int rows, int window, int n_sink)
    {
        len = rows > 0 ? rows : 0;
        a = b = len;
        if (window > 0 && window < len) { b = len - window; a = n_sink < b ? n_sink : b; }
        const int n_t = tiles_for(len, kKeys);
        n_a = tiles_for(a, kKeys);
        t_b = b / kKeys > n_a ? b / kKeys : n_a;
        n_tiles = n_a + (b < len ? n_t - t_b : 0);
    }
    // the first key of a tile of the walk
    __host__ __device__ int key0(int tile) const { return (tile < n_a ? tile : t_b + (tile - n_a)) * kKeys; }
    __host__ __device__ bool sees(int key) const { return key < a || (key >= b && key < len); }
    // whether it sees kKeys keys from key0 on
    __host__ __device__ bool sees_all(int key0) const 
    {
        const unsigned end = (unsigned)key0 + kKeys;            // up to 2^31
        return end <= (unsigned)a || (key0 >= b && end <= (unsigned)len);
    }
};

}  // namespace fedattn
