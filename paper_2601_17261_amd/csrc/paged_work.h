// What attention over a cache in pages reckons a row tile's work as, on the device and, for what it comes to at the ends of its ranges, on the host.
#pragma once
#include <stdint.h>

namespace agzo {

// A row tile's work is about the keys that its rows see: first + t step of row tile t of a sequence, so that the work in front of one is a whole number that every
// workgroup finds alike
struct PgWork { int tiles, first, step; };      // of a sequence: its row tiles, the first one's work, and what each has more than the one before

// nq new tokens of G rows each behind and among nk keys, `rows` rows to a tile; start: what a tile's start costs, in keys.  tree: its rows may see all keys.  nq G, nk: below 2^31 - 1024
__host__ __device__ __forceinline__ PgWork pg_work(int nq, int nk, int G, int rows, bool tree, int start) {
    PgWork w;
    w.tiles = (int)(((uint32_t)nq * (uint32_t)G + (rows - 1)) / rows);
    // (rounded up, but down where the last row tile's work, which then is more than the keys, would not be of 32 bits)
    w.step = tree ? 0 : (rows + G - 1) / G;
    if (!tree && nk + (int64_t)w.step * w.tiles > 0x7FFFFFFF - 1024) w.step -= w.step * G != rows;
    const int seen = tree ? nk : nk - nq + w.step;
    w.first = (seen > 0 ? seen : 0) + start;
    return w;
}
__host__ __device__ __forceinline__ int64_t pg_before(const PgWork& w, int t) { return (int64_t)w.first * t + (int64_t)w.step * ((int64_t)t * (t - 1) / 2); }
__host__ __device__ __forceinline__ int pg_of(const PgWork& w, int t) { return w.first + w.step * t; }

}  // namespace agzo
