// How a call of the fully-connected layer in 8-bit integers runs, and where everything lies in its workspace: decided in one place,
// for the query of the workspace's size and for the launches.  Plain host code, no HIP.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace dc {

constexpr int kI8FewRows = 64;           // rows of the kernel of few rows, at most
constexpr int kI8TileSums = 64 * 64;     // sums of a tile that workgroups share

struct I8Plan {
    struct Area { size_t at = 0, bytes = 0; };
    size_t width = 0;          // bytes of a row in 8 bits: K padded with zeros to whole steps
    long tiles = 0;            // of 64 rows x 64 channels
    int splits = 1;            // workgroups that share a tile's K
    bool few = false;          // the kernel of few rows (the rows in tiles, in the order of its fragments) instead of the GEMM
    bool copy = false;         // the GEMM reads padded copies of the weights
    // one row needs none: the kernel rounds it for itself
    Area rows, scales, weights, part, done;      // `part`, `done`: the sums and counters of tiles that workgroups share
    size_t bytes = 0;
};

// Workgroups that share a tile of 64 x 64: as many as give every CU one, with eight stages of K each at least.  Putting the sums together
// costs 2.5 us, so K has to be long: with more than 64 rows (us, alone -> shared) 2048 -> 1000 on 128 rows 10.4 -> 10.7, 4096 -> 1024
// 14.7 -> 13.4, 9216 -> 4096 30.5 -> 24.9, 25088 -> 512 50.1 -> 28.9; where the other side is the kernel of few rows 4096 -> 4096 on 64
// rows 14.8 -> 15.5, 9216 -> 4096 23.7 -> 20.7, 25088 -> 512 36.8 -> 27.6, on 17 rows 13.3 -> 15.1, 18.4 -> 18.6, 28.0 -> 25.1.
inline int i8_splits(int n_rows, int K, long tiles) {
    const int stages = (K + 127) / 128;
    if (n_rows <= 16 || stages < (n_rows <= kI8FewRows ? 64 : 32)) return 1;
    return (int)std::max(1l, std::min(256 / tiles, (long)stages / 8));
}

// vectors: rows of weights are whole 16-byte vectors (K and their address are multiples of 16), as the GEMM wants them: weights of
// another form are copied for many rows, and few rows have their own kernel.  room: bytes of the workspace; a copy that only saves
// time is made if they suffice for it.
inline I8Plan i8_plan(int n_rows, int K, int cout, bool vectors, size_t room = SIZE_MAX) {
    auto up = [](size_t v, size_t a) { return (v + a - 1) / a * a; };
    I8Plan p;
    p.width = up(K, 128);
    if (n_rows == 1) return p;
    p.tiles = ((long)n_rows + 63) / 64 * (((long)cout + 63) / 64);
    const int splits = i8_splits(n_rows, K, p.tiles);
    p.few = n_rows <= kI8FewRows && !(splits > 1 && vectors);
    if (!p.few) p.splits = splits;
    auto lay_out = [&](bool copy) {
        p.copy = copy;
        p.bytes = 0;
        auto take = [&](size_t bytes) {
            const I8Plan::Area a{p.bytes, bytes};
            p.bytes += up(bytes, 256);
            return a;
        };
        p.rows = take(up(n_rows, 16) * p.width);
        p.scales = take((size_t)n_rows * sizeof(float));
        p.weights = take(copy ? cout * p.width : 0);
        p.part = take(p.splits > 1 ? p.tiles * p.splits * (kI8TileSums * sizeof(int32_t)) : 0);
        p.done = take(p.splits > 1 ? p.tiles * sizeof(int32_t) : 0);
    };
    // Rows that begin inside a cache line cost more lines a stage: from 2.5e10 products on padded copies of the weights pay (us, as they are ->
    // copied: 2064 -> 2048 on 6272 rows 65.0 -> 61.3, 4112 -> 1024 on 12544 123 -> 111; 2064 -> 2048 on 3136 36.8 -> 38.8, 576 -> 256 on 12544 22.5 -> 24.5).
    // Up to 64 rows read every weight once, and a copy would read and write it besides.
    const bool many = n_rows > kI8FewRows;
    lay_out(many && (!vectors || (K % 128 && (double)n_rows * K * cout >= 2.5e10)));
    if (p.copy && vectors && p.bytes > room) lay_out(false);
    return p;
}

// Rows that a workspace of `room` bytes serves at once: all of them, or 64 at a time, which copy no weights (0: not even those).  A row's
// result does not depend on the others, nor on which kernel computes it.
inline int i8_rows(int n_rows, int K, int cout, bool vectors, size_t room) {
    for (int n : {n_rows, std::min(n_rows, kI8FewRows)})
        if (i8_plan(n, K, cout, vectors, room).bytes <= room) return n;
    return 0;
}

// What a call needs whatever its weights' address.
inline size_t i8_workspace(int n_rows, int K, int cout) {
    return std::max(i8_plan(n_rows, K, cout, false).bytes, K % 16 ? 0 : i8_plan(n_rows, K, cout, true).bytes);
}

}  // namespace dc
