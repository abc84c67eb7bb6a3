// How a product with low-rank adapters is cut into workgroups (lora.hip): a rule on the host, by sizes alone.
#pragma once
#include <cstddef>
#include <cstdint>

namespace abft {

constexpr int kLoraRows = 16;          // rows of a tile
constexpr int kLoraMostRank = 128;
constexpr int kLoraColumns = 64;       // columns of Y that a wavefront has at a time
constexpr int kLoraStep = 128;         // columns of X that a wavefront has at a time
constexpr int kLoraWaves = 4;
constexpr int kLoraMostSplits = 16;
constexpr int kLoraUpGroups = 1024;    // workgroups of the products with `up`

struct LoraCut {
    int tiles, slots, splits;   // tiles of rows; workgroups among which the adapters of a tile are dealt; parts of K
};
// Up to 128 rows any may have an adapter of its own: a workgroup for each row of a tile.  From 512 on most tiles are one request's, and one workgroup
// takes the adapters of a tile in turns.  (us, 16 / 8 / 4 / 1 workgroups for a tile: 256 rows of 64 adapters in no order, 4096 x 4096, rank 16 16.7 / 16.6 /
// 28 / -, of 4 in order 14.3 / 9.6 / 9.4 / -; 1024 rows of 4 in order 38.6 / 22.6 / - / 14.4; 4096 - / - / 41.5 / 26.2.)
// K is cut into so many parts that the sums have some workgroups for every compute unit, and a wavefront 128 columns at least; every part is read
// again by the products with `up` (4287 rows of prompts, 2 / 4 parts 44.9 / 43.8; 1024 rows, 4 / 8 parts 14.4 / 15.1).
inline LoraCut lora_cut(int64_t M, int K) {
    LoraCut c;
    c.tiles = (int)((M + kLoraRows - 1) / kLoraRows);
    c.slots = M < 1 ? 1 : M < kLoraRows ? (int)M : M <= 128 ? kLoraRows : M < 512 ? 8 : 1;
    const int64_t groups = (int64_t)(c.tiles < 1 ? 1 : c.tiles) * c.slots, long_k = ((int64_t)K + kLoraStep * kLoraWaves - 1) / (kLoraStep * kLoraWaves);
    int64_t s = M < 512 ? (512 + groups - 1) / groups : 1100 / groups;
    if (s > long_k) s = long_k;
    if (s > kLoraMostSplits) s = kLoraMostSplits;
    c.splits = s < 1 ? 1 : (int)s;
    return c;
}
// Workgroups among which the columns of a tile's rows are dealt, `blocks` times 64 of them.  (binary32 with more than two sixteens of ranks takes the
// registers of a whole SIMD: no more workgroups than are resident at once)
inline int lora_up_groups(const LoraCut& c, int blocks, int rank_tiles, bool f32) {
    const int64_t rows = (int64_t)c.tiles * c.slots, most = (blocks + kLoraWaves - 1) / kLoraWaves;
    const int64_t wanted = rank_tiles <= 2 ? kLoraUpGroups : f32 ? kLoraUpGroups / 4 : kLoraUpGroups;
    const int64_t groups = (wanted + rows - 1) / rows;
    return (int)(groups < most ? groups : most);
}
// Workgroups of 256 threads for the elements of an adapter's layout: no more than a launch may have, of fewer than 2^32 threads.
inline int64_t lora_load_groups(int64_t elements) {
    const int64_t groups = (elements + 255) / 256;
    return groups < 1 ? 1 : groups > 0xffffff ? 0xffffff : groups;
}
// floats of a call's sums over K
inline int64_t lora_sums(int64_t M, int K, int max_rank) { return (int64_t)lora_cut(M, K).splits * M * ((max_rank + 15) / 16 * 16); }
// ... that every call on up to M rows needs at most
inline int64_t lora_most_sums(int64_t M, int K, int max_rank) {
    int64_t most = 0;
    for (int64_t m = M; m > 0; m = m > 20000 ? 20000 : m - 1) {   // (beyond, one part of K)
        const int64_t n = lora_sums(m, K, max_rank);
        if (n > most) most = n;
    }
    return most;
}

}  // namespace abft
