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
constexpr int kLoraWanted = 512;       // workgroups of the sums over K
constexpr int kLoraUpGroups = 1024;    // workgroups of the products with `up`
constexpr int kLoraFewRows = 128;      // rows up to which any may have an adapter of its own: a workgroup for each
constexpr int kLoraManyRows = 512;     // rows from which on most tiles are one adapter's

struct LoraCut {
    int tiles, slots, splits;   // tiles of rows; workgroups among which the adapters of a tile are dealt; parts of K
    int waves;                  // of a workgroup of the sums over K
};
inline LoraCut lora_cut(int64_t M, int K) {
    LoraCut c;
    c.tiles = (int)((M + kLoraRows - 1) / kLoraRows);
    c.slots = M < kLoraRows ? (int)M : M <= kLoraFewRows ? kLoraRows : M < kLoraManyRows ? 8 : 1;
    if (c.slots < 1) c.slots = 1;
    c.waves = M >= kLoraManyRows ? 2 * kLoraWaves : kLoraWaves;
    const int64_t groups = (int64_t)c.tiles * c.slots, long_k = ((int64_t)K + kLoraStep * c.waves - 1) / (kLoraStep * c.waves);
    int64_t s = groups ? (kLoraWanted + groups - 1) / groups : 1;
    if (s > long_k) s = long_k;
    if (s > kLoraMostSplits) s = kLoraMostSplits;
    c.splits = (int)s;
    return c;
}
// floats of a call's sums over K
inline int64_t lora_sums(int64_t M, int K, int max_rank) { return (int64_t)lora_cut(M, K).splits * M * ((max_rank + 15) / 16 * 16); }
// ... that every call on up to M rows needs at most
inline int64_t lora_most_sums(int64_t M, int K, int max_rank) {
    int64_t most = 0;
    for (int64_t m = M; m > 0; m = m > 64 * kLoraWanted ? 64 * kLoraWanted : m - 1) {   // (beyond, one part of K)
        const int64_t n = lora_sums(m, K, max_rank);
        if (n > most) most = n;
    }
    return most;
}

}  // namespace abft
