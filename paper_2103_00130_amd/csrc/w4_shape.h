// How a product with a 4-bit weight is cut into workgroups (w4.hip): a rule on the host, by sizes alone.
#pragma once
#include <cstdint>

namespace abft {

struct W4Shape {
    int tiles, waves;   // NT, NW
};
// The most tiles of a wavefront that fit its registers.
constexpr int w4_most_tiles(bool f32, int group, int ct) { return ct == 2 || (f32 && group == 32) ? 2 : 4; }

// How a product is cut.  Workgroups of one tile of the weight while there are no more of them than compute units (us, 1 / 2 / 4 tiles:
// 1x4096x4096 4.24 / 5.52 / 7.69, 16 rows 6.65 / 7.57 / 10.7); beyond, X is fetched less often the more tiles share it (16x8192x8192
// 19.0 / 12.3 / 16.0, 16x16384x4096 19.0 / 15.1 / 12.9, 32 rows 36.2 / 22.7 / 22.8, 16 rows in 32 bits 34.6 / 23.3 / 15.8), which up to four rows
// hardly notice (1x16384x4096 10.4 / 9.2 / 9.9).  A long K with one workgroup to a compute unit: sixteen wavefronts, not eight
// (1x4096x16384 10.3 / 12.4; 1x4096x4096 4.3 / 4.2, 1x16384x4096 12.4 / 10.4).
inline W4Shape w4_shape(int M, int64_t tiles, int chunks) {
    const int64_t groups = tiles * ((M + 31) / 32);
    W4Shape s;
    s.tiles = groups <= 256 ? 1 : groups <= 512 || M <= 4 ? 2 : 4;
    s.waves = s.tiles == 1 && chunks >= 64 ? 16 : 8;
    return s;
}

}  // namespace abft
