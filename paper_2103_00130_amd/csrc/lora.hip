// Low-rank adapters of many requests at once (abft_lora_* in include/abft_gemm.h):
//     Y[m] = base[m] + scale[a] up[a] (down[a] X[m]),     a = ids[m].
//
// Two launches: the sums over K (of `rank` numbers a row, kept in 32 bits), then the products with `up`, whose epilogue adds base.  Rows are
// taken 16 at a time, the rows of a matrix-core operand; rows of a tile that share an adapter share one product, so that a prompt's rows cost one
// pass over the adapter for 16 rows and each adapter of a batch of single tokens is read once for every tile that has it.  X enters the matrix
// cores as it is (16-bit types, whose products are exact; binary32 by its own instruction); the sums over K are binary32 and meet `up` in binary32.
//
// Measured (4096 x 4096, bf16): one row of rank 16 6.8 us, both launches and two dependent trips to memory each (3.2 and 4.2); 64 rows through 36 adapters to
// 6144 columns 9.4 (10.3 MB; 3.9 and 6.0, as many workgroups as rows have adapters, each with little to do); 4287 rows of nine prompts 46 (14.5 and 32, the
// first at 2.4 TB/s, the second at 2.2 of base and Y; a copy of such rows, 16 of them and 128 bytes of each at a time, takes 17.7, rows end to end 15.7);
// 4096 rows of rank 16 / 32 / 128 26 / 33 / 80 (of rank 32 in float16 37); 2048 rows of rank 32 in binary32 44; 540 rows of rank 72 in binary32, 185 to 9239
// columns, 38; 8 rows of rank 128 15; 4000 rows of rank 20, 1001 to 4099 columns (no row at a multiple of 16 bytes) 45.  Where 16 rows have several adapters the tile is gone through for each (with tiles of 32 rows 51 us for nine
// prompts that begin anywhere, 43 for such that begin at multiples of 32; 4096 rows of 64 adapters in no order 120).
#include <hip/hip_runtime.h>

#include <cmath>
#include <type_traits>

#include "abft_internal.h"
#include "lora_cut.h"
#include "values.h"

namespace abft {
namespace {

typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef v4u v4u_any __attribute__((aligned(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef bf16 v8bf __attribute__((ext_vector_type(8)));
typedef f16 v8h __attribute__((ext_vector_type(8)));

// Layouts.  down: [adapter][rank / 16][chunk of K][lane][16 bytes], lane l of a chunk has row l % 16 of the sixteen and, of the chunk's 64 bytes a
// row, bytes 16 (l / 16)..: the first operand of a product with rows of X.  up: [adapter][columns / 64][rank / 16][lane][tile 0..3][4 elements]:
// lane l of a tile has the ranks 4 (l / 16).. of the sixteen for column_of(i / 4, 4 tile + i % 4) of the 64, i = l % 16, so that a
// lane's sums of the four tiles are pieces of 16 bytes of Y, those of four lanes side by side.
template <typename T>
constexpr int kChunkOf = 64 / sizeof(T);   // columns of a chunk
template <typename T>
constexpr int kPiece = 16 / sizeof(T);     // elements of 16 bytes
// the place of a lane's f-th sum among 64 columns, kg the lane's sixteen
template <typename T>
__device__ inline int column_of(int kg, int f) { return 4 * kPiece<T> * (f / kPiece<T>) + kPiece<T> * kg + f % kPiece<T>; }

struct LoraParams {
    const uint8_t* down;
    const uint8_t* up;
    const float* scale;
    const int32_t* rank;
    const void* X;
    const void* base;
    void* Y;
    const int32_t* ids;
    float* sums;     // [split][row][ranks]
    int64_t ldx, ldb, ldy;
    int M, N, K, adapters, max_rank, rank_tiles, chunks, blocks, splits, slots;
};

template <typename T>
__device__ inline v4f mma(v4u a, v4u b, v4f c) {
    if constexpr (sizeof(T) == 4) {
        const v4f x = __builtin_bit_cast(v4f, a), y = __builtin_bit_cast(v4f, b);
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[i], y[i], c, 0, 0, 0);
        return c;
    } else if constexpr (std::is_same<T, f16>::value) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, a), __builtin_bit_cast(v8h, b), c, 0, 0, 0);
    } else {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
    }
}

// Behind a loop of matrix instructions, ahead of what reads their sums: as many wait states as the longest needs.  The compiler counts them across
// branches by the first path that it finds to the instruction, which behind a loop may be the longer one: 640 columns in binary32 lost the
// last product of a lane's third sum.
__device__ inline void wait_for_products() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_nop 15" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// 16 bytes of a row of X from column k on; columns past K are zero.
template <typename T>
__device__ inline v4u load_x(const T* row, int k, int K) {
    constexpr int n = 16 / sizeof(T);
    if (k + n <= K) return *reinterpret_cast<const v4u_any*>(row + k);
    uint32_t v[n];
#pragma unroll
    for (int i = 0; i < n; ++i) {
        v[i] = 0;
        if (k + i < K) {
            if constexpr (sizeof(T) == 4) v[i] = __builtin_bit_cast(uint32_t, row[k + i]);
            else v[i] = __builtin_bit_cast(uint16_t, row[k + i]);
        }
    }
    if constexpr (sizeof(T) == 4) return v4u{v[0], v[1], v[2], v[3]};
    else return v4u{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4 % n] | v[5 % n] << 16, v[6 % n] | v[7 % n] << 16};
}

// The adapter of row m0 + lane % 16, or -1 (none, or no such row).
__device__ inline int adapter_of(const LoraParams& p, int m0) {
    const int m = m0 + (threadIdx.x & 15);
    const int a = m < p.M ? p.ids[m] : -1;
    return a >= 0 && a < p.adapters ? a : -1;
}
// The adapters among a tile's rows (and -1, where `none` says so), dealt to `slots` workgroups: to one for each row that has its adapter first, where there
// are as many, else in turns.
template <typename F>
__device__ __attribute__((always_inline)) inline void for_adapters(int mine, int slot, int slots, bool none, const F& f) {
    uint32_t left = (uint32_t)__ballot(none || mine >= 0) & 0xffffu;
    if (slots == kLoraRows) {
        const int a = __builtin_amdgcn_readlane(mine, slot);
        const uint32_t same = (uint32_t)__ballot(mine == a) & left;
        if (same && __builtin_ctz(same) == slot) f(a);
        return;
    }
    for (int n = 0; left; ++n) {
        const int a = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
        left &= ~(uint32_t)__ballot(mine == a);
        if (n % slots == slot) f(a);
    }
}
// (matrix instructions run whatever lanes are active: what decides about them is brought to one register for all)
__device__ inline int rank_of(const LoraParams& p, int a) { return __builtin_amdgcn_readfirstlane(min(max(p.rank[a], 0), p.max_rank)); }

// Sums over K.  RT: sixteens of ranks that a wavefront holds; an adapter of more is taken in turns.  The next step's loads are on their way while
// this one's are multiplied, without a branch about them, so that what is awaited is what is multiplied: rows that are not the adapter's are
// read from a row that is, and their sums left.
template <typename T, int RT>
__global__ __launch_bounds__(kLoraWaves * 64) void lora_down_kernel(const LoraParams p) {
    __shared__ v4f s_sum[kLoraWaves][RT][64];
    constexpr int kStep = RT > 2 ? 2 : 4;   // chunks of a step
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = lane >> 4;
    const int m0 = blockIdx.y * kLoraRows, mine = adapter_of(p, m0);
    const int each = (p.chunks + p.splits - 1) / p.splits, begin = min((int)blockIdx.z * each, p.chunks), end = min(p.chunks, begin + each);
    const int whole = min(end, p.K / kChunkOf<T>);   // (the last chunk may reach past K)
    for_adapters(mine, blockIdx.x, p.slots, false, [&](int a) __attribute__((always_inline)) {
        const uint32_t rows = (uint32_t)__ballot(mine == a) & 0xffffu;
        const int from = mine == a ? lane & 15 : __builtin_ctz(rows);
        const T* const row = static_cast<const T*>(p.X) + (int64_t)(m0 + from) * p.ldx + kg * kPiece<T>;
        const v4u* const down = reinterpret_cast<const v4u*>(p.down) + (int64_t)a * p.rank_tiles * p.chunks * 64 + lane;
        const int tiles = (rank_of(p, a) + 15) / 16;
        auto some = [&](auto nt, int t0) __attribute__((always_inline)) {
            constexpr int NT = decltype(nt)::value;
            struct Fetched {
                v4u x[kStep], w[kStep][NT];
            };
            v4f sum[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) sum[t] = v4f{0, 0, 0, 0};
            auto fetch = [&](Fetched& f, int c0) __attribute__((always_inline)) {
#pragma unroll
                for (int c = 0; c < kStep; ++c) {
                    const int ch = min(c0 + c, whole - 1);
                    f.x[c] = *reinterpret_cast<const v4u_any*>(row + ch * kChunkOf<T>);
#pragma unroll
                    for (int t = 0; t < NT; ++t) f.w[c][t] = down[((int64_t)(t0 + t) * p.chunks + ch) * 64];
                }
            };
            auto multiply = [&](const Fetched& f, int c0) __attribute__((always_inline)) {
#pragma unroll
                for (int c = 0; c < kStep; ++c) {
                    const v4u x = c0 + c < whole ? f.x[c] : v4u{0, 0, 0, 0}, none = {0, 0, 0, 0};
#pragma unroll
                    for (int t = 0; t < NT; ++t) sum[t] = mma<T>(c0 + c < whole ? f.w[c][t] : none, x, sum[t]);
                }
            };
            constexpr int kAll = kLoraWaves * kStep;
            int c0 = begin + wave * kStep;
            if (c0 < whole) {
                Fetched one, two;
                fetch(one, c0);
                for (;; c0 += 2 * kAll) {
                    fetch(two, c0 + kAll);
                    multiply(one, c0);
                    if (c0 + kAll >= whole) break;
                    fetch(one, c0 + 2 * kAll);
                    multiply(two, c0 + kAll);
                    if (c0 + 2 * kAll >= whole) break;
                }
            }
            if (wave == kLoraWaves - 1 && whole < end) {
                const int k = whole * kChunkOf<T> + kg * kPiece<T>;
                const v4u x = load_x<T>(row - kg * kPiece<T>, k, p.K);
#pragma unroll
                for (int t = 0; t < NT; ++t) sum[t] = mma<T>(down[((int64_t)(t0 + t) * p.chunks + whole) * 64], x, sum[t]);
            }
            wait_for_products();
#pragma unroll
            for (int t = 0; t < NT; ++t) s_sum[wave][t][lane] = sum[t];
            __syncthreads();
            for (int t = wave; t < NT; t += kLoraWaves) {
                v4f y = s_sum[0][t][lane];
#pragma unroll
                for (int w = 1; w < kLoraWaves; ++w) y += s_sum[w][t][lane];
                if (mine == a) *reinterpret_cast<v4f*>(p.sums + ((int64_t)blockIdx.z * p.M + m0 + (lane & 15)) * (16 * p.rank_tiles) + 16 * (t0 + t) + 4 * kg) = y;
            }
            __syncthreads();
        };
        int t0 = 0;
        if constexpr (RT == 1) some(std::integral_constant<int, 1>(), t0++);   // (nothing waits for the rank; of none, what is there is summed and not used)
        for (; t0 + RT <= tiles; t0 += RT) some(std::integral_constant<int, RT>(), t0);
        if constexpr (RT > 1)
            for (; t0 < tiles; ++t0) some(std::integral_constant<int, 1>(), t0);
    });
}

// Sixteen elements side by side, as they are stored.
template <typename T>
struct Sixteen {
    v4u w[sizeof(T)];
    __device__ inline void load(const T* at) {
#pragma unroll
        for (int h = 0; h < (int)sizeof(T); ++h) w[h] = reinterpret_cast<const v4u*>(at)[h];
    }
    __device__ inline float operator[](int i) const {
        constexpr int n = 16 / sizeof(T);
        const uint32_t v = w[i / n][i % n * (int)sizeof(T) / 4];
        if constexpr (sizeof(T) == 4) return __builtin_bit_cast(float, v);
        else return to_f32(__builtin_bit_cast(T, (uint16_t)(v >> (16 * (i % 2)))));
    }
};

// (Binary32 products of bfloat16 made binary32, four for sixteen ranks, kept the matrix cores busy for longer than memory: 64 rows of 64 columns a
// wavefront, rank 32, 37.3 us against 27.8.)
// The sums over K as the second product takes them: with bfloat16 adapters as three bfloat16 parts that add up to them bit for bit, sixteen ranks
// in two products of 32 places (first and second part, third part), else as they are.
template <typename T>
struct Factor {
    v4f h;
    __device__ inline void set(v4f v) { h = v; }
    // sum[t] += (the four tiles of `up`) . h
    __device__ inline void multiply(const Sixteen<T>& w, v4f (&sum)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[4 * t + i], h[i], sum[t], 0, 0, 0);
    }
};
template <>
struct Factor<bf16> {
    v4u high, low;
    __device__ inline void set(v4f v) {
        uint32_t part[3][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = v[i];
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                part[k][i] = __builtin_bit_cast(uint32_t, x) >> 16;
                x -= __builtin_bit_cast(float, part[k][i] << 16);
            }
        }
        high = v4u{part[0][0] | part[0][1] << 16, part[0][2] | part[0][3] << 16, part[1][0] | part[1][1] << 16, part[1][2] | part[1][3] << 16};
        low = v4u{part[2][0] | part[2][1] << 16, part[2][2] | part[2][3] << 16, 0, 0};
    }
    __device__ inline void multiply(const Sixteen<bf16>& w, v4f (&sum)[4]) const {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t u0 = w.w[t / 2][t % 2 * 2], u1 = w.w[t / 2][t % 2 * 2 + 1];
            const v4u u = {u0, u1, u0, u1};
            sum[t] = mma<bf16>(u, low, sum[t]);
            sum[t] = mma<bf16>(u, high, sum[t]);
        }
    }
};

// Rows of one adapter: base plus scale times the product with `up`, for the columns that a wavefront has (64 at a time, a lane 16 of a row).
// m: the lane's row, which exists; on: whether it is the adapter's, others being read as they are and left.  NT sixteens of ranks have their sums over K
// in registers, those of MORE in `more`.  What the next columns need is on its way while these are multiplied, as above.
// PIECES: a row has 16 bytes at least, so that whatever it has can be read 16 bytes at a time.
template <typename T, int NT, bool MORE, bool PIECES>
__device__ __attribute__((always_inline)) inline void up_pass(const LoraParams& p, int a, int tiles, int m, bool on, int first, int last, v4f* more) {
    constexpr int P = kPiece<T>, kPieces = 16 / P, kKept = NT < 1 ? 1 : NT;
    typedef T piece __attribute__((ext_vector_type(P)));
    typedef piece piece_any __attribute__((aligned(2)));
    const int lane = threadIdx.x & 63, kg = lane >> 4;
    const Sixteen<T>* const up = reinterpret_cast<const Sixteen<T>*>(p.up) + (int64_t)a * p.blocks * p.rank_tiles * 64 + lane;
    const T* const base = static_cast<const T*>(p.base) + (int64_t)m * p.ldb;
    T* const y = static_cast<T*>(p.Y) + (int64_t)m * p.ldy;
    struct Fetched {
        Sixteen<T> up[kKept];
        v4u base[kPieces];
    };
    auto fetch = [&](Fetched& f, int block) __attribute__((always_inline)) {
        block = min(block, last - 1);
        if constexpr (PIECES) {
#pragma unroll
            for (int h = 0; h < kPieces; ++h) f.base[h] = *reinterpret_cast<const v4u_any*>(base + min(block * kLoraColumns + column_of<T>(kg, h * P), p.N - P));
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) f.up[t].load(reinterpret_cast<const T*>(up + ((int64_t)block * p.rank_tiles + t) * 64));
    };
    auto sums_of = [&](int t) __attribute__((always_inline)) {
        const v4f* const at = reinterpret_cast<const v4f*>(p.sums + (int64_t)m * (16 * p.rank_tiles) + 16 * t + 4 * kg);
        const int64_t step = (int64_t)p.M * 4 * p.rank_tiles;
        v4f v = at[0];
        for (int i = 1; i < p.splits; i += 4) {
            v4f part[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) part[j] = at[min(i + j, p.splits - 1) * step];
#pragma unroll
            for (int j = 0; j < 4; ++j) v += i + j < p.splits ? part[j] : v4f{0, 0, 0, 0};
        }
        return v;
    };
    Factor<T> h[kKept];
    const float scale = p.scale[a];
    auto finish = [&](const Fetched& f, int block) __attribute__((always_inline)) {
        v4f sum[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sum[t] = v4f{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < NT; ++t) h[t].multiply(f.up[t], sum);
        if constexpr (MORE)
            for (int t = NT; t < tiles; ++t) {
                Sixteen<T> w;
                w.load(reinterpret_cast<const T*>(up + ((int64_t)block * p.rank_tiles + t) * 64));
                Factor<T> other;
                other.set(more[(t - NT) * 64 + lane]);
                other.multiply(w, sum);
            }
        wait_for_products();
        if (tiles == 0)
#pragma unroll
            for (int t = 0; t < 4; ++t) sum[t] = v4f{0, 0, 0, 0};
        if (!on) return;
#pragma unroll
        for (int h = 0; h < kPieces; ++h) {
            const int n = block * kLoraColumns + column_of<T>(kg, h * P);
            if (PIECES && n + P <= p.N) {
                const piece b = __builtin_bit_cast(piece, f.base[h]);
                piece v;
#pragma unroll
                for (int i = 0; i < P; ++i) v[i] = from_f32<T>(__builtin_fmaf(scale, sum[(h * P + i) / 4][i % 4], to_f32((T)b[i])));
                *reinterpret_cast<piece_any*>(y + n) = v;
            } else {
#pragma unroll
                for (int i = 0; i < P; ++i)
                    if (n + i < p.N) y[n + i] = from_f32<T>(__builtin_fmaf(scale, sum[(h * P + i) / 4][i % 4], to_f32(base[n + i])));
            }
        }
    };
    Fetched one, two;
    fetch(one, first);
#pragma unroll
    for (int t = 0; t < NT; ++t) h[t].set(sums_of(t));
    if constexpr (MORE)
        for (int t = NT; t < tiles; ++t) more[(t - NT) * 64 + lane] = sums_of(t);   // (read back by the lane that writes it)
    for (int block = first;; block += 2) {
        fetch(two, block + 1);
        finish(one, block);
        if (block + 1 >= last) break;
        fetch(one, block + 2);
        finish(two, block + 1);
        if (block + 2 >= last) break;
    }
}
// Rows without an adapter: as they are.
template <typename T, bool PIECES>
__device__ __attribute__((always_inline)) inline void copy_row(const LoraParams& p, int m, bool on, int first, int last) {
    constexpr int P = kPiece<T>;
    if (!on || m >= p.M) return;
    const T* const base = static_cast<const T*>(p.base) + (int64_t)m * p.ldb;
    T* const y = static_cast<T*>(p.Y) + (int64_t)m * p.ldy;
    for (int block = first; block < last; ++block) {
#pragma unroll
        for (int h = 0; h < 16 / P; ++h) {
            const int n = block * kLoraColumns + column_of<T>((threadIdx.x & 63) >> 4, h * P);
            if (PIECES && n + P <= p.N) *reinterpret_cast<v4u_any*>(y + n) = *reinterpret_cast<const v4u_any*>(base + n);
            else
                for (int i = n; i < min(n + P, p.N); ++i) y[i] = base[i];
        }
    }
}

// Y, 16 rows to a wavefront, and columns next to each other.  RT: the most sixteens of ranks whose sums it keeps in registers.
template <typename T, int RT, bool PIECES>
__global__ __launch_bounds__(kLoraWaves * 64) void lora_up_kernel(const LoraParams p) {
    constexpr int kMore = RT == 4 ? kLoraMostRank / 16 - RT : 0;
    __shared__ v4f s_more[kLoraWaves][kMore ? kMore * 64 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = gridDim.x * kLoraWaves, each = (p.blocks + waves - 1) / waves;
    const int m0 = blockIdx.y * kLoraRows, first = (blockIdx.x * kLoraWaves + wave) * each, last = min(first + each, p.blocks);
    if (first >= last) return;
    v4f* const more = s_more[wave];
    const int mine = adapter_of(p, m0);
    for_adapters(mine, blockIdx.z, p.slots, p.base != p.Y, [&](int a) __attribute__((always_inline)) {
        if (a < 0) {
            copy_row<T, PIECES>(p, m0 + (lane & 15), mine < 0, first, last);
            return;
        }
        // (the vote is taken by all lanes: inside the choice only those would vote that take that side of it, none for the adapter)
        const uint32_t rows = (uint32_t)__ballot(mine == a) & 0xffffu;
        const bool on = mine == a;
        const int m = m0 + (on ? lane & 15 : __builtin_ctz(rows));
        const int tiles = (rank_of(p, a) + 15) / 16;
        // (with one sixteen in the pool nothing waits for the rank: what is there is multiplied, and left if the adapter has none)
        if (RT == 1 || tiles == 1) up_pass<T, 1, false, PIECES>(p, a, tiles, m, on, first, last, more);
        else if (tiles == 0) up_pass<T, 0, false, PIECES>(p, a, tiles, m, on, first, last, more);
        else if (tiles == 2) up_pass<T, (RT > 1 ? 2 : 1), false, PIECES>(p, a, tiles, m, on, first, last, more);
        else if (tiles == 3) up_pass<T, (RT > 2 ? 3 : 1), false, PIECES>(p, a, tiles, m, on, first, last, more);
        else up_pass<T, (RT > 2 ? 4 : 1), (RT > 2), PIECES>(p, a, tiles, m, on, first, last, more);
    });
}

// An adapter into its place: an element of the layout to a thread, or several where there are more than a launch has threads; zeros where the adapter has none.
template <typename T>
__global__ __launch_bounds__(256) void lora_load_kernel(T* down, T* up, float* scale_at, int32_t* rank_at, const T* A, int64_t lda, const T* B, int64_t ldb,
                                                        int rank, float scale, int K, int N, int chunks, int blocks, int rank_tiles) {
    const int tiles = (rank + 15) / 16;
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x, n_down = (int64_t)tiles * chunks * (1024 / sizeof(T)), n_up = (int64_t)blocks * tiles * 1024;
    if (first == 0) {
        *scale_at = scale;
        *rank_at = rank;
    }
    for (int64_t t = first; t < n_down + n_up; t += (int64_t)gridDim.x * 256) {
        if (t < n_down) {
            constexpr int n = 16 / sizeof(T);   // elements of a lane
            const int e = (int)(t % n), lane = (int)(t / n) & 63;
            const int64_t piece = t / (64 * n);
            const int r = (int)(piece / chunks) * 16 + (lane & 15);
            const int64_t k = piece % chunks * kChunkOf<T> + (lane >> 4) * n + e;
            down[t] = r < rank && k < K ? A[r * lda + k] : (T)0.0f;
        } else {
            const int64_t u = t - n_down, piece = u / 1024;   // [block][rank tile]
            const int e = (int)(u & 3), tile = (int)(u / 4) & 3, lane = (int)(u / 16) & 63, i = lane & 15, rt = (int)(piece % tiles);
            const int64_t block = piece / tiles, col = block * kLoraColumns + column_of<T>(i >> 2, tile * 4 + (i & 3));
            const int r = rt * 16 + (lane >> 4) * 4 + e;
            up[(block * rank_tiles + rt) * 1024 + lane * 16 + tile * 4 + e] = r < rank && col < N ? B[col * ldb + r] : (T)0.0f;
        }
    }
}

const char* wrong_sizes(const abft_lora_t* L) {
    if (!L) return "null pool";
    if (!known_type(L->type)) return "unknown type";
    if (L->adapters < 1 || L->K < 1 || L->N < 1) return "a pool needs adapters, K and N";
    if (L->max_rank < 1 || L->max_rank > kLoraMostRank) return "max_rank must be 1..128";
    if (L->K > 0x7fffff00 || L->N > 0x7fffff00) return "K or N too large";
    return nullptr;
}
const char* wrong(const abft_lora_t* L) {
    if (const char* w = wrong_sizes(L)) return w;
    if (!L->down || !L->up || !L->scale || !L->rank) return "null pointer in the pool";
    if ((reinterpret_cast<uintptr_t>(L->down) | reinterpret_cast<uintptr_t>(L->up)) & 15) return "down and up must be 16-byte aligned";
    return nullptr;
}
int chunk_of(int type) { return 64 / type_size(type); }
int rank_tiles_of(const abft_lora_t* L) { return (L->max_rank + 15) / 16; }
int64_t chunks_of(const abft_lora_t* L) { return ((int64_t)L->K + chunk_of(L->type) - 1) / chunk_of(L->type); }
int64_t blocks_of(const abft_lora_t* L) { return ((int64_t)L->N + kLoraColumns - 1) / kLoraColumns; }

template <typename T>
void launch_load(const abft_lora_t* L, int slot, const void* A, int64_t lda, const void* B, int64_t ldb, int rank, float scale, hipStream_t s) {
    const int64_t chunks = chunks_of(L), blocks = blocks_of(L), tiles = (rank + 15) / 16;
    const int64_t count = tiles * chunks * (int64_t)(1024 / sizeof(T)) + blocks * tiles * 1024;
    T* const down = static_cast<T*>(L->down) + (int64_t)slot * rank_tiles_of(L) * chunks * (int64_t)(1024 / sizeof(T));
    T* const up = static_cast<T*>(L->up) + (int64_t)slot * blocks * rank_tiles_of(L) * 1024;
    lora_load_kernel<T><<<dim3((unsigned)lora_load_groups(count)), dim3(256), 0, s>>>(down, up, L->scale + slot, L->rank + slot, static_cast<const T*>(A), lda,
                                                                                          static_cast<const T*>(B), ldb, rank, scale, L->K, L->N, (int)chunks, (int)blocks, rank_tiles_of(L));
}

template <typename T>
void launch_gemv(const LoraParams& p, const LoraCut& c, hipStream_t s) {
    const dim3 threads(kLoraWaves * 64), down((unsigned)c.slots, (unsigned)c.tiles, (unsigned)c.splits);
    const dim3 up((unsigned)lora_up_groups(c, p.blocks, p.rank_tiles, sizeof(T) == 4), (unsigned)c.tiles, (unsigned)c.slots);
    auto launch = [&](auto rt) {
        constexpr int RT = decltype(rt)::value;
        lora_down_kernel<T, RT><<<down, threads, 0, s>>>(p);
        if (p.N < kPiece<T>) lora_up_kernel<T, RT, false><<<up, threads, 0, s>>>(p);
        else lora_up_kernel<T, RT, true><<<up, threads, 0, s>>>(p);
    };
    if (p.rank_tiles == 1) launch(std::integral_constant<int, 1>());
    else if (p.rank_tiles == 2) launch(std::integral_constant<int, 2>());
    else launch(std::integral_constant<int, 4>());
}

}  // namespace
}  // namespace abft

extern "C" {

int abft_lora_bytes(const abft_lora_t* pool, size_t* down, size_t* up) {
    if (const char* w = abft::wrong_sizes(pool)) return abft::set_error(ABFT_EINVAL, "abft_lora_bytes: %s", w);
    const size_t tiles = (size_t)pool->adapters * abft::rank_tiles_of(pool);
    if (down) *down = tiles * abft::chunks_of(pool) * 1024;
    if (up) *up = tiles * abft::blocks_of(pool) * 1024 * abft::type_size(pool->type);
    return ABFT_OK;
}

int abft_lora_load(const abft_lora_t* pool, int slot, const void* A, int64_t lda, const void* B, int64_t ldb, int rank, float scale, void* stream) {
    const char* fn = "abft_lora_load";
    if (const char* w = abft::wrong(pool)) return abft::set_error(ABFT_EINVAL, "%s: %s", fn, w);
    if (slot < 0 || slot >= pool->adapters) return abft::set_error(ABFT_EINVAL, "%s: slot=%d of %d", fn, slot, pool->adapters);
    if (rank < 0 || rank > pool->max_rank) return abft::set_error(ABFT_EINVAL, "%s: rank=%d (the pool takes up to %d)", fn, rank, pool->max_rank);
    if (!std::isfinite(scale)) return abft::set_error(ABFT_EINVAL, "%s: scale must be finite", fn);
    if (rank > 0 && (!A || !B)) return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    if (rank > 0 && (lda < pool->K || ldb < rank)) return abft::set_error(ABFT_EINVAL, "%s: lda=%lld or ldb=%lld smaller than a row", fn, (long long)lda, (long long)ldb);
    const uintptr_t es = (uintptr_t)abft::type_size(pool->type);
    if (reinterpret_cast<uintptr_t>(A) % es || reinterpret_cast<uintptr_t>(B) % es) return abft::set_error(ABFT_EINVAL, "%s: A or B is not aligned to its type", fn);
    hipStream_t s = (hipStream_t)stream;
    if (pool->type == ABFT_TYPE_F32) abft::launch_load<float>(pool, slot, A, lda, B, ldb, rank, scale, s);
    else if (pool->type == ABFT_TYPE_F16) abft::launch_load<abft::f16>(pool, slot, A, lda, B, ldb, rank, scale, s);
    else abft::launch_load<abft::bf16>(pool, slot, A, lda, B, ldb, rank, scale, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

size_t abft_lora_workspace_bytes(const abft_lora_t* pool, int M) {
    if (abft::wrong_sizes(pool) || M < 1) return 0;
    return (size_t)abft::lora_most_sums(M, pool->K, pool->max_rank) * sizeof(float);
}

int abft_lora_gemv(const void* X, int64_t ldx, int M, const abft_lora_t* pool, const int32_t* ids, const void* base, int64_t ldb, void* Y, int64_t ldy,
                   void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "abft_lora_gemv";
    if (const char* w = abft::wrong(pool)) return abft::set_error(ABFT_EINVAL, "%s: %s", fn, w);
    if (M < 0) return abft::set_error(ABFT_EINVAL, "%s: M=%d must be >= 0", fn, M);
    if (M == 0) return ABFT_OK;
    if (!X || !ids || !base || !Y || !workspace) return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    if (ldx < pool->K || ldb < pool->N || ldy < pool->N) return abft::set_error(ABFT_EINVAL, "%s: ldx=%lld, ldb=%lld or ldy=%lld smaller than a row", fn, (long long)ldx, (long long)ldb, (long long)ldy);
    if (base == Y && ldb != ldy) return abft::set_error(ABFT_EINVAL, "%s: base is Y, with another leading dimension", fn);
    const uintptr_t es = (uintptr_t)abft::type_size(pool->type), at = reinterpret_cast<uintptr_t>(base) | reinterpret_cast<uintptr_t>(Y);
    if (reinterpret_cast<uintptr_t>(X) % es || at % es) return abft::set_error(ABFT_EINVAL, "%s: X, base or Y is not aligned to its type", fn);
    if (reinterpret_cast<uintptr_t>(workspace) & 15) return abft::set_error(ABFT_EINVAL, "%s: workspace must be 16-byte aligned", fn);
    if (M > abft::kLoraRows * 65535) return abft::set_error(ABFT_EUNSUPPORTED, "%s: M=%d too large", fn, M);
    abft::LoraCut c = abft::lora_cut(M, pool->K);
    abft::LoraParams p;
    p.rank_tiles = abft::rank_tiles_of(pool);
    const int64_t one = (int64_t)M * 16 * p.rank_tiles * (int64_t)sizeof(float), room = (int64_t)workspace_bytes / one;
    if (room < 1) return abft::set_error(ABFT_EINVAL, "%s: workspace of %zu bytes, %lld are needed", fn, workspace_bytes, (long long)one);
    if (c.splits > room) c.splits = (int)room;
    p.down = static_cast<const uint8_t*>(pool->down);
    p.up = static_cast<const uint8_t*>(pool->up);
    p.scale = pool->scale;
    p.rank = pool->rank;
    p.X = X;
    p.base = base;
    p.Y = Y;
    p.ids = ids;
    p.sums = static_cast<float*>(workspace);
    p.ldx = ldx;
    p.ldb = ldb;
    p.ldy = ldy;
    p.M = M;
    p.N = pool->N;
    p.K = pool->K;
    p.adapters = pool->adapters;
    p.max_rank = pool->max_rank;
    p.chunks = (int)abft::chunks_of(pool);
    p.blocks = (int)abft::blocks_of(pool);
    p.splits = c.splits;
    p.slots = c.slots;
    hipStream_t s = (hipStream_t)stream;
    if (pool->type == ABFT_TYPE_F32) abft::launch_gemv<float>(p, c, s);
    else if (pool->type == ABFT_TYPE_F16) abft::launch_gemv<abft::f16>(p, c, s);
    else abft::launch_gemv<abft::bf16>(p, c, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

}  // extern "C"
