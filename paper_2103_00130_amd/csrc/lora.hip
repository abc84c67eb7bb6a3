// Low-rank adapters of many requests at once (abft_lora_* in include/abft_gemm.h):
//     Y[m] = base[m] + scale[a] up[a] (down[a] X[m]),     a = ids[m].
//
// Two launches: the sums over K (of `rank` numbers a row, kept in 32 bits), then the products with `up`, whose epilogue adds base.  Rows are
// taken 16 at a time, the rows of a matrix-core operand; rows of a tile that share an adapter share one product, so that a prompt's rows cost one
// pass over the adapter for 16 rows and each adapter of a batch of single tokens is read once for every tile that has it.  X enters the matrix
// cores as it is (16-bit types, whose products are exact; binary32 by its own instruction); the sums over K are binary32 and meet `up` in binary32.
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
// row, bytes 16 (l / 16)..: the first operand of a product with rows of X.  up: [adapter][columns / 64][rank / 16][tile 0..3][lane][4 elements]:
// lane l of a tile has the ranks 4 (l / 16).. of the sixteen for column 16 (i / 4) + 4 tile + i % 4 of the 64, i = l % 16, so that a
// lane's sums of the four tiles are 16 columns side by side.
template <typename T>
constexpr int kChunkOf = 64 / sizeof(T);   // columns of a chunk

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
    bool wide;       // rows of base and Y are whole aligned pieces of 16 bytes
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
// (matrix instructions run whatever lanes are active: what decides about them is brought to one register for all)
__device__ inline int rank_of(const LoraParams& p, int a) { return __builtin_amdgcn_readfirstlane(min(max(p.rank[a], 0), p.max_rank)); }

// Sums over K.  RT: sixteens of ranks that a wavefront holds; an adapter of more is taken in turns.
template <typename T, int RT>
__global__ __launch_bounds__(kLoraWaves * 64) void lora_down_kernel(const LoraParams p) {
    __shared__ v4f s_sum[kLoraWaves][RT][64];
    constexpr int kStep = RT > 2 ? 2 : 4;   // chunks under way
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = lane >> 4;
    const int m0 = blockIdx.y * kLoraRows, mine = adapter_of(p, m0);
    const int each = (p.chunks + p.splits - 1) / p.splits, begin = blockIdx.z * each, end = min(p.chunks, begin + each);
    const T* const row = static_cast<const T*>(p.X) + (int64_t)min(m0 + (lane & 15), p.M - 1) * p.ldx;
    uint32_t left = (uint32_t)__ballot(mine >= 0) & 0xffffu;
    for (int n = 0; left; ++n) {
        const int a = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
        left &= ~(uint32_t)__ballot(mine == a);
        if (n % p.slots != (int)blockIdx.x) continue;
        const int tiles = (rank_of(p, a) + 15) / 16;
        const v4u* const down = reinterpret_cast<const v4u*>(p.down) + (int64_t)a * p.rank_tiles * p.chunks * 64 + lane;
        for (int t0 = 0; t0 < tiles; t0 += RT) {
            v4f sum[RT];
#pragma unroll
            for (int t = 0; t < RT; ++t) sum[t] = v4f{0, 0, 0, 0};
            for (int c0 = begin + wave * kStep; c0 < end; c0 += kLoraWaves * kStep) {
                v4u x[kStep], w[kStep][RT];
#pragma unroll
                for (int c = 0; c < kStep; ++c) {
                    const int ch = c0 + c;
                    x[c] = v4u{0, 0, 0, 0};
                    if (mine == a && ch < end) x[c] = load_x<T>(row, ch * kChunkOf<T> + kg * (16 / (int)sizeof(T)), p.K);
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        if (t0 + t < tiles) w[c][t] = down[((int64_t)(t0 + t) * p.chunks + min(ch, end - 1)) * 64];
                }
#pragma unroll
                for (int c = 0; c < kStep; ++c)
#pragma unroll
                    for (int t = 0; t < RT; ++t)
                        if (t0 + t < tiles) sum[t] = mma<T>(w[c][t], x[c], sum[t]);
            }
            wait_for_products();
#pragma unroll
            for (int t = 0; t < RT; ++t) s_sum[wave][t][lane] = sum[t];
            __syncthreads();
            for (int t = wave; t < RT && t0 + t < tiles; t += kLoraWaves) {
                v4f y = s_sum[0][t][lane];
#pragma unroll
                for (int w = 1; w < kLoraWaves; ++w) y += s_sum[w][t][lane];
                if (mine == a) *reinterpret_cast<v4f*>(p.sums + ((int64_t)blockIdx.z * p.M + m0 + (lane & 15)) * (16 * p.rank_tiles) + 16 * (t0 + t) + 4 * kg) = y;
            }
            __syncthreads();
        }
    }
}

// Four elements of `up` as binary32.
template <typename T>
__device__ inline v4f load_up(const uint8_t* up, int64_t piece) {
    if constexpr (sizeof(T) == 4) {
        return reinterpret_cast<const v4f*>(up)[piece];
    } else {
        const v2u w = reinterpret_cast<const v2u*>(up)[piece];
        v4f f;
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = to_f32(__builtin_bit_cast(T, (uint16_t)(w[i / 2] >> (16 * (i % 2)))));
        return f;
    }
}

// Y.  A wavefront has 16 rows and 64 columns at a time, a lane 16 columns of one row.
template <typename T>
__global__ __launch_bounds__(kLoraWaves * 64) void lora_up_kernel(const LoraParams p) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), kg = lane >> 4;
    const int m0 = blockIdx.y * kLoraRows, m = m0 + (lane & 15), mine = adapter_of(p, m0);
    const int block = blockIdx.x * kLoraWaves + wave;
    if (block >= p.blocks) return;
    const int n0 = block * kLoraColumns + 16 * kg, columns = min(p.N - n0, 16);
    const T* const base = static_cast<const T*>(p.base) + (int64_t)min(m, p.M - 1) * p.ldb + n0;
    T* const y = static_cast<T*>(p.Y) + (int64_t)min(m, p.M - 1) * p.ldy + n0;
    // what the rows of the group get: base, and `sum` scaled
    auto store = [&](bool on, const v4f (&sum)[4], float scale) {
        if (!on || m >= p.M || columns <= 0) return;
        if (p.wide && columns == 16) {
            constexpr int n = 16 / sizeof(T);
            typedef T piece __attribute__((ext_vector_type(n)));
#pragma unroll
            for (int h = 0; h < 16 / n; ++h) {
                piece v = reinterpret_cast<const piece*>(base)[h];
#pragma unroll
                for (int i = 0; i < n; ++i) v[i] = from_f32<T>(__builtin_fmaf(scale, sum[(h * n + i) / 4][i % 4], to_f32((T)v[i])));
                reinterpret_cast<piece*>(y)[h] = v;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (i < columns) y[i] = from_f32<T>(__builtin_fmaf(scale, sum[i / 4][i % 4], to_f32(base[i])));
        }
    };
    uint32_t left = 0xffffu;
    for (int n = 0; left; ++n) {
        const int a = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
        left &= ~(uint32_t)__ballot(mine == a);
        if (n % p.slots != (int)blockIdx.z) continue;
        v4f sum[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) sum[t] = v4f{0, 0, 0, 0};
        if (a < 0) {
            // rows without an adapter: as they are
            if (p.base != p.Y && mine == a && m < p.M && columns > 0)
                for (int i = 0; i < columns; ++i) y[i] = base[i];
            continue;
        }
        const int tiles = (rank_of(p, a) + 15) / 16;
        for (int t0 = 0; t0 < tiles; ++t0) {
            v4f h = {0, 0, 0, 0};
            if (mine == a)
                for (int s = 0; s < p.splits; ++s) h += *reinterpret_cast<const v4f*>(p.sums + ((int64_t)s * p.M + m) * (16 * p.rank_tiles) + 16 * t0 + 4 * kg);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const v4f w = load_up<T>(p.up, ((((int64_t)a * p.blocks + block) * p.rank_tiles + t0) * 4 + t) * 64 + lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], h[i], sum[t], 0, 0, 0);
            }
        }
        wait_for_products();
        store(mine == a, sum, p.scale[a]);
    }
}

// An adapter into its place: one thread for each element of the layout, zeros where the adapter has none.
template <typename T>
__global__ __launch_bounds__(256) void lora_load_kernel(T* down, T* up, float* scale_at, int32_t* rank_at, const T* A, int64_t lda, const T* B, int64_t ldb,
                                                        int rank, float scale, int K, int N, int chunks, int blocks, int rank_tiles) {
    const int tiles = (rank + 15) / 16;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x, n_down = (int64_t)tiles * chunks * (1024 / sizeof(T)), n_up = (int64_t)blocks * tiles * 1024;
    if (t == 0) {
        *scale_at = scale;
        *rank_at = rank;
    }
    if (t < n_down) {
        constexpr int n = 16 / sizeof(T);   // elements of a lane
        const int e = (int)(t % n), lane = (int)(t / n) & 63;
        const int64_t piece = t / (64 * n);
        const int r = (int)(piece / chunks) * 16 + (lane & 15);
        const int64_t k = piece % chunks * kChunkOf<T> + (lane >> 4) * n + e;
        down[t] = r < rank && k < K ? A[r * lda + k] : (T)0.0f;
    } else if (t - n_down < n_up) {
        const int64_t u = t - n_down, piece = u / 256;   // [block][rank tile][tile]
        const int e = (int)(u & 3), lane = (int)(u / 4) & 63, i = lane & 15, tile = (int)(piece & 3), rt = (int)(piece / 4 % tiles);
        const int64_t block = piece / 4 / tiles, col = block * kLoraColumns + (i >> 2) * 16 + tile * 4 + (i & 3);
        const int r = rt * 16 + (lane >> 4) * 4 + e;
        up[((block * rank_tiles + rt) * 4 + tile) * 256 + lane * 4 + e] = r < rank && col < N ? B[col * ldb + r] : (T)0.0f;
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
    lora_load_kernel<T><<<dim3((unsigned)(count ? (count + 255) / 256 : 1)), dim3(256), 0, s>>>(down, up, L->scale + slot, L->rank + slot, static_cast<const T*>(A), lda,
                                                                                          static_cast<const T*>(B), ldb, rank, scale, L->K, L->N, (int)chunks, (int)blocks, rank_tiles_of(L));
}

template <typename T>
void launch_gemv(const LoraParams& p, const LoraCut& c, hipStream_t s) {
    const dim3 threads(kLoraWaves * 64), down((unsigned)c.slots, (unsigned)c.tiles, (unsigned)c.splits);
    if (p.rank_tiles == 1) lora_down_kernel<T, 1><<<down, threads, 0, s>>>(p);
    else if (p.rank_tiles == 2) lora_down_kernel<T, 2><<<down, threads, 0, s>>>(p);
    else lora_down_kernel<T, 4><<<down, threads, 0, s>>>(p);
    lora_up_kernel<T><<<dim3((unsigned)((p.blocks + kLoraWaves - 1) / kLoraWaves), (unsigned)c.tiles, (unsigned)c.slots), threads, 0, s>>>(p);
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
    p.wide = ((at | (uintptr_t)ldb * es | (uintptr_t)ldy * es) & 15) == 0;
    hipStream_t s = (hipStream_t)stream;
    if (pool->type == ABFT_TYPE_F32) abft::launch_gemv<float>(p, c, s);
    else if (pool->type == ABFT_TYPE_F16) abft::launch_gemv<abft::f16>(p, c, s);
    else abft::launch_gemv<abft::bf16>(p, c, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

}  // extern "C"
