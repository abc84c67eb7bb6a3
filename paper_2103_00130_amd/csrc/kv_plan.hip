// Block tables and slots of a step (abft_kv_plan in include/abft_eb.h): two prefix sums over the requests - rows of new
// tokens, and blocks they need - and then every row and every new block finds its request by bisection.
//
// One launch.  A workgroup that had to wait for another's part of the prefix sums would wait longer than it takes to read all
// lengths itself (8 bytes a request, which the caches hold), so each workgroup makes both sums of all requests in LDS and writes its
// share of the outputs.  Nothing is read that another workgroup writes: entries of the table are read below a request's blocks and
// written from there on, and rows in new blocks are numbered from free_blocks.  Bound by latency: two dependent loads, two scans,
// the bisections (64 requests of a token each 4.2 us, 3.4 for one request; 2000 of up to 1000 tokens 9.5).
#include <hip/hip_runtime.h>

#include "../../include/abft_eb.h"
#include "abft_internal.h"

namespace abft {
namespace {

constexpr int kMaxRequests = 16384;   // two words of LDS for each: 128 of 160 KiB
constexpr uint32_t kRefused = 0x80000000u;

struct PlanParams {
    const int32_t* ctx;
    const int32_t* fresh;
    const int32_t* free_blocks;
    int32_t* table;
    int32_t* seq_len;
    int32_t* cu_new;
    int64_t* slots;
    int32_t* req_flags;
    int32_t* taken;
    int64_t ldt, n_slots;
    uint64_t inverse;   // floor((2^64 - 1) / block) + 1
    int n_req, block, shift, width, n_free;   // shift: log2 of the block, or -1
};

// x / block for any 32-bit x: a shift, or the upper half of a product with the block's inverse, whose error of less than 2^-32 of a
// quotient cannot carry it to the next whole number (the general 64-bit division is a hundred instructions).
__device__ inline uint32_t blocks_below(const PlanParams& p, uint32_t x) { return p.shift >= 0 ? x >> p.shift : (uint32_t)__umul64hi(p.inverse, x); }
__device__ inline int64_t blocks_for(const PlanParams& p, int64_t tokens) { return tokens > 0 ? (int64_t)blocks_below(p, (uint32_t)(tokens - 1)) + 1 : 0; }

// Sums that stop at 2^31 - 1, which no count that matters reaches: so they fit 32 bits, and are in any order what they are in one.
__device__ inline uint32_t add31(uint32_t a, uint32_t b) { return min(a + b, 0x7fffffffu); }
// over the lanes up to and with this one: within rows of 16 lanes, then from row to row
__device__ inline uint32_t wave_scan(uint32_t x) {
    x = add31(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false));
    x = add31(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false));
    x = add31(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false));
    x = add31(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false));
    x = add31(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false));
    return add31(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false));
}
// Two sums over the threads before this one, and over all.  s: two words per wavefront
struct Two {
    uint32_t rows, need;
};
template <int NT>
__device__ inline Two block_scan(Two v, Two* s, Two* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Two upto = {wave_scan(v.rows), wave_scan(v.need)};
    if (lane == 63) s[wave] = upto;
    __syncthreads();
    Two before = {0, 0}, all = {0, 0};
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        const Two x = s[w];
        if (w < wave) before = {add31(before.rows, x.rows), add31(before.need, x.need)};
        all = {add31(all.rows, x.rows), add31(all.need, x.need)};
    }
    __syncthreads();
    *total = all;
    // (what the lanes before this one have, not a difference: a sum that stopped has lost it)
    const uint32_t r = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane - 1), (int)upto.rows), n = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (lane - 1), (int)upto.need);
    return {add31(before.rows, lane ? r : 0), add31(before.need, lane ? n : 0)};
}

// the first request whose sum, without its mark, is larger than v; n if none is
__device__ inline int first_above(const uint32_t* sums, int n, uint32_t v) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((sums[mid] & ~kRefused) > v) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

struct Range {
    uintptr_t at, bytes;
    bool overlaps(const Range& o) const { return bytes > 0 && o.bytes > 0 && at < o.at + o.bytes && o.at < at + bytes; }
};
template <typename T>
Range range(const T* p, int64_t n) {
    return {reinterpret_cast<uintptr_t>(p), p ? (uintptr_t)n * sizeof(T) : 0};
}

// NT threads, each of which takes up to PER neighbouring requests.
template <int NT, int PER>
__global__ __launch_bounds__(NT) void kv_plan_kernel(const PlanParams p) {
    constexpr bool kKeepCtx = PER <= 4;          // (for more requests there is no room in LDS)
    extern __shared__ uint32_t s_dyn[];
    uint32_t* const s_rows = s_dyn;              // rows up to and with a request, marked if it is refused
    uint32_t* const s_upto = s_dyn + p.n_req;    // blocks needed up to and with it
    int32_t* const s_ctx = reinterpret_cast<int32_t*>(s_dyn + 2 * p.n_req);
    __shared__ Two s_wave[NT / 64];
    __shared__ int s_taken;
    const int tid = threadIdx.x;
    if (tid == 0) s_taken = 0;

    const int per = (p.n_req + NT - 1) / NT, r0 = min(tid * per, p.n_req), count = min(per, p.n_req - r0);
    int32_t ctx_in[PER], fresh_in[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int r = min(r0 + i, p.n_req - 1);
        ctx_in[i] = i < count ? p.ctx[r] : 0;
        fresh_in[i] = i < count ? p.fresh[r] : 0;
    }
    // blocks a request holds and wants, unless its row of the table is too short
    auto held = [&](int i) __attribute__((always_inline)) { return blocks_for(p, max(ctx_in[i], 0)); };
    // (no row of the table has so many blocks as 2^31 tokens or more come to here: blocks can be so large that it has room for them, but
    // a length has 31 bits)
    auto wanted = [&](int i) __attribute__((always_inline)) {
        const uint32_t tokens = (uint32_t)max(ctx_in[i], 0) + (uint32_t)max(fresh_in[i], 0);
        return (int)tokens < 0 ? 0x80000000u : tokens ? blocks_below(p, tokens - 1) + 1 : 0u;
    };
    auto sums = [&](uint32_t rows_before, bool limited) __attribute__((always_inline)) {
        Two t = {0, 0};
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            t.rows = add31(t.rows, (uint32_t)max(fresh_in[i], 0));
            const uint32_t want = wanted(i);
            if (want <= (uint32_t)p.width && !(limited && add31(rows_before, t.rows) > p.n_slots)) t.need = add31(t.need, want - (uint32_t)held(i));
        }
        return t;
    };
    Two all, before = block_scan<NT>(sums(0, false), s_wave, &all);
    if (all.rows > p.n_slots) before.need = block_scan<NT>(sums(before.rows, true), s_wave, &all).need;   // some have no rows, and so need no blocks
    uint32_t rows = before.rows, need = before.need;
    int most = 0;
    // the requests whose outputs this workgroup writes
    const int wr = (p.n_req + gridDim.x - 1) / gridDim.x, w0 = min((int)blockIdx.x * wr, p.n_req), w1 = min(w0 + wr, p.n_req);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (i < count) {
            const int r = r0 + i;
            const int64_t ctx = max(ctx_in[i], 0), fresh = max(fresh_in[i], 0), have = held(i), want = wanted(i);
            rows = add31(rows, (uint32_t)fresh);
            int why = 0;
            if (want > p.width) why |= ABFT_KV_TABLE_FULL;
            if (rows > p.n_slots) why |= ABFT_KV_NO_ROW;
            const int64_t n = why == 0 ? want - have : 0;
            need = add31(need, (uint32_t)n);
            if (n > 0) {
                if (need > (uint32_t)p.n_free) why |= ABFT_KV_NO_BLOCK;
                else most = max(most, (int)need);
            }
            s_rows[r] = rows | (why ? kRefused : 0u);
            s_upto[r] = need;
            if (kKeepCtx) s_ctx[r] = (int32_t)ctx;
            if (r >= w0 && r < w1) {
                p.req_flags[r] = why | (ctx_in[i] < 0 || fresh_in[i] < 0 ? ABFT_KV_BAD_LENGTH : 0);
                p.seq_len[r] = (int32_t)(why ? ctx : ctx + fresh);
                p.cu_new[r + 1] = (int32_t)min((int64_t)rows, p.n_slots);
            }
        }
    }
    if (most > 0) atomicMax(&s_taken, most);
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        p.cu_new[0] = 0;
        *p.taken = s_taken;
    }
    auto ctx_of = [&](int r) __attribute__((always_inline)) { return (int64_t)(kKeepCtx ? s_ctx[r] : max(p.ctx[r], 0)); };

    // new blocks: the u-th free one belongs to the first request that needs more than u up to itself
    const int stride = (int)gridDim.x * NT, first = (int)blockIdx.x * NT + tid;
    for (int64_t u = first; u < s_taken; u += stride) {
        const int r = first_above(s_upto, p.n_req, (uint32_t)u);
        const int64_t have = blocks_for(p, ctx_of(r));
        p.table[(int64_t)r * p.ldt + have + (u - (r > 0 ? s_upto[r - 1] : 0u))] = p.free_blocks[u];
    }
    for (int64_t t = first; t < p.n_slots; t += stride) {
        const int r = first_above(s_rows, p.n_req, (uint32_t)t);
        int64_t slot = -1;
        if (r < p.n_req && !(s_rows[r] & kRefused)) {
            const int64_t ctx = ctx_of(r), have = blocks_for(p, ctx);
            const int64_t pos = ctx + (t - (r > 0 ? s_rows[r - 1] & ~kRefused : 0u)), at = blocks_below(p, (uint32_t)pos);
            const int64_t before = r > 0 ? s_upto[r - 1] : 0u;
            const int32_t b = at < have ? p.table[(int64_t)r * p.ldt + at] : p.free_blocks[before + at - have];
            slot = (int64_t)b * p.block + (pos - at * p.block);
        }
        p.slots[t] = slot;
    }
}

}  // namespace
}  // namespace abft

extern "C" int abft_kv_plan(const int32_t* ctx_len, const int32_t* new_len, int n_req, int block_tokens, int32_t* table, int64_t ldt, int width,
                            const int32_t* free_blocks, int n_free, int32_t* seq_len, int32_t* cu_new, int64_t* slots, int64_t n_slots,
                            int32_t* req_flags, int32_t* taken, void* stream) {
    const char* fn = "abft_kv_plan";
    if (n_req < 0 || n_free < 0 || n_slots < 0 || width < 0) return abft::set_error(ABFT_EINVAL, "%s: negative count", fn);
    if (block_tokens < 1) return abft::set_error(ABFT_EINVAL, "%s: block_tokens=%d must be >= 1", fn, block_tokens);
    if (!cu_new || !taken || (n_slots > 0 && !slots) || (n_free > 0 && !free_blocks) ||
        (n_req > 0 && (!ctx_len || !new_len || !seq_len || !req_flags || (width > 0 && !table))))
        return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    if (ldt < width) return abft::set_error(ABFT_EINVAL, "%s: ldt=%lld smaller than width=%d", fn, (long long)ldt, width);
    if (n_req > abft::kMaxRequests) return abft::set_error(ABFT_EUNSUPPORTED, "%s: n_req=%d (at most %d)", fn, n_req, abft::kMaxRequests);
    if (n_slots >= 0x7fffffffll) return abft::set_error(ABFT_EUNSUPPORTED, "%s: n_slots=%lld too large", fn, (long long)n_slots);
    // (every workgroup reads all lengths while others write: an update in place would come out in parts)
    const abft::Range inputs[] = {abft::range(ctx_len, n_req), abft::range(new_len, n_req), abft::range(free_blocks, n_free)};
    const abft::Range outputs[] = {abft::range(seq_len, n_req), abft::range(cu_new, (int64_t)n_req + 1), abft::range(req_flags, n_req), abft::range(taken, 1),
                                   abft::range(slots, n_slots), abft::range(table, n_req > 0 ? (n_req - 1) * ldt + width : 0)};
    for (const abft::Range& in : inputs)
        for (const abft::Range& out : outputs)
            if (in.overlaps(out)) return abft::set_error(ABFT_EINVAL, "%s: the lengths or free blocks overlap what is written", fn);
    abft::PlanParams p{ctx_len, new_len, free_blocks, table, seq_len, cu_new, slots, req_flags, taken, ldt, n_slots, ~0ull / (uint64_t)block_tokens + 1, n_req, block_tokens, -1, width, n_free};
    for (int k = 0; k < 31; ++k)
        if (block_tokens == 1 << k) p.shift = k;
    // As few threads to a workgroup as have the requests in four steps, or in one, while a thread has no more than a row then (us, workgroups
    // of 256 / 512 / 1024: 64 requests of a token 4.2 / 4.5 / 5.3, 250 of them 4.5 / 4.8 / 5.5, 300 5.4 / 5.0 / 5.6, 1000 6.5 / 5.6 /
    // 6.2, 2000 8.8 / 6.9 / 7.1; 2000 of up to 1000 tokens in blocks of 16 512 10.2, 1024 9.5).
    const bool middle = n_req > 256 && n_req <= 2048 && n_slots <= 256 * 512;
    const int nt = n_req <= 256 ? 256 : middle ? 512 : 1024;
    const int64_t groups = (n_slots + nt - 1) / nt;
    const dim3 grid((unsigned)(groups < 1 ? 1 : groups > 256 ? 256 : groups));
    hipStream_t s = (hipStream_t)stream;
    if (n_req <= 256) {
        abft::kv_plan_kernel<256, 1><<<grid, dim3(256), (size_t)n_req * 12, s>>>(p);
    } else if (middle) {
        abft::kv_plan_kernel<512, 4><<<grid, dim3(512), (size_t)n_req * 12, s>>>(p);
    } else if (n_req <= 4096) {
        abft::kv_plan_kernel<1024, 4><<<grid, dim3(1024), (size_t)n_req * 12, s>>>(p);
    } else {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = abft::allow_dynamic_lds(reinterpret_cast<const void*>(abft::kv_plan_kernel<1024, 16>), abft::kMaxRequests * 8, done);
        if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
        abft::kv_plan_kernel<1024, 16><<<grid, dim3(1024), (size_t)n_req * 8, s>>>(p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}
