// Block tables and slots of a step (abft_kv_plan in include/abft_eb.h): two prefix sums over the requests - rows of new
// tokens, and blocks they need - and then every row and every new block finds its request by bisection.
//
// One launch.  A workgroup that had to wait for another's part of the prefix sums would wait longer than it takes to read all
// lengths itself (8 bytes a request, which the caches hold), so each workgroup makes both sums of all requests in LDS and writes its
// share of the outputs.  Nothing is read that another workgroup writes: entries of the table are read below a request's blocks and
// written from there on, and rows in new blocks are numbered from free_blocks.  Bound by latency: two dependent loads, two scans,
// the bisections.
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
    int n_req, block, width, n_free;
};

// sum over the threads before this one; *total: over all.  s: one word per wavefront
template <int NT>
__device__ inline int64_t block_scan(int64_t v, int64_t* s, int64_t* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t x = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    if (lane == 63) s[wave] = x;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        if (w < wave) before += s[w];
        all += s[w];
    }
    __syncthreads();
    *total = all;
    return before + x - v;
}

__device__ inline uint32_t clamp31(int64_t v) { return v > 0x7fffffffll ? 0x7fffffffu : (uint32_t)v; }

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

template <int NT>
__global__ __launch_bounds__(NT) void kv_plan_kernel(const PlanParams p) {
    extern __shared__ uint32_t s_dyn[];
    uint32_t* const s_rows = s_dyn;              // rows up to and with a request, marked if it is refused
    uint32_t* const s_upto = s_dyn + p.n_req;    // blocks needed up to and with it
    __shared__ int64_t s_wave[NT / 64];
    __shared__ int s_taken;
    const int tid = threadIdx.x;
    if (tid == 0) s_taken = 0;

    // each thread takes neighbouring requests
    const int per = (p.n_req + NT - 1) / NT, r0 = min(tid * per, p.n_req), r1 = min(r0 + per, p.n_req);
    int64_t rows = 0, all_rows, all_need;
    for (int r = r0; r < r1; ++r) rows += max(p.fresh[r], 0);
    const int64_t rows_before = block_scan<NT>(rows, s_wave, &all_rows);
    int64_t need = 0;
    rows = rows_before;
    for (int r = r0; r < r1; ++r) {
        const int64_t ctx = max(p.ctx[r], 0), fresh = max(p.fresh[r], 0);
        rows += fresh;
        const int64_t have = (ctx + p.block - 1) / p.block, want = (ctx + fresh + p.block - 1) / p.block;
        if (want <= p.width && rows <= p.n_slots) need += want - have;
    }
    const int64_t need_before = block_scan<NT>(need, s_wave, &all_need);
    rows = rows_before;
    need = need_before;
    int most = 0;
    // the requests whose outputs this workgroup writes
    const int wr = (p.n_req + gridDim.x - 1) / gridDim.x, w0 = min((int)blockIdx.x * wr, p.n_req), w1 = min(w0 + wr, p.n_req);
    for (int r = r0; r < r1; ++r) {
        const int32_t ctx_in = p.ctx[r], fresh_in = p.fresh[r];
        const int64_t ctx = max(ctx_in, 0), fresh = max(fresh_in, 0);
        rows += fresh;
        const int64_t have = (ctx + p.block - 1) / p.block, want = (ctx + fresh + p.block - 1) / p.block;
        int why = 0;
        if (want > p.width) why |= ABFT_KV_TABLE_FULL;
        if (rows > p.n_slots) why |= ABFT_KV_NO_ROW;
        const int64_t n = why == 0 ? want - have : 0;
        need += n;
        if (n > 0) {
            if (need > p.n_free) why |= ABFT_KV_NO_BLOCK;
            else most = max(most, (int)need);
        }
        s_rows[r] = clamp31(rows) | (why ? kRefused : 0u);
        s_upto[r] = clamp31(need);
        if (r >= w0 && r < w1) {
            p.req_flags[r] = why | (ctx_in < 0 || fresh_in < 0 ? ABFT_KV_BAD_LENGTH : 0);
            p.seq_len[r] = (int32_t)(why ? ctx : ctx + fresh);
            p.cu_new[r + 1] = (int32_t)min(rows, p.n_slots);
        }
    }
    if (most > 0) atomicMax(&s_taken, most);
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        p.cu_new[0] = 0;
        *p.taken = s_taken;
    }

    // new blocks: the u-th free one belongs to the first request that needs more than u up to itself
    const int stride = (int)gridDim.x * NT, first = (int)blockIdx.x * NT + tid;
    for (int64_t u = first; u < s_taken; u += stride) {
        const int r = first_above(s_upto, p.n_req, (uint32_t)u);
        const int64_t have = ((int64_t)max(p.ctx[r], 0) + p.block - 1) / p.block;
        p.table[(int64_t)r * p.ldt + have + (u - (r > 0 ? s_upto[r - 1] : 0u))] = p.free_blocks[u];
    }
    for (int64_t t = first; t < p.n_slots; t += stride) {
        const int r = first_above(s_rows, p.n_req, (uint32_t)t);
        int64_t slot = -1;
        if (r < p.n_req && !(s_rows[r] & kRefused)) {
            const int64_t ctx = max(p.ctx[r], 0), have = (ctx + p.block - 1) / p.block;
            const int64_t pos = ctx + (t - (r > 0 ? s_rows[r - 1] & ~kRefused : 0u)), at = pos / p.block;
            const int64_t before = r > 0 ? s_upto[r - 1] : 0u;
            const int32_t b = at < have ? p.table[(int64_t)r * p.ldt + at] : p.free_blocks[before + at - have];
            slot = (int64_t)b * p.block + pos % p.block;
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
    abft::PlanParams p{ctx_len, new_len, free_blocks, table, seq_len, cu_new, slots, req_flags, taken, ldt, n_slots, n_req, block_tokens, width, n_free};
    const size_t lds = (size_t)n_req * 8;
    const int nt = n_req <= 256 ? 256 : 1024;
    const int64_t groups = (n_slots + nt - 1) / nt;
    const unsigned grid = (unsigned)(groups < 1 ? 1 : groups > 256 ? 256 : groups);
    if (nt == 256) abft::kv_plan_kernel<256><<<dim3(grid), dim3(256), lds, (hipStream_t)stream>>>(p);
    else {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = abft::allow_dynamic_lds(reinterpret_cast<const void*>(abft::kv_plan_kernel<1024>), abft::kMaxRequests * 8, done);
        if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
        abft::kv_plan_kernel<1024><<<dim3(grid), dim3(1024), lds, (hipStream_t)stream>>>(p);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}
