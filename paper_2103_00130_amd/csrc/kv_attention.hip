// abft_kv_attention: argument checks, how the work is cut, and the launch (the kernels are in kv_attention.h).
#include <cmath>

#include "kv_attention.h"

namespace abft {
namespace {

__global__ __launch_bounds__(256) void kv_clear_flags_kernel(int32_t* flags, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) flags[i] = 0;
}
hipError_t clear_flags(int32_t* flags, int n, hipStream_t s) {
    if (!flags) return hipSuccess;
    kv_clear_flags_kernel<<<dim3((unsigned)(((int64_t)n + 255) / 256)), dim3(256), 0, s>>>(flags, n);
    return hipGetLastError();
}

}  // namespace
}  // namespace abft

extern "C" {

size_t abft_kv_attention_workspace_bytes(const abft_kv_cache_t* cache, int n_req, int q_heads, int max_new, int max_len) {
    if (abft::kv_wrong_sizes(cache) || n_req < 1 || q_heads < 1 || q_heads % cache->heads != 0 || max_new < 1 || max_len < 1 || max_len > 0x7ffffe00) return 0;
    return abft::attn_workspace_bytes(abft::kv_columns(cache->head_dim), n_req, cache->heads, q_heads / cache->heads, max_new, max_len);
}

int abft_kv_attention(const abft_kv_cache_t* cache, const void* Q, int64_t q_token_stride, int64_t q_head_stride, int type,
                      int64_t n_rows, int q_heads, const int32_t* table, int64_t ldt, int width, const int32_t* seq_len,
                      const int32_t* cu_new, int n_req, int max_new, int max_len, float scale, void* O, int64_t o_token_stride,
                      int64_t o_head_stride, float* lse, int32_t* req_flags, void* workspace, size_t workspace_bytes, void* stream) {
    const char* fn = "abft_kv_attention";
    if (const char* w = abft::kv_wrong(cache)) return abft::set_error(ABFT_EINVAL, "%s: %s", fn, w);
    if (!abft::known_type(type)) return abft::set_error(ABFT_EINVAL, "%s: unknown type %d", fn, type);
    if (n_rows < 0 || n_req < 0 || width < 0) return abft::set_error(ABFT_EINVAL, "%s: negative count", fn);
    if (q_heads < 1 || q_heads % cache->heads != 0) return abft::set_error(ABFT_EINVAL, "%s: q_heads=%d must be a multiple of the cache's %d heads", fn, q_heads, cache->heads);
    const float scale2 = scale * 1.44269504f;
    if (!std::isfinite(scale2)) return abft::set_error(ABFT_EINVAL, "%s: scale must be finite, as must be scale * log2(e)", fn);
    if (n_req == 0) return ABFT_OK;
    hipStream_t s = (hipStream_t)stream;
    if (n_rows == 0) {   // nothing to do but to overwrite the flags
        const hipError_t e = abft::clear_flags(req_flags, n_req, s);
        return e == hipSuccess ? ABFT_OK : abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    }
    if (max_new < 1 || max_len < 1) return abft::set_error(ABFT_EINVAL, "%s: max_new=%d and max_len=%d must be >= 1", fn, max_new, max_len);
    if (!Q || !O || !table || !seq_len || !cu_new) return abft::set_error(ABFT_EINVAL, "%s: null pointer", fn);
    if (ldt < width) return abft::set_error(ABFT_EINVAL, "%s: ldt=%lld smaller than width=%d", fn, (long long)ldt, width);
    const uintptr_t es = (uintptr_t)abft::type_size(type);
    if (reinterpret_cast<uintptr_t>(Q) % es || reinterpret_cast<uintptr_t>(O) % es) return abft::set_error(ABFT_EINVAL, "%s: Q or O is not aligned to its type", fn);
    if (workspace && (reinterpret_cast<uintptr_t>(workspace) & 15)) return abft::set_error(ABFT_EINVAL, "%s: the workspace must be 16-byte aligned", fn);
    if (n_req > 65535) return abft::set_error(ABFT_EUNSUPPORTED, "%s: n_req=%d (at most 65535)", fn, n_req);
    // (positions are 32-bit: a tile begins below 2^31 - 512, whatever the lengths say)
    if (((int64_t)width * cache->block_tokens) > 0x7ffffe00ll || max_len > 0x7ffffe00) return abft::set_error(ABFT_EUNSUPPORTED, "%s: a request's tokens must be fewer than 2^31 - 512", fn);
    if (n_rows > 0x7fffffffll / q_heads) return abft::set_error(ABFT_EUNSUPPORTED, "%s: n_rows=%lld too large for one launch", fn, (long long)n_rows);

    const int cols = abft::kv_columns(cache->head_dim);
    const int64_t pairs = (int64_t)n_req * cache->heads;
    if (pairs > abft::kAttnMostWorkgroups) return abft::set_error(ABFT_EUNSUPPORTED, "%s: n_req=%d requests of %d heads are too many for one launch", fn, n_req, cache->heads);
    abft::AttnCut c = abft::attn_cut(cols, n_req, cache->heads, q_heads / cache->heads, (int)abft::attn_at_most(max_new, n_rows), max_len);
    const size_t each = abft::attn_part_bytes(n_rows * q_heads, cols);
    if (c.parts > 1 && (!workspace || workspace_bytes / each < (size_t)c.parts)) {
        const size_t fit = workspace ? workspace_bytes / each : 0;
        const int64_t parts = fit < 2 ? 1 : (int64_t)fit;
        c.chunk = (int)((((int64_t)max_len + parts - 1) / parts + 255) / 256 * 256);
        c.parts = (int)(((int64_t)max_len + c.chunk - 1) / c.chunk);
    }
    const int64_t workgroups = pairs * c.groups * c.parts;
    abft::AttnParams p;
    p.k_codes = cache->k_codes;
    p.v_codes = cache->v_codes;
    p.k_scale = cache->k_scale;
    p.v_scale = cache->v_scale;
    p.Q = Q;
    p.O = O;
    p.table = table;
    p.seq_len = seq_len;
    p.cu_new = cu_new;
    p.lse = lse;
    p.req_flags = req_flags;
    p.part_o = static_cast<float*>(workspace);
    p.part_ml = p.part_o ? p.part_o + (size_t)c.parts * n_rows * q_heads * cols : nullptr;
    p.q_token = q_token_stride;
    p.q_head = q_head_stride;
    p.o_token = o_token_stride;
    p.o_head = o_head_stride;
    p.ldt = ldt;
    p.n_rows = n_rows;
    p.n_blocks = cache->n_blocks;
    p.heads = cache->heads;
    p.q_heads = q_heads;
    p.group = q_heads / cache->heads;
    p.dim = cache->head_dim;
    p.block_shift = cache->block_tokens == 16 ? 4 : cache->block_tokens == 32 ? 5 : cache->block_tokens == 64 ? 6 : 7;
    p.width = width;
    p.n_req = n_req;
    p.groups = c.groups;
    p.parts = c.parts;
    p.stride = (int)(pairs * 382 / 1000 / 8 * 8 + 1);   // (far, by no simple fraction, and on to the next eighth of the chip)
    p.chunk = c.chunk;
    p.scale2 = scale2;
    p.q_wide = ((reinterpret_cast<uintptr_t>(Q) | (uintptr_t)(q_token_stride * (int64_t)es) | (uintptr_t)(q_head_stride * (int64_t)es) | (uintptr_t)(cache->head_dim * (int64_t)es)) & (4 * es - 1)) == 0;
    hipError_t e = abft::clear_flags(req_flags, n_req, s);
    const bool small_blocks = cache->block_tokens < abft::kKvTile;
    if (e == hipSuccess)
        e = type == ABFT_TYPE_F32 ? abft::launch_attention_f32(c.shape, cols, small_blocks, p, (unsigned)workgroups, s)
            : type == ABFT_TYPE_F16 ? abft::launch_attention_f16(c.shape, cols, small_blocks, p, (unsigned)workgroups, s)
                                    : abft::launch_attention_bf16(c.shape, cols, small_blocks, p, (unsigned)workgroups, s);
    if (e != hipSuccess) return abft::set_error(ABFT_EHIP, "%s: %s", fn, hipGetErrorString(e));
    return ABFT_OK;
}

}  // extern "C"
