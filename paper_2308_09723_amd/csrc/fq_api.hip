// C ABI of libfq: argument validation on the host, then dispatch to the launchers.
// Every check happens before the first HIP call, so invalid calls never touch the GPU.
#include <hip/hip_runtime.h>
#include <mutex>
#include <stdint.h>
#include <stdio.h>

#include "fq_internal.h"
#include "fq_layout.h"

namespace {

bool bits_ok(int bits) { return bits == 3 || bits == 4 || bits == 8; }

// Returns FQ_OK and the effective group size in *g_eff, or an error status.
int check_shape(int64_t K, int64_t N, int bits, int group_size, int* g_eff) {
    if (!bits_ok(bits) || K <= 0 || N <= 0 || group_size < 0) return FQ_ERR_INVALID_ARG;
    const int64_t g = (group_size == 0) ? K : (int64_t)group_size;
    if (g > K || K % g != 0) return FQ_ERR_INVALID_ARG;
    if (K > (int64_t)1 << 24 || N > (int64_t)1 << 24) return FQ_ERR_UNSUPPORTED;
    if (N % FQ_NTILE != 0 || K % fq_kblk(bits) != 0) return FQ_ERR_UNSUPPORTED;
    if (g % 32 != 0) return FQ_ERR_UNSUPPORTED;
    if (K / g > 65535) return FQ_ERR_UNSUPPORTED;
    if (g_eff) *g_eff = (int)g;
    return FQ_OK;
}

int halving_levels(int64_t g_top, int g_min) {
    int levels = 0;
    int64_t g = g_top;
    while (g % 2 == 0 && g / 2 >= g_min) {
        g /= 2;
        ++levels;
    }
    return levels;
}

// workspace bytes of a planned product
size_t plan_bytes(const fq_gemm_plan& plan, int64_t M, int64_t N, int64_t K, int act_dtype, int scale_format) {
    size_t need = fq_partial_bytes(plan, M, N);
    if (fq_via_f16(act_dtype, scale_format, plan, N)) need += fq_a16_bytes(M, K) + fq_rowscale_bytes(M);
    return need;
}

}  // namespace

extern "C" {

size_t fq_codes_bytes(int64_t K, int64_t N, int bits) {
    if (!bits_ok(bits) || K <= 0 || N <= 0) return 0;
    return (size_t)(K * N * bits / 8);
}

size_t fq_scales_bytes(int64_t K, int64_t N, int group_size) {
    if (K <= 0 || N <= 0 || group_size < 0) return 0;
    const int64_t g = group_size == 0 ? K : group_size;
    if (g > K || K % g != 0) return 0;
    return (size_t)((K / g) * N * 2);
}

size_t fq_gemm_workspace_bytes_for(int64_t M, int64_t N, int64_t K, int bits, int group_size, int act_dtype,
                                   int scale_format) {
    int g = 0;
    if (M <= 0 || check_shape(K, N, bits, group_size, &g) != FQ_OK) return 0;
    return plan_bytes(fq_plan_gemm(M, N, K, bits, g, act_dtype), M, N, K, act_dtype, scale_format);
}

size_t fq_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K, int bits, int group_size) {
    // the largest need over the activation types and scale formats
    return fq_gemm_workspace_bytes_for(M, N, K, bits, group_size, FQ_BF16, FQ_SCALE_F16);
}

size_t fq_gemm_grouped_workspace_bytes(int64_t total_rows, int E, int64_t N, int64_t K, int bits,
                                       int group_size) {
    (void)total_rows; (void)E; (void)N; (void)K; (void)bits; (void)group_size;
    return 0;
}

int fq_quantize_sf(const void* W_f16, int64_t K, int64_t N, int bits, int group_size, int scale_format,
                   void* codes, void* scales, void* stream) {
    if (!W_f16 || !codes || !scales) return FQ_ERR_INVALID_ARG;
    if (scale_format != FQ_SCALE_F16 && scale_format != FQ_SCALE_BF16) return FQ_ERR_INVALID_ARG;
    int g = 0;
    const int st = check_shape(K, N, bits, group_size, &g);
    if (st != FQ_OK) return st;
    return fq_launch_quantize(W_f16, K, N, bits, g, scale_format, codes, scales, (hipStream_t)stream);
}

int fq_quantize(const void* W_f16, int64_t K, int64_t N, int bits, int group_size, void* codes,
                void* scales_f16, void* stream) {
    return fq_quantize_sf(W_f16, K, N, bits, group_size, FQ_SCALE_F16, codes, scales_f16, stream);
}

int fq_unpack(const void* codes, int64_t K, int64_t N, int bits, int8_t* q, void* stream) {
    if (!codes || !q) return FQ_ERR_INVALID_ARG;
    const int st = check_shape(K, N, bits, 0, nullptr);
    if (st != FQ_OK) return st;
    return fq_launch_unpack(codes, K, N, bits, q, (hipStream_t)stream);
}

size_t fq_choose_group_workspace_bytes(int64_t K, int64_t N, int g_start, int g_min) {
    if (K <= 0 || N <= 0 || g_start < 0 || g_min <= 0) return 0;
    const int64_t g_top = g_start == 0 ? K : g_start;
    if (g_top > K || K % g_top != 0) return 0;
    const int levels = halving_levels(g_top, g_min);
    const int64_t f = g_top >> levels;
    return (size_t)(256 + (K / f) * N * 2);
}

int fq_choose_group(const void* W_f16, int64_t K, int64_t N, int g_start, int g_min, float alpha,
                    int* g_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!W_f16 || !g_out || K <= 0 || N <= 0 || g_start < 0 || g_min <= 0) return FQ_ERR_INVALID_ARG;
    if (!(alpha >= 0.0f && alpha <= 1.0f)) return FQ_ERR_INVALID_ARG;
    const int64_t g_top = g_start == 0 ? K : g_start;
    if (g_top > K || K % g_top != 0) return FQ_ERR_INVALID_ARG;
    // (the abs-max kernel reads eight columns per lane)
    if (N % FQ_NTILE != 0 || K > (int64_t)1 << 24 || N > (int64_t)1 << 24) return FQ_ERR_UNSUPPORTED;
    const int levels = halving_levels(g_top, g_min);
    if (levels == 0) {
        *g_out = (int)g_top;
        return FQ_OK;
    }
    const int64_t f = g_top >> levels;
    if (levels > 24 || K / f > 65535 || K / g_top > 65535) return FQ_ERR_UNSUPPORTED;
    if (!workspace || workspace_bytes < fq_choose_group_workspace_bytes(K, N, g_start, g_min))
        return FQ_ERR_WORKSPACE;
    uint32_t flags = 0;      // bit d: halving step d is taken
    const int st = fq_launch_choose_group(W_f16, K, N, (int)g_top, levels, alpha, &flags, workspace,
                                          (hipStream_t)stream);
    if (st != FQ_OK) return st;
    int64_t g = g_top;
    for (int d = 0; d < levels; ++d) {
        if (!(flags >> d & 1u)) break;
        g /= 2;
    }
    *g_out = (int)g;
    return FQ_OK;
}

size_t fq_quant_error_workspace_bytes(int64_t K, int64_t N) {
    if (K <= 0 || N <= 0) return 0;
    return (size_t)(16 + 16 * fq_quant_error_blocks(K, N));
}

int fq_quant_error(const void* W_f16, int64_t K, int64_t N, int bits, int group_size, const void* codes,
                   const void* scales_f16, double* sse_out, double* max_abs_out, void* workspace,
                   size_t workspace_bytes, void* stream) {
    return fq_quant_error_sf(W_f16, K, N, bits, group_size, FQ_SCALE_F16, codes, scales_f16, sse_out, max_abs_out,
                             workspace, workspace_bytes, stream);
}

int fq_quant_error_sf(const void* W_f16, int64_t K, int64_t N, int bits, int group_size, int scale_format,
                      const void* codes, const void* scales_f16, double* sse_out, double* max_abs_out,
                      void* workspace, size_t workspace_bytes, void* stream) {
    if (!W_f16 || !codes || !scales_f16 || !sse_out || !max_abs_out) return FQ_ERR_INVALID_ARG;
    if (scale_format != FQ_SCALE_F16 && scale_format != FQ_SCALE_BF16) return FQ_ERR_INVALID_ARG;
    int g = 0;
    const int st = check_shape(K, N, bits, group_size, &g);
    if (st != FQ_OK) return st;
    if (!workspace || workspace_bytes < fq_quant_error_workspace_bytes(K, N)) return FQ_ERR_WORKSPACE;
    double out[2] = {0.0, 0.0};
    const int rc = fq_launch_quant_error(W_f16, K, N, bits, g, scale_format, codes, scales_f16, out, workspace,
                                         (hipStream_t)stream);
    if (rc != FQ_OK) return rc;
    *sse_out = out[0];
    *max_abs_out = out[1];
    return FQ_OK;
}

// internal activation kind: FQ_F16, FQ_BF16, or 2 = bf16 activations with bf16 scales; -1 = refuse
static int act_kind(int act_dtype, int scale_format, int* status) {
    *status = FQ_OK;
    if (act_dtype != FQ_F16 && act_dtype != FQ_BF16) *status = FQ_ERR_INVALID_ARG;
    else if (scale_format != FQ_SCALE_F16 && scale_format != FQ_SCALE_BF16) *status = FQ_ERR_INVALID_ARG;
    else if (scale_format == FQ_SCALE_BF16 && act_dtype != FQ_BF16) *status = FQ_ERR_UNSUPPORTED;
    if (*status != FQ_OK) return -1;
    return scale_format == FQ_SCALE_BF16 ? 2 : act_dtype;
}

int fq_gemm(const void* A, int act_dtype, int64_t M, int64_t N, int64_t K, const void* codes,
            const void* scales_f16, int bits, int group_size, void* C, void* workspace,
            size_t workspace_bytes, void* stream) {
    return fq_gemm_sf(A, act_dtype, M, N, K, codes, scales_f16, FQ_SCALE_F16, bits, group_size, C, workspace,
                      workspace_bytes, stream);
}

int fq_gemm_sf(const void* A, int act_dtype, int64_t M, int64_t N, int64_t K, const void* codes,
               const void* scales_f16, int scale_format, int bits, int group_size, void* C, void* workspace,
               size_t workspace_bytes, void* stream) {
    if (M < 0) return FQ_ERR_INVALID_ARG;
    int kst = FQ_OK;
    const int kind = act_kind(act_dtype, scale_format, &kst);
    if (kst == FQ_ERR_INVALID_ARG) return kst;
    int g = 0;
    const int st = check_shape(K, N, bits, group_size, &g);
    if (st != FQ_OK) return st;
    if (kst != FQ_OK) return kst;
    if (M == 0) return FQ_OK;
    if (!A || !codes || !scales_f16 || !C) return FQ_ERR_INVALID_ARG;
    if (M > (int64_t)1 << 24) return FQ_ERR_UNSUPPORTED;
    const fq_gemm_plan plan = fq_plan_gemm(M, N, K, bits, g, act_dtype);
    const size_t need = plan_bytes(plan, M, N, K, act_dtype, scale_format);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FQ_ERR_WORKSPACE;
    return fq_launch_gemm(plan, A, kind, M, N, K, codes, scales_f16, bits, g, C, workspace,
                          (hipStream_t)stream);
}

}  // extern "C"

// Scratch of fq_gemm_noalloc: a file-scope device array (every GPU the library runs on holds its own copy,
// at its own address, until the process ends).  In host code the array's name is only a handle for
// hipGetSymbolAddress; the address kernels may use is asked for once per device and kept here.
static __device__ __align__(256) unsigned char scratch[FQ_NOALLOC_SCRATCH_BYTES];

namespace {
std::mutex g_scratch_mutex;
void* g_scratch_ptr[64];

// Device address of `scratch` on the current device, or nullptr (with *status set) on failure.
void* scratch_of_current_device(int* status) {
    int dev = 0;
    *status = FQ_OK;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) {
        *status = FQ_ERR_HIP;
        return nullptr;
    }
    std::lock_guard<std::mutex> lock(g_scratch_mutex);
    if (!g_scratch_ptr[dev]) {
        void* p = nullptr;
        if (hipGetSymbolAddress(&p, HIP_SYMBOL(scratch)) != hipSuccess || !p) {
            (void)hipGetLastError();
            *status = FQ_ERR_HIP;
            return nullptr;
        }
        g_scratch_ptr[dev] = p;
    }
    return g_scratch_ptr[dev];
}
}  // namespace

extern "C" {

int fq_gemm_noalloc(const void* A, int act_dtype, int64_t M, int64_t N, int64_t K, const void* codes,
                    const void* scales_f16, int bits, int group_size, void* C, void* stream) {
    if (M < 0) return FQ_ERR_INVALID_ARG;
    int kst = FQ_OK;
    const int kind = act_kind(act_dtype, FQ_SCALE_F16, &kst);
    if (kst != FQ_OK) return kst;
    int g = 0;
    const int st = check_shape(K, N, bits, group_size, &g);
    if (st != FQ_OK) return st;
    if (M == 0) return FQ_OK;
    if (!A || !codes || !scales_f16 || !C) return FQ_ERR_INVALID_ARG;
    if (M > (int64_t)1 << 24) return FQ_ERR_UNSUPPORTED;
    const fq_gemm_plan plan = fq_plan_gemm(M, N, K, bits, g, act_dtype);
    const size_t need = plan_bytes(plan, M, N, K, act_dtype, FQ_SCALE_F16);
    if (need > (size_t)FQ_NOALLOC_SCRATCH_BYTES) return FQ_ERR_WORKSPACE;   // beyond the static scratch
    void* ws = nullptr;
    if (need > 0) {
        int sst = FQ_OK;
        ws = scratch_of_current_device(&sst);
        if (!ws) return sst;
    }
    // Nothing in the scratch has to start at zero: every partial sum and every rewritten activation row that this
    // call reads it has written itself, in an earlier kernel or (fq_split_sum.h) in the blocks of the same one that
    // took their ticket before.
    return fq_launch_gemm(plan, A, kind, M, N, K, codes, scales_f16, bits, g, C, ws, (hipStream_t)stream);
}

size_t fq_gemm_noalloc_scratch_bytes(void) { return (size_t)FQ_NOALLOC_SCRATCH_BYTES; }

static int check_grouped(const int32_t* offsets_host, int E, int64_t N, int64_t K, int bits, int group_size, int* g) {
    if (E > 256) return FQ_ERR_UNSUPPORTED;
    const int st = check_shape(K, N, bits, group_size, g);
    if (st != FQ_OK || E == 0) return st;
    if (offsets_host[0] != 0) return FQ_ERR_INVALID_ARG;
    for (int e = 0; e < E; ++e)
        if (offsets_host[e + 1] < offsets_host[e]) return FQ_ERR_INVALID_ARG;
    return FQ_OK;
}

int fq_gemm_grouped(const void* A, int act_dtype, const int32_t* offsets_host, int E, int64_t N,
                    int64_t K, const void* codes, const void* scales_f16, int bits, int group_size,
                    void* C, void* workspace, size_t workspace_bytes, void* stream) {
    return fq_gemm_grouped_sf(A, act_dtype, offsets_host, E, N, K, codes, scales_f16, FQ_SCALE_F16, bits,
                              group_size, C, workspace, workspace_bytes, stream);
}

int fq_gemm_grouped_sf(const void* A, int act_dtype, const int32_t* offsets_host, int E, int64_t N,
                       int64_t K, const void* codes, const void* scales_f16, int scale_format, int bits,
                       int group_size, void* C, void* workspace, size_t workspace_bytes, void* stream) {
    (void)workspace; (void)workspace_bytes;
    if (!offsets_host || E < 0) return FQ_ERR_INVALID_ARG;
    int kst = FQ_OK;
    const int kind = act_kind(act_dtype, scale_format, &kst);
    if (kst != FQ_OK) return kst;
    int g = 0;
    const int st = check_grouped(offsets_host, E, N, K, bits, group_size, &g);
    if (st != FQ_OK) return st;
    if (E == 0 || offsets_host[E] == 0) return FQ_OK;
    if (!A || !codes || !scales_f16 || !C) return FQ_ERR_INVALID_ARG;
    return fq_launch_gemm_grouped(A, kind, offsets_host, E, N, K, codes, scales_f16, bits, g, C,
                                  (hipStream_t)stream);
}

int fq_gemm_grouped_describe(const int32_t* offsets_host, int E, int64_t N, int64_t K, int bits, int group_size,
                             char* buf, size_t buf_bytes) {
    if (!offsets_host || E < 0 || !buf || buf_bytes == 0) return FQ_ERR_INVALID_ARG;
    int g = 0;
    const int st = check_grouped(offsets_host, E, N, K, bits, group_size, &g);
    if (st != FQ_OK) return st;
    if (E == 0 || offsets_host[E] == 0) {
        snprintf(buf, buf_bytes, "empty");
        return FQ_OK;
    }
    const fq_grouped_plan p = fq_plan_grouped(offsets_host, E, N, K, bits, g);
    int count[FQ_TILE_CLASSES] = {}, classes = 0;
    for (int e = 0; e < E; ++e)
        for (int32_t left = offsets_host[e + 1] - offsets_host[e], take = 0; left > 0; left -= take)
            classes += count[fq_next_tile(p, left, &take)]++ == 0;
    snprintf(buf, buf_bytes, "rows128=%d rows64=%d mid-m=%d (gp=%d kw=%d) small-m=%d streams=%d", count[FQ_TILE_128],
             count[FQ_TILE_64], count[FQ_TILE_MID], p.mid.gp, p.mid.kw, count[FQ_TILE_SMALL], p.fork ? classes : 1);
    return FQ_OK;
}

// ------------------------------------------------------------------------------------------ attention
// FQ_OK, or what is wrong with types and head counts
static int check_heads(int act_dtype, int q_heads, int kv_heads, int head_dim) {
    if (act_dtype != FQ_F16 && act_dtype != FQ_BF16) return FQ_ERR_INVALID_ARG;
    if (q_heads <= 0 || kv_heads <= 0 || head_dim <= 0 || q_heads % kv_heads != 0) return FQ_ERR_INVALID_ARG;
    return head_dim % 8 != 0 || head_dim > 128 || q_heads > 4096 ? FQ_ERR_UNSUPPORTED : FQ_OK;
}

static bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Whether n things a stride apart reach further than any memory does (the sums of offsets below stay within 63 bits)
static bool too_far(int64_t n, int64_t stride) { return stride > ((int64_t)1 << 58) / (n > 0 ? n : 1); }

static int check_rows(const fq_heads* x, int64_t rows, int heads) {
    if (!x->data || x->row_stride < 0 || x->head_stride < 0) return FQ_ERR_INVALID_ARG;
    if (!aligned16(x->data) || x->row_stride % 8 != 0 || x->head_stride % 8 != 0 || too_far(rows, x->row_stride) ||
        too_far(heads, x->head_stride))
        return FQ_ERR_UNSUPPORTED;
    return FQ_OK;
}

static int check_cache(const fq_kv_pages* c, int kv_heads, int head_dim) {
    if (!c->k || !c->v || c->pages <= 0 || c->page_size <= 0) return FQ_ERR_INVALID_ARG;
    // (a slot's head_dim values are its own: no stride is shorter, unless there is only one of what it steps over)
    if ((c->pages > 1 && c->page_stride < head_dim) || (c->page_size > 1 && c->token_stride < head_dim) ||
        (kv_heads > 1 && c->head_stride < head_dim) || c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0)
        return FQ_ERR_INVALID_ARG;
    if (!aligned16(c->k) || !aligned16(c->v) || c->page_stride % 8 != 0 || c->token_stride % 8 != 0 || c->head_stride % 8 != 0)
        return FQ_ERR_UNSUPPORTED;
    if (too_far(c->pages, c->page_stride) || too_far(c->page_size, c->token_stride) || too_far(kv_heads, c->head_stride)) return FQ_ERR_UNSUPPORTED;
    return c->pages > INT32_MAX / c->page_size ? FQ_ERR_UNSUPPORTED : FQ_OK;
}

// Whether memory that a call writes lies among the cache's keys or values (from the first of them to the last)
static bool over_cache(const void* p, size_t bytes, const fq_kv_pages* c, int kv_heads, int head_dim) {
    const size_t all = (size_t)((c->pages - 1) * c->page_stride + (c->page_size - 1) * c->token_stride + (kv_heads - 1) * c->head_stride + head_dim) * 2;
    return fq_overlaps(p, bytes, {{c->k, all}, {c->v, all}});
}

int fq_qk_norm_rope(const void* qkv, int act_dtype, int64_t tokens, int64_t row_stride, int q_heads, int kv_heads, int head_dim,
                    const void* q_weight, const void* k_weight, float eps, const float* table, int64_t table_rows, int rot_dim,
                    int interleaved, const int32_t* positions, void* q_out, void* k_out, const fq_kv_pages* cache,
                    const int64_t* slots, void* stream) {
    if (tokens < 0 || rot_dim < 0 || rot_dim > head_dim || !(eps >= 0.0f && eps <= 3.4e38f)) return FQ_ERR_INVALID_ARG;
    const int st = check_heads(act_dtype, q_heads, kv_heads, head_dim);
    if (st != FQ_OK) return st;
    const int64_t row = ((int64_t)q_heads + 2 * (int64_t)kv_heads) * head_dim;
    if (row_stride < row && tokens > 1) return FQ_ERR_INVALID_ARG;
    if (tokens > 0 && (!cache != !slots || (!k_out && !cache))) return FQ_ERR_INVALID_ARG;
    if (rot_dim > 0 && (table_rows <= 0 || !table || (!positions && tokens > 0))) return FQ_ERR_INVALID_ARG;
    if (rot_dim % 8 != 0 || tokens >= (int64_t)1 << 24 || too_far(tokens, row_stride) || row_stride % 8 != 0) return FQ_ERR_UNSUPPORTED;
    if (cache) {
        const int cst = check_cache(cache, kv_heads, head_dim);
        if (cst != FQ_OK) return cst;
    }
    if (tokens == 0) return FQ_OK;
    if (!qkv || !q_out) return FQ_ERR_INVALID_ARG;
    if (!aligned16(qkv) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(q_weight) || !aligned16(k_weight)) return FQ_ERR_UNSUPPORTED;
    const size_t read = (size_t)((tokens - 1) * row_stride + row) * 2;
    const size_t q_bytes = (size_t)tokens * q_heads * head_dim * 2, k_bytes = (size_t)tokens * kv_heads * head_dim * 2;
    if (fq_overlaps(q_out, q_bytes, {{qkv, read}})) return FQ_ERR_INVALID_ARG;
    if (k_out && fq_overlaps(k_out, k_bytes, {{qkv, read}, {q_out, q_bytes}})) return FQ_ERR_INVALID_ARG;
    if (cache && (over_cache(qkv, read, cache, kv_heads, head_dim) || over_cache(q_out, q_bytes, cache, kv_heads, head_dim) ||
                  (k_out && over_cache(k_out, k_bytes, cache, kv_heads, head_dim))))
        return FQ_ERR_INVALID_ARG;
    fq_rope_args a = {qkv, tokens, row_stride, q_heads, kv_heads, head_dim, q_weight, k_weight, eps, table, table_rows, rot_dim, interleaved != 0,
                      positions, q_out, k_out, {}, slots};
    if (cache) a.cache = *cache;
    return fq_launch_qk_norm_rope(act_dtype, a, (hipStream_t)stream);
}

static constexpr int32_t MOST_PLACES = INT32_MAX - 1024;

static int check_offsets(const int32_t* offsets, int sequences) {
    if (offsets[0] != 0) return FQ_ERR_INVALID_ARG;
    for (int b = 0; b < sequences; ++b)
        if (offsets[b + 1] < offsets[b]) return FQ_ERR_INVALID_ARG;
    return FQ_OK;
}

// The checks that need no data pointer; fills what they have seen.
static int check_prompt(int act_dtype, int q_heads, int kv_heads, int head_dim, const int32_t* q_offsets, const int32_t* k_offsets,
                        int sequences, fq_prompt_args* a) {
    if (!q_offsets || sequences < 0) return FQ_ERR_INVALID_ARG;
    if (!k_offsets) k_offsets = q_offsets;
    int st = check_heads(act_dtype, q_heads, kv_heads, head_dim);
    if (st != FQ_OK) return st;
    if (sequences > 65536) return FQ_ERR_UNSUPPORTED;
    // (the kernels count up to a few tiles behind the last row)
    if (q_offsets[sequences] > MOST_PLACES || k_offsets[sequences] > MOST_PLACES) return FQ_ERR_UNSUPPORTED;
    st = check_offsets(q_offsets, sequences);
    if (st == FQ_OK && k_offsets != q_offsets) st = check_offsets(k_offsets, sequences);
    if (st != FQ_OK) return st;
    a->q_heads = q_heads;
    a->kv_heads = kv_heads;
    a->head_dim = head_dim;
    a->q_offsets = q_offsets;
    a->k_offsets = k_offsets;
    a->sequences = sequences;
    return fq_prompt_fits(*a) ? FQ_OK : FQ_ERR_UNSUPPORTED;
}

// 1 / sqrt(head_dim) for 0; false: not a scale
static bool effective_scale(float* scale, int head_dim) {
    if (*scale == 0.0f) *scale = 1.0f / __builtin_sqrtf((float)head_dim);
    return *scale > 0.0f && *scale <= 3.4e38f;
}

size_t fq_attention_prompt_workspace_bytes(int q_heads, int kv_heads, int head_dim, const int32_t* q_offsets_host,
                                           const int32_t* k_offsets_host, int sequences) {
    fq_prompt_args a = {};
    if (check_prompt(FQ_F16, q_heads, kv_heads, head_dim, q_offsets_host, k_offsets_host, sequences, &a) != FQ_OK) return 0;
    return fq_prompt_bytes(a);
}

int fq_attention_prompt(const fq_heads* q, const fq_heads* k, const fq_heads* v, int act_dtype, int q_heads, int kv_heads, int head_dim,
                        const int32_t* q_offsets_host, const int32_t* k_offsets_host, int sequences, float scale, void* out,
                        void* workspace, size_t workspace_bytes, void* stream) {
    fq_prompt_args a = {};
    int st = check_prompt(act_dtype, q_heads, kv_heads, head_dim, q_offsets_host, k_offsets_host, sequences, &a);
    if (st != FQ_OK) return st;
    if (!effective_scale(&scale, head_dim)) return FQ_ERR_INVALID_ARG;
    const int64_t rows = a.q_offsets[sequences], keys = a.k_offsets[sequences];
    if (rows == 0) return FQ_OK;
    if (!q || !out || (keys > 0 && (!k || !v))) return FQ_ERR_INVALID_ARG;
    if ((st = check_rows(q, rows, q_heads)) != FQ_OK) return st;
    if (keys > 0 && ((st = check_rows(k, keys, kv_heads)) != FQ_OK || (st = check_rows(v, keys, kv_heads)) != FQ_OK)) return st;
    if (!aligned16(out)) return FQ_ERR_UNSUPPORTED;
    const size_t bytes = (size_t)rows * q_heads * head_dim * 2;
    auto span = [&](const fq_heads* x, int64_t n, int heads) {
        return fq_span{x->data, (size_t)((n - 1) * x->row_stride + (heads - 1) * x->head_stride + head_dim) * 2};
    };
    if (fq_overlaps(out, bytes, {span(q, rows, q_heads)}) ||
        (keys > 0 && fq_overlaps(out, bytes, {span(k, keys, kv_heads), span(v, keys, kv_heads)})))
        return FQ_ERR_INVALID_ARG;
    const size_t need = fq_prompt_bytes(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FQ_ERR_WORKSPACE;
    a.q = *q;
    if (keys > 0) a.k = *k, a.v = *v;
    a.scale = scale;
    a.out = out;
    return fq_launch_attention_prompt(act_dtype, a, workspace, (hipStream_t)stream);
}

static int check_tree(int act_dtype, int64_t sequences, int64_t nodes, int q_heads, int kv_heads, int head_dim, int64_t table_width,
                      int page_size, fq_tree_args* a) {
    if (sequences < 0 || nodes < 0 || table_width < 0 || page_size <= 0) return FQ_ERR_INVALID_ARG;
    const int st = check_heads(act_dtype, q_heads, kv_heads, head_dim);
    if (st != FQ_OK) return st;
    if (sequences > 65536 || nodes > 1 << 20 || sequences * nodes > 1 << 24 || table_width > MOST_PLACES / page_size) return FQ_ERR_UNSUPPORTED;
    a->sequences = sequences;
    a->nodes = (int)nodes;
    a->q_heads = q_heads;
    a->kv_heads = kv_heads;
    a->head_dim = head_dim;
    a->table_width = table_width;
    a->cache.page_size = page_size;
    return fq_tree_fits(*a) ? FQ_OK : FQ_ERR_UNSUPPORTED;
}

size_t fq_attention_tree_workspace_bytes(int64_t sequences, int64_t nodes, int q_heads, int kv_heads, int head_dim, int64_t table_width,
                                         int page_size) {
    fq_tree_args a = {};
    if (check_tree(FQ_F16, sequences, nodes, q_heads, kv_heads, head_dim, table_width, page_size, &a) != FQ_OK) return 0;
    if (sequences == 0 || nodes == 0) return 0;
    return fq_tree_bytes(a);
}

int fq_attention_tree(const fq_heads* q, int act_dtype, int64_t sequences, int64_t nodes, int q_heads, int kv_heads, int head_dim,
                      const fq_kv_pages* cache, const int32_t* page_table, int64_t table_width, const int32_t* context_lens,
                      const uint64_t* mask, int64_t mask_stride, float scale, void* out, void* workspace, size_t workspace_bytes,
                      void* stream) {
    if (!cache) return FQ_ERR_INVALID_ARG;
    fq_tree_args a = {};
    int st = check_tree(act_dtype, sequences, nodes, q_heads, kv_heads, head_dim, table_width, cache->page_size, &a);
    if (st != FQ_OK) return st;
    if ((st = check_cache(cache, kv_heads, head_dim)) != FQ_OK) return st;
    if (!effective_scale(&scale, head_dim) || mask_stride < 0) return FQ_ERR_INVALID_ARG;
    if (sequences == 0 || nodes == 0) return FQ_OK;
    if (!q || !out || !context_lens || (!page_table && table_width > 0)) return FQ_ERR_INVALID_ARG;
    if (mask && mask_stride != 0 && mask_stride < nodes * ((nodes + 63) / 64)) return FQ_ERR_INVALID_ARG;
    if ((st = check_rows(q, sequences * nodes, q_heads)) != FQ_OK) return st;
    if (!aligned16(out) || too_far(sequences, mask_stride)) return FQ_ERR_UNSUPPORTED;
    const size_t bytes = (size_t)(sequences * nodes) * q_heads * head_dim * 2;
    const size_t words = (size_t)((mask_stride ? (sequences - 1) * mask_stride : 0) + nodes * ((nodes + 63) / 64));
    if (fq_overlaps(out, bytes, {{q->data, (size_t)((sequences * nodes - 1) * q->row_stride + (q_heads - 1) * q->head_stride + head_dim) * 2},
                                 {page_table, (size_t)(sequences * table_width) * 4}, {context_lens, (size_t)sequences * 4}, {mask, mask ? words * 8 : 0}}) ||
        over_cache(out, bytes, cache, kv_heads, head_dim))
        return FQ_ERR_INVALID_ARG;
    const size_t need = fq_tree_bytes(a);
    if (need > 0 && (!workspace || workspace_bytes < need)) return FQ_ERR_WORKSPACE;
    a.q = *q;
    a.cache = *cache;
    a.page_table = page_table;
    a.context_lens = context_lens;
    a.mask = mask;
    a.mask_stride = mask_stride;
    a.scale = scale;
    a.out = out;
    return fq_launch_attention_tree(act_dtype, a, workspace, (hipStream_t)stream);
}

int fq_gemm_describe(int64_t M, int64_t N, int64_t K, int bits, int group_size, char* buf,
                     size_t buf_bytes) {
    if (!buf || buf_bytes == 0 || M < 0) return FQ_ERR_INVALID_ARG;
    int g = 0;
    const int st = check_shape(K, N, bits, group_size, &g);
    if (st != FQ_OK) return st;
    if (M == 0) {
        snprintf(buf, buf_bytes, "empty");
        return FQ_OK;
    }
    const fq_gemm_plan p = fq_plan_gemm(M, N, K, bits, g, FQ_BF16);
    if (p.kind == 0) {
        snprintf(buf, buf_bytes, "small-m variant=%d gp=%d kw=%d au=%d waves=%d splits=%d", p.variant, p.gp,
                 p.kw, p.au, p.waves, p.splits);
        return FQ_OK;
    }
    // One form for all products of more than 16 rows.  mt and waves are the class of the block shape (32, 64 or 128
    // rows, 4 or 8 waves); a shape that is not its class's own follows behind it.  Described for bfloat16 activations; the
    // shape that binary16 ones take instead needs the same scratch.
    int kbs = p.kb_per_split, cls = p.mt <= 2 ? 2 : (p.mt <= 4 ? 4 : 8);
    const bool streams = p.kind == 2 || p.kind == 3;
    if (p.kind == 3 && M > 256) cls = 8;
    // (32- and 64-row blocks of more than 256 rows stand in the class of 128 rows and 4 waves, whose k-blocks are as long as theirs)
    auto below_class = [&](const fq_gemm_plan& q) { return q.kind == 1 && q.mt < 5 && M > 256; };
    const bool low = below_class(p);
    if (low) cls = 8;
    if (streams) {
        const int KB = (int)(K / fq_mma_kblk(bits, cls, 8, K, g));
        kbs = (KB + p.splits - 1) / p.splits;
    }
    const int n = snprintf(buf, buf_bytes, "tiled mt=%d waves=%d splits=%d kb_per_split=%d tail=%dx%d", cls,
                           streams ? 8 : (low ? 4 : p.waves), p.splits, kbs, p.tail_tiles, p.tail_tiles > 0 ? p.tail_splits : 1);
    if (n < 0 || (size_t)n >= buf_bytes) return FQ_OK;
    const fq_gemm_plan f = fq_plan_gemm(M, N, K, bits, g, FQ_F16);
    if (streams)
        snprintf(buf + n, buf_bytes - n, "%s mid-m rows=%d gp=%d kw=%d waves=%d", p.nt == 1 ? " cols=16" : "", 16 * p.mt, p.gp, p.kw,
                 p.waves);
    else if (low || fq_flexible(p))
        snprintf(buf + n, buf_bytes - n, " rows=%d cols=%d", 16 * p.mt, p.waves * p.nt * FQ_NTILE);
    else if (below_class(f) || fq_flexible(f))
        snprintf(buf + n, buf_bytes - n, " f16: rows=%d cols=%d", 16 * f.mt, f.waves * f.nt * FQ_NTILE);
    return FQ_OK;
}

int fq_stream_read_probe(const void* buf, size_t bytes, void* sink, void* stream) {
    if (!buf || !sink || bytes == 0 || bytes % 16 != 0) return FQ_ERR_INVALID_ARG;
    return fq_launch_stream_read_probe(buf, bytes, sink, (hipStream_t)stream);
}

size_t fq_mfma_rate_probe_operand_bytes(void) { return fq_mfma_probe_operand_bytes(); }
size_t fq_mfma_rate_probe_sink_bytes(void) { return fq_mfma_probe_sink_bytes(); }
double fq_mfma_rate_probe_flops(int iterations, int int8) {
    return iterations > 0 ? fq_mfma_probe_flops(iterations, int8 != 0) : 0.0;
}

int fq_mfma_rate_probe(const void* operands, size_t operand_bytes, void* sink, size_t sink_bytes, int iterations,
                       int lds_reads, int int8, void* stream) {
    if (!operands || !sink || iterations <= 0 || iterations > (1 << 16)) return FQ_ERR_INVALID_ARG;
    if (operand_bytes < fq_mfma_probe_operand_bytes() || sink_bytes < fq_mfma_probe_sink_bytes()) return FQ_ERR_WORKSPACE;
    return fq_launch_mfma_rate_probe(operands, sink, iterations, lds_reads != 0, int8 != 0, (hipStream_t)stream);
}

const char* fq_status_string(int status) {
    switch (status) {
        case FQ_OK: return "FQ_OK";
        case FQ_ERR_INVALID_ARG: return "FQ_ERR_INVALID_ARG";
        case FQ_ERR_UNSUPPORTED: return "FQ_ERR_UNSUPPORTED";
        case FQ_ERR_WORKSPACE: return "FQ_ERR_WORKSPACE";
        case FQ_ERR_HIP: return "FQ_ERR_HIP";
        default: return "FQ_ERR_UNKNOWN";
    }
}

const char* fq_version(void) { return "0.1"; }

}  // extern "C"
