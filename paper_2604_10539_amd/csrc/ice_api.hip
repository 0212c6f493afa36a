// Host side of the C ABI: argument validation, workspace layout, launch sequencing.
// No call here allocates device memory, synchronises, or reads device memory.
#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <mutex>
#include <new>
#include <unordered_map>

#include "ice_cache.h"
#include "ice_internal.h"

struct ice_index : ice::Host {};

namespace {

using namespace ice;

thread_local char g_err[512] = "";

ice_status_t fail(ice_status_t code, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return code;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

ice_status_t check_cfg(const ice_config_t *c) {
    if (!c) return fail(ICE_ERR_INVALID_ARG, "config is null");
    if (c->batch < 1 || c->n_kv_heads < 1 || c->max_tokens < 1 || c->kmeans_iters < 1)
        return fail(ICE_ERR_INVALID_ARG, "batch, n_kv_heads, max_tokens and kmeans_iters must be >= 1");
    if (c->head_dim != kD) return fail(ICE_ERR_UNSUPPORTED, "head_dim %d: only 128 is supported", c->head_dim);
    if (c->group_size != 1 && c->group_size != 2 && c->group_size != 4 && c->group_size != 8)
        return fail(ICE_ERR_UNSUPPORTED, "group_size %d: only 1, 2, 4, 8 are supported", c->group_size);
    if ((long long)c->batch * c->n_kv_heads > 65535) return fail(ICE_ERR_UNSUPPORTED, "more than 65535 units");
    return ICE_OK;
}

ice_status_t check_shape(int page_size, int n_clusters) {
    if (page_size != 16 && page_size != 32 && page_size != 64)
        return fail(ICE_ERR_UNSUPPORTED, "page_size %d: only 16, 32, 64 are supported", page_size);
    if (n_clusters < 1) return fail(ICE_ERR_INVALID_ARG, "n_clusters must be >= 1");
    if (n_clusters > 8192) return fail(ICE_ERR_UNSUPPORTED, "n_clusters %d: at most 8192", n_clusters);
    return ICE_OK;
}

// Carves the workspace; with base == nullptr only measures.  Every region is 256-byte aligned.
size_t lay_out(const ice_config_t &cfg, int s, int C, char *base, Dev *out) {
    Dev d{};
    d.U = cfg.batch * cfg.n_kv_heads;
    d.G = cfg.group_size;
    d.s = s;
    d.C = C;
    d.Cpad = round_up(C, 32);
    d.max_tokens = cfg.max_tokens;
    d.max_pages = cfg.max_tokens / s + C;
    const size_t U = d.U, MP = d.max_pages, MT = d.max_tokens, CP = d.Cpad;
    size_t off = 0;
    auto take = [&](size_t bytes) -> char * {
        char *p = base ? base + off : nullptr;
        off += (bytes + 255) / 256 * 256;
        return p;
    };
    d.Kp = (bf16_t *)take(U * MP * s * kD * 2);
    d.Vp = (bf16_t *)take(U * MP * s * kD * 2);
    d.page_cluster = (int *)take(U * MP * 4);
    d.page_fill = (int *)take(U * MP * 4);
    d.page_pos = (int *)take(U * MP * s * 4);
    d.cluster_tail = (int *)take(U * C * 4);
    d.cluster_cnt = (int *)take(U * C * 4);
    d.tail_fill = (int *)take(U * C * 4);
    d.tail_sum = (float *)take(U * C * kD * 4);
    d.cluster_sum = (float *)take(U * C * kD * 4);
    d.centroid = (float *)take(U * C * kD * 4);
    d.page_sum = (float *)take(U * MP * kD * 4);
    d.rep = (bf16_t *)take(U * MP * kD * 2);
    d.n_pages = (int *)take(U * 4);
    d.n_tokens = (int *)take(U * 4);
    for (int b = 0; b < 2; ++b) {
        d.cent_bf16[b] = (bf16_t *)take(U * CP * kD * 2);
        d.cnorm[b] = (float *)take(U * CP * 4);
    }
    d.kaug = (bf16_t *)take(U * MT * 2);
    for (int b = 0; b < 2; ++b) d.caug[b] = (bf16_t *)take(U * CP * 2);
    d.cent_aug = (float *)take(U * C * 4);
    d.csum_aug = (float *)take(U * C * 4);
    d.c2 = (float *)take(U * 4);
    d.top_cent = (float *)take(U * kTopMax * kD * 4);
    d.top_bf16 = (bf16_t *)take(U * kTopMax * kD * 2);
    d.top_of = (int *)take(U * C * 4);
    d.top_cnt = (int *)take(U * kTopMax * 4);
    d.top_init = (int *)take(U * kTopMax * 4);
    d.init_idx = (int *)take(U * C * 4);
    d.assign = (int *)take(U * MT * 4);
    d.packed = (unsigned long long *)take(U * MT * 8);
    d.order = (int *)take(U * MT * 4);
    d.moved = (uint32_t *)take(U * CP * 4);
    d.touched = (unsigned char *)take(U * CP);
    d.any_moved = (int *)take(U * 2 * 4);
    d.large_keys = (int *)take(U * 4);
    d.page_base = (int *)take(U * C * 4);
    d.range_off = (uint32_t *)take(sort_ranges_max(d.U, d.max_tokens, d.Cpad) * CP * 4);
    d.attn_part = (float *)take((size_t)256 * d.G * (kD + 2) * 4);
    d.attn_arrive = (int *)take(U * 4);
    d.scores = (uint32_t *)take(U * MP * 4);
    d.counter = (int *)take(U * 4);
    if (out) *out = d;
    return off;
}

ice_status_t ensure_layout(ice_index *ix, int s, int C) {
    if (ix->laid_out && ix->dev.s == s && ix->dev.C == C) return ICE_OK;
    const size_t need = lay_out(ix->cfg, s, C, nullptr, nullptr);
    if (need > ix->ws_bytes)
        return fail(ICE_ERR_CAPACITY, "workspace has %zu bytes, page_size %d / n_clusters %d need %zu", ix->ws_bytes, s,
                    C, need);
    lay_out(ix->cfg, s, C, ix->ws, &ix->dev);
    ix->dev.tk = ix->geometry;
    ix->laid_out = true;
    ix->built = false;
    return ICE_OK;
}

ice_status_t device_status(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(ICE_ERR_DEVICE, "%s: %s", what, hipGetErrorString(e));
    return ICE_OK;
}

// whether every array is 16-byte aligned device memory of the GPU that holds `ws`, which is the current one, and lies
// inside its allocation
bool all_on_device(const void *const *p, const size_t *bytes, int n, const void *ws) {
    int dev = -1;
    hipPointerAttribute_t at;
    if (hipGetDevice(&dev) != hipSuccess || hipPointerGetAttributes(&at, ws) != hipSuccess) {
        (void)hipGetLastError();
        return false;
    }
    if (at.type != hipMemoryTypeDevice || at.device != dev) return false;
    for (int i = 0; i < n; ++i) {
        if (!aligned16(p[i])) return false;
        if (hipPointerGetAttributes(&at, p[i]) != hipSuccess) {
            (void)hipGetLastError();  // (not an error of the call: the copy calls decide)
            return false;
        }
        if (at.type != hipMemoryTypeDevice || at.device != dev) return false;
        hipDeviceptr_t base = nullptr;
        size_t size = 0;
        if (hipMemGetAddressRange(&base, &size, const_cast<void *>(p[i])) != hipSuccess) {
            (void)hipGetLastError();
            return false;
        }
        if ((size_t)(static_cast<const char *>(p[i]) - static_cast<const char *>(base)) + bytes[i] > size) return false;
    }
    return true;
}

__global__ void fill_i32_kernel(int *p, int n, int v) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) p[i] = v;
}

// token counters, arrival counters and the empty marks of the score slots
void reset_decode_state(const Dev &d, int n_tokens, hipStream_t s) {
    hipLaunchKernelGGL(fill_i32_kernel, dim3((d.U + 255) / 256), dim3(256), 0, s, d.n_tokens, d.U, n_tokens);
    hipLaunchKernelGGL(fill_i32_kernel, dim3((d.U + 255) / 256), dim3(256), 0, s, d.counter, d.U, 0);
    hipLaunchKernelGGL(fill_i32_kernel, dim3((d.U + 255) / 256), dim3(256), 0, s, d.attn_arrive, d.U, 0);
    const int ns = d.U * d.max_pages;
    hipLaunchKernelGGL(fill_i32_kernel, dim3((ns + 255) / 256), dim3(256), 0, s, (int *)d.scores, ns, -1);
}

}  // namespace

namespace ice {

void allow_dynamic_lds(const void *kernel, size_t bytes) {
    static std::mutex mu;
    static std::unordered_map<uintptr_t, size_t> allowed;  // per (kernel, device): the largest size set so far
    int dev = 0;
    (void)hipGetDevice(&dev);
    std::lock_guard<std::mutex> lock(mu);
    size_t &have = allowed[reinterpret_cast<uintptr_t>(kernel) * 64u + (uintptr_t)(dev & 63)];
    if (bytes <= have) return;
    if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == hipSuccess) have = bytes;
}

}  // namespace ice

extern "C" {

const char *ice_last_error(void) { return g_err; }

size_t ice_workspace_bytes(const ice_config_t *cfg, int32_t page_size, int32_t n_clusters) {
    if (check_cfg(cfg) != ICE_OK || check_shape(page_size, n_clusters) != ICE_OK) return 0;
    return lay_out(*cfg, page_size, n_clusters, nullptr, nullptr);
}

ice_status_t ice_create(const ice_config_t *cfg, void *workspace, size_t workspace_bytes, ice_index_t **out) {
    if (!out) return fail(ICE_ERR_INVALID_ARG, "out is null");
    *out = nullptr;
    if (ice_status_t st = check_cfg(cfg)) return st;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
        return fail(ICE_ERR_INVALID_ARG, "workspace is null or not 256-byte aligned");
    if (workspace_bytes == 0) return fail(ICE_ERR_INVALID_ARG, "workspace_bytes is 0");
    ice_index *ix = new (std::nothrow) ice_index();
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "out of host memory");
    ix->cfg = *cfg;
    ix->ws = static_cast<char *>(workspace);
    ix->ws_bytes = workspace_bytes;
    ix->laid_out = false;
    ix->built = false;
    ix->n_tokens = 0;
    ix->build_n = 0;
    ix->n_top = 0;
    ix->cur = 0;
    ix->geometry = 0;
    *out = ix;
    return ICE_OK;
}

ice_status_t ice_destroy(ice_index_t *idx) {
    if (!idx) return fail(ICE_ERR_INVALID_ARG, "index is null");
    delete idx;
    return ICE_OK;
}

ice_status_t ice_build_index(ice_index_t *ix, const void *K, const void *V, int32_t n, int32_t page_size,
                             int32_t n_clusters, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!K || !V || !aligned16(K) || !aligned16(V)) return fail(ICE_ERR_INVALID_ARG, "K or V is null or misaligned");
    if (ix->cfg.init_idx && (reinterpret_cast<uintptr_t>(ix->cfg.init_idx) & 3u))
        return fail(ICE_ERR_INVALID_ARG, "init_idx is misaligned");
    if (ice_status_t st = check_shape(page_size, n_clusters)) return st;
    if (n < 1) return fail(ICE_ERR_INVALID_ARG, "n_tokens must be >= 1");
    if (n_clusters > n) return fail(ICE_ERR_SHAPE, "n_clusters %d exceeds n_tokens %d", n_clusters, n);
    if (n > ix->cfg.max_tokens) return fail(ICE_ERR_SHAPE, "n_tokens %d exceeds max_tokens %d", n, ix->cfg.max_tokens);
    if (ice_status_t st = ensure_layout(ix, page_size, n_clusters)) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    ix->dev.tk = ix->geometry;
    const Dev &d = ix->dev;
    const bf16_t *Kb = static_cast<const bf16_t *>(K), *Vb = static_cast<const bf16_t *>(V);
    ix->built = false;
    int cur = 0;
    if (d.tk) launch_key_aug(d, Kb, n, s);
    launch_init_centroids(d, Kb, n, ix->cfg.init_idx, ix->cfg.seed, cur, s);
    const bool fused = sort_is_fused(d, n);
    const bool near = near_pays(d, n, ix->cfg.kmeans_iters), later = near || (ix->cfg.kmeans_iters > 2 && reassign_pays(d, n));
    for (int t = 0; t < ix->cfg.kmeans_iters; ++t) {
        if (near && t >= 1 && t % kRoundNumbers != 0) launch_near(d, Kb, n, cur, t, fused, s);
        else if (later && t >= 2 && t % kRoundNumbers != 0) launch_reassign(d, Kb, n, cur, t, fused, s);
        else launch_assign(d, Kb, n, cur, t, fused, later && t == 0, s);
        if (!fused) launch_sort(d, n, t, nullptr, nullptr, s);
        launch_means(d, Kb, n, cur, t, t + 1 == ix->cfg.kmeans_iters, s);
        cur ^= 1;
    }
    launch_paginate(d, Kb, Vb, n, true, s);
    if (ice_status_t st = device_status("ice_build_index")) return st;
    ix->cur = cur;
    ix->n_tokens = n;
    ix->build_n = n;
    ix->n_top = 0;
    ix->built = true;
    return ICE_OK;
}

ice_status_t ice_insert_batch(ice_index_t *ix, const void *k, const void *v, int32_t m, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_insert before ice_build_index");
    if (!k || !v || !aligned16(k) || !aligned16(v)) return fail(ICE_ERR_INVALID_ARG, "k or v is null or misaligned");
    if (m < 1) return fail(ICE_ERR_SHAPE, "number of tokens to insert must be >= 1");
    if ((long long)ix->n_tokens + m > ix->cfg.max_tokens)
        return fail(ICE_ERR_CAPACITY, "index holds %d tokens per unit, %d more exceed max_tokens = %d", ix->n_tokens, m,
                    ix->cfg.max_tokens);
    launch_insert(ix->dev, static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v), m, ix->cur,
                  static_cast<hipStream_t>(stream));
    if (ice_status_t st = device_status("ice_insert")) return st;
    ix->n_tokens += m;
    return ICE_OK;
}

ice_status_t ice_insert(ice_index_t *ix, const void *k, const void *v, void *stream) {
    return ice_insert_batch(ix, k, v, 1, stream);
}

static ice_status_t check_select(ice_index_t *ix, const void *q, int32_t budget, const int32_t *ids,
                                 const int32_t *n_sel, const char *who) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "%s before ice_build_index", who);
    if (!q || !aligned16(q)) return fail(ICE_ERR_INVALID_ARG, "q is null or misaligned");
    if (!ids || !n_sel) return fail(ICE_ERR_INVALID_ARG, "page_ids or n_selected is null");
    if (budget < ix->dev.s) return fail(ICE_ERR_SHAPE, "token_budget %d is below page_size %d", budget, ix->dev.s);
    if (ix->dev.max_pages > decode_step_max_pages(ix->dev.G))
        return fail(ICE_ERR_UNSUPPORTED, "%d pages per unit exceed the selection kernel's limit of %d", ix->dev.max_pages,
                    decode_step_max_pages(ix->dev.G));
    if (!decode_step_plan(ix->dev, budget / ix->dev.s, ix->n_tokens / ix->dev.s + ix->dev.C).fits)
        return fail(ICE_ERR_UNSUPPORTED, "token_budget %d (%d pages) and %d pages per unit need more LDS than a CU has for the "
                    "winner lists", budget, budget / ix->dev.s, ix->dev.max_pages);
    return ICE_OK;
}

ice_status_t ice_select(ice_index_t *ix, const void *q, int32_t budget, int32_t *ids, int32_t *n_sel, float *scores,
                        void *stream) {
    if (ice_status_t st = check_select(ix, q, budget, ids, n_sel, "ice_select")) return st;
    launch_decode_step(ix->dev, static_cast<const bf16_t *>(q), budget / ix->dev.s, ix->n_tokens / ix->dev.s + ix->dev.C,
                       ids, n_sel, scores, nullptr, nullptr, 0, nullptr, static_cast<hipStream_t>(stream));
    return device_status("ice_select");
}

static ice_status_t check_resident(const void *rk, const void *rv, int32_t n_res) {
    if (n_res < 0 || n_res > (1 << 20)) return fail(ICE_ERR_SHAPE, "n_resident %d is outside [0, 2^20]", n_res);
    if (n_res > 0 && (!rk || !rv || !aligned16(rk) || !aligned16(rv)))
        return fail(ICE_ERR_INVALID_ARG, "resident_k or resident_v is null or misaligned");
    return ICE_OK;
}

ice_status_t ice_attend_resident(ice_index_t *ix, const void *q, const int32_t *ids, const int32_t *n_sel, int32_t P,
                                 const void *rk, const void *rv, int32_t n_res, float *out, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_attend before ice_build_index");
    if (!q || !aligned16(q)) return fail(ICE_ERR_INVALID_ARG, "q is null or misaligned");
    if (!ids || !n_sel || !out) return fail(ICE_ERR_INVALID_ARG, "page_ids, n_selected or out is null");
    if (P < 1) return fail(ICE_ERR_SHAPE, "n_ids_per_unit must be >= 1");
    if (ice_status_t st = check_resident(rk, rv, n_res)) return st;
    const Resident res = {static_cast<const bf16_t *>(rk), static_cast<const bf16_t *>(rv), n_res, nullptr, nullptr, 0};
    launch_attend(ix->dev, static_cast<const bf16_t *>(q), ids, n_sel, P, res, out, static_cast<hipStream_t>(stream));
    return device_status("ice_attend");
}

ice_status_t ice_attend(ice_index_t *ix, const void *q, const int32_t *ids, const int32_t *n_sel, int32_t P, float *out,
                        void *stream) {
    return ice_attend_resident(ix, q, ids, n_sel, P, nullptr, nullptr, 0, out, stream);
}

ice_status_t ice_attend_noalloc(ice_index_t *ix, const void *q, const int32_t *ids, const int32_t *n_sel, int32_t P, float *out,
                                void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_attend_noalloc before ice_build_index");
    if (!q || !aligned16(q)) return fail(ICE_ERR_INVALID_ARG, "q is null or misaligned");
    if (!ids || !n_sel || !out) return fail(ICE_ERR_INVALID_ARG, "page_ids, n_selected or out is null");
    if (P < 1) return fail(ICE_ERR_SHAPE, "n_ids_per_unit must be >= 1");
    if (ix->dev.U > attend_static_max_units())
        return fail(ICE_ERR_UNSUPPORTED, "%d units: the static scratch array holds the partial results of at most %d",
                    ix->dev.U, attend_static_max_units());
    const hipError_t e = launch_attend_static(ix->dev, static_cast<const bf16_t *>(q), ids, n_sel, P, out,
                                              static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return fail(ICE_ERR_DEVICE, "ice_attend_noalloc: %s", hipGetErrorString(e));
    return device_status("ice_attend_noalloc");
}

ice_status_t ice_select_attend_resident(ice_index_t *ix, const void *q, int32_t budget, const void *rk, const void *rv,
                                        int32_t n_res, int32_t *ids, int32_t *n_sel, float *out, void *stream) {
    if (ice_status_t st = check_select(ix, q, budget, ids, n_sel, "ice_select_attend")) return st;
    if (!out) return fail(ICE_ERR_INVALID_ARG, "out is null");
    if (ice_status_t st = check_resident(rk, rv, n_res)) return st;
    launch_decode_step(ix->dev, static_cast<const bf16_t *>(q), budget / ix->dev.s, ix->n_tokens / ix->dev.s + ix->dev.C, ids,
                       n_sel, nullptr, static_cast<const bf16_t *>(rk), static_cast<const bf16_t *>(rv), n_res, out,
                       static_cast<hipStream_t>(stream));
    return device_status("ice_select_attend");
}

ice_status_t ice_select_attend(ice_index_t *ix, const void *q, int32_t budget, int32_t *ids, int32_t *n_sel, float *out,
                               void *stream) {
    return ice_select_attend_resident(ix, q, budget, nullptr, nullptr, 0, ids, n_sel, out, stream);
}

ice_status_t ice_selected_tokens(ice_index_t *ix, const int32_t *ids, const int32_t *n_sel, int32_t P, int32_t *pos,
                                 int32_t *n_tok, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_selected_tokens before ice_build_index");
    if (!ids || !n_sel || !pos || !n_tok) return fail(ICE_ERR_INVALID_ARG, "a pointer is null");
    if (P < 1 || P > 1024) return fail(ICE_ERR_SHAPE, "n_ids_per_unit %d is outside [1, 1024]", P);
    launch_selected_tokens(ix->dev, ids, n_sel, P, pos, n_tok, static_cast<hipStream_t>(stream));
    return device_status("ice_selected_tokens");
}

ice_status_t ice_attend_tokens(ice_index_t *ix, const void *q, const void *K, const void *V, int32_t n_rows,
                               const int32_t *pos, const int32_t *n_tok, int32_t max_tok, float *out, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->laid_out) return fail(ICE_ERR_STATE, "ice_attend_tokens before ice_build_index or ice_import_index");
    if (!q || !aligned16(q) || !K || !V || !aligned16(K) || !aligned16(V))
        return fail(ICE_ERR_INVALID_ARG, "q, K or V is null or misaligned");
    if (!pos || !n_tok || !out) return fail(ICE_ERR_INVALID_ARG, "token_pos, n_tok or out is null");
    if (n_rows < 1 || max_tok < 1) return fail(ICE_ERR_SHAPE, "n_rows and max_tok must be >= 1");
    const Resident res = {static_cast<const bf16_t *>(K), static_cast<const bf16_t *>(V), max_tok, pos, n_tok, n_rows};
    launch_attend(ix->dev, static_cast<const bf16_t *>(q), nullptr, nullptr, 1, res, out, static_cast<hipStream_t>(stream));
    return device_status("ice_attend_tokens");
}

// ---- the 4-bit sequence cache

static ice_status_t check_cache(const ice_cache_t *c) {
    if (!c) return fail(ICE_ERR_INVALID_ARG, "cache is null");
    if (c->head_dim != kD) return fail(ICE_ERR_UNSUPPORTED, "head_dim %d: only 128 is supported", c->head_dim);
    if (c->block_size != 16 && c->block_size != 32 && c->block_size != 64)
        return fail(ICE_ERR_UNSUPPORTED, "block_size %d: only 16, 32, 64 are supported", c->block_size);
    if (c->n_blocks < 1 || c->n_kv_heads < 1) return fail(ICE_ERR_SHAPE, "n_blocks and n_kv_heads must be >= 1");
    if ((double)c->n_blocks * c->n_kv_heads * c->block_size >= 2147483648.0)
        return fail(ICE_ERR_UNSUPPORTED, "%d blocks of %d tokens for %d KV heads: 2^31 rows or more", c->n_blocks, c->block_size, c->n_kv_heads);
    return ICE_OK;
}

static ice_status_t check_cache_data(const ice_cache_t *c) {
    if (ice_status_t st = check_cache(c)) return st;
    if (!c->data || (reinterpret_cast<uintptr_t>(c->data) & 127u))
        return fail(ICE_ERR_INVALID_ARG, "the cache's data is null or not 128-byte aligned");
    return ICE_OK;
}

static CacheDims cache_dims(const ice_cache_t *c) {
    return {static_cast<uint8_t *>(c->data), c->n_blocks, c->n_kv_heads, c->block_size == 64 ? 2 : c->block_size == 32 ? 1 : 0};
}

static ice_status_t check_table(const ice_cache_t *c, int32_t n_requests, const int32_t *seq_len, const int32_t *table, int32_t max_blocks) {
    if (!seq_len || !table) return fail(ICE_ERR_INVALID_ARG, "seq_len or block_table is null");
    if (n_requests < 1 || n_requests > 65535) return fail(ICE_ERR_SHAPE, "n_requests %d is outside [1, 65535]", n_requests);
    if (max_blocks < 1 || (long long)max_blocks * c->block_size >= 2147483648ll)
        return fail(ICE_ERR_SHAPE, "max_blocks %d: at least 1, and fewer than 2^31 tokens", max_blocks);
    return ICE_OK;
}

size_t ice_cache_bytes(const ice_cache_t *c) {
    if (check_cache(c) != ICE_OK) return 0;
    return (size_t)c->n_blocks * c->n_kv_heads * (c->block_size / kCacheTile) * kCacheTileBytes;
}

ice_status_t ice_plan_blocks(int32_t n_requests, int32_t block_size, int32_t max_blocks, int32_t n_blocks, const int32_t *new_len,
                             const int32_t *cached_len, int32_t *seq_len, int32_t *table, int32_t *free_ids, const int32_t *n_free,
                             int32_t *n_free_left, int32_t *query_start, int32_t *slots, int32_t n_slots, int32_t *info, void *stream) {
    if (!new_len || !cached_len || !seq_len || !table || !free_ids || !n_free || !n_free_left || !query_start || !slots || !info)
        return fail(ICE_ERR_INVALID_ARG, "a pointer is null");
    if (block_size != 16 && block_size != 32 && block_size != 64)
        return fail(ICE_ERR_UNSUPPORTED, "block_size %d: only 16, 32, 64 are supported", block_size);
    if (n_requests < 1 || n_requests > kPlanRequests) return fail(ICE_ERR_SHAPE, "n_requests %d is outside [1, %d]", n_requests, kPlanRequests);
    if (n_slots < 1 || n_slots > (1 << 30)) return fail(ICE_ERR_SHAPE, "n_slots %d is outside [1, 2^30]", n_slots);
    if (n_blocks < 1 || (long long)n_blocks * block_size >= 2147483648ll)
        return fail(ICE_ERR_SHAPE, "n_blocks %d: at least 1, and fewer than 2^31 slots", n_blocks);
    if (max_blocks < 1 || (long long)max_blocks * block_size >= 2147483648ll)
        return fail(ICE_ERR_SHAPE, "max_blocks %d: at least 1, and fewer than 2^31 tokens", max_blocks);
    launch_cache_plan({n_requests, block_size == 64 ? 6 : block_size == 32 ? 5 : 4, max_blocks, n_blocks, new_len, cached_len, seq_len, table,
                       free_ids, n_free, n_free_left, query_start, slots, n_slots, info, false},
                      static_cast<hipStream_t>(stream));
    return device_status("ice_plan_blocks");
}

ice_status_t ice_cache_write(const ice_cache_t *c, const void *k, const void *v, int64_t k_stride, int64_t v_stride, const int32_t *slots,
                             int32_t n_tokens, void *stream) {
    if (ice_status_t st = check_cache_data(c)) return st;
    if (n_tokens < 0) return fail(ICE_ERR_SHAPE, "n_tokens must be >= 0");
    if (n_tokens == 0) return ICE_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return fail(ICE_ERR_INVALID_ARG, "k or v is null or misaligned");
    if (!slots) return fail(ICE_ERR_INVALID_ARG, "slots is null");
    const int64_t row = (int64_t)c->n_kv_heads * kD;
    if ((k_stride & 7) || (v_stride & 7) || (n_tokens > 1 && (k_stride < row || v_stride < row)))
        return fail(ICE_ERR_SHAPE, "strides must be multiples of 8 and at least n_kv_heads * 128");
    if ((double)((n_tokens + 15ll) / 16) * c->n_kv_heads > 1e7) return fail(ICE_ERR_UNSUPPORTED, "too many rows for one call");
    launch_cache_write(cache_dims(c), static_cast<const bf16_t *>(k), static_cast<const bf16_t *>(v), k_stride, v_stride, slots, n_tokens,
                       static_cast<hipStream_t>(stream));
    return device_status("ice_cache_write");
}

ice_status_t ice_cache_read(const ice_cache_t *c, int32_t n_requests, const int32_t *seq_len, const int32_t *table, int32_t max_blocks,
                            const int32_t *first, int32_t n_rows, void *K, void *V, void *stream) {
    if (ice_status_t st = check_cache_data(c)) return st;
    if (ice_status_t st = check_table(c, n_requests, seq_len, table, max_blocks)) return st;
    if (n_rows < 0) return fail(ICE_ERR_SHAPE, "n_rows must be >= 0");
    if (n_rows == 0) return ICE_OK;
    if (!K || !V || !aligned16(K) || !aligned16(V)) return fail(ICE_ERR_INVALID_ARG, "K or V is null or misaligned");
    if ((double)((n_rows + 15ll) / 16) * n_requests * c->n_kv_heads > 1e7) return fail(ICE_ERR_UNSUPPORTED, "too many rows for one call");
    launch_cache_read(cache_dims(c), n_requests, seq_len, table, max_blocks, first, n_rows, static_cast<bf16_t *>(K), static_cast<bf16_t *>(V),
                      static_cast<hipStream_t>(stream));
    return device_status("ice_cache_read");
}

// the sizes that say how an attention call is cut
static ice_status_t plan_attend(const ice_cache_t *c, int32_t G, int32_t n_requests, int32_t max_query, int32_t max_keys, bool listed,
                                CacheAttend &a, size_t *bytes) {
    if (ice_status_t st = check_cache(c)) return st;
    if (G < 1 || G > 16) return fail(ICE_ERR_UNSUPPORTED, "group_size %d: only 1 to 16 are supported", G);
    if (n_requests < 1 || n_requests > 65535) return fail(ICE_ERR_SHAPE, "n_requests %d is outside [1, 65535]", n_requests);
    if (max_query < 1 || max_query > (1 << 24)) return fail(ICE_ERR_SHAPE, "max_query %d is outside [1, 2^24]", max_query);
    if (max_keys < 1 || max_keys > (1 << 30)) return fail(ICE_ERR_SHAPE, "max_keys or max_tok %d is outside [1, 2^30]", max_keys);
    a.c = cache_dims(c);
    a.S = n_requests;
    a.G = G;
    a.max_query = max_query;
    a.max_keys = max_keys;
    a.scale_log2 = 0.12751743f;  // log2(e) / sqrt(128)
    *bytes = plan_cache_attend(a, listed);
    return ICE_OK;
}

size_t ice_cache_attend_bytes(const ice_cache_t *c, int32_t G, int32_t n_requests, int32_t max_query, int32_t max_keys) {
    CacheAttend a{};
    size_t bytes = 0;
    return plan_attend(c, G, n_requests, max_query, max_keys, false, a, &bytes) == ICE_OK ? bytes : 0;
}

size_t ice_cache_attend_tokens_bytes(const ice_cache_t *c, int32_t G, int32_t n_requests, int32_t max_tok) {
    CacheAttend a{};
    size_t bytes = 0;
    return plan_attend(c, G, n_requests, 1, max_tok, true, a, &bytes) == ICE_OK ? bytes : 0;
}

// (the sum of a launch's pieces of 128 keys is counted in 31 bits)
static ice_status_t check_count(const ice_cache_t *c, const CacheAttend &a, bool listed) {
    const double keys = listed ? a.max_keys : (double)a.max_blocks * c->block_size, rows = listed ? 1 : a.max_query * (double)a.G;
    if ((keys / 128 + 3) * (rows / 192 + 2) * (a.S < 1024 ? a.S : 1024) * c->n_kv_heads >= 2147483648.0)
        return fail(ICE_ERR_UNSUPPORTED, "%d requests x %d KV heads x %.0f keys x %.0f query rows: too many for one call", a.S, c->n_kv_heads, keys, rows);
    return ICE_OK;
}

static ice_status_t set_attend(const ice_cache_t *c, CacheAttend &a, const void *q, int64_t q_stride, void *out, int32_t out_type, float *lse, void *ws,
                               size_t ws_bytes, size_t need) {
    if (!q || !aligned16(q)) return fail(ICE_ERR_INVALID_ARG, "q is null or misaligned");
    // (positions are rounded up to steps in 32 bits)
    if ((long long)a.max_blocks * c->block_size > (1 << 30)) return fail(ICE_ERR_SHAPE, "max_blocks %d: more than 2^30 tokens", a.max_blocks);
    if (!a.list_start)  // (else the call has counted its work)
        if (ice_status_t st = check_count(c, a, a.pos != nullptr)) return st;
    if ((q_stride & 7) || (a.T > 1 && q_stride < (int64_t)c->n_kv_heads * a.G * kD))
        return fail(ICE_ERR_SHAPE, "q's stride must be a multiple of 8 and at least n_kv_heads * group_size * 128");
    if (!out || !aligned16(out)) return fail(ICE_ERR_INVALID_ARG, "out is null or misaligned");
    if (out_type != ICE_OUT_F32 && out_type != ICE_OUT_BF16) return fail(ICE_ERR_INVALID_ARG, "out_type %d: ICE_OUT_F32 or ICE_OUT_BF16", out_type);
    if (need && (!ws || !aligned16(ws))) return fail(ICE_ERR_INVALID_ARG, "workspace is null or misaligned");
    if (need > ws_bytes) return fail(ICE_ERR_CAPACITY, "workspace of %zu bytes, %zu are needed", ws_bytes, need);
    a.q = static_cast<const bf16_t *>(q);
    a.q_stride = q_stride;
    a.out = out;
    a.out_bf16 = out_type == ICE_OUT_BF16;
    a.lse = lse;
    a.part = static_cast<float *>(ws);
    return ICE_OK;
}

static ice_status_t cache_attend(const ice_cache_t *c, CacheAttend &a, const void *q, int64_t q_stride, void *out, int32_t out_type,
                                 float *lse, void *ws, size_t ws_bytes, size_t need, void *stream, const char *who) {
    if (ice_status_t st = set_attend(c, a, q, q_stride, out, out_type, lse, ws, ws_bytes, need)) return st;
    launch_cache_attend(a, static_cast<hipStream_t>(stream));
    return device_status(who);
}

ice_status_t ice_cache_attend(const ice_cache_t *c, const void *q, int64_t q_stride, int32_t G, int32_t n_requests, const int32_t *query_start,
                              int32_t n_tokens, int32_t max_query, const int32_t *seq_len, int32_t max_keys, const int32_t *table,
                              int32_t max_blocks, int32_t window, void *out, int32_t out_type, float *lse, void *ws, size_t ws_bytes,
                              void *stream) {
    if (ice_status_t st = check_cache_data(c)) return st;
    if (ice_status_t st = check_table(c, n_requests, seq_len, table, max_blocks)) return st;
    if (!query_start) return fail(ICE_ERR_INVALID_ARG, "query_start is null");
    if (n_tokens < 0) return fail(ICE_ERR_SHAPE, "n_tokens must be >= 0");
    if (window < 0) return fail(ICE_ERR_SHAPE, "window must be >= 0 (0: no window)");
    CacheAttend a{};
    size_t need = 0;
    if (ice_status_t st = plan_attend(c, G, n_requests, max_query, max_keys, false, a, &need)) return st;
    if (n_tokens == 0) return ICE_OK;
    a.T = n_tokens;
    a.query_start = query_start;
    a.seq_len = seq_len;
    a.table = table;
    a.max_blocks = max_blocks;
    a.window = window;
    return cache_attend(c, a, q, q_stride, out, out_type, lse, ws, ws_bytes, need, stream, "ice_cache_attend");
}

ice_status_t ice_cache_attend_tokens(const ice_cache_t *c, const void *q, int64_t q_stride, int32_t G, int32_t n_requests,
                                     const int32_t *seq_len, const int32_t *table, int32_t max_blocks, const int32_t *pos,
                                     const int32_t *n_tok, int32_t max_tok, void *out, int32_t out_type, float *lse, void *ws,
                                     size_t ws_bytes, void *stream) {
    if (ice_status_t st = check_cache_data(c)) return st;
    if (ice_status_t st = check_table(c, n_requests, seq_len, table, max_blocks)) return st;
    if (!pos || !n_tok) return fail(ICE_ERR_INVALID_ARG, "token_pos or n_tok is null");
    CacheAttend a{};
    size_t need = 0;
    if (ice_status_t st = plan_attend(c, G, n_requests, 1, max_tok, true, a, &need)) return st;
    a.T = n_requests;
    a.seq_len = seq_len;
    a.table = table;
    a.max_blocks = max_blocks;
    a.pos = pos;
    a.n_tok = n_tok;
    return cache_attend(c, a, q, q_stride, out, out_type, lse, ws, ws_bytes, need, stream, "ice_cache_attend_tokens");
}

// ---- rows of a table that requests share

ice_status_t ice_plan_sources(int32_t n_requests, int32_t n_rows, int32_t n_tokens, const int32_t *source, const int32_t *query_start,
                              const int32_t *seq_len, int32_t *plan, void *stream) {
    if (!source || !query_start || !plan) return fail(ICE_ERR_INVALID_ARG, "source, query_start or plan is null");
    if (n_requests < 1 || n_requests > kSourceRows) return fail(ICE_ERR_SHAPE, "n_requests %d is outside [1, %d]", n_requests, kSourceRows);
    if (n_rows < 1 || n_rows > kSourceRows) return fail(ICE_ERR_SHAPE, "n_rows %d is outside [1, %d]", n_rows, kSourceRows);
    if (n_tokens < 0 || n_tokens > (1 << 30)) return fail(ICE_ERR_SHAPE, "n_tokens %d is outside [0, 2^30]", n_tokens);
    launch_plan_sources({n_requests, n_rows, n_tokens, source, query_start, seq_len, plan}, static_cast<hipStream_t>(stream));
    return device_status("ice_plan_sources");
}

ice_status_t ice_cache_append(const ice_cache_t *c, const void *q, int64_t q_stride, int32_t n_q_heads, void *q_out, int64_t q_out_stride, const void *k,
                              const void *v, int64_t k_stride, int64_t v_stride, int32_t n_tokens, int32_t n_requests, const int32_t *query_start,
                              const int32_t *seq_len, const int32_t *source, const int32_t *table, int32_t max_blocks, const float *rope,
                              int32_t n_positions, int32_t rotated, int32_t neighbours, void *stream) {
    if (ice_status_t st = check_cache_data(c)) return st;
    if (ice_status_t st = check_table(c, n_requests, seq_len, table, max_blocks)) return st;
    if (!query_start) return fail(ICE_ERR_INVALID_ARG, "query_start is null");
    if (n_tokens < 0) return fail(ICE_ERR_SHAPE, "n_tokens must be >= 0");
    if (neighbours != 0 && neighbours != 1) return fail(ICE_ERR_INVALID_ARG, "neighbours %d: 0 or 1", neighbours);
    if (rope) {
        if (!aligned16(rope)) return fail(ICE_ERR_INVALID_ARG, "rope is misaligned");
        if (n_positions < 1) return fail(ICE_ERR_SHAPE, "n_positions must be >= 1");
        if (rotated < 16 || rotated > kD || rotated % 16) return fail(ICE_ERR_UNSUPPORTED, "rotated %d: a multiple of 16, at most %d", rotated, kD);
    } else if (q) {
        return fail(ICE_ERR_INVALID_ARG, "queries without a table of rotations: nothing to do with them");
    }
    if (q && (n_q_heads < 1 || n_q_heads > 65536)) return fail(ICE_ERR_SHAPE, "n_q_heads %d is outside [1, 65536]", n_q_heads);
    if (n_tokens == 0) return ICE_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return fail(ICE_ERR_INVALID_ARG, "k or v is null or misaligned");
    if (q && (!aligned16(q) || !q_out || !aligned16(q_out))) return fail(ICE_ERR_INVALID_ARG, "q or q_out is null or misaligned");
    const int64_t row = (int64_t)c->n_kv_heads * kD, q_row = (int64_t)n_q_heads * kD;
    if ((k_stride & 7) || (v_stride & 7) || (n_tokens > 1 && (k_stride < row || v_stride < row)))
        return fail(ICE_ERR_SHAPE, "strides must be multiples of 8 and at least n_kv_heads * 128");
    if (q && ((q_stride & 7) || (q_out_stride & 7) || (n_tokens > 1 && (q_stride < q_row || q_out_stride < q_row))))
        return fail(ICE_ERR_SHAPE, "strides of q and q_out must be multiples of 8 and at least n_q_heads * 128");
    CacheAppend a{};
    a.q_heads = q ? n_q_heads : 0;
    if ((double)((n_tokens + 3ll) / 4) * (a.q_heads + 2.0 * c->n_kv_heads) > 4e7) return fail(ICE_ERR_UNSUPPORTED, "too many rows for one call");
    a.c = cache_dims(c);
    a.q = static_cast<const bf16_t *>(q);
    a.k = static_cast<const bf16_t *>(k);
    a.v = static_cast<const bf16_t *>(v);
    a.q_out = static_cast<bf16_t *>(q_out);
    a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.q_out_stride = q_out_stride;
    a.n_tokens = n_tokens, a.n_requests = n_requests, a.max_blocks = max_blocks;
    a.query_start = query_start, a.seq_len = seq_len, a.table = table, a.source = source;
    a.rope = rope, a.n_positions = n_positions, a.half = rope ? rotated / 2 : 0, a.neighbours = neighbours != 0;
    launch_cache_append(a, static_cast<hipStream_t>(stream));
    return device_status("ice_cache_append");
}

static ice_status_t check_rows(int32_t n_rows) {
    return n_rows < 1 || n_rows > kSourceRows ? fail(ICE_ERR_SHAPE, "%d rows of the table: outside [1, %d]", n_rows, kSourceRows) : ICE_OK;
}

// The row tiles that `rows` requests or sources can have between them: each those of its most queries, and all together those of n_tokens, the last ones of
// each not full.  (A most beyond n_tokens, that no step can have, counts as it is given.)  The kernels take arrays of starts that do not ascend, where
// queries would count several times, for a step without queries.
static double row_tiles(const CacheAttend &a, int most, int rows) {
    const int tile = 192 / a.G;
    const double each = rows * (double)((most + (long long)tile - 1) / tile);
    return most > a.T ? each : std::min(each, (double)(a.T / tile) + std::min(rows, a.T));
}
// (the quanta of a launch's entries are counted in 31 bits; both sides of attention behind a source lie in one launch)
static ice_status_t check_sources_count(const ice_cache_t *c, const CacheAttend &a, double tiles) {
    if (((double)a.max_blocks * c->block_size / 128 + 4) * tiles * c->n_kv_heads >= 2147483648.0)
        return fail(ICE_ERR_UNSUPPORTED, "%d rows, %d tokens x %d KV heads x %d blocks: too many for one call", a.S, a.T, c->n_kv_heads, a.max_blocks);
    return ICE_OK;
}
static ice_status_t check_shared_count(const ice_cache_t *c, const CacheAttend &a) {
    return check_sources_count(c, a, row_tiles(a, a.max_query, a.S) + row_tiles(a, a.max_shared, a.S));
}
static ice_status_t check_cross_count(const ice_cache_t *c, const CacheAttend &a) {
    return check_sources_count(c, a, row_tiles(a, a.max_query, std::min(a.S, 1024)));
}

// where a list's parts lie (ice_plan_sources)
static void set_list(CacheAttend &a, const int32_t *plan) {
    a.list_start = plan;
    a.lowest = plan + a.S + 2;
    a.token = plan + 2 * (size_t)a.S + 2;
    a.place = a.token + a.T;
}

size_t ice_cache_attend_cross_bytes(const ice_cache_t *c, int32_t G, int32_t n_rows, int32_t max_shared, int32_t max_keys) {
    CacheAttend a{};
    size_t bytes = 0;
    if (check_rows(n_rows) != ICE_OK) return 0;
    return plan_attend(c, G, n_rows, max_shared, max_keys, false, a, &bytes) == ICE_OK ? bytes : 0;
}

ice_status_t ice_cache_attend_cross(const ice_cache_t *c, const void *q, int64_t q_stride, int32_t G, int32_t n_rows, const int32_t *plan, int32_t n_tokens,
                                    int32_t max_shared, const int32_t *seq_len, int32_t max_keys, const int32_t *table, int32_t max_blocks, void *out,
                                    int32_t out_type, float *lse, void *ws, size_t ws_bytes, void *stream) {
    if (ice_status_t st = check_cache_data(c)) return st;
    if (ice_status_t st = check_rows(n_rows)) return st;
    if (ice_status_t st = check_table(c, n_rows, seq_len, table, max_blocks)) return st;
    if (!plan) return fail(ICE_ERR_INVALID_ARG, "plan is null");
    if (n_tokens < 0) return fail(ICE_ERR_SHAPE, "n_tokens must be >= 0");
    CacheAttend a{};
    size_t need = 0;
    if (ice_status_t st = plan_attend(c, G, n_rows, max_shared, max_keys, false, a, &need)) return st;
    if (n_tokens == 0) return ICE_OK;
    a.T = n_tokens;
    set_list(a, plan);
    a.query_start = plan;
    a.seq_len = seq_len;
    a.table = table;
    a.max_blocks = max_blocks;
    if (ice_status_t st = check_cross_count(c, a)) return st;
    if (ice_status_t st = set_attend(c, a, q, q_stride, out, out_type, lse, ws, ws_bytes, need)) return st;
    launch_cache_cross(a, static_cast<hipStream_t>(stream));
    return device_status("ice_cache_attend_cross");
}

static ice_status_t plan_shared(const ice_cache_t *c, int32_t G, int32_t n_requests, int32_t n_tokens, int32_t max_query, int32_t max_shared,
                                int32_t max_keys, int32_t max_source_keys, CacheAttend &a, size_t *bytes) {
    if (ice_status_t st = check_rows(n_requests)) return st;
    if (n_tokens < 0 || n_tokens > (1 << 30)) return fail(ICE_ERR_SHAPE, "n_tokens %d is outside [0, 2^30]", n_tokens);
    if (ice_status_t st = plan_attend(c, G, n_requests, max_shared, max_source_keys, false, a, bytes)) return st;  // (its checks of these two)
    if (ice_status_t st = plan_attend(c, G, n_requests, max_query, max_keys, false, a, bytes)) return st;
    if ((double)n_tokens * c->n_kv_heads > 1e7) return fail(ICE_ERR_UNSUPPORTED, "%d tokens for %d KV heads: too many for one call", n_tokens, c->n_kv_heads);
    a.T = n_tokens;
    a.max_shared = max_shared;
    a.whole = false;
    *bytes = plan_cache_shared(a, max_source_keys);
    return ICE_OK;
}

size_t ice_cache_attend_shared_bytes(const ice_cache_t *c, int32_t G, int32_t n_requests, int32_t n_tokens, int32_t max_query, int32_t max_shared,
                                     int32_t max_keys, int32_t max_source_keys) {
    CacheAttend a{};
    size_t bytes = 0;
    return plan_shared(c, G, n_requests, n_tokens, max_query, max_shared, max_keys, max_source_keys, a, &bytes) == ICE_OK ? bytes : 0;
}

ice_status_t ice_cache_attend_shared(const ice_cache_t *c, const void *q, int64_t q_stride, int32_t G, int32_t n_requests, const int32_t *query_start,
                                     const int32_t *source, const int32_t *plan, int32_t n_tokens, int32_t max_query, int32_t max_shared,
                                     const int32_t *seq_len, int32_t max_keys, int32_t max_source_keys, const int32_t *table, int32_t max_blocks,
                                     int32_t window, void *out, int32_t out_type, float *lse, void *ws, size_t ws_bytes, void *stream) {
    if (ice_status_t st = check_cache_data(c)) return st;
    if (ice_status_t st = check_rows(n_requests)) return st;
    if (ice_status_t st = check_table(c, n_requests, seq_len, table, max_blocks)) return st;
    if (!query_start || !source || !plan) return fail(ICE_ERR_INVALID_ARG, "query_start, source or plan is null");
    if (window < 0) return fail(ICE_ERR_SHAPE, "window must be >= 0 (0: no window)");
    CacheAttend a{};
    size_t need = 0;
    if (ice_status_t st = plan_shared(c, G, n_requests, n_tokens, max_query, max_shared, max_keys, max_source_keys, a, &need)) return st;
    if (n_tokens == 0) return ICE_OK;
    a.seq_len = seq_len;
    a.table = table;
    a.max_blocks = max_blocks;
    a.window = window;
    a.source = source;
    a.query_start = query_start;
    set_list(a, plan);
    if (ice_status_t st = check_shared_count(c, a)) return st;
    if (ice_status_t st = set_attend(c, a, q, q_stride, out, out_type, lse, ws, ws_bytes, need)) return st;
    launch_cache_shared(a, ws, static_cast<hipStream_t>(stream));
    return device_status("ice_cache_attend_shared");
}

ice_status_t ice_debug_shared_cut(const ice_cache_t *c, int32_t G, int32_t n_requests, const int32_t *query_start, const int32_t *plan, int32_t n_tokens,
                                  int32_t max_query, int32_t max_shared, const int32_t *seq_len, int32_t max_keys, int32_t max_source_keys, int32_t max_blocks,
                                  int32_t window, int32_t *parts, int64_t max_parts, int64_t *n_parts) {
    if (ice_status_t st = check_cache(c)) return st;
    if (!query_start || !plan || !seq_len || !parts || !n_parts) return fail(ICE_ERR_INVALID_ARG, "a pointer is null");
    if (max_blocks < 1 || (long long)max_blocks * c->block_size > (1 << 30)) return fail(ICE_ERR_SHAPE, "max_blocks %d: at least 1, at most 2^30 tokens", max_blocks);
    if (window < 0 || max_parts < 0) return fail(ICE_ERR_SHAPE, "window and max_parts must be >= 0");
    CacheAttend a{};
    size_t need = 0;
    if (ice_status_t st = plan_shared(c, G, n_requests, n_tokens, max_query, max_shared, max_keys, max_source_keys, a, &need)) return st;
    a.max_blocks = max_blocks;
    a.window = window;
    a.seq_len = seq_len;
    a.query_start = query_start;
    set_list(a, plan);
    if (ice_status_t st = check_shared_count(c, a)) return st;
    try {
        *n_parts = cut_cache_shared(a, parts, max_parts);
    } catch (...) {
        return fail(ICE_ERR_CAPACITY, "no host memory for the sums of %d requests", n_requests);
    }
    return ICE_OK;
}

ice_status_t ice_debug_cross_cut(const ice_cache_t *c, int32_t G, int32_t n_rows, const int32_t *start, int32_t n_tokens, int32_t max_shared,
                                 const int32_t *len, int32_t max_keys, int32_t max_blocks, int32_t *parts, int64_t max_parts, int64_t *n_parts) {
    if (ice_status_t st = check_cache(c)) return st;
    if (ice_status_t st = check_rows(n_rows)) return st;
    if (!start || !len || !parts || !n_parts) return fail(ICE_ERR_INVALID_ARG, "a pointer is null");
    if (max_blocks < 1 || (long long)max_blocks * c->block_size > (1 << 30)) return fail(ICE_ERR_SHAPE, "max_blocks %d: at least 1, at most 2^30 tokens", max_blocks);
    if (n_tokens < 0 || max_parts < 0) return fail(ICE_ERR_SHAPE, "n_tokens and max_parts must be >= 0");
    CacheAttend a{};
    size_t need = 0;
    if (ice_status_t st = plan_attend(c, G, n_rows, max_shared, max_keys, false, a, &need)) return st;
    a.T = n_tokens;
    a.max_blocks = max_blocks;
    if (ice_status_t st = check_cross_count(c, a)) return st;
    try {
        *n_parts = cut_cache_cross(a, start, len, parts, max_parts);
    } catch (...) {
        return fail(ICE_ERR_CAPACITY, "no host memory for the sums of %d rows", n_rows);
    }
    return ICE_OK;
}

ice_status_t ice_debug_cache_cut(const ice_cache_t *c, int32_t G, int32_t n_requests, const int32_t *query_start, int32_t n_tokens, int32_t max_query,
                                 const int32_t *len, int32_t max_keys, int32_t max_blocks, int32_t window, int32_t *parts, int64_t max_parts,
                                 int64_t *n_parts) {
    if (ice_status_t st = check_cache(c)) return st;
    if (!len || !parts || !n_parts) return fail(ICE_ERR_INVALID_ARG, "a pointer is null");
    if (max_blocks < 1 || (long long)max_blocks * c->block_size > (1 << 30)) return fail(ICE_ERR_SHAPE, "max_blocks %d: at least 1, at most 2^30 tokens", max_blocks);
    if (window < 0 || n_tokens < 0 || max_parts < 0) return fail(ICE_ERR_SHAPE, "window, n_tokens and max_parts must be >= 0");
    CacheAttend a{};
    size_t need = 0;
    if (ice_status_t st = plan_attend(c, G, n_requests, max_query, max_keys, !query_start, a, &need)) return st;
    a.T = query_start ? n_tokens : n_requests;
    a.max_blocks = max_blocks;
    a.window = window;
    if (ice_status_t st = check_count(c, a, !query_start)) return st;
    try {
        *n_parts = cut_cache_attend(a, !query_start, query_start, len, parts, max_parts);
    } catch (...) {
        return fail(ICE_ERR_CAPACITY, "no host memory for the sums of %d requests", n_requests);
    }
    return ICE_OK;
}

static ice_status_t select_hier_common(ice_index_t *ix, const void *q, int32_t budget, int32_t n_top, int32_t n_probe_top,
                                       int32_t n_probe, int32_t n_refine, int32_t *ids, int32_t *n_sel, float *scores,
                                       int32_t *clusters, int32_t *tops, float *out, void *stream, const char *who) {
    if (!q || !aligned16(q)) return fail(ICE_ERR_INVALID_ARG, "q is null or misaligned");
    if (!ids || !n_sel) return fail(ICE_ERR_INVALID_ARG, "page_ids or n_selected is null");
    if (budget < ix->dev.s) return fail(ICE_ERR_SHAPE, "token_budget %d is below page_size %d", budget, ix->dev.s);
    if (n_probe < 1) return fail(ICE_ERR_SHAPE, "n_probe must be >= 1");
    const int P = budget / ix->dev.s;
    if (n_refine != 0 && n_refine < P)
        return fail(ICE_ERR_SHAPE, "n_refine %d must be 0 (off) or at least the %d pages of the budget", n_refine, P);
    if (n_refine > ix->dev.max_pages) n_refine = ix->dev.max_pages;
    if (ix->dev.max_pages > decode_hier_max_pages(ix->dev.G))
        return fail(ICE_ERR_UNSUPPORTED, "%d pages per unit exceed the selection kernel's limit of %d", ix->dev.max_pages,
                    decode_hier_max_pages(ix->dev.G));
    if (decode_hier_lds_bytes(ix->dev, P, n_probe, n_refine) > 160u * 1024u - 6144u)
        return fail(ICE_ERR_UNSUPPORTED, "%d pages per unit, n_probe %d, n_refine %d and token_budget %d need more LDS than a CU has",
                    ix->dev.max_pages, n_probe, n_refine, budget);
    launch_decode_hier(ix->dev, static_cast<const bf16_t *>(q), ix->cur, P, n_top, n_probe_top, n_probe, n_refine,
                       ix->n_tokens / ix->dev.s + ix->dev.C, ids, n_sel, scores, clusters, tops, out, static_cast<hipStream_t>(stream));
    return device_status(who);
}

ice_status_t ice_select_hier(ice_index_t *ix, const void *q, int32_t budget, int32_t n_probe, int32_t n_refine, int32_t *ids,
                             int32_t *n_sel, float *scores, int32_t *clusters, float *out, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_select_hier before ice_build_index");
    return select_hier_common(ix, q, budget, 0, 0, n_probe, n_refine, ids, n_sel, scores, clusters, nullptr, out, stream,
                              "ice_select_hier");
}

ice_status_t ice_select_hier3(ice_index_t *ix, const void *q, int32_t budget, int32_t n_probe_top, int32_t n_probe,
                              int32_t n_refine, int32_t *ids, int32_t *n_sel, float *scores, int32_t *clusters, int32_t *tops,
                              float *out, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_select_hier3 before ice_build_index");
    if (ix->n_top == 0) return fail(ICE_ERR_STATE, "ice_select_hier3 before ice_build_top_level");
    if (n_probe_top < 1) return fail(ICE_ERR_SHAPE, "n_probe_top must be >= 1");
    return select_hier_common(ix, q, budget, ix->n_top, n_probe_top, n_probe, n_refine, ids, n_sel, scores, clusters, tops, out,
                              stream, "ice_select_hier3");
}

ice_status_t ice_build_top_level(ice_index_t *ix, int32_t n_top, int32_t iters, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_build_top_level before ice_build_index");
    if (n_top == 0) {  // (drops the level)
        ix->n_top = 0;
        return ICE_OK;
    }
    if (n_top < 1 || n_top > kTopMax || n_top > ix->dev.C)
        return fail(ICE_ERR_SHAPE, "n_top %d is outside [1, min(%d, n_clusters = %d)]", n_top, kTopMax, ix->dev.C);
    if (iters < 1) return fail(ICE_ERR_INVALID_ARG, "iters must be >= 1");
    launch_top_level(ix->dev, ix->cur, n_top, iters, static_cast<hipStream_t>(stream));
    if (ice_status_t st = device_status("ice_build_top_level")) return st;
    ix->n_top = n_top;
    return ICE_OK;
}

ice_status_t ice_export_top_level(ice_index_t *ix, ice_top_view_t *v) {
    if (!ix || !v) return fail(ICE_ERR_INVALID_ARG, "index or view is null");
    if (!ix->built || ix->n_top == 0) return fail(ICE_ERR_STATE, "ice_export_top_level before ice_build_top_level");
    memset(v, 0, sizeof(*v));
    v->n_top = ix->n_top;
    v->n_top_max = kTopMax;
    v->top_centroid = ix->dev.top_cent;
    v->top_centroid_bf16 = ix->dev.top_bf16;
    v->top_of = ix->dev.top_of;
    v->top_count = ix->dev.top_cnt;
    v->top_init = ix->dev.top_init;
    return ICE_OK;
}

ice_status_t ice_set_geometry(ice_index_t *ix, int32_t geometry) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (geometry != ICE_GEOMETRY_RAW && geometry != ICE_GEOMETRY_TRANSFORMED)
        return fail(ICE_ERR_INVALID_ARG, "geometry %d: ICE_GEOMETRY_RAW or ICE_GEOMETRY_TRANSFORMED", geometry);
    if (geometry != ix->geometry) ix->built = false;  // takes effect with the next build
    ix->geometry = geometry;
    return ICE_OK;
}

ice_status_t ice_export_geometry(ice_index_t *ix, ice_geometry_view_t *v) {
    if (!ix || !v) return fail(ICE_ERR_INVALID_ARG, "index or view is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_export_geometry before ice_build_index");
    const Dev &d = ix->dev;
    memset(v, 0, sizeof(*v));
    v->geometry = d.tk;
    if (d.tk) {
        v->key_extra = d.kaug;
        v->centroid_extra = d.cent_aug;
        v->cluster_sum_extra = d.csum_aug;
        v->radius_sq = d.c2;
        v->assign_centroid_extra_bf16 = d.caug[ix->cur ^ 1];
    }
    return ICE_OK;
}

ice_status_t ice_export_index(ice_index_t *ix, ice_index_view_t *v) {
    if (!ix || !v) return fail(ICE_ERR_INVALID_ARG, "index or view is null");
    if (!ix->built) return fail(ICE_ERR_STATE, "ice_export_index before ice_build_index");
    const Dev &d = ix->dev;
    memset(v, 0, sizeof(*v));
    v->n_units = d.U;
    v->group_size = d.G;
    v->head_dim = kD;
    v->page_size = d.s;
    v->n_clusters = d.C;
    v->cpad = d.Cpad;
    v->max_pages = d.max_pages;
    v->max_tokens = d.max_tokens;
    v->n_tokens = ix->n_tokens;
    v->Kp = d.Kp;
    v->Vp = d.Vp;
    v->page_cluster = d.page_cluster;
    v->page_fill = d.page_fill;
    v->page_pos = d.page_pos;
    v->cluster_tail = d.cluster_tail;
    v->cluster_cnt = d.cluster_cnt;
    v->cluster_sum = d.cluster_sum;
    v->centroid = d.centroid;
    v->page_sum = d.page_sum;
    v->rep = d.rep;
    v->n_pages = d.n_pages;
    v->assign = d.assign;
    v->assign_centroid_bf16 = d.cent_bf16[ix->cur ^ 1];
    v->init_idx = d.init_idx;
    return ICE_OK;
}

ice_status_t ice_import_index(ice_index_t *ix, const ice_index_view_t *v, void *stream) {
    if (!ix || !v) return fail(ICE_ERR_INVALID_ARG, "index or view is null");
    if (ice_status_t st = check_shape(v->page_size, v->n_clusters)) return st;
    if (v->n_units != ix->cfg.batch * ix->cfg.n_kv_heads || v->group_size != ix->cfg.group_size || v->head_dim != kD ||
        v->max_tokens != ix->cfg.max_tokens || v->max_pages != ix->cfg.max_tokens / v->page_size + v->n_clusters)
        return fail(ICE_ERR_SHAPE, "view dimensions do not match the index configuration");
    if (v->n_tokens < 0 || v->n_tokens > ix->cfg.max_tokens) return fail(ICE_ERR_SHAPE, "view n_tokens out of range");
    if (!v->Kp || !v->Vp || !v->page_cluster || !v->page_fill || !v->page_pos || !v->cluster_tail || !v->cluster_cnt ||
        !v->cluster_sum || !v->centroid || !v->page_sum || !v->rep || !v->n_pages)
        return fail(ICE_ERR_INVALID_ARG, "a view array is null");
    if (ice_status_t st = ensure_layout(ix, v->page_size, v->n_clusters)) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Dev &d = ix->dev;
    const size_t U = d.U, MP = d.max_pages, C = d.C, ps = d.s;
    const void *src[12] = {v->Kp, v->Vp, v->page_sum, v->rep, v->page_pos, v->cluster_sum, v->centroid, v->page_cluster, v->page_fill,
                           v->cluster_tail, v->cluster_cnt, v->n_pages};
    void *dst[12] = {d.Kp, d.Vp, d.page_sum, d.rep, d.page_pos, d.cluster_sum, d.centroid, d.page_cluster, d.page_fill,
                     d.cluster_tail, d.cluster_cnt, d.n_pages};
    const size_t bytes[12] = {U * MP * ps * kD * 2, U * MP * ps * kD * 2, U * MP * kD * 4, U * MP * kD * 2, U * MP * ps * 4, U * C * kD * 4,
                              U * C * kD * 4, U * MP * 4, U * MP * 4, U * C * 4, U * C * 4, U * 4};
    // One launch when all arrays are aligned memory of the workspace's own GPU; anything else a copy call
    // takes (another GPU's memory, pinned or managed memory, an odd address) or refuses (an array that ends
    // before its size) goes through copy calls.
    if (all_on_device(src, bytes, 12, ix->ws)) {
        launch_import(d, src, dst, bytes, *v, s);
    } else {
        for (int i = 0; i < 12; ++i) {
            const hipError_t e = hipMemcpyAsync(dst[i], src[i], bytes[i], hipMemcpyDeviceToDevice, s);
            if (e != hipSuccess) return fail(ICE_ERR_DEVICE, "ice_import_index: %s", hipGetErrorString(e));
        }
        reset_decode_state(d, v->n_tokens, s);
        launch_refresh_centroids(d, 0, s);
        launch_refresh_centroids(d, 1, s);
        launch_refresh_tails(d, s);
    }
    ix->cur = 0;
    ix->geometry = 0;  // (an imported index carries no extra coordinate)
    ix->dev.tk = 0;
    if (ice_status_t st = device_status("ice_import_index")) return st;
    ix->n_tokens = v->n_tokens;
    ix->build_n = 0;  // (not the product of a build here: no stage to re-run)
    ix->n_top = 0;
    ix->built = true;
    return ICE_OK;
}

ice_status_t ice_debug_assign(ice_index_t *ix, const void *K, int32_t n, const void *cent, int32_t n_clusters,
                              int32_t *assign_out, float *best_out, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!K || !cent || !aligned16(K) || !aligned16(cent))
        return fail(ICE_ERR_INVALID_ARG, "K or centroids is null or misaligned");
    if (n < 1) return fail(ICE_ERR_INVALID_ARG, "n must be >= 1");
    if (n > ix->cfg.max_tokens) return fail(ICE_ERR_SHAPE, "n %d exceeds max_tokens %d", n, ix->cfg.max_tokens);
    const int s_cur = ix->laid_out ? ix->dev.s : 16;
    if (ice_status_t st = check_shape(s_cur, n_clusters)) return st;
    if (ice_status_t st = ensure_layout(ix, s_cur, n_clusters)) return st;
    ix->dev.tk = 0;  // (the debug assignment is always on the raw keys)
    ix->built = false;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Dev &d = ix->dev;
    launch_load_centroids(d, static_cast<const bf16_t *>(cent), 0, s);
    launch_assign(d, static_cast<const bf16_t *>(K), n, 0, 0, false, false, s);
    if (assign_out) launch_sort(d, n, 0, best_out, assign_out, s);  // (unpacks the winners; without it only the kernel is timed)
    return device_status("ice_debug_assign");
}

ice_status_t ice_debug_rerun_stage(ice_index_t *ix, const void *K, const void *V, int32_t stage, void *stream) {
    if (!ix) return fail(ICE_ERR_INVALID_ARG, "index is null");
    if (!ix->built || ix->build_n == 0 || ix->n_tokens != ix->build_n)
        return fail(ICE_ERR_STATE, "ice_debug_rerun_stage needs an index fresh from ice_build_index (no insertion since)");
    if (!K || !V || !aligned16(K) || !aligned16(V)) return fail(ICE_ERR_INVALID_ARG, "K or V is null or misaligned");
    hipStream_t s = static_cast<hipStream_t>(stream);
    const Dev &d = ix->dev;
    const bf16_t *Kb = static_cast<const bf16_t *>(K), *Vb = static_cast<const bf16_t *>(V);
    const int n = ix->build_n, prev = ix->cur ^ 1;  // the last round read buffer `prev` and wrote the live one
    switch (stage) {
        case ICE_STAGE_ASSIGN: launch_assign(d, Kb, n, prev, 0, false, false, s); break;
        case ICE_STAGE_SORT: launch_sort(d, n, 0, nullptr, nullptr, s); break;
        case ICE_STAGE_MEANS: launch_means(d, Kb, n, prev, 0, true, s); break;
        case ICE_STAGE_PAGINATE: launch_paginate(d, Kb, Vb, n, false, s); break;
        default: return fail(ICE_ERR_INVALID_ARG, "stage %d: one of ICE_STAGE_ASSIGN .. ICE_STAGE_PAGINATE", stage);
    }
    return device_status("ice_debug_rerun_stage");
}

ice_status_t ice_debug_build_plan(const ice_config_t *cfg, int32_t n, int32_t n_clusters, int32_t plan[6]) {
    if (ice_status_t st = check_cfg(cfg)) return st;
    if (!plan) return fail(ICE_ERR_INVALID_ARG, "plan is null");
    if (ice_status_t st = check_shape(16, n_clusters)) return st;
    if (n < 1) return fail(ICE_ERR_INVALID_ARG, "n_tokens must be >= 1");
    if (n_clusters > n) return fail(ICE_ERR_SHAPE, "n_clusters %d exceeds n_tokens %d", n_clusters, n);
    if (n > cfg->max_tokens) return fail(ICE_ERR_SHAPE, "n_tokens %d exceeds max_tokens %d", n, cfg->max_tokens);
    Dev d{};
    d.U = cfg->batch * cfg->n_kv_heads;
    d.C = n_clusters;
    d.Cpad = round_up(n_clusters, 32);
    build_plan(d, n, cfg->kmeans_iters, plan);
    return ICE_OK;
}

ice_status_t ice_debug_near_bounds(int32_t n, const float *k2, const float *a2, const float *sa, const float *sb, float *need, float *dist2) {
    if (n < 0) return fail(ICE_ERR_INVALID_ARG, "n must not be negative");
    if (!k2 || !a2 || !sa || !sb || !need || !dist2) return fail(ICE_ERR_INVALID_ARG, "a pointer is null");
    near_bounds(n, k2, a2, sa, sb, need, dist2);
    return ICE_OK;
}

ice_status_t ice_debug_select_fault(ice_index_t *ix, const void *q, int32_t budget, int32_t *ids, int32_t *n_sel, float *out,
                                    int32_t muted_chunk, int32_t wait_log2, void *stream) {
    if (ice_status_t st = check_select(ix, q, budget, ids, n_sel, "ice_debug_select_fault")) return st;
    const int np_hint = ix->n_tokens / ix->dev.s + ix->dev.C;
    const int chunks = decode_step_chunks(ix->dev, np_hint);
    if (chunks < 2) return fail(ICE_ERR_UNSUPPORTED, "this index is served by one workgroup per unit: there is no score hand-off to disturb");
    if (muted_chunk < 0 || muted_chunk >= chunks) return fail(ICE_ERR_SHAPE, "muted_chunk %d is outside [0, %d)", muted_chunk, chunks);
    if (wait_log2 < 0 || wait_log2 > 20) return fail(ICE_ERR_SHAPE, "wait_log2 %d is outside [0, 20]", wait_log2);
    launch_decode_step(ix->dev, static_cast<const bf16_t *>(q), budget / ix->dev.s, np_hint, ids, n_sel, nullptr, nullptr, nullptr, 0,
                       out, static_cast<hipStream_t>(stream), wait_log2 | ((muted_chunk + 1) << 8));
    return device_status("ice_debug_select_fault");
}

}  // extern "C"
