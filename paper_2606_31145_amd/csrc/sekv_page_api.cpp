// C ABI of the paged token store: host checks and launches.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>

#include "sekv.h"
#include "sekv_host.h"
#include "sekv_internal.h"
#include "sekv_page_index.h"
#include "sekv_page_internal.h"

namespace {

using sekv::fail;

bool misaligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

// The checks that the three calls share; *go is false when there is nothing to do.
sekv_status check_call(const sekv_page_dims *d, const sekv_pages *p, void *ws, size_t ws_bytes,
                       size_t need, bool empty, bool *go) {
    *go = false;
    sekv_status st = sekv::check_page_dims(d);
    if (st != SEKV_OK) return st;
    if (d->batch == 0 || empty) return SEKV_OK;
    st = sekv::check_pages(d, p);
    if (st != SEKV_OK) return st;
    if (!ws) return fail(SEKV_ERR_WORKSPACE, "workspace is NULL");
    if (misaligned(ws, 256)) return fail(SEKV_ERR_WORKSPACE, "workspace not 256-byte aligned");
    if (ws_bytes < need) return fail(SEKV_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, need);
    *go = true;
    return SEKV_OK;
}

// Consecutive tokens `stride` elements apart, each `heads` rows of d.
sekv_status check_rows(const sekv_page_dims *d, const void *p, int64_t stride, int heads, const char *name) {
    const int e = sekv::elem_bytes(d->dtype);
    if (!p) return fail(SEKV_ERR_INVALID_ARG, "%s is NULL", name);
    if (misaligned(p, 16)) return fail(SEKV_ERR_INVALID_ARG, "%s not 16-byte aligned", name);
    if (stride < int64_t(heads) * d->head_dim || stride % (16 / e))
        return fail(SEKV_ERR_INVALID_ARG, "%s: a token stride of %lld elements (at least %d, in 16-byte steps)", name,
                    (long long)stride, heads * d->head_dim);
    return SEKV_OK;
}

sekv::PageTables tables(const sekv_page_dims *d, const sekv_pages *p, const int32_t *tok_start, int n_tokens,
                        void *ws) {
    sekv::PageTables t{};
    t.table = p->table;
    t.seq_len = p->seq_len;
    t.tok_start = tok_start;
    t.error = &static_cast<sekv::WsHeader *>(ws)->error;
    t.B = d->batch;
    t.Hkv = d->n_kv_heads;
    t.n_pages = d->n_pages;
    t.max_pages = d->max_pages;
    t.page_shift = log2_of(d->page_size);
    t.n_tokens = n_tokens;
    return t;
}

// Work items aimed at: two workgroups a compute unit, two rounds of them, so that ragged chunks even out.
// A workgroup without an item still has to be started and to find that out.  Measured (us) with 512, 1024
// and 2048: one token of 8 sequences at 9000 in 8 bits 30.6, 30.5, 34.0; six of 16 under a window 30.8,
// 30.9, 32.8; one of 32 ragged sequences of up to 32768 in bfloat16 511, 465, 453; one of 5 of up to 131072
// in 8 bits 218, 188, 191; 9 ragged ones, one of 300 tokens, 467, 425, 434.
constexpr int kItems = 1024;

sekv::page::Launch plan(const sekv_page_dims *d, int n_tokens) {
    return sekv::page::plan_launch(d->batch, n_tokens, d->n_kv_heads, log2_of(d->n_q_heads / d->n_kv_heads),
                                   int64_t(d->max_pages) * d->page_size, kItems);
}

// The header, the counters, then the partials of split tiles.
size_t workspace_bytes(const sekv_page_dims *d, int32_t n_tokens) {
    const int64_t rows = sekv::page::partial_rows(n_tokens, d->n_kv_heads, log2_of(d->n_q_heads / d->n_kv_heads),
                                                  int64_t(d->max_pages) * d->page_size, kItems);
    return sizeof(sekv::WsHeader) + sekv::page::kCounters * sizeof(uint32_t) + size_t(rows) * (d->head_dim + 2) * sizeof(float);
}

}  // namespace

extern "C" {

sekv_status sekv_check_page_dims(const sekv_page_dims *dims) { return sekv::check_page_dims(dims); }

size_t sekv_page_workspace_size(const sekv_page_dims *dims, int32_t n_tokens) {
    if (sekv::check_page_dims(dims) != SEKV_OK) return 0;
    if (n_tokens < 0) {
        fail(SEKV_ERR_INVALID_ARG, "n_tokens < 0");
        return 0;
    }
    return workspace_bytes(dims, n_tokens);
}

sekv_status sekv_page_append(const sekv_page_dims *dims, const sekv_pages *pages, const void *k, const void *v,
                             int64_t k_stride, int64_t v_stride, const int32_t *tok_start, int32_t n_tokens,
                             void *ws, size_t ws_bytes, hipStream_t stream) {
    if (n_tokens < 0) return fail(SEKV_ERR_INVALID_ARG, "n_tokens < 0");
    bool go = false;
    sekv_status st = check_call(dims, pages, ws, ws_bytes, sizeof(sekv::WsHeader), n_tokens == 0, &go);
    if (st != SEKV_OK || !go) return st;
    if (!tok_start || misaligned(tok_start, 4))
        return fail(SEKV_ERR_INVALID_ARG, "tok_start is NULL or not 4-byte aligned");
    if ((st = check_rows(dims, k, k_stride, dims->n_kv_heads, "k")) != SEKV_OK) return st;
    if ((st = check_rows(dims, v, v_stride, dims->n_kv_heads, "v")) != SEKV_OK) return st;
    if (int64_t(n_tokens) * dims->n_kv_heads > 0x7fffffffll)
        return fail(SEKV_ERR_UNSUPPORTED, "%d new tokens of %d heads in one call", n_tokens, dims->n_kv_heads);
    sekv::PageAppendArgs a{};
    a.t = tables(dims, pages, tok_start, n_tokens, ws);
    a.src[0] = k; a.src[1] = v;
    a.stride[0] = k_stride; a.stride[1] = v_stride;
    a.pool[0] = pages->k; a.pool[1] = pages->v;
    a.scale[0] = pages->k_scale; a.scale[1] = pages->v_scale;
    const hipError_t e = sekv::launch_page_append(a, dims->dtype, dims->page_dtype, dims->head_dim, stream);
    if (e != hipSuccess) return fail(SEKV_ERR_HIP, "page append launch: %s", hipGetErrorString(e));
    return SEKV_OK;
}

sekv_status sekv_page_read(const sekv_page_dims *dims, const sekv_pages *pages, void *keys, void *values,
                           int32_t max_tokens, void *ws, size_t ws_bytes, hipStream_t stream) {
    if (max_tokens < 0) return fail(SEKV_ERR_INVALID_ARG, "max_tokens < 0");
    bool go = false;
    sekv_status st = check_call(dims, pages, ws, ws_bytes, sizeof(sekv::WsHeader), max_tokens == 0, &go);
    if (st != SEKV_OK || !go) return st;
    if (!keys || !values) return fail(SEKV_ERR_INVALID_ARG, "keys or values is NULL");
    if (misaligned(keys, 16) || misaligned(values, 16))
        return fail(SEKV_ERR_INVALID_ARG, "keys or values not 16-byte aligned");
    sekv::PageReadArgs a{};
    a.t = tables(dims, pages, nullptr, 0, ws);
    a.pool[0] = pages->k; a.pool[1] = pages->v;
    a.scale[0] = pages->k_scale; a.scale[1] = pages->v_scale;
    a.dst[0] = keys; a.dst[1] = values;
    a.max_tokens = max_tokens;
    const hipError_t e = sekv::launch_page_read(a, dims->dtype, dims->page_dtype, dims->head_dim, stream);
    if (e != hipSuccess) return fail(SEKV_ERR_HIP, "page read launch: %s", hipGetErrorString(e));
    return SEKV_OK;
}

sekv_status sekv_page_attend(const sekv_page_dims *dims, const sekv_pages *pages, const void *q, int64_t q_stride,
                             const int32_t *tok_start, int32_t n_tokens, void *out, float *lse, void *ws,
                             size_t ws_bytes, hipStream_t stream) {
    if (n_tokens < 0) return fail(SEKV_ERR_INVALID_ARG, "n_tokens < 0");
    bool go = false;
    sekv_status st = check_call(dims, pages, ws, ws_bytes, sizeof(sekv::WsHeader), n_tokens == 0, &go);
    if (st != SEKV_OK || !go) return st;
    if (!tok_start || misaligned(tok_start, 4))
        return fail(SEKV_ERR_INVALID_ARG, "tok_start is NULL or not 4-byte aligned");
    if ((st = check_rows(dims, q, q_stride, dims->n_q_heads, "q")) != SEKV_OK) return st;
    if (!out || misaligned(out, 16)) return fail(SEKV_ERR_INVALID_ARG, "out is NULL or not 16-byte aligned");
    if (misaligned(lse, 4)) return fail(SEKV_ERR_INVALID_ARG, "lse not 4-byte aligned");
    if (int64_t(n_tokens) * dims->n_q_heads > 0x7fffffffll)
        return fail(SEKV_ERR_UNSUPPORTED, "%d new tokens of %d heads in one call", n_tokens, dims->n_q_heads);
    if (ws_bytes < workspace_bytes(dims, n_tokens))
        return fail(SEKV_ERR_WORKSPACE, "workspace %zu bytes < %zu needed", ws_bytes, workspace_bytes(dims, n_tokens));
    sekv::PageAttendArgs a{};
    a.t = tables(dims, pages, tok_start, n_tokens, ws);
    a.q = q; a.q_stride = q_stride;
    a.k = pages->k; a.v = pages->v;
    a.k_scale = pages->k_scale; a.v_scale = pages->v_scale;
    a.out = out; a.lse = lse;
    a.group_shift = log2_of(dims->n_q_heads / dims->n_kv_heads);
    a.window = dims->window > 0 ? dims->window : 0x7fffffff;
    a.scale_log2 = float(dims->softmax_scale * 1.4426950408889634074);
    const sekv::page::Launch l = plan(dims, n_tokens);
    a.splits = l.splits; a.target = l.target; a.tiles = l.tiles; a.pairs = l.pairs;
    a.join_launch = sekv::page::join_in_launch(dims->batch, n_tokens, a.group_shift);
    a.arrived = reinterpret_cast<uint32_t *>(static_cast<unsigned char *>(ws) + sizeof(sekv::WsHeader));
    a.part_o = reinterpret_cast<float *>(a.arrived + sekv::page::kCounters);
    a.part_ml = a.part_o + size_t(l.splits) * n_tokens * dims->n_q_heads * dims->head_dim;
    if (sekv::page::blocks_of(l.pairs, dims->n_kv_heads) > (int64_t(1) << 23))
        return fail(SEKV_ERR_UNSUPPORTED, "%d new tokens of %d heads in one call", n_tokens, dims->n_q_heads);
    hipError_t e = l.splits > 1 ? sekv::ws_prepare_pages(ws, ws_bytes, sekv::page::kCounters, stream) : hipSuccess;
    if (e != hipSuccess) return fail(SEKV_ERR_HIP, "workspace zero kernel: %s", hipGetErrorString(e));
    e = sekv::launch_page_attend(a, dims->dtype, dims->page_dtype, dims->head_dim, stream);
    if (e != hipSuccess) return fail(SEKV_ERR_HIP, "page attention launch: %s", hipGetErrorString(e));
    return SEKV_OK;
}

}  // extern "C"
