// Launch structures of the paged token store (sekv_page.hip, sekv_page_attend_inst.hip,
// sekv_page_api.cpp).
#pragma once

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#include "sekv.h"

namespace sekv {

// Device error bit of the page calls (beside those of sekv_internal.h): a page outside the
// pool, or a token outside its sequence's pages.
constexpr int32_t kErrPageRange = 8;

// Sequences of a paged store: sekv_page_append keeps their token offsets in LDS.
constexpr int kMaxPageBatch = 4096;

// The tables that every page call reads.
struct PageTables {
    const int32_t *table;      // [B][max_pages]
    const int32_t *seq_len;    // [B]
    const int32_t *tok_start;  // [B + 1] (null in a read)
    int32_t *error;            // workspace error word
    int32_t B, Hkv, n_pages, max_pages, page_shift, n_tokens;
};

struct PageAppendArgs {
    PageTables t;
    const void *src[2];        // keys, values: [n_tokens][Hkv][d], token strides below
    int64_t stride[2];         // elements
    void *pool[2];
    uint8_t *scale[2];
};

// Rows turned by their positions: queries to q_out, and for a paged store keys, with values as they are, into the pools.
struct RotaryArgs {
    PageTables t;              // n_tokens; the rest for a paged store
    const int32_t *positions;  // [n_tokens], or null: a token's own in its sequence
    const double *freq;        // [rot_dim / 2]
    double scale;
    int32_t rot_dim, transpose;
    int32_t Hq;                // 0: no queries
    const void *q;             // [n_tokens][Hq][d]
    int64_t q_stride;
    void *q_out;
    int64_t out_stride;
    PageAppendArgs kv;         // a paged store's; its t is not read
    int32_t kv_chunks, kv_per, q_chunks, q_per;      // a token's heads in chunks of so many (queries: of rows side by side)
    int64_t kv_items, q_items; // a wave's work each, the keys first
};

struct PageReadArgs {
    PageTables t;
    const void *pool[2];
    const uint8_t *scale[2];
    void *dst[2];              // [B][Hkv][max_tokens][d]
    int32_t max_tokens;
};

struct PageAttendArgs {
    PageTables t;
    const void *q;             // [n_tokens][Hq][d], tokens q_stride elements apart
    int64_t q_stride;
    const void *k, *v;
    const uint8_t *k_scale, *v_scale;
    void *out;                 // [n_tokens][Hq][d]
    float *lse;                // [n_tokens][Hq] or null
    int32_t group_shift;       // log2(Hq / Hkv)
    int32_t window;            // > 0; 2^31 - 1: none
    int32_t splits, target;    // see sekv_page_index.h
    int64_t tiles, pairs;
    float scale_log2;          // softmax_scale * log2(e)
    int32_t join_launch;       // partials are joined by a second kernel, not by a tile's last workgroup
    uint32_t *arrived;         // [n_tokens][Hkv] by a tile's first token: its chunks that are done; zero between calls
    float *part_o;             // [splits][n_tokens][Hq][d]
    float *part_ml;            // [splits][n_tokens][Hq][2]: maximum (base 2), sum
};

// sekv_api.cpp: a page call with `words` counters behind the header is about to run on this workspace;
// they are zeroed on the stream unless the last call there left them so.
hipError_t ws_prepare_pages(void *ws, size_t bytes, size_t words, hipStream_t stream);

hipError_t launch_zero_words(void *p, size_t words, hipStream_t stream);
hipError_t launch_page_append(const PageAppendArgs &a, int dtype, int page_dtype, int head_dim, hipStream_t stream);
// page_dtype -1: no pages
hipError_t launch_rotary(RotaryArgs a, int layout, int dtype, int page_dtype, int head_dim, hipStream_t stream);
hipError_t launch_page_read(const PageReadArgs &a, int dtype, int page_dtype, int head_dim, hipStream_t stream);
hipError_t launch_page_attend(const PageAttendArgs &a, int dtype, int page_dtype, int head_dim, hipStream_t stream);

}  // namespace sekv
