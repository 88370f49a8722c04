// Internal declarations of the steps around a paged cache: what the host dispatcher hands to their kernels.
// Nothing here is part of the public ABI (include/snapkv.h).
#ifndef SNAPKV_SERVE_H_
#define SNAPKV_SERVE_H_

#include "snapkv_internal.h"

namespace snapkv {

// Appending tokens to a paged cache (snapkv_append.hip); strides in bytes.
struct AppendArgs {
    const char *q, *k, *v;                           // q: null with Hq = 0 (no queries)
    int64_t q_rs, q_hs, k_rs, k_hs, v_rs, v_hs;
    char *q_out, *k_out;                             // k_out: may be null
    int64_t qo_rs, qo_hs, ko_rs, ko_hs;
    char *k_pages, *v_pages;                         // [pages, page, Hkv, D]
    const int32_t* table;                            // [B, table_stride]
    int64_t table_stride, table_rows, pages;         // table_rows: rows that a sequence's table columns hold
    const int32_t *starts, *cu, *positions;          // [B]; [B + 1] or null: one token per sequence; [T] or null: the rows
    const float *cos, *sin;                          // [npos, rot / 2]
    int64_t npos, T;
    int B, Hq, Hkv, page, rot;
    int parts;                                       // waves that share a token's heads
};
hipError_t launch_append(int dtype, int D, bool interleaved, AppendArgs A, hipStream_t st);

// Causal attention over packed prompts (snapkv_prompt.hip); strides in bytes.
struct PromptArgs {
    const char *q, *k, *v;
    int64_t q_rs, q_hs, k_rs, k_hs, v_rs, v_hs;
    char* out;                                       // [T, Hq, D]
    float* lse;                                      // [Hq, T] or null
    const int32_t* cu;                               // [B + 1]
    int64_t T;
    int B, Hq, Hkv, g;
    int ranks;                                       // row tiles that a head can have
    float scale2;                                    // log2(e) / sqrt(D)
};
hipError_t launch_prompt(int dtype, int D, PromptArgs A, hipStream_t st);

// One new token per sequence over a paged cache (snapkv_paged.hip).
struct PagedArgs {
    const char *q, *k, *v;                           // [B, Hq, D]; pages [pages, page, Hkv, D]
    const int32_t *table, *lens;                     // [B, table_stride]; [B]
    int64_t table_stride, pages, max_len;
    int B, Hq, Hkv, g, page;
    int nchunk, least;                               // shares that a sequence's keys can have; keys of the shortest
    int places;                                      // of workgroups, per sequence and KV head
    bool by_xcd;                                     // how workgroups are dealt out
    unsigned page_magic;                             // r / page = r * page_magic >> page_shift, r < 2^31
    int page_shift;
    float scale2;
    char* out;                                       // [B, Hq, D]
    float* lse;                                      // [B, Hq] or null
    float* part_acc;                                 // [B, Hq, nchunk, D]
    float2* part_ml;                                 // [B, Hq, nchunk]
};
struct PagedPlan {
    int nchunk, least;
    size_t bytes;                                    // of workspace
};
PagedPlan paged_plan(int B, int Hq, int Hkv, int D, int64_t max_len);
hipError_t launch_paged(int dtype, int D, PagedArgs A, void* workspace, hipStream_t st);

}  // namespace snapkv

#endif
