// Paged key/value cache: arguments of its kernels.
#pragma once
#include "sa_internal.h"

namespace sa {

struct AppendArgs {
    const void* q;              // NULL: none
    void* q_out;
    const void* k;
    void* k_out;                // NULL: rotated keys go to the cache alone
    const void* v;
    const int32_t* pos;         // NULL: nothing is rotated
    const int32_t* slot;
    void* k_cache;
    void* v_cache;
    int rows, H, H_kv, d, page_size;
    int wg_rows;                // rows a workgroup
    int64_t n_slots;
    int64_t stride_h, stride_s, kv_stride_h, kv_stride_s, stride_page, stride_slot, stride_head;
    double log2_base;
};
hipError_t launch_cache_append(const AppendArgs& a, int dtype, hipStream_t st);

struct DecodeArgs {
    const void* q;
    const void* k_cache;
    const void* v_cache;
    const int32_t* table;
    const int32_t* lens;
    void* out;
    float* lse;                 // NULL: not wanted
    float* parts;               // workspace
    int B, H, H_kv, d, n_pages, page_size, max_pages;
    int64_t stride_b, stride_h, stat_stride_b, table_stride, stride_page, stride_slot, stride_head;
    float scale;
    int n_wgs;                  // workgroups of the launch
};
// The same under a window: a separate structure, which the plain kernels know nothing of.
struct WindowDecodeArgs : DecodeArgs {
    int window, sinks;
};
hipError_t launch_window_decode(const WindowDecodeArgs& a, int dtype, hipStream_t st);
int64_t decode_workspace(int H, int H_kv, int d);
hipError_t launch_decode(const DecodeArgs& a, int dtype, hipStream_t st);

struct TreeArgs {
    const void* q;
    const void* k_cache;
    const void* v_cache;
    const int32_t* table;
    const int32_t* lens;        // tokens in front of the draft
    const int32_t* drafts;      // drafted tokens; NULL: T each
    const int64_t* seen;
    void* out;
    float* lse;                 // NULL: not wanted
    float* parts;               // workspace
    int B, T, H, H_kv, d, n_pages, page_size, max_pages;
    int64_t stride_b, stride_t, stride_h, stat_stride_b, stat_stride_t, table_stride, seen_stride, stride_page, stride_slot, stride_head;
    float scale;
    int n_wgs;                  // workgroups of the launch
};
int64_t tree_workspace(int rows, int d, int dtype);         // rows: T H / H_kv
hipError_t launch_tree(const TreeArgs& a, int dtype, hipStream_t st);

// Whole pages, or their first tokens, onto others
struct CopyArgs {
    void* k_cache;
    void* v_cache;
    const int32_t* from;
    const int32_t* to;
    const int32_t* tokens;      // NULL: all of the page
    int n, H_kv, d, n_pages, page_size;
    int64_t stride_page, stride_slot, stride_head;
};
hipError_t launch_cache_copy(const CopyArgs& a, int dtype, hipStream_t st);

// The accepted tokens of drafts moved up
struct AcceptArgs {
    void* k_cache;
    void* v_cache;
    const int32_t* table;
    const int32_t* lens;
    const int32_t* chosen;
    const int32_t* accepted;
    int32_t* lens_after;        // NULL: not wanted
    int B, T, H_kv, d, n_pages, page_size, max_pages;
    int64_t table_stride, chosen_stride, stride_page, stride_slot, stride_head;
};
hipError_t launch_cache_accept(const AcceptArgs& a, int dtype, hipStream_t st);

}  // namespace sa
