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
int64_t decode_workspace(int H, int H_kv, int d);
hipError_t launch_decode(const DecodeArgs& a, int dtype, hipStream_t st);

}  // namespace sa
