// C ABI of libstriped_attn: argument validation, mask classification, dispatch to
// the kernels, and the single-GPU ring drivers (Algorithm 1 played in sequence).
#include <math.h>

#include <algorithm>
#include <vector>

#include "packed.h"
#include "window.h"
#include "paged.h"
#include "sa_internal.h"

namespace {

using sa::StepArgs;

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int64_t row_stride(const sa_shape* s) { return s->stride_s > 0 ? s->stride_s : s->d; }

// strides of one [B, heads, rows, d]-like tensor family
struct Geom { int heads; int64_t sb, sh, ss; };
inline Geom q_geom(const sa_shape* s) { return {s->H, s->stride_b, s->stride_h, row_stride(s)}; }
inline bool grouped(const sa_shape* s) { return s->H_kv > 0; }
inline Geom kv_geom(const sa_shape* s) {
    if (!grouped(s)) return q_geom(s);
    return {s->H_kv, s->kv_stride_b, s->kv_stride_h, s->kv_stride_s > 0 ? s->kv_stride_s : s->d};
}

// rows rows per (batch, head) must not overlap each other
int check_geom(const Geom& g, int B, int64_t rows, int d) {
    const int dmul = 4;      // rows are read four elements at a time (16 or 8 bytes)
    if (g.ss < d) return SA_ERR_SHAPE;
    // heads apart ([B, H, rows, d]-like) or interleaved within a row step ([B, rows, H, d]-like)
    const bool heads_apart = g.sh >= rows * g.ss;
    const bool heads_inside = g.sh >= d && g.ss >= (int64_t)g.heads * g.sh;
    if (!heads_apart && !heads_inside) return SA_ERR_SHAPE;
    if (B > 1 && g.sb < (heads_apart ? g.sh : rows * g.ss)) return SA_ERR_SHAPE;
    if (g.sb % dmul || g.sh % dmul || g.ss % dmul) return SA_ERR_ALIGN;
    return SA_OK;
}

int check_shape(const sa_shape* s) {
    if (!s) return SA_ERR_NULL;
    if (s->dtype != SA_F32 && s->dtype != SA_BF16) return SA_ERR_DTYPE;
    if (s->B < 1 || s->H < 1 || s->c < 1 || s->d < 1 || s->d > 256) return SA_ERR_SHAPE;
    if ((int64_t)s->B * s->H > 65535) return SA_ERR_SHAPE;
    if (s->d % 4) return SA_ERR_SHAPE;
    if (s->H_kv < 0 || (grouped(s) && s->H % s->H_kv)) return SA_ERR_SHAPE;
    if (s->stat_stride_h < s->c || (s->B > 1 && s->stat_stride_b < s->stat_stride_h)) return SA_ERR_SHAPE;
    if (int e = check_geom(q_geom(s), s->B, s->c, s->d)) return e;
    if (grouped(s))
        if (int e = check_geom(kv_geom(s), s->B, s->c, s->d)) return e;
    return SA_OK;
}

// the ring drivers address N shards of c rows inside the same tensors
int check_ring_extent(const sa_shape* s, int N) {
    const int64_t rows = (int64_t)N * s->c;
    if (s->stat_stride_h < rows) return SA_ERR_SHAPE;
    if (check_geom(q_geom(s), s->B, rows, s->d) || check_geom(kv_geom(s), s->B, rows, s->d))
        return SA_ERR_SHAPE;
    return SA_OK;
}

int check_step(int q_dev, int kv_dev, int N, int layout) {
    if (N < 1 || q_dev < 0 || q_dev >= N || kv_dev < 0 || kv_dev >= N) return SA_ERR_DEV;
    if (layout != SA_CONTIGUOUS && layout != SA_STRIPED) return SA_ERR_LAYOUT;
    return SA_OK;
}

// the block of query device q_dev and key device kv_dev
StepArgs make_args(const sa_shape* s, int q_dev = 0, int kv_dev = 0, int layout = SA_STRIPED) {
    StepArgs a{};
    a.layout = layout; a.q_dev = q_dev; a.n_q = 1; a.kv_dev = kv_dev; a.n_kv = 1;
    a.B = s->B; a.H = s->H; a.c = s->c; a.d = s->d;
    a.stride_b = s->stride_b; a.stride_h = s->stride_h;
    a.stat_stride_b = s->stat_stride_b; a.stat_stride_h = s->stat_stride_h;
    a.stride_s = row_stride(s);
    const Geom kv = kv_geom(s);
    a.H_kv = kv.heads; a.kv_stride_b = kv.sb; a.kv_stride_h = kv.sh; a.kv_stride_s = kv.ss;
    a.scale = s->softmax_scale > 0.f ? s->softmax_scale : 1.0f / sqrtf((float)s->d);
    return a;
}

int permute_common(const void* src, void* dst, int64_t outer, int64_t n_seq, int64_t inner_bytes,
                   int N, bool inverse, void* stream) {
    if (N < 1) return SA_ERR_DEV;
    if (outer < 0 || n_seq < 0 || inner_bytes < 1 || n_seq % N) return SA_ERR_SHAPE;
    if (outer == 0 || n_seq == 0) return SA_OK;   // empty: nothing to move, pointers may be NULL
    if (!src || !dst) return SA_ERR_NULL;
    if (src == dst) return SA_ERR_LAYOUT;
    int64_t al = 16;
    while (inner_bytes % al) al >>= 1;
    if ((reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst)) & (uintptr_t)(al - 1))
        return SA_ERR_ALIGN;
    return sa::launch_permute(src, dst, outer, n_seq, inner_bytes, N, inverse, (hipStream_t)stream) ==
                   hipSuccess ? SA_OK : SA_ERR_HIP;
}

// Emulated tile-skipping granularity (Sec. 3.1): both 0 (the kernels' own), or multiples of
// 128 dividing c on a shape the MFMA kernels take.
int check_skip(const sa_shape* s, int bq, int bk) {
    if (bq == 0 && bk == 0) return SA_OK;
    if (bq < 128 || bk < 128 || bq % 128 || bk % 128 || s->c % bq || s->c % bk) return SA_ERR_SHAPE;
    StepArgs a = make_args(s);
    return sa::fwd_mfma_supported(a, s->dtype) && sa::bwd_mfma_supported(a, s->dtype) ? SA_OK
                                                                                      : SA_ERR_SHAPE;
}

size_t elt_size(int dtype) { return dtype == SA_F32 ? 4 : 2; }

// HIP takes fewer than 2^32 threads a launch.  The kernels' grids are one-dimensional; at worst they
// hold one workgroup of 256 threads per 32 rows of each side (as many at d > 128, where a key-owning
// workgroup has 64 rows and half of the columns; the bf16 forward workgroups of 512 threads, on blocks of fewer
// than 128 rows or launches of a few workgroups, count as two; the fp32 ones of 512 threads per 32 rows are taken
// only where their launch fits: f32x3_split_supported).
constexpr int64_t kMostWorkgroups = (int64_t(1) << 24) - 1;
int64_t workgroups_per_kv_head(const StepArgs& a) {
    return ((int64_t)a.c / 32 + 2) * ((int64_t)a.n_q * (a.H / a.H_kv) * (a.c < 128 ? 2 : 1) + a.n_kv);
}
// Blocks of a launch that may hold more are played in parts of whole key/value heads and their groups.
template <typename Launch>
hipError_t in_parts(const StepArgs& a, int dtype, Launch launch) {
    const int64_t fit = std::max<int64_t>(1, kMostWorkgroups / workgroups_per_kv_head(a));
    if ((int64_t)a.B * a.H_kv <= fit) return launch(a);
    const int heads = (int)std::min<int64_t>(fit, a.H_kv), batches = (int)std::max<int64_t>(1, fit / a.H_kv);
    const int group = a.H / a.H_kv;
    const int64_t es = (int64_t)elt_size(dtype);
    for (int b = 0; b < a.B; b += batches)
        for (int h = 0; h < a.H_kv; h += heads) {
            StepArgs part = a;
            part.B = std::min(batches, a.B - b);
            part.H_kv = std::min(heads, a.H_kv - h);
            part.H = part.H_kv * group;
            const int64_t q = b * a.stride_b + (int64_t)h * group * a.stride_h, kv = b * a.kv_stride_b + h * a.kv_stride_h;
            const int64_t stat = b * a.stat_stride_b + (int64_t)h * group * a.stat_stride_h;
            auto in = [&](const void* p, int64_t at) -> const void* { return p ? (const char*)p + at * es : nullptr; };
            part.q = in(a.q, q); part.dout = in(a.dout, q); part.k = in(a.k, kv); part.v = in(a.v, kv);
            if (a.o) part.o = a.o + q;
            if (a.dq) part.dq = a.dq + q;
            if (a.dk) part.dk = a.dk + kv;
            if (a.dv) part.dv = a.dv + kv;
            part.lse = a.lse + stat;
            if (a.delta) part.delta = a.delta + stat;
            if (a.q_pos) part.q_pos = a.q_pos + b * a.pos_stride_b;
            if (hipError_t e = launch(part)) return e;
        }
    return hipSuccess;
}

hipError_t launch_fwd(const StepArgs& all, int dtype, hipStream_t st) {
    return in_parts(all, dtype, [&](const StepArgs& a) {
        if (!sa::fwd_mfma_supported(a, dtype)) return sa::launch_fwd_f32(a, dtype, st);
        return sa::fwd_split_wanted(a) ? sa::launch_fwd_split(a, st) : sa::launch_fwd_mfma(a, st);
    });
}
hipError_t launch_bwd(const StepArgs& all, int dtype, hipStream_t st) {
    return in_parts(all, dtype, [&](const StepArgs& a) {
        if (!sa::bwd_mfma_supported(a, dtype)) return sa::launch_bwd_f32(a, dtype, st);
        return sa::bwd_split_wanted(a) ? sa::launch_bwd_split(a, st) : sa::launch_bwd_mfma(a, st);
    });
}

int step_fwd(const void* q, const void* k, const void* v, float* o, float* lse, int q_dev, int kv_dev,
             int layout, const sa_shape* s, int bq, int bk, hipStream_t st, const int32_t* q_pos = nullptr,
             int64_t pos_stride_b = 0, float rope_base = 0.f) {
    StepArgs a = make_args(s, q_dev, kv_dev, layout);
    a.q = q; a.k = k; a.v = v; a.o = o; a.lse = lse;
    a.skip_bq = bq; a.skip_bk = bk;
    if (q_pos) {
        if (!sa::fwd_mfma_rope_supported(a, s->dtype)) return SA_ERR_SHAPE;
        a.q_pos = q_pos; a.pos_stride_b = pos_stride_b; a.rope_log2_base = log2((double)rope_base);
    }
    if (sa::block_kind(q_dev, kv_dev, layout) == sa::MASK_EMPTY) return SA_OK;   // nothing to launch
    return launch_fwd(a, s->dtype, st) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int step_bwd(const void* q, const void* k, const void* v, const void* dout, const float* lse,
             const float* delta, float* dq, float* dk, float* dv, int q_dev, int kv_dev, int layout,
             const sa_shape* s, int bq, int bk, hipStream_t st) {
    StepArgs a = make_args(s, q_dev, kv_dev, layout);
    if (sa::block_kind(q_dev, kv_dev, layout) == sa::MASK_EMPTY) return SA_OK;
    a.skip_bq = bq; a.skip_bk = bk;
    a.q = q; a.k = k; a.v = v; a.dout = dout; a.lse = const_cast<float*>(lse); a.delta = delta;
    a.dq = dq; a.dk = dk; a.dv = dv;
    return launch_bwd(a, s->dtype, st) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

// The ring drivers without per-step timings: one launch per kernel for all blocks of the played
// devices, where rows are numbered in 31 bits and a key/value head's blocks fit a launch.  Else,
// and when the caller wants each step's time, one launch per block and kernel.
bool one_launch(const StepArgs& a, int N) {
    return (int64_t)N * a.c < (int64_t(1) << 31) && workgroups_per_kv_head(a) <= kMostWorkgroups;
}

// ---- packed sequences
int check_packed(const sa_packed* s) {
    if (!s) return SA_ERR_NULL;
    if (s->dtype != SA_F32 && s->dtype != SA_BF16) return SA_ERR_DTYPE;
    if (s->n_seq < 0 || s->rows < 0 || s->max_len < 0) return SA_ERR_SHAPE;
    if (s->H < 1 || s->H > 65535 || s->H_kv < 1 || s->H % s->H_kv || s->d < 1 || s->d > 256 || s->d % 4) return SA_ERR_SHAPE;
    const Geom q{s->H, 0, s->stride_h, s->stride_s}, kv{s->H_kv, 0, s->kv_stride_h, s->kv_stride_s};
    if (s->stat_stride_h < s->rows) return SA_ERR_SHAPE;
    if (int e = check_geom(q, 1, s->rows, s->d)) return e;
    return check_geom(kv, 1, s->rows, s->d);
}
// The tile loads address a sequence through a buffer descriptor with 32-bit byte offsets: its last tile must end below 2^31
// bytes from its first row (in `stride`, elements between rows).
bool packed_in_reach(const sa_packed* s, int64_t stride) {
    const int64_t rows = ((int64_t)std::min(s->max_len, s->rows) + 127) / 128 * 128;
    return s->dtype == SA_F32 || stride < (int64_t(1) << 30) / (rows + 1);
}
// the pointers of a call, checked
int packed_fwd_args(const void* q, const void* k, const void* v, const int32_t* offsets, void* out, float* lse, const sa_packed* shape,
                    sa::PackedArgs& a) {
    if (!q || !k || !v || !offsets || !out || !lse) return SA_ERR_NULL;
    // (queries: a tile's 128 rows)
    if (!packed_in_reach(shape, shape->kv_stride_s) || (shape->dtype == SA_BF16 && shape->stride_s >= (1 << 23))) return SA_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || (reinterpret_cast<uintptr_t>(offsets) & 3u) ||
        (reinterpret_cast<uintptr_t>(lse) & 3u))
        return SA_ERR_ALIGN;
    a.q = q; a.k = k; a.v = v; a.o = (float*)out; a.lse = lse;
    return SA_OK;
}
int packed_bwd_args(const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse, const int32_t* offsets,
                    float* delta, void* dq, void* dk, void* dv, const sa_packed* shape, sa::PackedArgs& a) {
    if (!q || !k || !v || !out || !dout || !lse || !offsets || !delta || !dq || !dk || !dv) return SA_ERR_NULL;
    if (!packed_in_reach(shape, shape->kv_stride_s) || !packed_in_reach(shape, shape->stride_s)) return SA_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(dout) || !aligned16(dq) || !aligned16(dk) ||
        !aligned16(dv) || ((reinterpret_cast<uintptr_t>(offsets) | reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(delta)) & 3u))
        return SA_ERR_ALIGN;
    a.q = q; a.k = k; a.v = v; a.dout = dout; a.lse = const_cast<float*>(lse); a.delta = delta;
    a.o = (float*)const_cast<void*>(out);
    a.dq = (float*)dq; a.dk = (float*)dk; a.dv = (float*)dv;
    return SA_OK;
}
// One launch, or several of whole key/value heads and their groups where a launch would hold too many workgroups.
template <typename Args, typename Launch>
int play_packed(const sa_packed* s, const int32_t* offsets, Args a, Launch launch) {
    a.layout = SA_CONTIGUOUS; a.n_q = a.n_kv = 1; a.fresh = true;
    a.B = 1; a.H = s->H; a.H_kv = s->H_kv; a.d = s->d;
    a.stride_h = s->stride_h; a.stride_s = s->stride_s; a.kv_stride_h = s->kv_stride_h; a.kv_stride_s = s->kv_stride_s;
    a.stat_stride_h = s->stat_stride_h;
    a.scale = s->softmax_scale > 0.f ? s->softmax_scale : 1.0f / sqrtf((float)s->d);
    a.offsets = offsets; a.n_seq = s->n_seq; a.rows = s->rows; a.max_len = std::min(s->max_len, s->rows);
    a.es = (int)elt_size(s->dtype);
    const int group = s->H / s->H_kv;
    // per key/value head at most two workgroups for each tile and query head (fp32 ones of 32 rows have 512 threads) and as many for
    // its keys; bf16 launches of 32-row workgroups are kept small by their own rule (packed_split_wanted)
    const int64_t fit = kMostWorkgroups / (sa::most_tiles(a, s->dtype == SA_F32 ? 32 : 128) * 2 * (group + 1));
    if (fit < 1) return SA_ERR_SHAPE;
    const int heads = (int)std::min<int64_t>(fit, s->H_kv);
    for (int h = 0; h < s->H_kv; h += heads) {
        Args part = a;
        part.H_kv = std::min(heads, s->H_kv - h);
        part.H = part.H_kv * group;
        const int64_t q = (int64_t)h * group * a.stride_h * a.es, kv = (int64_t)h * a.kv_stride_h * a.es;
        auto at = [](const void* p, int64_t bytes) { return p ? (char*)p + bytes : nullptr; };
        part.q = at(a.q, q); part.k = at(a.k, kv); part.v = at(a.v, kv); part.dout = at(a.dout, q);
        part.o = (float*)at(a.o, q); part.dq = (float*)at(a.dq, q); part.dk = (float*)at(a.dk, kv); part.dv = (float*)at(a.dv, kv);
        part.lse = a.lse + (int64_t)h * group * a.stat_stride_h;
        if (a.delta) part.delta = a.delta + (int64_t)h * group * a.stat_stride_h;
        if (launch(part) != hipSuccess) return SA_ERR_HIP;
    }
    return SA_OK;
}
int check_window(const sa_window* w) {
    if (!w) return SA_ERR_NULL;
    return w->window < 1 || w->sinks < 0 ? SA_ERR_SHAPE : SA_OK;
}
// (rows and windows behind them are added in 32 bits)
bool too_long(const sa_packed* s) { return std::min(s->max_len, s->rows) > 1 << 30; }
// beyond the longest sequence neither says more
void set_window(sa::WindowArgs& a, const sa_packed* s, const sa_window* w) {
    a.n_seq = s->n_seq; a.rows = s->rows; a.max_len = std::min(s->max_len, s->rows);
    a.H = s->H; a.H_kv = s->H_kv; a.d = s->d; a.es = (int)elt_size(s->dtype);
    a.window = std::min(w->window, std::max(a.max_len, 1));
    a.sinks = std::min(w->sinks, a.max_len);
    sa::set_far(a);
    a.slot = -1;
}

// ---- paged cache
int check_cache(const sa_cache* c) {
    if (!c) return SA_ERR_NULL;
    if (c->dtype != SA_F32 && c->dtype != SA_BF16) return SA_ERR_DTYPE;
    if (c->n_pages < 1 || c->page_size < 16 || c->page_size % 16 || c->H_kv < 1 || c->H_kv > 65535 || c->d < 1 || c->d > 256 || c->d % 4)
        return SA_ERR_SHAPE;
    if ((int64_t)c->n_pages * c->page_size >= (int64_t(1) << 31)) return SA_ERR_SHAPE;
    if (int e = check_geom({c->H_kv, c->stride_page, c->stride_h, c->stride_s}, 1, c->page_size, c->d)) return e;
    // pages apart, and the tokens of a 16-row block within the 32-bit offsets of a descriptor
    const bool heads_apart = c->stride_h >= c->page_size * c->stride_s;
    if (c->n_pages > 1 && c->stride_page < (heads_apart ? c->H_kv * c->stride_h : c->page_size * c->stride_s)) return SA_ERR_SHAPE;
    if (c->stride_s >= (int64_t(1) << 24)) return SA_ERR_SHAPE;
    return c->stride_page % 4 ? SA_ERR_ALIGN : SA_OK;
}
int check_decode(const sa_decode* s, const sa_cache* c) {
    if (!s) return SA_ERR_NULL;
    if (int e = check_cache(c)) return e;
    if (s->B < 0 || s->H < 1 || s->H % c->H_kv || s->max_pages < 0) return SA_ERR_SHAPE;
    if ((int64_t)s->B * s->H > kMostWorkgroups || (int64_t)s->max_pages * c->page_size > (int64_t(1) << 30)) return SA_ERR_SHAPE;
    // (chunks of all units are numbered in 31 bits)
    if (((int64_t)s->max_pages * c->page_size / 64 + 1) * s->B * s->H >= (int64_t(1) << 31)) return SA_ERR_SHAPE;
    if (s->stride_h < c->d || (s->B > 1 && (s->stride_b < s->H * s->stride_h || s->stat_stride_b < s->H))) return SA_ERR_SHAPE;
    if (s->B > 1 && s->table_stride < s->max_pages) return SA_ERR_SHAPE;
    return s->stride_b % 4 || s->stride_h % 4 ? SA_ERR_ALIGN : SA_OK;
}

template <typename Args>
void set_cache(Args& a, const sa_cache* c) {
    a.H_kv = c->H_kv; a.d = c->d; a.n_pages = c->n_pages; a.page_size = c->page_size;
    a.stride_page = c->stride_page; a.stride_slot = c->stride_s; a.stride_head = c->stride_h;
}
// the pointers of a call, checked
int decode_args(const void* q, const void* k_cache, const void* v_cache, const int32_t* table, const int32_t* lens, void* out, float* lse, void* workspace,
                int64_t workspace_bytes, const sa_decode* shape, const sa_cache* cache, sa::DecodeArgs& a) {
    if (!q || !k_cache || !v_cache || !lens || !out || !workspace || (!table && shape->max_pages > 0)) return SA_ERR_NULL;
    if (workspace_bytes < sa::decode_workspace(shape->H, cache->H_kv, cache->d)) return SA_ERR_SHAPE;
    for (const void* p : {q, k_cache, v_cache, (const void*)out, (const void*)workspace})
        if (!aligned16(p)) return SA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(lens) | reinterpret_cast<uintptr_t>(lse)) & 3u) return SA_ERR_ALIGN;
    a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.table = table; a.lens = lens; a.out = out; a.lse = lse;
    a.parts = (float*)workspace;
    a.B = shape->B; a.H = shape->H; a.max_pages = shape->max_pages;
    a.stride_b = shape->stride_b; a.stride_h = shape->stride_h; a.stat_stride_b = shape->stat_stride_b; a.table_stride = shape->table_stride;
    set_cache(a, cache);
    a.scale = shape->softmax_scale > 0.f ? shape->softmax_scale : 1.0f / sqrtf((float)cache->d);
    return SA_OK;
}
int check_tree(const sa_tree* s, const sa_cache* c) {
    if (!s) return SA_ERR_NULL;
    if (int e = check_cache(c)) return e;
    if (s->B < 0 || s->T < 1 || s->T > 64 || s->H < 1 || s->H % c->H_kv || s->max_pages < 0) return SA_ERR_SHAPE;
    if ((int64_t)s->B * s->T * s->H > kMostWorkgroups || (int64_t)s->max_pages * c->page_size > (int64_t(1) << 30)) return SA_ERR_SHAPE;
    // (chunks of all units are numbered in 31 bits)
    const int64_t units = (int64_t)c->H_kv * (((int64_t)s->T * (s->H / c->H_kv) + 15) / 16) * s->B;
    if (((int64_t)s->max_pages * c->page_size / 64 + 1) >= (int64_t(1) << 31) / std::max<int64_t>(units, 1)) return SA_ERR_SHAPE;
    if (s->stride_h < c->d || (s->T > 1 && (s->stride_t < s->H * s->stride_h || s->stat_stride_t < s->H))) return SA_ERR_SHAPE;
    if (s->B > 1 && (s->stride_b < (s->T - 1) * s->stride_t + s->H * s->stride_h || s->stat_stride_b < (s->T - 1) * s->stat_stride_t + s->H)) return SA_ERR_SHAPE;
    if (s->B > 1 && (s->table_stride < s->max_pages || s->seen_stride < s->T)) return SA_ERR_SHAPE;
    return s->stride_b % 4 || s->stride_t % 4 || s->stride_h % 4 ? SA_ERR_ALIGN : SA_OK;
}

// Event bookkeeping for the drivers' optional per-step timings.
struct StepTimer {
    std::vector<hipEvent_t> ev;
    std::vector<int> slot;
    bool on;
    explicit StepTimer(bool enabled) : on(enabled) {}
    bool begin(hipStream_t st, int s) {
        if (!on) return true;
        hipEvent_t a, b;
        if (hipEventCreate(&a) != hipSuccess) return false;
        if (hipEventCreate(&b) != hipSuccess) { (void)hipEventDestroy(a); return false; }
        ev.push_back(a); ev.push_back(b); slot.push_back(s);
        return hipEventRecord(a, st) == hipSuccess;
    }
    bool end(hipStream_t st) { return !on || hipEventRecord(ev.back(), st) == hipSuccess; }
    bool collect(hipStream_t st, float* out) {
        if (!on) return true;
        bool ok = hipStreamSynchronize(st) == hipSuccess;
        for (size_t i = 0; i < slot.size(); ++i) {
            float ms = 0.f;
            if (ok && hipEventElapsedTime(&ms, ev[2 * i], ev[2 * i + 1]) == hipSuccess) out[slot[i]] = ms;
            else ok = false;
        }
        return ok;
    }
    ~StepTimer() { for (hipEvent_t e : ev) (void)hipEventDestroy(e); }
};

}  // namespace

extern "C" {

int sa_stripe_permute(const void* src, void* dst, int64_t outer, int64_t n_seq, int64_t inner_bytes,
                      int32_t N, void* stream) {
    return permute_common(src, dst, outer, n_seq, inner_bytes, N, false, stream);
}

int sa_unstripe_permute(const void* src, void* dst, int64_t outer, int64_t n_seq, int64_t inner_bytes,
                        int32_t N, void* stream) {
    return permute_common(src, dst, outer, n_seq, inner_bytes, N, true, stream);
}

int sa_state_init(float* o, float* lse, const sa_shape* shape, void* stream) {
    if (!o || !lse) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (!aligned16(o)) return SA_ERR_ALIGN;
    return sa::launch_state_init(o, lse, *shape, (hipStream_t)stream) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int sa_rope(const void* x, void* y, const int32_t* pos, int64_t pos_stride_b, const sa_shape* shape,
            float base, int32_t inverse, void* stream) {
    if (!x || !y || !pos) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (pos_stride_b < 0 || (pos_stride_b > 0 && pos_stride_b < shape->c) || !(base > 1.f)) return SA_ERR_SHAPE;
    if (!aligned16(x) || !aligned16(y) || (reinterpret_cast<uintptr_t>(pos) & 3u)) return SA_ERR_ALIGN;
    return sa::launch_rope(x, y, pos, pos_stride_b, *shape, base, inverse != 0, (hipStream_t)stream) ==
                   hipSuccess ? SA_OK : SA_ERR_HIP;
}

int sa_attn_step_fwd_tiled(const void* q, const void* k, const void* v, float* o, float* lse,
                           int32_t q_dev, int32_t kv_dev, int32_t N, int32_t layout, const sa_shape* shape,
                           int32_t skip_bq, int32_t skip_bk, void* stream) {
    if (!q || !k || !v || !o || !lse) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (int e = check_step(q_dev, kv_dev, N, layout)) return e;
    if (int e = check_skip(shape, skip_bq, skip_bk)) return e;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o)) return SA_ERR_ALIGN;
    return step_fwd(q, k, v, o, lse, q_dev, kv_dev, layout, shape, skip_bq, skip_bk, (hipStream_t)stream);
}

int sa_attn_step_fwd_rope(const void* q, const void* k, const void* v, float* o, float* lse,
                          const int32_t* q_pos, int64_t pos_stride_b, float rope_base, int32_t q_dev,
                          int32_t kv_dev, int32_t N, int32_t layout, const sa_shape* shape, void* stream) {
    if (!q || !k || !v || !o || !lse || !q_pos) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (int e = check_step(q_dev, kv_dev, N, layout)) return e;
    if (pos_stride_b < 0 || (pos_stride_b > 0 && pos_stride_b < shape->c) || !(rope_base > 1.f)) return SA_ERR_SHAPE;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(o) ||
        (reinterpret_cast<uintptr_t>(q_pos) & 3u))
        return SA_ERR_ALIGN;
    return step_fwd(q, k, v, o, lse, q_dev, kv_dev, layout, shape, 0, 0, (hipStream_t)stream, q_pos,
                    pos_stride_b, rope_base);
}

int sa_attn_step_fwd(const void* q, const void* k, const void* v, float* o, float* lse, int32_t q_dev,
                     int32_t kv_dev, int32_t N, int32_t layout, const sa_shape* shape, void* stream) {
    return sa_attn_step_fwd_tiled(q, k, v, o, lse, q_dev, kv_dev, N, layout, shape, 0, 0, stream);
}

int sa_finalize(const float* o, void* out, const sa_shape* shape, void* stream) {
    if (!o || !out) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (!aligned16(o) || !aligned16(out)) return SA_ERR_ALIGN;
    return sa::launch_finalize(o, out, *shape, (hipStream_t)stream) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int sa_bwd_preprocess(const float* o, const void* dout, float* delta, const sa_shape* shape,
                      void* stream) {
    if (!o || !dout || !delta) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (!aligned16(o) || !aligned16(dout)) return SA_ERR_ALIGN;
    return sa::launch_bwd_preprocess(o, dout, delta, *shape, shape->c, (hipStream_t)stream) == hipSuccess
               ? SA_OK : SA_ERR_HIP;
}

int sa_attn_step_bwd_tiled(const void* q, const void* k, const void* v, const void* dout,
                           const float* lse, const float* delta, float* dq, float* dk, float* dv,
                           int32_t q_dev, int32_t kv_dev, int32_t N, int32_t layout, const sa_shape* shape,
                           int32_t skip_bq, int32_t skip_bk, void* stream) {
    if (!q || !k || !v || !dout || !lse || !delta || !dq || !dk || !dv) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (int e = check_step(q_dev, kv_dev, N, layout)) return e;
    if (int e = check_skip(shape, skip_bq, skip_bk)) return e;
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(dout) || !aligned16(dq) ||
        !aligned16(dk) || !aligned16(dv))
        return SA_ERR_ALIGN;
    return step_bwd(q, k, v, dout, lse, delta, dq, dk, dv, q_dev, kv_dev, layout, shape, skip_bq, skip_bk,
                    (hipStream_t)stream);
}

int sa_attn_step_bwd(const void* q, const void* k, const void* v, const void* dout, const float* lse,
                     const float* delta, float* dq, float* dk, float* dv, int32_t q_dev, int32_t kv_dev,
                     int32_t N, int32_t layout, const sa_shape* shape, void* stream) {
    return sa_attn_step_bwd_tiled(q, k, v, dout, lse, delta, dq, dk, dv, q_dev, kv_dev, N, layout, shape,
                                  0, 0, stream);
}

int sa_ring_fwd_tiled(const void* Q, const void* K, const void* V, float* O, float* LSE, int32_t N,
                      int32_t layout, const sa_shape* shape, int32_t skip_bq, int32_t skip_bk,
                      int32_t q_dev_only, float* step_ms, void* stream) {
    if (!Q || !K || !V || !O || !LSE) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (int e = check_skip(shape, skip_bq, skip_bk)) return e;
    if (N < 1 || q_dev_only >= N) return SA_ERR_DEV;
    if (layout != SA_CONTIGUOUS && layout != SA_STRIPED) return SA_ERR_LAYOUT;
    if (int e = check_ring_extent(shape, N)) return e;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(O)) return SA_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    const size_t es = elt_size(shape->dtype);
    const int64_t shard = (int64_t)shape->c * row_stride(shape);     // elements between shards
    const int64_t kv_shard = (int64_t)shape->c * kv_geom(shape).ss;  // ... of K and V
    auto in_at = [&](const void* p, int dev) { return (const char*)p + (size_t)dev * shard * es; };
    auto kv_at = [&](const void* p, int dev) { return (const char*)p + (size_t)dev * kv_shard * es; };
    if (step_ms) for (int i = 0; i < N * N; ++i) step_ms[i] = 0.f;
    const int j0 = q_dev_only >= 0 ? q_dev_only : 0, j1 = q_dev_only >= 0 ? q_dev_only + 1 : N;
    StepArgs all = make_args(shape, j0, 0, layout);
    all.n_q = j1 - j0; all.n_kv = N; all.q_shard = shard; all.kv_shard = kv_shard; all.fresh = true;
    if (!step_ms && one_launch(all, N)) {
        all.q = in_at(Q, j0); all.k = K; all.v = V;
        all.o = O + j0 * shard; all.lse = LSE + (int64_t)j0 * shape->c;
        all.skip_bq = skip_bq; all.skip_bk = skip_bk;
        return launch_fwd(all, shape->dtype, st) == hipSuccess ? SA_OK : SA_ERR_HIP;
    }
    for (int j = j0; j < j1; ++j)
        if (sa::launch_state_init(O + j * shard, LSE + (int64_t)j * shape->c, *shape, st) != hipSuccess)
            return SA_ERR_HIP;
    StepTimer timer(step_ms != nullptr);
    for (int i = 0; i < N; ++i) {
        for (int j = j0; j < j1; ++j) {
            const int k = ((j - i) % N + N) % N;            // Algorithm 1: block held in round i
            if (!timer.begin(st, i * N + j)) return SA_ERR_HIP;
            int e = step_fwd(in_at(Q, j), kv_at(K, k), kv_at(V, k), O + j * shard,
                             LSE + (int64_t)j * shape->c, j, k, layout, shape, skip_bq, skip_bk, st);
            if (e) return e;
            if (!timer.end(st)) return SA_ERR_HIP;
        }
    }
    return timer.collect(st, step_ms) ? SA_OK : SA_ERR_HIP;
}

int sa_ring_fwd(const void* Q, const void* K, const void* V, float* O, float* LSE, int32_t N,
                int32_t layout, const sa_shape* shape, int32_t q_dev_only, float* step_ms, void* stream) {
    return sa_ring_fwd_tiled(Q, K, V, O, LSE, N, layout, shape, 0, 0, q_dev_only, step_ms, stream);
}

int sa_ring_bwd_tiled(const void* Q, const void* K, const void* V, const void* dO, const float* O,
                      const float* LSE, float* delta, float* dQ, float* dK, float* dV, int32_t N,
                      int32_t layout, const sa_shape* shape, int32_t skip_bq, int32_t skip_bk,
                      int32_t q_dev_only, float* step_ms, void* stream) {
    if (!Q || !K || !V || !dO || !O || !LSE || !delta || !dQ || !dK || !dV) return SA_ERR_NULL;
    if (int e = check_shape(shape)) return e;
    if (int e = check_skip(shape, skip_bq, skip_bk)) return e;
    if (N < 1 || q_dev_only >= N) return SA_ERR_DEV;
    if (layout != SA_CONTIGUOUS && layout != SA_STRIPED) return SA_ERR_LAYOUT;
    if (int e = check_ring_extent(shape, N)) return e;
    if (!aligned16(Q) || !aligned16(K) || !aligned16(V) || !aligned16(dO) || !aligned16(O) ||
        !aligned16(dQ) || !aligned16(dK) || !aligned16(dV))
        return SA_ERR_ALIGN;
    hipStream_t st = (hipStream_t)stream;
    const size_t es = elt_size(shape->dtype);
    const int64_t shard = (int64_t)shape->c * row_stride(shape);     // elements between shards
    const Geom kvg = kv_geom(shape);
    const int64_t kv_shard = (int64_t)shape->c * kvg.ss;             // ... of K, V, dK, dV
    auto in_at = [&](const void* p, int dev) { return (const char*)p + (size_t)dev * shard * es; };
    auto kv_at = [&](const void* p, int dev) { return (const char*)p + (size_t)dev * kv_shard * es; };
    if (step_ms) for (int i = 0; i < N * N; ++i) step_ms[i] = 0.f;
    const int j0 = q_dev_only >= 0 ? q_dev_only : 0, j1 = q_dev_only >= 0 ? q_dev_only + 1 : N;
    sa_shape kv_shape = *shape;          // dK and dV as a tensor family of their own
    kv_shape.H = kvg.heads; kv_shape.stride_b = kvg.sb; kv_shape.stride_h = kvg.sh; kv_shape.stride_s = kvg.ss;
    // rows first .. first + n - 1 of the devices' shards, as one tensor
    auto zero = [&](float* p, int64_t shard_elts, const sa_shape& s, int first, int n) {
        return n <= 0 || sa::launch_zero_f32(p + first * shard_elts, s, (int64_t)n * shape->c, st) == hipSuccess;
    };
    StepArgs all = make_args(shape, j0, 0, layout);
    all.n_q = j1 - j0; all.q_shard = shard; all.kv_shard = kv_shard; all.fresh = true;
    // key shards that some played device sees; contiguous layout: none further on than the last
    all.n_kv = layout == SA_STRIPED ? N : j1;
    if (!step_ms && one_launch(all, N)) {
        all.q = in_at(Q, j0); all.k = K; all.v = V; all.dout = in_at(dO, j0);
        all.lse = const_cast<float*>(LSE) + (int64_t)j0 * shape->c;
        all.delta = delta + (int64_t)j0 * shape->c;
        all.dq = dQ + j0 * shard; all.dk = dK; all.dv = dV;
        all.skip_bq = skip_bq; all.skip_bk = skip_bk;
        // what the kernels do not write: other devices' dQ, dK / dV of shards no played device sees
        if (!zero(dQ, shard, *shape, 0, j0) || !zero(dQ, shard, *shape, j1, N - j1) ||
            !zero(dK, kv_shard, kv_shape, all.n_kv, N - all.n_kv) ||
            !zero(dV, kv_shard, kv_shape, all.n_kv, N - all.n_kv) ||
            sa::launch_bwd_preprocess(O + j0 * shard, in_at(dO, j0), delta + (int64_t)j0 * shape->c, *shape,
                                      (int64_t)(j1 - j0) * shape->c, st) != hipSuccess)
            return SA_ERR_HIP;
        return launch_bwd(all, shape->dtype, st) == hipSuccess ? SA_OK : SA_ERR_HIP;
    }
    if (!zero(dQ, shard, *shape, 0, N) || !zero(dK, kv_shard, kv_shape, 0, N) ||
        !zero(dV, kv_shard, kv_shape, 0, N))
        return SA_ERR_HIP;
    for (int j = j0; j < j1; ++j)
        if (sa::launch_bwd_preprocess(O + j * shard, in_at(dO, j), delta + (int64_t)j * shape->c, *shape,
                                      shape->c, st) != hipSuccess)
            return SA_ERR_HIP;
    StepTimer timer(step_ms != nullptr);
    for (int i = 0; i < N; ++i) {
        for (int j = j0; j < j1; ++j) {
            const int k = ((j - i) % N + N) % N;
            if (!timer.begin(st, i * N + j)) return SA_ERR_HIP;
            int e = step_bwd(in_at(Q, j), kv_at(K, k), kv_at(V, k), in_at(dO, j),
                             LSE + (int64_t)j * shape->c, delta + (int64_t)j * shape->c, dQ + j * shard,
                             dK + k * kv_shard, dV + k * kv_shard, j, k, layout, shape, skip_bq, skip_bk,
                             st);
            if (e) return e;
            if (!timer.end(st)) return SA_ERR_HIP;
        }
    }
    return timer.collect(st, step_ms) ? SA_OK : SA_ERR_HIP;
}

int sa_ring_bwd(const void* Q, const void* K, const void* V, const void* dO, const float* O,
                const float* LSE, float* delta, float* dQ, float* dK, float* dV, int32_t N, int32_t layout,
                const sa_shape* shape, int32_t q_dev_only, float* step_ms, void* stream) {
    return sa_ring_bwd_tiled(Q, K, V, dO, O, LSE, delta, dQ, dK, dV, N, layout, shape, 0, 0, q_dev_only,
                             step_ms, stream);
}

int sa_attn_packed_fwd(const void* q, const void* k, const void* v, const int32_t* offsets, void* out, float* lse,
                       const sa_packed* shape, void* stream) {
    if (int e = check_packed(shape)) return e;
    if (shape->n_seq == 0 || shape->rows == 0 || shape->max_len == 0) return SA_OK;
    sa::PackedArgs a{};
    if (int e = packed_fwd_args(q, k, v, offsets, out, lse, shape, a)) return e;
    hipStream_t st = (hipStream_t)stream;
    return play_packed(shape, offsets, a, [&](const sa::PackedArgs& p) {
        return shape->dtype == SA_F32 ? sa::launch_packed_f32(p, false, st) : sa::launch_packed_fwd(p, st);
    });
}

int sa_attn_packed_bwd(const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse,
                       const int32_t* offsets, float* delta, void* dq, void* dk, void* dv, const sa_packed* shape, void* stream) {
    if (int e = check_packed(shape)) return e;
    if (shape->n_seq == 0 || shape->rows == 0 || shape->max_len == 0) return SA_OK;
    sa::PackedArgs a{};
    if (int e = packed_bwd_args(q, k, v, out, dout, lse, offsets, delta, dq, dk, dv, shape, a)) return e;
    hipStream_t st = (hipStream_t)stream;
    return play_packed(shape, offsets, a, [&](const sa::PackedArgs& p) {
        return shape->dtype == SA_F32 ? sa::launch_packed_f32(p, true, st) : sa::launch_packed_bwd(p, st);
    });
}

int sa_attn_window_fwd(const void* q, const void* k, const void* v, const int32_t* offsets, void* out, float* lse,
                       const sa_packed* shape, const sa_window* window, void* stream) {
    if (int e = check_packed(shape)) return e;
    if (int e = check_window(window)) return e;
    if (shape->n_seq == 0 || shape->rows == 0 || shape->max_len == 0) return SA_OK;
    if (too_long(shape)) return SA_ERR_SHAPE;
    sa::WindowArgs a{};
    if (int e = packed_fwd_args(q, k, v, offsets, out, lse, shape, a)) return e;
    set_window(a, shape, window);
    hipStream_t st = (hipStream_t)stream;
    return play_packed(shape, offsets, a, [&](const sa::WindowArgs& p) {
        return shape->dtype == SA_F32 ? sa::launch_window_f32(p, false, st) : sa::launch_window_fwd(p, st);
    });
}

int64_t sa_attn_window_bwd_workspace(const sa_packed* shape, const sa_window* window) {
    if (int e = check_packed(shape)) return e;
    if (int e = check_window(window)) return e;
    if (too_long(shape)) return SA_ERR_SHAPE;
    sa::WindowArgs a{};
    set_window(a, shape, window);
    return sa::far_bytes(a);
}

int sa_attn_window_bwd(const void* q, const void* k, const void* v, const void* out, const void* dout, const float* lse,
                       const int32_t* offsets, float* delta, void* dq, void* dk, void* dv, void* workspace, int64_t workspace_bytes,
                       const sa_packed* shape, const sa_window* window, void* stream) {
    if (int e = check_packed(shape)) return e;
    if (int e = check_window(window)) return e;
    if (shape->n_seq == 0 || shape->rows == 0 || shape->max_len == 0) return SA_OK;
    if (too_long(shape)) return SA_ERR_SHAPE;
    sa::WindowArgs a{};
    if (int e = packed_bwd_args(q, k, v, out, dout, lse, offsets, delta, dq, dk, dv, shape, a)) return e;
    const int64_t bytes = sa_attn_window_bwd_workspace(shape, window);
    if (workspace_bytes < bytes) return SA_ERR_SHAPE;
    if (bytes > 0 && !workspace) return SA_ERR_NULL;
    if (!aligned16(workspace)) return SA_ERR_ALIGN;
    set_window(a, shape, window);
    a.work = (float*)workspace;
    hipStream_t st = (hipStream_t)stream;
    return play_packed(shape, offsets, a, [&](const sa::WindowArgs& p) {
        return shape->dtype == SA_F32 ? sa::launch_window_f32(p, true, st) : sa::launch_window_bwd(p, st);
    });
}

int sa_cache_append(const void* q, void* q_out, const void* k, void* k_out, const void* v, const int32_t* pos, const int32_t* slot,
                    void* k_cache, void* v_cache, const sa_append* rows, const sa_cache* cache, void* stream) {
    if (!rows) return SA_ERR_NULL;
    if (int e = check_cache(cache)) return e;
    if (rows->rows < 0) return SA_ERR_SHAPE;
    if (rows->rows == 0) return SA_OK;
    if (!k || !v || !slot || !k_cache || !v_cache || !q != !q_out || (q && !pos)) return SA_ERR_NULL;
    if (q) {
        if (rows->H < 1 || rows->H > 65535) return SA_ERR_SHAPE;
        if (int e = check_geom({rows->H, 0, rows->stride_h, rows->stride_s}, 1, rows->rows, cache->d)) return e;
    }
    if (int e = check_geom({cache->H_kv, 0, rows->kv_stride_h, rows->kv_stride_s}, 1, rows->rows, cache->d)) return e;
    if (pos && !(rows->rope_base > 1.f)) return SA_ERR_SHAPE;
    for (const void* p : {q, (const void*)q_out, k, (const void*)k_out, v, (const void*)k_cache, (const void*)v_cache})
        if (!aligned16(p)) return SA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(pos) | reinterpret_cast<uintptr_t>(slot)) & 3u) return SA_ERR_ALIGN;
    sa::AppendArgs a{};
    a.q = q; a.q_out = q_out; a.k = k; a.k_out = k_out; a.v = v; a.pos = pos; a.slot = slot; a.k_cache = k_cache; a.v_cache = v_cache;
    a.rows = rows->rows; a.H = rows->H; a.H_kv = cache->H_kv; a.d = cache->d; a.page_size = cache->page_size;
    a.n_slots = (int64_t)cache->n_pages * cache->page_size;
    a.stride_h = rows->stride_h; a.stride_s = rows->stride_s; a.kv_stride_h = rows->kv_stride_h; a.kv_stride_s = rows->kv_stride_s;
    a.stride_page = cache->stride_page; a.stride_slot = cache->stride_s; a.stride_head = cache->stride_h;
    a.log2_base = pos ? log2((double)rows->rope_base) : 0.;
    return sa::launch_cache_append(a, cache->dtype, (hipStream_t)stream) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int64_t sa_attn_decode_workspace(const sa_decode* shape, const sa_cache* cache) {
    if (int e = check_decode(shape, cache)) return e;
    return sa::decode_workspace(shape->H, cache->H_kv, cache->d);
}

int sa_attn_decode(const void* q, const void* k_cache, const void* v_cache, const int32_t* table, const int32_t* lens, void* out,
                   float* lse, void* workspace, int64_t workspace_bytes, const sa_decode* shape, const sa_cache* cache, void* stream) {
    if (int e = check_decode(shape, cache)) return e;
    if (shape->B == 0) return SA_OK;
    sa::DecodeArgs a{};
    if (int e = decode_args(q, k_cache, v_cache, table, lens, out, lse, workspace, workspace_bytes, shape, cache, a)) return e;
    return sa::launch_decode(a, cache->dtype, (hipStream_t)stream) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int sa_attn_window_decode(const void* q, const void* k_cache, const void* v_cache, const int32_t* table, const int32_t* lens, void* out,
                          float* lse, void* workspace, int64_t workspace_bytes, const sa_decode* shape, const sa_cache* cache,
                          const sa_window* window, void* stream) {
    if (int e = check_decode(shape, cache)) return e;
    if (int e = check_window(window)) return e;
    if (shape->B == 0) return SA_OK;
    sa::WindowDecodeArgs a{};
    if (int e = decode_args(q, k_cache, v_cache, table, lens, out, lse, workspace, workspace_bytes, shape, cache, a)) return e;
    const int room = std::max(1, shape->max_pages * cache->page_size);         // (beyond it neither says more)
    a.window = std::min(window->window, room);
    a.sinks = std::min(window->sinks, room);
    return sa::launch_window_decode(a, cache->dtype, (hipStream_t)stream) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int64_t sa_attn_tree_workspace(const sa_tree* shape, const sa_cache* cache) {
    if (int e = check_tree(shape, cache)) return e;
    return sa::tree_workspace(shape->T * (shape->H / cache->H_kv), cache->d, cache->dtype);
}

int sa_attn_tree(const void* q, const void* k_cache, const void* v_cache, const int32_t* table, const int32_t* lens, const int32_t* drafts,
                 const int64_t* seen, void* out, float* lse, void* workspace, int64_t workspace_bytes, const sa_tree* shape,
                 const sa_cache* cache, void* stream) {
    if (int e = check_tree(shape, cache)) return e;
    if (shape->B == 0) return SA_OK;
    if (!q || !k_cache || !v_cache || !lens || !seen || !out || !workspace || (!table && shape->max_pages > 0)) return SA_ERR_NULL;
    if (workspace_bytes < sa_attn_tree_workspace(shape, cache)) return SA_ERR_SHAPE;
    for (const void* p : {q, k_cache, v_cache, (const void*)out, (const void*)workspace})
        if (!aligned16(p)) return SA_ERR_ALIGN;
    for (const void* p : {(const void*)table, (const void*)lens, (const void*)drafts, (const void*)lse})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return SA_ERR_ALIGN;
    if (reinterpret_cast<uintptr_t>(seen) & 7u) return SA_ERR_ALIGN;
    sa::TreeArgs a{};
    a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.table = table; a.lens = lens; a.drafts = drafts; a.seen = seen; a.out = out; a.lse = lse;
    a.parts = (float*)workspace;
    a.B = shape->B; a.T = shape->T; a.H = shape->H; a.max_pages = shape->max_pages;
    a.stride_b = shape->stride_b; a.stride_t = shape->stride_t; a.stride_h = shape->stride_h;
    a.stat_stride_b = shape->stat_stride_b; a.stat_stride_t = shape->stat_stride_t;
    a.table_stride = shape->table_stride; a.seen_stride = shape->seen_stride;
    set_cache(a, cache);
    a.scale = shape->softmax_scale > 0.f ? shape->softmax_scale : 1.0f / sqrtf((float)cache->d);
    return sa::launch_tree(a, cache->dtype, (hipStream_t)stream) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int sa_cache_accept(void* k_cache, void* v_cache, const int32_t* table, const int32_t* lens, const int32_t* chosen, const int32_t* accepted,
                    int32_t* lens_after, const sa_accept* shape, const sa_cache* cache, void* stream) {
    if (!shape) return SA_ERR_NULL;
    if (int e = check_cache(cache)) return e;
    if (shape->B < 0 || shape->B > 1 << 22 || shape->T < 1 || shape->T > 64 || shape->max_pages < 0) return SA_ERR_SHAPE;
    if ((int64_t)shape->max_pages * cache->page_size > (int64_t(1) << 30)) return SA_ERR_SHAPE;
    if (shape->B > 1 && (shape->table_stride < shape->max_pages || shape->chosen_stride < shape->T)) return SA_ERR_SHAPE;
    if (shape->B == 0) return SA_OK;
    if (!k_cache || !v_cache || !lens || !chosen || !accepted || (!table && shape->max_pages > 0)) return SA_ERR_NULL;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return SA_ERR_ALIGN;
    for (const void* p : {(const void*)table, (const void*)lens, (const void*)chosen, (const void*)accepted, (const void*)lens_after})
        if (reinterpret_cast<uintptr_t>(p) & 3u) return SA_ERR_ALIGN;
    sa::AcceptArgs a{};
    a.k_cache = k_cache; a.v_cache = v_cache; a.table = table; a.lens = lens; a.chosen = chosen; a.accepted = accepted; a.lens_after = lens_after;
    a.B = shape->B; a.T = shape->T; a.max_pages = shape->max_pages; a.table_stride = shape->table_stride; a.chosen_stride = shape->chosen_stride;
    set_cache(a, cache);
    return sa::launch_cache_accept(a, cache->dtype, (hipStream_t)stream) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int sa_cache_copy(void* k_cache, void* v_cache, const int32_t* from, const int32_t* to, const int32_t* tokens, int32_t n,
                  const sa_cache* cache, void* stream) {
    if (int e = check_cache(cache)) return e;
    if (n < 0 || n > 1 << 22) return SA_ERR_SHAPE;
    // (a page's units of 8 bytes are numbered in 31 bits)
    if ((double)cache->page_size * cache->H_kv * cache->d * (double)elt_size(cache->dtype) >= 17179869184.) return SA_ERR_SHAPE;
    if (n == 0) return SA_OK;
    if (!k_cache || !v_cache || !from || !to) return SA_ERR_NULL;
    if (!aligned16(k_cache) || !aligned16(v_cache)) return SA_ERR_ALIGN;
    if ((reinterpret_cast<uintptr_t>(from) | reinterpret_cast<uintptr_t>(to) | reinterpret_cast<uintptr_t>(tokens)) & 3u) return SA_ERR_ALIGN;
    sa::CopyArgs a{};
    a.k_cache = k_cache; a.v_cache = v_cache; a.from = from; a.to = to; a.tokens = tokens; a.n = n;
    set_cache(a, cache);
    return sa::launch_cache_copy(a, cache->dtype, (hipStream_t)stream) == hipSuccess ? SA_OK : SA_ERR_HIP;
}

int sa_step_mask(int32_t q_dev, int32_t kv_dev, int32_t N, int32_t layout, int32_t* kind, int32_t* off) {
    if (!kind || !off) return SA_ERR_NULL;
    if (int e = check_step(q_dev, kv_dev, N, layout)) return e;
    *kind = sa::block_kind(q_dev, kv_dev, layout);
    *off = sa::block_off(q_dev, kv_dev, layout);
    return SA_OK;
}

int64_t sa_step_pairs(int32_t q_dev, int32_t kv_dev, int32_t N, int32_t layout, int64_t c) {
    if (check_step(q_dev, kv_dev, N, layout) || c < 0) return -1;
    const int kind = sa::block_kind(q_dev, kv_dev, layout), off = sa::block_off(q_dev, kv_dev, layout);
    if (kind == sa::MASK_EMPTY) return 0;
    if (kind == sa::MASK_FULL) return c * c;
    return off ? c * (c - 1) / 2 : c * (c + 1) / 2;
}

int sa_step_tiles(int32_t q_dev, int32_t kv_dev, int32_t N, int32_t layout, int64_t c, int64_t skip_bq,
                  int64_t skip_bk, int64_t* computed, int64_t* total) {
    if (!computed || !total) return SA_ERR_NULL;
    if (int e = check_step(q_dev, kv_dev, N, layout)) return e;
    if (c < 1 || skip_bq < 1 || skip_bk < 1 || c % skip_bq || c % skip_bk) return SA_ERR_SHAPE;
    const int kind = sa::block_kind(q_dev, kv_dev, layout), off = sa::block_off(q_dev, kv_dev, layout);
    const int64_t nq = c / skip_bq, nk = c / skip_bk;
    *total = nq * nk;
    if (kind == sa::MASK_EMPTY) { *computed = 0; return SA_OK; }
    if (kind == sa::MASK_FULL) { *computed = nq * nk; return SA_OK; }
    // tile (r, s) holds an allowed pair iff its first key s*bk <= its last query (r+1)*bq - 1 - off
    int64_t n = 0;
    for (int64_t r = 0; r < nq; ++r) {
        const int64_t last = (r + 1) * skip_bq - 1 - off;       // last key any query of the tile sees
        if (last >= 0) n += (last / skip_bk + 1 < nk) ? last / skip_bk + 1 : nk;
    }
    *computed = n;
    return SA_OK;
}

int sa_device_props(int32_t* compute_units, int32_t* clock_khz, int64_t* memory_bytes) {
    if (!compute_units || !clock_khz || !memory_bytes) return SA_ERR_NULL;
    int dev = 0;
    hipDeviceProp_t prop;
    if (hipGetDevice(&dev) != hipSuccess || hipGetDeviceProperties(&prop, dev) != hipSuccess) return SA_ERR_HIP;
    *compute_units = prop.multiProcessorCount;
    *clock_khz = prop.clockRate;
    *memory_bytes = (int64_t)prop.totalGlobalMem;
    return SA_OK;
}

const char* sa_status_str(int status) {
    switch (status) {
        case SA_OK: return "ok";
        case SA_ERR_NULL: return "null pointer";
        case SA_ERR_SHAPE: return "bad shape";
        case SA_ERR_DEV: return "device index out of range";
        case SA_ERR_DTYPE: return "unsupported dtype";
        case SA_ERR_LAYOUT: return "bad layout";
        case SA_ERR_ALIGN: return "misaligned pointer or stride";
        case SA_ERR_HIP: return "HIP call failed";
        default: return "unknown status";
    }
}

}  // extern "C"
