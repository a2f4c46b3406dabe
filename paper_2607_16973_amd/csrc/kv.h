// Launch interface of the reader's kernels (prompt attention, the 8-bit cache
// and its pages) and what they share on the device.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "tq.h"

namespace tq {

constexpr int kPage = TQ_KV_PAGE;     // tokens of a page
constexpr int kBlock = TQ_KV_BLOCK;   // tokens under one scale

// One layer of a cache, as the kernels take it.
struct KvLayer {
    char *k, *v;                  // [pages][heads] tiles of 64 x D codes
    float *ks, *vs;               // [pages][heads][4]
    int *status;                  // or null
    int pages, heads;
};

// The packed new tokens of a call and the rows they belong to.
struct RowSet {
    const int *tables, *lens, *starts;   // starts null: one token per row
    int rows, width, total;
};

struct AppendArgs {
    KvLayer layer;
    RowSet set;
    const void *k, *v;
    int64_t kt, kh, vt, vh;       // strides in elements
    int bf16, wide;               // wide: 16-byte loads are aligned
};
hipError_t kv_append(const AppendArgs &a, int D, int type, hipStream_t stream);

struct AttendArgs {
    KvLayer layer;
    RowSet set;
    const void *q;
    int64_t qt, qh;
    void *out;
    float *lse;                   // or null
    int *info;                    // [units] first part and number of parts
    float *parts;                 // [2 shares][tile][D + 4]: sums, maximum, weight
    float scale2;                 // scale * log2(e)
    int heads, group, bf16, wide;
    int shares;
    int limit;                    // tokens of a row that are looked at
};
// How a call is split: query rows of a tile, tiles (units), waves that share
// the units' pages (0: a workgroup per unit).  line: a bound on the pages of all units.
struct AttendPlan {
    int tile, shares;
    int64_t units, line;
};
AttendPlan attend_plan(int64_t n, int rows, int group, int kv_heads, int width, int longest, int D, bool starts);
size_t attend_info_bytes(const AttendPlan &p);
size_t attend_bytes(const AttendPlan &p, int D);
hipError_t kv_attend(const AttendArgs &a, const AttendPlan &p, int D, int type, hipStream_t stream);

struct PromptArgs {
    const void *q, *k, *v;
    int64_t qt, qh, kt, kh, vt, vh;
    const int *starts, *key_starts;
    int rows, total, keys, heads, group, kv_heads, causal, wide;
    int levels;                   // tiles of the longest row where all are short, else 0
    float scale2;
    void *out;
    float *lse;
};
int prompt_levels(int group, int longest);
hipError_t prompt_attention(const PromptArgs &a, int D, int bf16, hipStream_t stream);

struct PagesArgs {
    int *tables, *lens, *refs;
    int pages, rows, width;
    KvLayer cache;                // layer 0
    int layers, D;
    void *ws;
};
size_t kv_rows_bytes(int64_t pages, int64_t rows, int64_t width, int64_t n);
hipError_t kv_resize(const PagesArgs &a, const int *goals, hipStream_t stream);
hipError_t kv_fork(const PagesArgs &a, const int *src, const int *dst, int n, hipStream_t stream);
hipError_t kv_compact(const PagesArgs &a, int *live, hipStream_t stream);

#ifdef __HIPCC__
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// The new tokens of row i within the packed tensor, kept inside it whatever
// starts holds.
__device__ inline void row_tokens(const int *starts, int i, int total, int *first, int *count) {
    if (!starts) {
        *first = min(i, total);
        *count = i < total ? 1 : 0;
        return;
    }
    const int a = min(max(starts[i], 0), total);
    *first = a;
    *count = min(max(starts[i + 1] - a, 0), total - a);
}

// The length of row i; negative ones count as 0, so that what is computed from it stays in range.
__device__ inline int row_length(const int *lens, int i) { return max(lens[i], 0); }

// Work slots of rows without a list made by the host: row i owns the slots
// from f(i) = starts[i] * num / den + i * extra on; the row of slot s is the last i
// with f(i) <= s.  (num / den slots per token, extra more per row.)
__device__ inline int64_t slot_begin(const int *starts, int i, int num, int den, int extra) {
    return (int64_t)starts[i] * num / den + (int64_t)i * extra;
}
// The last row i with begin(i) <= s, begin ascending.  Called by whole waves: the 64 lanes
// look at 64 places at once, so up to 64 rows take one round of loads, up to 4,096 two.
template <class F>
__device__ inline int row_of_slot(int rows, int64_t s, F begin) {
    const int lane = __lane_id();
    int lo = 0, n = rows;
    while (n > 1) {
        const int step = (n + 63) >> 6, i = lane * step;
        const bool le = i < n && begin(lo + i) <= s;
        const int past = __popcll(__ballot(le));
        if (past == 0) break;
        lo += (past - 1) * step;
        n = min(step, n - (past - 1) * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
__device__ inline int slot_row(const int *starts, int rows, int64_t s, int num, int den, int extra) {
    return row_of_slot(rows, s, [=](int i) { return slot_begin(starts, i, num, den, extra); });
}

// The larger; NaN if one is.  (One instruction each, also of values the matrix
// cores have just written: fmaxf would first quiet every operand.)
__device__ inline float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ inline float max3(float a, float b, float c) { return larger(larger(a, b), c); }

// Largest / sum over the lanes l, l ^ 16, l ^ 32, l ^ 48.
__device__ inline float max_of_groups(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = larger(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return larger(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float sum_of_groups(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// The same over l and l ^ 32.
__device__ inline float max_of_halves(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return larger(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ inline float sum_of_halves(float x) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(a[0]) + __uint_as_float(a[1]);
}

// x * f - m with both steps rounded: never fused, so that a value gives
// exactly 0 against its own rounded product.
__device__ inline float scaled_less(float x, float f, float m) {
#pragma clang fp contract(off)
    const float y = x * f;
    return y - m;
}

__device__ inline float bf16_float(unsigned short h) { return __uint_as_float((unsigned)h << 16); }
__device__ inline float f16_float(unsigned short h) {
    _Float16 x;
    __builtin_memcpy(&x, &h, 2);
    return (float)x;
}
__device__ inline unsigned short float_bits16(float x, int bf16) {
    unsigned short h;
    if (bf16) {
        const __bf16 y = (__bf16)x;
        __builtin_memcpy(&h, &y, 2);
    } else {
        const _Float16 y = (_Float16)x;
        __builtin_memcpy(&h, &y, 2);
    }
    return h;
}
// Eight 16-bit floats of a row, as float32: one 16-byte load where the row allows it.
__device__ inline void load8(const void *row, int64_t at, int bf16, int wide, float *x) {
    const unsigned short *p = static_cast<const unsigned short *>(row) + at;
    unsigned short h[8];
    if (wide) {
        const uint4 u = *reinterpret_cast<const uint4 *>(p);
        __builtin_memcpy(h, &u, 16);
    } else {
        for (int j = 0; j < 8; ++j) h[j] = p[j];
    }
    for (int j = 0; j < 8; ++j) x[j] = bf16 ? bf16_float(h[j]) : f16_float(h[j]);
}
#endif

}  // namespace tq
