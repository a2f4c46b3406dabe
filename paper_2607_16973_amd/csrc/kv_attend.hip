// Attention over the 8-bit cache.
//
// For one key head the rows of a tile are (new token, query head of the
// group) pairs, 16 per matrix-core tile.  A wave takes a page (64 tokens):
//   S^T = K Q^T     16x16x32 f16, four tiles of 16 tokens
//   O^T += V^T P^T  16x16x32 f16, D / 16 tiles of 16 coordinates
// The page's rows are dealt to the four S^T tiles so that the 16 results a
// lane gets -- four tiles of four -- are the 16 tokens of ONE block, block
// lane / 16: S^T tile t, row m holds token 16 (m / 4) + 4 t + m % 4.  So a
// lane multiplies its scores by one key scale and its weights by one value
// scale, and the weights it computed are, in order, the operand that the
// second product wants from it: nothing goes through LDS between the
// products, and one 16-byte load brings a lane the 16 tokens of a
// coordinate.  Query n = lane % 16 stays in its lane throughout, so the
// running maximum and sum of the softmax are lane values.
//
// Codes become float16 exactly (|z| <= 448).  Queries are brought to float16
// with one power of two per row that puts the largest at 2^14: what float16
// rounds away is 2^-39 of it.  The numerator has a running maximum of its own, over score +
// log2(value scale), so that weights times value scales stay in float16's
// range whatever the scales are; they are taken to the product in two
// float16 parts (22 bits: the product is far from its limit here, and the rounding of the weights
// would otherwise be as large as that of a float16 result).
#include <hip/hip_runtime.h>

#include "kv.h"

namespace tq {
namespace {

#ifndef WANT
#define WANT 4096
#define WHOLE 32
#endif

constexpr float kUnit = 6.f;      // weights are held in units of 2^-kUnit ...
constexpr float kLag = 8.f;       // ... and may pass the running maximum by 2^kLag before it follows

__device__ inline float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// 16 codes -> 2 x 8 float16.
template <bool FP8>
__device__ inline void to_half(const uint4 &c, f16x8 *lo, f16x8 *hi) {
    f16x2 h[8];
    const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if constexpr (FP8) {
            h[2 * q] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[q], 1.0f, false);
            h[2 * q + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w[q], 1.0f, true);
        } else {
            // bytes of code + 128 under 0x64: the float16 1024 + 128 + code
            const uint32_t u = w[q] ^ 0x80808080u;
            const uint32_t a = __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u);
            const uint32_t b = __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u);
            const f16x2 off = {(_Float16)-1152.f, (_Float16)-1152.f};
            h[2 * q] = __builtin_bit_cast(f16x2, a) + off;
            h[2 * q + 1] = __builtin_bit_cast(f16x2, b) + off;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        (*lo)[2 * j] = h[j].x;
        (*lo)[2 * j + 1] = h[j].y;
        (*hi)[2 * j] = h[4 + j].x;
        (*hi)[2 * j + 1] = h[4 + j].y;
    }
}

// Clears the codes of tokens at and past n of a 16-token line (n <= 16).
__device__ inline uint4 keep_tokens(uint4 c, int n) {
    auto mask = [n](int word) -> uint32_t {
        const int k = n - 4 * word;
        return k >= 4 ? ~0u : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
    };
    c.x &= mask(0);
    c.y &= mask(1);
    c.z &= mask(2);
    c.w &= mask(3);
    return c;
}

// Queries of 16 rows as operands, 8 coordinates (s/2) 64 + g 16 + (s%2) 8 of
// each step, in float16 with the power of two that is returned.
template <int D>
__device__ inline int load_queries(const AttendArgs &a, bool in, int64_t at, int g, f16x8 *q) {
    constexpr int KS = D / 32;
    float x[KS][8];
    float big = 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        if (in) load8(a.q, at + (s >> 1) * 64 + g * 16 + (s & 1) * 8, a.bf16, a.wide, x[s]);
        else for (int j = 0; j < 8; ++j) x[s][j] = 0.f;
        for (int j = 0; j < 8; ++j) {
            const float y = fabsf(x[s][j]);
            big = fmaxf(big, y < __builtin_inff() ? y : 0.f);
        }
    }
    big = max_of_groups(big);
    int e;
    frexpf(big, &e);
    e = big > 0.f ? 15 - e : 0;
    const float sign = a.scale2 < 0.f ? -1.f : 1.f;
#pragma unroll
    for (int s = 0; s < KS; ++s)
        for (int j = 0; j < 8; ++j) q[s][j] = (_Float16)(sign * ldexpf(x[s][j], e));
    return e;
}

// Rows of few queries (decoding, drafted tokens): NT tiles of 16 query rows that
// the W waves of the workgroup share.  Each wave takes every W-th page and
// has the next one's codes on the way while it works; the waves are joined
// through LDS.  Bound by the memory system: 16 pages of 64 D bytes in
// flight per compute unit.
template <int D, bool FP8, int NT, int W>
__global__ __launch_bounds__(64 * W) void attend_kernel(AttendArgs a) {
    constexpr int KS = D / 32;                       // 32-wide steps of the first product
    constexpr int DT = D / 16;
    constexpr int RT = 16 * NT;                      // rows of the workgroup
    extern __shared__ __align__(16) float lds[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int n = lane & 15, g = lane >> 4;

    int64_t slot = blockIdx.x / a.chunks;
    const int chunk = blockIdx.x % a.chunks, kvh = blockIdx.y;
    int row, first, count;
    if (a.set.starts) {
        row = slot_row(a.set.starts, a.set.rows, slot, a.group, RT, 1);
        slot -= slot_begin(a.set.starts, row, a.group, RT, 1);
    } else {   // one token per row: its group in ceil(group / RT) tiles
        const int per = (a.group + RT - 1) / RT;
        row = (int)(slot / per);
        slot %= per;
    }
    row_tokens(a.set.starts, row, a.set.total, &first, &count);
    const int rows = count * a.group;
    if (slot < 0 || slot * RT >= rows) return;       // the whole workgroup
    const int r0 = (int)slot * RT;
    const int true_len = a.set.lens[row];
    const int len = min(true_len, a.limit);

    // positions: the last key that each row, any row and every row sees
    int pos[NT], token[NT];
    const int last = min(rows - 1, r0 + RT - 1);
    const int top = min(true_len - count + last / a.group, len - 1);
    const int low = min(true_len - count + r0 / a.group, len - 1);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        token[i] = min(r0 + 16 * i + n, last) / a.group;
        pos[i] = min(true_len - count + token[i], len - 1);
    }
    const int begin = chunk * a.chunk_pages + wave;
    const int end = top < 0 ? 0 : min(top / kPage + 1, (chunk + 1) * a.chunk_pages);

    // what a page needs: its codes and the scales of the lane's block
    const int *table = a.set.tables + (int64_t)row * a.set.width;
    uint4 kc[4][D / 64], vc[DT];
    const int krow = (16 * (n >> 2) + (n & 3)) * D + g * 16, vrow = (g * D + n) * 16;
    int ahead = begin < end ? table[begin] : 0;      // page id of the next load
    bool fits = false;
    auto tile_of = [&](int page) {
        fits = page >= 0 && page < a.layer.pages;
        if (!fits && a.layer.status && lane == 0) atomicOr(a.layer.status, TQ_KV_BAD_PAGE);
        return (int64_t)(fits ? page : 0) * a.layer.heads + kvh;
    };
    auto load_keys = [&](int64_t tile) {
        const char *kp = a.layer.k + tile * (kPage * D) + krow;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int u = 0; u < D / 64; ++u) kc[s][u] = *reinterpret_cast<const uint4 *>(kp + 4 * s * D + u * 64);
    };
    auto load_values = [&](int64_t tile) {
        const char *vp = a.layer.v + tile * (kPage * D) + vrow;
#pragma unroll
        for (int d = 0; d < DT; ++d) vc[d] = *reinterpret_cast<const uint4 *>(vp + d * 256);
    };
    int64_t tile = 0;
    float ks = 0.f, vs = 0.f;
    if (begin < end) {
        tile = tile_of(__builtin_amdgcn_readfirstlane(ahead));
        load_keys(tile);
        ks = a.layer.ks[tile * 4 + g];
        vs = a.layer.vs[tile * 4 + g];
        load_values(tile);
        if (begin + W < end) ahead = table[begin + W];
    }

    f16x8 q[NT][KS];
    float factor[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int r = r0 + 16 * i + n;
        const int e = load_queries<D>(a, r < rows, (int64_t)(first + token[i]) * a.qt + (int64_t)(kvh * a.group + min(r, last) % a.group) * a.qh, g, q[i]);
        factor[i] = ldexpf(fabsf(a.scale2), -e);
    }
    float m[NT], mv[NT], l[NT];                      // maxima (log2 units) of scores and of scores with value scales; sum
    f32x4 o[NT][DT];                                 // in units of 2^(mv - kUnit)
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        m[i] = mv[i] = -__builtin_inff();
        l[i] = 0.f;
        for (int d = 0; d < DT; ++d) o[i][d] = {0.f, 0.f, 0.f, 0.f};
    }

    for (int p = begin; p < end; p += W) {
        // S^T of the page
        f32x4 x[NT][4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            for (int i = 0; i < NT; ++i) x[i][s] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < D / 64; ++u) {
                f16x8 lo, hi;
                to_half<FP8>(kc[s][u], &lo, &hi);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    x[i][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, q[i][2 * u], x[i][s], 0, 0, 0);
                    x[i][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, q[i][2 * u + 1], x[i][s], 0, 0, 0);
                }
            }
        }
        const bool here = fits, more = p + W < end;
        const float kscale = ks;
        if (more) {                                  // the next page's keys
            tile = tile_of(__builtin_amdgcn_readfirstlane(ahead));
            load_keys(tile);
            ks = a.layer.ks[tile * 4 + g];
            if (p + 2 * W < end) ahead = table[p + 2 * W];
        }
        __builtin_amdgcn_sched_barrier(0);
        const int base = p * kPage + 16 * g;         // position of the lane's first token
        float vlog = vs > 0.f ? __log2f(vs) : -__builtin_inff();
        // A page that holds the row's end may hold anything past it: those
        // codes and scales are taken out before they meet a zero weight.
        if ((p + 1) * kPage > len || !here) {
            const int left = here ? min(max(len - base, 0), 16) : 0;
            if (left == 0) vlog = -__builtin_inff();
#pragma unroll
            for (int d = 0; d < DT; ++d) vc[d] = keep_tokens(vc[d], left);
        }
        const bool masked = (p + 1) * kPage - 1 > low || !here;

        f16x8 w[NT][2], wl[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            // never 0, so that a masked score stays -inf (a NaN scale of an unused block goes too)
            const float f = fmaxf(factor[i] * kscale, 0x1p-126f);
            if (masked) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (base + j > pos[i] || !here) x[i][j >> 2][j & 3] = -__builtin_inff();
            }
            float big = max3(x[i][0][0], x[i][0][1], x[i][0][2]);
#pragma unroll
            for (int j = 3; j < 15; j += 2) big = max3(big, x[i][j >> 2][j & 3], x[i][(j + 1) >> 2][(j + 1) & 3]);
            big = fmaxf(big, x[i][3][3]) * f;
            const float top1 = max_of_groups(big), top2 = max_of_groups(big + vlog);
            if (__any(top1 > m[i] + kLag || top2 > mv[i] + kLag)) {
                const float m1 = fmaxf(m[i], top1), m2 = fmaxf(mv[i], top2);
                l[i] *= m[i] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(m[i] - m1);
                const float back = mv[i] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mv[i] - m2);
#pragma unroll
                for (int d = 0; d < DT; ++d) o[i][d] *= back;
                m[i] = m1;
                mv[i] = m2;
            }
            const float m1 = m[i] == -__builtin_inff() ? 0.f : m[i], m2 = mv[i] == -__builtin_inff() ? 0.f : mv[i];
            const float gain = __builtin_amdgcn_exp2f(fminf(vlog + (m1 - m2) + kUnit, 126.f));
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float e = __builtin_amdgcn_exp2f(scaled_less(x[i][j >> 2][j & 3], f, m1));
                sum += e;
                const float y = e * gain;
                const _Float16 hi = (_Float16)y;
                w[i][j >> 3][j & 7] = hi;
                wl[i][j >> 3][j & 7] = (_Float16)(y - (float)hi);
            }
            l[i] += sum;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            f16x8 lo, hi;
            to_half<FP8>(vc[d], &lo, &hi);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                o[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, w[i][0], o[i][d], 0, 0, 0);
                o[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, w[i][1], o[i][d], 0, 0, 0);
                o[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, wl[i][0], o[i][d], 0, 0, 0);
                o[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, wl[i][1], o[i][d], 0, 0, 0);
            }
        }
        if (more) {                                  // and its values
            load_values(tile);
            vs = a.layer.vs[tile * 4 + g];
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    constexpr int OS = D + 4;                        // LDS row, off the banks' period
    float *lm = lds + W * RT * OS;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const float sum = sum_of_groups(l[i]);
        // back to units of 2^m, which the waves and parts have in common with the sum
        const float back = mv[i] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mv[i] - m[i] - kUnit);
        for (int d = 0; d < DT; ++d)
            *reinterpret_cast<f32x4 *>(lds + ((wave * RT + 16 * i + n) * OS + d * 16 + g * 4)) = o[i][d] * back;
        if (g == 0) {
            lm[(wave * RT + 16 * i + n) * 2] = m[i];
            lm[(wave * RT + 16 * i + n) * 2 + 1] = sum;
        }
    }
    __syncthreads();
    // four coordinates of a row per thread
    for (int j = threadIdx.x; j < RT * (D / 4); j += 64 * W) {
        const int tr = j / (D / 4), d = (j % (D / 4)) * 4, r = r0 + tr;
        if (r >= rows) continue;
        float mt = -__builtin_inff();
        for (int w = 0; w < W; ++w) mt = fmaxf(mt, lm[(w * RT + tr) * 2]);
        const float mm = mt == -__builtin_inff() ? 0.f : mt;
        float sum = 0.f;
        f32x4 ot = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < W; ++w) {
            const float e = __builtin_amdgcn_exp2f(lm[(w * RT + tr) * 2] - mm);
            sum += e * lm[(w * RT + tr) * 2 + 1];
            ot += e * *reinterpret_cast<const f32x4 *>(lds + ((w * RT + tr) * OS + d));
        }
        const int64_t at = (int64_t)(first + r / a.group) * a.heads + kvh * a.group + r % a.group;
        if (a.chunks > 1) {
            *reinterpret_cast<f32x4 *>(a.part + (at * a.chunks + chunk) * D + d) = ot;
            if (d == 0) {
                float *pm = a.part + ((int64_t)a.set.total * a.heads * a.chunks * D + (at * a.chunks + chunk) * 2);
                pm[0] = mt;
                pm[1] = sum;
            }
        } else {
            const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
            unsigned short h[4];
            for (int k = 0; k < 4; ++k) h[k] = float_bits16(ot[k] * inv, a.bf16);
            uint2 u;
            __builtin_memcpy(&u, h, 8);
            *reinterpret_cast<uint2 *>(static_cast<unsigned short *>(a.out) + at * D + d) = u;
            if (a.lse && d == 0) a.lse[at] = sum == 0.f ? -__builtin_inff() : (mt + __log2f(sum)) * 0.69314718056f;
        }
    }
}

// Joins the parts of a (token, head): W waves, each takes every W-th part.
template <int D, int W>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
    constexpr int N = D / 64;
    __shared__ float lds[W > 1 ? W * (D + 1) : 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t at = W > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (at >= (int64_t)a.set.total * a.heads) return;
    const int token = (int)(at / a.heads);
    int row = token, first = token, count = 1;
    if (a.set.starts) {
        row = slot_row(a.set.starts, a.set.rows, token, 1, 1, 0);
        row_tokens(a.set.starts, row, a.set.total, &first, &count);
    }
    const int true_len = a.set.lens[row];
    const int len = min(true_len, a.limit);
    const int pos = min(true_len - count + (token - first), len - 1);
    // parts that hold tokens this query sees
    const int parts = pos < 0 ? 0 : pos / (a.chunk_pages * kPage) + 1;
    const float *po = a.part + at * a.chunks * D;
    const float *pm = a.part + ((int64_t)a.set.total * a.heads * D + at * 2) * a.chunks;
    float m = -__builtin_inff();
    for (int c = lane; c < parts; c += 64) m = fmaxf(m, pm[2 * c]);
    for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    const float mm = m == -__builtin_inff() ? 0.f : m;
    float l = 0.f, o[N];
    for (int j = 0; j < N; ++j) o[j] = 0.f;
#pragma unroll 4
    for (int c = W > 1 ? wave : 0; c < parts; c += W) {
        const float e = __builtin_amdgcn_exp2f(pm[2 * c] - mm);
        l += e * pm[2 * c + 1];
        for (int j = 0; j < N; ++j) o[j] += e * po[(int64_t)c * D + j * 64 + lane];
    }
    if constexpr (W > 1) {
        for (int j = 0; j < N; ++j) lds[wave * (D + 1) + j * 64 + lane] = o[j];
        if (lane == 0) lds[wave * (D + 1) + D] = l;
        __syncthreads();
        if (wave > 0) return;
        for (int w = 1; w < W; ++w) {
            for (int j = 0; j < N; ++j) o[j] += lds[w * (D + 1) + j * 64 + lane];
            l += lds[w * (D + 1) + D];
        }
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    for (int j = 0; j < N; ++j)
        static_cast<unsigned short *>(a.out)[at * D + j * 64 + lane] = float_bits16(o[j] * inv, a.bf16);
    if (a.lse && lane == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.69314718056f;
}

template <int D, bool FP8, int NT, int W>
hipError_t launch(const AttendArgs &a, hipStream_t stream) {
    constexpr int RT = 16 * NT;
    constexpr size_t lds = sizeof(float) * W * RT * (D + 4 + 2);
    if (lds > 65536) {
        static const hipError_t once = hipFuncSetAttribute(
            reinterpret_cast<const void *>(attend_kernel<D, FP8, NT, W>),
            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (once != hipSuccess) return once;
    }
    const int64_t slots = a.set.starts ? (int64_t)a.set.total * a.group / RT + a.set.rows
                                       : (int64_t)a.set.rows * ((a.group + RT - 1) / RT);
    attend_kernel<D, FP8, NT, W><<<dim3((unsigned)(slots * a.chunks), (unsigned)a.layer.heads), 64 * W, lds, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.chunks == 1) return e;
    const int64_t outs = (int64_t)a.set.total * a.heads;
    // many parts of few results: four waves each
    if (a.chunks > 8) join_kernel<D, 4><<<(unsigned)outs, 256, 0, stream>>>(a);
    else join_kernel<D, 1><<<(unsigned)((outs + 3) / 4), 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D, bool FP8>
hipError_t pick(const AttendArgs &a, const AttendPlan &p, hipStream_t stream) {
    if constexpr (D < 256) {   // at 256 neither fits the registers
        if (p.waves == 8) return launch<D, FP8, 1, 8>(a, stream);
        if (p.tile == 32) return launch<D, FP8, 2, 4>(a, stream);
    }
    return launch<D, FP8, 1, 4>(a, stream);
}

}  // namespace

AttendPlan attend_plan(int64_t n, int rows, int group, int kv_heads, int width, int longest, int D) {
    AttendPlan p;
    const int64_t tokens = (int64_t)width * kPage;
    const int64_t len = longest > 0 && longest < tokens ? longest : tokens;
    const int pages = (int)((len + kPage - 1) / kPage);
    // query rows of one key head and table row, on average
    const int64_t mean = (n * group + rows - 1) / rows;
    p.tile = mean > 16 && D < 256 ? 32 : 16;
    const int64_t units = ((n * group) / p.tile + rows) * kv_heads;
    p.waves = p.tile == 16 && D < 256 && pages <= WHOLE ? 8 : 4;
    int64_t each = pages <= WHOLE ? pages : pages * units / WANT;
    if (each < 8) each = 8;
    if (each > 64) each = 64;
    p.chunk_pages = (int)each;
    p.chunks = pages > 0 ? (int)((pages + each - 1) / each) : 1;
    return p;
}

size_t attend_part_bytes(const AttendPlan &p, int64_t n, int heads, int D) {
    return p.chunks > 1 ? sizeof(float) * (size_t)n * heads * p.chunks * (D + 2) : 0;
}

hipError_t kv_attend(const AttendArgs &a, const AttendPlan &p, int D, int type, hipStream_t stream) {
    const bool f = type == TQ_KV_FP8;
    if (D == 64) return f ? pick<64, true>(a, p, stream) : pick<64, false>(a, p, stream);
    if (D == 128) return f ? pick<128, true>(a, p, stream) : pick<128, false>(a, p, stream);
    return f ? pick<256, true>(a, p, stream) : pick<256, false>(a, p, stream);
}

}  // namespace tq
