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
// rounds away is 2^-39 of it.  Weights are rounded to float16 in units of
// 2^-kUnit and of a power of two no smaller than the value scales seen so far, which
// keeps 11 bits down to 2^-20 of the largest weight.
#include <hip/hip_runtime.h>

#include "kv.h"

namespace tq {
namespace {

constexpr int kUnit = 6;          // weights are at most 2^kUnit in float16
constexpr int kNoScale = -4096;   // exponent of "no value scale yet"

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

// What a wave has of a tile of 16 query rows after some pages.
template <int D>
struct Part {
    float m, l;                 // running maximum (log2 units) and the lane's share of the sum
    f32x4 o[D / 16];            // in units of 2^-kUnit 2^k of the wave
};

// The query rows of a tile and their position limits.
struct Tile {
    int row, kvh;               // row of the table, key head
    int first, count;           // its new tokens in the packed tensor
    int len;
    int r0;                     // first (token, head) row of the tile within the row's
};

// NT tiles of 16 query rows per wave.  APART: every wave has rows of its own
// and walks all pages of the part; else the four waves share the rows, take
// every fourth page, and are joined through LDS.
template <int D, bool FP8, int NT, bool APART>
__global__ __launch_bounds__(256) void attend_kernel(AttendArgs a) {
    constexpr int KS = D / 32;                       // 32-wide steps of the first product
    constexpr int DT = D / 16;
    constexpr int RW = 16 * NT;                      // rows of a wave
    constexpr int RT = APART ? 4 * RW : RW;          // rows of the workgroup
    extern __shared__ __align__(16) float lds[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int n = lane & 15, g = lane >> 4;

    Tile t;
    int64_t slot = blockIdx.x / a.chunks;
    const int chunk = blockIdx.x % a.chunks;
    t.kvh = blockIdx.y;
    if (a.set.starts) {
        t.row = slot_row(a.set.starts, a.set.rows, slot, a.group, RT, 1);
        slot -= slot_begin(a.set.starts, t.row, a.group, RT, 1);
    } else {   // one token per row: its group in ceil(group / RT) tiles
        const int per = (a.group + RT - 1) / RT;
        t.row = (int)(slot / per);
        slot %= per;
    }
    row_tokens(a.set.starts, t.row, a.set.total, &t.first, &t.count);
    const int rows = t.count * a.group;
    if (slot < 0 || slot * RT >= rows) return;       // the whole workgroup
    t.r0 = (int)slot * RT + (APART ? wave * RW : 0);
    const int true_len = a.set.lens[t.row];
    t.len = min(true_len, a.limit);

    // queries: rows r0 + 16 i + n, 8 coordinates (ks/2) 64 + g 16 + (ks%2) 8 of each step
    f16x8 q[NT][KS];
    float factor[NT];
    int pos[NT];
    int top = -1;                                    // last position any row of the wave sees
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const int r = t.r0 + 16 * i + n;
        const bool in = r < rows;
        const int token = in ? r / a.group : 0, head = t.kvh * a.group + (in ? r % a.group : 0);
        pos[i] = in ? min(true_len - t.count + token, t.len - 1) : -1;
        float x[KS][8];
        float big = 0.f;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            if (in) load8(a.q, (t.first + token) * a.qt + head * a.qh + (s >> 1) * 64 + g * 16 + (s & 1) * 8, a.bf16, a.wide, x[s]);
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
#pragma unroll
        for (int s = 0; s < KS; ++s)
            for (int j = 0; j < 8; ++j) q[i][s][j] = (_Float16)ldexpf(x[s][j], e);
        factor[i] = ldexpf(a.scale2, -e);
        top = max(top, pos[i]);
    }
    for (int m = 1; m < 16; m <<= 1) top = max(top, __shfl_xor(top, m));
    top = __builtin_amdgcn_readfirstlane(top);

    Part<D> part[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        part[i].m = -__builtin_inff();
        part[i].l = 0.f;
        for (int d = 0; d < DT; ++d) part[i].o[d] = {0.f, 0.f, 0.f, 0.f};
    }
    int unit = kNoScale;                             // the wave's value unit 2^unit

    const int page_end = min(top / kPage + 1, (chunk + 1) * a.chunk_pages);
    const int step = APART ? 1 : 4;
    const int *table = a.set.tables + (int64_t)t.row * a.set.width;
    for (int p = top < 0 ? page_end : chunk * a.chunk_pages + (APART ? 0 : wave); p < page_end; p += step) {
        const int page = __builtin_amdgcn_readfirstlane(table[p]);
        if (page < 0 || page >= a.layer.pages) {
            if (a.layer.status && lane == 0) atomicOr(a.layer.status, TQ_KV_BAD_PAGE);
            continue;
        }
        const int64_t tile = (int64_t)page * a.layer.heads + t.kvh;
        const char *kp = a.layer.k + tile * (kPage * D);
        const char *vp = a.layer.v + tile * (kPage * D);
        const float ks = a.layer.ks[tile * 4 + g];
        float vs = a.layer.vs[tile * 4 + g];
        uint4 kc[4][D / 64], vc[DT];
        const int krow = (16 * (n >> 2) + (n & 3)) * D + g * 16;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int u = 0; u < D / 64; ++u)
                kc[s][u] = *reinterpret_cast<const uint4 *>(kp + krow + 4 * s * D + u * 64);
#pragma unroll
        for (int d = 0; d < DT; ++d)
            vc[d] = *reinterpret_cast<const uint4 *>(vp + (g * D + d * 16 + n) * 16);

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
        const int base = p * kPage + 16 * g;         // position of the lane's first token
        // A page that holds the row's end may hold anything past it: those
        // codes and scales are taken out before they meet a zero weight.
        if ((p + 1) * kPage > t.len) {
            const int left = min(max(t.len - base, 0), 16);
            if (left == 0) vs = 0.f;
#pragma unroll
            for (int d = 0; d < DT; ++d) vc[d] = keep_tokens(vc[d], left);
        }
        // the value unit: a power of two above every scale so far
        int ve;
        frexpf(vs, &ve);
        ve = vs > 0.f ? ve : kNoScale;
        const int v01 = max(__builtin_amdgcn_readlane(ve, 0), __builtin_amdgcn_readlane(ve, 16));
        const int v23 = max(__builtin_amdgcn_readlane(ve, 32), __builtin_amdgcn_readlane(ve, 48));
        const int higher = max(unit, max(v01, v23));
        const float lower = unit == kNoScale ? 0.f : ldexpf(1.f, unit - higher);
        const float vn = ldexpf(vs, -higher);
        const bool moved = higher > unit;
        unit = higher;

        f16x8 w[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            const float f = factor[i] * ks;
            float y[16], big = -__builtin_inff();
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float z = x[i][s][r] * f;
                    if (base + 4 * s + r > pos[i]) z = -__builtin_inff();
                    y[4 * s + r] = z;
                    big = fmaxf(big, z);
                }
            const float m = fmaxf(part[i].m, max_of_groups(big));
            const float mm = m == -__builtin_inff() ? 0.f : m;
            const float alpha = __builtin_amdgcn_exp2f(part[i].m - mm);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float e = __builtin_amdgcn_exp2f(y[j] - mm);
                sum += e;
                w[i][j >> 3][j & 7] = (_Float16)(e * vn * (float)(1 << kUnit));
            }
            part[i].l = part[i].l * alpha + sum;
            if (moved || __any(m > part[i].m)) {
                const float both = alpha * lower;
                for (int d = 0; d < DT; ++d) part[i].o[d] *= both;
            }
            part[i].m = m;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            f16x8 lo, hi;
            to_half<FP8>(vc[d], &lo, &hi);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                part[i].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, w[i][0], part[i].o[d], 0, 0, 0);
                part[i].o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, w[i][1], part[i].o[d], 0, 0, 0);
            }
        }
    }

    const float back = unit == kNoScale ? 0.f : ldexpf(1.f, unit - kUnit);
    constexpr int OS = D + 4;                        // LDS row, off the banks' period
    float *lo = lds, *lm = lds + (APART ? 0 : 4 * RW * OS);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        const float l = sum_of_groups(part[i].l), m = part[i].m;
        if constexpr (!APART) {
            for (int d = 0; d < DT; ++d) {
                f32x4 o = part[i].o[d] * back;
                *reinterpret_cast<f32x4 *>(lo + ((wave * RW + 16 * i + n) * OS + d * 16 + g * 4)) = o;
            }
            if (g == 0) {
                lm[(wave * RW + 16 * i + n) * 2] = m;
                lm[(wave * RW + 16 * i + n) * 2 + 1] = l;
            }
        } else {
            const int r = t.r0 + 16 * i + n;
            if (r >= rows) continue;
            const int64_t at = (int64_t)(t.first + r / a.group) * a.heads + t.kvh * a.group + r % a.group;
            if (a.chunks > 1) {
                float *po = a.part + (at * a.chunks + chunk) * D;
                for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4 *>(po + d * 16 + g * 4) = part[i].o[d] * back;
                if (g == 0) {
                    float *pm = a.part + ((int64_t)a.set.total * a.heads * a.chunks * D + (at * a.chunks + chunk) * 2);
                    pm[0] = m;
                    pm[1] = l;
                }
            } else {
                const float inv = l > 0.f || l != l ? back / l : 0.f;
                for (int d = 0; d < DT; ++d) {
                    unsigned short h[4];
                    for (int j = 0; j < 4; ++j) h[j] = float_bits16(part[i].o[d][j] * inv, a.bf16);
                    uint2 u;
                    __builtin_memcpy(&u, h, 8);
                    *reinterpret_cast<uint2 *>(static_cast<unsigned short *>(a.out) + at * D + d * 16 + g * 4) = u;
                }
                if (a.lse && g == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.69314718056f;
            }
        }
    }
    if constexpr (!APART) {
        __syncthreads();
        // four coordinates of a row per thread
        for (int j = threadIdx.x; j < RW * (D / 4); j += 256) {
            const int row = j / (D / 4), d = (j % (D / 4)) * 4, r = t.r0 + row;
            if (r >= rows) continue;
            float m = -__builtin_inff();
            for (int w = 0; w < 4; ++w) m = fmaxf(m, lm[(w * RW + row) * 2]);
            const float mm = m == -__builtin_inff() ? 0.f : m;
            float l = 0.f;
            f32x4 o = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < 4; ++w) {
                const float e = __builtin_amdgcn_exp2f(lm[(w * RW + row) * 2] - mm);
                l += e * lm[(w * RW + row) * 2 + 1];
                o += e * *reinterpret_cast<const f32x4 *>(lo + ((w * RW + row) * OS + d));
            }
            const int64_t at = (int64_t)(t.first + r / a.group) * a.heads + t.kvh * a.group + r % a.group;
            if (a.chunks > 1) {
                *reinterpret_cast<f32x4 *>(a.part + (at * a.chunks + chunk) * D + d) = o;
                if (d == 0) {
                    float *pm = a.part + ((int64_t)a.set.total * a.heads * a.chunks * D + (at * a.chunks + chunk) * 2);
                    pm[0] = m;
                    pm[1] = l;
                }
            } else {
                const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
                unsigned short h[4];
                for (int k = 0; k < 4; ++k) h[k] = float_bits16(o[k] * inv, a.bf16);
                uint2 u;
                __builtin_memcpy(&u, h, 8);
                *reinterpret_cast<uint2 *>(static_cast<unsigned short *>(a.out) + at * D + d) = u;
                if (a.lse && d == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.69314718056f;
            }
        }
    }
}

// Joins the parts of a row: a wave per (token, head).
template <int D>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
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
    constexpr int N = D / 64;
    float l = 0.f, o[N];
    for (int j = 0; j < N; ++j) o[j] = 0.f;
    for (int c = 0; c < parts; ++c) {
        const float e = __builtin_amdgcn_exp2f(pm[2 * c] - mm);
        l += e * pm[2 * c + 1];
        for (int j = 0; j < N; ++j) o[j] += e * po[(int64_t)c * D + j * 64 + lane];
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    for (int j = 0; j < N; ++j)
        static_cast<unsigned short *>(a.out)[at * D + j * 64 + lane] = float_bits16(o[j] * inv, a.bf16);
    if (a.lse && lane == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.69314718056f;
}

template <int D, bool FP8, int NT, bool APART>
hipError_t launch(const AttendArgs &a, hipStream_t stream) {
    constexpr int RW = 16 * NT, RT = APART ? 4 * RW : RW;
    const size_t lds = APART ? 0 : sizeof(float) * 4 * RW * (D + 4 + 2);
    if (lds > 65536) {
        static const hipError_t once = hipFuncSetAttribute(
            reinterpret_cast<const void *>(attend_kernel<D, FP8, NT, APART>),
            hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (once != hipSuccess) return once;
    }
    const int64_t slots = a.set.starts ? (int64_t)a.set.total * a.group / RT + a.set.rows
                                       : (int64_t)a.set.rows * ((a.group + RT - 1) / RT);
    attend_kernel<D, FP8, NT, APART><<<dim3((unsigned)(slots * a.chunks), (unsigned)a.layer.heads), 256, lds, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.chunks == 1) return e;
    join_kernel<D><<<(unsigned)(((int64_t)a.set.total * a.heads + 3) / 4), 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D, bool FP8>
hipError_t pick(const AttendArgs &a, const AttendPlan &p, hipStream_t stream) {
    if (p.rows_apart) return launch<D, FP8, 2, true>(a, stream);
    return p.tile == 16 ? launch<D, FP8, 1, false>(a, stream) : launch<D, FP8, 2, false>(a, stream);
}

}  // namespace

AttendPlan attend_plan(int64_t n, int rows, int group, int kv_heads, int width, int longest, int D) {
    AttendPlan p;
    const int64_t tokens = (int64_t)width * kPage;
    const int64_t len = longest > 0 && longest < tokens ? longest : tokens;
    const int pages = (int)((len + kPage - 1) / kPage);
    // query rows of one key head and table row, on average
    const int64_t mean = (n * group + rows - 1) / rows;
    p.rows_apart = mean > 64;
    p.tile = p.rows_apart ? 128 : mean > 16 ? 32 : 16;
    const int64_t units = ((n * group) / p.tile + rows) * kv_heads;
    const int64_t want = 2048;
    int64_t chunks = (want + units - 1) / units;
    int each = (int)((pages + chunks - 1) / chunks);
    if (each < 4) each = 4;
    p.chunk_pages = each;
    p.chunks = pages > 0 ? (pages + each - 1) / each : 1;
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
