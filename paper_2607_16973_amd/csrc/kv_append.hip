// Appending keys and values to the 8-bit cache.
//
// A wave holds one block -- 16 tokens of one head, keys or values -- so that
// the block's scale, its old codes and its new ones have one owner and no
// atomics: amax over the new values (finite ones), s1 = max(s0, amax * (1 / qmax)),
// new codes round(x / s1), and the old ones brought to s1 where it grew.
// A key wave's lane has 8 coordinates of every (512 / D)-th token, so that its
// codes are a piece of a key row; a value wave's lane has all 16 tokens (8 at
// D = 64) of 2 or 4 coordinates, so that its codes are the store's
// tokens-innermost lines and nothing needs transposing.  amax is taken of
// the 16-bit values as integers, two at a time; a finite value needs no
// clamp then, and int8 rounding is one addition of 1.5 2^23.  Blocks with
// values that are not finite take the long way.
// Bound by memory: 2 bytes read and 1 written per element, plus one block of
// old value codes per row and head.  Measured: 16.6 us for 13,600 tokens of 8 heads,
// d = 128, float16 to e4m3 (5.0 TB/s, the rate of a large copy); 6 us, all of it latency, for
// one token of each of 64 rows.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "kv.h"

namespace tq {
namespace {

constexpr float kTiny = 0x1p-100f;   // amax below this counts as zero: 1 / s1 stays finite

template <bool FP8>
__device__ inline float code_top() {
    return FP8 ? 448.f : 127.f;
}

// x * r as a code, in the low byte (int8) or as the float to convert (e4m3).
// SAFE: x is finite and |x| r at most qmax up to rounding.
template <bool FP8, bool SAFE>
__device__ inline float code_of(float x, float r) {
#pragma clang fp contract(off)
    float z = x * r;
    if constexpr (!SAFE) {
        z = z != z ? 0.f : z;
        z = fminf(fmaxf(z, -code_top<FP8>()), code_top<FP8>());
    }
    if constexpr (FP8) return __builtin_amdgcn_fmed3f(z, -448.f, 448.f);
    else return z + 12582912.f;      // rounds to an integer, ties to even, in the low bits
}
template <bool FP8>
__device__ inline uint32_t pack4(float a, float b, float c, float d) {
    if constexpr (FP8) {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x0c0c0400u);
        const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d), __float_as_uint(c), 0x04000c0cu);
        return lo | hi;
    }
}
template <bool FP8>
__device__ inline void unpack4(uint32_t w, float *x) {
    if constexpr (FP8) {
        const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
        const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        x[0] = lo.x, x[1] = lo.y, x[2] = hi.x, x[3] = hi.y;
    } else {
        for (int j = 0; j < 4; ++j) x[j] = (float)((int)(w << (24 - 8 * j)) >> 24);
    }
}
// Old codes of a word under a grown scale: round(z * s0/s1).
template <bool FP8>
__device__ inline uint32_t shrink4(uint32_t w, float ratio) {
    float x[4];
    unpack4<FP8>(w, x);
    for (int j = 0; j < 4; ++j) x[j] = code_of<FP8, false>(x[j], ratio);
    return pack4<FP8>(x[0], x[1], x[2], x[3]);
}
__device__ inline float low_half(uint32_t w, int bf16) { return bf16 ? __uint_as_float(w << 16) : f16_float((unsigned short)w); }
__device__ inline float high_half(uint32_t w, int bf16) {
    return bf16 ? __uint_as_float(w & 0xffff0000u) : f16_float((unsigned short)(w >> 16));
}
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
// The larger of two magnitudes as integers, in both halves of a word.
__device__ inline uint32_t max_bits(uint32_t a, uint32_t w) {
    const u16x2 x = __builtin_bit_cast(u16x2, a), y = __builtin_bit_cast(u16x2, w & 0x7fff7fffu);
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(x, y));
}

// Words of N 16-bit values of a row.
template <int N>
__device__ inline void load_words(const void *row, int64_t at, int wide, uint32_t *w) {
    const unsigned short *p = static_cast<const unsigned short *>(row) + at;
    if (wide) {
        __builtin_memcpy(w, __builtin_assume_aligned(p, 2 * N), 2 * N);
    } else {
        for (int j = 0; j < N / 2; ++j) w[j] = p[2 * j] | (uint32_t)p[2 * j + 1] << 16;
    }
}

// The block's scale from the magnitudes in `bits` (two halves) and the words x[0..n).
struct Scaling {
    float s1, r, ratio;
    bool grown, safe;                // safe: all new values are finite
};
template <bool FP8, int N>
__device__ inline Scaling rescale(const AppendArgs &a, const uint32_t *x, float s0, int c, int lane) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) bits = max_bits(bits, x[i]);
    uint32_t top = max(bits & 0xffffu, bits >> 16);
    for (int m = 32; m; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
    Scaling s;
    s.safe = top < (a.bf16 ? 0x7f80u : 0x7c00u);
    float amax = low_half(top, a.bf16);
    if (!s.safe) {
        amax = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float lo = fabsf(low_half(x[i], a.bf16)), hi = fabsf(high_half(x[i], a.bf16));
            if (lo < __builtin_inff()) amax = fmaxf(amax, lo);
            if (hi < __builtin_inff()) amax = fmaxf(amax, hi);
        }
        for (int m = 32; m; m >>= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
        if (a.layer.status && lane == 0) atomicOr(a.layer.status, TQ_KV_NONFINITE);
    }
    s.s1 = fmaxf(s0, amax < kTiny ? 0.f : amax * (1.f / code_top<FP8>()));
    s.r = s.s1 > 0.f ? 1.f / s.s1 : 0.f;
    s.grown = c > 0 && s.s1 > s0;
    s.ratio = s.grown ? s0 / s.s1 : 1.f;
    return s;
}

// A block's place: tokens [c, e) of it are new, the first of them is number
// `token` of the packed tensor.
struct Block {
    int64_t token;
    int c, e;
    char *store;
    float *scale;
};

template <int D, bool FP8>
__device__ inline void append_keys(const AppendArgs &a, const Block &b, int head, int lane) {
    constexpr int LT = D / 8;         // lanes of one token
    constexpr int TP = 64 / LT;       // tokens of one pass
    constexpr int NP = kBlock / TP;   // passes
    const int t0 = lane / LT, e0 = (lane % LT) * 8;
    uint32_t x[NP * 4];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int t = p * TP + t0;
        if (t >= b.c && t < b.e) load_words<8>(a.k, (b.token + t - b.c) * a.kt + head * a.kh + e0, a.wide, x + 4 * p);
        else x[4 * p] = x[4 * p + 1] = x[4 * p + 2] = x[4 * p + 3] = 0;
    }
    const Scaling s = rescale<FP8, NP * 4>(a, x, b.c > 0 ? *b.scale : 0.f, b.c, lane);
    auto put = [&](auto safe) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int t = p * TP + t0;
            float z[8];
            for (int j = 0; j < 4; ++j) {
                z[2 * j] = code_of<FP8, decltype(safe)::value>(low_half(x[4 * p + j], a.bf16), s.r);
                z[2 * j + 1] = code_of<FP8, decltype(safe)::value>(high_half(x[4 * p + j], a.bf16), s.r);
            }
            uint2 *to = reinterpret_cast<uint2 *>(b.store + t * D + e0);
            if (t >= b.c && (t < b.e || b.c == 0)) {   // past e: zeros
                *to = make_uint2(pack4<FP8>(z[0], z[1], z[2], z[3]), pack4<FP8>(z[4], z[5], z[6], z[7]));
            } else if (s.grown) {                      // also what a retreat left past e
                const uint2 o = *to;
                *to = make_uint2(shrink4<FP8>(o.x, s.ratio), shrink4<FP8>(o.y, s.ratio));
            }
        }
    };
    if (s.safe) put(std::true_type());
    else put(std::false_type());
    if (lane == 0) *b.scale = s.s1;
}

template <int D, bool FP8>
__device__ inline void append_values(const AppendArgs &a, const Block &b, int head, int lane) {
    constexpr int E = D == 256 ? 4 : 2;              // coordinates of a lane
    constexpr int T = D == 64 ? 8 : 16;              // tokens of a lane
    const int d0 = lane % (D / E) * E, t0 = lane / (D / E) * T;
    uint32_t x[T * (E / 2)];
#pragma unroll
    for (int i = 0; i < T; ++i) {
        const int t = t0 + i;
        if (t >= b.c && t < b.e) load_words<E>(a.v, (b.token + t - b.c) * a.vt + head * a.vh + d0, a.wide, x + i * (E / 2));
        else for (int j = 0; j < E / 2; ++j) x[i * (E / 2) + j] = 0;
    }
    // the lines of T codes that are there: coordinate d0 + e
    uint32_t old[E][T / 4];
    uint32_t *line = reinterpret_cast<uint32_t *>(b.store + d0 * kBlock + t0);
#pragma unroll
    for (int e = 0; e < E; ++e)
        for (int q = 0; q < T / 4; ++q) old[e][q] = b.c > 0 ? line[e * (kBlock / 4) + q] : 0;
    const Scaling s = rescale<FP8, T * (E / 2)>(a, x, b.c > 0 ? *b.scale : 0.f, b.c, lane);
    auto put = [&](auto safe) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            uint32_t w[T / 4];
#pragma unroll
            for (int q = 0; q < T / 4; ++q) {
                float z[4];
                for (int j = 0; j < 4; ++j) {
                    const uint32_t u = x[(4 * q + j) * (E / 2) + e / 2];
                    z[j] = code_of<FP8, decltype(safe)::value>(e & 1 ? high_half(u, a.bf16) : low_half(u, a.bf16), s.r);
                }
                w[q] = pack4<FP8>(z[0], z[1], z[2], z[3]);
                if (b.c > 0) {       // the bytes of the new tokens among the old ones
                    const int lo = min(max(b.c - t0 - 4 * q, 0), 4), hi = min(max(b.e - t0 - 4 * q, 0), 4);
                    const uint32_t m = hi > lo ? (~0u >> (32 - 8 * (hi - lo))) << (8 * lo) : 0u;
                    const uint32_t o = s.grown ? shrink4<FP8>(old[e][q], s.ratio) : old[e][q];
                    w[q] = (w[q] & m) | (o & ~m);
                }
            }
            if constexpr (T == 16) *reinterpret_cast<uint4 *>(line + e * (kBlock / 4)) = make_uint4(w[0], w[1], w[2], w[3]);
            else *reinterpret_cast<uint2 *>(line + e * (kBlock / 4)) = make_uint2(w[0], w[1]);
        }
    };
    if (s.safe) put(std::true_type());
    else put(std::false_type());
    if (lane == 0) *b.scale = s.s1;
}

template <int D, bool FP8>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int item = blockIdx.y * 4 + wave;           // (head, keys or values)
    const RowSet &set = a.set;
    const int heads = a.layer.heads;

    // the block: row, first and one-past-last new position inside it
    int row, first, count;
    int64_t local;
    if (set.starts) {
        row = slot_row(set.starts, set.rows, blockIdx.x, 1, kBlock, 2);
        local = (int64_t)blockIdx.x - slot_begin(set.starts, row, 1, kBlock, 2);
    } else {
        row = blockIdx.x;
        local = 0;
    }
    row_tokens(set.starts, row, set.total, &first, &count);
    const int true_len = row_length(set.lens, row), len = min(true_len, set.width * kPage);
    const int begin = true_len - count;                // position of the first new token
    if (local < 0 || local > count / kBlock + 1) return;   // the whole workgroup
    const int blk = max(begin, 0) / kBlock + (int)local;
    const int lo = max(begin, blk * kBlock), hi = min(len, (blk + 1) * kBlock);
    if (count == 0 || lo >= hi) return;
    const int page = set.tables[(int64_t)row * set.width + blk / 4];
    if (page < 0 || page >= a.layer.pages) {
        if (a.layer.status && threadIdx.x == 0 && blockIdx.y == 0) atomicOr(a.layer.status, TQ_KV_BAD_PAGE);
        return;
    }
    if (item >= 2 * heads) return;
    const int head = item >> 1;
    const bool val = item & 1;
    const int64_t tile = (int64_t)page * heads + head;
    Block b;
    b.token = first + (lo - begin);
    b.c = lo - blk * kBlock;
    b.e = hi - blk * kBlock;
    b.store = (val ? a.layer.v : a.layer.k) + tile * (kPage * D) + (int64_t)(blk & 3) * (kBlock * D);
    b.scale = (val ? a.layer.vs : a.layer.ks) + tile * 4 + (blk & 3);
    if (val) append_values<D, FP8>(a, b, head, lane);
    else append_keys<D, FP8>(a, b, head, lane);
}

template <int D>
hipError_t launch(const AppendArgs &a, int type, dim3 grid, hipStream_t stream) {
    if (type == TQ_KV_FP8) append_kernel<D, true><<<grid, 256, 0, stream>>>(a);
    else append_kernel<D, false><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t kv_append(const AppendArgs &a, int D, int type, hipStream_t stream) {
    // a row of n tokens touches at most n / 16 + 2 blocks
    const int64_t slots = a.set.starts ? (int64_t)a.set.total / kBlock + 2 * (int64_t)a.set.rows : a.set.rows;
    const dim3 grid((unsigned)slots, (unsigned)((2 * a.layer.heads + 3) / 4));
    return D == 64 ? launch<64>(a, type, grid, stream) : D == 128 ? launch<128>(a, type, grid, stream)
                                                                  : launch<256>(a, type, grid, stream);
}

}  // namespace tq
