// Appending keys and values to the 8-bit cache.
//
// A wave holds one block -- 16 tokens of one head, keys or values -- so that
// the block's scale, its old codes and its new ones have one owner and no
// atomics: amax over the new values (finite ones), s1 = max(s0, amax * (1 / qmax)),
// new codes round(x / s1), and the old ones brought to s1 where it grew.
// Lane l holds the 8 elements (l mod D/8) * 8 .. + 7 of the tokens l / (D/8),
// + 512/D, ...: a wave's loads take whole rows of the head.  The value
// store wants a block's tokens innermost, so codes pass through LDS once.
// Bound by memory: 2 bytes read and 1 written per element, plus one block of
// old value codes per row and head.
#include <hip/hip_runtime.h>

#include "kv.h"

namespace tq {
namespace {

constexpr float kTiny = 0x1p-100f;   // amax below this counts as zero: 1 / s1 stays finite

template <bool FP8>
__device__ inline float code_top() {
    return FP8 ? 448.f : 127.f;
}

// round(clamp(z)) as float32, NaN as 0: what is packed next is exact (int8)
// or rounded once (e4m3).
template <bool FP8>
__device__ inline float clamp_code(float z) {
    z = z != z ? 0.f : z;
    z = fminf(fmaxf(z, -code_top<FP8>()), code_top<FP8>());
    return FP8 ? z : rintf(z);
}
template <bool FP8>
__device__ inline uint32_t pack4(float a, float b, float c, float d) {
    if constexpr (FP8) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    } else {
        return ((uint32_t)(int)a & 255u) | (((uint32_t)(int)b & 255u) << 8) |
               (((uint32_t)(int)c & 255u) << 16) | ((uint32_t)(int)d << 24);
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
    for (int j = 0; j < 4; ++j) x[j] = clamp_code<FP8>(x[j] * ratio);
    return pack4<FP8>(x[0], x[1], x[2], x[3]);
}

template <int D, bool FP8>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a) {
    constexpr int LT = D / 8;         // lanes of one token
    constexpr int TP = 64 / LT;       // tokens of one pass
    constexpr int NP = kBlock / TP;   // passes
    __shared__ __align__(16) uint8_t codes[4][kBlock * D];

    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int item = blockIdx.y * 4 + wave;           // (head, keys or values)
    const RowSet &set = a.set;
    const int heads = a.layer.heads;
    const bool active = item < 2 * heads;
    const int head = active ? item >> 1 : 0;
    const bool val = item & 1;

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
    const int len = min(set.lens[row], set.width * kPage);
    const int begin = set.lens[row] - count;           // position of the first new token
    if (local < 0 || local > count / kBlock + 1) return;   // the whole workgroup
    const int blk = max(begin, 0) / kBlock + (int)local;
    const int lo = max(begin, blk * kBlock), hi = min(len, (blk + 1) * kBlock);
    if (count == 0 || lo >= hi) return;
    const int page = set.tables[(int64_t)row * set.width + blk / 4];
    if (page < 0 || page >= a.layer.pages) {
        if (a.layer.status && threadIdx.x == 0 && blockIdx.y == 0) atomicOr(a.layer.status, TQ_KV_BAD_PAGE);
        return;
    }
    if (!active) return;
    const int c = max(begin - blk * kBlock, 0);        // tokens of the block there before
    const int e = hi - blk * kBlock;
    const int sub = blk & 3;

    const void *src = val ? a.v : a.k;
    const int64_t st = val ? a.vt : a.kt, sh = val ? a.vh : a.kh;
    const int64_t tile = (int64_t)page * heads + head;
    char *store = (val ? a.layer.v : a.layer.k) + tile * (kPage * D) + (int64_t)sub * (kBlock * D);
    float *scale = (val ? a.layer.vs : a.layer.ks) + tile * 4 + sub;

    const int t0 = lane / LT, e0 = (lane % LT) * 8;
    float x[NP][8];
    bool odd = false;
    float amax = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int t = p * TP + t0;
        if (t >= c && t < e) {
            const int64_t token = first + (blk * kBlock + t - begin);
            load8(src, token * st + head * sh + e0, a.bf16, a.wide, x[p]);
        } else {
            for (int j = 0; j < 8; ++j) x[p][j] = 0.f;
        }
    }
    // old value codes: D / 64 tokens-innermost lines of 16 bytes per lane
    uint4 old[D / 64];
#pragma unroll
    for (int i = 0; i < D / 64; ++i)
        old[i] = c > 0 && val ? reinterpret_cast<const uint4 *>(store)[i * 64 + lane] : make_uint4(0, 0, 0, 0);
    const float s0 = c > 0 ? *scale : 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p)
        for (int j = 0; j < 8; ++j) {
            const float y = fabsf(x[p][j]);
            const bool fin = y < __builtin_inff();
            odd |= !fin;
            amax = fmaxf(amax, fin ? y : 0.f);
        }
    for (int m = 32; m; m >>= 1) amax = fmaxf(amax, __shfl_xor(amax, m));
    if (__any(odd) && a.layer.status && lane == 0) atomicOr(a.layer.status, TQ_KV_NONFINITE);

    const float s1 = fmaxf(s0, amax < kTiny ? 0.f : amax * (1.f / code_top<FP8>()));
    const float r = s1 > 0.f ? 1.f / s1 : 0.f;
    const bool grown = c > 0 && s1 > s0;
    const float ratio = grown ? s0 / s1 : 1.f;

#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int t = p * TP + t0;
        float z[8];
        for (int j = 0; j < 8; ++j) z[j] = clamp_code<FP8>(x[p][j] * r);
        const uint2 w = make_uint2(pack4<FP8>(z[0], z[1], z[2], z[3]), pack4<FP8>(z[4], z[5], z[6], z[7]));
        if (val) {
            *reinterpret_cast<uint2 *>(&codes[wave][t * D + e0]) = w;
        } else {
            uint2 *to = reinterpret_cast<uint2 *>(store + t * D + e0);
            if (t >= c && (t < e || c == 0)) {
                *to = w;                               // past e: zeros
            } else if (grown) {   // also what a retreat left past e
                const uint2 o = *to;
                *to = make_uint2(shrink4<FP8>(o.x, ratio), shrink4<FP8>(o.y, ratio));
            }
        }
    }
    if (val) {
        // the wave's own LDS: its writes above are waited for, nobody else's matter
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            uint32_t w[4] = {old[i].x, old[i].y, old[i].z, old[i].w};
            if (grown)
                for (int q = 0; q < 4; ++q) w[q] = shrink4<FP8>(w[q], ratio);
            for (int t = 0; t < kBlock; ++t) {
                if (t >= c && (t < e || c == 0)) {
                    const uint32_t b = codes[wave][t * D + i * 64 + lane];
                    const int sh8 = 8 * (t & 3);
                    w[t >> 2] = (w[t >> 2] & ~(255u << sh8)) | (b << sh8);
                }
            }
            reinterpret_cast<uint4 *>(store)[i * 64 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    if (lane == 0) *scale = s1;
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
