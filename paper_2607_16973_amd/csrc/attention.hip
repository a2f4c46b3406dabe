// Attention over whole prompts, packed rows, grouped heads.
//
// The rows of a tile are (query, head of the group) pairs of one key head,
// 32 per wave and 128 per workgroup; a step takes 64 keys through LDS:
//   S^T = K Q^T     32x32x16, two tiles of 32 keys
//   O^T += V^T P^T  32x32x16, D / 32 tiles of 32 coordinates
// A query stays in lane n = lane % 32 (and n + 32): maximum, sum and
// correction are lane values, and the weights a lane computes are the operand
// the second product wants from it when its keys are taken in the order
// S^T hands them out: 8 j + 4 (lane / 32) + i, so P never leaves the registers.
// Bound by the matrix cores and the exponentials.
#include <hip/hip_runtime.h>

#include "kv.h"

namespace tq {
namespace {

constexpr int kKeys = 64;     // keys of a step
constexpr int kRows = 128;    // query rows of a workgroup

template <bool BF16>
struct Half;
template <>
struct Half<true> {
    typedef bf16x8 x8;
    static __device__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <>
struct Half<false> {
    typedef f16x8 x8;
    static __device__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

template <bool BF16>
__device__ inline bool finite16(unsigned short u) {
    constexpr unsigned e = BF16 ? 0x7f80 : 0x7c00;
    return (u & e) != e;
}

template <int D, bool BF16>
__global__ __launch_bounds__(256) void prompt_kernel(PromptArgs a) {
    typedef typename Half<BF16>::x8 x8;
    constexpr int KS = D / 16, DT = D / 32, CH = D / 8;   // CH: 16-byte pieces of a row
    __shared__ __align__(16) unsigned short kl[kKeys * D], vl[kKeys * D];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int n = lane & 31, h = lane >> 5;
    // key heads next to each other: workgroups go round the XCDs, so one
    // XCD's L2 sees few of the heads' keys.  A row's long tiles come first.
    const int kvh = blockIdx.x % a.kv_heads;
    int64_t slot = (int64_t)(gridDim.x - 1 - blockIdx.x) / a.kv_heads;
    const int row = slot_row(a.starts, a.rows, slot, a.group, kRows, 1);
    slot -= slot_begin(a.starts, row, a.group, kRows, 1);
    int first, count, kfirst, keys;
    row_tokens(a.starts, row, a.total, &first, &count);
    if (a.key_starts) row_tokens(a.key_starts, row, a.keys, &kfirst, &keys);
    else kfirst = first, keys = count;
    const int64_t rows = (int64_t)count * a.group;
    if (slot < 0 || slot * kRows >= rows) return;
    const int64_t r = slot * kRows + wave * 32 + n;
    const bool in = r < rows;
    const int token = in ? (int)(r / a.group) : 0, head = kvh * a.group + (in ? (int)(r % a.group) : 0);
    // last key the query sees, and the last one any row of the workgroup sees
    const int pos = !in ? -1 : a.causal ? token + keys - count : keys - 1;
    const int64_t last_row = min(rows, (slot + 1) * kRows) - 1;
    const int top = a.causal ? (int)(last_row / a.group) + keys - count : keys - 1;

    x8 q[KS];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        unsigned short u[8];
        const unsigned short *p = static_cast<const unsigned short *>(a.q) + (int64_t)(first + token) * a.qt + head * a.qh + s * 16 + h * 8;
        for (int j = 0; j < 8; ++j) u[j] = in ? p[j] : 0;
        __builtin_memcpy(&q[s], u, 16);
    }
    f32x16 o[DT];
    for (int d = 0; d < DT; ++d)
        for (int j = 0; j < 16; ++j) o[d][j] = 0.f;
    float m = -__builtin_inff(), l = 0.f;

    const int full = a.causal ? (int)(slot * kRows / a.group) + keys - count : keys - 1;   // keys that all rows see
    for (int k0 = 0; k0 <= top; k0 += kKeys) {
        const bool masked = k0 + kKeys - 1 > full;
        bool odd = false;
        __syncthreads();
        for (int c = threadIdx.x; c < kKeys * CH; c += 256) {
            const int kr = c / CH, piece = c % CH, key = k0 + kr;
            unsigned short uk[8], uv[8];
            for (int j = 0; j < 8; ++j) uk[j] = uv[j] = 0;
            if (key < keys) {
                const unsigned short *pk = static_cast<const unsigned short *>(a.k) + (int64_t)(kfirst + key) * a.kt + kvh * a.kh + piece * 8;
                const unsigned short *pv = static_cast<const unsigned short *>(a.v) + (int64_t)(kfirst + key) * a.vt + kvh * a.vh + piece * 8;
                for (int j = 0; j < 8; ++j) uk[j] = pk[j], uv[j] = pv[j];
            }
            __builtin_memcpy(&kl[kr * D + (piece ^ (kr % CH)) * 8], uk, 16);
            __builtin_memcpy(&vl[kr * D + piece * 8], uv, 16);
            for (int j = 0; j < 8; ++j) odd |= !finite16<BF16>(uv[j]);
        }
        // Values that are not finite must not meet the zero weights of the
        // rows that do not see them: where a step has both, they are taken
        // out of the product and added to the rows that do see them.
        odd = __syncthreads_or(odd && masked);
        f32x16 s[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            for (int j = 0; j < 16; ++j) s[t][j] = 0.f;
#pragma unroll
            for (int c = 0; c < KS; ++c) {
                x8 k;
                const int kr = t * 32 + n, piece = 2 * c + h;
                __builtin_memcpy(&k, &kl[kr * D + (piece ^ (kr % CH)) * 8], 16);
                s[t] = Half<BF16>::mfma(k, q[c], s[t]);
            }
        }
        float big = -__builtin_inff();
        float y[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const int key = k0 + (j >> 4) * 32 + ((j & 15) >> 2) * 8 + 4 * h + (j & 3);
            float z = s[j >> 4][j & 15] * a.scale2;
            if (key > pos) z = -__builtin_inff();
            y[j] = z;
            big = fmaxf(big, z);
        }
        const float mn = fmaxf(m, max_of_halves(big)), mm = mn == -__builtin_inff() ? 0.f : mn;
        const float alpha = __builtin_amdgcn_exp2f(m - mm);
        float sum = 0.f;
        unsigned short pw[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float e = __builtin_amdgcn_exp2f(y[j] - mm);
            sum += e;
            pw[j] = float_bits16(e, BF16);
        }
        l = l * alpha + sum;
        m = mn;
        for (int d = 0; d < DT; ++d) o[d] *= alpha;
#pragma unroll
        for (int c = 0; c < 4; ++c) {   // 16 keys: lane half h has 4h + i and 8 + 4h + i of them
            x8 p;
            __builtin_memcpy(&p, &pw[8 * c], 16);
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                unsigned short u[8];
                for (int i = 0; i < 4; ++i) {
                    u[i] = vl[(16 * c + 4 * h + i) * D + d * 32 + n];
                    u[4 + i] = vl[(16 * c + 8 + 4 * h + i) * D + d * 32 + n];
                }
                if (odd)
                    for (int i = 0; i < 8; ++i) u[i] = finite16<BF16>(u[i]) ? u[i] : 0;
                x8 v;
                __builtin_memcpy(&v, u, 16);
                o[d] = Half<BF16>::mfma(v, p, o[d]);
            }
        }
        if (odd) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    for (int kr = 0; kr < kKeys && k0 + kr <= pos; ++kr) {
                        const unsigned short u = vl[kr * D + d * 32 + (j >> 2) * 8 + 4 * h + (j & 3)];
                        if (!finite16<BF16>(u)) o[d][j] += BF16 ? bf16_float(u) : f16_float(u);
                    }
        }
    }
    if (!in) return;
    const int64_t at = (int64_t)(first + token) * a.heads + head;
    // the two lanes of a query hold the sum in two parts
    l = sum_of_halves(l);
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            unsigned short u[4];
            for (int i = 0; i < 4; ++i) u[i] = float_bits16(o[d][4 * j + i] * inv, BF16);
            __builtin_memcpy(static_cast<unsigned short *>(a.out) + at * D + d * 32 + 8 * j + 4 * h, u, 8);
        }
    if (a.lse && h == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * 0.69314718056f;
}

template <int D>
hipError_t launch(const PromptArgs &a, int bf16, hipStream_t stream) {
    const int64_t slots = (int64_t)a.total * a.group / kRows + a.rows;
    const unsigned grid = (unsigned)(slots * a.kv_heads);
    if (bf16) prompt_kernel<D, true><<<grid, 256, 0, stream>>>(a);
    else prompt_kernel<D, false><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t prompt_attention(const PromptArgs &a, int D, int bf16, hipStream_t stream) {
    return D == 64 ? launch<64>(a, bf16, stream) : D == 128 ? launch<128>(a, bf16, stream) : launch<256>(a, bf16, stream);
}

}  // namespace tq
