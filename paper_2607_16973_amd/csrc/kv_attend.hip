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

// Rows of few queries (decoding, drafted tokens).  A unit is a tile of 16 NT
// query rows of one key head of one table row, and has that row's pages to
// go through.  All units' pages form one line, which is cut into equal
// shares, one per wave of the grid: rows of very different lengths load the
// machine evenly, and a wave has the next page's codes on the way while it
// works, across units too.  A unit that lies in one share is written out at
// once; of the others each share leaves a part (at most two per wave: at
// its begin and at its end) for join_kernel.  Bound by the memory system:
// up to 16 pages of 64 D bytes in flight per compute unit.
struct Place {                       // a page of the line; the same in all lanes
    int row, tile, kvh, page;        // page of the row
    int tiles, pages;                // of the row
    int len, count, first;
};

// Tiles and pages of a table row.  A row without tokens has one page, which
// nobody sees.
template <int RT>
__device__ inline void row_shape(const AttendArgs &a, int row, Place *p) {
    row_tokens(a.set.starts, row, a.set.total, &p->first, &p->count);
    p->len = a.set.lens[row];
    p->tiles = (p->count * a.group + RT - 1) / RT;
    p->pages = max((min(p->len, a.limit) + kPage - 1) / kPage, 1);
}

template <int RT>
__device__ inline void to_row(const AttendArgs &a, int row, Place *p) {
    p->row = row;
    row_shape<RT>(a, row, p);
    p->len = __builtin_amdgcn_readfirstlane(p->len);
    p->count = __builtin_amdgcn_readfirstlane(p->count);
    p->first = __builtin_amdgcn_readfirstlane(p->first);
    p->tiles = __builtin_amdgcn_readfirstlane(p->tiles);
    p->pages = __builtin_amdgcn_readfirstlane(p->pages);
}

template <int RT>
__device__ inline void advance(const AttendArgs &a, Place *p) {
    if (++p->page < p->pages) return;
    p->page = 0;
    if (++p->kvh < a.layer.heads) return;
    p->kvh = 0;
    if (++p->tile < p->tiles) return;
    p->tile = 0;
    int row = p->row;
    do {
        if (++row >= a.set.rows) return;             // past the line: never used
        to_row<RT>(a, row, p);
    } while (p->tiles == 0);
}

// The number of a unit in the list of parts (first: the row's first token,
// which row_tokens keeps inside the call, and the number with it).
template <int RT>
__device__ inline int64_t unit_of(const AttendArgs &a, int row, int first, int tile, int kvh) {
    const int64_t slot = a.set.starts ? (int64_t)first * a.group / RT + row : (int64_t)row * ((a.group + RT - 1) / RT);
    return (slot + tile) * a.layer.heads + kvh;
}

template <int D, bool FP8, int NT>
__global__ __launch_bounds__(256) void attend_kernel(AttendArgs a) {
    constexpr int KS = D / 32;                       // 32-wide steps of the first product
    constexpr int DT = D / 16;
    constexpr int RT = 16 * NT;
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int share = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    const int heads = a.layer.heads;

    // the line's length, the wave's share [x, end) and where x lies
    auto pages_at = [&](int row) {
        Place p;
        if (row >= a.set.rows) return 0;
        row_shape<RT>(a, row, &p);
        return p.tiles * p.pages * heads;
    };
    auto running = [&](int v) {                      // inclusive sum over the lanes
        for (int k = 1; k < 64; k <<= 1) {
            const int y = __shfl_up(v, k);
            if (lane >= k) v += y;
        }
        return v;
    };
    int total = 0, sums = 0;
    for (int base = 0; base < a.set.rows; base += 64) {
        sums = running(pages_at(base + lane));
        total += __builtin_amdgcn_readlane(sums, 63);
    }
    const int each = (total + a.shares - 1) / a.shares;
    const int x = share * each, end = min(x + each, total);
    if (x >= end) return;
    Place cur;
    {
        int before = 0;
        for (int base = 0;; base += 64) {
            if (a.set.rows > 64) sums = running(pages_at(base + lane));
            const uint64_t past = __ballot(before + sums > x);
            if (past) {
                const int at = __builtin_ctzll(past);
                if (at) before += __builtin_amdgcn_readlane(sums, at - 1);
                to_row<RT>(a, base + at, &cur);
                break;
            }
            before += __builtin_amdgcn_readlane(sums, 63);
        }
        const int within = x - before, unit = within / cur.pages;
        cur.page = within % cur.pages;
        cur.tile = unit / heads;
        cur.kvh = unit % heads;
    }

    // what a page needs: its codes and the scales of the lane's block
    uint4 kc[4][D / 64], vc[DT];
    const int krow = (16 * (n >> 2) + (n & 3)) * D + g * 16, vrow = (g * D + n) * 16;
    auto any_in = [&](const Place &p) { return p.page * kPage < min(p.len, a.limit); };
    auto id_of = [&](const Place &p) { return any_in(p) ? a.set.tables[(int64_t)p.row * a.set.width + p.page] : -1; };
    bool fits = false;
    auto tile_of = [&](const Place &p, int page) {
        const bool in = page >= 0 && page < a.layer.pages, any = any_in(p);
        fits = in && any;
        if (!in && any && a.layer.status && lane == 0) atomicOr(a.layer.status, TQ_KV_BAD_PAGE);
        return (int64_t)(fits ? page : 0) * heads + p.kvh;
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
    int64_t tile = tile_of(cur, __builtin_amdgcn_readfirstlane(id_of(cur)));
    load_keys(tile);
    float ks = a.layer.ks[tile * 4 + g], vs = a.layer.vs[tile * 4 + g];
    load_values(tile);
    Place next = cur;                                // the page whose codes come next, its id on the way
    int ahead = 0;
    if (x + 1 < end) {
        advance<RT>(a, &next);
        ahead = id_of(next);
    }

    f16x8 q[NT][KS];
    float factor[NT];
    int pos[NT];                                     // the last key a row sees
    int top = -1, low = -1;                          // the last one any row and every row sees
    float m[NT], mv[NT], l[NT];                      // maxima (log2 units) of scores and of scores with value scales; sum
    f32x4 o[NT][DT];                                 // in units of 2^(mv - kUnit)
    int from = cur.page;                             // the first page of the unit in this share
    bool open = true;                                // a unit begins

    for (int at = x; at < end; ++at) {
        const int len = min(cur.len, a.limit);
        const int rows = cur.count * a.group, r0 = cur.tile * RT, last = min(rows - 1, r0 + RT - 1);
        if (open) {
            from = cur.page;
            top = min(cur.len - cur.count + last / a.group, len - 1);
            low = min(cur.len - cur.count + r0 / a.group, len - 1);
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const int r = min(r0 + 16 * i + n, last), token = r / a.group;
                pos[i] = min(cur.len - cur.count + token, len - 1);
                const int e = load_queries<D>(a, r0 + 16 * i + n <= last,
                                              (int64_t)(cur.first + token) * a.qt + (int64_t)(cur.kvh * a.group + r % a.group) * a.qh, g, q[i]);
                factor[i] = ldexpf(fabsf(a.scale2), -e);
                m[i] = mv[i] = -__builtin_inff();
                l[i] = 0.f;
                for (int d = 0; d < DT; ++d) o[i][d] = {0.f, 0.f, 0.f, 0.f};
            }
            open = false;
        }
        // S^T of the page
        f32x4 s[NT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            for (int i = 0; i < NT; ++i) s[i][j] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int u = 0; u < D / 64; ++u) {
                f16x8 lo, hi;
                to_half<FP8>(kc[j][u], &lo, &hi);
#pragma unroll
                for (int i = 0; i < NT; ++i) {
                    s[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lo, q[i][2 * u], s[i][j], 0, 0, 0);
                    s[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(hi, q[i][2 * u + 1], s[i][j], 0, 0, 0);
                }
            }
        }
        const bool here = fits, more = at + 1 < end;
        const float kscale = ks;
        const Place then = next;                     // the next page's keys
        if (more) {
            tile = tile_of(next, __builtin_amdgcn_readfirstlane(ahead));
            load_keys(tile);
            ks = a.layer.ks[tile * 4 + g];
            if (at + 2 < end) {
                advance<RT>(a, &next);
                ahead = id_of(next);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        const int base = cur.page * kPage + 16 * g;  // position of the lane's first token
        float vlog = vs > 0.f ? __log2f(vs) : -__builtin_inff();
        // A page that holds the row's end may hold anything past it: those
        // codes and scales are taken out before they meet a zero weight.
        if ((cur.page + 1) * kPage > len || !here) {
            const int left = here ? min(max(len - base, 0), 16) : 0;
            if (left == 0) vlog = -__builtin_inff();
#pragma unroll
            for (int d = 0; d < DT; ++d) vc[d] = keep_tokens(vc[d], left);
        }
        const bool masked = (cur.page + 1) * kPage - 1 > low || !here;

        f16x8 w[NT][2], wl[NT][2];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            // never 0, so that a masked score stays -inf (a NaN scale of an unused block goes too)
            const float f = fmaxf(factor[i] * kscale, 0x1p-126f);
            if (masked) {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (base + j > pos[i] || !here) s[i][j >> 2][j & 3] = -__builtin_inff();
            }
            float big = max3(s[i][0][0], s[i][0][1], s[i][0][2]);
#pragma unroll
            for (int j = 3; j < 15; j += 2) big = max3(big, s[i][j >> 2][j & 3], s[i][(j + 1) >> 2][(j + 1) & 3]);
            big = fmaxf(big, s[i][3][3]) * f;
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
                const float e = __builtin_amdgcn_exp2f(scaled_less(s[i][j >> 2][j & 3], f, m1));
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

        if (cur.page + 1 == cur.pages || !more) {    // the unit, or the share, ends here
            const bool whole = from == 0 && cur.page + 1 == cur.pages;
            const int place = 2 * share + (at - x == cur.page - from ? 0 : 1);   // the share's first unit, or its last
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                const float sum = sum_of_groups(l[i]);
                // to units of 2^m, which the parts have in common with the sum
                const float back = mv[i] == -__builtin_inff() ? 0.f : __builtin_amdgcn_exp2f(mv[i] - m[i] - kUnit);
                const int r = r0 + 16 * i + n;
                if (r <= last) {
                    if (whole) {
                        const int64_t to = (int64_t)(cur.first + r / a.group) * a.heads + cur.kvh * a.group + r % a.group;
                        const float inv = sum > 0.f || sum != sum ? back / sum : 0.f;
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            unsigned short h[4];
                            for (int k = 0; k < 4; ++k) h[k] = float_bits16(o[i][d][k] * inv, a.bf16);
                            uint2 u;
                            __builtin_memcpy(&u, h, 8);
                            *reinterpret_cast<uint2 *>(static_cast<unsigned short *>(a.out) + to * D + d * 16 + g * 4) = u;
                        }
                        if (a.lse && g == 0) a.lse[to] = sum == 0.f ? -__builtin_inff() : (m[i] + __log2f(sum)) * 0.69314718056f;
                    } else {
                        float *po = a.parts + ((int64_t)place * RT + 16 * i + n) * (D + 4);
#pragma unroll
                        for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4 *>(po + d * 16 + g * 4) = o[i][d] * back;
                        if (g == 0) {
                            po[D] = m[i];
                            po[D + 1] = sum;
                        }
                    }
                }
            }
            // who begins a unit says where its parts are
            if (from == 0 && lane == 0) {
                const int begin = at - cur.page, finish = begin + cur.pages - 1;   // in the line
                reinterpret_cast<int2 *>(a.info)[unit_of<RT>(a, cur.row, cur.first, cur.tile, cur.kvh)] =
                    make_int2(place, finish / each - begin / each + 1);
            }
            open = true;
        }
        cur = then;
    }
}

// Joins the parts of a (token, head) whose unit several shares have: W waves,
// each takes every W-th part.
template <int D, int RT, int W>
__global__ __launch_bounds__(256) void join_kernel(AttendArgs a) {
    constexpr int N = D / 64;
    __shared__ float lds[W > 1 ? W * (D + 1) : 1];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t at = W > 1 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (at >= (int64_t)a.set.total * a.heads) return;
    const int token = (int)(at / a.heads), head = (int)(at % a.heads);
    int row = token, first = token, count = 1;
    if (a.set.starts) {
        row = slot_row(a.set.starts, a.set.rows, token, 1, 1, 0);
        row_tokens(a.set.starts, row, a.set.total, &first, &count);
        if (token < first || token >= first + count) return;
    }
    const int r = (token - first) * a.group + head % a.group;
    const int2 info = reinterpret_cast<const int2 *>(a.info)[unit_of<RT>(a, row, first, r / RT, head / a.group)];
    const int place = info.x, parts = info.y;
    if (parts <= 1) return;                          // written already
    // (starts that do not ascend may leave a unit without an owner)
    if (place < 0 || parts > a.shares || (place & ~1) + 2 * (parts - 1) >= 2 * a.shares) return;
    // the first part, then the first unit of each following share
    const float *first_part = a.parts + ((int64_t)place * RT + r % RT) * (D + 4);
    const float *others = a.parts + ((int64_t)(place & ~1) * RT + r % RT) * (D + 4);
    auto part_of = [&](int c) { return c ? others + (int64_t)c * 2 * RT * (D + 4) : first_part; };
    float m = -__builtin_inff();
    for (int c = lane; c < parts; c += 64) m = fmaxf(m, part_of(c)[D]);
    for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    const float mm = m == -__builtin_inff() ? 0.f : m;
    float l = 0.f, o[N];
    for (int j = 0; j < N; ++j) o[j] = 0.f;
#pragma unroll 4
    for (int c = W > 1 ? wave : 0; c < parts; c += W) {
        const float *po = part_of(c);
        const float e = __builtin_amdgcn_exp2f(po[D] - mm);
        l += e * po[D + 1];
        for (int j = 0; j < N; ++j) o[j] += e * po[j * 64 + lane];
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

template <int D, bool FP8, int NT>
hipError_t launch(const AttendArgs &a, const AttendPlan &p, hipStream_t stream) {
    constexpr int RT = 16 * NT;
    attend_kernel<D, FP8, NT><<<(unsigned)((p.shares + 3) / 4), 256, 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.join) return e;
    const int64_t outs = (int64_t)a.set.total * a.heads;
    // results of many parts: four waves each
    if (p.shares > 8 * p.units) join_kernel<D, RT, 4><<<(unsigned)outs, 256, 0, stream>>>(a);
    else join_kernel<D, RT, 1><<<(unsigned)((outs + 3) / 4), 256, 0, stream>>>(a);
    return hipGetLastError();
}

template <int D, bool FP8>
hipError_t pick(const AttendArgs &a, const AttendPlan &p, hipStream_t stream) {
    if constexpr (D < 256) {   // at 256 two tiles do not fit the registers
        if (p.tile == 32) return launch<D, FP8, 2>(a, p, stream);
    }
    return launch<D, FP8, 1>(a, p, stream);
}

}  // namespace

AttendPlan attend_plan(int64_t n, int rows, int group, int kv_heads, int width, int longest, int D, bool starts) {
    AttendPlan p;
    const int64_t tokens = (int64_t)width * kPage;
    const int64_t len = longest > 0 && longest < tokens ? longest : tokens;
    const int64_t pages = len > 0 ? (len + kPage - 1) / kPage : 1;
    // query rows of one key head and table row, on average
    const int64_t mean = (n * group + rows - 1) / rows;
    p.tile = mean > 16 && D < 256 ? 32 : 16;
    p.units = (starts ? n * group / p.tile + rows : rows * (int64_t)((group + p.tile - 1) / p.tile)) * kv_heads;
    // as many waves as have their registers at once: 1 to 3 per SIMD
    const int64_t waves = D == 64 && p.tile == 16 ? 3072 : D == 256 || (D == 128 && p.tile == 32) ? 1024 : 2048;
    p.shares = (int)(p.units * pages < waves ? p.units * pages : waves);
    p.join = pages > 1;
    p.line = p.units * pages;
    return p;
}

size_t attend_info_bytes(const AttendPlan &p) { return ((size_t)p.units * 8 + 255) / 256 * 256; }
size_t attend_bytes(const AttendPlan &p, int D) {
    return attend_info_bytes(p) + (p.join ? sizeof(float) * 2 * (size_t)p.shares * p.tile * (D + 4) : 0);
}

hipError_t kv_attend(const AttendArgs &a, const AttendPlan &p, int D, int type, hipStream_t stream) {
    const bool f = type == TQ_KV_FP8;
    if (D == 64) return f ? pick<64, true>(a, p, stream) : pick<64, false>(a, p, stream);
    if (D == 128) return f ? pick<128, true>(a, p, stream) : pick<128, false>(a, p, stream);
    return f ? pick<256, true>(a, p, stream) : pick<256, false>(a, p, stream);
}

}  // namespace tq
