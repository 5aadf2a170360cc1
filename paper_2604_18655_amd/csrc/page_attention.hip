// Attention over a paged cache of 8 bits (see include/mlora_page_attention.h).
//
// A block takes up to 16 query vectors of one kv head: of one stream, or of several if they have few (a bundle).  What they may see is a list of
// items: pages of 64 tokens (those of the sink, then from the window's first on), chunks of 32 tokens of the tails, chunks of 32 rows of
// the step.  The block's waves take items in turn, each by itself, and merge their results through LDS at the end; where one block is not enough for
// the items several share them, and a second kernel merges what they leave in the workspace.  Streams of a bundle that hold the same page at the same
// place, as beams do, take it together: a page that all of four streams see costs what it costs one.
//
// Pages go from memory to the matrix units as they are: codes are multiplied as whole numbers (16x16x64 products of int8, exact in
// 32 bits), nothing is widened and nothing passes through LDS.  The other side is cut into three digits to the base 256, each a signed byte, of
// whole numbers of three bytes:
//     q = unit * whole         to 2^-22 of the vector's largest magnitude
//     p = whole / P_ONE        p = exp(score - the page's largest score) in (0, 1], to 2^-24
// so that a product of scores or outputs is three products of bytes, each half the work of one of bf16, and as near as fp32 arithmetic would come.  (Two
// digits for outputs in bf16: 4 x 8 beams on 4096 shared tokens 17.0 -> 15.6 us, 128 streams of 130 tokens 16.0 -> 12.3, 200000 tokens 78.6 -> 77.8; but query vectors
// with a feature 100 times the others were off by 10^-3, and 63 keys of a page that each weigh a little less than half a unit were lost, another 10^-3.)
// The weights are counted relative to the page's own maximum; a page's sum of weights is the sum of the very integers that multiply the values.  Scores are K . Q^T: a lane
// holds 16 keys of ONE query vector, and if the keys of a page are dealt to the products in the right order (key 16 * (i / 4) + 4 * t + i % 4 is
// row i of product t) these are the 16 that O^T += V^T . P^T wants from it.  Values are stored feature by feature for that.
// The tail and the step's rows are bf16, with scores and weights as in tree_attention.hip, the weights as three bf16 numbers each (two leave outputs off by
// 10^-6, which shows in fp32 where nearly all that a row sees is tail).
//
// What bounds a call of few query vectors is the bytes (200000 tokens of 8 heads of 128: 79 us, 5.2 TB/s), or, in short ones, the launch and the trips
// length, table, page (333 tokens 4.7 us); else the vector work around the weights, some 250 to 290 instructions per page and tile (8 trees of 30
// rows, 2048 tokens of window, 8 heads of 64: 21 us, of which a wave is 11 in its pages).  So whole numbers become floats and back by adding
// 1.5 * 2^23 or 2^23 where that is free (an accumulator's start, the addend of a multiplication) and not by conversions, and sums are rescaled
// only where a maximum rises by much.  The next page's keys are asked for behind the scores: without that 22 -> 39 us, with the values, too, on their way
// earlier no difference.
#include <algorithm>
#include <type_traits>

#include "common.hpp"

#include "../../include/mlora_page_attention.h"

namespace mlora {

mlora_status check_page_cache(const mlora_page_cache *c);

namespace {

constexpr int P = MLORA_PAGE_TOKENS, KC = 32;            // tokens of a page, of a chunk
constexpr int ALONE = 32;                                // a bundle's streams of fewer pages and chunks go alone (see below)
constexpr float UNSEEN = -__builtin_inff();
constexpr int N = 3;                                     // digits
// The largest weight as a whole number of N digits, 127 in each place, and what turns a float of such a size into its bits: with that addend the low
// bytes of the sum are the number, 128 added to all digits but the first (which has room for none).
constexpr float P_ONE = 8355711.f, P_BITS = 8388608.f + 32896.f;
constexpr int NUMBER = 0x4B400000;                       // the bits of 1.5 * 2^23: a whole number below 2^22 added to them is one added to it
constexpr float NUMBER_F = 12582912.f;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    const uint16_t *q;                                   // bf16 [M][Hq][D]
    const int8_t *k, *v;                                 // of the layer, like the scales and tails
    const float *k_scale, *v_scale;
    const uint16_t *k_tail, *v_tail, *k_new, *v_new;
    const int *slot, *len, *table, *parent;
    float *part_out;                                     // several blocks per query tile: [splits][S * R * Hq][D], not normalised
    float2 *part_ml;                                     // [splits][S * R * Hq]: maximum (of scores in units of log 2) and sum
    int *used;                                           // [S * R * Hq]: how many of the splits there are
    void *out;
    int Hq, Hkv, G, S, R, M;
    int pages, columns, window, sink;
    int splits, bundle;
    unsigned g_inv;                                      // ceil(2^16 / G): v / G = (v * g_inv) >> 16 for v < 512
    int out_fp32;
    float scale2;                                        // scale * log2(e)
};

// Into how many blocks a query tile's items go, of at most `most`
__host__ __device__ constexpr int splits_for(int items, int most) { return items < 32 || most < 1 ? 1 : most < items / 8 ? most : items / 8; }

// a value combined over the four quarters of a wave (lanes 16 and 32 apart); every lane gets the result
template <class Op>
__device__ __forceinline__ float over_quarters(float v, const Op &op)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float most(float x, float y) { return fmaxf(x, y); }
__device__ __forceinline__ float finite_or_0(float m) { return m == UNSEEN ? 0.f : m; }

// D[16 rows][16 cols] += A[16][64] * B[64][16] of signed bytes; lane l supplies row l % 16 of A and column l % 16 of B at
// 16 * (l / 16) .. + 15, and receives D[4 * (l / 16) + r][l % 16] in element r.
__device__ __forceinline__ i32x4 mfma_i8(u32x4 a, u32x4 b, i32x4 c)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// Byte n of four registers
__device__ __forceinline__ unsigned bytes_of(int n, unsigned y0, unsigned y1, unsigned y2, unsigned y3)
{
    const unsigned pair = 0x0C0C0400u + 0x0101u * n;
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(y3, y2, pair), __builtin_amdgcn_perm(y1, y0, pair), 0x05040100u);
}
// Digits of four whole numbers, 128 added to all but the first: d[0] the first (of four numbers), d[N - 1] the last
__device__ __forceinline__ void digits_of(const unsigned (&y)[4], unsigned (&d)[N])
{
    const unsigned lo01 = __builtin_amdgcn_perm(y[1], y[0], 0x05010400u), lo23 = __builtin_amdgcn_perm(y[3], y[2], 0x05010400u);   // {b0 b0 b1 b1}
    const unsigned b0 = __builtin_amdgcn_perm(lo23, lo01, 0x05040100u), b1 = __builtin_amdgcn_perm(lo23, lo01, 0x07060302u);
    d[2] = b0 ^ 0x80808080u;
    d[1] = b1 ^ 0x80808080u;
    d[0] = bytes_of(2, y[0], y[1], y[2], y[3]);
}
// The sum of N products of digits, as a number; NUMBER_F is added to it, as the last accumulator started from NUMBER.
__device__ __forceinline__ float joined(const i32x4 (&x)[N], int e)
{
    return __builtin_fmaf((float)((x[0][e] << 8) + x[1][e]), 256.f, __int_as_float(x[2][e]));
}

// LDS of a wave: the values of a chunk on their way to the matrix units, then its share of the result.
template <int D>
struct WaveLds {
    static constexpr int VROW = D * 2 + 32;              // bytes of a row of values; +32: eight rows cover all banks once
    static constexpr int OROW = D + 4;                   // floats of a query vector's output
    static constexpr int O_BYTES = 16 * OROW * 4, ML_BYTES = 16 * 8;
    static constexpr int BYTES = KC * VROW > O_BYTES + ML_BYTES ? KC * VROW : O_BYTES + ML_BYTES;
};

template <int D, int W, bool SPLIT>
__global__ __launch_bounds__(64 * W, (D == 64 ? 3 : 2)) void page_attn(const AttnArgs a)
{
    using L = WaveLds<D>;
    constexpr int DK = D / 64, DB = D / 16, VI = KC * D / 512;
    __shared__ __align__(16) unsigned char smem[W * L::BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    // blocks: (head, tile, stream and share), or, as a bundle has one tile, (head, bundle, share): those that have nothing to do come last.  In
    // between they left whole compute units without work (128 streams of 2500 tokens took half as long again).
    const int hk = blockIdx.x, per_stream = a.R * a.G;
    int bundle = a.bundle, s0, z = 0, qv0 = 0;
    if (bundle > 1) {
        s0 = (int)blockIdx.y * bundle, z = blockIdx.z;
    } else {
        s0 = SPLIT ? (int)blockIdx.z / a.splits : (int)blockIdx.z, qv0 = (int)blockIdx.y * 16;
        if (SPLIT) z = (int)blockIdx.z - s0 * a.splits;
    }
    int streams = min(bundle, a.S - s0), n_qv = streams * per_stream;

    // this lane's query vector: its stream, row and head
    int sb, row;
    const uint16_t *q_at;
    u32x4 qx[DK][2];
    const auto load_q = [&]() {
        const int vec = min(qv0 + l16, n_qv - 1);
        sb = bundle == 1 ? 0 : vec / per_stream;
        const int in_stream = vec - sb * per_stream;
        row = (int)((unsigned)in_stream * a.g_inv >> 16);
        q_at = a.q + ((size_t)((s0 + sb) * a.R + row) * a.Hq + hk * a.G + (in_stream - row * a.G)) * D;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk)
#pragma unroll
            for (int i = 0; i < 2; ++i) qx[kk][i] = *reinterpret_cast<const u32x4 *>(q_at + 64 * kk + 16 * lq + 8 * i);
    };
    load_q();

    // the items: page numbers that some stream of the bundle sees, then chunks
    int len = min(max(a.len[s0 + sb], 0), P * a.columns + P - 1), slot = min(max(a.slot[s0 + sb], 0), a.S - 1), full, first, sinks;
    int b_full, b_first, b_sinks;                        // of the bundle
    const int per_chunks = (P - 1 + a.R + KC - 1) / KC;
    const auto pages_of = [&]() {
        full = len / P, first = a.window > 0 ? min(max(len - a.window + 1, 0) / P, full) : 0, sinks = min((a.sink + P - 1) / P, first);
        b_full = full, b_first = first, b_sinks = sinks;
        if (bundle > 1)
#pragma unroll
            for (int d = 1; d < 16; d *= 2) {
                b_full = max(b_full, __shfl_xor(b_full, d));
                b_first = min(b_first, __shfl_xor(b_first, d));
                b_sinks = max(b_sinks, __shfl_xor(b_sinks, d));
            }
        b_full = __builtin_amdgcn_readfirstlane(b_full), b_first = __builtin_amdgcn_readfirstlane(b_first);
        b_sinks = min(__builtin_amdgcn_readfirstlane(b_sinks), b_first);
    };
    pages_of();
    // The host has cut the call for tables that are full.  Where the streams of a bundle are short, each has a block of its own; what the lengths call for
    // decides how many blocks share a bundle or stream.  The other blocks have nothing to do.  (In long tables, us in a graph, all blocks busy and so: 8
    // streams of 100 tokens 11.2 / 7.3, 21 of 70 13.8 / 7.0, 64 of 300 14.4 / 12.2, 8 of 1000 13.3 / 9.9; long ones are the same within 1 %.)
    if (bundle > 1 && b_sinks + b_full - b_first + per_chunks < ALONE) {
        if (z >= streams) return;
        len = __builtin_amdgcn_readlane(len, z * per_stream), slot = __builtin_amdgcn_readlane(slot, z * per_stream);
        s0 += z, z = 0, bundle = streams = 1, n_qv = per_stream;
        load_q();
        pages_of();
    }
    const int n_pages = b_sinks + b_full - b_first, items = n_pages + streams * per_chunks;
    const int use = SPLIT ? splits_for(streams * (n_pages + per_chunks), a.splits) : 1, stride = use * W;
    if (z >= use) return;
    const int *const table = a.table + (size_t)slot * a.columns;
    int c = z * W + wave;
    // the page that this lane's stream sees as item i, or -1
    const auto number_of = [&](int i) { return i < b_sinks ? i : b_first + i - b_sinks; };
    const auto look_up = [&](int i) {
        const int at = number_of(i);
        int page = -1;
        if (i < n_pages && at < full && (at >= first || at < sinks)) page = table[at];
        return page < a.pages ? page : -1;
    };
    int todo = look_up(c), ahead = look_up(c + stride);

    // its digits
    u32x4 qd[N][DK];
    float unit;                                          // score of a product of codes, but for the page's scale
    {
        unsigned top = 0;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, max(qx[kk][i / 4][i % 4] & 0x7FFFu, qx[kk][i / 4][i % 4] >> 16 & 0x7FFFu));
        top = __float_as_uint(over_quarters(__uint_as_float(top), [](float x, float y) { return __uint_as_float(max(__float_as_uint(x), __float_as_uint(y))); }));
        // (whole numbers below 2^22)
        const int e = (int)max(top >> 7, 1u) - 127;
        const bool ok = top < 0x7F80u;
        constexpr int BITS = 21;
        unit = ok ? __builtin_ldexpf(fabsf(a.scale2), e - BITS) : __builtin_nanf("");
        const int shift = BITS - e;
        const float sign = a.scale2 < 0.f ? -1.f : 1.f;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                unsigned n[4], d[N];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned pair = qx[kk][w / 2][2 * (w % 2) + j / 2];
                    const float f = sign * __builtin_ldexpf(bf16_bits_to_float(j & 1 ? pair >> 16 : pair & 0xFFFFu), shift);
                    n[j] = (unsigned)((ok ? (int)rintf(f) : 0) + 0x8080);
                }
                digits_of(n, d);
#pragma unroll
                for (int g = 0; g < N; ++g) qd[g][kk][w] = d[g];
            }
    }
    // lane b * R + r: the rows that row r of stream b may see, itself and what it continues.  A parent must be an earlier row, so a path has at most
    // 64; each step doubles what is known of all of them.
    const int my_row = bundle == 1 ? lane : lane % a.R, row_lane = sb * a.R + row;
    unsigned anc_lo = my_row < 32 ? 1u << my_row : 0u, anc_hi = my_row >= 32 ? 1u << (my_row - 32) : 0u;
    if (a.R > 1) {
        int up = lane < streams * a.R ? a.parent[s0 * a.R + lane] : -1;
        up = up < my_row ? up : -1;
        while (__ballot(up >= 0)) {
            const int of = lane - my_row + max(up, 0), further = __shfl(up, of);
            const unsigned lo = (unsigned)__shfl((int)anc_lo, of), hi = (unsigned)__shfl((int)anc_hi, of);
            anc_lo |= up >= 0 ? lo : 0u;
            anc_hi |= up >= 0 ? hi : 0u;
            up = up >= 0 ? further : -1;
        }
    }
    const int depth = __popc(anc_lo) + __popc(anc_hi) - 1;             // of row `my_row`
    unsigned long long path = (unsigned long long)(unsigned)__shfl((int)anc_hi, row_lane) << 32 | (unsigned)__shfl((int)anc_lo, row_lane);
    const int since = a.window > 0 ? len + __shfl(depth, row_lane) - a.window + 1 : 0;      // positions that the row sees begin here, but for the sink
    if (a.window > 0 && a.window < a.R)                  // the rows of the path that the window has left behind
        for (int j = 0; j < a.R; ++j) {
            const int pos = len + __shfl(depth, sb * a.R + j);
            if (pos < since && pos >= a.sink) path &= ~(1ull << j);
        }

    float m = UNSEEN, l = 0.f, over = 0.f;               // l: of the lane's own keys; over: what NUMBER_F adds to every output
    f32x4 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};

    // pages: the next one to look at, and who sees it
    int page = -1;
    bool mine = false;
    u32x4 kf[4][DK], vf[DB];
    float ks, vs;
    const auto next = [&]() {
        for (;;) {
            const unsigned long long left = __ballot(todo >= 0);
            if (left) {
                page = __builtin_amdgcn_readlane(todo, __builtin_ctzll(left));
                mine = todo == page;
                todo = mine ? -1 : todo;
                return true;
            }
            if (c + stride >= n_pages) return false;
            c += stride;
            todo = ahead;
            ahead = look_up(c + stride);
        }
    };
    const auto load_k = [&]() {
        const size_t at = (size_t)page * a.Hkv + hk;
        const int8_t *const kp = a.k + at * (P * D) + (16 * (l16 >> 2) + (l16 & 3)) * D + 16 * lq;
        ks = a.k_scale[at], vs = a.v_scale[at];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int kk = 0; kk < DK; ++kk) kf[t][kk] = *reinterpret_cast<const u32x4 *>(kp + 4 * t * D + 64 * kk);
    };
    const auto load_v = [&]() {
        const int8_t *const vp = a.v + ((size_t)page * a.Hkv + hk) * (P * D) + l16 * P + 16 * lq;
#pragma unroll
        for (int db = 0; db < DB; ++db) vf[db] = *reinterpret_cast<const u32x4 *>(vp + 16 * db * P);
    };
    bool more = c < n_pages && next();
    if (more) {
        load_k();
        load_v();
    }
#pragma nounroll
    while (more) {
        // scores: element e of sc[t] is key 16 * lq + 4 * t + e; in units of `per`, and NUMBER_F too large
        f32x4 sc[4];
        float per = unit * ks;
        const float vs_here = vs;
        // (a query vector or a page that is not finite: whoever sees a token becomes NaN below.  Zeros are all alike, and hidden keys stay hidden.)
        const bool bad = !(per >= 0.f && per < __builtin_inff()), seen = mine;
        if (bad || per == 0.f) per = 1e-30f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            i32x4 x[N];
#pragma unroll
            for (int g = 0; g < N; ++g) {
                x[g] = g == 2 ? i32x4{NUMBER, NUMBER, NUMBER, NUMBER} : i32x4{0, 0, 0, 0};
#pragma unroll
                for (int kk = 0; kk < DK; ++kk) x[g] = mfma_i8(kf[t][kk], qd[g][kk], x[g]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[t][e] = joined(x, e);
        }
        const int t0 = number_of(c) * P;
        more = next();
        if (more) load_k();
        if (__ballot(seen && t0 < since && t0 + P > a.sink)) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int pos = t0 + 16 * lq + 4 * t + e;
                    sc[t][e] = pos >= since || pos < a.sink ? sc[t][e] : UNSEEN;
                }
        }
        float top = UNSEEN;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[t][e]);
        top = over_quarters(top, most);
        // weights relative to the page's maximum, as whole numbers; nothing of a page that the lane's stream does not hold
        // (its maximum a little too large, since that of a product is rounded and no weight may be above 1)
        const float scaled = finite_or_0(top) * per, from = scaled + fabsf(scaled) * 0x1p-23f, one = seen ? P_ONE : 0.f;
        unsigned sum = 0;
        u32x4 pd[N];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            unsigned n[4], d[N];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                n[e] = __float_as_uint(__builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][e], per, -from)), one, P_BITS));
                sum += n[e];
            }
            digits_of(n, d);
#pragma unroll
            for (int g = 0; g < N; ++g) pd[g][t] = d[g];
        }
        sum -= 16u * __float_as_uint(P_BITS);
        top = top == UNSEEN || !seen ? UNSEEN : __builtin_fmaf(-NUMBER_F, per, from);
        // The sums so far are relative to a maximum that is raised only where a page's is more than 2^8 times as heavy: fp32 has the room, and what the
        // lane holds need not be scaled for every page that is a little heavier.
        if (__ballot(top > m + 8.f)) {
            const float m_new = top > m + 8.f ? top : m, keep = __builtin_amdgcn_exp2f(m - finite_or_0(m_new));
            m = m_new;
            l *= keep;
            over *= keep;
#pragma unroll
            for (int db = 0; db < DB; ++db) o[db] *= keep;
        }
        float w = __builtin_amdgcn_exp2f(top - finite_or_0(m)) * (1.f / P_ONE);
        if (bad && top != UNSEEN) w = __builtin_nanf("");
        l += (float)(int)sum * w;
        const float wv = top != UNSEEN ? w * vs_here : 0.f;              // (a page of NaN that the row does not see)
        over += NUMBER_F * wv;
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            i32x4 x[N];
#pragma unroll
            for (int g = 0; g < N; ++g) x[g] = mfma_i8(vf[db], pd[g], g == 2 ? i32x4{NUMBER, NUMBER, NUMBER, NUMBER} : i32x4{0, 0, 0, 0});
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][e] = __builtin_fmaf(joined(x, e), wv, o[db][e]);
        }
        if (more) load_v();
    }
    while (c < n_pages) c += stride;
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] -= over;

    // chunks of a tail and, behind it, the step's rows
    unsigned char *const piece_of = smem + wave * L::BYTES;
    unsigned char *const v_in = piece_of + (lane / (D / 8)) * L::VROW + (lane % (D / 8)) * 16;
    using Lds4 = __attribute__((address_space(3))) s16x4;
    const unsigned char *const v_out = piece_of + (4 * lq + (l16 >> 2)) * L::VROW + (l16 & 3) * 8;
    for (; c < items; c += stride) {
        const int cs = (c - n_pages) / per_chunks, k0 = (c - n_pages - cs * per_chunks) * KC;
        const int its_len = __builtin_amdgcn_readlane(len, cs * per_stream), its_slot = __builtin_amdgcn_readlane(slot, cs * per_stream);
        const int n_tail = its_len % P, n = min(n_tail + a.R - k0, KC);
        if (n <= 0) continue;
        const size_t tail_at = ((size_t)its_slot * a.Hkv + hk) * P * D, rows_at = ((size_t)(s0 + cs) * a.R * a.Hkv + hk) * D;
        // key number k0 + i, the last one behind the end
        const auto from = [&](const uint16_t *tail, const uint16_t *rows, int i) {
            const int k = k0 + min(i, n - 1);
            return k < n_tail ? tail + tail_at + k * D : rows + rows_at + (size_t)(k - n_tail) * (a.Hkv * D);
        };
        // scores: element e of sc[j] is key 16 * j + 4 * lq + e
        f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        u32x4 vr[VI];
        const uint16_t *const kp[2] = {from(a.k_tail, a.k_new, l16) + 8 * lq, from(a.k_tail, a.k_new, 16 + l16) + 8 * lq};
#pragma unroll
        for (int u = 0; u < VI; ++u) {
            const int piece = u * 64 + lane;
            vr[u] = *reinterpret_cast<const u32x4 *>(from(a.v_tail, a.v_new, piece / (D / 8)) + (piece % (D / 8)) * 8);
        }
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            const uint4 qf = *reinterpret_cast<const uint4 *>(q_at + 32 * kk + 8 * lq);
#pragma unroll
            for (int j = 0; j < 2; ++j) sc[j] = mfma16(*reinterpret_cast<const uint4 *>(kp[j] + 32 * kk), qf, sc[j]);
        }
        unsigned odd = 0;                                // values that are not finite (what a row does not see is weighed with 0)
#pragma unroll
        for (int u = 0; u < VI; ++u) {
#pragma unroll
            for (int j = 0; j < 4; ++j) odd |= (unsigned)((vr[u][j] & 0x7F80u) == 0x7F80u) | (unsigned)((vr[u][j] & 0x7F800000u) == 0x7F800000u);
            *reinterpret_cast<u32x4 *>(v_in + u * (512 / D) * L::VROW) = vr[u];
        }
        const auto first_bits = [](int n) { return n >= KC ? ~0u : n <= 0 ? 0u : (1u << n) - 1; };
        const int p0 = its_len - n_tail + k0, behind = n_tail - k0;      // position of the first; keys of the tail from here on
        const unsigned in_tail = first_bits(behind) & (~first_bits(since - p0) | first_bits(a.sink - p0));
        const unsigned rows = (unsigned)(behind >= 0 ? path << min(behind, 63) : path >> min(-behind, 63));
        unsigned see = in_tail | (rows & ~first_bits(behind) & first_bits(n));
        see = sb == cs ? see >> 4 * lq : 0u;
        float top = m;                                   // (which may lie below the largest score so far: see above)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sc[j][e] = (see >> (16 * j + e)) & 1 ? sc[j][e] * a.scale2 : UNSEEN;
                top = fmaxf(top, sc[j][e]);
            }
        top = over_quarters(top, most);
        const float base = finite_or_0(top), keep = __builtin_amdgcn_exp2f(m - base);
        m = top;
        float sum = 0.f, p[2][4];
        uint32_t part[N][4];                             // the weights as N bf16 numbers each
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[j][e] = __builtin_amdgcn_exp2f(sc[j][e] - base);
                sum += p[j][e];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float x = p[j][2 * i], y = p[j][2 * i + 1];
#pragma unroll
                for (int g = 0; g < N; ++g) {
                    part[g][2 * j + i] = pack_bf16(x, y);
                    x -= bf16_bits_to_float(part[g][2 * j + i] & 0xFFFFu);
                    y -= __uint_as_float(part[g][2 * j + i] & 0xFFFF0000u);
                }
            }
        }
        l = l * keep + sum;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= keep;
        if (!__ballot(odd)) {
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4 *)(v_out + db * 32)));
                const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4 *)(v_out + 16 * L::VROW + db * 32)));
                const uint4 vf = make_uint4(x.x, x.y, y.x, y.y);
#pragma unroll
                for (int g = 0; g < N; ++g) o[db] = mfma16(vf, make_uint4(part[g][0], part[g][1], part[g][2], part[g][3]), o[db]);
            }
        } else {
            // zeros times infinity would be NaN: key by key, those that the row sees
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll 1
                    for (int g = 0; g < 4; ++g) {
                        const float pk = __shfl(p[j][e], 16 * g + l16), sk = __shfl(sc[j][e], 16 * g + l16);
                        const unsigned char *const v = piece_of + (16 * j + 4 * g + e) * L::VROW;
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            const uint2 x = *reinterpret_cast<const uint2 *>(v + (16 * db + 4 * lq) * 2);
                            const float f[4] = {bf16_bits_to_float(x.x & 0xFFFFu), __uint_as_float(x.x & 0xFFFF0000u), bf16_bits_to_float(x.y & 0xFFFFu),
                                                __uint_as_float(x.y & 0xFFFF0000u)};
#pragma unroll
                            for (int r = 0; r < 4; ++r) o[db][r] = sk == UNSEEN ? o[db][r] : o[db][r] + pk * f[r];
                        }
                    }
        }
    }

    // the waves' results, merged in the order of the waves
    {
        float *const om = reinterpret_cast<float *>(piece_of);
        const float sum = over_quarters(l, [](float x, float y) { return x + y; });
        if (lq == 0) reinterpret_cast<float2 *>(piece_of + L::O_BYTES)[l16] = make_float2(m, sum);
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4 *>(om + l16 * L::OROW + 16 * db + 4 * lq) = o[db];
    }
    __syncthreads();
    for (int i = tid; i < 16 * (D / 4); i += 64 * W) {
        const int qv = i / (D / 4), f = i % (D / 4) * 4, v = qv0 + qv;
        if (v >= n_qv) break;
        auto ml_of = [&](int w) { return reinterpret_cast<const float2 *>(smem + w * L::BYTES + L::O_BYTES)[qv]; };
        float top = UNSEEN;
#pragma unroll
        for (int w = 0; w < W; ++w) top = fmaxf(top, ml_of(w).x);
        const float base = finite_or_0(top);
        f32x4 num = {0.f, 0.f, 0.f, 0.f};
        float den = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float2 x = ml_of(w);
            const float weight = __builtin_amdgcn_exp2f(x.x - base);
            num += weight * *reinterpret_cast<const f32x4 *>(smem + w * L::BYTES + (qv * L::OROW + f) * 4);
            den += weight * x.y;
        }
        const int b = bundle == 1 ? 0 : v / per_stream, in = v - b * per_stream, r = (int)((unsigned)in * a.g_inv >> 16);
        const size_t vec_at = (size_t)((s0 + b) * a.R + r) * a.Hq + hk * a.G + (in - r * a.G);
        if (SPLIT && z == 0 && f == 0) a.used[vec_at] = use;
        if (SPLIT && use > 1) {
            const size_t at = (size_t)z * a.M * a.Hq + vec_at;
            if (f == 0) a.part_ml[at] = make_float2(top, den);
            *reinterpret_cast<f32x4 *>(a.part_out + at * D + f) = num;
        } else {
            num /= den;                                        // (a row always sees itself)
            if (a.out_fp32) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) + vec_at * D + f) = num;
            else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(a.out) + vec_at * D + f) = make_uint2(pack_bf16(num[0], num[1]), pack_bf16(num[2], num[3]));
        }
    }
}

// Four features of a query vector per thread: merge what the blocks that shared its pages saw, in their order.
template <int D>
__global__ __launch_bounds__(256) void page_attn_combine(const AttnArgs a)
{
    const int i = (int)blockIdx.x * 256 + (int)threadIdx.x, vecs = a.M * a.Hq;
    if (i >= vecs * (D / 4)) return;
    const int vec = i / (D / 4), f = i % (D / 4) * 4;
    const int used = a.used[vec];                              // (1: a block has written the output; what nobody wrote holds anything)
    constexpr int RB = 8;                                      // results per trip to memory; the next ones are asked for before these are known
    float2 ml[2][RB];
    f32x4 pv[2][RB];
    const auto load = [&](int z0, float2 (&ml)[RB], f32x4 (&pv)[RB]) {
#pragma unroll
        for (int u = 0; u < RB; ++u) {
            const size_t at = (size_t)min(z0 + u, a.splits - 1) * vecs + vec;
            ml[u] = a.part_ml[at];
            pv[u] = *reinterpret_cast<const f32x4 *>(a.part_out + at * D + f);
        }
    };
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f, run_top = UNSEEN;
    const auto take = [&](int z0, float2 (&ml)[RB], f32x4 (&pv)[RB]) {
        float top = run_top;
#pragma unroll
        for (int u = 0; u < RB; ++u) {
            if (z0 + u >= used) ml[u] = make_float2(UNSEEN, 0.f), pv[u] = f32x4{0.f, 0.f, 0.f, 0.f};
            top = fmaxf(top, ml[u].x);
        }
        const float base = finite_or_0(top), keep = __builtin_amdgcn_exp2f(run_top - base);
        num *= keep;
        den *= keep;
#pragma unroll
        for (int u = 0; u < RB; ++u) {
            const float w = __builtin_amdgcn_exp2f(ml[u].x - base);
            num += w * pv[u];
            den += w * ml[u].y;
        }
        run_top = top;
    };
    load(0, ml[0], pv[0]);
    for (int z0 = 0;; z0 += 2 * RB) {
        if (z0 + RB < a.splits) load(z0 + RB, ml[1], pv[1]);
        take(z0, ml[0], pv[0]);
        if (!__any(used > z0 + RB)) break;
        if (z0 + 2 * RB < a.splits) load(z0 + 2 * RB, ml[0], pv[0]);
        take(z0 + RB, ml[1], pv[1]);
        if (!__any(used > z0 + 2 * RB)) break;
    }
    if (used == 1) return;
    num /= den;
    const size_t at = (size_t)vec * D + f;
    if (a.out_fp32) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) + at) = num;
    else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(a.out) + at) = make_uint2(pack_bf16(num[0], num[1]), pack_bf16(num[2], num[3]));
}

bool misaligned(const void *p, unsigned mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }

// How a call is cut.  Lines drawn from 28 calls with 4, 8 and 16 waves and 1 to 64 splits, us in a graph.
struct Plan {
    int waves, splits, bundle;
};
constexpr int MOST_SPLITS = 64;
Plan plan_of(const mlora_page_attn &t)
{
    Plan p;
    const long long pages = t.cache.max_pages;
    const long long seen = t.window > 0 ? std::min(pages, (long long)t.window / P + 2 + ((long long)t.sink + P - 1) / P) : pages;
    const int qv = t.rows_per_stream * (t.n_q_heads / t.cache.n_kv_heads);
    // Streams of a bundle may share pages, but each has a tail of its own to be gone through: 21 streams of one query vector and one page 4.5 us, in
    // bundles of 16 19.  Four beams on 4096 shared tokens take a quarter of the pages (22 -> 13 us without the merge).
    p.bundle = seen < 8 ? 1 : std::max(1, std::min(std::min(16 / qv, 8), t.cache.n_streams));
    const long long items = p.bundle * (seen + (P - 1 + t.rows_per_stream + KC - 1) / KC);
    const long long blocks = (long long)t.cache.n_kv_heads * ((t.cache.n_streams + p.bundle - 1) / p.bundle) * ((qv + 15) / 16);
    // Shared items cost a second launch (2.4 us at least) and pay from about four per wave on (8 items: 7.1 -> 4.7 with one block; 127: 27 -> 8.5 with 16),
    // up to some 200 blocks of eight waves (8 blocks of 3125 items, 24 / 32 splits: 78.5 / 80.1; 64 blocks would take 6 as well as 3: 16.9 / 15.4).  Calls that
    // fill the card without have blocks of four waves (512 blocks of 37 items: 21.4, of eight waves 22.4).  16 waves were first in 2 of 26, by 1.3 %.
    p.splits = splits_for((int)std::min(items, 1ll << 30), (int)std::min(std::max((200 + blocks / 2) / blocks, 1ll), (long long)MOST_SPLITS));
    p.waves = blocks * p.splits <= 256 ? 8 : 4;
    return p;
}
size_t workspace_floats(const mlora_page_attn &t)
{
    const int splits = plan_of(t).splits;
    return splits == 1 ? 0 : t.n_q_heads * (size_t)t.cache.n_streams * t.rows_per_stream * (splits * ((size_t)t.cache.head_dim + 2) + 1);
}

mlora_status check(const mlora_page_attn *t)
{
    if (!t) return MLORA_EINVAL;
    const mlora_status st = check_page_cache(&t->cache);
    if (st != MLORA_OK) return st;
    const mlora_page_cache &c = t->cache;
    if (t->layer < 0 || t->layer >= c.n_layers) return MLORA_ESHAPE;
    if (t->n_q_heads <= 0 || t->n_q_heads % c.n_kv_heads != 0 || t->n_q_heads / c.n_kv_heads > 8 || t->n_q_heads > 65535) return MLORA_ESHAPE;
    if (t->rows_per_stream <= 0 || t->rows_per_stream > 64 || (long long)c.n_streams * t->rows_per_stream > MLORA_MAX_ROWS) return MLORA_ESHAPE;
    if (t->window < 0 || t->sink < 0) return MLORA_ESHAPE;
    if (!t->k_new || !t->v_new || !t->parent) return MLORA_EINVAL;
    if (misaligned(t->k_new, 15u) || misaligned(t->v_new, 15u) || misaligned(t->parent, 3u)) return MLORA_EALIGN;
    return MLORA_OK;
}

}  // namespace
}  // namespace mlora

using namespace mlora;

extern "C" {

size_t mlora_page_attention_workspace_bytes(const mlora_page_attn *t)
{
    if (check(t) != MLORA_OK) return 0;
    return workspace_floats(*t) * sizeof(float) + 256;
}

mlora_status mlora_page_attention_plan(const mlora_page_attn *t, int32_t *info)
{
    if (!info) return MLORA_EINVAL;
    const mlora_status st = check(t);
    if (st != MLORA_OK) return st;
    const Plan p = plan_of(*t);
    info[0] = 1;
    info[1] = p.waves;
    info[2] = p.splits;
    return MLORA_OK;
}

mlora_status mlora_page_attention(const mlora_page_attn *t, const void *q, void *out, int32_t out_dtype, void *workspace,
                                  size_t workspace_bytes, void *stream)
{
    const mlora_status st = check(t);
    if (st != MLORA_OK) return st;
    if (!q || !out) return MLORA_EINVAL;
    if (out_dtype != MLORA_Y_BF16 && out_dtype != MLORA_Y_FP32) return MLORA_EINVAL;
    if (misaligned(q, 15u) || misaligned(out, 15u)) return MLORA_EALIGN;
    if (!workspace || workspace_bytes < workspace_floats(*t) * sizeof(float) + 256) return MLORA_EWORKSPACE;
    if (misaligned(workspace, 255u)) return MLORA_EALIGN;
    const Plan p = plan_of(*t);
    const mlora_page_cache &c = t->cache;
    const size_t pool = (size_t)t->layer * c.n_pages * c.n_kv_heads, tails = (size_t)t->layer * c.n_streams * c.n_kv_heads * P * c.head_dim;

    AttnArgs a;
    a.q = reinterpret_cast<const uint16_t *>(q);
    a.k = reinterpret_cast<const int8_t *>(c.k) + pool * P * c.head_dim;
    a.v = reinterpret_cast<const int8_t *>(c.v) + pool * P * c.head_dim;
    a.k_scale = c.k_scale + pool;
    a.v_scale = c.v_scale + pool;
    a.k_tail = reinterpret_cast<const uint16_t *>(c.k_tail) + tails;
    a.v_tail = reinterpret_cast<const uint16_t *>(c.v_tail) + tails;
    a.k_new = reinterpret_cast<const uint16_t *>(t->k_new);
    a.v_new = reinterpret_cast<const uint16_t *>(t->v_new);
    a.slot = c.slot;
    a.len = c.len;
    a.table = c.table;
    a.parent = t->parent;
    a.out = out;
    a.Hq = t->n_q_heads;
    a.Hkv = c.n_kv_heads;
    a.G = t->n_q_heads / c.n_kv_heads;
    a.S = c.n_streams;
    a.R = t->rows_per_stream;
    a.M = a.S * a.R;
    a.pages = c.n_pages;
    a.columns = c.max_pages;
    a.window = t->window;
    a.sink = std::min(t->sink, P * c.max_pages + 2 * P);
    a.splits = p.splits;
    a.bundle = p.bundle;
    a.part_out = reinterpret_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float2 *>(a.part_out + (size_t)p.splits * a.M * a.Hq * c.head_dim);
    a.used = reinterpret_cast<int *>(a.part_ml + (size_t)p.splits * a.M * a.Hq);
    a.g_inv = (65536u + (unsigned)a.G - 1) / (unsigned)a.G;
    a.out_fp32 = out_dtype == MLORA_Y_FP32;
    a.scale2 = t->scale * 1.44269504088896340736f;

    hipStream_t s = (hipStream_t)stream;
    const dim3 grid = p.bundle > 1 ? dim3((unsigned)a.Hkv, (unsigned)((a.S + p.bundle - 1) / p.bundle), (unsigned)std::max(p.splits, p.bundle))
                                   : dim3((unsigned)a.Hkv, (unsigned)((a.R * a.G + 15) / 16), (unsigned)(a.S * p.splits));
    const auto go = [&](auto d, auto waves) {
        constexpr int D = decltype(d)::value, W = decltype(waves)::value;
        if (p.splits == 1) {
            page_attn<D, W, false><<<grid, dim3(64 * W), 0, s>>>(a);
        } else {
            page_attn<D, W, true><<<grid, dim3(64 * W), 0, s>>>(a);
            page_attn_combine<D><<<dim3((unsigned)((a.M * a.Hq * (D / 4) + 255) / 256)), dim3(256), 0, s>>>(a);
        }
    };
    const auto by_waves = [&](auto d) {
        if (p.waves == 8) go(d, std::integral_constant<int, 8>{});
        else              go(d, std::integral_constant<int, 4>{});
    };
    if (c.head_dim == 64) by_waves(std::integral_constant<int, 64>{});
    else                  by_waves(std::integral_constant<int, 128>{});
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
