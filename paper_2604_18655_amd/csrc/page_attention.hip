// Attention over a paged cache of 8 bits (see include/mlora_page_attention.h).
//
// A block takes up to 16 query vectors of one stream and one kv head.  What they may see is a list of items: pages of 64
// tokens (those of the sink, then from the window's first on), chunks of 32 tokens of the tail, chunks of 32 rows of the step.  The block's waves
// take items in turn, each by itself, and merge their results through LDS at the end; where one block is not enough for the items several
// share them, and a second kernel merges what they leave in the workspace.
//
// Pages go from memory to the matrix units as they are: codes are multiplied as whole numbers (16x16x64 products of int8, exact in
// 32 bits), nothing is widened and nothing passes through LDS.  The other side is cut into digits to the base 256, each a signed byte:
//     q = 2^(e - 21) (65536 a + 256 b + c)         e the exponent of the vector's largest magnitude: to 2^-22 of that
//     p = (65536 a + 256 b + c) / 8355711          p = exp(score - the page's largest score) in (0, 1]: to 2^-24
// so that a product of scores or outputs is three products of bytes, half the work each of one of bf16.  The weights are counted relative to
// the page's own maximum; a page's sum of weights is the sum of the very integers that multiply the values.  Scores are K . Q^T: a lane
// holds 16 keys of ONE query vector, and if the keys of a page are dealt to the products in the right order (key 16 * (i / 4) + 4 * t + i % 4 is
// row i of product t) these are the 16 that O^T += V^T . P^T wants from it.  Values are stored feature by feature for that.
// The tail and the step's rows are bf16, with scores and weights (two bf16 halves) as in tree_attention.hip.
#include <algorithm>
#include <type_traits>

#include "common.hpp"

#include "../../include/mlora_page_attention.h"

namespace mlora {

mlora_status check_page_cache(const mlora_page_cache *c);

namespace {

constexpr int P = MLORA_PAGE_TOKENS, KC = 32;            // tokens of a page, of a chunk
constexpr float UNSEEN = -__builtin_inff();
constexpr float P_ONE = 8355711.f;                       // 127 * 65536 + 127 * 256 + 127

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
    void *out;
    int Hq, Hkv, G, S, R, M;
    int pages, columns, window, sink;
    int splits;
    unsigned g_inv;                                      // ceil(2^16 / G): v / G = (v * g_inv) >> 16 for v < 512
    int out_fp32;
    float scale2;                                        // scale * log2(e)
};

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

// Four whole numbers of at most 127 * 65536 + 127 * 256 + 127 in magnitude -> their digits, a register of four bytes for each place.
struct Digits {
    unsigned a, b, c;
};
__device__ __forceinline__ Digits digits_of(int x0, int x1, int x2, int x3)
{
    const unsigned y0 = (unsigned)(x0 + 0x808080), y1 = (unsigned)(x1 + 0x808080), y2 = (unsigned)(x2 + 0x808080), y3 = (unsigned)(x3 + 0x808080);
    const unsigned lo01 = __builtin_amdgcn_perm(y1, y0, 0x05010400u), lo23 = __builtin_amdgcn_perm(y3, y2, 0x05010400u);   // {b0 b0 b1 b1}
    const unsigned hi01 = __builtin_amdgcn_perm(y1, y0, 0x0C0C0602u), hi23 = __builtin_amdgcn_perm(y3, y2, 0x0C0C0602u);
    return Digits{__builtin_amdgcn_perm(hi23, hi01, 0x05040100u) ^ 0x80808080u, __builtin_amdgcn_perm(lo23, lo01, 0x07060302u) ^ 0x80808080u,
                  __builtin_amdgcn_perm(lo23, lo01, 0x05040100u) ^ 0x80808080u};
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
__global__ __launch_bounds__(64 * W, 2) void page_attn(const AttnArgs a)
{
    using L = WaveLds<D>;
    constexpr int DK = D / 64, DB = D / 16, VI = KC * D / 512;
    __shared__ __align__(16) unsigned char smem[W * L::BYTES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const int hk = blockIdx.x, s = SPLIT ? (int)blockIdx.z / a.splits : (int)blockIdx.z, z = SPLIT ? (int)blockIdx.z - s * a.splits : 0;
    const int n_qv = a.R * a.G, qv0 = (int)blockIdx.y * 16;

    // the items
    const int len = min(max(a.len[s], 0), P * a.columns + P - 1), slot = min(max(a.slot[s], 0), a.S - 1);
    const int full = len / P, n_tail = len % P;
    const int first = a.window > 0 ? min(max(len - a.window + 1, 0) / P, full) : 0, sinks = min((a.sink + P - 1) / P, first);
    const int n_pages = sinks + full - first, tail_chunks = (n_tail + KC - 1) / KC, end_t = n_pages + tail_chunks;
    const int items = end_t + (a.R + KC - 1) / KC;
    const int *const table = a.table + (size_t)slot * a.columns;
    const auto page_of = [&](int i) { return i < sinks ? i : first + i - sinks; };

    // this lane's query vector, its row and position
    const int vec = min(qv0 + l16, n_qv - 1), row = (int)((unsigned)vec * a.g_inv >> 16);
    const uint16_t *const q_at = a.q + ((size_t)(s * a.R + row) * a.Hq + hk * a.G + (vec - row * a.G)) * D;
    u32x4 qd[3][DK];
    float unit;                                          // score of a product of codes, but for the page's scale
    {
        u32x4 x[DK][2];
        unsigned top = 0;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[kk][i] = *reinterpret_cast<const u32x4 *>(q_at + 64 * kk + 16 * lq + 8 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) top = max(top, max(x[kk][i][j] & 0x7FFFu, x[kk][i][j] >> 16 & 0x7FFFu));
            }
        top = __float_as_uint(over_quarters(__uint_as_float(top), [](float p, float r) { return __uint_as_float(max(__float_as_uint(p), __float_as_uint(r))); }));
        const int e = (int)max(top >> 7, 1u) - 127;
        const bool ok = top < 0x7F80u;
        unit = ok ? __builtin_ldexpf(a.scale2, e - 21) : __builtin_nanf("");
#pragma unroll
        for (int kk = 0; kk < DK; ++kk)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                int n[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned pair = x[kk][w / 2][2 * (w % 2) + j / 2];
                    const float f = __builtin_ldexpf(bf16_bits_to_float(j & 1 ? pair >> 16 : pair & 0xFFFFu), 21 - e);
                    n[j] = ok ? (int)rintf(f) : 0;
                }
                const Digits d = digits_of(n[0], n[1], n[2], n[3]);
                qd[0][kk][w] = d.a, qd[1][kk][w] = d.b, qd[2][kk][w] = d.c;
            }
    }
    // lane r: the rows that row r may see, itself and what it continues (a parent must be an earlier row: the walk strictly
    // descends, so it ends and stays in bounds whatever the array holds)
    unsigned anc_lo = lane < 32 ? 1u << lane : 0u, anc_hi = lane >= 32 ? 1u << (lane - 32) : 0u;
    if (a.R > 1) {
        const int up0 = lane < a.R ? a.parent[s * a.R + lane] : -1;
        int r = lane < a.R && up0 < lane ? up0 : -1;
        while (__ballot(r >= 0)) {
            if (r >= 0) {
                anc_lo |= r < 32 ? 1u << r : 0u;
                anc_hi |= r >= 32 ? 1u << (r - 32) : 0u;
            }
            const int up = __shfl(up0, max(r, 0));
            r = r >= 0 && up < r ? up : -1;
        }
    }
    const int depth = __popc(anc_lo) + __popc(anc_hi) - 1;             // of row `lane`
    const unsigned sees_lo = (unsigned)__shfl((int)anc_lo, row), sees_hi = (unsigned)__shfl((int)anc_hi, row);
    const int since = a.window > 0 ? len + __shfl(depth, row) - a.window + 1 : 0;      // positions that the row sees begin here, but for the sink
    int latest = since;                                                                // of all rows of the tile
#pragma unroll
    for (int d = 1; d < 16; d *= 2) latest = max(latest, __shfl_xor(latest, d));

    float m = UNSEEN, l = 0.f;                           // l: of the lane's own keys
    f32x4 o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) o[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    int c = z * W + wave;
    const int stride = SPLIT ? a.splits * W : W;

    // pages
    const size_t unit_bytes = (size_t)P * D;
    for (; c < n_pages; c += stride) {
        const int i = page_of(c), page = table[i];
        if (page < 0 || page >= a.pages) continue;
        const size_t at = (size_t)page * a.Hkv + hk;
        const int8_t *const kp = a.k + at * unit_bytes + (16 * (l16 >> 2) + (l16 & 3)) * D + 16 * lq;
        const int8_t *const vp = a.v + at * unit_bytes + l16 * P + 16 * lq;
        u32x4 kf[4][DK], vf[DB];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int kk = 0; kk < DK; ++kk) kf[t][kk] = *reinterpret_cast<const u32x4 *>(kp + 4 * t * D + 64 * kk);
        const float ks = a.k_scale[at], vs = a.v_scale[at];
#pragma unroll
        for (int db = 0; db < DB; ++db) vf[db] = *reinterpret_cast<const u32x4 *>(vp + 16 * db * P);
        // scores: element e of sc[t] is key 16 * lq + 4 * t + e
        f32x4 sc[4];
        float per = unit * ks;
        const bool bad = !(fabsf(per) < __builtin_inff());
        if (bad) per = 0.f;                              // (a query vector or a page that is not finite: whoever sees a token becomes NaN below)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            i32x4 x[3];
#pragma unroll
            for (int g = 0; g < 3; ++g) {
                x[g] = i32x4{0, 0, 0, 0};
#pragma unroll
                for (int kk = 0; kk < DK; ++kk) x[g] = mfma_i8(kf[t][kk], qd[g][kk], x[g]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[t][e] = ((float)((x[0][e] << 8) + x[1][e]) * 256.f + (float)x[2][e]) * per;
        }
        const int t0 = i * P;
        if (t0 < latest && t0 + P > a.sink) {
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
        // weights relative to the page's maximum, as whole numbers
        const float from = finite_or_0(top);
        int sum = 0;
        u32x4 pd[3];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            int n[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                n[e] = (int)rintf(__builtin_amdgcn_exp2f(sc[t][e] - from) * P_ONE);
                sum += n[e];
            }
            const Digits d = digits_of(n[0], n[1], n[2], n[3]);
            pd[0][t] = d.a, pd[1][t] = d.b, pd[2][t] = d.c;
        }
        const float m_new = fmaxf(m, top), base = finite_or_0(m_new), keep = __builtin_amdgcn_exp2f(m - base);
        float w = __builtin_amdgcn_exp2f(top - base) * (1.f / P_ONE);
        if (bad && top != UNSEEN) w = __builtin_nanf("");
        m = m_new;
        l = l * keep + (float)sum * w;
        const float wv = top != UNSEEN ? w * vs : 0.f;   // (a page of NaN that the row does not see)
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            i32x4 x[3];
#pragma unroll
            for (int g = 0; g < 3; ++g) x[g] = mfma_i8(vf[db], pd[g], i32x4{0, 0, 0, 0});
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][e] = o[db][e] * keep + ((float)((x[0][e] << 8) + x[1][e]) * 256.f + (float)x[2][e]) * wv;
        }
    }

    // chunks of the tail and of the step's rows
    unsigned char *const mine = smem + wave * L::BYTES;
    unsigned char *const v_in = mine + (lane / (D / 8)) * L::VROW + (lane % (D / 8)) * 16;
    using Lds4 = __attribute__((address_space(3))) s16x4;
    const unsigned char *const v_out = mine + (4 * lq + (l16 >> 2)) * L::VROW + (l16 & 3) * 8;
    for (; c < items; c += stride) {
        const bool tail = c < end_t;
        const int k0 = (tail ? c - n_pages : c - end_t) * KC, n = min((tail ? n_tail : a.R) - k0, KC), pitch = tail ? D : a.Hkv * D;
        const size_t at = tail ? (((size_t)slot * a.Hkv + hk) * P + k0) * D : ((size_t)(s * a.R + k0) * a.Hkv + hk) * D;
        const uint16_t *const kp = (tail ? a.k_tail : a.k_new) + at, *const vp = (tail ? a.v_tail : a.v_new) + at;
        // scores: element e of sc[j] is key 16 * j + 4 * lq + e
        f32x4 sc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            const uint4 qf = *reinterpret_cast<const uint4 *>(q_at + 32 * kk + 8 * lq);
#pragma unroll
            for (int j = 0; j < 2; ++j) sc[j] = mfma16(*reinterpret_cast<const uint4 *>(kp + (unsigned)min(16 * j + l16, n - 1) * (unsigned)pitch + 32 * kk + 8 * lq), qf, sc[j]);
        }
        u32x4 vr[VI];
        unsigned odd = 0;                                // values that are not finite (what a row does not see is weighed with 0)
#pragma unroll
        for (int u = 0; u < VI; ++u) {
            const int piece = u * 64 + lane;
            vr[u] = *reinterpret_cast<const u32x4 *>(vp + (unsigned)min(piece / (D / 8), n - 1) * (unsigned)pitch + (piece % (D / 8)) * 8);
        }
#pragma unroll
        for (int u = 0; u < VI; ++u) {
#pragma unroll
            for (int j = 0; j < 4; ++j) odd |= (unsigned)((vr[u][j] & 0x7F80u) == 0x7F80u) | (unsigned)((vr[u][j] & 0x7F800000u) == 0x7F800000u);
            *reinterpret_cast<u32x4 *>(v_in + u * (512 / D) * L::VROW) = vr[u];
        }
        unsigned see;
        if (tail) {
            see = n < KC ? (1u << n) - 1 : ~0u;
            const int p0 = full * P + k0, skip = min(max(since - p0, 0), KC), still = min(max(a.sink - p0, 0), KC);
            see &= (skip < KC ? ~0u << skip : 0u) | (still < KC ? (1u << still) - 1 : ~0u);
        } else {
            see = k0 == 0 ? sees_lo : sees_hi;
            if (a.window > 0) {                          // the rows of the path whose positions the window has left behind
                for (int j = 0; j < n; ++j) {
                    const int pos = len + __shfl(depth, k0 + j);
                    if (pos < since && pos >= a.sink) see &= ~(1u << j);
                }
            }
        }
        see >>= 4 * lq;
        float top = m;
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
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                p[j][e] = __builtin_amdgcn_exp2f(sc[j][e] - base);
                sum += p[j][e];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                hi[2 * j + i] = pack_bf16(p[j][2 * i], p[j][2 * i + 1]);
                lo[2 * j + i] = pack_bf16(p[j][2 * i] - bf16_bits_to_float(hi[2 * j + i] & 0xFFFFu), p[j][2 * i + 1] - __uint_as_float(hi[2 * j + i] & 0xFFFF0000u));
            }
        }
        l = l * keep + sum;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[db] *= keep;
        if (!__ballot(odd)) {
            const uint4 ph = make_uint4(hi[0], hi[1], hi[2], hi[3]), pl = make_uint4(lo[0], lo[1], lo[2], lo[3]);
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4 *)(v_out + db * 32)));
                const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds4 *)(v_out + 16 * L::VROW + db * 32)));
                const uint4 vf = make_uint4(x.x, x.y, y.x, y.y);
                o[db] = mfma16(vf, ph, o[db]);
                o[db] = mfma16(vf, pl, o[db]);
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
                        const unsigned char *const v = mine + (16 * j + 4 * g + e) * L::VROW;
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
        float *const om = reinterpret_cast<float *>(mine);
        const float sum = over_quarters(l, [](float x, float y) { return x + y; });
        if (lq == 0) reinterpret_cast<float2 *>(mine + L::O_BYTES)[l16] = make_float2(m, sum);
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
        const int r = (int)((unsigned)v * a.g_inv >> 16);
        const size_t vec_at = (size_t)(s * a.R + r) * a.Hq + hk * a.G + (v - r * a.G);
        if constexpr (SPLIT) {
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
    constexpr int RB = 8;                                      // results per trip to memory
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    float den = 0.f, run_top = UNSEEN;
    for (int z0 = 0; z0 < a.splits; z0 += RB) {
        float2 ml[RB];
        f32x4 pv[RB];
#pragma unroll
        for (int u = 0; u < RB; ++u) {
            const size_t at = (size_t)min(z0 + u, a.splits - 1) * vecs + vec;
            ml[u] = a.part_ml[at];
            pv[u] = *reinterpret_cast<const f32x4 *>(a.part_out + at * D + f);
        }
        float top = run_top;
#pragma unroll
        for (int u = 0; u < RB; ++u) {
            if (z0 + u >= a.splits) ml[u] = make_float2(UNSEEN, 0.f), pv[u] = f32x4{0.f, 0.f, 0.f, 0.f};
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
    }
    num /= den;
    const size_t at = (size_t)vec * D + f;
    if (a.out_fp32) *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) + at) = num;
    else *reinterpret_cast<uint2 *>(reinterpret_cast<uint16_t *>(a.out) + at) = make_uint2(pack_bf16(num[0], num[1]), pack_bf16(num[2], num[3]));
}

bool misaligned(const void *p, unsigned mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }

// How a call is cut.
struct Plan {
    int waves, splits;
};
constexpr int MOST_SPLITS = 64;
long long most_items(const mlora_page_attn &t)
{
    const long long pages = t.cache.max_pages;
    const long long seen = t.window > 0 ? std::min(pages, (long long)t.window / P + 2 + ((long long)t.sink + P - 1) / P) : pages;
    return seen + 2 + (t.rows_per_stream + KC - 1) / KC;
}
Plan plan_of(const mlora_page_attn &t)
{
    Plan p;
    const long long items = most_items(t);
    const int qv = t.rows_per_stream * (t.n_q_heads / t.cache.n_kv_heads);
    const long long blocks = (long long)t.cache.n_kv_heads * t.cache.n_streams * ((qv + 15) / 16);
    p.waves = 4;
    const long long wanted = std::max(1ll, std::min(1024 / blocks, items / (2 * p.waves)));
    p.splits = (int)std::min((long long)MOST_SPLITS, wanted);
    return p;
}
size_t workspace_floats(const mlora_page_attn &t)
{
    const int splits = plan_of(t).splits;
    return splits == 1 ? 0 : (size_t)splits * t.n_q_heads * (size_t)t.cache.n_streams * t.rows_per_stream * ((size_t)t.cache.head_dim + 2);
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
    a.part_out = reinterpret_cast<float *>(workspace);
    a.part_ml = reinterpret_cast<float2 *>(a.part_out + (size_t)p.splits * a.M * a.Hq * c.head_dim);
    a.g_inv = (65536u + (unsigned)a.G - 1) / (unsigned)a.G;
    a.out_fp32 = out_dtype == MLORA_Y_FP32;
    a.scale2 = t->scale * 1.44269504088896340736f;

    hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)a.Hkv, (unsigned)((a.R * a.G + 15) / 16), (unsigned)(a.S * p.splits));
    const auto go = [&](auto d) {
        constexpr int D = decltype(d)::value, W = 4;
        if (p.splits == 1) {
            page_attn<D, W, false><<<grid, dim3(64 * W), 0, s>>>(a);
        } else {
            page_attn<D, W, true><<<grid, dim3(64 * W), 0, s>>>(a);
            page_attn_combine<D><<<dim3((unsigned)((a.M * a.Hq * (D / 4) + 255) / 256)), dim3(256), 0, s>>>(a);
        }
    };
    if (c.head_dim == 64) go(std::integral_constant<int, 64>{});
    else                  go(std::integral_constant<int, 128>{});
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
