// Attention weights of the newest rows, added to what every slot of the cache has received so far:
//
//     mass[t] = decay * mass[t] + sum over rows and query heads of exp(s[row][t] - max) / sum,   s = scale q . k
//
// A weight needs its row's maximum and sum over all keys first.  In general there are two launches: mass_stats leaves the maximum and
// sum of every query vector over each block's share of the keys, mass_add makes the scores again, key by key.  (Kept
// in between, the scores of a prompt's chunk would be gigabytes.)  Many query vectors take the wide forms of both.  Where the
// vectors are few and a block holds a stream's keys, mass_stream keeps the scores in registers and reads the keys once.
//
// Scores are products on the matrix units (16x16x32 bf16, fp32 accumulation).  A wave keeps one side in registers and its lanes
// own it (a lane's columns: its query vectors in mass_stats, its keys in mass_add), and the other side passes by, so that
// running maxima, sums and masses are a lane's own, without a trip through other lanes until the end.
//
// Query vectors are counted (stream, listed row, query head of the group): v = (s * N + j) * G + g.
#include <algorithm>
#include <type_traits>

#include "common.hpp"

#include "../../include/mlora_stream_cache.h"

namespace mlora {

namespace {

constexpr int MASS_WAVES = 4;
constexpr int KC = 32;                   // keys of a chunk in mass_stats
constexpr int BATCH = 512;               // query vectors whose maxima mass_add holds at a time
constexpr float NEG_BIG = -1.0e30f;      // "no key seen yet"
constexpr float NO_ROW = __builtin_inff();   // the maximum of a query vector that does not count: weights of 0
constexpr float FAR = 1.0995e12f;        // 2^40: how far sums may grow above their maximum before they are scaled down

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct MassArgs {
    const uint16_t *q, *k, *k_prefill;
    float *mass, *mass_prefill;
    const int *slot_pos, *len, *next_pos, *rows;
    float2 *rows_ml;                     // wide calls, and mass_stream beside a prefill segment: [L * H][vecs], maximum and 1 / sum
    int *q_row;                          // the same calls: [vecs], vector of a.q of a layer's first head (of its query heads); negative: does
                                         // not count (in wide calls ~ the place of a vector that does)
    float2 *part;                        // [L * H][p_splits + s_splits][vecs]: maximum (of scores in units of log 2) and sum
    int L, S, H, G, R, N, cap, P;        // N: listed rows of a stream
    int vecs;                            // S * N * G
    int p_splits, s_splits;              // blocks that share the keys of a query tile: prefill, stream segment
    int p_blocks, s_blocks;              // blocks of a layer and head: prefill; one stream (mass_stats)
    int p_per, s_per;                    // tiles of 16 query vectors of a block (mass_stats)
    int p_tiles, s_tiles;                // blocks of a layer and head: prefill; one stream (mass_add)
    float scale2, decay;                 // scale2 = scale * log2(e)
    float per_group, per_stream;         // 1 / G, 1 / N
};

// v / G and j / N in whole numbers (v < 2^16, j and N <= 2^12 and a little): (v + 1/2) / G lies 1 / 2G or more from the next whole number,
// farther than its roundings reach.  An integer division takes thirty instructions, in front of every look-up.
__device__ __forceinline__ int row_of(const MassArgs &a, int v) { return (int)(((float)v + 0.5f) * a.per_group); }
__device__ __forceinline__ int stream_of(const MassArgs &a, int j) { return (int)(((float)j + 0.5f) * a.per_stream); }

// listed rows of stream s that count; every wave finds it by itself
__device__ __forceinline__ int listed(const MassArgs &a, int s)
{
    if (!a.rows) return a.R;
    const int lane = threadIdx.x & 63;
    const int *const rows = a.rows + (size_t)s * a.N;
    for (int j0 = 0; j0 < a.N; j0 += 64) {
        const int r = j0 + lane < a.N ? rows[j0 + lane] : 0;
        const unsigned long long bad = __ballot(r < 0 || r >= a.R);
        if (bad) return j0 + __ffsll(bad) - 1;
    }
    return a.N;
}
// the same for one thread that looks at a row of its own: does entry j of stream s count?
__device__ __forceinline__ bool counts(const MassArgs &a, int s, int j)
{
    if (!a.rows) return true;
    const int *const rows = a.rows + (size_t)s * a.N;
    bool ok = true;
    for (int i = 0; i <= j; ++i) ok &= rows[i] >= 0 && rows[i] < a.R;
    return ok;
}
__device__ __forceinline__ size_t q_at(const MassArgs &a, int l, int h, int s, int j, int g, int D)
{
    const int r = a.rows ? a.rows[(size_t)s * a.N + j] : j;
    return ((((size_t)l * a.S + s) * a.R + r) * a.H * a.G + h * a.G + g) * D;
}

template <class Op>
__device__ __forceinline__ float over_quarters(float v, const Op &op)
{
    const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// One of two arguments of the kernel, by its value: chosen by its place, the arguments would be copied to memory for it.  The
// compiler no longer sees that they are global memory: what comes from them is read and written by the calls below.
template <class T>
__device__ __forceinline__ T *either(bool first, T *a, T *b)
{
    asm("" : "+s"(a), "+s"(b));
    return first ? a : b;
}
template <class T> using Global = __attribute__((address_space(1))) T;
__device__ __forceinline__ u32x4 global_piece(const uint16_t *p) { return *(const Global<u32x4> *)p; }
__device__ __forceinline__ float global_value(const float *p) { return *(const Global<float> *)p; }
__device__ __forceinline__ void global_put(float *p, float v) { *(Global<float> *)p = v; }

// What a block works on: a layer's and head's prefill segment or a stream's own, and a number within it.
struct Unit {
    int lh, l, h, s;
    int number;                          // of a tile of keys (the masses)
    int tile, z;                         // of query vectors, and which share of the keys (maxima and sums)
    bool prefill;
    int n, newest;                       // listed rows of the stream, and the position of the first one
    int vecs, keys;                      // query vectors and keys
    const uint16_t *k;
    const int *pos;
    size_t at;                           // of the segment's first slot
    // Blocks that share keys (a unit's tiles of query vectors) stand eight apart, on one die: its second-level cache has the
    // keys for all of them.
    __device__ __forceinline__ Unit(const MassArgs &a, int D)
    {
        int b = (int)blockIdx.x;
        const int heads = a.L * a.H, shared = heads * a.p_blocks;
        prefill = b < shared;
        if (!prefill) b -= shared;
        const int splits = prefill ? a.p_splits : a.s_splits, tiles = (prefill ? a.p_blocks : a.s_blocks) / splits;
        const int units = heads * splits * (prefill ? 1 : a.S);
        const int group = b / (8 * tiles), at_group = b - group * 8 * tiles, width = min(8, units - 8 * group);
        tile = at_group / width;
        int unit = 8 * group + at_group - tile * width;
        z = unit % splits;
        unit /= splits;
        lh = prefill ? unit : unit / a.S;
        s = prefill ? 0 : unit - lh * a.S;
        number = 0;
        rest(a, D);
    }
    __device__ __forceinline__ Unit(const MassArgs &a, int p_blocks, int s_blocks, int D)
    {
        const int per_head = p_blocks + a.S * s_blocks;
        lh = (int)blockIdx.x / per_head;
        tile = z = 0;
        number = (int)blockIdx.x - lh * per_head;
        prefill = number < p_blocks;
        s = 0;
        if (!prefill) {
            number -= p_blocks;
            s = number / s_blocks;
            number -= s * s_blocks;
        }
        rest(a, D);
    }
    __device__ __forceinline__ void rest(const MassArgs &a, int D)
    {
        l = lh / a.H;
        h = lh - l * a.H;
        keys = prefill ? a.P : max(0, min(a.len[s], a.cap));         // (asked for before the list is looked at)
        newest = prefill ? 0 : a.next_pos[s];
        n = prefill ? 0 : listed(a, s);
        newest -= n;
        vecs = prefill ? a.vecs : n * a.G;
        at = prefill ? (size_t)lh * a.P : (((size_t)l * a.S + s) * a.H + h) * a.cap;
        k = either(prefill, a.k_prefill, a.k) + at * D;
        pos = a.slot_pos + at;
    }
    // place of query vector v's features in a.q, and its number over all streams; false: it does not count
    __device__ __forceinline__ bool vector(const MassArgs &a, int v, int D, size_t &q, int &number_of) const
    {
        const int j = row_of(a, v), g = v - j * a.G;
        int st = s, row = j;
        if (prefill) st = stream_of(a, j), row = j - st * a.N;
        number_of = (st * a.N + row) * a.G + g;
        q = 0;
        if (prefill && !counts(a, st, row)) return false;
        q = q_at(a, l, h, st, row, g, D);
        return true;
    }
    // the same in two steps, where it may be any vector if v does not count
    __device__ __forceinline__ int listed_row(const MassArgs &a, int v) const
    {
        const int j = row_of(a, v);
        return a.rows ? a.rows[(prefill ? 0 : (size_t)s * a.N) + j] : prefill ? j - stream_of(a, j) * a.N : j;      // (of all streams, one behind the other)
    }
    __device__ __forceinline__ size_t some_vector(const MassArgs &a, int v, int row, int D) const
    {
        const int j = row_of(a, v), g = v - j * a.G, st = prefill ? stream_of(a, j) : s;
        row = row >= 0 && row < a.R ? row : 0;
        return ((((size_t)l * a.S + st) * a.R + row) * a.H * a.G + h * a.G + g) * D;
    }
    __device__ __forceinline__ size_t some_vector(const MassArgs &a, int v, int D) const { return some_vector(a, v, listed_row(a, v), D); }
};

// Maximum and sum of QT tiles of 16 query vectors over a share of the keys.
template <int D, int QT>
__device__ __forceinline__ void stats_tiles(const MassArgs &a, const Unit &w, float2 (*ml)[128])
{
    constexpr int DK = D / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lq = lane >> 4;
    const int splits = w.prefill ? a.p_splits : a.s_splits, tile = w.tile, z = w.z;
    const int per = w.prefill ? a.p_per : a.s_per, v0 = tile * per * 16, v_end = min(w.vecs, v0 + per * 16);
    if (v0 >= w.vecs) return;

    // keys as A operands (past the end: the last key), some chunks ahead of the one that is worked on
    struct Keys {
        uint4 f[KC / 16][DK];
        int pos;
    };
    const int chunks = (w.keys + KC - 1) / KC, stride = splits * MASS_WAVES;
    const auto ask = [&](Keys &x, int c) {
        const int k0 = c * KC, last = w.keys - 1;
#pragma unroll
        for (int j = 0; j < KC / 16; ++j) {
            const uint16_t *const kp = w.k + (size_t)min(k0 + 16 * j + l16, last) * D + 8 * lq;
#pragma unroll
            for (int kk = 0; kk < DK; ++kk) x.f[j][kk] = __builtin_bit_cast(uint4, global_piece(kp + 32 * kk));
        }
        x.pos = w.prefill ? 0 : w.pos[min(k0 + (lane & 31), last)];
    };
    // this lane's query vectors (B operands: lane (l16, lq) holds features 8 * lq .. of vector l16 of a tile).  Loads return in
    // their order: the rows' places first, a chunk of keys on its way beside them, the vectors, and the other chunks behind, because
    // the vectors are what all products need.
    constexpr int AHEAD = D == 64 ? 4 : 2;                           // chunks on their way
    Keys ring[AHEAD];
    int c = z * MASS_WAVES + wave;
    int listed_row[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) listed_row[t] = w.listed_row(a, min(v0 + 16 * t + l16, w.vecs - 1));
    if (c < chunks) ask(ring[0], c);
    uint4 qf[QT][DK];
    float m[QT], sum[QT];
    int pos[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int v = min(v0 + 16 * t + l16, w.vecs - 1);
        const size_t q = w.some_vector(a, v, listed_row[t], D);
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) qf[t][kk] = *reinterpret_cast<const uint4 *>(a.q + q + 8 * lq + 32 * kk);
        pos[t] = w.newest + row_of(a, v);
        m[t] = NEG_BIG;
        sum[t] = 0.f;
    }
#pragma unroll
    for (int i = 1; i < AHEAD; ++i)
        if (c + i * stride < chunks) ask(ring[i], c + i * stride);
    const auto work = [&](const Keys &x, int c) {
        const int nk = min(KC, w.keys - c * KC);
        const bool masked = nk < KC || (!w.prefill && __any(x.pos > w.newest));
        // Hidden scores are minus infinity at any scale.  Scores are scaled in the multiply-add of the exponential, as mass_add does: one
        // that had been rounded before would not be the one that is weighed (of 10^7, by as much as 2^0.9).
        const float factor = masked && a.scale2 == 0.f ? 1.f : a.scale2, kept = a.scale2 == 0.f ? 0.f : 1.f;
        const float hidden = a.scale2 < 0.f ? __builtin_inff() : -__builtin_inff();
        // (all tiles side by side, whether their vectors count or not: one after the other, each waits for its products)
        f32x4 sc[QT][KC / 16];
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int j = 0; j < KC / 16; ++j) {
                sc[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < DK; ++kk) sc[t][j] = mfma16(x.f[j][kk], qf[t][kk], sc[t][j]);
            }
        if (masked) {
#pragma unroll
            for (int j = 0; j < KC / 16; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = 16 * j + 4 * lq + e;
                    const int key_pos = __shfl(x.pos, key);          // (all lanes: before any condition)
#pragma unroll
                    for (int t = 0; t < QT; ++t)
                        sc[t][j][e] = key < nk && (w.prefill || key_pos <= pos[t]) ? sc[t][j][e] * kept : hidden;
                }
        }
        // Sums relative to maxima that may lie behind: the sums themselves tell when one does too far (the first chunk, and rarely
        // another), and they are made again.
        float add[QT], most;
        const auto take = [&](float by) {
            most = 0.f;
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                float of[2] = {0.f, 0.f};
#pragma unroll
                for (int j = 0; j < KC / 16; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) of[e & 1] += __builtin_amdgcn_exp2f(fmaf(sc[t][j][e], by, -m[t]));
                add[t] = of[0] + of[1];
                most = fmaxf(most, add[t]);
            }
        };
        take(factor);
        if (__any(most > FAR)) {
            float by = factor;
            asm volatile("" : "+v"(by));                             // (products that only this path needs are made here)
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                float top = m[t];
#pragma unroll
                for (int j = 0; j < KC / 16; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[t][j][e] * by);
                sum[t] *= __builtin_amdgcn_exp2f(m[t] - top);
                m[t] = top;
            }
            take(by);
        }
#pragma unroll
        for (int t = 0; t < QT; ++t) sum[t] += add[t];
    };
    while (c < chunks) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (c >= chunks) break;
            work(ring[i], c);
            if (c + AHEAD * stride < chunks) ask(ring[i], c + AHEAD * stride);
            c += stride;
        }
    }
    // the quarters' keys, then the waves'
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const float top = over_quarters(m[t], [](float x, float y) { return fmaxf(x, y); });
        const float all = over_quarters(sum[t] * __builtin_amdgcn_exp2f(m[t] - top), [](float x, float y) { return x + y; });
        if (lq == 0) ml[wave][16 * t + l16] = make_float2(top, all);
    }
    __syncthreads();
    const int v = v0 + (int)threadIdx.x;
    if (threadIdx.x < QT * 16 && v < v_end) {
        float top = NEG_BIG, all = 0.f;
#pragma unroll
        for (int i = 0; i < MASS_WAVES; ++i) top = fmaxf(top, ml[i][threadIdx.x].x);
#pragma unroll
        for (int i = 0; i < MASS_WAVES; ++i) all += ml[i][threadIdx.x].y * __builtin_amdgcn_exp2f(ml[i][threadIdx.x].x - top);
        const int row = (w.prefill ? 0 : a.p_splits) + z;
        a.part[((size_t)w.lh * (a.p_splits + a.s_splits) + row) * a.vecs + (w.prefill ? v : w.s * a.N * a.G + v)] = make_float2(top, all);
    }
}

template <int D, int PT, int QT>
__global__ __launch_bounds__(64 * MASS_WAVES, 2) void mass_stats(const MassArgs a)
{
    __shared__ float2 ml[MASS_WAVES][128];
    const Unit w(a, D);
    if (PT != QT && w.prefill) stats_tiles<D, PT>(a, w, ml);
    else                       stats_tiles<D, QT>(a, w, ml);
}

// a value combined over the 16 lanes of a quarter of the wave; every lane gets the result
template <class Op>
__device__ __forceinline__ float over_sixteen(float v, const Op &op)
{
    const auto ror = [](float x, auto n) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + decltype(n)::value, 0xF, 0xF, false));
    };
    v = op(v, ror(v, std::integral_constant<int, 8>{}));
    v = op(v, ror(v, std::integral_constant<int, 4>{}));
    v = op(v, ror(v, std::integral_constant<int, 2>{}));
    return op(v, ror(v, std::integral_constant<int, 1>{}));
}

// maximum and sum over what blocks left, four trips at a time
__device__ __forceinline__ void merge_parts(const float2 *part, int n, int stride, float &top, float &all)
{
    for (int z0 = 0; z0 < n; z0 += 4) {
        float2 x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = part[(size_t)min(z0 + u, n - 1) * stride];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if (z0 + u >= n) break;
            const float t2 = fmaxf(top, x[u].x);
            all = all * __builtin_amdgcn_exp2f(top - t2) + x[u].y * __builtin_amdgcn_exp2f(x[u].x - t2);
            top = t2;
        }
    }
}
// Maximum and 1 / sum of a row that counts; of one that sees nothing: 0.  Where the sum is NaN, 1 / sum is all that matters, and the
// maximum may be plus infinity, NO_ROW: it is not handed on.
__device__ __forceinline__ float2 counting_row(float top, float all)
{
    return make_float2(all == all ? top : 0.f, all > 0.f ? 1.f / all : all);
}
// the same of a query vector over all blocks that looked at its keys
__device__ __forceinline__ float2 whole_row(const MassArgs &a, int lh, int number)
{
    const int splits = a.p_splits + a.s_splits;
    float top = NEG_BIG, all = 0.f;
    merge_parts(a.part + (size_t)lh * splits * a.vecs + number, splits, a.vecs, top, all);
    return counting_row(top, all);
}

// One block: KT tiles of 16 keys per wave against all query vectors that may see them.  TABLE: their maxima, sums and places have been
// written down (mass_stream).
// SHARE: as many waves have the same keys, and take every SHARE-th tile of vectors each.
template <int D, int KT, bool TABLE, int SHARE>
__global__ __launch_bounds__(64 * MASS_WAVES * SHARE, 2) void mass_add(const MassArgs a)
{
    constexpr int DK = D / 32, KEYS = MASS_WAVES * KT * 16;
    __shared__ __align__(16) float top_of[BATCH], inv_of[BATCH];
    __shared__ int pos_of[BATCH];
    __shared__ const uint16_t *q_of[BATCH];
    const int tid = threadIdx.x, lane = tid & 63, all_waves = __builtin_amdgcn_readfirstlane(tid >> 6), wave = all_waves % MASS_WAVES, share = all_waves / MASS_WAVES, l16 = lane & 15, lq = lane >> 4;
    const Unit w(a, a.p_tiles, a.s_tiles, D);
    if (w.number * KEYS >= w.keys) return;
    const int k0 = w.number * KEYS + wave * KT * 16;

    const auto look_up = [&](int base, int pad) {
        if constexpr (!TABLE) {
            // Few vectors, of which many blocks had a share: sixteen lanes take turns with what these left, sixteen vectors at a time, where
            // that is fewer trips than a lane by itself makes, four parts at a time (one row on 2176 keys, nine parts: 5.6 -> 5.0 us;
            // three on 12000, both launches: 21.0 -> 16.3).
            const int splits = a.p_splits + a.s_splits;
            if (pad < 4 * splits) {
                for (int i = tid >> 4; i < pad; i += 4 * MASS_WAVES * SHARE) {
                    size_t q;
                    int number;
                    const int v = min(base + i, w.vecs - 1);
                    const bool ok = w.vector(a, v, D, q, number) && base + i < w.vecs;
                    float top = NEG_BIG, all = 0.f;
                    if (l16 < splits) merge_parts(a.part + ((size_t)w.lh * splits + l16) * a.vecs + number, (splits - l16 + 15) / 16, 16 * a.vecs, top, all);
                    const float most = over_sixteen(top, [](float x, float y) { return fmaxf(x, y); });
                    all = over_sixteen(all * __builtin_amdgcn_exp2f(top - most), [](float x, float y) { return x + y; });
                    if (l16 == 0) {
                        const float2 row = counting_row(most, all);
                        top_of[i] = ok ? row.x : NO_ROW;
                        inv_of[i] = ok ? row.y : 0.f;
                        pos_of[i] = ok ? w.newest + row_of(a, v) : (int)0x80000000;
                        q_of[i] = a.q + q;
                    }
                }
                return;
            }
        }
        for (int i = tid; i < pad; i += 64 * MASS_WAVES * SHARE) {
            const int v = min(base + i, w.vecs - 1);
            if constexpr (TABLE) {
                const float2 row = a.rows_ml[(size_t)w.lh * a.vecs + v];
                const int at_row = a.q_row[v];
                const bool ok = at_row >= 0 && base + i < w.vecs;
                top_of[i] = ok ? row.x : NO_ROW;
                inv_of[i] = ok ? row.y : 0.f;
                q_of[i] = a.q + (((size_t)w.l * a.S * a.R * a.H + w.h) * a.G + max(at_row, 0)) * D;
            } else {
                size_t q;
                int number;
                const bool ok = w.vector(a, v, D, q, number) && base + i < w.vecs;
                const float2 row = ok ? whole_row(a, w.lh, number) : make_float2(NO_ROW, 0.f);
                top_of[i] = row.x;
                inv_of[i] = row.y;
                pos_of[i] = ok ? w.newest + row_of(a, v) : (int)0x80000000;
                q_of[i] = a.q + q;
            }
        }
    };
    // (the first vectors are looked up before the keys are asked for: loads return in their order)
    look_up(0, (min(BATCH, w.vecs) + 15) / 16 * 16);

    // this lane's keys (B operands)
    uint4 kf[KT][DK];
    int at[KT];
    float acc[KT], old[KT];
    float *const mass = either(w.prefill, a.mass_prefill, a.mass) + w.at;
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        const int key = min(k0 + 16 * t + l16, w.keys - 1);
        old[t] = global_value(mass + key);
        const uint16_t *const kp = w.k + (size_t)key * D + 8 * lq;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) kf[t][kk] = __builtin_bit_cast(uint4, global_piece(kp + 32 * kk));
        at[t] = w.prefill ? 0 : w.pos[key];
        acc[t] = 0.f;
    }

    bool counted = false;                                            // any vector counts: without, a NaN key is no reason for a NaN
    for (int base = 0; base < w.vecs; base += BATCH) {
        const int here = min(BATCH, w.vecs - base), pad = (here + 15) / 16 * 16;
        if (base > 0) {
            __syncthreads();
            look_up(base, pad);
        }
        __syncthreads();
        bool masked = false;
#pragma unroll
        for (int t = 0; t < KT; ++t) masked |= !w.prefill && at[t] > w.newest;
        masked = __any(masked);
        // query vectors as A operands, a tile ahead: element e of a score belongs to vector 4 * lq + e
        // (in the place of one that does not count, another of the tile: it has no weight, but zeros times an infinite key would be NaN,
        // which a vector that sees the key makes of it by itself)
        uint4 qn[DK];
        unsigned counting_next;                                      // a bit for each of the tile's that counts
        const auto ask = [&](int t0) {
            const int first = min(t0, pad - 16);
            counting_next = (unsigned)__ballot(top_of[first + l16] != NO_ROW) & 0xFFFFu;
            const int from = counting_next >> l16 & 1 || !counting_next ? l16 : __ffs(counting_next) - 1;
            const uint16_t *const qp = q_of[first + from] + 8 * lq;
#pragma unroll
            for (int kk = 0; kk < DK; ++kk) qn[kk] = __builtin_bit_cast(uint4, global_piece(qp + 32 * kk));
        };
        ask(16 * share);
        for (int t0 = 16 * share; t0 < pad; t0 += 16 * SHARE) {
            uint4 qf[DK];
#pragma unroll
            for (int kk = 0; kk < DK; ++kk) qf[kk] = qn[kk];
            const bool none = counting_next == 0;
            ask(t0 + 16 * SHARE);
            if (none) continue;
            counted = true;
            const f32x4 top = *reinterpret_cast<const f32x4 *>(top_of + t0 + 4 * lq), inv = *reinterpret_cast<const f32x4 *>(inv_of + t0 + 4 * lq);
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < DK; ++kk) sc = mfma16(qf[kk], kf[t][kk], sc);
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], a.scale2, -top[e]));
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float with = fmaf(sc[e], inv[e], acc[t]);
                        acc[t] = at[t] > pos_of[t0 + 4 * lq + e] ? acc[t] : with;      // (a NaN row spoils what it sees, no more)
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[t] = fmaf(sc[e], inv[e], acc[t]);
                }
            }
        }
    }
    __shared__ float others[SHARE > 1 ? SHARE - 1 : 1][MASS_WAVES][KT][16];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        acc[t] = counted ? over_quarters(acc[t], [](float x, float y) { return x + y; }) : 0.f;
        if (SHARE > 1 && share > 0 && lq == 0) others[share - 1][wave][t][l16] = acc[t];
    }
    if (SHARE > 1) {
        __syncthreads();
        if (share > 0) return;
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        float add = acc[t];
#pragma unroll
        for (int i = 1; i < SHARE; ++i) add += others[i - 1][wave][t][l16];
        const int key = k0 + 16 * t + l16;
        if (lq == 0 && key < w.keys) global_put(mass + key, a.decay * old[t] + add);
    }
}

// Few query vectors (VT tiles of 16) on keys that a block holds at once: its scores stay in registers, and one pass over the keys is
// all there is.  The keys are a stream's own segment; where several streams share a prefill segment, its maxima and sums are
// there already (mass_stats) and what its masses need is left behind; where the stream is the only one (ALONE) they are the
// block's as well, in front of the others.
template <int D, int VT, int TK, int W, bool ALONE>
__global__ __launch_bounds__(64 * W) void mass_stream(const MassArgs a)
{
    constexpr int DK = D / 32, AHEAD = D == 64 ? (TK < 4 ? TK : 4) : 2, V = 16 * VT, GROUPS = (TK + 3) / 4;
    __shared__ __align__(16) float tops[W][V], sums[W][V], p_top[V], p_sum[V];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const Unit w(a, 0, 1, D);
    // tiles of 16 keys: wave, wave + W, ..; first those of the prefill segment.  Past a segment's end: its last key.
    const int p_tiles = ALONE ? (a.P + 15) / 16 : 0;
    struct Key {
        bool prefill, live;
        int at;                                                      // in its segment
    };
    const auto key_of = [&](int t) {
        const int tile = t * W + wave;
        Key k;
        k.prefill = ALONE && tile < p_tiles;
        const int key = (k.prefill ? tile : tile - p_tiles) * 16 + l16, keys = k.prefill ? a.P : w.keys;
        k.live = key < keys;
        k.at = min(key, max(keys - 1, 0));
        return k;
    };
    const auto tile_lives = [&](int t) {
        const int tile = t * W + wave;
        return ALONE && tile < p_tiles ? true : (tile - p_tiles) * 16 < w.keys;
    };
    const uint16_t *const pk = ALONE ? a.k_prefill + (size_t)w.lh * a.P * D : nullptr;
    float *const mass = a.mass + w.at, *const p_mass = ALONE ? a.mass_prefill + (size_t)w.lh * a.P : nullptr;
    // (vectors and what the prefill segment left come before the keys: loads return in their order.  In the place of a vector
    // that does not count stands the last one that does: without weight, but zeros times an infinite key would be NaN.)
    uint4 qf[VT][DK];
#pragma unroll
    for (int v = 0; v < VT; ++v) {
        const size_t q = w.some_vector(a, min(16 * v + l16, max(w.vecs, 1) - 1), D);
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) qf[v][kk] = *reinterpret_cast<const uint4 *>(a.q + q + 8 * lq + 32 * kk);
    }
    const int own = w.s * a.N * a.G;
    if (tid < V) {
        // this vector on the prefill segment
        float top = NEG_BIG, all = 0.f;
        if (!ALONE && tid < w.vecs && a.P > 0) merge_parts(a.part + (size_t)w.lh * a.p_splits * a.vecs + own + tid, a.p_splits, a.vecs, top, all);
        p_top[tid] = top;
        p_sum[tid] = all;
    }
    uint4 kf[AHEAD][DK];
    int at[TK];                                                      // positions; a prefill segment's lie before all
    const auto ask = [&](int t) {
        const Key k = key_of(t);
        const uint16_t *const kp = (k.prefill ? pk : w.k) + (size_t)k.at * D + 8 * lq;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) kf[t % AHEAD][kk] = __builtin_bit_cast(uint4, global_piece(kp + 32 * kk));
    };
#pragma unroll
    for (int t = 0; t < TK; ++t) {
        const Key k = key_of(t);
        at[t] = (int)0x80000000;
        if (!k.prefill) at[t] = w.pos[k.at];
    }
#pragma unroll
    for (int t = 0; t < AHEAD; ++t) ask(t);
    // Masses: a quarter of the wave takes one of four tiles.
    float old[GROUPS];
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const Key k = key_of(4 * g + lq);
        old[g] = global_value((k.prefill ? p_mass : mass) + k.at);
    }
    int pos[VT][4];
    float top[VT][4], sum[VT][4];
#pragma unroll
    for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int vec = 16 * v + 4 * lq + e;
            pos[v][e] = vec < w.vecs ? w.newest + row_of(a, vec) : (int)0x80000000;
            top[v][e] = NEG_BIG;
            sum[v][e] = 0.f;
        }
    // Scores, not yet scaled: element e of sc[v][t] is vector 16 * v + 4 * lq + e against key l16 of tile t; hidden ones are minus
    // infinity.  Tiles past the end are left out (their keys are asked for all the same: fewer loads on some ways make the
    // compiler wait for more on all).
    f32x4 sc[VT][TK];
#pragma unroll
    for (int t = 0; t < TK; ++t) {
        if (tile_lives(t)) {
#pragma unroll
            for (int v = 0; v < VT; ++v) {
                sc[v][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < DK; ++kk) sc[v][t] = mfma16(qf[v][kk], kf[t % AHEAD][kk], sc[v][t]);
            }
            const int key_pos = key_of(t).live ? at[t] : 0x7FFFFFFF;
            if (__any(key_pos > w.newest)) {
#pragma unroll
                for (int v = 0; v < VT; ++v)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sc[v][t][e] = key_pos <= pos[v][e] ? sc[v][t][e] : -__builtin_inff();
            }
#pragma unroll
            for (int v = 0; v < VT; ++v)
#pragma unroll
                for (int e = 0; e < 4; ++e) top[v][e] = fmaxf(top[v][e], sc[v][t][e]);
        }
        if (t + AHEAD < TK) ask(t + AHEAD);
    }
#pragma unroll
    for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            top[v][e] = over_sixteen(top[v][e], [](float x, float y) { return fmaxf(x, y); });
            if (l16 == 0) tops[wave][16 * v + 4 * lq + e] = top[v][e];
        }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < VT; ++v) {
        f32x4 m = *reinterpret_cast<const f32x4 *>(&tops[0][16 * v + 4 * lq]);
#pragma unroll
        for (int i = 1; i < W; ++i) {
            const f32x4 o = *reinterpret_cast<const f32x4 *>(&tops[i][16 * v + 4 * lq]);
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = fmaxf(m[e], o[e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) top[v][e] = m[e] * a.scale2;
    }
#pragma unroll
    for (int t = 0; t < TK; ++t) {
        if (!tile_lives(t)) continue;
#pragma unroll
        for (int v = 0; v < VT; ++v)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sc[v][t][e] = __builtin_amdgcn_exp2f(fmaf(sc[v][t][e], a.scale2, -top[v][e]));
                sum[v][e] += sc[v][t][e];
            }
    }
#pragma unroll
    for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sum[v][e] = over_sixteen(sum[v][e], [](float x, float y) { return x + y; });
            if (l16 == 0) sums[wave][16 * v + 4 * lq + e] = sum[v][e];
        }
    __syncthreads();
    float factor[VT][4];                                             // of a vector's weights
    bool spoils[VT][4];                                              // a NaN row spoils the slots that it sees, no more: below
#pragma unroll
    for (int v = 0; v < VT; ++v) {
        f32x4 all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < W; ++i) all += *reinterpret_cast<const f32x4 *>(&sums[i][16 * v + 4 * lq]);
        const f32x4 pt = *reinterpret_cast<const f32x4 *>(&p_top[16 * v + 4 * lq]), ps = *reinterpret_cast<const f32x4 *>(&p_sum[16 * v + 4 * lq]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int vec = 16 * v + 4 * lq + e;
            const float m = fmaxf(top[v][e], pt[e]), here = __builtin_amdgcn_exp2f(top[v][e] - m);
            const float total = all[e] * here + ps[e] * __builtin_amdgcn_exp2f(pt[e] - m), inv = total > 0.f ? 1.f / total : total;      // (NaN stays)
            const bool counts = vec < w.vecs;
            factor[v][e] = counts ? here * inv : 0.f;
            spoils[v][e] = factor[v][e] != factor[v][e];
            if (spoils[v][e]) factor[v][e] = 0.f;
            if (!ALONE && a.P > 0 && wave == 0 && l16 == 0 && vec < a.N * a.G) {
                a.rows_ml[(size_t)w.lh * a.vecs + own + vec] = make_float2(inv == inv ? m : 0.f, counts ? inv : 0.f);      // (see counting_row)
                if (w.lh == 0) {
                    const int j = row_of(a, vec);
                    a.q_row[own + vec] = counts ? (w.s * a.R + (a.rows ? a.rows[(size_t)w.s * a.N + j] : j)) * a.H * a.G + vec - j * a.G : -1;
                }
            }
        }
    }
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        float mine = 0.f;
#pragma unroll
        for (int t = 4 * g; t < TK && t < 4 * g + 4; ++t) {
            if (!tile_lives(t)) continue;
            float add = 0.f;
#pragma unroll
            for (int v = 0; v < VT; ++v)
#pragma unroll
                for (int e = 0; e < 4; ++e) add = fmaf(sc[v][t][e], factor[v][e], add);
            add = over_quarters(add, [](float x, float y) { return x + y; });
            mine = lq == t - 4 * g ? add : mine;
        }
        const Key k = key_of(4 * g + lq);
        if (k.live && 4 * g + lq < TK) global_put((k.prefill ? p_mass : mass) + k.at, a.decay * old[g] + (w.vecs > 0 ? mine : 0.f));
    }
    bool any_spoils = false;
#pragma unroll
    for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) any_spoils |= spoils[v][e];
    if (!__any(any_spoils)) return;
    int first = 4 * lq, spoiled_to = (int)0x80000000;                // (positions anew: kept from above, they cost a block per compute unit)
    asm volatile("" : "+v"(first));
#pragma unroll
    for (int v = 0; v < VT; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (spoils[v][e]) spoiled_to = max(spoiled_to, w.newest + row_of(a, 16 * v + first + e));
#pragma unroll 1
    for (int t = 0; t < TK; ++t) {                                   // (after the stores above: this wave's, to the same places)
        const Key k = key_of(t);
        if (any_spoils && k.live && (k.prefill || w.pos[k.at] <= spoiled_to)) global_put((k.prefill ? p_mass : mass) + k.at, __builtin_nanf(""));
    }
}

// ---------------------------------------------------------------------------------------------
// Many query vectors (a prompt's chunk): the side that a wave keeps is 64 vectors (or keys) in registers, the other passes by in
// chunks of 64 rows that the block's waves share through LDS, on the 32x32x16 products.  A row's 16-byte pieces are
// exchanged by its number, so that both the writes (rows side by side) and the reads (32 rows of one piece) use all banks.
// Bound by the vector unit, at the clock that products and exponentials side by side leave it: a score costs a multiply-add, an
// exponential (as long as three of them) and an addition, a tile of 32 x 32 scores half as long on the matrix unit.  512
// rows on 16384 slots, 8 heads of 128 features, 4 query heads each: 76 us for the maxima and sums, 86 for the masses (67.6
// GFLOP of products each: 0.89 and 0.79 PFLOP/s; a large library product 1.29).  Chunks that a wave's side does not see
// are passed over (the blocks of the last keys, where most are half seen or hidden, took 100 us).
// ---------------------------------------------------------------------------------------------
constexpr int WIDE_ROWS = 64;            // rows of a chunk
constexpr int WIDE_OWN = 256;            // vectors or keys of a block

template <int D>
struct Stage {
    static constexpr int PIECES = D / 8, PER = WIDE_ROWS * PIECES / 256;            // pieces of a row, of a thread
    static __device__ __forceinline__ int row(int i) { return (i * 256 + (int)threadIdx.x) / PIECES; }
    static __device__ __forceinline__ int piece() { return (int)threadIdx.x % PIECES; }
    static __device__ __forceinline__ int place(int row, int piece) { return row * PIECES + (piece ^ (D == 128 ? row & 15 : row >> 1 & 7)); }
};

// What the wave keeps is there before the loop: the compiler would wait for it inside, and for the loads on their way with it.
__device__ __forceinline__ void all_loaded() { __builtin_amdgcn_s_waitcnt(0x0F70); }              // vmcnt 0, the others unchanged

// Scores of 32 rows of a chunk against what the wave keeps: element i of sc[t] is row 8 * (i / 4) + 4 * (lane / 32) + i % 4
// against column 32 * t + lane % 32.  at[kk]: where the lane's pieces stand in the first half of the first buffer.  slice(i), i = 0 ..
// 15, is a share of the vector work on the last 32 rows' scores; product and slice are written in turn and kept so, because
// the matrix unit works beside the vector unit only if it is fed in between (two products in a row, of which the
// second waits for the first: maxima and sums of 2048 vectors on 16384 keys of 8 heads 80 us, in turn 76), and a chain of one exponential after the other waits for each.
template <int D, int BUFFER, int HALF, class Slice>
__device__ __forceinline__ void wide_scores(const u32x4 *chunks, const int (&at)[D / 16], const u32x4 (&own)[2][D / 16], f32x16 (&sc)[2], const Slice &slice)
{
    constexpr int DK = D / 16, FROM = (BUFFER * WIDE_ROWS + HALF * 32) * Stage<D>::PIECES;
    const auto piece = [&](int kk) { return __builtin_bit_cast(uint4, chunks[at[kk] + FROM]); };
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[t][i] = 0.f;
    uint4 f = piece(0);
#pragma unroll
    for (int kk = 0; kk < DK; ++kk) {
        const uint4 now = f;
        if (kk + 1 < DK) f = piece(kk + 1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            sc[t] = mfma32(now, __builtin_bit_cast(uint4, own[t][kk]), sc[t]);
#pragma unroll
            for (int i = 0; i < 8 / DK; ++i) slice((2 * kk + t) * (8 / DK) + i);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// Maximum and sum of 256 query vectors over every splits-th chunk of keys.
template <int D>
__global__ __launch_bounds__(256, 2) void mass_stats_wide(const MassArgs a)
{
    constexpr int DK = D / 16;
    using St = Stage<D>;
    __shared__ u32x4 chunk[2 * WIDE_ROWS * St::PIECES];
    __shared__ __align__(16) int key_pos[4][WIDE_ROWS];              // (read while the next but one is written)
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh2 = lane >> 5;
    const Unit w(a, D);
    const int splits = w.prefill ? a.p_splits : a.s_splits, tile = w.tile, z = w.z;
    const int v0 = tile * WIDE_OWN;
    if (v0 >= w.vecs) return;
    const int mine = v0 + wave * 64;                                 // first vector of the wave

    u32x4 qf[2][DK];
    float m[2], sum[2];
    int pos[2], at[DK];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int v = min(mine + 32 * t + l32, w.vecs - 1);
        const size_t q = w.some_vector(a, v, D);
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) qf[t][kk] = *reinterpret_cast<const u32x4 *>(a.q + q + 16 * kk + 8 * lh2);
        pos[t] = w.prefill ? 0 : w.newest + row_of(a, v);
        m[t] = NEG_BIG;
        sum[t] = 0.f;
    }
#pragma unroll
    for (int kk = 0; kk < DK; ++kk) at[kk] = St::place(l32, 2 * kk + lh2);
    const int first_pos = w.prefill ? 0 : w.newest + row_of(a, min(mine, w.vecs - 1)), last_pos = w.prefill ? 0 : w.newest + row_of(a, min(mine + 63, w.vecs - 1));
    const int chunks = (w.keys + WIDE_ROWS - 1) / WIDE_ROWS;
    u32x4 next[St::PER];
    int next_pos = 0, next_k0 = 0;
    bool masked = false, hidden = false;                             // the chunk holds keys that some of the wave's vectors do not see; no others
    // (what is loaded is not looked at here: that would wait for it)
    const auto ask = [&](int c) {
        next_k0 = min(c, chunks - 1) * WIDE_ROWS;
        const uint16_t *const rows = w.k + (size_t)next_k0 * D;
        const int last = w.keys - 1 - next_k0;
#pragma unroll
        for (int i = 0; i < St::PER; ++i) next[i] = global_piece(rows + (unsigned)(min(St::row(i), last) * D + St::piece() * 8));
        if (!w.prefill) next_pos = w.pos[next_k0 + min(lane, last)];
    };
    bool masked_next = false, hidden_next = false;
    const auto put = [&](int buffer, int c) {
#pragma unroll
        for (int i = 0; i < St::PER; ++i) chunk[buffer * WIDE_ROWS * St::PIECES + St::place(St::row(i), St::piece())] = next[i];
        // (a prefill segment hides what lies past its end)
        const int p = next_k0 + lane < w.keys ? next_pos : 0x7FFFFFFF;
        if (tid < WIDE_ROWS) key_pos[c & 3][lane] = p;
        masked_next = __any(p > first_pos);
        hidden_next = __all(p > last_pos);
    };
    const auto hide = [&](f32x16 (&sc)[2], int c, int half) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int p = key_pos[c & 3][32 * half + 8 * (i / 4) + 4 * lh2 + i % 4];
#pragma unroll
            for (int t = 0; t < 2; ++t) sc[t][i] = p <= pos[t] ? sc[t][i] : -__builtin_inff();
        }
    };
    // Sums relative to a maximum that may lie a little behind: the sum itself tells when it does too far.  A slice: two scores, and the
    // sum of the slice before.
    float more[2], e[2];
    const auto slice_of = [&](const f32x16 (&sc)[2]) {
        return [&](int i) {
            const int t = i / 8, first = i % 8 * 2;
            const float old = e[0] + e[1];
#pragma unroll
            for (int u = 0; u < 2; ++u) e[u] = __builtin_amdgcn_exp2f(fmaf(sc[t][first + u], a.scale2, -m[t]));
            if (i % 8 == 1) more[t] = old;
            else if (i > 0) more[(i - 1) / 8] += old;
        };
    };
    const auto settle = [&](const f32x16 (&sc)[2]) {
        more[1] += e[0] + e[1];
        if (__any(more[0] > FAR || more[1] > FAR)) {                 // rare, but for the first chunk: once more
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float high = sc[t][0];
#pragma unroll
                for (int i = 1; i < 16; ++i) high = fmaxf(high, sc[t][i]);
                high = fmaxf(high * a.scale2, m[t]);
                sum[t] *= __builtin_amdgcn_exp2f(m[t] - high);
                m[t] = high;
                more[t] = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) more[t] += __builtin_amdgcn_exp2f(fmaf(sc[t][i], a.scale2, -high));
            }
        }
        sum[0] += more[0];
        sum[1] += more[1];
    };
    f32x16 x[2], y[2] = {};
    if (chunks > 0) {
        ask(z);
        put(0, 0);
        masked = masked_next;
        hidden = hidden_next;
    }
    __syncthreads();
    all_loaded();
    if (chunks > 0) ask(z + splits);
    wide_scores<D, 0, 0>(chunk, at, qf, x, [](int) {});
    // a chunk: its second half's products beside its first half's exponentials, then the next chunk's first half's beside its second
    // half's (behind the last chunk: the last one again, of no use)
    const auto step = [&](auto buffer, int i) {
        constexpr int B = decltype(buffer)::value;
        if (!hidden) {
            if (masked) hide(x, i, 0);
            wide_scores<D, B, 1>(chunk, at, qf, y, slice_of(x));
            settle(x);
        }
        put(B ^ 1, i + 1);
        __syncthreads();
        ask(z + (i + 2) * splits);
        if (!hidden || !hidden_next) {                               // (a hidden chunk's second half is what it was: all of it is hidden here)
            if (masked) hide(y, i, 1);
            wide_scores<D, B ^ 1, 0>(chunk, at, qf, x, slice_of(y));
            settle(y);
        }
        masked = masked_next;
        hidden = hidden_next;
    };
    const int mine_chunks = z < chunks ? (chunks - z + splits - 1) / splits : 0;
    for (int i = 0; i < mine_chunks; i += 2) {
        step(std::integral_constant<int, 0>{}, i);
        if (i + 1 < mine_chunks) step(std::integral_constant<int, 1>{}, i + 1);
    }
    // the two halves' keys
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const float om = __shfl_xor(m[t], 32), os = __shfl_xor(sum[t], 32), high = fmaxf(m[t], om);
        const float all = sum[t] * __builtin_amdgcn_exp2f(m[t] - high) + os * __builtin_amdgcn_exp2f(om - high);
        const int v = mine + 32 * t + l32, row = (w.prefill ? 0 : a.p_splits) + z;
        if (lh2 == 0 && v < w.vecs)
            a.part[((size_t)w.lh * (a.p_splits + a.s_splits) + row) * a.vecs + (w.prefill ? v : w.s * a.N * a.G + v)] = make_float2(high, all);
    }
}

// Every query vector's maximum and 1 / sum, once for the blocks of mass_add_wide: eight lanes take turns with what the blocks of
// mass_stats_wide left (one lane by itself: 9 us for 32 of them).  A vector that does not count: a maximum that makes all weights 0.
__global__ __launch_bounds__(256) void mass_merge(const MassArgs a)
{
    const long long i = ((long long)blockIdx.x * 256 + threadIdx.x) / 8, all = (long long)a.L * a.H * a.vecs;
    const int lane = (int)threadIdx.x % 8;
    const long long at = i < all ? i : all - 1;
    const int lh = (int)(at / a.vecs), number = (int)(at - (long long)lh * a.vecs), j = row_of(a, number), splits = a.p_splits + a.s_splits;
    int s = stream_of(a, j);
    float top = NEG_BIG, sum = 0.f;
    if (lane < splits)
        merge_parts(a.part + ((size_t)lh * splits + lane) * a.vecs + number, (splits - lane + 7) / 8, 8 * a.vecs, top, sum);
    const bool ok = counts(a, s, j - s * a.N);
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        const float ot = __shfl_xor(top, d), os = __shfl_xor(sum, d), high = fmaxf(top, ot);
        sum = sum * __builtin_amdgcn_exp2f(top - high) + os * __builtin_amdgcn_exp2f(ot - high);
        top = high;
    }
    if (i >= all || lane != 0) return;
    a.rows_ml[i] = ok ? counting_row(top, sum) : make_float2(NO_ROW, 0.f);
    if (lh == 0) {
        int row = a.rows ? a.rows[j] : j - s * a.N;
        if (!ok) {
            // another row that counts, of this stream or of the next one that has any (or none does: any row)
            int t = s;
            for (int i = 0; i < a.S; ++i) {
                row = a.rows[(size_t)t * a.N];
                if (row >= 0 && row < a.R) break;
                row = 0;
                t = t + 1 < a.S ? t + 1 : 0;
            }
            s = t;
        }
        const int at = (s * a.R + row) * a.H * a.G + number - j * a.G;
        a.q_row[number] = ok ? at : ~at;
    }
}

// 256 keys of a segment against all query vectors that may see them.
template <int D>
__global__ __launch_bounds__(256, 2) void mass_add_wide(const MassArgs a)
{
    constexpr int DK = D / 16;
    using St = Stage<D>;
    __shared__ u32x4 chunk[2 * WIDE_ROWS * St::PIECES];
    __shared__ __align__(16) float top_of[4][WIDE_ROWS], inv_of[4][WIDE_ROWS];
    __shared__ __align__(16) int pos_of[4][WIDE_ROWS];
    __shared__ int counted;                                          // any vector counts: without, a NaN key is no reason for a NaN
    __shared__ long long spoiled_to;                                 // NaN rows spoil the slots that they see, no more: the last position
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, lh2 = lane >> 5;
    const Unit w(a, a.p_tiles, a.s_tiles, D);
    if (w.number * WIDE_OWN >= w.keys) return;
    if (tid == 0) counted = 0, spoiled_to = -(1ll << 40);            // (the first wave's alone, until the last chunk has gone by)
    const int k0 = w.number * WIDE_OWN + wave * 64;

    u32x4 kf[2][DK];
    int pos[2], at[DK];
    float acc[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int key = min(k0 + 32 * t + l32, w.keys - 1);
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) kf[t][kk] = global_piece(w.k + (size_t)key * D + 16 * kk + 8 * lh2);
        pos[t] = w.prefill ? 0 : w.pos[key];
        acc[t] = 0.f;
    }
#pragma unroll
    for (int kk = 0; kk < DK; ++kk) at[kk] = St::place(l32, 2 * kk + lh2);
    const bool any_hidden = !w.prefill && __any(pos[0] > w.newest || pos[1] > w.newest);          // from the first listed row, at least
    // the wave's keys are hidden from a chunk's rows, all of them
    const auto hidden_from = [&](int c) {
        if (!any_hidden) return false;
        const int last_pos = w.newest + row_of(a, min(c * WIDE_ROWS + WIDE_ROWS - 1, w.vecs - 1));
        return (bool)__all(pos[0] > last_pos && pos[1] > last_pos);
    };
    bool hidden = hidden_from(0);
    const int chunks = (w.vecs + WIDE_ROWS - 1) / WIDE_ROWS;
    const float2 *const ml = a.rows_ml + (size_t)w.lh * a.vecs + (w.prefill ? 0 : w.s * a.N * a.G);
    const int *const q_row = a.q_row + (w.prefill ? 0 : w.s * a.N * a.G);
    const uint16_t *const q = a.q + ((size_t)w.l * a.S * a.R * a.H + w.h) * a.G * D;
    u32x4 next[St::PER];
    float2 next_ml = make_float2(0.f, 0.f);
    int rows[St::PER], next_v0 = 0;                                  // where the next chunk's rows stand: a chunk ahead of them
    // (what is loaded is not looked at here: that would wait for it)
    const auto find = [&](int c) {
#pragma unroll
        for (int i = 0; i < St::PER; ++i) rows[i] = q_row[(unsigned)min(c * WIDE_ROWS + St::row(i), w.vecs - 1)];
    };
    const auto ask = [&](int c) {
        next_v0 = c * WIDE_ROWS;
        // (in the place of a row that does not count, one that does, and past the end the last: without weight, but zeros times an
        // infinite key would be NaN)
#pragma unroll
        for (int i = 0; i < St::PER; ++i)
            next[i] = *reinterpret_cast<const u32x4 *>(q + ((unsigned)max(rows[i], ~rows[i]) * D + St::piece() * 8));
        find(c + 1);
        next_ml = ml[(unsigned)min(next_v0 + lane, w.vecs - 1)];
    };
    const auto put = [&](int buffer, int c) {
#pragma unroll
        for (int i = 0; i < St::PER; ++i) chunk[buffer * WIDE_ROWS * St::PIECES + St::place(St::row(i), St::piece())] = next[i];
        if (tid < WIDE_ROWS) {
            const bool past = next_v0 + lane >= w.vecs;
            top_of[c & 3][lane] = past ? NO_ROW : next_ml.x;
            const int p = w.newest + row_of(a, next_v0 + lane);
            const bool spoils = !past && next_ml.y != next_ml.y;
            inv_of[c & 3][lane] = past || spoils ? 0.f : next_ml.y;
            const bool counts = !past && next_ml.x != NO_ROW;
            pos_of[c & 3][lane] = counts ? p : (int)0x80000000;
            if (counts) counted = 1;
            if (spoils) atomicMax(&spoiled_to, w.prefill ? 1ll << 40 : (long long)p);
        }
    };
    const auto hide = [&](f32x16 (&sc)[2], int c, int half) {
        const int first_pos = pos_of[c & 3][32 * half];
        if (!__any(pos[0] > first_pos || pos[1] > first_pos)) return;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int p = pos_of[c & 3][32 * half + 8 * (i / 4) + 4 * lh2 + i % 4];
#pragma unroll
            for (int t = 0; t < 2; ++t) sc[t][i] = pos[t] > p ? -__builtin_inff() : sc[t][i];
        }
    };
    // A slice: two scores, and the weights of the slice before.  Maxima and sums come from LDS four slices ahead.
    float e[2];
    f32x4 top, inv, old_inv = {0.f, 0.f, 0.f, 0.f}, top_next, inv_next;
    const auto slice_of = [&](const f32x16 (&sc)[2], int c, int half) {
        const float *const tops = &top_of[c & 3][32 * half + 4 * lh2], *const invs = &inv_of[c & 3][32 * half + 4 * lh2];
        top_next = *reinterpret_cast<const f32x4 *>(tops);
        inv_next = *reinterpret_cast<const f32x4 *>(invs);
        return [&, tops, invs](int i) {
            const int g = i / 4, t = i / 2 % 2, first = i % 2 * 2;               // rows 8 * g + 4 * lh2 + first and the next one
            if (i % 4 == 0) {
                old_inv = inv;
                top = top_next;
                inv = inv_next;
                if (g < 3) {
                    top_next = *reinterpret_cast<const f32x4 *>(tops + 8 * g + 8);
                    inv_next = *reinterpret_cast<const f32x4 *>(invs + 8 * g + 8);
                }
            }
            const float old[2] = {e[0], e[1]};
#pragma unroll
            for (int u = 0; u < 2; ++u) e[u] = __builtin_amdgcn_exp2f(fmaf(sc[t][4 * g + first + u], a.scale2, -top[first + u]));
            if (i > 0) {
                const int ot = (i - 1) / 2 % 2, of = (i - 1) % 2 * 2;
#pragma unroll
                for (int u = 0; u < 2; ++u) acc[ot] = fmaf(old[u], i % 4 == 0 ? old_inv[of + u] : inv[of + u], acc[ot]);
            }
        };
    };
    const auto settle = [&] {
#pragma unroll
        for (int u = 0; u < 2; ++u) acc[1] = fmaf(e[u], inv[2 + u], acc[1]);
    };
    f32x16 x[2], y[2] = {};
    if (chunks > 0) {
        find(0);
        ask(0);
        put(0, 0);
    }
    __syncthreads();
    all_loaded();
    if (chunks > 0) ask(1);
    wide_scores<D, 0, 0>(chunk, at, kf, x, [](int) {});
    const auto step = [&](auto buffer, int c) {                      // (see mass_stats_wide)
        constexpr int B = decltype(buffer)::value;
        const bool hidden_next = hidden_from(c + 1);
        if (!hidden) {
            if (any_hidden) hide(x, c, 0);
            wide_scores<D, B, 1>(chunk, at, kf, y, slice_of(x, c, 0));
            settle();
        }
        put(B ^ 1, c + 1);
        __syncthreads();
        ask(c + 2);
        if (!hidden || !hidden_next) {                               // (see mass_stats_wide)
            if (any_hidden) hide(y, c, 1);
            wide_scores<D, B ^ 1, 0>(chunk, at, kf, x, slice_of(y, c, 1));
            settle();
        }
        hidden = hidden_next;
    };
    for (int c = 0; c < chunks; c += 2) {
        step(std::integral_constant<int, 0>{}, c);
        if (c + 1 < chunks) step(std::integral_constant<int, 1>{}, c + 1);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const float sum = acc[t] + __shfl_xor(acc[t], 32), add = pos[t] <= spoiled_to ? __builtin_nanf("") : counted ? sum : 0.f;
        const int key = k0 + 32 * t + l32;
        float *const to = either(w.prefill, a.mass_prefill, a.mass) + w.at + key;
        if (lh2 == 0 && key < w.keys) global_put(to, a.decay * global_value(to) + add);
    }
}

mlora_status check(const mlora_attention_mass *d)
{
    if (!d) return MLORA_EINVAL;
    const mlora_stream_cache *c = &d->cache;
    if (c->head_dim != 64 && c->head_dim != 128) return MLORA_ESHAPE;
    if (c->n_layers <= 0 || c->n_streams <= 0 || c->n_kv_heads <= 0 || c->cap <= 0 || c->cap > MLORA_CACHE_MAX_SLOTS) return MLORA_ESHAPE;
    if ((double)c->n_layers * c->n_streams * c->n_kv_heads > MLORA_CACHE_MAX_HEADS) return MLORA_ESHAPE;
    if (d->n_q_heads <= 0 || d->n_q_heads % c->n_kv_heads != 0 || d->n_q_heads / c->n_kv_heads > 8) return MLORA_ESHAPE;
    if (d->rows_per_stream <= 0 || (long long)c->n_streams * d->rows_per_stream > MLORA_MAX_ROWS) return MLORA_ESHAPE;
    if (d->len_prefill < 0 || d->len_prefill > MLORA_CACHE_MAX_SLOTS) return MLORA_ESHAPE;
    if (!c->k || !c->mass || !c->slot_pos || !c->len || !c->next_pos) return MLORA_EINVAL;
    if (d->len_prefill > 0 && (!d->k_prefill || !d->mass_prefill)) return MLORA_EINVAL;
    if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(d->k_prefill)) & 15u) return MLORA_EALIGN;
    const void *words[] = {c->mass, c->slot_pos, c->len, c->next_pos, d->mass_prefill};
    for (const void *p : words)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return MLORA_EALIGN;
    return MLORA_OK;
}

// How a call is cut: blocks that share a query tile's keys, until the launch has about two blocks per compute unit (four: 8 streams of
// 1500 slots, 36 query vectors of 128 features 17.0 -> 19.6 us) or a block has fewer than two chunks per wave left.
struct Plan {
    bool wide;
    int stream;                          // 0, or the key tiles of a wave in mass_stream
    int stream_vecs, stream_waves;       // its vector tiles and waves
    bool alone;                          // the prefill segment is the one stream's
    int p_tiles, s_tiles;                // query tiles of a block: prefill, stream segment
    int p_splits, s_splits, p_blocks, s_blocks;
    int p_per, s_per;                    // query tiles of a block, evenly: 6 tiles are 3 and 3, not 4 and 2
    int key_tiles;                       // key tiles of a wave in mass_add
    int share;                           // waves of it that share keys
};
Plan plan_of(const mlora_attention_mass &d, int N)
{
    const mlora_stream_cache &c = d.cache;
    const int G = d.n_q_heads / c.n_kv_heads;
    const long long lh = (long long)c.n_layers * c.n_kv_heads, own = (long long)N * G, all = own * c.n_streams;
    Plan p;
    const auto ceil_div = [](long long x, long long y) { return (x + y - 1) / y; };
    // The wide products, which take three launches and 256 vectors a block, from half a tile of vectors on, and where scores times
    // vectors are many.  Of 64 features, 8 heads: 256 vectors on 3000 slots 21.5 us and by 16 vectors 19.2, on 12000 27.3 and 34.3; 800
    // on 1500 37.0 and 31.0, on 6000 39.3 and 52.3.  Of 128, 8 heads: 400 vectors on 400 slots 28.3 and 25.4, 256 on 3000 24.9
    // and 26.8, 128 on 12000 28.4 and 38.9.  The product does not part all of these: at 64 features 800 on 1500 slots (0.9 of 2^33)
    // go wide, where they lose 6 us, because 256 on 12000 (0.7 of 2^33) gain 7.  (A layer's query vectors are reached by 32-bit offsets.)
    p.wide = d.scale > 0.f && own >= WIDE_OWN / 2 && d.n_q_heads <= 1024
          && (double)lh * ((double)c.cap * own * c.n_streams + (double)d.len_prefill * all) * own >= (c.head_dim == 64 ? 0x1p32 : 0x1p29);
    // One pass where a block holds the keys: up to 16 tiles in each of eight waves (9 with 17 to 32 vectors, whose scores take twice the
    // registers), or 9 and 4 in sixteen, in which a block that is alone on its compute unit is through sooner (4, 9 and 16 are
    // built, and a number between takes the next; others were not timed).  As
    // the only launch it is always taken up to 64 tiles (32 with more vectors): 1000 keys on 8 or 32 blocks 8.6 and 8.5 us, in
    // two passes 11.5 and 11.3; 300 keys 5.6 and 9.8.  Beyond, a compute unit by itself draws too little from memory, so it
    // takes blocks: one per feature (32 blocks of 2000 keys of 64 features 11.8 and 11.5 us, 64 blocks 12.2 and 14.3; 64 blocks of
    // 1900 keys 14.6 and 14.1, 96 blocks 14.7 and 17.9; 64 blocks of 1800 keys of 128 features 18.8 and 19.8, 128 blocks 18.8
    // and 31.3).  As the second of three launches, for streams that share a prefill segment, 256 blocks (256 blocks 24.4 and
    // 25.8 us, 192 blocks 23.6 and 22.8).
    p.alone = d.len_prefill > 0 && c.n_streams == 1;
    p.stream_vecs = own <= 16 ? 1 : 2;
    const long long key_tiles = ceil_div(c.cap, 16) + (p.alone ? ceil_div(d.len_prefill, 16) : 0), stream_blocks = lh * c.n_streams;
    p.stream = 0;
    p.stream_waves = 8;
    const bool only = d.len_prefill == 0 || p.alone;
    const int few = own <= 16 ? 64 : 32;
    if (!p.wide && d.scale > 0.f && own <= 32 && (only ? key_tiles <= few || stream_blocks >= c.head_dim : stream_blocks >= 256)) {
        const int most = own <= 16 ? 16 : 9, most16 = own <= 16 ? 9 : 4;
        if (key_tiles > 32 && key_tiles <= 16 * most16 && (stream_blocks <= 256 || key_tiles > 8 * most)) p.stream_waves = 16;
        const int per_wave = (int)std::min(1000ll, ceil_div(key_tiles, p.stream_waves));
        if (per_wave <= (p.stream_waves == 16 ? most16 : most)) p.stream = per_wave <= 4 ? 4 : per_wave <= 9 ? 9 : 16;
    }
    if (!p.stream) p.alone = false;
    const auto tiles_of = [&](long long vecs) { return vecs <= 16 ? 1 : 4; };
    p.s_tiles = own <= 16 ? 1 : 4;
    p.p_tiles = tiles_of(all);
    const long long pt = d.len_prefill > 0 && !p.alone ? ceil_div(all, p.wide ? WIDE_OWN : 16 * p.p_tiles) : 0, st = ceil_div(own, p.wide ? WIDE_OWN : 16 * p.s_tiles);
    const long long blocks = std::max(1ll, lh * (pt + (p.stream ? 0 : c.n_streams * st))), want = std::max(1ll, ceil_div(512, blocks));
    const auto splits_of = [&](int keys) {
        const long long most = p.wide ? ceil_div(ceil_div(keys, WIDE_ROWS), 2) : ceil_div(ceil_div(keys, KC), 2 * MASS_WAVES);
        return (int)std::max(1ll, std::min({want, most, 32ll}));
    };
    p.p_splits = d.len_prefill > 0 && !p.alone ? splits_of(d.len_prefill) : 0;
    p.s_splits = p.stream ? 0 : splits_of(c.cap);
    p.p_per = pt > 0 ? (int)ceil_div(ceil_div(all, 16), pt) : 1;
    p.s_per = p.stream ? 1 : (int)ceil_div(ceil_div(own, 16), st);
    p.p_blocks = (int)(pt * p.p_splits);
    p.s_blocks = (int)(st * p.s_splits);
    const int many = 4, keys = MASS_WAVES * 16 * many;
    p.key_tiles = lh * (ceil_div(d.len_prefill, keys) + (p.stream ? 0 : c.n_streams * ceil_div(c.cap, keys))) < 512 ? 2 : many;
    // Few blocks with many vectors of 64 features are bound by the vectors' turns: two waves share keys and take turns (one head, 256
    // vectors on 400 slots 16.8 -> 15.2 us, 400 vectors 21.1 -> 17.1; 128 vectors 15.1 and 15.1, 64 vectors 11.6 and 12.2; of 128
    // features, whose keys are loaded twice for it, 256 vectors 20.2 and 21.0; four waves: 15.5 and 17.6 of the first two).
    p.share = p.key_tiles == 2 && c.head_dim == 64 && (d.len_prefill > 0 ? all : own) >= 256 ? 2 : 1;
    return p;
}
int listed_rows(const mlora_attention_mass &d, int n_rows) { return n_rows > 0 ? n_rows : d.rows_per_stream; }
size_t bytes_of(const mlora_attention_mass &d, int N)
{
    const Plan p = plan_of(d, N);
    const size_t vecs = (size_t)d.cache.n_streams * N * (d.n_q_heads / d.cache.n_kv_heads);
    return (size_t)d.cache.n_layers * d.cache.n_kv_heads * (p.p_splits + p.s_splits + 1) * vecs * sizeof(float2) + vecs * sizeof(int);
}

}  // namespace
}  // namespace mlora

using namespace mlora;

extern "C" {

size_t mlora_attention_mass_workspace_bytes(const mlora_attention_mass *d, int32_t n_rows)
{
    if (check(d) != MLORA_OK || n_rows < 0 || n_rows > d->rows_per_stream) return 0;
    return bytes_of(*d, listed_rows(*d, n_rows));
}

mlora_status mlora_attention_mass_add(const mlora_attention_mass *d, const void *q, const int32_t *rows, int32_t n_rows,
                                      void *workspace, size_t workspace_bytes, void *stream)
{
    const mlora_status st = check(d);
    if (st != MLORA_OK) return st;
    if (!q) return MLORA_EINVAL;
    if (reinterpret_cast<uintptr_t>(q) & 15u || reinterpret_cast<uintptr_t>(rows) & 3u) return MLORA_EALIGN;
    if (rows && (n_rows < 1 || n_rows > d->rows_per_stream)) return MLORA_ESHAPE;
    const int N = rows ? n_rows : d->rows_per_stream;
    if (!workspace || workspace_bytes < bytes_of(*d, N)) return MLORA_EWORKSPACE;
    if (reinterpret_cast<uintptr_t>(workspace) & 255u) return MLORA_EALIGN;
    const Plan p = plan_of(*d, N);
    const mlora_stream_cache &c = d->cache;
    MassArgs a;
    a.q = reinterpret_cast<const uint16_t *>(q);
    a.k = reinterpret_cast<const uint16_t *>(c.k);
    a.k_prefill = reinterpret_cast<const uint16_t *>(d->k_prefill);
    a.mass = c.mass;
    a.mass_prefill = d->mass_prefill;
    a.slot_pos = c.slot_pos;
    a.len = c.len;
    a.next_pos = c.next_pos;
    a.rows = rows;
    a.part = reinterpret_cast<float2 *>(workspace);
    a.L = c.n_layers;
    a.S = c.n_streams;
    a.H = c.n_kv_heads;
    a.G = d->n_q_heads / c.n_kv_heads;
    a.R = d->rows_per_stream;
    a.N = N;
    a.cap = c.cap;
    a.P = d->len_prefill;
    a.vecs = a.S * N * a.G;
    a.p_splits = p.p_splits;
    a.per_group = 1.f / (float)a.G;
    a.per_stream = 1.f / (float)a.N;
    a.s_splits = p.s_splits;
    a.p_per = p.p_per;
    a.s_per = p.s_per;
    a.p_blocks = p.p_blocks;
    a.s_blocks = p.s_blocks;
    a.scale2 = d->scale * 1.44269504088896340736f;
    a.decay = d->decay;
    a.rows_ml = a.part + (size_t)a.L * a.H * (p.p_splits + p.s_splits) * a.vecs;
    a.q_row = reinterpret_cast<int *>(a.rows_ml + (size_t)a.L * a.H * a.vecs);
    const int keys = p.wide ? WIDE_OWN : MASS_WAVES * 16 * p.key_tiles;
    a.p_tiles = (a.P + keys - 1) / keys;
    a.s_tiles = p.stream ? 0 : (a.cap + keys - 1) / keys;
    const long long lh = (long long)a.L * a.H, stats = lh * (a.p_blocks + (long long)a.S * a.s_blocks), add = lh * (a.p_tiles + (long long)a.S * a.s_tiles);
    if (stats > 0x7FFFFFFF || add > 0x7FFFFFFF) return MLORA_ESHAPE;
    hipStream_t s = (hipStream_t)stream;
    const dim3 block(64 * MASS_WAVES), stats_grid((unsigned)stats), add_grid((unsigned)add);
    const auto all = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        const auto stats = [&](auto prefill_tiles, auto stream_tiles) {
            mass_stats<D, decltype(prefill_tiles)::value, decltype(stream_tiles)::value><<<stats_grid, block, 0, s>>>(a);
        };
        constexpr std::integral_constant<int, 1> one{};
        constexpr std::integral_constant<int, 2> two{};
        constexpr std::integral_constant<int, 3> three{};
        constexpr std::integral_constant<int, 4> four{};
        const auto narrow_stats = [&] {
            const int per = std::max(p.p_per, p.s_per);
            const auto tiles = [&](auto q) { p.s_per == 1 ? stats(q, one) : stats(q, q); };
            per <= 1 ? tiles(one) : per == 2 ? tiles(two) : per == 3 ? tiles(three) : tiles(four);
        };
        const auto add_masses = [&](auto table) {
            constexpr bool TABLE = decltype(table)::value;
            if (p.key_tiles == 4) {
                mass_add<D, 4, TABLE, 1><<<add_grid, block, 0, s>>>(a);
            } else if (p.share == 1) {
                mass_add<D, 2, TABLE, 1><<<add_grid, block, 0, s>>>(a);
            } else if constexpr (D == 64) {
                mass_add<D, 2, TABLE, 2><<<add_grid, dim3(2 * 64 * MASS_WAVES), 0, s>>>(a);
            }
        };
        if (p.wide) {
            mass_stats_wide<D><<<stats_grid, block, 0, s>>>(a);
            mass_merge<<<dim3((unsigned)((lh * a.vecs + 31) / 32)), block, 0, s>>>(a);
            mass_add_wide<D><<<add_grid, block, 0, s>>>(a);
        } else if (p.stream) {
            if (a.P > 0 && !p.alone) narrow_stats();
            const auto stream_tiles = [&](auto vt, auto tk, auto waves) {
                constexpr int VT = decltype(vt)::value, TK = decltype(tk)::value, W = decltype(waves)::value;
                const dim3 grid((unsigned)(lh * a.S)), threads(64 * W);
                if (p.alone) mass_stream<D, VT, TK, W, true><<<grid, threads, 0, s>>>(a);
                else         mass_stream<D, VT, TK, W, false><<<grid, threads, 0, s>>>(a);
            };
            constexpr std::integral_constant<int, 8> eight{};
            constexpr std::integral_constant<int, 9> nine{};
            constexpr std::integral_constant<int, 16> sixteen{};
            if (p.stream_vecs == 1) {
                if (p.stream_waves == 16) p.stream == 4 ? stream_tiles(one, four, sixteen) : stream_tiles(one, nine, sixteen);
                else if (p.stream == 4)   stream_tiles(one, four, eight);
                else if (p.stream == 9)   stream_tiles(one, nine, eight);
                else                      stream_tiles(one, sixteen, eight);
            } else {
                if (p.stream_waves == 16) stream_tiles(two, four, sixteen);
                else if (p.stream == 4)   stream_tiles(two, four, eight);
                else                      stream_tiles(two, nine, eight);
            }
            if (a.P > 0 && !p.alone) {
                add_masses(std::true_type{});
            }
        } else {
            narrow_stats();
            add_masses(std::false_type{});
        }
    };
    if (c.head_dim == 64) all(std::integral_constant<int, 64>{});
    else                  all(std::integral_constant<int, 128>{});
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
