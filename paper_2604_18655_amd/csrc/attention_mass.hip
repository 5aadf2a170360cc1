// Attention weights of the newest rows, added to what every slot of the cache has received so far:
//
//     mass[t] = decay * mass[t] + sum over rows and query heads of exp(s[row][t] - max) / sum,   s = scale q . k
//
// A weight needs its row's maximum and sum over all keys first, so there are two launches: mass_stats leaves the maximum and
// sum of every query vector over each block's share of the keys, mass_add makes the scores again, key by key.  (Kept
// in between, the scores of a prompt's chunk would be gigabytes.)
//
// Scores are products on the matrix units (16x16x32 bf16, fp32 accumulation).  A wave keeps one side in registers and its lanes
// own it (a lane's columns: its query vectors in mass_stats, its keys in mass_add), and the other side passes by, so that
// running maxima, sums and masses are a lane's own, without a trip through other lanes until the end.
//
// Query vectors are counted (stream, listed row, query head of the group): v = (s * N + j) * G + g.
#include <algorithm>

#include "common.hpp"

#include "../../include/mlora_stream_cache.h"

namespace mlora {

namespace {

constexpr int MASS_WAVES = 4;
constexpr int KC = 32;                   // keys of a chunk in mass_stats
constexpr int KT = 2;                    // key tiles (of 16) of a wave in mass_add
constexpr int ADD_KEYS = MASS_WAVES * KT * 16;
constexpr int BATCH = 512;               // query vectors whose maxima mass_add holds at a time
constexpr float NEG_BIG = -1.0e30f;      // "no key seen yet"
constexpr float UNSEEN = -3.0e38f;       // score of a key that is not visible: exp2(UNSEEN - NEG_BIG) is 0

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct MassArgs {
    const uint16_t *q, *k, *k_prefill;
    float *mass, *mass_prefill;
    const int *slot_pos, *len, *next_pos, *rows;
    float2 *part;                        // [L * H][p_splits + s_splits][vecs]: maximum (of scores in units of log 2) and sum
    int L, S, H, G, R, N, cap, P;        // N: listed rows of a stream
    int vecs;                            // S * N * G
    int p_splits, s_splits;              // blocks that share the keys of a query tile: prefill, stream segment
    int p_blocks, s_blocks;              // blocks of a layer and head: prefill; one stream
    float scale2, decay;                 // scale2 = scale * log2(e)
};

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

// One block: QT tiles of 16 query vectors (of one stream, or of all streams on the prefill segment) against a share of the keys.
template <int D, int QT>
__global__ __launch_bounds__(64 * MASS_WAVES) void mass_stats(const MassArgs a)
{
    constexpr int DK = D / 32;
    __shared__ float2 ml[MASS_WAVES][QT * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l16 = lane & 15, lq = lane >> 4;
    const int per_head = a.p_blocks + a.S * a.s_blocks, lh = (int)blockIdx.x / per_head, l = lh / a.H, h = lh - l * a.H;
    int b = (int)blockIdx.x - lh * per_head;
    const bool prefill = b < a.p_blocks;
    int s = 0;
    if (!prefill) {
        b -= a.p_blocks;
        s = b / a.s_blocks;
        b -= s * a.s_blocks;
    }
    const int splits = prefill ? a.p_splits : a.s_splits, tile = b / splits, z = b - tile * splits;
    const int v0 = tile * QT * 16, n = prefill ? 0 : listed(a, s);
    const int mine = prefill ? a.vecs : n * a.G;                     // query vectors of this segment
    const int keys = prefill ? a.P : max(0, min(a.len[s], a.cap));
    if (v0 >= mine) return;
    const int newest = prefill ? 0 : a.next_pos[s] - n;              // position of the first listed row
    const size_t seg = prefill ? (size_t)lh * a.P : (((size_t)l * a.S + s) * a.H + h) * a.cap;
    const uint16_t *const kb = (prefill ? a.k_prefill : a.k) + seg * D;
    const int *const pb = a.slot_pos + seg;

    // this lane's query vectors (B operands: lane (l16, lq) holds features 8 * lq .. of vector l16 of a tile)
    uint4 qf[QT][DK];
    float m[QT], sum[QT];
    int pos[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int v = min(v0 + 16 * t + l16, mine - 1), j = v / a.G, g = v - j * a.G;
        int st = s, row = j;
        if (prefill) st = j / a.N, row = j - st * a.N;
        if (prefill && !counts(a, st, row)) row = -1;
        const uint16_t *const qp = a.q + (row < 0 ? 0 : q_at(a, l, h, st, row, g, D)) + 8 * lq;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) qf[t][kk] = *reinterpret_cast<const uint4 *>(qp + 32 * kk);
        pos[t] = newest + j;
        m[t] = NEG_BIG;
        sum[t] = 0.f;
    }
    const int chunks = (keys + KC - 1) / KC;
    for (int c = z * MASS_WAVES + wave; c < chunks; c += splits * MASS_WAVES) {
        const int k0 = c * KC, nk = min(KC, keys - k0);
        // keys as A operands (past the end: the last key)
        uint4 kf[KC / 16][DK];
#pragma unroll
        for (int j = 0; j < KC / 16; ++j) {
            const uint16_t *const kp = kb + (size_t)(k0 + min(16 * j + l16, nk - 1)) * D + 8 * lq;
#pragma unroll
            for (int kk = 0; kk < DK; ++kk) kf[j][kk] = *reinterpret_cast<const uint4 *>(kp + 32 * kk);
        }
        const int at = prefill ? 0 : pb[k0 + min(lane & 31, nk - 1)];
        const bool masked = nk < KC || (!prefill && __any(at > newest));
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            f32x4 sc[KC / 16];
#pragma unroll
            for (int j = 0; j < KC / 16; ++j) {
                sc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < DK; ++kk) sc[j] = mfma16(kf[j][kk], qf[t][kk], sc[j]);
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[j][e] *= a.scale2;
            }
            if (masked) {
#pragma unroll
                for (int j = 0; j < KC / 16; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = 16 * j + 4 * lq + e;
                        const int key_pos = __shfl(at, key);         // (all lanes: before any condition)
                        sc[j][e] = key < nk && (prefill || key_pos <= pos[t]) ? sc[j][e] : UNSEEN;
                    }
            }
            float top = m[t];
#pragma unroll
            for (int j = 0; j < KC / 16; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) top = fmaxf(top, sc[j][e]);
            float add = 0.f;
#pragma unroll
            for (int j = 0; j < KC / 16; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) add += __builtin_amdgcn_exp2f(sc[j][e] - top);
            sum[t] = sum[t] * __builtin_amdgcn_exp2f(m[t] - top) + add;
            m[t] = top;
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
    if (threadIdx.x < QT * 16 && v < mine) {
        float top = NEG_BIG, all = 0.f;
#pragma unroll
        for (int w = 0; w < MASS_WAVES; ++w) top = fmaxf(top, ml[w][threadIdx.x].x);
#pragma unroll
        for (int w = 0; w < MASS_WAVES; ++w) all += ml[w][threadIdx.x].y * __builtin_amdgcn_exp2f(ml[w][threadIdx.x].x - top);
        const int row = (prefill ? 0 : a.p_splits) + z;
        a.part[((size_t)lh * (a.p_splits + a.s_splits) + row) * a.vecs + (prefill ? v : s * a.N * a.G + v)] = make_float2(top, all);
    }
}

// One block: 128 keys of a segment against all query vectors that may see them.
template <int D>
__global__ __launch_bounds__(64 * MASS_WAVES) void mass_add(const MassArgs a)
{
    constexpr int DK = D / 32;
    __shared__ __align__(16) float top_of[BATCH], inv_of[BATCH];
    __shared__ int pos_of[BATCH];
    __shared__ const uint16_t *q_of[BATCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, lq = lane >> 4;
    const int p_blocks = (a.P + ADD_KEYS - 1) / ADD_KEYS, s_blocks = (a.cap + ADD_KEYS - 1) / ADD_KEYS;
    const int per_head = p_blocks + a.S * s_blocks, lh = (int)blockIdx.x / per_head, l = lh / a.H, h = lh - l * a.H;
    int b = (int)blockIdx.x - lh * per_head;
    const bool prefill = b < p_blocks;
    int s = 0;
    if (!prefill) {
        b -= p_blocks;
        s = b / s_blocks;
        b -= s * s_blocks;
    }
    const int keys = prefill ? a.P : max(0, min(a.len[s], a.cap));
    if (b * ADD_KEYS >= keys) return;
    const int n = prefill ? 0 : listed(a, s), newest = prefill ? 0 : a.next_pos[s] - n;
    const int mine = prefill ? a.vecs : n * a.G;
    const size_t seg = prefill ? (size_t)lh * a.P : (((size_t)l * a.S + s) * a.H + h) * a.cap;
    const int k0 = b * ADD_KEYS + wave * KT * 16;

    // this lane's keys (B operands)
    uint4 kf[KT][DK];
    int at[KT];
    float acc[KT];
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        const int key = min(k0 + 16 * t + l16, keys - 1);
        const uint16_t *const kp = (prefill ? a.k_prefill : a.k) + (seg + key) * D + 8 * lq;
#pragma unroll
        for (int kk = 0; kk < DK; ++kk) kf[t][kk] = *reinterpret_cast<const uint4 *>(kp + 32 * kk);
        at[t] = prefill ? 0 : a.slot_pos[seg + key];
        acc[t] = 0.f;
    }
    bool masked = false;
#pragma unroll
    for (int t = 0; t < KT; ++t) masked |= !prefill && at[t] > newest;
    masked = __any(masked);

    for (int base = 0; base < mine; base += BATCH) {
        const int here = min(BATCH, mine - base), pad = (here + 15) / 16 * 16;
        __syncthreads();
        for (int i = tid; i < pad; i += 64 * MASS_WAVES) {
            const int v = min(base + i, mine - 1), j = v / a.G, g = v - j * a.G;
            int st = s, row = j;
            if (prefill) st = j / a.N, row = j - st * a.N;
            const bool ok = base + i < mine && (!prefill || counts(a, st, row));
            float top = NEG_BIG, all = 0.f;
            const int splits = a.p_splits + a.s_splits;
            const float2 *const part = a.part + (size_t)lh * splits * a.vecs + ((size_t)st * a.N + row) * a.G + g;
            if (ok) {
                for (int z = 0; z < splits; ++z) {
                    const float2 x = part[(size_t)z * a.vecs];
                    const float t2 = fmaxf(top, x.x);
                    all = all * __builtin_amdgcn_exp2f(top - t2) + x.y * __builtin_amdgcn_exp2f(x.x - t2);
                    top = t2;
                }
            }
            top_of[i] = top;
            inv_of[i] = all > 0.f ? 1.f / all : all;                 // (a row that sees nothing adds nothing; NaN stays)
            pos_of[i] = newest + j;
            q_of[i] = a.q + (ok ? q_at(a, l, h, st, row, g, D) : 0);
        }
        __syncthreads();
        for (int t0 = 0; t0 < pad; t0 += 16) {
            // query vectors as A operands: element e of a score belongs to vector 4 * lq + e
            uint4 qf[DK];
            const uint16_t *const qp = q_of[t0 + l16] + 8 * lq;
#pragma unroll
            for (int kk = 0; kk < DK; ++kk) qf[kk] = *reinterpret_cast<const uint4 *>(qp + 32 * kk);
            const f32x4 top = *reinterpret_cast<const f32x4 *>(top_of + t0 + 4 * lq), inv = *reinterpret_cast<const f32x4 *>(inv_of + t0 + 4 * lq);
#pragma unroll
            for (int t = 0; t < KT; ++t) {
                f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < DK; ++kk) sc = mfma16(qf[kk], kf[t][kk], sc);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float w = __builtin_amdgcn_exp2f(sc[e] * a.scale2 - top[e]) * inv[e];
                    if (masked) w = at[t] <= pos_of[t0 + 4 * lq + e] ? w : 0.f;
                    acc[t] += inv[e] != 0.f ? w : 0.f;
                }
            }
        }
    }
#pragma unroll
    for (int t = 0; t < KT; ++t) {
        const float add = over_quarters(acc[t], [](float x, float y) { return x + y; });
        const int key = k0 + 16 * t + l16;
        float *const to = (prefill ? a.mass_prefill : a.mass) + seg + key;
        if (lq == 0 && key < keys) *to = a.decay * *to + add;
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

// How a call is cut: blocks that share a query tile's keys, until the launch has about four blocks per compute unit or a block
// has fewer than two chunks per wave left.
struct Plan {
    int tiles;                           // query tiles of a block
    int p_splits, s_splits, p_blocks, s_blocks;
};
Plan plan_of(const mlora_attention_mass &d, int N)
{
    const mlora_stream_cache &c = d.cache;
    const int G = d.n_q_heads / c.n_kv_heads;
    const long long lh = (long long)c.n_layers * c.n_kv_heads, own = (long long)N * G, all = own * c.n_streams;
    Plan p;
    p.tiles = own > 16 ? 4 : 1;
    const auto tiles_of = [&](long long vecs) { return (vecs + 16 * p.tiles - 1) / (16 * p.tiles); };
    const long long pt = d.len_prefill > 0 ? tiles_of(all) : 0, st = tiles_of(own);
    const long long blocks = lh * (pt + c.n_streams * st), want = std::max(1ll, (1024 + blocks - 1) / blocks);
    const auto splits_of = [&](int keys) {
        const long long chunks = (keys + KC - 1) / KC;
        return (int)std::max(1ll, std::min({want, (chunks + 2 * MASS_WAVES - 1) / (2 * MASS_WAVES), 32ll}));
    };
    p.p_splits = d.len_prefill > 0 ? splits_of(d.len_prefill) : 0;
    p.s_splits = splits_of(c.cap);
    p.p_blocks = (int)(pt * p.p_splits);
    p.s_blocks = (int)(st * p.s_splits);
    return p;
}
int listed_rows(const mlora_attention_mass &d, int n_rows) { return n_rows > 0 ? n_rows : d.rows_per_stream; }
size_t bytes_of(const mlora_attention_mass &d, int N)
{
    const Plan p = plan_of(d, N);
    const size_t vecs = (size_t)d.cache.n_streams * N * (d.n_q_heads / d.cache.n_kv_heads);
    return (size_t)d.cache.n_layers * d.cache.n_kv_heads * (p.p_splits + p.s_splits) * vecs * sizeof(float2);
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
    a.s_splits = p.s_splits;
    a.p_blocks = p.p_blocks;
    a.s_blocks = p.s_blocks;
    a.scale2 = d->scale * 1.44269504088896340736f;
    a.decay = d->decay;
    const long long lh = (long long)a.L * a.H, stats = lh * (a.p_blocks + (long long)a.S * a.s_blocks);
    const long long add = lh * ((a.P + ADD_KEYS - 1) / ADD_KEYS + (long long)a.S * ((a.cap + ADD_KEYS - 1) / ADD_KEYS));
    if (stats > 0x7FFFFFFF || add > 0x7FFFFFFF) return MLORA_ESHAPE;
    hipStream_t s = (hipStream_t)stream;
    const dim3 block(64 * MASS_WAVES);
    if (c.head_dim == 64) {
        if (p.tiles == 1) mass_stats<64, 1><<<dim3((unsigned)stats), block, 0, s>>>(a);
        else              mass_stats<64, 4><<<dim3((unsigned)stats), block, 0, s>>>(a);
        mass_add<64><<<dim3((unsigned)add), block, 0, s>>>(a);
    } else {
        if (p.tiles == 1) mass_stats<128, 1><<<dim3((unsigned)stats), block, 0, s>>>(a);
        else              mass_stats<128, 4><<<dim3((unsigned)stats), block, 0, s>>>(a);
        mass_add<128><<<dim3((unsigned)add), block, 0, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
