// Rotary position encodings: y_a = x_a cos - x_b sin, y_b = x_b cos + x_a sin for the pairs of a head, by the angle
// position * frequency.
//
// An angle is reduced in 64 bits: with t = position * (frequency in quarter turns), n = rint(t) and r = t - n from one fused
// multiply-add, sine and cosine of r quarter turns are short Taylor sums in 32 bits (|r| <= 1/2), and n mod 4 swaps and
// signs them.
//
// A call's bytes are read and written once.  A block makes the angles of its rows once, in LDS, for all heads of all tensors, and
// asks for its first 32 bytes per thread before it does.  The unit of work is two vectors of 16 bytes: V pairs in the half layout,
// 2 V features in the interleaved one and where features pass through.  Bound by memory: 4096 rows of 48 heads of 128 features,
// 100 MB read and written, 17 us from the memory-side cache and 23 from memory (4.4 TB/s); few rows by the launch.
#include <algorithm>
#include <cmath>

#include "common.hpp"

#include "../../include/mlora_rope.h"

namespace mlora {

namespace {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_BLOCK_ROWS = 8;       // most rows of a block

struct RopeRows {
    const int *base, *offset;
    const double *quarter_turns;
    int M, rows, half;                   // half: pairs of a head
};

__device__ __forceinline__ void rope_angle(const RopeRows &a, int m, int pair, float &c, float &s)
{
    const int stream = m / a.rows, row = m - stream * a.rows;
    const double pos = (a.base ? (double)a.base[stream] : 0.0) + (a.offset ? (double)a.offset[row] : (double)row);
    const double q = a.quarter_turns[pair], n = rint(pos * q), r = fma(pos, q, -n);
    const int quadrant = (int)(n - 4.0 * floor(n * 0.25));
    const float x = (float)(r * 1.57079632679489661923), z = x * x;
    const float sn = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
    const float cs = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    c = quadrant & 1 ? sn : cs;
    s = quadrant & 1 ? cs : sn;
    c = quadrant == 1 || quadrant == 2 ? -c : c;
    s = quadrant >= 2 ? -s : s;
}

__global__ __launch_bounds__(ROPE_THREADS) void rope_tables(const RopeRows a, float *cos_out, float *sin_out)
{
    const long long i = (long long)blockIdx.x * ROPE_THREADS + threadIdx.x;
    if (i >= (long long)a.M * a.half) return;
    const int m = (int)(i / a.half), pair = (int)(i - (long long)m * a.half);
    float c, s;
    rope_angle(a, m, pair, c, s);
    cos_out[i] = c;
    sin_out[i] = s;
}

struct RopeMove {
    const void *x;
    void *y;
    long long x_row, x_head, y_row, y_head;
    int begin;                           // first unit of a row
    int turning;                         // units of a head that turn pairs
    int units;                           // units of a head
    unsigned units_inv;                  // ceil(2^32 / units): i / units = umulhi(i, units_inv) while i * units < 2^32; units > 1
    int through;                         // first feature that passes through
};
struct RopeArgs {
    RopeRows at;
    RopeMove t[MLORA_ROPE_MAX_TENSORS];
    int n, row_units, block_rows, dim;
    float sign;
};

template <class T, int V>
struct alignas(16) RopeVec { T e[V]; };
// n of V elements, wherever they stand (a 16-byte access needs no more than its element's alignment)
typedef unsigned u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
template <class T, int V>
__device__ __forceinline__ RopeVec<T, V> rope_load(const T *p, int n)
{
    RopeVec<T, V> v;
    if (n >= V) v = __builtin_bit_cast(RopeVec<T, V>, *reinterpret_cast<const u32x4_at2 *>(p));
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) v.e[i] = i < n ? p[i] : T(0);
    }
    return v;
}
template <class T, int V>
__device__ __forceinline__ void rope_store(T *p, const RopeVec<T, V> &v, int n)
{
    if (n >= V) *reinterpret_cast<u32x4_at2 *>(p) = __builtin_bit_cast(u32x4_at2, v);
    else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < n) p[i] = v.e[i];
    }
}
__device__ __forceinline__ float rope_value(uint16_t b) { return bf16_bits_to_float(b); }
__device__ __forceinline__ float rope_value(float f) { return f; }
__device__ __forceinline__ void rope_put(uint16_t &to, float f) { to = __builtin_bit_cast(uint16_t, (__bf16)f); }
__device__ __forceinline__ void rope_put(float &to, float f) { to = f; }

template <class T, bool INTERLEAVED>
__global__ __launch_bounds__(ROPE_THREADS) void rope_apply(const RopeArgs a)
{
    constexpr int V = 16 / sizeof(T);
    extern __shared__ float table[];                     // [block_rows][2][half_pad]
    const int tid = threadIdx.x, row0 = (int)blockIdx.x * a.block_rows, rows = min(a.block_rows, a.at.M - row0);
    const int step = (int)gridDim.y * ROPE_THREADS;
    const int half = a.at.half, half_pad = (half + V - 1) / V * V, total = rows * a.row_units;

    struct Unit {
        const T *x0;
        T *y0;
        int apart;                                       // from the first vector to the second
        int n0, n1;                                      // elements of each
        int at;                                          // of its first pair in the table, or -1: passes through
    };
    auto unit_of = [&](int i) {
        int r = 0;
        while (i >= a.row_units) i -= a.row_units, ++r;
        int k = 0;
        while (k + 1 < a.n && i >= a.t[k + 1].begin) ++k;
        const RopeMove &t = a.t[k];
        const int j = i - t.begin, head = t.units > 1 ? (int)__umulhi((unsigned)j, t.units_inv) : j, u = j - head * t.units;
        Unit w;
        int first, left;
        if (u < t.turning) {
            w.at = r * 2 * half_pad + u * V;
            if (INTERLEAVED) { first = u * 2 * V; left = 2 * half - first; w.apart = V; }
            else             { first = u * V; left = 0; w.apart = half; w.n0 = w.n1 = min(V, half - first); }
        } else {
            w.at = -1;
            first = t.through + (u - t.turning) * 2 * V;
            left = a.dim - first;
            w.apart = V;
        }
        if (INTERLEAVED || w.at < 0) w.n0 = min(V, left), w.n1 = min(V, left - w.n0);
        const long long m = row0 + r;
        w.x0 = reinterpret_cast<const T *>(t.x) + m * t.x_row + head * t.x_head + first;
        w.y0 = reinterpret_cast<T *>(t.y) + m * t.y_row + head * t.y_head + first;
        return w;
    };
    int i = (int)blockIdx.y * ROPE_THREADS + tid;
    Unit w{};
    RopeVec<T, V> p, q;
    if (i < total) {
        w = unit_of(i);
        p = rope_load<T, V>(w.x0, w.n0);
        q = rope_load<T, V>(w.x0 + w.apart, w.n1);
    }
    for (int k = tid; k < rows * half; k += ROPE_THREADS) {
        const int r = k / half, pair = k - r * half;
        float c, s;
        rope_angle(a.at, row0 + r, pair, c, s);
        table[r * 2 * half_pad + pair] = c;
        table[r * 2 * half_pad + half_pad + pair] = s * a.sign;
    }
    __syncthreads();
    while (i < total) {
        const Unit now = w;
        RopeVec<T, V> x0 = p, x1 = q;
        i += step;
        if (i < total) {
            w = unit_of(i);
            p = rope_load<T, V>(w.x0, w.n0);
            q = rope_load<T, V>(w.x0 + w.apart, w.n1);
        }
        if (now.at >= 0) {
            float c[V], s[V];
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                *reinterpret_cast<f32x4 *>(c + e) = *reinterpret_cast<const f32x4 *>(table + now.at + e);
                *reinterpret_cast<f32x4 *>(s + e) = *reinterpret_cast<const f32x4 *>(table + now.at + half_pad + e);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                T &first = INTERLEAVED ? (2 * e < V ? x0.e[(2 * e) % V] : x1.e[(2 * e) % V]) : x0.e[e];
                T &second = INTERLEAVED ? (2 * e < V ? x0.e[(2 * e + 1) % V] : x1.e[(2 * e + 1) % V]) : x1.e[e];
                const float u = rope_value(first), v = rope_value(second);
                rope_put(first, fmaf(u, c[e], -v * s[e]));
                rope_put(second, fmaf(v, c[e], u * s[e]));
            }
        }
        rope_store<T, V>(now.y0, x0, now.n0);
        rope_store<T, V>(now.y0 + now.apart, x1, now.n1);
    }
}

bool turns_finite(double v) { return std::isfinite(v); }

mlora_status check(const mlora_rope *r)
{
    if (!r) return MLORA_EINVAL;
    if (r->layout != MLORA_ROPE_HALF && r->layout != MLORA_ROPE_INTERLEAVED) return MLORA_EINVAL;
    if (r->scaling < MLORA_ROPE_PLAIN || r->scaling > MLORA_ROPE_TURNS) return MLORA_EINVAL;
    if (r->head_dim < 2 || r->head_dim > MLORA_ROPE_MAX_DIM || r->rot < 2 || r->rot > r->head_dim || r->rot % 2 != 0) return MLORA_ESHAPE;
    if (r->scaling == MLORA_ROPE_BASE && r->rot < 4) return MLORA_ESHAPE;
    if (!(r->theta > 0) || !turns_finite(r->theta)) return MLORA_EINVAL;
    if (r->scaling != MLORA_ROPE_PLAIN && (!(r->factor > 0) || !turns_finite(r->factor))) return MLORA_EINVAL;
    if (r->scaling == MLORA_ROPE_TURNS && (!(r->low < r->high) || !turns_finite(r->low) || !turns_finite(r->high)
                                          || !(r->context > 0) || !turns_finite(r->context))) return MLORA_EINVAL;
    return MLORA_OK;
}

mlora_status check(const mlora_rope *r, const mlora_rope_rows *rows)
{
    const mlora_status st = check(r);
    if (st != MLORA_OK) return st;
    if (!rows || !rows->quarter_turns) return MLORA_EINVAL;
    if (rows->M < 0 || rows->M > MLORA_ROPE_MAX_ROWS || rows->rows_per_stream <= 0 || rows->M % rows->rows_per_stream != 0) return MLORA_ESHAPE;
    if ((reinterpret_cast<uintptr_t>(rows->base) | reinterpret_cast<uintptr_t>(rows->offset)) & 3u) return MLORA_EALIGN;
    if (reinterpret_cast<uintptr_t>(rows->quarter_turns) & 7u) return MLORA_EALIGN;
    return MLORA_OK;
}

RopeRows rows_of(const mlora_rope *r, const mlora_rope_rows *rows)
{
    return RopeRows{rows->base, rows->offset, rows->quarter_turns, rows->M, rows->rows_per_stream, r->rot / 2};
}

}  // namespace
}  // namespace mlora

using namespace mlora;

extern "C" {

mlora_status mlora_rope_frequencies(const mlora_rope *r, double *quarter_turns)
{
    const mlora_status st = check(r);
    if (st != MLORA_OK) return st;
    if (!quarter_turns) return MLORA_EINVAL;
    const double pi = 3.14159265358979323846;
    const double base = r->scaling == MLORA_ROPE_BASE ? r->theta * std::pow(r->factor, r->rot / (r->rot - 2.0)) : r->theta;
    for (int i = 0; i < r->rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / r->rot);
        if (r->scaling == MLORA_ROPE_LINEAR) f /= r->factor;
        if (r->scaling == MLORA_ROPE_TURNS) {
            const double u = std::min(1.0, std::max(0.0, (r->context * f / (2 * pi) - r->low) / (r->high - r->low)));
            f = (1 - u) * f / r->factor + u * f;
        }
        quarter_turns[i] = f * (2 / pi);
    }
    return MLORA_OK;
}

mlora_status mlora_rope_tables(const mlora_rope *r, const mlora_rope_rows *rows, float *cos_out, float *sin_out, void *stream)
{
    const mlora_status st = check(r, rows);
    if (st != MLORA_OK) return st;
    if (rows->M > 0 && (!cos_out || !sin_out)) return MLORA_EINVAL;
    if ((reinterpret_cast<uintptr_t>(cos_out) | reinterpret_cast<uintptr_t>(sin_out)) & 3u) return MLORA_EALIGN;
    if (rows->M == 0) return MLORA_OK;
    const RopeRows a = rows_of(r, rows);
    const long long n = (long long)a.M * a.half;
    rope_tables<<<dim3((unsigned)((n + ROPE_THREADS - 1) / ROPE_THREADS)), dim3(ROPE_THREADS), 0, (hipStream_t)stream>>>(a, cos_out, sin_out);
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

mlora_status mlora_rope_apply(const mlora_rope *r, const mlora_rope_rows *rows, const mlora_rope_tensor *tensors, int32_t n_tensors,
                              int32_t dtype, int32_t inverse, void *stream)
{
    const mlora_status st = check(r, rows);
    if (st != MLORA_OK) return st;
    if (!tensors || n_tensors < 1 || n_tensors > MLORA_ROPE_MAX_TENSORS) return MLORA_EINVAL;
    if (dtype != MLORA_Y_BF16 && dtype != MLORA_Y_FP32) return MLORA_EINVAL;
    if (inverse != 0 && inverse != 1) return MLORA_EINVAL;
    const int size = dtype == MLORA_Y_BF16 ? 2 : 4, V = 16 / size, dim = r->head_dim, half = r->rot / 2;
    RopeArgs a;
    a.at = rows_of(r, rows);
    a.n = n_tensors;
    a.dim = dim;
    a.sign = inverse ? -1.f : 1.f;
    int units = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const mlora_rope_tensor &t = tensors[i];
        if (rows->M > 0 && (!t.x || !t.y)) return MLORA_EINVAL;
        if (t.heads < 1 || t.heads > 4096) return MLORA_ESHAPE;
        if (t.x_row < 0 || t.x_head < 0 || t.y_row < 0 || t.y_head < 0) return MLORA_ESHAPE;
        if ((reinterpret_cast<uintptr_t>(t.x) | reinterpret_cast<uintptr_t>(t.y)) & (unsigned)(size - 1)) return MLORA_EALIGN;
        if (rows->M > 0 && t.x == t.y && (t.x_row != t.y_row || t.x_head != t.y_head)) return MLORA_EINVAL;
        if ((rows->M > 1 && t.y_row < dim) || (rows->M > 0 && t.heads > 1 && t.y_head < dim)) return MLORA_EINVAL;
        RopeMove &m = a.t[i];
        m.x = t.x;
        m.y = t.y;
        m.x_row = t.x_row, m.x_head = t.x_head, m.y_row = t.y_row, m.y_head = t.y_head;
        m.begin = units;
        m.turning = t.rotate ? (half + V - 1) / V : 0;
        m.through = t.rotate ? r->rot : 0;
        m.units = m.turning + (dim - m.through + 2 * V - 1) / (2 * V);
        m.units_inv = m.units > 1 ? (unsigned)((0x100000000ull + m.units - 1) / m.units) : 0;
        units += m.units * t.heads;
    }
    if (rows->M == 0) return MLORA_OK;
    a.row_units = units;
    // Few rows: a row per block, or several blocks where they leave room (240 rows of 40 heads in fp32 6.2 -> 5.0 us); from two
    // blocks per compute unit on rows share a block, up to four units per thread (4096 rows of 48 heads: two 18.6 us, four 16.8,
    // eight 21.9; loads past the caches save a tenth where the inputs are not in them and cost a quarter where they are).
    a.block_rows = std::max(1, std::min(std::min(ROPE_BLOCK_ROWS, a.at.M / 512), 4 * ROPE_THREADS / units));
    const size_t lds = (size_t)a.block_rows * 2 * ((half + V - 1) / V * V) * sizeof(float);
    const int blocks = (a.at.M + a.block_rows - 1) / a.block_rows;
    const int parts = std::max(1, std::min((units * a.block_rows + ROPE_THREADS - 1) / ROPE_THREADS, 1024 / blocks));
    const dim3 grid((unsigned)blocks, (unsigned)parts), block(ROPE_THREADS);
    hipStream_t s = (hipStream_t)stream;
    const bool inter = r->layout == MLORA_ROPE_INTERLEAVED;
    if (dtype == MLORA_Y_BF16) {
        if (inter) rope_apply<uint16_t, true><<<grid, block, lds, s>>>(a);
        else       rope_apply<uint16_t, false><<<grid, block, lds, s>>>(a);
    } else {
        if (inter) rope_apply<float, true><<<grid, block, lds, s>>>(a);
        else       rope_apply<float, false><<<grid, block, lds, s>>>(a);
    }
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
