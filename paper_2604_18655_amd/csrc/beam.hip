// One step of beam search on the logits (see include/mlora_beam.h).
//
// A candidate's rank inside its beam is its logit's, so the W best of a group lie in the W chunks of 64 tokens whose best candidates are the
// best W (an order without equals: ranked score, beam, logit, token).  beam_stats goes over the logits once and leaves the largest logit
// of every chunk, and of every slice of 64 chunks the maximum and the sum of exponentials.  beam_pick, a block per group, makes
// the beams' log-sums, finds the W chunks among all, and looks at the 64 logits of each once more.
#include <type_traits>

#include "common.hpp"

#include "../../include/mlora_beam.h"

namespace mlora {

namespace {

constexpr int CHUNK = 64, SLICE = 64 * CHUNK;            // tokens
constexpr int PICK = 1024;                               // threads of beam_pick
constexpr int W_MAX = MLORA_BEAM_MAX_BEAMS;
constexpr int LIST = W_MAX * CHUNK;                      // candidates that are ranked at once
constexpr float NONE = -__builtin_inff();

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));     // logits are aligned as one element

struct BeamArgs {
    const void *logits;
    const float *score;
    const int *length, *finished;
    int *source, *token;
    float *score_out;
    int *length_out, *finished_out;
    float *chunk_top;                                    // [rows][chunks]
    float *slice_top;                                    // [rows][slices]
    double *slice_sum;                                   // [rows][slices], of exp(logit - slice_top)
    int W, V, chunks, slices, eos, pad;
    float power;
};

template <bool FP32>
__device__ __forceinline__ float logit_at(const void *row, int v)
{
    if constexpr (FP32) return reinterpret_cast<const float *>(row)[v];
    else                return bf16_bits_to_float(reinterpret_cast<const uint16_t *>(row)[v]);
}

template <int CTRL>
__device__ __forceinline__ float max_with(float x)
{
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true)));
}

// A wave per slice and row: 16 bytes per lane and load, side by side, so that a chunk is 8 (bf16) or 16 (fp32) neighbouring lanes.
template <bool FP32>
__global__ __launch_bounds__(256) void beam_stats(const BeamArgs a)
{
    constexpr int E = FP32 ? 4 : 8, LOADS = SLICE / (64 * E);
    const int lane = threadIdx.x & 63, slice = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), row = blockIdx.y;
    if (slice >= a.slices || a.finished[row] != 0) return;
    const char *const z = reinterpret_cast<const char *>(a.logits) + (size_t)row * a.V * (FP32 ? 4 : 2);
    const int first = slice * SLICE;
    float x[LOADS][E];
    u32x4 raw[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int v = first + (i * 64 + lane) * E;
        if (v + E <= a.V) raw[i] = *reinterpret_cast<const u32x4_any *>(z + (size_t)v * (FP32 ? 4 : 2));
    }
    float top = NONE;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int v = first + (i * 64 + lane) * E;
        float most = NONE;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (v + E <= a.V) x[i][e] = FP32 ? __uint_as_float(raw[i][e % 4]) : bf16_bits_to_float(e & 1 ? raw[i][e / 2] >> 16 : raw[i][e / 2] & 0xFFFFu);
            else              x[i][e] = v + e < a.V ? logit_at<FP32>(z, v + e) : NONE;
            most = fmaxf(most, x[i][e]);
        }
        most = max_with<0xB1>(most);                     // neighbours, pairs, halves of 8, of 16
        most = max_with<0x4E>(most);
        most = max_with<0x141>(most);
        if constexpr (FP32) most = max_with<0x140>(most);
        if (lane % (CHUNK / E) == 0 && v < a.V) a.chunk_top[(size_t)row * a.chunks + v / CHUNK] = most;
        top = fmaxf(top, most);
    }
#pragma unroll
    for (int d = 8; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float from = top == NONE ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) sum += __builtin_amdgcn_exp2f((x[i][e] - from) * 1.44269504088896340736f);
    double all = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
    if (lane == 0) {
        a.slice_top[(size_t)row * a.slices + slice] = top;
        a.slice_sum[(size_t)row * a.slices + slice] = all;
    }
}

struct Beam {
    double score, lse, len;                              // len: what the score of its candidates is divided by
    int finished, live, tokens;                          // tokens: of its candidates
};
// What beam b makes of a logit; -infinity: no candidate
__device__ __forceinline__ double ranked(const Beam &b, float z)
{
    if (!b.live || !(z > NONE)) return (double)NONE;
    return (b.finished ? b.score : b.score + ((double)z - b.lse)) / b.len;
}
struct Candidate {
    double rank;
    float z;
    int beam, at;                                        // chunk, or token
};
__device__ __forceinline__ bool before(const Candidate &x, const Candidate &y)
{
    if (x.rank != y.rank) return x.rank > y.rank;
    if (x.beam != y.beam) return x.beam < y.beam;
    if (x.z != y.z) return x.z > y.z;
    return x.at < y.at;
}
// numbers, -infinity among them, as integers that order like them
__device__ __forceinline__ int in_order(float f)
{
    const int b = __float_as_int(f + 0.f);
    return b < 0 ? b ^ 0x7FFFFFFF : b;
}

template <bool FP32>
__global__ __launch_bounds__(PICK) void beam_pick(const BeamArgs a)
{
    __shared__ Beam beams[W_MAX];
    __shared__ Candidate list[LIST];
    __shared__ Candidate best[W_MAX];
    __shared__ int found, at_least;
    __shared__ Candidate wave_best[PICK / 64], winners[W_MAX];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, W = a.W, row0 = (int)blockIdx.x * W;
    for (int b = wave; b < W; b += PICK / 64) {
        const int row = row0 + b, done = a.finished[row];
        const float *const tops = a.slice_top + (size_t)row * a.slices;
        const double *const sums = a.slice_sum + (size_t)row * a.slices;
        float top = NONE;
        if (!done)
            for (int i = lane; i < a.slices; i += 64) top = fmaxf(top, tops[i]);
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        double sum = 0.;
        if (!done)
            for (int i = lane; i < a.slices; i += 64) sum += sums[i] * exp((double)tops[i] - (double)(top == NONE ? 0.f : top));
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        if (lane == 0) {
            const float score = a.score[row];
            const double lse = (double)top + log(sum);
            const int tokens = a.length[row] + (done ? 0 : 1);
            beams[b] = Beam{score, lse, pow(fmax(1., (double)tokens), (double)a.power), done, isfinite(score) && (done || isfinite(lse)), tokens};
        }
    }
    if (tid == 0) found = 0, at_least = in_order(NONE);
    __syncthreads();

    // The W best chunks.  Of each wave's 64 lanes, the W-th best best chunk: that many chunks are at least as good, so nothing below the largest
    // such bound of all waves counts.
    const int n = W * a.chunks;
    const auto chunk_at = [&](int i) {
        const int b = i / a.chunks, c = i - b * a.chunks;
        Candidate x{(double)NONE, NONE, b, c};
        if (beams[b].finished) x.z = c == 0 ? 0.f : NONE;
        else                   x.z = a.chunk_top[(size_t)(row0 + b) * a.chunks + c];
        x.rank = ranked(beams[b], x.z);
        return x;
    };
    float mine = NONE;
    for (int i = tid; i < n; i += PICK) mine = fmaxf(mine, (float)chunk_at(i).rank);
    {
        const int key = in_order(mine);
        int bound = in_order(NONE);
        unsigned lo = 0;                                 // the largest key that W lanes reach, bit by bit from above
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            const unsigned t = lo | 1u << bit;
            if (__popcll(__ballot(((unsigned)key ^ 0x80000000u) >= t)) >= W) lo = t;
        }
        bound = max(bound, (int)(lo ^ 0x80000000u));
        if (lane == 0) atomicMax(&at_least, bound);
    }
    __syncthreads();
    const int bound = at_least;
    for (int i = tid; i < n; i += PICK) {
        const Candidate x = chunk_at(i);
        if (x.rank > (double)NONE && in_order((float)x.rank) >= bound) {
            const int at = atomicAdd(&found, 1);
            if (at < LIST) list[at] = x;
        }
    }
    __syncthreads();
    int chunks = min(found, W);
    if (found <= LIST) {
        const int m = found;
        for (int i = tid; i < m; i += PICK) {
            int number = 0;
            for (int j = 0; j < m; ++j) number += before(list[j], list[i]);
            if (number < W) best[number] = list[i];
        }
        __syncthreads();
    } else {
        // (more equals than the list holds: one after the other)
        Candidate last{__builtin_inf(), 0.f, -1, -1};
        for (int k = 0; k < chunks; ++k) {
            Candidate top{(double)NONE, NONE, W, 0};
            for (int i = tid; i < n; i += PICK) {
                const Candidate x = chunk_at(i);
                if (x.rank > (double)NONE && before(last, x) && before(x, top)) top = x;
            }
#pragma unroll 1
            for (int d = 1; d < 64; d *= 2) {
                const Candidate x{__shfl_xor(top.rank, d), __shfl_xor(top.z, d), __shfl_xor(top.beam, d), __shfl_xor(top.at, d)};
                if (before(x, top)) top = x;
            }
            if (lane == 0) wave_best[wave] = top;
            __syncthreads();
            last = wave_best[0];
#pragma unroll 1
            for (int w = 1; w < PICK / 64; ++w)
                if (before(wave_best[w], last)) last = wave_best[w];
            if (tid == 0) best[k] = last;
            __syncthreads();
        }
    }

    // Their logits: none that is worse than the best of the W-th chunk counts.
    if (tid == 0) found = 0;
    __syncthreads();
    const Candidate worst = best[max(chunks - 1, 0)];
    for (int i = tid; i < chunks * CHUNK; i += PICK) {
        const Candidate of = best[i / CHUNK];
        const Beam &b = beams[of.beam];
        const int v = b.finished ? i % CHUNK : of.at * CHUNK + i % CHUNK;
        Candidate x{(double)NONE, NONE, of.beam, v};
        if (b.finished)   x.z = v == 0 ? 0.f : NONE;
        else if (v < a.V) x.z = logit_at<FP32>(reinterpret_cast<const char *>(a.logits) + (size_t)(row0 + of.beam) * a.V * (FP32 ? 4 : 2), v);
        x.rank = ranked(b, x.z);
        if (x.rank > (double)NONE && (chunks < W || x.rank >= worst.rank)) list[atomicAdd(&found, 1)] = x;
    }
    __syncthreads();
    const int m = found;
    for (int i = tid; i < m; i += PICK) {
        int number = 0;
        for (int j = 0; j < m; ++j) number += before(list[j], list[i]);
        if (number < W) winners[number] = list[i];
    }
    __syncthreads();
    if (tid < W) {
        const int row = row0 + tid;
        if (tid < m) {
            const Candidate x = winners[tid];
            const Beam &b = beams[x.beam];
            const int token = b.finished ? a.pad : x.at;
            a.source[row] = row0 + x.beam;
            a.token[row] = token;
            a.score_out[row] = (float)(b.finished ? b.score : b.score + ((double)x.z - b.lse));
            a.length_out[row] = b.tokens;
            a.finished_out[row] = b.finished || token == a.eos;
        } else {
            a.source[row] = row;
            a.token[row] = a.pad;
            a.score_out[row] = NONE;
            a.length_out[row] = 0;
            a.finished_out[row] = 0;
        }
    }
}

bool misaligned(const void *p, unsigned mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }

mlora_status check(const mlora_beam *d)
{
    if (!d) return MLORA_EINVAL;
    if (d->n_groups <= 0 || d->n_beams <= 0 || d->n_beams > MLORA_BEAM_MAX_BEAMS || d->vocab <= 0 || d->vocab > MLORA_BEAM_MAX_VOCAB) return MLORA_ESHAPE;
    if ((long long)d->n_groups * d->n_beams > MLORA_MAX_ROWS) return MLORA_ESHAPE;
    if (d->logits_dtype != MLORA_Y_BF16 && d->logits_dtype != MLORA_Y_FP32) return MLORA_EINVAL;
    if (!(d->length_power >= 0.f) || d->length_power > 3.0e38f) return MLORA_EINVAL;
    return MLORA_OK;
}

// Where the parts of the workspace begin: 8-byte numbers first.
struct Sizes {
    size_t rows, chunks, slices;
    size_t bytes() const { return rows * (slices * 12 + chunks * 4) + 256; }
};
Sizes sizes_of(const mlora_beam *d)
{
    return Sizes{(size_t)d->n_groups * d->n_beams, ((size_t)d->vocab + CHUNK - 1) / CHUNK, ((size_t)d->vocab + SLICE - 1) / SLICE};
}

}  // namespace
}  // namespace mlora

using namespace mlora;

extern "C" {

size_t mlora_beam_workspace_bytes(const mlora_beam *d)
{
    return check(d) == MLORA_OK ? sizes_of(d).bytes() : 0;
}

mlora_status mlora_beam_select(const mlora_beam *d, const void *logits, const float *score, const int32_t *length, const int32_t *finished,
                               int32_t *source, int32_t *token, float *score_out, int32_t *length_out, int32_t *finished_out,
                               void *workspace, size_t workspace_bytes, void *stream)
{
    const mlora_status st = check(d);
    if (st != MLORA_OK) return st;
    if (!logits || !score || !length || !finished || !source || !token || !score_out || !length_out || !finished_out) return MLORA_EINVAL;
    for (const void *p : {(const void *)score, (const void *)length, (const void *)finished, (const void *)source, (const void *)token,
                          (const void *)score_out, (const void *)length_out, (const void *)finished_out})
        if (misaligned(p, 3u)) return MLORA_EALIGN;
    if (misaligned(logits, d->logits_dtype == MLORA_Y_FP32 ? 3u : 1u)) return MLORA_EALIGN;
    const Sizes n = sizes_of(d);
    if (!workspace || workspace_bytes < n.bytes()) return MLORA_EWORKSPACE;
    if (misaligned(workspace, 255u)) return MLORA_EALIGN;
    BeamArgs a;
    a.logits = logits;
    a.score = score;
    a.length = length;
    a.finished = finished;
    a.source = source;
    a.token = token;
    a.score_out = score_out;
    a.length_out = length_out;
    a.finished_out = finished_out;
    a.slice_sum = reinterpret_cast<double *>(workspace);
    a.slice_top = reinterpret_cast<float *>(a.slice_sum + n.rows * n.slices);
    a.chunk_top = a.slice_top + n.rows * n.slices;
    a.W = d->n_beams;
    a.V = d->vocab;
    a.chunks = (int)n.chunks;
    a.slices = (int)n.slices;
    a.eos = d->eos;
    a.pad = d->pad;
    a.power = d->length_power;
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)((n.slices + 3) / 4), (unsigned)n.rows);
    const auto go = [&](auto fp32) {
        beam_stats<decltype(fp32)::value><<<grid, dim3(256), 0, s>>>(a);
        beam_pick<decltype(fp32)::value><<<dim3((unsigned)d->n_groups), dim3(PICK), 0, s>>>(a);
    };
    if (d->logits_dtype == MLORA_Y_FP32) go(std::true_type{});
    else                                 go(std::false_type{});
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
