// One step of beam search on the logits (see include/mlora_beam.h).
//
// A candidate's rank inside its beam is its logit's, so the W best of a group lie in the W chunks of 64 tokens whose best candidates are the
// best W (an order without equals: ranked score, beam, logit, token).  beam_stats goes over the logits once and leaves the largest logit
// of every chunk, and of every slice of 64 chunks the maximum and the sum of exponentials.  beam_pick, a block per group, makes
// the beams' log-sums, finds the best chunks by a bound that W of them reach, and looks at their logits once more.
//
// A large call is bound by the logits (8 groups of 16 beams over 128256 bf16 tokens: 9 to 11 us for 29.5 MB), and then by beam_pick's chain: what
// the slices left, the bound, the chunks above it, their logits, their order, 0.6 to 3.6 us each (12 to 14 us there; one group of 4 beams over
// 32003 fp32 tokens 3.5 to 5.5 us and 8, of which what the slices left and the bound are 2 each).  Ranks for all chunks in 64 bits, candidates
// ranked by one thread each and a bound found bit by bit were: 84 us for that block.
#include <type_traits>

#include "common.hpp"

#include "../../include/mlora_beam.h"

namespace mlora {

namespace {

constexpr int CHUNK = 64, SLICE = 64 * CHUNK;            // tokens
constexpr int PICK = 1024;                               // threads of beam_pick
constexpr int W_MAX = MLORA_BEAM_MAX_BEAMS;
constexpr int LIST = W_MAX * CHUNK;                      // candidates that are ranked at once
constexpr int FEW = 64, AT_ONCE = 4;                     // chunks that are looked at before they are ranked (256: 8 groups of 16 beams 13.2 -> 15.9 us); logits per thread at once
constexpr int QUADS = 1024;                              // groups of four chunks that are looked at one by one
constexpr int HELD = 8;                                  // loads of beam_pick at once
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
    float *chunk_top;                                    // [rows][slices][64]: -infinity behind the vocabulary
    float *slice_top;                                    // [rows][slices]
    double *slice_sum;                                   // [rows][slices], of exp(logit - slice_top)
    int W, V, slices, eos, pad;
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

// The largest of the lanes that hold a chunk together: neighbours, pairs, halves of 8 lanes, of 16
template <bool FP32>
__device__ __forceinline__ float chunk_max(float x)
{
    x = max_with<0xB1>(x);
    x = max_with<0x4E>(x);
    x = max_with<0x141>(x);
    if constexpr (FP32) x = max_with<0x140>(x);
    return x;
}

// e^d.  The fp32 number next to 1 / log 2 alone would make all exponentials of a row too large or too small together, by 10^-8 for each unit of d.
__device__ __forceinline__ float exp_of(float d)
{
    return __builtin_amdgcn_exp2f(__builtin_fmaf(d, 1.44269502162933349609f, d * 1.92596303350001e-8f));
}

// A wave per slice and row: 16 bytes per lane and load, side by side, so that a chunk is 8 (bf16) or 16 (fp32) neighbouring lanes.
template <bool FP32>
__global__ __launch_bounds__(256) void beam_stats(const BeamArgs a)
{
    constexpr int E = FP32 ? 4 : 8, LOADS = SLICE / (64 * E), SIZE = FP32 ? 4 : 2;
    const int lane = threadIdx.x & 63, slice = (int)blockIdx.x * 4 + (int)(threadIdx.x >> 6), row = blockIdx.y;
    if (slice >= a.slices) return;
    const char *const z = reinterpret_cast<const char *>(a.logits) + ((size_t)row * a.V + (size_t)slice * SLICE) * SIZE;
    float *const tops = a.chunk_top + ((size_t)row * a.slices + slice) * (SLICE / CHUNK);
    const int n = a.V - slice * SLICE;                   // tokens from here on
    const bool head = lane % (CHUNK / E) == 0;
    u32x4 raw[LOADS];
    if (n >= SLICE) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) raw[i] = *reinterpret_cast<const u32x4_any *>(z + (i * 64 + lane) * 16);
    } else {
        // the vocabulary's last slice: whole pieces, one that is not, and -infinity behind it
        constexpr unsigned NOTHING = FP32 ? 0xFF800000u : 0xFF80FF80u;
        u32x4 rest = {NOTHING, NOTHING, NOTHING, NOTHING};
        const int whole = n / E;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (whole * E + e < n) {
                if constexpr (FP32) rest[e] = reinterpret_cast<const unsigned *>(z)[whole * E + e];
                else                rest[e / 2] = e & 1 ? (rest[e / 2] & 0xFFFFu) | (unsigned)reinterpret_cast<const uint16_t *>(z)[whole * E + e] << 16
                                                        : (rest[e / 2] & 0xFFFF0000u) | reinterpret_cast<const uint16_t *>(z)[whole * E + e];
            }
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            raw[i] = u32x4{NOTHING, NOTHING, NOTHING, NOTHING};
            if (i * 64 + lane < whole) raw[i] = *reinterpret_cast<const u32x4_any *>(z + (i * 64 + lane) * 16);
            if (i * 64 + lane == whole) raw[i] = rest;
        }
    }
    if (a.finished[row] != 0) return;
    const auto at = [&](int i, int e) { return FP32 ? __uint_as_float(raw[i][e % 4]) : e & 1 ? __uint_as_float(raw[i][e / 2 % 4] & 0xFFFF0000u) : bf16_bits_to_float(raw[i][e / 2 % 4]); };
    float top = NONE, sum = 0.f;
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        float most = at(i, 0);
#pragma unroll
        for (int e = 1; e < E; ++e) most = fmaxf(most, at(i, e));
        most = chunk_max<FP32>(fmaxf(most, NONE));
        if (head) tops[(i * 64 + lane) * E / CHUNK] = most;
        top = fmaxf(top, most);
    }
#pragma unroll
    for (int d = 8; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    const float from = top == NONE ? 0.f : top;
#pragma unroll
    for (int i = 0; i < LOADS; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) sum += exp_of(at(i, e) - from);
    double all = sum;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d);
    if (lane == 0) {
        a.slice_top[(size_t)row * a.slices + slice] = top;
        a.slice_sum[(size_t)row * a.slices + slice] = all;
    }
}

struct Beam {
    double score, lse, per;                              // per: what the score of its candidates is multiplied by
    int finished, live, tokens;                          // tokens: of its candidates
};
// What beam b makes of a logit; -infinity: no candidate
__device__ __forceinline__ double ranked(const Beam &b, float z)
{
    return b.live && z > NONE ? (b.finished ? b.score : b.score + ((double)z - b.lse)) * b.per : (double)NONE;
}
// numbers, -infinity among them, as integers that order like them
__device__ __forceinline__ int in_order(float f)
{
    const int b = __float_as_int(f + 0.f);
    return b < 0 ? b ^ 0x7FFFFFFF : b;
}
__device__ __forceinline__ long long in_order(double f)
{
    const long long b = __double_as_longlong(f + 0.);
    return b < 0 ? b ^ 0x7FFFFFFFFFFFFFFFll : b;
}
struct Candidate {
    long long rank;
    float z;
    int beam, at;                                        // at: chunk, or token
};
__device__ __forceinline__ bool later(const Candidate &x, const Candidate &y)        // of equal rank: x behind y
{
    if (x.beam != y.beam) return x.beam > y.beam;
    if (x.z != y.z) return x.z < y.z;
    return x.at > y.at;
}
__device__ __forceinline__ bool before(const Candidate &x, const Candidate &y)
{
    return x.rank > y.rank || (x.rank == y.rank && later(y, x));
}

struct Quads {                                           // groups of four chunks with one that may count
    f32x4 z[QUADS];
    int task[QUADS], at[QUADS], found;
};
struct Place {
    int beam, at;
};
struct List {
    long long rank[LIST];
    float z[LIST];
    int beam[LIST], at[LIST], number[LIST];
    int found;
    __device__ Candidate get(int i) const { return Candidate{rank[i], z[i], beam[i], at[i]}; }
    __device__ void put(const Candidate &x)
    {
        const int i = atomicAdd(&found, 1);
        if (i < LIST) rank[i] = x.rank, z[i] = x.z, beam[i] = x.beam, at[i] = x.at;
    }
};
// The W best of a list of m <= LIST, each in its place.  Every wave looks at 64 of them and at a share of all.
__device__ __forceinline__ void best_of(List &list, int m, int W, Candidate *best)
{
    const int tid = threadIdx.x;
    int per = 64;
    while (per < m && per < PICK) per *= 2;
    for (int i = tid; i < m; i += PICK) list.number[i] = 0;
    __syncthreads();
    for (int i = tid & (per - 1); i < m; i += per) {
        const Candidate mine = list.get(i);
        int number = 0;
#pragma unroll 4
        for (int j = tid / per; j < m; j += PICK / per) {
            const long long other = list.rank[j];
            if (other > mine.rank) ++number;
            else if (other == mine.rank && j != i) number += later(mine, list.get(j));
        }
        if (number) atomicAdd(&list.number[i], number);
    }
    __syncthreads();
    for (int i = tid; i < m; i += PICK)
        if (list.number[i] < W) best[list.number[i]] = list.get(i);
    __syncthreads();
}

// A wave's shares are of one beam (two, if there are more beams than waves), so ranks are made for few of them: a bound on ranks is one on the logits of
// a beam.  Both passes over the chunks' best logits take four per lane and load.
template <bool FP32>
__global__ __launch_bounds__(PICK) void beam_pick(const BeamArgs a)
{
    constexpr int WAVES = PICK / 64;
    __shared__ Beam beams[W_MAX];
    __shared__ List list, picked;
    __shared__ Quads quads_of;
    __shared__ Candidate best[W_MAX], wave_best[WAVES];
    __shared__ int at_least;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), W = a.W, row0 = (int)blockIdx.x * W;
    // shares: `parts` waves per beam, its groups of four chunks dealt out in runs
    const int parts = W < WAVES ? WAVES / W : 1, quads = a.slices * 16, run = (quads + parts - 1) / parts;
    struct Share {
        const f32x4 *tops;
        int beam, first, n;                              // groups from first on
    };
    const auto share_of = [&](int t) {
        const int b = t / parts, first = (t - b * parts) * run;
        return Share{reinterpret_cast<const f32x4 *>(a.chunk_top) + (size_t)(row0 + b) * quads + first, b, first, min(run, quads - first)};
    };
    const auto load = [&](const Share &s, int q0, f32x4 (&z)[HELD]) {
#pragma unroll
        for (int u = 0; u < HELD; ++u) {
            const int q = q0 + u * 64 + lane;
            z[u] = f32x4{NONE, NONE, NONE, NONE};
            if (q < s.n) z[u] = s.tops[q];
        }
    };
    // (asked for before anything else; kept where a wave has no more than that)
    f32x4 z[HELD];
    const bool all = W * parts <= WAVES && run <= 64 * HELD;
    load(share_of(min(wave, W * parts - 1)), 0, z);
    // Few tokens: of groups, fewer lanes than W may have any, and nothing would be ruled out.  So here the bound is made from single chunks, and a second
    // beam's go to the other half of the lanes (32 beams: 4000 tokens 405 -> 27 us, 2000 118 -> 25; 24 beams, 4500 tokens 320 -> 20).
    const bool fine = run < 64;
    const auto load_fine = [&](const Share &s, int turn, float (&x)[4]) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int c = u * 64 + (lane ^ (turn & 1) * 32);
            x[u] = NONE;
            if (c < 4 * s.n) x[u] = reinterpret_cast<const float *>(s.tops)[c];
        }
    };
    float x[4] = {NONE, NONE, NONE, NONE};
    if (fine) load_fine(share_of(min(wave, W * parts - 1)), 0, x);
    const auto top_of = [&](const f32x4 &z) { return fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])); };

    for (int b = wave; b < W; b += WAVES) {
        const int row = row0 + b, done = a.finished[row], tokens = a.length[row] + (done ? 0 : 1);
        const float score = a.score[row];
        const float *const tops = a.slice_top + (size_t)row * a.slices;
        const double *const sums = a.slice_sum + (size_t)row * a.slices;
        float top = NONE;
        double sum = 0.;
        for (int i0 = 0; i0 < a.slices; i0 += 64) {      // (rows of finished beams hold anything)
            const int i = i0 + lane;
            const float here = i < a.slices ? tops[i] : NONE;
            const double part = i < a.slices ? sums[i] : 0.;
            float next = fmaxf(top, here);
#pragma unroll
            for (int d = 1; d < 64; d *= 2) next = fmaxf(next, __shfl_xor(next, d));
            const float from = next == NONE ? 0.f : next;
            sum = sum * (double)exp_of(top - from) + part * (double)exp_of(here - from);
            top = next;
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
        const double logs = log(lane == 1 ? fmax(1., (double)tokens) : sum), lse = (double)top + logs;
        const double per = a.power == 0.f ? 1. : exp(-(double)a.power * __shfl(logs, 1));
        if (lane == 0) beams[b] = Beam{score, lse, per, done, isfinite(score) && (done || isfinite(lse)), tokens};
    }
    if (tid == 0) list.found = picked.found = quads_of.found = 0, at_least = in_order(NONE);
    __syncthreads();

    // The W best chunks.  Of each wave's 64 lanes, the W-th best best chunk: that many chunks are at least as good, so nothing below the largest
    // such bound of all waves counts.
    float mine = NONE;
    for (int t = wave; t < W * parts; t += WAVES) {
        const Share s = share_of(t);
        const Beam &b = beams[s.beam];
        float most = NONE;
        if (b.finished) {
            most = s.first == 0 && lane == 0 ? 0.f : NONE;               // (its one candidate)
        } else if (fine) {
            if (t != wave) load_fine(s, t / WAVES, x);
            most = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
        } else {
            for (int q0 = 0; q0 < s.n; q0 += 64 * HELD) {
                if (t != wave || q0) load(s, q0, z);
#pragma unroll
                for (int u = 0; u < HELD; ++u) most = fmaxf(most, top_of(z[u]));
            }
        }
        mine = fmaxf(mine, (float)ranked(b, most));
    }
    {
        const unsigned key = (unsigned)in_order(mine) ^ 0x80000000u;
        unsigned lo = 0;                                 // the largest key that W lanes reach, two bits at a time from above, to 20 bits
#pragma unroll 1
        for (int bit = 30; bit >= 12; bit -= 2) {
            const unsigned t1 = lo | 1u << bit, t2 = lo | 2u << bit, t3 = lo | 3u << bit;
            const bool one = __popcll(__ballot(key >= t1)) >= W, two = __popcll(__ballot(key >= t2)) >= W, three = __popcll(__ballot(key >= t3)) >= W;
            lo = three ? t3 : two ? t2 : one ? t1 : lo;
        }
        if (lane == 0) atomicMax(&at_least, max((int)(lo ^ 0x80000000u), in_order(NONE)));
    }
    __syncthreads();
    const int bound = at_least;
    const float bound_rank = __int_as_float(bound < 0 ? bound ^ 0x7FFFFFFF : bound);
    // the bound as one on a live beam's logits, a little lower (ranks decide): what is below it has no part
    const auto lowest = [&](const Beam &b) {
        if (bound_rank == NONE) return -3.4028235e38f;
        const double low = ((double)bound_rank - fabs((double)bound_rank) * 0x1p-22 - 0x1p-148) / b.per - b.score, z = low + b.lse;
        return fmaxf((float)(z - (fabs(low) + fabs(b.lse)) * 0x1p-22), -3.4028235e38f);        // (a number, also where `per` is next to nothing)
    };
    for (int t = wave; t < W * parts; t += WAVES) {
        const Share s = share_of(t);
        const Beam &b = beams[s.beam];
        if (b.finished) {
            const double rank = ranked(b, 0.f);
            if (s.first == 0 && lane == 0 && b.live && in_order((float)rank) >= bound) list.put(Candidate{in_order(rank), 0.f, s.beam, 0});
            continue;
        }
        if (!b.live) continue;                           // (its logits may be +infinity, and reach any bound)
        const float from = lowest(b);
        for (int q0 = 0; q0 < s.n; q0 += 64 * HELD) {
            if (!all) load(s, q0, z);
#pragma unroll
            for (int u = 0; u < HELD; ++u)
                if (top_of(z[u]) >= from) {
                    const int i = atomicAdd(&quads_of.found, 1);
                    if (i < QUADS) quads_of.z[i] = z[u], quads_of.task[i] = t, quads_of.at[i] = q0 + u * 64 + lane;
                }
        }
    }
    __syncthreads();
    const int some = quads_of.found;
    for (int i = tid; i < 4 * min(some, QUADS); i += PICK) {
        const Share s = share_of(quads_of.task[i / 4]);
        const float x = quads_of.z[i / 4][i % 4];
        const double rank = ranked(beams[s.beam], x);
        if (rank > (double)NONE && in_order((float)rank) >= bound) list.put(Candidate{in_order(rank), x, s.beam, 4 * (s.first + quads_of.at[i / 4]) + i % 4});
    }
    __syncthreads();
    const int found = list.found;

    // The logits of n chunks that reach the bound, and rank `least`
    const auto look_at = [&](int n, const auto &chunk, long long least) {
        for (int i0 = tid; i0 < n * CHUNK; i0 += PICK * AT_ONCE) {
            float z[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = i0 + u * PICK;
                z[u] = NONE;
                if (i < n * CHUNK) {
                    const Place of = chunk(i / CHUNK);
                    const int v = of.at * CHUNK + i % CHUNK;
                    if (beams[of.beam].finished) z[u] = i % CHUNK == 0 ? 0.f : NONE;
                    else if (v < a.V)            z[u] = logit_at<FP32>(reinterpret_cast<const char *>(a.logits) + (size_t)(row0 + of.beam) * a.V * (FP32 ? 4 : 2), v);
                }
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                const int i = i0 + u * PICK;
                if (!(z[u] > NONE)) continue;
                const Place of = chunk(i / CHUNK);
                const double rank = ranked(beams[of.beam], z[u]);
                if (rank > (double)NONE && in_order((float)rank) >= bound && in_order(rank) >= least)
                    picked.put(Candidate{in_order(rank), z[u], of.beam, of.at * CHUNK + i % CHUNK});
            }
        }
        __syncthreads();
    };
    // As a rule few chunks reach the bound, and few of their logits.
    int m = LIST + 1;
    if (found <= FEW && some <= QUADS) {
        look_at(found, [&](int i) { return Place{list.beam[i], list.at[i]}; }, in_order((double)NONE));
        m = picked.found;
    }
    if (m > LIST) {
        // Else those of the W best chunks, of which there are W, that are no worse than the best of the W-th.
        __syncthreads();
        if (tid == 0) picked.found = 0;
        int chosen = min(W, found);
        if (found <= LIST && some <= QUADS) {
            best_of(list, found, W, best);
        } else {
            // (more equals than the list holds: one after the other)
            Candidate last{0x7FFFFFFFFFFFFFFFll, 0.f, -1, -1};
            for (chosen = 0; chosen < W; ++chosen) {
                Candidate top{in_order((double)NONE), NONE, W, 0};
                for (int t = wave; t < W * parts; t += WAVES) {
                    const Share s = share_of(t);
                    const Beam &b = beams[s.beam];
                    if (!b.live) continue;
                    const float from = lowest(b);
                    for (int c = lane; c < (b.finished ? 1 : 4 * s.n); c += 64) {
                        const float z = b.finished ? (s.first == 0 ? 0.f : NONE) : reinterpret_cast<const float *>(s.tops)[c];
                        const Candidate x{in_order(ranked(b, z)), z, s.beam, 4 * s.first + c};
                        if (z > NONE && (b.finished || z >= from) && x.rank > in_order((double)NONE) && before(last, x) && before(x, top)) top = x;
                    }
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
                for (int w = 1; w < WAVES; ++w)
                    if (before(wave_best[w], last)) last = wave_best[w];
                if (last.beam == W) break;               // (none is left: the same in all threads)
                if (tid == 0) best[chosen] = last;
                __syncthreads();
            }
        }
        look_at(chosen, [&](int i) { return Place{best[i].beam, best[i].at}; }, chosen < W ? in_order((double)NONE) : best[W - 1].rank);
        m = picked.found;
    }
    best_of(picked, m, W, best);
    if (tid < W) {
        const int row = row0 + tid;
        if (tid < m) {
            const Candidate x = best[tid];
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

// Rows, and what each leaves in the workspace.
struct Sizes {
    size_t rows, slices;
    size_t bytes() const { return rows * slices * (8 + 4 + 4 * (SLICE / CHUNK)) + 256; }
};
Sizes sizes_of(const mlora_beam *d)
{
    return Sizes{(size_t)d->n_groups * d->n_beams, ((size_t)d->vocab + SLICE - 1) / SLICE};
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
    a.chunk_top = reinterpret_cast<float *>(workspace);
    a.slice_sum = reinterpret_cast<double *>(a.chunk_top + n.rows * n.slices * (SLICE / CHUNK));
    a.slice_top = reinterpret_cast<float *>(a.slice_sum + n.rows * n.slices);
    a.W = d->n_beams;
    a.V = d->vocab;
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
