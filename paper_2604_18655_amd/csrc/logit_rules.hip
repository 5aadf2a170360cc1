// Penalties, biases and grammar masks on the logits of a draft tree's rows.
//
// Bound by one pass over the logits.  A block owns 512 tokens of one stream, eight per lane, and takes all rows of that
// stream, so counts and biases come from memory once, and new tokens enter the counts where they are read: no atomics, and
// no second launch.  Rows are dealt out to the block's waves, a wave asks for several at once, and everything that is looked up
// for a row or a token goes through LDS once: a wave that went through all 30 rows of a draft tree by itself, and looked
// masks and path tokens up in memory, spent its time waiting (8 streams, 128256 tokens: 60 us, now 27: 4.8 TB/s).  What a
// stream's counts and biases do to a token is the same in all its rows: one of two factors and a sum, made once (1 /
// repetition is rounded, which adds half a step to a logit); a token of a row's own path is looked up again, which is rare.  Rows of an odd vocabulary start anywhere: 16-byte accesses at their element's alignment.
#include <algorithm>
#include <type_traits>

#include "common.hpp"

#include "../../include/mlora_logit_rules.h"

namespace mlora {

namespace {

constexpr int RULES_V = 8;               // tokens of a thread

struct RulesArgs {
    const void *logits;
    void *out;
    const int *parent, *tokens, *new_tokens, *bias_row, *mask_row;
    int *counts;
    const float *repetition, *frequency, *presence, *bias;
    const unsigned *masks;
    size_t mask_words;                   // of a mask
    int S, R, T, V, n_new, n_bias, n_masks;
};

typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <class T> struct RulesPack;     // eight logits as they are stored, wherever they stand
template <> struct RulesPack<uint16_t> {
    u32x4_any w;
    __device__ __forceinline__ void load(const uint16_t *at) { w = *reinterpret_cast<const u32x4_any *>(at); }
    __device__ __forceinline__ float operator[](int i) const
    {
        const unsigned pair = w[i / 2];
        return i & 1 ? __uint_as_float(pair & 0xFFFF0000u) : __uint_as_float(pair << 16);
    }
};
template <> struct RulesPack<float> {
    u32x4_any w[2];
    __device__ __forceinline__ void load(const float *at)
    {
        w[0] = *reinterpret_cast<const u32x4_any *>(at);
        w[1] = *reinterpret_cast<const u32x4_any *>(at + 4);
    }
    __device__ __forceinline__ float operator[](int i) const
    {
        const unsigned x = w[i / 4][i % 4];
        return __uint_as_float(x);
    }
};
// PAST: by the caches
template <bool PAST>
__device__ __forceinline__ void rules_store(uint16_t *at, const float (&z)[RULES_V])
{
    const u32x4_any x = {pack_bf16(z[0], z[1]), pack_bf16(z[2], z[3]), pack_bf16(z[4], z[5]), pack_bf16(z[6], z[7])};
    if constexpr (PAST) __builtin_nontemporal_store(x, reinterpret_cast<u32x4_any *>(at));
    else                *reinterpret_cast<u32x4_any *>(at) = x;
}
template <bool PAST>
__device__ __forceinline__ void rules_store(float *at, const float (&z)[RULES_V])
{
    static_assert(!PAST, "(see the launch)");
    typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
    *reinterpret_cast<f32x4_any *>(at) = f32x4_any{z[0], z[1], z[2], z[3]};
    *reinterpret_cast<f32x4_any *>(at + 4) = f32x4_any{z[4], z[5], z[6], z[7]};
}
__device__ __forceinline__ float rules_one(uint16_t x) { return bf16_bits_to_float(x); }
__device__ __forceinline__ float rules_one(float x) { return x; }
__device__ __forceinline__ void rules_put(uint16_t &to, float x) { to = __builtin_bit_cast(uint16_t, (__bf16)x); }
__device__ __forceinline__ void rules_put(float &to, float x) { to = x; }

// What a stream's counts and biases do to a logit: z * (seen ? z > 0 ? inv : rep : 1) + (bias - penalty(count)).
struct Penalty {
    float rep, inv, freq, pres;
    __device__ __forceinline__ float add(int count, float bias) const { return count != 0 ? bias - fmaf(freq, (float)count, count > 0 ? pres : 0.f) : bias; }
    __device__ __forceinline__ float apply(float z, bool seen, float add) const
    {
        const float f = z > 0.f ? inv : rep;
        return fmaf(z, seen ? f : 1.f, add);
    }
};
// bit i of `allowed`: the value, or minus infinity
__device__ __forceinline__ float rules_mask(float z, int allowed, int i)
{
    const unsigned keep = (unsigned)__builtin_amdgcn_sbfe(allowed, i, 1);            // all bits or none
    return __uint_as_float((__float_as_uint(z) & keep) | (0xFF800000u & ~keep));
}

// A block takes 512 tokens of a stream, eight per lane, its waves every blockDim / 64-th row.  Where the vocabulary ends inside a
// lane's eight, they are the last eight and the first of them the lane before's: it stores its own only.
template <class T, int AHEAD, bool PAST>
__global__ __launch_bounds__(512) void logit_rules(const RulesArgs a)
{
    __shared__ unsigned long long path[MLORA_RULES_MAX_ROWS], same[MLORA_RULES_MAX_ROWS];
    __shared__ int token[MLORA_RULES_MAX_ROWS], mask_of[MLORA_RULES_MAX_ROWS];
    __shared__ int count_of[64 * RULES_V];
    __shared__ float bias_of[64 * RULES_V];
    const int s = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = (int)blockDim.x >> 6;
    const size_t row0 = (size_t)s * a.R, V = a.V;
    int v0 = ((int)blockIdx.x * 64 + lane) * RULES_V, first = 0;
    const bool mine = v0 < a.V;                                                  // this lane has tokens: v0 + first .. v0 + 7
    if (v0 + RULES_V > a.V) {
        first = min(RULES_V, v0 + RULES_V - a.V);
        v0 = a.V - RULES_V;
    }
    const T *const in = reinterpret_cast<const T *>(a.logits) + row0 * V + v0;
    T *const out = reinterpret_cast<T *>(a.out) + row0 * V + v0;

    // the wave's first rows are on their way while the rest is looked up
    RulesPack<T> raw[AHEAD];
    const auto ask = [&](int r0) {
        if (mine) {
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) raw[u].load(in + min(r0 + u * waves, a.R - 1) * V);
        }
    };
    ask(wave);
    Penalty p;
    p.rep = a.repetition ? a.repetition[s] : 1.f;
    p.inv = 1.f / p.rep;
    p.freq = a.frequency ? a.frequency[s] : 0.f;
    p.pres = a.presence ? a.presence[s] : 0.f;
    // the first wave looks up, for all of them, what the tokens and the rows are to get
    if (wave == 0) {
        const int table = a.n_bias > 0 ? a.bias_row[s] : -1;
        int *const counts = a.counts ? a.counts + (size_t)s * V + v0 : nullptr;
        int count[RULES_V];
        float bias[RULES_V];
#pragma unroll
        for (int e = 0; e < RULES_V; ++e) count[e] = counts && mine ? counts[e] : 0;
        // a row's mask, the token rows above it, the token rows of the same token; a parent is an earlier row: the walk ends
        const int at = min(lane, a.R - 1), up0 = a.parent[row0 + at], mask = a.n_masks > 0 ? a.mask_row[row0 + at] : -1;
        const int tok = a.tokens[(size_t)s * a.T + min(lane, a.T - 1)];
#pragma unroll
        for (int e = 0; e < RULES_V; ++e) bias[e] = mine && table >= 0 && table < a.n_bias ? a.bias[(size_t)table * V + v0 + e] : 0.f;
        mask_of[lane] = mask < a.n_masks ? mask : -1;
        token[lane] = tok;
        unsigned long long on = 0, alike = 0;
        int r = at;
        while (__ballot(r > 0)) {
            if (r > 0 && r < a.T) on |= 1ull << r;
            const int up = __shfl(up0, max(r, 0));
            r = r > 0 && up < r ? up : 0;
        }
        for (int t = 0; t < a.T; ++t) alike |= tok == __builtin_amdgcn_readlane(tok, t) ? 1ull << t : 0ull;
        path[lane] = on;
        same[lane] = alike;
        unsigned changed = 0;
        for (int i0 = 0; i0 < a.n_new; i0 += 64) {
            const int some = min(64, a.n_new - i0), its = a.new_tokens[(size_t)s * a.n_new + i0 + min(lane, some - 1)];
            for (int i = 0; i < some; ++i) {
                const int at = __builtin_amdgcn_readlane(its, i) - v0;
                if (mine && at >= first && at < RULES_V) {                       // (v0 + at: in [0, V))
                    changed |= 1u << at;
#pragma unroll
                    for (int e = 0; e < RULES_V; ++e) count[e] += e == at;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < RULES_V; ++e) {
            count_of[e * 64 + lane] = count[e];
            bias_of[e * 64 + lane] = bias[e];
            if (changed >> e & 1) counts[e] = count[e];
        }
    }
    __syncthreads();
    float add[RULES_V];
    bool seen[RULES_V];
#pragma unroll
    for (int e = 0; e < RULES_V; ++e) {
        const int count = count_of[e * 64 + lane];
        add[e] = p.add(count, bias_of[e * 64 + lane]);
        seen[e] = count > 0;
    }
    // the allowed tokens of a row, a bit each; without a branch: a row of no mask looks at the first one and forgets it
    const auto allowed = [&](int r) {
        const int m = mask_of[r];
        unsigned bits = ~0u;
        if (a.n_masks > 0) {
            const unsigned *const words = a.masks + max(m, 0) * a.mask_words;
            bits = words[v0 >> 5] >> (v0 & 31);
            if (first) bits |= words[(v0 + 7) >> 5] << 1 << (31 - (v0 & 31));    // (its eight may end in the next word)
        }
        return m >= 0 ? (int)bits : -1;
    };
    int bits[AHEAD];
    const auto ask_masks = [&](int r0) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) bits[u] = mine ? allowed(min(r0 + u * waves, a.R - 1)) : 0;
    };
    ask_masks(wave);
    unsigned long long hit = 0;                                                  // token rows whose token is one of this lane's
    for (int t = 1; t < a.T; ++t) {
        const int at = token[t] - v0;
        hit |= mine && at >= first && at < RULES_V ? 1ull << t : 0ull;
    }
    const bool hits = __any(hit != 0);
    if (!mine) return;                                                           // (no barrier from here on)

    for (int r0 = wave; r0 < a.R; r0 += AHEAD * waves) {
        if (r0 != wave) ask(r0), ask_masks(r0);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int r = r0 + u * waves;
            if (r >= a.R) break;
            float z[RULES_V];
#pragma unroll
            for (int e = 0; e < RULES_V; ++e) z[e] = p.apply(raw[u][e], seen[e], add[e]);
            if (hits) {
                // a token of the row's own path: counted on top
                for (unsigned long long m = hit & path[r]; m;) {
                    const int t = __ffsll(m) - 1, at = token[t] - v0;
                    const unsigned long long alike = same[t];
                    const int c = count_of[at * 64 + lane] + __popcll(m & alike);
                    float x = 0.f;
#pragma unroll
                    for (int e = 0; e < RULES_V; ++e) x = e == at ? raw[u][e] : x;
                    x = p.apply(x, c > 0, p.add(c, bias_of[at * 64 + lane]));
#pragma unroll
                    for (int e = 0; e < RULES_V; ++e) z[e] = e == at ? x : z[e];
                    m &= ~alike;
                }
            }
#pragma unroll
            for (int e = 0; e < RULES_V; ++e) z[e] = rules_mask(z[e], bits[u], e);
            if (first == 0) {
                rules_store<PAST>(out + r * V, z);
            } else {
#pragma unroll
                for (int e = 1; e < RULES_V; ++e)
                    if (e >= first) rules_put(out[r * V + e], z[e]);
            }
        }
    }
}

// Fewer than eight tokens: a thread per row, token by token.
template <class T>
__global__ __launch_bounds__(64) void logit_rules_few(const RulesArgs a)
{
    const int s = blockIdx.x, r = threadIdx.x;
    int *const counts = a.counts ? a.counts + (size_t)s * a.V : nullptr;
    int count[RULES_V];
    for (int v = 0; v < RULES_V; ++v) count[v] = counts && v < a.V ? counts[v] : 0;
    for (int i = 0; i < a.n_new; ++i)
        for (int v = 0; v < RULES_V; ++v) count[v] += v < a.V && a.new_tokens[(size_t)s * a.n_new + i] == v;
    __syncthreads();                                                             // all rows have read the counts
    if (r == 0 && a.n_new > 0)
        for (int v = 0; v < RULES_V; ++v)
            if (v < a.V) counts[v] = count[v];
    if (r >= a.R) return;
    const size_t row = (size_t)s * a.R + r;
    for (int at = r; at > 0;) {
        for (int v = 0; v < RULES_V; ++v) count[v] += at < a.T && v < a.V && a.tokens[(size_t)s * a.T + at] == v;
        const int up = a.parent[(size_t)s * a.R + at];
        at = up < at ? up : 0;
    }
    Penalty p;
    p.rep = a.repetition ? a.repetition[s] : 1.f;
    p.inv = 1.f / p.rep;
    p.freq = a.frequency ? a.frequency[s] : 0.f;
    p.pres = a.presence ? a.presence[s] : 0.f;
    const int table = a.n_bias > 0 ? a.bias_row[s] : -1, mask = a.n_masks > 0 ? a.mask_row[row] : -1;
    const bool biased = table >= 0 && table < a.n_bias, masked = mask >= 0 && mask < a.n_masks;
    for (int v = 0; v < RULES_V; ++v) {
        if (v >= a.V) break;
        const float z = p.apply(rules_one(reinterpret_cast<const T *>(a.logits)[row * a.V + v]), count[v] > 0,
                                p.add(count[v], biased ? a.bias[(size_t)table * a.V + v] : 0.f));
        rules_put(reinterpret_cast<T *>(a.out)[row * a.V + v], rules_mask(z, masked ? (int)a.masks[mask * a.mask_words] : -1, v));
    }
}

mlora_status check(const mlora_logit_rules *d)
{
    if (!d) return MLORA_EINVAL;
    if (d->logits_dtype != MLORA_Y_BF16 && d->logits_dtype != MLORA_Y_FP32) return MLORA_EINVAL;
    if (d->n_streams <= 0 || d->rows_per_stream <= 0 || d->rows_per_stream > MLORA_RULES_MAX_ROWS) return MLORA_ESHAPE;
    if ((long long)d->n_streams * d->rows_per_stream > MLORA_MAX_ROWS) return MLORA_ESHAPE;
    if (d->tokens_per_stream <= 0 || d->tokens_per_stream > d->rows_per_stream) return MLORA_ESHAPE;
    if (d->vocab <= 0 || d->vocab > (1 << 30) || d->n_bias < 0 || d->n_masks < 0) return MLORA_ESHAPE;
    if (!d->parent || (d->n_bias > 0 && (!d->bias || !d->bias_row)) || (d->n_masks > 0 && (!d->masks || !d->mask_row))) return MLORA_EINVAL;
    const void *words[] = {d->parent, d->counts, d->repetition, d->frequency, d->presence, d->bias, d->bias_row, d->masks, d->mask_row};
    for (const void *p : words)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return MLORA_EALIGN;
    return MLORA_OK;
}

}  // namespace
}  // namespace mlora

using namespace mlora;

extern "C" mlora_status mlora_logit_rules_apply(const mlora_logit_rules *d, const void *logits, const int32_t *tokens, const int32_t *new_tokens,
                                                int32_t n_new, void *out, void *stream)
{
    const mlora_status st = check(d);
    if (st != MLORA_OK) return st;
    if (n_new < 0 || n_new > MLORA_RULES_MAX_NEW) return MLORA_ESHAPE;
    if (!logits || !tokens || !out || (n_new > 0 && (!new_tokens || !d->counts))) return MLORA_EINVAL;
    const unsigned size = d->logits_dtype == MLORA_Y_BF16 ? 2 : 4;
    if ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out)) & (size - 1)) return MLORA_EALIGN;
    if ((reinterpret_cast<uintptr_t>(tokens) | reinterpret_cast<uintptr_t>(new_tokens)) & 3u) return MLORA_EALIGN;
    RulesArgs a;
    a.logits = logits;
    a.out = out;
    a.parent = d->parent;
    a.tokens = tokens;
    a.new_tokens = new_tokens;
    a.bias_row = d->bias_row;
    a.mask_row = d->mask_row;
    a.counts = d->counts;
    a.repetition = d->repetition;
    a.frequency = d->frequency;
    a.presence = d->presence;
    a.bias = d->bias;
    a.masks = d->masks;
    a.mask_words = (size_t)(d->vocab + 31) / 32;
    a.S = d->n_streams;
    a.R = d->rows_per_stream;
    a.T = d->tokens_per_stream;
    a.V = d->vocab;
    a.n_new = n_new;
    a.n_bias = d->n_bias;
    a.n_masks = d->n_masks;
    hipStream_t s = (hipStream_t)stream;
    if (d->vocab < RULES_V) {
        if (size == 2) logit_rules_few<uint16_t><<<dim3((unsigned)d->n_streams), dim3(64), 0, s>>>(a);
        else           logit_rules_few<float><<<dim3((unsigned)d->n_streams), dim3(64), 0, s>>>(a);
    } else {
        const int tiles = (d->vocab + 64 * RULES_V - 1) / (64 * RULES_V);
        // A wave per row up to four rows; then four rows at a time in up to four waves, or eight where there is no more than a
        // block per compute unit (us: 30 rows in 63 blocks 8.7 and 8.0, in 2008 31 and 33; 7 rows in 1004 blocks, one wave 9.3, two 7.8).
        const int most = (long long)tiles * a.S <= 256 ? 8 : 4, waves = a.R <= 4 ? a.R : std::min(most, (a.R + 3) / 4);
        const dim3 grid((unsigned)tiles, (unsigned)a.S), block(64u * (unsigned)waves);
        // bf16 results of their own that outgrow the second-level caches (8 x 4 MB) go past them: 8 streams x 30 rows x 128256 tokens
        // 33.0 -> 26.6 us, with the draft step that reads them 51.5 -> 46.6 (with a plain copy of them 52.6 -> 57.4); of 64000
        // tokens 17.5 -> 16.9, 33.7 -> 32.3.  In place 26.9 -> 27.7, and fp32 with the draft step 78.3 -> 80.2: not those.
        const bool past = out != logits && size == 2 && (double)a.S * a.R * a.V * 2 > (double)(32 << 20);
        const auto go = [&](auto ahead, auto by) {
            constexpr int AHEAD = decltype(ahead)::value;
            constexpr bool PAST = decltype(by)::value;
            if (PAST || size == 2) logit_rules<uint16_t, AHEAD, PAST><<<grid, block, 0, s>>>(a);
            else                   logit_rules<float, AHEAD, false><<<grid, block, 0, s>>>(a);
        };
        constexpr std::integral_constant<int, 1> one{};
        constexpr std::integral_constant<int, 4> four{};
        if (past) a.R <= 4 ? go(one, std::true_type{}) : go(four, std::true_type{});
        else      a.R <= 4 ? go(one, std::false_type{}) : go(four, std::false_type{});
    }
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}
