// Penalties, biases and grammar masks on the logits of a draft tree's rows.
//
// Bound by one pass over the logits.  A thread owns eight neighbouring tokens of one stream and takes all rows of that
// stream, so counts and biases are read once for all rows, and new tokens enter the counts where they are read: no atomics,
// and no second launch.  Most tokens have never been given out: where no lane of a wave has one that was, a row costs an add
// and a mask bit per token.  Rows of an odd vocabulary start anywhere: 16-byte accesses at their element's alignment.
#include "common.hpp"

#include "../../include/mlora_logit_rules.h"

namespace mlora {

namespace {

constexpr int RULES_V = 8;               // tokens of a thread
constexpr int RULES_AHEAD = 4;           // rows asked for at a time

struct RulesArgs {
    const void *logits;
    void *out;
    const int *parent, *tokens, *new_tokens, *bias_row, *mask_row;
    int *counts;
    const float *repetition, *frequency, *presence, *bias;
    const uint8_t *masks;
    size_t mask_bytes;                   // of a mask
    int R, T, V, n_new, n_bias, n_masks;
};

typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
template <class T> struct RulesPack;     // eight logits as they are stored
template <> struct RulesPack<uint16_t> { u32x4_any w; };
template <> struct RulesPack<float> { u32x4_any w[2]; };

__device__ __forceinline__ void rules_load(RulesPack<uint16_t> &p, const uint16_t *at, int n)
{
    if (n >= RULES_V) { p.w = *reinterpret_cast<const u32x4_any *>(at); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned lo = 2 * i < n ? at[2 * i] : 0u, hi = 2 * i + 1 < n ? at[2 * i + 1] : 0u;
        p.w[i] = lo | hi << 16;
    }
}
__device__ __forceinline__ void rules_load(RulesPack<float> &p, const float *at, int n)
{
    if (n >= RULES_V) {
        p.w[0] = *reinterpret_cast<const u32x4_any *>(at);
        p.w[1] = *reinterpret_cast<const u32x4_any *>(at + 4);
        return;
    }
#pragma unroll
    for (int i = 0; i < RULES_V; ++i) p.w[i / 4][i % 4] = i < n ? __float_as_uint(at[i]) : 0u;
}
__device__ __forceinline__ float rules_get(const RulesPack<uint16_t> &p, int i)
{
    const unsigned w = p.w[i / 2];
    return i & 1 ? __uint_as_float(w & 0xFFFF0000u) : __uint_as_float(w << 16);
}
__device__ __forceinline__ float rules_get(const RulesPack<float> &p, int i)
{
    const unsigned w = p.w[i / 4][i % 4];
    return __uint_as_float(w);
}
__device__ __forceinline__ void rules_store(uint16_t *at, const float (&z)[RULES_V], int n)
{
    u32x4_any w;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = pack_bf16(z[2 * i], z[2 * i + 1]);
    if (n >= RULES_V) { *reinterpret_cast<u32x4_any *>(at) = w; return; }
#pragma unroll
    for (int i = 0; i < RULES_V; ++i) {
        const unsigned pair = w[i / 2];
        if (i < n) at[i] = (uint16_t)(i & 1 ? pair >> 16 : pair & 0xFFFFu);
    }
}
__device__ __forceinline__ void rules_store(float *at, const float (&z)[RULES_V], int n)
{
    if (n >= RULES_V) {
        typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
        *reinterpret_cast<f32x4_any *>(at) = f32x4_any{z[0], z[1], z[2], z[3]};
        *reinterpret_cast<f32x4_any *>(at + 4) = f32x4_any{z[4], z[5], z[6], z[7]};
        return;
    }
#pragma unroll
    for (int i = 0; i < RULES_V; ++i)
        if (i < n) at[i] = z[i];
}

template <class T>
__global__ void logit_rules(const RulesArgs a)
{
    __shared__ unsigned long long path[MLORA_RULES_MAX_ROWS];
    __shared__ int token[MLORA_RULES_MAX_ROWS];
    const int s = blockIdx.y, tid = threadIdx.x;
    const int v0 = ((int)blockIdx.x * (int)blockDim.x + tid) * RULES_V;          // (below 2^30 + 2^14)
    const int n = min(RULES_V, a.V - v0);                                        // tokens of this thread; none where it is not positive
    const size_t row0 = (size_t)s * a.R;

    // (the block has 64 threads at least) the token rows above a row; a parent is an earlier row: the walk ends
    if (tid < a.T) token[tid] = a.tokens[s * a.T + tid];
    if (tid < a.R) {
        unsigned long long on = 0;
        for (int r = tid; r > 0;) {
            if (r < a.T) on |= 1ull << r;
            const int up = a.parent[row0 + r];
            r = up < r ? up : 0;
        }
        path[tid] = on;
    }
    int count[RULES_V];
    float bias[RULES_V];
    const int table = a.n_bias > 0 ? a.bias_row[s] : -1;
    const bool biased = table >= 0 && table < a.n_bias;
#pragma unroll
    for (int e = 0; e < RULES_V; ++e) {
        count[e] = a.counts && e < n ? a.counts[(size_t)s * a.V + v0 + e] : 0;
        bias[e] = biased && e < n ? a.bias[(size_t)table * a.V + v0 + e] : 0.f;
    }
    for (int i = 0; i < a.n_new; ++i) {
        const int at = a.new_tokens[(size_t)s * a.n_new + i] - v0;
        if (at >= 0 && at < n) {                                                 // (v0 + at: in [0, V))
            int now = 0;
#pragma unroll
            for (int e = 0; e < RULES_V; ++e) {
                count[e] += e == at;
                now = e == at ? count[e] : now;
            }
            a.counts[(size_t)s * a.V + v0 + at] = now;
        }
    }
    __syncthreads();
    unsigned long long hit = 0;                                                  // token rows whose token is one of this thread's
    for (int t = 1; t < a.T; ++t) {
        const int at = token[t] - v0;
        hit |= at >= 0 && at < n ? 1ull << t : 0ull;
    }
    bool seen = hit != 0;
#pragma unroll
    for (int e = 0; e < RULES_V; ++e) seen |= count[e] != 0;
    const bool wave_seen = __any(seen);
    const float rep = a.repetition ? a.repetition[s] : 1.f, freq = a.frequency ? a.frequency[s] : 0.f, pres = a.presence ? a.presence[s] : 0.f;
    if (n <= 0) return;

    const T *const in = reinterpret_cast<const T *>(a.logits) + row0 * a.V + v0;
    T *const out = reinterpret_cast<T *>(a.out) + row0 * a.V + v0;
    for (int r0 = 0; r0 < a.R; r0 += RULES_AHEAD) {
        RulesPack<T> raw[RULES_AHEAD];
        unsigned allowed[RULES_AHEAD];
#pragma unroll
        for (int u = 0; u < RULES_AHEAD; ++u) {
            const int r = min(r0 + u, a.R - 1);
            rules_load(raw[u], in + (size_t)r * a.V, n);
            const int mask = a.n_masks > 0 ? a.mask_row[row0 + r] : -1;
            allowed[u] = mask >= 0 && mask < a.n_masks ? a.masks[mask * a.mask_bytes + (v0 >> 3)] : 0xFFu;
        }
#pragma unroll
        for (int u = 0; u < RULES_AHEAD; ++u) {
            const int r = r0 + u;
            if (r >= a.R) break;
            float z[RULES_V];
#pragma unroll
            for (int e = 0; e < RULES_V; ++e) z[e] = rules_get(raw[u], e);
            if (wave_seen) {
                int c[RULES_V];
#pragma unroll
                for (int e = 0; e < RULES_V; ++e) c[e] = count[e];
                for (unsigned long long m = hit & path[r]; m; m &= m - 1) {
                    const int at = token[__ffsll((unsigned long long)m) - 1] - v0;
#pragma unroll
                    for (int e = 0; e < RULES_V; ++e) c[e] += e == at;
                }
#pragma unroll
                for (int e = 0; e < RULES_V; ++e)
                    if (c[e] != 0) {
                        const float f = (float)c[e];
                        if (c[e] > 0) z[e] = z[e] > 0.f ? z[e] / rep : z[e] * rep;
                        z[e] -= fmaf(freq, f, c[e] > 0 ? pres : 0.f);
                    }
            }
#pragma unroll
            for (int e = 0; e < RULES_V; ++e) {
                z[e] += bias[e];
                z[e] = allowed[u] >> e & 1 ? z[e] : -__builtin_inff();
            }
            rules_store(out + (size_t)r * a.V, z, n);
        }
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
    a.masks = reinterpret_cast<const uint8_t *>(d->masks);
    a.mask_bytes = (size_t)(d->vocab + 31) / 32 * 4;
    a.R = d->rows_per_stream;
    a.T = d->tokens_per_stream;
    a.V = d->vocab;
    a.n_new = n_new;
    a.n_bias = d->n_bias;
    a.n_masks = d->n_masks;
    // blocks of one wave until those of four would fill the compute units four times
    const int threads = (long long)d->n_streams * ((d->vocab + 2047) / 2048) < 1024 ? 64 : 256;
    const dim3 grid((unsigned)((d->vocab + threads * RULES_V - 1) / (threads * RULES_V)), (unsigned)d->n_streams), block((unsigned)threads);
    if (size == 2) logit_rules<uint16_t><<<grid, block, 0, (hipStream_t)stream>>>(a);
    else           logit_rules<float><<<grid, block, 0, (hipStream_t)stream>>>(a);
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}
