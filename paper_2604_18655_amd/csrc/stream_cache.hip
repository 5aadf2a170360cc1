// The streams' own cache segments at a bounded size: rows of a step enter them in the place of the slots with the least
// accumulated attention weight, and the heaviest slots of a long segment are copied into a smaller one.
//
// Both need the K highest-ranked of a head's live slots.  A slot's rank is a 32-bit number that orders like the stated
// rule (protected slots the largest, NaN the smallest), and equal numbers in the order of the slots.  A block finds
// the K-th largest number by histograms of 11, 11 and 10 bits in LDS, then counts slots in their order.
#include <algorithm>

#include "common.hpp"

#include "../../include/mlora_stream_cache.h"

namespace mlora {

namespace {

constexpr int BINS = 2048;

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned rank_of(float mass, int pos, int newest, int sink)
{
    unsigned b = __float_as_uint(mass);
    if (b == 0x80000000u) b = 0;                                     // -0 counts as +0
    const bool nan = (b & 0x7FFFFFFFu) > 0x7F800000u;
    const unsigned r = nan ? 0u : (b & 0x80000000u) ? ~b : b | 0x80000000u;
    return pos >= newest || pos < sink ? 0xFFFFFFFFu : r;
}

// What a head's slots are ranked by.
struct Head {
    const float *mass;
    const int *pos;
    int live;                            // slots
    int newest, sink;                    // protected: pos >= newest or pos < sink
};

// KPT consecutive slots per thread, a chunk of THREADS * KPT at a time
template <int THREADS, int KPT>
__device__ __forceinline__ void ranks_of(const Head &h, int first, unsigned (&r)[KPT])
{
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        const int t = min(first + i, h.live - 1);
        r[i] = rank_of(h.mass[t], h.pos[t], h.newest, h.sink);
    }
}

// sum of v over the threads before this one, and over all of them
template <int THREADS>
__device__ __forceinline__ int block_scan(int v, int *wave_sum, int &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int up = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(up, d);
        if (lane >= d) up += o;
    }
    if (lane == 63) wave_sum[wave] = up;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        const int x = wave_sum[w];
        before += w < wave ? x : 0;
        total += x;
    }
    __syncthreads();
    return before + up - v;
}

struct Cut {
    unsigned top;                        // ranks whose bits from `shift` on are above this are kept
    int shift;
    int ties;                            // of those equal to it, as many are kept, in the order of the slots
    __device__ __forceinline__ int side(unsigned r) const { return (r >> shift) > top ? 1 : (r >> shift) == top ? 0 : -1; }
};

template <int THREADS>
struct SelectLds {
    int bins[BINS];
    int wave_sum[THREADS / 64];
    int found[2];
};

// The cut that leaves the `keep` highest of the head's live slots, 0 < keep < live.  `held` are the ranks of the only chunk
// (live <= THREADS * KPT), else they are made anew in every pass.
template <int THREADS, int KPT>
__device__ __forceinline__ Cut find_cut(const Head &h, int keep, unsigned (&held)[KPT], SelectLds<THREADS> &lds)
{
    const int tid = threadIdx.x, lane = tid & 63;
    constexpr int CHUNK = THREADS * KPT, PER = BINS / THREADS;
    Cut cut{0u, 32, 0};
    unsigned prefix = 0;
    int left = keep, shift = 32;
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10, above = shift;
        shift -= bits;
#pragma unroll
        for (int i = 0; i < PER; ++i) lds.bins[i * THREADS + tid] = 0;
        __syncthreads();
        for (int c0 = 0; c0 < h.live; c0 += CHUNK) {
            unsigned r[KPT];
            if (h.live > CHUNK) ranks_of<THREADS, KPT>(h, c0 + tid * KPT, r);
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                const unsigned x = h.live > CHUNK ? r[i] : held[i];
                const bool mine = c0 + tid * KPT + i < h.live && (pass == 0 || x >> (above & 31) == prefix);
                const unsigned digit = x >> shift & ((1u << bits) - 1);
                // equal digits all over the wave (masses that are all zero) are added up first
                const unsigned long long all = __ballot(mine);
                if (all == 0) continue;
                const unsigned one = __shfl(digit, __ffsll(all) - 1);
                if (__ballot(mine && digit == one) == all) {
                    if (lane == __ffsll(all) - 1) atomicAdd(&lds.bins[one], __popcll(all));
                } else if (mine) {
                    atomicAdd(&lds.bins[digit], 1);
                }
            }
        }
        __syncthreads();
        // the bin that holds the left-th largest: thread t looks at bins from the top, PER each
        int n[PER], sum = 0, total;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            n[i] = lds.bins[BINS - 1 - (tid * PER + i)];
            sum += n[i];
        }
        int before = block_scan<THREADS>(sum, lds.wave_sum, total);
        if (before < left && left <= before + sum) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (before < left && left <= before + n[i]) {
                    lds.found[0] = BINS - 1 - (tid * PER + i);
                    lds.found[1] = before;
                    lds.bins[0] = n[i];                              // (all bins have been read)
                }
                before += n[i];
            }
        }
        __syncthreads();
        const int bin = lds.found[0], in_bin = lds.bins[0];
        left -= lds.found[1];
        prefix = prefix << bits | (unsigned)bin;
        cut = Cut{prefix, shift, left};
        __syncthreads();
        if (left == in_bin) break;                                   // all of them: no finer cut is needed
    }
    return cut;
}

// Calls use(slot, kept?, number) for every live slot, `number` counting the kept (KEPT) or the other slots in their order.
template <int THREADS, int KPT, bool KEPT, class Use>
__device__ __forceinline__ void in_order(const Head &h, const Cut &cut, unsigned (&held)[KPT], SelectLds<THREADS> &lds, const Use &use)
{
    const int tid = threadIdx.x;
    constexpr int CHUNK = THREADS * KPT;
    int ties = 0, count = 0;
    for (int c0 = 0; c0 < h.live; c0 += CHUNK) {
        unsigned r[KPT];
        if (h.live > CHUNK) ranks_of<THREADS, KPT>(h, c0 + tid * KPT, r);
        int equal = 0, total;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            if (h.live <= CHUNK) r[i] = held[i];
            equal += c0 + tid * KPT + i < h.live && cut.side(r[i]) == 0;
        }
        int tie = ties + block_scan<THREADS>(equal, lds.wave_sum, total);
        ties += total;
        unsigned wanted = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const bool live = c0 + tid * KPT + i < h.live;
            const int side = cut.side(r[i]);
            const bool kept = side > 0 || (side == 0 && tie < cut.ties);
            tie += live && side == 0;
            wanted |= live && kept == KEPT ? 1u << i : 0u;
        }
        int number = count + block_scan<THREADS>(__popc(wanted), lds.wave_sum, total);
        count += total;
#pragma unroll
        for (int i = 0; i < KPT; ++i)
            if (wanted >> i & 1) use(c0 + tid * KPT + i, number++);
    }
}

struct CacheArgs {
    uint16_t *k, *v;
    float *mass;
    int *slot_pos, *len, *next_pos;
    unsigned *tickets;
    int L, S, H, cap;
};

// entries of a stream's list before the first that names no row; every wave finds it by itself
__device__ __forceinline__ int listed(const int *rows, int n_rows, int R)
{
    if (!rows) return R;
    const int lane = threadIdx.x & 63;
    for (int j0 = 0; j0 < n_rows; j0 += 64) {
        const int r = j0 + lane < n_rows ? rows[j0 + lane] : 0;
        const unsigned long long bad = __ballot(r < 0 || r >= R);
        if (bad) return j0 + __ffsll(bad) - 1;
    }
    return n_rows;
}

struct AppendArgs {
    CacheArgs c;
    const uint16_t *k_new, *v_new;
    const int *rows;
    int R, n_rows, budget, sink, recent;
};

// A block per layer, stream and head.
template <int THREADS, int KPT, int D>
__global__ __launch_bounds__(THREADS) void cache_append(const AppendArgs a)
{
    __shared__ SelectLds<THREADS> lds;
    extern __shared__ int taken[];                                   // slots that give way
    const int tid = threadIdx.x, H = a.c.H, S = a.c.S, cap = a.c.cap;
    const int head = blockIdx.x, l = head / (S * H), s = head / H % S, h = head % H;
    const int *const rows = a.rows ? a.rows + (size_t)s * a.n_rows : nullptr;
    const int live = max(0, min(a.c.len[s], cap)), next = a.c.next_pos[s];
    const int n = listed(rows, a.n_rows, a.R);
    const int room = min(n, max(live, a.budget) - live), out = n - room;
    const size_t slots = (size_t)head * cap;
    if (out > 0) {
        const Head hd{a.c.mass + slots, a.c.slot_pos + slots, live, next - a.recent, a.sink};
        unsigned held[KPT];
        if (live <= THREADS * KPT) ranks_of<THREADS, KPT>(hd, tid * KPT, held);
        Cut cut{0xFFFFFFFFu, 0, 0};                                  // (all give way: ranks equal to it are ties beyond the count)
        if (out < live) cut = find_cut<THREADS, KPT>(hd, live - out, held, lds);
        in_order<THREADS, KPT, false>(hd, cut, held, lds, [&](int slot, int number) { taken[number] = slot; });
        __syncthreads();
    }
    constexpr int PIECES = D / 8;                                    // of 16 bytes in a row
    for (int i = tid; i < n * 2 * PIECES; i += THREADS) {
        const int j = i / (2 * PIECES), piece = i % PIECES, value = i / PIECES % 2;
        const int slot = j < room ? live + j : taken[j - room];
        const int r = rows ? rows[j] : j;
        const size_t from = (((size_t)l * S + s) * a.R + r) * H + h;
        const u32x4 *src = reinterpret_cast<const u32x4 *>((value ? a.v_new : a.k_new) + from * D) + piece;
        reinterpret_cast<u32x4 *>((value ? a.c.v : a.c.k) + (slots + slot) * D)[piece] = *src;
        if (piece == 0) {
            if (value) a.c.slot_pos[slots + slot] = next + j;
            else       a.c.mass[slots + slot] = 0.f;
        }
    }
    // the stream's last block moves its length on: all others have read it (a ticket is drawn behind the barrier)
    __syncthreads();
    if (tid == 0) {
        const unsigned last = (unsigned)(a.c.L * H) - 1;
        __threadfence();
        if (atomicInc(a.c.tickets + s, last) == last) {
            a.c.len[s] = live + room;
            a.c.next_pos[s] = next + n;
        }
    }
}

struct CompressArgs {
    CacheArgs from, to;
    int *kept;
    int budget, sink, recent;
};

template <int THREADS, int KPT>
__global__ __launch_bounds__(THREADS) void cache_select(const CompressArgs a)
{
    __shared__ SelectLds<THREADS> lds;
    const int tid = threadIdx.x, H = a.from.H, S = a.from.S;
    const int head = blockIdx.x, s = head / H % S;
    const int live = max(0, min(a.from.len[s], a.from.cap)), next = a.from.next_pos[s], keep = min(live, a.budget);
    const size_t slots = (size_t)head * a.from.cap;
    int *const kept = a.kept + (size_t)head * a.budget;
    if (keep < live) {
        const Head hd{a.from.mass + slots, a.from.slot_pos + slots, live, next - a.recent, a.sink};
        unsigned held[KPT];
        if (live <= THREADS * KPT) ranks_of<THREADS, KPT>(hd, tid * KPT, held);
        const Cut cut = find_cut<THREADS, KPT>(hd, keep, held, lds);
        in_order<THREADS, KPT, true>(hd, cut, held, lds, [&](int slot, int number) { kept[number] = slot; });
    } else {
        for (int i = tid; i < keep; i += THREADS) kept[i] = i;
    }
    for (int i = keep + tid; i < a.budget; i += THREADS) kept[i] = -1;
    if (tid == 0 && head % (S * H) == s * H && head < S * H) {
        a.to.len[s] = keep;
        a.to.next_pos[s] = next;
    }
}

// A wave copies 64 slots of a head, 64 lanes side by side along the rows.
template <int D>
__global__ __launch_bounds__(256) void cache_gather(const CompressArgs a)
{
    constexpr int PIECES = D / 8, AT_ONCE = 64 / PIECES, STEPS = 64 / AT_ONCE, AHEAD = 4;
    const int runs = (a.budget + 63) / 64, lane = threadIdx.x & 63;
    const long long task = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int head = (int)(task / runs), j0 = (int)(task - (long long)head * runs) * 64;
    if (head >= a.from.L * a.from.S * a.from.H) return;
    const int slot = j0 + lane < a.budget ? a.kept[(size_t)head * a.budget + j0 + lane] : -1;
    const size_t from = (size_t)head * a.from.cap, to = (size_t)head * a.to.cap + j0;
    if (slot >= 0) {
        a.to.mass[to + lane] = a.from.mass[from + slot];
        a.to.slot_pos[to + lane] = a.from.slot_pos[from + slot];
    }
    const int piece = lane % PIECES, row = lane / PIECES;
    const u32x4 *const ks = reinterpret_cast<const u32x4 *>(a.from.k + from * D) + piece, *const vs = reinterpret_cast<const u32x4 *>(a.from.v + from * D) + piece;
    u32x4 *const kt = reinterpret_cast<u32x4 *>(a.to.k + to * D) + piece, *const vt = reinterpret_cast<u32x4 *>(a.to.v + to * D) + piece;
    for (int i0 = 0; i0 < STEPS; i0 += AHEAD) {
        u32x4 kv[AHEAD], vv[AHEAD];
        int src[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            src[u] = __shfl(slot, (i0 + u) * AT_ONCE + row);
            if (src[u] >= 0) {
                kv[u] = ks[(size_t)src[u] * PIECES];
                vv[u] = vs[(size_t)src[u] * PIECES];
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (src[u] >= 0) {
                kt[((i0 + u) * AT_ONCE + row) * PIECES] = kv[u];
                vt[((i0 + u) * AT_ONCE + row) * PIECES] = vv[u];
            }
    }
}

mlora_status check(const mlora_stream_cache *c)
{
    if (!c) return MLORA_EINVAL;
    if (c->head_dim != 64 && c->head_dim != 128) return MLORA_ESHAPE;
    if (c->n_layers <= 0 || c->n_streams <= 0 || c->n_kv_heads <= 0 || c->cap <= 0 || c->cap > MLORA_CACHE_MAX_SLOTS) return MLORA_ESHAPE;
    if ((double)c->n_layers * c->n_streams * c->n_kv_heads > MLORA_CACHE_MAX_HEADS) return MLORA_ESHAPE;
    if (!c->k || !c->v || !c->mass || !c->slot_pos || !c->len || !c->next_pos || !c->tickets) return MLORA_EINVAL;
    if ((reinterpret_cast<uintptr_t>(c->k) | reinterpret_cast<uintptr_t>(c->v)) & 15u) return MLORA_EALIGN;
    const void *words[] = {c->mass, c->slot_pos, c->len, c->next_pos, c->tickets};
    for (const void *p : words)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return MLORA_EALIGN;
    return MLORA_OK;
}

CacheArgs args_of(const mlora_stream_cache *c)
{
    return CacheArgs{reinterpret_cast<uint16_t *>(c->k), reinterpret_cast<uint16_t *>(c->v), c->mass, c->slot_pos, c->len, c->next_pos, c->tickets,
                     c->n_layers, c->n_streams, c->n_kv_heads, c->cap};
}

}  // namespace
}  // namespace mlora

using namespace mlora;

extern "C" {

mlora_status mlora_stream_cache_append(const mlora_stream_cache *c, const void *k_new, const void *v_new, int32_t rows_per_stream,
                                       const int32_t *rows, int32_t n_rows, int32_t budget, int32_t sink, int32_t recent, void *stream)
{
    const mlora_status st = check(c);
    if (st != MLORA_OK) return st;
    if (!k_new || !v_new) return MLORA_EINVAL;
    if ((reinterpret_cast<uintptr_t>(k_new) | reinterpret_cast<uintptr_t>(v_new)) & 15u) return MLORA_EALIGN;
    if (reinterpret_cast<uintptr_t>(rows) & 3u) return MLORA_EALIGN;
    if (rows_per_stream <= 0 || (long long)c->n_streams * rows_per_stream > MLORA_MAX_ROWS) return MLORA_ESHAPE;
    const int n = rows ? n_rows : rows_per_stream;
    if (n < 1 || n > rows_per_stream || budget < n || budget > c->cap || sink < 0 || recent < 0) return MLORA_ESHAPE;
    AppendArgs a{args_of(c), reinterpret_cast<const uint16_t *>(k_new), reinterpret_cast<const uint16_t *>(v_new), rows, rows_per_stream, n,
                 budget, sink, recent};
    const dim3 grid((unsigned)(a.c.L * a.c.S * a.c.H));
    const size_t taken = (size_t)n * sizeof(int);
    hipStream_t s = (hipStream_t)stream;
    if (c->head_dim == 64) cache_append<256, 16, 64><<<grid, dim3(256), taken, s>>>(a);
    else                   cache_append<256, 16, 128><<<grid, dim3(256), taken, s>>>(a);
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

mlora_status mlora_stream_cache_compress(const mlora_stream_cache *from, const mlora_stream_cache *to, int32_t *kept,
                                         int32_t budget, int32_t sink, int32_t recent, void *stream)
{
    mlora_status st = check(from);
    if (st == MLORA_OK) st = check(to);
    if (st != MLORA_OK) return st;
    if (!kept) return MLORA_EINVAL;
    if (reinterpret_cast<uintptr_t>(kept) & 3u) return MLORA_EALIGN;
    if (from->n_layers != to->n_layers || from->n_streams != to->n_streams || from->n_kv_heads != to->n_kv_heads || from->head_dim != to->head_dim)
        return MLORA_ESHAPE;
    if (budget < 1 || budget > to->cap || sink < 0 || recent < 0) return MLORA_ESHAPE;
    if (from->k == to->k || from->v == to->v || from->mass == to->mass || from->slot_pos == to->slot_pos || from->len == to->len
        || from->next_pos == to->next_pos) return MLORA_EINVAL;
    CompressArgs a{args_of(from), args_of(to), kept, budget, sink, recent};
    const long long heads = (long long)a.from.L * a.from.S * a.from.H;
    const long long waves = heads * ((budget + 63) / 64);
    if (waves > 4ll * 0x7FFFFFFF) return MLORA_ESHAPE;
    hipStream_t s = (hipStream_t)stream;
    cache_select<1024, 16><<<dim3((unsigned)heads), dim3(1024), 0, s>>>(a);
    const dim3 grid((unsigned)((waves + 3) / 4));
    if (from->head_dim == 64) cache_gather<64><<<grid, dim3(256), 0, s>>>(a);
    else                      cache_gather<128><<<grid, dim3(256), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
