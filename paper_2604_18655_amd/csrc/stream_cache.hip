// The streams' own cache segments at a bounded size: rows of a step enter them in the place of the slots with the least
// accumulated attention weight, and the heaviest slots of a long segment are copied into a smaller one.
//
// Both need the K highest-ranked of a head's live slots.  A slot's rank is a 32-bit number that orders like the stated
// rule (protected slots the largest, NaN the smallest), and equal numbers in the order of the slots.  A block finds
// the K-th largest number by histograms of 11, 11 and 10 bits in LDS, then counts slots in their order.
//
// An append reads 8 bytes per live slot and moves few rows: it is bound by its dependent trips to memory (lengths and lists, then masses
// and positions, then the rows) and by the launch.  16 layers x 8 streams x 8 heads of 1024 slots, 3 rows of 30: 6.4 us a
// call.  The few lowest slots of a head are taken wave by wave, without histograms (33 -> 6.4 us together with a line of
// tickets per stream).
//
// A compression into a large cache is bound by its copy: 128 heads of 16384 slots with 128 features to 2048 slots, 268 MB read and written:
// 14.4 us to find the slots, a block per head (dependent passes over 64 KB of ranks in registers), and 52 us to copy them, by
// blocks all over the card (5.2 TB/s).  Up to COPY_ROWS slots a head the block that found them copies them as well (15
// heads of 1003 slots: 7.7 us a call).
#include <algorithm>
#include <type_traits>

#include "common.hpp"

#include "../../include/mlora_stream_cache.h"

namespace mlora {

namespace {

constexpr int BINS = 2048;
constexpr int COPY_ROWS = 512;           // budgets up to which the block that finds a head's slots copies them too

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned rank_of(float mass, int pos, int newest, int sink)
{
    const float m = mass + 0.f;                                      // -0 counts as +0
    const unsigned b = __float_as_uint(m), r = b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
    return pos >= newest || pos < sink ? 0xFFFFFFFFu : m != m ? 0u : r;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp(unsigned old, unsigned v) { return (unsigned)__builtin_amdgcn_update_dpp((int)old, (int)v, CTRL, ROWS, 0xF, false); }
// v combined over this lane and those below it
template <class Op>
__device__ __forceinline__ unsigned scan_wave(unsigned v, unsigned neutral, const Op &op)
{
    v = op(v, dpp<0x111, 0xF>(neutral, v));                          // from one, two, four and eight lanes below in a row of 16,
    v = op(v, dpp<0x112, 0xF>(neutral, v));
    v = op(v, dpp<0x114, 0xF>(neutral, v));
    v = op(v, dpp<0x118, 0xF>(neutral, v));
    v = op(v, dpp<0x142, 0xA>(neutral, v));                          // then from the last lane of the row below,
    return op(v, dpp<0x143, 0xC>(neutral, v));                       // and of the lower half
}
__device__ __forceinline__ unsigned wave_sums(unsigned v) { return scan_wave(v, 0u, [](unsigned x, unsigned y) { return x + y; }); }
__device__ __forceinline__ unsigned last_lane(unsigned v) { return (unsigned)__builtin_amdgcn_readlane((int)v, 63); }
__device__ __forceinline__ unsigned wave_min(unsigned v) { return last_lane(scan_wave(v, ~0u, [](unsigned x, unsigned y) { return min(x, y); })); }
__device__ __forceinline__ unsigned wave_max(unsigned v) { return last_lane(scan_wave(v, 0u, [](unsigned x, unsigned y) { return max(x, y); })); }

// What a head's slots are ranked by.
struct Head {
    const float *mass;
    const int *pos;
    int cap, live;                       // slots
    int newest, sink;                    // protected: pos >= newest or pos < sink
};

// KPT slots per thread of a chunk of THREADS * KPT: four in a row, KPT / 4 times, so that a wave asks for 1 KiB at a time.
template <int THREADS, int KPT>
struct Slots {
    static constexpr int CHUNK = THREADS * KPT;
    float mass[KPT];
    int pos[KPT];
    static __device__ __forceinline__ int slot(int first, int i) { return first + (i / 4) * (THREADS * 4) + (int)threadIdx.x * 4 + i % 4; }
    __device__ __forceinline__ void load(const Head &h, int first)
    {
        typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
        typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
        for (int g = 0; g < KPT; g += 4) {
            const int t = slot(first, g);
            if (t + 3 < h.cap) {
                const f32x4_any m = *reinterpret_cast<const f32x4_any *>(h.mass + t);
                const i32x4_any p = *reinterpret_cast<const i32x4_any *>(h.pos + t);
#pragma unroll
                for (int e = 0; e < 4; ++e) mass[g + e] = m[e], pos[g + e] = p[e];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    mass[g + e] = t + e < h.cap ? h.mass[t + e] : 0.f;
                    pos[g + e] = t + e < h.cap ? h.pos[t + e] : 0;
                }
            }
        }
    }
    // The ranks.  Dead slots have the lowest one, behind live slots with NaN because they are numbered higher.
    __device__ __forceinline__ void ranks(const Head &h, int first, unsigned (&r)[KPT]) const
    {
#pragma unroll
        for (int i = 0; i < KPT; ++i) r[i] = slot(first, i) < h.live ? rank_of(mass[i], pos[i], h.newest, h.sink) : 0u;
    }
};

// sums of W words over the threads before this one, and over all of them
template <int THREADS, int W>
__device__ __forceinline__ void block_scan(unsigned (&v)[W], unsigned (*wave_sum)[W], unsigned (&total)[W])
{
    const int wave = threadIdx.x >> 6;
    unsigned mine[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        mine[i] = v[i];
        v[i] = wave_sums(v[i]);
        if ((threadIdx.x & 63) == 63) wave_sum[wave][i] = v[i];
        total[i] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < W; ++i) {
        unsigned before = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            const unsigned x = wave_sum[w][i];
            before += w < wave ? x : 0u;
            total[i] += x;
        }
        v[i] += before - mine[i];
    }
    __syncthreads();
}

struct Cut {
    unsigned top;                        // ranks whose bits from `shift` on are above this are kept
    int shift;
    int ties;                            // of those equal to it, as many are kept, in the order of the slots
    bool all_ties;                       // they are all there are
};

template <int THREADS>
struct SelectLds {
    int bins[BINS];
    union {
        unsigned wave_sum[THREADS / 64][1];
        unsigned wave_sum2[THREADS / 64][2];
    };
    int found[3];
};
template <int THREADS, int W>
__device__ __forceinline__ unsigned (*sums_of(SelectLds<THREADS> &lds))[W]
{
    if constexpr (W == 1) return lds.wave_sum;
    else return lds.wave_sum2;
}

// The cut that leaves the `keep` highest of the head's live slots, 0 < keep < live.  `held` are the ranks of the only chunk
// (live <= THREADS * KPT), else they are made anew in every pass.
template <int THREADS, int KPT>
__device__ __forceinline__ Cut find_cut(const Head &h, int keep, const unsigned (&held)[KPT], SelectLds<THREADS> &lds)
{
    using Chunk = Slots<THREADS, KPT>;
    const int tid = threadIdx.x, lane = tid & 63;
    constexpr int PER = BINS / THREADS;
    Cut cut{0u, 0, 0, false};
    unsigned prefix = 0;
    int left = keep, shift = 32;
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass < 2 ? 11 : 10, above = shift;
        shift -= bits;
#pragma unroll
        for (int i = 0; i < PER; ++i) lds.bins[i * THREADS + tid] = 0;
        __syncthreads();
        for (int c0 = 0; c0 < h.live; c0 += Chunk::CHUNK) {
            unsigned r[KPT];
            if (h.live > Chunk::CHUNK) {
                Chunk now;
                now.load(h, c0);
                now.ranks(h, c0, r);
            } else {
#pragma unroll
                for (int i = 0; i < KPT; ++i) r[i] = held[i];
            }
            // equal ranks all over the wave (masses that are all zero) are counted at once; rank 0 (dead slots) is not
            // counted: what no other bin holds is in the last
            const unsigned one = __builtin_amdgcn_readfirstlane(r[0]);
            unsigned differ = 0;
#pragma unroll
            for (int i = 0; i < KPT; ++i) differ |= r[i] ^ one;
            if (!__any(differ != 0)) {
                if (lane == 0 && one && (pass == 0 || one >> (above & 31) == prefix)) atomicAdd(&lds.bins[one >> shift & ((1u << bits) - 1)], 64 * KPT);
                continue;
            }
            if (pass == 0) {
#pragma unroll
                for (int i = 0; i < KPT; ++i)
                    if (r[i]) atomicAdd(&lds.bins[r[i] >> 21], 1);
            } else {
#pragma unroll
                for (int i = 0; i < KPT; ++i)
                    if (r[i] >> above == prefix && r[i]) atomicAdd(&lds.bins[r[i] >> shift & ((1u << bits) - 1)], 1);
            }
        }
        __syncthreads();
        // the bin that holds the left-th largest: thread t looks at PER bins, counted from the top
        int n[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            n[i] = lds.bins[BINS - 1 - (tid * PER + i)];
            sum += n[i];
        }
        unsigned scan[1] = {(unsigned)sum}, total[1];
        block_scan<THREADS, 1>(scan, lds.wave_sum, total);
        int before = (int)scan[0];
        const bool in_last = left > (int)total[0];                   // (bin 0, where it holds rank 0)
        if (before < left && left <= before + sum) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                if (before < left && left <= before + n[i]) {
                    lds.found[0] = BINS - 1 - (tid * PER + i);
                    lds.found[1] = before;
                    lds.found[2] = n[i];
                }
                before += n[i];
            }
        }
        __syncthreads();
        if (in_last) {
            left -= (int)total[0];
            return Cut{0u, 0, left, false};                          // rank 0 itself
        }
        const int bin = lds.found[0], in_bin = lds.found[2];
        left -= lds.found[1];
        prefix = prefix << bits | (unsigned)bin;
        // (a bin 0 of the prefix 0 holds rank 0 too, uncounted)
        cut = Cut{prefix, shift, left, left == in_bin && prefix != 0};
        if (cut.all_ties) break;                                     // no finer cut is needed
    }
    return cut;
}

// Calls use(slot, number) for every live slot that is kept (KEPT) or that is not, numbered in the order of the slots.
template <int THREADS, int KPT, bool KEPT, class Use>
__device__ __forceinline__ void in_order(const Head &h, const Cut &cut, const unsigned (&held)[KPT], SelectLds<THREADS> &lds, const Use &use)
{
    using Chunk = Slots<THREADS, KPT>;
    static_assert(KPT <= 16 && THREADS <= 1024, "a field of 16 bits per four slots of a thread");
    constexpr int W = KPT > 8 ? 2 : 1;
    int ties = 0, count = 0;
    for (int c0 = 0; c0 < h.live; c0 += Chunk::CHUNK) {
        unsigned r[KPT];
        if (h.live > Chunk::CHUNK) {
            Chunk now;
            now.load(h, c0);
            now.ranks(h, c0, r);
        } else {
#pragma unroll
            for (int i = 0; i < KPT; ++i) r[i] = held[i];
        }
        // a bit per slot above the cut, and per slot at it
        unsigned wanted = 0, equal = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const unsigned x = r[i] >> cut.shift;
            wanted |= x > cut.top ? 1u << i : 0u;
            equal |= x == cut.top ? 1u << i : 0u;
        }
        if (cut.all_ties) {
            wanted |= equal;
        } else {
            // counts of each run of four slots, 16 bits each: of a run, the lower threads come first
            unsigned n[W] = {}, all[W];
#pragma unroll
            for (int g = 0; g < KPT; g += 4) n[g / 8] += (unsigned)__popc(equal >> g & 15u) << (g / 4 % 2 * 16);
            block_scan<THREADS, W>(n, sums_of<THREADS, W>(lds), all);
#pragma unroll
            for (int g = 0; g < KPT; g += 4) {
                int tie = ties + (int)(n[g / 8] >> (g / 4 % 2 * 16) & 0xFFFF);
#pragma unroll
                for (int i = g; i < g + 4; ++i) {
                    const bool is = equal >> i & 1;
                    wanted |= is && tie < cut.ties ? 1u << i : 0u;
                    tie += is;
                }
                ties += (int)(all[g / 8] >> (g / 4 % 2 * 16) & 0xFFFF);
            }
        }
        if (!KEPT) {
#pragma unroll
            for (int i = 0; i < KPT; ++i) wanted ^= Chunk::slot(c0, i) < h.live ? 1u << i : 0u;
        }
        unsigned n[W] = {}, all[W];
#pragma unroll
        for (int g = 0; g < KPT; g += 4) n[g / 8] += (unsigned)__popc(wanted >> g & 15u) << (g / 4 % 2 * 16);
        block_scan<THREADS, W>(n, sums_of<THREADS, W>(lds), all);
#pragma unroll
        for (int g = 0; g < KPT; g += 4) {
            int at = count + (int)(n[g / 8] >> (g / 4 % 2 * 16) & 0xFFFF);
#pragma unroll
            for (int i = g; i < g + 4; ++i)
                if (wanted >> i & 1) use(Chunk::slot(c0, i), at++);
            count += (int)(all[g / 8] >> (g / 4 % 2 * 16) & 0xFFFF);
        }
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

// The `out` slots of the lowest rank in the order of the slots, for out * waves <= 64: every wave takes its lowest one after
// the other, then all waves' candidates, one per lane, are counted against each other.
template <int THREADS, int KPT>
__device__ __forceinline__ void lowest_few(const Head &h, int out, const unsigned (&rank)[KPT], unsigned (*candidate)[64], int *taken)
{
    unsigned live = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) live |= Slots<THREADS, KPT>::slot(0, i) < h.live ? 1u << i : 0u;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned *const ranks = candidate[0], *const slots = candidate[1];          // slot + 1; 0: none
    for (int n = 0; n < out; ++n) {
        unsigned low = ~0u, at = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            const bool lower = (live >> i & 1) && rank[i] <= low;               // among equals the higher slot goes first
            low = lower ? rank[i] : low;
            at = lower ? i + 1 : at;
        }
        const unsigned least = wave_min(low);
        const unsigned slot = at && low == least ? (unsigned)Slots<THREADS, KPT>::slot(0, (int)at - 1) + 1 : 0u, last = wave_max(slot);
        if (slot == last && slot) live &= ~(1u << (at - 1));
        if (lane == 0) ranks[wave * out + n] = least, slots[wave * out + n] = last;
    }
    __syncthreads();
    if (wave == 0) {
        const int all = out * (THREADS / 64);
        const unsigned r = lane < all ? ranks[lane] : ~0u, t = lane < all ? slots[lane] : 0u;
        int before = 0;
        for (int c = 0; c < all; ++c) {
            const unsigned rc = (unsigned)__builtin_amdgcn_readlane((int)r, c), tc = (unsigned)__builtin_amdgcn_readlane((int)t, c);
            before += rc < r || (rc == r && tc > t);
        }
        const bool goes = t && before < out;
        int number = 0;
        for (unsigned long long m = __ballot(goes); m; m &= m - 1) number += (unsigned)__builtin_amdgcn_readlane((int)t, __ffsll(m) - 1) < t;
        if (goes) taken[number] = (int)t - 1;
    }
}

// A block per layer, stream and head.
template <int THREADS, int KPT, int D>
__global__ __launch_bounds__(THREADS) void cache_append(const AppendArgs a)
{
    __shared__ SelectLds<THREADS> lds;
    extern __shared__ int taken[];                                   // slots that give way
    using Chunk = Slots<THREADS, KPT>;
    const int tid = threadIdx.x, H = a.c.H, S = a.c.S, cap = a.c.cap;
    const int head = blockIdx.x, l = head / (S * H), s = head / H % S, h = head % H;
    const size_t slots = (size_t)head * cap;
    Head hd{a.c.mass + slots, a.c.slot_pos + slots, cap, 0, 0, a.sink};
    Chunk first;                                                     // asked for before it is known whether a slot gives way
    first.load(hd, 0);
    const int *const rows = a.rows ? a.rows + (size_t)s * a.n_rows : nullptr;
    const int live = max(0, min(a.c.len[s], cap)), next = a.c.next_pos[s];
    const int n = listed(rows, a.n_rows, a.R);
    const int room = min(n, max(live, a.budget) - live), out = n - room;
    constexpr int PIECES = D / 8;                                    // of 16 bytes in a row
    const auto source = [&](int i) {
        const int j = i / (2 * PIECES), piece = i % PIECES, value = i / PIECES % 2;
        const size_t from = (((size_t)l * S + s) * a.R + (rows ? rows[j] : j)) * H + h;
        return *(reinterpret_cast<const u32x4 *>((value ? a.v_new : a.k_new) + from * D) + piece);
    };
    u32x4 ahead = {0, 0, 0, 0};
    if (tid < n * 2 * PIECES) ahead = source(tid);
    if (out > 0) {
        hd.live = live;
        hd.newest = next - a.recent;
        unsigned held[KPT];
        first.ranks(hd, 0, held);
        if (out * (THREADS / 64) <= 64 && live <= Chunk::CHUNK) {
            lowest_few<THREADS, KPT>(hd, out, held, reinterpret_cast<unsigned (*)[64]>(lds.bins), taken);
        } else {
            Cut cut{0xFFFFFFFFu, 0, 0, false};                       // (all give way: ranks equal to it are ties beyond the count)
            if (out < live) cut = find_cut<THREADS, KPT>(hd, live - out, held, lds);
            in_order<THREADS, KPT, false>(hd, cut, held, lds, [&](int slot, int number) { taken[number] = slot; });
        }
        __syncthreads();
    }
    for (int i = tid; i < n * 2 * PIECES; i += THREADS) {
        const int j = i / (2 * PIECES), piece = i % PIECES, value = i / PIECES % 2;
        const int slot = j < room ? live + j : taken[j - room];
        reinterpret_cast<u32x4 *>((value ? a.c.v : a.c.k) + (slots + slot) * D)[piece] = i == tid ? ahead : source(i);
        if (piece == 0) {
            if (value) a.c.slot_pos[slots + slot] = next + j;
            else       a.c.mass[slots + slot] = 0.f;
        }
    }
    // The stream's last block moves its length on: all others have read it (a ticket is drawn behind the barrier; nothing that a
    // block has written is handed over, so no fence: with one, and all streams' tickets in one line, 16 layers x 8
    // streams x 8 heads took 27 us.)
    __syncthreads();
    if (tid == 0) {
        const unsigned last = (unsigned)(a.c.L * H) - 1;
        if (atomicInc(a.c.tickets + (size_t)s * MLORA_CACHE_TICKET_WORDS, last) == last) {
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

// One head's slots, all of them found: AT_ONCE rows of keys and of values side by side, AHEAD times.  from_slot(j) is the slot of
// row j, the same for all lanes of a row; j counts from the first row of `to`.
// PAST: read past the caches.  (Written past them, the call takes as long, and the attention that reads the copies next longer: 16
// layers' compression and attention 250 us instead of 238.)
template <int D, int LANES, bool PAST, class From>
__device__ __forceinline__ void copy_rows(const CompressArgs &a, size_t from, size_t to, int rows, int lane, const From &from_slot)
{
    constexpr int PIECES = D / 8, AT_ONCE = LANES / PIECES, AHEAD = 4;
    const int piece = lane % PIECES, row = lane / PIECES;
    const u32x4 *const ks = reinterpret_cast<const u32x4 *>(a.from.k + from * D) + piece, *const vs = reinterpret_cast<const u32x4 *>(a.from.v + from * D) + piece;
    u32x4 *const kt = reinterpret_cast<u32x4 *>(a.to.k + to * D) + piece, *const vt = reinterpret_cast<u32x4 *>(a.to.v + to * D) + piece;
    for (int j0 = 0; j0 < rows; j0 += AT_ONCE * AHEAD) {
        u32x4 kv[AHEAD], vv[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int j = j0 + u * AT_ONCE + row, src = from_slot(j);
            const u32x4 *const kp = ks + (size_t)src * PIECES, *const vp = vs + (size_t)src * PIECES;
            if (j < rows) kv[u] = PAST ? __builtin_nontemporal_load(kp) : *kp, vv[u] = PAST ? __builtin_nontemporal_load(vp) : *vp;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int j = j0 + u * AT_ONCE + row;
            if (j >= rows) continue;
            kt[(size_t)j * PIECES] = kv[u], vt[(size_t)j * PIECES] = vv[u];
        }
    }
}

// A block per layer, stream and head finds its slots.  D: and copies them, up to ROWS.
template <int THREADS, int KPT, int D>
__global__ __launch_bounds__(THREADS) void cache_select(const CompressArgs a)
{
    __shared__ SelectLds<THREADS> lds;
    __shared__ int slot_of[D ? COPY_ROWS : 1];
    const int tid = threadIdx.x, H = a.from.H, S = a.from.S;
    const int head = blockIdx.x, s = head / H % S;
    const size_t slots = (size_t)head * a.from.cap;
    Head hd{a.from.mass + slots, a.from.slot_pos + slots, a.from.cap, 0, 0, a.sink};
    Slots<THREADS, KPT> first;
    first.load(hd, 0);
    const int live = max(0, min(a.from.len[s], a.from.cap)), next = a.from.next_pos[s], keep = min(live, a.budget);
    int *const kept = a.kept + (size_t)head * a.budget;
    const auto put = [&](int slot, int number) {
        kept[number] = slot;
        if constexpr (D != 0) slot_of[number] = slot;
    };
    if (keep < live) {
        hd.live = live;
        hd.newest = next - a.recent;
        unsigned held[KPT];
        first.ranks(hd, 0, held);
        const Cut cut = find_cut<THREADS, KPT>(hd, keep, held, lds);
        in_order<THREADS, KPT, true>(hd, cut, held, lds, put);
    } else {
        for (int i = tid; i < keep; i += THREADS) put(i, i);
    }
    for (int i = keep + tid; i < a.budget; i += THREADS) kept[i] = -1;
    if (tid == 0 && head == s * H) {
        a.to.len[s] = keep;
        a.to.next_pos[s] = next;
    }
    if constexpr (D != 0) {
        __syncthreads();
        const size_t to = (size_t)head * a.to.cap;
        for (int i = tid; i < keep; i += THREADS) {
            a.to.mass[to + i] = hd.mass[slot_of[i]];
            a.to.slot_pos[to + i] = hd.pos[slot_of[i]];
        }
        copy_rows<D, THREADS, false>(a, slots, to, keep, tid, [&](int j) { return slot_of[min(j, keep - 1)]; });
    }
}

// A wave copies 64 slots of a head.
template <int D, bool PAST>
__global__ __launch_bounds__(256) void cache_gather(const CompressArgs a)
{
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
    copy_rows<D, 64, PAST>(a, from, to, __popcll(__ballot(slot >= 0)), lane, [&](int j) { return __shfl(slot, j); });
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
    // slots per thread: as few as hold a head (larger caches go over them in chunks)
    const auto go = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        if (c->cap <= 1024)      cache_append<256, 4, D><<<grid, dim3(256), taken, s>>>(a);
        else if (c->cap <= 2048) cache_append<256, 8, D><<<grid, dim3(256), taken, s>>>(a);
        else                     cache_append<256, 16, D><<<grid, dim3(256), taken, s>>>(a);
    };
    if (c->head_dim == 64) go(std::integral_constant<int, 64>{});
    else                   go(std::integral_constant<int, 128>{});
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
    const dim3 grid((unsigned)heads), gather((unsigned)((waves + 3) / 4));
    const auto select = [&](auto dim) {
        constexpr int D = decltype(dim)::value;
        if (from->cap <= 1024)      cache_select<256, 4, D><<<grid, dim3(256), 0, s>>>(a);
        else if (from->cap <= 4096) cache_select<1024, 4, D><<<grid, dim3(1024), 0, s>>>(a);
        else                        cache_select<1024, 16, D><<<grid, dim3(1024), 0, s>>>(a);
    };
    if (budget > COPY_ROWS) {
        select(std::integral_constant<int, 0>{});
        // From 128 MB read and copied on, half of the memory-side cache, what is read goes past the caches, which leaves them to the
        // copies: 128 heads of 16384 slots with 128 features to 2048, 268 MB, 75 -> 66 us, with a reader of the copies 140 -> 128;
        // 96 heads 62 -> 51 and 109 -> 97; 64 heads, 134 MB, 46 to 40 -> 40; to 700 of 8192, 92 MB, 31 -> 33.
        const bool past = (double)heads * budget * from->head_dim * 8 >= (double)(128 << 20);
        if (from->head_dim == 64) past ? cache_gather<64, true><<<gather, dim3(256), 0, s>>>(a) : cache_gather<64, false><<<gather, dim3(256), 0, s>>>(a);
        else                      past ? cache_gather<128, true><<<gather, dim3(256), 0, s>>>(a) : cache_gather<128, false><<<gather, dim3(256), 0, s>>>(a);
    } else {
        if (from->head_dim == 64) select(std::integral_constant<int, 64>{});
        else                      select(std::integral_constant<int, 128>{});
    }
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
