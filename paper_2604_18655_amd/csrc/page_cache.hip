// A paged cache of keys and values in 8 bits (see include/mlora_page_cache.h): rows that enter it, streams that become others, copies
// into another cache.
//
// A call of some hundred streams or fewer is one launch: every block works out what it needs of the bookkeeping (which pages, which slots) by itself,
// moves its share of the data, and the last block to have read the cache's lists writes them anew.  Who is the last is found by counters that wrap,
// a line of memory per stream and one above them.  Larger calls, and prompts, are two launches: a block for the bookkeeping, which leaves what the
// others need in the cache's own words, and blocks that move the data.  (Two launches for a step's calls, too, was: 8 beams of 16 layers reordered
// in 7.9 us, now 5.0, 64 streams with a window in 8.0, now 5.2.)
#include <algorithm>
#include <type_traits>

#include "common.hpp"

#include "../../include/mlora_page_cache.h"

namespace mlora {

namespace {

constexpr int P = MLORA_PAGE_TOKENS;
constexpr int CTRL = 1024;                               // threads of a bookkeeping block; at least MLORA_PAGE_MAX_STREAMS
constexpr int ONE = 256;                                 // of a block of a call that is one launch; its streams at most
static_assert(CTRL >= MLORA_PAGE_MAX_STREAMS, "a thread per stream");

// the cache's own words: where the search for free pages starts (no page below is free), then what a call's two launches hand over
constexpr int FAR = 32;                                  // pages per thread that are looked over at once where none is free
constexpr int OWN_LOW = 0, OWN_COUNT = 1, OWN_TICKETS = 64, TICKET_WORDS = 32;
__host__ __device__ constexpr int own_plan(int streams) { return OWN_TICKETS + TICKET_WORDS * (streams + 1); }
struct Plan {
    int first, count, slot, other;
};
constexpr int PLAN_WORDS = 4;

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

struct CacheArgs {
    int8_t *k, *v;
    float *k_scale, *v_scale;
    uint16_t *k_tail, *v_tail;
    int *slot, *len, *table, *refs, *own;
    int L, S, H, D, pages, columns;
};

__device__ __forceinline__ int slot_of(const CacheArgs &c, int s) { return min(max(c.slot[s], 0), c.S - 1); }
__device__ __forceinline__ int len_of(const CacheArgs &c, int s) { return min(max(c.len[s], 0), P * c.columns + P - 1); }
__device__ __forceinline__ Plan *plans(const CacheArgs &c) { return reinterpret_cast<Plan *>(c.own + own_plan(c.S)); }

// Sums over the threads before this one, and over all of them.  One __syncthreads before `part` is used again is the caller's.
struct Sums {
    int before, all;
};
template <int T>
__device__ __forceinline__ Sums sums_of(int x, int (&part)[T / 64])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int run = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int y = __shfl_up(run, d);
        run += lane >= d ? y : 0;
    }
    if (lane == 63) part[wave] = run;
    __syncthreads();
    int base = 0, all = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) {
        const int y = part[w];
        base += w < wave ? y : 0;
        all += y;
    }
    return Sums{base + run - x, all};
}

// Thread 0 of a block that has read the lists draws a ticket; true for the last of all (blocks_per_stream) * S blocks.  The counters are zero again then.
__device__ __forceinline__ bool last_to_read(const CacheArgs &c, int s, unsigned blocks_per_stream)
{
    unsigned *const tickets = reinterpret_cast<unsigned *>(c.own + OWN_TICKETS);
    if (atomicInc(tickets + TICKET_WORDS * (s + 1), blocks_per_stream - 1) != blocks_per_stream - 1) return false;
    return atomicInc(tickets, (unsigned)c.S - 1) == (unsigned)c.S - 1;
}

// The last of n ascending numbers, the first of them 0, that is at most i.
__device__ __forceinline__ int last_from(const int *start, int n, int i)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (start[mid] <= i) lo = mid;
        else                 hi = mid;
    }
    return lo;
}

// ---------------------------------------------------------------------------------------------- append

struct AppendArgs {
    CacheArgs c;
    const uint16_t *k_new, *v_new;
    const int *rows;
    int *appended;
    int R, n_rows;
};

// pages that one call can fill: (S * 63 + S * R) / 64
template <int T> constexpr int MOST_FILLED = MLORA_MAX_ROWS / P + T;

template <int T>
struct AppendLds {
    int count[T], start[T], place[T], part[T / 64], list[MOST_FILLED<T>], last;
};
// Who enters, and which pages fill: those of stream s are list[start[s]] and on.  The result is the stream's of the thread's number; `used`: all pages.
struct Entry {
    int len, slot, n, used, low;
};
template <int T>
__device__ __forceinline__ Entry append_plan_of(const AppendArgs &a, AppendLds<T> &lds)
{
    const CacheArgs &c = a.c;
    const int tid = threadIdx.x;
    lds.count[tid] = a.n_rows;
    if (tid == 0) lds.last = 0;
    const int low = min(max(c.own[OWN_LOW], 0), c.pages) & ~3;
    int len = 0, slot = 0, n = 0, wish = 0;
    if (tid < c.S) {
        len = len_of(c, tid);
        slot = slot_of(c, tid);
    }
    __syncthreads();
    if (a.rows)
        for (int i = tid; i < c.S * a.n_rows; i += T) {
            const int r = a.rows[i], s = i / a.n_rows;
            if (r < 0 || r >= a.R) atomicMin(&lds.count[s], i - s * a.n_rows);
        }
    __syncthreads();
    if (tid < c.S) {
        n = lds.count[tid];
        wish = (len % P + n) / P;
        if (len / P + wish > c.columns) n = wish = 0;
    }
    const Sums want = sums_of<T>(wish, lds.part);
    lds.start[tid] = want.before;
    lds.place[tid] = len / P;
    // the lowest free pages, as many as are wanted
    int found = 0;
    for (int p0 = low; found < want.all && p0 < c.pages; p0 += 4 * T) {
        int refs[4], some = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int p = p0 + 4 * tid + u;
            refs[u] = p < c.pages ? c.refs[p] : 1;
            some += refs[u] <= 0;
        }
        __syncthreads();
        const Sums at = sums_of<T>(some, lds.part);
        int number = found + at.before;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (refs[u] <= 0) {
                if (number < want.all) lds.list[number] = p0 + 4 * tid + u;
                ++number;
            }
        found += at.all;
        // In pools that are nearly full, whole stretches without a free page are passed over (none free of 250000: 400 -> 56 us).
        for (bool none = at.all == 0; none && p0 + 4 * T < c.pages;) {
            int least = 1;                               // (behind the end the last page again, which lies in the stretch)
#pragma unroll
            for (int u = 0; u < FAR; ++u) least = min(least, c.refs[min(p0 + 4 * T + u * T + tid, c.pages - 1)]);
            __syncthreads();
            none = sums_of<T>(least <= 0, lds.part).all == 0;
            if (none) p0 += FAR * T;
        }
    }
    found = min(found, want.all);
    const bool enters = wish == 0 || want.before + wish <= found;
    if (!enters) n = 0;
    else if (wish > 0) atomicMax(&lds.last, want.before + wish);
    __syncthreads();
    const int used = lds.last;                           // (streams that do not enter stand behind all that fill pages)
    // Where the next search starts: at the first page that was found and not taken; behind all pages, if more were wanted than are free; else behind the last one
    // taken.  (None free of 250000, asked for again: 56 -> 5 us.)
    const int next = want.all == 0 ? -1 : used < found ? lds.list[used] : found < want.all ? c.pages : lds.list[used - 1] + 1;
    return Entry{len, slot, n, used, next};
}
// and what is to be written of it
template <int T>
__device__ __forceinline__ void append_commit(const AppendArgs &a, const AppendLds<T> &lds, const Entry &e)
{
    const CacheArgs &c = a.c;
    const int tid = threadIdx.x;
    for (int i = tid; i < e.used; i += T) {
        const int s = last_from(lds.start, c.S, i);
        c.table[(size_t)slot_of(c, s) * c.columns + lds.place[s] + (i - lds.start[s])] = lds.list[i];
        c.refs[lds.list[i]] = 1;
    }
    if (tid < c.S) {
        c.len[tid] = e.len + e.n;
        if (a.appended) a.appended[tid] = e.n;
    }
    if (tid == 0 && e.low >= 0) c.own[OWN_LOW] = e.low;
}

__global__ __launch_bounds__(CTRL) void append_plan(const AppendArgs a)
{
    __shared__ AppendLds<CTRL> lds;
    const Entry e = append_plan_of<CTRL>(a, lds);
    append_commit<CTRL>(a, lds, e);
    if ((int)threadIdx.x < a.c.S) plans(a.c)[threadIdx.x] = Plan{e.len, e.n, e.slot, 0};
}

// A page's 64 x D numbers to codes and a scale: the largest magnitude, as the bits of a bf16 number (which order like it)
__device__ __forceinline__ unsigned top_bits(const u32x4 &x, unsigned top)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(x[i] & 0x7FFFu, x[i] >> 16 & 0x7FFFu));
    return top;
}
// Codes of 8 numbers.  All are moved by the power of two that brings `top` into [1/2, 1), since 127 x may not be a number.  127 x / top is a quotient of
// numbers of 15 and 8 bits: it is a half, which one correction of the product with the reciprocal gives exactly, or further from one than
// 2^-17, and the codes are those of the exact quotient.  1.5 * 2^23 added rounds to whole numbers; the low byte of the sum's bits is the code.
struct Divide {
    float top, inverse, by, more;                        // x is multiplied by `by`, and by `more` where that is not 1 (top below 2^-100)
};
__device__ __forceinline__ Divide divide_by(unsigned bits)
{
    const float top = bf16_bits_to_float(bits);
    const int e = __builtin_amdgcn_frexp_expf(top);
    const float t = __builtin_ldexpf(top, -e);
    return Divide{t, __builtin_amdgcn_rcpf(t), __builtin_ldexpf(127.f, min(-e, 100)), __builtin_ldexpf(1.f, max(-e - 100, 0))};
}
__device__ __forceinline__ u32x2 codes_of(const u32x4 &x, const Divide &d)
{
    unsigned n[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float f = (i & 1 ? __uint_as_float(x[i / 2] & 0xFFFF0000u) : bf16_bits_to_float(x[i / 2])) * d.by;
        if (d.more != 1.f) f *= d.more;
        const float near = f * d.inverse, quotient = __builtin_fmaf(__builtin_fmaf(-near, d.top, f), d.inverse, near);
        n[i] = __float_as_uint(quotient + 12582912.f);
    }
    u32x2 out;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        out[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(n[4 * i + 3], n[4 * i + 2], 0x0C0C0400u), __builtin_amdgcn_perm(n[4 * i + 1], n[4 * i], 0x0C0C0400u), 0x05040100u);
    return out;
}

// A prompt of 4096 rows of 8 heads of 128 features, 25 MB read and written: 7.2 to 8.9 us, a launch and three dependent trips among it (values turned
// byte by byte and divided by the hardware's steps: 10.9).
//
// The rows of a layer, stream and head: they fill its j-th page, `page` of the pool; with the first one the tail is written as well, behind the page that
// takes what was there.
template <int D>
struct PageLds {
    __align__(16) unsigned char turned[D * P];           // [feature][token], groups of 16 tokens in another order in each run of 8 features
    unsigned tops[2][4];
};
template <int D>
__device__ __forceinline__ void append_head(const AppendArgs &a, PageLds<D> &lds, const Plan &plan, int page, int l, int s, int h, int j)
{
    constexpr int PIECES = D / 8, NP = P * PIECES / 256;         // a thread has 8 features of NP tokens in a row
    auto &turned = lds.turned;
    auto &tops = lds.tops;
    const CacheArgs &c = a.c;
    const int tid = threadIdx.x;
    const int t = plan.first % P, filled = (t + plan.count) / P;
    const size_t tail = (((size_t)l * c.S + plan.slot) * c.H + h) * P * D, stream = ((size_t)l * c.S + s) * a.R;
    // token g of those behind the full pages (in the tail up to t), 8 of its features from f on
    const auto from = [&](int g) {
        const int i = min(g - t, plan.count - 1), row = a.rows ? a.rows[s * a.n_rows + i] : i;
        return ((stream + row) * c.H + h) * D;
    };
    if (j < filled) {
        const int f = tid % PIECES * 8, t0 = tid / PIECES * NP;
        u32x4 kx[NP], vx[NP];
        unsigned kt = 0, vt = 0;
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            const int g = j * P + t0 + u;
            const size_t at = g < t ? tail + (size_t)g * D + f : from(g) + f;
            kx[u] = *reinterpret_cast<const u32x4 *>((g < t ? c.k_tail : a.k_new) + at);
            vx[u] = *reinterpret_cast<const u32x4 *>((g < t ? c.v_tail : a.v_new) + at);
        }
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            kt = top_bits(kx[u], kt);
            vt = top_bits(vx[u], vt);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            kt = max(kt, (unsigned)__shfl_xor((int)kt, d));
            vt = max(vt, (unsigned)__shfl_xor((int)vt, d));
        }
        if ((tid & 63) == 0) tops[0][tid >> 6] = kt, tops[1][tid >> 6] = vt;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) kt = max(kt, tops[0][w]), vt = max(vt, tops[1][w]);
        const size_t unit = ((size_t)l * c.pages + page) * c.H + h;
        const bool k_ok = kt > 0 && kt < 0x7F80u, v_ok = vt > 0 && vt < 0x7F80u;
        const Divide k_by = divide_by(k_ok ? kt : 0x3F80u), v_by = divide_by(v_ok ? vt : 0x3F80u);
        u32x2 v[NP];
#pragma unroll
        for (int u = 0; u < NP; ++u) {
            *reinterpret_cast<u32x2 *>(c.k + (unit * P + t0 + u) * D + f) = k_ok ? codes_of(kx[u], k_by) : u32x2{0, 0};
            v[u] = v_ok ? codes_of(vx[u], v_by) : u32x2{0, 0};
        }
        // values feature by feature: the thread's tokens of a feature are NP bytes in a row
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            unsigned word = 0;
#pragma unroll
            for (int u = 0; u < NP; ++u) word |= (v[u][e / 4] >> 8 * (e % 4) & 0xFFu) << 8 * u;
            unsigned char *const to = turned + (f + e) * P + (t0 ^ (f / 8 & 3) * 16);
            if constexpr (NP == 4) *reinterpret_cast<unsigned *>(to) = word;
            else                   *reinterpret_cast<unsigned short *>(to) = (unsigned short)word;
        }
        if (tid == 0) {
            c.k_scale[unit] = kt < 0x7F80u ? bf16_bits_to_float(kt) / 127.f : __builtin_nanf("");
            c.v_scale[unit] = vt < 0x7F80u ? bf16_bits_to_float(vt) / 127.f : __builtin_nanf("");
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < D * P / 16 / 256; ++u) {
            const int i = u * 256 + tid, feature = i / 4, group = i % 4 ^ (feature / 8 & 3);
            *reinterpret_cast<u32x4 *>(c.v + unit * P * D + 16 * i) = *reinterpret_cast<const u32x4 *>(turned + feature * P + group * 16);
        }
    }
    if (j == 0) {
        // (everybody has read the old tail: the first barrier above)
        const int first = filled ? filled * P : t, n = t + plan.count - first;
        for (int piece = tid; piece < n * PIECES; piece += 256) {
            const int g = first + piece / PIECES, f = piece % PIECES * 8;
            const size_t at = from(g) + f, to = tail + (size_t)(g % P) * D + f;
            *reinterpret_cast<u32x4 *>(c.k_tail + to) = *reinterpret_cast<const u32x4 *>(a.k_new + at);
            *reinterpret_cast<u32x4 *>(c.v_tail + to) = *reinterpret_cast<const u32x4 *>(a.v_new + at);
        }
    }
}

// Block y of a layer, stream and head takes its y-th page.
template <int D>
__global__ __launch_bounds__(256) void append_rows(const AppendArgs a)
{
    __shared__ PageLds<D> lds;
    const CacheArgs &c = a.c;
    const int head = blockIdx.x, s = head / c.H % c.S, l = head / (c.H * c.S), h = head - (l * c.S + s) * c.H, j = blockIdx.y;
    const Plan plan = plans(c)[s];
    if (plan.first % P + plan.count < j * P) return;
    const int at = plan.first / P + j, page = at < c.columns ? min(max(c.table[(size_t)plan.slot * c.columns + at], 0), c.pages - 1) : 0;
    append_head<D>(a, lds, plan, page, l, s, h, j);
}

// A call of at most 64 rows per stream: a block per stream, layer and head, the stream fastest.
template <int D>
__global__ __launch_bounds__(ONE) void append_step(const AppendArgs a)
{
    __shared__ union Lds {
        AppendLds<ONE> plan;
        PageLds<D> page;
    } lds;
    __shared__ Plan mine;
    __shared__ int my_page, is_last;
    const CacheArgs &c = a.c;
    const int tid = threadIdx.x, s = (int)blockIdx.x % c.S, unit = (int)blockIdx.x / c.S, l = unit / c.H, h = unit - l * c.H;
    // its own rows; who else enters only where they fill a page
    if (tid < 64) {
        const int r = tid < a.n_rows ? (a.rows ? a.rows[s * a.n_rows + tid] : tid) : -1;
        const unsigned long long bad = __ballot(r < 0 || r >= a.R);
        const int n = bad ? __builtin_ctzll(bad) : 64;
        if (tid == 0) mine = Plan{len_of(c, s), n, slot_of(c, s), 0};
    }
    __syncthreads();
    Plan plan = mine;
    int page = 0;
    if (plan.first % P + plan.count >= P) {
        const Entry e = append_plan_of<ONE>(a, lds.plan);
        if (tid == s) {
            mine.count = e.n;
            my_page = e.n > 0 ? lds.plan.list[lds.plan.start[s]] : 0;
        }
        __syncthreads();
        plan = mine;
        page = my_page;
    }
    if (tid == 0) is_last = last_to_read(c, s, (unsigned)(c.L * c.H));
    __syncthreads();
    append_head<D>(a, lds.page, plan, page, l, s, h, 0);
    if (!is_last) return;
    __syncthreads();
    const Entry e = append_plan_of<ONE>(a, lds.plan);
    append_commit<ONE>(a, lds.plan, e);
}

// ---------------------------------------------------------------------------------------------- reorder

struct ReorderArgs {
    CacheArgs c;
    const int *source;
    int window, sink;
};

// Slots and lengths.  A stream's plan: its new length, whether its data moves (2: from a slot, 1: it becomes empty, 0: it stays), the slots
// to and from; and the tokens that its new slot held before.
template <int T>
struct ReorderLds {
    int first[T], taken[T], place[T], slot[T], len[T], held[T], part[T / 64];
};
struct Move {
    Plan plan;
    int held;
};
template <int T>
__device__ __forceinline__ Move reorder_plan_of(const ReorderArgs &a, ReorderLds<T> &lds)
{
    const CacheArgs &c = a.c;
    const int tid = threadIdx.x, S = c.S;
    lds.first[tid] = T;
    lds.taken[tid] = 0;
    lds.held[tid] = 0;
    int from = -1, was = 0, at = 0;
    if (tid < S) {
        from = a.source ? a.source[tid] : tid;
        was = len_of(c, tid);
        at = slot_of(c, tid);
        if (from < 0 || from >= S) from = -1;
        lds.slot[tid] = at;
        lds.len[tid] = was;
    }
    __syncthreads();
    if (tid < S) lds.held[at] = was;
    if (from >= 0) atomicMin(&lds.first[from], tid);
    __syncthreads();
    const int slot = from >= 0 ? lds.slot[from] : 0, len = from >= 0 ? lds.len[from] : 0;
    const bool keeps = from >= 0 && lds.first[from] == tid;
    if (keeps) lds.taken[slot] = 1;
    __syncthreads();
    // free slots and streams that look for one, both counted at once
    const bool open = tid < S && !lds.taken[tid], looks = tid < S && !keeps;
    const int before = sums_of<T>((int)open + ((int)looks << 16), lds.part).before;
    if (open) lds.place[before & 0xFFFF] = tid;
    __syncthreads();
    if (tid >= S) return Move{};
    const int to = keeps ? slot : lds.place[before >> 16];
    return Move{Plan{len, keeps ? 0 : from >= 0 ? 2 : 1, to, slot}, lds.held[to]};
}

__global__ __launch_bounds__(CTRL) void reorder_plan(const ReorderArgs a)
{
    __shared__ ReorderLds<CTRL> lds;
    const CacheArgs &c = a.c;
    const Move m = reorder_plan_of<CTRL>(a, lds);
    __syncthreads();                                     // (everybody has read slot and len)
    if ((int)threadIdx.x < c.S) {
        c.slot[threadIdx.x] = m.plan.slot;
        c.len[threadIdx.x] = m.plan.first;
        plans(c)[threadIdx.x] = m.plan;
        c.own[own_plan(c.S) + PLAN_WORDS * c.S + threadIdx.x] = m.held;
    }
}

// A table entry is given up: if nobody else holds its page, the page is free.
__device__ __forceinline__ void give_up(const CacheArgs &c, int page)
{
    if (page >= 0 && page < c.pages && atomicSub(&c.refs[page], 1) == 1) atomicMin(&c.own[OWN_LOW], page);
}

// Block x of n that a stream has: its share of the table row, 256 entries at a time, and of the tails, a layer and head at a time.  No page is free in between: who gives one up held it, and who takes one takes it from a slot that keeps it.
template <int D>
__device__ __forceinline__ void reorder_share(const ReorderArgs &a, const Move &m, int x, int n)
{
    const CacheArgs &c = a.c;
    const int len = m.plan.first, moves = m.plan.count, to = m.plan.slot, from = m.plan.other, full = len / P, old_full = m.held / P;
    for (int i = x * 256 + (int)threadIdx.x; i < max(full, moves ? old_full : 0); i += n * 256) {
        const bool gone = a.window > 0 && (i + 1) * P <= len - a.window + 1 && i * P >= a.sink;
        int *const mine = c.table + (size_t)to * c.columns + i;
        if (moves == 0) {
            if (!gone) continue;
            give_up(c, *mine);
            *mine = -1;
            continue;
        }
        const int page = moves == 2 && i < full && !gone ? c.table[(size_t)from * c.columns + i] : -1;
        if (page >= 0 && page < c.pages) atomicAdd(&c.refs[page], 1);
        if (i < old_full) give_up(c, *mine);
        *mine = page;
    }
    if (moves != 2) return;
    constexpr int HEAD = P * D / 8, PER = HEAD / 256;    // pieces of a head's tail, of them a thread's
    const int pieces = len % P * (D / 8), units = c.L * c.H;
    if (pieces == 0) return;
    u32x4 *const ks = reinterpret_cast<u32x4 *>(c.k_tail), *const vs = reinterpret_cast<u32x4 *>(c.v_tail);
    for (int unit = x; unit < units; unit += n) {
        const int l = unit / c.H;
        const size_t head = (size_t)l * (c.S - 1) * c.H + unit;        // [l][slot][h] is l * S * H + slot * H + h
        const size_t src = (head + (size_t)from * c.H) * HEAD + threadIdx.x, dst = (head + (size_t)to * c.H) * HEAD + threadIdx.x;
        u32x4 k[PER], v[PER];
#pragma unroll
        for (int u = 0; u < PER; ++u)
            if ((int)threadIdx.x + u * 256 < pieces) k[u] = ks[src + u * 256], v[u] = vs[src + u * 256];
#pragma unroll
        for (int u = 0; u < PER; ++u)
            if ((int)threadIdx.x + u * 256 < pieces) ks[dst + u * 256] = k[u], vs[dst + u * 256] = v[u];
    }
}

template <int D>
__global__ __launch_bounds__(256) void reorder_move(const ReorderArgs a)
{
    const int s = blockIdx.y;
    const Move m{plans(a.c)[s], a.c.own[own_plan(a.c.S) + PLAN_WORDS * a.c.S + s]};
    reorder_share<D>(a, m, blockIdx.x, gridDim.x);
}

template <int D>
__global__ __launch_bounds__(ONE) void reorder_step(const ReorderArgs a)
{
    __shared__ ReorderLds<ONE> lds;
    __shared__ Move mine;
    __shared__ int is_last;
    const CacheArgs &c = a.c;
    const int tid = threadIdx.x, s = blockIdx.y;
    const Move m = reorder_plan_of<ONE>(a, lds);
    if (tid == s) mine = m;
    __syncthreads();                                     // (the block has read slot and len)
    if (tid == 0) is_last = last_to_read(c, s, gridDim.x);
    reorder_share<D>(a, mine, blockIdx.x, gridDim.x);
    __syncthreads();
    if (is_last && tid < c.S) {
        c.slot[tid] = m.plan.slot;
        c.len[tid] = m.plan.first;
    }
}

// ---------------------------------------------------------------------------------------------- copy

constexpr int PAGE_BLOCKS = 4096;                        // of a copy, for all layers
struct CopyArgs {
    CacheArgs from, to;
    const int *source;
    int *n_used;
};

// Pages that the streams hold, how often, and which place each takes.  The marks of the pool's pages stand behind the plans of `from`, the list
// of pages to copy behind those of `to`.  As the lowest free pages are taken first, of large pools only what lies below the highest page held
// is looked at (a copy of little out of 250000 pages 300 -> 9 us).
__global__ __launch_bounds__(CTRL) void copy_plan(const CopyArgs a)
{
    constexpr int EACH = 4;
    __shared__ int part[CTRL / 64], start[CTRL], row[CTRL], too_long, above;
    const CacheArgs &f = a.from, &t = a.to;
    const int tid = threadIdx.x;
    int *const marks = f.own + own_plan(f.S) + (PLAN_WORDS + 1) * f.S, *const list = t.own + own_plan(t.S) + (PLAN_WORDS + 1) * t.S;
    const bool small = f.pages <= EACH * CTRL;           // (one round: not worth a search)
    const auto clear = [&](int pages) {
        for (int p = tid; p < pages; p += CTRL) __hip_atomic_store(&marks[p], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    if (small) clear(f.pages);
    if (tid == 0) too_long = above = 0;
    int len = 0, slot = 0, has = 0;
    if (tid < t.S) {
        const int s = a.source[tid];
        has = s >= 0 && s < f.S;
        if (has) {
            len = len_of(f, s);
            slot = slot_of(f, s);
        }
    }
    __syncthreads();
    if (len / P > t.columns) atomicOr(&too_long, 1);
    const Sums entries = sums_of<CTRL>(len / P, part);
    start[tid] = entries.before;
    row[tid] = slot;
    __syncthreads();
    const auto page_of = [&](int i) {
        const int s = last_from(start, t.S, i);
        return f.table[(size_t)row[s] * f.columns + (i - start[s])];
    };
    const int mine = tid < entries.all ? page_of(tid) : -1;     // (all that there is to read, as a rule)
    if (!small) {
        int highest = mine < f.pages ? mine : -1;
        for (int i = tid + CTRL; i < entries.all; i += CTRL) {
            const int page = page_of(i);
            if (page < f.pages) highest = max(highest, page);
        }
        if (highest >= 0) atomicMax(&above, highest + 1);
        __syncthreads();
        clear(above);
        __syncthreads();
    }
    const int pages = small ? f.pages : above;
    for (int i = tid; i < entries.all; i += CTRL) {
        const int page = i == tid ? mine : page_of(i);
        if (page >= 0 && page < f.pages) __hip_atomic_fetch_add(&marks[page], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    int used = 0;
    for (int p0 = 0; p0 < pages; p0 += EACH * CTRL) {
        int held[EACH], some = 0;
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int p = p0 + EACH * tid + u;
            held[u] = p < pages ? __hip_atomic_load(&marks[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
        }
#pragma unroll
        for (int u = 0; u < EACH; ++u) some += held[u] > 0;
        __syncthreads();
        const Sums at = sums_of<CTRL>(some, part);
        int place = used + at.before;
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int p = p0 + EACH * tid + u;
            if (p < pages) marks[p] = held[u] > 0 ? place : -1;
            if (held[u] > 0) {
                if (place < t.pages) list[place] = p, t.refs[place] = held[u];
                ++place;
            }
        }
        used += at.all;
    }
    __syncthreads();
    const bool fits = used <= t.pages && !too_long;
    if (tid < t.S) {
        t.slot[tid] = tid;
        t.len[tid] = fits ? len : 0;
        plans(t)[tid] = Plan{fits ? len : 0, has && fits, tid, slot};
    }
    if (tid == 0) {
        t.own[OWN_LOW] = t.own[OWN_COUNT] = fits ? used : 0;
        if (a.n_used) *a.n_used = used;
    }
}

// 384 pages of 2 layers of 8 heads of 64 features, 100 MB: 24 to 28 us (3.6 to 4.2 TB/s), and 6 for copy_plan.
// Blocks over the pages of a layer, then over the tails of its streams and heads, then (in the first layer) over the table and the pages that are free.
template <int D>
__global__ __launch_bounds__(256) void copy_move(const CopyArgs a, int page_blocks, int tail_blocks)
{
    const CacheArgs &f = a.from, &t = a.to;
    const int tid = threadIdx.x, l = blockIdx.y, b = blockIdx.x;
    if (b < page_blocks) {
        const int count = t.own[OWN_COUNT];
        for (int place = b; place < count; place += page_blocks) {
            const int page = t.own[own_plan(t.S) + (PLAN_WORDS + 1) * t.S + place];
            const size_t src = ((size_t)l * f.pages + page) * f.H, dst = ((size_t)l * t.pages + place) * t.H;
            const u32x4 *const ks = reinterpret_cast<const u32x4 *>(f.k + src * P * D), *const vs = reinterpret_cast<const u32x4 *>(f.v + src * P * D);
            u32x4 *const kt = reinterpret_cast<u32x4 *>(t.k + dst * P * D), *const vt = reinterpret_cast<u32x4 *>(t.v + dst * P * D);
            constexpr int AT_ONCE = 4;
            for (int i = tid; i < f.H * (P * D / 16); i += 256 * AT_ONCE) {
                u32x4 k[AT_ONCE], v[AT_ONCE];
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u)
                    if (i + u * 256 < f.H * (P * D / 16)) k[u] = ks[i + u * 256], v[u] = vs[i + u * 256];
#pragma unroll
                for (int u = 0; u < AT_ONCE; ++u)
                    if (i + u * 256 < f.H * (P * D / 16)) kt[i + u * 256] = k[u], vt[i + u * 256] = v[u];
            }
            for (int h = tid; h < f.H; h += 256) {
                t.k_scale[dst + h] = f.k_scale[src + h];
                t.v_scale[dst + h] = f.v_scale[src + h];
            }
        }
    } else if (b < page_blocks + tail_blocks) {
        const int unit = b - page_blocks, s = unit / t.H, h = unit - s * t.H;
        const Plan plan = plans(t)[s];
        const int n = plan.count ? plan.first % P : 0;
        const size_t src = (((size_t)l * f.S + plan.other) * f.H + h) * P * D, dst = (((size_t)l * t.S + s) * t.H + h) * P * D;
        for (int i = tid; i < n * (D / 8); i += 256) {
            reinterpret_cast<u32x4 *>(t.k_tail + dst)[i] = reinterpret_cast<const u32x4 *>(f.k_tail + src)[i];
            reinterpret_cast<u32x4 *>(t.v_tail + dst)[i] = reinterpret_cast<const u32x4 *>(f.v_tail + src)[i];
        }
    } else if (l == 0) {
        const int *const marks = f.own + own_plan(f.S) + (PLAN_WORDS + 1) * f.S;
        const long long i = (long long)(b - page_blocks - tail_blocks) * 256 + tid, threads = (long long)(gridDim.x - page_blocks - tail_blocks) * 256;
        for (long long p = t.own[OWN_COUNT] + i; p < t.pages; p += threads) t.refs[p] = 0;
        const int s = (int)(i / t.columns), column = (int)(i - (long long)s * t.columns);
        if (s >= t.S) return;
        const Plan plan = plans(t)[s];
        int page = -1;
        if (plan.count && column < plan.first / P) page = f.table[(size_t)plan.other * f.columns + column];
        t.table[i] = page >= 0 && page < f.pages ? marks[page] : -1;
    }
}

// ---------------------------------------------------------------------------------------------- host

bool misaligned(const void *p, unsigned mask) { return (reinterpret_cast<uintptr_t>(p) & mask) != 0; }

CacheArgs args_of(const mlora_page_cache *c)
{
    return CacheArgs{reinterpret_cast<int8_t *>(c->k), reinterpret_cast<int8_t *>(c->v), c->k_scale, c->v_scale,
                     reinterpret_cast<uint16_t *>(c->k_tail), reinterpret_cast<uint16_t *>(c->v_tail), c->slot, c->len, c->table, c->refs, c->own,
                     c->n_layers, c->n_streams, c->n_kv_heads, c->head_dim, c->n_pages, c->max_pages};
}

}  // namespace

mlora_status check_page_cache(const mlora_page_cache *c)
{
    if (!c) return MLORA_EINVAL;
    if (c->head_dim != 64 && c->head_dim != 128) return MLORA_ESHAPE;
    if (c->n_layers <= 0 || c->n_streams <= 0 || c->n_kv_heads <= 0 || c->n_pages <= 0 || c->max_pages <= 0) return MLORA_ESHAPE;
    if (c->n_streams > MLORA_PAGE_MAX_STREAMS || c->n_pages > MLORA_PAGE_MAX_PAGES || c->max_pages > MLORA_PAGE_MAX_COLUMNS) return MLORA_ESHAPE;
    if ((double)c->n_layers * c->n_streams * c->n_kv_heads > MLORA_PAGE_MAX_HEADS || c->n_layers > 65535) return MLORA_ESHAPE;
    if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !c->slot || !c->len || !c->table || !c->refs || !c->own)
        return MLORA_EINVAL;
    for (const void *p : {(const void *)c->k, (const void *)c->v, (const void *)c->k_tail, (const void *)c->v_tail})
        if (misaligned(p, 15u)) return MLORA_EALIGN;
    for (const void *p : {(const void *)c->k_scale, (const void *)c->v_scale, (const void *)c->slot, (const void *)c->len, (const void *)c->table,
                          (const void *)c->refs, (const void *)c->own})
        if (misaligned(p, 3u)) return MLORA_EALIGN;
    return MLORA_OK;
}

}  // namespace mlora

using namespace mlora;

extern "C" {

size_t mlora_page_cache_own_words(int32_t n_streams, int32_t n_pages)
{
    if (n_streams <= 0 || n_streams > MLORA_PAGE_MAX_STREAMS || n_pages <= 0 || n_pages > MLORA_PAGE_MAX_PAGES) return 0;
    return (size_t)own_plan(n_streams) + (size_t)(PLAN_WORDS + 1) * n_streams + n_pages;
}

mlora_status mlora_page_cache_append(const mlora_page_cache *c, const void *k_new, const void *v_new, int32_t rows_per_stream,
                                     const int32_t *rows, int32_t n_rows, int32_t *appended, void *stream)
{
    const mlora_status st = check_page_cache(c);
    if (st != MLORA_OK) return st;
    if (!k_new || !v_new) return MLORA_EINVAL;
    if (misaligned(k_new, 15u) || misaligned(v_new, 15u) || misaligned(rows, 3u) || misaligned(appended, 3u)) return MLORA_EALIGN;
    if (rows_per_stream <= 0 || (long long)c->n_streams * rows_per_stream > MLORA_MAX_ROWS) return MLORA_ESHAPE;
    const int n = rows ? n_rows : rows_per_stream;
    if (n < 1 || n > rows_per_stream) return MLORA_ESHAPE;
    const AppendArgs a{args_of(c), reinterpret_cast<const uint16_t *>(k_new), reinterpret_cast<const uint16_t *>(v_new), rows, appended, rows_per_stream, n};
    hipStream_t s = (hipStream_t)stream;
    const unsigned heads = (unsigned)(c->n_layers * c->n_streams * c->n_kv_heads);
    if (n <= P && c->n_streams <= ONE) {
        if (c->head_dim == 64) append_step<64><<<dim3(heads), dim3(ONE), 0, s>>>(a);
        else                   append_step<128><<<dim3(heads), dim3(ONE), 0, s>>>(a);
        return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
    }
    append_plan<<<dim3(1), dim3(CTRL), 0, s>>>(a);
    const dim3 grid(heads, (unsigned)((P - 1 + n) / P));
    if (c->head_dim == 64) append_rows<64><<<grid, dim3(256), 0, s>>>(a);
    else                   append_rows<128><<<grid, dim3(256), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

mlora_status mlora_page_cache_reorder(const mlora_page_cache *c, const int32_t *source, int32_t window, int32_t sink, void *stream)
{
    const mlora_status st = check_page_cache(c);
    if (st != MLORA_OK) return st;
    if (misaligned(source, 3u)) return MLORA_EALIGN;
    if (window < 0 || sink < 0) return MLORA_ESHAPE;
    const ReorderArgs a{args_of(c), source, window, sink};
    hipStream_t s = (hipStream_t)stream;
    // Blocks of a stream: one per layer and head, up to some 512 in all (each draws a ticket, and tickets of a stream are drawn one after the other: 129 of
    // each of 8 streams 5.4 us, 64 4.8).
    const int blocks = std::max(1, std::min(std::max(c->n_layers * c->n_kv_heads, (c->max_pages + 255) / 256), 512 / c->n_streams));
    const dim3 grid((unsigned)blocks, (unsigned)c->n_streams);
    if (c->n_streams <= ONE) {
        if (c->head_dim == 64) reorder_step<64><<<grid, dim3(ONE), 0, s>>>(a);
        else                   reorder_step<128><<<grid, dim3(ONE), 0, s>>>(a);
        return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
    }
    reorder_plan<<<dim3(1), dim3(CTRL), 0, s>>>(a);
    if (c->head_dim == 64) reorder_move<64><<<grid, dim3(256), 0, s>>>(a);
    else                   reorder_move<128><<<grid, dim3(256), 0, s>>>(a);
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

mlora_status mlora_page_cache_copy(const mlora_page_cache *from, const mlora_page_cache *to, const int32_t *source, int32_t *n_used, void *stream)
{
    mlora_status st = check_page_cache(from);
    if (st == MLORA_OK) st = check_page_cache(to);
    if (st != MLORA_OK) return st;
    if (!source) return MLORA_EINVAL;
    if (misaligned(source, 3u) || misaligned(n_used, 3u)) return MLORA_EALIGN;
    if (from->n_layers != to->n_layers || from->n_kv_heads != to->n_kv_heads || from->head_dim != to->head_dim) return MLORA_ESHAPE;
    if (from->k == to->k || from->v == to->v || from->k_scale == to->k_scale || from->v_scale == to->v_scale || from->k_tail == to->k_tail
        || from->v_tail == to->v_tail || from->slot == to->slot || from->len == to->len || from->table == to->table || from->refs == to->refs
        || from->own == to->own) return MLORA_EINVAL;
    const CopyArgs a{args_of(from), args_of(to), source, n_used};
    hipStream_t s = (hipStream_t)stream;
    copy_plan<<<dim3(1), dim3(CTRL), 0, s>>>(a);
    // (pools are larger than what is copied, as a rule: blocks that find nothing cost, too)
    const int page_blocks = std::min(std::min(from->n_pages, to->n_pages), std::max(PAGE_BLOCKS / to->n_layers, 256));
    const int tail_blocks = to->n_streams * to->n_kv_heads;
    const long long others = std::max(((long long)to->n_streams * to->max_pages + 255) / 256, std::min((to->n_pages + 1023ll) / 1024, 256ll));
    const dim3 grid((unsigned)(page_blocks + tail_blocks + others), (unsigned)to->n_layers);
    if (to->head_dim == 64) copy_move<64><<<grid, dim3(256), 0, s>>>(a, page_blocks, tail_blocks);
    else                    copy_move<128><<<grid, dim3(256), 0, s>>>(a, page_blocks, tail_blocks);
    return hipGetLastError() == hipSuccess ? MLORA_OK : MLORA_EHIP;
}

}  // extern "C"
