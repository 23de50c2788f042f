// Pages, slots and positions of a step's new tokens: block tables kept on the device from request lengths alone.
//
// The state is page_refs (rows that hold a page, 0 = free) and each row's pages.  With need_b = ceil((ctx_b + n_b) / P), base_b =
// pages the row holds or takes over from another row, grow_b = max(0, need_b - base_b) and the free pages in ascending order
// f_0 < f_1 < .., row b gets f_(g_b) .. f_(g_b + grow_b - 1), g_b = sum of grow before b: two sums over rows, one list of the
// free pages, and no list that would have to be kept from call to call.
//
// What bounds it: latency.  A step moves a few KB beside the 4 bytes a page of page_refs.  Three phases depend on one another:
//   rows    records, shared pages counted up and released ones down
//   pages   the free pages of every piece of the pool, in order (and the sums over the rows)
//   give    a thread per new token finds its row, its page, its slot; the thread of a page's first position writes the page's
//           entries, so tables and references cost no pass of their own
// Calls of up to kSmallPages pages, kSmallRows rows and some thousand tokens take one workgroup and one launch, in which a barrier separates the
// phases and the pages' counts stay as bits in LDS: 64 rows of 9 tokens, 16 384 pages, 12.3 us.  Beyond that they are three launches, 6.0 + 5.3 + 5.7 us for
// 512 rows and 327 680 pages, 8.7 + 5.7 + 6.4 for 64 whole prompts and a million pages (4 MB; all medians): each is a launch and three or four loads that wait for
// one another, and to release a row of 2048 pages is four rounds of 512 page ids, one behind the other, by the row's one wave.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/seer_verify.h"
#include "seer_device.h"

namespace seer {

constexpr int kReserveMaxB = 16384;
// one workgroup takes the call up to these sizes
constexpr int kSmallThreads = 1024, kSmallPages = 32 * kSmallThreads, kSmallRows = kSmallThreads, kSmallTokens = 8192;
constexpr int kThreads = 256;
constexpr int kPieceStep = kThreads * 16;            // pages that a workgroup looks at together
constexpr int kMaxPieces = 2048;

// A row of the call: positions and pages before it, pages it needs beside them (-1: refused, left as it is), new tokens (-1: over).
struct ReserveRow {
    int32_t ctx, base, grow, n;
};

struct ReserveArgs {
    const int32_t* ctx_len;
    const int32_t* n_new;
    const int32_t* share_from;
    const uint64_t* tree_mask;
    int32_t* block_table;
    int32_t* held;
    int32_t* refs;
    int32_t* step_len;
    int32_t* first;
    int32_t* slot;
    int32_t* position;
    int32_t* status;
    ReserveRow* rows;        // [B]
    int32_t* start;          // [B] sum of grow before the row
    int32_t* counts;         // [pieces] free pages of a piece
    int32_t* list;           // [pieces][piece] the free pages of a piece
    int B, P, num_pages, max_pages, n_tokens, piece, pieces;
    uint32_t inv_p;          // 2^32 / P, at most 2^32 - 1
};

// Page of a position: the product's upper half is the quotient or one less.
__device__ __forceinline__ int reserve_page(const ReserveArgs& a, int position) {
    const uint32_t x = static_cast<uint32_t>(position), d = static_cast<uint32_t>(a.P), q = __umulhi(x, a.inv_p);
    return static_cast<int>(q + ((d - 1u - (x - q * d)) >> 31));
}

__device__ __forceinline__ void raise(const ReserveArgs& a, int bits) {
    if (bits && a.status) atomicOr(a.status, bits);
}

// What the arrays hold for row b before the call (requested together).
struct ReserveInput {
    int n, ctx, held, share;
};
__device__ __forceinline__ ReserveInput reserve_input(const ReserveArgs& a, int b) {
    return ReserveInput{a.n_new[b], a.ctx_len[b], a.held[b], a.share_from ? a.share_from[b] : -1};
}
// The record of row b; `before`: new tokens of the rows before it.  error: status bits.
__device__ __forceinline__ ReserveRow reserve_row(const ReserveArgs& a, int b, const ReserveInput& in, int64_t before, int& error) {
    ReserveRow r{in.ctx, in.held, -1, in.n};
    error = 1;
    if (r.n < -1 || r.base < 0 || r.base > a.max_pages) return r;
    if (r.n < 0) {
        r.ctx = 0, r.grow = 0, error = 0;
        return r;
    }
    const int64_t end = static_cast<int64_t>(r.ctx) + r.n;
    if (r.ctx < 0 || end > static_cast<int64_t>(a.max_pages) * a.P) return r;
    if (in.share >= 0) {
        const int pages = reserve_page(a, r.ctx);
        if (in.share >= a.B || in.share == b || r.base != 0 || r.ctx != pages * a.P) return r;
        const int theirs = a.held[in.share];
        if (theirs < 0 || theirs > a.max_pages || pages > theirs) return r;
    } else if (r.ctx > static_cast<int64_t>(r.base) * a.P) {
        return r;
    }
    error = 4;
    if (before + r.n > a.n_tokens) return r;
    if (in.share >= 0) r.base = reserve_page(a, r.ctx);
    const int need = end == 0 ? 0 : reserve_page(a, static_cast<int>(end) - 1) + 1;
    r.grow = max(0, need - r.base), error = 0;
    return r;
}
__device__ __forceinline__ int reserve_need(const ReserveArgs& a, const ReserveRow& r) {
    return r.n < 0 || r.ctx + r.n == 0 ? 0 : reserve_page(a, r.ctx + r.n - 1) + 1;
}

// count(page) for the pages in row[from .. to), `lanes` threads to a row, several requested at a time.
template <class Count>
__device__ __forceinline__ int count_pages(const ReserveArgs& a, const int32_t* row, int from, int to, int lane, int lanes, Count&& count) {
    constexpr int kAhead = 8;
    int error = 0;
    for (int j0 = from + lane; j0 < to; j0 += kAhead * lanes) {
        int page[kAhead];
#pragma unroll
        for (int x = 0; x < kAhead; ++x) page[x] = row[min(j0 + x * lanes, to - 1)];
#pragma unroll
        for (int x = 0; x < kAhead; ++x)
            if (j0 + x * lanes < to) {
                if (page[x] >= 0 && page[x] < a.num_pages) count(page[x]);
                else error = 2;
            }
    }
    return error;
}
// Row b's shared pages up, or those that it no longer needs down.
template <class Count>
__device__ __forceinline__ int count_row(const ReserveArgs& a, int b, const ReserveRow& r, int share, int lane, int lanes, Count&& count) {
    if (r.grow < 0) return 0;
    if (share >= 0 && r.n >= 0) return count_pages(a, a.block_table + static_cast<size_t>(share) * a.max_pages, 0, r.base, lane, lanes, [&](int page) { count(page, 1); });
    return count_pages(a, a.block_table + static_cast<size_t>(b) * a.max_pages, reserve_need(a, r), r.base, lane, lanes, [&](int page) { count(page, -1); });
}
// What a row holds from now on; `granted`: it got its pages.
__device__ __forceinline__ int finish_row(const ReserveArgs& a, int b, const ReserveRow& r, int share, bool granted, int lane, int lanes) {
    int error = 0;
    if (share >= 0 && r.grow >= 0 && r.n >= 0) {
        const int32_t* from = a.block_table + static_cast<size_t>(share) * a.max_pages;
        if (granted) {
            int32_t* to = a.block_table + static_cast<size_t>(b) * a.max_pages;
#pragma unroll 8
            for (int j = lane; j < r.base; j += lanes) to[j] = from[j];
        } else {
            error = count_pages(a, from, 0, r.base, lane, lanes, [&](int page) { atomicAdd(a.refs + page, -1); });
        }
    }
    if (lane == 0) {
        if (granted) a.held[b] = reserve_need(a, r);
        a.step_len[b] = granted && r.n >= 0 ? r.ctx + r.n : 0;
        if (r.grow >= 0 && !granted) error |= 8;
    }
    return error;
}

// Slot and position of new token i, of row b whose tokens begin at `begin`; page_at(rank): the rank-th free page.
template <class PageAt>
__device__ __forceinline__ int place_token(const ReserveArgs& a, int i, int b, int begin, const ReserveRow& r, int start, bool granted, PageAt&& page_at) {
    int slot = -1, position = -1, error = 0;
    if (granted) {
        const int at = r.ctx + (i - begin), lp = reserve_page(a, at), inside = at - lp * a.P;
        int32_t* entry = a.block_table + static_cast<size_t>(b) * a.max_pages + lp;
        int page;
        if (lp < r.base) {
            page = *entry;
        } else {
            page = page_at(start + lp - r.base);
            if (inside == 0) *entry = page, a.refs[page] = 1;       // (every position of a new page is a new token's, its first one too)
        }
        position = at;
        if (page >= 0 && page < a.num_pages) slot = page * a.P + inside;
        else error = 2;
        if (a.tree_mask) {
            const uint64_t word = a.tree_mask[i];
            if (word) position = r.ctx + __popcll(word) - 1;
        }
    }
    a.slot[i] = slot;
    a.position[i] = position;
    return error;
}

// The row of token i: the last one whose tokens begin at or before it (first[0 .. B], ascending; rows without tokens come before).
__device__ __forceinline__ int row_of_token(const int32_t* first, int B, int i) {
    int lo = 0, hi = B;                              // first[lo] <= i; first[hi] > i or hi == B
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= i) lo = mid;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ int64_t wave_sum64(int64_t v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, kWave);
    return v;
}
// Sum of v over the threads before this one; total: over all.  Ends behind a barrier.
template <int THREADS>
__device__ __forceinline__ int64_t block_before(int64_t v, int64_t* s_sums, int64_t& total) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    int64_t up = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int64_t x = __shfl_up(up, o, kWave);
        if (lane >= o) up += x;
    }
    if (lane == kWave - 1) s_sums[wave] = up;
    __syncthreads();
    int64_t before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) {
        if (w < wave) before += s_sums[w];
        total += s_sums[w];
    }
    __syncthreads();
    return before + up - v;
}
__device__ __forceinline__ int32_t saturate(int64_t x) { return x > 0x7fffffff ? 0x7fffffff : static_cast<int32_t>(x); }

// Which of ROWS * 64 pages from page0 on are free: lane x < ROWS gets the bits of pages page0 + 64 x ...  below: the same for counts below 0 (BITS),
// or whether this lane saw one.  (Read past the vector cache: another workgroup may have counted them a moment ago.)
template <int ROWS, bool BITS>
__device__ __forceinline__ void look_at_pages(const ReserveArgs& a, int64_t page0, int64_t end, uint64_t& free, uint64_t& below) {
    const int lane = threadIdx.x & (kWave - 1);
    int refs[ROWS];
#pragma unroll
    for (int x = 0; x < ROWS; ++x)
        refs[x] = __hip_atomic_load(a.refs + min(page0 + x * kWave + lane, static_cast<int64_t>(a.num_pages) - 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    free = below = 0;
#pragma unroll
    for (int x = 0; x < ROWS; ++x) {
        const bool there = page0 + x * kWave + lane < end;
        const uint64_t f = __ballot(refs[x] == 0 && there);
        if (lane == x) free = f;
        if constexpr (BITS) {
            const uint64_t n = __ballot(refs[x] < 0 && there);
            if (lane == x) below = n;
        } else {
            if (refs[x] < 0 && there) below = 1;
        }
    }
}
// Writes those pages behind one another, lane x's at `at` and on, as far as `limit`.
template <int ROWS>
__device__ __forceinline__ void write_pages(int32_t* list, int limit, int page0, uint64_t mine, int at) {
    const int lane = threadIdx.x & (kWave - 1);
    for (int x = 0; x < ROWS; ++x) {
        const uint64_t bits = static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(mine >> 32), x))) << 32 |
                              static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(mine), x));
        const int to = __builtin_amdgcn_readlane(at, x) + __popcll(bits & ((1ull << lane) - 1));
        if (((bits >> lane) & 1) && to < limit) list[to] = page0 + x * kWave + lane;
    }
}

// ---------------------------------------------------------------------------
// one workgroup
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kSmallThreads) void reserve_small(ReserveArgs a) {
    __shared__ ReserveRow s_row[kSmallRows];
    __shared__ int32_t s_share[kSmallRows];
    __shared__ int32_t s_first[kSmallRows + 1], s_start[kSmallRows];
    __shared__ int32_t s_list[kSmallTokens];
    __shared__ unsigned long long s_free[kSmallPages / kWave], s_below[kSmallPages / kWave];
    __shared__ int64_t s_sums[kSmallThreads / kWave];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    int error = 0;
    int64_t total, all_tokens;
    constexpr int kRows = kSmallPages / kSmallThreads;                         // (of 64 pages, a wave)
    const int page0 = wave * kRows * kWave;
    {
        // the rows' numbers and the counts as they are before the call are requested together
        const ReserveInput in = reserve_input(a, min(tid, a.B - 1));
        uint64_t free = 0, below = 0;
        if (page0 < a.num_pages) look_at_pages<kRows, true>(a, page0, a.num_pages, free, below);
        if (lane < kRows) s_free[wave * kRows + lane] = free, s_below[wave * kRows + lane] = below;
        const int64_t before = block_before<kSmallThreads>(tid < a.B ? max(in.n, 0) : 0, s_sums, all_tokens);
        int64_t grow = 0;
        if (tid < a.B) {
            const ReserveRow r = reserve_row(a, tid, in, before, error);
            s_row[tid] = r, s_share[tid] = in.share, s_first[tid] = saturate(before), a.first[tid] = saturate(before);
            grow = max(r.grow, 0);
            if (tid == a.B - 1) s_first[a.B] = saturate(all_tokens), a.first[a.B] = saturate(all_tokens);
        }
        const int64_t start = block_before<kSmallThreads>(grow, s_sums, total);
        if (tid < a.B) s_start[tid] = saturate(start);
    }
    __syncthreads();
    // a count that comes to zero or leaves it turns its page's bit over, in whatever order that happens; one that passes below zero its other bit
    const int lanes = min(kWave, kSmallThreads >> (32 - __clz(a.B - 1 | 1))), at_lane = tid & (lanes - 1), at_row = tid / lanes;      // (all rows at once)
    if (at_row < a.B)
        error |= count_row(a, at_row, s_row[at_row], s_share[at_row], at_lane, lanes, [&](int page, int by) {
            const int was = atomicAdd(a.refs + page, by);
            if (was == 0 || was + by == 0) atomicXor(s_free + page / kWave, 1ull << (page % kWave));
            if ((was < 0) != (was + by < 0)) atomicXor(s_below + page / kWave, 1ull << (page % kWave));
        });
    __syncthreads();
    const int wanted = saturate(total);
    int64_t free_total;
    {
        const uint64_t mine = lane < kRows ? s_free[wave * kRows + lane] : 0;
        if (lane < kRows && s_below[wave * kRows + lane]) error |= 16;
        const int at = static_cast<int>(block_before<kSmallThreads>(__popcll(mine), s_sums, free_total));
        if (wanted > 0 && __any(mine != 0)) write_pages<kRows>(s_list, min(wanted, kSmallTokens), page0, mine, at);
    }
    __syncthreads();
    auto granted = [&](int b) { return s_row[b].grow == 0 || (s_row[b].grow > 0 && static_cast<int64_t>(s_start[b]) + s_row[b].grow <= free_total); };
    if (at_row < a.B) error |= finish_row(a, at_row, s_row[at_row], s_share[at_row], granted(at_row), at_lane, lanes);
    for (int i = tid; i < a.n_tokens; i += kSmallThreads) {
        const bool real = i < s_first[a.B];
        const int b = row_of_token(s_first, a.B, i);
        error |= place_token(a, i, b, s_first[b], s_row[b], s_start[b], real && granted(b), [&](int rank) { return s_list[rank]; });
    }
    raise(a, error);
}

// ---------------------------------------------------------------------------
// three launches
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(kThreads) void reserve_rows(ReserveArgs a) {
    constexpr int kRows = kThreads / kWave;
    __shared__ int64_t s_sums[kRows];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, b0 = blockIdx.x * kRows, b = b0 + wave;
    const ReserveInput in = reserve_input(a, min(b, a.B - 1));
    // tokens of the rows before this workgroup's, then of those before this wave's
    int64_t sum = 0;
#pragma unroll 4
    for (int i = tid; i < b0; i += kThreads) sum += max(a.n_new[i], 0);
    sum = wave_sum64(sum);
    if (lane == 0) s_sums[wave] = sum;
    __syncthreads();
    int64_t before = 0;
#pragma unroll
    for (int x = 0; x < kRows; ++x) before += s_sums[x];
    if (b >= a.B) return;
    for (int x = b0; x < b; ++x) before += max(a.n_new[x], 0);
    int error;
    const ReserveRow r = reserve_row(a, b, in, before, error);
    if (lane == 0) {
        a.rows[b] = r;
        a.first[b] = saturate(before);
        if (b == a.B - 1) a.first[a.B] = saturate(before + max(r.n, 0));
    }
    error |= count_row(a, b, r, in.share, lane, kWave, [&](int page, int by) { atomicAdd(a.refs + page, by); });
    raise(a, error);
}

// Workgroup 0: the sums of grow.  The others: the free pages of a piece of the pool, in order.
__global__ __launch_bounds__(kThreads) void reserve_pages(ReserveArgs a) {
    __shared__ int64_t s_sums[kThreads / kWave];
    const int tid = threadIdx.x;
    int64_t total;
    if (blockIdx.x == 0) {
        int64_t sum = 0;
        for (int b0 = 0; b0 < a.B; b0 += kThreads) {
            const int b = b0 + tid;
            const int64_t before = block_before<kThreads>(b < a.B ? max(a.rows[b].grow, 0) : 0, s_sums, total);
            if (b < a.B) a.start[b] = saturate(sum + before);
            sum += total;
        }
        return;
    }
    const int piece = blockIdx.x - 1, first = piece * a.piece, end = min(first + a.piece, a.num_pages);
    int32_t* list = a.list + first;
    int count = 0;
    for (int page0 = first; page0 < end; page0 += kPieceStep) {
        constexpr int kRows = kPieceStep / kThreads;
        const int wave0 = page0 + tid / kWave * kRows * kWave;
        uint64_t mine, below;
        look_at_pages<kRows, false>(a, wave0, end, mine, below);
        if (below) raise(a, 16);
        const int at = count + static_cast<int>(block_before<kThreads>(__popcll(mine), s_sums, total));
        write_pages<kRows>(list, a.piece, wave0, mine, at);
        count += static_cast<int>(total);
    }
    if (tid == 0) a.counts[piece] = count;
}

constexpr int kFirstInLds = 4096;

__global__ __launch_bounds__(kThreads) void reserve_give(ReserveArgs a, int token_blocks) {
    __shared__ int32_t s_before[kMaxPieces + 1];      // free pages of the pieces before
    __shared__ int32_t s_first[kFirstInLds + 1];
    __shared__ int64_t s_sums[kThreads / kWave];
    const int tid = threadIdx.x;
    int64_t sum = 0, total;
    for (int p0 = 0; p0 < a.pieces; p0 += kThreads) {
        const int64_t before = block_before<kThreads>(p0 + tid < a.pieces ? a.counts[p0 + tid] : 0, s_sums, total);
        if (p0 + tid < a.pieces) s_before[p0 + tid] = static_cast<int32_t>(sum + before);
        sum += total;
    }
    const int64_t free_total = sum;
    auto granted = [&](const ReserveRow& r, int start) { return r.grow == 0 || (r.grow > 0 && static_cast<int64_t>(start) + r.grow <= free_total); };
    int error = 0;
    if (static_cast<int>(blockIdx.x) >= token_blocks) {
        const int lane = tid & (kWave - 1), b = (blockIdx.x - token_blocks) * (kThreads / kWave) + tid / kWave;
        if (b < a.B) {
            const ReserveRow r = a.rows[b];
            error = finish_row(a, b, r, a.share_from ? a.share_from[b] : -1, granted(r, a.start[b]), lane, kWave);
        }
        raise(a, error);
        return;
    }
    const bool in_lds = a.B <= kFirstInLds;
    if (in_lds)
        for (int b = tid; b <= a.B; b += kThreads) s_first[b] = a.first[b];
    __syncthreads();
    const int32_t* first = in_lds ? s_first : a.first;
    auto page_at = [&](int rank) {
        int lo = 0, hi = a.pieces;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_before[mid] <= rank) lo = mid;
            else hi = mid;
        }
        return a.list[static_cast<size_t>(lo) * a.piece + (rank - s_before[lo])];
    };
    // (a token a thread: four behind one another, looked up once, took 8.3 us of the kernel against 6.5 for 349 708 tokens, and 10.4 against 5.4 for 512 rows of
    // five: the chain of loads is longer where they are of two rows or pages)
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + tid;
    if (i < a.n_tokens) {
        const int b = row_of_token(first, a.B, static_cast<int>(i));
        const ReserveRow r = a.rows[b];
        const int start = a.start[b];
        error = place_token(a, static_cast<int>(i), b, first[b], r, start, i < first[a.B] && granted(r, start), page_at);
    }
    raise(a, error);
}

// SEER_RESERVE_OWN_PAGES: slots in pages that more than one row holds are taken back.  In a launch of its own, since only behind the others a count is what it stays (shared
// pages of rows that got nothing are counted down again last), so that the result depends on nothing else.  64 rows of 9 tokens 12.9 -> 15.3 us, 64 whole prompts 19.7 -> 23.5:
// what shares no page that way does without.
__global__ __launch_bounds__(kThreads) void reserve_own_pages(ReserveArgs a) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= a.n_tokens) return;
    const int slot = a.slot[i];
    if (slot < 0 || a.refs[reserve_page(a, slot)] <= 1) return;
    a.slot[i] = -1, a.position[i] = -1;
    raise(a, 32);
}
static hipError_t launch_own_pages(const seer_reserve_params& p, const ReserveArgs& a, hipStream_t stream) {
    if (!(p.flags & SEER_RESERVE_OWN_PAGES) || p.n_tokens == 0) return hipSuccess;
    hipLaunchKernelGGL(reserve_own_pages, dim3((p.n_tokens + kThreads - 1) / kThreads), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static int check_reserve_params(const seer_reserve_params* p) {
    if (!p) return SEER_EINVAL;
    if (p->B < 0 || p->page_size < 1 || p->num_pages < 1 || p->max_pages_per_seq < 1 || p->n_tokens < 0) return SEER_EINVAL;
    if (p->flags & ~SEER_RESERVE_OWN_PAGES) return SEER_EINVAL;
    if (p->B > kReserveMaxB || p->num_pages > 1 << 30 || static_cast<int64_t>(p->num_pages) * p->page_size > 0x7fffffffLL || p->n_tokens > 0x7fffffff - (1 << 20)) return SEER_ESHAPE;
    if (static_cast<int64_t>(p->max_pages_per_seq) * p->page_size > 0x7fffffffLL) return SEER_ESHAPE;
    return SEER_OK;
}
// One workgroup against three launches, calls with their host part: 8 rows of a token in 1024 pages 12.8 | 18.8 us, 64 of 9 in 16 384 13.0 | 19.5; in 32 768 pages,
// 1000 of 1 14.2 | 19.4, 8 of 1000 16.7 | 19.7, 256 of 30 19.3 | 19.1, 500 of 8 16.8 | 19.6, of 16 21.1 | 19.5, 1000 of 4 17.5 | 19.4, of 6 20.1 | 19.5: a pass over 1024
// tokens costs more where they are of many rows.
inline bool reserve_is_small(const seer_reserve_params& p) {
    return p.num_pages <= kSmallPages && p.B <= kSmallRows && p.n_tokens <= (p.B <= kSmallRows / 4 ? kSmallTokens : kSmallTokens * 5 / 8);
}
struct ReserveLayout {
    int piece, pieces;
    size_t off_start, off_counts, off_list, total;
};
inline ReserveLayout reserve_layout(const seer_reserve_params& p) {
    ReserveLayout w{};
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const int64_t share = (static_cast<int64_t>(p.num_pages) + kMaxPieces - 1) / kMaxPieces;
    w.piece = static_cast<int>((share + kPieceStep - 1) / kPieceStep) * kPieceStep;
    w.pieces = static_cast<int>((static_cast<int64_t>(p.num_pages) + w.piece - 1) / w.piece);
    w.off_start = up(sizeof(ReserveRow) * p.B);
    w.off_counts = w.off_start + up(sizeof(int32_t) * p.B);
    w.off_list = w.off_counts + up(sizeof(int32_t) * w.pieces);
    w.total = reserve_is_small(p) ? 256 : w.off_list + up(sizeof(int32_t) * p.num_pages);
    return w;
}

}  // namespace seer

extern "C" size_t seer_kv_reserve_workspace(const seer_reserve_params* p) {
    if (seer::check_reserve_params(p) != SEER_OK || p->B == 0) return 0;
    return seer::reserve_layout(*p).total;
}

extern "C" int seer_kv_reserve(const seer_reserve_params* p, const int32_t* ctx_len, const int32_t* n_new, const int32_t* share_from,
                               const uint64_t* tree_mask, int32_t* block_table, int32_t* pages_held, int32_t* page_refs, int32_t* step_len,
                               int32_t* first_token, int32_t* slot, int32_t* position, int32_t* status, void* workspace,
                               size_t workspace_bytes, void* hip_stream) {
    const int rc = seer::check_reserve_params(p);
    if (rc != SEER_OK) return rc;
    if (p->B == 0) return SEER_OK;
    if (!ctx_len || !n_new || !block_table || !pages_held || !page_refs || !step_len || !first_token || (p->n_tokens > 0 && (!slot || !position)))
        return SEER_EINVAL;
    if (step_len == ctx_len || step_len == n_new) return SEER_EINVAL;
    const seer::ReserveLayout layout = seer::reserve_layout(*p);
    if (!workspace || workspace_bytes < layout.total) return SEER_EWORKSPACE;
    auto misaligned = [](const void* ptr, uintptr_t a) { return reinterpret_cast<uintptr_t>(ptr) % a != 0; };
    if (misaligned(page_refs, 16) || misaligned(workspace, 16) || misaligned(tree_mask, 8) || misaligned(ctx_len, 4) || misaligned(n_new, 4) ||
        misaligned(share_from, 4) || misaligned(block_table, 4) || misaligned(pages_held, 4) || misaligned(step_len, 4) || misaligned(first_token, 4) ||
        misaligned(slot, 4) || misaligned(position, 4) || misaligned(status, 4))
        return SEER_EALIGN;
    seer::ReserveArgs a{};
    a.ctx_len = ctx_len, a.n_new = n_new, a.share_from = share_from, a.tree_mask = tree_mask;
    a.block_table = block_table, a.held = pages_held, a.refs = page_refs, a.step_len = step_len, a.first = first_token;
    a.slot = slot, a.position = position, a.status = status;
    a.B = p->B, a.P = p->page_size, a.num_pages = p->num_pages, a.max_pages = p->max_pages_per_seq, a.n_tokens = p->n_tokens;
    a.piece = layout.piece, a.pieces = layout.pieces;
    a.inv_p = p->page_size > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / static_cast<uint32_t>(p->page_size)) : 0xffffffffu;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (seer::reserve_is_small(*p)) {
        hipLaunchKernelGGL(seer::reserve_small, dim3(1), dim3(seer::kSmallThreads), 0, stream, a);
        hipError_t err = hipGetLastError();
        if (err == hipSuccess) err = seer::launch_own_pages(*p, a, stream);
        return err == hipSuccess ? SEER_OK : static_cast<int>(err);
    }
    char* ws = static_cast<char*>(workspace);
    a.rows = reinterpret_cast<seer::ReserveRow*>(ws);
    a.start = reinterpret_cast<int32_t*>(ws + layout.off_start);
    a.counts = reinterpret_cast<int32_t*>(ws + layout.off_counts);
    a.list = reinterpret_cast<int32_t*>(ws + layout.off_list);
    const unsigned row_blocks = (p->B + seer::kThreads / seer::kWave - 1) / (seer::kThreads / seer::kWave);
    const int token_blocks = (p->n_tokens + seer::kThreads - 1) / seer::kThreads;
    hipLaunchKernelGGL(seer::reserve_rows, dim3(row_blocks), dim3(seer::kThreads), 0, stream, a);
    hipLaunchKernelGGL(seer::reserve_pages, dim3(1u + layout.pieces), dim3(seer::kThreads), 0, stream, a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return static_cast<int>(err);
    hipLaunchKernelGGL(seer::reserve_give, dim3(token_blocks + row_blocks), dim3(seer::kThreads), 0, stream, a, token_blocks);
    err = hipGetLastError();
    if (err == hipSuccess) err = seer::launch_own_pages(*p, a, stream);
    return err == hipSuccess ? SEER_OK : static_cast<int>(err);
}
