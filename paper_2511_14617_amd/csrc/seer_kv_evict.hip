// seer_kv_evict: requests whose cache has grown over a limit keep `budget` positions per KV head: the first ones, the newest ones,
// and of those between the ones with the largest sums of attention weight.
//
// Attention does not depend on the order of the positions that every query sees, so only what would lie behind the new end
// moves: with E = budget - keep_last, the i-th kept position from E on (ascending, the newest aside) goes to the i-th free slot below
// E, and the newest keep_last positions become E .. budget - 1, in order.  A step that drops a few positions so moves a few rows,
// however long the cache is; compacting in order would move nearly all of it.
//
// What bounds it: HBM where many rows move, else the chain select -> list -> rows.
//   evict_short    rows of sums of up to 8192: one workgroup per request and KV head holds them in LDS, finds the smallest sum that stays by
//                  counting, ranks free slots and moving positions and writes their list.
//   evict_bracket, evict_pick, evict_list   longer ones, cut into segments of 4096 positions.  A sample of 512 sums gives two keys that
//                  the smallest one that stays lies between (but for one row in some ten thousand); the workgroups of the segments count what
//                  lies above and list what lies between, about a fifth; one workgroup per row then searches the lists only
//                  (or, where the sample was wrong, in the whole row) and hands every segment the ranks it begins with; the
//                  segments' workgroups write the list.  (One workgroup for a whole row of 100 000 took 175 us, most of it instructions of one CU.)
//   evict_move     rows of the pools, and the sums and the `kept` entries that go with them.  A slot below E is free, so no row that moves there is
//                  read by another one that moves: any number of workgroups.  The newest rows may overlap their destination, and rows between E and
//                  budget have to leave before: columns of 128 bytes do not depend on each other, so a workgroup takes one
//                  column of all these rows, those that leave first, then the newest in ascending pieces, each read before it is written.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/seer_verify.h"
#include "seer_device.h"
#include "seer_plan.h"
#include "seer_tile.h"

namespace seer {

// (Loops over keys are not unrolled much: these kernels run a few microseconds, and code that is run once has to be fetched first.  With the
// keys in registers and 39 KB of unrolled code the search among 4300 sums took 35 us, 12 of them up to the first digit.)
constexpr int kBins = 2048;
constexpr int kShortThreads = 512, kShortKeys = 8192;    // evict_short: threads, keys in LDS
constexpr int kSegThreads = 256, kSegment = 4096;
constexpr int kPickThreads = 1024, kPickKeys = 32768, kPickSegments = 512;      // evict_pick: keys and segments that LDS holds
constexpr int kSamples = 512, kSampleSlack = 48;         // four standard deviations of a rank among 512 samples are at most 45.3
constexpr int kMoveThreads = 256;
constexpr int kMoveHold = 4;                 // 16-byte chunks a thread of a column holds between read and write
constexpr int kMoveAhead = 4;                // chunks a thread of the other rows has in flight
constexpr int kColumn = 128;                 // bytes of a row that one workgroup takes
constexpr int kMoveRows = 64;                // rows that move per workgroup, about

struct EvictHeader {
    int32_t cut;                             // 0: the request stays as it is
    int32_t n;                               // its length before the call
    int32_t moves, leaving;                  // rows that move to free slots; the first of them, which lie below budget
    uint32_t least;                          // the smallest sum that stays (its key), and how many equal to it stay
    int32_t equal;
    int32_t usable, pad;                     // 0: the request is one of those that the status word reports
};
struct EvictSegment {
    int32_t larger[2];                       // keys above the bracket at positions below `end`, from `end` on
    int32_t listed[2];                       // keys in the bracket, all of them listed: likewise
};
struct EvictRank {
    int32_t holes, movers, ties_left;        // free slots and moving positions in front of a segment; how many more equal sums stay from it on
};

struct EvictArgs {
    unsigned char* k_pages;
    unsigned char* v_pages;                  // nullptr: shared latent
    const int32_t* block_table;
    const int32_t* ctx_len;
    const int32_t* keep_first;               // nullptr: first for every request
    const float* weights;
    int32_t* new_ctx_len;
    float* new_weights;                      // nullptr, weights, or another array
    int32_t* kept;                           // may be nullptr
    int32_t* status;                         // may be nullptr
    EvictHeader* header;                     // [B][Hkv]
    // [B][Hkv][capacity]: where the i-th moving row goes, and, `ahead` further, where it is.  Two lists, since different segments write them: lines of memory that two
    // L2 caches hold parts of cost more than what is in them (64 rows of 65 536 .. 131 072 sums: evict_list 38 us with pairs in one list, 35 so).
    int32_t* moves;
    int64_t ahead;
    EvictSegment* segment;                   // [B][Hkv][segments], longer rows only, as the two below
    EvictRank* rank;                         // [B][Hkv][segments]
    uint2* bound;                            // [B][Hkv] the bracket
    uint32_t* list;                          // [B][Hkv][segments][kSegment]
    int64_t ldw, capacity;
    int B, Hkv, P, num_pages, max_pages, max_ctx, segments;
    int limit, budget, first, last;
    int k_chunks, v_chunks;                  // 16-byte chunks of a row
    uint32_t inv_p;                          // floor(2^32 / P), see divide()
    int columns, wgs;                        // workgroups of evict_move per request and KV head: columns (the sums' is the last), then rows
};

// Sums in ascending order as whole numbers above 0; a NaN comes before everything.
__device__ __forceinline__ uint32_t sum_key(float w) { return w != w ? 1u : ordered(w); }
__device__ __forceinline__ uint64_t first_bits(int count) { return count >= kWave ? ~0ull : count <= 0 ? 0ull : (1ull << count) - 1; }
// Sum of the values that the waves in front of this one left in `v`, and of all.
template <int WAVES>
__device__ __forceinline__ int2 before_and_all(const int* v, int wave) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1), mine = lane < WAVES ? v[lane] : 0, incl = wave_incl_scan(mine);
    return make_int2(__builtin_amdgcn_readlane(incl, wave) - __builtin_amdgcn_readlane(mine, wave), last_lane(incl));
}

// A request as the kernels see it: candidates first .. stop - 1, of which `slots` stay, below `end` in the end.
struct EvictRequest {
    int n, first, end, stop, slots;
    int bad;                                 // status bit of what is wrong with its numbers
    bool cut;
};
__device__ __forceinline__ EvictRequest evict_request(const EvictArgs& a, int b) {
    EvictRequest q{};
    q.n = a.ctx_len[b], q.first = a.keep_first ? a.keep_first[b] : a.first;
    q.bad = q.n < 0 || q.n > a.max_ctx ? 1 : 0;
    q.cut = !q.bad && q.n > a.limit;
    q.end = a.budget - a.last, q.stop = q.n - a.last;
    if (q.cut && (q.first < 0 || q.first > q.end)) q.bad = 4, q.cut = false;
    q.slots = q.end - q.first;
    return q;
}
// Rows are moved only where every page that a position from the first one on lies in is known to be in the pool (whole workgroup).
__device__ __forceinline__ bool pages_ok(const EvictArgs& a, int b, const EvictRequest& q, int threads) {
    const int32_t* table = a.block_table + static_cast<size_t>(b) * a.max_pages;
    bool wrong = false;
    const int last_page = divide(q.n - 1, a.P, a.inv_p);
#pragma unroll 4
    for (int l = divide(q.first, a.P, a.inv_p) + static_cast<int>(threadIdx.x); l <= last_page; l += threads) wrong |= table[l] < 0 || table[l] >= a.num_pages;
    return !__syncthreads_or(wrong);
}

// Keys of the `count` positions from `begin` on.
template <int THREADS>
__device__ __forceinline__ uint2 load_keys(uint32_t* s_key, const float* w, int begin, int count) {       // (the thread's smallest and largest)
    uint2 range = make_uint2(0xffffffffu, 0u);
    for (int i0 = threadIdx.x; i0 < count; i0 += 16 * THREADS) {
        float v[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) v[x] = w[begin + min(i0 + x * THREADS, count - 1)];
#pragma unroll
        for (int x = 0; x < 16; ++x)
            if (i0 + x * THREADS < count) {
                const uint32_t k = sum_key(v[x]);
                s_key[i0 + x * THREADS] = k;
                range.x = min(range.x, k), range.y = max(range.y, k);
            }
    }
    return range;
}

// Exclusive prefix of v over the threads of a workgroup.
template <int THREADS>
__device__ __forceinline__ int block_before(int v, int* s_wave, int wave) {
    const int incl = wave_incl_scan(v);
    if ((static_cast<int>(threadIdx.x) & (kWave - 1)) == kWave - 1) s_wave[wave] = incl;
    __syncthreads();
    return before_and_all<THREADS / kWave>(s_wave, wave).x + incl - v;
}

// One digit of the search for the want-th largest key (THREADS * PER bins in LDS, counted): the bin it lies in and its rank in there.
template <int THREADS>
__device__ __forceinline__ void pick_bin(const int* s_bins, int* s_wave, int* s_pick, int wave, int want) {
    constexpr int kPer = kBins / THREADS, kWaves = THREADS / kWave;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), high = kBins - 1 - kPer * tid;      // a thread's bins: high, high - 1, ..
    int count[kPer], sum = 0;
#pragma unroll
    for (int x = 0; x < kPer; ++x) count[x] = s_bins[high - x], sum += count[x];
    const int incl = wave_incl_scan(sum);
    if (lane == kWave - 1) s_wave[wave] = incl;
    __syncthreads();
    int above = before_and_all<kWaves>(s_wave, wave).x + incl - sum;
#pragma unroll
    for (int x = 0; x < kPer; ++x) {
        if (above < want && want <= above + count[x]) s_pick[0] = high - x, s_pick[1] = want - above, s_pick[2] = count[x];
        above += count[x];
    }
    __syncthreads();
}
// The want-th largest of the keys in low .. high that every(use) hands to `use` (1 <= want <= their number), and its rank among equals: they are counted in
// equal parts of that range (the first digit of a key would put most of them into a few bins, whose counters then take them one by one), the part
// it lies in becomes the range, until a thread for each key is enough to rank them by counting.
template <int THREADS, class Every>
__device__ __forceinline__ int2 nth_key(int* s_bins, int* s_wave, int* s_pick, int wave, int want, uint32_t low, uint32_t high, Every&& every) {
    const int tid = threadIdx.x;
    for (;;) {
        const int shift = max(0, 21 - __builtin_clz((high - low) | 1u));                  // (high - low) >> shift < kBins
        for (int i = tid; i < kBins; i += THREADS) s_bins[i] = 0;
        __syncthreads();
        every([&](uint32_t k) __attribute__((always_inline)) {
            if (k >= low && k <= high) atomicAdd(&s_bins[(k - low) >> shift], 1);
        });
        __syncthreads();
        pick_bin<THREADS>(s_bins, s_wave, s_pick, wave, want);
        low += static_cast<uint32_t>(s_pick[0]) << shift;
        high = min(high, low + ((1u << shift) - 1));
        want = s_pick[1];
        const int there = s_pick[2];                        // keys of the part
        if (shift == 0) return make_int2(static_cast<int>(low), want);
        if (there > THREADS) continue;
        __syncthreads();                                    // (the bins and the pick have been read)
        if (tid == 0) s_pick[2] = 0;
        __syncthreads();
        every([&](uint32_t k) __attribute__((always_inline)) {
            if (k >= low && k <= high) s_bins[atomicAdd(&s_pick[2], 1)] = static_cast<int>(k);
        });
        __syncthreads();
        if (tid < there) {
            const uint32_t mine = static_cast<uint32_t>(s_bins[tid]);
            int above = 0, same = 0;
#pragma unroll 4
            for (int i = 0; i < there; ++i) {
                const uint32_t k = static_cast<uint32_t>(s_bins[i]);
                above += k > mine ? 1 : 0, same += k == mine ? 1 : 0;
            }
            if (above < want && want <= above + same) s_pick[0] = static_cast<int>(mine), s_pick[1] = want - above;     // (equal ones write the same)
        }
        __syncthreads();
        return make_int2(s_pick[0], s_pick[1]);
    }
}

// The positions of one workgroup, begin .. begin + count - 1, from their keys: appends free slots and moving positions to the request's list from the given
// ranks on and writes what stays in place to kept and new_weights.  Every thread takes an odd number of consecutive keys (no bank conflicts).
// Returns, by thread, how many positions it has moving and how many of those lie below budget.
template <int THREADS>
__device__ __forceinline__ int2 list_positions(const EvictArgs& a, size_t bh, const EvictRequest& q, uint32_t* s_key, int begin, int count, uint32_t least,
                                               EvictRank from, int (*s_wave)[THREADS / kWave], int wave) {
    const int tid = threadIdx.x, per = ((count + THREADS - 1) / THREADS) | 1, i0 = min(tid * per, count), i1 = min(i0 + per, count);
    const int below = min(max(q.end - begin, 0), count);    // keys of positions below `end`
    int larger_below = 0, larger = 0, equal_below = 0, equal = 0;
#pragma unroll 4
    for (int i = i0; i < i1; ++i) {
        const uint32_t k = s_key[i];
        const int gt = k > least ? 1 : 0, tie = k == least ? 1 : 0;
        larger += gt, equal += tie;
        larger_below += i < below ? gt : 0, equal_below += i < below ? tie : 0;
    }
    int ties_left = max(0, from.ties_left - block_before<THREADS>(equal, s_wave[0], wave));
    const int ties_below = min(ties_left, equal_below), ties_above = min(ties_left - ties_below, equal - equal_below);
    const int my_holes = max(0, min(i1, below) - i0) - larger_below - ties_below, my_movers = larger - larger_below + ties_above;
    int hole = from.holes + block_before<THREADS>(my_holes, s_wave[1], wave);
    int mover = from.movers + block_before<THREADS>(my_movers, s_wave[2], wave);
    int leaving = 0;
    int32_t* slot = a.moves + bh * a.capacity;
    int32_t* position = slot + a.ahead;
#pragma unroll 4
    for (int i = i0; i < i1; ++i) {
        const uint32_t k = s_key[i];
        const bool stays = k > least || (k == least && ties_left-- > 0);
        const int j = begin + i;
        if (i < below) {
            if (!stays) slot[hole++] = j;
        } else if (stays) {
            position[mover++] = j;
            leaving += j < a.budget ? 1 : 0;
        }
        s_key[i] = stays ? 1u : 0u;
    }
    __syncthreads();
    const float* w = a.weights + bh * a.ldw + begin;
    float* to = a.new_weights && a.new_weights != a.weights ? a.new_weights + bh * a.ldw + begin : nullptr;
    int32_t* kept = a.kept ? a.kept + bh * a.budget + begin : nullptr;
    if (kept)                                               // (every slot: evict_move comes later and writes over the filled ones)
#pragma unroll 4
        for (int i = tid; i < below; i += THREADS) kept[i] = begin + i;
    if (to)
        for (int b0 = tid; b0 < below; b0 += 4 * THREADS) {
            float v[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) v[x] = w[min(b0 + x * THREADS, below - 1)];
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (b0 + x * THREADS < below && s_key[b0 + x * THREADS]) to[b0 + x * THREADS] = v[x];
        }
    return make_int2(my_movers, leaving);
}
// What no search decides: the first positions of a request that is cut, all of one that is not (threads `at`, at + step, ..).
__device__ __forceinline__ void fixed_positions(const EvictArgs& a, size_t bh, bool cut, int first, int n, bool usable, int at, int step) {
    const float* w = a.weights + bh * a.ldw;
    float* to = usable && a.new_weights && a.new_weights != a.weights ? a.new_weights + bh * a.ldw : nullptr;
    int32_t* kept = a.kept ? a.kept + bh * a.budget : nullptr;
    // (unsigned: a position and a stride on top may pass 2^31)
    if (kept)
        for (uint32_t j = at, stop = cut ? first : a.budget; j < stop; j += step) kept[j] = cut ? static_cast<int>(j) : -1;
    if (to)
        for (uint32_t j = at, stop = cut ? first : n; j < stop; j += step) to[j] = w[j];
}

__global__ __launch_bounds__(kShortThreads) void evict_short(EvictArgs a) {
    constexpr int kWaves = kShortThreads / kWave;
    __shared__ uint32_t s_key[kShortKeys], s_range[2];
    __shared__ int s_bins[kBins];
    __shared__ int s_wave[3][kWaves];
    __shared__ int s_pick[3];
    const int b = blockIdx.x / a.Hkv, tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const size_t bh = blockIdx.x;
    EvictRequest q = evict_request(a, b);
    const int count = q.stop - q.first;
    if (tid == 0) s_range[0] = 0xffffffffu, s_range[1] = 0u;
    __syncthreads();
    if (q.cut) {
        uint2 range = load_keys<kShortThreads>(s_key, a.weights + bh * a.ldw, q.first, count);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1)
            range.x = min(range.x, static_cast<uint32_t>(__shfl_xor(static_cast<int>(range.x), o, kWave))),
            range.y = max(range.y, static_cast<uint32_t>(__shfl_xor(static_cast<int>(range.y), o, kWave)));
        if ((tid & (kWave - 1)) == 0) atomicMin(&s_range[0], range.x), atomicMax(&s_range[1], range.y);
        if (!pages_ok(a, b, q, kShortThreads)) q.bad = 2, q.cut = false;
    }
    fixed_positions(a, bh, q.cut, q.first, q.n, !q.bad, tid, kShortThreads);
    if (!q.cut) {
        if (tid == 0) {
            a.header[bh] = EvictHeader{0, q.n, 0, 0, 0, 0, !q.bad, 0};
            if (q.bad && a.status) atomicOr(a.status, q.bad);
        }
        return;
    }
    int2 least = make_int2(-1, 0);                          // (nothing between the two ends stays)
    if (q.slots > 0)
        least = nth_key<kShortThreads>(s_bins, s_wave[0], s_pick, wave, q.slots, s_range[0], s_range[1], [&](auto&& use) __attribute__((always_inline)) {
#pragma unroll 4
            for (int i = tid; i < count; i += kShortThreads) use(s_key[i]);
        });
    __syncthreads();
    if (tid < 2) s_pick[tid] = 0;
    const int2 moved = list_positions<kShortThreads>(a, bh, q, s_key, q.first, count, static_cast<uint32_t>(least.x), EvictRank{0, 0, least.y}, s_wave, wave);
    if (moved.x) atomicAdd(&s_pick[0], moved.x);
    if (moved.y) atomicAdd(&s_pick[1], moved.y);
    __syncthreads();
    if (tid == 0) a.header[bh] = EvictHeader{1, q.n, s_pick[0], s_pick[1], 0, 0, 1, 0};
}

// Longer rows, first step: what of a segment lies above the bracket, and a list of what lies in it (in any order; the keys of positions below
// `end` from the front, the others from the back).
__global__ __launch_bounds__(kSegThreads) void evict_bracket(EvictArgs a) {
    constexpr int kPerLane = kSamples / kWave, kHold = kSegment / kSegThreads;
    __shared__ uint32_t s_bound[2];
    __shared__ int s_count[4];               // larger below `end` and from it on, listed likewise
    __shared__ int s_wave[2][kSegThreads / kWave];
    const size_t bh = blockIdx.x / a.segments;
    const int seg = static_cast<int>(blockIdx.x - bh * a.segments), b = static_cast<int>(bh) / a.Hkv, tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const EvictRequest q = evict_request(a, b);
    const int total = q.stop - q.first;
    if (!q.cut || seg * kSegment >= total) return;          // (before anything is added to `first`: the table's segments from there on may pass 2^31)
    const int begin = q.first + seg * kSegment;
    const float* w = a.weights + bh * a.ldw;
    const int count = min(kSegment, q.stop - begin), below = min(max(q.end - begin, 0), count);
    float v[kHold];
#pragma unroll
    for (int x = 0; x < kHold; ++x) v[x] = w[begin + min(x * kSegThreads + tid, count - 1)];
    if (tid < 4) s_count[tid] = 0;
    if (wave < 2) {                                         // wave 0: the lower bound, wave 1: the upper
        uint32_t sample[kPerLane];
#pragma unroll
        for (int x = 0; x < kPerLane; ++x)
            sample[x] = sum_key(w[q.first + static_cast<int>((2ll * (x * kWave + lane) + 1) * total / (2 * kSamples))]);
        // a key that at least `rank` samples reach, good to its upper 20 bits
        const int rank = static_cast<int>(static_cast<int64_t>(q.slots) * kSamples / total) + (wave == 0 ? kSampleSlack : -kSampleSlack);
        uint32_t at = 0;
        for (int bit = 31; bit >= 12; --bit) {
            const uint32_t probe = at | 1u << bit;
            int reach = 0;
#pragma unroll
            for (int x = 0; x < kPerLane; ++x) reach += __popcll(__ballot(sample[x] >= probe));
            if (reach >= rank) at = probe;
        }
        if (lane == 0) s_bound[wave] = wave == 0 ? (rank >= kSamples ? 1u : max(1u, at)) : (rank < 1 ? 0xffffffffu : at | 0xfffu);
    }
    __syncthreads();
    const uint32_t low = s_bound[0], high = s_bound[1];
    if (seg == 0 && tid == 0) a.bound[bh] = make_uint2(low, high);
    uint32_t* list = a.list + (bh * a.segments + seg) * kSegment;
    int larger[2] = {0, 0}, listed[2] = {0, 0};
#pragma unroll
    for (int x = 0; x < kHold; ++x) {
        const int i = x * kSegThreads + tid;
        const uint32_t k = i < count ? sum_key(v[x]) : 0u;
        const int gt = k > high ? 1 : 0, in = k >= low && k <= high ? 1 : 0;
        larger[0] += i < below ? gt : 0, larger[1] += i < below ? 0 : gt;
        listed[0] += i < below ? in : 0, listed[1] += i < below ? 0 : in;
    }
    int at = block_before<kSegThreads>(listed[0], s_wave[0], wave), behind = kSegment - 1 - block_before<kSegThreads>(listed[1], s_wave[1], wave);
    if (tid == kSegThreads - 1) s_count[2] = at + listed[0], s_count[3] = kSegment - 1 - behind + listed[1];
#pragma unroll
    for (int x = 0; x < kHold; ++x) {
        const int i = x * kSegThreads + tid;
        const uint32_t k = i < count ? sum_key(v[x]) : 0u;
        if (k >= low && k <= high) list[i < below ? at++ : behind--] = k;
    }
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const int sum = last_lane(wave_incl_scan(larger[side]));
        if (lane == 0 && sum) atomicAdd(&s_count[side], sum);
    }
    __syncthreads();
    if (tid == 0) a.segment[bh * a.segments + seg] = EvictSegment{{s_count[0], s_count[1]}, {s_count[2], s_count[3]}};
}

// Second step: the smallest sum that stays, and the ranks that every segment begins with.
__global__ __launch_bounds__(kPickThreads) void evict_pick(EvictArgs a) {
    constexpr int kWaves = kPickThreads / kWave;
    __shared__ int s_bins[kBins];
    __shared__ int s_wave[kWaves];
    __shared__ int s_pick[3];
    __shared__ uint32_t s_key[kPickKeys];
    __shared__ int s_at[kPickSegments];
    const int b = blockIdx.x / a.Hkv, tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const size_t bh = blockIdx.x;
    EvictRequest q = evict_request(a, b);
    if (q.cut && !pages_ok(a, b, q, kPickThreads)) q.bad = 2, q.cut = false;
    if (!q.cut) {
        if (tid == 0) {
            a.header[bh] = EvictHeader{0, q.n, 0, 0, 0, 0, !q.bad, 0};
            if (q.bad && a.status) atomicOr(a.status, q.bad);
        }
        return;
    }
    const int total = q.stop - q.first, segments = (total + kSegment - 1) / kSegment;
    const EvictSegment* segment = a.segment + bh * a.segments;
    EvictRank* rank = a.rank + bh * a.segments;
    const uint32_t* list = a.list + bh * a.segments * kSegment;
    const float* w = a.weights + bh * a.ldw;

    int larger = 0, listed = 0;
    for (int s = tid; s < segments; s += kPickThreads) larger += segment[s].larger[0] + segment[s].larger[1], listed += segment[s].listed[0] + segment[s].listed[1];
    larger = last_lane(wave_incl_scan(larger)), listed = last_lane(wave_incl_scan(listed));
    if (lane == 0) s_wave[wave] = larger;
    __syncthreads();
    larger = before_and_all<kWaves>(s_wave, 0).y;
    __syncthreads();
    if (lane == 0) s_wave[wave] = listed;
    __syncthreads();
    listed = before_and_all<kWaves>(s_wave, 0).y;
    __syncthreads();
    const int want = q.slots - larger;
    const bool bracketed = want >= 1 && want <= listed;     // (else the whole row is gone through)
    const bool held = bracketed && listed <= kPickKeys && segments <= kPickSegments;      // the lists in LDS, one behind the other
    if (held) {
        for (int s0 = 0; s0 < segments; s0 += kPickThreads) {                              // (once: kPickSegments of them at most)
            const int s = s0 + tid, mine = s < segments ? segment[s].listed[0] + segment[s].listed[1] : 0;
            const int before = block_before<kPickThreads>(mine, s_wave, wave);
            if (s < segments) s_at[s] = before;
        }
        __syncthreads();
        for (int s = wave; s < segments; s += kWaves) {
            const int below = segment[s].listed[0], count = below + segment[s].listed[1], to = s_at[s];
            for (int i0 = lane; i0 < count; i0 += 8 * kWave) {
                uint32_t k[8];
#pragma unroll
                for (int x = 0; x < 8; ++x) {
                    const int i = min(i0 + x * kWave, count - 1);
                    k[x] = list[static_cast<size_t>(s) * kSegment + (i < below ? i : kSegment - 1 - (i - below))];
                }
#pragma unroll
                for (int x = 0; x < 8; ++x)
                    if (i0 + x * kWave < count) s_key[to + i0 + x * kWave] = k[x];
            }
        }
        __syncthreads();
    }
    int2 least = make_int2(-1, 0);
    // keys(segment, use): use(its keys in the bracket, or all of them, 0: none, their number below `end`), 64 at a time
    auto keys = [&](int s, auto&& use) __attribute__((always_inline)) {
        const int from = q.first + s * kSegment;
        const int below = bracketed ? segment[s].listed[0] : max(0, min(q.end, min(q.stop, from + kSegment)) - from);
        const int count = bracketed ? below + segment[s].listed[1] : min(kSegment, q.stop - from);
        if (held) {
            const int at = s_at[s];
            for (int i0 = 0; i0 < count; i0 += kWave) use(i0 + lane < count ? s_key[at + i0 + lane] : 0u, below - i0);
            return;
        }
        for (int i0 = 0; i0 < count; i0 += 4 * kWave) {
            uint32_t k[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int i = min(i0 + x * kWave + lane, count - 1);
                k[x] = bracketed ? list[static_cast<size_t>(s) * kSegment + (i < below ? i : kSegment - 1 - (i - below))] : sum_key(w[from + i]);
            }
            for (int x = 0; x < 4; ++x) use(i0 + x * kWave + lane < count ? (x == 0 ? k[0] : x == 1 ? k[1] : x == 2 ? k[2] : k[3]) : 0u, below - i0 - x * kWave);
        }
    };
    if (q.slots > 0)
        least = nth_key<kPickThreads>(s_bins, s_wave, s_pick, wave, bracketed ? want : q.slots, bracketed ? a.bound[bh].x : 1u, bracketed ? a.bound[bh].y : 0xffffffffu, [&](auto&& use) __attribute__((always_inline)) {
            if (held) {
#pragma unroll 4
                for (int i = tid; i < listed; i += kPickThreads) use(s_key[i]);
            } else {
                for (int s = wave; s < segments; s += kWaves) keys(s, [&](uint32_t k, int) __attribute__((always_inline)) { use(k); });
            }
        });
    // counts of every segment, in the place of its ranks first: free slots without the equal sums, moving positions likewise, equal sums
    // below `end` in the lower half of ties_left's bits, from `end` on in the upper
    const uint32_t key = static_cast<uint32_t>(least.x);
    for (int s = wave; s < segments; s += kWaves) {
        int gt[2] = {0, 0}, tie[2] = {0, 0};
        if (bracketed) gt[0] = segment[s].larger[0], gt[1] = segment[s].larger[1];
        keys(s, [&](uint32_t k, int below_here) __attribute__((always_inline)) {
            const uint64_t above = __ballot(k > key), same = __ballot(k == key), below = first_bits(below_here);
            gt[0] += __popcll(above & below), gt[1] += __popcll(above & ~below);
            tie[0] += __popcll(same & below), tie[1] += __popcll(same & ~below);
        });
        const int from = q.first + s * kSegment, below = max(0, min(q.end, min(q.stop, from + kSegment)) - from);
        if (lane == 0) rank[s] = EvictRank{below - gt[0], gt[1], tie[0] | tie[1] << 16};
    }
    __syncthreads();
    if (wave) return;
    EvictRank before{0, 0, least.y};
    for (int s0 = 0; s0 < segments; s0 += kWave) {
        const bool in = s0 + lane < segments;
        EvictRank c = in ? rank[s0 + lane] : EvictRank{0, 0, 0};
        const int tie[2] = {c.ties_left & 0xffff, c.ties_left >> 16}, all = tie[0] + tie[1];
        const int ties = wave_incl_scan(all), left = max(0, before.ties_left - (ties - all));
        const int stay_below = min(left, tie[0]), stay_above = min(left - stay_below, tie[1]);
        const int holes = c.holes - stay_below, movers = c.movers + stay_above;
        const int holes_incl = wave_incl_scan(holes), movers_incl = wave_incl_scan(movers);
        if (in) rank[s0 + lane] = EvictRank{before.holes + holes_incl - holes, before.movers + movers_incl - movers, left};
        before.holes += last_lane(holes_incl), before.movers += last_lane(movers_incl);
        before.ties_left = max(0, before.ties_left - last_lane(ties));
    }
    if (lane == 0) a.header[bh] = EvictHeader{1, q.n, before.movers, 0, key, least.y, 1, 0};
}

// Third step: the segments' parts of the list.
__global__ __launch_bounds__(kSegThreads) void evict_list(EvictArgs a) {
    __shared__ uint32_t s_key[kSegment];
    __shared__ int s_wave[3][kSegThreads / kWave];
    const size_t bh = blockIdx.x / a.segments;
    const int seg = static_cast<int>(blockIdx.x - bh * a.segments), b = static_cast<int>(bh) / a.Hkv, tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const EvictRequest q = evict_request(a, b);
    const int count = q.cut ? min(kSegment, q.stop - q.first - seg * kSegment) : 0, begin = count > 0 ? q.first + seg * kSegment : 0;
    if (count > 0) load_keys<kSegThreads>(s_key, a.weights + bh * a.ldw, begin, count);
    const EvictHeader h = a.header[bh];
    fixed_positions(a, bh, h.cut, q.first, q.n, h.usable, seg * kSegThreads + tid, a.segments * kSegThreads);
    if (!h.cut || count <= 0) return;
    const EvictRank from = a.rank[bh * a.segments + seg];
    __syncthreads();
    const int2 moved = list_positions<kSegThreads>(a, bh, q, s_key, begin, count, h.least, from, s_wave, wave);
    const int leaving = last_lane(wave_incl_scan(moved.y));
    if ((tid & (kWave - 1)) == 0 && leaving) atomicAdd(&a.header[bh].leaving, leaving);
}

__global__ __launch_bounds__(kMoveThreads) void evict_move(EvictArgs a) {
    const size_t bh = blockIdx.x / a.wgs;
    const int part = static_cast<int>(blockIdx.x - bh * a.wgs), b = static_cast<int>(bh) / a.Hkv, kvh = static_cast<int>(bh) - b * a.Hkv, tid = threadIdx.x;
    const EvictHeader h = a.header[bh];
    if (kvh == 0 && part == 0 && tid == 0) a.new_ctx_len[b] = h.cut ? a.budget : h.n;
    if (!h.cut) return;
    const int32_t* __restrict__ table = a.block_table + static_cast<size_t>(b) * a.max_pages;
    const int32_t* __restrict__ slots = a.moves + bh * a.capacity;
    const int32_t* __restrict__ positions = slots + a.ahead;
    const float* w = a.weights + bh * a.ldw;
    float* new_w = a.new_weights ? a.new_weights + bh * a.ldw : nullptr;
    int32_t* kept = a.kept ? a.kept + bh * a.budget : nullptr;
    auto row_of = [&](int pos) __attribute__((always_inline)) {
        const int page = divide(pos, a.P, a.inv_p);
        return (static_cast<size_t>(table[page]) * a.Hkv + kvh) * a.P + (pos - page * a.P);
    };
    const int end = a.budget - a.last;
    if (part < a.columns) {
        // the rows that leave the slots from `end` on, then the newest ones (row i: slot, position)
        const int count = h.leaving + a.last;
        auto row = [&](int i) __attribute__((always_inline)) {
            return i < h.leaving ? make_int2(slots[i], positions[i]) : make_int2(end + i - h.leaving, h.n - count + i);
        };
        if (part == a.columns - 1) {                        // their sums
            for (int i0 = 0; i0 < count; i0 += kMoveThreads) {
                const int2 m = row(min(i0 + tid, count - 1));
                const float v = new_w ? w[m.y] : 0.f;
                wait_vmcnt<0>();
                __syncthreads();
                if (i0 + tid < count) {
                    if (new_w) new_w[m.x] = v;
                    if (kept) kept[m.x] = m.y;
                }
                __syncthreads();
            }
            return;
        }
        constexpr int kLanes = kColumn / 16, kRows = kMoveThreads / kLanes;
        const int k_columns = (a.k_chunks + kLanes - 1) / kLanes;
        const bool is_k = part < k_columns;
        const int chunk = (is_k ? part : part - k_columns) * kLanes + (tid & (kLanes - 1)), chunks = is_k ? a.k_chunks : a.v_chunks;
        const bool ok = chunk < chunks;
        u32x4* base = reinterpret_cast<u32x4*>(is_k ? a.k_pages : a.v_pages) + (ok ? chunk : 0);
        for (int i0 = 0; i0 < count; i0 += kRows * kMoveHold) {
            int2 m[kMoveHold];
            u32x4* from[kMoveHold];
            u32x4* to[kMoveHold];
            u32x4 hold[kMoveHold];
#pragma unroll
            for (int x = 0; x < kMoveHold; ++x) m[x] = row(min(i0 + x * kRows + tid / kLanes, count - 1));
#pragma unroll
            for (int x = 0; x < kMoveHold; ++x) from[x] = base + row_of(m[x].y) * chunks, to[x] = base + row_of(m[x].x) * chunks;
#pragma unroll
            for (int x = 0; x < kMoveHold; ++x) hold[x] = *from[x];
            wait_vmcnt<0>();
            __syncthreads();                                // everything has been read
#pragma unroll
            for (int x = 0; x < kMoveHold; ++x)
                if (ok && i0 + x * kRows + tid / kLanes < count) *to[x] = hold[x];
            __syncthreads();
        }
        return;
    }
    // the other rows: chunks of K, then of V; what a thread reads it requests in stages (list, table, rows), kMoveAhead chunks at a time
    const int per_row = a.k_chunks + a.v_chunks, threads = (a.wgs - a.columns) * kMoveThreads;
    const int64_t total = static_cast<int64_t>(h.moves - h.leaving) * per_row;
    for (int64_t x0 = static_cast<int64_t>(part - a.columns) * kMoveThreads + tid; x0 < total; x0 += static_cast<int64_t>(threads) * kMoveAhead) {
        int2 m[kMoveAhead];
        int c[kMoveAhead];
        u32x4* from[kMoveAhead];
        u32x4* to[kMoveAhead];
        u32x4 hold[kMoveAhead];
#pragma unroll
        for (int x = 0; x < kMoveAhead; ++x) {              // (behind the end: the last chunk again, not written)
            const int64_t at = min(x0 + static_cast<int64_t>(x) * threads, total - 1);
            const int i = static_cast<int>(at / per_row);
            c[x] = static_cast<int>(at - static_cast<int64_t>(i) * per_row);
            m[x] = make_int2(slots[h.leaving + i], positions[h.leaving + i]);
        }
#pragma unroll
        for (int x = 0; x < kMoveAhead; ++x) {
            const bool is_k = c[x] < a.k_chunks;
            u32x4* base = reinterpret_cast<u32x4*>(is_k ? a.k_pages : a.v_pages);
            const size_t chunks = is_k ? a.k_chunks : a.v_chunks, at = is_k ? c[x] : c[x] - a.k_chunks;
            from[x] = base + row_of(m[x].y) * chunks + at, to[x] = base + row_of(m[x].x) * chunks + at;
        }
#pragma unroll
        for (int x = 0; x < kMoveAhead; ++x) hold[x] = *from[x];
#pragma unroll
        for (int x = 0; x < kMoveAhead; ++x)
            if (x0 + static_cast<int64_t>(x) * threads < total) {
                *to[x] = hold[x];
                if (c[x] == 0) {
                    if (new_w) new_w[m[x].x] = w[m[x].y];
                    if (kept) kept[m[x].x] = m[x].y;
                }
            }
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
inline int evict_columns(int chunks) { return (chunks * 16 + kColumn - 1) / kColumn; }

static int check_evict_params(const seer_attn_params* p, const seer_evict_params* e) {
    if (!p || !e) return SEER_EINVAL;
    if (p->B < 0 || p->num_pages < 1 || p->max_pages_per_seq < 1 || p->page_size < 1) return SEER_EINVAL;
    const bool shared = p->kv_shared_latent != 0;
    if (p->Hkv < 1 || p->Dqk < 1 || p->Dqk % 8 != 0 || (!shared && (p->Dv < 1 || p->Dv % 8 != 0))) return SEER_ESHAPE;      // rows move in 16-byte chunks
    if (e->budget < 1 || e->limit < e->budget || e->keep_first < 0 || e->keep_last < 0) return SEER_EINVAL;
    if (static_cast<int64_t>(e->keep_first) + e->keep_last > e->budget) return SEER_ESHAPE;
    const int64_t ctx = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size;
    if (ctx > 0x7fffffffLL - 4096 || p->Dqk > 1 << 16 || p->Dv > 1 << 16) return SEER_ESHAPE;
    // launches count their threads in 32 bits: up to one workgroup per segment, or per column (and the sums', and one for the other rows, 8192 on top)
    const int64_t heads = static_cast<int64_t>(p->B) * p->Hkv, columns = e->keep_last > 0 ? evict_columns(p->Dqk / 8) + evict_columns(shared ? 0 : p->Dv / 8) + 1 : 0;
    const int64_t most = 0xffffffffLL / 256 - 8192;
    if (heads > 0x7fffffffLL / 4096 || heads > most / (ctx / kSegment + 1) || heads > most / (columns + 1)) return SEER_ESHAPE;
    return SEER_OK;
}
// Rows of one request and KV head that can move to free slots, at most.
inline int64_t evict_capacity(const seer_attn_params& p, const seer_evict_params& e) {
    const int64_t end = e.budget - e.keep_last, ctx = static_cast<int64_t>(p.max_pages_per_seq) * p.page_size;
    const int64_t most = ctx - e.keep_last - end;
    return most < 0 ? 0 : (most < end ? most : end);
}
struct EvictLayout {
    int segments;                            // of longer rows; 0: evict_short
    size_t off_moves, off_segment, off_rank, off_bound, off_list, total;
};
inline EvictLayout evict_layout(const seer_attn_params& p, const seer_evict_params& e) {
    EvictLayout w{};
    const size_t heads = static_cast<size_t>(p.B) * p.Hkv;
    const int64_t ctx = static_cast<int64_t>(p.max_pages_per_seq) * p.page_size;      // (what the host knows of the lengths)
    w.segments = ctx <= kShortKeys ? 0 : static_cast<int>((ctx + kSegment - 1) / kSegment);
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    w.off_moves = up(sizeof(EvictHeader) * heads);
    w.off_segment = w.off_moves + 2 * up(sizeof(int32_t) * static_cast<size_t>(evict_capacity(p, e)) * heads);
    w.off_rank = w.off_segment + up(sizeof(EvictSegment) * w.segments * heads);
    w.off_bound = w.off_rank + up(sizeof(EvictRank) * w.segments * heads);
    w.off_list = w.off_bound + (w.segments ? up(sizeof(uint2) * heads) : 0);
    w.total = w.off_list + up(sizeof(uint32_t) * kSegment * static_cast<size_t>(w.segments) * heads);
    return w;
}

}  // namespace seer

extern "C" size_t seer_kv_evict_workspace(const seer_attn_params* p, const seer_evict_params* e) {
    if (seer::check_evict_params(p, e) != SEER_OK || p->B == 0) return 0;
    return seer::evict_layout(*p, *e).total;
}

extern "C" int seer_kv_evict(const seer_attn_params* p, const seer_evict_params* e, void* k_pages, void* v_pages, const int32_t* block_table,
                             const int32_t* ctx_len, const int32_t* keep_first, const float* weights, int32_t* new_ctx_len,
                             float* new_weights, int32_t* kept, int32_t* status, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = seer::check_evict_params(p, e);
    if (rc != SEER_OK) return rc;
    if (p->B == 0) return SEER_OK;
    const bool shared = p->kv_shared_latent != 0;
    if (!k_pages || shared != !v_pages || !block_table || !ctx_len || !weights || !new_ctx_len) return SEER_EINVAL;
    const seer::EvictLayout layout = seer::evict_layout(*p, *e);
    if (!workspace || workspace_bytes < layout.total) return SEER_EWORKSPACE;
    auto misaligned = [](const void* ptr, uintptr_t a) { return reinterpret_cast<uintptr_t>(ptr) % a != 0; };
    if (misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(workspace, 16) || misaligned(weights, 4) || misaligned(new_weights, 4) ||
        misaligned(block_table, 4) || misaligned(ctx_len, 4) || misaligned(keep_first, 4) || misaligned(new_ctx_len, 4) || misaligned(kept, 4) || misaligned(status, 4))
        return SEER_EALIGN;
    seer::EvictArgs a{};
    a.k_pages = static_cast<unsigned char*>(k_pages), a.v_pages = static_cast<unsigned char*>(v_pages);
    a.block_table = block_table, a.ctx_len = ctx_len, a.keep_first = keep_first, a.weights = weights;
    a.new_ctx_len = new_ctx_len, a.new_weights = new_weights, a.kept = kept, a.status = status;
    char* ws = static_cast<char*>(workspace);
    a.header = reinterpret_cast<seer::EvictHeader*>(ws);
    a.moves = reinterpret_cast<int32_t*>(ws + layout.off_moves);
    a.ahead = static_cast<int64_t>((layout.off_segment - layout.off_moves) / 2 / sizeof(int32_t));
    a.segment = reinterpret_cast<seer::EvictSegment*>(ws + layout.off_segment);
    a.rank = reinterpret_cast<seer::EvictRank*>(ws + layout.off_rank);
    a.bound = reinterpret_cast<uint2*>(ws + layout.off_bound);
    a.list = reinterpret_cast<uint32_t*>(ws + layout.off_list);
    a.segments = layout.segments;
    a.ldw = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size, a.capacity = seer::evict_capacity(*p, *e);
    a.B = p->B, a.Hkv = p->Hkv, a.P = p->page_size, a.num_pages = p->num_pages, a.max_pages = p->max_pages_per_seq;
    a.max_ctx = static_cast<int>(a.ldw);
    a.inv_p = p->page_size > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / static_cast<uint32_t>(p->page_size)) : 0xffffffffu;
    a.limit = e->limit, a.budget = e->budget, a.first = e->keep_first, a.last = e->keep_last;
    a.k_chunks = p->Dqk / 8, a.v_chunks = shared ? 0 : p->Dv / 8;
    a.columns = e->keep_last > 0 ? seer::evict_columns(a.k_chunks) + seer::evict_columns(a.v_chunks) + 1 : 0;
    // workgroups for the other rows: one per 64 that may move, as long as the launch is no larger than the chip can use
    const int64_t heads = static_cast<int64_t>(p->B) * p->Hkv, most = (8192 + heads - 1) / heads;
    int64_t rows = (a.capacity + seer::kMoveRows - 1) / seer::kMoveRows;
    if (rows > most) rows = most;
    if (rows < 1) rows = 1;
    a.wgs = a.columns + static_cast<int>(rows);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const unsigned rows_of_sums = static_cast<unsigned>(heads);
    if (a.segments == 0) {
        hipLaunchKernelGGL(seer::evict_short, dim3(rows_of_sums), dim3(seer::kShortThreads), 0, stream, a);
    } else {
        const dim3 grid(rows_of_sums * static_cast<unsigned>(a.segments));
        hipLaunchKernelGGL(seer::evict_bracket, grid, dim3(seer::kSegThreads), 0, stream, a);
        hipLaunchKernelGGL(seer::evict_pick, dim3(rows_of_sums), dim3(seer::kPickThreads), 0, stream, a);
        hipLaunchKernelGGL(seer::evict_list, grid, dim3(seer::kSegThreads), 0, stream, a);
    }
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return static_cast<int>(err);
    hipLaunchKernelGGL(seer::evict_move, dim3(static_cast<unsigned>(heads * a.wgs)), dim3(seer::kMoveThreads), 0, stream, a);
    err = hipGetLastError();
    return err == hipSuccess ? SEER_OK : static_cast<int>(err);
}
