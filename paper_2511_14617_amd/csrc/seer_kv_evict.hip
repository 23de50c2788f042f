// seer_kv_evict: requests whose cache has grown over a limit keep `budget` positions per KV head: the first ones, the newest ones,
// and of those between the ones with the largest sums of attention weight.
//
// Attention does not depend on the order of the positions that every query sees, so only what would lie behind the new end
// moves: with E = budget - keep_last, the i-th kept position from E on (ascending, the newest aside) goes to the i-th free slot below
// E, and the newest keep_last positions become E .. budget - 1, in order.  A step that drops a few positions so moves a few rows,
// however long the cache is; compacting in order would move nearly all of it.
//
// What bounds it: HBM where many rows move, else the chain select -> lists -> rows.
//   evict_select   one workgroup per request and KV head: the M-th largest sum by three passes of counting digits of 11, 11 and 10 bits (the
//                  sums are read from the L2 after the first), then one ordered pass that ranks equal sums, free slots and moving
//                  positions by ballots; it also moves the sums themselves.
//   evict_move     rows of the pools.  A slot below E is free, so no row that moves there is read by another one that moves: any number of workgroups.  The newest
//                  rows may overlap their destination, and rows between E and budget have to leave before: columns of 128
//                  bytes do not depend on each other, so a workgroup takes one column of all these rows, those that leave
//                  first, then the newest in ascending pieces, each read before it is written.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/seer_verify.h"
#include "seer_device.h"
#include "seer_plan.h"
#include "seer_tile.h"

namespace seer {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / kWave;
constexpr int kSelBins = 2048;
constexpr int kMoveThreads = 256;
constexpr int kMoveHold = 8;                 // 16-byte chunks a thread of a column holds between read and write
constexpr int kColumn = 128;                 // bytes of a row that one workgroup takes
constexpr int kMoveRows = 64;                // rows that move per workgroup, about

struct EvictHeader {
    int32_t cut;                             // 0: the request stays as it is
    int32_t n;                               // its length before the call
    int32_t moves, leaving;                  // rows that move to free slots; the first of them, which lie below budget
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
    int2* moves;                             // [B][Hkv][capacity]: slot, position
    int64_t ldw, capacity;
    int B, Hkv, P, num_pages, max_pages, max_ctx;
    int limit, budget, first, last;
    int k_chunks, v_chunks;                  // 16-byte chunks of a row
    int columns, wgs;                        // workgroups of evict_move per request and KV head: columns, then rows
};

// Sums in ascending order as whole numbers; a NaN comes before everything.
__device__ __forceinline__ uint32_t sum_key(float w) { return w != w ? 0u : ordered(w); }

__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs a) {
    __shared__ int s_bins[kSelBins];
    __shared__ int s_wave[3][kSelWaves];
    __shared__ int s_pick[2];
    const int b = blockIdx.x / a.Hkv, tid = threadIdx.x, lane = tid & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const size_t bh = blockIdx.x;
    const int n = a.ctx_len[b], first = a.keep_first ? a.keep_first[b] : a.first;
    const float* w = a.weights + bh * a.ldw;
    float* to = a.new_weights ? a.new_weights + bh * a.ldw : nullptr;
    const bool in_place = to == w;
    int32_t* kept = a.kept ? a.kept + bh * a.budget : nullptr;

    int bad = n < 0 || n > a.max_ctx ? 1 : 0;
    bool cut = !bad && n > a.limit;
    if (cut && (first < 0 || first > a.budget - a.last)) bad = 4, cut = false;
    if (cut) {                                              // rows are moved only where every page is known to lie in the pool
        const int32_t* table = a.block_table + static_cast<size_t>(b) * a.max_pages;
        bool wrong = false;
        for (int l = first / a.P + tid; l <= (n - 1) / a.P; l += kSelThreads) wrong |= table[l] < 0 || table[l] >= a.num_pages;
        if (__syncthreads_or(wrong)) bad = 2, cut = false;
    }
    if (!cut) {
        if (tid == 0) {
            a.header[bh] = EvictHeader{0, n, 0, 0};
            if (bad && a.status) atomicOr(a.status, bad);
        }
        if (kept)
            for (int j = tid; j < a.budget; j += kSelThreads) kept[j] = -1;
        if (!bad && to && !in_place)
            for (int j = tid; j < n; j += kSelThreads) to[j] = w[j];
        return;
    }

    // ---- the smallest sum that stays, and how many of those equal to it -------------------------------------
    const int end = a.budget - a.last;                      // slots of the kept ones below the newest
    const int slots = end - first, stop = n - a.last;       // candidates: first .. stop - 1
    uint32_t least = 0xffffffffu;
    int equal = 0;                                          // how many equal to `least` stay
    if (slots > 0) {
        uint32_t prefix = 0;
        int want = slots;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
            for (int i = tid; i < kSelBins; i += kSelThreads) s_bins[i] = 0;
            __syncthreads();
            for (int j = first + tid; j < stop; j += kSelThreads) {
                const uint32_t k = sum_key(w[j]);
                if (pass == 0 || k >> (shift + bits) == prefix) atomicAdd(&s_bins[(k >> shift) & ((1u << bits) - 1)], 1);
            }
            __syncthreads();
            // thread t: bins kSelBins - 1 - 2 t and the one below
            const int high = s_bins[kSelBins - 1 - 2 * tid], low = s_bins[kSelBins - 2 - 2 * tid];
            const int incl = wave_incl_scan(high + low);
            if (lane == kWave - 1) s_wave[0][wave] = incl;
            __syncthreads();
            int above = incl - high - low;
            for (int x = 0; x < wave; ++x) above += s_wave[0][x];
            if (above < want && want <= above + high + low) {
                const bool in_high = want <= above + high;
                s_pick[0] = kSelBins - 1 - 2 * tid - (in_high ? 0 : 1);
                s_pick[1] = want - above - (in_high ? 0 : high);
            }
            __syncthreads();
            prefix = prefix << bits | static_cast<uint32_t>(s_pick[0]);
            want = s_pick[1];
        }
        least = prefix, equal = want;
    }

    // ---- ranks: every wave takes consecutive positions -----------------------------------------------------
    const int per_wave = ((stop - first + kSelWaves - 1) / kSelWaves + kWave - 1) / kWave * kWave;
    const int begin = min(stop, first + wave * per_wave), finish = min(stop, begin + per_wave);
    const uint64_t below_lane = (1ull << lane) - 1;
    int count = 0;
    for (int j0 = begin; j0 < finish; j0 += kWave) {
        const int j = j0 + lane;
        count += __popcll(__ballot(j < finish && sum_key(w[min(j, finish - 1)]) == least));
    }
    if (lane == 0) s_wave[0][wave] = count;
    __syncthreads();
    int equal_before = 0;
    for (int x = 0; x < wave; ++x) equal_before += s_wave[0][x];
    // walk(use): use(position, stays, free slots before it, moving positions before it) for the wave's positions; the totals come back
    auto walk = [&](int holes, int movers, auto&& use) __attribute__((always_inline)) {
        int ties = equal_before;
        for (int j0 = begin; j0 < finish; j0 += kWave) {
            const int j = j0 + lane;
            const bool in = j < finish;
            const uint32_t k = in ? sum_key(w[j]) : 0u;
            const uint64_t tie = __ballot(in && k == least);
            const bool stays = in && (k > least || (k == least && ties + __popcll(tie & below_lane) < equal));
            const uint64_t hole = __ballot(in && j < end && !stays), mover = __ballot(stays && j >= end);
            use(j, in, stays, holes + __popcll(hole & below_lane), movers + __popcll(mover & below_lane));
            ties += __popcll(tie), holes += __popcll(hole), movers += __popcll(mover);
        }
        return make_int2(holes, movers);
    };
    const int2 mine = walk(0, 0, [](int, bool, bool, int, int) {});
    if (lane == 0) s_wave[1][wave] = mine.x, s_wave[2][wave] = mine.y;
    if (tid == 0) s_pick[0] = 0;
    __syncthreads();
    int holes = 0, movers = 0, all = 0;
    for (int x = 0; x < kSelWaves; ++x) {
        if (x < wave) holes += s_wave[1][x], movers += s_wave[2][x];
        all += s_wave[2][x];
    }
    int2* moves = a.moves + bh * a.capacity;
    int leaving = 0;
    walk(holes, movers, [&](int j, bool in, bool stays, int hole, int mover) __attribute__((always_inline)) {
        if (in && j < end && !stays) moves[hole].x = j;
        if (stays && j >= end) {
            moves[mover].y = j;
            if (j < a.budget) ++leaving;
        }
        if (stays && j < end) {
            if (kept) kept[j] = j;
            if (to && !in_place) to[j] = w[j];
        }
    });
    if (leaving) atomicAdd(&s_pick[0], leaving);
    for (int j = tid; j < first; j += kSelThreads) {
        if (kept) kept[j] = j;
        if (to && !in_place) to[j] = w[j];
    }
    __syncthreads();                                        // (the list is whole)
    if (tid == 0) a.header[bh] = EvictHeader{1, n, all, s_pick[0]};
    for (int i = tid; i < all; i += kSelThreads) {
        const int2 m = moves[i];
        if (kept) kept[m.x] = m.y;
        if (to) to[m.x] = w[m.y];                           // (slots below `end`, positions from `end` on)
    }
    for (int i = tid; i < a.last; i += kSelThreads) {
        if (kept) kept[end + i] = stop + i;
        if (to && !in_place) to[end + i] = w[stop + i];
    }
    if (in_place) {
        __syncthreads();
        for (int i0 = 0; i0 < a.last; i0 += kSelThreads) {
            const int i = i0 + tid;
            const float v = i < a.last ? w[stop + i] : 0.f;
            __syncthreads();
            if (i < a.last) to[end + i] = v;
            __syncthreads();
        }
    }
}

__global__ __launch_bounds__(kMoveThreads) void evict_move(EvictArgs a) {
    const size_t bh = blockIdx.x / a.wgs;
    const int part = static_cast<int>(blockIdx.x - bh * a.wgs), b = static_cast<int>(bh) / a.Hkv, kvh = static_cast<int>(bh) - b * a.Hkv, tid = threadIdx.x;
    const EvictHeader h = a.header[bh];
    if (kvh == 0 && part == 0 && tid == 0) a.new_ctx_len[b] = h.cut ? a.budget : h.n;
    if (!h.cut) return;
    const int32_t* __restrict__ table = a.block_table + static_cast<size_t>(b) * a.max_pages;
    const int2* __restrict__ moves = a.moves + bh * a.capacity;
    const bool page_pow2 = (a.P & (a.P - 1)) == 0;
    const int page_shift = __builtin_ctz(static_cast<unsigned>(a.P));
    auto row_of = [&](int pos) __attribute__((always_inline)) {
        const int page = page_pow2 ? pos >> page_shift : pos / a.P;
        return (static_cast<size_t>(table[page]) * a.Hkv + kvh) * a.P + (pos - page * a.P);
    };
    const int end = a.budget - a.last;
    if (part < a.columns) {
        // one column of the rows that leave the slots from `end` on, then of the newest rows
        constexpr int kLanes = kColumn / 16, kRows = kMoveThreads / kLanes;
        const int k_columns = (a.k_chunks + kLanes - 1) / kLanes;
        const bool is_k = part < k_columns;
        const int chunk = (is_k ? part : part - k_columns) * kLanes + (tid & (kLanes - 1)), chunks = is_k ? a.k_chunks : a.v_chunks;
        u32x4* base = reinterpret_cast<u32x4*>(is_k ? a.k_pages : a.v_pages) + chunk;
        const bool ok = chunk < chunks;
        auto copy = [&](int count, auto&& rows) __attribute__((always_inline)) {       // rows(i): (to, from)
            for (int i0 = 0; i0 < count; i0 += kRows * kMoveHold) {
                u32x4 hold[kMoveHold];
                int to[kMoveHold];
#pragma unroll
                for (int x = 0; x < kMoveHold; ++x) {
                    const int i = i0 + x * kRows + tid / kLanes;
                    to[x] = -1;
                    if (ok && i < count) {
                        const int2 m = rows(i);
                        to[x] = m.x;
                        hold[x] = base[row_of(m.y) * chunks];
                    }
                }
                wait_vmcnt<0>();
                __syncthreads();                            // everything has been read
#pragma unroll
                for (int x = 0; x < kMoveHold; ++x)
                    if (to[x] >= 0) base[row_of(to[x]) * chunks] = hold[x];
                __syncthreads();
            }
        };
        copy(h.leaving, [&](int i) __attribute__((always_inline)) { return moves[i]; });
        copy(a.last, [&](int i) __attribute__((always_inline)) { return make_int2(end + i, h.n - a.last + i); });
        return;
    }
    const int per_row = a.k_chunks + a.v_chunks;
    const int64_t total = static_cast<int64_t>(h.moves - h.leaving) * per_row, stride = static_cast<int64_t>(a.wgs - a.columns) * kMoveThreads;
    u32x4* k = reinterpret_cast<u32x4*>(a.k_pages);
    u32x4* v = reinterpret_cast<u32x4*>(a.v_pages);
#pragma unroll 4
    for (int64_t x = static_cast<int64_t>(part - a.columns) * kMoveThreads + tid; x < total; x += stride) {
        const int i = static_cast<int>(x / per_row), c = static_cast<int>(x - static_cast<int64_t>(i) * per_row);
        const int2 m = moves[h.leaving + i];
        const size_t from = row_of(m.y), to = row_of(m.x);
        if (c < a.k_chunks) k[to * a.k_chunks + c] = k[from * a.k_chunks + c];
        else v[to * a.v_chunks + c - a.k_chunks] = v[from * a.v_chunks + c - a.k_chunks];
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static int check_evict_params(const seer_attn_params* p, const seer_evict_params* e) {
    if (!p || !e) return SEER_EINVAL;
    if (p->B < 0 || p->num_pages < 1 || p->max_pages_per_seq < 1 || p->page_size < 1) return SEER_EINVAL;
    const bool shared = p->kv_shared_latent != 0;
    if (p->Hkv < 1 || p->Dqk < 1 || p->Dqk % 8 != 0 || (!shared && (p->Dv < 1 || p->Dv % 8 != 0))) return SEER_ESHAPE;      // rows move in 16-byte chunks
    if (e->budget < 1 || e->limit < e->budget || e->keep_first < 0 || e->keep_last < 0) return SEER_EINVAL;
    if (static_cast<int64_t>(e->keep_first) + e->keep_last > e->budget) return SEER_ESHAPE;
    const int64_t ctx = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size;
    if (ctx > 0x7fffffffLL - 4096 || p->Dqk > 1 << 16 || p->Dv > 1 << 16) return SEER_ESHAPE;
    if (static_cast<int64_t>(p->B) * p->Hkv > 0x7fffffffLL / 4096) return SEER_ESHAPE;
    return SEER_OK;
}
// Rows of one request and KV head that can move to free slots, at most.
inline int64_t evict_capacity(const seer_attn_params& p, const seer_evict_params& e) {
    const int64_t end = e.budget - e.keep_last, ctx = static_cast<int64_t>(p.max_pages_per_seq) * p.page_size;
    const int64_t most = ctx - e.keep_last - end;
    return most < 0 ? 0 : (most < end ? most : end);
}
inline size_t evict_header_bytes(const seer_attn_params& p) { return (sizeof(EvictHeader) * static_cast<size_t>(p.B) * p.Hkv + 255) / 256 * 256; }

}  // namespace seer

extern "C" size_t seer_kv_evict_workspace(const seer_attn_params* p, const seer_evict_params* e) {
    if (seer::check_evict_params(p, e) != SEER_OK || p->B == 0) return 0;
    const size_t list = sizeof(int2) * static_cast<size_t>(seer::evict_capacity(*p, *e)) * p->B * p->Hkv;
    return seer::evict_header_bytes(*p) + (list + 255) / 256 * 256;
}

extern "C" int seer_kv_evict(const seer_attn_params* p, const seer_evict_params* e, void* k_pages, void* v_pages, const int32_t* block_table,
                             const int32_t* ctx_len, const int32_t* keep_first, const float* weights, int32_t* new_ctx_len,
                             float* new_weights, int32_t* kept, int32_t* status, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = seer::check_evict_params(p, e);
    if (rc != SEER_OK) return rc;
    if (p->B == 0) return SEER_OK;
    const bool shared = p->kv_shared_latent != 0;
    if (!k_pages || shared != !v_pages || !block_table || !ctx_len || !weights || !new_ctx_len) return SEER_EINVAL;
    if (!workspace || workspace_bytes < seer_kv_evict_workspace(p, e)) return SEER_EWORKSPACE;
    auto misaligned = [](const void* ptr, uintptr_t a) { return reinterpret_cast<uintptr_t>(ptr) % a != 0; };
    if (misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(workspace, 16) || misaligned(weights, 4) || misaligned(new_weights, 4) ||
        misaligned(block_table, 4) || misaligned(ctx_len, 4) || misaligned(keep_first, 4) || misaligned(new_ctx_len, 4) || misaligned(kept, 4) || misaligned(status, 4))
        return SEER_EALIGN;
    seer::EvictArgs a{};
    a.k_pages = static_cast<unsigned char*>(k_pages), a.v_pages = static_cast<unsigned char*>(v_pages);
    a.block_table = block_table, a.ctx_len = ctx_len, a.keep_first = keep_first, a.weights = weights;
    a.new_ctx_len = new_ctx_len, a.new_weights = new_weights, a.kept = kept, a.status = status;
    a.header = static_cast<seer::EvictHeader*>(workspace);
    a.moves = reinterpret_cast<int2*>(static_cast<char*>(workspace) + seer::evict_header_bytes(*p));
    a.ldw = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size, a.capacity = seer::evict_capacity(*p, *e);
    a.B = p->B, a.Hkv = p->Hkv, a.P = p->page_size, a.num_pages = p->num_pages, a.max_pages = p->max_pages_per_seq;
    a.max_ctx = static_cast<int>(a.ldw);
    a.limit = e->limit, a.budget = e->budget, a.first = e->keep_first, a.last = e->keep_last;
    a.k_chunks = p->Dqk / 8, a.v_chunks = shared ? 0 : p->Dv / 8;
    auto columns = [](int chunks) { return (chunks * 16 + seer::kColumn - 1) / seer::kColumn; };
    a.columns = e->keep_last > 0 ? columns(a.k_chunks) + columns(a.v_chunks) : 0;
    // workgroups for the other rows: one per 64 that may move, as long as the launch is no larger than the chip can use
    const int64_t heads = static_cast<int64_t>(p->B) * p->Hkv, most = (8192 + heads - 1) / heads;
    int64_t rows = (a.capacity + seer::kMoveRows - 1) / seer::kMoveRows;
    if (rows > most) rows = most;
    if (rows < 1) rows = 1;
    a.wgs = a.columns + static_cast<int>(rows);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipLaunchKernelGGL(seer::evict_select, dim3(static_cast<unsigned>(heads)), dim3(seer::kSelThreads), 0, stream, a);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return static_cast<int>(err);
    hipLaunchKernelGGL(seer::evict_move, dim3(static_cast<unsigned>(heads * a.wgs)), dim3(seer::kMoveThreads), 0, stream, a);
    err = hipGetLastError();
    return err == hipSuccess ? SEER_OK : static_cast<int>(err);
}
