// Work of the prompt attention kernels: how packed tokens of requests of any length are cut into equal shares, on the device.
//
// Rows: a request's n tokens times the G heads that share a KV head are n G consecutive query rows (row r = token r / G, head r % G), cut into
// row tiles of 128 (or 256).  A row tile reads the positions that its last row sees, so its cost grows along a prompt: with past = ctx - n
// cached positions before the new ones, row tile i of a request costs (in units of a position times a head of the group)
//     c_i = G (past + tile_cost) + 128 (i + 1),     i < R = ceil(n G / 128).
// All row tiles -- requests in order, their KV heads in order, their row tiles in order -- lie end to end on one line, whose
// prefix sums have closed forms in i and in the KV head, and whose sums over requests are one scan.  Workgroup w of W takes the stretch from
// x_w = total w / W to x_(w+1): equal work whatever the mix of lengths, one launch, no queue.
// A cut inside a row tile costs two partial results and their joining: one that comes within `snap` of a row tile's end is moved there, and row
// tiles of up to kWholePositions are never cut, their cuts are moved to where they begin.  Stretches are at least 2 `snap` long, or as many as
// there are row tiles, so that calls with little to do use one workgroup a row tile.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/seer_verify.h"
#include "seer_device.h"

namespace seer {

constexpr int kRowTile = 128;          // query rows of a workgroup: 32 of each of its four waves (twice that where it has eight)
constexpr int kPromptThreads = 256, kMostPromptThreads = 512;
// The exponent reference of a row that has seen no finite score: the lowest float, which no finite score is below.  Every difference of references is then a
// number or -inf, and a row that stays without a score asks for no rescaling.
constexpr float kNoScore = -3.402823466e38f;
// Measured with 128 | 256 | 512 positions a stretch: 8 single tokens behind 2048 positions, 8/1 heads, 30.7 | 26.3 | 27.7 us, 16 behind 4096 45.5 | 36.6 | 34.0, one prompt of 900
// 33.4 | 31.2 | 28.9, the 8 single tokens over the latent on 16 heads 44.8 | 43.2 | 54.0; large calls do not notice.  Row tiles left whole up to 128 | 512 | 1024: eight prompts of
// 17 .. 300 tokens 21.7 | 16.8 | 16.9, the single tokens 26.3 | 26.3 | 36.7, over the latent 43.4 | 43.2 | 77.3, 32 prompts of 600 62.1 | 53.4 | 52.9, one of 900 25.3 | 31.2 | 26.7.
constexpr int kMinStretch = 256;       // positions per head of the group
constexpr int kWholePositions = 512;

// The pieces that end a stretch inside a row tile: the row tile, and in how many stretches it lies (0: none begins here and goes on).
struct PromptCut {
    int32_t b, kvh, tile, pieces;
};

struct PromptArgs {
    uint16_t* out;
    const uint16_t* q;
    const unsigned char* k_pages;
    const unsigned char* v_pages;
    const int32_t* block_table;
    const int32_t* ctx_len;
    const int32_t* first;
    int32_t* status;
    PromptCut* cuts;       // [W]
    float* part_ml;        // [2 W][row tile][2]: reference (a raw score), sum
    float* part_acc;       // [2 W][row tile][Dv]: unnormalised output.  Slot 2 w: the row tile that began before stretch w, 2 w + 1: the one that goes on behind it
    int B, Hq, Hkv, G, P, num_pages, max_pages, n_tokens, Dqk, Dv;
    int W;
    int row_shift;         // a row tile has 2^row_shift rows
    int tile_cost;         // what a row tile costs beside its positions, in positions
    uint32_t inv_p, inv_g; // 2^32 / P and 2^32 / G, at most 2^32 - 1
    float scale_log2, move_at;      // scale in units of log2 e; raw scores by which a reference is exceeded before it moves, 8 / scale_log2
    int64_t max_ctx;
};

// x / d from inv = 2^32 / d rounded down (d = 1: 2^32 - 1): the product's upper half is the quotient or one less.
__device__ __forceinline__ uint32_t quotient(uint32_t x, uint32_t d, uint32_t inv) {
    const uint32_t q = __umulhi(x, inv);
    return q + ((d - 1u - (x - q * d)) >> 31);         // (rests of 2 d and more do not occur, so the sign says it)
}
// Page of a position.
__device__ __forceinline__ int prompt_page(const PromptArgs& a, int position) {
    return static_cast<int>(quotient(static_cast<uint32_t>(position), static_cast<uint32_t>(a.P), a.inv_p));
}
// Token of a query row of a request.
__device__ __forceinline__ int prompt_token(const PromptArgs& a, uint32_t row) { return static_cast<int>(quotient(row, static_cast<uint32_t>(a.G), a.inv_g)); }

// A row tile of a workgroup of THREADS has 2^kRowShift rows, half as many.
template <int THREADS>
constexpr int kRowShift = THREADS == kPromptThreads ? 7 : 8;
static_assert(1 << kRowShift<kPromptThreads> == kRowTile && 1 << kRowShift<kMostPromptThreads> == 2 * kRowTile, "");

// A request as the line counts it.
struct PromptRequest {
    int64_t past;          // positions before the new tokens
    int n, tiles, first;   // new tokens, row tiles per KV head (0: nothing to do), first packed token
    bool bad;              // a ctx_len that cannot be: rows of zeros
};

// Tokens of request b; 0 where first_token cannot be.
__device__ __forceinline__ int prompt_tokens(const PromptArgs& a, int b) {
    const int lo = a.first[b], hi = a.first[b + 1];
    return lo >= 0 && hi >= lo && hi <= a.n_tokens ? hi - lo : 0;
}
// before: the sum of prompt_tokens over the requests before b (with a limit to it the line is finite whatever the array holds).
template <int THREADS>
__device__ __forceinline__ PromptRequest prompt_request(const PromptArgs& a, int b, int64_t before, int& error) {
    PromptRequest r{0, 0, 0, 0, false};
    const int lo = a.first[b], hi = a.first[b + 1], ctx = a.ctx_len[b];
    if (lo < 0 || hi < lo || hi > a.n_tokens || before + (hi - lo) > a.n_tokens) {
        error |= 4;
        return r;
    }
    r.n = hi - lo, r.first = lo;
    if (r.n == 0) return r;
    r.bad = ctx < r.n || ctx > a.max_ctx;
    if (r.bad) error |= 1;
    r.past = r.bad ? 0 : ctx - r.n;
    r.tiles = static_cast<int>((static_cast<int64_t>(r.n) * a.G + (1 << kRowShift<THREADS>) - 1) >> kRowShift<THREADS>);
    return r;
}
// Cost of the first i row tiles of a KV head, and of row tile i.
template <int THREADS>
__device__ __forceinline__ int64_t tiles_before(const PromptArgs& a, int64_t past, int64_t i) {
    return i * (a.G * (past + a.tile_cost)) + ((i * (i + 1)) << (kRowShift<THREADS> - 1));
}
template <int THREADS>
__device__ __forceinline__ int64_t tile_cost(const PromptArgs& a, int64_t past, int64_t i) { return a.G * (past + a.tile_cost) + ((i + 1) << kRowShift<THREADS>); }

struct PromptLds {
    int64_t sums[3][kMostPromptThreads / kWave];
    int64_t base[2], before[2];
    int found[2];
};

// A row tile on the line: begins at `begin`, costs `cost`.
struct PromptTile {
    int b, kvh, i;
    int64_t begin, cost;
    int64_t before;        // tokens of the requests before
    PromptRequest r;
};

struct PromptPlan {
    int64_t total;                     // of the line
    int64_t snap, whole;               // row tiles of up to this cost are not cut
    int W;                             // stretches in use
};

__device__ __forceinline__ int64_t uniform64(int64_t x) {
    return static_cast<int64_t>(static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(x >> 32)))) << 32 |
                                static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(x))));
}

// Sum of v over the threads before this one, and over all; two barriers.
template <int THREADS>
__device__ __forceinline__ int64_t prompt_before(int64_t v, int64_t* s, int64_t& total) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    int64_t up = v;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int64_t x = __shfl_up(up, o, kWave);
        if (lane >= o) up += x;
    }
    if (lane == kWave - 1) s[wave] = up;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) {
        if (w < wave) before += s[w];
        all += s[w];
    }
    total = uniform64(all);
    return before + up - v;
}

// Where stretch w begins on the line, before cuts are moved.
__device__ __forceinline__ int64_t stretch_begin(const PromptPlan& p, int w) {
    const int64_t each = p.total / p.W, rest = p.total - each * p.W;
    return each * w + rest * w / p.W;
}

// The stretch of workgroup `block`, of W in use; -1: none.  Neighbouring stretches read the same positions: one XCD (ids are dealt round-robin to eight) takes
// an eighth of the line.  An eighth of what is in use, not of the launch: with wide block tables the host cannot see how little there is to do (8 single tokens behind
// 2048 positions, 8/1 heads, a table for 32 768: of 512 workgroups 73 have a stretch, by eighths of the launch on two XCDs 32.6 us, on all eight 26.3; eight prompts of 17 .. 300 18.4 | 16.8).
constexpr int kXcds = 8;
__host__ __device__ constexpr int stretch_of(int block, int W) {
    const int xcd = block % kXcds, w = xcd * W / kXcds + block / kXcds;
    return w < (xcd + 1) * W / kXcds ? w : -1;
}

// The line, by all threads of a workgroup (each looks at ceil(B / threads) requests behind one another), the workgroup's stretch w, and where on it
// that begins and ends: the row tiles there.  False: it has no stretch.  No barrier behind it.
template <int THREADS>
__device__ __forceinline__ bool prompt_plan(const PromptArgs& a, PromptLds& s, int& w, PromptPlan& p, int64_t (&x)[2], PromptTile (&t)[2], int& error) {
    const int per = (a.B + THREADS - 1) / THREADS, b0 = threadIdx.x * per, b1 = min(b0 + per, a.B);
    int64_t n = 0, all;
    for (int b = b0; b < b1; ++b) n += prompt_tokens(a, b);
    const int64_t mine_n = prompt_before<THREADS>(n, s.sums[0], all);
    int64_t mine_cost = 0, before = mine_n, tiles = 0;
    for (int b = b0; b < b1; ++b) {
        const PromptRequest r = prompt_request<THREADS>(a, b, before, error);
        before += prompt_tokens(a, b);
        mine_cost += a.Hkv * tiles_before<THREADS>(a, r.past, r.tiles);
        tiles += a.Hkv * static_cast<int64_t>(r.tiles);
    }
    int64_t all_tiles;
    prompt_before<THREADS>(tiles, s.sums[2], all_tiles);
    const int64_t mine = prompt_before<THREADS>(mine_cost, s.sums[1], p.total);
    const int64_t least = static_cast<int64_t>(a.G) * kMinStretch;
    const int64_t most = max((p.total + least - 1) / least, all_tiles);
    p.W = __builtin_amdgcn_readfirstlane(static_cast<int>(most < a.W ? most : a.W));
    p.snap = least / 2;
    p.whole = static_cast<int64_t>(a.G) * (kWholePositions + a.tile_cost);
    // (of stretches that are not in use nothing is joined)
    if (blockIdx.x == 0)
        for (int i = p.W + static_cast<int>(threadIdx.x); i < a.W; i += THREADS) a.cuts[i] = PromptCut{0, 0, 0, 0};
    w = __builtin_amdgcn_readfirstlane(stretch_of(static_cast<int>(blockIdx.x), p.W));
    if (w < 0) return false;
    int ignored = 0;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        x[e] = stretch_begin(p, w + e);
        const int64_t at = x[e] < p.total ? x[e] : p.total - 1;        // (the line's end: its last row tile)
        if (at < mine || at >= mine + mine_cost) continue;
        int64_t begin = mine;
        before = mine_n;
        for (int b = b0; b < b1; ++b) {
            const PromptRequest r = prompt_request<THREADS>(a, b, before, ignored);
            const int64_t cost = a.Hkv * tiles_before<THREADS>(a, r.past, r.tiles);
            if (at < begin + cost) {
                s.found[e] = b, s.base[e] = begin, s.before[e] = before;
                break;
            }
            begin += cost;
            before += prompt_tokens(a, b);
        }
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int64_t at = x[e] < p.total ? x[e] : p.total - 1;
        PromptTile& o = t[e];
        o.b = __builtin_amdgcn_readfirstlane(s.found[e]);
        o.before = uniform64(s.before[e]);
        o.r = prompt_request<THREADS>(a, o.b, o.before, ignored);
        const int64_t begin = uniform64(s.base[e]), head = tiles_before<THREADS>(a, o.r.past, o.r.tiles), d = at - begin;
        o.kvh = static_cast<int>(d / head);
        const int64_t inside = d - o.kvh * head;
        // the largest i with tiles_before(i) <= inside
        const double A = static_cast<double>(a.G * (o.r.past + a.tile_cost) + (1 << (kRowShift<THREADS> - 1))), row_tile = 1 << kRowShift<THREADS>;
        int64_t i = static_cast<int64_t>((sqrt(A * A + 2.0 * row_tile * static_cast<double>(inside)) - A) / row_tile);
        i = i < 0 ? 0 : (i >= o.r.tiles ? o.r.tiles - 1 : i);
        while (i > 0 && tiles_before<THREADS>(a, o.r.past, i) > inside) --i;
        while (i + 1 < o.r.tiles && tiles_before<THREADS>(a, o.r.past, i + 1) <= inside) ++i;
        o.i = static_cast<int>(i);
        o.begin = begin + o.kvh * head + tiles_before<THREADS>(a, o.r.past, i);
        o.cost = tile_cost<THREADS>(a, o.r.past, i);
    }
    return true;
}

// The row tile behind t on the line, which must not end there; by each wave for itself.  Of the KV head, of the next one, of the next request with
// tokens: 64 requests are looked at together.
template <int THREADS>
__device__ __forceinline__ void next_tile(const PromptArgs& a, PromptTile& t) {
    t.begin += t.cost;
    if (t.i + 1 < t.r.tiles) {
        ++t.i;
    } else if (t.kvh + 1 < a.Hkv) {
        ++t.kvh, t.i = 0;
    } else {
        int ignored = 0;
        const int lane = threadIdx.x & (kWave - 1);
        t.before += prompt_tokens(a, t.b);
        t.kvh = 0, t.i = 0, t.r.tiles = 0;
        for (int b0 = t.b + 1; b0 < a.B && t.r.tiles == 0; ) {
            const int n = b0 + lane < a.B ? prompt_tokens(a, b0 + lane) : 0;
            const uint64_t some = __ballot(n > 0);
            if (some == 0) {
                b0 += kWave;
                continue;
            }
            t.b = b0 + __builtin_ctzll(some);
            t.r = prompt_request<THREADS>(a, t.b, t.before, ignored);       // (nothing, if the tokens before it fill the array)
            if (t.r.tiles == 0) t.before += prompt_tokens(a, t.b), b0 = t.b + 1;
        }
        t.before = uniform64(t.before);
        t.b = __builtin_amdgcn_readfirstlane(t.b);
        t.r.past = uniform64(t.r.past), t.r.n = __builtin_amdgcn_readfirstlane(t.r.n), t.r.tiles = __builtin_amdgcn_readfirstlane(t.r.tiles);
        t.r.first = __builtin_amdgcn_readfirstlane(t.r.first), t.r.bad = __builtin_amdgcn_readfirstlane(t.r.bad);
    }
    t.cost = tile_cost<THREADS>(a, t.r.past, t.i);
}
// A cut at x inside row tile t, moved to the row tile's end if that is near.
__device__ __forceinline__ int64_t moved_cut(const PromptPlan& p, const PromptTile& t, int64_t x) {
    if (x >= t.begin + t.cost) return t.begin + t.cost;        // (the line's end)
    if (x - t.begin <= p.snap || t.cost <= p.whole) return t.begin;
    if (t.begin + t.cost - x <= p.snap) return t.begin + t.cost;
    return x;
}
// How many stretches the row tile lies in that begins in stretch w and is cut behind it.
__device__ __forceinline__ int pieces_of(const PromptPlan& p, const PromptTile& t, int w) {
    const int64_t last = t.begin + t.cost - p.snap;            // the first cut from here on is moved to the row tile's end
    int e = w + 1;
    const int64_t each = p.total / p.W > 0 ? p.total / p.W : 1;
    const int64_t guess = last / (each + 1);
    if (guess > e) e = static_cast<int>(guess < p.W ? guess : p.W);
    while (e > w + 1 && stretch_begin(p, e - 1) >= last) --e;
    while (e < p.W && stretch_begin(p, e) < last) ++e;
    return e - w;
}

// The partition kernel for the shared latent 576/512.
hipError_t launch_prompt_latent(const PromptArgs& a, hipStream_t stream);

}  // namespace seer
