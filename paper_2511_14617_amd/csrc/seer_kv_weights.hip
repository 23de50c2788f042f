// seer_kv_weights: the attention weight that the tokens of a step gave to every cached position, added to running sums.
//
// For a request whose cache now holds n positions, the last R of them from this step (the root and the accepted draft tokens), row i of
// the step sees positions 0 .. n - R + i.  With s_rj = scale q_r . k_j for every row r = (i, head g of the group) and
// lse_r = ln sum_j exp s_rj over what the row sees,
//   w_j <- decay w_j (0 for the step's own positions) + sum_r exp(s_rj - lse_r).
//
// What bounds it: HBM for a few rows, LDS reads and matrix products in turn for the many rows of a shared latent.  A weight needs its row's
// denominator first:
//   up to 16 rows   one sweep over the keys (kModeKeep) that leaves each row's maximum and sum per piece and the scores, kv_lse, which joins the
//                   denominators, and kv_apply, which reads the scores.  64 requests of 512 .. 32 768 tokens on 32/8 heads, one row each: 251 us with two
//                   sweeps, 168 with one.
//   more            the scores would cost more than the keys: two sweeps with the same loads and matrix products, kModeSums and
//                   kModeWeights, kv_lse between them.
//
// Work decomposition: per KV head the 32-token tiles of all requests, each times its row blocks of 32 NW rows, lie on one line, cut
// into equal stretches, one per workgroup, all of them resident at once.  Every workgroup finds its stretch from the lengths
// (for_pieces, one request per lane).  A piece is a request's part of a stretch; piece (w, b) has partial slot w + b (along the line every
// next piece raises one of the two).  Tiles go from the pool to LDS directly (32 rows of 16-byte chunks, swizzled as in
// seer_tile.h), wave i holds 32 query rows in registers.  The first sweep multiplies K.Q^T (a row per lane: its maximum and
// sum stay in the lane), the second Q.K^T (a token per lane: the sum over the rows stays in the lane).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "../../include/seer_verify.h"
#include "seer_device.h"
#include "seer_plan.h"
#include "seer_tile.h"

namespace seer {

constexpr int kSwTile = 32;            // tokens of a tile
constexpr int kSwChunk = 32;           // tiles whose sums are collected in LDS before they go to memory
constexpr int kModeSums = 0, kModeWeights = 1, kModeKeep = 2;          // (see kv_sweep)
// Stages of the ring of tiles in LDS, waves per SIMD that the registers have to leave room for.
constexpr int sweep_stages(int Dqk, int mode) { return mode == kModeKeep && Dqk <= 256 ? 3 : 2; }
constexpr int sweep_waves_per_simd(int Dqk) { return Dqk <= 128 ? 3 : 2; }
constexpr int kSwMaxStretches = 2048;
constexpr int64_t kCacheable = int64_t{192} << 20;
constexpr int kLseThreads = 256, kLseRows = 8;
constexpr int kApplyThreads = 256, kApplyPositions = 2048;

struct KvWeightsArgs {
    float* weights;
    const void* q;
    const void* k_pages;
    const int32_t* block_table;
    const int32_t* ctx_len;
    const int32_t* accepted_len;       // nullptr: all T slots of every request
    const int32_t* accepted_path;
    int32_t* status;                   // may be nullptr
    int32_t* line;                     // [B + 2]: units per stretch, then each request's first unit on the line and the line's end
    float2* part;                      // [W + B][Hkv][G T] maximum (log2 units, scaled) and sum
    float* lse;                        // [B][Hkv][G T] log2 of the denominators
    float* scores;                     // [B][Hkv][ldw][kept rows] scaled, in log2 units (few rows only)
    int64_t ldw;                       // positions of a row of weights
    int B, T, Hq, Hkv, G, P, num_pages, max_pages, max_ctx, W, block_rows;
    float scale_log2, decay;
};

struct StepRows {
    int n, rows;                       // positions of the request, rows of the step; rows = 0: left as it is
};
__device__ __forceinline__ StepRows step_rows(const KvWeightsArgs& a, int b, bool& bad) {
    StepRows s{a.ctx_len[b], a.accepted_len ? a.accepted_len[b] + 1 : a.T};
    bad = false;
    if (s.rows < 1 || s.rows > a.T) bad = true, s.rows = 0;
    if (s.n < s.rows || s.n < 1 || s.n > a.max_ctx) bad = true, s.rows = 0;
    return s;
}
__device__ __forceinline__ int row_blocks_of(const KvWeightsArgs& a, int rows) { return (rows * a.G + a.block_rows - 1) / a.block_rows; }
__device__ __forceinline__ int units_of(const KvWeightsArgs& a, const StepRows& s) { return s.rows ? (s.n + kSwTile - 1) / kSwTile * row_blocks_of(a, s.rows) : 0; }

// The step's slots (lane i: row i's), which have to ascend from the root; `wrong` if they do not.
__device__ __forceinline__ int step_slot(const KvWeightsArgs& a, int b, int rows, bool& wrong) {
    const int lane = static_cast<int>(threadIdx.x) & (kWave - 1);
    wrong = false;
    if (!a.accepted_path) return lane;
    const int slot = lane < rows ? a.accepted_path[static_cast<size_t>(b) * a.T + lane] : a.T, up = __shfl_up(slot, 1, kWave);
    wrong = __any(lane < rows && (lane == 0 ? slot != 0 : slot <= up || slot >= a.T));
    return slot;
}

// body(request, its positions, rows of the step, step_slot's, row blocks, first and last tile, units of the whole line) for every piece of stretch w.  The line: per KV head the
// tiles of all requests, each times the request's row blocks, cut into equal stretches.  PUBLISH: the first workgroup leaves the line for kv_lse,
// and status bits are raised.
template <bool PUBLISH, class Body>
__device__ __forceinline__ void for_pieces(const KvWeightsArgs& a, int w, int& found, Body&& body) {
    const int tid = threadIdx.x, lane = tid & (kWave - 1);
    const bool publish = PUBLISH && blockIdx.x == 0;
    int total = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {               // 64 requests at a time
        bool bad = false;
        int u = 0;
        if (b0 + lane < a.B) u = units_of(a, step_rows(a, b0 + lane, bad));
        if (publish && bad) found |= 1;
        const int incl = wave_incl_scan(u);
        if (publish && tid < kWave && b0 + lane < a.B) a.line[1 + b0 + lane] = total + incl - u;
        total += last_lane(incl);
    }
    const int step = max(1, (total + a.W - 1) / a.W);
    if (publish && tid == 0) a.line[0] = step, a.line[1 + a.B] = total;
    const int u_begin = min(w * step, total), u_end = min(u_begin + step, total);
    int before = 0;                                         // units of the requests in front of b0
    for (int b0 = 0; b0 < a.B && before < u_end; b0 += kWave) {
        bool bad = false;
        StepRows mine{0, 0};
        if (b0 + lane < a.B) mine = step_rows(a, b0 + lane, bad);
        const int my_units = units_of(a, mine), incl = wave_incl_scan(my_units), my_off = before + incl - my_units;
        uint64_t todo = __ballot(my_units > 0 && my_off < u_end && my_off + my_units > u_begin);
        before += last_lane(incl);
        for (; todo; todo &= todo - 1) {
            const int bit = __builtin_ctzll(todo), b = b0 + bit;
            const int off = __builtin_amdgcn_readlane(my_off, bit), n = __builtin_amdgcn_readlane(mine.n, bit);
            const int rows = __builtin_amdgcn_readlane(mine.rows, bit), blocks = row_blocks_of(a, rows);
            const int n_tiles = (n + kSwTile - 1) / kSwTile;
            const int t_begin = min(n_tiles, (max(u_begin - off, 0) + blocks - 1) / blocks);
            const int t_end = min(n_tiles, (u_end - off + blocks - 1) / blocks);
            bool wrong;
            const int slot = step_slot(a, b, rows, wrong);
            if (wrong) {
                if (PUBLISH) found |= 4;
                continue;
            }
            body(b, n, rows, slot, blocks, t_begin, t_end, total);
        }
    }
}

template <int DQK>
struct Keys {
    static constexpr int kRow = DQK * 2, kBytes = kSwTile * kRow, kSteps = DQK / 16, kRowChunks = kRow / 16;
};

// Scores of the tile at LDS address `at`, 32 tokens against this wave's 32 rows.  ROWS: register i of the result holds row (i/4)*8 + lg*4 + i%4
// for this lane's token, else that token for this lane's row.
template <int DQK, bool ROWS>
__device__ __forceinline__ f32x16 sweep_scores(int at, int k_rd, const bf16x8 (&q)[DQK / 16]) {
    constexpr int kXorBits = Keys<DQK>::kRow % 256 == 0 ? 4 : 3, kPerXor = 1 << (kXorBits - 1);
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
    const int ka = at + k_rd;
#pragma unroll
    for (int h = 0; h < DQK / 16; h += 4) {
        u32x4 kv[4];
        auto of = [&](int kk) { return (ka ^ ((kk % kPerXor) << 5)) + kk / kPerXor * (kPerXor * 32); };
        tile::read_k4(kv, of(h), of(h + 1), of(h + 2), of(h + 3));
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
            s = ROWS ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[h + kk], as_bf16x8(kv[kk]), s, 0, 0, 0)
                     : __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kv[kk]), q[h + kk], s, 0, 0, 0);
    }
    return s;
}

// The same from one of the stages, which are arrays of their own so that the compiler can tell a read of this one from the loads in flight into the other.  It waits for
// all reads at once while such loads are in flight: four reads go behind the first product of the four before, a product's time ahead of their use (16
// requests of 8192 .. 24 576 tokens on 128 heads: 300 us with reads and products in turn, 278 so).
template <int DQK, bool ROWS>
__device__ __forceinline__ f32x16 stage_scores(const unsigned char* stage, const int (&rd)[4], const bf16x8 (&q)[DQK / 16]) {
    constexpr int kXorBits = Keys<DQK>::kRow % 256 == 0 ? 4 : 3, kPerXor = 1 << (kXorBits - 1);
    static_assert(kPerXor == 4, "");
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < DQK / 16; ++kk) {
        const bf16x8 k = as_bf16x8(*reinterpret_cast<const u32x4*>(stage + rd[kk % kPerXor] + kk / kPerXor * (kPerXor * 32)));
        s = ROWS ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(q[kk], k, s, 0, 0, 0) : __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[kk], s, 0, 0, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);      // (0x100: reads, 0x008: products)
#pragma unroll
    for (int h = 1; h < DQK / 64; ++h) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, 3, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    return s;
}

// A word of LDS (as asm with its wait, like the tiles' reads: through the compiler it would wait for the tile loads in flight).
__device__ __forceinline__ float lds_word(int at) {
    float v;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v) : "v"(at) : "memory");
    return v;
}

// Sum of NW words 128 bytes apart, in their order.
template <int NW>
__device__ __forceinline__ float lds_sum(int at) {
    if constexpr (NW == 2) {
        float v[2];
        asm volatile("ds_read_b32 %0, %2\n\tds_read_b32 %1, %2 offset:128\n\ts_waitcnt lgkmcnt(0)" : "=&v"(v[0]), "=&v"(v[1]) : "v"(at) : "memory");
        return v[0] + v[1];
    } else {
        static_assert(NW == 8, "");
        float v[8];
        asm volatile("ds_read_b32 %0, %8\n\tds_read_b32 %1, %8 offset:128\n\tds_read_b32 %2, %8 offset:256\n\tds_read_b32 %3, %8 offset:384\n\t"
                     "ds_read_b32 %4, %8 offset:512\n\tds_read_b32 %5, %8 offset:640\n\tds_read_b32 %6, %8 offset:768\n\tds_read_b32 %7, %8 offset:896\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(v[0]), "=&v"(v[1]), "=&v"(v[2]), "=&v"(v[3]), "=&v"(v[4]), "=&v"(v[5]), "=&v"(v[6]), "=&v"(v[7])
                     : "v"(at)
                     : "memory");
        return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
    }
}

// MODE: kModeSums leaves each row's maximum and sum, kModeWeights the weights, kModeKeep (KEPT rows at most, one wave) maximum, sum and the scores themselves.
template <int DQK, int NW, int MODE, int KEPT>
__global__ __launch_bounds__(NW * kWave) __attribute__((amdgpu_waves_per_eu(NW == 8 ? 2 : 1))) void kv_sweep(KvWeightsArgs a) {
    using K = Keys<DQK>;
    constexpr bool WEIGHTS = MODE == kModeWeights;
    constexpr int kSwStages = sweep_stages(DQK, MODE);
    constexpr int kTileLoads = K::kBytes / 1024, kLoads = (kTileLoads + NW - 1) / NW;      // direct-to-LDS loads of a tile, of a wave at most
    static_assert(kSwStages == 2 || kLoads * (kSwStages - 1) < 64, "");
    constexpr bool APART = NW == 8;
    static_assert(APART || kTileLoads % NW == 0, "every wave has the same number of loads in flight");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[APART ? 1024 : kSwStages * K::kBytes];
    __shared__ __attribute__((aligned(1024))) unsigned char lds_even[APART ? K::kBytes : 1], lds_odd[APART ? K::kBytes : 1];
    __shared__ float s_sums[WEIGHTS ? kSwChunk * kSwTile : 1];
    __shared__ __attribute__((aligned(16))) float s_denom[NW][WEIGHTS ? 32 : 1];       // of the waves' rows
    __shared__ float s_part[2][WEIGHTS && NW > 1 ? NW : 1][WEIGHTS && NW > 1 ? kSwTile : 1];      // the waves' sums of a tile

    const int kvh = blockIdx.x % a.Hkv, w = blockIdx.x / a.Hkv;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), ln = lane & 31, lg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const unsigned char* __restrict__ kbase = static_cast<const unsigned char*>(a.k_pages);
    const int k_rd = ln * K::kRow + ((lg ^ tile::k_swz<K::kRow>(ln)) << 4);
    const bool page_pow2 = (a.P & (a.P - 1)) == 0;
    const int page_shift = __builtin_ctz(static_cast<unsigned>(a.P));
    auto page_of = [&](int tok) __attribute__((always_inline)) -> int { return page_pow2 ? tok >> page_shift : tok / a.P; };
    int rd[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) rd[x] = k_rd ^ x << 5;
    auto scores = [&](auto rows, const unsigned char* at, const bf16x8 (&q)[K::kSteps]) __attribute__((always_inline)) {
        if constexpr (APART) return stage_scores<DQK, decltype(rows)::value>(at, rd, q);
        else return sweep_scores<DQK, decltype(rows)::value>(tile::lds_addr(at), k_rd, q);
    };
    int found = 0;                                          // status bits

    for_pieces<MODE != kModeWeights>(a, w, found, [&](int b, int n, int rows, int slot, int blocks, int t_begin, int t_end, int total) __attribute__((always_inline)) {
            const int R = rows * a.G;
            // Keys that the memory-side cache cannot hold for the second sweep are streamed past it, and so are those that are read once.
            const bool stream = MODE == kModeKeep || static_cast<int64_t>(total) * K::kBytes * a.Hkv > kCacheable;

            // ---- tile loads --------------------------------------------------------------------------
            const int32_t* __restrict__ table = a.block_table + static_cast<size_t>(b) * a.max_pages;
            const int last_page = (n - 1) / a.P;
            int win = 0, pg_win = 0;                        // lane l holds the (clamped) page id of logical page win + l
            bool have_window = false;
            auto issue_tile = [&](int t, unsigned char* to) __attribute__((always_inline)) {
                const int tb = t * kSwTile, first = page_of(tb);
                if (!have_window || first < win || page_of(tb + kSwTile - 1) >= win + kWave) {       // (uniform; a tile spans at most 32 pages)
                    have_window = true;
                    win = first;
                    int pg = table[min(first + lane, a.max_pages - 1)];
                    if (pg < 0 || pg >= a.num_pages) {
                        if (first + lane <= last_page) found |= 2;
                        pg = min(max(pg, 0), a.num_pages - 1);
                    }
                    pg_win = pg;
                }
                const int tok = tb + ln, lp = page_of(tok);
                const int pg = __builtin_amdgcn_ds_bpermute((lp - win) << 2, pg_win);
                const uint32_t row_idx = (static_cast<uint32_t>(pg) * a.Hkv + kvh) * static_cast<uint32_t>(a.P) + (tok - lp * a.P);
                uint32_t at[kLoads];                        // (all asked for, then waited for once: a lane's value comes from another one through LDS)
#pragma unroll
                for (int j = 0; j < kLoads; ++j) at[j] = __builtin_amdgcn_ds_bpermute(((wave + j * NW) * kWave + lane) / K::kRowChunks << 2, row_idx);
                __builtin_amdgcn_sched_barrier(0);
                auto from = [&](int j) __attribute__((always_inline)) {
                    const int c = (wave + j * NW) * kWave + lane, row = c / K::kRowChunks, pos = c - row * K::kRowChunks;
                    return kbase + static_cast<size_t>(at[j]) * K::kRow + ((pos ^ tile::k_swz<K::kRow>(row)) << 4);
                };
                to += wave * 1024;
                if (stream) {
#pragma unroll
                    for (int j = 0; j < kLoads; ++j)
                        if (kTileLoads % NW == 0 || wave + j * NW < kTileLoads)
                            __builtin_amdgcn_global_load_lds((const SEER_AS1 void*)(from(j)), (SEER_AS3 void*)(to + j * NW * 1024), 16, 0, 2);
                } else {
#pragma unroll
                    for (int j = 0; j < kLoads; ++j)
                        if (kTileLoads % NW == 0 || wave + j * NW < kTileLoads)
                            __builtin_amdgcn_global_load_lds((const SEER_AS1 void*)(from(j)), (SEER_AS3 void*)(to + j * NW * 1024), 16, 0, 0);
                }
            };

            // Tiles t0 .. t1 - 1, each handed to `use` with its LDS address once it has landed for every wave; `after` is called behind the
            // barrier that follows a tile.
            auto sweep = [&](int t0, int t1, auto&& use, auto&& after) __attribute__((always_inline)) {
                if (NW > 1) bare_barrier();                 // every wave is done with the stages
                if constexpr (APART) {
                    auto one = [&](int t, unsigned char* here, unsigned char* other) __attribute__((always_inline)) {
                        asm volatile("" ::: "memory");      // (the barrier alone does not keep reads of the stage behind it)
                        wait_vmcnt<0>();
                        __builtin_amdgcn_s_waitcnt(0xc07f);
                        bare_barrier();
                        asm volatile("" ::: "memory");
                        if (t + 1 < t1) issue_tile(t + 1, other);
                        if (t > t0) after(t - 1);
                        use(t, here);
                    };
                    if (t0 < t1) issue_tile(t0, lds_even);
                    for (int t = t0; t < t1; t += 2) {
                        one(t, lds_even, lds_odd);
                        if (t + 1 < t1) one(t + 1, lds_odd, lds_even);
                    }
                    __builtin_amdgcn_s_waitcnt(0xc07f);
                    bare_barrier();
                    if (t1 > t0) after(t1 - 1);
                    return;
                }
#pragma unroll
                for (int s = 0; s < kSwStages - 1; ++s)
                    if (t0 + s < t1) issue_tile(t0 + s, lds + s * K::kBytes);
                int stage = 0;
                for (int t = t0; t < t1; ++t) {
                    // (this wave's loads of the tiles behind this one may be on their way; near the end none are waited for apart)
                    if (kSwStages == 2 || t + kSwStages - 1 > t1) wait_vmcnt<0>();
                    else wait_vmcnt<kLoads * (kSwStages - 2)>();
                    if (NW > 1) {
                        __builtin_amdgcn_s_waitcnt(0xc07f); // (lgkmcnt: what `use` wrote)
                        bare_barrier();
                    }
                    const int next = stage == 0 ? kSwStages - 1 : stage - 1;
                    if (t + kSwStages - 1 < t1) issue_tile(t + kSwStages - 1, lds + next * K::kBytes);
                    __builtin_amdgcn_sched_barrier(0);
                    if (t > t0) after(t - 1);
                    use(t, lds + stage * K::kBytes);
                    __builtin_amdgcn_sched_barrier(0);
                    stage = stage + 1 == kSwStages ? 0 : stage + 1;
                }
                if (NW > 1) {
                    __builtin_amdgcn_s_waitcnt(0xc07f);
                    bare_barrier();
                }
                if (t1 > t0) after(t1 - 1);
            };

            bf16x8 q[K::kSteps];
            auto load_rows = [&](int block) __attribute__((always_inline)) {       // this lane's row
                const int r = block * a.block_rows + wave * 32 + ln;
                const bool ok = r < R;
                const int i = ok ? r / a.G : 0, g = ok ? r - i * a.G : 0;
                const int t = __builtin_amdgcn_ds_bpermute(i << 2, slot);
                const u32x4* from = reinterpret_cast<const u32x4*>(
                    static_cast<const uint16_t*>(a.q) + ((static_cast<size_t>(b) * a.T + t) * a.Hq + kvh * a.G + g) * DQK + lg * 8);
#pragma unroll
                for (int kk = 0; kk < K::kSteps; ++kk) {
                    u32x4 v = {0u, 0u, 0u, 0u};
                    if (ok) v = from[kk * 2];
                    q[kk] = as_bf16x8(v);
                }
                return r;
            };
            const int first_own = n - rows;                 // row i sees positions up to first_own + i

            if constexpr (MODE == kModeSums) {
                for (int block = 0; block < blocks; ++block) {
                    const int r = load_rows(block);
                    const int seen = first_own + min(r, R - 1) / a.G + 1;
                    float m_run = kNegInf, l_run = 0.f;
                    const bool idle = block * a.block_rows + wave * 32 >= R;      // (uniform: none of the wave's rows exists)
                    sweep(t_begin, t_end, [&](int t, const unsigned char* at) __attribute__((always_inline)) {
                        if (NW > 1 && idle) return;
                        f32x16 s = scores(std::integral_constant<bool, false>{}, at, q);
                        const int tb = t * kSwTile;
                        if (tb + kSwTile > first_own + 1) {
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (tb + (i >> 2) * 8 + lg * 4 + (i & 3) >= seen) s[i] = kNegInf;
                        }
                        float mx = s[0];
#pragma unroll
                        for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
                        float alpha;
                        const float m_use = move_reference(mx, a.scale_log2, m_run, alpha);
                        float sum = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum += fast_exp2(fmaf(s[i], a.scale_log2, -m_use));
                        l_run = fmaf(l_run, alpha, sum);
                    }, [](int) {});
                    const float l = l_run + __shfl_xor(l_run, 32, kWave);
                    if (lg == 0 && r < R) a.part[(static_cast<size_t>(w + b) * a.Hkv + kvh) * (a.G * a.T) + r] = make_float2(m_run, l);
                }
            } else if constexpr (MODE == kModeKeep) {
                // a token per lane, its few rows in the first registers: maximum and sum per row and lane, joined at the end
                constexpr int kRegs = KEPT <= 8 ? 4 : 8;
                const int r_own = load_rows(0), row_i = min(r_own, R - 1) / a.G;
                float m[kRegs], l[kRegs];
#pragma unroll
                for (int i = 0; i < kRegs; ++i) m[i] = kNegInf, l[i] = 0.f;
                float* __restrict__ to = a.scores + (static_cast<size_t>(b) * a.Hkv + kvh) * a.ldw * KEPT;
                sweep(t_begin, t_end, [&](int t, const unsigned char* at) __attribute__((always_inline)) {
                    f32x16 s = scores(std::integral_constant<bool, true>{}, at, q);
                    const int tok = t * kSwTile + ln;
#pragma unroll
                    for (int i = 0; i < kRegs; ++i) s[i] *= a.scale_log2;
                    if (t * kSwTile + kSwTile > first_own + 1) {
#pragma unroll
                        for (int i = 0; i < kRegs; ++i)
                            if (__shfl(row_i, (i >> 2) * 8 + lg * 4 + (i & 3), kWave) < tok - first_own) s[i] = kNegInf;
                    }
#pragma unroll
                    for (int i = 0; i < kRegs; ++i) {
                        const float top = fmaxf(m[i], s[i]), use = top == kNegInf ? 0.f : top;
                        l[i] = fmaf(l[i], fast_exp2(m[i] - use), fast_exp2(s[i] - use));
                        m[i] = top;
                    }
                    if (tok < n && (KEPT > 4 || lg == 0)) {
#pragma unroll
                        for (int i = 0; i < kRegs; i += 4)
                            *reinterpret_cast<f32x4*>(to + static_cast<size_t>(tok) * KEPT + (i >> 2) * 8 + lg * 4) = f32x4{s[i], s[i + 1], s[i + 2], s[i + 3]};
                    }
                }, [](int) {});
#pragma unroll
                for (int i = 0; i < kRegs; ++i) {
                    float top = m[i];
#pragma unroll
                    for (int o = 16; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
                    float sum = m[i] == kNegInf ? l[i] * 0.f : l[i] * fast_exp2(m[i] - top);       // (nothing seen: 0, or a NaN that was)
#pragma unroll
                    for (int o = 16; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, kWave);
                    const int r = (i >> 2) * 8 + lg * 4 + (i & 3);
                    if (ln == 0 && r < R) a.part[(static_cast<size_t>(w + b) * a.Hkv + kvh) * (a.G * a.T) + r] = make_float2(top, sum);
                }
            } else {
                float* __restrict__ to = a.weights + (static_cast<size_t>(b) * a.Hkv + kvh) * a.ldw;
                for (int c0 = t_begin; c0 < t_end; c0 += kSwChunk) {
                    const int c1 = min(c0 + kSwChunk, t_end);
                    for (int block = 0; block < blocks; ++block) {
                        const int r = load_rows(block);
                        // the denominators of the wave's rows, register by register
                        float own = -kNegInf;               // (no such row: exp2 gives 0)
                        if (r < R) own = a.lse[(static_cast<size_t>(b) * a.Hkv + kvh) * (a.G * a.T) + r];
                        const bool partial = __any(!(own < -kNegInf));
                        if (lg == 0) s_denom[wave][ln] = own;
                        const int denom_at = tile::lds_addr(reinterpret_cast<const unsigned char*>(&s_denom[wave][lg * 4]));
                        const int row_i = min(r, R - 1) / a.G;
                        const bool idle = block * a.block_rows + wave * 32 >= R;
                        sweep(c0, c1, [&](int t, const unsigned char* at) __attribute__((always_inline)) {
                            if (NW > 1 && idle) {
                                if (lg == 0) s_part[t & 1][wave][ln] = 0.f;
                                return;
                            }
                            f32x16 s = scores(std::integral_constant<bool, true>{}, at, q);
                            const int tb = t * kSwTile;
                            u32x4 denom[4];                 // (read for every tile: kept in registers they are what the 576-wide rows have not)
                            tile::read_k4(denom, denom_at, denom_at + 32, denom_at + 64, denom_at + 96);
                            auto denom_of = [&](int i) __attribute__((always_inline)) { return __uint_as_float(denom[i >> 2][i & 3]); };
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[i] = fast_exp2(fmaf(s[i], a.scale_log2, -denom_of(i)));
                            if (partial) {
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    if (denom_of(i) == -kNegInf) s[i] = 0.f;
                            }
                            if (tb + kSwTile > first_own + 1) {
                                const int behind = tb + ln - first_own;     // rows from this one on see the position
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    if (__shfl(row_i, (i >> 2) * 8 + lg * 4 + (i & 3), kWave) < behind) s[i] = 0.f;
                            }
                            float sum = 0.f;
#pragma unroll
                            for (int i = 0; i < 16; ++i) sum += s[i];
                            sum += __shfl_xor(sum, 32, kWave);
                            if constexpr (NW > 1) {
                                if (lg == 0) s_part[t & 1][wave][ln] = sum;
                            } else {
                                const int to_sum = tile::lds_addr(reinterpret_cast<const unsigned char*>(&s_sums[(t - c0) * kSwTile + ln]));
                                if (block) sum += lds_word(to_sum);
                                if (lg == 0) s_sums[(t - c0) * kSwTile + ln] = sum;
                            }
                        }, [&](int t) __attribute__((always_inline)) {
                            if constexpr (NW > 1) {         // the waves' sums of the tile, in their order, by one of them
                                if (wave != (t & (NW - 1))) return;
                                const int from = tile::lds_addr(reinterpret_cast<const unsigned char*>(&s_part[t & 1][0][ln]));
                                float sum = lds_sum<NW>(from);
                                const int to_sum = tile::lds_addr(reinterpret_cast<const unsigned char*>(&s_sums[(t - c0) * kSwTile + ln]));
                                if (block) sum += lds_word(to_sum);
                                if (lg == 0) s_sums[(t - c0) * kSwTile + ln] = sum;
                            }
                        });
                    }
                    __syncthreads();
                    const int tokens = min(n, c1 * kSwTile) - c0 * kSwTile;
                    for (int j = tid; j < tokens; j += NW * kWave) {
                        const int pos = c0 * kSwTile + j;
                        to[pos] = pos < first_own ? fmaf(a.decay, to[pos], s_sums[j]) : s_sums[j];
                    }
                    __syncthreads();
                }
            }
    });
    if (!WEIGHTS && a.status && found) atomicOr(a.status, found);
}

// A piece's sum brought from its maximum to `to`.  Without a maximum nothing was seen there, or nothing but -inf and NaN: 0, or a NaN that has to stay.
__device__ __forceinline__ float part_sum(float2 p, float to) { return p.x == kNegInf ? p.y * 0.f : p.y * fast_exp2(p.x - to); }

// log2 of the denominators: eight rows of a request and KV head per workgroup, 32 threads of a row share its pieces.
__global__ __launch_bounds__(kLseThreads) void kv_lse(KvWeightsArgs a) {
    __shared__ float2 s_part[kLseThreads];
    const int GT = a.G * a.T, groups = (GT + kLseRows - 1) / kLseRows;
    const int b = blockIdx.x / (a.Hkv * groups), rest = blockIdx.x - b * a.Hkv * groups, kvh = rest / groups;
    const int tid = threadIdx.x, r = (rest - kvh * groups) * kLseRows + (tid & (kLseRows - 1)), slice = tid / kLseRows;
    constexpr int kSlices = kLseThreads / kLseRows;
    const int step = a.line[0], begin = a.line[1 + b], end = a.line[2 + b];
    if (begin >= end) return;                               // (nothing of this request is asked for)
    const int first = begin / step, last = (end - 1) / step;
    float m = kNegInf, l = 0.f;
    if (r < GT) {
        const float2* at = a.part + (static_cast<size_t>(b) * a.Hkv + kvh) * GT + r;
        const size_t stride = static_cast<size_t>(a.Hkv) * GT;
#pragma unroll 4
        for (int w = first + slice; w <= last; w += kSlices) {
            const float2 p = at[w * stride];
            const float top = fmaxf(m, p.x), use = top == kNegInf ? 0.f : top;
            l = l * fast_exp2(m - use) + part_sum(p, use);
            m = top;
        }
    }
    s_part[tid] = make_float2(m, l);
    __syncthreads();
    if (slice || r >= GT) return;
    float top = kNegInf;
    for (int s = 0; s < kSlices; ++s) top = fmaxf(top, s_part[s * kLseRows + tid].x);
    float sum = 0.f;
    for (int s = 0; s < kSlices; ++s) {
        sum += part_sum(s_part[s * kLseRows + tid], top);
    }
    // a row that weighs nothing (all its scores -inf): +inf, so that exp2 gives 0
    a.lse[(static_cast<size_t>(b) * a.Hkv + kvh) * GT + r] = top == kNegInf && sum == 0.f ? -kNegInf : top + log2f(sum);
}

// The weights from the scores that kModeKeep left: a position per thread.
template <int KEPT>
__global__ __launch_bounds__(kApplyThreads) void kv_apply(KvWeightsArgs a, int parts) {
    const size_t bh = blockIdx.x / parts;
    const int part = static_cast<int>(blockIdx.x - bh * parts), b = static_cast<int>(bh) / a.Hkv;
    bool bad, wrong;
    const StepRows step = step_rows(a, b, bad);
    if (part * kApplyPositions >= step.n || step.rows == 0) return;
    step_slot(a, b, step.rows, wrong);
    if (wrong) return;
    const int R = step.rows * a.G, first_own = step.n - step.rows;
    const float* lse = a.lse + bh * (a.G * a.T);
    float denom[KEPT];
#pragma unroll
    for (int r = 0; r < KEPT; ++r) denom[r] = r < R ? lse[r] : 0.f;
    const float* scores = a.scores + bh * a.ldw * KEPT;
    float* to = a.weights + bh * a.ldw;
    for (int p0 = part * kApplyPositions; p0 < step.n; p0 += parts * kApplyPositions)
#pragma unroll 4
        for (int x = 0; x < kApplyPositions / kApplyThreads; ++x) {
            const int pos = p0 + x * kApplyThreads + static_cast<int>(threadIdx.x);
            if (pos >= step.n) break;
            const int from_row = pos > first_own ? (pos - first_own) * a.G : 0;      // (a row whose denominator is a NaN leaves what it does not see alone)
            float sum = 0.f;
#pragma unroll
            for (int r = 0; r < KEPT; r += 4) {
                const f32x4 s = *reinterpret_cast<const f32x4*>(scores + static_cast<size_t>(pos) * KEPT + r);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (r + i < R && r + i >= from_row) sum += fast_exp2(s[i] - denom[r + i]);
            }
            to[pos] = pos < first_own ? fmaf(a.decay, to[pos], sum) : sum;
        }
}

// Short block tables: one workgroup per request and KV head keeps all scores in LDS, and the three launches become one.  Wave i takes tiles i, i + 4, .. (the keys
// go from memory to the operand registers, the next tile's while this one is multiplied), then a wave each row for its denominator, then a
// thread each position for its sum.  Against three launches: 4 requests of 64 .. 512 tokens, 8/2 heads, 20 rows at most 12.4 | 17.3 us, 64 of them with 32/8
// heads 20.3 | 30.6; but 16 of up to 3000 tokens with 4 rows 40.4 | 26.3 and 16 of up to 400 with 36 rows 21.9 | 18.9.  Between 512 and 3000 positions they cross at 768 .. 1536 for few
// requests (4 on 8/2 heads, one row: 768 positions 11.8 | 16.3, 1536 19.9 | 16.9; three rows: 1024 19.1 | 16.9), beyond 3000 for many (64 on 32/8, one
// row: 84 | 94): the limit is safe for both.
constexpr int kShortWaves = 4, kShortPositions = 512, kShortRows = 32, kShortScores = 16000;      // of the table, rows, scores in LDS at most
inline bool weights_short(int rows, int Dqk, int64_t positions) {
    return Dqk <= 256 && positions <= kShortPositions && rows <= kShortRows && (positions + 36) * rows <= kShortScores;
}

template <int DQK>
__global__ __launch_bounds__(kShortWaves * kWave) void kv_short(KvWeightsArgs a, int stride) {
    extern __shared__ __attribute__((aligned(16))) float s_score[];       // [rows][stride]: stride positions, a multiple of 32 and 4 more
    __shared__ float s_lse[kShortRows];
    constexpr int kSteps = DQK / 16;
    const int b = blockIdx.x / a.Hkv, kvh = blockIdx.x - b * a.Hkv, tid = threadIdx.x, lane = tid & (kWave - 1), ln = lane & 31, lg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    bool bad, wrong;
    const StepRows step = step_rows(a, b, bad);
    const int slot = step_slot(a, b, step.rows, wrong);
    if (bad || wrong) {
        if (tid == 0 && a.status) atomicOr(a.status, bad ? 1 : 4);
        return;
    }
    const int n = step.n, rows = step.rows, R = rows * a.G, first_own = n - rows, n_tiles = (n + kSwTile - 1) / kSwTile, last_page = (n - 1) / a.P;
    const int32_t* __restrict__ table = a.block_table + static_cast<size_t>(b) * a.max_pages;
    int found = 0;
    auto load_tile = [&](int t, u32x4 (&k)[kSteps]) __attribute__((always_inline)) {        // (behind the last one: it again)
        const int tok = min(t, n_tiles - 1) * kSwTile + ln, lp = tok / a.P;
        int pg = table[min(lp, a.max_pages - 1)];
        if (pg < 0 || pg >= a.num_pages) {
            if (lp <= last_page) found |= 2;
            pg = min(max(pg, 0), a.num_pages - 1);
        }
        const u32x4* from = reinterpret_cast<const u32x4*>(
            static_cast<const uint16_t*>(a.k_pages) + ((static_cast<size_t>(pg) * a.Hkv + kvh) * a.P + (tok - lp * a.P)) * DQK) + lg;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) k[kk] = from[2 * kk];
    };
    u32x4 key[2][kSteps];
    if (wave < n_tiles) load_tile(wave, key[0]);
    const int r = ln, rc = min(r, R - 1), i_row = rc / a.G;
    const int t_slot = __builtin_amdgcn_ds_bpermute(i_row << 2, slot), seen = first_own + i_row + 1;
    const u32x4* from = reinterpret_cast<const u32x4*>(
        static_cast<const uint16_t*>(a.q) + ((static_cast<size_t>(b) * a.T + t_slot) * a.Hq + kvh * a.G + (rc - i_row * a.G)) * DQK) + lg;
    u32x4 q[kSteps];
#pragma unroll
    for (int kk = 0; kk < kSteps; ++kk) q[kk] = from[2 * kk];
    auto scores = [&](int t, const u32x4 (&k)[kSteps]) __attribute__((always_inline)) {
        f32x16 s;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(k[kk]), as_bf16x8(q[kk]), s, 0, 0, 0);
        if (r < R) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const int tok = t * kSwTile + (i >> 2) * 8 + lg * 4;
                f32x4 v;
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = tok + x < seen ? s[i + x] * a.scale_log2 : kNegInf;
                *reinterpret_cast<f32x4*>(&s_score[r * stride + tok]) = v;
            }
        }
    };
    for (int t = wave; t < n_tiles; t += 2 * kShortWaves) {            // two tiles in turn, each requested a tile ahead
        load_tile(t + kShortWaves, key[1]);
        scores(t, key[0]);
        load_tile(t + 2 * kShortWaves, key[0]);
        if (t + kShortWaves < n_tiles) scores(t + kShortWaves, key[1]);
    }
    __syncthreads();
    for (int r = wave; r < R; r += kShortWaves) {
        float m = kNegInf, l = 0.f;
        for (int j = lane; j < n; j += kWave) m = fmaxf(m, s_score[r * stride + j]);
        m = wave_max(m);
        for (int j = lane; j < n; j += kWave) l += fast_exp2(s_score[r * stride + j] - (m == kNegInf ? 0.f : m));
        l = wave_sum(l);
        if (lane == 0) s_lse[r] = m == kNegInf && l == 0.f ? -kNegInf : m + log2f(l);      // (nothing weighs: +inf, so that exp2 gives 0)
    }
    __syncthreads();
    float* __restrict__ to = a.weights + (static_cast<size_t>(b) * a.Hkv + kvh) * a.ldw;
    for (int j = tid; j < n; j += kShortWaves * kWave) {
        const float old = j < first_own ? to[j] : 0.f;
        float sum = 0.f;
#pragma unroll 4
        for (int r = max(0, j - first_own) * a.G; r < R; ++r) sum += fast_exp2(s_score[r * stride + j] - s_lse[r]);       // (the rows that see the position)
        to[j] = j < first_own ? fmaf(a.decay, old, sum) : sum;
    }
    if (a.status && found) atomicOr(a.status, found);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// Rows whose scores are kept between the sweeps: written and read once they cost 8 bytes a position each, the second sweep
// 2 Dqk; up to a quarter of that, and up to 16.  The workspace holds them for every position of the block table, so not where that is more than 2 GiB (some cache of
// many requests on long tables would have no room for it; there the keys are read twice, 64 requests of 512 .. 32 768 tokens on 32/8 heads 251 us instead of
// 168, with 0.1 MB of workspace instead of 268).  0: none.
constexpr size_t kMaxScoreBytes = size_t{2} << 30;
static_assert(kMaxScoreBytes / 16 + size_t{8192} * kApplyPositions < (size_t{1} << 31), "kv_apply counts positions in 32 bits, with a stride of its launch on top");
inline int kept_rows(const seer_attn_params& p, int rows) {
    const int kept = rows <= 4 ? 4 : rows <= 8 ? 8 : 16;
    const int64_t positions = static_cast<int64_t>(p.max_pages_per_seq) * p.page_size, most = static_cast<int64_t>(kMaxScoreBytes / sizeof(float)) / kept;
    return rows <= 16 && kept <= p.Dqk / 8 && static_cast<int64_t>(p.B) * p.Hkv <= most / positions ? kept : 0;
}
struct KvWeightsLayout {
    int waves, W, kept;
    bool whole;                        // kv_short, which needs no workspace
    size_t off_part, off_lse, off_scores, total;
};
inline KvWeightsLayout kv_weights_layout(const seer_attn_params& p) {
    KvWeightsLayout w{};
    const int rows = (p.Hq / p.Hkv) * p.T;
    w.whole = weights_short(rows, p.Dqk, static_cast<int64_t>(p.max_pages_per_seq) * p.page_size);
    w.kept = kept_rows(p, rows);
    // Waves of a workgroup.  Up to 256-wide keys: one per 32 rows that a request may have, at most two (of a step's slots only the accepted ones come, so
    // most requests have fewer: 64 requests of 72 rows at most, two waves 53 us, four 58, one 62).  Shared latent: eight, since every
    // row block of a request reads its keys again (16 requests of 8192 .. 24 576 tokens, 640 rows at most: four waves 326 us, eight 300, 263 .. 280 with stage_scores).
    w.waves = p.Dqk > 256 ? (w.kept ? 1 : 8) : rows <= 32 ? 1 : 2;
    // what a CU holds at once, by LDS and by registers
    const int tile_bytes = kSwTile * p.Dqk * 2;
    const int lds = w.kept ? sweep_stages(p.Dqk, kModeKeep) * tile_bytes : sweep_stages(p.Dqk, kModeWeights) * tile_bytes + kSwChunk * kSwTile * 4 + 3 * w.waves * kSwTile * 4;
    const int waves_per_cu = 4 * sweep_waves_per_simd(p.Dqk);
    int per_cu = (159 << 10) / lds;
    if (per_cu > waves_per_cu / w.waves) per_cu = waves_per_cu / w.waves;
    if (per_cu < 1) per_cu = 1;
    w.W = 256 * per_cu / p.Hkv;
    if (w.W < 1) w.W = 1;
    if (w.W > kSwMaxStretches) w.W = kSwMaxStretches;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t per_head = static_cast<size_t>(p.Hq) * p.T;          // Hkv * G * T
    w.off_part = up(sizeof(int32_t) * (static_cast<size_t>(p.B) + 2));
    w.off_lse = w.off_part + up(sizeof(float2) * (static_cast<size_t>(w.W) + p.B) * per_head);
    w.off_scores = w.off_lse + up(sizeof(float) * static_cast<size_t>(p.B) * per_head);
    w.total = w.off_scores + sizeof(float) * w.kept * static_cast<size_t>(p.B) * p.Hkv * p.max_pages_per_seq * p.page_size;
    w.total = up(w.total);
    return w;
}

static int check_kv_weights_params(const seer_attn_params* p) {
    if (!p) return SEER_EINVAL;
    if (p->B < 0 || p->num_pages < 1 || p->max_pages_per_seq < 1 || p->page_size < 1) return SEER_EINVAL;
    if (p->T < 1 || p->T > SEER_MAX_T || p->Hq < 1 || p->Hkv < 1 || p->Hq % p->Hkv != 0 || p->Hq > 65535) return SEER_ESHAPE;
    if (!(p->scale > 0.f) || p->scale > 2.0e38f) return SEER_EINVAL;
    if (p->Dqk != 64 && p->Dqk != 128 && p->Dqk != 192 && p->Dqk != 256 && p->Dqk != 576) return SEER_EUNSUPPORTED;
    const int64_t ctx = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size;
    if (ctx > 0x7fffffffLL - 64) return SEER_ESHAPE;
    // units of a line, partial results and workgroups are counted in 32 bits
    const int64_t blocks = (static_cast<int64_t>(p->Hq / p->Hkv) * p->T + 31) / 32;
    if ((static_cast<int64_t>(p->B) + 1) * (ctx / 32 + 1) > 0x7fffffffLL / 2 / blocks || static_cast<int64_t>(p->B) * p->Hq * p->T > 0x7fffffffLL) return SEER_ESHAPE;
    if (static_cast<int64_t>(p->num_pages) * p->Hkv > 0xffffffffLL / p->page_size) return SEER_ESHAPE;
    // and so are the threads of a launch (kv_lse and kv_apply, whose 8192 workgroups come on top, have the most workgroups for many requests)
    const int64_t heads = static_cast<int64_t>(p->B) * p->Hkv, groups = (static_cast<int64_t>(p->Hq / p->Hkv) * p->T + kLseRows - 1) / kLseRows;
    if (heads * groups > 0xffffffffLL / 256 - 8192) return SEER_ESHAPE;
    return SEER_OK;
}

static void launch_kv_lse(const KvWeightsArgs& a, hipStream_t stream) {
    const unsigned groups = static_cast<unsigned>((a.G * a.T + kLseRows - 1) / kLseRows);
    hipLaunchKernelGGL(kv_lse, dim3(static_cast<unsigned>(a.B) * static_cast<unsigned>(a.Hkv) * groups), dim3(kLseThreads), 0, stream, a);
}
template <int DQK, int NW>
hipError_t launch_kv_weights(const KvWeightsArgs& a, int kept, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(a.W) * static_cast<unsigned>(a.Hkv)), block(NW * kWave);
    if constexpr (NW == 1) {
        const int64_t heads = static_cast<int64_t>(a.B) * a.Hkv, most = (8192 + heads - 1) / heads, chunks = (a.ldw + kApplyPositions - 1) / kApplyPositions;
        const int parts = static_cast<int>(chunks < most ? chunks : most);
        const dim3 apply(static_cast<unsigned>(heads * parts));
#define SEER_KEEP(KEPT)                                                                                       \
    if constexpr (KEPT <= DQK / 8)                                                                            \
        if (kept == KEPT) {                                                                                   \
            hipLaunchKernelGGL((kv_sweep<DQK, 1, kModeKeep, KEPT>), grid, block, 0, stream, a);                \
            launch_kv_lse(a, stream);                                                                         \
            hipLaunchKernelGGL((kv_apply<KEPT>), apply, dim3(kApplyThreads), 0, stream, a, parts);             \
            return hipGetLastError();                                                                         \
        }
        SEER_KEEP(4)
        SEER_KEEP(8)
        SEER_KEEP(16)
#undef SEER_KEEP
    }
    if constexpr (DQK <= 256 || NW == 8) {
        hipLaunchKernelGGL((kv_sweep<DQK, NW, kModeSums, 0>), grid, block, 0, stream, a);
        launch_kv_lse(a, stream);
        hipLaunchKernelGGL((kv_sweep<DQK, NW, kModeWeights, 0>), grid, block, 0, stream, a);
    }
    return hipGetLastError();
}

}  // namespace seer

extern "C" size_t seer_kv_weights_workspace(const seer_attn_params* p) {
    if (seer::check_kv_weights_params(p) != SEER_OK || p->B == 0) return 0;
    return seer::kv_weights_layout(*p).total;
}

extern "C" int seer_kv_weights(float* weights, const void* q, const void* k_pages, const int32_t* block_table, const int32_t* ctx_len,
                               const int32_t* accepted_len, const int32_t* accepted_path, float decay, const seer_attn_params* p,
                               int32_t* status, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = seer::check_kv_weights_params(p);
    if (rc != SEER_OK) return rc;
    if (!(decay >= 0.f) || decay > 1.f) return SEER_EINVAL;
    if (p->B == 0) return SEER_OK;
    if (!weights || !q || !k_pages || !block_table || !ctx_len || !accepted_len != !accepted_path) return SEER_EINVAL;
    const seer::KvWeightsLayout w = seer::kv_weights_layout(*p);
    if (!workspace || workspace_bytes < w.total) return SEER_EWORKSPACE;
    auto misaligned = [](const void* ptr, uintptr_t a) { return reinterpret_cast<uintptr_t>(ptr) % a != 0; };
    if (misaligned(q, 16) || misaligned(k_pages, 16) || misaligned(workspace, 256) || misaligned(weights, 4) || misaligned(block_table, 4) ||
        misaligned(ctx_len, 4) || misaligned(accepted_len, 4) || misaligned(accepted_path, 4) || misaligned(status, 4))
        return SEER_EALIGN;
    char* ws = static_cast<char*>(workspace);
    seer::KvWeightsArgs a{};
    a.weights = weights, a.q = q, a.k_pages = k_pages, a.block_table = block_table, a.ctx_len = ctx_len;
    a.accepted_len = accepted_len, a.accepted_path = accepted_path, a.status = status;
    a.line = reinterpret_cast<int32_t*>(ws);
    a.part = reinterpret_cast<float2*>(ws + w.off_part);
    a.lse = reinterpret_cast<float*>(ws + w.off_lse);
    a.scores = reinterpret_cast<float*>(ws + w.off_scores);
    a.ldw = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size;
    a.B = p->B, a.T = p->T, a.Hq = p->Hq, a.Hkv = p->Hkv, a.G = p->Hq / p->Hkv, a.P = p->page_size;
    a.num_pages = p->num_pages, a.max_pages = p->max_pages_per_seq, a.max_ctx = static_cast<int>(a.ldw);
    a.W = w.W, a.block_rows = 32 * w.waves;

    a.scale_log2 = p->scale * seer::kLog2e, a.decay = decay;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (w.whole) {
        const int stride = static_cast<int>((a.ldw + 31) / 32 * 32 + 4);
        const unsigned lds = static_cast<unsigned>(sizeof(float) * stride * a.G * a.T);
        const dim3 grid(static_cast<unsigned>(p->B) * static_cast<unsigned>(p->Hkv)), block(seer::kShortWaves * seer::kWave);
#define SEER_SHORT(DQK)                                                                                                        \
    if (p->Dqk == DQK) {                                                                                                       \
        hipLaunchKernelGGL(seer::kv_short<DQK>, grid, block, lds, stream, a, stride);                                          \
        return static_cast<int>(hipGetLastError());                                                                            \
    }
        SEER_SHORT(64)
        SEER_SHORT(128)
        SEER_SHORT(192)
        SEER_SHORT(256)
#undef SEER_SHORT
    }
#define SEER_SWEEP(DQK, NW) \
    if (p->Dqk == DQK && w.waves == NW) return static_cast<int>(seer::launch_kv_weights<DQK, NW>(a, w.kept, stream));
#define SEER_SWEEPS(DQK) SEER_SWEEP(DQK, 1) SEER_SWEEP(DQK, 2)
    SEER_SWEEPS(64)
    SEER_SWEEPS(128)
    SEER_SWEEPS(192)
    SEER_SWEEPS(256)
    SEER_SWEEP(576, 1)
    SEER_SWEEP(576, 8)
#undef SEER_SWEEPS
#undef SEER_SWEEP
    return SEER_EUNSUPPORTED;
}
