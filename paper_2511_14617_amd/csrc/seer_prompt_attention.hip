// Causal attention of packed tokens over the paged cache, separate K and V pools: (64, 64), (128, 128), (192, 128) and (256, 256),
// pages of any size.
//
// out = sum_j p_j V_j / sum_j p_j, p_j = exp(scale q.K_j - m) over the positions j that a token sees (those before it and itself), in one pass: a
// running reference m, sums and outputs in fp32.  Positions that no row of the tile sees are not read, a cached row is read once per row tile.
//
// Workgroup = 4 waves = a row tile of 128 query rows of one KV head, 32 rows a wave (8 waves and 256 rows where there are many); the work is cut into equal stretches of a line
// of row tiles (seer_prompt.h).  A tile of 32 positions goes HBM/L2 -> LDS directly into rings of four tiles, three of them in flight.  S^T = K.Q^T
// leaves a query row to a lane pair, so its softmax needs one exchange between two lanes, and the probabilities are, packed to bf16 (the matrix
// operand's type; the sum is taken of the rounded values, so what is common cancels), the operand of O^T += V^T.P^T as they are.
//
// Neighbouring tiles run side by side: behind every MFMA of the scores of tile u stand a K read for a later one and a few of tile u - 1's probabilities,
// behind those of its product with V the rest of them and the highest scores of tile u.  Before that, scores, softmax and product of a tile one
// after the other, one prompt of 32 768 tokens on 8/1 heads of 128 took 3.09 ms; side by side 2.67; with the arithmetic pinned beside its
// MFMA 2.53; with waits and loads without conditions and descriptors in scalar registers 2.25; with today's shares of the line 2.17; with eight waves on a
// tile 2.06 (1067 TFLOP/s, where an 8192^3 bf16 library product reaches 1378).
//
// What bounds it: the power that matrix cores, LDS and vector ALU take together.  In that prompt, with four waves a workgroup, the matrix cores are busy 56 % of
// the time, vector instructions 47 %, LDS 30 % (0.15 % of it conflicts), at 1.79 GHz instead of 2.4, and changes that saved cycles lowered the clock by nearly
// as much: without the exponentials the time is 1 % less, without tile loads 13 to 19, without the product with V 15; earlier K reads, loads in the shadow of the
// scores' MFMAs, other shares of probabilities, wave priorities changed nothing.  Eight waves take 4 % more cycles (54 % busy) and half the loads, at 1.92 GHz.
// Requests of one token are bound by HBM where they are alone: 64 of 16 384 positions on 8 KV heads read 4.8 TB/s (loads that stream past the caches gain 4 % there and cost
// prompts 30 %, which share what they read: not used).  A row tile costs its matrix work whether it has rows or not, though: one token on 32/8 heads has 4 rows, and the waves without
// rows compute scores and products of zeros.  Beside a piece of a prompt that takes power from it: 2048 tokens behind 16 384 and 63 single tokens need 1.15 TFLOP, the kernel executes 1.73
// (by its count of MFMAs), 0.6 of them for single tokens, at the 930 TFLOP/s that it reaches with prompts.
//
// Infinities and NaN: scores of positions that a row does not see are replaced by selection.  In the product with V a position's row is
// multiplied into all query rows, so in tiles with masked positions V rows that hold an infinity or NaN are taken out and added to the rows that see
// them.
#include <type_traits>

#include "seer_device.h"
#include "seer_prompt.h"
#include "seer_tile.h"

namespace seer {

// Slots of the K ring and of the V ring, one tile of 32 positions each: K of tile u and V of tile u - 1 are read in step u, so each ring
// has three tiles in flight behind the one in use.
constexpr int kSlots = 4;

template <int DQK, int DV, int WAVES>
struct PromptShape {
    static constexpr int kTile = 32;
    static constexpr int kKRow = DQK * 2, kVRow = DV * 2;                     // bytes of a position's row
    static constexpr int kKSlot = kTile * kKRow, kVSlot = kTile * kVRow;
    static constexpr int kVBase = kSlots * kKSlot;                           // the V ring follows the K ring
    static constexpr int kLds = kSlots * (kKSlot + kVSlot);
    static constexpr int kKSteps = DQK / 16, kDTiles = DV / 32, kPv = 2 * kDTiles;      // contraction steps; d-tiles; MFMAs of a product
    static constexpr int kRows = 32 * WAVES;                                 // of a row tile
    static constexpr int kMine = kTile / WAVES;                              // positions of a tile that a wave loads
    static constexpr int kKLoads = kKSlot / (1024 * WAVES), kVLoads = kVSlot / (1024 * WAVES);   // of 1 KB, per wave and tile
    static constexpr int kKAhead = kKSteps < 8 ? kKSteps : 8;                // K operands requested ahead of their MFMA
    static constexpr int kVAhead = kPv < 8 ? kPv : 8;                        // V operands (two reads each)
    // Waves that a SIMD holds, by registers (queries, outputs, scores of two tiles, operands) and LDS.  Heads of 192/128 with one: 531 us for four sequences
    // of 4096 on 16 heads, with two 431.
    static constexpr int kWavesPerSimd = DQK <= 64 ? 3 : (DQK <= 192 ? 2 : 1);
    static_assert(kKSlot % (1024 * WAVES) == 0 && kVSlot % (1024 * WAVES) == 0 && kLds <= 156 * 1024, "");
};

// One LDS read whose completion is waited for by count (LDS answers in order; see wait_lgkm): through the builtins the compiler would wait for the
// tile loads in flight, which it cannot tell apart.  Every result is used behind such a wait in the same straight line of code.
#define SEER_PROMPT_READ128(dst, addr, OFF) asm volatile("ds_read_b128 %0, %1 offset:%2" : "=&v"(dst) : "v"(addr), "n"(OFF))
#define SEER_PROMPT_READ_TR(dst, addr, OFF_LO, OFF_HI)                \
    asm volatile("ds_read_b64_tr_b16 %0, %2 offset:%3\n"              \
                 "ds_read_b64_tr_b16 %1, %2 offset:%4"                \
                 : "=&v"(dst[0]), "=&v"(dst[1])                       \
                 : "v"(addr), "n"(OFF_LO), "n"(OFF_HI))
// Keeps the computation of x where it is written: it would be moved behind the next branch, out of the shadow of the MFMAs.
#define SEER_PROMPT_PIN(x) asm volatile("" : "+v"(x))
template <int N>
__device__ __forceinline__ void wait_reads() {
    static_assert(N >= 0 && N < 16, "lgkmcnt is a 4-bit counter");
    __builtin_amdgcn_s_waitcnt(0xc07f | (N << 8));
    __builtin_amdgcn_sched_barrier(0);
}
template <int N>
using I = std::integral_constant<int, N>;
template <typename F, int... N>
__device__ __forceinline__ void each_index(F&& f, std::integer_sequence<int, N...>) {
    (f(I<N>{}), ...);
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const unsigned char* p, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(p), 0, bytes, 0x00020000);
}
__device__ __forceinline__ void load_to_lds(__amdgpu_buffer_rsrc_t rsrc, unsigned char* to, int offset) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (SEER_AS3 void*)(to), 16, offset, 0, 0, 0);
}
// Requests a wave's MINE rows of a tile: at_row = row of the pool of the first of them (ANY_PAGE: of the tile's position lane % 32).
template <int ROW, int LOADS, int MINE, bool ANY_PAGE>
__device__ __forceinline__ void issue_rows(const unsigned char* pool, uint32_t at_row, const int (&pat)[LOADS], unsigned char* slot, int wave, int lane) {
    if constexpr (ANY_PAGE) {
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int r = (j * kWave + lane) / (ROW / 16);
            const uint32_t from = __builtin_amdgcn_ds_bpermute((wave * MINE + r) << 2, at_row);
            const unsigned char* src = pool + static_cast<size_t>(from) * ROW + (pat[j] - r * ROW);
            __builtin_amdgcn_global_load_lds((const SEER_AS1 void*)(src), (SEER_AS3 void*)(slot + (wave * LOADS + j) * 1024), 16, 0, 0);
        }
    } else {
        const __amdgpu_buffer_rsrc_t rsrc = rows_at(pool + static_cast<size_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(at_row))) * ROW, MINE * ROW);
#pragma unroll
        for (int j = 0; j < LOADS; ++j) load_to_lds(rsrc, slot + (wave * LOADS + j) * 1024, pat[j]);
    }
}

// ANY_PAGE: pages of any size; else of a multiple of 16 positions, so that the rows of a tile that a wave loads lie in one page.
// WAVES: four, or eight with 256 query rows, which read the same tile.
template <int DQK, int DV, bool ANY_PAGE, int WAVES>
__global__ __launch_bounds__(WAVES * kWave) __attribute__((amdgpu_waves_per_eu(PromptShape<DQK, DV, WAVES>::kWavesPerSimd)))
void prompt_tile_kernel(PromptArgs a) {
    using S = PromptShape<DQK, DV, WAVES>;
    using O = tile::Operands<DQK, DV>;
    using tile::k_swz;
    using tile::v_swz;
    constexpr int kTile = S::kTile;
    // (nothing beside the rings: two workgroups of the 192/128 shape take all 160 KB of a CU; the plan's words lie where the rings come)
    __shared__ __attribute__((aligned(1024))) unsigned char lds[S::kLds];
    PromptLds& s_plan = *reinterpret_cast<PromptLds*>(lds);
    const int tid = threadIdx.x, lane = tid & (kWave - 1), ln = lane & 31, lg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    int w, error = 0;
    PromptPlan plan;
    int64_t x, x_end;
    PromptTile t;
    {
        int64_t at[2];
        PromptTile ends[2];
        const bool on = prompt_plan<WAVES * kWave>(a, s_plan, w, plan, at, ends, error);
        if (blockIdx.x == 0 && error && a.status) atomicOr(a.status, error);
        if (!on) return;
        x = moved_cut(plan, ends[0], at[0]);
        x_end = moved_cut(plan, ends[1], at[1]);
        t = ends[0];
        PromptCut cut{0, 0, 0, 0};                  // the row tile that begins in this stretch and goes on behind it
        if (x_end > ends[1].begin && x_end < ends[1].begin + ends[1].cost && ends[1].begin >= x && !ends[1].r.bad)
            cut = PromptCut{ends[1].b, ends[1].kvh, ends[1].i, pieces_of(plan, ends[1], w)};
        if (tid == 0) a.cuts[w] = cut;
        // (w is wanted next where a partial result is stored: in a vector register; in a scalar one it takes others' place through the tiles, 0.5 % of the time)
        asm volatile("" : "+v"(w));
    }
    bool bad_page = false;
    // ANY_PAGE: window of page ids: request, first logical page; lane l holds the (clamped) id of page win + l.
    // Else a window of rows: request, KV head, first tile; lane l holds the row of the pool where tile win + l's first position of this wave is; and the window of the request's
    // first tiles, with which most row tiles begin.
    int win_b = -1, win_h = -1, win = 0, in_win = 0, first_win = 0;
    const int lds0 = tile::lds_addr(lds);
    auto page_of = [&](int position) __attribute__((always_inline)) -> int { return prompt_page(a, position); };

    // ---- what stays for the whole stretch: operand addresses, byte offsets of this lane's loads in its wave's eight rows ----------
    const O operands;
    int k_at[O::kPerXor], v_at[O::kPerV], k_pat[S::kKLoads], v_pat[S::kVLoads];
#pragma unroll
    for (int i = 0; i < O::kPerXor; ++i) k_at[i] = (lds0 + operands.k_rd) ^ (i << 5);
#pragma unroll
    for (int i = 0; i < O::kPerV; ++i) v_at[i] = (lds0 + S::kVBase + (operands.v_rd - tile::Shape<DQK, DV>::kKBytes)) ^ (i << 6);
#pragma unroll
    for (int j = 0; j < S::kKLoads; ++j) {
        const int c = j * kWave + lane, r = c / (S::kKRow / 16), pos = c - r * (S::kKRow / 16);
        k_pat[j] = r * S::kKRow + ((pos ^ k_swz<S::kKRow>(wave * S::kMine + r)) << 4);
    }
#pragma unroll
    for (int j = 0; j < S::kVLoads; ++j) {
        const int c = j * kWave + lane, r = c / (S::kVRow / 16), pos = c - r * (S::kVRow / 16);
        v_pat[j] = r * S::kVRow + ((pos ^ v_swz<S::kVRow>(wave * S::kMine + r)) << 4);
    }

    while (x < x_end) {
        if (x >= t.begin + t.cost) next_tile<WAVES * kWave>(a, t);
        const int64_t end = min(x_end, t.begin + t.cost);
        const bool begins = x == t.begin, ends = end == t.begin + t.cost;
        // (rows of q are counted in 32 bits)
        const uint32_t row0 = static_cast<uint32_t>(t.i) * S::kRows;
        const int rows = static_cast<int>(min(static_cast<uint32_t>(t.r.n) * static_cast<uint32_t>(a.G) - row0, static_cast<uint32_t>(S::kRows)));
        const int token_first = prompt_token(a, row0), token_last = prompt_token(a, row0 + rows - 1);              // of the request's new tokens
        const int seen = static_cast<int>(t.r.past) + token_last + 1;                                              // positions that the last row sees
        const int all_see = static_cast<int>(t.r.past) + token_first;                                              // the last one that all rows see
        const int tiles = t.r.bad ? 0 : (seen + kTile - 1) / kTile;
        // the piece's tiles (the same rounding on both sides of a cut)
        int u0 = 0, u1 = tiles;
        if (!begins) u0 = static_cast<int>(static_cast<double>(x - t.begin) * tiles / static_cast<double>(t.cost));
        if (!ends) u1 = static_cast<int>(static_cast<double>(end - t.begin) * tiles / static_cast<double>(t.cost));
        x = end;
        if (t.r.bad && !begins) continue;
        const int n_tiles = u1 - u0, tok_begin = u0 * kTile;

        // ---- this lane's query row -------------------------------------------------------------------------
        const uint32_t row = row0 + wave * 32 + ln;
        const bool row_ok = wave * 32 + ln < rows;
        const int token = row_ok ? prompt_token(a, row) : 0;
        const uint32_t q_row = static_cast<uint32_t>(t.r.first + token) * a.Hq + t.kvh * a.G + (row_ok ? row - static_cast<uint32_t>(token) * a.G : 0u);
        const int sees = row_ok ? static_cast<int>(t.r.past) + token : -1;                                         // last position that it sees
        const int sees_lo = __builtin_amdgcn_readfirstlane(sees);                                                  // the wave's first row
        f32x16 acc[S::kDTiles];
#pragma unroll
        for (int dt = 0; dt < S::kDTiles; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
        float m_run = kNoScore, l_run = 0.f;
        __syncthreads();                            // every wave is done with the rings of the piece before
        if (n_tiles > 0) {
            u32x4 qreg[S::kKSteps];
            {
                const u32x4* qp = reinterpret_cast<const u32x4*>(a.q + static_cast<size_t>(q_row) * DQK + lg * 8);
#pragma unroll
                for (int kk = 0; kk < S::kKSteps; ++kk) {
                    qreg[kk] = u32x4{0u, 0u, 0u, 0u};
                    if (row_ok) qreg[kk] = qp[kk * 2];
                }
            }
            // ---- tile loads --------------------------------------------------------------------------------
            const int32_t* table = a.block_table + static_cast<size_t>(t.b) * a.max_pages;
            const int last_page = page_of(static_cast<int>(t.r.past) + t.r.n - 1);
            const int last = static_cast<int>(t.r.past) + t.r.n - 1;
            auto set_window = [&](int first) __attribute__((always_inline)) {
                win = first;
                int pg;
                if constexpr (ANY_PAGE) {
                    pg = table[min(first + lane, a.max_pages - 1)];
                    if ((pg < 0 || pg >= a.num_pages) && first + lane <= last_page) bad_page = true;
                    in_win = min(max(pg, 0), a.num_pages - 1);
                } else {
                    // (behind the request's last position: its last ones again)
                    const int position = min((first + lane) * kTile + wave * S::kMine, last & ~(S::kMine - 1)), lp = page_of(position);
                    pg = table[lp];
                    if (pg < 0 || pg >= a.num_pages) bad_page = true;
                    pg = min(max(pg, 0), a.num_pages - 1);
                    in_win = static_cast<int>((static_cast<uint32_t>(pg) * a.Hkv + t.kvh) * static_cast<uint32_t>(a.P) + static_cast<uint32_t>(position - lp * a.P));
                    if (first == 0) first_win = in_win;
                }
            };
            // Row of the pool (of 128 bytes or more each: 32 bits reach past the memory of the GPU) of tile u's first position of this wave; ANY_PAGE: of position ln.
            // Tiles are asked for in ascending order.
            auto tile_row = [&](int u) __attribute__((always_inline)) -> uint32_t {
                if constexpr (ANY_PAGE) {
                    const int tb = tok_begin + u * kTile;
                    if (page_of(tb) < win || page_of(tb + kTile - 1) >= win + kWave) set_window(page_of(tb));      // (uniform; a tile spans at most 32 pages)
                    const int lp = page_of(tb + ln);
                    const int pg = __builtin_amdgcn_ds_bpermute((lp - win) << 2, in_win);
                    return (static_cast<uint32_t>(pg) * a.Hkv + t.kvh) * static_cast<uint32_t>(a.P) + static_cast<uint32_t>(tb + ln - lp * a.P);
                } else {
                    if (u0 + u - win >= kWave) set_window(u0 + u);
                    return __builtin_amdgcn_readlane(in_win, u0 + u - win);
                }
            };
            auto issue_k = [&](int u, uint32_t at_row) __attribute__((always_inline)) {
                issue_rows<S::kKRow, S::kKLoads, S::kMine, ANY_PAGE>(a.k_pages, at_row, k_pat, lds + (u & (kSlots - 1)) * S::kKSlot, wave, lane);
            };
            auto issue_v = [&](int u, uint32_t at_row) __attribute__((always_inline)) {
                issue_rows<S::kVRow, S::kVLoads, S::kMine, ANY_PAGE>(a.v_pages, at_row, v_pat, lds + S::kVBase + (u & (kSlots - 1)) * S::kVSlot, wave, lane);
            };

            // ---- softmax ------------------------------------------------------------------------------------
            f32x16 s_a, s_b = {};
            uint32_t pk[8];
            // The exponent reference of a row: a score near its highest so far.  It moves only when a score exceeds it by more than 8 in units of log2 e
            // (probabilities stay below 2^8, which bf16 and fp32 hold as well as any), so that outputs are seldom rescaled and the arithmetic of a move stands in a
            // branch.  m_run: the reference as a raw score; m_use: scaled, what is taken from a scaled score in one fma.  m_use is rounded, which no other tile
            // or piece knows of: up to 2^10 that is 2^-15 at most in the exponent, far below the probabilities' own rounding; beyond, the raw reference is taken from the
            // raw scores first (far).
            float m_use = 0.f, alpha = 1.f, mx = 0.f;
            bool moved = false, far = false;        // uniform: alpha is not 1 for some row
            auto highest = [&](auto partc, const f32x16& s) __attribute__((always_inline)) {
                constexpr int part = decltype(partc)::value;
                if constexpr (part == 0) {
                    mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
                    for (int i = 3; i < 9; i += 2) mx = fmaxf(fmaxf(mx, s[i]), s[i + 1]);
                } else if constexpr (part == 1) {
#pragma unroll
                    for (int i = 9; i < 15; i += 2) mx = fmaxf(fmaxf(mx, s[i]), s[i + 1]);
                    mx = fmaxf(mx, s[15]);
                } else {
                    mx = max_across_halves(mx);
                }
            };
            auto reference = [&](f32x16& s) __attribute__((always_inline)) {
                const bool moves = mx > m_run + a.move_at;
                moved = __any(moves);
                if (moved) {
                    const float m_new = moves ? mx : m_run;
                    alpha = fast_exp2((m_run - m_new) * a.scale_log2);
                    m_run = m_new;
                    m_use = m_new == kNoScore ? 0.f : m_new * a.scale_log2;
                    far = far || __any(fabsf(m_use) > 1024.f);
                }
                if (far) {
                    m_use = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] -= m_run;
                }
            };
            // -inf into the scores of tile u that this lane's row does not see
            auto mask = [&](int u, f32x16& s) __attribute__((always_inline)) {
                const int tb = tok_begin + u * kTile;
                if (tb + kTile - 1 <= sees_lo) return;                 // (wave-uniform)
                const int lim = sees - tb;          // last position of the tile that the row sees
                uint32_t vis = lim < 0 ? 0u : (lim >= 31 ? 0xffffffffu : (2u << lim) - 1u);
                vis >>= lg * 4;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((vis >> ((i >> 2) * 8 + (i & 3))) & 1u)) s[i] = kNegInf;
            };
            float psum = 0.f, p_even = 0.f;
            auto probability = [&](auto ic, const f32x16& s) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                const float p = fast_exp2(fmaf(s[i], a.scale_log2, -m_use));
                if constexpr (i % 2 == 0) {
                    p_even = p;
                    SEER_PROMPT_PIN(p_even);
                    if constexpr (i >= 2) {         // the sum of what the product will see, one pair behind
                        psum = add_bf16_pair(pk[(i >> 1) - 1], psum);
                        SEER_PROMPT_PIN(psum);
                    }
                } else {
                    pk[i >> 1] = cvt_pk_bf16(p_even, p);
                    SEER_PROMPT_PIN(pk[i >> 1]);
                }
            };

            // ---- V rows with infinities or NaN of the tile in V slot `slot_at` (tile u), where some row does not see all of it ----------
            uint32_t left = 0;                      // uniform: positions whose V row is kept out of the product
            auto scan = [&](int u, int slot_at) __attribute__((always_inline)) {
                left = 0;
                if (tok_begin + u * kTile + kTile - 1 <= all_see) return;
                unsigned char* vl = lds + S::kVBase + slot_at;
                // (where the tile's K was, which all waves have left: the next K goes there behind this)
                uint32_t* found_in = reinterpret_cast<uint32_t*>(lds + (u & (kSlots - 1)) * S::kKSlot);
                if (tid == 0) *found_in = 0;
                wait_reads<0>();
                bare_barrier();
                const uint32_t found = tile::tile_nonfinite<DQK, DV>(vl, tid, WAVES * kWave);
                if (found) atomicOr(found_in, found);
                wait_reads<0>();
                bare_barrier();
                left = __builtin_amdgcn_readfirstlane(*const_cast<volatile uint32_t*>(found_in));
                if (left) {
                    tile::tile_clear_rows<DQK, DV>(vl, left, tid, WAVES * kWave);
                    wait_reads<0>();
                }
                bare_barrier();
            };

            // ---- step u: scores of tile u beside the probabilities of tile u - 1, then the product with V of tile u - 1 beside the loads and
            // the reference of tile u ----------------------------------------------------------------------------------------------------
            uint32_t row2 = 0;                      // row of tile u + 2: its K was requested in the step before
            // (SURE: u + 2 < n_tiles, and for the loads u + 3 < n_tiles)
            auto top = [&](auto surec, int u) __attribute__((always_inline)) {
                constexpr int K = S::kKLoads, V = S::kVLoads;        // loads that may be in flight behind those of K of tile u and V of tile u - 1
                if (decltype(surec)::value || u + 2 < n_tiles) wait_vmcnt<2 * K + 2 * V>();
                else if (u + 1 < n_tiles) wait_vmcnt<K + 2 * V>();
                else if (u < n_tiles) wait_vmcnt<V>();
                else wait_vmcnt<0>();
                bare_barrier();                     // they have landed for every wave, every wave is done with step u - 1
            };
            auto loads = [&](auto surec, int u) __attribute__((always_inline)) {
                uint32_t row3 = 0;
                if (decltype(surec)::value || u + 3 < n_tiles) {
                    row3 = tile_row(u + 3);
                    issue_k(u + 3, row3);
                }
                if (decltype(surec)::value || u + 2 < n_tiles) issue_v(u + 2, row2);
                row2 = row3;
            };
            u32x2 vr[S::kVAhead][2];
            // V operand m of a product (positions of half m / kDTiles, d-tile m % kDTiles) into its ring slot
            auto read_v = [&](auto mc, auto slotc, int shift) __attribute__((always_inline)) {
                constexpr int m = decltype(mc)::value, dt = m % S::kDTiles, half = m / S::kDTiles;
                constexpr int off = decltype(slotc)::value * S::kVSlot + dt / O::kPerV * (O::kPerV * 64) + half * 16 * S::kVRow;
                (void)&vr;
                const int from = v_at[dt % O::kPerV] + shift;
                SEER_PROMPT_READ_TR(vr[m % S::kVAhead], from, off, off + 8 * S::kVRow);
            };
            auto product = [&](auto slotc, int shift, auto&& beside) __attribute__((always_inline)) {
                each_index([&](auto mc) __attribute__((always_inline)) {
                    constexpr int m = decltype(mc)::value, later = S::kPv - 1 - m;
                    wait_reads<2 * (later < S::kVAhead - 1 ? later : S::kVAhead - 1)>();
                    const bf16x8 v = as_bf16x8(u32x4{vr[m % S::kVAhead][0][0], vr[m % S::kVAhead][0][1], vr[m % S::kVAhead][1][0], vr[m % S::kVAhead][1][1]});
                    constexpr int dt = m % S::kDTiles, h = m / S::kDTiles * 4;
                    acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, as_bf16x8(u32x4{pk[h], pk[h + 1], pk[h + 2], pk[h + 3]}), acc[dt], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (m + S::kVAhead < S::kPv) read_v(std::integral_constant<int, m + S::kVAhead>{}, slotc, shift);
                    beside(mc);
                    __builtin_amdgcn_sched_barrier(0);
                }, std::make_integer_sequence<int, S::kPv>{});
            };
            auto rescale = [&]() __attribute__((always_inline)) {
                if (moved) {
                    l_run *= alpha;
#pragma unroll
                    for (int dt = 0; dt < S::kDTiles; ++dt)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
                }
            };
            auto add_left = [&](int u) __attribute__((always_inline)) {
                if (!left) return;
                const int tb = tok_begin + u * kTile, lim = sees - tb;
                const uint64_t word = lim < 0 ? 0 : (lim >= 31 ? 0xffffffffull : (2ull << lim) - 1);
                uint32_t term[1][8];
#pragma unroll
                for (int i = 0; i < 8; ++i) term[0][i] = pk[i];
                tile::tile_add_rows<1>(left, term, word, 0, acc, [&](int j) __attribute__((always_inline)) -> const uint16_t* {
                    const int lp = page_of(tb + j);
                    const int pg = min(max(table[min(lp, a.max_pages - 1)], 0), a.num_pages - 1);
                    return reinterpret_cast<const uint16_t*>(a.v_pages) + ((static_cast<size_t>(pg) * a.Hkv + t.kvh) * a.P + (tb + j - lp * a.P)) * DV;
                });
            };
            // The step itself, behind top(): K of tile u in slot SLOT (+ k_shift), V of tile u - 1 in slot BEFORE (+ v_shift).  PREV: there is a tile
            // u - 1; EDGE, MASK: that some rows do not see all of tile u - 1, of tile u.
            auto step = [&](auto slotc, auto beforec, auto prevc, auto edgec, auto maskc, auto surec, int u, int k_shift, int v_shift, f32x16& s_new, const f32x16& s_old) __attribute__((always_inline)) {
                constexpr int SLOT = decltype(slotc)::value, kEarly = 10;          // probabilities beside the scores' MFMAs
                constexpr bool PREV = decltype(prevc)::value, EDGE = decltype(edgec)::value, MASK = decltype(maskc)::value;
                u32x4 kr[S::kKAhead];
                each_index([&](auto kc) __attribute__((always_inline)) {
                    constexpr int kk = decltype(kc)::value;
                    (void)&kr;                      // (asm operands alone do not capture)
                    const int from = k_at[kk % O::kPerXor] + k_shift;
                    SEER_PROMPT_READ128(kr[kk], from, SLOT * S::kKSlot + kk / O::kPerXor * (O::kPerXor * 32));
                }, std::make_integer_sequence<int, S::kKAhead>{});
                __builtin_amdgcn_sched_barrier(0);
                loads(surec, u);
                __builtin_amdgcn_sched_barrier(0);
                psum = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) s_new[i] = 0.f;
                each_index([&](auto kc) __attribute__((always_inline)) {
                    constexpr int kk = decltype(kc)::value;
                    (void)&kr;
                    // behind K operand kk: the K operands requested since, and the V operands, a pair behind each MFMA from kVFirst on
                    constexpr int kAfter = S::kKSteps - 1 - kk < S::kKAhead - 1 ? S::kKSteps - 1 - kk : S::kKAhead - 1;
                    constexpr int kVFirst = S::kKSteps - S::kVAhead;
                    constexpr int kVSoFar = PREV && kk > kVFirst ? 2 * (kk - kVFirst) : 0;
                    static_assert(kVFirst >= S::kKSteps - S::kKAhead && kAfter + kVSoFar < 16, "");
                    wait_reads<kAfter + kVSoFar>();
                    s_new = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(kr[kk % S::kKAhead]), as_bf16x8(qreg[kk]), s_new, 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (kk + S::kKAhead < S::kKSteps) {
                        const int from = k_at[(kk + S::kKAhead) % O::kPerXor] + k_shift;
                        SEER_PROMPT_READ128(kr[kk % S::kKAhead], from, SLOT * S::kKSlot + (kk + S::kKAhead) / O::kPerXor * (O::kPerXor * 32));
                    }
                    if constexpr (PREV && kk >= kVFirst) read_v(std::integral_constant<int, kk - kVFirst>{}, beforec, v_shift);
                    if constexpr (PREV) {
                        constexpr int e0 = kEarly * kk / S::kKSteps, e1 = kEarly * (kk + 1) / S::kKSteps;
                        each_index([&](auto ec) __attribute__((always_inline)) { probability(std::integral_constant<int, e0 + decltype(ec)::value>{}, s_old); },
                                   std::make_integer_sequence<int, e1 - e0>{});
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }, std::make_integer_sequence<int, S::kKSteps>{});
                if constexpr (PREV) {
                    rescale();
                    __builtin_amdgcn_sched_barrier(0);
                    product(beforec, v_shift, [&](auto mc) __attribute__((always_inline)) {
                        // beside the first half the other probabilities, which the second half takes; beside that the highest scores of tile u
                        constexpr int m = decltype(mc)::value, kHalf = S::kDTiles;
                        if constexpr (m < kHalf) {
                            constexpr int e0 = kEarly + (16 - kEarly) * m / kHalf, e1 = kEarly + (16 - kEarly) * (m + 1) / kHalf;
                            each_index([&](auto ec) __attribute__((always_inline)) { probability(I<e0 + decltype(ec)::value>{}, s_old); },
                                       std::make_integer_sequence<int, e1 - e0>{});
                        }
                        if constexpr (m == kHalf) l_run = add_bf16_pair(pk[7], psum) + l_run;
                        constexpr int r0 = m < kHalf ? 0 : 3 * (m - kHalf) / kHalf, r1 = m < kHalf ? 0 : 3 * (m + 1 - kHalf) / kHalf;
                        if constexpr (!MASK && r1 > r0)
                            each_index([&](auto rc) __attribute__((always_inline)) { highest(I<r0 + decltype(rc)::value>{}, s_new); },
                                       std::make_integer_sequence<int, r1 - r0>{});
                    });
                    if constexpr (EDGE) add_left(u - 1);
                }
                if constexpr (MASK) mask(u, s_new);
                if constexpr (MASK || !PREV) each_index([&](auto ic) __attribute__((always_inline)) { highest(ic, s_new); }, std::make_integer_sequence<int, 3>{});
                reference(s_new);
            };

            // the first tiles: K of 0, 1, 2 and V of 0, 1, in the order in which steps -3, -2, -1 would request them
            if constexpr (ANY_PAGE) {
                if (t.b != win_b) win_b = t.b, set_window(page_of(tok_begin));      // (else the window may do)
            } else if (t.b == win_b && t.kvh == win_h && u0 == 0) {
                win = 0, in_win = first_win;
            } else {
                win_b = u0 == 0 ? t.b : -1, win_h = t.kvh;
                set_window(u0);
            }
            {
                const uint32_t row0 = tile_row(0);
                uint32_t row1 = 0;
                issue_k(0, row0);
                if (n_tiles > 1) row1 = tile_row(1), issue_k(1, row1);
                issue_v(0, row0);
                if (n_tiles > 2) row2 = tile_row(2), issue_k(2, row2);
                if (n_tiles > 1) issue_v(1, row1);
            }
            using yes = std::true_type;
            using no = std::false_type;
            top(no{}, 0);
            step(I<0>{}, I<0>{}, no{}, no{}, yes{}, no{}, 0, 0, 0, s_a, s_b);
            // tiles that every row sees whole, with the next ones requested in any case, slots at fixed places; then the others
            const int whole = min(n_tiles - 3, (all_see + 1 - tok_begin) / kTile);      // (below 0: none)
            int u = 1;
            for (; u + 3 < whole; u += 4) {
                top(yes{}, u);
                step(I<1>{}, I<0>{}, yes{}, no{}, no{}, yes{}, u, 0, 0, s_b, s_a);
                top(yes{}, u + 1);
                step(I<2>{}, I<1>{}, yes{}, no{}, no{}, yes{}, u + 1, 0, 0, s_a, s_b);
                top(yes{}, u + 2);
                step(I<3>{}, I<2>{}, yes{}, no{}, no{}, yes{}, u + 2, 0, 0, s_b, s_a);
                top(yes{}, u + 3);
                step(I<0>{}, I<3>{}, yes{}, no{}, no{}, yes{}, u + 3, 0, 0, s_a, s_b);
            }
            for (; u < n_tiles; ++u) {
                top(no{}, u);
                scan(u - 1, ((u - 1) & (kSlots - 1)) * S::kVSlot);
                step(I<0>{}, I<0>{}, yes{}, yes{}, yes{}, no{}, u, (u & (kSlots - 1)) * S::kKSlot, ((u - 1) & (kSlots - 1)) * S::kVSlot, s_b, s_a);
#pragma unroll
                for (int i = 0; i < 16; ++i) s_a[i] = s_b[i];
            }
            // the last tile's probabilities and product
            top(no{}, n_tiles);
            const int shift = ((n_tiles - 1) & (kSlots - 1)) * S::kVSlot;
            scan(n_tiles - 1, shift);
            each_index([&](auto mc) __attribute__((always_inline)) { read_v(mc, I<0>{}, shift); }, std::make_integer_sequence<int, S::kVAhead>{});
            __builtin_amdgcn_sched_barrier(0);
            psum = 0.f;
            each_index([&](auto ec) __attribute__((always_inline)) { probability(ec, s_a); }, std::make_integer_sequence<int, 16>{});
            rescale();
            l_run += add_bf16_pair(pk[7], psum);
            __builtin_amdgcn_sched_barrier(0);
            product(I<0>{}, shift, [](auto) {});
            add_left(n_tiles - 1);
        }

        // ---- the row tile's output, or this piece's share of it ------------------------------------------
        const float l_tot = l_run + __shfl_xor(l_run, 32, kWave);
        if (begins && (ends || t.r.bad)) {
            const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;          // (a row of nothing but -inf: zeros)
            // through LDS, so that a store takes whole rows: 16-byte chunk c of row r at c ^ r (its low bits)
            constexpr int kChunks = DV / 8, kPerStore = kWave / (kChunks < kWave ? kChunks : kWave);      // rows of a store
            static_assert(S::kRows * DV * 2 <= S::kLds, "");
            int l = lane;
            asm volatile("" : "+v"(l));             // (the addresses below are made here, not kept in registers through the tiles)
            const int row_l = l & 31;
            unsigned char* mine = lds + wave * (32 * DV * 2);
            __syncthreads();                        // every wave is done with the rings
#pragma unroll
            for (int dt = 0; dt < S::kDTiles; ++dt)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4)
                    *reinterpret_cast<u32x2*>(mine + row_l * (DV * 2) + (((dt * 4 + i4) ^ (row_l & (kChunks - 1) & 15)) << 4) + (l >> 5) * 8) =
                        u32x2{cvt_pk_bf16(acc[dt][i4 * 4] * inv, acc[dt][i4 * 4 + 1] * inv), cvt_pk_bf16(acc[dt][i4 * 4 + 2] * inv, acc[dt][i4 * 4 + 3] * inv)};
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int j = 0; j < 32 / kPerStore; ++j) {
                const int r = j * kPerStore + l / kChunks, c = l % kChunks;
                const u32x4 v = *reinterpret_cast<const u32x4*>(mine + r * (DV * 2) + ((c ^ (r & (kChunks - 1) & 15)) << 4));
                const uint32_t to = __shfl(q_row, r, kWave);
                if (wave * 32 + r < rows) *reinterpret_cast<u32x4*>(a.out + static_cast<size_t>(to) * DV + c * 8) = v;
            }
            continue;
        }
        // a lane's registers as they are, so that a store takes 1 KB: see partial_at
        const size_t slot = 2 * static_cast<size_t>(__builtin_amdgcn_readfirstlane(w)) + (begins ? 1 : 0);
        if (lg == 0) {
            const size_t prow = slot * S::kRows + wave * 32 + ln;
            a.part_ml[2 * prow] = m_run, a.part_ml[2 * prow + 1] = l_tot;
        }
        f32x4* po = reinterpret_cast<f32x4*>(a.part_acc) + (slot * WAVES + wave) * (S::kDTiles * 4 * kWave) + lane;
#pragma unroll
        for (int dt = 0; dt < S::kDTiles; ++dt)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) po[(dt * 4 + i4) * kWave] = f32x4{acc[dt][i4 * 4], acc[dt][i4 * 4 + 1], acc[dt][i4 * 4 + 2], acc[dt][i4 * 4 + 3]};
    }
    if (a.status && __any(bad_page) && lane == 0) atomicOr(a.status, 2);
}

// Joins the pieces of the row tile that was cut at the end of stretch blockIdx.x, 256 vectors a workgroup.
// A workgroup takes a quarter of a wave's rows and outputs: one f32x4 of a lane (row ln, outputs dt * 32 + i4 * 8 + lg * 4 .. + 3) per thread.
template <int DV, int ROWS>
__global__ __launch_bounds__(kPromptThreads) void prompt_join_kernel(PromptArgs a) {
    constexpr int kVectors = ROWS * DV / 4, kBlocks = kVectors / kPromptThreads;
    const int w = blockIdx.x / kBlocks, e = blockIdx.x % kBlocks * kPromptThreads + threadIdx.x;
    const PromptCut cut = a.cuts[w];
    if (cut.pieces < 2) return;
    const int first = a.first[cut.b], n = a.first[cut.b + 1] - first;
    const int lane = e & (kWave - 1), vec = e / kWave % (DV / 8), wave = e / kWave / (DV / 8);
    const int r = wave * 32 + (lane & 31), d = vec * 8 + (lane >> 5) * 4;
    const int64_t row = static_cast<int64_t>(cut.tile) * ROWS + r;
    if (row >= static_cast<int64_t>(n) * a.G) return;
    auto slot = [&](int k) { return 2 * static_cast<size_t>(w + k) + (k == 0 ? 1 : 0); };
    float m = kNoScore;
    for (int k = 0; k < cut.pieces; ++k) m = fmaxf(m, a.part_ml[2 * (slot(k) * ROWS + r)]);
    float l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 0; k < cut.pieces; ++k) {
        const float mk = a.part_ml[2 * (slot(k) * ROWS + r)], lk = a.part_ml[2 * (slot(k) * ROWS + r) + 1];
        const float f = fast_exp2((mk - m) * a.scale_log2);
        const f32x4 v = *(reinterpret_cast<const f32x4*>(a.part_acc) + slot(k) * kVectors + e);
        l = fmaf(lk, f, l);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = fmaf(v[i], f, o[i]);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t token = row / a.G;
    uint16_t* out = a.out + ((static_cast<size_t>(first) + token) * a.Hq + cut.kvh * a.G + (row - token * a.G)) * DV + d;
    *reinterpret_cast<u32x2*>(out) = u32x2{cvt_pk_bf16(o[0] * inv, o[1] * inv), cvt_pk_bf16(o[2] * inv, o[3] * inv)};
}

static hipError_t launch_join(const PromptArgs& a, hipStream_t stream) {
    // (a block table so short that no row tile is cut leaves nothing to join)
    const int rows = 1 << a.row_shift;
    if (a.G * (a.max_ctx + a.tile_cost) + rows <= static_cast<int64_t>(a.G) * (kWholePositions + a.tile_cost)) return hipSuccess;
    const dim3 grid(a.W * (rows * a.Dv / 4 / kPromptThreads));
    if (a.Dv == 64) hipLaunchKernelGGL((prompt_join_kernel<64, kRowTile>), grid, dim3(kPromptThreads), 0, stream, a);
    else if (a.Dv == 128 && rows > kRowTile) hipLaunchKernelGGL((prompt_join_kernel<128, 2 * kRowTile>), grid, dim3(kPromptThreads), 0, stream, a);
    else if (a.Dv == 128) hipLaunchKernelGGL((prompt_join_kernel<128, kRowTile>), grid, dim3(kPromptThreads), 0, stream, a);
    else if (a.Dv == 256) hipLaunchKernelGGL((prompt_join_kernel<256, kRowTile>), grid, dim3(kPromptThreads), 0, stream, a);
    else hipLaunchKernelGGL((prompt_join_kernel<512, kRowTile>), grid, dim3(kPromptThreads), 0, stream, a);
    return hipGetLastError();
}

template <int DQK, int DV>
static hipError_t launch_prompt(const PromptArgs& a, hipStream_t stream) {
    if constexpr (DQK == 128) {
        if (1 << a.row_shift > kRowTile) {
            hipLaunchKernelGGL((prompt_tile_kernel<DQK, DV, false, 8>), dim3(a.W), dim3(8 * kWave), 0, stream, a);
            return hipGetLastError();
        }
    }
    // (pages of 16 through the form for any page, against their own: one prompt of 32 768 tokens on 8/1 heads 2553 | 2162 us, heads of 256 439 | 348, 64 253 | 226)
    if (a.P % 16 == 0) hipLaunchKernelGGL((prompt_tile_kernel<DQK, DV, false, 4>), dim3(a.W), dim3(kPromptThreads), 0, stream, a);
    else hipLaunchKernelGGL((prompt_tile_kernel<DQK, DV, true, 4>), dim3(a.W), dim3(kPromptThreads), 0, stream, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
// What a row tile costs beside its positions -- queries, first loads, masked tiles, output -- in positions.  Measured, with 1 | 128 | 256 | 384 | 512:
// heads of 64, 12 prompts of up to 6000 tokens 289 | 248 | 250 | 259 | 266 us; of 128, 16 prompts of up to 8192 4175 | 3499 | 3253 | 3297 | 3411 (256 rows a row tile, 128 | 256 | 384: 3643 | 3081 | 3131); of 256, four
// of 4096 531 | 392 | 346 | 353 | 358; shared latent, four pieces of up to 2048 2269 | 1667 | 1498 | 1482 | 1491.  Heads of 192 take what 128 and 256 take: four of 4096 on 16 heads 462 | 439 | 424 | 424
// (128 | 256 | 384 | 512, a slower card: heads of 256 415 | 375 | 380 | 382 there), 12 of up to 6000 542 | 524 | 522 | 527.
constexpr int prompt_tile_cost(int dqk) { return dqk <= 64 ? 128 : (dqk <= 256 ? 256 : 384); }
static int check_prompt_params(const seer_attn_params* p, int32_t n_tokens) {
    if (!p) return SEER_EINVAL;
    if (p->B < 0 || n_tokens < 0 || p->Hq < 1 || p->Hkv < 1 || p->page_size < 1 || p->num_pages < 1 || p->max_pages_per_seq < 1) return SEER_EINVAL;
    if (!(p->scale > 0.f) || !(p->scale <= 3.4028234e38f)) return SEER_EINVAL;
    if (p->Hq % p->Hkv != 0) return SEER_ESHAPE;
    const bool shared = p->kv_shared_latent != 0;
    const bool known = shared ? p->Dqk == 576 && p->Dv == 512
                              : (p->Dqk == 64 && p->Dv == 64) || (p->Dqk == 128 && p->Dv == 128) || (p->Dqk == 256 && p->Dv == 256) || (p->Dqk == 192 && p->Dv == 128);
    if (!known) return SEER_EUNSUPPORTED;
    const int64_t ctx = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size, G = p->Hq / p->Hkv;
    // positions are counted in 32 bits, the line of row tiles in 64, rows of the pool and of q in 32
    if (ctx > 0x7fffffffLL - 65536 || static_cast<int64_t>(p->num_pages) * p->page_size * p->Hkv > 0xffffffffLL) return SEER_ESHAPE;
    if (static_cast<int64_t>(n_tokens) * p->Hq > 0xffffffffLL) return SEER_ESHAPE;
    const double tiles = static_cast<double>(n_tokens) * G / kRowTile + p->B;
    if (tiles * p->Hkv * (static_cast<double>(G) * (ctx + prompt_tile_cost(p->Dqk)) + static_cast<double>(n_tokens) * G + 2 * kRowTile) > 4e15) return SEER_ESHAPE;
    return SEER_OK;
}
struct PromptLayout {
    int W, row_shift;
    size_t off_ml, off_acc, total;
};
constexpr int64_t kEightWavesRows = 131072, kEightWavesRequest = 8192;      // query rows, and those of a KV head and request on average
constexpr int prompt_waves_per_simd(int dqk) { return dqk <= 64 ? 3 : (dqk <= 192 ? 2 : 1); }
// Eight waves and 256 rows a workgroup, for heads of 128: half the tile loads.  Four | eight waves: 16 prompts of 256 .. 8192 tokens on 64/8 heads 3121 | 2999 us, one of 32 768
// on 8/1 2065 | 1990, one of 16 384 on 64/8 4210 | 3973, four of 8192 on 16/16 1204 | 1150, 16 of 2048 on 32/8 681 | 666.  With few rows a request or few of all, coarse
// row tiles cost more than that: 8 of 1024 on 32/8 105 | 113, four of 4096 on 16/16 335 | 340, one of 600 on 8/1 24.5 | 40, of 4096 62.6 | 64.6, one of 1024 on 64/8 47 | 52, single
// tokens 902 | 1127.  The host knows the rows and the requests, not which rows are padding and which requests have none: padding raises the average, requests without tokens lower it, and
// either may call for the dearer form of the two, whose results are within the same bounds.  (Heads of 64 and 256 hold three waves and one a SIMD, a tile of 192 components is no multiple of eight waves' loads.)
static bool prompt_has_eight_waves(const seer_attn_params& p, int32_t n_tokens) {
    const int64_t rows = static_cast<int64_t>(n_tokens) * p.Hq;
    return p.Dqk == 128 && p.page_size % 16 == 0 && rows >= kEightWavesRows && rows / p.Hkv >= kEightWavesRequest * static_cast<int64_t>(p.B);
}
static PromptLayout prompt_layout(const seer_attn_params& p, int32_t n_tokens) {
    PromptLayout w{};
    // no more stretches than the GPU holds at once, nor than the host can see work for
    const int row_tile = prompt_has_eight_waves(p, n_tokens) ? 2 * kRowTile : kRowTile;
    int resident = 256 * prompt_waves_per_simd(p.Dqk) * kRowTile / row_tile;
    const int64_t ctx = static_cast<int64_t>(p.max_pages_per_seq) * p.page_size, G = p.Hq / p.Hkv;
    const int64_t requests = p.B < n_tokens ? p.B : n_tokens;
    const double row_tiles = (static_cast<double>(n_tokens) * G / row_tile + requests) * p.Hkv;
    const double most = row_tiles * (static_cast<double>(ctx + prompt_tile_cost(p.Dqk) + row_tile) / kMinStretch + 1);
    if (most < resident) resident = static_cast<int>(most);
    w.W = (resident + 7) / 8 * 8;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    // (as many bytes for both row tiles: what does for more tokens does for fewer)
    w.off_ml = up(sizeof(PromptCut) * w.W * (row_tile / kRowTile));
    w.off_acc = w.off_ml + up(sizeof(float) * 2 * row_tile * 2 * w.W);
    w.total = w.off_acc + sizeof(float) * row_tile * p.Dv * 2 * w.W;
    w.row_shift = row_tile == kRowTile ? 7 : 8;
    return w;
}

}  // namespace seer

extern "C" size_t seer_prompt_attention_workspace(const seer_attn_params* p, int32_t n_tokens) {
    if (seer::check_prompt_params(p, n_tokens) != SEER_OK || p->B == 0 || n_tokens == 0) return 0;
    return seer::prompt_layout(*p, n_tokens).total;
}

extern "C" int seer_prompt_attention(void* out, const void* q, const void* k_pages, const void* v_pages, const int32_t* block_table,
                                     const int32_t* ctx_len, const int32_t* first_token, const seer_attn_params* p, int32_t n_tokens,
                                     int32_t* status, void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = seer::check_prompt_params(p, n_tokens);
    if (rc != SEER_OK) return rc;
    if (p->B == 0 || n_tokens == 0) return SEER_OK;
    const bool shared = p->kv_shared_latent != 0;
    if (!out || !q || !k_pages || shared != !v_pages || !block_table || !ctx_len || !first_token) return SEER_EINVAL;
    const seer::PromptLayout layout = seer::prompt_layout(*p, n_tokens);
    if (!workspace || workspace_bytes < layout.total) return SEER_EWORKSPACE;
    auto misaligned = [](const void* ptr, uintptr_t a) { return reinterpret_cast<uintptr_t>(ptr) % a != 0; };
    if (misaligned(out, 16) || misaligned(q, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16) || misaligned(workspace, 256) ||
        misaligned(block_table, 4) || misaligned(ctx_len, 4) || misaligned(first_token, 4) || misaligned(status, 4))
        return SEER_EALIGN;
    seer::PromptArgs a{};
    a.out = static_cast<uint16_t*>(out), a.q = static_cast<const uint16_t*>(q);
    a.k_pages = static_cast<const unsigned char*>(k_pages), a.v_pages = static_cast<const unsigned char*>(v_pages);
    a.block_table = block_table, a.ctx_len = ctx_len, a.first = first_token, a.status = status;
    char* ws = static_cast<char*>(workspace);
    a.cuts = reinterpret_cast<seer::PromptCut*>(ws);
    a.part_ml = reinterpret_cast<float*>(ws + layout.off_ml);
    a.part_acc = reinterpret_cast<float*>(ws + layout.off_acc);
    a.B = p->B, a.Hq = p->Hq, a.Hkv = p->Hkv, a.G = p->Hq / p->Hkv, a.P = p->page_size, a.num_pages = p->num_pages, a.max_pages = p->max_pages_per_seq;
    a.inv_g = a.G > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / static_cast<uint32_t>(a.G)) : 0xffffffffu;
    a.n_tokens = n_tokens, a.Dqk = p->Dqk, a.Dv = p->Dv, a.W = layout.W, a.row_shift = layout.row_shift, a.tile_cost = seer::prompt_tile_cost(p->Dqk);
    a.inv_p = p->page_size > 1 ? static_cast<uint32_t>((uint64_t{1} << 32) / static_cast<uint32_t>(p->page_size)) : 0xffffffffu;
    a.scale_log2 = p->scale * seer::kLog2e;
    a.move_at = a.scale_log2 > 1e-36f ? 8.f / a.scale_log2 : 8e36f;
    a.max_ctx = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    hipError_t err = hipErrorInvalidValue;
    if (p->Dqk == 64) err = seer::launch_prompt<64, 64>(a, stream);
    else if (p->Dqk == 128) err = seer::launch_prompt<128, 128>(a, stream);
    else if (p->Dqk == 192) err = seer::launch_prompt<192, 128>(a, stream);
    else if (p->Dqk == 256) err = seer::launch_prompt<256, 256>(a, stream);
    else err = seer::launch_prompt_latent(a, stream);
    if (err == hipSuccess) err = seer::launch_join(a, stream);
    return err == hipSuccess ? SEER_OK : static_cast<int>(err);
}
