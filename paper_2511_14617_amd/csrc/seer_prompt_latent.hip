// Causal attention of packed tokens over a cache of shared latents (576 components a position, its first 512 the value): the prompt form of
// the verify kernel for that shape, with that kernel's arithmetic (seer_mla.h) on the row tiles of seer_prompt.h.
//
// What bounds it: the matrix cores at the clock that the power limit leaves them, and what one wave per SIMD issues between their instructions
// (about 1200 flop per byte of a tile).  A workgroup of four waves takes 128 query rows; a tile of 32 positions (36 KB) goes HBM/L2 -> LDS
// directly, three stages; the scores of tile u run beside the softmax of tile u - 1, then its product with V beside the highest scores of tile u.  Four
// pieces of 256 .. 2048 tokens on 128 heads: 1.5 ms, 980 TFLOP/s; matrix cores busy 49 % of the time, LDS 34 % without conflicts.  With 128
// heads a row tile is one token, and neighbouring row tiles read the same latents: the stretches of one XCD are neighbours on the line.
// Queries and outputs (276 KB a row tile) pass through LDS, the outputs in a loop: unrolled they were 6 KB of code, fetched anew for every row tile
// (with that and row tiles counted without a fixed cost 2.10 ms).
//
// Infinities and NaN in positions that some row of the tile does not see: scores by selection; the value rows are taken out of LDS once
// all waves have the tile's scores.  A row that sees such a latent has it in its score as well, which is then NaN or +inf and makes the whole row NaN, or -inf:
// 0 times the latent, which is added at the end.
#include "seer_device.h"
#include "seer_mla.h"
#include "seer_prompt.h"
#include "seer_tile.h"

namespace seer {

// ANY_PAGE: pages of any size; a lane finds the row of its LDS slot through the block table instead of a descriptor of the tile.
template <bool ANY_PAGE>
__global__ __launch_bounds__(kPromptThreads) __attribute__((amdgpu_waves_per_eu(1, 1)))
void prompt_latent_kernel(PromptArgs a) {
    using namespace mla;
    static_assert(kRowsPerWg == kRowTile && kWaves * kWave == kPromptThreads, "");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kStages * kStageBytes];
    __shared__ __attribute__((aligned(16))) u32x4 q_tail[kWaves][kQLdsSteps][kWave];      // (see the verify kernel)
    __shared__ PromptLds s_plan;
    __shared__ uint32_t s_found;                    // positions with infinities or NaN in the scanned tile's values
    constexpr int kEdgeTiles = 8;                   // (that some row does not see whole: 128 tokens at most touch six)
    __shared__ uint32_t s_left[kWaves][kEdgeTiles]; // the positions left out, by tile (each wave its own copy)

    const int tid = threadIdx.x, lane = tid & (kWave - 1), ln = lane & 31, lg = lane >> 5, l16 = lane >> 4, p16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    int w, error = 0;
    PromptPlan plan;
    int64_t x, x_end;
    PromptTile t;
    {
        int64_t at[2];
        PromptTile ends[2];
        const bool on = prompt_plan<kPromptThreads>(a, s_plan, w, plan, at, ends, error);
        if (blockIdx.x == 0 && error && a.status) atomicOr(a.status, error);
        if (!on) return;
        x = moved_cut(plan, ends[0], at[0]);
        x_end = moved_cut(plan, ends[1], at[1]);
        t = ends[0];
        PromptCut cut{0, 0, 0, 0};                  // the row tile that begins in this stretch and goes on behind it
        if (x_end > ends[1].begin && x_end < ends[1].begin + ends[1].cost && ends[1].begin >= x && !ends[1].r.bad)
            cut = PromptCut{ends[1].b, ends[1].kvh, ends[1].i, pieces_of(plan, ends[1], w)};
        if (tid == 0) a.cuts[w] = cut;
    }
    bool bad_page = false;

    // operand addresses (see the verify kernel)
    int k_rd[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) k_rd[j] = ln * kRowBytes + (((2 * j + lg) ^ swz(ln)) << 4);
    const int v_k = p16 >> 2, v_c4 = p16 & 3, v_dhalf = l16 & 1;
    const int v_swz = swz(lg * 4 + v_k), v_row0 = (lg * 4 + v_k) * kRowBytes;
    const int v_even = v_row0 + (((v_dhalf * 2 + (v_c4 >> 1)) ^ v_swz) << 4) + (v_c4 & 1) * 8;
    const int v_odd = v_row0 + (((4 + v_dhalf * 2 + (v_c4 >> 1)) ^ v_swz) << 4) + (v_c4 & 1) * 8;
    const int v_even8 = v_row0 + (((v_dhalf * 2 + (v_c4 >> 1)) ^ v_swz ^ 1) << 4) + (v_c4 & 1) * 8;
    const int v_odd8 = v_row0 + (((4 + v_dhalf * 2 + (v_c4 >> 1)) ^ v_swz ^ 1) << 4) + (v_c4 & 1) * 8;
    int pat[5];
#pragma unroll
    for (int j = 0; j < 5; ++j) {
        const unsigned c = static_cast<unsigned>((j < 4 ? wave + 4 * j : 16 + (wave & 1)) * 64 + lane);
        const unsigned row = c / kChunksPerRow, pos = c - row * kChunksPerRow;
        pat[j] = static_cast<int>(row * kRowBytes + ((pos ^ static_cast<unsigned>(swz(static_cast<int>(row)))) << 4));
    }
    auto page_of = [&](int position) __attribute__((always_inline)) -> int { return prompt_page(a, position); };

    while (x < x_end) {
        if (x >= t.begin + t.cost) next_tile<kPromptThreads>(a, t);
        const int64_t end = min(x_end, t.begin + t.cost);
        const bool begins = x == t.begin, ends = end == t.begin + t.cost;
        // (rows of q are counted in 32 bits)
        const uint32_t row0 = static_cast<uint32_t>(t.i) * kRowTile;
        const int rows = static_cast<int>(min(static_cast<uint32_t>(t.r.n) * static_cast<uint32_t>(a.G) - row0, static_cast<uint32_t>(kRowTile)));
        const int token_first = prompt_token(a, row0), token_last = prompt_token(a, row0 + rows - 1);              // of the request's new tokens
        const int seen = static_cast<int>(t.r.past) + token_last + 1;
        const int tiles = t.r.bad ? 0 : (seen + kTile - 1) / kTile;
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
        const int sees = row_ok ? static_cast<int>(t.r.past) + token : -1;
        const int sees_lo = __builtin_amdgcn_readfirstlane(sees), all_see = static_cast<int>(t.r.past) + token_first;
        f32x16 acc[kDTiles];
#pragma unroll
        for (int dt = 0; dt < kDTiles; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
        float m_run = kNoScore, l_run = 0.f, alpha = 1.f;
        bool any_left = false;                      // uniform
        __syncthreads();                            // every wave is done with the stages of the piece before
        if (n_tiles > 0) {
            // Queries through LDS: a wave's 32 rows lie there as a tile does (waves 0 to 2 in the stages, wave 3 in the parked part), so that they are
            // loaded row by row and read as K operands are (straight from memory, 16 bytes of 32 rows an instruction, 20 000 clocks a row tile).
            u32x4 qreg[kQRegSteps];
            {
                static_assert(sizeof(q_tail) >= kStageBytes, "");
                unsigned char* mine = wave < 3 ? lds + wave * kStageBytes : reinterpret_cast<unsigned char*>(q_tail);
#pragma unroll 6
                for (int j = 0; j < kBlocks; ++j) {
                    const int c = j * kWave + lane, r = c / kChunksPerRow, pos = c - r * kChunksPerRow;
                    const uint32_t of = row0 + min(wave * 32 + r, rows - 1), at = prompt_token(a, of);      // (behind the last row: again that one)
                    const uint32_t from = static_cast<uint32_t>(t.r.first + at) * a.Hq + t.kvh * a.G + (of - at * a.G);
                    const unsigned char* src = reinterpret_cast<const unsigned char*>(a.q) + static_cast<size_t>(from) * kRowBytes + ((pos ^ swz(r)) << 4);
                    __builtin_amdgcn_global_load_lds((const SEER_AS1 void*)(src), (SEER_AS3 void*)(mine + j * 1024), 16, 0, 0);
                }
                wait_vmcnt<0>();
                __builtin_amdgcn_wave_barrier();
                u32x4 tail[kQLdsSteps];
#pragma unroll
                for (int kk = 0; kk < kKSteps; ++kk) {
                    const u32x4 v = *reinterpret_cast<const u32x4*>(mine + k_rd[kk & 3] + (kk >> 2) * 128);
                    if (kk < kQRegSteps) qreg[kk < kQRegSteps ? kk : 0] = v;
                    else tail[kk >= kQRegSteps ? kk - kQRegSteps : 0] = v;
                }
                __syncthreads();                    // every wave has its queries
#pragma unroll
                for (int kk = 0; kk < kQLdsSteps; ++kk) q_tail[wave][kk][lane] = tail[kk];
#pragma unroll
                for (int kk = 0; kk < kQRegSteps; ++kk) asm volatile("" : "+v"(qreg[kk]));
            }

            // ---- page ids, 64 at a time -------------------------------------------------------------------
            const int32_t* table = a.block_table + static_cast<size_t>(t.b) * a.max_pages;
            const int last_page = page_of(static_cast<int>(t.r.past) + t.r.n - 1);
            int win = -0x40000000, pg_win = 0;
            auto set_window = [&](int first) __attribute__((always_inline)) {
                win = first;
                int pg = table[min(first + lane, a.max_pages - 1)];
                if (pg < 0 || pg >= a.num_pages) {
                    if (first + lane <= last_page) bad_page = true;
                    pg = min(max(pg, 0), a.num_pages - 1);
                }
                pg_win = pg;
            };
            // loads through a descriptor of the tile, which lies in one page where pages hold a multiple of a tile (see the verify kernel)
            auto tile_rsrc = [&](int tile) __attribute__((always_inline)) {
                const int tb = tok_begin + tile * kTile, lp = page_of(tb);
                if (lp < win || lp >= win + kWave) set_window(lp);
                const int pg = __builtin_amdgcn_readlane(pg_win, __builtin_amdgcn_readfirstlane(lp - win));
                const unsigned char* src = a.k_pages + ((static_cast<size_t>(pg) * a.Hkv + t.kvh) * a.P + (tb - lp * a.P)) * kRowBytes;
                return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(src), 0, kStageBytes, 0x00020000);
            };
            auto issue_load = [&](auto ic, __amdgpu_buffer_rsrc_t rsrc, int stage_off) __attribute__((always_inline)) {
                constexpr int i = decltype(ic)::value;
                const int half = i < 8 ? (i & 1) : (wave >> 1);
                const int block = (i < 8 ? wave + 4 * (i >> 1) : 16 + (wave & 1)) + 18 * half;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (SEER_AS3 void*)(lds + stage_off + block * 1024), 16, pat[i < 8 ? (i >> 1) : 4],
                                                         half * (16 * kRowBytes), 0, 0);
            };
            // ... and through the row of every position
            auto issue_rows = [&](int tile, int stage_off) __attribute__((always_inline)) {
                const int tb = tok_begin + tile * kTile;
                if (page_of(tb) < win || page_of(tb + kTile - 1) >= win + kWave) set_window(page_of(tb));
                const int tok = tb + ln, lp = page_of(tok);
                const int pg = __builtin_amdgcn_ds_bpermute((lp - win) << 2, pg_win);
                const uint32_t row_idx = (static_cast<uint32_t>(pg) * a.Hkv + t.kvh) * static_cast<uint32_t>(a.P) + static_cast<uint32_t>(tok - lp * a.P);
                for (int j = 0; j < kLoadsPerWave; ++j) {
                    const int block = j * kWaves + wave, c = block * kWave + lane, r = c / kChunksPerRow, pos = c - r * kChunksPerRow;
                    const uint32_t from = __builtin_amdgcn_ds_bpermute(r << 2, row_idx);
                    const unsigned char* src = a.k_pages + static_cast<size_t>(from) * kRowBytes + ((pos ^ swz(r)) << 4);
                    __builtin_amdgcn_global_load_lds((const SEER_AS1 void*)(src), (SEER_AS3 void*)(lds + stage_off + block * 1024), 16, 0, 0);
                }
            };
            auto issue_tile = [&](int tile, int stage_off) __attribute__((always_inline)) {
                if constexpr (ANY_PAGE) {
                    issue_rows(tile, stage_off);
                } else {
                    const __amdgpu_buffer_rsrc_t rsrc = tile_rsrc(tile);
                    for_each_index([&](auto ic) __attribute__((always_inline)) { issue_load(ic, rsrc, stage_off); }, std::make_integer_sequence<int, kLoadsPerWave>{});
                }
            };

            // ---- the pipeline (see the verify kernel): step u = scores of tile u | softmax of tile u - 1, then P.V of tile u - 1 -------
            static_assert(kStages == 3, "the three stage offsets below rotate");
            int st_prev = 2 * kStageBytes, st_cur = 0, st_next = kStageBytes;
            const int lds_base = lds_addr(lds);
            const int qt = lds_addr(&q_tail[wave][0][lane]);
            f32x16 s_a, s_b;
            uint32_t pk[8];
            // positions of the tile before, and of this one, whose values are kept out of the product (uniform)
            uint32_t left_prev = 0, left_cur = 0;
            if (lane < kEdgeTiles) *const_cast<volatile uint32_t*>(&s_left[wave][lane]) = 0;
            auto step_top = [&](int u) __attribute__((always_inline)) {
                wait_vmcnt<0>();
                bare_barrier();                     // tile u has landed for every wave, every wave has the scores of tile u - 1
                if constexpr (ANY_PAGE) {
                    if (u + 1 < n_tiles) issue_rows(u + 1, st_next);
                }
                left_prev = left_cur, left_cur = 0;
                if (u < n_tiles && tok_begin + u * kTile + kTile - 1 > all_see) {
                    if (tid == 0) s_found = 0;
                    __builtin_amdgcn_s_waitcnt(0xc07f);
                    bare_barrier();
                    uint32_t found = 0;
#pragma unroll 1
                    for (int c = tid; c < kTile * (kDv / 8); c += kPromptThreads) {
                        const int r = c / (kDv / 8), pos = c - r * (kDv / 8);
                        const u32x4 v = *reinterpret_cast<const u32x4*>(lds + st_cur + r * kRowBytes + ((pos ^ swz(r)) << 4));
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if ((v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u) found |= 1u << r;
                    }
                    if (found) atomicOr(&s_found, found);
                    __builtin_amdgcn_s_waitcnt(0xc07f);
                    bare_barrier();
                    left_cur = __builtin_amdgcn_readfirstlane(*const_cast<volatile uint32_t*>(&s_found));
                    if (left_cur) {
                        const int edge = u0 + u - (all_see + 1) / kTile;
                        if (edge < kEdgeTiles) *const_cast<volatile uint32_t*>(&s_left[wave][edge]) = left_cur;
                        any_left = true;
                    }
                }
                if (left_prev) {
#pragma unroll 1
                    for (int c = tid; c < kTile * (kDv / 8); c += kPromptThreads) {
                        const int r = c / (kDv / 8), pos = c - r * (kDv / 8);
                        if ((left_prev >> r) & 1u) *reinterpret_cast<u32x4*>(lds + st_prev + r * kRowBytes + ((pos ^ swz(r)) << 4)) = u32x4{0u, 0u, 0u, 0u};
                    }
                    __builtin_amdgcn_s_waitcnt(0xc07f);
                }
                if (left_prev || (u < n_tiles && tok_begin + u * kTile + kTile - 1 > all_see)) bare_barrier();      // (also: s_found has been read)
            };
            auto apply_mask = [&](int j, f32x16& sc) __attribute__((always_inline)) {
                const int tb = tok_begin + j * kTile;
                if (tb + kTile - 1 <= sees_lo) return;
                const int lim = sees - tb;
                uint32_t vis = lim < 0 ? 0u : (lim >= 31 ? 0xffffffffu : (2u << lim) - 1u);
                vis >>= lg * 4;
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (!((vis >> ((i >> 2) * 8 + (i & 3))) & 1u)) sc[i] = kNegInf;
            };
            auto k_addrs = [&](int stage_off, int (&ka)[4]) __attribute__((always_inline)) {
                const int st = lds_base + stage_off;
#pragma unroll
                for (int j = 0; j < 4; ++j) ka[j] = st + k_rd[j];
            };
            auto v_addrs = [&](int stage_off, int (&va)[4]) __attribute__((always_inline)) {
                const int st = lds_base + stage_off;
                va[0] = st + v_even, va[1] = st + v_even8, va[2] = st + v_odd, va[3] = st + v_odd8;
            };
            // (references as in the kernel for separate pools; the move itself stands behind the product, where no read is in flight)
            float m_use = 0.f, mx = 0.f;
            bool moved = false, far = false;
            auto highest = [&](auto ic, const f32x16& sc) __attribute__((always_inline)) {
                constexpr int part = decltype(ic)::value;
                if constexpr (part == 0) {
                    mx = fmaxf(fmaxf(sc[0], sc[1]), sc[2]);
#pragma unroll
                    for (int i = 3; i < 9; i += 2) mx = fmaxf(fmaxf(mx, sc[i]), sc[i + 1]);
                    SEER_MLA_PIN(mx);
                } else if constexpr (part == 1) {
#pragma unroll
                    for (int i = 9; i < 15; i += 2) mx = fmaxf(fmaxf(mx, sc[i]), sc[i + 1]);
                    mx = fmaxf(mx, sc[15]);
                    SEER_MLA_PIN(mx);
                } else {
                    mx = max_across_halves(mx);
                    SEER_MLA_PIN(mx);
                }
            };
            auto reference = [&](f32x16& sc) __attribute__((always_inline)) {
                const bool moves = mx > m_run + a.move_at;
                moved = __any(moves);
                alpha = 1.f;
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
                    for (int i = 0; i < 16; ++i) sc[i] -= m_run;
                }
            };
            u32x2 vr[kVAhead][2];
            int va[4];
            auto pv = [&](int j, auto next, f32x16& sc_next, auto&& prepare) __attribute__((always_inline)) {
                constexpr bool NEXT = decltype(next)::value;
                if constexpr (NEXT) {
                    if (tok_begin + (j + 1) * kTile + kTile - 1 > sees_lo) {
                        mfma_drain();
                        apply_mask(j + 1, sc_next);
                    }
                }
                if (moved) {
                    mfma_drain();
#pragma unroll
                    for (int dt = 0; dt < kDTiles; ++dt) {
                        f32x16 tmp = acc[dt];
                        asm volatile("" : "+v"(tmp));
#pragma unroll
                        for (int i = 0; i < 16; ++i) tmp[i] *= alpha;
                        acc[dt] = tmp;
                        asm volatile("" : "+a"(acc[dt]));
                    }
                    asm volatile("s_nop 7");
                }
                constexpr int kRefFirst = 4;
                phase_b(va, vr, pk, acc, [&](auto ic) __attribute__((always_inline)) {
                    constexpr int m = decltype(ic)::value;
                    if constexpr (NEXT && m >= kRefFirst && (m - kRefFirst) % 2 == 0 && (m - kRefFirst) / 2 < 3)
                        highest(std::integral_constant<int, (m - kRefFirst) / 2>{}, sc_next);
                    prepare(ic);
                });
                if constexpr (NEXT) reference(sc_next);
            };
            using yes = std::true_type;
            using no = std::false_type;

            issue_tile(0, st_cur);
            int ka[4];
            __amdgpu_buffer_rsrc_t next_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(a.k_pages), 0, 0, 0x00020000);
            bool next_ok = false;
            auto next_setup = [&](int u) __attribute__((always_inline)) {
                if constexpr (!ANY_PAGE) {
                    next_ok = u + 1 < n_tiles;
                    if (next_ok) next_rsrc = tile_rsrc(u + 1);
                }
            };
            auto next_load = [&](auto ic) __attribute__((always_inline)) {
                if constexpr (!ANY_PAGE) {
                    if (next_ok) issue_load(ic, next_rsrc, st_next);
                }
            };
            auto nothing = [](auto) {};
            int u = 0;
            auto prepare_next = [&](auto ic) __attribute__((always_inline)) {
                constexpr int m = decltype(ic)::value;
                if constexpr (m == 14) {
                    const int st = st_prev;
                    st_prev = st_cur, st_cur = st_next, st_next = st;
                    k_addrs(st_cur, ka);
                } else if constexpr (m == 18) {
                    next_setup(u + 1);
                }
            };
            auto v_addrs_early = [&](auto ic) __attribute__((always_inline)) {
                if constexpr (decltype(ic)::value == 2) v_addrs(st_prev, va);
            };
            k_addrs(st_cur, ka);
            next_setup(0);
            step_top(0);
            phase_a<true, false>(ka, qt, qreg, s_a, s_b, pk, m_use, l_run, alpha, a.scale_log2, va, vr, next_load, nothing);
            mfma_drain();
            apply_mask(0, s_a);
            for_each_index([&](auto ic) __attribute__((always_inline)) { highest(ic, s_a); }, std::make_integer_sequence<int, 3>{});
            reference(s_a);
            prepare_next(std::integral_constant<int, 14>{});
            prepare_next(std::integral_constant<int, 18>{});
            for (u = 1; u + 1 < n_tiles;) {
                step_top(u);
                phase_a<true, true>(ka, qt, qreg, s_b, s_a, pk, m_use, l_run, alpha, a.scale_log2, va, vr, next_load, v_addrs_early);
                pv(u - 1, yes{}, s_b, prepare_next);
                ++u;
                step_top(u);
                phase_a<true, true>(ka, qt, qreg, s_a, s_b, pk, m_use, l_run, alpha, a.scale_log2, va, vr, next_load, v_addrs_early);
                pv(u - 1, yes{}, s_a, prepare_next);
                ++u;
            }
            if (u < n_tiles) {
                step_top(u);
                phase_a<true, true>(ka, qt, qreg, s_b, s_a, pk, m_use, l_run, alpha, a.scale_log2, va, vr, next_load, v_addrs_early);
                pv(u - 1, yes{}, s_b, prepare_next);
                asm volatile("" : "+v"(s_b));       // the copy below reads s_b after the P.V MFMAs, not right behind the score MFMAs
#pragma unroll
                for (int i = 0; i < 16; ++i) s_a[i] = s_b[i];
            }
            // the last tile's scores are in s_a, masked, and its reference is set; its stage is the one before the current
            if (left_cur) step_top(n_tiles);
            v_addrs(st_prev, va);
            phase_a<false, true>(ka, qt, qreg, s_b, s_a, pk, m_use, l_run, alpha, a.scale_log2, va, vr, nothing, nothing);
            pv(n_tiles - 1, no{}, s_a, nothing);
            mfma_drain();
        }

        // Positions that were left out, for the rows that see them: the probability is 0, or the row is NaN already, so what is added to component d is 0 times the
        // latent's.  each(latent, the last position that does not see it): for every one of them.
        auto left_out = [&](auto&& each) __attribute__((always_inline)) {
            const int32_t* table = a.block_table + static_cast<size_t>(t.b) * a.max_pages;
#pragma unroll 1
            for (int e = 0; e < kEdgeTiles; ++e) {
                uint32_t words = __builtin_amdgcn_readfirstlane(*const_cast<volatile uint32_t*>(&s_left[wave][e]));
#pragma unroll 1
                for (; words; words &= words - 1) {
                    const int position = ((all_see + 1) / kTile + e) * kTile + __builtin_ctz(words), lp = page_of(position);
                    const int pg = min(max(table[min(lp, a.max_pages - 1)], 0), a.num_pages - 1);
                    each(reinterpret_cast<const uint16_t*>(a.k_pages) + ((static_cast<size_t>(pg) * a.Hkv + t.kvh) * a.P + (position - lp * a.P)) * (kRowBytes / 2), position);
                }
            }
        };
        auto add_zero_times = [](const uint16_t* latent, f32x4& o) __attribute__((always_inline)) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(latent);
            o[0] = fmaf(0.f, bf16lo_to_f32(v[0]), o[0]), o[1] = fmaf(0.f, bf16hi_to_f32(v[0]), o[1]);
            o[2] = fmaf(0.f, bf16lo_to_f32(v[1]), o[2]), o[3] = fmaf(0.f, bf16hi_to_f32(v[1]), o[3]);
        };
        // ---- the row tile's output, or this piece's share of it ------------------------------------------
        const float l_tot = l_run + __shfl_xor(l_run, 32, kWave);
        if (begins && (ends || t.r.bad)) {
            const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;          // (a row of nothing but -inf: zeros)
            // Through LDS, so that a store takes 512 bytes of a row: the unscaled outputs of 256 components at a time, 16-byte chunk c of row r at
            // c ^ r; divided and rounded on the way out, in a loop (unrolled over all accumulators that is 6 KB of code for once a row tile, and
            // its fetch took longer than the work).
            constexpr int kPart = 256;
            static_assert(32 * kPart * 4 <= kStageBytes && kDv % kPart == 0, "");
            unsigned char* mine = wave < 3 ? lds + wave * kStageBytes : reinterpret_cast<unsigned char*>(q_tail);
            int l = lane;
            asm volatile("" : "+v"(l));             // (the addresses below are made here, not kept in registers through the tiles)
            __syncthreads();                        // every wave is done with the stages
            const int rows_here = min(rows - wave * 32, 32);
#pragma unroll
            for (int part = 0; part < kDv / kPart; ++part) {
#pragma unroll
                for (int dt = 0; dt < kPart / 32; ++dt)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4) {
                        const f32x16& o = acc[part * (kPart / 32) + dt];
                        *reinterpret_cast<f32x4*>(mine + (l & 31) * (kPart * 4) + (((dt * 8 + i4 * 2 + (l >> 5)) ^ (l & 31)) << 4)) =
                            f32x4{o[i4 * 4], o[i4 * 4 + 1], o[i4 * 4 + 2], o[i4 * 4 + 3]};
                    }
                __builtin_amdgcn_wave_barrier();
                if (any_left) {
                    left_out([&](const uint16_t* latent, int position) __attribute__((always_inline)) {
#pragma unroll 1
                        for (int r = 0; r < rows_here; ++r)
                            if (__builtin_amdgcn_readlane(sees, r) >= position)
                                add_zero_times(latent + part * kPart + l * 4, *reinterpret_cast<f32x4*>(mine + r * (kPart * 4) + ((l ^ r) << 4)));
                    });
                    __builtin_amdgcn_wave_barrier();
                }
                for (int r = 0; r < rows_here; ++r) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(mine + r * (kPart * 4) + ((l ^ r) << 4));
                    const uint32_t to = __builtin_amdgcn_readlane(q_row, r);
                    const float scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(inv), r));
                    *reinterpret_cast<u32x2*>(a.out + static_cast<size_t>(to) * kDv + part * kPart + l * 4) =
                        u32x2{cvt_pk_bf16(v[0] * scale, v[1] * scale), cvt_pk_bf16(v[2] * scale, v[3] * scale)};
                }
                __builtin_amdgcn_wave_barrier();
            }
            continue;
        }
        // a lane's registers as they are, so that a store takes 1 KB (see the joining kernel)
        const size_t slot = 2 * static_cast<size_t>(w) + (begins ? 1 : 0);
        if (lg == 0) {
            const size_t prow = slot * kRowTile + wave * 32 + ln;
            a.part_ml[2 * prow] = m_run, a.part_ml[2 * prow + 1] = l_tot;
        }
        f32x4* po = reinterpret_cast<f32x4*>(a.part_acc) + (slot * 4 + wave) * (kDTiles * 4 * kWave) + lane;
#pragma unroll
        for (int dt = 0; dt < kDTiles; ++dt)
#pragma unroll
            for (int i4 = 0; i4 < 4; ++i4) po[(dt * 4 + i4) * kWave] = f32x4{acc[dt][i4 * 4], acc[dt][i4 * 4 + 1], acc[dt][i4 * 4 + 2], acc[dt][i4 * 4 + 3]};
        if (any_left)
            left_out([&](const uint16_t* latent, int position) __attribute__((always_inline)) {
                if (sees < position) return;
#pragma unroll 1
                for (int i = 0; i < kDTiles * 4; ++i) {
                    f32x4 o = po[i * kWave];
                    add_zero_times(latent + i * 8 + lg * 4, o);
                    po[i * kWave] = o;
                }
            });
    }
    if (a.status && __any(bad_page) && lane == 0) atomicOr(a.status, 2);
}

hipError_t launch_prompt_latent(const PromptArgs& a, hipStream_t stream) {
    if (a.P % mla::kTile == 0) hipLaunchKernelGGL((prompt_latent_kernel<false>), dim3(a.W), dim3(kPromptThreads), 0, stream, a);
    else hipLaunchKernelGGL((prompt_latent_kernel<true>), dim3(a.W), dim3(kPromptThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace seer
