// Causal attention of packed tokens over the paged cache, separate K and V pools: (64, 64), (128, 128), (192, 128) and (256, 256),
// pages of any size.
//
// Workgroup = 4 waves = a row tile of 128 query rows of one KV head, 32 rows a wave; the work is cut into equal stretches of a line
// of row tiles (seer_prompt.h).  A tile of 32 positions goes HBM/L2 -> LDS directly, K rows then V rows, two stages; S^T = K.Q^T
// leaves a query row to a lane, so its softmax needs one exchange between two lanes, and the probabilities are, packed to bf16, the
// operand of O^T += V^T.P^T as they are.  Running maximum and sum: one pass over the positions.  Positions that no row of the tile sees are not
// read; a wave whose rows see nothing of a tile does not compute it; only tiles that some row does not see whole are masked.
//
// Infinities and NaN: scores of positions that a row does not see are replaced by selection.  In the product with V a position's row is
// multiplied into all query rows, so in tiles with masked positions V rows that hold an infinity or NaN are taken out and added to the rows that see
// them.
#include <type_traits>

#include "seer_device.h"
#include "seer_prompt.h"
#include "seer_tile.h"

namespace seer {

// Workgroups that a CU holds: by registers (queries and outputs of 32 rows) and by LDS.
constexpr int prompt_waves_per_simd(int dqk) { return dqk <= 128 ? 2 : 1; }

template <int DQK, int DV>
__global__ __launch_bounds__(kPromptThreads) __attribute__((amdgpu_waves_per_eu(prompt_waves_per_simd(DQK))))
void prompt_tile_kernel(PromptArgs a) {
    using namespace tile;
    using S = Shape<DQK, DV>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * S::kStage];
    __shared__ PromptLds s_plan;
    __shared__ uint32_t s_found;                    // V rows with infinities or NaN of the scanned tile
    const int tid = threadIdx.x, lane = tid & (kWave - 1), ln = lane & 31, lg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    // neighbouring stretches read the same positions: one XCD (ids are dealt round-robin to eight) takes an eighth of the line
    const int w = (blockIdx.x & 7) * (a.W >> 3) + (blockIdx.x >> 3);

    int error = 0;
    PromptPlan plan;
    int64_t x, x_end;
    PromptTile t;
    {
        int64_t at[2];
        PromptTile ends[2];
        const bool on = prompt_plan(a, s_plan, w, plan, at, ends, error);
        if (w == 0 && error && a.status) atomicOr(a.status, error);
        if (!on) {
            if (tid == 0) a.cuts[w] = PromptCut{0, 0, 0, 0};
            return;
        }
        x = moved_cut(plan, ends[0], at[0]);
        x_end = moved_cut(plan, ends[1], at[1]);
        t = ends[0];
    }
    PromptCut cut{0, 0, 0, 0};
    bool bad_page = false;
    const int lds0 = lds_addr(lds);
    auto page_of = [&](int64_t tok) __attribute__((always_inline)) -> int { return static_cast<int>(a.page_shift >= 0 ? tok >> a.page_shift : tok / a.P); };
    const Operands<DQK, DV> operands;

    while (x < x_end) {
        if (x >= t.begin + t.cost) next_tile(a, t);
        const int64_t end = min(x_end, t.begin + t.cost);
        const bool begins = x == t.begin, ends = end == t.begin + t.cost;
        const int rows = min(kRowTile, static_cast<int>(min(static_cast<int64_t>(t.r.n) * a.G - static_cast<int64_t>(t.i) * kRowTile, static_cast<int64_t>(kRowTile))));
        const int token_first = static_cast<int>(static_cast<int64_t>(t.i) * kRowTile / a.G);                      // of the request's new tokens
        const int token_last = static_cast<int>((static_cast<int64_t>(t.i) * kRowTile + rows - 1) / a.G);
        const int seen = static_cast<int>(t.r.past) + token_last + 1;                                              // positions that the last row sees
        const int tiles = t.r.bad ? 0 : (seen + kTile - 1) / kTile;
        // the piece's tiles (the same rounding on both sides of a cut)
        const int u0 = begins ? 0 : static_cast<int>(static_cast<double>(x - t.begin) * tiles / static_cast<double>(t.cost));
        const int u1 = ends ? tiles : static_cast<int>(static_cast<double>(end - t.begin) * tiles / static_cast<double>(t.cost));
        x = end;
        if (t.r.bad && !begins) continue;

        // ---- this lane's query row -------------------------------------------------------------------------
        const int64_t row = static_cast<int64_t>(t.i) * kRowTile + wave * 32 + ln;
        const bool row_ok = wave * 32 + ln < rows;
        const int token = row_ok ? static_cast<int>(row / a.G) : 0;
        const size_t q_row = (static_cast<size_t>(t.r.first) + token) * a.Hq + t.kvh * a.G + (row_ok ? row - static_cast<int64_t>(token) * a.G : 0);
        const int sees = row_ok ? static_cast<int>(t.r.past) + token : -1;                                         // last position that it sees
        // of the wave: its first row's, its last row's
        const int sees_lo = __builtin_amdgcn_readfirstlane(sees);
        const int sees_hi = sees_lo < 0 ? -1 : static_cast<int>(t.r.past) + static_cast<int>((static_cast<int64_t>(t.i) * kRowTile + min(wave * 32 + 31, rows - 1)) / a.G);
        bf16x8 qreg[S::kKSteps];
        {
            const u32x4* qp = reinterpret_cast<const u32x4*>(a.q + q_row * DQK + lg * 8);
#pragma unroll
            for (int kk = 0; kk < S::kKSteps; ++kk) {
                u32x4 v = {0u, 0u, 0u, 0u};
                if (row_ok) v = qp[kk * 2];
                qreg[kk] = as_bf16x8(v);
            }
        }
        f32x16 acc[S::kDTiles];
#pragma unroll
        for (int dt = 0; dt < S::kDTiles; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[dt][i] = 0.f;
        float m_run = kNegInf, l_run = 0.f, top = kNegInf;

        // ---- tile loads ------------------------------------------------------------------------------------
        const int32_t* table = a.block_table + static_cast<size_t>(t.b) * a.max_pages;
        const int last_page = page_of(static_cast<int64_t>(t.r.past) + t.r.n - 1);
        int win = 0, pg_win = 0;                    // lane l holds the (clamped) page id of logical page win + l
        auto set_window = [&](int first) __attribute__((always_inline)) {
            win = first;
            int pg = table[min(first + lane, a.max_pages - 1)];
            if (pg < 0 || pg >= a.num_pages) {
                if (first + lane <= last_page) bad_page = true;
                pg = min(max(pg, 0), a.num_pages - 1);
            }
            pg_win = pg;
        };
        auto issue_tile = [&](int u, int stage) __attribute__((always_inline)) {
            const int64_t tb = static_cast<int64_t>(u) * kTile;
            const int first = page_of(tb);
            if (u == u0 || page_of(tb + kTile - 1) >= win + kWave) set_window(first);           // (uniform; a tile spans at most 32 pages)
            const int64_t tok = tb + ln;
            const int lp = page_of(tok);
            const int pg = __builtin_amdgcn_ds_bpermute((lp - win) << 2, pg_win);
            // row index in the pool (of 128 bytes or more each: 32 bits reach past the memory of the GPU)
            const uint32_t row_idx = (static_cast<uint32_t>(pg) * a.Hkv + t.kvh) * static_cast<uint32_t>(a.P) + static_cast<uint32_t>(tok - static_cast<int64_t>(lp) * a.P);
            constexpr int kKChunks = S::kKRow / 16, kVChunks = S::kVRow / 16;
#pragma unroll
            for (int j0 = 0; j0 < S::kKBytes / 1024; j0 += 4) {
                const int c = (j0 + wave) * kWave + lane, r = c / kKChunks, pos = c - r * kKChunks;
                if (S::kKBytes / 1024 % 4 != 0 && j0 + wave >= S::kKBytes / 1024) break;
                const uint32_t from = __builtin_amdgcn_ds_bpermute(r << 2, row_idx);
                const unsigned char* src = a.k_pages + static_cast<size_t>(from) * S::kKRow + ((pos ^ k_swz<S::kKRow>(r)) << 4);
                __builtin_amdgcn_global_load_lds((const SEER_AS1 void*)(src), (SEER_AS3 void*)(lds + stage + (j0 + wave) * 1024), 16, 0, 0);
            }
#pragma unroll
            for (int j0 = 0; j0 < S::kVBytes / 1024; j0 += 4) {
                const int c = (j0 + wave) * kWave + lane, r = c / kVChunks, pos = c - r * kVChunks;
                if (S::kVBytes / 1024 % 4 != 0 && j0 + wave >= S::kVBytes / 1024) break;
                const uint32_t from = __builtin_amdgcn_ds_bpermute(r << 2, row_idx);
                const unsigned char* src = a.v_pages + static_cast<size_t>(from) * S::kVRow + ((pos ^ v_swz<S::kVRow>(r)) << 4);
                __builtin_amdgcn_global_load_lds((const SEER_AS1 void*)(src), (SEER_AS3 void*)(lds + stage + S::kKBytes + (j0 + wave) * 1024), 16, 0, 0);
            }
        };
        __syncthreads();                            // every wave is done with the stages of the piece before
        if (u0 < u1) issue_tile(u0, 0);
        for (int u = u0; u < u1; ++u) {
            const int stage = ((u - u0) & 1) * S::kStage;
            wait_vmcnt<0>();
            bare_barrier();                         // tile u has landed for every wave, every wave is done with tile u - 1
            if (u + 1 < u1) issue_tile(u + 1, S::kStage - stage);
            __builtin_amdgcn_sched_barrier(0);
            const int tb = u * kTile;
            uint32_t nonfinite = 0;                 // uniform: positions of this tile whose V row is kept out of the product
            if (tb + kTile - 1 > static_cast<int>(t.r.past) + token_first) {
                unsigned char* vl = lds + stage + S::kKBytes;
                if (tid == 0) s_found = 0;
                __builtin_amdgcn_s_waitcnt(0xc07f);
                bare_barrier();
                const uint32_t found = tile_nonfinite<DQK, DV>(vl, tid, kPromptThreads);
                if (found) atomicOr(&s_found, found);
                __builtin_amdgcn_s_waitcnt(0xc07f);
                bare_barrier();
                nonfinite = __builtin_amdgcn_readfirstlane(*const_cast<volatile uint32_t*>(&s_found));
                if (nonfinite) {
                    tile_clear_rows<DQK, DV>(vl, nonfinite, tid, kPromptThreads);
                    __builtin_amdgcn_s_waitcnt(0xc07f);
                }
                bare_barrier();
            }
            if (tb > sees_hi) continue;             // (wave-uniform)
            f32x16 s = tile_scores<DQK, DV>(lds0 + stage, operands, qreg);
            const int lim = sees - tb;              // last position of the tile that the row sees
            const uint64_t word = lim < 0 ? 0 : (lim >= 31 ? 0xffffffffull : (2ull << lim) - 1);
            if (tb + kTile - 1 > sees_lo) tile_mask(s, word, 0);
            float alpha;
            uint32_t term[1][8];
            tile_softmax<1>(s, a.scale_log2, top, m_run, l_run, alpha, term);
            if (__any(alpha != 1.f)) {
#pragma unroll
                for (int dt = 0; dt < S::kDTiles; ++dt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[dt][i] *= alpha;
            }
            tile_pv<DQK, DV, 1>(lds0 + stage, operands, term, acc);
            if (nonfinite)
                tile_add_rows<1>(nonfinite, term, word, 0, acc, [&](int j) __attribute__((always_inline)) -> const uint16_t* {
                    const int64_t tok = static_cast<int64_t>(tb) + j;
                    const int lp = page_of(tok);
                    const int pg = min(max(table[min(lp, a.max_pages - 1)], 0), a.num_pages - 1);
                    return reinterpret_cast<const uint16_t*>(a.v_pages) + ((static_cast<size_t>(pg) * a.Hkv + t.kvh) * a.P + (tok - static_cast<int64_t>(lp) * a.P)) * DV;
                });
        }

        // ---- the row tile's output, or this piece's share of it ------------------------------------------
        const float l_tot = l_run + __shfl_xor(l_run, 32, kWave);
        if (begins && (ends || t.r.bad)) {
            const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;          // (a row of nothing but -inf: zeros)
            if (row_ok) {
                uint16_t* o = a.out + q_row * DV + lg * 4;
#pragma unroll
                for (int dt = 0; dt < S::kDTiles; ++dt)
#pragma unroll
                    for (int i4 = 0; i4 < 4; ++i4)
                        *reinterpret_cast<u32x2*>(o + dt * 32 + i4 * 8) = u32x2{cvt_pk_bf16(acc[dt][i4 * 4] * inv, acc[dt][i4 * 4 + 1] * inv),
                                                                               cvt_pk_bf16(acc[dt][i4 * 4 + 2] * inv, acc[dt][i4 * 4 + 3] * inv)};
            }
            continue;
        }
        const size_t slot = 2 * static_cast<size_t>(w) + (begins ? 1 : 0);
        if (begins) cut = PromptCut{t.b, t.kvh, t.i, pieces_of(plan, t, w)};
        if (row_ok) {
            const size_t prow = slot * kRowTile + wave * 32 + ln;
            if (lg == 0) a.part_ml[2 * prow] = m_run, a.part_ml[2 * prow + 1] = l_tot;
            float* po = a.part_acc + prow * DV + lg * 4;
#pragma unroll
            for (int dt = 0; dt < S::kDTiles; ++dt)
#pragma unroll
                for (int i4 = 0; i4 < 4; ++i4)
                    *reinterpret_cast<f32x4*>(po + dt * 32 + i4 * 8) = f32x4{acc[dt][i4 * 4], acc[dt][i4 * 4 + 1], acc[dt][i4 * 4 + 2], acc[dt][i4 * 4 + 3]};
        }
    }
    if (tid == 0) a.cuts[w] = cut;
    if (a.status && __any(bad_page) && lane == 0) atomicOr(a.status, 2);
}

// Joins the pieces of the row tile that was cut at the end of stretch blockIdx.x, eight rows a workgroup.
constexpr int kJoinRows = 8;

template <int DV>
__global__ __launch_bounds__(kPromptThreads) void prompt_join_kernel(PromptArgs a) {
    const int w = blockIdx.x / (kRowTile / kJoinRows), part = blockIdx.x % (kRowTile / kJoinRows);
    const PromptCut cut = a.cuts[w];
    if (cut.pieces < 2) return;
    const int first = a.first[cut.b], n = a.first[cut.b + 1] - first;
    const int64_t row0 = static_cast<int64_t>(cut.tile) * kRowTile;
    constexpr int kThreadsPerRow = kPromptThreads / kJoinRows, kEach = DV / kThreadsPerRow;      // 32 threads a row
    const int r = part * kJoinRows + threadIdx.x / kThreadsPerRow, d = threadIdx.x % kThreadsPerRow * kEach;
    const int64_t row = row0 + r;
    if (row >= static_cast<int64_t>(n) * a.G) return;
    auto slot = [&](int k) { return (2 * static_cast<size_t>(w + k) + (k == 0 ? 1 : 0)) * kRowTile + r; };
    float m = kNegInf;
    for (int k = 0; k < cut.pieces; ++k) m = fmaxf(m, a.part_ml[2 * slot(k)]);
    float l = 0.f, o[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) o[i] = 0.f;
#pragma unroll 4
    for (int k = 0; k < cut.pieces; ++k) {
        const size_t at = slot(k);
        const float mk = a.part_ml[2 * at], lk = a.part_ml[2 * at + 1];
        const float f = mk == kNegInf ? 0.f : fast_exp2(mk - m);
        l = fmaf(lk, f, l);
#pragma unroll
        for (int i = 0; i < kEach; ++i) o[i] = fmaf(a.part_acc[at * DV + d + i], f, o[i]);
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int64_t token = row / a.G;
    uint16_t* out = a.out + ((static_cast<size_t>(first) + token) * a.Hq + cut.kvh * a.G + (row - token * a.G)) * DV + d;
#pragma unroll
    for (int i = 0; i < kEach; ++i) out[i] = f32_to_bf16(o[i] * inv);
}

static hipError_t launch_join(const PromptArgs& a, hipStream_t stream) {
    const dim3 grid(a.W * (kRowTile / kJoinRows));
    if (a.Dv == 64) hipLaunchKernelGGL((prompt_join_kernel<64>), grid, dim3(kPromptThreads), 0, stream, a);
    else if (a.Dv == 128) hipLaunchKernelGGL((prompt_join_kernel<128>), grid, dim3(kPromptThreads), 0, stream, a);
    else if (a.Dv == 256) hipLaunchKernelGGL((prompt_join_kernel<256>), grid, dim3(kPromptThreads), 0, stream, a);
    else hipLaunchKernelGGL((prompt_join_kernel<512>), grid, dim3(kPromptThreads), 0, stream, a);
    return hipGetLastError();
}

template <int DQK, int DV>
static hipError_t launch_prompt(const PromptArgs& a, hipStream_t stream) {
    hipLaunchKernelGGL((prompt_tile_kernel<DQK, DV>), dim3(a.W), dim3(kPromptThreads), 0, stream, a);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
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
    // positions are counted in 32 bits, the line of row tiles in 64, rows of the pool in 32
    if (ctx > 0x7fffffffLL - 65536 || static_cast<int64_t>(p->num_pages) * p->page_size * p->Hkv > 0xffffffffLL) return SEER_ESHAPE;
    const double tiles = static_cast<double>(n_tokens) * G / kRowTile + p->B;
    if (tiles * p->Hkv * (static_cast<double>(G) * (ctx + kTileCost) + static_cast<double>(n_tokens) * G + kRowTile) > 4e15) return SEER_ESHAPE;
    return SEER_OK;
}
struct PromptLayout {
    int W;
    size_t off_ml, off_acc, total;
};
static PromptLayout prompt_layout(const seer_attn_params& p, int32_t n_tokens) {
    PromptLayout w{};
    // no more stretches than the GPU holds at once, nor than the host can see work for
    int resident = 256 * prompt_waves_per_simd(p.Dqk);
    const int64_t ctx = static_cast<int64_t>(p.max_pages_per_seq) * p.page_size, G = p.Hq / p.Hkv;
    const int64_t requests = p.B < n_tokens ? p.B : n_tokens;
    const double row_tiles = (static_cast<double>(n_tokens) * G / kRowTile + requests) * p.Hkv;
    const double most = row_tiles * (static_cast<double>(ctx + kTileCost + kRowTile) / kMinStretch + 2);
    if (most < resident) resident = static_cast<int>(most);
    w.W = (resident + 7) / 8 * 8;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    w.off_ml = up(sizeof(PromptCut) * w.W);
    w.off_acc = w.off_ml + up(sizeof(float) * 2 * kRowTile * 2 * w.W);
    w.total = w.off_acc + sizeof(float) * kRowTile * p.Dv * 2 * w.W;
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
    a.n_tokens = n_tokens, a.Dqk = p->Dqk, a.Dv = p->Dv, a.W = layout.W;
    a.page_shift = (p->page_size & (p->page_size - 1)) == 0 ? __builtin_ctz(static_cast<unsigned>(p->page_size)) : -1;
    a.scale_log2 = p->scale * seer::kLog2e;
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
