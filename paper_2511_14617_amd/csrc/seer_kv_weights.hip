// seer_kv_weights: the attention weight that the tokens of a step gave to every cached position, added to running sums.
//
// For a request whose cache now holds n positions, the last R of them from this step (the root and the accepted draft tokens), row i of
// the step sees positions 0 .. n - R + i.  With s_rj = scale q_r . k_j for every row r = (i, head g of the group) and
// lse_r = ln sum_j exp s_rj over what the row sees,
//   w_j <- decay w_j (0 for the step's own positions) + sum_r exp(s_rj - lse_r).
//
// What bounds it: HBM for a few rows, the matrix cores for the many rows of a shared latent.  A weight needs its row's denominator, so the keys are swept
// twice, with the same loads and matrix products: kv_sweep<.., false> leaves each row's running maximum and sum per piece,
// kv_lse joins them, kv_sweep<.., true> exponentiates again and adds up the rows of each position.
//
// Work decomposition: per KV head the 32-token tiles of all requests, each times its row blocks of 32 NW rows, lie on one line, cut
// into equal stretches, one per workgroup, all of them resident at once.  Every workgroup finds its stretch from the lengths
// (line_of, one request per lane).  A piece is a request's part of a stretch; piece (w, b) has partial slot w + b (along the line every
// next piece raises one of the two).  Tiles go from the pool to LDS directly (32 rows of 16-byte chunks, swizzled as in
// seer_tile.h), wave i holds 32 query rows in registers.  The first sweep multiplies K.Q^T (a row per lane: its maximum and
// sum stay in the lane), the second Q.K^T (a token per lane: the sum over the rows stays in the lane).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/seer_verify.h"
#include "seer_device.h"
#include "seer_tile.h"

namespace seer {

constexpr int kSwTile = 32;            // tokens of a tile
constexpr int kSwChunk = 32;           // tiles whose sums are collected in LDS before they go to memory
constexpr int kSwStages = 2;
constexpr int kSwMaxStretches = 2048;
constexpr int kLseThreads = 256, kLseRows = 8;

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

__device__ __forceinline__ int wave_scan(int v) {          // inclusive
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
        const int x = __shfl_up(v, o, kWave);
        if ((static_cast<int>(threadIdx.x) & (kWave - 1)) >= o) v += x;
    }
    return v;
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

template <int DQK, int NW, bool WEIGHTS>
__global__ __launch_bounds__(NW * kWave) void kv_sweep(KvWeightsArgs a) {
    using K = Keys<DQK>;
    constexpr int kLoads = K::kBytes / 1024 / NW;           // direct-to-LDS loads of a wave per tile
    static_assert(K::kBytes % (1024 * NW) == 0 && kLoads * (kSwStages - 1) < 64, "");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[kSwStages * K::kBytes];
    __shared__ float s_sums[WEIGHTS ? NW : 1][WEIGHTS ? kSwChunk * kSwTile : 1];

    const int kvh = blockIdx.x % a.Hkv, w = blockIdx.x / a.Hkv;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), ln = lane & 31, lg = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
    const unsigned char* __restrict__ kbase = static_cast<const unsigned char*>(a.k_pages);
    const int lds0 = tile::lds_addr(lds);
    const int k_rd = ln * K::kRow + ((lg ^ tile::k_swz<K::kRow>(ln)) << 4);
    const bool page_pow2 = (a.P & (a.P - 1)) == 0;
    const int page_shift = __builtin_ctz(static_cast<unsigned>(a.P));
    auto page_of = [&](int tok) __attribute__((always_inline)) -> int { return page_pow2 ? tok >> page_shift : tok / a.P; };
    int found = 0;                                          // status bits

    // ---- the line: its length, then the pieces of this stretch, 64 requests at a time -------------------------------
    int total = 0;
    for (int b0 = 0; b0 < a.B; b0 += kWave) {
        bool bad = false;
        int u = 0;
        if (b0 + lane < a.B) u = units_of(a, step_rows(a, b0 + lane, bad));
        if (!WEIGHTS && blockIdx.x == 0 && bad) found |= 1;
        const int incl = wave_scan(u);
        if (!WEIGHTS && blockIdx.x == 0 && wave == 0 && b0 + lane < a.B) a.line[1 + b0 + lane] = total + incl - u;
        total += __builtin_amdgcn_readlane(incl, kWave - 1);
    }
    const int step = max(1, (total + a.W - 1) / a.W);
    if (!WEIGHTS && blockIdx.x == 0 && tid == 0) a.line[0] = step, a.line[1 + a.B] = total;
    const int u_begin = min(w * step, total), u_end = min(u_begin + step, total);

    int before = 0;                                         // units of the requests in front of b0
    for (int b0 = 0; b0 < a.B && before < u_end; b0 += kWave) {
        bool bad = false;
        StepRows mine{0, 0};
        if (b0 + lane < a.B) mine = step_rows(a, b0 + lane, bad);
        const int my_units = units_of(a, mine), incl = wave_scan(my_units), my_off = before + incl - my_units;
        uint64_t todo = __ballot(my_units > 0 && my_off < u_end && my_off + my_units > u_begin);
        before += __builtin_amdgcn_readlane(incl, kWave - 1);
        for (; todo; todo &= todo - 1) {
            const int bit = __builtin_ctzll(todo), b = b0 + bit;
            const int off = __builtin_amdgcn_readlane(my_off, bit), n = __builtin_amdgcn_readlane(mine.n, bit);
            const int rows = __builtin_amdgcn_readlane(mine.rows, bit), R = rows * a.G, blocks = row_blocks_of(a, rows);
            const int n_tiles = (n + kSwTile - 1) / kSwTile;
            const int t_begin = min(n_tiles, (max(u_begin - off, 0) + blocks - 1) / blocks);
            const int t_end = min(n_tiles, (u_end - off + blocks - 1) / blocks);

            // the step's slots (lane i: row i's), which have to ascend from the root
            int slot = lane;
            if (a.accepted_path) {
                slot = lane < rows ? a.accepted_path[static_cast<size_t>(b) * a.T + lane] : a.T;
                const int up = __shfl_up(slot, 1, kWave);
                const bool wrong = lane < rows && (lane == 0 ? slot != 0 : slot <= up || slot >= a.T);
                if (__any(wrong)) {
                    if (!WEIGHTS) found |= 4;
                    continue;
                }
            }

            // ---- tile loads --------------------------------------------------------------------------
            const int32_t* __restrict__ table = a.block_table + static_cast<size_t>(b) * a.max_pages;
            const int last_page = (n - 1) / a.P;
            int win = 0, pg_win = 0;                        // lane l holds the (clamped) page id of logical page win + l
            bool have_window = false;
            auto issue_tile = [&](int t, int stage) __attribute__((always_inline)) {
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
#pragma unroll
                for (int j = 0; j < kLoads; ++j) {
                    const int c = (wave * kLoads + j) * kWave + lane, row = c / K::kRowChunks, pos = c - row * K::kRowChunks;
                    const uint32_t r = __builtin_amdgcn_ds_bpermute(row << 2, row_idx);
                    const unsigned char* src = kbase + static_cast<size_t>(r) * K::kRow + ((pos ^ tile::k_swz<K::kRow>(row)) << 4);
                    __builtin_amdgcn_global_load_lds((const SEER_AS1 void*)(src), (SEER_AS3 void*)(lds + stage * K::kBytes + (wave * kLoads + j) * 1024), 16, 0, 0);
                }
            };

            // Tiles t0 .. t1 - 1, each handed to `use` with its LDS address once it has landed for every wave.
            auto sweep = [&](int t0, int t1, auto&& use) __attribute__((always_inline)) {
                if (NW > 1) bare_barrier();                 // every wave is done with the stages
#pragma unroll
                for (int s = 0; s < kSwStages - 1; ++s)
                    if (t0 + s < t1) issue_tile(t0 + s, s);
                int stage = 0;
                for (int t = t0; t < t1; ++t) {
                    if (t + kSwStages - 1 <= t1) wait_vmcnt<kLoads * (kSwStages - 2)>(); else wait_vmcnt<0>();
                    if (NW > 1) bare_barrier();
                    const int next = stage == 0 ? kSwStages - 1 : stage - 1;
                    if (t + kSwStages - 1 < t1) issue_tile(t + kSwStages - 1, next);
                    __builtin_amdgcn_sched_barrier(0);
                    use(t, lds0 + stage * K::kBytes);
                    __builtin_amdgcn_sched_barrier(0);
                    stage = stage + 1 == kSwStages ? 0 : stage + 1;
                }
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

            if constexpr (!WEIGHTS) {
                for (int block = 0; block < blocks; ++block) {
                    const int r = load_rows(block);
                    const int seen = first_own + min(r, R - 1) / a.G + 1;
                    float m_run = kNegInf, l_run = 0.f;
                    sweep(t_begin, t_end, [&](int t, int at) __attribute__((always_inline)) {
                        f32x16 s = sweep_scores<DQK, false>(at, k_rd, q);
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
                    });
                    const float l = l_run + __shfl_xor(l_run, 32, kWave);
                    if (lg == 0 && r < R) a.part[(static_cast<size_t>(w + b) * a.Hkv + kvh) * (a.G * a.T) + r] = make_float2(m_run, l);
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
                        float denom[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) denom[i] = __shfl(own, (i >> 2) * 8 + lg * 4 + (i & 3), kWave);
                        const int row_i = min(r, R - 1) / a.G;
                        sweep(c0, c1, [&](int t, int at) __attribute__((always_inline)) {
                            f32x16 s = sweep_scores<DQK, true>(at, k_rd, q);
                            const int tb = t * kSwTile;
#pragma unroll
                            for (int i = 0; i < 16; ++i) s[i] = fast_exp2(fmaf(s[i], a.scale_log2, -denom[i]));
                            if (partial) {
#pragma unroll
                                for (int i = 0; i < 16; ++i)
                                    if (denom[i] == -kNegInf) s[i] = 0.f;
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
                            float* at_sum = &s_sums[wave][(t - c0) * kSwTile + ln];
                            if (lg == 0) *at_sum = block ? *at_sum + sum : sum;
                        });
                    }
                    __syncthreads();
                    const int tokens = min(n, c1 * kSwTile) - c0 * kSwTile;
                    for (int j = tid; j < tokens; j += NW * kWave) {
                        float sum = s_sums[0][j];
#pragma unroll
                        for (int x = 1; x < NW; ++x) sum += s_sums[x][j];
                        const int pos = c0 * kSwTile + j;
                        to[pos] = pos < first_own ? fmaf(a.decay, to[pos], sum) : sum;
                    }
                    __syncthreads();
                }
            }
        }
    }
    if (!WEIGHTS && a.status && found) atomicOr(a.status, found);
}

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
            l = l * fast_exp2(m - use) + (p.x == kNegInf ? 0.f : p.y * fast_exp2(p.x - use));
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
        const float2 p = s_part[s * kLseRows + tid];
        sum += p.x == kNegInf ? 0.f : p.y * fast_exp2(p.x - top);
    }
    // a row that weighs nothing (all its scores -inf): +inf, so that exp2 gives 0
    a.lse[(static_cast<size_t>(b) * a.Hkv + kvh) * GT + r] = top == kNegInf ? -kNegInf : top + log2f(sum);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
struct KvWeightsLayout {
    int waves, W;
    size_t off_part, off_lse, total;
};
inline KvWeightsLayout kv_weights_layout(const seer_attn_params& p) {
    KvWeightsLayout w{};
    const int rows = (p.Hq / p.Hkv) * p.T;
    w.waves = rows <= 32 ? 1 : rows <= 64 ? 2 : 4;
    const int lds_kb = (kSwStages * kSwTile * p.Dqk * 2 + w.waves * kSwChunk * kSwTile * 4) / 1024 + 1;
    int per_cu = 159 / lds_kb;
    if (per_cu > 8 / w.waves) per_cu = 8 / w.waves;
    if (per_cu < 1) per_cu = 1;
    w.W = 256 * per_cu / p.Hkv;
    if (w.W < 1) w.W = 1;
    if (w.W > kSwMaxStretches) w.W = kSwMaxStretches;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t per_head = static_cast<size_t>(p.Hq) * p.T;          // Hkv * G * T
    w.off_part = up(sizeof(int32_t) * (static_cast<size_t>(p.B) + 2));
    w.off_lse = w.off_part + up(sizeof(float2) * (static_cast<size_t>(w.W) + p.B) * per_head);
    w.total = w.off_lse + up(sizeof(float) * static_cast<size_t>(p.B) * per_head);
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
    return SEER_OK;
}

template <int DQK, int NW>
hipError_t launch_kv_weights(const KvWeightsArgs& a, hipStream_t stream) {
    const dim3 grid(static_cast<unsigned>(a.W) * static_cast<unsigned>(a.Hkv)), block(NW * kWave);
    hipLaunchKernelGGL((kv_sweep<DQK, NW, false>), grid, block, 0, stream, a);
    const unsigned groups = static_cast<unsigned>((a.G * a.T + kLseRows - 1) / kLseRows);
    hipLaunchKernelGGL(kv_lse, dim3(static_cast<unsigned>(a.B) * static_cast<unsigned>(a.Hkv) * groups), dim3(kLseThreads), 0, stream, a);
    hipLaunchKernelGGL((kv_sweep<DQK, NW, true>), grid, block, 0, stream, a);
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
    a.ldw = static_cast<int64_t>(p->max_pages_per_seq) * p->page_size;
    a.B = p->B, a.T = p->T, a.Hq = p->Hq, a.Hkv = p->Hkv, a.G = p->Hq / p->Hkv, a.P = p->page_size;
    a.num_pages = p->num_pages, a.max_pages = p->max_pages_per_seq, a.max_ctx = static_cast<int>(a.ldw);
    a.W = w.W, a.block_rows = 32 * w.waves;
    a.scale_log2 = p->scale * seer::kLog2e, a.decay = decay;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
#define SEER_SWEEP(DQK, NW) \
    if (p->Dqk == DQK && w.waves == NW) return static_cast<int>(seer::launch_kv_weights<DQK, NW>(a, stream));
#define SEER_SWEEPS(DQK) SEER_SWEEP(DQK, 1) SEER_SWEEP(DQK, 2) SEER_SWEEP(DQK, 4)
    SEER_SWEEPS(64)
    SEER_SWEEPS(128)
    SEER_SWEEPS(192)
    SEER_SWEEPS(256)
    SEER_SWEEPS(576)
#undef SEER_SWEEPS
#undef SEER_SWEEP
    return SEER_EUNSUPPORTED;
}
