// seer_token_logprobs: log probability of given tokens under softmax(logits / temperature), the entropy of each row and
// its most probable alternatives; seer_token_logprobs_grad: the gradient of log probability and entropy with respect to the logits.
//
// With z = x / tau, m = max z, l = sum exp(z - m):  logsumexp = m + ln l,  log p_y = z_y - logsumexp,
// H = ln l - (sum exp(z - m) (z - m)) / l.  All three sums come from one pass over the row, and so do the alternatives.
// Gradient: d(log p_y)/dx_v = (1[v = y] - p_v) / tau,  dH/dx_v = -p_v (ln p_v + H) / tau, with p_v = exp(z_v - logsumexp).
//
// What bounds it: HBM, one read of the logits (gradient: one read and one write).  Rows are cut into chunks so that a launch
// fills the chip whatever rows * V is (logprob_scan); a second kernel joins the chunks of a row (logprob_join).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/seer_verify.h"
#include "seer_device.h"
#include "seer_plan.h"
#include "seer_tile.h"

namespace seer {

constexpr int kLpThreads = 256;
constexpr int kLpWaves = kLpThreads / kWave;
constexpr int kLpMaxCand = 1024;        // candidates for the alternatives that a workgroup keeps in LDS
constexpr float kLowest = -1e4f;        // exp2 of this is 0: keeps 0 * -inf out of the entropy's sum
constexpr float kLn2f = 0.693147181f;

// Rows begin at any element (odd vocabularies, padded strides): vector loads and stores that assume the element's alignment only.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <int DTYPE>
struct Elem;
template <>
struct Elem<SEER_F32> {
    typedef float T;
    static constexpr int kVec = 4;
    typedef f32x4 Vec;
    static __device__ __forceinline__ Vec load(const T* p) { return __builtin_nontemporal_load(reinterpret_cast<const f32x4_any*>(p)); }
    static __device__ __forceinline__ Vec none() { return f32x4{kNegInf, kNegInf, kNegInf, kNegInf}; }
    static __device__ __forceinline__ float get(const Vec& v, int i) { return v[i]; }
    static __device__ __forceinline__ float one(const T* p) { return *p; }
    static __device__ __forceinline__ void store(T* p, const float (&g)[kVec]) {
        __builtin_nontemporal_store(f32x4{g[0], g[1], g[2], g[3]}, reinterpret_cast<f32x4_any*>(p));
    }
    static __device__ __forceinline__ void store_one(T* p, float g) { *p = g; }
};
template <>
struct Elem<SEER_BF16> {
    typedef uint16_t T;
    static constexpr int kVec = 8;
    typedef u32x4 Vec;
    static __device__ __forceinline__ Vec load(const T* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p)); }
    static __device__ __forceinline__ Vec none() { return u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
    static __device__ __forceinline__ float get(const Vec& v, int i) { return i & 1 ? bf16hi_to_f32(v[i >> 1]) : bf16lo_to_f32(v[i >> 1]); }
    static __device__ __forceinline__ float one(const T* p) { return bf16_to_f32(*p); }
    static __device__ __forceinline__ void store(T* p, const float (&g)[kVec]) {
        __builtin_nontemporal_store(u32x4{cvt_pk_bf16(g[0], g[1]), cvt_pk_bf16(g[2], g[3]), cvt_pk_bf16(g[4], g[5]), cvt_pk_bf16(g[6], g[7])},
                                    reinterpret_cast<u32x4_any*>(p));
    }
    static __device__ __forceinline__ void store_one(T* p, float g) { *p = f32_to_bf16(g); }
};

// Over the lanes of a wave through DPP, in every lane.
__device__ __forceinline__ float all_sum(float v) { return last_lane(wave_incl_scan(v)); }
template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float max_step(float v) {
    const int x = __float_as_int(v);
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(x, x, CTRL, ROW_MASK, 0xf, false)));
}
__device__ __forceinline__ float all_max(float v) {
    v = max_step<0x111, 0xf>(v);
    v = max_step<0x112, 0xf>(v);
    v = max_step<0x114, 0xf>(v);
    v = max_step<0x118, 0xf>(v);
    v = max_step<0x142, 0xa>(v);
    v = max_step<0x143, 0xc>(v);
    return last_lane(v);
}

struct LogprobArgs {
    const void* logits;
    const int32_t* tokens;
    const int32_t* path;          // nullptr: output row = logits row
    int64_t ld;
    int T, V, n_chunks, chunk, top_n;      // chunk: elements of one
    float inv_tau;
    float* part;                  // [rows][n_chunks][3]: maximum of x, sum of exp2(d), sum of exp2(d) d, d = (x - maximum) log2(e) / tau
    uint64_t* part_top;           // [rows][n_chunks][top_n] keys, descending, 0 = none
    float* logprob;
    float* entropy;               // may be nullptr, as the two below
    float* logsumexp;
    float* top_logprob;
    int32_t* top_token;
};

// The logits row that output row r is about, -1: none (no token, or a place behind the accepted path).
__device__ __forceinline__ int64_t logits_row(const LogprobArgs& a, int r, int& token) {
    token = a.tokens[r];
    if (token < 0 || token >= a.V) return -1;
    if (!a.path) return r;
    const int slot = a.path[r];
    if (slot < 0 || slot >= a.T) return -1;
    return static_cast<int64_t>(r / a.T) * a.T + slot;
}

constexpr uint32_t kOrderedNegInf = 0x007fffffu;
// Keys of alternatives: larger value first, then lower index.
__device__ __forceinline__ uint64_t alt_key(uint32_t value, int index) { return static_cast<uint64_t>(value) << 32 | static_cast<uint32_t>(~index); }

// A value that at least n lanes' values reach (n <= 64): the n-th largest with its low 12 bits cleared, found bit by bit with one ballot each.
__device__ __forceinline__ uint32_t wave_nth_largest(uint32_t v, int n) {
    uint32_t at = 0;
    for (int bit = 31; bit >= 12; --bit) {
        const uint32_t probe = at | 1u << bit;
        if (__popcll(__ballot(v >= probe)) >= n) at = probe;
    }
    return at;
}

template <int DTYPE, int kChunk, bool TOP>
__global__ __launch_bounds__(kLpThreads) void logprob_scan(LogprobArgs a) {
    using E = Elem<DTYPE>;
    constexpr int kVec = E::kVec, kIter = kChunk / (kLpThreads * kVec);
    __shared__ float s_max[kLpWaves], s_sum[kLpWaves][2];
    const int r = blockIdx.x / a.n_chunks, chunk = blockIdx.x - r * a.n_chunks;
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
    const int begin = min(a.V, chunk * a.chunk), end = min(a.V, begin + a.chunk);
    // (without a path the logits are requested beside the token, not behind it)
    int token;
    int64_t row = r;
    if (a.path && (row = logits_row(a, r, token)) < 0) return;
    const typename E::T* base = static_cast<const typename E::T*>(a.logits) + row * a.ld;

    // whole vectors, then one element of the last, incomplete one
    typename E::Vec x[kIter];
#pragma unroll
    for (int it = 0; it < kIter; ++it) {
        const int i = begin + (it * kLpThreads + tid) * kVec;
        x[it] = i + kVec <= end ? E::load(base + i) : E::none();
    }
    const int rest = begin + (end - begin) / kVec * kVec + tid;
    const float x_rest = rest < end ? E::one(base + rest) : kNegInf;
    if (!a.path && logits_row(a, r, token) < 0) return;

    float top = x_rest;
#pragma unroll
    for (int it = 0; it < kIter; ++it)
#pragma unroll
        for (int c = 0; c < kVec; ++c) top = fmaxf(top, E::get(x[it], c));
    const float wave_top = all_max(top);
    if (lane == 0) s_max[wave] = wave_top;
    __syncthreads();
    float m = s_max[0];
#pragma unroll
    for (int w = 1; w < kLpWaves; ++w) m = fmaxf(m, s_max[w]);

    // d = v scale - c with c = m scale rounded: one fused multiply-add, exact but for its last rounding, and an unpacking, two sums and the exponential beside
    // it are what a logit costs (with the difference, the product and a clamp against -inf apart the bf16 scan was bound by them: 4096
    // rows of 151 936 in 215 us).  m itself then has the rounding of c for its d, a quarter at most below 2^22; beyond (chunks of a
    // finite mask value, small temperatures), where it would grow until exp2 overflows or vanishes, and where a logit of -inf makes the second sum a
    // NaN, a wave goes over its logits again, with the difference taken first.
    const float scale = a.inv_tau * kLog2e, c = m * scale;
    const bool usual = fabsf(c) < 0x1p22f;
    float l = 0.f, s = 0.f;
    auto add = [&](float v) __attribute__((always_inline)) {
        const float d = fmaf(v, scale, -c), e = fast_exp2(d);      // (a NaN reaches l, and through it every result of the row)
        l += e;
        s = fmaf(e, d, s);
    };
    auto add_with_care = [&](float v) __attribute__((always_inline)) {
        const float d = (v - (m == kNegInf ? 0.f : m)) * scale, e = fast_exp2(d);
        l += e;
        s = fmaf(e, fmaxf(d, kLowest), s);
    };
    auto every = [&](auto&& use) __attribute__((always_inline)) {
#pragma unroll
        for (int it = 0; it < kIter; ++it)
            if (begin + (it * kLpThreads + tid) * kVec + kVec <= end) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) use(E::get(x[it], i));
            }
    };
    every(add);
    if (rest < end) add(x_rest);
    if (!usual || __any(s != s)) {
        l = s = 0.f;
        every(add_with_care);
        add_with_care(x_rest);
        l = all_sum(l), s = all_sum(s);
    } else {
        l = all_sum(l), s = all_sum(s);
        // from c to m itself
        const float off = fmaf(m, scale, -c), f = fast_exp2(-off);
        s = f * fmaf(-off, l, s), l *= f;
    }
    if (lane == 0) s_sum[wave][0] = l, s_sum[wave][1] = s;

    if constexpr (TOP) {
        // Alternatives of the chunk: an element below the n-th largest of a wave's 64 lane maxima is none of the n first, so only
        // the few that reach the largest such bound of the four waves are ranked, each by counting the ones before it.  Elements of
        // -inf take no part (logprob_join puts them in where a row has too few others).
        __shared__ uint32_t s_bound[kLpWaves];
        __shared__ uint64_t s_cand[kLpMaxCand];
        __shared__ int s_count;
        const int n = a.top_n;
        const uint32_t mine = ordered(top), bound_wave = wave_nth_largest(mine, n);
        if (lane == 0) s_bound[wave] = bound_wave;
        if (tid == 0) s_count = 0;
        __syncthreads();
        uint32_t bound = kOrderedNegInf + 1;
#pragma unroll
        for (int w = 0; w < kLpWaves; ++w) bound = max(bound, s_bound[w]);
        auto offer = [&](float v, int index) __attribute__((always_inline)) {
            const uint32_t k = ordered(v);
            if (k >= bound) {
                const int at = atomicAdd(&s_count, 1);
                if (at < kLpMaxCand) s_cand[at] = alt_key(k, index);
            }
        };
        if (__any(mine >= bound)) {
#pragma unroll
            for (int it = 0; it < kIter; ++it) {
                float v = E::get(x[it], 0);
#pragma unroll
                for (int c = 1; c < kVec; ++c) v = fmaxf(v, E::get(x[it], c));
                if (ordered(v) >= bound) {
#pragma unroll
                    for (int c = 0; c < kVec; ++c) offer(E::get(x[it], c), begin + (it * kLpThreads + tid) * kVec + c);
                }
            }
            if (rest < end) offer(x_rest, rest);
        }
        __syncthreads();
        const int count = s_count;
        uint64_t* out = a.part_top + static_cast<size_t>(blockIdx.x) * n;
        if (count <= kLpMaxCand) {
            for (int i = tid; i < count; i += kLpThreads) {
                const uint64_t k = s_cand[i];
                int before = 0;
#pragma unroll 8
                for (int j = 0; j < count; ++j) before += s_cand[j] > k ? 1 : 0;
                if (before < n) out[before] = k;
            }
            for (int i = count + tid; i < n; i += kLpThreads) out[i] = 0;
        } else {
            // More equal values than the list holds (a flat row): one after the other, the largest key below the last one taken.
            // (Read again: with the chunk kept in registers for this, the kernel took 167 of them.)
            uint64_t last = ~0ull;
            for (int k = 0; k < n; ++k) {
                uint64_t best = 0;
                for (int i = begin + tid; i < end; i += kLpThreads) {
                    const float v = E::one(base + i);
                    const uint64_t key = alt_key(ordered(v), i);
                    if (v != kNegInf && key < last && key > best) best = key;
                }
#pragma unroll
                for (int o = 32; o >= 1; o >>= 1) best = max(best, static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(best), o, kWave)));
                __syncthreads();
                if (lane == 0) s_cand[wave] = best;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kLpWaves; ++w) best = max(best, s_cand[w]);
                if (tid == 0) out[k] = best;
                last = best;
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        float* p = a.part + static_cast<size_t>(blockIdx.x) * 3;
#pragma unroll
        for (int w = 1; w < kLpWaves; ++w) l += s_sum[w][0], s += s_sum[w][1];
        p[0] = m, p[1] = l, p[2] = s;
    }
}

// One wave per row: the sums of its chunks brought to the row's maximum, and the n first of their lists.  Few keys (up to kJoinHold * 64) are taken
// at once: each lane's largest gives a bound that n keys reach (as in logprob_scan), the keys that reach it are ranked by counting.
// More of them, or more than kJoinCand that reach it, are merged one by one, each lane holding the head of the lists lane, lane + 64, ..
// (always merged one by one, with the next head read from memory each time, it took 13 us for 38 lists of 20).
constexpr int kJoinHold = 20, kJoinCand = 256;

template <int DTYPE>
__global__ __launch_bounds__(kWave) void logprob_join(LogprobArgs a) {
    extern __shared__ uint8_t s_taken[];                    // per chunk: keys taken from its list
    __shared__ uint64_t s_cand[kJoinCand];
    const int r = blockIdx.x, lane = threadIdx.x, n = a.top_n;
    const float* part = a.part + static_cast<size_t>(r) * a.n_chunks * 3;
    const uint64_t* lists = a.part_top + static_cast<size_t>(r) * a.n_chunks * n;
    // (what a row without an entry finds here is not used)
    float m = kNegInf;
    for (int c = lane; c < a.n_chunks; c += kWave) m = fmaxf(m, part[c * 3]);
    const int64_t total = static_cast<int64_t>(a.n_chunks) * n;
    const bool few = total <= kJoinHold * kWave;
    uint64_t key[kJoinHold];
    if (few) {
#pragma unroll
        for (int x = 0; x < kJoinHold; ++x) {
            key[x] = 0;
            if (x * kWave < total && x * kWave + lane < total) key[x] = lists[x * kWave + lane];
        }
    }
    int token;
    const int64_t row = logits_row(a, r, token);
    float* const alt_logp = a.top_logprob + static_cast<size_t>(r) * n;
    int32_t* const alt_token = a.top_token + static_cast<size_t>(r) * n;
    if (row < 0) {
        if (lane == 0) {
            a.logprob[r] = 0.f;
            if (a.entropy) a.entropy[r] = 0.f;
            if (a.logsumexp) a.logsumexp[r] = 0.f;
        }
        if (lane < n) alt_logp[lane] = 0.f, alt_token[lane] = -1;
        return;
    }
    const float x_token = Elem<DTYPE>::one(static_cast<const typename Elem<DTYPE>::T*>(a.logits) + row * a.ld + token);
    m = all_max(m);
    const float scale = a.inv_tau * kLog2e;
    float l = 0.f, s = 0.f;
    for (int c = lane; c < a.n_chunks; c += kWave) {
        const float d = part[c * 3] == kNegInf ? kLowest : (part[c * 3] - m) * scale, w = fast_exp2(d);
        l += w * part[c * 3 + 1];
        s += w * fmaf(part[c * 3 + 1], fmaxf(d, kLowest), part[c * 3 + 2]);
    }
    l = all_sum(l), s = all_sum(s);
    const float ln_l = logf(l);
    const bool empty = m == kNegInf && l == 0.f;             // every logit is -inf
    // (a row with a NaN or +inf, whose sum is a NaN, has no log probabilities, not even of its logits of -inf)
    auto logp = [&](float x) __attribute__((always_inline)) { return x == kNegInf && ln_l == ln_l ? kNegInf : (x - m) * a.inv_tau - ln_l; };
    if (lane == 0) {
        a.logprob[r] = logp(x_token);
        if (a.entropy) a.entropy[r] = empty ? 0.f : ln_l - kLn2f * (s / l);
        if (a.logsumexp) a.logsumexp[r] = empty ? kNegInf : fmaf(m, a.inv_tau, ln_l);
    }
    if (n == 0) return;
    auto write = [&](int at, uint64_t k) __attribute__((always_inline)) {
        alt_logp[at] = logp(unordered(static_cast<uint32_t>(k >> 32)));
        alt_token[at] = static_cast<int>(~static_cast<uint32_t>(k));
    };

    uint64_t mine = 0;                                      // (fewer than n finite logits: lane k's is the k-th alternative)
    int got = kWave;                                        // how many there are
    bool ranked = false;
    if (few) {
        uint64_t top = 0;
#pragma unroll
        for (int x = 0; x < kJoinHold; ++x) top = max(top, key[x]);
        const uint32_t bound = wave_nth_largest(static_cast<uint32_t>(top >> 32), n);
        int count = 0;
#pragma unroll
        for (int x = 0; x < kJoinHold; ++x) {
            if (x * kWave < total) {
                const bool in = key[x] != 0 && static_cast<uint32_t>(key[x] >> 32) >= bound;
                const uint64_t who = __ballot(in);
                const int at = count + __popcll(who & ((1ull << lane) - 1));
                if (in && at < kJoinCand) s_cand[at] = key[x];
                count += __popcll(who);
            }
        }
        if (count <= kJoinCand) {
            ranked = true;
            __syncthreads();
            for (int i = lane; i < count; i += kWave) {
                const uint64_t k = s_cand[i];
                int before = 0;
#pragma unroll 8
                for (int j = 0; j < count; ++j) before += s_cand[j] > k ? 1 : 0;
                if (before < n) write(before, k);
            }
            got = count;
            if (count < n && lane < count) mine = s_cand[lane];
        }
    }
    if (!ranked) {
        for (int c = lane; c < a.n_chunks; c += kWave) s_taken[c] = 0;
        uint64_t head = 0;
        int from = 0;
        auto find_head = [&]() __attribute__((always_inline)) {
            head = 0;
            for (int c = lane; c < a.n_chunks; c += kWave) {
                const int at = s_taken[c];
                const uint64_t k = at < n ? lists[static_cast<size_t>(c) * n + at] : 0;
                if (k > head) head = k, from = c;
            }
        };
        find_head();
        for (got = 0; got < n; ++got) {
            uint64_t best = head;
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) best = max(best, static_cast<uint64_t>(__shfl_xor(static_cast<unsigned long long>(best), o, kWave)));
            if (best == 0) break;
            if (lane == got) mine = best, write(got, best);
            if (head == best) {
                ++s_taken[from];
                find_head();
            }
        }
    }
    // fewer than n finite logits: the lowest indices that are not among them, whose logits are -inf
    const int index = static_cast<int>(~static_cast<uint32_t>(mine)), found = got;
    for (int v = 0; got < n; ++v) {
        if (__ballot(lane < found && index == v)) continue;
        if (lane == 0) alt_logp[got] = logp(kNegInf), alt_token[got] = v;
        ++got;
    }
}

struct LogprobGradArgs {
    void* grad;
    const void* logits;
    const int32_t* tokens;
    const float* logsumexp;
    const float* entropy;         // nullptr iff grad_entropy is
    const float* grad_logprob;
    const float* grad_entropy;
    int64_t ld, grad_ld;
    int V, n_chunks;
    float inv_tau;
};

// d(row) / d(logit) from its log probability; c0 = -g_lp - g_h entropy.
__device__ __forceinline__ float logit_grad(float logp, float g_lp, float g_h, float c0, bool is_token) {
    return fast_exp2(logp * kLog2e) * fmaf(-g_h, fmaxf(logp, kLowest), c0) + (is_token ? g_lp : 0.f);
}

// fp32 holds a logsumexp beyond this to steps of which p = exp(z - logsumexp) takes 2^-12 and more, until ln l is lost (a row that -1e9 masks
// throughout: steps of 64).  Such a row is the business of its first workgroup alone, which takes the row's own maximum and sum and then every element from its distance to
// the maximum: 16 rows of 152 064 fp32 logits 114 us (9 where all are near zero), 4096 of bf16 1020 (452).
constexpr float kLpFar = 4096.f;
constexpr int kFarHold = 4;              // vectors that a thread has in flight there (eight: 82 registers for bf16, and five workgroups a CU for all rows)

template <int DTYPE>
__device__ __forceinline__ void far_row_grad(const typename Elem<DTYPE>::T* base, typename Elem<DTYPE>::T* out, int V, int token, float inv_tau, float g_lp, float g_h, float c0) {
    using E = Elem<DTYPE>;
    constexpr int kVec = E::kVec, kStep = kLpThreads * kVec;
    __shared__ float s_max[kLpWaves], s_sum[kLpWaves];
    const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave, rest = V / kVec * kVec + tid;
    const float x_rest = rest < V ? E::one(base + rest) : kNegInf, scale = inv_tau * kLog2e;
    typename E::Vec x[kFarHold];
    auto load = [&](int i0) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < kFarHold; ++k) x[k] = i0 + k * kStep + kVec <= V ? E::load(base + i0 + k * kStep) : E::none();
    };
    float m = x_rest, l = x_rest == kNegInf ? 0.f : fast_exp2((x_rest - x_rest) * scale);      // of the thread's elements (a NaN reaches l)
    for (int i0 = tid * kVec; i0 < V; i0 += kFarHold * kStep) {
        load(i0);
        const float before = m;
#pragma unroll
        for (int k = 0; k < kFarHold; ++k)
#pragma unroll
            for (int c = 0; c < kVec; ++c) m = fmaxf(m, E::get(x[k], c));
        const float from = m == kNegInf ? 0.f : m;
        l *= fast_exp2((before - from) * scale);
#pragma unroll
        for (int k = 0; k < kFarHold; ++k)
#pragma unroll
            for (int c = 0; c < kVec; ++c) l += fast_exp2((E::get(x[k], c) - from) * scale);
    }
    const float wave_top = all_max(m);
    if (lane == 0) s_max[wave] = wave_top;
    __syncthreads();
    float top = s_max[0];
#pragma unroll
    for (int w = 1; w < kLpWaves; ++w) top = fmaxf(top, s_max[w]);
    const float from = top == kNegInf ? 0.f : top;          // (every logit is -inf: l is 0, and so is the gradient)
    l = all_sum(l * fast_exp2((m - from) * scale));
    if (lane == 0) s_sum[wave] = l;
    __syncthreads();                                        // (everything has been read)
    l = s_sum[0];
#pragma unroll
    for (int w = 1; w < kLpWaves; ++w) l += s_sum[w];
    const float ln_l = logf(l);
    auto grad = [&](float v, int index) __attribute__((always_inline)) {
        return l == 0.f ? 0.f : logit_grad((v - from) * inv_tau - ln_l, g_lp, g_h, c0, index == token);
    };
    for (int i0 = tid * kVec; i0 < V; i0 += kFarHold * kStep) {
        load(i0);
#pragma unroll
        for (int k = 0; k < kFarHold; ++k) {
            const int i = i0 + k * kStep;
            if (i + kVec <= V) {
                float g[kVec];
#pragma unroll
                for (int c = 0; c < kVec; ++c) g[c] = grad(E::get(x[k], c), i + c);
                E::store(out + i, g);
            }
        }
    }
    if (rest < V) E::store_one(out + rest, grad(x_rest, rest));
}

// Every thread writes exactly the elements that it has read, so the gradient may take the logits' place.
template <int DTYPE, int kChunk>
__global__ __launch_bounds__(kLpThreads) void logprob_grad(LogprobGradArgs a) {
    using E = Elem<DTYPE>;
    constexpr int kVec = E::kVec, kIter = kChunk / (kLpThreads * kVec);
    const int r = blockIdx.x / a.n_chunks, chunk = blockIdx.x - r * a.n_chunks, tid = threadIdx.x;
    const int begin = chunk * kChunk, end = min(a.V, begin + kChunk);
    const typename E::T* base = static_cast<const typename E::T*>(a.logits) + r * a.ld;
    typename E::T* out = static_cast<typename E::T*>(a.grad) + r * a.grad_ld;
    typename E::Vec x[kIter];
#pragma unroll
    for (int it = 0; it < kIter; ++it) {
        const int i = begin + (it * kLpThreads + tid) * kVec;
        x[it] = i + kVec <= end ? E::load(base + i) : E::none();
    }
    const int rest = begin + (end - begin) / kVec * kVec + tid;
    const float x_rest = rest < end ? E::one(base + rest) : kNegInf;
    const int token = a.tokens[r];
    const float lse = a.logsumexp[r];
    const bool none = token < 0 || token >= a.V;            // no token: no gradient
    const float g_lp = a.grad_logprob ? a.grad_logprob[r] * a.inv_tau : 0.f;
    const float g_h = a.grad_entropy ? a.grad_entropy[r] * a.inv_tau : 0.f;
    const float h = a.grad_entropy ? a.entropy[r] : 0.f;
    const float c0 = -g_lp - g_h * h;
    if (__builtin_amdgcn_readfirstlane(!none && fabsf(lse) >= kLpFar)) {
        if (chunk == 0) far_row_grad<DTYPE>(base, out, a.V, token, a.inv_tau, g_lp, g_h, c0);
        return;
    }
    auto grad = [&](float v, int index) __attribute__((always_inline)) {
        return none ? 0.f : logit_grad(fmaf(v, a.inv_tau, -lse), g_lp, g_h, c0, index == token);
    };
#pragma unroll
    for (int it = 0; it < kIter; ++it) {
        const int i = begin + (it * kLpThreads + tid) * kVec;
        if (i + kVec <= end) {
            float g[kVec];
#pragma unroll
            for (int c = 0; c < kVec; ++c) g[c] = grad(E::get(x[it], c), i + c);
            E::store(out + i, g);
        }
    }
    if (rest < end) E::store_one(out + rest, grad(x_rest, rest));
}

// Elements of a workgroup's chunk, at most.
constexpr int kLpChunkLarge = 16384, kLpChunkSmall = 4096;
inline int lp_chunk(const seer_logprob_params& p) {
    const int64_t rows = static_cast<int64_t>(p.B) * p.T;
    return rows * ((p.V + kLpChunkLarge - 1) / kLpChunkLarge) >= 2048 ? kLpChunkLarge : kLpChunkSmall;
}
inline int lp_num_chunks(const seer_logprob_params& p) { return (p.V + lp_chunk(p) - 1) / lp_chunk(p); }
// With alternatives to find, which cost a workgroup much the same whatever its length, chunks of one length (in pieces of 512), else whole ones and a short last
// one, whose loads are all full: 1023 rows of 50 257 bf16 with one alternative 30.0 | 34.2 us, 576 rows of 152 064 fp32 with five 32.2 | 32.5; 4096 rows of
// 151 936 bf16 without 186 | 181.
inline int lp_chunk_length(const seer_logprob_params& p) {
    const int n = lp_num_chunks(p);
    return p.top_n > 0 ? ((p.V + n - 1) / n + 511) / 512 * 512 : lp_chunk(p);
}
inline size_t lp_sums_bytes(const seer_logprob_params& p) {
    return (static_cast<size_t>(p.B) * p.T * lp_num_chunks(p) * 3 * sizeof(float) + 255) / 256 * 256;
}

static int check_logprob_params(const seer_logprob_params* p) {
    if (!p) return SEER_EINVAL;
    if (p->B < 0 || p->V < 1) return SEER_EINVAL;
    if (!(p->temperature > 0.f) || p->temperature > 3.0e38f) return SEER_EINVAL;
    if (p->T < 1 || p->top_n < 0 || p->top_n > SEER_MAX_ALTERNATIVES || p->top_n > p->V || p->ld < p->V) return SEER_ESHAPE;
    if (p->dtype != SEER_F32 && p->dtype != SEER_BF16) return SEER_EUNSUPPORTED;
    if (p->V > SEER_LOGPROB_MAX_V) return SEER_EUNSUPPORTED;
    // a launch counts its threads in 32 bits
    const int64_t rows = static_cast<int64_t>(p->B) * p->T, most = 0xffffffffLL / kLpThreads;
    if (rows > most || (p->B > 0 && rows * lp_num_chunks(*p) > most)) return SEER_ESHAPE;
    if (!(1.0f / p->temperature < 2.0e38f)) return SEER_EINVAL;          // (its reciprocal has to be finite too, also times log2 e)
    return SEER_OK;
}

static bool lp_misaligned(const void* ptr, uintptr_t a) { return reinterpret_cast<uintptr_t>(ptr) % a != 0; }

}  // namespace seer

extern "C" size_t seer_token_logprobs_workspace(const seer_logprob_params* p) {
    if (seer::check_logprob_params(p) != SEER_OK || p->B == 0) return 0;
    const size_t keys = static_cast<size_t>(p->B) * p->T * seer::lp_num_chunks(*p) * p->top_n * sizeof(uint64_t);
    return seer::lp_sums_bytes(*p) + (keys + 255) / 256 * 256;
}

extern "C" int seer_token_logprobs(const void* logits, const int32_t* tokens, const int32_t* accepted_path, const seer_logprob_params* p,
                                   float* logprob, float* entropy, float* logsumexp, float* top_logprob, int32_t* top_token,
                                   void* workspace, size_t workspace_bytes, void* hip_stream) {
    const int rc = seer::check_logprob_params(p);
    if (rc != SEER_OK) return rc;
    if (p->B == 0) return SEER_OK;
    if (!logits || !tokens || !logprob || (p->top_n > 0 && (!top_logprob || !top_token))) return SEER_EINVAL;
    if (!workspace || workspace_bytes < seer_token_logprobs_workspace(p)) return SEER_EWORKSPACE;
    const bool f32 = p->dtype == SEER_F32;
    if (seer::lp_misaligned(logits, f32 ? 4 : 2) || seer::lp_misaligned(workspace, 16) || seer::lp_misaligned(tokens, 4) || seer::lp_misaligned(accepted_path, 4) ||
        seer::lp_misaligned(logprob, 4) || seer::lp_misaligned(entropy, 4) || seer::lp_misaligned(logsumexp, 4) || seer::lp_misaligned(top_logprob, 4) ||
        seer::lp_misaligned(top_token, 4))
        return SEER_EALIGN;
    seer::LogprobArgs a{};
    a.logits = logits, a.tokens = tokens, a.path = accepted_path;
    a.ld = p->ld, a.T = p->T, a.V = p->V, a.n_chunks = seer::lp_num_chunks(*p), a.chunk = seer::lp_chunk_length(*p), a.top_n = p->top_n;
    a.inv_tau = 1.0f / p->temperature;
    a.part = static_cast<float*>(workspace);
    a.part_top = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + seer::lp_sums_bytes(*p));
    a.logprob = logprob, a.entropy = entropy, a.logsumexp = logsumexp, a.top_logprob = top_logprob, a.top_token = top_token;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const unsigned rows = static_cast<unsigned>(p->B) * static_cast<unsigned>(p->T);
    const dim3 grid(rows * static_cast<unsigned>(a.n_chunks)), block(seer::kLpThreads);
    const int chunk = seer::lp_chunk(*p);
    const bool top = p->top_n > 0;
#define SEER_LP_SCAN(DTYPE, CHUNK, TOP) \
    if (p->dtype == DTYPE && chunk == CHUNK && top == TOP) hipLaunchKernelGGL((seer::logprob_scan<DTYPE, CHUNK, TOP>), grid, block, 0, stream, a);
    SEER_LP_SCAN(SEER_F32, seer::kLpChunkLarge, true)
    SEER_LP_SCAN(SEER_F32, seer::kLpChunkLarge, false)
    SEER_LP_SCAN(SEER_F32, seer::kLpChunkSmall, true)
    SEER_LP_SCAN(SEER_F32, seer::kLpChunkSmall, false)
    SEER_LP_SCAN(SEER_BF16, seer::kLpChunkLarge, true)
    SEER_LP_SCAN(SEER_BF16, seer::kLpChunkLarge, false)
    SEER_LP_SCAN(SEER_BF16, seer::kLpChunkSmall, true)
    SEER_LP_SCAN(SEER_BF16, seer::kLpChunkSmall, false)
#undef SEER_LP_SCAN
    hipError_t err = hipGetLastError();
    if (err != hipSuccess) return static_cast<int>(err);
    const unsigned lds = top ? static_cast<unsigned>(a.n_chunks) : 0u;
    if (f32) hipLaunchKernelGGL((seer::logprob_join<SEER_F32>), dim3(rows), dim3(seer::kWave), lds, stream, a);
    else hipLaunchKernelGGL((seer::logprob_join<SEER_BF16>), dim3(rows), dim3(seer::kWave), lds, stream, a);
    err = hipGetLastError();
    return err == hipSuccess ? SEER_OK : static_cast<int>(err);
}

extern "C" int seer_token_logprobs_grad(void* grad_logits, int64_t grad_ld, const void* logits, const int32_t* tokens, const float* logsumexp,
                                        const float* entropy, const float* grad_logprob, const float* grad_entropy,
                                        const seer_logprob_params* p, void* hip_stream) {
    const int rc = seer::check_logprob_params(p);
    if (rc != SEER_OK) return rc;
    if (grad_ld < p->V) return SEER_ESHAPE;
    if (p->B == 0) return SEER_OK;
    if (!grad_logits || !logits || !tokens || !logsumexp || (grad_entropy && !entropy)) return SEER_EINVAL;
    if (grad_logits == logits && grad_ld != p->ld) return SEER_EINVAL;        // in place: the same rows
    const bool f32 = p->dtype == SEER_F32;
    if (seer::lp_misaligned(logits, f32 ? 4 : 2) || seer::lp_misaligned(grad_logits, f32 ? 4 : 2) || seer::lp_misaligned(tokens, 4) ||
        seer::lp_misaligned(logsumexp, 4) || seer::lp_misaligned(entropy, 4) || seer::lp_misaligned(grad_logprob, 4) || seer::lp_misaligned(grad_entropy, 4))
        return SEER_EALIGN;
    seer::LogprobGradArgs a{};
    a.grad = grad_logits, a.logits = logits, a.tokens = tokens, a.logsumexp = logsumexp, a.entropy = entropy;
    a.grad_logprob = grad_logprob, a.grad_entropy = grad_entropy;
    a.ld = p->ld, a.grad_ld = grad_ld, a.V = p->V, a.n_chunks = seer::lp_num_chunks(*p);
    a.inv_tau = 1.0f / p->temperature;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const dim3 grid(static_cast<unsigned>(p->B) * static_cast<unsigned>(p->T) * static_cast<unsigned>(a.n_chunks)), block(seer::kLpThreads);
    const int chunk = seer::lp_chunk(*p);
#define SEER_LP_GRAD(DTYPE, CHUNK) \
    if (p->dtype == DTYPE && chunk == CHUNK) hipLaunchKernelGGL((seer::logprob_grad<DTYPE, CHUNK>), grid, block, 0, stream, a);
    SEER_LP_GRAD(SEER_F32, seer::kLpChunkLarge)
    SEER_LP_GRAD(SEER_F32, seer::kLpChunkSmall)
    SEER_LP_GRAD(SEER_BF16, seer::kLpChunkLarge)
    SEER_LP_GRAD(SEER_BF16, seer::kLpChunkSmall)
#undef SEER_LP_GRAD
    const hipError_t err = hipGetLastError();
    return err == hipSuccess ? SEER_OK : static_cast<int>(err);
}
