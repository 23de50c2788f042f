// Rows of new tokens into the paged cache: queries and keys rotated by their positions on the way, keys and values stored in the
// slots that the tokens were given.
//
// Rotation of pair (a, b) at position m with frequency f: (a cos mf - b sin mf, b cos mf + a sin mf), in fp32 from the bf16 inputs, rounded
// once.  The angle is taken in 64 bits and reduced to a fraction of a turn there: at position 10^6 fp32 would leave 0.06 of a radian, fp64
// leaves 10^-10, and what goes to the fp32 sine and cosine is at most half a turn.
//
// What bounds it: HBM.  2 bytes read and 2 written per component, nothing read twice.  A workgroup takes the heads of a few tokens: it makes
// the tokens' sines and cosines once (R / 2 of them a token, in LDS) and then moves 16-byte chunks; a thread of the rotated part takes
// both chunks whose components belong together, so q_out may be q.  16 384 tokens on 64/8 heads of 128: 131 us, 5.1 TB/s; 4096 on 128 heads of 576
// 235 us, 5.2 TB/s (a large copy: 4.9).  576 tokens: 10.9 us, a launch, two loads that wait for one another and a read and write of 41 KB a token.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/seer_verify.h"
#include "seer_device.h"
#include "seer_tile.h"

namespace seer {

constexpr int kAppendThreads = 256;
constexpr int kAppendMaxRotary = 512;                 // components rotated, at most
constexpr int kAppendTokens = 4;                      // tokens of a workgroup, at most
constexpr int kAppendHold = 4;                        // jobs that a thread has in flight
constexpr int kJobsWanted = kAppendThreads * kAppendHold;
constexpr int kManyBlocks = 1024;                     // workgroups that the GPU is full with

struct AppendArgs {
    const uint16_t* q;
    const uint16_t* k;
    const uint16_t* v;
    const int32_t* slot;
    const int32_t* position;
    const float* inv_freq;
    uint16_t* q_out;
    uint16_t* k_pages;
    uint16_t* v_pages;
    int32_t* status;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    int n_tokens, Hq, Hkv, Dqk, Dv, P, num_slots;
    int half, at, interleaved;        // pairs, first rotated component
    int jobs_qk, jobs_v;              // jobs of a head of q or k, and of v
    int jobs;                         // of a token
    int tokens, parts;                // of a workgroup: tokens; workgroups that share their jobs
    uint32_t inv_qk, inv_v;           // 2^32 / jobs_qk, rounded up; 2^32 / jobs_v
};

// x / d for x < 2^16, from 2^32 / d rounded up (d > 1; d = 1: the reciprocal does not fit, see the caller).
__device__ __forceinline__ int quotient(int x, uint32_t inv, int d) { return d == 1 ? x : static_cast<int>(__umulhi(static_cast<uint32_t>(x), inv)); }

struct AppendJob {
    const uint16_t* from;
    uint16_t* to;
    int second;                       // components from the first chunk to the second (0: one chunk)
    int trig;                         // first pair's entry of the table; -1: copied as it is
    bool on;
};

__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendArgs a) {
    __shared__ float2 s_trig[kAppendTokens * kAppendMaxRotary / 2];
    __shared__ int s_page[kAppendTokens], s_inside[kAppendTokens];       // (page -1: the token has no slot)
    const int tid = threadIdx.x;
    const int block = blockIdx.x / a.parts, part = blockIdx.x - block * a.parts;
    const int first = block * a.tokens, count = min(a.tokens, a.n_tokens - first);
    if (tid < count) {
        const int slot = a.slot[first + tid];
        const bool ok = slot >= 0 && slot < a.num_slots;
        s_page[tid] = ok ? slot / a.P : -1, s_inside[tid] = ok ? slot % a.P : 0;
        if (part == 0 && a.status && (slot < -1 || slot >= a.num_slots)) atomicOr(a.status, 1);
    }
    for (int x = tid; x < count * a.half; x += kAppendThreads) {
        const int t = x / a.half, i = x - t * a.half;
        const double turns = static_cast<double>(a.position[first + t]) * static_cast<double>(a.inv_freq[i]) * 0.15915494309189533577;
        float sine, cosine;
        sincospif(2.f * static_cast<float>(turns - rint(turns)), &sine, &cosine);
        s_trig[x] = make_float2(cosine, sine);
    }
    __syncthreads();
    // jobs of the tokens, one token's behind the other's: heads of q, of k, of v
    const int per_token = (a.jobs + a.parts - 1) / a.parts, job0 = part * per_token, mine = min(a.jobs - job0, per_token);
    if (mine <= 0) return;
    const int total = mine * count, q_jobs = a.Hq * a.jobs_qk, k_jobs = a.Hkv * a.jobs_qk, pair_jobs = a.interleaved ? 0 : a.half / 8;
    for (int x0 = tid; x0 < total; x0 += kAppendThreads * kAppendHold) {
        AppendJob job[kAppendHold];
        u32x4 one[kAppendHold], two[kAppendHold];
#pragma unroll
        for (int h = 0; h < kAppendHold; ++h) {
            const int x = x0 + h * kAppendThreads;
            AppendJob& o = job[h];
            o.on = x < total;
            int t = 0, y = o.on ? x : 0;
#pragma unroll
            for (int next = 1; next < kAppendTokens; ++next)
                if (y >= mine) y -= mine, ++t;
            const int page = s_page[t], inside = s_inside[t];
            o.on = o.on && page >= 0;
            y += job0;
            o.second = 0, o.trig = -1;
            const size_t token = static_cast<size_t>(first) + t;
            if (y < q_jobs + k_jobs) {
                const bool is_q = y < q_jobs;
                y -= is_q ? 0 : q_jobs;
                const int head = quotient(y, a.inv_qk, a.jobs_qk);
                int chunk = y - head * a.jobs_qk;
                // (the pairs' jobs come first, then the chunks beside the rotated part)
                if (chunk < pair_jobs) {
                    o.trig = t * a.half + chunk * 8, o.second = a.half;
                    chunk += a.at / 8;
                } else {
                    chunk -= pair_jobs;
                    if (!a.interleaved && chunk >= a.at / 8) chunk += a.half / 4;
                    if (a.interleaved && chunk >= a.at / 8 && chunk < (a.at + 2 * a.half) / 8) o.trig = t * a.half + (chunk - a.at / 8) * 4;
                }
                if (is_q) {
                    o.from = a.q + token * a.q_stride + head * a.Dqk + chunk * 8;
                    o.to = a.q_out + token * a.q_out_stride + head * a.Dqk + chunk * 8;
                } else {
                    o.from = a.k + token * a.k_stride + head * a.Dqk + chunk * 8;
                    o.to = a.k_pages + ((static_cast<size_t>(page) * a.Hkv + head) * a.P + inside) * a.Dqk + chunk * 8;
                }
            } else {
                y -= q_jobs + k_jobs;
                const int head = quotient(y, a.inv_v, a.jobs_v), chunk = y - head * a.jobs_v;
                o.from = a.v + token * a.v_stride + head * a.Dv + chunk * 8;
                o.to = a.v_pages + ((static_cast<size_t>(page) * a.Hkv + head) * a.P + inside) * a.Dv + chunk * 8;
            }
        }
#pragma unroll
        for (int h = 0; h < kAppendHold; ++h)
            if (job[h].on) {
                one[h] = *reinterpret_cast<const u32x4*>(job[h].from);
                if (job[h].second) two[h] = *reinterpret_cast<const u32x4*>(job[h].from + job[h].second);
            }
#pragma unroll
        for (int h = 0; h < kAppendHold; ++h) {
            const AppendJob& o = job[h];
            if (!o.on) continue;
            if (o.trig >= 0) {
                const float2* trig = s_trig + o.trig;
                if (o.second) {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 c0 = trig[2 * w], c1 = trig[2 * w + 1];
                        const float a0 = bf16lo_to_f32(one[h][w]), a1 = bf16hi_to_f32(one[h][w]);
                        const float b0 = bf16lo_to_f32(two[h][w]), b1 = bf16hi_to_f32(two[h][w]);
                        one[h][w] = cvt_pk_bf16(a0 * c0.x - b0 * c0.y, a1 * c1.x - b1 * c1.y);
                        two[h][w] = cvt_pk_bf16(b0 * c0.x + a0 * c0.y, b1 * c1.x + a1 * c1.y);
                    }
                } else {
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float2 c = trig[w];
                        const float a0 = bf16lo_to_f32(one[h][w]), b0 = bf16hi_to_f32(one[h][w]);
                        one[h][w] = cvt_pk_bf16(a0 * c.x - b0 * c.y, b0 * c.x + a0 * c.y);
                    }
                }
            }
            *reinterpret_cast<u32x4*>(o.to) = one[h];
            if (o.second) *reinterpret_cast<u32x4*>(o.to + o.second) = two[h];
        }
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
static int check_append_params(const seer_append_params* p) {
    if (!p) return SEER_EINVAL;
    if (p->n_tokens < 0 || p->Hq < 0 || p->Hkv < 1 || p->page_size < 1 || p->num_pages < 1) return SEER_EINVAL;
    const bool shared = p->kv_shared_latent != 0;
    // (a token's components: what its jobs and strides are counted with)
    if (p->Dqk < 8 || p->Dqk % 8 != 0 || p->Dqk > 4096 || (!shared && (p->Dv < 8 || p->Dv % 8 != 0 || p->Dv > 4096))) return SEER_ESHAPE;
    if (p->Hq > 4096 || p->Hkv > 4096) return SEER_ESHAPE;
    const int64_t chunks = (static_cast<int64_t>(p->Hq + p->Hkv) * p->Dqk + (shared ? 0 : static_cast<int64_t>(p->Hkv) * p->Dv)) / 8;
    if (chunks >= 1 << 16) return SEER_ESHAPE;
    const int R = p->rotary_dim, at = p->rotary_at;
    if (R < 0 || R > kAppendMaxRotary || R % (p->interleaved ? 8 : 16) != 0 || at < 0 || at % 8 != 0 || static_cast<int64_t>(at) + R > p->Dqk) return SEER_ESHAPE;
    if (static_cast<int64_t>(p->num_pages) * p->page_size > 0x7fffffffLL) return SEER_ESHAPE;
    const int64_t q_row = static_cast<int64_t>(p->Hq) * p->Dqk, k_row = static_cast<int64_t>(p->Hkv) * p->Dqk, v_row = shared ? 0 : static_cast<int64_t>(p->Hkv) * p->Dv;
    if (p->q_stride < q_row || p->q_out_stride < q_row || p->k_stride < k_row || (!shared && p->v_stride < v_row)) return SEER_ESHAPE;
    if (p->q_stride % 8 != 0 || p->q_out_stride % 8 != 0 || p->k_stride % 8 != 0 || (!shared && p->v_stride % 8 != 0)) return SEER_EALIGN;
    return SEER_OK;
}

}  // namespace seer

extern "C" int seer_kv_append(const seer_append_params* p, const void* q, const void* k, const void* v, const int32_t* slot, const int32_t* position,
                              const float* inv_freq, void* q_out, void* k_pages, void* v_pages, int32_t* status, void* hip_stream) {
    const int rc = seer::check_append_params(p);
    if (rc != SEER_OK) return rc;
    if (p->n_tokens == 0) return SEER_OK;
    const bool shared = p->kv_shared_latent != 0;
    if (!k || !k_pages || shared != !v || shared != !v_pages || !slot || (p->Hq > 0) != (q != nullptr) || (p->Hq > 0) != (q_out != nullptr)) return SEER_EINVAL;
    if (p->rotary_dim > 0 && (!position || !inv_freq)) return SEER_EINVAL;
    auto misaligned = [](const void* ptr, uintptr_t a) { return reinterpret_cast<uintptr_t>(ptr) % a != 0; };
    if (misaligned(q, 16) || misaligned(k, 16) || misaligned(v, 16) || misaligned(q_out, 16) || misaligned(k_pages, 16) || misaligned(v_pages, 16) ||
        misaligned(slot, 4) || misaligned(position, 4) || misaligned(inv_freq, 4) || misaligned(status, 4))
        return SEER_EALIGN;
    seer::AppendArgs a{};
    a.q = static_cast<const uint16_t*>(q), a.k = static_cast<const uint16_t*>(k), a.v = static_cast<const uint16_t*>(v);
    a.slot = slot, a.position = position, a.inv_freq = inv_freq, a.status = status;
    a.q_out = static_cast<uint16_t*>(q_out), a.k_pages = static_cast<uint16_t*>(k_pages), a.v_pages = static_cast<uint16_t*>(v_pages);
    a.q_stride = p->q_stride, a.k_stride = p->k_stride, a.v_stride = p->v_stride, a.q_out_stride = p->q_out_stride;
    a.n_tokens = p->n_tokens, a.Hq = p->Hq, a.Hkv = p->Hkv, a.Dqk = p->Dqk, a.Dv = shared ? 0 : p->Dv, a.P = p->page_size;
    a.num_slots = p->num_pages * p->page_size;
    a.half = p->rotary_dim / 2, a.at = p->rotary_at, a.interleaved = p->interleaved != 0;
    a.jobs_qk = p->Dqk / 8 - (a.interleaved ? 0 : a.half / 8), a.jobs_v = shared ? 1 : p->Dv / 8;
    a.jobs = (p->Hq + p->Hkv) * a.jobs_qk + (shared ? 0 : p->Hkv * a.jobs_v);
    auto reciprocal = [](int d) { return static_cast<uint32_t>(((uint64_t{1} << 32) + d - 1) / d); };     // (d = 1: not looked at)
    a.inv_qk = reciprocal(a.jobs_qk), a.inv_v = reciprocal(a.jobs_v);
    // Tokens of fewer than 1024 jobs are taken two, of fewer than 512 four at a time where there are enough of them; large ones are shared by several workgroups, as long as a thread has
    // its jobs in flight.  With one | two | four tokens, in us: 16 384 tokens on 8/1 heads of 128 (88 jobs) 33.6 | 24.1 | 18.2 (four taken), on 16/4 of 64 40.6 | 30.7 | 24.5 (four), on
    // 20/4 of 128 (256) 55.6 | 52.6 | 52.5 (four), on 32/8 (448) 85.8 | 83.6 | 83.7 (four; neighbouring pairs, 768: 91.1 | 87.1 | 83.2, two), on 16/16 of 192 (896) 117.9 | 115.0 | 116.1 (two), on
    // 40/8 with half of 128 rotated (704) 104.9 | 102.2 | 103.0 (two), on 64/8 (704) 129.7 | 131.6 | 136.7 (two, the one case here that loses by it); 2048 on 64/8 16.0 | 15.7 | 17.9; calls of a
    // few hundred are alike.
    a.tokens = 1, a.parts = 1;
    while (a.tokens < seer::kAppendTokens && a.tokens * a.jobs < seer::kJobsWanted && p->n_tokens / (2 * a.tokens) >= seer::kManyBlocks) a.tokens *= 2;
    if (a.tokens == 1) a.parts = (a.jobs + 2 * seer::kJobsWanted - 1) / (2 * seer::kJobsWanted);
    const int64_t blocks = (static_cast<int64_t>(p->n_tokens) + a.tokens - 1) / a.tokens * a.parts;
    if (blocks > 0xffffffffLL / seer::kAppendThreads) return SEER_ESHAPE;
    hipLaunchKernelGGL(seer::kv_append_kernel, dim3(static_cast<unsigned>(blocks)), dim3(seer::kAppendThreads), 0, static_cast<hipStream_t>(hip_stream), a);
    const hipError_t err = hipGetLastError();
    return err == hipSuccess ? SEER_OK : static_cast<int>(err);
}
