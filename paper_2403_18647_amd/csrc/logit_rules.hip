// Rules on logits ahead of verification: penalties for tokens that a row's context holds, biases, ids that are not
// allowed.  For row j of sequence b and id v, with said = the times v stands in the history behind the prompt and among
// the block's tokens that the row sees, seen = v stands in any of them or in the prompt:
//   z <- seen ? (z > 0 ? z / rep : z rep) : z
//   z <- z - freq said - pres [said > 0] + bias[v], -inf where v is not allowed.
//
// Bound by memory: a logit is read and written once.  A workgroup has a segment of the vocabulary and rows of one
// sequence.  It counts the history's ids of its segment in LDS (whole histories are read by every segment, from L2; integer
// counts, so their order is of no account), then adjusts its rows with the counts and the bias in registers, each thread
// the same ids in every row.  The block's tokens differ by row: an id's word names the block rows that hold it, as a mask
// that is cut with what the row sees.  The first rows' logits are requested behind the history's first ids, ahead of the
// counting, which then costs no time of its own.
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace sdsat {


typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef int i32x4u_t __attribute__((ext_vector_type(4), aligned(4)));

// An id's word: bit 31 in the prompt, bits 24-30 one more than the first block row that holds it, bits 0-23 its count
// behind the prompt.
// U rows are under way at once.
template <int kRuleThreads, int U>
__global__ void __launch_bounds__(kRuleThreads) logit_rules_kernel(LogitRuleArgs a, int segs, int row_groups, int group_rows) {
    constexpr int kRuleSegment = 4 * kRuleThreads;
    constexpr int AHEAD = 1024 / kRuleThreads;   // quads of the history ahead of the rows
    __shared__ __align__(16) uint32_t s_word[kRuleSegment];
    __shared__ unsigned long long s_who[64];   // block rows that hold the token of row i
    const int seg = (int)blockIdx.x % segs, rg = (int)blockIdx.x / segs % row_groups, b = (int)blockIdx.x / segs / row_groups;
    const int tid = threadIdx.x, v0 = seg * kRuleSegment, v = v0 + 4 * tid;
    const int r0 = rg * group_rows, r1 = min(a.q, r0 + group_rows), left = a.V - v;   // rows; ids of this thread
    const bool counted = a.history || a.tokens;

    float rep = 1.f, freq = 0.f, pres = 0.f;
    if (a.penalties) {
        rep = a.penalties[b];
        freq = a.penalties[a.B + b];
        pres = a.penalties[2 * a.B + b];
    }
    const int* hist = a.history + (size_t)b * a.history_ld;
    i32x4u_t h[AHEAD];
    int n = 0, prompt = 0;
    if (a.history) {
        n = a.history_len[b];
        prompt = a.prompt_len ? a.prompt_len[b] : 0;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {   // as far as a row goes: the length is on its way
            const int i = 4 * (tid + k * kRuleThreads);
            if (i + 4 <= a.history_ld) h[k] = *reinterpret_cast<const i32x4u_t*>(hist + i);
        }
    }
    const int token = a.tokens && tid < a.q && tid < 64 ? a.tokens[(size_t)b * a.q + tid] : -1;
    __builtin_amdgcn_sched_barrier(0);
    f32x4u_t z4[U];
    uint32_t al = 0;   // ids allowed: lane 8 u + i holds the wave's word i of row j0 + u
    const int lane = tid & 63;
    auto row = [&](int j) { return ((size_t)b * a.q + j) * a.V + v; };
    auto request = [&](int j0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j0 + u >= r1 || left <= 0) continue;
            const float* src = a.logits + row(j0 + u);
            if (left >= 4) z4[u] = *reinterpret_cast<const f32x4u_t*>(src);
            else z4[u] = f32x4u_t{src[0], left > 1 ? src[1] : 0.f, left > 2 ? src[2] : 0.f, 0.f};
        }
        if (a.allowed) {
            const int word = (v0 + 4 * (tid - lane)) / 32 + lane % 8;
            al = a.allowed[((size_t)b * a.q + min(j0 + lane / 8, r1 - 1)) * a.allowed_ld + min(word, a.allowed_ld - 1)];
        }
    };
    request(r0);
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.bias) {
        const float* p = a.bias + (size_t)b * a.bias_ld + v;
        if (left >= 4) {
            const f32x4u_t t = *reinterpret_cast<const f32x4u_t*>(p);
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[e] = t[e];
        } else {
            for (int e = 0; e < left; ++e) bias[e] = p[e];
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (counted) {
        reinterpret_cast<uint4*>(s_word)[tid] = uint4{0, 0, 0, 0};
        __syncthreads();
        if (a.history) {
            if (n < 0 || n > a.history_ld) {
                if (tid == 0) atomicOr(a.err, 64);
                n = n < 0 ? 0 : a.history_ld;
            }
            auto count = [&](int i, int id) {
                const uint32_t at = (uint32_t)id - (uint32_t)v0;
                if (at < (uint32_t)kRuleSegment && id < a.V) {
                    if (i < prompt) atomicOr(&s_word[at], 0x80000000u);
                    else atomicAdd(&s_word[at], 1u);
                }
            };
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int i = 4 * (tid + k * kRuleThreads);
                if (i + 4 <= a.history_ld) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (i + e < n) count(i + e, h[k][e]);
                } else {   // a row's last ids
                    for (int e = 0; i + e < n; ++e) count(i + e, hist[i + e]);
                }
            }
            for (int i = 4 * (tid + AHEAD * kRuleThreads); i < n; i += 4 * kRuleThreads) {
                if (i + 4 <= n) {
                    const i32x4u_t t = *reinterpret_cast<const i32x4u_t*>(hist + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) count(i + e, t[e]);
                } else {
                    for (int e = 0; i + e < n; ++e) count(i + e, hist[i + e]);
                }
            }
        }
        if (a.tokens && tid < 64) {
            unsigned long long who = 0;
            for (int j = 0; j < a.q; ++j) who |= (unsigned long long)(__shfl(token, j, 64) == token) << j;
            const uint32_t at = (uint32_t)token - (uint32_t)v0;
            s_who[tid] = who;
            if (token >= 0 && at < (uint32_t)kRuleSegment && token < a.V && __ffsll((long long)who) - 1 == tid)
                atomicAdd(&s_word[at], (uint32_t)(tid + 1) << 24);
        }
        __syncthreads();
    }
    uint4 w4{0, 0, 0, 0};
    if (counted) w4 = reinterpret_cast<const uint4*>(s_word)[tid];
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
    const bool any = (w4.x | w4.y | w4.z | w4.w) != 0;
    for (int j0 = r0; j0 < r1; j0 += U) {
        if (j0 > r0) request(j0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u;
            const uint32_t allowed = a.allowed ? (uint32_t)__shfl((int)al, 8 * u + lane / 8, 64) >> (v % 32) : 15u;
            if (j >= r1 || left <= 0) continue;
            float z[4] = {z4[u][0], z4[u][1], z4[u][2], z4[u][3]};
            if (any) {
                const unsigned long long sees =
                    a.mask ? a.mask[(size_t)b * a.q + j] : j >= 63 ? ~0ull : (2ull << j) - 1;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (!w[e]) continue;
                    int said = w[e] & 0xFFFFFF;
                    const uint32_t at = (w[e] >> 24) & 127u;
                    if (at) said += __popcll(s_who[at - 1] & sees);
                    if (said || w[e] >> 31) z[e] = z[e] > 0.f ? z[e] / rep : z[e] * rep;
                    if (said) z[e] = z[e] - freq * (float)said - pres;
                }
            }
            if (a.bias) {
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] += bias[e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!((allowed >> e) & 1u)) z[e] = -INFINITY;
            float* dst = a.out + row(j);
            if (left >= 4) {
                *reinterpret_cast<f32x4u_t*>(dst) = f32x4u_t{z[0], z[1], z[2], z[3]};
            } else {
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (e < left) dst[e] = z[e];
            }
        }
    }
}

hipError_t launch_logit_rules(const LogitRuleArgs& a, hipStream_t s) {
    if (!a.logits || !a.out || a.B < 1 || a.q < 1 || a.V < 1 || (a.tokens && a.q > 64) || (a.history && (!a.history_len || a.history_ld < 0)) ||
        (a.mask && a.q > 64) || a.history_ld >= 1 << 24 || a.bias_ld < 0 || (a.allowed && a.allowed_ld < (a.V + 31) / 32) || !a.err)
        return hipErrorInvalidValue;
    // Large calls: 2048 ids a workgroup, each of which reads the history, and six rows under way; 96 rows of 128256 ids with
    // histories of 4000: 25 us (a copy of the logits takes 20), 26.3 with 1024 ids and two rows.  Small ones are over sooner
    // in more workgroups of less code: 6 rows of 32016 ids 5.7 us, 6.0.
    const bool large = (long)((a.V + 2047) / 2048) * a.B >= 256;
    const int threads = large ? 512 : 256;
    const int segs = (a.V + 4 * threads - 1) / (4 * threads);
    // rows of a sequence in as many groups (of four rows at least) as fill the compute units twice
    const long wgs = (long)segs * a.B;
    const int most = (a.q + 3) / 4;
    const int want = (int)std::min<long>(most, std::max<long>(1, 512 / wgs));
    const int group_rows = (a.q + want - 1) / want, groups = (a.q + group_rows - 1) / group_rows;
    if (wgs * groups > 0x7FFFFFFFl / threads) return hipErrorInvalidValue;
    auto kern = large ? logit_rules_kernel<512, 6> : logit_rules_kernel<256, 2>;
    hipLaunchKernelGGL(kern, dim3((unsigned)(wgs * groups)), dim3((unsigned)threads), 0, s, a, segs, groups, group_rows);
    return hipGetLastError();
}

}  // namespace sdsat
