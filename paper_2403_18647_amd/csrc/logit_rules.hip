// Rules on logits ahead of verification: penalties for tokens that a row's context holds, biases, ids that are not
// allowed.  For row j of sequence b and id v, with said = the times v stands in the history behind the prompt and among
// the block's tokens that the row sees, seen = v stands in any of them or in the prompt:
//   z <- seen ? (z > 0 ? z / rep : z rep) : z
//   z <- z - freq said - pres [said > 0] + bias[v], -inf where v is not allowed.
//
// Bound by memory: a logit is read and written once.  A workgroup has a segment of the vocabulary and rows of one
// sequence.  It counts the history's ids of its segment in LDS (whole histories are read by every segment, from L2; integer
// counts, so their order is of no account), then streams its rows with the counts and the bias in registers, each thread
// the same ids in every row.  The block's tokens differ by row: an id's word names the block rows that hold it, as a mask
// that is cut with what the row sees.
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace sdsat {

static constexpr int kRuleThreads = 256;

typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));
typedef int i32x4u_t __attribute__((ext_vector_type(4), aligned(4)));

// An id's word: bit 31 in the prompt, bits 24-30 one more than the first block row that holds it, bits 0-23 its count
// behind the prompt.
template <int CH>
__global__ void __launch_bounds__(kRuleThreads) logit_rules_kernel(LogitRuleArgs a, int segs, int row_groups, int group_rows) {
    constexpr int SEG = 4 * kRuleThreads * CH;
    __shared__ __align__(16) uint32_t s_word[SEG];
    __shared__ unsigned long long s_who[64];   // block rows that hold the token of row i
    const int seg = (int)blockIdx.x % segs, rg = (int)blockIdx.x / segs % row_groups, b = (int)blockIdx.x / segs / row_groups;
    const int tid = threadIdx.x, v0 = seg * SEG;
    const bool counted = a.history || a.tokens;
    if (counted) {
        for (int i = tid; i < SEG / 4; i += kRuleThreads) reinterpret_cast<uint4*>(s_word)[i] = uint4{0, 0, 0, 0};
        __syncthreads();
        if (a.history) {
            int n = a.history_len[b], prompt = a.prompt_len ? a.prompt_len[b] : 0;
            if (n < 0 || n > a.history_ld) {
                if (tid == 0) atomicOr(a.err, 64);
                n = n < 0 ? 0 : a.history_ld;
            }
            const int* hist = a.history + (size_t)b * a.history_ld;
            auto count = [&](int i, int v) {
                const uint32_t at = (uint32_t)v - (uint32_t)v0;
                if (at < (uint32_t)SEG && v < a.V) {
                    if (i < prompt) atomicOr(&s_word[at], 0x80000000u);
                    else atomicAdd(&s_word[at], 1u);
                }
            };
            int i = 4 * tid;
            for (; i + 4 <= n; i += 4 * kRuleThreads) {
                const i32x4u_t v = *reinterpret_cast<const i32x4u_t*>(hist + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) count(i + e, v[e]);
            }
            for (; i < n; ++i) count(i, hist[i]);   // at most one thread has a rest
        }
        if (a.tokens && tid < 64) {
            const int t = tid < a.q ? a.tokens[(size_t)b * a.q + tid] : -1;
            unsigned long long who = 0;
            for (int j = 0; j < a.q; ++j) who |= (unsigned long long)(__shfl(t, j, 64) == t) << j;
            const uint32_t at = (uint32_t)t - (uint32_t)v0;
            s_who[tid] = who;
            if (t >= 0 && at < (uint32_t)SEG && t < a.V && __ffsll((long long)who) - 1 == tid)
                atomicAdd(&s_word[at], (uint32_t)(tid + 1) << 24);
        }
        __syncthreads();
    }
    float rep = 1.f, freq = 0.f, pres = 0.f;
    if (a.penalties) {
        rep = a.penalties[b];
        freq = a.penalties[a.B + b];
        pres = a.penalties[2 * a.B + b];
    }
    const int r0 = rg * group_rows, r1 = min(a.q, r0 + group_rows);
#pragma unroll
    for (int ch = 0; ch < CH; ++ch) {
        const int v = v0 + 4 * (ch * kRuleThreads + tid);
        const int left = a.V - v;   // ids of this thread
        if (left <= 0) break;
        uint4 w4{0, 0, 0, 0};
        if (counted) w4 = reinterpret_cast<const uint4*>(s_word)[ch * kRuleThreads + tid];
        const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
        const bool any = (w4.x | w4.y | w4.z | w4.w) != 0;
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
        auto adjust = [&](int j, float (&z)[4], uint32_t allowed) {
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
        };
        auto bits = [&](int j) -> uint32_t {
            return a.allowed ? a.allowed[((size_t)b * a.q + j) * a.allowed_ld + v / 32] >> (v % 32) : 15u;
        };
        if (left >= 4) {
            int j = r0;
            for (; j + 4 <= r1; j += 4) {
                float z[4][4];
                uint32_t al[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const f32x4u_t t = *reinterpret_cast<const f32x4u_t*>(a.logits + ((size_t)b * a.q + j + u) * a.V + v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[u][e] = t[e];
                    al[u] = bits(j + u);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    adjust(j + u, z[u], al[u]);
                    *reinterpret_cast<f32x4u_t*>(a.out + ((size_t)b * a.q + j + u) * a.V + v) =
                        f32x4u_t{z[u][0], z[u][1], z[u][2], z[u][3]};
                }
            }
            for (; j < r1; ++j) {
                const f32x4u_t t = *reinterpret_cast<const f32x4u_t*>(a.logits + ((size_t)b * a.q + j) * a.V + v);
                float z[4] = {t[0], t[1], t[2], t[3]};
                adjust(j, z, bits(j));
                *reinterpret_cast<f32x4u_t*>(a.out + ((size_t)b * a.q + j) * a.V + v) = f32x4u_t{z[0], z[1], z[2], z[3]};
            }
        } else {
            for (int j = r0; j < r1; ++j) {
                const float* src = a.logits + ((size_t)b * a.q + j) * a.V + v;
                float z[4] = {src[0], left > 1 ? src[1] : 0.f, left > 2 ? src[2] : 0.f, 0.f};
                adjust(j, z, bits(j));
                float* dst = a.out + ((size_t)b * a.q + j) * a.V + v;
                for (int e = 0; e < left; ++e) dst[e] = z[e];
            }
        }
    }
}

hipError_t launch_logit_rules(const LogitRuleArgs& a, hipStream_t s) {
    if (!a.logits || !a.out || a.B < 1 || a.q < 1 || a.V < 1 || (a.tokens && a.q > 64) || (a.history && (!a.history_len || a.history_ld < 0)) ||
        (a.mask && a.q > 64) || a.history_ld >= 1 << 24 || a.bias_ld < 0 || (a.allowed && a.allowed_ld < (a.V + 31) / 32) || !a.err)
        return hipErrorInvalidValue;
    const int segs = (a.V + 4 * kRuleThreads - 1) / (4 * kRuleThreads);
    // rows of a sequence in as many groups (of four rows at least) as fill the compute units twice
    const long wgs = (long)segs * a.B;
    const int most = (a.q + 3) / 4;
    const int want = (int)std::min<long>(most, std::max<long>(1, 512 / wgs));
    const int group_rows = (a.q + want - 1) / want, groups = (a.q + group_rows - 1) / group_rows;
    if (wgs * groups > 0x7FFFFFFFl / kRuleThreads) return hipErrorInvalidValue;
    hipLaunchKernelGGL(logit_rules_kernel<1>, dim3((unsigned)(wgs * groups)), dim3(kRuleThreads), 0, s, a, segs, groups, group_rows);
    return hipGetLastError();
}

}  // namespace sdsat
