// Log probabilities of given tokens under logits rows, each row's entropy and
// its most probable alternatives.
//
// With z = x / T over the V ids of a row and M = max z:
//   log p_t = (z_t - M) - log S,   S = sum_i e^(z_i - M)
//   H       = log S + sum_i (M - z_i) e^(z_i - M) / S
// and the n_top ids of the largest logits (ties to the lower id) with their
// log p.  S is held without its largest term (which is 1) and log S formed by
// log1p, so that rows with nearly all mass on one id keep their small
// differences; both terms of H are sums of positive numbers.  All sums are
// float32 in a fixed order.
//
// A row is cut into chunks of 8192 ids, one workgroup each, which are read once
// into registers (8 vector loads per thread in flight): the maximum, then the
// sums, then the chunk's n_top largest.  For these, ids are held as 64-bit keys
// (the logit as an order-preserving integer above the complement of the id), so
// that every key differs and ties need no care.  64 groups of threads know
// their largest keys; the n_top-th largest of those is at most the n_top-th
// largest of the chunk, so only keys from it on are candidates (about 1.3
// n_top for logits in no order); they are gathered in LDS and each is ranked
// by counting the larger ones.  The chunk that arrives last joins the row's
// results in chunk order.
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace sdsat {

static constexpr int kLpNT = 256;
static constexpr int kLpVec = 8;                              // vector loads per thread
static constexpr int kLpChunk = kLpNT * 4 * kLpVec;           // ids per workgroup
static constexpr int kLpGroups = 64;
static constexpr int kLpMost = (kMaxTop - 1) * (kLpChunk / kLpGroups) + 1;   // candidates, at most
static_assert(kMaxTop <= kLpGroups && kLpMost <= kMaxTopKeys, "one threshold key per group; candidates fit LDS");

typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));   // logits rows are float-aligned
typedef unsigned long long u64;

// Order-preserving integer of a logit: -0 as +0, NaN below everything.
__device__ __forceinline__ uint32_t logit_key(float f) {
    uint32_t u = __float_as_uint(f);
    if (f != f) return 1u;
    if (u == 0x80000000u) u = 0u;
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float key_logit(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

__device__ __forceinline__ u64 max64(u64 a, u64 b) { return a > b ? a : b; }

__device__ __forceinline__ u64 shfl_xor64(u64 v, int o) {
    return (u64)__shfl_xor((int)(v >> 32), o, 64) << 32 | (uint32_t)__shfl_xor((int)(uint32_t)v, o, 64);
}

template <typename V>
__device__ __forceinline__ void agent_store(V* p, V v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <typename V>
__device__ __forceinline__ V agent_load(const V* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The n largest of cand[0..count), in order, to out (agent-scope where another workgroup reads it)
template <typename F>
__device__ __forceinline__ void rank_candidates(const u64* cand, int count, int n, F out) {
    for (int i = threadIdx.x; i < count; i += kLpNT) {
        const u64 k = cand[i];
        int r = 0;
        for (int j = 0; j < count; ++j) r += cand[j] > k;
        if (r < n) out(r, k);
    }
}

struct LogprobArgs {
    const float* logits; int M, V, chunks;
    const int* tokens; float inv_t; int n_top;
    float* lp; float* ent; int* ids; float* top_lp;
    // [M][chunks]: the chunk's largest key, S without it and the weighted sum, then n_top keys
    u64* part; int* counter;
    int* err;
};

__global__ void __launch_bounds__(kLpNT) token_logprobs_kernel(LogprobArgs a) {
    __shared__ u64 s_cand[kMaxTopKeys];
    __shared__ u64 s_group[kLpGroups];
    __shared__ u64 s_key[kLpNT / 64];
    __shared__ float s_s[kLpNT / 64], s_w[kLpNT / 64];
    __shared__ int s_count, s_last;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int row = (int)blockIdx.x / a.chunks, ch = (int)blockIdx.x % a.chunks, lo = ch * kLpChunk;
    const int n = min(kLpChunk, a.V - lo);
    const float* x = a.logits + (size_t)row * a.V + lo;

    float v[kLpVec][4];
#pragma unroll
    for (int i = 0; i < kLpVec; ++i) {
        const int id = (i * kLpNT + tid) * 4;
        if (id + 4 <= n) {
            const f32x4u_t t = *reinterpret_cast<const f32x4u_t*>(x + id);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = t[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[i][j] = id + j < n ? x[id + j] : -INFINITY;
        }
    }
    if (tid == 0) s_count = 0;
    // this thread's largest key; ids past the row have none
    auto key = [&](int i, int j) -> u64 {
        const int id = (i * kLpNT + tid) * 4 + j;
        return id < n ? (u64)logit_key(v[i][j]) << 32 | (uint32_t)~(uint32_t)(lo + id) : 0ull;
    };
    u64 best = 0;
#pragma unroll
    for (int i = 0; i < kLpVec; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) best = max64(best, key(i, j));
    u64 grp = max64(best, shfl_xor64(best, 1));   // groups of 4 threads
    grp = max64(grp, shfl_xor64(grp, 2));
    if ((tid & 3) == 0) s_group[tid >> 2] = grp;
#pragma unroll
    for (int o = 4; o < 64; o <<= 1) grp = max64(grp, shfl_xor64(grp, o));
    if (lane == 0) s_key[wave] = grp;
    __syncthreads();
    u64 top = s_key[0];
#pragma unroll
    for (int w = 1; w < kLpNT / 64; ++w) top = max64(top, s_key[w]);
    const float m = key_logit((uint32_t)(top >> 32));
    const float base = m == -INFINITY || m != m ? 0.f : m;

    // sums without the largest id's term
    float s = 0.f, w = 0.f;
#pragma unroll
    for (int i = 0; i < kLpVec; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float t = (v[i][j] - base) * a.inv_t;
            float e = __builtin_amdgcn_exp2f(t * 1.44269504f);
            if (key(i, j) == top && e == e) e = 0.f;   // NaN stays
            s += e;
            w += e == 0.f ? 0.f : -t * e;              // t may be -inf there
        }
    s = wave_sum(s);
    w = wave_sum(w);
    if (lane == 0) { s_s[wave] = s; s_w[wave] = w; }

    // the chunk's n_top largest keys, in order, at s_group[0..]
    if (a.n_top > 0) {
        u64 mine = s_group[lane];
        int r = 0;
        for (int j = 0; j < kLpGroups; ++j) r += s_group[j] > mine;
        // groups past the row's end have key 0 and are tied at the end; the threshold is then 0 (every id)
        const u64 at = __ballot(r == a.n_top - 1 && mine != 0);
        const int src = at ? __builtin_ctzll(at) : 0;
        const u64 thr = at ? s_group[src] : 1ull;
#pragma unroll
        for (int i = 0; i < kLpVec; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u64 k = key(i, j);
                if (k >= thr) s_cand[atomicAdd(&s_count, 1)] = k;
            }
        __syncthreads();   // candidates complete; every wave has read the group keys
        if (tid < kLpGroups) s_group[tid] = 0;
        __syncthreads();
        rank_candidates(s_cand, s_count, a.n_top, [&](int r, u64 k) { s_group[r] = k; });
    }
    __syncthreads();
    s = s_s[0]; w = s_w[0];
#pragma unroll
    for (int k = 1; k < kLpNT / 64; ++k) { s += s_s[k]; w += s_w[k]; }

    const int stride = 2 + a.n_top;
    u64* part = a.part + (size_t)row * a.chunks * stride;
    if (a.chunks > 1) {
        // the chunk's results, stored device-coherent: the row's last chunk may run on another XCD
        u64* mine = part + (size_t)ch * stride;
        if (tid == 0) {
            agent_store(mine, top);
            agent_store(mine + 1, (u64)__float_as_uint(w) << 32 | __float_as_uint(s));
        }
        if (tid < a.n_top) agent_store(mine + 2 + tid, s_group[tid]);
        __builtin_amdgcn_s_waitcnt(0);   // performed before the count is raised
        __syncthreads();
        if (tid == 0) {
            s_last = __hip_atomic_fetch_add(&a.counter[row], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.chunks - 1;
            if (s_last) agent_store(&a.counter[row], 0);
        }
        __syncthreads();
        if (!s_last) return;
        // join: the largest key, then each chunk's sums relative to it, in chunk order
        for (int c = 0; c < a.chunks; ++c) top = max64(top, agent_load(part + (size_t)c * stride));
        const float mm = key_logit((uint32_t)(top >> 32));
        s = w = 0.f;
        for (int c = 0; c < a.chunks; ++c) {
            const u64 k = agent_load(part + (size_t)c * stride), sw = agent_load(part + (size_t)c * stride + 1);
            const float cs = __uint_as_float((uint32_t)sw), cw = __uint_as_float((uint32_t)(sw >> 32));
            const float cm = key_logit((uint32_t)(k >> 32));
            if (k == top) {
                s += cs;
                w += cw;
            } else if (cm == -INFINITY || cm != cm) {   // a chunk of banned ids has no mass (NaN stays)
                s += cs;
            } else {
                const float d = (cm - mm) * a.inv_t, f = __builtin_amdgcn_exp2f(d * 1.44269504f);
                s += f * (1.f + cs);
                w += f == 0.f ? f * cs : f * (cw - d * (1.f + cs));   // d may be -inf there
            }
        }
        if (a.n_top > 0) {
            // each chunk's keys are in order: a candidate's rank is its place there plus the larger keys of the others
            for (int i = tid; i < a.chunks * a.n_top; i += kLpNT)
                s_cand[i] = agent_load(part + (size_t)(i / a.n_top) * stride + 2 + i % a.n_top);
            __syncthreads();
            rank_candidates(s_cand, a.chunks * a.n_top, a.n_top, [&](int r, u64 k) { s_group[r] = k; });
            __syncthreads();
        }
    }
    // the row's results; without a finite largest logit they are NaN
    const float mm = key_logit((uint32_t)(top >> 32));
    const float log_s = log1pf(s);
    if (tid == 0) {
        if (a.ent) a.ent[row] = isfinite(mm) ? log_s + w / (1.f + s) : NAN;
        if (a.lp) {
            const int t = a.tokens[row];
            float r = 0.f;   // no token in this row
            if (t >= a.V) {
                atomicOr(a.err, 1);
                r = NAN;
            } else if (t >= 0) {
                r = isfinite(mm) ? (a.logits[(size_t)row * a.V + t] - mm) * a.inv_t - log_s : NAN;
            }
            a.lp[row] = r;
        }
    }
    if (tid < a.n_top) {
        const u64 k = s_group[tid];
        a.ids[(size_t)row * a.n_top + tid] = (int)~(uint32_t)k;
        a.top_lp[(size_t)row * a.n_top + tid] =
            isfinite(mm) ? (key_logit((uint32_t)(k >> 32)) - mm) * a.inv_t - log_s : NAN;
    }
}

int logprob_chunks(int V) { return (V + kLpChunk - 1) / kLpChunk; }

size_t logprob_part_bytes(int M, int V) {
    const int c = logprob_chunks(V);
    return c > 1 ? (size_t)M * c * (2 + kMaxTop) * 8 : 0;
}

hipError_t launch_token_logprobs(const float* logits, int M, int V, const int* tokens, float temperature, int n_top, float* lp,
                                 float* ent, int* ids, float* top_lp, void* part, int* counter, int* err, hipStream_t s) {
    const int chunks = logprob_chunks(V);
    if (M < 1 || V < 1 || !(temperature > 0.f) || n_top < 0 || n_top > kMaxTop || n_top > V || (lp && !tokens) ||
        (n_top && (!ids || !top_lp)) || (chunks > 1 && (!part || !counter)) || (long)chunks * n_top > kMaxTopKeys)
        return hipErrorInvalidValue;
    LogprobArgs a{logits, M, V, chunks, tokens, 1.0f / temperature, n_top, lp, ent, ids, top_lp, static_cast<u64*>(part), counter,
                  err};
    hipLaunchKernelGGL(token_logprobs_kernel, dim3((unsigned)((size_t)M * chunks)), dim3(kLpNT), 0, s, a);
    return hipGetLastError();
}

}  // namespace sdsat
