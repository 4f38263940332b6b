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
// A row is one segment, or several where there are few rows; one workgroup
// streams each.  Its threads keep their own running maximum, sum and weighted
// sum (no exchange while data arrives) and join them at the end.  For the n_top
// largest, the threads' maxima serve: at least n_top ids reach the n_top-th
// largest maximum of 64 groups of threads, so only ids that do are candidates,
// little more than n_top for logits in no order, and only threads whose own
// maximum does have any.  The workgroup reads those threads' ids once more (from
// a cache), gathers the candidates in LDS as 64-bit keys (the logit as an
// order-preserving integer above the complement of the id: all differ, and ties
// need no care), and ranks each by counting the larger ones.  Segments with more
// candidates than LDS holds (many equal values) take their ids one after the
// other.  The segment that arrives last joins the row's results in segment order.
//
// The threshold has the 16 leading bits of a logit, steps of 2^-7 of its size: rows
// whose logits lie close together for their size, or are equal in many ids, have
// more candidates than LDS holds and pay for it (us with 1, 5 and 20 alternatives;
// ordinary rows of N(0, 4) take 47, 49 and 63, every row 42 without any): 2047 rows
// of 32016 ids of 20 + N(0, 0.01) 176, 428, 1421; of 1000 + N(0, 4) 57, 71, 408; all
// equal 174, 401, 1226.
//
// Bound by HBM over many rows: 2047 rows of 32016 ids with one alternative take
// 50 us, 5.2 TB/s (a large copy here reaches 4.9, a read 6.3).  Over few rows the
// way from the last load to the result counts: 96 rows of 128256 ids take 17.7 us
// with 20 alternatives and 12.3 with none, 8 to 10 of which the logits need; 6
// rows of 32016 with 5 take 8.3, an empty launch 4.4.  There a workgroup runs each
// part of its code for the first time, and what is short counts more than what is
// unrolled: picking candidates while the logits stream, with its code in each of
// the loop's tiles, took 22.3 us for the 96 rows and 57 for the 2047.
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace sdsat {

static constexpr int kLpNT = 256, kLpWaves = kLpNT / 64;
static constexpr int kLpVec = 4;                              // vector loads per thread and tile
static constexpr int kLpTile = 64 * 4 * kLpVec;               // ids a wave takes at a time
static constexpr int kLpStep = kLpWaves * kLpTile;            // segments are multiples of it
static constexpr int kLpFew = 384;                            // candidates of a segment that are ranked, at most
static constexpr int kLpGrid = 1024;                          // rows are cut into as many segments together, at most: four
                                                              // workgroups a CU; 96 rows of 128256 take 17.7 us, with 512
                                                              // 17.9, with 2048 20.9
static constexpr int kLpSegments = 64, kLpKeys = 1024;        // segments of a row, and their keys in the join, at most
static_assert(kMaxTop <= 64, "lanes for the thresholds");

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

__device__ __forceinline__ u64 id_key(float f, int id) { return (u64)logit_key(f) << 32 | (uint32_t)~(uint32_t)id; }

template <typename V>
__device__ __forceinline__ void agent_store(V* p, V v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

template <typename V>
__device__ __forceinline__ V agent_load(const V* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ u64 pack2(float lo, float hi) { return (u64)__float_as_uint(hi) << 32 | __float_as_uint(lo); }

// The n largest of cand[0..count), all different, in order to out[0..n): eight lanes count the keys above one
__device__ __forceinline__ void rank_candidates(const u64* cand, int count, int n, u64* out) {
    const int sub = threadIdx.x & 7;
    for (int i0 = 0; i0 < count; i0 += kLpNT / 8) {   // every lane takes part in the sums
        const int i = i0 + (threadIdx.x >> 3);
        const u64 k = cand[min(i, count - 1)];
        int r = 0;
        for (int j0 = 0; j0 < count; j0 += 32) {      // past the end the last is read again
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int j = j0 + 8 * u + sub;
                r += j < count && cand[min(j, count - 1)] > k;
            }
        }
        float f = across_quads((float)r, OpSum());
        f += lane_perm<0x141>(f);
        r = (int)f;
        if (sub == 0 && i < count && r < n) out[r] = k;
    }
}

// A value that at least n of the wave's 64 reach: the n-th largest, to the 16 leading bits of its key.
__device__ __forceinline__ float nth_largest(float v, int n) {
    const uint32_t key = logit_key(v);
    u64 in = ~0ull;   // lanes whose leading bits are those of the n-th largest
    uint32_t got = 0;
#pragma unroll 4
    for (int b = 31; b >= 16; --b) {
        const u64 set = in & __ballot((key >> b) & 1u);
        const int k = __popcll(set);
        if (k >= n) {
            in = set;
            got |= 1u << b;
        } else {
            n -= k;
            in &= ~set;
        }
    }
    return got > 0x007FFFFFu ? key_logit(got) : -INFINITY;   // below the key of -inf: everything
}

// The running sums of a part of a row, with z in units of log 2: the maximum m, the sum of 2^(z - m) without one
// largest term, and the sum of (z - m) 2^(z - m).
struct LpSums { float m, s, w; };

// a and b joined (z = x * scale); of equal maxima, a's term stays the one left out
__device__ __forceinline__ LpSums lp_join(const LpSums& a, const LpSums& b, float scale) {
    const float m = fmaxf(a.m, b.m);
    const bool of_a = a.m >= b.m;
    const float hi_s = of_a ? a.s : b.s, hi_w = of_a ? a.w : b.w, lo_m = of_a ? b.m : a.m;
    const float lo_s = of_a ? b.s : a.s, lo_w = of_a ? b.w : a.w;
    if (lo_m == -INFINITY) return {m, hi_s + lo_s, hi_w};   // no mass (NaN stays)
    const float d = (lo_m - m) * scale, f = __builtin_amdgcn_exp2f(d);
    return {m, hi_s + f * (1.f + lo_s), fmaf(f, fmaf(fmaxf(d, -1000.f), 1.f + lo_s, lo_w), hi_w)};   // 2^-1000 is 0
}

// The wave's sums joined; of equal maxima, the first lane's term stays the one left out.
__device__ __forceinline__ LpSums lp_join_wave(const LpSums& v, float scale) {
    const float m = across_wave(v.m, OpMax());
    const u64 top = __ballot(v.m == m);
    const float one = top && (int)(threadIdx.x & 63) == __builtin_ctzll(top) ? 0.f : 1.f;
    const bool none = v.m == -INFINITY;   // no mass (NaN stays)
    const float d = none ? 0.f : (v.m - m) * scale, f = __builtin_amdgcn_exp2f(d);
    const float s = none ? v.s : f * (one + v.s), w = none ? 0.f : f * fmaf(fmaxf(d, -1000.f), 1.f + v.s, v.w);
    return {m, across_wave(s, OpSum()), across_wave(w, OpSum())};
}

struct LogprobArgs {
    const float* logits; int M, V, segs, seg;   // segments of a row, ids of each (the last takes the rest)
    const int* tokens; float inv_t; int n_top;
    float* lp; float* ent; int* ids; float* top_lp;
    int tiles_log;                              // a segment is at most 2^tiles_log steps
    u64* part; u64* keys;                       // [M][segs][2]: the sums; [M][segs][n_top]: the largest keys
    int* counter;
    int per, per_inv;                           // join: first keys of each segment behind the threshold; ceil(2^16 / per)
    int* err;
};

// SMALL: fewer ids than a tile
template <bool SMALL>
__global__ void __launch_bounds__(kLpNT, 7) token_logprobs_kernel(LogprobArgs a) {
    __shared__ u64 s_cand[kLpKeys];
    __shared__ u64 s_top[kMaxTop], s_key[kLpWaves];   // the largest keys, in order
    __shared__ u64 s_few[kLpFew];
    __shared__ float s_group[kLpWaves][64];
    __shared__ LpSums s_sums[kLpWaves];
    __shared__ uint8_t s_from[kLpNT];
    __shared__ int s_threads, s_left, s_last;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int row = (int)blockIdx.x / a.segs, sg = (int)blockIdx.x % a.segs, lo = sg * a.seg;
    const int n = min(a.seg, a.V - lo), n_top = a.n_top;
    const float* x = a.logits + (size_t)row * a.V + lo;
    if (tid == 0) s_left = s_threads = 0;
    const float scale = a.inv_t * 1.44269504f;

    // The wave's tile at `base`: ids first(base) + 256 i + 4 lane + j.  A tile that ends past the segment begins earlier, and
    // `trim` takes out what belongs to the one before; of a tile behind the last, lane 0's part is read and not used: each
    // tile is four loads, so that a wait for one leaves the next in flight
    auto first = [&](int base) { return SMALL ? base : min(base, n - kLpTile); };
    auto load = [&](float (&v)[kLpVec][4], int base) {
        if constexpr (SMALL) {
#pragma unroll
            for (int i = 0; i < kLpVec; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int id = base + 256 * i + 4 * lane + j;
                    v[i][j] = id < n ? x[id] : -INFINITY;
                }
        } else {
            const float* at = x + first(base) + (base < n ? 4 * lane : 0);
#pragma unroll
            for (int i = 0; i < kLpVec; ++i) {
                const f32x4u_t t = *reinterpret_cast<const f32x4u_t*>(at + 256 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] = t[j];
            }
        }
    };
    auto trim = [&](float (&v)[kLpVec][4], int base) {
        if (SMALL || base + kLpTile <= n) return;
#pragma unroll
        for (int i = 0; i < kLpVec; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (base >= n || first(base) + 256 * i + 4 * lane + j < base) v[i][j] = -INFINITY;
    };
    LpSums r{-INFINITY, 0.f, 0.f};
    float ones = 0.f;                       // terms of 1 at the present maximum (none while it is -inf)
    auto add = [&](const float (&v)[kLpVec][4]) {
        float tm = -INFINITY;
#pragma unroll
        for (int i = 0; i < kLpVec; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) tm = fmaxf(tm, v[i][j]);
        if (tm > r.m) {   // the sums so far relative to the new maximum, their largest terms ordinary ones now
            const float d = fmaxf((r.m - tm) * scale, -1000.f), f = __builtin_amdgcn_exp2f(d);
            r.w = f * fmaf(d, ones + r.s, r.w);
            r.s = f * (ones + r.s);
            r.m = tm;
            ones = 0.f;
        }
        const float at = r.m == -INFINITY ? 0.f : r.m;
        float all = 0.f, some = 0.f, w = 0.f;
#pragma unroll
        for (int i = 0; i < kLpVec; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float t = (v[i][j] - at) * scale, e = __builtin_amdgcn_exp2f(t);
                all += e;
                some += __builtin_amdgcn_fractf(e);   // 0 for the largest terms, which are 1
                w = fmaf(fmaxf(t, -1000.f), e, w);    // -inf adds nothing
            }
        ones += rintf(all - some);
        r.s += some;
        r.w += w;
    };
    int tok = -1;
    float tok_x;
    {
        float v0[kLpVec][4], v1[kLpVec][4];
        int base = wave * kLpTile;
        load(v0, base);
        // the row's token and its logit, asked for now: only the row's last workgroup needs them
        if (a.lp) tok = a.tokens[row];
        tok_x = a.logits[(size_t)row * a.V + (tok >= 0 && tok < a.V ? tok : 0)];
        while (base < n) {
            const int next = base + kLpStep, after = next + kLpStep;
            if constexpr (!SMALL) load(v1, next);
            trim(v0, base);
            add(v0);
            if constexpr (!SMALL) load(v0, after);
            if (!SMALL && next < n) {
                trim(v1, next);
                add(v1);
            }
            base = after;
        }
    }
    if (ones > 1.f) r.s += ones - 1.f;   // one of the largest terms stays out

    // The largest keys of xs[0..len) (ids from id0), one after the other: for more candidates than LDS holds, and for
    // rows with fewer finite logits than n_top.
    auto one_by_one = [&](const float* xs, int len, int id0) {
        u64 last = ~0ull, best = 0;
        for (int k = 0; k < min(n_top, len); ++k) {
            if (k == 0 || best == last) {   // this thread's was taken: its next one
                best = 0;
                for (int id = tid; id < len; id += kLpNT) {
                    const u64 key = id_key(xs[id], id0 + id);
                    if (key < last && key > best) best = key;
                }
            }
            u64 top = best;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                const u64 other = (u64)(uint32_t)__shfl_xor((int)(top >> 32), o, 64) << 32 |
                                  (uint32_t)__shfl_xor((int)(uint32_t)top, o, 64);
                if (other > top) top = other;
            }
            __syncthreads();   // the round before has read s_key
            if (lane == 0) s_key[wave] = top;
            __syncthreads();
            last = s_key[0];
#pragma unroll
            for (int o = 1; o < kLpWaves; ++o) if (s_key[o] > last) last = s_key[o];
            if (tid == 0) s_top[k] = last;
        }
    };

    // the segment's sums and its n_top largest keys (of finite logits, if it is one of several), in order, in s_top
    {
        const LpSums u = lp_join_wave(r, scale);
        if (lane == 0) s_sums[wave] = u;
    }
    if (tid < kMaxTop) s_top[tid] = 0;
    const float mine = r.m;   // the largest of this thread's ids
    if (n_top > 0) {
        s_group[wave][lane] = mine;   // groups across the waves: a short row lies in the first one
    }
    __syncthreads();
    r = s_sums[0];
#pragma unroll
    for (int k = 1; k < kLpWaves; ++k) r = lp_join(r, s_sums[k], scale);
    if (n_top > 0) {
        // the ids that reach the threshold: what the threads that have one read is read again, four ids a thread
        float group = s_group[0][lane];
#pragma unroll
        for (int k = 1; k < kLpWaves; ++k) group = fmaxf(group, s_group[k][lane]);
        const float least = fmaxf(nth_largest(group, n_top), -3.402823466e38f);   // banned ids (-inf) are not taken
        if (mine >= least) s_from[atomicAdd(&s_threads, 1)] = (uint8_t)tid;
        __syncthreads();
        const int items = s_threads << a.tiles_log << 2;   // each four ids
#pragma unroll 1
        for (int i = tid; i < items; i += kLpNT) {
            const int t = s_from[i >> a.tiles_log >> 2], k = (i >> 2) & ((1 << a.tiles_log) - 1);
            const int base = k * kLpStep + (t >> 6) * kLpTile, id = first(base) + 256 * (i & 3) + 4 * (t & 63);
            if (base >= n) continue;
            float v[4];
            if constexpr (SMALL) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = id + j < n ? x[id + j] : -INFINITY;
            } else {
                const f32x4u_t u = *reinterpret_cast<const f32x4u_t*>(x + id);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = id + j >= base ? u[j] : -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v[j] >= least) {
                    const int p = atomicAdd(&s_left, 1);
                    if (p < kLpFew) s_few[p] = id_key(v[j], lo + id + j);
                }
        }
        __syncthreads();
        const int left = s_left;
        if (left <= kLpFew && (left >= n_top || a.segs > 1)) rank_candidates(s_few, left, n_top, s_top);
        else one_by_one(x, n, lo);
        __syncthreads();
    }

    if (a.segs > 1) {
        u64* part = a.part + (size_t)row * a.segs * 2;
        u64* keys = a.keys + (size_t)row * a.segs * n_top;
        // the segment's results, stored device-coherent: the row's last segment may run on another XCD
        if (tid == 0) {
            agent_store(part + 2 * sg, pack2(r.m, r.s));
            agent_store(part + 2 * sg + 1, pack2(r.w, 0.f));
        }
        if (tid < n_top) agent_store(keys + sg * n_top + tid, s_top[tid]);
        __builtin_amdgcn_s_waitcnt(0);   // performed before the count is raised (wave 0 stored everything)
        if (tid == 0) {
            s_last = __hip_atomic_fetch_add(&a.counter[row], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == a.segs - 1;
            if (s_last) agent_store(&a.counter[row], 0);
            s_left = 0;
        }
        __syncthreads();
        if (!s_last) return;
        // join: a segment per lane; of the keys, if they are many, those that reach a threshold from the first keys of each
        // segment.  Everything is asked for at once
        const int n_keys = a.segs * n_top;
        const bool thin = n_keys > 96;
        u64 key[kLpKeys / kLpNT], first = 0;
#pragma unroll
        for (int i = 0; i < kLpKeys / kLpNT; ++i)
            key[i] = tid + i * kLpNT < n_keys ? agent_load(keys + tid + i * kLpNT) : 0;
        if (thin) {
            const int c = (int)((uint32_t)(lane * a.per_inv) >> 16);   // lane / per
            if (c < a.segs) first = agent_load(keys + c * n_top + lane - c * a.per);
        }
        const u64 ms = lane < a.segs ? agent_load(part + 2 * lane) : pack2(-INFINITY, 0.f);
        const u64 ww = lane < a.segs ? agent_load(part + 2 * lane + 1) : 0;
        if (n_top > 0) {
            // an empty place (a segment of fewer ids) is below every logit
            const uint32_t least =
                thin ? logit_key(nth_largest(first ? key_logit((uint32_t)(first >> 32)) : -INFINITY, n_top)) : 0;
#pragma unroll
            for (int i = 0; i < kLpKeys / kLpNT; ++i)
                if (key[i] && (uint32_t)(key[i] >> 32) >= least) s_cand[atomicAdd(&s_left, 1)] = key[i];
            __syncthreads();
            if (s_left >= n_top) rank_candidates(s_cand, s_left, n_top, s_top);
            else one_by_one(a.logits + (size_t)row * a.V, a.V, 0);
        }
        r = lp_join_wave({__uint_as_float((uint32_t)ms), __uint_as_float((uint32_t)(ms >> 32)), __uint_as_float((uint32_t)ww)}, scale);
        if (n_top > 0) __syncthreads();
    }
    // the row's results; without a finite largest logit they are NaN
    const float log_s = log1pf(r.s);
    if (tid == 0) {
        if (a.ent) a.ent[row] = isfinite(r.m) ? log_s - r.w * 0.693147181f / (1.f + r.s) : NAN;
        if (a.lp) {
            float y = 0.f;   // no token in this row
            if (tok >= a.V) {
                atomicOr(a.err, 1);
                y = NAN;
            } else if (tok >= 0) {
                y = isfinite(r.m) ? (tok_x - r.m) * a.inv_t - log_s : NAN;
            }
            a.lp[row] = y;
        }
    }
    if (tid < n_top) {
        const u64 k = s_top[tid];
        a.ids[(size_t)row * n_top + tid] = (int)~(uint32_t)k;
        a.top_lp[(size_t)row * n_top + tid] =
            isfinite(r.m) ? (key_logit((uint32_t)(k >> 32)) - r.m) * a.inv_t - log_s : NAN;
    }
}

// Ids per segment: the fewest steps for which all segments run at a time (or each row is one), within what a join takes.
static int logprob_segment(int M, int V, int n_top) {
    const long steps = (V + kLpStep - 1) / kLpStep;
    const long most = std::min<long>(kLpSegments, n_top > 0 ? kLpKeys / n_top : kLpSegments);
    const long segs = std::max<long>(1, std::min<long>({steps, most, kLpGrid / M}));
    return (int)((steps + segs - 1) / segs * kLpStep);
}

// Rows are cut while kLpGrid segments hold them all.
size_t logprob_part_bytes(int M, int V) { return V > kLpStep ? (size_t)std::min<long>((long)M * kLpSegments, kLpGrid) * (2 + kMaxTop) * 8 : 0; }

hipError_t launch_token_logprobs(const float* logits, int M, int V, const int* tokens, float temperature, int n_top, float* lp,
                                 float* ent, int* ids, float* top_lp, void* part, int* counter, int* err, hipStream_t s) {
    if (M < 1 || V < 1 || V > (1 << 30) || !logprob_temperature_ok(temperature) || n_top < 0 || n_top > kMaxTop || n_top > V || (lp && !tokens) ||
        (n_top && (!ids || !top_lp)))
        return hipErrorInvalidValue;
    const int seg = logprob_segment(M, V, n_top), segs = (int)(((long)V + seg - 1) / seg);
    if (segs > 1 && (!part || !counter)) return hipErrorInvalidValue;
    const int per = n_top > 0 ? std::min(n_top, 64 / segs) : 1;
    int tiles_log = 0;
    while (((long)kLpStep << tiles_log) < std::min(seg, V)) ++tiles_log;
    u64* sums = static_cast<u64*>(part);
    LogprobArgs a{logits, M, V, segs, seg, tokens, 1.0f / temperature, n_top, lp, ent, ids, top_lp, tiles_log,
                  sums, sums + (size_t)2 * M * segs, counter, per, (65536 + per - 1) / per, err};
    hipLaunchKernelGGL(V < kLpTile ? token_logprobs_kernel<true> : token_logprobs_kernel<false>, dim3((unsigned)((size_t)M * segs)), dim3(kLpNT), 0, s, a);
    return hipGetLastError();
}

}  // namespace sdsat
