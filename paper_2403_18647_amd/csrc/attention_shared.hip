// Block attention of sequences that share a long prefix (samples of one
// prompt, questions behind one instruction).
//
// Sequences come in groups of n.  The group's first `pages` 32-slot pages lie
// in the cache of its first sequence and are the same for all of it; behind
// them each sequence has its own slots.  For sequence b, head h and block row
// r (query at position L_b + r):
//   O_r = softmax(Q_r [K_shared; K_own]^T / sqrt(Dh)) [V_shared; V_own]
// over the shared keys, its own committed keys and the block rows it may see
// (0..r, or the rows set in its ancestor mask).
//
// The softmax is cut into parts, each with its own maximum and sum:
//  * a prefix part: rows of all sequences of a group (n * q rows, RT 16-row
//    tiles per workgroup) against a range of shared pages, which are so read
//    once for the group instead of once per sequence; no mask;
//  * an own part: the q rows of one sequence against a range of its own pages.
// A second kernel joins a row's parts (prefix parts in page order, then own
// parts) by log-sum-exp.  Blocks of more than kAttnSplitRows rows have
// workgroups enough and take both phases in one workgroup per 64 rows (WHOLE),
// which writes the result itself.
//
// Within a workgroup the 4 waves take the range's 32-key blocks round-robin;
// each forms the scores of its block for all row tiles with K straight from the
// cache as matrix-core fragments (S^T = K Q^T; Q in LDS), the softmax in
// registers (rows in lanes, keys in registers and lane groups), and O^T += V^T
// P^T with P as it stands; the next block's K and V are in flight meanwhile.
// On bf16 models Q and P enter the matrix cores as value and remainder, so that
// float accuracy is kept.  Scores are in units of log 2 (the scale is folded
// into Q) and a row's maximum is only raised when a score exceeds it by more
// than kRaise: the weights then stay below 2^kRaise, exact in float, and most
// blocks need no rescaling of O and no exchange between lanes.
//
// Key ranges depend on the prefix lengths, the number of sequences and the cache
// capacity, never on q: a row's result is bitwise the same in blocks of any
// size up to kAttnSplitRows rows.
#include <hip/hip_ext.h>

#include <algorithm>

#include "attention_device.h"

namespace sdsat {

static constexpr int kShareWaves = 4;
static constexpr float kRaise = 8.f;

SharedPlan plan_shared(int B, int group, int H, int q, int dtype, const int* pages, int max_len, int S_max) {
    SharedPlan p{};
    const int G = B / group;
    int most = 0, least = S_max / 32;
    for (int g = 0; g < G; ++g) {
        most = std::max(most, pages[g]);
        least = std::min(least, pages[g]);
    }
    p.whole = q > kAttnSplitRows;
    // 16-row tiles per workgroup: float models keep one (registers); bf16 as many as a group's rows fill, up to 4
    const int rows = p.whole ? q : group * q;
    p.rt = dtype == 0 ? 1 : rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    const int tile = 16 * p.rt;
    if (p.whole) {
        p.grid = B * H * ((q + tile - 1) / tile);
        p.slots = 0;
        return p;
    }
    // pages per prefix part: one for each wave at the least, and parts enough for kSharedParts workgroups
    const int parts = std::min(kSharedMaxParts, std::max(1, (kSharedParts + G * H - 1) / (G * H)));
    p.chunk = std::max(kShareWaves, (most + parts - 1) / parts);
    p.prefix_parts = (most + p.chunk - 1) / p.chunk;
    // pages per own part: the own slots of a full cache in as many parts as fit kSharedParts workgroups
    const int cap = S_max / 32 - least;
    const int own = std::min(kSharedMaxOwn, std::max(1, kSharedParts / (B * H)));
    p.own_chunk = std::max(kShareWaves, (cap + own - 1) / own);
    const int nblk = std::max(1, std::min(cap, (max_len + q + 31) / 32 - least));
    p.own_parts = (nblk + p.own_chunk - 1) / p.own_chunk;
    p.slots = p.prefix_parts + p.own_parts;
    p.tiles = (rows + tile - 1) / tile;
    p.own_tiles = (q + tile - 1) / tile;
    p.prefix_grid = ((G * H * p.prefix_parts + 7) / 8 * 8) * p.tiles;
    p.grid = p.prefix_grid + B * H * p.own_tiles * p.own_parts;
    return p;
}

size_t shared_partial_floats(const SharedPlan& p, int B, int q, int H, int head_dim) {
    return (size_t)B * q * H * p.slots * (head_dim + 4);
}

// The most any call can need: every row of a decode block, both kinds of part at their most.
size_t shared_partial_floats_most(int B_max, int H, int q_max, int head_dim) {
    if (B_max < 2) return 0;   // a group of one takes the plain attention
    const int parts = std::min(kSharedMaxParts, std::max(1, (kSharedParts + H - 1) / H));
    size_t most = 0;
    for (int B = 2; B <= B_max; ++B) {
        const int own = std::min(kSharedMaxOwn, std::max(1, kSharedParts / (B * H)));
        most = std::max(most, (size_t)B * std::min(q_max, kAttnSplitRows) * H * (parts + own) * (head_dim + 4));
    }
    return most;
}

// Four floats at float alignment (the caller's queries).
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));

// f with its elements e of invisible keys zero (a slot no row sees may hold anything)
template <typename T>
__device__ __forceinline__ void drop_keys(Frag<T>& f, int key0, int g, int Tb) {
    auto gone = [&](int e) { return key0 + 16 * (e / 4) + 4 * g + e % 4 >= Tb; };
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
            f.v[w] &= (gone(2 * w) ? 0u : 0x0000FFFFu) | (gone(2 * w + 1) ? 0u : 0xFFFF0000u);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f.lo[e] = gone(e) ? 0.f : f.lo[e];
            f.hi[e] = gone(4 + e) ? 0.f : f.hi[e];
        }
    }
}

// What a block's rows may see: keys below L all, keys below Tb by the causal order or the ancestor masks.
struct Sight { int L, Tb, q; const uint64_t* mask; };

// One 32-key block for up to RT 16-row tiles (nt of them in use).  Row tile t's column c is block row m0 + 16 t + c;
// only blocks with keys from L on look at it.
template <typename T, int NDS, int NDT, int RT>
__device__ __forceinline__ void attend(const Frag<T> (&kf)[2][NDS], Frag<T> (&vf)[NDT], const Frag<T>* qs, int lane, int nt,
                                       int m0, const Sight& see, int blk, float (&rmax)[RT], float (&rsum)[RT],
                                       f32x4_t (&o)[RT][NDT]) {
    constexpr bool two = sizeof(T) == 2;
    const int c = lane & 15, g = lane >> 4;
    const bool whole = 32 * blk + 32 <= see.L;
    if (32 * blk + 32 > see.Tb) {
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) drop_keys<T>(vf[dt], 32 * blk, g, see.Tb);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (t >= nt) break;
        f32x4_t s0 = f32x4_t{0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
        for (int ds = 0; ds < NDS; ++ds) {
            constexpr int P = two ? 2 : 1;
            const Frag<T> qh = lds_frag<T>(qs, (t * P * NDS + ds) * 64 + lane);
            mma(s0, kf[0][ds], qh);
            mma(s1, kf[1][ds], qh);
            if constexpr (two) {
                const Frag<T> ql = lds_frag<T>(qs, (t * P * NDS + NDS + ds) * 64 + lane);
                mma(s0, kf[0][ds], ql);
                mma(s1, kf[1][ds], ql);
            }
        }
        float sv[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) sv[e] = e < 4 ? s0[e] : s1[e - 4];
        if (!whole) {
            const int m = m0 + 16 * t + c;
            const uint64_t mrow = see.mask && m < see.q ? see.mask[m] : 0ull;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int key = 32 * blk + 16 * (e / 4) + 4 * g + e % 4;
                bool v = key < see.Tb && m < see.q;
                if (see.mask) v = v && (key < see.L || ((mrow >> (key - see.L)) & 1ull));
                else v = v && key <= see.L + m;
                if (!v) sv[e] = -INFINITY;
            }
        }
        const float lm = fmaxf(fmaxf(fmaxf(sv[0], sv[1]), fmaxf(sv[2], sv[3])),
                               fmaxf(fmaxf(sv[4], sv[5]), fmaxf(sv[6], sv[7])));
        if (__any(lm > rmax[t] + kRaise)) {
            float bm = fmaxf(lm, __shfl_xor(lm, 16, 64));
            bm = fmaxf(bm, __shfl_xor(bm, 32, 64));
            if (bm > rmax[t] + kRaise) {   // rows whose maximum stays are left as they are
                const float alpha = __builtin_amdgcn_exp2f(rmax[t] - bm);
                rmax[t] = bm;
                rsum[t] *= alpha;
#pragma unroll
                for (int dt = 0; dt < NDT; ++dt) o[t][dt] *= alpha;
            }
        }
        const float base = rmax[t] == -INFINITY ? 0.f : rmax[t];   // a row that has seen no key yet
        float p[8];
        float ps = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(sv[e] - base);
            ps += p[e];
        }
        rsum[t] += ps;
        Frag<T> ph, pl;
        split_frag<T>(p, ph, pl);
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) {
            mma(o[t][dt], vf[dt], ph);
            if constexpr (two) mma(o[t][dt], vf[dt], pl);
        }
    }
}

// Blocks lo + wave, lo + wave + 4, ... below hi of the cache behind kr, vr.  A block past the wave's last is asked for
// past the end of the buffer: no memory is read.
template <typename T, int NDS, int NDT, int RT>
__device__ __forceinline__ void attend_range(__amdgpu_buffer_rsrc_t kr, __amdgpu_buffer_rsrc_t vr, int none, int lo, int hi,
                                             const Frag<T>* qs, int lane, int wave, int nt, int m0, const Sight& see,
                                             float (&rmax)[RT], float (&rsum)[RT], f32x4_t (&o)[RT][NDT]) {
    const int c = lane & 15, g = lane >> 4;
    constexpr bool ahead = sizeof(T) == 2 || NDS == 2;   // float heads of 128: one block's registers are all there are
    Frag<T> kA[2][NDS], vA[NDT];
    if constexpr (ahead) {
        Frag<T> kB[2][NDS], vB[NDT];
        int i = lo + wave;
        load_kv<T, NDS, NDT>(kA, vA, kr, vr, i < hi ? i : none, c, g, 0);
        while (i < hi) {
            const int j = i + kShareWaves, l = j + kShareWaves;
            load_kv<T, NDS, NDT>(kB, vB, kr, vr, j < hi ? j : none, c, g, 0);
            attend<T, NDS, NDT, RT>(kA, vA, qs, lane, nt, m0, see, i, rmax, rsum, o);
            if (j >= hi) break;
            load_kv<T, NDS, NDT>(kA, vA, kr, vr, l < hi ? l : none, c, g, 0);
            attend<T, NDS, NDT, RT>(kB, vB, qs, lane, nt, m0, see, j, rmax, rsum, o);
            i = l;
        }
    } else {
        for (int i = lo + wave; i < hi; i += kShareWaves) {
            load_kv<T, NDS, NDT>(kA, vA, kr, vr, i, c, g, 0);
            attend<T, NDS, NDT, RT>(kA, vA, qs, lane, nt, m0, see, i, rmax, rsum, o);
        }
    }
}

template <typename T, int DH, int RT, bool WHOLE>
__global__ void __launch_bounds__(64 * kShareWaves, RT == 4 ? 1 : 2) shared_attn_kernel(SharedArgs a) {
    constexpr int NDS = DH / 32, NDT = DH / 16, P = sizeof(T) == 2 ? 2 : 1, TILE = 16 * RT;
    constexpr int Q_BYTES = RT * P * NDS * 64 * (int)sizeof(Frag<T>), M_BYTES = kShareWaves * NDT * 64 * 16;
    __shared__ __align__(16) unsigned char smem[Q_BYTES > M_BYTES ? Q_BYTES : M_BYTES];
    __shared__ float s_max[RT][kShareWaves][16], s_sum[RT][kShareWaves][16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int c = lane & 15, g = lane >> 4;
    const AttnArgs& at = a.at;
    const int q = at.q, n = a.group;

    // the workgroup's part: rows row0 .. row0 + rows - 1 of the batch (nt tiles), key blocks of two caches
    int h, grp, b, row0, rows, m0, slot, lo, hi;
    bool prefix;
    if (!WHOLE && (int)blockIdx.x < a.prefix_grid) {
        // the row tiles of a part are neighbours on one XCD (workgroups go to the 8 of them in turn)
        const int x = blockIdx.x & 7, y = blockIdx.x >> 3, tile = y % a.tiles, part = (y / a.tiles) * 8 + x;
        slot = part % a.prefix_parts;
        h = part / a.prefix_parts % at.H;
        grp = part / a.prefix_parts / at.H;
        if (grp * n >= at.B) return;
        lo = slot * a.chunk;
        hi = min(lo + a.chunk, a.pages[grp]);
        if (lo >= hi) return;   // a shorter prefix than the longest group's: the join skips the part too
        b = grp * n;
        m0 = tile * TILE;
        row0 = b * q + m0;
        rows = min(TILE, n * q - m0);
        prefix = true;
    } else {
        int i = WHOLE ? (int)blockIdx.x : (int)blockIdx.x - a.prefix_grid;
        const int part = WHOLE ? 0 : i % a.own_parts;
        if (!WHOLE) i /= a.own_parts;
        const int tiles = (q + TILE - 1) / TILE;
        const int tile = i % tiles;
        i /= tiles;
        h = i % at.H;
        b = i / at.H;
        grp = b / n;
        m0 = tile * TILE;
        row0 = b * q + m0;
        rows = min(TILE, q - m0);
        slot = a.prefix_parts + part;
        lo = a.pages[grp] + part * a.own_chunk;
        hi = !WHOLE && part < a.own_parts - 1 ? lo + a.own_chunk : 0x7FFFFFF;   // the last part runs on to the true end
        prefix = false;
    }
    const int nt = (rows + 15) / 16;

    // the rows' queries, scaled into units of log 2, as fragments in LDS (rows past the last repeat it)
    Frag<T>* s_q = reinterpret_cast<Frag<T>*>(smem);
    for (int i = threadIdx.x; i < RT * NDS * 64; i += 64 * kShareWaves) {
        const int t = i / (NDS * 64), ds = i / 64 % NDS, r = min(16 * t + (i & 15), rows - 1);
        if (t >= nt) break;
        const f32x4u_t* src = reinterpret_cast<const f32x4u_t*>(at.qbuf + ((size_t)(row0 + r) * at.H + h) * DH + 32 * ds +
                                                                8 * ((i >> 4) & 3));
        const f32x4u_t q0 = src[0], q1 = src[1];
        const float x8[8] = {q0.x * at.scale, q0.y * at.scale, q0.z * at.scale, q0.w * at.scale,
                             q1.x * at.scale, q1.y * at.scale, q1.z * at.scale, q1.w * at.scale};
        Frag<T> hi8, lo8;
        split_frag<T>(x8, hi8, lo8);
        s_q[(t * P * NDS + ds) * 64 + (i & 63)] = hi8;
        if constexpr (P == 2) s_q[(t * P * NDS + NDS + ds) * 64 + (i & 63)] = lo8;
    }
    __syncthreads();

    float rmax[RT], rsum[RT];
    f32x4_t o[RT][NDT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        rmax[t] = -INFINITY;
        rsum[t] = 0.f;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) o[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const uint32_t bytes = (uint32_t)at.S_max * DH * sizeof(T);
    const int none = at.S_max / 32;
    if (prefix || WHOLE) {
        const size_t off = ((size_t)grp * n * at.H + h) * at.S_max * DH;
        const Sight all{0x7FFFFFFF, 0x7FFFFFFF, 0, nullptr};
        attend_range<T, NDS, NDT, RT>(buf_rsrc(reinterpret_cast<const T*>(at.kc) + off, bytes),
                                      buf_rsrc(reinterpret_cast<const T*>(at.vc) + off, bytes), none, WHOLE ? 0 : lo,
                                      WHOLE ? a.pages[grp] : hi, s_q, lane, wave, nt, m0, all, rmax, rsum, o);
    }
    if (!prefix) {
        const int L = at.cache_len[b];
        const bool over = L < 0 || L + q > at.S_max;   // the host checks capacity; never read past this sequence's cache
        if (threadIdx.x == 0 && (over || L < 32 * a.pages[grp])) atomicOr(at.err, over ? 4 : 16);
        const int nblk = over ? 0 : (L + min(m0 + TILE, q) + 31) / 32;   // what the tile's last row can see
        const size_t off = ((size_t)b * at.H + h) * at.S_max * DH;
        const Sight see{L, L + q, q, at.mask ? at.mask + (size_t)b * q : nullptr};
        attend_range<T, NDS, NDT, RT>(buf_rsrc(reinterpret_cast<const T*>(at.kc) + off, bytes),
                                      buf_rsrc(reinterpret_cast<const T*>(at.vc) + off, bytes), none, lo, min(hi, nblk),
                                      s_q, lane, wave, nt, m0, see, rmax, rsum, o);
    }

    // the waves' results joined by log-sum-exp in wave order, tile by tile through LDS
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        rsum[t] += __shfl_xor(rsum[t], 16, 64);
        rsum[t] += __shfl_xor(rsum[t], 32, 64);
        if (g == 0) {
            s_max[t][wave][c] = rmax[t];
            s_sum[t][wave][c] = rsum[t];
        }
    }
    f32x4_t* s_o = reinterpret_cast<f32x4_t*>(smem);   // [wave][dt][lane], in place of Q
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        if (t >= nt) break;
        __syncthreads();
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) s_o[(wave * NDT + dt) * 64 + lane] = o[t][dt];
        __syncthreads();
        const int r = 16 * t + c;
        float w[kShareWaves], top = -INFINITY, den = 0.f;
#pragma unroll
        for (int k = 0; k < kShareWaves; ++k) top = fmaxf(top, s_max[t][k][c]);
#pragma unroll
        for (int k = 0; k < kShareWaves; ++k) {
            const float m = s_max[t][k][c];
            w[k] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
            den = fmaf(w[k], s_sum[t][k][c], den);
        }
        if (r >= rows) continue;
#pragma unroll
        for (int i = 0; i < NDT / kShareWaves; ++i) {
            const int dt = wave + kShareWaves * i, d = 16 * dt + 4 * g;
            f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < kShareWaves; ++k) {
                const f32x4_t ov = s_o[(k * NDT + dt) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(ov[e], w[k], acc[e]);
            }
            if constexpr (WHOLE) {
                const float inv = den == 0.f ? 0.f : 1.0f / den;   // a row that sees no key: zeros
                store_out<T>(at, out_off<DH>(at, b, h, m0 + r, d), acc * inv);
            } else {
                float* pr = a.part + (((size_t)(row0 + r) * at.H + h) * a.slots + slot) * (DH + 4);
                *reinterpret_cast<f32x4_t*>(pr + d) = acc;
                if (dt == 0 && g == 0) *reinterpret_cast<float2*>(pr + DH) = float2{top, den};
            }
        }
    }
}

// Joins the parts of each row and head: DH / 4 threads each, four columns per thread.
template <typename T, int DH>
__global__ void __launch_bounds__(256) shared_join_kernel(SharedArgs a) {
    constexpr int D4 = DH / 4;
    const AttnArgs& at = a.at;
    const int e = (int)(blockIdx.x * 256 + threadIdx.x);
    const int rh = e / D4, d = 4 * (e % D4), row = rh / at.H, h = rh % at.H;
    if (row >= at.B * at.q) return;
    const int b = row / at.q, pages = a.pages[b / a.group];
    const int np = (pages + a.chunk - 1) / a.chunk;   // the group's prefix parts
    const float* base = a.part + (size_t)rh * a.slots * (DH + 4);
    float top = -INFINITY;
    for (int i = 0; i < a.slots; ++i)
        if (i < np || i >= a.prefix_parts) top = fmaxf(top, base[(size_t)i * (DH + 4) + DH]);
    float den = 0.f;
    f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < a.slots; ++i) {
        if (i >= np && i < a.prefix_parts) continue;
        const float* pr = base + (size_t)i * (DH + 4);
        const float2 ms = *reinterpret_cast<const float2*>(pr + DH);
        const f32x4_t ov = *reinterpret_cast<const f32x4_t*>(pr + d);
        const float w = ms.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms.x - top);
        den = fmaf(w, ms.y, den);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = fmaf(ov[k], w, acc[k]);
    }
    const float inv = den == 0.f ? 0.f : 1.0f / den;   // a row that sees no key: zeros
    store_out<T>(at, out_off<DH>(at, b, h, row - b * at.q, d), acc * inv);
}

template <typename T, int DH>
static hipError_t launch_shared_dh(const SharedPlan& p, const SharedArgs& a, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
    void (*kern)(SharedArgs);
    if constexpr (sizeof(T) == 2) {
        if (p.whole) kern = shared_attn_kernel<T, DH, 4, true>;   // more than 64 rows: four tiles
        else if (p.rt == 4) kern = shared_attn_kernel<T, DH, 4, false>;
        else if (p.rt == 2) kern = shared_attn_kernel<T, DH, 2, false>;
        else kern = shared_attn_kernel<T, DH, 1, false>;
    } else {
        kern = p.whole ? shared_attn_kernel<T, DH, 1, true> : shared_attn_kernel<T, DH, 1, false>;
    }
    const dim3 block(64 * kShareWaves);
    if (ev0) hipExtLaunchKernelGGL(kern, dim3(p.grid), block, 0, s, ev0, p.whole ? ev1 : nullptr, 0, a);
    else hipLaunchKernelGGL(kern, dim3(p.grid), block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.whole) return e;
    const unsigned grid = (unsigned)(((size_t)a.at.B * a.at.q * a.at.H * (DH / 4) + 255) / 256);
    if (ev1) hipExtLaunchKernelGGL((shared_join_kernel<T, DH>), dim3(grid), dim3(256), 0, s, nullptr, ev1, 0, a);
    else hipLaunchKernelGGL((shared_join_kernel<T, DH>), dim3(grid), dim3(256), 0, s, a);
    return hipGetLastError();
}

hipError_t launch_attention_shared(int dtype, int head_dim, const SharedPlan& p, SharedArgs a, hipStream_t s, hipEvent_t ev0,
                                   hipEvent_t ev1) {
    const AttnArgs& at = a.at;
    if (at.q < 1 || at.q > 4096 || (at.mask && at.q > 64) || at.B < 1 || at.H < 1 || a.group < 1 || at.B % a.group ||
        at.B / a.group > kMaxShareGroups || at.S_max < 32 || at.S_max % 32 || at.ldo % 4 || !at.qbuf || !at.kc || !at.vc ||
        !at.cache_len || !at.out || !at.err || p.whole != (at.q > kAttnSplitRows) || (!p.whole && !a.part) ||
        (dtype == 1 ? p.rt != 4 && (p.whole || (p.rt != 1 && p.rt != 2)) : p.rt != 1))
        return hipErrorInvalidValue;
    for (int g = 0; g < at.B / a.group; ++g)
        if (a.pages[g] < 0 || a.pages[g] > at.S_max / 32 || (!p.whole && a.pages[g] > p.chunk * p.prefix_parts))
            return hipErrorInvalidValue;
    a.chunk = p.chunk; a.prefix_parts = p.prefix_parts; a.own_chunk = p.own_chunk; a.own_parts = p.own_parts;
    a.slots = p.slots; a.tiles = p.tiles; a.prefix_grid = p.prefix_grid;
    if (p.whole) a.chunk = a.prefix_parts = a.own_parts = 1;
    if (dtype == 1) {
        if (head_dim == 128) return launch_shared_dh<uint16_t, 128>(p, a, s, ev0, ev1);
        if (head_dim == 64) return launch_shared_dh<uint16_t, 64>(p, a, s, ev0, ev1);
    } else {
        if (head_dim == 128) return launch_shared_dh<float, 128>(p, a, s, ev0, ev1);
        if (head_dim == 64) return launch_shared_dh<float, 64>(p, a, s, ev0, ev1);
    }
    return hipErrorInvalidValue;
}

}  // namespace sdsat
