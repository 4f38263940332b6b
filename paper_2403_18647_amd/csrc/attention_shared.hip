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
//  * prefix parts: rows of all sequences of a group (n * q rows) against a
//    range of shared pages, which are so read once for the group instead of
//    once per sequence; no mask;
//  * own parts: the q rows of one sequence against a range of its own pages.
// A second kernel joins a row's parts, prefix parts in page order, then own
// parts, by log-sum-exp.  Blocks of more than kAttnSplitRows rows have workgroups
// enough and take both phases in one workgroup per row tile, which writes the
// result.
//
// A part's 32-key blocks go round-robin over key lanes (2 for a prefix, 4 for
// own slots), waves that keep their own maximum, sum and O, joined in lane order
// at the end.  Scores are formed as S^T = K Q^T, the softmax runs in registers
// (rows in lanes, keys in registers and lane groups), and O^T += V^T P^T takes P
// as it stands.  Two kinds of workgroup do this, with the same values:
//  * few rows, and float models: a wave per key lane and 16 rows, K and V
//    straight from the cache into registers; bound by HBM: two groups of 8
//    sequences, one row each over 2011 shared and 300 own slots of 32 heads of 128
//    (119 MB) 31 us, 3.8 TB/s (a read stream 6.3); a second launch, the join, 4.5 of it;
//  * many rows of bf16 models: 64 rows, two key lanes of two waves with 32 rows
//    each; the blocks go straight into LDS while the ones before are used, Q
//    stays in registers; bound by the matrix cores, the softmax beside them and, where
//    rows are few for their keys, by the loads: 16 sequences of 11 rows over 16384
//    shared and 400 own slots of 40 heads of 128 (121 GFLOP with the remainders)
//    150-152 us, 130 without products and softmax and 120 without the loads; 8 blocks
//    of 128 rows over 4000 slots (136 GFLOP) 120 us, 1.1 PFLOP/s (a large product
//    1.19); two workgroups a CU, so 4 such blocks take 90 us.
// Float models take the first kind for every block: 4 blocks of 150 rows over 2000
// slots 35 us with 4 heads of 64, 302 with 32 heads of 128 (20 GFLOP, 68 TFLOP/s).
// On bf16 models Q and P enter the matrix cores as value and remainder, as in
// attention.hip: 16 bits of each, outputs within 3.5e-6 of their size of the
// 64-bit result (float32 arithmetic 0.7e-6 to 2.3e-6); a third term would add
// half as many products again, and the many-row kernel is bound by them.
// Scores are in units of log 2 (the scale is folded into Q).  A row keeps a base,
// and its products are added to minus the base, so that the weights are 2 to what
// comes out.  The base begins at the maximum of the row's first block and is only
// raised, to the maximum at hand, when a score exceeds it by more than kRaise: the
// weights stay below 2^kRaise, far from the end of float's range, and most blocks
// need no rescaling of O and no exchange between lanes.
//
// Key ranges depend on the prefix lengths, the number of sequences and the cache
// capacity, never on q: a row's result is bitwise the same in blocks of any
// size up to kAttnSplitRows rows.
#include <hip/hip_ext.h>

#include <algorithm>

#include "attention_device.h"

namespace sdsat {

static constexpr float kRaise = 8.f;
static constexpr int kPrefixLanes = 2, kOwnLanes = 4;   // key lanes
static constexpr int kTileRows = 64;                    // rows of a workgroup that stages K and V in LDS

// Parts of all groups and heads.  More of them bring more waves where rows are few, fewer of them fewer partial results
// where there are many: of one group over 6000 shared and 100 own slots, 32 heads of 128, us per call with 256, 384 and 512
// parts: 2 sequences of 6 rows 24.6, 22.3, 26.0; 4 of 1 row 25.0, 24.4, 25.8; 12 of 6 rows 41.7, 42.7, 49.9; over 4000
// slots, 16 of 6 rows 36.3, 40.9, 45.1; 32 of 6 rows 57.1, 65.8, 74.5.  The rows of a block have no say (16 of 1 row: 27.2,
// 24.9, 25.4), so large groups are cut for speculative blocks.
static int shared_parts(int group) { return group < kSharedMany ? kSharedParts : kSharedManyParts; }

static constexpr int kOwnPages = 32;   // pages of an own part at the least: 1024 slots
static int prefix_parts_most(int G, int group, int H) { return std::min(kSharedMaxParts, std::max(1, shared_parts(group) / (G * H))); }
static int own_parts_most(int B, int group, int H) { return std::min(kSharedMaxOwn, std::max(1, shared_parts(group) / (B * H))); }

SharedPlan plan_shared(int B, int group, int H, int q, int dtype, const int* pages, int max_len, int S_max) {
    SharedPlan p{};
    const int G = B / group;
    int most = 0, least = S_max / 32;
    for (int g = 0; g < G; ++g) {
        most = std::max(most, pages[g]);
        least = std::min(least, pages[g]);
    }
    p.whole = q > kAttnSplitRows;
    const int rows = p.whole ? q : group * q;
    p.staged = dtype == 1 && rows > kSharedFewRows;
    const int tile = p.staged ? kTileRows : 16;
    p.tiles = (rows + tile - 1) / tile;
    if (p.whole) {
        p.grid = B * H * p.tiles;
        return p;
    }
    // pages per prefix part: four for each lane at the least
    const int parts = prefix_parts_most(G, group, H);
    p.chunk = std::max(4 * kPrefixLanes, (most + parts - 1) / parts);
    p.prefix_parts = (most + p.chunk - 1) / p.chunk;
    // pages per own part: the own slots of a full cache in as many parts as that allows
    const int cap = S_max / 32 - least;
    const int own = own_parts_most(B, group, H);
    p.own_chunk = std::max(kOwnPages, (cap + own - 1) / own);
    const int nblk = std::max(1, std::min(cap, (max_len + q + 31) / 32 - least));
    p.own_parts = (nblk + p.own_chunk - 1) / p.own_chunk;
    p.slots = p.prefix_parts + p.own_parts;
    // workgroups of the prefix: one per part and row tile, of 64 rows or two of 16; then those of the own parts
    const int units = (G * H * p.prefix_parts + 7) / 8 * 8 * p.tiles;
    p.prefix_grid = p.staged ? units : (units + 15) / 16 * 8;
    p.grid = p.prefix_grid + B * H * ((q + 15) / 16) * p.own_parts;
    return p;
}

size_t shared_partial_floats(const SharedPlan& p, int B, int q, int H, int head_dim) {
    return (size_t)B * q * H * p.slots * (head_dim + 4);
}

// The most any call can need: every row of a decode block, for any groups (of two sequences or more: one takes the plain
// attention), both kinds of part at their most for a cache of S_max slots.
size_t shared_partial_floats_most(int B_max, int H, int q_max, int head_dim, int S_max) {
    const int pages = S_max / 32;
    size_t most = 0;
    for (int G = 1; G <= kMaxShareGroups; ++G)
        for (int group = 2; (long)G * group <= B_max; ++group) {
            const int B = G * group, parts = std::min(prefix_parts_most(G, group, H), pages / (4 * kPrefixLanes) + 1),
                      own = std::min(own_parts_most(B, group, H), pages / kOwnPages + 1);
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

// One wave's share of an attention over 32-key blocks: RT 16-row tiles of queries, the scores of the block at hand, and
// the bases, sums and weighted V of each row (row tile t's column c is row 16 t + c).
template <typename T, int DH, int RT>
struct WaveAttention {
    static constexpr int NDT = DH / 16;
    f32x4_t s[RT][2], o[RT][NDT];   // s[t][kt][r] = S^T[key 16 kt + 4 g + r][row 16 t + c] less the row's base
    f32x4_t minus[RT];              // minus the row's base (0 before its first key): what the products are added to
    float rise[RT], rsum[RT];       // scores above it raise the base: kRaise, or -inf before the first key

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            minus[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            rise[t] = -INFINITY;
            rsum[t] = 0.f;
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) o[t][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
    }
    // The scores of block blk as its rows see them, and the bases raised where they have to be.  m0: block row of tile 0.
    __device__ __forceinline__ void look(int blk, int m0, const Sight& see, int lane) {
        const int c = lane & 15, g = lane >> 4;
        if (32 * blk + 32 > see.L) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const int m = m0 + 16 * t + c;
                const uint64_t mrow = see.mask && m < see.q ? see.mask[m] : 0ull;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int key = 32 * blk + 16 * (e / 4) + 4 * g + e % 4;
                    bool v = key < see.Tb && m < see.q;
                    if (see.mask) v = v && (key < see.L || ((mrow >> (key - see.L)) & 1ull));
                    else v = v && key <= see.L + m;
                    if (!v) s[t][e / 4][e % 4] = -INFINITY;
                }
            }
        }
        // the larger of two as the median with infinity (that the compiler cannot see): fmaxf would first quiet each product
        // sum, an instruction more
        float lm[RT], inf = INFINITY;
        asm("" : "+s"(inf));
        bool any = false;
#pragma unroll
        for (int t = 0; t < RT; ++t) {
            auto larger = [&](float a, float b) { return __builtin_amdgcn_fmed3f(a, b, inf); };
            lm[t] = larger(larger(larger(s[t][0][0], s[t][0][1]), larger(s[t][0][2], s[t][0][3])),
                           larger(larger(s[t][1][0], s[t][1][1]), larger(s[t][1][2], s[t][1][3])));
            any |= lm[t] > rise[t];
        }
        if (__any(any)) {
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                const float bm = across_rows(lm[t], OpMax());
                if (bm > rise[t]) {   // rows whose base stays are left as they are
                    const float next = minus[t][0] - bm, up = minus[t][0] - next;   // up: by what the base rises as it is rounded
                    const float alpha = rise[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(-up);
                    minus[t] = f32x4_t{next, next, next, next};
                    rise[t] = kRaise;
                    rsum[t] *= alpha;
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[t][e / 4][e % 4] -= up;
#pragma unroll
                    for (int dt = 0; dt < NDT; ++dt) o[t][dt] *= alpha;
                }
            }
        }
    }
    // The row's base, -inf where it has seen no key.
    __device__ __forceinline__ float top(int t) const { return rise[t] == -INFINITY ? -INFINITY : -minus[t][0]; }
    // The weights of tile t's scores as matrix operands, and their sum.
    __device__ __forceinline__ void weigh(int t, Frag<T>& ph, Frag<T>& pl) {
        float p[8], ps = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            p[e] = __builtin_amdgcn_exp2f(s[t][e / 4][e % 4]);
            ps += p[e];
        }
        rsum[t] += ps;
        split_frag<T>(p, ph, pl);
    }
};

// The cache rows of a head that an attention reads: pages below `pages` from the group's first sequence, the others from
// the sequence itself.
template <typename T>
struct HeadCache {
    const T *k0, *v0, *k1, *v1;
    int pages;
};
template <typename T, int DH>
__device__ __forceinline__ HeadCache<T> head_cache(const AttnArgs& at, int first, int own, int h, int pages) {
    const size_t o0 = ((size_t)first * at.H + h) * at.S_max * DH, o1 = ((size_t)own * at.H + h) * at.S_max * DH;
    const T* kc = reinterpret_cast<const T*>(at.kc);
    const T* vc = reinterpret_cast<const T*>(at.vc);
    return {kc + o0, vc + o0, kc + o1, vc + o1, pages};
}

// Eight query columns scaled into units of log 2, as value and remainder.
template <typename T>
__device__ __forceinline__ void query_frag(const AttnArgs& at, f32x4u_t a, f32x4u_t b, Frag<T>& hi, Frag<T>& lo) {
    const float x[8] = {a.x * at.scale, a.y * at.scale, a.z * at.scale, a.w * at.scale,
                        b.x * at.scale, b.y * at.scale, b.z * at.scale, b.w * at.scale};
    split_frag<T>(x, hi, lo);
}

// ------------------------------------------------------------------ 16 rows, K and V from the cache to registers
// The attention of rows row0 .. row0 + rows - 1 (at most 16) over blocks from lo, a wave per key lane (`wave` of LANES).
// K of the next block is requested as soon as the scores of the present one are formed, V of the next after its products:
// one block's registers, so that three waves share a SIMD and one's loads fill the others' waits.  Loads return in order:
// the sequence's length (len, null for a prefix) and the queries are asked for ahead of the first block, which is
// requested below hi before late(length, hi) says what the rows see and where the blocks end; a block past the wave's
// last is asked for past the end of the buffer, which reads no memory.
template <typename T, int DH, int LANES, typename F>
__device__ __forceinline__ void attend_few(WaveAttention<T, DH, 1>& w, const AttnArgs& at, const HeadCache<T>& hc, int lo, int hi,
                                           int row0, int rows, int h, int m0, int wave, int lane, const int* len, F late) {
    constexpr int NDS = DH / 32, NDT = DH / 16;
    constexpr uint32_t E = sizeof(T);
    const int c = lane & 15, g = lane >> 4, none = at.S_max / 32;
    const uint32_t bytes = (uint32_t)at.S_max * DH * E;
    const __amdgpu_buffer_rsrc_t k0 = buf_rsrc(hc.k0, bytes), v0 = buf_rsrc(hc.v0, bytes), k1 = buf_rsrc(hc.k1, bytes),
                                 v1 = buf_rsrc(hc.v1, bytes);
    int zero = 0;
    asm volatile("" : "+v"(zero));   // a vector load: a scalar one would be placed behind the requests
    const int L = len ? len[zero] : 0;
    f32x4u_t q8[NDS][2];
    {
        const float* q0 = at.qbuf + ((size_t)(row0 + min(c, rows - 1)) * at.H + h) * DH + 8 * g;   // rows past the last repeat it
#pragma unroll
        for (int ds = 0; ds < NDS; ++ds)
#pragma unroll
            for (int u = 0; u < 2; ++u) q8[ds][u] = reinterpret_cast<const f32x4u_t*>(q0 + 32 * ds)[u];
    }
    Frag<T> kf[2][NDS], vf[NDT], qh[NDS], ql[NDS];
    auto get_k = [&](int j) {
        const __amdgpu_buffer_rsrc_t r = j < hc.pages ? k0 : k1;
        const int blk = j < hi ? j : none;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const uint32_t ko = ((uint32_t)(blk * 32 + 16 * kt + c) * DH + 8 * g) * E;
#pragma unroll
            for (int ds = 0; ds < NDS; ++ds) kf[kt][ds] = buf_frag<T>(r, ko, ds * 32 * E);
        }
    };
    auto get_v = [&](int j) {
        const __amdgpu_buffer_rsrc_t r = j < hc.pages ? v0 : v1;
        const uint32_t vo = ((uint32_t)(j < hi ? j : none) * DH * 32 + c * 32 + 8 * g) * E;
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) vf[dt] = buf_frag<T>(r, vo, dt * 16 * 32 * E);
    };
    int i = lo + wave;
    get_k(i);
    get_v(i);
    __builtin_amdgcn_sched_barrier(0);   // the requests stay ahead of the wait for the queries
#pragma unroll
    for (int ds = 0; ds < NDS; ++ds) query_frag<T>(at, q8[ds][0], q8[ds][1], qh[ds], ql[ds]);
    w.clear();
    const Sight see = late(__builtin_amdgcn_readfirstlane(L), hi);
    for (; i < hi; i += LANES) {
        w.s[0][0] = w.s[0][1] = w.minus[0];
#pragma unroll
        for (int ds = 0; ds < NDS; ++ds) {
            // products that follow each other go to different sums: each waits for its sum's last one
            mma(w.s[0][0], kf[0][ds], qh[ds]);
            mma(w.s[0][1], kf[1][ds], qh[ds]);
            if constexpr (E == 2) {
                mma(w.s[0][0], kf[0][ds], ql[ds]);
                mma(w.s[0][1], kf[1][ds], ql[ds]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        get_k(i + LANES);
        w.look(i, m0, see, lane);
        if (32 * i + 32 > see.Tb) {   // keys that no row sees: their V may be anything
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) drop_keys<T>(vf[dt], 32 * i, g, see.Tb);
        }
        Frag<T> ph, pl;
        w.weigh(0, ph, pl);
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) mma(w.o[0][dt], vf[dt], ph);
        if constexpr (E == 2) {
#pragma unroll
            for (int dt = 0; dt < NDT; ++dt) mma(w.o[0][dt], vf[dt], pl);
        }
        __builtin_amdgcn_sched_barrier(0);
        get_v(i + LANES);
    }
}

// The key lanes of a workgroup of 4 waves (4 lanes, or twice 2 of different parts) joined by log-sum-exp in lane order:
// out(row, columns d.., O to the maximum, maximum, sum) for four columns of each row.  smem: FewBytes.
template <int DH> constexpr int FewBytes = DH * 256 + 2 * 4 * 16 * 4;
template <typename T, int DH, int LANES, typename F>
__device__ __forceinline__ void join_few(const WaveAttention<T, DH, 1>& w, unsigned char* smem, int rows, int wave4, int lane, F out) {
    constexpr int NDT = DH / 16;
    const int c = lane & 15, g = lane >> 4, wave = wave4 % LANES;
    f32x4_t* s_o = reinterpret_cast<f32x4_t*>(smem) + (wave4 - wave) * NDT * 64;   // [lane][dt][64]
    float (*s_max)[16] = reinterpret_cast<float (*)[16]>(smem + DH * 256) + wave4 - wave, (*s_sum)[16] = s_max + 4;
    const float sum = across_rows(w.rsum[0], OpSum());
    if (g == 0) {
        s_max[wave][c] = w.top(0);
        s_sum[wave][c] = sum;
    }
#pragma unroll
    for (int dt = 0; dt < NDT; ++dt) s_o[(wave * NDT + dt) * 64 + lane] = w.o[0][dt];
    __syncthreads();
    if (c >= rows) return;
    float wt[LANES], top = -INFINITY, den = 0.f;
#pragma unroll
    for (int k = 0; k < LANES; ++k) top = fmaxf(top, s_max[k][c]);
#pragma unroll
    for (int k = 0; k < LANES; ++k) {
        const float m = s_max[k][c];
        wt[k] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        den = fmaf(wt[k], s_sum[k][c], den);
    }
#pragma unroll
    for (int i = 0; i < NDT / LANES; ++i) {
        const int dt = wave + LANES * i;
        f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < LANES; ++k) {
            const f32x4_t ov = s_o[(k * NDT + dt) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(ov[e], wt[k], acc[e]);
        }
        out(c, 16 * dt + 4 * g, acc, top, den);
    }
}

// ------------------------------------------------------------------ 64 rows, K and V through LDS (bf16)
// The kernels that load into LDS hold one shared array: with several, the compiler takes every read of LDS for one that may
// depend on the loads in flight and waits for them.
template <int DH>
struct TileShape {
    static constexpr int CPR = DH / 8;                        // 16-byte chunks per K row
    static constexpr int HALF = 32 * DH * 2, BLK = 2 * HALF;  // bytes of a block's K (or V), of both
    static constexpr int STAGE = kPrefixLanes * BLK;          // a step's blocks, one per key lane
    static constexpr int BYTES = 2 * STAGE + 1024;            // two stages, and the rows' maxima and sums
    __device__ __forceinline__ static int swz(int row) { return CPR == 16 ? row & 15 : (row >> 1) & 7; }
};

// One block for a wave's 32 rows, from a stage's K and V, while the next step's blocks come into the other stage (pieces
// at offsets ko of its K and vo of its V).
template <int DH>
__device__ __forceinline__ void tile_step(WaveAttention<uint16_t, DH, 2>& w, unsigned char* next, const unsigned char* stage, bool load, bool use,
                                          const unsigned char* kb, const unsigned char* vb,
                                          const uint32_t (&ko)[DH / 32], const uint32_t (&vo)[DH / 32],
                                          const Frag<uint16_t> (&qh)[2][DH / 32], const Frag<uint16_t> (&ql)[2][DH / 32], int blk,
                                          int m0, const Sight& see, int lane) {
    using T = uint16_t;
    using S = TileShape<DH>;
    constexpr int NDS = DH / 32, NDT = DH / 16, PIECES = DH / 32;
    const int c = lane & 15, g = lane >> 4;
    if (load) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(kb + ko[i]),
                                             (__attribute__((address_space(3))) void*)(next + vo[i]), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(vb + vo[i] + c * 64 + g * 16),
                                             (__attribute__((address_space(3))) void*)(next + S::HALF + vo[i]), 16, 0, 0);
        }
    }
    if (!use) return;
#pragma unroll
    for (int t = 0; t < 2; ++t) w.s[t][0] = w.s[t][1] = w.minus[t];
    // K and V fragments are read one product group ahead of their use (the scheduler would move the reads next to it)
    auto k_frags = [&](Frag<T> (&kf)[2], int ds) {
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
            const int row = 16 * kt + c;
            kf[kt] = Frag<T>::load(reinterpret_cast<const T*>(stage + (row * S::CPR + ((ds * 4 + g) ^ S::swz(row))) * 16));
        }
    };
    const bool junk = 32 * blk + 32 > see.Tb;   // keys that no row sees: their V may be anything
    auto v_frags = [&](Frag<T> (&vf)[2], int dt) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            vf[u] = Frag<T>::load(reinterpret_cast<const T*>(stage + S::HALF + (dt + u) * 1024 + lane * 16));
    };
    // While loads into LDS are in flight the compiler waits for every read of LDS where it needs one: what a group needs is
    // waited for here, before the next one's reads are issued
    auto landed = [] {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);   // lgkmcnt 0
        __builtin_amdgcn_sched_barrier(0);
    };
    Frag<T> f[2][2];
    k_frags(f[0], 0);
#pragma unroll
    for (int ds = 0; ds < NDS; ++ds) {
        const Frag<T> (&kf)[2] = f[ds & 1];
        landed();
        if (ds + 1 < NDS) k_frags(f[(ds + 1) & 1], ds + 1);
        else v_frags(f[(ds + 1) & 1], 0);
        __builtin_amdgcn_sched_barrier(0);
        // products that follow each other go to different sums: each waits for its sum's last one
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) mma(w.s[t][kt], kf[kt], qh[t][ds]);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) mma(w.s[t][kt], kf[kt], ql[t][ds]);
        __builtin_amdgcn_sched_barrier(0);
    }
    w.look(blk, m0, see, lane);
    Frag<T> ph[2], pl[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) w.weigh(t, ph[t], pl[t]);
#pragma unroll
    for (int dt = 0; dt < NDT; dt += 2) {
        Frag<T> (&vf)[2] = f[(NDS + dt / 2) & 1];
        landed();
        if (dt + 2 < NDT) v_frags(f[(NDS + dt / 2 + 1) & 1], dt + 2);
        __builtin_amdgcn_sched_barrier(0);
        if (junk) {
            int key0 = 32 * blk;
            asm volatile("" : "+v"(key0));   // the masks are made here, in the last block, not in every one
#pragma unroll
            for (int u = 0; u < 2; ++u) drop_keys<T>(vf[u], key0, g, see.Tb);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int t = 0; t < 2; ++t) mma(w.o[t][dt + u], vf[u], ph[t]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int t = 0; t < 2; ++t) mma(w.o[t][dt + u], vf[u], pl[t]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The attention of rows row0 .. row0 + rows - 1 (at most 64) over blocks lo .. hi - 1 by 4 waves: wave 2 rs + kp has rows
// 32 rs .. of key lane kp.  K's rows are stored with their 16-byte chunks permuted by row (applied to the source address),
// so that 16 rows' same chunk lies in 16 different banks; V's fragments lie as the lanes read them.  smem: two stages.
template <int DH>
__device__ __forceinline__ void attend_tile(WaveAttention<uint16_t, DH, 2>& w, const AttnArgs& at, const HeadCache<uint16_t>& hc,
                                            int lo, int hi, int row0, int rows, int h, int m0, const Sight& see,
                                            unsigned char* smem, int wave, int lane) {
    using T = uint16_t;
    using S = TileShape<DH>;
    constexpr int NDS = DH / 32, PIECES = DH / 32;   // 1 KiB loads per operand and wave
    const int rs = wave >> 1, kp = wave & 1, c = lane & 15, g = lane >> 4;
    const int nstep = (hi - lo + 1) / 2;
    // waves 0, 1 load lane 0's block, waves 2, 3 lane 1's, half of its K and of its V each
    uint32_t ko[PIECES], vo[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int piece = (wave & 1) * PIECES + i, ch = piece * 64 + lane, row = ch / S::CPR;
        vo[i] = (uint32_t)piece * 1024;
        ko[i] = (uint32_t)(row * S::CPR + ((ch % S::CPR) ^ S::swz(row))) * 16;
    }
    Frag<T> qh[2][NDS], ql[2][NDS];
    // step i: its block is used (i >= 0), step i + 1's requested; a block past the last repeats it: in bounds, never used
    auto step = [&](int i) {
        const int j = min(lo + 2 * (i + 1) + (wave >> 1), hi - 1), blk = lo + 2 * i + kp;
        const bool shared = j < hc.pages;
        const unsigned char* kb = reinterpret_cast<const unsigned char*>(shared ? hc.k0 : hc.k1) + (size_t)j * S::HALF;
        const unsigned char* vb = reinterpret_cast<const unsigned char*>(shared ? hc.v0 : hc.v1) + (size_t)j * S::HALF;
        tile_step<DH>(w, smem + ((i + 1) & 1) * S::STAGE + (wave >> 1) * S::BLK, smem + (i & 1) * S::STAGE + kp * S::BLK,
                      i + 1 < nstep, i >= 0 && blk < hi && 32 * rs < rows, kb, vb, ko, vo, qh, ql, blk, m0 + 32 * rs, see, lane);
    };
    w.clear();
    if (nstep <= 0) return;
    f32x4u_t q8[2][NDS][2];   // loads return in order: the queries ahead of the first blocks
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int r = min(32 * rs + 16 * t + c, rows - 1);   // rows past the last repeat it
        const float* q0 = at.qbuf + ((size_t)(row0 + r) * at.H + h) * DH + 8 * g;
#pragma unroll
        for (int ds = 0; ds < NDS; ++ds)
#pragma unroll
            for (int u = 0; u < 2; ++u) q8[t][ds][u] = reinterpret_cast<const f32x4u_t*>(q0 + 32 * ds)[u];
    }
    step(-1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int ds = 0; ds < NDS; ++ds) query_frag<T>(at, q8[t][ds][0], q8[t][ds][1], qh[t][ds], ql[t][ds]);
    for (int i = 0; i < nstep; ++i) {
        // this wave's loads of step i have landed; after the barrier everyone's have, and nobody still reads the other stage
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(7 << 4);   // vmcnt 0, lgkmcnt 0
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        step(i);
    }
}

// The key lanes joined by log-sum-exp in lane order, as join_few; smem: the stages.
template <int DH, typename F>
__device__ __forceinline__ void join_tile(const WaveAttention<uint16_t, DH, 2>& w, unsigned char* smem, int rows, int wave, int lane,
                                          F out) {
    constexpr int NDT = DH / 16;
    static_assert(4 * 2 * NDT * 1024 <= 2 * TileShape<DH>::STAGE, "the waves' results fit the stages");
    f32x4_t* s_o = reinterpret_cast<f32x4_t*>(smem);   // [wave][t][dt][lane]
    float (*s_max)[2][16] = reinterpret_cast<float (*)[2][16]>(smem + 2 * TileShape<DH>::STAGE), (*s_sum)[2][16] = s_max + 4;
    const int rs = wave >> 1, kp = wave & 1, c = lane & 15, g = lane >> 4;
    __syncthreads();   // the stages are free
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const float sum = across_rows(w.rsum[t], OpSum());
        if (g == 0) {
            s_max[wave][t][c] = w.top(t);
            s_sum[wave][t][c] = sum;
        }
#pragma unroll
        for (int dt = 0; dt < NDT; ++dt) s_o[((wave * 2 + t) * NDT + dt) * 64 + lane] = w.o[t][dt];
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int r = 32 * rs + 16 * t + c;
        if (r >= rows) continue;
        float wt[2], top = -INFINITY, den = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) top = fmaxf(top, s_max[2 * rs + k][t][c]);
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const float m = s_max[2 * rs + k][t][c];
            wt[k] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
            den = fmaf(wt[k], s_sum[2 * rs + k][t][c], den);
        }
#pragma unroll
        for (int i = 0; i < NDT / 2; ++i) {
            const int dt = kp + 2 * i;
            f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x4_t ov = s_o[(((2 * rs + k) * 2 + t) * NDT + dt) * 64 + lane];
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(ov[e], wt[k], acc[e]);
            }
            out(r, 16 * dt + 4 * g, acc, top, den);
        }
    }
}

// ------------------------------------------------------------------ kernels
// A prefix part: head, group, pages and rows of unit `unit` (part and row tile); false where it has none.  The row tiles
// of a part are neighbours on one XCD (workgroups go to the 8 of them in turn).
struct PrefixPart { int h, b, lo, hi, row0, rows, slot; };
__device__ __forceinline__ bool prefix_part(const SharedArgs& a, int unit, int tile_rows, PrefixPart& p) {
    const int x = unit & 7, y = unit >> 3, tile = y % a.tiles, part = (y / a.tiles) * 8 + x;
    const int grp = part / a.prefix_parts / a.at.H;
    p.slot = part % a.prefix_parts;
    p.h = part / a.prefix_parts % a.at.H;
    p.b = grp * a.group;
    if (p.b >= a.at.B) return false;
    p.lo = p.slot * a.chunk;
    p.hi = min(p.lo + a.chunk, a.pages[grp]);
    p.row0 = p.b * a.at.q + tile * tile_rows;
    p.rows = min(tile_rows, a.group * a.at.q - tile * tile_rows);
    return p.lo < p.hi;   // else a shorter prefix than the longest group's: the join skips the part too
}

template <int DH>
__device__ __forceinline__ void store_part(const SharedArgs& a, int row, int h, int slot, int d, f32x4_t acc, float top, float den) {
    float* pr = a.part + (((size_t)row * a.at.H + h) * a.slots + slot) * (DH + 4);
    *reinterpret_cast<f32x4_t*>(pr + d) = acc;
    if (d == 0) *reinterpret_cast<float2*>(pr + DH) = float2{top, den};
}

// The rows of a block of sequence b that a workgroup has, of head h.
struct OwnRows { int h, b, m0, row0, rows, pages, prefix; };
__device__ __forceinline__ OwnRows own_rows(const SharedArgs& a, int i, int tile, int tile_rows) {
    OwnRows o;
    o.h = i % a.at.H;
    o.b = i / a.at.H;
    o.m0 = tile * tile_rows;
    o.row0 = o.b * a.at.q + o.m0;
    o.rows = min(tile_rows, a.at.q - o.m0);
    o.pages = a.pages[o.b / a.group];
    o.prefix = 32 * o.pages + a.rest[o.b / a.group];
    return o;
}
// Key blocks of sequence b (rows up to m of its block): none where the cache is too short (the host checks capacity;
// never read past this sequence's cache).
__device__ __forceinline__ int key_blocks(const SharedArgs& a, int L, int m) {
    return L < 0 || L + a.at.q > a.at.S_max ? 0 : (L + min(m, a.at.q) + 31) / 32;
}
__device__ __forceinline__ void report(const SharedArgs& a, int L, int prefix) {
    const bool over = L < 0 || L + a.at.q > a.at.S_max;
    if (threadIdx.x == 0 && (over || L < prefix)) atomicOr(a.at.err, over ? 4 : 16);
}
__device__ __forceinline__ Sight own_sight(const SharedArgs& a, int b, int L) {
    return {L, L + a.at.q, a.at.q, a.at.mask ? a.at.mask + (size_t)b * a.at.q : nullptr};
}

// The parts: workgroups of the prefix, then those of the own slots.
template <typename T, int DH, bool STAGED>
__global__ void __launch_bounds__(256, STAGED || sizeof(T) * DH > 256 ? 2 : 3) shared_parts_kernel(SharedArgs a) {
    __shared__ __align__(1024) unsigned char smem[STAGED ? TileShape<DH>::BYTES : FewBytes<DH>];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if ((int)blockIdx.x < a.prefix_grid) {
        PrefixPart p;
        auto store = [&](int r, int d, f32x4_t acc, float top, float den) {
            store_part<DH>(a, p.row0 + r, p.h, p.slot, d, acc, top, den);
        };
        const Sight all{0x7FFFFFFF, 0x7FFFFFFF, 0, nullptr};
        if constexpr (STAGED) {
            if (!prefix_part(a, blockIdx.x, kTileRows, p)) return;
            WaveAttention<T, DH, 2> w;
            attend_tile<DH>(w, a.at, head_cache<T, DH>(a.at, p.b, p.b, p.h, 0), p.lo, p.hi, p.row0, p.rows, p.h, 0, all, smem,
                            wave, lane);
            join_tile<DH>(w, smem, p.rows, wave, lane, store);
        } else {
            // two units: waves 0, 1 and waves 2, 3 (of neighbours on one XCD)
            const int unit = ((int)blockIdx.x >> 3) * 16 + (wave >> 1) * 8 + (blockIdx.x & 7);
            const bool any = prefix_part(a, unit, 16, p);
            WaveAttention<T, DH, 1> w;
            w.clear();
            if (any)
                attend_few<T, DH, kPrefixLanes>(w, a.at, head_cache<T, DH>(a.at, p.b, p.b, p.h, 0), p.lo, p.hi, p.row0, p.rows,
                                                p.h, 0, wave & 1, lane, nullptr, [&](int, int&) { return all; });
            join_few<T, DH, kPrefixLanes>(w, smem, any ? p.rows : 0, wave, lane, store);
        }
        return;
    }
    const int tiles = (a.at.q + 15) / 16, i = (int)blockIdx.x - a.prefix_grid, part = i % a.own_parts, j = i / a.own_parts;
    const OwnRows o = own_rows(a, j / tiles, j % tiles, 16);
    // the last part takes what is left: the device's lengths may exceed the host's (a replayed graph)
    const int lo = o.pages + part * a.own_chunk, most = a.at.S_max / 32, end = part == a.own_parts - 1 ? most : min(lo + a.own_chunk, most);
    WaveAttention<T, DH, 1> w;
    attend_few<T, DH, kOwnLanes>(w, a.at, head_cache<T, DH>(a.at, o.b, o.b, o.h, 0), lo, end, o.row0, o.rows, o.h, o.m0, wave,
                                 lane, a.at.cache_len + o.b, [&](int L, int& hi) {
        if (part == 0) report(a, L, o.prefix);
        hi = min(hi, key_blocks(a, L, a.at.q));
        return own_sight(a, o.b, L);
    });
    join_few<T, DH, kOwnLanes>(w, smem, o.rows, wave, lane, [&](int r, int d, f32x4_t acc, float top, float den) {
        store_part<DH>(a, o.row0 + r, o.h, a.prefix_parts + part, d, acc, top, den);
    });
}

// Joins the parts of each row and head, DH / 4 threads with four columns each: parts that hold no key of the row (maximum
// -inf) count nothing.
template <typename T, int DH>
__global__ void __launch_bounds__(256) shared_join_kernel(SharedArgs a) {
    constexpr int D4 = DH / 4, U = 8;   // parts whose loads are in flight together
    const int e = (int)(blockIdx.x * 256 + threadIdx.x), rh = e / D4, d = 4 * (e % D4), row = rh / a.at.H, h = rh % a.at.H;
    if (row >= a.at.B * a.at.q) return;
    const int b = row / a.at.q, np = (a.pages[b / a.group] + a.chunk - 1) / a.chunk, all = np + a.own_parts;
    const float* base = a.part + (size_t)rh * a.slots * (DH + 4);
    f32x4_t sum = f32x4_t{0.f, 0.f, 0.f, 0.f};
    float total = 0.f, top = -INFINITY;
    for (int k = 0; k < all; k += U) {   // past the last it is read again
        f32x4_t ov[U];
        float2 ms[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = min(k + u, all - 1);
            const float* pr = base + (size_t)(i < np ? i : a.prefix_parts + i - np) * (DH + 4);
            ov[u] = *reinterpret_cast<const f32x4_t*>(pr + d);
            ms[u] = *reinterpret_cast<const float2*>(pr + DH);
        }
        float m = top;
#pragma unroll
        for (int u = 0; u < U; ++u) m = fmaxf(m, ms[u].x);
        const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - m);
        top = m;
        total *= f;
        sum *= f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float wt = k + u >= all || ms[u].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ms[u].x - m);
            total = fmaf(wt, ms[u].y, total);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(ov[u][i], wt, sum[i]);
        }
    }
    const float inv = total == 0.f ? 0.f : 1.0f / total;   // a row that sees no key: zeros
    store_out<T>(a.at, out_off<DH>(a.at, b, h, row - b * a.at.q, d), sum * inv);
}

// Blocks of more than kAttnSplitRows rows: prefix and own pages in one workgroup per row tile, the longest first.
template <typename T, int DH>
__global__ void __launch_bounds__(256, 2) shared_rows_kernel(SharedArgs a) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    constexpr int TILE = sizeof(T) == 2 ? kTileRows : 16;
    __shared__ __align__(1024) unsigned char smem[sizeof(T) == 2 ? TileShape<DH>::BYTES : FewBytes<DH>];
    // a ragged last tile of few rows after the others, beside which it fits; a head's tiles on one XCD where heads come in
    // eights
    const int nth = (int)blockIdx.x / (a.at.B * a.at.H), last = a.at.q % TILE;
    const int tile = last && 2 * last <= TILE ? (nth + 1 == a.tiles ? nth : a.tiles - 2 - nth) : a.tiles - 1 - nth;
    const OwnRows o = own_rows(a, (int)blockIdx.x % (a.at.B * a.at.H), tile, TILE);
    const int L = __builtin_amdgcn_readfirstlane(a.at.cache_len[o.b]), nblk = key_blocks(a, L, o.m0 + TILE);   // what the tile's last row can see
    report(a, L, o.prefix);
    const Sight see = own_sight(a, o.b, L);
    const HeadCache<T> hc = head_cache<T, DH>(a.at, o.b / a.group * a.group, o.b, o.h, o.pages);
    auto write = [&](int r, int d, f32x4_t acc, float, float den) {
        const float inv = den == 0.f ? 0.f : 1.0f / den;   // a row that sees no key: zeros
        store_out<T>(a.at, out_off<DH>(a.at, o.b, o.h, o.m0 + r, d), acc * inv);
    };
    if constexpr (sizeof(T) == 2) {
        WaveAttention<T, DH, 2> w;
        attend_tile<DH>(w, a.at, hc, 0, nblk, o.row0, o.rows, o.h, o.m0, see, smem, wave, lane);
        join_tile<DH>(w, smem, o.rows, wave, lane, write);
    } else {
        WaveAttention<T, DH, 1> w;
        attend_few<T, DH, 4>(w, a.at, hc, 0, nblk, o.row0, o.rows, o.h, o.m0, wave, lane, nullptr, [&](int, int&) { return see; });
        join_few<T, DH, 4>(w, smem, o.rows, wave, lane, write);
    }
}

template <typename T, int DH>
static hipError_t launch_shared_dh(const SharedPlan& p, const SharedArgs& a, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
    auto go = [&](void (*kern)(SharedArgs), size_t grid, hipEvent_t begin, hipEvent_t end) {
        if (begin || end) hipExtLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), 0, s, begin, end, 0, a);
        else hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), 0, s, a);
        return hipGetLastError();
    };
    if (p.whole) return go(shared_rows_kernel<T, DH>, p.grid, ev0, ev1);
    void (*parts)(SharedArgs) = shared_parts_kernel<T, DH, false>;
    if constexpr (sizeof(T) == 2) {
        if (p.staged) parts = shared_parts_kernel<T, DH, true>;
    }
    const hipError_t e = go(parts, p.grid, ev0, nullptr);
    if (e != hipSuccess) return e;
    return go(shared_join_kernel<T, DH>, ((size_t)a.at.B * a.at.q * a.at.H * (DH / 4) + 255) / 256, nullptr, ev1);
}

hipError_t launch_attention_shared(int dtype, int head_dim, const SharedPlan& p, SharedArgs a, hipStream_t s, hipEvent_t ev0,
                                   hipEvent_t ev1) {
    const AttnArgs& at = a.at;
    if (at.q < 1 || at.q > 4096 || (at.mask && at.q > 64) || at.B < 1 || at.H < 1 || a.group < 1 || at.B % a.group ||
        at.B / a.group > kMaxShareGroups || at.S_max < 32 || at.S_max % 32 || !shared_supported(at.S_max, head_dim, dtype == 1 ? 2 : 4) ||
         at.ldo % 4 || !at.qbuf || !at.kc || !at.vc ||
        !at.cache_len || !at.out || !at.err || p.whole != (at.q > kAttnSplitRows) || (!p.whole && !a.part) ||
        (dtype != 1 && p.staged) || (dtype == 1 && p.whole && !p.staged))
        return hipErrorInvalidValue;
    for (int g = 0; g < at.B / a.group; ++g)
        if (a.pages[g] < 0 || a.pages[g] > at.S_max / 32 || a.rest[g] < 0 || a.rest[g] > 31 ||
            (!p.whole && a.pages[g] > p.chunk * p.prefix_parts))
            return hipErrorInvalidValue;
    a.chunk = p.chunk; a.prefix_parts = p.prefix_parts; a.own_chunk = p.own_chunk; a.own_parts = p.own_parts;
    a.slots = p.slots; a.tiles = p.tiles; a.prefix_grid = p.prefix_grid;
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
