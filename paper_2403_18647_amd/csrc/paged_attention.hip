// Attention over a paged cache: the rows of a call's chunks (pieces of prompts, draft and verify blocks, single tokens)
// against the pages of their sequences, whose last slots the chunk itself has filled.
//
// For sequence b, query head h and the chunk's row i (at slot s = len_b + i):
//   O = softmax(scale q [K]^T) [V] over the slots it sees: s - window + 1 .. s, or all below len_b and the chunk's slots of
//   its mask.  A row that sees nothing gives zeros.
// The H / Hkv query heads that share a key head are rows of one product: packed row i * group + head.
//
// The scores of 32 slots and 32 packed rows are formed as S^T = K Q^T, so that a lane has 16 slots of one row (its row's
// others are in lane ^ 32), and enter O^T += V^T P^T as they stand: K's rows are read in the order in which V's pages hold
// their slots.  Scores, sums and O are float.  On bf16 pools P enters as value and remainder (16 bits), which costs short
// chunks 0 to 3% (a token each of 64 sequences 143 and 144.5 us, 11 rows of 8 over 4000 slots 47.6 and 49.0) and tiles half
// the time again (4096 rows behind 4096 slots 434 and 652 us).  So tiles round P to bf16 where the output is rounded to it
// too (half a step, 2^-8 of each weight at the most; error 0.0023 of the output's size, 0.0017 being its own rounding; the
// row's sum takes the unrounded weights) and take it whole where the output is float.
// A row keeps a base, in units of log 2, that its weights are 2 to the score above; the base is raised, and O scaled, only
// when a score of the row's own passes it by more than kRaise: in most blocks nothing is scaled.
//
// Two kinds of workgroup of four waves, in one launch:
//  * tiles, of chunks of more than kPagedFewRows packed rows: 128 rows, 32 for each wave; two pages at a time go straight
//    into LDS while the two before are used;
//  * short chunks, up to kPagedFewRows packed rows: 32 rows and a part of the sequence's pages, which the waves take in
//    turn; a wave's page goes into its own piece of LDS, K's half while the page before is weighed with V, V's half while
//    the next scores are formed; no barriers.  The waves' results are joined by log-sum-exp in wave order.
// A short chunk's part is 2^part_shift pages from a slot that is a multiple of them, the same for the handle's every call:
// a row's result depends neither on what else is in its call nor on the chunk's other rows.  Tiles are in as many parts as
// the call's number of them leaves room for, so that their results depend on the call's chunks in the order of summation.
// Results of parts go to scratch; a second launch joins them (in the workgroup that comes last it took longer: 11 rows of 8
// sequences over 3000 slots 47 us, 39 so).
//
// Bound by memory where rows are few: a token each of 64 sequences of up to 4000 slots, 8 key heads of 128 in bf16 (893 MB),
// 144 us, 6.2 TB/s; of one of 130000 (533 MB) 88, 6.1; and by the way to the first page and the second launch where slots
// are few too (11 rows each of 4 sequences of 1500, 98 MB: 26 us, 14 at the rate of a read stream).  Long chunks keep
// neither pipe full: 4096 rows behind 4096 slots, 32 heads, 412 GFLOP, take 417 to 435 us, 950 to 990 TFLOP/s (a large
// product 1180 to 1230), with the vector pipes busy 58% of the cycles, for the softmax, and the matrix pipes 49%, at the
// clock of 1.7 GHz that the card holds under both; without the softmax, or without loads and barriers, it took about a
// tenth less.  A chunk of 1001 rows beside 31 single tokens: 165 us, 74 at both rates.
#include <algorithm>
#include <type_traits>

#include "paged_device.h"

namespace sdsat {

static constexpr float kRaise = 8.f;

static constexpr int kWaves = 4;

typedef float f32x16_t __attribute__((ext_vector_type(16)));

// acc += A(32 x 16) B(16 x 32): lane l holds A's row and B's column l % 32, contraction indices 8 (l / 32) .. + 7; of the
// result column l % 32, rows 8 (i / 4) + 4 (l / 32) + i % 4
__device__ __forceinline__ void mma32(f32x16_t& acc, const Frag<uint16_t>& a, const Frag<uint16_t>& b) {
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a.v), __builtin_bit_cast(bf16x8_t, b.v), acc, 0, 0, 0);
}
__device__ __forceinline__ void mma32(f32x16_t& acc, const Frag<float>& a, const Frag<float>& b) {
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.lo[e], b.lo[e], acc, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a.hi[e], b.hi[e], acc, 0, 0, 0);
}

// A page's K (32 rows of DH) or V (DH rows of 32) in LDS: rows as in memory, their 16-byte chunks exchanged by row, so that
// a chunk of neighbouring rows lies in different banks.
template <typename T, int DH>
struct PageTile {
    static constexpr int E = (int)sizeof(T), HALF = 32 * DH * E, BLK = 2 * HALF, PIECES = HALF / 1024;
    template <int RB>
    __device__ __forceinline__ static int swz(int row) {
        constexpr int CPR = RB / 16;
        return RB >= 256 ? row & 15 : (row * RB / 256) & (CPR - 1);
    }
    // where lane `lane` of the piece's load (1 KiB, linear in LDS) reads in the page's K (RB = DH * E) or V (RB = 32 * E)
    template <int RB>
    __device__ __forceinline__ static uint32_t source(int piece, int lane) {
        constexpr int CPR = RB / 16;
        const int ch = piece * 64 + lane, row = ch / CPR;
        return (uint32_t)(row * CPR + ((ch % CPR) ^ swz<RB>(row))) * 16;
    }
    template <int RB>
    __device__ __forceinline__ static Frag<T> frag(const unsigned char* at, int row, int first) {   // 8 elements from chunk `first`
        Frag<T> f;
        const unsigned char* r = at + row * RB;
        const int z = swz<RB>(row);
        if constexpr (sizeof(T) == 2) {
            f.v = *reinterpret_cast<const u32x4_t*>(r + ((first ^ z) << 4));
        } else {
            f.lo = *reinterpret_cast<const f32x4_t*>(r + ((first ^ z) << 4));
            f.hi = *reinterpret_cast<const f32x4_t*>(r + (((first + 1) ^ z) << 4));
        }
        return f;
    }
    // K's row of result row l % 32 (lane l): bits 3 and 4 exchanged, the slots' order in V's pages
    __device__ __forceinline__ static Frag<T> k(const unsigned char* at, int ks, int lane) {
        const int r = lane & 31, row = (r & 7) | (r & 8) << 1 | (r & 16) >> 1;
        return frag<DH * E>(at, row, (16 * ks + 8 * (lane >> 5)) * E / 16);
    }
    __device__ __forceinline__ static Frag<T> v(const unsigned char* at, int dt, int s, int lane) {
        return frag<32 * E>(at, 32 * dt + (lane & 31), 8 * (2 * s + (lane >> 5)) * E / 16);
    }
};

// A page's K or V on its way into LDS (at dst, the wave's), through a buffer resource over it: the pieces' addresses repeat
// after 16 rows, so a few lane offsets and the instruction's own offset (which counts on both sides) make them.
template <typename T, int DH, int RB>
struct Fetch {
    using P = PageTile<T, DH>;
    static constexpr int VARS = RB / 64;
    uint32_t off[VARS];
    __device__ __forceinline__ explicit Fetch(int lane) {
#pragma unroll
        for (int i = 0; i < VARS; ++i) off[i] = P::template source<RB>(i, lane) - i * 1024;
    }
    template <int N, int AUX, int I = 0>   // pieces first .. first + N - 1 (first a multiple of VARS), to their places
    __device__ __forceinline__ void pieces(const unsigned char* src, unsigned char* dst, int first) const {
#ifdef __HIP_DEVICE_COMPILE__   // the host's pass over several kernels that load alike does not know the builtin
        if constexpr (I < N) {
            const int at = (first + I / 4 * 4) * 1024;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(buf_rsrc(src, P::HALF), (__attribute__((address_space(3))) void*)(dst + at), 16,
                                                     off[I % VARS], at, I % 4 * 1024, AUX);
            pieces<N, AUX, I + 1>(src, dst, first);
        }
#else
        (void)src, (void)dst, (void)first;
#endif
    }
};
// Eight fragments out of LDS, and the wait for them.  In one piece of assembly: the compiler holds every read of LDS behind
// all loads into it that are in flight, the ones for the next page too.
template <int O0, int O1, int O2, int O3, int O4, int O5, int O6, int O7>
__device__ __forceinline__ void read8(Frag<uint16_t> (&f)[8], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t a4,
                                      uint32_t a5, uint32_t a6, uint32_t a7) {
    asm volatile(
        "ds_read_b128 %0, %8 offset:%16\n\tds_read_b128 %1, %9 offset:%17\n\tds_read_b128 %2, %10 offset:%18\n\t"
        "ds_read_b128 %3, %11 offset:%19\n\tds_read_b128 %4, %12 offset:%20\n\tds_read_b128 %5, %13 offset:%21\n\t"
        "ds_read_b128 %6, %14 offset:%22\n\tds_read_b128 %7, %15 offset:%23\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(f[0].v), "=&v"(f[1].v), "=&v"(f[2].v), "=&v"(f[3].v), "=&v"(f[4].v), "=&v"(f[5].v), "=&v"(f[6].v), "=&v"(f[7].v)
        : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "v"(a4), "v"(a5), "v"(a6), "v"(a7), "i"(O0), "i"(O1), "i"(O2), "i"(O3), "i"(O4),
          "i"(O5), "i"(O6), "i"(O7)
        : "memory");
}
template <int O0, int O1, int O2, int O3>
__device__ __forceinline__ void read4(Frag<uint16_t> (&f)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
    asm volatile(
        "ds_read_b128 %0, %4 offset:%8\n\tds_read_b128 %1, %5 offset:%9\n\tds_read_b128 %2, %6 offset:%10\n\t"
        "ds_read_b128 %3, %7 offset:%11\n\ts_waitcnt lgkmcnt(0)"
        : "=&v"(f[0].v), "=&v"(f[1].v), "=&v"(f[2].v), "=&v"(f[3].v)
        : "v"(a0), "v"(a1), "v"(a2), "v"(a3), "i"(O0), "i"(O1), "i"(O2), "i"(O3)
        : "memory");
}
// A lane's reads of a page in LDS, K at `base` (bytes into smem), V behind it: all fragments of a head, and the wait.
template <typename T, int DH>
struct PageRead {
    using P = PageTile<T, DH>;
    static constexpr int KS = DH / 16, DT = DH / 32;
    const unsigned char* at;
    int lane;
    __device__ __forceinline__ PageRead(const unsigned char* smem, int base, int l) : at(smem + base), lane(l) {}
    __device__ __forceinline__ void move(int by) { at += by; }
    template <int AT>   // the page AT bytes further
    __device__ __forceinline__ void k(Frag<T> (&f)[KS]) const {
#pragma unroll
        for (int i = 0; i < KS; ++i) f[i] = P::k(at + AT, i, lane);
    }
    template <int AT>   // fragment s * DT + dt
    __device__ __forceinline__ void v(Frag<T> (&f)[KS]) const {
#pragma unroll
        for (int i = 0; i < KS; ++i) f[i] = P::v(at + AT + P::HALF, i % DT, i / DT, lane);
    }
};
template <int DH>
struct PageRead<uint16_t, DH> {
    using P = PageTile<uint16_t, DH>;
    static constexpr int KS = DH / 16;
    uint32_t ka[KS], va[2];
    __device__ __forceinline__ PageRead(const unsigned char* smem, int base, int lane) {
        const uint32_t at = (uint32_t)(size_t)(const __attribute__((address_space(3))) unsigned char*)smem + base;
        const int r = lane & 31, g = lane >> 5, row = (r & 7) | (r & 8) << 1 | (r & 16) >> 1;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) ka[ks] = at + row * DH * 2 + ((2 * ks + g) ^ P::template swz<DH * 2>(row)) * 16;
#pragma unroll
        for (int s = 0; s < 2; ++s) va[s] = at + P::HALF + r * 64 + ((2 * s + g) ^ P::template swz<64>(r)) * 16;
    }
    __device__ __forceinline__ void move(int by) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) ka[ks] += by;
        va[0] += by;
        va[1] += by;
    }
    template <int AT>
    __device__ __forceinline__ void k(Frag<uint16_t> (&f)[KS]) const {
        if constexpr (KS == 8) read8<AT, AT, AT, AT, AT, AT, AT, AT>(f, ka[0], ka[1], ka[2], ka[3], ka[4], ka[5], ka[6], ka[7]);
        else read4<AT, AT, AT, AT>(f, ka[0], ka[1], ka[2], ka[3]);
    }
    template <int AT>
    __device__ __forceinline__ void v(Frag<uint16_t> (&f)[KS]) const {
        if constexpr (KS == 8)
            read8<AT, AT + 2048, AT + 4096, AT + 6144, AT, AT + 2048, AT + 4096, AT + 6144>(f, va[0], va[0], va[0], va[0], va[1], va[1], va[1], va[1]);
        else
            read4<AT, AT + 2048, AT, AT + 2048>(f, va[0], va[0], va[1], va[1]);
    }
};

// at most N loads are outstanding
template <int N>
__device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void wait_lds() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// The slots that a lane's row sees, and those that every row of the wave does.
struct Sight {
    int first, last;    // slots of this row (of the tree mask: up to the chunk's end)
    int len;            // tree: the slots below it
    uint64_t bits;      // ... and of the chunk's those
    bool tree;
    int all_first, all_last;
    __device__ __forceinline__ bool sees(int slot) const {
        const bool v = (slot >= first) & (slot <= last);
        return tree ? v & ((slot < len) | (bool)(bits >> ((slot - len) & 63) & 1)) : v;
    }
};

// want 0: finite values as they are, others as zero; ones where +inf (1), -inf (2), NaN (3), any of them (4)
template <typename T>
__device__ __forceinline__ Frag<T> select_values(Frag<T> f, int want) {
    // opaque: nothing of this is formed ahead for the steps that do not need it
    if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(f.v));
    else asm volatile("" : "+v"(f.lo), "+v"(f.hi));
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float v = f.get(j);
        const bool nan = v != v, inf = !nan && fabsf(v) == INFINITY;
        const bool hit = want == 1 ? inf && v > 0.f : want == 2 ? inf && v < 0.f : nan || (want == 4 && inf);
        x[j] = want == 0 ? (nan || inf ? 0.f : v) : hit ? 1.f : 0.f;
    }
    return Frag<T>::from_f32(x);
}
// a value's sign bit set in `seen` where an exponent is all ones: one more there carries into it
__device__ __forceinline__ void mark_not_finite(const Frag<uint16_t>& f, uint32_t& seen) {
#pragma unroll
    for (int j = 0; j < 4; ++j) seen |= (f.v[j] & 0x7F807F80u) + 0x00800080u;
}
__device__ __forceinline__ void mark_not_finite(const Frag<float>& f, uint32_t& seen) {
#pragma unroll
    for (int j = 0; j < 8; ++j) seen |= (__float_as_uint(f.get(j)) & 0x7F800000u) + 0x00800000u;
}
template <typename T>
constexpr uint32_t kSignBits = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;

// The weights of a page, as the second product takes them.  FINE, bf16 pools: as value and remainder (16 bits of each), so
// that they are no rounding point.
template <typename T, bool FINE>
struct Weights {
    static constexpr bool REST = FINE && sizeof(T) == 2;
    Frag<T> p[2], rest[REST ? 2 : 1];
    __device__ __forceinline__ void set(const float (&w)[16]) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            p[s] = Frag<T>::from_f32(w + 8 * s);
            if constexpr (REST) {
                float r[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) r[j] = w[8 * s + j] - p[s].get(j);
                rest[s] = Frag<T>::from_f32(r);
            }
        }
    }
};

// A wave's 32 rows: queries, and the running softmax over NB pages at a time.
template <typename T, int DH, int NB, bool FINE>
struct RowWave {
    static constexpr int KS = DH / 16, DT = DH / 32;
    using W = Weights<T, FINE>;
    Frag<T> q[KS];
    f32x16_t o[DT];
    float base, sum;   // base -inf: nothing seen yet

    __device__ __forceinline__ void clear() {
        base = -INFINITY;
        sum = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[dt][i] = 0.f;
    }
    __device__ __forceinline__ void load_q(const T* row, int lane) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = Frag<T>::load(row + 16 * ks + 8 * (lane >> 5));
    }
    // the queries are here: their loads, ahead of those into LDS, are waited for once and not in every step
    __device__ __forceinline__ void have_q() {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if constexpr (sizeof(T) == 2) asm volatile("" : "+v"(q[ks].v));
            else asm volatile("" : "+v"(q[ks].lo), "+v"(q[ks].hi));
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    __device__ __forceinline__ void scores(f32x16_t& s, const Frag<T> (&k)[KS]) const {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) mma32(s, k[ks], q[ks]);
    }
    // the slot of a lane's i-th score of a page
    __device__ __forceinline__ static int slot_of(int page, int i, int lane) {
        return 32 * page + 16 * (i / 4 % 2) + 8 * (i / 8) + 4 * (lane >> 5) + i % 4;
    }
    // scores of pages blk .. to weights; masked: some row does not see all of them (pages from `end` on: none does)
    __device__ __forceinline__ void weigh(const f32x16_t (&s)[NB], W (&p)[NB], int blk, int end, bool masked, const Sight& see,
                                          float scale, int lane) {
        float x[NB][16];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[n][i] = s[n][i];
        if (masked) {
            asm volatile("" : "+v"(lane));   // nothing of the masks is formed ahead for the steps that need none
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[n][i] = ((blk + n < end) & see.sees(slot_of(blk + n, i, lane))) ? x[n][i] : -INFINITY;
                }
        }
        float top = x[0][0];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, x[n][i]);
        {
            const uint32_t u = __float_as_uint(top);
            const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
            top = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])) * scale;   // scale > 0
        }
        // each row for itself: what the wave's other rows do must not move its base, which its weights are rounded to
        const bool raise = (top > base + kRaise) | ((base == -INFINITY) & (top > base));
        if (__any(raise)) {
            const float to = raise ? top : base;   // top > base
            const float alpha = !raise ? 1.f : base == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(base - to);
            sum *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[dt] *= alpha;
            base = to;
        }
        const float minus = base == -INFINITY ? 0.f : -base;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            float w[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                w[i] = __builtin_amdgcn_exp2f(fmaf(x[n][i], scale, minus));
                sum += w[i];
            }
            p[n].set(w);
        }
    }
    // O += P V of page blk.  Values that are not finite must not meet weights of slots that a row does not see, which are
    // zero, nor remainders, which have either sign: they are taken out of the product, and infinities and NaN of slots that
    // do count are put in by products with where they stand (NaN where a slot is seen, but its weight is below the smallest
    // float: zero times infinity).
    __device__ __forceinline__ void weighted(const W& p, Frag<T> (&v)[KS], int blk, int end, bool masked, const Sight& see, int lane) {
        bool odd = false;
        int fine = FINE;
        asm volatile("" : "+s"(fine));   // a branch all the same: without it O and V are copied ahead of the rare part, into scratch
        const bool look = masked || fine != 0;
        if (look) {
            uint32_t seen = 0;
#pragma unroll
            for (int i = 0; i < KS; ++i) mark_not_finite(v[i], seen);
            odd = __any((seen & kSignBits<T>) != 0);
        }
        if (look && odd) {
            asm volatile("" : "+v"(lane));
            Frag<T> none[2];   // ones where a slot is seen with a weight of zero
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    x[j] = (!masked || (blk < end && see.sees(slot_of(blk, 8 * s + j, lane)))) && p.p[s].get(j) == 0.f ? 1.f : 0.f;
                none[s] = Frag<T>::from_f32(x);
            }
            // one copy of this, on tile 0, the tiles taking turns there
#pragma unroll 1
            for (int dt = 0; dt < DT; ++dt) {
#pragma unroll 1
                for (int want = 1; want < 5; ++want) {
                    f32x16_t d;
#pragma unroll
                    for (int i = 0; i < 16; ++i) d[i] = 0.f;
#pragma unroll
                    for (int s = 0; s < 2; ++s) mma32(d, select_values(v[s * DT], want), want == 4 ? none[s] : p.p[s]);
                    const float x = want == 1 ? INFINITY : want == 2 ? -INFINITY : NAN;
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[0][i] += d[i] > 0.f ? x : 0.f;
                }
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const Frag<T> f = select_values(v[s * DT], 0);
#pragma unroll
                    for (int t = 0; t + 1 < DT; ++t) v[s * DT + t] = v[s * DT + t + 1];
                    v[s * DT + DT - 1] = f;
                }
                const f32x16_t o0 = o[0];
#pragma unroll
                for (int t = 0; t + 1 < DT; ++t) o[t] = o[t + 1];
                o[DT - 1] = o0;
            }
        }
#pragma unroll
        for (int i = 0; i < KS; ++i) mma32(o[i % DT], v[i], p.p[i / DT]);
        if constexpr (W::REST) {
#pragma unroll
            for (int i = 0; i < KS; ++i) mma32(o[i % DT], v[i], p.rest[i / DT]);
        }
    }
    __device__ __forceinline__ float whole_sum() const {
        const uint32_t u = __float_as_uint(sum);
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
};

__device__ __forceinline__ void put4(__amdgpu_buffer_rsrc_t r, uint32_t off, f32x4_t v) {
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, v), r, off, 0, 0);
}

// packed rows row0 .. row0 + rows - 1 of a chunk and key head
struct Rows {
    int b, h, row0, rows, group;
    PagedSeq seq;
    uint32_t inv;   // of short chunks: ceil(2^16 / group); 0: divide
    // the chunk's row of packed row p (p + 1 <= kPagedFewRows where inv is given: then p * inv < 2^16 (p / group + 1))
    __device__ __forceinline__ int row(int p) const { return inv ? (int)(((uint32_t)p * inv) >> 16) : p / group; }
};

template <typename T, int DH>
__device__ __forceinline__ const T* q_row(const PagedAttnArgs& a, const Rows& r, int n) {
    const int p = r.row0 + min(n, r.rows - 1);
    const int i = r.row(p);
    return reinterpret_cast<const T*>(a.q) + (size_t)(r.seq.start + i) * a.ldq + (size_t)(r.h * r.group + p - i * r.group) * DH;
}

template <typename T, int DH>
__device__ __forceinline__ void store_row(const PagedAttnArgs& a, const Rows& r, int n, int d, f32x4_t v) {
    const int p = r.row0 + n, i = r.row(p);
    const size_t off = (size_t)(r.seq.start + i) * a.ldo + (size_t)(r.h * r.group + p - i * r.group) * DH + d;
    if (sizeof(T) == 4 || a.out_f32) *reinterpret_cast<f32x4_t*>(reinterpret_cast<float*>(a.out) + off) = v;
    else *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(a.out) + off) = uint2{f32x2_to_bf16x2(v[0], v[1]), f32x2_to_bf16x2(v[2], v[3])};
}

template <typename T, int DH>
__device__ __forceinline__ Sight sight_of(const PagedAttnArgs& a, const Rows& r, int w0, int lane) {
    Sight s;
    const int end = r.rows - 1;   // rows past it, and those of a wave that has none, look like the last
    const int i = r.row(r.row0 + min(w0 + (lane & 31), end));
    const int i0 = r.row(r.row0 + min(w0, end)), i1 = r.row(r.row0 + min(w0 + 31, end));
    s.tree = a.mask != nullptr;
    s.len = r.seq.len;
    s.first = a.window && !s.tree ? max(0, r.seq.len + i - a.window + 1) : 0;
    s.last = r.seq.len + (s.tree ? r.seq.n - 1 : i);
    s.bits = s.tree ? a.mask[r.seq.start + i] : 0;
    s.all_first = a.window && !s.tree ? max(0, r.seq.len + i1 - a.window + 1) : 0;
    s.all_last = s.tree ? r.seq.len - 1 : r.seq.len + i0;
    return s;
}

// A part of R rows (32 at most): [DH / 4][R] quads of O to the part's base, whole lines as the waves hold them, then [R]
// quads of the base and the sum.
template <int DH>
constexpr int kPartFloats = 32 * (DH + 4);
template <int DH>
__device__ __forceinline__ uint32_t part_quad(int R, int i, int d4) { return (uint32_t)(d4 * R + i) * 16; }   // d4 = DH / 4: base, sum

// LDS: pages, the waves' bases and sums.
template <typename T, int DH>
constexpr int kLdsBytes = kWaves * PageTile<T, DH>::BLK + 2 * kWaves * 32 * 4;

// A call's work in pieces, numbered through the sequences: where piece `want` is, and how many there are.  pieces(lane's
// sequence) counts those of one; 64 sequences are looked at at once.
struct Found { bool ok; int b, k; PagedSeq seq; };
template <typename F>
__device__ __forceinline__ Found find_piece(const PagedSeqs& s, int want, int lane, F pieces) {
    for (int b0 = 0; b0 < s.B; b0 += 64) {
        const int b = b0 + lane;
        PagedSeq q = load_seq(s, min(b, s.B - 1));
        const int mine = b < s.B ? pieces(q) : 0;
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o, 64);
            if (lane >= o) upto += v;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (want < all) {
            const int at = __popcll(__ballot(upto <= want));   // the first lane whose sum passes it
            const int k = want - (__builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at));
            return Found{true, b0 + at, k, PagedSeq{__builtin_amdgcn_readlane(q.start, at), __builtin_amdgcn_readlane(q.n, at),
                                                    __builtin_amdgcn_readlane(q.len, at), true}};
        }
        want -= all;
    }
    return Found{false, 0, 0, PagedSeq{0, 0, 0, false}};
}
template <typename F>
__device__ __forceinline__ int count_pieces(const PagedSeqs& s, int lane, F pieces) {
    int all = 0;
    for (int b0 = 0; b0 < s.B; b0 += 64) {
        const int b = b0 + lane;
        all = min(all + (b < s.B ? pieces(load_seq(s, b)) : 0), 1 << 24);   // starts that do not ascend: no overflow either
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o, 64);
    return __builtin_amdgcn_readfirstlane(all);
}

// Pages lo .. hi - 1 that the chunk's rows i0 .. i1 see between them.
__device__ __forceinline__ void page_range(const PagedAttnArgs& a, const PagedSeq& q, int i0, int i1, int& lo, int& hi) {
    const bool tree = a.mask != nullptr;
    lo = a.window && !tree ? max(0, q.len + i0 - a.window + 1) / kPage : 0;
    hi = (q.len + (tree ? q.n - 1 : i1)) / kPage + 1;
}
__device__ __forceinline__ void page_range(const PagedAttnArgs& a, const Rows& r, int& lo, int& hi) {
    page_range(a, r.seq, r.row(r.row0), r.row(r.row0 + r.rows - 1), lo, hi);
}
// A short chunk: its pages, its first part and their number.
struct FewParts { int lo, hi, first, parts; };
__device__ __forceinline__ FewParts few_parts(const PagedAttnArgs& a, const PagedSeq& q) {
    FewParts f;
    page_range(a, q, 0, q.n - 1, f.lo, f.hi);
    f.first = f.lo >> a.part_shift;
    f.parts = ((f.hi - 1) >> a.part_shift) - f.first + 1;
    return f;
}

// ------------------------------------------------------------------ short chunks
// Where a part of rows row0 .. of a short chunk goes.
template <int DH>
__device__ __forceinline__ float* few_part(const PagedAttnArgs& a, const Rows& r, int part) {
    return a.part + ((((size_t)r.b * a.Hkv + r.h) * a.max_parts + part) * (kPagedFewRows / 32) + r.row0 / 32) * kPartFloats<DH>;
}

// Rows (at most 32) over pages lo .. hi - 1 of part sp (of `parts`, the first being part sp0).
template <typename T, int DH>
__device__ __forceinline__ void few_rows(const PagedAttnArgs& a, const Rows& r, int lo, int hi, int sp, int sp0, int parts,
                                         unsigned char* smem, int wave, int lane) {
    using P = PageTile<T, DH>;
    constexpr int DT = DH / 32, QUADS = 4 * DT;
    RowWave<T, DH, 1, true> w;
    w.clear();
    const Sight see = sight_of<T, DH>(a, r, 0, lane);
    const int begin = sp << a.part_shift;
    const int from = max(lo, begin), to = min(hi, begin + (1 << a.part_shift));
    const int first = begin + (from - begin + 3 - wave) / kWaves * kWaves + wave;   // this wave's first page
    const int cnt = first < to ? (to - first + kWaves - 1) / kWaves : 0;
    unsigned char* s_k = smem + wave * P::BLK;
    unsigned char* s_v = s_k + P::HALF;
    if (cnt > 0) {
        const size_t page_bytes = (size_t)a.Hkv * P::HALF;
        const unsigned char* kb = reinterpret_cast<const unsigned char*>(a.kp) + (size_t)r.h * P::HALF;
        const unsigned char* vb = reinterpret_cast<const unsigned char*>(a.vp) + (size_t)r.h * P::HALF;
        const Fetch<T, DH, DH * P::E> fk(lane);
        const Fetch<T, DH, 32 * P::E> fv(lane);
        int ids = 0;   // lane j: the page of this wave's block j of 64
        bool bad = false;
        auto load_ids = [&](int i0) {
            bool ok = true;
            if (i0 + lane < cnt) ids = page_of(a.seq, r.b, first + (i0 + lane) * kWaves, ok);
            bad |= !ok;
        };
        load_ids(0);
        w.load_q(q_row<T, DH>(a, r, lane & 31), lane);
        __builtin_amdgcn_sched_barrier(0);
        int id = __builtin_amdgcn_readlane(ids, 0);
        fk.template pieces<P::PIECES, 2>(kb + (size_t)id * page_bytes, s_k, 0);
        fv.template pieces<P::PIECES, 2>(vb + (size_t)id * page_bytes, s_v, 0);
        w.have_q();
        const PageRead<T, DH> rd(smem, wave * P::BLK, lane);
        for (int i = 0; i < cnt; ++i) {
            const int blk = first + i * kWaves;
            const bool more = i + 1 < cnt, masked = 32 * blk + 31 > see.all_last || 32 * blk < see.all_first;
            f32x16_t s[1];
            Weights<T, true> p[1];
            wait_loads<P::PIECES>();   // K; V's are behind
            Frag<T> f[DH / 16];
            rd.template k<0>(f);
            if constexpr (sizeof(T) == 4) wait_lds();
            if (more) {
                if (((i + 1) & 63) == 0) load_ids(i + 1);
                id = __builtin_amdgcn_readlane(ids, (i + 1) & 63);
                fk.template pieces<P::PIECES, 2>(kb + (size_t)id * page_bytes, s_k, 0);
            }
            w.scores(s[0], f);
            w.weigh(s, p, blk, to, masked, see, a.scale, lane);
            if (more) wait_loads<P::PIECES>();   // V; the next K's are behind
            else wait_loads<0>();
            rd.template v<0>(f);
            if constexpr (sizeof(T) == 4) wait_lds();
            if (more) fv.template pieces<P::PIECES, 2>(vb + (size_t)id * page_bytes, s_v, 0);
            w.weighted(p[0], f, blk, to, masked, see, lane);
        }
        if (bad) atomicOr(a.seq.err, 1);
    }
    // the waves' results, in their pieces of LDS, joined in wave order
    float (*s_base)[32] = reinterpret_cast<float (*)[32]>(smem + kWaves * P::BLK), (*s_sum)[32] = s_base + kWaves;
    f32x4_t* own = reinterpret_cast<f32x4_t*>(smem + wave * P::BLK);
    static_assert(QUADS * 1024 <= P::BLK, "a wave's O fits its page");
    const float sum = w.whole_sum();
    if (lane < 32) {
        s_base[wave][lane] = w.base;
        s_sum[wave][lane] = sum;
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            own[(dt * 4 + j) * 64 + lane] = f32x4_t{w.o[dt][4 * j], w.o[dt][4 * j + 1], w.o[dt][4 * j + 2], w.o[dt][4 * j + 3]};
    __syncthreads();
    const int i = lane & 31;
    float wt[kWaves], top = -INFINITY, den = 0.f;
#pragma unroll
    for (int k = 0; k < kWaves; ++k) top = fmaxf(top, s_base[k][i]);
#pragma unroll
    for (int k = 0; k < kWaves; ++k) {
        const float m = s_base[k][i];
        wt[k] = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        den = fmaf(wt[k], s_sum[k][i], den);
    }
    const __amdgpu_buffer_rsrc_t rs = buf_rsrc(few_part<DH>(a, r, sp - sp0), kPartFloats<DH> * 4);
    const float inv = den == 0.f ? 0.f : 1.0f / den;
    for (int qd = wave; qd < QUADS; qd += kWaves) {
        f32x4_t acc = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < kWaves; ++k) {
            const f32x4_t v = reinterpret_cast<const f32x4_t*>(smem + k * P::BLK)[qd * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = fmaf(v[e], wt[k], acc[e]);
        }
        if (i >= r.rows) continue;
        const int d = 8 * qd + 4 * (lane >> 5);   // quad 4 dt + j: columns 32 dt + 8 j + 4 (lane / 32)
        if (parts == 1) {
            store_row<T, DH>(a, r, i, d, acc * inv);
        } else {
            put4(rs, part_quad<DH>(r.rows, i, d / 4), acc);
            if (qd == 0 && lane < 32) put4(rs, part_quad<DH>(r.rows, i, DH / 4), f32x4_t{top, den, 0.f, 0.f});
        }
    }
}

// Workgroup `wg` of `wgs` takes pieces wg, wg + wgs, ... of the short chunks': per sequence its parts, row tiles, key heads.
template <typename T, int DH>
__device__ __forceinline__ void few_work(const PagedAttnArgs& a, int wg, int wgs, unsigned char* smem, int wave, int lane) {
    const int group = a.H / a.Hkv;
    auto pieces = [&](const PagedSeq& q) {
        return q.n == 0 || q.n * (long)group > kPagedFewRows ? 0 : few_parts(a, q).parts * ((q.n * group + 31) / 32) * a.Hkv;
    };
    for (int want = wg;; want += wgs) {
        const Found f = find_piece(a.seq, want, lane, pieces);
        if (!f.ok) return;
        const FewParts fp = few_parts(a, f.seq);
        const int two = f.seq.n * group > 32, k = f.k / a.Hkv;   // 32 rows or twice
        Rows r{f.b, f.k - k * a.Hkv, (k & two) * 32, 0, group, f.seq, (65535u + group) / group};
        r.rows = min(32, f.seq.n * group - r.row0);
        few_rows<T, DH>(a, r, fp.lo, fp.hi, fp.first + (k >> two), fp.first, fp.parts, smem, wave, lane);
        if (a.few_once) return;
        __syncthreads();   // smem is free
    }
}
static_assert(kPagedFewRows == 64, "a short chunk is 32 rows or twice");

// ------------------------------------------------------------------ tiles
// Where rows 32 sub .. of a tile's part go.
template <int DH>
__device__ __forceinline__ float* tile_part(const PagedAttnArgs& a, int part, int sub) {
    return a.part + a.tile_part + ((size_t)part * (kPagedTileRows / 32) + sub) * kPartFloats<DH>;
}

// Piece `want` of the tiles: a tile and key head (numbered `slot` among them) and one of its parts, pages lo .. hi - 1 of it.
struct TileWork { bool ok; Rows r; int slot, splits, sp, parts, lo, hi; };
__device__ __forceinline__ TileWork tile_work(const PagedAttnArgs& a, int want, bool by_slot, int lane) {
    const int group = a.H / a.Hkv;
    auto tiles_of = [&](const PagedSeq& q) {
        return q.n * (long)group > kPagedFewRows ? (q.n * group + kPagedTileRows - 1) / kPagedTileRows : 0;
    };
    TileWork t{};
    t.splits = paged_tile_splits(count_pieces(a.seq, lane, tiles_of), a.Hkv);
    const int each = by_slot ? 1 : t.splits;
    const Found f = find_piece(a.seq, want, lane, [&](const PagedSeq& q) { return tiles_of(q) * each * a.Hkv; });
    if (!f.ok) return t;
    const int h = f.k % a.Hkv, nth = f.k / a.Hkv / each;
    t.sp = f.k / a.Hkv % each;
    t.slot = (want - f.k) / each + nth * a.Hkv + h;
    t.r = Rows{f.b, h, (tiles_of(f.seq) - 1 - nth) * kPagedTileRows, 0, group, f.seq, 0};   // the longest first
    t.r.rows = min(kPagedTileRows, f.seq.n * group - t.r.row0);
    page_range(a, t.r, t.lo, t.hi);
    const int per = max((t.hi - t.lo + t.splits - 1) / t.splits, 4);
    t.parts = (t.hi - t.lo + per - 1) / per;
    t.ok = t.sp < t.parts;
    t.lo += t.sp * per;
    t.hi = min(t.hi, t.lo + per);
    return t;
}

template <typename T, int DH, bool FINE>
__device__ __forceinline__ void tile_rows(const PagedAttnArgs& a, int wg, unsigned char* smem, int wave, int lane) {
    using P = PageTile<T, DH>;
    constexpr int DT = DH / 32, NL = P::PIECES / 2;   // 1 KiB loads of a wave per step, of K and of V
    const TileWork t = tile_work(a, wg, false, lane);
    if (!t.ok) return;
    const Rows r = t.r;
    const int b = r.b, h = r.h, lo = t.lo, hi = t.hi, parts = t.parts;
    const int w0 = 32 * wave;
    const Sight see = sight_of<T, DH>(a, r, w0, lane);
    // pages this wave's rows see
    int wlo = lo, whi = lo;
    if (w0 < r.rows) {
        Rows x = r;
        x.row0 += w0;
        x.rows = min(32, r.rows - w0);
        page_range(a, x, wlo, whi);
    }
    RowWave<T, DH, 2, FINE> w;
    w.clear();
    const size_t page_bytes = (size_t)a.Hkv * P::HALF;
    const unsigned char* kb = reinterpret_cast<const unsigned char*>(a.kp) + (size_t)h * P::HALF;
    const unsigned char* vb = reinterpret_cast<const unsigned char*>(a.vp) + (size_t)h * P::HALF;
    // waves 0, 1 load a step's first page, waves 2, 3 its second, half of K and of V each
    const int part0 = (wave & 1) * NL;
    const Fetch<T, DH, DH * P::E> fk(lane);
    const Fetch<T, DH, 32 * P::E> fv(lane);
    int ids = 0;
    bool bad = false;
    auto load_ids = [&](int i0) {   // of pages lo + i0 + lane
        bool ok = true;
        if (lo + i0 + lane < hi) ids = page_of(a.seq, b, lo + i0 + lane, ok);
        bad |= !ok;
    };
    const int nstep = (hi - lo + 1) / 2;
    auto request = [&](int i) {   // a page past the last repeats it: in bounds, weighed with nothing
        if ((i & 31) == 0) load_ids(2 * i);
        const int j = min(2 * i + (wave >> 1), hi - lo - 1);
        const size_t off = (size_t)__builtin_amdgcn_readlane(ids, j & 63) * page_bytes;
        unsigned char* dst = smem + (i & 1) * 2 * P::BLK + (wave >> 1) * P::BLK;
        fk.template pieces<NL, 0>(kb + off, dst, part0);
        fv.template pieces<NL, 0>(vb + off, dst + P::HALF, part0);
    };
    w.load_q(q_row<T, DH>(a, r, w0 + (lane & 31)), lane);
    __builtin_amdgcn_sched_barrier(0);
    request(0);
    w.have_q();
    PageRead<T, DH> rd(smem, 0, lane);
    for (int i = 0; i < nstep; ++i) {
        // this wave's loads of step i have landed; after the barrier everyone's have, and nobody still reads the other stage
        wait_lds();
        wait_loads<0>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (i + 1 < nstep) request(i + 1);
        const int blk = lo + 2 * i;
        if (blk < whi && blk + 2 > wlo) {
            const bool masked = 32 * blk + 63 > see.all_last || 32 * blk < see.all_first || blk + 2 > hi;
            f32x16_t s[2];
            Weights<T, FINE> p[2];
            Frag<T> f[DH / 16];
            rd.template k<0>(f);
            w.scores(s[0], f);
            rd.template k<P::BLK>(f);
            w.scores(s[1], f);
            w.weigh(s, p, blk, hi, masked, see, a.scale, lane);
            rd.template v<0>(f);
            w.weighted(p[0], f, blk, hi, masked, see, lane);
            rd.template v<P::BLK>(f);
            w.weighted(p[1], f, blk + 1, hi, masked, see, lane);
        }
        rd.move(i & 1 ? -2 * P::BLK : 2 * P::BLK);
    }
    if (bad) atomicOr(a.seq.err, 1);
    const float den = w.whole_sum(), inv = den == 0.f ? 0.f : 1.0f / den;
    const __amdgpu_buffer_rsrc_t rs = buf_rsrc(tile_part<DH>(a, t.slot * t.splits + t.sp, wave), kPartFloats<DH> * 4);
    const int own = min(32, r.rows - w0), i = lane & 31;   // rows of this wave
    if (i >= own) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const f32x4_t v = f32x4_t{w.o[dt][4 * j], w.o[dt][4 * j + 1], w.o[dt][4 * j + 2], w.o[dt][4 * j + 3]};
            const int d = 32 * dt + 8 * j + 4 * (lane >> 5);
            if (parts == 1) store_row<T, DH>(a, r, w0 + i, d, v * inv);
            else put4(rs, part_quad<DH>(own, i, d / 4), v);
        }
    if (parts > 1 && lane < 32) put4(rs, part_quad<DH>(own, i, DH / 4), f32x4_t{w.base, den, 0.f, 0.f});
}

// ------------------------------------------------------------------ joining parts
// Parts 0 .. n - 1 of rows (at most 32) joined by log-sum-exp, part p's at part + p * stride quads; columns
// of slice `slice` of `slices`.  Even parts in order, odd ones in order, then both: half a wave each.  Parts that a row sees
// nothing of add zeros, and the sums are taken over lanes that stand for the sequence's parts from its beginning (the first
// here is its part `first`): a row's bits do not depend on which parts the chunk's other rows see.
template <typename T, int DH>
__device__ __forceinline__ void join_parts(const PagedAttnArgs& a, const Rows& r, const f32x4_t* part, int stride, int first, int n,
                                           int slice, int slices, float (*s_w)[32]) {
    constexpr int D4 = DH / 4;
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    static_assert(kPagedMaxParts <= 64, "a lane for each part");
    // a row's bases and sums in the lanes of a wave; the waves take the rows in turn
    const int p = lane - first;
    const bool mine = p >= 0 && p < n;
    for (int i = tid / 64; i < r.rows; i += 4) {
        const f32x4_t v = part[(size_t)min(max(p, 0), n - 1) * stride + D4 * r.rows + i];
        const float m = mine ? v[0] : -INFINITY, top = across_wave(m, OpMax());
        const float w = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
        const float den = across_wave(mine ? w * v[1] : 0.f, OpSum());
        if (mine) s_w[p][i] = w * (den == 0.f ? 0.f : 1.0f / den);
    }
    __syncthreads();
    const int quads = r.rows * (D4 / slices);
    const int e0 = tid / 64 * 32 + (lane & 31);
    auto join = [&](auto ahead) {   // so many parts' loads of a half wave under way at once, of 16 / AHEAD quads
        constexpr int AHEAD = decltype(ahead)::value, Q = 16 / AHEAD > 8 ? 8 : 16 / AHEAD;
        for (int eb = e0; eb - e0 < quads; eb += 128 * Q) {
            f32x4_t acc[Q];
#pragma unroll
            for (int k = 0; k < Q; ++k) acc[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
            for (int p0 = half; p0 < n; p0 += 2 * AHEAD) {
                f32x4_t u[Q][AHEAD];
#pragma unroll
                for (int k = 0; k < Q; ++k)
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j)   // past the last: the last again, not used
                        u[k][j] = part[(size_t)min(p0 + 2 * j, n - 1) * stride + slice * (D4 / slices) * r.rows + min(eb + 128 * k, quads - 1)];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int k = 0; k < Q; ++k)
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j) {
                        const bool in = p0 + 2 * j < n;
                        const float w = s_w[min(p0 + 2 * j, n - 1)][min(eb + 128 * k, quads - 1) % r.rows];
#pragma unroll
                        for (int c = 0; c < 4; ++c) acc[k][c] = in ? fmaf(w, u[k][j][c], acc[k][c]) : acc[k][c];
                    }
            }
#pragma unroll
            for (int k = 0; k < Q; ++k) {
                const int e = eb + 128 * k;
                f32x4_t out;
#pragma unroll
                for (int c = 0; c < 4; ++c) out[c] = acc[k][c] + __shfl_xor(acc[k][c], 32, 64);
                if (half == 0 && e < quads) store_row<T, DH>(a, r, e % r.rows, 4 * (slice * (D4 / slices) + e / r.rows), out);
            }
        }
    };
    if (n <= 2) join(std::integral_constant<int, 1>());
    else if (n <= 8) join(std::integral_constant<int, 4>());
    else join(std::integral_constant<int, 16>());
}

// Workgroups of short chunks, `slices` for each sequence, key head and one of `subs` times 32 rows; then of tiles, four for
// each 32 rows of one.
template <typename T, int DH>
__global__ void __launch_bounds__(256) paged_join_kernel(PagedAttnArgs a, int few, int subs, int slices) {
    __shared__ float s_w[kPagedMaxParts][32];
    const int lane = threadIdx.x & 63;
    int x = (int)blockIdx.x;
    const int group = a.H / a.Hkv;
    if (x < few) {
        const int slice = x % slices;
        x /= slices;
        const int sub = x % subs;
        x /= subs;
        const int b = x / a.Hkv;
        Rows r{b, x - b * a.Hkv, sub * 32, 0, group, load_seq(a.seq, b), (65535u + group) / group};
        const int rows = r.seq.n * group;
        if (rows <= r.row0 || rows > kPagedFewRows) return;
        const FewParts fp = few_parts(a, r.seq);
        if (fp.parts < 2) return;
        r.rows = min(32, rows - r.row0);
        join_parts<T, DH>(a, r, reinterpret_cast<const f32x4_t*>(few_part<DH>(a, r, 0)), kPagedFewRows / 32 * kPartFloats<DH> / 4,
                          fp.first, fp.parts, slice, slices, s_w);
        return;
    }
    x -= few;
    const int sub = x % (kPagedTileRows / 32);
    const TileWork t = tile_work(a, x / (kPagedTileRows / 32), true, lane);
    if (!t.ok || t.parts < 2 || 32 * sub >= t.r.rows) return;
    Rows r = t.r;
    r.row0 += 32 * sub;
    r.rows = min(32, r.rows - 32 * sub);
    join_parts<T, DH>(a, r, reinterpret_cast<const f32x4_t*>(tile_part<DH>(a, t.slot * t.splits, sub)),
                      kPagedTileRows / 32 * kPartFloats<DH> / 4, 0, t.parts, 0, 1, s_w);
}

// ------------------------------------------------------------------ the launch
template <typename T, int DH, bool TILES, bool FINE>
__global__ void __launch_bounds__(64 * kWaves, sizeof(T) * DH > 256 ? 1 : 2) paged_attn_kernel(PagedAttnArgs a) {
    __shared__ __align__(1024) unsigned char smem[kLdsBytes<T, DH>];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (blockIdx.x == 0 && wave == 0) check_seqs(a.seq, lane);
    int few = (int)blockIdx.x;
    if constexpr (TILES) {
        if (few < a.tile_wgs) {
            tile_rows<T, DH, FINE>(a, few, smem, wave, lane);
            return;
        }
        few -= a.tile_wgs;
    }
    few_work<T, DH>(a, few, a.few_wgs, smem, wave, lane);
}

// ------------------------------------------------------------------ plans
PagedPlan plan_paged(int Hkv, int max_batch, int max_ctx) {
    PagedPlan p{};
    const long cap = std::max(1, (max_ctx + kPage - 1) / kPage), pairs = (long)Hkv * max_batch;
    // pages of a part: a full cache in about 1024 parts, four for each wave at the least.  us with 4, 8 and 16 at the least: a
    // token over 1500 slots of 8 key heads 15.1, 14.1, 15.1; 6 tokens of 4 sequences over 3000 37, 26, 20; 64 tokens over 500
    // slots 39, 39, 26; 11 rows of 4 sequences over 1500 slots of 32 heads 33, 31, 28.  512 to 4096 parts, 64 tokens over 4000
    // slots: 167, 167, 173, 181.  (All on handles of the call's own size.  Parts follow the handle, so that a row's bits do
    // not follow the batch, and a handle for more has longer ones: one for 64 sequences of 16384 slots and more takes a token
    // over 2000, 8000 and 16000 slots of 8 key heads in 23.5, 26.9 and 28.4 us, one of the call's size in 14.3, 14.7 and 16.9;
    // 6 rows of 4 sequences over 3000 slots in 30, 19.4.)
    // (A power of two, as the kernels shift, near the number, and enough of them for a full cache in kPagedMaxParts.)
    const long want = std::min<long>((cap * pairs + 1023) / 1024, 64), least = (cap + kPagedMaxParts - 1) / kPagedMaxParts;
    p.part_shift = 4;
    while ((2l << p.part_shift) * 3 <= want * 4 || (1l << p.part_shift) < least) ++p.part_shift;
    const long per = 1l << p.part_shift;
    p.max_parts = (int)((cap + per - 1) / per);
    return p;
}

// tiles of a call and key head, at most
static long most_tiles(int H, int Hkv, long rows, int B) { return rows * (H / Hkv) / kPagedTileRows + B; }

void plan_paged_call(PagedPlan& p, int H, int Hkv, int B, int rows, int max_q, int max_len) {
    const int group = H / Hkv;
    p.tile_wgs = 0;
    if ((long)max_q * group > kPagedFewRows)
        p.tile_wgs = (int)std::min<long>(std::max<long>(most_tiles(H, Hkv, rows, B) * Hkv, kPagedTileParts), 0x7FFFFFFF);
    const int tiles = (int)std::min<long>(((long)max_q * group + 31) / 32, kPagedFewRows / 32);
    const long parts = ((long)max_len + ((long)kPage << p.part_shift) - 1) / ((long)kPage << p.part_shift);
    p.call_parts = (int)parts;
    const long pieces = parts * B * tiles * Hkv;
    p.few_wgs = (int)std::max<long>(1, std::min<long>(pieces, 2048));
    p.few_once = pieces <= p.few_wgs;
}

size_t paged_part_floats(const PagedPlan& p, int H, int Hkv, int head_dim, int max_batch, int max_rows, size_t* tile_part) {
    *tile_part = p.max_parts > 1 ? (size_t)max_batch * Hkv * p.max_parts * kPagedFewRows * (head_dim + 4) : 0;
    return *tile_part + ((long)max_rows * (H / Hkv) > kPagedFewRows ? (size_t)kPagedTileParts * kPagedTileRows * (head_dim + 4) : 0);
}

template <typename T, int DH>
static hipError_t launch_dh(const PagedPlan& p, const PagedAttnArgs& a, hipStream_t s) {
    const unsigned grid = (unsigned)p.tile_wgs + (unsigned)p.few_wgs;
    auto kern = p.tile_wgs ? paged_attn_kernel<T, DH, true, false> : paged_attn_kernel<T, DH, false, false>;
    if constexpr (sizeof(T) == 2) {
        if (p.tile_wgs && a.out_f32) kern = paged_attn_kernel<T, DH, true, true>;
    }
    hipLaunchKernelGGL(kern, dim3(grid), dim3(64 * kWaves), 0, s, a);
    // tiles in several parts are kPagedTileParts / 2 at the most, with key heads
    const int subs = (long)a.seq.max_q * (a.H / a.Hkv) > 32 ? kPagedFewRows / 32 : 1, slices = p.call_parts > 8 ? 4 : 1;
    const int few = p.call_parts > 1 ? a.seq.B * a.Hkv * subs * slices : 0;
    const int join = few + (p.tile_wgs ? kPagedTileParts / 2 * (kPagedTileRows / 32) : 0);
    if (join) hipLaunchKernelGGL((paged_join_kernel<T, DH>), dim3((unsigned)join), dim3(256), 0, s, a, few, subs, slices);
    return hipGetLastError();
}

hipError_t launch_paged_attention(int dtype, int head_dim, const PagedPlan& p, const PagedAttnArgs& a, hipStream_t s) {
    const PagedSeqs& q = a.seq;
    const int group = a.Hkv > 0 ? a.H / a.Hkv : 0;
    if (group < 1 || a.H % a.Hkv || q.B < 1 || q.rows < 0 || q.pages_ld < 1 || q.n_pages < 1 || q.max_q < 0 || q.max_len < 0 ||
        q.max_len > (long)q.pages_ld * kPage || !q.start || !q.len || !q.pages || !q.err || !a.kp || !a.vp || !a.q || !a.out ||
        (a.mask && (q.max_q > 64 || a.window)) || a.window < 0 || !(a.scale > 0.f) || a.ldq % 8 || a.ldo % 4 || p.part_shift < 0 || p.part_shift > 20 ||
        a.part_shift != p.part_shift || a.few_once != p.few_once || a.tile_wgs != p.tile_wgs || a.few_wgs != p.few_wgs || a.max_parts != p.max_parts ||
        p.few_wgs < 1 || p.max_parts > kPagedMaxParts ||
        (long)p.tile_wgs + p.few_wgs > 0xFFFFFFFFl / (64 * kWaves) || q.max_len > ((long)p.max_parts * kPage << p.part_shift) || p.call_parts < 1 ||
        ((long)p.call_parts * kPage << p.part_shift) < q.max_len || (long)q.B * a.Hkv > kPagedMaxPairs ||
        ((long)p.max_parts << p.part_shift) > 0x7FFFFFFFl / kPage || !a.part ||
        ((long)q.max_q * group > kPagedFewRows && p.tile_wgs < std::max<long>(most_tiles(a.H, a.Hkv, q.rows, q.B) * a.Hkv, kPagedTileParts)))
        return hipErrorInvalidValue;
    if (dtype == 1) {
        if (head_dim == 128) return launch_dh<uint16_t, 128>(p, a, s);
        if (head_dim == 64) return launch_dh<uint16_t, 64>(p, a, s);
    } else {
        if (head_dim == 128) return launch_dh<float, 128>(p, a, s);
        if (head_dim == 64) return launch_dh<float, 64>(p, a, s);
    }
    return hipErrorInvalidValue;
}

}  // namespace sdsat
