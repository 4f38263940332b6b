// Appending to a paged cache: the new tokens' rows q | k | v, as a linear layer leaves them, become queries for the
// attention and keys and values in the pages of their sequences.
//
// For a query or key head x of Dh columns of the token at position p, in float:
//   x <- gain o x / sqrt(mean(x^2) + eps)                        (where a gain is given)
//   (a, c) <- (a cos w - c sin w, c cos w + a sin w) * mscale    for the pairs j < R / 2 of the R rotated columns,
//                                                                w = p f_j; pairs (j, j + R/2) or (2j, 2j + 1)
// and one rounding to the cache's type.  Turns p f_j / 2 pi are formed in double and reduced to an eighth of one before
// they become float: positions of 10^6 and more lose nothing (the angle is off by 2.3e-8 at most).
//
// A workgroup has the tokens of one page (up to 32) and a slice of the heads.  Eight columns of a head are one lane's:
// 4 pairs' both sides, so that a rotation needs no exchange, and a lane that keeps its token while it goes through the
// heads forms its 4 sines once; U heads' columns are on their way at once.  K's rows are written whole.  V's lie transposed
// in a page (32 slots beside each other for one column): pages of more than kScatterTokens new tokens are turned in LDS and
// written 16 bytes at a time where all of a chunk's slots are new; fewer tokens are written element by element.
// Bound by memory, and by latency for single tokens: 4 prompts of 2047 tokens, 48 heads of 128 in bf16 (201 MB) 54 us,
// 3.7 TB/s (a large copy 4.9; without the norms 51, one head at a time 73); one token of 64 sequences 7.8 us, a block
// of 6 tokens of the tiny decoder 5.2 (called from Python 9.0 and 6.8: the host's time; a launch alone is 4.4).
#include <algorithm>

#include "paged_device.h"

namespace sdsat {

static constexpr int kAppendThreads = 256;
static constexpr int kScatterTokens = 8;
static constexpr int kTurned = 2;   // V's heads turned at once

// 4 neighbouring columns, as they are stored
template <typename T>
struct Raw4 {
    uint2 v;
    __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ void get(float* x) const {
        x[0] = __uint_as_float(v.x << 16);
        x[1] = __uint_as_float(v.x & 0xFFFF0000u);
        x[2] = __uint_as_float(v.y << 16);
        x[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
};
template <>
struct Raw4<float> {
    f32x4_t v;
    __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const f32x4_t*>(p); }
    __device__ __forceinline__ void get(float* x) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = v[i];
    }
};
template <typename T>
__device__ __forceinline__ void load4(const T* p, float* x) {
    Raw4<T> r;
    r.load(p);
    r.get(x);
}
template <typename T>
__device__ __forceinline__ void store4(T* p, const float* x) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<f32x4_t*>(p) = f32x4_t{x[0], x[1], x[2], x[3]};
    else *reinterpret_cast<uint2*>(p) = uint2{f32x2_to_bf16x2(x[0], x[1]), f32x2_to_bf16x2(x[2], x[3])};
}

// The sum over the 8 or 16 neighbouring lanes of a head.
template <int GL>
__device__ __forceinline__ float across_head(float v) {
    v = across_quads(v, OpSum());
    v += lane_perm<0x141>(v);   // mirrored within 8 lanes
    if constexpr (GL == 16) v += lane_perm<0x140>(v);
    return v;
}
// 1 / sqrt(x) within a step; the instruction takes subnormal numbers for zero
__device__ __forceinline__ float inverse_root(float x) {
    const bool tiny = x < 0x1p-100f;
    const float r = __builtin_amdgcn_rsqf(tiny ? x * 0x1p100f : x);
    return tiny ? r * 0x1p50f : r;
}

// cos and sin of 2 pi t
__device__ __forceinline__ void turn(double t, float& c, float& s) {
    const double f = t - rint(t), q = rint(4.0 * f);   // [-1/2, 1/2]; quarters, -2 .. 2
    float s0, c0;
    sincospif((float)(2.0 * f - 0.5 * q), &s0, &c0);   // an eighth of a turn at most
    const int k = (int)q & 3;
    const float a = (k & 1) ? s0 : c0, b = (k & 1) ? c0 : s0;
    c = (k == 1 || k == 2) ? -a : a;
    s = (k >= 2) ? -b : b;
}

template <typename TX, typename T, int DH>
__global__ void __launch_bounds__(kAppendThreads) paged_append_kernel(PagedAppendArgs a, int slices, int slice_heads, int v_heads) {
    constexpr int U = 4;
    constexpr int GL = DH / 8, NG = kAppendThreads / GL;   // lanes of a head, heads at a time
    constexpr int VLD = DH + 16 / (int)sizeof(T);          // a row of V in LDS, elements: four of them lie 16 banks apart
    __shared__ __align__(16) T s_v[kTurned * kPage * VLD];
    const int lane = threadIdx.x & 63;
    if (blockIdx.x == 0 && threadIdx.x < 64) check_seqs(a.seq, lane);
    const int pieces = (int)gridDim.x / slices, slice = (int)blockIdx.x / pieces, piece = (int)blockIdx.x % pieces;
    const PieceSeq found = seq_of_piece(a.seq, piece, 1, kPage, 2, lane);
    const int b = __builtin_amdgcn_readfirstlane(found.b);
    const PagedSeq seq = found.seq;
    const int nth = piece - piece_begin(seq.start, 1, kPage, 2, b);
    if (!seq.ok || nth < 0) return;
    const int page = seq.len / kPage + nth;
    const int s0 = max(seq.len, page * kPage), s1 = min(seq.len + seq.n, (page + 1) * kPage);   // new slots of this page
    if (s0 >= s1) return;
    bool ok;   // looked at where something is stored: the rows' loads do not wait for the page's number
    const int id = page_of(a.seq, b, page, ok);
    const int tokens = s1 - s0, row0 = seq.start + s0 - seq.len;
    const int grp = (int)threadIdx.x / GL, l = (int)threadIdx.x % GL;
    // token-wise groups for full pages, head-wise ones for single tokens
    int tp = 1;
    while (tp < NG && tp < tokens) tp *= 2;
    const int hp = NG / tp, tok = grp % tp;
    const TX* x = reinterpret_cast<const TX*>(a.x);
    const int qk = a.H + a.Hkv, qk_slices = (qk + slice_heads - 1) / slice_heads;
    T* kp = reinterpret_cast<T*>(a.kp) + (size_t)id * a.Hkv * kPage * DH;
    T* vp = reinterpret_cast<T*>(a.vp) + (size_t)id * a.Hkv * kPage * DH;
    if (slice < qk_slices) {
        const int h0 = slice * slice_heads, h1 = min(h0 + slice_heads, qk);
        // this lane's columns: 4 at c0, 4 at c1, 4 pairs of them rotated
        const bool turned = 8 * l < a.rot;
        const int c0 = a.interleaved || !turned ? 8 * l : 4 * l;
        const int c1 = a.interleaved || !turned ? 8 * l + 4 : a.rot / 2 + 4 * l;
        float gq[8], gk[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) gq[i] = gk[i] = 1.f;
        if (a.q_gain) {
#pragma unroll
            for (int i = 0; i < 8; ++i) gq[i] = a.q_gain[(i < 4 ? c0 : c1 - 4) + i];
        }
        if (a.k_gain) {
#pragma unroll
            for (int i = 0; i < 8; ++i) gk[i] = a.k_gain[(i < 4 ? c0 : c1 - 4) + i];
        }
        for (int t = tok; t < tokens; t += tp) {
            const int row = row0 + t;
            const int pos = a.pos ? a.pos[row] : s0 + t;
            float cs[4], sn[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                cs[j] = 1.f;
                sn[j] = 0.f;
                if (turned) {
                    turn((double)pos * a.turns[4 * l + j], cs[j], sn[j]);
                    cs[j] *= a.mscale;
                    sn[j] *= a.mscale;
                }
            }
            const TX* src = x + (size_t)row * a.ldx;
            for (int h = h0 + grp / tp; h < h1; h += U * hp) {
                Raw4<TX> raw[U][2];   // U heads under way
#pragma unroll
                for (int u = 0; u < U; ++u) {   // past the last: the last again, not used
                    const TX* head = src + (size_t)min(h + u * hp, h1 - 1) * DH;
                    raw[u][0].load(head + c0);
                    raw[u][1].load(head + c1);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int hh = h + u * hp;
                    if (hh >= h1) continue;
                    const bool is_q = hh < a.H;
                    float v[8];
                    raw[u][0].get(v);
                    raw[u][1].get(v + 4);
                    if (is_q ? a.q_gain != nullptr : a.k_gain != nullptr) {
                        float ss = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) ss = fmaf(v[i], v[i], ss);
                        const float inv = inverse_root(across_head<GL>(ss) * (1.0f / DH) + a.eps);
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = v[i] * inv * (is_q ? gq[i] : gk[i]);
                    }
                    if (turned) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float& p = v[a.interleaved ? 2 * j : j];
                            float& r = v[a.interleaved ? 2 * j + 1 : 4 + j];
                            const float m = p * cs[j] - r * sn[j], w = r * cs[j] + p * sn[j];
                            p = m;
                            r = w;
                        }
                    }
                    T* dst = is_q ? reinterpret_cast<T*>(a.qout) + (size_t)row * a.ldq + (size_t)hh * DH
                                  : kp + ((size_t)(hh - a.H) * kPage + (s0 + t) % kPage) * DH;
                    if (!is_q && !ok) continue;
                    store4(dst + c0, v);
                    store4(dst + c1, v + 4);
                }
            }
        }
        if (!ok && slice == 0 && threadIdx.x == 0) atomicOr(a.seq.err, 1);
        return;
    }
    const int h0 = (slice - qk_slices) * v_heads, h1 = min(h0 + v_heads, a.Hkv);
    if (tokens <= kScatterTokens) {
        for (int t = tok; t < tokens; t += tp)
            for (int h = h0 + grp / tp; h < h1; h += hp) {
                const TX* src = x + (size_t)(row0 + t) * a.ldx + (size_t)(qk + h) * DH + 8 * l;
                float v[8];
                load4(src, v);
                load4(src + 4, v + 4);
                T* dst = vp + ((size_t)h * DH + 8 * l) * kPage + vperm((s0 + t) % kPage);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (ok) dst[i * kPage] = to_elem<T>(v[i]);
            }
        return;
    }
    // kTurned heads at a time: rows into LDS as they are, columns out of it, neighbouring lanes a column's chunks
    constexpr int CH = 16 / (int)sizeof(T), PER_COL = 32 / CH;   // elements of a chunk, chunks of a column
    for (int hb = h0; hb < h1; hb += kTurned) {
        const int heads = min(kTurned, h1 - hb);
        if (hb > h0) __syncthreads();
        for (int t = grp; t < tokens; t += NG) {
            const TX* src = x + (size_t)(row0 + t) * a.ldx + (size_t)(qk + hb) * DH + 8 * l;
            Raw4<TX> raw[kTurned][2];
#pragma unroll
            for (int u = 0; u < kTurned; ++u) {
                raw[u][0].load(src + (size_t)min(u, heads - 1) * DH);
                raw[u][1].load(src + (size_t)min(u, heads - 1) * DH + 4);
            }
#pragma unroll
            for (int u = 0; u < kTurned; ++u) {
                float v[8];
                raw[u][0].get(v);
                raw[u][1].get(v + 4);
                T* dst = s_v + (u * kPage + (s0 + t) % kPage) * VLD + 8 * l;
                store4(dst, v);
                store4(dst + 4, v + 4);
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; ok && i < heads * DH * PER_COL; i += kAppendThreads) {
            const int u = i / (DH * PER_COL), d = i / PER_COL % DH, at = i % PER_COL * CH;
            T* dst = vp + ((size_t)(hb + u) * DH + d) * kPage + at;
            const T* src = s_v + u * kPage * VLD + d;
            // places at .. at + 3 hold slots 16 (at / 4 % 2) + 4 (at / 8) .., the next four those 16 further
            bool all = true;
            T v[CH];
#pragma unroll
            for (int e = 0; e < CH; ++e) {
                const int in = ((at + e) & 4) * 4 + (at + e) / 8 * 4 + (e & 3), slot = page * kPage + in;
                v[e] = src[in * VLD];
                all = all && slot >= s0 && slot < s1;
            }
            if (all) {
                __builtin_memcpy(dst, v, 16);
                continue;
            }
#pragma unroll
            for (int e = 0; e < CH; ++e) {
                const int slot = page * kPage + ((at + e) & 4) * 4 + (at + e) / 8 * 4 + (e & 3);
                if (slot >= s0 && slot < s1) dst[e] = v[e];
            }
        }
    }
}

template <typename TX, typename T>
static hipError_t launch_append_dh(int head_dim, const PagedAppendArgs& a, hipStream_t s) {
    const int pieces = a.seq.rows / kPage + 2 * a.seq.B;
    // heads of a slice: 20, fewer where that leaves compute units idle; V's, which whole pages turn one pair after another,
    // in pairs
    int per = 20;
    while (per > 5 && (long)pieces * ((a.H + a.Hkv + per - 1) / per + (a.Hkv + per - 1) / per) < 1024) per /= 2;
    int pv = a.seq.max_q > kScatterTokens ? kTurned : per;
    if ((long)pieces * (a.Hkv / pv) > 1 << 22) pv = std::max(pv, per);   // a launch's 2^32 threads
    const int slices = (a.H + a.Hkv + per - 1) / per + (a.Hkv + pv - 1) / pv;
    if ((long)pieces * slices > 0xFFFFFFFFl / kAppendThreads) return hipErrorInvalidValue;
    auto kern = head_dim == 128 ? paged_append_kernel<TX, T, 128> : paged_append_kernel<TX, T, 64>;
    hipLaunchKernelGGL(kern, dim3((unsigned)(pieces * slices)), dim3(kAppendThreads), 0, s, a, slices, per, pv);
    return hipGetLastError();
}

__global__ void __launch_bounds__(64) paged_check_kernel(PagedSeqs seq) { check_seqs(seq, threadIdx.x); }

hipError_t launch_paged_check(const PagedSeqs& q, hipStream_t s) {
    if (q.B < 1 || !q.start || !q.len || !q.err) return hipErrorInvalidValue;
    hipLaunchKernelGGL(paged_check_kernel, dim3(1), dim3(64), 0, s, q);
    return hipGetLastError();
}

hipError_t launch_paged_append(int dtype, int x_dtype, int head_dim, const PagedAppendArgs& a, hipStream_t s) {
    const PagedSeqs& q = a.seq;
    if ((head_dim != 64 && head_dim != 128) || q.B < 1 || q.rows < 0 || q.pages_ld < 1 || q.n_pages < 1 || q.max_q < 0 ||
        q.max_len < 0 || q.max_len > (long)q.pages_ld * kPage || !q.start || !q.len || !q.pages || !q.err || !a.kp || !a.vp ||
        !a.x || !a.qout || a.H < 1 || a.Hkv < 1 || a.H % a.Hkv || a.rot < 0 || a.rot > head_dim || a.rot % 8 || a.ldx % 8 ||
        a.ldq % 8)
        return hipErrorInvalidValue;
    if (dtype == 1) return x_dtype == 1 ? launch_append_dh<uint16_t, uint16_t>(head_dim, a, s) : launch_append_dh<float, uint16_t>(head_dim, a, s);
    return x_dtype == 1 ? launch_append_dh<uint16_t, float>(head_dim, a, s) : launch_append_dh<float, float>(head_dim, a, s);
}

}  // namespace sdsat
