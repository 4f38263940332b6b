// Device-side helpers shared by the kernels of the paged cache: a call's sequences, checked, and how workgroups find
// theirs.
#pragma once

#include "device.h"
#include "kernels.h"

namespace sdsat {

// Sequence b of a call: its first row, new tokens and cached ones; none and ok false where its numbers do not fit.
struct PagedSeq { int start, n, len; bool ok; };

__device__ __forceinline__ PagedSeq check_seq(const PagedSeqs& s, int start, int end, int len) {
    const bool ok = start >= 0 && end >= start && end <= s.rows && end - start <= s.max_q && len >= 0 &&
                    len <= s.max_len - (end - start);
    return {ok ? start : 0, ok ? end - start : 0, ok ? len : 0, ok};
}

__device__ __forceinline__ PagedSeq load_seq(const PagedSeqs& s, int b) {
    return check_seq(s, s.start[b], s.start[b + 1], s.len[b]);
}

// The page of slots 32 i .. of sequence b, clamped into the pool; i < pages_ld.
__device__ __forceinline__ int page_of(const PagedSeqs& s, int b, int i, bool& ok) {
    const int id = s.pages[(size_t)b * s.pages_ld + i];
    ok = id >= 0 && id < s.n_pages;
    return ok ? id : 0;
}

// Every sequence's numbers are looked at once per launch, by one wave of it.
__device__ __forceinline__ void check_seqs(const PagedSeqs& s, int lane) {
    bool bad = false;
    for (int b = lane; b < s.B; b += 64) bad |= !load_seq(s, b).ok;
    if (bad) atomicOr(s.err, 4);
}

// A call's work in pieces: those of sequence b begin at piece floor(start[b] * mul / unit) + extra * b, which leaves every
// sequence enough of them (floor(x + y) >= floor(x) + floor(y)) without sums over the sequences.  The sequence of a piece
// is the last that begins at it or before; the whole wave takes part.  Where starts do not ascend (which check_seqs
// reports) the answer is some sequence, and the piece's number in it may be negative.
__device__ __forceinline__ int piece_begin(int start, int mul, int unit, int extra, int b) {
    return (int)((long)start * mul / unit) + extra * b;
}
struct PieceSeq { int b; PagedSeq seq; };
__device__ __forceinline__ PieceSeq seq_of_piece(const PagedSeqs& s, int piece, int mul, int unit, int extra, int lane) {
    int before = 0, b0 = 0, start, end, len;   // this lane's sequence's
    for (;; b0 += 64) {
        const int b = b0 + lane, bc = min(b, s.B - 1);
        start = s.start[bc];
        end = s.start[bc + 1];
        len = s.len[bc];
        const unsigned long long in = __ballot(b < s.B && piece_begin(start, mul, unit, extra, b) <= piece);
        before += __popcll(in);
        if (in != ~0ull || b0 + 64 >= s.B) break;
    }
    const int b = max(before, 1) - 1;
    if (b < b0) return {b, load_seq(s, b)};   // the last of the 64 before
    const int l = b - b0;
    return {b, check_seq(s, __builtin_amdgcn_readlane(start, l), __builtin_amdgcn_readlane(end, l), __builtin_amdgcn_readlane(len, l))};
}

}  // namespace sdsat
