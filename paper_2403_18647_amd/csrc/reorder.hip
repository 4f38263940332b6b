// Reordering the KV cache: sequence b of a batch continues from sequence src[b]
// (a prompt forked into samples, beams that follow their parents, survivors
// moved into the rows of finished sequences; src[b] = -1 frees sequence b).
//
//   K[l][b][h][p], V[l][b][h][p] <- those of sequence src[b], as they stood
//   before the call, for the 32-slot pages p from the one that holds
//   first_slot to the last with a committed slot of src[b];
//   cache_len[b] <- cache_len[src[b]]  (0 for src[b] = -1).
//
// The map may be any: one source for many, chains (0 <- 1 <- 2), swaps and
// cycles, all in place.  A cell (layer, K or V, head, 16 bytes of a page) of
// one sequence only ever moves to the same cell of another, so one thread
// owns a cell of every sequence and walks a list of steps that is the same
// for all cells: load a source, store it to its destinations.  A source is
// loaded before anything is stored over it (destinations that are sources
// themselves first); each cycle begins by holding one member's cell in a second
// register.  For up to 64 sequences and 8192 workgroups every workgroup makes
// the list itself, in one wave, and the last one to finish writes the new
// lengths (one launch instead of two: four sequences of a tiny decoder 8.2 ->
// 5.3 us, one page of eight sequences in eight 7B layers 10.4 -> 9.3, 8192
// workgroups 41.7 -> 39.0; but 20160 209.7 -> 213.8, 40000 436 -> 452); else one
// workgroup makes it in a launch ahead.
// Nothing is computed: each source's pages are read once, each destination's
// written once, and the copy is bound by HBM: 16 sequences of 4000 slots
// compacted in four 13B layers (2.47 GB) 432-437 us, 5.7 TB/s; nontemporal stores,
// which nothing of this call reads again (ordinary ones 456 us; eight beams of 790
// slots in eight 7B layers 40 and 54).
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace sdsat {

// A step: x = operation * 65536 + sequence; y = for loads, the end of the source's pages (slots)
enum { RS_LOAD = 0, RS_STORE = 1, RS_HOLD = 2, RS_USE = 3 };

// One thread per sequence.  Every source gets a run of steps (its load, then a store per destination) at an offset
// given out in rounds: a source is ready once every destination of its that is itself a source has its run.  What
// is left are the cycles, walked one after the other.
__global__ void __launch_bounds__(kReorderMaxBatch) reorder_plan_kernel(int* cache_len, int batch, int all, int S_max,
                                                                        const int* d_src, int2* steps, int* n_steps,
                                                                        int* err) {
    __shared__ int s_src[kReorderMaxBatch], s_len[kReorderMaxBatch];
    __shared__ int s_dests[kReorderMaxBatch];    // destinations of a source
    __shared__ int s_wait[kReorderMaxBatch];     // of which are sources without a run
    __shared__ int s_at[kReorderMaxBatch];       // where its run begins, -1 without one
    __shared__ int s_op[kReorderMaxBatch], s_put[kReorderMaxBatch];
    __shared__ int s_total, s_more, s_end;
    const int b = threadIdx.x;
    int src = b;   // sequences from `batch` on stay
    int len = 0;
    if (b < all) {
        len = min(max(cache_len[b], 0), S_max);
        if (b < batch) {
            src = d_src[b];
            if (src < -1 || src >= all) {
                atomicOr(err, 32);
                src = b;
            }
        }
        s_src[b] = src;
        s_len[b] = len;
        s_dests[b] = s_wait[b] = s_put[b] = 0;
        s_at[b] = -1;
        s_op[b] = RS_LOAD;
    }
    if (b == 0) s_total = s_end = 0;
    __syncthreads();
    const bool moves = b < all && src >= 0 && src != b;
    if (moves) atomicAdd(&s_dests[src], 1);
    __syncthreads();
    if (moves && s_dests[b] > 0) atomicAdd(&s_wait[src], 1);
    bool todo = b < all && s_dests[b] > 0;
    if (todo) atomicMax(&s_end, (len + 31) / 32 * 32);
    for (;;) {
        __syncthreads();
        if (b == 0) s_more = 0;
        const bool ready = todo && s_wait[b] == 0;
        __syncthreads();
        if (ready) {
            s_at[b] = atomicAdd(&s_total, 1 + s_dests[b]);
            if (moves) atomicAdd(&s_wait[src], -1);
            todo = false;
            s_more = 1;
        }
        __syncthreads();
        if (!s_more) break;
    }
    if (b == 0) {
        int total = s_total;
        for (int c0 = 0; c0 < all; ++c0) {
            if (s_dests[c0] == 0 || s_at[c0] >= 0) continue;
            steps[total++] = int2{RS_HOLD * 65536 + c0, (s_len[c0] + 31) / 32 * 32};
            for (int c = s_src[c0]; c != c0; c = s_src[c]) {
                s_at[c] = total;
                total += 1 + s_dests[c];
            }
            s_at[c0] = total;
            s_op[c0] = RS_USE;
            total += 1 + s_dests[c0];
        }
        n_steps[0] = total;
        n_steps[1] = s_end;
    }
    __syncthreads();
    if (b < all && s_dests[b] > 0) steps[s_at[b]] = int2{s_op[b] * 65536 + b, (len + 31) / 32 * 32};
    if (moves) steps[s_at[src] + 1 + atomicAdd(&s_put[src], 1)] = int2{RS_STORE * 65536 + b, 0};
    if (b < batch) cache_len[b] = src < 0 ? 0 : s_len[src];
}

// The same list in one wave, a lane per sequence, left in LDS; returns its length and the longest source's slots.  src: the
// lane's (-1: none, lane itself: stays), slots: its committed ones in whole pages.
__device__ __forceinline__ int2 reorder_list(int src, int slots, int lane, int2* steps) {
    typedef unsigned long long u64;
    const bool moves = src >= 0 && src != lane;
    u64 dests = 0;   // of this lane as a source
    for (u64 left = __ballot(moves); left;) {
        const int a = __builtin_amdgcn_readlane(src, __builtin_ctzll(left));
        const u64 m = __ballot(moves && src == a);
        if (lane == a) dests = m;
        left &= ~m;
    }
    const u64 sources = __ballot(dests != 0);
    const uint32_t d_lo = (uint32_t)dests, d_hi = (uint32_t)(dests >> 32);
    auto count = [&](int a) {
        return __builtin_popcount(__builtin_amdgcn_readlane(d_lo, a)) + __builtin_popcount(__builtin_amdgcn_readlane(d_hi, a));
    };
    int total = 0, at = 0, op = RS_LOAD;
    u64 done = 0;
    for (;;) {   // sources whose destinations have all been loaded, or are none themselves
        u64 ready = __ballot(dests != 0 && !(done >> lane & 1) && (dests & sources & ~done) == 0);
        if (!ready) break;
        done |= ready;
        for (; ready; ready &= ready - 1) {
            const int a = __builtin_ctzll(ready);
            if (lane == a) at = total;
            total += 1 + count(a);
        }
    }
    for (u64 left = sources & ~done; left; left = sources & ~done) {   // cycles
        const int c0 = __builtin_ctzll(left);
        if (lane == c0) {
            steps[total] = int2{RS_HOLD * 65536 + lane, slots};
            op = RS_USE;
        }
        ++total;
        int c = c0;
        do {
            c = __builtin_amdgcn_readlane(src, c);
            done |= 1ull << c;
            if (lane == c) at = total;
            total += 1 + count(c);
        } while (c != c0);
    }
    if (dests) steps[at] = int2{op * 65536 + lane, slots};
    const int s = moves ? src : lane;
    const u64 of = (u64)(uint32_t)__shfl((int)d_hi, s, 64) << 32 | (uint32_t)__shfl((int)d_lo, s, 64);
    const int base = __shfl(at, s, 64);
    if (moves) steps[base + 1 + __popcll(of & ((1ull << lane) - 1))] = int2{RS_STORE * 65536 + lane, 0};
    return int2{total, (int)across_wave(dests ? (float)slots : 0.f, OpMax())};   // exact: capacities are below 2^24
}

struct ReorderArgs {
    u32x4_t* kc; u32x4_t* vc;
    size_t layer_cells, head_cells;    // 16-byte cells of a layer's K (or V), of a sequence's head
    int n_layers, batch, all, H, S_max, slot_cells, first;
    int* cache_len; const int* src;
    const int2* steps; const int* n_steps;   // made ahead: the list, its length and the longest source's slots
    int* arrived; int* err;
};

// Chunks of 256 * kReorderCells cells of the pages from `first` on, of each layer, K and V, and head.  The host's grid holds
// them all as far as it knows the lengths and a launch may; workgroups take further ones where the device's lengths are
// longer (a replayed graph), or there are more.
static constexpr int kReorderCells = 2, kReorderAlone = 8192;   // cells per thread; workgroups that make the list themselves, at most
template <bool AHEAD>
__global__ void __launch_bounds__(256) reorder_copy_kernel(ReorderArgs a) {
    __shared__ int2 s_steps[AHEAD ? 1 : 3 * 64];
    __shared__ int2 s_n;
    const int2* steps = a.steps;
    int2 made;
    int now = 0;
    bool wrong = false;   // wave 0: the lane's new length, and whether its source is out of range
    if constexpr (AHEAD) {
        made = int2{a.n_steps[0], a.n_steps[1]};
    } else {
        if (threadIdx.x < 64) {
            const int lane = threadIdx.x;
            int src = lane < a.batch ? a.src[lane] : lane;   // sequences from `batch` on stay
            const int len = lane < a.all ? min(max(a.cache_len[lane], 0), a.S_max) : 0;
            const bool bad = lane < a.batch && (src < -1 || src >= a.all);
            if (bad) src = lane;
            const int2 list = reorder_list(src, (len + 31) / 32 * 32, lane, s_steps);
            if (lane == 0) s_n = list;
            now = __shfl(len, max(src, 0), 64);
            if (src < 0) now = 0;
            wrong = bad;
        }
        __syncthreads();
        made = s_n;
        steps = s_steps;
    }
    const int n = __builtin_amdgcn_readfirstlane(made.x), end_slot = __builtin_amdgcn_readfirstlane(made.y);
    const uint32_t chunks = (uint32_t)(((size_t)max(0, end_slot - a.first) * a.slot_cells + 256 * kReorderCells - 1) / (256 * kReorderCells));
    const size_t items = (size_t)chunks * 2 * a.H * a.n_layers;
    const size_t seq_cells = (size_t)a.H * a.head_cells;
    for (size_t at = blockIdx.x; at < items; at += gridDim.x) {
        const uint32_t item = (uint32_t)at, chunk = item % chunks, of = item / chunks, y = of % (2 * a.H), layer = of / (2 * a.H);
        u32x4_t* base = (y & 1 ? a.vc : a.kc) + layer * a.layer_cells + (y >> 1) * a.head_cells;
        size_t cell[kReorderCells];
#pragma unroll
        for (int u = 0; u < kReorderCells; ++u)
            cell[u] = (size_t)a.first * a.slot_cells + ((size_t)chunk * kReorderCells + u) * 256 + threadIdx.x;
        u32x4_t v[kReorderCells], held[kReorderCells];
        size_t end = 0, held_end = 0;
        for (int i = 0; i < n; ++i) {
            const int x = __builtin_amdgcn_readfirstlane(steps[i].x), slots = __builtin_amdgcn_readfirstlane(steps[i].y);
            u32x4_t* row = base + (size_t)(x & 0xFFFF) * seq_cells;
            switch (x >> 16) {
                case RS_LOAD:
                    end = (size_t)slots * a.slot_cells;
#pragma unroll
                    for (int u = 0; u < kReorderCells; ++u)
                        if (cell[u] < end) v[u] = row[cell[u]];
                    break;
                case RS_HOLD:
                    held_end = (size_t)slots * a.slot_cells;
#pragma unroll
                    for (int u = 0; u < kReorderCells; ++u)
                        if (cell[u] < held_end) held[u] = row[cell[u]];
                    break;
                case RS_USE:
                    end = held_end;
#pragma unroll
                    for (int u = 0; u < kReorderCells; ++u) v[u] = held[u];
                    break;
                default:
#pragma unroll
                    for (int u = 0; u < kReorderCells; ++u)
                        if (cell[u] < end) __builtin_nontemporal_store(v[u], row + cell[u]);
            }
        }
    }
    if constexpr (!AHEAD) {   // every workgroup has read the lengths: the last one here writes the new ones
        if (threadIdx.x >= 64) return;
        const int lane = threadIdx.x;
        int last = 0;
        if (lane == 0) {   // counted in kReorderCounts places first: 512 additions to one take 5 us
            auto arrive = [&](int* p, int all) {
                const bool full = __hip_atomic_fetch_add(p, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == all - 1;
                if (full) __hip_atomic_store(p, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                return full;
            };
            const int k = blockIdx.x % kReorderCounts;
            last = arrive(a.arrived + 32 * (1 + k), ((int)gridDim.x - k + kReorderCounts - 1) / kReorderCounts) &&
                   arrive(a.arrived, min((int)gridDim.x, kReorderCounts));
        }
        if (__builtin_amdgcn_readfirstlane(last) && lane < a.batch) {
            if (wrong) atomicOr(a.err, 32);
            a.cache_len[lane] = now;
        }
    }
}

// Sequences that one workgroup's threads hold, slots that a float holds, chunks that their 32-bit number holds.
bool reorder_supported(int esz, int all, int n_layers, int H, int Dh, int S_max) {
    const long cells = (long)S_max * (Dh * esz / 16), most = (cells + 256 * kReorderCells - 1) / (256 * kReorderCells) * 2 * H * n_layers;
    return all <= kReorderMaxBatch && S_max < 1 << 24 && most <= 0x7FFFFFFF;
}

// One workgroup per chunk as far as the host knows the lengths; a launch holds fewer than 2^32 threads, so of larger caches
// (7B heads and layers: from 262144 slots on) each workgroup takes several.
long reorder_workgroups(int esz, int n_layers, int H, int Dh, int max_len, int first_slot) {
    const int first = first_slot / 32 * 32, end = (max_len + 31) / 32 * 32;
    const size_t cells = (size_t)std::max(0, end - first) * (Dh * esz / 16);
    const long chunks = (long)((cells + 256 * kReorderCells - 1) / (256 * kReorderCells));
    return std::min<long>(std::max<long>(1, chunks * 2 * H * n_layers), 0xFFFFFFFFu / 256);
}

hipError_t launch_reorder(int esz, void* kc, void* vc, size_t layer_elems, int n_layers, int batch, int all, int H, int Dh,
                          int S_max, int* cache_len, int max_len, const int* src, int first_slot, int* steps, int* err,
                          hipStream_t s) {
    if (batch < 1 || batch > all || all > kReorderMaxBatch || (Dh * esz) % 16 || first_slot < 0 || S_max % 32 ||
        max_len < 0 || max_len > S_max || !src || !steps)
        return hipErrorInvalidValue;
    if (!reorder_supported(esz, all, n_layers, H, Dh, S_max)) return hipErrorInvalidValue;
    const int slot_cells = Dh * esz / 16;
    const long groups = reorder_workgroups(esz, n_layers, H, Dh, max_len, first_slot);
    const bool ahead = all > 64 || groups > kReorderAlone;
    if (ahead) {
        hipLaunchKernelGGL(reorder_plan_kernel, dim3(1), dim3((all + 63) / 64 * 64), 0, s, cache_len, batch, all, S_max, src,
                           reinterpret_cast<int2*>(steps + kReorderHead), steps + kReorderHead - 2, err);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    ReorderArgs a{};
    a.kc = static_cast<u32x4_t*>(kc); a.vc = static_cast<u32x4_t*>(vc);
    a.layer_cells = layer_elems * esz / 16; a.head_cells = (size_t)S_max * slot_cells;
    a.n_layers = n_layers; a.batch = batch; a.all = all; a.H = H; a.S_max = S_max; a.slot_cells = slot_cells;
    a.first = first_slot / 32 * 32;
    a.cache_len = cache_len; a.src = src; a.steps = reinterpret_cast<const int2*>(steps + kReorderHead);
    a.n_steps = steps + kReorderHead - 2;
    a.arrived = steps; a.err = err;
    const dim3 grid((unsigned)groups);
    if (ahead) hipLaunchKernelGGL(reorder_copy_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(reorder_copy_kernel<false>, grid, dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace sdsat
