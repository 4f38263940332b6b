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
// loaded before anything is stored over it (children first); each cycle
// begins by holding one member's cell in a second register.  The list is made
// by one workgroup in a launch of its own, which also updates the lengths.
// Nothing is computed: each source's pages are read once, each destination's
// written once, and the copy is bound by HBM.
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
    __shared__ int s_total, s_more;
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
    if (b == 0) s_total = 0;
    __syncthreads();
    const bool moves = b < all && src >= 0 && src != b;
    if (moves) atomicAdd(&s_dests[src], 1);
    __syncthreads();
    if (moves && s_dests[b] > 0) atomicAdd(&s_wait[src], 1);
    bool todo = b < all && s_dests[b] > 0;
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
        *n_steps = total;
    }
    __syncthreads();
    if (b < all && s_dests[b] > 0) steps[s_at[b]] = int2{s_op[b] * 65536 + b, (len + 31) / 32 * 32};
    if (moves) steps[s_at[src] + 1 + atomicAdd(&s_put[src], 1)] = int2{RS_STORE * 65536 + b, 0};
    if (b < batch) cache_len[b] = src < 0 ? 0 : s_len[src];
}

// Workgroup (x, y, z): 16-byte cells x * 256 * kReorderCells .. of head y's K (even) or V (odd) in layer z.
static constexpr int kReorderCells = 4;
__global__ void __launch_bounds__(256) reorder_copy_kernel(u32x4_t* kc, u32x4_t* vc, size_t layer_cells, int H,
                                                           size_t head_cells, int slot_cells, int first,
                                                           const int2* steps, const int* n_steps) {
    const int n = *n_steps;
    const int h = (int)blockIdx.y >> 1;
    u32x4_t* base = (blockIdx.y & 1 ? vc : kc) + blockIdx.z * layer_cells + h * head_cells;
    const size_t seq_cells = (size_t)H * head_cells;
    size_t cell[kReorderCells];
#pragma unroll
    for (int u = 0; u < kReorderCells; ++u)
        cell[u] = (size_t)first * slot_cells + ((size_t)blockIdx.x * kReorderCells + u) * 256 + threadIdx.x;
    u32x4_t v[kReorderCells], held[kReorderCells];
    size_t end = 0, held_end = 0;
    for (int i = 0; i < n; ++i) {
        const int2 st = steps[i];
        u32x4_t* row = base + (size_t)(st.x & 0xFFFF) * seq_cells;
        switch (st.x >> 16) {
            case RS_LOAD:
                end = (size_t)st.y * slot_cells;
#pragma unroll
                for (int u = 0; u < kReorderCells; ++u)
                    if (cell[u] < end) v[u] = row[cell[u]];
                break;
            case RS_HOLD:
                held_end = (size_t)st.y * slot_cells;
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
                    if (cell[u] < end) row[cell[u]] = v[u];
        }
    }
}

hipError_t launch_reorder(int esz, void* kc, void* vc, size_t layer_elems, int n_layers, int batch, int all, int H, int Dh,
                          int S_max, int* cache_len, int max_len, const int* src, int first_slot, int* steps, int* err,
                          hipStream_t s) {
    if (batch < 1 || batch > all || all > kReorderMaxBatch || (Dh * esz) % 16 || first_slot < 0 || S_max % 32 ||
        max_len < 0 || max_len > S_max || !src || !steps)
        return hipErrorInvalidValue;
    // steps: the count, then (8-byte aligned) the list
    hipLaunchKernelGGL(reorder_plan_kernel, dim3(1), dim3((all + 63) / 64 * 64), 0, s, cache_len, batch, all, S_max, src,
                       reinterpret_cast<int2*>(steps + 2), steps, err);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int first = first_slot / 32 * 32, end = (max_len + 31) / 32 * 32;
    if (end <= first) return hipSuccess;   // no page to move
    const int slot_cells = Dh * esz / 16;
    const size_t cells = (size_t)(end - first) * slot_cells;
    const unsigned gx = (unsigned)((cells + 256 * kReorderCells - 1) / (256 * kReorderCells));
    hipLaunchKernelGGL(reorder_copy_kernel, dim3(gx, 2 * H, n_layers), dim3(256), 0, s, static_cast<u32x4_t*>(kc),
                       static_cast<u32x4_t*>(vc), layer_elems * esz / 16, H, (size_t)S_max * slot_cells, slot_cells, first,
                       reinterpret_cast<const int2*>(steps + 2), steps);
    return hipGetLastError();
}

}  // namespace sdsat
