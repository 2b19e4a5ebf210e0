// Block tables, slot maps and row offsets of a step, from the lengths of its requests, on the GPU: an engine whose lengths live there
// (decoding steps replayed from a graph) needs no round trip to the host to give its sequences cache blocks.
//
// The free blocks are a stack.  Everything follows from three prefix sums over the sequences: rows asked for by chunks, blocks
// needed, and rows taken.  A sequence is refused where the rows or blocks that it and those in front of it ask for are not there, so
// the sequences that get blocks stand in front of those that do not: the blocks needed in front of one that gets some were all
// given, and its place on the stack is the plain prefix sum.
// Bound: latency.  A step's lengths are a few KB, its slot map 8 bytes a row; what is there to save is round trips.
#include "internal.h"

namespace shiftattn {

namespace {

constexpr int kScanThreads = 1024;
constexpr uint32_t kMost = 0x7FFFFFFFu;   // sums saturate here (which keeps them monotone, and saturating addition is associative)

__device__ inline uint32_t add_sat(uint32_t a, uint32_t b) { return min(a + b, kMost); }

// inclusive prefix sum over the workgroup plus `carry`, which moves on to the sum of all; call with all threads
__device__ inline uint32_t scan(uint32_t v, uint32_t& carry, uint32_t* wave_sum) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = static_cast<uint32_t>(__shfl_up(static_cast<int>(v), o));
        if (lane >= o) v = add_sat(v, up);
    }
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    uint32_t front = carry, all = carry;
    for (int w = 0; w < kScanThreads / 64; ++w) {
        if (w < wave) front = add_sat(front, wave_sum[w]);
        all = add_sat(all, wave_sum[w]);
    }
    __syncthreads();
    carry = all;
    return add_sat(v, front);
}

__device__ inline int blocks_of(int tokens) { return tokens / kBlockSize + (tokens % kBlockSize != 0); }

// last index in [0, n) with from[index] <= x, for from[0] <= x and a non-decreasing array
__device__ inline int last_at_most(const int32_t* from, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (from[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

// ws: [num_seqs] blocks given to the sequences in front, then the blocks given in all and the stack's height before
__global__ __launch_bounds__(kScanThreads) void tables_append_scan_kernel(shiftattn_tables t, const int32_t* new_lens, int num_prefill,
                                                                          int total_prefill_q, int32_t* cu, int32_t* taken, int32_t* ws) {
    __shared__ uint32_t wave_sum[kScanThreads / 64];
    __shared__ int given_s;
    const int64_t room = static_cast<int64_t>(t.max_blocks_per_seq) * kBlockSize;
    const int height = min(max(*t.free_count, 0), t.num_blocks);
    uint32_t asked_c = 0, need_c = 0, rows_c = 0;
    if (threadIdx.x == 0) given_s = 0;
    for (int base = 0; base < t.num_seqs; base += kScanThreads) {
        const int s = base + threadIdx.x;
        const bool there = s < t.num_seqs, chunk = s < num_prefill;
        const int had = there ? max(t.seq_lens[s], 0) : 0, n = there ? max(new_lens[s], 0) : 0;
        bool ok = there && static_cast<int64_t>(had) + n <= room && (chunk || n <= 1);
        const uint32_t asked = scan(ok && chunk ? n : 0, asked_c, wave_sum);
        ok = ok && (!chunk || asked <= static_cast<uint32_t>(total_prefill_q));
        const uint32_t need = ok ? blocks_of(had + n) - blocks_of(had) : 0;
        const uint32_t needed = scan(need, need_c, wave_sum);
        ok = ok && (need == 0 || needed <= static_cast<uint32_t>(height));
        const int take = ok ? n : 0;
        const uint32_t rows = scan(chunk ? take : 0, rows_c, wave_sum);
        if (!there) continue;   // (no barrier is left in this round)
        if (ok && need > 0) atomicMax(&given_s, static_cast<int>(needed));
        taken[s] = take;
        if (take > 0) t.seq_lens[s] = had + take;
        ws[s] = static_cast<int32_t>(needed - need);
        if (chunk) cu[s + 1] = static_cast<int32_t>(rows);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        cu[0] = 0;
        ws[t.num_seqs] = given_s;
        ws[t.num_seqs + 1] = height;
        *t.free_count = height - given_s;
    }
}

// table entries of the blocks given, then a slot per row
__global__ __launch_bounds__(256) void tables_append_fill_kernel(shiftattn_tables t, int num_prefill, int total_prefill_q, int rows,
                                                                 const int32_t* cu, int64_t* slots, const int32_t* taken, const int32_t* ws) {
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256, first = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const int given = ws[t.num_seqs], height = ws[t.num_seqs + 1];
    for (int64_t k = first; k < given; k += stride) {
        const int s = last_at_most(ws, t.num_seqs, static_cast<int>(k));
        const int had = max(t.seq_lens[s], 0) - taken[s];
        t.block_table[static_cast<size_t>(s) * t.max_blocks_per_seq + blocks_of(had) + (static_cast<int>(k) - ws[s])] = t.free_blocks[height - 1 - k];
    }
    const int num_decode = t.num_seqs - num_prefill;
    for (int64_t r = first; r < rows; r += stride) {
        int s = -1, row = 0;
        if (r < total_prefill_q) {
            if (num_prefill > 0 && r < cu[num_prefill]) {
                s = last_at_most(cu, num_prefill, static_cast<int>(r));
                row = static_cast<int>(r) - cu[s];
            }
        } else if (r - total_prefill_q < num_decode) {
            s = num_prefill + static_cast<int>(r - total_prefill_q);
            if (taken[s] == 0) s = -1;
        }
        int64_t slot = -1;
        if (s >= 0) {
            const int had = max(t.seq_lens[s], 0) - taken[s], p = had + row, i = p / kBlockSize, kept = blocks_of(had);
            const int64_t blk = i < kept ? t.block_table[static_cast<size_t>(s) * t.max_blocks_per_seq + i] : t.free_blocks[height - 1 - ws[s] - (i - kept)];
            slot = blk * kBlockSize + p % kBlockSize;
        }
        slots[r] = slot;
    }
}

// ws: [num_seqs] blocks given back by the sequences in front, then those given back in all and the stack's height before
__global__ __launch_bounds__(kScanThreads) void tables_truncate_scan_kernel(shiftattn_tables t, const int32_t* keep_lens, int32_t* ws) {
    __shared__ uint32_t wave_sum[kScanThreads / 64];
    const int height = min(max(*t.free_count, 0), t.num_blocks);
    uint32_t gone_c = 0;
    for (int base = 0; base < t.num_seqs; base += kScanThreads) {
        const int s = base + threadIdx.x;
        const bool there = s < t.num_seqs;
        const int had = there ? t.seq_lens[s] : 0, keep = there ? keep_lens[s] : -1;
        const bool cut = keep >= 0 && keep < had;
        const uint32_t gone = cut ? blocks_of(had) - blocks_of(keep) : 0;
        const uint32_t all = scan(gone, gone_c, wave_sum);
        if (!there) continue;
        ws[s] = static_cast<int32_t>(all - gone);
        if (cut) t.seq_lens[s] = keep;
    }
    if (threadIdx.x == 0) {
        ws[t.num_seqs] = static_cast<int32_t>(gone_c);
        ws[t.num_seqs + 1] = height;
        *t.free_count = static_cast<int>(min(static_cast<uint32_t>(height) + gone_c, static_cast<uint32_t>(t.num_blocks)));
    }
}

__global__ __launch_bounds__(256) void tables_truncate_fill_kernel(shiftattn_tables t, const int32_t* ws) {
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
    const int gone = ws[t.num_seqs];
    const int64_t top = static_cast<int64_t>(ws[t.num_seqs + 1]) + gone;
    for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < gone; k += stride) {
        const int s = last_at_most(ws, t.num_seqs, static_cast<int>(k));
        const int i = blocks_of(max(t.seq_lens[s], 0)) + (static_cast<int>(k) - ws[s]);
        // (a stack that would outgrow its memory has been given a block twice: what lies past the end is dropped)
        if (top - 1 - k < t.num_blocks) t.free_blocks[top - 1 - k] = t.block_table[static_cast<size_t>(s) * t.max_blocks_per_seq + i];
    }
}

unsigned fill_grid(int64_t items) {
    const int64_t wgs = (items + 255) / 256;
    return static_cast<unsigned>(wgs < 1 ? 1 : wgs > 2048 ? 2048 : wgs);
}

}  // namespace

size_t tables_workspace(int num_seqs) { return (static_cast<size_t>(num_seqs) + 2) * sizeof(int32_t); }

hipError_t launch_tables_append(const shiftattn_tables& t, const int32_t* new_lens, int num_prefill, int total_prefill_q, int rows, int32_t* cu,
                                int64_t* slots, int32_t* taken, void* workspace, hipStream_t st) {
    int32_t* ws = static_cast<int32_t*>(workspace);
    tables_append_scan_kernel<<<1, kScanThreads, 0, st>>>(t, new_lens, num_prefill, total_prefill_q, cu, taken, ws);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    tables_append_fill_kernel<<<fill_grid(rows), 256, 0, st>>>(t, num_prefill, total_prefill_q, rows, cu, slots, taken, ws);
    return hipGetLastError();
}

hipError_t launch_tables_truncate(const shiftattn_tables& t, const int32_t* keep_lens, void* workspace, hipStream_t st) {
    int32_t* ws = static_cast<int32_t*>(workspace);
    tables_truncate_scan_kernel<<<1, kScanThreads, 0, st>>>(t, keep_lens, ws);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t entries = static_cast<int64_t>(t.num_seqs) * t.max_blocks_per_seq;
    tables_truncate_fill_kernel<<<fill_grid(entries < t.num_blocks ? entries : t.num_blocks), 256, 0, st>>>(t, ws);
    return hipGetLastError();
}

}  // namespace shiftattn
