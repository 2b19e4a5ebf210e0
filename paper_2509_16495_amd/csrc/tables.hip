// Block tables, slot maps and row offsets of a step, from the lengths of its requests, on the GPU: an engine whose lengths live there
// (decoding steps replayed from a graph) needs no round trip to the host to give its sequences cache blocks.
//
// The free blocks are a stack.  Everything follows from three prefix sums over the sequences: rows asked for by chunks, blocks
// needed, and rows taken.  A sequence is refused where the rows or blocks that it and those in front of it ask for are not there, so
// the sequences that get blocks stand in front of those that do not: the blocks needed in front of one that gets some were all
// given, and its place on the stack is the plain prefix sum.
// Bound: latency.  A step's lengths are a few KB, its slot map 8 bytes a row; what is there to save is launches and round trips.
#include "internal.h"

#include <type_traits>

namespace shiftattn {

namespace {

constexpr int kOnePass = 1024;            // sequences that a launch of one workgroup holds, one a thread
constexpr uint32_t kMost = 0x7FFFFFFFu;   // sums saturate here (which keeps them monotone, and saturating addition is associative)

__device__ inline uint32_t add_sat(uint32_t a, uint32_t b) { return min(a + b, kMost); }

template <int kV>
using Int = std::integral_constant<int, kV>;

// inclusive prefix sum over the workgroup plus `carry`, which moves on to the sum of all; call with all threads
template <int kThreads>
__device__ inline uint32_t scan(uint32_t v, uint32_t& carry, uint32_t* wave_sum) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // over the wavefront with cross-lane moves: rows of 16, then row to row (a lane without a source adds 0)
    auto add_from = [&](auto ctrl, auto rows) {
        v = add_sat(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, false)));
    };
    add_from(Int<0x111>{}, Int<0xf>{});   // row_shr:1, 2, 4, 8
    add_from(Int<0x112>{}, Int<0xf>{});
    add_from(Int<0x114>{}, Int<0xf>{});
    add_from(Int<0x118>{}, Int<0xf>{});
    add_from(Int<0x142>{}, Int<0xa>{});   // lane 15 of a row into rows 1 and 3
    add_from(Int<0x143>{}, Int<0xc>{});   // lane 31 into rows 2 and 3
    if constexpr (kThreads == 64) {
        v = add_sat(v, carry);
        carry = static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(v), 63));
        return v;
    }
    if (lane == 63) wave_sum[wave] = v;
    __syncthreads();
    uint32_t front = carry, all = carry;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        if (w < wave) front = add_sat(front, wave_sum[w]);
        all = add_sat(all, wave_sum[w]);
    }
    __syncthreads();
    carry = all;
    return add_sat(v, front);
}

// tokens that a sequence's row of block_table can hold (lengths are int32)
__device__ inline int64_t room_of(const shiftattn_tables& t) {
    return min(static_cast<int64_t>(t.max_blocks_per_seq) * kBlockSize, static_cast<int64_t>(kMost));
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

// What the second half of either call needs of the first, per sequence: blocks given to (or back by) the sequences in front, chunks'
// first rows, and tokens in front of the new ones.  In LDS where one workgroup does it all, in the workspace and the results otherwise.
struct Shared {
    int32_t front[kOnePass], row[kOnePass + 1], had[kOnePass];
};

// The slot of one row and the table entry of one block given.  kInLds: by the arrays above.
template <bool kInLds>
struct AppendView {
    const shiftattn_tables& t;
    int num_prefill, total_prefill_q, given, height;
    const int32_t *front, *cu, *had_s;      // had_s: LDS only
    const int32_t* taken;
    __device__ int had(int s) const { return kInLds ? had_s[s] : max(t.seq_lens[s], 0) - taken[s]; }
    __device__ int32_t popped(int k) const { return t.free_blocks[height - 1 - k]; }
    __device__ void entry(int k) const {
        const int s = last_at_most(front, t.num_seqs, k);
        t.block_table[static_cast<size_t>(s) * t.max_blocks_per_seq + blocks_of(had(s)) + (k - front[s])] = popped(k);
    }
    __device__ int64_t slot(int s, int row) const {
        const int h = had(s), p = h + row, i = p / kBlockSize, kept = blocks_of(h);
        const int64_t blk = i < kept ? t.block_table[static_cast<size_t>(s) * t.max_blocks_per_seq + i] : popped(front[s] + (i - kept));
        return blk * kBlockSize + p % kBlockSize;
    }
    __device__ int64_t chunk_row(int r) const {   // r < total_prefill_q
        if (num_prefill == 0 || r >= cu[num_prefill]) return -1;
        const int s = last_at_most(cu, num_prefill, r);
        return slot(s, r - cu[s]);
    }
};

// kOne: one workgroup does the whole call (at most kThreads sequences): everything stays in LDS, and each decode sequence's thread writes its
// row.  Else the first of two launches, whose second one needs ws: [num_seqs] blocks given to the sequences in front, then the blocks
// given in all and the stack's height before.
template <bool kOne, int kThreads>
__global__ __launch_bounds__(kThreads) void tables_append_kernel(shiftattn_tables t, const int32_t* new_lens, int num_prefill, int total_prefill_q,
                                                                 int rows, int32_t* cu, int64_t* slots, int32_t* taken, int32_t* ws) {
    __shared__ uint32_t wave_sum[kThreads / 64];
    __shared__ int given_s;
    __shared__ Shared sh;
    const int64_t room = room_of(t);
    const int height = min(max(*t.free_count, 0), t.num_blocks);
    uint32_t asked_c = 0, need_c = 0, rows_c = 0;
    if (threadIdx.x == 0) given_s = 0;
    if constexpr (kThreads > 64) __syncthreads();
    for (int base = 0; base < t.num_seqs; base += kThreads) {
        const int s = base + threadIdx.x;
        const bool there = s < t.num_seqs, chunk = s < num_prefill, chunks_here = base < num_prefill;   // (the last: uniform)
        const int had = there ? max(t.seq_lens[s], 0) : 0, n = there ? max(new_lens[s], 0) : 0;
        bool ok = there && static_cast<int64_t>(had) + n <= room && (chunk || n <= 1);
        if (chunks_here) {
            const uint32_t asked = scan<kThreads>(ok && chunk ? n : 0, asked_c, wave_sum);
            ok = ok && (!chunk || asked <= static_cast<uint32_t>(total_prefill_q));
        }
        const uint32_t need = ok ? blocks_of(had + n) - blocks_of(had) : 0;
        const uint32_t needed = scan<kThreads>(need, need_c, wave_sum);
        ok = ok && (need == 0 || needed <= static_cast<uint32_t>(height));
        const int take = ok ? n : 0;
        uint32_t row = 0;
        if (chunks_here) row = scan<kThreads>(chunk ? take : 0, rows_c, wave_sum);
        // blocks given so far: the sum behind the last sequence that got some (one lane of a wavefront says it)
        const uint64_t got = __builtin_amdgcn_ballot_w64(ok && need > 0);
        if (got != 0 && static_cast<int>(threadIdx.x & 63) == 63 - __builtin_clzll(got)) atomicMax(&given_s, static_cast<int>(needed));
        if (!there) continue;   // (no barrier is left in this round)
        const int front = static_cast<int>(needed - need);
        taken[s] = take;
        if (take > 0) t.seq_lens[s] = had + take;
        if (chunk) cu[s + 1] = static_cast<int32_t>(row);
        if constexpr (kOne) {
            sh.front[s] = front, sh.had[s] = had;
            if (chunk) {
                sh.row[s + 1] = static_cast<int32_t>(row);
            } else {   // its one row, and block
                int64_t slot = -1;
                if (take > 0) {
                    const int i = had / kBlockSize;
                    int32_t* at = t.block_table + static_cast<size_t>(s) * t.max_blocks_per_seq + i;
                    slot = static_cast<int64_t>(need > 0 ? t.free_blocks[height - 1 - front] : *at) * kBlockSize + had % kBlockSize;
                }
                slots[total_prefill_q + s - num_prefill] = slot;
            }
        } else {
            ws[s] = front;
        }
    }
    __syncthreads();
    const int given = given_s;
    if (threadIdx.x == 0) {
        cu[0] = 0;
        *t.free_count = height - given;
        if constexpr (!kOne) {
            ws[t.num_seqs] = given;
            ws[t.num_seqs + 1] = height;
        }
    }
    if constexpr (kOne) {
        if (threadIdx.x == 0) sh.row[0] = 0;
        __syncthreads();
        const AppendView<true> v{t, num_prefill, total_prefill_q, given, height, sh.front, sh.row, sh.had, nullptr};
        for (int k = threadIdx.x; k < given; k += kThreads) v.entry(k);
        for (int r = threadIdx.x; r < total_prefill_q; r += kThreads) slots[r] = v.chunk_row(r);
        for (int r = total_prefill_q + t.num_seqs - num_prefill + threadIdx.x; r < rows; r += kThreads) slots[r] = -1;
    }
}

// the second of two launches: table entries of the blocks given, then a slot per row
__global__ __launch_bounds__(256) void tables_append_fill_kernel(shiftattn_tables t, int num_prefill, int total_prefill_q, int rows,
                                                                 const int32_t* cu, int64_t* slots, const int32_t* taken, const int32_t* ws) {
    __shared__ int32_t cu_s[kOnePass + 1], front_s[kOnePass];
    const bool staged = t.num_seqs <= kOnePass;   // searched in LDS where they fit
    if (staged) {
        for (int i = threadIdx.x; i <= num_prefill; i += 256) cu_s[i] = cu[i];
        for (int i = threadIdx.x; i < t.num_seqs; i += 256) front_s[i] = ws[i];
        __syncthreads();
    }
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256, first = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    const AppendView<false> v{t, num_prefill, total_prefill_q, ws[t.num_seqs], ws[t.num_seqs + 1], staged ? front_s : ws, staged ? cu_s : cu, nullptr, taken};
    for (int64_t k = first; k < v.given; k += stride) v.entry(static_cast<int>(k));
    for (int64_t r = first; r < rows; r += stride) {
        int64_t slot = -1;
        const int64_t j = r - total_prefill_q;   // decode row
        if (j < 0) slot = v.chunk_row(static_cast<int>(r));
        else if (j < t.num_seqs - num_prefill && taken[num_prefill + j] > 0) slot = v.slot(num_prefill + static_cast<int>(j), 0);
        slots[r] = slot;
    }
}

// Block k of those given back, to its place.  front, keep: blocks given back by the sequences in front, and tokens kept.
__device__ inline void give_back(const shiftattn_tables& t, const int32_t* front, const int32_t* keep, int64_t top, int k) {
    const int s = last_at_most(front, t.num_seqs, k);
    const int i = blocks_of(max(keep[s], 0)) + (k - front[s]);
    // (a stack that would outgrow its memory has been given a block twice: what lies past the end is dropped)
    if (top - 1 - k < t.num_blocks) t.free_blocks[top - 1 - k] = t.block_table[static_cast<size_t>(s) * t.max_blocks_per_seq + i];
}

// kOne as above; else ws: [num_seqs] blocks given back by the sequences in front, then those given back in all and the stack's height before
template <bool kOne, int kThreads>
__global__ __launch_bounds__(kThreads) void tables_truncate_kernel(shiftattn_tables t, const int32_t* keep_lens, int32_t* ws) {
    __shared__ uint32_t wave_sum[kThreads / 64];
    __shared__ Shared sh;
    const int64_t room = room_of(t);
    const int height = min(max(*t.free_count, 0), t.num_blocks);
    uint32_t gone_c = 0;
    for (int base = 0; base < t.num_seqs; base += kThreads) {
        const int s = base + threadIdx.x;
        const bool there = s < t.num_seqs;
        const int had = there ? t.seq_lens[s] : 0, keep = there ? keep_lens[s] : -1;
        const bool cut = keep >= 0 && keep < had && had <= room;   // (blocks behind the row are nobody's to give back)
        const uint32_t gone = cut ? blocks_of(had) - blocks_of(keep) : 0;
        const uint32_t all = scan<kThreads>(gone, gone_c, wave_sum);
        if (!there) continue;
        if constexpr (kOne) sh.front[s] = static_cast<int32_t>(all - gone), sh.had[s] = cut ? keep : had;
        else ws[s] = static_cast<int32_t>(all - gone);
        if (cut) t.seq_lens[s] = keep;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        if constexpr (!kOne) {
            ws[t.num_seqs] = static_cast<int32_t>(gone_c);
            ws[t.num_seqs + 1] = height;
        }
        *t.free_count = static_cast<int>(min(static_cast<uint32_t>(height) + gone_c, static_cast<uint32_t>(t.num_blocks)));
    }
    if constexpr (kOne) {
#pragma unroll 4
        for (int k = threadIdx.x; k < static_cast<int>(gone_c); k += kThreads)
            give_back(t, sh.front, sh.had, static_cast<int64_t>(height) + gone_c, k);
    }
}

__global__ __launch_bounds__(256) void tables_truncate_fill_kernel(shiftattn_tables t, const int32_t* ws) {
    __shared__ int32_t front_s[kOnePass];
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
    const int gone = ws[t.num_seqs];
    if (static_cast<int64_t>(blockIdx.x) * 256 >= gone) return;   // uniform
    const bool staged = t.num_seqs <= kOnePass;
    if (staged) {
        for (int i = threadIdx.x; i < t.num_seqs; i += 256) front_s[i] = ws[i];
        __syncthreads();
    }
    for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < gone; k += stride)
        give_back(t, staged ? front_s : ws, t.seq_lens, static_cast<int64_t>(ws[t.num_seqs + 1]) + gone, static_cast<int>(k));
}

unsigned fill_grid(int64_t items) {
    const int64_t wgs = (items + 255) / 256;   // (more items a thread: 136456 rows 13.1 -> 14.1 us with two, 15.8 with four)
    return static_cast<unsigned>(wgs < 1 ? 1 : wgs > 2048 ? 2048 : wgs);
}

}  // namespace

size_t tables_workspace(int num_seqs) { return (static_cast<size_t>(num_seqs) + 2) * sizeof(int32_t); }

// One launch of one workgroup, or a scan and a launch that fills.  Append and truncate of a step, us in a replayed graph, one / two launches
// for the append: 61 decode rows 5.2 / 7.0, 1000 9.5 / 12.2, 2120 rows 10.1 / 11.2, 2456 10.7 / 10.8, 11520 18.7 / 16.1, 136456 112 / 17.6 (the
// last two before both were made faster; now 12.6 and 13.1 in two).  How many blocks a truncate gives back is known on the GPU only, so its line lies
// where the most that it can be costs a workgroup some 80 us: of few blocks one launch saves 1.6 us, of 8500 two save 11.  Threads of that one workgroup,
// 256 / 512 / 1024: append and truncate of 61 decode rows 5.2 / 5.3 / 5.7 us, of 25 prompts (5400 blocks back) 21 / 16.2 / 12.8.
constexpr int kOneLaunchRows = 2560, kOneLaunchBlocks = 65536;

// threads of the workgroup that scans: as few wavefronts as hold the sequences
template <class Launch>
hipError_t by_threads(int num_seqs, Launch launch) {
    if (num_seqs <= 64) launch(std::integral_constant<int, 64>{});
    else if (num_seqs <= 256) launch(std::integral_constant<int, 256>{});
    else if (num_seqs <= 512) launch(std::integral_constant<int, 512>{});
    else launch(std::integral_constant<int, kOnePass>{});
    return hipGetLastError();
}

hipError_t launch_tables_append(const shiftattn_tables& t, const int32_t* new_lens, int num_prefill, int total_prefill_q, int rows, int32_t* cu,
                                int64_t* slots, int32_t* taken, void* workspace, hipStream_t st) {
    int32_t* ws = static_cast<int32_t*>(workspace);
    if (t.num_seqs <= kOnePass && rows <= kOneLaunchRows)
        return by_threads(rows > 1024 ? kOnePass : t.num_seqs, [&](auto threads) {
            tables_append_kernel<true, decltype(threads)::value><<<1, decltype(threads)::value, 0, st>>>(t, new_lens, num_prefill, total_prefill_q, rows, cu, slots, taken, ws);
        });
    hipError_t e = by_threads(t.num_seqs, [&](auto threads) {
        tables_append_kernel<false, decltype(threads)::value><<<1, decltype(threads)::value, 0, st>>>(t, new_lens, num_prefill, total_prefill_q, rows, cu, slots, taken, ws);
    });
    if (e != hipSuccess) return e;
    tables_append_fill_kernel<<<fill_grid(rows), 256, 0, st>>>(t, num_prefill, total_prefill_q, rows, cu, slots, taken, ws);
    return hipGetLastError();
}

hipError_t launch_tables_truncate(const shiftattn_tables& t, const int32_t* keep_lens, void* workspace, hipStream_t st) {
    int32_t* ws = static_cast<int32_t*>(workspace);
    const int64_t entries = static_cast<int64_t>(t.num_seqs) * t.max_blocks_per_seq, most = entries < t.num_blocks ? entries : t.num_blocks;
    if (t.num_seqs <= kOnePass && most <= kOneLaunchBlocks)
        return by_threads(most > 4096 && t.num_seqs < 512 ? 512 : most > 1024 && t.num_seqs < 256 ? 256 : t.num_seqs, [&](auto threads) {
            tables_truncate_kernel<true, decltype(threads)::value><<<1, decltype(threads)::value, 0, st>>>(t, keep_lens, ws);
        });
    hipError_t e = by_threads(t.num_seqs, [&](auto threads) {
        tables_truncate_kernel<false, decltype(threads)::value><<<1, decltype(threads)::value, 0, st>>>(t, keep_lens, ws);
    });
    if (e != hipSuccess) return e;
    tables_truncate_fill_kernel<<<fill_grid(most), 256, 0, st>>>(t, ws);
    return hipGetLastError();
}

}  // namespace shiftattn
