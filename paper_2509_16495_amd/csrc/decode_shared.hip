// Decode attention of a batch whose groups of sequences have the first blocks of their tables in common (shiftattn_decode_shared).
#include "decode_body.h"

namespace shiftattn {

namespace {

using namespace decode_flat;

constexpr int kWaves = 4;
constexpr int kWorkgroups = 512;      // two resident per compute unit
constexpr int kMaxPairs = 1024;       // (sequence, KV head) pairs of a launch
constexpr int kMaxGroups = 512;
constexpr int kStep = 64;             // keys a workgroup takes at once: four blocks, one loaded by each wavefront
constexpr int kTileCols = 128;        // (sequence, head) columns of a tile; groups of up to 64 take the two halves of a step's keys apart
constexpr int kMaxRanges = 240;       // ranges that the shared keys of a tile are cut into
constexpr int kMinSteps = 4;          // steps of a range
constexpr int kPrefixWeight = 1, kSuffixWeight = 3;   // time of a step, and of 32 tokens for each of a workgroup's wavefronts

// the shared part of a sequence, for the merge: items (tile, KV head) of its group start at line0, `steps` each
struct alignas(32) SharedRow {
    int line0, steps, tiles, base, col0, range, wide, reserved;   // tiles 0: it shares nothing
};

struct GroupIndex {
    int eff[kMaxGroups];               // blocks in common
    int line[kMaxGroups + 1];          // steps of all items of the groups in front
    uint16_t offs[kMaxGroups + 1], base[kMaxGroups + 1], leader[kMaxGroups];   // first sequence, items in front, the sequence whose table is read
    int sums[2][kWaves];
};

struct SharedArgs {
    const uint16_t* q;
    uint16_t* cache;
    const int32_t* block_table;
    const int32_t* seq_lens;
    const int32_t* group_offsets;
    const int32_t* shared_lens;
    const float* scales;
    float* o_part;        // partial results of the sequences' own keys, as in decode_flat_body
    float* ml_part;
    int2* plan;
    float* o_shared;      // [workgroup + item][column][D], and (reference, sum) pairs
    float* ml_shared;
    SharedRow* rows;
    int64_t q_stride;
    int num_groups, first_seq, num_seqs, max_blocks, hq_l, hkv_l, r_min, range_min;
    float c;
};

__device__ inline int wave_scan(int v) {   // inclusive
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // row_shr:2
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);  // row_shr:4
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);  // row_shr:8
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // lane 15 of a row into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 into rows 2 and 3
    return v;
}

// items (tiles) of a group of m sequences for one KV head
__device__ inline int tiles_of(int m, int G) { return (m * G + kTileCols - 1) / kTileCols; }

// A workgroup's share of the line of shared keys: steps [start, end).
template <bool kFp8, int kScales>
__device__ __attribute__((always_inline)) inline void shared_keys_body(const SharedArgs& a, const GroupIndex& gi, unsigned char* smem, int start, int end, int wg) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int G = a.hq_l / a.hkv_l;
    const int col = lane & 15, grp = lane >> 4;
    // LDS: two buffers of a step, each two groups of 32 tokens parked as in decode_flat_body (its comment has the layout)
    const int b = wave & 1;                         // this wavefront's block of its group
    unsigned char* const park = smem + (wave >> 1) * kStageBytes;
    int kw[4], kr[4];
    {
        const int r0 = lane >> 4, p = lane & 15;
        const int at = r0 * 256 + ((p ^ r0) << 4);
        const int tau_a = ((col >> 2) << 3) + (col & 3);
        const int k_sel = tau_a >> 4, k_off_a = tau_a & 15;
        const int rat = k_sel * 4096 + k_off_a * 256 + ((grp ^ k_off_a ^ (4 * k_sel)) << 4);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            kw[x] = at ^ (64 * x) ^ (64 * b);
            kr[x] = rat ^ (64 * x);
        }
    }
    const int vw = 8192 + ((lane ^ ((lane >> 4) & 1)) << 4);
    const int vr = 8192 + (grp >> 1) * 4096 + (((2 * col + (grp & 1)) ^ ((col >> 3) & 1)) << 4);
    int kw8 = 0, vw8 = 0;
    if constexpr (kFp8) {
        const int r8 = lane >> 3, pc = lane & 7;
        kw8 = r8 * 256 + (((2 * pc) ^ (r8 & 3) ^ (4 * (lane >> 5))) << 4);
        const int l31 = lane & 31;
        vw8 = 8192 + 1024 * (lane >> 5) + (((2 * l31) ^ ((l31 >> 3) & 1)) << 4);
    }

    // ---- a position on the line: its group, item and the item's first and last step (all scalar) ----
    struct Item {
        int group, local, begin, end;
    };
    auto item_at = [&](int pos) -> Item {
        int g = 0;
        for (int at = 0; at < a.num_groups; at += 64) {   // the last group that starts at or before pos and is not empty
            const int i = at + lane;
            const uint64_t m = __builtin_amdgcn_ballot_w64(i < a.num_groups && gi.line[i] <= pos && gi.line[min(i, a.num_groups - 1) + 1] > pos);
            if (m) {
                g = at + __builtin_ctzll(m);
                break;
            }
        }
        g = __builtin_amdgcn_readfirstlane(g);
        const int line0 = __builtin_amdgcn_readfirstlane(gi.line[g]);
        const int steps = (__builtin_amdgcn_readfirstlane(gi.eff[g]) + 3) / 4;
        const int local = (pos - line0) / steps;
        return {g, local, line0 + local * steps, line0 + (local + 1) * steps};
    };
    u32x4 fk[4], fv[4];
    float sc_k = 1.f, sc_v = 1.f;
    auto load_step = [&](const Item& it, int pos) {
        const int eff = __builtin_amdgcn_readfirstlane(gi.eff[it.group]);
        const int m = __builtin_amdgcn_readfirstlane(gi.offs[it.group + 1]) - __builtin_amdgcn_readfirstlane(gi.offs[it.group]);
        const int head = it.local / tiles_of(m, G);
        const int leader = __builtin_amdgcn_readfirstlane(gi.leader[it.group]);
        const int64_t blk = a.block_table[static_cast<size_t>(leader) * a.max_blocks + min((pos - it.begin) * 4 + wave, eff - 1)];
        if constexpr (kFp8) {
            if constexpr (kScales != 0) {
                sc_k = a.scales[(static_cast<size_t>(blk) * a.hkv_l + head) * 2];
                sc_v = a.scales[(static_cast<size_t>(blk) * a.hkv_l + head) * 2 + 1];
            }
            const u32x4* src = reinterpret_cast<const u32x4*>(reinterpret_cast<const unsigned char*>(a.cache) + cache_part_offset(blk, head, 0, a.hkv_l, kD)) + lane;
#pragma unroll
            for (int j = 0; j < 2; ++j) fk[j] = src[64 * j], fv[j] = src[128 + 64 * j];
        } else {
            const u32x4* src = reinterpret_cast<const u32x4*>(a.cache + cache_part_offset(blk, head, 0, a.hkv_l, kD)) + lane;
#pragma unroll
            for (int j = 0; j < 4; ++j) fk[j] = src[64 * j], fv[j] = src[256 + 64 * j];
        }
    };
    auto park_step = [&](int buffer) {
        unsigned char* my = park + buffer * 2 * kStageBytes;
        if constexpr (kFp8) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 lo, hi;
                widen_fp8(fk[j], lo, hi, sc_k);
                const int ka = (kw8 ^ (64 * ((2 * j) ^ b))) + 4096 * b + 2048 * j;
                *reinterpret_cast<u32x4*>(my + ka) = lo;
                *reinterpret_cast<u32x4*>(my + (ka ^ 16)) = hi;
                widen_fp8(fv[j], lo, hi, sc_v);
                const int va = vw8 + 4096 * b + 2048 * j;
                *reinterpret_cast<u32x4*>(my + va) = lo;
                *reinterpret_cast<u32x4*>(my + (va ^ 16)) = hi;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                *reinterpret_cast<u32x4*>(my + kw[j] + 4096 * b + 1024 * j) = fk[j];
                *reinterpret_cast<u32x4*>(my + vw + 4096 * b + 1024 * j) = fv[j];
            }
        }
    };

    bf16x8 qf[2][4];
    f32x4 o[2][8];
    float m_run[2], l_run[2];
    const float ref_least = -3.4e38f / fmaxf(a.c, 1.f);   // the reference stays finite (times c too) where all logits are minus infinity
    int cols = 0, col0 = 0, first = 0, head = 0;          // columns of the group, this wavefront's first one, the group's first sequence
    bool wide = true;
    auto open_item = [&](const Item& it) {
        first = __builtin_amdgcn_readfirstlane(gi.offs[it.group]);
        const int m = __builtin_amdgcn_readfirstlane(gi.offs[it.group + 1]) - first;
        const int tiles = tiles_of(m, G);
        head = it.local / tiles;
        cols = m * G;
        wide = cols > kTileCols / 2;
        col0 = (it.local - head * tiles) * kTileCols + 32 * (wide ? wave : wave & 1);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int cc = col0 + 16 * x + col;
            const int member = cc / G;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                u32x4 v = {0u, 0u, 0u, 0u};
                if (cc < cols)
                    v = *reinterpret_cast<const u32x4*>(a.q + static_cast<size_t>(first + member) * a.q_stride +
                                                        static_cast<size_t>(head * G + cc - member * G) * kD + 8 * (grp + 4 * kk));
                qf[x][kk] = as_bf16x8(v);
            }
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) o[x][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
            m_run[x] = -INFINITY;
            l_run[x] = 0.f;
        }
    };
    auto close_item = [&](const Item& it) {   // this workgroup's partial of the item
        const size_t slot = static_cast<size_t>(wg) + __builtin_amdgcn_readfirstlane(gi.base[it.group]) + it.local;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float l = l_run[x] + __shfl_xor(l_run[x], 16);
            l += __shfl_xor(l, 32);
            if (col0 + 16 * x + col < cols) {
                const size_t row = slot * kTileCols + 32 * wave + 16 * x + col;   // (narrow: the second half of the keys is 64 columns on)
                float* dst = a.o_shared + row * kD + 4 * grp;
#pragma unroll
                for (int mt = 0; mt < 8; ++mt) *reinterpret_cast<f32x4*>(dst + 16 * mt) = o[x][mt];
                if (grp == 0) {
                    a.ml_shared[row * 2] = m_run[x] * a.c;
                    a.ml_shared[row * 2 + 1] = l;
                }
            }
        }
    };
    // the 32 tokens of a parked group, `there` of which exist
    auto take_group = [&](const unsigned char* my, int there) {
        f32x4 sa[2], sb[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) sa[x] = sb[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const bf16x8 ka = as_bf16x8(*reinterpret_cast<const u32x4*>(my + kr[kk]));
            const bf16x8 kb = as_bf16x8(*reinterpret_cast<const u32x4*>(my + kr[kk ^ 1] + 1024));
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                sa[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, qf[x][kk], sa[x], 0, 0, 0);
                sb[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, qf[x][kk], sb[x], 0, 0, 0);
            }
        }
        u32x4 vf[8];
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) vf[mt] = *reinterpret_cast<const u32x4*>(my + vr + 512 * mt);
        if (there < kGroup) {   // uniform; whole blocks are shared, so a lane's eight tokens exist or do not
            const bool gone = 8 * grp >= there;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (gone) sa[x][r] = sb[x][r] = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < 8; ++mt)
                if (gone) vf[mt] = u32x4{0u, 0u, 0u, 0u};
        }
        bf16x8 pf[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float mx = fmaxf(fmaxf(fmaxf(sa[x][0], sa[x][1]), fmaxf(sa[x][2], sa[x][3])), fmaxf(fmaxf(sb[x][0], sb[x][1]), fmaxf(sb[x][2], sb[x][3])));
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float m_new = fmaxf(fmaxf(m_run[x], mx), ref_least);
            const float alpha = __builtin_amdgcn_exp2f((m_run[x] - m_new) * a.c);
            const float mc = m_new * a.c;
            float pa[4], pb[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                pa[r] = __builtin_amdgcn_exp2f(fmaf(sa[x][r], a.c, -mc));
                pb[r] = __builtin_amdgcn_exp2f(fmaf(sb[x][r], a.c, -mc));
            }
            l_run[x] = l_run[x] * alpha + ((pa[0] + pa[1]) + (pa[2] + pa[3])) + ((pb[0] + pb[1]) + (pb[2] + pb[3]));
            m_run[x] = m_new;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                pf[x][r] = static_cast<__bf16>(pa[r]);
                pf[x][4 + r] = static_cast<__bf16>(pb[r]);
            }
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) o[x][mt] *= alpha;
        }
#pragma unroll
        for (int mt = 0; mt < 8; ++mt)
#pragma unroll
            for (int x = 0; x < 2; ++x) o[x][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[mt]), pf[x], o[x][mt], 0, 0, 0);
    };

    // ---- steps: while step i is computed from one buffer, step i + 1 is parked in the other and the loads of step i + 2 are in flight ----
    Item now = item_at(start), next = now;
    load_step(now, start);
    open_item(now);
    park_step(0);
    if (start + 1 < end) {
        if (start + 1 >= next.end) next = item_at(start + 1);
        load_step(next, start + 1);
    }
    __syncthreads();
    for (int pos = start; pos < end; ++pos) {
        const int buffer = (pos - start) & 1;
        Item after = next;
        if (pos + 1 < end) {   // uniform over the workgroup, as all branches around barriers here
            park_step(buffer ^ 1);
            if (pos + 2 < end) {
                if (pos + 2 >= after.end) after = item_at(pos + 2);
                load_step(after, pos + 2);
            }
        }
        const unsigned char* at = smem + buffer * 2 * kStageBytes;
        const int left = (__builtin_amdgcn_readfirstlane(gi.eff[now.group]) - (pos - now.begin) * 4) * kBlockSize;
        if (wide) {
            take_group(at, left);
            take_group(at + kStageBytes, left - kGroup);
        } else {
            take_group(at + (wave >> 1) * kStageBytes, left - (wave >> 1) * kGroup);
        }
        if (pos + 1 >= end || pos + 1 >= now.end) {
            close_item(now);
            if (pos + 1 < end) open_item(next);
        }
        now = next;
        next = after;
        __syncthreads();
    }
}

template <bool kFp8, bool kAppend, bool kBlockScales>
__global__ __launch_bounds__(kWaves * 64, 2) void decode_shared_kernel(SharedArgs a, AppendArgs ap) {
    __shared__ __attribute__((aligned(16))) unsigned char smem[kWaves * kStageBytes];
    __shared__ int index[kMaxPairs + 1 + 16];
    __shared__ int from[kMaxPairs];
    __shared__ GroupIndex gi;
    const int G = a.hq_l / a.hkv_l, n = a.num_seqs;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kThreads = kWaves * 64, kSeqs = kMaxPairs / kThreads, kGroupsPer = kMaxGroups / kThreads;

    // ---- which sequences share how many blocks: the least that any of a group's sequences has in front of its last token's block ----
    int len[kSeqs];
#pragma unroll
    for (int x = 0; x < kSeqs; ++x) len[x] = tid + x * kThreads < n ? a.seq_lens[tid + x * kThreads] : 0;
    for (int g = tid; g <= a.num_groups; g += kThreads) {
        gi.offs[g] = static_cast<uint16_t>(min(max(a.group_offsets[g] - a.first_seq, 0), n));
        if (g < a.num_groups) {
            gi.eff[g] = max(a.shared_lens[g], 0) / kBlockSize;
            gi.line[g] = n;   // the first sequence that is no padding
        }
    }
    __syncthreads();
    int mine[kSeqs];
#pragma unroll
    for (int x = 0; x < kSeqs; ++x) {
        const int s = tid + x * kThreads;
        mine[x] = -1;
        if (s < n && len[x] > 0 && a.num_groups > 0 && s >= gi.offs[0] && s < gi.offs[a.num_groups]) {
            int lo = 0, hi = a.num_groups;   // the last group with offs <= s: the one that is not empty among those that start alike
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (gi.offs[mid] <= s) lo = mid; else hi = mid;
            }
            mine[x] = lo;
            atomicMin(&gi.eff[lo], (len[x] - 1) / kBlockSize);
            atomicMin(&gi.line[lo], s);
        }
    }
    __syncthreads();
    int steps_of[kGroupsPer], items_of[kGroupsPer], line = 0, items = 0;
#pragma unroll
    for (int x = 0; x < kGroupsPer; ++x) {   // thread t owns kGroupsPer groups from kGroupsPer t on
        const int g = tid * kGroupsPer + x;
        steps_of[x] = items_of[x] = 0;
        if (g < a.num_groups) {
            const int m = gi.offs[g + 1] - gi.offs[g];
            if (m < 2 || gi.line[g] >= n) gi.eff[g] = 0;
            gi.leader[g] = static_cast<uint16_t>(gi.line[g]);
            if (gi.eff[g] > 0) {
                items_of[x] = a.hkv_l * tiles_of(m, G);
                steps_of[x] = items_of[x] * ((gi.eff[g] + 3) / 4);
            }
        }
        line += steps_of[x];
        items += items_of[x];
    }
    const int line_incl = wave_scan(line), items_incl = wave_scan(items);
    if (lane == 63) gi.sums[0][wave] = line_incl, gi.sums[1][wave] = items_incl;
    __syncthreads();
    int line_run = line_incl - line, items_run = items_incl - items, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) line_run += gi.sums[0][w], items_run += gi.sums[1][w];
        total += gi.sums[0][w];
    }
#pragma unroll
    for (int x = 0; x < kGroupsPer; ++x) {
        const int g = tid * kGroupsPer + x;
        if (g <= a.num_groups) {
            gi.line[g] = line_run;
            gi.base[g] = static_cast<uint16_t>(items_run);
        }
        line_run += steps_of[x];
        items_run += items_of[x];
    }
    if (tid == 0 && a.num_groups == kMaxGroups) gi.line[kMaxGroups] = total;
    int own = 0;   // groups of 32 tokens that the sequences have to themselves
#pragma unroll
    for (int x = 0; x < kSeqs; ++x) {
        const int s = tid + x * kThreads;
        const int f = mine[x] >= 0 ? gi.eff[mine[x]] : 0;
        from[s] = f;
        own += (max(len[x], 0) - f * kBlockSize + kGroup - 1) / kGroup;
    }
    own = wave_scan(own);
    __syncthreads();
    if (lane == 63) gi.sums[0][wave] = own;
    __syncthreads();
    own = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) own += gi.sums[0][w];

    // ---- how many workgroups take shared keys (the first ones), and how many steps each ----
    const int64_t cost_p = static_cast<int64_t>(total) * kPrefixWeight, cost_s = static_cast<int64_t>(own) * a.hkv_l * kSuffixWeight / kWaves + 1;
    int n_p = 0, range = a.range_min;
    if (total > 0) {
        n_p = min(max(static_cast<int>(kWorkgroups * cost_p / (cost_p + cost_s)), 1), kWorkgroups - 1);
        range = max((total + n_p - 1) / n_p, a.range_min);
        n_p = (total + range - 1) / range;
    }
    n_p = __builtin_amdgcn_readfirstlane(n_p);
    range = __builtin_amdgcn_readfirstlane(range);
    const int wg = blockIdx.x;
    if (wg == n_p) {   // for the merge
#pragma unroll
        for (int x = 0; x < kSeqs; ++x) {
            const int s = tid + x * kThreads;
            if (s >= n) continue;
            SharedRow r = {0, 0, 0, 0, 0, range, 0, 0};
            const int g = mine[x];
            if (g >= 0 && gi.eff[g] > 0) {
                const int m = gi.offs[g + 1] - gi.offs[g];
                r = SharedRow{gi.line[g], (gi.eff[g] + 3) / 4, tiles_of(m, G), gi.base[g], (s - gi.offs[g]) * G, range, m * G > kTileCols / 2, 0};
            }
            a.rows[s] = r;
        }
    }
    if (wg < n_p) {
        shared_keys_body<kFp8, kBlockScales ? 1 : 0>(a, gi, smem, wg * range, min((wg + 1) * range, total), wg);
        return;
    }
    decode_flat_body<kFp8, kAppend, kWaves, false, kBlockScales ? 1 : 0, kMaxPairs, true>(
        a.q, a.q_stride, a.cache, a.block_table, a.max_blocks, a.seq_lens, a.o_part, a.ml_part, a.plan, n, a.hq_l, a.hkv_l, a.c, a.r_min, ap, smem, index, wg - n_p,
        kWorkgroups - n_p, a.scales, from);
}

// One workgroup per output row: the parts of its own keys, then those of the shared ones, summed in that order with the weights of their
// references.  32 threads (four elements of the head each) form a group; group i sums parts i, i + groups, ...
constexpr int kMergeParts = kMaxParts;
template <int kGroups>
__global__ __launch_bounds__(32 * kGroups) void combine_shared_kernel(const float* __restrict__ o_part, const float* __restrict__ ml_part, const int2* __restrict__ plan,
                                                                      const float* __restrict__ o_shared, const float* __restrict__ ml_shared,
                                                                      const SharedRow* __restrict__ rows, const int32_t* __restrict__ seq_lens, int hq_l, int G,
                                                                      uint16_t* __restrict__ out, int64_t out_stride, float out_scale) {
    constexpr int kThreads = 32 * kGroups;
    __shared__ float w_s[kMergeParts];
    __shared__ float red_s[2][kThreads / 64];
    __shared__ __attribute__((aligned(16))) float acc_s[kGroups][kD];
    const int seq = blockIdx.x / hq_l, j = blockIdx.x % hq_l, tid = threadIdx.x, pg = tid >> 5, lane = tid & 63;
    uint16_t* dst = out + static_cast<size_t>(seq) * out_stride + static_cast<size_t>(j) * kD;
    const int2 e = plan[seq * (hq_l / G) + j / G];
    const SharedRow r = rows[seq];
    const bool there = seq_lens[seq] > 0;
    const size_t own0 = static_cast<size_t>(e.x) * G + j % G;
    size_t shared0 = 0;
    int shared_parts = 0;
    if (r.tiles > 0) {
        const int c = r.col0 + j % G, tile = r.wide ? c / kTileCols : 0, local = tile + r.tiles * (j / G);
        const int begin = r.line0 + local * r.steps, w0 = begin / r.range, w1 = (begin + r.steps - 1) / r.range;
        shared0 = (static_cast<size_t>(w0) + r.base + local) * kTileCols + (c - tile * kTileCols);
        shared_parts = (w1 - w0 + 1) * (r.wide ? 1 : 2);
    }
    const int np = there ? min(e.y + shared_parts, kMergeParts) : 0;
    const int stride = r.wide ? kTileCols : kTileCols / 2;   // rows between a shared part and the next
    auto part = [&](int c, const float*& o, const float*& ml) {
        if (c < e.y) {
            const size_t row = own0 + static_cast<size_t>(c) * G;
            o = o_part + row * kD;
            ml = ml_part + row * 2;
        } else {
            const size_t row = shared0 + static_cast<size_t>(c - e.y) * stride;
            o = o_shared + row * kD;
            ml = ml_shared + row * 2;
        }
    };
    float m_loc = -INFINITY;
    for (int c = tid; c < np; c += kThreads) {
        const float *o, *ml;
        part(c, o, ml);
        w_s[c] = ml[0];
        m_loc = fmaxf(m_loc, ml[0]);
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) m_loc = fmaxf(m_loc, __shfl_xor(m_loc, x));
    if (lane == 0) red_s[0][tid >> 6] = m_loc;
    __syncthreads();
    float m_star = red_s[0][0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) m_star = fmaxf(m_star, red_s[0][w]);
    float l_loc = 0.f;
    for (int c = tid; c < np; c += kThreads) {
        const float *o, *ml;
        part(c, o, ml);
        const float w = w_s[c] == -INFINITY ? 0.f : exp2f(w_s[c] - m_star);
        w_s[c] = w;
        l_loc = fmaf(ml[1], w, l_loc);
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) l_loc += __shfl_xor(l_loc, x);
    if (lane == 0) red_s[1][tid >> 6] = l_loc;
    __syncthreads();
    float l_star = red_s[1][0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) l_star += red_s[1][w];
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int c = pg; c < np; c += kGroups) {
        const float *o, *ml;
        part(c, o, ml);
        const f32x4 v = *reinterpret_cast<const f32x4*>(o + 4 * (tid & 31));
        const float w = w_s[c];
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[x] = fmaf(v[x], w, acc[x]);
    }
    *reinterpret_cast<f32x4*>(&acc_s[pg][4 * (tid & 31)]) = acc;
    __syncthreads();
    if (tid < kD) {
        float sum = acc_s[0][tid];
#pragma unroll
        for (int g = 1; g < kGroups; ++g) sum += acc_s[g][tid];
        const float inv = l_star > 0.f ? out_scale / l_star : 0.f;   // (a row without keys is zero)
        dst[tid] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(sum * inv));
    }
}

// sequences per launch: what its index holds, and a token line below 2^31
int seqs_per_launch(int max_seq_len, const AttnShape& a) {
    const int64_t padded = static_cast<int64_t>(max_seq_len > 0 ? max_seq_len : 1) / kGroup * kGroup + kGroup;
    const int64_t by_line = (static_cast<int64_t>(0x7FFFFFFF) - kGroup) / padded / a.hkv_l, by_index = kMaxPairs / a.hkv_l;
    return static_cast<int>(by_line < by_index ? by_line : by_index);
}
int64_t most_items(int n, int num_groups, const AttnShape& a) {
    return static_cast<int64_t>(a.hkv_l) * (static_cast<int64_t>(n) * (a.hq_l / a.hkv_l) / kTileCols + (num_groups < n ? num_groups : n));
}
// tokens per wavefront so that no row has more than 480 parts of its own, steps per range so that it has no more than 482 shared ones
int own_r_min(int max_seq_len) {
    const int r = (max_seq_len / 480 + kGroup) / kGroup * kGroup;
    return r < 2 * kGroup ? 2 * kGroup : r;
}
int range_min(int max_seq_len) {
    const int r = (max_seq_len / kStep + kMaxRanges) / kMaxRanges;
    return r < kMinSteps ? kMinSteps : r;
}
size_t rows_of(int n, const AttnShape& a) { return decode_mfma_rows_for(kWorkgroups * kWaves, n, a); }
size_t slots_of(int n, int num_groups, const AttnShape& a) { return kWorkgroups + static_cast<size_t>(most_items(n, num_groups, a)); }

}  // namespace

bool decode_shared_supported(const AttnShape& a, int num_seqs, int max_seq_len, int num_groups) {
    if (num_groups < 1 || num_groups > kMaxGroups || !decode_mfma_supported(a, num_seqs, max_seq_len) || a.hkv_l > kMaxPairs) return false;
    const int per = seqs_per_launch(max_seq_len, a), n = num_seqs < per ? num_seqs : per;
    return per >= 1 && most_items(n, num_groups, a) < 0xFFFF && most_items(n, num_groups, a) * (max_seq_len / kStep + 1) < 0x7FFFFFFF;
}

size_t decode_shared_workspace(int num_seqs, int max_seq_len, int num_groups, const AttnShape& a) {
    const int per = seqs_per_launch(max_seq_len, a), n = num_seqs < per ? num_seqs : per;
    return (rows_of(n, a) + slots_of(n, num_groups, a) * kTileCols) * (kD + 2) * sizeof(float) + static_cast<size_t>(n) * (a.hkv_l * sizeof(int2) + sizeof(SharedRow)) + 32;
}

hipError_t launch_decode_shared(const void* q, const void* k_new, const void* v_new, const int64_t* slots, void* cache, const int32_t* block_table,
                                const int32_t* seq_lens, int num_seqs, int max_seq_len, const int32_t* group_offsets, const int32_t* shared_lens,
                                int num_groups, void* out, void* workspace, const AttnShape& a, hipStream_t st) {
    const bool append = k_new != nullptr;
    const int per = seqs_per_launch(max_seq_len, a), G = a.hq_l / a.hkv_l;
    for (int s0 = 0; s0 < num_seqs; s0 += per) {  // runs share the workspace: same stream, one after the other
        const int n = num_seqs - s0 < per ? num_seqs - s0 : per;
        const size_t rows = rows_of(n, a), shared = slots_of(n, num_groups, a) * kTileCols;
        float* o_part = static_cast<float*>(workspace);
        float* o_shared = o_part + rows * kD;
        float* ml_part = o_shared + shared * kD;
        float* ml_shared = ml_part + rows * 2;
        int2* plan = reinterpret_cast<int2*>(ml_shared + shared * 2);
        SharedRow* info = reinterpret_cast<SharedRow*>((reinterpret_cast<uintptr_t>(plan + static_cast<size_t>(n) * a.hkv_l) + 31) & ~static_cast<uintptr_t>(31));
        const SharedArgs args = {static_cast<const uint16_t*>(q) + static_cast<size_t>(s0) * a.q_stride, static_cast<uint16_t*>(cache),
                                 block_table + static_cast<size_t>(s0) * a.max_blocks, seq_lens + s0, group_offsets, shared_lens, a.kv_scales, o_part, ml_part, plan,
                                 o_shared, ml_shared, info, a.q_stride, num_groups, s0, n, a.max_blocks, a.hq_l, a.hkv_l, own_r_min(max_seq_len),
                                 range_min(max_seq_len), a.scale * a.k_scale * 1.4426950408889634f};
        const AppendArgs ap = {append ? static_cast<const uint16_t*>(k_new) + static_cast<size_t>(s0) * a.kv_stride : nullptr,
                               append ? static_cast<const uint16_t*>(v_new) + static_cast<size_t>(s0) * a.kv_stride : nullptr,
                               append ? slots + s0 : nullptr, a.kv_stride, a.k_scale, a.v_scale, a.kv_scales};
        auto launch = [&](auto kernel) { kernel<<<kWorkgroups, kWaves * 64, 0, st>>>(args, ap); };
        if (a.block_scales) {
            if (append) launch(decode_shared_kernel<true, true, true>);
            else launch(decode_shared_kernel<true, false, true>);
        } else if (a.kv_fp8()) {
            if (append) launch(decode_shared_kernel<true, true, false>);
            else launch(decode_shared_kernel<true, false, false>);
        } else {
            if (append) launch(decode_shared_kernel<false, true, false>);
            else launch(decode_shared_kernel<false, false, false>);
        }
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        const unsigned grid = static_cast<unsigned>(n) * a.hq_l;
        uint16_t* out_run = static_cast<uint16_t*>(out) + static_cast<size_t>(s0) * a.out_stride;
        if (grid >= 1024)
            combine_shared_kernel<4><<<grid, 128, 0, st>>>(o_part, ml_part, plan, o_shared, ml_shared, info, seq_lens + s0, a.hq_l, G, out_run, a.out_stride, a.v_scale);
        else
            combine_shared_kernel<16><<<grid, 512, 0, st>>>(o_part, ml_part, plan, o_shared, ml_shared, info, seq_lens + s0, a.hq_l, G, out_run, a.out_stride, a.v_scale);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace shiftattn
