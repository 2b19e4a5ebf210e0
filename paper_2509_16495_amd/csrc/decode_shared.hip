// Decode attention of a batch whose groups of sequences have the first blocks of their tables in common (shiftattn_decode_shared).
//
// The keys of a sequence are two ranges: S, the blocks in common, and E, its own.  With a reference m_R for each range (any finite number;
// the result does not depend on it) and
//     l_R = sum_{t in R} 2^(c z_t - m_R),   o_R = sum_{t in R} 2^(c z_t - m_R) v_t,   m = max m_R,
// the row is  sum_R 2^(m_R - m) o_R / sum_R 2^(m_R - m) l_R.  o_S needs keys and values of S once for all (sequence, head) pairs of a group,
// which are then columns of a matrix product (S^T = K Q^T, O^T = V^T P^T) like the heads of one sequence are in the plain kernel.
//
// One launch takes both kinds of ranges, a second one joins them.  Every workgroup works out the same plan from lengths and offsets, about
// 3 us of which most is dependent loads; a launch of its own for the plan took 4 us more.  Workgroups are dealt out by the work that either
// kind weighs (shared_deal.h); a unit of shared keys is (tile of columns, KV head, range of keys), a workgroup's own keys are the plain kernel's.
//
// What bounds it: the bytes read once are few (256 sequences of 8 heads behind 32768 tokens: 160 MB, 29 us at the copy rate), but each 32
// tokens cost a tile of 128 columns 128 matrix instructions of 16.4 clocks and 4096 exponentials: a wavefront's share of the matrix and of the
// vector instructions takes about 880 clocks of a SIMD (0.37 us).  Two tiles on a compute unit, a wavefront of each on a SIMD, take 0.8 to 1.0 us for
// a group of both: that sum and a tenth to a third on top of it.  A lone tile takes 0.85 us for its group, twice its sum: it waits (for operands out of LDS, for the
// products that its exponentials need, for the other wavefronts), with nothing beside it that would fill the time.  A launch has both, and wavefronts
// that read the sequences' own keys: over all of 256 sequences behind 32768 tokens the matrix units are busy for a quarter of the time, and so is LDS.
// Neither the barrier (1 us of 55 without it), nor keys out of a hot L2, nor 32x32x16 instructions (4 % less for one workgroup, 5 % more for two), nor
// exponentials in front of the first matrix instructions change that.  Few sequences are bounded by the fixed parts: plan 3 us, first loads 3, partial
// results 2, the merge 4 to 9.  256 sequences behind 32768 tokens: 67 us, where the plain kernel reads 17 GB in 607.
// Workgroups of eight wavefronts whose halves take every other group and add their sums in LDS write half as many parts (64 sequences behind
// 32768 tokens 28.1 us against 31.7), but a compute unit draws only so many bytes, and those with the sequences' own keys are then fewer (256 with
// up to 2000 of their own 84 to 113 us against 67): not taken.
#include "decode_body.h"
#include "shared_deal.h"

namespace shiftattn {

namespace {

using namespace decode_flat;
using namespace shared_deal;

constexpr int kWaves = 4;
constexpr int kMaxPairs = 1024;       // (sequence, KV head) pairs of a launch
constexpr int kMaxGroups = 512;
constexpr double kPlainBytes = 40.0e6;   // cache up to which a batch is the plain kernel's
constexpr int kMaxRanges = 480;       // ranges that the shared keys of a tile are cut into
constexpr int kMinSteps = 2;          // steps of a range
// A column's reference is set this much (in powers of two) above the largest logit so far, and moves from a sum of a lane's eight weights of kMostSum
// on: weights may grow by 2^13 until it does, and are at most one in the mean, so that a product overflows where the plain kernel's would.  (Rounding
// to bf16 does not depend on the exponent.)  On tiles of 128 columns a growth of 2^8 was 2 % slower, one of 2^40 no faster than one of 2^16.
constexpr float kLead = 13.f, kMostSum = 8.f;

// the shared part of a sequence, for the merge: `parts` partial results in units base + (tile + tiles * head) * ranges and on
struct alignas(32) SharedRow {
    int base, ranges, parts, tiles, col0, cols, reserved[2];   // tiles 0: it shares nothing; cols: of a tile
};

struct GroupIndex {
    int eff[kMaxGroups];                                       // blocks in common
    int units[kMaxGroups + 1];                                 // units (tile, KV head, range) of the groups in front
    uint16_t offs[kMaxGroups + 1], ranges[kMaxGroups], leader[kMaxGroups];   // first sequence, ranges of an item, the sequence whose table is read
    int sums[3][kWaves];
};

// logits become powers of two by c; how far above the largest one a reference is set, and the least one: it stays finite (times c too) where all
// logits are minus infinity
struct Reference {
    float c, lead, least;
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
    float* o_shared;      // [unit][column of the tile][D], and (reference, sum) pairs
    float* ml_shared;
    SharedRow* rows;
    int64_t q_stride;
    int num_groups, first_seq, num_seqs, max_blocks, hq_l, hkv_l, r_min, range_min;
    bool always;          // groups share whatever that costs
    Reference ref;
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

// One unit: the keys of blocks [first_block, end_block) of a group's table for one KV head, met by the columns [col_first, col_end) of
// the group ((sequence, head) pairs of that KV head's heads), up to 128, or up to 32 (kNarrow).
struct Unit {
    const int32_t* table;
    int first_block, end_block, head, col_first, col_end, seq_first, slot;
};

// A wavefront's 32 columns: queries, sums and references.  S^T = K Q^T and O^T += V^T P^T as in decode_flat_body, two tiles of 16 columns
// for each K and V operand read from LDS.
struct Columns {
    bf16x8 q[2][4];
    f32x4 o[2][8];
    float m[2], l[2];

    __device__ void open(const SharedArgs& a, const Unit& u, int col0, int G) {
        const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int cc = col0 + 16 * x + col, member = cc / G;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                u32x4 v = {0u, 0u, 0u, 0u};
                if (cc < u.col_end)
                    v = *reinterpret_cast<const u32x4*>(a.q + static_cast<size_t>(u.seq_first + member) * a.q_stride +
                                                        static_cast<size_t>(u.head * G + cc - member * G) * kD + 8 * (grp + 4 * kk));
                q[x][kk] = as_bf16x8(v);
            }
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) o[x][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
            m[x] = -INFINITY;
            l[x] = 0.f;
        }
    }

    // logits of the 32 tokens parked at `my`: of column tile x, tokens 8 grp .. 8 grp + 3 in s[x] and the next four in s[2 + x]
    __device__ __attribute__((always_inline)) void scores(const unsigned char* my, const int (&kr)[4], f32x4 (&s)[4]) const {
#pragma unroll
        for (int x = 0; x < 4; ++x) s[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const bf16x8 ka = as_bf16x8(*reinterpret_cast<const u32x4*>(my + kr[kk]));
            const bf16x8 kb = as_bf16x8(*reinterpret_cast<const u32x4*>(my + kr[kk ^ 1] + 1024));
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                s[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka, q[x][kk], s[x], 0, 0, 0);
                s[2 + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb, q[x][kk], s[2 + x], 0, 0, 0);
            }
        }
    }

    // P and O += V^T P^T of those tokens, `there` of which exist: 16 or all (blocks that do not are zeros).  kAhead: and the logits of the
    // group parked at `ahead`, their matrix instructions one by one between those of the exponentials, which take about as long.
    template <bool kAhead>
    __device__ __attribute__((always_inline)) void weigh(const unsigned char* my, int vr, f32x4 (&s)[4], int there, const Reference& r, const unsigned char* ahead = nullptr,
                                                         const int* kr = nullptr, f32x4* next = nullptr) {
        u32x4 vf[8];
        const float c = r.c;
        // P is taken against a reference that moves when a sum says that logits are far above it (rounding to bf16 does not depend on the
        // exponent): no maximum is looked for, which was a fifth of the instructions, and the sums are rarely scaled
        float p[4][4], sum[2];
        const float mc0 = m[0] * c, mc1 = m[1] * c;
        auto exp_of = [&](int i) {
            const int x = i & 1, h = (i >> 1) & 1, r = i >> 2;
            p[x + 2 * h][r] = __builtin_amdgcn_exp2f(fmaf(s[x + 2 * h][r], c, x ? -mc1 : -mc0));
        };
        auto add_up = [&](int x) { sum[x] = ((p[x][0] + p[x][1]) + (p[x][2] + p[x][3])) + ((p[2 + x][0] + p[2 + x][1]) + (p[2 + x][2] + p[2 + x][3])); };
        if constexpr (kAhead) {
            bf16x8 kf[8];
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                kf[2 * kk] = as_bf16x8(*reinterpret_cast<const u32x4*>(ahead + kr[kk]));
                kf[2 * kk + 1] = as_bf16x8(*reinterpret_cast<const u32x4*>(ahead + kr[kk ^ 1] + 1024));
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) next[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int kk = i >> 2, h = (i >> 1) & 1, x = i & 1;
                __builtin_amdgcn_sched_barrier(0);
                next[x + 2 * h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[2 * kk + h], q[x][kk], next[x + 2 * h], 0, 0, 0);
                exp_of(i);
                asm volatile("" : "+v"(p[x + 2 * h][kk]));   // (stays here: the compiler would put all of them behind the matrix instructions)
                if (i & 1) vf[i >> 1] = *reinterpret_cast<const u32x4*>(my + vr + 512 * (i >> 1));
            }
            __builtin_amdgcn_sched_barrier(0);
        } else {
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) vf[mt] = *reinterpret_cast<const u32x4*>(my + vr + 512 * mt);
#pragma unroll
            for (int i = 0; i < 16; ++i) exp_of(i);
        }
        add_up(0);
        add_up(1);
        if (there < kGroup || __builtin_amdgcn_ballot_w64(!(sum[0] < kMostSum) || !(sum[1] < kMostSum))) [[unlikely]] {
            // the unit's first tokens, a reference that is too low, NaN, or a block that does not exist
            const int grp = (threadIdx.x & 63) >> 4;
            const bool gone = 8 * grp >= there;             // a lane's eight tokens exist or do not
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (gone) s[x][i] = s[2 + x][i] = -INFINITY;
                    mx = fmaxf(mx, fmaxf(s[x][i], s[2 + x][i]));
                }
                mx = fmaxf(mx, __shfl_xor(mx, 16));
                mx = fmaxf(mx, __shfl_xor(mx, 32));
                const float m_new = fmaxf(fmaxf(m[x], fminf(mx + r.lead, -r.least)), r.least);
                const float alpha = __builtin_amdgcn_exp2f((m[x] - m_new) * c);
                m[x] = m_new;
                l[x] *= alpha;
#pragma unroll
                for (int mt = 0; mt < 8; ++mt) o[x][mt] *= alpha;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[x][i] = __builtin_amdgcn_exp2f(fmaf(s[x][i], c, -m_new * c));
                    p[2 + x][i] = __builtin_amdgcn_exp2f(fmaf(s[2 + x][i], c, -m_new * c));
                }
                add_up(x);
            }
        }
        // P to bf16, off by at most 2^-8 of itself: what the matrix instructions take, as in every decode kernel here (float32 ones are 16 times slower).
        // The sums l are of P as it is, in 32 bits.
        bf16x8 pf[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            l[x] += sum[x];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                pf[x][r] = static_cast<__bf16>(p[x][r]);
                pf[x][4 + r] = static_cast<__bf16>(p[2 + x][r]);
            }
        }
#pragma unroll
        for (int mt = 0; mt < 8; ++mt)
#pragma unroll
            for (int x = 0; x < 2; ++x) o[x][mt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[mt]), pf[x], o[x][mt], 0, 0, 0);
    }

    // the sums of P over all lanes of a column
    __device__ void sum_lanes() {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            l[x] += __shfl_xor(l[x], 16);
            l[x] += __shfl_xor(l[x], 32);
        }
    }
};

// A block of 16 tokens on its way from the cache to LDS, by one wavefront: eight (FP8: four) loads of 1 KiB, parked as decode_flat_body's
// comment says (the block's place b in its group of 32 tokens is 0 or 1).
template <bool kFp8, int kScales>
struct Block {
    static constexpr int kLoads = kFp8 ? 2 : 4;
    u32x4 k[kLoads], v[kLoads];
    float sc_k, sc_v;

    __device__ void load(const SharedArgs& a, int64_t blk, int head) {
        const int lane = threadIdx.x & 63;
        if constexpr (kScales != 0) {
            sc_k = a.scales[(static_cast<size_t>(blk) * a.hkv_l + head) * 2];
            sc_v = a.scales[(static_cast<size_t>(blk) * a.hkv_l + head) * 2 + 1];
        }
        const size_t at = cache_part_offset(blk, head, 0, a.hkv_l, kD);
        const u32x4* src = (kFp8 ? reinterpret_cast<const u32x4*>(reinterpret_cast<const unsigned char*>(a.cache) + at) : reinterpret_cast<const u32x4*>(a.cache + at)) + lane;
#pragma unroll
        for (int j = 0; j < kLoads; ++j) k[j] = src[64 * j], v[j] = src[64 * (kLoads + j)];
    }
    __device__ void clear() {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) k[j] = v[j] = u32x4{0u, 0u, 0u, 0u};
        sc_k = sc_v = 1.f;
    }
    __device__ void park(unsigned char* my, int kw, int vw, int b) const {
        if constexpr (kFp8) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                u32x4 lo, hi;
                widen_fp8(k[j], lo, hi, kScales ? sc_k : 1.f);
                const int ka = (kw ^ (64 * ((2 * j) ^ b))) + 4096 * b + 2048 * j;
                *reinterpret_cast<u32x4*>(my + ka) = lo;
                *reinterpret_cast<u32x4*>(my + (ka ^ 16)) = hi;
                widen_fp8(v[j], lo, hi, kScales ? sc_v : 1.f);
                const int va = vw + 4096 * b + 2048 * j;
                *reinterpret_cast<u32x4*>(my + va) = lo;
                *reinterpret_cast<u32x4*>(my + (va ^ 16)) = hi;
            }
        } else {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                *reinterpret_cast<u32x4*>(my + (kw ^ (64 * (j ^ b))) + 4096 * b + 1024 * j) = k[j];
                *reinterpret_cast<u32x4*>(my + vw + 4096 * b + 1024 * j) = v[j];
            }
        }
    }
};

// A unit's block ids, 64 at a time, one per lane: ids that came one by one through scalar loads made every wait for LDS data wait for them
// too (they share a counter), 1 us a step.  (As built, the load of the window behind is waited for where it is made, with everything else that
// is on its way: once in 32 groups.)
struct BlockIds {
    const int32_t* table;
    int last, at, now, next;   // the window from block `at` on, and the one behind it
    __device__ void open(const Unit& u) {
        table = u.table, last = u.end_block - 1, at = u.first_block;
        now = fetch(at);
        next = fetch(at + 64);
    }
    __device__ int fetch(int from) const { return table[min(from + static_cast<int>(threadIdx.x & 63), last)]; }
    // the id of block i, between `at` and `at` + 127; blocks in front of i are not asked for again
    __device__ int get(int i) {
        if (i >= at + 64) {   // uniform
            at += 64;
            now = next;
            next = fetch(at + 64);
        }
        return __builtin_amdgcn_readlane(now, i - at);
    }
};

// LDS addresses of this lane's pieces
struct Places {
    int kw, vw, kr[4], vr;
    template <bool kFp8>
    __device__ static Places get() {
        const int lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
        Places p;
        if constexpr (kFp8) {
            const int r8 = lane >> 3, pc = lane & 7, l31 = lane & 31;
            p.kw = r8 * 256 + (((2 * pc) ^ (r8 & 3) ^ (4 * (lane >> 5))) << 4);
            p.vw = 8192 + 1024 * (lane >> 5) + (((2 * l31) ^ ((l31 >> 3) & 1)) << 4);
        } else {
            p.kw = (lane >> 4) * 256 + (((lane & 15) ^ (lane >> 4)) << 4);
            p.vw = 8192 + ((lane ^ ((lane >> 4) & 1)) << 4);
        }
        const int tau_a = ((col >> 2) << 3) + (col & 3), k_sel = tau_a >> 4, k_off_a = tau_a & 15;
#pragma unroll
        for (int x = 0; x < 4; ++x) p.kr[x] = (k_sel * 4096 + k_off_a * 256 + ((grp ^ k_off_a ^ (4 * k_sel)) << 4)) ^ (64 * x);
        p.vr = 8192 + (grp >> 1) * 4096 + (((2 * col + (grp & 1)) ^ ((col >> 3) & 1)) << 4);
        return p;
    }
};

// A tile of up to 128 columns, 32 per wavefront, all of which read every key.  LDS is a ring of four groups of 32 tokens (two blocks), of
// which wavefront w brings block w / 2's K or V^T (w % 2).  While the weights and the second product of group g are computed, the
// logits of group g + 1 are (matrix instructions between the vector ones), and groups g + 2 and g + 3 are on their way: straight into LDS, or
// in two sets of registers where codes are widened.  One barrier per group: behind it group g + 1 is there for all, and all are done with
// group g - 1, whose place the next load takes.
// What bounds it stands at the head of this file; LDS, 64 KiB read for each group by the four wavefronts (512 clocks of a compute unit), is not it.
template <bool kFp8, int kScales>
__device__ __attribute__((always_inline)) inline void wide_unit(const SharedArgs& a, const Unit& u, unsigned char* smem) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const Places at = Places::get<kFp8>();
    const int b = wave >> 1, part = wave & 1;
    const int blocks = u.end_block - u.first_block, n = (blocks + 1) / 2;   // groups
    // this lane's places in the 4 KiB of its wavefront's block and part: where it reads (loads into LDS: what belongs to its 16 bytes there) or writes
    int place[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (kFp8) place[j] = j >= 2 ? 0 : (part ? at.vw : at.kw ^ (64 * ((2 * j) ^ b))) + 4096 * b + 2048 * j;
        else place[j] = part ? (lane ^ ((lane >> 4) & 1)) << 4 : ((lane & 48) | ((lane & 15) ^ (lane >> 4) ^ (4 * (j ^ b)))) << 4;
    }
    const int zero_at = 8192 * part + 4096 * b;
    BlockIds ids;
    ids.open(u);
    u32x4 set[2][kFp8 ? 2 : 1];
    float scale[2] = {1.f, 1.f};
    // groups come in order; the block that an odd count leaves out of the last one is zeros
    auto fetch = [&](int g, int which) {
        const int i = u.first_block + 2 * g + b;
        if (i < u.end_block) {
            const int64_t blk = ids.get(i);
            const size_t from = cache_part_offset(blk, u.head, part, a.hkv_l, kD);
            if constexpr (kFp8) {
                if constexpr (kScales != 0) scale[which] = a.scales[(static_cast<size_t>(blk) * a.hkv_l + u.head) * 2 + part];
                const u32x4* src = reinterpret_cast<const u32x4*>(reinterpret_cast<const unsigned char*>(a.cache) + from) + lane;
                set[which][0] = src[0];
                set[which][1] = src[64];
            } else {
                // (no registers are written; the compiler does not count these loads: they are waited for below)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\t"
                             "global_load_lds_dwordx4 %1, %5\n\t"
                             "global_load_lds_dwordx4 %2, %5 offset:1024\n\t"
                             "global_load_lds_dwordx4 %3, %5 offset:2048\n\t"
                             "global_load_lds_dwordx4 %4, %5 offset:0xc00"
                             :: "s"(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(smem)) + (g & 3) * kStageBytes + zero_at), "v"(place[0]), "v"(place[1]), "v"(place[2]),
                                "v"(place[3]), "s"(a.cache + from) : "memory");
            }
        } else if constexpr (kFp8) {
            set[which][0] = set[which][1] = u32x4{0u, 0u, 0u, 0u};
            scale[which] = 1.f;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<u32x4*>(smem + (g & 3) * kStageBytes + zero_at + 1024 * j + 16 * lane) = u32x4{0u, 0u, 0u, 0u};
        }
    };
    auto park = [&](int g, int which) {
        if constexpr (kFp8) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                u32x4 lo, hi;
                widen_fp8(set[which][j], lo, hi, kScales ? scale[which] : 1.f);
                unsigned char* my = smem + (g & 3) * kStageBytes;
                *reinterpret_cast<u32x4*>(my + place[j]) = lo;
                *reinterpret_cast<u32x4*>(my + (place[j] ^ 16)) = hi;
            }
        }
    };
    // loads of all but the newest `kLeft` groups have arrived, LDS is written, for all wavefronts
    auto meet = [&](auto left) {
        if constexpr (kFp8) __syncthreads();
        else if constexpr (decltype(left)::value == 2) asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else if constexpr (decltype(left)::value == 1) asm volatile("s_waitcnt vmcnt(4) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    using Int0 = std::integral_constant<int, 0>;
    using Int1 = std::integral_constant<int, 1>;
    Columns c;
    const int col0 = u.col_first + 32 * wave;
    c.open(a, u, col0, a.hq_l / a.hkv_l);
    fetch(0, 0);
    if (n > 1) fetch(1, 1);
    if constexpr (kFp8) {
        park(0, 0);
        if (n > 1) park(1, 1);
        if (n > 2) fetch(2, 0);
        if (n > 3) fetch(3, 1);
    } else if (n > 2) {
        fetch(2, 0);
    }
    // (the newest groups have no loads where their block does not exist: a wait by count is for those in front of the last one)
    if (n > 3) meet(std::integral_constant<int, 2>{});
    else meet(Int0{});
    f32x4 s0[4], s1[4];
    c.scores(smem, at.kr, s0);
    auto group = [&](int g, f32x4 (&now)[4], f32x4 (&next)[4], auto which) {
        if (g + 3 < n) meet(Int1{});
        else meet(Int0{});
        constexpr int w = decltype(which)::value;
        if constexpr (kFp8) {
            if (g + 2 < n) park(g + 2, w);
            if (g + 4 < n) fetch(g + 4, w);
        } else {
            if (g + 3 < n) fetch(g + 3, 0);
        }
        // (behind the last group: logits of whatever lies there, not used)
        c.weigh<true>(smem + (g & 3) * kStageBytes, at.vr, now, (blocks - 2 * g) * kBlockSize, a.ref, smem + ((g + 1) & 3) * kStageBytes, at.kr, next);
    };
    int g = 0;
#pragma unroll 1
    for (; g + 1 < n; g += 2) {
        group(g, s0, s1, Int0{});
        group(g + 1, s1, s0, Int1{});
    }
    if (g < n) group(g, s0, s1, Int0{});
    __syncthreads();   // (a next unit loads where this one reads)
    c.sum_lanes();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        if (col0 + 16 * x + col < u.col_end) {
            const size_t row = static_cast<size_t>(u.slot) * kTileCols + 32 * wave + 16 * x + col;
            float* dst = a.o_shared + row * kD + 4 * grp;
#pragma unroll
            for (int mt = 0; mt < 8; ++mt) *reinterpret_cast<f32x4*>(dst + 16 * mt) = c.o[x][mt];
            if (grp == 0) *reinterpret_cast<f32x2*>(a.ml_shared + row * 2) = f32x2{c.m[x] * a.ref.c, c.l[x]};
        }
    }
    if constexpr (!kFp8) __builtin_amdgcn_s_waitcnt(0x0F70);   // (vmcnt(0): a next unit counts its own loads only)
}

// A tile of up to 32 columns, which all wavefronts take, each with every fourth group of 32 keys: nothing is shared until the end, where
// their sums are added in LDS.
template <bool kFp8, int kScales>
__device__ __attribute__((always_inline)) inline void narrow_unit(const SharedArgs& a, const Unit& u, unsigned char* smem, float (&ref)[kWaves][kNarrowCols],
                                                                 float (&sums)[kWaves][kNarrowCols]) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, grp = lane >> 4;
    const Places at = Places::get<kFp8>();
    unsigned char* const my = smem + wave * kStageBytes;
    Block<kFp8, kScales> blk[2];
    BlockIds ids;
    ids.open(u);
    auto load = [&](int first) {
        blk[0].load(a, ids.get(first), u.head);
        if (first + 1 < u.end_block) blk[1].load(a, ids.get(first + 1), u.head);
        else blk[1].clear();
    };
    constexpr int kStride = 2 * kWaves;   // blocks from a wavefront's group to its next
    int i = u.first_block + 2 * wave;
    if (i < u.end_block) load(i);
    Columns c;
    c.open(a, u, u.col_first, a.hq_l / a.hkv_l);
#pragma unroll 1
    for (; i < u.end_block; i += kStride) {
        blk[0].park(my, at.kw, at.vw, 0);
        blk[1].park(my, at.kw, at.vw, 1);
        if (i + kStride < u.end_block) load(i + kStride);
        f32x4 s[4];
        c.scores(my, at.kr, s);
        c.weigh<false>(my, at.vr, s, (u.end_block - i) * kBlockSize, a.ref);
    }
    c.sum_lanes();
    if (grp == 0) ref[wave][col] = c.m[0], ref[wave][16 + col] = c.m[1];
    __syncthreads();
    float* mine = reinterpret_cast<float*>(my);   // [column][D], 16 bytes swizzled by the column so that the lanes of a column spread over the banks
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        float top = ref[0][16 * x + col];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ref[w][16 * x + col]);
        const float f = c.m[x] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((c.m[x] - top) * a.ref.c);
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) *reinterpret_cast<f32x4*>(mine + (16 * x + col) * kD + 4 * ((grp + 4 * mt) ^ (col & 7))) = c.o[x][mt] * f;
        if (grp == 0) sums[wave][16 * x + col] = c.l[x] * f;
    }
    __syncthreads();
    // a wavefront adds eight columns, eight lanes each
    {
        const int cc = 8 * wave + (lane >> 3);
        const size_t row = static_cast<size_t>(u.slot) * kTileCols + cc;
        if (u.col_first + cc < u.col_end) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int piece = (lane & 7) + 8 * j;
                f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    v += *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(smem + w * kStageBytes) + cc * kD + 4 * (piece ^ (cc & 7)));
                *reinterpret_cast<f32x4*>(a.o_shared + row * kD + 4 * piece) = v;
            }
            if ((lane & 7) == 0) {
                float top = ref[0][cc], l = sums[0][cc];
#pragma unroll
                for (int w = 1; w < kWaves; ++w) top = fmaxf(top, ref[w][cc]), l += sums[w][cc];
                *reinterpret_cast<f32x2*>(a.ml_shared + row * 2) = f32x2{top * a.ref.c, l};
            }
        }
    }
    __syncthreads();   // (a next unit writes where this one reads)
}

// the first unit that begins at weight x of the line or behind it (weights: where each group's units begin; uniform)
__device__ inline int first_unit(const SharedArgs& a, const GroupIndex& gi, const int* weights, uint32_t x) {
    const int lane = threadIdx.x & 63;
    for (int at = 0; at < a.num_groups; at += 64) {
        const int i = min(at + lane, a.num_groups - 1);
        const uint64_t m = __builtin_amdgcn_ballot_w64(static_cast<uint32_t>(weights[i]) < x && static_cast<uint32_t>(weights[i + 1]) >= x);
        if (m) {
            const int g = __builtin_amdgcn_readfirstlane(at + __builtin_ctzll(m));
            const uint32_t from = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(weights[g])), to = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(weights[g + 1]));
            const int first = __builtin_amdgcn_readfirstlane(gi.units[g]), n = __builtin_amdgcn_readfirstlane(gi.units[g + 1]) - first;
            return first + units_before(x, from, (to - from) / n, n);
        }
    }
    return 0;   // x = 0
}

// units [first, end)
template <bool kFp8, int kScales>
__device__ __attribute__((always_inline)) inline void shared_units(const SharedArgs& a, const GroupIndex& gi, unsigned char* smem, float (&ref)[kWaves][kNarrowCols],
                                                                  float (&sums)[kWaves][kNarrowCols], int first, int end) {
    const int lane = threadIdx.x & 63;
    const int G = a.hq_l / a.hkv_l;
    auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
#pragma unroll 1
    for (int unit = first; unit < end; ++unit) {
        int g = 0;
        for (int at = 0; at < a.num_groups; at += 64) {   // the group that the unit belongs to
            const int i = min(at + lane, a.num_groups - 1);
            const uint64_t m = __builtin_amdgcn_ballot_w64(gi.units[i] <= unit && gi.units[i + 1] > unit);
            if (m) {
                g = uniform(at + __builtin_ctzll(m));
                break;
            }
        }
        const int eff = uniform(gi.eff[g]), ranges = uniform(gi.ranges[g]), seq_first = uniform(gi.offs[g]), cols = (uniform(gi.offs[g + 1]) - seq_first) * G;
        const int local = unit - uniform(gi.units[g]), item = uniform(local / ranges), range = local - item * ranges, tiles = tiles_of(cols);
        const int per = uniform(range_steps(steps_of(eff), ranges)) * 4, head = uniform(item / tiles), col_first = (item - head * tiles) * tile_cols(cols);
        Unit u = {a.block_table + static_cast<size_t>(uniform(gi.leader[g])) * a.max_blocks, range * per, min((range + 1) * per, eff), head, col_first,
                  min(col_first + tile_cols(cols), cols), seq_first, unit};
        if (u.first_block >= eff) continue;   // (uniform) the last ranges of a group may have no keys
        if (cols > kNarrowCols) wide_unit<kFp8, kScales>(a, u, smem);
        else narrow_unit<kFp8, kScales>(a, u, smem, ref, sums);
    }
}

// Every workgroup works out the same plan from the lengths and offsets (a launch of its own for that took longer), and takes its part of it:
// the first ones units of shared keys, the others the sequences' own keys as decode_flat_body deals them out.
template <bool kFp8, bool kAppend, bool kBlockScales>
__global__ __launch_bounds__(kWaves * 64, 2) void decode_shared_kernel(SharedArgs a, AppendArgs ap) {
    __shared__ __attribute__((aligned(16))) unsigned char smem[kWaves * kStageBytes];
    __shared__ int index[kMaxPairs + 1 + 16];
    __shared__ int from[kMaxPairs];
    __shared__ GroupIndex gi;
    float(&ref)[kWaves][kNarrowCols] = *reinterpret_cast<float(*)[kWaves][kNarrowCols]>(index);   // (a workgroup needs the index or these)
    float(&sums)[kWaves][kNarrowCols] = *reinterpret_cast<float(*)[kWaves][kNarrowCols]>(index + kWaves * kNarrowCols);
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
            gi.units[g] = n;   // the first sequence that is no padding
        }
    }
    __syncthreads();
    int mine[kSeqs];
    {
        const int first = gi.offs[0], end = gi.offs[a.num_groups];
#pragma unroll
        for (int x = 0; x < kSeqs; ++x) {
            const int s = tid + x * kThreads;
            mine[x] = -1;
            if (s < n && len[x] > 0 && s >= first && s < end) {
                int lo = 0, hi = a.num_groups;   // the last group with offs <= s: the one that is not empty among those that start alike
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (gi.offs[mid] <= s) lo = mid; else hi = mid;
                }
                if (s < gi.offs[lo + 1] && gi.offs[lo + 1] - gi.offs[lo] >= 2) {   // (a group of one shares nothing)
                    mine[x] = lo;
                    atomicMin(&gi.eff[lo], (len[x] - 1) / kBlockSize);
                    atomicMin(&gi.units[lo], s);
                }
            }
        }
    }
    __syncthreads();
    // ---- what there is to do: steps of all tiles, weighted, and groups of 32 tokens that the sequences have to themselves ----
    auto eff_of = [&](int g) -> int {
        const int members = gi.offs[g + 1] - gi.offs[g];
        return a.always || pays(gi.eff[g], members, members * G) ? gi.eff[g] : 0;
    };
    int cols[kGroupsPer], steps[kGroupsPer];   // thread t owns groups kGroupsPer t and following
    int weight = 0, own = 0;
#pragma unroll
    for (int x = 0; x < kGroupsPer; ++x) {
        const int g = tid * kGroupsPer + x;
        cols[x] = steps[x] = 0;
        if (g < a.num_groups) {
            const int leader = gi.units[g];
            gi.leader[g] = static_cast<uint16_t>(leader);
            if (leader < n) {
                cols[x] = (gi.offs[g + 1] - gi.offs[g]) * G;
                steps[x] = steps_of(eff_of(g));
            }
            weight += steps[x] * a.hkv_l * tiles_of(cols[x]) * cost_of(cols[x]);
        }
    }
#pragma unroll
    for (int x = 0; x < kSeqs; ++x) {
        const int f = mine[x] >= 0 ? eff_of(mine[x]) : 0;
        from[tid + x * kThreads] = f;
        own += (max(len[x], 0) - f * kBlockSize + kGroup - 1) / kGroup;
    }
    weight = wave_scan(weight);
    own = wave_scan(own);
    if (lane == 63) gi.sums[0][wave] = weight, gi.sums[1][wave] = own;
    __syncthreads();
    float cost_p = 0.f, cost_s = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) cost_p += static_cast<float>(gi.sums[0][w]), cost_s += static_cast<float>(gi.sums[1][w]);
    cost_s *= static_cast<float>(a.hkv_l * kOwnCost) / kWaves;
#pragma unroll
    for (int x = 0; x < kGroupsPer; ++x)
        if (steps[x] == 0 && tid * kGroupsPer + x < a.num_groups) gi.eff[tid * kGroupsPer + x] = 0;   // (all have read it)
    // ---- ranges: so long that the shared keys take the workgroups that are theirs by weight ----
    const int wg = blockIdx.x;
    int n_p = 0, all = 0;
    if (cost_p > 0) {   // uniform
        const int range = range_of(cost_p, cost_s);
        int units_of[kGroupsPer], each_of[kGroupsPer], units = 0;
#pragma unroll
        for (int x = 0; x < kGroupsPer; ++x) {
            units_of[x] = each_of[x] = 0;
            if (steps[x] > 0) {
                const int ranges = ranges_of(steps[x], cols[x], range, a.range_min);
                gi.ranges[tid * kGroupsPer + x] = static_cast<uint16_t>(ranges);
                units_of[x] = ranges * a.hkv_l * tiles_of(cols[x]);
                each_of[x] = among(range_steps(steps[x], ranges), cols[x]);
            }
            units += units_of[x];
        }
        const int incl = wave_scan(units);
        if (lane == 63) gi.sums[2][wave] = incl;
        __syncthreads();
        int run = incl - units;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) run += gi.sums[2][w];
            all += gi.sums[2][w];
        }
#pragma unroll
        for (int x = 0; x < kGroupsPer; ++x) {
            const int g = tid * kGroupsPer + x;
            if (g < a.num_groups) gi.units[g] = run;
            run += units_of[x];
        }
        if (tid == 0) gi.units[a.num_groups] = all;
        n_p = all;
        if (!one_each(all, cost_p, cost_s)) {   // uniform
            uint32_t weighs = 0, longest = 0;   // as the units are: their last ranges may be shorter
#pragma unroll
            for (int x = 0; x < kGroupsPer; ++x) {
                weighs += static_cast<uint32_t>(units_of[x]) * each_of[x];
                longest = max(longest, static_cast<uint32_t>(each_of[x]));
            }
            const uint32_t weighs_to = static_cast<uint32_t>(wave_scan(static_cast<int>(weighs)));
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) longest = max(longest, static_cast<uint32_t>(__shfl_xor(static_cast<int>(longest), o)));
            if (lane == 63) gi.sums[0][wave] = static_cast<int>(weighs_to), gi.sums[1][wave] = static_cast<int>(longest);
            __syncthreads();
            uint32_t line = 0, at = weighs_to - weighs;
            longest = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                if (w < wave) at += static_cast<uint32_t>(gi.sums[0][w]);
                line += static_cast<uint32_t>(gi.sums[0][w]);
                longest = max(longest, static_cast<uint32_t>(gi.sums[1][w]));
            }
            n_p = workgroups_of(all, static_cast<float>(line), static_cast<float>(longest), cost_s);
            if (wg < n_p && n_p < all) {   // (a workgroup needs the weights or the sequences' first blocks)
#pragma unroll
                for (int x = 0; x < kGroupsPer; ++x) {
                    const int g = tid * kGroupsPer + x;
                    if (g <= a.num_groups) from[g] = static_cast<int>(at);
                    at += static_cast<uint32_t>(units_of[x]) * each_of[x];
                }
                if (tid == 0) from[a.num_groups] = static_cast<int>(line);
            }
        }
    }
    n_p = __builtin_amdgcn_readfirstlane(n_p);
    all = __builtin_amdgcn_readfirstlane(all);
    if (wg == kWorkgroups - 1) {   // for the merge
        __syncthreads();
#pragma unroll
        for (int x = 0; x < kSeqs; ++x) {
            const int s = tid + x * kThreads;
            if (s >= n) continue;
            SharedRow r = {};
            const int g = mine[x];
            if (g >= 0 && gi.eff[g] > 0) {
                const int c = (gi.offs[g + 1] - gi.offs[g]) * G, st = steps_of(gi.eff[g]), per = range_steps(st, gi.ranges[g]);
                r = SharedRow{gi.units[g], gi.ranges[g], (st + per - 1) / per, tiles_of(c), (s - gi.offs[g]) * G, tile_cols(c), {0, 0}};
            }
            a.rows[s] = r;
        }
    }
    if (wg < n_p) {
        __syncthreads();
        int first = wg, end = wg + 1;
        if (n_p < all) {
            const uint32_t line = static_cast<uint32_t>(from[a.num_groups]);
            first = first_unit(a, gi, from, first_of(line, n_p, wg));
            end = first_unit(a, gi, from, first_of(line, n_p, wg + 1));
        }
        shared_units<kFp8, kBlockScales ? 1 : 0>(a, gi, smem, ref, sums, first, end);
        return;
    }
    decode_flat_body<kFp8, kAppend, kWaves, false, kBlockScales ? 1 : 0, kMaxPairs, true>(
        a.q, a.q_stride, a.cache, a.block_table, a.max_blocks, a.seq_lens, a.o_part, a.ml_part, a.plan, n, a.hq_l, a.hkv_l, a.ref.c, a.r_min, ap, smem, index, wg - n_p,
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
        const int c = r.col0 + j % G, tile = c / r.cols;
        shared0 = (static_cast<size_t>(r.base) + static_cast<size_t>(tile + r.tiles * (j / G)) * r.ranges) * kTileCols + (c - tile * r.cols);
        shared_parts = r.parts;
    }
    const int np = there ? min(e.y + shared_parts, kMergeParts) : 0;
    auto row_of = [&](int c) -> size_t { return c < e.y ? own0 + static_cast<size_t>(c) * G : shared0 + static_cast<size_t>(c - e.y) * kTileCols; };
    auto o_of = [&](int c) -> f32x4 { return *reinterpret_cast<const f32x4*>((c < e.y ? o_part : o_shared) + row_of(c) * kD + 4 * (tid & 31)); };
    auto pair_of = [&](int c) -> f32x2 {
        return c < np ? *reinterpret_cast<const f32x2*>((c < e.y ? ml_part : ml_shared) + row_of(c) * 2) : f32x2{-INFINITY, 0.f};
    };
    // this thread's first parts are requested before the weights are known: the time is that of dependent loads
    constexpr int kEarly = kGroups == 4 ? 4 : 8;
    f32x4 early[kEarly];
#pragma unroll
    for (int x = 0; x < kEarly; ++x) early[x] = pg + kGroups * x < np ? o_of(pg + kGroups * x) : f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    auto add_part = [&](float w, f32x4 v) {
#pragma unroll
        for (int x = 0; x < 4; ++x) acc[x] = fmaf(v[x], w, acc[x]);
    };
    float l_star;
    if (np <= 64) {   // uniform: a pair per lane, every wavefront has all weights without LDS
        const f32x2 ml = pair_of(lane);
        float m_star = ml[0];
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) m_star = fmaxf(m_star, __shfl_xor(m_star, x));
        const float w_lane = ml[0] == -INFINITY ? 0.f : exp2f(ml[0] - m_star);
        l_star = ml[1] * w_lane;
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) l_star += __shfl_xor(l_star, x);
#pragma unroll
        for (int x = 0; x < kEarly; ++x)
            if (kGroups * x < 64) add_part(__shfl(w_lane, (pg + kGroups * x) & 63), early[x]);
        for (int c = kEarly * kGroups; c < np; c += kGroups) {
            const float w = __shfl(w_lane, min(c + pg, 63));
            if (c + pg < np) add_part(w, o_of(c + pg));
        }
    } else {
        float m_loc = -INFINITY;
        for (int c = tid; c < np; c += kThreads) {
            w_s[c] = pair_of(c)[0];
            m_loc = fmaxf(m_loc, w_s[c]);
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
            const float w = w_s[c] == -INFINITY ? 0.f : exp2f(w_s[c] - m_star);   // (each slot is read and rewritten by the same thread)
            w_s[c] = w;
            l_loc = fmaf(pair_of(c)[1], w, l_loc);
        }
#pragma unroll
        for (int x = 32; x > 0; x >>= 1) l_loc += __shfl_xor(l_loc, x);
        if (lane == 0) red_s[1][tid >> 6] = l_loc;
        __syncthreads();
        l_star = red_s[1][0];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) l_star += red_s[1][w];
#pragma unroll
        for (int x = 0; x < kEarly; ++x)
            if (pg + kGroups * x < np) add_part(w_s[pg + kGroups * x], early[x]);
#pragma unroll 4
        for (int c = pg + kEarly * kGroups; c < np; c += kGroups) add_part(w_s[c], o_of(c));
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
// units: a launch of `share` workgroups has up to that many ranges and one more for each item (tile, KV head); the work is summed in float32
int64_t most_items(int n, int num_groups, const AttnShape& a) {
    return static_cast<int64_t>(a.hkv_l) * (static_cast<int64_t>(n) * (a.hq_l / a.hkv_l) / kNarrowCols + (num_groups < n ? num_groups : n));
}
int64_t most_units(int n, int num_groups, const AttnShape& a) { return (kWorkgroups + most_items(n, num_groups, a)) * 9 / 8; }
// tokens per wavefront so that no row has more than 482 parts of its own, steps per range so that it has no more than 484 shared ones
int own_r_min(int max_seq_len) {
    const int r = (max_seq_len / 480 + kGroup) / kGroup * kGroup;
    return r < 2 * kGroup ? 2 * kGroup : r;
}
int range_min(int max_seq_len) {
    const int r = (max_seq_len / kStep + kMaxRanges) / kMaxRanges;
    return r < kMinSteps ? kMinSteps : r;
}
size_t rows_of(int n, const AttnShape& a) { return decode_mfma_rows_for(kWorkgroups * kWaves, n, a); }

// is a batch the kernel's that shares?
bool large_enough(int num_seqs, int max_seq_len, const AttnShape& a) {
    if (option_decode_shared() != 0) return option_decode_shared() == 1;
    // A batch that is small even if every sequence has max_seq_len tokens reads its shared keys again and again from the caches, and the plain
    // kernel, which has no groups to work out and fewer parts to merge, is done first: of 48 batches it was 1.0 to 3.5 us faster in all but one
    // below 40 MB (10.9 against 13.5 us at 10 MB), even at 45 to 60, slower above (27 against 22 at 98, 150 against 45 at 1061).
    const double bytes = 2.0 * kD * a.kv_elem * a.hkv_l * num_seqs * max_seq_len;
    return bytes > kPlainBytes;
}
size_t size_of(int n, int num_groups, const AttnShape& a) {
    return (rows_of(n, a) + static_cast<size_t>(most_units(n, num_groups, a)) * kTileCols) * (kD + 2) * sizeof(float) + static_cast<size_t>(n) * (a.hkv_l * sizeof(int2) + sizeof(SharedRow)) + 32;
}

}  // namespace

bool decode_shared_supported(const AttnShape& a, int num_seqs, int max_seq_len, int num_groups) {
    if (num_groups < 1 || num_groups > kMaxGroups || !decode_mfma_supported(a, num_seqs, max_seq_len) || a.hkv_l > kMaxPairs) return false;
    if (!large_enough(num_seqs, max_seq_len, a)) return false;
    const int per = seqs_per_launch(max_seq_len, a), n = num_seqs < per ? num_seqs : per;
    return per >= 1 && most_items(n, num_groups, a) * (max_seq_len / kStep + 1) < 0x7FFFFFFF / kWideCost;
}

size_t decode_shared_workspace(int num_seqs, int max_seq_len, int num_groups, const AttnShape& a) {
    const int per = seqs_per_launch(max_seq_len, a);
    return size_of(num_seqs < per ? num_seqs : per, num_groups, a);
}

size_t decode_shared_most_workspace(int num_seqs, int max_seq_len, int num_groups, const AttnShape& a) {
    if (num_groups < 1 || (num_groups > kMaxGroups && num_groups > num_seqs) || !decode_mfma_supported(a, num_seqs, 0) || a.hkv_l > kMaxPairs ||
        !large_enough(num_seqs, max_seq_len, a))
        return 0;
    const int per = seqs_per_launch(0, a);   // a launch of shorter sequences has more of them
    return size_of(num_seqs < per ? num_seqs : per, num_groups < kMaxGroups ? num_groups : kMaxGroups, a);
}

hipError_t launch_decode_shared(const void* q, const void* k_new, const void* v_new, const int64_t* slots, void* cache, const int32_t* block_table,
                                const int32_t* seq_lens, int num_seqs, int max_seq_len, const int32_t* group_offsets, const int32_t* shared_lens,
                                int num_groups, void* out, void* workspace, const AttnShape& a, hipStream_t st) {
    const bool append = k_new != nullptr;
    const int per = seqs_per_launch(max_seq_len, a), G = a.hq_l / a.hkv_l;
    const float c = a.scale * a.k_scale * 1.4426950408889634f;
    for (int s0 = 0; s0 < num_seqs; s0 += per) {  // runs share the workspace: same stream, one after the other
        const int n = num_seqs - s0 < per ? num_seqs - s0 : per;
        const size_t rows = rows_of(n, a), shared = static_cast<size_t>(most_units(n, num_groups, a)) * kTileCols;
        float* o_part = static_cast<float*>(workspace);
        float* o_shared = o_part + rows * kD;
        float* ml_part = o_shared + shared * kD;
        float* ml_shared = ml_part + rows * 2;
        int2* plan = reinterpret_cast<int2*>(ml_shared + shared * 2);
        SharedRow* info = reinterpret_cast<SharedRow*>((reinterpret_cast<uintptr_t>(plan + static_cast<size_t>(n) * a.hkv_l) + 31) & ~static_cast<uintptr_t>(31));
        const SharedArgs args = {static_cast<const uint16_t*>(q) + static_cast<size_t>(s0) * a.q_stride, static_cast<uint16_t*>(cache),
                                 block_table + static_cast<size_t>(s0) * a.max_blocks, seq_lens + s0, group_offsets, shared_lens, a.kv_scales, o_part, ml_part, plan,
                                 o_shared, ml_shared, info, a.q_stride, num_groups, s0, n, a.max_blocks, a.hq_l, a.hkv_l, own_r_min(max_seq_len),
                                 range_min(max_seq_len), option_decode_shared() == 1, {c, fminf(kLead / c, 3.4e38f / fmaxf(c, 1.f)), -3.4e38f / fmaxf(c, 1.f)}};
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
        auto merge = [&](auto kernel, int threads) {
            kernel<<<grid, threads, 0, st>>>(o_part, ml_part, plan, o_shared, ml_shared, info, seq_lens + s0, a.hq_l, G, out_run, a.out_stride, a.v_scale);
        };
        // many rows have few parts and fill the chip by themselves (4032 rows of four parts: 17.5 us with four groups, 20.1 with eight); few rows
        // have many, all of which should be on their way at once (1520 rows: 44.3 us with four, 42.6 with eight)
        if (grid >= 2048) merge(combine_shared_kernel<4>, 128);
        else if (grid >= 1024) merge(combine_shared_kernel<8>, 256);
        else merge(combine_shared_kernel<16>, 512);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace shiftattn
