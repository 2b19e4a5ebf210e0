// Attention over an FP8 cache with block scales, for the shapes that the MFMA kernels do not take: fp32 tensors, head dimensions
// other than 128, batches whose widened copy would be too large.  Prefill and decode rows alike.
//
// One workgroup takes a row (token) and up to HG query heads of one KV head, so that K and V are fetched and widened once for all of
// them; its wavefronts take the context in chunks of 64 tokens in turn, each with a running maximum and sum of its own, and
// meet in LDS at the end, in wavefront order.  Within a chunk lanes are tokens for q.k (a lane walks its token's row of codes, q comes from
// LDS for all lanes at once) and head-dim rows for p.V (a lane's 16 bytes are 16 tokens of its row, the probabilities come from LDS).
// The scales are applied by the widening instruction, which costs nothing and keeps the products in range: a query times a code may
// overflow where the query times the element does not.  All sums are float32.
// Bound: the LDS reads that hand q and the probabilities round (16 bytes for four multiply-adds of a wavefront; a compute unit's wavefronts share
// one LDS), and for few rows the walk over a context.  So a workgroup takes one head, and four only where rows fill the chip many times
// over and fetching and widening K and V four times weighs more: 2000 rows x 8 heads of 256 734 -> 474 us, but 16 decode rows x 4 heads
// of 64 (fp32, up to 1500 tokens, with the append) 14.2 -> 29.0, 550 rows x 4 of 64 34.0 -> 37.4.  Wavefronts by how many
// workgroups there are, 16 / 8 / 4: 64 workgroups 14.2 / 14.7 / 20.0 us, 400 19.9 / 14.7 / 16.7, 1200 53 / 40 / 35.  One wavefront per (row,
// head) that walked the whole context alone took 97 us for the 16 rows.
#include "block_scale.h"
#include "query_rows.h"

#include <type_traits>

namespace shiftattn {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxD = 256, kMaxWaves = 16, kChunk = 64;

__device__ inline float to_float(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ inline float to_float(float f) { return f; }
__device__ inline void store_elem(uint16_t* p, float f) {
    uint32_t u = __float_as_uint(f);
    u = f != f ? 0x7FC00000u : u + 0x7FFFu + ((u >> 16) & 1u);
    *p = static_cast<uint16_t>(u >> 16);
}
__device__ inline void store_elem(float* p, float f) { *p = f; }

__device__ inline float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// values of four codes times their block's scale
__device__ inline f32x4 widen4(uint32_t codes, float scale) {
    const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(static_cast<int>(codes), scale, false);
    const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(static_cast<int>(codes), scale, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// HG: heads at most; DV: head-dim rows per lane (64 DV >= D)
template <typename Elem, int HG, int DV>
__global__ __launch_bounds__(64 * kMaxWaves) void attn_scaled_rows_kernel(const Elem* __restrict__ q, const uint8_t* __restrict__ cache,
                                                                         const float* __restrict__ scales, const int32_t* __restrict__ block_table,
                                                                         const int32_t* __restrict__ cu_seqlens_q, const int32_t* __restrict__ seq_lens,
                                                                         int num_seqs, int head_groups, int first_row, Elem* __restrict__ out, AttnShape a) {
    __shared__ __attribute__((aligned(16))) float q_s[HG * kMaxD];
    constexpr int kPerWave = HG > DV ? HG * kChunk : DV * 64;                       // a chunk's probabilities, then one head's sums
    __shared__ __attribute__((aligned(16))) float p_s[kMaxWaves * kPerWave];
    __shared__ float m_s[kMaxWaves][HG], l_s[kMaxWaves][HG];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int per_row = a.hkv_l * head_groups;
    const int row = blockIdx.x / per_row, rest = blockIdx.x - row * per_row, g = rest / head_groups, hg = rest - g * head_groups;
    const int tok = first_row + row;
    const int G = a.hq_l / a.hkv_l, D = a.D, h0 = g * G + hg * HG, heads = min(HG, G - hg * HG);

    const auto [s, pos] = query_row(cu_seqlens_q, seq_lens, num_seqs, tok);
    if (s < 0) return;   // uniform
    const int32_t* table = block_table + static_cast<size_t>(s) * a.max_blocks;
    const Elem* q_row = q + static_cast<size_t>(tok) * a.q_stride + static_cast<size_t>(h0) * D;
    for (int i = threadIdx.x; i < HG * D; i += blockDim.x) q_s[i] = i < heads * D ? to_float(q_row[i]) : 0.f;
    __syncthreads();

    float m_run[HG], l_lane[HG], o[HG][DV];
#pragma unroll
    for (int h = 0; h < HG; ++h) {
        m_run[h] = -INFINITY, l_lane[h] = 0.f;
#pragma unroll
        for (int x = 0; x < DV; ++x) o[h][x] = 0.f;
    }
    float* p_w = p_s + wave * kPerWave;
    for (int64_t t0 = static_cast<int64_t>(wave) * kChunk; t0 <= pos; t0 += static_cast<int64_t>(waves) * kChunk) {
        const int t = static_cast<int>(t0) + lane;
        const bool sees = t <= pos;
        float logit[HG];
#pragma unroll
        for (int h = 0; h < HG; ++h) logit[h] = -INFINITY;
        if (sees) {
            const size_t at = static_cast<size_t>(table[t / kBlockSize]) * a.hkv_l + g;
            const uint8_t* k_row = cache + at * 2 * kBlockSize * D + static_cast<size_t>(t % kBlockSize) * D;
            const float k_scale = scales[at * 2];
            f32x4 acc[HG];   // four sums a head: shorter chains, smaller rounding errors
#pragma unroll
            for (int h = 0; h < HG; ++h) acc[h] = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int d = 0; d < D; d += 16) {
                const u32x4 codes = *reinterpret_cast<const u32x4*>(k_row + d);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const f32x4 k4 = widen4(codes[w], k_scale);
#pragma unroll
                    for (int h = 0; h < HG; ++h) {
                        const f32x4 q4 = *reinterpret_cast<const f32x4*>(q_s + h * D + d + 4 * w);
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[h][e] = fmaf(q4[e], k4[e], acc[h][e]);
                    }
                }
            }
#pragma unroll
            for (int h = 0; h < HG; ++h) logit[h] = ((acc[h][0] + acc[h][1]) + (acc[h][2] + acc[h][3])) * a.scale;
        }
#pragma unroll
        for (int h = 0; h < HG; ++h) {
            const float m_new = fmaxf(m_run[h], wave_max(logit[h]));
            const float m_ref = m_new == -INFINITY ? 0.f : m_new;   // (no logit above minus infinity yet)
            const float p = sees ? expf(logit[h] - m_ref) : 0.f;
            const float alpha = expf(m_run[h] - m_ref);   // exp(-inf) = 0 on the first chunk
            l_lane[h] = fmaf(l_lane[h], alpha, p);
            m_run[h] = m_new;
            p_w[h * kChunk + lane] = p;
#pragma unroll
            for (int x = 0; x < DV; ++x) o[h][x] *= alpha;
        }
        __builtin_amdgcn_wave_barrier();
        for (int b = 0; b < kChunk / kBlockSize; ++b) {
            const int left = pos - (static_cast<int>(t0) + b * kBlockSize) + 1;   // tokens of the block that are seen
            if (left <= 0) break;
            const size_t at = static_cast<size_t>(table[static_cast<int>(t0) / kBlockSize + b]) * a.hkv_l + g;
            const uint8_t* v_part = cache + (at * 2 + 1) * kBlockSize * D;
            const float v_scale = scales[at * 2 + 1];
#pragma unroll
            for (int x = 0; x < DV; ++x) {
                const int d = lane + 64 * x;
                if (d >= D) continue;
                u32x4 codes = *reinterpret_cast<const u32x4*>(v_part + static_cast<size_t>(d) * kBlockSize);
                if (left < kBlockSize) {   // slots behind the context may hold anything (also NaN)
#pragma unroll
                    for (int w = 0; w < 4; ++w)
                        codes[w] &= left >= 4 * w + 4 ? 0xFFFFFFFFu : left <= 4 * w ? 0u : (1u << (8 * (left - 4 * w))) - 1u;
                }
                f32x4 v4[4];
#pragma unroll
                for (int w = 0; w < 4; ++w) v4[w] = widen4(codes[w], v_scale);
#pragma unroll
                for (int h = 0; h < HG; ++h) {
                    f32x4 part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const f32x4 p4 = *reinterpret_cast<const f32x4*>(p_w + h * kChunk + b * kBlockSize + 4 * w);
#pragma unroll
                        for (int e = 0; e < 4; ++e) part[e] = fmaf(p4[e], v4[w][e], part[e]);
                    }
                    o[h][x] += (part[0] + part[1]) + (part[2] + part[3]);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
    // the wavefronts' parts meet, head by head
#pragma unroll
    for (int h = 0; h < HG; ++h) {
        const float l = wave_sum(l_lane[h]);
        if (lane == 0) m_s[wave][h] = m_run[h], l_s[wave][h] = l;
    }
    __syncthreads();
    Elem* o_row = out + static_cast<size_t>(tok) * a.out_stride + static_cast<size_t>(h0) * D;
#pragma unroll
    for (int h = 0; h < HG; ++h) {
        if (h >= heads) break;   // uniform
        float m_star = -INFINITY;
        for (int w = 0; w < waves; ++w) m_star = fmaxf(m_star, m_s[w][h]);
        const float mine = m_run[h] == -INFINITY ? 0.f : expf(m_run[h] - m_star);
        float l_star = 0.f;
        for (int w = 0; w < waves; ++w) l_star = fmaf(l_s[w][h], m_s[w][h] == -INFINITY ? 0.f : expf(m_s[w][h] - m_star), l_star);
#pragma unroll
        for (int x = 0; x < DV; ++x) p_w[lane + 64 * x] = o[h][x] * mine;
        __syncthreads();
        const float inv = l_star > 0.f ? 1.f / l_star : 0.f;   // a row without visible keys (padding) is zero
        for (int d = threadIdx.x; d < D; d += blockDim.x) {
            float sum = p_s[d];
            for (int w = 1; w < waves; ++w) sum += p_s[w * kPerWave + d];
            store_elem(o_row + static_cast<size_t>(h) * D + d, sum * inv);
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_attn_scaled(const void* q, const void* cache, const int32_t* block_table, const int32_t* cu_seqlens_q, const int32_t* seq_lens,
                              int num_seqs, int rows, int max_seq_len, void* out, const AttnShape& a, hipStream_t st) {
    if (rows == 0) return hipSuccess;
    const int G = a.hq_l / a.hkv_l;
    auto run = [&](auto elem, auto hg, auto dv) {
        using Elem = decltype(elem);
        constexpr int HG = decltype(hg)::value;
        const int groups = (G + HG - 1) / HG;
        const int64_t wgs = static_cast<int64_t>(rows) * a.hkv_l * groups;
        const int chunks = max_seq_len / kChunk + (max_seq_len % kChunk != 0);
        int waves = wgs <= 256 ? 16 : wgs <= 1024 ? 8 : 4;
        while (waves > 1 && waves >= 2 * chunks) waves /= 2;   // (none without a chunk)
        const int per_row = a.hkv_l * groups;
        const int64_t piece = most_workgroups(64 * waves) / per_row;   // rows a launch
        if (piece == 0) return hipErrorInvalidValue;
        for (int64_t row = 0; row < rows; row += piece) {
            const int n = static_cast<int>(rows - row < piece ? rows - row : piece);
            attn_scaled_rows_kernel<Elem, HG, decltype(dv)::value><<<static_cast<unsigned>(n) * per_row, 64 * waves, 0, st>>>(
                static_cast<const Elem*>(q), static_cast<const uint8_t*>(cache), a.kv_scales, block_table, cu_seqlens_q, seq_lens, num_seqs, groups,
                static_cast<int>(row), static_cast<Elem*>(out), a);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    auto by_heads = [&](auto elem, auto dv) {
        if (G > 1 && static_cast<int64_t>(rows) * a.hq_l >= 8192) return run(elem, std::integral_constant<int, 4>{}, dv);
        return run(elem, std::integral_constant<int, 1>{}, dv);
    };
    auto by_dim = [&](auto elem) {
        if (a.D <= 64) return by_heads(elem, std::integral_constant<int, 1>{});
        if (a.D <= 128) return by_heads(elem, std::integral_constant<int, 2>{});
        return by_heads(elem, std::integral_constant<int, 4>{});
    };
    return a.elem == 2 ? by_dim(uint16_t{}) : by_dim(float{});
}

}  // namespace shiftattn
