// K/V append into the FP8 E4M3 cache with a scale per (block, KV head, part); see block_scale.h for the scales.
//
// A run is a stretch of consecutive new tokens whose slots are consecutive inside one block.  All new tokens of a block that a call
// brings are one run (the caller's contract), so whoever takes a run owns the block's codes and scales: it finds the largest finite
// magnitude of the run's K and of its V, takes the least scale that holds them - and, unless the run starts at the block's first
// slot, the scale that the block has - moves the codes in front of the run to the new scale where that grew, and writes the
// run's codes.
#include "block_scale.h"

namespace shiftattn {

namespace {

constexpr int kWavesPerWg = 4;

__device__ inline float value_of(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ inline float value_of(float f) { return f; }

__device__ inline uint32_t wave_max_bits(uint32_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o)));
    return v;
}

// A wavefront per (new token, KV head); those whose token starts a run take it, lanes over the head dimension.
template <typename Elem>
__global__ __launch_bounds__(64 * kWavesPerWg) void kv_write_scaled_kernel(const Elem* __restrict__ k_new, const Elem* __restrict__ v_new,
                                                                           const int64_t* __restrict__ slots, int n_tokens, uint8_t* cache,
                                                                           float* scales, int hkv_l, int D, int64_t kv_stride) {
    const int lane = threadIdx.x & 63;
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kWavesPerWg + (threadIdx.x >> 6);
    if (id >= static_cast<int64_t>(n_tokens) * hkv_l) return;
    const int64_t i = id / hkv_l;
    const int g = static_cast<int>(id - i * hkv_l);
    const int64_t slot = slots[i];
    if (slot < 0) return;
    const int off = static_cast<int>(slot % kBlockSize);
    if (off != 0 && i > 0 && slots[i - 1] == slot - 1) return;   // continues a run
    const int64_t at = i + lane;
    const bool goes_on = lane < kBlockSize - off && at < n_tokens && slots[at] == slot + lane;
    const int len = __builtin_ctzll(~__builtin_amdgcn_ballot_w64(goes_on));
    const int64_t blk = slot / kBlockSize;
    uint8_t* part[2] = {cache + cache_part_offset(blk, g, 0, hkv_l, D), cache + cache_part_offset(blk, g, 1, hkv_l, D)};
    float* s_blk = scales + (static_cast<size_t>(blk) * hkv_l + g) * 2;
#pragma unroll
    for (int x = 0; x < 2; ++x) {   // K, V
        const Elem* src = (x == 0 ? k_new : v_new) + static_cast<size_t>(i) * kv_stride + static_cast<size_t>(g) * D;
        uint32_t top = 0;
        for (int t = 0; t < len; ++t)
            for (int d = lane; d < D; d += 64) top = max(top, finite_magnitude(value_of(src[static_cast<size_t>(t) * kv_stride + d])));
        float s = block_scale(wave_max_bits(top));
        // element (token offset, d): K token-major, V dimension-major
        auto code_at = [&](int t, int d) -> uint8_t* { return part[x] + (x == 0 ? t * D + d : d * kBlockSize + t); };
        if (off > 0) {
            const float had = s_blk[x];
            s = fmaxf(s, had);
            if (s > had)   // uniform
                for (int t = 0; t < off; ++t)
                    for (int d = lane; d < D; d += 64) *code_at(t, d) = static_cast<uint8_t>(rescale_codes(*code_at(t, d), had / s));
        }
        for (int t = 0; t < len; ++t)
            for (int d = lane; d < D; d += 64)
                *code_at(off + t, d) = static_cast<uint8_t>(e4m3_pair(value_of(src[static_cast<size_t>(t) * kv_stride + d]), 0.f, s));
        if (lane == 0) s_blk[x] = s;
    }
}

}  // namespace

hipError_t launch_kv_write_scaled(const void* k_new, const void* v_new, const int64_t* slots, int n_tokens, void* cache,
                                  const AttnShape& a, hipStream_t st) {
    const int64_t waves = static_cast<int64_t>(n_tokens) * a.hkv_l;
    if (waves == 0) return hipSuccess;
    const int64_t wgs = (waves + kWavesPerWg - 1) / kWavesPerWg;
    if (wgs > 0x7FFFFFFF) return hipErrorInvalidValue;
    auto run = [&](auto elem) {
        using Elem = decltype(elem);
        kv_write_scaled_kernel<Elem><<<static_cast<unsigned>(wgs), 64 * kWavesPerWg, 0, st>>>(
            static_cast<const Elem*>(k_new), static_cast<const Elem*>(v_new), slots, n_tokens, static_cast<uint8_t*>(cache), a.kv_scales,
            a.hkv_l, a.D, a.kv_stride);
        return hipGetLastError();
    };
    return a.elem == 2 ? run(uint16_t{}) : run(float{});
}

}  // namespace shiftattn
