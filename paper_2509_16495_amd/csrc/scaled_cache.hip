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
                                                                           float* scales, int hkv_l, int D, int64_t kv_stride, int64_t first) {
    const int lane = threadIdx.x & 63;
    const int64_t id = first + static_cast<int64_t>(blockIdx.x) * kWavesPerWg + (threadIdx.x >> 6);
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

// bf16, D = 128 or 64: a wavefront takes the runs that start in its window of tokens.  Lane (q, dv) = (lane / 16, lane % 16) holds elements 8 dv ..
// 8 dv + 7 (where D has them) of the tokens at block offsets 4 q .. 4 q + 3, so that the four codes of a head-dim row that lie next to each other in V's
// block come from one lane: a 4 x 4 byte transposition in registers, a word per head-dim row through LDS, and V goes out as whole rows of
// 16 codes.  Where the run does not fill the block those rows are read first and merged.
// Bound: bytes for large launches, for small ones the chain of round trips slot - rows - stores.  Windows: of one token up to 4096 (token,
// head) and for decode rows, whose runs are one token each and a wavefront takes one behind the other (1024 rows, windows of 1 / 4 / 8 /
// 16 tokens: 4.9 / 10.6 / 18.5 / 34.3 us); of eight beyond, where a wavefront for every token would be launched in vain (16384 tokens of
// prompts 12.4 / 5.4 / 4.9 / 4.9, 65536 42.1 / 14.0 / 12.2 / 11.9, 600000 363 / 106 / 90 / 90: 5.1 TB/s read and written).
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
constexpr int kTileBytes = 128 * 16 + 16 * 16;   // per wavefront: 128 rows of 16 codes, 16 bytes more behind every eight (banks)

template <int D>
__global__ __launch_bounds__(64 * kWavesPerWg) void kv_write_scaled_rows_kernel(const uint16_t* __restrict__ k_new, const uint16_t* __restrict__ v_new,
                                                                                const int64_t* __restrict__ slots, int n_tokens, int window_of_chunks,
                                                                                int chunk_rows, uint8_t* cache, float* scales, int hkv_l, int64_t kv_stride) {
    __shared__ __attribute__((aligned(16))) unsigned char tile_all[kWavesPerWg * kTileBytes];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    unsigned char* tile = tile_all + wave * kTileBytes;
    const int g = blockIdx.y;
    // rows of chunks in windows, the rows behind them one by one
    const int64_t id = static_cast<int64_t>(blockIdx.x) * kWavesPerWg + wave, chunk_windows = (static_cast<int64_t>(chunk_rows) + window_of_chunks - 1) / window_of_chunks;
    const bool in_chunks = id < chunk_windows;
    const int64_t w0 = in_chunks ? id * window_of_chunks : chunk_rows + id - chunk_windows;
    if (w0 >= n_tokens) return;
    const int window = !in_chunks ? 1 : static_cast<int>(min(static_cast<int64_t>(window_of_chunks), chunk_rows - w0));
    // slots of the window and of the 16 tokens behind it, a token per lane: bit t of `starts` says that token t starts a run, bit t of
    // `breaks` that it does not continue the run of the one before
    const int64_t i_lane = w0 + (lane & 31);
    const int64_t s_lane = i_lane < n_tokens ? slots[i_lane] : -1;
    const int64_t s_prev = i_lane > 0 && i_lane < n_tokens ? slots[i_lane - 1] : -2;
    const bool st = s_lane >= 0 && (s_lane % kBlockSize == 0 || s_prev != s_lane - 1);
    uint32_t starts = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(st)) & ((1u << window) - 1u);
    const uint32_t breaks = static_cast<uint32_t>(__builtin_amdgcn_ballot_w64(st || s_lane < 0));
    const int q = lane >> 4, dv = lane & 15;
    while (starts) {   // uniform
        const int t0 = __builtin_ctz(starts);
        starts &= starts - 1;
        const int len = __builtin_ctz((breaks >> 1) >> t0) + 1;   // at most 16: a multiple of 16 starts the next run
        const int s_lo = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint64_t>(s_lane)), t0);
        const int s_hi = __builtin_amdgcn_readlane(static_cast<int>(static_cast<uint64_t>(s_lane) >> 32), t0);
        const uint64_t slot = (static_cast<uint64_t>(static_cast<uint32_t>(s_hi)) << 32) | static_cast<uint32_t>(s_lo);
        const int off = static_cast<int>(slot % kBlockSize);
        const int64_t blk = static_cast<int64_t>(slot / kBlockSize);
        uint8_t* k_at = cache + cache_part_offset(blk, g, 0, hkv_l, D);
        uint8_t* v_at = cache + cache_part_offset(blk, g, 1, hkv_l, D);
        float* s_blk = scales + (static_cast<size_t>(blk) * hkv_l + g) * 2;
        const bool whole = len == kBlockSize;
        u32x4 kx[4], vx[4], v_old[2];
        float had_k = 0.f, had_v = 0.f;
        const size_t src = static_cast<size_t>(w0 + t0) * kv_stride + static_cast<size_t>(g) * D + dv * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * q + i - off;
            kx[i] = vx[i] = u32x4{0u, 0u, 0u, 0u};
            if (t >= 0 && t < len && 8 * dv < D) {
                const size_t at = src + static_cast<size_t>(t) * kv_stride;
                kx[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(k_new + at));
                vx[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(v_new + at));
            }
        }
        if (!whole) {
#pragma unroll
            for (int j = 0; j < D / 64; ++j) v_old[j] = *reinterpret_cast<const u32x4*>(v_at + 1024 * j + 16 * lane);
        }
        if (off > 0) had_k = s_blk[0], had_v = s_blk[1];
        // largest magnitudes as bits, K's in the upper half of a word, V's in the lower
        u16x2 top_k = {0, 0}, top_v = {0, 0};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                top_k = __builtin_elementwise_max(top_k, __builtin_bit_cast(u16x2, kx[i][j] & 0x7FFF7FFFu));
                top_v = __builtin_elementwise_max(top_v, __builtin_bit_cast(u16x2, vx[i][j] & 0x7FFF7FFFu));
            }
        auto wave_top = [&](u16x2 both) {
#pragma unroll
            for (int o = 32; o > 0; o >>= 1)
                both = __builtin_elementwise_max(both, __builtin_bit_cast(u16x2, __shfl_xor(__builtin_bit_cast(int, both), o)));
            return both;
        };
        u16x2 top = wave_top(u16x2{max(top_v[0], top_v[1]), max(top_k[0], top_k[1])});
        const bool finite = top[0] < 0x7F80 && top[1] < 0x7F80;   // uniform
        if (!finite) {   // rare: maxima of the finite elements
            auto finite_top = [](const u32x4 (&x)[4]) {
                uint16_t m = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const uint16_t b = static_cast<uint16_t>((x[i][j >> 1] >> (16 * (j & 1))) & 0x7FFFu);
                        if (b < 0x7F80) m = max(m, b);
                    }
                return m;
            };
            top = wave_top(u16x2{finite_top(vx), finite_top(kx)});
        }
        float now_k = block_scale(static_cast<uint32_t>(top[1]) << 16), now_v = block_scale(static_cast<uint32_t>(top[0]) << 16);
        if (off > 0) now_k = fmaxf(now_k, had_k), now_v = fmaxf(now_v, had_v);
        // a finite element is at most 448 scales but at the largest scale, where codes saturate
        const bool clamp = !finite || now_k >= 0x1p119f || now_v >= 0x1p119f;
        auto encode = [&](u32x4 x, float scale) -> u32x2 {
            float f[8];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f[2 * j] = __uint_as_float(x[j] << 16);
                f[2 * j + 1] = __uint_as_float(x[j] & 0xFFFF0000u);
            }
            if (clamp)
                return u32x2{e4m3_pair(f[0], f[1], scale) | (e4m3_pair(f[2], f[3], scale) << 16),
                             e4m3_pair(f[4], f[5], scale) | (e4m3_pair(f[6], f[7], scale) << 16)};
            const float inv = __uint_as_float((254u << 23) - __float_as_uint(scale));   // exact: a power of two
            u32x2 r;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h] * inv, f[4 * h + 1] * inv, 0, false);
                r[h] = static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2] * inv, f[4 * h + 3] * inv, w, true));
            }
            return r;
        };
        u32x2 vc[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = 4 * q + i - off;
            if (t >= 0 && t < len && 8 * dv < D)
                __builtin_nontemporal_store(encode(kx[i], now_k), reinterpret_cast<u32x2*>(k_at + (4 * q + i) * D + dv * 8));
            vc[i] = encode(vx[i], now_v);
        }
        // word (d, q): codes of head-dim row d at offsets 4 q .. 4 q + 3
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t a = __builtin_amdgcn_perm(vc[1][h], vc[0][h], 0x05010400u), b = __builtin_amdgcn_perm(vc[1][h], vc[0][h], 0x07030602u);
            const uint32_t c = __builtin_amdgcn_perm(vc[3][h], vc[2][h], 0x05010400u), d = __builtin_amdgcn_perm(vc[3][h], vc[2][h], 0x07030602u);
            uint32_t* w = reinterpret_cast<uint32_t*>(tile + dv * 144 + h * 64 + q * 4);
            w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
            w[4] = __builtin_amdgcn_perm(c, a, 0x07060302u);
            w[8] = __builtin_amdgcn_perm(d, b, 0x05040100u);
            w[12] = __builtin_amdgcn_perm(d, b, 0x07060302u);
        }
        __builtin_amdgcn_wave_barrier();
        const bool grown_k = off > 0 && now_k > had_k, grown_v = off > 0 && now_v > had_v;   // uniform
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const int d = lane + 64 * j;
            u32x4 row = *reinterpret_cast<const u32x4*>(tile + d * 16 + (d >> 3) * 16);
            if (!whole) {
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    auto below = [&](int n) { return n >= 4 * w + 4 ? 0xFFFFFFFFu : n <= 4 * w ? 0u : (1u << (8 * (n - 4 * w))) - 1u; };
                    uint32_t old = v_old[j][w];
                    if (grown_v) old = (rescale_codes(old, had_v / now_v) & below(off)) | (old & ~below(off));
                    const uint32_t mine = below(off + len) & ~below(off);
                    row[w] = (row[w] & mine) | (old & ~mine);
                }
            }
            __builtin_nontemporal_store(row, reinterpret_cast<u32x4*>(v_at + 1024 * j + 16 * lane));
        }
        if (grown_k) {   // K rows in front of the run: 1 KiB of rows a load
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                if ((1024 * j + 16 * lane) / D < off) {
                    u32x4* at = reinterpret_cast<u32x4*>(k_at + 1024 * j + 16 * lane);
                    u32x4 x = *at;
#pragma unroll
                    for (int w = 0; w < 4; ++w) x[w] = rescale_codes(x[w], had_k / now_k);
                    *at = x;
                }
            }
        }
        if (lane == 0) s_blk[0] = now_k, s_blk[1] = now_v;
        __builtin_amdgcn_wave_barrier();   // the next run reuses the tile
    }
}

}  // namespace

hipError_t launch_kv_write_scaled(const void* k_new, const void* v_new, const int64_t* slots, int n_tokens, int chunk_rows, void* cache,
                                  const AttnShape& a, hipStream_t st) {
    const int64_t waves = static_cast<int64_t>(n_tokens) * a.hkv_l;
    if (waves == 0) return hipSuccess;
    const int window = static_cast<int64_t>(chunk_rows) * a.hkv_l <= 4096 ? 1 : 8;
    const int64_t windows = (static_cast<int64_t>(chunk_rows) + window - 1) / window + n_tokens - chunk_rows;
    const int64_t wgs = (windows + kWavesPerWg - 1) / kWavesPerWg;
    if (a.elem == 2 && (a.D == 128 || a.D == 64) && a.hkv_l <= 65535 && wgs <= most_workgroups(64 * kWavesPerWg)) {
        const dim3 grid(static_cast<unsigned>(wgs), static_cast<unsigned>(a.hkv_l));
        auto rows = [&](auto kernel) {
            kernel<<<grid, 64 * kWavesPerWg, 0, st>>>(static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new), slots, n_tokens, window,
                                                      chunk_rows, static_cast<uint8_t*>(cache), a.kv_scales, a.hkv_l, a.kv_stride);
            return hipGetLastError();
        };
        return a.D == 128 ? rows(kv_write_scaled_rows_kernel<128>) : rows(kv_write_scaled_rows_kernel<64>);
    }
    auto run = [&](auto elem) {
        using Elem = decltype(elem);
        const int64_t piece = most_workgroups(64 * kWavesPerWg) * kWavesPerWg;   // (token, head) a launch
        for (int64_t first = 0; first < waves; first += piece) {
            const int64_t n = waves - first < piece ? waves - first : piece;
            kv_write_scaled_kernel<Elem><<<static_cast<unsigned>((n + kWavesPerWg - 1) / kWavesPerWg), 64 * kWavesPerWg, 0, st>>>(
                static_cast<const Elem*>(k_new), static_cast<const Elem*>(v_new), slots, n_tokens, static_cast<uint8_t*>(cache), a.kv_scales,
                a.hkv_l, a.D, a.kv_stride, first);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    return a.elem == 2 ? run(uint16_t{}) : run(float{});
}

}  // namespace shiftattn
