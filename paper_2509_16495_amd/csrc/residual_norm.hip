// Residual addition and root-mean-square norm of rows (shiftattn_add_rms_norm), written as values or as the 8-bit codes that the
// projections take.
//
//   h = x + residual, rounded to the residual's type and stored there;  inv = 1 / sqrt(sum h^2 / cols + eps);  y = (h * inv) * (w + offset)
//
// The squares are summed in 64 bits (a bf16 value's square is exact in 32, a float32 value's in 64) and inv is rounded once to float32, so
// that y, and with it every code and scale, is what the definition says in any order of the sum, unless 1 / sqrt lies within the sum's and the root's few
// 2^-53 of a border between two float32 values: about one row in 2^27, whose inv may be the neighbouring value.  A row's instance follows from
// `cols` alone, so the same row gives the same bits in every call.
#include "internal.h"

namespace shiftattn {

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int kMaxWaves = 16;

struct NormArgs {
    const void* x;
    void* res;            // nullptr: the rows have no residual
    const void* w;
    void* out;
    float* scales;
    int64_t x_stride, res_stride, out_stride;
    int cols;
    bool w_f32;
    int out_kind;         // SHIFTATTN_BF16, SHIFTATTN_F32, SHIFTATTN_CODES_FP8, SHIFTATTN_CODES_INT8
    float offset;
    double eps;
};

// eight elements of a row in float32
template <bool kF32>
__device__ inline void load8(const void* base, int64_t at, float (&f)[8]) {
    if constexpr (kF32) {
        const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const float*>(base) + at);
        const u32x4 a = p[0], b = p[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(a[j]), f[4 + j] = __uint_as_float(b[j]);
    } else {
        const u32x4 v = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[2 * j] = __uint_as_float(v[j] << 16), f[2 * j + 1] = __uint_as_float(v[j] & 0xFFFF0000u);
    }
}

__device__ inline uint32_t bf16_pair(float a, float b) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, bf16x2{static_cast<__bf16>(a), static_cast<__bf16>(b)});
}

template <bool kF32>
__device__ inline void store8(void* base, int64_t at, const float (&f)[8]) {
    if constexpr (kF32) {
        u32x4* p = reinterpret_cast<u32x4*>(static_cast<float*>(base) + at);
        p[0] = u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
        p[1] = u32x4{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])};
    } else {
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(base) + at) = u32x4{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7])};
    }
}

// 1 / sqrt(x) rounded from an error of a few 2^-53 (two Newton steps on the hardware's estimate); 0 for an infinity
__device__ inline float inverse_root(double x) {
    double r = __builtin_amdgcn_rsq(x);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = fma(r, fma(-0.5 * x * r, r, 0.5), r);
    return x < __builtin_inf() ? static_cast<float>(r) : x > 0.0 ? 0.f : static_cast<float>(x);
}

// One workgroup per row, kPieces stretches of eight elements per thread, held in registers from the load to the store.
// Bound: a row's bytes through HBM once (x and the residual in, the residual and the output out).  Threads for two stretches each: with one, a
// row of 8192 took a workgroup of 16 wavefronts that waits at two barriers with nothing beside it on its compute unit (16384 rows, int8: 208
// us), with four there are too few loads in flight (180; with two 170, 5.5 TB/s, what a copy reaches).
template <bool kXF32, bool kResF32, int kPieces>
__global__ __launch_bounds__(kMaxWaves * 64) void add_rms_norm_kernel(NormArgs a) {
    __shared__ double sums[kMaxWaves];
    __shared__ uint32_t tops[kMaxWaves];
    const int64_t row = blockIdx.x;
    const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    float h[kPieces][8];
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int col = (threadIdx.x + i * blockDim.x) * 8;
        if (col >= a.cols) {
#pragma unroll
            for (int j = 0; j < 8; ++j) h[i][j] = 0.f;
            continue;
        }
        load8<kXF32>(a.x, row * a.x_stride + col, h[i]);
        if (a.res) {
            float r[8];
            load8<kResF32>(a.res, row * a.res_stride + col, r);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[i][j] += r[j];
                if (!kResF32) h[i][j] = static_cast<float>(static_cast<__bf16>(h[i][j]));
            }
            store8<kResF32>(a.res, row * a.res_stride + col, h[i]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fma(static_cast<double>(h[i][j]), static_cast<double>(h[i][j]), sum);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) sums[wave] = sum;
    __syncthreads();
    sum = sums[0];
    for (int w = 1; w < waves; ++w) sum += sums[w];
    const double mean = sum / a.cols + a.eps;
    const float inv = inverse_root(mean);

    const bool codes = a.out_kind >= SHIFTATTN_CODES_FP8;
    const uint32_t below = a.out_kind == SHIFTATTN_CODES_FP8 ? 0x7F800001u : 0x7F800000u;
    uint32_t all = 0;     // largest |y|, as bits (NaN is above everything)
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int col = (threadIdx.x + i * blockDim.x) * 8;
        if (col >= a.cols) continue;
        float w[8];
        if (a.w_f32) load8<true>(a.w, col, w);
        else load8<false>(a.w, col, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            h[i][j] = (h[i][j] * inv) * (w[j] + a.offset);
            const uint32_t b = __float_as_uint(h[i][j]) & 0x7FFFFFFFu;
            all = max(all, b);
        }
        if (a.out_kind == SHIFTATTN_BF16) store8<false>(a.out, row * a.out_stride + col, h[i]);
        else if (a.out_kind == SHIFTATTN_F32) store8<true>(a.out, row * a.out_stride + col, h[i]);
    }
    if (!codes) return;
    auto over_row = [&](uint32_t v) -> uint32_t {
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o)));
        if (lane == 0) tops[wave] = v;
        __syncthreads();
        v = tops[0];
        for (int w = 1; w < waves; ++w) v = max(v, tops[w]);
        return v;
    };
    uint32_t top = over_row(all);   // largest |y| as bits
    const bool numbers = top < 0x7F800000u;
    if (!numbers) {   // (uniform, rare) of those that are numbers (FP8: infinities too)
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t b = __float_as_uint(h[i][j]) & 0x7FFFFFFFu;
                if ((threadIdx.x + i * blockDim.x) * 8 < a.cols) m = max(m, b < below ? b : 0u);
            }
        __syncthreads();
        top = over_row(m);
    }
    const float amax = __uint_as_float(top);
    uint8_t* out = static_cast<uint8_t*>(a.out) + row * a.out_stride;
    if (a.out_kind == SHIFTATTN_CODES_FP8) {
        const float scale = amax > 0.f ? amax / 448.f : 1.f;
        if (threadIdx.x == 0) a.scales[row] = scale;
        // The quotient correctly rounded, as a division gives it, in five instructions instead of ten: with y the rounded reciprocal, two steps
        // q += (v - q scale) y, whose remainders are exact (Markstein's theorem; it needs a reciprocal whose divisor's
        // mantissa is not all ones, and a range without underflow: below 2^-11 a quotient's code is 0 whatever its last bits).
        if (numbers && scale > 0x1p-60f && scale < 0x1p60f && (__float_as_uint(scale) & 0x7FFFFFu) != 0x7FFFFFu) {
            const float y = 1.f / scale;
            auto quotient = [&](float v) {
                float q = v * y;
                q = fmaf(fmaf(-q, scale, v), y, q);
                return copysignf(fmaf(fmaf(-q, scale, v), y, q), v);   // (-0 keeps its sign) at most 448 (1 + 2^-23): rounds to a code without a clamp
            };
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
                const int col = (threadIdx.x + i * blockDim.x) * 8;
                if (col >= a.cols) continue;
                u32x2 r;
#pragma unroll
                for (int h2 = 0; h2 < 2; ++h2) {
                    int w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(h[i][4 * h2]), quotient(h[i][4 * h2 + 1]), 0, false);
                    w = __builtin_amdgcn_cvt_pk_fp8_f32(quotient(h[i][4 * h2 + 2]), quotient(h[i][4 * h2 + 3]), w, true);
                    r[h2] = static_cast<uint32_t>(w);
                }
                *reinterpret_cast<u32x2*>(out + col) = r;
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int col = (threadIdx.x + i * blockDim.x) * 8;
            if (col >= a.cols) continue;
            *reinterpret_cast<u32x2*>(out + col) = u32x2{e4m3_pair(h[i][0], h[i][1], scale) | (e4m3_pair(h[i][2], h[i][3], scale) << 16),
                                                         e4m3_pair(h[i][4], h[i][5], scale) | (e4m3_pair(h[i][6], h[i][7], scale) << 16)};
        }
        return;
    }
    const bool tiny = amax < 0x1p-100f;
    const float to_code = tiny ? 1.f : 127.f * (1.f / amax);
    if (threadIdx.x == 0) a.scales[row] = tiny ? 1.f : amax * (1.f / 127.f);
    auto code = [&](float v) -> uint32_t {
        // adding 1.5 * 2^23 rounds the exact product to an integer, ties to even; its low byte is the code
        const uint32_t c = __float_as_uint(fmaf(v, to_code, 12582912.f)) & 0xFFu;
        return numbers || fabsf(v) < INFINITY ? c : v != v ? 0u : v > 0.f ? 127u : 129u;
    };
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int col = (threadIdx.x + i * blockDim.x) * 8;
        if (col >= a.cols) continue;
        u32x2 r;
#pragma unroll
        for (int q = 0; q < 2; ++q)
            r[q] = code(h[i][4 * q]) | (code(h[i][4 * q + 1]) << 8) | (code(h[i][4 * q + 2]) << 16) | (code(h[i][4 * q + 3]) << 24);
        *reinterpret_cast<u32x2*>(out + col) = r;
    }
}

}  // namespace

hipError_t launch_add_rms_norm(const void* x, void* residual, const void* weight, void* out, float* scales, int rows, const NormShape& s,
                               hipStream_t st) {
    if (rows == 0) return hipSuccess;
    const int pieces = s.cols / 8;
    int threads = (pieces + 127) / 128 * 64;
    threads = threads < kMaxWaves * 64 ? threads : kMaxWaves * 64;
    const int per = (pieces + threads - 1) / threads;
    NormArgs a{x, residual, weight, out, scales, s.x_stride, s.res_stride, s.out_stride, s.cols, s.w_f32, s.out_kind, s.offset,
               static_cast<double>(s.eps)};
    auto run = [&](auto kernel) -> hipError_t {
        const int64_t piece = most_workgroups(threads);
        const int x_elem = s.x_f32 ? 4 : 2, res_elem = s.res_f32 ? 4 : 2, out_elem = s.out_kind == SHIFTATTN_F32 ? 4 : s.out_kind == SHIFTATTN_BF16 ? 2 : 1;
        for (int64_t row = 0; row < rows; row += piece) {
            NormArgs b = a;
            b.x = static_cast<const char*>(x) + row * s.x_stride * x_elem;
            if (residual) b.res = static_cast<char*>(residual) + row * s.res_stride * res_elem;
            b.out = static_cast<char*>(out) + row * s.out_stride * out_elem;
            if (scales) b.scales = scales + row;
            kernel<<<static_cast<unsigned>(rows - row < piece ? rows - row : piece), threads, 0, st>>>(b);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    auto typed = [&](auto pieces_c) -> hipError_t {
        constexpr int kP = decltype(pieces_c)::value;
        if (s.x_f32) return s.res_f32 ? run(add_rms_norm_kernel<true, true, kP>) : run(add_rms_norm_kernel<true, false, kP>);
        return s.res_f32 ? run(add_rms_norm_kernel<false, true, kP>) : run(add_rms_norm_kernel<false, false, kP>);
    };
    if (per <= 1) return typed(std::integral_constant<int, 1>{});
    if (per <= 2) return typed(std::integral_constant<int, 2>{});
    if (per <= 4) return typed(std::integral_constant<int, 4>{});
    return typed(std::integral_constant<int, 8>{});
}

}  // namespace shiftattn
