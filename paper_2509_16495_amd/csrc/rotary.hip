// Rotary positions (shiftattn_rotary, shiftattn_rotary_mixed): pairs of elements of the query and key heads of a row turned in place by
// angles that grow with the row's position, (a, b) -> m (a cos t - b sin t, b cos t + a sin t), t = position * frequency.
//
// The angle is reduced to a fraction of a turn in 64 bits: at position 10^6 a float32 product would have no fraction left that is worth
// anything (2^20 radians have a last place of 2^-3).  A quarter of a turn around the nearest axis remains, where the Taylor series of
// sine to the ninth and of cosine to the tenth power are exact to 2 * 10^-9, a thirtieth of float32's last place.
#include "internal.h"
#include "query_rows.h"

namespace shiftattn {

namespace {

constexpr int kThreads = 256;

struct RotaryArgs {
    void* heads[2];                 // queries, keys
    int num_heads[2];
    int64_t stride[2];
    const int32_t* positions;       // nullptr: from the two below
    const int32_t* cu_seqlens_q;
    const int32_t* seq_lens;
    const double* frequencies;
    int64_t first, rows;            // those of this launch
    int num_prefill, total_prefill_q, head_dim, half, slices;
    float magnitude;
};

__device__ inline float to_float(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ inline float to_float(float f) { return f; }
__device__ inline void set(uint16_t& p, float f) { p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
__device__ inline void set(float& p, float f) { p = f; }

// sine and cosine of position * frequency radians
__device__ inline void angle_of(int position, double frequency, float& sin_t, float& cos_t) {
    double turns = position * (frequency * 0.15915494309189535);   // 1 / (2 pi)
    turns -= rint(turns);                                          // [-1/2, 1/2]
    const double quarter = rint(turns * 4.0);
    const float t = static_cast<float>((turns - quarter * 0.25) * 6.283185307179586), u = t * t;
    const float s = t * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
    const float c = fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const int n = static_cast<int>(quarter) & 3;
    const float a = n & 1 ? c : s, b = n & 1 ? s : c;
    sin_t = n & 2 ? -a : a;
    cos_t = n == 1 || n == 2 ? -b : b;
}

// A thread takes one 16-byte piece of a head's first elements (kPer pairs) and its partners, computes their angles once and goes through
// its share of the row's heads; heads are dealt to `slices` threads where rows are few.
template <typename Elem, bool kPairs>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
    constexpr int kPer = 16 / sizeof(Elem);
    const int chunks = a.half / kPer;
    const int64_t item = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    const int chunk = static_cast<int>(item % chunks);
    const int64_t rest = item / chunks;
    if (rest >= a.rows * a.slices) return;
    const int row = static_cast<int>(a.first + rest / a.slices), slice = static_cast<int>(rest % a.slices);
    int pos;
    if (a.positions) pos = a.positions[row];
    else if (row >= a.total_prefill_q) pos = a.seq_lens[a.num_prefill + row - a.total_prefill_q] - 1;
    else pos = a.num_prefill > 0 ? query_row(a.cu_seqlens_q, a.seq_lens, a.num_prefill, row).pos : -1;
    if (pos < 0) return;   // no token
    float sin_t[kPer], cos_t[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        angle_of(pos, a.frequencies[chunk * kPer + j], sin_t[j], cos_t[j]);
        sin_t[j] *= a.magnitude;
        cos_t[j] *= a.magnitude;
    }
    union Piece { u32x4 v; Elem e[kPer]; };
    const int total = a.num_heads[0] + a.num_heads[1];
    for (int head = slice; head < total; head += a.slices) {
        const int which = head < a.num_heads[0] ? 0 : 1;
        Elem* p = static_cast<Elem*>(a.heads[which]) + row * a.stride[which] + static_cast<int64_t>(head - (which ? a.num_heads[0] : 0)) * a.head_dim;
        u32x4* lo = reinterpret_cast<u32x4*>(p + (kPairs ? 2 * chunk : chunk) * kPer);
        u32x4* hi = kPairs ? lo + 1 : reinterpret_cast<u32x4*>(p + a.half + chunk * kPer);
        Piece x, y;
        x.v = *lo;
        y.v = *hi;
        if constexpr (kPairs) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                Piece& z = j < kPer / 2 ? x : y;
                const int at = 2 * (j % (kPer / 2));
                const float u = to_float(z.e[at]), v = to_float(z.e[at + 1]);
                set(z.e[at], u * cos_t[j] - v * sin_t[j]);
                set(z.e[at + 1], v * cos_t[j] + u * sin_t[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const float u = to_float(x.e[j]), v = to_float(y.e[j]);
                set(x.e[j], u * cos_t[j] - v * sin_t[j]);
                set(y.e[j], v * cos_t[j] + u * sin_t[j]);
            }
        }
        *lo = x.v;
        *hi = y.v;
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryShape& s, void* q, void* k, const int32_t* positions, const int32_t* cu_seqlens_q, const int32_t* seq_lens,
                         int num_prefill, int total_prefill_q, int rows, const double* frequencies, hipStream_t st) {
    const int heads = (q ? s.hq : 0) + (k ? s.hkv : 0);
    if (rows == 0 || heads == 0) return hipSuccess;
    RotaryArgs a{{q, k}, {q ? s.hq : 0, k ? s.hkv : 0}, {s.q_stride, s.k_stride}, positions, cu_seqlens_q, seq_lens, frequencies, 0, 0,
                 num_prefill, total_prefill_q, s.head_dim, s.rot_dim / 2, 1, s.magnitude};
    const int chunks = a.half * s.elem / 16;
    // enough threads for every compute unit; beyond that a thread's angles serve all heads of its row
    while (a.slices < heads && static_cast<int64_t>(rows) * chunks * a.slices < 256 * 256) a.slices *= 2;
    a.slices = a.slices < heads ? a.slices : heads;
    // rows beyond the threads of one launch go into further ones
    const int64_t per_row = static_cast<int64_t>(chunks) * a.slices, most = most_workgroups(kThreads) * kThreads / per_row;
    auto run = [&](auto kernel) -> hipError_t {
        for (a.first = 0; a.first < rows; a.first += most) {
            a.rows = rows - a.first < most ? rows - a.first : most;
            kernel<<<static_cast<unsigned>((a.rows * per_row + kThreads - 1) / kThreads), kThreads, 0, st>>>(a);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    if (s.elem == 2) return s.pairs ? run(rotary_kernel<uint16_t, true>) : run(rotary_kernel<uint16_t, false>);
    return s.pairs ? run(rotary_kernel<float, true>) : run(rotary_kernel<float, false>);
}

}  // namespace shiftattn
