// Rotary positions (shiftattn_rotary, shiftattn_rotary_mixed): pairs of elements of the query and key heads of a row turned in place by
// angles that grow with the row's position, (a, b) -> m (a cos t - b sin t, b cos t + a sin t), t = position * frequency.
//
// The angle is reduced to a fraction of a turn in 64 bits: at position 10^6 a float32 product would have no fraction left that is worth
// anything (2^20 radians have a last place of 2^-3).  Both products, by 1 / (2 pi) and by the position, keep what their rounding leaves off: at position
// 2^31 that is up to 4e-7 radians for a frequency of 1, and more for higher ones.  A quarter of a turn around the nearest axis remains, where the Taylor series of
// sine to the ninth and of cosine to the tenth power are exact to 2 * 10^-9, a thirtieth of float32's last place.
#include "internal.h"
#include "query_rows.h"

namespace shiftattn {

namespace {

constexpr int kThreads = 256;
constexpr int kBatch = 2;         // heads of a lane whose loads are in flight together
constexpr int kMostPairs = 128;   // head_dim up to 256

struct RotaryArgs {
    void* heads[2];                 // queries, keys
    int num_heads[2];
    int64_t stride[2];
    const int32_t* positions;       // nullptr: from the two below
    const int32_t* cu_seqlens_q;
    const int32_t* seq_lens;
    const double* frequencies;
    int64_t first, rows;            // those of this launch
    int num_prefill, total_prefill_q, head_dim, half;
    float magnitude;
};

__device__ inline float to_float(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
__device__ inline float to_float(float f) { return f; }
__device__ inline void set(uint16_t& p, float f) { p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(f)); }
__device__ inline void set(float& p, float f) { p = f; }

// sine and cosine of position * frequency radians
__device__ inline void angle_of(int position, double frequency, float& sin_t, float& cos_t) {
    float t;
    double quarter;
    {
#pragma clang fp contract(off)   // (a product that joined a sum would bring the part that is added below)
        const double high = frequency * 0.15915494309189535;   // 1 / (2 pi), whose next 53 bits are those of -9.839338337591243e-18
        const double low = fma(frequency, 0.15915494309189535, -high) + frequency * -9.839338337591243e-18;
        const double turns = position * high, rest = fma(static_cast<double>(position), high, -turns) + position * low;
        const double part = turns - rint(turns);   // [-1/2, 1/2], exact
        quarter = rint(part * 4.0);
        t = static_cast<float>(((part - quarter * 0.25) + rest) * 6.283185307179586);
    }
    const float u = t * t;
    const float s = t * fmaf(u, fmaf(u, fmaf(u, fmaf(u, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
    const float c = fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const int n = static_cast<int>(quarter) & 3;
    const float a = n & 1 ? c : s, b = n & 1 ? s : c;
    sin_t = n & 2 ? -a : a;
    cos_t = n == 1 || n == 2 ? -b : b;
}

// A wavefront takes a row.  Its lanes compute the angles, a pair (or two) each, and hand them round through LDS; then a lane owns one
// 16-byte piece of a head's first elements (kPer pairs) and its partners, and the lanes lie side by side in memory over several heads.
// What bounds it is HBM, where it counts that neighbouring lanes' places lie side by side and that instructions are few: threads that went down a
// row's heads one by one touched 128 bytes here and there (65536 rows of 18 heads 124 us), and with the heads side by side but the angles
// worked out by every thread batches that fit the caches were bound by those (8192 rows of 9 heads 9.9 us).  This takes 115 (5.2 TB/s
// read + written) and 8.1.
template <typename Elem, bool kPairs>
__global__ __launch_bounds__(kThreads) void rotary_kernel(RotaryArgs a) {
    constexpr int kPer = 16 / sizeof(Elem);
    __shared__ float angles[kThreads / 64][2][kMostPairs];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t at = static_cast<int64_t>(blockIdx.x) * (kThreads / 64) + wave;
    if (at >= a.rows) return;   // (a wavefront as a whole; there is no barrier)
    const int row = static_cast<int>(a.first + at);
    int pos;
    if (a.positions) pos = a.positions[row];
    else if (row >= a.total_prefill_q) pos = a.seq_lens[a.num_prefill + row - a.total_prefill_q] - 1;
    else pos = a.num_prefill > 0 ? query_row(a.cu_seqlens_q, a.seq_lens, a.num_prefill, row).pos : -1;
    if (pos < 0) return;   // no token
    for (int i = lane; i < a.half; i += 64) {
        float sin_i, cos_i;
        angle_of(pos, a.frequencies[i], sin_i, cos_i);
        angles[wave][0][i] = sin_i * a.magnitude;
        angles[wave][1][i] = cos_i * a.magnitude;
    }
    __builtin_amdgcn_wave_barrier();
    const int chunks = a.half / kPer;                       // pieces of a head
    const int beside = 64 / chunks;                         // heads that the wavefront takes at once
    const int chunk = lane % chunks, slice = lane / chunks;
    if (slice >= beside) return;
    float sin_t[kPer], cos_t[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        sin_t[j] = angles[wave][0][chunk * kPer + j];
        cos_t[j] = angles[wave][1][chunk * kPer + j];
    }
    union Piece { u32x4 v; Elem e[kPer]; };
    const int total = a.num_heads[0] + a.num_heads[1];
    auto place = [&](int head) -> u32x4* {
        const int which = head < a.num_heads[0] ? 0 : 1;
        return reinterpret_cast<u32x4*>(static_cast<Elem*>(a.heads[which]) + row * a.stride[which] + static_cast<int64_t>(head - (which ? a.num_heads[0] : 0)) * a.head_dim +
                                        (kPairs ? 2 * chunk : chunk) * kPer);
    };
    const int partner = kPairs ? 1 : chunks;   // 16-byte pieces from the first to the second
    auto turn = [&](Piece& x, Piece& y) {
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
    };
    // heads in batches, all of a batch's loads in front of its stores (in place, the compiler cannot move a load up by itself)
    for (int first = slice; first < total; first += kBatch * beside) {
        Piece x[kBatch], y[kBatch];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int head = first + i * beside;
            if (head < total) {
                const u32x4* p = place(head);
                x[i].v = p[0];
                y[i].v = p[partner];
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const int head = first + i * beside;
            if (head < total) {
                turn(x[i], y[i]);
                u32x4* p = place(head);
                p[0] = x[i].v;
                p[partner] = y[i].v;
            }
        }
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryShape& s, void* q, void* k, const int32_t* positions, const int32_t* cu_seqlens_q, const int32_t* seq_lens,
                         int num_prefill, int total_prefill_q, int rows, const double* frequencies, hipStream_t st) {
    const int heads = (q ? s.hq : 0) + (k ? s.hkv : 0);
    if (rows == 0 || heads == 0) return hipSuccess;
    RotaryArgs a{{q, k}, {q ? s.hq : 0, k ? s.hkv : 0}, {s.q_stride, s.k_stride}, positions, cu_seqlens_q, seq_lens, frequencies, 0, 0,
                 num_prefill, total_prefill_q, s.head_dim, s.rot_dim / 2, s.magnitude};
    // rows beyond the threads of one launch go into further ones
    constexpr int64_t kRows = kThreads / 64, kMost = most_workgroups(kThreads) * kRows;
    auto run = [&](auto kernel) -> hipError_t {
        for (a.first = 0; a.first < rows; a.first += kMost) {
            a.rows = rows - a.first < kMost ? rows - a.first : kMost;
            kernel<<<static_cast<unsigned>((a.rows + kRows - 1) / kRows), kThreads, 0, st>>>(a);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        return hipSuccess;
    };
    if (s.elem == 2) return s.pairs ? run(rotary_kernel<uint16_t, true>) : run(rotary_kernel<uint16_t, false>);
    return s.pairs ? run(rotary_kernel<float, true>) : run(rotary_kernel<float, false>);
}

}  // namespace shiftattn
