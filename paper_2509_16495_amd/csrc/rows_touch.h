// Do the rows of two strided arrays have bytes in common?  Nothing of HIP in here: the library and a host test share the function.
#pragma once
#include <stdint.h>

namespace shiftattn {

// sum of floor((a i + b) / m) over i = 0 .. n - 1, by the steps of Euclid's algorithm: after the whole parts of a / m and b / m, the sum counts the
// points below a line, which seen from the other axis are those of a line with m and a exchanged
inline unsigned __int128 sum_of_floors(unsigned __int128 n, unsigned __int128 m, unsigned __int128 a, unsigned __int128 b) {
    unsigned __int128 sum = 0;
    for (;;) {
        sum += n * (n - 1) / 2 * (a / m) + n * (b / m);
        a %= m, b %= m;
        const unsigned __int128 top = a * n + b;
        if (top < m) return sum;
        n = top / m, b = top % m;
        const unsigned __int128 t = m;
        m = a, a = t;
    }
}

// n rows of a_bytes from a on, a_stride apart, and n of b_bytes from b on, b_stride apart (strides and sizes in bytes, at least 1)
inline bool rows_touch(uint64_t a, int64_t a_bytes, __int128 a_stride, uint64_t b, int64_t b_bytes, __int128 b_stride, int64_t n) {
    // With t = a - b + i a_stride, row i meets row j where t - b_bytes < j b_stride < t + a_bytes.
    const __int128 d = static_cast<__int128>(a) - static_cast<__int128>(b), end = (n - 1) * b_stride;   // (j's last place)
    if (n < 1 || d >= end + b_bytes || -d >= (n - 1) * a_stride + a_bytes) return false;
    // the rows i that lie between the first and the last j
    const __int128 first = d > -a_bytes ? 0 : (-a_bytes - d) / a_stride + 1, behind = (end + b_bytes - 1 - d) / a_stride, last = behind < n - 1 ? behind : n - 1;
    if (first > last) return false;
    const __int128 t = d + first * a_stride;
    if (t < b_bytes || d + last * a_stride + a_bytes > end) return true;   // they meet the first j, or the last
    // else every multiple of b_stride that one of them meets is some j's
    const auto meets = static_cast<unsigned __int128>(last - first + 1);
    return sum_of_floors(meets, b_stride, a_stride, t + a_bytes - 1) != sum_of_floors(meets, b_stride, a_stride, t - b_bytes);
}

}  // namespace shiftattn
