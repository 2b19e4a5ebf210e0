// Which token a row of q and out stands for, in the kernels that take a row at a time.  Nothing of HIP in here: the kernels and a
// host test that walks batches share the function.
#pragma once
#include <stdint.h>

namespace shiftattn {

// seq < 0: the row stands for no token (it has no keys, and its place in out stays as it was)
struct QueryRow {
    int seq, pos;   // sequence, position in it: the row sees positions 0 .. pos
};

// cu_seqlens_q null: decode rows, one a sequence.  Else the rows of chunks, of which there may be more than cu_seqlens_q[num_seqs] says:
// the count comes from the host, the lengths from the device, where a chunk may have been refused.  num_seqs >= 1.
constexpr QueryRow query_row(const int32_t* cu_seqlens_q, const int32_t* seq_lens, int num_seqs, int tok) {
    if (cu_seqlens_q == nullptr) return {tok, seq_lens[tok] - 1};
    if (tok >= cu_seqlens_q[num_seqs]) return {-1, -1};
    int lo = 0, hi = num_seqs;  // last s with cu[s] <= tok
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (cu_seqlens_q[mid] <= tok) lo = mid; else hi = mid;
    }
    return {lo, seq_lens[lo] - cu_seqlens_q[lo + 1] + tok};
}

}  // namespace shiftattn
