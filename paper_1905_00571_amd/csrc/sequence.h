// Layers on packed sequences: what the causal convolution and the selective scan share.
#pragma once

#include "internal.h"

namespace cadnn {

// Tokens of several sequences lie one behind the other.  `start` (device, seqs + 1 offsets, or NULL: all sequences are
// tokens / seqs long) is the caller's; it cannot be checked before the launch, so what it says is cut to [0, tokens] here.
struct Sequences {
    const int32_t* start;
    int tokens, seqs;
};

__device__ __forceinline__ void seq_range(const Sequences& q, int s, int* lo, int* hi) {
    if (q.start) {
        const int a = min(max(q.start[s], 0), q.tokens), b = min(max(q.start[s + 1], 0), q.tokens);
        *lo = a;
        *hi = max(a, b);
    } else {
        const int per = q.tokens / q.seqs;
        *lo = s * per;
        *hi = *lo + per;
    }
}

// Work is cut into pieces of `chunk` tokens of one sequence.  The host does not know the sequences' lengths, so their
// pieces get places ("slots") by a rule that needs no sums: sequence s begins at slot start[s] / chunk + s, which leaves
// it floor(end / chunk) - floor(start / chunk) + 1 >= ceil(length / chunk) places.  Sequences of one length have none to spare.
inline int64_t seq_slots(int tokens, int seqs, bool ragged, int chunk) {
    if (ragged) return (int64_t)tokens / chunk + seqs;
    const int per = tokens / seqs;
    return (int64_t)seqs * ((per + chunk - 1) / chunk);
}

__device__ __forceinline__ int seq_first_slot(const Sequences& q, int s, int chunk) {
    if (q.start) return min(max(q.start[s], 0), q.tokens) / chunk + s;
    return s * ((q.tokens / q.seqs + chunk - 1) / chunk);
}

// The sequence that owns a slot (the last one that begins at or before it) and the slot's place in it.
__device__ __forceinline__ int seq_of_slot(const Sequences& q, int slot, int chunk, int* piece) {
    if (!q.start) {
        const int pieces = (q.tokens / q.seqs + chunk - 1) / chunk;
        *piece = slot % pieces;
        return slot / pieces;
    }
    int s = 0, n = q.seqs;            // the owner is among s .. s + n - 1
    while (n > 1) {
        const int half = n >> 1;
        if (seq_first_slot(q, s + half, chunk) <= slot) { s += half; n -= half; }
        else n = half;
    }
    *piece = slot - seq_first_slot(q, s, chunk);
    return s;
}

cadnn_status check_sequences(const char* who, int tokens, int seqs, const int32_t* seq_start);

}  // namespace cadnn
