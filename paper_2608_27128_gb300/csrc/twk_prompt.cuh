// twk_prompt.cuh -- the sequences of a packed call and what their tokens see.
#pragma once
#include <cstdint>

#include "twk_prompt_internal.h"

namespace twk {

struct Sequence {
    int t0, n;       // first row of q, tokens
    int j0, m;       // first row of k, keys
    bool ok;         // false: a data error, n = m = 0
};

__device__ __forceinline__ void rows_of(const int* offsets, const int* lens, int b, int rows,
                                        int& first, int& count, bool& ok)
{
    first = offsets ? offsets[b] : 0;
    const int end = offsets ? offsets[b + 1] : rows;
    ok = ok && first >= 0 && first <= end && end <= rows;
    count = end - first;
    if (lens) {
        const int n = lens[b];
        ok = ok && n >= 0 && n <= count;
        count = n;
    }
}

__device__ __forceinline__ Sequence sequence_of(const PromptArgs& a, int b)
{
    Sequence q;
    q.ok = true;
    rows_of(a.seqs.offsets, a.seqs.lens, b, a.s.tokens, q.t0, q.n, q.ok);
    const bool own = a.seqs.k_offsets || !a.seqs.offsets;
    rows_of(own ? a.seqs.k_offsets : a.seqs.offsets,
            a.seqs.k_lens ? a.seqs.k_lens : own ? nullptr : a.seqs.lens, b, a.s.keys, q.j0, q.m,
            q.ok);
    if (!q.ok) q.n = q.m = 0;
    return q;
}

}  // namespace twk
