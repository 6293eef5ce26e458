// What the softmax attention kernels share: their arguments, and the keys that a block takes.
#pragma once

#include "packed.cuh"

namespace flex {

struct AttnArgs {
    Packed p;
    const void *q, *k, *v;
    const int *cu_q, *cu_k;
    float scale;
    int causal, splits;
    void* out;
    float* lse;       // [T][H] or NULL
    float* part;      // [splits][T][H][d] and
    float* part_lse;  // [splits][T][H], with splits > 1
    int* status;
};

// Blocks [first, last) of `size` keys that range `split` of a tile takes: those up to the key
// `newest` that its last row sees (causal), cut evenly.
__device__ __forceinline__ void key_range(const AttnArgs& x, int size, int lk, int newest, int split,
                                          int& first, int& last)
{
    const int n = x.causal ? min(lk, max(newest + 1, 0)) : lk;
    const long long blocks = (n + size - 1) / size;
    first = (int)(blocks * split / x.splits);
    last = (int)(blocks * (split + 1) / x.splits);
}

}  // namespace flex
