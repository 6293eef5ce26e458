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

// Key heads and ranges of a tile side by side, then the tiles, longest first (find_tile's rank is
// blockIdx.z * gridDim.y + blockIdx.y).
inline dim3 softattn_grid(const AttnArgs& x, int tokens)
{
    const int slots = block_slots(x.p.T, x.p.n, tokens), y = slots < 65535 ? slots : 65535;
    return dim3((unsigned)(x.p.Hk * x.splits), (unsigned)y, (unsigned)((slots + y - 1) / y));
}

// One or two tokens a sequence on average: the step of a serving batch.
inline bool softattn_few(const Packed& p) { return p.T <= 2LL * p.n; }

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

// The tile of rows that CTA `rank` of a packed call takes: tiles of `tokens` tokens of all
// sequences, those with the most keys first, so that the last CTAs to start are the short ones
// (in the order of the rows, prompts of 4000, 1531, 700, .. tokens, H12 d64, took 84 us: the
// longest tiles started last).  A tile's work is the newest key it sees, in units of `tokens`; how
// many tiles have at least w units is a sum over the sequences, and a search for the largest w
// that still leaves more than `rank` tiles finds the tile.  Executed by a whole warp, whose lanes
// hold the sequences; more of them than kSorted go in the order of the rows (find_block).
constexpr int kSorted = 128;

__device__ __forceinline__ bool find_tile(const AttnArgs& x, int tokens, int rank, int& s, int& block,
                                          int& qlo, int& qhi)
{
    const Packed& pk = x.p;
    if (pk.n > kSorted) return find_block(x.cu_q, pk.n, pk.T, tokens, rank, s, block, qlo, qhi);
    constexpr int R = kSorted / 32;
    const int lane = threadIdx.x & 31, step = x.causal ? 1 : 0;
    int tiles[R] = {}, work[R] = {};  // of sequence lane + 32 i: tiles, and the first one's work
    int most = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        if (lane + 32 * i >= pk.n) continue;
        int a, b, c, d;
        seq_rows(x.cu_q, lane + 32 * i, pk.T, a, b);
        seq_rows(x.cu_k, lane + 32 * i, pk.Tk, c, d);
        tiles[i] = (b - a + tokens - 1) / tokens;
        work[i] = max((step ? (d - c) - (b - a) : d - c) / tokens, 0);
        if (tiles[i] > 0) most = max(most, work[i] + step * (tiles[i] - 1));
    }
    auto at_least = [&](int i, int w) {  // tiles of sequence i with at least w units
        return step ? max(min(tiles[i] - (w - work[i]), tiles[i]), 0) : work[i] >= w ? tiles[i] : 0;
    };
    auto count = [&](int w) {
        int c = 0;
#pragma unroll
        for (int i = 0; i < R; ++i) c += at_least(i, w);
        return (int)__reduce_add_sync(0xffffffffu, (unsigned)c);
    };
    if (rank >= count(0)) return false;
    int low = 0, high = __reduce_max_sync(0xffffffffu, most);  // count(low) > rank >= count(high + 1)
    while (low < high) {
        const int mid = (low + high + 1) >> 1;
        if (count(mid) > rank) low = mid;
        else high = mid - 1;
    }
    int left = rank - count(low + 1);  // among the tiles of exactly `low` units, in sequence order
    bool found = false;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const int all = at_least(i, low), here = all - at_least(i, low + 1);
        int upto = here;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const int o = __shfl_up_sync(0xffffffffu, upto, m);
            if (lane >= m) upto += o;
        }
        const int sum = __shfl_sync(0xffffffffu, upto, 31);
        if (!found && left < sum) {
            const int owner = __ffs(__ballot_sync(0xffffffffu, left < upto)) - 1;
            // its tiles with at least `low` units are its last `all`
            block = __shfl_sync(0xffffffffu, tiles[i] - all + left - (upto - here), owner);
            s = 32 * i + owner;
            found = true;
        }
        left -= found ? 0 : sum;
    }
    if (found) seq_rows(x.cu_q, s, pk.T, qlo, qhi);
    return found;
}

}  // namespace flex
