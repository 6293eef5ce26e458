// Selective state space scan: what its kernels share.  Per channel c and state i, with
// D_t = softplus(dt_t + bias),
//   h_t[i] = exp(D_t A[c][i]) h_{t-1}[i] + D_t x_t B_t[i],  y_t = sum_i C_t[i] h_t[i] + Ds x_t,
//   out_t = y_t silu(z_t).
#pragma once

#include "packed.cuh"
#include "tc_util.cuh"

namespace flex {

struct SsmArgs {
    int n, T, D, G, N, bf16, softplus;
    long long xs, ds, bs, cs, zs;  // row strides in elements
    const void *x, *dt, *B, *C, *z;
    const float *A, *Ds, *bias;
    const int* cu;
    const float* h0;
    float* h1;
    void* out;
    int rows;     // tokens of a block; T + 1: sequences are not cut
    float* ends;  // [slots][D][N]: what a block's tokens alone leave behind, then what it starts from
    float* sums;  // [slots][D]: sum of its D_t
    bool joined;  // ends are joined before the walk
    float* marks; // NULL, or the states ahead of every kMark tokens, [mark slots][D][N]
    // backward
    const void* dout;
    void *dx, *ddt, *dB, *dC, *dz;
    float *dA, *dDs, *dbias;
    float *part_bc;  // [tiles of a group][T][G][2 N]: sums of dB, dC over a tile's channels
    float *part_a;   // [slots][D][N]
    float *part_d;   // [slots][2][D]: dDs, dbias
};

// Tokens of a block (64 of them and more, or 32 backward), or T + 1 where sequences stay whole.
int ssm_rows(const SsmArgs& a, bool backward);
bool ssm_joined(const SsmArgs& a);    // forward
int ssm_bwd_tiles(const SsmArgs& a);  // blocks of a group's channels in the backward
cudaError_t launch_ssm_fwd(const SsmArgs& a, cudaStream_t s);        // 1 kernel, cut: 2, or 3 if joined
cudaError_t launch_ssm_back_ends(const SsmArgs& a, cudaStream_t s);  // 2
cudaError_t launch_ssm_bwd(const SsmArgs& a, cudaStream_t s);        // 2 kernels, cut: 4
cudaError_t launch_ssm_decode(const SsmArgs& a, cudaStream_t s);     // 1

namespace ssm {

constexpr int kTile = 16;  // tokens of the forward's tiles
constexpr int kMark = 8;   // tokens between two marks, and of the backward's tiles
constexpr int kSMs = 152;  // of a GB300: a workspace's size is to depend on the shape alone

inline int group_tiles(const SsmArgs& a, int channels)
{
    return (a.D / a.G + channels - 1) / channels;
}

// Sums of L values over L lanes (lane p of them): lane p returns the one of value slot(p).  Every
// step halves the values that a lane still adds up.
template <int L>
__device__ __forceinline__ float lane_sums(float (&x)[L], int p)
{
#pragma unroll
    for (int m = L / 2; m >= 1; m /= 2) {
        const bool up = p & m;
#pragma unroll
        for (int i = 0; i < m; ++i) {
            const float give = up ? x[i] : x[i + m], keep = up ? x[i + m] : x[i];
            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, m);
        }
    }
    return x[0];
}

__device__ __forceinline__ float max_nan(float x, float y)  // a NaN stays one
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}
// exp(-|x|), 0 from 111 on; off by 3e-7 at 7, where steps near 0.001 lie (the product's rounding)
__device__ __forceinline__ float exp_neg(float x)
{
    return ex2(max_nan(-fabsf(x), -111.f) * kLog2e);
}

// softplus(x) = max(x, 0) + log1p(t), t = exp(-|x|) in [0, 1], of 4 values.  log1p(t) / t is a
// polynomial of degree 8 (least relative error, 3e-8, found by exchange), so that small steps keep
// their relative accuracy.  0 for -inf, exactly.
__device__ constexpr float soft(int k)
{
    constexpr float c[9] = {9.9999996988e-01f, -4.9999493140e-01f, 3.3319096808e-01f,
                            -2.4842982216e-01f, 1.9106006770e-01f, -1.3663245815e-01f,
                            7.8225952120e-02f, -2.9505238928e-02f, 5.2326943023e-03f};
    return c[k];
}
__device__ __forceinline__ void softplus4(float (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        float a = max_nan(-fabsf(x[i]), -111.f), b = max_nan(-fabsf(x[i + 1]), -111.f);
        tc::f2_unpack(tc::f2_mul(tc::f2_pack(a, b), tc::f2_pack(kLog2e, kLog2e)), a, b);
        const uint64_t t = tc::f2_pack(ex2(a), ex2(b));
        uint64_t p = tc::f2_pack(soft(8), soft(8));
#pragma unroll
        for (int k = 7; k >= 0; --k) p = tc::f2_fma(p, t, tc::f2_pack(soft(k), soft(k)));
        p = tc::f2_fma(p, t, tc::f2_pack(fmaxf(x[i], 0.f), fmaxf(x[i + 1], 0.f)));
        tc::f2_unpack(p, x[i], x[i + 1]);
    }
}
__device__ __forceinline__ float softplus(float x)
{
    const float t = exp_neg(x);
    float p = soft(8);
#pragma unroll
    for (int k = 7; k >= 0; --k) p = fmaf(p, t, soft(k));
    return fmaf(p, t, fmaxf(x, 0.f));
}
// its derivative
__device__ __forceinline__ float sigmoid(float x)
{
    const float t = exp_neg(x), r = rcp(1.f + t);
    return x < 0.f ? t * r : r;
}
__device__ __forceinline__ float silu(float x) { return x * logistic(x); }

// ex2.approx comes out 0 to 5e-8 low on average (by up to 2.7e-8 where a state lasts for tens of
// tokens), which adds up over the tokens a state lasts; kUp in the exponent makes half of that good, at
// no cost (dA of 8 x 1024 tokens: 1.3e-6 off without, 4.9e-7 with it and sums of sums).
constexpr float kUp = 2e-8f;

// SP states as packed pairs.
template <int SP>
struct States {
    uint64_t v[SP / 2];
    __device__ __forceinline__ void read(const float* p)
    {
#pragma unroll
        for (int i = 0; i < SP / 4; ++i) {
            const ulonglong2 u = *(const ulonglong2*)(p + 4 * i);
            v[2 * i] = u.x;
            v[2 * i + 1] = u.y;
        }
    }
    __device__ __forceinline__ void write(float* p) const
    {
#pragma unroll
        for (int i = 0; i < SP / 4; ++i) *(ulonglong2*)(p + 4 * i) = make_ulonglong2(v[2 * i], v[2 * i + 1]);
    }
    __device__ __forceinline__ void zero()
    {
#pragma unroll
        for (int i = 0; i < SP / 2; ++i) v[i] = 0;
    }
};
// The second half's own barrier: each thread's copies are there for all of it.
__device__ __forceinline__ void bring_barrier(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }

__device__ __forceinline__ uint64_t ex2_pair(uint64_t x)
{
    float a, b;
    tc::f2_unpack(x, a, b);
    return tc::f2_pack(ex2(a), ex2(b));
}
__device__ __forceinline__ uint64_t twice(float x) { return tc::f2_pack(x, x); }

// Where a block of threads stands: its channels and its rows of one sequence.
struct Place {
    int slot, s, block, lo, hi, first, last;  // rows [first, last) of sequence [lo, hi)
    int g, c0, nc, tile;                      // group, first channel, channels, tile of the group
};
// false where the slot has no rows (an empty sequence has one such slot, block 0, to itself)
template <int CT>
__device__ __forceinline__ bool find_place(const SsmArgs& a, int index, Place& p)
{
    const int Dg = a.D / a.G, tiles = (Dg + CT - 1) / CT, all = tiles * a.G;
    p.slot = index / all;
    const int t = index % all;
    p.g = t / tiles;
    p.tile = t % tiles;
    p.c0 = p.g * Dg + p.tile * CT;
    p.nc = min(CT, Dg - p.tile * CT);
    const bool found = find_block(a.cu, a.n, a.T, a.rows, p.slot, p.s, p.block, p.lo, p.hi);
    p.first = found ? p.lo + p.block * a.rows : p.lo;
    p.last = min((long long)p.hi, (long long)p.first + a.rows);
    return found;
}

}  // namespace ssm
}  // namespace flex
