// Selective state space scan: what its kernels share.  Per channel c and state i, with
// D_t = softplus(dt_t + bias),
//   h_t[i] = exp(D_t A[c][i]) h_{t-1}[i] + D_t x_t B_t[i],  y_t = sum_i C_t[i] h_t[i] + Ds x_t,
//   out_t = y_t silu(z_t).
#pragma once

#include "packed.cuh"
#include "tc_util.cuh"

namespace flex {

struct SsmArgs {  // (declared in flex_internal.h)
    int n, T, D, G, N, bf16, softplus;
    long long xs, ds, bs, cs, zs;  // row strides in elements
    const void *x, *dt, *B, *C, *z;
    const float *A, *Ds, *bias;
    const int* cu;
    const float* h0;
    float* h1;
    void* out;
    int rows;     // tokens of a block; T + 1: sequences are not cut
    float* ends;  // [slots][D][N]: what a block's tokens alone leave behind
    float* sums;  // [slots][D]: sum of its D_t
    float* marks; // NULL, or the states ahead of every kTile tokens, [mark slots][D][N]
    // backward
    const void* dout;
    void *dx, *ddt, *dB, *dC, *dz;
    float *dA, *dDs, *dbias;
    float *part_bc;  // [tiles of a group][T][G][2 N]: sums of dB, dC over a tile's channels
    float *part_a;   // [slots][D][N]
    float *part_d;   // [slots][2][D]: dDs, dbias
};

namespace ssm {

constexpr int kTile = 16;  // tokens staged at a time, and between two marks
constexpr int kSMs = 152;  // of a GB300: a workspace's size is to depend on the shape alone

// A thread holds 4 states of one channel; L = N / 4 lanes hold a channel.  Blocks of 64 channels,
// or 32 where a channel takes 8 lanes and more.
template <int L>
struct Cfg {
    static constexpr int N = 4 * L, CT = L <= 4 ? 64 : 32, THREADS = CT * L;
    static constexpr int QUADS = kTile * CT / 4;  // groups of 4 channels of a token in a tile
    static constexpr int PT = QUADS > THREADS ? QUADS / THREADS : 1;  // of them a thread stages
    static constexpr int BC = kTile * N / 2;      // groups of 4 values of B and C in a tile
    static constexpr int PBC = BC > THREADS ? BC / THREADS : 1;
};
inline int tile_channels(int N) { return N <= 16 ? 64 : 32; }
inline int group_tiles(const SsmArgs& a)
{
    const int c = tile_channels(a.N);
    return (a.D / a.G + c - 1) / c;
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

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x)
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLog2eLow = 1.925963033500e-08f;  // log2(e) - float(log2(e))

// exp(x) for x <= 0 and above -80: 2^hi with the product's own rounding made good
__device__ __forceinline__ float exp_neg(float x)
{
    const float hi = x * kLog2e;
    const float lo = fmaf(x, kLog2eLow, fmaf(x, kLog2e, -hi));
    const float y = ex2(hi);
    return fmaf(y, lo * 0.693147180559945f, y);
}

// softplus(x) = max(x, 0) + log1p(t), t = exp(-|x|), with log1p(t) = 2 atanh(s), s = t / (2 + t)
// <= 1/3, by its series in s^2 up to s^15 (the next term is 7e-10 of the sum); t is exact to its
// last bits however small, as a step near 0.001 needs it.
__device__ __forceinline__ float softplus(float x)
{
    const float t = exp_neg(fmaxf(-fabsf(x), -80.f));
    const float s = t * rcp(2.f + t), y = s * s;
    float p = fmaf(y, 1.f / 15, 1.f / 13);
    p = fmaf(p, y, 1.f / 11);
    p = fmaf(p, y, 1.f / 9);
    p = fmaf(p, y, 1.f / 7);
    p = fmaf(p, y, 1.f / 5);
    p = fmaf(p, y, 1.f / 3);
    p = fmaf(p, y, 1.f);
    const float top = x > 0.f ? x : (x == x ? 0.f : x);  // (a NaN stays one)
    return fmaf(2.f * s, p, top);
}
// its derivative
__device__ __forceinline__ float sigmoid(float x)
{
    const float t = exp_neg(fmaxf(-fabsf(x), -80.f)), r = rcp(1.f + t);
    const float y = x > 0.f ? r : t * r;
    return x == x ? y : x;
}

// Four elements as they lie in memory.
template <typename T>
struct Quad;
template <>
struct Quad<float> {
    float4 r;
    __device__ __forceinline__ void load(const float* p) { r = *(const float4*)p; }
    __device__ __forceinline__ void zero() { r = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ float4 get() const { return r; }
};
template <>
struct Quad<__nv_bfloat16> {
    uint2 r;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = *(const uint2*)p; }
    __device__ __forceinline__ void zero() { r = make_uint2(0u, 0u); }
    __device__ __forceinline__ float4 get() const
    {
        return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u),
                           __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
    }
};

struct alignas(16) F2x2 {  // a thread's 4 states as packed pairs
    uint64_t x, y;
    __device__ __forceinline__ void from(float4 v)
    {
        x = tc::f2_pack(v.x, v.y);
        y = tc::f2_pack(v.z, v.w);
    }
    __device__ __forceinline__ float4 get() const
    {
        float4 v;
        tc::f2_unpack(x, v.x, v.y);
        tc::f2_unpack(y, v.z, v.w);
        return v;
    }
    __device__ __forceinline__ float dot(const F2x2& o) const
    {
        float lo, hi;
        tc::f2_unpack(tc::f2_fma(y, o.y, tc::f2_mul(x, o.x)), lo, hi);
        return lo + hi;
    }
};
// exp(d A) for A2 = A log2(e)
__device__ __forceinline__ F2x2 decay(const F2x2& A2, uint64_t dd)
{
    F2x2 e;
    e.x = tc::f2_mul(A2.x, dd);
    e.y = tc::f2_mul(A2.y, dd);
    const float4 v = e.get();
    e.from(make_float4(ex2(v.x), ex2(v.y), ex2(v.z), ex2(v.w)));
    return e;
}

// Where a block of threads stands: its channels and its rows of one sequence.
struct Place {
    int slot, s, block, lo, hi, first, last;  // rows [first, last) of sequence [lo, hi)
    int g, c0, nc, tile;                      // group, first channel, channels, tile of the group
};
// false where the slot has no rows (an empty sequence has one such slot, block 0, to itself)
template <int L>
__device__ __forceinline__ bool find_place(const SsmArgs& a, int index, Place& p)
{
    const int Dg = a.D / a.G, tiles = (Dg + Cfg<L>::CT - 1) / Cfg<L>::CT, all = tiles * a.G;
    p.slot = index / all;
    const int t = index % all;
    p.g = t / tiles;
    p.tile = t % tiles;
    p.c0 = p.g * Dg + p.tile * Cfg<L>::CT;
    p.nc = min(Cfg<L>::CT, Dg - p.tile * Cfg<L>::CT);
    const bool found = find_block(a.cu, a.n, a.T, a.rows, p.slot, p.s, p.block, p.lo, p.hi);
    p.first = found ? p.lo + p.block * a.rows : p.lo;
    p.last = min((long long)p.hi, (long long)p.first + a.rows);
    return found;
}

}  // namespace ssm
}  // namespace flex
