// Short causal convolution and norms around the recurrence: what their kernels share.
#pragma once

#include "packed.cuh"
#include "tc_util.cuh"

namespace flex {

struct ConvArgs {
    int n, T, D, W, bf16, silu;
    long long xs;  // row stride in elements
    const void* x;
    const float *w, *bias;  // [D][W], [D]
    const int* cu;
    const void* S0;  // [n][W - 1][D], oldest row first
    void* S1;
    void* out;
    int run;  // rows of a thread
    // backward
    const void* dout;
    void* dx;
    float *dw, *dbias;
    float* part;  // [blocks of rows][W + 1][D]
};

struct NormArgs {
    int T, H, d, bf16, heads;  // heads: of the parameters, 1 or H
    float eps;
    long long xs, zs, rs;
    const void *x, *z, *res;
    const float *w, *scale;
    const int* end;  // NULL, or how many rows there are
    void *out, *total;
    float* rstd;
    // backward
    const void *dout, *dtotal;
    void *dx, *dres, *dz;
    float *dw, *dscale;
    float* part;  // [groups of threads][1 or 2][d]
};

// N consecutive elements of 16 bytes in all (8 bytes: half of them), as they lie in memory.
template <typename T>
struct Pack;
template <>
struct Pack<float> {
    static constexpr int N = 4;
    float4 r;
    __device__ __forceinline__ void load(const float* p) { r = *(const float4*)p; }
    __device__ __forceinline__ void store(float* p) const { *(float4*)p = r; }
    __device__ __forceinline__ void zero() { r = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&v)[4]) const { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
    __device__ __forceinline__ void set(const float (&v)[4]) { r = make_float4(v[0], v[1], v[2], v[3]); }
};
template <>
struct Pack<__nv_bfloat16> {
    static constexpr int N = 8;
    uint4 r;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = *(const uint4*)p; }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *(uint4*)p = r; }
    __device__ __forceinline__ void zero() { r = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void get(float (&v)[8]) const
    {
        const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(u[i] << 16);
            v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&v)[8])
    {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            u[i] = *(const uint32_t*)&b;
        }
        r = make_uint4(u[0], u[1], u[2], u[3]);
    }
};

// N consecutive fp32 parameters (16-byte aligned).
template <int N>
__device__ __forceinline__ void load_params(float (&v)[N], const float* p)
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const float4 u = *(const float4*)(p + i);
        v[i] = u.x; v[i + 1] = u.y; v[i + 2] = u.z; v[i + 3] = u.w;
    }
}

// Sums of a matrix's columns in a fixed order (conv.cu): to[k][c] for c < cols, over rows
// first + k + i * step, i < count, of `from` [..][cols].  `split` columns go to to0, the rest to to1
// (or nowhere, if NULL), both [sums][their columns].
cudaError_t launch_column_sums(const float* from, int cols, int split, int sums, int step, int count,
                               float* to0, float* to1, cudaStream_t s);

int conv_run(const ConvArgs& a);         // rows of a thread (ConvArgs::run)
int conv_bwd_blocks(const ConvArgs& a);  // blocks of rows, of which each leaves sums
cudaError_t launch_conv_fwd(const ConvArgs& a, cudaStream_t s);     // 1 kernel
cudaError_t launch_conv_bwd(const ConvArgs& a, cudaStream_t s);     // 2
cudaError_t launch_conv_decode(const ConvArgs& a, cudaStream_t s);  // 1
int norm_bwd_blocks(const NormArgs& a);
size_t norm_part_floats(const NormArgs& a);
cudaError_t launch_norm_fwd(const NormArgs& a, cudaStream_t s);     // 1
cudaError_t launch_norm_bwd(const NormArgs& a, cudaStream_t s);     // 2

}  // namespace flex
