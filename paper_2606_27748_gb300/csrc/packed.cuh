// Packed batches: rows of several sequences one after the other, found through int32 offsets.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

namespace flex {

// A packed call as the kernels see it (include/flexattn.h, flex_packed).  Strides in elements.
struct Packed {
    int n, T, Tk, H, Hk, d, bf16;
    long long qs, ks, vs;
};

// Rows [lo, hi) of sequence s; offsets outside [0, T] are clamped and a decreasing pair counts
// as an empty sequence, so that whatever the offsets hold no row outside the tensors is touched.
__device__ __forceinline__ void seq_rows(const int* cu, int s, int T, int& lo, int& hi)
{
    lo = min(max(__ldg(cu + s), 0), T);
    hi = max(min(__ldg(cu + s + 1), T), lo);
}

// Blocks of `rows` rows, counted per sequence.  Sequence s starts at slot lo / rows + s: since
// floor((a + b) / r) + 1 >= floor(a / r) + ceil(b / r), no two sequences share a slot and
// T / rows + n slots hold them all; a slot that no block takes is skipped.  So a slot's place
// in memory is known without summing over the sequences before it.
inline __host__ __device__ int block_slots(int T, int n, int rows) { return T / rows + n; }

// The sequence and its block that a slot stands for; false for a slot that none takes.
// Executed by a whole warp (every lane gets the answer): 32 sequences are looked at at once,
// two rounds of loads for up to 1024 sequences.
__device__ __forceinline__ bool find_block(const int* cu, int n, int T, int rows, int slot, int& s,
                                           int& block, int& lo, int& hi)
{
    const int lane = threadIdx.x & 31;
    int first = 0, count = n;  // the last sequence whose first slot is <= slot lies in here
    while (count > 1) {
        const int step = (count + 31) / 32;
        const int i = first + lane * step;
        bool le = false;
        if (lane * step < count) le = min(max(__ldg(cu + i), 0), T) / rows + i <= slot;
        const unsigned hit = __ballot_sync(0xffffffffu, le);
        const int at = hit ? 31 - __clz(hit) : 0;
        const int end = first + count;
        first += at * step;
        count = min(step, end - first);
    }
    s = first;
    seq_rows(cu, s, T, lo, hi);
    block = slot - (lo / rows + s);
    return block >= 0 && (long long)block * rows < hi - lo;
}

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f32(float& y, float x) { y = x; }
__device__ __forceinline__ void from_f32(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

// Four consecutive elements (16 or 8 bytes, aligned) as floats.  Plain loads: some of what goes
// through them was written by the kernel before (see grid_dep_wait).
__device__ __forceinline__ float4 load4(const float* p) { return *(const float4*)p; }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p)
{
    const uint2 r = *(const uint2*)p;
    return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u),
                       __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
}
__device__ __forceinline__ void store4(float* p, float4 v) { *(float4*)p = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, float4 v)
{
    __nv_bfloat162 a = __floats2bfloat162_rn(v.x, v.y), b = __floats2bfloat162_rn(v.z, v.w);
    *(uint2*)p = make_uint2(*(uint32_t*)&a, *(uint32_t*)&b);
}

// Four elements as they lie in memory.
template <typename T>
struct Quad;
template <>
struct Quad<float> {
    float4 r;
    __device__ __forceinline__ void load(const float* p) { r = *(const float4*)p; }
    __device__ __forceinline__ void store(float* p) const { *(float4*)p = r; }
    __device__ __forceinline__ void zero() { r = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void low() { r.x = r.y = r.z = r.w = __uint_as_float(0xff800000u); }
    __device__ __forceinline__ float4 get() const { return r; }
};
template <>
struct Quad<__nv_bfloat16> {
    uint2 r;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { r = *(const uint2*)p; }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *(uint2*)p = r; }
    __device__ __forceinline__ void zero() { r = make_uint2(0u, 0u); }
    __device__ __forceinline__ void low() { r = make_uint2(0xff80ff80u, 0xff80ff80u); }  // -inf
    __device__ __forceinline__ float4 get() const
    {
        return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u),
                           __uint_as_float(r.y << 16), __uint_as_float(r.y & 0xffff0000u));
    }
};

// Four elements to shared memory, not waited for; zeros where `in` is false.
__device__ __forceinline__ void copy_quad(float* to, const float* from, bool in)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)),
                 "l"(from), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_quad(__nv_bfloat16* to, const __nv_bfloat16* from, bool in)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)),
                 "l"(from), "r"(in ? 8 : 0) : "memory");
}

// Copies since the last call are a group; all groups but the youngest N have arrived (for this thread).
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// 2^x and 1 / x, one instruction each: two units in the last place and one, denormals as 0.
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
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
// 1 / (1 + exp(-x)), a few units in the last place; 0 and 1 where exp(-x) leaves fp32.
__device__ __forceinline__ float logistic(float x) { return rcp(1.f + ex2(-kLog2e * x)); }

}  // namespace flex
