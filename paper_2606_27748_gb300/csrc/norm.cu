// Norms around a block: r = x, or res + scale x (the residual stream, which is written too); out =
// r rstd w, rstd = (mean r^2 + eps)^-1/2 over the d elements of a head, times silu(z) where a gate is
// given; and the gradients.
//
// A group of threads, a power of two of them, takes a (row, head), 16 bytes at a time, and holds all of
// it in registers between the sum and what it is for.  Bound by DRAM: every tensor is read or written
// once.  The backward's groups stay with their head and walk rows, keeping sums for dw and dscale, with
// the rows ahead on their way to shared memory.  32768 x 16 heads of 128 with the gate: 71 us, 5.7 TB/s
// (1 unit of 16 bytes a thread instead of 2: 80); 16384 rows of 2048 with the residual sum: 47 us, and
// gradients 66 for 403 MB (88 with one row ahead in registers).  A backward row of more than 256 units (2048
// elements in bf16, 1024 in fp32) is 2 to 8 units a thread, 8 warps an SM in bf16, whose parameters are
// loaded again for every row: the same 403 MB as rows of 4096 take its two kernels 115 us, of 8192 107 (72 as
// rows of 2048).
#include "flex_internal.h"
#include "layer.cuh"

#include <type_traits>

namespace flex {
namespace {

constexpr int kThreads = 256;

// Sum over a group of `tpr` threads; past a warp through shared memory, two slots in turn.
__device__ __forceinline__ float group_sum(float v, int tpr, float* slots)
{
#pragma unroll
    for (int m = 16; m >= 1; m /= 2)
        if (m < tpr) v += __shfl_xor_sync(0xffffffffu, v, m);
    if (tpr <= 32) return v;
    const int warp = threadIdx.x / 32, per = tpr / 32, first = warp / per * per;
    if (threadIdx.x % 32 == 0) slots[warp] = v;
    __syncthreads();
    v = 0.f;
    for (int k = 0; k < per; ++k) v += slots[first + k];
    return v;
}

__device__ __forceinline__ int row_count(const NormArgs& a)
{
    return a.end ? min(max(__ldg(a.end), 0), a.T) : a.T;
}

template <typename T, int K>
__global__ void __launch_bounds__(kThreads) norm_fwd_kernel(NormArgs a, int tpr)
{
    constexpr int V = Pack<T>::N;
    __shared__ float slots[kThreads / 32];
    // (tpr is a power of two, and rows times heads fit 31 bits)
    const int lane = threadIdx.x & (tpr - 1), shift = 31 - __clz(tpr);
    const unsigned item = blockIdx.x * (kThreads >> shift) + (threadIdx.x >> shift);
    const unsigned t = item / (unsigned)a.H, h = item - t * a.H;
    const bool in = t < (unsigned)row_count(a);
    const size_t out = (size_t)item * a.d;
    Pack<T> xr[K], zr[K], rr[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (lane + k * tpr) * V;
        xr[k].zero(); zr[k].zero(); rr[k].zero();
        if (!in || e >= a.d) continue;
        xr[k].load((const T*)a.x + t * a.xs + h * a.d + e);
        if (a.res) rr[k].load((const T*)a.res + t * a.rs + h * a.d + e);
        if (a.z) zr[k].load((const T*)a.z + t * a.zs + h * a.d + e);
    }
    const int p = a.heads > 1 ? (int)h * a.d : 0;
    float r[K][V], sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (lane + k * tpr) * V;
        xr[k].get(r[k]);
        if (a.res) {
            float y[V], s[V];
            rr[k].get(y);
            if (a.scale && e < a.d) load_params<V>(s, a.scale + p + e);
#pragma unroll
            for (int q = 0; q < V; ++q) r[k][q] = a.scale ? fmaf(e < a.d ? s[q] : 0.f, r[k][q], y[q]) : r[k][q] + y[q];
            if (in && e < a.d) {
                rr[k].set(r[k]);
                rr[k].store((T*)a.total + out + e);
            }
        }
#pragma unroll
        for (int q = 0; q < V; ++q) sum = fmaf(r[k][q], r[k][q], sum);
    }
    sum = group_sum(sum, tpr, slots);
    const float rstd = rsqrtf(sum / (float)a.d + a.eps);
    if (!in) return;
    if (a.rstd && lane == 0) a.rstd[item] = rstd;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (lane + k * tpr) * V;
        if (e >= a.d) continue;
        float w[V], g[V];
        load_params<V>(w, a.w + p + e);
        zr[k].get(g);
#pragma unroll
        for (int q = 0; q < V; ++q) {
            r[k][q] *= rstd * w[q];
            if (a.z) r[k][q] *= g[q] * logistic(g[q]);
        }
        xr[k].set(r[k]);
        xr[k].store((T*)a.out + out + e);
    }
}

// With n = r rstd and g = dout silu(z): dn = g w, dr = rstd (dn - n mean(dn n)) + dtotal;
// dres = dr, dx = scale dr, dscale += dr x, dw += g n, dz = dout silu'(z) n w.  r is found again from
// x and res, since a rounded sum would leave its rounding in the parameters' gradients.
// Rows of a group on their way: x, dout, res and dtotal, z.
template <int K, bool RES, bool GATE>
struct Ring {
    static constexpr int TENSORS = 2 + 2 * RES + GATE, STAGES = K == 1 ? 4 : K <= 4 ? 2 : 1;
    static constexpr int BYTES = STAGES * TENSORS * K * kThreads * 16;
};
__device__ __forceinline__ void copy_unit(uint4* to, const void* from, bool in)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to)),
                 "l"(from), "r"(in ? 16 : 0) : "memory");
}

template <typename T, int K, bool RES, bool GATE>
__global__ void __launch_bounds__(kThreads, K == 1 ? 2 : 1) norm_bwd_kernel(NormArgs a, int tpr)
{
    constexpr int V = Pack<T>::N;
    __shared__ float slots[2][kThreads / 32];
    const int lane = threadIdx.x & (tpr - 1), shift = 31 - __clz(tpr), per = kThreads >> shift;
    const int mine = threadIdx.x >> shift;
    const unsigned group = blockIdx.x * per + mine, groups = gridDim.x * per;
    const unsigned items = (unsigned)row_count(a) * a.H;
    // groups % H == 0 where the parameters are a head's own: a group's head is always the same
    const int p = a.heads > 1 ? (int)(group % a.H) * a.d : 0;
    float dw[K][V] = {}, ds[RES ? K : 1][V] = {};
    // one unit a thread: its parameters stay
    float w1[V], s1[V];
    auto params = [&](int e, float (&w)[V], float (&s)[V]) {
#pragma unroll
        for (int q = 0; q < V; ++q) {
            w[q] = 0.f;
            s[q] = a.scale || e >= a.d ? 0.f : 1.f;
        }
        if (e >= a.d) return;
        load_params<V>(w, a.w + p + e);
        if (RES && a.scale) load_params<V>(s, a.scale + p + e);
    };
    if (K == 1) params(lane * V, w1, s1);
    // the row and head that are loaded next
    unsigned t = group / (unsigned)a.H, h = group - t * a.H;
    const unsigned rows_on = groups / (unsigned)a.H, heads_on = groups - rows_on * a.H;
    // A thread's own units of the rows ahead, [stage][tensor][K][threads]: nobody else reads them, so
    // their arrival is all that is waited for.
    constexpr int TENSORS = Ring<K, RES, GATE>::TENSORS, STAGES = Ring<K, RES, GATE>::STAGES;
    extern __shared__ __align__(16) uint4 ring[];
    auto slot = [&](int stage, int tensor, int k) {
        return ring + ((stage * TENSORS + tensor) * K + k) * kThreads + threadIdx.x;
    };
    auto load = [&](unsigned item, int stage) {
        const size_t at = h * a.d, out = (size_t)item * a.d;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (lane + k * tpr) * V;
            const bool in = item < items && e < a.d;
            const size_t xe = in ? at + e : 0, oe = in ? out + e : 0, r = in ? t : 0;
            copy_unit(slot(stage, 0, k), (const T*)a.x + r * a.xs + xe, in);
            copy_unit(slot(stage, 1, k), (const T*)a.dout + oe, in);
            if (RES) copy_unit(slot(stage, 2, k), (const T*)a.res + r * a.rs + xe, in);
            if (RES && a.dtotal) copy_unit(slot(stage, 3, k), (const T*)a.dtotal + oe, in);
            if (GATE) copy_unit(slot(stage, TENSORS - 1, k), (const T*)a.z + r * a.zs + xe, in);
        }
        copies_commit();
        t += rows_on;
        h += heads_on;
        if (h >= (unsigned)a.H) { h -= a.H; ++t; }
    };
    int turn = 0, stage = 0;
    float ahead = group < items ? a.rstd[group] : 0.f;
    for (int k = 0; k < STAGES - 1; ++k) load(group + k * groups, k);
    // (every group of a block makes the same number of rounds: the sums may have block barriers)
    for (unsigned base = blockIdx.x * per; base < items; base += groups, turn ^= 1) {
        const unsigned item = base + mine;
        load(item + (STAGES - 1) * groups, (stage + STAGES - 1) % STAGES);
        copies_wait<STAGES - 1>();
        Pack<T> xr[K], tr[RES ? K : 1];
        const size_t out = (size_t)item * a.d;
        const bool in = item < items;
        const float rstd = ahead;
        ahead = item + groups < items ? a.rstd[item + groups] : 0.f;
        float n[K][V], dn[K][V], sum = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (lane + k * tpr) * V;
            float w[V], s[V], g[V], x[V];
            if (K > 1) params(e, w, s);
#pragma unroll
            for (int q = 0; q < V; ++q)
                if (K == 1) { w[q] = w1[q]; s[q] = s1[q]; }
            Pack<T> in_;
            xr[k].load((const T*)slot(stage, 0, k));
            xr[k].get(n[k]);
            if (RES) {
                float y[V];
                in_.load((const T*)slot(stage, 2, k));
                in_.get(y);
#pragma unroll
                for (int q = 0; q < V; ++q) n[k][q] = fmaf(s[q], n[k][q], y[q]);
            }
            in_.load((const T*)slot(stage, 1, k));
            in_.get(g);
            if (GATE) {
                in_.load((const T*)slot(stage, TENSORS - 1, k));
                in_.get(x);
            }
            float dz[V];
#pragma unroll
            for (int q = 0; q < V; ++q) {
                n[k][q] *= rstd;
                if (GATE) {
                    const float l = logistic(x[q]);
                    dz[q] = g[q] * l * fmaf(x[q], 1.f - l, 1.f) * n[k][q] * w[q];
                    g[q] *= x[q] * l;
                }
                dw[k][q] = fmaf(g[q], n[k][q], dw[k][q]);
                dn[k][q] = g[q] * w[q];
                sum = fmaf(dn[k][q], n[k][q], sum);
            }
            if (GATE && in && e < a.d) {
                in_.set(dz);
                in_.store((T*)a.dz + out + e);
            }
        }
        sum = group_sum(sum, tpr, slots[turn]) / (float)a.d;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int e = (lane + k * tpr) * V;
            if (!in || e >= a.d) continue;
            float dr[V];
#pragma unroll
            for (int q = 0; q < V; ++q) dr[q] = rstd * fmaf(-n[k][q], sum, dn[k][q]);
            Pack<T> o;
            if (RES) {
                float y[V], x[V];
                if (a.dtotal) tr[k].load((const T*)slot(stage, 3, k)); else tr[k].zero();
                tr[k].get(y);
                xr[k].get(x);
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    dr[q] += y[q];
                    ds[k][q] = fmaf(dr[q], x[q], ds[k][q]);
                }
                o.set(dr);
                o.store((T*)a.dres + out + e);
                if (!a.scale) continue;
                float w[V], s[V];
                if (K > 1) params(e, w, s);
#pragma unroll
                for (int q = 0; q < V; ++q) dr[q] *= K > 1 ? s[q] : s1[q];
            }
            o.set(dr);
            o.store((T*)a.dx + out + e);
        }
        stage = (stage + 1) % STAGES;
    }
    const int cols = RES && a.scale ? 2 * a.d : a.d;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int e = (lane + k * tpr) * V;
        if (e >= a.d) continue;
        float* to = a.part + (size_t)group * cols + e;
#pragma unroll
        for (int q = 0; q < V; q += 4) {
            *(float4*)(to + q) = make_float4(dw[k][q], dw[k][q + 1], dw[k][q + 2], dw[k][q + 3]);
            if (RES && a.scale)
                *(float4*)(to + a.d + q) = make_float4(ds[k][q], ds[k][q + 1], ds[k][q + 2], ds[k][q + 3]);
        }
    }
}

struct Plan { int tpr, K; };
// Threads of a group and 16-byte units of each: at most 2 forward and 1 backward, which holds more of
// each in registers; more where a row has more than 512 or 256 units.
Plan plan(const NormArgs& a, bool backward)
{
    const int units = a.d / (a.bf16 ? 8 : 4);
    int tpr = 1;
    while (tpr < kThreads && (backward ? 1 : 2) * tpr < units) tpr *= 2;
    const int need = (units + tpr - 1) / tpr;
    return {tpr, need <= 2 ? need : need <= 4 ? 4 : 8};
}

template <typename T>
cudaError_t fwd(const NormArgs& a, cudaStream_t s)
{
    const Plan p = plan(a, false);
    const int per = kThreads / p.tpr;
    const dim3 grid((unsigned)(((long long)a.T * a.H + per - 1) / per));
    constexpr int most = 32 / Pack<T>::N;  // (rows of 8192 elements)
    auto kernel = p.K == 1 ? norm_fwd_kernel<T, 1> : p.K == 2 ? norm_fwd_kernel<T, 2>
                : p.K == 4 ? norm_fwd_kernel<T, 4> : norm_fwd_kernel<T, most>;
    return tc::launch_after(kernel, grid, kThreads, 0, 0, false, s, a, p.tpr);
}
template <typename T, int K>
cudaError_t bwd_k(const NormArgs& a, const Plan& p, cudaStream_t s)
{
    const int blocks = norm_bwd_blocks(a), groups = blocks * (kThreads / p.tpr);
    auto launch = [&](auto res, auto gate) {
        auto kernel = norm_bwd_kernel<T, K, res, gate>;
        constexpr int bytes = Ring<K, res, gate>::BYTES;
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e != cudaSuccess) return e;
        return tc::launch_after(kernel, dim3((unsigned)blocks), kThreads, bytes, 0, false, s, a, p.tpr);
    };
    const std::true_type yes;
    const std::false_type no;
    const cudaError_t e = a.res ? (a.z ? launch(yes, yes) : launch(yes, no)) : (a.z ? launch(no, yes) : launch(no, no));
    if (e != cudaSuccess) return e;
    const bool two = a.res && a.scale;
    return launch_column_sums(a.part, two ? 2 * a.d : a.d, a.d, a.heads, a.heads, groups / a.heads, a.dw,
                              two ? a.dscale : nullptr, s);
}
template <typename T>
cudaError_t bwd(const NormArgs& a, cudaStream_t s)
{
    const Plan p = plan(a, true);
    return p.K == 1 ? bwd_k<T, 1>(a, p, s) : p.K == 2 ? bwd_k<T, 2>(a, p, s)
         : p.K == 4 ? bwd_k<T, 4>(a, p, s) : bwd_k<T, 32 / Pack<T>::N>(a, p, s);
}

}  // namespace

// Blocks of the backward, 2 an SM at most; whole groups for every head that has its own parameters.
int norm_bwd_blocks(const NormArgs& a)
{
    const int per = kThreads / plan(a, true).tpr;
    const long long all = ((long long)a.T * a.H + per - 1) / per;
    int unit = a.heads;  // blocks whose groups are a multiple of the heads
    while (unit % 2 == 0 && unit / 2 * per % a.heads == 0) unit /= 2;
    const long long blocks = all < 304 ? all : 304;
    return (int)((blocks + unit - 1) / unit * unit);
}
size_t norm_part_floats(const NormArgs& a)
{
    return (size_t)norm_bwd_blocks(a) * (kThreads / plan(a, true).tpr) * 2 * a.d;
}

cudaError_t launch_norm_fwd(const NormArgs& a, cudaStream_t s)
{
    return a.bf16 ? fwd<__nv_bfloat16>(a, s) : fwd<float>(a, s);
}
cudaError_t launch_norm_bwd(const NormArgs& a, cudaStream_t s)
{
    return a.bf16 ? bwd<__nv_bfloat16>(a, s) : bwd<float>(a, s);
}

}  // namespace flex
