// Short causal convolution over packed sequences, channel by channel:
//   pre_t = b + sum_j w_j x_{t - (W - 1) + j},  out_t = silu(pre_t) or pre_t,
// rows ahead of a sequence's first being its state's (the last W - 1 rows of what came before) or 0.
//
// A thread walks a run of rows of 4 channels with the last rows in registers, so every row is read once
// but for the W - 1 ahead of each run; runs are cut from all rows alike, whatever the sequences.  Bound
// by DRAM: x read once and out written once, 32768 rows of 4096 channels (bf16) in 94 us, 5.7 TB/s; 16
// bytes of channels a thread took 127 registers and 177 us.
#include "flex_internal.h"
#include "layer.cuh"

namespace flex {
namespace {

// The sequence that row t lies in (t < cu[n]): the last that starts at or before it.
__device__ __forceinline__ int find_row(const int* cu, int n, int t)
{
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (__ldg(cu + mid) <= t) lo = mid; else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ int rows_end(const int* cu, int n, int T) { return min(max(__ldg(cu + n), 0), T); }

constexpr int kAhead = 8;  // rows whose loads are in flight together

struct Four {  // 4 channels' values as packed pairs
    uint64_t a, b;
    __device__ __forceinline__ void set(float4 v) { a = tc::f2_pack(v.x, v.y); b = tc::f2_pack(v.z, v.w); }
    __device__ __forceinline__ float4 get() const
    {
        float4 v;
        tc::f2_unpack(a, v.x, v.y);
        tc::f2_unpack(b, v.z, v.w);
        return v;
    }
    __device__ __forceinline__ void add(const Four& x, const Four& y)  // += x y
    {
        a = tc::f2_fma(x.a, y.a, a);
        b = tc::f2_fma(x.b, y.b, b);
    }
};
// 4 channels' parameters: w [D][W], fp32.
template <int W>
__device__ __forceinline__ void load_taps(Four (&w)[W], Four& bias, const ConvArgs& a, int c)
{
    float v[4 * W];
    load_params<4 * W>(v, a.w + (size_t)c * W);
    bias.set(a.bias ? *(const float4*)(a.bias + c) : make_float4(0.f, 0.f, 0.f, 0.f));
#pragma unroll
    for (int j = 0; j < W; ++j) w[j].set(make_float4(v[j], v[W + j], v[2 * W + j], v[3 * W + j]));
}

template <typename T, int W>
__global__ void __launch_bounds__(128) conv_fwd_kernel(ConvArgs a, long long run_blocks)
{
    const int CQ = a.D / 4;
    const T* x = (const T*)a.x;
    if (blockIdx.x >= run_blocks) {  // the sequences' last rows
        const long long i = (blockIdx.x - run_blocks) * 128 + threadIdx.x;
        const long long row = i / CQ;
        const int c = (int)(i % CQ) * 4, s = (int)(row / (W - 1)), j = (int)(row % (W - 1));
        if (s >= a.n) return;
        int lo, hi;
        seq_rows(a.cu, s, a.T, lo, hi);
        const int t = hi - (W - 1) + j;
        Quad<T> v;
        v.zero();
        if (t >= lo) v.load(x + (long long)t * a.xs + c);
        else if (a.S0) v.load((const T*)a.S0 + ((long long)s * (W - 1) + (t - lo + W - 1)) * a.D + c);
        v.store((T*)a.S1 + row * a.D + c);
        return;
    }
    const long long i = blockIdx.x * 128LL + threadIdx.x;
    const int c = (int)(i % CQ) * 4;
    const int end = rows_end(a.cu, a.n, a.T);
    const long long first = i / CQ * a.run;
    if (first >= end) return;
    const int t0 = (int)first, t1 = min(end, t0 + a.run);
    int s = find_row(a.cu, a.n, t0), lo, hi;
    seq_rows(a.cu, s, a.T, lo, hi);
    Four w[W], b, win[W - 1];
    load_taps<W>(w, b, a, c);
    // the rows ahead of row t of sequence s
    auto before = [&](int t) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int u = t - (W - 1) + j;
            Quad<T> v;
            v.zero();
            if (u >= lo) v.load(x + (long long)u * a.xs + c);
            // (no row ahead of the state's first, whatever the offsets)
            else if (a.S0) v.load((const T*)a.S0 + ((long long)s * (W - 1) + max(u - lo + W - 1, 0)) * a.D + c);
            win[j].set(v.get());
        }
    };
    before(t0);
    const T* from = x + (long long)t0 * a.xs + c;
    T* to = (T*)a.out + (long long)t0 * a.D + c;
    auto step = [&](const Quad<T>& row, T* at) {
        Four v, p = b;
        v.set(row.get());
#pragma unroll
        for (int j = 0; j < W - 1; ++j) p.add(w[j], win[j]);
        p.add(w[W - 1], v);
        float4 y = p.get();
        if (a.silu) {
            y.x *= logistic(y.x); y.y *= logistic(y.y); y.z *= logistic(y.z); y.w *= logistic(y.w);
        }
        store4(at, y);
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) win[j] = win[j + 1];
        win[W - 2] = v;
    };
    for (int t = t0; t < t1; t += kAhead, from += kAhead * a.xs, to += (long long)kAhead * a.D) {
        Quad<T> rows[kAhead];
        if (t + kAhead <= min(t1, hi)) {  // one sequence's rows, as most are: nothing to look at
#pragma unroll
            for (int k = 0; k < kAhead; ++k) rows[k].load(from + k * a.xs);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) step(rows[k], to + (long long)k * a.D);
            continue;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (t + k < t1) rows[k].load(from + k * a.xs);
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (t + k >= t1) break;
            if (t + k >= hi && s + 1 < a.n) {  // the next sequence that has rows
                do {
                    ++s;
                    seq_rows(a.cu, s, a.T, lo, hi);
                } while (t + k >= hi && s + 1 < a.n);
                before(t + k);
            }
            step(rows[k], to + (long long)k * a.D);
        }
    }
}

// Gradients: dpre_t = dout_t silu'(pre_t), dx_t = sum_j w_j dpre_{t + (W - 1) - j} within the
// sequence, dw_j = sum_t dpre_t x_{t - (W - 1) + j}, db = sum_t dpre_t.  A thread walks its run and the
// W - 1 rows behind it, whose dpre its last rows' dx wants; dw and db are summed over a block's 8 runs
// in their order, and over blocks by a kernel of their own.  12817 rows of 2048 channels: 48 us for 157 MB,
// 57% of the issue slots, 816 blocks of which 304 run at a time (52 with rows in registers; three blocks an
// SM spill: 80).
constexpr int kBack = 4;
// Batches of rows on their way, a thread's own: 64 KB a block.
template <typename T>
constexpr int kStages = 32 / (kBack * sizeof(T));

template <typename T, int W>
__global__ void __launch_bounds__(256, 2) conv_bwd_kernel(ConvArgs a)
{
    __shared__ float4 sums[8][W + 1][32];
    extern __shared__ __align__(16) unsigned char ring[];
    const int c = (blockIdx.y * 32 + threadIdx.x) * 4;
    const bool mine = c < a.D;
    const int end = rows_end(a.cu, a.n, a.T);
    const long long first = ((long long)blockIdx.x * 8 + threadIdx.y) * a.run;
    Four dw[W], db;
    db.a = db.b = 0;
#pragma unroll
    for (int j = 0; j < W; ++j) dw[j].a = dw[j].b = 0;
    if (mine && first < end) {
        const int t0 = (int)first, t1 = min(end, t0 + a.run), t2 = min(end, t1 + W - 1);
        int s = find_row(a.cu, a.n, t0), lo, hi;
        seq_rows(a.cu, s, a.T, lo, hi);
        Four w[W], b, win[W - 1], acc[W];
        load_taps<W>(w, b, a, c);
#pragma unroll
        for (int j = 0; j < W; ++j) acc[j].a = acc[j].b = 0;
        const T *x = (const T*)a.x + (long long)t0 * a.xs + c, *dout = (const T*)a.dout + (long long)t0 * a.D + c;
        T* dx = (T*)a.dx + (long long)(t0 - (W - 1)) * a.D + c;  // (the row that row t0 completes)
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            Quad<T> v;
            v.zero();
            if (t0 - (W - 1) + j >= lo) v.load(x + (long long)(j - (W - 1)) * a.xs);
            win[j].set(v.get());
        }
        // Row u's share in its own and the rows' ahead; `at` of these are of its sequence.
        auto add = [&](const Quad<T>& px, const Quad<T>& pd, bool own, int at) {
            Four v, p = b, dp;
            v.set(px.get());
#pragma unroll
            for (int j = 0; j < W - 1; ++j) p.add(w[j], win[j]);
            p.add(w[W - 1], v);
            float4 g = pd.get();
            if (a.silu) {
                const float4 q = p.get();
                const float4 l = make_float4(logistic(q.x), logistic(q.y), logistic(q.z), logistic(q.w));
                g.x *= l.x * fmaf(q.x, 1.f - l.x, 1.f);
                g.y *= l.y * fmaf(q.y, 1.f - l.y, 1.f);
                g.z *= l.z * fmaf(q.z, 1.f - l.z, 1.f);
                g.w *= l.w * fmaf(q.w, 1.f - l.w, 1.f);
            }
            dp.set(g);
            if (own) {
                Four one;
                one.a = one.b = tc::f2_pack(1.f, 1.f);
                db.add(dp, one);
#pragma unroll
                for (int j = 0; j < W - 1; ++j) dw[j].add(dp, win[j]);
                dw[W - 1].add(dp, v);
            }
#pragma unroll
            for (int j = 0; j < W; ++j)
                if (W - 1 - j <= at) acc[j].add(w[j], dp);
#pragma unroll
            for (int j = 0; j + 1 < W - 1; ++j) win[j] = win[j + 1];
            win[W - 2] = v;
        };
        auto next = [&]() {
#pragma unroll
            for (int j = 0; j + 1 < W; ++j) acc[j] = acc[j + 1];
            acc[W - 1].a = acc[W - 1].b = 0;
        };
        // row k of a stage's batch: x, and dout 256 quads on
        auto slot = [&](int stage, int k) {
            return (T*)ring + 4 * ((stage * kBack + k) * 512 + threadIdx.y * 32 + threadIdx.x);
        };
        auto fetch = [&](int t, int stage) {
#pragma unroll
            for (int k = 0; k < kBack; ++k) {
                const bool in = t + k < t2;
                const long long row = in ? t + k - t0 : 0;
                copy_quad(slot(stage, k), x + row * a.xs, in);
                copy_quad(slot(stage, k) + 1024, dout + row * a.D, in);
            }
            copies_commit();
        };
        int stage = 0;
        constexpr int STAGES = kStages<T>;
#pragma unroll
        for (int k = 0; k < STAGES - 1; ++k) fetch(t0 + k * kBack, k);
        for (int t = t0; t < t1 + W - 1; t += kBack, dx += (long long)kBack * a.D) {
            fetch(t + (STAGES - 1) * kBack, (stage + STAGES - 1) % STAGES);
            copies_wait<STAGES - 1>();
            Quad<T> px[kBack], pd[kBack];
#pragma unroll
            for (int k = 0; k < kBack; ++k) {
                px[k].load(slot(stage, k));
                pd[k].load(slot(stage, k) + 1024);
            }
            stage = (stage + 1) % STAGES;
            if (t >= t0 + W - 1 && t >= lo + W - 1 && t + kBack <= min(t1, hi)) {  // nothing to look at
#pragma unroll
                for (int k = 0; k < kBack; ++k) {
                    add(px[k], pd[k], true, W - 1);
                    store4(dx + (long long)k * a.D, acc[0].get());
                    next();
                }
                continue;
            }
#pragma unroll
            for (int k = 0; k < kBack; ++k) {
                const int u = t + k;
                if (u >= t1 + W - 1) break;
                if (u < t2) {
                    if (u >= hi && s + 1 < a.n) {
                        do {
                            ++s;
                            seq_rows(a.cu, s, a.T, lo, hi);
                        } while (u >= hi && s + 1 < a.n);
#pragma unroll
                        for (int j = 0; j < W - 1; ++j) win[j].a = win[j].b = 0;
                    }
                    add(px[k], pd[k], u < t1, u - lo);
                }
                // nothing more is added to this row's dx
                if (u - (W - 1) >= t0) store4(dx + (long long)k * a.D, acc[0].get());
                next();
            }
        }
    }
#pragma unroll
    for (int j = 0; j < W; ++j) sums[threadIdx.y][j][threadIdx.x] = dw[j].get();
    sums[threadIdx.y][W][threadIdx.x] = db.get();
    __syncthreads();
    if (threadIdx.y <= W && mine) {
        float4 v = sums[0][threadIdx.y][threadIdx.x];
#pragma unroll
        for (int k = 1; k < 8; ++k) {
            const float4 u = sums[k][threadIdx.y][threadIdx.x];
            v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
        // dw as [D][W], then db: columns of a matrix of one row a block
        float* to = a.part + (size_t)blockIdx.x * (W + 1) * a.D;
        const float f[4] = {v.x, v.y, v.z, v.w};
        const int j = threadIdx.y;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (j < W) to[(size_t)(c + q) * W + j] = f[q];
            else to[(size_t)a.D * W + c + q] = f[q];
        }
    }
}

// One row of every sequence, the state moved on by it.
template <typename T, int W>
__global__ void __launch_bounds__(128) conv_decode_kernel(ConvArgs a)
{
    constexpr int V = Pack<T>::N;
    const int CV = a.D / V;
    const long long i = blockIdx.x * 128LL + threadIdx.x;
    const long long s = i / CV;
    const int c = (int)(i % CV) * V;
    if (s >= a.n) return;
    T* state = (T*)a.S1 + s * (W - 1) * a.D + c;
    Pack<T> rows[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) rows[j].load(state + (long long)j * a.D);
    rows[W - 1].load((const T*)a.x + s * a.xs + c);
    float p[V];
#pragma unroll
    for (int k = 0; k < V; ++k) p[k] = a.bias ? a.bias[c + k] : 0.f;
#pragma unroll
    for (int j = 0; j < W; ++j) {
        float v[V];
        rows[j].get(v);
#pragma unroll
        for (int k = 0; k < V; ++k) p[k] = fmaf(a.w[(size_t)(c + k) * W + j], v[k], p[k]);
    }
    if (a.silu)
#pragma unroll
        for (int k = 0; k < V; ++k) p[k] *= logistic(p[k]);
    Pack<T> o;
    o.set(p);
    o.store((T*)a.out + s * a.D + c);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) rows[j + 1].store(state + (long long)j * a.D);
}

// Blocks of 32 columns.  Where some hundred rows are summed, as for the convolution and for norms of 2048
// elements, what costs is their loads' latency (5 to 8 us).  A norm of few elements leaves a row for each of
// its groups of threads, up to 77824 of them for d 8, all in one block's hands: its gradients for 20000 rows
// take 82 us, of 128 elements 30.
constexpr int kSlices = 32;
__global__ void __launch_bounds__(8 * kSlices) column_sums_kernel(const float* from, int cols, int split,
                                                                  int step, int count, float* to0, float* to1)
{
    __shared__ float4 sums[kSlices][8];
    tc::grid_dep_wait();
    const int c = (blockIdx.x * 8 + threadIdx.x) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (c < cols) {
#pragma unroll 8
        for (int k = threadIdx.y; k < count; k += kSlices) {
            const float4 u = *(const float4*)(from + (size_t)(blockIdx.y + (size_t)k * step) * cols + c);
            v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
    }
    sums[threadIdx.y][threadIdx.x] = v;
    __syncthreads();
    if (threadIdx.y || c >= cols) return;
#pragma unroll
    for (int k = 1; k < kSlices; ++k) {
        const float4 u = sums[k][threadIdx.x];
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    if (c < split) *(float4*)(to0 + (size_t)blockIdx.y * split + c) = v;
    else if (to1) *(float4*)(to1 + (size_t)blockIdx.y * (cols - split) + c - split) = v;
}

template <typename T, int W>
cudaError_t fwd(const ConvArgs& a, cudaStream_t s)
{
    const int CQ = a.D / 4;
    const long long blocks = ((long long)(a.T + a.run - 1) / a.run * CQ + 127) / 128;
    const long long more = a.S1 ? ((long long)a.n * (W - 1) * CQ + 127) / 128 : 0;
    return tc::launch_after(conv_fwd_kernel<T, W>, dim3((unsigned)(blocks + more)), 128, 0, 0, false, s, a,
                            blocks);
}
template <typename T, int W>
cudaError_t bwd(const ConvArgs& a, cudaStream_t s)
{
    const int rows = conv_bwd_blocks(a);
    constexpr int bytes = kStages<T> * kBack * 512 * 4 * sizeof(T);
    cudaError_t e = cudaFuncSetAttribute(conv_bwd_kernel<T, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    conv_bwd_kernel<T, W><<<dim3(rows, (a.D + 127) / 128), dim3(32, 8), bytes, s>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_column_sums(a.part, (W + 1) * a.D, W * a.D, 1, 1, rows, a.dw, a.dbias, s);
}
template <typename T, int W>
cudaError_t decode(const ConvArgs& a, cudaStream_t s)
{
    const long long items = (long long)a.n * (a.D / Pack<T>::N);
    return tc::launch_after(conv_decode_kernel<T, W>, dim3((unsigned)((items + 127) / 128)), 128, 0, 0, false,
                            s, a);
}

enum What { kFwd, kBwd, kDecode };
template <typename T, int W>
cudaError_t call(const ConvArgs& a, What what, cudaStream_t s)
{
    return what == kFwd ? fwd<T, W>(a, s) : what == kBwd ? bwd<T, W>(a, s) : decode<T, W>(a, s);
}
template <typename T>
cudaError_t call_w(const ConvArgs& a, What what, cudaStream_t s)
{
    return a.W == 2 ? call<T, 2>(a, what, s) : a.W == 3 ? call<T, 3>(a, what, s) : call<T, 4>(a, what, s);
}
cudaError_t call_t(const ConvArgs& a, What what, cudaStream_t s)
{
    return a.bf16 ? call_w<__nv_bfloat16>(a, what, s) : call_w<float>(a, what, s);
}

}  // namespace

cudaError_t launch_column_sums(const float* from, int cols, int split, int sums, int step, int count,
                               float* to0, float* to1, cudaStream_t s)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((cols + 31) / 32), (unsigned)sums);
    cfg.blockDim = dim3(8, kSlices);
    cfg.stream = s;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, column_sums_kernel, from, cols, split, step, count, to0, to1);
}

// Rows of a thread's run: long ones read fewer rows twice, short ones fill the SMs.
int conv_run(const ConvArgs& a)
{
    const long long lanes = a.D / 4, want = 152LL * 1024;
    int run = 32;
    while (run > 4 && (a.T + run - 1) / run * lanes < want) run /= 2;
    return run;
}
int conv_bwd_blocks(const ConvArgs& a) { return (a.T + 8 * a.run - 1) / (8 * a.run); }

cudaError_t launch_conv_fwd(const ConvArgs& a, cudaStream_t s) { return call_t(a, kFwd, s); }
cudaError_t launch_conv_bwd(const ConvArgs& a, cudaStream_t s) { return call_t(a, kBwd, s); }
cudaError_t launch_conv_decode(const ConvArgs& a, cudaStream_t s) { return call_t(a, kDecode, s); }

}  // namespace flex
