// Softmax attention over packed sequences in fp32 arithmetic, and the join of partial results
// over ranges of keys.  out_i = sum_j softmax_j(scale q_i . k_j) v_j over the keys that row i
// sees; one pass over the keys with the running maximum and sum of every row.
//
// The G = H / Hk heads that share a key head are rows of one tile (row = token * G + head), so
// their keys and values are read once, and one token of a sequence fills G rows.  Where the
// tiles are too few for the SMs, the keys are cut into ranges of which each block takes one;
// ranges leave their rows' output and log sum, which a second kernel joins.
#include "flex_internal.h"
#include "packed.cuh"
#include "softattn.cuh"
#include "tc_util.cuh"

namespace flex {
namespace {

constexpr int kRows = 64, kKeys = 64, kThreads = 256;

// fp32: tiles of 64 rows x 64 keys, 256 threads.  A thread holds 4 x 4 scores (rows 4 ty ..,
// keys tx, tx + 16, ..) and 4 x D / 16 outputs; each 16-byte shared read feeds 8 (scores) to
// 10 (outputs) FMAs.  Row pads of 4 floats keep the reads of 16 keys apart by banks.  V's loads are
// in flight behind the scores, the next K's behind the outputs.
template <int D>
struct SimtSmem {
    float q[kRows][D + 4];
    float kv[kKeys][D + 4];  // k, then v
    float p[kRows][kKeys + 4];
};

template <int D>
__global__ void __launch_bounds__(kThreads) softattn_simt_kernel(AttnArgs x)
{
    extern __shared__ __align__(16) char raw[];
    SimtSmem<D>& sm = *reinterpret_cast<SimtSmem<D>*>(raw);
    const Packed& pk = x.p;
    const int G = pk.H / pk.Hk, tpt = kRows / G;  // tokens of a tile
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int hk = blockIdx.x % pk.Hk, split = blockIdx.x / pk.Hk;
    int s, block, qlo, qhi, klo, khi;
    if (!find_tile(x, tpt, (int)(blockIdx.z * gridDim.y + blockIdx.y), s, block, qlo, qhi)) return;
    seq_rows(x.cu_k, s, pk.Tk, klo, khi);
    const int t0 = block * tpt, nt = min(tpt, qhi - qlo - t0);  // tokens of this tile
    const int lk = khi - klo, shift = lk - (qhi - qlo);
    int first, last;  // blocks of keys
    key_range(x, kKeys, lk, t0 + nt - 1 + shift, split, first, last);

    for (int e = tid; e < kRows * D / 4; e += kThreads) {
        const int r = e / (D / 4), c = e % (D / 4) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < nt * G)
            v = load4((const float*)x.q + (qlo + t0 + r / G) * pk.qs + (hk * G + r % G) * D + c);
        *(float4*)&sm.q[r][c] = v;
    }
    float o[4][D / 16] = {}, m[4], l[4] = {};
    int see[4];  // keys of the sequence that each row sees
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY;
        const int r = 4 * ty + i;
        see[i] = r >= nt * G ? 0 : x.causal ? min(lk, t0 + r / G + shift + 1) : lk;
    }
    float4 held[D / 16];  // this thread's part of the tile that comes next
    auto fetch = [&](const float* base, long long stride, int j0) {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            const int e = tid + kThreads * i, r = e / (D / 4), c = e % (D / 4) * 4;
            held[i] = j0 + r < lk ? load4(base + (klo + j0 + r) * stride + hk * D + c)
                                  : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    };
    auto put = [&] {
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            const int e = tid + kThreads * i;
            *(float4*)&sm.kv[e / (D / 4)][e % (D / 4) * 4] = held[i];
        }
    };
    if (first < last) fetch((const float*)x.k, pk.ks, first * kKeys);
    for (int b = first; b < last; ++b) {
        const int j0 = b * kKeys;
        __syncthreads();
        put();
        __syncthreads();
        fetch((const float*)x.v, pk.vs, j0);
        float sc[4][4] = {};
#pragma unroll 4
        for (int c = 0; c < D; c += 4) {
            float4 a[4], k[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = *(const float4*)&sm.q[4 * ty + i][c];
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = *(const float4*)&sm.kv[tx + 16 * i][c];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sc[i][j] = fmaf(a[i].w, k[j].w, fmaf(a[i].z, k[j].z, fmaf(a[i].y, k[j].y,
                                                                          fmaf(a[i].x, k[j].x, sc[i][j]))));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float top = m[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sc[i][j] = j0 + tx + 16 * j < see[i] ? sc[i][j] * x.scale : -INFINITY;
                top = fmaxf(top, sc[i][j]);
            }
#pragma unroll
            for (int w = 1; w < 16; w *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
            const float base = top == -INFINITY ? 0.f : top;  // a row that has seen no key yet
            const float keep = expf(m[i] - base);
            m[i] = top;
            l[i] *= keep;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = expf(sc[i][j] - base);
                l[i] += p;
                sm.p[4 * ty + i][tx + 16 * j] = p;
            }
#pragma unroll
            for (int c = 0; c < D / 16; ++c) o[i][c] *= keep;
        }
        __syncthreads();
        put();
        __syncthreads();
        if (b + 1 < last) fetch((const float*)x.k, pk.ks, j0 + kKeys);
#pragma unroll 2
        for (int j = 0; j < kKeys; j += 4) {
            float4 p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = *(const float4*)&sm.p[4 * ty + i][j];
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                float4 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = *(const float4*)&sm.kv[j + k][4 * tx + 64 * c];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float* y = &o[i][4 * c];
                    y[0] = fmaf(p[i].w, v[3].x, fmaf(p[i].z, v[2].x, fmaf(p[i].y, v[1].x, fmaf(p[i].x, v[0].x, y[0]))));
                    y[1] = fmaf(p[i].w, v[3].y, fmaf(p[i].z, v[2].y, fmaf(p[i].y, v[1].y, fmaf(p[i].x, v[0].y, y[1]))));
                    y[2] = fmaf(p[i].w, v[3].z, fmaf(p[i].z, v[2].z, fmaf(p[i].y, v[1].z, fmaf(p[i].x, v[0].z, y[2]))));
                    y[3] = fmaf(p[i].w, v[3].w, fmaf(p[i].z, v[2].w, fmaf(p[i].y, v[1].w, fmaf(p[i].x, v[0].w, y[3]))));
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int w = 1; w < 16; w *= 2) l[i] += __shfl_xor_sync(0xffffffffu, l[i], w);
        const int r = 4 * ty + i;
        if (r >= nt * G) continue;
        const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];  // (no key seen; a NaN sum goes on)
        const size_t row = (size_t)(qlo + t0 + r / G) * pk.H + hk * G + r % G;
        if (tx == 0) {
            const float z = m[i] + logf(l[i]);
            if (x.splits > 1) x.part_lse[(size_t)split * pk.T * pk.H + row] = z;
            else if (x.lse) x.lse[row] = z;
        }
#pragma unroll
        for (int c = 0; c < D / 64; ++c) {
            const float4 y = make_float4(o[i][4 * c] * inv, o[i][4 * c + 1] * inv,
                                         o[i][4 * c + 2] * inv, o[i][4 * c + 3] * inv);
            const int col = 4 * tx + 64 * c;
            if (x.splits > 1)
                store4(x.part + ((size_t)split * pk.T * pk.H + row) * D + col, y);
            else
                store4((float*)x.out + row * D + col, y);
        }
    }
}

// Joins the ranges of every row: out = sum_s exp(lse_s - lse) out_s, lse = log sum_s exp(lse_s),
// ranges in order.  A warp per row; a range that saw no key (lse -inf) has weight 0, one that met a
// NaN (lse NaN) makes the sum NaN.  Bound by the partial results' bytes (in L2: splitting is for few
// rows).
template <typename T>
__global__ void __launch_bounds__(128) softattn_join_kernel(AttnArgs x)
{
    tc::grid_dep_wait();
    const Packed& pk = x.p;
    const int lane = threadIdx.x & 31;
    const long long rows = (long long)pk.T * pk.H;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (row >= rows) return;
    const int t = (int)(row / pk.H);
    if (t < min(max(__ldg(x.cu_q), 0), pk.T) || t >= min(__ldg(x.cu_q + pk.n), pk.T)) return;
    float z = lane < x.splits ? x.part_lse[lane * rows + row] : -INFINITY;
    float top = z;
#pragma unroll
    for (int w = 1; w < 32; w *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, w));
    const float weight = z == -INFINITY ? 0.f : expf(z - top);
    float total = weight;
#pragma unroll
    for (int w = 1; w < 32; w *= 2) total += __shfl_xor_sync(0xffffffffu, total, w);
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int c = 4 * lane;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* part = x.part + row * pk.d + min(c, pk.d - 4);
#pragma unroll 8
    for (int s = 0; s < x.splits; ++s) {  // (every range has written its rows: 0 if it saw no key)
        const float w = __shfl_sync(0xffffffffu, weight, s) * inv;
        const float4 v = load4(part + s * rows * pk.d);
        y.x = fmaf(w, v.x, y.x); y.y = fmaf(w, v.y, y.y);
        y.z = fmaf(w, v.z, y.z); y.w = fmaf(w, v.w, y.w);
    }
    if (c < pk.d) store4((T*)x.out + row * pk.d + c, y);
    if (lane == 0 && x.lse) x.lse[row] = total == 0.f ? -INFINITY : top + logf(total);
}

template <int D>
cudaError_t launch_simt(const AttnArgs& x, cudaStream_t s)
{
    const Packed& p = x.p;
    const int smem = (int)sizeof(SimtSmem<D>);
    cudaError_t e = cudaFuncSetAttribute(softattn_simt_kernel<D>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    return tc::launch_after(softattn_simt_kernel<D>, softattn_grid(x, kRows / (p.H / p.Hk)), kThreads, smem, 0, false, s, x);
}

}  // namespace

int softattn_splits(const Packed& p)
{
    // Ranges of keys per tile.  Rows that fill their tiles are cut only as far as it takes to
    // give every SM a block: each range costs 4 (d + 1) bytes a row, written and read.  A few rows
    // (single tokens) cost next to nothing to join, and two blocks fit an SM; more of them pay their
    // start and end without filling it better (16 sequences of 8000 and 16 of 1777 keys, H16 Hk4
    // d128: 66 us for one block an SM, 61 for two, 64 for three, 68 for four, 73 for eight).  A range
    // is 256 keys (fp32: 128) of an average sequence or more; 32 ranges (the join's lanes) at most.
    // (152 SMs as a constant: the workspace's size must not go by the device that is current when it
    // is asked for, and the order of a row's sums not by where it runs.)
    const int G = p.H / p.Hk;
    const bool tc = tc_softattn_supported(p);
    const int rows = tc ? tc_softattn_rows(p) : kRows;
    const int tokens = rows == 256 ? 2 * (128 / G) : rows / G;  // of a block
    const long long blocks = (long long)block_slots(p.T, p.n, tokens) * p.Hk;
    const long long want = ((softattn_few(p) || !tc ? 2 : 1) * 152 + blocks - 1) / blocks;
    const long long most = (long long)p.Tk / p.n / (tc ? 256 : 128);
    const long long n = want < most ? want : most;
    return n < 1 ? 1 : n > 32 ? 32 : (int)n;
}

cudaError_t launch_softattn_simt(const AttnArgs& x, cudaStream_t s)
{
    return x.p.d == 64 ? launch_simt<64>(x, s) : launch_simt<128>(x, s);
}

cudaError_t launch_softattn_join(const AttnArgs& x, cudaStream_t s)
{
    const long long rows = (long long)x.p.T * x.p.H;
    const dim3 grid((unsigned)((rows + 3) / 4));
    return x.p.bf16 ? tc::launch_after(softattn_join_kernel<__nv_bfloat16>, grid, 128, 0, 0, true, s, x)
                    : tc::launch_after(softattn_join_kernel<float>, grid, 128, 0, 0, true, s, x);
}

}  // namespace flex
