// Gated delta rule token by token, in fp32: whole sequences forward and backward, and the
// single-token step.  Per sequence and head, with a_t = exp(g_t),
//   e_t = v_t - a_t S^T k_t,  S <- a_t S + beta_t k_t e_t^T,  out_t = scale S^T q_t.
//
// Every column S[:, j] of the state depends on no other column (e_t[j] needs only column j), and
// once e is known every row S[i, :] depends on no other row.  So a state is cut into lines
// (columns, or rows) of which a few lanes each hold 16 entries in registers, and no block waits
// for another.  The backward runs three such scans: columns in reverse for D^T k (D: the gradient
// of the state), then rows forward (dq, and S_{t-1} dv) and rows in reverse (D u), the two halves
// of one grid.  Sums over a line are a few shuffles; sums over lines never occur.
#include "flex_internal.h"
#include "packed.cuh"
#include "tc_util.cuh"

namespace flex {
namespace {

constexpr int kThreads = 128;

// One line per P lanes, 16 entries each: entry 4 i + e of lane p is element 4 (p + P i) + e, so a
// warp's 16-byte reads of a staged vector touch P consecutive pieces.
template <int D>
struct Lines {
    static constexpr int P = D / 16;
    static constexpr int N = kThreads / P;   // lines of a block
    static constexpr int TT = 1024 / D;      // tokens staged at a time
};

template <int P>
__device__ __forceinline__ float line_sum(float x)
{
#pragma unroll
    for (int m = 1; m < P; m *= 2) x += __shfl_xor_sync(0xffffffffu, x, m);
    return x;
}

__device__ __forceinline__ float dot16(const float (&s)[16], const float4 (&x)[4])
{
    float a = 0.f, b = 0.f, c = 0.f, d = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a = fmaf(s[4 * i], x[i].x, a);
        b = fmaf(s[4 * i + 1], x[i].y, b);
        c = fmaf(s[4 * i + 2], x[i].z, c);
        d = fmaf(s[4 * i + 3], x[i].w, d);
    }
    return (a + b) + (c + d);
}
// s = a s + w x
__device__ __forceinline__ void axpy16(float (&s)[16], float a, float w, const float4 (&x)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        s[4 * i] = fmaf(w, x[i].x, a * s[4 * i]);
        s[4 * i + 1] = fmaf(w, x[i].y, a * s[4 * i + 1]);
        s[4 * i + 2] = fmaf(w, x[i].z, a * s[4 * i + 2]);
        s[4 * i + 3] = fmaf(w, x[i].w, a * s[4 * i + 3]);
    }
}
template <int P>
__device__ __forceinline__ void read16(float4 (&x)[4], const float* vec, int p)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = *(const float4*)(vec + 4 * (p + P * i));
}

// A tile of tokens in shared memory: up to three vectors of D elements and two values per line
// for every token, and the token's a and beta.
template <int D>
struct Tile {
    float vec[3][Lines<D>::TT][D];
    float line[2][Lines<D>::TT][Lines<D>::N];
    float a[Lines<D>::TT], beta[Lines<D>::TT];
};

// A vector operand: rows of D elements at base + t * stride, times `mul`, times beta_t if asked.
struct Rows {
    const void* base;
    long long stride;
    float mul;
    bool f32, by_beta;
};

// The loads of one tile, held in registers while the tile before it is worked on.
template <typename T, int D, int NV, int NL>
struct Fetch {
    static constexpr int TT = Lines<D>::TT, LN = Lines<D>::N;
    static constexpr int LP = (TT * LN + kThreads - 1) / kThreads;
    float4 v[NV][2];
    float l[NL][LP];
    float a, beta;
    float vb[2];

    // Tokens t0 .. t0 + TT - 1 of which those in [lo, hi) exist; the others read as zero (and
    // are not worked on).
    __device__ __forceinline__ void load(const Rows (&rows)[NV], const Rows (&line)[NL], int line0,
                                         const T* g, const T* beta_p, int H, int h, int t0, int lo,
                                         int hi, int tid)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 4 * (tid + kThreads * i), t = t0 + e / D, c = e % D;
            const bool in = t >= lo && t < hi;
            vb[i] = 0.f;
            if (in) vb[i] = to_f32(beta_p[(size_t)t * H + h]);
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                v[n][i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (!in) continue;
                if (rows[n].f32)
                    v[n][i] = load4((const float*)rows[n].base + t * rows[n].stride + c);
                else
                    v[n][i] = load4((const T*)rows[n].base + t * rows[n].stride + c);
            }
        }
#pragma unroll
        for (int i = 0; i < LP; ++i) {
            const int e = tid + kThreads * i, t = t0 + e / LN, c = line0 + e % LN;
            const bool in = e < TT * LN && t >= lo && t < hi;
#pragma unroll
            for (int n = 0; n < NL; ++n)
                l[n][i] = in ? to_f32(((const T*)line[n].base)[t * line[n].stride + c]) : 0.f;
        }
        if (tid < TT) {
            const int t = t0 + tid;
            const bool in = t >= lo && t < hi;
            a = in ? expf(to_f32(g[(size_t)t * H + h])) : 0.f;
            beta = in ? to_f32(beta_p[(size_t)t * H + h]) : 0.f;
        }
    }
    __device__ __forceinline__ void put(Tile<D>& s, const Rows (&rows)[NV], const Rows (&line)[NL],
                                        int tid) const
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int e = 4 * (tid + kThreads * i);
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const float m = rows[n].by_beta ? rows[n].mul * vb[i] : rows[n].mul;
                float4 x = v[n][i];
                x.x *= m; x.y *= m; x.z *= m; x.w *= m;
                *(float4*)(&s.vec[n][0][0] + e) = x;
            }
        }
#pragma unroll
        for (int i = 0; i < LP; ++i) {
            const int e = tid + kThreads * i;
            if (e < TT * LN) {
#pragma unroll
                for (int n = 0; n < NL; ++n) (&s.line[n][0][0])[e] = l[n][i] * line[n].mul;
            }
        }
        if (tid < TT) {
            s.a[tid] = a;
            s.beta[tid] = beta;
        }
    }
};

// Runs `step(tile, j, t)` over the rows [lo, hi) of a sequence, forward or in reverse, the next
// tile's loads in flight behind the current one's work.
template <typename T, int D, int NV, int NL, bool REV, typename Step>
__device__ __forceinline__ void scan(Tile<D>* tiles, const Rows (&rows)[NV], const Rows (&line)[NL],
                                     int line0, const T* g, const T* beta, int H, int h, int lo,
                                     int hi, Step step)
{
    constexpr int TT = Lines<D>::TT;
    const int tid = threadIdx.x, nt = (hi - lo + TT - 1) / TT;
    Fetch<T, D, NV, NL> f;
    auto start = [&](int i) { return REV ? hi - (i + 1) * TT : lo + i * TT; };
    if (nt > 0) {
        f.load(rows, line, line0, g, beta, H, h, start(0), lo, hi, tid);
        f.put(tiles[0], rows, line, tid);
    }
    __syncthreads();
    for (int i = 0; i < nt; ++i) {
        const int t0 = start(i);
        if (i + 1 < nt) f.load(rows, line, line0, g, beta, H, h, start(i + 1), lo, hi, tid);
        const Tile<D>& s = tiles[i & 1];
        if (REV) {
            for (int j = TT - 1; j >= 0 && t0 + j >= lo; --j) step(s, j, t0 + j);
        } else {
            for (int j = 0; j < TT && t0 + j < hi; ++j) step(s, j, t0 + j);
        }
        if (i + 1 < nt) f.put(tiles[(i + 1) & 1], rows, line, tid);
        __syncthreads();
    }
}

struct ScanArgs {
    Packed p;
    const void *q, *k, *v, *g, *beta, *dout;
    const int* cu;
    float scale;
    const float* S0;
    float* S1;
    void* out;
    float *e, *du, *dqh, *rh, *wh;  // [T][H][d]
};

// Which line block, head and sequence this block works on (line blocks of a head side by side).
template <int D>
__device__ __forceinline__ void place(const Packed& p, int b, int& line0, int& h, int& s)
{
    constexpr int LB = D / Lines<D>::N;
    line0 = (b % LB) * Lines<D>::N;
    h = (b / LB) % p.H;
    s = b / LB / p.H;
}

// Forward, one column per P lanes.  e (NULL or [T][H][d] fp32) receives v - a S^T k.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) delta_fwd_kernel(ScanArgs x)
{
    using L = Lines<D>;
    __shared__ Tile<D> tiles[2];
    const Packed& pk = x.p;
    int col0, h, s, lo, hi;
    place<D>(pk, blockIdx.x, col0, h, s);
    seq_rows(x.cu, s, pk.T, lo, hi);
    const int tid = threadIdx.x, p = tid % L::P, cl = tid / L::P, col = col0 + cl;
    const int H = pk.H, hk = h / (H / pk.Hk);
    float S[16];
    const size_t at = ((size_t)s * H + h) * D * D;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int r = 4 * (p + L::P * (i / 4)) + i % 4;
        S[i] = x.S0 ? x.S0[at + (size_t)r * D + col] : 0.f;
    }
    const Rows rows[2] = {{(const T*)x.k + hk * D, pk.ks, 1.f, false, false},
                          {(const T*)x.q + hk * D, pk.qs, x.scale, false, false}};
    const Rows line[1] = {{(const T*)x.v + h * D, pk.vs, 1.f, false, false}};
    T* out = (T*)x.out + h * D + col;
    float* e_out = x.e ? x.e + h * D + col : nullptr;
    const long long os = (long long)H * D;
    scan<T, D, 2, 1, false>(tiles, rows, line, col0, (const T*)x.g, (const T*)x.beta, H, h, lo, hi,
                            [&](const Tile<D>& tile, int j, int t) {
        float4 k[4], q[4];
        read16<L::P>(k, tile.vec[0][j], p);
        read16<L::P>(q, tile.vec[1][j], p);
        const float a = tile.a[j];
        const float e = tile.line[0][j][cl] - a * line_sum<L::P>(dot16(S, k));
        axpy16(S, a, tile.beta[j] * e, k);
        const float o = line_sum<L::P>(dot16(S, q));
        if (p == 0) {
            from_f32(out[t * os], o);
            if (e_out) e_out[t * os] = e;
        }
    });
    if (x.S1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = 4 * (p + L::P * (i / 4)) + i % 4;
            x.S1[at + (size_t)r * D + col] = S[i];
        }
    }
}

// Backward, first scan: columns of D in reverse; du_t = D_t^T k_t, D <- a (D - k dv^T).
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) delta_bwd_cols_kernel(ScanArgs x)
{
    using L = Lines<D>;
    __shared__ Tile<D> tiles[2];
    const Packed& pk = x.p;
    int col0, h, s, lo, hi;
    place<D>(pk, blockIdx.x, col0, h, s);
    seq_rows(x.cu, s, pk.T, lo, hi);
    const int tid = threadIdx.x, p = tid % L::P, cl = tid / L::P;
    const int H = pk.H, hk = h / (H / pk.Hk);
    const long long os = (long long)H * D;
    float S[16] = {};
    const Rows rows[2] = {{(const T*)x.k + hk * D, pk.ks, 1.f, false, false},
                          {(const T*)x.q + hk * D, pk.qs, x.scale, false, false}};
    const Rows line[1] = {{(const T*)x.dout + h * D, os, 1.f, false, false}};
    float* du_out = x.du + h * D + col0 + cl;
    scan<T, D, 2, 1, true>(tiles, rows, line, col0, (const T*)x.g, (const T*)x.beta, H, h, lo, hi,
                           [&](const Tile<D>& tile, int j, int t) {
        float4 k[4], q[4];
        read16<L::P>(k, tile.vec[0][j], p);
        read16<L::P>(q, tile.vec[1][j], p);
        axpy16(S, 1.f, tile.line[0][j][cl], q);
        const float du = line_sum<L::P>(dot16(S, k)), a = tile.a[j];
        axpy16(S, a, -a * tile.beta[j] * du, k);
        if (p == 0) du_out[t * os] = du;
    });
}

// Backward, the row scans: even blocks rows of S forward (dq = scale S dout, r = a S_{t-1} dv),
// odd blocks rows of D in reverse (w = D u, u = beta e).
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) delta_bwd_rows_kernel(ScanArgs x)
{
    using L = Lines<D>;
    __shared__ Tile<D> tiles[2];
    tc::grid_dep_wait();  // du
    const Packed& pk = x.p;
    int row0, h, s, lo, hi;
    place<D>(pk, blockIdx.x / 2, row0, h, s);
    seq_rows(x.cu, s, pk.T, lo, hi);
    const int tid = threadIdx.x, p = tid % L::P, rl = tid / L::P;
    const int H = pk.H, hk = h / (H / pk.Hk);
    const long long os = (long long)H * D;
    float S[16] = {};
    const Rows rows[3] = {{x.e + h * D, os, 1.f, true, true},
                          {x.du + h * D, os, 1.f, true, true},
                          {(const T*)x.dout + h * D, os, x.scale, false, false}};
    const Rows line[2] = {{(const T*)x.k + hk * D, pk.ks, 1.f, false, false},
                          {(const T*)x.q + hk * D, pk.qs, 1.f, false, false}};
    const size_t out0 = h * D + row0 + rl;
    if (blockIdx.x % 2 == 0) {
        scan<T, D, 3, 2, false>(tiles, rows, line, row0, (const T*)x.g, (const T*)x.beta, H, h, lo,
                                hi, [&](const Tile<D>& tile, int j, int t) {
            float4 u[4], dv[4], dO[4];
            read16<L::P>(u, tile.vec[0][j], p);
            read16<L::P>(dv, tile.vec[1][j], p);
            read16<L::P>(dO, tile.vec[2][j], p);
            const float a = tile.a[j];
            const float r = a * line_sum<L::P>(dot16(S, dv));
            axpy16(S, a, tile.line[0][j][rl], u);
            const float dq = line_sum<L::P>(dot16(S, dO));
            if (p == 0) {
                x.rh[out0 + t * os] = r;
                x.dqh[out0 + t * os] = dq;
            }
        });
    } else {
        scan<T, D, 3, 2, true>(tiles, rows, line, row0, (const T*)x.g, (const T*)x.beta, H, h, lo,
                               hi, [&](const Tile<D>& tile, int j, int t) {
            float4 u[4], dv[4], dO[4];
            read16<L::P>(u, tile.vec[0][j], p);
            read16<L::P>(dv, tile.vec[1][j], p);
            read16<L::P>(dO, tile.vec[2][j], p);
            const float a = tile.a[j];
            axpy16(S, 1.f, tile.line[1][j][rl], dO);
            const float w = line_sum<L::P>(dot16(S, u));
            axpy16(S, a, -a * tile.line[0][j][rl], dv);
            if (p == 0) x.wh[out0 + t * os] = w;
        });
    }
}

struct FinishArgs {
    Packed p;
    const void *q, *k, *beta;
    const int* cu;
    const float *e, *du, *dqh, *rh, *wh;
    void *dq, *dk, *dv, *dbeta, *dg;
    float* dG;  // [H][T]
};

// Row by row: dq and dk summed over the heads of a key head, dv = beta du, dbeta = e . du, and
// the gradient of the summed log decay, dG = q.dq - k.r - k.w (q_t and the reading k_t come with
// exp(+G_t), the writing k_t with exp(-G_t)).  One warp per (row, key head), D / 32 elements a lane.
template <typename T, int D>
__global__ void __launch_bounds__(128) delta_bwd_finish_kernel(FinishArgs x)
{
    tc::grid_dep_wait();
    const Packed& pk = x.p;
    const int lane = threadIdx.x & 31;
    const long long item = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    const int t = (int)(item / pk.Hk), hk = (int)(item % pk.Hk), G = pk.H / pk.Hk;
    const int lo = min(max(__ldg(x.cu), 0), pk.T), hi = min(__ldg(x.cu + pk.n), pk.T);
    if (t < lo || t >= hi) return;  // a row of no sequence: left as it was
    constexpr int E = D / 32;
    float q[E], k[E], dq[E] = {}, dk[E] = {};
#pragma unroll
    for (int i = 0; i < E; ++i) {
        q[i] = to_f32(((const T*)x.q)[t * pk.qs + hk * D + lane + 32 * i]);
        k[i] = to_f32(((const T*)x.k)[t * pk.ks + hk * D + lane + 32 * i]);
    }
    for (int h = hk * G; h < (hk + 1) * G; ++h) {
        const size_t at = ((size_t)t * pk.H + h) * D + lane;
        const float beta = to_f32(((const T*)x.beta)[(size_t)t * pk.H + h]);
        float sg = 0.f, sb = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const float a = x.dqh[at + 32 * i], r = x.rh[at + 32 * i], w = x.wh[at + 32 * i];
            const float du = x.du[at + 32 * i];
            dq[i] += a;
            dk[i] += w - r;
            sg += q[i] * a - k[i] * (r + w);
            sb += x.e[at + 32 * i] * du;
            from_f32(((T*)x.dv)[at + 32 * i], beta * du);
        }
        sg = line_sum<32>(sg);
        sb = line_sum<32>(sb);
        if (lane == 0) {
            from_f32(((T*)x.dbeta)[(size_t)t * pk.H + h], sb);
            x.dG[(size_t)h * pk.T + t] = sg;
        }
    }
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const size_t at = ((size_t)t * pk.Hk + hk) * D + lane + 32 * i;
        from_f32(((T*)x.dq)[at], dq[i]);
        from_f32(((T*)x.dk)[at], dk[i]);
    }
}

// dg_t = the sum of dG from t to the end of t's sequence.  The terms nearly cancel over a long
// sequence, so they are added up in 64 bits.
template <typename T>
__global__ void __launch_bounds__(256) delta_bwd_gate_kernel(FinishArgs x)
{
    tc::grid_dep_wait();
    __shared__ double part[8];
    const Packed& pk = x.p;
    const int h = blockIdx.x % pk.H, s = blockIdx.x / pk.H, tid = threadIdx.x, lane = tid & 31;
    int lo, hi;
    seq_rows(x.cu, s, pk.T, lo, hi);
    const float* dG = x.dG + (size_t)h * pk.T;
    double behind = 0.;
    for (int end = hi; end > lo; end -= 256) {
        const int t = end - 1 - tid;
        double v = t >= lo ? (double)dG[t] : 0.;
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const double o = __shfl_up_sync(0xffffffffu, v, m);
            if (lane >= m) v += o;
        }
        if (lane == 31) part[tid >> 5] = v;
        __syncthreads();
        double before = behind;
        for (int w = 0; w < (tid >> 5); ++w) before += part[w];
        for (int w = 0; w < 8; ++w) behind += part[w];
        if (t >= lo) from_f32(((T*)x.dg)[(size_t)t * pk.H + h], (float)(before + v));
        __syncthreads();
    }
}

// One token of a sequence: block (i, h) holds the state S [D][D] in registers, a float4 of
// columns and D / R rows (R apart) a thread, reads it once, and writes it once.  Both products
// with the old state, S^T k and S^T q, are taken in one pass over the registers and joined over
// the R row groups in shared memory; out = scale (a S^T q + (k.q) u) then needs no second pass.
// Bound by the state's bytes: all of a block's loads are in flight together.
template <typename T, int D, int NT>
__global__ void __launch_bounds__(NT) delta_decode_kernel(ScanArgs x)
{
    constexpr int Q = D / 4, R = NT / Q, N = D / R;
    __shared__ float4 part[2][R][Q];
    __shared__ float ks[D], qs[D];
    const Packed& pk = x.p;
    const int h = blockIdx.x % pk.H, s = blockIdx.x / pk.H, tid = threadIdx.x, c = tid % Q, r = tid / Q;
    const int H = pk.H, hk = h / (H / pk.Hk);
    float4* S = (float4*)(x.S1 + ((size_t)s * H + h) * D * D) + c;
    float4 st[N];
#pragma unroll
    for (int i = 0; i < N; ++i) st[i] = S[(size_t)(r + R * i) * Q];
    if (tid < D) {
        ks[tid] = to_f32(((const T*)x.k)[s * pk.ks + hk * D + tid]);
        qs[tid] = to_f32(((const T*)x.q)[s * pk.qs + hk * D + tid]);
    }
    const float a = expf(to_f32(((const T*)x.g)[(size_t)s * H + h]));
    const float beta = to_f32(((const T*)x.beta)[(size_t)s * H + h]);
    const float4 v = load4((const T*)x.v + s * pk.vs + h * D + 4 * c);
    __syncthreads();
    float4 sk = make_float4(0.f, 0.f, 0.f, 0.f), sq = sk;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float k = ks[r + R * i], q = qs[r + R * i];
        sk.x = fmaf(st[i].x, k, sk.x); sk.y = fmaf(st[i].y, k, sk.y);
        sk.z = fmaf(st[i].z, k, sk.z); sk.w = fmaf(st[i].w, k, sk.w);
        sq.x = fmaf(st[i].x, q, sq.x); sq.y = fmaf(st[i].y, q, sq.y);
        sq.z = fmaf(st[i].z, q, sq.z); sq.w = fmaf(st[i].w, q, sq.w);
    }
    part[0][r][c] = sk;
    part[1][r][c] = sq;
    float kq = 0.f;
    for (int i = tid & 31; i < D; i += 32) kq += ks[i] * qs[i];
    kq = line_sum<32>(kq);
    __syncthreads();
    sk = make_float4(0.f, 0.f, 0.f, 0.f);
    sq = sk;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const float4 y = part[0][i][c], z = part[1][i][c];
        sk.x += y.x; sk.y += y.y; sk.z += y.z; sk.w += y.w;
        sq.x += z.x; sq.y += z.y; sq.z += z.z; sq.w += z.w;
    }
    const float4 u = make_float4(beta * (v.x - a * sk.x), beta * (v.y - a * sk.y),
                                 beta * (v.z - a * sk.z), beta * (v.w - a * sk.w));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float k = ks[r + R * i];
        S[(size_t)(r + R * i) * Q] = make_float4(fmaf(k, u.x, a * st[i].x), fmaf(k, u.y, a * st[i].y),
                                                 fmaf(k, u.z, a * st[i].z), fmaf(k, u.w, a * st[i].w));
    }
    if (r == 0)
        store4((T*)x.out + ((size_t)s * H + h) * D + 4 * c,
               make_float4(x.scale * fmaf(kq, u.x, a * sq.x), x.scale * fmaf(kq, u.y, a * sq.y),
                           x.scale * fmaf(kq, u.z, a * sq.z), x.scale * fmaf(kq, u.w, a * sq.w)));
}

template <int D>
long long scan_blocks(const Packed& p) { return (long long)p.n * p.H * (D / Lines<D>::N); }

template <typename T, int D>
cudaError_t fwd(const ScanArgs& x, cudaStream_t s)
{
    return tc::launch_after(delta_fwd_kernel<T, D>, dim3((unsigned)scan_blocks<D>(x.p)), kThreads, 0,
                            0, false, s, x);
}

template <typename T, int D>
cudaError_t bwd(const ScanArgs& x, const FinishArgs& f, cudaStream_t s)
{
    const Packed& p = x.p;
    const unsigned blocks = (unsigned)scan_blocks<D>(p);
    cudaError_t e = tc::launch_after(delta_bwd_cols_kernel<T, D>, dim3(blocks), kThreads, 0, 0,
                                     false, s, x);
    if (e == cudaSuccess)
        e = tc::launch_after(delta_bwd_rows_kernel<T, D>, dim3(2 * blocks), kThreads, 0, 0, true, s, x);
    const long long items = (long long)p.T * p.Hk;
    if (e == cudaSuccess)
        e = tc::launch_after(delta_bwd_finish_kernel<T, D>, dim3((unsigned)((items + 3) / 4)), 128, 0,
                             0, true, s, f);
    if (e == cudaSuccess)
        e = tc::launch_after(delta_bwd_gate_kernel<T>, dim3((unsigned)(p.n * p.H)), 256, 0, 0, true,
                             s, f);
    return e;
}

template <typename T>
cudaError_t decode(const ScanArgs& x, cudaStream_t s)
{
    const dim3 grid((unsigned)((long long)x.p.n * x.p.H));
    if (x.p.d == 64)
        return tc::launch_after(delta_decode_kernel<T, 64, 128>, grid, 128, 0, 0, false, s, x);
    return tc::launch_after(delta_decode_kernel<T, 128, 256>, grid, 256, 0, 0, false, s, x);
}

}  // namespace

size_t delta_scan_save_floats(const Packed& p) { return (size_t)p.T * p.H * p.d; }
// du, dq, r, w per head, and dG
size_t delta_scan_ws_floats(const Packed& p) { return 4 * delta_scan_save_floats(p) + (size_t)p.T * p.H; }

cudaError_t launch_delta_scan_fwd(const Packed& p, const void* q, const void* k, const void* v,
                                  const void* g, const void* beta, const int* cu, float scale,
                                  const float* S0, float* S1, void* out, float* e, cudaStream_t s)
{
    ScanArgs x = {};
    x.p = p;
    x.q = q; x.k = k; x.v = v; x.g = g; x.beta = beta;
    x.cu = cu; x.scale = scale; x.S0 = S0; x.S1 = S1; x.out = out; x.e = e;
    if (p.bf16) return p.d == 64 ? fwd<__nv_bfloat16, 64>(x, s) : fwd<__nv_bfloat16, 128>(x, s);
    return p.d == 64 ? fwd<float, 64>(x, s) : fwd<float, 128>(x, s);
}

cudaError_t launch_delta_scan_bwd(const Packed& p, const void* q, const void* k, const void* g,
                                  const void* beta, const int* cu, float scale, const void* dout,
                                  const float* e, void* dq, void* dk, void* dv, void* dg,
                                  void* dbeta, float* scratch, cudaStream_t s)
{
    const size_t n = delta_scan_save_floats(p);
    ScanArgs x = {};
    x.p = p;
    x.q = q; x.k = k; x.g = g; x.beta = beta; x.dout = dout;
    x.cu = cu; x.scale = scale; x.e = const_cast<float*>(e);
    x.du = scratch; x.dqh = scratch + n; x.rh = scratch + 2 * n; x.wh = scratch + 3 * n;
    FinishArgs f = {};
    f.p = p;
    f.q = q; f.k = k; f.beta = beta; f.cu = cu;
    f.e = e; f.du = x.du; f.dqh = x.dqh; f.rh = x.rh; f.wh = x.wh;
    f.dq = dq; f.dk = dk; f.dv = dv; f.dbeta = dbeta; f.dg = dg;
    f.dG = scratch + 4 * n;
    if (p.bf16) return p.d == 64 ? bwd<__nv_bfloat16, 64>(x, f, s) : bwd<__nv_bfloat16, 128>(x, f, s);
    return p.d == 64 ? bwd<float, 64>(x, f, s) : bwd<float, 128>(x, f, s);
}

cudaError_t launch_delta_decode(const Packed& p, const void* q, const void* k, const void* v,
                                const void* g, const void* beta, float scale, float* S, void* out,
                                cudaStream_t s)
{
    ScanArgs x = {};
    x.p = p;
    x.q = q; x.k = k; x.v = v; x.g = g; x.beta = beta;
    x.scale = scale; x.S1 = S; x.out = out;
    return p.bf16 ? decode<__nv_bfloat16>(x, s) : decode<float>(x, s);
}

}  // namespace flex
