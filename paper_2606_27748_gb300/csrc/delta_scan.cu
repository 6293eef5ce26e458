// Gated delta rule in fp32: whole sequences forward and backward, and the single-token step.  Per
// sequence and head, with a_t = exp(g_t),
//   e_t = v_t - a_t S^T k_t,  S <- a_t S + beta_t k_t e_t^T,  out_t = scale S^T q_t.
//
// Every column S[:, j] of the state depends on no other column (e_t[j] needs only column j), and
// once e is known every row S[i, :] depends on no other row.  So a state is cut into lines
// (columns, or rows) of which a few lanes each hold 8 or 16 entries in registers, and no block waits
// for another.  The backward runs three such scans: columns in reverse for Y = D^T k (D: the
// gradient of the state), then rows forward (dq, and S_{t-1} dv) and rows in reverse (D u), the
// two halves of one grid.  Sums over a line are a few shuffles; sums over lines never occur.
//
// A column's next step needs the sum of its last one, so what bounds a scan is one warp's chain of
// product (90 cycles a token), shuffles (130) and update, and how many warps share a
// scheduler and the shared memory meanwhile.  Measured, H4 d64: forward, 1000 tokens, with 8 lanes
// to a line 181 us, with 4 208 (blocks of 32 lines; 137 in blocks of 16, see narrow()); reverse,
// 4 x 1000, with 4 lanes 142, with 8 156; 8 tokens at once with their mutual products (a triangular
// system), 4 lanes 222 us (890 instructions a warp for 8 tokens), 16 lanes 255 (bound by
// shared-memory reads).
#include "flex_internal.h"
#include "packed.cuh"
#include "tc_util.cuh"

namespace flex {
namespace {

constexpr int kNarrow = 16, kWide = 32;  // lines of a block (see narrow())
constexpr int kMark = 64;   // tokens between two marks of a sequence (see delta_bwd_gate_kernel)

template <int D>
struct Cfg {
    // lanes of a line: columns forward, columns in reverse, rows
    static constexpr int PF = D / 8, PB = D / 16, PR = D / 8;
    static constexpr int COL = 16, ROW = 1024 / D;  // tokens staged at a time
};

template <int P>
__device__ __forceinline__ float line_sum(float x)
{
#pragma unroll
    for (int m = 1; m < P; m *= 2) x += __shfl_xor_sync(0xffffffffu, x, m);
    return x;
}
// Two sums over a line at once: their shuffles run side by side.
template <int P>
__device__ __forceinline__ void line_sum2(float& x, float& y)
{
#pragma unroll
    for (int m = 1; m < P; m *= 2) {
        const float a = __shfl_xor_sync(0xffffffffu, x, m), b = __shfl_xor_sync(0xffffffffu, y, m);
        x += a;
        y += b;
    }
}

// Sums of 8 values over a line's lanes, each of which returns the one of value p / (P / 8): every
// step halves the values that a lane still adds up, 7 or 8 shuffles instead of 24 or 32.
template <int P>
__device__ __forceinline__ float line_sums8(float (&x)[8], int p)
{
#pragma unroll
    for (int m = P / 2, n = 4; n >= 1; m /= 2, n /= 2) {
        const bool up = p & m;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float give = up ? x[i] : x[i + n], keep = up ? x[i + n] : x[i];
            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, m);
        }
    }
    return P == 16 ? x[0] + __shfl_xor_sync(0xffffffffu, x[0], 1) : x[0];
}

// A lane's D / P entries of a line (elements 4 p + 0 .. 3 of every 4 P) as packed pairs.
template <int D, int P>
struct Vec {
    static constexpr int N = D / P / 2;
    uint64_t x[N];

    __device__ __forceinline__ void read(const float* vec, int p)
    {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const ulonglong2 y = *(const ulonglong2*)(vec + 4 * (P * i + p));
            x[2 * i] = y.x;
            x[2 * i + 1] = y.y;
        }
    }
    __device__ __forceinline__ float dot(const Vec& y) const
    {
        uint64_t a[N / 2];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) a[i] = tc::f2_fma(x[i + N / 2], y.x[i + N / 2], tc::f2_mul(x[i], y.x[i]));
        float c[N];
#pragma unroll
        for (int i = 0; i < N / 2; ++i) tc::f2_unpack(a[i], c[2 * i], c[2 * i + 1]);
#pragma unroll
        for (int m = 1; m < N; m *= 2)
#pragma unroll
            for (int i = 0; i + m < N; i += 2 * m) c[i] += c[i + m];
        return c[0];
    }
    __device__ __forceinline__ void add(float w, const Vec& y)  // += w y
    {
        const uint64_t ww = tc::f2_pack(w, w);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = tc::f2_fma(ww, y.x[i], x[i]);
    }
    __device__ __forceinline__ void scale(float a)
    {
        const uint64_t aa = tc::f2_pack(a, a);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = tc::f2_mul(aa, x[i]);
    }
};
template <int P>
__device__ __forceinline__ int element(int i, int p) { return 4 * (P * (i / 4) + p) + i % 4; }

// The tile of tokens that a column scan works on: k, q and the lines' values (v, or dout).
template <int D, int L>
struct ColTile {
    float k[Cfg<D>::COL][D], q[Cfg<D>::COL][D];
    float line[Cfg<D>::COL][L];
    float a[Cfg<D>::COL], beta[Cfg<D>::COL];
};

// Runs `step(tile, j, t)` over the rows [lo, hi) of a sequence, forward or in reverse; the next
// tile's loads are in flight behind the current one's work, and nothing is computed from them before
// that is done (an exponential of the gates ahead of it cost 50 of 480 cycles a token).  Steps are
// unrolled, and leave for the next one the sums that nothing waits for.
template <typename T, int D, int L, int P, bool REV, typename Step>
__device__ __forceinline__ void col_scan(ColTile<D, L>* tiles, const T* k, long long ks, const T* q,
                                         long long qs, const T* line, long long ls, const T* g,
                                         const T* beta, int H, int lo, int hi, Step step)
{
    constexpr int TT = Cfg<D>::COL, NT = L * P, LP = TT * L / NT, V4 = TT * D / 4 / NT;
    const int tid = threadIdx.x, nt = (hi - lo + TT - 1) / TT;
    float4 kr[V4], qr[V4];
    float lr[LP], ar = 0.f, br = 0.f;
    auto start = [&](int i) { return REV ? hi - (i + 1) * TT : lo + i * TT; };
    auto load = [&](int t0) {
#pragma unroll
        for (int i = 0; i < V4; ++i) {
            const int e = 4 * (tid + NT * i), t = t0 + e / D, c = e % D;
            const bool in = t >= lo && t < hi;
            kr[i] = in ? load4(k + t * ks + c) : make_float4(0.f, 0.f, 0.f, 0.f);
            qr[i] = in ? load4(q + t * qs + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int i = 0; i < LP; ++i) {
            const int e = tid + NT * i, t = t0 + e / L;
            lr[i] = t >= lo && t < hi ? to_f32(line[t * ls + e % L]) : 0.f;
        }
        if (tid < TT) {
            const int t = t0 + tid;
            const bool in = t >= lo && t < hi;
            ar = in ? to_f32(g[(size_t)t * H]) : 0.f;
            br = in ? to_f32(beta[(size_t)t * H]) : 0.f;
        }
    };
    auto put = [&](ColTile<D, L>& s) {
#pragma unroll
        for (int i = 0; i < V4; ++i) {
            *(float4*)(&s.k[0][0] + 4 * (tid + NT * i)) = kr[i];
            *(float4*)(&s.q[0][0] + 4 * (tid + NT * i)) = qr[i];
        }
#pragma unroll
        for (int i = 0; i < LP; ++i) (&s.line[0][0])[tid + NT * i] = lr[i];
        if (tid < TT) {
            s.a[tid] = expf(ar);  // (rows that do not exist are staged but not worked on)
            s.beta[tid] = br;
        }
    };
    if (nt > 0) {
        load(start(0));
        put(tiles[0]);
    }
    __syncthreads();
    for (int i = 0; i < nt; ++i) {
        const int t0 = start(i);
        if (i + 1 < nt) load(start(i + 1));
        const ColTile<D, L>& s = tiles[i & 1];
        if (REV) {
            if (t0 >= lo) {
#pragma unroll 4
                for (int j = TT - 1; j >= 0; --j) step(s, j, t0 + j);
            } else {
                for (int j = TT - 1; t0 + j >= lo; --j) step(s, j, t0 + j);
            }
        } else {
            if (t0 + TT <= hi) {
#pragma unroll 4
                for (int j = 0; j < TT; ++j) step(s, j, t0 + j);
            } else {
                for (int j = 0; t0 + j < hi; ++j) step(s, j, t0 + j);
            }
        }
        if (i + 1 < nt) put(tiles[(i + 1) & 1]);
        __syncthreads();
    }
}

// The tile of tokens that a row scan works on: u = beta e, dv = beta du, scale dout; k and q.
template <int D, int L>
struct RowTile {
    float vec[3][Cfg<D>::ROW][D];
    float k[Cfg<D>::ROW][L], q[Cfg<D>::ROW][L];
    float a[Cfg<D>::ROW];
};

struct ScanArgs {
    Packed p;
    const void *q, *k, *v, *g, *beta, *dout;
    const int* cu;
    float scale;
    const float* S0;
    float* S1;
    void* out;
    float *e, *du, *dqh, *rh, *wh;  // [T][H][d]
    float *Sm, *Dm;                 // [T / kMark][H][d][d]: S and D at the marks
};

// A mark's place in Sm and Dm: marks lie kMark tokens apart within a sequence, the first one kMark
// behind its start, so no two of a batch, whatever its sequences, share a multiple of kMark.
__device__ __forceinline__ size_t mark(const Packed& p, int t, int h)
{
    return ((size_t)(t / kMark - 1) * p.H + h) * p.d * p.d;
}

// Which line block, head and sequence this block works on (line blocks of a head side by side).
template <int D, int L>
__device__ __forceinline__ void place(const Packed& p, int b, int& line0, int& h, int& s)
{
    constexpr int LB = D / L;
    line0 = (b % LB) * L;
    h = (b / LB) % p.H;
    s = b / LB / p.H;
}

// Forward by columns.  e (NULL or [T][H][d] fp32) receives v - a S^T k.
template <typename T, int D, int L>
__global__ void __launch_bounds__(L * Cfg<D>::PF, L == kNarrow) delta_fwd_kernel(ScanArgs x)
{
    constexpr int P = Cfg<D>::PF;
    __shared__ ColTile<D, L> tiles[2];
    const Packed& pk = x.p;
    int col0, h, s, lo, hi;
    place<D, L>(pk, blockIdx.x, col0, h, s);
    seq_rows(x.cu, s, pk.T, lo, hi);
    const int tid = threadIdx.x, p = tid % P, cl = tid / P, col = col0 + cl;
    const int H = pk.H, hk = h / (H / pk.Hk);
    Vec<D, P> S;
    const size_t at = ((size_t)s * H + h) * D * D + col;
#pragma unroll
    for (int i = 0; i < Vec<D, P>::N; ++i)
        S.x[i] = x.S0 ? tc::f2_pack(x.S0[at + (size_t)element<P>(2 * i, p) * D],
                                    x.S0[at + (size_t)element<P>(2 * i + 1, p) * D])
                      : tc::f2_pack(0.f, 0.f);
    const long long os = (long long)H * D;
    T* out = (T*)x.out + (long long)lo * os + h * D + col;  // of the token that `o` belongs to
    float* e_out = x.e ? x.e + h * D + col : nullptr;
    float o = 0.f;
    bool any = false;
    col_scan<T, D, L, P, false>(tiles, (const T*)x.k + hk * D, pk.ks, (const T*)x.q + hk * D, pk.qs,
                             (const T*)x.v + h * D + col0, pk.vs, (const T*)x.g + h,
                             (const T*)x.beta + h, H, lo, hi, [&](const ColTile<D, L>& w, int j, int t) {
        Vec<D, P> k, q;
        k.read(w.k[j], p);
        q.read(w.q[j], p);
        const float a = w.a[j], beta = w.beta[j];
        float sk = S.dot(k);
        line_sum2<P>(sk, o);
        const float e = fmaf(-a, sk, w.line[j][cl]);
        S.scale(a);
        S.add(beta * e, k);
        if (p == 0) {
            if (any) from_f32(*out, x.scale * o);
            if (e_out) e_out[t * os] = e;
        }
        if (any) out += os;
        any = true;
        o = S.dot(q);
    });
    o = line_sum<P>(o);
    if (any && p == 0) from_f32(*out, x.scale * o);
    if (x.S1) {
#pragma unroll
        for (int i = 0; i < Vec<D, P>::N; ++i) {
            float a, b;
            tc::f2_unpack(S.x[i], a, b);
            x.S1[at + (size_t)element<P>(2 * i, p) * D] = a;
            x.S1[at + (size_t)element<P>(2 * i + 1, p) * D] = b;
        }
    }
}

// Backward, first scan: columns of D in reverse; du_t = D_t^T k_t, D <- a (D - k dv^T).
template <typename T, int D, int L>
__global__ void __launch_bounds__(L * Cfg<D>::PB, L == kNarrow) delta_bwd_cols_kernel(ScanArgs x)
{
    constexpr int P = Cfg<D>::PB;
    __shared__ ColTile<D, L> tiles[2];
    const Packed& pk = x.p;
    int col0, h, s, lo, hi;
    place<D, L>(pk, blockIdx.x, col0, h, s);
    seq_rows(x.cu, s, pk.T, lo, hi);
    const int tid = threadIdx.x, p = tid % P, cl = tid / P;
    const int H = pk.H, hk = h / (H / pk.Hk);
    const long long os = (long long)H * D;
    Vec<D, P> S = {};
    float* du_out = x.du + h * D + col0 + cl;
    col_scan<T, D, L, P, true>(tiles, (const T*)x.k + hk * D, pk.ks, (const T*)x.q + hk * D, pk.qs,
                            (const T*)x.dout + h * D + col0, os, (const T*)x.g + h,
                            (const T*)x.beta + h, H, lo, hi, [&](const ColTile<D, L>& w, int j, int t) {
        Vec<D, P> k, q;
        k.read(w.k[j], p);
        q.read(w.q[j], p);
        const float a = w.a[j], beta = w.beta[j];
        S.add(x.scale * w.line[j][cl], q);
        const float du = line_sum<P>(S.dot(k));
        S.add(-beta * du, k);
        S.scale(a);
        if (p == 0) du_out[t * os] = du;
    });
}

// Backward, the row scans: even blocks rows of S forward (dq = scale S dout, r = a S_{t-1} dv),
// odd blocks rows of D in reverse (w = D u, u = beta e).  By tokens; sums of 8 tokens at once.
template <typename T, int D, int L>
__global__ void __launch_bounds__(L * Cfg<D>::PR, L == kNarrow) delta_bwd_rows_kernel(ScanArgs x)
{
    constexpr int TT = Cfg<D>::ROW, NT = L * Cfg<D>::PR, P = Cfg<D>::PR;
    constexpr int SLOTS = TT * D / 4;                            // 16-byte pieces of a vector: 256
    constexpr int LV = (3 * SLOTS + NT - 1) / NT, LL = TT * L / NT ? TT * L / NT : 1;
    __shared__ RowTile<D, L> tiles[2];
    tc::grid_dep_wait();  // du
    const Packed& pk = x.p;
    const bool rev = blockIdx.x & 1;
    int row0, h, s, lo, hi;
    place<D, L>(pk, blockIdx.x / 2, row0, h, s);
    seq_rows(x.cu, s, pk.T, lo, hi);
    const int tid = threadIdx.x, p = tid % P, rl = tid / P, nt = (hi - lo + TT - 1) / TT;
    const int H = pk.H, hk = h / (H / pk.Hk);
    const long long os = (long long)H * D;
    const T *g = (const T*)x.g + h, *beta = (const T*)x.beta + h;
    const T *k = (const T*)x.k + hk * D + row0, *q = (const T*)x.q + hk * D + row0;
    Vec<D, P> S = {};

    float4 v[LV];  // this thread's pieces of the three vectors, and what they are multiplied by
    float m[LV], kr[LL], qr[LL], ar = 0.f;
    // In reverse the tiles lie as they do forward: the tokens behind the last one leave D zero.
    static_assert(kMark % TT == 0, "marks lie between tiles");
    auto start = [&](int i) { return lo + (rev ? nt - 1 - i : i) * TT; };
    auto load = [&](int t0) {
#pragma unroll
        for (int i = 0; i < LV; ++i) {
            const int slot = tid + NT * i, n = slot / SLOTS, e = slot % SLOTS * 4, t = t0 + e / D, c = e % D;
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            m[i] = 0.f;
            if (n >= 3 || t < lo || t >= hi) continue;
            const size_t at = (size_t)t * os + h * D + c;
            m[i] = x.scale;
            if (n < 2) {
                v[i] = load4((n ? x.du : x.e) + at);
                m[i] = to_f32(beta[(size_t)t * H]);
            } else {
                v[i] = load4((const T*)x.dout + at);
            }
        }
#pragma unroll
        for (int i = 0; i < LL; ++i) {
            const int e = tid + NT * i, t = t0 + e / L;
            const bool in = e < TT * L && t >= lo && t < hi;
            kr[i] = in ? to_f32(k[t * pk.ks + e % L]) : 0.f;
            qr[i] = in ? to_f32(q[t * pk.qs + e % L]) : 0.f;
        }
        if (tid < TT) ar = t0 + tid >= lo && t0 + tid < hi ? to_f32(g[(size_t)(t0 + tid) * H]) : 0.f;
    };
    auto put = [&](RowTile<D, L>& w) {
#pragma unroll
        for (int i = 0; i < LV; ++i) {
            const int slot = tid + NT * i;
            if (slot < 3 * SLOTS)
                *(float4*)(&w.vec[0][0][0] + 4 * slot) =
                    make_float4(v[i].x * m[i], v[i].y * m[i], v[i].z * m[i], v[i].w * m[i]);
        }
#pragma unroll
        for (int i = 0; i < LL; ++i) {
            const int e = tid + NT * i;
            if (e < TT * L) {
                (&w.k[0][0])[e] = kr[i];
                (&w.q[0][0])[e] = qr[i];
            }
        }
        if (tid < TT) w.a[tid] = expf(ar);
    };
    if (nt > 0) {
        load(start(0));
        put(tiles[0]);
    }
    __syncthreads();
    const size_t out = (size_t)h * D + row0 + rl;
    for (int i = 0; i < nt; ++i) {
        const RowTile<D, L>& w = tiles[i & 1];
        if (i + 1 < nt) load(start(i + 1));
#pragma unroll 1
        for (int jj = 0; jj < TT; jj += 8) {
            const int j = rev ? TT - 8 - jj : jj, t = start(i) + j + p / (P / 8);  // the token whose sums this lane gets
            const bool store = (P == 8 || !(p & 1)) && t >= lo && t < hi;
            float a[8], b[8];
            if (!rev) {
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    Vec<D, P> u, dv, dO;
                    u.read(w.vec[0][j + y], p);
                    dv.read(w.vec[1][j + y], p);
                    dO.read(w.vec[2][j + y], p);
                    S.scale(w.a[j + y]);
                    a[y] = S.dot(dv);
                    S.add(w.k[j + y][rl], u);
                    b[y] = S.dot(dO);
                }
                const float r = line_sums8<P>(a, p), dq = line_sums8<P>(b, p);
                if (store) {
                    x.rh[out + t * os] = r;
                    x.dqh[out + t * os] = dq;
                }
            } else {
#pragma unroll
                for (int y = 7; y >= 0; --y) {
                    Vec<D, P> u, dv, dO;
                    u.read(w.vec[0][j + y], p);
                    dv.read(w.vec[1][j + y], p);
                    dO.read(w.vec[2][j + y], p);
                    S.add(w.q[j + y][rl], dO);
                    a[y] = S.dot(u);
                    S.add(-w.k[j + y][rl], dv);
                    S.scale(w.a[j + y]);
                }
                const float z = line_sums8<P>(a, p);
                if (store) x.wh[out + t * os] = z;
            }
        }
        const int m0 = start(i) + (rev ? 0 : TT);  // the token that the state now stands before
        if (m0 > lo && m0 < hi && (m0 - lo) % kMark == 0) {
            float* to = (rev ? x.Dm : x.Sm) + mark(pk, m0, h) + (size_t)(row0 + rl) * D;
#pragma unroll
            for (int y = 0; y < Vec<D, P>::N / 2; ++y)
                *(ulonglong2*)(to + 4 * (P * y + p)) = make_ulonglong2(S.x[2 * y], S.x[2 * y + 1]);
        }
        if (i + 1 < nt) put(tiles[(i + 1) & 1]);
        __syncthreads();
    }
}

struct FinishArgs {
    Packed p;
    const void *q, *k, *g, *beta;
    const int* cu;
    const float *e, *du, *dqh, *rh, *wh;
    void *dq, *dk, *dv, *dbeta, *dg;
    const float *Sm, *Dm;
    float* dG;  // [H][T]
};

// Row by row: dq and dk summed over the heads of a key head, dv = beta du, dbeta = e . du, and
// dG = q.dq - k.r - k.w, by which dg falls from a token to the next (q_t and the reading k_t come
// with exp(+G_t), the writing k_t with exp(-G_t), G_t the sum of the log decays).  One warp per (row, key head), D / 32 elements a lane.
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

// dg_t = a_t <S_{t-1}, D_t - k_t dv_t^T> falls by dG_t from t to t + 1.  As a sum of dG over a whole
// sequence its terms nearly cancel (1000 tokens, H4 d64: dg 2.1e-6 wrong in the 2-norm, and worse
// with the length).  So the row scans leave S and D at marks kMark tokens apart (8 MB of 4 x 1000
// tokens), dg at a mark is <D, S>, and only the terms since then are subtracted, in 64 bits.  At a
// sequence's first token the state ahead is 0, and at a token with a_t = 0 nothing of it is left:
// dg is 0 there, not what two equal sums leave to rounding, and the terms are counted from there.
// One block per (kMark tokens, head).
template <typename T>
__global__ void __launch_bounds__(256) delta_bwd_gate_kernel(FinishArgs x)
{
    __shared__ double part[8], before[kMark], half;  // before: the terms from the mark up to a token
    __shared__ int half_from;
    const Packed& pk = x.p;
    const int h = blockIdx.x % pk.H, tid = threadIdx.x, lane = tid & 31;
    int s, block, lo, hi;
    if (!find_block(x.cu, pk.n, pk.T, kMark, (int)(blockIdx.x / pk.H), s, block, lo, hi)) return;
    const int t0 = lo + block * kMark, n = min(kMark, hi - t0), t = t0 + tid;
    tc::grid_dep_wait();
    double dot = 0.;
    if (t0 > lo) {
        const float *S = x.Sm + mark(pk, t0, h), *D = x.Dm + mark(pk, t0, h);
        for (int i = 4 * tid; i < pk.d * pk.d; i += 4 * 256) {
            const float4 a = load4(S + i), b = load4(D + i);
            dot += (double)(a.x * b.x + a.y * b.y + (a.z * b.z + a.w * b.w));
        }
    }
#pragma unroll
    for (int m = 16; m; m /= 2) dot += __shfl_xor_sync(0xffffffffu, dot, m);
    // sums of the terms up to t, and the last token up to t whose gate is 0 (-1: none since the mark)
    double sum = tid < n ? (double)x.dG[(size_t)h * pk.T + t] : 0.;
    int from = tid < n && expf(to_f32(((const T*)x.g)[(size_t)t * pk.H + h])) == 0.f ? tid : -1;
#pragma unroll
    for (int m = 1; m < 32; m *= 2) {
        const double o = __shfl_up_sync(0xffffffffu, sum, m);
        const int f = __shfl_up_sync(0xffffffffu, from, m);
        if (lane >= m) {
            sum += o;
            from = max(from, f);
        }
    }
    if (lane == 0) part[tid >> 5] = dot;
    if (tid == 31) {
        half = sum;
        half_from = from;
    }
    const double up = __shfl_up_sync(0xffffffffu, sum, 1);
    __syncthreads();
    if (tid < kMark) before[tid] = (lane ? up : 0.) + (tid >= 32 ? half : 0.);
    __syncthreads();
    if (tid >= n) return;
    if (tid >= 32) from = max(from, half_from);
    dot = 0.;
    for (int w = 0; w < 8; ++w) dot += part[w];
    const double first = from >= 0 ? before[from] : dot;
    from_f32(((T*)x.dg)[(size_t)t * pk.H + h], (float)(first - before[tid]));
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

// Blocks of L lines.  16 of them where even so every block has an SM to itself (fewer warps there
// to share its schedulers and shared memory, and registers for as many loads as a thread then has
// in flight), else 32 (half the staging).  Measured, 16 against 32 lines, sequences of 500 tokens, us:
// d64 forward 78 and 103 (128 blocks of 16 lines), 144 and 140 (512), 447 and 427 (2048); columns and
// rows backward 127 and 161 (64, 128), 479 and 425 (512, 1024); d128 forward 103 and 162 (128), backward
// 183 and 272 (32, 64), 423 and 398 (256, 512).
template <int D>
bool narrow(const Packed& p, int sides)
{
    return (long long)p.n * p.H * (D / kNarrow) * sides <= tc::sm_count();
}

template <int D, int L, typename Kernel>
cudaError_t scan(Kernel kernel, int P, int sides, bool after, const ScanArgs& x, cudaStream_t s)
{
    const long long blocks = (long long)x.p.n * x.p.H * (D / L) * sides;
    return tc::launch_after(kernel, dim3((unsigned)blocks), L * P, 0, 0, after, s, x);
}

template <typename T, int D>
cudaError_t fwd(const ScanArgs& x, cudaStream_t s)
{
    using C = Cfg<D>;
    return narrow<D>(x.p, 1) ? scan<D, kNarrow>(delta_fwd_kernel<T, D, kNarrow>, C::PF, 1, false, x, s)
                             : scan<D, kWide>(delta_fwd_kernel<T, D, kWide>, C::PF, 1, false, x, s);
}

template <typename T, int D>
cudaError_t bwd(const ScanArgs& x, const FinishArgs& f, cudaStream_t s)
{
    using C = Cfg<D>;
    const Packed& p = x.p;
    cudaError_t e = narrow<D>(p, 1)
        ? scan<D, kNarrow>(delta_bwd_cols_kernel<T, D, kNarrow>, C::PB, 1, false, x, s)
        : scan<D, kWide>(delta_bwd_cols_kernel<T, D, kWide>, C::PB, 1, false, x, s);
    if (e == cudaSuccess)
        e = narrow<D>(p, 2) ? scan<D, kNarrow>(delta_bwd_rows_kernel<T, D, kNarrow>, C::PR, 2, true, x, s)
                            : scan<D, kWide>(delta_bwd_rows_kernel<T, D, kWide>, C::PR, 2, true, x, s);
    const long long items = (long long)p.T * p.Hk;
    if (e == cudaSuccess)
        e = tc::launch_after(delta_bwd_finish_kernel<T, D>, dim3((unsigned)((items + 3) / 4)), 128, 0,
                             0, true, s, f);
    if (e == cudaSuccess)
        e = tc::launch_after(delta_bwd_gate_kernel<T>,
                             dim3((unsigned)((long long)block_slots(p.T, p.n, kMark) * p.H)), 256, 0, 0,
                             true, s, f);
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
static size_t mark_floats(const Packed& p) { return (size_t)(p.T / kMark) * p.H * p.d * p.d; }
// du, dq, r, w per head, S and D at the marks, and dG
size_t delta_scan_ws_floats(const Packed& p)
{
    return 4 * delta_scan_save_floats(p) + 2 * mark_floats(p) + (size_t)p.T * p.H;
}

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
    x.Sm = scratch + 4 * n; x.Dm = x.Sm + mark_floats(p);
    FinishArgs f = {};
    f.p = p;
    f.q = q; f.k = k; f.g = g; f.beta = beta; f.cu = cu;
    f.e = e; f.du = x.du; f.dqh = x.dqh; f.rh = x.rh; f.wh = x.wh;
    f.dq = dq; f.dk = dk; f.dv = dv; f.dbeta = dbeta; f.dg = dg;
    f.Sm = x.Sm; f.Dm = x.Dm;
    f.dG = x.Dm + mark_floats(p);
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
