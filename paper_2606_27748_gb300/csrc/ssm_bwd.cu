// Selective state space scan, backward.  With dy_t = dout_t silu(z_t) and e_t the gradient of h_t
// (later tokens included), from a sequence's last token to its first:
//   e_t += dy_t C_t;  dC_t = sum_c dy_t h_t;  dB_t = sum_c D_t x_t e_t;  s_t = <e_t, B_t>;
//   q_t = e_t exp(D_t A) h_{t-1};  dA += D_t q_t;  dD_t = s_t x_t + <q_t, A>;
//   dx_t = s_t D_t + Ds dy_t;  dDs += dy_t x_t;  e_{t-1} = exp(D_t A) e_t.
//
// A thread holds 4 states of each of 2 channels, as in the forward, and walks tiles of 8 tokens from
// the marks that the forward left: the tile's states again, kept in registers, then back.  The other
// half of the threads brings tiles, finishes what the walk has summed over states (s_t, <q_t, A>,
// <C_t, h_t>, by shuffles) and sums dB and dC over the block's channels, which the walk leaves in shared
// memory for 4 tokens at a time.  Sums over blocks go through global memory to a kernel of their own.
// Every order is fixed.  What bounds it is shared memory's bandwidth: B, C and steps twice, and dB and dC
// out and in again, 7 of its 128-byte wavefronts for 32 elements (token, channel, state), 65% of what an
// SM has, and 23 instructions, 51% of the issue slots: 321 us for 8 x 1024 tokens of 2048 channels of 16
// states (1 channel a thread, all threads alike: 651).
#include "flex_internal.h"
#include "ssm.cuh"

namespace flex {
namespace {

using namespace ssm;

constexpr int kHalf = kMark / 2;
// Channels of a block.
constexpr int channels(int N) { return N <= 16 ? 64 : 32; }

template <typename T, int N_>
struct Layout {
    static constexpr int N = N_, CT = channels(N), L = N / 4, CG = CT / 2;  // CG: pairs of channels
    static constexpr int WALK = CG * L, BRING = 2 * CT;
    static constexpr int RING = 4;
    struct Raw {
        T x[kMark][CT], dt[kMark][CT], z[kMark][CT], dout[kMark][CT], bc[kMark][2][N];
        float mark[CT][N];
    };
    struct Smem {
        Raw raw[RING];
        float2 td[2][kMark][CT];            // D_t, D_t x_t
        float dy[2][kMark][CT];
        float bc[2][kMark][2][N];
        float sums[2][3][kMark][CT + 8];    // s_t, <q_t, A>, <C_t, h_t>
        float pair[2][kHalf][2][CG][N];     // dB and dC of a pair of channels
    };
    static_assert(kMark * CT / 4 == BRING, "a group of 4 channels of a token for each");
};

__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Sums of 4 tokens' values over a channel's L lanes; lane sub returns those of tokens
// sub, sub + L, ... (L = 8: sub % 4, twice).
template <int L>
__device__ __forceinline__ void token_sums(const float (&x)[4], int sub, float (&out)[L == 2 ? 2 : 1])
{
    if constexpr (L == 2) {
        float a[2] = {x[0], x[1]}, b[2] = {x[2], x[3]};
        out[0] = lane_sums<2>(a, sub);
        out[1] = lane_sums<2>(b, sub);
    } else {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = L == 8 ? x[i] + __shfl_xor_sync(0xffffffffu, x[i], 4) : x[i];
        out[0] = lane_sums<4>(v, sub % 4);
    }
}

template <typename T, int N>
__global__ void __launch_bounds__(Layout<T, N>::WALK + Layout<T, N>::BRING, 2) ssm_bwd_kernel(SsmArgs a)
{
    using Y = Layout<T, N>;
    constexpr int CT = Y::CT, L = Y::L, CG = Y::CG, NT = Y::BRING, CQ = CT / 4;
    extern __shared__ __align__(16) unsigned char smem[];
    typename Y::Smem& sm = *(typename Y::Smem*)smem;
    const bool walks = threadIdx.x < Y::WALK;
    const int tid = walks ? threadIdx.x : threadIdx.x - Y::WALK;
    Place p;
    const bool found = find_place<CT>(a, blockIdx.x, p);
    const int cg = tid / L, ch = 2 * cg, sub = tid % L;
    const bool mine = walks && ch < p.nc;  // (channels come in fours)
    const size_t DN = (size_t)a.D * N, state = (size_t)(p.c0 + ch) * N + 4 * sub;
    const int q4 = 4 * (tid % CQ), tt = tid / CQ;  // a bringing thread's group of 4 channels of a token
    const bool stages = !walks && q4 < p.nc;
    tc::grid_dep_wait();
    if (!found) {  // no rows, no gradients
        const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mine)
            for (int c = 0; c < 2; ++c) *(float4*)(a.part_a + p.slot * DN + state + c * N) = zero;
        if (stages && tt < 2) *(float4*)(a.part_d + ((size_t)p.slot * 2 + tt) * a.D + p.c0 + q4) = zero;
        return;
    }
    const int blocks = (p.hi - p.lo + a.rows - 1) / a.rows;
    const int nt = (p.last - p.first + kMark - 1) / kMark;
    const bool gate = a.z != nullptr;

    if (!walks) {
        const T *x = (const T*)a.x, *dt = (const T*)a.dt, *z = (const T*)a.z, *dout = (const T*)a.dout;
        float4 bias = make_float4(0.f, 0.f, 0.f, 0.f), Ds = bias, dDs = bias, dbias = bias;
        if (stages) {
            if (a.bias) bias = *(const float4*)(a.bias + p.c0 + q4);
            if (a.Ds) Ds = *(const float4*)(a.Ds + p.c0 + q4);
        }
        const float* marks = a.marks + ((size_t)(p.lo / kMark + p.s) + (p.first - p.lo) / kMark) * DN
                           + (size_t)p.c0 * N;
        // a thread's groups in memory (the walk goes from the last tile to the first)
        const long long t0 = p.first + (nt - 1) * kMark + tt;
        const T* from[4] = {x + t0 * a.xs + p.c0 + q4, dt + t0 * a.ds + p.c0 + q4, dout + t0 * a.D + p.c0 + q4,
                            gate ? z + t0 * a.zs + p.c0 + q4 : z};
        const long long back[4] = {kMark * a.xs, kMark * a.ds, (long long)kMark * a.D, kMark * a.zs};
        constexpr int ROWS_BC = kMark * 2 * L / NT > 0 ? kMark * 2 * L / NT : 1;  // groups of B and C
        const int bw = tid / (kMark * L) % 2, bu = tid / L % kMark, bm = 4 * (tid % L);
        auto fetch = [&](int i) {  // (called for one tile after the other)
            typename Y::Raw& r = sm.raw[i % Y::RING];
            const int left = p.last - (p.first + i * kMark);  // rows that exist, from the tile's first
            const bool in = stages && tt < left;
            // (what is not read has a valid address too: the tensor's)
            copy_quad(&r.x[tt][q4], in ? from[0] : x, in);
            copy_quad(&r.dt[tt][q4], in ? from[1] : x, in);
            copy_quad(&r.dout[tt][q4], in ? from[2] : x, in);
            if (gate) copy_quad(&r.z[tt][q4], in ? from[3] : x, in);
#pragma unroll
            for (int k = 0; k < 4; ++k) from[k] -= back[k];
#pragma unroll
            for (int k = 0; k < ROWS_BC; ++k) {
                const int f = tid + k * NT, which = ROWS_BC > 1 ? f / (kMark * L) : bw;
                if (f >= kMark * 2 * L) break;
                const bool row = bu < left;
                const long long at = row ? p.first + i * kMark + bu : p.first;
                if (which) copy_quad(&r.bc[bu][1][bm], (const T*)a.C + at * a.cs + p.g * N + bm, row);
                else copy_quad(&r.bc[bu][0][bm], (const T*)a.B + at * a.bs + p.g * N + bm, row);
            }
#pragma unroll
            for (int k = 0; k < CT * L / NT; ++k) {
                const int f = tid + k * NT;
                const bool row = f / L < p.nc;
                copy_quad(&r.mark[0][0] + 4 * f, marks + i * DN + (row ? 4 * f : 0), row);
            }
        };
        auto convert = [&](int i) {
            const typename Y::Raw& r = sm.raw[i % Y::RING];
            Quad<T> xr, dr, zr, gr;
            xr.load(&r.x[tt][q4]);
            dr.load(&r.dt[tt][q4]);
            gr.load(&r.dout[tt][q4]);
            const bool in = stages && p.first + i * kMark + tt < p.last;
            if (a.softplus && !in) dr.low();  // a token that does not exist takes a step of 0
            const float4 xv = xr.get(), w = dr.get();
            float4 dy = gr.get();
            if (gate) {
                zr.load(&r.z[tt][q4]);
                const float4 g = zr.get();
                dy.x *= silu(g.x); dy.y *= silu(g.y); dy.z *= silu(g.z); dy.w *= silu(g.w);
            }
            float d[4] = {w.x + bias.x, w.y + bias.y, w.z + bias.z, w.w + bias.w};
            if (a.softplus) softplus4(d);
            else if (!in) d[0] = d[1] = d[2] = d[3] = 0.f;
            float4* to = (float4*)&sm.td[i & 1][tt][q4];
            const float4 lo = make_float4(d[0], d[0] * xv.x, d[1], d[1] * xv.y);
            const float4 hi = make_float4(d[2], d[2] * xv.z, d[3], d[3] * xv.w);
            const bool odd = tid / 4 % 2;  // (halves in turn: 8 lanes' 128 bytes are in 32 banks)
            to[odd] = odd ? hi : lo;
            to[!odd] = odd ? lo : hi;
            *(float4*)&sm.dy[i & 1][tt][q4] = dy;
#pragma unroll
            for (int k = 0; k < ROWS_BC; ++k) {
                const int f = tid + k * NT, which = ROWS_BC > 1 ? f / (kMark * L) : bw;
                if (f >= kMark * 2 * L) break;
                Quad<T> v;
                v.load(&r.bc[bu][which][bm]);
                *(float4*)&sm.bc[i & 1][bu][which][bm] = v.get();
            }
        };
        // dx, ddt, dz of a tile
        auto finish = [&](int i) {
            const long long t = p.first + i * kMark + tt;
            if (!stages || t >= p.last) return;
            const typename Y::Raw& r = sm.raw[i % Y::RING];
            Quad<T> xr, dr, zr, gr;
            xr.load(&r.x[tt][q4]);
            dr.load(&r.dt[tt][q4]);
            const float4 xq = xr.get(), dq = dr.get(), dyq = *(const float4*)&sm.dy[i & 1][tt][q4];
            const float4 s1 = *(const float4*)&sm.sums[i & 1][0][tt][q4];
            const float4 s2 = *(const float4*)&sm.sums[i & 1][1][tt][q4];
            const float xv[4] = {xq.x, xq.y, xq.z, xq.w}, dy[4] = {dyq.x, dyq.y, dyq.z, dyq.w};
            const float raw[4] = {dq.x + bias.x, dq.y + bias.y, dq.z + bias.z, dq.w + bias.w};
            const float Dv[4] = {Ds.x, Ds.y, Ds.z, Ds.w};
            const float s[4] = {s1.x, s1.y, s1.z, s1.w}, q[4] = {s2.x, s2.y, s2.z, s2.w};
            float gx[4], gd[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                gx[j] = fmaf(s[j], sm.td[i & 1][tt][q4 + j].x, Dv[j] * dy[j]);
                gd[j] = fmaf(s[j], xv[j], q[j] * kLn2);
                if (a.softplus) gd[j] *= sigmoid(raw[j]);
            }
            dDs.x = fmaf(dy[0], xv[0], dDs.x); dDs.y = fmaf(dy[1], xv[1], dDs.y);
            dDs.z = fmaf(dy[2], xv[2], dDs.z); dDs.w = fmaf(dy[3], xv[3], dDs.w);
            dbias.x += gd[0]; dbias.y += gd[1]; dbias.z += gd[2]; dbias.w += gd[3];
            const size_t at = t * a.D + p.c0 + q4;
            store4((T*)a.dx + at, make_float4(gx[0], gx[1], gx[2], gx[3]));
            store4((T*)a.ddt + at, make_float4(gd[0], gd[1], gd[2], gd[3]));
            if (gate) {
                zr.load(&r.z[tt][q4]);
                gr.load(&r.dout[tt][q4]);
                const float4 zq = zr.get(), oq = gr.get(), yq = *(const float4*)&sm.sums[i & 1][2][tt][q4];
                const float zv[4] = {zq.x, zq.y, zq.z, zq.w}, o[4] = {oq.x, oq.y, oq.z, oq.w};
                const float y[4] = {yq.x, yq.y, yq.z, yq.w};
                float gz[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float g = logistic(zv[j]);
                    gz[j] = o[j] * fmaf(Dv[j], xv[j], y[j]) * g * fmaf(zv[j], 1.f - g, 1.f);
                }
                store4((T*)a.dz + at, make_float4(gz[0], gz[1], gz[2], gz[3]));
            }
        };
        // dB and dC of 4 tokens: 4 threads add up a quarter of the pairs of channels each, in turn
        auto sum_pairs = [&](int i, int half) {
#pragma unroll
            for (int k4 = 0; k4 < (32 * L + NT - 1) / NT; ++k4) {
                const int f = tid + k4 * NT;
                if (32 * L < NT && f >= 32 * L) break;  // (whole warps)
                const int m = f % L, part = f / L % 4, which = f / (4 * L) % 2, u = f / (8 * L);
                const float* from = &sm.pair[half][u][which][part][4 * m];
                States<4> v, w;
                v.read(from);
#pragma unroll
                for (int k = 1; k < CG / 4; ++k) {
                    w.read(from + 4 * k * N);
                    v.v[0] = f2_add(v.v[0], w.v[0]);
                    v.v[1] = f2_add(v.v[1], w.v[1]);
                }
#pragma unroll
                for (int k = L; k <= 2 * L; k *= 2)
#pragma unroll
                    for (int q = 0; q < 2; ++q)
                        v.v[q] = f2_add(v.v[q], __shfl_xor_sync(0xffffffffu, (unsigned long long)v.v[q], k));
                const int t = i * kMark + half * kHalf + u + p.first;
                if (part == 0 && t < p.last)
                    v.write(a.part_bc + (((size_t)p.tile * a.T + t) * a.G + p.g) * 2 * N + which * N + 4 * m);
            }
        };
        fetch(nt - 1);
        copies_commit();
        if (nt > 1) fetch(nt - 2);
        copies_commit();
        copies_wait<1>();
        bring_barrier(NT);
        convert(nt - 1);
        for (int i = nt - 1; i >= 0; --i) {
            copies_wait<0>();
            __syncthreads();  // tile i is there, and i + 1 walked
            if (i > 1) fetch(i - 2);
            copies_commit();
            if (i + 1 < nt) {
                sum_pairs(i + 1, 0);
                finish(i + 1);
            }
            if (i > 0) convert(i - 1);
            __syncthreads();  // the tile's later tokens are walked
            sum_pairs(i, 1);
        }
        __syncthreads();
        sum_pairs(0, 0);
        finish(0);
        // dDs and dbias over the tokens of a tile, which 8 threads hold; all of them are done with sums
        bring_barrier(NT);
        *(float4*)&sm.sums[0][0][tt][q4] = dDs;
        *(float4*)&sm.sums[0][1][tt][q4] = dbias;
        bring_barrier(NT);
        if (stages && tt < 2) {
            float4 v = *(const float4*)&sm.sums[0][tt][0][q4];
#pragma unroll
            for (int k = 1; k < kMark; ++k) {
                const float4 u = *(const float4*)&sm.sums[0][tt][k][q4];
                v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
            }
            *(float4*)(a.part_d + ((size_t)p.slot * 2 + tt) * a.D + p.c0 + q4) = v;
        }
        return;
    }

    States<4> A2[2], e[2], dA[2];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        A2[c].zero(); e[c].zero(); dA[c].zero();
        if (!mine) continue;
        A2[c].read(a.A + state + c * N);
#pragma unroll
        for (int k = 0; k < 2; ++k) A2[c].v[k] = tc::f2_mul(A2[c].v[k], twice(kLog2e));
        // the gradient of the state behind the block
        if (blocks > 1) e[c].read(a.ends + p.slot * DN + state + c * N);
    }
    for (int i = nt - 1; i >= 0; --i) {
        __syncthreads();
        const float2(*td)[CT] = sm.td[i & 1];
        const float(*dys)[CT] = sm.dy[i & 1];
        const float(*bc)[2][N] = sm.bc[i & 1];
        States<4> h0[2], hh[kMark][2], dAt[2];  // dAt: the tile's part, so that long sums are sums of sums
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            h0[c].read(&sm.raw[i % Y::RING].mark[ch + c][4 * sub]);
            dAt[c].zero();
        }
#pragma unroll
        for (int t = 0; t < kMark; ++t) {
            const float4 v = *(const float4*)&td[t][ch];
            States<4> B;
            B.read(&bc[t][0][4 * sub]);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint64_t d = twice(c ? v.z : v.x), u = twice(c ? v.w : v.y);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint64_t w = ex2_pair(tc::f2_fma(A2[c].v[k], d, twice(kUp)));
                    hh[t][c].v[k] = tc::f2_fma(w, t ? hh[t - 1][c].v[k] : h0[c].v[k], tc::f2_mul(u, B.v[k]));
                }
            }
        }
#pragma unroll
        for (int half = 1; half >= 0; --half) {
            float s1[2][kHalf], s2[2][kHalf], y[2][kHalf];
#pragma unroll
            for (int u = kHalf - 1; u >= 0; --u) {
                const int t = half * kHalf + u;
                const float4 v = *(const float4*)&td[t][ch];
                const float2 g = *(const float2*)&dys[t][ch];
                States<4> B, Cv, dB, dC;
                B.read(&bc[t][0][4 * sub]);
                Cv.read(&bc[t][1][4 * sub]);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint64_t dy = twice(c ? g.y : g.x), d = twice(c ? v.z : v.x), dx = twice(c ? v.w : v.y);
                    uint64_t ya = 0, sa = 0, qa = 0;
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const uint64_t h = hh[t][c].v[k], hp = t ? hh[t - 1][c].v[k] : h0[c].v[k];
                        uint64_t& ek = e[c].v[k];
                        ya = k ? tc::f2_fma(h, Cv.v[k], ya) : tc::f2_mul(h, Cv.v[k]);
                        dC.v[k] = c ? tc::f2_fma(dy, h, dC.v[k]) : tc::f2_mul(dy, h);
                        ek = tc::f2_fma(dy, Cv.v[k], ek);
                        dB.v[k] = c ? tc::f2_fma(dx, ek, dB.v[k]) : tc::f2_mul(dx, ek);
                        sa = k ? tc::f2_fma(ek, B.v[k], sa) : tc::f2_mul(ek, B.v[k]);
                        ek = tc::f2_mul(ex2_pair(tc::f2_fma(A2[c].v[k], d, twice(kUp))), ek);
                        const uint64_t q = tc::f2_mul(ek, hp);
                        qa = k ? tc::f2_fma(q, A2[c].v[k], qa) : tc::f2_mul(q, A2[c].v[k]);
                        dAt[c].v[k] = tc::f2_fma(d, q, dAt[c].v[k]);
                    }
                    float lo, hi;
                    tc::f2_unpack(ya, lo, hi);
                    y[c][u] = lo + hi;
                    tc::f2_unpack(sa, lo, hi);
                    s1[c][u] = lo + hi;
                    tc::f2_unpack(qa, lo, hi);
                    s2[c][u] = lo + hi;
                }
                dB.write(&sm.pair[half][u][0][cg][4 * sub]);
                dC.write(&sm.pair[half][u][1][cg][4 * sub]);
            }
            constexpr int M = L == 2 ? 2 : 1;
            float r[3][2][M];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                token_sums<L>(s1[c], sub, r[0][c]);
                token_sums<L>(s2[c], sub, r[1][c]);
                if (gate) token_sums<L>(y[c], sub, r[2][c]);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
#pragma unroll
                for (int m = 0; m < M; ++m)
                    if (k < 2 || gate)
                        *(float2*)&sm.sums[i & 1][k][half * kHalf + sub % 4 + m * L][ch] =
                            make_float2(r[k][0][m], r[k][1][m]);
            if (half) __syncthreads();
        }
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int k = 0; k < 2; ++k) dA[c].v[k] = f2_add(dA[c].v[k], dAt[c].v[k]);
    }
    __syncthreads();
    if (!mine) return;
#pragma unroll
    for (int c = 0; c < 2; ++c) dA[c].write(a.part_a + p.slot * DN + state + c * N);
}

// Sums over blocks, in their order: dB and dC over the blocks of a group (4 values a thread), then dA,
// dDs and dbias over the slots.
template <typename T>
__global__ void __launch_bounds__(256) ssm_bwd_sum_kernel(SsmArgs a, int tiles, int slots, long long bc_blocks)
{
    tc::grid_dep_wait();
    if (blockIdx.x < bc_blocks) {
        const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
        const int per = a.G * 2 * a.N / 4;
        const long long t = i / per;
        if (t >= min(max(__ldg(a.cu + a.n), 0), a.T)) return;
        const int f = (int)(i % per) * 4, g = f / (2 * a.N), k = f / a.N % 2, m = f % a.N;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        const size_t row = (size_t)a.G * 2 * a.N;
#pragma unroll 8
        for (int j = 0; j < tiles; ++j) {
            const float4 u = *(const float4*)(a.part_bc + ((size_t)j * a.T + t) * row + f);
            v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
        }
        store4((T*)(k ? a.dC : a.dB) + ((size_t)t * a.G + g) * a.N + m, v);
        return;
    }
    const long long i = ((long long)(blockIdx.x - bc_blocks) * 256 + threadIdx.x) * 4;
    const long long DN = (long long)a.D * a.N;
    const float* from;
    float* to;
    size_t step;
    if (i < DN) {
        from = a.part_a + i; to = a.dA + i; step = DN;
    } else {
        const long long c = i - DN;
        if (c >= 2 * a.D) return;
        float* base = c < a.D ? a.dDs : a.dbias;
        if (!base) return;
        from = a.part_d + c; to = base + c % a.D; step = 2 * (size_t)a.D;
    }
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
    for (int j = 0; j < slots; ++j) {
        const float4 u = *(const float4*)(from + j * step);
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    *(float4*)to = v;
}

template <typename T, int N>
cudaError_t bwd(const SsmArgs& a, bool after, cudaStream_t s)
{
    using Y = Layout<T, N>;
    const int slots = block_slots(a.T, a.n, a.rows), tiles = group_tiles(a, Y::CT);
    auto kernel = ssm_bwd_kernel<T, N>;
    constexpr int bytes = sizeof(typename Y::Smem);
    static_assert(bytes <= 112 * 1024, "two blocks an SM");
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    e = tc::launch_after(kernel, dim3((unsigned)((long long)slots * tiles * a.G)), Y::WALK + Y::BRING, bytes, 0,
                         after, s, a);
    if (e != cudaSuccess) return e;
    const long long bc = ((long long)a.T * a.G * 2 * a.N / 4 + 255) / 256;
    const long long par = (((long long)a.D * (a.N + 2)) / 4 + 255) / 256;
    return tc::launch_after(ssm_bwd_sum_kernel<T>, dim3((unsigned)(bc + par)), 256, 0, 0, true, s, a, tiles,
                            slots, bc);
}
template <typename T>
cudaError_t bwd_n(const SsmArgs& a, bool after, cudaStream_t s)
{
    return a.N == 8 ? bwd<T, 8>(a, after, s) : a.N == 16 ? bwd<T, 16>(a, after, s) : bwd<T, 32>(a, after, s);
}

}  // namespace

int ssm_bwd_tiles(const SsmArgs& a) { return group_tiles(a, channels(a.N)); }

cudaError_t launch_ssm_bwd(const SsmArgs& a, cudaStream_t s)
{
    const bool cut = a.rows <= a.T;
    if (cut) {
        const cudaError_t e = launch_ssm_back_ends(a, s);
        if (e != cudaSuccess) return e;
    }
    return a.bf16 ? bwd_n<__nv_bfloat16>(a, cut, s) : bwd_n<float>(a, cut, s);
}

}  // namespace flex
