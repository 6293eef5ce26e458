// Selective state space scan, backward.  With dy_t = dout_t silu(z_t) and e_t the gradient of h_t
// (later tokens included), from a sequence's last token to its first:
//   e_t += dy_t C_t;  dC_t = sum_c dy_t h_t;  dB_t = sum_c D_t x_t e_t;  s_t = <e_t, B_t>;
//   q_t = e_t exp(D_t A) h_{t-1};  dA += D_t q_t;  dD_t = s_t x_t + <q_t, A>;
//   dx_t = s_t D_t + Ds dy_t;  dDs += dy_t x_t;  e_{t-1} = exp(D_t A) e_t.
//
// A thread holds 4 states of one channel, as in the forward.  The states themselves are found again
// from the marks that the forward left every 16 tokens, and kept in registers for the 16 tokens on
// the way back.  Sums over a channel's states go by shuffles; sums over channels (dB, dC) through
// shared memory, first within a warp for two tokens at a time, then over its warps once a tile,
// then over the blocks of a group in a kernel of its own: every order is fixed.
#include "flex_internal.h"
#include "ssm.cuh"

namespace flex {
namespace {

using namespace ssm;

// Channels of a block.
constexpr int channels(int L) { return L <= 4 ? 64 : 32; }

template <int L>
struct Smem {
    using C = Cfg<L, channels(L)>;
    static constexpr int WARPS = C::THREADS / 32, SPLIT = 8 / L, PARTS = WARPS * SPLIT;
    struct Tile {
        float2 td[kTile][C::CT];       // D_t, D_t x_t
        float dy[kTile][C::CT];
        float bc[kTile][2][C::N];
    } tiles[2];
    float sums[3][kTile][C::CT + 8];   // s_t, <q_t, A>, <C_t, h_t>
    float pair[WARPS][2][2][128];      // a warp's two tokens, dB and dC: [channel][N]
    float parts[PARTS][kTile][2][C::N];
};

template <typename T, int L>
__global__ void __launch_bounds__(channels(L) * L, 512 / (channels(L) * L))
ssm_bwd_kernel(SsmArgs a)
{
    using C = Cfg<L, channels(L)>;
    using S = Smem<L>;
    constexpr int N = C::N, CT = C::CT, NT = C::THREADS, PT = C::PT, PBC = C::PBC;
    constexpr int YB = L < 4 ? 4 : L;
    extern __shared__ __align__(16) unsigned char raw[];
    S& sm = *(S*)raw;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    Place p;
    const bool found = find_place<channels(L)>(a, blockIdx.x, p);
    const int ch = tid / L, sub = tid % L;
    const bool mine = ch < p.nc;
    const size_t DN = (size_t)a.D * N, state = (size_t)(p.c0 + ch) * N + 4 * sub;
    constexpr int CQ = CT / 4;
    const int q4 = 4 * (tid % CQ), tq = tid / CQ;
    const bool stages = tid < C::QUADS && q4 < p.nc;
    tc::grid_dep_wait();
    if (!found) {  // no rows, no gradients
        const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
        if (mine) *(float4*)(a.part_a + p.slot * DN + state) = zero;
        if (tid < CQ && q4 < p.nc)
            for (int k = 0; k < 2; ++k)
                *(float4*)(a.part_d + ((size_t)p.slot * 2 + k) * a.D + p.c0 + q4) = zero;
        return;
    }
    const int blocks = (p.hi - p.lo + a.rows - 1) / a.rows;
    F2x2 A2, e, dA;
    {
        const float4 v = mine ? *(const float4*)(a.A + state) : make_float4(0.f, 0.f, 0.f, 0.f);
        A2.from(make_float4(v.x * kLog2e, v.y * kLog2e, v.z * kLog2e, v.w * kLog2e));
        e.x = e.y = dA.x = dA.y = 0;
    }
    // the gradient of the state behind the block, from the blocks after it
    if (mine)
        for (int j = p.slot - p.block + blocks - 1; j > p.slot; --j) {
            const float sum = a.sums[(size_t)j * a.D + p.c0 + ch];
            const F2x2 w = decay(A2, tc::f2_pack(sum, sum));
            F2x2 v;
            v.from(*(const float4*)(a.ends + j * DN + state));
            e.x = tc::f2_fma(w.x, e.x, v.x);
            e.y = tc::f2_fma(w.y, e.y, v.y);
        }

    const T *x = (const T*)a.x, *dt = (const T*)a.dt, *z = (const T*)a.z, *dout = (const T*)a.dout;
    float4 bias = make_float4(0.f, 0.f, 0.f, 0.f), Ds = bias, dDs = bias, dbias = bias;
    if (stages) {
        if (a.bias) bias = *(const float4*)(a.bias + p.c0 + q4);
        if (a.Ds) Ds = *(const float4*)(a.Ds + p.c0 + q4);
    }
    const int nt = (p.last - p.first + kTile - 1) / kTile;

    struct Raw { Quad<T> x[PT], d[PT], z[PT], o[PT], bc[PBC]; } r;
    auto load = [&](int i) {
        const int t0 = p.first + i * kTile;
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const long long t = t0 + tq + k * (NT / CQ);
            r.x[k].zero(); r.z[k].zero(); r.o[k].zero();
            if (a.softplus) r.d[k].low(); else r.d[k].zero();  // a step of 0
            if (stages && t < p.last) {
                r.x[k].load(x + t * a.xs + p.c0 + q4);
                r.d[k].load(dt + t * a.ds + p.c0 + q4);
                r.o[k].load(dout + t * a.D + p.c0 + q4);
                if (z) r.z[k].load(z + t * a.zs + p.c0 + q4);
            }
        }
#pragma unroll
        for (int k = 0; k < PBC; ++k) {
            const int f = tid + k * NT, which = f / (C::BC / 2), i4 = f % (C::BC / 2);
            const long long t = t0 + i4 / L;
            r.bc[k].zero();
            if (f < C::BC && t < p.last) {
                const int at = p.g * N + 4 * (i4 % L);
                if (which == 0) r.bc[k].load((const T*)a.B + t * a.bs + at);
                else r.bc[k].load((const T*)a.C + t * a.cs + at);
            }
        }
    };
    auto put = [&](typename S::Tile& s) {
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const int tt = tq + k * (NT / CQ);
            if (tid >= C::QUADS) break;
            const float4 dv = r.d[k].get(), xv = r.x[k].get();
            float4 o = r.o[k].get();
            if (z) {
                const float4 g = r.z[k].get();
                o.x *= silu(g.x); o.y *= silu(g.y); o.z *= silu(g.z); o.w *= silu(g.w);
            }
            float d[4] = {dv.x + bias.x, dv.y + bias.y, dv.z + bias.z, dv.w + bias.w};
            if (a.softplus) softplus4(d);
            float4* to = (float4*)&s.td[tt][q4];
            to[0] = make_float4(d[0], d[0] * xv.x, d[1], d[1] * xv.y);
            to[1] = make_float4(d[2], d[2] * xv.z, d[3], d[3] * xv.w);
            *(float4*)&s.dy[tt][q4] = o;
        }
#pragma unroll
        for (int k = 0; k < PBC; ++k) {
            const int f = tid + k * NT, which = f / (C::BC / 2), i4 = f % (C::BC / 2);
            if (f < C::BC) *(float4*)&s.bc[i4 / L][which][4 * (i4 % L)] = r.bc[k].get();
        }
    };

    const float* marks = a.marks + ((size_t)(p.lo / kTile + p.s) + (p.first - p.lo) / kTile) * DN + state;
    load(nt - 1);
    F2x2 dAt;  // a tile's part, so that long sums are sums of sums
    for (int i = nt - 1; i >= 0; --i) {
        typename S::Tile& s = sm.tiles[i & 1];
        put(s);
        F2x2 h0;
        h0.from(mine ? *(const float4*)(marks + i * DN) : make_float4(0.f, 0.f, 0.f, 0.f));
        __syncthreads();
        dAt.x = dAt.y = 0;
        // the states again, and y
        F2x2 hh[kTile];
#pragma unroll
        for (int b = 0; b < kTile; b += YB) {
            float y[YB];
#pragma unroll
            for (int j = 0; j < YB; ++j) {
                const float2 td = s.td[b + j][ch];
                const F2x2 B = *(const F2x2*)&s.bc[b + j][0][4 * sub];
                const F2x2 w = decay(A2, tc::f2_pack(td.x, td.x)), &h = b + j ? hh[b + j - 1] : h0;
                const uint64_t dx = tc::f2_pack(td.y, td.y);
                hh[b + j].x = tc::f2_fma(w.x, h.x, tc::f2_mul(dx, B.x));
                hh[b + j].y = tc::f2_fma(w.y, h.y, tc::f2_mul(dx, B.y));
                if (z) y[j] = hh[b + j].dot(*(const F2x2*)&s.bc[b + j][1][4 * sub]);
            }
            if (z) {
#pragma unroll
                for (int j = 0; j < YB; j += L) {
                    float v[L];
#pragma unroll
                    for (int k = 0; k < L; ++k) v[k] = y[j + k];
                    sm.sums[2][b + j + sub][ch] = lane_sums<L>(v, sub);
                }
            }
        }
        // and back
#pragma unroll
        for (int b = kTile - YB; b >= 0; b -= YB) {
            float s1[YB], s2[YB];
#pragma unroll
            for (int j2 = YB - 2; j2 >= 0; j2 -= 2) {
#pragma unroll
                for (int j = j2 + 1; j >= j2; --j) {
                    const int t = b + j;
                    const float2 td = s.td[t][ch];
                    const float dyv = s.dy[t][ch];
                    const F2x2 B = *(const F2x2*)&s.bc[t][0][4 * sub];
                    const F2x2 Cv = *(const F2x2*)&s.bc[t][1][4 * sub];
                    const uint64_t dy = tc::f2_pack(dyv, dyv), dx = tc::f2_pack(td.y, td.y);
                    const uint64_t dd = tc::f2_pack(td.x, td.x);
                    F2x2 v;
                    v.x = tc::f2_mul(dy, hh[t].x);
                    v.y = tc::f2_mul(dy, hh[t].y);
                    *(F2x2*)&sm.pair[warp][t & 1][1][4 * lane] = v;
                    e.x = tc::f2_fma(dy, Cv.x, e.x);
                    e.y = tc::f2_fma(dy, Cv.y, e.y);
                    v.x = tc::f2_mul(dx, e.x);
                    v.y = tc::f2_mul(dx, e.y);
                    *(F2x2*)&sm.pair[warp][t & 1][0][4 * lane] = v;
                    s1[j] = e.dot(B);
                    const F2x2 w = decay(A2, dd);
                    e.x = tc::f2_mul(w.x, e.x);
                    e.y = tc::f2_mul(w.y, e.y);
                    const F2x2& h = t ? hh[t - 1] : h0;
                    v.x = tc::f2_mul(e.x, h.x);
                    v.y = tc::f2_mul(e.y, h.y);
                    s2[j] = v.dot(A2);
                    dAt.x = tc::f2_fma(dd, v.x, dAt.x);
                    dAt.y = tc::f2_fma(dd, v.y, dAt.y);
                }
                // Sums over the warp's channels for two tokens: 4 L groups of 4 values, of which a
                // lane adds those of 4 channels.  They are read in turn, since two groups' rows
                // start in the same bank.
                __syncwarp();
                {
                    const int group = lane % (4 * L), part = lane / (4 * L), k = group / L, m = group % L;
                    const float* from = &sm.pair[warp][k / 2][k % 2][4 * m];
                    F2x2 v = *(const F2x2*)(from + (4 * part + (k & 3)) * N);
#pragma unroll
                    for (int c = 1; c < 4; ++c) {
                        const F2x2 u = *(const F2x2*)(from + (4 * part + ((k + c) & 3)) * N);
                        v.x = tc::f2_fma(u.x, tc::f2_pack(1.f, 1.f), v.x);
                        v.y = tc::f2_fma(u.y, tc::f2_pack(1.f, 1.f), v.y);
                    }
                    *(F2x2*)&sm.parts[warp * S::SPLIT + part][b + j2 + k / 2][k % 2][4 * m] = v;
                }
                __syncwarp();
            }
#pragma unroll
            for (int j = 0; j < YB; j += L) {
                float v[L], u[L];
#pragma unroll
                for (int k = 0; k < L; ++k) { v[k] = s1[j + k]; u[k] = s2[j + k]; }
                sm.sums[0][b + j + sub][ch] = lane_sums<L>(v, sub);
                sm.sums[1][b + j + sub][ch] = lane_sums<L>(u, sub);
            }
        }
        __syncthreads();
        dA.x = tc::f2_fma(dAt.x, tc::f2_pack(1.f, 1.f), dA.x);
        dA.y = tc::f2_fma(dAt.y, tc::f2_pack(1.f, 1.f), dA.y);
        // the tile's gradients
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const int tt = tq + k * (NT / CQ);
            const long long t = p.first + i * kTile + tt;
            if (!stages || t >= p.last) continue;
            const float4 xq = r.x[k].get(), dq = r.d[k].get(), oq = r.o[k].get(), zq = r.z[k].get();
            const float xv[4] = {xq.x, xq.y, xq.z, xq.w};
            const float rv[4] = {dq.x + bias.x, dq.y + bias.y, dq.z + bias.z, dq.w + bias.w};
            const float ov[4] = {oq.x, oq.y, oq.z, oq.w}, zv[4] = {zq.x, zq.y, zq.z, zq.w};
            const float Dv[4] = {Ds.x, Ds.y, Ds.z, Ds.w};
            float gx[4], gd[4], gz[4], gD[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float s1 = sm.sums[0][tt][q4 + j], s2 = sm.sums[1][tt][q4 + j] * kLn2;
                const float dy = s.dy[tt][q4 + j], d = s.td[tt][q4 + j].x;
                gx[j] = fmaf(s1, d, Dv[j] * dy);
                gd[j] = fmaf(s1, xv[j], s2);
                if (a.softplus) gd[j] *= sigmoid(rv[j]);
                gD[j] = dy * xv[j];
                if (z) {
                    const float y = fmaf(Dv[j], xv[j], sm.sums[2][tt][q4 + j]), g = sigmoid(zv[j]);
                    gz[j] = ov[j] * y * g * fmaf(zv[j], 1.f - g, 1.f);
                }
            }
            dDs.x += gD[0]; dDs.y += gD[1]; dDs.z += gD[2]; dDs.w += gD[3];
            dbias.x += gd[0]; dbias.y += gd[1]; dbias.z += gd[2]; dbias.w += gd[3];
            const size_t at = t * a.D + p.c0 + q4;
            store4((T*)a.dx + at, make_float4(gx[0], gx[1], gx[2], gx[3]));
            store4((T*)a.ddt + at, make_float4(gd[0], gd[1], gd[2], gd[3]));
            if (z) store4((T*)a.dz + at, make_float4(gz[0], gz[1], gz[2], gz[3]));
        }
        for (int f = tid; f < kTile * 2 * L; f += NT) {  // groups of 4 values of dB and dC
            const int tt = f / (2 * L);
            const long long t = p.first + i * kTile + tt;
            const float* from = &sm.parts[0][0][0][0] + 4 * f;
            float4 v = *(const float4*)from;
#pragma unroll
            for (int k = 1; k < S::PARTS; ++k) {
                const float4 u = *(const float4*)(from + (size_t)k * kTile * 2 * N);
                v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
            }
            if (t < p.last)
                *(float4*)(a.part_bc + (((size_t)p.tile * a.T + t) * a.G + p.g) * 2 * N + 4 * (f % (2 * L))) = v;
        }
        if (i > 0) load(i - 1);
        __syncthreads();
    }
    if (mine) *(float4*)(a.part_a + p.slot * DN + state) = dA.get();
    // dDs and dbias: over the tokens of a tile, which NT / CQ threads hold
    constexpr int ROWS = C::QUADS / CQ / PT;
    if (tid < C::QUADS) {
        *(float4*)&sm.sums[0][tq][q4] = dDs;
        *(float4*)&sm.sums[1][tq][q4] = dbias;
    }
    __syncthreads();
    for (int f = tid; f < 2 * CT; f += NT) {
        const int k = f / CT, c = f % CT;
        if (c >= p.nc) continue;
        float v = 0.f;
#pragma unroll
        for (int j = 0; j < ROWS; ++j) v += sm.sums[k][j][c];
        a.part_d[((size_t)p.slot * 2 + k) * a.D + p.c0 + c] = v;
    }
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
    for (int j = 0; j < slots; ++j) {
        const float4 u = *(const float4*)(from + j * step);
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    *(float4*)to = v;
}

template <typename T, int L>
cudaError_t bwd(const SsmArgs& a, bool after, cudaStream_t s)
{
    const int slots = block_slots(a.T, a.n, a.rows), tiles = group_tiles(a, channels(L));
    auto kernel = ssm_bwd_kernel<T, L>;
    static_assert(sizeof(Smem<L>) <= 113 * 1024, "two blocks an SM");
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Smem<L>));
    if (e != cudaSuccess) return e;
    e = tc::launch_after(kernel, dim3((unsigned)((long long)slots * tiles * a.G)), channels(L) * L,
                         sizeof(Smem<L>), 0, after, s, a);
    if (e != cudaSuccess) return e;
    const long long bc = ((long long)a.T * a.G * 2 * a.N / 4 + 255) / 256;
    const long long par = (((long long)a.D * (a.N + 2)) / 4 + 255) / 256;
    return tc::launch_after(ssm_bwd_sum_kernel<T>, dim3((unsigned)(bc + par)), 256, 0, 0, true, s, a, tiles,
                            slots, bc);
}
template <typename T>
cudaError_t bwd_n(const SsmArgs& a, bool after, cudaStream_t s)
{
    switch (a.N) {
    case 8: return bwd<T, 2>(a, after, s);
    case 16: return bwd<T, 4>(a, after, s);
    default: return bwd<T, 8>(a, after, s);
    }
}

}  // namespace

int ssm_bwd_tiles(const SsmArgs& a) { return group_tiles(a, channels(a.N / 4)); }

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
