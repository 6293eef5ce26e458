// Selective state space scan, forward: whole sequences, and the single-token step.
//
// Channels and states are independent of one another but for y's sum over a channel's states, so a
// thread walks 4 states of one channel through the tokens with everything in registers; lanes of a
// channel add their y's up four tokens at a time.  What bounds it is arithmetic: per token and
// state one exponential and four multiplications or additions.
//
// Where sequences and channels leave SMs idle, sequences are cut into blocks of `rows` tokens.  A
// first kernel finds what each block's tokens leave behind by themselves and the sum of their
// steps, exp(A sum) being the decay over the whole block; the second starts every block from the
// ends ahead of it, joined in order.
#include "flex_internal.h"
#include "ssm.cuh"

namespace flex {
namespace {

using namespace ssm;

enum Mode { kOut, kEnds, kBack };

// One tile of tokens in shared memory.
template <int L, int MODE>
struct Tile {
    float2 td[kTile][Cfg<L>::CT];     // D_t, and D_t x_t (kBack: dy_t)
    float bc[kTile][2][Cfg<L>::N];    // B and C (kEnds: B, kBack: C)
};

// kOut: outputs, last states and marks.  kEnds: what a block leaves behind, without outputs.  kBack:
// the same of the gradient of the state, from the block's last token to its first:
// e_{t-1} = exp(D_t A) (e_t + dy_t C_t).
template <typename T, int L, int MODE>
__global__ void __launch_bounds__(Cfg<L>::THREADS) ssm_scan_kernel(SsmArgs a)
{
    using C = Cfg<L>;
    constexpr int N = C::N, CT = C::CT, NT = C::THREADS, PT = C::PT, PBC = C::PBC;
    constexpr int YB = L < 4 ? 4 / L * L : L;  // tokens whose y's are added up together
    __shared__ alignas(16) Tile<L, MODE> tiles[2];
    __shared__ alignas(16) float sy[MODE == kOut ? 2 : 1][MODE == kOut ? kTile : 1][CT + 8];
    const int tid = threadIdx.x;
    Place p;
    const bool found = find_place<L>(a, blockIdx.x, p);
    const int ch = tid / L, sub = tid % L;
    const bool mine = ch < p.nc;
    const size_t state = (size_t)(p.c0 + ch) * N + 4 * sub;  // within [D][N]
    const size_t DN = (size_t)a.D * N;
    // the kernel ahead left ends and sums; nothing is read of them before this
    tc::grid_dep_wait();
    if (!found) {
        if (MODE == kOut && a.h1 && p.block == 0 && p.lo == p.hi && mine)
            *(float4*)(a.h1 + p.s * DN + state) =
                a.h0 ? *(const float4*)(a.h0 + p.s * DN + state) : make_float4(0.f, 0.f, 0.f, 0.f);
        return;
    }
    const int blocks = (p.hi - p.lo + a.rows - 1) / a.rows;
    if (MODE == kEnds && p.block == blocks - 1) return;  // nothing comes after it
    if (MODE == kBack && p.block == 0) return;

    F2x2 A2, h;
    {
        float4 v = mine ? *(const float4*)(a.A + state) : make_float4(0.f, 0.f, 0.f, 0.f);
        A2.from(make_float4(v.x * kLog2e, v.y * kLog2e, v.z * kLog2e, v.w * kLog2e));
        v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (MODE != kBack && p.block == 0 && a.h0 && mine) {
            // h1 may be h0: of a sequence in several blocks the first kernel keeps a copy, in the
            // place of the last block's end, which nothing else takes
            float* copy = a.ends + (size_t)(p.slot + blocks - 1) * DN + state;
            v = *(const float4*)(MODE == kOut && blocks > 1 ? copy : a.h0 + p.s * DN + state);
            if (MODE == kEnds) *(float4*)copy = v;
        }
        h.from(v);
    }
    if (MODE == kOut && p.block > 0 && mine) {
        for (int j = p.slot - p.block; j < p.slot; ++j) {
            const float sum = a.sums[(size_t)j * a.D + p.c0 + ch];
            const F2x2 w = decay(A2, tc::f2_pack(sum, sum));
            F2x2 e;
            e.from(*(const float4*)(a.ends + j * DN + state));
            h.x = tc::f2_fma(w.x, h.x, e.x);
            h.y = tc::f2_fma(w.y, h.y, e.y);
        }
    }

    const T *x = (const T*)a.x, *dt = (const T*)a.dt, *z = (const T*)a.z, *dout = (const T*)a.dout;
    Quad<T> xr[2][PT], zr[2][PT], dr[PT], bcr[PBC];
    // a thread's groups of 4 channels: tokens tid / (CT / 4) + ..., channels 4 (tid % (CT / 4)) + ...
    constexpr int CQ = CT / 4;
    const int q4 = 4 * (tid % CQ), tq = tid / CQ;
    const bool stages = tid < C::QUADS && q4 < p.nc;
    float4 bias = make_float4(0.f, 0.f, 0.f, 0.f), Ds = bias;
    if (stages) {
        if (a.bias) bias = *(const float4*)(a.bias + p.c0 + q4);
        if (MODE == kOut && a.Ds) Ds = *(const float4*)(a.Ds + p.c0 + q4);
    }
    const int nt = (p.last - p.first + kTile - 1) / kTile;
    auto start = [&](int i) { return MODE == kBack ? p.first + (nt - 1 - i) * kTile : p.first + i * kTile; };
    auto load = [&](int i, Quad<T>(&xq)[PT], Quad<T>(&zq)[PT]) {
        const int t0 = start(i);
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const long long t = t0 + tq + k * (NT / CQ);
            xq[k].zero(); zq[k].zero(); dr[k].zero();
            if (stages && t < p.last) {
                dr[k].load(dt + t * a.ds + p.c0 + q4);
                if (MODE == kBack) xq[k].load(dout + t * a.D + p.c0 + q4);
                else xq[k].load(x + t * a.xs + p.c0 + q4);
                if (MODE != kEnds && z) zq[k].load(z + t * a.zs + p.c0 + q4);
            }
        }
#pragma unroll
        for (int k = 0; k < PBC; ++k) {
            const int e = tid + k * NT, which = e / (C::BC / 2), i4 = e % (C::BC / 2);
            const long long t = t0 + i4 / L;
            bcr[k].zero();
            if (e < C::BC && t < p.last) {
                const int at = p.g * N + 4 * (i4 % L);
                if (which == 0 && MODE != kBack) bcr[k].load((const T*)a.B + t * a.bs + at);
                if (which == 1 && MODE != kEnds) bcr[k].load((const T*)a.C + t * a.cs + at);
            }
        }
    };
    auto silu = [](float v) { return __fdividef(v, 1.f + __expf(-v)); };
    auto put = [&](int i, Tile<L, MODE>& s, const Quad<T>(&xq)[PT], const Quad<T>(&zq)[PT]) {
        const int t0 = start(i);
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const int tt = tq + k * (NT / CQ);
            if (tid >= C::QUADS) break;
            // a token that does not exist takes a step of 0: it changes nothing
            const bool in = stages && t0 + tt < p.last;
            const float4 r = dr[k].get();
            float4 v = xq[k].get();
            if (MODE == kBack && z) {
                const float4 g = zq[k].get();
                v.x *= silu(g.x); v.y *= silu(g.y); v.z *= silu(g.z); v.w *= silu(g.w);
            }
            float d[4] = {r.x + bias.x, r.y + bias.y, r.z + bias.z, r.w + bias.w};
            float u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                d[j] = in ? (a.softplus ? softplus(d[j]) : d[j]) : 0.f;
                if (MODE != kBack) u[j] *= d[j];
                if (!in) u[j] = 0.f;
            }
            float4* to = (float4*)&s.td[tt][q4];
            to[0] = make_float4(d[0], u[0], d[1], u[1]);
            to[1] = make_float4(d[2], u[2], d[3], u[3]);
        }
#pragma unroll
        for (int k = 0; k < PBC; ++k) {
            const int e = tid + k * NT, which = e / (C::BC / 2), i4 = e % (C::BC / 2);
            if (e < C::BC) *(float4*)&s.bc[i4 / L][which][4 * (i4 % L)] = bcr[k].get();
        }
    };
    auto finish = [&](int i, const Quad<T>(&xq)[PT], const Quad<T>(&zq)[PT]) {
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const int tt = tq + k * (NT / CQ);
            const long long t = start(i) + tt;
            if (!stages || t >= p.last) continue;
            float4 y = *(const float4*)&sy[i & 1][MODE == kOut ? tt : 0][q4];
            const float4 v = xq[k].get();
            y.x = fmaf(Ds.x, v.x, y.x); y.y = fmaf(Ds.y, v.y, y.y);
            y.z = fmaf(Ds.z, v.z, y.z); y.w = fmaf(Ds.w, v.w, y.w);
            if (z) {
                const float4 g = zq[k].get();
                y.x *= silu(g.x); y.y *= silu(g.y); y.z *= silu(g.z); y.w *= silu(g.w);
            }
            store4((T*)a.out + t * a.D + p.c0 + q4, y);
        }
    };

    float sum = 0.f;
    float* marks = MODE == kOut && a.marks && mine
        ? a.marks + ((size_t)(p.lo / kTile + p.s) + (p.first - p.lo) / kTile) * DN + state : nullptr;
    load(0, xr[0], zr[0]);
    put(0, tiles[0], xr[0], zr[0]);
    __syncthreads();
    auto body = [&](int i, auto par) {
        constexpr int P = decltype(par)::value;
        if (i + 1 < nt) load(i + 1, xr[P ^ 1], zr[P ^ 1]);
        if (marks) {
            *(float4*)marks = h.get();
            marks += DN;
        }
        const Tile<L, MODE>& s = tiles[P];
        if (MODE == kOut) {
#pragma unroll
            for (int b = 0; b < kTile; b += YB) {
                float y[YB];
#pragma unroll
                for (int j = 0; j < YB; ++j) {
                    const float2 td = s.td[b + j][ch];
                    const F2x2 B = *(const F2x2*)&s.bc[b + j][0][4 * sub];
                    const F2x2 Cv = *(const F2x2*)&s.bc[b + j][1][4 * sub];
                    const F2x2 w = decay(A2, tc::f2_pack(td.x, td.x));
                    const uint64_t dx = tc::f2_pack(td.y, td.y);
                    h.x = tc::f2_fma(w.x, h.x, tc::f2_mul(dx, B.x));
                    h.y = tc::f2_fma(w.y, h.y, tc::f2_mul(dx, B.y));
                    y[j] = h.dot(Cv);
                }
#pragma unroll
                for (int j = 0; j < YB; j += L) {
                    float v[L];
#pragma unroll
                    for (int k = 0; k < L; ++k) v[k] = y[j + k];
                    sy[P][b + j + sub][ch] = lane_sums<L>(v, sub);
                }
            }
        } else {
#pragma unroll 8
            for (int k = 0; k < kTile; ++k) {
                const int j = MODE == kBack ? kTile - 1 - k : k;
                const float2 td = s.td[j][ch];
                const F2x2 v = *(const F2x2*)&s.bc[j][MODE == kBack][4 * sub];
                const F2x2 w = decay(A2, tc::f2_pack(td.x, td.x));
                const uint64_t u = tc::f2_pack(td.y, td.y);
                if (MODE == kEnds) {
                    h.x = tc::f2_fma(w.x, h.x, tc::f2_mul(u, v.x));
                    h.y = tc::f2_fma(w.y, h.y, tc::f2_mul(u, v.y));
                } else {
                    h.x = tc::f2_mul(w.x, tc::f2_fma(u, v.x, h.x));
                    h.y = tc::f2_mul(w.y, tc::f2_fma(u, v.y, h.y));
                }
                sum += td.x;
            }
        }
        if (i + 1 < nt) put(i + 1, tiles[P ^ 1], xr[P ^ 1], zr[P ^ 1]);
        __syncthreads();
        if (MODE == kOut) finish(i, xr[P], zr[P]);
    };
    for (int i = 0; i < nt; i += 2) {
        body(i, std::integral_constant<int, 0>());
        if (i + 1 < nt) body(i + 1, std::integral_constant<int, 1>());
    }
    if (!mine) return;
    if (MODE == kOut) {
        if (a.h1 && p.last == p.hi) *(float4*)(a.h1 + p.s * DN + state) = h.get();
    } else {
        *(float4*)(a.ends + p.slot * DN + state) = h.get();
        if (sub == 0) a.sums[(size_t)p.slot * a.D + p.c0 + ch] = sum;
    }
}

// One token of every sequence.  Bound by the state, read and written once; a thread takes 4 states
// of a channel through several sequences, so that A is read once for them and their states' loads
// are in flight together.
constexpr int kSeqs = 4;
template <typename T, int L>
__global__ void __launch_bounds__(256) ssm_decode_kernel(SsmArgs a)
{
    constexpr int N = 4 * L;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(i / L), sub = (int)(i % L), s0 = blockIdx.y * kSeqs;
    const bool mine = c < a.D;
    const size_t DN = (size_t)a.D * N, state = (size_t)c * N + 4 * sub;
    const int g = mine ? c / (a.D / a.G) : 0;
    float4 h[kSeqs];
#pragma unroll
    for (int k = 0; k < kSeqs; ++k)
        if (mine && s0 + k < a.n) h[k] = *(const float4*)(a.h1 + (s0 + k) * DN + state);
    const unsigned lanes = __ballot_sync(0xffffffffu, mine);
    if (!mine) return;  // (the lanes of a channel go together)
    const float4 A = *(const float4*)(a.A + state);
    const float bias = a.bias ? a.bias[c] : 0.f, Ds = a.Ds ? a.Ds[c] : 0.f;
#pragma unroll
    for (int k = 0; k < kSeqs; ++k) {
        const long long t = s0 + k;
        if (t >= a.n) break;
        const float x = to_f32(((const T*)a.x)[t * a.xs + c]);
        float d = to_f32(((const T*)a.dt)[t * a.ds + c]) + bias;
        if (a.softplus) d = softplus(d);
        const float4 B = load4((const T*)a.B + t * a.bs + g * N + 4 * sub);
        const float4 C = load4((const T*)a.C + t * a.cs + g * N + 4 * sub);
        const float dx = d * x;
        float4 v = h[k];
        v.x = fmaf(expf(d * A.x), v.x, dx * B.x);
        v.y = fmaf(expf(d * A.y), v.y, dx * B.y);
        v.z = fmaf(expf(d * A.z), v.z, dx * B.z);
        v.w = fmaf(expf(d * A.w), v.w, dx * B.w);
        *(float4*)(a.h1 + t * DN + state) = v;
        float y = fmaf(v.x, C.x, v.y * C.y) + fmaf(v.z, C.z, v.w * C.w);
#pragma unroll
        for (int m = 1; m < L; m *= 2) y += __shfl_xor_sync(lanes, y, m);
        if (sub == 0) {
            y = fmaf(Ds, x, y);
            if (a.z) {
                const float z = to_f32(((const T*)a.z)[t * a.zs + c]);
                y *= z / (1.f + expf(-z));
            }
            from_f32(((T*)a.out)[t * a.D + c], y);
        }
    }
}

template <typename T, int L>
cudaError_t scan(const SsmArgs& a, int mode, bool after, cudaStream_t s)
{
    const long long blocks = (long long)block_slots(a.T, a.n, a.rows) * group_tiles(a) * a.G;
    auto kernel = mode == kOut ? ssm_scan_kernel<T, L, kOut>
                : mode == kEnds ? ssm_scan_kernel<T, L, kEnds> : ssm_scan_kernel<T, L, kBack>;
    return tc::launch_after(kernel, dim3((unsigned)blocks), Cfg<L>::THREADS, 0, 0, after, s, a);
}
template <typename T, int L>
cudaError_t decode(const SsmArgs& a, cudaStream_t s)
{
    const dim3 grid((unsigned)(((long long)a.D * L + 255) / 256), (unsigned)((a.n + kSeqs - 1) / kSeqs));
    return tc::launch_after(ssm_decode_kernel<T, L>, grid, 256, 0, 0, false, s, a);
}

template <typename T>
cudaError_t scan_n(const SsmArgs& a, int mode, bool after, cudaStream_t s)
{
    switch (a.N) {
    case 8: return scan<T, 2>(a, mode, after, s);
    case 16: return scan<T, 4>(a, mode, after, s);
    default: return scan<T, 8>(a, mode, after, s);
    }
}
template <typename T>
cudaError_t decode_n(const SsmArgs& a, cudaStream_t s)
{
    switch (a.N) {
    case 8: return decode<T, 2>(a, s);
    case 16: return decode<T, 4>(a, s);
    default: return decode<T, 8>(a, s);
    }
}

}  // namespace

// Sequences stay whole where their channels fill the SMs at 2 blocks each; else they are cut, so
// that as many blocks as that are there.
int ssm_rows(const SsmArgs& a, bool backward)
{
    const long long tiles = (long long)group_tiles(a) * a.G, want = 2LL * kSMs;
    if (!backward && a.n * tiles >= want) return a.T + 1;
    long long rows = (a.T * tiles + want - 1) / want;
    rows = (rows + 4 * kTile - 1) / (4 * kTile) * (4 * kTile);
    return rows > a.T ? a.T + 1 : (int)rows;
}

cudaError_t launch_ssm_fwd(const SsmArgs& a, cudaStream_t s)
{
    cudaError_t e = cudaSuccess;
    if (a.rows <= a.T) e = a.bf16 ? scan_n<__nv_bfloat16>(a, kEnds, false, s) : scan_n<float>(a, kEnds, false, s);
    if (e != cudaSuccess) return e;
    return a.bf16 ? scan_n<__nv_bfloat16>(a, kOut, a.rows <= a.T, s) : scan_n<float>(a, kOut, a.rows <= a.T, s);
}
cudaError_t launch_ssm_back_ends(const SsmArgs& a, cudaStream_t s)
{
    return a.bf16 ? scan_n<__nv_bfloat16>(a, kBack, false, s) : scan_n<float>(a, kBack, false, s);
}
cudaError_t launch_ssm_decode(const SsmArgs& a, cudaStream_t s)
{
    return a.bf16 ? decode_n<__nv_bfloat16>(a, s) : decode_n<float>(a, s);
}

}  // namespace flex
