// Selective state space scan, forward: whole sequences, and the single-token step.
//
// Channels and states are independent of one another but for y's sum over a channel's states, so a
// thread walks 4 states of each of 2 channels through the tokens with everything in registers; lanes
// of a channel add their y's up four tokens at a time.  Per token, channel and state that is one
// exponential (32 a clock and SM) and four multiplications or additions (128): 107 us for 8 x 4096
// tokens of 2048 channels of 16 states, 81 for their bytes.  Measured 386: 8.1 instructions a warp for
// 32 of them (steps, sums over lanes and what feeds them), 63% of the issue slots, and 2.1 wavefronts of
// shared memory, 63% of what an SM has.  1 channel a thread reads B and C twice as often (582 us), 4
// leave too few warps (531).
//
// Where sequences and channels leave SMs idle, sequences are cut into blocks of `rows` tokens.  A
// first kernel finds what each block's tokens leave behind by themselves and the sum of their
// steps, exp(A sum) being the decay over the whole block; a second joins these ends in order to the
// states that the blocks start from, and the third starts from them.
#include "flex_internal.h"
#include "ssm.cuh"

namespace flex {
namespace {

using namespace ssm;

enum Mode { kOut, kEnds, kBack };

// How a block's threads divide a tile of tokens.  A thread holds SP states of each of CH channels.
template <typename T, int N_, int CH, int SP, int CT_>
struct Layout {
    static constexpr int N = N_, CT = CT_, L = N / SP;
    static constexpr int WALK = CT / CH * L, BRING = 2 * CT;  // threads that walk, and that bring tiles
    static constexpr int QUADS = kTile * CT / 4, PT = QUADS / BRING;  // groups of 4 channels of a token
    static constexpr int BC = kTile * N / 2, PBC = (BC + BRING - 1) / BRING;  // of 4 values of B and C
    static constexpr int RING = 4;
    struct Raw {  // a tile as it lies in memory
        T x[kTile][CT], dt[kTile][CT], z[kTile][CT], bc[kTile][2][N];
    };
    struct Smem {
        Raw raw[RING];
        float2 td[2][kTile][CT];       // D_t, and D_t x_t (kBack: dy_t)
        float bc[2][kTile][2][N];      // B and C
        float y[2][kTile][CT + 8];
    };
};

// kOut: outputs, last states and marks.  kEnds: what a block leaves behind, without outputs.  kBack:
// the same of the gradient of the state, from the block's last token to its first:
// e_{t-1} = exp(D_t A) (e_t + dy_t C_t).
//
// Tiles of 16 tokens are copied to shared memory two ahead, their steps and inputs computed one
// ahead, once for all states; a tile's outputs are finished after the next block barrier, of which
// there is one a tile.  That is the second half of the threads' work: a walk's tokens follow one
// another, and few sequences leave few warps to hide it behind.
template <typename T, int N, int CH, int SP, int CT, int MODE, int MIN>
__global__ void __launch_bounds__(CT / CH * (N / SP) + 2 * CT, MIN) ssm_scan_kernel(SsmArgs a)
{
    using Y = Layout<T, N, CH, SP, CT>;
    constexpr int L = Y::L, NT = Y::BRING, PT = Y::PT, PBC = Y::PBC, CQ = CT / 4;
    extern __shared__ __align__(16) unsigned char smem[];
    typename Y::Smem& sm = *(typename Y::Smem*)smem;
    // some threads walk the tokens, the others bring them and take the outputs away
    const bool walks = threadIdx.x < Y::WALK;
    const int tid = walks ? threadIdx.x : threadIdx.x - Y::WALK;
    Place p;
    const bool found = find_place<CT>(a, blockIdx.x, p);
    const int ch = tid / L * CH, sub = tid % L;
    const bool mine = walks && ch < p.nc;  // (channels come in fours)
    const size_t state = (size_t)(p.c0 + ch) * N + SP * sub;  // within [D][N]; the next channel's + N
    const size_t DN = (size_t)a.D * N;
    // the kernel ahead left ends and sums; nothing is read of them before this
    tc::grid_dep_wait();
    if (!found) {
        if (MODE == kOut && a.h1 && p.block == 0 && p.lo == p.hi && mine) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                States<SP> v;
                v.zero();
                if (a.h0) v.read(a.h0 + p.s * DN + state + c * N);
                v.write(a.h1 + p.s * DN + state + c * N);
            }
        }
        return;
    }
    const int blocks = (p.hi - p.lo + a.rows - 1) / a.rows;
    if (MODE == kEnds && p.block == blocks - 1) return;  // nothing comes after it
    if (MODE == kBack && p.block == 0) return;

    States<SP> A2[CH], h[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        A2[c].zero();
        h[c].zero();
        if (!mine) continue;
        A2[c].read(a.A + state + c * N);
#pragma unroll
        for (int i = 0; i < SP / 2; ++i) A2[c].v[i] = tc::f2_mul(A2[c].v[i], twice(kLog2e));
        if (MODE == kOut && blocks > 1 && a.joined) h[c].read(a.ends + p.slot * DN + state + c * N);
        else if (MODE == kOut && a.h0) h[c].read(a.h0 + p.s * DN + state + c * N);
        if (MODE == kOut && p.block > 0 && !a.joined) {  // few blocks: each joins the ends ahead of it
            for (int j = p.slot - p.block; j < p.slot; j += 4) {
                States<SP> e[4];
                float sum[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    e[k].zero();
                    sum[k] = 0.f;
                    if (j + k >= p.slot) continue;
                    e[k].read(a.ends + (size_t)(j + k) * DN + state + c * N);
                    sum[k] = a.sums[(size_t)(j + k) * a.D + p.c0 + ch + c];
                }
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int i = 0; i < SP / 2; ++i)
                        if (j + k < p.slot)
                            h[c].v[i] = tc::f2_fma(ex2_pair(tc::f2_mul(A2[c].v[i], twice(sum[k]))), h[c].v[i], e[k].v[i]);
            }
        }
    }

    const int q4 = 4 * (tid % CQ), tq = tid / CQ;  // a thread's groups of channels: tokens tq + k NT / CQ
    const bool stages = q4 < p.nc;
    float4 bias = make_float4(0.f, 0.f, 0.f, 0.f), Ds = bias;
    if (stages) {
        if (a.bias) bias = *(const float4*)(a.bias + p.c0 + q4);
        if (MODE == kOut && a.Ds) Ds = *(const float4*)(a.Ds + p.c0 + q4);
    }
    const bool gate = MODE != kEnds && a.z;
    const int nt = (p.last - p.first + kTile - 1) / kTile;
    auto start = [&](int i) { return MODE == kBack ? p.first + (nt - 1 - i) * kTile : p.first + i * kTile; };
    // a thread's first groups in memory, and how far on the next ones and the next tile's are
    const long long t0 = (MODE == kBack ? p.first + (nt - 1) * kTile : p.first) + tq;
    const T* from[3] = {(const T*)a.dt + t0 * a.ds + p.c0 + q4,
                        MODE == kBack ? (const T*)a.dout + t0 * a.D + p.c0 + q4
                                      : (const T*)a.x + t0 * a.xs + p.c0 + q4,
                        (const T*)a.z + (gate ? t0 * a.zs + p.c0 + q4 : 0)};
    const long long per_row[3] = {a.ds, MODE == kBack ? (long long)a.D : a.xs, a.zs};
    auto fetch = [&](int i) {
        typename Y::Raw& r = sm.raw[i % Y::RING];
        const int t0 = start(i), left = p.last - t0;  // rows that exist, from the tile's first
        const long long tiles = MODE == kBack ? -i : i;
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const int tt = tq + k * (NT / CQ);
            const bool in = stages && tt < left;
            const long long row = in ? tiles * kTile + k * (NT / CQ) : 0;
            // (what is not read has a valid address too: the tensor's)
            copy_quad(&r.dt[tt][q4], in ? from[0] + row * per_row[0] : (const T*)a.dt, in);
            copy_quad(&r.x[tt][q4], in ? from[1] + row * per_row[1] : (const T*)a.dt, in);
            if (gate) copy_quad(&r.z[tt][q4], in ? from[2] + row * per_row[2] : (const T*)a.dt, in);
        }
#pragma unroll
        for (int k = 0; k < PBC; ++k) {
            const int e = tid + k * NT;
            if (Y::BC % NT && e >= Y::BC) break;
            const int which = e / (Y::BC / 2), i4 = e % (Y::BC / 2), tt = i4 / (N / 4), m = 4 * (i4 % (N / 4));
            const bool in = tt < left;
            const long long row = in ? t0 + tt : p.first;
            if (which == 0 && MODE != kBack) copy_quad(&r.bc[tt][0][m], (const T*)a.B + row * a.bs + p.g * N + m, in);
            if (which == 1 && MODE != kEnds) copy_quad(&r.bc[tt][1][m], (const T*)a.C + row * a.cs + p.g * N + m, in);
        }
    };
    auto convert = [&](int i) {
        const typename Y::Raw& r = sm.raw[i % Y::RING];
        const int t0 = start(i);
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const int tt = tq + k * (NT / CQ);
            Quad<T> dr, xr, zr;
            dr.load(&r.dt[tt][q4]);
            xr.load(&r.x[tt][q4]);
            // a token that does not exist takes a step of 0: it changes nothing
            if (a.softplus && !(stages && t0 + tt < p.last)) dr.low();
            float4 v = xr.get();
            const float4 w = dr.get();
            if (MODE == kBack && gate) {
                zr.load(&r.z[tt][q4]);
                const float4 g = zr.get();
                v.x *= silu(g.x); v.y *= silu(g.y); v.z *= silu(g.z); v.w *= silu(g.w);
            }
            float d[4] = {w.x + bias.x, w.y + bias.y, w.z + bias.z, w.w + bias.w};
            if (a.softplus) softplus4(d);
            else if (!(stages && t0 + tt < p.last)) d[0] = d[1] = d[2] = d[3] = 0.f;
            if (MODE != kBack) { v.x *= d[0]; v.y *= d[1]; v.z *= d[2]; v.w *= d[3]; }
            float4* to = (float4*)&sm.td[i & 1][tt][q4];
            const float4 lo = make_float4(d[0], v.x, d[1], v.y), hi = make_float4(d[2], v.z, d[3], v.w);
            const bool odd = tid / 4 % 2;  // (halves in turn: 8 lanes' 128 bytes are in 32 banks)
            to[odd] = odd ? hi : lo;
            to[!odd] = odd ? lo : hi;
        }
#pragma unroll
        for (int k = 0; k < PBC; ++k) {
            const int e = tid + k * NT;
            if (Y::BC % NT && e >= Y::BC) break;
            const int which = e / (Y::BC / 2), i4 = e % (Y::BC / 2), tt = i4 / (N / 4), m = 4 * (i4 % (N / 4));
            if (which != (MODE == kBack ? 0 : MODE == kEnds ? 1 : 2)) {
                Quad<T> v;
                v.load(&r.bc[tt][which][m]);
                *(float4*)&sm.bc[i & 1][tt][which][m] = v.get();
            }
        }
    };
    auto finish = [&](int i) {
        const typename Y::Raw& r = sm.raw[i % Y::RING];
#pragma unroll
        for (int k = 0; k < PT; ++k) {
            const int tt = tq + k * (NT / CQ);
            const long long t = start(i) + tt;
            if (!stages || t >= p.last) continue;
            float4 y = *(const float4*)&sm.y[i & 1][tt][q4];
            Quad<T> xr, zr;
            xr.load(&r.x[tt][q4]);
            const float4 v = xr.get();
            y.x = fmaf(Ds.x, v.x, y.x); y.y = fmaf(Ds.y, v.y, y.y);
            y.z = fmaf(Ds.z, v.z, y.z); y.w = fmaf(Ds.w, v.w, y.w);
            if (gate) {
                zr.load(&r.z[tt][q4]);
                const float4 g = zr.get();
                y.x *= silu(g.x); y.y *= silu(g.y); y.z *= silu(g.z); y.w *= silu(g.w);
            }
            store4((T*)a.out + t * a.D + p.c0 + q4, y);
        }
    };

    float sum[CH] = {};
    float* marks = MODE == kOut && a.marks && mine
        ? a.marks + ((size_t)(p.lo / kMark + p.s) + (p.first - p.lo) / kMark) * DN + state : nullptr;
    if (!walks) {
        fetch(0);
        copies_commit();
        if (nt > 1) fetch(1);
        copies_commit();
        copies_wait<1>();
        bring_barrier(NT);
        convert(0);
        for (int i = 0; i < nt; ++i) {
            copies_wait<0>();
            __syncthreads();  // tile i's steps are there, and i - 1's outputs
            if (i + 2 < nt) fetch(i + 2);
            copies_commit();
            if (MODE == kOut && i > 0) finish(i - 1);
            if (i + 1 < nt) convert(i + 1);
        }
        if (MODE == kOut) {
            __syncthreads();
            finish(nt - 1);
        }
        return;
    }
    for (int i = 0; i < nt; ++i) {
        __syncthreads();
        const float2(*td)[CT] = sm.td[i & 1];
        const float(*bc)[2][N] = sm.bc[i & 1];
        constexpr int YB = MODE == kOut && L > 2 ? L : 2;
#pragma unroll
        for (int b = 0; b < kTile; b += YB) {
            float y[CH][YB];
            // (a mark only where tokens are: the slot after a sequence's last is another's)
            if (b % kMark == 0 && marks && start(i) + b < p.last) {
#pragma unroll
                for (int c = 0; c < CH; ++c) h[c].write(marks + c * N);
                marks += DN;
            }
#pragma unroll
            for (int jj = 0; jj < YB; ++jj) {
                const int j = MODE == kBack ? kTile - 1 - b - jj : b + jj;
                States<SP> B, C;
                if (MODE != kBack) B.read(&bc[j][0][SP * sub]);
                if (MODE != kEnds) C.read(&bc[j][1][SP * sub]);
                float2 du[CH];
#pragma unroll
                for (int c = 0; c < CH; c += 2) {
                    const float4 v = *(const float4*)&td[j][ch + c];
                    du[c] = make_float2(v.x, v.y);
                    du[c + 1] = make_float2(v.z, v.w);
                }
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    const uint64_t d = twice(du[c].x), u = twice(du[c].y);
                    uint64_t acc = 0;
#pragma unroll
                    for (int i2 = 0; i2 < SP / 2; ++i2) {
                        const uint64_t w = ex2_pair(tc::f2_fma(A2[c].v[i2], d, twice(kUp)));
                        uint64_t& s = h[c].v[i2];
                        if (MODE == kBack) s = tc::f2_mul(w, tc::f2_fma(u, C.v[i2], s));
                        else s = tc::f2_fma(w, s, tc::f2_mul(u, B.v[i2]));
                        if (MODE == kOut) acc = i2 ? tc::f2_fma(s, C.v[i2], acc) : tc::f2_mul(s, C.v[i2]);
                    }
                    if (MODE == kOut) {
                        float lo, hi;
                        tc::f2_unpack(acc, lo, hi);
                        y[c][jj] = lo + hi;
                    } else {
                        sum[c] += du[c].x;
                    }
                }
            }
            if (MODE == kOut) {
#pragma unroll
                for (int j = 0; j < YB; j += L) {
                    float v[CH];
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        float x[L];
#pragma unroll
                        for (int k = 0; k < L; ++k) x[k] = y[c][j + k];
                        v[c] = lane_sums<L>(x, sub);
                    }
                    float* to = &sm.y[i & 1][b + j + sub][ch];
#pragma unroll
                    for (int c = 0; c < CH; c += 2) *(float2*)(to + c) = make_float2(v[c], v[c + 1]);
                }
            }
        }
    }
    if (MODE == kOut) __syncthreads();
    if (!mine) return;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        if (MODE == kOut) {
            if (a.h1 && p.last == p.hi) h[c].write(a.h1 + p.s * DN + state + c * N);
        } else {
            h[c].write(a.ends + p.slot * DN + state + c * N);
            if (sub == 0) a.sums[(size_t)p.slot * a.D + p.c0 + ch + c] = sum[c];
        }
    }
}

// Blocks' ends to what their walks start from, in their place: of every sequence in several blocks the
// states ahead of each (from S0), or (back) the gradients of the states behind each.  A thread takes 4
// states of a channel through a sequence's blocks, the loads of 8 of them in flight (16384 tokens, D 256,
// 256 blocks: 77 us, 111 where every block joined the ends ahead of it by itself; D 1280, 43 blocks of
// 8192 tokens: 107 either way).
constexpr int kJoin = 8;
template <bool BACK>
__global__ void __launch_bounds__(128) ssm_join_kernel(SsmArgs a)
{
    tc::grid_dep_wait();
    const long long i = ((long long)blockIdx.x * 128 + threadIdx.x) * 4;
    const size_t DN = (size_t)a.D * a.N;
    const int s = blockIdx.y, c = (int)(i / a.N);
    int lo, hi;
    seq_rows(a.cu, s, a.T, lo, hi);
    const int blocks = (hi - lo + a.rows - 1) / a.rows, first = lo / a.rows + s;
    if (blocks < 2 || c >= a.D) return;
    States<4> A2, h;
    A2.read(a.A + i);
#pragma unroll
    for (int k = 0; k < 2; ++k) A2.v[k] = tc::f2_mul(A2.v[k], twice(kLog2e));
    h.zero();
    if (!BACK && a.h0) h.read(a.h0 + s * DN + i);
    for (int j0 = 0; j0 < blocks; j0 += kJoin) {
        States<4> e[kJoin];
        float sum[kJoin];
#pragma unroll
        for (int k = 0; k < kJoin; ++k) {
            const int j = BACK ? blocks - 1 - j0 - k : j0 + k;
            e[k].zero();
            sum[k] = 0.f;
            if (j0 + k + 1 >= blocks) continue;  // (the last one's end is nobody's start)
            e[k].read(a.ends + (size_t)(first + j) * DN + i);
            sum[k] = a.sums[(size_t)(first + j) * a.D + c];
        }
#pragma unroll
        for (int k = 0; k < kJoin; ++k) {
            const int j = BACK ? blocks - 1 - j0 - k : j0 + k;
            if (j0 + k >= blocks) break;
            h.write(a.ends + (size_t)(first + j) * DN + i);
#pragma unroll
            for (int q = 0; q < 2; ++q)
                h.v[q] = tc::f2_fma(ex2_pair(tc::f2_mul(A2.v[q], twice(sum[k]))), h.v[q], e[k].v[q]);
        }
    }
}

// One token of every sequence.  Bound by the state, read and written once; a thread takes 4 states
// of a channel through several sequences, so that A is read once for them and their states' loads
// are in flight together.
constexpr int kSeqs = 4;
template <typename T, int L>
__global__ void __launch_bounds__(256, 4) ssm_decode_kernel(SsmArgs a)
{
    constexpr int N = 4 * L;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(i / L), sub = (int)(i % L), s0 = blockIdx.y * kSeqs;
    const bool mine = c < a.D;
    const size_t DN = (size_t)a.D * N, state = (size_t)c * N + 4 * sub;
    const int g = mine ? c / (a.D / a.G) : 0;
    const unsigned lanes = __ballot_sync(0xffffffffu, mine);
    if (!mine) return;  // (the lanes of a channel go together)
    float4 h[kSeqs];
    Quad<T> B[kSeqs], C[kSeqs];
    T x[kSeqs], d[kSeqs], z[kSeqs];
#pragma unroll
    for (int k = 0; k < kSeqs; ++k) {
        const long long t = min(s0 + k, a.n - 1);
        h[k] = *(const float4*)(a.h1 + t * DN + state);
        B[k].load((const T*)a.B + t * a.bs + g * N + 4 * sub);
        C[k].load((const T*)a.C + t * a.cs + g * N + 4 * sub);
        x[k] = ((const T*)a.x)[t * a.xs + c];
        d[k] = ((const T*)a.dt)[t * a.ds + c];
        if (a.z) z[k] = ((const T*)a.z)[t * a.zs + c];
    }
    float4 A2 = *(const float4*)(a.A + state);
    A2.x *= kLog2e; A2.y *= kLog2e; A2.z *= kLog2e; A2.w *= kLog2e;
    const float bias = a.bias ? a.bias[c] : 0.f, Ds = a.Ds ? a.Ds[c] : 0.f;
#pragma unroll
    for (int k = 0; k < kSeqs; ++k) {
        const long long t = s0 + k;
        if (t >= a.n) break;
        const float xv = to_f32(x[k]);
        float dv = to_f32(d[k]) + bias;
        if (a.softplus) dv = softplus(dv);
        const float4 Bv = B[k].get(), Cv = C[k].get();
        const float dx = dv * xv;
        float4 v = h[k];
        v.x = fmaf(ex2(dv * A2.x), v.x, dx * Bv.x);
        v.y = fmaf(ex2(dv * A2.y), v.y, dx * Bv.y);
        v.z = fmaf(ex2(dv * A2.z), v.z, dx * Bv.z);
        v.w = fmaf(ex2(dv * A2.w), v.w, dx * Bv.w);
        *(float4*)(a.h1 + t * DN + state) = v;
        float y = fmaf(v.x, Cv.x, v.y * Cv.y) + fmaf(v.z, Cv.z, v.w * Cv.w);
#pragma unroll
        for (int m = 1; m < L; m *= 2) y += __shfl_xor_sync(lanes, y, m);
        if (sub == 0) {
            y = fmaf(Ds, xv, y);
            if (a.z) y *= silu(to_f32(z[k]));
            from_f32(((T*)a.out)[t * a.D + c], y);
        }
    }
}

template <typename T, int N, int CH, int SP, int CT>
cudaError_t scan(const SsmArgs& a, int mode, bool after, cudaStream_t s)
{
    using Y = Layout<T, N, CH, SP, CT>;
    const long long blocks = (long long)block_slots(a.T, a.n, a.rows) * group_tiles(a, CT) * a.G;
    // Whole sequences: registers for loads ahead, which at 16 states leaves 2 blocks an SM; a few long
    // sequences do not fill those (8 x 4096, D 2048: 384 us, 406 at 3), and where more blocks wait it costs
    // little (64 x 512: 338 us, 330 at 3).  Blocks of sequences run 3 an SM (8192, D 1280: 107 us, 113 at
    // 2); in fp32 shared memory, 87 KB a block, holds 2 all the same, and 32 states' 384 threads 1.
    constexpr int MIN = N <= 16 ? 3 : 1;
    auto kernel = mode == kEnds ? ssm_scan_kernel<T, N, CH, SP, CT, kEnds, MIN>
                : mode == kBack ? ssm_scan_kernel<T, N, CH, SP, CT, kBack, MIN>
                : a.rows > a.T ? ssm_scan_kernel<T, N, CH, SP, CT, kOut, 1>
                               : ssm_scan_kernel<T, N, CH, SP, CT, kOut, MIN>;
    constexpr int bytes = sizeof(typename Y::Smem);
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return e;
    return tc::launch_after(kernel, dim3((unsigned)blocks), Y::WALK + Y::BRING, bytes, 0, after, s, a);
}
template <typename T>
cudaError_t scan_n(const SsmArgs& a, int mode, bool after, cudaStream_t s)
{
    switch (a.N) {
    case 8: return scan<T, 8, 2, 4, 64>(a, mode, after, s);
    case 16: return scan<T, 16, 2, 4, 64>(a, mode, after, s);
    default: return scan<T, 32, 2, 4, 64>(a, mode, after, s);
    }
}
template <typename T, int L>
cudaError_t decode(const SsmArgs& a, cudaStream_t s)
{
    const dim3 grid((unsigned)(((long long)a.D * L + 255) / 256), (unsigned)((a.n + kSeqs - 1) / kSeqs));
    return tc::launch_after(ssm_decode_kernel<T, L>, grid, 256, 0, 0, false, s, a);
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

// Sequences stay whole where their blocks fill the SMs (8 x 4096, D 2048: 390 us whole, 544 cut);
// else they are cut, so that there are 8 blocks an SM (8192, D 1280: 4 115 us, 8 107, 12 117).  The
// backward's are cut in any case: its walk is the longer one, and blocks of sequences of different
// lengths fill the SMs evenly (8 x 1024, D 2048, training: 2 an SM 533 us, 4 530, 8 502, 12 506).  Small
// batches: blocks of 64 tokens forward (2000, D 512: 23 us, of 32 29, more of them to join), of 32
// backward (600 tokens of three sequences, D 256, training: 33 us, of 64 42).
// The forward's rule sees how many sequences there are, empty ones among them, and not their lengths, which
// the host does not know: one far longer than the others then keeps few blocks busy (8192 tokens and four of
// 1, D 2048: 463 us, as 8196 tokens of one sequence, cut, 156; 25 documents of 1 to 5003 tokens 291 us, as
// many tokens in 8 of one length 158).
int ssm_rows(const SsmArgs& a, bool backward)
{
    const long long tiles = (long long)group_tiles(a, 64) * a.G, want = 8LL * kSMs;
    if (!backward && a.n * tiles >= kSMs) return a.T + 1;
    long long rows = (a.T * tiles + want - 1) / want;
    const int unit = backward ? 32 : 64;
    rows = (rows + unit - 1) / unit * unit;
    return rows > a.T ? a.T + 1 : (int)rows;
}

// Whether the ends are joined by a kernel of their own: not where no sequence can have more than 24 blocks
// (5 short prompts, 530 tokens, D 1024, captured: 17 us with it, 15 without), unless S1 is S0, which a
// sequence's last block may write before the others have read it.
bool ssm_joined(const SsmArgs& a) { return a.T / a.rows + 1 > 24 || (a.h0 && a.h0 == a.h1); }

static cudaError_t join(const SsmArgs& a, bool back, cudaStream_t s)
{
    const dim3 grid((unsigned)(((long long)a.D * a.N / 4 + 127) / 128), (unsigned)a.n);
    return tc::launch_after(back ? ssm_join_kernel<true> : ssm_join_kernel<false>, grid, 128, 0, 0, true, s, a);
}

cudaError_t launch_ssm_fwd(const SsmArgs& a, cudaStream_t s)
{
    const bool cut = a.rows <= a.T;
    if (cut) {
        cudaError_t e = a.bf16 ? scan_n<__nv_bfloat16>(a, kEnds, false, s) : scan_n<float>(a, kEnds, false, s);
        if (e == cudaSuccess && a.joined) e = join(a, false, s);
        if (e != cudaSuccess) return e;
    }
    return a.bf16 ? scan_n<__nv_bfloat16>(a, kOut, cut, s) : scan_n<float>(a, kOut, cut, s);
}
cudaError_t launch_ssm_back_ends(const SsmArgs& a, cudaStream_t s)
{
    const cudaError_t e = a.bf16 ? scan_n<__nv_bfloat16>(a, kBack, false, s) : scan_n<float>(a, kBack, false, s);
    return e != cudaSuccess ? e : join(a, true, s);
}
cudaError_t launch_ssm_decode(const SsmArgs& a, cudaStream_t s)
{
    return a.bf16 ? decode_n<__nv_bfloat16>(a, s) : decode_n<float>(a, s);
}

}  // namespace flex
