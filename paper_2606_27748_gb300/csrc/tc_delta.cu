// Gated delta rule on the tensor cores (bf16 storage, d 64 or 128), in chunks of 64 tokens.
//
// With G_i the sum of the log decays from the chunk's first token to token i, Y_ij = exp(G_i - G_j)
// for i >= j, and S the state ahead of the chunk, the recurrence over a chunk is the linear system
//   (I + L diag(beta)) E = R,  L = tril(Y o K K^T, -1),  R = V - e^G K S
// whose solution is E = R - M (beta R) with M = (I + L diag(beta))^-1 L, strictly lower; then
//   U = beta E,  O = scale e^G Q S + P U,  P = scale tril(Y o Q K^T),
//   S <- e^{G_C} S + (e^{G_C - G} K)^T U.
// M and P depend on no state: one kernel computes them for all chunks and heads at once.  A
// second one walks each (sequence, head)'s chunks with three dependent products a chunk; what
// bounds it is their latency, then the tensor cores.
//
// Everything of the walk is held transposed, a row of the state or of a chunk's E for one value
// dimension in one lane of tensor memory: S^T, R^T, U^T are then "A" operands in tensor memory
// that the threads write straight from registers, K, Q, M and P are "B" operands as they lie in
// shared memory (read along their rows or across them), and no operand is ever transposed.
// For d = 64 the lower 64 of the 128 lanes carry the state; the others compute on whatever they hold.
//
// Precision: K and Q are exact.  What multiplies them on the way of the state (S, beta R, U, and
// M) is split into bf16 high and low parts (2^-17), so that the state, held in fp32 registers, is
// accurate to fp32's order.  The output's own products take S, U and P as bf16: it is rounded to
// bf16 anyway.
#include <cuda.h>

#include "flex_internal.h"
#include "packed.cuh"
#include "tc_util.cuh"

namespace flex {
namespace {

using namespace tc;

constexpr int kC = 64;             // tokens of a chunk
constexpr float kLog2e = 1.4426950408889634f;
// A log decay of -88 is exp(-88) = 6e-39, no factor in fp32 sums; -inf is taken as that, since
// the differences of the sums G have to be finite.
constexpr float kLeastGate = -88.f;

// What the walk needs of a chunk, as it is copied to shared memory: M's high and low parts and P
// (64 x 64 bf16, 128-byte rows, swizzled), then e^G, e^{G_C - G}, beta (64 floats each; 0 behind
// the sequence's end) and e^{G_C}.
struct Rec {
    static constexpr uint32_t M_HI = 0, M_LO = 8192, P = 16384, AUX = 24576, BYTES = 25600;
    static constexpr uint32_t GAMMA = AUX, KAPPA = AUX + 256, BETA = AUX + 512, LAST = AUX + 768;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// (a, b) as bf16 pairs hi + lo.
__device__ __forceinline__ void split(float a, float b, uint32_t& hi, uint32_t& lo)
{
    hi = pack_bf16(a, b);
    lo = pack_bf16(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xffff0000u));
}

__device__ __forceinline__ uint64_t adv(uint64_t d, uint32_t bytes) { return d + (bytes >> 4); }

// ---- M, P and the gates' factors of every chunk ------------------------------------------
// One CTA of 128 threads per (chunk, head).  [K; Q] K^T is one tcgen05 product of 128 rows: rows
// 0-63 (threads 0-63) K K^T, rows 64-127 Q K^T.  The system is solved in fp32: the two diagonal
// blocks of 32 by forward substitution, a thread per column with the column in registers; then
// the block below, M21 = X - M22 (beta X) with X = L21 - L21 (beta M11), by all threads.
struct PrepSmem {
    float L[64][68];  // over the operand tiles, once the product is done
    float M[64][68];  // columns 32-63 of rows 0-31 hold X
};

template <int D>
__global__ void __launch_bounds__(128)
    delta_prep_kernel(const __grid_constant__ CUtensorMap tmap_q,
                      const __grid_constant__ CUtensorMap tmap_k, Packed pk,
                      const __nv_bfloat16* __restrict__ g, const __nv_bfloat16* __restrict__ beta,
                      const int* __restrict__ cu, float scale, uint8_t* rec, int* status)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t sb = smem_u32(sm);
    PrepSmem& w = *reinterpret_cast<PrepSmem*>(sm);
    __shared__ uint64_t bar_load, bar_mma;
    __shared__ uint32_t tmem_base_sh;
    __shared__ volatile int abort_flag;
    __shared__ __align__(16) float Gs[64], Bs[64];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, h = blockIdx.y;
    int s, chunk, lo, hi;
    if (!find_block(cu, pk.n, pk.T, kC, (int)blockIdx.x, s, chunk, lo, hi)) return;
    const int t0 = lo + chunk * kC, n = min(kC, hi - t0), hk = h / (pk.H / pk.Hk);
    if (tid == 0) {
        mbar_init(&bar_load, 1);
        mbar_init(&bar_mma, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(&tmem_base_sh, 64);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tm = tmem_base_sh;
    bool ok = true;
    if (warp == 0) {
        wmbar_arrive_expect_tx(&bar_load, 2 * kC * D * 2);
        for (int b = 0; b < D / 64; ++b) {
            wtma_load_3d(sb + b * 16384, &tmap_k, 64 * b, hk, t0, &bar_load);
            wtma_load_3d(sb + b * 16384 + 8192, &tmap_q, 64 * b, hk, t0, &bar_load);
        }
    }
    if (warp == 1) {  // sums of the gates, two tokens a lane
        float a[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * lane + i;
            const size_t at = (size_t)(t0 + j) * pk.H + h;
            a[i] = j < n ? fmaxf(__bfloat162float(g[at]), kLeastGate) * kLog2e : 0.f;
            Bs[j] = j < n ? __bfloat162float(beta[at]) : 0.f;
        }
        float sum = a[0] + a[1];
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const float o = __shfl_up_sync(0xffffffffu, sum, m);
            if (lane >= m) sum += o;
        }
        float before = __shfl_up_sync(0xffffffffu, sum, 1);
        if (lane == 0) before = 0.f;
        Gs[2 * lane] = before + a[0];
        Gs[2 * lane + 1] = sum;
    }
    if (warp == 0) {
        ok = bar_wait_w(&bar_load, 0, &abort_flag, status);
        if (ok) {
            constexpr uint32_t I = idesc_bf16(128, kC, 0, 0);
            const uint64_t d = sdesc(sb, 16, 1024);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const uint32_t o = (ks >> 2) * 16384 + (ks & 3) * 32;
                wmma_bf16(tm, adv(d, o), adv(d, o), I, ks > 0);
            }
            wmma_commit(&bar_mma);
        }
    }
    __syncthreads();
    ok = bar_wait_w(&bar_mma, 0, &abort_flag, status);
    if (!__syncthreads_and(ok)) {  // (also: the operand tiles may be overwritten from here on)
        drain_after_abort(true);
        if (warp == 0) tmem_dealloc(tm, 64);
        return;
    }
    fence_after_sync();
    rec += ((size_t)blockIdx.x * pk.H + h) * Rec::BYTES;
    const int row = tid & 63;
    {
        float v[64];
        const uint32_t ta = tm + ((uint32_t)warp << 21);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x[16];
            tmem_ld16(ta + 16 * i, x);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[16 * i + e] = x[e];
        }
        tmem_wait_ld();
        const float G = Gs[row];
        if (tid < 64) {  // L, rows behind the end zero (and with them columns: beta is 0 there)
#pragma unroll
            for (int j = 0; j < 64; j += 4) {
                float4 x;
                float* y = &x.x;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    y[e] = j + e < row && row < n ? v[j + e] * ex2(G - Gs[j + e]) : 0.f;
                *(float4*)&w.L[row][j] = x;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 64; j += 8) {
                float p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    p[e] = j + e <= row && row < n ? scale * v[j + e] * ex2(G - Gs[j + e]) : 0.f;
                *(uint4*)(rec + Rec::P + swz128(row, j)) =
                    make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]), pack_bf16(p[4], p[5]),
                               pack_bf16(p[6], p[7]));
            }
            const float last = Gs[63];
            float* aux = (float*)rec;
            aux[Rec::GAMMA / 4 + row] = ex2(G);
            aux[Rec::KAPPA / 4 + row] = row < n ? ex2(last - G) : 0.f;
            aux[Rec::BETA / 4 + row] = Bs[row];
            if (row == 0) aux[Rec::LAST / 4] = ex2(last);
        }
    }
    __syncthreads();
    if (tid < 64) {  // column `lane` of diagonal block `warp`: x_i = L_ic - sum_k L_ik beta_k x_k
        const int b = 32 * warp;
        float y[32];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            float a[4] = {};
#pragma unroll
            for (int k = 0; k < i; k += 4) {
                const float4 l = *(const float4*)&w.L[b + i][b + k];
                a[0] = fmaf(l.x, y[k], a[0]);
                if (k + 1 < i) a[1] = fmaf(l.y, y[k + 1], a[1]);
                if (k + 2 < i) a[2] = fmaf(l.z, y[k + 2], a[2]);
                if (k + 3 < i) a[3] = fmaf(l.w, y[k + 3], a[3]);
            }
            const float x = i > lane ? w.L[b + i][b + lane] - ((a[0] + a[1]) + (a[2] + a[3])) : 0.f;
            w.M[b + i][b + lane] = x;
            y[i] = Bs[b + i] * x;
        }
    }
    __syncthreads();
    const int i0 = 2 * (tid >> 3), j0 = 4 * (tid & 7);  // 2 rows x 4 columns of the block below
    auto below = [&](const float (*a)[68], int acol, const float (*x)[68], int xcol, int brow,
                     float4 (&out)[2]) {  // out = sum_k a[i0 + r][acol + k] beta[brow + k] x[k][xcol + j0 ..]
        out[0] = out[1] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
        for (int k = 0; k < 32; k += 4) {
            float4 l[2], m[4];
            const float4 bt = *(const float4*)&Bs[brow + k];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                l[r] = *(const float4*)&a[i0 + r][acol + k];
                l[r].x *= bt.x; l[r].y *= bt.y; l[r].z *= bt.z; l[r].w *= bt.w;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) m[e] = *(const float4*)&x[k + e][xcol + j0];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                out[r].x = fmaf(l[r].w, m[3].x, fmaf(l[r].z, m[2].x, fmaf(l[r].y, m[1].x, fmaf(l[r].x, m[0].x, out[r].x))));
                out[r].y = fmaf(l[r].w, m[3].y, fmaf(l[r].z, m[2].y, fmaf(l[r].y, m[1].y, fmaf(l[r].x, m[0].y, out[r].y))));
                out[r].z = fmaf(l[r].w, m[3].z, fmaf(l[r].z, m[2].z, fmaf(l[r].y, m[1].z, fmaf(l[r].x, m[0].z, out[r].z))));
                out[r].w = fmaf(l[r].w, m[3].w, fmaf(l[r].z, m[2].w, fmaf(l[r].y, m[1].w, fmaf(l[r].x, m[0].w, out[r].w))));
            }
        }
    };
    float4 acc[2], X[2];
    below(w.L + 32, 0, w.M, 0, 0, acc);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const float4 l = *(const float4*)&w.L[32 + i0 + r][j0];
        X[r] = make_float4(l.x - acc[r].x, l.y - acc[r].y, l.z - acc[r].z, l.w - acc[r].w);
        *(float4*)&w.M[i0 + r][32 + j0] = X[r];
    }
    __syncthreads();
    below(w.M + 32, 32, w.M, 32, 32, acc);
#pragma unroll
    for (int r = 0; r < 2; ++r)
        *(float4*)&w.M[32 + i0 + r][j0] = make_float4(X[r].x - acc[r].x, X[r].y - acc[r].y,
                                                      X[r].z - acc[r].z, X[r].w - acc[r].w);
    __syncthreads();
    for (int e = tid; e < 64 * 8; e += 128) {
        const int i = e >> 3, j = (e & 7) * 8;
        uint32_t mh[4], ml[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int a = j + 2 * c;
            split(a < i ? w.M[i][a] : 0.f, a + 1 < i ? w.M[i][a + 1] : 0.f, mh[c], ml[c]);
        }
        *(uint4*)(rec + Rec::M_HI + swz128(i, j)) = make_uint4(mh[0], mh[1], mh[2], mh[3]);
        *(uint4*)(rec + Rec::M_LO + swz128(i, j)) = make_uint4(ml[0], ml[1], ml[2], ml[3]);
    }
    if (warp == 0) tmem_dealloc(tm, 64);
}

// ---- the walk over a sequence's chunks ---------------------------------------------------

template <int D>
struct Walk {
    static constexpr int THREADS = 448;
    static constexpr int WARPS = D == 128 ? 8 : 4;  // computing warps (lanes of tensor memory in use)
    static constexpr int EPI = D == 128 ? 4 : 2;    // output warps
    static constexpr uint32_t TILE = kC * D * 2;    // 64 rows of K, Q or V
    static constexpr uint32_t K = 0, Q = TILE, V = 2 * TILE, REC = 3 * TILE;
    static constexpr uint32_t STAGE = (REC + Rec::BYTES + 1023) / 1024 * 1024;
    static constexpr int ST = D == 128 ? 3 : 4;
    static constexpr uint32_t SMEM = ST * STAGE + 1024;
    // tensor memory columns: S high, low; the chunk's product (K S, then M (beta R), then P U);
    // beta R, then kappa U, high and low; U; the state's increment; Q S
    static constexpr int T_SH = 0, T_SL = D / 2, T_X = D, T_AH = D + 64, T_AL = D + 96, T_U = D + 128,
                         T_D = D + 160, T_Q = 2 * D + 160;
    static_assert(2 * D + 224 <= 512, "tensor memory");
};
constexpr int kWalkMma = 12, kWalkTma = 13;

struct WalkArgs {
    Packed p;
    const int* cu;
    float scale;
    const float* S0;
    float* S1;
    __nv_bfloat16* out;
    const uint8_t* rec;
    __nv_bfloat16 *e_save, *s_save;  // NULL, or E^T [slot][H][d][64] and S^T [slot][H][d][d] of each chunk
    int* status;
};

// Warps 0-7 (d = 64: 0, 1, 4, 5) compute: quadrant w % 4 of the lanes, half w / 4 of the tokens
// (R, U) or of the state's columns, whose fp32 master they hold in registers.  Warps 8-11 (8, 9)
// write the output, 12 issues the products, 13 loads.  A chunk:
//   compute  S += last chunk's increment; S high, low -> tensor memory            (s_ready)
//   issue    X = K S                                                              (x_full)
//   compute  R = V - e^G X; beta R high, low                                      (r_ready)
//   issue    X = M (beta R)                                                       (e_full)
//   compute  E = R - X, U = beta E; e^{G_C - G} U high, low; U                    (u_ready)
//   issue    increment = (e^{G_C - G} U) K (s_full), then X = P U                 (o_full)
//   output   scale e^G (Q S) + P U                                                (o_free)
template <int D>
__global__ void __launch_bounds__(Walk<D>::THREADS, 1)
    delta_walk_kernel(const __grid_constant__ CUtensorMap tmap_q,
                      const __grid_constant__ CUtensorMap tmap_k,
                      const __grid_constant__ CUtensorMap tmap_v, WalkArgs x)
{
    using W = Walk<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = reinterpret_cast<uint8_t*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    const uint32_t sb = smem_u32(sm);
    __shared__ uint64_t full[W::ST], empty[W::ST], s_ready, x_full, r_ready, e_full, u_ready, s_full,
        o_full, o_free;
    __shared__ uint32_t tmem_base_sh;
    __shared__ volatile int abort_flag;

    const Packed& pk = x.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.x % pk.H, s = blockIdx.x / pk.H, hk = h / (pk.H / pk.Hk);
    int lo, hi;
    seq_rows(x.cu, s, pk.T, lo, hi);
    const int chunks = (hi - lo + kC - 1) / kC;
    const size_t rec0 = ((size_t)(lo / kC + s)) * pk.H + h;  // of chunk 0; pk.H further for each

    if (tid == 0) {
        for (int i = 0; i < W::ST; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], W::WARPS + W::EPI + 1);
        }
        mbar_init(&s_ready, W::WARPS);
        mbar_init(&r_ready, W::WARPS);
        mbar_init(&u_ready, W::WARPS);
        mbar_init(&o_free, W::EPI);
        mbar_init(&x_full, 1);
        mbar_init(&e_full, 1);
        mbar_init(&s_full, 1);
        mbar_init(&o_full, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == kWalkMma) {
        tmem_alloc(&tmem_base_sh, 512);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tm = tmem_base_sh;
    auto stage = [&](int c) { return (uint32_t)(c % W::ST) * W::STAGE; };
    auto landed = [&](int c) {
        return bar_wait_w(&full[c % W::ST], (uint32_t)(c / W::ST) & 1, &abort_flag, x.status);
    };

    if (warp == kWalkTma) {
        grid_dep_wait();  // the records
        for (int c = 0; c < chunks; ++c) {
            uint64_t* bar = &full[c % W::ST];
            if (c >= W::ST &&
                !bar_wait_w(&empty[c % W::ST], (uint32_t)(c / W::ST - 1) & 1, &abort_flag, x.status))
                break;
            const uint32_t st = sb + stage(c);
            const int t = lo + c * kC;
            wmbar_arrive_expect_tx(bar, 3 * W::TILE + Rec::BYTES);
            for (int b = 0; b < D / 64; ++b) {
                wtma_load_3d(st + W::K + 8192 * b, &tmap_k, 64 * b, hk, t, bar);
                wtma_load_3d(st + W::V + 8192 * b, &tmap_v, 64 * b, h, t, bar);
                wtma_load_3d(st + W::Q + 8192 * b, &tmap_q, 64 * b, hk, t, bar);
            }
            if (elect_one())
                bulk_load(st + W::REC, x.rec + (rec0 + (size_t)c * pk.H) * Rec::BYTES, Rec::BYTES, bar);
        }
    } else if (warp == kWalkMma) {
        constexpr uint32_t I_C = idesc_bf16(128, kC, 0, 0), I_D = idesc_bf16(128, D, 0, 1);
        bool ok = true;
        auto wait = [&](uint64_t* bar, int phase) {
            if (ok) ok = bar_wait_w(bar, (uint32_t)phase & 1, &abort_flag, x.status);
            fence_after_sync();
        };
        for (int c = 0; c < chunks && ok; ++c) {
            const uint32_t st = sb + stage(c);
            const int n = hi - lo - c * kC;
            ok = landed(c);
            if (!ok) break;
            if (n < kC) {  // K behind the sequence's end is another's, and 0 * NaN is NaN
                for (int e = n * 8 + lane; e < kC * 8; e += 32)
                    for (int b = 0; b < D / 64; ++b)
                        st_shared_v4(st + W::K + 8192 * b + e * 16, 0, 0, 0, 0);
                fence_proxy_async();
                __syncwarp();
            }
            const uint64_t dk = sdesc(st + W::K, 16, 1024), dq = sdesc(st + W::Q, 16, 1024);
            const uint64_t dkn = sdesc(st + W::K, 8192, 1024);
            const uint64_t dmh = sdesc(st + W::REC + Rec::M_HI, 16, 1024);
            const uint64_t dml = sdesc(st + W::REC + Rec::M_LO, 16, 1024);
            const uint64_t dp = sdesc(st + W::REC + Rec::P, 16, 1024);
            if (c > 0) wait(&o_free, c - 1);  // X and Q S of the last chunk have been read
            wait(&s_ready, c);
            if (!ok) break;
#pragma unroll
            for (int ks = 0; ks < D / 8; ++ks) {
                const int k = ks % (D / 16);
                wmma_bf16_tmem_a(tm + W::T_X, tm + (ks < D / 16 ? W::T_SH : W::T_SL) + 8 * k,
                                 adv(dk, (k >> 2) * 8192 + (k & 3) * 32), I_C, ks > 0);
            }
            wmma_commit(&x_full);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                wmma_bf16_tmem_a(tm + W::T_Q, tm + W::T_SH + 8 * k,
                                 adv(dq, (k >> 2) * 8192 + (k & 3) * 32), I_C, k > 0);
            wait(&r_ready, c);
            if (!ok) break;
#pragma unroll
            for (int ks = 0; ks < 12; ++ks) {  // high high, low high, high low
                const int k = ks & 3;
                wmma_bf16_tmem_a(tm + W::T_X, tm + (ks >> 2 == 1 ? W::T_AL : W::T_AH) + 8 * k,
                                 adv(ks >> 2 == 2 ? dml : dmh, k * 32), I_C, ks > 0);
            }
            wmma_commit(&e_full);
            wait(&u_ready, c);
            if (!ok) break;
#pragma unroll
            for (int ks = 0; ks < 8; ++ks)
                wmma_bf16_tmem_a(tm + W::T_D, tm + (ks < 4 ? W::T_AH : W::T_AL) + 8 * (ks & 3),
                                 adv(dkn, (ks & 3) * 2048), I_D, ks > 0);
            wmma_commit(&s_full);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                wmma_bf16_tmem_a(tm + W::T_X, tm + W::T_U + 8 * k, adv(dp, k * 32), I_C, k > 0);
            wmma_commit(&o_full);
            wmma_commit(&empty[c % W::ST]);
        }
    } else if (warp >= 8 && (warp & 3) < W::EPI) {
        // ---- output rows ----
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const int v = 32 * (warp & 3) + lane;
        const size_t os = (size_t)pk.H * D;
        __nv_bfloat16* out = x.out + (size_t)(lo + (lane & 1)) * os + h * D + (v & ~1);
        for (int c = 0; c < chunks; ++c) {
            const float* gamma = (const float*)(sm + stage(c) + W::REC + Rec::GAMMA);
            if (!landed(c)) break;
            if (!bar_wait_w(&o_full, (uint32_t)c & 1, &abort_flag, x.status)) break;
            fence_after_sync();
            const int n = min(kC, hi - lo - c * kC);
            float o[kC];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float a[16], b[16];
                tmem_ld16(tm + lanes + W::T_Q + 16 * i, a);
                tmem_ld16(tm + lanes + W::T_X + 16 * i, b);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) o[16 * i + e] = fmaf(x.scale * gamma[16 * i + e], a[e], b[e]);
            }
            fence_before_sync();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&o_free);
                mbar_arrive(&empty[c % W::ST]);
            }
            // neighbouring lanes exchange halves of two rows: each writes two elements of one row
#pragma unroll
            for (int i = 0; i < kC; i += 2) {
                const float other = __shfl_xor_sync(0xffffffffu, lane & 1 ? o[i] : o[i + 1], 1);
                const uint32_t w = lane & 1 ? pack_bf16(other, o[i + 1]) : pack_bf16(o[i], other);
                if (i + (lane & 1) < n) *(uint32_t*)(out + (size_t)(c * kC + i) * os) = w;
            }
        }
    } else if (warp < 8 && (warp & 3) < W::EPI) {
        // ---- the state ----
        const int half = warp >> 2, v = 32 * (warp & 3) + lane;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const uint32_t vcol = (uint32_t)(v >> 6) * 8192;
        constexpr int N = D / 2;  // columns of the state a thread holds
        float S[N];
        const size_t at = ((size_t)s * pk.H + h) * D * D + (size_t)half * N * D + v;
#pragma unroll
        for (int i = 0; i < N; ++i) S[i] = x.S0 ? x.S0[at + (size_t)i * D] : 0.f;
        float decay = 1.f;
        bool ok = true;
        auto increment = [&](int c) {  // S = decay S + the increment of chunk c
            ok = bar_wait_w(&s_full, (uint32_t)c & 1, &abort_flag, x.status);
            fence_after_sync();
#pragma unroll
            for (int i = 0; i < N / 16; ++i) {
                float d[16];
                tmem_ld16(tm + lanes + W::T_D + half * N + 16 * i, d);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) S[16 * i + e] = fmaf(decay, S[16 * i + e], d[e]);
            }
        };
        auto ready = [&](uint64_t* bar) {
            tmem_wait_st();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        for (int c = 0; c < chunks; ++c) {
            if (c > 0) increment(c - 1);
            if (!ok) break;
#pragma unroll
            for (int i = 0; i < N / 32; ++i) {
                uint32_t wh[16], wl[16];
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    split(S[32 * i + 2 * e], S[32 * i + 2 * e + 1], wh[e], wl[e]);
                tmem_st16(tm + lanes + W::T_SH + half * (N / 2) + 16 * i, wh);
                tmem_st16(tm + lanes + W::T_SL + half * (N / 2) + 16 * i, wl);
                if (x.s_save) {
                    uint4* dst = (uint4*)(x.s_save + ((rec0 + (size_t)c * pk.H) * D + v) * D + half * N + 32 * i);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        dst[e] = make_uint4(wh[4 * e], wh[4 * e + 1], wh[4 * e + 2], wh[4 * e + 3]);
                }
            }
            ready(&s_ready);
            if (!(ok = landed(c))) break;
            const uint8_t* st = sm + stage(c);
            const float* aux = (const float*)(st + W::REC) + 32 * half;
            const int n = hi - lo - c * kC - 32 * half;
            float R[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const uint32_t r = 32 * half + i;
                R[i] = __uint_as_float((uint32_t) * (const uint16_t*)(st + W::V + vcol + swz128(r, v & 63)) << 16);
            }
            if (!(ok = bar_wait_w(&x_full, (uint32_t)c & 1, &abort_flag, x.status))) break;
            fence_after_sync();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float d[16];
                uint32_t wh[8], wl[8];
                tmem_ld16(tm + lanes + W::T_X + 32 * half + 16 * i, d);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int t = 16 * i + e;
                    R[t] = t < n ? fmaf(-aux[Rec::GAMMA / 4 + t], d[e], R[t]) : 0.f;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = 16 * i + 2 * e;
                    split(aux[Rec::BETA / 4 + t] * R[t], aux[Rec::BETA / 4 + t + 1] * R[t + 1], wh[e], wl[e]);
                }
                tmem_st8(tm + lanes + W::T_AH + 16 * half + 8 * i, wh);
                tmem_st8(tm + lanes + W::T_AL + 16 * half + 8 * i, wl);
            }
            ready(&r_ready);
            if (!(ok = bar_wait_w(&e_full, (uint32_t)c & 1, &abort_flag, x.status))) break;
            fence_after_sync();
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float d[16];
                uint32_t wh[8], wl[8], wu[8];
                tmem_ld16(tm + lanes + W::T_X + 32 * half + 16 * i, d);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int t = 16 * i + 2 * e;
                    R[t] -= d[2 * e];
                    R[t + 1] -= d[2 * e + 1];
                    const float u0 = aux[Rec::BETA / 4 + t] * R[t], u1 = aux[Rec::BETA / 4 + t + 1] * R[t + 1];
                    wu[e] = pack_bf16(u0, u1);
                    split(aux[Rec::KAPPA / 4 + t] * u0, aux[Rec::KAPPA / 4 + t + 1] * u1, wh[e], wl[e]);
                }
                tmem_st8(tm + lanes + W::T_AH + 16 * half + 8 * i, wh);
                tmem_st8(tm + lanes + W::T_AL + 16 * half + 8 * i, wl);
                tmem_st8(tm + lanes + W::T_U + 16 * half + 8 * i, wu);
            }
            decay = *(const float*)(st + W::REC + Rec::LAST);
            ready(&u_ready);
            if (lane == 0) mbar_arrive(&empty[c % W::ST]);
            if (x.e_save) {
                uint4* dst = (uint4*)(x.e_save + ((rec0 + (size_t)c * pk.H) * D + v) * kC + 32 * half);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    dst[i] = make_uint4(pack_bf16(R[8 * i], R[8 * i + 1]), pack_bf16(R[8 * i + 2], R[8 * i + 3]),
                                        pack_bf16(R[8 * i + 4], R[8 * i + 5]), pack_bf16(R[8 * i + 6], R[8 * i + 7]));
            }
        }
        if (ok && chunks > 0) increment(chunks - 1);
        if (ok && x.S1) {
#pragma unroll
            for (int i = 0; i < N; ++i) x.S1[at + (size_t)i * D] = S[i];
        }
        fence_before_sync();
    }
    __syncthreads();
    drain_after_abort(abort_flag);
    if (warp == kWalkMma) {
        fence_after_sync();
        tmem_dealloc(tm, 512);
    }
}

// [rows][heads][d] bf16 with a row stride (elements): boxes of 64 elements of one head in 64 rows,
// 128-byte swizzle; rows outside read as zero.
bool make_chunk_map(CUtensorMap* m, const void* base, int T, int heads, int d, long long stride)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)T};
    cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)stride * 2};
    cuuint32_t box[3] = {64, 1, (cuuint32_t)kC};
    cuuint32_t es[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box,
               es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t fwd(const Packed& p, const void* q, const void* k, const void* v, const void* g,
                const void* beta, WalkArgs& x, uint8_t* rec, cudaStream_t s)
{
    CUtensorMap mq, mk, mv;
    if (!make_chunk_map(&mq, q, p.T, p.Hk, D, p.qs) || !make_chunk_map(&mk, k, p.T, p.Hk, D, p.ks) ||
        !make_chunk_map(&mv, v, p.T, p.H, D, p.vs))
        return cudaErrorInvalidValue;
    const int prep = (D * 256 > (int)sizeof(PrepSmem) ? D * 256 : (int)sizeof(PrepSmem)) + 1024;
    const int walk = (int)Walk<D>::SMEM;
    cudaError_t e = cudaFuncSetAttribute(delta_prep_kernel<D>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, prep);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(delta_walk_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, walk);
    if (e == cudaSuccess)
        e = launch_after(delta_prep_kernel<D>,
                         dim3((unsigned)block_slots(p.T, p.n, kC), (unsigned)p.H), 128, prep, 0, false,
                         s, mq, mk, p, (const __nv_bfloat16*)g, (const __nv_bfloat16*)beta, x.cu,
                         x.scale, rec, x.status);
    if (e == cudaSuccess)
        e = launch_after(delta_walk_kernel<D>, dim3((unsigned)(p.n * p.H)), Walk<D>::THREADS, walk, 0,
                         true, s, mq, mk, mv, x);
    return e;
}

}  // namespace

bool tc_delta_supported(const Packed& p) { return p.bf16 && p.T >= 32 * (long long)p.n; }

size_t tc_delta_rec_bytes(const Packed& p)
{
    return (size_t)block_slots(p.T, p.n, kC) * p.H * Rec::BYTES;
}

cudaError_t launch_tc_delta_fwd(const Packed& p, const void* q, const void* k, const void* v,
                                const void* g, const void* beta, const int* cu, float scale,
                                const float* S0, float* S1, void* out, void* rec, int* status,
                                cudaStream_t s)
{
    WalkArgs x = {};
    x.p = p;
    x.cu = cu; x.scale = scale; x.S0 = S0; x.S1 = S1;
    x.out = (__nv_bfloat16*)out; x.rec = (const uint8_t*)rec; x.status = status;
    return p.d == 64 ? fwd<64>(p, q, k, v, g, beta, x, (uint8_t*)rec, s)
                     : fwd<128>(p, q, k, v, g, beta, x, (uint8_t*)rec, s);
}

}  // namespace flex
