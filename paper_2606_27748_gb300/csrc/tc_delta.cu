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

// (a, b) as bf16 pairs hi + lo, from a packed pair.
__device__ __forceinline__ void split2(uint64_t ab, uint32_t& hi, uint32_t& lo)
{
    float a, b;
    f2_unpack(ab, a, b);
    hi = pack_bf16(a, b);
    const uint64_t h = f2_pack(__uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u));
    f2_unpack(f2_fma(h, f2_pack(-1.f, -1.f), ab), a, b);
    lo = pack_bf16(a, b);
}
__device__ __forceinline__ void split(float a, float b, uint32_t& hi, uint32_t& lo)
{
    split2(f2_pack(a, b), hi, lo);
}

// Matrix descriptors as their varying low words (address and leading offset); the high word is
// the same for all (1024 bytes between groups of 8 rows, 128-byte swizzle), so that an issuing
// warp keeps one register for each.
__device__ __forceinline__ uint32_t dlow(uint32_t addr, uint32_t lbo) { return (addr >> 4) | (lbo >> 4) << 16; }
__device__ __forceinline__ uint64_t desc(uint32_t low, uint32_t bytes)
{
    constexpr uint32_t kHigh = (1024u >> 4) | 1u << 14 | 2u << 29;
    return (uint64_t)kHigh << 32 | (low + (bytes >> 4));
}

// ---- M, P and the gates' factors of every chunk ------------------------------------------
// One CTA of 128 threads per (chunk, head).  [K; Q] K^T is one tcgen05 product of 128 rows: rows
// 0-63 (threads 0-63) K K^T, rows 64-127 Q K^T.  The system is solved in fp32: the four diagonal
// blocks of 16 by forward substitution, a thread per column with the column in registers; then
// the blocks of 16, and the block of 32, below, M21 = X - M22 (beta X) with X = L21 - L21 (beta M11).
struct PrepSmem {
    float L[64][68];  // over the operand tiles, once the product is done
    float M[64][68];  // X stands where M's upper triangle would
};

// x[r] -= sum_k a[r][k] beta[k] m[k][0..3], k < K, R rows (pitch 68).
template <int K, int R>
__device__ __forceinline__ void minus_product(float4* x, const float* a, const float* m, const float* beta)
{
#pragma unroll 2
    for (int k = 0; k < K; k += 4) {
        float4 l[R], y[4];
        const float4 bt = *(const float4*)(beta + k);
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = *(const float4*)(m + (k + e) * 68);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            l[r] = *(const float4*)(a + r * 68 + k);
            l[r].x *= -bt.x; l[r].y *= -bt.y; l[r].z *= -bt.z; l[r].w *= -bt.w;
            x[r].x = fmaf(l[r].w, y[3].x, fmaf(l[r].z, y[2].x, fmaf(l[r].y, y[1].x, fmaf(l[r].x, y[0].x, x[r].x))));
            x[r].y = fmaf(l[r].w, y[3].y, fmaf(l[r].z, y[2].y, fmaf(l[r].y, y[1].y, fmaf(l[r].x, y[0].y, x[r].y))));
            x[r].z = fmaf(l[r].w, y[3].z, fmaf(l[r].z, y[2].z, fmaf(l[r].y, y[1].z, fmaf(l[r].x, y[0].z, x[r].z))));
            x[r].w = fmaf(l[r].w, y[3].w, fmaf(l[r].z, y[2].w, fmaf(l[r].y, y[1].w, fmaf(l[r].x, y[0].w, x[r].w))));
        }
    }
}

template <int D>
__global__ void __launch_bounds__(128)
    delta_prep_kernel(const __grid_constant__ CUtensorMap tmap_q,
                      const __grid_constant__ CUtensorMap tmap_k, Packed pk,
                      const __nv_bfloat16* __restrict__ g, const __nv_bfloat16* __restrict__ beta,
                      const int* __restrict__ cu, float scale, uint8_t* rec, int* status)
{
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);  // (stays a shared-memory pointer)
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
            const uint32_t d = dlow(sb, 16);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const uint32_t o = (ks >> 2) * 16384 + (ks & 3) * 32;
                wmma_bf16(tm, desc(d, o), desc(d, o), I, ks > 0);
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
        const int cols = 32 + 32 * (warp & 1);  // columns up to the diagonal of this warp's rows
        const bool in = row < n;
        if (tid < 64) {  // L, rows behind the end zero (and with them columns: beta is 0 there)
#pragma unroll
            for (int j = 0; j < 64; j += 4) {
                if (j >= cols) break;
                const float4 gj = *(const float4*)&Gs[j];
                const float y[4] = {gj.x, gj.y, gj.z, gj.w};
                float4 x;
                float* z = &x.x;
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = j + e < row && in ? v[j + e] * ex2(G - y[e]) : 0.f;
                *(float4*)&w.L[row][j] = x;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 64; j += 8) {
                uint4 out = make_uint4(0, 0, 0, 0);
                if (j < cols) {
                    const float4 g0 = *(const float4*)&Gs[j], g1 = *(const float4*)&Gs[j + 4];
                    const float y[8] = {g0.x, g0.y, g0.z, g0.w, g1.x, g1.y, g1.z, g1.w};
                    float p[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        p[e] = j + e <= row && in ? scale * v[j + e] * ex2(G - y[e]) : 0.f;
                    out = make_uint4(pack_bf16(p[0], p[1]), pack_bf16(p[2], p[3]),
                                     pack_bf16(p[4], p[5]), pack_bf16(p[6], p[7]));
                }
                *(uint4*)(rec + Rec::P + swz128(row, j)) = out;
            }
            const float last = Gs[63];
            float* aux = (float*)rec;
            aux[Rec::GAMMA / 4 + row] = ex2(G);
            aux[Rec::KAPPA / 4 + row] = in ? ex2(last - G) : 0.f;
            aux[Rec::BETA / 4 + row] = Bs[row];
            if (row == 0) aux[Rec::LAST / 4] = ex2(last);
        }
    }
    __syncthreads();
    if (lane < 16) {  // column `lane` of diagonal block `warp`: x_i = L_ic - sum_k L_ik beta_k x_k
        const int b = 16 * warp;
        float y[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
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
    {  // two blocks of 16 below the diagonal, one row x 4 columns a thread
        const int b = 32 * (tid >> 6), i = (tid & 63) >> 2, j = 4 * (tid & 3);
        float4 x = *(const float4*)&w.L[b + 16 + i][b + j];
        minus_product<16, 1>(&x, &w.L[b + 16 + i][b], &w.M[b][b + j], &Bs[b]);
        *(float4*)&w.M[b + i][b + 16 + j] = x;
        __syncthreads();
        minus_product<16, 1>(&x, &w.M[b + 16 + i][b + 16], &w.M[b][b + 16 + j], &Bs[b + 16]);
        *(float4*)&w.M[b + 16 + i][b + j] = x;
        __syncthreads();
        // (X is dead: its place belongs to M's upper triangle, which the products below read as 0)
        *(float4*)&w.M[b + i][b + 16 + j] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    __syncthreads();
    {  // the block of 32 below, two rows x 4 columns a thread
        const int i = 2 * (tid >> 3), j = 4 * (tid & 7);
        float4 x[2] = {*(const float4*)&w.L[32 + i][j], *(const float4*)&w.L[33 + i][j]};
        minus_product<32, 2>(x, &w.L[32 + i][0], &w.M[0][j], &Bs[0]);
        *(float4*)&w.M[i][32 + j] = x[0];
        *(float4*)&w.M[i + 1][32 + j] = x[1];
        __syncthreads();
        minus_product<32, 2>(x, &w.M[32 + i][32], &w.M[0][32 + j], &Bs[32]);
        *(float4*)&w.M[32 + i][j] = x[0];
        *(float4*)&w.M[33 + i][j] = x[1];
    }
    __syncthreads();
    for (int e = tid; e < 64 * 8; e += 128) {
        const int i = e >> 3, j = (e & 7) * 8;
        uint32_t mh[4], ml[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int a = j + 2 * c;
            const float2 m = *(const float2*)&w.M[i][a];
            split(a < i ? m.x : 0.f, a + 1 < i ? m.y : 0.f, mh[c], ml[c]);
        }
        *(uint4*)(rec + Rec::M_HI + swz128(i, j)) = make_uint4(mh[0], mh[1], mh[2], mh[3]);
        *(uint4*)(rec + Rec::M_LO + swz128(i, j)) = make_uint4(ml[0], ml[1], ml[2], ml[3]);
    }
    if (warp == 0) tmem_dealloc(tm, 64);
}

// ---- the walk over a sequence's chunks ---------------------------------------------------

template <int D>
struct Walk {
    static constexpr int QUADS = D / 32;            // quadrants of tensor memory's lanes in use
    static constexpr int WARPS = 2 * QUADS;         // state warps, and as many token warps
    static constexpr int PIECES = D / 64;           // of the state: 64 key dimensions each
    static constexpr uint32_t TILE = kC * D * 2;    // 64 rows of K, Q or V
    static constexpr uint32_t K = 0, Q = TILE, V = 2 * TILE, REC = 3 * TILE;
    static constexpr uint32_t STAGE = (REC + Rec::BYTES + 1023) / 1024 * 1024;
    static constexpr int ST = D == 128 ? 3 : 4;
    static constexpr uint32_t SMEM = ST * STAGE + 1024;
    // tensor memory columns: S high, low; the chunk's product (K S, then M (beta R), then P U);
    // beta R, then kappa U, high and low; U high and low; the state's increment; Q S
    static constexpr int T_SH = 0, T_SL = D / 2, T_X = D, T_AH = D + 64, T_AL = D + 96, T_UH = D + 128,
                         T_UL = D + 160, T_D = D + 192, T_Q = 2 * D + 192;
    static_assert(2 * D + 256 <= 512, "tensor memory");
};
constexpr int kWalkThreads = 640, kWalkMma = 16, kWalkTma = 17;

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

// State warps (0-7; d = 64: 0, 1, 4, 5) hold the state's fp32 master in registers: quadrant w % 4
// of the lanes, half w / 4 % 2 of each piece of 64 key dimensions.  Token warps (8-15) work on the
// chunk's tokens, half of them each, and write the output while the state warps are busy.  Warp
// 16 issues the products, 17 loads.  A chunk:
//   state   S += last chunk's increment; S high, low -> tensor memory, by pieces   (s_ready)
//   issue   X = K S                                                                (x_full)
//   tokens  R = V - e^G X; beta R high, low                                        (r_ready)
//   issue   X = M (beta R)                                                         (e_full)
//   tokens  E = R - X, U = beta E; e^{G_C - G} U and U high, low                   (u_ready)
//   issue   increment = (e^{G_C - G} U) K, by pieces (s_full), then X = P U        (o_full)
//   tokens  out = scale e^G (Q S) + P U                                    (x_free, q_free)
// The pieces let the products of one piece run beside the arithmetic of the other.  (One set of
// warps for state and tokens needs 168 registers a thread and spills what it holds on the way.)
template <int D>
__global__ void __launch_bounds__(kWalkThreads, 1)
    delta_walk_kernel(const __grid_constant__ CUtensorMap tmap_q,
                      const __grid_constant__ CUtensorMap tmap_k,
                      const __grid_constant__ CUtensorMap tmap_v, WalkArgs x)
{
    using W = Walk<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);  // (stays a shared-memory pointer)
    const uint32_t sb = smem_u32(sm);
    __shared__ uint64_t full[W::ST], empty[W::ST], s_ready[2], s_full[2], x_full, r_ready, e_full,
        u_ready, o_full, x_free, q_free;
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
            mbar_init(&empty[i], 2 * W::WARPS + 1);
        }
        for (int i = 0; i < W::PIECES; ++i) {
            mbar_init(&s_ready[i], W::WARPS);
            mbar_init(&s_full[i], 1);
        }
        mbar_init(&r_ready, W::WARPS);
        mbar_init(&u_ready, W::WARPS);
        mbar_init(&x_free, W::WARPS);
        mbar_init(&q_free, W::WARPS);
        mbar_init(&x_full, 1);
        mbar_init(&e_full, 1);
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

    // registers: launched with 96 a thread; 2 x 104 + 2 x 104 + 64 = 480 = 5 x 96
    if (warp >= 16) {
        setmaxnreg_dec<64>();
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
            constexpr uint32_t I_C = idesc_bf16(128, kC, 0, 0), I_D = idesc_bf16(128, 64, 0, 1);
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
                const uint32_t dk = dlow(st + W::K, 16), dq = dlow(st + W::Q, 16);
                const uint32_t dkn = dlow(st + W::K, 8192);
                const uint32_t dmh = dlow(st + W::REC + Rec::M_HI, 16);
                const uint32_t dml = dlow(st + W::REC + Rec::M_LO, 16);
                const uint32_t dp = dlow(st + W::REC + Rec::P, 16);
                if (c > 0) wait(&x_free, c - 1);  // P U of the last chunk has been read from X
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
                    wait(&s_ready[p], c);
                    if (!ok) break;
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        wmma_bf16_tmem_a(tm + W::T_X, tm + (ks < 4 ? W::T_SH : W::T_SL) + 32 * p + 8 * (ks & 3),
                                         desc(dk, 8192 * p + (ks & 3) * 32), I_C, p > 0 || ks > 0);
                }
                if (!ok) break;
                wmma_commit(&x_full);
                if (c > 0) wait(&q_free, c - 1);
                if (!ok) break;
#pragma unroll
                for (int ks = 0; ks < D / 8; ++ks) {
                    const int k = ks % (D / 16);
                    wmma_bf16_tmem_a(tm + W::T_Q, tm + (ks < D / 16 ? W::T_SH : W::T_SL) + 8 * k,
                                     desc(dq, (k >> 2) * 8192 + (k & 3) * 32), I_C, ks > 0);
                }
                wait(&r_ready, c);
                if (!ok) break;
#pragma unroll
                for (int ks = 0; ks < 12; ++ks) {  // high high, low high, high low
                    const int k = ks & 3;
                    wmma_bf16_tmem_a(tm + W::T_X, tm + (ks >> 2 == 1 ? W::T_AL : W::T_AH) + 8 * k,
                                     desc(ks >> 2 == 2 ? dml : dmh, k * 32), I_C, ks > 0);
                }
                wmma_commit(&e_full);
                wait(&u_ready, c);
                if (!ok) break;
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
#pragma unroll
                    for (int ks = 0; ks < 8; ++ks)
                        wmma_bf16_tmem_a(tm + W::T_D + 64 * p, tm + (ks < 4 ? W::T_AH : W::T_AL) + 8 * (ks & 3),
                                         desc(dkn, 8192 * p + (ks & 3) * 2048), I_D, ks > 0);
                    wmma_commit(&s_full[p]);
                }
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    wmma_bf16_tmem_a(tm + W::T_X, tm + (ks < 4 ? W::T_UH : W::T_UL) + 8 * (ks & 3),
                                     desc(dp, (ks & 3) * 32), I_C, ks > 0);
                wmma_commit(&o_full);
                wmma_commit(&empty[c % W::ST]);
            }
        }
    } else {
        setmaxnreg_inc<104>();
        const int half = (warp >> 2) & 1, v = 32 * (warp & 3) + lane;
        const uint32_t lanes = tm + ((uint32_t)(warp & 3) << 21);
        auto ready = [&](uint64_t* bar) {
            tmem_wait_st();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        bool ok = true;
        auto wait = [&](uint64_t* bar, int phase) {
            ok = bar_wait_w(bar, (uint32_t)phase & 1, &abort_flag, x.status);
            fence_after_sync();
            return ok;
        };
        if ((warp & 3) >= W::QUADS) {
            // (no lane of this quadrant holds a value dimension)
        } else if (warp < 8) {
            // ---- the state ----
            float S[W::PIECES][32];  // key dimensions 64 p + 32 half + 0 .. 31
            const size_t at = ((size_t)s * pk.H + h) * D * D + (size_t)half * 32 * D + v;
#pragma unroll
            for (int p = 0; p < W::PIECES; ++p)
#pragma unroll
                for (int i = 0; i < 32; ++i) S[p][i] = x.S0 ? x.S0[at + (size_t)(64 * p + i) * D] : 0.f;
            float decay = 1.f;
            for (int c = 0; c <= chunks; ++c) {
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
                    if (c > 0 && !wait(&s_full[p], c - 1)) break;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (c > 0) {  // S = decay S + the increment of the last chunk
                            float a[16];
                            tmem_ld16(lanes + W::T_D + 64 * p + 32 * half + 16 * j, a);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) S[p][16 * j + e] = fmaf(decay, S[p][16 * j + e], a[e]);
                        }
                        if (c < chunks) {
                            uint32_t wh[8], wl[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                split(S[p][16 * j + 2 * e], S[p][16 * j + 2 * e + 1], wh[e], wl[e]);
                            tmem_st8(lanes + W::T_SH + 32 * p + 16 * half + 8 * j, wh);
                            tmem_st8(lanes + W::T_SL + 32 * p + 16 * half + 8 * j, wl);
                            if (x.s_save) {
                                uint4* dst = (uint4*)(x.s_save + ((rec0 + (size_t)c * pk.H) * D + v) * D +
                                                      64 * p + 32 * half + 16 * j);
                                dst[0] = make_uint4(wh[0], wh[1], wh[2], wh[3]);
                                dst[1] = make_uint4(wh[4], wh[5], wh[6], wh[7]);
                            }
                        }
                    }
                    if (c < chunks) ready(&s_ready[p]);
                }
                if (!ok || c == chunks || !(ok = landed(c))) break;
                decay = *(const float*)(sm + stage(c) + W::REC + Rec::LAST);
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty[c % W::ST]);
            }
            if (ok && x.S1) {
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p)
#pragma unroll
                    for (int i = 0; i < 32; ++i) x.S1[at + (size_t)(64 * p + i) * D] = S[p][i];
            }
        } else {
            // ---- the tokens ----
            const size_t os = (size_t)pk.H * D;
            __nv_bfloat16* out = x.out + (size_t)(lo + 32 * half + (lane & 1)) * os + h * D + (v & ~1);
            for (int c = 0; c < chunks; ++c) {
                if (!(ok = landed(c))) break;
                const uint8_t* st = sm + stage(c);
                const float* aux = (const float*)(st + W::REC) + 32 * half;
                const int n = hi - lo - c * kC - 32 * half;
                float R[32];
                {
                    const uint8_t* col = st + W::V + (uint32_t)(v >> 6) * 8192 + half * 4096;
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        R[i] = __uint_as_float((uint32_t) * (const uint16_t*)(col + swz128(i, v & 63)) << 16);
                }
                if (n < 32) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) R[i] = i < n ? R[i] : 0.f;
                }
                if (!wait(&x_full, c)) break;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16];
                    tmem_ld16(lanes + W::T_X + 32 * half + 16 * j, d);
                    tmem_wait_ld();
                    uint32_t wh[8], wl[8];
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {  // (X is 0 behind the end: K is)
                        const float4 gm = *(const float4*)(aux + Rec::GAMMA / 4 + 16 * j + i);
                        const float4 bt = *(const float4*)(aux + Rec::BETA / 4 + 16 * j + i);
                        float* r = R + 16 * j + i;
                        r[0] = fmaf(-gm.x, d[i], r[0]);
                        r[1] = fmaf(-gm.y, d[i + 1], r[1]);
                        r[2] = fmaf(-gm.z, d[i + 2], r[2]);
                        r[3] = fmaf(-gm.w, d[i + 3], r[3]);
                        split2(f2_mul(f2_pack(bt.x, bt.y), f2_pack(r[0], r[1])), wh[i / 2], wl[i / 2]);
                        split2(f2_mul(f2_pack(bt.z, bt.w), f2_pack(r[2], r[3])), wh[i / 2 + 1], wl[i / 2 + 1]);
                    }
                    tmem_st8(lanes + W::T_AH + 16 * half + 8 * j, wh);
                    tmem_st8(lanes + W::T_AL + 16 * half + 8 * j, wl);
                }
                ready(&r_ready);
                if (!wait(&e_full, c)) break;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16];
                    tmem_ld16(lanes + W::T_X + 32 * half + 16 * j, d);
                    tmem_wait_ld();
                    uint32_t wh[8], wl[8], uh[8], ul[8];
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const float4 bt = *(const float4*)(aux + Rec::BETA / 4 + 16 * j + i);
                        const float4 kp = *(const float4*)(aux + Rec::KAPPA / 4 + 16 * j + i);
                        float* r = R + 16 * j + i;
                        r[0] -= d[i];
                        r[1] -= d[i + 1];
                        r[2] -= d[i + 2];
                        r[3] -= d[i + 3];
                        const uint64_t u0 = f2_mul(f2_pack(bt.x, bt.y), f2_pack(r[0], r[1]));
                        const uint64_t u1 = f2_mul(f2_pack(bt.z, bt.w), f2_pack(r[2], r[3]));
                        split2(f2_mul(f2_pack(kp.x, kp.y), u0), wh[i / 2], wl[i / 2]);
                        split2(f2_mul(f2_pack(kp.z, kp.w), u1), wh[i / 2 + 1], wl[i / 2 + 1]);
                        split2(u0, uh[i / 2], ul[i / 2]);
                        split2(u1, uh[i / 2 + 1], ul[i / 2 + 1]);
                    }
                    tmem_st8(lanes + W::T_AH + 16 * half + 8 * j, wh);
                    tmem_st8(lanes + W::T_AL + 16 * half + 8 * j, wl);
                    tmem_st8(lanes + W::T_UH + 16 * half + 8 * j, uh);
                    tmem_st8(lanes + W::T_UL + 16 * half + 8 * j, ul);
                }
                ready(&u_ready);
                if (x.e_save) {
                    uint4* dst = (uint4*)(x.e_save + ((rec0 + (size_t)c * pk.H) * D + v) * kC + 32 * half);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        dst[i] = make_uint4(pack_bf16(R[8 * i], R[8 * i + 1]), pack_bf16(R[8 * i + 2], R[8 * i + 3]),
                                            pack_bf16(R[8 * i + 4], R[8 * i + 5]), pack_bf16(R[8 * i + 6], R[8 * i + 7]));
                }
                if (!wait(&o_full, c)) break;
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    tmem_ld16(lanes + W::T_X + 32 * half + 16 * j, *(float(*)[16])(R + 16 * j));
                tmem_wait_ld();
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&x_free);
                // neighbouring lanes exchange halves of two rows: each writes two elements of one
                __nv_bfloat16* dst = out + (size_t)(c * kC) * os;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16];
                    tmem_ld16(lanes + W::T_Q + 32 * half + 16 * j, d);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        const float2 gm = *(const float2*)(aux + Rec::GAMMA / 4 + 16 * j + e);
                        const float o0 = fmaf(x.scale * gm.x, d[e], R[16 * j + e]);
                        const float o1 = fmaf(x.scale * gm.y, d[e + 1], R[16 * j + e + 1]);
                        const float other = __shfl_xor_sync(0xffffffffu, lane & 1 ? o0 : o1, 1);
                        const uint32_t w = lane & 1 ? pack_bf16(other, o1) : pack_bf16(o0, other);
                        if (16 * j + e + (lane & 1) < n) *(uint32_t*)dst = w;
                        dst += 2 * os;
                    }
                }
                fence_before_sync();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&q_free);
                    mbar_arrive(&empty[c % W::ST]);
                }
            }
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
        e = launch_after(delta_walk_kernel<D>, dim3((unsigned)(p.n * p.H)), kWalkThreads, walk, 0,
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
