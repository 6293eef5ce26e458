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
// Precision: K and Q are exact.  What multiplies them (S, beta R, U, M and P) is split into bf16 high
// and low parts (2^-17), so that the output is off by little more than its own rounding (with P as
// bf16 by 1.6 times it).  The state, held in fp32 registers, would be off by 2.8e-6 so, nearly all of
// it from e^{G_C - G} U, what a chunk adds.  A prompt's walk takes that and beta R in three parts and
// multiplies M's and beta R's low parts too: 6e-7 to 7e-7 (8 x 4096, H16 d128: 371 -> 394 us; S and M
// need no third part: emulated, 5e-8 and 5e-7).  The walk that saves for the backward, whose results
// are bf16, does without (third parts for both: 371 us instead of 355 for 8 x 2048 H12 d64).
// The backward's results are bf16 and held to 1.2 times their own rounding: of its operands P, E and
// Zq (below) are split, which left 1.8 times it as bf16 (E and Zq 1.7e-3 each of dq's 3.0e-3, dk's and
// dg's 3.1e-3; splitting them took 331 us to 355, 8 x 2048 H12 d64); the state and its gradient of a
// chunk, dV and the walk's own operands, bf16 too, leave 0.6e-3 or less each.
#include <cuda.h>

#include "flex_internal.h"
#include "packed.cuh"
#include "tc_util.cuh"

namespace flex {
namespace {

using namespace tc;

constexpr int kC = 64;             // tokens of a chunk
constexpr double kLog2e = 1.4426950408889634;
// A log decay of -88 is exp(-88) = 6e-39, no factor in fp32 sums; -inf is taken as that, since
// the differences of the sums G have to be finite.  A chunk's G may so reach -8000 (powers of two),
// where fp32 knows a difference to 2^-12 only and with it the decay between two tokens behind a few
// resets: 32 of them, then slow decays, made the last state 1e-4 wrong.  So G is summed in 64 bits
// and kept as a high and a low float.
constexpr float kLeastGate = -88.f;

// What the walk needs of a chunk, as it is copied to shared memory: M's low and high parts and
// P's high and low ones (64 x 64 bf16, 128-byte rows, swizzled), then -e^G, e^{G_C - G}, beta (0
// behind the sequence's end), G's high part in powers of two (64 floats each) and e^{G_C}.
struct Rec {
    static constexpr uint32_t M_LO = 0, M_HI = 8192, P = 16384, P_LO = 24576, AUX = 32768, BYTES = 34048;
    static constexpr uint32_t GAMMA = AUX, KAPPA = AUX + 256, BETA = AUX + 512, G = AUX + 768, LAST = AUX + 1024;
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

// ... and, if `third`, what those leave.
__device__ __forceinline__ void split23(uint64_t ab, bool third, uint32_t& hi, uint32_t& lo, uint32_t& rest)
{
    split2(ab, hi, lo);
    if (!third) return;
    const uint64_t minus = f2_pack(-1.f, -1.f);
    ab = f2_fma(f2_pack(__uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u)), minus, ab);
    ab = f2_fma(f2_pack(__uint_as_float(lo << 16), __uint_as_float(lo & 0xffff0000u)), minus, ab);
    float a, b;
    f2_unpack(ab, a, b);
    rest = pack_bf16(a, b);
}

// Eight packed pairs rounded to bf16.
__device__ __forceinline__ void pack8(const uint64_t* x, uint32_t (&w)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float a, b;
        f2_unpack(x[i], a, b);
        w[i] = pack_bf16(a, b);
    }
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

// Four products of 16 along K with A in tensor memory (8 columns a step) and B in shared memory
// (`bstep` bytes a step), into one accumulator.
__device__ __forceinline__ void mma4(uint32_t d, uint32_t a, uint32_t b_low, uint32_t bstep, uint32_t idesc,
                                     uint32_t accumulate)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        wmma_bf16_tmem_a(d, a + 8 * i, desc(b_low, bstep * i), idesc, i > 0 ? 1u : accumulate);
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
    __shared__ __align__(16) float Gs[64], Gl[64], Bs[64];  // G, high and low; beta

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
        double a[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = 2 * lane + i;
            const size_t at = (size_t)(t0 + j) * pk.H + h;
            const float gate = j < n ? __bfloat162float(g[at]) : 0.f;
            a[i] = (double)(gate < kLeastGate ? kLeastGate : gate) * kLog2e;  // (NaN stays)
            Bs[j] = j < n ? __bfloat162float(beta[at]) : 0.f;
        }
        double sum = a[0] + a[1];
#pragma unroll
        for (int m = 1; m < 32; m *= 2) {
            const double o = __shfl_up_sync(0xffffffffu, sum, m);
            if (lane >= m) sum += o;
        }
        double before = __shfl_up_sync(0xffffffffu, sum, 1);
        if (lane == 0) before = 0.;
        const double G[2] = {before + a[0], sum};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            Gs[2 * lane + i] = (float)G[i];
            Gl[2 * lane + i] = (float)(G[i] - (double)(float)G[i]);
        }
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
        const uint64_t G2 = f2_pack(G, G), Gl2 = f2_pack(Gl[row], Gl[row]), one = f2_pack(1.f, 1.f);
        const uint64_t minus = f2_pack(-1.f, -1.f);
        // (G down to -32 is known to 2^-20, and the low part would change a decay by 1e-6 at most)
        const bool far = !(Gs[63] >= -32.f);
        auto decays = [&](int j, float (&y)[4]) {  // of this row against columns j .. j + 3
            const ulonglong2 h = *(const ulonglong2*)&Gs[j];
            uint64_t a = f2_fma(h.x, minus, G2), b = f2_fma(h.y, minus, G2);
            if (far) {
                const ulonglong2 l = *(const ulonglong2*)&Gl[j];
                a = f2_fma(f2_fma(l.x, minus, Gl2), one, a);
                b = f2_fma(f2_fma(l.y, minus, Gl2), one, b);
            }
            f2_unpack(a, y[0], y[1]);
            f2_unpack(b, y[2], y[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = ex2(y[e]);
        };
        const int cols = 32 + 32 * (warp & 1);  // columns up to the diagonal of this warp's rows
        const bool in = row < n;
        if (tid < 64) {  // L, rows behind the end zero (and with them columns: beta is 0 there)
#pragma unroll
            for (int j = 0; j < 64; j += 4) {
                if (j >= cols) break;
                float y[4];
                decays(j, y);
                float4 x;
                float* z = &x.x;
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = j + e < row && in ? v[j + e] * y[e] : 0.f;
                *(float4*)&w.L[row][j] = x;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 64; j += 8) {
                uint4 out = make_uint4(0, 0, 0, 0), out_lo = out;
                if (j < cols) {
                    float y[2][4], p[8];
                    decays(j, y[0]);
                    decays(j + 4, y[1]);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        p[e] = j + e <= row && in ? scale * v[j + e] * y[e / 4][e % 4] : 0.f;
                    split(p[0], p[1], out.x, out_lo.x);
                    split(p[2], p[3], out.y, out_lo.y);
                    split(p[4], p[5], out.z, out_lo.z);
                    split(p[6], p[7], out.w, out_lo.w);
                }
                *(uint4*)(rec + Rec::P + swz128(row, j)) = out;
                *(uint4*)(rec + Rec::P_LO + swz128(row, j)) = out_lo;
            }
            const float last = Gs[63];
            float* aux = (float*)rec;
            aux[Rec::GAMMA / 4 + row] = -ex2(G);
            aux[Rec::KAPPA / 4 + row] = in ? ex2((last - G) + (Gl[63] - Gl[row])) : 0.f;
            aux[Rec::BETA / 4 + row] = Bs[row];
            aux[Rec::G / 4 + row] = G;
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
    // The issuing and the loading warp: for d = 64, which computes on quadrants 0 and 1 and so on
    // schedulers 0 and 1, they go to the others (training, 8 x 2048 H12: 356 -> 350 us; d = 128 is the
    // slower for it).
    static constexpr int MMA = D == 64 ? 18 : 16, TMA = D == 64 ? 19 : 17;
    static constexpr uint32_t TILE = kC * D * 2;    // 64 rows of K, Q or V
    static constexpr uint32_t K = 0, Q = TILE, V = 2 * TILE, REC = 3 * TILE;
    static constexpr uint32_t STAGE = (REC + Rec::BYTES + 1023) / 1024 * 1024;
    static constexpr int ST = D == 128 ? 2 : 3;
    static constexpr uint32_t SMEM = ST * STAGE + 1024;
    // tensor memory columns: S high, low; the chunk's product (K S, then M (beta R), then P U);
    // beta R, then kappa U, high and low; U high and low; the state's increment; Q S
    static constexpr int T_SH = 0, T_SL = D / 2, T_X = D, T_AH = D + 64, T_AL = D + 96, T_UH = D + 128,
                         T_UL = D + 160, T_D = D + 192, T_Q = 2 * D + 192;
    // The third parts: of beta R where U comes once the product with M is done, of kappa U where the
    // state's last piece stands, which that product's completion frees and s_full of that piece hands on.
    static constexpr int T_RM = T_UH, T_KM = T_SH + 32 * (PIECES - 1);
    static_assert(2 * D + 256 <= 512, "tensor memory");
};
constexpr int kWalkThreads = 640;

struct WalkArgs {
    Packed p;
    const int* cu;
    float scale;
    const float* S0;
    float* S1;
    __nv_bfloat16* out;
    const uint8_t* rec;
    // (saving) E^T [slot][H][high, low][d][64] and S^T [slot][H][d][d] of each chunk
    __nv_bfloat16 *e_save, *s_save;
    int* status;
};

// State warps (0-7; d = 64: 0, 1, 4, 5) hold the state's fp32 master in registers: quadrant w % 4
// of the lanes, half w / 4 % 2 of each piece of 64 key dimensions.  Token warps (8-15) work on the
// chunk's tokens, half of them each, and write the output while the state warps are busy.  Warp
// MMA issues the products, warp TMA loads.  A chunk:
//   state   S += last chunk's increment; S high, low -> tensor memory, by pieces   (s_ready)
//   issue   X = K S                                                                (x_full)
//   tokens  R = V - e^G X; beta R high, low                                        (r_ready)
//   issue   X = M (beta R)                                                         (e_full)
//   tokens  E = R - X, U = beta E; e^{G_C - G} U, then U, high, low        (u_ready, p_ready)
//   issue   increment = (e^{G_C - G} U) K, by pieces (s_full), then X = P U        (o_full)
//   tokens  out = scale e^G (Q S) + P U                                    (x_free, q_free)
// The pieces let the products of one piece run beside the arithmetic of the other.  (One set of
// warps for state and tokens would need 168 registers a thread, of 96.)  SAVE: leave E and S for the
// backward, without third parts (see the top).
template <int D, bool SAVE>
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
        u_ready, p_ready, o_full, x_free, q_free;
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
        mbar_init(&p_ready, W::WARPS);
        mbar_init(&x_free, W::WARPS);
        mbar_init(&q_free, W::WARPS);
        mbar_init(&x_full, 1);
        mbar_init(&e_full, 1);
        mbar_init(&o_full, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == W::MMA) {
        tmem_alloc(&tmem_base_sh, 512);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tm = tmem_base_sh;
    if (tm != 0 && tid == 0) {  // (cannot be; nothing is issued then)
        abort_flag = 1;
        if (x.status) atomicExch(x.status, (int)FLEX_ECUDA);
    }
    auto stage = [&](int c) { return (uint32_t)(c % W::ST) * W::STAGE; };
    auto landed = [&](int c) {
        return bar_wait_w(&full[c % W::ST], (uint32_t)(c / W::ST) & 1, &abort_flag, x.status);
    };

    // registers: launched with 96 a thread; 2 x 104 + 2 x 104 + 64 = 480 = 5 x 96
    if (warp >= 16) {
        setmaxnreg_dec<64>();
        if (warp == W::TMA) {
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
        } else if (warp == W::MMA && tm == 0) {  // all of tensor memory starts at its address 0
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
                const uint32_t dp = dlow(st + W::REC + Rec::P, 16), dpl = dlow(st + W::REC + Rec::P_LO, 16);
                if (c > 0) wait(&x_free, c - 1);  // P U of the last chunk has been read from X
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
                    wait(&s_ready[p], c);
                    if (!ok) break;
                    mma4(W::T_X, W::T_SH + 32 * p, dk + 512 * p, 32, I_C, p > 0);
                    mma4(W::T_X, W::T_SL + 32 * p, dk + 512 * p, 32, I_C, 1);
                }
                if (!ok) break;
                wmma_commit(&x_full);
                if (c > 0) wait(&q_free, c - 1);
                if (!ok) break;
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
                    mma4(W::T_Q, W::T_SH + 32 * p, dq + 512 * p, 32, I_C, p > 0);
                    mma4(W::T_Q, W::T_SL + 32 * p, dq + 512 * p, 32, I_C, 1);
                }
                wait(&r_ready, c);
                if (!ok) break;
                mma4(W::T_X, W::T_AH, dmh, 32, I_C, 0);
                mma4(W::T_X, W::T_AL, dmh, 32, I_C, 1);
                mma4(W::T_X, W::T_AH, dml, 32, I_C, 1);
                if (!SAVE) {
                    mma4(W::T_X, W::T_RM, dmh, 32, I_C, 1);
                    mma4(W::T_X, W::T_AL, dml, 32, I_C, 1);
                }
                wmma_commit(&e_full);
                wait(&u_ready, c);
                if (!ok) break;
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
                    mma4(W::T_D + 64 * p, W::T_AH, dkn + 512 * p, 2048, I_D, 0);
                    mma4(W::T_D + 64 * p, W::T_AL, dkn + 512 * p, 2048, I_D, 1);
                    if (!SAVE) mma4(W::T_D + 64 * p, W::T_KM, dkn + 512 * p, 2048, I_D, 1);
                    wmma_commit(&s_full[p]);
                }
                wait(&p_ready, c);
                if (!ok) break;
                mma4(W::T_X, W::T_UH, dp, 32, I_C, 0);
                mma4(W::T_X, W::T_UL, dp, 32, I_C, 1);
                mma4(W::T_X, W::T_UH, dpl, 32, I_C, 1);
                wmma_commit(&o_full);
                // (only where a later load waits for it: no arrival may be on its way when the block ends)
                if (c + W::ST < chunks) wmma_commit(&empty[c % W::ST]);
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
            uint64_t S[W::PIECES][16];  // pairs of key dimensions 64 p + 32 half + 0 .. 31
            const size_t at = ((size_t)s * pk.H + h) * D * D + (size_t)half * 32 * D + v;
#pragma unroll
            for (int p = 0; p < W::PIECES; ++p)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float* y = x.S0 + at + (size_t)(64 * p + 2 * i) * D;
                    S[p][i] = x.S0 ? f2_pack(y[0], y[D]) : f2_pack(0.f, 0.f);
                }
            uint64_t decay = f2_pack(1.f, 1.f);
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
                            for (int e = 0; e < 8; ++e)
                                S[p][8 * j + e] = f2_fma(decay, S[p][8 * j + e], f2_pack(a[2 * e], a[2 * e + 1]));
                        }
                        if (c < chunks) {
                            uint32_t wh[8], wl[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) split2(S[p][8 * j + e], wh[e], wl[e]);
                            tmem_st8(lanes + W::T_SH + 32 * p + 16 * half + 8 * j, wh);
                            tmem_st8(lanes + W::T_SL + 32 * p + 16 * half + 8 * j, wl);
                        }
                    }
                    if (c < chunks) ready(&s_ready[p]);
                }
                if (SAVE && ok && c < chunks) {  // (rounded again: the walk waits for the pieces)
#pragma unroll
                    for (int p = 0; p < W::PIECES; ++p) {
                        __nv_bfloat16* dst = x.s_save + ((rec0 + (size_t)c * pk.H) * D + v) * D + 64 * p + 32 * half;
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint32_t w[8];
                            pack8(S[p] + 8 * j, w);
                            store_32b(dst + 16 * j, make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7]));
                        }
                    }
                }
                if (!ok || c == chunks || !(ok = landed(c))) break;
                const float last = *(const float*)(sm + stage(c) + W::REC + Rec::LAST);
                decay = f2_pack(last, last);
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty[c % W::ST]);
            }
            if (ok && x.S1) {
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float* y = x.S1 + at + (size_t)(64 * p + 2 * i) * D;
                        float a, b;
                        f2_unpack(S[p][i], a, b);
                        y[0] = a;
                        y[D] = b;
                    }
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
                uint64_t R[16];  // pairs of tokens
                {
                    const uint8_t* col = st + W::V + (uint32_t)(v >> 6) * 8192 + half * 4096;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t a = *(const uint16_t*)(col + swz128(2 * i, v & 63));
                        const uint32_t b = *(const uint16_t*)(col + swz128(2 * i + 1, v & 63));
                        R[i] = f2_pack(__uint_as_float(a << 16), __uint_as_float(b << 16));
                    }
                }
                if (n < 32) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float a, b;
                        f2_unpack(R[i], a, b);
                        R[i] = f2_pack(2 * i < n ? a : 0.f, 2 * i + 1 < n ? b : 0.f);
                    }
                }
                if (!wait(&x_full, c)) break;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16];
                    tmem_ld16(lanes + W::T_X + 32 * half + 16 * j, d);
                    tmem_wait_ld();
                    uint32_t wh[8], wl[8], wm[8];
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {  // (X is 0 behind the end: K is)
                        const ulonglong2 gm = *(const ulonglong2*)(aux + Rec::GAMMA / 4 + 16 * j + 2 * i);
                        const ulonglong2 bt = *(const ulonglong2*)(aux + Rec::BETA / 4 + 16 * j + 2 * i);
                        uint64_t* r = R + 8 * j + i;
                        // (e^G holds its negative in the record: R = V - e^G X)
                        r[0] = f2_fma(gm.x, f2_pack(d[2 * i], d[2 * i + 1]), r[0]);
                        r[1] = f2_fma(gm.y, f2_pack(d[2 * i + 2], d[2 * i + 3]), r[1]);
                        split23(f2_mul(bt.x, r[0]), !SAVE, wh[i], wl[i], wm[i]);
                        split23(f2_mul(bt.y, r[1]), !SAVE, wh[i + 1], wl[i + 1], wm[i + 1]);
                    }
                    tmem_st8(lanes + W::T_AH + 16 * half + 8 * j, wh);
                    tmem_st8(lanes + W::T_AL + 16 * half + 8 * j, wl);
                    if (!SAVE) tmem_st8(lanes + W::T_RM + 16 * half + 8 * j, wm);
                }
                ready(&r_ready);
                if (!wait(&e_full, c)) break;
                const uint64_t minus = f2_pack(-1.f, -1.f);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16];
                    tmem_ld16(lanes + W::T_X + 32 * half + 16 * j, d);
                    tmem_wait_ld();
                    uint32_t wh[8], wl[8], wm[8];
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const ulonglong2 bt = *(const ulonglong2*)(aux + Rec::BETA / 4 + 16 * j + 2 * i);
                        const ulonglong2 kp = *(const ulonglong2*)(aux + Rec::KAPPA / 4 + 16 * j + 2 * i);
                        uint64_t* r = R + 8 * j + i;
                        r[0] = f2_fma(f2_pack(d[2 * i], d[2 * i + 1]), minus, r[0]);
                        r[1] = f2_fma(f2_pack(d[2 * i + 2], d[2 * i + 3]), minus, r[1]);
                        split23(f2_mul(f2_mul(kp.x, bt.x), r[0]), !SAVE, wh[i], wl[i], wm[i]);
                        split23(f2_mul(f2_mul(kp.y, bt.y), r[1]), !SAVE, wh[i + 1], wl[i + 1], wm[i + 1]);
                    }
                    tmem_st8(lanes + W::T_AH + 16 * half + 8 * j, wh);
                    tmem_st8(lanes + W::T_AL + 16 * half + 8 * j, wl);
                    if (!SAVE) tmem_st8(lanes + W::T_KM + 16 * half + 8 * j, wm);
                }
                ready(&u_ready);
#pragma unroll
                for (int j = 0; j < 2; ++j) {  // (the output waits for nothing but the next chunk's X)
                    uint32_t uh[8], ul[8];
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const ulonglong2 bt = *(const ulonglong2*)(aux + Rec::BETA / 4 + 16 * j + 2 * i);
                        split2(f2_mul(bt.x, R[8 * j + i]), uh[i], ul[i]);
                        split2(f2_mul(bt.y, R[8 * j + i + 1]), uh[i + 1], ul[i + 1]);
                    }
                    tmem_st8(lanes + W::T_UH + 16 * half + 8 * j, uh);
                    tmem_st8(lanes + W::T_UL + 16 * half + 8 * j, ul);
                }
                ready(&p_ready);
                if (SAVE) {
                    __nv_bfloat16* dst = x.e_save + ((rec0 + (size_t)c * pk.H) * 2 * D + v) * kC + 32 * half;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t w[8], y[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) split2(R[8 * i + e], w[e], y[e]);
                        store_32b(dst + 16 * i, make_uint4(w[0], w[1], w[2], w[3]), make_uint4(w[4], w[5], w[6], w[7]));
                        store_32b(dst + D * kC + 16 * i, make_uint4(y[0], y[1], y[2], y[3]),
                                  make_uint4(y[4], y[5], y[6], y[7]));
                    }
                }
                if (!wait(&o_full, c)) break;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16];
                    tmem_ld16(lanes + W::T_X + 32 * half + 16 * j, d);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 8; ++e) R[8 * j + e] = f2_pack(d[2 * e], d[2 * e + 1]);
                }
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&x_free);
                // neighbouring lanes exchange halves of two rows: each writes two elements of one
                __nv_bfloat16* dst = out + (size_t)(c * kC) * os;
                const uint32_t pick = lane & 1 ? 0x3276u : 0x5410u;
                const uint64_t factor = f2_pack(-x.scale, -x.scale);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16];
                    tmem_ld16(lanes + W::T_Q + 32 * half + 16 * j, d);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const uint64_t gm = *(const uint64_t*)(aux + Rec::GAMMA / 4 + 16 * j + 2 * e);
                        float o0, o1;
                        f2_unpack(f2_fma(f2_mul(factor, gm), f2_pack(d[2 * e], d[2 * e + 1]), R[8 * j + e]), o0, o1);
                        const uint32_t w = pack_bf16(o0, o1);
                        const uint32_t y = __byte_perm(w, __shfl_xor_sync(0xffffffffu, w, 1), pick);
                        if (16 * j + 2 * e + (lane & 1) < n) *(uint32_t*)dst = y;
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
    if (warp == W::MMA) {
        fence_after_sync();
        tmem_dealloc(tm, 512);
    }
}

// ---- backward, the walk in reverse -------------------------------------------------------
// With D the gradient of the state behind a chunk (the scale folded into P),
//   dU = P^T dO + e^{G_C - G} K D,  Y = dU - M^T (beta dU),  dV = beta Y,  dbeta = E . Y,
//   D <- e^{G_C} D + Q^T (scale e^G dO) - K^T (e^G dV).
// Held transposed like the forward's walk, with the same roles and steps.  All results are bf16,
// so the products' operands but P are bf16 without a low part (see the top); D itself stays fp32 in
// registers.  D of every chunk, dV and the products E . Y (in fp32, summed over a quadrant's 32 value
// dimensions) go to memory.
template <int D>
struct Back {
    static constexpr uint32_t TILE = kC * D * 2;
    static constexpr uint32_t REC_BYTES = Rec::BYTES - Rec::M_HI;  // M's high part, P, the factors
    // (E: a value dimension a row, high parts, then low ones)
    static constexpr uint32_t K = 0, Q = TILE, DO = 2 * TILE, E = 3 * TILE, REC = 5 * TILE;
    static constexpr uint32_t STAGE = (REC + REC_BYTES + 1023) / 1024 * 1024;
    static constexpr int ST = D == 128 ? 2 : 3;
    static constexpr uint32_t SMEM = ST * STAGE + 1024;
    static constexpr uint32_t M = REC, P = REC + Rec::P - Rec::M_HI, AUX = REC + Rec::AUX - Rec::M_HI;
    // tensor memory: D; K D, then M^T (beta dU); P^T dO; beta dU; -e^G dV; scale e^G dO; increment
    static constexpr int T_S = 0, T_X = D / 2, T_P = T_X + 64, T_A = T_P + 64, T_R = T_A + 32,
                         T_O = T_R + 32, T_D = T_O + 32;
    static_assert(T_D + D <= 512, "tensor memory");
};

struct BackArgs {
    Packed p;
    const int* cu;
    float scale;
    const uint8_t* rec;
    __nv_bfloat16* ds;       // D^T [slot][H][d][d]
    float* db;               // [slot][H][4][64]
    __nv_bfloat16* dv;
    int* status;
};

// 32 lanes x 32 bits, 8 consecutive columns.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float (&v)[8])
{
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
                   "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}

// sum_lane x[i] for 16 values i: lanes 2 i and 2 i + 1 return the sum of value i.
__device__ __forceinline__ float transpose_sum16(float (&x)[16])
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int m = 16, n = 8; n >= 1; m >>= 1, n >>= 1) {
        const bool up = lane & m;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float give = up ? x[i] : x[i + n], keep = up ? x[i + n] : x[i];
            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, m);
        }
    }
    return x[0] + __shfl_xor_sync(0xffffffffu, x[0], 1);
}

// sum_lane x[i] for 32 values i: lane i returns the sum of value i.  Every step halves the values.
__device__ __forceinline__ float transpose_sum(float (&x)[32])
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int m = 16; m >= 1; m >>= 1) {
        const bool up = lane & m;
#pragma unroll
        for (int i = 0; i < m; ++i) {
            const float give = up ? x[i] : x[i + m], keep = up ? x[i + m] : x[i];
            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, m);
        }
    }
    return x[0];
}

template <int D>
__global__ void __launch_bounds__(kWalkThreads, 1)
    delta_back_kernel(const __grid_constant__ CUtensorMap tmap_q,
                      const __grid_constant__ CUtensorMap tmap_k,
                      const __grid_constant__ CUtensorMap tmap_do,
                      const __grid_constant__ CUtensorMap tmap_e, BackArgs x)
{
    using W = Walk<D>;
    using B = Back<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);  // (stays a shared-memory pointer)
    const uint32_t sb = smem_u32(sm);
    __shared__ uint64_t full[B::ST], empty[B::ST], s_ready[2], s_full[2], x_full, r_ready, e_full, u_ready;
    __shared__ uint32_t tmem_base_sh;
    __shared__ volatile int abort_flag;

    const Packed& pk = x.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int h = blockIdx.x % pk.H, s = blockIdx.x / pk.H, hk = h / (pk.H / pk.Hk);
    int lo, hi;
    seq_rows(x.cu, s, pk.T, lo, hi);
    const int chunks = (hi - lo + kC - 1) / kC;
    const size_t rec0 = ((size_t)(lo / kC + s)) * pk.H + h;

    if (tid == 0) {
        for (int i = 0; i < B::ST; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 2 * W::WARPS + 1);
        }
        for (int i = 0; i < W::PIECES; ++i) {
            mbar_init(&s_ready[i], W::WARPS);
            mbar_init(&s_full[i], 1);
        }
        mbar_init(&r_ready, W::WARPS);
        mbar_init(&u_ready, W::WARPS);
        mbar_init(&x_full, 1);
        mbar_init(&e_full, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == W::MMA) {
        tmem_alloc(&tmem_base_sh, 512);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tm = tmem_base_sh;
    if (tm != 0 && tid == 0) {  // (cannot be; nothing is issued then)
        abort_flag = 1;
        if (x.status) atomicExch(x.status, (int)FLEX_ECUDA);
    }
    // step r works on chunk chunks - 1 - r
    auto stage = [&](int r) { return (uint32_t)(r % B::ST) * B::STAGE; };
    auto landed = [&](int r) {
        return bar_wait_w(&full[r % B::ST], (uint32_t)(r / B::ST) & 1, &abort_flag, x.status);
    };

    // registers: launched with 96 a thread; 4 x 104 + 64 = 480 = 5 x 96
    if (warp >= 16) {
        setmaxnreg_dec<64>();
        if (warp == W::TMA) {
            for (int r = 0; r < chunks; ++r) {
                uint64_t* bar = &full[r % B::ST];
                if (r >= B::ST &&
                    !bar_wait_w(&empty[r % B::ST], (uint32_t)(r / B::ST - 1) & 1, &abort_flag, x.status))
                    break;
                const uint32_t st = sb + stage(r);
                const int c = chunks - 1 - r, t = lo + c * kC;
                wmbar_arrive_expect_tx(bar, 5 * B::TILE + B::REC_BYTES);
                for (int b = 0; b < D / 64; ++b) {
                    wtma_load_3d(st + B::DO + 8192 * b, &tmap_do, 64 * b, h, t, bar);
                    wtma_load_3d(st + B::K + 8192 * b, &tmap_k, 64 * b, hk, t, bar);
                    wtma_load_3d(st + B::Q + 8192 * b, &tmap_q, 64 * b, hk, t, bar);
                }
                wtma_load_3d(st + B::E, &tmap_e, 0, 0, (int)(rec0 + (size_t)c * pk.H), bar);
                if (elect_one())
                    bulk_load(st + B::REC, x.rec + (rec0 + (size_t)c * pk.H) * Rec::BYTES + Rec::M_HI,
                              B::REC_BYTES, bar);
            }
        } else if (warp == W::MMA && tm == 0) {
            constexpr uint32_t I_C = idesc_bf16(128, kC, 0, 0), I_CM = idesc_bf16(128, kC, 0, 1);
            constexpr uint32_t I_P = idesc_bf16(128, kC, 1, 1), I_D = idesc_bf16(128, 64, 0, 1);
            bool ok = true;
            auto wait = [&](uint64_t* bar, int phase) {
                if (ok) ok = bar_wait_w(bar, (uint32_t)phase & 1, &abort_flag, x.status);
                fence_after_sync();
            };
            for (int r = 0; r < chunks && ok; ++r) {
                const uint32_t st = sb + stage(r);
                const int n = hi - lo - (chunks - 1 - r) * kC;
                ok = landed(r);
                if (!ok) break;
                if (n < kC) {  // rows behind the sequence's end are another's, and 0 * NaN is NaN
                    for (int e = n * 8 + lane; e < kC * 8; e += 32)
                        for (int b = 0; b < 3 * D / 64; ++b)  // K, Q, dO
                            st_shared_v4(st + 8192 * b + e * 16, 0, 0, 0, 0);
                    fence_proxy_async();
                    __syncwarp();
                }
                const uint32_t dk = dlow(st + B::K, 16), dkn = dlow(st + B::K, 8192);
                const uint32_t dqn = dlow(st + B::Q, 8192), dod = dlow(st + B::DO, 8192);
                const uint32_t dm = dlow(st + B::M, 16), dp = dlow(st + B::P, 16);
#pragma unroll
                for (int k = 0; k < 8; ++k)  // P^T dO, A across the rows of dO; P_LO follows P
                    wmma_bf16(B::T_P, desc(dod, 2048 * (k & 3)), desc(dp, 2048 * k), I_P, k > 0);
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
                    wait(&s_ready[p], r);
                    if (!ok) break;
                    mma4(B::T_X, B::T_S + 32 * p, dk + 512 * p, 32, I_C, p > 0);
                }
                if (!ok) break;
                wmma_commit(&x_full);
                wait(&r_ready, r);
                if (!ok) break;
                mma4(B::T_X, B::T_A, dm, 2048, I_CM, 0);
                wmma_commit(&e_full);
                // The first chunk's increment is used by nobody, and nobody would wait for it: the
                // block would free its tensor memory with products on their way into it.
                if (r + 1 == chunks) break;
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) mma4(B::T_D + 64 * p, B::T_O, dqn + 512 * p, 2048, I_D, 0);
                wait(&u_ready, r);
                if (!ok) break;
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
                    mma4(B::T_D + 64 * p, B::T_R, dkn + 512 * p, 2048, I_D, 1);
                    wmma_commit(&s_full[p]);
                }
                if (r + B::ST < chunks) wmma_commit(&empty[r % B::ST]);  // (see the forward's)
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
            // ---- the state's gradient ----
            uint64_t S[W::PIECES][16];  // pairs of key dimensions 64 p + 32 half + 0 .. 31
#pragma unroll
            for (int p = 0; p < W::PIECES; ++p)
#pragma unroll
                for (int i = 0; i < 16; ++i) S[p][i] = f2_pack(0.f, 0.f);
            uint64_t decay = f2_pack(1.f, 1.f);
            for (int r = 0; r < chunks; ++r) {
                __nv_bfloat16* ds = x.ds + ((rec0 + (size_t)(chunks - 1 - r) * pk.H) * D + v) * D + 32 * half;
#pragma unroll
                for (int p = 0; p < W::PIECES; ++p) {
                    if (r > 0 && !wait(&s_full[p], r - 1)) break;
                    const uint32_t inc = lanes + B::T_D + 64 * p + 32 * half;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        if (r > 0) {  // S = decay S + the increment of the chunk behind
                            float a[16];
                            tmem_ld16(inc + 16 * j, a);
                            tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                S[p][8 * j + e] = f2_fma(decay, S[p][8 * j + e], f2_pack(a[2 * e], a[2 * e + 1]));
                        }
                        uint32_t w[8];
                        pack8(S[p] + 8 * j, w);
                        tmem_st8(lanes + B::T_S + 32 * p + 16 * half + 8 * j, w);
                    }
                    ready(&s_ready[p]);
                }
                if (ok) {  // (rounded again: the walk waits for the pieces)
#pragma unroll
                    for (int p = 0; p < W::PIECES; ++p)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            uint32_t w[8];
                            pack8(S[p] + 8 * j, w);
                            store_32b(ds + 64 * p + 16 * j, make_uint4(w[0], w[1], w[2], w[3]),
                                      make_uint4(w[4], w[5], w[6], w[7]));
                        }
                }
                if (!ok || !(ok = landed(r))) break;
                const float last = *(const float*)(sm + stage(r) + B::AUX + Rec::LAST - Rec::AUX);
                decay = f2_pack(last, last);
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty[r % B::ST]);
            }
        } else {
            // ---- the tokens ----
            const size_t os = (size_t)pk.H * D;
            __nv_bfloat16* dv = x.dv + (size_t)(lo + 32 * half + (lane & 1)) * os + h * D + (v & ~1);
            const uint32_t pick = lane & 1 ? 0x3276u : 0x5410u;
            const uint64_t minus = f2_pack(-1.f, -1.f), factor = f2_pack(-x.scale, -x.scale);
            for (int r = 0; r < chunks; ++r) {
                const int c = chunks - 1 - r, n = hi - lo - c * kC - 32 * half;
                const size_t slot = rec0 + (size_t)c * pk.H;
                if (!(ok = landed(r))) break;
                const uint8_t* st = sm + stage(r);
                const float* aux = (const float*)(st + B::AUX) + 32 * half;
                constexpr int kG = 0, kK = (Rec::KAPPA - Rec::AUX) / 4, kB = (Rec::BETA - Rec::AUX) / 4;
                // the products of the last step have read scale e^G dO
                if (r > 0 && !wait(&s_full[W::PIECES - 1], r - 1)) break;
                {
                    const uint8_t* col = st + B::DO + (uint32_t)(v >> 6) * 8192 + half * 4096;
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const uint32_t a = *(const uint16_t*)(col + swz128(2 * i, v & 63));
                        const uint32_t b = *(const uint16_t*)(col + swz128(2 * i + 1, v & 63));
                        const uint64_t gm = *(const uint64_t*)(aux + kG + 2 * i);
                        float y, z;
                        f2_unpack(f2_mul(f2_mul(factor, gm), f2_pack(__uint_as_float(a << 16), __uint_as_float(b << 16))), y, z);
                        w[i] = pack_bf16(2 * i < n ? y : 0.f, 2 * i + 1 < n ? z : 0.f);
                    }
                    tmem_st16(lanes + B::T_O + 16 * half, w);
                }
                if (!wait(&x_full, r)) break;
                uint64_t U[16];  // dU, then Y: pairs of tokens
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16], y[16];
                    tmem_ld16(lanes + B::T_X + 32 * half + 16 * j, d);
                    tmem_ld16(lanes + B::T_P + 32 * half + 16 * j, y);
                    tmem_wait_ld();
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint64_t kp = *(const uint64_t*)(aux + kK + 16 * j + 2 * i);
                        const uint64_t bt = *(const uint64_t*)(aux + kB + 16 * j + 2 * i);
                        U[8 * j + i] = f2_fma(kp, f2_pack(d[2 * i], d[2 * i + 1]), f2_pack(y[2 * i], y[2 * i + 1]));
                        float a, b;
                        f2_unpack(f2_mul(bt, U[8 * j + i]), a, b);
                        w[i] = pack_bf16(a, b);
                    }
                    tmem_st8(lanes + B::T_A + 16 * half + 8 * j, w);
                }
                ready(&r_ready);
                if (!wait(&e_full, r)) break;
                uint32_t wv[16];  // dV
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float d[16];
                    tmem_ld16(lanes + B::T_X + 32 * half + 16 * j, d);
                    tmem_wait_ld();
                    uint32_t w[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint64_t gm = *(const uint64_t*)(aux + kG + 16 * j + 2 * i);  // -e^G
                        const uint64_t bt = *(const uint64_t*)(aux + kB + 16 * j + 2 * i);
                        U[8 * j + i] = f2_fma(f2_pack(d[2 * i], d[2 * i + 1]), minus, U[8 * j + i]);
                        const uint64_t y = f2_mul(bt, U[8 * j + i]);
                        float a, b;
                        f2_unpack(y, a, b);
                        wv[8 * j + i] = pack_bf16(a, b);
                        f2_unpack(f2_mul(gm, y), a, b);
                        w[i] = pack_bf16(a, b);
                    }
                    tmem_st8(lanes + B::T_R + 16 * half + 8 * j, w);
                }
                ready(&u_ready);
                __nv_bfloat16* dst = dv + (size_t)(c * kC) * os;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const uint32_t y = __byte_perm(wv[i], __shfl_xor_sync(0xffffffffu, wv[i], 1), pick);
                    if (2 * i + (lane & 1) < n) *(uint32_t*)dst = y;
                    dst += 2 * os;
                }
                float prod[32];  // E . Y of this lane's value dimension
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint4 eh = *(const uint4*)(st + B::E + swz128(v, 32 * half + 8 * i));
                    const uint4 el = *(const uint4*)(st + B::E + D * 128 + swz128(v, 32 * half + 8 * i));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t y = (&eh.x)[e], z = (&el.x)[e];
                        float a, b;
                        f2_unpack(U[4 * i + e], a, b);
                        prod[8 * i + 2 * e] = a * (__uint_as_float(y << 16) + __uint_as_float(z << 16));
                        prod[8 * i + 2 * e + 1] = b * (__uint_as_float(y & 0xffff0000u) + __uint_as_float(z & 0xffff0000u));
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&empty[r % B::ST]);
                x.db[(slot * 4 + (warp & 3)) * 64 + 32 * half + lane] = transpose_sum(prod);
            }
        }
        fence_before_sync();
    }
    __syncthreads();
    drain_after_abort(abort_flag);
    if (warp == W::MMA) {
        fence_after_sync();
        tmem_dealloc(tm, 512);
    }
}

// ---- backward, the gradients of every chunk ----------------------------------------------
// With S the state ahead of the chunk, D the gradient of the one behind, and the walk's dV:
//   Zq = scale tril(Y o dO U^T),  Zk = -tril(Y o dV U^T, -1)       (U = beta E)
//   dQ = scale e^G (dO S^T) + Zq K
//   dK = Zq^T Q + (Zk + Zk^T) K + e^{G_C - G} (U D^T) - e^G (dV S^T)
//   dg_t = sum_{i >= t > j} W_ij + sum_{i >= t} a_i + sum_{j < t} b_j + e^{G_C} <S, D>,
//   W = Zq o Q K^T + Zk o K K^T,  a_i = scale e^G q_i.(S dO_i) - e^G k_i.(S dV_i),
//   b_j = e^{G_C - G_j} beta_j k_j.(D E_j)
// (W as sum_{j < t} of its column j minus its row j: the sums are of the same fp32 values, so what
// cancels does so exactly.)  One CTA of 8 warps per (chunk, key head) runs over the heads that share
// it; dQ^T and dK^T are products of key dimension x token, summed over the heads in registers: a
// lane holds one key dimension (quadrant w % 4) and a warp half of the tokens (w / 4).  256 columns
// of tensor memory, taken twice: [dO E, dV E | Q K^T, K K^T | S dO | S dV], then [Zq K | Zq^T Q +
// (Zk + Zk^T) K | D E], E and Zq as high and low parts.  For d = 64 products have rows 64-127 that read
// whatever lies behind a tile (within shared memory) and are not looked at.
template <int D>
struct Grad {
    static constexpr uint32_t TILE = kC * D * 2, BLOCK = D * 128;  // 64 tokens; D rows of 64 elements
    // [Q; K] and [dO; dV]: per 64 elements, 64 rows of the one and 64 of the other
    // (E and Zq: high parts, then low ones)
    static constexpr uint32_t QK = 0, OV = 2 * TILE, E = 4 * TILE, S = E + 2 * BLOCK, DS = S + BLOCK * (D / 64),
                              ZQ = DS + BLOCK * (D / 64), ZK = ZQ + 16384, END = ZK + 8192;
    static constexpr uint32_t SMEM = END + 1024;
};

struct GradArgs {
    Packed p;
    const int* cu;
    float scale;
    const uint8_t* rec;
    const float* db;
    const __nv_bfloat16* g;
    __nv_bfloat16 *dq, *dk, *dg, *dbeta;
    int* status;
};

template <int D>
__global__ void __launch_bounds__(256, D == 64 ? 2 : 1)
    delta_grad_kernel(const __grid_constant__ CUtensorMap tmap_q,
                      const __grid_constant__ CUtensorMap tmap_k,
                      const __grid_constant__ CUtensorMap tmap_do,
                      const __grid_constant__ CUtensorMap tmap_dv,
                      const __grid_constant__ CUtensorMap tmap_e,
                      const __grid_constant__ CUtensorMap tmap_s,
                      const __grid_constant__ CUtensorMap tmap_ds, GradArgs x)
{
    using L = Grad<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);  // (stays a shared-memory pointer)
    const uint32_t sb = smem_u32(sm);
    __shared__ uint64_t bar_load, bar_mma;
    __shared__ uint32_t tmem_base_sh;
    __shared__ volatile int abort_flag;
    __shared__ __align__(16) float aux[256];  // -e^G, e^{G_C - G}, beta, G (in powers of two)
    __shared__ __align__(16) float sums_a[4][64], sums_b[4][64], cols[4][64], rows[2][128], ab[2][64], dots[8], last_sh;

    const Packed& pk = x.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, hk = blockIdx.y, G = pk.H / pk.Hk;
    int s, chunk, lo, hi;
    if (!find_block(x.cu, pk.n, pk.T, kC, (int)blockIdx.x, s, chunk, lo, hi)) return;
    const int t0 = lo + chunk * kC, n = min(kC, hi - t0);
    if (tid == 0) {
        mbar_init(&bar_load, 1);
        mbar_init(&bar_mma, 1);
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == 0) {
        tmem_alloc(&tmem_base_sh, 256);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tm = tmem_base_sh;
    const int quad = warp & 3, half = warp >> 2, kd = 32 * quad + lane;
    const bool mine = kd < D;  // this lane holds a key dimension (whole warps)
    const uint32_t lanes = tm + ((uint32_t)quad << 21);
    uint64_t dq[16], dk[16];  // pairs of tokens 32 half + 0 .. 31
#pragma unroll
    for (int i = 0; i < 16; ++i) dq[i] = dk[i] = f2_pack(0.f, 0.f);
    grid_dep_wait();  // dV, D and the products E . Y
    bool ok = true;
    uint32_t ph = 0, ph_mma = 0;
    auto products_done = [&] {  // every thread; false when a wait gave up
        ok = bar_wait_w(&bar_mma, ph_mma, &abort_flag, x.status);
        ph_mma ^= 1;
        fence_after_sync();
        return ok;
    };
    for (int h = hk * G; h < (hk + 1) * G; ++h) {
        const size_t slot = (size_t)blockIdx.x * pk.H + h;
        if (warp == 0) {
            wmbar_arrive_expect_tx(&bar_load, 2 * L::TILE + L::BLOCK * (2 + 2 * (D / 64)) +
                                                  (h == hk * G ? 2 * L::TILE : 0));
            for (int b = 0; b < D / 64; ++b) {
                if (h == hk * G) {
                    wtma_load_3d(sb + L::QK + 16384 * b, &tmap_q, 64 * b, hk, t0, &bar_load);
                    wtma_load_3d(sb + L::QK + 16384 * b + 8192, &tmap_k, 64 * b, hk, t0, &bar_load);
                }
                wtma_load_3d(sb + L::OV + 16384 * b, &tmap_do, 64 * b, h, t0, &bar_load);
                wtma_load_3d(sb + L::OV + 16384 * b + 8192, &tmap_dv, 64 * b, h, t0, &bar_load);
                wtma_load_3d(sb + L::S + L::BLOCK * b, &tmap_s, 64 * b, 0, (int)slot, &bar_load);
                wtma_load_3d(sb + L::DS + L::BLOCK * b, &tmap_ds, 64 * b, 0, (int)slot, &bar_load);
            }
            wtma_load_3d(sb + L::E, &tmap_e, 0, 0, (int)slot, &bar_load);
        }
        const float* rec = (const float*)(x.rec + slot * Rec::BYTES + Rec::AUX);
        aux[tid] = rec[tid];
        if (tid == 0) last_sh = rec[256];
        ok = bar_wait_w(&bar_load, ph, &abort_flag, x.status);
        ph ^= 1;
        if (h == hk * G && n < kC && ok) {  // rows behind the end are another's, and 0 * NaN is NaN
            for (int e = n * 8 + tid; e < kC * 8; e += 256)
                for (int b = 0; b < 2 * (D / 64); ++b)
                    st_shared_v4(sb + L::QK + 8192 * b + e * 16, 0, 0, 0, 0);
            fence_proxy_async();
        }
        if (!__syncthreads_and(ok)) {
            ok = false;
            break;
        }
        fence_after_sync();  // the other warps' loads of the head before, whose columns are overwritten
        const uint32_t qk = dlow(sb + L::QK, 16), ov = dlow(sb + L::OV, 16), de = dlow(sb + L::E, 8192);
        if (warp == 0) {
#pragma unroll
            for (int k = 0; k < D / 8; ++k) {  // (E low follows E)
                const uint32_t o = (k % (D / 16) >> 2) * 16384 + (k & 3) * 32;
                wmma_bf16(tm, desc(ov, o), desc(de, 2048 * k), idesc_bf16(128, kC, 0, 1), k > 0);
            }
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t o = (k >> 2) * 16384 + (k & 3) * 32;
                wmma_bf16(tm + 64, desc(qk, o), desc(qk, o + 8192), idesc_bf16(128, kC, 0, 0), k > 0);
            }
#pragma unroll
            for (int y = 0; y < 2; ++y)
#pragma unroll
                for (int k = 0; k < D / 16; ++k)
                    wmma_bf16(tm + 128 + 64 * y, desc(dlow(sb + L::S, L::BLOCK), 2048 * k),
                              desc(ov, 8192 * y + (k >> 2) * 16384 + (k & 3) * 32),
                              idesc_bf16(128, kC, 1, 0), k > 0);
            wmma_commit(&bar_mma);
        }
        {  // <S, D> while the products run
            float dot = 0.f;
            for (int e = tid; e < D * D / 8; e += 256) {
                const uint4 a = *(const uint4*)(sm + L::S + 16 * e), b = *(const uint4*)(sm + L::DS + 16 * e);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t u = (&a.x)[i], w = (&b.x)[i];
                    dot = fmaf(__uint_as_float(u << 16), __uint_as_float(w << 16), dot);
                    dot = fmaf(__uint_as_float(u & 0xffff0000u), __uint_as_float(w & 0xffff0000u), dot);
                }
            }
#pragma unroll
            for (int m = 1; m < 32; m *= 2) dot += __shfl_xor_sync(0xffffffffu, dot, m);
            if (lane == 0) dots[warp] = dot;
        }
        ok = products_done();
        if (ok) {
            // Z: row i = kd % 64 of Zq (quadrants 0, 1) or Zk, columns 32 half + 0 .. 31
            const int i = kd & 63;
            const bool key = quad >= 2;
            // (G without its low part leaves a decay off by 3.4e-4 at most; Z is rounded by up to 2^-8)
            const float Gi = aux[192 + i], f = key ? -1.f : x.scale;
            const int jmax = (i < n ? (key ? i : i + 1) : 0) - 32 * half;  // columns below it count
            const uint32_t dst = sb + (key ? L::ZK : L::ZQ);
            const bool none = half == 1 && !(quad & 1);  // all of this warp's lies above the diagonal
            float row = 0.f;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                uint32_t w[8] = {}, wl[8] = {};
                float col = 0.f;
                if (!none) {
                    float c1[16], W[16];
                    tmem_ld16(lanes + 32 * half + 16 * y, c1);
                    tmem_ld16(lanes + 64 + 32 * half + 16 * y, W);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const float4 bt = *(const float4*)&aux[128 + 32 * half + 16 * y + j];
                        const float4 gj = *(const float4*)&aux[192 + 32 * half + 16 * y + j];
                        const float b4[4] = {bt.x, bt.y, bt.z, bt.w}, g4[4] = {gj.x, gj.y, gj.z, gj.w};
                        float z[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const bool in = 16 * y + j + e < jmax;
                            z[e] = in ? f * b4[e] * ex2(Gi - g4[e]) * c1[j + e] : 0.f;
                            W[j + e] = in ? z[e] * W[j + e] : 0.f;
                            row += W[j + e];
                        }
                        split(z[0], z[1], w[j / 2], wl[j / 2]);
                        split(z[2], z[3], w[j / 2 + 1], wl[j / 2 + 1]);
                    }
                    col = transpose_sum16(W);
                }
                st_shared_v4(dst + swz128(i, 32 * half + 16 * y), w[0], w[1], w[2], w[3]);
                st_shared_v4(dst + swz128(i, 32 * half + 16 * y + 8), w[4], w[5], w[6], w[7]);
                if (!key) {
                    st_shared_v4(dst + 8192 + swz128(i, 32 * half + 16 * y), wl[0], wl[1], wl[2], wl[3]);
                    st_shared_v4(dst + 8192 + swz128(i, 32 * half + 16 * y + 8), wl[4], wl[5], wl[6], wl[7]);
                }
                if (!(lane & 1)) cols[quad][32 * half + 16 * y + lane / 2] = col;
            }
            rows[half][kd] = row;
        }
        const uint8_t* qcol = sm + L::QK + (kd >> 6) * 16384 + half * 4096;
        if (ok && mine) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float dot[16];
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const int c0 = 32 * half + 16 * y + 8 * z;
                    float a[8], b[8];
                    tmem_ld8(lanes + 128 + c0, a);
                    tmem_ld8(lanes + 192 + c0, b);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 8; j += 4) {
                        const float4 g4 = *(const float4*)&aux[c0 + j];
                        const float gm[4] = {g4.x, g4.y, g4.z, g4.w};  // -e^G
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int jj = 16 * y + 8 * z + j + e;
                            const bool in = 32 * half + jj < n;
                            a[j + e] = in ? -x.scale * gm[e] * a[j + e] : 0.f;
                            b[j + e] = in ? gm[e] * b[j + e] : 0.f;
                            const uint32_t qv = *(const uint16_t*)(qcol + swz128(jj, kd & 63));
                            const uint32_t kv = *(const uint16_t*)(qcol + 8192 + swz128(jj, kd & 63));
                            dot[8 * z + j + e] = a[j + e] * __uint_as_float(qv << 16) + b[j + e] * __uint_as_float(kv << 16);
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const int at = 8 * y + 4 * z + j / 2;
                        dq[at] = f2_fma(f2_pack(a[j], a[j + 1]), f2_pack(1.f, 1.f), dq[at]);
                        dk[at] = f2_fma(f2_pack(b[j], b[j + 1]), f2_pack(1.f, 1.f), dk[at]);
                    }
                }
                const float sum = transpose_sum16(dot);
                if (!(lane & 1)) sums_a[quad][32 * half + 16 * y + lane / 2] = sum;
            }
        }
        fence_proxy_async();  // Z
        fence_before_sync();
        if (!__syncthreads_and(ok)) {
            ok = false;
            break;
        }
        fence_after_sync();
        if (warp == 0) {
            const uint32_t zq = dlow(sb + L::ZQ, 16), zk = dlow(sb + L::ZK, 16);
            const uint32_t zqn = dlow(sb + L::ZQ, 8192), zkn = dlow(sb + L::ZK, 8192);
            const uint32_t qn = dlow(sb + L::QK, 16384), kn = dlow(sb + L::QK + 8192, 16384);
            constexpr uint32_t I_KM = idesc_bf16(128, kC, 1, 0), I_MM = idesc_bf16(128, kC, 1, 1);
#pragma unroll
            for (int k = 0; k < 8; ++k)  // (high, then low parts of Zq)
                wmma_bf16(tm, desc(kn, 2048 * (k & 3)), desc(zq, (k >> 2) * 8192 + 32 * (k & 3)), I_KM, k > 0);
#pragma unroll
            for (int k = 0; k < 8; ++k)
                wmma_bf16(tm + 64, desc(qn, 2048 * (k & 3)), desc(zqn, 2048 * k), I_MM, k > 0);
#pragma unroll
            for (int k = 0; k < 4; ++k) wmma_bf16(tm + 64, desc(kn, 2048 * k), desc(zkn, 2048 * k), I_MM, 1);
#pragma unroll
            for (int k = 0; k < 4; ++k) wmma_bf16(tm + 64, desc(kn, 2048 * k), desc(zk, 32 * k), I_KM, 1);
#pragma unroll
            for (int k = 0; k < D / 8; ++k)
                wmma_bf16(tm + 128, desc(dlow(sb + L::DS, L::BLOCK), 2048 * (k % (D / 16))), desc(de, 2048 * k), I_MM, k > 0);
            wmma_commit(&bar_mma);
        }
        ok = products_done();
        if (ok && mine) {
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                float dot[16];
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const int c0 = 32 * half + 16 * y + 8 * z;
                    float a[8], b[8], e2[8];
                    tmem_ld8(lanes + c0, a);         // Zq K
                    tmem_ld8(lanes + 64 + c0, b);    // Zq^T Q + (Zk + Zk^T) K
                    tmem_ld8(lanes + 128 + c0, e2);  // D E
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 8; j += 4) {
                        const float4 k4 = *(const float4*)&aux[64 + c0 + j], b4 = *(const float4*)&aux[128 + c0 + j];
                        const float kb[4] = {k4.x * b4.x, k4.y * b4.y, k4.z * b4.z, k4.w * b4.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int jj = 16 * y + 8 * z + j + e;
                            const uint32_t kv = *(const uint16_t*)(qcol + 8192 + swz128(jj, kd & 63));
                            const float write = kb[e] * e2[j + e];
                            dot[8 * z + j + e] = write * __uint_as_float(kv << 16);
                            b[j + e] += write;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 8; j += 2) {
                        const int at = 8 * y + 4 * z + j / 2;
                        dq[at] = f2_fma(f2_pack(a[j], a[j + 1]), f2_pack(1.f, 1.f), dq[at]);
                        dk[at] = f2_fma(f2_pack(b[j], b[j + 1]), f2_pack(1.f, 1.f), dk[at]);
                    }
                }
                const float sum = transpose_sum16(dot);
                if (!(lane & 1)) sums_b[quad][32 * half + 16 * y + lane / 2] = sum;
            }
        }
        fence_before_sync();
        if (!__syncthreads_and(ok)) {  // (also: tensor memory and the tiles are free for the next head)
            ok = false;
            break;
        }
        if (tid < 64) {
            float A = 0.f, B = 0.f;
#pragma unroll
            for (int y = 0; y < D / 32; ++y) {
                A += sums_a[y][tid];
                B += sums_b[y][tid];
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) B += cols[y][tid];
            B -= (rows[0][tid] + rows[1][tid]) + (rows[0][64 + tid] + rows[1][64 + tid]);
            ab[0][tid] = A;
            ab[1][tid] = B;
        }
        __syncthreads();
        if (tid < n) {
            float g = 0.f, db = 0.f;
#pragma unroll
            for (int y = 0; y < 8; ++y) g += dots[y];
            g *= last_sh;
            float behind = 0.f, ahead = 0.f;
#pragma unroll
            for (int j = 0; j < 64; j += 4) {
                const float4 a4 = *(const float4*)&ab[0][j], b4 = *(const float4*)&ab[1][j];
                behind += (j >= tid ? a4.x : b4.x) + (j + 1 >= tid ? a4.y : b4.y);
                ahead += (j + 2 >= tid ? a4.z : b4.z) + (j + 3 >= tid ? a4.w : b4.w);
            }
            g += behind + ahead;
            const float* part = x.db + slot * 256 + tid;
#pragma unroll
            for (int y = 0; y < D / 32; ++y) db += part[64 * y];
            const size_t at = (size_t)(t0 + tid) * pk.H + h;
            // (a reset, a_t = 0: the sums leave their rounding where dg is 0)
            x.dg[at] = __float2bfloat16_rn(__bfloat162float(x.g[at]) <= kLeastGate ? 0.f : g);
            x.dbeta[at] = __float2bfloat16_rn(db);
        }
        __syncthreads();
    }
    if (ok && mine) {  // neighbouring lanes exchange halves of two rows: each writes two elements of one
        const uint32_t pick = lane & 1 ? 0x3276u : 0x5410u;
        const size_t os = (size_t)pk.Hk * D;
        const size_t at = (size_t)(t0 + 32 * half + (lane & 1)) * os + hk * D + (kd & ~1);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            float a, b;
            f2_unpack(dq[i], a, b);
            const uint32_t w = pack_bf16(a, b);
            f2_unpack(dk[i], a, b);
            const uint32_t y = pack_bf16(a, b);
            const uint32_t w2 = __byte_perm(w, __shfl_xor_sync(0xffffffffu, w, 1), pick);
            const uint32_t y2 = __byte_perm(y, __shfl_xor_sync(0xffffffffu, y, 1), pick);
            if (32 * half + 2 * i + (lane & 1) < n) {
                *(uint32_t*)(x.dq + at + 2 * i * os) = w2;
                *(uint32_t*)(x.dk + at + 2 * i * os) = y2;
            }
        }
    }
    __syncthreads();
    drain_after_abort(abort_flag);
    if (warp == 0) {
        fence_after_sync();
        tmem_dealloc(tm, 256);
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
    const auto kernel = x.e_save ? delta_walk_kernel<D, true> : delta_walk_kernel<D, false>;
    cudaError_t e = cudaFuncSetAttribute(delta_prep_kernel<D>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, prep);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, walk);
    if (e == cudaSuccess)
        e = launch_after(delta_prep_kernel<D>,
                         dim3((unsigned)block_slots(p.T, p.n, kC), (unsigned)p.H), 128, prep, 0, false,
                         s, mq, mk, p, (const __nv_bfloat16*)g, (const __nv_bfloat16*)beta, x.cu,
                         x.scale, rec, x.status);
    if (e == cudaSuccess)
        e = launch_after(kernel, dim3((unsigned)(p.n * p.H)), kWalkThreads, walk, 0,
                         true, s, mq, mk, mv, x);
    return e;
}

template <int D>
cudaError_t back(const Packed& p, const void* q, const void* k, const void* dout, const void* e,
                 const void* st, BackArgs& x, GradArgs& g, cudaStream_t s)
{
    CUtensorMap mq, mk, mo, mv, me, ms, md;
    const int slots = block_slots(p.T, p.n, kC) * p.H;
    if (!make_chunk_map(&mq, q, p.T, p.Hk, D, p.qs) || !make_chunk_map(&mk, k, p.T, p.Hk, D, p.ks) ||
        !make_chunk_map(&mo, dout, p.T, p.H, D, (long long)p.H * D) ||
        !make_chunk_map(&mv, x.dv, p.T, p.H, D, (long long)p.H * D) ||
        !make_feat_map(&me, e, slots, 2 * D, kC, 2 * D) || !make_feat_map(&ms, st, slots, D, D, D) ||
        !make_feat_map(&md, x.ds, slots, D, D, D))
        return cudaErrorInvalidValue;
    const int walk = (int)Back<D>::SMEM, grad = (int)Grad<D>::SMEM;
    cudaError_t r = cudaFuncSetAttribute(delta_back_kernel<D>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, walk);
    if (r == cudaSuccess)
        r = cudaFuncSetAttribute(delta_grad_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, grad);
    if (r == cudaSuccess)
        r = launch_after(delta_back_kernel<D>, dim3((unsigned)(p.n * p.H)), kWalkThreads, walk, 0,
                         false, s, mq, mk, mo, me, x);
    if (r == cudaSuccess)
        r = launch_after(delta_grad_kernel<D>,
                         dim3((unsigned)block_slots(p.T, p.n, kC), (unsigned)p.Hk), 256, grad, 0, true,
                         s, mq, mk, mo, mv, me, ms, md, g);
    return r;
}

// The parts of a save buffer: records, E^T (high and low parts), S^T.
struct SaveParts {
    size_t e, s, total;
};
SaveParts save_parts(const Packed& p)
{
    const size_t slots = (size_t)block_slots(p.T, p.n, kC) * p.H;
    SaveParts x;
    x.e = align_up(slots * Rec::BYTES, 256);
    x.s = x.e + slots * 2 * p.d * kC * 2;
    x.total = x.s + slots * p.d * p.d * 2;
    return x;
}

}  // namespace

// By the average length (the lengths are on the device).  A walk costs a sequence 10 us and 3.6 us (d =
// 128: 4.4) for each 64 tokens, the scans 0.2 us (0.32) for each token.  Measured, H16, scans / chunks
// in us:
//   d = 64:  64 x 16 tokens 33 / 65, 64 x 32 57 / 66, 64 x 64 107 / 69; training, 64 x 16 128 / 144,
//            64 x 32 233 / 149
//   d = 128: 8 x 16 tokens 24 / 17, 64 x 16 146 / 79, 64 x 64 468 / 85
//   one prompt of 4000 among 100 single tokens: d = 64 797 / 241, d = 128 1280 / 292
// so the chunks take over at 16 and 8 tokens: below what uniform short sequences of d = 64 would
// like, for the sake of prompts among single tokens (too many of which, 266 beside 4000 tokens for
// d = 64, still bring the scans).
bool tc_delta_supported(const Packed& p) { return p.bf16 && (long long)p.T * p.d >= 1024LL * p.n; }

size_t tc_delta_rec_bytes(const Packed& p)
{
    return (size_t)block_slots(p.T, p.n, kC) * p.H * Rec::BYTES;
}
size_t tc_delta_save_bytes(const Packed& p) { return save_parts(p).total; }
size_t tc_delta_bwd_bytes(const Packed& p)  // D^T, then the products E . Y
{
    return (size_t)block_slots(p.T, p.n, kC) * p.H * ((size_t)p.d * p.d * 2 + 4 * 64 * 4);
}

cudaError_t launch_tc_delta_fwd(const Packed& p, const void* q, const void* k, const void* v,
                                const void* g, const void* beta, const int* cu, float scale,
                                const float* S0, float* S1, void* out, void* rec, bool saving,
                                int* status, cudaStream_t s)
{
    WalkArgs x = {};
    x.p = p;
    x.cu = cu; x.scale = scale; x.S0 = S0; x.S1 = S1;
    x.out = (__nv_bfloat16*)out; x.rec = (const uint8_t*)rec; x.status = status;
    if (saving) {
        const SaveParts at = save_parts(p);
        x.e_save = (__nv_bfloat16*)((char*)rec + at.e);
        x.s_save = (__nv_bfloat16*)((char*)rec + at.s);
    }
    return p.d == 64 ? fwd<64>(p, q, k, v, g, beta, x, (uint8_t*)rec, s)
                     : fwd<128>(p, q, k, v, g, beta, x, (uint8_t*)rec, s);
}

cudaError_t launch_tc_delta_bwd(const Packed& p, const void* q, const void* k, const void* g,
                                const int* cu, float scale, const void* dout, const void* save,
                                void* dq, void* dk, void* dv, void* dg, void* dbeta, void* scratch,
                                int* status, cudaStream_t s)
{
    const SaveParts at = save_parts(p);
    const char* base = (const char*)save;
    BackArgs x = {};
    x.p = p;
    x.cu = cu; x.scale = scale; x.rec = (const uint8_t*)save;
    x.ds = (__nv_bfloat16*)scratch;
    x.db = (float*)((char*)scratch + (size_t)block_slots(p.T, p.n, kC) * p.H * p.d * p.d * 2);
    x.dv = (__nv_bfloat16*)dv; x.status = status;
    GradArgs y = {};
    y.p = p;
    y.cu = cu; y.scale = scale; y.rec = (const uint8_t*)save; y.db = x.db;
    y.g = (const __nv_bfloat16*)g;
    y.dq = (__nv_bfloat16*)dq; y.dk = (__nv_bfloat16*)dk; y.dg = (__nv_bfloat16*)dg;
    y.dbeta = (__nv_bfloat16*)dbeta; y.status = status;
    return p.d == 64 ? back<64>(p, q, k, dout, base + at.e, base + at.s, x, y, s)
                     : back<128>(p, q, k, dout, base + at.e, base + at.s, x, y, s);
}

}  // namespace flex
