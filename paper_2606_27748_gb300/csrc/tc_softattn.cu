// Softmax attention over packed sequences on the tensor cores (bf16 storage, d 64 or 128):
// out_i = sum_j softmax_j(scale q_i . k_j) v_j, one pass over the keys with the running maximum
// and sum of every row.
//
// A CTA takes two tiles (short sequences: one) of 128 rows of one sequence and key head.  The G = H / Hk heads that
// share the key head are rows of a tile (row = token * G + head, 128 / G tokens), so K and V
// are read once for all of them, and one TMA box (64 elements, G heads, 128 / G tokens) brings
// a tile in that order.  While one tile's scores are turned into weights, the tensor core works
// on the other tile:
//   warps 0-3, 4-7  softmax of tile A, B: a thread per row
//   then            S = Q K^T (tcgen05, both operands in shared memory) and O += P V (P as bf16 in
//                   tensor memory) issued by one warp that takes the tiles in turn; for d = 64 by a
//                   warp for each
//   the last warp   TMA: Q once, then K and V tiles of 128 keys through a ring of buffers
// Tensor memory (512 columns; one tile 256): S of A and B, O of A and B.  For d = 128 that is all of
// it, P takes the place of its scores, and the products (2050 cycles for a block of 128 keys and both
// tiles) bound the kernel; a warp for each tile's products made it slower (16384 keys, H16 Hk4: 699 ->
// 907 us).  For d = 64 the softmax does (maxima, exponentials and sums in turn, 1350 cycles a tile):
// P has columns of its own, so that the next scores are there when the softmax wants them, and each
// tile's products are issued when that tile is ready (packed prompts 4000, 1531, .., H12: 53 -> 47 us).
// Two threads to a row, 16 softmax warps, were slower for both (764 us, 54 us).
// Sequences of at most 128 rows would leave tile B empty; with one tile a CTA takes half the
// tensor memory and shared memory, and the two CTAs of an SM hide each other's start and end.  Of
// at most 32 rows (single tokens above all) one softmax warp is enough, and only 32 rows of Q are
// kept: the product's other 96 rows read whatever lies behind them and are not looked at.
//
// The maximum that a row's weights refer to only has to keep them in range: it is raised (and
// O and the sum rescaled) when the true one exceeds it by more than 2^8, so after the first
// blocks O is hardly ever touched; the sum and O are exact for any reference.  (A published step of
// such kernels.)
//
// P is rounded to bf16 for its product with V; its sum is taken before.  With random v the error of
// the output's own rounding, 1.5e-3 to 1.7e-3 (2-norm), so becomes 1.9e-3 to 2.3e-3 (sqrt(2) of it at
// most).  A low part of P would do without, but half again the products, which bound d = 128, and a
// conversion more in the softmax, which bounds d = 64.
#include <cuda.h>

#include "flex_internal.h"
#include "softattn.cuh"
#include "tc_util.cuh"

namespace flex {
namespace {

using namespace tc;

constexpr int kKeys = 128;
constexpr float kSlack = 8.f;  // in powers of two

// ROWS: of a CTA, 256 (two tiles), 128 or 32.
template <int D, int ROWS>
struct Lay {
    static constexpr int TILES = ROWS == 256 ? 2 : 1, R = ROWS / TILES;  // rows in use of a tile
    static constexpr bool OWN_P = D == 64;             // see above
    static constexpr int ISSUERS = OWN_P ? TILES : 1;  // warps that issue products
    static constexpr int SW = R / 32, MMA = SW * TILES, TMA = MMA + ISSUERS;
    // whole warpgroups, so that the softmax warps can take registers that the others give back:
    // 384 x 168 = 256 x 216 + 128 x 72; 256 x 128 = 128 x 184 + 128 x 72
    static constexpr int THREADS = ROWS == 32 ? 96 : 128 * (TILES + 1);
    static constexpr int MORE = ROWS == 256 ? 216 : 184, LESS = 72;
    static constexpr uint32_t TILE = 128 * D * 2;  // one K or V tile
    static constexpr uint32_t QB = R * 128, QT = QB * (D / 64);  // 64 elements of a Q tile, a Q tile
    static constexpr int NB = ROWS == 256 ? (D == 128 ? 5 : 8) : ROWS == 128 ? (D == 128 ? 2 : 5) : (D == 128 ? 3 : 6);
    static constexpr uint32_t Q = 0, KV = TILES * QT;
    static constexpr uint32_t SMEM = KV + NB * TILE + 1024;  // + alignment
    static constexpr int T_S = 0, T_O = 128 * TILES, COLS = 256 * TILES;
    static constexpr int T_P = OWN_P ? T_O + D * TILES : T_S, P_STEP = OWN_P ? 64 : 128;  // of a tile
};

struct Bars {
    uint64_t q_full[2], full[8], empty[8], s_full[2], s_loaded[2], p_ready[2], pv_done[2];
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 32 lanes x 32 consecutive columns.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v)
{
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
        "%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
          "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
          "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
          "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
          "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

template <int D, int ROWS>
__global__ void __launch_bounds__(Lay<D, ROWS>::THREADS, ROWS == 256 ? 1 : 2)
    tc_softattn_kernel(const __grid_constant__ CUtensorMap tmap_q,
                       const __grid_constant__ CUtensorMap tmap_k,
                       const __grid_constant__ CUtensorMap tmap_v, AttnArgs x)
{
    using L = Lay<D, ROWS>;
    constexpr int TILES = L::TILES;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* sm = smem_raw + ((0u - smem_u32(smem_raw)) & 1023u);  // (stays a shared-memory pointer)
    const uint32_t sb = smem_u32(sm);
    __shared__ Bars bars;
    __shared__ uint32_t tmem_base_sh;
    __shared__ volatile int abort_flag;

    const Packed& pk = x.p;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int G = pk.H / pk.Hk, tpt = L::R / G;  // tokens of a tile
    const int hk = blockIdx.x % pk.Hk, split = blockIdx.x / pk.Hk;
    int s, block, qlo, qhi, klo, khi;
    if (!find_tile(x, TILES * tpt, (int)(blockIdx.z * gridDim.y + blockIdx.y), s, block, qlo, qhi)) return;
    seq_rows(x.cu_k, s, pk.Tk, klo, khi);
    const int t0 = block * TILES * tpt, rows_left = qhi - qlo - t0;
    const int lk = khi - klo, shift = lk - (qhi - qlo);
    // tokens and key blocks [first, last) of each tile; a tile without tokens takes none
    const int ntA = min(tpt, rows_left), ntB = TILES == 2 ? min(tpt, max(rows_left - tpt, 0)) : 0;
    int firstA, lastA, firstB, lastB;
    key_range(x, kKeys, lk, t0 + ntA - 1 + shift, split, firstA, lastA);
    key_range(x, kKeys, lk, t0 + tpt + ntB - 1 + shift, split, firstB, lastB);
    // The CTA walks over both tiles' blocks.  B's tokens are at most 128 behind A's, so B has at
    // most one block more in all and its range starts at most one block behind A's start: every
    // block of the walk belongs to A or to B, once an empty range is put at the other's start.
    if (ntB == 0) firstB = lastB = firstA;
    if (firstA == lastA) firstA = lastA = firstB;
    if (firstB == lastB) firstB = lastB = firstA;
    const int first = min(firstA, firstB), last = max(lastA, lastB);

    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.q_full[i], 1);
            mbar_init(&bars.s_full[i], 1);
            mbar_init(&bars.p_ready[i], L::SW);
            mbar_init(&bars.s_loaded[i], L::SW);
            mbar_init(&bars.pv_done[i], 1);
        }
        for (int i = 0; i < L::NB; ++i) {
            mbar_init(&bars.full[i], 1);
            mbar_init(&bars.empty[i], L::ISSUERS);
        }
        abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == L::MMA) {
        tmem_alloc(&tmem_base_sh, L::COLS);
        tmem_relinquish();
    }
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    // All of tensor memory starts at its address 0; as a constant it spares the issuing warps moves
    // to uniform registers.
    const uint32_t tm = L::COLS == 512 && L::OWN_P ? 0u : tmem_base_sh;
    if (tmem_base_sh != tm && tid == 0) {  // (cannot be; nothing is issued then)
        abort_flag = 1;
        if (x.status) atomicExch(x.status, (int)FLEX_ECUDA);
    }

    if (warp >= L::MMA) {
    if (ROWS != 32) setmaxnreg_dec<L::LESS>();
    if (tmem_base_sh != tm) {
    } else if (warp == L::TMA) {
        // ---- Q of the tiles at work, then K and V of every block: tile 2 i is K of block first + i,
        // tile 2 i + 1 its V; tile n goes to buffer n % NB ----
        for (int X = 0; X < TILES; ++X) {
            // (an empty range's tile is waited for by nobody, and the CTA may end ahead of its copy)
            if (X ? firstB == lastB : firstA == lastA) continue;
            wmbar_arrive_expect_tx(&bars.q_full[X], (uint32_t)(tpt * G * D * 2));
            for (int b = 0; b < D / 64; ++b)
                wtma_load_3d(sb + L::Q + X * L::QT + b * L::QB, &tmap_q, 64 * b, hk * G,
                             qlo + t0 + X * tpt, &bars.q_full[X]);
        }
        uint32_t ph = 0;  // parity of `empty` per buffer
        for (int n = 0; n < 2 * (last - first); ++n) {
            const int buf = n % L::NB;
            if (n >= L::NB) {
                if (!bar_wait_w(&bars.empty[buf], (ph >> buf) & 1, &abort_flag, x.status)) break;
                ph ^= 1u << buf;
            }
            const int row = klo + (first + n / 2) * kKeys;
            wmbar_arrive_expect_tx(&bars.full[buf], L::TILE);
            for (int b = 0; b < D / 64; ++b)
                wtma_load_3d(sb + L::KV + buf * L::TILE + b * 16384, n & 1 ? &tmap_v : &tmap_k,
                             64 * b, hk, row, &bars.full[buf]);
        }
    } else if (warp < L::TMA) {
        constexpr uint32_t I_S = idesc_bf16(128, kKeys, 0, 0), I_O = idesc_bf16(128, D, 0, 1);
        auto adv = [](uint64_t d, uint32_t bytes) { return d + (bytes >> 4); };
        const int f[2] = {firstA, firstB}, l[2] = {lastA, lastB};
        bool ok = true;
        auto wait = [&](uint64_t* bar, int phase) {
            if (ok) ok = bar_wait_w(bar, (uint32_t)phase & 1, &abort_flag, x.status);
            fence_after_sync();
            return ok;
        };
        // K of block j is tile 2 (j - first), its V the next
        auto buffer = [&](int n) { return sb + L::KV + (uint32_t)(n % L::NB) * L::TILE; };
        auto landed = [&](int n) { return wait(&bars.full[n % L::NB], n / L::NB); };
        // (only where a later load waits for it: no arrival may be on its way when the CTA ends)
        auto again = [&](int n) { return n + L::NB < 2 * (last - first); };
        auto release = [&](int n) {
            if (again(n)) wmma_commit(&bars.empty[n % L::NB]);
        };
        auto scores = [&](int X, int j) {  // S = Q K_j^T
            const int n = 2 * (j - first);
            if (L::OWN_P && (!landed(n) || (j > f[X] && !wait(&bars.s_loaded[X], j - 1 - f[X])))) return;
            const uint64_t dq = sdesc(sb + L::Q + X * L::QT, 16, 1024), dk = sdesc(buffer(n), 16, 1024);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                wmma_bf16(tm + L::T_S + 128 * X, adv(dq, (ks >> 2) * L::QB + (ks & 3) * 32),
                          adv(dk, (ks >> 2) * 16384 + (ks & 3) * 32), I_S, ks > 0);
            wmma_commit(&bars.s_full[X]);
        };
        auto have_v = [&](int j) {
            const int n = 2 * (j - first) + 1;
            // rows behind the sequence's end are another's, and 0 * NaN is NaN (every issuing warp
            // clears them: what it then reads is cleared)
            if (landed(n) && (j + 1) * kKeys > lk) {
                for (int e = (lk - j * kKeys) * 8 + lane; e < kKeys * 8; e += 32)
                    for (int b = 0; b < D / 64; ++b) st_shared_v4(buffer(n) + b * 16384 + e * 16, 0, 0, 0, 0);
                fence_proxy_async();
                __syncwarp();
            }
        };
        auto weighted = [&](int X, int j) {  // O += P V_j
            const int n = 2 * (j - first) + 1;
            if (L::OWN_P) have_v(j);
            if (!wait(&bars.p_ready[X], j - f[X])) return;
            const uint64_t dv = sdesc(buffer(n), 16384, 1024);
#pragma unroll
            for (int ks = 0; ks < kKeys / 16; ++ks)
                wmma_bf16_tmem_a(tm + L::T_O + D * X, tm + L::T_P + L::P_STEP * X + 8 * ks,
                                 adv(dv, ks * 2048), I_O, (j > f[X]) || ks > 0);
            if (L::OWN_P || j + 1 == l[X]) wmma_commit(&bars.pv_done[X]);
        };
        if (L::OWN_P) {
            const int X = warp - L::MMA;
            auto pass = [&](int j) {  // a block of the other tile's only
                for (int n = 2 * (j - first); n < 2 * (j - first) + 2; ++n)
                    if (landed(n) && again(n) && lane == 0) mbar_arrive(&bars.empty[n % L::NB]);
            };
            auto both = [&](int j, bool k, bool v) {  // the scores of block j + 1, then block j's O
                if (k) {
                    scores(X, j + 1);
                    if (ok) release(2 * (j + 1 - first));
                }
                if (v && ok) {
                    weighted(X, j);
                    if (ok) release(2 * (j - first) + 1);
                }
            };
            const int begin = f[X] < l[X] ? f[X] : last, end = f[X] < l[X] ? l[X] : last;
            for (int j = first; j < begin && ok; ++j) pass(j);
            if (begin < end) wait(&bars.q_full[X], 0);
            for (int j = begin - 1; j < end && begin < end && ok; ++j) both(j, j + 1 < end, j >= begin);
            for (int j = end; j < last && ok; ++j) pass(j);
        } else {
            for (int X = 0; X < TILES; ++X)
                if (f[X] < l[X]) wait(&bars.q_full[X], 0);
            for (int j = first - 1; j < last && ok; ++j) {
                bool k_here = false, v_here = false;
                for (int X = 0; X < TILES; ++X) {
                    if (j >= f[X] && j < l[X]) {
                        if (!v_here) have_v(j);
                        v_here = true;
                        if (ok) weighted(X, j);
                    }
                    if (j + 1 >= f[X] && j + 1 < l[X]) {
                        if (!k_here) landed(2 * (j + 1 - first));
                        k_here = true;
                        if (ok) scores(X, j + 1);
                    }
                }
                // every block has a reader among A and B; its buffers are free behind the last one's
                if (ok && j >= first) release(2 * (j - first) + 1);
                if (ok && j + 1 < last) release(2 * (j + 1 - first));
            }
        }
    }
    } else {
        if (ROWS != 32) setmaxnreg_inc<L::MORE>();
        // ---- softmax: one row per thread ----
        const int X = warp / L::SW, r = 32 * (warp % L::SW) + lane, fX = X ? firstB : firstA, lX = X ? lastB : lastA;
        const int nt = X ? ntB : ntA, tok = t0 + X * tpt + r / G;
        const bool mine = r < nt * G;
        // keys this row sees; a row of no token takes them all (its result goes nowhere)
        const int see = !mine || !x.causal ? lk : min(lk, tok + shift + 1);
        const int see_all = __reduce_min_sync(0xffffffffu, see);
        const float sign = x.scale < 0.f ? -1.f : 1.f;
        // a zero scale becomes one that leaves every score at 0 but a masked one at -inf
        const float c = fmaxf(fabsf(x.scale) * 1.4426950408889634f, 1e-37f);
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const uint32_t ts = tm + lanes + L::T_S + 128 * X, to = tm + lanes + L::T_O + D * X;
        const uint32_t tp = tm + lanes + L::T_P + L::P_STEP * X;
        float m = -INFINITY, l = 0.f;  // reference (powers of two) and sum
        bool ok = true;
        for (int j = fX; j < lX; ++j) {
            if (!(ok = bar_wait_w(&bars.s_full[X], (uint32_t)(j - fX) & 1, &abort_flag, x.status))) break;
            fence_after_sync();
            float v[kKeys];
#pragma unroll
            for (int i = 0; i < kKeys / 32; ++i) tmem_ld32(ts + 32 * i, v + 32 * i);
            tmem_wait_ld();
            if (L::OWN_P) {
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.s_loaded[X]);
            }
            if (sign < 0.f) {
#pragma unroll
                for (int i = 0; i < kKeys; ++i) v[i] = -v[i];
            }
            if ((j + 1) * kKeys > see_all) {
                const int n = see - j * kKeys;
#pragma unroll
                for (int i = 0; i < kKeys; ++i) v[i] = i < n ? v[i] : -INFINITY;
            }
            float top[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int i = 4; i < kKeys; i += 8) {  // (pairs: a maximum of three takes one instruction)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e + 4 < kKeys) top[e] = fmaxf(top[e], fmaxf(v[i + e], v[i + e + 4]));
                    else top[e] = fmaxf(top[e], v[i + e]);
            }
            const float now = c * fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            if (L::OWN_P && j > fX) {  // P and O of the block before are done with
                if (!(ok = bar_wait_w(&bars.pv_done[X], (uint32_t)(j - 1 - fX) & 1, &abort_flag, x.status))) break;
                fence_after_sync();
            }
            const bool raise = now > m + kSlack;  // (from -inf on the first key seen)
            if (__any_sync(0xffffffffu, raise)) {
                const float keep = raise ? ex2(m - now) : 1.f;  // 0 from -inf
                if (raise) m = now;
                l *= keep;
                if (j > fX) {  // (d = 128: S_j was issued after P_{j-1} V_{j-1}, so O is complete)
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {
                        float o[32];
                        tmem_ld32(to + 32 * i, o);
                        tmem_wait_ld();
                        uint32_t w[16];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
#pragma unroll
                            for (int e = 0; e < 16; ++e) w[e] = __float_as_uint(o[16 * h + e] * keep);
                            tmem_st16(to + 32 * i + 16 * h, w);
                        }
                    }
                }
            }
            const float base = m == -INFINITY ? 0.f : -m;
            const uint64_t cc = f2_pack(c, c), bb = f2_pack(base, base), one = f2_pack(1.f, 1.f);
            uint64_t sum[2] = {f2_pack(0.f, 0.f), f2_pack(0.f, 0.f)};
#pragma unroll
            for (int i = 0; i < kKeys / 32; ++i) {
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float p0, p1;
                    f2_unpack(f2_fma(f2_pack(v[32 * i + 2 * e], v[32 * i + 2 * e + 1]), cc, bb), p0, p1);
                    p0 = ex2(p0);
                    p1 = ex2(p1);
                    sum[e & 1] = f2_fma(f2_pack(p0, p1), one, sum[e & 1]);
                    w[e] = pack_bf16(p0, p1);
                }
                tmem_st16(tp + 16 * i, w);
            }
            {
                float a, b, d, e;
                f2_unpack(sum[0], a, b);
                f2_unpack(sum[1], d, e);
                l += (a + b) + (d + e);
            }
            tmem_wait_st();
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.p_ready[X]);
        }
        if (ok && fX < lX)
            ok = bar_wait_w(&bars.pv_done[X], L::OWN_P ? (uint32_t)(lX - 1 - fX) & 1 : 0u, &abort_flag, x.status);
        fence_after_sync();
        const size_t rows = (size_t)pk.T * pk.H;
        const size_t row = (size_t)(qlo + tok) * pk.H + hk * G + r % G;
        const bool none = l == 0.f;  // no key seen (a NaN or infinite score leaves a sum of NaN, and goes on)
        const float inv = 1.f / l;
        if (ok && mine) {
            const float z = none ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
            if (x.splits > 1)
                x.part_lse[split * rows + row] = z;
            else if (x.lse)
                x.lse[row] = z;
        }
        if (ok) {  // (the loads from tensor memory are the whole warp's)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                float o[32] = {};
                if (fX < lX) {
                    tmem_ld32(to + 32 * i, o);
                    tmem_wait_ld();
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = none ? 0.f : o[e] * inv;
                if (!mine) continue;
                if (x.splits > 1) {
                    float4* dst = (float4*)(x.part + (split * rows + row) * D + 32 * i);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        dst[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                } else {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = pack_bf16(o[2 * e], o[2 * e + 1]);
                    char* dst = (char*)((__nv_bfloat16*)x.out + row * D + 32 * i);
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        store_32b(dst + 32 * e, make_uint4(w[8 * e], w[8 * e + 1], w[8 * e + 2], w[8 * e + 3]),
                                  make_uint4(w[8 * e + 4], w[8 * e + 5], w[8 * e + 6], w[8 * e + 7]));
                }
            }
        }
        fence_before_sync();
    }
    __syncthreads();
    drain_after_abort(abort_flag);
    if (warp == L::MMA) {
        fence_after_sync();
        tmem_dealloc(tmem_base_sh, L::COLS);
    }
}

// [rows][heads][d] bf16 with a row stride (elements), as boxes of 64 elements, `bh` heads and
// `bt` rows, 128-byte swizzle: in shared memory row (t, h) of the box is 128 bytes at
// (t * bh + h) * 128.  Rows outside read as zero.
bool make_rows_map(CUtensorMap* m, const void* base, int T, int heads, int d, long long stride, int bh,
                   int bt)
{
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)T};
    cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)stride * 2};
    cuuint32_t box[3] = {64, (cuuint32_t)bh, (cuuint32_t)bt};
    cuuint32_t es[3] = {1, 1, 1};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box,
               es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, int ROWS>
cudaError_t launch(const AttnArgs& x, cudaStream_t s)
{
    using L = Lay<D, ROWS>;
    const Packed& p = x.p;
    const int G = p.H / p.Hk, tpt = L::R / G;
    CUtensorMap mq, mk, mv;
    if (!make_rows_map(&mq, x.q, p.T, p.H, D, p.qs, G, tpt) ||
        !make_rows_map(&mk, x.k, p.Tk, p.Hk, D, p.ks, 1, kKeys) ||
        !make_rows_map(&mv, x.v, p.Tk, p.Hk, D, p.vs, 1, kKeys))
        return cudaErrorInvalidValue;
    cudaError_t e = cudaFuncSetAttribute(tc_softattn_kernel<D, ROWS>,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::SMEM);
    if (e != cudaSuccess) return e;
    return launch_after(tc_softattn_kernel<D, ROWS>, softattn_grid(x, L::TILES * tpt), L::THREADS, (int)L::SMEM, 0, false, s, mq, mk,
                        mv, x);
}

template <int D>
cudaError_t launch(const AttnArgs& x, cudaStream_t s)
{
    const int rows = tc_softattn_rows(x.p);
    return rows == 32 ? launch<D, 32>(x, s) : rows == 128 ? launch<D, 128>(x, s) : launch<D, 256>(x, s);
}

}  // namespace

bool tc_softattn_supported(const Packed& p) { return p.bf16; }

// One or two tokens a sequence: 32 rows; else what holds an average sequence's rows.  (The lengths
// are on the device: a long prompt among single tokens raises the average and takes large blocks.)
int tc_softattn_rows(const Packed& p)
{
    const int G = p.H / p.Hk;
    if (softattn_few(p) && G <= 32) return 32;
    return (long long)p.T * G <= 128LL * p.n ? 128 : 256;
}

cudaError_t launch_tc_softattn(const AttnArgs& x, cudaStream_t s)
{
    return x.p.d == 64 ? launch<64>(x, s) : launch<128>(x, s);
}

}  // namespace flex
