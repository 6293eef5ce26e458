// Host side of the packed-batch entry points of include/flexattn.h: argument checks, workspace
// layout and dispatch.  Nothing here allocates device memory or synchronises.
#include "flex_internal.h"
#include "packed.cuh"
#include "softattn.cuh"

#include <initializer_list>

using flex::Packed;

namespace {

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// Delta rule: q and k have Hk heads, v has H.  Attention: q has H, k and v have Hk.
int make_packed(const flex_packed* s, bool attention, Packed* p)
{
    if (!s) return FLEX_EINVAL;
    if (s->n < 1 || s->T < 1 || s->Tk < 1 || s->H < 1 || s->Hk < 1 || s->H % s->Hk != 0)
        return FLEX_EINVAL;
    if (!attention && s->Tk != s->T) return FLEX_EINVAL;
    if (s->dtype != FLEX_F32 && s->dtype != FLEX_BF16) return FLEX_EINVAL;
    if (s->d != 64 && s->d != 128) return FLEX_EUNSUPPORTED;
    if (s->n > 65535 || s->H > 1024 || s->T > (1 << 30) || s->Tk > (1 << 30)) return FLEX_EUNSUPPORTED;
    if (attention && s->H / s->Hk > 64) return FLEX_EUNSUPPORTED;
    const int unit = s->dtype == FLEX_BF16 ? 8 : 4;  // elements of 16 bytes
    const int qh = attention ? s->H : s->Hk, vh = attention ? s->Hk : s->H;
    if (s->q_stride % unit || s->k_stride % unit || s->v_stride % unit) return FLEX_EINVAL;
    if (s->q_stride < qh * s->d || s->k_stride < s->Hk * s->d || s->v_stride < vh * s->d)
        return FLEX_EINVAL;
    p->n = s->n; p->T = s->T; p->Tk = s->Tk; p->H = s->H; p->Hk = s->Hk; p->d = s->d;
    p->bf16 = s->dtype == FLEX_BF16;
    p->qs = s->q_stride; p->ks = s->k_stride; p->vs = s->v_stride;
    return FLEX_OK;
}

int check_ws(void* ws, size_t ws_bytes, size_t need)
{
    if (!ws || !aligned(ws, 256)) return FLEX_EINVAL;
    return ws_bytes < need ? FLEX_EWORKSPACE : FLEX_OK;
}

bool all16(std::initializer_list<const void*> ps)
{
    for (const void* p : ps)
        if (!p || !aligned(p, 16)) return false;
    return true;
}

// Gates are read and written element by element.
bool gates(const Packed& p, std::initializer_list<const void*> ps)
{
    for (const void* x : ps)
        if (!x || !aligned(x, p.bf16 ? 2 : 4)) return false;
    return true;
}

constexpr size_t kHeader = sizeof(flex::WsHeader);

// The fp32 scans' scratch of the backward, or the tensor-core kernels': the chunks' records
// (forward without a save buffer), the states' gradients (backward).
size_t delta_ws_bytes(const Packed& p, bool backward)
{
    if (!flex::tc_delta_supported(p))
        return kHeader + (backward ? flex::align_up(flex::delta_scan_ws_floats(p) * 4, 256) : 0);
    const size_t f = flex::tc_delta_rec_bytes(p), b = backward ? flex::tc_delta_bwd_bytes(p) : 0;
    return kHeader + flex::align_up(f > b ? f : b, 256);
}
size_t delta_save(const Packed& p)
{
    return flex::align_up(flex::tc_delta_supported(p) ? flex::tc_delta_save_bytes(p)
                                                      : flex::delta_scan_save_floats(p) * 4, 256);
}

// Partial outputs, then partial log sums, when the keys are split.
size_t attn_ws_bytes(const Packed& p)
{
    const size_t rows = (size_t)p.T * p.H, n = flex::softattn_splits(p);
    return kHeader + (n > 1 ? flex::align_up(n * rows * p.d * 4, 256) + flex::align_up(n * rows * 4, 256) : 0);
}

int counted(int n, cudaError_t e)
{
    if (e != cudaSuccess) return FLEX_ECUDA;
    flex::add_launches(n);
    return FLEX_OK;
}

}  // namespace

extern "C" {

size_t flex_delta_workspace_bytes(const flex_packed* shape, int backward)
{
    Packed p;
    return make_packed(shape, false, &p) == FLEX_OK ? delta_ws_bytes(p, backward != 0) : 0;
}

size_t flex_delta_save_bytes(const flex_packed* shape)
{
    Packed p;
    return make_packed(shape, false, &p) == FLEX_OK ? delta_save(p) : 0;
}

int flex_delta_fwd(const flex_packed* shape, const void* q, const void* k, const void* v,
                   const void* g, const void* beta, const int* cu, float scale, const float* S0,
                   float* S1, void* out, void* save, void* ws, size_t ws_bytes, void* stream)
{
    Packed p;
    int rc = make_packed(shape, false, &p);
    if (rc) return rc;
    if (!all16({q, k, v, out}) || !gates(p, {g, beta}) || !cu || !aligned(cu, 4)) return FLEX_EINVAL;
    if ((S0 && !aligned(S0, 16)) || (S1 && !aligned(S1, 16)) || (save && !aligned(save, 256)))
        return FLEX_EINVAL;
    if (save && S0) return FLEX_EINVAL;
    // (with save the chunks' records go there)
    if ((rc = check_ws(ws, ws_bytes, save ? kHeader : delta_ws_bytes(p, false)))) return rc;
    if (flex::tc_delta_supported(p))
        return counted(2, flex::launch_tc_delta_fwd(p, q, k, v, g, beta, cu, scale, S0, S1, out,
                                                    save ? save : (char*)ws + kHeader, save != nullptr,
                                                    &((flex::WsHeader*)ws)->status,
                                                    (cudaStream_t)stream));
    return counted(1, flex::launch_delta_scan_fwd(p, q, k, v, g, beta, cu, scale, S0, S1, out,
                                                  (float*)save, (cudaStream_t)stream));
}

int flex_delta_bwd(const flex_packed* shape, const void* q, const void* k, const void* v,
                   const void* g, const void* beta, const int* cu, float scale, const void* dout,
                   const void* save, void* dq, void* dk, void* dv, void* dg, void* dbeta, void* ws,
                   size_t ws_bytes, void* stream)
{
    Packed p;
    int rc = make_packed(shape, false, &p);
    if (rc) return rc;
    if (!all16({q, k, v, dout, dq, dk, dv}) || !gates(p, {g, beta, dg, dbeta}) || !cu ||
        !aligned(cu, 4))
        return FLEX_EINVAL;
    if (!save || !aligned(save, 256)) return FLEX_EINVAL;
    if ((rc = check_ws(ws, ws_bytes, delta_ws_bytes(p, true)))) return rc;
    if (flex::tc_delta_supported(p))
        return counted(2, flex::launch_tc_delta_bwd(p, q, k, g, cu, scale, dout, save, dq, dk, dv, dg,
                                                    dbeta, (char*)ws + kHeader,
                                                    &((flex::WsHeader*)ws)->status,
                                                    (cudaStream_t)stream));
    return counted(4, flex::launch_delta_scan_bwd(p, q, k, g, beta, cu, scale, dout,
                                                  (const float*)save, dq, dk, dv, dg, dbeta,
                                                  (float*)((char*)ws + kHeader),
                                                  (cudaStream_t)stream));
}

int flex_delta_decode(const flex_packed* shape, const void* q, const void* k, const void* v,
                      const void* g, const void* beta, float scale, float* S, void* out,
                      void* stream)
{
    Packed p;
    int rc = make_packed(shape, false, &p);
    if (rc) return rc;
    if (p.T != p.n) return FLEX_EINVAL;
    if (!all16({q, k, v, S, out}) || !gates(p, {g, beta})) return FLEX_EINVAL;
    return counted(1, flex::launch_delta_decode(p, q, k, v, g, beta, scale, S, out,
                                                (cudaStream_t)stream));
}

size_t flex_softattn_workspace_bytes(const flex_packed* shape)
{
    Packed p;
    return make_packed(shape, true, &p) == FLEX_OK ? attn_ws_bytes(p) : 0;
}

int flex_softattn_fwd(const flex_packed* shape, const void* q, const void* k, const void* v,
                      const int* cu_q, const int* cu_k, float scale, int causal, void* out,
                      float* lse, void* ws, size_t ws_bytes, void* stream)
{
    Packed p;
    int rc = make_packed(shape, true, &p);
    if (rc) return rc;
    if (!all16({q, k, v, out}) || !cu_q || !cu_k || !aligned(cu_q, 4) || !aligned(cu_k, 4))
        return FLEX_EINVAL;
    if (lse && !aligned(lse, 4)) return FLEX_EINVAL;
    if ((rc = check_ws(ws, ws_bytes, attn_ws_bytes(p)))) return rc;
    flex::AttnArgs x = {};
    x.p = p;
    x.q = q; x.k = k; x.v = v; x.cu_q = cu_q; x.cu_k = cu_k;
    x.scale = scale; x.causal = causal != 0; x.splits = flex::softattn_splits(p);
    x.out = out; x.lse = lse;
    x.part = (float*)((char*)ws + kHeader);
    x.part_lse = (float*)((char*)x.part + flex::align_up((size_t)x.splits * p.T * p.H * p.d * 4, 256));
    x.status = &((flex::WsHeader*)ws)->status;
    cudaStream_t s = (cudaStream_t)stream;
    rc = counted(1, flex::tc_softattn_supported(p) ? flex::launch_tc_softattn(x, s)
                                                   : flex::launch_softattn_simt(x, s));
    if (rc) return rc;
    return x.splits > 1 ? counted(1, flex::launch_softattn_join(x, s)) : FLEX_OK;
}

}  // extern "C"
