// Host side of the entry points around the recurrence (include/flexattn.h): argument checks,
// workspace layout and dispatch.  Nothing here allocates device memory or synchronises.
#include "flex_internal.h"
#include "layer.cuh"
#include "ssm.cuh"

#include <initializer_list>

namespace {

constexpr size_t kHeader = sizeof(flex::WsHeader);

bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }
// All given and on 16-byte boundaries.
bool all16(std::initializer_list<const void*> ps)
{
    for (const void* p : ps)
        if (!p || !aligned(p, 16)) return false;
    return true;
}
// On 16-byte boundaries where given.
bool opt16(std::initializer_list<const void*> ps)
{
    for (const void* p : ps)
        if (!aligned(p, 16)) return false;
    return true;
}
bool offsets(const int* cu) { return cu && aligned(cu, 4); }
int check_ws(const void* ws, size_t ws_bytes, size_t need)
{
    if (!ws || !aligned(ws, 256)) return FLEX_EINVAL;
    return ws_bytes < need ? FLEX_EWORKSPACE : FLEX_OK;
}
int counted(int n, cudaError_t e)
{
    if (e != cudaSuccess) return FLEX_ECUDA;
    flex::add_launches(n);
    return FLEX_OK;
}
int unit(int dtype) { return dtype == FLEX_BF16 ? 8 : 4; }  // elements of 16 bytes
bool strides(int dtype, std::initializer_list<int> stride, int least)
{
    for (int s : stride)
        if (s % unit(dtype) || s < least) return false;
    return true;
}

// Whether an output lies over an input that is a slice of wider rows: its rows then replace others that
// are still to be read.  Over an input of contiguous rows every value is read before it is replaced.
struct Rows {
    const void* p;
    int stride;
};
bool over_slice(std::initializer_list<const void*> outs, std::initializer_list<Rows> ins, int row, int rows)
{
    for (const void* o : outs)
        for (const Rows& i : ins)
            if (o && o == i.p && rows > 1 && i.stride != row) return true;
    return false;
}

int make_ssm(const flex_ssm* s, bool z, flex::SsmArgs* a)
{
    if (!s || s->n < 1 || s->T < 1 || s->D < 1 || s->G < 1 || s->N < 1) return FLEX_EINVAL;
    if (s->dtype != FLEX_F32 && s->dtype != FLEX_BF16) return FLEX_EINVAL;
    if (s->D % s->G) return FLEX_EINVAL;
    if (s->N != 8 && s->N != 16 && s->N != 32) return FLEX_EUNSUPPORTED;
    if (s->D % unit(s->dtype) || s->D / s->G % 4) return FLEX_EUNSUPPORTED;
    if (s->n > 65535 || s->T >= (1 << 30) || s->D > 65536 || s->G > 1024) return FLEX_EUNSUPPORTED;
    if (!strides(s->dtype, {s->x_stride, s->dt_stride}, s->D)) return FLEX_EINVAL;
    if (!strides(s->dtype, {s->b_stride, s->c_stride}, s->G * s->N)) return FLEX_EINVAL;
    if (z && !strides(s->dtype, {s->z_stride}, s->D)) return FLEX_EINVAL;
    *a = {};
    a->n = s->n; a->T = s->T; a->D = s->D; a->G = s->G; a->N = s->N;
    a->bf16 = s->dtype == FLEX_BF16; a->softplus = s->softplus != 0;
    a->xs = s->x_stride; a->ds = s->dt_stride; a->bs = s->b_stride; a->cs = s->c_stride;
    a->zs = s->z_stride;
    return FLEX_OK;
}

size_t floats(size_t n) { return flex::align_up(n * 4, 256); }

// Blocks' ends and sums of steps where sequences are cut; backward: sums over blocks' channels and
// tokens too.  With ws the pointers into it are set.
size_t ssm_layout(flex::SsmArgs* a, bool backward, char* ws)
{
    size_t at = kHeader;
    auto take = [&](size_t n) {
        float* p = (float*)(ws + at);
        at += floats(n);
        return ws ? p : nullptr;
    };
    a->rows = flex::ssm_rows(*a, backward);
    const size_t slots = flex::block_slots(a->T, a->n, a->rows), DN = (size_t)a->D * a->N;
    if (a->rows <= a->T) {
        a->ends = take(slots * DN);
        a->sums = take(slots * a->D);
    }
    if (backward) {
        a->part_bc = take((size_t)flex::ssm_bwd_tiles(*a) * a->T * a->G * 2 * a->N);
        a->part_a = take(slots * DN);
        a->part_d = take(slots * 2 * a->D);
    }
    return at;
}
size_t ssm_ws_bytes(const flex::SsmArgs& a, bool backward)
{
    flex::SsmArgs x = a;
    const size_t f = ssm_layout(&x, false, nullptr), b = backward ? ssm_layout(&x, true, nullptr) : 0;
    return f > b ? f : b;
}
size_t ssm_save_bytes(const flex::SsmArgs& a)
{
    return floats((size_t)flex::block_slots(a.T, a.n, flex::ssm::kMark) * a.D * a.N);
}

int make_conv(const flex_conv* s, flex::ConvArgs* a)
{
    if (!s || s->n < 1 || s->T < 1 || s->D < 1 || s->W < 1) return FLEX_EINVAL;
    if (s->dtype != FLEX_F32 && s->dtype != FLEX_BF16) return FLEX_EINVAL;
    if (s->W < 2 || s->W > 4 || s->D % unit(s->dtype)) return FLEX_EUNSUPPORTED;
    if (s->n > 65535 || s->T >= (1 << 30) || s->D > 65536) return FLEX_EUNSUPPORTED;
    if (!strides(s->dtype, {s->x_stride}, s->D)) return FLEX_EINVAL;
    *a = {};
    a->n = s->n; a->T = s->T; a->D = s->D; a->W = s->W;
    a->bf16 = s->dtype == FLEX_BF16; a->silu = s->silu != 0; a->xs = s->x_stride;
    return FLEX_OK;
}
size_t conv_ws_bytes(flex::ConvArgs* a)
{
    a->run = flex::conv_run(*a);
    return kHeader + floats((size_t)flex::conv_bwd_blocks(*a) * (a->W + 1) * a->D);
}

int make_norm(const flex_norm* s, bool z, bool res, flex::NormArgs* a)
{
    if (!s || s->T < 1 || s->H < 1 || s->d < 1 || !(s->eps >= 0.f)) return FLEX_EINVAL;
    if (s->dtype != FLEX_F32 && s->dtype != FLEX_BF16) return FLEX_EINVAL;
    if (s->heads != 1 && s->heads != s->H) return FLEX_EINVAL;
    if (s->d % unit(s->dtype) || s->d > 8192) return FLEX_EUNSUPPORTED;
    if (s->T >= (1 << 30) || s->H > 1024 || (long long)s->T * s->H >= 1LL << 31) return FLEX_EUNSUPPORTED;
    const int row = s->H * s->d;
    if (!strides(s->dtype, {s->x_stride}, row)) return FLEX_EINVAL;
    if (z && !strides(s->dtype, {s->z_stride}, row)) return FLEX_EINVAL;
    if (res && !strides(s->dtype, {s->res_stride}, row)) return FLEX_EINVAL;
    *a = {};
    a->T = s->T; a->H = s->H; a->d = s->d; a->heads = s->heads; a->eps = s->eps;
    a->bf16 = s->dtype == FLEX_BF16;
    a->xs = s->x_stride; a->zs = s->z_stride; a->rs = s->res_stride;
    return FLEX_OK;
}

}  // namespace

extern "C" {

size_t flex_ssm_workspace_bytes(const flex_ssm* shape, int backward)
{
    flex::SsmArgs a;
    return make_ssm(shape, false, &a) == FLEX_OK ? ssm_ws_bytes(a, backward != 0) : 0;
}

size_t flex_ssm_save_bytes(const flex_ssm* shape)
{
    flex::SsmArgs a;
    return make_ssm(shape, false, &a) == FLEX_OK ? ssm_save_bytes(a) : 0;
}

int flex_ssm_fwd(const flex_ssm* shape, const void* x, const void* dt, const float* A, const void* B,
                 const void* C, const float* D, const void* z, const float* dt_bias, const int* cu,
                 const float* S0, float* S1, void* out, void* save, void* ws, size_t ws_bytes,
                 void* stream)
{
    flex::SsmArgs a;
    int rc = make_ssm(shape, z != nullptr, &a);
    if (rc) return rc;
    if (!all16({x, dt, A, B, C, out}) || !opt16({D, z, dt_bias, S0, S1}) || !offsets(cu)) return FLEX_EINVAL;
    if (save && (S0 || !aligned(save, 256))) return FLEX_EINVAL;
    if (over_slice({out}, {{x, shape->x_stride}, {dt, shape->dt_stride}, {z, shape->z_stride}}, a.D, a.T))
        return FLEX_EINVAL;
    const size_t need = ssm_layout(&a, false, nullptr);
    if ((rc = check_ws(ws, ws_bytes, need))) return rc;
    ssm_layout(&a, false, (char*)ws);
    a.x = x; a.dt = dt; a.A = A; a.B = B; a.C = C; a.Ds = D; a.z = z; a.bias = dt_bias; a.cu = cu;
    a.h0 = S0; a.h1 = S1; a.out = out; a.marks = (float*)save;
    a.joined = flex::ssm_joined(a);
    return counted(a.rows > a.T ? 1 : a.joined ? 3 : 2, flex::launch_ssm_fwd(a, (cudaStream_t)stream));
}

int flex_ssm_bwd(const flex_ssm* shape, const void* x, const void* dt, const float* A, const void* B,
                 const void* C, const float* D, const void* z, const float* dt_bias, const int* cu,
                 const void* dout, const void* save, void* dx, void* ddt, float* dA, void* dB,
                 void* dC, float* dD, void* dz, float* ddt_bias, void* ws, size_t ws_bytes,
                 void* stream)
{
    flex::SsmArgs a;
    int rc = make_ssm(shape, z != nullptr, &a);
    if (rc) return rc;
    if (!all16({x, dt, A, B, C, dout, dx, ddt, dA, dB, dC}) || !opt16({D, z, dt_bias, dD, dz, ddt_bias}))
        return FLEX_EINVAL;
    if (!offsets(cu) || !save || !aligned(save, 256)) return FLEX_EINVAL;
    if (!D != !dD || !z != !dz || !dt_bias != !ddt_bias) return FLEX_EINVAL;
    if (over_slice({dx, ddt, dz}, {{x, shape->x_stride}, {dt, shape->dt_stride}, {z, shape->z_stride}}, a.D, a.T))
        return FLEX_EINVAL;
    const size_t need = ssm_layout(&a, true, nullptr);
    if ((rc = check_ws(ws, ws_bytes, need))) return rc;
    ssm_layout(&a, true, (char*)ws);
    a.x = x; a.dt = dt; a.A = A; a.B = B; a.C = C; a.Ds = D; a.z = z; a.bias = dt_bias; a.cu = cu;
    a.marks = (float*)save; a.dout = dout;
    a.dx = dx; a.ddt = ddt; a.dA = dA; a.dB = dB; a.dC = dC; a.dDs = dD; a.dz = dz; a.dbias = ddt_bias;
    return counted(a.rows <= a.T ? 4 : 2, flex::launch_ssm_bwd(a, (cudaStream_t)stream));
}

int flex_ssm_decode(const flex_ssm* shape, const void* x, const void* dt, const float* A,
                    const void* B, const void* C, const float* D, const void* z,
                    const float* dt_bias, float* S, void* out, void* stream)
{
    flex::SsmArgs a;
    const int rc = make_ssm(shape, z != nullptr, &a);
    if (rc) return rc;
    if (a.T != a.n) return FLEX_EINVAL;
    if (!all16({x, dt, A, B, C, S, out}) || !opt16({D, z, dt_bias})) return FLEX_EINVAL;
    if (over_slice({out}, {{x, shape->x_stride}, {dt, shape->dt_stride}, {z, shape->z_stride}}, a.D, a.T))
        return FLEX_EINVAL;
    a.x = x; a.dt = dt; a.A = A; a.B = B; a.C = C; a.Ds = D; a.z = z; a.bias = dt_bias;
    a.h1 = S; a.out = out;
    return counted(1, flex::launch_ssm_decode(a, (cudaStream_t)stream));
}

size_t flex_conv_workspace_bytes(const flex_conv* shape)
{
    flex::ConvArgs a;
    return make_conv(shape, &a) == FLEX_OK ? conv_ws_bytes(&a) : 0;
}

int flex_conv_fwd(const flex_conv* shape, const void* x, const float* w, const float* bias,
                  const int* cu, const void* S0, void* S1, void* out, void* stream)
{
    flex::ConvArgs a;
    const int rc = make_conv(shape, &a);
    if (rc) return rc;
    if (!all16({x, w, out}) || !opt16({bias, S0, S1}) || !offsets(cu)) return FLEX_EINVAL;
    if ((S0 && S0 == S1) || out == x) return FLEX_EINVAL;  // (rows are read by others than write them)
    a.x = x; a.w = w; a.bias = bias; a.cu = cu; a.S0 = S0; a.S1 = S1; a.out = out;
    a.run = flex::conv_run(a);
    return counted(1, flex::launch_conv_fwd(a, (cudaStream_t)stream));
}

int flex_conv_bwd(const flex_conv* shape, const void* x, const float* w, const float* bias,
                  const int* cu, const void* dout, void* dx, float* dw, float* dbias, void* ws,
                  size_t ws_bytes, void* stream)
{
    flex::ConvArgs a;
    int rc = make_conv(shape, &a);
    if (rc) return rc;
    if (!all16({x, w, dout, dx, dw}) || !opt16({bias, dbias}) || !offsets(cu)) return FLEX_EINVAL;
    if (!bias != !dbias || dx == x || dx == dout) return FLEX_EINVAL;
    const size_t need = conv_ws_bytes(&a);
    if ((rc = check_ws(ws, ws_bytes, need))) return rc;
    a.x = x; a.w = w; a.bias = bias; a.cu = cu; a.dout = dout; a.dx = dx; a.dw = dw; a.dbias = dbias;
    a.part = (float*)((char*)ws + kHeader);
    return counted(2, flex::launch_conv_bwd(a, (cudaStream_t)stream));
}

int flex_conv_decode(const flex_conv* shape, const void* x, const float* w, const float* bias,
                     void* S, void* out, void* stream)
{
    flex::ConvArgs a;
    const int rc = make_conv(shape, &a);
    if (rc) return rc;
    if (a.T != a.n) return FLEX_EINVAL;
    if (!all16({x, w, S, out}) || !opt16({bias})) return FLEX_EINVAL;
    if (over_slice({out}, {{x, shape->x_stride}}, a.D, a.T)) return FLEX_EINVAL;
    a.x = x; a.w = w; a.bias = bias; a.S1 = S; a.out = out;
    return counted(1, flex::launch_conv_decode(a, (cudaStream_t)stream));
}

size_t flex_norm_workspace_bytes(const flex_norm* shape)
{
    flex::NormArgs a;
    return make_norm(shape, false, false, &a) == FLEX_OK ? kHeader + floats(flex::norm_part_floats(a)) : 0;
}

int flex_norm_fwd(const flex_norm* shape, const void* x, const float* w, const void* z,
                  const void* res, const float* scale, const int* end, void* out, void* total,
                  float* rstd, void* stream)
{
    flex::NormArgs a;
    const int rc = make_norm(shape, z != nullptr, res != nullptr, &a);
    if (rc) return rc;
    if (!all16({x, w, out}) || !opt16({z, res, scale, total}) || !aligned(end, 4) || !aligned(rstd, 4))
        return FLEX_EINVAL;
    if (!res != !total || (scale && !res)) return FLEX_EINVAL;
    if (over_slice({out, total}, {{x, shape->x_stride}, {z, shape->z_stride}, {res, shape->res_stride}},
                   a.H * a.d, a.T))
        return FLEX_EINVAL;
    a.x = x; a.w = w; a.z = z; a.res = res; a.scale = scale; a.end = end;
    a.out = out; a.total = total; a.rstd = rstd;
    return counted(1, flex::launch_norm_fwd(a, (cudaStream_t)stream));
}

int flex_norm_bwd(const flex_norm* shape, const void* x, const float* w, const void* z,
                  const void* res, const float* scale, const int* end, const float* rstd,
                  const void* dout, const void* dtotal, void* dx, void* dres, void* dz, float* dw,
                  float* dscale, void* ws, size_t ws_bytes, void* stream)
{
    flex::NormArgs a;
    int rc = make_norm(shape, z != nullptr, res != nullptr, &a);
    if (rc) return rc;
    if (!all16({x, w, dout, dw}) || !opt16({z, res, scale, dtotal, dx, dres, dz, dscale})) return FLEX_EINVAL;
    if (!rstd || !aligned(rstd, 4) || !aligned(end, 4)) return FLEX_EINVAL;
    if (!res != !dres || !z != !dz || !scale != !dscale || (scale && !res) || (dtotal && !res))
        return FLEX_EINVAL;
    if (!dx != (res && !scale)) return FLEX_EINVAL;  // (without a scale dres is dx too)
    if (over_slice({dx, dres, dz}, {{x, shape->x_stride}, {z, shape->z_stride}, {res, shape->res_stride}},
                   a.H * a.d, a.T))
        return FLEX_EINVAL;
    if ((rc = check_ws(ws, ws_bytes, kHeader + floats(flex::norm_part_floats(a))))) return rc;
    a.x = x; a.w = w; a.z = z; a.res = res; a.scale = scale; a.end = end; a.rstd = const_cast<float*>(rstd);
    a.dout = dout; a.dtotal = dtotal; a.dx = dx; a.dres = dres; a.dz = dz; a.dw = dw; a.dscale = dscale;
    a.part = (float*)((char*)ws + kHeader);
    return counted(2, flex::launch_norm_bwd(a, (cudaStream_t)stream));
}

}  // extern "C"
