// dart_api.cpp -- the C ABI of libdart.so (declared in include/dart.h):
// argument validation on the host, workspace sizing, dispatch to the kernel
// launchers, status codes and a per-thread error message.  Nothing here
// allocates device memory or keeps state between calls.
#include "dart.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <new>

#include "dart_internal.hpp"

namespace {

thread_local char g_err[512] = "";

dart_status fail(dart_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof g_err, fmt, ap);
    va_end(ap);
    return st;
}

dart_status ok() {
    g_err[0] = '\0';
    return DART_OK;
}

// Checks shared by every entry point; fills `s` on success.
dart_status make_shape(const dart_dims* d, bool need_seqlen, dart::Shape& s) {
    if (!d) return fail(DART_ERR_INVALID_ARG, "dims is NULL");
    if (d->batch < 1) return fail(DART_ERR_INVALID_ARG, "batch must be >= 1 (got %lld)", (long long)d->batch);
    if (need_seqlen && d->seqlen < 1)
        return fail(DART_ERR_INVALID_ARG, "seqlen must be >= 1 (got %lld)", (long long)d->seqlen);
    if (d->nheads < 1 || d->ngroups < 1)
        return fail(DART_ERR_INVALID_ARG, "nheads and ngroups must be >= 1");
    if (d->nheads % d->ngroups != 0)
        return fail(DART_ERR_INVALID_ARG, "nheads (%d) must be a multiple of ngroups (%d)", d->nheads, d->ngroups);
    if (d->headdim < 1 || d->dstate < 1 || d->chunk < 1)
        return fail(DART_ERR_INVALID_ARG, "headdim, dstate and chunk must be >= 1");
    if (d->dtype != DART_FP32 && d->dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "dtype must be DART_FP32 or DART_BF16 (got %d)", d->dtype);
    if (d->mem_capacity < 0) return fail(DART_ERR_INVALID_ARG, "mem_capacity must be >= 0");
    if (d->headdim != 64)
        return fail(DART_ERR_UNSUPPORTED, "headdim %d not supported (the library has kernels for 64)", d->headdim);
    if (d->dstate != 16 && d->dstate != 32 && d->dstate != 64 && d->dstate != 128)
        return fail(DART_ERR_UNSUPPORTED, "dstate %d not supported (16, 32, 64 or 128)", d->dstate);
    if (d->chunk > 4096)
        return fail(DART_ERR_UNSUPPORTED, "chunk %d not supported (at most 4096)", d->chunk);
    if (d->batch > 65535 || d->nheads > 65535)
        return fail(DART_ERR_UNSUPPORTED, "batch and nheads must be <= 65535");
    s.B = d->batch;
    s.L = need_seqlen ? d->seqlen : 0;
    s.H = d->nheads;
    s.G = d->ngroups;
    s.P = d->headdim;
    s.N = d->dstate;
    s.S = d->chunk;
    s.M = need_seqlen ? (s.L + s.S - 1) / s.S : 0;
    s.Mcap = d->mem_capacity ? d->mem_capacity : s.M;
    s.dtype = d->dtype;
    if (need_seqlen && s.Mcap < s.M)
        return fail(DART_ERR_INVALID_ARG, "mem_capacity %lld < ceil(L/S) = %lld", (long long)s.Mcap,
                    (long long)s.M);
    if (need_seqlen && s.M > 2147483647LL) return fail(DART_ERR_UNSUPPORTED, "too many chunks");
    return DART_OK;
}

dart_status check_opts(const dart_sma_opts* o) {
    if (!o) return fail(DART_ERR_INVALID_ARG, "opts is NULL");
    if (o->normalize != 0 && o->normalize != 1) return fail(DART_ERR_INVALID_ARG, "normalize must be 0 or 1");
    if (o->z_per_head != 0 && o->z_per_head != 1) return fail(DART_ERR_INVALID_ARG, "z_per_head must be 0 or 1");
    if (o->normalize && !(o->eps > 0.0f)) return fail(DART_ERR_INVALID_ARG, "eps must be > 0 when normalize = 1");
    if (!(o->eps >= 0.0f)) return fail(DART_ERR_INVALID_ARG, "eps must be >= 0");
    return DART_OK;
}

// The norm weights belong to RMSNorm: without normalisation they are unused.
dart::SmaArgs sma_args(const dart_sma_opts* o) {
    return dart::SmaArgs{o->eps, o->normalize ? o->q_norm_w : nullptr,
                         o->normalize ? o->e_norm_w : nullptr, o->normalize, o->z_per_head};
}

dart_status hip_status(hipError_t e, const char* what) {
    if (e != hipSuccess) return fail(DART_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
    return ok();
}

// The bytes that `rows` rows of `width` elements at a stride take, from p.
struct Range {
    uintptr_t a, b;  // first byte, one past the last
    Range(const void* p, int64_t rows, int64_t stride, int64_t width, int dtype)
        : a((uintptr_t)p), b(p && rows > 0 ? a + (uintptr_t)((rows - 1) * stride + width) * dart::elem_bytes(dtype) : a) {}
    Range(const void* p, size_t bytes) : a((uintptr_t)p), b(p ? a + bytes : a) {}
    bool meets(const Range& o) const { return a < o.b && o.a < b && a < b && o.a < o.b; }
};

// What is written meets nothing that is read and nothing else that is written.
struct Named {
    const char* name;
    Range r;
};
dart_status check_apart(std::initializer_list<Named> written, std::initializer_list<Named> read) {
    for (const Named* w = written.begin(); w != written.end(); ++w) {
        for (const Named* o = written.begin(); o != w; ++o)
            if (w->r.meets(o->r)) return fail(DART_ERR_INVALID_ARG, "%s overlaps %s", w->name, o->name);
        for (const Named& o : read)
            if (w->r.meets(o.r)) return fail(DART_ERR_INVALID_ARG, "%s overlaps %s", w->name, o.name);
    }
    return DART_OK;
}

// rows x stride elements have to be addressable.
bool too_large(int64_t rows, int64_t stride) { return rows > 0 && stride > ((int64_t)1 << 56) / rows; }

dart_status check_dtypes(int dtype, int grad_dtype) {
    if (dtype != DART_FP32 && dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "dtype must be DART_FP32 or DART_BF16 (got %d)", dtype);
    if (grad_dtype != DART_FP32 && grad_dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "grad_dtype must be DART_FP32 or DART_BF16 (got %d)", grad_dtype);
    if (grad_dtype == DART_BF16 && dtype == DART_FP32)
        return fail(DART_ERR_UNSUPPORTED, "grad_dtype DART_BF16 needs dtype DART_BF16");
    return DART_OK;
}

#define REQUIRE_PTR(p) \
    if (!(p)) return fail(DART_ERR_INVALID_ARG, "required pointer '%s' is NULL", #p)

}  // namespace

extern "C" {

size_t dart_scan_workspace_bytes(const dart_dims* dims) {
    dart::Shape s;
    if (make_shape(dims, true, s) != DART_OK) return 0;
    return dart::scan_workspace_bytes(s);
}

dart_status dart_ssd_chunk_scan(const dart_dims* dims, const void* x, const float* dt,
                                const float* A, const void* Bm, const void* Cm, const float* h0,
                                void* y_ssd, void* mem, float* h_last, void* workspace,
                                size_t workspace_bytes, void* stream) {
    dart::Shape s;
    dart_status st = make_shape(dims, true, s);
    if (st != DART_OK) return st;
    REQUIRE_PTR(x);
    REQUIRE_PTR(dt);
    REQUIRE_PTR(A);
    REQUIRE_PTR(Bm);
    REQUIRE_PTR(Cm);
    REQUIRE_PTR(y_ssd);
    REQUIRE_PTR(mem);
    REQUIRE_PTR(workspace);
    const size_t need = dart::scan_workspace_bytes(s);
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    return hip_status(dart::launch_scan(s, x, dt, A, Bm, Cm, h0, y_ssd, mem, h_last, workspace,
                                        (hipStream_t)stream),
                      "dart_ssd_chunk_scan launch");
}

size_t dart_ssd_bwd_workspace_bytes(const dart_dims* dims) {
    dart::Shape s;
    if (make_shape(dims, true, s) != DART_OK) return 0;
    return dart::ssd_bwd_workspace_bytes(s);
}

dart_status dart_ssd_bwd(const dart_dims* dims, const void* x, const float* dt, const float* A,
                         const void* Bm, const void* Cm, const float* h0, const void* dy,
                         const float* dmem, const float* dh_last, float* dx, float* ddt, float* dA,
                         float* dB, float* dC, float* dh0, void* workspace, size_t workspace_bytes,
                         void* stream) {
    dart::Shape s;
    dart_status st = make_shape(dims, true, s);
    if (st != DART_OK) return st;
    REQUIRE_PTR(x);
    REQUIRE_PTR(dt);
    REQUIRE_PTR(A);
    REQUIRE_PTR(Bm);
    REQUIRE_PTR(Cm);
    REQUIRE_PTR(dy);
    REQUIRE_PTR(dx);
    REQUIRE_PTR(ddt);
    REQUIRE_PTR(dA);
    REQUIRE_PTR(dB);
    REQUIRE_PTR(dC);
    REQUIRE_PTR(workspace);
    const size_t need = dart::ssd_bwd_workspace_bytes(s);
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    return hip_status(dart::launch_ssd_bwd(s, x, dt, A, Bm, Cm, h0, dy, dmem, dh_last, dx, ddt, dA,
                                           dB, dC, dh0, workspace, (hipStream_t)stream),
                      "dart_ssd_bwd launch");
}

size_t dart_sma_workspace_bytes(const dart_dims* dims) {
    dart::Shape s;
    if (make_shape(dims, true, s) != DART_OK) return 0;
    return dart::sma_workspace_bytes(s);
}

dart_status dart_sma_fwd(const dart_dims* dims, const dart_sma_opts* opts, const void* q,
                         const void* e, const void* Cm, const void* mem, const void* z,
                         const void* y_ssd, void* y, float* lse, void* workspace,
                         size_t workspace_bytes, void* stream) {
    dart::Shape s;
    dart_status st = make_shape(dims, true, s);
    if (st != DART_OK) return st;
    st = check_opts(opts);
    if (st != DART_OK) return st;
    REQUIRE_PTR(q);
    REQUIRE_PTR(e);
    REQUIRE_PTR(Cm);
    REQUIRE_PTR(mem);
    REQUIRE_PTR(z);
    REQUIRE_PTR(y_ssd);
    REQUIRE_PTR(y);
    const size_t need = dart::sma_workspace_bytes(s);
    if (need > 0 && !workspace) return fail(DART_ERR_INVALID_ARG, "required pointer 'workspace' is NULL");
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    if (y != y_ssd) {
        // partial overlap between y and y_ssd is not allowed (exact aliasing is)
        const size_t bytes = (size_t)s.B * s.L * s.H * s.P * dart::elem_bytes(s.dtype);
        const char* a0 = (const char*)y;
        const char* b0 = (const char*)y_ssd;
        if (a0 < b0 + bytes && b0 < a0 + bytes)
            return fail(DART_ERR_INVALID_ARG, "y partially overlaps y_ssd (only exact aliasing is allowed)");
    }
    const dart::SmaArgs a = sma_args(opts);
    return hip_status(dart::launch_sma(s, a, q, e, Cm, mem, z, y_ssd, y, lse, workspace,
                                       (hipStream_t)stream),
                      "dart_sma_fwd launch");
}

size_t dart_sma_bwd_workspace_bytes(const dart_dims* dims) {
    dart::Shape s;
    if (make_shape(dims, true, s) != DART_OK) return 0;
    return dart::sma_bwd_workspace_bytes(s);
}

dart_status dart_sma_bwd(const dart_dims* dims, const dart_sma_opts* opts, const void* q,
                         const void* e, const void* Cm, const void* mem, const void* z,
                         const float* lse, const void* dy, float* dq, float* de, float* dC,
                         float* dmem, float* dz, void* workspace, size_t workspace_bytes,
                         void* stream) {
    dart::Shape s;
    dart_status st = make_shape(dims, true, s);
    if (st != DART_OK) return st;
    st = check_opts(opts);
    if (st != DART_OK) return st;
    REQUIRE_PTR(q);
    REQUIRE_PTR(e);
    REQUIRE_PTR(Cm);
    REQUIRE_PTR(mem);
    REQUIRE_PTR(z);
    REQUIRE_PTR(lse);
    REQUIRE_PTR(dy);
    REQUIRE_PTR(dq);
    REQUIRE_PTR(de);
    REQUIRE_PTR(dC);
    REQUIRE_PTR(dmem);
    REQUIRE_PTR(dz);
    REQUIRE_PTR(workspace);
    const size_t need = dart::sma_bwd_workspace_bytes(s);
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    return hip_status(dart::launch_sma_bwd(s, sma_args(opts), q, e, Cm, mem, z, lse, dy, dq, de, dC,
                                           dmem, dz, workspace, (hipStream_t)stream),
                      "dart_sma_bwd launch");
}

dart_status dart_conv1d_silu(int64_t batch, int64_t seqlen, int32_t channels, int64_t row_stride,
                             int32_t dtype, const void* in, const float* weight, const float* bias,
                             const float* state_in, float* state_out, void* out, void* stream) {
    if (batch < 1 || seqlen < 1 || channels < 1)
        return fail(DART_ERR_INVALID_ARG, "batch, seqlen and channels must be >= 1");
    if (batch > 65535 || (seqlen + 31) / 32 > 65535)
        return fail(DART_ERR_UNSUPPORTED, "batch <= 65535 and seqlen <= 32 * 65535");
    if (row_stride < channels)
        return fail(DART_ERR_INVALID_ARG, "row_stride (%lld) < channels (%d)", (long long)row_stride, channels);
    if (dtype != DART_FP32 && dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "dtype must be DART_FP32 or DART_BF16 (got %d)", dtype);
    REQUIRE_PTR(in);
    REQUIRE_PTR(weight);
    REQUIRE_PTR(out);
    if (state_out && state_out == state_in && seqlen > 32)
        return fail(DART_ERR_INVALID_ARG, "state_out may alias state_in only for seqlen <= 32");
    return hip_status(dart::launch_conv1d_silu(dtype, batch, seqlen, channels, row_stride, in, weight,
                                               bias, state_in, state_out, out, (hipStream_t)stream),
                      "dart_conv1d_silu launch");
}

dart_status dart_dt_softplus(int64_t rows, int32_t nheads, int64_t row_stride, int32_t dtype,
                             const void* raw, const float* bias, float* dt, void* stream) {
    if (rows < 1 || nheads < 1) return fail(DART_ERR_INVALID_ARG, "rows and nheads must be >= 1");
    if (row_stride < nheads)
        return fail(DART_ERR_INVALID_ARG, "row_stride (%lld) < nheads (%d)", (long long)row_stride, nheads);
    if (dtype != DART_FP32 && dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "dtype must be DART_FP32 or DART_BF16 (got %d)", dtype);
    if ((rows * nheads + 255) / 256 > 2147483647LL) return fail(DART_ERR_UNSUPPORTED, "too many rows");
    REQUIRE_PTR(raw);
    REQUIRE_PTR(dt);
    return hip_status(dart::launch_dt_softplus(dtype, rows, nheads, raw, row_stride, bias, dt,
                                               (hipStream_t)stream),
                      "dart_dt_softplus launch");
}

dart_status dart_gated_rmsnorm(int64_t rows, int32_t dim, int32_t group, int32_t dtype,
                               const void* y, const void* z, int64_t z_row_stride,
                               const float* weight, float eps, void* out, void* stream) {
    if (rows < 1 || dim < 1 || group < 1) return fail(DART_ERR_INVALID_ARG, "rows, dim and group must be >= 1");
    if (dim % group != 0 || group % 8 != 0)
        return fail(DART_ERR_INVALID_ARG, "group must divide dim and be a multiple of 8 (dim %d, group %d)", dim, group);
    if (z_row_stride < dim || z_row_stride % 8 != 0)
        return fail(DART_ERR_INVALID_ARG, "z_row_stride must be >= dim and a multiple of 8");
    if (dtype != DART_FP32 && dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "dtype must be DART_FP32 or DART_BF16 (got %d)", dtype);
    if (!(eps > 0.0f)) return fail(DART_ERR_INVALID_ARG, "eps must be > 0");
    REQUIRE_PTR(y);
    REQUIRE_PTR(z);
    REQUIRE_PTR(out);
    if (((uintptr_t)y | (uintptr_t)z | (uintptr_t)out | (uintptr_t)weight) % 16 != 0)
        return fail(DART_ERR_INVALID_ARG, "y, z, out and weight must be 16-byte aligned");
    if ((rows * (dim / group) + 3) / 4 > 2147483647LL) return fail(DART_ERR_UNSUPPORTED, "too many rows");
    return hip_status(dart::launch_gated_rmsnorm(dtype, rows, dim, group, y, z, z_row_stride, weight,
                                                 eps, out, (hipStream_t)stream),
                      "dart_gated_rmsnorm launch");
}

size_t dart_conv1d_silu_bwd_workspace_bytes(int64_t batch, int64_t seqlen, int32_t channels) {
    if (batch < 1 || seqlen < 1 || channels < 1) return 0;
    return dart::conv1d_silu_bwd_workspace_bytes(batch, seqlen, channels);
}

dart_status dart_conv1d_silu_bwd(int64_t batch, int64_t seqlen, int32_t channels,
                                 int64_t row_stride, int32_t dtype, const void* in,
                                 const float* weight, const float* bias, const float* state_in,
                                 const float* dout, float* din, int64_t din_row_stride,
                                 float* dweight, float* dbias, float* dstate_in, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    if (batch < 1 || seqlen < 1 || channels < 1)
        return fail(DART_ERR_INVALID_ARG, "batch, seqlen and channels must be >= 1");
    if (batch > 65535 || (seqlen + 31) / 32 > 65535)
        return fail(DART_ERR_UNSUPPORTED, "batch <= 65535 and seqlen <= 32 * 65535");
    if (row_stride < channels || din_row_stride < channels)
        return fail(DART_ERR_INVALID_ARG, "row strides must be >= channels (%d)", channels);
    if (dtype != DART_FP32 && dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "dtype must be DART_FP32 or DART_BF16 (got %d)", dtype);
    REQUIRE_PTR(in);
    REQUIRE_PTR(weight);
    REQUIRE_PTR(dout);
    REQUIRE_PTR(din);
    REQUIRE_PTR(dweight);
    REQUIRE_PTR(workspace);
    const size_t need = dart::conv1d_silu_bwd_workspace_bytes(batch, seqlen, channels);
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    return hip_status(dart::launch_conv1d_silu_bwd(dtype, batch, seqlen, channels, row_stride, in,
                                                   weight, bias, state_in, dout, din,
                                                   din_row_stride, dweight, dbias, dstate_in,
                                                   workspace, (hipStream_t)stream),
                      "dart_conv1d_silu_bwd launch");
}

size_t dart_dt_softplus_bwd_workspace_bytes(int64_t rows, int32_t nheads) {
    if (rows < 1 || nheads < 1) return 0;
    return dart::dt_softplus_bwd_workspace_bytes(rows, nheads);
}

dart_status dart_dt_softplus_bwd(int64_t rows, int32_t nheads, int64_t row_stride, int32_t dtype,
                                 const void* raw, const float* bias, const float* ddt, float* draw,
                                 int64_t draw_row_stride, float* dbias, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    if (rows < 1 || nheads < 1) return fail(DART_ERR_INVALID_ARG, "rows and nheads must be >= 1");
    if (row_stride < nheads || draw_row_stride < nheads)
        return fail(DART_ERR_INVALID_ARG, "row strides must be >= nheads (%d)", nheads);
    if (dtype != DART_FP32 && dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "dtype must be DART_FP32 or DART_BF16 (got %d)", dtype);
    if ((rows + 255) / 256 > 65535) return fail(DART_ERR_UNSUPPORTED, "too many rows");
    REQUIRE_PTR(raw);
    REQUIRE_PTR(ddt);
    REQUIRE_PTR(draw);
    REQUIRE_PTR(workspace);
    const size_t need = dart::dt_softplus_bwd_workspace_bytes(rows, nheads);
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    return hip_status(dart::launch_dt_softplus_bwd(dtype, rows, nheads, raw, row_stride, bias, ddt,
                                                   draw, draw_row_stride, dbias, workspace,
                                                   (hipStream_t)stream),
                      "dart_dt_softplus_bwd launch");
}

size_t dart_gated_rmsnorm_bwd_workspace_bytes(int64_t rows, int32_t dim) {
    if (rows < 1 || dim < 1) return 0;
    return dart::gated_rmsnorm_bwd_workspace_bytes(rows, dim);
}

dart_status dart_gated_rmsnorm_bwd(int64_t rows, int32_t dim, int32_t group, int32_t dtype,
                                   const void* y, const void* z, int64_t z_row_stride,
                                   const float* weight, float eps, const float* dout, float* dy,
                                   float* dz, int64_t dz_row_stride, float* dweight,
                                   void* workspace, size_t workspace_bytes, void* stream) {
    if (rows < 1 || dim < 1 || group < 1) return fail(DART_ERR_INVALID_ARG, "rows, dim and group must be >= 1");
    if (dim % group != 0 || group % 8 != 0)
        return fail(DART_ERR_INVALID_ARG, "group must divide dim and be a multiple of 8 (dim %d, group %d)", dim, group);
    if (group > 2048) return fail(DART_ERR_UNSUPPORTED, "the backward supports groups of at most 2048 channels");
    if (z_row_stride < dim || z_row_stride % 8 != 0 || dz_row_stride < dim || dz_row_stride % 8 != 0)
        return fail(DART_ERR_INVALID_ARG, "z and dz row strides must be >= dim and multiples of 8");
    if (dtype != DART_FP32 && dtype != DART_BF16)
        return fail(DART_ERR_INVALID_ARG, "dtype must be DART_FP32 or DART_BF16 (got %d)", dtype);
    if (!(eps > 0.0f)) return fail(DART_ERR_INVALID_ARG, "eps must be > 0");
    REQUIRE_PTR(y);
    REQUIRE_PTR(z);
    REQUIRE_PTR(dout);
    REQUIRE_PTR(dy);
    REQUIRE_PTR(dz);
    REQUIRE_PTR(workspace);
    if (((uintptr_t)y | (uintptr_t)z | (uintptr_t)dout | (uintptr_t)dy | (uintptr_t)dz) % 32 != 0)
        return fail(DART_ERR_INVALID_ARG, "y, z, dout, dy and dz must be 32-byte aligned");
    const size_t need = dart::gated_rmsnorm_bwd_workspace_bytes(rows, dim);
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    if ((rows / 16 + 1) * (dim / group) / 4 + 1 > 2147483647LL) return fail(DART_ERR_UNSUPPORTED, "too many rows");
    return hip_status(dart::launch_gated_rmsnorm_bwd(dtype, rows, dim, group, y, z, z_row_stride,
                                                     weight, eps, dout, dy, dz, dz_row_stride,
                                                     dweight, workspace, (hipStream_t)stream),
                      "dart_gated_rmsnorm_bwd launch");
}

// ---- the steps around the blocks ---------------------------------------------

static dart_status check_norm(int64_t rows, int32_t dim, int32_t center, int64_t x_row_stride, float eps) {
    if (rows < 0 || dim < 1) return fail(DART_ERR_INVALID_ARG, "rows must be >= 0 and dim >= 1");
    if (dim > 16384) return fail(DART_ERR_UNSUPPORTED, "dim %d not supported (at most 16384)", dim);
    if (center != 0 && center != 1) return fail(DART_ERR_INVALID_ARG, "center must be 0 or 1");
    if (x_row_stride < dim)
        return fail(DART_ERR_INVALID_ARG, "x_row_stride (%lld) < dim (%d)", (long long)x_row_stride, dim);
    if (too_large(rows, x_row_stride)) return fail(DART_ERR_UNSUPPORTED, "too many rows");
    if (!(eps > 0.0f)) return fail(DART_ERR_INVALID_ARG, "eps must be > 0");
    return DART_OK;
}

dart_status dart_layernorm(int64_t rows, int32_t dim, int32_t dtype, int32_t center, const void* x,
                           int64_t x_row_stride, const void* residual, int64_t residual_row_stride,
                           const float* weight, const float* bias, float eps, void* out, void* sum,
                           void* stream) {
    dart_status st = check_norm(rows, dim, center, x_row_stride, eps);
    if (st != DART_OK) return st;
    st = check_dtypes(dtype, DART_FP32);
    if (st != DART_OK) return st;
    if (!residual && sum) return fail(DART_ERR_INVALID_ARG, "sum needs a residual");
    if (residual && residual_row_stride < dim)
        return fail(DART_ERR_INVALID_ARG, "residual_row_stride (%lld) < dim (%d)", (long long)residual_row_stride, dim);
    if (residual && too_large(rows, residual_row_stride)) return fail(DART_ERR_UNSUPPORTED, "too many rows");
    if (rows == 0) return ok();
    REQUIRE_PTR(x);
    REQUIRE_PTR(out);
    const Range rx(x, rows, x_row_stride, dim, dtype), rr(residual, rows, residual_row_stride, dim, dtype);
    const Range ro(out, rows, dim, dim, dtype), rs(sum, rows, dim, dim, dtype);
    const Range rw(weight, 1, dim, dim, DART_FP32), rb(bias, 1, dim, dim, DART_FP32);
    for (const Range* o : {&ro, &rs}) {
        const bool is_x = o->a == rx.a && (x_row_stride == dim || rows == 1);
        const bool is_r = o->a == rr.a && (residual_row_stride == dim || rows == 1);
        if ((!is_x && o->meets(rx)) || (!is_r && o->meets(rr)) || o->meets(rw) || o->meets(rb))
            return fail(DART_ERR_INVALID_ARG, "an output overlaps an input (only x or residual itself, at row stride dim, is allowed)");
    }
    if (ro.meets(rs)) return fail(DART_ERR_INVALID_ARG, "out overlaps sum");
    return hip_status(dart::launch_layernorm(dtype, rows, dim, center, x, x_row_stride, residual,
                                             residual_row_stride, weight, bias, eps, out, sum,
                                             (hipStream_t)stream),
                      "dart_layernorm launch");
}

size_t dart_layernorm_bwd_workspace_bytes(int64_t rows, int32_t dim) {
    if (rows < 0 || dim < 1 || dim > 16384 || too_large(rows, dim)) return 0;
    return dart::layernorm_bwd_workspace_bytes(rows, dim);
}

dart_status dart_layernorm_bwd(int64_t rows, int32_t dim, int32_t dtype, int32_t grad_dtype,
                               int32_t center, const void* x, int64_t x_row_stride,
                               const float* weight, float eps, const void* dout, const void* dsum,
                               void* dx, float* dweight, float* dbias, void* workspace,
                               size_t workspace_bytes, void* stream) {
    dart_status st = check_norm(rows, dim, center, x_row_stride, eps);
    if (st != DART_OK) return st;
    st = check_dtypes(dtype, grad_dtype);
    if (st != DART_OK) return st;
    const size_t need = dart::layernorm_bwd_workspace_bytes(rows, dim);
    if (rows > 0) {
        REQUIRE_PTR(x);
        REQUIRE_PTR(dout);
        REQUIRE_PTR(dx);
        REQUIRE_PTR(workspace);
        const Range rx(x, rows, x_row_stride, dim, dtype), ro(dout, rows, dim, dim, grad_dtype);
        const Range rs(dsum, rows, dim, dim, grad_dtype), rd(dx, rows, dim, dim, grad_dtype);
        const Range rw(weight, 1, dim, dim, DART_FP32), rdw(dweight, 1, dim, dim, DART_FP32);
        const Range rdb(dbias, 1, dim, dim, DART_FP32);
        if (rd.meets(rx) || rd.meets(rw) || (rd.a != ro.a && rd.meets(ro)) || (rd.a != rs.a && rd.meets(rs)))
            return fail(DART_ERR_INVALID_ARG, "dx overlaps an input (only dout or dsum itself is allowed)");
        for (const Range* o : {&rdw, &rdb})
            if (o->meets(rx) || o->meets(ro) || o->meets(rs) || o->meets(rd) || o->meets(rw))
                return fail(DART_ERR_INVALID_ARG, "dweight or dbias overlaps another argument");
        if (rdw.meets(rdb)) return fail(DART_ERR_INVALID_ARG, "dweight overlaps dbias");
        st = check_apart({{"workspace", Range(workspace, need)}},
                         {{"x", rx}, {"weight", rw}, {"dout", ro}, {"dsum", rs}, {"dx", rd}, {"dweight", rdw}, {"dbias", rdb}});
        if (st != DART_OK) return st;
    }
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    if (workspace && (uintptr_t)workspace % 16 != 0)
        return fail(DART_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    return hip_status(dart::launch_layernorm_bwd(dtype, grad_dtype, rows, dim, center, x, x_row_stride,
                                                 weight, eps, dout, dsum, dx, dweight, dbias,
                                                 workspace, (hipStream_t)stream),
                      "dart_layernorm_bwd launch");
}

static dart_status check_logits(int64_t rows, int64_t vocab, int64_t row_stride, int32_t dtype,
                                int32_t grad_dtype, int32_t top_k) {
    if (rows < 0 || vocab < 1) return fail(DART_ERR_INVALID_ARG, "rows must be >= 0 and vocab >= 1");
    if (vocab > (1 << 24)) return fail(DART_ERR_UNSUPPORTED, "vocab %lld not supported (at most 2^24)", (long long)vocab);
    if (row_stride < vocab)
        return fail(DART_ERR_INVALID_ARG, "row_stride (%lld) < vocab (%lld)", (long long)row_stride, (long long)vocab);
    if (too_large(rows, row_stride)) return fail(DART_ERR_UNSUPPORTED, "too many rows");
    if (top_k < 0 || top_k > vocab)
        return fail(DART_ERR_INVALID_ARG, "top_k must be in [0, vocab] (got %d)", top_k);
    if (top_k > DART_MAX_TOP_K)
        return fail(DART_ERR_UNSUPPORTED, "top_k %d not supported (at most %d)", top_k, DART_MAX_TOP_K);
    return check_dtypes(dtype, grad_dtype);
}

static dart_status check_dlogits(int64_t rows, int64_t vocab, int64_t row_stride, int32_t dtype,
                                 int32_t grad_dtype, const void* logits, const void* dlogits,
                                 int64_t dlogits_row_stride) {
    if (dlogits_row_stride < vocab)
        return fail(DART_ERR_INVALID_ARG, "dlogits_row_stride (%lld) < vocab (%lld)",
                    (long long)dlogits_row_stride, (long long)vocab);
    if (too_large(rows, dlogits_row_stride)) return fail(DART_ERR_UNSUPPORTED, "too many rows");
    const Range rl(logits, rows, row_stride, vocab, dtype), rd(dlogits, rows, dlogits_row_stride, vocab, grad_dtype);
    const bool same = logits == dlogits && dtype == grad_dtype && (row_stride == dlogits_row_stride || rows == 1);
    if (!same && rl.meets(rd))
        return fail(DART_ERR_INVALID_ARG, "dlogits overlaps logits (only logits itself, of the same type and stride, is allowed)");
    return DART_OK;
}

// `n` values of the rows' results or weights.
static Range of_rows(const float* p, int64_t n) { return Range(p, (size_t)n * sizeof(float)); }
static Range of_rows(const int64_t* p, int64_t n) { return Range(p, (size_t)n * sizeof(int64_t)); }

size_t dart_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int32_t dtype, int32_t top_k) {
    if (check_logits(rows, vocab, vocab, dtype, DART_FP32, top_k) != DART_OK) return 0;
    return dart::token_logprobs_workspace_bytes(rows, vocab, dtype, top_k);
}

// The forward's checks, then the launch with `grad` (or NULL).
static dart_status run_token_logprobs(const dart::LogprobArgs& a, const dart::LogprobGrad* grad,
                                      void* workspace, size_t workspace_bytes, void* stream,
                                      const char* what) {
    if (a.rows == 0) return ok();
    if (!a.logits) return fail(DART_ERR_INVALID_ARG, "required pointer 'logits' is NULL");
    if (a.logprob && !a.targets) return fail(DART_ERR_INVALID_ARG, "logprob needs targets");
    if (a.top_k > 0 && (!a.top_ids || !a.top_logprobs))
        return fail(DART_ERR_INVALID_ARG, "top_k > 0 needs top_ids and top_logprobs");
    const size_t need = dart::token_logprobs_workspace_bytes(a.rows, a.vocab, a.dtype, a.top_k);
    if (need > 0 && !workspace) return fail(DART_ERR_INVALID_ARG, "required pointer 'workspace' is NULL");
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    if (workspace && (uintptr_t)workspace % 16 != 0)
        return fail(DART_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    const int64_t n = a.rows, k = a.rows * a.top_k;
    const dart::LogprobGrad g = grad ? *grad : dart::LogprobGrad{};
    const Range dlogits(g.dlogits, n, g.stride, a.vocab, g.dtype);
    // (dlogits against logits has rules of its own)
    dart_status st = check_apart(
        {{"logprob", of_rows(a.logprob, n)}, {"entropy", of_rows(a.entropy, n)}, {"row_max", of_rows(a.row_max, n)},
         {"log_sum", of_rows(a.log_sum, n)}, {"top_ids", of_rows(a.top_ids, k)}, {"top_logprobs", of_rows(a.top_logprobs, k)},
         {"workspace", Range(workspace, need)}},
        {{"logits", Range(a.logits, n, a.stride, a.vocab, a.dtype)}, {"targets", of_rows(a.targets, n)},
         {"dlogprob", of_rows(g.dlogprob, n)}, {"dentropy", of_rows(g.dentropy, n)}, {"dlse", of_rows(g.dlse, n)}, {"dlogits", dlogits}});
    if (st == DART_OK)
        st = check_apart({{"dlogits", dlogits}}, {{"targets", of_rows(a.targets, n)}, {"dlogprob", of_rows(g.dlogprob, n)},
                                                  {"dentropy", of_rows(g.dentropy, n)}, {"dlse", of_rows(g.dlse, n)}});
    if (st != DART_OK) return st;
    return hip_status(dart::launch_token_logprobs(a, grad, workspace, (hipStream_t)stream), what);
}

dart_status dart_token_logprobs(int64_t rows, int64_t vocab, int64_t row_stride, int32_t dtype,
                                const void* logits, const int64_t* targets, int64_t ignore_index,
                                int32_t top_k, float* logprob, float* entropy, float* row_max,
                                float* log_sum, int64_t* top_ids, float* top_logprobs,
                                void* workspace, size_t workspace_bytes, void* stream) {
    dart_status st = check_logits(rows, vocab, row_stride, dtype, DART_FP32, top_k);
    if (st != DART_OK) return st;
    const dart::LogprobArgs a{rows, vocab, row_stride, dtype, top_k, logits, targets, ignore_index,
                              logprob, entropy, row_max, log_sum, top_ids, top_logprobs};
    return run_token_logprobs(a, nullptr, workspace, workspace_bytes, stream, "dart_token_logprobs launch");
}

dart_status dart_token_logprobs_bwd(int64_t rows, int64_t vocab, int64_t row_stride, int32_t dtype,
                                    int32_t grad_dtype, const void* logits, const int64_t* targets,
                                    int64_t ignore_index, const float* row_max,
                                    const float* log_sum, const float* entropy,
                                    const float* dlogprob, const float* dentropy,
                                    const float* dlse, void* dlogits, int64_t dlogits_row_stride,
                                    void* stream) {
    dart_status st = check_logits(rows, vocab, row_stride, dtype, grad_dtype, 0);
    if (st != DART_OK) return st;
    st = check_dlogits(rows, vocab, row_stride, dtype, grad_dtype, logits, dlogits, dlogits_row_stride);
    if (st != DART_OK) return st;
    if (dlogprob && !targets) return fail(DART_ERR_INVALID_ARG, "dlogprob needs targets");
    if (rows == 0) return ok();
    REQUIRE_PTR(logits);
    REQUIRE_PTR(row_max);
    REQUIRE_PTR(log_sum);
    REQUIRE_PTR(dlogits);
    if (dentropy && !entropy) return fail(DART_ERR_INVALID_ARG, "dentropy needs entropy");
    st = check_apart({{"dlogits", Range(dlogits, rows, dlogits_row_stride, vocab, grad_dtype)}},
                     {{"targets", of_rows(targets, rows)}, {"row_max", of_rows(row_max, rows)}, {"log_sum", of_rows(log_sum, rows)},
                      {"entropy", of_rows(entropy, rows)}, {"dlogprob", of_rows(dlogprob, rows)},
                      {"dentropy", of_rows(dentropy, rows)}, {"dlse", of_rows(dlse, rows)}});
    if (st != DART_OK) return st;
    const dart::LogprobArgs a{rows, vocab, row_stride, dtype, 0, logits, targets, ignore_index,
                              nullptr, const_cast<float*>(entropy), const_cast<float*>(row_max),
                              const_cast<float*>(log_sum), nullptr, nullptr};
    const dart::LogprobGrad g{grad_dtype, dlogits_row_stride, dlogprob, dentropy, dlse, dlogits};
    return hip_status(dart::launch_token_logprobs_bwd(a, g, (hipStream_t)stream), "dart_token_logprobs_bwd launch");
}

dart_status dart_token_logprobs_grad(int64_t rows, int64_t vocab, int64_t row_stride, int32_t dtype,
                                     int32_t grad_dtype, const void* logits, const int64_t* targets,
                                     int64_t ignore_index, int32_t top_k, const float* dlogprob,
                                     const float* dentropy, const float* dlse, float* logprob,
                                     float* entropy, float* row_max, float* log_sum,
                                     int64_t* top_ids, float* top_logprobs, void* dlogits,
                                     int64_t dlogits_row_stride, void* workspace,
                                     size_t workspace_bytes, void* stream) {
    dart_status st = check_logits(rows, vocab, row_stride, dtype, grad_dtype, top_k);
    if (st != DART_OK) return st;
    st = check_dlogits(rows, vocab, row_stride, dtype, grad_dtype, logits, dlogits, dlogits_row_stride);
    if (st != DART_OK) return st;
    if (dlogprob && !targets) return fail(DART_ERR_INVALID_ARG, "dlogprob needs targets");
    if (rows > 0) {
        REQUIRE_PTR(row_max);
        REQUIRE_PTR(log_sum);
        REQUIRE_PTR(dlogits);
        if (dentropy && !entropy) return fail(DART_ERR_INVALID_ARG, "dentropy needs entropy");
    }
    const dart::LogprobArgs a{rows, vocab, row_stride, dtype, top_k, logits, targets, ignore_index,
                              logprob, entropy, row_max, log_sum, top_ids, top_logprobs};
    const dart::LogprobGrad g{grad_dtype, dlogits_row_stride, dlogprob, dentropy, dlse, dlogits};
    return run_token_logprobs(a, &g, workspace, workspace_bytes, stream, "dart_token_logprobs_grad launch");
}

// Checks of a list of tensors; outs == NULL: they are only read.
static dart_status check_grads(int64_t n, const void* const* grads, void* const* outs, const int64_t* numels,
                               const int32_t* dtypes, const int32_t* out_dtypes, float scale,
                               const float* norm, const void* workspace, size_t workspace_bytes) {
    if (n < 0) return fail(DART_ERR_INVALID_ARG, "n must be >= 0 (got %lld)", (long long)n);
    if (n > (1 << 24)) return fail(DART_ERR_UNSUPPORTED, "at most 2^24 tensors");
    if (!std::isfinite(scale)) return fail(DART_ERR_INVALID_ARG, "scale must be finite");
    REQUIRE_PTR(norm);
    REQUIRE_PTR(workspace);
    if (workspace_bytes < dart::grad_norm_workspace_bytes(n))
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes,
                    dart::grad_norm_workspace_bytes(n));
    if ((uintptr_t)workspace % 16 != 0) return fail(DART_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    const Range rn(norm, sizeof(float)), rws(workspace, dart::grad_norm_workspace_bytes(n));
    if (rn.meets(rws)) return fail(DART_ERR_INVALID_ARG, "norm overlaps workspace");
    if (n == 0) return DART_OK;
    REQUIRE_PTR(grads);
    REQUIRE_PTR(numels);
    REQUIRE_PTR(dtypes);
    int64_t total = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (numels[i] < 0 || numels[i] > ((int64_t)1 << 42) || (total += numels[i]) > ((int64_t)1 << 42))
            return fail(DART_ERR_INVALID_ARG, "tensor %lld: element counts must be >= 0, and at most 2^42 in all", (long long)i);
        for (int d : {dtypes[i], outs ? out_dtypes[i] : dtypes[i]})
            if (d != DART_FP32 && d != DART_BF16)
                return fail(DART_ERR_INVALID_ARG, "tensor %lld: dtype must be DART_FP32 or DART_BF16 (got %d)", (long long)i, d);
        if (numels[i] == 0) continue;
        if (!grads[i] || (outs && !outs[i])) return fail(DART_ERR_INVALID_ARG, "tensor %lld: pointer is NULL", (long long)i);
        if ((uintptr_t)grads[i] % dart::elem_bytes(dtypes[i]) != 0 ||
            (outs && (uintptr_t)outs[i] % dart::elem_bytes(out_dtypes[i]) != 0))
            return fail(DART_ERR_INVALID_ARG, "tensor %lld: not aligned to its elements", (long long)i);
        const Range g(grads[i], 1, 0, numels[i], dtypes[i]);
        const Range o = outs ? Range(outs[i], 1, 0, numels[i], out_dtypes[i]) : g;
        if (g.meets(rn) || g.meets(rws) || o.meets(rn) || o.meets(rws))
            return fail(DART_ERR_INVALID_ARG, "tensor %lld: overlaps norm or workspace", (long long)i);
    }
    if (!outs) return DART_OK;
    // Whatever is written may meet nothing else: the ranges in order of their
    // start, each against the furthest end so far.
    struct Span {
        uintptr_t a, b;
        bool written;
    };
    Span* v = new (std::nothrow) Span[2 * (size_t)n];
    if (!v) return fail(DART_ERR_INVALID_ARG, "out of host memory");
    size_t m = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (numels[i] == 0) continue;
        const Range g(grads[i], 1, 0, numels[i], dtypes[i]), o(outs[i], 1, 0, numels[i], out_dtypes[i]);
        if (g.a != o.a || dtypes[i] != out_dtypes[i]) v[m++] = Span{g.a, g.b, false};
        v[m++] = Span{o.a, o.b, true};
    }
    std::sort(v, v + m, [](const Span& p, const Span& q) { return p.a < q.a; });
    uintptr_t end = 0, end_written = 0;
    bool clash = false;
    for (size_t i = 0; i < m; ++i) {
        clash = clash || v[i].a < (v[i].written ? end : end_written);
        end = std::max(end, v[i].b);
        if (v[i].written) end_written = std::max(end_written, v[i].b);
    }
    delete[] v;
    if (clash)
        return fail(DART_ERR_INVALID_ARG, "an output overlaps another tensor (the same one twice?)");
    return DART_OK;
}

size_t dart_grad_norm_workspace_bytes(int64_t n) {
    if (n < 0 || n > (1 << 24)) return 0;
    return dart::grad_norm_workspace_bytes(n);
}

dart_status dart_grad_norm(int64_t n, const void* const* grads, const int64_t* numels,
                           const int32_t* dtypes, float scale, float* norm, void* workspace,
                           size_t workspace_bytes, void* stream) {
    const dart_status st = check_grads(n, grads, nullptr, numels, dtypes, nullptr, scale, norm, workspace, workspace_bytes);
    if (st != DART_OK) return st;
    return hip_status(dart::launch_clip_grad_norm(n, grads, nullptr, numels, dtypes, nullptr, INFINITY,
                                                  scale, norm, workspace, (hipStream_t)stream),
                      "dart_grad_norm launch");
}

dart_status dart_clip_grad_norm(int64_t n, const void* const* grads, void* const* outs,
                                const int64_t* numels, const int32_t* dtypes,
                                const int32_t* out_dtypes, float max_norm, float scale, float* norm,
                                void* workspace, size_t workspace_bytes, void* stream) {
    if (!(max_norm >= 0.0f)) return fail(DART_ERR_INVALID_ARG, "max_norm must be >= 0");
    if (n > 0) {
        REQUIRE_PTR(outs);
        REQUIRE_PTR(out_dtypes);
    }
    const dart_status st = check_grads(n, grads, outs, numels, dtypes, out_dtypes, scale, norm, workspace, workspace_bytes);
    if (st != DART_OK) return st;
    return hip_status(dart::launch_clip_grad_norm(n, grads, outs, numels, dtypes, out_dtypes, max_norm,
                                                  scale, norm, workspace, (hipStream_t)stream),
                      "dart_clip_grad_norm launch");
}

size_t dart_decode_workspace_bytes(const dart_dims* dims) {
    dart::Shape s;
    if (make_shape(dims, false, s) != DART_OK) return 0;
    if (s.Mcap < 1) return 0;
    return dart::decode_workspace_bytes(s);
}

dart_status dart_decode_step(const dart_dims* dims, const dart_sma_opts* opts, int64_t pos,
                             const void* x, const float* dt, const float* A, const void* Bm,
                             const void* Cm, const void* q, const void* e, const void* z,
                             float* h_state, float* chunk_acc, void* mem_cache, void* y,
                             void* workspace, size_t workspace_bytes, void* stream) {
    dart::Shape s;
    dart_status st = make_shape(dims, false, s);
    if (st != DART_OK) return st;
    st = check_opts(opts);
    if (st != DART_OK) return st;
    if (s.Mcap < 1) return fail(DART_ERR_INVALID_ARG, "decode needs mem_capacity >= 1");
    if (pos < 0) return fail(DART_ERR_INVALID_ARG, "pos must be >= 0 (got %lld)", (long long)pos);
    const int64_t m = pos / s.S;
    if (m > s.Mcap)
        return fail(DART_ERR_INVALID_ARG, "pos %lld needs %lld cached memories > capacity %lld",
                    (long long)pos, (long long)m, (long long)s.Mcap);
    if (pos % s.S == s.S - 1 && m >= s.Mcap)
        return fail(DART_ERR_INVALID_ARG, "pos %lld closes chunk %lld but the cache holds %lld memories",
                    (long long)pos, (long long)m, (long long)s.Mcap);
    REQUIRE_PTR(x);
    REQUIRE_PTR(dt);
    REQUIRE_PTR(A);
    REQUIRE_PTR(Bm);
    REQUIRE_PTR(Cm);
    REQUIRE_PTR(q);
    REQUIRE_PTR(e);
    REQUIRE_PTR(z);
    REQUIRE_PTR(h_state);
    REQUIRE_PTR(chunk_acc);
    REQUIRE_PTR(mem_cache);
    REQUIRE_PTR(y);
    REQUIRE_PTR(workspace);
    const size_t need = dart::decode_workspace_bytes(s);
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    const dart::SmaArgs a = sma_args(opts);
    return hip_status(dart::launch_decode(s, a, pos, nullptr, x, dt, A, Bm, Cm, q, e, z, h_state,
                                          chunk_acc, mem_cache, y, workspace, (hipStream_t)stream),
                      "dart_decode_step launch");
}

dart_status dart_decode_step_noalloc(const dart_dims* dims, const dart_sma_opts* opts, int64_t pos,
                                     const void* x, const float* dt, const float* A,
                                     const void* Bm, const void* Cm, const void* q, const void* e,
                                     const void* z, float* h_state, float* chunk_acc,
                                     void* mem_cache, void* y, void* stream) {
    dart::Shape s;
    dart_status st = make_shape(dims, false, s);
    if (st != DART_OK) return st;
    st = check_opts(opts);
    if (st != DART_OK) return st;
    if (s.Mcap < 1) return fail(DART_ERR_INVALID_ARG, "decode needs mem_capacity >= 1");
    if (pos < 0) return fail(DART_ERR_INVALID_ARG, "pos must be >= 0 (got %lld)", (long long)pos);
    const int64_t m = pos / s.S;
    if (m > s.Mcap)
        return fail(DART_ERR_INVALID_ARG, "pos %lld needs %lld cached memories > capacity %lld",
                    (long long)pos, (long long)m, (long long)s.Mcap);
    if (pos % s.S == s.S - 1 && m >= s.Mcap)
        return fail(DART_ERR_INVALID_ARG, "pos %lld closes chunk %lld but the cache holds %lld memories",
                    (long long)pos, (long long)m, (long long)s.Mcap);
    REQUIRE_PTR(x);
    REQUIRE_PTR(dt);
    REQUIRE_PTR(A);
    REQUIRE_PTR(Bm);
    REQUIRE_PTR(Cm);
    REQUIRE_PTR(q);
    REQUIRE_PTR(e);
    REQUIRE_PTR(z);
    REQUIRE_PTR(h_state);
    REQUIRE_PTR(chunk_acc);
    REQUIRE_PTR(mem_cache);
    REQUIRE_PTR(y);
    const size_t need = dart::decode_noalloc_scratch_bytes(s, pos);
    if (need > (size_t)DART_DECODE_NOALLOC_SCRATCH_BYTES)
        return fail(DART_ERR_UNSUPPORTED,
                    "this step needs %zu bytes of scratch; the library's fixed scratch holds %zu "
                    "(use dart_decode_step with a workspace)",
                    need, (size_t)DART_DECODE_NOALLOC_SCRATCH_BYTES);
    const dart::SmaArgs a = sma_args(opts);
    return hip_status(dart::launch_decode_noalloc(s, a, pos, x, dt, A, Bm, Cm, q, e, z, h_state,
                                                  chunk_acc, mem_cache, y, (hipStream_t)stream),
                      "dart_decode_step_noalloc launch");
}

dart_status dart_decode_step_ragged(const dart_dims* dims, const dart_sma_opts* opts,
                                    const int64_t* pos, int64_t pos_max, const void* x,
                                    const float* dt, const float* A, const void* Bm,
                                    const void* Cm, const void* q, const void* e, const void* z,
                                    float* h_state, float* chunk_acc, void* mem_cache, void* y,
                                    void* workspace, size_t workspace_bytes, void* stream) {
    dart::Shape s;
    dart_status st = make_shape(dims, false, s);
    if (st != DART_OK) return st;
    st = check_opts(opts);
    if (st != DART_OK) return st;
    if (s.Mcap < 1) return fail(DART_ERR_INVALID_ARG, "decode needs mem_capacity >= 1");
    if (pos_max < 0)
        return fail(DART_ERR_INVALID_ARG, "pos_max must be >= 0 (got %lld)", (long long)pos_max);
    if (pos_max >= s.Mcap * s.S)
        return fail(DART_ERR_INVALID_ARG,
                    "pos_max %lld needs more than the %lld memories the cache holds",
                    (long long)pos_max, (long long)s.Mcap);
    REQUIRE_PTR(pos);
    REQUIRE_PTR(x);
    REQUIRE_PTR(dt);
    REQUIRE_PTR(A);
    REQUIRE_PTR(Bm);
    REQUIRE_PTR(Cm);
    REQUIRE_PTR(q);
    REQUIRE_PTR(e);
    REQUIRE_PTR(z);
    REQUIRE_PTR(h_state);
    REQUIRE_PTR(chunk_acc);
    REQUIRE_PTR(mem_cache);
    REQUIRE_PTR(y);
    REQUIRE_PTR(workspace);
    const size_t need = dart::decode_workspace_bytes(s);
    if (workspace_bytes < need)
        return fail(DART_ERR_INVALID_ARG, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    const dart::SmaArgs a = sma_args(opts);
    return hip_status(dart::launch_decode(s, a, pos_max, pos, x, dt, A, Bm, Cm, q, e, z, h_state,
                                          chunk_acc, mem_cache, y, workspace, (hipStream_t)stream),
                      "dart_decode_step_ragged launch");
}

dart_status dart_decode_handoff(const dart_dims* dims, const int64_t* lengths, const void* mem,
                                const float* h_last, float* h_state, float* chunk_acc,
                                void* stream) {
    dart::Shape s;
    dart_status st = make_shape(dims, false, s);
    if (st != DART_OK) return st;
    if (s.Mcap < 1) return fail(DART_ERR_INVALID_ARG, "handoff needs mem_capacity >= 1");
    REQUIRE_PTR(lengths);
    REQUIRE_PTR(mem);
    REQUIRE_PTR(h_last);
    REQUIRE_PTR(h_state);
    REQUIRE_PTR(chunk_acc);
    return hip_status(dart::launch_decode_handoff(s, mem, h_last, lengths, h_state, chunk_acc,
                                                  (hipStream_t)stream),
                      "dart_decode_handoff launch");
}

int64_t dart_decode_cache_elems(const dart_dims* dims, int64_t context) {
    if (!dims || context < 0 || dims->batch < 1 || dims->nheads < 1 || dims->headdim < 1 ||
        dims->dstate < 1 || dims->chunk < 1)
        return 0;
    const int64_t mems = (context + dims->chunk - 1) / dims->chunk;
    return dims->batch * mems * dims->nheads * (int64_t)dims->dstate * dims->headdim;
}

const char* dart_status_string(dart_status status) {
    switch (status) {
        case DART_OK: return "DART_OK";
        case DART_ERR_INVALID_ARG: return "DART_ERR_INVALID_ARG";
        case DART_ERR_UNSUPPORTED: return "DART_ERR_UNSUPPORTED";
        case DART_ERR_HIP: return "DART_ERR_HIP";
    }
    return "DART_ERR_UNKNOWN";
}

const char* dart_last_error(void) { return g_err; }

}  // extern "C"
