// C entry points of the operators around the convolutions (include/patdnn.h): checks of the arguments, and the launches.
#include <cmath>
#include <initializer_list>
#include <new>
#include <string>

#include "../../include/patdnn.h"
#include "operators.hpp"

using namespace patdnn;

namespace patdnn {
void set_last_error(const std::string& msg);     // patdnn_api.hip
}

static_assert(PATDNN_F32 == kF32 && PATDNN_F16 == kF16 && PATDNN_BF16 == kBF16 && PATDNN_MXFP4 == kMxfp4, "one numbering");
static_assert(PATDNN_ACT_NONE == kActNone && PATDNN_ACT_RELU == kActRelu && PATDNN_ACT_SILU == kActSilu, "one numbering");

namespace {

// No exception leaves the C interface: a text that finds no memory is dropped.
patdnn_status_t fail(patdnn_status_t s, const char* what, const char* more = "")
{
    try {
        set_last_error(std::string(what) + more);
    } catch (const std::bad_alloc&) {
    }
    return s;
}
patdnn_status_t done(hipError_t e, const char* what)
{
    if (e == hipSuccess) return PATDNN_OK;
    try {
        set_last_error(std::string(what) + ": " + hipGetErrorString(e));
    } catch (const std::bad_alloc&) {
    }
    return PATDNN_EHIP;
}

bool real_type(int32_t t) { return t == kF32 || t == kF16 || t == kBF16; }
bool aligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

// A strided tensor [n][pixels][channels], or [1][rows][values]: its bytes from the first element to the last, in runs of `width` that all start a
// multiple of `pitch` behind the first (0: not in such a rhythm).
struct Span {
    const void* p;
    long long bytes, pitch = 0, width = 0;
};
// False if the elements from the first to the last are more than addresses can count.
bool span_of(long long n, long long image, long long pixels, long long pixel, long long channels, int type, const void* p, Span& s)
{
    const __int128 elements = (__int128)(n - 1) * image + (__int128)(pixels - 1) * pixel + channels;
    if (elements > ((__int128)1 << 56)) return false;
    const long long size = (long long)element_bytes(type);
    s = Span{p, (long long)elements * size};
    const long long pitch = pixels > 1 ? pixel : n > 1 ? image : 0;
    if (pitch && (n == 1 || image % pitch == 0)) s.pitch = pitch * size, s.width = channels * size;
    return true;
}
bool overlap(const Span& a, const Span& b)
{
    const char* p = static_cast<const char*>(a.p);
    const char* q = static_cast<const char*>(b.p);
    if (!(p && q && p < q + b.bytes && q < p + a.bytes)) return false;
    if (!a.pitch || a.pitch != b.pitch) return true;
    // slices of one wider tensor: b's runs start `d` behind a's
    const long long ahead = (q - p) % a.pitch, d = ahead < 0 ? ahead + a.pitch : ahead;
    return d < a.width || d + b.width > a.pitch;
}
// Whether an output shares memory with an input or with another output (NULL: not there).
bool outputs_overlap(std::initializer_list<Span> inputs, std::initializer_list<Span> outputs)
{
    for (const Span& a : outputs) {
        for (const Span& b : inputs)
            if (overlap(a, b)) return true;
        for (const Span& b : outputs)
            if (&a != &b && overlap(a, b)) return true;
    }
    return false;
}

patdnn_status_t reorder(bool last, const void* in, int32_t in_type, int32_t n, int32_t channels, int32_t pixels, void* out, int32_t out_type,
                        int64_t image, int64_t pixel, void* stream)
{
    if (!real_type(in_type) || !real_type(out_type)) return fail(PATDNN_EINVAL, "unknown element type");
    if (n < 0 || channels <= 0 || pixels <= 0) return fail(PATDNN_EINVAL, "n must be >= 0 and channels, pixels positive");
    if (image < 0 || pixel < 0) return fail(PATDNN_EINVAL, "strides must be >= 0");
    const long long dense = (long long)channels * pixels;
    if (last && ((pixels > 1 && pixel < channels) || (n > 1 && (__int128)image < (__int128)(pixels - 1) * pixel + channels)))
        return fail(PATDNN_EINVAL, "output strides make pixels or images overlap");
    if (n == 0) return PATDNN_OK;
    if (!in || !out) return fail(PATDNN_EINVAL, "input / output is NULL");
    if (!aligned(in, element_bytes(in_type)) || !aligned(out, element_bytes(out_type))) return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    Span a, b;
    if (!span_of(n, dense, 1, 0, dense, last ? in_type : out_type, last ? in : out, a) ||
        !span_of(n, image, pixels, pixel, channels, last ? out_type : in_type, last ? out : in, b))
        return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    if (overlap(a, b)) return fail(PATDNN_EINVAL, "output overlaps input");
    const TransposeShape s = last ? TransposeShape{n, channels, pixels, in_type, out_type, dense, pixels, image, pixel}
                                  : TransposeShape{n, pixels, channels, in_type, out_type, image, pixel, dense, pixels};
    if (!transpose_fits(s)) return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    return done(launch_transpose(s, in, out, static_cast<hipStream_t>(stream)), "launching the change of channel order");
}

patdnn_status_t norm_shape(const patdnn_norm_desc_t* d, bool backward, NormShape& s)
{
    if (!d) return fail(PATDNN_EINVAL, "desc is NULL");
    if (d->n < 0 || d->pixels <= 0 || d->channels <= 0 || d->groups <= 0 || d->channels % d->groups != 0)
        return fail(PATDNN_EINVAL, "n must be >= 0, pixels, channels and groups positive, and groups divide channels");
    if (!real_type(d->type)) return fail(PATDNN_EINVAL, "unknown element type");
    if (d->act < kActNone || d->act > kActSilu) return fail(PATDNN_EINVAL, "unknown activation");
    if (!backward && !(d->eps >= 0.0f && std::isfinite(d->eps))) return fail(PATDNN_EINVAL, "eps must be finite and >= 0");
    if (d->x_image < 0 || d->x_pixel < 0 || (backward && (d->dy_image < 0 || d->dy_pixel < 0))) return fail(PATDNN_EINVAL, "strides must be >= 0");
    if ((d->pixels > 1 && d->y_pixel < d->channels) || d->y_pixel < 0 || d->y_image < 0 ||
        (d->n > 1 && (__int128)d->y_image < (__int128)(d->pixels - 1) * d->y_pixel + d->channels))
        return fail(PATDNN_EINVAL, "output strides make pixels or images overlap");
    s = NormShape{d->n, d->pixels, d->channels, d->groups, d->type, d->act, d->eps, d->x_image, d->x_pixel, d->y_image, d->y_pixel,
                  backward ? d->dy_image : 0, backward ? d->dy_pixel : 0};
    if (!norm_fits(s)) return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    return PATDNN_OK;
}

patdnn_status_t check_workspace(const void* p, size_t has, size_t needs, const char* name)
{
    if (needs && (!p || has < needs)) return fail(PATDNN_EINVAL, "the workspace is NULL or too small: see ", name);
    return PATDNN_OK;
}

bool linear_shape(const patdnn_linear_desc_t* d, LinearShape& s, const char*& why)
{
    why = "desc is NULL";
    if (!d) return false;
    why = "rows must be >= 0 and in_features, out_features positive";
    if (d->rows < 0 || d->in_features <= 0 || d->out_features <= 0) return false;
    why = "unknown element type";
    if (!(real_type(d->x_type) || d->x_type == kMxfp4) || !real_type(d->out_type)) return false;
    why = "unknown activation";
    if (d->act < kActNone || d->act > kActSilu) return false;
    why = "strides must be >= 0, and output rows must not overlap";
    if ((d->x_type != kMxfp4 && d->x_row < 0) || d->out_row < 0 || (d->rows > 1 && d->out_row < d->out_features)) return false;
    s = LinearShape{d->rows, d->in_features, d->out_features, d->x_type, d->out_type, d->act, d->x_type == kMxfp4 ? 0 : d->x_row, d->out_row};
    return true;
}

long long code_bytes(long long rows, long long cols) { return rows * mxfp4_pieces(cols) * 64; }

patdnn_status_t check_codes(const void* codes, const void* scales)
{
    if (!codes || !scales) return fail(PATDNN_EINVAL, "codes / scales is NULL");
    if (!aligned(codes, 16) || !aligned(scales, 4)) return fail(PATDNN_EINVAL, "codes must be 16-byte aligned and scales 4-byte aligned");
    return PATDNN_OK;
}

patdnn_status_t convert(bool quantize, void* values, int32_t type, int32_t rows, int32_t cols, int64_t row, uint8_t* codes, uint8_t* scales,
                        void* stream)
{
    if (!real_type(type)) return fail(PATDNN_EINVAL, "unknown element type");
    if (rows < 0 || cols <= 0) return fail(PATDNN_EINVAL, "rows must be >= 0 and cols positive");
    if (row < 0 || (!quantize && rows > 1 && row < cols)) return fail(PATDNN_EINVAL, "strides must be >= 0, and output rows must not overlap");
    if (rows == 0) return PATDNN_OK;
    if (!values) return fail(PATDNN_EINVAL, "x / out is NULL");
    if (const patdnn_status_t st = check_codes(codes, scales)) return st;
    if (!aligned(values, element_bytes(type))) return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    const Mxfp4Shape s{rows, cols, type, row};
    Span a;
    if (!mxfp4_fits(s) || !span_of(1, 0, rows, row, cols, type, values, a)) return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    const Span b{codes, code_bytes(rows, cols)}, c{scales, code_bytes(rows, cols) / 16};
    if (overlap(a, b) || overlap(a, c) || (quantize && overlap(b, c))) return fail(PATDNN_EINVAL, "output overlaps input");
    return quantize ? done(launch_mxfp4_quantize(s, values, codes, scales, static_cast<hipStream_t>(stream)), "launching the quantisation")
                    : done(launch_mxfp4_dequantize(s, codes, scales, values, static_cast<hipStream_t>(stream)), "launching the dequantisation");
}

}  // namespace

extern "C" {

patdnn_status_t patdnn_channels_last(const void* input, int32_t in_type, int32_t n, int32_t channels, int32_t pixels, void* output,
                                     int32_t out_type, int64_t out_image, int64_t out_pixel, void* stream)
{
    return reorder(true, input, in_type, n, channels, pixels, output, out_type, out_image, out_pixel, stream);
}

patdnn_status_t patdnn_channels_first(const void* input, int32_t in_type, int64_t in_image, int64_t in_pixel, int32_t n, int32_t channels,
                                      int32_t pixels, void* output, int32_t out_type, void* stream)
{
    return reorder(false, input, in_type, n, channels, pixels, output, out_type, in_image, in_pixel, stream);
}

size_t patdnn_group_norm_workspace_floats(const patdnn_norm_desc_t* desc, int32_t backward)
{
    NormShape s{};
    return norm_shape(desc, backward != 0, s) == PATDNN_OK ? norm_workspace_floats(s, backward != 0) : 0;
}

patdnn_status_t patdnn_group_norm(const patdnn_norm_desc_t* desc, const void* x, const float* gamma, const float* beta, void* y, float* mean,
                                  float* rstd, float* workspace, size_t workspace_floats, void* stream)
{
    NormShape s{};
    if (const patdnn_status_t st = norm_shape(desc, false, s)) return st;
    if (s.n == 0) return PATDNN_OK;
    if (!x || !y) return fail(PATDNN_EINVAL, "x / y is NULL");
    if (!aligned(x, element_bytes(s.type)) || !aligned(y, element_bytes(s.type)) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) ||
        !aligned(rstd, 4) || !aligned(workspace, 4))
        return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    Span in, out;
    if (!span_of(s.n, s.x_image, s.pixels, s.x_pixel, s.c, s.type, x, in) || !span_of(s.n, s.y_image, s.pixels, s.y_pixel, s.c, s.type, y, out))
        return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    if (overlap(in, out)) return fail(PATDNN_EINVAL, "output overlaps input");
    const size_t needs = norm_workspace_floats(s, false);
    if (const patdnn_status_t st = check_workspace(workspace, workspace_floats, needs, "patdnn_group_norm_workspace_floats")) return st;
    const Span work{workspace, (long long)needs * 4};
    if (overlap(work, in) || overlap(work, out)) return fail(PATDNN_EINVAL, "workspace overlaps input or output");
    const long long channels = 4ll * s.c, statistics = 4ll * s.n * s.groups;
    if (outputs_overlap({in, {gamma, channels}, {beta, channels}}, {out, work, {mean, statistics}, {rstd, statistics}}))
        return fail(PATDNN_EINVAL, "an output or the workspace overlaps another tensor");
    return done(launch_norm(s, x, gamma, beta, y, mean, rstd, workspace, static_cast<hipStream_t>(stream)), "launching the group norm");
}

patdnn_status_t patdnn_group_norm_backward(const patdnn_norm_desc_t* desc, const void* dy, const void* x, const float* mean, const float* rstd,
                                           const float* gamma, const float* beta, void* dx, float* dgamma, float* dbeta, float* workspace,
                                           size_t workspace_floats, void* stream)
{
    NormShape s{};
    if (const patdnn_status_t st = norm_shape(desc, true, s)) return st;
    if (!aligned(dgamma, 4) || !aligned(dbeta, 4)) return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    if (s.n > 0) {
        if (!x || !dy || !dx || !mean || !rstd) return fail(PATDNN_EINVAL, "x / dy / dx / mean / rstd is NULL");
        if (!aligned(x, element_bytes(s.type)) || !aligned(dy, element_bytes(s.type)) || !aligned(dx, element_bytes(s.type)) || !aligned(mean, 4) ||
            !aligned(rstd, 4) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(workspace, 4))
            return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
        Span in, grad, out;
        if (!span_of(s.n, s.x_image, s.pixels, s.x_pixel, s.c, s.type, x, in) || !span_of(s.n, s.dy_image, s.pixels, s.dy_pixel, s.c, s.type, dy, grad) ||
            !span_of(s.n, s.y_image, s.pixels, s.y_pixel, s.c, s.type, dx, out))
            return fail(PATDNN_EUNSUPPORTED, "tensor too large");
        if (overlap(in, out) || overlap(grad, out)) return fail(PATDNN_EINVAL, "output overlaps input");
        const size_t needs = norm_workspace_floats(s, true);
        if (const patdnn_status_t st = check_workspace(workspace, workspace_floats, needs, "patdnn_group_norm_workspace_floats")) return st;
        const Span work{workspace, (long long)needs * 4};
        if (overlap(work, in) || overlap(work, grad) || overlap(work, out)) return fail(PATDNN_EINVAL, "workspace overlaps input or output");
        const long long channels = 4ll * s.c, statistics = 4ll * s.n * s.groups;
        if (outputs_overlap({in, grad, {mean, statistics}, {rstd, statistics}, {gamma, channels}, {beta, channels}},
                            {out, work, {dgamma, channels}, {dbeta, channels}}))
            return fail(PATDNN_EINVAL, "an output or the workspace overlaps another tensor");
    }
    return done(launch_norm_backward(s, dy, x, mean, rstd, gamma, beta, dx, dgamma, dbeta, workspace, static_cast<hipStream_t>(stream)),
                "launching the group norm's backward pass");
}

// For tests: how a call would be launched (norm_plan_numbers).
patdnn_status_t patdnn_internal_norm_plan(const patdnn_norm_desc_t* desc, int32_t backward, int32_t out[8])
{
    NormShape s{};
    int32_t numbers[8] = {};
    const patdnn_status_t st = norm_shape(desc, backward != 0, s);
    if (st == PATDNN_OK) norm_plan_numbers(s, backward != 0, numbers);
    for (int i = 0; i < 8; ++i) out[i] = numbers[i];
    return st;
}

patdnn_status_t patdnn_mxfp4_quantize(const void* x, int32_t type, int32_t rows, int32_t cols, int64_t row, uint8_t* codes, uint8_t* scales,
                                      void* stream)
{
    return convert(true, const_cast<void*>(x), type, rows, cols, row, codes, scales, stream);
}

patdnn_status_t patdnn_mxfp4_dequantize(const uint8_t* codes, const uint8_t* scales, int32_t rows, int32_t cols, void* out, int32_t type,
                                        int64_t row, void* stream)
{
    return convert(false, out, type, rows, cols, row, const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), stream);
}

size_t patdnn_mxfp4_linear_workspace_bytes(const patdnn_linear_desc_t* desc)
{
    LinearShape s{};
    const char* why;
    return linear_shape(desc, s, why) && s.rows > 0 && linear_fits(s) ? linear_workspace_bytes(s) : 0;
}

patdnn_status_t patdnn_mxfp4_linear(const patdnn_linear_desc_t* desc, const void* x, const uint8_t* x_scales, const uint8_t* w,
                                    const uint8_t* w_scales, const float* bias, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    LinearShape s{};
    const char* why;
    if (!linear_shape(desc, s, why)) return fail(PATDNN_EINVAL, why);
    if (s.rows == 0) return PATDNN_OK;
    if (!linear_fits(s)) return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    if (!x || !out) return fail(PATDNN_EINVAL, "x / out is NULL");
    if (const patdnn_status_t st = check_codes(w, w_scales)) return st;
    const bool codes = s.x_type == kMxfp4;
    if (codes)
        if (const patdnn_status_t st = check_codes(x, x_scales)) return st;
    if ((!codes && !aligned(x, element_bytes(s.x_type))) || !aligned(out, element_bytes(s.out_type)) || !aligned(bias, 4))
        return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    Span in{x, code_bytes(s.rows, s.in)}, to;
    if ((!codes && !span_of(1, 0, s.rows, s.x_row, s.in, s.x_type, x, in)) || !span_of(1, 0, s.rows, s.out_row, s.out, s.out_type, out, to))
        return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    const Span weights{w, code_bytes(s.out, s.in)}, weight_scales{w_scales, code_bytes(s.out, s.in) / 16};
    const Span scales{codes ? x_scales : nullptr, code_bytes(s.rows, s.in) / 16}, b{bias, 4ll * s.out};
    for (const Span& from : {in, weights, weight_scales, scales, b})
        if (overlap(from, to)) return fail(PATDNN_EINVAL, "output overlaps input");
    const size_t needs = linear_workspace_bytes(s);
    if (const patdnn_status_t st = check_workspace(workspace, workspace_bytes, needs, "patdnn_mxfp4_linear_workspace_bytes")) return st;
    if (needs) {
        if (!aligned(workspace, 16)) return fail(PATDNN_EINVAL, "workspace must be 16-byte aligned");
        const Span work{workspace, (long long)needs};
        for (const Span& from : {in, weights, weight_scales, scales, b, to})
            if (overlap(from, work)) return fail(PATDNN_EINVAL, "workspace overlaps input or output");
    }
    return done(launch_linear(s, x, x_scales, w, w_scales, bias, out, workspace, static_cast<hipStream_t>(stream)), "launching the linear layer");
}

}  // extern "C"
