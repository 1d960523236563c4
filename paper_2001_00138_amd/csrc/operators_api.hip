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

static_assert(PATDNN_F32 == kF32 && PATDNN_F16 == kF16 && PATDNN_BF16 == kBF16 && PATDNN_MXFP4 == kMxfp4 && PATDNN_FP8 == kFp8,
              "one numbering");
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

// ---- the feed-forward block in fp8 ----

// Spans of a stored matrix: codes in whole pieces of 128, scales a row or 128 rows.
Span fp8_codes(const void* p, long long rows, long long cols) { return Span{p, rows * fp8_pieces(cols) * 128}; }
Span fp8_scales(const void* p, long long rows, long long cols, bool squares) { return Span{p, fp8_scale_rows(rows, squares) * fp8_pieces(cols)}; }

patdnn_status_t fp8_convert(bool quantize, void* values, int32_t type, int32_t rows, int32_t cols, int64_t row, int32_t blocks, bool transposed,
                            uint8_t* codes, uint8_t* scales, void* stream)
{
    if (!real_type(type)) return fail(PATDNN_EINVAL, "unknown element type");
    if (rows < 0 || cols <= 0) return fail(PATDNN_EINVAL, "rows must be >= 0 and cols positive");
    if (blocks != PATDNN_FP8_ROWS && blocks != PATDNN_FP8_SQUARES) return fail(PATDNN_EINVAL, "unknown blocks");
    if (row < 0 || (!quantize && rows > 1 && row < cols)) return fail(PATDNN_EINVAL, "strides must be >= 0, and output rows must not overlap");
    if (rows == 0) return PATDNN_OK;
    if (!values) return fail(PATDNN_EINVAL, "x / out is NULL");
    if (!codes || !scales) return fail(PATDNN_EINVAL, "codes / scales is NULL");
    if (!aligned(codes, 16)) return fail(PATDNN_EINVAL, "codes must be 16-byte aligned");
    if (!aligned(values, element_bytes(type))) return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    // the matrix as it is stored
    const Fp8Shape s{transposed ? cols : rows, transposed ? rows : cols, type, blocks == PATDNN_FP8_SQUARES, transposed, row};
    Span a;
    if (!fp8_fits(s, quantize) || !span_of(1, 0, rows, row, cols, type, values, a)) return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    const Span b = fp8_codes(codes, s.rows, s.cols), c = fp8_scales(scales, s.rows, s.cols, s.squares);
    if (overlap(a, b) || overlap(a, c) || (quantize && overlap(b, c))) return fail(PATDNN_EINVAL, "output overlaps input");
    return quantize ? done(launch_fp8_quantize(s, values, codes, scales, static_cast<hipStream_t>(stream)), "launching the quantisation")
                    : done(launch_fp8_dequantize(s, codes, scales, values, static_cast<hipStream_t>(stream)), "launching the dequantisation");
}

patdnn_status_t rms_shape(const patdnn_rms_desc_t* d, bool backward, RmsShape& s)
{
    if (!d) return fail(PATDNN_EINVAL, "desc is NULL");
    if (d->rows < 0 || d->cols <= 0) return fail(PATDNN_EINVAL, "rows must be >= 0 and cols positive");
    if (!real_type(d->type) || !(real_type(d->y_type) || (!backward && d->y_type == kFp8))) return fail(PATDNN_EINVAL, "unknown element type");
    if (!backward && !(d->eps >= 0.0f && std::isfinite(d->eps))) return fail(PATDNN_EINVAL, "eps must be finite and >= 0");
    const bool codes = d->y_type == kFp8;
    if (d->x_row < 0 || d->residual_row < 0 || d->sum_row < 0 || (!codes && d->y_row < 0)) return fail(PATDNN_EINVAL, "strides must be >= 0");
    s = RmsShape{d->rows, d->cols, d->type, d->y_type, d->eps, d->x_row, d->residual_row, d->sum_row, codes ? 0 : d->y_row};
    if (!rms_fits(s, backward)) return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    return PATDNN_OK;
}
bool rows_of(const RmsShape& s, const void* p, long long row, int type, Span& span) { return span_of(1, 0, s.rows, row, s.cols, type, p, span); }
// An output may be the very tensor that an input is.
bool same_rows(const RmsShape& s, const void* a, long long a_row, const void* b, long long b_row) { return a && a == b && (s.rows == 1 || a_row == b_row); }

patdnn_status_t product_shape(const patdnn_fp8_desc_t* d, int kind, ProductShape& s)
{
    if (!d) return fail(PATDNN_EINVAL, "desc is NULL");
    if (d->rows < 0 || d->in_features <= 0 || d->out_features <= 0)
        return fail(PATDNN_EINVAL, "rows must be >= 0 and in_features, out_features positive");
    if (d->w_blocks != PATDNN_FP8_ROWS && d->w_blocks != PATDNN_FP8_SQUARES) return fail(PATDNN_EINVAL, "unknown blocks");
    const bool codes = kind == kGated && d->out_type == kFp8, backward = kind == kGatedBackward;
    if (!(real_type(d->out_type) || codes) || (backward && !real_type(d->dh_type))) return fail(PATDNN_EINVAL, "unknown element type");
    if (d->act < kActNone || d->act > kActSilu) return fail(PATDNN_EINVAL, "unknown activation");
    if ((!codes && (d->out_row < 0 || (d->rows > 1 && d->out_row < d->out_features))) || (backward && d->dh_row < 0))
        return fail(PATDNN_EINVAL, "strides must be >= 0, and output rows must not overlap");
    s = ProductShape{kind, d->rows, d->in_features, d->out_features, d->w_blocks == PATDNN_FP8_SQUARES, d->out_type, d->act, backward ? d->dh_type : 0,
                     codes ? 0 : d->out_row, backward ? d->dh_row : 0};
    if (s.rows && !product_fits(s)) return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    return PATDNN_OK;
}
size_t product_workspace(const patdnn_fp8_desc_t* d, int kind)
{
    ProductShape s{};
    return product_shape(d, kind, s) == PATDNN_OK && s.rows ? product_workspace_bytes(s) : 0;
}

patdnn_status_t product(const patdnn_fp8_desc_t* d, int kind, const ProductTensors& t, void* workspace, size_t workspace_bytes, const char* sizes,
                        void* stream)
{
    ProductShape s{};
    if (const patdnn_status_t st = product_shape(d, kind, s)) return st;
    if (s.rows == 0) return PATDNN_OK;
    const bool two = kind != kLinear, backward = kind == kGatedBackward, codes = s.out_type == kFp8;
    if (!t.x || !t.x_scales || !t.w || !t.w_scales || (two && (!t.w2 || !t.w2_scales))) return fail(PATDNN_EINVAL, "codes / scales is NULL");
    if (!t.out || (backward && (!t.out2 || !t.dh)) || (codes && !t.out_scales)) return fail(PATDNN_EINVAL, "an output, or dh, is NULL");
    if (!aligned(t.x, 16) || !aligned(t.w, 16) || !aligned(t.w2, 16) || (codes && !aligned(t.out, 16))) return fail(PATDNN_EINVAL, "codes must be 16-byte aligned");
    const size_t element = element_bytes(s.out_type);
    if ((!codes && !aligned(t.out, element)) || (backward && (!aligned(t.out2, element) || !aligned(t.dh, element_bytes(s.dh_type)))) || !aligned(t.bias, 4))
        return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    Span out{}, out2{}, dh{};
    if (codes) out = fp8_codes(t.out, s.rows, s.out);
    else if (!span_of(1, 0, s.rows, s.out_row, s.out, s.out_type, t.out, out)) return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    if (backward && (!span_of(1, 0, s.rows, s.out_row, s.out, s.out_type, t.out2, out2) || !span_of(1, 0, s.rows, s.dh_row, s.out, s.dh_type, t.dh, dh)))
        return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    const size_t needs = product_workspace_bytes(s);
    if (const patdnn_status_t st = check_workspace(workspace, workspace_bytes, needs, sizes)) return st;
    if (needs && !aligned(workspace, 16)) return fail(PATDNN_EINVAL, "workspace must be 16-byte aligned");
    const Span work{needs ? workspace : nullptr, (long long)needs};
    if (outputs_overlap({fp8_codes(t.x, s.rows, s.in), fp8_scales(t.x_scales, s.rows, s.in, false), fp8_codes(t.w, s.out, s.in),
                         fp8_scales(t.w_scales, s.out, s.in, s.squares), fp8_codes(two ? t.w2 : nullptr, s.out, s.in),
                         fp8_scales(two ? t.w2_scales : nullptr, s.out, s.in, s.squares), {t.bias, 4ll * s.out}, dh},
                        {out, out2, {codes ? t.out_scales : nullptr, (long long)s.rows * fp8_pieces(s.out)}, work}))
        return fail(PATDNN_EINVAL, "an output or the workspace overlaps another tensor");
    return done(launch_product(s, t, workspace, static_cast<hipStream_t>(stream)), "launching the product");
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

patdnn_status_t patdnn_fp8_quantize(const void* x, int32_t type, int32_t rows, int32_t cols, int64_t row, int32_t blocks, int32_t transposed,
                                    uint8_t* codes, uint8_t* scales, void* stream)
{
    return fp8_convert(true, const_cast<void*>(x), type, rows, cols, row, blocks, transposed != 0, codes, scales, stream);
}

patdnn_status_t patdnn_fp8_dequantize(const uint8_t* codes, const uint8_t* scales, int32_t rows, int32_t cols, int32_t blocks, void* out, int32_t type,
                                      int64_t row, void* stream)
{
    return fp8_convert(false, out, type, rows, cols, row, blocks, false, const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), stream);
}

size_t patdnn_rms_norm_workspace_floats(const patdnn_rms_desc_t* desc)
{
    RmsShape s{};
    return rms_shape(desc, true, s) == PATDNN_OK ? rms_workspace_floats(s) : 0;
}

patdnn_status_t patdnn_rms_norm(const patdnn_rms_desc_t* desc, const void* x, const void* residual, const float* gamma, void* sum, void* y,
                                uint8_t* y_scales, float* rstd, void* stream)
{
    RmsShape s{};
    if (const patdnn_status_t st = rms_shape(desc, false, s)) return st;
    const bool codes = s.y_type == kFp8;
    if (s.rows > 1 && ((sum && s.sum_row < s.cols) || (!codes && s.y_row < s.cols))) return fail(PATDNN_EINVAL, "output rows must not overlap");
    if (s.rows == 0) return PATDNN_OK;
    if (!x || !y || (codes && !y_scales)) return fail(PATDNN_EINVAL, "x / y / y_scales is NULL");
    const size_t element = element_bytes(s.type);
    if (codes && !aligned(y, 16)) return fail(PATDNN_EINVAL, "codes must be 16-byte aligned");
    if (!aligned(x, element) || !aligned(residual, element) || !aligned(sum, element) || (!codes && !aligned(y, element_bytes(s.y_type))) ||
        !aligned(gamma, 4) || !aligned(rstd, 4))
        return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    Span in, add, total, out = fp8_codes(y, s.rows, s.cols);
    if (!rows_of(s, x, s.x_row, s.type, in) || !rows_of(s, residual, s.residual_row, s.type, add) || !rows_of(s, sum, s.sum_row, s.type, total) ||
        (!codes && !rows_of(s, y, s.y_row, s.y_type, out)))
        return fail(PATDNN_EUNSUPPORTED, "tensor too large");
    if (same_rows(s, sum, s.sum_row, residual, s.residual_row)) add.p = nullptr;
    if (outputs_overlap({in, add, {gamma, 4ll * s.cols}},
                        {total, out, {codes ? y_scales : nullptr, (long long)s.rows * fp8_pieces(s.cols)}, {rstd, 4ll * s.rows}}))
        return fail(PATDNN_EINVAL, "an output overlaps another tensor");
    return done(launch_rms(s, x, residual, gamma, sum, y, y_scales, rstd, static_cast<hipStream_t>(stream)), "launching the root-mean-square norm");
}

patdnn_status_t patdnn_rms_norm_backward(const patdnn_rms_desc_t* desc, const void* dy, const void* dsum, const void* x, const float* rstd,
                                         const float* gamma, void* dx, float* dgamma, float* workspace, size_t workspace_floats, void* stream)
{
    RmsShape s{};
    if (const patdnn_status_t st = rms_shape(desc, true, s)) return st;
    if (s.rows > 1 && s.sum_row < s.cols) return fail(PATDNN_EINVAL, "output rows must not overlap");
    if (!aligned(dgamma, 4)) return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
    if (s.rows > 0) {
        if (!dy || !x || !rstd || !dx) return fail(PATDNN_EINVAL, "dy / s / rstd / dx is NULL");
        const size_t element = element_bytes(s.type);
        if (!aligned(dy, element_bytes(s.y_type)) || !aligned(dsum, element) || !aligned(x, element) || !aligned(dx, element) || !aligned(rstd, 4) ||
            !aligned(gamma, 4) || !aligned(workspace, 4))
            return fail(PATDNN_EINVAL, "a tensor is not aligned to its elements");
        Span grad, add, in, out;
        if (!rows_of(s, dy, s.y_row, s.y_type, grad) || !rows_of(s, dsum, s.residual_row, s.type, add) || !rows_of(s, x, s.x_row, s.type, in) ||
            !rows_of(s, dx, s.sum_row, s.type, out))
            return fail(PATDNN_EUNSUPPORTED, "tensor too large");
        const size_t needs = dgamma ? rms_workspace_floats(s) : 0;
        if (const patdnn_status_t st = check_workspace(workspace, workspace_floats, needs, "patdnn_rms_norm_workspace_floats")) return st;
        if (same_rows(s, dx, s.sum_row, dsum, s.residual_row)) add.p = nullptr;
        if (outputs_overlap({grad, add, in, {rstd, 4ll * s.rows}, {gamma, 4ll * s.cols}},
                            {out, {dgamma, 4ll * s.cols}, {needs ? workspace : nullptr, (long long)needs * 4}}))
            return fail(PATDNN_EINVAL, "an output or the workspace overlaps another tensor");
    }
    return done(launch_rms_backward(s, dy, dsum, x, rstd, gamma, dx, dgamma, workspace, static_cast<hipStream_t>(stream)),
                "launching the root-mean-square norm's backward pass");
}

size_t patdnn_fp8_linear_workspace_bytes(const patdnn_fp8_desc_t* desc) { return product_workspace(desc, kLinear); }
size_t patdnn_fp8_gated_workspace_bytes(const patdnn_fp8_desc_t* desc) { return product_workspace(desc, kGated); }
size_t patdnn_fp8_gated_backward_workspace_bytes(const patdnn_fp8_desc_t* desc) { return product_workspace(desc, kGatedBackward); }

patdnn_status_t patdnn_fp8_linear(const patdnn_fp8_desc_t* desc, const uint8_t* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales,
                                  const float* bias, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    return product(desc, kLinear, ProductTensors{x, x_scales, w, w_scales, nullptr, nullptr, bias, nullptr, out, nullptr, nullptr}, workspace,
                   workspace_bytes, "patdnn_fp8_linear_workspace_bytes", stream);
}

patdnn_status_t patdnn_fp8_gated(const patdnn_fp8_desc_t* desc, const uint8_t* x, const uint8_t* x_scales, const uint8_t* gate, const uint8_t* gate_scales,
                                 const uint8_t* up, const uint8_t* up_scales, void* out, uint8_t* out_scales, void* workspace, size_t workspace_bytes,
                                 void* stream)
{
    return product(desc, kGated, ProductTensors{x, x_scales, gate, gate_scales, up, up_scales, nullptr, nullptr, out, nullptr, out_scales}, workspace,
                   workspace_bytes, "patdnn_fp8_gated_workspace_bytes", stream);
}

patdnn_status_t patdnn_fp8_gated_backward(const patdnn_fp8_desc_t* desc, const void* dh, const uint8_t* x, const uint8_t* x_scales, const uint8_t* gate,
                                          const uint8_t* gate_scales, const uint8_t* up, const uint8_t* up_scales, void* dgate, void* dup,
                                          void* workspace, size_t workspace_bytes, void* stream)
{
    return product(desc, kGatedBackward, ProductTensors{x, x_scales, gate, gate_scales, up, up_scales, nullptr, dh, dgate, dup, nullptr}, workspace,
                   workspace_bytes, "patdnn_fp8_gated_backward_workspace_bytes", stream);
}

}  // extern "C"
