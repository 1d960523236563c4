// Launchers of the operators around the pruned convolutions: order of channels, group norm, MXFP4, and the feed-forward block in fp8.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "element.hpp"

namespace patdnn {

// Most workgroups of 256 threads that one launch may have (a grid has fewer than 2^32 threads).
constexpr long long kMostBlocks = (1ll << 24) - 1;

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// ---- order of channels (kernel_reorder.hip) ----
// out[b][j][i] = in[b][i][j]: `rows` x `cols` of each of `batch` matrices; strides in elements, columns adjacent.
struct TransposeShape {
    int batch, rows, cols, in_type, out_type;
    long long in_batch, in_row, out_batch, out_row;
};
bool transpose_fits(const TransposeShape& s);
hipError_t launch_transpose(const TransposeShape& s, const void* in, void* out, hipStream_t stream);

// ---- group norm, channels last (kernel_norm.hip) ----
struct NormShape {
    int n, pixels, c, groups, type, act;
    float eps;
    long long x_image, x_pixel, y_image, y_pixel, dy_image, dy_pixel;      // strides in elements
};
constexpr int kMostNormLength = INT32_MAX - 1024;        // pixels, and channels
bool norm_fits(const NormShape& s);
// (the rest only for what fits)
size_t norm_workspace_floats(const NormShape& s, bool backward);
void norm_plan_numbers(const NormShape& s, bool backward, int32_t (&out)[8]);
hipError_t launch_norm(const NormShape& s, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
                       float* workspace, hipStream_t stream);
// y_* of the shape are dx's strides here.
hipError_t launch_norm_backward(const NormShape& s, const void* dy, const void* x, const float* mean, const float* rstd, const float* gamma,
                                const float* beta, void* dx, float* dgamma, float* dbeta, float* workspace, hipStream_t stream);

// ---- MXFP4 (kernel_mxfp4.hip) ----
// Bytes of a row of `cols` values: codes and scales, in whole pieces of 128 values.
inline long long mxfp4_pieces(long long cols) { return (cols + 127) / 128; }
struct Mxfp4Shape {
    int rows, cols, type;
    long long row;                       // elements between rows of the values
};
bool mxfp4_fits(const Mxfp4Shape& s);
hipError_t launch_mxfp4_quantize(const Mxfp4Shape& s, const void* x, uint8_t* codes, uint8_t* scales, hipStream_t stream);
hipError_t launch_mxfp4_dequantize(const Mxfp4Shape& s, const uint8_t* codes, const uint8_t* scales, void* out, hipStream_t stream);

struct LinearShape {
    int rows, in, out, x_type, out_type, act;
    long long x_row, out_row;            // elements between rows of x (unless MXFP4) and out
};
bool linear_fits(const LinearShape& s);
size_t linear_workspace_bytes(const LinearShape& s);
hipError_t launch_linear(const LinearShape& s, const void* x, const uint8_t* x_scales, const uint8_t* w, const uint8_t* w_scales, const float* bias,
                         void* out, void* workspace, hipStream_t stream);

// ---- fp8 (kernel_fp8.hip) ----
// The stored matrix has `rows` x `cols` values; x is it, or (transposed) its transpose, with `row` elements between x's rows.
struct Fp8Shape {
    int rows, cols, type;
    bool squares, transposed;
    long long row;
};
inline long long fp8_pieces(long long cols) { return (cols + 127) / 128; }
// Rows of scales of a stored matrix.
inline long long fp8_scale_rows(long long rows, bool squares) { return squares ? (rows + 127) / 128 : rows; }
bool fp8_fits(const Fp8Shape& s, bool quantize);
hipError_t launch_fp8_quantize(const Fp8Shape& s, const void* x, uint8_t* codes, uint8_t* scales, hipStream_t stream);
hipError_t launch_fp8_dequantize(const Fp8Shape& s, const uint8_t* codes, const uint8_t* scales, void* out, hipStream_t stream);

// ---- root-mean-square norm (kernel_rms.hip) ----
struct RmsShape {
    int rows, cols, type, y_type;        // y_type: of y (kFp8: codes), or of dy
    float eps;
    long long x_row, residual_row, sum_row, y_row;       // backward: of s, dsum, dx, dy
};
bool rms_fits(const RmsShape& s, bool backward);
size_t rms_workspace_floats(const RmsShape& s);          // of the backward call, for a gradient of gamma
hipError_t launch_rms(const RmsShape& s, const void* x, const void* residual, const float* gamma, void* sum, void* y, uint8_t* y_scales,
                      float* rstd, hipStream_t stream);
hipError_t launch_rms_backward(const RmsShape& s, const void* dy, const void* dsum, const void* x, const float* rstd, const float* gamma, void* dx,
                               float* dgamma, float* workspace, hipStream_t stream);

// ---- products of fp8 codes (kernel_fp8_rows.hip, kernel_fp8_tiles.hip) ----
enum { kLinear = 0, kGated = 1, kGatedBackward = 2 };
struct ProductShape {
    int kind;
    int rows, in, out;                   // of x, along the sums, of the weights (of each of the two)
    bool squares;                        // the weights' scales
    int out_type, act, dh_type;
    long long out_row, dh_row;
};
struct ProductTensors {
    const uint8_t *x, *x_scales, *w, *w_scales, *w2, *w2_scales;         // w2: the second projection
    const float* bias;
    const void* dh;
    void *out, *out2;                    // out2: the second projection's gradient
    uint8_t* out_scales;                 // of codes
};
bool product_fits(const ProductShape& s);
size_t product_workspace_bytes(const ProductShape& s);
hipError_t launch_product(const ProductShape& s, const ProductTensors& t, void* workspace, hipStream_t stream);

}  // namespace patdnn
