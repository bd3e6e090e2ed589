// Shared by the host runtime (block_runtime.cpp) and the kernels of the operators
// that a model's blocks and their gradients take (clip.hip, norm.hip, linear.hip).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "dsm.h"

namespace dsm {

// ---- Clipping by the global norm (clip.hip) ----

constexpr int kClipChunk = 16384;  // elements that a work-group takes
constexpr int kClipEntries = 48;   // tensors of a launch
constexpr int kClipGroups = 256;   // groups of a call
constexpr int64_t kClipOnce = int64_t(256) << 20;  // bytes of a call that the last-level cache does not hold
constexpr int kClipFewGroups = 64, kClipFewChunks = 2048;  // of a call whose norms take no launch of their own

struct ClipEntry {
    void* data;
    int64_t first, numel, block, stride;  // as in dsm_clip_tensor
    int32_t chunk;                        // first chunk of the launch
    uint16_t group, bf16;
};
// Part of a call's tensors, passed to the kernels by value.
struct ClipTable {
    ClipEntry e[kClipEntries];
    int32_t count, chunks;
    int64_t slot;  // of the launch's first chunk among the call's
};
// Where each group's chunks start among the call's; by value.
template <class Index, int GROUPS>
struct ClipStarts {
    Index start[GROUPS + 1];
    int32_t count;
    float max_norm, eps;
};
using ClipGroups = ClipStarts<int64_t, kClipGroups>;
using ClipFew = ClipStarts<int32_t, kClipFewGroups>;

// `bytes`: of all the call's tensors.
hipError_t launch_clip_squares(const ClipTable& t, int64_t bytes, double* parts, hipStream_t stream);
hipError_t launch_clip_norms(const ClipGroups& g, const double* parts, float* norm, double* factor, hipStream_t stream);
hipError_t launch_clip_scale(const ClipTable& t, const double* factor, hipStream_t stream);
// The last two in one, where every work-group sums its group's parts itself.
hipError_t launch_clip_rest(const ClipTable& t, const ClipFew& g, const double* parts, float* norm, hipStream_t stream);

// ---- Norms around a block (norm.hip) ----

constexpr int kNormSums = 5;  // weight, bias, gate, post_weight, post_bias
constexpr int kNormMaxDim = 8192;

struct NormCall {
    int32_t tokens, dim, f32;
    int32_t norm, post;  // dsm_norm_kind
    float eps, post_eps, scale;
    const void *h, *f, *dy, *ds;
    const float *weight, *bias, *gate, *post_weight, *post_bias;
    void *s, *y, *dh, *df;
    float* sums[kNormSums];  // dweight, dbias, dgate, dpost_weight, dpost_bias; NULL where not wanted
    int64_t h_stride, f_stride, s_stride, y_stride, dy_stride, ds_stride, dh_stride, df_stride;
    float* parts;     // [kNormSums][groups][dim]
    int32_t groups;   // work-groups of the backward kernel
};

// Work-groups that norm_backward's rows are spread over.
int norm_groups(int64_t tokens, int64_t dim);

hipError_t launch_norm(const NormCall& c, hipStream_t stream);
hipError_t launch_norm_backward(const NormCall& c, hipStream_t stream);

// ---- Linear layer with bias, activation and residual (linear.hip) ----

constexpr int kLinearFew = 64;       // tokens that are answered by one launch without tiles
constexpr int kLinearTopParts = 512; // work-groups that look for w's largest magnitude
constexpr int kDzRows = 64;          // tokens of a work-group that makes dz

enum LinearForm { kLinearBf16, kLinearHalves, kLinearSingle };  // what the products' operands hold (linear.hip)

// How a problem is cut and where the parts of the workspace lie (bytes from its start).
struct LinearPlan {
    int32_t tokens, dim, wide, act;
    int32_t f32, dw_f32;
    int32_t dz_halves;           // dz is two bf16 arrays, for dw
    LinearForm form, back_form;
    int32_t few, back_few;       // no tiles
    int32_t tile, splits;        // forward: tile, and parts that its sums run over side by side
    int32_t front;               // tile columns of 256; tiles of 128 take what follows
    int32_t back_tile, dx_splits, dw_splits;
    int32_t split_rows;          // tokens of a work-group that makes dz as halves
    int32_t bias_parts;          // rows of sums that dbias is joined from
    int64_t ld_dim, ld_wide;     // 16-bit elements of a row of x's and w's copies, of dz
    int64_t pad_tokens;          // rows of dz
    int64_t ld_y, ld_dx;         // floats of a row of the parts of y; of dx and dw
    int64_t x, w, dz;            // operands, where they are not read in place (of few tokens x and w always are)
    int64_t x_exp, w_exp, z_exp; // halves: powers of two of the rows of x, w and dz
    int64_t w_tops, tops;        // halves, backward: largest magnitudes of w by work-group; least exponents of x dz
    int64_t y_parts, dx_parts, dw_parts, bias_sums;
    int64_t forward_bytes, backward_bytes;
};

struct LinearCall {
    LinearPlan p;
    const void *x, *w, *residual, *dy, *z_in;
    const float* bias;
    void *y, *z, *dx, *dw;
    float* dbias;
    int64_t x_stride, w_stride, residual_stride, y_stride, z_stride, dy_stride, dx_stride, dw_stride;
    int32_t x_direct, w_direct, dz_direct;  // read where they lie
    char* workspace;
};

hipError_t launch_linear(const LinearCall& c, hipStream_t stream);
hipError_t launch_linear_backward(const LinearCall& c, hipStream_t stream);

}  // namespace dsm
