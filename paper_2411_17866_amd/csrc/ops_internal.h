// Shared by the host runtime (ops_runtime.cpp) and the kernels of the
// language-model operators (ortho.hip, linear_ce.hip).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "dsm.h"

namespace dsm {

// ---- Orthogonalised updates (ortho.hip) ----

constexpr int kOrthoGroup = 64;     // matrices that one set of launches takes
constexpr int kOrthoMaxSteps = 32;  // iterations

struct OrthoOffsets {
    int64_t at[kOrthoGroup];  // elements from the buffers' start to each matrix
};

// Power-of-two exponents of one iteration's stored operands: X * 2^x, A * 2^a,
// B * 2^b, and X * 2^x_next after it; an X below 1 grows by less than 2^growth.
struct OrthoScales {
    int x, a, b, x_next, growth;
};

// One group of matrices, all of one shape.  The iteration works on the wide
// orientation: m = min(rows, cols) rows of n = max columns.
struct OrthoGroup {
    int32_t count;
    int32_t m, n;
    int32_t tall;   // the matrix in memory is n x m
    int32_t bf16;   // bf16 buffers, operands as one fp16; else fp32 buffers, two fp16 halves
    int32_t vector;  // rows start where four elements can be moved at once (not for the
                     // transposed stores of a tall matrix)
    int64_t row_stride;
    OrthoOffsets off;
    // Workspace (per matrix strides follow from m and n, see ortho.hip).
    void* workspace;
    // Buffers.  in: the update (orthogonalize) or the gradient (step).
    const void* in;
    void* out;    // orthogonalised update, or the scaled direction; NULL if x is updated
    float* mom;   // momentum, updated; NULL without
    float* x;     // parameters, updated; NULL if out is written
    float mu, lr, scale, weight_decay, eps;
    int32_t nesterov;
};

// Bytes of workspace that a group of `count` m x n matrices needs (0 for matrices
// that are worked on in LDS).
int64_t ortho_group_bytes(int count, int m, int n, bool bf16);

hipError_t launch_ortho(const OrthoGroup& g, const float* coeffs, const OrthoScales* scales, int steps,
                        hipStream_t stream);

// ---- Linear layer with softmax cross entropy (linear_ce.hip) ----

// What the products' operands hold (linear_ce.hip).
enum CeForm { kCeBf16, kCeHalf, kCeHalves, kCeF32 };

// The plan's `scalars`: largest magnitudes, and those of kCeParts work-groups each.
constexpr int kCeParts = 512;
constexpr int64_t kCeScalars = 64 + 8 * kCeParts;

// Where the parts of the workspace lie (bytes from its start), and how the
// vocabulary is cut.
struct CePlan {
    int32_t tokens, dim, vocab;
    CeForm form;
    int32_t grads;
    int32_t tile;        // tokens of a work-group's tile: 32, 64, 128 or 256
    int32_t front;       // losses alone: tile columns of 256 words; tiles of 128 take what follows
    int32_t piece;       // columns of the vocabulary whose gradients are in memory at once
    int32_t dh_splits;   // parts of a piece that dh is summed over side by side
    int32_t sample;      // tile columns of the vocabulary that a row's reference is taken from (0: none)
    int32_t every;       // one of so many tile columns is
    int64_t scalars, coef, lse, hit, stats, tops, refs, rows, h, ht, w, wt, p, dh, bytes;
    int64_t ld_h, ld_w, ld_p;  // 16-bit elements of a row
    int64_t p_lo;              // bf16 form: from G's upper halves to its lower ones
    int64_t ld_dh;             // floats of a row of dh's sums
    int64_t ld_ht;             // with references: of a row of h transposed
    int64_t ld_wt;             // of a row of w transposed (0: there is none)
};

struct CeBuffers {
    const void* h;
    const void* w;
    const int64_t* target;
    const float* weight;
    float* total;
    float* loss;
    float* lse;
    void* dh;
    void* dw;
    int64_t h_stride, w_stride, dh_stride, dw_stride;
    char* workspace;
    int32_t mean;
    int32_t w_direct;  // w is read where it lies
    int32_t h_direct;  // and h
    // Rows whose elements can be moved by four.
    int32_t h_vector, w_vector, dh_vector, dw_vector;
};

hipError_t launch_linear_ce(const CePlan& plan, const CeBuffers& buf, hipStream_t stream);

}  // namespace dsm
