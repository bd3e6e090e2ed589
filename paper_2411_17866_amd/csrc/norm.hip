// The norms before and after a block, fused with its gate and residual scale, and
// their gradients, on gfx950.
//
//   p = post(f);  s = h + scale gate p;  y = norm(s)
//   a norm of a row v:  "layer"  (v - mean) r weight + bias,  r = 1 / sqrt(var + eps)
//                       "rms"    v r weight + bias,           r = 1 / sqrt(mean of v^2 + eps)
//
// Backward, with e = dy weight and v' = v - mean (or v):
//   d = ds + r e - v' r^3 mean(e v') [- r mean(e)]      (dh = d)
//   the same formula again takes scale gate d post_weight back through post, to df;
//   the vectors' gradients are sums over the tokens.
// Statistics are computed anew from s and f, which have to be read anyway: they are in
// registers, and nothing but s is kept from the forward pass.
//
// Everything is bound by memory: each tensor is read or written once.  A work-group of
// W waves takes R rows at a time, eight columns a lane in registers, and sums over them
// by turns of lanes and one exchange through LDS; variances are those of v - mean, not
// differences of sums.  In the backward kernel a lane keeps its columns of the
// vectors' gradients in registers over all of its work-group's rows; the work-groups'
// sums are joined by a second launch, in a fixed order.
#include <type_traits>

#include "block_internal.h"
#include "elements.h"

#pragma clang fp contract(off)

namespace dsm {
namespace {

using rows::V8;

// Rows that a work-group takes at a time (sixteen waves have 128 registers).
constexpr int rows_of(int waves) { return waves == 16 ? 1 : 2; }

// This lane's columns: 8 from `col` on, of which `have` exist.
struct Cols {
    int col, have;
};
__device__ __forceinline__ Cols cols_of(int dim) {
    const int c = static_cast<int>(threadIdx.x) * 8;
    return {c, max(0, min(dim - c, 8))};
}

// Columns past the row count as 0 in every sum.
__device__ __forceinline__ V8 vector8(const float* p, const Cols& c, float otherwise) {
    if (p) return rows::load8<true>(p, c.col, c.have);
    V8 v;
#pragma unroll
    for (int q = 0; q < 8; ++q) v.v[q] = q < c.have ? otherwise : 0.f;
    return v;
}

// What a kernel's sums over a row share.
template <int W, int R>
struct Sums {
    static constexpr int kFloats = 4 * R * W;  // two buffers of up to 2 R sums
    float* lds;
    int turn;
    template <int K>
    __device__ __forceinline__ void operator()(float (&x)[K]) {
        static_assert(K <= 2 * R, "a buffer's sums");
        rows::group_sums<W, K>(x, lds + turn * 2 * R * W);
        turn ^= 1;
    }
};

// R rows -> (v - mean) r (layer) or v r, and r; 0 for rows from `count` on and in the
// columns past the row.
template <int W, int R>
__device__ __forceinline__ void standardise(V8 (&v)[R], float (&r)[R], const Cols& c, int count, bool layer, float eps,
                                            float dim, Sums<W, R>& sum) {
    float s[R];
    if (layer) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            s[k] = 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) s[k] += v[k].v[q];
        }
        sum(s);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const float mean = s[k] / dim;
#pragma unroll
            for (int q = 0; q < 8; ++q) v[k].v[q] = q < c.have ? v[k].v[q] - mean : 0.f;
        }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        s[k] = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) s[k] = __builtin_fmaf(v[k].v[q], v[k].v[q], s[k]);
    }
    sum(s);
#pragma unroll
    for (int k = 0; k < R; ++k) {
        r[k] = k < count ? 1.0f / sqrtf(s[k] / dim + eps) : 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[k].v[q] *= r[k];
    }
}

// 8192 rows of 1600 in bf16 onto the residual, layer: 26 us, 4.1 TB/s.
template <bool F32, int W, int R>
__global__ __launch_bounds__(W * 64) void k_norm(NormCall p) {
    __shared__ float lds[Sums<W, R>::kFloats];
    Sums<W, R> sum{lds, 0};
    const float dim = static_cast<float>(p.dim);
    const Cols c = cols_of(p.dim);
    const V8 weight = vector8(p.weight, c, 1.f), bias = vector8(p.bias, c, 0.f);
    const V8 post_weight = vector8(p.post_weight, c, 1.f), post_bias = vector8(p.post_bias, c, 0.f);
    V8 share = vector8(p.gate, c, 1.f);
#pragma unroll
    for (int q = 0; q < 8; ++q) share.v[q] *= p.scale;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * R; row < p.tokens; row += static_cast<int64_t>(gridDim.x) * R) {
        const int count = static_cast<int>(min(static_cast<int64_t>(R), p.tokens - row));
        V8 v[R], f[R];
        float r[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int have = k < count ? c.have : 0;
            v[k] = rows::load8<F32>(p.h, (row + k) * p.h_stride + c.col, have);
            if (p.f) f[k] = rows::load8<F32>(p.f, (row + k) * p.f_stride + c.col, have);
        }
        if (p.f) {
            if (p.post != DSM_NORM_NONE) {
                standardise<W, R>(f, r, c, count, p.post == DSM_NORM_LAYER, p.post_eps, dim, sum);
#pragma unroll
                for (int k = 0; k < R; ++k)
#pragma unroll
                    for (int q = 0; q < 8; ++q) f[k].v[q] = f[k].v[q] * post_weight.v[q] + post_bias.v[q];
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
#pragma unroll
                for (int q = 0; q < 8; ++q) v[k].v[q] += f[k].v[q] * share.v[q];
                if (p.s && k < count) rows::store8<F32>(p.s, (row + k) * p.s_stride + c.col, v[k], c.have);
            }
        }
        if (p.norm == DSM_NORM_NONE) continue;
        standardise<W, R>(v, r, c, count, p.norm == DSM_NORM_LAYER, p.eps, dim, sum);
#pragma unroll
        for (int k = 0; k < R; ++k) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[k].v[q] = v[k].v[q] * weight.v[q] + bias.v[q];
            if (k < count) rows::store8<F32>(p.y, (row + k) * p.y_stride + c.col, v[k], c.have);
        }
    }
}

// d = the gradient of the standardised rows `hat` -> that of the rows.
template <int W, int R>
__device__ __forceinline__ void back(V8 (&d)[R], const V8 (&hat)[R], const float (&r)[R], bool layer, float dim,
                                     Sums<W, R>& sum) {
    float s[2 * R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        s[k] = s[R + k] = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            s[k] = __builtin_fmaf(d[k].v[q], hat[k].v[q], s[k]);
            s[R + k] += d[k].v[q];
        }
    }
    sum(s);
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const float along = s[k] / dim, mean = layer ? s[R + k] / dim : 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) d[k].v[q] = r[k] * (d[k].v[q] - hat[k].v[q] * along - mean);
    }
}

template <bool F32, int W, int R>
__global__ __launch_bounds__(W * 64) void k_norm_backward(NormCall p) {
    __shared__ float lds[Sums<W, R>::kFloats];
    Sums<W, R> sum{lds, 0};
    const float dim = static_cast<float>(p.dim);
    const bool normed = p.norm != DSM_NORM_NONE, posted = p.post != DSM_NORM_NONE;
    const bool branch = p.df || p.sums[2] || p.sums[3] || p.sums[4];
    const bool reads_f = branch && p.f;
    const Cols c = cols_of(p.dim);
    const V8 weight = vector8(p.weight, c, 1.f), gate = vector8(p.gate, c, 1.f);
    const V8 post_weight = vector8(p.post_weight, c, 1.f), post_bias = vector8(p.post_bias, c, 0.f);
    V8 sums[kNormSums];
#pragma unroll
    for (int s = 0; s < kNormSums; ++s)
#pragma unroll
        for (int q = 0; q < 8; ++q) sums[s].v[q] = 0.f;
    // The rows after these are on their way while these are worked on (sixteen waves have
    // no registers for that).
    constexpr bool kAhead = W < 16;
    struct {
        rows::Raw8<F32> dy[R], h[R], ds[R], f[R];
    } next;
    const auto load = [&](int64_t row) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int have = row + k < p.tokens ? c.have : 0;
            if (normed) {
                next.dy[k] = rows::raw8<F32>(p.dy, (row + k) * p.dy_stride + c.col, have);
                next.h[k] = rows::raw8<F32>(p.h, (row + k) * p.h_stride + c.col, have);
            }
            if (p.ds) next.ds[k] = rows::raw8<F32>(p.ds, (row + k) * p.ds_stride + c.col, have);
            if (reads_f) next.f[k] = rows::raw8<F32>(p.f, (row + k) * p.f_stride + c.col, have);
        }
    };
    const int64_t step = static_cast<int64_t>(gridDim.x) * R;
    if (kAhead) load(static_cast<int64_t>(blockIdx.x) * R);
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * R; row < p.tokens; row += step) {
        const int count = static_cast<int>(min(static_cast<int64_t>(R), p.tokens - row));
        V8 d[R], hat[R], f[R], ds[R];
        float r[R];
        if (!kAhead) load(row);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (normed) {
                d[k] = rows::wide8(next.dy[k]);
                hat[k] = rows::wide8(next.h[k]);
            }
            if (p.ds) ds[k] = rows::wide8(next.ds[k]);
            if (reads_f) f[k] = rows::wide8(next.f[k]);
        }
        if (kAhead) load(row + step);
        if (normed) {
            standardise<W, R>(hat, r, c, count, p.norm == DSM_NORM_LAYER, p.eps, dim, sum);
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float dy = d[k].v[q];
                    sums[0].v[q] += dy * hat[k].v[q];
                    sums[1].v[q] += dy;
                    d[k].v[q] = dy * weight.v[q];
                }
            back<W, R>(d, hat, r, p.norm == DSM_NORM_LAYER, dim, sum);
            if (p.ds) {
#pragma unroll
                for (int k = 0; k < R; ++k)
#pragma unroll
                    for (int q = 0; q < 8; ++q) d[k].v[q] += ds[k].v[q];
            }
        } else {
#pragma unroll
            for (int k = 0; k < R; ++k) d[k] = ds[k];
        }
        if (p.dh) {
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (k < count) rows::store8<F32>(p.dh, (row + k) * p.dh_stride + c.col, d[k], c.have);
        }
        if (!branch) continue;
        if (posted) standardise<W, R>(f, r, c, count, p.post == DSM_NORM_LAYER, p.post_eps, dim, sum);
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float sd = p.scale * d[k].v[q], dp = sd * gate.v[q];
                d[k].v[q] = dp;
                if (posted) {
                    sums[2].v[q] += sd * (f[k].v[q] * post_weight.v[q] + post_bias.v[q]);
                    sums[3].v[q] += dp * f[k].v[q];
                    sums[4].v[q] += dp;
                    d[k].v[q] = dp * post_weight.v[q];
                } else if (reads_f) {
                    sums[2].v[q] += sd * f[k].v[q];
                }
            }
        if (!p.df) continue;
        if (posted) back<W, R>(d, f, r, p.post == DSM_NORM_LAYER, dim, sum);
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (k < count) rows::store8<F32>(p.df, (row + k) * p.df_stride + c.col, d[k], c.have);
    }
#pragma unroll
    for (int s = 0; s < kNormSums; ++s)
        if (p.sums[s])
            rows::store8<true>(p.parts + (static_cast<int64_t>(s) * p.groups + blockIdx.x) * p.dim, c.col, sums[s], c.have);
}

// A vector's gradient from the work-groups' sums: 64 columns a work-group, whose 16
// waves take every 16th part each.
__global__ __launch_bounds__(1024) void k_norm_sums(NormCall p) {
    __shared__ float parts[16][64];
    float* out = p.sums[blockIdx.y];
    if (!out) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float s = 0.f;
    if (col < p.dim) {
        const float* at = p.parts + static_cast<int64_t>(blockIdx.y) * p.groups * p.dim + col;
#pragma unroll 8
        for (int g = wave; g < p.groups; g += 16) s += at[static_cast<int64_t>(g) * p.dim];
    }
    parts[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || col >= p.dim) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += parts[w][lane];
    out[col] = s;
}

// Waves of a row: eight columns a lane.
int waves_of(int64_t dim) {
    int w = 1;
    while (w < 16 && w * 512 < dim) w *= 2;
    return w;
}
template <class F>
void with_waves(int dim, F launch) {
    switch (waves_of(dim)) {
        case 1: return launch(std::integral_constant<int, 1>());
        case 2: return launch(std::integral_constant<int, 2>());
        case 4: return launch(std::integral_constant<int, 4>());
        case 8: return launch(std::integral_constant<int, 8>());
        default: return launch(std::integral_constant<int, 16>());
    }
}

}  // namespace

int norm_groups(int64_t tokens, int64_t dim) {
    const int w = waves_of(dim);
    const int64_t most = 2048 / w, turns = (tokens + rows_of(w) - 1) / rows_of(w);
    return static_cast<int>(turns < most ? turns : most);
}

hipError_t launch_norm(const NormCall& c, hipStream_t stream) {
    with_waves(c.dim, [&](auto waves) {
        constexpr int W = decltype(waves)::value, R = rows_of(W);
        const int64_t turns = (static_cast<int64_t>(c.tokens) + R - 1) / R, most = 8192 / W;
        const unsigned groups = static_cast<unsigned>(turns < most ? turns : most);
        if (c.f32)
            k_norm<true, W, R><<<groups, W * 64, 0, stream>>>(c);
        else
            k_norm<false, W, R><<<groups, W * 64, 0, stream>>>(c);
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormCall& c, hipStream_t stream) {
    with_waves(c.dim, [&](auto waves) {
        constexpr int W = decltype(waves)::value, R = rows_of(W);
        if (c.groups > 0) {
            if (c.f32)
                k_norm_backward<true, W, R><<<c.groups, W * 64, 0, stream>>>(c);
            else
                k_norm_backward<false, W, R><<<c.groups, W * 64, 0, stream>>>(c);
        }
    });
    bool any = false;
    for (float* s : c.sums) any = any || s != nullptr;
    if (any) k_norm_sums<<<dim3((c.dim + 63) / 64, kNormSums), 1024, 0, stream>>>(c);
    return hipGetLastError();
}

}  // namespace dsm
