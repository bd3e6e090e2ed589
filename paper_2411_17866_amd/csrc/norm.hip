// The norms before and after a block, fused with its gate and residual scale, and
// their gradients, on gfx950.
//
//   p = post(f);  s = h + scale gate p;  y = norm(s)
//   a norm of a row v:  "layer"  (v - mean) r weight + bias,  r = 1 / sqrt(var + eps)
//                       "rms"    v r weight + bias,           r = 1 / sqrt(mean of v^2 + eps)
//
// Backward, with v^ = (v - mean) r (or v r) and e = dy weight:
//   dh = d = ds + r (e - v^ mean(e v^) [- mean(e)])
//   the same formula takes g = scale gate d post_weight back through post, to df;
//   the vectors' gradients are sums over the tokens.
// Statistics are computed anew from s and f, which have to be read anyway: they are in
// registers, and nothing but s is kept from the forward pass.
//
// Everything is bound by memory: each tensor is read or written once.  A row is worked
// on by L lanes of a wave (several rows a wave) or by W waves, with 8 columns a lane
// in registers; sums over it go by turns of lanes and one exchange through LDS.
// Variances are those of v - mean, not differences of sums.  In the backward kernel a
// lane keeps its columns of the vectors' gradients in registers over all of its
// work-group's rows; the work-groups' sums are joined by a second launch, in a fixed
// order.  Few registers and many waves hide the rows' latency better than rows ahead
// of their turn: two rows at a time, or loads of the next ones, took 8192 x 1600 in fp32
// from 74 us to 103, 85 and with both 135 us.
#include "block_internal.h"
#include "elements.h"

#pragma clang fp contract(off)

namespace dsm {
namespace {

using rows::V8;

// Who works on a row: L lanes, or all 64 of W waves, with 8 columns each.
template <int W_, int L_>
struct Team {
    static constexpr int W = W_, L = L_;
    static constexpr int kRows = 64 / L;  // of a work-group at a time
    static constexpr int kFloats = 2 * 4 * W;
    static_assert(L == 64 || W == 1, "parts of a wave");

    float* lds;
    int turn, col, have;  // this lane's columns: 8 from col on, of which `have` exist
    int row;              // of the work-group's rows
    int back;             // where a row ends among them: how far before col eight columns are whole
    bool ragged;          // there are such lanes

    __device__ __forceinline__ Team(float* lds_, int dim) : lds(lds_), turn(0) {
        col = (static_cast<int>(threadIdx.x) % (W * L)) * 8;
        row = W == 1 ? static_cast<int>(threadIdx.x) / L : 0;
        have = max(0, min(dim - col, 8));
        ragged = dim % 8 != 0;
        // (Columns of another wave may be written in place before they are read here.)
        back = have > 0 && have < 8 && col > 0 && (threadIdx.x & 63) != 0 ? 8 - have : 0;
    }
    // Eight columns, on their way: a row's end takes the eight before it and moves them to
    // their places when they are there (taken one by one they would be waited for at once).
    template <bool F32>
    __device__ __forceinline__ rows::Raw8<F32> raw(const void* base, int64_t r, int64_t stride, bool there = true) const {
        return rows::raw8<F32>(base, r * stride + col - back, there ? have + back : 0);
    }
    template <bool F32>
    __device__ __forceinline__ V8 wide(const rows::Raw8<F32>& x) const {
        V8 v = rows::wide8(x);
        if (ragged) rows::shift(v, back);
        return v;
    }
    // Sums over the row; two buffers of LDS take turns.
    template <int K>
    __device__ __forceinline__ void sum(float (&x)[K]) {
        static_assert(K <= 4, "a buffer's sums");
        if constexpr (L < 64) {
#pragma unroll
            for (int k = 0; k < K; ++k) x[k] = rows::lanes_sum<L>(x[k]);
        } else {
            rows::group_sums<W, K>(x, lds + turn * 4 * W);
            turn ^= 1;
        }
    }
    // A vector, or `otherwise`; columns past the row count as 0 in every sum.
    __device__ __forceinline__ rows::Raw8<true> vector(const float* p) const {
        return p ? raw<true>(p, 0, 0) : rows::Raw8<true>{};
    }
    __device__ __forceinline__ V8 vector(const float* p, const rows::Raw8<true>& x, float otherwise) const {
        if (p) return wide(x);
        V8 v;
#pragma unroll
        for (int q = 0; q < 8; ++q) v.v[q] = q < have ? otherwise : 0.f;
        return v;
    }
    __device__ __forceinline__ float total(const V8& v) const {
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) s += v.v[q];
        return s;
    }
    __device__ __forceinline__ float squares(const V8& v) const {
        float s = 0.f;
#pragma unroll
        for (int q = 0; q < 8; ++q) s = __builtin_fmaf(v.v[q], v.v[q], s);
        return s;
    }
    __device__ __forceinline__ void subtract(V8& v, float mean) const {
#pragma unroll
        for (int q = 0; q < 8; ++q) v.v[q] = q < have ? v.v[q] - mean : 0.f;
    }
    template <bool F32>
    __device__ __forceinline__ void store(const V8& v, void* base, int64_t r, int64_t stride, bool there) const {
        rows::store8<F32>(base, r * stride + col, v, there ? have : 0);
    }
};

// A row standardised in place.
template <class T>
__device__ __forceinline__ void standardise(T& t, V8& v, bool layer, float eps, float dim) {
    if (layer) {
        float s[1] = {t.total(v)};
        t.sum(s);
        t.subtract(v, s[0] / dim);
    }
    float s[1] = {t.squares(v)};
    t.sum(s);
    const float r = 1.0f / sqrtf(s[0] / dim + eps);
#pragma unroll
    for (int q = 0; q < 8; ++q) v.v[q] *= r;
}

// 8192 rows of 1600 in bf16 onto the residual, layer: 20.4 us, 5.1 TB/s.
template <bool F32, class T>
__global__ __launch_bounds__(T::W * 64) void k_norm(NormCall p) {
    __shared__ float lds[T::kFloats];
    T t(lds, p.dim);
    const float dim = static_cast<float>(p.dim);
    const auto raw_weight = t.vector(p.weight), raw_bias = t.vector(p.bias), raw_gate = t.vector(p.gate);
    const auto raw_post_weight = t.vector(p.post_weight), raw_post_bias = t.vector(p.post_bias);
    // The first row is on its way before the vectors are there.
    rows::Raw8<F32> h{}, x{};
    const auto load = [&](int64_t row) {
        h = t.template raw<F32>(p.h, row, p.h_stride, row < p.tokens);
        if (p.f) x = t.template raw<F32>(p.f, row, p.f_stride, row < p.tokens);
    };
    load(static_cast<int64_t>(blockIdx.x) * T::kRows + t.row);
    const V8 weight = t.vector(p.weight, raw_weight, 1.f), bias = t.vector(p.bias, raw_bias, 0.f);
    const V8 post_weight = t.vector(p.post_weight, raw_post_weight, 1.f), post_bias = t.vector(p.post_bias, raw_post_bias, 0.f);
    V8 share = t.vector(p.gate, raw_gate, 1.f);
#pragma unroll
    for (int q = 0; q < 8; ++q) share.v[q] *= p.scale;
    const int64_t step = static_cast<int64_t>(gridDim.x) * T::kRows;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * T::kRows; first < p.tokens; first += step) {
        const int64_t row = first + t.row;
        const bool there = row < p.tokens;
        V8 v = t.wide(h), f;
        if (p.f) {
            f = t.wide(x);
            if (p.post != DSM_NORM_NONE) {
                standardise(t, f, p.post == DSM_NORM_LAYER, p.post_eps, dim);
#pragma unroll
                for (int q = 0; q < 8; ++q) f.v[q] = __builtin_fmaf(f.v[q], post_weight.v[q], post_bias.v[q]);
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) v.v[q] = __builtin_fmaf(f.v[q], share.v[q], v.v[q]);
            if (p.s) t.template store<F32>(v, p.s, row, p.s_stride, there);
        }
        load(row + step);
        if (p.norm == DSM_NORM_NONE) continue;
        standardise(t, v, p.norm == DSM_NORM_LAYER, p.eps, dim);
#pragma unroll
        for (int q = 0; q < 8; ++q) v.v[q] = __builtin_fmaf(v.v[q], weight.v[q], bias.v[q]);
        t.template store<F32>(v, p.y, row, p.y_stride, there);
    }
}

// Sums that need each other's results go by one exchange each:
//   means of v and f (layer);  (v - mean)^2, e (v - mean), e and f's squares;  g f^ and g.
// 8192 rows of 1600 in bf16, rms on both sides with a gate: 39 us, 4.0 TB/s, and 5 for the sums;
// the exchanges' latency and 45 instructions an element are what is above memory's 34.
template <bool F32, class T, bool POST>
__global__ __launch_bounds__(T::W * 64) void k_norm_backward(NormCall p) {
    __shared__ float lds[T::kFloats];
    T t(lds, p.dim);
    const float dim = static_cast<float>(p.dim);
    const bool normed = p.norm != DSM_NORM_NONE, layer = p.norm == DSM_NORM_LAYER, post_layer = POST && p.post == DSM_NORM_LAYER;
    const bool branch = p.df || p.sums[2] || p.sums[3] || p.sums[4];
    const bool reads_f = branch && p.f;
    // Sixteen waves have 128 registers each: there the vectors are read again for every row.
    constexpr bool kKept = !(T::W == 16 && POST);
    V8 weight, gate, post_weight, post_bias, sums[kNormSums];
    if (kKept) {
        const auto raw_weight = t.vector(p.weight), raw_gate = t.vector(p.gate);
        const auto raw_post_weight = POST ? t.vector(p.post_weight) : rows::Raw8<true>{};
        const auto raw_post_bias = POST ? t.vector(p.post_bias) : rows::Raw8<true>{};
        weight = t.vector(p.weight, raw_weight, 1.f);
        gate = t.vector(p.gate, raw_gate, 1.f);
        if (POST) {
            post_weight = t.vector(p.post_weight, raw_post_weight, 1.f);
            post_bias = t.vector(p.post_bias, raw_post_bias, 0.f);
        }
    }
#pragma unroll
    for (int s = 0; s < kNormSums; ++s)
#pragma unroll
        for (int q = 0; q < 8; ++q) sums[s].v[q] = 0.f;
    const int64_t step = static_cast<int64_t>(gridDim.x) * T::kRows;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * T::kRows; first < p.tokens; first += step) {
        const int64_t row = first + t.row;
        const bool there = row < p.tokens;
        rows::Raw8<F32> raw_d{}, raw_v{}, raw_ds{}, raw_f{};
        if (normed) {
            raw_d = t.template raw<F32>(p.dy, row, p.dy_stride, there);
            raw_v = t.template raw<F32>(p.h, row, p.h_stride, there);
        }
        if (p.ds) raw_ds = t.template raw<F32>(p.ds, row, p.ds_stride, there);
        if (reads_f) raw_f = t.template raw<F32>(p.f, row, p.f_stride, there);
        V8 d = t.wide(raw_d), v = t.wide(raw_v), f = t.wide(raw_f);
        const V8 ds = t.wide(raw_ds);
        if (layer || post_layer) {
            float s[2] = {layer ? t.total(v) : 0.f, post_layer ? t.total(f) : 0.f};
            t.sum(s);
            if (layer) t.subtract(v, s[0] / dim);
            if (post_layer) t.subtract(f, s[1] / dim);
        }
        float post_r = 0.f;
        if (normed || POST) {
            float s[4] = {0.f, 0.f, 0.f, POST ? t.squares(f) : 0.f};
            if (!kKept) weight = t.vector(p.weight, t.vector(p.weight), 1.f);
            if (normed) {
                s[0] = t.squares(v);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float e = d.v[q] * weight.v[q];
                    s[1] = __builtin_fmaf(e, v.v[q], s[1]);
                    s[2] += e;
                }
            }
            t.sum(s);
            // (0 for a row that is not there, which has no statistics.)
            const float r = there ? 1.0f / sqrtf(s[0] / dim + p.eps) : 0.f;
            post_r = there ? 1.0f / sqrtf(s[3] / dim + p.post_eps) : 0.f;
            if (normed) {
                const float along = s[1] * r / dim, mean = layer ? s[2] / dim : 0.f;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float dy = d.v[q], hat = v.v[q] * r;
                    sums[0].v[q] = __builtin_fmaf(dy, hat, sums[0].v[q]);
                    sums[1].v[q] += dy;
                    d.v[q] = r * __builtin_fmaf(-hat, along, __builtin_fmaf(dy, weight.v[q], -mean));
                    if (p.ds) d.v[q] += ds.v[q];
                }
            }
        }
        if (!normed) d = ds;
        if (p.dh) t.template store<F32>(d, p.dh, row, p.dh_stride, there);
        if (!branch) continue;
        if (!kKept) {
            const auto raw_gate = t.vector(p.gate), raw_post_weight = t.vector(p.post_weight), raw_post_bias = t.vector(p.post_bias);
            gate = t.vector(p.gate, raw_gate, 1.f);
            post_weight = t.vector(p.post_weight, raw_post_weight, 1.f);
            post_bias = t.vector(p.post_bias, raw_post_bias, 0.f);
        }
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            // (Columns past the row: gate is 0 there.)
            const float sd = p.scale * d.v[q], dp = sd * gate.v[q];
            d.v[q] = dp;
            if constexpr (POST) {
                const float hat = f.v[q] * post_r, g = dp * post_weight.v[q];
                f.v[q] = hat;
                const float value = __builtin_fmaf(hat, post_weight.v[q], post_bias.v[q]);
                sums[2].v[q] = __builtin_fmaf(sd, value, sums[2].v[q]);
                sums[3].v[q] = __builtin_fmaf(dp, hat, sums[3].v[q]);
                sums[4].v[q] += dp;
                d.v[q] = g;
                s[0] = __builtin_fmaf(g, hat, s[0]);
                s[1] += g;
            } else if (reads_f) {
                sums[2].v[q] = __builtin_fmaf(sd, f.v[q], sums[2].v[q]);
            }
        }
        if (!p.df) continue;
        if constexpr (POST) {
            t.sum(s);
            const float along = s[0] / dim, mean = post_layer ? s[1] / dim : 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) d.v[q] = post_r * __builtin_fmaf(-f.v[q], along, d.v[q] - mean);
        }
        t.template store<F32>(d, p.df, row, p.df_stride, there);
    }
#pragma unroll
    for (int s = 0; s < kNormSums; ++s) {
        if (!p.sums[s]) continue;
        if constexpr (T::L < 64) {  // the wave's rows
#pragma unroll
            for (int q = 0; q < 8; ++q)
#pragma unroll
                for (int w = T::L; w < 64; w *= 2) sums[s].v[q] += __shfl_xor(sums[s].v[q], w);
        }
        t.template store<true>(sums[s], p.parts + static_cast<int64_t>(s) * p.groups * p.dim, blockIdx.x, p.dim, t.row == 0);
    }
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

template <class T>
struct Type {
    using type = T;
};
// The team for a row's columns: use(team as a type).
template <class F>
void with_team(int64_t dim, F use) {
    if (dim <= 64)
        use(Type<Team<1, 8>>());
    else if (dim <= 128)
        use(Type<Team<1, 16>>());
    else if (dim <= 256)
        use(Type<Team<1, 32>>());
    else if (dim <= 512)
        use(Type<Team<1, 64>>());
    else if (dim <= 1024)
        use(Type<Team<2, 64>>());
    else if (dim <= 2048)
        use(Type<Team<4, 64>>());
    else if (dim <= 4096)
        use(Type<Team<8, 64>>());
    else
        use(Type<Team<16, 64>>());
}

// Work-groups for `tokens` rows, of `waves` a CU at most.
template <class T>
int groups_for(int64_t tokens, int64_t waves) {
    const int64_t turns = (tokens + T::kRows - 1) / T::kRows, most = waves * 256 / T::W;
    return static_cast<int>(turns < most ? turns : most);
}
constexpr int64_t kForwardWaves = 64;
// As many as a CU holds at once, whole work-groups of them.  8192 x 1600 in bf16 with post: 47 us by 12
// waves a CU, 55 by 8, 58 by 16; 4096 x 2500 in fp32: 68 by 8, 84 by 12; 2048 x 5000 in bf16: 70 by 16, 81 by 12.
template <class T>
constexpr int64_t kBackwardWaves = T::W == 16 ? 16 : T::W == 8 ? 8 : 12;

}  // namespace

int norm_groups(int64_t tokens, int64_t dim) {
    int groups = 0;
    with_team(dim, [&](auto team) {
        using T = typename decltype(team)::type;
        // A row takes a work-group 2 us, and each work-group's sums are written and read: 333 x 1001 in fp32
        // 15.6 us by a row each, 13.9 by two, 17.9 by four; 64 x 1001 10.2, 11.4 and 15.6.
        const int most = groups_for<T>(tokens, kBackwardWaves<T>), pairs = groups_for<T>((tokens + 1) / 2, kBackwardWaves<T>);
        groups = most <= 160 ? most : pairs > 160 ? pairs : 160;
    });
    return groups;
}

hipError_t launch_norm(const NormCall& c, hipStream_t stream) {
    with_team(c.dim, [&](auto team) {
        using T = typename decltype(team)::type;
        const int groups = groups_for<T>(c.tokens, kForwardWaves);
        if (c.f32)
            k_norm<true, T><<<groups, T::W * 64, 0, stream>>>(c);
        else
            k_norm<false, T><<<groups, T::W * 64, 0, stream>>>(c);
    });
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormCall& c, hipStream_t stream) {
    with_team(c.dim, [&](auto team) {
        using T = typename decltype(team)::type;
        if (c.groups == 0) return;
        // (f is not read where nothing of post is wanted.)
        const bool post = c.post != DSM_NORM_NONE && c.f;
        if (c.f32 && post)
            k_norm_backward<true, T, true><<<c.groups, T::W * 64, 0, stream>>>(c);
        else if (c.f32)
            k_norm_backward<true, T, false><<<c.groups, T::W * 64, 0, stream>>>(c);
        else if (post)
            k_norm_backward<false, T, true><<<c.groups, T::W * 64, 0, stream>>>(c);
        else
            k_norm_backward<false, T, false><<<c.groups, T::W * 64, 0, stream>>>(c);
    });
    bool any = false;
    for (float* s : c.sums) any = any || s != nullptr;
    if (any) k_norm_sums<<<dim3((c.dim + 63) / 64, kNormSums), 1024, 0, stream>>>(c);
    return hipGetLastError();
}

}  // namespace dsm
