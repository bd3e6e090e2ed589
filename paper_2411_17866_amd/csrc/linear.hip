// The linear layer with bias, activation and residual, and its gradients, on gfx950.
//
//   z = x w^T + bias;  y = act(z) + residual
//   dz = dy act'(z);  dx = dz w;  dw = dz^T x;  dbias = sum over the tokens of dz
//
// Up to kLinearFew tokens the forward pass is bound by reading w once: k_few does it
// without tiles in LDS and without copies, in one launch, or where few rows of w leave
// CUs idle in parts of k that a second one joins.  More tokens go through the tiles of
// gemm_tile.h with bias, activation and residual in their epilogue.  The
// gradients are two products of dz in one launch, dz being made by a pass of its own,
// which also sums dbias; where there is no activation, dy is taken where it lies.
//
// What the products take:
//   bf16  the operands as they are, where rows of 64 columns (k-contiguous) or of 8
//         (k-strided) are whole and aligned, else copies with zeros behind the rows.
//         dz is rounded to bf16: an error of half a step for each term of a sum, which is
//         about what the rounding of a bf16 result costs (0.0024 of its norm with both,
//         0.0017 with one).  A dw in fp32 takes dz as two bf16 halves, 16 bits, with twice
//         the matrix instructions.
//   fp32  two fp16 halves of every number (gemm_tile.h).  Powers of two bring a row's
//         largest magnitude just under fp16's, so rows of any size keep their bits:
//         x's and w's rows forward, dz's for dx.  In dw the sum runs over the tokens,
//         so there x_t is taken times 2^(c - e_t), e_t being dz_t's power: dz_t x_t
//         comes out right up to one power, and c brings the largest of them to fp16's
//         range.  w in dx, whose sum runs over w's rows, has one power for all.
//   fp32 itself, for few tokens, where reading w costs more than multiplying it: w is
//         read where it lies, and the matrix cores multiply fp32 at a 16th of the rate.
// Products accumulate in fp32.
//
// Sums over a long axis with few tiles are cut into parts that run side by side; they
// are joined by a launch that then has the epilogue.
#include <type_traits>

#include "block_internal.h"
#include "elements.h"
#include "gemm_tile.h"

#pragma clang fp contract(off)

namespace dsm {
namespace {

using rows::f4;
using rows::u16;
using rows::u16x8;
using rows::V8;
using tile::kContig;
using tile::kStrided;
using tile::Operand;

template <class T_>
struct Type {
    using type = T_;
};

// What the products' operands hold (the plan's `form`).
constexpr bool is_f32(LinearForm f) { return f != kLinearBf16; }
constexpr tile::Elem elem(LinearForm f) {
    return f == kLinearBf16 ? tile::kBF16 : f == kLinearHalves ? tile::kSplit : tile::kF32;
}
constexpr int units(LinearForm f) { return tile::units(elem(f)); }

constexpr int kNoExponent = 10000;  // of a row of zeros: brings everything to 0

// ---- Activations ----
//
// FAST, for results that are rounded to bf16: the hardware's exp2 and reciprocal
// (2^-22).  The epilogue's arithmetic does not overlap the next tile's products, so
// every instruction of it counts.  (silu and gelu_tanh are 0 where 1 + exp(-v) passes
// fp32's range, or its reciprocal falls below the normal numbers: results under 2^-119.)

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kTanhA = 1.59576912160573071f;  // 2 sqrt(2 / pi): (1 + tanh(u)) / 2 = logistic(2 u)
constexpr float kTanhB = 0.044715f;

template <bool FAST>
__device__ __forceinline__ float one_over(float v) {
    return FAST ? __builtin_amdgcn_rcpf(v) : 1.0f / v;
}
// exp(-v), of the logistic 1 / (1 + exp(-v)).
template <bool FAST>
__device__ __forceinline__ float exp_minus(float v) {
    return FAST ? __builtin_amdgcn_exp2f(v * -kLog2e) : expf(-v);
}

// The normal distribution's share below z, and exp(-z^2 / 2).  FAST: erfc(x) exp(x^2) is
// t Q(t) with t = 1 / (1 + 0.35 x) and Q a polynomial of degree 7, a least-squares fit of
// its relative error in Chebyshev's basis over x in [0, 40] (1.3e-6 in fp32 arithmetic).
template <bool FAST>
__device__ __forceinline__ float normal_share(float z, float* bell) {
    if constexpr (!FAST) {
        *bell = expf(-0.5f * z * z);
        return 0.5f * erfcf(z * -0.707106781186547524f);
    }
    constexpr float kQ[8] = {0.19746625423431396f, 0.1974421590566635f,     0.18609043955802917f, 0.1536107361316681f,
                             0.16591569781303406f, -0.018850743770599365f, 0.20431290566921234f, -0.08598839491605759f};
    *bell = __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2e));
    const float u = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(z), 0.35f * 0.707106781186547524f, 1.0f));
    float q = kQ[7];
#pragma unroll
    for (int k = 6; k >= 0; --k) q = __builtin_fmaf(q, u, kQ[k]);
    const float less = 0.5f * u * q * *bell;
    return z < 0.f ? less : 1.0f - less;
}

template <int ACT, bool FAST>
__device__ __forceinline__ float activation(float z) {
    if constexpr (ACT == DSM_ACT_RELU) {
        return z < 0.f ? 0.f : z;
    } else if constexpr (ACT == DSM_ACT_GELU) {
        float bell;
        return z * normal_share<FAST>(z, &bell);
    } else {
        const float v = ACT == DSM_ACT_SILU ? z : z * __builtin_fmaf(z * z, kTanhA * kTanhB, kTanhA);
        return z * one_over<FAST>(1.0f + exp_minus<FAST>(v));
    }
}

template <int ACT, bool FAST>
__device__ __forceinline__ float slope(float z) {
    if constexpr (ACT == DSM_ACT_RELU) return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
    // (Beyond 200 every slope is 0 or 1 in fp32, and its terms would overflow.)
    const float v = z > 200.f ? 200.f : z < -200.f ? -200.f : z;
    if constexpr (ACT == DSM_ACT_GELU) {
        float bell;
        const float share = normal_share<FAST>(v, &bell);
        return __builtin_fmaf(v * 0.398942280401432678f, bell, share);
    }
    float u = v, rate = 1.f;
    if constexpr (ACT == DSM_ACT_GELU_TANH) {
        const float square = v * v;
        u = v * __builtin_fmaf(square, kTanhA * kTanhB, kTanhA);
        rate = __builtin_fmaf(square, 3.f * kTanhA * kTanhB, kTanhA);
    }
    // With t = exp(-|u|) the logistic of u is 1 / (1 + t) or t / (1 + t), and its slope their product: no
    // difference, no overflow, and the slopes far below 0 keep their size (the hardware's exp2 takes t to 0 below 2^-126).
    const float t = exp_minus<FAST>(fabsf(u)), near = one_over<FAST>(1.0f + t), far = t * near;
    return __builtin_fmaf(v * rate, far * near, u < 0.f ? far : near);
}

// use(an activation's number as a type): one branch for eight entries.
template <class F>
__device__ __forceinline__ void with_act(int act, F use) {
    switch (act) {
        case DSM_ACT_RELU: return use(std::integral_constant<int, DSM_ACT_RELU>());
        case DSM_ACT_GELU: return use(std::integral_constant<int, DSM_ACT_GELU>());
        case DSM_ACT_GELU_TANH: return use(std::integral_constant<int, DSM_ACT_GELU_TANH>());
        case DSM_ACT_SILU: return use(std::integral_constant<int, DSM_ACT_SILU>());
        default: return;
    }
}
template <bool FAST>
__device__ __forceinline__ void activate(int act, V8& v) {
    with_act(act, [&](auto a) {
#pragma unroll
        for (int q = 0; q < 8; ++q) v.v[q] = activation<decltype(a)::value, FAST>(v.v[q]);
    });
}
// d times the slopes at z, of the columns that there are.
template <bool FAST>
__device__ __forceinline__ void times_slope(int act, V8& d, const V8& z, int have) {
    with_act(act, [&](auto a) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < have) d.v[q] *= slope<decltype(a)::value, FAST>(z.v[q]);
    });
}

// ---- Epilogue of the forward pass ----

// Eight columns of a row of x w^T: bias, z, activation, residual, y.
template <bool F32>
__device__ __forceinline__ void finish(const LinearCall& c, int64_t row, int col, V8 v, const V8& bias) {
    const int have = min(c.p.wide - col, 8);
#pragma unroll
    for (int q = 0; q < 8; ++q) v.v[q] += bias.v[q];
    if (c.z) rows::store8<F32>(c.z, row * c.z_stride + col, v, have);
    activate<!F32>(c.p.act, v);
    if (c.residual) {
        const V8 r = rows::load8<F32>(c.residual, row * c.residual_stride + col, have);
#pragma unroll
        for (int q = 0; q < 8; ++q) v.v[q] += r.v[q];
    }
    rows::store8<F32>(c.y, row * c.y_stride + col, v, have);
}

__device__ __forceinline__ V8 bias8(const LinearCall& c, int col) {
    V8 v;
    if (c.bias) return rows::load8<true>(c.bias, col, c.p.wide - col);
#pragma unroll
    for (int q = 0; q < 8; ++q) v.v[q] = 0.f;
    return v;
}

// ---- Few tokens ----

typedef __bf16 bfloat8 __attribute__((ext_vector_type(8)));

// 16 rows of w by G times 16 tokens a work-group, whose waves take every eighth run of
// 128 bytes of k each (of their part of k: few rows of w leave CUs idle otherwise).  Four
// neighbouring lanes load 64 bytes of a row; lanes that are neighbours in a fragment hold
// neighbouring rows instead, and loads in that order take the L1 a turn for each lane
// (24 tokens of 6400 -> 1600: 19 us).  So runs go through LDS on their way, in a corner of each
// wave's own, without barriers.  The waves' sums meet in LDS.
// Rows past the last one are the last one again, and not stored.
constexpr int kFewWaves = 8;
constexpr int few_runs(int g) { return g < 4 ? 2 : 1; }  // of a wave on their way at once

template <bool F32>
struct Run {  // a lane's part of 16 rows' runs
    static constexpr int kSteps = F32 ? 32 : 64, kEach = F32 ? 4 : 8;
    f4 v[2];
    // `row`: of the lane, from its 16 bytes of each 64 on.
    __device__ __forceinline__ void load(const char* row, int k) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char* at = row + static_cast<int64_t>(k) * (F32 ? 4 : 2) + h * 64;
            if constexpr (F32)
                v[h] = rows::from<false>(reinterpret_cast<const float*>(at));
            else
                v[h] = __builtin_bit_cast(f4, rows::from<false>(reinterpret_cast<const u16*>(at)));
        }
    }
    // The row's last run, shorter than the others: `left` from the lane's bytes on.
    __device__ __forceinline__ void load_end(const char* row, int k, int left) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char* at = row + static_cast<int64_t>(k) * (F32 ? 4 : 2) + h * 64;
            const int have = left - h * (kSteps / 2);
            if constexpr (F32) {
                v[h] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (e < have) v[h][e] = reinterpret_cast<const float*>(at)[e];
            } else {
                u16x8 u = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < have) u[e] = reinterpret_cast<const u16*>(at)[e];
                v[h] = __builtin_bit_cast(f4, u);
            }
        }
    }
    // From lane (row, 16 bytes) = (l / 4, l % 4) to (l % 16, l / 16); the 16 bytes of a row change places
    // so that neither side meets a bank twice.
    __device__ __forceinline__ void turn(f4* lds, int lane) {
        const int r = lane >> 2, l = lane & 15;
#pragma unroll
        for (int h = 0; h < 2; ++h) lds[h * 64 + r * 4 + ((lane & 3) ^ (r >> 2))] = v[h];
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int h = 0; h < 2; ++h) v[h] = lds[h * 64 + l * 4 + ((lane >> 4) ^ (l >> 2))];
        __builtin_amdgcn_wave_barrier();
    }
};

template <bool F32>
__device__ __forceinline__ f4 multiply(const Run<F32>& w, const Run<F32>& x, f4 acc) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w.v[h][e], x.v[h][e], acc, 0, 0, 0);
        } else {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloat8, w.v[h]),
                                                          __builtin_bit_cast(bfloat8, x.v[h]), acc, 0, 0, 0);
        }
    }
    return acc;
}

template <bool F32, int G>
__global__ __launch_bounds__(kFewWaves * 64) void k_few(LinearCall c) {
    using R = Run<F32>;
    constexpr int kBytes = F32 ? 4 : 2, kFewRuns = few_runs(G);
    __shared__ f4 lds[kFewWaves][G < 2 ? 2 : G][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = blockIdx.x * 16, parts = c.p.splits;
    const int dim = c.p.dim, runs = (dim + R::kSteps - 1) / R::kSteps, whole = dim / R::kSteps;
    const int each = (runs + parts - 1) / parts, begin = min(static_cast<int>(blockIdx.y) * each, runs);
    const int end = min(begin + each, runs), full = min(end, whole);
    // Lane l of a fragment has token l % 16, rows l / 16 * 4 .. + 3 of w: eight rows are
    // those of lanes l and l + 16.  What a lane that ends with them adds is on its way early.
    const int g = (threadIdx.x >> 5) % G, l = (threadIdx.x & 15) + ((threadIdx.x >> 4) & 1) * 32;
    const int token = g * 16 + (l & 15), col = n0 + (l >> 5) * 8;
    const bool ends = threadIdx.x < G * 32 && token < c.p.tokens && col < c.p.wide;
    const V8 bias = ends && parts == 1 ? bias8(c, col) : V8{};
    const char* w = static_cast<const char*>(c.w) +
                    static_cast<int64_t>(min(n0 + (lane >> 2), c.p.wide - 1)) * c.w_stride * kBytes + (lane & 3) * 16;
    const char* x[G];
    f4 acc[G];
#pragma unroll
    for (int k = 0; k < G; ++k) {
        x[k] = static_cast<const char*>(c.x) +
               static_cast<int64_t>(min(k * 16 + (lane >> 2), c.p.tokens - 1)) * c.x_stride * kBytes + (lane & 3) * 16;
        acc[k] = f4{0.f, 0.f, 0.f, 0.f};
    }
    f4* corner = &lds[wave][0][0];
    for (int first = begin + wave; first < full; first += kFewWaves * kFewRuns) {
        R a[kFewRuns], b[kFewRuns][G];
#pragma unroll
        for (int u = 0; u < kFewRuns; ++u) {
            const int r = first + u * kFewWaves;
            if (r < full) {
                a[u].load(w, r * R::kSteps);
#pragma unroll
                for (int k = 0; k < G; ++k) b[u][k].load(x[k], r * R::kSteps);
            }
        }
#pragma unroll
        for (int u = 0; u < kFewRuns; ++u)
            if (first + u * kFewWaves < full) {
                a[u].turn(corner, lane);
#pragma unroll
                for (int k = 0; k < G; ++k) {
                    b[u][k].turn(corner, lane);
                    acc[k] = multiply(a[u], b[u][k], acc[k]);
                }
            }
    }
    if (full < end && wave == (full - begin) % kFewWaves) {
        R a, b;
        const int left = dim - full * R::kSteps - (lane & 3) * R::kEach;
        a.load_end(w, full * R::kSteps, left);
        a.turn(corner, lane);
#pragma unroll
        for (int k = 0; k < G; ++k) {
            b.load_end(x[k], full * R::kSteps, left);
            b.turn(corner, lane);
            acc[k] = multiply(a, b, acc[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < G; ++k) lds[wave][k][lane] = acc[k];
    __syncthreads();
    if (!ends) return;
    f4 lo = lds[0][g][l], hi = lds[0][g][l + 16];
#pragma unroll
    for (int q = 1; q < kFewWaves; ++q) {
        lo += lds[q][g][l];
        hi += lds[q][g][l + 16];
    }
    V8 v;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        v.v[q] = lo[q];
        v.v[4 + q] = hi[q];
    }
    if (parts > 1)
        rows::store8<true>(c.workspace + c.p.y_parts, (static_cast<int64_t>(blockIdx.y) * c.p.tokens + token) * c.p.ld_y + col, v, 8);
    else
        finish<F32>(c, token, col, v, bias);
}

// ---- Operands ----

__device__ __forceinline__ u16 float_to_half(float v) { return __builtin_bit_cast(u16, static_cast<_Float16>(v)); }
__device__ __forceinline__ float half_to_float(u16 v) { return static_cast<float>(__builtin_bit_cast(_Float16, v)); }

__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}
__device__ __forceinline__ uint32_t top_of(const V8& x, uint32_t top) {
#pragma unroll
    for (int q = 0; q < 8; ++q) top = max(top, finite_bits(x.v[q]));
    return top;
}
__device__ __forceinline__ uint32_t wave_top(uint32_t top) {
    for (int w = 32; w > 0; w >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), w)));
    return top;
}
// The power of two that brings a largest magnitude into [2^14, 2^15).
__device__ __forceinline__ int exponent_for(uint32_t bits) {
    if (bits == 0) return kNoExponent;
    int e;
    frexpf(__builtin_bit_cast(float, bits), &e);
    return 15 - e;
}

// Eight numbers times 2^e as two halves each, at column col of a row.
__device__ __forceinline__ void store_halves(u16* row, int col, const V8& x, int e) {
    u16x8 hi, lo;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const float v = ldexpf(x.v[q], e);
        hi[q] = float_to_half(v);
        lo[q] = float_to_half(v - half_to_float(hi[q]));
    }
    u16* at = row + ((col >> 5) << 6) + (col & 31);
    *reinterpret_cast<u16x8*>(at) = hi;
    *reinterpret_cast<u16x8*>(at + 32) = lo;
}

// x and w (blockIdx.y) with zeros behind their rows, one wave a row: copies, or, forward, halves
// and the rows' exponents.
template <LinearForm FORM>
__global__ __launch_bounds__(256) void k_copies(LinearCall c, int from, bool twice) {
    const bool of_w = from + blockIdx.y != 0;
    // (x twice, for dz as two halves: its rows from the last token on are zeros then.)
    const int rows = of_w ? c.p.wide : twice ? static_cast<int>(c.p.pad_tokens) : c.p.tokens, lane = threadIdx.x & 63;
    const void* src = of_w ? c.w : c.x;
    const int64_t stride = of_w ? c.w_stride : c.x_stride, ld = c.p.ld_dim;
    const int cols = static_cast<int>(ld / units(FORM));
    u16* dst = reinterpret_cast<u16*>(c.workspace + (of_w ? c.p.w : c.p.x));
    for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += gridDim.x * 4) {
        int e = 0;
        if constexpr (FORM == kLinearHalves) {
            uint32_t top = 0;
#pragma unroll 4
            for (int k = lane * 8; k < c.p.dim; k += 512) top = top_of(rows::load8<true>(src, r * stride + k, c.p.dim - k), top);
            e = exponent_for(wave_top(top));
            if (lane == 0) reinterpret_cast<int32_t*>(c.workspace + (of_w ? c.p.w_exp : c.p.x_exp))[r] = e;
        }
#pragma unroll 4
        for (int k = lane * 8; k < cols; k += 512) {
            const V8 v = rows::load8<is_f32(FORM)>(src, r * stride + k, of_w || r < c.p.tokens ? c.p.dim - k : 0);
            if constexpr (FORM == kLinearHalves) {
                store_halves(dst + r * ld, k, v, e);
            } else {
                const int64_t at = r * (ld / units(FORM)) + k;
                rows::store8<is_f32(FORM)>(dst, at, v, 8);
                if (twice && !of_w) rows::store8<is_f32(FORM)>(dst, at + c.p.pad_tokens * (ld / units(FORM)), v, 8);
            }
        }
    }
}

// dz with zeros behind its rows (unless it is dy, read where it lies) and dbias's sums:
// kDzRows tokens from row0 on by kDzCols columns from col0 on, by a work-group of THREADS;
// 16 lanes have a row's columns, eight each.  (64 lanes for 512 columns: few tokens then
// have few work-groups, whose rows wait for each other; 64 x 1600 in fp32 27 us.)
constexpr int kDzCols = 128;
template <bool F32, int THREADS>
__device__ __forceinline__ void dz_block(const LinearCall& c, int64_t row0, int col0, V8 (*sums)[16]) {
    constexpr int kLanes = THREADS / 16;
    const int lane = threadIdx.x & 15, first = threadIdx.x >> 4, col = col0 + lane * 8;
    const int wide = c.p.wide, have = max(0, min(wide - col, 8));
    const int64_t ld = c.p.ld_wide / (F32 ? 2 : 1);
    V8 sum;
#pragma unroll
    for (int q = 0; q < 8; ++q) sum.v[q] = 0.f;
#pragma unroll
    for (int k = 0; k < kDzRows / kLanes; ++k) {
        const int64_t row = row0 + first + k * kLanes;
        const int here = row < c.p.tokens ? have : 0;
        V8 d = rows::load8<F32>(c.dy, row * c.dy_stride + col, here);
        if (c.p.act != DSM_ACT_NONE)
            times_slope<!F32>(c.p.act, d, rows::load8<F32>(c.z_in, row * c.z_stride + col, here), here);
#pragma unroll
        for (int q = 0; q < 8; ++q) sum.v[q] += d.v[q];
        if (!c.dz_direct && row < c.p.pad_tokens && col < ld) {
            rows::store8<F32>(c.workspace + c.p.dz, row * ld + col, d, 8);
            if (!F32 && c.p.dz_halves) {
#pragma unroll
                for (int q = 0; q < 8; ++q) d.v[q] -= rows::bf16_to_float(rows::float_to_bf16(d.v[q]));
                rows::store8<false>(c.workspace + c.p.dz, (c.p.pad_tokens + row) * ld + col, d, 8);
            }
        }
    }
    if (!c.dbias) return;
    sums[first][lane] = sum;
    __syncthreads();
    if (first != 0) return;
#pragma unroll
    for (int w = 1; w < kLanes; ++w)
#pragma unroll
        for (int q = 0; q < 8; ++q) sum.v[q] += sums[w][lane].v[q];
    if (c.p.bias_parts == 1)
        rows::store8<true>(c.dbias, col, sum, have);
    else
        rows::store8<true>(c.workspace + c.p.bias_sums, row0 / kDzRows * wide + col, sum, have);
}
template <bool F32>
__global__ __launch_bounds__(256) void k_dz(LinearCall c) {
    __shared__ V8 sums[16][16];
    dz_block<F32, 256>(c, static_cast<int64_t>(blockIdx.y) * kDzRows, blockIdx.x * kDzCols, sums);
}

// Halves: dz, its rows' exponents, dbias's sums, and the least exponent of x dz, R tokens a
// work-group (two, where there are too few of them for every CU); the work-groups before those look for w's largest magnitude.  A
// work-group's threads have a row's columns between them, eight each, so that the rows stay in
// registers until their exponents are known (HOLD: up to 8192 columns; wider rows are read
// again).  2045 x 4096 with an activation: 39 us by 256 threads that read twice.
template <bool HOLD, int R>
__global__ __launch_bounds__(1024) void k_dz_split(LinearCall c, int top_groups) {
    __shared__ uint32_t tops[R][16];
    __shared__ uint32_t x_tops[R];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, span = blockDim.x * 8;
    if (static_cast<int>(blockIdx.x) < top_groups) {
        uint32_t top = 0;
        for (int r = blockIdx.x * waves + wave; r < c.p.wide; r += top_groups * waves)
#pragma unroll 4
            for (int k = lane * 8; k < c.p.dim; k += 512)
                top = top_of(rows::load8<true>(c.w, r * c.w_stride + k, c.p.dim - k), top);
        top = wave_top(top);
        if (lane == 0) tops[0][wave] = top;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int k = 1; k < waves; ++k) top = max(top, tops[0][k]);
            reinterpret_cast<uint32_t*>(c.workspace + c.p.w_tops)[blockIdx.x] = top;
        }
        return;
    }
    const int group = blockIdx.x - top_groups, wide = c.p.wide;
    const int64_t first = static_cast<int64_t>(group) * R;
    u16* dz = reinterpret_cast<u16*>(c.workspace + c.p.dz);
    const auto load = [&](int k, int col, int have) {
        const int64_t row = first + k;
        const int here = row < c.p.tokens ? have : 0;
        V8 d = rows::load8<true>(c.dy, row * c.dy_stride + col, here);
        if (c.p.act != DSM_ACT_NONE)
            times_slope<false>(c.p.act, d, rows::load8<true>(c.z_in, row * c.z_stride + col, here), here);
        return d;
    };
    uint32_t top[R];
    V8 held[HOLD ? R : 1];
#pragma unroll
    for (int k = 0; k < R; ++k) top[k] = 0;
    for (int col = threadIdx.x * 8; col < (HOLD ? span : wide); col += span) {
        const int have = max(0, min(wide - col, 8));
        V8 sum;
#pragma unroll
        for (int q = 0; q < 8; ++q) sum.v[q] = 0.f;
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const V8 d = load(k, col, have);
            top[k] = top_of(d, top[k]);
#pragma unroll
            for (int q = 0; q < 8; ++q) sum.v[q] += d.v[q];
            if constexpr (HOLD) held[k] = d;
        }
        if (c.dbias && first < c.p.tokens)
            rows::store8<true>(c.workspace + c.p.bias_sums, static_cast<int64_t>(group) * wide + col, sum, have);
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        top[k] = wave_top(top[k]);
        if (lane == 0) tops[k][wave] = top[k];
    }
    if (c.dw) {  // x's rows
        for (int k = wave; k < R; k += waves) {
            uint32_t t = 0;
            const int64_t row = first + k;
            if (row < c.p.tokens)
                for (int col = lane * 8; col < c.p.dim; col += 512)
                    t = top_of(rows::load8<true>(c.x, row * c.x_stride + col, c.p.dim - col), t);
            t = wave_top(t);
            if (lane == 0) x_tops[k] = t;
        }
    }
    __syncthreads();
    int e[R], least = kNoExponent;
#pragma unroll
    for (int k = 0; k < R; ++k) {
        uint32_t t = 0;
        for (int w = 0; w < waves; ++w) t = max(t, tops[k][w]);
        e[k] = exponent_for(t);
        if (c.dw) least = min(least, e[k] + exponent_for(x_tops[k]));
    }
    if (threadIdx.x == 0) {
        if (c.dw) reinterpret_cast<int32_t*>(c.workspace + c.p.tops)[group] = least;
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (first + k < c.p.tokens) reinterpret_cast<int32_t*>(c.workspace + c.p.z_exp)[first + k] = e[k];
    }
    const int cols = static_cast<int>(c.p.ld_wide / 2);
    for (int col = threadIdx.x * 8; col < cols; col += span) {
        const int have = max(0, min(wide - col, 8));
#pragma unroll
        for (int k = 0; k < R; ++k) store_halves(dz + (first + k) * c.p.ld_wide, col, HOLD ? held[HOLD ? k : 0] : load(k, col, have), e[k]);
    }
}

// The largest of a work-group of 256.
__device__ __forceinline__ int largest(int v) {
    __shared__ int waves[4];
    for (int w = 32; w > 0; w >>= 1) v = max(v, __shfl_xor(v, w));
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    return max(max(waves[0], waves[1]), max(waves[2], waves[3]));
}

// Halves: w (blockIdx.y = 1) times one power of two, and x (0) times those that make its rows meet dz's.
__global__ __launch_bounds__(256) void k_back_copies(LinearCall c, int from, int top_groups, int dz_groups) {
    const bool of_w = from + blockIdx.y != 0;
    int e;
    if (of_w) {
        int top = 0;  // (bits of a magnitude: at least 0)
        const int* tops = reinterpret_cast<const int*>(c.workspace + c.p.w_tops);
        for (int q = threadIdx.x; q < top_groups; q += 256) top = max(top, tops[q]);
        e = exponent_for(static_cast<uint32_t>(largest(top)));
    } else {
        int least = -kNoExponent;
        const int* tops = reinterpret_cast<const int*>(c.workspace + c.p.tops);
        for (int q = threadIdx.x; q < dz_groups; q += 256) least = max(least, -tops[q]);
        e = -largest(least);
    }
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *reinterpret_cast<int32_t*>(c.workspace + (of_w ? c.p.w_exp : c.p.x_exp)) = e;
    const int rows = of_w ? c.p.wide : c.p.tokens, lane = threadIdx.x & 63;
    const void* src = of_w ? c.w : c.x;
    const int64_t stride = of_w ? c.w_stride : c.x_stride, ld = c.p.ld_dim;
    const int cols = static_cast<int>(ld / 2);
    u16* dst = reinterpret_cast<u16*>(c.workspace + (of_w ? c.p.w : c.p.x));
    const int32_t* z_exp = reinterpret_cast<const int32_t*>(c.workspace + c.p.z_exp);
    for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += gridDim.x * 4) {
        // (A row that dz has no entries for meets zeros alone.)
        const int by = of_w ? e : z_exp[r] == kNoExponent ? -kNoExponent : e - z_exp[r];
#pragma unroll 4
        for (int k = lane * 8; k < cols; k += 512)
            store_halves(dst + r * ld, k, rows::load8<true>(src, r * stride + k, c.p.dim - k), by);
    }
}

// ---- Products ----

// 16-bit elements of a row that lies where the caller has it.
template <LinearForm FORM>
__device__ __forceinline__ Operand rows_at(const void* p, int64_t stride, int rows, int cols) {
    return Operand{static_cast<const u16*>(p), stride * units(FORM), rows, cols * units(FORM)};
}
template <LinearForm FORM, bool BACK = false>
__device__ __forceinline__ Operand x_rows(const LinearCall& c) {
    if (FORM != kLinearHalves && c.x_direct) return rows_at<FORM>(c.x, c.x_stride, c.p.tokens, c.p.dim);
    const int rows = BACK && c.p.dz_halves ? static_cast<int>(2 * c.p.pad_tokens) : c.p.tokens;
    return Operand{reinterpret_cast<const u16*>(c.workspace + c.p.x), c.p.ld_dim, rows, static_cast<int32_t>(c.p.ld_dim)};
}
template <LinearForm FORM>
__device__ __forceinline__ Operand w_rows(const LinearCall& c) {
    if (FORM != kLinearHalves && c.w_direct) return rows_at<FORM>(c.w, c.w_stride, c.p.wide, c.p.dim);
    return Operand{reinterpret_cast<const u16*>(c.workspace + c.p.w), c.p.ld_dim, c.p.wide, static_cast<int32_t>(c.p.ld_dim)};
}
template <LinearForm FORM>
__device__ __forceinline__ Operand dz_rows(const LinearCall& c) {
    if (FORM != kLinearHalves && c.dz_direct) return rows_at<FORM>(c.dy, c.dy_stride, c.p.tokens, c.p.wide);
    return Operand{reinterpret_cast<const u16*>(c.workspace + c.p.dz), c.p.ld_wide,
                   static_cast<int32_t>(c.p.pad_tokens * (c.p.dz_halves ? 2 : 1)), static_cast<int32_t>(c.p.ld_wide)};
}

// Work-groups go to the XCDs in turn; every XCD gets one run of the tiles in order.
constexpr int kXcds = 8;
__device__ __forceinline__ int xcd_run(int b, int total) {
    const int x = b & 7, q = total >> 3, r = total & 7;
    return x * q + min(x, r) + (b >> 3);
}
__host__ __device__ inline int per_xcd(int tiles) { return (tiles + kXcds - 1) / kXcds; }

// Part `part` of `parts` of a sum of `all` steps: whole runs of 64.
__device__ __forceinline__ void part_of(int all, int parts, int part, int* begin, int* end) {
    const int each = ((all + 63) / 64 + parts - 1) / parts * 64;
    *begin = min(part * each, all);
    *end = min(*begin + each, all);
}

__device__ __forceinline__ V8 eight_of(const tile::Eight& x) {
    V8 v;
#pragma unroll
    for (int q = 0; q < 8; ++q) v.v[q] = x.v[q];
    return v;
}

// Four columns from `col` on, of which `have` exist.  (fp32 results go to memory as they lie in a
// tile's fragments, four columns a lane and 64 bytes of a row side by side; eight columns a lane would be
// pieces of 16 bytes: 2045 x 1024 x 4096 in fp32, both gradients 126.8 us instead of 124.1.)
__device__ __forceinline__ void store_four(float* row, int col, int have, f4 v) {
    if (have >= 4) {
        *reinterpret_cast<rows::f4_at*>(row + col) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 3; ++e)
        if (e < have) row[col + e] = v[e];
}

// y, or a part of its sums: the tile of rows from row0 on, columns from col0 on.
template <LinearForm FORM, class T, bool PARTS>
__device__ __forceinline__ void forward_tile(const LinearCall& c, int row0, int col0, int part, DSM_LDS char* lds) {
    // (Rows that are read where they lie end with a whole stage, copies have zeros up to one at least.)
    int k0 = 0, k1 = (c.p.dim + T::kSteps - 1) / T::kSteps * T::kSteps;
    if (PARTS) part_of(k1, c.p.splits, part, &k0, &k1);
    T t;
    t.clear();
    t.add(x_rows<FORM>(c), w_rows<FORM>(c), row0, col0, k0, k1, lds, c.p.tokens - row0, c.p.wide - col0);
    const int32_t* x_exp = reinterpret_cast<const int32_t*>(c.workspace + c.p.x_exp);
    const int32_t* w_exp = reinterpret_cast<const int32_t*>(c.workspace + c.p.w_exp);
#pragma unroll
    for (int q = 0; q < T::FJ / 2; ++q) {
        const int col = col0 + t.col8(q);
        const V8 bias = PARTS ? V8{} : bias8(c, col);
        int we[8];
        if constexpr (FORM == kLinearHalves) {
#pragma unroll
            for (int e = 0; e < 8; ++e) we[e] = w_exp[min(col + e, c.p.wide - 1)];
        }
#pragma unroll
        for (int f = 0; f < T::FI; ++f) {
            const int row = row0 + t.row(f);
            V8 v = eight_of(t.eight(f, q));
            if (row >= c.p.tokens || col >= c.p.wide) continue;
            if constexpr (FORM == kLinearHalves) {
                const int xe = x_exp[row];
#pragma unroll
                for (int e = 0; e < 8; ++e) v.v[e] = ldexpf(v.v[e], -(xe + we[e]));
            }
            if constexpr (PARTS)
                rows::store8<true>(c.workspace + c.p.y_parts,
                                   (static_cast<int64_t>(part) * c.p.tokens + row) * c.p.ld_y + col, v, 8);
            else
                finish<is_f32(FORM)>(c, row, col, v, bias);
        }
    }
}

// Tile `id` of tiles_t x tiles_n: eight rows of tiles side by side, so that the tiles an
// XCD has at once share rows of both operands.
__device__ __forceinline__ void place_tile(int id, int tiles_t, int tiles_n, int* tt, int* tn) {
    constexpr int kRows = 8;
    const int group = id / (kRows * tiles_n), rows = min(kRows, tiles_t - group * kRows);
    id -= group * kRows * tiles_n;
    *tn = id / rows;
    *tt = group * kRows + id - *tn * rows;
}

// By tiles of BM.  Tiles of 256 take the first `tiles_n` columns of tiles alone; what a
// last turn that leaves most CUs idle would take goes by tiles of 128.
template <LinearForm FORM, int BM, bool PARTS>
__global__ __launch_bounds__(tile::threads_of(BM)) void k_forward(LinearCall c, int tiles_t, int tiles_n, int groups) {
    using T = tile::Pick<elem(FORM), BM, kContig, kContig>;
    __shared__ __align__(1024) char lds[T::kLdsBytes];
    int tt, tn;
    if constexpr (BM == 256 && !PARTS) {
        if (static_cast<int>(blockIdx.x) >= groups) {
            const int col0 = tiles_n * 256, rest_t = (c.p.tokens + 127) / 128, rest_n = (c.p.wide - col0 + 127) / 128;
            place_tile(xcd_run(blockIdx.x - groups, gridDim.x - groups), rest_t, rest_n, &tt, &tn);
            forward_tile<FORM, tile::Pick<elem(FORM), 128, kContig, kContig>, false>(c, tt * 128, col0 + tn * 128, 0,
                                                                                    (DSM_LDS char*)lds);
            return;
        }
    }
    int id = xcd_run(blockIdx.x, groups);
    const int part = PARTS ? id / (tiles_t * tiles_n) : 0;
    place_tile(id - part * tiles_t * tiles_n, tiles_t, tiles_n, &tt, &tn);
    forward_tile<FORM, T, PARTS>(c, tt * BM, tn * BM, part, (DSM_LDS char*)lds);
}

// Eight columns of the sum of `parts` arrays of `rows` rows.
__device__ __forceinline__ V8 joined(const char* at, int64_t row, int col, int64_t rows, int64_t ld, int parts) {
    V8 v = rows::load8<true>(at, row * ld + col, 8);
    for (int s = 1; s < parts; ++s) {
        const V8 a = rows::load8<true>(at, (s * rows + row) * ld + col, 8);
#pragma unroll
        for (int q = 0; q < 8; ++q) v.v[q] += a.v[q];
    }
    return v;
}

template <bool F32>
__global__ __launch_bounds__(256) void k_forward_join(LinearCall c) {
    const int eights = (c.p.wide + 7) / 8;
    const int64_t all = static_cast<int64_t>(c.p.tokens) * eights, step = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < all; e += step) {
        const int64_t row = e / eights;
        const int col = static_cast<int>(e - row * eights) * 8;
        finish<F32>(c, row, col, joined(c.workspace + c.p.y_parts, row, col, c.p.tokens, c.p.ld_y, c.p.splits), bias8(c, col));
    }
}

__device__ __forceinline__ void store_dx(const LinearCall& c, int64_t row, int col, const V8& v) {
    const int have = min(c.p.dim - col, 8);
    if (c.p.f32)
        rows::store8<true>(c.dx, row * c.dx_stride + col, v, have);
    else
        rows::store8<false>(c.dx, row * c.dx_stride + col, v, have);
}
__device__ __forceinline__ void store_dw(const LinearCall& c, int64_t row, int col, const V8& v) {
    const int have = min(c.p.dim - col, 8);
    if (c.p.f32 || c.p.dw_f32)
        rows::store8<true>(c.dw, row * c.dw_stride + col, v, have);
    else
        rows::store8<false>(c.dw, row * c.dw_stride + col, v, have);
}

// A tile's rows from row0 on, columns from col0 on, of `rows` x `cols`: in fp32, times 2^exponent(row), or in bf16.
template <LinearForm FORM, class T, class E>
__device__ __forceinline__ void store_tile(T& t, int row0, int col0, int rows, int cols, float* to, int64_t stride, E exponent) {
#pragma unroll
    for (int f = 0; f < T::FI; ++f) {
        const int row = row0 + t.row(f);
        if (row >= rows) continue;
        const int e = exponent(row);
#pragma unroll
        for (int q = 0; q < T::FJ; ++q) {
            const int col = col0 + t.col(q);
            f4 v = t.acc[f][q];
            if constexpr (FORM == kLinearHalves) {
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = ldexpf(v[k], e);
            }
            store_four(to + row * stride, col, cols - col, v);
        }
    }
}
template <class T>
__device__ __forceinline__ void store_tile(T& t, int row0, int col0, int high, int cols, u16* to, int64_t stride) {
#pragma unroll
    for (int f = 0; f < T::FI; ++f) {
        const int row = row0 + t.row(f);
#pragma unroll
        for (int q = 0; q < T::FJ / 2; ++q) {
            const int col = col0 + t.col8(q);
            const V8 v = eight_of(t.eight(f, q));
            if (row < high && col < cols) rows::store8<false>(to, row * stride + col, v, min(cols - col, 8));
        }
    }
}

// dx: the tile of tokens from row0 on, columns from col0 on; a part of its sums, or all.
template <LinearForm FORM, class T>
__device__ __forceinline__ void dx_tile(const LinearCall& c, int row0, int col0, int part, int parts, DSM_LDS char* lds) {
    int k0, k1;
    part_of(FORM == kLinearHalves || !c.dz_direct ? static_cast<int>(c.p.ld_wide / units(FORM)) : c.p.wide, parts, part, &k0, &k1);
    T t;
    t.clear();
    t.add(dz_rows<FORM>(c), w_rows<FORM>(c), row0, col0, k0, k1, lds, c.p.tokens - row0, c.p.dim - col0);
    const int32_t* z_exp = reinterpret_cast<const int32_t*>(c.workspace + c.p.z_exp);
    const int we = FORM == kLinearHalves ? *reinterpret_cast<const int32_t*>(c.workspace + c.p.w_exp) : 0;
    const auto exponent = [&](int row) { return FORM == kLinearHalves ? -(z_exp[row] + we) : 0; };
    float* to = reinterpret_cast<float*>(c.workspace + c.p.dx_parts) + static_cast<int64_t>(part) * c.p.tokens * c.p.ld_dx;
    if (is_f32(FORM) && parts == 1) to = static_cast<float*>(c.dx);
    if (is_f32(FORM) || parts > 1)
        store_tile<FORM>(t, row0, col0, c.p.tokens, parts > 1 ? static_cast<int>(c.p.ld_dx) : c.p.dim, to,
                         parts > 1 ? c.p.ld_dx : c.dx_stride, exponent);
    else
        store_tile(t, row0, col0, c.p.tokens, c.p.dim, static_cast<u16*>(c.dx), c.dx_stride);
}

// dw: rows of w from row0 on, columns from col0 on.
template <LinearForm FORM, class T>
__device__ __forceinline__ void dw_tile(const LinearCall& c, int row0, int col0, int part, int parts, DSM_LDS char* lds) {
    int k0, k1;
    // (dz as two halves: one behind the other, and x twice.)
    const int steps = c.p.dz_halves ? static_cast<int>(2 * c.p.pad_tokens) : (c.p.tokens + T::kSteps - 1) / T::kSteps * T::kSteps;
    part_of(steps, parts, part, &k0, &k1);
    T t;
    t.clear();
    t.add(dz_rows<FORM>(c), x_rows<FORM, true>(c), row0, col0, k0, k1, lds, c.p.wide - row0, c.p.dim - col0);
    const int e = FORM == kLinearHalves ? -*reinterpret_cast<const int32_t*>(c.workspace + c.p.x_exp) : 0;
    const auto exponent = [&](int) { return e; };
    float* to = reinterpret_cast<float*>(c.workspace + c.p.dw_parts) + static_cast<int64_t>(part) * c.p.wide * c.p.ld_dx;
    if (parts == 1) to = static_cast<float*>(c.dw);
    if (is_f32(FORM) || parts > 1 || c.p.dw_f32)
        store_tile<FORM>(t, row0, col0, c.p.wide, parts > 1 ? static_cast<int>(c.p.ld_dx) : c.p.dim, to,
                         parts > 1 ? c.p.ld_dx : c.dw_stride, exponent);
    else
        store_tile(t, row0, col0, c.p.wide, c.p.dim, static_cast<u16*>(c.dw), c.dw_stride);
}

// Tile `id` of one of the products, by BM.
template <LinearForm FORM, int BM, bool DW>
__device__ __forceinline__ void back_tile(const LinearCall& c, int id, DSM_LDS char* lds) {
    constexpr tile::Kind KI = DW ? kStrided : kContig;
    const int rows = ((DW ? c.p.wide : c.p.tokens) + BM - 1) / BM, tiles_d = (c.p.dim + BM - 1) / BM;
    const int part = id / (rows * tiles_d), parts = DW ? c.p.dw_splits : c.p.dx_splits;
    id -= part * rows * tiles_d;
    const int tt = id / tiles_d, td = id - tt * tiles_d;
    const auto run = [&](auto as) {
        using T = typename decltype(as)::type;
        if constexpr (DW)
            dw_tile<FORM, T>(c, tt * BM, td * BM, part, parts, lds);
        else
            dx_tile<FORM, T>(c, tt * BM, td * BM, part, parts, lds);
    };
    // Tiles of 256 whose last 128 columns lie past the row are a type of their own.
    if constexpr (BM == 256) {
        if (c.p.dim - td * 256 <= 128)
            run(Type<tile::BigTile<elem(FORM), KI, kStrided, false, true>>());
        else
            run(Type<tile::BigTile<elem(FORM), KI, kStrided, false, false>>());
    } else {
        run(Type<tile::Pick<elem(FORM), BM, KI, kStrided>>());
    }
}

// dx, dw and, where dz is dy, dbias's sums in one launch: neither product fills the CUs'
// last turn by itself.  Each XCD has its run of the product's tiles that have more steps,
// then its run of the other's, then of the sums.  4093 x 1600 x 6400 in bf16: 0.86 PFLOP/s; the CUs'
// clock falls to 1.8 GHz when all of them multiply, and k-strided operands take LDS twice as long.
struct BackJobs {
    int32_t count[3];
    int32_t dw_first;
};
template <LinearForm FORM, int BM>
__global__ __launch_bounds__(tile::threads_of(BM)) void k_backward(LinearCall c, BackJobs jobs) {
    using TX = tile::Pick<elem(FORM), BM, kContig, kStrided>;
    using TW = tile::Pick<elem(FORM), BM, kStrided, kStrided>;
    constexpr int kLds = TX::kLdsBytes > TW::kLdsBytes ? TX::kLdsBytes : TW::kLdsBytes;
    __shared__ __align__(1024) char lds[kLds];
    const int x = blockIdx.x % kXcds;
    int at = blockIdx.x / kXcds, kind = 0;
    while (kind < 2 && at >= per_xcd(jobs.count[kind])) at -= per_xcd(jobs.count[kind++]);
    const int id = x * per_xcd(jobs.count[kind]) + at;
    if (id >= jobs.count[kind]) return;
    if (kind == 2) {
        if constexpr (FORM != kLinearHalves) {
            const int across = (c.p.wide + kDzCols - 1) / kDzCols, down = id / across;
            dz_block<is_f32(FORM), tile::threads_of(BM)>(c, static_cast<int64_t>(down) * kDzRows, (id - down * across) * kDzCols,
                                                         reinterpret_cast<V8(*)[16]>(lds));
        }
    } else if ((kind == 0) == (jobs.dw_first != 0)) {
        back_tile<FORM, BM, true>(c, id, (DSM_LDS char*)lds);
    } else {
        back_tile<FORM, BM, false>(c, id, (DSM_LDS char*)lds);
    }
}

// ---- Few tokens: gradients ----
//
// Both products straight from memory, four columns a lane, without tiles in LDS and without
// copies of w and x.  A matrix instruction takes 16 of its first operand's rows across the
// lanes; element e of what lane i loaded stands for column 4 i + e, so that four instructions
// take four times 16 columns and their sums lie side by side again.  bf16 multiplies eight
// steps of k a lane: its eight rows of four change places in registers first.
//   dx  4 x 16 columns of d and a part of n to a wave: w is read once, dz from the caches.
//   dw  4 x 16 columns of d by kFewRows rows of n to a wave, whose x stays in registers:
//       every row is written in pieces of 128 or 256 bytes.
// 13 tokens of 6400 -> 4800, both products, with dz's and the join's launches: in fp32 56 us, 4.4 TB/s;
// in bf16 28.6, 4.3 TB/s.

constexpr int kFewBackWaves = 4, kFewRows = 64;

struct FewJobs {
    int32_t slabs, dx, dw, bias;  // slabs of 64 columns of d; work-groups
};

// Four columns from `col` on, of which `have` exist.
__device__ __forceinline__ f4 four(const float* row, int col, int have) {
    if (have >= 4) return *reinterpret_cast<const rows::f4_at*>(row + col);
    f4 v = {0.f, 0.f, 0.f, 0.f};
    if (have > 0) {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            const float a = row[col + min(e, have - 1)];
            v[e] = e < have ? a : 0.f;
        }
    }
    return v;
}
typedef u16 u16x4 __attribute__((ext_vector_type(4)));
typedef u16x4 u16x4_at __attribute__((aligned(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct Two {  // four columns in bf16
    uint32_t v[2];
};
__device__ __forceinline__ Two four(const u16* row, int col, int have) {
    u16x4 v = {0, 0, 0, 0};
    if (have >= 4) {
        v = *reinterpret_cast<const u16x4_at*>(row + col);
    } else if (have > 0) {
#pragma unroll
        for (int e = 0; e < 3; ++e) {
            const u16 a = row[col + min(e, have - 1)];
            v[e] = e < have ? a : static_cast<u16>(0);
        }
    }
    return __builtin_bit_cast(Two, v);
}
// Eight rows of four columns: four columns of eight.
__device__ __forceinline__ void turn(const Two (&rows)[8], bfloat8 (&cols)[4]) {
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        u32x4 even, odd;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            even[q] = __builtin_amdgcn_perm(rows[2 * q + 1].v[p], rows[2 * q].v[p], 0x05040100u);
            odd[q] = __builtin_amdgcn_perm(rows[2 * q + 1].v[p], rows[2 * q].v[p], 0x07060302u);
        }
        cols[2 * p] = __builtin_bit_cast(bfloat8, even);
        cols[2 * p + 1] = __builtin_bit_cast(bfloat8, odd);
    }
}

// The waves' sums of dx.  Lane l's acc[g][e][r] is token 16 g + l % 16, column
// d0 + 16 (l / 16) + 4 r + e; wave r sums it.
template <bool F32, int G>
__device__ __forceinline__ void few_dx_end(const LinearCall& c, const f4 (&acc)[G][4], int part, int d0, f4 (*sums)[4][64]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = d0 + 16 * (lane >> 4) + 4 * wave;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        if (g > 0) __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[wave][e][lane] = acc[g][e];
        __syncthreads();
        f4 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float* from = reinterpret_cast<const float*>(&sums[0][e][lane]) + wave;
            v[e] = from[0];
#pragma unroll
            for (int o = 1; o < kFewBackWaves; ++o) v[e] += from[o * 4 * 64 * 4];
        }
        const int token = g * 16 + (lane & 15);
        if (token >= c.p.tokens) continue;
        if (c.p.dx_splits > 1) {
            store_four(reinterpret_cast<float*>(c.workspace + c.p.dx_parts) + (static_cast<int64_t>(part) * c.p.tokens + token) * c.p.ld_dx,
                       at, static_cast<int>(c.p.ld_dx) - at, v);
        } else if constexpr (F32) {
            store_four(static_cast<float*>(c.dx) + token * c.dx_stride, at, c.p.dim - at, v);
        } else {
            u16* row = static_cast<u16*>(c.dx) + token * c.dx_stride;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (at + e < c.p.dim) row[at + e] = rows::float_to_bf16(v[e]);
        }
    }
}

template <int G>
__global__ __launch_bounds__(kFewBackWaves * 64) void k_few_backward(LinearCall c, FewJobs jobs) {
    __shared__ f4 sums[kFewBackWaves][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, k = lane >> 4;
    const int dim = c.p.dim, wide = c.p.wide;
    const int64_t ld = c.p.ld_wide / 2;
    const float* dz = reinterpret_cast<const float*>(c.workspace + c.p.dz);
    if (static_cast<int>(blockIdx.x) < jobs.dx) {
        const int part = blockIdx.x / jobs.slabs, d0 = (blockIdx.x - part * jobs.slabs) * 64, col = d0 + 4 * i, have = dim - col;
        const float* w = static_cast<const float*>(c.w);
        // Runs of 16 rows of w, every fourth one to a wave.
        const int runs = (wide + 15) / 16, each = (runs + c.p.dx_splits - 1) / c.p.dx_splits;
        const int begin = part * each, end = min(begin + each, runs);
        f4 acc[G][4];
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[g][e] = f4{0.f, 0.f, 0.f, 0.f};
        constexpr int kAhead = G < 4 ? 4 : 2;
        for (int first = begin + wave; first < end; first += kFewBackWaves * kAhead) {
            f4 a[kAhead][4], b[kAhead][G];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int n0 = (first + u * kFewBackWaves) * 16;
                if (first + u * kFewBackWaves < end) {
                    // (Rows past the last one meet zeros in dz.)
#pragma unroll
                    for (int s = 0; s < 4; ++s) a[u][s] = four(w + min(n0 + 4 * k + s, wide - 1) * c.w_stride, col, have);
#pragma unroll
                    for (int g = 0; g < G; ++g) b[u][g] = *reinterpret_cast<const f4*>(dz + (g * 16 + i) * ld + n0 + 4 * k);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (first + u * kFewBackWaves < end) {
#pragma unroll
                    for (int s = 0; s < 4; ++s)
#pragma unroll
                        for (int g = 0; g < G; ++g)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                acc[g][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[u][s][e], b[u][g][s], acc[g][e], 0, 0, 0);
                }
        }
        few_dx_end<true, G>(c, acc, part, d0, sums);
        return;
    }
    // (Columns go to lanes so that a store's four lanes of a row have 64 bytes of it side by side: 13 tokens
    // of 6400 -> 4800 28 us for dw, dz's launch included; 46 by pieces of 16 bytes.)
    const int id = blockIdx.x - jobs.dx, down = id / jobs.slabs, d0 = (id - down * jobs.slabs) * 64;
    const int col = d0 + 4 * (4 * (i & 3) + (i >> 2)), have = dim - col;
    const int n = (down * kFewBackWaves + wave) * kFewRows + 4 * i;
    if (n >= c.p.ld_wide / 2) return;
    const float* x = static_cast<const float*>(c.x);
    f4 a[4 * G], b[4 * G];
    // (dz has zeros for the tokens that x does not have, and 64 columns a run.)
#pragma unroll
    for (int s = 0; s < 4 * G; ++s) {
        a[s] = four(x + min(4 * s + k, c.p.tokens - 1) * c.x_stride, col, have);
        b[s] = *reinterpret_cast<const f4*>(dz + (4 * s + k) * ld + n);
    }
    // Lane l's acc[e][r] is row n + q, column d0 + 16 r + 4 (l / 16) + e.
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        f4 acc[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < 4 * G; ++s)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s][e], b[s][q], acc[e], 0, 0, 0);
        if (n + q >= wide) continue;
        float* row = static_cast<float*>(c.dw) + (n + q) * c.dw_stride;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int at = d0 + 16 * r + 4 * k;
            store_four(row, at, dim - at, f4{acc[0][r], acc[1][r], acc[2][r], acc[3][r]});
        }
    }
}

// bf16: dz is dy where it lies, or its copy, in HALVES for dw.
template <int G, int HALVES>
__global__ __launch_bounds__(kFewBackWaves * 64) void k_few_backward_bf16(LinearCall c, FewJobs jobs) {
    __shared__ f4 sums[kFewBackWaves][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = lane & 15, k = lane >> 4;
    const int dim = c.p.dim, wide = c.p.wide, tokens = c.p.tokens;
    const u16* dz = c.dz_direct ? static_cast<const u16*>(c.dy) : reinterpret_cast<const u16*>(c.workspace + c.p.dz);
    const int64_t ld = c.dz_direct ? c.dy_stride : c.p.ld_wide;
    int id = blockIdx.x;
    if (id < jobs.dx) {
        const int part = id / jobs.slabs, d0 = (id - part * jobs.slabs) * 64, col = d0 + 4 * i, have = dim - col;
        const u16* w = static_cast<const u16*>(c.w);
        // Runs of 32 rows of w, every fourth one to a wave.
        const int runs = (wide + 31) / 32, each = (runs + c.p.dx_splits - 1) / c.p.dx_splits;
        const int begin = part * each, end = min(begin + each, runs);
        f4 acc[G][4];
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[g][e] = f4{0.f, 0.f, 0.f, 0.f};
        constexpr int kAhead = 2;
        for (int first = begin + wave; first < end; first += kFewBackWaves * kAhead) {
            Two a[kAhead][8];
            rows::Raw8<false> b[kAhead][G];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int n0 = (first + u * kFewBackWaves) * 32 + 8 * k;
                if (first + u * kFewBackWaves < end) {
                    // (Rows past the last one meet zeros in dz; tokens past the last one are not stored.)
#pragma unroll
                    for (int j = 0; j < 8; ++j) a[u][j] = four(w + min(n0 + j, wide - 1) * c.w_stride, col, have);
#pragma unroll
                    for (int g = 0; g < G; ++g) b[u][g] = rows::raw8<false>(dz, min(g * 16 + i, tokens - 1) * ld + n0, wide - n0);
                }
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
                if (first + u * kFewBackWaves < end) {
                    bfloat8 f[4];
                    turn(a[u], f);
#pragma unroll
                    for (int g = 0; g < G; ++g)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[g][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f[e], __builtin_bit_cast(bfloat8, b[u][g].v), acc[g][e], 0, 0, 0);
                }
        }
        few_dx_end<false, G>(c, acc, part, d0, sums);
        return;
    }
    id -= jobs.dx;
    if (id >= jobs.dw) {  // dbias, where dz is dy
        dz_block<false, kFewBackWaves * 64>(c, 0, (id - jobs.dw) * kDzCols, reinterpret_cast<V8(*)[16]>(&sums[0][0][0]));
        return;
    }
    // (As above, of two columns' fours a store.)
    const int down = id / jobs.slabs, d0 = (id - down * jobs.slabs) * 64;
    const int col = d0 + 4 * (8 * ((i >> 1) & 1) + 2 * (i >> 2) + (i & 1)), have = dim - col;
    const int n = (down * kFewBackWaves + wave) * kFewRows + 4 * i;
    static_assert(G <= 2, "one step of 32 tokens");
    bfloat8 a[4], b[HALVES][4];
    Two r[8], d[HALVES][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        // (Tokens past the last one: x's last row, and zeros in dz.)
        const int token = 8 * k + j, row = min(token, tokens - 1);
        r[j] = four(static_cast<const u16*>(c.x) + row * c.x_stride, col, have);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) d[h][j] = four(dz + (row + h * c.p.pad_tokens) * ld, n, token < tokens ? wide - n : 0);
    }
    turn(r, a);
#pragma unroll
    for (int h = 0; h < HALVES; ++h) turn(d[h], b[h]);
    // Lane l's acc[e][r] is row n + q, column d0 + 32 (r / 2) + 8 (l / 16) + 4 (r % 2) + e.
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        f4 acc[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[e], b[h][q], acc[e], 0, 0, 0);
        if (n + q >= wide) continue;
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            const int at = d0 + 32 * o + 8 * k;
            if (at >= dim) continue;
            V8 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v.v[e] = acc[e][2 * o];
                v.v[4 + e] = acc[e][2 * o + 1];
            }
            store_dw(c, n + q, at, v);
        }
    }
}

// What is left: dbias from its sums (the first work-groups, 16 columns each), and dx
// and dw where their sums are in parts.
__global__ __launch_bounds__(256) void k_backward_join(LinearCall c, int bias_groups) {
    __shared__ float sums[16][16];
    if (static_cast<int>(blockIdx.x) < bias_groups) {
        const int lane = threadIdx.x & 15, first = threadIdx.x >> 4, col = blockIdx.x * 16 + lane;
        float s = 0.f;
        if (col < c.p.wide) {
            const float* at = reinterpret_cast<const float*>(c.workspace + c.p.bias_sums) + col;
#pragma unroll 8
            for (int q = first; q < c.p.bias_parts; q += 16) s += at[static_cast<int64_t>(q) * c.p.wide];
        }
        sums[first][lane] = s;
        __syncthreads();
        if (first != 0 || col >= c.p.wide) return;
#pragma unroll
        for (int w = 1; w < 16; ++w) s += sums[w][lane];
        c.dbias[col] = s;
        return;
    }
    const int eights = (c.p.dim + 7) / 8;
    const int64_t of_dx = c.dx && c.p.dx_splits > 1 ? static_cast<int64_t>(c.p.tokens) * eights : 0;
    const int64_t of_dw = c.dw && c.p.dw_splits > 1 ? static_cast<int64_t>(c.p.wide) * eights : 0;
    const int64_t step = static_cast<int64_t>(gridDim.x - bias_groups) * 256;
    for (int64_t e = static_cast<int64_t>(blockIdx.x - bias_groups) * 256 + threadIdx.x; e < of_dx + of_dw; e += step) {
        const bool dw = e >= of_dx;
        const int64_t at = dw ? e - of_dx : e, row = at / eights;
        const int col = static_cast<int>(at - row * eights) * 8;
        if (dw)
            store_dw(c, row, col, joined(c.workspace + c.p.dw_parts, row, col, c.p.wide, c.p.ld_dx, c.p.dw_splits));
        else
            store_dx(c, row, col, joined(c.workspace + c.p.dx_parts, row, col, c.p.tokens, c.p.ld_dx, c.p.dx_splits));
    }
}

// No tokens: dw and dbias are zero.
__global__ __launch_bounds__(256) void k_no_tokens(LinearCall c) {
    V8 zero;
#pragma unroll
    for (int q = 0; q < 8; ++q) zero.v[q] = 0.f;
    if (c.dbias)
        for (int n = blockIdx.x * 256 + threadIdx.x; n < c.p.wide; n += gridDim.x * 256) c.dbias[n] = 0.f;
    if (!c.dw) return;
    for (int row = blockIdx.x; row < c.p.wide; row += gridDim.x)
        for (int col = threadIdx.x * 8; col < c.p.dim; col += 2048) store_dw(c, row, col, zero);
}

// ---- Launches ----

unsigned groups_for(int64_t wanted, int64_t most) { return static_cast<unsigned>(wanted < most ? wanted : most); }

template <bool F32>
void forward_join(const LinearCall& c, hipStream_t stream) {
    const int64_t eights = static_cast<int64_t>(c.p.tokens) * ((c.p.wide + 7) / 8);
    k_forward_join<F32><<<groups_for((eights + 255) / 256, 4096), 256, 0, stream>>>(c);
}

template <LinearForm FORM, int BM>
void forward(const LinearCall& c, hipStream_t stream) {
    const int tiles_t = (c.p.tokens + BM - 1) / BM, all = (c.p.wide + BM - 1) / BM;
    const int tiles_n = BM == 256 && c.p.splits == 1 ? c.p.front : all, groups = tiles_t * tiles_n * c.p.splits;
    if (c.p.splits > 1) {
        k_forward<FORM, BM, true><<<groups, tile::threads_of(BM), 0, stream>>>(c, tiles_t, tiles_n, groups);
        forward_join<is_f32(FORM)>(c, stream);
    } else {
        const int rest = tiles_n < all ? (c.p.tokens + 127) / 128 * ((c.p.wide - tiles_n * 256 + 127) / 128) : 0;
        k_forward<FORM, BM, false><<<groups + rest, tile::threads_of(BM), 0, stream>>>(c, tiles_t, tiles_n, groups);
    }
}

template <LinearForm FORM>
void forward(const LinearCall& c, hipStream_t stream) {
    // x from 0, w from 1: whichever is not read where it lies.
    const int from = c.x_direct ? 1 : 0, to = c.w_direct ? 1 : 2;
    if (from < to) {
        const int rows = c.p.tokens > c.p.wide ? c.p.tokens : c.p.wide;
        k_copies<FORM><<<dim3(groups_for((rows + 3) / 4, 4096), to - from), 256, 0, stream>>>(c, from, false);
    }
    if constexpr (FORM != kLinearSingle) {
        if (c.p.tile == 128) return forward<FORM, 128>(c, stream);
        if (c.p.tile == 256) return forward<FORM, 256>(c, stream);
    }
    forward<FORM, 64>(c, stream);
}

// use(groups of 16 tokens as a type)
template <class F>
void with_groups(int tokens, F use) {
    if (tokens <= 16)
        use(std::integral_constant<int, 1>());
    else if (tokens <= 32)
        use(std::integral_constant<int, 2>());
    else
        use(std::integral_constant<int, 4>());
}

template <bool F32>
void few(const LinearCall& c, hipStream_t stream) {
    const dim3 n((c.p.wide + 15) / 16, c.p.splits);
    with_groups(c.p.tokens, [&](auto g) { k_few<F32, decltype(g)::value><<<n, kFewWaves * 64, 0, stream>>>(c); });
    if (c.p.splits > 1) forward_join<F32>(c, stream);
}

template <LinearForm FORM, int BM>
void backward(const LinearCall& c, bool with_bias, hipStream_t stream) {
    const auto tiles = [](int n, int of) { return (n + of - 1) / of; };
    const int dx = c.dx ? tiles(c.p.tokens, BM) * tiles(c.p.dim, BM) * c.p.dx_splits : 0;
    const int dw = c.dw ? tiles(c.p.wide, BM) * tiles(c.p.dim, BM) * c.p.dw_splits : 0;
    BackJobs jobs;
    jobs.dw_first = static_cast<int64_t>(c.p.tokens) * c.p.dx_splits > static_cast<int64_t>(c.p.wide) * c.p.dw_splits;
    jobs.count[0] = jobs.dw_first ? dw : dx;
    jobs.count[1] = jobs.dw_first ? dx : dw;
    jobs.count[2] = with_bias ? static_cast<int>((c.p.wide + kDzCols - 1) / kDzCols * (c.p.pad_tokens / kDzRows)) : 0;
    const int groups = per_xcd(jobs.count[0]) + per_xcd(jobs.count[1]) + per_xcd(jobs.count[2]);
    k_backward<FORM, BM><<<kXcds * groups, tile::threads_of(BM), 0, stream>>>(c, jobs);
}

void few_backward(const LinearCall& c, hipStream_t stream) {
    FewJobs jobs;
    jobs.slabs = (c.p.dim + 63) / 64;
    jobs.dx = c.dx ? jobs.slabs * c.p.dx_splits : 0;
    jobs.dw = c.dw ? jobs.slabs * ((c.p.wide + kFewBackWaves * kFewRows - 1) / (kFewBackWaves * kFewRows)) : 0;
    jobs.bias = c.dz_direct && c.dbias ? (c.p.wide + kDzCols - 1) / kDzCols : 0;
    const int groups = jobs.dx + jobs.dw + jobs.bias;
    with_groups(c.p.tokens, [&](auto g) {
        constexpr int G = decltype(g)::value;
        if (c.p.f32) {
            k_few_backward<G><<<groups, kFewBackWaves * 64, 0, stream>>>(c, jobs);
        } else if constexpr (G <= 2) {
            if (c.p.dz_halves)
                k_few_backward_bf16<G, 2><<<groups, kFewBackWaves * 64, 0, stream>>>(c, jobs);
            else
                k_few_backward_bf16<G, 1><<<groups, kFewBackWaves * 64, 0, stream>>>(c, jobs);
        }
    });
}

template <LinearForm FORM>
void backward(const LinearCall& c, hipStream_t stream) {
    const int copies_rows = c.p.tokens > c.p.wide ? c.p.tokens : c.p.wide;
    // x is wanted for dw, w for dx.
    const int from = c.dw && !c.x_direct ? 0 : 1, to = c.dx && !c.w_direct ? 2 : 1;
    if constexpr (FORM == kLinearHalves) {
        const int top_groups = c.dx ? static_cast<int>(groups_for((c.p.wide + 3) / 4, kLinearTopParts)) : 0;
        const int dz_groups = static_cast<int>(c.p.pad_tokens / c.p.split_rows);
        // (ld_wide counts halves: its columns, eight a thread, are a multiple of 64.  Four waves or more, for x's rows.)
        const int threads = static_cast<int>((c.p.ld_wide / 16 + 63) / 64 * 64), groups = top_groups + dz_groups;
        if (threads > 1024)
            k_dz_split<false, 8><<<groups, 1024, 0, stream>>>(c, top_groups);
        else if (c.p.split_rows == 8)
            k_dz_split<true, 8><<<groups, threads < 256 ? 256 : threads, 0, stream>>>(c, top_groups);
        else
            k_dz_split<true, 2><<<groups, threads < 256 ? 256 : threads, 0, stream>>>(c, top_groups);
        if (from < to)
            k_back_copies<<<dim3(groups_for((copies_rows + 3) / 4, 2048), to - from), 256, 0, stream>>>(c, from, top_groups,
                                                                                                      dz_groups);
    } else {
        // (Where dz is dy, dbias's sums run beside the products.)
        if (!c.dz_direct || (c.dbias && !c.dx && !c.dw))
            k_dz<is_f32(FORM)><<<dim3((c.p.ld_wide / units(FORM) + kDzCols - 1) / kDzCols, c.p.pad_tokens / kDzRows), 256, 0, stream>>>(c);
        if (!c.p.back_few && from < to)
            k_copies<FORM><<<dim3(groups_for((copies_rows + 3) / 4, 4096), to - from), 256, 0, stream>>>(c, from, c.p.dz_halves);
    }
    if (c.dx || c.dw) {
        const bool with_bias = FORM != kLinearHalves && c.dz_direct && c.dbias;
        if (c.p.back_few)
            few_backward(c, stream);
        else if constexpr (FORM != kLinearSingle) {
            if (c.p.back_tile == 64)
                backward<FORM, 64>(c, with_bias, stream);
            else if (c.p.back_tile == 128)
                backward<FORM, 128>(c, with_bias, stream);
            else
                backward<FORM, 256>(c, with_bias, stream);
        }
    }
    const int bias_groups = c.dbias && c.p.bias_parts > 1 ? (c.p.wide + 15) / 16 : 0;
    const int64_t eights = (c.p.dim + 7) / 8;
    const int64_t join = (c.dx && c.p.dx_splits > 1 ? c.p.tokens * eights : 0) + (c.dw && c.p.dw_splits > 1 ? c.p.wide * eights : 0);
    const unsigned groups = bias_groups + groups_for((join + 255) / 256, 4096);
    if (groups > 0) k_backward_join<<<groups, 256, 0, stream>>>(c, bias_groups);
}

}  // namespace

hipError_t launch_linear(const LinearCall& c, hipStream_t stream) {
    if (c.p.few) {
        if (c.p.f32)
            few<true>(c, stream);
        else
            few<false>(c, stream);
    } else if (c.p.form == kLinearSingle) {
        forward<kLinearSingle>(c, stream);
    } else if (c.p.form == kLinearHalves) {
        forward<kLinearHalves>(c, stream);
    } else {
        forward<kLinearBf16>(c, stream);
    }
    return hipGetLastError();
}

hipError_t launch_linear_backward(const LinearCall& c, hipStream_t stream) {
    if (c.p.tokens == 0)
        k_no_tokens<<<groups_for(c.p.wide, 2048), 256, 0, stream>>>(c);
    else if (c.p.back_form == kLinearSingle)
        backward<kLinearSingle>(c, stream);
    else if (c.p.back_form == kLinearHalves)
        backward<kLinearHalves>(c, stream);
    else
        backward<kLinearBf16>(c, stream);
    return hipGetLastError();
}

}  // namespace dsm
