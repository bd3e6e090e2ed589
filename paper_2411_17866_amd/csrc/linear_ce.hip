// Softmax cross entropy of a linear layer over a large vocabulary on gfx950,
// with the gradients of the layer's input and weight.
//
//   z = h w^T;  lse_t = log sum_v exp z_tv;  loss_t = lse_t - z_t,target
//   G_tv = c_t (exp(z_tv - lse_t) - [v = target_t]);  dh = G w;  dw = G^T h
//
// A first pass over the vocabulary computes the logits tile by tile and keeps of
// each row of a tile its largest logit and the sum of exp(z - largest); joined over
// the tiles they give lse.  With gradients, G has to be in memory, for two products
// read it: it is made for a piece of the vocabulary at a time, at most 1 GiB, in 16
// bits or two halves an entry.  The logits themselves are never in memory.
//   * For the first piece, which is most often the only one, the first pass leaves
//     exp(z - largest of a wave's columns) in G's place, and a light pass multiplies
//     it by c exp(largest - lse); the target's entry, where p - 1 cancels, it
//     computes anew.  6 T V D operations of the matrix cores.
//   * For the others the logits are computed again, 8 T V D in all.
// 8192 tokens of 50257 x 768 in bf16, whose G is 0.8 GB: 2.87 ms by two pieces, both
// computed again; 2.28 ms by one; 1.93 ms with what follows.
//
// The light pass itself is saved, with many tokens and a large vocabulary, by a
// reference r_t for each row that is near lse_t and known before the first pass: the
// logarithm of the sum over a few tiles of the vocabulary, a turn of the CUs, scaled
// to all of it.  Exponentials are then kept relative to r_t and stay as they are:
//   G_tv = s_t E_tv,  E_tv = 2^k (exp(z_tv - x_t) - [v = target] exp(lse_t - x_t)),
//   s_t = 2^-k c_t exp(x_t - lse_t),  x_t = r_t
// dh's sums are multiplied by s_t where they are joined, and dw is the product of E
// with s_t h_t, which is written transposed on the way.  Only a row whose lse_t turns
// out too far from r_t for fp16's range is passed over once more (x_t = lse_t).
//
// The target's exponential stays out of the sums: the first pass keeps the target's
// logit and adds up the others, R = sum over v != target of exp(z_tv - x), so that a row
// that is nearly sure of its target keeps the digits of what is left,
//   loss_t = log(1 + R / exp(z_target - x)),  p_target - 1 = expm1(-loss_t)
// Arguments of exponentials are near 0 where they count: powers of two that use fp16's
// range are multiplied in afterwards.  (With those in the argument and the target among
// the rest, losses were off by 4e-7, all of a loss of 1e-6.)
//
// What the products take ("form", chosen by the host from type and tokens):
//   fp16, scaled     bf16 buffers, many tokens.  A power of two brings an
//                    operand's largest finite entry just under fp16's largest
//                    number; a bf16 number then keeps all its bits down to 2^-32
//                    of the largest, and G keeps 11 bits where bf16 would leave
//                    it 8: a row of G is mostly its target's entry, whose
//                    rounding no sum averages out, and in bf16 it alone would
//                    cost the gradients what their own rounding to bf16 does.
//   two fp16 halves  fp32 buffers, many tokens (gemm_tile.h)
//   bf16             bf16 buffers, few tokens or no gradients: w is read where it
//                    lies, which saves the passes over w that find its largest
//                    entry and convert it, and G goes as two bf16 halves (twice
//                    the matrix instructions in the products of G)
//   fp32             fp32 buffers, few tokens: w is read where it lies
// Few tokens are those for which reading w costs more than multiplying it.
// Logits, softmax statistics, losses and sums are fp32.
//
// A token whose target lies outside [0, vocab) has no loss and no gradient, and
// what its row of h holds, NaN included, reaches no output but its own zeros.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "gemm_tile.h"
#include "ops_internal.h"

#pragma clang fp contract(off)

namespace dsm {
namespace {

using tile::f4;
using tile::kContig;
using tile::kStrided;
using tile::Operand;

typedef unsigned short u16;
typedef u16 u16x4 __attribute__((ext_vector_type(4)));
typedef u16 u16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ u16 float_to_bf16(float v) {
    return __builtin_bit_cast(u16, static_cast<__bf16>(v));
}
__device__ __forceinline__ float half_to_float(u16 v) {
    return static_cast<float>(__builtin_bit_cast(_Float16, v));
}
__device__ __forceinline__ u16 float_to_half(float v) {
    return __builtin_bit_cast(u16, static_cast<_Float16>(v));
}

__device__ __forceinline__ float bf16_to_float(u16 v) {
    return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16);
}

constexpr bool is_f32(CeForm f) { return f == kCeHalves || f == kCeF32; }
constexpr bool is_scaled(CeForm f) { return f == kCeHalf || f == kCeHalves; }
constexpr tile::Elem elem(CeForm f) {
    return f == kCeHalf ? tile::kF16 : f == kCeBf16 ? tile::kBF16 : f == kCeHalves ? tile::kSplit : tile::kF32;
}
constexpr int units(CeForm f) { return tile::units(elem(f)); }

struct Scalars {
    uint32_t h_max, w_max;  // bits of the largest finite |h| and |w| (scaled forms)
    uint32_t c_max;         // bits of the largest finite |c_t|
    uint32_t parts[2][kCeParts];  // of the work-groups that look for h_max and w_max
};
static_assert(sizeof(Scalars) <= kCeScalars, "the host's plan leaves room for this");

// The power of two that brings a largest magnitude into [2^14, 2^15).
__device__ __forceinline__ int exponent_for(uint32_t bits) {
    if (bits == 0) return 0;
    int e;
    frexpf(__builtin_bit_cast(float, bits), &e);
    return min(15 - e, 120);
}

__device__ __forceinline__ bool is_valid(int64_t target, int vocab) { return target >= 0 && target < vocab; }

__device__ __forceinline__ uint32_t finite_bits(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// c_t of a token with a valid target, of which there are `count`.
__device__ __forceinline__ float coefficient(const CeBuffers& b, int t, int count) {
    return (b.weight ? b.weight[t] : 1.0f) / (b.mean ? static_cast<float>(max(count, 1)) : 1.0f);
}

// c_t of every token and their largest magnitude, for the gradients; by one
// work-group.
__device__ void coefficients(const CePlan& p, const CeBuffers& b) {
    __shared__ int count;
    __shared__ uint32_t c_max;
    if (threadIdx.x == 0) {
        count = 0;
        c_max = 0;
    }
    __syncthreads();
    int mine = 0;
#pragma unroll 8
    for (int t = threadIdx.x; t < p.tokens; t += blockDim.x) mine += is_valid(b.target[t], p.vocab);
    for (int w = 32; w > 0; w >>= 1) mine += __shfl_xor(mine, w);
    if ((threadIdx.x & 63) == 0) atomicAdd(&count, mine);
    __syncthreads();
    float* coef = reinterpret_cast<float*>(b.workspace + p.coef);
    uint32_t top = 0;
    // (Eight tokens' loads before their stores, which might overlap them.)
    for (int first = threadIdx.x; first < p.tokens; first += 8 * blockDim.x) {
        float c[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int t = min(first + q * static_cast<int>(blockDim.x), p.tokens - 1);
            const bool valid = is_valid(b.target[t], p.vocab);
            c[q] = coefficient(b, t, count);
            c[q] = valid ? c[q] : 0.f;
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int t = first + q * static_cast<int>(blockDim.x);
            if (t < p.tokens) coef[t] = c[q];
            top = max(top, finite_bits(c[q]));
        }
    }
    atomicMax(&c_max, top);
    __syncthreads();
    if (threadIdx.x == 0) {
        reinterpret_cast<Scalars*>(b.workspace + p.scalars)->c_max = c_max;
    }
}

template <bool F32>
__device__ __forceinline__ f4 load4(const void* base, int64_t at, int have, bool vec) {
    f4 v = {0.f, 0.f, 0.f, 0.f};
    if constexpr (F32) {
        const float* p = static_cast<const float*>(base) + at;
        if (vec) return *reinterpret_cast<const f4*>(p);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < have) v[q] = p[q];
    } else {
        const u16* p = static_cast<const u16*>(base) + at;
        if (vec) {
            const u16x4 b = *reinterpret_cast<const u16x4*>(p);
#pragma unroll
            for (int q = 0; q < 4; ++q) v[q] = bf16_to_float(b[q]);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (q < have) v[q] = bf16_to_float(p[q]);
        }
    }
    return v;
}

// The largest of a work-group of 256.
__device__ __forceinline__ uint32_t largest_of_group(uint32_t top) {
    __shared__ uint32_t tops[4];
    for (int w = 32; w > 0; w >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), w)));
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = top;
    __syncthreads();
    return max(max(tops[0], tops[1]), max(tops[2], tops[3]));
}

// The largest finite magnitude of h's valid rows (blockIdx.y = 0) and of w (1), one
// of each work-group.  (Atomics on one address would take turns: 54 us where this
// takes 19 for w of 50257 x 768 in bf16, 4.0 TB/s.)  A work-group past those computes
// the coefficients, for which nothing waits here.
template <bool F32>
__global__ __launch_bounds__(256) void k_largest(CePlan p, CeBuffers b) {
    const bool of_w = blockIdx.y != 0;
    const int groups = static_cast<int>(gridDim.x) - 1;
    if (static_cast<int>(blockIdx.x) >= groups) {
        if (!of_w && p.grads) coefficients(p, b);
        return;
    }
    const void* src = of_w ? b.w : b.h;
    const bool vec = of_w ? b.w_vector : b.h_vector;
    const int64_t stride = of_w ? b.w_stride : b.h_stride;
    const int rows = of_w ? p.vocab : p.tokens;
    uint32_t top = 0;
    if (of_w && vec && stride == p.dim) {  // one run of elements
        const int64_t all = static_cast<int64_t>(rows) * p.dim / 4;
        const int64_t step = static_cast<int64_t>(groups) * 256;
#pragma unroll 8
        for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < all; e += step) {
            const f4 v = load4<F32>(src, e * 4, 4, true);
#pragma unroll
            for (int q = 0; q < 4; ++q) top = max(top, finite_bits(v[q]));
        }
    } else {
        for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += groups * 4) {
            if (!of_w && !is_valid(b.target[r], p.vocab)) continue;
#pragma unroll 4
            for (int c = (threadIdx.x & 63) * 4; c < p.dim; c += 256) {
                const f4 v = load4<F32>(src, r * stride + c, p.dim - c, vec);
#pragma unroll
                for (int q = 0; q < 4; ++q) top = max(top, finite_bits(v[q]));
            }
        }
    }
    top = largest_of_group(top);
    if (threadIdx.x == 0)
        reinterpret_cast<Scalars*>(b.workspace + p.scalars)->parts[of_w][blockIdx.x] = top;
}

// h (blockIdx.y = 0) and w (1) as the products take them: rows of a multiple of
// 64 columns, h with a multiple of 64 rows; zeros in the padding and in h's rows
// without a valid target.  In the forms without a scale the last work-group of h computes
// the coefficients.  `parts`: of the largest magnitudes.
template <CeForm FORM>
__global__ __launch_bounds__(256) void k_operands(CePlan p, CeBuffers b, int parts) {
    const bool of_w = blockIdx.y != 0;
    const int groups = static_cast<int>(gridDim.x) - (is_scaled(FORM) ? 0 : 1);
    if (static_cast<int>(blockIdx.x) >= groups) {
        if (!of_w && p.grads) coefficients(p, b);
        return;
    }
    const int rows = of_w ? p.vocab : (p.tokens + 63) / 64 * 64;
    const void* src = of_w ? b.w : b.h;
    const bool vec = of_w ? b.w_vector : b.h_vector;
    const int64_t stride = of_w ? b.w_stride : b.h_stride;
    const int64_t ld = of_w ? p.ld_w : p.ld_h;
    const int cols = static_cast<int>(ld / units(FORM));
    u16* dst = reinterpret_cast<u16*>(b.workspace + (of_w ? p.w : p.h));
    float scale = 1.f;
    if constexpr (is_scaled(FORM)) {
        Scalars* s = reinterpret_cast<Scalars*>(b.workspace + p.scalars);
        uint32_t top = 0;
        for (int q = threadIdx.x; q < parts; q += 256) top = max(top, s->parts[of_w][q]);
        top = largest_of_group(top);
        if (blockIdx.x == 0 && threadIdx.x == 0) *(of_w ? &s->w_max : &s->h_max) = top;
        scale = ldexpf(1.f, exponent_for(top));
    }
    for (int r = blockIdx.x * 4 + (threadIdx.x >> 6); r < rows; r += groups * 4) {
        const bool keep = of_w || (r < p.tokens && is_valid(b.target[r], p.vocab));
        u16* out = dst + r * ld;
#pragma unroll 4
        for (int c = (threadIdx.x & 63) * 4; c < cols; c += 256) {
            f4 v = {0.f, 0.f, 0.f, 0.f};
            if (keep && c < p.dim) v = load4<is_f32(FORM)>(src, r * stride + c, p.dim - c, vec);
            if constexpr (FORM == kCeF32) {
                *reinterpret_cast<f4*>(out + 2 * c) = v;
                continue;
            }
            u16x4 hi, lo;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                if constexpr (FORM == kCeBf16) {
                    hi[q] = float_to_bf16(v[q]);
                } else {
                    const float x = v[q] * scale;
                    hi[q] = float_to_half(x);
                    lo[q] = float_to_half(x - half_to_float(hi[q]));
                }
            }
            if constexpr (FORM == kCeHalves) {
                u16* at = out + ((c >> 5) << 6) + (c & 31);
                *reinterpret_cast<u16x4*>(at) = hi;
                *reinterpret_cast<u16x4*>(at + 32) = lo;
            } else {
                *reinterpret_cast<u16x4*>(out + c) = hi;
            }
        }
    }
}

// w as the logits take it and transposed, as dh does (one half; a k-contiguous operand
// gives the matrix cores 9% more than a k-strided one, and quarters past dim take
// none): 64 words by up to 256 columns a work-group.  50257 x 768 bf16: 47 us, 4.9
// TB/s; dh and dw of 8192 tokens 1.17 -> 1.09 ms by it.
__global__ __launch_bounds__(256) void k_both(CePlan p, CeBuffers b, int parts) {
    __shared__ u16 tile[64][64 + 4];
    Scalars* s = reinterpret_cast<Scalars*>(b.workspace + p.scalars);
    uint32_t top = 0;
    for (int q = threadIdx.x; q < parts; q += 256) top = max(top, s->parts[1][q]);
    top = largest_of_group(top);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) s->w_max = top;
    const float scale = ldexpf(1.f, exponent_for(top));
    const int v0 = blockIdx.x * 64, four = (threadIdx.x & 15) * 4;
    u16* w = reinterpret_cast<u16*>(b.workspace + p.w);
    u16* wt = reinterpret_cast<u16*>(b.workspace + p.wt);
    for (int d0 = blockIdx.y * 256; d0 < min(static_cast<int>(blockIdx.y + 1) * 256, static_cast<int>(p.ld_w)); d0 += 64) {
        f4 in[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int v = v0 + k * 16 + (threadIdx.x >> 4), d = d0 + four;
            in[k] = f4{0.f, 0.f, 0.f, 0.f};
            if (v < p.vocab && d < p.dim) in[k] = load4<false>(b.w, v * b.w_stride + d, p.dim - d, b.w_vector);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = k * 16 + (threadIdx.x >> 4);
            u16x4 x;
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = float_to_half(in[k][q] * scale);
            if (v0 + r < p.vocab) *reinterpret_cast<u16x4*>(w + (v0 + r) * p.ld_w + d0 + four) = x;
            *reinterpret_cast<u16x4*>(&tile[r][four]) = x;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = k * 16 + (threadIdx.x >> 4);
            u16x4 x;
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = tile[four + q][r];
            if (d0 + r < p.dim) *reinterpret_cast<u16x4*>(wt + (d0 + r) * p.ld_wt + v0 + four) = x;
        }
        __syncthreads();
    }
}

// Work-groups go to the XCDs in turn; every XCD gets one run of the tiles in
// order, so that the tiles that share rows share an L2.
__device__ __forceinline__ int xcd_run(int b, int total) {
    const int x = b & 7, q = total >> 3, r = total & 7;
    return x * q + min(x, r) + (b >> 3);
}

// Tiles of TM tokens: with the vocabulary (or dim) side by side 256 or 128 of it,
// and, for products summed over the tokens, squares of 256 or 128.
template <CeForm FORM, int TM, tile::Kind KI, tile::Kind KJ>
struct TokenTile {
    using T = tile::Tile<elem(FORM), TM, 128, 1, 4, TM == 32 ? 4 : 3, KI, KJ>;
};
template <CeForm FORM, tile::Kind KI, tile::Kind KJ>
struct TokenTile<FORM, 128, KI, KJ> {
    using T = tile::Pick<elem(FORM), 128, KI, KJ>;
};
template <CeForm FORM, tile::Kind KI, tile::Kind KJ>
struct TokenTile<FORM, 256, KI, KJ> {
    using T = tile::Pick<elem(FORM), 256, KI, KJ>;
};
__host__ __device__ constexpr int square_of(int tm) { return tm == 256 ? 256 : 128; }
constexpr int threads_of(int tm) { return tm >= 128 ? 512 : 256; }

__device__ __forceinline__ Operand h_rows(const CePlan& p, const CeBuffers& b) {
    if (b.h_direct)
        return Operand{static_cast<const u16*>(b.h), p.form == kCeF32 ? 2 * b.h_stride : b.h_stride, p.tokens,
                       static_cast<int32_t>(p.ld_h)};
    return Operand{reinterpret_cast<const u16*>(b.workspace + p.h), p.ld_h, (p.tokens + 63) / 64 * 64,
                   static_cast<int32_t>(p.ld_h)};
}
__device__ __forceinline__ Operand w_rows(const CePlan& p, const CeBuffers& b, int first) {
    const u16* w = b.w_direct ? static_cast<const u16*>(b.w) : reinterpret_cast<const u16*>(b.workspace + p.w);
    const int64_t ld = !b.w_direct ? p.ld_w : p.form == kCeF32 ? 2 * b.w_stride : b.w_stride;
    return Operand{w + first * ld, ld, p.vocab - first, static_cast<int32_t>(p.ld_w)};
}

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;

// What brings a tile's accumulators to logits in units of log2: a positive normal
// number, so that logits of -inf (the columns past the vocabulary) stay -inf, and 0 stays
// 0, where h and w are both tiny or both huge.  (Accumulators stay below 2^46: times
// 2^-126 nothing is left of them beside 1, as of the logits they stand for.)
__device__ __forceinline__ float logit_unit(CeForm form, const CePlan& p, const CeBuffers& b) {
    if (!is_scaled(form)) return kLog2e;
    const Scalars* s = reinterpret_cast<const Scalars*>(b.workspace + p.scalars);
    return ldexpf(kLog2e, max(-126, min(126, -(exponent_for(s->h_max) + exponent_for(s->w_max)))));
}

// What logits are taken relative to, at least the largest or a reference, and the sum
// of exp2(z2 - that) over all but the targets, of two sets of logits.
__device__ __forceinline__ float2 joined(float2 a, float2 c) {
    const float top = fmaxf(a.x, c.x);
    if (top == -__builtin_inff()) return make_float2(top, a.y + c.y);
    return make_float2(top, a.y * __builtin_amdgcn_exp2f(a.x - top) + c.y * __builtin_amdgcn_exp2f(c.x - top));
}

// The logits' tiles in order: eight rows of tokens side by side, along the
// vocabulary, so that the 32 tiles that an XCD has at once share 8 tiles of h and 4
// of w.  (With every token's tile in turn, 8192 tokens, h went through each L2 again
// for every tile of w; so, 1.0 GB come from beyond the L2s at 50257 x 768.)
__device__ __forceinline__ void logit_tile(int id, int tiles_t, int tiles_v, int* tt, int* tv) {
    constexpr int kRows = 8;
    const int group = id / (kRows * tiles_v), rows = min(kRows, tiles_t - group * kRows);
    id -= group * kRows * tiles_v;
    *tv = id / rows;
    *tt = group * kRows + id - *tv * rows;
}

// Eight neighbouring entries of a row of G, or of what is kept in its place.
template <CeForm FORM>
__device__ __forceinline__ void store_g(const CePlan& p, u16* row, int at, const float (&v)[8]) {
    if constexpr (FORM == kCeF32) {
        float* out = reinterpret_cast<float*>(row) + at;
        *reinterpret_cast<f4*>(out) = f4{v[0], v[1], v[2], v[3]};
        *reinterpret_cast<f4*>(out + 4) = f4{v[4], v[5], v[6], v[7]};
    } else {
        u16x8 hi, lo;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            if constexpr (FORM == kCeBf16) {
                hi[r] = float_to_bf16(v[r]);
                lo[r] = float_to_bf16(v[r] - bf16_to_float(hi[r]));
            } else {
                hi[r] = float_to_half(v[r]);
                lo[r] = float_to_half(v[r] - half_to_float(hi[r]));
            }
        }
        u16* out = row + (FORM == kCeHalves ? ((at >> 5) << 6) + (at & 31) : at);
        *reinterpret_cast<u16x8*>(out) = hi;
        if constexpr (FORM == kCeHalves) *reinterpret_cast<u16x8*>(out + 32) = lo;
        if constexpr (FORM == kCeBf16) *reinterpret_cast<u16x8*>(out + p.p_lo) = lo;
    }
}
template <CeForm FORM>
__device__ __forceinline__ void load_g(const CePlan& p, const u16* row, int at, float (&v)[8]) {
    if constexpr (FORM == kCeF32) {
        const float* in = reinterpret_cast<const float*>(row) + at;
        const f4 a = *reinterpret_cast<const f4*>(in), b = *reinterpret_cast<const f4*>(in + 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            v[r] = a[r];
            v[4 + r] = b[r];
        }
    } else {
        const u16* in = row + (FORM == kCeHalves ? ((at >> 5) << 6) + (at & 31) : at);
        const u16x8 hi = *reinterpret_cast<const u16x8*>(in);
        u16x8 lo = {};
        if constexpr (FORM == kCeHalves) lo = *reinterpret_cast<const u16x8*>(in + 32);
        if constexpr (FORM == kCeBf16) lo = *reinterpret_cast<const u16x8*>(in + p.p_lo);
#pragma unroll
        for (int r = 0; r < 8; ++r) {
            v[r] = FORM == kCeBf16 ? bf16_to_float(hi[r]) : half_to_float(hi[r]);
            if constexpr (FORM == kCeHalves) v[r] += half_to_float(lo[r]);
            if constexpr (FORM == kCeBf16) v[r] += bf16_to_float(lo[r]);
        }
    }
}

// Which of the four columns of waves has column j of a tile.
__device__ __forceinline__ int wave_of(int j) { return (j >> 5) & 3; }

// Exponentials relative to a largest one are kept times two to this: fp16's upper
// range.
template <CeForm FORM>
constexpr int kKept = is_scaled(FORM) ? 14 : 0;

// References: lse_t may pass r_t by 2^room and lie 2^kLow below it, so exp(z - r_t) is
// kept times 2^k, k = 15 - room: of c_t, entries of G keep what is above 2^-34 (one half:
// rows whose sample misses a word of up to 15/16 of the sum stay in range) or 2^-36
// (two halves; 3/4 of it).
constexpr int kLow = 2;
__host__ __device__ constexpr int room(CeForm f) { return f == kCeHalves ? 2 : 4; }
__host__ __device__ constexpr int shift(CeForm f) { return 15 - room(f); }
__host__ __device__ constexpr float pow2(int e) { return e < 0 ? 1.f / static_cast<float>(1 << -e) : static_cast<float>(1 << e); }
// s_t is at most c_t 2^(kLow + room - 15), so s_t h_t is taken times this and the powers
// of two that bring the largest c and h to 2^15: at most 2^15.
constexpr int turned(CeForm f) { return -kLow - room(f); }

// First pass: each row's largest logit and sum of exp(z - largest) in a tile, without the
// target's, and the target's logit.  KEEP also writes the exponentials in G's place for
// the first piece, relative to the largest logit of a wave's columns of the tile
// (wave_of), or to the row's reference, and what they are relative to.  Of the tile
// columns from `skip` on tiles_v are taken, one of every `every`, into slots from `slot`;
// `done` tiles were taken by launches before this one.
//
// Many tokens, bf16: 8192 of 50257 x 768 in 0.81 ms, 0.78 PFLOP/s.  Of a tile's 32 us
// the products take 18 (1.44 PFLOP/s), the writes of exponentials 6 (at 5.7 TB/s; one
// work-group fills a CU, so nothing runs beside them), exponentials, sums and the start
// of the next tile 8: the matrix cores are busy 42% of the time, at 2.0 GHz.  One token
// reads w, 77 MB, in 15 us at 5.1 TB/s; tiles of 32 tokens by 128 words with four stages
// on their way fill two work-groups a CU for that.
template <CeForm FORM, int TM, bool KEEP>
__global__ __launch_bounds__(threads_of(TM)) void k_stats(CePlan p, CeBuffers b, int tiles_v, int every, int skip,
                                                          int slot, int done) {
    using T = typename TokenTile<FORM, TM, kContig, kContig>::T;
    constexpr int TN = T::kBN;
    __shared__ __align__(1024) char lds[T::kLdsBytes];
    const int tiles_t = (p.tokens + TM - 1) / TM;
    int tt, at;
    logit_tile(done + xcd_run(blockIdx.x, gridDim.x), tiles_t, tiles_v, &tt, &at);
    const int tv = skip + at * every;
    T t;
    t.clear();
    t.add(h_rows(p, b), w_rows(p, b, 0), tt * TM, tv * TN, 0, static_cast<int>(p.ld_h / units(FORM)),
          (DSM_LDS char*)lds, p.tokens - tt * TM, p.vocab - tv * TN);
    // In units of log2: z2 = acc * unit, exp(z) = exp2(z2).
    const float unit = logit_unit(FORM, p, b);
    float* hit = reinterpret_cast<float*>(b.workspace + p.hit);
    float2* part = reinterpret_cast<float2*>(lds);  // [T::WN][TM]
    u16* g = reinterpret_cast<u16*>(b.workspace + p.p) + (tt * TM + t.row(0)) * p.ld_p;
    float* tops = reinterpret_cast<float*>(b.workspace + p.tops);
    const bool keep = KEEP && tv * TN < p.piece;
    int rel[T::FI];  // the target's column in the tile, or -1
    float ref[T::FI];
#pragma unroll
    for (int fi = 0; fi < T::FI; ++fi) {
        const int token = tt * TM + t.row(fi);
        const int64_t target = b.target[min(token, p.tokens - 1)];
        rel[fi] = token < p.tokens && is_valid(target, p.vocab) ? static_cast<int>(target) - tv * TN : -1;
        ref[fi] = -__builtin_inff();
        if (KEEP && p.sample > 0) ref[fi] = reinterpret_cast<const float*>(b.workspace + p.refs)[min(token, p.tokens - 1)];
    }
    if (tv * TN + TN > p.vocab) {  // columns past the vocabulary
#pragma unroll
        for (int fj = 0; fj < T::FJ; ++fj)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (tv * TN + t.col(fj) + r >= p.vocab)
#pragma unroll
                    for (int fi = 0; fi < T::FI; ++fi) t.acc[fi][fj][r] = -__builtin_inff();
    }
    // The rows' largest logits, all before the first store: one wait for the exchange.
    float top[T::FI];
#pragma unroll
    for (int fi = 0; fi < T::FI; ++fi) {
        top[fi] = t.acc[fi][0][0];
#pragma unroll
        for (int fj = 0; fj < T::FJ; ++fj)
#pragma unroll
            for (int r = 0; r < 4; ++r) top[fi] = fmaxf(top[fi], t.acc[fi][fj][r]);
    }
#pragma unroll
    for (int w = 16; w <= 32; w *= 2)
#pragma unroll
        for (int fi = 0; fi < T::FI; ++fi) top[fi] = fmaxf(top[fi], __shfl_xor(top[fi], w));
    float sum[T::FI], kept[T::FI];
#pragma unroll
    for (int fi = 0; fi < T::FI; ++fi) {
        const int token = tt * TM + t.row(fi);
        // Few waves hold a target's column.
        if (__any(rel[fi] >= 0 && rel[fi] < TN && wave_of(rel[fi]) == t.wj)) {
#pragma unroll
            for (int fj = 0; fj < T::FJ; ++fj)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (rel[fi] == t.col(fj) + r) {
                        hit[token] = t.acc[fi][fj][r];
                        t.acc[fi][fj][r] = -__builtin_inff();
                    }
        }
        top[fi] *= unit;
        // All logits -inf: no exponential counts (and -inf - -inf is none).
        const bool none = top[fi] == -__builtin_inff();
        const bool near = KEEP && is_scaled(FORM) && top[fi] - ref[fi] <= room(FORM);
        const float from = near ? ref[fi] : none ? 0.f : top[fi], by = near ? pow2(shift(FORM)) : pow2(kKept<FORM>);
        top[fi] = none ? top[fi] : from;
        kept[fi] = from;
        sum[fi] = 0.f;
        if (keep) {
#pragma unroll
            for (int q = 0; q < T::FJ / 2; ++q) {
                const tile::Eight z = t.eight(fi, q);
                float e[8];
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z.v[r], unit, -from));
                    sum[fi] += e[r];
                }
                if constexpr (is_scaled(FORM)) {
#pragma unroll
                    for (int r = 0; r < 8; ++r) e[r] *= by;
                }
                if (token < p.tokens)
                    store_g<FORM>(p, g + (t.row(fi) - t.row(0)) * p.ld_p, tv * TN + t.col8(q), e);
            }
        } else {
#pragma unroll
            for (int fj = 0; fj < T::FJ; ++fj)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    sum[fi] += __builtin_amdgcn_exp2f(__builtin_fmaf(t.acc[fi][fj][r], unit, -from));
        }
    }
#pragma unroll
    for (int w = 16; w <= 32; w *= 2)
#pragma unroll
        for (int fi = 0; fi < T::FI; ++fi) sum[fi] += __shfl_xor(sum[fi], w);
    if (t.lane < 16) {
#pragma unroll
        for (int fi = 0; fi < T::FI; ++fi) {
            const int token = tt * TM + t.row(fi);
            part[t.wj * TM + t.row(fi)] = make_float2(top[fi], sum[fi]);
            if (keep && token < p.tokens)
                tops[static_cast<int64_t>(token) * (p.piece / TN * 4) + tv * 4 + t.wj] = kept[fi];
        }
    }
    __syncthreads();
    float2* stats = reinterpret_cast<float2*>(b.workspace + p.stats) + static_cast<int64_t>(slot + at) * p.tokens;
    for (int r = threadIdx.x; r < TM; r += T::kThreads) {
        if (tt * TM + r >= p.tokens) break;
        float2 a = part[r];
#pragma unroll
        for (int w = 1; w < T::WN; ++w) a = joined(a, part[w * TM + r]);
        stats[tt * TM + r] = a;
    }
}

// The rows' references, from the sampled tiles: 16 tokens a work-group, 16 lanes each.
// A target in the sample counts once, the other words for those that are not in it.
__global__ __launch_bounds__(256) void k_refs(CePlan p, CeBuffers b) {
    __shared__ float2 part[16][16];
    const int lane = threadIdx.x & 15, share = threadIdx.x >> 4;
    const int token = blockIdx.x * 16 + lane;
    const float2* stats = reinterpret_cast<const float2*>(b.workspace + p.stats) + min(token, p.tokens - 1);
    float2 a = make_float2(-__builtin_inff(), 0.f);
#pragma unroll 4
    for (int v = share; v < p.sample; v += 16) a = joined(a, stats[static_cast<int64_t>(v) * p.tokens]);
    part[share][lane] = a;
    __syncthreads();
    if (share != 0 || token >= p.tokens) return;
#pragma unroll
    for (int q = 1; q < 16; ++q) a = joined(a, part[q][lane]);
    const float all = static_cast<float>(p.vocab) / (p.sample * 256.f);
    const int64_t target = b.target[token], column = target / 256;
    float own = 0.f;
    if (is_valid(target, p.vocab) && column % p.every == 0 && column / p.every < p.sample)
        own = __builtin_amdgcn_exp2f(
            __builtin_fmaf(reinterpret_cast<const float*>(b.workspace + p.hit)[token], logit_unit(p.form, p, b), -a.x));
    const float ref = a.x + __builtin_amdgcn_logf(a.y * all + own);
    reinterpret_cast<float*>(b.workspace + p.refs)[token] = fabsf(ref) < __builtin_inff() ? ref : -__builtin_inff();
}

// The weighted total, in a fixed order, by one work-group.
template <int N>
__device__ __forceinline__ void total_loss(const CePlan& p, const CeBuffers& b) {
    __shared__ double s[N];
    __shared__ int count;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    int mine = 0;
#pragma unroll 8
    for (int t = threadIdx.x; t < p.tokens; t += N) mine += is_valid(b.target[t], p.vocab);
    atomicAdd(&count, mine);
    __syncthreads();
    double sum = 0.0;
#pragma unroll 8
    for (int t = threadIdx.x; t < p.tokens; t += N)
        sum += is_valid(b.target[t], p.vocab) ? static_cast<double>(coefficient(b, t, count)) * b.loss[t] : 0.0;
    s[threadIdx.x] = sum;
    __syncthreads();
    for (int w = N / 2; w > 0; w >>= 1) {
        if (static_cast<int>(threadIdx.x) < w) s[threadIdx.x] += s[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0) b.total[0] = static_cast<float>(s[0]);
}
__global__ __launch_bounds__(1024) void k_total(CePlan p, CeBuffers b) { total_loss<1024>(p, b); }

// The kept exponentials become G of the first piece, eight columns a lane; with
// references, E: there only the target's entry changes, and rows that do not fit.  A
// work-group past the rows' sums the total, which would take a launch of its own.
template <CeForm FORM>
__global__ __launch_bounds__(256) void k_settle(CePlan p, CeBuffers b, int groups_of_row) {
    const int token = blockIdx.x / groups_of_row, first = blockIdx.x - token * groups_of_row;
    if (token >= p.tokens) {
        total_loss<256>(p, b);
        return;
    }
    const float lse = reinterpret_cast<const float*>(b.workspace + p.lse)[token];
    const int64_t target = b.target[token];
    const bool valid = is_valid(target, p.vocab);
    u16* g = reinterpret_cast<u16*>(b.workspace + p.p) + token * p.ld_p;
    const int square = square_of(p.tile);
    const float* tops = reinterpret_cast<const float*>(b.workspace + p.tops) + static_cast<int64_t>(token) * (p.piece / square * 4);
    // G is exp(z - lse) mul, the target's entry p - 1 = expm1(-loss) of it.
    float mul, ref = -__builtin_inff();
    if (is_scaled(FORM) && p.sample > 0) {
        ref = reinterpret_cast<const float*>(b.workspace + p.refs)[token];
        mul = pow2(shift(FORM));
        if (reinterpret_cast<const float2*>(b.workspace + p.rows)[token].x == ref) {
            if (threadIdx.x != 0 || !valid || target >= p.piece) return;
            const int at = static_cast<int>(target) & ~7;
            float v[8];
            load_g<FORM>(p, g, at, v);
            const float e = mul * __builtin_amdgcn_exp2f(lse - ref) * expm1f(-b.loss[token]);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (target == at + r) v[r] = e;
            store_g<FORM>(p, g, at, v);
            return;
        }
    } else {
        const int eg = !is_scaled(FORM) ? 0 : exponent_for(reinterpret_cast<const Scalars*>(b.workspace + p.scalars)->c_max);
        mul = ldexpf(reinterpret_cast<const float*>(b.workspace + p.coef)[token], eg);
    }
    for (int at = (first * 256 + threadIdx.x) * 8; at < p.piece; at += groups_of_row * 2048) {
        float v[8];
        load_g<FORM>(p, g, at, v);
        const float from = tops[at / square * 4 + wave_of(at)];
        const float by = mul * (from == ref ? pow2(-shift(FORM)) : pow2(-kKept<FORM>)) * __builtin_amdgcn_exp2f(from - lse);
#pragma unroll
        for (int r = 0; r < 8; ++r) v[r] = valid ? v[r] * by : 0.f;
        if (valid && target >= at && target < at + 8) {
            const float e = mul * expm1f(-b.loss[token]);
#pragma unroll
            for (int r = 0; r < 8; ++r)
                if (target == at + r) v[r] = e;
        }
        store_g<FORM>(p, g, at, v);
    }
}

// s_t h_t transposed, as dw takes it (a k-contiguous operand, which LDS gives at twice
// the rate): 8192 x 768 in 8 us.  64 tokens by 64 columns a work-group, zeros for
// tokens past the last one and those without a valid target.
template <CeForm FORM>
__global__ __launch_bounds__(256) void k_turn(CePlan p, CeBuffers b) {
    __shared__ float tile[64][65];
    const int t0 = blockIdx.x * 64, d0 = blockIdx.y * 64;
    const Scalars* sc = reinterpret_cast<const Scalars*>(b.workspace + p.scalars);
    const int es = exponent_for(sc->c_max) + turned(FORM);
    const u16* h = reinterpret_cast<const u16*>(b.workspace + p.h);
    const float2* rows = reinterpret_cast<const float2*>(b.workspace + p.rows);
    const int four = (threadIdx.x & 15) * 4;  // of a row's columns, then of its tokens
#pragma unroll
    for (int r = threadIdx.x >> 4; r < 64; r += 16) {
        const int token = t0 + r, d = d0 + four;
        f4 v = {0.f, 0.f, 0.f, 0.f};
        if (token < p.tokens && is_valid(b.target[token], p.vocab)) {
            const u16* at = h + token * p.ld_h + (FORM == kCeHalves ? ((d >> 5) << 6) + (d & 31) : d);
            const u16x4 hi = *reinterpret_cast<const u16x4*>(at);
            u16x4 lo = {};
            if constexpr (FORM == kCeHalves) lo = *reinterpret_cast<const u16x4*>(at + 32);
            const float by = ldexpf(rows[token].y, es);
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[q] = (FORM == kCeHalves ? half_to_float(hi[q]) + half_to_float(lo[q]) : half_to_float(hi[q])) * by;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) tile[r][four + q] = v[q];
    }
    __syncthreads();
    u16* ht = reinterpret_cast<u16*>(b.workspace + p.ht);
#pragma unroll
    for (int r = threadIdx.x >> 4; r < 64; r += 16) {
        const int d = d0 + r, token = t0 + four;
        if (d >= p.dim) break;
        u16x4 hi, lo;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float v = tile[four + q][r];
            hi[q] = float_to_half(v);
            lo[q] = float_to_half(v - half_to_float(hi[q]));
        }
        u16* at = ht + d * p.ld_ht + (FORM == kCeHalves ? ((token >> 5) << 6) + (token & 31) : token);
        *reinterpret_cast<u16x4*>(at) = hi;
        if constexpr (FORM == kCeHalves) *reinterpret_cast<u16x4*>(at + 32) = lo;
    }
}

// lse and loss of 16 tokens by a work-group: 64 lanes share a token's tiles, for which
// it waits (8192 tokens by 197 tiles: 10 us).  With
// one work-group it sums the total as well.
constexpr int kJoinTokens = 16;
__global__ __launch_bounds__(1024) void k_join(CePlan p, CeBuffers b, int tiles) {
    __shared__ float2 part[64][kJoinTokens];
    const int lane = threadIdx.x % kJoinTokens, share = threadIdx.x / kJoinTokens;
    const int token = blockIdx.x * kJoinTokens + lane, at = min(token, p.tokens - 1);
    const float2* stats = reinterpret_cast<const float2*>(b.workspace + p.stats) + at;
    float2 a = make_float2(-__builtin_inff(), 0.f);
#pragma unroll 4
    for (int v = share; v < tiles; v += 64) a = joined(a, stats[static_cast<int64_t>(v) * p.tokens]);
    part[share][lane] = a;
    __syncthreads();
    for (int w = 32; w > 0; w >>= 1) {
        if (share < w) part[share][lane] = joined(part[share][lane], part[share + w][lane]);
        __syncthreads();
    }
    if (share != 0) return;
    a = part[0][lane];
    const bool valid = token < p.tokens && is_valid(b.target[at], p.vocab);
    // The target's logit over what the sum is relative to, in one rounding.  (-inf over
    // -inf is NaN: a row without a logit has no loss, and its sum is 0.)
    const float hit = reinterpret_cast<const float*>(b.workspace + p.hit)[at];
    float over = __builtin_fmaf(hit, logit_unit(p.form, p, b), -a.x);
    if (!(fabsf(a.x) < __builtin_inff())) over = hit - a.x;
    const float own = valid && a.x != -__builtin_inff() ? exp2f(over) : 0.f;
    const float sum2 = log2f(a.y + own), lse2 = a.x + sum2, odds = a.y * exp2f(-over);
    const float loss = !valid ? 0.f : odds < 1.f ? log1pf(odds) : (sum2 - over) * kLn2;
    if (token < p.tokens) {
        reinterpret_cast<float*>(b.workspace + p.lse)[token] = lse2;
        if (b.lse) b.lse[token] = valid ? lse2 * kLn2 : 0.f;
        b.loss[token] = loss;
        if (p.sample > 0) {
            // In range of its reference, and every wave kept exponentials relative to it
            // (a larger logit elsewhere would be what the joined sum is relative to).
            const float ref = reinterpret_cast<const float*>(b.workspace + p.refs)[token];
            const bool fits = a.x == ref && lse2 - ref <= room(p.form) && lse2 - ref >= -kLow;
            const float below = fits ? ref - lse2 : 0.f;
            reinterpret_cast<float2*>(b.workspace + p.rows)[token] = make_float2(
                fits ? ref : lse2, reinterpret_cast<const float*>(b.workspace + p.coef)[token] *
                                       __builtin_amdgcn_exp2f(below) * pow2(-shift(p.form)));
        }
    }
    if (gridDim.x > 1) return;
    const int count = __popcll(__ballot(valid));
    double sum = valid ? static_cast<double>(coefficient(b, at, count)) * loss : 0.0;
    for (int w = kJoinTokens / 2; w > 0; w >>= 1) sum += __shfl_xor(sum, w);
    if (lane == 0) b.total[0] = static_cast<float>(sum);
}

// G of one piece of the vocabulary, [first, first + cols), after the first: the logits
// computed again, at the rate of the first pass.
template <CeForm FORM, int TM>
__global__ __launch_bounds__(threads_of(TM)) void k_piece(CePlan p, CeBuffers b, int first, int cols) {
    using T = typename TokenTile<FORM, TM, kContig, kContig>::T;
    constexpr int TN = T::kBN;
    __shared__ __align__(1024) char lds[T::kLdsBytes];
    const int cols_pad = (cols + 63) / 64 * 64;
    const int tiles_t = (p.tokens + TM - 1) / TM, tiles_v = (cols + TN - 1) / TN;
    int tt, tv;
    logit_tile(xcd_run(blockIdx.x, tiles_t * tiles_v), tiles_t, tiles_v, &tt, &tv);
    T t;
    t.run(h_rows(p, b), w_rows(p, b, first), tt * TM, tv * TN, 0, static_cast<int>(p.ld_h / units(FORM)),
          (DSM_LDS char*)lds, p.tokens - tt * TM, cols - tv * TN);
    const float unit = logit_unit(FORM, p, b);
    const int eg = !is_scaled(FORM) ? 0 : exponent_for(reinterpret_cast<const Scalars*>(b.workspace + p.scalars)->c_max);
    const float* lse = reinterpret_cast<const float*>(b.workspace + p.lse);
    const float* coef = reinterpret_cast<const float*>(b.workspace + p.coef);
    u16* g = reinterpret_cast<u16*>(b.workspace + p.p) + (tt * TM + t.row(0)) * p.ld_p;
    // What the rows need, all loaded before the first store.  A row without a
    // valid target gets 0 throughout.  With references, E.
    const bool refs = is_scaled(FORM) && p.sample > 0;
    const float2* rows = reinterpret_cast<const float2*>(b.workspace + p.rows);
    int rel[T::FI];
    bool counts[T::FI];
    float l[T::FI], c[T::FI], less[T::FI];  // less: the target's entry, p - 1, before c
#pragma unroll
    for (int fi = 0; fi < T::FI; ++fi) {
        const int token = tt * TM + t.row(fi), at = min(token, p.tokens - 1);
        const int64_t target = b.target[at];
        const bool valid = token < p.tokens && is_valid(target, p.vocab);
        rel[fi] = valid ? static_cast<int>(target) - first - tv * TN : -1;
        const float x = refs ? rows[at].x : lse[at];
        counts[fi] = valid;
        l[fi] = x;
        c[fi] = refs ? pow2(shift(FORM)) : ldexpf(coef[at], eg);
        less[fi] = (refs ? __builtin_amdgcn_exp2f(lse[at] - x) : 1.f) * expm1f(-b.loss[at]);
    }
    const bool ragged = tv * TN + TN > cols;
#pragma unroll
    for (int fi = 0; fi < T::FI; ++fi) {
        const int token = tt * TM + t.row(fi);
        // Few waves hold a target's column.
        const bool hits = __any(rel[fi] >= 0 && rel[fi] < TN && wave_of(rel[fi]) == t.wj);
        if (token >= p.tokens) continue;
#pragma unroll
        for (int q = 0; q < T::FJ / 2; ++q) {
            const int col = t.col8(q);
            const tile::Eight z = t.eight(fi, q);
            float v[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) v[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(z.v[r], unit, -l[fi]));
            if (hits) {
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (rel[fi] == col + r) v[r] = less[fi];
            }
            const int at = tv * TN + col;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                v[r] = counts[fi] ? v[r] * c[fi] : 0.f;
                if (ragged && at + r >= cols) v[r] = 0.f;
            }
            if (at < cols_pad) store_g<FORM>(p, g + (t.row(fi) - t.row(0)) * p.ld_p, at, v);
        }
    }
}

// G of the piece as an operand of its products; in the bf16 form its upper halves
// or (LO) its lower ones.  (Where a product runs over the tokens, those past the
// last one meet h's rows of zeros.)
template <bool LO = false>
__device__ __forceinline__ Operand g_rows(const CePlan& p, const CeBuffers& b) {
    return Operand{reinterpret_cast<const u16*>(b.workspace + p.p) + (LO ? p.p_lo : 0), p.ld_p, p.tokens,
                   static_cast<int32_t>(p.ld_p)};
}

// dh's sums over one piece, each of dh_splits parts into its own fp32 buffer: dh has few
// tiles (96 of 256 x 256 for 8192 x 768), whose sums run over the whole vocabulary.
// Tiles of the products of G: NARROW ones (of 256, whose last 128 columns lie past dim)
// are types of their own, for loops beside each other in one tile spill registers.  fp32,
// 600 tokens of 20000 x 100: 105 -> 96 us; bf16, 2048 of 50257 x 384: 429 -> 420.
template <CeForm FORM, int TM, tile::Kind KI, tile::Kind KJ, bool NARROW>
struct GradTile {
    using T = typename TokenTile<FORM, TM, KI, KJ>::T;
};
template <tile::Elem E, tile::Kind KI, tile::Kind KJ, bool NARROW>
using BigGradTile = tile::BigTile<E, KI, KJ, false, NARROW>;
template <tile::Kind KI, tile::Kind KJ, bool NARROW>
struct GradTile<kCeHalf, 256, KI, KJ, NARROW> {
    using T = BigGradTile<elem(kCeHalf), KI, KJ, NARROW>;
};
template <tile::Kind KI, tile::Kind KJ, bool NARROW>
struct GradTile<kCeHalves, 256, KI, KJ, NARROW> {
    using T = BigGradTile<elem(kCeHalves), KI, KJ, NARROW>;
};

template <CeForm FORM, int TM, bool TURNED, bool NARROW = false>
using DhTile = typename GradTile<FORM, TM, kContig, TURNED ? kContig : kStrided, NARROW>::T;

template <CeForm FORM, int TM, bool TURNED, bool NARROW>
__device__ __forceinline__ void dh_tile(const CePlan& p, const CeBuffers& b, int first, int cols, int id,
                                        DSM_LDS char* lds) {
    using T = DhTile<FORM, TM, TURNED, NARROW>;
    constexpr int TN = T::kBN;
    const int tiles_t = (p.tokens + TM - 1) / TM, tiles_d = (p.dim + TN - 1) / TN;
    const int part = id / (tiles_t * tiles_d);
    id -= part * tiles_t * tiles_d;
    const int tt = id / tiles_d, td = id - tt * tiles_d;
    const int cols_pad = (cols + 63) / 64 * 64;
    const int each = (cols_pad / 64 + p.dh_splits - 1) / p.dh_splits * 64;
    const int k0 = min(part * each, cols_pad), k1 = min(k0 + each, cols_pad);
    T t;
    t.clear();
    const Operand w = TURNED ? Operand{reinterpret_cast<const u16*>(b.workspace + p.wt) + first, p.ld_wt, p.dim,
                                       static_cast<int32_t>(p.ld_wt - first)}
                             : w_rows(p, b, first);
    t.add(g_rows(p, b), w, tt * TM, td * TN, k0, k1, lds, p.tokens - tt * TM, p.dim - td * TN);
    if constexpr (FORM == kCeBf16)
        t.add(g_rows<true>(p, b), w, tt * TM, td * TN, k0, k1, lds, p.tokens - tt * TM, p.dim - td * TN);
    float* out = reinterpret_cast<float*>(b.workspace + p.dh) + part * p.tokens * p.ld_dh;
    const int ld = static_cast<int>(p.ld_dh);
    constexpr int kBatch = T::FI < 4 ? T::FI : 4;
#pragma unroll
    for (int f0 = 0; f0 < T::FI; f0 += kBatch) {
        f4 old[kBatch][T::FJ];
#pragma unroll
        for (int fi = 0; fi < kBatch; ++fi)
#pragma unroll
            for (int fj = 0; fj < T::FJ; ++fj) {
                const int64_t q = static_cast<int64_t>(min(tt * TM + t.row(f0 + fi), p.tokens - 1)) * ld +
                                  min(td * TN + t.col(fj), ld - 4);
                old[fi][fj] = first == 0 ? f4{0.f, 0.f, 0.f, 0.f} : *reinterpret_cast<const f4*>(out + q);
            }
#pragma unroll
        for (int fi = 0; fi < kBatch; ++fi) {
            const int token = tt * TM + t.row(f0 + fi);
#pragma unroll
            for (int fj = 0; fj < T::FJ; ++fj) {
                const int d = td * TN + t.col(fj);
                if (token < p.tokens && d < ld)
                    *reinterpret_cast<f4*>(out + static_cast<int64_t>(token) * ld + d) = old[fi][fj] + t.acc[f0 + fi][fj];
            }
        }
    }
}

// Four entries of a gradient, of which `have` exist.
template <bool F32>
__device__ __forceinline__ void store_grad(void* base, int64_t at, f4 v, int have, bool vec) {
    if constexpr (F32) {
        float* p = static_cast<float*>(base) + at;
        if (vec && have >= 4) {
            *reinterpret_cast<f4*>(p) = v;
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < have) p[r] = v[r];
        }
    } else {
        u16* p = static_cast<u16*>(base) + at;
        u16x4 w;
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = float_to_bf16(v[r]);
        if (vec && have >= 4) {
            *reinterpret_cast<u16x4*>(p) = w;
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < have) p[r] = w[r];
        }
    }
}

// dh from its parts (8192 x 768: 24 us, 4 TB/s): 256 columns of a row by a work-group, whose four waves add a
// quarter of the parts each; the order is fixed.
template <CeForm FORM>
__global__ __launch_bounds__(256) void k_dh_join(CePlan p, CeBuffers b, int first) {
    __shared__ f4 sums[4][64];
    const Scalars* s = reinterpret_cast<const Scalars*>(b.workspace + p.scalars);
    const bool refs = is_scaled(FORM) && p.sample > 0;
    const int ex = is_scaled(FORM) ? -((refs ? 0 : exponent_for(s->c_max)) + exponent_for(s->w_max)) : 0;
    const int64_t each = p.tokens * p.ld_dh;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = first + blockIdx.y, d = blockIdx.x * 256 + lane * 4;
    const int quarter = (p.dh_splits + 3) / 4, q1 = min((wave + 1) * quarter, p.dh_splits);
    f4 v = {0.f, 0.f, 0.f, 0.f};
    if (d < p.dim) {
        const float* parts = reinterpret_cast<const float*>(b.workspace + p.dh) + row * p.ld_dh + d;
#pragma unroll 8
        for (int q = wave * quarter; q < q1; ++q) v += *reinterpret_cast<const f4*>(parts + q * each);
    }
    sums[wave][lane] = v;
    __syncthreads();
    if (wave != 0 || d >= p.dim) return;
    v = (v + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
    const float by = refs ? reinterpret_cast<const float2*>(b.workspace + p.rows)[row].y : 1.f;
    // (A row of zeros in G meets what w holds, NaN included.)
    const bool valid = is_valid(b.target[row], p.vocab);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = valid ? ldexpf(v[r], ex) * by : 0.f;
    store_grad<is_f32(FORM)>(b.dh, row * b.dh_stride + d, v, p.dim - d, b.dh_vector);
}

// dw of one piece; REFS: of E by s_t h_t transposed.
template <CeForm FORM, int TM, bool REFS, bool NARROW = false>
using DwTile = std::conditional_t<TM == 256, typename GradTile<FORM, 256, kStrided, REFS ? kContig : kStrided, NARROW>::T,
                                  tile::Pick<elem(FORM), square_of(TM), kStrided, kStrided>>;

template <CeForm FORM, int TM, bool REFS, bool NARROW>
__device__ __forceinline__ void dw_tile(const CePlan& p, const CeBuffers& b, int first, int cols, int id,
                                        DSM_LDS char* lds) {
    constexpr int BM = square_of(TM);
    using T = DwTile<FORM, TM, REFS, NARROW>;
    const int tiles_d = (p.dim + BM - 1) / BM;
    const int tv = id / tiles_d, td = id - tv * tiles_d;
    constexpr int kSteps = T::kSteps;
    const int rows_pad = (p.tokens + kSteps - 1) / kSteps * kSteps;
    const Operand h = REFS ? Operand{reinterpret_cast<const u16*>(b.workspace + p.ht), p.ld_ht, p.dim,
                                     static_cast<int32_t>(p.ld_ht)}
                           : h_rows(p, b);
    T t;
    t.clear();
    t.add(g_rows(p, b), h, tv * BM, td * BM, 0, rows_pad, lds, cols - tv * BM, p.dim - td * BM);
    if constexpr (FORM == kCeBf16)
        t.add(g_rows<true>(p, b), h, tv * BM, td * BM, 0, rows_pad, lds, cols - tv * BM, p.dim - td * BM);
    int ex = 0;
    if constexpr (is_scaled(FORM)) {
        const Scalars* s = reinterpret_cast<const Scalars*>(b.workspace + p.scalars);
        ex = -(exponent_for(s->c_max) + exponent_for(s->h_max) + (REFS ? turned(FORM) : 0));
    }
#pragma unroll
    for (int fi = 0; fi < T::FI; ++fi) {
        const int v = tv * BM + t.row(fi);
        if (v >= cols) continue;
#pragma unroll
        for (int q = 0; q < T::FJ / 2; ++q) {
            const int d = td * BM + t.col8(q);
            const tile::Eight x = t.eight(fi, q);
            f4 lo, hi;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                lo[r] = ldexpf(x.v[r], ex);
                hi[r] = ldexpf(x.v[4 + r], ex);
            }
            const int64_t at = (first + v) * b.dw_stride + d;
            if (d < p.dim) store_grad<is_f32(FORM)>(b.dw, at, lo, p.dim - d, b.dw_vector);
            if (d + 4 < p.dim) store_grad<is_f32(FORM)>(b.dw, at + 4, hi, p.dim - d - 4, b.dw_vector);
        }
    }
}

// The two products of G in one launch: neither fills the CUs' last turn by itself,
// and their tiles take different times.  Each XCD has its run of dh's tiles, the
// longer ones, then its run of dw's.  8192 tokens of 50257 x 768 in bf16: 1.09 ms, 1.16
// PFLOP/s, the matrix cores busy 69% of the time at 1.8 GHz; what bounds it is LDS, whose
// transposing reads of k-strided operands give half as much as plain ones, and the clock.
constexpr int kXcds = 8;
__host__ __device__ inline int per_xcd(int tiles) { return (tiles + kXcds - 1) / kXcds; }

template <CeForm FORM, int TM, bool REFS>
__global__ __launch_bounds__(threads_of(TM)) void k_gradients(CePlan p, CeBuffers b, int first, int cols,
                                                              int dh_tiles, int dw_tiles) {
    constexpr bool kTurned = REFS && FORM == kCeHalf;
    using TD = DhTile<FORM, TM, kTurned>;
    using TW = DwTile<FORM, TM, REFS>;
    constexpr int kLds = TD::kLdsBytes > TW::kLdsBytes ? TD::kLdsBytes : TW::kLdsBytes;
    __shared__ __align__(1024) char lds[kLds];
    const int x = blockIdx.x % kXcds, at = blockIdx.x / kXcds, front = per_xcd(dh_tiles);
    // Tile columns of dim, and those with more than 128 columns.
    const int tiles_d = (p.dim + square_of(TM) - 1) / square_of(TM), wide = (p.dim + 127) / 256;
    if (at < front) {
        const int id = x * front + at;
        if (id >= dh_tiles) return;
        if (TM == 256 && id % tiles_d >= wide)
            dh_tile<FORM, TM, kTurned, TM == 256>(p, b, first, cols, id, (DSM_LDS char*)lds);
        else
            dh_tile<FORM, TM, kTurned, false>(p, b, first, cols, id, (DSM_LDS char*)lds);
    } else {
        const int id = x * per_xcd(dw_tiles) + at - front;
        if (id >= dw_tiles) return;
        if (TM == 256 && id % tiles_d >= wide)
            dw_tile<FORM, TM, REFS, TM == 256>(p, b, first, cols, id, (DSM_LDS char*)lds);
        else
            dw_tile<FORM, TM, REFS, false>(p, b, first, cols, id, (DSM_LDS char*)lds);
    }
}

// Few tokens: one by one, their tiles being of different shapes.
template <CeForm FORM, int TM>
__global__ __launch_bounds__(threads_of(TM)) void k_dh(CePlan p, CeBuffers b, int first, int cols) {
    __shared__ __align__(1024) char lds[DhTile<FORM, TM, false>::kLdsBytes];
    dh_tile<FORM, TM, false, false>(p, b, first, cols, xcd_run(blockIdx.x, gridDim.x), (DSM_LDS char*)lds);
}
template <CeForm FORM, int TM>
__global__ __launch_bounds__(tile::threads_of(square_of(TM))) void k_dw(CePlan p, CeBuffers b, int first, int cols) {
    __shared__ __align__(1024) char lds[DwTile<FORM, TM, false>::kLdsBytes];
    dw_tile<FORM, TM, false, false>(p, b, first, cols, xcd_run(blockIdx.x, gridDim.x), (DSM_LDS char*)lds);
}

// No tokens: the total and dw are zero.
template <bool F32>
__global__ __launch_bounds__(256) void k_nothing(CePlan p, CeBuffers b) {
    if (blockIdx.x == 0 && threadIdx.x == 0) b.total[0] = 0.f;
    if (!p.grads) return;
    for (int r = blockIdx.x; r < p.vocab; r += gridDim.x)
        for (int c = threadIdx.x * 4; c < p.dim; c += 1024)
            store_grad<F32>(b.dw, r * b.dw_stride + c, f4{0.f, 0.f, 0.f, 0.f}, p.dim - c, b.dw_vector);
}

// A launch holds fewer than 2^32 threads, which 2^20 tokens by 2^19 words have.
constexpr int kMostGroups = 1 << 22;
template <CeForm FORM, int TM, bool KEEP>
void stats(const CePlan& p, const CeBuffers& b, int tiles_v, int every, int skip, int slot, hipStream_t stream) {
    const int tiles = (p.tokens + TM - 1) / TM * tiles_v;
    for (int done = 0; done < tiles; done += kMostGroups)
        k_stats<FORM, TM, KEEP><<<std::min(tiles - done, kMostGroups), threads_of(TM), 0, stream>>>(p, b, tiles_v, every, skip,
                                                                                                 slot, done);
}

template <CeForm FORM, int TM>
void products(const CePlan& p, const CeBuffers& b, hipStream_t stream) {
    constexpr int kThreads = threads_of(TM), TN = square_of(TM);
    constexpr bool kRefs = TM == 256 && is_scaled(FORM);  // rows may have references
    const int tt = (p.tokens + TM - 1) / TM, td = (p.dim + TN - 1) / TN, tv = (p.vocab + TN - 1) / TN;
    if constexpr (FORM != kCeBf16 || TM < 256) {  // (many tokens with gradients take fp16)
        if (p.grads) {
            if constexpr (kRefs) {
                if (p.sample > 0) {
                    stats<FORM, TM, false>(p, b, p.sample, p.every, 0, 0, stream);
                    k_refs<<<(p.tokens + 15) / 16, 256, 0, stream>>>(p, b);
                }
            }
            stats<FORM, TM, true>(p, b, tv, 1, 0, 0, stream);
        }
    }
    int slots = tv;
    if (!p.grads) {
        int front = tv;
        if constexpr (TM == 256) front = p.front;
        stats<FORM, TM, false>(p, b, front, 1, 0, 0, stream);
        if constexpr (TM == 256) {
            if (front < tv) {
                const int rest = (p.vocab - front * 256 + 127) / 128;
                stats<FORM, 128, false>(p, b, rest, 1, front * 2, front, stream);
                slots = front + rest;
            }
        }
    }
    k_join<<<(p.tokens + kJoinTokens - 1) / kJoinTokens, 1024, 0, stream>>>(p, b, slots);
    if (!p.grads && p.tokens > kJoinTokens) k_total<<<1, 1024, 0, stream>>>(p, b);
    if constexpr (FORM != kCeBf16 || TM < 256) {
        if (!p.grads) return;
        for (int first = 0; first < p.vocab; first += p.piece) {
            const int cols = p.vocab - first < p.piece ? p.vocab - first : p.piece;
            const int tp = (cols + TN - 1) / TN;
            if (first == 0) {
                // With references few rows change: one group each.
                const int groups = p.sample > 0 ? 1 : (p.piece + 2047) / 2048;
                k_settle<FORM><<<p.tokens * groups + (p.tokens > kJoinTokens), 256, 0, stream>>>(p, b, groups);
                if constexpr (kRefs) {
                    if (p.sample > 0)
                        k_turn<FORM><<<dim3((p.tokens + 63) / 64, (p.dim + 63) / 64), 256, 0, stream>>>(p, b);
                }
            } else {
                k_piece<FORM, TM><<<tt * tp, kThreads, 0, stream>>>(p, b, first, cols);
            }
            const int dh_tiles = tt * td * p.dh_splits, dw_tiles = tp * td;
            if constexpr (TM >= 128) {
                const int groups = kXcds * (per_xcd(dh_tiles) + per_xcd(dw_tiles));
                if (kRefs && p.sample > 0)
                    k_gradients<FORM, TM, kRefs><<<groups, kThreads, 0, stream>>>(p, b, first, cols, dh_tiles, dw_tiles);
                else
                    k_gradients<FORM, TM, false><<<groups, kThreads, 0, stream>>>(p, b, first, cols, dh_tiles, dw_tiles);
            } else {
                k_dh<FORM, TM><<<dh_tiles, kThreads, 0, stream>>>(p, b, first, cols);
                k_dw<FORM, TM><<<dw_tiles, tile::threads_of(TN), 0, stream>>>(p, b, first, cols);
            }
        }
        for (int row = 0; row < p.tokens; row += 32768)  // (a grid dimension holds 65535)
            k_dh_join<FORM><<<dim3((p.dim + 255) / 256, std::min(p.tokens - row, 32768)), 256, 0, stream>>>(p, b, row);
    }
}

}  // namespace

hipError_t launch_linear_ce(const CePlan& p, const CeBuffers& b, hipStream_t stream) {
    if (p.tokens == 0) {
        const unsigned rows = static_cast<unsigned>(p.grads ? std::min(p.vocab, 2048) : 1);
        if (is_f32(p.form))
            k_nothing<true><<<rows, 256, 0, stream>>>(p, b);
        else
            k_nothing<false><<<rows, 256, 0, stream>>>(p, b);
        return hipGetLastError();
    }
    const int most = b.w_direct || p.tokens > p.vocab ? p.tokens : p.vocab;
    const unsigned groups = static_cast<unsigned>(most < 8192 ? (most + 3) / 4 : 2048);
    const unsigned parts = std::min(groups, static_cast<unsigned>(kCeParts));
    switch (p.form) {
        case kCeBf16:
            if (!b.h_direct)
                k_operands<kCeBf16><<<dim3(groups + 1, b.w_direct ? 1 : 2), 256, 0, stream>>>(p, b, 0);
            if (p.tile == 32)
                products<kCeBf16, 32>(p, b, stream);
            else if (p.tile == 64)
                products<kCeBf16, 64>(p, b, stream);
            else if (p.tile == 128)
                products<kCeBf16, 128>(p, b, stream);
            else
                products<kCeBf16, 256>(p, b, stream);
            break;
        case kCeF32:
            if (!b.h_direct)
                k_operands<kCeF32><<<dim3(groups + 1, b.w_direct ? 1 : 2), 256, 0, stream>>>(p, b, 0);
            if (p.tile == 32)
                products<kCeF32, 32>(p, b, stream);
            else
                products<kCeF32, 64>(p, b, stream);
            break;
        case kCeHalf:
            k_largest<false><<<dim3(parts + 1, 2), 256, 0, stream>>>(p, b);
            k_operands<kCeHalf><<<dim3(groups, p.ld_wt ? 1 : 2), 256, 0, stream>>>(p, b, parts);
            if (p.ld_wt)
                k_both<<<dim3((p.vocab + 63) / 64, (p.dim + 255) / 256), 256, 0, stream>>>(p, b, parts);
            if (p.tile == 128)
                products<kCeHalf, 128>(p, b, stream);
            else
                products<kCeHalf, 256>(p, b, stream);
            break;
        case kCeHalves:
            k_largest<true><<<dim3(parts + 1, 2), 256, 0, stream>>>(p, b);
            k_operands<kCeHalves><<<dim3(groups, 2), 256, 0, stream>>>(p, b, parts);
            if (p.tile == 128)
                products<kCeHalves, 128>(p, b, stream);
            else
                products<kCeHalves, 256>(p, b, stream);
            break;
    }
    return hipGetLastError();
}

}  // namespace dsm
