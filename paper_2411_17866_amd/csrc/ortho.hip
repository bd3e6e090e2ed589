// Orthogonalised updates on gfx950: Newton-Schulz iteration on batches of
// matrices, with the momentum before it and the parameter update after it.
//
//   X = U / (||U||_F + eps);  then for each step, with A = X X^T,
//   B = b A + c A A,  X <- a X + B X
//
// on the wide orientation (m <= n), so A and B are m x m.  A step is three
// matrix products, m^2 n + m^3 + 2 m^2 n operations with the symmetry of A and
// of A A used: the two symmetric products compute the tiles on and below the
// diagonal and store each tile below it a second time, transposed.
//
// Precision.  Products accumulate in fp32.  fp32 matrices go through the
// products as two fp16 halves (gemm_tile.h: 22 bits, three matrix instructions),
// which keeps the result as near to 64-bit arithmetic as fp32 products do.
// bf16 matrices go through them as one fp16 (11 bits, against bf16's 8: the
// iteration multiplies small singular values by up to 3.4445^5 = 485, and with
// them what rounding X, A or B to 8 bits put there).  Two rules keep 11 bits
// enough: A is rounded once and that same A enters b A and c A A, and the term
// a X takes X from 22 bits (hi + lo), the products hi alone.  (With 14 bits there a
// rank of 5 over noise of 1e-4 is off by 0.3-0.7%; rounding the result to bf16 costs
// 0.17%, all of it in bf16 1-5%.)
//   Near the end all singular values are near 1, so A is near I and B near -2.5 I: their
// diagonals are most of what is rounded, and a X + B X nearly cancels.  So the diagonals
// D of A and E of B stay apart, in fp32, and with A' = A - D, B' = B - E
//   A A = A' A' + D A' + A' D + D D,   a X + B X = (a + E) X + B' X
// where the epilogues add what is not a product of matrices.  E X is part of a product
// that takes hi alone, and in an early iteration it has to take hi too: B X is 0 where X
// is small, and E X and B' X cancel there, with X's rounding on both sides or on neither.
// When what is left multiplies small singular values little (late), (a + E) X takes hi
// and lo.  Against 64 bits results are then off by 1.01-1.12 times what rounding them
// to bf16 costs; by 1.2-1.6 times with the diagonals inside (noise, orthogonal rows).
//   The fewer the singular values, the less their errors average: matrices small enough
// for LDS take two halves (bf16 64 x 48: 0.28% so, with one half; 0.17% with two).
//
// Range.  ||X||_2 <= 1 at the start, and the polynomial bounds it after each
// step, so the host picks for each stored operand the power of two that brings
// its bound just under fp16's largest number; entries then keep their bits down
// to 2^-40 of that bound.  Where eps outweighs the norm, X starts far below 1: it is
// then stored times 2^e, e its own for each matrix, with which b A and c A A lose
// 2^-2e and 2^-4e, and e falls with each iteration by what X can grow.
#include <hip/hip_runtime.h>

#include <cmath>

#include "gemm_tile.h"
#include "ops_internal.h"
#include "ortho_plan.h"

#pragma clang fp contract(off)

namespace dsm {
namespace {

using tile::Eight;
using tile::f4;
using tile::kContig;
using tile::kStrided;
using tile::Operand;

typedef unsigned short u16;
typedef u16 u16x4 __attribute__((ext_vector_type(4)));
typedef u16 u16x8 __attribute__((ext_vector_type(8)));

constexpr int kPad = 64;          // k of every operand is padded to this with zeros
constexpr int kNormParts = 256;   // partial sums of squares of a matrix, at most
constexpr int kPrepTile = 64;

__host__ __device__ inline int pad(int v) { return (v + kPad - 1) / kPad * kPad; }
__host__ __device__ inline int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

// Workspace of one matrix: the partial sums, two X, A and B.  A split operand
// keeps hi and lo interleaved in blocks of 32 columns (twice the columns); with
// one half, X's lo lies apart, where only the epilogue reads it.
struct Parts {
    int64_t x[2], a, b, bytes;
    int64_t lo;           // from an X to its lo half (one half only)
    int64_t diag_a, diag_b;  // diagonals of A and B in fp32 (one half only)
    __host__ __device__ Parts(int m, int n, bool split) {
        const int64_t xb = up256(static_cast<int64_t>(m) * pad(n) * 2) * 2;
        const int64_t ab = up256(static_cast<int64_t>(m) * pad(m) * 2 * (split ? 2 : 1));
        lo = xb / 2;
        x[0] = up256(kNormParts * 8 + 4);
        x[1] = x[0] + xb;
        a = x[1] + xb;
        b = a + ab;
        diag_a = b + ab;
        const int64_t db = split ? 0 : up256(static_cast<int64_t>(pad(m)) * 4);
        diag_b = diag_a + db;
        bytes = diag_b + db;
    }
};

__device__ __forceinline__ float from_bits(u16 v) {
    return static_cast<float>(__builtin_bit_cast(_Float16, v));
}
__device__ __forceinline__ u16 to_bits(float v) {
    return __builtin_bit_cast(u16, static_cast<_Float16>(v));
}
__device__ __forceinline__ float bf16_to_float(u16 v) {
    return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16);
}
__device__ __forceinline__ u16 float_to_bf16(float v) {
    return __builtin_bit_cast(u16, static_cast<__bf16>(v));
}

// Where element (i, j) of a stored operand lies; the lo half is 32 further.
template <int S>
__device__ __forceinline__ int64_t at(int64_t i, int j, int64_t ld) {
    return S == 1 ? i * ld + j : i * ld + ((j >> 5) << 6) + (j & 31);
}

// The update u = g + mu m, m, or the matrix itself, at four elements from e on
// (`have` of them exist); FIRST computes and stores the new momentum, which a
// later call reads.
template <bool STEP, bool BF16, bool FIRST>
__device__ __forceinline__ f4 update_at(const OrthoGroup& g, int64_t e, int have) {
    f4 v = {0.f, 0.f, 0.f, 0.f};
    if constexpr (BF16) {
        const u16* in = static_cast<const u16*>(g.in) + e;
        if (g.vector && have >= 4) {
            const u16x4 b = *reinterpret_cast<const u16x4*>(in);
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = bf16_to_float(b[r]);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < have) v[r] = bf16_to_float(in[r]);
        }
        return v;
    }
    const float* in = static_cast<const float*>(g.in) + e;
    const bool vec = g.vector && have >= 4;
    if (vec) {
        v = *reinterpret_cast<const f4*>(in);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < have) v[r] = in[r];
    }
    if constexpr (STEP) {
        if (!g.mom) return v;
        float* mom = g.mom + e;
        f4 m = {0.f, 0.f, 0.f, 0.f};
        if (vec) {
            m = *reinterpret_cast<const f4*>(mom);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (r < have) m[r] = mom[r];
        }
        if constexpr (FIRST) {
#pragma unroll
            for (int r = 0; r < 4; ++r) m[r] = g.mu * m[r] + v[r];
            if (vec) {
                *reinterpret_cast<f4*>(mom) = m;
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (r < have) mom[r] = m[r];
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = g.nesterov ? v[r] + g.mu * m[r] : m[r];
    }
    return v;
}

// Memory bounds it: twelve fp32 768 x 2304 with momentum in 51 us, 4.9 TB/s.
// Momentum and the partial sums of squares, in double so that no fp32 update
// overflows or vanishes in its square; a fixed order, so reruns give the same
// bits.  A work-group takes every n_parts-th row of a matrix, or, where rows are
// short, that run of them; four elements a lane.
template <bool STEP, bool BF16>
__global__ __launch_bounds__(256) void k_norm(OrthoGroup g, Parts parts, int n_parts) {
    const int rows = g.tall ? g.n : g.m, cols = g.tall ? g.m : g.n;
    const int64_t base = g.off.at[blockIdx.y];
    const int quads = (cols + 3) / 4;
    double sum = 0.0;
    // Lanes over (row, quad) pairs: lanes of a row side by side, rows to fill 256.
    const int per_row = quads < 256 ? quads : 256;
    const int rows_at_once = 256 / per_row;
    const int mine = threadIdx.x / per_row, q0 = threadIdx.x - mine * per_row;
    if (mine < rows_at_once) {
        for (int r = blockIdx.x * rows_at_once + mine; r < rows; r += n_parts * rows_at_once)
#pragma unroll 4
            for (int q = q0; q < quads; q += per_row) {
                const f4 v = update_at<STEP, BF16, true>(g, base + r * g.row_stride + q * 4, cols - q * 4);
                sum += static_cast<double>(v[0]) * v[0] + static_cast<double>(v[1]) * v[1] +
                       (static_cast<double>(v[2]) * v[2] + static_cast<double>(v[3]) * v[3]);
            }
    }
    __shared__ double s[256];
    s[threadIdx.x] = sum;
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
        if (static_cast<int>(threadIdx.x) < w) s[threadIdx.x] += s[threadIdx.x + w];
        __syncthreads();
    }
    if (threadIdx.x == 0)
        reinterpret_cast<double*>(static_cast<char*>(g.workspace) + blockIdx.y * parts.bytes)[blockIdx.x] = s[0];
}

// The power of two that brings norm / (norm + eps) into (1/2, 1].
__device__ __forceinline__ int lift_of(double norm, double eps) {
    const double share = norm / (norm + eps);
    return share > 0.0 && share < 0.5 ? -ilogb(share) - 1 : 0;
}
// 2^e / (norm + eps); zeros stay zeros where eps is 0 too.
__device__ __forceinline__ double inverse_of(double norm, double eps, int e) {
    const double size = norm + eps;
    return size == 0.0 ? 0.0 : ldexp(1.0 / size, e);
}
__host__ __device__ inline int64_t lift_at() { return kNormParts * 8; }  // bytes into a matrix's workspace

// X_0 in the stored form, wide, its padding zero: 64 x 64 of it per work-group, turned
// in LDS where the matrix is tall.  Memory bounds it: eight bf16 6400 x 1600 in 94 us,
// 4.4 TB/s.
template <int S, bool STEP, bool BF16>
__global__ __launch_bounds__(256) void k_start(OrthoGroup g, Parts parts, int n_parts, int x_exp) {
    __shared__ float t[kPrepTile][kPrepTile + 1];
    __shared__ double s[256];
    char* ws = static_cast<char*>(g.workspace) + blockIdx.z * parts.bytes;
    const double* p = reinterpret_cast<const double*>(ws);
    s[threadIdx.x] = static_cast<int>(threadIdx.x) < n_parts ? p[threadIdx.x] : 0.0;
    // Rows of memory: i of the wide orientation, or j where the matrix is tall.
    const int64_t base = g.off.at[blockIdx.z];
    const int i0 = blockIdx.y * kPrepTile, j0 = blockIdx.x * kPrepTile;
    const int r0 = g.tall ? j0 : i0, c0 = g.tall ? i0 : j0;
    const int rows = g.tall ? g.n : g.m, cols = g.tall ? g.m : g.n;
    const int c = threadIdx.x & 15;
    f4 v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = r0 + k * 16 + (threadIdx.x >> 4);
        const int have = r < rows ? cols - (c0 + c * 4) : 0;
        v[k] = have > 0 ? update_at<STEP, BF16, false>(g, base + r * g.row_stride + c0 + c * 4, have)
                        : f4{0.f, 0.f, 0.f, 0.f};
    }
    __syncthreads();
    for (int w = 128; w > 0; w >>= 1) {
        if (static_cast<int>(threadIdx.x) < w) s[threadIdx.x] += s[threadIdx.x + w];
        __syncthreads();
    }
    const double norm = sqrt(s[0]);
    const int lift = lift_of(norm, g.eps);
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *reinterpret_cast<int*>(ws + lift_at()) = lift;
    const double inv = inverse_of(norm, g.eps, x_exp + lift);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int r = k * 16 + (threadIdx.x >> 4);
            const float x = static_cast<float>(v[k][q] * inv);
            if (g.tall)
                t[c * 4 + q][r] = x;
            else
                t[r][c * 4 + q] = x;
        }
    __syncthreads();
    const int np = pad(g.n);
    u16* x = reinterpret_cast<u16*>(ws + parts.x[0]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = k * 16 + (threadIdx.x >> 4);
        const int i = i0 + r, j = j0 + c * 4;
        if (i >= g.m || j >= np) continue;
        u16x4 hi, lo;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float w = t[r][c * 4 + q];
            hi[q] = to_bits(w);
            lo[q] = to_bits(w - from_bits(hi[q]));
        }
        u16* to = x + at<S>(i, j, static_cast<int64_t>(np) * S);
        *reinterpret_cast<u16x4*>(to) = hi;
        *reinterpret_cast<u16x4*>(to + (S == 2 ? 32 : parts.lo / 2)) = lo;
    }
}

enum Product { kGram, kPoly, kUpdate, kLast };

// Work-groups go to the XCDs in turn; every XCD gets one run of the tiles in
// order, so that the tiles that share rows share an L2.
__device__ __forceinline__ int xcd_run(int b, int total) {
    const int x = b & 7, q = total >> 3, r = total & 7;
    return x * q + min(x, r) + (b >> 3);
}

// Eight parameters of row i, columns j .. j + 7 of the wide orientation (0 outside).
__device__ __forceinline__ Eight load_old(const OrthoGroup& g, int which, int i, int j) {
    Eight e = {};
    if (i >= g.m) return e;
    const float* x = g.x + g.off.at[which] + (g.tall ? j * g.row_stride + i : i * g.row_stride + j);
    if (g.vector && !g.tall && j + 7 < g.n) {
        const f4 a = *reinterpret_cast<const f4*>(x), b = *reinterpret_cast<const f4*>(x + 4);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            e.v[r] = a[r];
            e.v[4 + r] = b[r];
        }
        return e;
    }
#pragma unroll
    for (int r = 0; r < 8; ++r)
        if (j + r < g.n) e.v[r] = x[g.tall ? r * g.row_stride : r];
    return e;
}

// fp16 halves of eight numbers.
__device__ __forceinline__ u16x8 upper(const Eight& e) {
    u16x8 h;
#pragma unroll
    for (int r = 0; r < 8; ++r) h[r] = to_bits(e.v[r]);
    return h;
}
__device__ __forceinline__ u16x8 lower(const Eight& e) {
    u16x8 l;
#pragma unroll
    for (int r = 0; r < 8; ++r) l[r] = to_bits(e.v[r] - from_bits(to_bits(e.v[r])));
    return l;
}

// A = X X^T, B = c A A + b A, and a X + B X as the next X or as the result: tiles of
// BM x BM.  The symmetric two take the tiles on and below the diagonal, tile (i, j)
// before (i, j + 1), and write each a second time, turned in LDS.
//
// Eight bf16 6400 x 1600: A in 137-150 us (224 tiles, 0.9 PFLOP/s of what the symmetry
// leaves; the matrix cores are busy 78% of the time in which a CU has work, 73% of all),
// B in 50-55 (of which 17 a launch, its first loads and the turned stores), X in 374-403
// (1400 tiles in six turns, matrix cores busy 41%: their products take 231 us, the
// epilogue's 655 MB the rest: one work-group fills a CU, so they do not overlap).  Four fp32
// 5120 x 1280: A in 127-135 us, B 40-42, X 184-194 (two halves: three matrix instructions
// for one, 1.3-1.5 PFLOP/s of them).  Twelve bf16 768 x 768: 14, 16 and 26 us of one turn
// or two, a launch's start and end for the most part.
template <int S, int BM, Product P>
__global__ __launch_bounds__(tile::threads_of(BM)) void k_product(OrthoGroup g, Parts parts, int from, float mul,
                                                                    float add, int fallen, int next, int late) {
    using T = tile::Pick<S == 1 ? tile::kF16 : tile::kSplit, BM, kContig, P == kGram || P == kPoly ? kContig : kStrided>;
    constexpr bool kSymmetric = P == kGram || P == kPoly;
    __shared__ __align__(1024) char lds[T::kLdsBytes];
    const int m = g.m, n = g.n, mp = pad(m), np = pad(n);
    const int ti_n = (m + BM - 1) / BM, tj_n = ((kSymmetric ? m : n) + BM - 1) / BM;
    const int each = kSymmetric ? ti_n * (ti_n + 1) / 2 : ti_n * tj_n;
    const int id = xcd_run(blockIdx.x, each * g.count);
    const int which = id / each;
    int ti = 0, tj = id - which * each;
    if (kSymmetric) {
        while (tj > ti) tj -= ++ti;
    } else {
        // Down the columns of tiles: the next work-group takes the same columns of X.
        ti = tj % ti_n;
        tj /= ti_n;
    }
    char* ws = static_cast<char*>(g.workspace) + which * parts.bytes;
    u16* X = reinterpret_cast<u16*>(ws + parts.x[from]);
    u16* Y = reinterpret_cast<u16*>(ws + parts.x[from ^ 1]);
    u16* A = reinterpret_cast<u16*>(ws + parts.a);
    u16* B = reinterpret_cast<u16*>(ws + parts.b);
    const int64_t ldx = static_cast<int64_t>(np) * S, lda = static_cast<int64_t>(mp) * S;
    const Operand ox{X, ldx, m, np * S}, oa{A, lda, m, mp * S}, ob{B, lda, m, mp * S};
    T t;
    t.run(P == kGram ? ox : P == kPoly ? oa : ob, P == kPoly ? oa : ox, ti * BM, tj * BM, 0,
          P == kGram ? np : mp, (DSM_LDS char*)lds, m - ti * BM, (kSymmetric ? m : n) - tj * BM);

    // X is stored times 2^lift more, and after this iteration 2^after.
    const int lift = max(*reinterpret_cast<const int*>(ws + lift_at()) - fallen, 0);
    if constexpr (P == kPoly) {
        mul = ldexpf(mul, -4 * lift);
        add = ldexpf(add, -2 * lift);
    } else if constexpr (P == kUpdate || P == kLast) {
        const int after = P == kLast ? 0 : max(lift - next, 0);
        mul = ldexpf(mul, after - lift);
        add = ldexpf(add, after - lift);
    }
    // mul, add: powers of two and coefficients that bring the accumulator and
    // the stored A or X to the stored result.  What a batch of fragments needs of
    // them is loaded before the batch's first store, which the compiler must
    // assume to overlap it: one wait a batch, not one a fragment.
    constexpr int kBatch = T::FI < 4 ? T::FI : 4, kPairs = T::FJ / 2;
    const int64_t lo_at = S == 2 ? 32 : parts.lo / 2;  // of an X
    const u16* old = P == kPoly ? A : X;
    const int64_t ld_old = P == kPoly ? lda : ldx, old_lo = P == kPoly ? 32 : lo_at;
    const int last_col = (P == kPoly ? mp : np) - 8;
    // One half: A and B are stored without their diagonals.
    constexpr bool kApart = S == 1;
    float* diag_a = reinterpret_cast<float*>(ws + parts.diag_a);
    float* diag_b = reinterpret_cast<float*>(ws + parts.diag_b);
    Eight dj[kPairs];
    if constexpr (kApart && P == kPoly) {
#pragma unroll
        for (int p = 0; p < kPairs; ++p) {
            const float* d = diag_a + min(tj * BM + t.col8(p), last_col);
            const f4 lo = *reinterpret_cast<const f4*>(d), hi = *reinterpret_cast<const f4*>(d + 4);
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                dj[p].v[r] = lo[r];
                dj[p].v[4 + r] = hi[r];
            }
        }
    }
#pragma unroll
    for (int f0 = 0; f0 < T::FI; f0 += kBatch) {
        if (!kSymmetric && t.idle(f0)) break;
        u16x8 oh[kBatch][kPairs], ol[kBatch][kPairs];
        float di[kBatch];
        if constexpr (kApart && P != kGram) {
#pragma unroll
            for (int fi = 0; fi < kBatch; ++fi)
                di[fi] = (P == kPoly ? diag_a : diag_b)[min(ti * BM + t.row(f0 + fi), m - 1)];
        }
        if constexpr (P != kGram) {
#pragma unroll
            for (int fi = 0; fi < kBatch; ++fi)
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    const int64_t q = at<S>(min(ti * BM + t.row(f0 + fi), m - 1),
                                            min(tj * BM + t.col8(p), last_col), ld_old);
                    oh[fi][p] = *reinterpret_cast<const u16x8*>(old + q);
                    if constexpr (P != kPoly || S == 2)
                        ol[fi][p] = *reinterpret_cast<const u16x8*>(old + q + old_lo);
                }
        }
#pragma unroll
        for (int fi = 0; fi < kBatch; ++fi) {
            const int i = ti * BM + t.row(f0 + fi);
            // a X, with one half (a + E) X.
            const float add_hi = kApart && !kSymmetric ? __builtin_fmaf(mul, di[fi], add) : add, add_lo = late ? add_hi : add;
            Eight px[kPairs];
            if constexpr (P == kLast && S == 2) {
                if (g.x) {
#pragma unroll
                    for (int p = 0; p < kPairs; ++p) px[p] = load_old(g, which, i, tj * BM + t.col8(p));
                }
            }
#pragma unroll
            for (int p = 0; p < kPairs; ++p) {
                const int j = tj * BM + t.col8(p);
                Eight v = t.eight(f0 + fi, p);
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    v.v[r] *= mul;
                    if constexpr (P == kGram) {
                        continue;
                    } else if constexpr (S == 2) {
                        v.v[r] = __builtin_fmaf(add, from_bits(oh[fi][p][r]) + from_bits(ol[fi][p][r]), v.v[r]);
                    } else if constexpr (P == kPoly) {
                        v.v[r] = __builtin_fmaf(__builtin_fmaf(mul, di[fi] + dj[p].v[r], add), from_bits(oh[fi][p][r]), v.v[r]);
                    } else {
                        v.v[r] = __builtin_fmaf(add_lo, from_bits(ol[fi][p][r]), v.v[r]);
                        v.v[r] = __builtin_fmaf(add_hi, from_bits(oh[fi][p][r]), v.v[r]);
                    }
                }
                if constexpr (kApart && kSymmetric) {
                    if (ti == tj && i >= j && i < j + 8 && i < m) {
                        float d = 0.f;
#pragma unroll
                        for (int r = 0; r < 8; ++r)
                            if (i == j + r) {
                                d = v.v[r];
                                v.v[r] = 0.f;
                            }
                        if constexpr (P == kPoly) d = __builtin_fmaf(__builtin_fmaf(mul, di[fi], add), di[fi], d);
                        (P == kGram ? diag_a : diag_b)[i] = d;
                    }
                }
                if constexpr (kSymmetric) {
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        if (i >= m || j + r >= m) v.v[r] = 0.f;  // the padding of k
#pragma unroll
                    for (int r = 0; r < 4; ++r) {  // for the mirror image
                        t.acc[f0 + fi][2 * p][r] = v.v[r];
                        t.acc[f0 + fi][2 * p + 1][r] = v.v[4 + r];
                    }
                    if (i >= m || j >= mp) continue;
                    u16* out = (P == kGram ? A : B) + at<S>(i, j, lda);
                    *reinterpret_cast<u16x8*>(out) = upper(v);
                    if constexpr (S == 2) *reinterpret_cast<u16x8*>(out + 32) = lower(v);
                } else if constexpr (P == kUpdate) {
                    if (i >= m || j >= np) continue;
                    u16* out = Y + at<S>(i, j, ldx);
                    *reinterpret_cast<u16x8*>(out) = upper(v);
                    *reinterpret_cast<u16x8*>(out + lo_at) = lower(v);
                } else {
                    if (i >= m || j >= n) continue;
                    const int64_t e = g.off.at[which] + (g.tall ? j * g.row_stride + i : i * g.row_stride + j);
                    const bool whole = g.vector && !g.tall && j + 7 < n;
                    const int64_t step = g.tall ? g.row_stride : 1;
                    if constexpr (S == 2) {
                        float* out = (g.x ? g.x : static_cast<float*>(g.out)) + e;
#pragma unroll
                        for (int r = 0; r < 8; ++r) {
                            v.v[r] *= g.scale;
                            if (g.x) v.v[r] = px[p].v[r] - g.lr * (v.v[r] + g.weight_decay * px[p].v[r]);
                        }
                        if (whole) {
                            *reinterpret_cast<f4*>(out) = f4{v.v[0], v.v[1], v.v[2], v.v[3]};
                            *reinterpret_cast<f4*>(out + 4) = f4{v.v[4], v.v[5], v.v[6], v.v[7]};
                            continue;
                        }
#pragma unroll
                        for (int r = 0; r < 8; ++r)
                            if (j + r < n) out[r * step] = v.v[r];
                    } else {
                        u16* out = static_cast<u16*>(g.out) + e;
                        u16x8 b;
#pragma unroll
                        for (int r = 0; r < 8; ++r) b[r] = float_to_bf16(v.v[r]);
                        if (whole) {
                            *reinterpret_cast<u16x4*>(out) = u16x4{b[0], b[1], b[2], b[3]};
                            *reinterpret_cast<u16x4*>(out + 4) = u16x4{b[4], b[5], b[6], b[7]};
                            continue;
                        }
#pragma unroll
                        for (int r = 0; r < 8; ++r)
                            if (j + r < n) out[r * step] = b[r];
                    }
                }
            }
        }
    }
    // The tile above the diagonal: the same values through LDS, read transposed.
    if constexpr (kSymmetric) {
        if (ti == tj) return;
        using Turn = tile::Turned<BM>;
        DSM_LDS char* turned = (DSM_LDS char*)lds;
#pragma unroll
        for (int half = 0; half < S; ++half) {
#pragma unroll
            for (int fi = 0; fi < T::FI; ++fi)
#pragma unroll
                for (int p = 0; p < kPairs; ++p) {
                    Eight v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        v.v[r] = t.acc[fi][2 * p][r];
                        v.v[4 + r] = t.acc[fi][2 * p + 1][r];
                    }
                    Turn::put(turned, t.row(fi), t.col8(p),
                              __builtin_bit_cast(tile::short8v, half == 0 ? upper(v) : lower(v)));
                }
            __syncthreads();
            // 16 rows of the mirror image by 32 of its columns for each wave and turn.
            for (int c = t.wave; c < BM / 16 * (BM / 32); c += tile::threads_of(BM) / 64) {
                const int j0 = c / (BM / 32) * 16, i0 = c % (BM / 32) * 32;
                const int j = tj * BM + j0 + (t.lane & 15), i = ti * BM + i0 + (t.lane >> 4) * 8;
                const tile::short8v v = Turn::get(turned, i0, j0, t.lane);
                if (j < m && i < mp)
                    *reinterpret_cast<tile::short8v*>((P == kGram ? A : B) + at<S>(j, i, lda) + half * 32) = v;
            }
            if (half + 1 < S) __syncthreads();
        }
    }
}

// ---- Small matrices: the whole iteration in one work-group's LDS ----
//
// A matrix whose X and A fit LDS as split operands takes one launch: a work-group
// of eight waves keeps X and A (then B in its place) and iterates between barriers.
// With the products' kernels it would be 2 + 3 * steps launches of little work, each
// 3-5 us on the host and on the device: one 64 x 48 matrix 57-67 us so, 29 us here.
// Operands are stored as gemm_tile.h's stages are: for each 32 columns all rows of
// 128 bytes (hi x 32, lo x 32), the 16-byte pieces of a row exchanged by its number.

__host__ __device__ inline int pad32(int v) { return (v + 31) / 32 * 32; }

// Factors of the accumulators and of what is added to them, for each iteration.
struct SmallSteps {
    int steps;
    struct {
        float gram, poly, poly_add, update, update_add;
        int growth;
    } f[kOrthoMaxSteps];
};

struct SmallOperand {
    DSM_LDS char* p;
    int rows;  // padded
    __device__ __forceinline__ DSM_LDS char* piece(int row, int col, int half) const {
        const int byte = (col & 31) * 2;
        return p + ((col >> 5) * rows + row) * 128 + ((((byte >> 4) + half * 4) ^ (row & 7)) << 4) + (byte & 15);
    }
    // Rows 16 f .. of columns 32 kb .. : operand k-contiguous.
    __device__ __forceinline__ tile::short8v along(int f, int kb, int half, int lane) const {
        return *reinterpret_cast<const DSM_LDS tile::short8v*>(
            piece(f * 16 + (lane & 15), kb * 32 + (lane >> 4) * 8, half));
    }
    // Columns 16 f .. of rows 32 kb .. : operand k-strided.
    __device__ __forceinline__ tile::short8v across(int f, int kb, int half, int lane) const {
        const int k = kb * 32 + (lane >> 4) * 8 + ((lane & 15) >> 2), c = f * 16 + (lane & 3) * 4;
        const tile::short4v a =
            __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<DSM_LDS tile::short4v*>(piece(k, c, half)));
        const tile::short4v b =
            __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<DSM_LDS tile::short4v*>(piece(k + 4, c, half)));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ __forceinline__ f4 get(int row, int col) const {
        const u16x4 h = *reinterpret_cast<const DSM_LDS u16x4*>(piece(row, col, 0));
        const u16x4 l = *reinterpret_cast<const DSM_LDS u16x4*>(piece(row, col, 1));
        f4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = from_bits(h[r]) + from_bits(l[r]);
        return v;
    }
    __device__ __forceinline__ void put(int row, int col, f4 v) const {
        u16x4 h, l;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            h[r] = to_bits(v[r]);
            l[r] = to_bits(v[r] - from_bits(h[r]));
        }
        *reinterpret_cast<DSM_LDS u16x4*>(piece(row, col, 0)) = h;
        *reinterpret_cast<DSM_LDS u16x4*>(piece(row, col, 1)) = l;
    }
};

__device__ __forceinline__ f4 triple(tile::short8v ih, tile::short8v il, tile::short8v jh, tile::short8v jl, f4 c) {
    c = tile::mfma<tile::kSplit>(jl, ih, c);
    c = tile::mfma<tile::kSplit>(jh, il, c);
    return tile::mfma<tile::kSplit>(jh, ih, c);
}

template <bool STEP, bool BF16>
__global__ __launch_bounds__(kSmallWaves * 64) void k_small(OrthoGroup g, SmallSteps it, int x_exp) {
    __shared__ __align__(1024) char lds[kSmallLds];
    __shared__ double sums[kSmallWaves];
    const int m = g.m, n = g.n, mp = pad32(m), np = pad32(n);
    const SmallOperand X{(DSM_LDS char*)lds, mp}, A{(DSM_LDS char*)lds + mp * np * 4, mp};
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t base = g.off.at[blockIdx.x];
    const int rows = g.tall ? n : m, cols = g.tall ? m : n, quads = (cols + 3) / 4;

    // Momentum, norm, X_0.  A thread comes back to the elements it has written.
    double sum = 0.0;
    for (int q = threadIdx.x; q < rows * quads; q += kSmallWaves * 64) {
        const int r = q / quads, c = (q - r * quads) * 4;
        const f4 v = update_at<STEP, BF16, true>(g, base + r * g.row_stride + c, cols - c);
        sum += static_cast<double>(v[0]) * v[0] + static_cast<double>(v[1]) * v[1] +
               (static_cast<double>(v[2]) * v[2] + static_cast<double>(v[3]) * v[3]);
    }
    for (int w = 32; w > 0; w >>= 1) sum += __shfl_xor(sum, w);
    if (lane == 0) sums[wave] = sum;
    for (int e = threadIdx.x; e < mp * np / 4; e += kSmallWaves * 64)
        reinterpret_cast<DSM_LDS f4*>((DSM_LDS char*)lds)[e] = f4{0.f, 0.f, 0.f, 0.f};
    __syncthreads();
    sum = 0.0;
    for (int w = 0; w < kSmallWaves; ++w) sum += sums[w];
    const double norm = sqrt(sum);
    int lift = __builtin_amdgcn_readfirstlane(lift_of(norm, g.eps));
    const double inv = inverse_of(norm, g.eps, x_exp + lift);
    for (int q = threadIdx.x; q < rows * quads; q += kSmallWaves * 64) {
        const int r = q / quads, c = (q - r * quads) * 4;
        const f4 v = update_at<STEP, BF16, false>(g, base + r * g.row_stride + c, cols - c);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= cols) break;
            const float x = static_cast<float>(v[e] * inv);
            const int i = g.tall ? c + e : r, j = g.tall ? r : c + e;
            const u16 hi = to_bits(x);
            *reinterpret_cast<DSM_LDS u16*>(X.piece(i, j, 0)) = hi;
            *reinterpret_cast<DSM_LDS u16*>(X.piece(i, j, 1)) = to_bits(x - from_bits(hi));
        }
    }
    __syncthreads();

    const int mi = mp / 16, square = mi * mi, wide = mi * (np / 16);
    for (int s = 0; s < it.steps; ++s) {
        auto f = it.f[s];
        const bool last = s + 1 == it.steps;
        const int after = last ? 0 : max(lift - f.growth, 0);
        f.poly = ldexpf(f.poly, -4 * lift);
        f.poly_add = ldexpf(f.poly_add, -2 * lift);
        f.update = ldexpf(f.update, after - lift);
        f.update_add = ldexpf(f.update_add, after - lift);
        lift = after;
        // Unknown to the compiler in each iteration, or it would keep the LDS
        // addresses of every fragment in registers over all of them.
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const int i0 = ln & 15, j0 = (ln >> 4) * 4;
        for (int id = wave; id < square; id += kSmallWaves) {
            const int fi = id / mi, fj = id - fi * mi;
            f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
            for (int kb = 0; kb < np / 32; ++kb)
                acc = triple(X.along(fi, kb, 0, ln), X.along(fi, kb, 1, ln), X.along(fj, kb, 0, ln),
                             X.along(fj, kb, 1, ln), acc);
            A.put(fi * 16 + i0, fj * 16 + j0, acc * f.gram);
        }
        __syncthreads();
        f4 b[kSmallSquare];
#pragma unroll
        for (int t = 0; t < kSmallSquare; ++t) {
            const int id = t * kSmallWaves + wave;
            if (id >= square) continue;
            const int fi = id / mi, fj = id - fi * mi;
            f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int kb = 0; kb < mp / 32; ++kb)
                acc = triple(A.along(fi, kb, 0, ln), A.along(fi, kb, 1, ln), A.along(fj, kb, 0, ln),
                             A.along(fj, kb, 1, ln), acc);
            const f4 a = A.get(fi * 16 + i0, fj * 16 + j0);
#pragma unroll
            for (int r = 0; r < 4; ++r) b[t][r] = __builtin_fmaf(f.poly_add, a[r], acc[r] * f.poly);
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kSmallSquare; ++t) {
            const int id = t * kSmallWaves + wave;
            if (id >= square) continue;
            const int fi = id / mi;
            A.put(fi * 16 + i0, (id - fi * mi) * 16 + j0, b[t]);
        }
        __syncthreads();
        f4 x[kSmallWide];
#pragma unroll
        for (int t = 0; t < kSmallWide; ++t) {
            const int id = t * kSmallWaves + wave;
            if (id >= wide) continue;
            const int fj = id / mi, fi = id - fj * mi;
            f4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int kb = 0; kb < mp / 32; ++kb)
                acc = triple(A.along(fi, kb, 0, ln), A.along(fi, kb, 1, ln), X.across(fj, kb, 0, ln),
                             X.across(fj, kb, 1, ln), acc);
            const f4 a = X.get(fi * 16 + i0, fj * 16 + j0);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[t][r] = __builtin_fmaf(f.update_add, a[r], acc[r] * f.update);
        }
        __syncthreads();
#pragma unroll
        for (int t = 0; t < kSmallWide; ++t) {
            const int id = t * kSmallWaves + wave;
            if (id >= wide) continue;
            const int fj = id / mi, i = (id - fj * mi) * 16 + i0, j = fj * 16 + j0;
            if (!last) {
                X.put(i, j, x[t]);
                continue;
            }
            if (i >= m) continue;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (j + r >= n) continue;
                const int64_t e = base + (g.tall ? (j + r) * g.row_stride + i : i * g.row_stride + j + r);
                if constexpr (BF16) {
                    static_cast<u16*>(g.out)[e] = float_to_bf16(x[t][r]);
                } else {
                    const float d = g.scale * x[t][r];
                    if (g.x) {
                        const float p = g.x[e];
                        g.x[e] = p - g.lr * (d + g.weight_decay * p);
                    } else {
                        static_cast<float*>(g.out)[e] = d;
                    }
                }
            }
        }
        __syncthreads();
    }
}

float pow2(int e) { return __builtin_ldexpf(1.0f, e); }

template <int S, Product P>
void product(const OrthoGroup& g, const Parts& parts, int from, float mul, float add, int fallen, int next,
             bool late, hipStream_t stream) {
    constexpr bool kSymmetric = P == kGram || P == kPoly;
    const int bm = ortho_tile(g.count, g.m, g.n, kSymmetric);
    const unsigned groups = ortho_groups(g.count, g.m, g.n, bm, kSymmetric);
    if (bm == 64)
        k_product<S, 64, P><<<groups, tile::threads_of(64), 0, stream>>>(g, parts, from, mul, add, fallen, next, late);
    else if (bm == 128)
        k_product<S, 128, P><<<groups, tile::threads_of(128), 0, stream>>>(g, parts, from, mul, add, fallen, next, late);
    else
        k_product<S, 256, P><<<groups, tile::threads_of(256), 0, stream>>>(g, parts, from, mul, add, fallen, next, late);
}

// From which growth on the iterations left are "late" (k_product).
constexpr float kLate = 16.f;

template <int S>
void iterate(const OrthoGroup& g, const Parts& parts, const float* coeffs, const OrthoScales* scales,
             int steps, hipStream_t stream) {
    int fallen = 0;  // by how much X's lift has fallen
    for (int s = 0; s < steps; ++s) {
        const OrthoScales sc = scales[s];
        const float a = coeffs[3 * s], b = coeffs[3 * s + 1], c = coeffs[3 * s + 2];
        // Small singular values grow by this much in the iterations that follow.
        float growth = 1.f;
        for (int k = s + 1; k < steps; ++k) growth *= std::fabs(coeffs[3 * k]);
        const bool late = growth <= kLate;
        product<S, kGram>(g, parts, s & 1, pow2(sc.a - 2 * sc.x), 0.f, 0, 0, late, stream);
        product<S, kPoly>(g, parts, s & 1, c * pow2(sc.b - 2 * sc.a), b * pow2(sc.b - sc.a), fallen, 0, late, stream);
        const float mul = pow2(sc.x_next - sc.b - sc.x), add = a * pow2(sc.x_next - sc.x);
        if (s + 1 < steps)
            product<S, kUpdate>(g, parts, s & 1, mul, add, fallen, sc.growth, late, stream);
        else
            product<S, kLast>(g, parts, s & 1, mul, add, fallen, 0, late, stream);
        fallen += sc.growth;
    }
}

template <bool STEP, bool BF16>
void small(const OrthoGroup& g, const float* coeffs, const OrthoScales* scales, int steps, hipStream_t stream) {
    SmallSteps it;
    it.steps = steps;
    for (int s = 0; s < steps; ++s) {
        const OrthoScales sc = scales[s];
        it.f[s] = {pow2(sc.a - 2 * sc.x), coeffs[3 * s + 2] * pow2(sc.b - 2 * sc.a), coeffs[3 * s + 1] * pow2(sc.b - sc.a),
                   pow2(sc.x_next - sc.b - sc.x), coeffs[3 * s] * pow2(sc.x_next - sc.x), sc.growth};
    }
    k_small<STEP, BF16><<<g.count, kSmallWaves * 64, 0, stream>>>(g, it, scales[0].x);
}

template <int S, bool STEP, bool BF16>
void start(const OrthoGroup& g, const Parts& parts, int x_exp, hipStream_t stream) {
    // Some 4096 elements a work-group, and enough of them for all CUs.
    const int64_t total = static_cast<int64_t>(g.m) * g.n;
    const int n_parts = static_cast<int>(total < kNormParts * 4096 ? (total + 4095) / 4096 : kNormParts);
    k_norm<STEP, BF16><<<dim3(n_parts, g.count), 256, 0, stream>>>(g, parts, n_parts);
    const dim3 grid((pad(g.n) + kPrepTile - 1) / kPrepTile, (g.m + kPrepTile - 1) / kPrepTile, g.count);
    k_start<S, STEP, BF16><<<grid, 256, 0, stream>>>(g, parts, n_parts, x_exp);
}

}  // namespace

int64_t ortho_group_bytes(int count, int m, int n, bool bf16) {
    return is_small(m, n) ? 0 : Parts(m, n, !bf16).bytes * count;
}

hipError_t launch_ortho(const OrthoGroup& g, const float* coeffs, const OrthoScales* scales, int steps,
                        hipStream_t stream) {
    if (is_small(g.m, g.n)) {
        if (g.bf16)
            small<false, true>(g, coeffs, scales, steps, stream);
        else if (g.mom || g.x)
            small<true, false>(g, coeffs, scales, steps, stream);
        else
            small<false, false>(g, coeffs, scales, steps, stream);
        return hipGetLastError();
    }
    const Parts parts(g.m, g.n, g.bf16 == 0);
    if (g.bf16)
        start<1, false, true>(g, parts, scales[0].x, stream);
    else if (g.mom || g.x)
        start<2, true, false>(g, parts, scales[0].x, stream);
    else
        start<2, false, false>(g, parts, scales[0].x, stream);
    if (g.bf16)
        iterate<1>(g, parts, coeffs, scales, steps, stream);
    else
        iterate<2>(g, parts, coeffs, scales, steps, stream);
    return hipGetLastError();
}

}  // namespace dsm
