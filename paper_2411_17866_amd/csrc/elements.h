// Rows of fp32 or bf16 elements, eight to a lane, and sums over a wave or a
// work-group, for the kernels that stream rows (clip.hip, norm.hip, linear.hip).
//
// Rows may start at any element: 16-byte accesses of global memory need no more than
// the element's own alignment on gfx950, so odd widths and strides take the same path.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dsm {
namespace rows {

typedef unsigned short u16;
typedef u16 u16x8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
// The same at any element's address.
typedef u16x8 u16x8_at __attribute__((aligned(2)));
typedef f4 f4_at __attribute__((aligned(4)));

__device__ __forceinline__ u16 float_to_bf16(float v) { return __builtin_bit_cast(u16, static_cast<__bf16>(v)); }
__device__ __forceinline__ float bf16_to_float(u16 v) {
    return __builtin_bit_cast(float, static_cast<uint32_t>(v) << 16);
}

struct V8 {
    float v[8];
};

// Eight elements as they lie in memory.
template <bool F32>
struct Raw8 {
    u16x8 v;
};
template <>
struct Raw8<true> {
    f4 a, b;
};

// 16 bytes from any element's address; ONCE leaves the caches to what is read again.  (A
// type's lesser alignment does not pass through a template's argument.)
template <bool ONCE>
__device__ __forceinline__ f4 from(const float* p) {
    const f4_at* at = reinterpret_cast<const f4_at*>(p);
    if constexpr (ONCE)
        return __builtin_nontemporal_load(at);
    else
        return *at;
}
template <bool ONCE>
__device__ __forceinline__ u16x8 from(const u16* p) {
    const u16x8_at* at = reinterpret_cast<const u16x8_at*>(p);
    if constexpr (ONCE)
        return __builtin_nontemporal_load(at);
    else
        return *at;
}

// Eight elements from element `at` on, of which `have` exist (the others are 0); in fp32 all
// eight may also be two fours, `apart` from each other.
template <bool F32, bool ONCE = false>
__device__ __forceinline__ Raw8<F32> raw8(const void* base, int64_t at, int have, int apart = 4) {
    Raw8<F32> o;
    if constexpr (F32) {
        const float* p = static_cast<const float*>(base) + at;
        o.a = o.b = f4{0.f, 0.f, 0.f, 0.f};
        if (have >= 8) {
            o.a = from<ONCE>(p);
            o.b = from<ONCE>(p + apart);
        } else if (have > 0) {
            // The last one again for those that are missing: loads side by side, no branches.
            // (Their places are not kept in registers from one row to the next.)
            int last = have - 1;
            asm volatile("" : "+v"(last));
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float a = p[min(q, last)], b = p[min(4 + q, last)];
                o.a[q] = q < have ? a : 0.f;
                o.b[q] = 4 + q < have ? b : 0.f;
            }
        }
    } else {
        const u16* p = static_cast<const u16*>(base) + at;
        o.v = u16x8{0, 0, 0, 0, 0, 0, 0, 0};
        if (have >= 8) {
            o.v = from<ONCE>(p);
        } else if (have > 0) {
            int last = have - 1;
            asm volatile("" : "+v"(last));
#pragma unroll
            for (int q = 0; q < 7; ++q) {
                const u16 a = p[min(q, last)];
                o.v[q] = q < have ? a : static_cast<u16>(0);
            }
        }
    }
    return o;
}
template <bool F32>
__device__ __forceinline__ V8 wide8(const Raw8<F32>& x) {
    V8 o;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        if constexpr (F32)
            o.v[q] = q < 4 ? x.a[q & 3] : x.b[q & 3];
        else
            o.v[q] = bf16_to_float(x.v[q]);
    }
    return o;
}
// Moves elements `back` places to the front, zeros behind them.
__device__ __forceinline__ void shift(V8& v, int back) {
#pragma unroll
    for (int by = 4; by > 0; by /= 2)
#pragma unroll
        for (int q = 0; q < 8; ++q) v.v[q] = (back & by) ? (q + by < 8 ? v.v[q + by] : 0.f) : v.v[q];
}
template <bool F32, bool ONCE = false>
__device__ __forceinline__ V8 load8(const void* base, int64_t at, int have, int apart = 4) {
    return wide8(raw8<F32, ONCE>(base, at, have, apart));
}

template <bool F32>
__device__ __forceinline__ void store8(void* base, int64_t at, const V8& x, int have, int apart = 4) {
    if constexpr (F32) {
        float* p = static_cast<float*>(base) + at;
        if (have >= 8) {
            f4 a, b;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                a[q] = x.v[q];
                b[q] = x.v[4 + q];
            }
            *reinterpret_cast<f4_at*>(p) = a;
            *reinterpret_cast<f4_at*>(p + apart) = b;
        } else if (have > 0) {
#pragma unroll
            for (int q = 0; q < 7; ++q)
                if (q < have) p[q] = x.v[q];
        }
    } else {
        u16* p = static_cast<u16*>(base) + at;
        if (have >= 8) {
            u16x8 a;
#pragma unroll
            for (int q = 0; q < 8; ++q) a[q] = float_to_bf16(x.v[q]);
            *reinterpret_cast<u16x8_at*>(p) = a;
        } else if (have > 0) {
#pragma unroll
            for (int q = 0; q < 7; ++q)
                if (q < have) p[q] = float_to_bf16(x.v[q]);
        }
    }
}

// x of the lane that a DPP control names.
template <int CTRL>
__device__ __forceinline__ float from_lane(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// The sum over every L lanes that lie together, in each of them, in a fixed order: within
// 16 lanes by turns, then rows of 16 change places.
template <int L>
__device__ __forceinline__ float lanes_sum(float x) {
    static_assert(L == 8 || L == 16 || L == 32 || L == 64, "parts of a wave");
    if constexpr (L == 8) {
        x += from_lane<0xb1>(x);   // quad_perm: lane ^ 1
        x += from_lane<0x4e>(x);   // quad_perm: lane ^ 2
        x += from_lane<0x141>(x);  // half of a row mirrored: the other quad
        return x;
    }
    x += from_lane<0x128>(x);  // turned by 8, 4, 2, 1 in a row of 16
    x += from_lane<0x124>(x);
    x += from_lane<0x122>(x);
    x += from_lane<0x121>(x);
    if constexpr (L >= 32) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        const unsigned p = a[0], q = a[1];
        x = __builtin_bit_cast(float, p) + __builtin_bit_cast(float, q);
    }
    if constexpr (L == 64) {
        const unsigned u = __builtin_bit_cast(unsigned, x);
        const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        const unsigned p = b[0], q = b[1];
        x = __builtin_bit_cast(float, p) + __builtin_bit_cast(float, q);
    }
    return x;
}

// Sums of K values over a work-group of W waves, in every lane, through K * W floats
// of LDS.  Two calls in a row take two buffers, so one barrier is enough: whoever
// writes a buffer again has passed the barrier that follows everyone's reads of it.
template <int W, int K>
__device__ __forceinline__ void group_sums(float (&x)[K], float* lds) {
#pragma unroll
    for (int k = 0; k < K; ++k) x[k] = lanes_sum<64>(x[k]);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) lds[k * W + (threadIdx.x >> 6)] = x[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float s = lds[k * W];
#pragma unroll
            for (int w = 1; w < W; ++w) s += lds[k * W + w];
            x[k] = s;
        }
    }
}

}  // namespace rows
}  // namespace dsm
