// The global norm of many gradients, and clipping by it, on gfx950.
//
//   norm = sqrt(sum of g^2 over a group's tensors);  g <- g min(1, max / (norm + eps))
//
// A work-group takes a chunk of a tensor; squares are taken and summed in fp64, so
// that no magnitude of fp32 overflows or vanishes in them and the order of the sums
// does not show in the norm.  (A conversion and an fma an element, a fifth of what
// the CUs can do while memory brings them.)  Sums of chunks go to the workspace and
// are joined in a fixed order.
//
// It is bound by memory: all gradients are read, and where the norm exceeds the
// maximum read again and written.  The second pass takes the chunks from the last to
// the first: what was read last is still in the last-level cache.
#include "block_internal.h"
#include "elements.h"

#pragma clang fp contract(off)

namespace dsm {
namespace {

using rows::V8;

struct Chunk {
    ClipEntry e;
    int64_t at;  // of the tensor's elements
    int n;
};

__device__ __forceinline__ Chunk chunk_of(const ClipTable& t, int c) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (t.e[mid].chunk <= c)
            lo = mid;
        else
            hi = mid - 1;
    }
    Chunk k;
    k.e = t.e[lo];
    k.at = static_cast<int64_t>(c - k.e.chunk) * kClipChunk;
    k.n = static_cast<int>(min(static_cast<int64_t>(kClipChunk), k.e.numel - k.at));
    return k;
}

// Where up to eight elements lie, as offsets from data.
struct Run {  // side by side; in fp32 also two fours, `apart` from each other
    int64_t at;
    int have, apart;
};
struct Spread {  // each by itself
    int64_t at[8];
    int have;
};
template <bool F32, bool ONCE = false>
__device__ __forceinline__ V8 load(const void* data, const Run& r) {
    return rows::load8<F32, ONCE>(data, r.at, r.have, r.apart);
}
template <bool F32>
__device__ __forceinline__ void store(void* data, const Run& r, const V8& x) {
    rows::store8<F32>(data, r.at, x, r.have, r.apart);
}
template <bool F32, bool ONCE = false>
__device__ __forceinline__ V8 load(const void* data, const Spread& s) {
    V8 x;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        x.v[q] = 0.f;
        if (q >= s.have) continue;
        if constexpr (F32)
            x.v[q] = static_cast<const float*>(data)[s.at[q]];
        else
            x.v[q] = rows::bf16_to_float(static_cast<const rows::u16*>(data)[s.at[q]]);
    }
    return x;
}
template <bool F32>
__device__ __forceinline__ void store(void* data, const Spread& s, const V8& x) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        if (q >= s.have) continue;
        if constexpr (F32)
            static_cast<float*>(data)[s.at[q]] = x.v[q];
        else
            static_cast<rows::u16*>(data)[s.at[q]] = rows::float_to_bf16(x.v[q]);
    }
}

// Calls use(array of Runs or Spreads, whose loads go side by side) for all elements of a chunk.  In fp32 neighbouring lanes load whole
// lines as two fours (496 MB clipped in 261 us instead of 272).  Rows apart whose width or first element is no
// multiple of eight have no eights in common with the chunk's: there a lane takes eight elements 256 from
// each other, and its neighbours those beside them (16384 x 1601 in fp32 99 us, where an element at a time
// took 171; x 1600 55).
template <bool F32, class F>
__device__ __forceinline__ void each_run(const Chunk& k, F use) {
    const int64_t start = k.e.first + k.at;
    if (k.e.block >= k.e.first + k.e.numel) {  // one run
        const auto whole = [&](int u) { return Run{static_cast<int64_t>(start + u + threadIdx.x * (F32 ? 4 : 8)), 8, F32 ? 1024 : 4}; };
        int u = 0;
        for (; u + 8192 <= k.n; u += 8192) {
            const Run runs[4] = {whole(u), whole(u + 2048), whole(u + 4096), whole(u + 6144)};
            use(runs);
        }
        for (; u + 2048 <= k.n; u += 2048) {
            const Run runs[1] = {whole(u)};
            use(runs);
        }
        u += static_cast<int>(threadIdx.x) * 8;
        const Run runs[1] = {Run{start + u, k.n - u, 4}};
        if (u < k.n) use(runs);
        return;
    }
    const int64_t row = start / k.e.block, col = start - row * k.e.block;
    const bool eights = start % 8 == 0 && k.e.block % 8 == 0;
    const auto elements = [&](auto place) {
        if (eights) {
            int u = threadIdx.x * 8;
            for (; u + 6144 + 8 <= k.n; u += 8192) {
                const Run runs[4] = {{place(u), 8, 4}, {place(u + 2048), 8, 4}, {place(u + 4096), 8, 4}, {place(u + 6144), 8, 4}};
                use(runs);
            }
            for (; u < k.n; u += 2048) {
                const Run runs[1] = {{place(u), min(8, k.n - u), 4}};
                use(runs);
            }
            return;
        }
        for (int u = threadIdx.x; u < k.n; u += 2048) {
            Spread s[1];
            s[0].have = min(8, (k.n - u + 255) / 256);
#pragma unroll
            for (int q = 0; q < 8; ++q) s[0].at[q] = place(u + q * 256);
            use(s);
        }
    };
    if (k.e.block >= kClipChunk) {  // at most one row ends inside
        const int left = static_cast<int>(min(k.e.block - col, static_cast<int64_t>(kClipChunk)));
        elements([&](int u) { return u < left ? row * k.e.stride + col + u : (row + 1) * k.e.stride + u - left; });
    } else {
        const unsigned block = static_cast<unsigned>(k.e.block), c0 = static_cast<unsigned>(col);
        elements([&](int u) {
            const unsigned c = c0 + u, r = c / block;
            return static_cast<int64_t>((row + r) * k.e.stride + (c - r * block));
        });
    }
}

// The sum of a work-group's values, in its first lane.
__device__ __forceinline__ double group_sum(double v) {
    __shared__ double waves[16];
    for (int w = 32; w > 0; w >>= 1) v += __shfl_xor(v, w);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
    for (unsigned w = 0; w < blockDim.x / 64; ++w) s += waves[w];
    return s;
}

template <bool F32, bool ONCE>
__device__ __forceinline__ double squares(const Chunk& k) {
    double a = 0.0, b = 0.0;
    each_run<F32>(k, [&](const auto& at) {
        constexpr int N = sizeof(at) / sizeof(at[0]);
        V8 x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = load<F32, ONCE>(k.e.data, at[i]);
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int q = 0; q < 8; q += 2) {
                const double u = x[i].v[q], v = x[i].v[q + 1];
                a = __builtin_fma(u, u, a);
                b = __builtin_fma(v, v, b);
            }
    });
    return a + b;
}

// ONCE: of more bytes than the last-level cache holds.
template <bool ONCE>
__global__ __launch_bounds__(256) void k_clip_squares(ClipTable t, double* parts) {
    const Chunk k = chunk_of(t, blockIdx.x);
    const double s = group_sum(k.e.bf16 ? squares<false, ONCE>(k) : squares<true, ONCE>(k));
    if (threadIdx.x == 0) parts[t.slot + blockIdx.x] = s;
}

// A group's norm from its chunks' sums.
template <class Groups>
__device__ __forceinline__ double group_norm(const Groups& g, int group, const double* parts) {
    double s = 0.0;
    for (int64_t c = g.start[group] + threadIdx.x; c < g.start[group + 1]; c += blockDim.x) s += parts[c];
    return sqrt(group_sum(s));
}
// Gradients whose norm is not a finite number stay as they are: no factor mends them.
// (In fp64, as the products: a norm near fp32's largest number has a factor below its
// smallest.)
template <class Groups>
__device__ __forceinline__ double factor_of(const Groups& g, double norm) {
    if (!(norm < __builtin_inf())) return 1.0;
    return fmin(1.0, static_cast<double>(g.max_norm) / (norm + static_cast<double>(g.eps)));
}

__global__ __launch_bounds__(1024) void k_clip_norms(ClipGroups g, const double* parts, float* norm, double* factor) {
    const double v = group_norm(g, blockIdx.x, parts);
    if (threadIdx.x != 0) return;
    norm[blockIdx.x] = static_cast<float>(v);
    factor[blockIdx.x] = factor_of(g, v);
}

// Ten of v's bits, the last of them set where anything follows: exact in fp32 down to where bf16 is 0, and rounded
// to bf16 as v itself.
__device__ __forceinline__ float ten_bits(double v) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const uint32_t high = static_cast<uint32_t>(bits >> 32), low = static_cast<uint32_t>(bits);
    const uint32_t rest = ((high & 0x3ffu) | low) != 0 ? 0x400u : 0u;
    return static_cast<float>(__builtin_bit_cast(double, static_cast<uint64_t>((high & ~0x3ffu) | rest) << 32));
}

// Products in fp64.  bf16 is rounded by way of fp32, which comes to one rounding of the product but where fp32's falls
// on a middle of bf16's (its lower half is 0x8000, the least of 16 signed bits), as one in 2^16 does by chance: where one of
// a lane's eight does, they go by their first ten bits.  (Nine tensors of 100 x 201 and less, both launches: 6.63 us,
// 6.92 with every product's ten bits, 6.48 with neither; loads of four runs go before their first store.)
template <bool F32>
__device__ __forceinline__ void scale(const Chunk& k, double by) {
    typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
    each_run<F32>(k, [&](const auto& at) {
        constexpr int N = sizeof(at) / sizeof(at[0]);
        V8 x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = load<F32>(k.e.data, at[i]);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            V8 f;
            i16x2 least = {0, 0};
#pragma unroll
            for (int q = 0; q < 8; ++q) f.v[q] = static_cast<float>(x[i].v[q] * by);
            if constexpr (!F32) {
#pragma unroll
                for (int q = 0; q < 8; q += 2) {
                    const i16x2 halves = {static_cast<int16_t>(__builtin_bit_cast(uint32_t, f.v[q])),
                                          static_cast<int16_t>(__builtin_bit_cast(uint32_t, f.v[q + 1]))};
                    least = __builtin_elementwise_min(least, halves);
                }
                if (__builtin_expect(min(least[0], least[1]) == INT16_MIN, 0)) {
#pragma unroll
                    for (int q = 0; q < 8; ++q) f.v[q] = ten_bits(x[i].v[q] * by);
                }
            }
            store<F32>(k.e.data, at[i], f);
        }
    });
}
__device__ __forceinline__ void scale(const Chunk& k, double by) {
    if (by == 1.0) return;
    if (k.e.bf16)
        scale<false>(k, by);
    else
        scale<true>(k, by);
}

__global__ __launch_bounds__(256) void k_clip_scale(ClipTable t, const double* factor) {
    const Chunk k = chunk_of(t, t.chunks - 1 - blockIdx.x);
    scale(k, factor[k.e.group]);
}

// Few chunks: a launch less.  The work-groups past the chunks write the norms.
__global__ __launch_bounds__(256) void k_clip_rest(ClipTable t, ClipFew g, const double* parts, float* norm) {
    const int c = blockIdx.x;
    if (c >= t.chunks) {
        const double v = group_norm(g, c - t.chunks, parts);
        if (threadIdx.x == 0) norm[c - t.chunks] = static_cast<float>(v);
        return;
    }
    const Chunk k = chunk_of(t, c);
    scale(k, factor_of(g, group_norm(g, k.e.group, parts)));
}

}  // namespace

hipError_t launch_clip_squares(const ClipTable& t, int64_t bytes, double* parts, hipStream_t stream) {
    // 496 MB in fp32: the norm alone 83 us, 6.0 TB/s, and 94 by loads that stay in the caches; 37 MB 9.6 and 8.8.
    if (bytes > kClipOnce)
        k_clip_squares<true><<<t.chunks, 256, 0, stream>>>(t, parts);
    else
        k_clip_squares<false><<<t.chunks, 256, 0, stream>>>(t, parts);
    return hipGetLastError();
}

hipError_t launch_clip_norms(const ClipGroups& g, const double* parts, float* norm, double* factor, hipStream_t stream) {
    k_clip_norms<<<g.count, 1024, 0, stream>>>(g, parts, norm, factor);
    return hipGetLastError();
}

hipError_t launch_clip_scale(const ClipTable& t, const double* factor, hipStream_t stream) {
    k_clip_scale<<<t.chunks, 256, 0, stream>>>(t, factor);
    return hipGetLastError();
}

hipError_t launch_clip_rest(const ClipTable& t, const ClipFew& g, const double* parts, float* norm, hipStream_t stream) {
    k_clip_rest<<<t.chunks + g.count, 256, 0, stream>>>(t, g, parts, norm);
    return hipGetLastError();
}

}  // namespace dsm
