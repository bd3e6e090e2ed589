// Matrix-core tiles of the language-model operators on gfx950.
//
// A work-group computes a BM x BN tile of C[i][j] = sum_k I(i,k) J(j,k) from
// 16-bit operands with fp32 accumulation.  An operand lies in memory either
// "k-contiguous" (a row for each i, k along the row) or "k-strided" (a row for
// each k, i along the row); the second kind is read from LDS with the
// transposing reads (ds_read_b64_tr_b16), so no operand is transposed in memory.
//
// Split operands (S = 2) carry 22 bits: x = hi + lo, both fp16, kept side by
// side in blocks of 32 (hi x 32, then lo x 32), and a product takes three matrix
// instructions, hi hi + hi lo + lo hi; the lo lo term is below 2^-22 of the
// largest.  A stage of LDS then holds 32 steps of k in the bytes that 64 take
// with S = 1, so the loader is the same.
//
// Stages are filled by direct global-to-LDS loads (16 bytes a lane) into two
// buffers: the loads of the next stage are in flight while one is multiplied.
// The load writes lane l's 16 bytes at l * 16 of a 1 KiB piece, so the swizzles
// that keep the reads free of bank conflicts are put on the global side: which
// 16 bytes a lane fetches.
//
// C is accumulated with j in the registers (4 consecutive j a lane) and i across
// the lanes: lane l of a 16 x 16 fragment holds i = l % 16, j = (l / 16) * 4 + r.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace dsm {
namespace tile {

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bfloat8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

#define DSM_LDS __attribute__((address_space(3)))
#define DSM_GLOBAL __attribute__((address_space(1)))

enum Kind { kContig, kStrided };  // how an operand lies in memory

// Zero-based 16-bit elements; `rows` is the number of rows that may be read
// (rows past it are replaced by the last one: what they give is never used, or
// meets zeros in the other operand), `cols` the same for the columns of a
// k-strided operand.
struct Operand {
    const uint16_t* p;
    int64_t ld;    // 16-bit elements from one row to the next
    int32_t rows;
    int32_t cols;  // k-strided only: 16-bit elements that may be read in a row
};

template <bool BF16>
__device__ __forceinline__ f4 mfma(short8v a, short8v b, f4 c) {
    if constexpr (BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloat8, a),
                                                       __builtin_bit_cast(bfloat8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a),
                                                      __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// One operand's loader and fragment reader: R rows (or columns) of the tile,
// NW waves in the work-group.
template <int R, int NW, Kind KIND, int S>
struct Side {
    static constexpr int kStageBytes = R * 128;
    static constexpr int kLoads = kStageBytes / 1024 / NW;  // wave loads of 1 KiB each
    static constexpr int kSteps = S == 1 ? 64 : 32;         // k of one stage
    static_assert(kStageBytes % (1024 * NW) == 0, "whole pieces for each wave");
    // k-strided: bytes of one k row of the tile.
    static constexpr int kRowBytes = R * 2 * S;
    static_assert(kRowBytes <= 1024 && 1024 % kRowBytes == 0, "whole rows in a piece");

    const char* base;        // of the tile at k = 0 (uniform)
    int64_t ld_bytes;
    uint32_t off[kLoads];
    int32_t k_rows;          // k-strided: rows that may be read from base on

    // swizzle of a k-strided row: 32-byte columns are exchanged so that the
    // rows that one transposing read touches fall into different banks.
    static __device__ __forceinline__ int swz(int k) { return (k & 3) | ((k >> 1) & 4); }

    __device__ __forceinline__ void init(const Operand& o, int64_t first, int lane, int wave) {
        ld_bytes = o.ld * 2;
        if constexpr (KIND == kContig) {
            base = reinterpret_cast<const char*>(o.p) + first * ld_bytes;
            const int last = static_cast<int>(o.rows - 1 - first);
#pragma unroll
            for (int q = 0; q < kLoads; ++q) {
                const int r = (q * NW + wave) * 8 + (lane >> 3);
                const int chunk = (lane & 7) ^ (r & 7);
                off[q] = static_cast<uint32_t>(min(r, last)) * static_cast<uint32_t>(ld_bytes) +
                         chunk * 16;
            }
        } else {
            base = reinterpret_cast<const char*>(o.p) + first * 2 * S;
            k_rows = o.rows;
            const int last = (o.cols - static_cast<int>(first) * S - 8) * 2;
#pragma unroll
            for (int q = 0; q < kLoads; ++q) off[q] = strided_off(q, lane, wave, last, 1 << 30);
            last_col = last;
        }
    }
    int last_col;
    __device__ __forceinline__ uint32_t strided_off(int q, int lane, int wave, int last, int k_max) {
        const int byte = (q * NW + wave) * 1024 + lane * 16;
        const int k = byte / kRowBytes;
        const int slot = (byte % kRowBytes) >> 4;
        const int col = ((((slot >> 1) ^ swz(k)) << 1) | (slot & 1)) * 16;
        return static_cast<uint32_t>(min(k, k_max)) * static_cast<uint32_t>(ld_bytes) + min(col, last);
    }
    // Starts the loads of the stage that begins at step k0 (a multiple of kSteps).
    __device__ __forceinline__ void issue(int k0, DSM_LDS char* lds, int lane, int wave) {
        const char* b;
        if constexpr (KIND == kContig) {
            b = base + static_cast<int64_t>(k0 / kSteps) * 128;
        } else {
            b = base + static_cast<int64_t>(min(k0, k_rows - 1)) * ld_bytes;
            if (k0 + kSteps > k_rows) {  // rows past the end read the last one
                const int last_k = max(k_rows - 1 - k0, 0);
#pragma unroll
                for (int q = 0; q < kLoads; ++q) off[q] = strided_off(q, lane, wave, last_col, last_k);
            }
        }
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            __builtin_amdgcn_global_load_lds(
                reinterpret_cast<const DSM_GLOBAL uint32_t*>(reinterpret_cast<uintptr_t>(b + off[q])),
                reinterpret_cast<DSM_LDS uint32_t*>(lds + (q * NW + wave) * 1024), 16, 0, 0);
    }
    // Fragment f (16 rows of the tile), part `part`: with S = 1 the 32 steps
    // part * 32 .., with S = 2 the hi (0) or lo (1) halves of the 32 steps.
    static __device__ __forceinline__ short8v fragment(const DSM_LDS char* lds, int f, int part,
                                                       int lane) {
        if constexpr (KIND == kContig) {
            const int r = lane & 15;
            const int chunk = (part * 4 + (lane >> 4)) ^ (r & 7);
            return *reinterpret_cast<const DSM_LDS short8v*>(lds + f * 2048 + r * 128 + chunk * 16);
        } else {
            const int g = lane >> 4, i = lane & 15;
            const int k = (S == 1 ? part * 32 : 0) + g * 8 + (i >> 2);
            const int sw = (i >> 2) | ((g & 1) << 2);
            const int chunk = (S == 1 ? f : (f >> 1) * 4 + part * 2 + (f & 1)) ^ sw;
            const DSM_LDS char* at = lds + k * kRowBytes + chunk * 32 + (i & 3) * 8;
            short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                reinterpret_cast<DSM_LDS short4v*>(const_cast<DSM_LDS char*>(at)));
            short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                reinterpret_cast<DSM_LDS short4v*>(const_cast<DSM_LDS char*>(at + 4 * kRowBytes)));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// BM x BN tile by WM x WN waves.
template <bool BF16, int S, int BM, int BN, int WM, int WN, Kind KI, Kind KJ>
struct Tile {
    static constexpr int kWaves = WM * WN;
    static constexpr int kThreads = kWaves * 64;
    static constexpr int FI = BM / WM / 16, FJ = BN / WN / 16;  // fragments of a wave
    using SideI = Side<BM, kWaves, KI, S>;
    using SideJ = Side<BN, kWaves, KJ, S>;
    static constexpr int kSteps = SideI::kSteps;
    static constexpr int kStageBytes = SideI::kStageBytes + SideJ::kStageBytes;
    static constexpr int kLdsBytes = 2 * kStageBytes;
    static constexpr int kLoads = SideI::kLoads + SideJ::kLoads;

    f4 acc[FI][FJ];
    int lane, wave, wi, wj;

    __device__ __forceinline__ void compute(const DSM_LDS char* st) {
        const DSM_LDS char* li = st;
        const DSM_LDS char* lj = st + SideI::kStageBytes;
        if constexpr (S == 1) {
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                short8v fj[FJ];
#pragma unroll
                for (int j = 0; j < FJ; ++j) fj[j] = SideJ::fragment(lj, wj * FJ + j, part, lane);
#pragma unroll
                for (int i = 0; i < FI; ++i) {
                    const short8v fi = SideI::fragment(li, wi * FI + i, part, lane);
#pragma unroll
                    for (int j = 0; j < FJ; ++j) acc[i][j] = mfma<BF16>(fj[j], fi, acc[i][j]);
                }
            }
        } else {
            short8v hj[FJ], lo[FJ];
#pragma unroll
            for (int j = 0; j < FJ; ++j) {
                hj[j] = SideJ::fragment(lj, wj * FJ + j, 0, lane);
                lo[j] = SideJ::fragment(lj, wj * FJ + j, 1, lane);
            }
#pragma unroll
            for (int i = 0; i < FI; ++i) {
                const short8v hi = SideI::fragment(li, wi * FI + i, 0, lane);
                const short8v li_ = SideI::fragment(li, wi * FI + i, 1, lane);
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[i][j] = mfma<BF16>(lo[j], hi, acc[i][j]);
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[i][j] = mfma<BF16>(hj[j], li_, acc[i][j]);
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[i][j] = mfma<BF16>(hj[j], hi, acc[i][j]);
            }
        }
    }

    // The products of steps [k_begin, k_end); k_begin is a multiple of kSteps,
    // and what lies between k_end and the next multiple is zero in one operand.
    __device__ __forceinline__ void run(const Operand& oi, const Operand& oj, int64_t i0, int64_t j0,
                                        int k_begin, int k_end, DSM_LDS char* lds) {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wi = wave / WN;
        wj = wave % WN;
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
        SideI si;
        SideJ sj;
        si.init(oi, i0, lane, wave);
        sj.init(oj, j0, lane, wave);
        if (k_begin >= k_end) return;
        si.issue(k_begin, lds, lane, wave);
        sj.issue(k_begin, lds + SideI::kStageBytes, lane, wave);
        int buf = 0;
        for (int k = k_begin; k < k_end; k += kSteps) {
            if (k + kSteps < k_end) {
                DSM_LDS char* next = lds + (buf ^ 1) * kStageBytes;
                si.issue(k + kSteps, next, lane, wave);
                sj.issue(k + kSteps, next + SideI::kStageBytes, lane, wave);
                wait_loads<kLoads>();
            } else {
                wait_loads<0>();
            }
            __builtin_amdgcn_s_barrier();
            fence();
            compute(lds + buf * kStageBytes);
            fence();
            __builtin_amdgcn_s_barrier();  // the buffer is read: the next stage may fill it
            buf ^= 1;
        }
    }

    // Until at most N loads are in flight (vmcnt, 6 bits; the other counters untouched).
    template <int N>
    static __device__ __forceinline__ void wait_loads() {
        fence();
        __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
        fence();
    }
    static __device__ __forceinline__ void fence() { asm volatile("" ::: "memory"); }

    // i and j of acc[fi][fj][r] inside the tile.
    __device__ __forceinline__ int row(int fi) const { return (wi * FI + fi) * 16 + (lane & 15); }
    __device__ __forceinline__ int col(int fj) const { return (wj * FJ + fj) * 16 + (lane >> 4) * 4; }
};

}  // namespace tile
}  // namespace dsm
