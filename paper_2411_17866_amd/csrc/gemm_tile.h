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

// What the operands hold: 16-bit numbers; two fp16 halves of each number; or fp32
// itself, for tiles that wait for memory rather than for the matrix cores (fp32
// products run at a sixteenth of the 16-bit ones' rate).  Sizes of operands count
// 16-bit units, two for each number of the last two.
enum Elem { kF16, kBF16, kSplit, kF32 };
constexpr int units(Elem e) { return e == kSplit || e == kF32 ? 2 : 1; }

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

template <Elem E>
__device__ __forceinline__ f4 mfma(short8v a, short8v b, f4 c) {
    if constexpr (E == kBF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bfloat8, a),
                                                       __builtin_bit_cast(bfloat8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a),
                                                      __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// Eight consecutive columns of one row from two neighbouring fragments, of which
// each lane holds four and four: the odd rows of 16 lanes of the first fragment
// change places with the even ones of the second.  Lane l then holds columns
// (l / 16 % 2) * 16 + l / 32 * 8 and the next seven of the two fragments' 32, so
// that four lanes move 64 bytes of fp16 in a row at once.
struct Eight {
    float v[8];
};
__device__ __forceinline__ Eight join(const f4& a, const f4& b) {
    Eight e;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        // Copies: a bit cast of a vector's element takes its first element.
        const float x = a[r], y = b[r];
        const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x),
                                                        __builtin_bit_cast(unsigned, y), false, false);
        const unsigned p = s[0], q = s[1];
        e.v[r] = __builtin_bit_cast(float, p);
        e.v[4 + r] = __builtin_bit_cast(float, q);
    }
    return e;
}
__device__ __forceinline__ int joined_col(int lane) { return ((lane >> 4) & 1) * 16 + (lane >> 5) * 8; }

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
    static_assert(KIND == kContig || (kRowBytes <= 1024 && 1024 % kRowBytes == 0), "whole rows in a piece");

    const char* base;        // of the tile at k = 0 (uniform)
    int64_t ld_bytes;
    uint32_t off[kLoads];
    int32_t k_rows;          // k-strided: rows that may be read from base on

    // swizzle of a k-strided row: 32-byte columns are exchanged so that the
    // rows that one transposing read touches fall into different banks.
    static __device__ __forceinline__ int swz(int k) {
        constexpr int kMask = (kRowBytes / 32 < 8 ? kRowBytes / 32 : 8) - 1;
        return ((k & 3) | ((k >> 1) & 4)) & kMask;
    }

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
            const int sw = swz(k);  // (that of k + 4 too)
            const int chunk = (S == 1 ? f : (f >> 1) * 4 + part * 2 + (f & 1)) ^ sw;
            const DSM_LDS char* at = lds + k * kRowBytes + chunk * 32 + (i & 3) * 8;
            short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                reinterpret_cast<DSM_LDS short4v*>(const_cast<DSM_LDS char*>(at)));
            short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                reinterpret_cast<DSM_LDS short4v*>(const_cast<DSM_LDS char*>(at + 4 * kRowBytes)));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    // fp32: steps part * 16 + lane / 16 * 4 and the next three, one for each of
    // four matrix instructions.
    static __device__ __forceinline__ f4 fragment32(const DSM_LDS char* lds, int f, int part, int lane) {
        if constexpr (KIND == kContig) {
            return __builtin_bit_cast(f4, fragment(lds, f, part, lane));
        } else {
            const int k = part * 16 + (lane >> 4) * 4, at = f * 64 + (lane & 15) * 4;
            f4 v;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = *reinterpret_cast<const DSM_LDS float*>(lds + (k + e) * kRowBytes +
                                                               (((at >> 5) ^ swz(k + e)) << 5) + (at & 31));
            return v;
        }
    }
};

// BM x BN tile by WM x WN waves, with STAGES buffers for stages of k: the loads of
// STAGES - 1 stages are in flight while one is multiplied.  Two suffice where a
// second work-group on the CU fills the waits; a CU with one work-group of small
// tiles waits for memory in every step and takes more.
template <Elem E, int BM, int BN, int WM, int WN_, int STAGES, Kind KI, Kind KJ>
struct Tile {
    static constexpr int S = units(E), kBM = BM, kBN = BN;
    static constexpr int WN = WN_;
    static constexpr int kWaves = WM * WN;
    static constexpr int kThreads = kWaves * 64;
    static constexpr int FI = BM / WM / 16, FJ = BN / WN / 16;  // fragments of a wave
    using SideI = Side<BM, kWaves, KI, S>;
    using SideJ = Side<BN, kWaves, KJ, S>;
    static constexpr int kSteps = SideI::kSteps;
    static constexpr int kStageBytes = SideI::kStageBytes + SideJ::kStageBytes;
    static constexpr int kLdsBytes = STAGES * kStageBytes;
    static constexpr int kLoads = SideI::kLoads + SideJ::kLoads;

    f4 acc[FI][FJ];
    int lane, wave, wi, wj;

    // Adds a stage.  Where tiles wait for memory anyway, fp32 and low bf16 ones, a stage
    // sums by itself: 1600 products as 50 sums of 32, not as one chain of 400 roundings
    // (single tokens' losses: off by 1e-7 for 4e-7).
    __device__ __forceinline__ void compute(const DSM_LDS char* st) {
        const DSM_LDS char* li = st;
        const DSM_LDS char* lj = st + SideI::kStageBytes;
        if constexpr (E == kF32) {
            f4 sum[FI][FJ] = {};
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                f4 fj[FJ];
#pragma unroll
                for (int j = 0; j < FJ; ++j) fj[j] = SideJ::fragment32(lj, wj * FJ + j, part, lane);
#pragma unroll
                for (int i = 0; i < FI; ++i) {
                    const f4 fi = SideI::fragment32(li, wi * FI + i, part, lane);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
#pragma unroll
                        for (int j = 0; j < FJ; ++j)
                            sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(fj[j][e], fi[e], sum[i][j], 0, 0, 0);
                }
            }
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[i][j] += sum[i][j];
        } else if constexpr (S == 1) {
            f4 sum[FI][FJ] = {};
            constexpr bool kApart = E == kBF16 && BM <= 64;  // (more rows' errors average)
#pragma unroll
            for (int part = 0; part < 2; ++part) {
                short8v fj[FJ];
#pragma unroll
                for (int j = 0; j < FJ; ++j) fj[j] = SideJ::fragment(lj, wj * FJ + j, part, lane);
#pragma unroll
                for (int i = 0; i < FI; ++i) {
                    const short8v fi = SideI::fragment(li, wi * FI + i, part, lane);
#pragma unroll
                    for (int j = 0; j < FJ; ++j) {
                        if constexpr (kApart)
                            sum[i][j] = mfma<E>(fj[j], fi, sum[i][j]);
                        else
                            acc[i][j] = mfma<E>(fj[j], fi, acc[i][j]);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FJ; ++j)
                    if constexpr (kApart) acc[i][j] += sum[i][j];
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
                for (int j = 0; j < FJ; ++j) acc[i][j] = mfma<E>(lo[j], hi, acc[i][j]);
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[i][j] = mfma<E>(hj[j], li_, acc[i][j]);
#pragma unroll
                for (int j = 0; j < FJ; ++j) acc[i][j] = mfma<E>(hj[j], hi, acc[i][j]);
            }
        }
    }

    __device__ __forceinline__ void clear() {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wi = wave / WN;
        wj = wave % WN;
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    }
    __device__ __forceinline__ void run(const Operand& oi, const Operand& oj, int64_t i0, int64_t j0,
                                        int k_begin, int k_end, DSM_LDS char* lds, int = 0, int = 0) {
        clear();
        add(oi, oj, i0, j0, k_begin, k_end, lds);
    }
    // Adds the products of steps [k_begin, k_end); k_begin is a multiple of kSteps,
    // and what lies between k_end and the next multiple is zero in one operand.
    __device__ __forceinline__ void add(const Operand& oi, const Operand& oj, int64_t i0, int64_t j0,
                                        int k_begin, int k_end, DSM_LDS char* lds, int = 0, int = 0) {
        SideI si;
        SideJ sj;
        si.init(oi, i0, lane, wave);
        sj.init(oj, j0, lane, wave);
        const int n = (k_end - k_begin + kSteps - 1) / kSteps;
        const auto load = [&](int s) {
            DSM_LDS char* at = lds + s % STAGES * kStageBytes;
            si.issue(k_begin + s * kSteps, at, lane, wave);
            sj.issue(k_begin + s * kSteps, at + SideI::kStageBytes, lane, wave);
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            if (s < n) load(s);
        for (int s = 0; s < n; ++s) {
            wait_loads_of(min(n - 1 - s, STAGES - 2));
            // The stage is there, and the one before it read: its products come before the
            // barrier in the compiled code (tests look), so its reads are over.
            __builtin_amdgcn_s_barrier();
            fence();
            if (s + STAGES - 1 < n) load(s + STAGES - 1);
            compute(lds + s % STAGES * kStageBytes);
            fence();
        }
        __builtin_amdgcn_s_barrier();
        fence();
    }

    // Until at most this many stages are in flight.
    static __device__ __forceinline__ void wait_loads_of(int stages) {
        if (STAGES > 3 && stages >= 2)
            wait_loads<2 * kLoads>();
        else if (STAGES > 2 && stages >= 1)
            wait_loads<kLoads>();
        else
            wait_loads<0>();
    }
    // Until at most N loads are in flight (vmcnt, 6 bits; the other counters untouched).
    template <int N>
    static __device__ __forceinline__ void wait_loads() {
        fence();
        __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
        fence();
    }
    static __device__ __forceinline__ void fence() { asm volatile("" ::: "memory"); }

    // Whether no row of the fragments from fi on is wanted.
    __device__ __forceinline__ bool idle(int) const { return false; }
    // i and j of acc[fi][fj][r] inside the tile.
    __device__ __forceinline__ int row(int fi) const { return (wi * FI + fi) * 16 + (lane & 15); }
    __device__ __forceinline__ int col(int fj) const { return (wj * FJ + fj) * 16 + (lane >> 4) * 4; }
    // Fragments 2 p and 2 p + 1 of row(fi), and their first column.
    __device__ __forceinline__ Eight eight(int fi, int p) const { return join(acc[fi][2 * p], acc[fi][2 * p + 1]); }
    __device__ __forceinline__ int col8(int p) const { return (wj * FJ + 2 * p) * 16 + joined_col(lane); }
};

// One side of a big tile (BigTile below): two half tiles of 128 rows (or
// columns), each a buffer of its own in LDS.
template <Kind KIND, int S>
struct HalfSide {
    static constexpr int kRows = 128;
    static constexpr int kBytes = kRows * 128;
    static constexpr int kWaves = 8;
    static constexpr int kLoads = kBytes / 1024 / kWaves;
    static constexpr int kSteps = S == 1 ? 64 : 32;
    static constexpr int kRowBytes = kRows * 2 * S;  // k-strided: one k row

    const char* base;
    int64_t ld_bytes;
    uint32_t off[2][kLoads];
    int32_t k_rows, last_col;

    static __device__ __forceinline__ int swz(int k) { return (k & 3) | ((k >> 1) & 4); }

    __device__ __forceinline__ void init(const Operand& o, int64_t first, int lane, int wave) {
        ld_bytes = o.ld * 2;
        if constexpr (KIND == kContig) {
            base = reinterpret_cast<const char*>(o.p) + first * ld_bytes;
            const int last = static_cast<int>(o.rows - 1 - first);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < kLoads; ++q) {
                    const int r = (q * kWaves + wave) * 8 + (lane >> 3);
                    const int chunk = (lane & 7) ^ (r & 7);
                    off[h][q] = static_cast<uint32_t>(min(h * kRows + r, last)) * static_cast<uint32_t>(ld_bytes) +
                                chunk * 16;
                }
        } else {
            base = reinterpret_cast<const char*>(o.p) + first * 2 * S;
            k_rows = o.rows;
            last_col = (o.cols - static_cast<int>(first) * S - 8) * 2;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < kLoads; ++q) off[h][q] = strided_off(h, q, lane, wave, 1 << 30);
        }
    }
    __device__ __forceinline__ uint32_t strided_off(int h, int q, int lane, int wave, int k_max) const {
        const int byte = (q * kWaves + wave) * 1024 + lane * 16;
        const int k = byte / kRowBytes;
        const int slot = (byte % kRowBytes) >> 4;
        const int at = (((slot >> 1) ^ swz(k)) << 1) | (slot & 1);  // 16-byte column of the half tile
        const int col = h * kRowBytes + at * 16;
        return static_cast<uint32_t>(min(k, k_max)) * static_cast<uint32_t>(ld_bytes) + min(col, last_col);
    }
    // Starts this wave's loads of half h of the stage at step k0.
    template <int H>
    __device__ __forceinline__ void issue(int k0, DSM_LDS char* lds, int lane, int wave) {
        const char* b;
        if constexpr (KIND == kContig) {
            b = base + static_cast<int64_t>(k0 / kSteps) * 128;
        } else {
            b = base + static_cast<int64_t>(min(k0, k_rows - 1)) * ld_bytes;
            if (k0 + kSteps > k_rows) {  // rows past the end read the last one
                const int last_k = max(k_rows - 1 - k0, 0);
#pragma unroll
                for (int q = 0; q < kLoads; ++q) off[H][q] = strided_off(H, q, lane, wave, last_k);
            }
        }
#pragma unroll
        for (int q = 0; q < kLoads; ++q)
            __builtin_amdgcn_global_load_lds(
                reinterpret_cast<const DSM_GLOBAL uint32_t*>(reinterpret_cast<uintptr_t>(b + off[H][q])),
                reinterpret_cast<DSM_LDS uint32_t*>(lds + (q * kWaves + wave) * 1024), 16, 0, 0);
    }
    static __device__ __forceinline__ short8v fragment(const DSM_LDS char* lds, int f, int part, int lane) {
        return Side<kRows, kWaves, KIND, S>::fragment(lds, f, part, lane);
    }
};

// A 256 x 256 tile by 8 waves, two on each SIMD.  A wave has 64 rows and 32 columns
// of each 128 x 128 quarter, so that a quarter where nothing is wanted (past the
// matrix's last row or column) costs no wave a matrix instruction.
//
// The two waves of a SIMD take turns: while one feeds the matrix core the other
// reads fragments from LDS and starts global loads, then they change over at a
// barrier (waves 4-7 run one turn behind).  A stage of k has two such turns, one
// for each half of the wave's rows:
//
//   turn  reads          multiplies      starts the loads of
//   0     I0 J1          I0 (J0 J1)      I1 one stage on, J0 two
//   1     I1, next J0    I1 (J0 J1)      I0 J1 two stages on
//
// so that both turns read as much, about what LDS gives while the other wave
// multiplies.  (Split operands multiply half as long again and need the registers:
// there J0 is read in turn 0 of its own stage, and loaded in turn 1.)  A turn's
// reads are waited for before the barrier that ends it, so the next turn's loads may
// overwrite what was read, by the waves that run behind too.  Each load has two
// turns or more to arrive: before the barrier a wave waits until at most 8 of its
// loads are in flight, which is all but those that the next turn's reads need.
//
// 8192 x 8192 x 4096, bf16: 1260 TFLOP/s with both operands k-contiguous, 1150 with
// one k-strided (1070 with J0 read in its own stage), 1060 with both; split operands
// 1440-1500 TFLOP/s of matrix instructions.  In the cross entropy's gradients the clock
// is at 1.8 GHz (of 2.4) and the matrix cores are busy 69% of the time in which a CU has
// work with one k-strided operand in fp16, 85% with split ones: the rest is the k-strided
// reads, starts and epilogues.
template <Elem E, Kind KI, Kind KJ, bool QUARTERS = KI == kContig && KJ == kContig, bool NARROW = false>
struct BigTile {
    static_assert(E != kF32, "fp32 products are for tiles that wait for memory");
    static constexpr int S = units(E);
    static constexpr int kBM = 256, kBN = 256, kThreads = 512;
    static constexpr int WN = 4, FI = 8, FJ = 4;
    using SideI = HalfSide<KI, S>;
    using SideJ = HalfSide<KJ, S>;
    static constexpr int kSteps = SideI::kSteps;
    static constexpr int kHalf = SideI::kBytes;
    static constexpr bool kAhead = S == 1;  // J0 is read a turn before its stage
    // Quarters without wanted rows or columns are left out by loops of their own.  (A
    // branch in the loop, or these loops beside k-strided loads, spill registers.)
    // NARROW: 128 columns at most are wanted, without asking.
    static constexpr bool kQuarters = QUARTERS;
    static constexpr int kStageBytes = 4 * kHalf;  // J0, I0, J1, I1
    static constexpr int kLdsBytes = 2 * kStageBytes;

    f4 acc[FI][FJ];
    int lane, wave, wi, wj;
    bool tall, wide;  // more than 128 rows, columns are wanted
    short8v fi[4][2], j0[kAhead ? 2 : 1][2][2], j1[2][2];  // j0: this stage's and the next one's

    static __device__ __forceinline__ void fence() {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("" ::: "memory");
    }
    // Until this wave's reads are done and at most N of its loads are in flight.
    template <int N>
    static __device__ __forceinline__ void wait() {
        fence();
        __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));
        fence();
    }
    static __device__ __forceinline__ void turn_over() {
        fence();
        __builtin_amdgcn_s_barrier();
        fence();
    }
    __device__ __forceinline__ void read_i(const DSM_LDS char* half) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int f = 0; f < 4; ++f) fi[f][part] = SideI::fragment(half, wi * 4 + f, part, lane);
    }
    __device__ __forceinline__ void read_j(const DSM_LDS char* half, short8v (&to)[2][2]) {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int f = 0; f < 2; ++f) to[f][part] = SideJ::fragment(half, wj * 2 + f, part, lane);
    }
    // The first N fragments of columns by half H of the rows.
    template <int H, int N>
    __device__ __forceinline__ void multiply(const short8v (&front)[2][2]) {
        fence();
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int t = 0; t < (S == 1 ? 2 : 3); ++t) {
            // S = 2: lo hi, hi lo, hi hi.
            const int pi = S == 1 ? t : t == 1, pj = S == 1 ? t : t == 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j)
                    acc[H * 4 + i][j] = mfma<E>(j < 2 ? front[j][pj] : j1[j - 2][pj], fi[i][pi], acc[H * 4 + i][j]);
        }
        __builtin_amdgcn_s_setprio(0);
        fence();
    }

    __device__ __forceinline__ void clear() {
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wi = wave / WN;
        wj = wave % WN;
#pragma unroll
        for (int i = 0; i < FI; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    }
    // Of the tile rows x cols are wanted.
    __device__ __forceinline__ void run(const Operand& oi, const Operand& oj, int64_t first_i, int64_t first_j,
                                        int k_begin, int k_end, DSM_LDS char* lds, int rows, int cols) {
        clear();
        add(oi, oj, first_i, first_j, k_begin, k_end, lds, rows, cols);
    }
    __device__ __forceinline__ void add(const Operand& oi, const Operand& oj, int64_t first_i, int64_t first_j,
                                        int k_begin, int k_end, DSM_LDS char* lds, int rows, int cols) {
        tall = rows > 128;
        wide = cols > 128;
        if (k_begin >= k_end) return;
        SideI si;
        SideJ sj;
        si.init(oi, first_i, lane, wave);
        sj.init(oj, first_j, lane, wave);
        const bool second = k_begin + kSteps < k_end;
        sj.template issue<0>(k_begin, lds, lane, wave);
        load_middle(si, sj, k_begin, lds);
        si.template issue<1>(k_begin, lds + 3 * kHalf, lane, wave);
        if (second) {
            sj.template issue<0>(k_begin + kSteps, lds + kStageBytes, lane, wave);
            load_middle(si, sj, k_begin + kSteps, lds + kStageBytes);
            wait<8>();  // all of the first stage but I1 is there
        } else {
            wait<0>();
        }
        turn_over();
        if constexpr (kAhead) {
            read_j(lds, j0[0]);
            wait<8>();
            turn_over();  // J0 is read: its next load may start
        }
        if (wave >= 4) turn_over();
        if (!kQuarters || (tall && wide))
            stages<2, NARROW ? 2 : 4>(si, sj, k_begin, k_end, lds);
        else if (tall)
            stages<2, 2>(si, sj, k_begin, k_end, lds);
        else if (wide)
            stages<1, 4>(si, sj, k_begin, k_end, lds);
        else
            stages<1, 2>(si, sj, k_begin, k_end, lds);
        if (wave < 4) turn_over();
        turn_over();  // every wave is done with LDS
    }
    // HALVES of the rows by N fragments of a wave's columns.
    template <int HALVES, int N>
    __device__ __forceinline__ void stages(SideI& si, SideJ& sj, int k, int k_end, DSM_LDS char* lds) {
        for (;;) {
            stage<0, HALVES, N>(si, sj, k, k_end, lds);
            if ((k += kSteps) >= k_end) break;
            stage<1, HALVES, N>(si, sj, k, k_end, lds);
            if ((k += kSteps) >= k_end) break;
        }
    }
    __device__ __forceinline__ void load_middle(SideI& si, SideJ& sj, int k, DSM_LDS char* st) {
        si.template issue<0>(k, st + kHalf, lane, wave);
        sj.template issue<1>(k, st + 2 * kHalf, lane, wave);
    }
    // The stage at step k, in buffer B.
    template <int B, int HALVES, int N>
    __device__ __forceinline__ void stage(SideI& si, SideJ& sj, int k, int k_end, DSM_LDS char* lds) {
        DSM_LDS char* st = lds + B * kStageBytes;
        DSM_LDS char* other = lds + (B ^ 1) * kStageBytes;
        const bool next = k + kSteps < k_end, more = k + 2 * kSteps < k_end;
        constexpr int kNow = kAhead ? B : 0;
        if constexpr (!kAhead) read_j(st, j0[0]);
        read_i(st + kHalf);
        if constexpr (N > 2) read_j(st + 2 * kHalf, j1);
        if (next) si.template issue<1>(k + kSteps, other + 3 * kHalf, lane, wave);
        if (kAhead ? more : next) {
            if constexpr (kAhead) sj.template issue<0>(k + 2 * kSteps, st, lane, wave);
            wait<8>();
        } else {
            wait<0>();
        }
        turn_over();
        multiply<0, N>(j0[kNow]);
        turn_over();
        if constexpr (HALVES > 1) read_i(st + 3 * kHalf);
        if constexpr (kAhead) {
            if (next) read_j(other, j0[B ^ 1]);
        }
        if (more) {
            if constexpr (!kAhead) sj.template issue<0>(k + 2 * kSteps, st, lane, wave);
            load_middle(si, sj, k + 2 * kSteps, st);
            wait<8>();
        } else {
            wait<0>();
        }
        turn_over();
        if constexpr (HALVES > 1) multiply<1, N>(j0[kNow]);
        turn_over();
    }

    // i and j of acc[fi][fj][r] inside the tile.
    __device__ __forceinline__ int row(int f) const { return (f >> 2) * 128 + wi * 64 + (f & 3) * 16 + (lane & 15); }
    __device__ __forceinline__ int col(int f) const { return (f >> 1) * 128 + wj * 32 + (f & 1) * 16 + (lane >> 4) * 4; }
    // Fragments 2 p and 2 p + 1 of row(fi), and their first column.
    __device__ __forceinline__ Eight eight(int f, int p) const { return join(acc[f][2 * p], acc[f][2 * p + 1]); }
    __device__ __forceinline__ int col8(int p) const { return p * 128 + wj * 32 + joined_col(lane); }
    __device__ __forceinline__ bool idle(int f) const { return f >= 4 && !tall; }
};

// A BM x BM tile of 16-bit values in LDS (rows of BM * 2 bytes, their 32-byte
// columns exchanged as a k-strided operand's are), to be read transposed.
template <int BM>
struct Turned {
    static __device__ __forceinline__ int at(int i, int j) {
        constexpr int kMask = (BM / 16 < 8 ? BM / 16 : 8) - 1;
        return i * BM * 2 + (((j >> 4) ^ (((i & 3) | ((i >> 1) & 4)) & kMask)) << 5) + (j & 15) * 2;
    }
    static __device__ __forceinline__ void put(DSM_LDS char* lds, int i, int j8, short8v v) {
        *reinterpret_cast<DSM_LDS short8v*>(lds + at(i, j8)) = v;
    }
    // Rows i .. i + 7 (i = i0 + lane / 16 * 8) of column j0 + lane % 16; i0 a
    // multiple of 32, j0 of 16.
    static __device__ __forceinline__ short8v get(DSM_LDS char* lds, int i0, int j0, int lane) {
        const int i = i0 + (lane >> 4) * 8 + ((lane & 15) >> 2), j = j0 + (lane & 3) * 4;
        short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<DSM_LDS short4v*>(lds + at(i, j)));
        short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<DSM_LDS short4v*>(lds + at(i + 4, j)));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

template <Elem E, int BM, Kind KI, Kind KJ>
struct Picked {
    static_assert(BM == 128, "tiles are 64, 128 or 256 square");
    using T = Tile<E, 128, 128, 2, 4, 2, KI, KJ>;
};
template <Elem E, Kind KI, Kind KJ>
struct Picked<E, 64, KI, KJ> {
    using T = Tile<E, 64, 64, 4, 2, 4, KI, KJ>;
};
template <Elem E, Kind KI, Kind KJ>
struct Picked<E, 256, KI, KJ> {
    using T = BigTile<E, KI, KJ>;
};
// The tile of BM x BM.  128 takes eight waves, two on a SIMD, so that one reads
// LDS while the other multiplies where a CU has one work-group: 8-16% less time
// than four waves there with split operands, 2-4% with fp16, and no more where two
// work-groups share a CU.
constexpr int threads_of(int) { return 512; }
template <Elem E, int BM, Kind KI, Kind KJ>
using Pick = typename Picked<E, BM, KI, KJ>::T;

}  // namespace tile
}  // namespace dsm
