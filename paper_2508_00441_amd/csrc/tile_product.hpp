// The product of a tile of vectors X (rows of the matrix unit's result) with a tile of vectors Y (its columns), both contiguous along
// the inner dimension: FP8 codes with a scale per 128 of them, BF16 or FP16.
//
// A step is 128 bytes of the inner dimension of every vector of the tile: 128 FP8 codes, which are one v_mfma_f32_16x16x128 deep and
// share their scales, or 64 elements of 16 bits, two v_mfma_f32_16x16x32 deep.  Steps travel from memory to LDS with direct loads
// through a ring of NST buffers; a wave reads its fragments from there.
//
// LDS rows are 128 bytes; the eight 16-byte pieces of row r lie at place piece ^ ((r >> 1) & 7).  Lane l reads pieces l / 16 and l / 16 + 4
// of row l % 16 of a 16-row tile: the sixteen lanes that a 128-bit LDS read serves together (0-3, 12-15, 20-23, 24-27 and the like)
// then meet sixteen different places of the 256 bytes that the banks hold.  (Which elements of the inner dimension a lane takes is
// free, as long as both operands agree.)  A direct load writes lane l's 16 bytes at a fixed place, base + 16 l, so each lane
// fetches the piece that belongs there.
//
// Vectors beyond the matrix repeat the last one; their results are not stored.  Pieces beyond the end of the vectors are read from
// sixteen zero bytes, and where the end lies inside a piece the bytes behind it are cleared in LDS, in both operands: what the
// caller's memory holds there may be a NaN.
#pragma once
#include "low_precision.hpp"

namespace ozaki {
namespace {

// FP8: X's scales per 128 x 128 block or per 128 elements of a vector (Y's always the latter), on the FP8 or on the FP16 instructions
constexpr int KIND_FP8_BLOCKS = 0, KIND_FP8_VECTORS = 1, KIND_WIDE_BLOCKS = 2, KIND_WIDE_VECTORS = 3, KIND_BF16 = 4, KIND_F16 = 5;
constexpr int STEP_BYTES = 128;

#define OZAKI_TILE_GPTR(p) ((const __attribute__((address_space(1))) void*)(p))
#define OZAKI_TILE_LPTR(p) ((__attribute__((address_space(3))) void*)(p))

__device__ __attribute__((aligned(16))) uint8_t no_elements[16];

// A lane's share of 16 vectors' 128 codes, and the product of two such shares over the 128 elements.  The matrix unit's FP8 instructions align
// the products of eight neighbouring codes to the largest of them and cut them 13 bits below its exponent (measured; the sums of
// eight are then added in 24 bits): 1.4e-5 of the result's norm on normally distributed codes, a hundredth of a 16-bit result's rounding but
// two hundred of a 32-bit one's.  Its FP16 instructions, at half the rate, do not, and FP16 holds every E4M3 code: `WIDE`.
template <bool WIDE> struct Fragment {
    typedef v8i32 type;
    static __device__ __forceinline__ type of(v8i32 codes) { return codes; }
    static __device__ __forceinline__ v4f32 product(const type& x, const type& y) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, v4f32{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
    }
};
template <> struct Fragment<true> {
    struct type { v8f16 part[4]; };
    static __device__ __forceinline__ type of(v8i32 codes) {
        type f;
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v2f16 two = (q & 1) ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[2 * p + (q >> 1)], 1.0f, true)
                                          : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[2 * p + (q >> 1)], 1.0f, false);
                f.part[p][2 * q] = two[0];
                f.part[p][2 * q + 1] = two[1];
            }
        return f;
    }
    static __device__ __forceinline__ v4f32 product(const type& x, const type& y) {
        v4f32 t = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int p = 0; p < 4; ++p) t = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.part[p], y.part[p], t, 0, 0, 0);
        return t;
    }
};

struct TileOperand {
    const uint8_t* vectors;      // the tile's first vector
    int64_t stride;              // bytes
    int rows;                    // vectors from there to the matrix's last, at least 1
    const float* scales;         // FP8: of the tile's first vector (or block of vectors) in inner block 0
    int64_t scale_stride;        // between inner blocks
};

// four neighbouring elements of a row of D, the first `left` of them; `wide`: D's rows start at multiples of four elements
template <typename T>
__device__ __forceinline__ void put_four(T* at, v4f32 v, int64_t left, bool wide, bool accumulate) {
    typedef T four __attribute__((ext_vector_type(4)));
    if (wide && left >= 4) {
        if (accumulate) {
            const four old = *reinterpret_cast<const four*>(at);
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] += (float)old[r];
        }
        *reinterpret_cast<four*>(at) = four{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < left) at[r] = (T)(accumulate ? v[r] + (float)at[r] : v[r]);
    }
}

// Waits until at most N vector-memory operations of this wave are outstanding and its LDS operations are done, then meets the others.
template <int N>
__device__ __forceinline__ void tile_wait() {
    static_assert(N >= 0 && N < 64, "range of the counter");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | 0x0070);   // vmcnt(N) expcnt(7) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// WN x WM waves, each FN x FM tiles of 16 x 16
template <int KIND, int WN_, int WM_, int FN_, int FM_, int NST_>
struct Tile {
    static constexpr bool FP8 = KIND < KIND_BF16, WIDE = KIND == KIND_WIDE_BLOCKS || KIND == KIND_WIDE_VECTORS;
    static constexpr bool BLOCKS = KIND == KIND_FP8_BLOCKS || KIND == KIND_WIDE_BLOCKS;
    static constexpr int WN = WN_, WM = WM_, FN = FN_, FM = FM_, NST = NST_;
    static constexpr int WAVES = WN * WM, THREADS = 64 * WAVES, TN = WN * FN * 16, TM = WM * FM * 16, ROWS = TN + TM;
    static constexpr int SCALE_BYTES = FP8 ? (ROWS * 4 + 255) / 256 * 256 : 0;
    static constexpr int STAGE_BYTES = ROWS * STEP_BYTES + SCALE_BYTES;
    static constexpr int LDS_BYTES = NST * STAGE_BYTES;
    static constexpr int PIECE_LOADS = ROWS / 8, SCALE_LOADS = SCALE_BYTES / 256;                  // wave instructions of a stage
    static constexpr int LPW = (PIECE_LOADS + WAVES - 1) / WAVES, SPW = (SCALE_LOADS + WAVES - 1) / WAVES;
    static_assert((WN * FN * 16) % 8 == 0, "");

    // acc[i][j][r] += X row wn * FN * 16 + 16 i + 4 (lane / 16) + r  times  Y row wm * FM * 16 + 16 j + lane % 16, over the steps
    // [step0, step1) of vectors of `bytes` bytes.  Ends with nothing in flight and all waves past their last LDS read.
    __device__ static void multiply(uint8_t* lds, const TileOperand& X, const TileOperand& Y, int64_t bytes, int step0, int step1,
                                    v4f32 (&acc)[FN][FM]) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wn = wave / WM, wm = wave % WM;
        const int steps = step1 - step0;
        const int64_t rest = bytes - (int64_t)(step1 - 1) * STEP_BYTES;
        const int last_bytes = rest < STEP_BYTES ? (int)rest : STEP_BYTES;              // of the last step
        const bool ragged = last_bytes < STEP_BYTES;

        // what this lane loads: LPW pieces, at `from` (uniform) + voff, and SPW scales
        unsigned voff[LPW];
        const uint8_t* from[LPW];
        int to[LPW];
        {
            const int r = lane >> 3;
#pragma unroll
            for (int i = 0; i < LPW; ++i) {
                int at = wave * LPW + i;
                at = at < PIECE_LOADS ? at : PIECE_LOADS - 1;                           // (the same bytes to the same place twice)
                const bool x = at * 8 < TN;
                const int row = at * 8 + r, mine = x ? row : row - TN, rows = x ? X.rows : Y.rows;
                const unsigned piece = (lane & 7) ^ ((row >> 1) & 7);
                voff[i] = (unsigned)(mine < rows ? mine : rows - 1) * (unsigned)(x ? X.stride : Y.stride) + piece * 16;
                from[i] = (x ? X.vectors : Y.vectors) + (int64_t)step0 * STEP_BYTES;
                to[i] = at * 1024;
            }
        }
        const float* sfrom[SPW > 0 ? SPW : 1];
        int64_t sstride[SPW > 0 ? SPW : 1];
        int sto[SPW > 0 ? SPW : 1];
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < SPW; ++i) {
                int at = wave * SPW + i;
                at = at < SCALE_LOADS ? at : SCALE_LOADS - 1;
                const int row = at * 64 + lane < ROWS ? at * 64 + lane : ROWS - 1;
                const bool x = row < TN;
                const int mine = x ? row : row - TN, rows = x ? X.rows : Y.rows, real = mine < rows ? mine : rows - 1;
                const int index = x && BLOCKS ? real / SCALE_BLOCK : real;
                sfrom[i] = (x ? X.scales + (int64_t)step0 * X.scale_stride : Y.scales + (int64_t)step0 * Y.scale_stride) + index;
                sstride[i] = x ? X.scale_stride : Y.scale_stride;
                sto[i] = ROWS * STEP_BYTES + at * 256;
            }
        }
        int issue_buf = 0;
        auto issue_scales = [&]() {
            if constexpr (FP8) {
#pragma unroll
                for (int i = 0; i < SPW; ++i) {
                    __builtin_amdgcn_global_load_lds(OZAKI_TILE_GPTR(sfrom[i]), OZAKI_TILE_LPTR(lds + issue_buf * STAGE_BYTES + sto[i]), 4, 0, 0);
                    sfrom[i] += sstride[i];
                }
            }
        };
        auto issue_full = [&]() {
#pragma unroll
            for (int i = 0; i < LPW; ++i) {
                __builtin_amdgcn_global_load_lds(OZAKI_TILE_GPTR(from[i] + voff[i]), OZAKI_TILE_LPTR(lds + issue_buf * STAGE_BYTES + to[i]), 16, 0, 0);
                from[i] += STEP_BYTES;
            }
            issue_scales();
            issue_buf = issue_buf + 1 == NST ? 0 : issue_buf + 1;
        };
        // the last step, or (none) none at all: loads that keep the count of those in flight even
        auto issue_last = [&](bool none) {
#pragma unroll
            for (int i = 0; i < LPW; ++i) {
                int at = wave * LPW + i;
                at = at < PIECE_LOADS ? at : PIECE_LOADS - 1;
                const int piece = (lane & 7) ^ (((at * 8 + (lane >> 3)) >> 1) & 7);
                const uint8_t* src = none || piece * 16 >= last_bytes ? no_elements : from[i] + voff[i];
                __builtin_amdgcn_global_load_lds(OZAKI_TILE_GPTR(src), OZAKI_TILE_LPTR(lds + issue_buf * STAGE_BYTES + to[i]), 16, 0, 0);
            }
            if constexpr (FP8) {
#pragma unroll
                for (int i = 0; i < SPW; ++i) {
                    const float* src = none ? reinterpret_cast<const float*>(no_elements) : sfrom[i];
                    __builtin_amdgcn_global_load_lds(OZAKI_TILE_GPTR(src), OZAKI_TILE_LPTR(lds + issue_buf * STAGE_BYTES + sto[i]), 4, 0, 0);
                }
            }
            issue_buf = issue_buf + 1 == NST ? 0 : issue_buf + 1;
        };

        const int frow = lane & 15, g = lane >> 4, fsw = (frow >> 1) & 7;
        const int piece0 = (g ^ fsw) << 4, piece1 = ((g + 4) ^ fsw) << 4;
        const int xbase = (wn * FN * 16 + frow) * STEP_BYTES, ybase = (TN + wm * FM * 16 + frow) * STEP_BYTES;
        int read_buf = 0;
        auto fragment = [&](const uint8_t* at) -> v8i32 {
            const v4i32 lo = *reinterpret_cast<const v4i32*>(at + piece0), hi = *reinterpret_cast<const v4i32*>(at + piece1);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        auto compute = [&]() {
            const uint8_t* const stage = lds + read_buf * STAGE_BYTES;
            typedef typename Fragment<WIDE>::type operand;
            operand y[FM];
#pragma unroll
            for (int j = 0; j < FM; ++j) y[j] = Fragment<WIDE>::of(fragment(stage + ybase + j * 16 * STEP_BYTES));
            if constexpr (FP8) {
                const float* const scales = reinterpret_cast<const float*>(stage + ROWS * STEP_BYTES);
                float sy[FM];
#pragma unroll
                for (int j = 0; j < FM; ++j) sy[j] = scales[TN + (wm * FM + j) * 16 + frow];
                if constexpr (BLOCKS) {
                    // the wave's rows lie in one block of 128 vectors
                    static_assert(SCALE_BLOCK % (FN * 16) == 0, "");
                    const float sx = scales[wn * FN * 16];
#pragma unroll
                    for (int j = 0; j < FM; ++j) sy[j] *= sx;
                }
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    const operand x = Fragment<WIDE>::of(fragment(stage + xbase + i * 16 * STEP_BYTES));
                    v4f32 sx = {};
                    if constexpr (!BLOCKS) sx = *reinterpret_cast<const v4f32*>(scales + (wn * FN + i) * 16 + 4 * g);
#pragma unroll
                    for (int j = 0; j < FM; ++j) {
                        const v4f32 t = Fragment<WIDE>::product(x, y[j]);
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[i][j][r] = __builtin_fmaf(t[r], BLOCKS ? sy[j] : sx[r] * sy[j], acc[i][j][r]);
                    }
                    if constexpr (WIDE) __builtin_amdgcn_sched_barrier(0);              // no second row's fragment beside this one: registers
                }
            } else {
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    const v8i32 x = fragment(stage + xbase + i * 16 * STEP_BYTES);
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int j = 0; j < FM; ++j) {
                            const v4i32 xh = h ? __builtin_shufflevector(x, x, 4, 5, 6, 7) : __builtin_shufflevector(x, x, 0, 1, 2, 3);
                            const v4i32 yh = h ? __builtin_shufflevector(y[j], y[j], 4, 5, 6, 7) : __builtin_shufflevector(y[j], y[j], 0, 1, 2, 3);
                            if constexpr (KIND == KIND_BF16)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf16, xh), __builtin_bit_cast(v8bf16, yh), acc[i][j], 0, 0, 0);
                            else
                                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8f16, xh), __builtin_bit_cast(v8f16, yh), acc[i][j], 0, 0, 0);
                        }
                }
            }
            read_buf = read_buf + 1 == NST ? 0 : read_buf + 1;
        };

        // NST - 1 steps are in flight; step s is awaited, everybody is then done with step s - 1, and its buffer takes step s + NST - 1
#pragma unroll
        for (int s = 0; s < NST - 1; ++s) {
            if (s + 1 < steps || (s + 1 == steps && !ragged)) issue_full();
            else issue_last(s + 1 > steps);
        }
        int s = 0;
        for (; s + NST < steps; ++s) {
            tile_wait<(NST - 2) * (LPW + SPW)>();
            issue_full();
            compute();
        }
        for (; s < steps; ++s) {
            tile_wait<(NST - 2) * (LPW + SPW)>();
            const int next = s + NST - 1;
            if (next + 1 == steps && !ragged) issue_full();
            else issue_last(next >= steps);
            if (s + 1 == steps && (last_bytes & 15) != 0) {
                // the end lies inside a piece
                for (int row = tid; row < ROWS; row += THREADS) {
                    uint8_t* const at = lds + read_buf * STAGE_BYTES + row * STEP_BYTES + (((last_bytes >> 4) ^ ((row >> 1) & 7)) << 4);
                    for (int b = last_bytes & 15; b < 16; ++b) at[b] = 0;
                }
                tile_wait<(NST - 1) * (LPW + SPW)>();
            }
            compute();
        }
        tile_wait<0>();
    }
};

}  // namespace
}  // namespace ozaki
