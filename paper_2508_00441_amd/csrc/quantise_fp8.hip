// Quantisation to OCP E4M3 with a 32-bit scale for each block of 128 elements of a vector, or for each 128 x 128 square.
//
// For a block with the largest finite magnitude a (at least 2^-100):
//     scale = a / 448, rounded to 32 bits,     code = E4M3(x * 448 / a), rounded once, to nearest, ties to even.
// 448 is the largest value of E4M3.  The quotient is rounded once (of_block): a tie between two codes is common with 16-bit elements
// (a and x have 8 or 11 significant bits), and x times a rounded 448 / a would decide it by that factor's error.  An element that is not
// finite gets the code NaN and does not count for the scale, so one of them spoils only itself.
//
// The scales lie [block of the inner dimension][vector]: a product's step over 128 elements then reads the scales of neighbouring
// vectors as one contiguous piece.
//
// Bound by memory: the elements are read once, the codes written once.  The transposed result comes from the same read (a second pass would
// read 2 or 4 bytes per element again to write 1).  16384 x 4096 in 32 bits, both ways: 85 us, 4.75 TB/s, what a copy reaches; 8192 x 4096 in 16 bits,
// both ways: 34 us, 4.0 TB/s; one vector of 4096: 2.6 us, a launch's own time.
#include "low_precision.hpp"

namespace ozaki {

namespace {

constexpr float E4M3_MAX = 448.0f;
constexpr float SMALLEST_AMAX = 7.888609052210118e-31f;      // 2^-100

template <typename T>
__device__ __forceinline__ float finite_magnitude(T x) {
    const float a = fabsf((float)x);
    return a < __builtin_inff() ? a : 0.0f;                  // (false for NaN too)
}

// x * 448 / a, in a form that rounds to E4M3 as the exact quotient does: as 0.875 x over 2^-9 a, which cannot overflow.  Division by the
// correctly rounded reciprocal with one correction gives the nearest 32-bit number.  With 16-bit elements 0.875 x is exact and no quotient
// comes so near a tie between two codes without being it; with 32-bit ones it may, and the quotient is then made odd (in its last
// bit) on the side of the exact one, which is never a tie.
struct Divisor {
    float a, inverse;
    __device__ __forceinline__ explicit Divisor(float amax) : a(amax * 0.001953125f), inverse(1.0f / (amax * 0.001953125f)) {}
};
template <typename T>
__device__ __forceinline__ float of_block(float x, const Divisor& d) {
    const float y = x * 0.875f, p = y * d.inverse;
    float r = __builtin_fmaf(-p, d.a, y);
    if constexpr (sizeof(T) == 2) return __builtin_fmaf(r, d.inverse, p);
    const float lost = __builtin_fmaf(x, 0.875f, -y);
    float q = __builtin_fmaf(r + lost, d.inverse, p);
    r = __builtin_fmaf(-q, d.a, y) + lost;
    const int bits = __float_as_int(q);
    if (r != 0.0f && (bits & 1) == 0 && q != 0.0f) q = __int_as_float(bits + ((__float_as_int(r) ^ bits) < 0 ? -1 : 1));
    return q;
}

// codes of eight quotients, the first in the lowest byte
__device__ __forceinline__ v2i32 codes_of(const float (&x)[8]) {
    v2i32 q;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        int w = 0;
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h], x[4 * h + 1], w, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * h + 2], x[4 * h + 3], w, true);
        q[h] = w;
    }
    return q;
}
template <typename T>
__device__ __forceinline__ v2i32 quantised(const float (&x)[8], float amax) {
    const Divisor d(amax);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = of_block<T>(x[i], d);
    return codes_of(y);
}

// eight elements of a vector as they are in memory
template <typename T> struct Eight {
    static constexpr int PER = 16 / sizeof(T), PIECES = 8 / PER;
    typedef T piece __attribute__((ext_vector_type(PER)));
    piece p[PIECES];
    __device__ __forceinline__ float operator[](int i) const { return (float)p[i / PER][i % PER]; }
    // from `at`, which is 16-byte aligned; zeros from element `left` on
    __device__ __forceinline__ void load(const T* at, int64_t left) {
#pragma unroll
        for (int q = 0; q < PIECES; ++q) {
            p[q] = piece{};
            if (q * PER < left) p[q] = *reinterpret_cast<const piece*>(at + q * PER);
            if (left < (q + 1) * PER) {
#pragma unroll
                for (int i = 0; i < PER; ++i)
                    if (q * PER + i >= left) p[q][i] = (T)0.0f;
            }
        }
    }
};

// eight codes to `at`, which is 8-byte aligned, the first `left` of them
__device__ __forceinline__ void store_eight(uint8_t* at, int64_t left, v2i32 q) {
    if (left >= 8) {
        *reinterpret_cast<v2i32*>(at) = q;
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) at[i] = (uint8_t)((unsigned)q[i >> 2] >> (8 * (i & 3)));
    }
}

// largest of the sixteen lanes of a row, and of the same lane of the wave's four rows
template <int CONTROL>
__device__ __forceinline__ float moved(float a) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(a), CONTROL, 0xF, 0xF, true));
}
__device__ __forceinline__ float row_max(float a) {
    a = fmaxf(a, moved<0x128>(a));           // from eight lanes on in the row, round
    a = fmaxf(a, moved<0x124>(a));           // four
    a = fmaxf(a, moved<0x4E>(a));            // two, in fours
    return fmaxf(a, moved<0xB1>(a));
}
__device__ __forceinline__ float column_max(float a) {
    a = fmaxf(a, __shfl_xor(a, 16));
    return fmaxf(a, __shfl_xor(a, 32));
}

// Vectors only: sixteen lanes take 128 elements, a wave four vectors, a workgroup sixteen vectors of one block.
template <int TYPE>
__global__ void __launch_bounds__(256) quantise_vectors_kernel(const QuantiseArgs a, const unsigned blocks_k) {
    typedef typename Element<TYPE>::type T;
    const int part = threadIdx.x & 15;
    const int64_t row = (int64_t)(blockIdx.x / blocks_k) * 16 + (threadIdx.x >> 4), kb = blockIdx.x % blocks_k, e = kb * SCALE_BLOCK + part * 8;
    const bool real = row < a.rows;
    Eight<T> raw;
    raw.load(static_cast<const T*>(a.X) + (real ? row : a.rows - 1) * a.ldx + e, a.k - e);
    float x[8], most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = raw[i];
        most = fmaxf(most, finite_magnitude(x[i]));
    }
    most = fmaxf(row_max(most), SMALLEST_AMAX);
    if (!real) return;
    store_eight(a.Q + row * a.ldq + e, a.k - e, quantised<T>(x, most));
    if (part == 0) a.S[kb * a.lds + row] = most / E4M3_MAX;
}

// A 128 x 128 square: thread (g, part) holds rows 8 g .. 8 g + 7 of columns 8 part .. 8 part + 7, as they are in memory (as 32-bit numbers they
// would leave room for one wave per SIMD, and nothing would cover the loads).  The eight rows of a column are eight bytes of the transposed
// result, which travels through LDS so that its vectors too are written in 128-byte pieces.
// There the eight bytes of column c and rows 8 g lie at c * TURNED + 8 * (g ^ (c / 8)): the sixteen columns that a wave's lanes write to
// together are eight apart, and the pitch alone would put them on four places of the banks.
constexpr int TURNED = SCALE_BLOCK + 8;

template <int TYPE, int SCALING, bool TRANSPOSED>
__global__ void __launch_bounds__(256) quantise_tile_kernel(const QuantiseArgs a, const unsigned blocks_k) {
    typedef typename Element<TYPE>::type T;
    constexpr bool SQUARE = SCALING == SCALE_BLOCKS;
    __shared__ __attribute__((aligned(16))) uint8_t turned[TRANSPOSED ? SCALE_BLOCK * TURNED : 16];
    __shared__ __attribute__((aligned(16))) float of_wave[4][SCALE_BLOCK];
    const int part = threadIdx.x & 15, g = threadIdx.x >> 4, wave = threadIdx.x >> 6;
    const int64_t rb = blockIdx.x / blocks_k, kb = blockIdx.x % blocks_k, row0 = rb * SCALE_BLOCK, e0 = kb * SCALE_BLOCK;
    const int64_t e = e0 + part * 8, left = a.k - e, first_row = row0 + g * 8;
    Eight<T> x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i].load(static_cast<const T*>(a.X) + (first_row + i) * a.ldx + e, first_row + i < a.rows ? left : 0);
    float in_row[8], in_column[8], of_square = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) in_row[i] = in_column[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float m = finite_magnitude(x[i][j]);
            if constexpr (SQUARE) {
                of_square = fmaxf(of_square, m);
            } else {
                in_row[i] = fmaxf(in_row[i], m);
                in_column[j] = fmaxf(in_column[j], m);
            }
        }
    if constexpr (SQUARE) {
        of_square = column_max(row_max(of_square));
        if ((threadIdx.x & 63) == 0) of_wave[0][wave] = of_square;
        __syncthreads();
        const v4f32 all = *reinterpret_cast<const v4f32*>(&of_wave[0][0]);
        of_square = fmaxf(fmaxf(fmaxf(all[0], all[1]), fmaxf(all[2], all[3])), SMALLEST_AMAX);
        if (threadIdx.x == 0) {
            if (a.Q != nullptr) a.S[kb * a.lds + rb] = of_square / E4M3_MAX;
            if (TRANSPOSED) a.St[rb * a.ldst + kb] = of_square / E4M3_MAX;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            in_column[j] = column_max(in_column[j]);
            if ((g & 3) == 0) of_wave[wave][part * 8 + j] = in_column[j];
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4f32 most = {SMALLEST_AMAX, SMALLEST_AMAX, SMALLEST_AMAX, SMALLEST_AMAX};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const v4f32 one = *reinterpret_cast<const v4f32*>(&of_wave[w][part * 8 + 4 * h]);
#pragma unroll
                for (int q = 0; q < 4; ++q) most[q] = fmaxf(most[q], one[q]);
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) in_column[4 * h + q] = most[q];
        }
        if (a.Q != nullptr) {
            float mine = SMALLEST_AMAX;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                in_row[i] = fmaxf(row_max(in_row[i]), SMALLEST_AMAX);
                mine = part == i ? in_row[i] : mine;
            }
            if (part < 8 && first_row + part < a.rows) a.S[kb * a.lds + first_row + part] = mine / E4M3_MAX;
        }
        if (threadIdx.x < SCALE_BLOCK && e0 + threadIdx.x < a.k) {
            float most = SMALLEST_AMAX;
#pragma unroll
            for (int w = 0; w < 4; ++w) most = fmaxf(most, of_wave[w][threadIdx.x]);
            a.St[rb * a.ldst + e0 + threadIdx.x] = most / E4M3_MAX;
        }
    }
    if (a.Q != nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (first_row + i >= a.rows) continue;
            const float row[8] = {x[i][0], x[i][1], x[i][2], x[i][3], x[i][4], x[i][5], x[i][6], x[i][7]};
            store_eight(a.Q + (first_row + i) * a.ldq + e, left, quantised<T>(row, SQUARE ? of_square : in_row[i]));
        }
    }
    if constexpr (TRANSPOSED) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float column[8] = {x[0][j], x[1][j], x[2][j], x[3][j], x[4][j], x[5][j], x[6][j], x[7][j]};
            *reinterpret_cast<v2i32*>(turned + (part * 8 + j) * TURNED + ((g ^ part) << 3)) = quantised<T>(column, SQUARE ? of_square : in_column[j]);
        }
        __syncthreads();
        // eight lanes write the 128 bytes of a column
        const int piece = threadIdx.x & 7;
        const int64_t r = row0 + piece * 16;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int column = (threadIdx.x >> 3) + 32 * c;
            if (e0 + column >= a.k || r >= a.rows) continue;
            const uint8_t* const from = turned + column * TURNED;
            const v2i32 lo = *reinterpret_cast<const v2i32*>(from + (((2 * piece) ^ (column >> 3)) << 3));
            const v2i32 hi = *reinterpret_cast<const v2i32*>(from + (((2 * piece + 1) ^ (column >> 3)) << 3));
            uint8_t* const to = a.Qt + (e0 + column) * a.ldqt + r;
            if (r + 16 <= a.rows) {
                *reinterpret_cast<v4i32*>(to) = v4i32{lo[0], lo[1], hi[0], hi[1]};
            } else {
                store_eight(to, a.rows - r, lo);
                if (r + 8 < a.rows) store_eight(to + 8, a.rows - r - 8, hi);
            }
        }
    }
}

// (one dimension, blocks of the inner dimension fastest: neighbours read neighbouring pieces of the same vectors, and the grid's other dimensions
// end at 65535)
template <int TYPE>
hipError_t launch_typed(const QuantiseArgs& a, int scaling, hipStream_t st) {
    const unsigned blocks_k = (unsigned)div_up(a.k, SCALE_BLOCK);
    if (scaling == SCALE_VECTORS && a.Qt == nullptr) {
        hipLaunchKernelGGL((quantise_vectors_kernel<TYPE>), dim3(blocks_k * (unsigned)div_up(a.rows, 16)), dim3(256), 0, st, a, blocks_k);
        return hipGetLastError();
    }
    const dim3 grid(blocks_k * (unsigned)div_up(a.rows, SCALE_BLOCK));
    if (scaling == SCALE_VECTORS) hipLaunchKernelGGL((quantise_tile_kernel<TYPE, SCALE_VECTORS, true>), grid, dim3(256), 0, st, a, blocks_k);
    else if (a.Qt != nullptr) hipLaunchKernelGGL((quantise_tile_kernel<TYPE, SCALE_BLOCKS, true>), grid, dim3(256), 0, st, a, blocks_k);
    else hipLaunchKernelGGL((quantise_tile_kernel<TYPE, SCALE_BLOCKS, false>), grid, dim3(256), 0, st, a, blocks_k);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantise_fp8(const QuantiseArgs& a, int type, int scaling, hipStream_t st) {
    if (a.rows == 0 || a.k == 0) return hipSuccess;
    return type == TYPE_F32 ? launch_typed<TYPE_F32>(a, scaling, st) : type == TYPE_BF16 ? launch_typed<TYPE_BF16>(a, scaling, st)
                                                                                         : launch_typed<TYPE_F16>(a, scaling, st);
}

}  // namespace ozaki
