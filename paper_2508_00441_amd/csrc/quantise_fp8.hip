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
// read 2 or 4 bytes per element again to write 1).
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

// eight elements from `at`, which is 16-byte aligned; zeros from element `left` on
template <typename T>
__device__ __forceinline__ void load_eight(const T* at, int64_t left, float (&x)[8]) {
    constexpr int PER = 16 / sizeof(T);
    typedef T piece __attribute__((ext_vector_type(PER)));
#pragma unroll
    for (int p = 0; p < 8 / PER; ++p) {
        piece v = {};
        if (p * PER < left) v = *reinterpret_cast<const piece*>(at + p * PER);
#pragma unroll
        for (int i = 0; i < PER; ++i) x[p * PER + i] = p * PER + i < left ? (float)v[i] : 0.0f;
    }
}

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

// largest of the sixteen lanes of a row
__device__ __forceinline__ float row_max(float a) {
#pragma unroll
    for (int s = 1; s < 16; s <<= 1) a = fmaxf(a, __shfl_xor(a, s, 16));
    return a;
}

// Vectors only: sixteen lanes take 128 elements, a wave four vectors, a workgroup sixteen vectors of one block.
template <int TYPE>
__global__ void __launch_bounds__(256) quantise_vectors_kernel(const QuantiseArgs a) {
    typedef typename Element<TYPE>::type T;
    const int part = threadIdx.x & 15;
    const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), kb = blockIdx.y, e = kb * SCALE_BLOCK + part * 8;
    const bool real = row < a.rows;
    float x[8];
    load_eight(static_cast<const T*>(a.X) + (real ? row : a.rows - 1) * a.ldx + e, a.k - e, x);
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = fmaxf(most, finite_magnitude(x[i]));
    most = fmaxf(row_max(most), SMALLEST_AMAX);
    if (!real) return;
    store_eight(a.Q + row * a.ldq + e, a.k - e, quantised<T>(x, most));
    if (part == 0) a.S[kb * a.lds + row] = most / E4M3_MAX;
}

// A 128 x 128 square: thread (g, part) holds rows 8 g .. 8 g + 7 of columns 8 part .. 8 part + 7.  The eight rows of a column are
// eight bytes of the transposed result, which travels through LDS so that its vectors too are written in 128-byte pieces.
constexpr int TURNED = SCALE_BLOCK + 16;                     // bytes between columns of the transposed tile (16-byte pieces)

template <int TYPE, int SCALING, bool TRANSPOSED>
__global__ void __launch_bounds__(256) quantise_tile_kernel(const QuantiseArgs a) {
    typedef typename Element<TYPE>::type T;
    __shared__ __attribute__((aligned(16))) uint8_t turned[TRANSPOSED ? SCALE_BLOCK * TURNED : 16];
    __shared__ float reduced[16][SCALE_BLOCK];
    const int part = threadIdx.x & 15, g = threadIdx.x >> 4;
    const int64_t row0 = (int64_t)blockIdx.x * SCALE_BLOCK, e0 = (int64_t)blockIdx.y * SCALE_BLOCK;
    const int64_t e = e0 + part * 8, left = a.k - e;
    float x[8][8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + g * 8 + i;
        load_eight(static_cast<const T*>(a.X) + row * a.ldx + e, row < a.rows ? left : 0, x[i]);
    }
    float in_row[8], in_column[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) in_row[i] = in_column[i] = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float m = finite_magnitude(x[i][j]);
            in_row[i] = fmaxf(in_row[i], m);
            in_column[j] = fmaxf(in_column[j], m);
        }
    float of_square = SMALLEST_AMAX;
    if (SCALING == SCALE_BLOCKS || TRANSPOSED) {
#pragma unroll
        for (int j = 0; j < 8; ++j) reduced[g][part * 8 + j] = in_column[j];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float most = 0.0f;
#pragma unroll
            for (int h = 0; h < 16; ++h) most = fmaxf(most, reduced[h][part * 8 + j]);
            in_column[j] = fmaxf(most, SMALLEST_AMAX);
            of_square = fmaxf(of_square, most);
        }
        of_square = row_max(of_square);
    }
    if (a.Q != nullptr) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t row = row0 + g * 8 + i;
            const float most = SCALING == SCALE_BLOCKS ? of_square : fmaxf(row_max(in_row[i]), SMALLEST_AMAX);
            if (row >= a.rows) continue;
            store_eight(a.Q + row * a.ldq + e, left, quantised<T>(x[i], most));
            if (SCALING == SCALE_VECTORS && part == 0) a.S[blockIdx.y * a.lds + row] = most / E4M3_MAX;
        }
        if (SCALING == SCALE_BLOCKS && threadIdx.x == 0) a.S[blockIdx.y * a.lds + blockIdx.x] = of_square / E4M3_MAX;
    }
    if constexpr (TRANSPOSED) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float most = SCALING == SCALE_BLOCKS ? of_square : in_column[j];
            const float column[8] = {x[0][j], x[1][j], x[2][j], x[3][j], x[4][j], x[5][j], x[6][j], x[7][j]};
            *reinterpret_cast<v2i32*>(turned + (part * 8 + j) * TURNED + g * 8) = quantised<T>(column, most);
            if (SCALING == SCALE_VECTORS && g == 0 && j < left) a.St[blockIdx.x * a.ldst + e + j] = most / E4M3_MAX;
        }
        if (SCALING == SCALE_BLOCKS && threadIdx.x == 0) a.St[blockIdx.x * a.ldst + blockIdx.y] = of_square / E4M3_MAX;
        __syncthreads();
        // eight lanes write the 128 bytes of a column
        const int piece = threadIdx.x & 7;
        const int64_t r = row0 + piece * 16;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int column = (threadIdx.x >> 3) + 32 * c;
            if (e0 + column >= a.k || r >= a.rows) continue;
            const uint8_t* from = turned + column * TURNED + piece * 16;
            uint8_t* to = a.Qt + (e0 + column) * a.ldqt + r;
            if (r + 16 <= a.rows) {
                *reinterpret_cast<v4i32*>(to) = *reinterpret_cast<const v4i32*>(from);
            } else {
                for (int i = 0; i < (int)(a.rows - r); ++i) to[i] = from[i];
            }
        }
    }
}

template <int TYPE>
hipError_t launch_typed(const QuantiseArgs& a, int scaling, hipStream_t st) {
    if (scaling == SCALE_VECTORS && a.Qt == nullptr) {
        const dim3 grid((unsigned)div_up(a.rows, 16), (unsigned)div_up(a.k, SCALE_BLOCK));
        hipLaunchKernelGGL((quantise_vectors_kernel<TYPE>), grid, dim3(256), 0, st, a);
        return hipGetLastError();
    }
    const dim3 grid((unsigned)div_up(a.rows, SCALE_BLOCK), (unsigned)div_up(a.k, SCALE_BLOCK));
    if (scaling == SCALE_VECTORS) hipLaunchKernelGGL((quantise_tile_kernel<TYPE, SCALE_VECTORS, true>), grid, dim3(256), 0, st, a);
    else if (a.Qt != nullptr) hipLaunchKernelGGL((quantise_tile_kernel<TYPE, SCALE_BLOCKS, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((quantise_tile_kernel<TYPE, SCALE_BLOCKS, false>), grid, dim3(256), 0, st, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantise_fp8(const QuantiseArgs& a, int type, int scaling, hipStream_t st) {
    if (a.rows == 0 || a.k == 0) return hipSuccess;
    return type == TYPE_F32 ? launch_typed<TYPE_F32>(a, scaling, st) : type == TYPE_BF16 ? launch_typed<TYPE_BF16>(a, scaling, st)
                                                                                         : launch_typed<TYPE_F16>(a, scaling, st);
}

}  // namespace ozaki
