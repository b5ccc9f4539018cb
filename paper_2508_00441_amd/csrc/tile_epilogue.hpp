// What becomes of a tile that tile_product.hpp has left: through LDS to rows of 16-byte pieces, with whatever happens to the elements on the way.
#pragma once
#include "block_operators.hpp"
#include "tile_product.hpp"

namespace ozaki {
namespace {

// A share of the inner dimension: sums as they are, [share][m][n in fours], a pair's second factor behind all shares of the first.
struct Partial {
    float* to;
    int64_t ld, second;
    static constexpr bool wide = true;
    typedef float eight;             // (nothing beside the sums)
    __device__ __forceinline__ float columns(int64_t) const { return 0.0f; }
    __device__ __forceinline__ float column(int64_t) const { return 0.0f; }
    __device__ __forceinline__ float ahead(int64_t, int64_t) const { return 0.0f; }
    template <typename V> __device__ __forceinline__ void put(int64_t at, V v) const { *reinterpret_cast<V*>(to + at) = v; }
    __device__ __forceinline__ void piece(int64_t m, int64_t c, v8f32 v, v8f32 u, float, float) const {
        const int64_t at = m * ld + c;
        put(at, __builtin_shufflevector(v, v, 0, 1, 2, 3));
        put(at + 4, __builtin_shufflevector(v, v, 4, 5, 6, 7));
        if (second == 0) return;
        put(at + second, __builtin_shufflevector(u, u, 0, 1, 2, 3));
        put(at + second + 4, __builtin_shufflevector(u, u, 4, 5, 6, 7));
    }
    __device__ __forceinline__ void one(int64_t m, int64_t c, float v, float u) const {
        to[m * ld + c] = v;
        if (second != 0) to[m * ld + c + second] = u;
    }
    template <int N> __device__ __forceinline__ void rows(int64_t m0, const int (&m)[N], unsigned there, int64_t c, float (&v)[N], const float (&u)[N], float) const {
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (there >> q & 1) one(m0 + m[q], c, v[q], u[q]);
    }
};

// The tile that P::multiply has left goes through LDS, 16 rows of every wave at a time in 32 bits: from there eight neighbouring columns are a
// thread's, so that rows are read and written in 16-byte pieces of neighbouring lanes.  Where matrices' rows are not aligned to that, a thread has a column (100 x 5001 x 2048: 12.3 us,
// in pieces that lie anywhere 13.1).
template <typename P, typename E>
__device__ __forceinline__ void put_tile(uint8_t* lds, const v4f32 (&acc)[P::FN][P::FM], int64_t m0, int64_t n0, int64_t left_m, int64_t left_n, const E& e) {
    constexpr int COLUMNS = P::PAIR ? P::TN / 2 : P::TN, STRIDE = P::TN * 4 + 16, PIECES = COLUMNS / 8, ROWS = P::WM * 16, HALF = P::PAIR ? P::FN / 2 : P::FN;
    static_assert(ROWS * STRIDE <= P::LDS_BYTES && P::THREADS % PIECES == 0 && P::THREADS % COLUMNS == 0, "");
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wn = wave / P::WM, wm = wave % P::WM;
    const int columns = left_n < COLUMNS ? (int)left_n : COLUMNS, whole = e.wide ? columns / 8 * 8 : 0;
#pragma unroll
    for (int j = 0; j < P::FM; ++j) {
        uint8_t* const mine = lds + (wm * 16 + (lane & 15)) * STRIDE + (wn * HALF * 16 + 4 * (lane >> 4)) * 4;
#pragma unroll
        for (int i = 0; i < P::FN; ++i) *reinterpret_cast<v4f32*>(mine + (i < HALF ? i * 64 : COLUMNS * 4 + (i - HALF) * 64)) = acc[i][j];
        __syncthreads();
        const auto row_of = [&](int r) { return ((r >> 4) * P::FM + j) * 16 + (r & 15); };
        const int column = threadIdx.x % PIECES * 8;
        if (column < whole) {
            constexpr int APART = P::THREADS / PIECES, EACH = ROWS < APART ? 1 : ROWS / APART, AT_ONCE = P::PAIR ? 1 : EACH < 4 ? EACH : 4;
            static_assert(EACH % AT_ONCE == 0, "");
            const auto bias = e.columns(n0 + column);
#pragma unroll 1
            for (int first = threadIdx.x / PIECES; first < ROWS; first += AT_ONCE * APART) {
                typename E::eight ahead[AT_ONCE];
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q) {
                    const int m = row_of(first + q * APART);
                    ahead[q] = e.ahead(m0 + (m < left_m ? m : 0), n0 + column);
                }
#pragma unroll
                for (int q = 0; q < AT_ONCE; ++q) {
                    const int r = first + q * APART;
                    const int m = row_of(r);
                    if (m >= left_m) continue;
                    const v4f32* const from = reinterpret_cast<const v4f32*>(lds + r * STRIDE + column * 4);
                    const v8f32 v = __builtin_shufflevector(from[0], from[1], 0, 1, 2, 3, 4, 5, 6, 7);
                    v8f32 u = {};
                    if (P::PAIR) u = __builtin_shufflevector(from[COLUMNS / 4], from[COLUMNS / 4 + 1], 0, 1, 2, 3, 4, 5, 6, 7);
                    e.piece(m0 + m, n0 + column, v, u, bias, ahead[q]);
                }
            }
        }
        const int c = whole + threadIdx.x % COLUMNS;
        if (c < columns) {
            constexpr int APART = P::THREADS / COLUMNS, N = P::PAIR && P::TM == 256 ? 4 : 8;       // (of registers for eight the largest tiles leave too few)
            const float bias = e.column(n0 + c);
#pragma unroll 1
            for (int first = threadIdx.x / COLUMNS; first < ROWS; first += N * APART) {
                int m[N];
                unsigned there = 0;
                float v[N], u[N];
#pragma unroll
                for (int q = 0; q < N; ++q) {
                    const int r = first + q * APART < ROWS ? first + q * APART : 0;
                    m[q] = row_of(r);
                    there |= first + q * APART < ROWS && m[q] < left_m ? 1u << q : 0u;
                    const float* const from = reinterpret_cast<const float*>(lds + r * STRIDE) + c;
                    v[q] = from[0];
                    u[q] = P::PAIR ? from[COLUMNS] : 0.0f;
                }
                e.rows(m0, m, there, n0 + c, v, u, bias);
            }
        }
        __syncthreads();
    }
}

// A result as it is, rounded once.
template <typename T, bool STREAMED> struct Plain {
    typedef float eight;
    T* to;
    int64_t ld;
    bool wide;
    __device__ __forceinline__ Plain(T* D, int64_t ldd) : to(D), ld(ldd), wide(rows_aligned(D, ldd)) {}
    __device__ __forceinline__ float columns(int64_t) const { return 0.0f; }
    __device__ __forceinline__ float column(int64_t) const { return 0.0f; }
    __device__ __forceinline__ float ahead(int64_t, int64_t) const { return 0.0f; }
    __device__ __forceinline__ void piece(int64_t m, int64_t c, v8f32 v, v8f32, float, float) const { put_eight<STREAMED>(to + m * ld + c, v); }
    template <int N> __device__ __forceinline__ void rows(int64_t m0, const int (&m)[N], unsigned there, int64_t c, float (&v)[N], const float (&)[N], float) const {
#pragma unroll
        for (int q = 0; q < N; ++q)
            if (there >> q & 1) to[(m0 + m[q]) * ld + c] = (T)v[q];
    }
};

}  // namespace
}  // namespace ozaki
