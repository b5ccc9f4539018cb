// D (+)= the product of two matrices of FP8 E4M3 codes with a scale for each 128 elements of the inner dimension:
//     D[i][j] = sum over blocks b of  Sa[b][i] * Sb[b][j or j / 128] * (sum over e in b of A[i][e] * B[j][e])
// A block's products are summed by the matrix unit in FP32, the blocks' sums by FP32 fused multiply-adds with the product of their two
// scales; D is rounded once.  A D of 16 bits takes the FP8 instructions, a D of 32 bits the FP16 ones (Fragment in tile_product.hpp).
// Few vectors of A are bound by the read of B, many by the matrix unit's issue (4096 x 4096 x 4096: 61 - 63 us, 2.2 PFLOP/s), 32-bit results by the
// vector unit, which widens the codes (16384 x 4096 x 8192: 1.03 - 1.07 ms, 1.03 - 1.07 PFLOP/s).
#include "layout.hpp"
#include "tile_product.hpp"

namespace ozaki {
namespace {

struct GemmFp8Work {
    GemmFp8Args g;
    int steps, splits;
    int tiles_m, tiles_n;
    WorkOrder order;
};

template <typename P, int TYPE>
__device__ __forceinline__ void gemm_fp8_body(const GemmFp8Work& w) {
    typedef typename Element<TYPE>::type T;
    __shared__ __attribute__((aligned(16))) uint8_t lds[P::LDS_BYTES];
    const GemmFp8Args& a = w.g;
    const WorkItem item = work_item(blockIdx.x, gridDim.x, w.order, w.tiles_m, w.tiles_n);
    const int64_t m0 = (int64_t)item.bm * P::TM, n0 = (int64_t)item.bn * P::TN;
    const int64_t left_m = a.m - m0, left_n = a.n - n0;
    constexpr bool BLOCKS = P::BLOCKS;
    const TileOperand X{a.B + n0 * a.ldb, a.ldb, (int)(left_n < P::TN ? left_n : P::TN), a.Sb + (BLOCKS ? n0 / SCALE_BLOCK : n0), a.ldsb};
    const TileOperand Y{a.A + m0 * a.lda, a.lda, (int)(left_m < P::TM ? left_m : P::TM), a.Sa + m0, a.ldsa};
    const int split = item.gi;
    v4f32 acc[P::FN][P::FM] = {};
    P::multiply(lds, X, Y, a.k, split_begin(w.steps, w.splits, split), split_begin(w.steps, w.splits, split + 1), acc);

    const auto one = [](int64_t) { return 1.0f; };
    if (w.splits > 1)
        store_tile<P, false>(lds, acc, a.partial + ((int64_t)split * a.m + m0) * in_fours(a.n) + n0, in_fours(a.n), left_m, in_fours(left_n), false, one);
    else
        store_tile<P, (P::THREADS > 256)>(lds, acc, static_cast<T*>(a.D) + m0 * a.ldd + n0, a.ldd, left_m, left_n, a.accumulate != 0, one);
}

template <int TYPE, int SCALING> constexpr int kind_of() {
    return TYPE == TYPE_F32 ? (SCALING == SCALE_BLOCKS ? KIND_WIDE_BLOCKS : KIND_WIDE_VECTORS) : (SCALING == SCALE_BLOCKS ? KIND_FP8_BLOCKS : KIND_FP8_VECTORS);
}

template <int SCALING, int TYPE>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) gemm_fp8_large_kernel(const GemmFp8Work w) {
    gemm_fp8_body<PairedTile<kind_of<TYPE, SCALING>()>, TYPE>(w);
}
template <int SCALING, int TYPE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) gemm_fp8_middle_kernel(const GemmFp8Work w) {
    gemm_fp8_body<Tile<kind_of<TYPE, SCALING>(), 2, 2, 4, 4, 2>, TYPE>(w);
}
template <int SCALING, int TYPE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) gemm_fp8_small_kernel(const GemmFp8Work w) {
    gemm_fp8_body<Tile<kind_of<TYPE, SCALING>(), 2, 2, 2, 2, 3>, TYPE>(w);
}

// Up to sixteen vectors of A: no tile in LDS.  A workgroup of FEW_WAVES waves takes sixteen vectors of B, a wave every FEW_WAVES-th step, straight
// from memory into registers; the waves' sums are added in LDS, in their order.  B is read once and bounds it.  A wave has AHEAD steps (2 KiB of B
// each) under way.  1 x 8192 x 4096: 8.0 us; by 16 x 64 tiles with the inner dimension in shares that meet in memory 11.6 us.  1 x 16384 x 16384: 53 us,
// 5.1 TB/s.
constexpr int FEW = 16, FEW_WAVES = 8, AHEAD = 4;

struct FewPieces {
    v4i32 x[AHEAD][2], y[AHEAD][2];
    const uint8_t* x_at;         // this lane's vector, from piece lane / 16 on
    const uint8_t* y_at;
    int64_t bytes;
    int g, steps;
    __device__ __forceinline__ FewPieces(const TileOperand& X, const TileOperand& Y, int64_t bytes_, int lane)
        : bytes(bytes_), g(lane >> 4), steps((int)div_up(bytes_, STEP_BYTES)) {
        const int row = lane & 15;
        x_at = X.vectors + (int64_t)(row < X.rows ? row : X.rows - 1) * X.stride + g * 16;
        y_at = Y.vectors + (int64_t)(row < Y.rows ? row : Y.rows - 1) * Y.stride + g * 16;
    }
    // (behind the end of the vectors something that is there is read and not used)
    __device__ __forceinline__ void load(int u, int s) {
        const int64_t at = (int64_t)s * STEP_BYTES;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t from = at + g * 16 + h * 64 < bytes ? at + h * 64 : -(int64_t)g * 16;
            x[u][h] = *reinterpret_cast<const v4i32*>(x_at + from);
            y[u][h] = *reinterpret_cast<const v4i32*>(y_at + from);
        }
    }
    __device__ __forceinline__ void clear_end(int u, int s) {
        if ((int64_t)(s + 1) * STEP_BYTES <= bytes) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int left = (int)(bytes - (int64_t)s * STEP_BYTES) - g * 16 - h * 64, keep = left < 0 ? 0 : left;
            x[u][h] = first_bytes(x[u][h], keep);
            y[u][h] = first_bytes(y[u][h], keep);
        }
    }
};

// the sum over a workgroup's waves of element (vector m of Y, n of X) of their products, for thread 16 m + n < 256
__device__ __forceinline__ float few_sum(v4f32 (&sums)[FEW_WAVES][64], v4f32 mine) {
    sums[threadIdx.x >> 6][threadIdx.x & 63] = mine;
    __syncthreads();
    const int n = threadIdx.x & 15, m = (threadIdx.x >> 4) & 15;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w) sum += reinterpret_cast<const float*>(&sums[w][(n >> 2) * 16 + m])[n & 3];
    return sum;
}

template <int SCALING, int TYPE>
__global__ void __launch_bounds__(FEW_WAVES * 64) gemm_fp8_few_kernel(const GemmFp8Args a, const int splits) {
    typedef typename Element<TYPE>::type T;
    typedef Fragment<TYPE == TYPE_F32> F;
    __shared__ __attribute__((aligned(16))) v4f32 sums[FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int split = blockIdx.x % splits;
    const int64_t n0 = (int64_t)(blockIdx.x / splits) * 16;
    const int left_n = a.n - n0 < 16 ? (int)(a.n - n0) : 16;
    FewPieces p(TileOperand{a.B + n0 * a.ldb, a.ldb, left_n, nullptr, 0}, TileOperand{a.A, a.lda, (int)a.m, nullptr, 0}, a.k, lane);
    const int begin = split_begin(p.steps, splits, split), end = split_begin(p.steps, splits, split + 1);
    const float* const sx_at = SCALING == SCALE_BLOCKS ? a.Sb + n0 / SCALE_BLOCK : a.Sb + n0;
    const float* const sy_at = a.Sa + ((lane & 15) < a.m ? lane & 15 : a.m - 1);
    int four[4];                                     // this lane's four columns of the result
#pragma unroll
    for (int r = 0; r < 4; ++r) four[r] = 4 * g + r < left_n ? 4 * g + r : left_n - 1;
    v4f32 sx[AHEAD];
    float sy[AHEAD];
    auto load = [&](int u, int s) {
        s = s < end ? s : end - 1;
        p.load(u, s);
        sy[u] = sy_at[s * a.ldsa];
        if constexpr (SCALING == SCALE_BLOCKS) {
            sx[u][0] = sx_at[s * a.ldsb];
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) sx[u][r] = sx_at[s * a.ldsb + four[r]];
        }
    };
    v4f32 acc = {};
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(u, begin + wave + u * FEW_WAVES);
    for (int first = begin + wave; first < end; first += FEW_WAVES * AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int s = first + u * FEW_WAVES;
            if (s >= end) break;
            p.clear_end(u, s);
            const v4f32 t = F::product(F::of(__builtin_shufflevector(p.x[u][0], p.x[u][1], 0, 1, 2, 3, 4, 5, 6, 7)),
                                       F::of(__builtin_shufflevector(p.y[u][0], p.y[u][1], 0, 1, 2, 3, 4, 5, 6, 7)));
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[r] = __builtin_fmaf(t[r], sx[u][SCALING == SCALE_BLOCKS ? 0 : r] * sy[u], acc[r]);
            if (first + FEW_WAVES * AHEAD < end) load(u, s + FEW_WAVES * AHEAD);
        }
    }
    const float sum = few_sum(sums, acc);
    const int n = threadIdx.x & 15, m = threadIdx.x >> 4;
    if (threadIdx.x >= 256 || m >= a.m || n >= left_n) return;
    if (splits > 1) {
        a.partial[((int64_t)split * a.m + m) * in_fours(a.n) + n0 + n] = sum;
        return;
    }
    T* const to = static_cast<T*>(a.D) + m * a.ldd + n0 + n;
    *to = (T)(a.accumulate ? (float)*to + sum : sum);
}

// sums the pieces of the inner dimension in their order
template <int TYPE>
__global__ void __launch_bounds__(256) gemm_fp8_join_kernel(const GemmFp8Args a, const int splits) {
    typedef typename Element<TYPE>::type T;
    const int64_t j = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, i = blockIdx.y, ld = in_fours(a.n);
    if (j >= a.n) return;
    v4f32 sum = {};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) sum += *reinterpret_cast<const v4f32*>(a.partial + ((int64_t)s * a.m + i) * ld + j);
    T* const D = static_cast<T*>(a.D);
    const bool wide = a.ldd % 4 == 0 && reinterpret_cast<uintptr_t>(D) % (4 * sizeof(T)) == 0;
    put_four(D + i * a.ldd + j, sum, a.n - j, wide, a.accumulate != 0);
}

enum { VECTORS, SMALL, MIDDLE, LARGE };
struct Shape { int kind, tm, tn, splits; };
// By how many tiles of 128 x 128 there are for 256 compute units, each of which holds two (times with blocks of scales, 16-bit results, in us):
//     fewer than 256, or up to 64 rows or columns    64 x 64       512 x 4096 x 4096: 17.7, by 128 x 128 23.8;  1000 x 1000 x 1024 (32 bits) 9.1, 16.9
//     up to 512, or up to 128 rows or columns        128 x 128     2048 x 4096 x 4096: 40, by 256 x 256 50;  900 x 4000 x 2048: 17.8, by 64 x 64 20.6
//     more                                           256 x 256     2304 x 4096 x 4096: 51, by 128 x 128 60;  200 x 65536 x 2048: 43, 55
// 32-bit results: no tiles of 256 x 256.  The widened fragments do not fit beside their accumulators, and two workgroups of 128 x 128, which pause
// at different times, do better than one of 256 x 128 (16384 x 4096 x 8192: 1030 and 1080).
// Where 64 x 64 tiles are too few, the inner dimension is cut, into shares of at least four steps (64 x 4096 x 16384: 17.3 for 256 shares in all,
// 18.4 for 512; shares of eight steps: 64 x 2048 x 2048 9.5 against 8.5).  Where few vectors meet few of B: from 96 steps on, into shares
// of at least 32 (1 x 64 x 65536: 7.5, uncut 37.7; 1 x 1024 x 16384: 8.4, 11.9, in shares of 64 steps 10.0; 1 x 2048 x 12288, two shares: 10.9, uncut 11.6;
// but two shares of 1 x 2048 x 8192, 64 steps: 8.1, uncut 7.7).
Shape shape_of(int64_t m, int64_t n, int64_t k) {
    const int64_t steps = div_up(k, SCALE_BLOCK);
    const auto shares = [](int64_t want, int64_t most) {
        const int64_t s = want < most ? want : most;
        return (int)(s < 1 ? 1 : s > 16 ? 16 : s);
    };
    if (m <= FEW) return Shape{VECTORS, FEW, 16, steps < 96 ? 1 : shares(256 / div_up(n, 16), steps / 32)};
    const int64_t middle = div_up(m, 128) * div_up(n, 128), least = m < n ? m : n;
    if (middle >= 256 && least > 64) return middle <= 512 || least <= 128 ? Shape{MIDDLE, 128, 128, 1} : Shape{LARGE, 256, 256, 1};
    return Shape{SMALL, 64, 64, shares(256 / (div_up(m, 64) * div_up(n, 64)), steps / 4)};
}

// Large tiles run in rounds of one for every compute unit.  Where the last round has few of them, the rows or columns of D that they hold, of the
// longer dimension, are left to smaller tiles in a launch of their own, if these run in one round (4608 x 4096 x 4096, 288 tiles: 83 us against 112,
// x 512 27 against 37; 5500 x 4096 x 4096, 352 tiles: 102 against 118).
int64_t in_rounds(int64_t length, int64_t across) {
    const int64_t tiles = across * div_up(length, 256), over = tiles % 256, whole = (tiles - over) / across;
    return over == 0 || whole == 0 || tiles - whole * across > 128 ? length : whole * 256;
}

template <int SCALING, int TYPE>
hipError_t launch_kind(const GemmFp8Args& a, int splits, Shape s, hipStream_t st) {
    GemmFp8Work w;
    w.g = a;
    w.steps = (int)div_up(a.k, SCALE_BLOCK);
    w.splits = splits;
    w.tiles_m = (int)div_up(a.m, s.tm);
    w.tiles_n = (int)div_up(a.n, s.tn);
    const int64_t tiles = (int64_t)w.tiles_m * w.tiles_n;
    w.order = WorkOrder{s.kind == LARGE ? 32 : 64, 8};             // 4096 x 4096 x 4096: 63.1 us, in plain order 63.7; 2048 x 4096 x 4096: 42.7, 43.4
    const unsigned blocks = (unsigned)(tiles * splits);
    if (s.kind == VECTORS) hipLaunchKernelGGL((gemm_fp8_few_kernel<SCALING, TYPE>), dim3(blocks), dim3(FEW_WAVES * 64), 0, st, a, splits);
    else if (s.kind == SMALL) hipLaunchKernelGGL((gemm_fp8_small_kernel<SCALING, TYPE>), dim3(blocks), dim3(256), 0, st, w);
    else if (s.kind == MIDDLE) hipLaunchKernelGGL((gemm_fp8_middle_kernel<SCALING, TYPE>), dim3(blocks), dim3(256), 0, st, w);
    else if constexpr (TYPE != TYPE_F32) hipLaunchKernelGGL((gemm_fp8_large_kernel<SCALING, TYPE>), dim3(blocks), dim3(512), 0, st, w);
    if (splits > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((gemm_fp8_join_kernel<TYPE>), dim3((unsigned)div_up(a.n, 1024), (unsigned)a.m), dim3(256), 0, st, a, splits);
    }
    return hipGetLastError();
}

template <int SCALING, int TYPE>
hipError_t launch_scaled(GemmFp8Args a, int splits, hipStream_t st) {
    const Shape s = shape_of(a.m, a.n, a.k);
    if (s.kind != LARGE) return launch_kind<SCALING, TYPE>(a, splits, s, st);
    if (TYPE == TYPE_F32) return launch_kind<SCALING, TYPE>(a, 1, Shape{MIDDLE, 128, 128, 1}, st);
    const int64_t m = a.m, n = a.n;
    if (m >= n) a.m = in_rounds(m, div_up(n, 256));
    else a.n = in_rounds(n, div_up(m, 256));
    const hipError_t e = launch_kind<SCALING, TYPE>(a, 1, s, st);
    if (e != hipSuccess || (a.m == m && a.n == n)) return e;
    typedef typename Element<TYPE>::type T;
    if (a.m < m) {
        a.A = static_cast<const uint8_t*>(a.A) + a.m * a.lda;
        a.Sa += a.m;
        a.D = static_cast<T*>(a.D) + a.m * a.ldd;
        a.m = m - a.m;
    } else {
        a.B = static_cast<const uint8_t*>(a.B) + a.n * a.ldb;
        a.Sb += SCALING == SCALE_BLOCKS ? a.n / SCALE_BLOCK : a.n;
        a.D = static_cast<T*>(a.D) + a.n;
        a.n = n - a.n;
    }
    return launch_kind<SCALING, TYPE>(a, 1, shape_of(a.m, a.n, a.k), st);
}

template <int TYPE>
__global__ void __launch_bounds__(256) gemm_fp8_empty_kernel(const GemmFp8Args a) {
    typedef typename Element<TYPE>::type T;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < a.m * a.n; at += (int64_t)gridDim.x * 256)
        static_cast<T*>(a.D)[at / a.n * a.ldd + at % a.n] = (T)0.0f;
}

template <int TYPE>
hipError_t launch_typed(const GemmFp8Args& a, int scaling, int splits, hipStream_t st) {
    if (a.k == 0) {
        if (a.accumulate) return hipSuccess;
        hipLaunchKernelGGL((gemm_fp8_empty_kernel<TYPE>), dim3((unsigned)(a.m * a.n < 1 << 24 ? div_up(a.m * a.n, 256) : 1 << 16)), dim3(256), 0, st, a);
        return hipGetLastError();
    }
    return scaling == SCALE_BLOCKS ? launch_scaled<SCALE_BLOCKS, TYPE>(a, splits, st) : launch_scaled<SCALE_VECTORS, TYPE>(a, splits, st);
}

}  // namespace

int gemm_fp8_splits(int64_t m, int64_t n, int64_t k) { return m > 0 && n > 0 && k > 0 ? shape_of(m, n, k).splits : 1; }

hipError_t launch_gemm_fp8(const GemmFp8Args& a, int scaling, int type_d, int splits, hipStream_t st) {
    if (a.m == 0 || a.n == 0) return hipSuccess;
    return type_d == TYPE_F32 ? launch_typed<TYPE_F32>(a, scaling, splits, st) : type_d == TYPE_BF16 ? launch_typed<TYPE_BF16>(a, scaling, splits, st)
                                                                                                    : launch_typed<TYPE_F16>(a, scaling, splits, st);
}

}  // namespace ozaki
