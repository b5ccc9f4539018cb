// D (+)= the product of two matrices of FP8 E4M3 codes with a scale for each 128 elements of the inner dimension:
//     D[i][j] = sum over blocks b of  Sa[b][i] * Sb[b][j or j / 128] * (sum over e in b of A[i][e] * B[j][e])
// A block's products are summed by the matrix unit in FP32, the blocks' sums by FP32 fused multiply-adds with the product of their two
// scales; D is rounded once.  A D of 16 bits takes the FP8 instructions, a D of 32 bits the FP16 ones (Fragment in tile_product.hpp).
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

__device__ __forceinline__ int split_begin(int steps, int splits, int s) { return (int)((int64_t)steps * s / splits); }

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
        store_tile<P, false>(lds, acc, a.partial + ((int64_t)split * a.m + m0) * a.n + n0, a.n, left_m, left_n, false, one);
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
// 256 x 128 for 32-bit results: the widened fragments of 256 x 256 do not fit beside its accumulators
template <int SCALING>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) gemm_fp8_wide_kernel(const GemmFp8Work w) {
    gemm_fp8_body<Tile<kind_of<TYPE_F32, SCALING>(), 4, 2, 4, 4, 3>, TYPE_F32>(w);
}
template <int SCALING, int TYPE>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) gemm_fp8_middle_kernel(const GemmFp8Work w) {
    gemm_fp8_body<Tile<kind_of<TYPE, SCALING>(), 2, 2, 4, 4, 2>, TYPE>(w);
}
template <int SCALING, int TYPE>
__global__ void __launch_bounds__(256) gemm_fp8_few_kernel(const GemmFp8Work w) {
    gemm_fp8_body<Tile<kind_of<TYPE, SCALING>(), 4, 1, 1, 1, 6>, TYPE>(w);
}

// sums the pieces of the inner dimension in their order
template <int TYPE>
__global__ void __launch_bounds__(256) gemm_fp8_join_kernel(const GemmFp8Args a, const int splits) {
    typedef typename Element<TYPE>::type T;
    const int64_t j = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, i = blockIdx.y;
    if (j >= a.n) return;
    v4f32 sum = {};
    if (a.n % 4 == 0) {
        for (int s = 0; s < splits; ++s) sum += *reinterpret_cast<const v4f32*>(a.partial + ((int64_t)s * a.m + i) * a.n + j);
    } else {
        for (int s = 0; s < splits; ++s)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (j + r < a.n) sum[r] += a.partial[((int64_t)s * a.m + i) * a.n + j + r];
    }
    T* const D = static_cast<T*>(a.D);
    const bool wide = a.ldd % 4 == 0 && reinterpret_cast<uintptr_t>(D) % (4 * sizeof(T)) == 0;
    put_four(D + i * a.ldd + j, sum, a.n - j, wide, a.accumulate != 0);
}

constexpr int FEW = 16;                   // vectors of A up to which the kernel for few of them runs
struct Shape { int tm, tn, splits; };
Shape shape_of(int64_t m, int64_t n, int64_t k) {
    const int64_t steps = div_up(k, SCALE_BLOCK);
    Shape s{256, 256, 1};
    if (m <= FEW) s = {16, 64, 1};
    else if (div_up(m, 256) * div_up(n, 256) < 192) s = {128, 128, 1};
    if (s.tm < 256) {
        const int64_t tiles = div_up(m, s.tm) * div_up(n, s.tn), want = 512 / tiles;
        int64_t splits = want < steps / 4 ? want : steps / 4;
        s.splits = (int)(splits < 1 ? 1 : splits > 16 ? 16 : splits);
    }
    return s;
}

template <int SCALING, int TYPE>
hipError_t launch_kind(const GemmFp8Args& a, int splits, hipStream_t st) {
    const Shape s = shape_of(a.m, a.n, a.k);
    GemmFp8Work w;
    w.g = a;
    w.steps = (int)div_up(a.k, SCALE_BLOCK);
    w.splits = splits;
    const int tm = TYPE == TYPE_F32 && s.tm == 256 ? 128 : s.tm;
    w.tiles_m = (int)div_up(a.m, tm);
    w.tiles_n = (int)div_up(a.n, s.tn);
    const int64_t tiles = (int64_t)w.tiles_m * w.tiles_n;
        w.order = tiles * splits >= 512 ? WorkOrder{32, w.tiles_m > 8 ? 4 : 8} : WorkOrder{0, 0};
    const unsigned blocks = (unsigned)(tiles * splits);
    if (s.tm == 16) hipLaunchKernelGGL((gemm_fp8_few_kernel<SCALING, TYPE>), dim3(blocks), dim3(256), 0, st, w);
    else if (s.tm == 128) hipLaunchKernelGGL((gemm_fp8_middle_kernel<SCALING, TYPE>), dim3(blocks), dim3(256), 0, st, w);
    else if constexpr (TYPE == TYPE_F32) hipLaunchKernelGGL((gemm_fp8_wide_kernel<SCALING>), dim3(blocks), dim3(512), 0, st, w);
    else hipLaunchKernelGGL((gemm_fp8_large_kernel<SCALING, TYPE>), dim3(blocks), dim3(512), 0, st, w);
    if (splits > 1) {
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((gemm_fp8_join_kernel<TYPE>), dim3((unsigned)div_up(a.n, 1024), (unsigned)a.m), dim3(256), 0, st, a, splits);
    }
    return hipGetLastError();
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
    return scaling == SCALE_BLOCKS ? launch_kind<SCALE_BLOCKS, TYPE>(a, splits, st) : launch_kind<SCALE_VECTORS, TYPE>(a, splits, st);
}

}  // namespace

int gemm_fp8_splits(int64_t m, int64_t n, int64_t k) { return m > 0 && n > 0 && k > 0 ? shape_of(m, n, k).splits : 1; }

hipError_t launch_gemm_fp8(const GemmFp8Args& a, int scaling, int type_d, int splits, hipStream_t st) {
    if (a.m == 0 || a.n == 0) return hipSuccess;
    return type_d == TYPE_F32 ? launch_typed<TYPE_F32>(a, scaling, splits, st) : type_d == TYPE_BF16 ? launch_typed<TYPE_BF16>(a, scaling, splits, st)
                                                                                                    : launch_typed<TYPE_F16>(a, scaling, splits, st);
}

}  // namespace ozaki
