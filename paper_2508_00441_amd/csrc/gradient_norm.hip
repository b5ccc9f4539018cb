// The norm of many tensors together, and the tensors scaled so that it stays within bounds:
//     norm = |scale| sqrt(sum over all elements of x^2),        out = x * scale * min(1, max_norm / norm).
//
// Bound by memory: every element is read for the norm and once more to be scaled.  Tensors are named in the kernel's arguments, as many to a launch as fit there;
// elements go to workgroups in chunks, whatever the tensors' sizes.  Squares are summed in 64 bits, in an order that depends on the sizes only, so that no
// element's square leaves the range and the norm is the same for every call.
#include "block_operators.hpp"

namespace ozaki {
namespace {

constexpr int64_t CHUNK = 32768;         // elements
constexpr int TABLE = 96;                // tensors in a launch's arguments, which hold 4 KiB
constexpr unsigned MOST_BLOCKS = 2048;   // of a launch, and partial sums that it leaves
constexpr int THREADS = 256;

struct ClipTable {
    const void* x[TABLE];
    void* out[TABLE];
    int64_t size[TABLE];
    uint32_t first[TABLE + 1];           // chunk
    uint8_t type[TABLE];
    int count;
};
static_assert(sizeof(ClipTable) < 3840, "kernel arguments");

// f(x, first element, elements, type's constant) for chunk `at`
template <typename F> __device__ __forceinline__ void with_chunk(const ClipTable& t, uint32_t at, F f) {
    int lo = 0, hi = t.count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= at) lo = mid;
        else hi = mid - 1;
    }
    const int64_t from = (int64_t)(at - t.first[lo]) * CHUNK, left = t.size[lo] - from, n = left < CHUNK ? left : CHUNK;
    switch (t.type[lo]) {
        case TYPE_BF16: f(lo, from, n, std::integral_constant<int, TYPE_BF16>()); break;
        case TYPE_F16: f(lo, from, n, std::integral_constant<int, TYPE_F16>()); break;
        default: f(lo, from, n, std::integral_constant<int, TYPE_F32>()); break;
    }
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double lds[THREADS / 64];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ void __launch_bounds__(THREADS) gradient_squares_kernel(const ClipTable t, double* partial) {
    double sum[2] = {};
    for (uint32_t at = blockIdx.x; at < t.first[t.count]; at += gridDim.x)
        with_chunk(t, at, [&](int i, int64_t from, int64_t n, auto type) {
            typedef typename Element<decltype(type)::value>::type T;
            constexpr int PER = 16 / sizeof(T);
            typedef T piece __attribute__((ext_vector_type(PER)));
            const T* const x = static_cast<const T*>(t.x[i]) + from;
            if (reinterpret_cast<uintptr_t>(x) % 16 == 0) {
                const int64_t pieces = n / PER;
#pragma unroll 4
                for (int64_t p = threadIdx.x; p < pieces; p += THREADS) {
                    const piece v = reinterpret_cast<const piece*>(x)[p];
#pragma unroll
                    for (int q = 0; q < PER; ++q) sum[q & 1] = __builtin_fma((double)(float)v[q], (double)(float)v[q], sum[q & 1]);
                }
                for (int64_t e = pieces * PER + threadIdx.x; e < n; e += THREADS) sum[0] = __builtin_fma((double)(float)x[e], (double)(float)x[e], sum[0]);
            } else {
#pragma unroll 8
                for (int64_t e = threadIdx.x; e < n; e += THREADS) sum[0] = __builtin_fma((double)(float)x[e], (double)(float)x[e], sum[0]);
            }
        });
    const double all = block_sum(sum[0] + sum[1]);
    if (threadIdx.x == 0) partial[blockIdx.x] = all;
}

__global__ void __launch_bounds__(THREADS) gradient_norm_kernel(const double* partial, int64_t count, float scale, float* norm) {
    double sum = 0.0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < count; i += THREADS) sum += partial[i];
    sum = block_sum(sum);
    if (threadIdx.x == 0) *norm = (float)(fabs((double)scale) * sqrt(sum));
}

__global__ void __launch_bounds__(THREADS) gradient_clip_kernel(const ClipTable t, const float* norm_at, float scale, float max_norm) {
    // (a norm that is no number makes the factor none, one that is infinite makes it zero)
    const float norm = *norm_at, factor = norm <= max_norm ? scale : scale * (max_norm / norm);
    for (uint32_t at = blockIdx.x; at < t.first[t.count]; at += gridDim.x)
        with_chunk(t, at, [&](int i, int64_t from, int64_t n, auto type) {
            typedef typename Element<decltype(type)::value>::type T;
            constexpr int PER = 16 / sizeof(T);
            typedef T piece __attribute__((ext_vector_type(PER)));
            const T* const x = static_cast<const T*>(t.x[i]) + from;
            T* const out = static_cast<T*>(t.out[i]) + from;
            if (factor == 1.0f && x == out) return;
            int64_t e = threadIdx.x;
            if (reinterpret_cast<uintptr_t>(x) % 16 == 0 && reinterpret_cast<uintptr_t>(out) % 16 == 0) {
                const int64_t pieces = n / PER;
#pragma unroll 4
                for (int64_t p = threadIdx.x; p < pieces; p += THREADS) {
                    piece v = reinterpret_cast<const piece*>(x)[p];
#pragma unroll
                    for (int q = 0; q < PER; ++q) v[q] = (T)((float)v[q] * factor);
                    reinterpret_cast<piece*>(out)[p] = v;
                }
                e += pieces * PER;
            }
#pragma unroll 8
            for (; e < n; e += THREADS) out[e] = (T)((float)x[e] * factor);
        });
}

// f(table, blocks, index of the launch) for each launch
template <typename F> hipError_t with_tables(const ClipArgs& a, F f) {
    ClipTable t;
    t.count = 0;
    t.first[0] = 0;
    int launch = 0;
    const auto flush = [&]() -> hipError_t {
        if (t.count == 0) return hipSuccess;
        const uint32_t chunks = t.first[t.count];
        f(t, chunks < MOST_BLOCKS ? chunks : MOST_BLOCKS, launch++);
        t.count = 0;
        return hipGetLastError();
    };
    for (int i = 0; i < a.count; ++i) {
        if (a.sizes[i] == 0) continue;
        const int64_t chunks = div_up(a.sizes[i], CHUNK);
        if (t.count == TABLE) {      // (no tensor has more than 2^38 elements: their chunks' numbers stay inside 32 bits)
            const hipError_t e = flush();
            if (e != hipSuccess) return e;
        }
        t.x[t.count] = a.tensors[i];
        t.out[t.count] = a.out != nullptr ? a.out[i] : nullptr;
        t.size[t.count] = a.sizes[i];
        t.type[t.count] = (uint8_t)a.types[i];
        t.first[t.count + 1] = t.first[t.count] + (uint32_t)chunks;
        ++t.count;
    }
    return flush();
}

}  // namespace

size_t gradient_norm_bytes(int64_t count) { return (size_t)div_up(count, TABLE) * MOST_BLOCKS * sizeof(double); }

hipError_t launch_clip(const ClipArgs& a, hipStream_t st) {
    if (!a.given) {
        int64_t partials = 0;
        hipError_t e = with_tables(a, [&](const ClipTable& t, unsigned blocks, int) {
            hipLaunchKernelGGL(gradient_squares_kernel, dim3(blocks), dim3(THREADS), 0, st, t, a.partial + partials);
            partials += blocks;
        });
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(gradient_norm_kernel, dim3(1), dim3(THREADS), 0, st, a.partial, partials, a.scale, a.norm);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.out == nullptr) return hipSuccess;
    return with_tables(a, [&](const ClipTable& t, unsigned blocks, int) {
        hipLaunchKernelGGL(gradient_clip_kernel, dim3(blocks), dim3(THREADS), 0, st, t, a.norm, a.scale, a.max_norm);
    });
}

}  // namespace ozaki
