// The norm of many tensors together, and the tensors scaled so that it stays within bounds:
//     norm = |scale| sqrt(sum over all elements of x^2),        out = x * scale * min(1, max_norm / norm).
//
// Bound by memory: every element is read for the norm and once more to be scaled.  Tensors are named in the kernel's arguments, as many to a launch as fit there;
// elements go to workgroups in chunks, whatever the tensors' sizes.  
// Squares are summed in 32 bits by a thread over its elements of a chunk, and from there on in pairs of 32-bit numbers, a sum and what it lacks, in an order that
// depends on the sizes only.  Where a thread's squares leave the range of 32 bits, it reads its elements again and squares them times 2^-90 or 2^90; such sums are kept apart
// and join at the end.
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

// hi + lo, with lo less than hi's last place
struct Sum { float hi, lo; };
__device__ __forceinline__ Sum operator+(Sum a, Sum b) {
    const float s = a.hi + b.hi, from_b = s - a.hi, lacks = ((a.hi - (s - from_b)) + (b.hi - from_b)) + (a.lo + b.lo), hi = s + lacks;
    return fabsf(s) < __builtin_inff() ? Sum{hi, lacks - (hi - s)} : Sum{s, 0.0f};
}
// Sums of squares: as they are, of elements times 2^-90 and times 2^90.
enum { PLAIN, LARGE, SMALL, LEVELS };
constexpr float LEVEL_FACTOR[LEVELS] = {1.0f, 0x1p-90f, 0x1p90f};
struct Squares { Sum level[LEVELS]; };
__device__ __forceinline__ Squares block_sum(Squares v) {
    __shared__ Squares lds[THREADS / 64];
#pragma unroll
    for (int l = 0; l < LEVELS; ++l)
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) v.level[l] = v.level[l] + Sum{__shfl_xor(v.level[l].hi, d), __shfl_xor(v.level[l].lo, d)};
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    Squares all;
#pragma unroll
    for (int l = 0; l < LEVELS; ++l) all.level[l] = (lds[0].level[l] + lds[1].level[l]) + (lds[2].level[l] + lds[3].level[l]);
    return all;
}

// A thread's squares of the n elements of a chunk, each times `factor` first: eight sums, of CHUNK / THREADS / 8 = 16 elements each at most.
template <typename T> __device__ __forceinline__ float chunk_squares(const T* x, int64_t n, float factor) {
    typedef T eight __attribute__((ext_vector_type(8), aligned(16)));
    float sum[8] = {};
    const auto add = [&](int q, T v) { sum[q] = __builtin_fmaf((float)v * factor, (float)v * factor, sum[q]); };
    int64_t e = 0;
    if (reinterpret_cast<uintptr_t>(x) % 16 == 0) {
        const int64_t pieces = n / 8;
#pragma unroll 4
        for (int64_t p = threadIdx.x; p < pieces; p += THREADS) {
            const eight v = reinterpret_cast<const eight*>(x)[p];
#pragma unroll
            for (int q = 0; q < 8; ++q) add(q, v[q]);
        }
        e = pieces * 8;
    } else {
        for (; e + 8 * THREADS <= n; e += 8 * THREADS)
#pragma unroll
            for (int q = 0; q < 8; ++q) add(q, x[e + q * THREADS + threadIdx.x]);
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        const int64_t at = e + q * THREADS + threadIdx.x;
        if (at < n) add(q, x[at]);
    }
    return ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
}

__global__ void __launch_bounds__(THREADS) gradient_squares_kernel(const ClipTable t, Squares* partial) {
    Squares all = {};
    for (uint32_t at = blockIdx.x; at < t.first[t.count]; at += gridDim.x)
        with_chunk(t, at, [&](int i, int64_t from, int64_t n, auto type) {
            typedef typename Element<decltype(type)::value>::type T;
            const T* const x = static_cast<const T*>(t.x[i]) + from;
            const float sum = chunk_squares(x, n, 1.0f);
            if (sum >= 0x1p-80f && sum < 0x1p90f) {
                all.level[PLAIN] = all.level[PLAIN] + Sum{sum, 0.0f};
            } else if (sum < 1.0f) {
                all.level[SMALL] = all.level[SMALL] + Sum{chunk_squares(x, n, LEVEL_FACTOR[SMALL]), 0.0f};
            } else {                                 // (also what is no number)
                all.level[LARGE] = all.level[LARGE] + Sum{chunk_squares(x, n, LEVEL_FACTOR[LARGE]), 0.0f};
            }
        });
    all = block_sum(all);
    if (threadIdx.x == 0) partial[blockIdx.x] = all;
}

__global__ void __launch_bounds__(THREADS) gradient_norm_kernel(const Squares* partial, int64_t count, float scale, float* norm) {
    Squares all = {};
    for (int64_t i = threadIdx.x; i < count; i += THREADS) {
        const Squares p = partial[i];
#pragma unroll
        for (int l = 0; l < LEVELS; ++l) all.level[l] = all.level[l] + p.level[l];
    }
    all = block_sum(all);
    if (threadIdx.x != 0) return;
    // the highest level that is there, with the next one's share of it (the one below that is less than its last place)
    const auto scaled = [](Sum s, float f) { return Sum{s.hi * f, s.lo * f}; };
    const bool large = all.level[LARGE].hi != 0.0f, plain = all.level[PLAIN].hi != 0.0f;
    const Sum sum = large ? all.level[LARGE] + scaled(scaled(all.level[PLAIN], LEVEL_FACTOR[LARGE]), LEVEL_FACTOR[LARGE])
                  : plain ? all.level[PLAIN] + scaled(scaled(all.level[SMALL], LEVEL_FACTOR[LARGE]), LEVEL_FACTOR[LARGE])
                          : all.level[SMALL];
    const float by = fabsf(scale), back = large ? LEVEL_FACTOR[SMALL] : plain ? 1.0f : LEVEL_FACTOR[LARGE];
    // the root with what it lacks, times the scale: one rounding
    const float root = sqrtf(sum.hi), lacks = root > 0.0f && root < __builtin_inff() ? (__builtin_fmaf(-root, root, sum.hi) + sum.lo) / (2.0f * root) : 0.0f;
    const float n = root * by, rest = root < __builtin_inff() ? __builtin_fmaf(root, by, -n) + lacks * by : 0.0f;
    *norm = (n + rest) * back;
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

size_t gradient_norm_bytes(int64_t count) { return (size_t)div_up(count, TABLE) * MOST_BLOCKS * sizeof(Squares); }

hipError_t launch_clip(const ClipArgs& a, hipStream_t st) {
    if (!a.given) {
        int64_t partials = 0;
        Squares* const partial = reinterpret_cast<Squares*>(a.ws);
        hipError_t e = with_tables(a, [&](const ClipTable& t, unsigned blocks, int) {
            hipLaunchKernelGGL(gradient_squares_kernel, dim3(blocks), dim3(THREADS), 0, st, t, partial + partials);
            partials += blocks;
        });
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(gradient_norm_kernel, dim3(1), dim3(THREADS), 0, st, partial, partials, a.scale, a.norm);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.out == nullptr) return hipSuccess;
    return with_tables(a, [&](const ClipTable& t, unsigned blocks, int) {
        hipLaunchKernelGGL(gradient_clip_kernel, dim3(blocks), dim3(THREADS), 0, st, t, a.norm, a.scale, a.max_norm);
    });
}

}  // namespace ozaki
