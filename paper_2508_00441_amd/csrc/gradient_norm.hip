// The norm of many tensors together, and the tensors scaled so that it stays within bounds:
//     norm = |scale| sqrt(sum over all elements of x^2),        out = x * scale * min(1, max_norm / norm).
//
// Bound by memory: every element is read for the norm and once more to be scaled, from the end, which the last-level cache still has (268 million BF16 elements: 121 us
// for the squares, 4.4 TB/s, 175 - 181 for the second reading, 5.9 - 6.1 TB/s read and written).  Tensors are named in the kernel's arguments, as many to a launch as fit there;
// elements go to workgroups in chunks, whatever the tensors' sizes.
// Squares are summed in 32 bits by a thread over its elements of a chunk, and from there on in pairs of 32-bit numbers, a sum and what it lacks, in an order that
// depends on the sizes only.  Where a thread's squares leave the range of 32 bits, it reads its elements again and squares them times 2^-90 or 2^90; such sums are kept apart
// and join at the end.
#include "block_operators.hpp"

namespace ozaki {
namespace {

// Elements of a chunk, and workgroups of a launch, each of which leaves a partial sum.  268 million BF16 elements: 126 us for the squares, 174 for the second reading; chunks of
// 32768 129 and 183, of 4096 148 and 184; 2048 workgroups add 2 us to the join.
constexpr uint32_t MOST_CHUNK = 8192, LEAST_CHUNK = 2048;
constexpr unsigned MOST_BLOCKS = 1024;
// Tensors in a launch's arguments: what 4 KiB hold, but for one.  One more is two more launches: 144 tensors of 2.6 million BF16 elements 13 us, 153 of 2.8 million 24; 144 of 42 million 55, 153 of 45
// million 67.
constexpr int TABLE = 144;
constexpr int MOST_REVERSED = 64;        // launches that the second reading takes from the last one on
constexpr int THREADS = 256, MOST_JOINED = 1024;     // partial sums that every workgroup of the second reading adds up itself: 3 us, a launch of its own 5

struct ClipTable {
    const void* x[TABLE];
    void* out[TABLE];
    uint64_t size[TABLE];                // and the type, in the two highest bits
    uint32_t first[TABLE];               // chunk; behind the last tensor the number of all chunks
    uint32_t chunks, chunk;              // elements of a chunk
};
static_assert(sizeof(ClipTable) + 2 * sizeof(void*) + sizeof(int) + 2 * sizeof(float) <= 4096, "kernel arguments");
static_assert(MAX_CLIPPED / MOST_CHUNK + TABLE + MOST_BLOCKS <= 0x7FFFFFFF, "chunks of a launch, counted in 32 bits");
static_assert((MAX_TENSORS / TABLE + 1) * MOST_BLOCKS <= 0x7FFFFFFF, "partial sums, counted in 32 bits");

// The table in a wave's registers, a tensor a lane, read in one go: a search in memory would wait for each of its steps, since arguments come from far away.
struct ClipLanes {
    static constexpr int ROUNDS = (TABLE + 63) / 64;
    const void* x[ROUNDS];
    void* out[ROUNDS];
    uint64_t size[ROUNDS];
    uint32_t first[ROUNDS];
    __device__ __forceinline__ explicit ClipLanes(const ClipTable& t, bool results) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int i = r * 64 + lane < TABLE ? r * 64 + lane : TABLE - 1;
            x[r] = t.x[i];
            out[r] = results ? t.out[i] : nullptr;
            size[r] = t.size[i];
            first[r] = t.first[i];
        }
    }
    // f(x, out, elements, type's constant) for chunk `at`
    template <typename F> __device__ __forceinline__ void with_chunk(uint32_t at, uint32_t chunk, F f) const {
        int i = -1;                      // tensors that begin there or before it (the places behind the last hold the number of all chunks)
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) i += __popcll(__ballot(first[r] <= at && r * 64 + (threadIdx.x & 63) < TABLE));
        const int lane = i & 63, round = i >> 6;
        const auto lanes = [&](uint64_t v) {
            return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32;
        };
        uint64_t p = 0, q = 0, n = 0;
        uint32_t begin = 0;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            if (r == round) {
                p = lanes(reinterpret_cast<uint64_t>(x[r]));
                q = lanes(reinterpret_cast<uint64_t>(out[r]));
                n = lanes(size[r]);
                begin = (uint32_t)__builtin_amdgcn_readlane((int)first[r], lane);
            }
        const int type = (int)(n >> 62);
        n &= ((uint64_t)1 << 62) - 1;
        const uint64_t from = (uint64_t)(at - begin) * chunk, left = n - from;
        const int elements = (int)(left < chunk ? left : chunk);
        const auto of = [&](auto c) {
            typedef typename Element<decltype(c)::value>::type T;
            f(reinterpret_cast<const T*>(p) + from, reinterpret_cast<T*>(q) + from, elements);
        };
        if (type == TYPE_BF16) of(std::integral_constant<int, TYPE_BF16>());
        else if (type == TYPE_F16) of(std::integral_constant<int, TYPE_F16>());
        else of(std::integral_constant<int, TYPE_F32>());
    }
};

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
    for (int l = 0; l < LEVELS; ++l) {
        if (__ballot(v.level[l].hi != 0.0f) == 0) continue;            // (most levels, as a rule: 12 exchanges instead of 36)
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) v.level[l] = v.level[l] + Sum{__shfl_xor(v.level[l].hi, d), __shfl_xor(v.level[l].lo, d)};
    }
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    Squares all;
#pragma unroll
    for (int l = 0; l < LEVELS; ++l) all.level[l] = (lds[0].level[l] + lds[1].level[l]) + (lds[2].level[l] + lds[3].level[l]);
    return all;
}

// A thread's squares of the n elements of a chunk, each times `factor` first: eight sums, of MOST_CHUNK / THREADS / 8 = 4 elements each at most; a chunk that
// ends inside a piece has up to seven more, one for each of the first threads.
template <typename T> __device__ __forceinline__ float chunk_squares(const T* x, int n, float factor) {
    float sum[8] = {};
    const auto add = [&](int q, T v) { sum[q] = __builtin_fmaf((float)v * factor, (float)v * factor, sum[q]); };
    const int pieces = n / 8, e = pieces * 8;
#pragma unroll 4
    for (int p = threadIdx.x; p < pieces; p += THREADS) {
        const Eight<T> v = *reinterpret_cast<const Eight<T>*>(x + 8 * p);
#pragma unroll
        for (int q = 0; q < 8; ++q) add(q, v[q]);
    }
    if (e + (int)threadIdx.x < n) add(0, x[e + threadIdx.x]);
    return ((sum[0] + sum[1]) + (sum[2] + sum[3])) + ((sum[4] + sum[5]) + (sum[6] + sum[7]));
}

__global__ void __launch_bounds__(THREADS) gradient_squares_kernel(const ClipTable t, Squares* partial) {
    const ClipLanes lanes(t, false);
    Squares all = {};
    for (uint32_t at = blockIdx.x; at < t.chunks; at += gridDim.x)
        lanes.with_chunk(at, t.chunk, [&](auto x, auto, int n) {
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

// the norm from `count` partial sums, for all threads of a workgroup
__device__ __forceinline__ float norm_of(const Squares* partial, int count, float scale) {
    Squares all = {};
#pragma unroll 4
    for (int i = threadIdx.x; i < count; i += THREADS) {
        const Squares p = partial[i];
#pragma unroll
        for (int l = 0; l < LEVELS; ++l) all.level[l] = all.level[l] + p.level[l];
    }
    all = block_sum(all);
    // the highest level that is there, with the next one's share of it (the one below that is less than its last place)
    const auto scaled = [](Sum s, float f) { return Sum{s.hi * f, s.lo * f}; };
    const bool large = all.level[LARGE].hi != 0.0f, plain = all.level[PLAIN].hi != 0.0f;
    const Sum sum = large ? all.level[LARGE] + scaled(scaled(all.level[PLAIN], LEVEL_FACTOR[LARGE]), LEVEL_FACTOR[LARGE])
                  : plain ? all.level[PLAIN] + scaled(scaled(all.level[SMALL], LEVEL_FACTOR[LARGE]), LEVEL_FACTOR[LARGE])
                          : all.level[SMALL];
    float by = fabsf(scale), back = large ? LEVEL_FACTOR[SMALL] : plain ? 1.0f : LEVEL_FACTOR[LARGE];
    // a scale on the other side of one takes the level's power of two with it: no product on the way leaves the range unless the norm does
    if (large ? by < 1.0f : by > 1.0f) {
        by *= back;
        back = 1.0f;
    }
    // the root with what it lacks, times the scale: one rounding
    const float root = sqrtf(sum.hi), lacks = root > 0.0f && root < __builtin_inff() ? (__builtin_fmaf(-root, root, sum.hi) + sum.lo) / (2.0f * root) : 0.0f;
    const float n = root * by, rest = n < __builtin_inff() ? __builtin_fmaf(root, by, -n) + lacks * by : 0.0f;
    return (n + rest) * back;
}

__global__ void __launch_bounds__(THREADS) gradient_norm_kernel(const Squares* partial, int count, float scale, float* norm) {
    const float n = norm_of(partial, count, scale);
    if (threadIdx.x == 0) *norm = n;
}

// `count` partial sums, each workgroup adding them up itself; 0: the norm is there.
__global__ void __launch_bounds__(THREADS) gradient_clip_kernel(const ClipTable t, float* norm_at, const Squares* partial, int count, float scale, float max_norm) {
    const ClipLanes lanes(t, true);
    float norm;
    if (count > 0) {
        norm = norm_of(partial, count, scale);
        if (blockIdx.x == 0 && threadIdx.x == 0) *norm_at = norm;
    } else {
        norm = *norm_at;
    }
    // (a norm that is no number makes the factor none, one that is infinite makes it zero)
    const float ratio = max_norm / norm, factor = norm <= max_norm ? scale : scale * ratio;
    // A factor below the normal numbers would lose its bits: then elements meet the scale first, which keeps them within the norm, and the ratio after that; a ratio
    // as small is formed times 2^100, which the elements give back in between.
    const bool far = norm > max_norm && norm < __builtin_inff() && (ratio < 0x1p-126f || fabsf(factor) < 0x1p-126f);
    const float back = ratio < 0x1p-126f ? 0x1p-100f : 1.0f, rest = ratio < 0x1p-126f ? 0x1p100f * max_norm / norm : ratio;
    for (uint32_t i = blockIdx.x; i < t.chunks; i += gridDim.x)
        lanes.with_chunk(t.chunks - 1 - i, t.chunk, [&](auto x, auto out, int n) {
            typedef std::remove_pointer_t<decltype(out)> T;
            constexpr int PER = 16 / sizeof(T);
            typedef T piece __attribute__((ext_vector_type(PER), aligned(sizeof(T))));
            if (factor == 1.0f && x == out) return;
            const auto write = [&](auto times) {
                const int pieces = n / PER, e = pieces * PER + threadIdx.x;
#pragma unroll 4
                for (int p = threadIdx.x; p < pieces; p += THREADS) {
                    piece v = *reinterpret_cast<const piece*>(x + PER * p);
#pragma unroll
                    for (int q = 0; q < PER; ++q) v[q] = (T)times((float)v[q]);
                    *reinterpret_cast<piece*>(out + PER * p) = v;
                }
                if (e < n) out[e] = (T)times((float)x[e]);
            };
            if (far) write([&](float v) { return v * scale * back * rest; });
            else write([&](float v) { return v * factor; });
        });
}

// A launch's tensors: from `begin` on, as many as fit; returns where the next one begins.
int fill_table(const ClipArgs& a, int begin, ClipTable& t) {
    int at[TABLE], count = 0, i = begin;
    uint64_t total = 0;
    for (; i < a.count && count < TABLE; ++i)
        if (a.sizes[i] > 0) {
            at[count++] = i;
            total += a.sizes[i];
        }
    // as short as makes 512 of them, within the bounds
    t.chunk = LEAST_CHUNK;
    while (t.chunk < MOST_CHUNK && total / t.chunk > MOST_JOINED / 2) t.chunk *= 2;
    t.chunks = 0;
    for (int j = 0; j < TABLE; ++j) {
        t.first[j] = t.chunks;
        t.x[j] = j < count ? a.tensors[at[j]] : nullptr;
        t.out[j] = j < count && a.out != nullptr ? a.out[at[j]] : nullptr;
        t.size[j] = j < count ? (uint64_t)a.sizes[at[j]] | (uint64_t)a.types[at[j]] << 62 : 0;
        if (j < count) t.chunks += (uint32_t)div_up(a.sizes[at[j]], t.chunk);
    }
    return i;
}
unsigned blocks_of(const ClipTable& t) { return t.chunks < MOST_BLOCKS ? t.chunks : MOST_BLOCKS; }

}  // namespace

size_t gradient_norm_bytes(int64_t count) { return (size_t)div_up(count, TABLE) * MOST_BLOCKS * sizeof(Squares); }

hipError_t launch_clip(const ClipArgs& a, hipStream_t st) {
    Squares* const partial = reinterpret_cast<Squares*>(a.ws);
    int partials = 0, launches = 0;
    int begins[MOST_REVERSED];           // of the launches' tensors
    ClipTable t;
    for (int i = 0; i < a.count && !a.given;) {
        if (launches < MOST_REVERSED) begins[launches] = i;
        i = fill_table(a, i, t);
        if (t.chunks == 0) break;
        hipLaunchKernelGGL(gradient_squares_kernel, dim3(blocks_of(t)), dim3(THREADS), 0, st, t, partial + partials);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        partials += blocks_of(t);
        ++launches;
    }
    // Few partial sums are added up by every workgroup of the second reading, without a launch in between.
    const bool apart = !a.given && (a.out == nullptr || launches == 0 || partials > MOST_JOINED);
    if (apart) {
        hipLaunchKernelGGL(gradient_norm_kernel, dim3(1), dim3(THREADS), 0, st, partial, partials, a.scale, a.norm);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const auto clip = [&](int begin, int& next) {
        next = fill_table(a, begin, t);
        if (t.chunks == 0) return hipSuccess;
        hipLaunchKernelGGL(gradient_clip_kernel, dim3(blocks_of(t)), dim3(THREADS), 0, st, t, a.norm, partial, a.given || apart ? 0 : partials, a.scale, a.max_norm);
        return hipGetLastError();
    };
    if (a.out == nullptr) return hipSuccess;
    int next = 0;
    if (launches > 0 && launches <= MOST_REVERSED) {                   // what was read last comes first
        for (int l = launches - 1; l >= 0; --l) {
            const hipError_t e = clip(begins[l], next);
            if (e != hipSuccess) return e;
        }
    } else {
        while (next < a.count) {
            const hipError_t e = clip(next, next);
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace ozaki
