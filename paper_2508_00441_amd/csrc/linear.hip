// A linear layer with what follows it, and a pair of linear layers whose results are multiplied:
//     z = x W^T + bias,  y = act(z) + r            and            g = x Wg^T,  u = x Wu^T,  y = act(g) * u.
//
// One product of 16-bit elements in FP32 on the matrix unit (tile_product.hpp); everything behind it happens on a tile in LDS on its way to memory, in
// FP32, with one rounding of each result.  Of a pair, half of a tile's vectors of weights are Wg's and half are Wu's, so that a lane holds both
// factors of its elements and neither reaches memory unless it is asked for.
// Few vectors of X are bound by the read of the weights (below), many by the matrix unit and power (pair of 4096 x 8192 x 4096, both factors kept: 394 - 416 us, 1.32 - 1.40 PFLOP/s;
// 8192 x 16384 x 2048 426 - 440 us, with bias and GELU, which no product covers, 483), in between by a step's latency.
#include "block_operators.hpp"
#include "layout.hpp"
#include "tile_epilogue.hpp"

namespace ozaki {
namespace {

constexpr int kind_of(int type) { return type == TYPE_F16 ? KIND_F16 : KIND_BF16; }

// What becomes of the sums of row m, column c (both of the whole matrices) and its seven neighbours, or of one alone.
template <int TYPE, bool PAIR, bool STREAMED>
struct Epilogue {
    typedef typename Element<TYPE>::type T;
    typedef Eight<T> eight;
    const LinearArgs& a;
    bool wide;                       // every matrix has rows that start at multiples of 16 bytes

    __device__ __forceinline__ explicit Epilogue(const LinearArgs& args) : a(args) {
        wide = rows_aligned(static_cast<T*>(a.Y), a.ldy) && rows_aligned(static_cast<T*>(a.Z), a.ldz) &&
               (PAIR ? rows_aligned(static_cast<T*>(a.U), a.ldu) : rows_aligned(static_cast<const T*>(a.R), a.ldr));
    }
    __device__ __forceinline__ void put(void* to, int64_t at, v8f32 v) const { put_eight<STREAMED>(static_cast<T*>(to) + at, v); }
    __device__ __forceinline__ v8f32 activate(v8f32 v) const {
        with_activation(a.activation, [&](auto act) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = activated<decltype(act)::value>(v[q]);
        });
        return v;
    }
    // What eight columns, or one, need beside their sums, for every row: the bias.
    __device__ __forceinline__ v8f32 columns(int64_t c) const { return !PAIR && a.bias != nullptr ? get_eight(static_cast<const T*>(a.bias) + c) : v8f32{}; }
    __device__ __forceinline__ float column(int64_t c) const { return !PAIR && a.bias != nullptr ? (float)static_cast<const T*>(a.bias)[c] : 0.0f; }
    // ... and for one row: the residual, asked for in front of the others' arithmetic
    __device__ __forceinline__ eight ahead(int64_t m, int64_t c) const {
        return !PAIR && a.R != nullptr ? *reinterpret_cast<const Eight<T>*>(static_cast<const T*>(a.R) + m * a.ldr + c) : eight{};
    }
    __device__ __forceinline__ void piece(int64_t m, int64_t c, v8f32 v, v8f32 u, v8f32 bias, eight r) const {
        v += bias;
        if (a.Z != nullptr) {
            put(a.Z, m * a.ldz + c, v);
            if constexpr (PAIR) put(a.U, m * a.ldu + c, u);
        }
        v = activate(v);
        if constexpr (PAIR) v *= u;
        else v += __builtin_convertvector(r, v8f32);
        put(a.Y, m * a.ldy + c, v);
    }
    // the sums of one column of rows m0 + m[q]; `there`: bit q, that row exists
    template <int N> __device__ __forceinline__ void rows(int64_t m0, const int (&m)[N], unsigned there, int64_t c, float (&v)[N], const float (&u)[N], float bias) const {
        T r[N];
        if constexpr (!PAIR) {
#pragma unroll
            for (int q = 0; q < N; ++q) r[q] = a.R != nullptr && (there >> q & 1) ? static_cast<const T*>(a.R)[(m0 + m[q]) * a.ldr + c] : (T)0.0f;
        }
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] += bias;
        if (a.Z != nullptr) {
#pragma unroll
            for (int q = 0; q < N; ++q)
                if (there >> q & 1) {
                    static_cast<T*>(a.Z)[(m0 + m[q]) * a.ldz + c] = (T)v[q];
                    if constexpr (PAIR) static_cast<T*>(a.U)[(m0 + m[q]) * a.ldu + c] = (T)u[q];
                }
        }
        with_activation(a.activation, [&](auto act) {
#pragma unroll
            for (int q = 0; q < N; ++q) v[q] = activated<decltype(act)::value>(v[q]);
        });
#pragma unroll
        for (int q = 0; q < N; ++q) {
            if constexpr (PAIR) v[q] *= u[q];
            else v[q] += (float)r[q];
            if (there >> q & 1) static_cast<T*>(a.Y)[(m0 + m[q]) * a.ldy + c] = (T)v[q];
        }
    }
    __device__ __forceinline__ void one(int64_t m, int64_t c, float v, float u) const {
        v += column(c);
        if (a.Z != nullptr) {
            static_cast<T*>(a.Z)[m * a.ldz + c] = (T)v;
            if constexpr (PAIR) static_cast<T*>(a.U)[m * a.ldu + c] = (T)u;
        }
        with_activation(a.activation, [&](auto act) { v = activated<decltype(act)::value>(v); });
        if constexpr (PAIR) v *= u;
        else if (a.R != nullptr) v += (float)static_cast<const T*>(a.R)[m * a.ldr + c];
        static_cast<T*>(a.Y)[m * a.ldy + c] = (T)v;
    }
};

struct LinearWork {
    LinearArgs a;
    int steps, splits;
    int tiles_m, tiles_n;
    WorkOrder order;
};

template <typename P, int TYPE>
__device__ __forceinline__ void linear_body(const LinearWork& w) {
    constexpr bool PAIR = P::PAIR;
    constexpr int COLUMNS = PAIR ? P::TN / 2 : P::TN;
    __shared__ __attribute__((aligned(16))) uint8_t lds[P::LDS_BYTES];
    const LinearArgs& a = w.a;
    const WorkItem item = work_item(blockIdx.x, gridDim.x, w.order, w.tiles_m, w.tiles_n);
    const int64_t m0 = (int64_t)item.bm * P::TM, n0 = (int64_t)item.bn * COLUMNS, left_m = a.m - m0, left_n = a.n - n0;
    TileOperand X{static_cast<const uint8_t*>(a.W) + n0 * a.ldw * 2, a.ldw * 2, (int)(left_n < COLUMNS ? left_n : COLUMNS), nullptr, 0};
    if constexpr (PAIR) X.second = static_cast<const uint8_t*>(a.W2) + n0 * a.ldw * 2;
    const TileOperand Y{static_cast<const uint8_t*>(a.X) + m0 * a.ldx * 2, a.ldx * 2, (int)(left_m < P::TM ? left_m : P::TM), nullptr, 0};
    const int split = item.gi;
    v4f32 acc[P::FN][P::FM] = {};
    P::multiply(lds, X, Y, a.k * 2, split_begin(w.steps, w.splits, split), split_begin(w.steps, w.splits, split + 1), acc);
    if (w.splits > 1) {
        const int64_t ld = in_fours(a.n);
        put_tile<P>(lds, acc, m0, n0, left_m, in_fours(left_n), Partial{a.partial + split * a.m * ld, ld, PAIR ? w.splits * a.m * ld : 0});
    } else {
        put_tile<P>(lds, acc, m0, n0, left_m, left_n, Epilogue<TYPE, PAIR, (P::TM == 256)>(a));
    }
}

template <int TYPE, bool PAIR>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) linear_large_kernel(const LinearWork w) {
    linear_body<PairedTile<kind_of(TYPE), false, false, PAIR>, TYPE>(w);
}
template <int TYPE, bool PAIR>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) linear_middle_kernel(const LinearWork w) {
    linear_body<Tile<kind_of(TYPE), 2, 2, 4, 4, 2, false, false, PAIR>, TYPE>(w);
}
// Smaller tiles in eight waves, two to a SIMD: with one, a step's wait, LDS reads and products follow each other (100 x 5001 x 2048: 13.1 us against 14.2 in four waves)
template <int TYPE, bool PAIR>
__global__ void __launch_bounds__(512) linear_half_kernel(const LinearWork w) {
    linear_body<Tile<kind_of(TYPE), 2, 4, 4, 1, 3, false, false, PAIR>, TYPE>(w);
}
template <int TYPE, bool PAIR>
__global__ void __launch_bounds__(512) linear_small_kernel(const LinearWork w) {
    linear_body<Tile<kind_of(TYPE), 2, 4, 2, 1, 4, false, false, PAIR>, TYPE>(w);
}
// (of a pair a wave has both factors' vectors: half as many waves)
template <int TYPE, bool PAIR>
__global__ void __launch_bounds__(PAIR ? 256 : 512) linear_narrow_kernel(const LinearWork w) {
    linear_body<Tile<kind_of(TYPE), PAIR ? 1 : 2, 4, PAIR ? 2 : 1, 1, 4, false, false, PAIR>, TYPE>(w);
}

// Up to sixteen vectors of X: no tile in LDS.  A workgroup takes sixteen vectors of W (of each, of a pair), its waves take steps of 64 elements in turn, straight
// from memory into registers; the waves' sums are added in LDS, in their order.  W is read once, past the caches, and bounds it.  A wave has AHEAD steps under way.
// 1 x 4096 x 8192: 15.5 us, 4.3 TB/s.  Eight waves without a pair: 1 x 16384 x 2048 13.7, in sixteen 23.7;  4 x 4096 x 1024 6.3, 8.1;  16 x 11001 x 4096 26.6, 29.1;  longer vectors are
// about even, 16 x 16384 x 16384 144, 152, but 1 x 4096 x 8192 13.5 in sixteen, 1 x 16384 x 16384 106, 100.  A pair of 8192 x 4096: 25.3, 5.3 TB/s, in eight waves with four steps under way 29.1.
constexpr int FEW = 16;
constexpr int few_waves(bool pair) { return pair ? 16 : 8; }

template <int TYPE, bool PAIR>
__global__ void __launch_bounds__(few_waves(PAIR) * 64) linear_few_kernel(const LinearArgs a, const int splits) {
    constexpr int FACTORS = PAIR ? 2 : 1, FEW_WAVES = few_waves(PAIR), AHEAD = PAIR ? 2 : 4;
    __shared__ __attribute__((aligned(16))) v4f32 sums[FACTORS][FEW_WAVES][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, row = lane & 15;
    const int split = blockIdx.x % splits;
    const int64_t n0 = (int64_t)(blockIdx.x / splits) * 16, bytes = a.k * 2;
    const int left_n = a.n - n0 < 16 ? (int)(a.n - n0) : 16, steps = (int)div_up(bytes, STEP_BYTES);
    const int begin = split_begin(steps, splits, split), end = split_begin(steps, splits, split + 1);
    const uint8_t* at[FACTORS + 1];                  // this lane's vectors, from piece lane / 16 on: of W, of W2, of X
    const int64_t w_row = (n0 + (row < left_n ? row : left_n - 1)) * a.ldw * 2 + g * 16;
    at[0] = static_cast<const uint8_t*>(a.W) + w_row;
    if constexpr (PAIR) at[1] = static_cast<const uint8_t*>(a.W2) + w_row;
    at[FACTORS] = static_cast<const uint8_t*>(a.X) + (row < a.m ? row : a.m - 1) * a.ldx * 2 + g * 16;
    v4i32 pieces[AHEAD][FACTORS + 1][2];
    // (behind the end of the vectors something that is there is read and not used)
    const auto load = [&](int u, int s) {
        const int64_t from = (int64_t)(s < end ? s : end - 1) * STEP_BYTES;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t off = from + g * 16 + h * 64 < bytes ? from + h * 64 : -(int64_t)g * 16;
#pragma unroll
            for (int o = 0; o <= FACTORS; ++o) {
                const v4i32* const p = reinterpret_cast<const v4i32*>(at[o] + off);
                pieces[u][o][h] = o < FACTORS ? __builtin_nontemporal_load(p) : *p;
            }
        }
    };
    v4f32 acc[FACTORS] = {};
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(u, begin + wave + u * FEW_WAVES);
    for (int first = begin + wave; first < end; first += FEW_WAVES * AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int s = first + u * FEW_WAVES;
            if (s >= end) break;
            const int64_t left = bytes - (int64_t)s * STEP_BYTES;
            if (left < STEP_BYTES) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int o = 0; o <= FACTORS; ++o) {
                        const int keep = (int)left - g * 16 - h * 64;
                        pieces[u][o][h] = first_bytes(pieces[u][o][h], keep < 0 ? 0 : keep);
                    }
            }
#pragma unroll
            for (int o = 0; o < FACTORS; ++o)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if constexpr (TYPE == TYPE_BF16)
                        acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf16, pieces[u][o][h]), __builtin_bit_cast(v8bf16, pieces[u][FACTORS][h]), acc[o], 0, 0, 0);
                    else
                        acc[o] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8f16, pieces[u][o][h]), __builtin_bit_cast(v8f16, pieces[u][FACTORS][h]), acc[o], 0, 0, 0);
                }
            if (first + FEW_WAVES * AHEAD < end) load(u, s + FEW_WAVES * AHEAD);
        }
    }
#pragma unroll
    for (int o = 0; o < FACTORS; ++o) sums[o][wave][lane] = acc[o];
    __syncthreads();
    const int n = threadIdx.x & 15, m = threadIdx.x >> 4;
    if (threadIdx.x >= 256 || m >= a.m || n >= left_n) return;
    float total[2] = {};
#pragma unroll
    for (int w = 0; w < FEW_WAVES; ++w)
#pragma unroll
        for (int o = 0; o < FACTORS; ++o) total[o] += reinterpret_cast<const float*>(&sums[o][w][(n >> 2) * 16 + m])[n & 3];
    if (splits > 1) {
        const int64_t ld = in_fours(a.n);
        Partial{a.partial + split * a.m * ld, ld, PAIR ? splits * a.m * ld : 0}.one(m, n0 + n, total[0], total[1]);
    } else {
        Epilogue<TYPE, PAIR, false>(a).one(m, n0 + n, total[0], total[1]);
    }
}

// sums the shares of the inner dimension in their order, eight columns a thread
template <int TYPE, bool PAIR>
__global__ void __launch_bounds__(256) linear_join_kernel(const LinearArgs a, const int splits) {
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8, ld = in_fours(a.n);
    if (c >= a.n) return;
    const Epilogue<TYPE, PAIR, false> e(a);
    const bool more = c + 4 < ld;
    for (int64_t m = blockIdx.y; m < a.m; m += gridDim.y) {
        v8f32 v[2] = {};
#pragma unroll
        for (int o = 0; o < (PAIR ? 2 : 1); ++o) {
            const float* from = a.partial + (o * splits * a.m + m) * ld + c;
            v4f32 lo = {}, hi = {};
#pragma unroll 4
            for (int s = 0; s < splits; ++s, from += a.m * ld) {
                lo += *reinterpret_cast<const v4f32*>(from);
                if (more) hi += *reinterpret_cast<const v4f32*>(from + 4);
            }
            v[o] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        if (e.wide && c + 8 <= a.n) {
            e.piece(m, c, v[0], v[1], e.columns(c), e.ahead(m, c));
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (c + q < a.n) e.one(m, c + q, v[0][q], v[1][q]);
        }
    }
}

enum { VECTORS, NARROW, SMALL, HALF, MIDDLE, LARGE };
struct Shape { int kind, tm, tn, splits; };
// By how many tiles there are for 256 compute units; `columns` counts both factors of a pair.  Times in us, with bias and GELU in BF16, W in the last-level cache (from memory the
// order is the same: 300 x 11000 x 4096 56, 67, 65;  1024 x 4096 x 4096 54, 68, 64):
//     tiles of 64 tokens and 64 columns, up to 128 of them: 32 columns     200 x 2048 x 2048: 11.2, by 64 x 64 12.9;  128 x 4096 x 4096: 17.2, 19.6
//     fewer than 256 of 64 x 128: 64 x 64                                  1000 x 1000 x 1000: 9.7, by 32 columns 12.0, by 64 x 128 11.8
//     up to 768 of 64 x 128                                                1024 x 4096 x 4096: 49, by 64 x 64 62, by 128 x 128 51;  300 x 11000 x 4096: 42, 53, 54
//     up to 512 of 128 x 128                                               2048 x 4096 x 2048: 42.4, by 64 x 128 52.5, by 256 x 256 57
//     more: 256 x 256                                                      2048 x 8192 x 512: 31, by 128 x 128 36
// The narrowest tiles where they are fewer than compute units: in shares of the inner dimension of sixteen steps at least (20 x 1000 x 8192: 13.1 in eight, 26.8 uncut;
// but 48 x 1000 x 500, eight steps: 7.0, in two shares 8.6).  64 x 64 tiles are not cut, however long the inner dimension is (128 x 4160 x 16384, 130 of them: 75, where W's read is 30).  Few
// vectors: from 96 steps on, in shares of at least 32 (1 x 1000 x 16384: 12.5, uncut 20.4); from 256 steps on in two also where there are enough workgroups (1 x 5000 x 16384: 37.5, uncut 45; a pair
// of 16384 x 16384: 192, 204; not so without a pair, 1 x 16384 x 16384: 106, uncut 100).
Shape shape_of(int64_t m, int64_t n, int64_t k, bool pair) {
    const int64_t steps = div_up(k * 2, STEP_BYTES), columns = pair ? 2 * n : n;
    const auto shares = [](int64_t want, int64_t most) {
        const int64_t s = want < most ? want : most;
        return (int)(s < 1 ? 1 : s > 16 ? 16 : s);
    };
    if (m <= FEW) return Shape{VECTORS, FEW, 16, steps < 96 ? 1 : shares(256 / div_up(n, 16) > 1 || steps < 256 ? 256 / div_up(n, 16) : 2, steps / 32)};
    const auto tiles = [&](int64_t tm, int64_t tn) { return div_up(m, tm) * div_up(columns, tn); };
    const auto shape = [&](int kind, int tm, int tn, int splits) { return Shape{kind, tm, pair ? tn / 2 : tn, splits}; };
    if (tiles(64, 64) <= 128) return shape(NARROW, 64, 32, shares(256 / tiles(64, 32), steps / 16));
    if (tiles(64, 128) < 256) return shape(SMALL, 64, 64, 1);
    if (tiles(64, 128) <= 768) return shape(HALF, 64, 128, 1);
    return tiles(128, 128) <= 512 || m <= 128 || columns <= 128 ? shape(MIDDLE, 128, 128, 1) : shape(LARGE, 256, 256, 1);
}

template <int TYPE, bool PAIR>
hipError_t launch_kind(const LinearArgs& a, Shape s, hipStream_t st) {
    LinearWork w;
    w.a = a;
    w.steps = (int)div_up(a.k * 2, STEP_BYTES);
    w.splits = s.splits;
    w.tiles_m = (int)div_up(a.m, s.tm);
    w.tiles_n = (int)div_up(a.n, s.tn);
    w.order = WorkOrder{s.kind == LARGE ? 32 : 64, 8};
    const unsigned blocks = (unsigned)((int64_t)w.tiles_m * w.tiles_n * s.splits);
    if (s.kind == VECTORS) hipLaunchKernelGGL((linear_few_kernel<TYPE, PAIR>), dim3(blocks), dim3(few_waves(PAIR) * 64), 0, st, a, s.splits);
    else if (s.kind == NARROW) hipLaunchKernelGGL((linear_narrow_kernel<TYPE, PAIR>), dim3(blocks), dim3(PAIR ? 256 : 512), 0, st, w);
    else if (s.kind == SMALL) hipLaunchKernelGGL((linear_small_kernel<TYPE, PAIR>), dim3(blocks), dim3(512), 0, st, w);
    else if (s.kind == HALF) hipLaunchKernelGGL((linear_half_kernel<TYPE, PAIR>), dim3(blocks), dim3(512), 0, st, w);
    else if (s.kind == MIDDLE) hipLaunchKernelGGL((linear_middle_kernel<TYPE, PAIR>), dim3(blocks), dim3(256), 0, st, w);
    else hipLaunchKernelGGL((linear_large_kernel<TYPE, PAIR>), dim3(blocks), dim3(512), 0, st, w);
    if (s.splits > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((linear_join_kernel<TYPE, PAIR>), dim3((unsigned)div_up(a.n, 2048), (unsigned)(a.m < 65535 ? a.m : 65535)), dim3(256), 0, st, a, s.splits);
    }
    return hipGetLastError();
}

// Large tiles run in rounds of one for every compute unit.  Where the last round has few of them, the rows or columns that they hold, of the longer
// dimension, are left to smaller tiles in a launch of their own (4608 x 4096 x 4096, 288 tiles: 136 us against 190; 2304 x 8192 x 4096, the same: 148, 189).
int64_t in_rounds(int64_t length, int64_t edge, int64_t across) {
    const int64_t tiles = across * div_up(length, edge), over = tiles % 256, whole = (tiles - over) / across;
    return over == 0 || whole == 0 || tiles - whole * across > 128 ? length : whole * edge;
}

template <int TYPE, bool PAIR>
hipError_t launch_shaped(LinearArgs a, hipStream_t st) {
    const Shape s = shape_of(a.m, a.n, a.k, PAIR);
    if (s.kind != LARGE) return launch_kind<TYPE, PAIR>(a, s, st);
    const int64_t m = a.m, n = a.n;
    if (m >= (PAIR ? 2 * n : n)) a.m = in_rounds(m, s.tm, div_up(n, s.tn));
    else a.n = in_rounds(n, s.tn, div_up(m, s.tm));
    const hipError_t e = launch_kind<TYPE, PAIR>(a, s, st);
    if (e != hipSuccess || (a.m == m && a.n == n)) return e;
    const auto rows = [](auto*& p, int64_t elements) {
        if (p != nullptr) p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(reinterpret_cast<uintptr_t>(p) + elements * 2);
    };
    if (a.m < m) {
        rows(a.X, a.m * a.ldx);
        rows(a.R, a.m * a.ldr);
        rows(a.Y, a.m * a.ldy);
        rows(a.Z, a.m * a.ldz);
        rows(a.U, a.m * a.ldu);
        a.m = m - a.m;
    } else {
        rows(a.W, a.n * a.ldw);
        rows(a.W2, a.n * a.ldw);
        rows(a.bias, a.n);
        rows(a.R, a.n);
        rows(a.Y, a.n);
        rows(a.Z, a.n);
        rows(a.U, a.n);
        a.n = n - a.n;
    }
    Shape rest = shape_of(a.m, a.n, a.k, PAIR);
    rest.splits = 1;
    return launch_kind<TYPE, PAIR>(a, rest, st);
}

template <int TYPE>
hipError_t launch_typed(const LinearArgs& a, hipStream_t st) { return a.W2 != nullptr ? launch_shaped<TYPE, true>(a, st) : launch_shaped<TYPE, false>(a, st); }

}  // namespace

size_t linear_bytes(int64_t m, int64_t n, int64_t k, bool pair) {
    const int splits = shape_of(m, n, k, pair).splits;
    return splits > 1 ? (size_t)splits * m * in_fours(n) * sizeof(float) * (pair ? 2 : 1) : 0;
}
hipError_t launch_linear(const LinearArgs& a, int type, hipStream_t st) { return type == TYPE_F16 ? launch_typed<TYPE_F16>(a, st) : launch_typed<TYPE_BF16>(a, st); }

}  // namespace ozaki
