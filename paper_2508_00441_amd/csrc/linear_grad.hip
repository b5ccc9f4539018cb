// Gradients of a linear layer with its activation, and of a pair of linear layers whose results are multiplied (linear.hip):
//     dz = dy act'(z),                         dx = dz W,               dW = dz^T x,   dbias = sum over rows of dz
//     dg = dy u act'(g),  du = dy act(g),      dx = dg Wg + du Wu,      dWg = dg^T x,  dWu = du^T x.
//
// dz (dg, du) is formed once, in 16 bits: its rounding is of the size of the results' own.  dbias is summed in the same pass, of what has not been
// rounded.  Without an activation dz is dy itself.  Both products are sums over 16-bit elements in FP32 on the matrix unit (tile_product.hpp); W in dx, and
// dz and x in dW, lie across the inner dimension and are turned on the way from LDS to registers.  The two terms of a pair's dx are one sum.
// Both products go in one launch, so that the tiles of one fill up what the other leaves of the compute units.  Where there are few tiles all the same, the inner
// dimension is cut into shares whose sums meet in work memory, in their order.
// Bound by the matrix unit and power, and by memory where dz is formed: pair of 4096 x 8192 x 4096 842 - 882 us, of which 68 form dg and du (4.8 TB/s) and the rest is the
// products' (1.36 - 1.40 PFLOP/s); 4096 x 8192 x 2048 with bias 249 - 255 us, 41 of them for dz.
#include "block_operators.hpp"
#include "layout.hpp"
#include "tile_epilogue.hpp"

namespace ozaki {
namespace {

constexpr int kind_of(int type) { return type == TYPE_F16 ? KIND_F16 : KIND_BF16; }
size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
int64_t in_eights(int64_t n) { return div_up(n, 8) * 8; }

// ---- dz and dbias ------------------------------------------------------------------------------------------------
struct SlopeWork {
    const void* Z;
    const void* U;
    const void* dY;
    void* dZ;                // null: only dbias is wanted
    void* dU;
    float* sums;             // null: no dbias; [chunk][columns in eights], or dbias itself where there is one chunk
    int64_t m, n, ldz, ldu, lddy, ld;        // ld: of dZ and dU
    int64_t rows;            // of a chunk
    int activation;
    bool whole;              // `sums` is dbias
};
constexpr int SLOPE_WAVES = 4, SLOPE_COLUMNS = 512;

// A wave has eight columns a lane and every fourth row of a chunk.  Memory at copy rate (4096 x 8192 of a pair: 335 MB in 68 us).
template <int TYPE, bool PAIR>
__global__ void __launch_bounds__(SLOPE_WAVES * 64) linear_slope_kernel(const SlopeWork w) {
    typedef typename Element<TYPE>::type T;
    typedef T eight __attribute__((ext_vector_type(8)));
    __shared__ v8f32 shares[SLOPE_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * 8, first = (int64_t)blockIdx.y * w.rows, end = first + w.rows < w.m ? first + w.rows : w.m;
    const int there = w.n - c < 8 ? (int)(w.n - c) : 8;          // columns; behind them the pieces hold anything
    v8f32 sum = {};
    if (there > 0) {
        with_activation(w.activation, [&](auto act) {
            constexpr int ACT = decltype(act)::value;
            const auto read = [&](const void* p, int64_t ld, int64_t r) { return __builtin_convertvector(*reinterpret_cast<const eight*>(static_cast<const T*>(p) + r * ld + c), v8f32); };
            const auto write = [&](void* p, int64_t r, v8f32 v) { *reinterpret_cast<eight*>(static_cast<T*>(p) + r * w.ld + c) = __builtin_convertvector(v, eight); };
#pragma unroll 2
            for (int64_t r = first + wave; r < end; r += SLOPE_WAVES) {
                v8f32 d = read(w.dY, w.lddy, r), z = {}, u = {};
                if constexpr (ACT != ACT_NONE || PAIR) z = read(w.Z, w.ldz, r);
                if constexpr (PAIR) u = read(w.U, w.ldu, r);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const Activation a = activation_of<ACT>(z[q]);
                    if constexpr (PAIR) {
                        z[q] = q < there ? d[q] * u[q] * a.slope : 0.0f;
                        u[q] = q < there ? d[q] * a.value : 0.0f;
                    } else {
                        z[q] = q < there ? d[q] * a.slope : 0.0f;
                    }
                }
                if (w.dZ != nullptr) write(w.dZ, r, z);
                if constexpr (PAIR) write(w.dU, r, u);
                sum += z;
            }
        });
    }
    if (PAIR || w.sums == nullptr) return;
    shares[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || there <= 0) return;
#pragma unroll
    for (int i = 1; i < SLOPE_WAVES; ++i) sum += shares[i][lane];
    float* const to = w.sums + (w.whole ? 0 : blockIdx.y * w.ld) + c;
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < there) to[q] = sum[q];
}

// The chunks' sums, in an order that depends on sizes only: 64 columns a workgroup, its waves each with a share of the chunks.
struct BiasJoin {
    const float* sums;       // null: nothing to do
    float* dbias;
    int64_t chunks, n, ld;
    unsigned blocks;
};
constexpr int BIAS_COLUMNS = 64, BIAS_WAVES = 4;
__device__ __forceinline__ void bias_join(const BiasJoin& w, float* lds, unsigned block) {
    const int lane = threadIdx.x & 63, share = threadIdx.x >> 6;
    const int64_t c = (int64_t)block * BIAS_COLUMNS + lane;
    float sum = 0.0f;
    if (c < w.n && share < BIAS_WAVES) {
#pragma unroll 8
        for (int64_t i = share; i < w.chunks; i += BIAS_WAVES) sum += w.sums[i * w.ld + c];
    }
    if (share < BIAS_WAVES) lds[share * 64 + lane] = sum;
    __syncthreads();
    if (share == 0 && c < w.n) w.dbias[c] = ((lds[lane] + lds[64 + lane]) + lds[128 + lane]) + lds[192 + lane];
}
__global__ void __launch_bounds__(BIAS_WAVES * 64) linear_bias_join_kernel(const BiasJoin w) {
    __shared__ float lds[BIAS_WAVES * 64];
    bias_join(w, lds, blockIdx.x);
}

// ---- products ----------------------------------------------------------------------------------------------------
// D = sum of the terms X Y^T; rows of Y are D's rows.  A pair's dX has two terms; a pair's dW is two results, one behind the other in `tiles_m`.
struct ProductWork {
    const uint8_t* X[2];
    const uint8_t* Y[2];
    void* D[2];
    int64_t ldx, ldy, ldd;   // ldx, ldy in bytes
    int64_t elements;        // of the inner dimension
    int64_t m, n;
    float* partial;          // splits > 1: [result][split][m][n in fours]
    int terms, results;
    int steps, splits;       // steps: of one term
    int tiles_m, tiles_n;    // of one result
    WorkOrder order;
};

// `b` of `blocks` workgroups
template <typename P, typename T, bool YT>
__device__ __forceinline__ void product_body(const ProductWork& w, uint8_t* lds, unsigned b, unsigned blocks) {
    const WorkItem item = work_item(b, blocks, w.order, w.tiles_m * w.results, w.tiles_n);
    const int result = item.bm >= (unsigned)w.tiles_m ? 1 : 0, split = item.gi;
    const int64_t m0 = (int64_t)(item.bm - result * w.tiles_m) * P::TM, n0 = (int64_t)item.bn * P::TN, left_m = w.m - m0, left_n = w.n - n0;
    const int begin = split_begin(w.steps * w.terms, w.splits, split), end = split_begin(w.steps * w.terms, w.splits, split + 1);
    v4f32 acc[P::FN][P::FM] = {};
#pragma unroll 1
    for (int t = 0; t < w.terms; ++t) {
        const int from = begin - t * w.steps > 0 ? begin - t * w.steps : 0, to = end - t * w.steps < w.steps ? end - t * w.steps : w.steps;
        if (from >= to) continue;
        const TileOperand X{w.X[t] + n0 * 2, w.ldx, (int)(left_n < P::TN ? left_n : P::TN), nullptr, 0, w.elements};
        const TileOperand Y{w.Y[YT ? result : t] + m0 * (YT ? 2 : w.ldy), w.ldy, (int)(left_m < P::TM ? left_m : P::TM), nullptr, 0, w.elements};
        P::multiply(lds, X, Y, w.elements * 2, from, to, acc);
    }
    if (w.splits > 1) {
        const int64_t ld = in_fours(w.n);
        put_tile<P>(lds, acc, m0, n0, left_m, in_fours(left_n), Partial{w.partial + ((int64_t)result * w.splits + split) * w.m * ld, ld, 0});
    } else {
        put_tile<P>(lds, acc, m0, n0, left_m, left_n, Plain<T, (P::TM == 256)>(static_cast<T*>(w.D[result]), w.ldd));
    }
}

// Both products, or one: `dx_blocks` workgroups have tiles of dX, the others of dW; `dx_first` says whose go out first.  Behind them the join of dbias.
struct BothWork {
    ProductWork dx, dw;
    BiasJoin bias;
    unsigned dx_blocks, dw_blocks;
    bool dx_first;
};
template <typename PX, typename PW, typename T>
__device__ __forceinline__ void both_body(const BothWork& w) {
    static_assert(PX::THREADS == PW::THREADS, "");
    __shared__ __attribute__((aligned(16))) uint8_t lds[PX::LDS_BYTES > PW::LDS_BYTES ? PX::LDS_BYTES : PW::LDS_BYTES];
    if (blockIdx.x >= w.dx_blocks + w.dw_blocks) {
        bias_join(w.bias, reinterpret_cast<float*>(lds), blockIdx.x - w.dx_blocks - w.dw_blocks);
        return;
    }
    const unsigned front = w.dx_first ? w.dx_blocks : w.dw_blocks, b = blockIdx.x < front ? blockIdx.x : blockIdx.x - front;
    if ((blockIdx.x < front) == w.dx_first) product_body<PX, T, false>(w.dx, lds, b, w.dx_blocks);
    else product_body<PW, T, true>(w.dw, lds, b, w.dw_blocks);
}

template <int TYPE>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) linear_grad_large_kernel(const BothWork w) {
    both_body<PairedTile<kind_of(TYPE), true, false>, PairedTile<kind_of(TYPE), true, true>, typename Element<TYPE>::type>(w);
}
// Of dX 64 x 128 elements or (FEW) 16 x 128, of dW 128 x 128, in eight waves: with four a step's wait, LDS reads and products follow each other (512 x 1024 x 1024:
// 14.7 us against 18); twice the steps under way in one workgroup to a compute unit are no faster.
template <int TYPE, bool FEW>
__global__ void __launch_bounds__(512) linear_grad_middle_kernel(const BothWork w) {
    constexpr int KIND = kind_of(TYPE);
    typedef std::conditional_t<FEW, Tile<KIND, 8, 1, 1, 1, 4, true, false>, Tile<KIND, 4, 2, 2, 2, 3, true, false>> DX;
    both_body<DX, Tile<KIND, 4, 2, 2, 4, 2, true, true>, typename Element<TYPE>::type>(w);
}

// the shares' sums in their order; blockIdx.z: the result
template <int TYPE>
__global__ void __launch_bounds__(256) linear_product_join_kernel(const ProductWork w) {
    typedef typename Element<TYPE>::type T;
    const int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, ld = in_fours(w.n);
    if (c >= w.n) return;
    T* const D = static_cast<T*>(w.D[blockIdx.z]);
    const bool wide = w.ldd % 4 == 0 && reinterpret_cast<uintptr_t>(D) % (4 * sizeof(T)) == 0;
    for (int64_t m = blockIdx.y; m < w.m; m += gridDim.y) {
        const float* from = w.partial + ((int64_t)blockIdx.z * w.splits * w.m + m) * ld + c;
        v4f32 sum = {};
#pragma unroll 4
        for (int s = 0; s < w.splits; ++s, from += w.m * ld) sum += *reinterpret_cast<const v4f32*>(from);
        put_four(D + m * w.ldd + c, sum, w.n - c, wide, false);
    }
}

enum { FEW, MIDDLE, LARGE };
struct Shape { int kind, tm, tn, splits; };
// Of dX, which is m x k, and of dW, `results` of n x k; `dx`, `dw`: which are wanted.  A size that has none: 0 tiles.
struct Shapes {
    Shape dx, dw;
    int64_t dx_tiles, dw_tiles, dx_steps, dw_steps;
};
Shapes shapes_of(int64_t m, int64_t n, int64_t k, bool pair, bool dx, bool dw) {
    const int results = pair ? 2 : 1;
    Shapes s = {};
    s.dx_steps = div_up(n, 64) * results;
    s.dw_steps = div_up(m, 64);
    const auto tiles = [](int64_t rows, int64_t columns, int64_t tm, int64_t tn) { return div_up(rows, tm) * div_up(columns, tn); };
    const int64_t dx_large = tiles(m, k, 256, 256), dw_large = results * tiles(n, k, 256, 256);
    // Large tiles where they are sixteen steps of every compute unit (1024 x 4096 x 2048, just that: 48.7 us, by smaller ones 50; half of it, 2048 x 2048 x 1024: 47, 37).
    const int64_t work = (dx ? dx_large * s.dx_steps : 0) + (dw ? dw_large * s.dw_steps : 0);
    const bool large = m > 128 && k > 128 && n > 128 && work >= 256 * 16;
    s.dx = large ? Shape{LARGE, 256, 256, 1} : m <= 16 ? Shape{FEW, 16, 128, 1} : Shape{MIDDLE, 64, 128, 1};
    s.dw = large ? Shape{LARGE, 256, 256, 1} : Shape{MIDDLE, 128, 128, 1};
    s.dx_tiles = dx ? tiles(m, k, s.dx.tm, s.dx.tn) : 0;
    s.dw_tiles = dw ? results * tiles(n, k, s.dw.tm, s.dw.tn) : 0;
    // Shares as long as a compute unit has steps to do in all, in which a step of dW's smaller tiles counts twice, and of eight steps at least.  Up to sixteen steps stay
    // uncut: the join costs more (333 x 1000 x 1001: 15.5, in shares of eight 18.1).
    const int64_t weight = large ? 1 : 2, all = s.dx_tiles * s.dx_steps + s.dw_tiles * s.dw_steps * weight, each = div_up(all, 256);
    const auto shares = [&](int64_t steps, int64_t weighted) {
        const int64_t want = (2 * weighted + each) / (2 * each), most = steps > 16 ? steps / 8 : 1, splits = want < most ? want : most;
        return (int)(splits < 1 ? 1 : splits > 32 ? 32 : splits);
    };
    s.dx.splits = shares(s.dx_steps, s.dx_steps);
    s.dw.splits = shares(s.dw_steps, s.dw_steps * weight);
    return s;
}

struct Places {
    uint8_t* dZ;
    uint8_t* dU;
    float* sums;
    uint8_t* partial;
    size_t total;
};
// Rows of a chunk.  With dbias: at most 128 chunks, whose sums the join reads.
int64_t chunk_rows(int64_t m, int64_t n, bool pair) {
    const int64_t strips = div_up(n, SLOPE_COLUMNS), want = 2048 / strips, most = pair ? 65535 : 128, chunks = want < 1 ? 1 : want > most ? most : want, rows = div_up(m, chunks);
    return rows < SLOPE_WAVES ? SLOPE_WAVES : rows;
}
size_t partial_bytes(const Shapes& s, int64_t m, int64_t n, int64_t k, int results, size_t& for_dx) {
    for_dx = s.dx.splits > 1 && s.dx_tiles > 0 ? up((size_t)s.dx.splits * m * in_fours(k) * 4) : 0;
    return for_dx + (s.dw.splits > 1 && s.dw_tiles > 0 ? up((size_t)results * s.dw.splits * n * in_fours(k) * 4) : 0);
}
Places places_of(uint8_t* ws, int64_t m, int64_t n, int64_t k, bool pair) {
    Places p;
    size_t at = 0, unused;
    const auto take = [&](size_t bytes) { uint8_t* const here = ws + at; at += up(bytes); return here; };
    p.dZ = take((size_t)m * in_eights(n) * 2);
    p.dU = take(pair ? (size_t)m * in_eights(n) * 2 : 0);
    p.sums = reinterpret_cast<float*>(take(pair ? 0 : (size_t)div_up(m, chunk_rows(m, n, pair)) * in_eights(n) * 4));
    // the shares' sums, of whatever results a call asks for
    size_t most = 0;
    for (int which = 1; which < 4; ++which) {
        const size_t need = partial_bytes(shapes_of(m, n, k, pair, which & 1, which & 2), m, n, k, pair ? 2 : 1, unused);
        most = need > most ? need : most;
    }
    p.partial = take(most);
    p.total = at;
    return p;
}

#define OZAKI_LINEAR_TRY(expr) do { const hipError_t e_ = (expr); if (e_ != hipSuccess) return e_; } while (0)

template <int TYPE>
hipError_t launch_join(const ProductWork& w, hipStream_t st) {
    if (w.splits == 1) return hipSuccess;
    hipLaunchKernelGGL((linear_product_join_kernel<TYPE>), dim3((unsigned)div_up(w.n, 1024), (unsigned)(w.m < 65535 ? w.m : 65535), (unsigned)w.results), dim3(256), 0, st, w);
    return hipGetLastError();
}
unsigned set_tiles(ProductWork& w, const Shape& s) {
    w.splits = s.splits;
    w.tiles_m = (int)div_up(w.m, s.tm);
    w.tiles_n = (int)div_up(w.n, s.tn);
    w.order = WorkOrder{s.kind == LARGE ? 32 : 64, 8};
    return (unsigned)((int64_t)w.tiles_m * w.results * w.tiles_n * w.splits);
}
template <int TYPE>
hipError_t launch_both(BothWork w, const Shapes& s, bool dx, bool dw, hipStream_t st) {
    w.dx_blocks = dx ? set_tiles(w.dx, s.dx) : 0;
    w.dw_blocks = dw ? set_tiles(w.dw, s.dw) : 0;
    w.dx_first = s.dx_steps / s.dx.splits >= s.dw_steps / s.dw.splits;
    const dim3 blocks(w.dx_blocks + w.dw_blocks + w.bias.blocks);
    if (s.dw.kind == LARGE) hipLaunchKernelGGL((linear_grad_large_kernel<TYPE>), blocks, dim3(512), 0, st, w);
    else if (s.dx.kind == FEW) hipLaunchKernelGGL((linear_grad_middle_kernel<TYPE, true>), blocks, dim3(512), 0, st, w);
    else hipLaunchKernelGGL((linear_grad_middle_kernel<TYPE, false>), blocks, dim3(512), 0, st, w);
    OZAKI_LINEAR_TRY(hipGetLastError());
    if (dx) OZAKI_LINEAR_TRY(launch_join<TYPE>(w.dx, st));
    return dw ? launch_join<TYPE>(w.dw, st) : hipSuccess;
}

template <int TYPE>
hipError_t grad_typed(const LinearGradArgs& a, hipStream_t st) {
    const bool pair = a.pair, products = a.dX != nullptr || a.dW != nullptr || a.dW2 != nullptr;
    const Places p = places_of(a.ws, a.m, a.n, a.k, pair);
    // (dY's pieces behind the end of a row hold anything, which dX's product, only one of whose operands is turned, would take)
    const bool formed = pair || a.activation != ACT_NONE || a.n % 8 != 0;
    SlopeWork w = {};
    w.Z = a.Z;
    w.U = a.U;
    w.dY = a.dY;
    w.dZ = formed && products ? p.dZ : nullptr;
    w.dU = p.dU;
    w.m = a.m;
    w.n = a.n;
    w.ldz = a.ldz;
    w.ldu = a.ldu;
    w.lddy = a.lddy;
    w.ld = in_eights(a.n);
    w.activation = a.activation;
    w.rows = chunk_rows(a.m, a.n, pair);
    const int64_t chunks = div_up(a.m, w.rows);
    w.whole = chunks == 1;
    w.sums = a.dbias == nullptr ? nullptr : w.whole ? a.dbias : p.sums;
    if (w.dZ != nullptr || w.sums != nullptr) {
        const dim3 blocks((unsigned)div_up(a.n, SLOPE_COLUMNS), (unsigned)chunks);
        if (pair) hipLaunchKernelGGL((linear_slope_kernel<TYPE, true>), blocks, dim3(SLOPE_WAVES * 64), 0, st, w);
        else hipLaunchKernelGGL((linear_slope_kernel<TYPE, false>), blocks, dim3(SLOPE_WAVES * 64), 0, st, w);
        OZAKI_LINEAR_TRY(hipGetLastError());
    }
    const uint8_t* const dz[2] = {formed ? p.dZ : static_cast<const uint8_t*>(a.dY), p.dU};
    const int64_t lddz = (formed ? w.ld : a.lddy) * 2;
    const bool dx = a.dX != nullptr, both = a.dW != nullptr && a.dW2 != nullptr, dw = a.dW != nullptr || a.dW2 != nullptr;
    BothWork d = {};
    if (w.sums != nullptr && !w.whole) d.bias = BiasJoin{p.sums, a.dbias, chunks, a.n, w.ld, (unsigned)div_up(a.n, BIAS_COLUMNS)};
    if (!dx && !dw) {
        if (d.bias.blocks > 0) hipLaunchKernelGGL(linear_bias_join_kernel, dim3(d.bias.blocks), dim3(BIAS_WAVES * 64), 0, st, d.bias);
        return hipGetLastError();
    }
    // (of a pair one dW is cut as both are, so that it has the same bits)
    const Shapes s = shapes_of(a.m, a.n, a.k, pair, dx, dw);
    size_t for_dx;
    partial_bytes(s, a.m, a.n, a.k, pair ? 2 : 1, for_dx);
    if (dx) {
        d.dx.X[0] = static_cast<const uint8_t*>(a.W);
        d.dx.X[1] = static_cast<const uint8_t*>(a.W2);
        d.dx.Y[0] = dz[0];
        d.dx.Y[1] = dz[1];
        d.dx.D[0] = a.dX;
        d.dx.ldx = a.ldw * 2;
        d.dx.ldy = lddz;
        d.dx.ldd = a.lddx;
        d.dx.elements = a.n;
        d.dx.m = a.m;
        d.dx.n = a.k;
        d.dx.partial = reinterpret_cast<float*>(p.partial);
        d.dx.terms = pair ? 2 : 1;
        d.dx.results = 1;
        d.dx.steps = (int)div_up(a.n, 64);
    }
    if (dw) {
        d.dw.X[0] = static_cast<const uint8_t*>(a.X);
        d.dw.Y[0] = a.dW != nullptr ? dz[0] : dz[1];
        d.dw.Y[1] = dz[1];
        d.dw.D[0] = a.dW != nullptr ? a.dW : a.dW2;
        d.dw.D[1] = a.dW2;
        d.dw.ldx = a.ldx * 2;
        d.dw.ldy = lddz;
        d.dw.ldd = a.lddw;
        d.dw.elements = a.m;
        d.dw.m = a.n;
        d.dw.n = a.k;
        d.dw.partial = reinterpret_cast<float*>(p.partial + for_dx);
        d.dw.terms = 1;
        d.dw.results = both ? 2 : 1;
        d.dw.steps = (int)div_up(a.m, 64);
    }
    return launch_both<TYPE>(d, s, dx, dw, st);
}

}  // namespace

size_t linear_grad_bytes(int64_t m, int64_t n, int64_t k, bool pair) { return places_of(nullptr, m, n, k, pair).total; }
hipError_t launch_linear_grad(const LinearGradArgs& a, int type, hipStream_t st) { return type == TYPE_F16 ? grad_typed<TYPE_F16>(a, st) : grad_typed<TYPE_BF16>(a, st); }

}  // namespace ozaki
