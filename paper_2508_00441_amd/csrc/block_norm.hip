// What lies between two blocks of a model: the norm behind a block, its gate and scale, the sum that runs through the model, the norm in front of the
// next block; and the gradient of all of it.
//     u = x * rho(x) * w_post (or x),   r' = r + scale * gate * u,   h = r' * rho(r') * w_pre,        rho(v) = 1 / sqrt(mean(v^2) + eps)
// with, for the gradient, n = r' rho(r'), m = x rho(x):
//     dn = dh w_pre          dr = dr' + rho(r') (dn - n mean(dn n))          dw_pre = sum over rows of dh n
//     dm = scale gate dr w_post      dx = rho(x) (dm - m mean(dm m))         s = sum over rows of dr m,  dw_post = scale gate s,  dgate = scale w_post s.
//
// Every element is read and written once: a workgroup keeps a row in registers from the loads to the stores.  Sums are in
// 32 bits; where a row's squares leave their range, above or below, its sums are formed again with the row times a power of two.  Sums over rows
// are kept in registers over the rows that a workgroup has one after another, and meet in work memory; a second launch adds them up, in an order that
// depends on sizes only.
#include "block_operators.hpp"

namespace ozaki {
namespace {

template <typename T> struct Eight { typedef T type __attribute__((ext_vector_type(8))); };

// eight elements of a vector, of which `there` exist (zeros for the others); the 16 bytes in which a vector ends may be read whole
template <typename T> __device__ __forceinline__ v8f32 load_eight(const T* p, int there) {
    v8f32 v = {};
    if (there <= 0) return v;
    if constexpr (sizeof(T) == 4) {
        const v4f32 lo = *reinterpret_cast<const v4f32*>(p);
        v4f32 hi = {};
        if (there > 4) hi = *reinterpret_cast<const v4f32*>(p + 4);
        v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        v = __builtin_convertvector(*reinterpret_cast<const typename Eight<T>::type*>(p), v8f32);
    }
    if (there < 8) {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = q < there ? v[q] : 0.0f;
    }
    return v;
}
// of weights, which lie anywhere
__device__ __forceinline__ v8f32 load_weights(const float* p, int there, bool wide) {
    if (wide && there >= 8) return load_eight(p, 8);
    v8f32 v = {};
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < there) v[q] = p[q];
    return v;
}
template <typename T> __device__ __forceinline__ void store_eight(T* p, v8f32 v, int there, bool wide) {
    if (wide && there >= 8) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<v4f32*>(p) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
            *reinterpret_cast<v4f32*>(p + 4) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
        } else {
            *reinterpret_cast<typename Eight<T>::type*>(p) = __builtin_convertvector(v, typename Eight<T>::type);
        }
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < there) p[q] = (T)v[q];
    }
}
template <typename T> __device__ __forceinline__ bool rows_wide(const T* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * sizeof(T) % 16 == 0; }

// The sums of N numbers over a workgroup, for all its threads; `lds` has room for N numbers a wave and is free again when the next call's first barrier is passed.
template <int THREADS, int N> __device__ __forceinline__ void row_sums(float (&v)[N], float* lds) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], d);
    if constexpr (THREADS > 64) {
        constexpr int WAVES = THREADS / 64;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) lds[(threadIdx.x >> 6) * N + i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = lds[(threadIdx.x & (WAVES - 1)) * N + i];
#pragma unroll
            for (int d = 1; d < WAVES; d <<= 1) v[i] += __shfl_xor(v[i], d);
        }
    }
}
__device__ __forceinline__ float dot(v8f32 a, v8f32 b, float s) {
#pragma unroll
    for (int q = 0; q < 8; ++q) s = __builtin_fmaf(a[q], b[q], s);
    return s;
}

// rho of a row and (ALONG) mean(d n) with n = row * rho; through(p): piece p of d
struct RowNorm { float rho, along; };
template <int THREADS, bool ALONG, int PIECES, typename F>
__device__ __forceinline__ RowNorm row_norm(const v8f32 (&x)[PIECES], F through, float k, float eps, float* lds) {
    float s[ALONG ? 2 : 1] = {};
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        s[0] = dot(x[p], x[p], s[0]);
        if constexpr (ALONG) s[1] = dot(through(p), x[p], s[1]);
    }
    row_sums<THREADS>(s, lds);
    RowNorm r = {__builtin_amdgcn_rsqf(s[0] / k + eps), 0.0f};
    const bool above = !(s[0] < 0x1p126f), below = s[0] < 0x1p-90f && eps < 0x1p-80f;
    bool again = above || below;
    if constexpr (ALONG) {
        r.along = s[1] * r.rho / k;
        again = again || !(fabsf(s[1]) < __builtin_inff());
    }
    if (again) {                                     // (the same for all threads)
        // times 2^-72 no row's squares are too large, times 2^100 no row's that came to so little too small
        const float f = above ? 0x1p-72f : below ? 0x1p100f : 1.0f;
        float q[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < PIECES; ++p) q[0] = dot(x[p] * f, x[p] * f, q[0]);
        row_sums<THREADS>(q, lds);
        r.rho = f * __builtin_amdgcn_rsqf(q[0] / k + eps * f * f);
        if constexpr (ALONG) {
            q[0] = 0.0f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) q[0] = dot(through(p), x[p] * r.rho, q[0]);
            row_sums<THREADS>(q, lds);
            r.along = q[0] / k;
        }
    }
    return r;
}

template <int TYPE, int TYPE_R, int THREADS, int PIECES>
__global__ void __launch_bounds__(THREADS) block_norm_kernel(const BlockNormArgs a) {
    typedef typename Element<TYPE>::type T;
    typedef typename Element<TYPE_R>::type TR;
    __shared__ float lds[THREADS / 64];
    const auto none = [](int) { return v8f32{}; };
    const T* const X = static_cast<const T*>(a.X);
    const TR* const R = static_cast<const TR*>(a.R);
    TR* const R_out = static_cast<TR*>(a.R_out);
    T* const H = static_cast<T*>(a.H);
    const bool wide_r = rows_wide(R_out, a.ldro), wide_h = rows_wide(H, a.ldh);
    const bool wide_post = rows_wide(a.w_post, 0), wide_pre = rows_wide(a.w_pre, 0), wide_gate = rows_wide(a.gate, a.k);
    int c[PIECES], there[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        c[p] = (p * THREADS + threadIdx.x) * 8;
        there[p] = (int)a.k - c[p];
    }
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        v8f32 x[PIECES], r[PIECES];
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            x[p] = X != nullptr ? load_eight(X + row * a.ldx + c[p], there[p]) : v8f32{};
            r[p] = R != nullptr ? load_eight(R + row * a.ldr + c[p], there[p]) : v8f32{};
        }
        if (X != nullptr) {
            const float rho = a.w_post != nullptr ? row_norm<THREADS, false>(x, none, (float)a.k, a.eps, lds).rho : 1.0f;
            const float* const gate = a.gate != nullptr ? a.gate + row / a.group * a.k : nullptr;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                v8f32 u = x[p];
                if (a.w_post != nullptr) u = u * rho * load_weights(a.w_post + c[p], there[p], wide_post);
                if (gate != nullptr) u *= load_weights(gate + c[p], there[p], wide_gate);
                r[p] += u * a.scale;
                if (R_out != nullptr) store_eight(R_out + row * a.ldro + c[p], r[p], there[p], wide_r);
            }
        }
        if (H == nullptr) continue;
        const float rho = row_norm<THREADS, false>(r, none, (float)a.k, a.eps, lds).rho;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) store_eight(H + row * a.ldh + c[p], r[p] * rho * load_weights(a.w_pre + c[p], there[p], wide_pre), there[p], wide_h);
    }
}

// ---- gradient ----------------------------------------------------------------------------------------------------
// A workgroup has a chunk of neighbouring rows.  Where a gate's rows are more than a chunk, a chunk lies inside them and leaves its s; where they are fewer, a chunk
// is some gates' rows and leaves each one's s.
struct NormChunks {
    int64_t group, groups;   // rows of a gate (or all, without one), and how many gates
    int64_t rows, per_group; // of a chunk; chunks in a group, 0: groups in a chunk
    int64_t chunks, units;   // units: of s
};
struct NormGradWork {
    BlockNormArgs a;
    NormChunks n;
    float* t;                // [chunk][k]: sums of dh n; null: not wanted
    float* s;                // [unit][k]; null: not wanted
};

template <int TYPE, int TYPE_R, int THREADS, int PIECES>
__global__ void __launch_bounds__(THREADS) block_norm_grad_kernel(const NormGradWork w) {
    typedef typename Element<TYPE>::type T;
    typedef typename Element<TYPE_R>::type TR;
    __shared__ float lds[2 * (THREADS / 64)];
    // The sums over rows, t and s: in registers, or (the longest rows, which leave no registers) a thread's own places in LDS.
    constexpr bool HELD = THREADS == 1024 && PIECES == 2;
    __shared__ v4f32 held[HELD ? 4 * PIECES : 1][HELD ? THREADS : 1];
    v8f32 kept[2][HELD ? 1 : PIECES] = {};
    const auto add = [&](int which, int p, v8f32 v) {
        if constexpr (HELD) {
            held[which * 4 + 2 * p][threadIdx.x] += __builtin_shufflevector(v, v, 0, 1, 2, 3);
            held[which * 4 + 2 * p + 1][threadIdx.x] += __builtin_shufflevector(v, v, 4, 5, 6, 7);
        } else {
            kept[which][p] += v;
        }
    };
    if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < 4 * PIECES; ++i) held[i][threadIdx.x] = v4f32{};
    }
    const BlockNormArgs& a = w.a;
    const T* const X = static_cast<const T*>(a.X);
    const T* const dH = static_cast<const T*>(a.dH);
    const TR* const R = static_cast<const TR*>(a.R);
    const TR* const dR_out = static_cast<const TR*>(a.dR_out);
    T* const dX = static_cast<T*>(a.dX);
    TR* const dR = static_cast<TR*>(a.dR);
    const bool wide_x = rows_wide(dX, a.lddx), wide_r = rows_wide(dR, a.lddr);
    const bool wide_post = rows_wide(a.w_post, 0), wide_pre = rows_wide(a.w_pre, 0), wide_gate = rows_wide(a.gate, a.k);
    const bool post = X != nullptr && a.w_post != nullptr, branch = X != nullptr && (dX != nullptr || w.s != nullptr);
    int c[PIECES], there[PIECES];
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        c[p] = (p * THREADS + threadIdx.x) * 8;
        there[p] = (int)a.k - c[p];
    }
    const auto leave = [&](float* to, int which) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            v8f32 v;
            if constexpr (HELD) {
                v = __builtin_shufflevector(held[which * 4 + 2 * p][threadIdx.x], held[which * 4 + 2 * p + 1][threadIdx.x], 0, 1, 2, 3, 4, 5, 6, 7);
                held[which * 4 + 2 * p][threadIdx.x] = held[which * 4 + 2 * p + 1][threadIdx.x] = v4f32{};
            } else {
                v = kept[which][p];
                kept[which][p] = v8f32{};
            }
            store_eight(to + c[p], v, there[p], a.k % 4 == 0);
        }
    };
    const NormChunks& n = w.n;
    int64_t row, end, left;                          // left: rows to the end of the unit
    int64_t unit;
    if (n.per_group > 0) {
        const int64_t g = blockIdx.x / n.per_group, j = blockIdx.x - g * n.per_group, last = (g + 1) * n.group < a.rows ? (g + 1) * n.group : a.rows;
        row = g * n.group + j * n.rows;
        end = row + n.rows < last ? row + n.rows : last;
        left = end - row;
        unit = blockIdx.x;
    } else {
        row = blockIdx.x * n.rows;
        end = row + n.rows < a.rows ? row + n.rows : a.rows;
        left = n.group;
        unit = blockIdx.x * (n.rows / n.group);
    }
    for (; row < end; ++row) {
        v8f32 x[PIECES], r[PIECES], dh[PIECES], dr[PIECES];
        const auto load_x = [&]() {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) x[p] = branch ? load_eight(X + row * a.ldx + c[p], there[p]) : v8f32{};
        };
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            dr[p] = dR_out != nullptr ? load_eight(dR_out + row * a.lddro + c[p], there[p]) : v8f32{};
            dh[p] = dH != nullptr ? load_eight(dH + row * a.lddh + c[p], there[p]) : v8f32{};
            r[p] = dH != nullptr ? load_eight(R + row * a.ldr + c[p], there[p]) : v8f32{};
        }
        if constexpr (!HELD) load_x();
        if (dH != nullptr) {
            const RowNorm rn = row_norm<THREADS, true>(r, [&](int p) { return dh[p] * load_weights(a.w_pre + c[p], there[p], wide_pre); }, (float)a.k, a.eps, lds);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const v8f32 n = r[p] * rn.rho;
                dr[p] += (dh[p] * load_weights(a.w_pre + c[p], there[p], wide_pre) - n * rn.along) * rn.rho;
                add(0, p, dh[p] * n);
            }
        }
        if (dR != nullptr) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) store_eight(dR + row * a.lddr + c[p], dr[p], there[p], wide_r);
        }
        if (branch) {
            if constexpr (HELD) load_x();
            // what the gradient of m is, or of x without a norm
            const float* const gate = a.gate != nullptr ? a.gate + row / a.group * a.k : nullptr;
            const auto through = [&](int p) {
                v8f32 d = dr[p] * a.scale;
                if (gate != nullptr) d *= load_weights(gate + c[p], there[p], wide_gate);
                return post ? d * load_weights(a.w_post + c[p], there[p], wide_post) : d;
            };
            RowNorm xn = {1.0f, 0.0f};
            if (post) xn = row_norm<THREADS, true>(x, through, (float)a.k, a.eps, lds);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const v8f32 m = x[p] * xn.rho;
                add(1, p, dr[p] * m);
                if (dX != nullptr) store_eight(dX + row * a.lddx + c[p], post ? (through(p) - m * xn.along) * xn.rho : through(p), there[p], wide_x);
            }
        }
        if (--left == 0 && n.per_group == 0) {
            if (w.s != nullptr) leave(w.s + unit * a.k, 1);
            ++unit;
            left = n.group;
        }
    }
    if (w.s != nullptr && (n.per_group > 0 || left < n.group)) leave(w.s + unit * a.k, 1);
    if (w.t != nullptr) leave(w.t + blockIdx.x * a.k, 0);
}

// Sums over chunks and units: 32 columns a workgroup, in 32 shares.  blockIdx.y: 0 dw_pre, 1 dw_post, from 2 on a gate's gradient.
constexpr int JOIN_COLUMNS = 32, JOIN_SHARES = 32;
__global__ void __launch_bounds__(JOIN_COLUMNS * JOIN_SHARES) block_norm_join_kernel(const NormGradWork w) {
    __shared__ float shares[JOIN_SHARES][JOIN_COLUMNS + 1];
    const BlockNormArgs& a = w.a;
    const NormChunks& n = w.n;
    const int in = threadIdx.x % JOIN_COLUMNS, share = threadIdx.x / JOIN_COLUMNS;
    const int64_t c = (int64_t)blockIdx.x * JOIN_COLUMNS + in, what = blockIdx.y;
    if (what == 0 ? a.dw_pre == nullptr : what == 1 ? a.dw_post == nullptr : false) return;
    float sum = 0.0f;
    if (c < a.k) {
        if (what == 0) {
#pragma unroll 8
            for (int64_t i = share; i < n.chunks; i += JOIN_SHARES) sum += w.t[i * a.k + c];
        } else if (what == 1) {
#pragma unroll 8
            for (int64_t i = share; i < n.units; i += JOIN_SHARES)
                sum += w.s[i * a.k + c] * (a.gate != nullptr ? a.gate[(n.per_group > 0 ? i / n.per_group : i) * a.k + c] : 1.0f);
        } else {
            const float* const from = w.s + (what - 2) * n.per_group * a.k + c;
#pragma unroll 8
            for (int64_t i = share; i < n.per_group; i += JOIN_SHARES) sum += from[i * a.k];
        }
    }
    shares[share][in] = sum;
    __syncthreads();
    // share i of the 32 takes column i: a wave has two columns' 32 sums
    const int column = threadIdx.x / JOIN_SHARES, from = threadIdx.x % JOIN_SHARES;
    sum = shares[from][column];
#pragma unroll
    for (int d = 1; d < JOIN_SHARES; d <<= 1) sum += __shfl_xor(sum, d);
    const int64_t to = (int64_t)blockIdx.x * JOIN_COLUMNS + column;
    if (from != 0 || to >= a.k) return;
    if (what == 0) a.dw_pre[to] = sum;
    else if (what == 1) a.dw_post[to] = sum * a.scale;
    else a.dgate[(what - 2) * a.k + to] = sum * a.scale * (a.w_post != nullptr ? a.w_post[to] : 1.0f);
}
// a gate's gradient where its rows are one unit
__global__ void __launch_bounds__(256) block_norm_gate_kernel(const NormGradWork w) {
    const BlockNormArgs& a = w.a;
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= a.k) return;
    const float factor = a.scale * (a.w_post != nullptr ? a.w_post[c] : 1.0f);
    for (int64_t g = blockIdx.y; g < w.n.groups; g += gridDim.y) a.dgate[g * a.k + c] = w.s[g * a.k + c] * factor;
}

// ---- launches ----------------------------------------------------------------------------------------------------
// threads and pieces of eight elements a thread that hold a row
struct RowShape { int threads, pieces; };
RowShape row_shape(int64_t k) {
    return k <= 512 ? RowShape{64, 1} : k <= 1024 ? RowShape{64, 2} : k <= 2048 ? RowShape{256, 1} : k <= 4096 ? RowShape{256, 2} : k <= 8192 ? RowShape{1024, 1} : RowShape{1024, 2};
}
NormChunks norm_chunks(int64_t rows, int64_t k, int64_t group) {
    const int threads = row_shape(k).threads;
    const int64_t most = threads == 64 ? 2048 : threads == 256 ? 768 : 256;
    NormChunks n;
    n.group = group > 0 && group < rows ? group : rows;
    n.groups = div_up(rows, n.group);
    n.rows = div_up(rows, most);
    if (n.group >= n.rows) {
        n.per_group = div_up(n.group, n.rows);
        n.chunks = n.units = n.groups * n.per_group;
    } else {
        n.rows = n.rows / n.group * n.group;
        n.per_group = 0;
        n.chunks = div_up(rows, n.rows);
        n.units = n.groups;
    }
    return n;
}
size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

template <typename F> hipError_t with_shape(int64_t k, F f) {
    const RowShape s = row_shape(k);
    if (s.threads == 64) return s.pieces == 1 ? f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>()) : f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    if (s.threads == 256) return s.pieces == 1 ? f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>()) : f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    return s.pieces == 1 ? f(std::integral_constant<int, 1024>(), std::integral_constant<int, 1>()) : f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
}
template <typename F> hipError_t with_types(int type, int type_r, F f) {
    if (type == TYPE_F32) return f(std::integral_constant<int, TYPE_F32>(), std::integral_constant<int, TYPE_F32>());
    if (type == TYPE_BF16) return type_r == TYPE_F32 ? f(std::integral_constant<int, TYPE_BF16>(), std::integral_constant<int, TYPE_F32>())
                                                     : f(std::integral_constant<int, TYPE_BF16>(), std::integral_constant<int, TYPE_BF16>());
    return type_r == TYPE_F32 ? f(std::integral_constant<int, TYPE_F16>(), std::integral_constant<int, TYPE_F32>())
                              : f(std::integral_constant<int, TYPE_F16>(), std::integral_constant<int, TYPE_F16>());
}

}  // namespace

size_t block_norm_grad_bytes(int64_t rows, int64_t k, int64_t group) {
    if (rows == 0) return 0;
    const NormChunks n = norm_chunks(rows, k, group);
    return up((size_t)n.chunks * k * 4) + up((size_t)n.units * k * 4);
}

hipError_t launch_block_norm(const BlockNormArgs& a, int type, int type_r, hipStream_t st) {
    return with_types(type, type_r, [&](auto t, auto tr) {
        return with_shape(a.k, [&](auto threads, auto pieces) {
            constexpr int T = decltype(t)::value, TR = decltype(tr)::value, THREADS = decltype(threads)::value, PIECES = decltype(pieces)::value;
            const int64_t most = 256 * (2048 / THREADS);
            hipLaunchKernelGGL((block_norm_kernel<T, TR, THREADS, PIECES>), dim3((unsigned)(a.rows < most ? a.rows : most)), dim3(THREADS), 0, st, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_block_norm_grad(const BlockNormArgs& a, int type, int type_r, hipStream_t st) {
    NormGradWork w;
    w.a = a;
    w.n = norm_chunks(a.rows, a.k, a.gate != nullptr ? a.group : 0);
    float* const t = reinterpret_cast<float*>(a.ws);
    w.t = a.dw_pre != nullptr ? t : nullptr;
    w.s = a.dw_post != nullptr || a.dgate != nullptr ? reinterpret_cast<float*>(a.ws + up((size_t)w.n.chunks * a.k * 4)) : nullptr;
    const hipError_t e = with_types(type, type_r, [&](auto ty, auto tr) {
        return with_shape(a.k, [&](auto threads, auto pieces) {
            constexpr int T = decltype(ty)::value, TR = decltype(tr)::value, THREADS = decltype(threads)::value, PIECES = decltype(pieces)::value;
            hipLaunchKernelGGL((block_norm_grad_kernel<T, TR, THREADS, PIECES>), dim3((unsigned)w.n.chunks), dim3(THREADS), 0, st, w);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || (w.t == nullptr && w.s == nullptr)) return e;
    const bool gates = a.dgate != nullptr && w.n.per_group > 0;
    if (a.dw_pre != nullptr || a.dw_post != nullptr || gates) {
        hipLaunchKernelGGL(block_norm_join_kernel, dim3((unsigned)div_up(a.k, JOIN_COLUMNS), (unsigned)(gates ? 2 + w.n.groups : 2)), dim3(JOIN_COLUMNS * JOIN_SHARES), 0, st, w);
        const hipError_t j = hipGetLastError();
        if (j != hipSuccess) return j;
    }
    if (a.dgate != nullptr && !gates) {
        hipLaunchKernelGGL(block_norm_gate_kernel, dim3((unsigned)div_up(a.k, 256), (unsigned)(w.n.groups < 65535 ? w.n.groups : 65535)), dim3(256), 0, st, w);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace ozaki
