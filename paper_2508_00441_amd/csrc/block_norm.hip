// What lies between two blocks of a model: the norm behind a block, its gate and scale, the sum that runs through the model, the norm in front of the
// next block; and the gradient of all of it.
//     u = x * rho(x) * w_post (or x),   r' = r + scale * gate * u,   h = r' * rho(r') * w_pre,        rho(v) = 1 / sqrt(mean(v^2) + eps)
// with, for the gradient, n = r' rho(r'), m = x rho(x):
//     dn = dh w_pre          dr = dr' + rho(r') (dn - n mean(dn n))          dw_pre = sum over rows of dh n
//     dm = scale gate dr w_post      dx = rho(x) (dm - m mean(dm m))         s = sum over rows of dr m,  dw_post = scale gate s,  dgate = scale w_post s.
//
// Every element is read and written once: a workgroup keeps a row in registers from the loads to the stores (the gradient of rows of more than 8192, in 32 bits 4096, reads
// them again from the caches).  Sums are in 32 bits; where a row's squares leave their range, above or below, its sums are formed again with the row
// times a power of two.  Sums over rows are kept in LDS over the rows that a workgroup has one after another, and meet in work memory; a second launch adds them
// up, in an order that depends on sizes only.
// Bound by memory: 8192 x 4096 with both norms, gates and 32-bit sums 81 us, 5.0 TB/s; its gradient in 16 bits 95 us, 4.4 TB/s in the kernel and 6 us for the join.
#include "block_operators.hpp"

namespace ozaki {
namespace {

// Eight elements of a vector as they are in memory, and as numbers: `there` of them exist (zeros for the others); the 16 bytes in which a vector ends
// may be read whole.
template <typename T> struct Raw { v4i32 part[sizeof(T) / 2]; };
// (a row's address is the same for all lanes and stays in scalar registers; a lane adds 32 bits to it)
template <typename T> __device__ __forceinline__ const T* place(const T* row, unsigned c) {
    return reinterpret_cast<const T*>(reinterpret_cast<const uint8_t*>(row) + c * (unsigned)sizeof(T));
}
template <typename T> __device__ __forceinline__ T* place(T* row, unsigned c) { return const_cast<T*>(place(const_cast<const T*>(row), c)); }
template <typename T> __device__ __forceinline__ Raw<T> load_raw(const T* row, unsigned c, int there) {
    Raw<T> r = {};
    if (there > 0) r.part[0] = *reinterpret_cast<const v4i32*>(place(row, c));
    if constexpr (sizeof(T) == 4)
        if (there > 4) r.part[1] = *reinterpret_cast<const v4i32*>(place(row, c + 4));
    return r;
}
template <typename T> __device__ __forceinline__ v8f32 numbers(const Raw<T>& r, int there) {
    v8f32 v;
    if constexpr (sizeof(T) == 4) v = __builtin_bit_cast(v8f32, r);
    else v = __builtin_convertvector(__builtin_bit_cast(Eight<T>, r), v8f32);
    if (there < 8) {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = q < there ? v[q] : 0.0f;
    }
    return v;
}
// of weights and results, which lie anywhere
__device__ __forceinline__ v8f32 load_weights(const float* p, int there) {
    if (there >= 8) return get_eight(p);
    v8f32 v = {};
#pragma unroll
    for (int q = 0; q < 8; ++q)
        if (q < there) v[q] = p[q];
    return v;
}
template <typename T> __device__ __forceinline__ void store_eight(T* p, v8f32 v, int there) {
    if (there >= 8) {
        put_eight<false>(p, v);
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (q < there) p[q] = (T)v[q];
    }
}

// Sums over a wave, without LDS: rows of sixteen lanes, then across them.
template <int CONTROL, int ROWS> __device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CONTROL, ROWS, 0xF, false));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += moved<0x111, 0xF>(v);           // from 1, 2, 4, 8 lanes below
    v += moved<0x112, 0xF>(v);
    v += moved<0x114, 0xF>(v);
    v += moved<0x118, 0xF>(v);
    v += moved<0x142, 0xA>(v);           // the last lane of a row to the next one
    v += moved<0x143, 0xC>(v);           // lane 31 to the upper half
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}
// The same over 16 or 32 neighbouring lanes, for each of them: with the other pair's, the other four's, the other eight's.
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
    static_assert(LANES == 16 || LANES == 32, "");
    v += moved<0xB1, 0xF>(v);            // lane ^ 1
    v += moved<0x4E, 0xF>(v);            // lane ^ 2
    v += moved<0x141, 0xF>(v);           // eight lanes the other way round
    v += moved<0x140, 0xF>(v);           // sixteen
    if constexpr (LANES == 32) v += __shfl_xor(v, 16);
    return v;
}
// The sums of N numbers over a row's threads, for all of them: some lanes of a wave, a wave, or a whole workgroup; there calls take the two halves of `places` in
// turn, so that one meeting is enough.
template <int THREADS> struct Meeting {
    static constexpr int WAVES = THREADS < 64 ? 1 : THREADS / 64;
    float (*places)[2][WAVES];           // [half][number][wave]
    int half = 0;
    template <int N> __device__ __forceinline__ void sums(float (&v)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if constexpr (THREADS < 64) v[i] = lanes_sum<THREADS>(v[i]);
            else v[i] = wave_sum(v[i]);
        }
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) places[half][i][threadIdx.x >> 6] = v[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                // a lane has a wave's
                float all = places[half][i][threadIdx.x & (WAVES - 1)];
                all += moved<0x111, 0xF>(all);
                if constexpr (WAVES > 2) all += moved<0x112, 0xF>(all);
                if constexpr (WAVES > 4) all += moved<0x114, 0xF>(all);
                if constexpr (WAVES > 8) all += moved<0x118, 0xF>(all);
                v[i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, all), WAVES - 1));
            }
            half ^= 1;
        }
    }
};
__device__ __forceinline__ v8f32 multiply_add(v8f32 a, v8f32 b, v8f32 c) { return __builtin_elementwise_fma(a, b, c); }
__device__ __forceinline__ float dot(v8f32 a, v8f32 b, float s) {
#pragma unroll
    for (int q = 0; q < 8; ++q) s = __builtin_fmaf(a[q], b[q], s);
    return s;
}

// rho of a row x and (ALONG) mean(d n) with n = x * rho; x(p), d(p): piece p
struct RowNorm { float rho, along; };
template <bool ALONG, int PIECES, int THREADS, typename X, typename F>
__device__ __forceinline__ RowNorm row_norm(X x, F d, float k, float eps, Meeting<THREADS>& meeting) {
    float s[ALONG ? 2 : 1] = {};
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        const v8f32 xp = x(p);
        s[0] = dot(xp, xp, s[0]);
        if constexpr (ALONG) s[1] = dot(d(p), xp, s[1]);
    }
    meeting.sums(s);
    RowNorm r = {__builtin_amdgcn_rsqf(s[0] / k + eps), 0.0f};
    const bool above = !(s[0] < 0x1p126f), below = s[0] < 0x1p-90f && eps < 0x1p-80f;
    bool again = above || below;
    if constexpr (ALONG) {
        r.along = s[1] * r.rho / k;
        again = again || !(fabsf(r.along) < __builtin_inff());
    }
    if (again) {                                     // (the same for all of a row's threads)
        // times 2^-72 no row's squares are too large, times 2^100 no row's that came to so little too small
        const float f = above ? 0x1p-72f : below ? 0x1p100f : 1.0f;
        float q[1] = {0.0f};
#pragma unroll
        for (int p = 0; p < PIECES; ++p) q[0] = dot(x(p) * f, x(p) * f, q[0]);
        meeting.sums(q);
        r.rho = f * __builtin_amdgcn_rsqf(q[0] / k + eps * f * f);
        if constexpr (ALONG) {
            // (divided before it is summed: the mean may be a number where the sum is none)
            q[0] = 0.0f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) q[0] = dot(d(p), x(p) * r.rho / k, q[0]);
            meeting.sums(q);
            r.along = q[0];
        }
    }
    return r;
}

// A thread's columns, and their weights: w_pre, and what of w_post, gate and scale goes with x.
template <int ROW, int PIECES> struct Columns {
    unsigned c[PIECES];
    int there[PIECES];
    __device__ __forceinline__ explicit Columns(const BlockNormArgs& a) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            c[p] = (p * ROW + threadIdx.x % ROW) * 8;
            there[p] = (int)a.k - (int)c[p];
        }
    }
    __device__ __forceinline__ v8f32 pre(const BlockNormArgs& a, int p) const { return load_weights(place(a.w_pre, c[p]), there[p]); }
    // scale * gate * w_post for the rows of a gate
    __device__ __forceinline__ v8f32 behind(const BlockNormArgs& a, int64_t gate, int p) const {
        v8f32 f = v8f32{} + a.scale;
        if (a.gate != nullptr) f *= load_weights(place(a.gate + gate * a.k, c[p]), there[p]);
        if (a.w_post != nullptr) f *= load_weights(place(a.w_post, c[p]), there[p]);
        return f;
    }
};

// A row has ROW threads of eight elements, twice eight for the longest.  Rows of a wave or less lie side by side in workgroups of 256: one to a workgroup, most
// lanes of short ones would have nothing to do, and the chains of reads and sums would follow one another.
constexpr int workgroup_threads(int row) { return row > 64 ? row : 256; }
// which of a workgroup's rows a thread has (the same for a whole wave where that has one)
template <int ROW> __device__ __forceinline__ int beside() {
    return ROW > 64 ? 0 : ROW == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : threadIdx.x / ROW;
}

template <int TYPE, int TYPE_R, int ROW, int PIECES>
__global__ void __launch_bounds__(workgroup_threads(ROW)) block_norm_kernel(const BlockNormArgs a) {
    typedef typename Element<TYPE>::type T;
    typedef typename Element<TYPE_R>::type TR;
    constexpr int AT_ONCE = workgroup_threads(ROW) / ROW;
    __shared__ float places[2][2][ROW > 64 ? ROW / 64 : 1];
    Meeting<ROW> meeting{places};
    constexpr bool AHEAD = ROW < 1024;               // the next row is asked for in front of this one's sums; the longest rows leave no registers for it
    const auto none = [](int) { return v8f32{}; };
    const T* const X = static_cast<const T*>(a.X);
    const TR* const R = static_cast<const TR*>(a.R);
    TR* const R_out = static_cast<TR*>(a.R_out);
    T* const H = static_cast<T*>(a.H);
    const Columns<ROW, PIECES> at(a);
    // weights stay in registers from row to row; those of the longest rows are read again for each
    constexpr bool KEPT = PIECES == 1;
    v8f32 pre = KEPT && H != nullptr ? at.pre(a, 0) : v8f32{}, behind = {};
    int64_t gate = -1;
    Raw<T> next_x[PIECES];
    Raw<TR> next_r[PIECES];
    const auto load = [&](int64_t row) {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            if (X != nullptr) next_x[p] = load_raw(X + row * a.ldx, at.c[p], at.there[p]);
            if (R != nullptr) next_r[p] = load_raw(R + row * a.ldr, at.c[p], at.there[p]);
        }
    };
    int64_t row = (int64_t)blockIdx.x * AT_ONCE + beside<ROW>();
    const int64_t step = (int64_t)gridDim.x * AT_ONCE;
    if (AHEAD && row < a.rows) load(row);
    for (; row < a.rows; row += step) {
        v8f32 x[PIECES], r[PIECES];
        if (!AHEAD) load(row);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            x[p] = X != nullptr ? numbers<T>(next_x[p], at.there[p]) : v8f32{};
            r[p] = R != nullptr ? numbers<TR>(next_r[p], at.there[p]) : v8f32{};
        }
        if (AHEAD && row + step < a.rows) load(row + step);
        if (X != nullptr) {
            const int64_t g = a.gate != nullptr ? (uint32_t)row / (uint32_t)a.group : 0;
            if (KEPT && g != gate) behind = at.behind(a, gate = g, 0);
            const float rho = a.w_post != nullptr ? row_norm<false, PIECES>([&](int p) { return x[p]; }, none, (float)a.k, a.eps, meeting).rho : 1.0f;
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                r[p] = multiply_add(x[p] * rho, KEPT ? behind : at.behind(a, g, p), r[p]);
                if (R_out != nullptr) store_eight(place(R_out + row * a.ldro, at.c[p]), r[p], at.there[p]);
            }
        }
        if (H == nullptr) continue;
        const float rho = row_norm<false, PIECES>([&](int p) { return r[p]; }, none, (float)a.k, a.eps, meeting).rho;
#pragma unroll
        for (int p = 0; p < PIECES; ++p) store_eight(place(H + row * a.ldh, at.c[p]), r[p] * rho * (KEPT ? pre : at.pre(a, p)), at.there[p]);
    }
}

// ---- gradient ----------------------------------------------------------------------------------------------------
// A workgroup has a chunk of neighbouring rows.  Where a gate's rows are more than a chunk, a chunk lies inside them and leaves its s for the join.  Where they are
// fewer, a chunk is some gates' rows: the workgroup writes their gradients itself and leaves the sum of gate s (16384 x 2048 with a gate for each row 187 us, 371 where
// every s went through memory).
struct NormChunks {
    int64_t group, groups;   // rows of a gate (or all, without one), and how many gates
    int64_t rows;            // of a chunk; where gates end inside: of what one of the rows side by side has, whole gates
    int64_t per_group;       // chunks in a group, 0: groups in a chunk
    int64_t chunks;
};
struct NormGradWork {
    BlockNormArgs a;
    NormChunks n;
    float* t;                // [chunk][k]: sums of dh n; null: not wanted
    float* s;                // [chunk][k]: sums of s, of gate s where gates end inside a chunk; null: not wanted
};

template <int TYPE, int TYPE_R, int ROW, int PIECES>
__global__ void __launch_bounds__(workgroup_threads(ROW)) block_norm_grad_kernel(const NormGradWork w) {
    typedef typename Element<TYPE>::type T;
    typedef typename Element<TYPE_R>::type TR;
    constexpr int THREADS = workgroup_threads(ROW), AT_ONCE = THREADS / ROW;
    __shared__ float places[2][2][ROW > 64 ? ROW / 64 : 1];
    Meeting<ROW> meeting{places};
    // What goes with columns lies in LDS, each thread's in places of its own: the sums over rows, t and s, and the weights (those of the longest rows are read again
    // for each).  In registers they would leave room for half as many waves.  Where gates end inside the chunk, BEHIND's place has the sum of gate s, the longest
    // rows' is in work memory.
    enum { SUM_T, SUM_S, PRE, BEHIND };
    constexpr bool LONG = PIECES > 1 || (TYPE == TYPE_F32 && ROW == 1024), AHEAD = ROW < 1024;
    __shared__ v4f32 held[LONG ? 2 : 4][2 * PIECES][THREADS];
    const auto get = [&](int which, int p) { return __builtin_shufflevector(held[which][2 * p][threadIdx.x], held[which][2 * p + 1][threadIdx.x], 0, 1, 2, 3, 4, 5, 6, 7); };
    const auto put = [&](int which, int p, v8f32 v) {
        held[which][2 * p][threadIdx.x] = __builtin_shufflevector(v, v, 0, 1, 2, 3);
        held[which][2 * p + 1][threadIdx.x] = __builtin_shufflevector(v, v, 4, 5, 6, 7);
    };
    const auto add = [&](int which, int p, v8f32 a, v8f32 b) { put(which, p, multiply_add(a, b, get(which, p))); };
    const BlockNormArgs& a = w.a;
    const T* const X = static_cast<const T*>(a.X);
    const T* const dH = static_cast<const T*>(a.dH);
    const TR* const R = static_cast<const TR*>(a.R);
    const TR* const dR_out = static_cast<const TR*>(a.dR_out);
    T* const dX = static_cast<T*>(a.dX);
    TR* const dR = static_cast<TR*>(a.dR);
    const NormChunks& n = w.n;
    const bool post = a.w_post != nullptr, branch = X != nullptr && (dX != nullptr || w.s != nullptr), inside = n.per_group == 0;
    const Columns<ROW, PIECES> at(a);
    // gate: the one of the next row; left: rows to its end
    int64_t row, end, gate, left = n.group;
    const int64_t step = inside ? 1 : AT_ONCE;
    if (inside) {
        row = ((int64_t)blockIdx.x * AT_ONCE + beside<ROW>()) * n.rows;
        end = row + n.rows < a.rows ? row + n.rows : a.rows;
        gate = (uint32_t)row / (uint32_t)n.group;
    } else {
        gate = (uint32_t)blockIdx.x / (uint32_t)n.per_group;
        const int64_t last = (gate + 1) * n.group < a.rows ? (gate + 1) * n.group : a.rows;
        row = gate * n.group + (blockIdx.x - gate * n.per_group) * n.rows;
        end = row + n.rows < last ? row + n.rows : last;
        row += beside<ROW>();
    }
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
        put(SUM_T, p, v8f32{});
        put(SUM_S, p, v8f32{});
    }
    if (!LONG && dH != nullptr) put(PRE, 0, at.pre(a, 0));
    if (!LONG) put(BEHIND, 0, inside || !branch ? v8f32{} : at.behind(a, gate, 0));
    bool first = true;
    // a gate's rows are done: its gradient, and gate s
    const auto finish = [&]() {
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            const v8f32 s = get(SUM_S, p);
            put(SUM_S, p, v8f32{});
            if (a.dgate != nullptr) {
                v8f32 d = s * a.scale;
                if (post) d *= load_weights(place(a.w_post, at.c[p]), at.there[p]);
                store_eight(place(a.dgate + gate * a.k, at.c[p]), d, at.there[p]);
            }
            if (a.dw_post != nullptr) {
                const v8f32 f = load_weights(place(a.gate + gate * a.k, at.c[p]), at.there[p]);
                if constexpr (LONG) {
                    float* const to = place(w.s + blockIdx.x * a.k, at.c[p]);
                    store_eight(to, first ? f * s : multiply_add(f, s, load_weights(to, at.there[p])), at.there[p]);
                } else add(BEHIND, p, f, s);
            }
        }
        first = false;
    };
    // A row's pieces: in registers, the next row's on their way; of the longest rows read again whenever they are needed, which the caches serve.
    Raw<T> next_x, next_dh;
    Raw<TR> next_r, next_dr;
    const auto load = [&](int64_t i) {
        if (dH != nullptr) {
            next_r = load_raw(R + i * a.ldr, at.c[0], at.there[0]);
            next_dh = load_raw(dH + i * a.lddh, at.c[0], at.there[0]);
        }
        if (dR_out != nullptr) next_dr = load_raw(dR_out + i * a.lddro, at.c[0], at.there[0]);
        if (branch) next_x = load_raw(X + i * a.ldx, at.c[0], at.there[0]);
    };
    if (AHEAD && row < end) load(row);
    for (; row < end; row += step) {
        v8f32 x0, r0, dh0, dr[PIECES];
        asm volatile("" ::: "memory");               // (nothing of LDS is kept in registers from row to row)
        if constexpr (!LONG) {
            if (!AHEAD) load(row);
            dr[0] = dR_out != nullptr ? numbers<TR>(next_dr, at.there[0]) : v8f32{};
            if (dH != nullptr) {
                r0 = numbers<TR>(next_r, at.there[0]);
                dh0 = numbers<T>(next_dh, at.there[0]);
            }
            if (branch) x0 = numbers<T>(next_x, at.there[0]);
            if (AHEAD && row + step < end) load(row + step);
        }
        const auto x = [&](int p) { return LONG ? numbers<T>(load_raw(X + row * a.ldx, at.c[p], at.there[p]), at.there[p]) : x0; };
        const auto r = [&](int p) { return LONG ? numbers<TR>(load_raw(R + row * a.ldr, at.c[p], at.there[p]), at.there[p]) : r0; };
        const auto dh = [&](int p) { return LONG ? numbers<T>(load_raw(dH + row * a.lddh, at.c[p], at.there[p]), at.there[p]) : dh0; };
        const auto dn = [&](int p) { return dh(p) * (LONG ? at.pre(a, p) : get(PRE, p)); };
        RowNorm rn = {0.0f, 0.0f};
        if (dH != nullptr) rn = row_norm<true, PIECES>(r, dn, (float)a.k, a.eps, meeting);
#pragma unroll
        for (int p = 0; p < PIECES; ++p) {
            if (LONG) dr[p] = dR_out != nullptr ? numbers<TR>(load_raw(dR_out + row * a.lddro, at.c[p], at.there[p]), at.there[p]) : v8f32{};
            if (dH != nullptr) {
                const v8f32 m = r(p) * rn.rho;
                dr[p] = multiply_add(multiply_add(-m, v8f32{} + rn.along, dn(p)), v8f32{} + rn.rho, dr[p]);
                add(SUM_T, p, dh(p), m);
            }
            if (dR != nullptr) store_eight(place(dR + row * a.lddr, at.c[p]), dr[p], at.there[p]);
        }
        if (branch) {
            v8f32 behind;
            if (!LONG) behind = inside ? at.behind(a, gate, 0) : get(BEHIND, 0);
            const auto dm = [&](int p) { return dr[p] * (LONG ? at.behind(a, gate, p) : behind); };       // the gradient of m, or of x where that has no norm
            RowNorm xn = {1.0f, 0.0f};
            if (post) xn = row_norm<true, PIECES>(x, dm, (float)a.k, a.eps, meeting);
#pragma unroll
            for (int p = 0; p < PIECES; ++p) {
                const v8f32 m = x(p) * xn.rho;
                add(SUM_S, p, dr[p], m);
                if (dX != nullptr) store_eight(place(dX + row * a.lddx, at.c[p]), post ? multiply_add(-m, v8f32{} + xn.along, dm(p)) * xn.rho : dm(p), at.there[p]);
            }
        }
        if (inside && (--left == 0 || row + 1 == end)) {
            if (w.s != nullptr) finish();
            ++gate;
            left = n.group;
        }
    }
    // the chunk's sums: of what lies side by side together, in its order
    const auto leave = [&](float* to, int which) {
        if constexpr (AT_ONCE == 1) {
#pragma unroll
            for (int p = 0; p < PIECES; ++p) store_eight(place(to, at.c[p]), get(which, p), at.there[p]);
        } else if (threadIdx.x < 2 * ROW) {
            const int half = threadIdx.x / ROW, lane = threadIdx.x % ROW, c = lane * 8 + half * 4;
            v4f32 sum = held[which][half][lane];
#pragma unroll
            for (int j = 1; j < AT_ONCE; ++j) sum += held[which][half][lane + j * ROW];
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (c + q < a.k) to[c + q] = sum[q];
        }
    };
    if (AT_ONCE > 1) __syncthreads();
    if (w.t != nullptr) leave(w.t + blockIdx.x * a.k, SUM_T);
    if (w.s != nullptr && !inside) leave(w.s + blockIdx.x * a.k, SUM_S);
    if (!LONG && a.dw_post != nullptr && inside) leave(w.s + blockIdx.x * a.k, BEHIND);
}

// Sums over chunks: 32 columns a workgroup, in 32 shares.  blockIdx.y: 0 dw_pre, 1 dw_post, from 2 on the gradients of gates, of as many as there are shares for
// (a gate of few chunks has few shares); a single gate's comes from the same sum as dw_post.
constexpr int JOIN_COLUMNS = 32, JOIN_SHARES = 32;
__host__ __device__ __forceinline__ int gate_shares(const NormChunks& n) {
    int shares = 1;
    while (shares < JOIN_SHARES && shares < n.per_group) shares *= 2;
    return shares;
}
__global__ void __launch_bounds__(JOIN_COLUMNS * JOIN_SHARES) block_norm_join_kernel(const NormGradWork w) {
    __shared__ float shares[JOIN_SHARES][JOIN_COLUMNS + 1];
    const BlockNormArgs& a = w.a;
    const NormChunks& n = w.n;
    const int in = threadIdx.x % JOIN_COLUMNS, share = threadIdx.x / JOIN_COLUMNS;
    const int64_t c = (int64_t)blockIdx.x * JOIN_COLUMNS + in;
    const int what = blockIdx.y, each = what < 2 ? JOIN_SHARES : gate_shares(n), first = (what - 2) * (JOIN_SHARES / each);     // first: of the gates
    const bool single = a.gate != nullptr && n.groups == 1;
    if (what == 0 ? a.dw_pre == nullptr : what == 1 ? a.dw_post == nullptr && !(single && a.dgate != nullptr) : false) return;
    float sum = 0.0f;
    if (c < a.k) {
        if (what == 0) {
#pragma unroll 8
            for (int64_t i = share; i < n.chunks; i += JOIN_SHARES) sum += w.t[i * a.k + c];
        } else if (what == 1) {
            if (a.gate != nullptr && !single && n.per_group > 0) {
#pragma unroll 8
                for (int64_t i = share; i < n.chunks; i += JOIN_SHARES) sum += w.s[i * a.k + c] * a.gate[(uint32_t)i / (uint32_t)n.per_group * a.k + c];
            } else {
#pragma unroll 8
                for (int64_t i = share; i < n.chunks; i += JOIN_SHARES) sum += w.s[i * a.k + c];
            }
        } else if (first + share / each < n.groups) {
            const float* const from = w.s + (first + share / each) * n.per_group * a.k + c;
#pragma unroll 8
            for (int64_t i = share % each; i < n.per_group; i += each) sum += from[i * a.k];
        }
    }
    shares[share][in] = sum;
    __syncthreads();
    // share i of the 32 takes column i: a wave has two columns' 32 sums
    const int column = threadIdx.x / JOIN_SHARES, from = threadIdx.x % JOIN_SHARES;
    sum = shares[from][column];
    for (int d = 1; d < each; d <<= 1) sum += __shfl_xor(sum, d);
    const int64_t to = (int64_t)blockIdx.x * JOIN_COLUMNS + column;
    if (from % each != 0 || to >= a.k) return;
    if (what == 0) a.dw_pre[to] = sum;
    else if (what == 1) {
        if (a.dw_post != nullptr) a.dw_post[to] = sum * (single ? a.gate[to] * a.scale : a.scale);
        if (single && a.dgate != nullptr) a.dgate[to] = sum * a.scale * (a.w_post != nullptr ? a.w_post[to] : 1.0f);
    } else if (first + from / each < n.groups) a.dgate[(first + from / each) * a.k + to] = sum * a.scale * (a.w_post != nullptr ? a.w_post[to] : 1.0f);
}

// ---- launches ----------------------------------------------------------------------------------------------------
// threads and pieces of eight elements a thread that hold a row
struct RowShape { int threads, pieces; };
RowShape row_shape(int64_t k) {
    int threads = 16;
    while (threads < 1024 && threads * 8 < k) threads *= 2;
    return RowShape{threads, threads * 8 < k ? 2 : 1};
}
NormChunks norm_chunks(int64_t rows, int64_t k, int64_t group) {
    const int threads = row_shape(k).threads, at_once = workgroup_threads(threads) / threads;
    // as many as run at a time, of short rows fewer, whose join counts: 8192 x 4096 in 512 chunks 95 us, in 256 111, in 768 102;  16384 x 1024 in 1024 70, in 2048 71;
    // 16384 x 255 in 512 21, in 256 23, in 1024 25;  16384 x 32 in 512 11.6, in 256 13.2, in 1024 13.6
    const int64_t most = threads <= 64 ? 512 : threads == 128 ? 1024 : 262144 / threads;
    NormChunks n;
    n.group = group > 0 && group < rows ? group : rows;
    n.groups = div_up(rows, n.group);
    n.rows = div_up(div_up(rows, most), at_once) * at_once;
    // gates of fewer rows whose rows fill a workgroup are a chunk each, if they are not too many: one after another they would take longer than more chunks to join
    // (16384 x 128 with a gate for 16 rows 21 us, inside chunks 34)
    if (at_once > 1 && n.group < n.rows && n.group >= at_once && n.groups <= 4 * most) n.rows = n.group;
    if (n.group >= n.rows || n.groups == 1) {
        n.per_group = div_up(n.group, n.rows);
        n.chunks = n.groups * n.per_group;
    } else {
        const int64_t each = n.rows / at_once / n.group;
        n.rows = (each > 1 ? each : 1) * n.group;
        n.per_group = 0;
        n.chunks = div_up(rows, n.rows * at_once);
    }
    return n;
}
size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

template <typename F> hipError_t with_shape(int64_t k, F f) {
    const RowShape s = row_shape(k);
    const std::integral_constant<int, 1> one;
    switch (s.threads) {
        case 16: return f(std::integral_constant<int, 16>(), one);
        case 32: return f(std::integral_constant<int, 32>(), one);
        case 64: return f(std::integral_constant<int, 64>(), one);
        case 128: return f(std::integral_constant<int, 128>(), one);
        case 256: return f(std::integral_constant<int, 256>(), one);
        case 512: return f(std::integral_constant<int, 512>(), one);
        default: return s.pieces == 1 ? f(std::integral_constant<int, 1024>(), one) : f(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
    }
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
    return 2 * up((size_t)n.chunks * k * 4);
}

hipError_t launch_block_norm(const BlockNormArgs& args, int type, int type_r, hipStream_t st) {
    BlockNormArgs a = args;
    if (a.group > a.rows) a.group = a.rows;          // (rows are divided by it in 32 bits)
    return with_types(type, type_r, [&](auto t, auto tr) {
        return with_shape(a.k, [&](auto threads, auto pieces) {
            constexpr int T = decltype(t)::value, TR = decltype(tr)::value, ROW = decltype(threads)::value, PIECES = decltype(pieces)::value, THREADS = workgroup_threads(ROW);
            const int64_t most = 256 * (2048 / THREADS), wanted = div_up(a.rows, THREADS / ROW);
            hipLaunchKernelGGL((block_norm_kernel<T, TR, ROW, PIECES>), dim3((unsigned)(wanted < most ? wanted : most)), dim3(THREADS), 0, st, a);
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
            constexpr int T = decltype(ty)::value, TR = decltype(tr)::value, ROW = decltype(threads)::value, PIECES = decltype(pieces)::value;
            hipLaunchKernelGGL((block_norm_grad_kernel<T, TR, ROW, PIECES>), dim3((unsigned)w.n.chunks), dim3(workgroup_threads(ROW)), 0, st, w);
            return hipGetLastError();
        });
    });
    if (e != hipSuccess || (w.t == nullptr && w.s == nullptr)) return e;
    const bool gates = a.dgate != nullptr && w.n.per_group > 0;
    if (a.dw_pre == nullptr && a.dw_post == nullptr && !gates) return hipSuccess;
    const int64_t ys = gates && w.n.groups > 1 ? div_up(w.n.groups, JOIN_SHARES / gate_shares(w.n)) : 0;
    hipLaunchKernelGGL(block_norm_join_kernel, dim3((unsigned)div_up(a.k, JOIN_COLUMNS), (unsigned)(2 + ys)), dim3(JOIN_COLUMNS * JOIN_SHARES), 0, st, w);
    return hipGetLastError();
}

}  // namespace ozaki
