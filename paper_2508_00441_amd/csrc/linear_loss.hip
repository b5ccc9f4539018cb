// Softmax cross entropy of a linear layer's outputs over a vocabulary, and its gradient, without keeping the outputs:
//     z[t][v] = H[t] . W[v],   lse[t] = log sum_v exp(z[t][v]),   loss[t] = lse[t] - z[t][target[t]]
//     g[t][v] = (exp(z[t][v] - lse[t]) - [v == target[t]]) * dloss[t],   dH = g W,   dW = g^T H.
//
// Forward: a workgroup forms a tile of z in registers and leaves each token's largest value and sum of exponentials over the tile's
// words, 8 bytes per token and tile; a second launch joins them and takes the target's z, which the lane that held it has written.
// Gradient: the vocabulary is taken in pieces.  A piece's z are formed again and become g in the 16-bit type of H and W (its rounding is of the
// size of the result's own), stored as [token][word]; the two products read it from there.  All products are sums over 16-bit elements in
// FP32 on the matrix unit (tile_product.hpp).  W in dH, and g and H in dW, lie across the inner dimension; they are turned on the way from LDS
// to registers (with copies turned in memory the gradient of 4096 x 65536 x 4096 took 5.3 ms, of 16 x 65536 x 2048 0.44 ms).
//
// What is held of g is (exp(z - lse) - [v == target]) * 2^12, without dloss.  Its largest entries, the targets', are then near a power of two
// and lose nothing to 16 bits; times dloss they all lose alike, which does not average out (1.7 times the error of the result's own
// rounding in FP16).  2^12 keeps the words down to a probability of 2^-26 among FP16's normal numbers.  dloss comes in where it costs no
// rounding: as a factor of the rows of dH, and for dW with a copy of H times dloss over the largest |dloss|, which is one for a mean.
// Where the shares differ, that copy is rounded to 16 bits once more (on normally distributed numbers dW's error grows from 1.8e-3 of its norm
// to 2.5e-3 in BF16, from 2.5e-4 to 3.3e-4 in FP16; the result's own rounding is 1.7e-3 and 2.1e-4).  In FP16, whose smallest normal number is 2^-14, H times a share below 2^-10 would
// run out of bits; there g takes up to 2^8 of the share, a power of two that costs it nothing but the words below a probability of 2^-18 of
// that token, whose error stays below 2^-29 (share_exponent).  So shares down to 2^-19 are as good as others.
// Only the tokens that count take part (tokens_body).
//
// Few tokens are bound by the read of W (16 x 65536 x 2048: 52 us and 5 for the join, 5.1 TB/s; the gradient reads it twice, 166 us), many by the matrix
// unit (4096 x 131072 x 4096: 3.07 ms, 1.43 PFLOP/s; gradient of 4096 x 65536 x 4096: 4.83 ms, 1.36 PFLOP/s).
#include "layout.hpp"
#include "tile_product.hpp"

namespace ozaki {
namespace {

constexpr float LOG2_E = 1.44269504088896340736f, LN_2 = 0.69314718055994530942f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * LOG2_E); }
__device__ __forceinline__ float log_of(float x) { return __builtin_amdgcn_logf(x) * LN_2; }
// What exponentials are taken relative to: the largest number.  Where that is infinite, zero: nothing but minus infinity gives a sum of zero,
// and plus infinity, less itself, would give NaN instead of an infinite sum.
__device__ __forceinline__ float base_of(float most) { return fabsf(most) == __builtin_inff() ? 0.0f : most; }

// per token, what a tile of z needs
struct TokenState {
    const float* lse;
    const int* target;
    const float* held;       // what its g is held times
};
// What g is held times, HELD / 2^a, where H is held times dloss / (the largest) * 2^a.
constexpr float HELD = 4096.0f;
template <typename T>
__device__ __forceinline__ int share_exponent(float share) {
    if constexpr (!std::is_same_v<T, _Float16>) return 0;
    const int a = 117 - ((__float_as_int(share) >> 23) & 0xFF);       // how far below 2^-10
    return a < 0 ? 0 : a < 8 ? a : 8;
}

struct LogitWork {
    const uint8_t* H;
    const uint8_t* W;        // of the piece
    int64_t ldh, ldw, bytes; // in bytes
    int64_t tokens, words, first_word;    // words: of the piece
    const int* count;        // not null: how many tokens there really are
    int tiles_m, tiles_n, steps;
    WorkOrder order;
    // forward
    const int64_t* targets;
    float2* part;            // [tile of words][token]
    float* target_z;
    // gradient
    TokenState token;
    uint8_t* G;              // [token][ldg]; zeros behind the piece's words, up to a whole tile
    int64_t ldg;             // elements
};

// the tile of z that this workgroup has; false where it has none
template <typename P>
__device__ __forceinline__ bool logits(const LogitWork& w, uint8_t* lds, int64_t tokens, int64_t& m0, int64_t& n0, v4f32 (&acc)[P::FN][P::FM]) {
    const unsigned tiles_m = (unsigned)div_up(tokens, P::TM), total = tiles_m * (unsigned)w.tiles_n;
    if (blockIdx.x >= total) return false;
    const WorkItem item = work_item(blockIdx.x, total, w.order, tiles_m, w.tiles_n);
    m0 = (int64_t)item.bm * P::TM;
    n0 = (int64_t)item.bn * P::TN;
    const int64_t left_m = tokens - m0, left_n = w.words - n0;
    const TileOperand X{w.W + n0 * w.ldw, w.ldw, (int)(left_n < P::TN ? left_n : P::TN), nullptr, 0};
    const TileOperand Y{w.H + m0 * w.ldh, w.ldh, (int)(left_m < P::TM ? left_m : P::TM), nullptr, 0};
    P::multiply(lds, X, Y, w.bytes, 0, w.steps, acc);
    return true;
}

template <typename P>
__device__ __forceinline__ void loss_forward_body(const LogitWork& w) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[P::LDS_BYTES];
    int64_t m0, n0;
    v4f32 acc[P::FN][P::FM] = {};
    if (!logits<P>(w, lds, w.tokens, m0, n0, acc)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wn = wave / P::WM, wm = wave % P::WM, g = lane >> 4;
    float2* const joined = reinterpret_cast<float2*>(lds);            // [wn][token]
    const int first = wn * P::FN * 16 + 4 * g;                        // this lane's first word in the tile
    const int words = (int)(w.words - n0 < P::TN ? w.words - n0 : P::TN);
#pragma unroll
    for (int j = 0; j < P::FM; ++j) {
        const int t = (wm * P::FM + j) * 16 + (lane & 15);
        const int64_t target = m0 + t < w.tokens ? w.targets[m0 + t] - w.first_word - n0 : -1;
        float most = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < P::FN; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int v = first + 16 * i + r;
                if (v >= words) acc[i][j][r] = -__builtin_inff();
                most = fmaxf(most, acc[i][j][r]);
                if (v < words && v == target) w.target_z[m0 + t] = acc[i][j][r];
            }
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float base = base_of(most);
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < P::FN; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) sum += exp_of(acc[i][j][r] - base);
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (g == 0) joined[wn * P::TM + t] = make_float2(most, sum);
    }
    __syncthreads();
    for (int t = threadIdx.x; t < P::TM; t += P::THREADS) {
        if (m0 + t >= w.tokens) break;
        float most = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int i = 0; i < P::WN; ++i) most = fmaxf(most, joined[i * P::TM + t].x);
        const float base = base_of(most);
#pragma unroll
        for (int i = 0; i < P::WN; ++i) sum += joined[i * P::TM + t].y * exp_of(joined[i * P::TM + t].x - base);
        w.part[(n0 / P::TN) * w.tokens + m0 + t] = make_float2(most, sum);
    }
}

// TOKENS tokens a workgroup, 256 / TOKENS shares of the tiles of words for each.
template <int TOKENS>
__global__ void __launch_bounds__(256) loss_join_kernel(const float2* part, const float* target_z, const int64_t* targets, int64_t tokens,
                                                        int64_t vocab, int64_t ignore, int tiles, float* loss, float* lse, int* flags) {
    constexpr int SHARES = 256 / TOKENS, AT_ONCE = 4;
    __shared__ float2 share[4][TOKENS];
    const int tl = threadIdx.x % TOKENS, s = threadIdx.x / TOKENS;
    const int64_t t = (int64_t)blockIdx.x * TOKENS + tl, at = t < tokens ? t : tokens - 1;
    float most = -__builtin_inff(), sum = 0.0f;
    const auto add = [&](float m, float v) {
        const float higher = fmaxf(most, m), base = base_of(higher);
        sum = sum * exp_of(most - base) + v * exp_of(m - base);
        most = higher;
    };
    for (int i = s; i < tiles; i += SHARES * AT_ONCE) {
        float2 p[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) p[u] = i + u * SHARES < tiles ? part[(int64_t)(i + u * SHARES) * tokens + at] : make_float2(-__builtin_inff(), 0.0f);
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) add(p[u].x, p[u].y);
    }
    // the shares of a token lie TOKENS lanes apart in a wave, and in four waves
#pragma unroll
    for (int d = TOKENS; d < 64; d <<= 1) {
        const float m = __shfl_xor(most, d), v = __shfl_xor(sum, d);
        add(m, v);
    }
    if ((threadIdx.x & 63) < TOKENS) share[threadIdx.x >> 6][tl] = make_float2(most, sum);
    __syncthreads();
    if (threadIdx.x >= TOKENS || t >= tokens) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) add(share[w][tl].x, share[w][tl].y);
    const float l = base_of(most) + log_of(sum);
    const int64_t target = targets[t];
    const bool counts = target != ignore, real = target >= 0 && target < vocab;
    lse[t] = l;
    loss[t] = !counts ? 0.0f : real ? l - target_z[t] : __builtin_nanf("");
    if (counts && !real) atomicOr(flags, TARGET_FLAG);
}

// Gradient, in front of everything.  Tokens that do not count (often more than half: prompts, padding) cost the products nothing: those that do are
// copied together, in their order, H as it is and (for dW) times the token's share of the largest |dloss|; with them go their targets, lse and
// factors of dH's rows, and where in dH those lie.  How many there are only the card knows: the kernels behind this one are launched for all tokens,
// and workgroups without any end at once.  Rows of dH of the other tokens become zeros here.
// A workgroup has `each` neighbouring tokens; it finds the largest |dloss| and how many count in front of its own by itself (12 bytes a token; a
// launch of its own for that took 2.5 us, and 4.6 with 1003 tokens).
struct GradTokens {
    const int64_t* targets;
    const float* lse;
    const float* dloss;
    int64_t tokens, vocab, ignore, k, each;
    // of the tokens that count, in their order
    int* count;
    int* place;              // in dH
    int* target_out;
    float* lse_out;
    float* row_factor;
    float* held_out;
    float* dw_factor;        // one number
    int* flags;
};
constexpr int TOKEN_THREADS = 512;

template <typename T>
__device__ __forceinline__ void tokens_body(const GradTokens& w, const T* H, int64_t ldh, T* Hc, T* Hs, int64_t ld, T* dH, int64_t lddh) {
    typedef T eight __attribute__((ext_vector_type(8)));
    constexpr int WAVES = TOKEN_THREADS / 64;
    __shared__ float most_of[WAVES];
    __shared__ int before_of[WAVES], all_of[WAVES], at_of[TOKEN_THREADS];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int64_t first = (int64_t)blockIdx.x * w.each, end = first + w.each < w.tokens ? first + w.each : w.tokens;
    const auto counts = [&](int64_t target) { return target != w.ignore && target >= 0 && target < w.vocab; };
    float most = 0.0f;
    int before = 0, all = 0;
#pragma unroll 4
    for (int64_t t = tid; t < w.tokens; t += TOKEN_THREADS) {
        const bool c = counts(w.targets[t]);
        const float d = c ? fabsf(w.dloss[t]) : 0.0f;
        most = d < __builtin_inff() ? fmaxf(most, d) : most;
        all += c;
        before += c && t < first;
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        most = fmaxf(most, __shfl_xor(most, s));
        before += __shfl_xor(before, s);
        all += __shfl_xor(all, s);
    }
    if (lane == 0) {
        most_of[wave] = most;
        before_of[wave] = before;
        all_of[wave] = all;
    }
    __syncthreads();
    before = all = 0;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        most = fmaxf(most, most_of[i]);
        before += before_of[i];
        all += all_of[i];
    }
    if (most == 0.0f) most = 1.0f;
    if (blockIdx.x == 0 && tid == 0) {
        *w.count = all;
        *w.dw_factor = most * (1.0f / HELD);
    }
    const int64_t pieces = ld / 8;
    const bool wide = lddh % 8 == 0 && reinterpret_cast<uintptr_t>(dH) % 16 == 0;
    for (int64_t from = first; from < end; from += TOKEN_THREADS) {
        // the places of the next tokens, one a thread
        const int64_t t = from + tid;
        const bool c = t < end && counts(w.targets[t]);
        const unsigned long long in_wave = __ballot(c);
        __syncthreads();
        if (lane == 0) all_of[wave] = __popcll(in_wave);
        __syncthreads();
        int at = before + __popcll(in_wave & ((1ull << lane) - 1));
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            at += i < wave ? all_of[i] : 0;
            before += all_of[i];
        }
        at_of[tid] = c ? at : -1;
        if (c) {
            w.place[at] = (int)t;
            w.target_out[at] = (int)w.targets[t];
            w.lse_out[at] = w.lse[t];
            const float d = w.dloss[t];
            const int a = share_exponent<T>(d / most);
            w.row_factor[at] = ldexpf(d, a) * (1.0f / HELD);
            w.held_out[at] = ldexpf(HELD, -a);
        } else if (t < end && w.targets[t] != w.ignore) {
            atomicOr(w.flags, TARGET_FLAG);
        }
        __syncthreads();
        const int64_t here = end - from < TOKEN_THREADS ? end - from : TOKEN_THREADS;
        for (int64_t p = tid; p < here * pieces; p += TOKEN_THREADS) {
            const int64_t i = p / pieces, e = p % pieces * 8;
            const int to = at_of[i];
            if (to >= 0) {
                eight x = *reinterpret_cast<const eight*>(H + (from + i) * ldh + e);
                *reinterpret_cast<eight*>(Hc + to * ld + e) = x;
                if (Hs == nullptr) continue;
                const float share = w.dloss[from + i] / most, f = ldexpf(share, share_exponent<T>(share));
#pragma unroll
                for (int q = 0; q < 8; ++q) x[q] = (T)((float)x[q] * f);
                *reinterpret_cast<eight*>(Hs + to * ld + e) = x;
            } else if (dH != nullptr) {
                T* const row = dH + (from + i) * lddh + e;
                if (wide && e + 8 <= w.k) {
                    *reinterpret_cast<eight*>(row) = eight{};
                } else {
#pragma unroll
                    for (int q = 0; q < 8; ++q)
                        if (e + q < w.k) row[q] = (T)0.0f;
                }
            }
        }
    }
}

// A tile of g, through LDS so that it is written in rows of 16-byte pieces.
template <typename P, typename T>
__device__ __forceinline__ void loss_g_body(const LogitWork& w) {
    constexpr int STRIDE = P::TN * 2 + 16;            // bytes between tokens
    __shared__ __attribute__((aligned(16))) uint8_t lds[P::LDS_BYTES > P::TM * STRIDE ? P::LDS_BYTES : P::TM * STRIDE];
    int64_t m0, n0;
    v4f32 acc[P::FN][P::FM] = {};
    const int64_t tokens = *w.count;
    if (!logits<P>(w, lds, tokens, m0, n0, acc)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wn = wave / P::WM, wm = wave % P::WM, g = lane >> 4;
    const int first = wn * P::FN * 16 + 4 * g;
    const int words = (int)(w.words - n0 < P::TN ? w.words - n0 : P::TN);
    typedef T four __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int j = 0; j < P::FM; ++j) {
        const int t = (wm * P::FM + j) * 16 + (lane & 15);
        const bool real = m0 + t < tokens;
        const float lse = real ? w.token.lse[m0 + t] : 0.0f, held = real ? w.token.held[m0 + t] : 0.0f;
        const int at = real ? (int)(w.token.target[m0 + t] - w.first_word - n0) : -1;
#pragma unroll
        for (int i = 0; i < P::FN; ++i) {
            four v;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int word = first + 16 * i + r;
                const float p = exp_of(acc[i][j][r] - lse) - (word == at ? 1.0f : 0.0f);
                v[r] = (T)(word < words ? p * held : 0.0f);
            }
            *reinterpret_cast<four*>(lds + t * STRIDE + (first + 16 * i) * 2) = v;
        }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < P::TM * P::TN / 8; c += P::THREADS) {
        const int t = c / (P::TN / 8), p = c % (P::TN / 8);
        if (m0 + t >= tokens) break;
        *reinterpret_cast<v4i32*>(w.G + ((m0 + t) * w.ldg + n0 + p * 8) * 2) = *reinterpret_cast<const v4i32*>(lds + t * STRIDE + p * 16);
    }
}

// In how many shares the inner dimension of dH is cut: as many as the workgroups launched for all tokens' tiles make of the tiles that there are
// (`tiles` of `rows` rows, over all shares), but no more than `most`.
struct ProductRoom {
    int tiles, rows, most;
    __device__ __forceinline__ int splits(int64_t count) const {
        const int64_t there = div_up(count, rows), s = there > 0 ? tiles / there : 1;
        return (int)(s < most ? s : most);
    }
};

// D = X Y^T of 16-bit operands; rows of Y are D's rows
struct ProductWork {
    const uint8_t* X;
    const uint8_t* Y;
    int64_t ldx, ldy;        // in bytes
    int64_t elements;        // of the inner dimension: the words of dH; of dW the tokens
    int64_t m, n;            // rows of D (dH: for all tokens) and its columns
    const int* count;        // how many tokens there really are
    const int* place;        // dH: which row of D a token's is
    int tiles_n;
    ProductRoom room;
    WorkOrder order;
    void* D;
    int64_t ldd;
    const float* row_factor; // what the sums are multiplied by, of dH: one for every row,
    const float* factor;     // of dW: the same for all
    float* partial;          // not null: unscaled sums go there, [split][token that counts][n in fours]
};

template <typename P, typename T, bool DW>
__device__ __forceinline__ void loss_product_body(const ProductWork& w) {
    __shared__ __attribute__((aligned(16))) uint8_t lds[P::LDS_BYTES];
    const int64_t count = *w.count, m = DW ? w.m : count, elements = DW ? count : w.elements;
    const int steps = (int)div_up(elements * 2, STEP_BYTES), splits = DW ? 1 : w.room.splits(count);
    const unsigned tiles_m = (unsigned)div_up(m, P::TM), total = tiles_m * (unsigned)w.tiles_n * (unsigned)splits;
    if (blockIdx.x >= total) return;
    const WorkItem item = work_item(blockIdx.x, total, w.order, tiles_m, w.tiles_n);
    const int64_t m0 = (int64_t)item.bm * P::TM, n0 = (int64_t)item.bn * P::TN, left_m = m - m0, left_n = w.n - n0;
    const TileOperand X{w.X + n0 * 2, w.ldx, (int)(left_n < P::TN ? left_n : P::TN), nullptr, 0, elements};
    const TileOperand Y{w.Y + m0 * (DW ? 2 : w.ldy), w.ldy, (int)(left_m < P::TM ? left_m : P::TM), nullptr, 0, elements};
    v4f32 acc[P::FN][P::FM] = {};
    const int split = item.gi;
    if (steps > 0) P::multiply(lds, X, Y, elements * 2, split_begin(steps, splits, split), split_begin(steps, splits, split + 1), acc);
    if constexpr (DW) {
        const float all = *w.factor;
        store_tile<P, (P::THREADS > 256)>(lds, acc, static_cast<T*>(w.D) + m0 * w.ldd + n0, w.ldd, left_m, left_n, false, [&](int64_t) { return all; });
    } else if (w.partial != nullptr) {
        store_tile<P, false>(lds, acc, w.partial + ((int64_t)split * m + m0) * in_fours(w.n) + n0, in_fours(w.n), left_m, in_fours(left_n), false,
                             [](int64_t) { return 1.0f; });
    } else {
        store_tile<P, (P::THREADS > 256)>(lds, acc, static_cast<T*>(w.D) + n0, w.ldd, left_m, left_n, false, [&](int64_t r) { return w.row_factor[m0 + r]; },
                                          [&](int64_t r) { return (int64_t)w.place[m0 + r]; });
    }
}

// The sums of a piece's shares of the inner dimension, on top of the pieces' before it (`sum`, unless it is the first); the last piece's go to D.
// A workgroup a row.
template <typename T>
__device__ __forceinline__ void join_body(const float* partial, const ProductRoom& room, int64_t n, float* sum, bool first, bool last,
                                          const int* count, const int* place, const float* row_factor, T* D, int64_t ldd) {
    const int64_t ld = in_fours(n), rows = *count;
    const int splits = room.splits(rows);
    for (int64_t i = blockIdx.x; i < rows; i += gridDim.x)
        for (int64_t j = threadIdx.x * 4; j < n; j += 1024) {
            v4f32 s = {};
            if (!first) s = *reinterpret_cast<const v4f32*>(sum + i * ld + j);
#pragma unroll 4
            for (int p = 0; p < splits; ++p) s += *reinterpret_cast<const v4f32*>(partial + ((int64_t)p * rows + i) * ld + j);
            if (last) put_four(D + place[i] * ldd + j, s * row_factor[i], n - j, ldd % 4 == 0 && reinterpret_cast<uintptr_t>(D) % (4 * sizeof(T)) == 0, false);
            else *reinterpret_cast<v4f32*>(sum + i * ld + j) = s;
        }
}

__global__ void __launch_bounds__(256) zero_rows_kernel(uint16_t* D, int64_t rows, int64_t k, int64_t ldd) {
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < rows * k; at += (int64_t)gridDim.x * 256) D[at / k * ldd + at % k] = 0;
}

constexpr int kind_of(int type) { return type == TYPE_F16 ? KIND_F16 : KIND_BF16; }
template <int TYPE> using LargeTile = PairedTile<kind_of(TYPE)>;      // 256 words or columns, 256 tokens or rows
template <int TYPE> using MiddleTile = Tile<kind_of(TYPE), 2, 2, 4, 2, 3>;     // 128, 64
template <int TYPE> using SmallTile = Tile<kind_of(TYPE), 2, 2, 2, 2, 4>;      // 64, 64
// 64, 16: 16 tokens, 65536 words of 2048 in 57 us; 128 words a workgroup 62, straight from memory into registers 75 (there the tokens are read as
// often as the words).  One token, 131072 words of 4096: 190, 203, 180.
template <int TYPE> using FewTile = Tile<kind_of(TYPE), 4, 1, 1, 1, 4>;

template <int TYPE>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) loss_forward_large_kernel(const LogitWork w) { loss_forward_body<LargeTile<TYPE>>(w); }
template <int TYPE>
__global__ void __launch_bounds__(256) loss_forward_middle_kernel(const LogitWork w) { loss_forward_body<MiddleTile<TYPE>>(w); }
template <int TYPE>
__global__ void __launch_bounds__(256) loss_forward_small_kernel(const LogitWork w) { loss_forward_body<SmallTile<TYPE>>(w); }
template <int TYPE>
__global__ void __launch_bounds__(256) loss_forward_few_kernel(const LogitWork w) { loss_forward_body<FewTile<TYPE>>(w); }
template <int TYPE>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) loss_g_large_kernel(const LogitWork w) { loss_g_body<LargeTile<TYPE>, typename Element<TYPE>::type>(w); }
template <int TYPE>
__global__ void __launch_bounds__(256) loss_g_middle_kernel(const LogitWork w) { loss_g_body<MiddleTile<TYPE>, typename Element<TYPE>::type>(w); }
template <int TYPE>
__global__ void __launch_bounds__(256) loss_g_small_kernel(const LogitWork w) { loss_g_body<SmallTile<TYPE>, typename Element<TYPE>::type>(w); }
template <int TYPE>
__global__ void __launch_bounds__(256) loss_g_few_kernel(const LogitWork w) { loss_g_body<FewTile<TYPE>, typename Element<TYPE>::type>(w); }
// dH = g W, and dW = g^T H
template <int TYPE>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) loss_dh_large_kernel(const ProductWork w) {
    loss_product_body<PairedTile<kind_of(TYPE), true, false>, typename Element<TYPE>::type, false>(w);
}
template <int TYPE>
__global__ void __launch_bounds__(256) loss_dh_middle_kernel(const ProductWork w) {
    loss_product_body<Tile<kind_of(TYPE), 2, 2, 4, 2, 3, true, false>, typename Element<TYPE>::type, false>(w);
}
template <int TYPE>
__global__ void __launch_bounds__(256) loss_dh_few_kernel(const ProductWork w) {
    loss_product_body<Tile<kind_of(TYPE), 4, 1, 2, 1, 4, true, false>, typename Element<TYPE>::type, false>(w);
}
template <int TYPE>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) loss_dw_large_kernel(const ProductWork w) {
    loss_product_body<PairedTile<kind_of(TYPE), true, true>, typename Element<TYPE>::type, true>(w);
}
template <int TYPE>
__global__ void __launch_bounds__(256) loss_dw_middle_kernel(const ProductWork w) {
    loss_product_body<Tile<kind_of(TYPE), 2, 2, 4, 4, 2, true, true>, typename Element<TYPE>::type, true>(w);
}
template <int TYPE>
__global__ void __launch_bounds__(256) loss_product_join_kernel(const float* partial, const ProductRoom room, int64_t n, float* sum, bool first, bool last,
                                                                const int* count, const int* place, const float* row_factor, void* D, int64_t ldd) {
    join_body(partial, room, n, sum, first, last, count, place, row_factor, static_cast<typename Element<TYPE>::type*>(D), ldd);
}

template <int TYPE>
__global__ void __launch_bounds__(TOKEN_THREADS) loss_tokens_kernel(const GradTokens w, const void* H, int64_t ldh, void* Hc, void* Hs, int64_t ld, void* dH,
                                                                    int64_t lddh) {
    typedef typename Element<TYPE>::type T;
    tokens_body(w, static_cast<const T*>(H), ldh, static_cast<T*>(Hc), static_cast<T*>(Hs), ld, static_cast<T*>(dH), lddh);
}

// ---- shapes and work memory ------------------------------------------------------------------------------------
enum { FEW, SMALL, MIDDLE, LARGE };
// Up to 16 rows tiles of that many; of 256 x 256 from 128 of them on, but not for few rows; in between 128 x 64, two to a compute unit (forward, in us:
// 512 tokens, 8000 words of 1024: 19, by large tiles 31; 1024, 12288 of 2048: 49, by middle ones 69; 100, 32768 of 2048: 42, by large ones 52).
int shape_for(int64_t m, int64_t n) { return m <= 16 ? FEW : div_up(m, 256) * div_up(n, 256) < 128 || m <= 128 ? MIDDLE : LARGE; }
// Of the kernels that form z: where tiles of 128 words and 64 tokens leave compute units without work, tiles of 64 words
// (81 tokens, 7855 words of 3136: 19.7 us against 26.2; 400, 3053 of 1296: 15.4 against 16.0).
int logit_shape(int64_t tokens, int64_t words) {
    const int shape = shape_for(tokens, words);
    return shape == MIDDLE && div_up(tokens, 64) * div_up(words, 128) < 256 ? SMALL : shape;
}
int tile_m(int shape) { return shape == FEW ? 16 : shape == LARGE ? 256 : 64; }
int tile_n(int shape) { return shape == LARGE ? 256 : 128; }
int tile_words(int shape) { return shape == FEW || shape == SMALL ? 64 : tile_n(shape); }      // of the kernels that form z
// tiles that run on an XCD at a time share its L2: 4096 tokens, 65536 words of 4096, gradient 4.98 ms, in plain order 5.37
WorkOrder order_for(int shape) { return WorkOrder{shape == LARGE ? 32 : 64, 8}; }
// Large tiles run in rounds of one for every compute unit.  Where the last round has few of them, the words that they hold are left to smaller
// tiles in a launch of their own (1003 tokens and 50001 words, 784 tiles: of 1000 elements 129 us against 144, of 256 58 against 66, the gradient
// 353 against 376 and 150 against 157).  Up to 64 tiles: of z 512 of 128 x 64, two to a compute unit, of dW 256 of 128 x 128.
int64_t words_in_rounds(int64_t across, int64_t words) {
    const int64_t tiles = across * div_up(words, 256), over = tiles % 256, whole = (tiles - over) / across;
    return over == 0 || whole == 0 || tiles - whole * across > 64 ? words : whole * 256;
}
struct LogitPlan { int shape[2]; int64_t words[2]; };
LogitPlan logit_plan(int64_t tokens, int64_t words) {
    LogitPlan p = {{logit_shape(tokens, words), 0}, {words, 0}};
    if (p.shape[0] == LARGE) p.words[0] = words_in_rounds(div_up(tokens, 256), words);
    p.words[1] = words - p.words[0];
    p.shape[1] = logit_shape(tokens, p.words[1]);
    return p;
}
int64_t logit_tiles(const LogitPlan& p) { return div_up(p.words[0], tile_words(p.shape[0])) + div_up(p.words[1], tile_words(p.shape[1])); }
struct ProductShape {
    int shape, splits, most;
    ProductRoom room(int64_t m, bool joined) const {
        const int tiles = (int)div_up(m, tile_m(shape));
        return joined || splits > 1 ? ProductRoom{tiles * splits, tile_m(shape), most} : ProductRoom{tiles, tile_m(shape), 1};
    }
};
// dH, whose inner dimension is the vocabulary: large tiles also where they are few, if that leaves every compute unit a share of it of
// some length (1003 x 1024 over 50001 words: 16 tiles in 16 shares; the whole gradient 339 us, with middle tiles 383).  Shares of at least eight steps,
// as many as run at a time (twice as many: 365).
ProductShape dh_shape(int64_t m, int64_t n, int64_t steps) {
    int shape = shape_for(m, n);
    if (shape == MIDDLE && m > 128 && div_up(m, 256) * div_up(n, 256) * (steps / 16) >= 128) shape = LARGE;
    const int64_t tiles = div_up(m, tile_m(shape)) * div_up(n, tile_n(shape)), want = (shape == LARGE ? 256 : 512) / tiles, least = steps / 8, most = least < 1 ? 1 : least > 32 ? 32 : least;
    return ProductShape{shape, (int)(want < 1 ? 1 : want < most ? want : most), (int)most};
}

size_t up(size_t bytes) { return (bytes + 255) & ~(size_t)255; }
constexpr int64_t EDGE = 256;            // what g is padded to, with zeros
int64_t padded(int64_t n) { return div_up(n, EDGE) * EDGE; }
int64_t in_eights(int64_t n) { return div_up(n, 8) * 8; }

struct GradPlaces {
    float* dw_factor;
    float* row_factor;
    float* lse;
    float* held;
    int* target;
    int* place;
    int* count;
    uint8_t* Hc;
    uint8_t* Hs;
    uint8_t* G;
    float* partial;
    float* sum;
    size_t total;
};
GradPlaces grad_places(uint8_t* ws, int64_t tokens, int64_t vocab, int64_t k, int64_t piece) {
    GradPlaces p;
    size_t at = 256;                     // the flag words
    auto take = [&](size_t bytes) { uint8_t* const here = ws + at; at += up(bytes); return here; };
    const int64_t words = piece < vocab ? piece : vocab;
    const ProductShape dh = dh_shape(tokens, k, div_up(words * 2, STEP_BYTES));
    p.dw_factor = reinterpret_cast<float*>(take(4));
    p.row_factor = reinterpret_cast<float*>(take((size_t)tokens * 4));
    p.count = reinterpret_cast<int*>(take(4));
    p.lse = reinterpret_cast<float*>(take((size_t)tokens * 4));
    p.held = reinterpret_cast<float*>(take((size_t)tokens * 4));
    p.target = reinterpret_cast<int*>(take((size_t)tokens * 4));
    p.place = reinterpret_cast<int*>(take((size_t)tokens * 4));
    p.Hc = take((size_t)tokens * in_eights(k) * 2);
    p.Hs = take((size_t)tokens * in_eights(k) * 2);
    p.G = take((size_t)tokens * padded(words) * 2);
    const bool joined = dh.splits > 1 || piece < vocab;
    p.partial = reinterpret_cast<float*>(take(joined ? (size_t)dh.splits * div_up(tokens, tile_m(dh.shape)) * tile_m(dh.shape) * in_fours(k) * 4 : 0));
    p.sum = reinterpret_cast<float*>(take(piece < vocab ? (size_t)tokens * in_fours(k) * 4 : 0));
    p.total = at;
    return p;
}

#define OZAKI_LOSS_TRY(expr) do { const hipError_t e_ = (expr); if (e_ != hipSuccess) return e_; } while (0)

template <int TYPE>
hipError_t launch_dh(ProductWork w, int shape, hipStream_t st) {
    w.tiles_n = (int)div_up(w.n, tile_n(shape));
    w.order = order_for(shape);
    const dim3 blocks((unsigned)((int64_t)w.room.tiles * w.tiles_n));
    if (shape == FEW) hipLaunchKernelGGL((loss_dh_few_kernel<TYPE>), blocks, dim3(256), 0, st, w);
    else if (shape == MIDDLE) hipLaunchKernelGGL((loss_dh_middle_kernel<TYPE>), blocks, dim3(256), 0, st, w);
    else hipLaunchKernelGGL((loss_dh_large_kernel<TYPE>), blocks, dim3(512), 0, st, w);
    return hipGetLastError();
}
template <int TYPE>
hipError_t launch_dw(ProductWork w, hipStream_t st) {
    const bool large = shape_for(w.m, w.n) == LARGE;
    const int edge = large ? 256 : 128;
    w.tiles_n = (int)div_up(w.n, edge);
    w.order = order_for(large ? LARGE : MIDDLE);
    const dim3 blocks((unsigned)(div_up(w.m, edge) * w.tiles_n));
    if (large) hipLaunchKernelGGL((loss_dw_large_kernel<TYPE>), blocks, dim3(512), 0, st, w);
    else hipLaunchKernelGGL((loss_dw_middle_kernel<TYPE>), blocks, dim3(256), 0, st, w);
    return hipGetLastError();
}

void set_tiles(LogitWork& w, int shape) {
    w.steps = (int)div_up(w.bytes, STEP_BYTES);
    w.tiles_m = (int)div_up(w.tokens, tile_m(shape));
    w.tiles_n = (int)div_up(w.words, tile_words(shape));
    w.order = order_for(shape);
}
// the second share of a plan, behind the first
void second_share(LogitWork& w, const LogitPlan& p) {
    w.W += p.words[0] * w.ldw;
    w.first_word += p.words[0];
    w.words = p.words[1];
    if (w.G != nullptr) w.G += p.words[0] * 2;
    else w.part += w.tiles_n * w.tokens;
}

template <int TYPE>
hipError_t forward_typed(const LossArgs& a, uint8_t* ws, hipStream_t st) {
    const LogitPlan plan = logit_plan(a.tokens, a.vocab);
    LogitWork w = {};
    w.H = static_cast<const uint8_t*>(a.H);
    w.W = static_cast<const uint8_t*>(a.W);
    w.ldh = a.ldh * 2;
    w.ldw = a.ldw * 2;
    w.bytes = a.k * 2;
    w.tokens = a.tokens;
    w.targets = a.targets;
    w.target_z = reinterpret_cast<float*>(ws + 256);
    float2* const part = reinterpret_cast<float2*>(ws + 256 + up((size_t)a.tokens * 4));
    w.part = part;
    for (int share = 0; share < 2 && plan.words[share] > 0; ++share) {
        const int shape = plan.shape[share];
        w.words = plan.words[share];
        if (share == 1) second_share(w, plan);
        set_tiles(w, shape);
        const unsigned blocks = (unsigned)(w.tiles_m * (int64_t)w.tiles_n);
        if (shape == FEW) hipLaunchKernelGGL((loss_forward_few_kernel<TYPE>), dim3(blocks), dim3(256), 0, st, w);
        else if (shape == SMALL) hipLaunchKernelGGL((loss_forward_small_kernel<TYPE>), dim3(blocks), dim3(256), 0, st, w);
        else if (shape == MIDDLE) hipLaunchKernelGGL((loss_forward_middle_kernel<TYPE>), dim3(blocks), dim3(256), 0, st, w);
        else hipLaunchKernelGGL((loss_forward_large_kernel<TYPE>), dim3(blocks), dim3(512), 0, st, w);
        OZAKI_LOSS_TRY(hipGetLastError());
    }
    const auto join = [&](auto kernel, int tokens) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)div_up(a.tokens, tokens)), dim3(256), 0, st, part, w.target_z, a.targets, a.tokens, a.vocab, a.ignore,
                           (int)logit_tiles(plan), a.loss, a.lse, a.flags);
    };
    if (a.tokens <= 64) join(loss_join_kernel<1>, 1);
    else join(loss_join_kernel<4>, 4);
    return hipGetLastError();
}

template <int TYPE>
hipError_t grad_typed(const LossArgs& a, int64_t piece, uint8_t* ws, hipStream_t st) {
    const GradPlaces p = grad_places(ws, a.tokens, a.vocab, a.k, piece);
    const int64_t ldhs = in_eights(a.k), each = div_up(a.tokens, 512);
    const GradTokens tokens{a.targets, a.lse_in, a.dloss, a.tokens, a.vocab, a.ignore, a.k, each, p.count, p.place, p.target, p.lse, p.row_factor, p.held, p.dw_factor, a.flags};
    hipLaunchKernelGGL((loss_tokens_kernel<TYPE>), dim3((unsigned)div_up(a.tokens, each)), dim3(TOKEN_THREADS), 0, st, tokens, a.H, a.ldh, p.Hc,
                       a.dW != nullptr ? p.Hs : nullptr, ldhs, a.dH, a.lddh);
    OZAKI_LOSS_TRY(hipGetLastError());
    const bool joined = piece < a.vocab;
    for (int64_t first = 0; first < a.vocab; first += piece) {
        const int64_t words = a.vocab - first < piece ? a.vocab - first : piece;
        const uint8_t* const W = static_cast<const uint8_t*>(a.W) + first * a.ldw * 2;
        LogitWork w = {};
        w.H = p.Hc;
        w.W = W;
        w.ldh = ldhs * 2;
        w.ldw = a.ldw * 2;
        w.bytes = a.k * 2;
        w.tokens = a.tokens;
        w.first_word = first;
        w.count = p.count;
        w.token = TokenState{p.lse, p.target, p.held};
        w.G = p.G;
        w.ldg = padded(words);
        const LogitPlan plan = logit_plan(a.tokens, words);
        for (int share = 0; share < 2 && plan.words[share] > 0; ++share) {
            const int shape = plan.shape[share];
            w.words = plan.words[share];
            if (share == 1) second_share(w, plan);
            set_tiles(w, shape);
            const unsigned blocks = (unsigned)(w.tiles_m * (int64_t)w.tiles_n);
            if (shape == FEW) hipLaunchKernelGGL((loss_g_few_kernel<TYPE>), dim3(blocks), dim3(256), 0, st, w);
            else if (shape == SMALL) hipLaunchKernelGGL((loss_g_small_kernel<TYPE>), dim3(blocks), dim3(256), 0, st, w);
            else if (shape == MIDDLE) hipLaunchKernelGGL((loss_g_middle_kernel<TYPE>), dim3(blocks), dim3(256), 0, st, w);
            else hipLaunchKernelGGL((loss_g_large_kernel<TYPE>), dim3(blocks), dim3(512), 0, st, w);
            OZAKI_LOSS_TRY(hipGetLastError());
        }
        if (a.dH != nullptr) {
            ProductWork d = {};
            d.X = W;
            d.Y = p.G;
            d.ldx = a.ldw * 2;
            d.ldy = padded(words) * 2;
            d.elements = words;                      // (behind them g has zeros to the end of the piece)
            d.count = p.count;
            d.place = p.place;
            d.m = a.tokens;
            d.n = a.k;
            const ProductShape ps = dh_shape(d.m, d.n, div_up(words * 2, STEP_BYTES));
            d.room = ps.room(d.m, joined);
            d.D = a.dH;
            d.ldd = a.lddh;
            d.row_factor = p.row_factor;
            d.partial = joined || ps.splits > 1 ? p.partial : nullptr;
            OZAKI_LOSS_TRY(launch_dh<TYPE>(d, ps.shape, st));
            if (d.partial != nullptr) {
                hipLaunchKernelGGL((loss_product_join_kernel<TYPE>), dim3((unsigned)(d.m < 65536 ? d.m : 65536)), dim3(256), 0, st, p.partial, d.room, d.n, p.sum, first == 0, first + piece >= a.vocab, p.count, p.place, d.row_factor, a.dH, a.lddh);
                OZAKI_LOSS_TRY(hipGetLastError());
            }
        }
        if (a.dW != nullptr) {
            ProductWork d = {};
            d.X = p.Hs;
            d.Y = p.G;
            d.ldx = ldhs * 2;
            d.ldy = padded(words) * 2;
            d.count = p.count;
            d.m = words;
            d.n = a.k;
            d.D = static_cast<uint8_t*>(a.dW) + first * a.lddw * 2;
            d.ldd = a.lddw;
            d.factor = p.dw_factor;
            if (shape_for(d.m, d.n) == LARGE) d.m = words_in_rounds(div_up(d.n, 256), words);
            OZAKI_LOSS_TRY(launch_dw<TYPE>(d, st));
            if (d.m < words) {
                d.Y += d.m * 2;
                d.D = static_cast<uint8_t*>(d.D) + d.m * d.ldd * 2;
                d.m = words - d.m;
                OZAKI_LOSS_TRY(launch_dw<TYPE>(d, st));
            }
        }
    }
    return hipSuccess;
}

}  // namespace

size_t loss_bytes(int64_t tokens, int64_t vocab) {
    return 256 + up((size_t)tokens * 4) + up((size_t)logit_tiles(logit_plan(tokens, vocab)) * tokens * sizeof(float2));
}
size_t loss_grad_bytes(int64_t tokens, int64_t vocab, int64_t k, int64_t piece) { return grad_places(nullptr, tokens, vocab, k, piece).total; }

// As few pieces as keep one piece's g within 1 GiB, all of a length.
int64_t loss_grad_piece(int64_t tokens, int64_t vocab, int64_t k) {
    const int64_t fits = ((int64_t)1 << 30) / (2 * tokens), most = fits < LOSS_PIECE ? LOSS_PIECE : fits;
    const int64_t piece = padded(div_up(vocab, div_up(vocab, most)));
    return piece < LOSS_PIECE ? LOSS_PIECE : piece;
}

hipError_t launch_zero_rows(void* D, int64_t rows, int64_t k, int64_t ldd, hipStream_t st) {
    const int64_t blocks = div_up(rows * k, 256);
    hipLaunchKernelGGL(zero_rows_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, st, static_cast<uint16_t*>(D), rows, k, ldd);
    return hipGetLastError();
}
hipError_t launch_linear_loss(const LossArgs& a, int type, uint8_t* ws, hipStream_t st) {
    return type == TYPE_F16 ? forward_typed<TYPE_F16>(a, ws, st) : forward_typed<TYPE_BF16>(a, ws, st);
}
hipError_t launch_linear_loss_grad(const LossArgs& a, int type, int64_t piece, uint8_t* ws, hipStream_t st) {
    return type == TYPE_F16 ? grad_typed<TYPE_F16>(a, piece, ws, st) : grad_typed<TYPE_BF16>(a, piece, ws, st);
}

}  // namespace ozaki
