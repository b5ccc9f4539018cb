// Shared by the operators of a feed-forward block and its training step: activations, the launchers' arguments and prototypes.
#pragma once
#include <type_traits>

#include "low_precision.hpp"

namespace ozaki {

// values of the activation argument
constexpr int ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4;
inline bool activation_ok(int a) { return a >= ACT_NONE && a <= ACT_SILU; }

// ---- linear.hip ----------------------------------------------------------------------------------------------
// Y = act(X W^T + bias) + R, Z what the activation is taken of; a pair: Y = act(X W^T) * (X W2^T), Z and U the two factors' products.
struct LinearArgs {
    const void* X;           // m vectors of k elements
    const void* W;           // n vectors
    const void* W2;          // pair: n vectors
    const void* bias;        // may be null
    const void* R;           // may be null
    void* Y;
    void* Z;                 // may be null
    void* U;                 // pair: null if Z is
    int64_t m, n, k, ldx, ldw, ldr, ldy, ldz, ldu;
    int activation;
    float* partial;          // the shares of the inner dimension, where it is cut
};
size_t linear_bytes(int64_t m, int64_t n, int64_t k, bool pair);           // of `partial`; 0: none is needed
hipError_t launch_linear(const LinearArgs& a, int type, hipStream_t st);

// ---- linear_grad.hip -----------------------------------------------------------------------------------------
struct LinearGradArgs {
    const void* X;
    const void* W;
    const void* W2;          // pair
    const void* Z;           // what the forward call left; may be null without an activation
    const void* U;           // pair
    const void* dY;
    void* dX;                // any of the results may be null
    void* dW;
    void* dW2;
    float* dbias;
    int64_t m, n, k, ldx, ldw, ldz, ldu, lddy, lddx, lddw;
    int activation;
    bool pair;
    uint8_t* ws;
};
size_t linear_grad_bytes(int64_t m, int64_t n, int64_t k, bool pair);
hipError_t launch_linear_grad(const LinearGradArgs& a, int type, hipStream_t st);

// ---- block_norm.hip ------------------------------------------------------------------------------------------
constexpr int64_t MAX_NORM = 16384;       // elements of a row: a workgroup keeps it in registers
struct BlockNormArgs {
    const void* X;
    const float* w_post;
    const float* gate;       // [row / group][k]
    const float* w_pre;
    const void* R;           // gradient: the sum that the forward call left
    int64_t rows, k, ldx, ldr, group;
    float scale, eps;
    // forward: out
    void* R_out;
    void* H;
    int64_t ldro, ldh;
    // gradient: what arrives, and out
    const void* dH;
    const void* dR_out;
    void* dX;
    void* dR;
    float* dw_post;
    float* dgate;
    float* dw_pre;
    int64_t lddh, lddro, lddx, lddr;
    uint8_t* ws;
};
size_t block_norm_grad_bytes(int64_t rows, int64_t k, int64_t group);
hipError_t launch_block_norm(const BlockNormArgs& a, int type, int type_r, hipStream_t st);
hipError_t launch_block_norm_grad(const BlockNormArgs& a, int type, int type_r, hipStream_t st);

// ---- gradient_norm.hip ---------------------------------------------------------------------------------------
constexpr int64_t MAX_TENSORS = (int64_t)1 << 27, MAX_CLIPPED = (int64_t)1 << 43;       // of a call; elements of all of them
struct ClipArgs {
    int count;
    const void* const* tensors;      // HOST
    const int64_t* sizes;            // HOST
    const int* types;                // HOST
    void* const* out;                // HOST; null: only the norm
    float scale, max_norm;
    float* norm;
    bool given;                      // the norm is there already
    uint8_t* ws;
};
size_t gradient_norm_bytes(int64_t count);
hipError_t launch_clip(const ClipArgs& a, hipStream_t st);

#if defined(__HIPCC__)

typedef float v8f32 __attribute__((ext_vector_type(8)));
// Eight neighbouring elements, wherever they lie: the memory takes 16-byte accesses at any element.
template <typename T> using Eight = T __attribute__((ext_vector_type(8), aligned(sizeof(T))));
template <typename T> __device__ __forceinline__ v8f32 get_eight(const T* p) { return __builtin_convertvector(*reinterpret_cast<const Eight<T>*>(p), v8f32); }
template <bool STREAMED, typename T> __device__ __forceinline__ void put_eight(T* to, v8f32 v) {
    const Eight<T> w = __builtin_convertvector(v, Eight<T>);
    if constexpr (STREAMED) __builtin_nontemporal_store(w, reinterpret_cast<Eight<T>*>(to));
    else *reinterpret_cast<Eight<T>*>(to) = w;
}
template <typename T> __device__ __forceinline__ bool rows_aligned(const T* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * sizeof(T) % 16 == 0; }

// 1 / (1 + exp(-x)) and what it lacks of one, each with its own few roundings: the exponential is of -|x|, so that it neither overflows nor cancels.
struct Sigmoid { float p, rest; };
__device__ __forceinline__ Sigmoid sigmoid_of(float x) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896340736f * fabsf(x)), r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
    return x < 0.0f ? Sigmoid{er, r} : Sigmoid{r, er};
}
constexpr float GELU_C = 0.79788456080286535588f, GELU_CUBE = 0.044715f;       // sqrt(2 / pi)
// (beyond 20 the tanh is one; the cube of what is far beyond would not be finite)
__device__ __forceinline__ float gelu_argument(float z) {
    const float c = fminf(fmaxf(z, -20.0f), 20.0f);
    return 2.0f * GELU_C * (c + GELU_CUBE * c * c * c);
}
// Phi(z) and exp(-z^2 / 2).  With x = |z| / sqrt(2) and r = 1 / (1 + 0.4 x), erfc(x) exp(x^2) / r is a polynomial of degree 8 in 2 r - 1 to within 1.6e-7 of itself for
// all x, with the coefficients in 32 bits (least squares, reweighted until the largest relative error is least); so the tail keeps its relative precision, and 20 instructions do what the library's erfc takes
// several times as many for.
struct Normal { float phi, e; };
__device__ __forceinline__ Normal normal_of(float z) {
    const float r = __builtin_amdgcn_rcpf(__builtin_fmaf(0.4f * 0.70710678118654752440f, fabsf(z), 1.0f)), t = __builtin_fmaf(2.0f, r, -1.0f);
    float q = 1.963244576472789e-04f;
    q = __builtin_fmaf(q, t, 1.4176529657561332e-04f);
    q = __builtin_fmaf(q, t, -1.8630237318575382e-03f);
    q = __builtin_fmaf(q, t, -3.3358947839587927e-03f);
    q = __builtin_fmaf(q, t, 1.1324104852974415e-02f);
    q = __builtin_fmaf(q, t, 6.849516183137894e-02f);
    q = __builtin_fmaf(q, t, 1.8156789243221283e-01f);
    q = __builtin_fmaf(q, t, 3.218610882759094e-01f);
    q = __builtin_fmaf(q, t, 4.216126799583435e-01f);
    const float e = __builtin_amdgcn_exp2f(-0.72134752044448170368f * z * z), half = 0.5f * q * r * e;
    return Normal{z < 0.0f ? half : 1.0f - half, e};
}
template <int ACT> __device__ __forceinline__ float activated(float z) {
    if constexpr (ACT == ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == ACT_GELU) return z * normal_of(z).phi;
    if constexpr (ACT == ACT_GELU_TANH) return z * sigmoid_of(gelu_argument(z)).p;                 // (1 + tanh y) / 2 = 1 / (1 + exp(-2 y))
    if constexpr (ACT == ACT_SILU) return z * sigmoid_of(z).p;
    return z;
}
// the activation's value and derivative
struct Activation { float value, slope; };
template <int ACT> __device__ __forceinline__ Activation activation_of(float z) {
    if constexpr (ACT == ACT_RELU) return Activation{z < 0.0f ? 0.0f : z, z > 0.0f ? 1.0f : z <= 0.0f ? 0.0f : z};
    if constexpr (ACT == ACT_GELU) {
        const Normal n = normal_of(z);
        return Activation{z * n.phi, n.phi + z * (0.39894228040143267794f * n.e)};
    }
    if constexpr (ACT == ACT_GELU_TANH) {
        const Sigmoid s = sigmoid_of(gelu_argument(z));
        const float c = fminf(fmaxf(z, -20.0f), 20.0f);
        return Activation{z * s.p, s.p + z * s.p * s.rest * (2.0f * GELU_C * (1.0f + 3.0f * GELU_CUBE * c * c))};
    }
    if constexpr (ACT == ACT_SILU) {
        const Sigmoid s = sigmoid_of(z);
        return Activation{z * s.p, s.p * (1.0f + z * s.rest)};
    }
    return Activation{z, 1.0f};
}
// f(constant) for the activation that the argument names
template <typename F> __device__ __forceinline__ void with_activation(int activation, F f) {
    switch (activation) {
        case ACT_RELU: f(std::integral_constant<int, ACT_RELU>()); break;
        case ACT_GELU: f(std::integral_constant<int, ACT_GELU>()); break;
        case ACT_GELU_TANH: f(std::integral_constant<int, ACT_GELU_TANH>()); break;
        case ACT_SILU: f(std::integral_constant<int, ACT_SILU>()); break;
        default: f(std::integral_constant<int, ACT_NONE>()); break;
    }
}

#endif

}  // namespace ozaki
