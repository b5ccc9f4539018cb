// Shared by the low-precision operators: element types, the blocks that share a scale, and the launchers' prototypes.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ozaki {

// values of the type, scaling arguments
constexpr int TYPE_F32 = 0, TYPE_BF16 = 1, TYPE_F16 = 2;
constexpr int SCALE_VECTORS = 0, SCALE_BLOCKS = 1;
constexpr int SCALE_BLOCK = 128;          // elements that share a scale, along one axis or both
constexpr int64_t MAX_VECTOR_BYTES = (int64_t)1 << 22;      // between vectors, and of one: 255 of them stay inside a 32-bit offset

inline bool type_ok(int type) { return type >= TYPE_F32 && type <= TYPE_F16; }
inline int type_bytes(int type) { return type == TYPE_F32 ? 4 : 2; }
__host__ __device__ inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }
__host__ __device__ inline int64_t in_fours(int64_t n) { return (n + 3) & ~(int64_t)3; }

// ---- quantise_fp8.hip ----------------------------------------------------------------------------------------
struct QuantiseArgs {
    const void* X;
    int64_t rows, k, ldx;
    uint8_t* Q;              // null: not wanted
    int64_t ldq;
    float* S;
    int64_t lds;
    uint8_t* Qt;             // of the transpose; null: not wanted
    int64_t ldqt;
    float* St;
    int64_t ldst;
};
hipError_t launch_quantise_fp8(const QuantiseArgs& a, int type, int scaling, hipStream_t st);

// ---- gemm_fp8.hip --------------------------------------------------------------------------------------------
struct GemmFp8Args {
    const uint8_t* A;        // m vectors of k bytes, lda apart
    const uint8_t* B;        // n vectors
    const float* Sa;         // [k block][m]
    const float* Sb;         // [k block][n], or [k block][n / 128]
    void* D;                 // m x n, rows ldd apart
    float* partial;          // splits > 1: [split][m][n in fours]
    int64_t m, n, k, lda, ldb, ldsa, ldsb, ldd;
    int accumulate;
};
// How many pieces the inner dimension is cut into, whose sums meet in work memory; 1: none is needed.
int gemm_fp8_splits(int64_t m, int64_t n, int64_t k);
hipError_t launch_gemm_fp8(const GemmFp8Args& a, int scaling, int type_d, int splits, hipStream_t st);

// ---- linear_loss.hip -----------------------------------------------------------------------------------------
struct LossArgs {
    const void* H;           // tokens x k
    const void* W;           // vocab x k
    const int64_t* targets;
    int64_t tokens, vocab, k, ldh, ldw, ignore;
    float* loss;             // forward: out
    float* lse;              // forward: out
    const float* lse_in;     // gradient
    const float* dloss;
    void* dH;                // gradient: out, either may be null
    void* dW;
    int64_t lddh, lddw;
    int* flags;              // work memory's flag words
};
// Work memory: of the forward pass; of the gradient with the vocabulary in pieces of `piece` words (a multiple of LOSS_PIECE).
constexpr int LOSS_PIECE = 256;
size_t loss_bytes(int64_t tokens, int64_t vocab);
size_t loss_grad_bytes(int64_t tokens, int64_t vocab, int64_t k, int64_t piece);
int64_t loss_grad_piece(int64_t tokens, int64_t vocab, int64_t k);        // what is recommended
hipError_t launch_linear_loss(const LossArgs& a, int type, uint8_t* ws, hipStream_t st);
hipError_t launch_zero_rows(void* D, int64_t rows, int64_t k, int64_t ldd, hipStream_t st);       // of 16-bit elements
hipError_t launch_linear_loss_grad(const LossArgs& a, int type, int64_t piece, uint8_t* ws, hipStream_t st);

// bits of flag word 0: an FP64 product's input was not finite; a target was neither a word of the vocabulary nor `ignore`
constexpr int NONFINITE_FLAG = 1, TARGET_FLAG = 2;

#if defined(__HIPCC__)

typedef int v2i32 __attribute__((ext_vector_type(2)));
typedef int v4i32 __attribute__((ext_vector_type(4)));
typedef int v8i32 __attribute__((ext_vector_type(8)));
typedef float v4f32 __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));
typedef _Float16 v2f16 __attribute__((ext_vector_type(2)));
typedef _Float16 v8f16 __attribute__((ext_vector_type(8)));

template <int TYPE> struct Element;
template <> struct Element<TYPE_F32> { typedef float type; };
template <> struct Element<TYPE_BF16> { typedef __bf16 type; };
template <> struct Element<TYPE_F16> { typedef _Float16 type; };

#endif

}  // namespace ozaki
