// The product of a tile of vectors X (rows of the matrix unit's result) with a tile of vectors Y (its columns), both contiguous along
// the inner dimension: FP8 codes with a scale per 128 of them, BF16 or FP16.
//
// A step is 128 bytes of the inner dimension of every vector of the tile: 128 FP8 codes, which are one v_mfma_f32_16x16x128 deep and
// share their scales, or 64 elements of 16 bits, two v_mfma_f32_16x16x32 deep.  Steps travel from memory to LDS with direct loads
// through a ring of NST buffers; a wave reads its fragments from there.
//
// LDS rows are 128 bytes; the eight 16-byte pieces of row r lie at place piece ^ ((r >> 1) & 7).  Lane l reads pieces l / 16 and l / 16 + 4
// of row l % 16 of a 16-row tile: the sixteen lanes that a 128-bit LDS read serves together (0-3, 12-15, 20-23, 24-27 and the like)
// then meet sixteen different places of the 256 bytes that the banks hold.  (Which elements of the inner dimension a lane takes is
// free, as long as both operands agree.)  A direct load writes lane l's 16 bytes at a fixed place, base + 16 l, so each lane
// fetches the piece that belongs there.
//
// Vectors beyond the matrix repeat the last one; their results are not stored.  Pieces beyond the end of the vectors are read from
// sixteen zero bytes, and where the end lies inside a piece the bytes behind it are cleared in LDS, in both operands: what the
// caller's memory holds there may be a NaN.
#pragma once
#include <type_traits>

#include "low_precision.hpp"

namespace ozaki {
namespace {

// FP8: X's scales per 128 x 128 block or per 128 elements of a vector (Y's always the latter), on the FP8 or on the FP16 instructions
constexpr int KIND_FP8_BLOCKS = 0, KIND_FP8_VECTORS = 1, KIND_WIDE_BLOCKS = 2, KIND_WIDE_VECTORS = 3, KIND_BF16 = 4, KIND_F16 = 5;
constexpr int STEP_BYTES = 128;

#define OZAKI_TILE_GPTR(p) ((const __attribute__((address_space(1))) void*)(p))
#define OZAKI_TILE_LPTR(p) ((__attribute__((address_space(3))) void*)(p))

__device__ __attribute__((aligned(16))) uint8_t no_elements[16];

// A lane's share of 16 vectors' 128 codes, and the product of two such shares over the 128 elements.  The matrix unit's FP8 instructions align
// the products of eight neighbouring codes to the largest of them and cut them 13 bits below its exponent (measured; the sums of
// eight are then added in 24 bits): 1.4e-5 of the result's norm on normally distributed codes, a hundredth of a 16-bit result's rounding but
// two hundred of a 32-bit one's.  Its FP16 instructions, at half the rate, do not, and FP16 holds every E4M3 code: `WIDE`.
template <bool WIDE> struct Fragment {
    typedef v8i32 type;
    static __device__ __forceinline__ type of(v8i32 codes) { return codes; }
    static __device__ __forceinline__ v4f32 product(const type& x, const type& y) {
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, v4f32{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
    }
};
template <> struct Fragment<true> {
    struct type { v8f16 part[4]; };
    static __device__ __forceinline__ type of(v8i32 codes) {
        type f;
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v2f16 two = (q & 1) ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[2 * p + (q >> 1)], 1.0f, true)
                                          : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(codes[2 * p + (q >> 1)], 1.0f, false);
                f.part[p][2 * q] = two[0];
                f.part[p][2 * q + 1] = two[1];
            }
        return f;
    }
    static __device__ __forceinline__ v4f32 product(const type& x, const type& y) {
        v4f32 t = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int p = 0; p < 4; ++p) t = __builtin_amdgcn_mfma_f32_16x16x32_f16(x.part[p], y.part[p], t, 0, 0, 0);
        return t;
    }
};

struct TileOperand {
    const uint8_t* vectors;      // the tile's first vector
    int64_t stride;              // bytes
    int rows;                    // vectors from there to the matrix's last, at least 1
    const float* scales;         // FP8: of the tile's first vector (or block of vectors) in inner block 0
    int64_t scale_stride;        // between inner blocks
    // Turned operands (16 bits): the matrix lies the other way, element e of all vectors in a row; `vectors` is element 0 of the tile's first
    // vector, `stride` the distance between rows, and `rows` the vectors from there on; there are `elements` rows.
    int64_t elements = 0;
    // Pairs of matrices (XP): the second one's vectors of the tile, as far apart; `rows` is each one's.
    const uint8_t* second = nullptr;
};

// A turned operand in LDS: 64 rows of 128 vectors, 256 bytes each, to a panel.  A fragment is read with ds_read_b64_tr_b16, which gives a lane four
// elements of one vector: the sixteen lanes of a group address four rows of 32 bytes, row (lane % 16) / 4, and get vector lane % 16 of them.
// Lanes that are served together read rows 0 - 3 of each eight at the same 32 bytes; piece p (32 bytes) of row r lies at p ^ turned_place(r),
// which spreads them over the banks.
constexpr int PANEL_BYTES = 64 * 256;
__device__ __forceinline__ int turned_place(int row) { return (row & 3) | ((row >> 3) & 1) << 2; }
// Direct loads beside ds_read_b64_tr_b16: the compiler takes every such read to depend on every direct load under way and waits for all of
// them, which the pipelines here are built not to do, so the loads are written out.  (They have no register to return to; who reads what
// they bring waits for them in tile_wait.  The pause is for m0, and for scalar registers that a vector instruction may have written just before.)
__device__ __forceinline__ unsigned lds_place(const uint8_t* lds) { return __builtin_amdgcn_readfirstlane((unsigned)(uintptr_t)OZAKI_TILE_LPTR(lds)); }
__device__ __forceinline__ void direct_load(const uint8_t* from, const uint8_t* lds) {
    int m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds_place(lds)), "v"(from) : "memory");
}
__device__ __forceinline__ void direct_load(v4i32 resource, unsigned offset, int step, const uint8_t* lds) {
    int m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 4\n\tbuffer_load_dwordx4 %2, %3, %4 offen lds\n\ts_mov_b32 m0, %0"
                 : "=&s"(m0) : "s"(lds_place(lds)), "v"(offset), "s"(resource), "s"(step) : "memory");
}
// the words of a raw buffer resource
__device__ __forceinline__ v4i32 resource_of(const uint8_t* base, unsigned records) {
    const uint64_t at = reinterpret_cast<uint64_t>(base);
    return v4i32{__builtin_amdgcn_readfirstlane((int)(unsigned)at), __builtin_amdgcn_readfirstlane((int)(unsigned)(at >> 32) & 0xFFFF), (int)records, 0x00027000};
}

// the lane's share of 16 vectors (piece `p` of a panel) and 64 elements, in the order in which a lane reads pieces g and g + 4 of an ordinary row
__device__ __forceinline__ v8i32 turned_fragment(const uint8_t* panel, int p, int lane) {
    typedef short v4i16 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4i16* place;
    const int g = lane >> 4, in = (lane >> 2) & 3, at = (8 * g + in) * 256 + ((p ^ (in | (g & 1) << 2)) << 5) + (lane & 3) * 8;
    v8i32 out;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const v2i32 two = __builtin_bit_cast(v2i32, __builtin_amdgcn_ds_read_tr16_b64_v4i16((place)OZAKI_TILE_LPTR(panel + at + (32 * h + 4 * t) * 256)));
            out[4 * h + 2 * t] = two[0];
            out[4 * h + 2 * t + 1] = two[1];
        }
    return out;
}

// where share s of the steps begins
__device__ __forceinline__ int split_begin(int steps, int splits, int s) { return (int)((int64_t)steps * s / splits); }

// four neighbouring elements of a row of D, the first `left` of them; `wide`: D's rows start at multiples of four elements
template <typename T>
__device__ __forceinline__ void put_four(T* at, v4f32 v, int64_t left, bool wide, bool accumulate) {
    typedef T four __attribute__((ext_vector_type(4)));
    if (wide && left >= 4) {
        if (accumulate) {
            const four old = *reinterpret_cast<const four*>(at);
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] += (float)old[r];
        }
        *reinterpret_cast<four*>(at) = four{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < left) at[r] = (T)(accumulate ? v[r] + (float)at[r] : v[r]);
    }
}

// the first `keep` of sixteen bytes, zeros behind them
__device__ __forceinline__ v4i32 first_bytes(v4i32 v, int keep) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int bytes = keep - 4 * q;
        v[q] = bytes >= 4 ? v[q] : bytes <= 0 ? 0 : v[q] & (int)((1u << (8 * bytes)) - 1);
    }
    return v;
}

// Waits until at most N vector-memory operations of this wave are outstanding and its LDS operations are done, then meets the others.
template <int N>
__device__ __forceinline__ void tile_wait() {
    static_assert(N >= 0 && N < 64, "range of the counter");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | 0x0070);   // vmcnt(N) expcnt(7) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// WN x WM waves, each FN x FM tiles of 16 x 16; XT, YT: the operand is turned; XP: X is a pair of matrices, TN / 2 vectors of each, and a lane that has
// element r of acc[i][j] from the first has the same vector of the second in acc[i + FN / 2][j].
template <int KIND, int WN_, int WM_, int FN_, int FM_, int NST_, bool XT = false, bool YT = false, bool XP = false>
struct Tile {
    static constexpr bool FP8 = KIND < KIND_BF16, WIDE = KIND == KIND_WIDE_BLOCKS || KIND == KIND_WIDE_VECTORS;
    static constexpr bool BLOCKS = KIND == KIND_FP8_BLOCKS || KIND == KIND_WIDE_BLOCKS;
    static constexpr int WN = WN_, WM = WM_, FN = FN_, FM = FM_, NST = NST_;
    static constexpr int WAVES = WN * WM, THREADS = 64 * WAVES, TN = WN * FN * 16, TM = WM * FM * 16, ROWS = TN + TM;
    static constexpr int SCALE_BYTES = FP8 ? (ROWS * 4 + 255) / 256 * 256 : 0;
    static constexpr int STAGE_BYTES = ROWS * STEP_BYTES + SCALE_BYTES;
    static constexpr int LDS_BYTES = NST * STAGE_BYTES;
    static constexpr int PIECE_LOADS = ROWS / 8, SCALE_LOADS = SCALE_BYTES / 256;                  // wave instructions of a stage
    static constexpr int LPW = (PIECE_LOADS + WAVES - 1) / WAVES, SPW = (SCALE_LOADS + WAVES - 1) / WAVES;
    static_assert(!FP8 || (!XT && !YT), "");
    static_assert((!XT || TN % 128 == 0) && (!YT || TM % 128 == 0), "");
    static_assert(!XP || (!FP8 && !XT && FN % 2 == 0), "");
    static constexpr bool PAIR = XP;

    // acc[i][j][r] += X row wn * FN * 16 + 16 i + 4 (lane / 16) + r  times  Y row wm * FM * 16 + 16 j + lane % 16, over the steps
    // [step0, step1) of vectors of `bytes` bytes (if only one operand is turned, the other has zeros behind them to the end of the 16 bytes).  Ends
    // with nothing in flight and all waves past their last LDS read.
    __device__ static void multiply(uint8_t* lds, const TileOperand& X, const TileOperand& Y, int64_t bytes, int step0, int step1,
                                    v4f32 (&acc)[FN][FM]) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wn = wave / WM, wm = wave % WM;
        const int steps = step1 - step0;
        const int64_t rest = bytes - (int64_t)(step1 - 1) * STEP_BYTES;
        const int last_bytes = rest < STEP_BYTES ? (int)rest : STEP_BYTES;              // of the last step
        const bool ragged = last_bytes < STEP_BYTES;

        // what this lane loads: LPW pieces, at `from` (uniform) + voff, and SPW scales
        unsigned voff[LPW];
        const uint8_t* from[LPW];
        int to[LPW];
        {
            const int r = lane >> 3;
#pragma unroll
            for (int i = 0; i < LPW; ++i) {
                int at = wave * LPW + i;
                at = at < PIECE_LOADS ? at : PIECE_LOADS - 1;                           // (the same bytes to the same place twice)
                const bool x = at * 8 < TN;
                const int row = at * 8 + r, rows = x ? X.rows : Y.rows;
                const int mine = !x ? row - TN : XP ? row / (FN * 16) * (FN * 8) + row % (FN * 8) : row;
                const unsigned piece = (lane & 7) ^ ((row >> 1) & 7);
                voff[i] = (unsigned)(mine < rows ? mine : rows - 1) * (unsigned)(x ? X.stride : Y.stride) + piece * 16;
                from[i] = (x ? X.vectors : Y.vectors) + (int64_t)step0 * STEP_BYTES;
                to[i] = at * 1024;
                if (XP && x && at * 8 % (FN * 16) >= FN * 8) from[i] = X.second + (int64_t)step0 * STEP_BYTES;
                if ((x && XT) || (!x && YT)) {
                    // four rows of a panel
                    const int q = x ? at : at - TN / 8, e = (q & 15) * 4 + (lane >> 4);
                    const int v = (q >> 4) * 128 + (((lane & 15) >> 1) ^ turned_place(e)) * 16 + (lane & 1) * 8;
                    voff[i] = (unsigned)e * (unsigned)(x ? X.stride : Y.stride) + 2 * (unsigned)(v < rows ? v : 0);
                    from[i] = (x ? X.vectors : Y.vectors) + (int64_t)step0 * 64 * (x ? X.stride : Y.stride);
                }
            }
        }
        const float* sfrom[SPW > 0 ? SPW : 1];
        int64_t sstride[SPW > 0 ? SPW : 1];
        int sto[SPW > 0 ? SPW : 1];
        if constexpr (FP8) {
#pragma unroll
            for (int i = 0; i < SPW; ++i) {
                int at = wave * SPW + i;
                at = at < SCALE_LOADS ? at : SCALE_LOADS - 1;
                const int row = at * 64 + lane < ROWS ? at * 64 + lane : ROWS - 1;
                const bool x = row < TN;
                const int mine = x ? row : row - TN, rows = x ? X.rows : Y.rows, real = mine < rows ? mine : rows - 1;
                const int index = x && BLOCKS ? real / SCALE_BLOCK : real;
                sfrom[i] = (x ? X.scales + (int64_t)step0 * X.scale_stride : Y.scales + (int64_t)step0 * Y.scale_stride) + index;
                sstride[i] = x ? X.scale_stride : Y.scale_stride;
                sto[i] = ROWS * STEP_BYTES + at * 256;
            }
        }
        auto is_x = [&](int i) {
            const int at = wave * LPW + i;
            return (at < PIECE_LOADS ? at : PIECE_LOADS - 1) * 8 < TN;
        };
        auto step_of = [&](int i) -> int64_t {
            if (XT || YT) return is_x(i) ? (XT ? 64 * X.stride : STEP_BYTES) : (YT ? 64 * Y.stride : STEP_BYTES);
            return STEP_BYTES;
        };
        int issue_buf = 0;
        auto issue_scales = [&]() {
            if constexpr (FP8) {
#pragma unroll
                for (int i = 0; i < SPW; ++i) {
                    __builtin_amdgcn_global_load_lds(OZAKI_TILE_GPTR(sfrom[i]), OZAKI_TILE_LPTR(lds + issue_buf * STAGE_BYTES + sto[i]), 4, 0, 0);
                    sfrom[i] += sstride[i];
                }
            }
        };
        auto issue_full = [&]() {
#pragma unroll
            for (int i = 0; i < LPW; ++i) {
                if constexpr (XT || YT) direct_load(from[i] + voff[i], lds + issue_buf * STAGE_BYTES + to[i]);
                else __builtin_amdgcn_global_load_lds(OZAKI_TILE_GPTR(from[i] + voff[i]), OZAKI_TILE_LPTR(lds + issue_buf * STAGE_BYTES + to[i]), 16, 0, 0);
                from[i] += step_of(i);
            }
            issue_scales();
            issue_buf = issue_buf + 1 == NST ? 0 : issue_buf + 1;
        };
        // the last step, or (none) none at all: loads that keep the count of those in flight even
        auto issue_last = [&](bool none) {
#pragma unroll
            for (int i = 0; i < LPW; ++i) {
                int at = wave * LPW + i;
                at = at < PIECE_LOADS ? at : PIECE_LOADS - 1;
                const int piece = (lane & 7) ^ (((at * 8 + (lane >> 3)) >> 1) & 7);
                bool there = !none && piece * 16 < last_bytes;
                if (XT || YT) {
                    const bool x = at * 8 < TN;
                    const int e = ((x ? at : at - TN / 8) & 15) * 4 + (lane >> 4);
                    if (x ? XT : YT) there = !none && (int64_t)(step1 - 1) * 64 + e < (x ? X.elements : Y.elements);
                }
                const uint8_t* src = there ? from[i] + voff[i] : no_elements;
                if constexpr (XT || YT) direct_load(src, lds + issue_buf * STAGE_BYTES + to[i]);
                else __builtin_amdgcn_global_load_lds(OZAKI_TILE_GPTR(src), OZAKI_TILE_LPTR(lds + issue_buf * STAGE_BYTES + to[i]), 16, 0, 0);
            }
            if constexpr (FP8) {
#pragma unroll
                for (int i = 0; i < SPW; ++i) {
                    const float* src = none ? reinterpret_cast<const float*>(no_elements) : sfrom[i];
                    __builtin_amdgcn_global_load_lds(OZAKI_TILE_GPTR(src), OZAKI_TILE_LPTR(lds + issue_buf * STAGE_BYTES + sto[i]), 4, 0, 0);
                }
            }
            issue_buf = issue_buf + 1 == NST ? 0 : issue_buf + 1;
        };

        const int frow = lane & 15, g = lane >> 4, fsw = (frow >> 1) & 7;
        const int piece0 = (g ^ fsw) << 4, piece1 = ((g + 4) ^ fsw) << 4;
        const int xbase = (wn * FN * 16 + frow) * STEP_BYTES, ybase = (TN + wm * FM * 16 + frow) * STEP_BYTES;
        int read_buf = 0;
        auto fragment = [&](const uint8_t* at) -> v8i32 {
            const v4i32 lo = *reinterpret_cast<const v4i32*>(at + piece0), hi = *reinterpret_cast<const v4i32*>(at + piece1);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        // A step's products.  The order is fixed: a product's fused multiply-adds come behind the next products, which cover the matrix
        // unit's latency, and a row's fragment is read while the row two before it is multiplied.
        auto compute = [&]() {
            const uint8_t* const stage = lds + read_buf * STAGE_BYTES;
            typedef typename Fragment<WIDE>::type operand;
            constexpr int AHEAD = FN > 1 ? 2 : 1;                     // rows whose fragments are read in front
            operand y[FM], x[AHEAD + 1];
            auto row = [&](int i) {
                if constexpr (XT) {
                    const int t = wn * FN + i;
                    return turned_fragment(stage + (t >> 3) * PANEL_BYTES, t & 7, lane);
                } else {
                    return Fragment<WIDE>::of(fragment(stage + xbase + i * 16 * STEP_BYTES));
                }
            };
            auto column = [&](int j) {
                if constexpr (YT) {
                    const int t = wm * FM + j;
                    return turned_fragment(stage + TN * STEP_BYTES + (t >> 3) * PANEL_BYTES, t & 7, lane);
                } else {
                    return Fragment<WIDE>::of(fragment(stage + ybase + j * 16 * STEP_BYTES));
                }
            };
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (FP8) {
                const float* const scales = reinterpret_cast<const float*>(stage + ROWS * STEP_BYTES);
                constexpr int MOST = BLOCKS ? 3 : 2, LAG = FM * FN > MOST ? MOST : FM * FN - 1, T = LAG + 1;
                float sy[FM], sx_all = 0.0f;
                v4f32 t[T], sx[2] = {};
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    y[j] = column(j);
                    if (j < AHEAD && j < FN) x[j] = row(j);
                }
                if (AHEAD > FM) x[1] = row(1);
#pragma unroll
                for (int j = 0; j < FM; ++j) sy[j] = scales[TN + (wm * FM + j) * 16 + frow];
                // (the wave's rows lie in one block of 128 vectors)
                static_assert(!BLOCKS || SCALE_BLOCK % (FN * 16) == 0, "");
                if constexpr (BLOCKS) sx_all = scales[wn * FN * 16];
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < FN * FM + LAG; ++n) {
                    if (n < FN * FM) {
                        const int i = n / FM, j = n % FM;
                        if (j == 0 && i + AHEAD < FN) x[(i + AHEAD) % (AHEAD + 1)] = row(i + AHEAD);
                        if (!BLOCKS && j == 0) sx[i & 1] = *reinterpret_cast<const v4f32*>(scales + (wn * FN + i) * 16 + 4 * g);
                        t[n % T] = Fragment<WIDE>::product(x[i % (AHEAD + 1)], y[j]);
                    }
                    if (BLOCKS && n == LAG) {
#pragma unroll
                        for (int j = 0; j < FM; ++j) sy[j] *= sx_all;
                    }
                    if (n >= LAG) {
                        const int d = n - LAG, i = d / FM, j = d % FM;
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            acc[i][j][r] = __builtin_fmaf(t[d % T][r], BLOCKS ? sy[j] : sx[i & 1][r] * sy[j], acc[i][j][r]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int j = 0; j < FM; ++j) {
                    y[j] = column(j);
                    if (j < AHEAD && j < FN) x[j] = row(j);
                }
                if (AHEAD > FM) x[1] = row(1);
#pragma unroll
                for (int i = 0; i < FN; ++i) {
                    if (i + AHEAD < FN) x[(i + AHEAD) % (AHEAD + 1)] = row(i + AHEAD);
                    const v8i32 xi = x[i % (AHEAD + 1)];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int j = 0; j < FM; ++j) {
                            const v4i32 xh = h ? __builtin_shufflevector(xi, xi, 4, 5, 6, 7) : __builtin_shufflevector(xi, xi, 0, 1, 2, 3);
                            const v4i32 yh = h ? __builtin_shufflevector(y[j], y[j], 4, 5, 6, 7) : __builtin_shufflevector(y[j], y[j], 0, 1, 2, 3);
                            if constexpr (KIND == KIND_BF16)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf16, xh), __builtin_bit_cast(v8bf16, yh), acc[i][j], 0, 0, 0);
                            else
                                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8f16, xh), __builtin_bit_cast(v8f16, yh), acc[i][j], 0, 0, 0);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            read_buf = read_buf + 1 == NST ? 0 : read_buf + 1;
        };

        // NST - 1 steps are in flight; step s is awaited, everybody is then done with step s - 1, and its buffer takes step s + NST - 1
#pragma unroll
        for (int s = 0; s < NST - 1; ++s) {
            if (s + 1 < steps || (s + 1 == steps && !ragged)) issue_full();
            else issue_last(s + 1 > steps);
        }
        int s = 0;
        for (; s + NST < steps; ++s) {
            tile_wait<(NST - 2) * (LPW + SPW)>();
            issue_full();
            compute();
        }
        for (; s < steps; ++s) {
            tile_wait<(NST - 2) * (LPW + SPW)>();
            const int next = s + NST - 1;
            if (next + 1 == steps && !ragged) issue_full();
            else issue_last(next >= steps);
            if (!XT && !YT && s + 1 == steps && (last_bytes & 15) != 0) {
                // the end lies inside a piece
                for (int row = tid; row < ROWS; row += THREADS) {
                    v4i32* const at = reinterpret_cast<v4i32*>(lds + read_buf * STAGE_BYTES + row * STEP_BYTES + (((last_bytes >> 4) ^ ((row >> 1) & 7)) << 4));
                    *at = first_bytes(*at, last_bytes & 15);
                }
                tile_wait<(NST - 1) * (LPW + SPW)>();
            }
            compute();
        }
        tile_wait<0>();
    }
};

// The product of 256 X with 256 Y in eight waves, two to a SIMD, for large results: Tile's layout and arithmetic with another pipeline.
//
// Two steps' vectors fit into LDS (128 of its 160 KiB), and with one meeting per step a step's loads get no more than a step's time to arrive
// and all waves start a step together, with LDS reads and nothing to multiply.  Here a step's loads come in two parts, each asked for as
// soon as the part it replaces has been read and met one and a half steps later:
//     part 1: all of Y and rows 0 - 63 of each 128 of X (what rows 0 - 3 of a wave's tiles need), and the scales
//     part 2: rows 64 - 127 of each 128 of X.
// Rows of products 0 .. 7 of step s (each of FM tiles):
//     head of row 3: part 2 of step s has arrived; part 1 of s has been read: part 1 of s + 2 is asked for
//     head of row 7: part 1 of step s + 1 has arrived; part 2 of s has been read: part 2 of s + 2 is asked for
// X's fragments are read a row in front, across the end of the step; Y's fragment j of the next step in row 7, where the last product
// that reads it has been issued.  So no wave waits for LDS at a step's head.
// Whole steps are loaded with buffer instructions, whose addresses are 32-bit offsets of a lane and of the step: 256 accumulators of two waves
// leave no registers for 64-bit ones.
// FP8, 8192 x 8192 x 8192: 460 us, 2.39 PFLOP/s, the matrix unit busy 60 % of the cycles at 1.9 GHz; without loads and LDS reads it would be 3.2 PFLOP/s.
// BF16, 4096 x 65536 x 4096: 1.43 PFLOP/s, busy 74 %; 2.07 without.  Bound by the two together: LDS reads and scales hold up the issue.
template <int KIND, bool XT = false, bool YT = false, bool XP = false>
struct PairedTile {
    typedef Tile<KIND, 2, 4, 8, 4, 2, false, false, XP> Base;
    static constexpr bool PAIR = XP;
    static_assert(!XP || !XT, "");
    static constexpr bool FP8 = Base::FP8, BLOCKS = Base::BLOCKS;
    static_assert(!Base::WIDE, "registers");
    static constexpr int WN = 2, WM = 4, FN = 8, FM = 4, WAVES = 8, THREADS = 512, TN = 256, TM = 256, ROWS = 512;
    static constexpr int STAGE_BYTES = ROWS * STEP_BYTES, SCALE_BYTES = FP8 ? ROWS * 4 : 0, SCALE_RING = 3;
    static constexpr int LDS_BYTES = 2 * STAGE_BYTES + SCALE_RING * SCALE_BYTES;
    static_assert(LDS_BYTES >= Base::LDS_BYTES, "");
    static constexpr int P1 = 6, P2 = 2, S = FP8 ? 1 : 0;            // loads of a wave

    // Vectors that end inside a piece: their last step on its own, by Tile.  (Clearing the piece in the pipeline costs it a hundred registers.)
    __device__ static void multiply(uint8_t* lds, const TileOperand& X, const TileOperand& Y, int64_t bytes, int step0, int step1,
                                    v4f32 (&acc)[FN][FM]) {
        if constexpr (XT || YT) {                    // (a turned operand ends at a row)
            pipeline(lds, X, Y, bytes, step0, step1, acc);
            return;
        }
        const bool inside = (bytes & 15) != 0 && bytes < (int64_t)step1 * STEP_BYTES;
        const int whole = step1 - (inside ? 1 : 0);
        if (whole > step0) pipeline(lds, X, Y, bytes, step0, whole, acc);
        if (inside) Base::multiply(lds, offset(X, whole), offset(Y, whole), bytes - (int64_t)whole * STEP_BYTES, 0, 1, acc);
    }

    __device__ static TileOperand offset(const TileOperand& o, int step) {
        return TileOperand{o.vectors + (int64_t)step * STEP_BYTES, o.stride, o.rows, o.scales + (int64_t)step * o.scale_stride, o.scale_stride, 0,
                           XP ? o.second + (int64_t)step * STEP_BYTES : nullptr};
    }

    __device__ static void pipeline(uint8_t* lds, const TileOperand& X, const TileOperand& Y, int64_t bytes, int step0, int step1,
                                    v4f32 (&acc)[FN][FM]) {
        const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wn = wave / WM, wm = wave % WM;
        const int steps = step1 - step0;
        const int64_t rest = bytes - (int64_t)(step1 - 1) * STEP_BYTES;
        const int last_bytes = rest < STEP_BYTES ? (int)rest : STEP_BYTES;
        const bool ragged = last_bytes < STEP_BYTES;

        // Load i of a wave brings eight rows of the stage (X's 256, then Y's): Y for i < 4, X's of part 1 for i = 4, 5, of part 2 for i = 6, 7.
        const int y_first = TN + wave * 32, x_first = (wave >> 2) * 128 + (wave & 3) * 16;
        auto row_of = [&](int i) { return i < 4 ? y_first + 8 * i : x_first + (i < P1 ? 8 * (i - 4) : 64 + 8 * (i - P1)); };
        // (beyond `RECORDS` bytes these resources give zeros)
        constexpr unsigned RECORDS = 0x7FFFFFFFu;
        const __amdgpu_buffer_rsrc_t in_x = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(X.vectors), 0, RECORDS, 0x00027000);
        // (a pair's second matrix is part 2 of X: rows 64 - 127 of each 128)
        const __amdgpu_buffer_rsrc_t in_x2 = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(XP ? X.second : X.vectors), 0, RECORDS, 0x00027000);
        const __amdgpu_buffer_rsrc_t in_y = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(Y.vectors), 0, RECORDS, 0x00027000);
        // A turned operand's loads bring four rows of a panel of 128 vectors: of X, panel 0 is part 1 and panel 1 part 2.
        auto panel_load = [&](int i) { return i < 4 ? wave * 4 + i : (i < P1 ? wave * 2 + i - 4 : 16 + wave * 2 + i - P1); };
        auto element_of = [&](int i) { return (panel_load(i) & 15) * 4 + (lane >> 4); };
        unsigned voff[P1 + P2];
#pragma unroll
        for (int i = 0; i < P1 + P2; ++i) {
            const TileOperand& o = i < 4 ? Y : X;
            const int row = row_of(i) + (lane >> 3), mine = i < 4 ? row - TN : XP ? (row >> 7) * 64 + (row & 63) : row;
            voff[i] = (unsigned)(mine < o.rows ? mine : o.rows - 1) * (unsigned)o.stride + (((lane & 7) ^ ((row >> 1) & 7)) << 4);
            if (i < 4 ? YT : XT) {
                const int e = element_of(i), panel = panel_load(i) >> 4, c = (((lane & 15) >> 1) ^ turned_place(e)) * 16 + (lane & 1) * 8;
                const int v = i < 4 ? panel * 128 + c : (c >> 6) * 128 + panel * 64 + (c & 63);
                voff[i] = (unsigned)e * (unsigned)o.stride + 2 * (unsigned)(v < o.rows ? v : 0);
            }
        }
        // the scales of a wave's 64 rows of the stage
        const bool x_scales = wave < 4;
        unsigned soff = 0;
        if constexpr (FP8) {
            const int row = (wave & 3) * 64 + lane, rows = x_scales ? X.rows : Y.rows, real = row < rows ? row : rows - 1;
            soff = 4 * (unsigned)(x_scales && BLOCKS ? real / SCALE_BLOCK : real);
        }
        // load i of step `s`; `plain`: a whole step is there to be read; otherwise zeros come from behind the vectors' end
        auto load = [&](int i, int s, bool plain) {
            unsigned at = voff[i];
            const bool turned = i < 4 ? YT : XT;
            const TileOperand& o = i < 4 ? Y : X;
            if (!plain) {
                const int limit = s + 1 < steps ? STEP_BYTES : s + 1 == steps ? last_bytes : 0;
                const bool there = turned ? s < steps && (int64_t)(step0 + s) * 64 + element_of(i) < o.elements
                                          : (int)((lane & 7) ^ (((row_of(i) + (lane >> 3)) >> 1) & 7)) * 16 < limit;
                if (!there) at = RECORDS;
            }
            uint8_t* const to = lds + (s & 1) * STAGE_BYTES + (turned ? (i < 4 ? TN * STEP_BYTES : 0) + panel_load(i) * 1024 : row_of(i) * STEP_BYTES);
            if (turned) {
                // (a step is 64 rows on, which may pass 32 bits)
                direct_load(resource_of(o.vectors + (int64_t)(step0 + s) * 64 * o.stride, RECORDS), at, 0, to);
            } else if (XT || YT) {
                direct_load(resource_of(o.vectors, RECORDS), at, (step0 + s) * STEP_BYTES, to);
            } else {
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i < 4 ? in_y : XP && i >= P1 ? in_x2 : in_x, OZAKI_TILE_LPTR(to), 16, at, (step0 + s) * STEP_BYTES, 0, 0);
            }
        };
        int scale_to = 0, scale_at = 0;                               // places in the ring of scales
        auto load_scales = [&](int s, bool plain) {
            if constexpr (FP8) {
                const float* const block = x_scales ? X.scales + (int64_t)(step0 + s) * X.scale_stride : Y.scales + (int64_t)(step0 + s) * Y.scale_stride;
                const __amdgpu_buffer_rsrc_t in = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(block), 0, plain || s < steps ? RECORDS : 0, 0x00027000);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(in, OZAKI_TILE_LPTR(lds + 2 * STAGE_BYTES + scale_to * SCALE_BYTES + wave * 256), 4, soff, 0, 0, 0);
                scale_to = scale_to + 1 == SCALE_RING ? 0 : scale_to + 1;
            }
        };
        const int frow = lane & 15, g = lane >> 4, fsw = (frow >> 1) & 7;
        const int piece0 = (g ^ fsw) << 4, piece1 = ((g + 4) ^ fsw) << 4;
        const int xbase = (wn * FN * 16 + frow) * STEP_BYTES, ybase = (TN + wm * FM * 16 + frow) * STEP_BYTES;
        auto fragment = [&](int at, int s) -> v8i32 {
            const uint8_t* const p = lds + (s & 1) * STAGE_BYTES + at;
            const v4i32 lo = *reinterpret_cast<const v4i32*>(p + piece0), hi = *reinterpret_cast<const v4i32*>(p + piece1);
            return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        auto half = [](const v8i32& v, int h) {
            return h ? __builtin_shufflevector(v, v, 4, 5, 6, 7) : __builtin_shufflevector(v, v, 0, 1, 2, 3);
        };
        // fragment i of this wave's rows of X, j of its rows of Y, in step s
        auto x_fragment = [&](int i, int s) -> v8i32 {
            if constexpr (XT) return turned_fragment(lds + (s & 1) * STAGE_BYTES + (i >> 2) * PANEL_BYTES, wn * 4 + (i & 3), lane);
            else return fragment(xbase + i * 16 * STEP_BYTES, s);
        };
        auto y_fragment = [&](int j, int s) -> v8i32 {
            if constexpr (YT) return turned_fragment(lds + (s & 1) * STAGE_BYTES + TN * STEP_BYTES + (wm >> 1) * PANEL_BYTES, (wm & 1) * 4 + j, lane);
            else return fragment(ybase + j * 16 * STEP_BYTES, s);
        };
        v8i32 y[FM], x[2];

        // in front of step 0: all four parts of two steps
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const bool plain = s + 1 < steps || (s + 1 == steps && !ragged);
#pragma unroll
            for (int i = 0; i < P1; ++i) load(i, s, plain);
            load_scales(s, plain);
#pragma unroll
            for (int i = P1; i < P1 + P2; ++i) load(i, s, plain);
        }
        tile_wait<P2 + P1 + S + P2>();
#pragma unroll
        for (int j = 0; j < FM; ++j) y[j] = y_fragment(j, 0);
        x[0] = x_fragment(0, 0);

        // one step; `plain`: the loads that it asks for are of whole steps, and there is a next one
        auto step = [&](int s, auto plain_c) {
            constexpr bool PLAIN = decltype(plain_c)::value;
            const bool full = PLAIN || s + 3 < steps || (s + 3 == steps && !ragged);
            const float* const scales = reinterpret_cast<const float*>(lds + 2 * STAGE_BYTES + scale_at * SCALE_BYTES);
            scale_at = scale_at + 1 == SCALE_RING ? 0 : scale_at + 1;
            constexpr int LAG = !FP8 ? 0 : BLOCKS ? 3 : 2;
            float sy[FM], sx_all = 0.0f;
            v4f32 t[LAG + 1], sx[2] = {};
            if constexpr (FP8) {
#pragma unroll
                for (int j = 0; j < FM; ++j) sy[j] = scales[TN + (wm * FM + j) * 16 + frow];
                if constexpr (BLOCKS) sx_all = scales[wn * FN * 16];
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < FN * FM + LAG; ++n) {
                const int i = n / FM, j = n % FM;
                if (n < FN * FM) {
                    if (j == 0 && i == 3) tile_wait<P1 + S + P2>();
                    if (j == 0 && i == 7) tile_wait<P2 + P1 + S>();
                    // (behind the last step these read what is there and nobody uses)
                    if (j == 0) x[(i + 1) & 1] = x_fragment((i + 1) % FN, i + 1 < FN ? s : s + 1);
                    if (FP8 && !BLOCKS && j == 0) sx[i & 1] = *reinterpret_cast<const v4f32*>(scales + (wn * FN + i) * 16 + 4 * g);
                    const v8i32 xi = x[i & 1];
                    if constexpr (FP8) {
                        t[n % (LAG + 1)] = Fragment<false>::product(xi, y[j]);
                    } else {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            if constexpr (KIND == KIND_BF16)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf16, half(xi, h)), __builtin_bit_cast(v8bf16, half(y[j], h)), acc[i][j], 0, 0, 0);
                            else
                                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8f16, half(xi, h)), __builtin_bit_cast(v8f16, half(y[j], h)), acc[i][j], 0, 0, 0);
                        }
                    }
                    if (i == FN - 1) y[j] = y_fragment(j, s + 1);
                    // the loads, one behind a product
                    const int l = n - 3 * FM;
                    if (l >= 0 && l < P1) load(l, s + 2, PLAIN || full);
                    if (l == P1) load_scales(s + 2, PLAIN || full);
                    if (n >= 7 * FM && n < 7 * FM + P2) load(P1 + n - 7 * FM, s + 2, PLAIN || full);
                }
                if (BLOCKS && n == LAG) {
#pragma unroll
                    for (int q = 0; q < FM; ++q) sy[q] *= sx_all;
                }
                if (FP8 && n >= LAG) {
                    const int d = n - LAG, di = d / FM, dj = d % FM;
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[di][dj][r] = __builtin_fmaf(t[d % (LAG + 1)][r], BLOCKS ? sy[dj] : sx[di & 1][r] * sy[dj], acc[di][dj][r]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        const std::integral_constant<bool, true> plain;
        const std::integral_constant<bool, false> checked;
        int s = 0;
        for (; s + 4 < steps; s += 2) {
            step(s, plain);
            step(s + 1, plain);
        }
        for (; s < steps; ++s) step(s, checked);
        tile_wait<0>();
    }
};

// Stores the tile that P::multiply has left, times factor(row of D) and (accumulate) on top of what D holds, D being its first element: `left_m` rows
// and `left_n` columns of it are there.  A lane has four neighbouring columns of sixteen rows; through LDS, 16 rows of every wave at a time
// in 32 bits, D's rows are written in whole 16-byte pieces of neighbouring lanes.  Rows of D that are not aligned to that are written by element.
// STREAMED: results of the large shapes, more than the L2 caches hold (FP8, 4096 x 4096 x 256 19.3 -> 17.0 us, 8192 x 8192 x 4096 252 -> 244).
// place(row): which row of D it becomes.
struct SameRow {
    __device__ __forceinline__ int64_t operator()(int64_t m) const { return m; }
};
template <typename P, bool STREAMED, typename T, typename F, typename R = SameRow>
__device__ __forceinline__ void store_tile(uint8_t* lds, const v4f32 (&acc)[P::FN][P::FM], T* D, int64_t ldd, int64_t left_m, int64_t left_n,
                                           bool accumulate, F factor, R place = R()) {
    constexpr int STRIDE = P::TN * 4 + 16, PER = 16 / sizeof(T), PIECES = P::TN / PER, ROWS = P::WM * 16;
    static_assert(ROWS * STRIDE <= P::LDS_BYTES && P::THREADS % PIECES == 0 && P::THREADS % P::TN == 0, "");
    typedef T piece __attribute__((ext_vector_type(PER)));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wn = wave / P::WM, wm = wave % P::WM;
    const int columns = left_n < P::TN ? (int)left_n : P::TN;
    const bool wide = ldd % PER == 0 && reinterpret_cast<uintptr_t>(D) % 16 == 0;
    const int whole = wide ? columns / PER * PER : 0, loose = columns - whole;
#pragma unroll
    for (int j = 0; j < P::FM; ++j) {
        uint8_t* const mine = lds + (wm * 16 + (lane & 15)) * STRIDE + (wn * P::FN * 16 + 4 * (lane >> 4)) * 4;
#pragma unroll
        for (int i = 0; i < P::FN; ++i) *reinterpret_cast<v4f32*>(mine + i * 64) = acc[i][j];
        __syncthreads();
        const int column = threadIdx.x % PIECES * PER;
        if (column < whole) {
#pragma unroll 2
            for (int r = threadIdx.x / PIECES; r < ROWS; r += P::THREADS / PIECES) {
                const int64_t m = ((r >> 4) * P::FM + j) * 16 + (r & 15);
                if (m >= left_m) continue;
                const float* const from = reinterpret_cast<const float*>(lds + r * STRIDE) + column;
                piece* const to = reinterpret_cast<piece*>(D + place(m) * ldd + column);
                const float f = factor(m);
                piece v = {};
                if (accumulate) v = *to;
#pragma unroll
                for (int q = 0; q < PER; ++q) v[q] = (T)(accumulate ? (float)v[q] + from[q] * f : from[q] * f);
                if constexpr (STREAMED) __builtin_nontemporal_store(v, to);
                else *to = v;
            }
        }
        // what is left, a thread a column (all of them where D's rows are not aligned)
        if (loose > 0) {
            constexpr int AT_ONCE = P::THREADS / P::TN;
            const int c = whole + threadIdx.x % P::TN;
            if (c < columns) {
#pragma unroll 4
                for (int r = threadIdx.x / P::TN; r < ROWS; r += AT_ONCE) {
                    const int64_t m = ((r >> 4) * P::FM + j) * 16 + (r & 15);
                    if (m >= left_m) continue;
                    const float v = reinterpret_cast<const float*>(lds + r * STRIDE)[c] * factor(m);
                    T* const to = D + place(m) * ldd + c;
                    *to = (T)(accumulate ? (float)*to + v : v);
                }
            }
        }
        __syncthreads();
    }
}

}  // namespace
}  // namespace ozaki
