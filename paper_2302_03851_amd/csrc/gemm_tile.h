// Matrix product C = A B on the matrix cores, fp32 or bf16 operands in any
// layout, stride and alignment, fp32 sums.
//
// A work-group owns a TM x TN tile of C.  Every thread loads pieces of 8
// elements of both operands into registers a step ahead, and writes them to
// LDS as bf16:
//   * bf16 as it is, 64 k a step;
//   * fp32 as three bf16 values that add up to it to the last bit (8 + 8 + 8
//     significant bits), 32 k a step.  Of the nine products the six largest are
//     formed, which leaves out less than 2^-24 of a term; they take 6/16 of the
//     time of the fp32 matrix instructions.  (The last piece is a multiple of
//     2^-133, bf16's least number: factors below 2^-109 lose digits.  First pieces
//     are rounded up by 2^-8 of them at most, and their product by 2^-7: it may
//     leave fp32's range where the term does not.)
// v_mfma_f32_16x16x32_bf16 wants 8 consecutive k of one row (or column) a lane.
// An operand whose k are contiguous in memory (K_LINES) is kept line by line and
// read 16 bytes at a time; one whose rows (columns) are (MN_LINES) is kept as it
// is, k by k, and turned by ds_read_b64_tr_b16, which hands a lane 4 k of its
// column.  Both are permuted within LDS so that no read meets its own banks.
//
// The products are formed as B^T A^T, so that a lane holds 4 neighbouring
// columns of a row of C; each wave passes its sums through LDS once more, to be
// finished (bias, activation, residual) and written by whole pieces of rows.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "row_access.h"

namespace edb {
namespace gemm {

using namespace edb::rows;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));

enum Layout { K_LINES, MN_LINES };

template <class T>
struct Kind;
template <>
struct Kind<bf16> {
    static constexpr int kPlanes = 1, kDepth = 64, kStages = 2;
};
template <>
struct Kind<float> {
    static constexpr int kPlanes = 3, kDepth = 32, kStages = 1;
};

// ---- activations ------------------------------------------------------------
//
// On the hardware's exponential and reciprocal (1 unit in the last place each);
// with the library's erfc, exp and tanh a layer of 28629 x 512 x 1536 took twice
// as long.  Infinities give the limits, NaN stays NaN.

constexpr float kLog2e = 1.4426950408889634f;

// 2^x for x <= 0 as e times scale, so that what is multiplied with it before
// `scale` keeps its digits where 2^x itself is below the normal numbers.
struct Power {
    float e, scale;
    __device__ __forceinline__ explicit Power(float x) {
        const bool far = x < -100.f;
        e = __builtin_amdgcn_exp2f(far ? x + 64.f : x);
        scale = far ? 0x1p-64f : 1.f;
    }
};

// erfc(z) exp(z^2) / 2 of z = a / sqrt(2) >= 0, as t Q(t) with t = 1 / (1 + z / 2)
// and Q fitted for the least largest relative error up to z = 10.6 (6.0e-8; in
// fp32 3.2e-7).
__device__ __forceinline__ float tail(float a) {
    const float t = __builtin_amdgcn_rcpf(fmaf(a, 0.35355339059327376f, 1.f));
    float q = -0.029606621712446213f;
    q = fmaf(q, t, 0.14263999462127686f);
    q = fmaf(q, t, -0.2443310022354126f);
    q = fmaf(q, t, 0.13987129926681519f);
    q = fmaf(q, t, -0.013890879228711128f);
    q = fmaf(q, t, 0.1015884131193161f);
    q = fmaf(q, t, 0.12148986756801605f);
    q = fmaf(q, t, 0.14119619131088257f);
    q = fmaf(q, t, 0.14104272425174713f);
    return q * t;
}

__device__ __forceinline__ float relu(float v) { return v < 0.f ? 0.f : v; }

// v Phi(v) = max(v, 0) - |v| Phi(-|v|)
__device__ __forceinline__ float gelu(float v) {
    const float a = fminf(fabsf(v), 20.f);
    return relu(v) - a * (__builtin_amdgcn_exp2f(-0.5f * kLog2e * (a * a)) * tail(a));
}
__device__ __forceinline__ float gelu_slope(float v) {
    const float a = fminf(fabsf(v), 20.f);
    const Power p(-0.5f * kLog2e * (a * a));
    // Phi(-a) and a phi(a)
    const float beyond = p.e * tail(a), bent = p.e * a * 0.39894228040143268f;
    return v != v ? v : v < 0.f ? (beyond - bent) * p.scale : 1.f - (beyond - bent) * p.scale;
}

__device__ __forceinline__ float silu(float v) {
    const float a = fminf(fabsf(v), 200.f);
    const Power p(-kLog2e * a);
    const float r = __builtin_amdgcn_rcpf(1.f + p.e * p.scale);
    return v < 0.f ? -(a * r * p.e) * p.scale : v * r;
}
__device__ __forceinline__ float silu_slope(float v) {
    const float a = fminf(fabsf(v), 200.f);
    const Power p(-kLog2e * a);
    const float r = __builtin_amdgcn_rcpf(1.f + p.e * p.scale);
    // s (1 + v (1 - s)) with s = r or e r, 1 - s the other one
    return v != v ? v : v < 0.f ? p.e * r * (1.f - a * r) * p.scale : r * fmaf(a * r * p.e, p.scale, 1.f);
}

// By (1 - e) / (1 + e), e = exp(-2 |v|), and next to 0 by v + v^3 P(v^2), P
// fitted for the least largest relative error (1.5e-7 of P).
__device__ __forceinline__ float tanh_of(float v) {
    const float a = fabsf(v), s = v * v;
    float p = -0.006045394577085972f;
    p = fmaf(p, s, 0.020961513742804527f);
    p = fmaf(p, s, -0.05384330824017525f);
    p = fmaf(p, s, 0.1333271861076355f);
    p = fmaf(p, s, -0.333333283662796f);
    const float e = __builtin_amdgcn_exp2f(-2.f * kLog2e * a);
    const float far = (1.f - e) * __builtin_amdgcn_rcpf(1.f + e);
    return a < 0.63f ? fmaf(v * s, p, v) : copysignf(far, v);
}
// 1 / cosh^2: keeps its digits where tanh is next to 1
__device__ __forceinline__ float tanh_slope(float v) {
    const Power p(-2.f * kLog2e * fabsf(v));
    const float r = __builtin_amdgcn_rcpf(1.f + p.e * p.scale);
    return 4.f * p.e * r * r * p.scale;
}

template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N]) {
#define EDB_EACH(f)               \
    _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = f(v[i])
    if (act == EDB_ACT_RELU) {
        EDB_EACH(relu);
    } else if (act == EDB_ACT_GELU) {
        EDB_EACH(gelu);
    } else if (act == EDB_ACT_SILU) {
        EDB_EACH(silu);
    } else if (act == EDB_ACT_TANH) {
        EDB_EACH(tanh_of);
    }
}
// x times the derivative at v
__device__ __forceinline__ void slope8(int act, const float (&v)[8], float (&x)[8]) {
#define EDB_TIMES(f)              \
    _Pragma("unroll") for (int i = 0; i < 8; ++i) x[i] *= f
    if (act == EDB_ACT_RELU) {
        EDB_TIMES((v[i] > 0.f ? 1.f : v[i] != v[i] ? v[i] : 0.f));
    } else if (act == EDB_ACT_GELU) {
        EDB_TIMES(gelu_slope(v[i]));
    } else if (act == EDB_ACT_SILU) {
        EDB_TIMES(silu_slope(v[i]));
    } else if (act == EDB_ACT_TANH) {
        EDB_TIMES(tanh_slope(v[i]));
    }
}
#undef EDB_EACH
#undef EDB_TIMES

// ---- what becomes of a sum ---------------------------------------------------

struct Finish {
    const void* bias;        // or NULL
    const void* residual;    // or NULL
    int64_t residual_stride;
    void* out;
    int64_t out_stride;
    void* pre;               // the sums with the bias, before the activation; or NULL
    int64_t pre_stride;
    int32_t act;
    bool bias_bf16, residual_bf16, out_bf16, pre_bf16;
};

__device__ __forceinline__ void load8(const void* p, bool half, int64_t at, float (&v)[8]) {
    if (half) load_k<bf16, 8>(static_cast<const bf16*>(p) + at, v);
    else load_k<float, 8>(static_cast<const float*>(p) + at, v);
}
__device__ __forceinline__ void store8(void* p, bool half, int64_t at, const float (&v)[8]) {
    if (half) store_k<bf16, 8>(static_cast<bf16*>(p) + at, v);
    else store_k<float, 8>(static_cast<float*>(p) + at, v);
}
__device__ __forceinline__ float load1(const void* p, bool half, int64_t at) {
    return half ? Elem<bf16>::get(static_cast<const bf16*>(p) + at) : static_cast<const float*>(p)[at];
}
__device__ __forceinline__ void store1(void* p, bool half, int64_t at, float v) {
    if (half) Elem<bf16>::put(static_cast<bf16*>(p) + at, v);
    else static_cast<float*>(p)[at] = v;
}

// 8 elements as they lie in memory.
struct Raw8 {
    u32x4 w[2];
    __device__ __forceinline__ void load(const void* p, bool half, int64_t at) {
        if (half) {
            w[0] = Elem<bf16>::load(static_cast<const bf16*>(p) + at);
        } else {
            w[0] = Elem<float>::load(static_cast<const float*>(p) + at);
            w[1] = Elem<float>::load(static_cast<const float*>(p) + at + 4);
        }
    }
    __device__ __forceinline__ void add_to(bool half, float (&v)[8]) const {
        float t[8];
        if (half) {
            Elem<bf16>::unpack(w[0], t);
        } else {
            Elem<float>::unpack(w[0], t);
            Elem<float>::unpack(w[1], t + 4);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += t[i];
    }
};

// Of the 8 columns from col, `left` are the matrix's.
__device__ __forceinline__ void load_bias(const Finish& f, int col, int left, float (&b)[8]) {
    if (!f.bias) return;
    if (left >= 8) {
        load8(f.bias, f.bias_bf16, col, b);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < left) b[i] = load1(f.bias, f.bias_bf16, col + i);
    }
}

// 8 columns of a row of sums with the bias; more: the residual's.
__device__ __forceinline__ void finish8(const Finish& f, int64_t row, int col, float (&v)[8], const Raw8& more) {
    if (f.pre) store8(f.pre, f.pre_bf16, row * f.pre_stride + col, v);
    activate(f.act, v);
    if (f.residual) more.add_to(f.residual_bf16, v);
    store8(f.out, f.out_bf16, row * f.out_stride + col, v);
}

// Up to 8 columns one by one.
template <int N>
__device__ __forceinline__ void finish_edge(const Finish& f, int64_t row, int col, int left, float (&v)[N]) {
    if (f.pre) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < left) store1(f.pre, f.pre_bf16, row * f.pre_stride + col + i, v[i]);
    }
    activate(f.act, v);
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < left) {
            if (f.residual) v[i] += load1(f.residual, f.residual_bf16, row * f.residual_stride + col + i);
            store1(f.out, f.out_bf16, row * f.out_stride + col + i, v[i]);
        }
}

// ---- operands ------------------------------------------------------------------

// The three pieces of 8 fp32 values, each rounded to nearest.  A value whose
// first piece would round to infinity takes the largest finite one; an infinity
// goes into the last piece, beside a first piece of its sign: its products are
// then with the other operand's first piece, which is zero for zeros only.  A
// NaN is one in its pieces.
__device__ __forceinline__ void split8(const u32x4 (&raw)[2], u32x4 (&o)[3]) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __builtin_bit_cast(float, (uint32_t)raw[i >> 2][i & 3]);
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) asm("v_max3_f32 %0, |%1|, |%2|, %0" : "+v"(most) : "v"(x[i]), "v"(x[i + 1]));
    constexpr float kLargest = 0x1.FEp127f;   // of the bf16 values
    const bool far = most > kLargest;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a = x[2 * i], b = x[2 * i + 1];
        if (__builtin_expect(far, 0)) {
            v2f p[3];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float v = j ? b : a;
                const bool inf = fabsf(v) == INFINITY;
                const float hi = inf ? copysignf(1.f, v) : fabsf(v) > kLargest ? copysignf(kLargest, v) : (float)static_cast<__bf16>(v);
                const float mid = inf ? 0.f : (float)static_cast<__bf16>(v - hi);
                p[0][j] = hi;
                p[1][j] = mid;
                p[2][j] = inf ? v : v - hi - mid;
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) o[k][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p[k], v2bf));
        } else {
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                const uint32_t u = __builtin_bit_cast(uint32_t, __builtin_convertvector((v2f{a, b}), v2bf));
                o[k][i] = u;
                a -= __builtin_bit_cast(float, u << 16);
                b -= __builtin_bit_cast(float, u & 0xFFFF0000u);
            }
        }
    }
}

// A tile's operand: R rows (columns) by kDepth k a step, by NT threads.
template <class T, Layout L, int R, int NT>
struct Operand {
    static constexpr int BK = Kind<T>::kDepth, P = Kind<T>::kPlanes;
    static constexpr int NP = (L == K_LINES ? BK : R) / 8;       // pieces of a line
    static constexpr int PIECES = R * BK / 8, PER = (PIECES + NT - 1) / NT;
    static constexpr int PLANE = R * BK * 2;                     // bytes of one plane
    static constexpr int WORDS = sizeof(T) / 2;                  // 16-byte words of a piece in memory

    const T* p[PER];
    u32x4 raw[PER][WORDS];
    int64_t step;

    static __device__ __forceinline__ int index(int j) { return min((int)threadIdx.x + j * NT, PIECES - 1); }

    // mn0: the tile's first row (column) of mn; k0: the first k.
    __device__ __forceinline__ void start(const T* base, int64_t stride, int mn0, int mn, int k0) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int line = index(j) / NP, q = index(j) % NP * 8;
            // rows (columns) past the end: the last one again, whose results nobody writes
            p[j] = L == K_LINES ? base + (int64_t)min(mn0 + line, mn - 1) * stride + k0 + q
                                : base + (int64_t)(k0 + line) * stride + min(mn0 + q, mn - 1);
        }
        step = L == K_LINES ? BK : BK * stride;
    }
    __device__ __forceinline__ void load() {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) raw[j][i] = Elem<T>::load(p[j] + i * Elem<T>::kVec);
            p[j] += step;
        }
    }
    // The same where the step leaves the k before kend or the tile the matrix: zeros from there on.
    __device__ __forceinline__ void load_edge(int mn0, int mn, int k0, int kend) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int line = index(j) / NP, q = index(j) % NP * 8;
            const int left = L == K_LINES ? kend - (k0 + q) : k0 + line < kend ? mn - (mn0 + q) : 0;
            if (left >= 8) {
#pragma unroll
                for (int i = 0; i < WORDS; ++i) raw[j][i] = Elem<T>::load(p[j] + i * Elem<T>::kVec);
            } else {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = i < left ? Elem<T>::get(p[j] + i) : 0.f;
#pragma unroll
                for (int i = 0; i < WORDS; ++i) raw[j][i] = Elem<T>::pack(v + i * Elem<T>::kVec);
            }
            p[j] += step;
        }
    }
    // Adds the pieces up (MN_LINES: all of a thread's are of the same 8 columns).
    __device__ __forceinline__ void add_to(float (&sum)[8]) const {
        static_assert(L == MN_LINES && NT % NP == 0, "a thread keeps its columns");
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            float v[8];
#pragma unroll
            for (int i = 0; i < WORDS; ++i) Elem<T>::unpack(raw[j][i], v + i * Elem<T>::kVec);
            if (PIECES % NT && (int)threadIdx.x + j * NT >= PIECES) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += v[i];
        }
    }
    // The columns' sums over the threads, through LDS of NT x 32 bytes; the caller's barriers are around it.
    static __device__ __forceinline__ void sums_out(const float (&sum)[8], float* lds, float* out, int mn0, int mn) {
#pragma unroll
        for (int i = 0; i < 8; ++i) lds[i * NT + threadIdx.x] = sum[i];
        __syncthreads();
        const int c = threadIdx.x;
        if (c >= R || mn0 + c >= mn) return;
        float s = 0.f;
        for (int t = c >> 3; t < NT; t += NP) s += lds[(c & 7) * NT + t];
        out[mn0 + c] = s;
    }
    // Byte offset of a piece in a plane.
    static __device__ __forceinline__ int place(int line, int q) {
        // 16 lines of one q, and the lines that the hardware reads in one go from two q, keep to different banks
        if constexpr (L == K_LINES) return line * BK * 2 + 16 * (q ^ ((BK == 64 ? line >> 1 : -(line >> 2)) & (NP - 1)));
        else return line * R * 2 + 32 * ((q >> 1) ^ turn(line)) + 16 * (q & 1);
    }
    // Where the 32-byte blocks of line k go: the 8 lines that two groups of 16
    // lanes read at once (k = 8 g + 0..3) are kept in different banks.
    static __device__ __forceinline__ int turn(int k) {
        constexpr int NB = R / 16;
        if constexpr (NB >= 8) return (k & 3) | (k >> 1 & 4);
        else if constexpr (NB == 4) return (k >> 1 & 1) | (k >> 2 & 2);
        else if constexpr (NB == 2) return k >> 3 & 1;
        else return 0;
    }
    __device__ __forceinline__ void store(char* lds) const {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int at = place(index(j) / NP, index(j) % NP);
            if constexpr (P == 1) {
                *reinterpret_cast<u32x4*>(lds + at) = raw[j][0];
            } else {
                u32x4 o[3];
                split8(raw[j], o);
#pragma unroll
                for (int k = 0; k < 3; ++k) *reinterpret_cast<u32x4*>(lds + k * PLANE + at) = o[k];
            }
        }
    }
    // The 16 rows (columns) from r0, k = 32 kk + 8 (lane / 16) + 0..7.
    static __device__ __forceinline__ v8bf fragment(const char* plane, int r0, int kk, int lane) {
        if constexpr (L == K_LINES) {
            return __builtin_bit_cast(v8bf, *reinterpret_cast<const u32x4*>(plane + place(r0 + (lane & 15), kk * 4 + (lane >> 4))));
        } else {
            v4s h[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = kk * 32 + (lane >> 4) * 8 + i * 4 + ((lane & 15) >> 2);
                const char* at = plane + k * R * 2 + 32 * ((r0 >> 4) ^ turn(k)) + (lane & 3) * 8;
                h[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)at);
            }
            return __builtin_bit_cast(v8bf, __builtin_shufflevector(h[0], h[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
    }
};

struct Args {
    const void *a, *b;
    int64_t a_stride, b_stride;
    int32_t m, n, k;            // C is m x n
    int32_t splits, k_per;      // k of a split (a multiple of the step's depth)
    float* partial;             // splits > 1: [split][m][n rounded up to 8]
    // both operands MN_LINES: sums over k of A's rows (1) or B's columns (2) besides, [split][m or n]
    int32_t sums;
    float* sums_out;
    Finish finish;
};

template <class T, Layout AL, Layout BL, int TM, int TN, int WM, int WN>
struct Shape {
    static constexpr int NT = 64 * WM * WN;
    typedef Operand<T, AL, TM, NT> A;
    typedef Operand<T, BL, TN, NT> B;
    static constexpr int STAGE = Kind<T>::kPlanes * (A::PLANE + B::PLANE);
    static constexpr int ROWS = TM / WM, COLS = TN / WN;         // of a wave
    static constexpr int OUT = ROWS >= 32 ? 2 : 1;               // blocks of 16 rows on their way out
    static constexpr int PITCH = COLS + 4;                       // floats of a row there
    static constexpr int IN = Kind<T>::kStages * STAGE, WAY = WM * WN * OUT * 16 * PITCH * 4;
    static constexpr int LDS = IN > WAY ? IN : WAY;
};

// Bound by what a compute unit's waves wait for each other: 8192^3 bf16 907 us
// (1212 TFLOP/s; a library product, in turn with it, 668), the matrix cores busy 60%
// of it, LDS 40%, without bank conflicts; with 128 x 128 tiles, whose operands pass
// through LDS half as often again, 1165.  fp32 4096^3 683 us (201 TFLOP/s of fp32; a
// library product 922), where splitting the operands takes the vector units half as long
// as the products take the matrix cores and two work-groups of a unit overlap
// the two only in part.  B by its columns (MN_LINES) from row-major memory takes
// 6% longer than by K_LINES (8192^3 964 us; a library product 770): twice the LDS reads.
template <class T, Layout AL, Layout BL, int TM, int TN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 2) void gemm_kernel(Args g) {
    using S = Shape<T, AL, BL, TM, TN, WM, WN>;
    using A = typename S::A;
    using B = typename S::B;
    constexpr int P = Kind<T>::kPlanes, BK = Kind<T>::kDepth, STAGES = Kind<T>::kStages;
    constexpr int FM = S::ROWS / 16, FN = S::COLS / 16;
    __shared__ __align__(16) char lds[S::LDS];

    // Work-groups go round the 8 XCDs in turn; each XCD takes a run of tiles, by
    // bands of 8 tile rows, so that what runs on it at once shares operands in its L2.
    const int mt = (g.m + TM - 1) / TM, nt = (g.n + TN - 1) / TN, tiles = mt * nt, all = tiles * g.splits;
    const int per = (all + 7) / 8, id = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if (id >= all) return;
    constexpr int kBand = 8;
    const int split = id / tiles, t = id % tiles, band = t / (kBand * nt), rest = t % (kBand * nt);
    const int high = min(kBand, mt - band * kBand);
    const int m0 = (band * kBand + rest % high) * TM, n0 = rest / high * TN;

    const int kbeg = split * g.k_per, kend = min(kbeg + g.k_per, g.k);
    const int steps = (kend - kbeg + BK - 1) / BK;
    // a piece that leaves its line's end (MN_LINES) reads on in the next line, if there is one: up to k_fast
    const bool inside = (AL == K_LINES || m0 + TM <= g.m) && (BL == K_LINES || n0 + TN <= g.n);
    const bool longer = (AL == K_LINES || g.a_stride >= 8) && (BL == K_LINES || g.b_stride >= 8);
    const int k_fast = inside ? kend : longer ? min(kend, g.k - 1) : 0;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN * S::ROWS, wn = wave % WN * S::COLS;

    A a;
    B b;
    a.start(static_cast<const T*>(g.a), g.a_stride, m0, g.m, kbeg);
    b.start(static_cast<const T*>(g.b), g.b_stride, n0, g.n, kbeg);
    auto load = [&](int s) {
        const int k0 = kbeg + s * BK;
        if (k0 + BK <= k_fast) {
            a.load();
            b.load();
        } else {
            a.load_edge(m0, g.m, k0, kend);
            b.load_edge(n0, g.n, k0, kend);
        }
    };
    // the sums, in registers, by the work-groups of the first tiles across; every kFold
    // steps they go on in other registers, so that long ones are no chains of additions
    // (262144 numbers of one sign, of the worst size: 1968 units off in one chain, 46 so)
    constexpr int kFold = 64;
    constexpr bool SUMS = AL == MN_LINES && BL == MN_LINES;
    const int sums = SUMS && (g.sums == 1 ? n0 == 0 : m0 == 0) ? g.sums : 0;
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, folded[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto store = [&](char* stage, int step) {
        if constexpr (SUMS) {
            if (sums == 1) a.add_to(sum);
        }
        a.store(stage);
        if constexpr (SUMS) {
            if (sums == 2) b.add_to(sum);
        }
        b.store(stage + P * A::PLANE);
        if constexpr (SUMS) {
            if (sums && (step & (kFold - 1)) == kFold - 1) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    folded[i] += sum[i];
                    sum[i] = 0.f;
                }
            }
        }
    };

    v4f acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = v4f{0.f, 0.f, 0.f, 0.f};
    auto compute = [&](const char* stage) {
        const char* as = stage;
        const char* bs = stage + P * A::PLANE;
#pragma unroll
        for (int kk = 0; kk < BK / 32; ++kk) {
            v8bf bf[P][FN];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int j = 0; j < FN; ++j) bf[p][j] = B::fragment(bs + p * B::PLANE, wn + j * 16, kk, lane);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                v8bf af[P];
#pragma unroll
                for (int p = 0; p < P; ++p) af[p] = A::fragment(as + p * A::PLANE, wm + i * 16, kk, lane);
                // smallest products first
#pragma unroll
                for (int o = P - 1; o >= 0; --o)
#pragma unroll
                    for (int p = 0; p <= o; ++p)
#pragma unroll
                        for (int j = 0; j < FN; ++j)
                            acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bf[o - p][j], af[p], acc[i][j], 0, 0, 0);
            }
        }
    };

    // Two stages: while a step is multiplied from one, the next is written to the
    // other and the one after it is on its way into registers.
    if (steps > 0) load(0);
    if constexpr (STAGES == 2) {
        if (steps > 0) store(lds, 0);
        if (steps > 1) load(1);
        __syncthreads();
        for (int s = 0; s < steps; ++s) {
            if (s + 1 < steps) store(lds + (~s & 1) * S::STAGE, s + 1);
            if (s + 2 < steps) load(s + 2);
            compute(lds + (s & 1) * S::STAGE);
            __syncthreads();
        }
    } else {
        for (int s = 0; s < steps; ++s) {
            store(lds, s);
            __syncthreads();
            if (s + 1 < steps) load(s + 1);
            compute(lds);
            __syncthreads();
        }
    }

    if constexpr (SUMS) {
        if (sums) {
            float* to = g.sums_out + (int64_t)split * (sums == 1 ? g.m : g.n);
            float* scratch = reinterpret_cast<float*>(lds);
            static_assert(S::LDS >= S::NT * 32, "room for the sums");
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += folded[i];
            if (sums == 1) A::sums_out(sum, scratch, to, m0, g.m);
            else B::sums_out(sum, scratch, to, n0, g.n);
            __syncthreads();
        }
    }

    // out: every wave passes OUT blocks of 16 rows at a time through its own
    // part of the LDS and finishes them by pieces of rows, AT a lane; the residual's
    // are loaded a turn ahead.  The turns are not unrolled: they are long code.
    constexpr int OUT = S::OUT, ROWS = OUT * 16, ACROSS = S::COLS / 8, DOWN = 64 / ACROSS, AT = ROWS / DOWN;
    float* buf = reinterpret_cast<float*>(lds) + wave * ROWS * S::PITCH;
    const Finish& f = g.finish;
    const int np = (g.n + 7) / 8 * 8, col = n0 + wn + lane % ACROSS * 8;
    const bool whole = col + 8 <= g.n;
    float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (g.splits == 1 && col < g.n) load_bias(f, col, g.n - col, bias);
    Raw8 more[AT], next[AT];
    auto load_more = [&](int part, Raw8 (&to)[AT]) {
        if (!f.residual || !whole || g.splits > 1) return;
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            const int row = m0 + wm + part * ROWS + i * DOWN + lane / ACROSS;
            if (row < g.m) to[i].load(f.residual, f.residual_bf16, row * f.residual_stride + col);
        }
    };
    load_more(0, next);
#pragma unroll 1
    for (int part = 0; part < FM / OUT; ++part) {
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            if (i / OUT != part) continue;
#pragma unroll
            for (int j = 0; j < FN; ++j)
                *reinterpret_cast<v4f*>(buf + (i % OUT * 16 + (lane & 15)) * S::PITCH + j * 16 + (lane >> 4) * 4) = acc[i][j];
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < AT; ++i) more[i] = next[i];
        if (part + 1 < FM / OUT) load_more(part + 1, next);
#pragma unroll
        for (int i = 0; i < AT; ++i) {
            const int r = i * DOWN + lane / ACROSS;
            const int64_t row = m0 + wm + part * ROWS + r;
            const v4f* q = reinterpret_cast<const v4f*>(buf + r * S::PITCH + lane % ACROSS * 8);
            if (row < g.m && col < g.n) {
                if (g.splits > 1) {
                    v4f* to = reinterpret_cast<v4f*>(g.partial + ((int64_t)split * g.m + row) * np + col);
                    to[0] = q[0];
                    to[1] = q[1];
                } else {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = q[e >> 2][e & 3] + bias[e];
                    if (whole) finish8(f, row, col, v, more[i]);
                    else finish_edge(f, row, col, g.n - col, v);
                }
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// The splits' sums, finished: a thread takes 8 columns of a row, of every
// SHARES-th split, and the shares are added through LDS, so that few pieces of
// many splits fill the card too.
template <int SHARES>
__global__ __launch_bounds__(256) void join_kernel(Args g) {
    constexpr int AT = 256 / SHARES;
    __shared__ float held[SHARES > 1 ? SHARES - 1 : 1][SHARES > 1 ? AT : 1][8];
    const int pieces = (g.n + 7) / 8, mine = threadIdx.x % AT, share = threadIdx.x / AT;
    const int64_t at = (int64_t)blockIdx.x * AT + mine, row = at / pieces;
    const int col = (int)(at - row * pieces) * 8;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (row < g.m) {
#pragma unroll 4
        for (int s = share; s < g.splits; s += SHARES) {
            const v4f* q = reinterpret_cast<const v4f*>(g.partial + (((int64_t)s * g.m + row) * pieces) * 8 + col);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += q[e >> 2][e & 3];
        }
    }
    if constexpr (SHARES > 1) {
        if (share)
#pragma unroll
            for (int e = 0; e < 8; ++e) held[share - 1][mine][e] = v[e];
        __syncthreads();
        if (share) return;
#pragma unroll
        for (int i = 0; i < SHARES - 1; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += held[i][mine][e];
    }
    if (row >= g.m) return;
    float bias[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    load_bias(g.finish, col, g.n - col, bias);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += bias[e];
    if (col + 8 <= g.n) {
        Raw8 more;
        if (g.finish.residual) more.load(g.finish.residual, g.finish.residual_bf16, row * g.finish.residual_stride + col);
        finish8(g.finish, row, col, v, more);
    } else {
        finish_edge(g.finish, row, col, g.n - col, v);
    }
}

}  // namespace gemm
}  // namespace edb
