// Layer norm and its gradients.
//
//   mean_i = 1/D sum_j x_ij,  r_i = 1 / sqrt(1/D sum_j (x_ij - mean_i)^2 + eps)
//   y_ij   = (x_ij - mean_i) r_i w_j + b_j
//
// with h_ij = (x_ij - mean_i) r_i and g_ij = dy_ij w_j, backwards
//
//   dx_ij = r_i (g_ij - 1/D sum_j g_ij - h_ij 1/D sum_j g_ij h_ij)
//   dw_j  = sum_i dy_ij h_ij,   db_j = sum_i dy_ij
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "column_sums.h"
#include "edb_internal.h"
#include "lane_sums.h"
#include "row_access.h"

using edb::fail;
using edb::Region;
using namespace edb::rows;

namespace {

struct NormArgs {
    const void* x;
    int64_t x_stride;
    const void *weight, *bias;
    bool weight_bf16;
    double eps, per;          // per: 1 / dim
    void* out;
    int64_t out_stride;
    float* stats;
    int32_t n, dim;
    bool past;
};

// K elements of the scale or the shift, `none` where there is no such array.
template <int K>
__device__ __forceinline__ void load_weight(const void* p, bool half, int col, float none, float* v) {
    if (!p) {
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] = none;
    } else if (half) {
        load_k<bf16, K>(static_cast<const bf16*>(p) + col, v);
    } else {
        load_k<float, K>(static_cast<const float*>(p) + col, v);
    }
}

// Sums of two values over the LANES threads of a row, in every one of them.
// Over several waves: `held` has a place for each (the caller's barriers
// separate its uses).
template <int LANES, class V>
__device__ __forceinline__ void row_sums(V& a, V& b, V (*held)[2]) {
    a = edb::lanes::sum<LANES < 64 ? LANES : 64>(a);
    b = edb::lanes::sum<LANES < 64 ? LANES : 64>(b);
    if constexpr (LANES > 64) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            held[wave][0] = a;
            held[wave][1] = b;
        }
        __syncthreads();
        a = b = V(0);
#pragma unroll
        for (int w = 0; w < LANES / 64; ++w) {
            a += held[w][0];
            b += held[w][1];
        }
    }
}

// Threads of a row's group, pieces a thread, rows at once: a work-group has 256
// threads, or one row's.
template <int LANES>
constexpr int threads() {
    return LANES > 256 ? LANES : 256;
}

// K elements as they lie in memory, read once: asked for a turn before they are used.
template <class T, int K>
struct RawPiece {
    static constexpr int kWords = K * (int)sizeof(T) / 16;
    u32x4 w[kWords > 0 ? kWords : 1];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (K == 1) w[0][0] = __builtin_bit_cast(uint32_t, Elem<T>::get(p));
        else if constexpr (kWords == 0) {
            const u32x2 h = Elem<T>::load_half_nt(p);
            w[0][0] = h[0];
            w[0][1] = h[1];
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) w[i] = Elem<T>::load_nt(p + i * Elem<T>::kVec);
        }
    }
    __device__ __forceinline__ void unpack(float* v) const {
        if constexpr (K == 1) v[0] = __builtin_bit_cast(float, (uint32_t)w[0][0]);
        else if constexpr (kWords == 0) Elem<T>::unpack_half(u32x2{w[0][0], w[0][1]}, v);
        else {
#pragma unroll
            for (int i = 0; i < kWords; ++i) Elem<T>::unpack(w[i], v + i * Elem<T>::kVec);
        }
    }
};

// The statistics are sums of differences from a value of the row's own, c: one
// pass over the row.  By pieces in 32 bits, c being the average of the row's
// first K elements, and over the pieces in 64, as long as that is safe: squares
// within fp32's range and c within two deviations of the mean, so that no digits
// cancel.  Other rows (an outlier at the front, constant, very large or very small
// ones) are done again in 64 bits with c = the first element, whose own square
// distance bounds the variance from below.  All rows in 64 bits took 158 us for
// 262144 x 512 bf16: conversions and 64-bit operations, not memory, bound it.
struct Moments {
    double mean, rstd;
    bool safe;
    // per = 1 / dim
    __device__ __forceinline__ Moments(double c, double sum, double squares, double per, double eps) {
        const double d = sum * per, all = squares * per, var = all - d * d, v = var + eps;
        mean = c + d;
        // one step of Newton's from the hardware's 22 bits and more
        const double y = (double)__builtin_amdgcn_rsqf((float)v);
        rstd = y * fma(-0.5 * v * y, y, 1.5);
        safe = squares >= 1e-25 && squares <= 1e30 && all <= 4.0 * var && v <= 1e37;
    }
    // whatever the numbers: the divisions and the root take as long as a row of 512 otherwise
    __device__ __forceinline__ void wide(double c, double sum, double squares, int dim, double eps) {
        const double d = sum / dim, var = squares / dim - d * d;
        mean = var == var ? c + d : var;
        rstd = 1.0 / sqrt((var > 0.0 ? var : var == var ? 0.0 : var) + eps);
    }
};

// Sums of the differences of K elements from c, the first `skip` left out, by a tree.
template <int K>
__device__ __forceinline__ void piece_sums(const float* e, float c, int skip, float& sum, float& squares) {
    float s[K], q[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        s[k] = K > 1 && k < skip ? 0.f : e[k] - c;
        q[k] = s[k] * s[k];
    }
#pragma unroll
    for (int w = K / 2; w; w >>= 1)
#pragma unroll
        for (int k = 0; k < w; ++k) {
            s[k] += s[k + w];
            q[k] += q[k + w];
        }
    sum = s[0];
    squares = q[0];
}
template <int K>
__device__ __forceinline__ void piece_sums(const float* e, double c, int skip, double& sum, double& squares) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const double d = (double)e[k] - c;
        if (K > 1 && k < skip) continue;
        sum += d;
        squares = fma(d, d, squares);
    }
}
template <int K>
__device__ __forceinline__ float average(const float* e) {
    float s = e[0];
#pragma unroll
    for (int k = 1; k < K; ++k) s += e[k];
    return s * (1.f / K);
}

// (x - mean) rstd: the mean as two floats where the row is safe.
struct Scaled {
    float high, low, rstd;
    const Moments& m;
    __device__ __forceinline__ explicit Scaled(const Moments& m) : high((float)m.mean), low((float)(m.mean - (double)high)), rstd((float)m.rstd), m(m) {}
    __device__ __forceinline__ float safe(float x) const { return ((x - high) - low) * rstd; }
    __device__ __forceinline__ float wide(float x) const { return (float)(((double)x - m.mean) * m.rstd); }
};

// Memory bound: 262144 x 512 bf16 107 us (5.0 TB/s), 30000 x 1024 fp32 42 (5.8);
// 28629 x 512 bf16, two turns of a work-group, 15.3 (3.8).  112 x 64 fp32: 2.6, a launch.
template <class T, class O, int K, int LANES, int V, int ROWS>
__global__ __launch_bounds__(threads<LANES>()) void norm_kernel(NormArgs a) {
    constexpr int kGroups = threads<LANES>() / LANES;
    constexpr bool kHoldWeights = V * K <= 16;
    __shared__ double held[LANES > 64 ? 2 : 1][LANES > 64 ? LANES / 64 : 1][2];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    float w[V][K], b[V][K];
    if constexpr (kHoldWeights) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int nominal = (v * LANES + lane) * K;
            const Piece<K> p(nominal < a.dim ? nominal : 0, a.dim);
            load_weight<K>(a.weight, a.weight_bf16, p.col, 1.f, w[v]);
            load_weight<K>(a.bias, a.weight_bf16, p.col, 0.f, b[v]);
        }
    }
    const T* x = static_cast<const T*>(a.x);
    O* out = static_cast<O*>(a.out);
    int turn = 0;
    const int64_t apart = (int64_t)gridDim.x * kGroups * ROWS;
    int64_t row0 = ((int64_t)blockIdx.x * kGroups + group) * ROWS;
    RawPiece<T, K> raw[ROWS][V], front[ROWS];
    auto load = [&](int64_t from) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const T* row = x + min(from + r, (int64_t)a.n - 1) * a.x_stride;
            front[r].load(row);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int nominal = (v * LANES + lane) * K;
                if (nominal < a.dim) raw[r][v].load(row + Piece<K>(nominal, a.dim).col);
            }
        }
    };
    if (row0 < a.n) load(row0);
    // (rows that share barriers are a work-group's only ones)
    for (; row0 < a.n; row0 += apart) {
        float e[ROWS][V][K], c[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float f[K];
            front[r].unpack(f);
            c[r] = average<K>(f);
#pragma unroll
            for (int v = 0; v < V; ++v) raw[r][v].unpack(e[r][v]);
        }
        if (row0 + apart < a.n) load(row0 + apart);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            double sum = 0.0, squares = 0.0;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int nominal = (v * LANES + lane) * K;
                if (nominal >= a.dim) continue;
                float s, q;
                piece_sums<K>(e[r][v], c[r], Piece<K>(nominal, a.dim).skip, s, q);
                sum += (double)s;
                squares += (double)q;
            }
            row_sums<LANES>(sum, squares, held[LANES > 64 ? turn : 0]);
            turn ^= 1;
            Moments m(c[r], sum, squares, a.per, a.eps);
            const bool safe = m.safe;
            if (!safe) {
                const double first = Elem<T>::get(x + min(row0 + r, (int64_t)a.n - 1) * a.x_stride);
                sum = squares = 0.0;
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int nominal = (v * LANES + lane) * K;
                    if (nominal < a.dim) piece_sums<K>(e[r][v], first, Piece<K>(nominal, a.dim).skip, sum, squares);
                }
                row_sums<LANES>(sum, squares, held[LANES > 64 ? turn : 0]);
                turn ^= 1;
                m.wide(first, sum, squares, a.dim, a.eps);
            }
            if (row0 + r >= a.n) break;
            if (lane == 0 && a.stats) {
                a.stats[2 * (row0 + r)] = (float)m.mean;
                a.stats[2 * (row0 + r) + 1] = (float)m.rstd;
            }
            const Scaled scaled(m);
            O* to = out + (row0 + r) * a.out_stride;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int nominal = (v * LANES + lane) * K;
                if (nominal >= a.dim) continue;
                const Piece<K> p(nominal, a.dim);
                if constexpr (!kHoldWeights) {
                    load_weight<K>(a.weight, a.weight_bf16, p.col, 1.f, w[v]);
                    load_weight<K>(a.bias, a.weight_bf16, p.col, 0.f, b[v]);
                }
                float y[K];
                if (safe) {
#pragma unroll
                    for (int k = 0; k < K; ++k) y[k] = fmaf(scaled.safe(e[r][v][k]), w[v][k], b[v][k]);
                } else {
#pragma unroll
                    for (int k = 0; k < K; ++k) y[k] = fmaf(scaled.wide(e[r][v][k]), w[v][k], b[v][k]);
                }
                // results that no cache could hold go past them (30000 x 1024 fp32 45.3 to 41.6 us)
                if (K == Elem<O>::kVec && a.past && p.skip == 0) Elem<O>::store_nt(to + p.col, Elem<O>::pack(y));
                else store_from<O, K>(to + p.col, y, p.skip);
            }
        }
    }
}

// Rows that no work-group holds: read twice.
constexpr int kLong = 1024;
template <class T, class O>
__global__ __launch_bounds__(kLong) void norm_long_kernel(NormArgs a) {
    constexpr int K = Elem<T>::kVec;
    __shared__ double held[2][kLong / 64][2];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const double first = Elem<T>::get(x);
        double sum = 0.0, squares = 0.0;
        for (int nominal = threadIdx.x * K; nominal < a.dim; nominal += kLong * K) {
            const Piece<K> p(nominal, a.dim);
            float e[K];
            load_k<T, K>(x + p.col, e);
            piece_sums<K>(e, first, p.skip, sum, squares);
        }
        row_sums<kLong>(sum, squares, held[turn]);
        turn ^= 1;
        Moments m(first, sum, squares, a.per, a.eps);
        m.wide(first, sum, squares, a.dim, a.eps);
        if (threadIdx.x == 0 && a.stats) {
            a.stats[2 * row] = (float)m.mean;
            a.stats[2 * row + 1] = (float)m.rstd;
        }
        const Scaled scaled(m);
        O* to = static_cast<O*>(a.out) + row * a.out_stride;
        for (int nominal = threadIdx.x * K; nominal < a.dim; nominal += kLong * K) {
            const Piece<K> p(nominal, a.dim);
            float e[K], w[K], b[K];
            load_k<T, K>(x + p.col, e);
            load_weight<K>(a.weight, a.weight_bf16, p.col, 1.f, w);
            load_weight<K>(a.bias, a.weight_bf16, p.col, 0.f, b);
#pragma unroll
            for (int k = 0; k < K; ++k) e[k] = fmaf(scaled.wide(e[k]), w[k], b[k]);
            store_from<O, K>(to + p.col, e, p.skip);
        }
    }
}

struct GradArgs {
    const void* x;
    int64_t x_stride;
    const float* stats;
    const void* dout;
    int64_t dout_stride;
    const void* weight;
    bool weight_bf16;
    void* dx;          // or NULL
    int64_t dx_stride;
    float* part;       // [work-group][2][dim], or NULL: dw and db are not wanted
    int32_t n, dim;
};

// (x - mean) rstd, by halves: the difference itself could leave fp32's range.
__device__ __forceinline__ float scaled(float x, float mean, float rstd) { return fmaf(x, 0.5f, -0.5f * mean) * (2.f * rstd); }

// A work-group's rows give their gradients and, in registers, their share of
// dw and db, which it writes once; a second launch adds up the shares.  Memory
// bound: 262144 x 512 bf16 151 us with the second launch's 5 (5.2 TB/s), 8000 x 8192 85
// (4.6); 1627 x 100 fp32 4.1 and 3.1.
template <class T, class O, int K, int LANES, int V, int ROWS>
__global__ __launch_bounds__(threads<LANES>()) void norm_grad_kernel(GradArgs a) {
    constexpr int kGroups = threads<LANES>() / LANES;
    __shared__ float held[LANES > 64 ? 2 : 1][LANES > 64 ? LANES / 64 : 1][2];
    __shared__ float shares[kGroups > 1 ? kGroups : 1][kGroups > 1 ? LANES * V * K : 1];
    const int lane = threadIdx.x % LANES, group = threadIdx.x / LANES;
    const T* x = static_cast<const T*>(a.x);
    const O* dout = static_cast<const O*>(a.dout);
    T* dx = static_cast<T*>(a.dx);
    float w[V][K], dw[V][K], db[V][K];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int nominal = (v * LANES + lane) * K;
        load_weight<K>(a.weight, a.weight_bf16, Piece<K>(nominal < a.dim ? nominal : 0, a.dim).col, 1.f, w[v]);
#pragma unroll
        for (int k = 0; k < K; ++k) dw[v][k] = db[v][k] = 0.f;
    }
    const float per = 1.f / (float)a.dim;
    int turn = 0;
    const int64_t apart = (int64_t)gridDim.x * kGroups * ROWS;
    int64_t row0 = ((int64_t)blockIdx.x * kGroups + group) * ROWS;
    RawPiece<T, K> raw_x[ROWS][V];
    RawPiece<O, K> raw_d[ROWS][V];
    float raw_mean[ROWS], raw_rstd[ROWS];
    auto load = [&](int64_t from) {
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const int64_t row = min(from + r, (int64_t)a.n - 1);
            raw_mean[r] = a.stats[2 * row];
            raw_rstd[r] = a.stats[2 * row + 1];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int nominal = (v * LANES + lane) * K;
                if (nominal >= a.dim) continue;
                const int col = Piece<K>(nominal, a.dim).col;
                raw_x[r][v].load(x + row * a.x_stride + col);
                raw_d[r][v].load(dout + row * a.dout_stride + col);
            }
        }
    };
    if (row0 < a.n) load(row0);
    for (; row0 < a.n; row0 += apart) {
        float h[ROWS][V][K], d[ROWS][V][K], mean[ROWS], rstd[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            mean[r] = raw_mean[r];
            rstd[r] = raw_rstd[r];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                raw_x[r][v].unpack(h[r][v]);
                raw_d[r][v].unpack(d[r][v]);
            }
        }
        if (row0 + apart < a.n) load(row0 + apart);
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            if (row0 + r >= a.n) break;
            float c1 = 0.f, c2 = 0.f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int nominal = (v * LANES + lane) * K;
                if (nominal >= a.dim) continue;
                const int skip = Piece<K>(nominal, a.dim).skip;
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    h[r][v][k] = scaled(h[r][v][k], mean[r], rstd[r]);
                    if (K > 1 && k < skip) continue;
                    const float g = d[r][v][k] * w[v][k];
                    c1 += g;
                    c2 = fmaf(g, h[r][v][k], c2);
                    dw[v][k] = fmaf(d[r][v][k], h[r][v][k], dw[v][k]);
                    db[v][k] += d[r][v][k];
                }
            }
            if (!dx) continue;
            row_sums<LANES>(c1, c2, held[LANES > 64 ? turn : 0]);
            turn ^= 1;
            c1 *= per;
            c2 *= per;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int nominal = (v * LANES + lane) * K;
                if (nominal >= a.dim) continue;
                const Piece<K> p(nominal, a.dim);
                float y[K];
#pragma unroll
                for (int k = 0; k < K; ++k) y[k] = rstd[r] * (fmaf(d[r][v][k], w[v][k], -c1) - h[r][v][k] * c2);
                store_from<T, K>(dx + (row0 + r) * a.dx_stride + p.col, y, p.skip);
            }
        }
    }
    if (!a.part) return;
    float* part = a.part + (int64_t)blockIdx.x * 2 * a.dim;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float(&s)[V][K] = which ? db : dw;
        if constexpr (kGroups > 1) {
            if (which) __syncthreads();
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int k = 0; k < K; ++k) shares[group][(v * K + k) * LANES + lane] = s[v][k];
            __syncthreads();
            if (group > 0) continue;
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int nominal = (v * LANES + lane) * K;
            if (nominal >= a.dim) continue;
            const Piece<K> p(nominal, a.dim);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if constexpr (kGroups > 1)
                    for (int g = 1; g < kGroups; ++g) s[v][k] += shares[g][(v * K + k) * LANES + lane];
                if (K == 1 || k >= p.skip) part[which * a.dim + p.col + k] = s[v][k];
            }
        }
    }
}

// Gradients of rows that no work-group holds: read twice; their columns' sums
// are another kernel's.
template <class T, class O>
__global__ __launch_bounds__(kLong) void norm_grad_long_kernel(GradArgs a) {
    constexpr int K = Elem<T>::kVec;
    __shared__ float held[2][kLong / 64][2];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const O* dout = static_cast<const O*>(a.dout) + row * a.dout_stride;
        const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
        float c1 = 0.f, c2 = 0.f;
        for (int nominal = threadIdx.x * K; nominal < a.dim; nominal += kLong * K) {
            const Piece<K> p(nominal, a.dim);
            float e[K], d[K], w[K];
            load_k<T, K>(x + p.col, e);
            load_k<O, K>(dout + p.col, d);
            load_weight<K>(a.weight, a.weight_bf16, p.col, 1.f, w);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (k < p.skip) continue;
                const float g = d[k] * w[k];
                c1 += g;
                c2 = fmaf(g, scaled(e[k], mean, rstd), c2);
            }
        }
        row_sums<kLong>(c1, c2, held[turn]);
        turn ^= 1;
        c1 *= 1.f / (float)a.dim;
        c2 *= 1.f / (float)a.dim;
        T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
        for (int nominal = threadIdx.x * K; nominal < a.dim; nominal += kLong * K) {
            const Piece<K> p(nominal, a.dim);
            float e[K], d[K], w[K];
            load_k<T, K>(x + p.col, e);
            load_k<O, K>(dout + p.col, d);
            load_weight<K>(a.weight, a.weight_bf16, p.col, 1.f, w);
#pragma unroll
            for (int k = 0; k < K; ++k) e[k] = rstd * (fmaf(d[k], w[k], -c1) - scaled(e[k], mean, rstd) * c2);
            store_from<T, K>(dx + p.col, e, p.skip);
        }
    }
}

// dw and db of such rows: a thread adds up K columns over a work-group's rows.
template <class T, class O>
__global__ __launch_bounds__(256) void norm_columns_kernel(GradArgs a, int rows_per) {
    constexpr int K = Elem<T>::kVec;
    const int nominal = (blockIdx.x * 256 + threadIdx.x) * K;
    if (nominal >= a.dim) return;
    const Piece<K> p(nominal, a.dim);
    float dw[K], db[K];
#pragma unroll
    for (int k = 0; k < K; ++k) dw[k] = db[k] = 0.f;
    const int64_t first = (int64_t)blockIdx.y * rows_per, end = min(first + rows_per, (int64_t)a.n);
    for (int64_t row = first; row < end; ++row) {
        const float mean = a.stats[2 * row], rstd = a.stats[2 * row + 1];
        float e[K], d[K];
        load_k<T, K>(static_cast<const T*>(a.x) + row * a.x_stride + p.col, e);
        load_k<O, K>(static_cast<const O*>(a.dout) + row * a.dout_stride + p.col, d);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            dw[k] = fmaf(d[k], scaled(e[k], mean, rstd), dw[k]);
            db[k] += d[k];
        }
    }
    float* part = a.part + (int64_t)blockIdx.y * 2 * a.dim + p.col;
    store_from<float, K>(part, dw, p.skip);
    store_from<float, K>(part + a.dim, db, p.skip);
}

constexpr int64_t kMaxElems = INT64_C(1) << 48;
constexpr int32_t kMaxDim = 1 << 20;
constexpr int64_t kPast = 96 << 20;

int32_t elem_bytes(int32_t dtype) { return dtype == EDB_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == EDB_F32 || dtype == EDB_BF16; }
bool element_aligned(const void* p, int32_t dtype) { return !(reinterpret_cast<uintptr_t>(p) & (elem_bytes(dtype) - 1)); }

Region matrix(const void* p, int32_t dtype, int32_t n, int32_t dim, int64_t stride) {
    return {n > 0 ? p : nullptr, n, (int64_t)dim * elem_bytes(dtype), stride * elem_bytes(dtype)};
}

edb_status launched(const char* who) {
    const hipError_t he = hipGetLastError();
    if (he != hipSuccess) return fail(EDB_ERR_HIP, std::string(who) + ": " + hipGetErrorString(he));
    edb::clear_error();
    return EDB_OK;
}

edb_status check_sizes(const char* who, int32_t n, int32_t dim) {
    const std::string w(who);
    if (n < 0 || dim < 1) return fail(EDB_ERR_INVALID, w + ": n >= 0 and dim >= 1 are needed");
    if (dim > kMaxDim) return fail(EDB_ERR_UNSUPPORTED, w + ": dim must not exceed 2^20");
    return EDB_OK;
}

edb_status check_matrix(const char* who, const char* name, const void* p, int32_t dtype, int32_t n, int32_t dim, int64_t stride) {
    const std::string w = std::string(who) + ": " + name;
    if (!known(dtype)) return fail(EDB_ERR_INVALID, w + ": dtype must be F32 or BF16");
    if (stride < dim) return fail(EDB_ERR_INVALID, w + ": the row stride is below dim");
    if (stride > kMaxElems / (n > 0 ? n : 1)) return fail(EDB_ERR_INVALID, w + ": the rows span more than 2^48 elements");
    if (n && !p) return fail(EDB_ERR_INVALID, w + ": NULL");
    if (!element_aligned(p, dtype)) return fail(EDB_ERR_INVALID, w + ": must be aligned to its elements");
    return EDB_OK;
}

int64_t pieces_of(int32_t dim, int k) { return ((int64_t)dim + k - 1) / k; }

template <class T, class O, int K, int LANES, int V, int ROWS>
void start(const NormArgs& a, hipStream_t st) {
    constexpr int kRows = threads<LANES>() / LANES * ROWS;
    // a few turns each at most sizes (262144 x 512 bf16 109 us, with 2048 work-groups 112; 28629 x 512 16.3, with one
    // turn each, of 3579, 17.2)
    const int64_t groups = ((int64_t)a.n + kRows - 1) / kRows, most = groups > 8192 ? 8192 : 2048;
    norm_kernel<T, O, K, LANES, V, ROWS><<<(unsigned)(groups < most ? groups : most), threads<LANES>(), 0, st>>>(a);
}

// As few threads a row as hold it.
template <class T, class O>
void launch_norm(const NormArgs& a, hipStream_t st) {
    constexpr int K = Elem<T>::kVec;
    const int64_t pieces = pieces_of(a.dim, K);
    if (a.dim < K) start<T, O, 1, 8, 1, 2>(a, st);
    else if (pieces <= 16) start<T, O, K, 16, 1, 2>(a, st);
    else if (pieces <= 32) start<T, O, K, 32, 1, 2>(a, st);
    else if (pieces <= 64) start<T, O, K, 64, 1, 2>(a, st);
    else if (pieces <= 128) start<T, O, K, 64, 2, 2>(a, st);
    else if (pieces <= 256) start<T, O, K, 64, 4, 1>(a, st);
    else if (pieces <= 512) start<T, O, K, 256, 2, 1>(a, st);
    else if (pieces <= 1024) start<T, O, K, 256, 4, 1>(a, st);
    else if (pieces <= 2048) start<T, O, K, 1024, 2, 1>(a, st);
    else {
        if constexpr (K == 4) {   // 8 elements a piece: no registers for it
            if (pieces <= 4096) return start<T, O, K, 1024, 4, 1>(a, st);
        }
        norm_long_kernel<T, O><<<(unsigned)(a.n < 2048 ? a.n : 2048), kLong, 0, st>>>(a);
    }
}

constexpr int64_t kMostParts = 1024;

// Work-groups of the gradient (each writes a part of dw and db).
struct GradPlan {
    int32_t lanes, pieces, rows;   // lanes == 0: rows that no work-group holds
    int32_t parts, rows_per;
    int64_t bytes;
};

GradPlan grad_plan(int32_t n, int32_t dim, int k) {
    GradPlan g{};
    const int64_t pieces = pieces_of(dim, k);
    if (dim < k) g = {8, 1, 2, 0, 0, 0};
    else if (pieces <= 16) g = {16, 1, 2, 0, 0, 0};
    else if (pieces <= 32) g = {32, 1, 2, 0, 0, 0};
    else if (pieces <= 64) g = {64, 1, 2, 0, 0, 0};
    else if (pieces <= 128) g = {64, 2, 1, 0, 0, 0};
    else if (pieces <= 256) g = {256, 1, 1, 0, 0, 0};
    else if (pieces <= 512) g = {256, 2, 1, 0, 0, 0};
    else if (pieces <= 1024) g = {1024, 1, 1, 0, 0, 0};
    else if (pieces <= 2048) g = {1024, 2, 1, 0, 0, 0};
    int64_t parts;
    if (g.lanes) {
        const int rows = (g.lanes > 256 ? 1 : 256 / g.lanes) * g.rows;
        parts = ((int64_t)n + rows - 1) / rows;
        // the parts are a twentieth of what the rows are, but enough to fill the card
        const int64_t most = n / 32 > kMostParts ? kMostParts : n / 32 > 256 ? n / 32 : 256;
        if (parts > most) parts = most;
    } else {
        const int64_t wide = (pieces + 255) / 256;
        parts = (2048 + wide - 1) / wide;
        if (parts > n / 8 + 1) parts = n / 8 + 1;
        g.rows_per = (int32_t)(((int64_t)n + parts - 1) / parts);
        parts = g.rows_per ? ((int64_t)n + g.rows_per - 1) / g.rows_per : 0;
    }
    g.parts = (int32_t)parts;
    g.bytes = parts * 2 * dim * 4;
    return g;
}

template <class T, class O>
void launch_grad(const GradPlan& g, const GradArgs& a, hipStream_t st) {
    constexpr int K = Elem<T>::kVec;
    const unsigned parts = g.parts;
    if (g.lanes == 8) norm_grad_kernel<T, O, 1, 8, 1, 2><<<parts, 256, 0, st>>>(a);
    else if (g.lanes == 16) norm_grad_kernel<T, O, K, 16, 1, 2><<<parts, 256, 0, st>>>(a);
    else if (g.lanes == 32) norm_grad_kernel<T, O, K, 32, 1, 2><<<parts, 256, 0, st>>>(a);
    else if (g.lanes == 64 && g.pieces == 1) norm_grad_kernel<T, O, K, 64, 1, 2><<<parts, 256, 0, st>>>(a);
    else if (g.lanes == 64) norm_grad_kernel<T, O, K, 64, 2, 1><<<parts, 256, 0, st>>>(a);
    else if (g.lanes == 256 && g.pieces == 1) norm_grad_kernel<T, O, K, 256, 1, 1><<<parts, 256, 0, st>>>(a);
    else if (g.lanes == 256) norm_grad_kernel<T, O, K, 256, 2, 1><<<parts, 256, 0, st>>>(a);
    else if (g.lanes == 1024 && g.pieces == 1) norm_grad_kernel<T, O, K, 1024, 1, 1><<<parts, 1024, 0, st>>>(a);
    else if (g.lanes == 1024) norm_grad_kernel<T, O, K, 1024, 2, 1><<<parts, 1024, 0, st>>>(a);
    else {
        if (a.dx) norm_grad_long_kernel<T, O><<<(unsigned)(a.n < 2048 ? a.n : 2048), kLong, 0, st>>>(a);
        if (a.part) {
            const dim3 grid((unsigned)((pieces_of(a.dim, K) + 255) / 256), parts);
            norm_columns_kernel<T, O><<<grid, 256, 0, st>>>(a, g.rows_per);
        }
    }
}

}  // namespace

extern "C" edb_status edb_layer_norm(const void* x, int32_t x_dtype, int32_t n, int32_t dim, int64_t x_stride,
                                     const void* weight, const void* bias, int32_t weight_dtype, double eps, void* out,
                                     int32_t out_dtype, int64_t out_stride, float* stats, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_layer_norm";
        if (edb_status st = check_sizes(who, n, dim)) return st;
        if (edb_status st = check_matrix(who, "x", x, x_dtype, n, dim, x_stride)) return st;
        if (edb_status st = check_matrix(who, "out", out, out_dtype, n, dim, out_stride)) return st;
        if (!known(weight_dtype)) return fail(EDB_ERR_INVALID, "edb_layer_norm: weight: dtype must be F32 or BF16");
        if (!(eps >= 0.0) || !std::isfinite(eps)) return fail(EDB_ERR_INVALID, "edb_layer_norm: eps must be finite and not negative");
        if (!element_aligned(weight, weight_dtype) || !element_aligned(bias, weight_dtype) || !edb::word_aligned({stats}))
            return fail(EDB_ERR_INVALID, "edb_layer_norm: weight, bias and stats must be aligned to their elements");
        if (n == 0) {
            edb::clear_error();
            return EDB_OK;
        }
        const int64_t wide = (int64_t)dim * elem_bytes(weight_dtype);
        if (edb_status st = edb::apart(who, {matrix(out, out_dtype, n, dim, out_stride), Region::array(stats, n * INT64_C(8))},
                                       {matrix(x, x_dtype, n, dim, x_stride), Region::array(weight, wide), Region::array(bias, wide)}))
            return st;
        const NormArgs a{x, x_stride, weight, bias, weight_dtype == EDB_BF16, eps, 1.0 / dim, out, out_stride, stats, n, dim,
                         (int64_t)n * dim * elem_bytes(out_dtype) >= kPast};
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        if (x_dtype == EDB_F32) {
            if (out_dtype == EDB_F32) launch_norm<float, float>(a, st);
            else launch_norm<float, bf16>(a, st);
        } else {
            if (out_dtype == EDB_F32) launch_norm<bf16, float>(a, st);
            else launch_norm<bf16, bf16>(a, st);
        }
        return launched(who);
    });
}

extern "C" edb_status edb_layer_norm_grad_bytes(int32_t n, int32_t dim, int32_t x_dtype, int64_t* bytes) {
    return edb::guarded([&]() -> edb_status {
        if (!bytes) return fail(EDB_ERR_INVALID, "edb_layer_norm_grad_bytes: NULL argument");
        if (!known(x_dtype)) return fail(EDB_ERR_INVALID, "edb_layer_norm_grad_bytes: dtype must be F32 or BF16");
        if (edb_status st = check_sizes("edb_layer_norm_grad_bytes", n, dim)) return st;
        *bytes = grad_plan(n, dim, x_dtype == EDB_BF16 ? 8 : 4).bytes;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_layer_norm_grad(const void* x, int32_t x_dtype, int32_t n, int32_t dim, int64_t x_stride,
                                          const float* stats, const void* dout, int32_t dout_dtype, int64_t dout_stride,
                                          const void* weight, int32_t weight_dtype, void* dx, int64_t dx_stride,
                                          float* dweight, float* dbias, void* workspace, int64_t workspace_bytes,
                                          void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_layer_norm_grad";
        if (edb_status st = check_sizes(who, n, dim)) return st;
        if (edb_status st = check_matrix(who, "x", x, x_dtype, n, dim, x_stride)) return st;
        if (edb_status st = check_matrix(who, "dout", dout, dout_dtype, n, dim, dout_stride)) return st;
        if (dx)
            if (edb_status st = check_matrix(who, "dx", dx, x_dtype, n, dim, dx_stride)) return st;
        if (!known(weight_dtype)) return fail(EDB_ERR_INVALID, "edb_layer_norm_grad: weight: dtype must be F32 or BF16");
        if (n && !stats) return fail(EDB_ERR_INVALID, "edb_layer_norm_grad: NULL stats");
        if (!element_aligned(weight, weight_dtype) || !edb::word_aligned({stats, dweight, dbias}))
            return fail(EDB_ERR_INVALID, "edb_layer_norm_grad: weight, stats and sums must be aligned to their elements");
        const bool sums = dweight || dbias;
        GradPlan g = grad_plan(n, dim, x_dtype == EDB_BF16 ? 8 : 4);
        if (!sums) g.bytes = 0;
        if (workspace_bytes < g.bytes || (g.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
            return fail(EDB_ERR_INVALID, "edb_layer_norm_grad: a 16-byte aligned workspace of " + std::to_string(g.bytes) +
                                             " bytes is needed");
        if (edb_status st = edb::apart(
                who,
                {matrix(dx, x_dtype, n, dim, dx_stride), Region::array(dweight, dim * INT64_C(4)),
                 Region::array(dbias, dim * INT64_C(4)), Region::array(workspace, g.bytes)},
                {matrix(x, x_dtype, n, dim, x_stride), matrix(dout, dout_dtype, n, dim, dout_stride),
                 Region::array(stats, n * INT64_C(8)), Region::array(weight, (int64_t)dim * elem_bytes(weight_dtype))}))
            return st;
        if ((n == 0 || !dx) && !sums) {
            edb::clear_error();
            return EDB_OK;
        }
        GradArgs a{x, x_stride, stats, dout, dout_stride, weight, weight_dtype == EDB_BF16, dx, dx_stride,
                   sums ? static_cast<float*>(workspace) : nullptr, n, dim};
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        if (n) {
            if (x_dtype == EDB_F32) {
                if (dout_dtype == EDB_F32) launch_grad<float, float>(g, a, st);
                else launch_grad<float, bf16>(g, a, st);
            } else {
                if (dout_dtype == EDB_F32) launch_grad<bf16, float>(g, a, st);
                else launch_grad<bf16, bf16>(g, a, st);
            }
        }
        if (sums) edb::join_columns(a.part, g.parts, dim, 2, dweight, dbias, st);
        return launched(who);
    });
}
