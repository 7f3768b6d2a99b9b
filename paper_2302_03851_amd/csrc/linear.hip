// Linear layers: matrix product with bias, activation and residual in its
// epilogue, and its gradients.
//
//   v = x W + b,  y = act(v) + r;       g = dy act'(v),  dx = g W^T,  dW = x^T g,  db = sum_i g_i
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "column_sums.h"
#include "edb_internal.h"
#include "gemm_tile.h"

using edb::fail;
using edb::Region;
using namespace edb::rows;
using edb::gemm::Args;
using edb::gemm::Finish;
using edb::gemm::K_LINES;
using edb::gemm::Layout;
using edb::gemm::MN_LINES;

namespace {

struct SlopeArgs {
    const void* dout;
    int64_t dout_stride;
    const void* pre;
    int64_t pre_stride;
    int32_t act, n, m, rows_per;
    void* g;               // [n][m rounded up to 8], or NULL
    float* part;           // [chunk][m], or NULL
};

// g = dy act'(v) as the products take it, and the sums of its columns before
// that rounding: 32 pieces of 8 columns by 8 rows at once a work-group.
// For bf16 operands g is rounded to bf16, as the matrix instructions need it (two
// pieces would double the products).  Sums over more than 64 rows of a thread's go
// on in a second register, so that long columns are no chains of additions.
// Memory bound: the sums alone of 8192 x 65536 bf16 189 us, 5.7 TB/s.
template <class D, class T>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a) {
    __shared__ float held[8][32][9];
    const int piece = threadIdx.x & 31, line = threadIdx.x >> 5;
    const int col = (blockIdx.x * 32 + piece) * 8, left = min(a.m - col, 8);
    const int64_t gm = (a.m + 7) / 8 * 8;
    const int64_t first = (int64_t)blockIdx.y * a.rows_per, end = min(first + a.rows_per, (int64_t)a.n);
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, folded[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    int turn = 0;
    if (left > 0)
        for (int64_t row = first + line; row < end; row += 8) {
            const D* d = static_cast<const D*>(a.dout) + row * a.dout_stride + col;
            const T* v = static_cast<const T*>(a.pre) + row * a.pre_stride + col;
            float x[8], y[8];
            if (left == 8) {
                load_k<D, 8>(d, x);
                if (a.act != EDB_ACT_NONE) load_k<T, 8>(v, y);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = i < left ? Elem<D>::get(d + i) : 0.f;
                    y[i] = i < left && a.act != EDB_ACT_NONE ? Elem<T>::get(v + i) : 0.f;
                }
            }
            edb::gemm::slope8(a.act, y, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum[i] += x[i];
            if ((++turn & 63) == 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    folded[i] += sum[i];
                    sum[i] = 0.f;
                }
            }
            if (a.g) store_k<T, 8>(static_cast<T*>(a.g) + row * gm + col, x);
        }
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) held[line][piece][i] = folded[i] + sum[i];
    __syncthreads();
    const int c = threadIdx.x, to = blockIdx.x * 256 + c;
    if (to >= a.m) return;
    float s = 0.f;
#pragma unroll
    for (int l = 0; l < 8; ++l) s += held[l][c >> 3][c & 7];
    a.part[(int64_t)blockIdx.y * a.m + to] = s;
}

constexpr int64_t kMaxElems = INT64_C(1) << 48;
constexpr int32_t kMaxWide = 1 << 24;

int32_t elem_bytes(int32_t dtype) { return dtype == EDB_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == EDB_F32 || dtype == EDB_BF16; }
bool element_aligned(const void* p, int32_t dtype) { return !(reinterpret_cast<uintptr_t>(p) & (elem_bytes(dtype) - 1)); }

Region matrix(const void* p, int32_t dtype, int32_t n, int32_t dim, int64_t stride) {
    return {n > 0 && dim > 0 ? p : nullptr, n, (int64_t)dim * elem_bytes(dtype), stride * elem_bytes(dtype)};
}

edb_status launched(const char* who) {
    const hipError_t he = hipGetLastError();
    if (he != hipSuccess) return fail(EDB_ERR_HIP, std::string(who) + ": " + hipGetErrorString(he));
    edb::clear_error();
    return EDB_OK;
}

edb_status check_sizes(const char* who, int32_t n, int32_t k, int32_t m) {
    const std::string w(who);
    if (n < 0 || k < 1 || m < 1) return fail(EDB_ERR_INVALID, w + ": n >= 0, k >= 1 and m >= 1 are needed");
    if (k > kMaxWide || m > kMaxWide) return fail(EDB_ERR_UNSUPPORTED, w + ": k and m must not exceed 2^24");
    const int64_t wide = k > m ? k : m;
    auto tiles = [](int64_t rows, int64_t cols) { return (rows + 127) / 128 * ((cols + 127) / 128); };
    if (tiles(n, wide) > (1 << 23) || tiles(k, m) > (1 << 23))
        return fail(EDB_ERR_UNSUPPORTED, w + ": a matrix of more than 2^23 tiles of 128 x 128");
    return EDB_OK;
}

edb_status check_matrix(const char* who, const char* name, const void* p, int32_t dtype, int32_t n, int32_t dim, int64_t stride) {
    const std::string w = std::string(who) + ": " + name;
    if (!known(dtype)) return fail(EDB_ERR_INVALID, w + ": dtype must be F32 or BF16");
    if (stride < dim) return fail(EDB_ERR_INVALID, w + ": the row stride is below the row's length");
    if (stride > kMaxElems / (n > 0 ? n : 1)) return fail(EDB_ERR_INVALID, w + ": the rows span more than 2^48 elements");
    if (n && !p) return fail(EDB_ERR_INVALID, w + ": NULL");
    if (!element_aligned(p, dtype)) return fail(EDB_ERR_INVALID, w + ": must be aligned to its elements");
    return EDB_OK;
}

// ---- which tile, and how k is split --------------------------------------------

struct Product {
    int32_t tile, splits, k_per;
    int64_t bytes;                // of the partial sums
};

// Tiles of the products, with what a step of k and the way out of a work-group
// take in us: among as many others as its compute unit holds (busy, a share of
// the unit's time) and from beginning to end (alone).  Fitted to products from
// 1 x 512 x 131072 to 8192^3, whose best tile and split they find within 10%, as
// (bf16, us) 8192^3 256 x 256 907, 256 x 128 1097, 128 x 128 1165; 28629 x 512 x
// 1536 68, 80, 75; 2048 x 512 x 1536 23, 15, 13 and 64 x 64 9.8.
struct Tile {
    int32_t rows, cols, held;     // held: work-groups that a compute unit holds
    double busy, busy_out, alone, alone_out;
};
constexpr int kWide = 2;          // the tile of few rows
constexpr Tile kBf16[5] = {{128, 128, 2, 0.59, 3.3, 0.8, 4.0}, {64, 64, 5, 0.25, 0.2, 0.35, 2.0}, {16, 256, 2, 1.2, 0.0, 1.2, 0.0},
                           {256, 256, 1, 1.77, 10.0, 1.77, 10.0}, {256, 128, 1, 1.04, 5.8, 1.04, 5.8}};
constexpr Tile kF32[3] = {{128, 128, 2, 1.39, 2.5, 2.2, 4.0}, {64, 64, 4, 0.43, 0.3, 1.6, 2.5}, {16, 256, 2, 1.2, 0.0, 1.2, 0.0}};

Product product_plan(int32_t m, int32_t n, int32_t k, int32_t dtype) {
    constexpr int32_t kUnits = 256;
    const int depth = dtype == EDB_BF16 ? 64 : 32, count = dtype == EDB_BF16 ? 5 : 3;
    const Tile* tiles = dtype == EDB_BF16 ? kBf16 : kF32;
    const int64_t steps = ((int64_t)k + depth - 1) / depth;
    const double sums = 8.0 * m * n / 5e6;    // us for a split's sums to be written and read again, at 5 TB/s
    // Few rows of many columns are read as fast as memory gives them by a tile as
    // wide as high ones (1 x 512 x 131072 bf16 22.0 us, by 64 x 64 24.4; fp32 44 and
    // 60), of fewer columns not (16 x 1024 x 1024 fp32 13.6 and 11.9).
    const bool wide = m <= 16 && n >= 16384;
    Product p{kWide, 1, 0, 0};
    double best = 0.0;
    for (int t = 0; t < count; ++t) {
        if ((t == kWide) != wide) continue;
        const Tile& c = tiles[t];
        const int64_t all = (((int64_t)m + c.rows - 1) / c.rows) * (((int64_t)n + c.cols - 1) / c.cols);
        if (all > (1 << 23)) continue;    // a launch has less than 2^32 threads; tiles of 128 x 128 are never more
        // no splits, or such that fill the units one to four times
        int64_t last = 0;
        for (int turns = 0; turns <= 4; ++turns) {
            int64_t splits = turns && all ? kUnits * turns / all : 1;
            if (splits > 64) splits = 64;
            if (turns && splits > steps) splits = steps;
            if (splits <= last) continue;
            last = splits;
            const double each = (double)((steps + splits - 1) / splits), unit = (double)((all * splits + kUnits - 1) / kUnits);
            const double busy = unit * (each * c.busy + c.busy_out),
                         alone = (double)(((int64_t)unit + c.held - 1) / c.held) * (each * c.alone + c.alone_out);
            const double us = (busy > alone ? busy : alone) + (splits > 1 ? 5.0 + splits * sums : 0.0);
            if (best == 0.0 || us < best) {
                best = us;
                p.tile = t;
                p.splits = (int32_t)splits;
            }
        }
    }
    const int64_t per = steps > 0 ? (steps + p.splits - 1) / p.splits : 1;
    p.k_per = (int32_t)(per * depth);
    p.splits = steps > 0 ? (int32_t)((steps + per - 1) / per) : 1;
    p.bytes = p.splits > 1 ? (int64_t)p.splits * m * ((n + 7) / 8 * 8) * 4 : 0;
    return p;
}

template <class T, Layout AL, Layout BL, int TM, int TN, int WM, int WN>
void start(const Args& g, hipStream_t st) {
    const int64_t all = (((int64_t)g.m + TM - 1) / TM) * (((int64_t)g.n + TN - 1) / TN) * g.splits;
    edb::gemm::gemm_kernel<T, AL, BL, TM, TN, WM, WN><<<(unsigned)((all + 7) / 8 * 8), 64 * WM * WN, 0, st>>>(g);
}

template <class T, Layout AL, Layout BL>
void start(const Product& p, const Args& g, hipStream_t st) {
    if (p.tile == 0) start<T, AL, BL, 128, 128, 2, 2>(g, st);
    else if (p.tile == 1) start<T, AL, BL, 64, 64, 2, 2>(g, st);
    else if (p.tile == 2) start<T, AL, BL, 16, 256, 1, 4>(g, st);
    else if constexpr (sizeof(T) == 2) {
        if (p.tile == 3) start<T, AL, BL, 256, 256, 2, 4>(g, st);
        else start<T, AL, BL, 256, 128, 4, 2>(g, st);
    }
}

// C = A B.  a_lines, b_lines: how the operands lie in memory.
void multiply(const Product& p, int32_t dtype, Layout a_lines, Layout b_lines, Args g, void* workspace, hipStream_t st) {
    if (g.m == 0 || g.n == 0) return;
    g.splits = p.splits;
    g.k_per = p.k_per;
    g.partial = static_cast<float*>(workspace);
    auto go = [&](auto one) {
        using T = decltype(one);
        if (a_lines == MN_LINES) start<T, MN_LINES, MN_LINES>(p, g, st);
        else if (b_lines == MN_LINES) start<T, K_LINES, MN_LINES>(p, g, st);
        else start<T, K_LINES, K_LINES>(p, g, st);
    };
    if (dtype == EDB_BF16) go(bf16());
    else go(float());
    if (p.splits > 1) {
        const int64_t pieces = ((int64_t)g.n + 7) / 8 * g.m;
        if (pieces < 65536 && p.splits >= 8) edb::gemm::join_kernel<8><<<(unsigned)((pieces + 31) / 32), 256, 0, st>>>(g);
        else edb::gemm::join_kernel<1><<<(unsigned)((pieces + 255) / 256), 256, 0, st>>>(g);
    }
}

// Scratch memory of the gradients: g, the parts of its columns' sums, the products' partial sums.
struct GradPlan {
    bool own_g, summed;           // summed: the weight's product adds up the bias's gradient
    Product to_dx, to_dw, to_turned;
    int32_t chunks, rows_per;
    int64_t part, partial, bytes;
};

GradPlan grad_plan(int32_t n, int32_t k, int32_t m, int32_t dtype, int32_t dout_dtype, int32_t act, bool dx, bool dw, bool db) {
    GradPlan p{};
    p.own_g = (dx || dw) && (act != EDB_ACT_NONE || dtype != dout_dtype);
    p.summed = db && dw && !p.own_g;
    const int64_t wide = ((int64_t)m + 255) / 256;
    int64_t chunks = (2048 + wide - 1) / wide;
    if (chunks > (n + 31) / 32) chunks = (n + 31) / 32;
    if (chunks > 1024) chunks = 1024;
    if (chunks < 1) chunks = 1;
    p.rows_per = (int32_t)(((int64_t)n + chunks - 1) / chunks);
    p.chunks = p.rows_per ? (int32_t)(((int64_t)n + p.rows_per - 1) / p.rows_per) : 0;
    int64_t at = p.own_g ? (int64_t)n * ((m + 7) / 8 * 8) * elem_bytes(dtype) : 0;
    p.part = at = (at + 15) / 16 * 16;
    int64_t most = 0;
    if (dx) {
        p.to_dx = product_plan(n, k, m, dtype);
        most = p.to_dx.bytes;
    }
    if (dw) {
        // either way round: the weight may be stored output by output
        p.to_dw = product_plan(k, m, n, dtype);
        p.to_turned = product_plan(m, k, n, dtype);
        if (p.to_dw.bytes > most) most = p.to_dw.bytes;
        if (p.to_turned.bytes > most) most = p.to_turned.bytes;
        if (p.summed) p.chunks = p.to_dw.splits > p.to_turned.splits ? p.to_dw.splits : p.to_turned.splits;
    }
    if (db) at += (int64_t)p.chunks * m * 4;
    p.partial = at = (at + 15) / 16 * 16;
    p.bytes = at + most;
    return p;
}

edb_status check_act(const char* who, int32_t act) {
    if (act < EDB_ACT_NONE || act > EDB_ACT_TANH) return fail(EDB_ERR_INVALID, std::string(who) + ": unknown activation");
    return EDB_OK;
}

}  // namespace

extern "C" edb_status edb_linear_bytes(int32_t n, int32_t k, int32_t m, int32_t dtype, int64_t* bytes) {
    return edb::guarded([&]() -> edb_status {
        if (!bytes) return fail(EDB_ERR_INVALID, "edb_linear_bytes: NULL argument");
        if (!known(dtype)) return fail(EDB_ERR_INVALID, "edb_linear_bytes: dtype must be F32 or BF16");
        if (edb_status st = check_sizes("edb_linear_bytes", n, k, m)) return st;
        *bytes = n ? product_plan(n, m, k, dtype).bytes : 0;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_linear_plan(int32_t n, int32_t k, int32_t m, int32_t dtype, int32_t* rows, int32_t* cols, int32_t* splits) {
    return edb::guarded([&]() -> edb_status {
        if (!rows || !cols || !splits) return fail(EDB_ERR_INVALID, "edb_linear_plan: NULL argument");
        if (!known(dtype)) return fail(EDB_ERR_INVALID, "edb_linear_plan: dtype must be F32 or BF16");
        if (edb_status st = check_sizes("edb_linear_plan", n, k, m)) return st;
        const Product p = product_plan(n, m, k, dtype);
        const Tile& t = dtype == EDB_BF16 ? kBf16[p.tile] : kF32[p.tile];
        *rows = t.rows;
        *cols = t.cols;
        *splits = p.splits;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_linear(const void* x, const void* weight, int32_t dtype, int32_t n, int32_t k, int32_t m,
                                 int64_t x_stride, int64_t weight_stride, int32_t turned, const void* bias,
                                 int32_t bias_dtype, int32_t act, const void* residual, int32_t residual_dtype,
                                 int64_t residual_stride, void* out, int32_t out_dtype, int64_t out_stride, void* pre,
                                 int64_t pre_stride, void* workspace, int64_t workspace_bytes, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_linear";
        if (edb_status st = check_sizes(who, n, k, m)) return st;
        if (edb_status st = check_act(who, act)) return st;
        const int32_t lines = turned ? m : k, line = turned ? k : m;
        if (edb_status st = check_matrix(who, "x", x, dtype, n, k, x_stride)) return st;
        if (edb_status st = check_matrix(who, "weight", weight, dtype, lines, line, weight_stride)) return st;
        if (edb_status st = check_matrix(who, "out", out, out_dtype, n, m, out_stride)) return st;
        if (bias && (!known(bias_dtype) || !element_aligned(bias, bias_dtype)))
            return fail(EDB_ERR_INVALID, "edb_linear: bias: F32 or BF16, aligned to its elements, is needed");
        if (residual)
            if (edb_status st = check_matrix(who, "residual", residual, residual_dtype, n, m, residual_stride)) return st;
        if (pre)
            if (edb_status st = check_matrix(who, "pre", pre, dtype, n, m, pre_stride)) return st;
        if (n == 0) {
            edb::clear_error();
            return EDB_OK;
        }
        const Product p = product_plan(n, m, k, dtype);
        const int64_t bytes = p.bytes;
        if (workspace_bytes < bytes || (bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
            return fail(EDB_ERR_INVALID, "edb_linear: a 16-byte aligned workspace of " + std::to_string(bytes) + " bytes is needed");
        const Region in = matrix(x, dtype, n, k, x_stride), w = matrix(weight, dtype, lines, line, weight_stride),
                     shift = Region::array(bias, bias ? (int64_t)m * elem_bytes(bias_dtype) : 0),
                     add = matrix(residual, residual_dtype, n, m, residual_stride), to = matrix(out, out_dtype, n, m, out_stride),
                     before = matrix(pre, dtype, n, m, pre_stride), scratch = Region::array(workspace, bytes);
        if (edb_status st = edb::apart(who, {before, scratch}, {in, w, shift, add, to})) return st;
        if (edb_status st = edb::apart(who, {to}, {in, w, shift})) return st;
        // the residual's place may take the result
        if (residual && !(residual == out && residual_dtype == out_dtype && (n == 1 || residual_stride == out_stride)))
            if (edb_status st = edb::apart(who, {to}, {add})) return st;
        Args g{};
        g.a = x;
        g.b = weight;
        g.a_stride = x_stride;
        g.b_stride = weight_stride;
        g.m = n;
        g.n = m;
        g.k = k;
        g.finish = Finish{bias, residual, residual_stride, out, out_stride, pre, pre_stride, act, bias_dtype == EDB_BF16,
                          residual_dtype == EDB_BF16, out_dtype == EDB_BF16, dtype == EDB_BF16};
        multiply(p, dtype, K_LINES, turned ? K_LINES : MN_LINES, g, workspace, reinterpret_cast<hipStream_t>(stream));
        return launched(who);
    });
}

extern "C" edb_status edb_linear_grad_bytes(int32_t n, int32_t k, int32_t m, int32_t dtype, int32_t dout_dtype, int32_t act,
                                            int32_t results, int64_t* bytes) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_linear_grad_bytes";
        if (!bytes) return fail(EDB_ERR_INVALID, "edb_linear_grad_bytes: NULL argument");
        if (!known(dtype) || !known(dout_dtype)) return fail(EDB_ERR_INVALID, "edb_linear_grad_bytes: dtype must be F32 or BF16");
        if (edb_status st = check_sizes(who, n, k, m)) return st;
        if (edb_status st = check_act(who, act)) return st;
        if (results & ~(EDB_LINEAR_DX | EDB_LINEAR_DWEIGHT | EDB_LINEAR_DBIAS))
            return fail(EDB_ERR_INVALID, "edb_linear_grad_bytes: unknown result");
        *bytes = grad_plan(n, k, m, dtype, dout_dtype, act, results & EDB_LINEAR_DX, results & EDB_LINEAR_DWEIGHT,
                           results & EDB_LINEAR_DBIAS).bytes;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_linear_grad(const void* x, const void* weight, int32_t dtype, int32_t n, int32_t k, int32_t m,
                                      int64_t x_stride, int64_t weight_stride, int32_t turned, const void* dout,
                                      int32_t dout_dtype, int64_t dout_stride, int32_t act, const void* pre,
                                      int64_t pre_stride, void* dx, int64_t dx_stride, void* dweight,
                                      int64_t dweight_stride, float* dbias, void* workspace, int64_t workspace_bytes,
                                      void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_linear_grad";
        if (edb_status st = check_sizes(who, n, k, m)) return st;
        if (edb_status st = check_act(who, act)) return st;
        const int32_t lines = turned ? m : k, line = turned ? k : m;
        if (!known(dtype)) return fail(EDB_ERR_INVALID, "edb_linear_grad: dtype must be F32 or BF16");
        if (edb_status st = check_matrix(who, "dout", dout, dout_dtype, n, m, dout_stride)) return st;
        if (act != EDB_ACT_NONE)
            if (edb_status st = check_matrix(who, "pre", pre, dtype, n, m, pre_stride)) return st;
        if (dweight) {
            if (edb_status st = check_matrix(who, "x", x, dtype, n, k, x_stride)) return st;
            if (edb_status st = check_matrix(who, "dweight", dweight, dtype, lines, line, dweight_stride)) return st;
        }
        if (dx) {
            if (edb_status st = check_matrix(who, "weight", weight, dtype, lines, line, weight_stride)) return st;
            if (edb_status st = check_matrix(who, "dx", dx, dtype, n, k, dx_stride)) return st;
        }
        const GradPlan p = grad_plan(n, k, m, dtype, dout_dtype, act, dx, dweight, dbias);
        if (workspace_bytes < p.bytes || (p.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
            return fail(EDB_ERR_INVALID, "edb_linear_grad: a 16-byte aligned workspace of " + std::to_string(p.bytes) +
                                             " bytes is needed");
        if (!edb::word_aligned({dbias})) return fail(EDB_ERR_INVALID, "edb_linear_grad: dbias must be aligned to 4 bytes");
        if (edb_status st = edb::apart(who,
                                       {matrix(dx, dtype, n, k, dx_stride), matrix(dweight, dtype, lines, line, dweight_stride),
                                        Region::array(dbias, m * INT64_C(4)), Region::array(workspace, p.bytes)},
                                       {matrix(dweight ? x : nullptr, dtype, n, k, x_stride),
                                        matrix(dx ? weight : nullptr, dtype, lines, line, weight_stride),
                                        matrix(dout, dout_dtype, n, m, dout_stride),
                                        matrix(act != EDB_ACT_NONE ? pre : nullptr, dtype, n, m, pre_stride)}))
            return st;
        if ((n == 0 || !dx) && !dweight && !dbias) {
            edb::clear_error();
            return EDB_OK;
        }
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        char* ws = static_cast<char*>(workspace);
        const void* g = p.own_g ? ws : dout;
        const int64_t g_stride = p.own_g ? (m + 7) / 8 * 8 : dout_stride;
        float* part = dbias ? reinterpret_cast<float*>(ws + p.part) : nullptr;
        if (n && (p.own_g || (dbias && !p.summed))) {
            const SlopeArgs s{dout, dout_stride, pre, pre_stride, act, n, m, p.rows_per, p.own_g ? ws : nullptr, part};
            const dim3 grid((unsigned)(((int64_t)m + 255) / 256), (unsigned)p.chunks);
            if (dout_dtype == EDB_F32) {
                if (dtype == EDB_F32) slope_kernel<float, float><<<grid, 256, 0, st>>>(s);
                else slope_kernel<float, bf16><<<grid, 256, 0, st>>>(s);
            } else {
                if (dtype == EDB_F32) slope_kernel<bf16, float><<<grid, 256, 0, st>>>(s);
                else slope_kernel<bf16, bf16><<<grid, 256, 0, st>>>(s);
            }
        }
        if (dbias && !p.summed) edb::join_columns(part, p.chunks, m, 1, dbias, nullptr, st);
        const bool half = dtype == EDB_BF16;
        Args a{};
        a.finish.act = EDB_ACT_NONE;
        a.finish.out_bf16 = half;
        if (dx) {
            a.a = g;
            a.a_stride = g_stride;
            a.b = weight;
            a.b_stride = weight_stride;
            a.m = n;
            a.n = k;
            a.k = m;
            a.finish.out = dx;
            a.finish.out_stride = dx_stride;
            multiply(p.to_dx, dtype, K_LINES, turned ? MN_LINES : K_LINES, a, ws + p.partial, st);
        }
        if (dweight) {
            a.a = turned ? g : x;
            a.a_stride = turned ? g_stride : x_stride;
            a.b = turned ? x : g;
            a.b_stride = turned ? x_stride : g_stride;
            a.m = lines;
            a.n = line;
            a.k = n;
            a.finish.out = dweight;
            a.finish.out_stride = dweight_stride;
            const Product& q = turned ? p.to_turned : p.to_dw;
            if (p.summed) {
                a.sums = turned ? 1 : 2;
                a.sums_out = q.splits > 1 ? part : dbias;
            }
            multiply(q, dtype, MN_LINES, MN_LINES, a, ws + p.partial, st);
            if (p.summed && q.splits > 1) edb::join_columns(part, q.splits, m, 1, dbias, nullptr, st);
        }
        return launched(who);
    });
}
