// Embedding lookup with scaling, and the table's gradient.
//
//   y_i  = s W[id_i]                              (a zero row where id_i is outside [0, V))
//   dW_v = s sum over i with id_i = v of dy_i     (in fp32, the i in ascending order)
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "edb_internal.h"
#include "row_access.h"

using edb::fail;
using namespace edb::rows;

namespace {

// K consecutive elements in registers as fp32: K = 1, or 8 where every row
// starts on 16 bytes and holds whole 16-byte pieces on both sides.
template <class T, int K>
__device__ __forceinline__ void load_k(const T* p, float* v) {
    if constexpr (K == 1) {
        v[0] = Elem<T>::get(p);
    } else {
#pragma unroll
        for (int i = 0; i < K; i += Elem<T>::kVec) Elem<T>::unpack(Elem<T>::load(p + i), v + i);
    }
}
template <class T, int K>
__device__ __forceinline__ void store_k(T* p, const float* v) {
    if constexpr (K == 1) {
        Elem<T>::put(p, v[0]);
    } else {
#pragma unroll
        for (int i = 0; i < K; i += Elem<T>::kVec) Elem<T>::store(p + i, Elem<T>::pack(v + i));
    }
}

struct EmbedArgs {
    const int32_t* ids;
    int32_t n, vocab, dim;
    const void* table;
    int64_t table_stride;
    float scale;
    void* out;
    int64_t out_stride;
};

// One thread per K elements of a row.
template <class T, class O, int K>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
    const int pieces = a.dim / K;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / pieces;
    if (row >= a.n) return;
    const int col = (int)(at - row * pieces) * K, id = a.ids[row];
    float v[K];
    if (id < 0 || id >= a.vocab) {
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] = 0.f;
    } else {
        load_k<T, K>(static_cast<const T*>(a.table) + id * a.table_stride + col, v);
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] *= a.scale;
    }
    store_k<O, K>(static_cast<O*>(a.out) + row * a.out_stride + col, v);
}

struct EmbedGradArgs {
    const int32_t* ids;
    int32_t n, vocab, dim;
    const void* dout;
    int64_t dout_stride;
    float scale;
    int32_t accumulate;
    void* dtable;
    int64_t dtable_stride;
};

// A work-group owns one word and 256 K columns of the gradient and looks
// through all ids.
template <class T, class O, int K>
__global__ __launch_bounds__(256) void embed_grad_kernel(EmbedGradArgs a) {
    const int word = blockIdx.x, col = (blockIdx.y * 256 + threadIdx.x) * K;
    const bool here = col < a.dim;
    float sum[K] = {};
    bool any = false;
    for (int i = 0; i < a.n; ++i) {
        if (a.ids[i] != word) continue;
        any = true;
        if (!here) continue;
        float v[K];
        load_k<T, K>(static_cast<const T*>(a.dout) + i * a.dout_stride + col, v);
#pragma unroll
        for (int k = 0; k < K; ++k) sum[k] += v[k];
    }
    if (!here || (a.accumulate && !any)) return;
    O* d = static_cast<O*>(a.dtable) + word * a.dtable_stride + col;
    float old[K] = {};
    if (a.accumulate) load_k<O, K>(d, old);
#pragma unroll
    for (int k = 0; k < K; ++k) sum[k] = __builtin_fmaf(sum[k], a.scale, old[k]);
    store_k<O, K>(d, sum);
}

int64_t elem_bytes(int32_t dtype) { return dtype == EDB_BF16 ? 2 : 4; }

constexpr int64_t kMaxElems = INT64_C(1) << 48;  // of a matrix, gaps included: offsets in bytes stay far inside 64 bits

// t0, s0: dtype and row stride of the matrix of n rows; t1, s1: of the one of vocab rows.
edb_status check_table(const std::string& who, int32_t n, int32_t vocab, int32_t dim, int32_t t0, int32_t t1,
                       int64_t s0, int64_t s1, float scale) {
    for (int32_t t : {t0, t1})
        if (t != EDB_F32 && t != EDB_BF16) return fail(EDB_ERR_INVALID, who + ": dtype must be F32 or BF16");
    if (n < 0 || vocab < 1 || dim < 1) return fail(EDB_ERR_INVALID, who + ": n >= 0, vocab >= 1 and dim >= 1 are needed");
    if (vocab > (1 << 30) || dim > (1 << 20)) return fail(EDB_ERR_UNSUPPORTED, who + ": vocab up to 2^30 and dim up to 2^20");
    if (s0 < dim || s1 < dim) return fail(EDB_ERR_INVALID, who + ": a row stride is below dim");
    if (s0 > kMaxElems / (n > 0 ? n : 1) || s1 > kMaxElems / vocab)
        return fail(EDB_ERR_INVALID, who + ": a matrix spans more than 2^48 elements");
    if (!std::isfinite(scale)) return fail(EDB_ERR_INVALID, who + ": the scale must be finite");
    return EDB_OK;
}

bool element_aligned(const void* p, int32_t dtype) {
    return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(elem_bytes(dtype) - 1)) == 0;
}

// Whether rows come in whole, aligned 16-byte pieces.
bool pieces16(const void* p, int64_t stride, int32_t dtype) {
    return (reinterpret_cast<uintptr_t>(p) & 15u) == 0 && (stride * elem_bytes(dtype) & 15) == 0;
}

bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

edb_status launched(const char* who) {
    const hipError_t he = hipGetLastError();
    if (he != hipSuccess) return fail(EDB_ERR_HIP, std::string(who) + ": " + hipGetErrorString(he));
    edb::clear_error();
    return EDB_OK;
}

template <class T, class O>
void launch_embed(const EmbedArgs& a, bool wide, hipStream_t st) {
    const int64_t pieces = a.dim / (wide ? 8 : 1);
    const dim3 grid((unsigned)((a.n * pieces + 255) / 256));
    if (wide) embed_kernel<T, O, 8><<<grid, 256, 0, st>>>(a);
    else embed_kernel<T, O, 1><<<grid, 256, 0, st>>>(a);
}

template <class T, class O>
void launch_embed_grad(const EmbedGradArgs& a, bool wide, hipStream_t st) {
    const int pieces = a.dim / (wide ? 8 : 1);
    const dim3 grid(a.vocab, (pieces + 255) / 256);
    if (wide) embed_grad_kernel<T, O, 8><<<grid, 256, 0, st>>>(a);
    else embed_grad_kernel<T, O, 1><<<grid, 256, 0, st>>>(a);
}

}  // namespace

extern "C" edb_status edb_embed(const int32_t* ids, int32_t n, const void* table, int32_t table_dtype, int32_t vocab,
                                int32_t dim, int64_t table_stride, float scale, void* out, int32_t out_dtype,
                                int64_t out_stride, void* stream) {
    const char* who = "edb_embed";
    if (edb_status st = check_table(who, n, vocab, dim, out_dtype, table_dtype, out_stride, table_stride, scale)) return st;
    if (n == 0) {
        edb::clear_error();
        return EDB_OK;
    }
    if (!ids || !table || !out) return fail(EDB_ERR_INVALID, "edb_embed: NULL argument");
    if (!element_aligned(table, table_dtype) || !element_aligned(out, out_dtype))
        return fail(EDB_ERR_INVALID, "edb_embed: the table and the result must be aligned to their elements");
    if (overlap(table, ((vocab - 1) * table_stride + dim) * elem_bytes(table_dtype), out,
                ((n - 1) * out_stride + dim) * elem_bytes(out_dtype)))
        return fail(EDB_ERR_INVALID, "edb_embed: the result overlaps the table");
    if ((int64_t)n * dim > (INT64_C(1) << 38)) return fail(EDB_ERR_UNSUPPORTED, "edb_embed: n * dim exceeds 2^38");
    const EmbedArgs a{ids, n, vocab, dim, table, table_stride, scale, out, out_stride};
    const bool wide = dim % 8 == 0 && pieces16(table, table_stride, table_dtype) && pieces16(out, out_stride, out_dtype);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (table_dtype == EDB_F32) {
        if (out_dtype == EDB_F32) launch_embed<float, float>(a, wide, st);
        else launch_embed<float, bf16>(a, wide, st);
    } else {
        if (out_dtype == EDB_F32) launch_embed<bf16, float>(a, wide, st);
        else launch_embed<bf16, bf16>(a, wide, st);
    }
    return launched(who);
}

extern "C" edb_status edb_embed_grad_bytes(int32_t n, int32_t vocab, int32_t dim, int64_t* bytes) {
    if (!bytes) return fail(EDB_ERR_INVALID, "edb_embed_grad_bytes: NULL argument");
    if (edb_status st = check_table("edb_embed_grad_bytes", n, vocab, dim, EDB_F32, EDB_F32, dim, dim, 1.f)) return st;
    *bytes = 0;
    edb::clear_error();
    return EDB_OK;
}

extern "C" edb_status edb_embed_grad(const int32_t* ids, int32_t n, const void* dout, int32_t dout_dtype, int32_t vocab,
                                     int32_t dim, int64_t dout_stride, float scale, int32_t accumulate, void* dtable,
                                     int32_t dtable_dtype, int64_t dtable_stride, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
    const char* who = "edb_embed_grad";
    if (edb_status st = check_table(who, n, vocab, dim, dout_dtype, dtable_dtype, dout_stride, dtable_stride, scale)) return st;
    (void)workspace;
    (void)workspace_bytes;
    if (!dtable || (n && (!ids || !dout))) return fail(EDB_ERR_INVALID, "edb_embed_grad: NULL argument");
    if (!element_aligned(dout, dout_dtype) || !element_aligned(dtable, dtable_dtype))
        return fail(EDB_ERR_INVALID, "edb_embed_grad: both gradients must be aligned to their elements");
    if (n && overlap(dout, ((n - 1) * dout_stride + dim) * elem_bytes(dout_dtype), dtable,
                     ((vocab - 1) * dtable_stride + dim) * elem_bytes(dtable_dtype)))
        return fail(EDB_ERR_INVALID, "edb_embed_grad: the table's gradient overlaps the rows' gradients");
    const EmbedGradArgs a{ids, n, vocab, dim, dout, dout_stride, scale, accumulate, dtable, dtable_stride};
    const bool wide = dim % 8 == 0 && pieces16(dout, dout_stride, dout_dtype) && pieces16(dtable, dtable_stride, dtable_dtype);
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (dout_dtype == EDB_F32) {
        if (dtable_dtype == EDB_F32) launch_embed_grad<float, float>(a, wide, st);
        else launch_embed_grad<float, bf16>(a, wide, st);
    } else {
        if (dtable_dtype == EDB_F32) launch_embed_grad<bf16, float>(a, wide, st);
        else launch_embed_grad<bf16, bf16>(a, wide, st);
    }
    return launched(who);
}
