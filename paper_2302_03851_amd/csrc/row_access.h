// Typed access to the rows of the operators around the cells (embedding, layer
// norm, linear layers, log probabilities, distillation): elements are fp32 or bf16 in memory and fp32 in
// registers, 16 bytes at a time.  A row of an odd length leaves the next one
// on an element boundary only, so vector accesses state the element's
// alignment; the hardware takes 16-byte accesses at any address.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "edb.h"

namespace edb {
namespace rows {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef u32x2 u32x2_a2 __attribute__((aligned(2)));

struct bf16 {
    uint16_t bits;
};

template <class T>
struct Elem;

template <>
struct Elem<float> {
    static constexpr int kVec = 4;  // elements per 16 bytes
    static constexpr int kDtype = EDB_F32;
    static __device__ __forceinline__ float get(const float* p) { return *p; }
    static __device__ __forceinline__ void put(float* p, float v) { *p = v; }
    static __device__ __forceinline__ u32x4 load(const float* p) { return *reinterpret_cast<const u32x4_a4*>(p); }
    static __device__ __forceinline__ u32x4 load_nt(const float* p) {
        return __builtin_nontemporal_load(reinterpret_cast<const u32x4_a4*>(p));
    }
    static __device__ __forceinline__ void store(float* p, u32x4 v) { *reinterpret_cast<u32x4_a4*>(p) = v; }
    static __device__ __forceinline__ void store_nt(float* p, u32x4 v) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4_a4*>(p));
    }
    static __device__ __forceinline__ void unpack(u32x4 v, float* x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __builtin_bit_cast(float, (uint32_t)v[i]);
    }
    static __device__ __forceinline__ u32x4 pack(const float* x) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(uint32_t, x[i]);
        return v;
    }
};

// bf16 -> fp32 is exact; fp32 -> bf16 rounds to nearest even (the storage
// type's own rounding, once per result).
template <>
struct Elem<bf16> {
    static constexpr int kVec = 8;
    static constexpr int kDtype = EDB_BF16;
    static __device__ __forceinline__ float get(const bf16* p) {
        return __builtin_bit_cast(float, (uint32_t)p->bits << 16);
    }
    static __device__ __forceinline__ uint16_t round(float v) {
        return __builtin_bit_cast(uint16_t, static_cast<__bf16>(v));
    }
    static __device__ __forceinline__ void put(bf16* p, float v) { p->bits = round(v); }
    static __device__ __forceinline__ u32x4 load(const bf16* p) { return *reinterpret_cast<const u32x4_a2*>(p); }
    static __device__ __forceinline__ u32x4 load_nt(const bf16* p) {
        return __builtin_nontemporal_load(reinterpret_cast<const u32x4_a2*>(p));
    }
    static __device__ __forceinline__ void store(bf16* p, u32x4 v) { *reinterpret_cast<u32x4_a2*>(p) = v; }
    static __device__ __forceinline__ void store_nt(bf16* p, u32x4 v) {
        __builtin_nontemporal_store(v, reinterpret_cast<u32x4_a2*>(p));
    }
    static __device__ __forceinline__ void unpack(u32x4 v, float* x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __builtin_bit_cast(float, (uint32_t)v[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, (uint32_t)v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ u32x2 load_half(const bf16* p) { return *reinterpret_cast<const u32x2_a2*>(p); }
    static __device__ __forceinline__ u32x2 load_half_nt(const bf16* p) {
        return __builtin_nontemporal_load(reinterpret_cast<const u32x2_a2*>(p));
    }
    static __device__ __forceinline__ void unpack_half(u32x2 v, float* x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[2 * i] = __builtin_bit_cast(float, (uint32_t)v[i] << 16);
            x[2 * i + 1] = __builtin_bit_cast(float, (uint32_t)v[i] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store_half(bf16* p, const float* x) {
        *reinterpret_cast<u32x2_a2*>(p) = u32x2{pack_pair(x[0], x[1]), pack_pair(x[2], x[3])};
    }
    // one conversion instruction a pair
    static __device__ __forceinline__ uint32_t pack_pair(float a, float b) {
        typedef float f2 __attribute__((ext_vector_type(2)));
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), b2));
    }
    static __device__ __forceinline__ u32x4 pack(const float* x) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pack_pair(x[2 * i], x[2 * i + 1]);
        return v;
    }
};

// K consecutive elements of a row as fp32, at any alignment.  K is 8 or 4, or 1
// for rows shorter than 4.
// ONCE: read once only, not worth a place in the caches.
template <class T, int K, bool ONCE = false>
__device__ __forceinline__ void load_k(const T* p, float* v) {
    if constexpr (K == 1) {
        v[0] = Elem<T>::get(p);
    } else if constexpr (K < Elem<T>::kVec) {
        Elem<T>::unpack_half(ONCE ? Elem<T>::load_half_nt(p) : Elem<T>::load_half(p), v);
    } else {
#pragma unroll
        for (int i = 0; i < K; i += Elem<T>::kVec)
            Elem<T>::unpack(ONCE ? Elem<T>::load_nt(p + i) : Elem<T>::load(p + i), v + i);
    }
}
template <class T, int K>
__device__ __forceinline__ void store_k(T* p, const float* v) {
    if constexpr (K == 1) {
        Elem<T>::put(p, v[0]);
    } else if constexpr (K < Elem<T>::kVec) {
        Elem<T>::store_half(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < K; i += Elem<T>::kVec) Elem<T>::store(p + i, Elem<T>::pack(v + i));
    }
}

// Where the piece of K elements that starts at `nominal` is taken from in a row
// of dim >= K: the last one, if the row ends inside it, from the row's end
// backwards, and the `skip` elements that it shares with the piece before it
// are left to that one (so that no element has two writers).
template <int K>
struct Piece {
    int col, skip;
    __device__ __forceinline__ Piece(int nominal, int dim) : col(min(nominal, dim - K)), skip(nominal - col) {}
};
template <class T, int K>
__device__ __forceinline__ void store_from(T* p, const float* v, int skip) {
    if (K == 1 || skip <= 0) {
        store_k<T, K>(p, v);
    } else {
#pragma unroll
        for (int k = 1; k < K; ++k)
            if (k >= skip) Elem<T>::put(p + k, v[k]);
    }
}

}  // namespace rows
}  // namespace edb
