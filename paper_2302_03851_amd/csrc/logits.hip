// Operators over rows of vocabulary logits: the log probability of a given
// token with the row's entropy and best alternatives, its gradient, and
// distillation from a teacher's listed logits.
//
// With x a row of V logits, T the temperature, m = max_j x_j and
// e_j = exp((x_j - m) / T):  S = sum_j e_j, l = ln S,
//   lp_j = (x_j - m) / T - l,  p_j = exp(lp_j),
//   H    = -sum_j p_j lp_j = l - (sum_j e_j (x_j - m) / T) / S.
// Both terms of H are >= 0, so nothing cancels.  Exponents are taken in base 2
// (y = (x - m) c with c = log2(e) / T, e = 2^y) against a reference that is m c to
// its rounding error (see Stats): l and H are corrected by it, which cancels
// terms of its size, 2^-5 at most, and leaves fp32's rounding of those.  So l and H
// are cut off at 0, below which they cannot lie; log probabilities then stay at
// or below 0.  Sums are fp32.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>
#include <type_traits>

#include "edb_internal.h"
#include "row_access.h"

using edb::fail;
using edb::Region;
using namespace edb::rows;

namespace {

constexpr float kLn2 = 0.69314718055994531f;
// 2^kLow is 0.  Exponents are raised to it where a product with an exponential
// of 0 would be inf * 0 (a logit of -inf, or a difference past the fp32 range).
constexpr float kLow = -1.0e4f;
constexpr float kInf = __builtin_huge_valf();

__device__ __forceinline__ float exp2_hw(float y) { return __builtin_amdgcn_exp2f(y); }  // 0 below 2^-126

// 2^y k from e = 2^(y/2), which is a normal number where 2^y is not: 0 only where the product itself is too small.
__device__ __forceinline__ float squared_times(float e, float k) { return e * (e * k); }

// The value of lane (l ^ D), by data-parallel moves inside rows of 16 lanes.
template <int D>
__device__ __forceinline__ uint32_t from_lane_xor(uint32_t v) {
    if constexpr (D == 4) return from_lane_xor<3>(from_lane_xor<7>(v));
    else if constexpr (D == 1 || D == 2 || D == 3 || D == 7 || D == 8 || D == 15) {
        // quad permutations 1,0,3,2 / 2,3,0,1 / 3,2,1,0, half-row and row mirrors, row rotation by 8
        constexpr int kMove = D == 1 ? 0xb1 : D == 2 ? 0x4e : D == 3 ? 0x1b : D == 7 ? 0x141 : D == 15 ? 0x140 : 0x128;
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kMove, 0xf, 0xf, false);
    } else {
        return (uint32_t)__shfl_xor((int)v, D);
    }
}

template <int D>
__device__ __forceinline__ float from_lane_xor(float v) {
    return __builtin_bit_cast(float, from_lane_xor<D>(__builtin_bit_cast(uint32_t, v)));
}
// Both rows of 16 lanes, or halves of the wave, of which the lane is in one: an
// exchange of rows between two copies, in a few cycles.  (A shuffle through LDS
// takes over a hundred, but fewer instructions where one side is wanted only.)
template <class T>
struct Both {
    T a, b;
};
template <class T>
__device__ __forceinline__ Both<T> both_rows(T v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
    return {__builtin_bit_cast(T, (uint32_t)p[0]), __builtin_bit_cast(T, (uint32_t)p[1])};
}
template <class T>
__device__ __forceinline__ Both<T> both_halves(T v) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return {__builtin_bit_cast(T, (uint32_t)p[0]), __builtin_bit_cast(T, (uint32_t)p[1])};
}
// Over the wave, in every lane; sums in the same order in every run.
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, from_lane_xor<1>(v));
    v = fmaxf(v, from_lane_xor<2>(v));
    v = fmaxf(v, from_lane_xor<7>(v));
    v = fmaxf(v, from_lane_xor<8>(v));
    const auto rows = both_rows(v);
    const auto halves = both_halves(fmaxf(rows.a, rows.b));
    return fmaxf(halves.a, halves.b);
}
__device__ __forceinline__ float wave_sum(float v) {
    v += from_lane_xor<1>(v);
    v += from_lane_xor<2>(v);
    v += from_lane_xor<7>(v);
    v += from_lane_xor<8>(v);
    const auto rows = both_rows(v);
    const auto halves = both_halves(rows.a + rows.b);
    return halves.a + halves.b;
}

// Sums over the lanes up to this one: inside rows of 16, then from row to row.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    auto from = [](uint32_t v, auto move, auto rows) {
        return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(move)::value, decltype(rows)::value, 0xf, false);
    };
    using std::integral_constant;
    constexpr integral_constant<int, 0xf> every;
    v += from(v, integral_constant<int, 0x111>(), every);  // the lane 1, 2, 4, 8 before, 0 from outside the row
    v += from(v, integral_constant<int, 0x112>(), every);
    v += from(v, integral_constant<int, 0x114>(), every);
    v += from(v, integral_constant<int, 0x118>(), every);
    v += from(v, integral_constant<int, 0x142>(), integral_constant<int, 0xa>());  // each row's last lane to the next row
    v += from(v, integral_constant<int, 0x143>(), integral_constant<int, 0xc>());  // lane 31 to the upper half
    return v;
}

// ---- rows of bf16 at odd addresses
//
// A row of an odd number of bf16 leaves the next one 2 bytes off a dword, where
// 16-byte accesses are slow (log probabilities of 8192 x 65533: 227 us so, at
// dwords, 65532, 189).  Such a row is read from the dword before, the vectors of
// a wave being neighbours, and shifted by one element with the next lane's first
// dword (206 us; distillation 505 and 439); it is written from the dword after.
// Which elements a thread holds does not depend on the address, so neither do
// the results.

template <class T>
__device__ __forceinline__ bool odd_row(const T* p) {
    return sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(p) & 2);
}

__device__ __forceinline__ uint32_t from_next_lane(uint32_t v, uint32_t last) {  // `last` in lane 63
    constexpr int kDown = 0x130;  // DPP: every lane takes the value of the one after it
    return (uint32_t)__builtin_amdgcn_update_dpp((int)last, (int)v, kDown, 0xf, 0xf, false);
}

// The elements 0..7 of every lane's vector from the elements -1..6; the low
// half of `last` is element 7 of lane 63.
__device__ __forceinline__ u32x4 shift_in(u32x4 v, uint32_t last) {
    const uint32_t n = from_next_lane(v[0], last);
    return u32x4{__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16),
                 __builtin_amdgcn_alignbit(v[3], v[2], 16), __builtin_amdgcn_alignbit(n, v[3], 16)};
}

// `count` (the same in every lane) neighbouring vectors of a wave, read one
// element early; `last`: the element after the last of them that was read.
template <class T, int M>
__device__ __forceinline__ void shift_in_all(u32x4 (&raw)[M], int count, const T* last) {
    if constexpr (sizeof(T) == 2) {
        const uint32_t end = last->bits;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            if (i < count) {
                uint32_t next = end;
                if (i + 1 < M && i + 1 < count) next = (uint32_t)__builtin_amdgcn_readlane((int)raw[i + 1 < M ? i + 1 : i][0], 0);
                raw[i] = shift_in(raw[i], next);
            }
        }
    }
}

// 16 bytes of a result that is not read again here: past the caches where a
// wave writes whole lines, through them where two waves share some (gradient of
// log probabilities with four vectors a turn, 8192 x 65536 bf16: 397 us past the
// caches, 418 through them; 8192 x 65532: 463 and 436).  Where the caches could hold
// the result, the next kernel pays for it: gradient of 1000 x 65536 and a product
// with it 260 us, written through the caches 247; distillation 263 and 253.
template <class T>
__device__ __forceinline__ void store_piece(T* p, u32x4 v, bool straight) {
    if (straight) {
        Elem<T>::store_nt(p, v);
    } else {
        asm volatile("" ::: "memory");  // these two keep the compiler from making one plain store of both
        Elem<T>::store(p, v);
        asm volatile("" ::: "memory");
    }
}
template <class T>
__device__ __forceinline__ bool straight_row(const T* p) {
    return (reinterpret_cast<uintptr_t>(p) & 127) == 0;
}

// Writes every lane's vector v to d + j (j = the lane's place), up to V; all
// lanes of the wave call it, with neighbouring vectors.
template <class T>
__device__ __forceinline__ void store_vector(T* d, int j, int V, u32x4 v, bool odd, bool straight, int lane) {
    constexpr int N = Elem<T>::kVec;
    if (j >= V && !odd) return;
    if constexpr (sizeof(T) == 2) {
        if (odd) {
            const uint32_t n = from_next_lane(v[0], 0);
            const u32x4 o{__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16),
                          __builtin_amdgcn_alignbit(v[3], v[2], 16), __builtin_amdgcn_alignbit(n, v[3], 16)};
            if (lane == 0 && j < V) d[j].bits = (uint16_t)v[0];
            if (lane != 63 && j + N < V) {
                Elem<T>::store(d + j + 1, o);
            } else {
#pragma unroll
                for (int k = 1; k < N; ++k)
                    if (j + k < V) d[j + k].bits = (uint16_t)(v[k >> 1] >> (16 * (k & 1)));
            }
            return;
        }
    }
    if (j + N <= V) {
        store_piece(d + j, v, straight);
    } else {
        float e[N];
        Elem<T>::unpack(v, e);
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (j + k < V) Elem<T>::put(d + j + k, e[k]);
    }
}

// A lane's 16 bytes of a wave's vector at p, the same in every lane: a scalar
// base and a 32-bit offset, so that a row's many vectors need no address registers.
template <class T>
__device__ __forceinline__ T* lane_place(T* p, int lane) {
    return p + (uint32_t)(lane * (int)(16 / sizeof(T)));
}

template <class T>
__device__ __forceinline__ void store_first(T* d, u32x4 v) {  // the vector's first element
    float e[Elem<T>::kVec];
    Elem<T>::unpack(v, e);
    Elem<T>::put(d, e[0]);
}

template <class T>
__device__ __forceinline__ uint32_t element_bits(const T* p) {
    if constexpr (sizeof(T) == 2) return p->bits;
    else return __builtin_bit_cast(uint32_t, *p);
}

// Writes the elements from 1 on of every lane's vector v at an odd address d (the first lane's), the last lane's too.
template <class T>
__device__ __forceinline__ void store_end(T* d, u32x4 v, int lane) {
    if constexpr (sizeof(T) == 2) {
        const u32x4 o = shift_in(v, 0);
        T* p = lane_place(d, lane) + 1;
        if (lane != 63) {
            Elem<T>::store(p, o);
        } else {
            uint32_t* q = reinterpret_cast<uint32_t*>(p);  // an odd address and one element more: a dword's
            q[0] = o[0];
            q[1] = o[1];
            q[2] = o[2];
            p[6].bits = (uint16_t)(v[3] >> 16);
        }
    }
}

// The vector at place j of a row of V, from `early` (0 or 1) elements before it; -inf past its end.
template <class T>
__device__ __forceinline__ u32x4 load_vector(const T* x, int j, int V, int early) {
    constexpr int N = Elem<T>::kVec;
    if (j - early + N <= V) return Elem<T>::load_nt(x + j - early);
    float e[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int at = j - early + k;
        e[k] = at >= 0 && at < V ? Elem<T>::get(x + at) : -kInf;
    }
    return Elem<T>::pack(e);
}

// Running softmax statistics: the largest logit m, and s = sum 2^y, t = sum y 2^y
// with y = x c - r(m).  The reference r is m c rounded to fp32, so that y is one
// fused multiply-add and its own rounding the only one.  At x = m it leaves the
// rounding error of r there, which has to stay far below 1: from |m c| = 2^20 on
// (where it reaches 2^-5; at 2^32 2^y would leave the fp32 range) r is m c itself
// and y = (x - m) c, which is 0 there.  A NaN or +inf logit makes s NaN.
struct Stats {
    float m, s, t;

    static __device__ __forceinline__ Stats none() { return {-kInf, 0.f, 0.f}; }
    static __device__ __forceinline__ bool plain(float mc) { return fabsf(mc) < 1048576.f; }
    // r(m) - r(to), each rounded or not
    static __device__ __forceinline__ float between(float m, float to, float c) {
        const float a = m * c, b = to * c;
        if (plain(b)) return plain(a) ? a - b : __builtin_fmaf(m, c, -b);
        return plain(a) ? __builtin_fmaf(-to, c, a) : (m - to) * c;
    }
    // the sums taken to the reference of `to`, a number at or above m
    __device__ __forceinline__ void rescale(float to, float c) {
        const float d = fmaxf(between(m, to, c), kLow), f = exp2_hw(d);
        t = (t + s * d) * f;
        s = s * f;
        m = to;
    }
    // N values, with `top` their largest.  `masked` (the same in every lane) says
    // that logits of -inf have come: until then y 2^y is taken as it is, and a NaN
    // in t sends the values through again with y raised to kLow.
    template <int N>
    __device__ __forceinline__ void add(const float* x, float top, float c, bool& masked) {
        const float to = fmaxf(m, top), ref = to == -kInf ? 0.f : to, r = ref * c;
        rescale(ref, c);
        m = to;
        const float s0 = s, t0 = t;
        const bool all_plain = __ballot(!plain(r)) == 0;
        if (all_plain && !masked) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float y = __builtin_fmaf(x[i], c, -r), e = exp2_hw(y);
                s += e;
                t = __builtin_fmaf(y, e, t);
            }
            if (__ballot(t != t) == 0) return;
            masked = true;
            s = s0;
            t = t0;
        }
        if (all_plain) {
#pragma unroll
            for (int i = 0; i < N; ++i) count(__builtin_fmaf(x[i], c, -r));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) count(plain(r) ? __builtin_fmaf(x[i], c, -r) : (x[i] - ref) * c);
        }
    }
    __device__ __forceinline__ void count(float y) {
        const float e = exp2_hw(y);
        s += e;
        t = __builtin_fmaf(fmaxf(y, kLow), e, t);
    }
    // the lanes' statistics joined, in every lane
    __device__ __forceinline__ void join_wave(float c) {
        const float to = wave_max(m);
        rescale(to == -kInf ? 0.f : to, c);
        m = to;
        s = wave_sum(s);
        t = wave_sum(t);
    }
    __device__ __forceinline__ bool empty() const { return m == -kInf && s == 0.f; }
    static __device__ __forceinline__ float not_below_0(float v) { return v < 0.f ? 0.f : v; }  // NaN stays
    // ln sum exp((x - m) / T), 0 for a row that is masked out whole
    __device__ __forceinline__ float log_sum(float c) const {
        const float r = m * c;
        return empty() ? 0.f : not_below_0(plain(r) ? __builtin_fmaf(-kLn2, __builtin_fmaf(m, c, -r), logf(s)) : logf(s));
    }
    __device__ __forceinline__ float entropy() const {
        return empty() ? 0.f : not_below_0(__builtin_fmaf(-kLn2, t / s, logf(s)));
    }
};

template <int N>
__device__ __forceinline__ float largest(const float* x) {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
    return top;
}

// ---- the best entries of a row
//
// An entry (value, index) is a 64-bit key that orders it: larger values first,
// the lowest index first among equal ones (+0 and -0 are equal).  -inf and NaN
// are no entries, key 0.
typedef uint64_t Key;

__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ Key key_of(float v, int j) {
    return v > -kInf ? (Key)ordered(v) << 32 | (uint32_t)~j : 0;
}
__device__ __forceinline__ float key_value(Key k) {
    const uint32_t u = (uint32_t)(k >> 32);
    return __builtin_bit_cast(float, u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_index(Key k) { return (int)~(uint32_t)k; }

// Lanes l and l ^ D end with their larger key in the lower lane.
template <int D>
__device__ __forceinline__ Key order_with(Key k, int lane) {
    constexpr int kHigh = D & 32 ? 32 : D & 16 ? 16 : D & 8 ? 8 : D & 4 ? 4 : D & 2 ? 2 : 1;
    const Key o = (Key)from_lane_xor<D>((uint32_t)(k >> 32)) << 32 | from_lane_xor<D>((uint32_t)k);
    return (o > k) == ((lane & kHigh) == 0) ? o : k;
}

// Sorts a wave's keys, the largest in lane 0 (bitonic, the first step of every
// merge against the mirrored half, so that all steps order the same way).
__device__ __forceinline__ Key merge_down(Key k, int lane) {  // of a bitonic sequence over the wave
    k = order_with<32>(k, lane);
    k = order_with<16>(k, lane);
    k = order_with<8>(k, lane);
    k = order_with<4>(k, lane);
    k = order_with<2>(k, lane);
    return order_with<1>(k, lane);
}
template <int D>
__device__ __forceinline__ uint32_t order_with(uint32_t k, int lane) {
    constexpr int kHigh = D & 32 ? 32 : D & 16 ? 16 : D & 8 ? 8 : D & 4 ? 4 : D & 2 ? 2 : 1;
    const uint32_t o = from_lane_xor<D>(k);
    return (lane & kHigh) == 0 ? max(o, k) : min(o, k);
}

// `first`: the lanes (the same number everywhere) from which on all keys are 0.
template <class K>
__device__ __forceinline__ K sort_down(K k, int lane, int first = 64) {
    k = order_with<1>(k, lane);
    k = order_with<3>(k, lane);
    k = order_with<1>(k, lane);
    k = order_with<7>(k, lane);
    k = order_with<2>(k, lane);
    k = order_with<1>(k, lane);
    k = order_with<15>(k, lane);
    k = order_with<4>(k, lane);
    k = order_with<2>(k, lane);
    k = order_with<1>(k, lane);
    if (first <= 16) return k;
    k = order_with<31>(k, lane);
    k = order_with<8>(k, lane);
    k = order_with<4>(k, lane);
    k = order_with<2>(k, lane);
    k = order_with<1>(k, lane);
    if (first <= 32) return k;
    k = order_with<63>(k, lane);
    k = order_with<16>(k, lane);
    k = order_with<8>(k, lane);
    k = order_with<4>(k, lane);
    k = order_with<2>(k, lane);
    return order_with<1>(k, lane);
}

// The best entries among those pushed by a wave, sorted, lane i holding the i-th.
// Pushed entries wait in LDS until `sort` puts them into the list.  Sorting is
// a few hundred instructions, so it stands where a loop comes by, not behind
// every push.
constexpr int kWait = 320;

struct Best {
    Key key = 0;
    int waiting = 0;
    uint32_t bound;  // order of a value that at least `top` entries reach

    // A bound from the orders of values of different entries, four a lane (0 for
    // none): for short lists the top-th largest of the lanes' own largest (for very
    // short ones of four lanes' each, which takes half the sorting), else
    // the top-th largest of all, its lower 16 bits left open.
    __device__ __forceinline__ static uint32_t bound_of(const uint32_t (&u)[4], int top, int lane) {
        if (top <= 8) {  // of 16 values, each the largest of four lanes
            const auto rows = both_rows(max(max(u[0], u[1]), max(u[2], u[3])));
            const auto halves = both_halves(max(rows.a, rows.b));
            const uint32_t all = max(halves.a, halves.b);
            return (uint32_t)__builtin_amdgcn_readlane((int)sort_down(all, lane, 16), top - 1);
        }
        if (top <= 32)
            return (uint32_t)__builtin_amdgcn_readlane((int)sort_down(max(max(u[0], u[1]), max(u[2], u[3])), lane), top - 1);
        uint32_t b = 0;
#pragma unroll
        for (int bit = 31; bit >= 16; --bit) {
            const uint32_t t = b | 1u << bit;
            int n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(u[i] >= t));
            if (n >= top) b = t;
        }
        return b;
    }
    // the least value that reaches the bound
    __device__ __forceinline__ float bound_value() const { return bound ? key_value((Key)bound << 32) : -kInf; }
    __device__ __forceinline__ Key key_at(int lane) const {  // lane: the same in every lane
        return (Key)(uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), lane) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((int)key, lane);
    }
    // the least value that an entry can have and reach the bound
    __device__ __forceinline__ float least() const { return fmaxf(bound_value(), -__FLT_MAX__); }
    // One entry a lane, 0 for none; at most kWait - 64 wait already.
    __device__ __forceinline__ void push(Key k, Key* wait, int lane) {
        const uint64_t who = __ballot(k && (uint32_t)(k >> 32) >= bound);
        if (!who) return;
        if ((who >> lane) & 1) wait[waiting + __popcll(who & ((1ull << lane) - 1))] = k;
        waiting += __popcll(who);
    }
    __device__ __forceinline__ void sort(const Key* wait, int top, int lane) {
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int i = 0; i < waiting; i += 64) {
            Key k = sort_down(i + lane < waiting ? wait[i + lane] : 0, lane, waiting - i);
            if (key_at(0)) {  // the larger ones of the list and the mirrored newcomers: a bitonic sequence
                const Key o = (Key)from_lane_xor<63>((uint32_t)(k >> 32)) << 32 | from_lane_xor<63>((uint32_t)k);
                k = merge_down(o > key ? o : key, lane);
            }
            key = k;
        }
        waiting = 0;
        bound = max(bound, (uint32_t)(key_at(top - 1) >> 32));
        __builtin_amdgcn_wave_barrier();
    }
};

struct LogprobArgs {
    const void* logits;
    int64_t stride;
    int32_t n, vocab;
    const int32_t* ids;
    float c, inv_t;
    int32_t top;
    float *logprob, *entropy, *stats;
    int32_t* top_ids;
    float* top_logprobs;
    int32_t part, parts;  // a row is split into `parts` parts of `part` logits
    Stats* part_stats;    // [n][parts]
    Key* part_keys;       // [n][parts][top]
};

__device__ __forceinline__ void put_left_out(const LogprobArgs& a, int64_t row, int lane) {
    if (lane < a.top) {
        a.top_ids[row * a.top + lane] = -1;
        a.top_logprobs[row * a.top + lane] = -kInf;
    }
    if (lane == 0) {
        if (a.logprob) a.logprob[row] = 0.f;
        if (a.entropy) a.entropy[row] = 0.f;
        if (a.stats) a.stats[2 * row] = a.stats[2 * row + 1] = 0.f;
    }
}

// The results of a row from its joined statistics and best entries (one wave).
__device__ __forceinline__ void put_row(const LogprobArgs& a, int64_t row, const Stats& st, Key best, float given,
                                        int lane) {
    const float l = st.log_sum(a.c), ref = st.empty() ? 0.f : st.m;
    if (lane < a.top) {
        a.top_ids[row * a.top + lane] = best ? key_index(best) : -1;
        a.top_logprobs[row * a.top + lane] = best ? (key_value(best) - ref) * a.inv_t - l : -kInf;
    }
    if (lane == 0) {
        if (a.logprob) a.logprob[row] = (given - ref) * a.inv_t - l;
        if (a.entropy) a.entropy[row] = st.entropy();
        if (a.stats) {
            const bool none = st.s != st.s;
            a.stats[2 * row] = none ? st.s : st.m;
            a.stats[2 * row + 1] = l;
        }
    }
}

// A quad is four neighbouring lanes: together they load 64 bytes of the row.
__device__ __forceinline__ float quad_max(float v) {
    v = fmaxf(v, from_lane_xor<1>(v));
    return fmaxf(v, from_lane_xor<2>(v));
}

constexpr int kLoads = 2;  // 16-byte loads of a thread in flight, beside as many at work

// A work-group takes a row (a part of it past 131072 logits) in one pass, 16
// bytes a load: per logit a difference, an exponential and two sums against the
// running maximum (see Stats).  For the alternatives each quad of lanes leaves
// the largest of its 64 bytes in LDS: the best `top` logits lie in the best
// `top` of these groups (a group that does not belong to them has `top` groups
// with a better logit before it), so at the end one wave looks for those groups
// and reads them again.  Memory bound where there are many logits: 8192 x 65536
// bf16, 1.07 GB, 171 us without alternatives (6.3 TB/s), 178 with 5, 204 with
// 63.  Few or short rows are bound by the chain of steps of the choice, about 3
// us a row and wave: 23 x 3801 bf16 4 us, 7 with 5 alternatives.
// (W: row_waves; at most 64 registers, for eight waves a SIMD: 4381 x 4108 fp32,
// 5 alternatives, 21 us, without the limit 25)
template <class T, bool TOP, int W>
__global__ __launch_bounds__(64 * W, 8) void logprobs_kernel(LogprobArgs a) {
    constexpr int N = Elem<T>::kVec, kStep = kLoads * W * 64 * N;
    extern __shared__ float group_max[];
    __shared__ float part_m[W], part_s[W], part_t[W];
    __shared__ Key wait[TOP ? kWait : 1];
    const int64_t row = blockIdx.x / a.parts;
    const int which = blockIdx.x - (int)row * a.parts;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    const int V = a.vocab, begin = which * a.part, end = min(V, begin + a.part);
    const int id = a.ids ? a.ids[row] : 0;
    int j = begin + (wave * kLoads * 64 + lane) * N;  // a wave's loads are neighbours
    const int whole = (end - begin) / kStep;
    const bool odd = odd_row(x);
    const T* from = x - (odd ? 1 : 0);
    u32x4 raw[kLoads];
    if (whole > 0) {
#pragma unroll
        for (int u = 0; u < kLoads; ++u) raw[u] = Elem<T>::load_nt(from + j + u * 64 * N);
    }
    if (id < 0 || id >= V) {
        if (a.parts == 1 && wave == 0) put_left_out(a, row, lane);
        return;
    }
    const float given = a.ids ? Elem<T>::get(x + id) : 0.f;
    Stats st = Stats::none();
    bool masked = false;
    auto use = [&](const float(&v)[kLoads][N]) {
        float top[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) top[u] = largest<N>(v[u]);
        st.add<kLoads * N>(&v[0][0], largest<kLoads>(top), a.c, masked);
        if constexpr (TOP) {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const float q = quad_max(top[u]);
                if ((lane & 3) == 0 && j + u * 64 * N < end) group_max[(j + u * 64 * N - begin) / (4 * N)] = q;
            }
        }
    };
    for (int i = 0; i < whole; ++i) {
        float v[kLoads][N];
        if (odd) shift_in_all(raw, kLoads, x + j + (kLoads * 64 - lane) * N - 1);
#pragma unroll
        for (int u = 0; u < kLoads; ++u) Elem<T>::unpack(raw[u], v[u]);
        if (i + 1 < whole) {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) raw[u] = Elem<T>::load_nt(from + j + kStep + u * 64 * N);
        }
        use(v);
        j += kStep;
    }
    if (begin + whole * kStep < end) {
        float v[kLoads][N];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) {
            const int k = j + u * 64 * N;
            if (k + N <= end) {
                Elem<T>::unpack(Elem<T>::load(x + k), v[u]);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) v[u][i] = k + i < end ? Elem<T>::get(x + k + i) : -kInf;
            }
        }
        use(v);
    }
    st.join_wave(a.c);
    if constexpr (W > 1) {
        if (lane == 0) {
            part_m[wave] = st.m;
            part_s[wave] = st.s;
            part_t[wave] = st.t;
        }
        __syncthreads();
        if (wave) return;
        st = lane < W ? Stats{part_m[lane], part_s[lane], part_t[lane]} : Stats::none();
        st.join_wave(a.c);
    } else {
        __builtin_amdgcn_wave_barrier();
    }
    Best best;
    if constexpr (TOP) {
        constexpr int kGroup = 4 * N;  // logits
        const int n = (end - begin + kGroup - 1) / kGroup;
        // kLook x 256 groups at a time, more where rows are longer, all on their way before the first is looked at
        constexpr int kLook = W == 1 ? 1 : W == 4 ? 2 : 4;
        float w[kLook][4];
        auto look = [&](int i0) {
#pragma unroll
            for (int c = 0; c < kLook; ++c)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = i0 + (c * 4 + u) * 64 + lane;
                    w[c][u] = -kInf;
                    if (i0 + c * 256 < n) w[c][u] = i < n ? group_max[min(i, n - 1)] : -kInf;
                }
        };
        float own[4] = {-kInf, -kInf, -kInf, -kInf};
        for (int i0 = 0; i0 < n; i0 += kLook * 256) {
            look(i0);
#pragma unroll
            for (int c = 0; c < kLook; ++c)
                if (i0 + c * 256 < n) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) own[u] = fmaxf(own[u], w[c][u]);
                }
        }
        uint32_t order[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) order[u] = own[u] > -kInf ? ordered(own[u]) : 0;
        Best groups;
        groups.bound = Best::bound_of(order, a.top, lane);
        for (int i0 = 0; i0 < n; i0 += kLook * 256) {
            if (n > kLook * 256) look(i0);
            const float least = groups.least();
            uint32_t reach = 0;
#pragma unroll
            for (int c = 0; c < kLook; ++c)
                if (i0 + c * 256 < n) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) reach |= (w[c][u] >= least ? 1u : 0u) << (c * 4 + u);
                }
            const uint32_t upto = wave_scan(__popc(reach));
            const int all = __builtin_amdgcn_readlane((int)upto, 63);
            if (all == 0) continue;
            if (groups.waiting + all <= kWait) {
                int to = groups.waiting + (int)(upto - __popc(reach));
#pragma unroll
                for (int c = 0; c < kLook; ++c)
                    if (i0 + c * 256 < n) {
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if ((reach >> (c * 4 + u)) & 1) wait[to++] = key_of(w[c][u], i0 + (c * 4 + u) * 64 + lane);
                    }
                groups.waiting += all;
            } else {  // many equal ones: 64 at a time
                if (groups.waiting > kWait - 64) groups.sort(wait, a.top, lane);  // as many as push() expects
                for (int i = i0 + lane; i - lane < min(n, i0 + kLook * 256); i += 64) {
                    groups.push(i < n ? key_of(group_max[i], i) : 0, wait, lane);
                    if (groups.waiting > kWait - 64) groups.sort(wait, a.top, lane);
                }
            }
        }
        if (groups.waiting > 64 || groups.key_at(0)) groups.sort(wait, a.top, lane);
        // up to 64 groups reach the bound: all of them are read again; more: the best ones
        int there = groups.waiting;
        __builtin_amdgcn_wave_barrier();
        int mine = lane < there ? key_index(wait[lane]) : 0;
        if (groups.key_at(0)) {
            there = __popcll(__ballot(lane < a.top && groups.key));
            mine = key_index(groups.key);
        }
        __builtin_amdgcn_wave_barrier();
        best.bound = groups.bound;
        // 16 groups a load, all of them on their way before the first is looked at
        constexpr uint32_t kNone = N == 4 ? 0xff800000u : 0xff80ff80u;  // -inf
        u32x4 again[4];
        int at[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int g = u * 16 + lane / 4;
            at[u] = begin + __shfl(mine, g) * kGroup + lane % 4 * N;
            again[u] = u32x4{kNone, kNone, kNone, kNone};
            if (g < there && at[u] < end) {
                if (at[u] + N <= end) {
                    again[u] = Elem<T>::load(x + at[u]);
                } else {
                    float w[N];
#pragma unroll
                    for (int k = 0; k < N; ++k) w[k] = at[u] + k < end ? Elem<T>::get(x + at[u] + k) : -kInf;
                    again[u] = Elem<T>::pack(w);
                }
            }
        }
        if (there > 32 || 2 * n < 3 * a.top) {  // a closer bound from the loads' own largest values: fewer entries to sort
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                float w[N];
                Elem<T>::unpack(again[u], w);
                const float most = largest<N>(w);
                order[u] = most > -kInf ? ordered(most) : 0;
                asm volatile("" : "+v"(again[u]));  // unpacked anew below: the values would take too many registers
            }
            best.bound = max(best.bound, Best::bound_of(order, a.top, lane));
        }
        // the entries that reach the bound, a bit each; their places in the list follow from the lanes' counts
        const float least = best.least();
        uint32_t reach = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (u * 16 < there) {
                float w[N];
                Elem<T>::unpack(again[u], w);
#pragma unroll
                for (int k = 0; k < N; ++k) reach |= (w[k] >= least ? 1u : 0u) << (u * N + k);
                asm volatile("" : "+v"(again[u]));
            }
        const uint32_t upto = wave_scan(__popc(reach));
        const int all = __builtin_amdgcn_readlane((int)upto, 63);
        const bool many = all > kWait;  // equal ones: 256 at a time
        if (!many) {
            int to = (int)(upto - __popc(reach));
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (u * 16 < there) {
                    float w[N];
                    Elem<T>::unpack(again[u], w);
#pragma unroll
                    for (int k = 0; k < N; ++k)
                        if ((reach >> (u * N + k)) & 1) wait[to++] = key_of(w[k], at[u] + k);
                }
            best.waiting = all;
        }
        int i0 = 0;
        do {
            if (many) {
                float w[4];
                int j[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int g = i0 + (u * 64 + lane) / kGroup;
                    j[u] = begin + __shfl(mine, g & 63) * kGroup + lane % kGroup;
                    w[u] = g < there && j[u] < end ? Elem<T>::get(x + j[u]) : -kInf;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) best.push(key_of(w[u], j[u]), wait, lane);
                i0 += 256 / kGroup;
            } else {
                i0 = there;
            }
            if (i0 >= there || best.waiting > kWait - 256) best.sort(wait, a.top, lane);
        } while (i0 < there);
    }
    if (a.parts == 1) {
        put_row(a, row, st, best.key, given, lane);
    } else {
        const int64_t at = row * a.parts + which;
        if (lane == 0) a.part_stats[at] = st;
        if (lane < a.top) a.part_keys[at * a.top + lane] = best.key;
    }
}

// The statistics of a row's parts joined, in every lane of the wave.
__device__ __forceinline__ Stats join_parts(const Stats* part, int parts, float c, int lane) {
    Stats st = lane < parts ? part[lane] : Stats::none();
    st.join_wave(c);
    for (int i0 = 64; i0 < parts; i0 += 63) {  // lane 63 carries the parts before these
        if (lane != 63) st = i0 + lane < parts ? part[i0 + lane] : Stats::none();
        st.join_wave(c);
    }
    return st;
}

// Joins the parts of split rows: a wave a row; bound by its chain of loads and
// steps, 4 us for the 32 parts of 1 x 131072 with 8 alternatives.
template <class T>
__global__ __launch_bounds__(64) void logprobs_join(LogprobArgs a) {
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    const int id = a.ids ? a.ids[row] : 0;
    if (id < 0 || id >= a.vocab) {
        put_left_out(a, row, lane);
        return;
    }
    const float given = a.ids ? Elem<T>::get(static_cast<const T*>(a.logits) + row * a.stride + id) : 0.f;
    const Stats st = join_parts(a.part_stats + row * a.parts, a.parts, a.c, lane);
    Best best;
    if (a.top) {
        __shared__ Key wait[kWait];
        const Key* keys = a.part_keys + row * a.parts * a.top;
        const int n = a.parts * a.top;
        // bounds: every part's last entry, and the lanes' own largest ones
        Key k[4][4];
        auto look = [&](int i0) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = i0 + (c * 4 + u) * 64 + lane;
                    k[c][u] = 0;
                    if (i0 + c * 256 < n) k[c][u] = i < n ? keys[i] : 0;
                }
        };
        uint32_t own[4] = {}, last = 0;
        for (int i0 = 0; i0 < n; i0 += 1024) {
            look(i0);
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int u = 0; u < 4; ++u) own[u] = max(own[u], (uint32_t)(k[c][u] >> 32));
        }
        for (int i = lane; i < a.parts; i += 64) last = max(last, (uint32_t)(keys[(i + 1) * a.top - 1] >> 32));
        for (int d = 1; d < 64; d <<= 1) last = max(last, (uint32_t)__shfl_xor((int)last, d));
        best.bound = max(last, Best::bound_of(own, a.top, lane));
        for (int i0 = 0; i0 < n; i0 += 1024) {
            if (n > 1024) look(i0);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (i0 + c * 256 >= n) break;
#pragma unroll
                for (int u = 0; u < 4; ++u) best.push(k[c][u], wait, lane);
                if (best.waiting > 64) best.sort(wait, a.top, lane);
            }
        }
        best.sort(wait, a.top, lane);
    }
    put_row(a, row, st, best.key, given, lane);
}

template <class T>
__device__ __forceinline__ void zero_row(T* d, int V, int threads, int before = 0) {
    constexpr int N = Elem<T>::kVec;
    for (int j = (before + threadIdx.x) * N; j < V; j += threads * N) {
        if (j + N <= V) Elem<T>::store(d + j, u32x4{0u, 0u, 0u, 0u});
        else
            for (int k = j; k < V; ++k) Elem<T>::put(d + k, 0.f);
    }
}

struct GradArgs {
    const void* logits;
    int64_t stride;
    int32_t n, vocab;
    const int32_t* ids;
    float c, inv_t;
    const float *stats, *entropy, *g_logprob, *g_entropy;
    void* out;
    int64_t out_stride;
};

// dx_j = (g_lp (1[j = id] - p_j) - g_H p_j (lp_j + H)) / T, in one pass that
// takes p_j from the row's statistics.  The waves of a row's work-groups (several
// in y where there are few rows: 2 x 131072 bf16 4 us, by one each 15) take LOADS
// neighbouring vectors of 1 KB in turn: eight, of which fewer begin or end in a
// line that two waves write (8192 x 65533: 422 us, with four 432), or four where
// rows are few (300 x 10007 fp32: 6.4 us, with eight 6.9).  Memory bound: 8192 x
// 65536 bf16, read and written, 2.15 GB, 385 us (5.6 TB/s; a copy reaches 5.4).
constexpr int kGradWaves = 8;  // waves of a work-group at most

template <class T, int LOADS, bool CACHED>
__global__ __launch_bounds__(64 * kGradWaves) void logprobs_grad_kernel(GradArgs a) {
    constexpr int N = Elem<T>::kVec, kAll = 64 * N;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    T* d = static_cast<T*>(a.out) + row * a.out_stride;
    const int V = a.vocab, id = a.ids[row];
    const float g1 = a.g_logprob ? a.g_logprob[row] * a.inv_t : 0.f, g2 = a.g_entropy ? a.g_entropy[row] * a.inv_t : 0.f;
    const float m = a.stats[2 * row], l2 = a.stats[2 * row + 1] * (1.f / kLn2);
    if (id < 0 || id >= V || (g1 == 0.f && g2 == 0.f) || m == -kInf) {
        zero_row(d, V, gridDim.y * blockDim.x, blockIdx.y * blockDim.x);
        return;
    }
    // p (k0 + k1 log2 p / 2), k0 = -(g_lp + g_H H) / T, k1 = -2 g_H ln 2 / T
    const float k0 = -(g1 + (a.g_entropy ? g2 * a.entropy[row] : 0.f)), k1 = -2.f * (g2 * kLn2);
    const float half_c = 0.5f * a.c, half_l2 = 0.5f * l2;
    const bool odd = odd_row(x), odd_out = odd_row(d), straight = straight_row(d);
    auto slope = [&](u32x4 q, int j) {
        float v[N];
        Elem<T>::unpack(q, v);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = __builtin_fmaf(v[i] - m, half_c, -half_l2), e = exp2_hw(y);
            v[i] = squared_times(e, __builtin_fmaf(k1, fmaxf(y, kLow), k0));
        }
        const int at = id - j;
        if (at >= 0 && at < N) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += i == at ? g1 : 0.f;
        }
        return Elem<T>::pack(v);
    };
    const int all = V / kAll;
    const T* from = x - (odd ? 1 : 0);
    const int waves = blockDim.x >> 6, turn = blockIdx.y * waves + wave, turns = gridDim.y * waves;
    for (int g = turn * LOADS; g < all; g += turns * LOADS) {
        const int count = min(LOADS, all - g);
        u32x4 raw[LOADS];
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            const T* at = lane_place(from + min(g + u, all - 1) * kAll, lane);
            raw[u] = CACHED ? Elem<T>::load(at) : Elem<T>::load_nt(at);
        }
        if (odd) shift_in_all(raw, count, x + (g + count) * kAll - 1);
        u32x4 held{0u, 0u, 0u, 0u};
#pragma unroll
        for (int u = 0; u < LOADS; ++u) {
            if (u >= count) break;
            const u32x4 o = slope(raw[u], (g + u) * kAll + lane * N);
            T* at = d + (g + u) * kAll;
            if (!odd_out) {
                store_piece(lane_place(at, lane), o, straight);
            } else {
                if (u == 0) {
                    if (lane == 0) store_first(at, o);
                } else {
                    Elem<T>::store(lane_place(at - kAll + 1, lane),
                                   shift_in(held, (uint32_t)__builtin_amdgcn_readlane((int)o[0], 0)));
                }
                if (u + 1 == count) store_end(at, o, lane);
                held = o;
            }
        }
    }
    if (V % kAll != 0 && all / LOADS % turns == turn) {
        const int j = all * kAll + lane * N;
        u32x4 q = load_vector(x, j, V, odd ? 1 : 0);
        if (odd) q = shift_in(q, 0);
        store_vector(d, j, V, slope(q, j), odd_out, straight, lane);
    }
}

constexpr int kMaxListed = EDB_DISTILL_MAX_TOP;

struct DistillArgs {
    const void* logits;
    int64_t stride;
    int32_t n, vocab;
    const int32_t* top_ids;
    const float* top_logits;
    int32_t top;
    float c, inv_t, t;
    const float* weight;
    float* loss;
    void* out;
    int64_t out_stride;
    bool cached;          // all logits fit the caches of the memory side
    int32_t part, parts;  // a split row: `parts` parts of `part` logits
    Stats* part_stats;    // [n][parts]
    float* listed;        // [n][top]: the student's logits at the listed tokens
};

// The teacher's list of a row as masses: one entry a thread (the first
// kMaxListed threads), equal ids as one, at the first of them.
struct Listed {
    int id;      // -1: nothing to account for here
    float mass;
};

constexpr int kTable = 2 * kMaxListed;

struct ListedShared {
    int ids[kMaxListed];
    float q[kMaxListed];
    float part[2][kMaxListed / 64];
    int table[kTable];
    int twice;
};

// Called by all waves of the work-group (four at least); `total` is 0 where
// nothing is listed.  A table of the ids tells whether one comes twice; only
// then does every entry look through the others.
__device__ __forceinline__ Listed take_list(const DistillArgs& a, int id, float u, ListedShared& sh, float& total) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    constexpr int kWaves = kMaxListed / 64;
    const float um = wave_max(u);
    if (lane == 0 && wave < kWaves) sh.part[0][wave] = um;
    for (int i = tid; i < kTable; i += blockDim.x) sh.table[i] = -1;
    if (tid == 0) sh.twice = 0;
    __syncthreads();
    float tm = sh.part[0][0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) tm = fmaxf(tm, sh.part[0][i]);
    const float e = id < 0 ? 0.f : exp2_hw((u - (tm == -kInf ? 0.f : tm)) * a.c);
    const float es = wave_sum(e);
    if (lane == 0 && wave < kWaves) sh.part[1][wave] = es;
    if (id >= 0) {
        // at most half of the places are taken: the search ends at a free one
        for (uint32_t at = (uint32_t)id * 2654435761u >> 16;; ++at) {
            const int before = atomicCAS(&sh.table[at & (kTable - 1)], -1, id);
            if (before == id) sh.twice = 1;
            if (before == id || before == -1) break;
        }
    }
    __syncthreads();
    total = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) total += sh.part[1][i];
    Listed l{total == 0.f ? -1 : id, e / total};
    if (!sh.twice) return l;
    if (tid < kMaxListed) {
        sh.ids[tid] = id;
        sh.q[tid] = l.mass;
    }
    __syncthreads();
    if (l.id >= 0) {
        l.mass = 0.f;
        for (int k = 0; k < a.top; ++k)
            if (sh.ids[k] == id) {
                if (k < tid) l.id = -1;
                l.mass += sh.q[k];
            }
    }
    return l;
}

__device__ __forceinline__ void read_list(const DistillArgs& a, int64_t row, int& id, float& u) {
    id = -1;
    u = -kInf;
    if ((int)threadIdx.x < a.top) {
        id = a.top_ids[row * a.top + threadIdx.x];
        const float v = a.top_logits[row * a.top + threadIdx.x];
        if (id < 0 || id >= a.vocab) id = -1;
        else u = v;
    }
}

// The row's loss: the sum of the listed entries' terms, in the same order in every run.
template <int W>
__device__ __forceinline__ void put_loss(const DistillArgs& a, int64_t row, const Listed& l, float lp, float* part) {
    float each = l.id >= 0 && !(l.mass == 0.f) ? l.mass * (logf(l.mass) - lp) : 0.f;
    each = wave_sum(each);
    constexpr int kWaves = kMaxListed / 64 < W ? kMaxListed / 64 : W;
    if ((threadIdx.x & 63) == 0 && (int)(threadIdx.x >> 6) < kWaves) part[threadIdx.x >> 6] = each;
    __syncthreads();
    if (threadIdx.x == 0) {
        float sum = 0.f;
        for (int i = 0; i < kWaves; ++i) sum += part[i];
        a.loss[row] = a.t * (a.t * sum);  // T^2 can leave fp32's range where the loss does not
    }
}

// W waves hold a whole row in registers, up to NV 16-byte vectors a thread, so
// that it is read once and the gradient written once.  2^y with y = x c - r(m)
// (see Stats) is summed up in one pass over the registers, w T p_j = 2^y (w T / S)
// written in another; the owners of the listed entries then write
// w T (p_j - q_j).  Memory bound with many rows: 8192 x 65536 bf16, 2.15 GB, 383
// us (5.6 TB/s); 4096 x 131072 453 (4.7), where a row fills the registers of a
// compute unit, so that no other one is read while it is summed up; the chain of
// these steps with few: 128 x 8192 fp32 6 us.
constexpr int kBlock = 2;

template <class T, int W, int NV, bool CACHED>
__global__ __launch_bounds__(64 * W) void distill_kernel(DistillArgs a) {
    constexpr int N = Elem<T>::kVec, kThreads = 64 * W, kAll = 64 * N;  // elements of a wave's vector
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int V = a.vocab;
    __shared__ ListedShared sh;
    __shared__ float part[3][W];
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    T* d = a.out ? static_cast<T*>(a.out) + row * a.out_stride : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (tid == 0) a.loss[row] = 0.f;
        if (d) zero_row(d, V, kThreads);
        return;
    }
    // The row's vectors of a wave's 1 KB are dealt to the waves in turn, kBlock neighbouring ones at a time: the
    // wave's i-th is the row's number(i)-th.  `whole` of them are whole (in raw); the row's last, partial one is
    // in its wave's rest.  The row has a whole one at least, and the registers past a wave's own take the row's
    // last one, unused: loads without a condition keep the array in registers.
    const int all = V / kAll;
    auto number = [&](int i) { return (i / kBlock * W + wave) * kBlock + i % kBlock; };
    int whole = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) whole += number(i) < all;
    const bool has_rest = V % kAll != 0 && all / kBlock % W == wave, odd = odd_row(x);
    const int j_rest = all * kAll + lane * N;
    auto place = [&](int i) { return min(number(i), all - 1) * kAll; };
    u32x4 raw[NV], rest{0u, 0u, 0u, 0u};
    int id;
    float u, total;
    read_list(a, row, id, u);
    const T* from = x - (odd ? 1 : 0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const T* at = lane_place(from + place(i), lane);
        raw[i] = CACHED ? Elem<T>::load(at) : Elem<T>::load_nt(at);
    }
    if (has_rest) rest = load_vector(x, j_rest, V, odd ? 1 : 0);
    const Listed l = take_list(a, id, u, sh, total);
    const bool out = total == 0.f;
    const float z = l.id >= 0 ? Elem<T>::get(x + l.id) : 0.f;
    if (odd) {
        uint32_t after[NV / kBlock];  // the last element of each block
#pragma unroll
        for (int i = 0; i < NV; i += kBlock) after[i / kBlock] = element_bits(x + place(i + kBlock - 1) + kAll - 1);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            uint32_t next = after[i / kBlock];
            if (i % kBlock != kBlock - 1 && i + 1 < whole)
                next = (uint32_t)__builtin_amdgcn_readlane((int)raw[i + 1 < NV ? i + 1 : i][0], 0);
            raw[i] = shift_in(raw[i], next);
        }
        if (has_rest) rest = shift_in(rest, 0xff80);  // the row ends before lane 63 does: -inf
    }

    float m = -kInf;
    auto top = [&](u32x4 q) {
        float v[N];
        Elem<T>::unpack(q, v);
        m = fmaxf(m, largest<N>(v));
    };
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i < whole) top(raw[i]);
    if (has_rest) top(rest);
    m = wave_max(m);
    if (lane == 0) part[0][wave] = m;
    __syncthreads();
    m = wave_max(lane < W ? part[0][lane] : -kInf);
    // y = (x - low) c - r, low 0 but for rows whose reference is not rounded (see Stats)
    const float ref = m == -kInf ? 0.f : m;
    const bool plain = Stats::plain(ref * a.c);
    const float low = plain ? 0.f : ref, r = plain ? ref * a.c : 0.f;
    float s = 0.f;
    auto add = [&](u32x4 q) {
        float v[N];
        Elem<T>::unpack(q, v);
#pragma unroll
        for (int k = 0; k < N; ++k) s += exp2_hw(__builtin_fmaf(v[k] - low, a.c, -r));
    };
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i < whole) add(raw[i]);
    if (has_rest) add(rest);
    s = wave_sum(s);
    if (lane == 0) part[1][wave] = s;
    __syncthreads();
    const Stats st{m, wave_sum(lane < W ? part[1][lane] : 0.f), 0.f};
    put_loss<W>(a, row, l, (z - ref) * a.inv_t - st.log_sum(a.c), part[2]);
    if (out && tid == 0) a.loss[row] = 0.f;
    if (!d) return;

    // A factor w T / S of 1 or more takes its power of two into the exponent, so that a result is 0 only where it is too
    // small itself, not its 2^y.  (A square as in the other gradients costs 3% here: 4096 x 131072, 475 us for 460.)
    const float k = w * a.t;
    const int lift = max(0, __builtin_amdgcn_frexp_expf(k / st.s));
    const float ks = __builtin_amdgcn_ldexpf(k / st.s, -lift), base = lift ? ref : low, shift = lift ? -(float)lift : r;
    const bool zero = out || st.empty();
    auto slope = [&](u32x4 q) {
        float v[N];
        Elem<T>::unpack(q, v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = exp2_hw(__builtin_fmaf(v[e] - base, a.c, -shift)) * ks;
        const u32x4 o = Elem<T>::pack(v);
        return zero ? u32x4{0u, 0u, 0u, 0u} : o;
    };
    const bool odd_out = odd_row(d), straight = straight_row(d);
    u32x4 held{0u, 0u, 0u, 0u};  // at an odd address: the vector before, whose last lane wants this one's first element
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (i < whole) {
            const u32x4 o = slope(raw[i]);
            T* at = d + place(i);
            if (!odd_out) {
                store_piece(lane_place(at, lane), o, straight);
            } else {
                if (i % kBlock == 0) {
                    if (lane == 0) store_first(at, o);
                } else {
                    Elem<T>::store(lane_place(at - kAll + 1, lane),
                                   shift_in(held, (uint32_t)__builtin_amdgcn_readlane((int)o[0], 0)));
                }
                if (i % kBlock == kBlock - 1 || i + 1 == whole) store_end(at, o, lane);
                held = o;
            }
        }
    }
    if (has_rest) store_vector(d, j_rest, V, slope(rest), odd_out, straight, lane);
    __syncthreads();
    if (l.id >= 0 && !zero) {
        Elem<T>::put(d + l.id, exp2_hw(__builtin_fmaf(z - base, a.c, -shift)) * ks - l.mass * k);
    }
}

// 2^y ks of a logit, y = x c - r(m) (see Stats).
__device__ __forceinline__ float mass_of(float v, float c, float ref, float ks) {
    const float r = ref * c, half_c = 0.5f * c;
    return squared_times(exp2_hw(Stats::plain(r) ? __builtin_fmaf(v, half_c, -0.5f * r) : (v - ref) * half_c), ks);
}

template <class T>
__device__ __forceinline__ void load_up_to(const T* x, int j, int end, float (&v)[Elem<T>::kVec]) {
    constexpr int N = Elem<T>::kVec;
    if (j + N <= end) {
        Elem<T>::unpack(Elem<T>::load(x + j), v);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = j + i < end ? Elem<T>::get(x + j + i) : -kInf;
    }
}

// d_j = 2^y_j ks for begin <= j < end, by all threads of the work-group.
template <class T>
__device__ __forceinline__ void put_masses(const T* x, T* d, int begin, int end, int threads, float c, float ref, float ks) {
    constexpr int N = Elem<T>::kVec;
    for (int j = begin + (int)threadIdx.x * N; j < end; j += threads * N) {
        float v[N];
        load_up_to<T>(x, j, end, v);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = mass_of(v[i], c, ref, ks);
        if (j + N <= end) {
            Elem<T>::store_nt(d + j, Elem<T>::pack(v));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (j + i < end) Elem<T>::put(d + j + i, v[i]);
        }
    }
}

// Rows shorter than one vector of a wave, elements past the end taken one by one;
// bound by the chain of steps (128 x 100 fp32: 5 us).
constexpr int kShortWaves = 4;
template <class T>
__global__ __launch_bounds__(64 * kShortWaves) void distill_short(DistillArgs a) {
    constexpr int N = Elem<T>::kVec, kThreads = 64 * kShortWaves;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    T* d = a.out ? static_cast<T*>(a.out) + row * a.out_stride : nullptr;
    const int V = a.vocab;
    __shared__ ListedShared sh;
    __shared__ float part[4][kShortWaves];
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (tid == 0) a.loss[row] = 0.f;
        if (d) zero_row(d, V, kThreads);
        return;
    }
    int id;
    float u, total;
    read_list(a, row, id, u);
    const Listed l = take_list(a, id, u, sh, total);
    const bool out = total == 0.f;
    const float z = l.id >= 0 ? Elem<T>::get(x + l.id) : 0.f;

    Stats st = Stats::none();
    bool masked = false;
    for (int j = tid * N; j < V; j += kThreads * N) {
        float v[N];
        load_up_to<T>(x, j, V, v);
        st.add<N>(v, largest<N>(v), a.c, masked);
    }
    st.join_wave(a.c);
    if (lane == 0) {
        part[0][wave] = st.m;
        part[1][wave] = st.s;
    }
    __syncthreads();
    st = lane < kShortWaves ? Stats{part[0][lane], part[1][lane], 0.f} : Stats::none();
    st.join_wave(a.c);
    const float ref = st.m == -kInf ? 0.f : st.m, r = ref * a.c;
    put_loss<kShortWaves>(a, row, l, (z - ref) * a.inv_t - st.log_sum(a.c), part[2]);
    if (out && tid == 0) a.loss[row] = 0.f;
    if (!d) return;
    if (out || st.empty()) {
        zero_row(d, V, kThreads);
        return;
    }
    const float k = w * a.t, ks = k / st.s;
    put_masses<T>(x, d, 0, V, kThreads, a.c, ref, ks);
    __syncthreads();
    if (l.id >= 0) Elem<T>::put(d + l.id, mass_of(z, a.c, ref, ks) - l.mass * k);
}

// Rows that are split over work-groups (see distill_plan).  A first launch takes the statistics of every part,
// and the logits of the listed tokens before a gradient in their place can
// overwrite them; a second one joins them, every work-group for itself, and
// writes the gradient of its part (the first part's the loss).  Bound by the two
// launches' chains of steps for few rows (1 x 131072 bf16: 8 us), by memory, with
// the logits read twice, for long ones (1000 x 262144 bf16: 309 us, 5.1 TB/s of
// the 1.57 GB).
constexpr int kPartWaves = 4, kPartLoads = 4;  // 16-byte loads of a thread in flight

template <class T>
__global__ __launch_bounds__(64 * kPartWaves) void distill_parts(DistillArgs a) {
    constexpr int N = Elem<T>::kVec, kThreads = 64 * kPartWaves;
    __shared__ float part[2][kPartWaves];
    const int64_t row = blockIdx.x / a.parts;
    const int which = blockIdx.x - (int)row * a.parts, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (a.weight && a.weight[row] == 0.f) return;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    const int begin = which * a.part, end = min(a.vocab, begin + a.part);
    if (which == 0 && tid < a.top) {
        const int id = a.top_ids[row * a.top + tid];
        a.listed[row * a.top + tid] = id >= 0 && id < a.vocab ? Elem<T>::get(x + id) : 0.f;
    }
    Stats st = Stats::none();
    bool masked = false;
    int j = begin + tid * N;
    for (; j - tid * N + kPartLoads * kThreads * N <= end; j += kPartLoads * kThreads * N) {
        u32x4 raw[kPartLoads];
#pragma unroll
        for (int u = 0; u < kPartLoads; ++u) raw[u] = Elem<T>::load(x + j + u * kThreads * N);
        float v[kPartLoads * N];
#pragma unroll
        for (int u = 0; u < kPartLoads; ++u) Elem<T>::unpack(raw[u], v + u * N);
        st.add<kPartLoads * N>(v, largest<kPartLoads * N>(v), a.c, masked);
    }
    for (; j < end; j += kThreads * N) {
        float v[N];
        load_up_to<T>(x, j, end, v);
        st.add<N>(v, largest<N>(v), a.c, masked);
    }
    st.join_wave(a.c);
    if (lane == 0) {
        part[0][wave] = st.m;
        part[1][wave] = st.s;
    }
    __syncthreads();
    if (wave) return;
    st = lane < kPartWaves ? Stats{part[0][lane], part[1][lane], 0.f} : Stats::none();
    st.join_wave(a.c);
    if (lane == 0) a.part_stats[row * a.parts + which] = st;
}

template <class T>
__global__ __launch_bounds__(64 * kPartWaves) void distill_parts_grad(DistillArgs a) {
    constexpr int N = Elem<T>::kVec, kThreads = 64 * kPartWaves;
    __shared__ ListedShared sh;
    __shared__ float part[kPartWaves];
    const int groups = a.out ? a.parts : 1;
    const int64_t row = blockIdx.x / groups;
    const int which = blockIdx.x - (int)row * groups, tid = threadIdx.x, lane = tid & 63;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    const int begin = which * a.part, end = min(a.vocab, begin + a.part);
    T* d = a.out ? static_cast<T*>(a.out) + row * a.out_stride : nullptr;
    const float w = a.weight ? a.weight[row] : 1.f;
    if (w == 0.f) {
        if (which == 0 && tid == 0) a.loss[row] = 0.f;
        if (d) zero_row(d + begin, end - begin, kThreads);
        return;
    }
    int id;
    float u, total;
    read_list(a, row, id, u);
    const float z = tid < a.top ? a.listed[row * a.top + tid] : 0.f;
    const Stats st = join_parts(a.part_stats + row * a.parts, a.parts, a.c, lane);
    const Listed l = take_list(a, id, u, sh, total);
    const bool out = total == 0.f;
    const float ref = st.m == -kInf ? 0.f : st.m, r = ref * a.c;
    if (which == 0) {
        put_loss<kPartWaves>(a, row, l, (z - ref) * a.inv_t - st.log_sum(a.c), part);
        if (out && tid == 0) a.loss[row] = 0.f;
    }
    if (!d) return;
    if (out || st.empty()) {
        zero_row(d + begin, end - begin, kThreads);
        return;
    }
    const float k = w * a.t, ks = k / st.s;
    put_masses<T>(x, d, begin, end, kThreads, a.c, ref, ks);
    __syncthreads();
    if (l.id >= begin && l.id < end) Elem<T>::put(d + l.id, mass_of(z, a.c, ref, ks) - l.mass * k);
}

constexpr int64_t kMaxElems = INT64_C(1) << 48;  // of a matrix, gaps included: offsets in bytes stay far inside 64 bits

bool aligned(const void* p, int32_t dtype) {
    return (reinterpret_cast<uintptr_t>(p) & (dtype == EDB_BF16 ? 1u : 3u)) == 0;
}

float log2e_over(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

// Arguments that every operator over rows of logits shares.
edb_status check_rows(const char* who, const void* logits, int32_t dtype, int32_t n, int32_t vocab, int64_t stride,
                      float temperature) {
    const std::string w(who);
    if (dtype != EDB_F32 && dtype != EDB_BF16) return fail(EDB_ERR_INVALID, w + ": dtype must be F32 or BF16");
    if (n < 0 || vocab < 1) return fail(EDB_ERR_INVALID, w + ": n >= 0 and vocab >= 1 are needed");
    if (vocab > (1 << 30)) return fail(EDB_ERR_UNSUPPORTED, w + ": vocab must not exceed 2^30");
    if (stride < vocab) return fail(EDB_ERR_INVALID, w + ": the row stride is below vocab");
    if (stride > kMaxElems / (n > 0 ? n : 1)) return fail(EDB_ERR_INVALID, w + ": the rows span more than 2^48 elements");
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(log2e_over(temperature)))
        return fail(EDB_ERR_INVALID, w + ": the temperature must be positive and finite, and log2(e) / temperature too");
    if (n && !logits) return fail(EDB_ERR_INVALID, w + ": NULL logits");
    if (!aligned(logits, dtype)) return fail(EDB_ERR_INVALID, w + ": logits must be aligned to their elements");
    return EDB_OK;
}

Region matrix(const void* p, int32_t dtype, int32_t n, int32_t vocab, int64_t stride) {
    const int64_t bytes = dtype == EDB_BF16 ? 2 : 4;
    return {p, n, vocab * bytes, stride * bytes};
}

// An array of `each` 32-bit words a row.
Region words(const void* p, int32_t n, int64_t each = 1) { return Region::array(p, n * each * 4); }

edb_status misaligned(const char* who) {
    return fail(EDB_ERR_INVALID, std::string(who) + ": ids and fp32 arrays must be aligned to 4 bytes");
}

// The gradient's rows: apart from the logits, or exactly in their place.
edb_status check_grad(const char* who, const void* logits, int64_t stride, const void* out, int64_t out_stride,
                      int32_t dtype, int32_t n, int32_t vocab) {
    const std::string w(who);
    if (out_stride < vocab) return fail(EDB_ERR_INVALID, w + ": the gradient's row stride is below vocab");
    if (out_stride > kMaxElems / (n > 0 ? n : 1))
        return fail(EDB_ERR_INVALID, w + ": the gradient's rows span more than 2^48 elements");
    if (!aligned(out, dtype)) return fail(EDB_ERR_INVALID, w + ": the gradient must be aligned to its elements");
    if (n == 0 || (out == logits && out_stride == stride)) return EDB_OK;
    if (edb::overlap(matrix(logits, dtype, n, vocab, stride), matrix(out, dtype, n, vocab, out_stride)))
        return fail(EDB_ERR_INVALID, w + ": the gradient overlaps the logits without being in their place");
    return EDB_OK;
}

edb_status launched(const char* who) {
    const hipError_t he = hipGetLastError();
    if (he != hipSuccess) return fail(EDB_ERR_HIP, std::string(who) + ": " + hipGetErrorString(he));
    edb::clear_error();
    return EDB_OK;
}

// Waves that take a row.  One up to 4 KB; and where there are enough rows to
// fill the card with single waves, up to 16 KB, and up to 32 KB unless four
// waves' last step together finds three quarters of its places filled (8000 x
// 9001 bf16: 29 us, by four 39; 8000 x 6000 fp32: 34 and 32).  Eight for long
// rows where there are too few to fill the card with four.
constexpr int kFewRows = 512, kManyRows = 2048;
int row_waves(int32_t n, int64_t bytes) {
    constexpr int64_t kStep = 4 * kLoads * 64 * 16;
    if (bytes <= 4096) return 1;
    if (n >= kManyRows && (bytes <= 16384 || (bytes <= 32768 && bytes % kStep && bytes % kStep < kStep / 4 * 3))) return 1;
    return n < kFewRows && bytes >= 32768 ? 8 : 4;
}

// How a forward call splits its rows, and its scratch memory.
struct RowPlan {
    int32_t part, parts;
    int64_t stats, keys, bytes;  // offsets
};

// Rows are split into parts, joined by a second launch, where too few of them
// would fill the card: up to 255 from 65536 logits on, up to 127 from 32768 on
// (24 x 40602 fp32, 31 alternatives: 14 us, unsplit 17; 250 x 33000: 20 and 18);
// and so is any row whose group maxima would pass 32 KB of LDS.
RowPlan row_plan(int32_t n, int32_t vocab, int32_t top) {
    constexpr int32_t kSplit = 32768, kMost = 131072, kLeast = 4096, kFill = 512;
    int64_t parts = 1;
    if (n > 0 && vocab >= kSplit && n < (vocab < 2 * kSplit ? kFill / 4 : kFill / 2)) {
        parts = kFill / n;
        if (parts > vocab / kLeast) parts = vocab / kLeast;
    }
    if (parts * kMost < vocab) parts = ((int64_t)vocab + kMost - 1) / kMost;
    RowPlan r{};
    const int64_t part = ((int64_t)vocab + parts - 1) / parts;
    r.part = (int32_t)(parts > 1 ? (part + kLeast - 1) / kLeast * kLeast : vocab);
    r.parts = (int32_t)(((int64_t)vocab + r.part - 1) / r.part);
    if (r.parts == 1) return r;
    const int64_t all = (int64_t)n * r.parts;
    r.keys = (all * (int64_t)sizeof(Stats) + 15) / 16 * 16;
    r.bytes = r.keys + all * top * (int64_t)sizeof(Key);
    return r;
}

// LDS for the group maxima of a part.
template <class T>
size_t group_bytes(const RowPlan& r, int32_t vocab) {
    const size_t places = r.parts > 1 ? (size_t)r.part : (size_t)vocab;
    return (places / (4 * Elem<T>::kVec) + 1) * 4;
}

template <class T, int W>
void launch_logprobs(const LogprobArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    if (a.top) logprobs_kernel<T, true, W><<<grid, 64 * W, lds, st>>>(a);
    else logprobs_kernel<T, false, W><<<grid, 64 * W, 0, st>>>(a);
}

template <class T>
void launch_logprobs(const LogprobArgs& a, dim3 grid, size_t lds, hipStream_t st) {
    const int waves = a.parts > 1 ? 4 : row_waves(a.n, (int64_t)a.vocab * sizeof(T));
    if (waves == 1) launch_logprobs<T, 1>(a, grid, lds, st);
    else if (waves == 4) launch_logprobs<T, 4>(a, grid, lds, st);
    else launch_logprobs<T, 8>(a, grid, lds, st);
}

constexpr int64_t kHeld = 16 * 1024;  // vectors of the longest row that a work-group holds

// Whether the caches of the memory side can hold all logits, and may do so since
// they were written.  A gradient then reads them by plain loads, else past the
// caches (distillation of 1000 x 65536 bf16: 46 and 52 us, of 1500 x 131072 179
// and 170; gradient of log probabilities of 1000 x 65536: 43 and 54 us, of 8192
// x 65536 406 and 398).
bool caches_hold(int32_t n, int32_t vocab, int32_t dtype) {
    return (int64_t)n * vocab <= (INT64_C(128) << 20) / (dtype == EDB_BF16 ? 2 : 4);
}

constexpr int32_t kGradFill = 1024;  // work-groups of the gradient of log probabilities where rows can be split

template <class T, int LOADS>
void launch_grad(const GradArgs& a, bool cached, hipStream_t st) {
    // work-groups of as many waves as a row has vectors for, and enough of them for the card
    constexpr int32_t kTurn = 64 * Elem<T>::kVec * LOADS;
    const int32_t turns = (a.vocab + kTurn - 1) / kTurn;
    const int32_t waves = turns < kGradWaves ? turns : kGradWaves, most = (turns + waves - 1) / waves;
    const int32_t wanted = a.n < kGradFill ? (kGradFill + a.n - 1) / a.n : 1;
    const dim3 grid(a.n, wanted < most ? wanted : most);
    if (cached) logprobs_grad_kernel<T, LOADS, true><<<grid, 64 * waves, 0, st>>>(a);
    else logprobs_grad_kernel<T, LOADS, false><<<grid, 64 * waves, 0, st>>>(a);
}

template <class T>
void launch_grad(const GradArgs& a, bool cached, hipStream_t st) {
    if (a.n < kGradFill / 2) launch_grad<T, 4>(a, cached, st);
    else launch_grad<T, 8>(a, cached, st);
}

// How a distillation splits its rows, and its scratch memory.
struct DistillPlan {
    bool cached;
    int32_t part, parts;  // parts == 0: rows are not split
    int64_t stats, listed, bytes;
};

// Rows are split that no work-group holds.  So are those of which a work-group
// needs more than half of a compute unit, while the second read can find the
// logits in the caches (400 x 66001 bf16: 32 us, by a work-group a row 35; 1500 x
// 131072: 231 and 172), and from three eighths on where there are few rows (1 x
// 131072: 8 and 19 us, 64 x 65536: 9 and 12; 256 rows: 20 and 16).
DistillPlan distill_plan(int32_t n, int32_t vocab, int32_t dtype, int32_t top) {
    constexpr int32_t kFill = 4096, kFew = 128;
    const int32_t bytes = dtype == EDB_BF16 ? 2 : 4, vec = 16 / bytes, least = kPartLoads * 64 * kPartWaves * vec;
    DistillPlan r{};
    r.cached = caches_hold(n, vocab, dtype);
    const int64_t held = n <= kFew ? kHeld / 8 * 3 : r.cached ? kHeld / 2 : kHeld;
    if (n == 0 || vocab <= held * vec) return r;
    int64_t parts = n < kFill ? kFill / n : 1;
    if (parts > vocab / least) parts = vocab / least;
    if (parts < 1) parts = 1;
    r.part = (int32_t)((((int64_t)vocab + parts - 1) / parts + least - 1) / least * least);
    r.parts = (int32_t)(((int64_t)vocab + r.part - 1) / r.part);
    r.listed = ((int64_t)n * r.parts * (int64_t)sizeof(Stats) + 15) / 16 * 16;
    r.bytes = r.listed + (int64_t)n * top * 4;
    return r;
}

// As few registers as hold a row, so that several work-groups share a compute
// unit (one reads while another is at its sums); more waves rather than more
// vectors a thread from 32 KB on (8192 x 65536 bf16: 383 us with 16 waves of 8,
// 403 with 8 of 16).
template <class T, bool CACHED>
void launch_held(const DistillArgs& a, hipStream_t st) {
    const int64_t vectors = ((int64_t)a.vocab + Elem<T>::kVec - 1) / Elem<T>::kVec;
    if (vectors <= 2 * 256) distill_kernel<T, 4, 2, CACHED><<<a.n, 256, 0, st>>>(a);
    else if (vectors <= 4 * 256) distill_kernel<T, 4, 4, CACHED><<<a.n, 256, 0, st>>>(a);
    else if (vectors <= 8 * 256) distill_kernel<T, 4, 8, CACHED><<<a.n, 256, 0, st>>>(a);
    else if (vectors <= 8 * 512) distill_kernel<T, 8, 8, CACHED><<<a.n, 512, 0, st>>>(a);
    else if (vectors <= 8 * 1024) distill_kernel<T, 16, 8, CACHED><<<a.n, 1024, 0, st>>>(a);
    else distill_kernel<T, 16, 16, CACHED><<<a.n, 1024, 0, st>>>(a);
}

template <class T>
void launch_distill(const DistillArgs& a, hipStream_t st) {
    if (a.parts) {
        distill_parts<T><<<a.n * a.parts, 64 * kPartWaves, 0, st>>>(a);
        distill_parts_grad<T><<<a.out ? a.n * a.parts : a.n, 64 * kPartWaves, 0, st>>>(a);
        return;
    }
    if (a.vocab < 64 * Elem<T>::kVec) distill_short<T><<<a.n, 64 * kShortWaves, 0, st>>>(a);
    else if (a.cached) launch_held<T, true>(a, st);
    else launch_held<T, false>(a, st);
}

// A launch has less than 2^32 threads: more rows than this are taken in equal slices, one after the other.
constexpr int32_t kMostRows = 1 << 21;

template <class F>
edb_status in_slices(int32_t n, F&& call) {
    const int64_t slices = ((int64_t)n + kMostRows - 1) / kMostRows, per = (n + slices - 1) / slices;
    for (int64_t i = 0; i < n; i += per)
        if (edb_status st = call(i, (int32_t)(n - i < per ? n - i : per))) return st;
    return EDB_OK;
}

template <class P>
P* rows_from(P* p, int64_t elems) {
    return p ? p + elems : nullptr;
}
const void* rows_from(const void* p, int64_t row, int64_t stride, int32_t dtype) {
    return static_cast<const char*>(p) + row * stride * (dtype == EDB_BF16 ? 2 : 4);
}

}  // namespace

extern "C" edb_status edb_logprobs_bytes(int32_t n, int32_t vocab, int32_t dtype, int32_t top, int64_t* bytes) {
    return edb::guarded([&]() -> edb_status {
        if (!bytes) return fail(EDB_ERR_INVALID, "edb_logprobs_bytes: NULL argument");
        if (edb_status st = check_rows("edb_logprobs_bytes", bytes, dtype, n, vocab, vocab, 1.f)) return st;
        if (top < 0 || top > EDB_LOGPROBS_MAX_TOP)
            return fail(EDB_ERR_UNSUPPORTED, "edb_logprobs_bytes: top must be in [0, " +
                                                 std::to_string(EDB_LOGPROBS_MAX_TOP) + "]");
        *bytes = row_plan(n, vocab, top).bytes;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_logprobs(const void* logits, int32_t dtype, int32_t n, int32_t vocab, int64_t stride,
                                   const int32_t* ids, float temperature, int32_t top, float* logprob, float* entropy,
                                   float* stats, int32_t* top_ids, float* top_logprobs, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_logprobs";
        if (edb_status st = check_rows(who, logits, dtype, n, vocab, stride, temperature)) return st;
        if (top < 0 || top > EDB_LOGPROBS_MAX_TOP)
            return fail(EDB_ERR_UNSUPPORTED, "edb_logprobs: top must be in [0, " + std::to_string(EDB_LOGPROBS_MAX_TOP) + "]");
        if (logprob && !ids) return fail(EDB_ERR_INVALID, "edb_logprobs: log probabilities need the given tokens");
        if (n && top && (!top_ids || !top_logprobs)) return fail(EDB_ERR_INVALID, "edb_logprobs: NULL list of alternatives");
        if (n == 0) {
            edb::clear_error();
            return EDB_OK;
        }
        const RowPlan r = row_plan(n, vocab, top);
        if (workspace_bytes < r.bytes || (r.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
            return fail(EDB_ERR_INVALID, "edb_logprobs: a 16-byte aligned workspace of " + std::to_string(r.bytes) +
                                             " bytes is needed");
        if (!edb::word_aligned({ids, logprob, entropy, stats, top_ids, top_logprobs})) return misaligned(who);
        if (edb_status st = edb::apart(who,
                                       {words(logprob, n), words(entropy, n), words(stats, n, 2), words(top_ids, n, top),
                                        words(top_logprobs, n, top), Region::array(workspace, r.bytes)},
                                       {matrix(logits, dtype, n, vocab, stride), words(ids, n)}))
            return st;
        if (n > kMostRows)
            return in_slices(n, [&](int64_t i, int32_t m) {
                return edb_logprobs(rows_from(logits, i, stride, dtype), dtype, m, vocab, stride, rows_from(ids, i),
                                    temperature, top, rows_from(logprob, i), rows_from(entropy, i),
                                    rows_from(stats, 2 * i), rows_from(top_ids, i * top),
                                    rows_from(top_logprobs, i * top), workspace, workspace_bytes, stream);
            });
        if ((int64_t)n * r.parts > kMostRows * INT64_C(4))
            return fail(EDB_ERR_UNSUPPORTED, "edb_logprobs: more than 2^23 parts of rows");
        char* ws = static_cast<char*>(workspace);
        const LogprobArgs a{logits,
                            stride,
                            n,
                            vocab,
                            ids,
                            log2e_over(temperature),
                            (float)(1.0 / (double)temperature),
                            top,
                            logprob,
                            entropy,
                            stats,
                            top_ids,
                            top_logprobs,
                            r.part,
                            r.parts,
                            reinterpret_cast<Stats*>(ws + r.stats),
                            reinterpret_cast<Key*>(ws + r.keys)};
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        const dim3 grid(n * r.parts);
        if (dtype == EDB_F32) {
            const size_t lds = group_bytes<float>(r, vocab);
            launch_logprobs<float>(a, grid, lds, st);
            if (r.parts > 1) logprobs_join<float><<<n, 64, 0, st>>>(a);
        } else {
            const size_t lds = group_bytes<bf16>(r, vocab);
            launch_logprobs<bf16>(a, grid, lds, st);
            if (r.parts > 1) logprobs_join<bf16><<<n, 64, 0, st>>>(a);
        }
        return launched(who);
    });
}

extern "C" edb_status edb_logprobs_grad(const void* logits, int32_t dtype, int32_t n, int32_t vocab, int64_t stride,
                                        const int32_t* ids, float temperature, const float* stats,
                                        const float* entropy, const float* g_logprob, const float* g_entropy,
                                        void* dlogits, int64_t dlogits_stride, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_logprobs_grad";
        if (edb_status st = check_rows(who, logits, dtype, n, vocab, stride, temperature)) return st;
        if (n && (!ids || !stats || !dlogits)) return fail(EDB_ERR_INVALID, "edb_logprobs_grad: NULL argument");
        if (g_entropy && !entropy) return fail(EDB_ERR_INVALID, "edb_logprobs_grad: the entropies' gradient needs the entropies");
        if (edb_status st = check_grad(who, logits, stride, dlogits, dlogits_stride, dtype, n, vocab)) return st;
        if (n == 0) {
            edb::clear_error();
            return EDB_OK;
        }
        if (!edb::word_aligned({ids, stats, entropy, g_logprob, g_entropy})) return misaligned(who);
        const Region slopes = matrix(dlogits, dtype, n, vocab, dlogits_stride);
        for (const Region& r : {words(ids, n), words(stats, n, 2), words(entropy, n), words(g_logprob, n), words(g_entropy, n)})
            if (edb::overlap(r, slopes)) return fail(EDB_ERR_INVALID, "edb_logprobs_grad: the gradient overlaps another argument");
        if (n > kMostRows)
            return in_slices(n, [&](int64_t i, int32_t m) {
                return edb_logprobs_grad(rows_from(logits, i, stride, dtype), dtype, m, vocab, stride, ids + i,
                                         temperature, stats + 2 * i, rows_from(entropy, i), rows_from(g_logprob, i),
                                         rows_from(g_entropy, i),
                                         const_cast<void*>(rows_from(dlogits, i, dlogits_stride, dtype)),
                                         dlogits_stride, stream);
            });
        GradArgs a{logits, stride,  n,         vocab,     ids,     log2e_over(temperature), (float)(1.0 / (double)temperature),
                   stats,  entropy, g_logprob, g_entropy, dlogits, dlogits_stride};
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        const bool cached = caches_hold(n, vocab, dtype);
        if (dtype == EDB_F32) launch_grad<float>(a, cached, st);
        else launch_grad<bf16>(a, cached, st);
        return launched(who);
    });
}

extern "C" edb_status edb_distill_bytes(int32_t n, int32_t vocab, int32_t dtype, int32_t top, int64_t* bytes) {
    return edb::guarded([&]() -> edb_status {
        if (!bytes) return fail(EDB_ERR_INVALID, "edb_distill_bytes: NULL argument");
        if (edb_status st = check_rows("edb_distill_bytes", bytes, dtype, n, vocab, vocab, 1.f)) return st;
        if (top < 1 || top > EDB_DISTILL_MAX_TOP)
            return fail(EDB_ERR_UNSUPPORTED, "edb_distill_bytes: top must be in [1, " +
                                                 std::to_string(EDB_DISTILL_MAX_TOP) + "]");
        *bytes = distill_plan(n, vocab, dtype, top).bytes;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_distill(const void* logits, int32_t dtype, int32_t n, int32_t vocab, int64_t stride,
                                  const int32_t* top_ids, const float* top_logits, int32_t top, float temperature,
                                  const float* weight, float* loss, void* dlogits, int64_t dlogits_stride,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_distill";
        if (edb_status st = check_rows(who, logits, dtype, n, vocab, stride, temperature)) return st;
        if (top < 1 || top > EDB_DISTILL_MAX_TOP)
            return fail(EDB_ERR_UNSUPPORTED, "edb_distill: top must be in [1, " + std::to_string(EDB_DISTILL_MAX_TOP) + "]");
        if (n && (!top_ids || !top_logits || !loss)) return fail(EDB_ERR_INVALID, "edb_distill: NULL argument");
        if (dlogits)
            if (edb_status st = check_grad(who, logits, stride, dlogits, dlogits_stride, dtype, n, vocab)) return st;
        if (n == 0) {
            edb::clear_error();
            return EDB_OK;
        }
        const DistillPlan r = distill_plan(n, vocab, dtype, top);
        if (workspace_bytes < r.bytes || (r.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
            return fail(EDB_ERR_INVALID, "edb_distill: a 16-byte aligned workspace of " + std::to_string(r.bytes) +
                                             " bytes is needed");
        if (!edb::word_aligned({top_ids, top_logits, weight, loss})) return misaligned(who);
        const Region ids = words(top_ids, n, top), listed = words(top_logits, n, top), weights = words(weight, n),
                     slopes = matrix(dlogits, dtype, n, vocab, dlogits_stride);
        if (edb_status st = edb::apart(who, {words(loss, n), Region::array(workspace, r.bytes)},
                                       {ids, listed, weights, matrix(logits, dtype, n, vocab, stride), slopes}))
            return st;
        for (const Region& in : {ids, listed, weights})
            if (edb::overlap(in, slopes)) return fail(EDB_ERR_INVALID, "edb_distill: the gradient overlaps another argument");
        if (n > kMostRows)
            return in_slices(n, [&](int64_t i, int32_t m) {
                return edb_distill(rows_from(logits, i, stride, dtype), dtype, m, vocab, stride, top_ids + i * top,
                                   top_logits + i * top, top, temperature, rows_from(weight, i), loss + i,
                                   dlogits ? const_cast<void*>(rows_from(dlogits, i, dlogits_stride, dtype)) : nullptr,
                                   dlogits_stride, workspace, workspace_bytes, stream);
            });
        if ((int64_t)n * r.parts > kMostRows * INT64_C(4))
            return fail(EDB_ERR_UNSUPPORTED, "edb_distill: more than 2^23 parts of rows");
        char* ws = static_cast<char*>(workspace);
        const DistillArgs a{logits,
                            stride,
                            n,
                            vocab,
                            top_ids,
                            top_logits,
                            top,
                            log2e_over(temperature),
                            (float)(1.0 / (double)temperature),
                            temperature,
                            weight,
                            loss,
                            dlogits,
                            dlogits_stride,
                            r.cached,
                            r.part,
                            r.parts,
                            reinterpret_cast<Stats*>(ws + r.stats),
                            reinterpret_cast<float*>(ws + r.listed)};
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        if (dtype == EDB_F32) launch_distill<float>(a, st);
        else launch_distill<bf16>(a, st);
        return launched(who);
    });
}
