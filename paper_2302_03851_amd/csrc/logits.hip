// Operators over rows of vocabulary logits: the log probability of a given
// token with the row's entropy and best alternatives, its gradient, and
// distillation from a teacher's listed logits.
//
// With x a row of V logits, T the temperature, m = max_j x_j and
// e_j = exp((x_j - m) / T):  S = sum_j e_j, l = ln S,
//   lp_j = (x_j - m) / T - l,  p_j = exp(lp_j),
//   H    = -sum_j p_j lp_j = l - (sum_j e_j (x_j - m) / T) / S.
// Both terms of H are >= 0, so nothing cancels.  Exponents are taken in base 2
// (y = (x - m) c with c = log2(e) / T, e = 2^y); the difference comes first,
// because x c can pass the largest fp32 number where x does not.  Sums are fp32.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "edb_internal.h"
#include "row_access.h"

using edb::fail;
using namespace edb::rows;

namespace {

constexpr float kLn2 = 0.69314718055994531f;
// 2^kLow is 0.  Exponents are raised to it where a product with an exponential
// of 0 would be inf * 0 (a logit of -inf, or a difference past the fp32 range).
constexpr float kLow = -1.0e4f;
constexpr float kInf = __builtin_huge_valf();
constexpr int kNoIndex = 0x7fffffff;

__device__ __forceinline__ float exp2_hw(float y) { return __builtin_amdgcn_exp2f(y); }

// Running softmax statistics relative to the maximum so far: s = sum 2^y and
// t = sum y 2^y with y = (x - m) c.  A NaN or +inf logit makes s NaN.
struct Stats {
    float m, s, t;

    static __device__ __forceinline__ Stats none() { return {-kInf, 0.f, 0.f}; }
    // the sums rescaled to the reference `ref` (the maximum, 0 while it is -inf)
    __device__ __forceinline__ void rescale(float ref, float c) {
        const float d = fmaxf((m - ref) * c, kLow), f = exp2_hw(d);
        t = (t + s * d) * f;
        s = s * f;
    }
    // N values, with `top` their largest
    template <int N>
    __device__ __forceinline__ void add(const float* x, float top, float c) {
        const float nm = fmaxf(m, top), ref = nm == -kInf ? 0.f : nm;
        rescale(ref, c);
        m = nm;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float y = (x[i] - ref) * c, e = exp2_hw(y);
            s += e;
            t = __builtin_fmaf(fmaxf(y, kLow), e, t);
        }
    }
    __device__ __forceinline__ void join(const Stats& o, float c) {
        const float nm = fmaxf(m, o.m), ref = nm == -kInf ? 0.f : nm;
        Stats b = o;
        rescale(ref, c);
        b.rescale(ref, c);
        m = nm;
        s += b.s;
        t += b.t;
    }
};

// Every lane of the wave gets the join over its 64 lanes (a butterfly: the
// same order of additions in every run).
__device__ __forceinline__ Stats wave_join(Stats a, float c) {
    for (int d = 1; d < 64; d <<= 1) {
        Stats o;
        o.m = __shfl_xor(a.m, d);
        o.s = __shfl_xor(a.s, d);
        o.t = __shfl_xor(a.t, d);
        a.join(o, c);
    }
    return a;
}

template <int N>
__device__ __forceinline__ float largest(const float* x) {
    float top = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
    return top;
}

__device__ __forceinline__ float lane_value(float v, int lane) {  // lane: the same in every lane
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// The best entries seen by a wave, lane i holding the i-th best: larger
// values first, the lowest index first among equal ones.  -inf and NaN are no
// entries.
struct Best {
    float v = -kInf;
    int j = kNoIndex;

    __device__ __forceinline__ static bool better(float v, int j, float w, int k) { return v > w || (v == w && j < k); }
    // nv, nj: the same in every lane
    __device__ __forceinline__ void insert(float nv, int nj, int lane) {
        constexpr int kUp = 0x138;  // DPP: every lane takes the value of the one before it
        const int at = __popcll(__ballot(better(v, j, nv, nj)));
        const float pv = __builtin_bit_cast(
            float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kUp, 0xf, 0xf, false));
        const int pj = __builtin_amdgcn_update_dpp(0, j, kUp, 0xf, 0xf, false);
        v = lane < at ? v : lane == at ? nv : pv;
        j = lane < at ? j : lane == at ? nj : pj;
    }
    // takes one candidate per lane; `top`: entries that count
    __device__ __forceinline__ void offer(float nv, int nj, int top, int lane) {
        for (;;) {
            const float wv = lane_value(v, top - 1);
            const int wj = lane_value(j, top - 1);
            const uint64_t who = __ballot(nv > -kInf && better(nv, nj, wv, wj));
            if (!who) return;
            const int src = __ffsll((unsigned long long)who) - 1;
            insert(lane_value(nv, src), lane_value(nj, src), lane);
            if (lane == src) nv = -kInf;
        }
    }
    // The best `top` of n candidates, get(i) giving value and index.  The lanes'
    // own largest values come first: the top-th of these is a bound that at
    // least `top` candidates reach, and only few more do, so that there are
    // about `top` insertions whatever the candidates' order.
    template <class Get>
    __device__ __forceinline__ static Best of(int n, int top, int lane, Get get) {
        float own = -kInf;
        int j;
        for (int i = lane; i < n; i += 64) {
            float w;
            get(i, w, j);
            own = fmaxf(own, w);
        }
        int above = 0;
#pragma unroll
        for (int k = 0; k < 64; ++k) above += better(lane_value(own, k), k, own, lane);
        const float bound = lane_value(own, __ffsll((unsigned long long)__ballot(above == top - 1)) - 1);
        Best b;
        for (int i = lane; i - lane < n; i += 64) {
            float w = -kInf;
            j = kNoIndex;
            if (i < n) get(i, w, j);
            b.offer(w >= bound ? w : -kInf, j, top, lane);
        }
        return b;
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
    float* part_v;        // [n][parts][top]
    int32_t* part_j;
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
__device__ __forceinline__ void put_row(const LogprobArgs& a, int64_t row, const Stats& st, const Best& best,
                                        float given, int lane) {
    const bool empty = st.m == -kInf && st.s == 0.f;
    const float l = empty ? 0.f : logf(st.s), ref = empty ? 0.f : st.m;
    if (lane < a.top) {
        const bool there = best.v > -kInf;
        a.top_ids[row * a.top + lane] = there ? best.j : -1;
        a.top_logprobs[row * a.top + lane] = there ? (best.v - ref) * a.inv_t - l : -kInf;
    }
    if (lane == 0) {
        if (a.logprob) a.logprob[row] = (given - ref) * a.inv_t - l;
        if (a.entropy) a.entropy[row] = empty ? 0.f : l - kLn2 * (st.t / st.s);
        if (a.stats) {
            const bool none = st.s != st.s;
            a.stats[2 * row] = none ? st.s : st.m;
            a.stats[2 * row + 1] = l;
        }
    }
}

// A quad is four neighbouring lanes: together they load 64 bytes of the row.
__device__ __forceinline__ float quad_max(float v) {
    constexpr int kSwap1 = 0xb1, kSwap2 = 0x4e;  // DPP quad permutations 1,0,3,2 and 2,3,0,1
    v = fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kSwap1, 0xf, 0xf, false)));
    return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kSwap2, 0xf, 0xf, false)));
}

constexpr int kLogThreads = 256, kLogWaves = kLogThreads / 64;
constexpr int kLoads = 4;  // 16-byte loads of a thread in flight

// A work-group takes a part of a row (mostly all of it) in one pass, 16 bytes a
// load.  For the alternatives each quad of lanes leaves the largest of its 64
// bytes in LDS: the best `top` logits lie in the best `top` of these groups (a
// group that does not belong to them has `top` groups with a better logit
// before it), so at the end one wave looks for those groups and reads them again.
template <class T, bool TOP>
__global__ __launch_bounds__(kLogThreads) void logprobs_kernel(LogprobArgs a) {
    constexpr int N = Elem<T>::kVec, kStep = kLogThreads * N;
    extern __shared__ float group_max[];
    __shared__ float part_m[kLogWaves], part_s[kLogWaves], part_t[kLogWaves];
    const int64_t row = blockIdx.x / a.parts;
    const int which = blockIdx.x - (int)row * a.parts;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    const int V = a.vocab, begin = which * a.part, end = min(V, begin + a.part);
    const int id = a.ids ? a.ids[row] : 0;
    if (id < 0 || id >= V) {
        if (a.parts == 1 && wave == 0) put_left_out(a, row, lane);
        return;
    }
    Stats st = Stats::none();
    for (int j0 = begin; j0 < end; j0 += kLoads * kStep) {
        const int j = j0 + tid * N;
        float v[kLoads][N];
        if (j0 + kLoads * kStep <= end) {
            u32x4 raw[kLoads];
#pragma unroll
            for (int u = 0; u < kLoads; ++u) raw[u] = Elem<T>::load_nt(x + j + u * kStep);
#pragma unroll
            for (int u = 0; u < kLoads; ++u) Elem<T>::unpack(raw[u], v[u]);
        } else {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const int k = j + u * kStep;
                if (k + N <= end) {
                    Elem<T>::unpack(Elem<T>::load(x + k), v[u]);
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) v[u][i] = k + i < end ? Elem<T>::get(x + k + i) : -kInf;
                }
            }
        }
        float top[kLoads];
#pragma unroll
        for (int u = 0; u < kLoads; ++u) top[u] = largest<N>(v[u]);
        st.add<kLoads * N>(&v[0][0], largest<kLoads>(top), a.c);
        if constexpr (TOP) {
#pragma unroll
            for (int u = 0; u < kLoads; ++u) {
                const float q = quad_max(top[u]);
                if ((lane & 3) == 0 && j + u * kStep < end) group_max[(j + u * kStep - begin) / (4 * N)] = q;
            }
        }
    }
    st = wave_join(st, a.c);
    if (lane == 0) {
        part_m[wave] = st.m;
        part_s[wave] = st.s;
        part_t[wave] = st.t;
    }
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < kLogWaves; ++w) st.join(Stats{part_m[w], part_s[w], part_t[w]}, a.c);
    Best best;
    if constexpr (TOP) {
        constexpr int kGroup = 4 * N, kAtOnce = 64 / kGroup;
        const Best groups = Best::of((end - begin + kGroup - 1) / kGroup, a.top, lane, [&](int i, float& w, int& j) {
            w = group_max[i];
            j = i;
        });
        const int there = __popcll(__ballot(lane < a.top && groups.v > -kInf));
        const float bound = lane_value(groups.v, a.top - 1);
        for (int g0 = 0; g0 < there; g0 += 4 * kAtOnce) {
            float w[4];
            int j[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int g = g0 + u * kAtOnce + lane / kGroup;
                j[u] = begin + __shfl(groups.j, g & 63) * kGroup + lane % kGroup;
                w[u] = g < there && j[u] < end ? Elem<T>::get(x + j[u]) : -kInf;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) best.offer(w[u] >= bound ? w[u] : -kInf, j[u], a.top, lane);
        }
    }
    if (a.parts == 1) {
        put_row(a, row, st, best, a.ids ? Elem<T>::get(x + id) : 0.f, lane);
    } else {
        const int64_t at = row * a.parts + which;
        if (lane == 0) a.part_stats[at] = st;
        if (lane < a.top) {
            a.part_v[at * a.top + lane] = best.v;
            a.part_j[at * a.top + lane] = best.j;
        }
    }
}

// Joins the parts of split rows: a wave a row.
template <class T>
__global__ __launch_bounds__(64) void logprobs_join(LogprobArgs a) {
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    const int id = a.ids ? a.ids[row] : 0;
    if (id < 0 || id >= a.vocab) {
        put_left_out(a, row, lane);
        return;
    }
    Stats st = Stats::none();
    for (int i = lane; i < a.parts; i += 64) st.join(a.part_stats[row * a.parts + i], a.c);
    st = wave_join(st, a.c);
    Best best;
    if (a.top) {
        const float* v = a.part_v + row * a.parts * a.top;
        const int32_t* idx = a.part_j + row * a.parts * a.top;
        best = Best::of(a.parts * a.top, a.top, lane, [&](int i, float& w, int& j) {
            w = v[i];
            j = idx[i];
        });
    }
    put_row(a, row, st, best, a.ids ? Elem<T>::get(static_cast<const T*>(a.logits) + row * a.stride + id) : 0.f, lane);
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

// dx_j = (g_lp (1[j = id] - p_j) - g_H p_j (lp_j + H)) / T.
template <class T>
__global__ __launch_bounds__(256) void logprobs_grad_kernel(GradArgs a) {
    constexpr int N = Elem<T>::kVec;
    const int64_t row = blockIdx.x;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    T* d = static_cast<T*>(a.out) + row * a.out_stride;
    const int V = a.vocab, id = a.ids[row];
    const float g1 = a.g_logprob ? a.g_logprob[row] * a.inv_t : 0.f, g2 = a.g_entropy ? a.g_entropy[row] * a.inv_t : 0.f;
    const float m = a.stats[2 * row], l2 = a.stats[2 * row + 1] * (1.f / kLn2);
    const bool zero = id < 0 || id >= V || (g1 == 0.f && g2 == 0.f) || m == -kInf;
    // p (k0 + k1 log2 p), k0 = -(g_lp + g_H H) / T, k1 = -g_H ln 2 / T
    const float k0 = -(g1 + (a.g_entropy ? g2 * a.entropy[row] : 0.f)), k1 = -g2 * kLn2;
    for (int j = threadIdx.x * N; j < V; j += 256 * N) {
        float v[N];
        const bool whole = j + N <= V;
        if (zero) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 0.f;
        } else {
            if (whole) {
                Elem<T>::unpack(Elem<T>::load(x + j), v);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = j + i < V ? Elem<T>::get(x + j + i) : -kInf;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float y = (v[i] - m) * a.c - l2;
                v[i] = exp2_hw(y) * __builtin_fmaf(k1, fmaxf(y, kLow), k0) + (j + i == id ? g1 : 0.f);
            }
        }
        if (whole) {
            Elem<T>::store(d + j, Elem<T>::pack(v));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (j + i < V) Elem<T>::put(d + j + i, v[i]);
        }
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
};

__device__ __forceinline__ float wave_max(float v) {
    for (int d = 1; d < 64; d <<= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d);
    return v;
}

// One work-group a row.  The teacher's list (one entry a thread) becomes
// masses q, equal ids as one; a first pass takes the student's statistics, a
// second writes w T p_j, and the list's owners then write w T (p_j - q_j).
template <class T>
__global__ __launch_bounds__(256) void distill_kernel(DistillArgs a) {
    constexpr int N = Elem<T>::kVec;
    static_assert(kMaxListed == 256, "one listed entry a thread");
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T* x = static_cast<const T*>(a.logits) + row * a.stride;
    T* d = a.out ? static_cast<T*>(a.out) + row * a.out_stride : nullptr;
    const int V = a.vocab;
    __shared__ int ids[256];
    __shared__ float q[256];
    __shared__ Stats part[4];
    __shared__ float red[4], red2[4];
    const float w = a.weight ? a.weight[row] : 1.f;

    int id = -1;
    float u = -kInf;
    if (tid < a.top) {
        id = a.top_ids[row * a.top + tid];
        if (id < 0 || id >= V) id = -1;
        else u = a.top_logits[row * a.top + tid];
    }
    const float um = wave_max(u);
    if (lane == 0) red[wave] = um;
    __syncthreads();
    const float tm = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float e = id < 0 ? 0.f : exp2_hw((u - (tm == -kInf ? 0.f : tm)) * a.c);
    const float es = wave_sum(e);
    if (lane == 0) red2[wave] = es;
    __syncthreads();
    const float total = (red2[0] + red2[1]) + (red2[2] + red2[3]);
    const bool out = w == 0.f || total == 0.f;
    ids[tid] = id;
    q[tid] = e / total;
    __syncthreads();
    float mass = 0.f;
    bool first = id >= 0 && !out;
    if (first)
        for (int k = 0; k < a.top; ++k)
            if (ids[k] == id) {
                if (k < tid) first = false;
                mass += q[k];
            }
    const float z = first ? Elem<T>::get(x + id) : 0.f;

    Stats st = Stats::none();
    if (!out)
        for (int j = tid * N; j < V; j += 256 * N) {
            float v[N];
            if (j + N <= V) {
                Elem<T>::unpack(Elem<T>::load(x + j), v);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = j + i < V ? Elem<T>::get(x + j + i) : -kInf;
            }
            st.add<N>(v, largest<N>(v), a.c);
        }
    st = wave_join(st, a.c);
    if (lane == 0) part[wave] = st;
    __syncthreads();
    st = part[0];
    for (int k = 1; k < 4; ++k) st.join(part[k], a.c);
    const bool empty = st.m == -kInf && st.s == 0.f;
    const float l = empty ? 0.f : logf(st.s), m = empty ? 0.f : st.m, l2 = l * (1.f / kLn2);

    float each = 0.f;
    if (first && !(mass == 0.f)) each = mass * (logf(mass) - ((z - m) * a.inv_t - l));
    each = wave_sum(each);
    __syncthreads();
    if (lane == 0) red[wave] = each;
    __syncthreads();
    if (tid == 0) a.loss[row] = out ? 0.f : a.t * a.t * ((red[0] + red[1]) + (red[2] + red[3]));
    if (!d) return;

    const float k = w * a.t;
    const bool zero = out || empty;
    for (int j = tid * N; j < V; j += 256 * N) {
        float v[N];
        const bool whole = j + N <= V;
        if (zero) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = 0.f;
        } else {
            if (whole) {
                Elem<T>::unpack(Elem<T>::load(x + j), v);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) v[i] = j + i < V ? Elem<T>::get(x + j + i) : -kInf;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = exp2_hw((v[i] - m) * a.c - l2) * k;
        }
        if (whole) {
            Elem<T>::store(d + j, Elem<T>::pack(v));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (j + i < V) Elem<T>::put(d + j + i, v[i]);
        }
    }
    __syncthreads();
    if (first && !zero) Elem<T>::put(d + id, (exp2_hw((z - m) * a.c - l2) - mass) * k);
}

constexpr int64_t kMaxElems = INT64_C(1) << 48;  // of a matrix, gaps included: offsets in bytes stay far inside 64 bits

bool aligned(const void* p, int32_t dtype) {
    return (reinterpret_cast<uintptr_t>(p) & (dtype == EDB_BF16 ? 1u : 3u)) == 0;
}

// Arguments that every operator over rows of logits shares.
edb_status check_rows(const char* who, const void* logits, int32_t dtype, int32_t n, int32_t vocab, int64_t stride,
                      float temperature) {
    const std::string w(who);
    if (dtype != EDB_F32 && dtype != EDB_BF16) return fail(EDB_ERR_INVALID, w + ": dtype must be F32 or BF16");
    if (n < 0 || vocab < 1) return fail(EDB_ERR_INVALID, w + ": n >= 0 and vocab >= 1 are needed");
    if (vocab > (1 << 30)) return fail(EDB_ERR_UNSUPPORTED, w + ": vocab must not exceed 2^30");
    if (stride < vocab) return fail(EDB_ERR_INVALID, w + ": the row stride is below vocab");
    if (stride > kMaxElems / (n > 0 ? n : 1)) return fail(EDB_ERR_INVALID, w + ": the rows span more than 2^48 elements");
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.0f / temperature))
        return fail(EDB_ERR_INVALID, w + ": the temperature must be positive and finite");
    if (n && !logits) return fail(EDB_ERR_INVALID, w + ": NULL logits");
    if (!aligned(logits, dtype)) return fail(EDB_ERR_INVALID, w + ": logits must be aligned to their elements");
    return EDB_OK;
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
    const int64_t es = dtype == EDB_BF16 ? 2 : 4;
    const uintptr_t x0 = reinterpret_cast<uintptr_t>(logits), d0 = reinterpret_cast<uintptr_t>(out);
    const uintptr_t x1 = x0 + (uintptr_t)(((n - 1) * stride + vocab) * es),
                    d1 = d0 + (uintptr_t)(((n - 1) * out_stride + vocab) * es);
    if (x0 < d1 && d0 < x1)
        return fail(EDB_ERR_INVALID, w + ": the gradient overlaps the logits without being in their place");
    return EDB_OK;
}

edb_status launched(const char* who) {
    const hipError_t he = hipGetLastError();
    if (he != hipSuccess) return fail(EDB_ERR_HIP, std::string(who) + ": " + hipGetErrorString(he));
    edb::clear_error();
    return EDB_OK;
}

// How a forward call splits its rows, and its scratch memory.
struct RowPlan {
    int32_t part, parts;
    int64_t stats, v, j, bytes;  // offsets
};

// A row is split where there are too few rows for the card, and where a part's
// group maxima would pass 32 KB of LDS.  Parts are whole steps of a work-group.
RowPlan row_plan(int32_t n, int32_t vocab, int32_t dtype, int32_t top) {
    constexpr int32_t kMost = 131072;
    const int32_t step = kLoads * kLogThreads * (dtype == EDB_BF16 ? Elem<bf16>::kVec : Elem<float>::kVec);
    const int64_t steps = ((int64_t)vocab + step - 1) / step;
    int64_t parts = n >= 512 ? 1 : (512 + n - 1) / (n < 1 ? 1 : n);
    if (parts > steps) parts = steps;
    if (parts * kMost < vocab) parts = ((int64_t)vocab + kMost - 1) / kMost;
    RowPlan r{};
    r.part = (int32_t)((steps + parts - 1) / parts * step);
    r.parts = (int32_t)(((int64_t)vocab + r.part - 1) / r.part);
    if (r.parts == 1) return r;
    const int64_t all = (int64_t)n * r.parts;
    auto aligned16 = [](int64_t b) { return (b + 15) / 16 * 16; };
    r.v = aligned16(all * (int64_t)sizeof(Stats));
    r.j = r.v + aligned16(all * top * 4);
    r.bytes = r.j + all * top * 4;
    return r;
}

float log2e_over(float temperature) { return (float)(1.4426950408889634 / (double)temperature); }

}  // namespace

extern "C" edb_status edb_logprobs_bytes(int32_t n, int32_t vocab, int32_t dtype, int32_t top, int64_t* bytes) {
    if (!bytes) return fail(EDB_ERR_INVALID, "edb_logprobs_bytes: NULL argument");
    if (edb_status st = check_rows("edb_logprobs_bytes", bytes, dtype, n, vocab, vocab, 1.f)) return st;
    if (top < 0 || top > EDB_LOGPROBS_MAX_TOP)
        return fail(EDB_ERR_UNSUPPORTED, "edb_logprobs_bytes: top must be in [0, " +
                                             std::to_string(EDB_LOGPROBS_MAX_TOP) + "]");
    *bytes = row_plan(n, vocab, dtype, top).bytes;
    edb::clear_error();
    return EDB_OK;
}

extern "C" edb_status edb_logprobs(const void* logits, int32_t dtype, int32_t n, int32_t vocab, int64_t stride,
                                   const int32_t* ids, float temperature, int32_t top, float* logprob, float* entropy,
                                   float* stats, int32_t* top_ids, float* top_logprobs, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
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
    const RowPlan r = row_plan(n, vocab, dtype, top);
    if (workspace_bytes < r.bytes || (r.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
        return fail(EDB_ERR_INVALID, "edb_logprobs: a 16-byte aligned workspace of " + std::to_string(r.bytes) +
                                         " bytes is needed");
    if ((int64_t)n * r.parts > INT32_MAX) return fail(EDB_ERR_UNSUPPORTED, "edb_logprobs: more than 2^31 parts of rows");
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
                        reinterpret_cast<float*>(ws + r.v),
                        reinterpret_cast<int32_t*>(ws + r.j)};
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const dim3 grid(n * r.parts);
    if (dtype == EDB_F32) {
        const size_t lds = ((size_t)(r.part < vocab ? r.part : vocab) / (4 * Elem<float>::kVec) + 1) * 4;
        if (top) logprobs_kernel<float, true><<<grid, kLogThreads, lds, st>>>(a);
        else logprobs_kernel<float, false><<<grid, kLogThreads, 0, st>>>(a);
        if (r.parts > 1) logprobs_join<float><<<n, 64, 0, st>>>(a);
    } else {
        const size_t lds = ((size_t)(r.part < vocab ? r.part : vocab) / (4 * Elem<bf16>::kVec) + 1) * 4;
        if (top) logprobs_kernel<bf16, true><<<grid, kLogThreads, lds, st>>>(a);
        else logprobs_kernel<bf16, false><<<grid, kLogThreads, 0, st>>>(a);
        if (r.parts > 1) logprobs_join<bf16><<<n, 64, 0, st>>>(a);
    }
    return launched(who);
}

extern "C" edb_status edb_logprobs_grad(const void* logits, int32_t dtype, int32_t n, int32_t vocab, int64_t stride,
                                        const int32_t* ids, float temperature, const float* stats,
                                        const float* entropy, const float* g_logprob, const float* g_entropy,
                                        void* dlogits, int64_t dlogits_stride, void* stream) {
    const char* who = "edb_logprobs_grad";
    if (edb_status st = check_rows(who, logits, dtype, n, vocab, stride, temperature)) return st;
    if (n && (!ids || !stats || !dlogits)) return fail(EDB_ERR_INVALID, "edb_logprobs_grad: NULL argument");
    if (g_entropy && !entropy) return fail(EDB_ERR_INVALID, "edb_logprobs_grad: the entropies' gradient needs the entropies");
    if (edb_status st = check_grad(who, logits, stride, dlogits, dlogits_stride, dtype, n, vocab)) return st;
    if (n == 0) {
        edb::clear_error();
        return EDB_OK;
    }
    GradArgs a{logits, stride,  n,         vocab,     ids,     log2e_over(temperature), (float)(1.0 / (double)temperature),
               stats,  entropy, g_logprob, g_entropy, dlogits, dlogits_stride};
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const dim3 grid(n), block(256);
    if (dtype == EDB_F32) logprobs_grad_kernel<float><<<grid, block, 0, st>>>(a);
    else logprobs_grad_kernel<bf16><<<grid, block, 0, st>>>(a);
    return launched(who);
}

extern "C" edb_status edb_distill(const void* logits, int32_t dtype, int32_t n, int32_t vocab, int64_t stride,
                                  const int32_t* top_ids, const float* top_logits, int32_t top, float temperature,
                                  const float* weight, float* loss, void* dlogits, int64_t dlogits_stride,
                                  void* stream) {
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
    DistillArgs a{logits, stride,      n,      vocab, top_ids, top_logits, top, log2e_over(temperature),
                  (float)(1.0 / (double)temperature), temperature, weight, loss, dlogits, dlogits_stride};
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const dim3 grid(n), block(256);
    if (dtype == EDB_F32) distill_kernel<float><<<grid, block, 0, st>>>(a);
    else distill_kernel<bf16><<<grid, block, 0, st>>>(a);
    return launched(who);
}
