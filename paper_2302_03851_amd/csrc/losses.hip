// Losses over the log probabilities of sequences' tokens, with the gradients
// of the log probabilities.
//
// A sequence s is the tokens first[s] .. first[s + 1] - 1; T_s of them count
// (those with an id, where ids are given), and c_s is 1, or 1 / T_s where the
// loss goes by means.
//
// Preference of the sequence 2p over 2p + 1, with
//   R_s = c_s sum_t (lp_t - ref_t),  D = R_2p - R_2p+1,  f one of
//   (1 - e) ln(1 + exp(-b D)) + e ln(1 + exp(b D)),  max(0, 1 - b D),  (D - 1 / (2 b))^2:
//   loss_p = f(D),  g_t = +-weight_p f'(D) c_s
//
// Policy, with r_t = exp(lp_t - old_t), q_t = ref_t - lp_t:
//   loss_s = c_s sum_t -min(r A, clip(r, 1 - low, 1 + high) A) + k (exp q - 1 - q)
//   g_t    = weight_s c_s (-A r [not clipped] - k (exp q - 1))
//
// All of it is computed in 64 bits and rounded once: log ratios of long
// sequences are differences of large sums, exp q - 1 - q is what is left of
// terms up to 10^7 times as large, and a ratio next to the clip's border has to
// fall on its side of it.
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "edb_internal.h"
#include "lane_sums.h"

using edb::fail;
using edb::Region;

namespace {

struct alignas(8) Sums {
    double a, b;              // preference: log ratios; policy: surrogate, divergence
    int32_t live, clipped;
};

__device__ __forceinline__ Sums operator+(const Sums& x, const Sums& y) {
    return {x.a + y.a, x.b + y.b, x.live + y.live, x.clipped + y.clipped};
}

template <int LANES>
__device__ __forceinline__ Sums lanes_sum(const Sums& s) {
    using edb::lanes::sum;
    return {sum<LANES>(s.a), sum<LANES>(s.b), sum<LANES>(s.live), sum<LANES>(s.clipped)};
}

struct Loss {
    const float *logprob, *other;   // other: the reference (or NULL), the old log probabilities
    const float* reference;         // policy: or NULL
    const int32_t* ids;             // or NULL
    int32_t n;
    const int32_t* first;
    int32_t items;                  // pairs, sequences
    const float* advantage;         // policy
    int32_t per_token, mean, kind;
    double beta, smoothing;         // preference
    double low, high, coef;         // policy: the clip's borders (ratios), the divergence's factor
    double log_low, log_high;       // the borders' logarithms
    const float* weight;            // or NULL
    float *loss, *second;           // second: rewards, divergences
    int32_t* clipped;
    float* grad;
    // long calls only
    int32_t* places;                // [chunk]
    Sums *parts, *whole;            // [chunk][2], [sequence]
    bool counted;                   // policy, means over the tokens with an id: whole's live come before all else
    double* slopes;                 // preference: [sequence]
};

struct Range {
    int32_t from, to;
};
// Tokens of a sequence; offsets that fall or leave [0, n] give no tokens outside of it.
__device__ __forceinline__ Range range_of(const Loss& l, int s) {
    const int from = min(max(l.first[s], 0), l.n);
    return {from, min(max(l.first[s + 1], from), l.n)};
}
__device__ __forceinline__ bool is_live(const Loss& l, int64_t t) { return !l.ids || l.ids[t] >= 0; }

__device__ __forceinline__ double log_ratio(const Loss& l, int64_t t) {
    return (double)l.logprob[t] - (l.other ? (double)l.other[t] : 0.0);
}

// f(D) and f'(D)
__device__ __forceinline__ void preference(const Loss& l, double diff, double& loss, double& slope) {
    const double y = l.beta * diff;
    if (l.kind == EDB_PREFERENCE_LOGISTIC) {
        // a term of factor 0 is left out: the other's limit stands where it is infinite
        const double small = exp(-fabs(y)), near = log1p(small), won = (y < 0.0 ? -y : 0.0) + near, lost = (y > 0.0 ? y : 0.0) + near;
        const double few = small / (1.0 + small), most = 1.0 / (1.0 + small);
        const double p = y > 0.0 ? few : most, q = y > 0.0 ? most : few;   // of the other being preferred, and of this one
        const double e = l.smoothing;
        loss = e == 0.0 ? won : e == 1.0 ? lost : (1.0 - e) * won + e * lost;
        slope = l.beta * (e == 0.0 ? -p : e * q - (1.0 - e) * p);
    } else if (l.kind == EDB_PREFERENCE_HINGE) {
        loss = y < 1.0 ? 1.0 - y : y != y ? y : 0.0;
        slope = y < 1.0 ? -l.beta : y != y ? y : 0.0;
    } else {
        const double off = diff - 0.5 / l.beta;
        loss = off * off;
        slope = 2.0 * off;
    }
}

// exp x = 2^k (1 + r + r^2 H(r)) with r in [-ln 2 / 2, ln 2 / 2] and the series
// of H(r) = (exp r - 1 - r) / r^2 up to r^9 (what is left out is below 10^-13 of
// it): a third of the library's instructions, and exp x - 1 - x without
// cancellation next to 0.  The library's exp and expm1 took 40 of the 53 us of
// policy_terms over 4 M tokens.
struct Exp {
    int k;
    double r, h;
    __device__ __forceinline__ explicit Exp(double x) {
        const double c = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;   // NaN stays
        const double n = rint(c * 1.4426950408889634);
        k = (int)n;
        r = fma(n, -0.6931471805599453, c);
        h = 1.0 / 39916800.0;
        h = fma(h, r, 1.0 / 3628800.0);
        h = fma(h, r, 1.0 / 362880.0);
        h = fma(h, r, 1.0 / 40320.0);
        h = fma(h, r, 1.0 / 5040.0);
        h = fma(h, r, 1.0 / 720.0);
        h = fma(h, r, 1.0 / 120.0);
        h = fma(h, r, 1.0 / 24.0);
        h = fma(h, r, 1.0 / 6.0);
        h = fma(h, r, 0.5);
    }
    __device__ __forceinline__ double more() const { return fma(r * r, h, r); }      // exp r - 1
    __device__ __forceinline__ double value() const { return ldexp(1.0 + more(), k); }
    __device__ __forceinline__ double less_one() const { return k ? value() - 1.0 : more(); }
    __device__ __forceinline__ double less_line(double x) const { return k ? value() - 1.0 - x : r * r * h; }
};

struct Token {
    double gain, kl, slope;
    bool clipped;
};
__device__ __forceinline__ Token policy(const Loss& l, float logprob, float old, float reference, double a) {
    const double lp = logprob, d = lp - (double)old, r = Exp(d).value();
    const bool beyond = a > 0.0 ? d > l.log_high : a < 0.0 && d < l.log_low;
    const double moved = a == 0.0 && r == r ? 0.0 : a * r;
    Token t{beyond ? a * (a > 0.0 ? l.high : l.low) : moved, 0.0, beyond ? 0.0 : -moved, beyond};
    if (l.reference) {
        const double q = (double)reference - lp;
        const Exp e(q);
        t.kl = q == HUGE_VAL ? q : e.less_line(q);
        if (l.coef != 0.0) t.slope -= l.coef * e.less_one();
    }
    return t;
}
__device__ __forceinline__ double policy_loss(const Loss& l, double gain, double kl) {
    return l.coef != 0.0 ? l.coef * kl - gain : -gain;
}

// ---- few tokens: one launch, a group of threads for every pair or sequence ----

template <int THREADS>
__device__ __forceinline__ Sums group_sum(Sums s, Sums* held) {
    s = lanes_sum<64>(s);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) held[threadIdx.x >> 6] = s;
        __syncthreads();
        s = held[0];
        for (int w = 1; w < THREADS / 64; ++w) s = s + held[w];
    }
    return s;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS > 256 ? THREADS : 256) void preference_kernel(Loss l) {
    constexpr int kBlock = THREADS > 256 ? THREADS : 256;
    __shared__ Sums held[kBlock / 64];
    const int tid = threadIdx.x % THREADS, item = blockIdx.x * (kBlock / THREADS) + threadIdx.x / THREADS;
    if (item >= l.items) return;
    const double weight = l.weight ? (double)l.weight[item] : 1.0;
    Range range[2];
    double mean[2], ratio[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        range[i] = range_of(l, 2 * item + i);
        Sums s{0.0, 0.0, 0, 0};
        if (weight != 0.0)
            for (int64_t t = range[i].from + tid; t < range[i].to; t += THREADS)
                if (is_live(l, t)) {
                    s.a += log_ratio(l, t);
                    ++s.live;
                }
        s = group_sum<THREADS>(s, held);
        mean[i] = l.mean && s.live ? 1.0 / s.live : 1.0;
        ratio[i] = s.a * mean[i];
    }
    double loss = 0.0, slope = 0.0;
    if (weight != 0.0) preference(l, ratio[0] - ratio[1], loss, slope);
    if (tid == 0) {
        l.loss[item] = (float)loss;
        l.second[2 * item] = (float)(l.beta * ratio[0]);
        l.second[2 * item + 1] = (float)(l.beta * ratio[1]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float g = weight != 0.0 ? (float)((i ? -slope : slope) * weight * mean[i]) : 0.f;
        for (int64_t t = range[i].from + tid; t < range[i].to; t += THREADS) l.grad[t] = is_live(l, t) ? g : 0.f;
    }
    // tokens before the first sequence and behind the last
    if (item == 0)
        for (int64_t t = tid; t < range[0].from; t += THREADS) l.grad[t] = 0.f;
    if (item == l.items - 1)
        for (int64_t t = range[1].to + tid; t < l.n; t += THREADS) l.grad[t] = 0.f;
}

template <int THREADS>
__global__ __launch_bounds__(THREADS > 256 ? THREADS : 256) void policy_kernel(Loss l) {
    constexpr int kBlock = THREADS > 256 ? THREADS : 256;
    __shared__ Sums held[kBlock / 64];
    const int tid = threadIdx.x % THREADS, item = blockIdx.x * (kBlock / THREADS) + threadIdx.x / THREADS;
    if (item >= l.items) return;
    const Range range = range_of(l, item);
    const double weight = l.weight ? (double)l.weight[item] : 1.0;
    Sums s{0.0, 0.0, 0, 0};
    double mean = 1.0;
    if (weight == 0.0) {
        for (int64_t t = range.from + tid; t < range.to; t += THREADS) l.grad[t] = 0.f;
    } else {
        if (l.mean) {
            int live = range.to - range.from;
            if (l.ids) {
                for (int64_t t = range.from + tid; t < range.to; t += THREADS) s.live += l.ids[t] >= 0;
                live = group_sum<THREADS>(s, held).live;
                s.live = 0;
            }
            if (live) mean = 1.0 / live;
        }
        for (int64_t t = range.from + tid; t < range.to; t += THREADS) {
            float g = 0.f;
            if (is_live(l, t)) {
                const Token k = policy(l, l.logprob[t], l.other[t], l.reference ? l.reference[t] : 0.f,
                                       l.advantage[l.per_token ? t : item]);
                s.a += k.gain;
                s.b += k.kl;
                s.clipped += k.clipped;
                g = (float)(k.slope * weight * mean);
            }
            l.grad[t] = g;
        }
        s = group_sum<THREADS>(s, held);
    }
    if (tid == 0) {
        l.loss[item] = (float)(policy_loss(l, s.a, s.b) * mean);
        l.second[item] = (float)(s.b * mean);
        l.clipped[item] = s.clipped;
    }
    if (item == 0)
        for (int64_t t = tid; t < range.from; t += THREADS) l.grad[t] = 0.f;
    if (item == l.items - 1)
        for (int64_t t = range.to + tid; t < l.n; t += THREADS) l.grad[t] = 0.f;
}

// ---- many tokens: chunks of them, whatever sequences they belong to ----
//
// A chunk adds up each of its sequences' tokens.  What lies inside the chunk is
// whole; the sequence that comes in from the chunk before leaves its share in
// parts[chunk][0], the one that begins here and goes on in parts[chunk][1].

constexpr int kChunk = 1024, kThreads = 256, kEach = kChunk / kThreads;

struct Chunk {
    int32_t from, to;       // tokens
    int32_t s0, s1;         // sequences that may have tokens here: s0 <= s < s1
};

// First of the launches: for every chunk, how many sequences begin up to its
// first token.  The sequence that holds the token writes it (the one after the
// last: for chunks before the first sequence).  A search by each work-group of
// the other launches took 16 of policy_terms' 48 us over 4 M tokens.  A long
// sequence's chunks are the whole wave's: one thread's stores, one after the
// other, took 1.0 ms for the 65536 chunks of 2^26 tokens.
__global__ __launch_bounds__(kThreads) void place_chunks(Loss l, int sequences) {
    const int s = blockIdx.x * kThreads + threadIdx.x;
    constexpr int kOwn = 4;
    if (l.counted && s < sequences) l.whole[s].live = 0;
    int c0 = 0, c1 = 0;
    if (s <= sequences) {
        const int64_t from = s < sequences ? min(max(l.first[s], 0), l.n) : 0;
        const int64_t to = s == sequences ? min(max(l.first[0], 0), l.n) : s + 1 < sequences ? min(max(l.first[s + 1], 0), l.n) : l.n;
        c0 = (int)((from + kChunk - 1) / kChunk);
        c1 = (int)((to + kChunk - 1) / kChunk);
    }
    const int begun = s < sequences ? s + 1 : 0;
    if (c1 - c0 <= kOwn)
        for (int c = c0; c < c1; ++c) l.places[c] = begun;
    for (uint64_t left = __ballot(c1 - c0 > kOwn); left; left &= left - 1) {
        const int lane = __ffsll((unsigned long long)left) - 1, of = __shfl(begun, lane), end = __shfl(c1, lane);
        for (int c = __shfl(c0, lane) + (int)(threadIdx.x & 63); c < end; c += 64) l.places[c] = of;
    }
}

__device__ __forceinline__ Chunk chunk_of(const Loss& l, int sequences, int chunk) {
    Chunk c;
    c.from = chunk * kChunk;
    c.to = (int)min((int64_t)c.from + kChunk, (int64_t)l.n);
    // (offsets that fall may leave places unwritten: any number then)
    c.s0 = min(max(l.places[chunk] - 1, 0), sequences);
    c.s1 = c.to < l.n ? min(max(l.places[chunk + 1], 0), sequences) : sequences;
    return c;
}

// The chunk's sequences that have tokens there, in order.  `from` and `to` count
// from the chunk's first token; kOn marks one that came in or goes on.
constexpr uint32_t kOn = 0x8000, kPlace = 0x7fff;
struct List {
    int32_t seq[kChunk];
    uint16_t from[kChunk], to[kChunk];
    int32_t waves[2][kThreads / 64];
};

// Where more sequences than kWalk may lie here, most of them are empty: then every
// token looks for its own by halving, and those that are their sequence's first
// here name it (2^20 empty ones one after the other took the chunk 1.0 ms).
constexpr int kWalk = 2 * kChunk;
__device__ __forceinline__ int list_sequences(const Loss& l, const Chunk& c, List& list) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const bool search = c.s1 - c.s0 > kWalk;
    int of[kEach];
    if (search) {
        int high[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            of[i] = c.s0;
            high[i] = c.s1;
        }
        // the last that begins up to the token, all steps for all tokens (a span of 1 stays)
        for (int span = c.s1 - c.s0; span > 1; span -= span / 2) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int middle = of[i] + (high[i] - of[i]) / 2;
                if (l.first[middle] <= c.from + (int)threadIdx.x + i * kThreads) of[i] = middle;
                else high[i] = middle;
            }
        }
    }
    int count = 0, turn = 0;
    auto add = [&](int s, const Range& r, bool mine) {
        const int from = max(r.from, c.from), to = min(r.to, c.to);
        const bool listed = mine && from < to;
        const uint64_t there = __ballot(listed);
        if (lane == 0) list.waves[turn][wave] = __popcll(there);
        __syncthreads();
        int at = count + __popcll(there & ((1ull << lane) - 1));
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w) {
            const int n = list.waves[turn][w];
            if (w < wave) at += n;
            count += n;
        }
        if (listed && at < kChunk) {   // offsets that fall could name more
            list.seq[at] = s;
            list.from[at] = (uint16_t)((from - c.from) | (r.from < c.from ? kOn : 0));
            list.to[at] = (uint16_t)((to - c.from) | (r.to > c.to ? kOn : 0));
        }
        turn ^= 1;
    };
    if (search) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int64_t t = (int64_t)c.from + threadIdx.x + i * kThreads;
            const Range r = range_of(l, of[i]);
            add(of[i], r, t < c.to && t == max(r.from, c.from));
        }
    } else {
        for (int base = c.s0; base < c.s1; base += kThreads) {
            const int s = base + (int)threadIdx.x;
            Range r{0, 0};
            if (s < c.s1) r = range_of(l, s);
            add(s, r, true);
        }
    }
    __syncthreads();
    return min(count, kChunk);
}

// Calls body(i, lane) with a group of lanes for every sequence of the list, more
// lanes where there are fewer (and longer) ones.
constexpr int kLong = 8;
template <class F>
__device__ __forceinline__ void by_sequence(int count, F&& body) {
    auto go = [&](auto lanes) {
        constexpr int kLanes = decltype(lanes)::value;
        for (int i = (int)threadIdx.x / kLanes; i < count; i += kThreads / kLanes) body(i, (int)threadIdx.x % kLanes, lanes);
    };
    if (count <= kLong) go(std::integral_constant<int, 64>());
    else if (count <= 128) go(std::integral_constant<int, 16>());
    else go(std::integral_constant<int, 2>());
}

// The places in the list of the sequences of a thread's tokens (kOn: none).
__device__ __forceinline__ void find_sequences(const List& list, int count, uint16_t* scratch, uint32_t (&of)[kEach]) {
    if (count <= kLong) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) of[i] = kOn;
        for (int s = 0; s < count; ++s) {
            const int from = list.from[s] & kPlace, to = list.to[s] & kPlace;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int t = (int)threadIdx.x + i * kThreads;
                if (t >= from && t < to) of[i] = s;
            }
        }
        return;
    }
    for (int i = threadIdx.x; i < kChunk; i += kThreads) scratch[i] = kOn;
    __syncthreads();
    by_sequence(count, [&](int i, int lane, auto lanes) {
        const int to = list.to[i] & kPlace;
        for (int t = (list.from[i] & kPlace) + lane; t < to; t += decltype(lanes)::value) scratch[t] = (uint16_t)i;
    });
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i) of[i] = scratch[threadIdx.x + i * kThreads];
}

// Adds up the sequences' tokens and hands every sum on.  A thread has the tokens
// threadIdx.x + i kThreads, of the sequences of[] in the list, with terms term[].
// Few sequences (long ones) are added up from the registers, a sequence after the
// other by all waves; many one field after the other through LDS, so that it
// leaves room for more work-groups.  SUMS: doubles that are wanted, 0 to 2.
template <int SUMS>
__device__ __forceinline__ void sum_sequences(const Loss& l, const List& list, int count, Sums (&held)[kThreads / 64][kLong],
                                              double* scratch, const uint32_t (&of)[kEach], const Sums (&term)[kEach]) {
    // the counts alone are whole numbers, and added up right there, in whatever order
    auto count_to = [&](int i, int32_t live) {
        int32_t& to = l.whole[list.seq[i]].live;
        if ((list.from[i] | list.to[i]) & kOn) atomicAdd(&to, live);
        else to = live;
    };
    auto place = [&](int i) -> Sums& {
        if (list.from[i] & kOn) return l.parts[2 * blockIdx.x];
        if (list.to[i] & kOn) return l.parts[2 * blockIdx.x + 1];
        return l.whole[list.seq[i]];
    };
    if (count <= kLong) {
        for (int s = 0; s < count; ++s) {
            Sums sum{0.0, 0.0, 0, 0};
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                if (of[i] == (uint32_t)s) sum = sum + term[i];
            const uint32_t counts = edb::lanes::sum<64>((uint32_t)sum.live | (uint32_t)sum.clipped << 16);
            if (SUMS > 0) sum.a = edb::lanes::sum<64>(sum.a);
            if (SUMS > 1) sum.b = edb::lanes::sum<64>(sum.b);
            sum.live = (int)(counts & 0xffff);
            sum.clipped = (int)(counts >> 16);
            if ((threadIdx.x & 63) == 0) held[threadIdx.x >> 6][s] = sum;
        }
        __syncthreads();
        if ((int)threadIdx.x < count) {
            Sums sum = held[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < kThreads / 64; ++w) sum = sum + held[w][threadIdx.x];
            if (SUMS) place(threadIdx.x) = sum;
            else count_to(threadIdx.x, sum.live);
        }
        return;
    }
    auto field = [&](auto get, auto put) {
        typedef decltype(get(term[0])) V;
        V* values = reinterpret_cast<V*>(scratch);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i) values[i * kThreads + threadIdx.x] = get(term[i]);
        __syncthreads();
        by_sequence(count, [&](int i, int lane, auto lanes) {
            constexpr int kLanes = decltype(lanes)::value;
            const int to = list.to[i] & kPlace;
            V sum = 0;
            for (int t = (list.from[i] & kPlace) + lane; t < to; t += kLanes) sum += values[t];
            sum = edb::lanes::sum<kLanes>(sum);
            if (lane == 0) put(i, sum);
        });
    };
    if (SUMS > 0) field([](const Sums& s) { return s.a; }, [&](int i, double v) { place(i).a = v; });
    if (SUMS > 1) field([](const Sums& s) { return s.b; }, [&](int i, double v) { place(i).b = v; });
    field([](const Sums& s) { return (uint32_t)s.live | (uint32_t)s.clipped << 16; },
          [&](int i, uint32_t v) {
              if (SUMS) {
                  Sums& to = place(i);
                  to.live = (int)(v & 0xffff);
                  to.clipped = (int)(v >> 16);
              } else {
                  count_to(i, (int)v);
              }
          });
}

// A sequence's sums over its chunks, by a wave.
__device__ __forceinline__ Sums sequence_sum(const Loss& l, int s) {
    const Range r = range_of(l, s);
    Sums sum{0.0, 0.0, 0, 0};
    if (r.from >= r.to) return sum;
    const int c0 = r.from / kChunk, c1 = (r.to - 1) / kChunk;
    if (c0 == c1) return l.whole[s];
    // the first chunk's share began there, the others' came in; eight asked for at once
    constexpr int kOnce = 8;
    int c = c0 + (int)(threadIdx.x & 63);
    for (; c + (kOnce - 1) * 64 <= c1; c += kOnce * 64) {
        Sums part[kOnce];
#pragma unroll
        for (int i = 0; i < kOnce; ++i) part[i] = l.parts[2 * (c + i * 64) + (c + i * 64 == c0 ? 1 : 0)];
#pragma unroll
        for (int i = 0; i < kOnce; ++i) sum = sum + part[i];
    }
    for (; c <= c1; c += 64) sum = sum + l.parts[2 * c + (c == c0 ? 1 : 0)];
    return lanes_sum<64>(sum);
}

template <class T>
__device__ __forceinline__ void load_tokens(const T* p, int64_t at, int64_t end, T none, T (&v)[kEach]) {
#pragma unroll
    for (int i = 0; i < kEach; ++i) v[i] = p && at + i * kThreads < end ? p[at + i * kThreads] : none;
}

// Preference 1 of 3: the sequences' sums.
__global__ __launch_bounds__(kThreads) void preference_sums(Loss l) {
    __shared__ List list;
    __shared__ Sums held[kThreads / 64][kLong];
    __shared__ double scratch[kChunk];
    const int64_t at = (int64_t)blockIdx.x * kChunk + threadIdx.x;
    float lp[kEach], ref[kEach];
    int32_t id[kEach];
    load_tokens(l.logprob, at, l.n, 0.f, lp);
    load_tokens(l.other, at, l.n, 0.f, ref);
    load_tokens(l.ids, at, l.n, 0, id);
    const Chunk c = chunk_of(l, 2 * l.items, blockIdx.x);
    const int count = list_sequences(l, c, list);
    uint32_t of[kEach];
    find_sequences(list, count, reinterpret_cast<uint16_t*>(scratch), of);
    Sums term[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) term[i] = {id[i] >= 0 ? (double)lp[i] - (double)ref[i] : 0.0, 0.0, id[i] >= 0, 0};
    sum_sequences<1>(l, list, count, held, scratch, of, term);
}

// 2 of 3: the pairs' losses, a wave each.
__global__ __launch_bounds__(kThreads) void preference_pairs(Loss l) {
    const int item = blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    if (item >= l.items) return;
    const double weight = l.weight ? (double)l.weight[item] : 1.0;
    double mean[2], ratio[2], loss = 0.0, slope = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        Sums s = sequence_sum(l, 2 * item + i);
        if (weight == 0.0) s = {0.0, 0.0, 0, 0};
        mean[i] = l.mean && s.live ? 1.0 / s.live : 1.0;
        ratio[i] = s.a * mean[i];
    }
    if (weight != 0.0) preference(l, ratio[0] - ratio[1], loss, slope);
    if (threadIdx.x & 63) return;
    l.loss[item] = (float)loss;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l.second[2 * item + i] = (float)(l.beta * ratio[i]);
        l.slopes[2 * item + i] = weight != 0.0 ? (i ? -slope : slope) * weight * mean[i] : 0.0;
    }
}

// 3 of 3: the tokens' gradients.
__global__ __launch_bounds__(kThreads) void preference_grad(Loss l) {
    __shared__ List list;
    __shared__ float slope[kChunk];
    __shared__ uint16_t scratch[kChunk];
    const int64_t at = (int64_t)blockIdx.x * kChunk + threadIdx.x;
    int32_t id[kEach];
    load_tokens(l.ids, at, l.n, 0, id);
    const Chunk c = chunk_of(l, 2 * l.items, blockIdx.x);
    const int count = list_sequences(l, c, list);
    for (int i = threadIdx.x; i < count; i += kThreads) slope[i] = (float)l.slopes[list.seq[i]];
    uint32_t of[kEach];
    find_sequences(list, count, scratch, of);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        if (at + i * kThreads < c.to) l.grad[at + i * kThreads] = of[i] < kOn && id[i] >= 0 ? slope[of[i] & (kChunk - 1)] : 0.f;
}

// Policy 1 of 3, for means over the tokens with an id: how many there are.  A
// work-group takes up to kCounted chunks one after the other; where one sequence
// covers several of them, it adds to that one's number once (65536 additions to
// one place took 0.7 ms).
constexpr int kCounted = 32;
__global__ __launch_bounds__(kThreads) void policy_counts(Loss l, int chunks, int each) {
    __shared__ List list;
    __shared__ Sums held[kThreads / 64][kLong];
    __shared__ double scratch[kChunk / 2];
    __shared__ int32_t counts[kThreads / 64];
    const int begin = blockIdx.x * each, end = min(begin + each, chunks);
    int32_t mine = 0, whose = -1;     // this thread's tokens of the sequence that covers the chunks
    auto hand_over = [&]() {
        if (whose < 0) return;
        const int32_t n = edb::lanes::sum<64>(mine);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) counts[threadIdx.x >> 6] = n;
        __syncthreads();
        if (threadIdx.x == 0) {
            int32_t all = 0;
#pragma unroll
            for (int w = 0; w < kThreads / 64; ++w) all += counts[w];
            atomicAdd(&l.whole[whose].live, all);
        }
        mine = 0;
        whose = -1;
    };
    for (int chunk = begin; chunk < end; ++chunk) {
        const int64_t at = (int64_t)chunk * kChunk + threadIdx.x;
        int32_t id[kEach];
        load_tokens(l.ids, at, l.n, 0, id);
        const Chunk c = chunk_of(l, l.items, chunk);
        __syncthreads();              // the list of the chunk before is done with
        const int count = list_sequences(l, c, list);
        if (count == 1 && (list.from[0] & list.to[0] & kOn)) {
            const int seq = list.seq[0];
            if (seq != whose) hand_over();
            whose = seq;
#pragma unroll
            for (int i = 0; i < kEach; ++i) mine += id[i] >= 0;
            continue;
        }
        hand_over();
        uint32_t of[kEach];
        find_sequences(list, count, reinterpret_cast<uint16_t*>(scratch), of);
        Sums term[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) term[i] = {0.0, 0.0, id[i] >= 0, 0};
        sum_sequences<0>(l, list, count, held, scratch, of, term);
    }
    hand_over();
}

// 2 of 3: the tokens' terms and gradients, and the sequences' sums.
__global__ __launch_bounds__(kThreads) void policy_terms(Loss l) {
    __shared__ List list;
    __shared__ Sums held[kThreads / 64][kLong];
    __shared__ double scratch[kChunk];     // a sequence's weight over its tokens, then the tokens' terms
    __shared__ float advantages[kChunk];
    const int64_t at = (int64_t)blockIdx.x * kChunk + threadIdx.x;
    float lp[kEach], old[kEach], ref[kEach], each[kEach];
    int32_t id[kEach];
    load_tokens(l.logprob, at, l.n, 0.f, lp);
    load_tokens(l.other, at, l.n, 0.f, old);
    load_tokens(l.reference, at, l.n, 0.f, ref);
    load_tokens(l.ids, at, l.n, 0, id);
    load_tokens(l.per_token ? l.advantage : nullptr, at, l.n, 0.f, each);
    const Chunk c = chunk_of(l, l.items, blockIdx.x);
    const int count = list_sequences(l, c, list);
    for (int i = threadIdx.x; i < count; i += kThreads) {
        const int s = list.seq[i];
        const double weight = l.weight ? (double)l.weight[s] : 1.0;
        int live = 1;
        if (l.counted) live = l.whole[s].live;
        else if (l.mean) {
            const Range r = range_of(l, s);
            live = r.to - r.from;
        }
        scratch[i] = live ? weight / live : weight;
        advantages[i] = l.per_token ? 0.f : l.advantage[s];
    }
    __shared__ uint16_t places[kChunk];
    uint32_t of[kEach];
    find_sequences(list, count, places, of);
    __syncthreads();
    double scale[kEach], a[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t s = of[i];
        scale[i] = s < kOn && id[i] >= 0 ? scratch[s & (kChunk - 1)] : 0.0;
        a[i] = l.per_token ? each[i] : advantages[s & (kChunk - 1)];
    }
    Sums term[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int64_t t = at + i * kThreads;
        const bool live = scale[i] != 0.0;
        const Token k = policy(l, lp[i], old[i], ref[i], a[i]);
        term[i] = {live ? k.gain : 0.0, live ? k.kl : 0.0, live, live && k.clipped};
        if (t < c.to) l.grad[t] = live ? (float)(k.slope * scale[i]) : 0.f;
    }
    sum_sequences<2>(l, list, count, held, scratch, of, term);
}

// 3 of 3: the sequences' losses, a wave each.
__global__ __launch_bounds__(kThreads) void policy_losses(Loss l) {
    const int s = blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    if (s >= l.items) return;
    const Sums sum = sequence_sum(l, s);
    if (threadIdx.x & 63) return;
    const double mean = l.mean && sum.live ? 1.0 / sum.live : 1.0;
    l.loss[s] = (float)(policy_loss(l, sum.a, sum.b) * mean);
    l.second[s] = (float)(sum.b * mean);
    l.clipped[s] = sum.clipped;
}

// Up to so many tokens, and so many a pair or sequence, are taken by one launch
// (policy, us: 32768 in 64 sequences 8.0, by the long calls' four launches 17; in 2
// sequences 22 and 17, in one 40 and 17).  Where most are in one of many sequences
// after all, its group is alone with them: 32768 in one of 64 take 95, in one of 4096,
// where a group is a wave, 340.
constexpr int32_t kFew = 32768, kFewEach = 8192;
constexpr int32_t kShort = 128;    // tokens a pair or sequence, on average, up to which a wave takes it
constexpr int32_t kMostItems = 1 << 24;

struct Plan {
    int32_t chunks;          // 0: one launch
    int64_t places, whole, slopes, bytes;
};
Plan plan_of(int32_t n, int32_t sequences, bool pairs) {
    Plan p{};
    const int32_t items = pairs ? sequences / 2 : sequences;
    if (items == 0 || (n <= kFew && n / items <= kFewEach)) return p;
    p.chunks = (int32_t)(((int64_t)n + kChunk - 1) / kChunk);
    p.places = (int64_t)p.chunks * 2 * sizeof(Sums);
    p.whole = p.places + ((int64_t)p.chunks * 4 + 15) / 16 * 16;
    p.slopes = p.whole + (int64_t)sequences * sizeof(Sums);
    p.bytes = p.slopes + (pairs ? (int64_t)sequences * 8 : 0);
    return p;
}

Region words(const void* p, int64_t n) { return Region::array(p, n * 4); }

edb_status launched(const char* who) {
    const hipError_t he = hipGetLastError();
    if (he != hipSuccess) return fail(EDB_ERR_HIP, std::string(who) + ": " + hipGetErrorString(he));
    edb::clear_error();
    return EDB_OK;
}

edb_status check_items(const char* who, int32_t n, int32_t items, const char* name) {
    const std::string w(who);
    if (n < 0 || items < 0) return fail(EDB_ERR_INVALID, w + ": n >= 0 and " + name + " >= 0 are needed");
    if (items > kMostItems) return fail(EDB_ERR_UNSUPPORTED, w + ": " + name + " must not exceed 2^24");
    return EDB_OK;
}

bool in_range(double v, double lo, double hi) { return v >= lo && v <= hi && std::isfinite(v); }

__global__ __launch_bounds__(256) void no_sequences(float* grad, int32_t n) {
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < n) grad[t] = 0.f;
}

unsigned groups(int64_t n, int64_t per) { return (unsigned)((n + per - 1) / per); }

}  // namespace

extern "C" edb_status edb_preference_loss_bytes(int32_t n, int32_t pairs, int64_t* bytes) {
    return edb::guarded([&]() -> edb_status {
        if (!bytes) return fail(EDB_ERR_INVALID, "edb_preference_loss_bytes: NULL argument");
        if (edb_status st = check_items("edb_preference_loss_bytes", n, pairs, "pairs")) return st;
        *bytes = plan_of(n, 2 * pairs, true).bytes;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_preference_loss(const float* logprob, const float* reference, const int32_t* ids, int32_t n,
                                     const int32_t* first, int32_t pairs, int32_t kind, double beta, double smoothing,
                                     int32_t mean, const float* weight, float* loss, float* reward, float* g_logprob,
                                     void* workspace, int64_t workspace_bytes, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_preference_loss";
        if (edb_status st = check_items(who, n, pairs, "pairs")) return st;
        if (kind < EDB_PREFERENCE_LOGISTIC || kind > EDB_PREFERENCE_SQUARED)
            return fail(EDB_ERR_INVALID, "edb_preference_loss: unknown kind of loss");
        if (!(beta > 0.0) || !std::isfinite(beta)) return fail(EDB_ERR_INVALID, "edb_preference_loss: beta must be positive and finite");
        if (!in_range(smoothing, 0.0, 1.0) || (smoothing != 0.0 && kind != EDB_PREFERENCE_LOGISTIC))
            return fail(EDB_ERR_INVALID, "edb_preference_loss: smoothing must be in [0, 1], and 0 but for the logistic loss");
        if ((n && (!logprob || !g_logprob)) || (pairs && (!first || !loss || !reward)))
            return fail(EDB_ERR_INVALID, "edb_preference_loss: NULL argument");
        const Plan p = plan_of(n, 2 * pairs, true);
        if (workspace_bytes < p.bytes || (p.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
            return fail(EDB_ERR_INVALID, "edb_preference_loss: a 16-byte aligned workspace of " + std::to_string(p.bytes) +
                                             " bytes is needed");
        if (!edb::word_aligned({logprob, reference, ids, first, weight, loss, reward, g_logprob}))
            return fail(EDB_ERR_INVALID, "edb_preference_loss: all arrays must be aligned to 4 bytes");
        if (edb_status st = edb::apart(who,
                                       {words(loss, pairs), words(reward, 2 * (int64_t)pairs), words(g_logprob, n),
                                        Region::array(workspace, p.bytes)},
                                       {words(logprob, n), words(reference, n), words(ids, n),
                                        words(first, pairs ? 2 * (int64_t)pairs + 1 : 0), words(weight, pairs)}))
            return st;
        if (n == 0 && pairs == 0) {
            edb::clear_error();
            return EDB_OK;
        }
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        Loss l{};
        l.logprob = logprob;
        l.other = reference;
        l.ids = ids;
        l.n = n;
        l.first = first;
        l.items = pairs;
        l.kind = kind;
        l.beta = beta;
        l.smoothing = smoothing;
        l.mean = mean != 0;
        l.weight = weight;
        l.loss = loss;
        l.second = reward;
        l.grad = g_logprob;
        if (pairs == 0) {
            if (n) no_sequences<<<groups(n, 256), 256, 0, st>>>(g_logprob, n);
        } else if (p.chunks == 0) {
            if (n / pairs < kShort) preference_kernel<64><<<groups(pairs, 4), 256, 0, st>>>(l);
            else if (n / pairs < 16 * kShort) preference_kernel<256><<<pairs, 256, 0, st>>>(l);
            else preference_kernel<1024><<<pairs, 1024, 0, st>>>(l);
        } else {
            char* ws = static_cast<char*>(workspace);
            l.parts = reinterpret_cast<Sums*>(ws);
            l.places = reinterpret_cast<int32_t*>(ws + p.places);
            l.whole = reinterpret_cast<Sums*>(ws + p.whole);
            place_chunks<<<groups(2 * (int64_t)pairs + 1, kThreads), kThreads, 0, st>>>(l, 2 * pairs);
            l.slopes = reinterpret_cast<double*>(ws + p.slopes);
            preference_sums<<<p.chunks, kThreads, 0, st>>>(l);
            preference_pairs<<<groups(pairs, kThreads / 64), kThreads, 0, st>>>(l);
            preference_grad<<<p.chunks, kThreads, 0, st>>>(l);
        }
        return launched(who);
    });
}

extern "C" edb_status edb_policy_loss_bytes(int32_t n, int32_t sequences, int64_t* bytes) {
    return edb::guarded([&]() -> edb_status {
        if (!bytes) return fail(EDB_ERR_INVALID, "edb_policy_loss_bytes: NULL argument");
        if (edb_status st = check_items("edb_policy_loss_bytes", n, sequences, "sequences")) return st;
        *bytes = plan_of(n, sequences, false).bytes;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_policy_loss(const float* logprob, const float* old_logprob, const float* reference, const int32_t* ids,
                                 int32_t n, const int32_t* first, int32_t sequences, const float* advantage,
                                 int32_t per_token, double low, double high, double kl, int32_t mean, const float* weight,
                                 float* loss, float* divergence, int32_t* clipped, float* g_logprob, void* workspace,
                                 int64_t workspace_bytes, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_policy_loss";
        if (edb_status st = check_items(who, n, sequences, "sequences")) return st;
        if (!in_range(low, 0.0, 1.0) || !(high >= 0.0) || !std::isfinite(high))
            return fail(EDB_ERR_INVALID, "edb_policy_loss: low must be in [0, 1], high finite and not negative");
        if (!(kl >= 0.0) || !std::isfinite(kl)) return fail(EDB_ERR_INVALID, "edb_policy_loss: kl must be finite and not negative");
        if (kl != 0.0 && !reference) return fail(EDB_ERR_INVALID, "edb_policy_loss: the divergence needs a reference");
        if ((n && (!logprob || !old_logprob || !g_logprob)) || (sequences && (!first || !loss || !divergence || !clipped)) ||
            ((per_token ? n : sequences) && !advantage))
            return fail(EDB_ERR_INVALID, "edb_policy_loss: NULL argument");
        const Plan p = plan_of(n, sequences, false);
        if (workspace_bytes < p.bytes || (p.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
            return fail(EDB_ERR_INVALID, "edb_policy_loss: a 16-byte aligned workspace of " + std::to_string(p.bytes) +
                                             " bytes is needed");
        if (!edb::word_aligned({logprob, old_logprob, reference, ids, first, advantage, weight, loss, divergence, clipped, g_logprob}))
            return fail(EDB_ERR_INVALID, "edb_policy_loss: all arrays must be aligned to 4 bytes");
        if (edb_status st = edb::apart(who,
                                       {words(loss, sequences), words(divergence, sequences), words(clipped, sequences),
                                        words(g_logprob, n), Region::array(workspace, p.bytes)},
                                       {words(logprob, n), words(old_logprob, n), words(reference, n), words(ids, n),
                                        words(first, sequences ? (int64_t)sequences + 1 : 0),
                                        words(advantage, per_token ? n : sequences), words(weight, sequences)}))
            return st;
        if (n == 0 && sequences == 0) {
            edb::clear_error();
            return EDB_OK;
        }
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        Loss l{};
        l.logprob = logprob;
        l.other = old_logprob;
        l.reference = reference;
        l.ids = ids;
        l.n = n;
        l.first = first;
        l.items = sequences;
        l.advantage = advantage;
        l.per_token = per_token != 0;
        l.low = 1.0 - low;
        l.high = 1.0 + high;
        l.log_low = std::log(l.low);
        l.log_high = std::log(l.high);
        l.coef = kl;
        l.mean = mean != 0;
        l.weight = weight;
        l.loss = loss;
        l.second = divergence;
        l.clipped = clipped;
        l.grad = g_logprob;
        if (sequences == 0) {
            if (n) no_sequences<<<groups(n, 256), 256, 0, st>>>(g_logprob, n);
        } else if (p.chunks == 0) {
            if (n / sequences < kShort) policy_kernel<64><<<groups(sequences, 4), 256, 0, st>>>(l);
            else if (n / sequences < 16 * kShort) policy_kernel<256><<<sequences, 256, 0, st>>>(l);
            else policy_kernel<1024><<<sequences, 1024, 0, st>>>(l);
        } else {
            char* ws = static_cast<char*>(workspace);
            l.parts = reinterpret_cast<Sums*>(ws);
            l.places = reinterpret_cast<int32_t*>(ws + p.places);
            l.whole = reinterpret_cast<Sums*>(ws + p.whole);
            l.counted = l.mean && ids;
            place_chunks<<<groups((int64_t)sequences + 1, kThreads), kThreads, 0, st>>>(l, sequences);
            if (l.counted) {
                // (2048 work-groups fill the card)
                const int each = p.chunks >= 2048 * kCounted ? kCounted : (p.chunks + 2047) / 2048;
                policy_counts<<<groups(p.chunks, each), kThreads, 0, st>>>(l, p.chunks, each);
            }
            policy_terms<<<p.chunks, kThreads, 0, st>>>(l);
            policy_losses<<<groups(sequences, kThreads / 64), kThreads, 0, st>>>(l);
        }
        return launched(who);
    });
}
