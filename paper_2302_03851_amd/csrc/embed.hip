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

// K consecutive elements of a row as fp32: 8 or 4 where rows hold whole groups
// of so many (at any alignment), else 1.
template <class T, int K>
__device__ __forceinline__ void load_k(const T* p, float* v) {
    if constexpr (K == 1) {
        v[0] = Elem<T>::get(p);
    } else if constexpr (K < Elem<T>::kVec) {
        Elem<T>::unpack_half(Elem<T>::load_half(p), v);
    } else {
#pragma unroll
        for (int i = 0; i < K; i += Elem<T>::kVec) Elem<T>::unpack(Elem<T>::load(p + i), v + i);
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

// ---- the gradient: positions sorted by word, then sums over the runs of a word
//
// The sort is a stable radix sort of (word, position), so a word's rows are
// added in ascending position and the result does not depend on timing.  Ids
// that are no token get the word V and sort to the end.  Up to kBlockSort ids
// are sorted by one work-group in LDS; more by passes over digits of up to
// kMaxDigit bits, three launches each (counts per tile, their prefix sums, the
// scatter).  The zero rows of the result are written by further work-groups of
// the sorting launches, which leave the memory idle.

constexpr int kBlockSort = 8192;   // ids of the one-work-group sort: keys, positions and counts fill 56 KB of LDS
constexpr int kMaxDigit = 10;
constexpr int kTile = 2048;        // ids a work-group of the large sort ranks: 4 waves of 8 rounds
constexpr int kRounds = 8;

struct FillArgs {  // rows to zero: `share` of `shares` equal parts, by the work-groups from `first` on
    void* rows;
    int64_t stride_bytes, row_bytes, n_rows;
    int32_t share, shares, first;
};

// Zeroes its part of the rows: as one range of 16-byte pieces where the rows
// are dense, otherwise row by row in 2-byte units.
__device__ __forceinline__ void fill_share(const FillArgs& f, int threads) {
    const int64_t r0 = f.n_rows * f.share / f.shares, r1 = f.n_rows * (f.share + 1) / f.shares;
    const int64_t step = (int64_t)(gridDim.x - f.first) * threads;
    const int64_t me = (int64_t)(blockIdx.x - f.first) * threads + threadIdx.x;
    char* base = static_cast<char*>(f.rows);
    if (f.stride_bytes == f.row_bytes) {
        char* p = base + r0 * f.row_bytes;
        const int64_t bytes = (r1 - r0) * f.row_bytes, whole = bytes >> 4;
        for (int64_t i = me; i < whole; i += step) *reinterpret_cast<u32x4_a2*>(p + (i << 4)) = u32x4{0u, 0u, 0u, 0u};
        const int64_t rest = (bytes - (whole << 4)) >> 1;
        if (me < rest) *reinterpret_cast<uint16_t*>(p + (whole << 4) + 2 * me) = 0;
    } else {
        const int64_t units = f.row_bytes >> 1;
        for (int64_t r = r0 + me / units, c = me % units; r < r1;) {
            *reinterpret_cast<uint16_t*>(base + r * f.stride_bytes + 2 * c) = 0;
            c += step;
            r += c / units;
            c %= units;
        }
    }
}

__device__ __forceinline__ uint32_t word_of(int32_t id, uint32_t vocab) {
    return (uint32_t)id < vocab ? (uint32_t)id : vocab;
}

// Lanes of the wave with this lane's digit (of `bits` bits), among those of `valid`.
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, int bits, uint64_t valid) {
    uint64_t m = valid;
    for (int b = 0; b < bits; ++b) {
        const bool one = (digit >> b) & 1;
        const uint64_t v = __ballot(one);
        m &= one ? v : ~v;
    }
    return m;
}

__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }

__device__ __forceinline__ uint32_t wave_scan_inclusive(uint32_t v) {
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(v, d);
        if (lane_id() >= d) v += o;
    }
    return v;
}

struct SortArgs {
    const int32_t* ids;          // pass 0 reads the ids
    const uint32_t *keys, *pos;  // later passes read these
    uint32_t *keys_out, *pos_out;
    uint32_t* counts;            // [bin][tile]; their prefix sums after sort_scan
    uint32_t* totals;            // [bin]
    int32_t n, tiles, shift, bits;
    uint32_t vocab;
    FillArgs fill;
};

// One work-group, everything in LDS: passes of 8 bits.  Each of the 16 waves
// ranks a contiguous eighth-kilo of ids, so the order (digit, wave, round,
// lane) is the stable one.
__global__ __launch_bounds__(1024) void sort_block(SortArgs a) {
    if (blockIdx.x) {
        fill_share(a.fill, 1024);
        return;
    }
    constexpr int kWaves = 16, kBins = 256, kPer = kBlockSort / 1024;
    __shared__ uint32_t keys[kBlockSort];
    __shared__ uint16_t pos[kBlockSort];
    __shared__ uint16_t count[kBins][kWaves];
    __shared__ uint32_t wave_sum[kWaves];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    const int rounds = (a.n + 1023) / 1024, first = wave * rounds * 64;
    uint32_t k[kPer], p[kPer], rank[kPer];
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
        const int i = first + r * 64 + lane;
        p[r] = i;
        k[r] = r < rounds && i < a.n ? word_of(a.ids[i], a.vocab) : a.vocab;
    }
    for (int shift = 0;; shift += 8) {
        for (int i = tid; i < kBins * kWaves; i += 1024) (&count[0][0])[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kPer; ++r)
            if (r < rounds) {
                const bool valid = first + r * 64 + lane < a.n;
                const uint32_t d = (k[r] >> shift) & 255;
                const uint64_t m = same_digit(d, 8, __ballot(valid));
                const int before = __popcll(m & ((1ull << lane) - 1));
                if (valid) rank[r] = count[d][wave] + before;
                // the last lane of a digit updates its count, after every lane has read it
                __builtin_amdgcn_wave_barrier();
                if (valid && (m >> lane) == 1) count[d][wave] = (uint16_t)(rank[r] + 1);
                __builtin_amdgcn_wave_barrier();
            }
        __syncthreads();
        // exclusive sums in the order (digit, wave): four counts a thread
        uint32_t c[4], sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            c[i] = (&count[0][0])[4 * tid + i];
            sum += c[i];
        }
        const uint32_t upto = wave_scan_inclusive(sum);
        if (lane == 63) wave_sum[wave] = upto;
        __syncthreads();
        uint32_t base = upto - sum;
        for (int w = 0; w < wave; ++w) base += wave_sum[w];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            (&count[0][0])[4 * tid + i] = (uint16_t)base;
            base += c[i];
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kPer; ++r)
            if (r < rounds && first + r * 64 + lane < a.n) {
                const int to = count[(k[r] >> shift) & 255][wave] + (int)rank[r];
                keys[to] = k[r];
                pos[to] = (uint16_t)p[r];
            }
        __syncthreads();
        if (shift + 8 >= a.bits) break;
#pragma unroll
        for (int r = 0; r < kPer; ++r) {
            const int i = first + r * 64 + lane;
            if (r < rounds && i < a.n) {
                k[r] = keys[i];
                p[r] = pos[i];
            }
        }
    }
    for (int i = tid; i < a.n; i += 1024) {
        a.keys_out[i] = keys[i];
        a.pos_out[i] = pos[i];
    }
}

__device__ __forceinline__ uint32_t sort_key(const SortArgs& a, int i) {
    return a.ids ? word_of(a.ids[i], a.vocab) : a.keys[i];
}

// counts[bin][tile] of one digit.
__global__ __launch_bounds__(256) void sort_count(SortArgs a) {
    if ((int)blockIdx.x >= a.tiles) {
        fill_share(a.fill, 256);
        return;
    }
    __shared__ uint32_t count[1 << kMaxDigit];
    const int bins = 1 << a.bits, tile = blockIdx.x;
    for (int b = threadIdx.x; b < bins; b += 256) count[b] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kTile / 256; ++r) {
        const int64_t i = (int64_t)tile * kTile + r * 256 + threadIdx.x;
        if (i < a.n) atomicAdd(&count[(sort_key(a, (int)i) >> a.shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += 256) a.counts[(int64_t)b * a.tiles + tile] = count[b];
}

// Prefix sums of a bin's counts over the tiles: a wave a bin.
__global__ __launch_bounds__(256) void sort_scan(SortArgs a) {
    const int scanners = ((1 << a.bits) + 3) / 4;
    if ((int)blockIdx.x >= scanners) {
        fill_share(a.fill, 256);
        return;
    }
    const int bin = blockIdx.x * 4 + (threadIdx.x >> 6), lane = lane_id();
    if (bin >= 1 << a.bits) return;
    uint32_t* c = a.counts + (int64_t)bin * a.tiles;
    uint32_t base = 0;
    for (int t = 0; t < a.tiles; t += 64) {
        const uint32_t v = t + lane < a.tiles ? c[t + lane] : 0, upto = wave_scan_inclusive(v);
        if (t + lane < a.tiles) c[t + lane] = base + upto - v;
        base += __shfl(upto, 63);
    }
    if (lane == 0) a.totals[bin] = base;
}

// Ranks a tile's ids and writes them to their places.
__global__ __launch_bounds__(256) void sort_scatter(SortArgs a) {
    if ((int)blockIdx.x >= a.tiles) {
        fill_share(a.fill, 256);
        return;
    }
    constexpr int kBins = 1 << kMaxDigit;
    __shared__ uint32_t at[4][kBins];  // per wave: counts, then the next place of a digit
    __shared__ uint32_t wave_sum[4];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6, tile = blockIdx.x, bins = 1 << a.bits;
    for (int b = lane; b < bins; b += 64) at[wave][b] = 0;
    // each thread owns four neighbouring bins
    uint32_t total[kBins / 256], sum = 0;
#pragma unroll
    for (int i = 0; i < kBins / 256; ++i) {
        const int b = tid * (kBins / 256) + i;
        total[i] = b < bins ? a.totals[b] : 0;
        sum += total[i];
    }
    const uint32_t upto = wave_scan_inclusive(sum);
    if (lane == 63) wave_sum[wave] = upto;
    const int64_t first = (int64_t)tile * kTile + wave * (kTile / 4);
    uint32_t k[kRounds], p[kRounds], rank[kRounds];
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int64_t i = first + r * 64 + lane;
        k[r] = i < a.n ? sort_key(a, (int)i) : 0;
        p[r] = i < a.n ? (a.ids ? (uint32_t)i : a.pos[i]) : 0;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const bool valid = first + r * 64 + lane < a.n;
        const uint32_t d = (k[r] >> a.shift) & (bins - 1);
        const uint64_t m = same_digit(d, a.bits, __ballot(valid));
        if (valid) rank[r] = at[wave][d] + __popcll(m & ((1ull << lane) - 1));
        __builtin_amdgcn_wave_barrier();
        if (valid && (m >> lane) == 1) at[wave][d] = rank[r] + 1;
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    uint32_t base = upto - sum;
    for (int w = 0; w < wave; ++w) base += wave_sum[w];
#pragma unroll
    for (int i = 0; i < kBins / 256; ++i) {
        const int b = tid * (kBins / 256) + i;
        if (b < bins) {
            uint32_t next = base + a.counts[(int64_t)b * a.tiles + tile];
            for (int w = 0; w < 4; ++w) {
                const uint32_t c = at[w][b];
                at[w][b] = next;
                next += c;
            }
        }
        base += total[i];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRounds; ++r)
        if (first + r * 64 + lane < a.n) {
            const uint32_t to = at[wave][(k[r] >> a.shift) & (bins - 1)] + rank[r];
            a.keys_out[to] = k[r];
            a.pos_out[to] = p[r];
        }
}

struct SumArgs {
    const uint32_t *keys, *pos;  // sorted; readable to a multiple of 8
    int32_t n, chunk;            // chunk: a multiple of 8
    uint32_t vocab;
    int32_t dim, lanes;          // lanes: a power of two up to 64 that share a row
    const void* dout;
    int64_t dout_stride;
    float scale;
    int32_t accumulate;
    void* dtable;
    int64_t dtable_stride;
    float* partial;              // [chunks][2][dim]
};

template <class O, int K>
__device__ __forceinline__ void put_word(const SumArgs& a, uint32_t word, int col, const float* sum) {
    O* d = static_cast<O*>(a.dtable) + word * a.dtable_stride + col;
    float v[K];
    if (a.accumulate) {
        load_k<O, K>(d, v);
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = __builtin_fmaf(sum[k], a.scale, v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = sum[k] * a.scale;
    }
    store_k<O, K>(d, v);
}

// Eight neighbouring entries of the sorted lists.  WAVE: the same ones in every
// lane of the wave, kept in scalar registers.
template <bool WAVE>
struct Eight {
    uint32_t key[8], pos[8];

    __device__ __forceinline__ void load(const SumArgs& a, int i) {
        u32x4 v[4];
        v[0] = *reinterpret_cast<const u32x4*>(a.keys + i);
        v[1] = *reinterpret_cast<const u32x4*>(a.keys + i + 4);
        v[2] = *reinterpret_cast<const u32x4*>(a.pos + i);
        v[3] = *reinterpret_cast<const u32x4*>(a.pos + i + 4);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            key[u] = v[u >> 2][u & 3];
            pos[u] = v[2 + (u >> 2)][u & 3];
        }
    }
    __device__ __forceinline__ void settle() {
        if constexpr (WAVE)
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                key[u] = __builtin_amdgcn_readfirstlane(key[u]);
                pos[u] = __builtin_amdgcn_readfirstlane(pos[u]);
            }
    }
};

// A group of lanes adds up the runs of one chunk of the sorted positions, K
// columns a lane, eight rows in flight.  A run that lies inside the chunk is
// final; the part of one that came in from the chunk before goes to the
// chunk's first partial row, of one that only goes on to the next to the second.
// All eight entries are there before the first row is asked for (loads return
// in order: a wait for a later entry would wait for the rows before it too),
// and a place without a row reads its chunk's first one, without a branch.
template <class T, class O, int K, bool WAVE>
__global__ __launch_bounds__(256) void sum_chunks(SumArgs a) {
    int chunk;
    if constexpr (WAVE) chunk = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    else chunk = (int)(((int64_t)blockIdx.x * 256 + threadIdx.x) / a.lanes);
    const int lanes = WAVE ? 64 : a.lanes;
    const int col = (blockIdx.y * lanes + (threadIdx.x & (lanes - 1))) * K;
    const int64_t begin64 = (int64_t)chunk * a.chunk;
    if (begin64 >= a.n || col >= a.dim) return;
    const int begin = (int)begin64, end = (int)min((int64_t)a.n, begin64 + a.chunk);
    const T* rows = static_cast<const T*>(a.dout) + col;
    float* partial = a.partial + 2 * (int64_t)chunk * a.dim + col;
    Eight<WAVE> at;
    at.load(a, begin);
    const uint32_t before = begin > 0 ? a.keys[begin - 1] : a.vocab, after = end < a.n ? a.keys[end] : a.vocab;
    at.settle();
    uint32_t cur = at.key[0];
    if (cur >= a.vocab) return;  // only ids that are no token
    bool from_before = before == cur;
    const uint32_t some = at.pos[0];
    float sum[K] = {};
    for (int i = begin; i < end; i += 8) {
        float v[8][K];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const uint32_t p = i + u < end ? at.pos[u] : some;
            load_k<T, K>(rows + p * a.dout_stride, v[u]);
        }
        const Eight<WAVE> now = at;
        if (i + 8 < end) at.load(a, i + 8);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (i + u >= end) break;
            if (now.key[u] != cur) {
                if (from_before) store_k<float, K>(partial, sum);
                else put_word<O, K>(a, cur, col, sum);
                from_before = false;
                cur = now.key[u];
                if (cur >= a.vocab) return;
#pragma unroll
                for (int k = 0; k < K; ++k) sum[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < K; ++k) sum[k] += v[u][k];
        }
        at.settle();
    }
    if (from_before) store_k<float, K>(partial, sum);
    else if (after == cur) store_k<float, K>(partial + a.dim, sum);
    else put_word<O, K>(a, cur, col, sum);
}

constexpr int kJoinThreads = 256;

// A work-group a chunk: where a run begins in the chunk and goes on after it,
// adds the run's partial rows, a contiguous part of them for each group of lanes.
template <class O, int K>
__global__ __launch_bounds__(kJoinThreads) void join_chunks(SumArgs a) {
    const int64_t chunk = blockIdx.x, begin = chunk * a.chunk, end = begin + a.chunk;
    if (end >= a.n) return;
    const uint32_t word = a.keys[end - 1];
    if (word >= a.vocab || a.keys[end] != word) return;
    if (begin > 0 && a.keys[begin] == word && a.keys[begin - 1] == word) return;
    // the chunks after this one that begin with the word
    int64_t more = 0;
    const int lane = lane_id();
    for (;;) {
        const int64_t at = end + (more + lane) * a.chunk;
        const uint64_t m = __ballot(at < a.n && a.keys[at < a.n ? at : 0] == word);
        const int run = m == ~0ull ? 64 : __ffsll((unsigned long long)~m) - 1;
        more += run;
        if (run < 64) break;
    }
    const int64_t n = more + 1;  // partial rows: this chunk's second, then the others' first ones
    const int group = threadIdx.x / a.lanes, groups = kJoinThreads / a.lanes;
    const int col = (blockIdx.y * a.lanes + (threadIdx.x & (a.lanes - 1))) * K;
    const int64_t per = (n + groups - 1) / groups, i0 = group * per, i1 = min(n, i0 + per);
    float sum[K] = {};
    if (col < a.dim) {
        for (int64_t i = i0; i < i1; i += 8) {
            float v[8][K];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u < i1) load_k<float, K>(a.partial + (2 * (chunk + i + u) + (i + u == 0 ? 1 : 0)) * a.dim + col, v[u]);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u < i1)
#pragma unroll
                    for (int k = 0; k < K; ++k) sum[k] += v[u][k];
        }
    }
    __shared__ float part[kJoinThreads][K];
#pragma unroll
    for (int k = 0; k < K; ++k) part[threadIdx.x][k] = sum[k];
    __syncthreads();
    if (group || col >= a.dim) return;
    const int used = (int)((n + per - 1) / per);
    for (int g = 1; g < used; ++g)
#pragma unroll
        for (int k = 0; k < K; ++k) sum[k] += part[g * a.lanes + threadIdx.x][k];
    put_word<O, K>(a, word, col, sum);
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

// Elements a lane takes of a row of `dim`.
int piece_of(int dim) { return dim % 8 == 0 ? 8 : dim % 4 == 0 ? 4 : 1; }

template <class T, class O>
void launch_embed(const EmbedArgs& a, hipStream_t st) {
    const int k = piece_of(a.dim);
    const dim3 grid((unsigned)(((int64_t)a.n * (a.dim / k) + 255) / 256));
    if (k == 8) embed_kernel<T, O, 8><<<grid, 256, 0, st>>>(a);
    else if (k == 4) embed_kernel<T, O, 4><<<grid, 256, 0, st>>>(a);
    else embed_kernel<T, O, 1><<<grid, 256, 0, st>>>(a);
}

// How the gradient's work is laid out, and its scratch memory.
struct GradPlan {
    int32_t piece, lanes, tiles_y, chunk, chunks;
    int32_t passes, digit, sort_tiles;
    int64_t keys[2], pos[2], counts, totals, partial, bytes;  // offsets
};

GradPlan grad_plan(int32_t n, int32_t vocab, int32_t dim) {
    GradPlan g{};
    g.piece = piece_of(dim);
    const int pieces = dim / g.piece;
    g.lanes = 1;
    while (g.lanes < 64 && g.lanes < pieces) g.lanes *= 2;
    g.tiles_y = (pieces + g.lanes - 1) / g.lanes;
    // enough chunks for every SIMD to hold several waves, and long ones where there are more than that
    int64_t chunk = (int64_t)n * g.lanes * g.tiles_y / (64 * 4096) / 8 * 8;
    g.chunk = (int32_t)(chunk < 8 ? 8 : chunk > 64 ? 64 : chunk);
    g.chunks = (int32_t)(((int64_t)n + g.chunk - 1) / g.chunk);
    int bits = 1;
    while ((int64_t)vocab >> bits) ++bits;   // the words and V itself
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    const int64_t list = ((int64_t)n + 7) / 8 * 8 * 4;
    if (n <= kBlockSort) {
        g.passes = 0;
        g.digit = bits;
        g.keys[0] = take(list);
        g.pos[0] = take(list);
    } else {
        g.passes = (bits + kMaxDigit - 1) / kMaxDigit;
        g.digit = (bits + g.passes - 1) / g.passes;
        g.sort_tiles = (int32_t)(((int64_t)n + kTile - 1) / kTile);
        for (int i = 0; i < 2; ++i) {
            g.keys[i] = take(list);
            g.pos[i] = take(list);
        }
        g.counts = take((int64_t)g.sort_tiles * 4 << g.digit);
        g.totals = take(INT64_C(4) << g.digit);
    }
    g.partial = take((int64_t)g.chunks * 2 * dim * 4);
    g.bytes = n ? at : 0;
    return g;
}

template <class T, class O, int K>
void launch_sums(const GradPlan& g, const SumArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)g.chunks * g.lanes + 255) / 256), g.tiles_y);
    if (g.lanes == 64) sum_chunks<T, O, K, true><<<grid, 256, 0, st>>>(a);
    else sum_chunks<T, O, K, false><<<grid, 256, 0, st>>>(a);
    if (g.chunks > 1) join_chunks<O, K><<<dim3(g.chunks, g.tiles_y), kJoinThreads, 0, st>>>(a);
}

template <class T, class O>
void launch_sums(const GradPlan& g, const SumArgs& a, hipStream_t st) {
    if (g.piece == 8) launch_sums<T, O, 8>(g, a, st);
    else if (g.piece == 4) launch_sums<T, O, 4>(g, a, st);
    else launch_sums<T, O, 1>(g, a, st);
}

// Work-groups that fill, beside the sorting ones of a launch.
int fill_groups(int64_t bytes, int threads) {
    const int64_t n = (bytes + 64 * threads - 1) / (64 * threads);
    return (int)(n > 2048 ? 2048 : n);
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
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    if (table_dtype == EDB_F32) {
        if (out_dtype == EDB_F32) launch_embed<float, float>(a, st);
        else launch_embed<float, bf16>(a, st);
    } else {
        if (out_dtype == EDB_F32) launch_embed<bf16, float>(a, st);
        else launch_embed<bf16, bf16>(a, st);
    }
    return launched(who);
}

extern "C" edb_status edb_embed_grad_bytes(int32_t n, int32_t vocab, int32_t dim, int64_t* bytes) {
    if (!bytes) return fail(EDB_ERR_INVALID, "edb_embed_grad_bytes: NULL argument");
    if (edb_status st = check_table("edb_embed_grad_bytes", n, vocab, dim, EDB_F32, EDB_F32, dim, dim, 1.f)) return st;
    *bytes = grad_plan(n, vocab, dim).bytes;
    edb::clear_error();
    return EDB_OK;
}

extern "C" edb_status edb_embed_grad(const int32_t* ids, int32_t n, const void* dout, int32_t dout_dtype, int32_t vocab,
                                     int32_t dim, int64_t dout_stride, float scale, int32_t accumulate, void* dtable,
                                     int32_t dtable_dtype, int64_t dtable_stride, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
    const char* who = "edb_embed_grad";
    if (edb_status st = check_table(who, n, vocab, dim, dout_dtype, dtable_dtype, dout_stride, dtable_stride, scale)) return st;
    if (!dtable || (n && (!ids || !dout))) return fail(EDB_ERR_INVALID, "edb_embed_grad: NULL argument");
    if (!element_aligned(dout, dout_dtype) || !element_aligned(dtable, dtable_dtype))
        return fail(EDB_ERR_INVALID, "edb_embed_grad: both gradients must be aligned to their elements");
    if (n && overlap(dout, ((n - 1) * dout_stride + dim) * elem_bytes(dout_dtype), dtable,
                     ((vocab - 1) * dtable_stride + dim) * elem_bytes(dtable_dtype)))
        return fail(EDB_ERR_INVALID, "edb_embed_grad: the table's gradient overlaps the rows' gradients");
    const GradPlan g = grad_plan(n, vocab, dim);
    if (workspace_bytes < g.bytes || (g.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
        return fail(EDB_ERR_INVALID, "edb_embed_grad: a 16-byte aligned workspace of " + std::to_string(g.bytes) +
                                         " bytes is needed");
    hipStream_t st = reinterpret_cast<hipStream_t>(stream);
    const int64_t row_bytes = dim * elem_bytes(dtable_dtype);
    FillArgs fill{dtable, dtable_stride * elem_bytes(dtable_dtype), row_bytes, accumulate ? 0 : vocab, 0, 1, 1};
    char* ws = static_cast<char*>(workspace);
    auto at = [&](int64_t off) { return reinterpret_cast<uint32_t*>(ws + off); };
    SortArgs s{};
    s.n = n;
    s.vocab = (uint32_t)vocab;
    int last = 0;
    if (g.passes == 0) {
        s.ids = ids;
        s.keys_out = at(g.keys[0]);
        s.pos_out = at(g.pos[0]);
        s.bits = g.digit;
        s.fill = fill;
        sort_block<<<1 + fill_groups(fill.n_rows * row_bytes, 1024), 1024, 0, st>>>(s);
    } else {
        s.tiles = g.sort_tiles;
        s.counts = at(g.counts);
        s.totals = at(g.totals);
        s.bits = g.digit;
        fill.shares = 3 * g.passes;
        const int beside = fill_groups(fill.n_rows * row_bytes / fill.shares, 256), scanners = ((1 << g.digit) + 3) / 4;
        for (int p = 0; p < g.passes; ++p) {
            s.ids = p ? nullptr : ids;
            s.keys = at(g.keys[(p + 1) & 1]);
            s.pos = at(g.pos[(p + 1) & 1]);
            s.keys_out = at(g.keys[p & 1]);
            s.pos_out = at(g.pos[p & 1]);
            s.shift = p * g.digit;
            last = p & 1;
            s.fill = fill;
            s.fill.first = g.sort_tiles;
            s.fill.share = 3 * p;
            sort_count<<<g.sort_tiles + beside, 256, 0, st>>>(s);
            s.fill.first = scanners;
            s.fill.share = 3 * p + 1;
            sort_scan<<<scanners + beside, 256, 0, st>>>(s);
            s.fill.first = g.sort_tiles;
            s.fill.share = 3 * p + 2;
            sort_scatter<<<g.sort_tiles + beside, 256, 0, st>>>(s);
        }
    }
    if (n) {
        const SumArgs a{at(g.keys[last]), at(g.pos[last]), n, g.chunk, (uint32_t)vocab, dim, g.lanes, dout, dout_stride,
                        scale, accumulate, dtable, dtable_stride, reinterpret_cast<float*>(ws + g.partial)};
        if (dout_dtype == EDB_F32) {
            if (dtable_dtype == EDB_F32) launch_sums<float, float>(g, a, st);
            else launch_sums<float, bf16>(g, a, st);
        } else {
            if (dtable_dtype == EDB_F32) launch_sums<bf16, float>(g, a, st);
            else launch_sums<bf16, bf16>(g, a, st);
        }
    }
    return launched(who);
}
