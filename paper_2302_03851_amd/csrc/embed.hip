// Embedding lookup with scaling, and the table's gradient.
//
//   y_i  = s W[id_i]                              (a zero row where id_i is outside [0, V))
//   dW_v = s sum over i with id_i = v of dy_i     (in fp32, in an order that the places of v fix)
#include <hip/hip_runtime.h>

#include <cmath>
#include <string>

#include "edb_internal.h"
#include "row_access.h"

using edb::fail;
using edb::Region;
using namespace edb::rows;

namespace {

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

struct EmbedArgs {
    const int32_t* ids;
    int32_t n, vocab, dim;
    const void* table;
    int64_t table_stride;
    float scale;
    void* out;
    int64_t out_stride;
};

// One thread per K elements of a row: 16 bytes of the result, so that a wave
// writes whole lines, past the caches.  Memory bound: 262144 x 512 bf16, 268 MB
// written and 59 MB of rows that occur read, 61 us (5.4 TB/s; through the caches
// 99); 28629 x 512 from fp32 to bf16 11.5 us.  112 x 64: 2.5 us, a launch.  A
// result that the caches could hold costs the next kernel what this one saves:
// 4000 x 512 and a product with it 13.7 us, written through the caches 11.9.
template <class T, class O, int K>
__global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
    const int pieces = (a.dim + K - 1) / K;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / pieces;
    if (row >= a.n) return;
    const Piece<K> piece((int)(at - row * pieces) * K, a.dim);
    const int id = a.ids[row];
    float v[K];
    if (id < 0 || id >= a.vocab) {
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] = 0.f;
    } else {
        load_k<T, K>(static_cast<const T*>(a.table) + id * a.table_stride + piece.col, v);
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] *= a.scale;
    }
    O* to = static_cast<O*>(a.out) + row * a.out_stride + piece.col;
    if constexpr (K == Elem<O>::kVec) {
        if (piece.skip == 0) return Elem<O>::store_nt(to, Elem<O>::pack(v));
    }
    store_from<O, K>(to, v, piece.skip);
}

// ---- the gradient: positions sorted by word, then sums over the runs of a word
//
// The sort is a stable radix sort of (word, position), so a word's rows come in
// ascending position.  They are added in that order inside a chunk, and the parts
// of a run over several chunks by groups of lanes, then waves: an order that the
// places fix, so that the result does not depend on timing.  Ids
// that are no token get the word V and sort to the end.  It takes a pass for
// every digit of up to kMaxDigit bits, of counts per tile, their prefix sums and
// the scatter.  These launches leave the memory idle, so further work-groups of
// theirs write the zero rows: of all words, because those that occur are not
// known yet; the sums come over them later (rows of 512 bf16 into 65536 rows of
// fp32, with the zeros of the other words beside the sums in brackets: 5000 ids
// 42 us [51], 20000 51 [58], 262144 120 [119]).

constexpr int kMaxDigit = 10;
constexpr int kRounds = 4, kFewRounds = 2;  // a work-group of the sort ranks the ids of 4 waves of so many rounds
constexpr int kFewIds = 32768;     // ids up to which it takes fewer (20000: 2 us less, 33000: 2 us more)
constexpr int kSumTiles = 64;      // tiles up to which the scatter adds up the counts itself

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

struct alignas(8) Pair {
    uint32_t word, pos;
};

// A launch's share of the zero rows: the work-groups from `from` on write them.
struct Fill {
    char* table;
    int64_t row, stride;    // bytes
    uint32_t first, rows;
    int32_t from, per;      // per: rows of a work-group
};

constexpr int kFillBytes = 65536;  // a work-group's, about

__device__ __forceinline__ void fill_rows(const Fill& f, int group) {
    const uint32_t first = group * (uint32_t)f.per, rows = min((uint32_t)f.per, f.rows - first);
    char* base = f.table + (int64_t)(f.first + first) * f.stride;
    if (f.row == f.stride) {  // one piece of memory: 16 bytes a store where it is aligned, 2 before and after
        char* end = base + rows * f.row;
        char* body = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(base) + 15) & ~(uintptr_t)15);
        char* stop = reinterpret_cast<char*>(reinterpret_cast<uintptr_t>(end) & ~(uintptr_t)15);
        for (char* p = body + threadIdx.x * 16; p < stop; p += 256 * 16)
            __builtin_nontemporal_store(u32x4{0u, 0u, 0u, 0u}, reinterpret_cast<u32x4*>(p));
        const int at = threadIdx.x * 2;
        if (base + at < min(body, end)) *reinterpret_cast<uint16_t*>(base + at) = 0;
        if (stop >= body && stop + at < end) *reinterpret_cast<uint16_t*>(stop + at) = 0;
        return;
    }
    const uint32_t pieces = (uint32_t)((f.row + 15) / 16), items = rows * pieces;
    for (uint32_t i = threadIdx.x; i < items; i += 256) {
        const uint32_t r = i / pieces, c = (i - r * pieces) * 16;
        char* d = base + r * f.stride + c;
        if (c + 16 <= f.row) Elem<bf16>::store_nt(reinterpret_cast<bf16*>(d), u32x4{0u, 0u, 0u, 0u});
        else
            for (uint32_t k = 0; c + k < f.row; k += 2) *reinterpret_cast<uint16_t*>(d + k) = 0;
    }
}

struct SortArgs {
    const int32_t* ids;  // pass 0 reads the ids
    const Pair* in;      // later passes read these
    Pair* out;
    uint32_t* counts;    // [tile][bin]; their prefix sums over the tiles after sort_scan
    uint32_t* totals;    // [bin]
    int32_t n, tiles, shift, bits;
    uint32_t vocab;
    Fill fill;
};

__device__ __forceinline__ Pair sort_pair(const SortArgs& a, int64_t i) {
    return a.ids ? Pair{word_of(a.ids[i], a.vocab), (uint32_t)i} : a.in[i];
}

// counts[tile][bin] of one digit.
template <int ROUNDS>
__global__ __launch_bounds__(256) void sort_count(SortArgs a) {
    constexpr int kTile = 256 * ROUNDS;
    __shared__ uint32_t count[1 << kMaxDigit];
    if ((int)blockIdx.x >= a.fill.from) return fill_rows(a.fill, blockIdx.x - a.fill.from);
    const int bins = 1 << a.bits, tile = blockIdx.x;
    for (int b = threadIdx.x; b < bins; b += 256) count[b] = 0;
    uint32_t k[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t i = (int64_t)tile * kTile + r * 256 + threadIdx.x;
        k[r] = i < a.n ? sort_pair(a, i).word : 0;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
        if ((int64_t)tile * kTile + r * 256 + threadIdx.x < a.n) atomicAdd(&count[(k[r] >> a.shift) & (bins - 1)], 1u);
    __syncthreads();
    for (int b = threadIdx.x; b < bins; b += 256) a.counts[(int64_t)tile * bins + b] = count[b];
}

// Prefix sums of every bin's counts over the tiles: a work-group takes 16 bins,
// each of its 16 x 16 threads a bin's counts of a sixteenth of the tiles.
constexpr int kScanBins = 16;
__global__ __launch_bounds__(256) void sort_scan(SortArgs a) {
    const int bins = 1 << a.bits;
    __shared__ uint32_t part[16][kScanBins];
    if ((int)blockIdx.x >= a.fill.from) return fill_rows(a.fill, blockIdx.x - a.fill.from);
    const int mine = threadIdx.x >> 4, bin = blockIdx.x * kScanBins + (threadIdx.x & 15);
    const int per = (a.tiles + 15) / 16, t0 = min(a.tiles, mine * per), t1 = min(a.tiles, t0 + per);
    uint32_t* c = a.counts + bin;
    uint32_t sum = 0;
    if (bin < bins) {
#pragma unroll 8
        for (int t = t0; t < t1; ++t) sum += c[(int64_t)t * bins];
    }
    part[mine][threadIdx.x & 15] = sum;
    __syncthreads();
    uint32_t base = 0;
    for (int i = 0; i < mine; ++i) base += part[i][threadIdx.x & 15];
    if (bin >= bins) return;
#pragma unroll 8
    for (int t = t0; t < t1; ++t) {
        const uint32_t v = c[(int64_t)t * bins];
        c[(int64_t)t * bins] = base;
        base += v;
    }
    if (mine == 15) a.totals[bin] = base;
}

// Ranks a tile's ids and writes them to their places.  SUM: the counts are
// still those of single tiles, and every work-group adds them up for itself,
// which for few tiles takes less than another launch (the gradient of 9000 ids
// x 300 into 65536 words: 44 us, with a launch for the sums 48; 60000 ids: 70 both).
template <bool SUM, int ROUNDS>
__global__ __launch_bounds__(256) void sort_scatter(SortArgs a) {
    constexpr int kTile = 256 * ROUNDS;
    constexpr int kBins = 1 << kMaxDigit;
    __shared__ uint32_t at[4][kBins];  // per wave: counts, then the next place of a digit
    __shared__ uint32_t wave_sum[4];
    if ((int)blockIdx.x >= a.fill.from) return fill_rows(a.fill, blockIdx.x - a.fill.from);
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6, tile = blockIdx.x, bins = 1 << a.bits;
    // each thread owns four neighbouring bins
    constexpr int kOwn = kBins / 256;
    uint32_t total[kOwn], prior[kOwn], sum = 0;
    if constexpr (SUM) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) total[i] = prior[i] = 0;
        if (tid * kOwn < bins) {
#pragma unroll 8
            for (int t = 0; t < a.tiles; ++t) {
                const u32x4 c = *reinterpret_cast<const u32x4*>(a.counts + (int64_t)t * bins + tid * kOwn);
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    total[i] += c[i];
                    prior[i] += t < tile ? c[i] : 0;
                }
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            const int b = tid * kOwn + i;
            total[i] = b < bins ? a.totals[b] : 0;
            prior[i] = b < bins ? a.counts[(int64_t)tile * bins + b] : 0;
        }
    }
    const int64_t first = (int64_t)tile * kTile + wave * (kTile / 4);
    Pair k[ROUNDS];
    uint32_t rank[ROUNDS];
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int64_t i = first + r * 64 + lane;
        k[r] = i < a.n ? sort_pair(a, i) : Pair{0, 0};
    }
    for (int b = lane; b < bins; b += 64) at[wave][b] = 0;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) sum += total[i];
    const uint32_t upto = wave_scan_inclusive(sum);
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const bool valid = first + r * 64 + lane < a.n;
        const uint32_t d = (k[r].word >> a.shift) & (bins - 1);
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
    for (int i = 0; i < kOwn; ++i) {
        const int b = tid * kOwn + i;
        if (b < bins) {
            uint32_t next = base + prior[i];
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
    for (int r = 0; r < ROUNDS; ++r)
        if (first + r * 64 + lane < a.n) a.out[at[wave][(k[r].word >> a.shift) & (bins - 1)] + rank[r]] = k[r];
}

struct SumArgs {
    const Pair* sorted;  // readable to a multiple of 8
    int32_t n, chunk;    // chunk: a multiple of 8
    uint32_t vocab;
    int32_t dim, lanes;  // lanes: a power of two up to 64 that share a row
    const void* dout;
    int64_t dout_stride;
    float scale;
    int32_t accumulate;
    void* dtable;
    int64_t dtable_stride;
    float* partial;      // [chunks][2][dim]
};

constexpr int kFillRows = 256;

// Zeroes the rows first .. first + rows of the table's gradient but those marked in `there`.
template <class O>
__device__ __forceinline__ void zero_rows(void* dtable, int64_t stride, int32_t dim, uint32_t first, uint32_t rows,
                                          const uint8_t* there, uint32_t threads) {
    constexpr int kPer = 16 / (int)sizeof(O);
    const uint32_t pieces = (dim + kPer - 1) / kPer, items = rows * pieces;
    O* base = static_cast<O*>(dtable) + first * stride;
    for (uint32_t i = threadIdx.x; i < items; i += threads) {
        const uint32_t r = i / pieces, c = (i - r * pieces) * kPer;
        if (there[r]) continue;
        O* d = base + r * stride + c;
        if ((int)c + kPer <= dim) Elem<O>::store_nt(d, u32x4{0u, 0u, 0u, 0u});
        else
            for (int k = c; k < dim; ++k) Elem<O>::put(d + (k - c), 0.f);
    }
}

// The sums over the groups of `lanes` lanes of a wave, in every group.
template <int K>
__device__ __forceinline__ void add_groups(float* sum, int lanes) {
    for (int d = lanes; d < 64; d <<= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) sum[k] += __shfl_xor(sum[k], d);
}

template <class O, int K, class A>
__device__ __forceinline__ void put_word(const A& a, uint32_t word, Piece<K> piece, const float* sum) {
    O* d = static_cast<O*>(a.dtable) + word * a.dtable_stride + piece.col;
    float v[K];
    if (a.accumulate) {
        load_k<O, K>(d, v);
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = __builtin_fmaf(sum[k], a.scale, v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = sum[k] * a.scale;
    }
    store_from<O, K>(d, v, piece.skip);
}

// Eight neighbouring entries of the sorted lists.  WAVE: the same ones in every
// lane of the wave, kept in scalar registers.
template <bool WAVE>
struct Eight {
    uint32_t key[8], pos[8];

    __device__ __forceinline__ void load(const SumArgs& a, int i) {
        u32x4 v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = *reinterpret_cast<const u32x4*>(a.sorted + i + 2 * u);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            key[u] = v[u >> 1][2 * (u & 1)];
            pos[u] = v[u >> 1][2 * (u & 1) + 1];
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
// Memory bound: 262144 rows of 512 bf16 (268 MB) into those that occur of 131072
// in fp32: 78 us.
template <class T, class O, int K, bool WAVE>
__global__ __launch_bounds__(256) void sum_chunks(SumArgs a) {
    int chunk;
    if constexpr (WAVE) chunk = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    else chunk = (int)(((int64_t)blockIdx.x * 256 + threadIdx.x) / a.lanes);
    const int lanes = WAVE ? 64 : a.lanes;
    const int nominal = (blockIdx.y * lanes + (threadIdx.x & (lanes - 1))) * K;
    const int64_t begin64 = (int64_t)chunk * a.chunk;
    if (begin64 >= a.n || nominal >= a.dim) return;
    const Piece<K> piece(nominal, a.dim);
    const int begin = (int)begin64, end = (int)min((int64_t)a.n, begin64 + a.chunk);
    const T* rows = static_cast<const T*>(a.dout) + piece.col;
    float* partial = a.partial + 2 * (int64_t)chunk * a.dim + piece.col;
    Eight<WAVE> at;
    at.load(a, begin);
    const uint32_t before = begin > 0 ? a.sorted[begin - 1].word : a.vocab, after = end < a.n ? a.sorted[end].word : a.vocab;
    at.settle();
    uint32_t cur = at.key[0];
    if (cur >= a.vocab) return;  // only ids that are no token
    bool from_before = before == cur;
    const uint32_t some = at.pos[0];
    float sum[K] = {};
    for (int left = end - begin; left > 0; left -= 8) {  // counted down: a position and 8 can pass 2^31
        float v[8][K];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const uint32_t p = u < left ? at.pos[u] : some;
            load_k<T, K, true>(rows + p * a.dout_stride, v[u]);
        }
        const Eight<WAVE> now = at;
        if (left > 8) at.load(a, end - left + 8);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (u >= left) break;
            if (now.key[u] != cur) {
                if (from_before) store_from<float, K>(partial, sum, piece.skip);
                else put_word<O, K>(a, cur, piece, sum);
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
    if (from_before) store_from<float, K>(partial, sum, piece.skip);
    else if (after == cur) store_from<float, K>(partial + a.dim, sum, piece.skip);
    else put_word<O, K>(a, cur, piece, sum);
}

constexpr int kJoinWaves = 16;
constexpr int kJoinAlone = 32;  // partial rows that a wave adds up by itself
constexpr int kJoinLanes = 16;  // lanes to a row of a long run

// The sum of the partial rows i0 .. i1 of the run that begins in `chunk`: the
// chunk's second row, then the first rows of the chunks after it.
template <int K>
__device__ __forceinline__ void add_partial(const SumArgs& a, int64_t chunk, int64_t i0, int64_t i1, int col, float* sum) {
    for (int64_t i = i0; i < i1; i += 8) {
        float v[8][K];
#pragma unroll
        for (int u = 0; u < 8; ++u) {  // a place past the end reads the part's last row
            const int64_t j = min(i + u, i1 - 1);
            load_k<float, K>(a.partial + (2 * (chunk + j) + (j == 0 ? 1 : 0)) * a.dim + col, v[u]);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i + u < i1)
#pragma unroll
                for (int k = 0; k < K; ++k) sum[k] += v[u][k];
    }
}

// A wave a chunk: where a run begins in the chunk and goes on after it, its
// partial rows are added up, by the wave or, of a run over more than kJoinAlone
// chunks (at most one begins in a work-group's), by all waves together, each
// group of lanes a contiguous part.  A long run's columns are split over the
// work-groups along z, which a CU by itself would take too long for (262144 ids
// x 512 fp32, half of them one word: 210 us, 239 without the split); those but
// the first have nothing else to do.
template <class O, int K>
__global__ __launch_bounds__(64 * kJoinWaves) void join_chunks(SumArgs a) {
    static_assert(kJoinAlone >= kJoinWaves, "one long run a work-group");
    __shared__ float part[kJoinWaves][64][K];
    __shared__ int64_t long_chunk, long_rows;
    __shared__ uint32_t long_word;
    const int lane = lane_id(), wave = threadIdx.x >> 6;
    const int64_t chunk = (int64_t)blockIdx.x * kJoinWaves + wave, begin = chunk * a.chunk, end = begin + a.chunk;
    if (threadIdx.x == 0) long_rows = 0;
    int64_t rows = 0;
    uint32_t word = a.vocab;
    const int64_t far = blockIdx.z ? begin + (int64_t)kJoinAlone * a.chunk : end;
    if (far < a.n) {
        word = a.sorted[end - 1].word;
        const uint32_t after = a.sorted[far].word, head = a.sorted[begin].word,
                       before = begin > 0 ? a.sorted[begin - 1].word : a.vocab;
        if (word < a.vocab && after == word && !(head == word && before == word)) {
            // the chunks after this one that begin with the word: the first 64 looked at one by one, then 64
            // places of what is left at a time
            int64_t step = 1, limit = (a.n - end + a.chunk - 1) / a.chunk;
            while (rows < limit) {
                const int64_t at = rows + lane * step;
                const uint64_t m = __ballot(at < limit && a.sorted[end + min(at, limit - 1) * a.chunk].word == word);
                const int run = m == ~0ull ? 64 : __ffsll((unsigned long long)~m) - 1;
                if (run < 64) limit = min(limit, rows + run * step);
                if (run) rows += (run - 1) * step + 1;
                step = (limit - rows + 63) / 64;
            }
            ++rows;  // and its own second row
        }
    }
    __syncthreads();
    if (rows > kJoinAlone) {
        if (lane == 0) {
            long_chunk = chunk;
            long_rows = rows;
            long_word = word;
        }
    } else if (rows && blockIdx.z == 0) {
        const int groups = 64 / a.lanes, nominal = (blockIdx.y * a.lanes + (lane & (a.lanes - 1))) * K;
        const Piece<K> piece(nominal, a.dim);
        const int64_t per = (rows + groups - 1) / groups, i0 = min(rows, (lane / a.lanes) * per), i1 = min(rows, i0 + per);
        float sum[K] = {};
        if (nominal < a.dim) add_partial<K>(a, chunk, i0, i1, piece.col, sum);
        add_groups<K>(sum, a.lanes);
        if (lane < a.lanes && nominal < a.dim) put_word<O, K>(a, word, piece, sum);
    }
    __syncthreads();
    if (!long_rows) return;
    const int lanes = a.lanes / gridDim.z, groups = 64 / lanes;
    const int nominal = (blockIdx.y * a.lanes + blockIdx.z * lanes + (lane & (lanes - 1))) * K;
    const Piece<K> piece(nominal, a.dim);
    const int64_t n = long_rows, all = kJoinWaves * groups, per = (n + all - 1) / all;
    const int64_t i0 = min(n, (threadIdx.x / lanes) * per), i1 = min(n, i0 + per);
    float sum[K] = {};
    if (nominal < a.dim) add_partial<K>(a, long_chunk, i0, i1, piece.col, sum);
    add_groups<K>(sum, lanes);
#pragma unroll
    for (int k = 0; k < K; ++k) part[wave][lane][k] = sum[k];
    __syncthreads();
    if ((int)threadIdx.x >= lanes || nominal >= a.dim) return;
    for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
        for (int k = 0; k < K; ++k) sum[k] += part[w][lane][k];
    put_word<O, K>(a, long_word, piece, sum);
}

// ---- a few ids: one launch, without a sort
//
// A work-group an id looks through all ids.  The one at a word's first place
// adds up the word's rows (a contiguous part of them for each group of lanes),
// of a frequent word the ones at its first up to eight places a part of the
// columns each; the others end.  The first work-groups zero the rows of the
// other words, which is what most of the time goes to where the table is large.
// 1627 ids x 100 fp32 into 20011 words: 7 us, by sorting 24; 4000 x 512 into
// 65536: 34 and 43, also where one word has half of the ids (90 without the parts).
constexpr int kSmall = 4096;
constexpr int kSmallOften = 64;   // rows from which on a word's columns are split
constexpr int kSmallThreads = 256, kSmallWaves = kSmallThreads / 64;
constexpr int kMostFill = 1 << 22;  // work-groups that zero rows: a launch has less than 2^32 threads

struct SmallArgs {
    const int32_t* ids;
    int32_t n;
    uint32_t vocab;
    int32_t dim, lanes, tiles;
    const void* dout;
    int64_t dout_stride;
    float scale;
    int32_t accumulate;
    void* dtable;
    int64_t dtable_stride;
    // the first work-groups zero the rows of words that do not occur, so many at a time each
    int32_t fill_rows, fill_groups;
};

// kLook: ids that a thread looks at.
template <class T, class O, int K, int kLook>
__global__ __launch_bounds__(kSmallThreads) void sum_small(SmallArgs a) {
    __shared__ uint8_t there[kFillRows];
    __shared__ uint16_t list[kLook * kSmallThreads];
    __shared__ int count[kSmallWaves], early[kSmallWaves];
    __shared__ float part[kSmallWaves][64][K];
    const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
    int32_t id[kLook];
    if ((int)blockIdx.x < a.fill_groups) {
#pragma unroll
        for (int r = 0; r < kLook; ++r) id[r] = r * kSmallThreads + tid < a.n ? a.ids[r * kSmallThreads + tid] : -1;
        uint32_t first = blockIdx.x * (uint32_t)a.fill_rows;
        while (true) {  // once, but for the largest tables
            const uint32_t rows = min((uint32_t)a.fill_rows, a.vocab - first);
            if (tid < kFillRows) there[tid] = 0;
            __syncthreads();
#pragma unroll
            for (int r = 0; r < kLook; ++r)
                if (id[r] >= 0 && (uint32_t)id[r] - first < rows) there[(uint32_t)id[r] - first] = 1;
            __syncthreads();
            zero_rows<O>(a.dtable, a.dtable_stride, a.dim, first, rows, there, kSmallThreads);
            first += (uint32_t)a.fill_groups * (uint32_t)a.fill_rows;
            if (first >= a.vocab) return;
            __syncthreads();
        }
    }
    const int me = blockIdx.x - a.fill_groups, span = (a.n + kSmallThreads - 1) / kSmallThreads * 64, first = wave * span;
    const uint32_t word = word_of(a.ids[me], a.vocab);
#pragma unroll
    for (int r = 0; r < kLook; ++r) {
        const int i = first + r * 64 + lane;
        id[r] = r * 64 < span && i < a.n ? a.ids[i] : -1;
    }
    if (word >= a.vocab) return;
    uint64_t same[kLook];
    int mine = 0;
    bool before = false;
#pragma unroll
    for (int r = 0; r < kLook; ++r) {
        same[r] = __ballot((uint32_t)id[r] == word);
        mine += __popcll(same[r]);
        before |= same[r] && first + r * 64 + __ffsll((unsigned long long)same[r]) - 1 < me;
    }
    if (lane == 0) {
        count[wave] = mine;
        early[wave] = before;
    }
    __syncthreads();
    int at = 0, n = 0, turn = 0;
    for (int w = 0; w < kSmallWaves; ++w) {
        turn |= early[w];
        if (w < wave) at += count[w];
        n += count[w];
    }
    const int parts = n >= kSmallOften ? max(1, min(8, a.lanes / 4)) : 1, lanes = a.lanes / parts;
    if (turn) {  // not the first: which place of the word's is it
        if (parts == 1) return;
        __syncthreads();
        int places = 0;
#pragma unroll
        for (int r = 0; r < kLook; ++r) {
            const int to_me = me - (first + r * 64);
            places += __popcll(to_me >= 64 ? same[r] : to_me > 0 ? same[r] & ((1ull << to_me) - 1) : 0ull);
        }
        if (lane == 0) early[wave] = places;
        __syncthreads();
        turn = 0;
        for (int w = 0; w < kSmallWaves; ++w) turn += early[w];
        if (turn >= parts) return;
    }
#pragma unroll
    for (int r = 0; r < kLook; ++r) {
        if ((same[r] >> lane) & 1) list[at + __popcll(same[r] & ((1ull << lane) - 1))] = (uint16_t)(first + r * 64 + lane);
        at += __popcll(same[r]);
    }
    __syncthreads();
    const int per = (n * lanes + kSmallThreads - 1) / kSmallThreads;  // rows a group of lanes
    const int i0 = min(n, (tid / lanes) * per), i1 = min(n, i0 + per);
    const int used = (n * lanes + 64 * per - 1) / (64 * per);         // waves with rows
    for (int t = 0; t < a.tiles; ++t) {
        const int nominal = (t * a.lanes + turn * lanes + (tid & (lanes - 1))) * K;
        const Piece<K> piece(nominal, a.dim);
        float sum[K] = {};
        if (nominal < a.dim) {
            const T* rows = static_cast<const T*>(a.dout) + piece.col;
            for (int i = i0; i < i1; i += 8) {
                float v[8][K];
#pragma unroll
                for (int u = 0; u < 8; ++u)  // a place past the end reads its part's last row
                    load_k<T, K>(rows + list[min(i + u, i1 - 1)] * a.dout_stride, v[u]);
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    if (i + u < i1)
#pragma unroll
                        for (int k = 0; k < K; ++k) sum[k] += v[u][k];
            }
        }
        add_groups<K>(sum, lanes);
        if (used > 1) {
            if (t) __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) part[wave][lane][k] = sum[k];
            __syncthreads();
            if (wave == 0)
                for (int w = 1; w < used; ++w)
#pragma unroll
                    for (int k = 0; k < K; ++k) sum[k] += part[w][lane][k];
        }
        if (tid < lanes && nominal < a.dim) put_word<O, K>(a, word, piece, sum);
    }
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

Region matrix(const void* p, int32_t dtype, int32_t rows, int32_t dim, int64_t stride) {
    return {rows ? p : nullptr, rows, dim * elem_bytes(dtype), stride * elem_bytes(dtype)};
}

edb_status launched(const char* who) {
    const hipError_t he = hipGetLastError();
    if (he != hipSuccess) return fail(EDB_ERR_HIP, std::string(who) + ": " + hipGetErrorString(he));
    edb::clear_error();
    return EDB_OK;
}

// Elements that a lane of the gradient's kernels takes of a row.  Short rows by
// four, since a row's lanes are a power of two and more of them are used
// (262144 ids of 64 fp32: 50 us, by eight 63; 150: 75 and 85); from 256 on by
// eight, which asks for more bytes at a time (300 bf16: 98 us, by four 115).
int piece_of(int dim) { return dim >= 256 ? 8 : dim >= 4 ? 4 : 1; }

template <class T, class O>
void launch_embed(const EmbedArgs& a, hipStream_t st) {
    // 16 bytes of the result a lane, so that a wave writes whole lines
    constexpr int kWhole = Elem<O>::kVec;
    const int k = a.dim >= kWhole ? kWhole : a.dim >= 4 ? 4 : 1;
    // a launch has less than 2^32 threads: more are taken in slices of rows
    const int64_t pieces = (a.dim + k - 1) / k, most = (INT64_C(1) << 31) / pieces;
    for (int64_t i = 0; i < a.n; i += most) {
        EmbedArgs b = a;
        b.ids = a.ids + i;
        b.n = (int32_t)(a.n - i < most ? a.n - i : most);
        b.out = static_cast<O*>(a.out) + i * a.out_stride;
        const dim3 grid((unsigned)((b.n * pieces + 255) / 256));
        if (k == kWhole) embed_kernel<T, O, kWhole><<<grid, 256, 0, st>>>(b);
        else if (k == 4) embed_kernel<T, O, 4><<<grid, 256, 0, st>>>(b);
        else embed_kernel<T, O, 1><<<grid, 256, 0, st>>>(b);
    }
}

// How the gradient's work is laid out, and its scratch memory.
struct GradPlan {
    int32_t piece, lanes, tiles_y, chunk, chunks;
    int32_t passes, digit, sort_tiles;
    int64_t sorted[2], counts, totals, partial, bytes;  // offsets
};

GradPlan grad_plan(int32_t n, int32_t vocab, int32_t dim) {
    GradPlan g{};
    g.piece = piece_of(dim);
    const int pieces = (dim + g.piece - 1) / g.piece;
    g.lanes = 1;
    while (g.lanes < 64 && g.lanes < pieces) g.lanes *= 2;
    g.tiles_y = (pieces + g.lanes - 1) / g.lanes;
    // two waves a SIMD, more where chunks would pass 64 rows: short chunks cost partial rows
    int64_t chunk = (int64_t)n * g.lanes * g.tiles_y / (64 * 2048) / 8 * 8;
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
    const int64_t list = ((int64_t)n + 7) / 8 * 8 * (int64_t)sizeof(Pair);
    g.passes = (bits + kMaxDigit - 1) / kMaxDigit;
    g.digit = (bits + g.passes - 1) / g.passes;
    if (g.digit < 2) g.digit = 2;            // the scatter reads the counts by fours
    const int tile = 256 * (n <= kFewIds ? kFewRounds : kRounds);
    g.sort_tiles = (int32_t)(((int64_t)n + tile - 1) / tile);
    g.sorted[0] = take(list);
    g.sorted[1] = take(list);
    g.counts = take((int64_t)g.sort_tiles * 4 << g.digit);
    g.totals = take(INT64_C(4) << g.digit);
    g.partial = take((int64_t)g.chunks * 2 * dim * 4);
    g.bytes = n > kSmall ? at : 0;
    return g;
}

template <class T, class O, int K>
void launch_small(const SmallArgs& a, hipStream_t st) {
    const unsigned groups = a.n + a.fill_groups;
    if (groups == 0) return;
    // no more looks than the ids need (1627 ids x 100 into 20011 words: 7.4 us with 8, 9.1 with 16)
    if (a.n <= 4 * kSmallThreads) sum_small<T, O, K, 4><<<groups, kSmallThreads, 0, st>>>(a);
    else if (a.n <= 8 * kSmallThreads) sum_small<T, O, K, 8><<<groups, kSmallThreads, 0, st>>>(a);
    else sum_small<T, O, K, kSmall / kSmallThreads><<<groups, kSmallThreads, 0, st>>>(a);
}

template <class T, class O>
void launch_small(int piece, const SmallArgs& a, hipStream_t st) {
    if (piece == 8) launch_small<T, O, 8>(a, st);
    else if (piece == 4) launch_small<T, O, 4>(a, st);
    else launch_small<T, O, 1>(a, st);
}

template <class T, class O, int K>
void launch_sums(const GradPlan& g, const SumArgs& a, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)g.chunks * g.lanes + 255) / 256), g.tiles_y);
    if (g.lanes == 64) sum_chunks<T, O, K, true><<<grid, 256, 0, st>>>(a);
    else sum_chunks<T, O, K, false><<<grid, 256, 0, st>>>(a);
    if (g.chunks > 1) {
        const int parts = g.chunks > kJoinAlone && a.lanes > kJoinLanes ? a.lanes / kJoinLanes : 1;
        join_chunks<O, K><<<dim3((g.chunks + kJoinWaves - 1) / kJoinWaves, g.tiles_y, parts), 64 * kJoinWaves, 0, st>>>(a);
    }
}

template <class T, class O>
void launch_sums(const GradPlan& g, const SumArgs& a, hipStream_t st) {
    if (g.piece == 8) launch_sums<T, O, 8>(g, a, st);
    else if (g.piece == 4) launch_sums<T, O, 4>(g, a, st);
    else launch_sums<T, O, 1>(g, a, st);
}

}  // namespace

extern "C" edb_status edb_embed(const int32_t* ids, int32_t n, const void* table, int32_t table_dtype, int32_t vocab,
                                int32_t dim, int64_t table_stride, float scale, void* out, int32_t out_dtype,
                                int64_t out_stride, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_embed";
        if (edb_status st = check_table(who, n, vocab, dim, out_dtype, table_dtype, out_stride, table_stride, scale)) return st;
        if (n == 0) {
            edb::clear_error();
            return EDB_OK;
        }
        if (!ids || !table || !out) return fail(EDB_ERR_INVALID, "edb_embed: NULL argument");
        if (!element_aligned(table, table_dtype) || !element_aligned(out, out_dtype))
            return fail(EDB_ERR_INVALID, "edb_embed: the table and the result must be aligned to their elements");
        if (!edb::word_aligned({ids})) return fail(EDB_ERR_INVALID, "edb_embed: the ids must be aligned to 4 bytes");
        const Region result = matrix(out, out_dtype, n, dim, out_stride);
        if (edb::overlap(Region::array(ids, n * INT64_C(4)), result))
            return fail(EDB_ERR_INVALID, "edb_embed: the result overlaps the ids");
        if (edb::overlap(matrix(table, table_dtype, vocab, dim, table_stride), result))
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
    });
}

extern "C" edb_status edb_embed_grad_bytes(int32_t n, int32_t vocab, int32_t dim, int64_t* bytes) {
    return edb::guarded([&]() -> edb_status {
        if (!bytes) return fail(EDB_ERR_INVALID, "edb_embed_grad_bytes: NULL argument");
        if (edb_status st = check_table("edb_embed_grad_bytes", n, vocab, dim, EDB_F32, EDB_F32, dim, dim, 1.f)) return st;
        *bytes = grad_plan(n, vocab, dim).bytes;
        edb::clear_error();
        return EDB_OK;
    });
}

extern "C" edb_status edb_embed_grad(const int32_t* ids, int32_t n, const void* dout, int32_t dout_dtype, int32_t vocab,
                                     int32_t dim, int64_t dout_stride, float scale, int32_t accumulate, void* dtable,
                                     int32_t dtable_dtype, int64_t dtable_stride, void* workspace,
                                     int64_t workspace_bytes, void* stream) {
    return edb::guarded([&]() -> edb_status {
        const char* who = "edb_embed_grad";
        if (edb_status st = check_table(who, n, vocab, dim, dout_dtype, dtable_dtype, dout_stride, dtable_stride, scale)) return st;
        if (!dtable || (n && (!ids || !dout))) return fail(EDB_ERR_INVALID, "edb_embed_grad: NULL argument");
        if (!element_aligned(dout, dout_dtype) || !element_aligned(dtable, dtable_dtype))
            return fail(EDB_ERR_INVALID, "edb_embed_grad: both gradients must be aligned to their elements");
        const Region id_array = Region::array(ids, n * INT64_C(4)), rows = matrix(dtable, dtable_dtype, vocab, dim, dtable_stride),
                     drows = matrix(dout, dout_dtype, n, dim, dout_stride);
        if (edb::overlap(drows, rows))
            return fail(EDB_ERR_INVALID, "edb_embed_grad: the table's gradient overlaps the rows' gradients");
        if (!edb::word_aligned({ids})) return fail(EDB_ERR_INVALID, "edb_embed_grad: the ids must be aligned to 4 bytes");
        const GradPlan g = grad_plan(n, vocab, dim);
        if (workspace_bytes < g.bytes || (g.bytes && !workspace) || (reinterpret_cast<uintptr_t>(workspace) & 15u))
            return fail(EDB_ERR_INVALID, "edb_embed_grad: a 16-byte aligned workspace of " + std::to_string(g.bytes) +
                                             " bytes is needed");
        if (edb_status st = edb::apart(who, {Region::array(workspace, g.bytes)}, {id_array, rows, drows})) return st;
        if (edb::overlap(id_array, rows)) return fail(EDB_ERR_INVALID, "edb_embed_grad: the table's gradient overlaps the ids");
        hipStream_t st = reinterpret_cast<hipStream_t>(stream);
        const int64_t row_bytes = rows.row;
        if (n <= kSmall) {
            const int64_t fit = 16384 / row_bytes;  // rows that a work-group zeroes
            const int fill_rows = (int)(fit < 1 ? 1 : fit > kFillRows ? kFillRows : fit);
            const int64_t fills = ((int64_t)vocab + fill_rows - 1) / fill_rows;
            const int fill_groups = accumulate ? 0 : (int)(fills < kMostFill ? fills : kMostFill);
            const SmallArgs a{ids,   n,          (uint32_t)vocab, dim,           g.lanes,   g.tiles_y,  dout, dout_stride,
                              scale, accumulate, dtable,          dtable_stride, fill_rows, fill_groups};
            if (dout_dtype == EDB_F32) {
                if (dtable_dtype == EDB_F32) launch_small<float, float>(g.piece, a, st);
                else launch_small<float, bf16>(g.piece, a, st);
            } else {
                if (dtable_dtype == EDB_F32) launch_small<bf16, float>(g.piece, a, st);
                else launch_small<bf16, bf16>(g.piece, a, st);
            }
            return launched(who);
        }
        char* ws = static_cast<char*>(workspace);
        auto sorted = [&](int i) { return reinterpret_cast<Pair*>(ws + g.sorted[i]); };
        SortArgs s{};
        s.n = n;
        s.vocab = (uint32_t)vocab;
        int last = 0;
        s.tiles = g.sort_tiles;
        s.counts = reinterpret_cast<uint32_t*>(ws + g.counts);
        s.totals = reinterpret_cast<uint32_t*>(ws + g.totals);
        s.bits = g.digit;
        const bool scan = g.sort_tiles > kSumTiles;
        const int launches = g.passes * (scan ? 3 : 2);
        int launch = 0;
        // the work-groups of the next launch, its share of the zero rows behind `groups` of its own
        auto next = [&](int groups) {
            const int64_t first = (int64_t)vocab * launch / launches, end = (int64_t)vocab * (launch + 1) / launches;
            const int64_t per = row_bytes < kFillBytes ? kFillBytes / row_bytes : 1;
            ++launch;
            s.fill = Fill{static_cast<char*>(dtable), row_bytes, dtable_stride * elem_bytes(dtable_dtype), (uint32_t)first,
                          (uint32_t)(end - first), groups, (int32_t)per};
            return (unsigned)(groups + (accumulate ? 0 : (end - first + per - 1) / per));
        };
        for (int p = 0; p < g.passes; ++p) {
            s.ids = p ? nullptr : ids;
            s.in = sorted((p + 1) & 1);
            s.out = sorted(p & 1);
            s.shift = p * g.digit;
            last = p & 1;
            const unsigned count = next(g.sort_tiles);
            if (n <= kFewIds) sort_count<kFewRounds><<<count, 256, 0, st>>>(s);
            else sort_count<kRounds><<<count, 256, 0, st>>>(s);
            if (scan) {
                const unsigned sums = next(((1 << g.digit) + kScanBins - 1) / kScanBins);
                sort_scan<<<sums, 256, 0, st>>>(s);
            }
            const unsigned scatter = next(g.sort_tiles);
            if (scan) sort_scatter<false, kRounds><<<scatter, 256, 0, st>>>(s);
            else if (n <= kFewIds) sort_scatter<true, kFewRounds><<<scatter, 256, 0, st>>>(s);
            else sort_scatter<true, kRounds><<<scatter, 256, 0, st>>>(s);
        }
        const SumArgs a{sorted(last), n, g.chunk, (uint32_t)vocab, dim, g.lanes, dout, dout_stride, scale,
                        accumulate, dtable, dtable_stride, reinterpret_cast<float*>(ws + g.partial)};
        if (dout_dtype == EDB_F32) {
            if (dtable_dtype == EDB_F32) launch_sums<float, float>(g, a, st);
            else launch_sums<float, bf16>(g, a, st);
        } else {
            if (dtable_dtype == EDB_F32) launch_sums<bf16, float>(g, a, st);
            else launch_sums<bf16, bf16>(g, a, st);
        }
        return launched(who);
    });
}
