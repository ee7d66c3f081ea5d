// Embedding lookup and its gradient.
//
// Lookup: out[t, :] = scale * table[ids[t], :].  Bound by memory: a row read
// and a row written a token.  A wavefront moves 64 16-byte vectors of a row:
// short rows and few tokens still give the card enough of them.  16384 rows of
// 4096 bf16: 47 us, 5.7 TB/s; 8 rows: the launch.
//
// Gradient: dtable[v, :] = scale * sum of dout[t, :] over ids[t] = v.  The
// tokens are sorted by id, stably, so that the tokens of one row are adjacent
// and in increasing order; each row's sum is then one fold, with no atomics on
// it and one association: runs of kRun tokens, then the runs' sums in order.
// Three launches: the sort and the list of runs by one block, in LDS, while
// the others fill the table with zeros (most of its rows have no token, so
// that is most of the bytes); the runs; the rows of more than one run.
// 16384 tokens over a table of 131072 x 4096 bf16, frequencies falling as
// 1 / rank: 259 us, 4.7 TB/s of the bytes that have to pass; the sort and the
// zeros 177 (6.1 TB/s), the runs 76, which also wait for the zeros on their way
// from the caches to memory, the long rows 7 (medians of a trace).  5003 tokens,
// 32003 x 1001 fp32: 55 us; the sort, in two passes and longer than the zeros, 33,
// the runs 19, the long rows 5.
#include <algorithm>
#include <type_traits>

#include "replica.hpp"

namespace arp {
namespace {

constexpr int kRun = AR_EMBED_RUN;

// ------------------------------------------------------------- lookup

// The wavefront's number within its block, as a scalar.
__device__ __forceinline__ uint32_t wave_id() {
    return uint32_t(__builtin_amdgcn_readfirstlane(int(threadIdx.x >> 6)));
}

template <class T>
__global__ __launch_bounds__(256) void lookup_kernel(const T* table, int64_t table_stride,
                                                     const int64_t* ids, int64_t V, int64_t D,
                                                     int64_t rows, float scale, T* out,
                                                     int64_t out_stride) {
    constexpr int VEC = Num<T>::VEC;
    const uint32_t slices = uint32_t((D + 64 * VEC - 1) / (64 * VEC));  // of a row, one a wavefront
    const uint32_t units = uint32_t(rows) * slices, step = gridDim.x * 4;
    for (uint32_t u = blockIdx.x * 4 + wave_id(); u < units; u += step) {
        const int64_t t = u / slices;
        const int64_t at = int64_t(u % slices) * 64 * VEC + int64_t(threadIdx.x & 63) * VEC;
        const int64_t id = ids[t];
        const bool is = id >= 0 && id < V;
        const T* src = table + (is ? id : 0) * table_stride + at;
        T* dst = out + t * out_stride + at;
        if (D - at >= VEC) {
            float f[VEC] = {};
            if (is) Num<T>::unpack(load_vec(src), f);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] *= scale;
            store_vec(dst, is ? Num<T>::pack(f) : u32x4{0, 0, 0, 0});
        } else if (D > at) {
            for (int i = 0; i < int(D - at); ++i)
                dst[i] = is ? Num<T>::down(Num<T>::up(src[i]) * scale) : T(0);
        }
        if (units - u <= step) break;  // (u + step may pass 32 bits)
    }
}

// --------------------------------------------------------------- sort
//
// More than kSmallSort tokens (fewer: below).  Stable counting sort of the
// tokens by id, 8 bits a pass, lowest first.  A
// block takes kSortBlock tokens, each of its wavefronts a contiguous quarter
// in rounds of 64.  Three launches a pass: the blocks' digit counts, their
// exclusive sums in (digit, block) order, and the move.

constexpr int kDigits = 256;
constexpr int kSortBlock = 4096;
constexpr int kSortWaves = 4;
constexpr int kSortRounds = kSortBlock / (64 * kSortWaves);

struct SortSrc {  // a pass's input: the ids at first, then keys and tokens
    const int64_t* ids;
    const uint32_t* key;
    const uint32_t* tok;
    int64_t V, T;
};

__device__ __forceinline__ uint32_t sort_key(const SortSrc& s, int64_t i) {
    if (!s.ids) return s.key[i];
    const int64_t id = s.ids[i];
    return id >= 0 && id < s.V ? uint32_t(id) : uint32_t(s.V);  // no token: behind all rows
}

__global__ __launch_bounds__(256) void sort_count_kernel(SortSrc s, int shift, uint32_t* hist,
                                                         int64_t blocks) {
    __shared__ uint32_t n[kDigits];
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        n[threadIdx.x] = 0;
        __syncthreads();
        for (int r = 0; r < kSortBlock / 256; ++r) {
            const int64_t i = b * kSortBlock + r * 256 + threadIdx.x;
            if (i < s.T) atomicAdd(&n[(sort_key(s, i) >> shift) & (kDigits - 1)], 1u);
        }
        __syncthreads();
        hist[int64_t(threadIdx.x) * blocks + b] = n[threadIdx.x];
        __syncthreads();
    }
}

// Exclusive sums of n counts in place, by one block.
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t* hist, int64_t n,
                                                         uint32_t* count) {
    __shared__ uint32_t wave[16];
    if (threadIdx.x < 2) count[threadIdx.x] = 0;  // the lists that follow start empty
    uint32_t carry = 0;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int64_t base = 0; base < n; base += 1024) {
        const int64_t i = base + threadIdx.x;
        const uint32_t own = i < n ? hist[i] : 0;
        uint32_t sum = own;
        for (int d = 1; d < 64; d *= 2) {
            const uint32_t o = __shfl_up(sum, d);
            if (lane >= d) sum += o;
        }
        if (lane == 63) wave[w] = sum;
        __syncthreads();
        uint32_t before = carry, all = 0;
        for (int j = 0; j < 16; ++j) {
            if (j < w) before += wave[j];
            all += wave[j];
        }
        if (i < n) hist[i] = before + sum - own;
        carry += all;
        __syncthreads();
    }
}

__global__ __launch_bounds__(256) void sort_move_kernel(SortSrc s, int shift,
                                                        const uint32_t* offset, int64_t blocks,
                                                        uint32_t* key, uint32_t* tok) {
    __shared__ uint32_t at[kSortWaves][kDigits];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        for (int i = 0; i < kSortWaves; ++i) at[i][threadIdx.x] = 0;
        __syncthreads();
        const int64_t first = b * kSortBlock + int64_t(w) * 64 * kSortRounds;
        for (int r = 0; r < kSortRounds; ++r) {
            const int64_t i = first + r * 64 + lane;
            if (i < s.T) atomicAdd(&at[w][(sort_key(s, i) >> shift) & (kDigits - 1)], 1u);
        }
        __syncthreads();
        {   // counts -> each wavefront's first place for each digit
            uint32_t sum = offset[int64_t(threadIdx.x) * blocks + b];
            for (int i = 0; i < kSortWaves; ++i) {
                const uint32_t c = at[i][threadIdx.x];
                at[i][threadIdx.x] = sum;
                sum += c;
            }
        }
        __syncthreads();
        for (int r = 0; r < kSortRounds; ++r) {
            const int64_t i = first + r * 64 + lane;
            const bool is = i < s.T;
            const uint32_t k = is ? sort_key(s, i) : 0;
            const uint32_t d = (k >> shift) & (kDigits - 1);
            uint64_t same = __ballot(is);  // the lanes with this lane's digit
            for (int bit = 0; bit < 8; ++bit) {
                const uint64_t on = __ballot((d >> bit) & 1);
                same &= (d >> bit) & 1 ? on : ~on;
            }
            const int rank = __popcll(same & ((uint64_t(1) << lane) - 1));
            uint32_t place = 0;
            if (is) place = at[w][d];
            __builtin_amdgcn_wave_barrier();
            if (is && rank == 0) at[w][d] = place + uint32_t(__popcll(same));
            __builtin_amdgcn_wave_barrier();
            if (is) {
                key[place + rank] = k;
                tok[place + rank] = s.ids ? uint32_t(i) : s.tok[i];
            }
        }
        __syncthreads();
    }
}

// --------------------------------------------------------------- runs

// A run: `n` sorted places from `start`, of row v; n < 0: the only run of its
// row, -n places.
struct alignas(16) Run {
    uint32_t v, start;
    int32_t n;
    uint32_t tok;  // its first token
};
// A row of more than one run: its sorted places.
struct LongRow {
    uint32_t v, start, end;
};

struct RunList {
    Run* runs;
    LongRow* rows;
    uint32_t* count;  // of runs, of long rows
};

// The first sorted place in [lo, hi) whose key is above (or, with `from`, not
// below) k, or hi.
template <class Key>
__device__ __forceinline__ int64_t key_bound(const Key& key, int64_t lo, int64_t hi, uint32_t k,
                                             bool from) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (key(mid) > k || (from && key(mid) == k)) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// Lists the run that starts at sorted place i, and the long row; their order
// in the lists decides nothing.
template <class Key, class Tok, class Next>
__device__ __forceinline__ void list_run(const Key& key, const Tok& tok, int64_t i, int64_t T, int64_t V,
                                         const RunList& l, const Next& next) {
    const uint32_t v = key(i);
    if (v >= V) return;
    const bool first = i == 0 || key(i - 1) != v;
    if (!first) {
        if (i < kRun || key(i - kRun) != v) return;
        if ((i - key_bound(key, 0, i, v, true)) % kRun) return;
    }
    const int64_t cap = i + kRun < T ? i + kRun : T;
    const int64_t end = key(cap - 1) == v ? cap : key_bound(key, i, cap, v, false);
    const int n = int(end - i);
    const bool more = end < T && key(end) == v;
    l.runs[next(0)] = Run{v, uint32_t(i), first && !more ? -n : n, tok(i)};
    if (first && more)
        l.rows[next(1)] = LongRow{v, uint32_t(i), uint32_t(key_bound(key, end, T, v, false))};
}

// Up to kSmallSort tokens: one block sorts them in LDS, kSmallBits of the keys
// a pass.  A wavefront takes a contiguous share, 64 tokens a round, kept in
// registers between passes; a token's place is the sum of those of lower
// digits, of its digit in earlier wavefronts, in earlier rounds and in lower
// lanes.  16384 tokens are what LDS holds.  Against the launches above: 16384
// tokens, 131072 x 4096 bf16, the whole gradient 268 and 349 us; 4096 tokens,
// 32000 x 1024 fp32, 30 and 77.
constexpr int kSmallSort = 16384;
constexpr int kSmallBits = 9;
constexpr int kSmallDigits = 1 << kSmallBits;
constexpr int kSmallRounds = kSmallSort / 1024;

struct SmallSort {
    uint32_t key[kSmallSort];
    uint16_t tok[kSmallSort];
    uint32_t at[16][kSmallDigits];
    uint32_t wave[16];
    uint32_t count[2];
};

// f(0), f(1), .. as constants: what they index stays in registers.
template <int N, class F>
__device__ __forceinline__ void each_round(F&& f) {
    if constexpr (N > 0) {
        each_round<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

__device__ __forceinline__ void small_sort(SmallSort& s, const int64_t* ids, int T, int64_t V,
                                           uint32_t* tok, const RunList& l) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int rounds = (T + 1023) / 1024, first = w * rounds * 64 + lane;
    uint32_t k[kSmallRounds], n[kSmallRounds];
    uint32_t rank[kSmallRounds];
    each_round<kSmallRounds>([&](auto r_) {
        constexpr int r = decltype(r_)::value;
        const int i = first + r * 64;
        k[r] = 0;
        n[r] = uint32_t(i);
        if (r < rounds && i < T) {
            const int64_t id = ids[i];
            k[r] = id >= 0 && id < V ? uint32_t(id) : uint32_t(V);  // no token: behind all rows
        }
    });
    for (int shift = 0; (V >> shift) > 0; shift += kSmallBits) {
        for (int i = threadIdx.x; i < 16 * kSmallDigits; i += 1024) (&s.at[0][0])[i] = 0;
        __syncthreads();
        each_round<kSmallRounds>([&](auto r_) {
            constexpr int r = decltype(r_)::value;
            if (r >= rounds) return;
            const bool is = first + r * 64 < T;
            const uint32_t d = (k[r] >> shift) & (kSmallDigits - 1);
            uint64_t same = __ballot(is);  // the lanes with this lane's digit
            for (int bit = 0; bit < kSmallBits; ++bit) {
                const uint64_t on = __ballot((d >> bit) & 1);
                same &= (d >> bit) & 1 ? on : ~on;
            }
            const uint32_t below = uint32_t(__popcll(same & ((uint64_t(1) << lane) - 1)));
            const uint32_t before = s.at[w][d];
            __builtin_amdgcn_wave_barrier();
            if (is && below == 0) s.at[w][d] = before + uint32_t(__popcll(same));
            __builtin_amdgcn_wave_barrier();
            rank[r] = before + below;
        });
        __syncthreads();
        uint32_t own = 0, sum = 0;
        if (threadIdx.x < kSmallDigits) {  // a digit a thread
            for (int i = 0; i < 16; ++i) own += s.at[i][threadIdx.x];
            sum = own;
            for (int d = 1; d < 64; d *= 2) {
                const uint32_t o = __shfl_up(sum, d);
                if (lane >= d) sum += o;
            }
            if (lane == 63) s.wave[w] = sum;
        }
        __syncthreads();
        if (threadIdx.x < kSmallDigits) {
            sum -= own;
            for (int i = 0; i < w; ++i) sum += s.wave[i];
            for (int i = 0; i < 16; ++i) {
                const uint32_t c = s.at[i][threadIdx.x];
                s.at[i][threadIdx.x] = sum;
                sum += c;
            }
        }
        __syncthreads();
        each_round<kSmallRounds>([&](auto r_) {
            constexpr int r = decltype(r_)::value;
            if (r >= rounds || first + r * 64 >= T) return;
            const uint32_t at = s.at[w][(k[r] >> shift) & (kSmallDigits - 1)] + rank[r];
            s.key[at] = k[r];
            s.tok[at] = uint16_t(n[r]);
        });
        __syncthreads();
        each_round<kSmallRounds>([&](auto r_) {
            constexpr int r = decltype(r_)::value;
            if (r >= rounds || first + r * 64 >= T) return;
            k[r] = s.key[first + r * 64];
            n[r] = s.tok[first + r * 64];
        });
    }
    if (threadIdx.x < 2) s.count[threadIdx.x] = 0;
    __syncthreads();
    const auto key = [&](int64_t i) { return s.key[i]; };
    const auto at = [&](int64_t i) { return uint32_t(s.tok[i]); };
    for (int i = threadIdx.x; i < T; i += 1024) {
        tok[i] = s.tok[i];
        list_run(key, at, i, T, V, l, [&](int which) { return atomicAdd(&s.count[which], 1u); });
    }
    __syncthreads();
    if (threadIdx.x < 2) l.count[threadIdx.x] = s.count[threadIdx.x];
}

// Zeros over a matrix, by `blocks` blocks of which this is one, a wavefront
// kZeroVecs slices of 64 vectors of a row at a time.
constexpr int kZeroVecs = 8;

template <class T, int BLOCK>
__device__ __forceinline__ void zero_rows(T* m, uint32_t rows, int64_t cols, int64_t stride,
                                          uint32_t block, uint32_t blocks) {
    constexpr int VEC = Num<T>::VEC, WAVES = BLOCK / 64, UNIT = kZeroVecs * 64 * VEC;
    const uint32_t per = uint32_t((cols + UNIT - 1) / UNIT), units = rows * per;
    const uint32_t step = blocks * WAVES;
    for (uint32_t u = block * WAVES + wave_id(); u < units; u += step) {
        const int64_t at = int64_t(u % per) * UNIT + int64_t(threadIdx.x & 63) * VEC;
        T* const dst = m + int64_t(u / per) * stride + at;
#pragma unroll
        for (int i = 0; i < kZeroVecs; ++i) {
            const int64_t left = cols - at - i * 64 * VEC;
            if (left >= VEC) store_vec(dst + i * 64 * VEC, u32x4{0, 0, 0, 0});
            else if (left > 0) store_part(dst + i * 64 * VEC, u32x4{0, 0, 0, 0}, int(left));
        }
        if (units - u <= step) break;  // (u + step may pass 32 bits)
    }
}

// Block 0 sorts; the others, if any, fill the table with zeros.
template <class T>
__global__ __launch_bounds__(1024) void sort_zero_kernel(const int64_t* ids, int64_t tokens,
                                                         int64_t V, uint32_t* tok, RunList l,
                                                         T* m, int64_t rows, int64_t cols,
                                                         int64_t stride) {
    extern __shared__ char lds[];
    if (blockIdx.x == 0)
        small_sort(*reinterpret_cast<SmallSort*>(lds), ids, int(tokens), V, tok, l);
    else
        zero_rows<T, 1024>(m, uint32_t(rows), cols, stride, blockIdx.x - 1, gridDim.x - 1);
}

template <class T>
__global__ __launch_bounds__(256) void zero_kernel(T* m, int64_t rows, int64_t cols,
                                                   int64_t stride) {
    zero_rows<T, 256>(m, uint32_t(rows), cols, stride, blockIdx.x, gridDim.x);
}

// More tokens: the list of runs from the sorted keys in memory.
__global__ __launch_bounds__(256) void list_kernel(const uint32_t* keys, const uint32_t* tok,
                                                   int64_t tokens, int64_t V, RunList l) {
    const auto key = [&](int64_t i) { return keys[i]; };
    const auto at = [&](int64_t i) { return tok[i]; };
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < tokens;
         i += int64_t(gridDim.x) * 256)
        list_run(key, at, i, tokens, V, l, [&](int which) { return atomicAdd(&l.count[which], 1u); });
}

// --------------------------------------------------------------- fold

struct FoldArgs {
    RunList l;
    const uint32_t* tok;  // the sorted tokens
    int64_t D;
    int64_t dout_stride, dtable_stride;
    float scale;
    int accumulate;
    // fp32 sums of the runs of long rows, `pitch` apart: a full run that starts
    // at sorted place i is at i / kRun of `full`, the run of fewer tokens that
    // ends the row at (i - kRun) / kRun of `tail` (its place less a run is where
    // a full run of the row starts; two full runs are at least kRun apart).
    float* full;
    float* tail;
    int64_t pitch;
};

// W columns from `at` of a row's sum to the table.
template <class T, int W = Num<T>::VEC>
__device__ __forceinline__ void finish_row(const FoldArgs& a, T* dtable, uint32_t v, int64_t at,
                                           const float* sum) {
    T* const dst = dtable + int64_t(v) * a.dtable_stride + at;
    if constexpr (W == Num<T>::VEC) if (a.D - at >= W) {
        float f[W];
#pragma unroll
        for (int i = 0; i < W; ++i) f[i] = sum[i] * a.scale;
        if (a.accumulate) {
            float old[W];
            Num<T>::unpack(load_vec(dst), old);
#pragma unroll
            for (int i = 0; i < W; ++i) f[i] += old[i];
        }
        store_vec(dst, Num<T>::pack(f));
        return;
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (a.D - at <= i) continue;
        const float f = sum[i] * a.scale;
        dst[i] = Num<T>::down(a.accumulate ? f + Num<T>::up(dst[i]) : f);
    }
}

// The sums of N more rows over S slices of 64 vectors, their loads in flight
// together; `row(i)` is row i, `left` what the matrix has from the lane's first
// element on.
template <class T, int N, int S, class Row>
__device__ __forceinline__ void add_rows(float (*sum)[Num<T>::VEC], int64_t left, Row&& row) {
    constexpr int VEC = Num<T>::VEC;
    u32x4 x[N][S];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const T* src = row(i);
#pragma unroll
        for (int s = 0; s < S; ++s) {
            const int64_t n = left - s * 64 * VEC;
            x[i][s] = u32x4{0, 0, 0, 0};
            if (n >= VEC) x[i][s] = load_vec(src + s * 64 * VEC);
            else if (n > 0) x[i][s] = load_part(src + s * 64 * VEC, int(n));
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int s = 0; s < S; ++s) {
            float f[VEC];
            Num<T>::unpack(x[i][s], f);
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[s][e] += f[e];
        }
}
// The same for n rows, n a scalar, at most kFoldLoads vectors in flight.
constexpr int kFoldLoads = 8;
template <class T, int S, class Row>
__device__ __forceinline__ void add_all(float (*sum)[Num<T>::VEC], int64_t left, int n, Row&& row) {
    constexpr int N = kFoldLoads / S;
    int j = 0;
    const auto at = [&](int i) { return row(j + i); };
    for (; j + N <= n; j += N) add_rows<T, N, S>(sum, left, at);
    if constexpr (N > 4)
        if ((n - j) & 4) {
            add_rows<T, 4, S>(sum, left, at);
            j += 4;
        }
    if constexpr (N > 2)
        if ((n - j) & 2) {
            add_rows<T, 2, S>(sum, left, at);
            j += 2;
        }
    if ((n - j) & 1) add_rows<T, 1, S>(sum, left, at);
}

// One wavefront a (run, S slices of 64 vectors of the row).
template <class T, int S>
__global__ __launch_bounds__(256) void fold_kernel(FoldArgs a, const T* dout, T* dtable) {
    constexpr int VEC = Num<T>::VEC, UNIT = S * 64 * VEC;
    const int lane = threadIdx.x & 63;
    const uint32_t per = uint32_t((a.D + UNIT - 1) / UNIT);
    const uint32_t units = a.l.count[0] * per, step = gridDim.x * 4;
    for (uint32_t u = blockIdx.x * 4 + wave_id(); u < units; u += step) {
        const Run run = a.l.runs[u / per];
        const uint32_t v = scalar(run.v), start = scalar(run.start);
        const int size = int(scalar(uint32_t(run.n))), n = size < 0 ? -size : size;
        const int64_t at = int64_t(u % per) * UNIT + int64_t(lane) * VEC;
        const int64_t left = a.D - at;  // of the row, from the lane's first element on
        float sum[S][VEC] = {};
        if (n == 1) {
            const T* const src = dout + int64_t(scalar(run.tok)) * a.dout_stride + at;
            add_rows<T, 1, S>(sum, left, [&](int) { return src; });
        } else {
            const uint32_t mine = lane < n ? a.tok[start + lane] : 0;
            add_all<T, S>(sum, left, n, [&](int i) {
                return dout + int64_t(uint32_t(__builtin_amdgcn_readlane(int(mine), i))) * a.dout_stride + at;
            });
        }
        float* const part = (n == kRun ? a.full + int64_t(start / kRun) * a.pitch
                                       : a.tail + int64_t((start - kRun) / kRun) * a.pitch) + at;
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (left <= s * 64 * VEC) continue;
            if (size < 0) {
                finish_row(a, dtable, v, at + s * 64 * VEC, sum[s]);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; e += 4)
                    store_vec(part + s * 64 * VEC + e, Num<float>::pack(sum[s] + e));
            }
        }
        if (units - u <= step) break;  // (u + step may pass 32 bits)
    }
}

// Rows with more than one run: a wavefront a (row, slice of 64 fp32 vectors).
template <class T>
__global__ __launch_bounds__(256) void join_kernel(FoldArgs a, T* dtable) {
    constexpr int W = 4;  // columns a lane
    const uint32_t slices = uint32_t((a.D + 64 * W - 1) / (64 * W));
    const uint32_t units = a.l.count[1] * slices, step = gridDim.x * 4;
    for (uint32_t u = blockIdx.x * 4 + wave_id(); u < units; u += step) {
        const LongRow* const r = a.l.rows + u / slices;
        const uint32_t v = scalar(r->v), start = scalar(r->start), end = scalar(r->end);
        const int64_t at = int64_t(u % slices) * 64 * W + int64_t(threadIdx.x & 63) * W;
        const int64_t left = at < a.D ? W : 0;  // (the sums' rows are padded)
        const int full = int((end - start) / kRun), rest = int((end - start) % kRun);
        float sum[1][W] = {};
        const float* const src = a.full + int64_t(start / kRun) * a.pitch + at;
        add_all<float, 1>(sum, left, full, [&](int i) { return src + i * a.pitch; });
        if (rest) {
            const float* const last = a.tail + int64_t((end - rest - kRun) / kRun) * a.pitch + at;
            add_rows<float, 1, 1>(sum, left, [&](int) { return last; });
        }
        if (left) finish_row<T, W>(a, dtable, v, at, sum[0]);
        if (units - u <= step) break;
    }
}

struct GradSpace {  // the workspace's parts, in bytes from its start
    int64_t key[2], tok[2], hist, runs, rows, count, full, tail, end;
    int64_t blocks, pitch;
};

GradSpace grad_space(int64_t D, int64_t T) {
    GradSpace g{};
    g.blocks = ceil_div(T, kSortBlock);
    g.pitch = round_up(D, 8);
    const int64_t stretches = ceil_div(T, kRun);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at = round_up(at + bytes, 256);
        return here;
    };
    const bool small = T <= kSmallSort;
    for (int i = 0; i < 2; ++i) {
        g.key[i] = take(small ? 0 : 4 * T);
        g.tok[i] = take(small && i ? 0 : 4 * T);
    }
    g.hist = take(small ? 0 : 4 * kDigits * g.blocks);
    g.runs = take(int64_t(sizeof(Run)) * T);
    g.rows = take(int64_t(sizeof(LongRow)) * stretches);
    g.count = take(8);
    g.full = take(4 * stretches * g.pitch);
    g.tail = take(4 * stretches * g.pitch);
    g.end = at;
    return g;
}

// Blocks of 1024 threads, beside the sort (256 take the same time).
constexpr int64_t kZeroBlocks = 1024;
// Of 4 wavefronts: the card's 256 CUs hold them at once (8 times as many take
// the same time).
constexpr int64_t kFoldBlocks = 2048;

unsigned grid_of(int64_t blocks) { return unsigned(std::min<int64_t>(blocks, 1 << 20)); }

template <class T>
ar_status run_lookup(int64_t V, int64_t D, int64_t rows, const void* table, int64_t table_stride,
                     const int64_t* ids, float scale, void* out, int64_t out_stride,
                     hipStream_t st) {
    const int64_t units = rows * ceil_div(D, 64 * Num<T>::VEC);
    hipLaunchKernelGGL((lookup_kernel<T>), dim3(grid_of(ceil_div(units, 4))), dim3(256), 0, st,
                       static_cast<const T*>(table), table_stride, ids, V, D, rows, scale,
                       static_cast<T*>(out), out_stride);
    return launch_status("embedding lookup");
}

template <class T>
ar_status run_grad(int64_t V, int64_t D, int64_t rows, const void* dout, int64_t dout_stride,
                   const int64_t* ids, float scale, int32_t accumulate, void* dtable,
                   int64_t dtable_stride, char* ws, hipStream_t st) {
    T* const out = static_cast<T*>(dtable);
    // adjacent rows are zeroed as one
    const bool flat = dtable_stride == D;
    const int64_t zr = flat ? 1 : V, zc = flat ? V * D : D;
    const int64_t zeros = accumulate ? 0 : zr * ceil_div(zc, kZeroVecs * 64 * Num<T>::VEC);
    if (rows == 0) {
        if (zeros)
            hipLaunchKernelGGL((zero_kernel<T>), dim3(grid_of(ceil_div(zeros, 4))), dim3(256), 0,
                               st, out, zr, zc, dtable_stride);
        return launch_status("embedding gradient");
    }
    const GradSpace g = grad_space(D, rows);
    uint32_t* key[2] = {reinterpret_cast<uint32_t*>(ws + g.key[0]),
                        reinterpret_cast<uint32_t*>(ws + g.key[1])};
    uint32_t* tok[2] = {reinterpret_cast<uint32_t*>(ws + g.tok[0]),
                        reinterpret_cast<uint32_t*>(ws + g.tok[1])};
    const RunList l{reinterpret_cast<Run*>(ws + g.runs), reinterpret_cast<LongRow*>(ws + g.rows),
                    reinterpret_cast<uint32_t*>(ws + g.count)};
    const uint32_t* sorted = tok[0];
    if (rows <= kSmallSort) {
        const unsigned blocks = unsigned(std::min<int64_t>(ceil_div(zeros, 16), kZeroBlocks));
        hipLaunchKernelGGL((sort_zero_kernel<T>), dim3(1 + blocks), dim3(1024), sizeof(SmallSort),
                           st, ids, rows, V, tok[0], l, out, zr, zc, dtable_stride);
    } else {
        if (zeros)
            hipLaunchKernelGGL((zero_kernel<T>), dim3(grid_of(ceil_div(zeros, 4))), dim3(256), 0,
                               st, out, zr, zc, dtable_stride);
        uint32_t* hist = reinterpret_cast<uint32_t*>(ws + g.hist);
        SortSrc src{ids, nullptr, nullptr, V, rows};
        int to = 0;
        for (int shift = 0; (V >> shift) > 0; shift += 8, to ^= 1) {  // keys are 0 .. V
            hipLaunchKernelGGL(sort_count_kernel, dim3(grid_of(g.blocks)), dim3(256), 0, st, src,
                               shift, hist, g.blocks);
            hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), 0, st, hist,
                               kDigits * g.blocks, l.count);
            hipLaunchKernelGGL(sort_move_kernel, dim3(grid_of(g.blocks)), dim3(256), 0, st, src,
                               shift, hist, g.blocks, key[to], tok[to]);
            src = SortSrc{nullptr, key[to], tok[to], V, rows};
        }
        hipLaunchKernelGGL(list_kernel, dim3(grid_of(ceil_div(rows, 256))), dim3(256), 0, st,
                           src.key, src.tok, rows, V, l);
        sorted = src.tok;
    }
    const FoldArgs a{l, sorted, D, dout_stride, dtable_stride, scale, accumulate,
                     reinterpret_cast<float*>(ws + g.full), reinterpret_cast<float*>(ws + g.tail),
                     g.pitch};
    const auto grid = [](int64_t units) {  // at most so many wavefronts, which then loop
        return dim3(unsigned(std::min<int64_t>(ceil_div(units, 4), kFoldBlocks)));
    };
    // two slices a wavefront where a row has them: twice the loads in flight, most
    // of all for the rows of one token (4096 tokens, 32000 x 4096 bf16: the whole
    // gradient 54 us against 60, 32000 x 1024 fp32 30 against 31; 16384 tokens,
    // 131072 x 4096 bf16 the same within what runs differ by)
    if (D > 64 * Num<T>::VEC)
        hipLaunchKernelGGL((fold_kernel<T, 2>), grid(rows * ceil_div(D, 128 * Num<T>::VEC)), dim3(256),
                           0, st, a, static_cast<const T*>(dout), out);
    else
        hipLaunchKernelGGL((fold_kernel<T, 1>), grid(rows), dim3(256), 0, st, a,
                           static_cast<const T*>(dout), out);
    if (rows > kRun)
        hipLaunchKernelGGL((join_kernel<T>), grid(ceil_div(rows, kRun) * ceil_div(D, 256)), dim3(256),
                           0, st, a, out);
    return launch_status("embedding gradient");
}

// The kernels count a matrix's slices, a wavefront's share of a row, in 32 bits.
ar_status check_slices(int64_t rows, int64_t D) {
    if (rows > 0 && ceil_div(D, 256) > int64_t(UINT32_MAX) / rows)
        return fail(AR_ERR_UNSUPPORTED, "a matrix of more than 2^40 elements");
    return AR_OK;
}

ar_status check_ids(const int64_t* ids, int64_t T) {
    return check_matrix({"ids", ids, 1, T, T, 8});
}

}  // namespace
}  // namespace arp

using namespace arp;

AR_EXPORT ar_status ar_embed_lookup(int32_t dtype, int64_t V, int64_t D, int64_t T,
                                    const void* table, int64_t table_stride, const int64_t* ids,
                                    float scale, void* out, int64_t out_stride, void* stream) try {
    clear_error();
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_extent("V", V));
    AR_TRY(check_extent("D", D));
    AR_TRY(check_extent("T", T));
    const MatArg mt{"table", table, V, D, table_stride, es}, mo{"out", out, T, D, out_stride, es};
    const MatArg mi{"ids", ids, 1, T, T, 8};
    AR_TRY(check_matrix(mt));
    AR_TRY(check_matrix(mo));
    AR_TRY(check_ids(ids, T));
    AR_TRY(check_apart(mo, mt));
    AR_TRY(check_apart(mo, mi));
    AR_TRY(check_slices(T, D));
    if (T == 0 || D == 0) return AR_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == AR_F32 ? run_lookup<float>(V, D, T, table, table_stride, ids, scale, out, out_stride, st)
                           : run_lookup<uint16_t>(V, D, T, table, table_stride, ids, scale, out, out_stride, st);
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_embed_grad_workspace(int64_t V, int64_t D, int64_t T, int64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    AR_TRY(check_extent("V", V));
    AR_TRY(check_extent("D", D));
    AR_TRY(check_extent("T", T));
    *bytes = V == 0 || D == 0 || T == 0 ? 0 : grad_space(D, T).end;
    return AR_OK;
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_embed_grad(int32_t dtype, int64_t V, int64_t D, int64_t T, const void* dout,
                                  int64_t dout_stride, const int64_t* ids, float scale,
                                  int32_t accumulate, void* dtable, int64_t dtable_stride,
                                  void* workspace, int64_t workspace_bytes, void* stream) try {
    clear_error();
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    int64_t need = 0;
    AR_TRY(ar_embed_grad_workspace(V, D, T, &need));
    const MatArg md{"dout", dout, T, D, dout_stride, es},
        mt{"dtable", dtable, V, D, dtable_stride, es}, mi{"ids", ids, 1, T, T, 8},
        mw{"the workspace", workspace, 1, need, need, 1};
    AR_TRY(check_matrix(md));
    AR_TRY(check_matrix(mt));
    AR_TRY(check_ids(ids, T));
    AR_TRY(check_workspace(workspace, workspace_bytes, need));
    AR_TRY(check_apart(mt, md));
    AR_TRY(check_apart(mt, mi));
    for (const MatArg& m : {md, mt, mi}) AR_TRY(check_apart(mw, m));
    AR_TRY(check_slices(V, D));
    AR_TRY(check_slices(T, D));
    if (V == 0 || D == 0) return AR_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    return dtype == AR_F32 ? run_grad<float>(V, D, T, dout, dout_stride, ids, scale, accumulate, dtable, dtable_stride, ws, st)
                           : run_grad<uint16_t>(V, D, T, dout, dout_stride, ids, scale, accumulate, dtable, dtable_stride, ws, st);
} catch (...) {
    return thrown();
}
