// Attention's relative position bias by buckets of distance, and its table's gradient.
//
// The bias depends on j - i alone: along a diagonal of a head's Q x K matrix it is one
// number, and all of a diagonal's gradients go to one bucket.  So buckets are looked up
// a diagonal, not an element: a patch of the bias is stored from its diagonals' values
// in LDS, and a patch of gradients is first summed along its diagonals, in registers, and
// those sums are sorted into buckets.  An element costs its way through memory and, in
// the gradient, one addition.
//
// The distance on diagonal d = j - i is n = offset - d.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "replica.hpp"

namespace arp {
namespace {

constexpr int kBlock = 256, kWaves = kBlock / 64;

// The distances at which the buckets of a side begin: bucket b of `side` from at[b] on.
struct Borders {
    int32_t side;
    bool causal;
    int32_t at[AR_POSITION_MAX_BUCKETS];
};

struct BiasShape {
    int64_t H, Q, K, offset;
    int64_t rows, row_tiles, chunks;  // rows of a tile, and chunks of columns
};

// The place of a block: head, rows [i0, i1) and its first column.
struct Patch {
    int64_t h, i0, i1, j0;
};
__device__ __forceinline__ Patch patch_of(const BiasShape& s, int64_t n, int width) {
    const int64_t over = quotient(n, s.chunks), chunk = n - over * s.chunks;
    Patch p;
    p.h = quotient(over, s.row_tiles);
    const int64_t tile = over - p.h * s.row_tiles;
    p.i0 = tile * s.rows;
    p.i1 = p.i0 + s.rows < s.Q ? p.i0 + s.rows : s.Q;
    p.j0 = chunk * width;
    return p;
}

// The bucket of distance n from the borders `at`; behind the query in buckets of their
// own, or (causal) none.
__device__ __forceinline__ int bucket_of(const int32_t* at, int side, bool causal, int64_t n) {
    if (causal && n < 0) return -1;
    const int64_t d = n < 0 ? -n : n;
    int lo = 0, hi = side;  // at[lo] <= d < at[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (at[mid] <= d) lo = mid;
        else hi = mid;
    }
    return n < 0 ? side + lo : lo;
}

// The bias: a wavefront stores kBiasRows rows of 64 vectors, the block's wavefronts lie
// side by side as far as the rows are long.
constexpr int kBiasRows = 16;
// (Few rows: a block a chunk of 64 vectors, for there the lookups are what takes time: one
// query over 4001 keys 5.0 us, side by side 7.4.)
int bias_side(int64_t Q, int64_t K, int width) {
    return Q < kBiasRows ? 1 : K > 2 * width ? 4 : K > width ? 2 : 1;
}

// A lane's vectors of VEC rows from the 2 VEC diagonals' values that hold them all: row
// r's begins VEC - r further on.
__device__ __forceinline__ void vectors_of(const u32x4 a, const u32x4 b, float, u32x4* v) {
    v[0] = b;
    v[1] = u32x4{a[3], b[0], b[1], b[2]};
    v[2] = u32x4{a[2], a[3], b[0], b[1]};
    v[3] = u32x4{a[1], a[2], a[3], b[0]};
}
__device__ __forceinline__ void vectors_of(const u32x4 a, const u32x4 b, uint16_t, u32x4* v) {
    const uint32_t even[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    uint32_t odd[7];
#pragma unroll
    for (int k = 0; k < 7; ++k) odd[k] = __builtin_amdgcn_alignbyte(even[k + 1], even[k], 2);
#pragma unroll
    for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int x = 8 - r + 2 * e;
            v[r][e] = x % 2 ? odd[x / 2] : even[x / 2];
        }
}

template <class T>
__device__ __forceinline__ T element(const u32x4 v, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[e]);
    else return T(v[e / 2] >> (16 * (e % 2)));
}

// The values of a patch's diagonals lie in LDS; a lane reads those of VEC rows at once,
// and their vectors are parts of them.  Bound by memory, the matrix is written once: 16 x
// 2048 x 2048 bf16, 134 MB, 26.4 us, 5.1 TB/s (a fill of that size 24), f32 51, 5.3.  Lanes that keep a
// vector of diagonals and store it one element further on in each row, off 16 bytes, took 28.3;
// rows of 1 KB a block in place of whole ones of 4 KB 31.8.  One query over 4001 keys for 32
// heads: 5.0, the borders' and the table's way to LDS and the lookups.
template <class T>
__global__ __launch_bounds__(kBlock) void bias_kernel(BiasShape s, Borders borders, const T* table,
                                                      int64_t table_stride, int buckets, T* out,
                                                      int64_t head_stride, int64_t row_stride,
                                                      int64_t patches, int side) {
    constexpr int VEC = Num<T>::VEC, WIDTH = 64 * VEC;
    __shared__ __attribute__((aligned(16))) T value[kWaves * WIDTH + kWaves * kBiasRows];
    __shared__ int32_t at[AR_POSITION_MAX_BUCKETS];
    __shared__ T column[AR_POSITION_MAX_BUCKETS];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6);
    const int across = wave % side, down = wave / side;
    for (int64_t n = blockIdx.x; n < patches; n += gridDim.x) {
        const Patch p = patch_of(s, n, side * WIDTH);
        const int rows = int(p.i1 - p.i0);
        const int ceiling = (rows + VEC - 1) / VEC * VEC;
        if (int(threadIdx.x) < buckets) {
            at[threadIdx.x] = borders.at[threadIdx.x];
            column[threadIdx.x] = table[threadIdx.x * table_stride + p.h];
        }
        __syncthreads();
        // diagonal j0 - i0 - ceiling + x at x
        for (int x = threadIdx.x; x < side * WIDTH + ceiling; x += kBlock) {
            const int b = bucket_of(at, borders.side, borders.causal, s.offset - (p.j0 - p.i0 - ceiling + x));
            value[x] = b < 0 ? Num<T>::down(-INFINITY) : column[b];
        }
        __syncthreads();
        const int x = (across * 64 + lane) * VEC;
        const int64_t j = p.j0 + x;
        const int end = (down + 1) * kBiasRows < rows ? (down + 1) * kBiasRows : rows;
        for (int i = down * kBiasRows; i < end; i += VEC) {
            const AR_LDS u32x4* const from = (const AR_LDS u32x4*)((const AR_LDS T*)value + x + ceiling - i - VEC);
            u32x4 v[VEC];
            const u32x4 a = from[0], b = from[1];
            vectors_of(a, b, T(0), v);
            T* const to = out + p.h * head_stride + (p.i0 + i) * row_stride + j;
#pragma unroll
            for (int r = 0; r < VEC; ++r) {
                if (i + r >= end) break;
                if (j + VEC <= s.K) {
                    store_vec(to + r * row_stride, v[r]);
                } else if (j < s.K) {
                    // (bits: a conversion would change those of a NaN)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        if (j + e < s.K) ((AR_GLOBAL T*)to)[r * row_stride + e] = element<T>(v[r], e);
                }
            }
        }
        __syncthreads();
    }
}

struct GradArgs {
    int64_t B, batch_stride, head_stride, row_stride;
    int64_t span;     // elements from the first to the last one, and itself
    int64_t batches;  // of one block
    int64_t splits;
    int32_t rows;  // of a wavefront
    int32_t across, down;  // a block's wavefronts side by side, and one below the other; of
                           // less than four the others take other batches
};

// A lane's sums of its vector's diagonals, as it goes down the rows of a patch, VEC
// rows a step.  With b the diagonal of the vector's first element in a step's first
// row, `main` holds diagonals b .. b + VEC - 1 and `low` the VEC - 1 before them.  In the
// next step b is VEC less: `low` becomes main, and main the next lane's main, whose
// vector has now come to those diagonals; the last lane's leaves the wavefront.
template <int VEC>
struct Diagonals {
    float main[VEC], low[VEC];  // (low[0] is not used)
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int e = 0; e < VEC; ++e) main[e] = low[e] = 0.0f;
    }
    __device__ __forceinline__ void add(int row, const float* f) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            if (e >= row) main[e - row] += f[e];
            else low[e - row + VEC] += f[e];
        }
    }
    __device__ __forceinline__ void step() {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            // (lane l from lane l - 1, the first from none)
            const float from = __uint_as_float(uint32_t(__builtin_amdgcn_mov_dpp(
                int(__float_as_uint(main[e])), 0x138, 0xF, 0xF, true)));
            main[e] = low[e] + from;
            low[e] = 0.0f;
        }
    }
    __device__ __forceinline__ void put(AR_LDS float* to, bool first) const {
        typedef float f4 __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int e = 0; e < VEC; e += 4) {
            f4 v = {main[e], main[e + 1], main[e + 2], main[e + 3]};
            if (!first) v += *(const AR_LDS f4*)(to + e);
            *(AR_LDS f4*)(to + e) = v;
        }
    }
};

constexpr int kGradRows = 64;  // of a wavefront at most

// A wavefront's sums by diagonal of a patch, `rows` rows (a multiple of 2 VEC) from i0,
// of which those below i1 are there, and 64 VEC columns from j0 on, to LDS, or added to
// what is there: diagonal j0 - i0 - rows + x at x.  EDGE: the patch is not whole, or not
// all of it seen; a vector that passes a row's end is read whole and what lies behind the
// row left out, where that lies before the tensor's last element.
template <class T, bool EDGE>
__device__ __forceinline__ void sum_patch(const T* from, const T* end, int64_t stride, int rows,
                                          int64_t i0, int64_t i1, int64_t j0, int64_t K, int64_t seen,
                                          bool first, AR_LDS float* sums) {
    constexpr int VEC = Num<T>::VEC;
    const int lane = threadIdx.x & 63, steps = rows / VEC;
    // a lane's columns that are there, and the rows that see any of them and can be read whole
    int n = VEC, begin = 0, there = rows, safe = rows;
    if constexpr (EDGE) {
        const int64_t left = K - j0 - lane * VEC, late = j0 + lane * VEC - seen - i0;
        n = int(left < 0 ? 0 : left < VEC ? left : VEC);
        begin = n == 0 ? rows : int(late < 0 ? 0 : late < rows ? late : rows);
        if (i1 - i0 < rows) there = int(i1 - i0);
        safe = there;
        // (vectors reach that far into a row)
        const int64_t reach = K - j0 < 64 * VEC ? (K - j0 + VEC - 1) / VEC * VEC : 64 * VEC;
        while (safe > 0 && from + (safe - 1) * stride + reach > end) --safe;
    }
    Diagonals<VEC> d;
    d.clear();
    const T* p = from;
    // The steps' rows one after the other, read once and past the caches: 537 MB 80 us, as
    // ordinary loads 88.
    auto load = [&](int step, u32x4* v) {
        // (one address after the other, not each row's kept in registers of its own)
        int64_t next = stride;
        asm volatile("" : "+s"(next));
#pragma unroll
        for (int r = 0; r < VEC; ++r, p += next) {
            const int i = step * VEC + r;
            if (EDGE) v[r] = u32x4{0, 0, 0, 0};
            if (!EDGE || (i >= begin && i < safe))
                v[r] = __builtin_nontemporal_load((const typename Num<T>::V*)(p + lane * VEC));
        }
    };
    auto add = [&](int step, const u32x4* v) {
#pragma unroll
        for (int r = 0; r < VEC; ++r) {
            float f[VEC];
            Num<T>::unpack(v[r], f);
            if (EDGE) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = e < n ? f[e] : 0.0f;
            }
            d.add(r, f);
        }
        if (lane == 63) d.put(sums + (63 + steps - step) * VEC, first);
        d.step();
    };
    // (Of bf16, with another step's vectors there are registers too few; fp32's are half as
    // many, and its steps wait here all the same: a second one in flight has not been built.)
    if constexpr (EDGE) {
        u32x4 w[VEC];
#pragma unroll 1
        for (int step = 0; step < steps; ++step) {
            load(step, w);
            add(step, w);
        }
    } else {
        u32x4 v[VEC], w[VEC];
        int step = 0;
        load(0, v);
#pragma unroll 1
        for (; step + 2 < steps; step += 2) {
            load(step + 1, w);
            add(step, v);
            load(step + 2, v);
            add(step + 1, w);
        }
        load(step + 1, w);
        add(step, v);
        add(step + 1, w);
    }
    d.put(sums + lane * VEC, first);
    if constexpr (EDGE) {  // the tensor's last rows, an element at a time
#pragma unroll 1
        for (int i = safe; i < there; ++i) {
            wave_sync();
#pragma unroll 1
            for (int e = 0; e < n && i >= begin; ++e)
                sums[lane * VEC + e + rows - i] += Num<T>::up(((const AR_GLOBAL T*)(from + i * stride))[lane * VEC + e]);
        }
    }
}

// A block's sums by bucket, to its slot of `part`, or straight to the table where a
// head has one slot.  Bound by memory, the gradients pass once: 4 x 16 x 2048 x 2048 bf16, 537
// MB, 85 us, 6.3 TB/s, its join 4.6.  (Lanes that walk down their diagonals, each row's
// vector off 16 bytes by one element more: 113.)  In f32, 1074 MB, 195, 5.5 TB/s, and 4.8.  3 x 5
// x 509 x 1021 f32, of which 23 MB are seen: 13.8 and 4.0, the steps of a block one after the other.
// Keys fewer than 64 vectors leave lanes idle: 32 x 16 x 1024 x 48, 50 MB in bf16 and 101 in f32,
// 47 and 43.
template <class T>
__global__ __launch_bounds__(kBlock, 4) void bias_grad_kernel(BiasShape s, Borders borders, GradArgs a,
                                                           const T* d, int32_t buckets, float* part,
                                                           T* dtable, int64_t table_stride,
                                                           int32_t accumulate) {
    constexpr int VEC = Num<T>::VEC, WIDTH = 64 * VEC, LENGTH = WIDTH + kGradRows;
    __shared__ __attribute__((aligned(16))) float sums[kWaves][LENGTH];
    __shared__ float total[kWaves * (WIDTH + kGradRows)];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6);
    const int64_t per_head = s.row_tiles * s.chunks, patches = s.H * per_head;
    const int64_t seen = borders.causal ? s.offset : INT64_MAX / 2;
    const int rows = a.rows, tile = a.down * rows, width = a.across * WIDTH;
    const int fold = a.across * a.down;     // wavefronts with patches of their own
    for (int64_t n = blockIdx.x; n < patches * a.splits; n += gridDim.x) {
        const int64_t split = quotient(n, patches), in = n - split * patches;
        const Patch p = patch_of(s, in, width);
        const int64_t i0 = p.i0 + wave % fold / a.across * rows, j0 = p.j0 + wave % a.across * WIDTH;
        const int64_t i1 = i0 + rows < p.i1 ? i0 + rows : p.i1;
        const int64_t b0 = split * a.batches + wave / fold;
        const int64_t b1 = (split + 1) * a.batches < a.B ? (split + 1) * a.batches : a.B;
        AR_LDS float* const mine = (AR_LDS float*)sums[wave];
        // A lane looks at a bucket, wavefronts in turn.  Its distances [near, far) are
        // diagonals (offset - far, offset - near], or, behind the query, [offset + near,
        // offset + far).
        const int b = lane * kWaves + wave;
        int from = 0, to = 0;
        if (b < buckets) {
            const bool behind = b >= borders.side;
            const int m = behind ? b - borders.side : b;
            const int64_t near = borders.at[m], d0 = p.j0 - p.i0 - tile;
            int64_t lo = behind ? s.offset + (near ? near : 1) : INT64_MIN / 2;
            int64_t hi = behind ? INT64_MAX / 2 : s.offset - near + 1;
            if (m + 1 < borders.side) {
                if (behind) hi = s.offset + borders.at[m + 1];
                else lo = s.offset - borders.at[m + 1] + 1;
            }
            lo = lo > d0 ? lo - d0 : 0;
            hi = hi - d0 < width + tile ? hi - d0 : width + tile;
            if (lo < hi) {
                from = int(lo);
                to = int(hi);
            }
        }
        if (i0 < i1 && j0 < s.K && b0 < b1 && j0 - (i1 - 1) <= seen) {
            const bool whole = j0 + WIDTH <= s.K && i0 + rows <= i1 && j0 + WIDTH - 1 - i0 <= seen;
            for (int64_t k = b0; k < b1; k += kWaves / fold) {
                const T* const at = d + k * a.batch_stride + p.h * a.head_stride + i0 * a.row_stride + j0;
                if (whole)
                    sum_patch<T, false>(at, d + a.span, a.row_stride, rows, i0, i1, j0, s.K, seen, k == b0, mine);
                else
                    sum_patch<T, true>(at, d + a.span, a.row_stride, rows, i0, i1, j0, s.K, seen, k == b0, mine);
            }
        } else {
            for (int x = lane; x < WIDTH + rows; x += 64) mine[x] = 0.0f;
        }
        __syncthreads();
        // the wavefronts', diagonal j0 - i0 - tile + x at x
        for (int x = threadIdx.x; x < width + tile; x += kBlock) {
            float t = 0.0f;
#pragma unroll
            for (int v = 0; v < kWaves; ++v) {
                const int y = x - (v % a.across * WIDTH + tile - (v % fold / a.across + 1) * rows);
                if (y >= 0 && y < WIDTH + rows) t += sums[v][y];
            }
            total[x] = t;
        }
        __syncthreads();
        auto result = [&](int bucket, float t) {
            if (part) {
                const int64_t slots = per_head * a.splits;
                part[(p.h * buckets + bucket) * slots + split * per_head + in - p.h * per_head] = t;
            } else {
                T* const at = dtable + bucket * table_stride + p.h;
                *at = Num<T>::down(accumulate ? t + Num<T>::up(*at) : t);
            }
        };
        // few diagonals by the lane alone, many by the wavefront
        constexpr int FEW = 16;
        float few = 0.0f;
        for (int x = 0; x < FEW && __builtin_amdgcn_ballot_w64(to - from <= FEW && from + x < to); ++x)
            few += to - from <= FEW && from + x < to ? total[from + x] : 0.0f;
        if (b < buckets && to - from <= FEW) result(b, few);
        for (uint64_t left = __builtin_amdgcn_ballot_w64(to - from > FEW); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            const int end = __builtin_amdgcn_readlane(to, l);
            float t = 0.0f;
            for (int x = __builtin_amdgcn_readlane(from, l) + lane; x < end; x += 64) t += total[x];
            t = wave_sum(t);
            if (lane == 0) result(l * kWaves + wave, t);
        }
        __syncthreads();
    }
}

// The slots' sums, a wavefront a bucket of a head.
template <class T>
__global__ __launch_bounds__(kBlock) void bias_join_kernel(int64_t H, int32_t buckets, int64_t slots,
                                                           const float* part, T* dtable,
                                                           int64_t table_stride, int32_t accumulate) {
    const int lane = threadIdx.x & 63;
    for (int64_t n = int64_t(blockIdx.x) * kWaves + (threadIdx.x >> 6); n < H * buckets;
         n += int64_t(gridDim.x) * kWaves) {
        float t = 0.0f;
        for (int64_t x = lane; x < slots; x += 64) t += part[n * slots + x];
        t = wave_sum(t);
        if (lane == 0) {
            T* const to = dtable + n % buckets * table_stride + n / buckets;
            *to = Num<T>::down(accumulate ? t + Num<T>::up(*to) : t);
        }
    }
}

template <class T>
__global__ __launch_bounds__(kBlock) void table_zero_kernel(int64_t H, int32_t buckets, T* dtable,
                                                            int64_t table_stride) {
    for (int64_t n = int64_t(blockIdx.x) * kBlock + threadIdx.x; n < H * buckets;
         n += int64_t(gridDim.x) * kBlock)
        dtable[n / H * table_stride + n % H] = T(0);
}

// ---------------------------------------------------------------- host

// Products of up to AR_POSITION_MAX_BUCKETS / 2 numbers below 2^32, little ends first.
struct Whole {
    uint32_t word[AR_POSITION_MAX_BUCKETS / 2];
    int words = 1;
    Whole() { word[0] = 1; }
    void times(uint32_t by) {
        uint64_t carry = 0;
        for (int i = 0; i < words; ++i) {
            carry += uint64_t(word[i]) * by;
            word[i] = uint32_t(carry);
            carry >>= 32;
        }
        if (carry) word[words++] = uint32_t(carry);
    }
    bool at_least(const Whole& o) const {
        if (words != o.words) return words > o.words;
        for (int i = words; i-- > 0;)
            if (word[i] != o.word[i]) return word[i] > o.word[i];
        return true;
    }
};

// Where far bucket ones + m begins: the least n with (n / ones)^q >= (most / ones)^m,
// q = side - ones.  The powers of the root are within 3e-14 of their value; where one lies so
// near a whole number that this may decide wrongly, whole numbers decide.
Borders borders_of(int32_t buckets, int32_t most, bool causal) {
    Borders s{};
    s.causal = causal;
    s.side = causal ? buckets : buckets / 2;
    const int32_t ones = s.side / 2, q = s.side - ones;
    for (int32_t b = 0; b <= ones; ++b) s.at[b] = b;
    const double ratio = std::pow(double(most) / ones, 1.0 / q);
    double v = ones;
    for (int32_t m = 1; m < q; ++m) {
        v *= ratio;
        int64_t n = int64_t(std::ceil(v));
        const int64_t near = int64_t(v + 0.5);
        if (std::fabs(v - double(near)) <= 1e-12 * v) {
            Whole left, right;
            for (int32_t i = 0; i < q; ++i) left.times(uint32_t(near));
            for (int32_t i = 0; i < q; ++i) right.times(uint32_t(i < m ? most : ones));
            n = left.at_least(right) ? near : near + 1;
        }
        s.at[ones + m] = int32_t(std::min<int64_t>(n, most));
    }
    return s;
}

template <class T> constexpr int width_of() { return 64 * Num<T>::VEC; }

BiasShape shape_of(int64_t H, int64_t Q, int64_t K, int64_t offset, int64_t rows, int width) {
    BiasShape s{H, Q, K, offset, rows, 0, 0};
    s.row_tiles = ceil_div(Q, rows);
    s.chunks = ceil_div(K, width);
    return s;
}

// How a gradient is shared out: as many rows a wavefront as leave two wavefronts for each
// of the card's 1024 SIMDs, but two steps; a block's side by side along long rows, below each
// other in many, or else in other batches; and few batches a block, whose sums run on.  (Four
// wavefronts a SIMD: 32 x 1024 x 1024 bf16 20.1 us a call, two 18.8.  4 x 16 x 2048 x 2048
// bf16: side by side 86 us, below each other 100.  3 x 5 x 509 x 1021 f32 with 64 rows a
// wavefront 23, with 8 14.)
GradArgs split_of(int64_t B, int64_t H, int64_t Q, int64_t K, int width) {
    GradArgs a{};
    a.B = B;
    const int64_t least = width / 32, chunks = ceil_div(K, width);
    // A head in one block, without a join, where a lane gets at most 256 elements: 8 x 128 x
    // 128 bf16 10.3 us a call against 15.4, f32 9.8 and 15.1, 8 x 256 x 256 f32 9.9 and 14.5;
    // with twice as many in bf16 14.3 and 15.1, with four times 22 and 15.  256 of f32 rows that
    // end inside a wavefront's columns are the longest: a call as long as with the join, 8 x 250 x
    // 250 12.6 and 14.6, 8 x 8 x 32 x 32 14.9 and 14.4, but in a graph 12.2 and 8.7, 14.5 and 8.5.
    for (int64_t rows = least; rows <= kGradRows; rows *= 2) {
        a.across = chunks > 1 ? 4 : 1;
        a.down = a.across == 1 && Q > rows ? 4 : 1;
        a.batches = B;
        a.splits = 1;
        a.rows = int32_t(rows);
        if (chunks <= a.across && Q <= rows * a.down &&
            ceil_div(B * a.across * a.down, kWaves) * rows * (width / 64) <= 256)
            return a;
    }
    int64_t rows = kGradRows;
    while (rows > least && (rows >= 2 * Q || B * H * chunks * ceil_div(Q, rows) < 2048)) rows /= 2;
    a.rows = int32_t(rows);
    a.across = chunks >= 3 ? 4 : 1;
    a.down = a.across == 1 && Q > rows ? 4 : 1;
    const int64_t alone = kWaves / (a.across * a.down);     // batches at a time
    const int64_t blocks = H * ceil_div(chunks, a.across) * ceil_div(Q, rows * a.down);
    const int64_t splits = std::max(ceil_div(2048, blocks), ceil_div(B, 8));
    a.batches = ceil_div(B, std::max<int64_t>(1, std::min(ceil_div(B, alone), splits)));
    a.splits = ceil_div(B, a.batches);
    return a;
}
int64_t slots_of(const BiasShape& s, const GradArgs& a) { return s.row_tiles * s.chunks * a.splits; }

ar_status check_bias(int32_t buckets, int32_t most, int32_t causal, int64_t B, int64_t H, int64_t Q,
                     int64_t K, int64_t offset) {
    AR_TRY(check_extent("B", B));
    AR_TRY(check_extent("H", H));
    AR_TRY(check_extent("Q", Q));
    AR_TRY(check_extent("K", K));
    if (double(B) * double(H) * double(Q) * double(K) > 4e18)
        return fail(AR_ERR_UNSUPPORTED, "the sizes' product is beyond 2^62");
    if (buckets > AR_POSITION_MAX_BUCKETS)
        return fail(AR_ERR_UNSUPPORTED, "buckets is at most AR_POSITION_MAX_BUCKETS");
    if (buckets < (causal ? 2 : 4) || (!causal && buckets % 2))
        return fail(AR_ERR_INVALID_ARG, "buckets is at least 2, or, of two sides, even and at least 4");
    if (most <= (causal ? buckets : buckets / 2) / 2)
        return fail(AR_ERR_INVALID_ARG, "max_distance is above the distances with buckets of their own");
    if (offset > (int64_t(1) << 62) || offset < -(int64_t(1) << 62))
        return fail(AR_ERR_INVALID_ARG, "offset is beyond 2^62");
    return AR_OK;
}

// A tensor of batches, heads and rows, as one matrix row that spans it: its elements
// from the first to the last.
ar_status check_span(const char* name, const void* p, int32_t es, int64_t B, int64_t sb, int64_t H,
                     int64_t sh, int64_t Q, int64_t sq, int64_t K, int64_t* span) {
    *span = 0;
    if (B == 0 || H == 0 || Q == 0 || K == 0) return AR_OK;
    const std::string what = name;
    if (!p) return fail(AR_ERR_INVALID_ARG, what + " is NULL");
    if (reinterpret_cast<uintptr_t>(p) % uintptr_t(es))
        return fail(AR_ERR_INVALID_ARG, what + " is not aligned to its elements");
    int64_t most = K, at = 0;
    for (const auto& [n, s] : {std::pair<int64_t, int64_t>{B, sb}, {H, sh}, {Q, sq}}) {
        if (s < 0) return fail(AR_ERR_INVALID_ARG, what + ": a stride is negative");
        if (__builtin_mul_overflow(n - 1, s, &at) || __builtin_add_overflow(most, at, &most))
            return fail(AR_ERR_INVALID_ARG, what + ": its last element's offset overflows");
    }
    if (most > INT64_MAX / 16) return fail(AR_ERR_INVALID_ARG, what + ": its last element's offset overflows");
    *span = most;
    return AR_OK;
}

}  // namespace
}  // namespace arp

using namespace arp;

AR_EXPORT ar_status ar_position_bias(int32_t dtype, int32_t buckets, int32_t max_distance,
                                     int32_t causal, int64_t H, int64_t Q, int64_t K, int64_t offset,
                                     const void* table, int64_t table_stride, void* out,
                                     int64_t head_stride, int64_t row_stride, void* stream) try {
    clear_error();
    int32_t es = 0;
    int64_t span = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_bias(buckets, max_distance, causal, 1, H, Q, K, offset));
    const MatArg mt{"table", table, buckets, H, table_stride, es};
    AR_TRY(check_matrix(mt));
    AR_TRY(check_span("out", out, es, 1, 0, H, head_stride, Q, row_stride, K, &span));
    if (span == 0) return AR_OK;
    // rows within a head, or heads within a row: no element is another's
    const auto within = [K](int64_t n, int64_t inner, int64_t m, int64_t outer) {
        return (n == 1 || inner >= K) &&
               (m == 1 || (outer >= K && (n == 1 || (outer - K) / inner >= n - 1)));
    };
    if (!within(Q, row_stride, H, head_stride) && !within(H, head_stride, Q, row_stride))
        return fail(AR_ERR_INVALID_ARG, "out: its heads or rows overlap by their strides");
    AR_TRY(check_apart(MatArg{"out", out, 1, span, span, es}, mt));
    const Borders borders = borders_of(buckets, max_distance, causal != 0);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        const int side = bias_side(Q, K, width_of<T>());
        const BiasShape s = shape_of(H, Q, K, offset, kWaves / side * kBiasRows, side * width_of<T>());
        const int64_t patches = H * s.row_tiles * s.chunks;
        hipLaunchKernelGGL((bias_kernel<T>), dim3(unsigned(std::min<int64_t>(patches, 1 << 20))),
                           dim3(kBlock), 0, static_cast<hipStream_t>(stream), s, borders,
                           static_cast<const T*>(table), table_stride, buckets, static_cast<T*>(out),
                           head_stride, row_stride, patches, side);
        return launch_status("position bias");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}

static ar_status grad_need(int32_t dtype, int32_t buckets, int64_t B, int64_t H, int64_t Q, int64_t K,
                           BiasShape* s, GradArgs* a, int64_t* bytes) {
    *bytes = 0;
    if (B == 0 || H == 0 || Q == 0 || K == 0) return AR_OK;
    const int width = dtype == AR_F32 ? width_of<float>() : width_of<uint16_t>();
    *a = split_of(B, H, Q, K, width);
    *s = shape_of(H, Q, K, 0, a->down * a->rows, a->across * width);
    int64_t parts = 0;
    if (__builtin_mul_overflow(slots_of(*s, *a), H * buckets * 4, &parts))
        return fail(AR_ERR_UNSUPPORTED, "the sizes' product is beyond 2^63");
    if (slots_of(*s, *a) > 1) *bytes = round_up(parts, 16);
    return AR_OK;
}

AR_EXPORT ar_status ar_position_bias_grad_workspace(int32_t dtype, int32_t buckets, int64_t B, int64_t H,
                                                    int64_t Q, int64_t K, int64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_bias(buckets, INT32_MAX, 1, B, H, Q, K, 0));
    BiasShape s{};
    GradArgs a{};
    int64_t need = 0;
    AR_TRY(grad_need(dtype, buckets, B, H, Q, K, &s, &a, &need));
    *bytes = need;
    return AR_OK;
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_position_bias_grad(int32_t dtype, int32_t buckets, int32_t max_distance,
                                          int32_t causal, int64_t B, int64_t H, int64_t Q, int64_t K,
                                          int64_t offset, const void* dbias, int64_t batch_stride,
                                          int64_t head_stride, int64_t row_stride, int32_t accumulate,
                                          void* dtable, int64_t table_stride, void* workspace,
                                          int64_t workspace_bytes, void* stream) try {
    clear_error();
    int32_t es = 0;
    int64_t span = 0, need = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_bias(buckets, max_distance, causal, B, H, Q, K, offset));
    const MatArg mt{"dtable", dtable, buckets, H, table_stride, es};
    AR_TRY(check_matrix(mt));
    AR_TRY(check_span("dbias", dbias, es, B, batch_stride, H, head_stride, Q, row_stride, K, &span));
    BiasShape s{};
    GradArgs a{};
    AR_TRY(grad_need(dtype, buckets, B, H, Q, K, &s, &a, &need));
    AR_TRY(check_workspace(workspace, workspace_bytes, need));
    const MatArg md{"dbias", dbias, span ? 1 : 0, span, span, es},
        mw{"the workspace", workspace, 1, need, need, 1};
    AR_TRY(check_apart(mt, md));
    AR_TRY(check_apart(mw, md));
    AR_TRY(check_apart(mw, mt));
    if (H == 0) return AR_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        T* const to = static_cast<T*>(dtable);
        const auto grid = [](int64_t n, int64_t most) { return dim3(unsigned(std::min(n, most))); };
        if (span == 0) {
            if (!accumulate)
                hipLaunchKernelGGL((table_zero_kernel<T>), grid(ceil_div(H * buckets, kBlock), 1 << 16),
                                   dim3(kBlock), 0, st, H, buckets, to, table_stride);
            return launch_status("position bias gradient");
        }
        s.offset = offset;
        a.batch_stride = batch_stride;
        a.head_stride = head_stride;
        a.row_stride = row_stride;
        a.span = span;
        const int64_t slots = slots_of(s, a);
        hipLaunchKernelGGL((bias_grad_kernel<T>), grid(H * slots, 1 << 20), dim3(kBlock), 0, st, s,
                           borders_of(buckets, max_distance, causal != 0), a,
                           static_cast<const T*>(dbias), buckets,
                           slots > 1 ? static_cast<float*>(workspace) : nullptr, to, table_stride,
                           accumulate);
        if (slots > 1)
            hipLaunchKernelGGL((bias_join_kernel<T>), grid(ceil_div(H * buckets, kWaves), 1 << 16),
                               dim3(kBlock), 0, st, H, buckets, slots,
                               static_cast<const float*>(workspace), to, table_stride, accumulate);
        return launch_status("position bias gradient");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}
