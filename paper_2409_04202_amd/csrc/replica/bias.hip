// Attention's relative position bias by buckets of distance, and its table's gradient.
//
// The bias depends on j - i alone: along a diagonal of a head's Q x K matrix it is one
// number, and all of a diagonal's gradients go to one bucket.  So a lane owns a vector
// of adjacent diagonals and walks down the rows: the bias is looked up once and stored
// row after row, one element further on in each; the gradients are added in registers,
// and only the diagonals' sums are sorted into buckets.  An element costs its way
// through memory and, in the gradient, one addition.  Rows start at any element, and so
// do the vectors.
//
// Diagonals are counted g = j - i + Q - 1 >= 0; the distance is n = c - g with
// c = offset + Q - 1.
#include <algorithm>
#include <cmath>
#include <type_traits>
#include <vector>

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
    int64_t H, Q, K, c;
    int64_t rows, row_tiles, chunks;  // rows of a tile; chunks of diagonals a tile has
};

// The bucket of distance n; behind the query in buckets of their own, or (causal) none.
__device__ __forceinline__ int bucket_of(const Borders& s, int64_t n) {
    if (s.causal && n < 0) return -1;
    const int64_t d = n < 0 ? -n : n;
    int lo = 0, hi = s.side;  // at[lo] <= d < at[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s.at[mid] <= d) lo = mid;
        else hi = mid;
    }
    return n < 0 ? s.side + lo : lo;
}

// The place of a block: head, rows [i0, i1) and its first diagonal.
struct Patch {
    int64_t h, i0, i1, g0;
};
__device__ __forceinline__ Patch patch_of(const BiasShape& s, int64_t n, int width) {
    const int64_t chunk = n % s.chunks, tile = n / s.chunks % s.row_tiles;
    Patch p;
    p.h = n / s.chunks / s.row_tiles;
    p.i0 = tile * s.rows;
    p.i1 = p.i0 + s.rows < s.Q ? p.i0 + s.rows : s.Q;
    p.g0 = s.Q - p.i1 + chunk * width;
    return p;
}

// Bound by memory: the matrix is written once.
template <class T>
__global__ __launch_bounds__(kBlock) void bias_kernel(BiasShape s, Borders borders, const T* table,
                                                      int64_t table_stride, T* out, int64_t head_stride,
                                                      int64_t row_stride, int64_t patches) {
    constexpr int VEC = Num<T>::VEC, WIDTH = 64 * VEC;
    __shared__ __attribute__((aligned(16))) T value[WIDTH];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6);
    for (int64_t n = blockIdx.x; n < patches; n += gridDim.x) {
        const Patch p = patch_of(s, n, WIDTH);
        for (int x = threadIdx.x; x < WIDTH; x += kBlock) {
            const int b = bucket_of(borders, s.c - (p.g0 + x));
            value[x] = b < 0 ? Num<T>::down(-INFINITY) : table[b * table_stride + p.h];
        }
        __syncthreads();
        const u32x4 v = *(const AR_LDS u32x4*)((AR_LDS T*)value + lane * VEC);
        const int64_t per = (s.rows + kWaves - 1) / kWaves, i0 = p.i0 + wave * per;
        const int64_t i1 = i0 + per < p.i1 ? i0 + per : p.i1;
        int64_t j = p.g0 + lane * VEC + i0 - (s.Q - 1);
        T* to = out + p.h * head_stride + i0 * row_stride + j;
        for (int64_t i = i0; i < i1; ++i, ++j, to += row_stride + 1) {
            if (j >= 0 && j + VEC <= s.K) {
                store_vec(to, v);
            } else if (j > -VEC && j < s.K) {
                float f[VEC];
                Num<T>::unpack(v, f);
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    if (j + e >= 0 && j + e < s.K) ((AR_GLOBAL T*)to)[e] = Num<T>::down(f[e]);
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
};

// The sums of a wavefront's diagonals over rows [i0, i1): EDGE where some of its vectors
// pass a row's ends.  Such a vector is read whole and what lies outside the row is
// left out, where it lies between the tensor's first and last element.
template <class T, bool EDGE>
__device__ __forceinline__ void add_rows(const T* first, const T* end, const T* from, int64_t step,
                                         int64_t rows, int64_t j, int64_t K, float* sum) {
    constexpr int VEC = Num<T>::VEC, DEEP = 8;
    auto add = [&](const u32x4 w, int64_t at) {
        float f[VEC];
        Num<T>::unpack(w, f);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            sum[e] += !EDGE || (at + e >= 0 && at + e < K) ? f[e] : 0.0f;
    };
    auto load = [&](const T* p, int64_t at) {
        if constexpr (!EDGE) return load_vec(p);
        if (at <= -VEC || at >= K) return u32x4{0, 0, 0, 0};
        if (p >= first && p + VEC <= end) return load_vec(p);
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            f[e] = at + e >= 0 && at + e < K ? Num<T>::up(((const AR_GLOBAL T*)p)[e]) : 0.0f;
        return Num<T>::pack(f);
    };
    int64_t i = 0;
    for (; i + DEEP <= rows; i += DEEP, from += DEEP * step) {
        u32x4 w[DEEP];
#pragma unroll
        for (int d = 0; d < DEEP; ++d) w[d] = load(from + d * step, j + i + d);
#pragma unroll
        for (int d = 0; d < DEEP; ++d) add(w[d], j + i + d);
    }
    for (; i < rows; ++i, from += step) add(load(from, j + i), j + i);
}

// A block's sums by bucket, to its slot of `part`, or straight to the table where a
// head has one slot.  Bound by memory: the scores' gradients pass once.
template <class T>
__global__ __launch_bounds__(kBlock) void bias_grad_kernel(BiasShape s, Borders borders, GradArgs a,
                                                           const T* d, int32_t buckets, float* part,
                                                           T* dtable, int64_t table_stride,
                                                           int32_t accumulate) {
    constexpr int VEC = Num<T>::VEC, WIDTH = 64 * VEC;
    __shared__ __attribute__((aligned(16))) float sums[kWaves][WIDTH];
    const int lane = threadIdx.x & 63, wave = scalar(threadIdx.x >> 6);
    const int64_t per_head = s.row_tiles * s.chunks, patches = s.H * per_head;
    for (int64_t n = blockIdx.x; n < patches * a.splits; n += gridDim.x) {
        const int64_t split = n / patches, in = n % patches;
        const Patch p = patch_of(s, in, WIDTH);
        // a tile's rows are shared out to the wavefronts, or, of few rows, the batches
        const bool by_rows = s.rows >= kWaves;
        const int64_t per = by_rows ? (s.rows + kWaves - 1) / kWaves : s.rows;
        const int64_t i0 = p.i0 + (by_rows ? wave * per : 0);
        const int64_t i1 = i0 + per < p.i1 ? i0 + per : p.i1;
        const int64_t b0 = split * a.batches, b1 = b0 + a.batches < a.B ? b0 + a.batches : a.B;
        const int64_t g = p.g0 + lane * VEC, j = g + i0 - (s.Q - 1);
        float sum[VEC] = {};
        const bool seen = !borders.causal || p.g0 <= s.c;
        if (seen && i0 < i1) {
            const bool whole = p.g0 + i0 - (s.Q - 1) >= 0 && p.g0 + WIDTH - 1 + i1 - 1 - (s.Q - 1) < s.K;
            for (int64_t b = b0 + (by_rows ? 0 : wave); b < b1; b += by_rows ? 1 : kWaves) {
                const T* const from = d + b * a.batch_stride + p.h * a.head_stride + i0 * a.row_stride + j;
                if (whole) add_rows<T, false>(d, d + a.span, from, a.row_stride + 1, i1 - i0, j, s.K, sum);
                else add_rows<T, true>(d, d + a.span, from, a.row_stride + 1, i1 - i0, j, s.K, sum);
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            sums[wave][lane * VEC + e] = borders.causal && g + e > s.c ? 0.0f : sum[e];
        __syncthreads();
        for (int b = wave; b < buckets; b += kWaves) {
            // the bucket's distances [near, far) are diagonals (c - far, c - near], or,
            // behind the query, [c + near, c + far)
            const bool behind = b >= borders.side;
            const int m = behind ? b - borders.side : b;
            const int64_t near = borders.at[m];
            int64_t lo = behind ? s.c + (near ? near : 1) : 0, hi = behind ? INT64_MAX : s.c - near + 1;
            if (m + 1 < borders.side) {
                const int64_t far = borders.at[m + 1];
                if (behind) hi = s.c + far;
                else lo = s.c - far + 1;
            } else if (!behind) {
                lo = INT64_MIN;
            }
            lo = lo > p.g0 ? lo - p.g0 : 0;
            hi = hi > p.g0 ? (hi - p.g0 < WIDTH ? hi - p.g0 : WIDTH) : 0;
            float t = 0.0f;
            for (int x = int(lo < WIDTH ? lo : WIDTH) + lane; x < int(hi); x += 64)
                t += (sums[0][x] + sums[1][x]) + (sums[2][x] + sums[3][x]);
            t = wave_sum(t);
            if (lane == 0) {
                if (part) {
                    const int64_t slots = per_head * a.splits;
                    part[(p.h * buckets + b) * slots + split * per_head + in % per_head] = t;
                } else {
                    T* const to = dtable + b * table_stride + p.h;
                    *to = Num<T>::down(accumulate ? t + Num<T>::up(*to) : t);
                }
            }
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

// Whether a >= b, for products of whole numbers: little ends first.
using Whole = std::vector<uint32_t>;
void times(Whole* w, uint32_t by) {
    uint64_t carry = 0;
    for (uint32_t& x : *w) {
        carry += uint64_t(x) * by;
        x = uint32_t(carry);
        carry >>= 32;
    }
    if (carry) w->push_back(uint32_t(carry));
}
bool at_least(const Whole& a, const Whole& b) {
    if (a.size() != b.size()) return a.size() > b.size();
    for (size_t i = a.size(); i-- > 0;)
        if (a[i] != b[i]) return a[i] > b[i];
    return true;
}

// Where far bucket ones + m begins: the least n with (n / ones)^q >= (most / ones)^m,
// q = side - ones.  The root is taken in 64 bits of significand; where it lies so near a
// whole number that this may have decided wrongly, whole numbers decide.
Borders borders_of(int32_t buckets, int32_t most, bool causal) {
    Borders s{};
    s.causal = causal;
    s.side = causal ? buckets : buckets / 2;
    const int32_t ones = s.side / 2, q = s.side - ones;
    for (int32_t b = 0; b <= ones; ++b) s.at[b] = b;
    const long double ratio = powl((long double)most / ones, 1.0L / q);
    long double v = ones;
    for (int32_t m = 1; m < q; ++m) {
        v *= ratio;
        int64_t n = int64_t(ceill(v));
        const int64_t near = int64_t(llroundl(v));
        if (fabsl(v - near) <= 1e-14L * v) {
            Whole left{1}, right{1};
            for (int32_t i = 0; i < q; ++i) times(&left, uint32_t(near));
            for (int32_t i = 0; i < q; ++i) times(&right, uint32_t(i < m ? most : ones));
            n = at_least(left, right) ? near : near + 1;
        }
        s.at[ones + m] = int32_t(std::min<int64_t>(n, most));
    }
    return s;
}

template <class T> constexpr int width_of() { return 64 * Num<T>::VEC; }

BiasShape shape_of(int64_t H, int64_t Q, int64_t K, int64_t offset, int64_t rows, int width) {
    BiasShape s{H, Q, K, offset + Q - 1, std::min(rows, Q), 0, 0};
    s.row_tiles = ceil_div(Q, s.rows);
    s.chunks = ceil_div(K + s.rows - 1, width);
    return s;
}

constexpr int64_t kGradRows = 128, kBiasRows = 64;

// How a gradient's batches are shared out: enough blocks for the card, and few of
// them a block, whose sums run on.
GradArgs split_of(const BiasShape& s, int64_t B) {
    GradArgs a{};
    a.B = B;
    const int64_t patches = s.H * s.row_tiles * s.chunks;
    const int64_t want = std::max(ceil_div(2048, patches), ceil_div(B, 8));
    a.batches = ceil_div(B, std::max<int64_t>(1, std::min(B, want)));
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
        const BiasShape s = shape_of(H, Q, K, offset, kBiasRows, width_of<T>());
        const int64_t patches = H * s.row_tiles * s.chunks;
        hipLaunchKernelGGL((bias_kernel<T>), dim3(unsigned(std::min<int64_t>(patches, 1 << 20))),
                           dim3(kBlock), 0, static_cast<hipStream_t>(stream), s, borders,
                           static_cast<const T*>(table), table_stride, static_cast<T*>(out), head_stride,
                           row_stride, patches);
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
    *s = shape_of(H, Q, K, 0, kGradRows, dtype == AR_F32 ? width_of<float>() : width_of<uint16_t>());
    *a = split_of(*s, B);
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
        s.c = offset + Q - 1;
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
