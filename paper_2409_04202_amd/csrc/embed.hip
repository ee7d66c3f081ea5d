// Embedding lookup and its gradient.
//
// Lookup: out[t, :] = scale * table[ids[t], :].  Bound by memory: a row read
// and a row written a token.  A wavefront moves 64 16-byte vectors of a row.
//
// Gradient: dtable[v, :] = scale * sum of dout[t, :] over ids[t] = v.  The
// tokens are sorted by id, stably, so that the tokens of one row are adjacent
// and in increasing order; each row's sum is then one fold, with no atomics
// and one association: runs of kRun tokens, then the runs' sums in order.
#include <algorithm>

#include "replica.hpp"

namespace arp {
namespace {

constexpr int kRun = AR_EMBED_RUN;

// ------------------------------------------------------------- lookup

template <class T>
__global__ __launch_bounds__(256) void lookup_kernel(const T* table, int64_t table_stride,
                                                     const int64_t* ids, int64_t V, int64_t D,
                                                     int64_t rows, float scale, T* out,
                                                     int64_t out_stride) {
    constexpr int VEC = Num<T>::VEC;
    const int64_t slices = (D + 64 * VEC - 1) / (64 * VEC);  // of a row, one a wavefront
    const int64_t units = rows * slices;
    const int lane = threadIdx.x & 63;
    for (int64_t u = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6); u < units;
         u += int64_t(gridDim.x) * 4) {
        const int64_t t = u / slices, at = (u % slices) * 64 * VEC + int64_t(lane) * VEC;
        if (at >= D) continue;
        const int64_t id = ids[t];
        const bool is = id >= 0 && id < V;
        const T* src = table + (is ? id : 0) * table_stride + at;
        T* dst = out + t * out_stride + at;
        const int n = int(D - at < VEC ? D - at : VEC);
        u32x4 v = u32x4{0, 0, 0, 0};
        if (is) {
            float f[VEC];
            Num<T>::unpack(n == VEC ? load_vec(src) : load_part(src, n), f);
            for (int i = 0; i < VEC; ++i) f[i] *= scale;
            v = Num<T>::pack(f);
        }
        if (n == VEC) store_vec(dst, v);
        else store_part(dst, v, n);
    }
}

// --------------------------------------------------------------- sort
//
// Stable counting sort of the tokens by id, 8 bits a pass, lowest first.  A
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
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t* hist, int64_t n) {
    __shared__ uint32_t wave[16];
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

// --------------------------------------------------------------- fold

template <class T>
__global__ __launch_bounds__(256) void zero_kernel(T* m, int64_t rows, int64_t cols,
                                                   int64_t stride) {
    constexpr int VEC = Num<T>::VEC;
    const int64_t slices = (cols + 64 * VEC - 1) / (64 * VEC), units = rows * slices;
    for (int64_t u = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6); u < units;
         u += int64_t(gridDim.x) * 4) {
        const int64_t at = (u % slices) * 64 * VEC + int64_t(threadIdx.x & 63) * VEC;
        if (at >= cols) continue;
        T* dst = m + (u / slices) * stride + at;
        if (cols - at >= VEC) store_vec(dst, u32x4{0, 0, 0, 0});
        else store_part(dst, u32x4{0, 0, 0, 0}, int(cols - at));
    }
}

struct FoldArgs {
    const uint32_t* key;  // sorted ids, T of them, V where there is no token
    const uint32_t* tok;  // their tokens
    int64_t V, D, T;
    int64_t dout_stride, dtable_stride;
    float scale;
    int accumulate;
    // fp32 sums of runs of rows with more than kRun tokens, D apart: a full
    // run that starts at sorted place i is at i / kRun of `full`, the run of
    // fewer tokens that ends the row at (i - kRun) / kRun of `tail` (its
    // place less a run is where a full run of the row starts; two full runs
    // are at least kRun apart).
    float* full;
    float* tail;
};

template <class T>
__device__ __forceinline__ void finish_row(const FoldArgs& a, T* dtable, int64_t v, int64_t at,
                                           const float* sum) {
    constexpr int VEC = Num<T>::VEC;
    T* dst = dtable + v * a.dtable_stride + at;
    const int n = int(a.D - at < VEC ? a.D - at : VEC);
    float f[VEC];
    for (int i = 0; i < VEC; ++i) f[i] = sum[i] * a.scale;
    if (a.accumulate) {
        float old[VEC];
        Num<T>::unpack(n == VEC ? load_vec(dst) : load_part(dst, n), old);
        for (int i = 0; i < VEC; ++i) f[i] += old[i];
    }
    if (n == VEC) store_vec(dst, Num<T>::pack(f));
    else store_part(dst, Num<T>::pack(f), n);
}

// The first sorted place whose key is above (or, with `from`, not below) k.
__device__ __forceinline__ int64_t key_bound(const uint32_t* key, int64_t lo, int64_t hi,
                                             uint32_t k, bool from) {
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (key[mid] > k || (from && key[mid] == k)) hi = mid;
        else lo = mid + 1;
    }
    return lo;
}

// One wavefront a (run, slice of 64 vectors of the row).
template <class T>
__global__ __launch_bounds__(256) void fold_kernel(FoldArgs a, const T* dout, T* dtable) {
    constexpr int VEC = Num<T>::VEC;
    const int64_t slices = (a.D + 64 * VEC - 1) / (64 * VEC), units = a.T * slices;
    for (int64_t u = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6); u < units;
         u += int64_t(gridDim.x) * 4) {
        const int64_t i = u / slices, at = (u % slices) * 64 * VEC + int64_t(threadIdx.x & 63) * VEC;
        const uint32_t v = a.key[i];
        if (v >= a.V) continue;
        bool first = i == 0 || a.key[i - 1] != v;
        if (!first) {  // a later run of the row, or no run's start
            if (i < kRun || a.key[i - kRun] != v) continue;
            const int64_t start = key_bound(a.key, 0, i, v, true);
            if ((i - start) % kRun) continue;
        }
        int n = 1;
        while (n < kRun && i + n < a.T && a.key[i + n] == v) ++n;
        if (at >= a.D) continue;
        const int left = int(a.D - at < VEC ? a.D - at : VEC);
        float sum[VEC] = {};
        for (int j = 0; j < n; ++j) {
            const T* src = dout + int64_t(a.tok[i + j]) * a.dout_stride + at;
            float f[VEC];
            Num<T>::unpack(left == VEC ? load_vec(src) : load_part(src, left), f);
            for (int e = 0; e < VEC; ++e) sum[e] += f[e];
        }
        if (first && (i + n >= a.T || a.key[i + n] != v)) {
            finish_row(a, dtable, v, at, sum);
        } else {
            float* dst = (n == kRun ? a.full + i / kRun * a.D : a.tail + (i - kRun) / kRun * a.D) + at;
            for (int e = 0; e < left; ++e) dst[e] = sum[e];
        }
    }
}

// Rows with more than one run: a block a stretch of kRun sorted places, in
// which at most one of them starts.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(FoldArgs a, T* dtable) {
    constexpr int VEC = Num<T>::VEC;
    const int64_t stretches = (a.T + kRun - 1) / kRun;
    for (int64_t w = blockIdx.x; w < stretches; w += gridDim.x) {
        const int lane = threadIdx.x & 63;
        const int64_t i = w * kRun + lane;
        bool starts = false;
        if (lane < kRun && i + kRun < a.T) {
            const uint32_t k = a.key[i];
            starts = k < a.V && a.key[i + kRun] == k && (i == 0 || a.key[i - 1] != k);
        }
        const uint64_t who = __ballot(starts);
        if (!who) continue;
        const int64_t start = w * kRun + __ffsll((unsigned long long)who) - 1;
        const uint32_t v = a.key[start];
        const int64_t end = key_bound(a.key, start, a.T, v, false);
        for (int64_t at = int64_t(threadIdx.x) * VEC; at < a.D; at += 256 * VEC) {
            const int left = int(a.D - at < VEC ? a.D - at : VEC);
            float sum[VEC] = {};
            for (int64_t r = start; r < end; r += kRun) {
                const float* src = (end - r >= kRun ? a.full + r / kRun * a.D
                                                    : a.tail + (r - kRun) / kRun * a.D) + at;
                for (int e = 0; e < left; ++e) sum[e] += src[e];
            }
            finish_row(a, dtable, v, at, sum);
        }
    }
}

struct GradSpace {  // the workspace's parts, in bytes from its start
    int64_t key[2], tok[2], hist, full, tail, end;
    int64_t blocks;
};

GradSpace grad_space(int64_t D, int64_t T) {
    GradSpace g{};
    g.blocks = ceil_div(T, kSortBlock);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at = round_up(at + bytes, 256);
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        g.key[i] = take(4 * T);
        g.tok[i] = take(4 * T);
    }
    g.hist = take(4 * kDigits * g.blocks);
    g.full = take(4 * ceil_div(T, kRun) * D);
    g.tail = take(4 * ceil_div(T, kRun) * D);
    g.end = at;
    return g;
}

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
    const int64_t slices = ceil_div(D, 64 * Num<T>::VEC);
    if (!accumulate) {
        hipLaunchKernelGGL((zero_kernel<T>), dim3(grid_of(ceil_div(V * slices, 4))), dim3(256), 0,
                           st, out, V, D, dtable_stride);
    }
    if (rows > 0) {
        const GradSpace g = grad_space(D, rows);
        uint32_t* key[2] = {reinterpret_cast<uint32_t*>(ws + g.key[0]),
                            reinterpret_cast<uint32_t*>(ws + g.key[1])};
        uint32_t* tok[2] = {reinterpret_cast<uint32_t*>(ws + g.tok[0]),
                            reinterpret_cast<uint32_t*>(ws + g.tok[1])};
        uint32_t* hist = reinterpret_cast<uint32_t*>(ws + g.hist);
        SortSrc src{ids, nullptr, nullptr, V, rows};
        int to = 0;
        for (int shift = 0; (V >> shift) > 0; shift += 8, to ^= 1) {  // keys are 0 .. V
            hipLaunchKernelGGL(sort_count_kernel, dim3(grid_of(g.blocks)), dim3(256), 0, st, src,
                               shift, hist, g.blocks);
            hipLaunchKernelGGL(sort_scan_kernel, dim3(1), dim3(1024), 0, st, hist,
                               kDigits * g.blocks);
            hipLaunchKernelGGL(sort_move_kernel, dim3(grid_of(g.blocks)), dim3(256), 0, st, src,
                               shift, hist, g.blocks, key[to], tok[to]);
            src = SortSrc{nullptr, key[to], tok[to], V, rows};
        }
        const FoldArgs a{src.key, src.tok, V, D, rows, dout_stride, dtable_stride, scale,
                         accumulate, reinterpret_cast<float*>(ws + g.full),
                         reinterpret_cast<float*>(ws + g.tail)};
        hipLaunchKernelGGL((fold_kernel<T>), dim3(grid_of(ceil_div(rows * slices, 4))), dim3(256),
                           0, st, a, static_cast<const T*>(dout), out);
        hipLaunchKernelGGL((join_kernel<T>), dim3(grid_of(ceil_div(rows, kRun))), dim3(256), 0, st,
                           a, out);
    }
    return launch_status("embedding gradient");
}

ar_status check_ids(const int64_t* ids, int64_t T) {
    return check_matrix({"ids", ids, 1, T, T, 8});
}

}  // namespace
}  // namespace arp

using namespace arp;

AR_EXPORT ar_status ar_embed_lookup(int32_t dtype, int64_t V, int64_t D, int64_t T,
                                    const void* table, int64_t table_stride, const int64_t* ids,
                                    float scale, void* out, int64_t out_stride, void* stream) {
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
    if (T == 0 || D == 0) return AR_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == AR_F32 ? run_lookup<float>(V, D, T, table, table_stride, ids, scale, out, out_stride, st)
                           : run_lookup<uint16_t>(V, D, T, table, table_stride, ids, scale, out, out_stride, st);
}

AR_EXPORT ar_status ar_embed_grad_workspace(int64_t V, int64_t D, int64_t T, int64_t* bytes) {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    AR_TRY(check_extent("V", V));
    AR_TRY(check_extent("D", D));
    AR_TRY(check_extent("T", T));
    *bytes = V == 0 || D == 0 || T == 0 ? 0 : grad_space(D, T).end;
    return AR_OK;
}

AR_EXPORT ar_status ar_embed_grad(int32_t dtype, int64_t V, int64_t D, int64_t T, const void* dout,
                                  int64_t dout_stride, const int64_t* ids, float scale,
                                  int32_t accumulate, void* dtable, int64_t dtable_stride,
                                  void* workspace, int64_t workspace_bytes, void* stream) {
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
    if (V == 0 || D == 0) return AR_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    return dtype == AR_F32 ? run_grad<float>(V, D, T, dout, dout_stride, ids, scale, accumulate, dtable, dtable_stride, ws, st)
                           : run_grad<uint16_t>(V, D, T, dout, dout_stride, ids, scale, accumulate, dtable, dtable_stride, ws, st);
}
