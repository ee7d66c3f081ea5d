// Activations kept in 8 bits between a forward and a backward pass, and fetched
// again.
#include <algorithm>

#include "block8.hpp"

namespace arp {

ar_status check_block8(const char* name, const void* p, int64_t rows, int64_t width, int64_t stride) {
    if (rows == 0 || width == 0) return AR_OK;
    const std::string what = name;
    if (!p) return fail(AR_ERR_INVALID_ARG, what + " is NULL");
    if (reinterpret_cast<uintptr_t>(p) % 16 || stride % 16)
        return fail(AR_ERR_INVALID_ARG, what + ": rows of 8 bits lie at 16 bytes");
    if (stride < block8_row(width))
        return fail(AR_ERR_INVALID_ARG, what + ": the row stride is below the row's bytes");
    if (stride > (INT64_MAX - stride) / rows)
        return fail(AR_ERR_INVALID_ARG, what + ": stride * rows overflows");
    return AR_OK;
}

namespace {

constexpr int kLane = 16;  // elements a lane holds, half a run

// Lanes of a row, as a power of two, and how many blocks side by side a row takes.
struct Cover {
    int log;
    int64_t chunks, blocks;
};
Cover cover(int64_t M, int64_t N) {
    const int64_t lanes = 2 * runs_of(N);
    int log = 1;
    while (log < 8 && (int64_t(1) << log) < lanes) ++log;
    const int64_t chunks = ceil_div(lanes, int64_t(1) << log);
    return {log, chunks, chunks * ceil_div(M, int64_t(1) << (8 - log))};
}
dim3 grid_of(const Cover& c) { return dim3(unsigned(std::min<int64_t>(c.blocks, 1 << 22))); }

// A block's 256 lanes lie over `1 << log` lanes of a row and as many rows as that
// leaves, so no lane divides to find its place.
struct Place {
    int64_t row, col;
};
__device__ __forceinline__ Place place(int64_t block, int log, int64_t chunks) {
    const int64_t rows = block / chunks, chunk = block % chunks;
    return {(rows << (8 - log)) + (threadIdx.x >> log),
            ((chunk << log) + (threadIdx.x & ((1u << log) - 1))) * kLane};
}

// Bound by memory.
template <class T>
__global__ __launch_bounds__(256) void keep_kernel(int64_t M, int64_t N, Cover c, const T* x,
                                                   int64_t x_stride, uint8_t* kept, int64_t stride) {
  constexpr int VEC = Num<T>::VEC;
  const int64_t runs = runs_of(N);
  for (int64_t b = blockIdx.x; b < c.blocks; b += gridDim.x) {
    const Place at = place(b, c.log, c.chunks);
    if (at.row >= M || at.col >= runs * kRun) continue;  // (pairs of lanes together)
    const T* const from = x + at.row * x_stride + at.col;
    const int64_t left = N - at.col;
    float v[kLane];
    if (left >= kLane) {
        u32x4 w[kLane / VEC];
#pragma unroll
        for (int i = 0; i < kLane / VEC; ++i) w[i] = load_vec(from + i * VEC);
#pragma unroll
        for (int i = 0; i < kLane / VEC; ++i) Num<T>::unpack(w[i], v + i * VEC);
    } else {
#pragma unroll
        for (int i = 0; i < kLane; ++i) v[i] = i < left ? Num<T>::up(from[i]) : 0.0f;
    }
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kLane; ++i) top = max(top, magnitude(v[i]));
    top = max(top, uint32_t(__builtin_amdgcn_mov_dpp(int(top), 0xB1, 0xF, 0xF, true)));  // the pair's
    const uint32_t byte = run_byte(top);
    const float inverse = run_inverse(byte);
    uint8_t* const row = kept + at.row * stride;
    u32x4 codes;
#pragma unroll
    for (int i = 0; i < 4; ++i) codes[i] = four_numbers(v + 4 * i, inverse);
    *(AR_GLOBAL u32x4*)(row + at.col) = codes;
    if ((threadIdx.x & 1) == 0) row[runs * kRun + at.col / kRun] = uint8_t(byte);
  }
}

template <class T>
__global__ __launch_bounds__(256) void fetch_kernel(int64_t M, int64_t N, Cover c,
                                                    const uint8_t* kept, int64_t stride, T* x,
                                                    int64_t x_stride) {
  constexpr int VEC = Num<T>::VEC;
  for (int64_t b = blockIdx.x; b < c.blocks; b += gridDim.x) {
    const Place at = place(b, c.log, c.chunks);
    if (at.row >= M || at.col >= N) continue;
    const uint8_t* const row = kept + at.row * stride;
    const u32x4 codes = *(const AR_GLOBAL u32x4*)(row + at.col);
    const float scale = run_scale(row[runs_of(N) * kRun + at.col / kRun]);
    float v[kLane];
#pragma unroll
    for (int i = 0; i < 4; ++i) four_values(codes[i], scale, v + 4 * i);
    T* const to = x + at.row * x_stride + at.col;
    const int64_t left = N - at.col;
    if (left >= kLane) {
#pragma unroll
        for (int i = 0; i < kLane / VEC; ++i) store_vec(to + i * VEC, Num<T>::pack(v + i * VEC));
    } else {
#pragma unroll
        for (int i = 0; i < kLane; ++i)
            if (i < left) to[i] = Num<T>::down(v[i]);
    }
  }
}

ar_status check_sizes(int64_t M, int64_t N) {
    AR_TRY(check_extent("M", M));
    return check_extent("N", N);
}

}  // namespace
}  // namespace arp

using namespace arp;

AR_EXPORT ar_status ar_checkpoint_row(int64_t N, int64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    AR_TRY(check_extent("N", N));
    *bytes = block8_row(N);
    return AR_OK;
} catch (...) {
    return thrown();
}

static ar_status check_call(int32_t dtype, int64_t M, int64_t N, const void* x, int64_t x_stride,
                            const void* kept, int64_t kept_stride, Cover* c) {
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_sizes(M, N));
    const MatArg mx{"x", x, M, N, x_stride, es}, mk{"kept", kept, M, block8_row(N), kept_stride, 1};
    AR_TRY(check_matrix(mx));
    AR_TRY(check_block8("kept", kept, M, N, kept_stride));
    AR_TRY(check_apart(mx, mk));
    *c = cover(M, N);
    return AR_OK;
}

AR_EXPORT ar_status ar_checkpoint_store(int32_t dtype, int64_t M, int64_t N, const void* x,
                                        int64_t x_stride, void* kept, int64_t kept_stride,
                                        void* stream) try {
    clear_error();
    Cover c{};
    AR_TRY(check_call(dtype, M, N, x, x_stride, kept, kept_stride, &c));
    if (M == 0 || N == 0) return AR_OK;
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL((keep_kernel<T>), grid_of(c), dim3(256), 0,
                           static_cast<hipStream_t>(stream), M, N, c,
                           static_cast<const T*>(x), x_stride, static_cast<uint8_t*>(kept), kept_stride);
        return launch_status("checkpoint store");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_checkpoint_load(int32_t dtype, int64_t M, int64_t N, const void* kept,
                                       int64_t kept_stride, void* x, int64_t x_stride,
                                       void* stream) try {
    clear_error();
    Cover c{};
    AR_TRY(check_call(dtype, M, N, x, x_stride, kept, kept_stride, &c));
    if (M == 0 || N == 0) return AR_OK;
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL((fetch_kernel<T>), grid_of(c), dim3(256), 0,
                           static_cast<hipStream_t>(stream), M, N, c,
                           static_cast<const uint8_t*>(kept), kept_stride, static_cast<T*>(x), x_stride);
        return launch_status("checkpoint load");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}
