// Activations kept in 8 bits between a forward and a backward pass, and fetched
// again.
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

// 16 elements a lane, half of a run, whose numbers are one vector.  Bound by memory: 8192 x
// 16384 bf16 84 us, 4.9 TB/s.  (8 elements a lane, or stores past the caches: 89.)  Of fp32 a
// load takes 16 of every 64 bytes: 8192 x 8192 78 us, 4.3 TB/s.
template <class T>
__global__ __launch_bounds__(256) void keep_kernel(int64_t M, int64_t N, Cover c, const T* x,
                                                   int64_t x_stride, uint8_t* kept, int64_t stride) {
    constexpr int VEC = Num<T>::VEC, UNIT = 16;
    const int64_t runs = runs_of(N);
    for (int64_t s = blockIdx.x; s < c.strips; s += gridDim.x) {
        const Place at = place<UNIT>(s, c);
        if (at.row >= M || at.col >= runs * kRun) continue;  // (pairs of lanes together)
        const T* const from = x + at.row * x_stride + at.col;
        const int64_t left = N - at.col;
        float v[UNIT];
        u32x4 w[UNIT / VEC];
        if (left >= UNIT) {
#pragma unroll
            for (int i = 0; i < UNIT / VEC; ++i) w[i] = load_vec(from + i * VEC);
        } else {
#pragma unroll
            for (int i = 0; i < UNIT / VEC; ++i) {
                w[i] = u32x4{0, 0, 0, 0};
                if (left >= (i + 1) * VEC) w[i] = load_vec(from + i * VEC);
                else if (left > i * VEC) w[i] = load_part(from + i * VEC, int(left - i * VEC));
            }
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < UNIT / VEC; ++i) Num<T>::unpack(w[i], v + i * VEC);
#pragma unroll
        for (int i = 0; i < UNIT; ++i) top = max(top, magnitude(v[i]));
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

// 8 elements a lane, so that a wavefront's every store of bf16 is to adjacent bytes, and two
// strips at a time, whose loads are in flight together.  Bound by memory: 8192 x 16384 bf16 63
// us, 6.5 TB/s (16 elements a lane 71).  Of fp32 a store takes 16 of every 32 bytes: 8192 x 8192
// 79 us, 4.3 TB/s.
template <class T>
__global__ __launch_bounds__(256) void fetch_kernel(int64_t M, int64_t N, Cover c,
                                                    const uint8_t* kept, int64_t stride, T* x,
                                                    int64_t x_stride) {
    constexpr int VEC = Num<T>::VEC, UNIT = 8;
    const int64_t runs = runs_of(N);
    for (int64_t s = int64_t(blockIdx.x) * 2; s < c.strips; s += int64_t(gridDim.x) * 2) {
        Place at[2];
        uint64_t codes[2];
        uint32_t byte[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            at[h] = place<UNIT>(s + h, c);
            if (s + h >= c.strips || at[h].col >= N) at[h].row = M;
            codes[h] = byte[h] = 0;
            if (at[h].row >= M) continue;
            const uint8_t* const row = kept + at[h].row * stride;
            codes[h] = *(const AR_GLOBAL uint64_t*)(row + at[h].col);
            byte[h] = row[runs * kRun + at[h].col / kRun];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (at[h].row >= M) continue;
            float v[UNIT];
            const float scale = run_scale(byte[h]);
            four_values(uint32_t(codes[h]), scale, v);
            four_values(uint32_t(codes[h] >> 32), scale, v + 4);
            T* const to = x + at[h].row * x_stride + at[h].col;
            const int64_t left = N - at[h].col;
#pragma unroll
            for (int i = 0; i < UNIT; i += VEC) {
                if (left >= i + VEC) store_vec(to + i, Num<T>::pack(v + i));
                else if (left > i) store_part(to + i, Num<T>::pack(v + i), int(left - i));
            }
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
                            const void* kept, int64_t kept_stride) {
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_sizes(M, N));
    const MatArg mx{"x", x, M, N, x_stride, es}, mk{"kept", kept, M, block8_row(N), kept_stride, 1};
    AR_TRY(check_matrix(mx));
    AR_TRY(check_block8("kept", kept, M, N, kept_stride));
    AR_TRY(check_apart(mx, mk));
    return AR_OK;
}

AR_EXPORT ar_status ar_checkpoint_store(int32_t dtype, int64_t M, int64_t N, const void* x,
                                        int64_t x_stride, void* kept, int64_t kept_stride,
                                        void* stream) try {
    clear_error();
    AR_TRY(check_call(dtype, M, N, x, x_stride, kept, kept_stride));
    if (M == 0 || N == 0) return AR_OK;
    const Cover c = cover(M, N, 16);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL((keep_kernel<T>), cover_grid(c, 1), dim3(256), 0,
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
    AR_TRY(check_call(dtype, M, N, x, x_stride, kept, kept_stride));
    if (M == 0 || N == 0) return AR_OK;
    const Cover c = cover(M, N, 8);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL((fetch_kernel<T>), cover_grid(c, 2), dim3(256), 0,
                           static_cast<hipStream_t>(stream), M, N, c,
                           static_cast<const uint8_t*>(kept), kept_stride, static_cast<T*>(x), x_stride);
        return launch_status("checkpoint load");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}
