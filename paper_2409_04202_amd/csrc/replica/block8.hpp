// Activations kept in 8 bits: runs of 32 elements of a row share a power of two
// 2^e, and an element is a whole number times that, between -127 and 127.  e is
// the least for which no number leaves that range, at least -126 and at most 121.
//
// A power of two makes all of it exact but the one rounding: x 2^-e and the number
// times 2^e are exact in fp32, and since a number has 7 bits its value is one of
// bf16 too, so that what is fetched again can be a matrix instruction's operand as
// it is.  The error is at most 2^(e-1), that is 2^-7 of the run's largest element
// (1/127.5 at the worst place of that element between two powers of two); 33 bytes
// hold what takes 64 in bf16.
//
// A row is its numbers, in whole runs (zeros behind the row's end), then a byte a
// run, e + 127, or 255 for a run that holds a NaN or an infinity and reads as NaN.
// Rows lie at 16 bytes, so a lane writes and reads 16 numbers at once.
#pragma once

#include <algorithm>

#include "replica.hpp"

namespace arp {

constexpr int kRun = AR_BLOCK8_RUN;  // elements that share a power of two

__host__ __device__ inline int64_t runs_of(int64_t width) { return (width + kRun - 1) / kRun; }

// Bytes of a row.
inline int64_t block8_row(int64_t width) { return round_up(runs_of(width) * (kRun + 1), 16); }

// AR_OK, or the reason why rows of 8 bits cannot lie there.
ar_status check_block8(const char* name, const void* p, int64_t rows, int64_t width, int64_t stride);

// The largest magnitude of some elements, as bits: a NaN's are above an
// infinity's, and are kept where a maximum of floats would drop them.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

// The run's byte from its largest magnitude 1.f 2^(E - 127).  With e = E - 133 the
// largest number is 1.f 2^6, which rounds to 128 from 127.5 on, where 1.f's
// fraction is 0x7F0000 or more: adding 0x10000 then carries into the exponent.
__device__ __forceinline__ uint32_t run_byte(uint32_t top) {
    const int e = int((top + 0x10000u) >> 23) - 6;
    return top >= 0x7F800000u ? 255u : uint32_t(e < 1 ? 1 : e > 248 ? 248 : e);
}

// 2^-e of a run's byte; zero for a run of NaN, whose numbers are zeros.
__device__ __forceinline__ float run_inverse(uint32_t byte) {
    return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23);
}
__device__ __forceinline__ float run_scale(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte << 23);
}

// Four numbers.  Adding 1.5 2^23 rounds to whole numbers, ties to even, and leaves
// them in the sum's low bits.  (A limit is met where e is at its upper bound.  The
// maximum of a NaN, an infinity times zero, and a limit is the limit: zeroed.)
__device__ __forceinline__ uint32_t four_numbers(const float* x, float inverse) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float v = fminf(fmaxf(x[i] * inverse, -127.0f), 127.0f);
        w[i] = __float_as_uint(v + 12582912.0f);
    }
    const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0C0C0400u),
                   hi = __builtin_amdgcn_perm(w[3], w[2], 0x04000C0Cu);
    return inverse == 0.0f ? 0u : lo | hi;
}

// The values of four numbers.
__device__ __forceinline__ void four_values(uint32_t w, float scale, float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = float(int32_t(w << (24 - 8 * i)) >> 24) * scale;
}

// ------------------------------------------------- passes over rows of runs

// The work in strips of 256 units of 8 or 16 elements, a lane's: `1 << log` units of a
// row, `chunks` of those to a row, and as many rows as the 256 lanes have left.  No lane
// divides to find its place.
struct Cover {
    int log;
    int64_t chunks, strips;
};
inline Cover cover(int64_t M, int64_t N, int unit) {
    const int64_t units = kRun / unit * runs_of(N);
    int log = unit == 8 ? 2 : 1;
    while (log < 8 && (int64_t(1) << log) < units) ++log;
    const int64_t chunks = ceil_div(units, int64_t(1) << log);
    return {log, chunks, chunks * ceil_div(M, int64_t(1) << (8 - log))};
}
inline dim3 cover_grid(const Cover& c, int strips) {
    return dim3(unsigned(std::min<int64_t>(ceil_div(c.strips, strips), 1 << 22)));
}

struct Place {
    int64_t row, col;
};
template <int UNIT>
__device__ __forceinline__ Place place(int64_t strip, const Cover& c) {
    const int64_t rows = quotient(strip, c.chunks), chunk = strip - rows * c.chunks;
    return {(rows << (8 - c.log)) + (threadIdx.x >> c.log),
            ((chunk << c.log) + (threadIdx.x & ((1u << c.log) - 1))) * UNIT};
}

}  // namespace arp
