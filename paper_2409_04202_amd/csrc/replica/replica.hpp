// Shared by the replica operators' translation units (embed.hip, distill.hip,
// glu.hip): argument checks on the host, and the vector and element accesses
// of their kernels.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "../internal.hpp"
#include "../kernels.hpp"

namespace arp {

// ---------------------------------------------------------------- host

constexpr int64_t kMaxExtent = (int64_t(1) << 31) - 1;

struct MatArg {
    const char* name;
    const void* ptr;
    int64_t rows, cols, stride;  // stride in elements
    int32_t esize;
};

// AR_OK, or the reason why the matrix cannot be used (the error is set).
ar_status check_matrix(const MatArg& m);
// AR_OK unless the output shares an element with the other matrix.
ar_status check_apart(const MatArg& out, const MatArg& other);
ar_status check_dtype(const char* what, int32_t dtype, int32_t* esize);
ar_status check_extent(const char* what, int64_t v);
ar_status check_workspace(const void* ws, int64_t have, int64_t need);
ar_status launch_status(const char* what);

// The status of what a C entry has caught.  The entries' bodies are function try
// blocks: the text of an error takes memory, and may throw.
ar_status thrown() noexcept;

inline int64_t round_up(int64_t v, int64_t unit) { return (v + unit - 1) / unit * unit; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

#define AR_TRY(call)                          \
    do {                                      \
        const ar_status s_ = (call);          \
        if (s_ != AR_OK) return s_;           \
    } while (0)

// -------------------------------------------------------------- device

// Vectors of 16 bytes at the element's alignment: rows start at any element,
// and global_load_dwordx4 takes any address, so only a row's tail needs
// element-wise care.
typedef u32x4 u32x4_e4 __attribute__((aligned(4)));
typedef u32x4 u32x4_e2 __attribute__((aligned(2)));

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ uint32_t scalar(uint32_t v) {
    return uint32_t(__builtin_amdgcn_readfirstlane(int(v)));
}

template <class T> struct Num;
template <> struct Num<float> {
    static constexpr int VEC = 4;  // elements of a 16-byte vector
    using V = AR_GLOBAL u32x4_e4;
    static __device__ __forceinline__ float up(float x) { return x; }
    static __device__ __forceinline__ float down(float x) { return x; }
    static __device__ __forceinline__ void unpack(const u32x4 x, float* f) {
        for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(x[i]);
    }
    static __device__ __forceinline__ u32x4 pack(const float* f) {
        return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                     __float_as_uint(f[3])};
    }
};
template <> struct Num<uint16_t> {  // bf16 bits
    static constexpr int VEC = 8;
    using V = AR_GLOBAL u32x4_e2;
    static __device__ __forceinline__ float up(uint16_t x) {
        return __uint_as_float(uint32_t(x) << 16);
    }
    static __device__ __forceinline__ uint16_t down(float x) {
        return uint16_t(bf16_pack(x, 0.0f));
    }
    static __device__ __forceinline__ void unpack(const u32x4 x, float* f) {
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = bf16_lo(x[i]);
            f[2 * i + 1] = bf16_hi(x[i]);
        }
    }
    static __device__ __forceinline__ u32x4 pack(const float* f) {
        return u32x4{bf16_pack(f[0], f[1]), bf16_pack(f[2], f[3]), bf16_pack(f[4], f[5]),
                     bf16_pack(f[6], f[7])};
    }
};

template <class T>
__device__ __forceinline__ u32x4 load_vec(const T* p) {
    return *(const typename Num<T>::V*)p;
}
template <class T>
__device__ __forceinline__ void store_vec(T* p, const u32x4 v) {
    *(typename Num<T>::V*)p = v;
}
// The first n < VEC elements of a vector; the others read as zero, and are
// not stored.
template <class T>
__device__ __forceinline__ u32x4 load_part(const T* p, int n) {
    float f[Num<T>::VEC];
    for (int i = 0; i < Num<T>::VEC; ++i)
        f[i] = i < n ? Num<T>::up(((const AR_GLOBAL T*)p)[i]) : 0.0f;
    return Num<T>::pack(f);
}
template <class T>
__device__ __forceinline__ void store_part(T* p, const u32x4 v, int n) {
    float f[Num<T>::VEC];
    Num<T>::unpack(v, f);
    for (int i = 0; i < Num<T>::VEC; ++i)
        if (i < n) ((AR_GLOBAL T*)p)[i] = Num<T>::down(f[i]);
}

// Reductions over a wavefront, in the register file: after four shifts within
// the rows of 16 lanes and two broadcasts from row to row lane 63 has them all.
template <int CTRL, int ROWS>
__device__ __forceinline__ float from_lane(float v, float none) {
    return __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(
        int(__float_as_uint(none)), int(__float_as_uint(v)), CTRL, ROWS, 0xF, false)));
}
template <class F>
__device__ __forceinline__ float wave_reduce(float v, float none, F&& f) {
    v = f(v, from_lane<0x111, 0xF>(v, none));
    v = f(v, from_lane<0x112, 0xF>(v, none));
    v = f(v, from_lane<0x114, 0xF>(v, none));
    v = f(v, from_lane<0x118, 0xF>(v, none));
    v = f(v, from_lane<0x142, 0xA>(v, none));
    v = f(v, from_lane<0x143, 0xC>(v, none));
    return __uint_as_float(uint32_t(__builtin_amdgcn_readlane(int(__float_as_uint(v)), 63)));
}
__device__ __forceinline__ float wave_sum(float v) {
    return wave_reduce(v, 0.0f, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
    return wave_reduce(v, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace arp
