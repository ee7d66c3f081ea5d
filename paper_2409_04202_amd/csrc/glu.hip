// The gated feed-forward block's products.
#include <algorithm>

#include "replica.hpp"

namespace arp {
namespace {

// a(g) and a'(g).
__device__ __forceinline__ void activate(int act, float g, float* value, float* slope) {
    if (act == AR_ACT_SILU) {
        const float s = 1.0f / (1.0f + expf(-g));
        // at infinities the limits, not inf * 0
        *value = g == -INFINITY ? 0.0f : g * s;
        *slope = s == 0.0f ? 0.0f : s * (1.0f + (s == 1.0f ? 0.0f : g * (1.0f - s)));
    } else {
        const float cdf = 0.5f * erfcf(g * -0.70710678118654752f);
        const float pdf = 0.39894228040143268f * expf(-0.5f * g * g);
        *value = g == -INFINITY ? 0.0f : g * cdf;
        *slope = cdf + (pdf == 0.0f ? 0.0f : g * pdf);
    }
}

// One product, C (rows x cols) = sum over k of A(row, k) B(col, k) over one
// or two segments of k; any element strides.
template <class T>
struct Operand {
    const T* p;
    int64_t row, k;  // strides
    __device__ __forceinline__ float at(int64_t r, int64_t i) const {
        return Num<T>::up(p[r * row + i * k]);
    }
};

constexpr int kTile = 64, kDepth = 16;

// A 64 x 64 tile of A B^T by 256 threads, 4 x 4 each.
template <class T>
__device__ __forceinline__ void tile_product(const Operand<T> A, const Operand<T> B, int64_t r0,
                                             int64_t rows, int64_t c0, int64_t cols, int64_t K,
                                             float (*sa)[kTile + 4], float (*sb)[kTile + 4],
                                             float acc[4][4]) {
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    for (int64_t k0 = 0; k0 < K; k0 += kDepth) {
        __syncthreads();
        for (int e = threadIdx.x; e < kTile * kDepth; e += 256) {
            const int r = e / kDepth, k = e % kDepth;
            sa[k][r] = r0 + r < rows && k0 + k < K ? A.at(r0 + r, k0 + k) : 0.0f;
            sb[k][r] = c0 + r < cols && k0 + k < K ? B.at(c0 + r, k0 + k) : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < kDepth; ++k)
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = fmaf(sa[k][ty * 4 + i], sb[k][tx * 4 + j], acc[i][j]);
    }
}

struct ForwardArgs {
    int64_t M, D, F, x_stride, w_stride, h_stride, saved_stride;
    int act;
};

template <class T>
__global__ __launch_bounds__(256) void forward_kernel(ForwardArgs a, const T* x, const T* wg,
                                                      const T* wu, T* h, T* sg, T* su) {
    __shared__ float sa[kDepth][kTile + 4], sb[kDepth][kTile + 4];
    const int64_t r0 = int64_t(blockIdx.y) * kTile, c0 = int64_t(blockIdx.x) * kTile;
    float g[4][4] = {}, u[4][4] = {};
    const Operand<T> X{x, a.x_stride, 1};
    tile_product<T>(X, {wg, a.w_stride, 1}, r0, a.M, c0, a.F, a.D, sa, sb, g);
    tile_product<T>(X, {wu, a.w_stride, 1}, r0, a.M, c0, a.F, a.D, sa, sb, u);
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 4; ++j) {
            const int64_t r = r0 + (threadIdx.x >> 4) * 4 + i, c = c0 + (threadIdx.x & 15) * 4 + j;
            if (r >= a.M || c >= a.F) continue;
            float value, slope;
            activate(a.act, g[i][j], &value, &slope);
            h[r * a.h_stride + c] = Num<T>::down(value * u[i][j]);
            if (sg) {
                sg[r * a.saved_stride + c] = Num<T>::down(slope * u[i][j]);
                su[r * a.saved_stride + c] = Num<T>::down(value);
            }
        }
    }
}

// dg = dh * saved_gate and du = dh * saved_up.
template <class T>
__global__ __launch_bounds__(256) void factors_kernel(int64_t M, int64_t F, const T* dh,
                                                      int64_t dh_stride, const T* sg, const T* su,
                                                      int64_t saved_stride, T* dg, T* du,
                                                      int64_t stride) {
    for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < M * F;
         e += int64_t(gridDim.x) * 256) {
        const int64_t r = e / F, c = e % F;
        const float d = Num<T>::up(dh[r * dh_stride + c]);
        dg[r * stride + c] = Num<T>::down(d * Num<T>::up(sg[r * saved_stride + c]));
        du[r * stride + c] = Num<T>::down(d * Num<T>::up(su[r * saved_stride + c]));
    }
}

// C = A1 B1^T + A2 B2^T (K2 = 0: the first alone), or C += with accumulate.
template <class T>
__global__ __launch_bounds__(256) void product_kernel(Operand<T> A1, Operand<T> B1, int64_t K1,
                                                      Operand<T> A2, Operand<T> B2, int64_t K2,
                                                      int64_t rows, int64_t cols, int accumulate,
                                                      T* out, int64_t stride) {
    __shared__ float sa[kDepth][kTile + 4], sb[kDepth][kTile + 4];
    const int64_t r0 = int64_t(blockIdx.y) * kTile, c0 = int64_t(blockIdx.x) * kTile;
    float acc[4][4] = {};
    tile_product<T>(A1, B1, r0, rows, c0, cols, K1, sa, sb, acc);
    tile_product<T>(A2, B2, r0, rows, c0, cols, K2, sa, sb, acc);
    for (int i = 0; i < 4; ++i) {
        for (int j = 0; j < 4; ++j) {
            const int64_t r = r0 + (threadIdx.x >> 4) * 4 + i, c = c0 + (threadIdx.x & 15) * 4 + j;
            if (r >= rows || c >= cols) continue;
            T* const at = out + r * stride + c;
            *at = Num<T>::down(accumulate ? Num<T>::up(*at) + acc[i][j] : acc[i][j]);
        }
    }
}

int64_t factor_stride(int64_t F) { return round_up(F, 8); }

dim3 tiles(int64_t rows, int64_t cols) {
    return dim3(unsigned(ceil_div(cols, kTile)), unsigned(ceil_div(rows, kTile)));
}

}  // namespace
}  // namespace arp

using namespace arp;

// Rows and columns of a product: a launch's grid holds this many tiles.
static ar_status check_glu_sizes(int64_t M, int64_t D, int64_t F) {
    AR_TRY(check_extent("M", M));
    AR_TRY(check_extent("D", D));
    AR_TRY(check_extent("F", F));
    for (int64_t v : {M, D, F})
        if (v > AR_GLU_MAX_EXTENT)
            return fail(AR_ERR_UNSUPPORTED, "M, D and F are at most AR_GLU_MAX_EXTENT");
    return AR_OK;
}

AR_EXPORT ar_status ar_glu_workspace(int32_t dtype, int64_t M, int64_t D, int64_t F,
                                     int32_t backward, int64_t* bytes) {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_glu_sizes(M, D, F));
    *bytes = backward ? round_up(2 * M * factor_stride(F) * es, 256) : 0;
    return AR_OK;
}

AR_EXPORT ar_status ar_glu_forward(int32_t dtype, int32_t act, int64_t M, int64_t D, int64_t F,
                                   const void* x, int64_t x_stride, const void* wg, const void* wu,
                                   int64_t w_stride, void* h, int64_t h_stride, void* saved_gate,
                                   void* saved_up, int64_t saved_stride, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
    clear_error();
    int32_t es = 0;
    int64_t need = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    if (act != AR_ACT_SILU && act != AR_ACT_GELU)
        return fail(AR_ERR_INVALID_ARG, "unknown activation");
    AR_TRY(ar_glu_workspace(dtype, M, D, F, 0, &need));
    if (!saved_gate != !saved_up)
        return fail(AR_ERR_INVALID_ARG, "saved_gate and saved_up are given together");
    const int64_t sr = saved_gate ? M : 0;
    const MatArg mx{"x", x, M, D, x_stride, es}, mg{"wg", wg, F, D, w_stride, es},
        mu{"wu", wu, F, D, w_stride, es}, mh{"h", h, M, F, h_stride, es},
        sg{"saved_gate", saved_gate, sr, F, saved_stride, es},
        su{"saved_up", saved_up, sr, F, saved_stride, es},
        mw{"the workspace", workspace, 1, need, need, 1};
    for (const MatArg& m : {mx, mg, mu, mh, sg, su}) AR_TRY(check_matrix(m));
    AR_TRY(check_workspace(workspace, workspace_bytes, need));
    for (const MatArg& o : {mh, sg, su, mw})
        for (const MatArg& i : {mx, mg, mu}) AR_TRY(check_apart(o, i));
    for (const MatArg& o : {sg, su, mw}) AR_TRY(check_apart(o, mh));
    for (const MatArg& o : {su, mw}) AR_TRY(check_apart(o, sg));
    AR_TRY(check_apart(mw, su));
    if (M == 0 || F == 0) return AR_OK;
    const ForwardArgs a{M, D, F, x_stride, w_stride, h_stride, saved_stride, act};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        hipLaunchKernelGGL((forward_kernel<T>), tiles(M, F), dim3(256), 0, st, a,
                           static_cast<const T*>(x), static_cast<const T*>(wg),
                           static_cast<const T*>(wu), static_cast<T*>(h),
                           static_cast<T*>(saved_gate), static_cast<T*>(saved_up));
        return launch_status("gated feed-forward");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
}

AR_EXPORT ar_status ar_glu_backward(int32_t dtype, int64_t M, int64_t D, int64_t F, const void* dh,
                                    int64_t dh_stride, const void* x, int64_t x_stride,
                                    const void* wg, const void* wu, int64_t w_stride,
                                    const void* saved_gate, const void* saved_up,
                                    int64_t saved_stride, int32_t accumulate, void* dx,
                                    int64_t dx_stride, void* dwg, void* dwu, int64_t dw_stride,
                                    void* workspace, int64_t workspace_bytes, void* stream) {
    clear_error();
    int32_t es = 0;
    int64_t need = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(ar_glu_workspace(dtype, M, D, F, 1, &need));
    if (!dwg != !dwu && F > 0 && D > 0)
        return fail(AR_ERR_INVALID_ARG, "dwg and dwu are given together");
    const MatArg mh{"dh", dh, M, F, dh_stride, es}, mx{"x", x, dwg ? M : 0, D, x_stride, es},
        mg{"wg", wg, dx ? F : 0, D, w_stride, es}, mu{"wu", wu, dx ? F : 0, D, w_stride, es},
        sg{"saved_gate", saved_gate, M, F, saved_stride, es},
        su{"saved_up", saved_up, M, F, saved_stride, es},
        ox{"dx", dx, dx ? M : 0, D, dx_stride, es},
        og{"dwg", dwg, dwg ? F : 0, D, dw_stride, es}, ou{"dwu", dwu, dwg ? F : 0, D, dw_stride, es},
        mw{"the workspace", workspace, 1, need, need, 1};
    for (const MatArg& m : {mh, mx, mg, mu, sg, su, ox, og, ou}) AR_TRY(check_matrix(m));
    AR_TRY(check_workspace(workspace, workspace_bytes, need));
    for (const MatArg& o : {ox, og, ou, mw})
        for (const MatArg& i : {mh, mx, mg, mu, sg, su}) AR_TRY(check_apart(o, i));
    for (const MatArg& o : {og, ou, mw}) AR_TRY(check_apart(o, ox));
    for (const MatArg& o : {ou, mw}) AR_TRY(check_apart(o, og));
    AR_TRY(check_apart(mw, ou));
    if (D == 0 || (!dx && !dwg)) return AR_OK;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        const int64_t fs = factor_stride(F);
        T* const dg = static_cast<T*>(workspace);
        T* const du = dg + M * fs;
        if (M > 0 && F > 0)
            hipLaunchKernelGGL((factors_kernel<T>),
                               dim3(unsigned(std::min<int64_t>(ceil_div(M * F, 256), 1 << 16))),
                               dim3(256), 0, st, M, F, static_cast<const T*>(dh), dh_stride,
                               static_cast<const T*>(saved_gate), static_cast<const T*>(saved_up),
                               saved_stride, dg, du, fs);
        const T* const X = static_cast<const T*>(x);
        if (dx && M > 0)
            hipLaunchKernelGGL((product_kernel<T>), tiles(M, D), dim3(256), 0, st,
                               (Operand<T>{dg, fs, 1}),
                               (Operand<T>{static_cast<const T*>(wg), 1, w_stride}), F,
                               (Operand<T>{du, fs, 1}),
                               (Operand<T>{static_cast<const T*>(wu), 1, w_stride}), F, M, D, 0,
                               static_cast<T*>(dx), dx_stride);
        if (dwg && F > 0) {
            for (int i = 0; i < 2; ++i)
                hipLaunchKernelGGL((product_kernel<T>), tiles(F, D), dim3(256), 0, st,
                                   (Operand<T>{i ? du : dg, 1, fs}), (Operand<T>{X, 1, x_stride}), M,
                                   (Operand<T>{}), (Operand<T>{}), int64_t(0), F, D, accumulate,
                                   static_cast<T*>(i ? dwu : dwg), dw_stride);
        }
        return launch_status("gated feed-forward gradients");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
}
