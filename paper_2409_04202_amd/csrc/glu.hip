// The gated feed-forward block's products.
#include <algorithm>
#include <type_traits>

#include "product.hpp"

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

struct ForwardArgs {
    int64_t h_stride, saved_stride;
    int act;
};

template <class T, int BR, int BC, int WR, int WC, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WC) void forward_kernel(ProductShape p, ForwardArgs a,
                                                               Side<T> x, Side<T> w, T* h, T* sg,
                                                               T* su) {
    using P = Tile<T, BR, BC, WR, WC, true, true, true, DIRECT>;
    using S = Store<1>;
    static_assert(P::LDS >= WR * WC * S::BYTES, "");
    __shared__ __attribute__((aligned(16))) char lds[P::LDS];
    int64_t rt, ct;
    if (!tile_of(p, blockIdx.x, &rt, &ct)) return;
    f32x16 acc[P::SR][2] = {};
    P::run(p, x, w, rt * BR, ct * (BC / 2), (AR_LDS char*)lds, acc);
    const int wave = int(threadIdx.x) >> 6, wr = wave / WC, wc = wave % WC;
    AR_LDS float* const part = (AR_LDS float*)((AR_LDS char*)lds + wave * S::BYTES);
#pragma unroll
    for (int i = 0; i < P::SR; ++i) {
        const int64_t r0 = rt * BR + (wr * P::SR + i) * 32, c0 = ct * (BC / 2) + wc * 32;
        float value[16], slope[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) activate(a.act, acc[i][0][e], &value[e], &slope[e]);
        auto pass = [&](T* out, int64_t stride, auto f) {
            S::fill(part, f);
            wave_sync();
            S::store(part, out, stride, r0, p.rows, c0, p.cols, false);
            wave_sync();
        };
        pass(h, a.h_stride, [&](int, int e) { return value[e] * acc[i][1][e]; });
        if (sg) {
            pass(sg, a.saved_stride, [&](int, int e) { return slope[e] * acc[i][1][e]; });
            pass(su, a.saved_stride, [&](int, int e) { return value[e]; });
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

// C = R L^T, or C += with accumulate.
template <class T, int BR, int BC, int WR, int WC, bool RKC, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WC) void product_kernel(ProductShape p, Side<T> r, Side<T> l,
                                                               int accumulate, T* out,
                                                               int64_t stride) {
    using P = Tile<T, BR, BC, WR, WC, RKC, false, false, DIRECT>;
    using S = Store<P::SC>;
    static_assert(P::LDS >= WR * WC * S::BYTES, "");
    __shared__ __attribute__((aligned(16))) char lds[P::LDS];
    int64_t rt, ct;
    if (!tile_of(p, blockIdx.x, &rt, &ct)) return;
    f32x16 acc[P::SR][P::SC] = {};
    P::run(p, r, l, rt * BR, ct * BC, (AR_LDS char*)lds, acc);
    const int wave = int(threadIdx.x) >> 6, wr = wave / WC, wc = wave % WC;
    AR_LDS float* const part = (AR_LDS float*)((AR_LDS char*)lds + wave * S::BYTES);
#pragma unroll
    for (int i = 0; i < P::SR; ++i) {
        S::fill(part, [&](int j, int e) { return acc[i][j][e]; });
        wave_sync();
        S::store(part, out, stride, rt * BR + (wr * P::SR + i) * 32, p.rows,
                 ct * BC + wc * P::SC * 32, p.cols, accumulate);
        wave_sync();
    }
}

// Whether a tile's copies may go straight to LDS: 16-byte chunks at 16-byte
// places, within 32-bit offsets of the tile's first row.
template <class T>
bool direct(const void* a, const void* b, int64_t stride, int64_t extent, bool kc) {
    constexpr int VEC = Num<T>::VEC;
    if ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) % kChunk) return false;
    if (stride % VEC || stride * int64_t(sizeof(T)) > (int64_t(1) << 22)) return false;
    return kc || extent % VEC == 0;
}

int64_t factor_stride(int64_t F) { return round_up(F, 8); }

ProductShape shape(int64_t rows, int64_t cols, int64_t K, int segments, int br, int bc) {
    return ProductShape{rows, cols, K, segments, ceil_div(rows, br), ceil_div(cols, bc)};
}

dim3 grid_of(const ProductShape& p) {
    return dim3(unsigned(tile_blocks(p.row_tiles * p.col_tiles)));
}

template <class T, bool RKC, int BR, int BC, int WR, int WC>
void launch_product(const ProductShape& p, const Side<T>& r, const Side<T>& l, int accumulate,
                    T* out, int64_t stride, hipStream_t st) {
    const bool fast = direct<T>(r.p[0], r.p[1], r.stride, p.rows, RKC) &&
                      direct<T>(l.p[0], l.p[1], l.stride, p.cols, false);
    const dim3 block(64 * WR * WC);
    if (fast)
        hipLaunchKernelGGL((product_kernel<T, BR, BC, WR, WC, RKC, true>), grid_of(p), block, 0, st,
                           p, r, l, accumulate, out, stride);
    else
        hipLaunchKernelGGL((product_kernel<T, BR, BC, WR, WC, RKC, false>), grid_of(p), block, 0,
                           st, p, r, l, accumulate, out, stride);
}

template <class T, int BR, int BC, int WR, int WC>
void launch_forward(const ForwardArgs& a, int64_t M, int64_t D, int64_t F, const Side<T>& x,
                    const Side<T>& w, T* h, T* sg, T* su, hipStream_t st) {
    const ProductShape p = shape(M, F, D, 1, BR, BC / 2);
    const bool fast = direct<T>(x.p[0], x.p[1], x.stride, M, true) &&
                      direct<T>(w.p[0], w.p[1], w.stride, F, true);
    const dim3 block(64 * WR * WC);
    if (fast)
        hipLaunchKernelGGL((forward_kernel<T, BR, BC, WR, WC, true>), grid_of(p), block, 0, st, p, a,
                           x, w, h, sg, su);
    else
        hipLaunchKernelGGL((forward_kernel<T, BR, BC, WR, WC, false>), grid_of(p), block, 0, st, p,
                           a, x, w, h, sg, su);
}

}  // namespace
}  // namespace arp

using namespace arp;

// Whether a product of so many 256 x 256 tiles takes those, and not four times
// as many of 128 x 128: where they fill the card's 256 CUs.
static bool large_tiles(int64_t tiles) { return tiles >= 192; }

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
    const ForwardArgs a{h_stride, saved_stride, act};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        const Side<T> sx{{static_cast<const T*>(x), static_cast<const T*>(x)}, x_stride},
            sw{{static_cast<const T*>(wg), static_cast<const T*>(wu)}, w_stride};
        T *const oh = static_cast<T*>(h), *const og = static_cast<T*>(saved_gate),
                 *const ou = static_cast<T*>(saved_up);
        if (large_tiles(ceil_div(M, 256) * ceil_div(F, 128)))
            launch_forward<T, 256, 256, 2, 4>(a, M, D, F, sx, sw, oh, og, ou, st);
        else
            launch_forward<T, 128, 128, 2, 2>(a, M, D, F, sx, sw, oh, og, ou, st);
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
        auto product = [&](auto rkc, const Side<T>& r, const Side<T>& l, int64_t rows, int64_t K,
                           int segments, int acc, void* out, int64_t stride) {
            constexpr bool RKC = decltype(rkc)::value;
            T* const o = static_cast<T*>(out);
            if (large_tiles(ceil_div(rows, 256) * ceil_div(D, 256)))
                launch_product<T, RKC, 256, 256, 2, 4>(shape(rows, D, K, segments, 256, 256), r, l,
                                                       acc, o, stride, st);
            else
                launch_product<T, RKC, 128, 128, 2, 2>(shape(rows, D, K, segments, 128, 128), r, l,
                                                       acc, o, stride, st);
        };
        if (dx && M > 0)
            product(std::true_type{}, Side<T>{{dg, du}, fs},
                    Side<T>{{static_cast<const T*>(wg), static_cast<const T*>(wu)}, w_stride}, M, F,
                    2, 0, dx, dx_stride);
        if (dwg && F > 0) {
            const Side<T> sx{{static_cast<const T*>(x), static_cast<const T*>(x)}, x_stride};
            product(std::false_type{}, Side<T>{{dg, dg}, fs}, sx, F, M, 1, accumulate, dwg,
                    dw_stride);
            product(std::false_type{}, Side<T>{{du, du}, fs}, sx, F, M, 1, accumulate, dwu,
                    dw_stride);
        }
        return launch_status("gated feed-forward gradients");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
}
