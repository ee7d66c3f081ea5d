// Distillation from a teacher's top logits, forward and backward.
//
// A block takes a row.  In units of log2, with c = log2(e) / temperature:
//   m = max z,  S = sum 2^((z - m) c),  log2 q_j = (z_j - m) c - log2 S
// and the same for the teacher's entries; the loss and the gradient follow
// from these.  The difference comes before the product, which could overflow
// at a mask of the type's lowest value.  The first pass over the row takes the running maximum and sum
// (a sum is rescaled where the maximum rises); the second computes the
// gradient.  Bound by memory: the row read and the gradient written.
#include <algorithm>
#include <cmath>

#include "replica.hpp"

namespace arp {
namespace {

constexpr int kBlock = 1024;
constexpr int kWaves = kBlock / 64;

struct DistillArgs {
    const int64_t* ids;
    const float* weights;
    float* loss;
    int64_t T, V, K;
    int64_t logits_stride, teacher_stride, ids_stride, grad_stride;
    float c;            // log2(e) / temperature
    float temperature;
};

// A maximum and the sum of 2^((x - maximum) c); an empty one is (-inf, 0).
struct MaxSum {
    float m, s;
    __device__ __forceinline__ void add(const MaxSum o, float c) {
        const float top = fmaxf(m, o.m);
        // nothing but -inf so far: the sums are 0 (or NaN) and stay so
        const float base = top == -INFINITY ? 0.0f : top;
        s = s * exp2f((m - base) * c) + o.s * exp2f((o.m - base) * c);
        m = top;
    }
};

__device__ __forceinline__ MaxSum wave_sum(MaxSum a, float c) {
    for (int d = 32; d > 0; d /= 2) a.add({__shfl_xor(a.m, d), __shfl_xor(a.s, d)}, c);
    return a;
}

__device__ __forceinline__ float wave_sum(float v) {
    for (int d = 32; d > 0; d /= 2) v += __shfl_xor(v, d);
    return v;
}

template <class T, class S>
__global__ __launch_bounds__(kBlock) void distill_kernel(DistillArgs a, const T* logits,
                                                         const S* teacher, T* grad) {
    constexpr int VEC = Num<T>::VEC;
    extern __shared__ char lds[];
    __shared__ MaxSum part[kWaves];
    __shared__ float terms[kWaves];
    int32_t* const eid = reinterpret_cast<int32_t*>(lds);      // an entry's id, -1 if absent
    float* const ep = reinterpret_cast<float*>(lds) + a.K;     // the teacher's logit, then p
    float* const ez = reinterpret_cast<float*>(lds) + 2 * a.K; // the student's logit there, then log2 q
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;

    auto all = [&](MaxSum v) {  // over the block
        v = wave_sum(v, a.c);
        __syncthreads();
        if (lane == 0) part[w] = v;
        __syncthreads();
        MaxSum r = part[0];
        for (int i = 1; i < kWaves; ++i) r.add(part[i], a.c);
        return r;
    };

    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T* const z = logits + t * a.logits_stride;
        T* const g = grad ? grad + t * a.grad_stride : nullptr;
        const float weight = a.weights ? a.weights[t] : 1.0f;
        MaxSum tea{-INFINITY, 0.0f}, stu{-INFINITY, 0.0f};
        __syncthreads();  // the entries of the row before are done with
        if (weight != 0.0f) {
            for (int64_t k = threadIdx.x; k < a.K; k += kBlock) {
                const int64_t id = a.ids[t * a.ids_stride + k];
                const float s = Num<S>::up(teacher[t * a.teacher_stride + k]);
                const bool is = id >= 0 && id < a.V && s != -INFINITY;
                eid[k] = is ? int32_t(id) : -1;
                ep[k] = s;
                ez[k] = is ? Num<T>::up(z[id]) : 0.0f;
                if (is) tea.add({s, 1.0f}, a.c);
            }
            tea = all(tea);
        }
        bool live = weight != 0.0f && (tea.s != 0.0f);
        if (live) {
            for (int64_t at = int64_t(threadIdx.x) * VEC; at < a.V; at += kBlock * VEC) {
                const int n = int(a.V - at < VEC ? a.V - at : VEC);
                float f[VEC];
                Num<T>::unpack(n == VEC ? load_vec(z + at) : load_part(z + at, n), f);
                for (int i = 0; i < VEC; ++i) f[i] = i < n ? f[i] : -INFINITY;
                float top = stu.m;
                for (int i = 0; i < VEC; ++i) top = fmaxf(top, f[i]);
                const float base = top == -INFINITY ? 0.0f : top;
                float s = stu.s * exp2f((stu.m - base) * a.c);
                for (int i = 0; i < VEC; ++i) s += exp2f((f[i] - base) * a.c);
                stu = {top, s};
            }
            stu = all(stu);
            live = stu.s != 0.0f;
        }
        if (!live) {
            if (threadIdx.x == 0) a.loss[t] = 0.0f;
            if (g) {
                for (int64_t at = int64_t(threadIdx.x) * VEC; at < a.V; at += kBlock * VEC) {
                    if (a.V - at >= VEC) store_vec(g + at, u32x4{0, 0, 0, 0});
                    else store_part(g + at, u32x4{0, 0, 0, 0}, int(a.V - at));
                }
            }
            continue;
        }
        const float ls = log2f(stu.s), lt = log2f(tea.s);
        float sum = 0.0f;
        for (int64_t k = threadIdx.x; k < a.K; k += kBlock) {
            if (eid[k] < 0) continue;
            const float lp = (ep[k] - tea.m) * a.c - lt, lq = (ez[k] - stu.m) * a.c - ls;
            const float p = exp2f(lp);
            ep[k] = p;
            ez[k] = lq;
            if (p != 0.0f) sum += p * (lp - lq);
        }
        sum = wave_sum(sum);
        if (lane == 0) terms[w] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            float v = 0.0f;
            for (int i = 0; i < kWaves; ++i) v += terms[i];
            a.loss[t] = weight * a.temperature * a.temperature * (v * 0.6931471805599453f);
        }
        if (!g) continue;
        const float scale = weight * a.temperature;
        for (int64_t at = int64_t(threadIdx.x) * VEC; at < a.V; at += kBlock * VEC) {
            const int n = int(a.V - at < VEC ? a.V - at : VEC);
            float f[VEC];
            Num<T>::unpack(n == VEC ? load_vec(z + at) : load_part(z + at, n), f);
            for (int i = 0; i < VEC; ++i) f[i] = scale * exp2f((f[i] - stu.m) * a.c - ls);
            if (n == VEC) store_vec(g + at, Num<T>::pack(f));
            else store_part(g + at, Num<T>::pack(f), n);
        }
        __syncthreads();  // the entries' elements are written once more, after these
        for (int64_t k = threadIdx.x; k < a.K; k += kBlock) {
            const int32_t id = eid[k];
            if (id < 0) continue;
            float p = 0.0f;  // of every entry with this id: each of them stores the same
            for (int64_t j = 0; j < a.K; ++j)
                if (eid[j] == id) p += ep[j];
            g[id] = Num<T>::down(scale * (exp2f(ez[k]) - p));
        }
    }
}

template <class T, class S>
ar_status run_distill(const DistillArgs& a, const void* logits, const void* teacher, void* grad,
                      hipStream_t st) {
    const unsigned grid = unsigned(std::min<int64_t>(a.T, 1 << 20));
    hipLaunchKernelGGL((distill_kernel<T, S>), dim3(grid), dim3(kBlock), size_t(12 * a.K), st, a,
                       static_cast<const T*>(logits), static_cast<const S*>(teacher),
                       static_cast<T*>(grad));
    return launch_status("distillation");
}

}  // namespace
}  // namespace arp

using namespace arp;

AR_EXPORT ar_status ar_distill_workspace(int64_t T, int64_t V, int64_t K, int64_t* bytes) {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    AR_TRY(check_extent("T", T));
    AR_TRY(check_extent("V", V));
    AR_TRY(check_extent("K", K));
    if (K > AR_DISTILL_MAX_K) return fail(AR_ERR_UNSUPPORTED, "K exceeds AR_DISTILL_MAX_K");
    *bytes = 0;
    return AR_OK;
}

AR_EXPORT ar_status ar_distill(int32_t dtype, int64_t T, int64_t V, int64_t K, const void* logits,
                               int64_t logits_stride, int32_t teacher_dtype, const void* teacher,
                               int64_t teacher_stride, const int64_t* ids, int64_t ids_stride,
                               float temperature, const float* weights, float* loss, void* grad,
                               int64_t grad_stride, void* workspace, int64_t workspace_bytes,
                               void* stream) {
    clear_error();
    int32_t es = 0, ts = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_dtype("teacher_dtype", teacher_dtype, &ts));
    int64_t need = 0;
    AR_TRY(ar_distill_workspace(T, V, K, &need));
    if (!(temperature > 0.0f) || std::isinf(temperature))
        return fail(AR_ERR_INVALID_ARG, "temperature must be finite and > 0");
    const MatArg ml{"logits", logits, T, V, logits_stride, es},
        mt{"teacher", teacher, T, K, teacher_stride, ts}, mi{"ids", ids, T, K, ids_stride, 8},
        mw{"weights", weights, 1, weights ? T : 0, T, 4}, mo{"loss", loss, 1, T, T, 4},
        mg{"grad", grad, grad ? T : 0, V, grad_stride, es},
        ms{"the workspace", workspace, 1, need, need, 1};
    for (const MatArg& m : {ml, mt, mi, mw, mo, mg}) AR_TRY(check_matrix(m));
    AR_TRY(check_workspace(workspace, workspace_bytes, need));
    for (const MatArg& m : {ml, mt, mi, mw}) AR_TRY(check_apart(mo, m));
    if (!(grad == logits && grad_stride == logits_stride)) AR_TRY(check_apart(mg, ml));
    for (const MatArg& m : {mt, mi, mw, mo}) AR_TRY(check_apart(mg, m));
    for (const MatArg& m : {ml, mt, mi, mw, mo, mg}) AR_TRY(check_apart(ms, m));
    if (T == 0) return AR_OK;
    const DistillArgs a{ids, weights, loss, T, V, K, logits_stride, teacher_stride, ids_stride,
                        grad_stride, float(1.4426950408889634 / double(temperature)), temperature};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == AR_F32)
        return teacher_dtype == AR_F32 ? run_distill<float, float>(a, logits, teacher, grad, st)
                                       : run_distill<float, uint16_t>(a, logits, teacher, grad, st);
    return teacher_dtype == AR_F32 ? run_distill<uint16_t, float>(a, logits, teacher, grad, st)
                                   : run_distill<uint16_t, uint16_t>(a, logits, teacher, grad, st);
}
