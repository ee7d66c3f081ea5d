// Routing of tokens to experts, and the balance loss with its gradient.
//
// A row's logits stay in registers: a group of 2^g lanes holds a row, each lane P
// adjacent ones, so a wavefront has several short rows or one long row, and the
// softmax, the choice and the gradient are reductions over a group's lanes.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "replica.hpp"

namespace arp {
namespace {

constexpr int kBlock = 256;
constexpr int kMaxParts = 512;  // blocks whose sums are joined

// exp(x) for x <= 0, to a few units in the last place: 2^(x log2 e) with what the
// product was rounded by put back.
__device__ __forceinline__ float exp_below(float x) {
    const float t = x * 1.44269504f, lost = fmaf(x, 1.44269504f, -t) + x * 1.92596299e-8f;
    const float e = __builtin_amdgcn_exp2f(t);
    return t > -120.0f ? fmaf(e, lost * 0.69314718f, e) : e;
}

// Another lane's value: lanes change places in pairs 2^STEP apart, or mirrored
// within the next larger group, which a reduction does not tell apart.
template <int STEP>
__device__ __forceinline__ uint32_t other(uint32_t v) {
    if constexpr (STEP == 0) return uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0xB1, 0xF, 0xF, true));
    else if constexpr (STEP == 1) return uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x4E, 0xF, 0xF, true));
    else if constexpr (STEP == 2) return uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x141, 0xF, 0xF, true));
    else if constexpr (STEP == 3) return uint32_t(__builtin_amdgcn_mov_dpp(int(v), 0x140, 0xF, 0xF, true));
    else return uint32_t(__shfl_xor(int(v), 1 << STEP));
}
template <int LOG, int STEP = 0, class V, class F>
__device__ __forceinline__ V group_reduce(V v, F&& f) {
    if constexpr (STEP < LOG) {
        if constexpr (sizeof(V) == 4) {
            v = f(v, __builtin_bit_cast(V, other<STEP>(__builtin_bit_cast(uint32_t, v))));
        } else {
            const uint32_t lo = other<STEP>(uint32_t(v)), hi = other<STEP>(uint32_t(v >> 32));
            v = f(v, V(hi) << 32 | lo);
        }
        return group_reduce<LOG, STEP + 1>(v, f);
    } else {
        return v;
    }
}
template <int LOG> __device__ __forceinline__ float group_sum(float v) {
    return group_reduce<LOG>(v, [](float a, float b) { return a + b; });
}
template <int LOG> __device__ __forceinline__ float group_max(float v) {
    return group_reduce<LOG>(v, [](float a, float b) { return fmaxf(a, b); });
}

// A logit and its place as one number: larger for a larger logit, and of equal
// ones for the lower place.  A NaN is above everything; 0 is an absent expert's.
// bf16's 16 bits and the place fit 32 bits.
template <class T> struct Rank;
template <> struct Rank<uint16_t> {
    using K = uint32_t;
    static __device__ __forceinline__ K of(float z, uint32_t place) {
        const uint32_t u = __float_as_uint(z + 0.0f);   // (-0 is 0)
        const uint32_t o = z != z ? 0xFFFF0000u : (u ^ uint32_t(int32_t(u) >> 31 | int32_t(0x80000000)));
        return z == -INFINITY ? 0u : (o & 0xFFFF0000u) | (0xFFFFu - place);
    }
    static __device__ __forceinline__ uint32_t place(K k) { return 0xFFFFu - (k & 0xFFFFu); }
    static __device__ __forceinline__ float logit(K k) {
        const uint32_t o = k & 0xFFFF0000u;
        return __uint_as_float((int32_t(o) < 0 ? o ^ 0x80000000u : ~o) & 0xFFFF0000u);
    }
};
template <> struct Rank<float> {
    using K = uint64_t;
    static __device__ __forceinline__ K of(float z, uint32_t place) {
        const uint32_t u = __float_as_uint(z + 0.0f);
        const uint32_t o = z != z ? 0xFFFFFFFFu : u ^ uint32_t(int32_t(u) >> 31 | int32_t(0x80000000));
        return z == -INFINITY ? 0u : K(o) << 32 | (0xFFFFFFFFu - place);
    }
    static __device__ __forceinline__ uint32_t place(K k) { return 0xFFFFFFFFu - uint32_t(k); }
    static __device__ __forceinline__ float logit(K k) {
        const uint32_t o = uint32_t(k >> 32);
        return __uint_as_float(int32_t(o) < 0 ? o ^ 0x80000000u : ~o);
    }
};

// A lane's P logits from `first` on; behind the row's end -inf.
template <class T, int P>
__device__ __forceinline__ void load_logits(const T* row, int first, int E, float* z) {
    constexpr int VEC = Num<T>::VEC;
#pragma unroll
    for (int i = 0; i < P; i += VEC) {
        if (first + i + VEC <= E) {
            Num<T>::unpack(load_vec(row + first + i), z + i);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                z[i + e] = first + i + e < E ? Num<T>::up(((const AR_GLOBAL T*)row)[first + i + e])
                                             : -INFINITY;
        }
    }
}

// The row's probabilities; false where no logit is above -inf.
template <int LOG, int P>
__device__ __forceinline__ bool softmax(const float* z, float* p, float* top, float* inverse) {
    float m = z[0];
#pragma unroll
    for (int i = 1; i < P; ++i) m = fmaxf(m, z[i]);
    m = group_max<LOG>(m);
    // (a NaN is no maximum: a row of NaN and -inf has a NaN for its sum)
    float s = 0.0f, any = m;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        p[i] = exp_below(z[i] - m);
        s += p[i];
        if (z[i] != z[i]) any = 0.0f;
    }
    s = group_sum<LOG>(s);
    any = group_max<LOG>(any);
    const float r = 1.0f / s;
#pragma unroll
    for (int i = 0; i < P; ++i) p[i] *= r;
    *top = m;
    *inverse = r;
    return any != -INFINITY;
}

struct RouteArgs {
    int64_t T, stride;
    int E, k, normalize;
    const uint8_t* live;
    int64_t* ids;
    float* gates;
    int32_t* counts;  // E + 1, or a part of that a block
    float* mass;      // E, or a part a block
};

__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Bound by the choice's reductions, then by memory.
template <class T, int LOG, int P>
__global__ __launch_bounds__(kBlock) void route_kernel(const T* logits, RouteArgs a) {
    using R = Rank<T>;
    using K = typename R::K;
    constexpr int LANES = 1 << LOG, GROUPS = 64 / LANES, WAVES = kBlock / 64;
    constexpr int WIDE = LANES * P;                     // experts at most
    constexpr int PICKS = WIDE < AR_ROUTE_MAX_K ? WIDE : AR_ROUTE_MAX_K;
    __shared__ int32_t hist[WIDE + 1];
    __shared__ float sums[WAVES * GROUPS][WIDE];
    __shared__ int32_t place[WAVES][GROUPS * PICKS];
    __shared__ float gate[WAVES][GROUPS * PICKS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> LOG;
    const int sub = lane & (LANES - 1), first = sub * P;
    for (int i = threadIdx.x; i <= WIDE; i += kBlock) hist[i] = 0;
    __syncthreads();
    float mass[P] = {};
    const int64_t step = int64_t(gridDim.x) * WAVES * GROUPS;
    for (int64_t r0 = (int64_t(blockIdx.x) * WAVES + wave) * GROUPS; r0 < a.T; r0 += step) {
        const int64_t r = r0 + group;
        const bool live = r < a.T && (!a.live || a.live[r]);
        float z[P], p[P], top, inverse;
        if (live) {
            load_logits<T, P>(logits + r * a.stride, first, a.E, z);
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) z[i] = -INFINITY;
        }
        const bool any = softmax<LOG, P>(z, p, &top, &inverse) && live;
        K key[P];
#pragma unroll
        for (int i = 0; i < P; ++i) {
            mass[i] += any ? p[i] : 0.0f;
            key[i] = R::of(z[i], uint32_t(first + i));
        }
        float total = 0.0f;
        for (int j = 0; j < a.k; ++j) {
            K best = key[0];
#pragma unroll
            for (int i = 1; i < P; ++i) best = key[i] > best ? key[i] : best;
            best = group_reduce<LOG>(best, [](K x, K y) { return x > y ? x : y; });
            const bool here = best != 0;
            const float g = here ? exp_below(R::logit(best) - top) * inverse : 0.0f;
            total += g;
#pragma unroll
            for (int i = 0; i < P; ++i) key[i] = key[i] == best ? K(0) : key[i];
            if (sub == 0) {
                const int e = here ? int(R::place(best)) : -1;
                place[wave][group * a.k + j] = e;
                gate[wave][group * a.k + j] = g;
                if (here) atomicAdd(&hist[e], 1);
            }
        }
        if (sub == 0 && any) atomicAdd(&hist[a.E], 1);
        if (a.normalize) {
            wave_sync();
            for (int j = sub; j < a.k; j += LANES)
                if (any) gate[wave][group * a.k + j] /= total;
        }
        wave_sync();
        // the wavefront's rows are adjacent: so are their choices
        const int64_t rows = a.T - r0 < GROUPS ? a.T - r0 : GROUPS;
        for (int i = lane; i < int(rows) * a.k; i += 64) {
            a.ids[r0 * a.k + i] = place[wave][i];
            a.gates[r0 * a.k + i] = gate[wave][i];
        }
        wave_sync();
    }
#pragma unroll
    for (int i = 0; i < P; ++i) sums[wave * GROUPS + group][first + i] = mass[i];
    __syncthreads();
    int32_t* const counts = a.counts + int64_t(blockIdx.x) * (a.E + 1);
    float* const masses = a.mass + int64_t(blockIdx.x) * a.E;
    for (int e = threadIdx.x; e <= a.E; e += kBlock) {
        counts[e] = hist[e];
        if (e == a.E) break;
        float s = 0.0f;
        for (int i = 0; i < WAVES * GROUPS; ++i) s += sums[i][e];
        masses[e] = s;
    }
}

// The blocks' counts and sums, added in order: 16 experts a block of 64 x 16 lanes,
// each lane every 64th part.
__global__ __launch_bounds__(1024) void route_join_kernel(int parts, int E, const int32_t* counts,
                                                          const float* mass, int32_t* counts_out,
                                                          float* mass_out) {
    __shared__ int32_t c[64][16];
    __shared__ float m[64][16];
    const int e = int(blockIdx.x) * 16 + (threadIdx.x & 15), at = threadIdx.x >> 4;
    int32_t n = 0;
    float s = 0.0f;
    if (e <= E)
        for (int i = at; i < parts; i += 64) {
            n += counts[int64_t(i) * (E + 1) + e];
            if (e < E) s += mass[int64_t(i) * E + e];
        }
    c[at][threadIdx.x & 15] = n;
    m[at][threadIdx.x & 15] = s;
    for (int half = 32; half; half >>= 1) {
        __syncthreads();
        if (at < half) {
            c[at][threadIdx.x & 15] += c[at + half][threadIdx.x & 15];
            m[at][threadIdx.x & 15] += m[at + half][threadIdx.x & 15];
        }
    }
    if (at) return;
    if (e <= E) counts_out[e] = c[0][threadIdx.x];
    if (e < E) mass_out[e] = m[0][threadIdx.x];
}

struct BalanceArgs {
    int64_t T, stride, grad_stride;
    int E, k, normalize;
    float coefficient;
    const int64_t* ids;
    const int32_t* counts;
    const float *mass, *dgates;
    float* loss;
};

// The loss' slope at an expert's probability: coefficient E counts_e / (k N^2).
__device__ __forceinline__ float slope_of(const BalanceArgs& a, int e) {
    const float n = float(a.counts[a.E]);
    return n > 0.0f ? a.coefficient * float(a.E) / float(a.k) * (float(a.counts[e]) / n) / n : 0.0f;
}

// The loss, by one wavefront, in 64 bits.
__device__ __forceinline__ void loss_of(const BalanceArgs& a) {
    double s = 0.0;
    for (int e = threadIdx.x; e < a.E; e += 64) s += double(a.counts[e]) * double(a.mass[e]);
    for (int step = 32; step; step >>= 1) s += __shfl_xor(s, step);
    const double n = double(a.counts[a.E]);
    if (threadIdx.x == 0)
        *a.loss = a.counts[a.E] > 0 ? float(s * double(a.coefficient) * a.E / a.k / n / n) : 0.0f;
}
__global__ __launch_bounds__(64) void loss_kernel(BalanceArgs a) { loss_of(a); }

// The gradient, and in the last block the loss.
template <class T, int LOG, int P>
__global__ __launch_bounds__(kBlock) void balance_kernel(const T* logits, T* grad, BalanceArgs a) {
    constexpr int VEC = Num<T>::VEC;
    constexpr int LANES = 1 << LOG, GROUPS = 64 / LANES, WAVES = kBlock / 64;
    if (blockIdx.x == gridDim.x - 1) {
        if (threadIdx.x < 64) loss_of(a);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> LOG;
    const int first = (lane & (LANES - 1)) * P;
    float slope[P];
#pragma unroll
    for (int i = 0; i < P; ++i) slope[i] = first + i < a.E ? slope_of(a, first + i) : 0.0f;
    const int64_t step = int64_t(gridDim.x - 1) * WAVES * GROUPS;
    for (int64_t r0 = (int64_t(blockIdx.x) * WAVES + wave) * GROUPS; r0 < a.T; r0 += step) {
        const int64_t r = r0 + group;
        const int64_t* const ids = a.ids + r * a.k;
        const bool live = r < a.T && ids[0] >= 0;
        float z[P], p[P], top, inverse;
        if (live) {
            load_logits<T, P>(logits + r * a.stride, first, a.E, z);
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) z[i] = -INFINITY;
        }
        const bool any = softmax<LOG, P>(z, p, &top, &inverse) && live;
        // at[i]: the slope at p_i; with normalized gates apart, what is chosen: how often, and
        // the sum of its gates' gradients
        float at[P], times[P], wants[P];
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            at[i] = slope[i];
            times[i] = wants[i] = 0.0f;
        }
        if (a.dgates && live) {
            const float* const dg = a.dgates + r * a.k;
            for (int j = 0; j < a.k; ++j) {
                const int64_t rel = ids[j] - first;
                const float g = dg[j];
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    wants[i] += rel == i ? g : 0.0f;
                    times[i] += rel == i ? 1.0f : 0.0f;
                }
            }
            if (!a.normalize) {
#pragma unroll
                for (int i = 0; i < P; ++i) at[i] += wants[i];
            }
        }
#pragma unroll
        for (int i = 0; i < P; ++i) sum += p[i] * at[i];
        sum = group_sum<LOG>(sum);
        float d[P];
#pragma unroll
        for (int i = 0; i < P; ++i) d[i] = p[i] * (at[i] - sum);
        if (a.normalize && a.dgates) {
            float total = 0.0f, dot = 0.0f;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                total += times[i] != 0.0f ? p[i] * times[i] : 0.0f;
                dot += times[i] != 0.0f ? p[i] * wants[i] : 0.0f;
            }
            total = group_sum<LOG>(total);
            dot = group_sum<LOG>(dot) / total;
#pragma unroll
            for (int i = 0; i < P; ++i)
                d[i] += times[i] != 0.0f ? p[i] / total * (wants[i] - times[i] * dot) : 0.0f;
        }
        if (r >= a.T) continue;
        T* const to = grad + r * a.grad_stride;
#pragma unroll
        for (int i = 0; i < P; ++i) d[i] = any ? d[i] : 0.0f;
#pragma unroll
        for (int i = 0; i < P; i += VEC) {
            if (first + i + VEC <= a.E) store_vec(to + first + i, Num<T>::pack(d + i));
            else if (first + i < a.E) store_part(to + first + i, Num<T>::pack(d + i), a.E - first - i);
        }
    }
}

// Lanes that hold a row: 8 logits each, 16 above 512 experts.
template <class F>
void by_width(int E, F&& f) {
    const auto go = [&](auto log, auto p) { f(log, p); };
    const auto eight = std::integral_constant<int, 8>{};
    if (E <= 8) go(std::integral_constant<int, 0>{}, eight);
    else if (E <= 16) go(std::integral_constant<int, 1>{}, eight);
    else if (E <= 32) go(std::integral_constant<int, 2>{}, eight);
    else if (E <= 64) go(std::integral_constant<int, 3>{}, eight);
    else if (E <= 128) go(std::integral_constant<int, 4>{}, eight);
    else if (E <= 256) go(std::integral_constant<int, 5>{}, eight);
    else if (E <= 512) go(std::integral_constant<int, 6>{}, eight);
    else go(std::integral_constant<int, 6>{}, std::integral_constant<int, 16>{});
}
int group_log(int64_t E) {
    int log = 0;
    while (log < 6 && (8 << log) < E) ++log;
    return log;
}

// Blocks of a routing: as many as the rows fill, each with `4 passes` at least.
int64_t parts_of(int64_t T, int64_t E) {
    const int64_t rows = (kBlock / 64) * (64 >> group_log(E));
    return std::max<int64_t>(1, std::min<int64_t>(kMaxParts, ceil_div(T, 4 * rows)));
}
int64_t part_bytes(int64_t T, int64_t E) {
    const int64_t parts = parts_of(T, E);
    return parts > 1 ? round_up(parts * (2 * E + 1) * 4, 16) : 0;
}

ar_status check_route_sizes(int64_t T, int64_t E, int64_t k) {
    AR_TRY(check_extent("T", T));
    AR_TRY(check_extent("E", E));
    AR_TRY(check_extent("k", k));
    if (E > AR_ROUTE_MAX_EXPERTS)
        return fail(AR_ERR_UNSUPPORTED, "E is at most AR_ROUTE_MAX_EXPERTS");
    if (k > AR_ROUTE_MAX_K) return fail(AR_ERR_UNSUPPORTED, "k is at most AR_ROUTE_MAX_K");
    if (k < 1 || k > E) return fail(AR_ERR_INVALID_ARG, "k is at least 1 and at most E");
    return AR_OK;
}

}  // namespace
}  // namespace arp

using namespace arp;

AR_EXPORT ar_status ar_route_workspace(int64_t T, int64_t E, int64_t k, int64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    AR_TRY(check_route_sizes(T, E, k));
    *bytes = part_bytes(T, E);
    return AR_OK;
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_route(int32_t dtype, int64_t T, int64_t E, int64_t k, const void* logits,
                             int64_t logits_stride, const uint8_t* live, int32_t normalize,
                             int64_t* ids, float* gates, int32_t* counts, float* mass,
                             void* workspace, int64_t workspace_bytes, void* stream) try {
    clear_error();
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_route_sizes(T, E, k));
    const int64_t need = part_bytes(T, E);
    const MatArg ml{"logits", logits, T, E, logits_stride, es}, mv{"live", live, live ? 1 : 0, T, T, 1},
        mi{"ids", ids, T, k, k, 8}, mg{"gates", gates, T, k, k, 4},
        mc{"counts", counts, 1, E + 1, E + 1, 4}, mm{"mass", mass, 1, E, E, 4},
        mw{"the workspace", workspace, 1, need, need, 1};
    for (const MatArg& m : {ml, mv, mi, mg, mc, mm}) AR_TRY(check_matrix(m));
    AR_TRY(check_workspace(workspace, workspace_bytes, need));
    const MatArg outs[] = {mi, mg, mc, mm, mw};
    for (int o = 0; o < 5; ++o) {
        AR_TRY(check_apart(outs[o], ml));
        AR_TRY(check_apart(outs[o], mv));
        for (int p = 0; p < o; ++p) AR_TRY(check_apart(outs[o], outs[p]));
    }
    const int64_t parts = parts_of(T, E);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    int32_t* const part_counts = static_cast<int32_t*>(workspace);
    float* const part_mass = reinterpret_cast<float*>(part_counts + parts * (E + 1));
    const RouteArgs a{T, logits_stride, int(E), int(k), normalize, live, ids, gates,
                      parts > 1 ? part_counts : counts, parts > 1 ? part_mass : mass};
    auto go = [&](auto zero) {
        using U = decltype(zero);
        by_width(int(E), [&](auto log, auto p) {
            hipLaunchKernelGGL((route_kernel<U, decltype(log)::value, decltype(p)::value>),
                               dim3(unsigned(parts)), dim3(kBlock), 0, st,
                               static_cast<const U*>(logits), a);
        });
        if (parts > 1)
            hipLaunchKernelGGL(route_join_kernel, dim3(unsigned(ceil_div(E + 1, 16))), dim3(1024), 0,
                               st, int(parts), int(E), part_counts, part_mass, counts, mass);
        return launch_status("routing");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_balance(int32_t dtype, int64_t T, int64_t E, int64_t k, const void* logits,
                               int64_t logits_stride, const int64_t* ids, const int32_t* counts,
                               const float* mass, float coefficient, int32_t normalize,
                               const float* dgates, float* loss, void* grad, int64_t grad_stride,
                               void* stream) try {
    clear_error();
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_route_sizes(T, E, k));
    if (!(std::abs(coefficient) <= 3.4e38f))
        return fail(AR_ERR_INVALID_ARG, "the coefficient is not finite");
    const int64_t rows = grad ? T : 0;
    const MatArg ml{"logits", logits, rows, E, logits_stride, es}, mi{"ids", ids, rows, k, k, 8},
        mc{"counts", counts, 1, E + 1, E + 1, 4}, mm{"mass", mass, 1, E, E, 4},
        md{"dgates", dgates, dgates ? rows : 0, k, k, 4}, mo{"loss", loss, 1, 1, 1, 4},
        mg{"grad", grad, rows, E, grad_stride, es};
    for (const MatArg& m : {ml, mi, mc, mm, md, mo, mg}) AR_TRY(check_matrix(m));
    for (const MatArg& i : {mi, mc, mm, md}) AR_TRY(check_apart(mg, i));
    if (grad != logits || grad_stride != logits_stride) AR_TRY(check_apart(mg, ml));
    for (const MatArg& i : {ml, mi, mc, mm, md, mg}) AR_TRY(check_apart(mo, i));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const BalanceArgs a{T, logits_stride, grad_stride, int(E), int(k), normalize, coefficient,
                        ids, counts, mass, dgates, loss};
    if (rows == 0) {
        hipLaunchKernelGGL(loss_kernel, dim3(1), dim3(64), 0, st, a);
        return launch_status("balance loss");
    }
    auto go = [&](auto zero) {
        using U = decltype(zero);
        by_width(int(E), [&](auto log, auto p) {
            const int64_t blocks = ceil_div(T, (kBlock / 64) * (64 >> decltype(log)::value));
            hipLaunchKernelGGL((balance_kernel<U, decltype(log)::value, decltype(p)::value>),
                               dim3(unsigned(std::min<int64_t>(blocks, 2048)) + 1), dim3(kBlock), 0, st,
                               static_cast<const U*>(logits), static_cast<U*>(grad), a);
        });
        return launch_status("balance loss");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}
