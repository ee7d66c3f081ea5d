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

constexpr int kBalanceBlock = 256;
constexpr int kWideRow = 512;   // experts above which a lane holds 16 logits
// (Of blocks with 16 logits a lane a CU's registers hold one of 1024 lanes, and all 512 parts
// at once as blocks of 512: 65536 x 512 46.4 and 44.2 us with the join.)
constexpr int route_block(int logits) { return logits == 16 ? 512 : 1024; }
constexpr int kMaxParts = 512;  // blocks whose sums are joined: two a CU, all its wavefronts

// exp(x) for x <= 0, to a few units in the last place: 2^(x log2 e) with what the
// product was rounded by put back.  (Zero below -200; a NaN counts as that: the rows
// that have one get it back from their sum of zero.)
__device__ __forceinline__ float exp_below(float x) {
    x = fmaxf(x, -200.0f);
    const float t = x * 1.44269504f, lost = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269504f, -t));
    const float e = __builtin_amdgcn_exp2f(t);
    return fmaf(e, lost * 0.69314718f, e);
}
// The same where what is made of it is rounded to bf16: as the hardware has it, |x| units
// off, 2^-17 of the value at most, of which a rounding of 2^-9 leaves nothing.  (A routing's
// masses and gates are fp32: they take exp_below, 65536 x 512 bf16 44.8 us for 42.2.)
template <bool ROUGH>
__device__ __forceinline__ float exp_of_logit(float x) {
    if constexpr (ROUGH) return __builtin_amdgcn_exp2f(fmaxf(x, -200.0f) * 1.44269504f);
    else return exp_below(x);
}
// The larger number, or a NaN where there is one.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// v combined with another lane's: lanes change places in pairs 2^STEP apart, or
// mirrored within the next larger group, which a reduction does not tell apart.
// (RING: rotated by 4 and by 8 lanes of 16 instead, for sums over all groups, whose
// lanes are not alike.)
template <int STEP, bool RING, class F>
__device__ __forceinline__ uint32_t with_other(uint32_t v, F&& f) {
    if constexpr (STEP < 4) {
        constexpr int CTRL = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? (RING ? 0x124 : 0x141)
                                                                             : (RING ? 0x128 : 0x140);
        return f(v, uint32_t(__builtin_amdgcn_mov_dpp(int(v), CTRL, 0xF, 0xF, true)));
    } else if constexpr (STEP == 4) {  // rows of 16 lanes: {0, 0, 2, 2} and {1, 1, 3, 3}
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return f(r[0], r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return f(r[0], r[1]);
    }
}
// Over a group's 2^TO lanes, or with FROM over the same lane of all groups; every lane
// has the result.
template <int TO, int FROM = 0, bool RING = false, class F>
__device__ __forceinline__ uint32_t group_reduce(uint32_t v, F&& f) {
    if constexpr (FROM < TO) return group_reduce<TO, FROM + 1, RING>(with_other<FROM, RING>(v, f), f);
    else return v;
}
struct AddBits {
    __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const {
        return __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    }
};
template <int LOG> __device__ __forceinline__ float group_sum(float v) {
    return __uint_as_float(group_reduce<LOG>(__float_as_uint(v), AddBits{}));
}
template <int LOG> __device__ __forceinline__ float groups_sum(float v) {
    return __uint_as_float(group_reduce<6, LOG, true>(__float_as_uint(v), AddBits{}));
}
template <int LOG> __device__ __forceinline__ float group_max(float v) {
    return __uint_as_float(group_reduce<LOG>(__float_as_uint(v), [](uint32_t a, uint32_t b) {
        return __float_as_uint(larger(__uint_as_float(a), __uint_as_float(b)));
    }));
}
template <int LOG> __device__ __forceinline__ uint32_t group_most(uint32_t v) {
    return group_reduce<LOG>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
// The largest of a whole wavefront's lanes, to a scalar register.
__device__ __forceinline__ uint32_t wave_most(uint32_t v) {
    auto step = [&](auto ctrl, auto rows) {
        const uint32_t o = uint32_t(__builtin_amdgcn_update_dpp(0, int(v), decltype(ctrl)::value,
                                                                decltype(rows)::value, 0xF, false));
        v = o > v ? o : v;
    };
    using std::integral_constant;
    const integral_constant<int, 0xF> all{};
    step(integral_constant<int, 0x111>{}, all);     // as wave_reduce's
    step(integral_constant<int, 0x112>{}, all);
    step(integral_constant<int, 0x114>{}, all);
    step(integral_constant<int, 0x118>{}, all);
    step(integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});
    step(integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});
    return uint32_t(__builtin_amdgcn_readlane(int(v), 63));
}
// The largest of ranks; one of 64 bits by its upper and then its lower half.
template <int LOG> __device__ __forceinline__ uint32_t group_best(uint32_t v) {
    if constexpr (LOG == 6) return wave_most(v);
    else return group_most<LOG>(v);
}
template <int LOG> __device__ __forceinline__ uint64_t group_best(uint64_t v) {
    const uint32_t hi = group_best<LOG>(uint32_t(v >> 32));
    const uint32_t lo = group_best<LOG>(uint32_t(v >> 32) == hi ? uint32_t(v) : 0u);
    return uint64_t(hi) << 32 | lo;
}

// A logit and its place as one number: larger for a larger logit, and of equal ones for
// the lower place.  ODD: where a NaN, which is above everything, or a -0, which is 0, may be
// among them.  Up to NONE it is -inf's, an absent expert.  bf16's 16 bits and the place fit 32
// bits.
__device__ __forceinline__ uint32_t ordered(float z) {
    const uint32_t u = __float_as_uint(z);
    return u ^ uint32_t(int32_t(u) >> 31 | int32_t(0x80000000));
}
__device__ __forceinline__ float unordered(uint32_t o) {
    return __uint_as_float(int32_t(o) < 0 ? o ^ 0x80000000u : ~o);
}
template <class T> struct Rank;
template <> struct Rank<uint16_t> {
    using K = uint32_t;
    static constexpr K NONE = 0x007FFFFFu;
    template <bool ODD> static __device__ __forceinline__ K of(float z, uint32_t place) {
        const uint32_t o = ODD && z != z ? 0xFFFF0000u : ordered(ODD ? z + 0.0f : z);
        return (o & 0xFFFF0000u) | (0xFFFFu - place);
    }
    static __device__ __forceinline__ uint32_t place(K k) { return 0xFFFFu - (k & 0xFFFFu); }
    static __device__ __forceinline__ float logit(K k) {
        return __uint_as_float(__float_as_uint(unordered(k)) & 0xFFFF0000u);
    }
};
template <> struct Rank<float> {
    using K = uint64_t;
    static constexpr K NONE = 0x007FFFFFFFFFFFFFull;
    template <bool ODD> static __device__ __forceinline__ K of(float z, uint32_t place) {
        const uint32_t o = ODD && z != z ? 0xFFFFFFFFu : ordered(ODD ? z + 0.0f : z);
        return K(o) << 32 | (0xFFFFFFFFu - place);
    }
    static __device__ __forceinline__ uint32_t place(K k) { return 0xFFFFFFFFu - uint32_t(k); }
    static __device__ __forceinline__ float logit(K k) { return unordered(uint32_t(k >> 32)); }
};

// A lane's P logits from `first` on, as they lie; the rest of a row's last vector, and
// what is behind the row, is not read.
template <class T, int P>
struct Logits {
    static constexpr int VEC = Num<T>::VEC, VECS = P / VEC;
    u32x4 raw[VECS];
    __device__ __forceinline__ void load(const T* row, int first, int E) {
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int left = E - first - i * VEC;
            raw[i] = u32x4{0, 0, 0, 0};
            if (left >= VEC) raw[i] = load_vec(row + first + i * VEC);
            else if (left > 0) raw[i] = load_part(row + first + i * VEC, left);
        }
    }
    // behind the row's end -inf
    __device__ __forceinline__ void get(float* z, int first, int E) const {
#pragma unroll
        for (int i = 0; i < VECS; ++i) Num<T>::unpack(raw[i], z + i * VEC);
        if (E % P) {
#pragma unroll
            for (int i = 0; i < P; ++i) z[i] = first + i < E ? z[i] : -INFINITY;
        } else if (first >= E) {
#pragma unroll
            for (int i = 0; i < P; ++i) z[i] = -INFINITY;
        }
    }
};

// exp of the logits less the largest, and the inverse of their sum: NaN and an infinity, so
// that their product is NaN, where the largest is a NaN or an infinity; zero for no row.
template <bool ROUGH, int LOG, int P>
__device__ __forceinline__ float softmax(const float* z, float top, bool any, float* e) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < P; ++i) {
        e[i] = exp_of_logit<ROUGH>(z[i] - top);
        s += e[i];
    }
    s = group_sum<LOG>(s);
    return any ? 1.0f / s : 0.0f;
}

// Compares and exchanges until the larger are in front: merges of sorted halves, odd and
// even places apart.
template <int P, class V>
__device__ __forceinline__ void sort_falling(V& key) {
#pragma unroll
    for (int size = 1; size < P; size *= 2)
#pragma unroll
        for (int step = size; step > 0; step /= 2)
#pragma unroll
            for (int j = step % size; j + step < P; j += 2 * step)
#pragma unroll
                for (int i = 0; i < step; ++i)
                    if (j + i + step < P && (j + i) / (2 * size) == (j + i + step) / (2 * size)) {
                        const auto a = key[j + i], b = key[j + i + step];
                        key[j + i] = a > b ? a : b;
                        key[j + i + step] = a > b ? b : a;
                    }
}

// The elements behind the first, and a zero.
template <int P, class V>
__device__ __forceinline__ V moved_up(V v) {
    const V zero = 0;
    if constexpr (P == 8) return __builtin_shufflevector(v, zero, 1, 2, 3, 4, 5, 6, 7, 8);
    else return __builtin_shufflevector(v, zero, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 16);
}
// The first of a lane's sorted ranks, as many as can be chosen.
template <int LIST, class V>
__device__ __forceinline__ auto front(V v) {
    if constexpr (LIST == sizeof(V) / sizeof(v[0])) return v;
    else return __builtin_shufflevector(v, v, 0, 1, 2, 3, 4, 5, 6, 7);
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

// A lane's logits are sorted once; each choice is then a reduction over the lanes'
// first ones, and the lane that it came from moves on to its next.  Lane j keeps choice
// j, so gates, counts and stores are made for all of them at once.  The block's sums over its
// rows go to a part of their own, added in order by another launch: no atomics on floats.
// Bound by the vector units, by the ranks' sort and the choices, 43 operations a bf16 logit:
// they are busy for nearly all of the time that 65536 x 512 bf16, k = 8, takes, 44.8 us (a maximum
// over all logits for each choice 129); 16384 x 128 7.6.  fp32's ranks of 64 bits take twice that,
// 92 us, and 10.2.
template <class T, int LOG, int P, int LIST>
__global__ __launch_bounds__(route_block(P)) void route_kernel(const T* logits, RouteArgs a) {
    constexpr int BLOCK = route_block(P);
    using R = Rank<T>;
    using K = typename R::K;
    typedef K V __attribute__((ext_vector_type(P)));
    constexpr int LANES = 1 << LOG, GROUPS = 64 / LANES, WAVES = BLOCK / 64;
    constexpr int WIDE = LANES * P;                     // experts at most
    constexpr int MOST = LIST < P ? LIST : AR_ROUTE_MAX_K;
    constexpr int PICKS = WIDE < MOST ? WIDE : MOST;
    constexpr int SLOTS = (PICKS + LANES - 1) / LANES;  // choices a lane keeps
    __shared__ int32_t hist[WIDE + 1];
    __shared__ float sums[WAVES][WIDE];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> LOG;
    const int sub = lane & (LANES - 1), first = sub * P;
    const int64_t step = int64_t(gridDim.x) * WAVES * GROUPS;
    int64_t r0 = (int64_t(blockIdx.x) * WAVES + wave) * GROUPS;
    Logits<T, P> next;
    uint8_t next_live = 0;
    auto fetch = [&](int64_t r) {
        const bool in = r < a.T;
        next.load(logits + r * a.stride, in ? first : a.E, a.E);
        next_live = in ? (a.live ? a.live[r] : 1) : 0;
    };
    fetch(r0 + group);
    for (int i = threadIdx.x; i <= WIDE; i += BLOCK) hist[i] = 0;
    __syncthreads();
    float mass[P] = {};
    for (; r0 < a.T; r0 += step) {
        const int64_t r = r0 + group;
        const bool in = r < a.T, live = next_live;
        float z[P], e[P];
        next.get(z, first, a.E);
        fetch(r + step);
        // (a vector, not an array: a choice between its elements is one of registers)
        V all;
        K mine[SLOTS];
        bool odd = false;
#pragma unroll
        for (int i = 0; i < P; ++i) odd |= __builtin_amdgcn_classf(z[i], 0x23);  // NaN, -0
        if (__builtin_amdgcn_ballot_w64(odd)) {
#pragma unroll
            for (int i = 0; i < P; ++i) all[i] = R::template of<true>(z[i], uint32_t(first + i));
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i) all[i] = R::template of<false>(z[i], uint32_t(first + i));
        }
        sort_falling<P>(all);
        auto key = front<LIST>(all);
        K best = group_best<LOG>(key[0]);
        const bool any = live && best > R::NONE;
        const float top = R::logit(best), inverse = softmax<false, LOG, P>(z, top, any, e);
#pragma unroll
        for (int i = 0; i < P; ++i) mass[i] = fmaf(e[i], inverse, mass[i]);
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            mine[s] = 0;
            for (int j = 0; j < LANES && s * LANES + j < a.k; ++j) {
                mine[s] = sub == j ? best : mine[s];
                key = key[0] == best ? moved_up<LIST>(key) : key;
                best = group_best<LOG>(key[0]);
            }
        }
        float gate[SLOTS], total = 0.0f;
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            if (!live || mine[s] <= R::NONE) mine[s] = 0;
            gate[s] = mine[s] ? exp_below(R::logit(mine[s]) - top) * inverse : 0.0f;
            total += gate[s];
        }
        float scale = 1.0f;
        if (a.normalize) {
            total = group_sum<LOG>(total);
            scale = any ? 1.0f / total : 0.0f;
        }
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const int j = s * LANES + sub;
            if (j < a.k && in) {
                const int id = mine[s] ? int(R::place(mine[s])) : -1;
                a.ids[r * a.k + j] = id;
                a.gates[r * a.k + j] = gate[s] * scale;
                if (mine[s]) atomicAdd(&hist[id], 1);
            }
        }
        if (sub == 0 && any) atomicAdd(&hist[a.E], 1);
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const float m = groups_sum<LOG>(mass[i]);       // the wavefront's rows
        if (group == 0) sums[wave][first + i] = m;
    }
    __syncthreads();
    int32_t* const counts = a.counts + int64_t(blockIdx.x) * (a.E + 1);
    float* const masses = a.mass + int64_t(blockIdx.x) * a.E;
    for (int e = threadIdx.x; e <= a.E; e += BLOCK) {
        counts[e] = hist[e];
        if (e == a.E) break;
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) s += sums[i][e];
        masses[e] = s;
    }
}

// The blocks' counts and sums, added in order: 16 experts a block of 64 x 16 lanes,
// each lane every 64th part, all of its loads in flight together.  512 parts of 512 experts
// 4.8 us.
__global__ __launch_bounds__(1024) void route_join_kernel(int parts, int E, const int32_t* counts,
                                                          const float* mass, int32_t* counts_out,
                                                          float* mass_out) {
    __shared__ int32_t c[64][16];
    __shared__ float m[64][16];
    const int e = int(blockIdx.x) * 16 + (threadIdx.x & 15), at = threadIdx.x >> 4;
    int32_t n = 0;
    float s = 0.0f;
    int32_t x[kMaxParts / 64];
    float y[kMaxParts / 64];
#pragma unroll
    for (int i = 0; i < kMaxParts / 64; ++i) {
        const int64_t part = at + 64 * i;
        x[i] = part < parts && e <= E ? counts[part * (E + 1) + e] : 0;
        y[i] = part < parts && e < E ? mass[part * E + e] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kMaxParts / 64; ++i) {
        n += x[i];
        s += y[i];
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

// The gradient, and in the last block the loss.  What is chosen reaches the lanes that
// hold its logits through LDS: a place a logit, with the choice's number (0: none) and
// its gate's gradient.  65536 x 512 bf16, k = 8: 35 us, 3.9 TB/s, bound by the vector units
// (with every choice compared at every logit 87); fp32 52, 5.2 TB/s.  At most five blocks a CU, all
// that fit its registers: 16384 blocks, each of which gets the slopes first, took 87.
template <class T, int LOG, int P>
__global__ __launch_bounds__(kBalanceBlock) void balance_kernel(const T* logits, T* grad, BalanceArgs a) {
    constexpr int VEC = Num<T>::VEC;
    constexpr int LANES = 1 << LOG, GROUPS = 64 / LANES, WAVES = kBalanceBlock / 64, WIDE = LANES * P;
    constexpr int PICKS = WIDE < AR_ROUTE_MAX_K ? WIDE : AR_ROUTE_MAX_K;
    constexpr int SLOTS = (PICKS + LANES - 1) / LANES;
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) int chosen[WAVES][64 * P];
    __shared__ __attribute__((aligned(16))) float wanted[WAVES][64 * P];
    if (blockIdx.x == gridDim.x - 1) {
        if (threadIdx.x < 64) loss_of(a);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane >> LOG;
    const int sub = lane & (LANES - 1), first = sub * P;
    const int64_t step = int64_t(gridDim.x - 1) * WAVES * GROUPS;
    int64_t r0 = (int64_t(blockIdx.x) * WAVES + wave) * GROUPS;
    Logits<T, P> next;
    int next_id[SLOTS];
    int64_t next_first = -1;
    float next_g[SLOTS];
    auto fetch = [&](int64_t r) {
        const bool in = r < a.T;
        next.load(logits + r * a.stride, in ? first : a.E, a.E);
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            const int j = s * LANES + sub;
            const int64_t id = in && j < a.k ? a.ids[r * a.k + j] : -1;
            next_id[s] = id >= 0 && id < a.E ? int(id) : -1;
            next_g[s] = in && j < a.k && a.dgates ? a.dgates[r * a.k + j] : 0.0f;
        }
        next_first = in ? a.ids[r * a.k] : -1;
    };
    fetch(r0 + group);
    // the slopes of the loss: coefficient E counts_e / (k N^2), all counts in flight together.
    // (Made in 64 bits and rounded once: in 32 the factor before counts_e is infinite or
    // denormal for coefficients whose slopes are neither.)
    Logits<float, P> counts;
    counts.load(reinterpret_cast<const float*>(a.counts), first, a.E);
    const double n = double(a.counts[a.E]);
    const double unit = n > 0.0 ? double(a.coefficient) * a.E / a.k / n / n : 0.0;
    float slope[P];
#pragma unroll
    for (int i = 0; i < P; ++i) slope[i] = float(double(int32_t(counts.raw[i / 4][i % 4])) * unit);
    const float plain = a.normalize ? 0.0f : 1.0f;
    for (; r0 < a.T; r0 += step) {
        const int64_t r = r0 + group;
        const bool in = r < a.T, live = next_first >= 0;
        float z[P], p[P];
        next.get(z, first, a.E);
        int id[SLOTS];
        float g[SLOTS];
#pragma unroll
        for (int s = 0; s < SLOTS; ++s) {
            id[s] = next_id[s];
            g[s] = next_g[s];
        }
        fetch(r + step);
        float top = z[0];
#pragma unroll
        for (int i = 1; i < P; ++i) top = larger(top, z[i]);
        top = group_max<LOG>(top);
        const bool any = live && top != -INFINITY;
        const float inverse = softmax<sizeof(T) == 2, LOG, P>(z, top, any, p);
#pragma unroll
        for (int i = 0; i < P; ++i) p[i] *= inverse;
        // wants: the sum of the gates' gradients, of those chosen `times` times
        float times[P], wants[P];
#pragma unroll
        for (int i = 0; i < P; ++i) times[i] = wants[i] = 0.0f;
        if (a.dgates) {
            AR_LDS int* const number = (AR_LDS int*)chosen[wave] + group * WIDE;
            AR_LDS float* const want = (AR_LDS float*)wanted[wave] + group * WIDE;
            wave_sync();
#pragma unroll
            for (int i = 0; i < P; i += 4) {
                *(AR_LDS f32x4*)(want + first + i) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (a.normalize) *(AR_LDS i32x4*)(number + first + i) = i32x4{0, 0, 0, 0};
            }
            wave_sync();
            bool twice = false;
#pragma unroll
            for (int s = 0; s < SLOTS; ++s)
                if (id[s] >= 0) {
                    number[id[s]] = s * LANES + sub + 1;
                    want[id[s]] = g[s];
                }
            wave_sync();
#pragma unroll
            for (int s = 0; s < SLOTS; ++s)
                if (id[s] >= 0) twice |= number[id[s]] != s * LANES + sub + 1;
            if (!__builtin_amdgcn_ballot_w64(twice)) {
#pragma unroll
                for (int i = 0; i < P; i += 4) {
                    const f32x4 w = *(AR_LDS f32x4*)(want + first + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) wants[i + e] = w[e];
                    if (a.normalize) {
                        const i32x4 m = *(AR_LDS i32x4*)(number + first + i);
#pragma unroll
                        for (int e = 0; e < 4; ++e) times[i + e] = m[e] ? 1.0f : 0.0f;
                    }
                }
            } else if (in) {  // an expert more than once in a row: every choice at every lane
                for (int j = 0; j < a.k; ++j) {
                    const int64_t rel = a.ids[r * a.k + j] - first;
                    const float w = a.dgates[r * a.k + j];
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        wants[i] += rel == i && first + i < a.E ? w : 0.0f;
                        times[i] += rel == i && first + i < a.E ? 1.0f : 0.0f;
                    }
                }
            }
        }
        float d[P], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < P; ++i) {
            d[i] = fmaf(wants[i], plain, slope[i]);
            sum = fmaf(p[i], d[i], sum);
        }
        sum = group_sum<LOG>(sum);
#pragma unroll
        for (int i = 0; i < P; ++i) d[i] = p[i] * (d[i] - sum);
        if (a.normalize && a.dgates) {
            float total = 0.0f, dot = 0.0f;
#pragma unroll
            for (int i = 0; i < P; ++i) {
                total = fmaf(p[i], times[i], total);
                dot = fmaf(p[i], wants[i], dot);
            }
            total = group_sum<LOG>(total);
            const float share = total > 0.0f ? 1.0f / total : 0.0f;
            dot = group_sum<LOG>(dot) * share;
#pragma unroll
            for (int i = 0; i < P; ++i) d[i] = fmaf(p[i] * share, fmaf(-times[i], dot, wants[i]), d[i]);
        }
        if (!in) continue;
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

// Lanes that hold a row: 8 logits each, 16 of the widest.
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
    else if (E <= kWideRow) go(std::integral_constant<int, 6>{}, eight);
    else go(std::integral_constant<int, 6>{}, std::integral_constant<int, 16>{});
}
int group_log(int64_t E) {
    int log = 0;
    while (log < 6 && (8 << log) < E) ++log;
    return log;
}

// Blocks of a routing: as many as the rows fill, but one where its passes over its
// wavefronts' rows take less than a call with the join does, which are fewer for fp32's ranks
// of 64 bits, and for many choices or all of few experts.  us of a call, and of its launches in a
// graph, in one block and with the join:
//   192 x 128, k = 8   bf16, 3 passes: 13.1 and 18.0, 11.7 and 8.2; fp32: 16.3 and 17.7, 16.1 and 9.6
//   128 x 128, k = 8   2 passes: bf16 13.3 and 17.9, 8.7 and 8.2; fp32 13.2 and 17.8, 11.5 and 9.6
//   128 x 128, k = 32  bf16, 2 passes: 14.5 and 17.7, 14.1 and 10.8; fp32: 23.0 and 17.6, 23.0 and 15.6
//   16 x 1024, k = 32  bf16, 2 passes: 14.3 and 17.8, 13.7 and 12.6; fp32: 23.2 and 17.6, 23.0 and 15.9
//   2048 x 8, k = 8    bf16, 2 passes: 15.8 and 17.7, 15.7 and 10.7; fp32: 15.6 and 17.5, 15.3 and 11.5
// (In calls alone fp32's third pass of k = 8, and its second of 8 of 8, gain little beside what
// they cost a graph; bf16's third of 8 of 8 takes 20.9 and 16.3.)
int64_t parts_of(int32_t dtype, int64_t T, int64_t E, int64_t k, int log) {
    const int64_t rows = (route_block(E > kWideRow ? 16 : 8) / 64) * (64 >> log);
    const int64_t passes = (dtype == AR_F32 ? 1 : 2) + (k <= 8 && k < E ? 1 : 0);
    return T <= passes * rows ? 1 : std::min<int64_t>(kMaxParts, ceil_div(T, rows));
}

// Many bf16 rows of which up to 8 are chosen: 16 logits a lane of half as many lanes, of whose
// ranks the first 8 can be chosen.  A wavefront then has twice the rows for each of its
// reductions, but there are half as many wavefronts: it takes longer until blocks of 8 logits a
// lane are more than the card's 256 CUs, of long rows more than four a CU.  us of the launches,
// with 8 and with 16 logits a lane, k = 8:
//   16384 x 128 (256 blocks) 10.1 and 11.6, 16547 x 128 (259) 14.0 and 11.7, 24576 x 128 14.7 and
//   12.0, 40960 x 128 18.9 and 16.0, 65536 x 128 22.3 and 17.5, 66 experts alike
//   8192 x 256 (256 blocks) 9.3 and 11.4, 16384 x 256 13.6 and 12.3, but 24576 x 256 15.9 and
//   16.7, 32768 x 256 (1024) 19.1 and 17.7, 65536 x 256 29.6 and 26.2
//   4096 x 512 (256 blocks) 9.5 and 11.4, 8192 x 512 13.9 and 12.4, but 12288 x 512 16.1 and
//   17.3, 16384 x 512 (1024) 19.2 and 18.6, 32768 x 512 29.2 and 26.7, 65536 x 512 50.0 and 44.1
// (k = 2: 128 experts alike; 32768 x 512 22.6 and 23.0, 65536 x 512 37.4 and 36.8.)
bool doubled(int32_t dtype, int64_t T, int64_t E, int64_t k, int log) {
    const int64_t rows = (route_block(8) / 64) * (64 >> log);
    return dtype == AR_BF16 && k <= 8 && E > 64 && E <= kWideRow && T > (E <= 128 ? 256 : 1024) * rows;
}
int64_t part_bytes(int64_t T, int64_t E, int64_t k) {
    const int64_t parts = parts_of(AR_F32, T, E, k, group_log(E));  // (bf16 has as many or fewer)
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
    *bytes = part_bytes(T, E, k);
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
    const int64_t need = part_bytes(T, E, k);
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
    const bool twice = doubled(dtype, T, E, k, group_log(E));
    const int64_t parts = parts_of(dtype, T, E, k, group_log(E) - (twice ? 1 : 0));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    int32_t* const part_counts = static_cast<int32_t*>(workspace);
    float* const part_mass = reinterpret_cast<float*>(part_counts + parts * (E + 1));
    const RouteArgs a{T, logits_stride, int(E), int(k), normalize, live, ids, gates,
                      parts > 1 ? part_counts : counts, parts > 1 ? part_mass : mass};
    auto go = [&](auto zero) {
        using U = decltype(zero);
        by_width(int(E), [&](auto log, auto p) {
            constexpr int LOG = decltype(log)::value, P = decltype(p)::value;
            auto run = [&](auto kernel, int list) {
                hipLaunchKernelGGL(kernel, dim3(unsigned(parts)), dim3(route_block(list)), 0, st,
                                   static_cast<const U*>(logits), a);
            };
            if constexpr (sizeof(U) == 2 && P == 8 && LOG > 3) {
                if (twice) return run(route_kernel<U, LOG - 1, 16, 8>, 16);
            }
            run(route_kernel<U, LOG, P, P>, P);
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
    if (!std::isfinite(coefficient))
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
            const int64_t blocks = ceil_div(T, (kBalanceBlock / 64) * (64 >> decltype(log)::value));
            hipLaunchKernelGGL((balance_kernel<U, decltype(log)::value, decltype(p)::value>),
                               dim3(unsigned(std::min<int64_t>(blocks, 1280)) + 1), dim3(kBalanceBlock),
                               0, st,
                               static_cast<const U*>(logits), static_cast<U*>(grad), a);
        });
        return launch_status("balance loss");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}
