// Distillation from a teacher's top logits, forward and backward.
//
// In units of log2, with c = log2(e) / temperature and any base m near the
// row's maximum:
//   S = sum 2^((z - m) c),  log2 q_j = (z_j - m) c - log2 S
// and the same for the teacher's entries; the loss and the gradient follow
// from these.  Over a row (z - m) c is computed as z c - r with r = m c
// rounded, one fused multiply-add; what that is off by, m c - r, is the same
// for every z, known exactly by one more, and taken out of the sum.  m need
// not be the maximum, only near enough for the sum to stay in range: a
// wavefront takes the largest of the first vectors it holds, and looks for its
// true maximum, and takes differences, only where its sum shows that this
// would not do (a mask of the type's lowest value throughout, say).
//
// Bound by memory: the row read once and the gradient written once.  Two forms:
//  * kept: a block takes rows in turn and holds each in registers between the
//    sum and the gradient, so that it is read once; as it stores the gradient
//    it loads the next row into the registers that become free.  4096 rows of
//    131072 bf16 and their gradient: 467 us (473 the median of a trace), 4.3 of the
//    6.2 TB/s of a large copy, the vector units 45 % busy; 1021 rows of 32003 fp32,
//    the loss alone: 29 us, 4.5 TB/s;
//  * split: rows longer than a block holds, and rows too few to fill the card.
//    Each row is cut into parts of a block; one launch leaves the parts' sums,
//    a second one reads the parts again and writes the gradient.  4096 rows of
//    140000 bf16: 646 us, 5.3 TB/s of three passes; 8 rows of 131072, the loss
//    alone: 4 us each.
#include <algorithm>
#include <cmath>

#include "replica.hpp"

namespace arp {
namespace {

// Vectors of a row that a thread keeps: 64 registers, which leaves a CU its 16
// wavefronts.  (With 1024 threads three values that hold for all rows are spilled,
// written once and read once a row.)
constexpr int kKeep = 16;

__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// The sum S of 2^((z - m) c) over some elements; an empty one is (-inf, 0).
struct PartSum {
    float m, S;
};

// Whether z c - r with r = m c is near enough to (z - m) c.
__device__ __forceinline__ bool near_base(float r) { return fabsf(r) < 0x1p24f; }

struct DistillArgs {
    const int64_t* ids;
    const float* weights;
    float* loss;
    int64_t T, V, K;
    int64_t logits_stride, teacher_stride, ids_stride, grad_stride;
    float c;            // log2(e) / temperature
    float temperature;
    // split form
    int64_t first, parts, part;  // the launch's first row; parts of a row, elements of one
    PartSum* sums;               // of each part of each row of the launch
    float* at;                   // the student's logits at the entries, K a row
};

// The sum of n parts.
__device__ __forceinline__ PartSum join(const PartSum* part, int64_t n, float c) {
    PartSum all{-INFINITY, 0.0f};
    for (int64_t i = 0; i < n; i += 64) {
        const int64_t at = i + (threadIdx.x & 63);
        const PartSum p = at < n ? part[at] : PartSum{-INFINITY, 0.0f};
        const float high = fmaxf(all.m, wave_max(p.m));
        // (an empty one adds nothing, not 0 * inf)
        const float s = wave_sum(p.S == 0.0f ? 0.0f : p.S * pow2((p.m - high) * c));
        all.S = (all.S == 0.0f ? 0.0f : all.S * pow2((all.m - high) * c)) + s;
        all.m = high;
    }
    return all;
}

// A block's part of a row, elements [0, len) of z, in its threads' registers:
// vectors i * B + thread, and up to VEC - 1 elements at the end one a thread.
// A thread with no vector in the last round holds the last one once more, and
// takes it as -inf.
template <class T, int B>
struct Part {
    static constexpr int VEC = Num<T>::VEC;
    static constexpr int64_t LEN = int64_t(B) * kKeep * VEC;
    u32x4 v[kKeep];
    float last;
    int vecs, tail, rounds;  // whole vectors, elements after them, rounds of B vectors
    bool beyond;             // this thread has no vector in the last round
    uint32_t off, off_last;  // the thread's elements within a round, and the last one

    __device__ __forceinline__ void extent(int64_t len) {
        vecs = int(len / VEC);
        tail = int(len % VEC);
        rounds = (vecs + B - 1) / B;
        last = -INFINITY;
        beyond = (rounds - 1) * B + int(threadIdx.x) >= vecs;
        off = threadIdx.x * VEC;
        off_last = beyond ? uint32_t(vecs - 1 - (rounds - 1) * B) * VEC : off;
    }
    __device__ __forceinline__ u32x4 vec_of(const T* z, int i) const {
        return load_vec(z + i * B * VEC + (i == rounds - 1 ? off_last : off));
    }
    __device__ __forceinline__ void load(const T* z) {
#pragma unroll
        for (int i = 0; i < kKeep; ++i)
            if (i < rounds) v[i] = vec_of(z, i);
        last = int(threadIdx.x) < tail ? Num<T>::up(z[vecs * VEC + int(threadIdx.x)]) : -INFINITY;
    }
    // Within a loop over rows: what follows from the extent is worked out where
    // it is used, not kept in registers for all rounds of the loop.
    __device__ __forceinline__ void again() { asm volatile("" : "+s"(rounds)); }
    __device__ __forceinline__ void get(int i, float* x) const {
        constexpr uint32_t none = sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
        Num<T>::unpack(i == rounds - 1 && beyond ? u32x4{none, none, none, none} : v[i], x);
    }
    template <class F>
    __device__ __forceinline__ void each(F&& f) const {
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            if (i < rounds) {
                float x[VEC];
                get(i, x);
#pragma unroll
                for (int e = 0; e < VEC; ++e) f(x[e]);
            }
        }
        f(last);
    }
    // This wavefront's sum (the same in every lane).
    __device__ __forceinline__ PartSum sum(float c) const {
        float m = last;
        if (rounds > 0) {
            float x[VEC];
            get(0, x);
#pragma unroll
            for (int e = 0; e < VEC; ++e) m = fmaxf(m, x[e]);
        }
        m = wave_max(m);
        const float r = m * c;
        if (near_base(r)) {
            float S[2] = {0.0f, 0.0f};
            int n = 0;
            // (less +inf, what a thread holds once more adds 0; it is finite, or
            // the sum is of no use anyway)
            const float r_last = beyond ? INFINITY : r;
#pragma unroll
            for (int i = 0; i < kKeep; ++i) {
                if (i < rounds) {
                    float x[VEC];
                    Num<T>::unpack(v[i], x);
                    const float ri = i == rounds - 1 ? r_last : r;
#pragma unroll
                    for (int e = 0; e < VEC; ++e) S[n++ & 1] += pow2(fmaf(x[e], c, -ri));
                }
            }
            S[0] += pow2(fmaf(last, c, -r));
            const float s = wave_sum(S[0] + S[1]);
            // (the largest of the sample adds 1)
            if (s >= 0.5f && s < 0x1p60f) return {m, s * pow2(-fmaf(m, c, -r))};
        }
        // by the true maximum: the sample was far from it, or empty, or there
        // is a NaN
        m = -INFINITY;
        each([&](float z) { m = fmaxf(m, z); });
        m = wave_max(m);
        const float base = m == -INFINITY ? 0.0f : m;
        float s = 0.0f;
        each([&](float z) { s += pow2((z - base) * c); });
        s = wave_sum(s);
        return {s == 0.0f ? -INFINITY : base, s};
    }
    // g = f(z), where g is given; then the registers take `next`, where that is.
    template <class F>
    __device__ __forceinline__ void store_load(T* g, const T* next, F&& f) {
#pragma unroll
        for (int i = 0; i < kKeep; ++i) {
            if (i < rounds) {
                if (g) {
                    float x[VEC];
                    Num<T>::unpack(v[i], x);
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[e] = f(x[e]);
                    if (i < rounds - 1 || !beyond)
                        store_vec(g + (i * B + int(threadIdx.x)) * VEC, Num<T>::pack(x));
                }
                if (next) v[i] = vec_of(next, i);
            }
        }
        if (int(threadIdx.x) < tail) {
            if (g) g[vecs * VEC + int(threadIdx.x)] = Num<T>::down(f(last));
            if (next) last = Num<T>::up(next[vecs * VEC + int(threadIdx.x)]);
        }
    }
    // g = f(z) with z from memory.
    template <class F>
    __device__ __forceinline__ void store_from(T* g, const T* z, F&& f) const {
        for (int i = int(threadIdx.x); i < vecs; i += B) {
            float x[VEC];
            Num<T>::unpack(load_vec(z + i * VEC), x);
            for (int e = 0; e < VEC; ++e) x[e] = f(x[e]);
            store_vec(g + i * VEC, Num<T>::pack(x));
        }
        if (int(threadIdx.x) < tail) g[vecs * VEC + int(threadIdx.x)] = Num<T>::down(f(last));
    }
    // The thread that holds element j.
    __device__ __forceinline__ int owner(int j) const {
        return j < vecs * VEC ? (j / VEC) % B : j - vecs * VEC;
    }
    __device__ __forceinline__ void store_zero(T* g) const {
        for (int i = int(threadIdx.x); i < vecs; i += B) store_vec(g + i * VEC, u32x4{0, 0, 0, 0});
        if (int(threadIdx.x) < tail) g[vecs * VEC + int(threadIdx.x)] = T(0);
    }
};

// A row's statistics.
struct Row {
    float m, S, c;
    __device__ __forceinline__ float log2q(float z) const {
        return (z - m) * c - __builtin_amdgcn_logf(S);
    }
};

// The teacher's entries of a row, in LDS, one a thread at a time.
struct Entries {
    int32_t* id;  // -1 if absent
    float* p;     // the teacher's logit, then p
    float* z;     // the student's logit
};

template <int B>
struct Shared {
    PartSum part[B / 64];
    float term[B / 64];
    int any[B / 64];
};

// Reads the entries; false if none is present (the same for every thread).
// `logit(k, id)` is the student's logit at entry k.
template <class S, int B, class F>
__device__ __forceinline__ bool read_entries(const DistillArgs& a, int64_t t, const S* teacher,
                                             const Entries& e, F&& logit) {
    int any = 0;
    for (int64_t k = threadIdx.x; k < a.K; k += B) {
        const int64_t id = a.ids[t * a.ids_stride + k];
        const float s = Num<S>::up(teacher[t * a.teacher_stride + k]);
        const bool is = id >= 0 && id < a.V && s != -INFINITY;
        e.id[k] = is ? int32_t(id) : -1;
        e.p[k] = s;
        e.z[k] = is ? logit(k, id) : 0.0f;
        any |= is;
    }
    return __syncthreads_or(any) != 0;
}

// The entries' p, by differences to their largest; the row's loss, with
// scale = weight * temperature.  The difference of the logits is taken in their
// own units and each term scaled before the sum: a student's logit of the type's
// lowest value, which is beyond fp32 in units of log2, leaves the loss finite.
// By the whole block, or, if `alone`, by its first wavefront.
template <int B>
__device__ __forceinline__ float finish_entries(const DistillArgs& a, const Entries& e,
                                                const Row& row, float scale, Shared<B>& sh,
                                                bool alone) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t step = alone ? 64 : B;
    auto all = [&](float v, bool max) {
        v = max ? wave_max(v) : wave_sum(v);
        if (alone) return v;
        __syncthreads();
        if (lane == 0) sh.term[w] = v;
        __syncthreads();
        v = sh.term[0];
        for (int i = 1; i < B / 64; ++i) v = max ? fmaxf(v, sh.term[i]) : v + sh.term[i];
        return v;
    };
    float top = -INFINITY, sum = 0.0f, loss = 0.0f;
    for (int64_t k = threadIdx.x; k < a.K; k += step)
        if (e.id[k] >= 0) top = fmaxf(top, e.p[k]);
    top = all(top, true);
    for (int64_t k = threadIdx.x; k < a.K; k += step)
        if (e.id[k] >= 0) sum += pow2((e.p[k] - top) * a.c);
    sum = all(sum, false);
    const float ls = __builtin_amdgcn_logf(sum);
    // temperature (ln S - ln sum): what log p - log q has beside the logits
    const float sums = (__builtin_amdgcn_logf(row.S) - ls) * 0.6931471805599453f * a.temperature;
    for (int64_t k = threadIdx.x; k < a.K; k += step) {
        if (e.id[k] < 0) continue;
        const float s = e.p[k] - top, p = pow2(s * a.c - ls);
        e.p[k] = p;
        if (p != 0.0f) loss += scale * (p * (s - (e.z[k] - row.m) + sums));
    }
    return all(loss, false);
}

// The gradient at the entries in [lo, hi): every entry with an id stores the
// same, less the p of all of them.
template <class T, int B>
__device__ __forceinline__ void store_entries(const DistillArgs& a, const Entries& e,
                                              const Row& row, float scale, int64_t lo, int64_t hi,
                                              T* g) {
    for (int64_t k = threadIdx.x; k < a.K; k += B) {
        const int32_t id = e.id[k];
        if (id < lo || id >= hi || id < 0) continue;
        float p = 0.0f;
        for (int64_t j = 0; j < a.K; ++j)
            if (e.id[j] == id) p += e.p[j];
        g[id] = Num<T>::down(scale * (pow2(row.log2q(e.z[k])) - p));
    }
}

// The gradient of a part (z, to g; where g is given), and then the registers'
// next contents.
template <class T, int B>
__device__ __forceinline__ void store_gradient(Part<T, B>& part, const Row& row, float scale,
                                               const T* z, T* g, const T* next) {
    const float r = row.m * row.c;
    if (g && !near_base(r)) {  // rare: not worth registers
        const float f = scale / row.S;
        part.store_from(g, z, [&](float x) { return f * pow2((x - row.m) * row.c); });
        g = nullptr;
    }
    const float f = scale / row.S * pow2(-fmaf(row.m, row.c, -r));
    part.store_load(g, next, [&](float x) { return f * pow2(fmaf(x, row.c, -r)); });
}

// What a thread reads ahead of a row: its weight, and the thread's entry.
struct Ahead {
    float weight;
    int64_t id;
    float s;
};
template <class S>
__device__ __forceinline__ Ahead look_ahead(const DistillArgs& a, int64_t t, const S* teacher) {
    Ahead h{0.0f, -1, 0.0f};
    if (t >= a.T) return h;
    h.weight = a.weights ? a.weights[t] : 1.0f;
    if (h.weight != 0.0f && int64_t(threadIdx.x) < a.K) {
        h.id = a.ids[t * a.ids_stride + threadIdx.x];
        h.s = Num<S>::up(teacher[t * a.teacher_stride + threadIdx.x]);
    }
    return h;
}

template <class T, class S, int B>
__global__ __launch_bounds__(B, 4) void kept_kernel(DistillArgs a, const T* logits, const S* teacher,
                                                 T* grad) {
    extern __shared__ char lds[];
    __shared__ Shared<B> sh;
    __shared__ int32_t head[B];  // the entries whose elements a thread stores, chained
    const Entries e{reinterpret_cast<int32_t*>(lds), reinterpret_cast<float*>(lds) + a.K,
                    reinterpret_cast<float*>(lds) + 2 * a.K};
    int32_t* const chain = reinterpret_cast<int32_t*>(lds) + 3 * a.K;
    // few entries are the first wavefront's, and the others go on meanwhile
    const bool alone = a.K <= 64;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, tid = threadIdx.x;
    Part<T, B> part;
    part.extent(a.V);
    Ahead now{0.0f, -1, 0.0f};
    // (the first round only loads the first row)
    for (int64_t t = int64_t(blockIdx.x) - gridDim.x; t < a.T; t += gridDim.x) {
        part.again();
        const T* const z = logits + t * a.logits_stride;
        const int64_t tn = t + gridDim.x;
        T* g = grad && t >= 0 ? grad + t * a.grad_stride : nullptr;
        const float weight = now.weight, scale = weight * a.temperature;
        const Ahead was = now;
        now = look_ahead(a, tn, teacher);
        Row row{};
        bool live = false;
        if (weight != 0.0f) {
            // the thread's first entry; the student's logit there arrives during the sum
            float zs = 0.0f;
            const bool is0 = was.id >= 0 && was.id < a.V && was.s != -INFINITY;
            if (is0) zs = Num<T>::up(z[was.id]);
            const PartSum own = part.sum(a.c);
            if (lane == 0) sh.part[w] = own;
            head[tid] = -1;
            int any = is0;
            if (tid < a.K) {
                e.id[tid] = is0 ? int32_t(was.id) : -1;
                e.p[tid] = was.s;
                e.z[tid] = zs;
            }
            for (int64_t k = tid + B; k < a.K; k += B) {
                const int64_t id = a.ids[t * a.ids_stride + k];
                const float s = Num<S>::up(teacher[t * a.teacher_stride + k]);
                const bool is = id >= 0 && id < a.V && s != -INFINITY;
                e.id[k] = is ? int32_t(id) : -1;
                e.p[k] = s;
                e.z[k] = is ? Num<T>::up(z[id]) : 0.0f;
                any |= is;
            }
            const uint64_t some = __ballot(any);
            if (lane == 0) sh.any[w] = some != 0;
            __syncthreads();
            const PartSum s = join(sh.part, B / 64, a.c);
            row = Row{s.m, s.S, a.c};
            live = s.S != 0.0f && __ballot(lane < B / 64 ? sh.any[lane % (B / 64)] : 0) != 0;
        }
        if (live) {
            if (!alone || w == 0) {
                const float loss = finish_entries<B>(a, e, row, scale, sh, alone);
                if (tid == 0) a.loss[t] = loss;
                if (!alone) __syncthreads();
                for (int64_t k = tid; g && k < a.K; k += alone ? 64 : B) {
                    const int32_t id = e.id[k];
                    if (id < 0) continue;
                    // less the p of every entry with this id: each stores the same
                    float p = 0.0f;
                    for (int64_t j = 0; j < a.K; ++j)
                        if (e.id[j] == id) p += e.p[j];
                    e.z[k] = scale * (pow2(row.log2q(e.z[k])) - p);
                    chain[k] = atomicExch(&head[part.owner(id)], int32_t(k));
                }
            }
        } else if (t >= 0) {
            if (tid == 0) a.loss[t] = 0.0f;
            if (g) part.store_zero(g);
        }
        store_gradient(part, row, scale, z, live ? g : nullptr,
                       now.weight != 0.0f ? logits + tn * a.logits_stride : nullptr);
        __syncthreads();
        if (live && g) {
            // The entries' elements once more, each by the thread that has just
            // stored what lies around it, so that these stores come second.
            for (int32_t k = head[tid]; k >= 0; k = chain[k]) g[e.id[k]] = Num<T>::down(e.z[k]);
        }
        __syncthreads();  // LDS is free again
    }
}

// Split form, first launch: the parts' sums, and the student's logits at the
// entries (the second launch may write over them).
template <class T, int B>
__global__ __launch_bounds__(B) void parts_kernel(DistillArgs a, const T* logits) {
    __shared__ Shared<B> sh;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t i = blockIdx.x / a.parts, t = a.first + i, j = blockIdx.x % a.parts;
    if (a.weights && a.weights[t] == 0.0f) return;
    const T* const z = logits + t * a.logits_stride;
    if (j == 0) {
        for (int64_t k = threadIdx.x; k < a.K; k += B) {
            const int64_t id = a.ids[t * a.ids_stride + k];
            a.at[i * a.K + k] = id >= 0 && id < a.V ? Num<T>::up(z[id]) : 0.0f;
        }
    }
    Part<T, B> part;
    part.extent(a.V - j * a.part < a.part ? a.V - j * a.part : a.part);
    part.load(z + j * a.part);
    const PartSum own = part.sum(a.c);
    if (lane == 0) sh.part[w] = own;
    __syncthreads();
    const PartSum s = join(sh.part, B / 64, a.c);
    if (threadIdx.x == 0) a.sums[blockIdx.x] = s;
}

// Split form, second launch: every part's block joins its row's sums; the
// first one stores the loss, each its part of the gradient.
template <class T, class S, int B>
__global__ __launch_bounds__(B) void split_kernel(DistillArgs a, const T* logits, const S* teacher,
                                                  T* grad) {
    extern __shared__ char lds[];
    __shared__ Shared<B> sh;
    const Entries e{reinterpret_cast<int32_t*>(lds), reinterpret_cast<float*>(lds) + a.K,
                    reinterpret_cast<float*>(lds) + 2 * a.K};
    const int64_t blocks = grad ? a.parts : 1;  // a row's
    const int64_t i = blockIdx.x / blocks, t = a.first + i, j = blockIdx.x % blocks;
    const int64_t lo = j * a.part, hi = a.V - lo < a.part ? a.V : lo + a.part;
    const T* const z = logits + t * a.logits_stride + lo;
    T* const g = grad ? grad + t * a.grad_stride : nullptr;
    const float weight = a.weights ? a.weights[t] : 1.0f;
    Part<T, B> part;
    part.extent(hi - lo);
    Row row{};
    bool live = weight != 0.0f;
    if (live) {
        if (g) part.load(z);
        live = read_entries<S, B>(a, t, teacher, e, [&](int64_t k, int64_t) { return a.at[i * a.K + k]; });
    }
    if (live) {
        const PartSum s = join(a.sums + i * a.parts, a.parts, a.c);
        row = Row{s.m, s.S, a.c};
        live = s.S != 0.0f;
    }
    if (!live) {
        if (threadIdx.x == 0 && j == 0) a.loss[t] = 0.0f;
        if (g) part.store_zero(g + lo);
        return;
    }
    const float scale = weight * a.temperature;
    const float loss = finish_entries<B>(a, e, row, scale, sh, false);
    if (threadIdx.x == 0 && j == 0) a.loss[t] = loss;
    if (!g) return;
    store_gradient(part, row, scale, z, g + lo, static_cast<const T*>(nullptr));
    __syncthreads();  // the entries' elements are written once more, after these
    store_entries<T, B>(a, e, row, scale, lo, hi, g);
}

// ------------------------------------------------------------- launches

constexpr int kSplitBlock = 256;
// Rows from which each takes a block of its own: fewer leave CUs without one.
// Kept against split, on the device: 8 rows of 131072 bf16 18.7 and 10.7 us, 128
// rows 25.1 and 23.7, 192 rows 34 and 38, 256 rows 37 and 49; of 32000 bf16 8 rows
// 12.9 and 9.7 us, 128 rows 14.5 and 14.1.
constexpr int64_t kKeptRows = 192;
// Logits of one pair of launches, which bounds the parts' workspace.  Pairs so
// short that the second launch finds its rows in the 256 MiB last-level cache
// are slower: 4096 rows of 140000 bf16 646 us as one pair, 706 in pairs of
// 400 MiB, 753 of 192, 795 of 96.
constexpr int64_t kSplitBytes = int64_t(4) << 30;

struct Form {
    bool kept;
    int64_t part, parts, rows;  // split form: elements a part, parts a row, rows a launch
};

Form form_of(int64_t T, int64_t V, int esize) {
    const int64_t vec = 16 / esize;
    Form f{};
    f.kept = T >= kKeptRows && V <= 1024 * kKeep * vec;
    if (V <= 64 * kKeep * vec) f.kept = true;  // a wavefront holds the row
    // as many rounds as a thread keeps, fewer where that leaves CUs without a
    // part (between 256 and 1024 parts as a target no difference was measured)
    int64_t rounds = kKeep;
    while (rounds > 1 && T * ceil_div(V, kSplitBlock * vec * rounds) < 1024) rounds /= 2;
    f.part = kSplitBlock * vec * rounds;
    f.parts = std::max<int64_t>(1, ceil_div(V, f.part));
    f.rows = std::max<int64_t>(1, std::min(T, kSplitBytes / std::max<int64_t>(1, V * esize)));
    return f;
}

struct Space {
    int64_t at, end;  // the entries' logits, behind the sums
};
Space space_of(const Form& f, int64_t K) {
    Space s{};
    if (f.kept) return s;
    s.at = round_up(f.rows * f.parts * int64_t(sizeof(PartSum)), 256);
    s.end = s.at + round_up(f.rows * K * 4, 256);
    return s;
}

template <class T, class S, int B>
void launch_kept(const DistillArgs& a, const T* z, const S* teacher, T* grad, hipStream_t st) {
    // as many blocks as the 256 CUs hold at 16 wavefronts each
    const int64_t blocks = std::min<int64_t>(a.T, 256 * 1024 / B);
    hipLaunchKernelGGL((kept_kernel<T, S, B>), dim3(unsigned(blocks)), dim3(B), size_t(16 * a.K),
                       st, a, z, teacher, grad);
}

template <class T, class S>
ar_status run_distill(DistillArgs a, const void* logits, const void* teacher, void* grad,
                      char* workspace, hipStream_t st) {
    const T* const z = static_cast<const T*>(logits);
    const S* const s = static_cast<const S*>(teacher);
    T* const g = static_cast<T*>(grad);
    const Form f = form_of(a.T, a.V, int(sizeof(T)));
    if (f.kept) {
        const int64_t threads = ceil_div(a.V, kKeep * Num<T>::VEC);
        if (threads <= 64) launch_kept<T, S, 64>(a, z, s, g, st);
        else if (threads <= 128) launch_kept<T, S, 128>(a, z, s, g, st);
        else if (threads <= 256) launch_kept<T, S, 256>(a, z, s, g, st);
        else if (threads <= 512) launch_kept<T, S, 512>(a, z, s, g, st);
        else launch_kept<T, S, 1024>(a, z, s, g, st);
        return launch_status("distillation");
    }
    a.part = f.part;
    a.parts = f.parts;
    a.sums = reinterpret_cast<PartSum*>(workspace);
    a.at = reinterpret_cast<float*>(workspace + space_of(f, a.K).at);
    for (a.first = 0; a.first < a.T; a.first += f.rows) {
        const int64_t rows = std::min(f.rows, a.T - a.first);
        hipLaunchKernelGGL((parts_kernel<T, kSplitBlock>), dim3(unsigned(rows * f.parts)),
                           dim3(kSplitBlock), 0, st, a, z);
        hipLaunchKernelGGL((split_kernel<T, S, kSplitBlock>),
                           dim3(unsigned(rows * (g ? f.parts : 1))), dim3(kSplitBlock),
                           size_t(12 * a.K), st, a, z, s, g);
    }
    return launch_status("distillation");
}

}  // namespace
}  // namespace arp

using namespace arp;

AR_EXPORT ar_status ar_distill_workspace(int64_t T, int64_t V, int64_t K, int64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    AR_TRY(check_extent("T", T));
    AR_TRY(check_extent("V", V));
    AR_TRY(check_extent("K", K));
    if (K > AR_DISTILL_MAX_K) return fail(AR_ERR_UNSUPPORTED, "K exceeds AR_DISTILL_MAX_K");
    *bytes = std::max(space_of(form_of(T, V, 4), K).end, space_of(form_of(T, V, 2), K).end);
    return AR_OK;
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_distill(int32_t dtype, int64_t T, int64_t V, int64_t K, const void* logits,
                               int64_t logits_stride, int32_t teacher_dtype, const void* teacher,
                               int64_t teacher_stride, const int64_t* ids, int64_t ids_stride,
                               float temperature, const float* weights, float* loss, void* grad,
                               int64_t grad_stride, void* workspace, int64_t workspace_bytes,
                               void* stream) try {
    clear_error();
    int32_t es = 0, ts = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_dtype("teacher_dtype", teacher_dtype, &ts));
    int64_t need = 0;
    AR_TRY(ar_distill_workspace(T, V, K, &need));
    if (!(temperature > 0.0f) || std::isinf(temperature))
        return fail(AR_ERR_INVALID_ARG, "temperature must be finite and > 0");
    if (temperature < AR_DISTILL_MIN_TEMPERATURE || temperature > AR_DISTILL_MAX_TEMPERATURE)
        return fail(AR_ERR_UNSUPPORTED,
                    "temperature is outside AR_DISTILL_MIN_TEMPERATURE .. AR_DISTILL_MAX_TEMPERATURE");
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
    DistillArgs a{};
    a.ids = ids;
    a.weights = weights;
    a.loss = loss;
    a.T = T;
    a.V = V;
    a.K = K;
    a.logits_stride = logits_stride;
    a.teacher_stride = teacher_stride;
    a.ids_stride = ids_stride;
    a.grad_stride = grad_stride;
    a.c = float(1.4426950408889634 / double(temperature));
    a.temperature = temperature;
    char* const ws = static_cast<char*>(workspace);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (dtype == AR_F32)
        return teacher_dtype == AR_F32 ? run_distill<float, float>(a, logits, teacher, grad, ws, st)
                                       : run_distill<float, uint16_t>(a, logits, teacher, grad, ws, st);
    return teacher_dtype == AR_F32 ? run_distill<uint16_t, float>(a, logits, teacher, grad, ws, st)
                                   : run_distill<uint16_t, uint16_t>(a, logits, teacher, grad, ws, st);
} catch (...) {
    return thrown();
}
