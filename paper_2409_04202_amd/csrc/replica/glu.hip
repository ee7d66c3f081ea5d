// The gated feed-forward block's products.
#include <algorithm>
#include <type_traits>

#include "product.hpp"

namespace arp {
namespace {

// exp(x), to a few units in the last place: 2^(x log2 e) with what the product
// was rounded by put back.
__device__ __forceinline__ float exp_of(float x) {
    const float t = x * 1.44269504f, lost = fmaf(x, 1.44269504f, -t) + x * 1.92596299e-8f;
    const float e = __builtin_amdgcn_exp2f(t);
    return fabsf(t) < 127.0f ? fmaf(e, lost * 0.69314718f, e) : e;
}
// 1 / x for x >= 1, to a unit in the last place.
__device__ __forceinline__ float inverse(float x) {
    const float r = __builtin_amdgcn_rcpf(x);
    return r == 0.0f ? r : fmaf(fmaf(-x, r, 1.0f), r, r);
}

// a(g) and a'(g).  For bf16 the hardware's exponential and reciprocal as they
// are: their errors, some units of fp32 and about |g| more of the exponent's rounding,
// are far below the rounding of h, and of dg and du, which is all that the
// factors are for, those saved in fp32 too.
template <class T>
__device__ __forceinline__ void activate(int act, float g, float* value, float* slope) {
    if (act == AR_ACT_SILU) {
        float s;
        if constexpr (sizeof(T) == 2) s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504f));
        else s = inverse(1.0f + exp_of(-g));
        // at infinities the limits, not inf * 0
        *value = g == -INFINITY ? 0.0f : g * s;
        *slope = s == 0.0f ? 0.0f : s * (1.0f + (s == 1.0f ? 0.0f : g * (1.0f - s)));
    } else {
        const float cdf = 0.5f * erfcf(g * -0.70710678118654752f);
        const float pdf = 0.39894228040143268f * exp_of(-0.5f * g * g);
        *value = g == -INFINITY ? 0.0f : g * cdf;
        *slope = cdf + (pdf == 0.0f ? 0.0f : g * pdf);
    }
}

struct ForwardArgs {
    int64_t h_stride, saved_stride;
    int act;
    // the saved factors, or NULL: in fp32, or in the matrices' type
    void *sg, *su;
    bool saved_f32;
};

// Where the sums of a part of a tile (rows x cols) are.
__device__ __forceinline__ int64_t part_at(const ProductShape& p, int64_t tile, int split, int rows,
                                           int cols) {
    return ((tile - p.whole) * p.splits + split) * (int64_t(rows) * cols);
}

// h, and the saved factors where they are wanted, of a tile; or, split along k,
// the tile's sums of g and of u.  A panel holds rows of both weights, so that a
// lane has g and u of the same element and the activation is its epilogue.
// Bound by the matrix cores and the copies' issue: 2048 x 4096 x 16384 bf16 469
// us, 1172 TFLOP/s, in calls that follow each other (504 the median of a trace, whose
// launches stand apart); in traces 8192 rows with the factors saved 2.02 ms; 777 x
// 1003 x 2731 fp32 101 us, 85 TFLOP/s, and its join 6.
template <class T, int BR, int BC, int WR, int WC, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WC) void forward_kernel(ProductShape p, ForwardArgs a,
                                                               Side<T> x, Side<T> w, T* h) {
    using P = Tile<T, BR, BC, WR, WC, true, true, true, DIRECT>;
    using S = Store<1>;
    constexpr int LDS = P::LDS > WR * WC * S::BYTES ? P::LDS : WR * WC * S::BYTES;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    Unit unit;
    int64_t rt, ct;
    if (!unit_of(p, blockIdx.x, &unit)) return;
    place_of(p, unit.tile, &rt, &ct);
    f32x16 acc[P::SR][2] = {};
    P::run(p, x, w, rt * BR, ct * (BC / 2), unit, (AR_LDS char*)lds, acc);
    const int wave = int(threadIdx.x) >> 6, wr = wave / WC, wc = wave % WC;
    AR_LDS float* const part = (AR_LDS float*)((AR_LDS char*)lds + wave * S::BYTES);
#pragma unroll
    for (int i = 0; i < P::SR; ++i) {
        const int64_t tr = (wr * P::SR + i) * 32, tc = wc * 32;  // within the tile
        const int64_t r0 = rt * BR + tr, c0 = ct * (BC / 2) + tc;
        auto pass = [&](auto* out, int64_t stride, auto f) {
            S::fill(part, f);
            wave_sync();
            S::store(part, out, stride, r0, p.rows, c0, p.cols, false, 0, 0);
            wave_sync();
        };
        if (unit.splits > 1) {  // g on the left, u on the right
            float* const to = p.part + part_at(p, unit.tile, unit.split, BR, BC);
            auto sums = [&](int j) {
                S::fill(part, [&](int, int e) { return acc[i][j][e]; });
                wave_sync();
                S::store(part, to, BC, tr, BR, tc + j * (BC / 2), BC, false, 0, 0);
                wave_sync();
            };
            sums(0);
            sums(1);
            continue;
        }
        float value[16], slope[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) activate<T>(a.act, acc[i][0][e], &value[e], &slope[e]);
        pass(h, a.h_stride, [&](int, int e) { return value[e] * acc[i][1][e]; });
        auto save = [&](auto* sg, auto* su) {
            pass(sg, a.saved_stride, [&](int, int e) { return slope[e] * acc[i][1][e]; });
            pass(su, a.saved_stride, [&](int, int e) { return value[e]; });
        };
        if (a.sg && a.saved_f32) save(static_cast<float*>(a.sg), static_cast<float*>(a.su));
        else if (a.sg) save(static_cast<T*>(a.sg), static_cast<T*>(a.su));
    }
}

// Up to kFewRows rows of x: the weights pass once, so a wavefront takes whole
// rows of them, two of each, its lanes side by side along D, and one
// accumulator a (weight row, row of x).  Bound by memory: the weights' bytes.
// 2 x 16384 x 4096 bf16: 45 us for one row, 5.9 TB/s.  For 8 rows 69 us, on
// the tiles below 78; fp32, 2 x 8192 x 4096: 60 and 147.  From 9 rows on the
// registers for a sum each would leave too few loads in flight; on the tiles 16 rows
// take 76.
constexpr int kFewRows = 8;

template <class T, int ROWS>
__global__ __launch_bounds__(256) void few_rows_kernel(int64_t M, int64_t D, int64_t F,
                                                       ForwardArgs a, Side<T> x, Side<T> w, T* h) {
    constexpr int VEC = Num<T>::VEC, WIDE = ROWS <= 2 ? 4 : ROWS <= 4 ? 2 : 1;
    const int lane = threadIdx.x & 63;
    const int64_t f = (int64_t(blockIdx.x) * 4 + scalar(threadIdx.x >> 6)) * 2;
    if (f >= F) return;
    const int64_t next = f + 1 < F ? w.stride : 0;  // (an odd last row: twice)
    const T* const wr[4] = {w.p[0] + f * w.stride, w.p[0] + f * w.stride + next,
                            w.p[1] + f * w.stride, w.p[1] + f * w.stride + next};
    const T* xr[ROWS];
#pragma unroll
    for (int m = 0; m < ROWS; ++m) xr[m] = x.p[0] + (m < M ? m : M - 1) * x.stride;
    float sum[4][ROWS] = {};
    const int64_t whole = D / VEC * VEC;
    auto multiply_add = [&](const u32x4* wv, const u32x4* xv) {
        float a[4][VEC];
#pragma unroll
        for (int i = 0; i < 4; ++i) Num<T>::unpack(wv[i], a[i]);
#pragma unroll
        for (int m = 0; m < ROWS; ++m) {
            float b[VEC];
            Num<T>::unpack(xv[m], b);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum[i][m] = fmaf(a[i][e], b[e], sum[i][m]);
        }
    };
    auto add = [&](int64_t d, auto load) {
        u32x4 wv[4], xv[ROWS];
#pragma unroll
        for (int i = 0; i < 4; ++i) wv[i] = load(wr[i] + d);
#pragma unroll
        for (int m = 0; m < ROWS; ++m) xv[m] = load(xr[m] + d);
        multiply_add(wv, xv);
    };
    const auto vec = [](const T* p) { return load_vec(p); };
    int64_t d = int64_t(lane) * VEC;
    for (; d + (WIDE - 1) * 64 * VEC < whole; d += WIDE * 64 * VEC) {
        u32x4 wv[WIDE][4], xv[WIDE][ROWS];
#pragma unroll
        for (int k = 0; k < WIDE; ++k) {
#pragma unroll
            for (int i = 0; i < 4; ++i) wv[k][i] = load_vec(wr[i] + d + k * 64 * VEC);
#pragma unroll
            for (int m = 0; m < ROWS; ++m) xv[k][m] = load_vec(xr[m] + d + k * 64 * VEC);
        }
        __builtin_amdgcn_sched_barrier(0);  // all of them in flight
#pragma unroll
        for (int k = 0; k < WIDE; ++k) multiply_add(wv[k], xv[k]);
    }
    for (; d < whole; d += 64 * VEC) add(d, vec);
    const int rest = int(D - whole);
    if (rest && lane == 63) add(whole, [&](const T* p) { return load_part(p, rest); });
    // (feature f, row m) to lane 2 m + (0 or 1)
    float g = 0.0f, u = 0.0f;
#pragma unroll
    for (int m = 0; m < ROWS; ++m)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float sg = wave_sum(sum[i][m]), su = wave_sum(sum[2 + i][m]);
            if (lane == 2 * m + i) {
                g = sg;
                u = su;
            }
        }
    const int64_t m = lane >> 1, c = f + (lane & 1);
    if (m >= M || m >= ROWS || c >= F) return;
    float value, slope;
    activate<T>(a.act, g, &value, &slope);
    h[m * a.h_stride + c] = Num<T>::down(value * u);
    const int64_t at = m * a.saved_stride + c;
    if (a.sg && a.saved_f32) {
        static_cast<float*>(a.sg)[at] = slope * u;
        static_cast<float*>(a.su)[at] = value;
    } else if (a.sg) {
        static_cast<T*>(a.sg)[at] = Num<T>::down(slope * u);
        static_cast<T*>(a.su)[at] = Num<T>::down(value);
    }
}

// Four values to adjacent elements, of which n are there.
template <class T>
__device__ __forceinline__ void store_four(T* p, const float* v, int64_t n) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2), aligned(2)));
    if (n < 4) {
        for (int e = 0; e < int(n); ++e) p[e] = Num<T>::down(v[e]);
    } else if constexpr (sizeof(T) == 4) {
        store_vec(p, Num<T>::pack(v));
    } else {
        *(AR_GLOBAL u32x2*)p = u32x2{bf16_pack(v[0], v[1]), bf16_pack(v[2], v[3])};
    }
}

// The sums of the tiles that are split along k, added in order, to the output:
// `rows` of a tile and `cols` of the output in it are powers of two.
template <class T>
__global__ __launch_bounds__(256) void forward_join_kernel(ProductShape p, ForwardArgs a, T* h,
                                                           int rows, int cols) {
    const int64_t rest = (p.tiles - p.whole) * rows * (cols / 4), step = int64_t(gridDim.x) * 256;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < rest; i += step) {
        const int n = int(i & (rows * (cols / 4) - 1)), tr = n / (cols / 4), tc = n % (cols / 4) * 4;
        const int64_t tile = p.whole + i / (rows * (cols / 4));
        int64_t rt, ct;
        place_of(p, tile, &rt, &ct);
        const int64_t r = rt * rows + tr, c = ct * cols + tc;
        if (r >= p.rows || c >= p.cols) continue;
        float g[4] = {}, u[4] = {};
        for (int s = 0; s < p.splits; ++s) {
            const float* const from = p.part + part_at(p, tile, s, rows, 2 * cols) + tr * (2 * cols) + tc;
            float x[4], y[4];
            Num<float>::unpack(load_vec(from), x);
            Num<float>::unpack(load_vec(from + cols), y);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                g[e] += x[e];
                u[e] += y[e];
            }
        }
        float value[4], slope[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            activate<T>(a.act, g[e], &value[e], &slope[e]);
            slope[e] *= u[e];
            g[e] = value[e] * u[e];
        }
        const int64_t left = p.cols - c, at = r * a.saved_stride + c;
        store_four(h + r * a.h_stride + c, g, left);
        if (a.sg && a.saved_f32) {
            store_four(static_cast<float*>(a.sg) + at, slope, left);
            store_four(static_cast<float*>(a.su) + at, value, left);
        } else if (a.sg) {
            store_four(static_cast<T*>(a.sg) + at, slope, left);
            store_four(static_cast<T*>(a.su) + at, value, left);
        }
    }
}

// dg = dh * saved_gate and du = dh * saved_up (of type S), a vector of T a
// lane.  Bound by memory: five matrices pass once (8192 x 16384 bf16 with fp32
// factors: 0.37 ms, 5.1 TB/s).  A pass of its own because both gradients read dg and
// du, each element of them in several tiles.  For bf16 the rounding is that of the
// matrix instruction's operands: it takes the gradients' error from 0.0017 of their
// norm, the last rounding's, to 0.0023.
template <class T, class S>
__global__ __launch_bounds__(256) void factors_kernel(int64_t M, int64_t F, const T* dh,
                                                      int64_t dh_stride, const S* sg, const S* su,
                                                      int64_t saved_stride, T* dg, T* du,
                                                      int64_t stride) {
    constexpr int VEC = Num<T>::VEC, SV = Num<S>::VEC;
    const int64_t per = (F + VEC - 1) / VEC, step = int64_t(gridDim.x) * 256;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < M * per; i += step) {
        const int64_t r = i / per, c = i % per * VEC;
        const int n = int(F - c < VEC ? F - c : VEC);
        const T* pd = dh + r * dh_stride + c;
        const S *pg = sg + r * saved_stride + c, *pu = su + r * saved_stride + c;
        float d[VEC], g[VEC], u[VEC];
        if (n == VEC) {
            Num<T>::unpack(load_vec(pd), d);
#pragma unroll
            for (int e = 0; e < VEC; e += SV) {
                Num<S>::unpack(load_vec(pg + e), g + e);
                Num<S>::unpack(load_vec(pu + e), u + e);
            }
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                d[e] = e < n ? Num<T>::up(pd[e]) : 0.0f;
                g[e] = e < n ? Num<S>::up(pg[e]) : 0.0f;
                u[e] = e < n ? Num<S>::up(pu[e]) : 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            g[e] *= d[e];
            u[e] *= d[e];
        }
        // (their rows are whole vectors: the last one's rest is zero)
        store_vec(dg + r * stride + c, Num<T>::pack(g));
        store_vec(du + r * stride + c, Num<T>::pack(u));
    }
}

// One or two products C = R L^T of one shape (the two weight gradients have
// row operands of their own, and share a launch), or C += with accumulate.
// 8192 x 4096 x 16384 bf16, medians of a trace: dx 1.71 ms, 1.29 PFLOP/s, both
// weight gradients 1.70.  777 x 1003 x 2731 fp32: 102 us, its join 5, and 89.
template <class T>
struct Products {
    Side<T> r[2], l;
    T* out[2];
    int64_t stride;
    int count, accumulate;
};

template <class T, int BR, int BC, int WR, int WC, bool RKC, bool DIRECT>
__global__ __launch_bounds__(64 * WR * WC) void product_kernel(ProductShape p, Products<T> a) {
    using P = Tile<T, BR, BC, WR, WC, RKC, false, false, DIRECT>;
    using S = Store<P::SC>;
    constexpr int LDS = P::LDS > WR * WC * S::BYTES ? P::LDS : WR * WC * S::BYTES;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    constexpr int VEC = Num<T>::VEC;
    const int64_t tiles = p.row_tiles * p.col_tiles;
    Unit unit;
    int64_t rt, ct;
    if (!unit_of(p, blockIdx.x, &unit)) return;
    const bool second = unit.tile >= tiles;
    place_of(p, second ? unit.tile - tiles : unit.tile, &rt, &ct);
    f32x16 acc[P::SR][P::SC] = {};
    P::run(p, second ? a.r[1] : a.r[0], a.l, rt * BR, ct * BC, unit, (AR_LDS char*)lds, acc);
    const int wave = int(threadIdx.x) >> 6, wr = wave / WC, wc = wave % WC;
    AR_LDS float* const part = (AR_LDS float*)((AR_LDS char*)lds + wave * S::BYTES);
    const int shift = DIRECT ? int((VEC - a.l.extent % VEC) % VEC) : 0;
#pragma unroll
    for (int i = 0; i < P::SR; ++i) {
        S::fill(part, [&](int j, int e) { return acc[i][j][e]; });
        wave_sync();
        const int64_t tr = (wr * P::SR + i) * 32, tc = wc * P::SC * 32;  // within the tile
        const int64_t r0 = rt * BR + tr, c0 = ct * BC + tc;
        if (unit.splits > 1)
            S::store(part, p.part + part_at(p, unit.tile, unit.split, BR, BC), BC, tr,
                     p.rows - rt * BR < BR ? p.rows - rt * BR : BR, tc,
                     p.cols - ct * BC < BC ? p.cols - ct * BC : BC, false, VEC,
                     ct + 1 == p.col_tiles ? shift : 0);
        else
            S::store(part, second ? a.out[1] : a.out[0], a.stride, r0, p.rows, c0, p.cols,
                     a.accumulate, VEC, shift);
        wave_sync();
    }
}

template <class T>
__global__ __launch_bounds__(256) void product_join_kernel(ProductShape p, Products<T> a, int rows,
                                                           int cols) {
    const int64_t rest = (p.tiles - p.whole) * rows * (cols / 4), step = int64_t(gridDim.x) * 256;
    const int64_t tiles = p.row_tiles * p.col_tiles;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < rest; i += step) {
        const int n = int(i & (rows * (cols / 4) - 1)), tr = n / (cols / 4), tc = n % (cols / 4) * 4;
        const int64_t tile = p.whole + i / (rows * (cols / 4));
        const bool second = tile >= tiles;
        int64_t rt, ct;
        place_of(p, second ? tile - tiles : tile, &rt, &ct);
        const int64_t r = rt * rows + tr, c = ct * cols + tc;
        if (r >= p.rows || c >= p.cols) continue;
        float v[4] = {};
        for (int s = 0; s < p.splits; ++s) {
            float x[4];
            Num<float>::unpack(load_vec(p.part + part_at(p, tile, s, rows, cols) + tr * cols + tc), x);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += x[e];
        }
        T* const at = (second ? a.out[1] : a.out[0]) + r * a.stride + c;
        if (a.accumulate) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < p.cols) v[e] += Num<T>::up(at[e]);
        }
        store_four(at, v, p.cols - c);
    }
}

// Whether a tile's copies may go straight to LDS: 16-byte chunks at 16-byte
// places (fp32: at any element), within 32-bit offsets of the tile's first row,
// and, K-major, at least one chunk a row (fp32) or whole ones (bf16).
template <class T>
bool direct(const Side<T>& s, bool kc) {
    constexpr int VEC = Num<T>::VEC;
    if (s.stride * int64_t(sizeof(T)) > (int64_t(1) << 22)) return false;
    if (sizeof(T) == 2 &&
        (s.stride % VEC ||
         (reinterpret_cast<uintptr_t>(s.p[0]) | reinterpret_cast<uintptr_t>(s.p[1])) % kChunk))
        return false;
    return kc || (sizeof(T) == 4 ? s.extent >= VEC : s.extent % VEC == 0);
}

int64_t factor_stride(int64_t F) { return round_up(F, 8); }

// How a product is cut: square tiles of 256, 128 or 64, and parts along k, of all
// tiles or of those that are left after whole rounds of the 256 CUs.
// The time is estimated as the most that one of the CUs gets, at a rate a CU
// that grows with the tile (a larger tile reads less from LDS for its
// products), and, where k is split, the parts' way through memory and a launch.
// The rates are those of long products that were given each tile in turn.  1531 x
// 2051 x 5465 bf16: the forward's 258 tiles as 256 whole ones and two split by 8
// 124 us, as 1032 smaller ones 163; 777 x 1003 x 2731 fp32: 256 of 301 whole and the
// others split by 5 109 us, all split by 2 122.
struct Cut {
    int tile, splits;
    int64_t whole;  // tiles that are not split
};

constexpr double kCuFlops[2][4] = {
    // 64, 128, 256, and 64 of the gated product (two wavefronts a block), in
    // 1e12 a second
    {0.45, 0.54, 0.54, 0.34},  // fp32
    {1.7, 3.4, 4.6, 1.4},      // bf16
};

// A CU holds two and more blocks of the smaller tiles, and one of them alone,
// with no part beside it any more, does not reach the rate.
constexpr double kAlone = 1.2;

Cut cut_of(int64_t rows, int64_t cols, int64_t K, int outputs, int esize, bool gated) {
    Cut best{64, 1, 0};
    double least = 0;
    for (int i = 0; i < 3; ++i) {
        const int tile = 64 << i;
        const int64_t tiles = ceil_div(rows, tile) * ceil_div(cols, gated ? tile / 2 : tile) * outputs;
        const double one = 2.0 * tile * tile * double(K) /
                           (kCuFlops[esize == 2][gated && i == 0 ? 3 : i] * 1e12);
        auto consider = [&](int64_t whole, int s) {
            const int64_t rest = tiles - whole;
            double t = double(ceil_div(whole, 256)) * (one + 1.5e-6);
            if (rest)
                t += double(ceil_div(rest * s, 256)) * (one / s + 1.5e-6) + 4e-6 +
                     8.0 * s * double(rest) * tile * tile / 4e12;
            if (rest && whole && tile < 256) t *= kAlone;
            if (least == 0 || t < least) {
                least = t;
                best = Cut{tile, s, whole};
            }
        };
        consider(tiles, 1);
        for (int s = 2; s <= 16; ++s) {
            if (K / s < 4 * (kStepBytes / esize)) break;
            if ((s & (s - 1)) == 0) consider(0, s);
            if (tiles > 256 && tiles % 256) consider(tiles / 256 * 256, s);
        }
    }
    return best;
}

// The workspace of a cut's parts.
int64_t part_bytes(const Cut& c, int64_t rows, int64_t cols, int outputs, bool gated) {
    const int64_t tiles = ceil_div(rows, c.tile) * ceil_div(cols, gated ? c.tile / 2 : c.tile) * outputs;
    return c.splits > 1 ? 4 * c.splits * (tiles - c.whole) * c.tile * c.tile : 0;
}

ProductShape shape(int64_t rows, int64_t cols, int64_t K, int segments, const Cut& c, int width,
                   int outputs, void* part) {
    const int64_t rt = ceil_div(rows, c.tile), ct = ceil_div(cols, width);
    return ProductShape{rows, cols, K, segments, rt, ct, rt * ct * outputs,
                        c.splits > 1 ? c.whole : rt * ct * outputs, c.splits,
                        static_cast<float*>(part)};
}

dim3 grid_of(const ProductShape& p) { return dim3(unsigned(unit_blocks(p))); }
dim3 join_grid(int64_t vecs) {
    return dim3(unsigned(std::min<int64_t>(ceil_div(vecs, 256), 1 << 14)));
}

template <class T, bool RKC, int B, int WR, int WC>
void launch_product(const ProductShape& p, const Products<T>& a, bool fast, hipStream_t st) {
    const dim3 grid = grid_of(p), block(64 * WR * WC);
    if (fast)
        hipLaunchKernelGGL((product_kernel<T, B, B, WR, WC, RKC, true>), grid, block, 0, st, p, a);
    else
        hipLaunchKernelGGL((product_kernel<T, B, B, WR, WC, RKC, false>), grid, block, 0, st, p, a);
}

template <class T, bool RKC>
void run_product(int64_t rows, int64_t cols, int64_t K, int segments, const Products<T>& a,
                 void* part, hipStream_t st) {
    const Cut c = cut_of(rows, cols, K * segments, a.count, int(sizeof(T)), false);
    const ProductShape p = shape(rows, cols, K, segments, c, c.tile, a.count, part);
    bool fast = direct(a.l, false);
    for (int i = 0; i < a.count; ++i) fast = fast && direct(a.r[i], RKC);
    if (c.tile == 256) launch_product<T, RKC, 256, 2, 4>(p, a, fast, st);
    else if (c.tile == 128) launch_product<T, RKC, 128, 2, 2>(p, a, fast, st);
    else launch_product<T, RKC, 64, 2, 2>(p, a, fast, st);
    if (c.splits > 1)
        hipLaunchKernelGGL((product_join_kernel<T>), join_grid((p.tiles - p.whole) * c.tile * c.tile / 4),
                           dim3(256), 0, st, p, a, c.tile, c.tile);
}

template <class T, int B, int WR, int WC>
void launch_forward(const ProductShape& p, const ForwardArgs& a, const Side<T>& x, const Side<T>& w,
                    T* h, bool fast, hipStream_t st) {
    const dim3 grid = grid_of(p), block(64 * WR * WC);
    if (fast)
        hipLaunchKernelGGL((forward_kernel<T, B, B, WR, WC, true>), grid, block, 0, st, p, a, x, w, h);
    else
        hipLaunchKernelGGL((forward_kernel<T, B, B, WR, WC, false>), grid, block, 0, st, p, a, x, w, h);
}

template <class T>
void run_forward(const ForwardArgs& a, int64_t M, int64_t D, int64_t F, const Side<T>& x,
                 const Side<T>& w, T* h, void* part, hipStream_t st) {
    if (M <= kFewRows) {
        const dim3 grid(unsigned(ceil_div(F, 8))), block(256);
        auto go = [&](auto rows) {
            hipLaunchKernelGGL((few_rows_kernel<T, decltype(rows)::value>), grid, block, 0, st, M, D,
                               F, a, x, w, h);
        };
        if (M <= 1) go(std::integral_constant<int, 1>{});
        else if (M <= 2) go(std::integral_constant<int, 2>{});
        else if (M <= 4) go(std::integral_constant<int, 4>{});
        else go(std::integral_constant<int, 8>{});
        return;
    }
    const Cut c = cut_of(M, F, D, 1, int(sizeof(T)), true);
    const ProductShape p = shape(M, F, D, 1, c, c.tile / 2, 1, part);
    const bool fast = direct(x, true) && direct(w, true);
    if (c.tile == 256) launch_forward<T, 256, 2, 4>(p, a, x, w, h, fast, st);
    else if (c.tile == 128) launch_forward<T, 128, 2, 2>(p, a, x, w, h, fast, st);
    else launch_forward<T, 64, 2, 1>(p, a, x, w, h, fast, st);
    if (c.splits > 1)
        hipLaunchKernelGGL((forward_join_kernel<T>), join_grid((p.tiles - p.whole) * c.tile * c.tile / 8),
                           dim3(256), 0, st, p, a, h, c.tile, c.tile / 2);
}

// bf16 rows that do not lie at 16 bytes, by their width, stride or address, cannot
// be copied straight to LDS: x and the weights are laid out once more, in rows of
// whole vectors, where enough rows of x read the weights to pay for it.
template <class T>
__global__ __launch_bounds__(256) void pack_kernel(int64_t rows, int64_t cols, const T* from,
                                                   int64_t stride, T* to, int64_t pitch) {
    constexpr int VEC = Num<T>::VEC;
    const int64_t per = pitch / VEC, step = int64_t(gridDim.x) * 256;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < rows * per; i += step) {
        const int64_t r = i / per, c = i % per * VEC, left = cols - c;
        const T* const p = from + r * stride + c;
        store_vec(to + r * pitch + c, left >= VEC ? load_vec(p) : load_part(p, int(left)));
    }
}

// The forward's panels lie along their rows, the backward's across them, where
// rows that all start at another place within 16 bytes are the slowest.  M x D x F,
// us as they lie and laid out anew.  Forward, 2048 x 1003 x 4096 71 and 77, 2048 x
// 2048 x 5464 161 and 139, 512 x 4099 x 16384 195 and 276, 4096 x 4099 x 16384 1334 and
// 1241, 4096 x 4096 x 16384 1541 and 1042.  Backward, 128 x 4099 x 16384 316 and
// 365, 256 x 4099 x 16384 454 and 416, 1536 x 2051 x 5465 717 and 302; of whole vectors 512
// x 4096 x 16384 436 and 470, 768 x 1024 x 4096 107 and 98, 4096 x 2048 x 5464 551 and
// 475.
bool packs(int64_t M, int64_t D, int64_t F, int esize, bool backward) {
    const int64_t rows = !backward ? 2048 : D % 8 ? 256 : 768;
    return esize == 2 && M >= rows && double(M) * double(D) * double(F) > 5e8;
}
int64_t pack_bytes(int64_t M, int64_t D, int64_t F, int esize, bool backward) {
    return packs(M, D, F, esize, backward) ? round_up((M + 2 * F) * round_up(D, 8) * esize, 256) : 0;
}
// Replaces x and w by their copies in `space`.
template <class T>
void pack(int64_t M, int64_t D, int64_t F, Side<T>* x, Side<T>* w, void* space, hipStream_t st) {
    const int64_t pitch = round_up(D, 8);
    T* to = static_cast<T*>(space);
    auto one = [&](const T* from, int64_t rows, int64_t stride) {
        hipLaunchKernelGGL((pack_kernel<T>), join_grid(rows * pitch / Num<T>::VEC), dim3(256), 0, st, rows,
                           D, from, stride, to, pitch);
        T* const at = to;
        to += rows * pitch;
        return at;
    };
    if (x && x->p[0]) {
        const T* const px = one(x->p[0], M, x->stride);
        *x = Side<T>{{px, px}, pitch, pitch};
    }
    if (w && w->p[0]) {
        const T* const pg = one(w->p[0], F, w->stride);
        const T* const pu = one(w->p[1], F, w->stride);
        *w = Side<T>{{pg, pu}, pitch, pitch};
    }
}

// The backward call's workspace: the factors, the parts of dx, those of dwg and
// dwu, and x and the weights laid out anew.
struct BackSpace {
    int64_t dx, dw, packed, end;
};
BackSpace back_space(int64_t M, int64_t D, int64_t F, int esize) {
    BackSpace b{};
    b.dx = round_up(2 * M * factor_stride(F) * esize, 256);
    b.dw = b.dx + part_bytes(cut_of(M, D, 2 * F, 1, esize, false), M, D, 1, false);
    b.packed = b.dw + part_bytes(cut_of(F, D, M, 2, esize, false), F, D, 2, false);
    b.end = b.packed + pack_bytes(M, D, F, esize, true);
    return b;
}

}  // namespace
}  // namespace arp

using namespace arp;

static ar_status check_saved_dtype(int32_t dtype, int32_t saved, int32_t* esize) {
    AR_TRY(check_dtype("saved_dtype", saved, esize));
    if (saved != dtype && saved != AR_F32)
        return fail(AR_ERR_UNSUPPORTED, "saved_dtype is dtype or AR_F32");
    return AR_OK;
}

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
                                     int32_t backward, int64_t* bytes) try {
    clear_error();
    if (!bytes) return fail(AR_ERR_INVALID_ARG, "bytes is NULL");
    int32_t es = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_glu_sizes(M, D, F));
    *bytes = M <= kFewRows || D == 0 || F == 0
                 ? 0
                 : part_bytes(cut_of(M, F, D, 1, es, true), M, F, 1, true) +
                       pack_bytes(M, D, F, es, false);
    if (backward) *bytes = std::max(*bytes, back_space(M, D, F, es).end);
    return AR_OK;
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_glu_forward(int32_t dtype, int32_t act, int64_t M, int64_t D, int64_t F,
                                   const void* x, int64_t x_stride, const void* wg, const void* wu,
                                   int64_t w_stride, void* h, int64_t h_stride, void* saved_gate,
                                   void* saved_up, int64_t saved_stride, int32_t saved_dtype,
                                   void* workspace, int64_t workspace_bytes, void* stream) try {
    clear_error();
    int32_t es = 0, ss = 0;
    int64_t need = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    if (act != AR_ACT_SILU && act != AR_ACT_GELU)
        return fail(AR_ERR_INVALID_ARG, "unknown activation");
    AR_TRY(check_saved_dtype(dtype, saved_dtype, &ss));
    AR_TRY(ar_glu_workspace(dtype, M, D, F, 0, &need));
    if (!saved_gate != !saved_up)
        return fail(AR_ERR_INVALID_ARG, "saved_gate and saved_up are given together");
    const int64_t sr = saved_gate ? M : 0;
    const MatArg mx{"x", x, M, D, x_stride, es}, mg{"wg", wg, F, D, w_stride, es},
        mu{"wu", wu, F, D, w_stride, es}, mh{"h", h, M, F, h_stride, es},
        sg{"saved_gate", saved_gate, sr, F, saved_stride, ss},
        su{"saved_up", saved_up, sr, F, saved_stride, ss},
        mw{"the workspace", workspace, 1, need, need, 1};
    for (const MatArg& m : {mx, mg, mu, mh, sg, su}) AR_TRY(check_matrix(m));
    AR_TRY(check_workspace(workspace, workspace_bytes, need));
    for (const MatArg& o : {mh, sg, su, mw})
        for (const MatArg& i : {mx, mg, mu}) AR_TRY(check_apart(o, i));
    for (const MatArg& o : {sg, su, mw}) AR_TRY(check_apart(o, mh));
    for (const MatArg& o : {su, mw}) AR_TRY(check_apart(o, sg));
    AR_TRY(check_apart(mw, su));
    if (M == 0 || F == 0) return AR_OK;
    const ForwardArgs a{h_stride, saved_stride, act, saved_gate, saved_up, saved_dtype == AR_F32};
    const hipStream_t st = static_cast<hipStream_t>(stream);
    auto go = [&](auto zero) {
        using T = decltype(zero);
        Side<T> sx{{static_cast<const T*>(x), static_cast<const T*>(x)}, x_stride, D},
            sw{{static_cast<const T*>(wg), static_cast<const T*>(wu)}, w_stride, D};
        if (packs(M, D, F, es, false))
            pack<T>(M, D, F, direct(sx, true) ? nullptr : &sx, direct(sw, true) ? nullptr : &sw,
                    static_cast<char*>(workspace) + part_bytes(cut_of(M, F, D, 1, es, true), M, F, 1, true), st);
        run_forward<T>(a, M, D, F, sx, sw, static_cast<T*>(h), workspace, st);
        return launch_status("gated feed-forward");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}

AR_EXPORT ar_status ar_glu_backward(int32_t dtype, int64_t M, int64_t D, int64_t F, const void* dh,
                                    int64_t dh_stride, const void* x, int64_t x_stride,
                                    const void* wg, const void* wu, int64_t w_stride,
                                    const void* saved_gate, const void* saved_up,
                                    int64_t saved_stride, int32_t saved_dtype,
                                    int32_t accumulate, void* dx,
                                    int64_t dx_stride, void* dwg, void* dwu, int64_t dw_stride,
                                    void* workspace, int64_t workspace_bytes, void* stream) try {
    clear_error();
    int32_t es = 0, ss = 0;
    int64_t need = 0;
    AR_TRY(check_dtype("dtype", dtype, &es));
    AR_TRY(check_saved_dtype(dtype, saved_dtype, &ss));
    AR_TRY(ar_glu_workspace(dtype, M, D, F, 1, &need));
    if (!dwg != !dwu && F > 0 && D > 0)
        return fail(AR_ERR_INVALID_ARG, "dwg and dwu are given together");
    const MatArg mh{"dh", dh, M, F, dh_stride, es}, mx{"x", x, dwg ? M : 0, D, x_stride, es},
        mg{"wg", wg, dx ? F : 0, D, w_stride, es}, mu{"wu", wu, dx ? F : 0, D, w_stride, es},
        sg{"saved_gate", saved_gate, M, F, saved_stride, ss},
        su{"saved_up", saved_up, M, F, saved_stride, ss},
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
        auto factors = [&](auto saved) {
            using S = decltype(saved);
            const int64_t blocks = ceil_div(M * ceil_div(F, Num<T>::VEC), 256);
            hipLaunchKernelGGL((factors_kernel<T, S>),
                               dim3(unsigned(std::min<int64_t>(blocks, 1 << 16))), dim3(256), 0, st,
                               M, F, static_cast<const T*>(dh), dh_stride,
                               static_cast<const S*>(saved_gate), static_cast<const S*>(saved_up),
                               saved_stride, dg, du, fs);
        };
        if (M > 0 && F > 0) {
            if (saved_dtype == AR_F32) factors(float(0));
            else factors(T(0));
        }
        const BackSpace space = back_space(M, D, F, es);
        char* const ws = static_cast<char*>(workspace);
        Side<T> sx{{static_cast<const T*>(x), static_cast<const T*>(x)}, x_stride, D},
            sw{{static_cast<const T*>(wg), static_cast<const T*>(wu)}, w_stride, D};
        if (packs(M, D, F, es, true))
            pack<T>(M, D, F, dwg && !direct(sx, false) ? &sx : nullptr,
                    dx && !direct(sw, false) ? &sw : nullptr, ws + space.packed, st);
        const Side<T> sg{{dg, du}, fs, fs};
        if (dx && M > 0)
            run_product<T, true>(M, D, F, 2,
                                 Products<T>{{sg, sg}, sw, {static_cast<T*>(dx), nullptr}, dx_stride, 1, 0},
                                 ws + space.dx, st);
        if (dwg && F > 0)
            run_product<T, false>(F, D, M, 1,
                                  Products<T>{{Side<T>{{dg, dg}, fs, fs}, Side<T>{{du, du}, fs, fs}},
                                              sx, {static_cast<T*>(dwg), static_cast<T*>(dwu)},
                                              dw_stride, 2, accumulate},
                                  ws + space.dw, st);
        return launch_status("gated feed-forward gradients");
    };
    return dtype == AR_F32 ? go(float(0)) : go(uint16_t(0));
} catch (...) {
    return thrown();
}
