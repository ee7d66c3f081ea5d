// Tiled matrix products on the matrix cores, for the gated feed-forward block:
// C (rows x cols) = sum over k of R(row, k) L(col, k), R the row operand and L
// the column operand, each stored with k along its rows ("K-contiguous") or
// across them ("K-major"), both in fp32 or bf16 with fp32 accumulation.
//
// A block computes a tile of C; its wavefronts split it into 32 x 32 squares
// of accumulators.  Per step of 128 bytes of k (64 bf16 or 32 fp32) the
// operands' panels are copied into LDS, two buffers in turn: the copies of
// the next step run while this one's products do, and the fragments of the next
// quarter of a step are read while this quarter's products run.  The column
// operand is the matrix instruction's first, so a lane holds, of one row of C,
// runs of four adjacent columns.
//
// LDS layouts.  K-contiguous: a row of the panel is 8 chunks of 16 bytes,
// chunk c of row r at place c ^ swz(r), so that any 8 and any 16 successive
// rows' chunks of one k lie in different banks.  K-major bf16: a row is one k,
// read with the transposing LDS load (16 lanes read 4 k of 16 columns and each
// receives 4 k of its column); chunk c of row k at c ^ swzk(k), which puts the
// 32-byte pieces of 4 successive k, and of two neighbouring squares, into
// different banks.  K-major fp32: a row is one k, unswizzled; a lane reads
// single elements, 32 lanes 128 adjacent bytes.
//
// Edges.  Rows beyond an operand's end repeat its last row (their results are
// not stored); a step's k beyond the end reads as zero in both operands, so
// what lies there, NaN included, has no effect.  Where copies go straight to
// LDS, the last chunk of a K-major row that has fewer elements is moved back to
// end with the row: what it holds lies `shift` further on, in the accumulators
// too, and the store reads it from there.  (Column operands only: the rows of a
// K-major row operand, the factors in the workspace, are whole chunks.)
//
// Tiles that do not fill the card.  The last tiles, or all of them, may be split
// along k (`splits`), each part's sums going to memory in fp32; a second kernel
// adds them in order.
#pragma once

#include "replica.hpp"

namespace arp {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kChunk = 16;       // bytes a copy moves a lane
constexpr int kStepBytes = 128;  // bytes of k a step

template <class T> struct StepOf { static constexpr int K = kStepBytes / int(sizeof(T)); };

// An operand: up to two matrices one after the other in k (the second may be
// absent), or, in a panel of the gated product, side by side (half the panel's
// rows from each).
template <class T>
struct Side {
    const T* p[2];
    int64_t stride;
    int64_t extent;  // K-major: the rows' elements in memory, at least the product's
};

struct ProductShape {
    int64_t rows, cols;  // of C (cols: of each half in the gated product)
    int64_t K;           // of one segment
    int segments;        // 1 or 2
    int64_t row_tiles, col_tiles;
    int64_t tiles, whole;  // of all outputs; the first `whole` of them are not split
    int splits;            // parts along k of the others
    float* part;           // their sums, [tile][split][rows of a tile][its columns]
};

// A block's work: a tile, or part `split` of its `splits`.
struct Unit {
    int64_t tile;
    int split, splits;
};

__device__ __forceinline__ int swz(int r) { return ((r >> 1) ^ ((r & 1) << 2)) & 7; }
// (of a K-major row of `chunks` chunks)
__device__ __forceinline__ int swzk(int k, int chunks) {
    return 2 * ((k & 3) ^ ((k & 3) << 1)) & (chunks - 1);
}

// One operand's panel: N rows (K-contiguous) or columns (K-major) of the step.
template <class T, int N, int THREADS, bool KC, bool GATED>
struct Panel {
    static constexpr int E = int(sizeof(T));
    static constexpr int VEC = kChunk / E;
    static constexpr int BYTES = N * kStepBytes;
    static constexpr int LOADS = BYTES / (kChunk * THREADS);  // chunks a thread
    static constexpr int ROWCHUNKS = KC ? kStepBytes / kChunk : N * E / kChunk;
    static constexpr int ROWSTEP = THREADS / ROWCHUNKS;  // panel rows from load to load
    static_assert(THREADS % ROWCHUNKS == 0 && BYTES % (kChunk * THREADS) == 0, "");
    static_assert(!GATED || (KC && (N / 2) % ROWSTEP == 0), "");

    const Side<T> s;
    int64_t first;      // the panel's first row (column) in the operand
    int64_t end;        // the operand's rows (columns)
    uint32_t off[LOADS];
    int back;           // columns that the copies' origin lies before the first one

    // The thread's place in load i: panel row and chunk (logical).
    static __device__ __forceinline__ int row_of(int i) {
        return i * ROWSTEP + int(threadIdx.x) / ROWCHUNKS;
    }
    static __device__ __forceinline__ int chunk_of(int i) {
        const int phys = int(threadIdx.x) % ROWCHUNKS, r = row_of(i);
        return KC ? phys ^ swz(r) : (E == 2 ? phys ^ swzk(r, ROWCHUNKS) : phys);
    }
    // The matrix and its row behind panel row r.
    __device__ __forceinline__ int64_t source(int r, int seg, const T** p) const {
        if constexpr (GATED) {
            *p = r >= N / 2 ? s.p[1] : s.p[0];
            return first + (r & (N / 2 - 1));
        } else {
            *p = seg ? s.p[1] : s.p[0];
            return first + r;
        }
    }

    __device__ __forceinline__ Panel(const Side<T>& side, int64_t f, int64_t e)
        : s(side), first(f), end(e), back(0) {
        if constexpr (KC) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int r = GATED ? row_of(i) & (N / 2 - 1) : row_of(i);
                const int64_t last = end - 1 - first;
                off[i] = uint32_t((r < last ? r : last) * s.stride * E) + chunk_of(i) * kChunk;
            }
        } else {
            // a chunk that ends behind the row: its last whole one
            const int64_t last = end - VEC - first;
            if (last < 0) back = int(-last);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const int64_t c = int64_t(chunk_of(i)) * VEC;
                off[i] = uint32_t((row_of(i) * s.stride + (c < last ? c : last) + back) * E);
            }
        }
    }

    // Where the copies of the first step of segment `seg` (of half `seg` of a
    // gated panel) start, as a scalar, and how far on the next step's do.
    __device__ __forceinline__ uint64_t origin(int seg, int64_t k0) const {
        const T* const p = (seg ? s.p[1] : s.p[0]) +
                           (KC ? first * s.stride + k0 : k0 * s.stride + first - back);
        const uint64_t at = reinterpret_cast<uint64_t>(p);
        return uint64_t(scalar(uint32_t(at >> 32))) << 32 | scalar(uint32_t(at));
    }
    __device__ __forceinline__ uint64_t advance() const {
        return KC ? kStepBytes : uint64_t(s.stride) * kStepBytes;
    }
    // Start copy i of a whole step straight into LDS, `lds` the panel's address
    // there: lane l's 16 bytes go to the wavefront's 1 KiB at 16 l.  It is
    // written as assembly because of the waits: the compiler would hold every
    // LDS read back until all copies have landed, those of the other buffer
    // among them.  Whoever reads what they bring waits for the vector memory
    // counter and passes a barrier first (see landed()).  (m0 is reserved: the
    // compiler keeps nothing in it, and takes no clobber of it.)
    __device__ __forceinline__ void copy(int i, uint64_t at, uint32_t lds) const {
        // a raw buffer from there on, without a bound below 4 GiB
        const u32x4 rsrc = {uint32_t(at), uint32_t(at >> 32) & 0xFFFFu, 0xFFFFFFFFu, 0x00020000u};
        const uint32_t to = lds + uint32_t(i * THREADS) * kChunk;
        // (a write of m0 has to be a state old, a scalar that a vector
        // instruction wrote five, before the load reads them)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                     :: "s"(to), "v"(off[i]), "s"(rsrc) : "memory");
    }
    // Whether copy i belongs to the second half of a gated panel.
    static __device__ __forceinline__ bool upper(int i) { return GATED && i * ROWSTEP >= N / 2; }

    // The same through registers, for any alignment and with elements beyond
    // the ends of k and of a K-major row as zeros.
    // MOVE: a K-major row's last chunk as the copies place it.
    template <bool MOVE>
    __device__ __forceinline__ void fetch(int seg, int64_t k0, int64_t K, u32x4* v) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = row_of(i), c = chunk_of(i) * VEC;
            const T* p;
            int64_t at = source(KC ? r : 0, seg, &p), n;
            if constexpr (KC) {
                at = at < end ? at : end - 1;
                p += at * s.stride + k0 + c;
                n = K - k0 - c;
            } else {
                const int64_t last = end - VEC - first, cc = MOVE && c > last ? last : c;
                p += (k0 + r) * s.stride + first + cc;
                n = k0 + r < K ? end - first - cc : 0;
            }
            if (n >= VEC) v[i] = load_vec(p);
            else if (n > 0) v[i] = load_part(p, int(n));
            else v[i] = u32x4{0, 0, 0, 0};
        }
    }
    static __device__ __forceinline__ void put(AR_LDS char* lds, const u32x4* v) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            *(AR_LDS u32x4*)(lds + (i * THREADS + int(threadIdx.x)) * kChunk) = v[i];
    }
};

// A lane's reader of one operand's fragments: 16 bytes, k 8 (4) to a half of
// the wavefront, of row (column) lane % 32 of a square.
template <class T, int N, bool KC>
struct Frags {
    static constexpr int E = int(sizeof(T));
    int lane_off[4];

    // `base`: the wavefront's first row in the panel, a multiple of 32.
    __device__ __forceinline__ Frags(int base) {
        const int lane = int(threadIdx.x) & 63;
        if constexpr (KC) {
            const int r = base + (lane & 31);
#pragma unroll
            for (int s = 0; s < 4; ++s)
                lane_off[s] = r * kStepBytes + (((2 * s + (lane >> 5)) ^ swz(r)) * kChunk);
        } else if constexpr (E == 2) {
            const int l = lane & 15, g = lane >> 4;
            const int k = 8 * (g >> 1) + (l >> 2);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = base / 8 + 4 * j + 2 * (g & 1) + ((l & 3) >> 1);
                lane_off[j] = k * (N * 2) + ((c ^ swzk(k, N / 8)) * kChunk) + (l & 1) * 8;
            }
        } else {
            lane_off[0] = (4 * (lane >> 5)) * (N * 4) + (base + (lane & 31)) * 4;
        }
    }
    // Square j (32 rows on) of the panel at `lds`, substep s of the step's 4.
    __device__ __forceinline__ u32x4 read(const AR_LDS char* lds, int j, int s) const {
        if constexpr (KC) {
            return *(const AR_LDS u32x4*)(lds + lane_off[s] + j * 32 * kStepBytes);
        } else if constexpr (E == 2) {
            typedef AR_LDS s16x4* P;
            const AR_LDS char* at = lds + lane_off[j & 3] + (j >> 2) * 256 + s * 16 * (N * 2);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(at + 4 * (N * 2)));
            struct { s16x4 a, b; } both{lo, hi};
            return __builtin_bit_cast(u32x4, both);
        } else {
            u32x4 v;
            const AR_LDS char* at = lds + lane_off[0] + j * 128 + s * 8 * (N * 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = *(const AR_LDS uint32_t*)(at + e * (N * 4));
            return v;
        }
    }
};

template <class T>
__device__ __forceinline__ void multiply(const u32x4 l, const u32x4 r, f32x16& acc) {
    if constexpr (sizeof(T) == 2) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, l),
                                                      __builtin_bit_cast(bf16x8, r), acc, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(l[e]), __uint_as_float(r[e]),
                                                       acc, 0, 0, 0);
    }
}

// The block's work: blocks go to the 8 XCDs in turn, so XCD x takes a
// contiguous eighth of the tiles, in strips of `kStrip` tile rows that are
// walked along the columns: what its 32 CUs work on at a time shares panels
// in its L2.  The parts of the tiles that are split follow, an eighth each too.
constexpr int kStrip = 4;
__device__ __forceinline__ bool unit_of(const ProductShape& p, int64_t block, Unit* u) {
    const int64_t x = block & 7, i = block >> 3, share = (p.whole + 7) / 8;
    if (i < share) {
        *u = Unit{x * share + i, 0, 1};
        return u->tile < p.whole;
    }
    const int64_t rest = p.tiles - p.whole, parts = rest * p.splits, eighth = (parts + 7) / 8;
    const int64_t n = x * eighth + i - share;
    if (i - share >= eighth || n >= parts) return false;
    *u = Unit{p.whole + n % rest, int(n / rest), p.splits};
    return true;
}
// Where the tile lies in its product.
__device__ __forceinline__ void place_of(const ProductShape& p, int64_t t, int64_t* r, int64_t* c) {
    const int64_t per = kStrip * p.col_tiles, strip = t / per, in = t % per;
    const int64_t h = p.row_tiles - strip * kStrip < kStrip ? p.row_tiles - strip * kStrip : kStrip;
    *r = strip * kStrip + in % h;
    *c = in / h;
}
inline int64_t unit_blocks(const ProductShape& p) {
    return 8 * (ceil_div(p.whole, 8) + ceil_div((p.tiles - p.whole) * p.splits, 8));
}

// This wavefront's copies have landed in LDS and its own LDS stores are done;
// after the barrier that follows, so have all the block's.
__device__ __forceinline__ void landed() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
}

// The products of one tile: acc[i][j] is the square of row square i and column
// square j of the wavefront (gated: j = 0 the gate's, 1 the up projection's).
template <class T, int BR, int BC, int WR, int WC, bool RKC, bool LKC, bool GATED, bool DIRECT>
struct Tile {
    static constexpr int THREADS = 64 * WR * WC;
    static constexpr int SR = BR / (32 * WR), SC = BC / (32 * WC);  // squares of a wavefront
    static_assert(!GATED || SC == 2, "");
    using RP = Panel<T, BR, THREADS, RKC, false>;
    using LP = Panel<T, BC, THREADS, LKC, GATED>;
    static constexpr int HALF = RP::BYTES + LP::BYTES;  // one of the two buffers
    static constexpr int LDS = 2 * HALF;

    static __device__ __forceinline__ void run(const ProductShape& p, const Side<T>& R,
                                               const Side<T>& L, int64_t r0, int64_t c0, const Unit& u,
                                               AR_LDS char* lds, f32x16 (&acc)[SR][SC]) {
        const int wave = int(threadIdx.x) >> 6, wr = wave / WC, wc = wave % WC;
        const RP rp(R, r0, RKC ? p.rows : R.extent);
        const LP lp(L, c0, LKC ? p.cols : L.extent);
        const Frags<T, BR, RKC> rf(wr * SR * 32);
        const Frags<T, BC, LKC> lf(wc * (GATED ? 32 : SC * 32));
        constexpr int KS = StepOf<T>::K;
        const int per = int((p.K + KS - 1) / KS), all = per * p.segments;
        // this part's steps
        const int from = int(int64_t(all) * u.split / u.splits);
        const int steps = int(int64_t(all) * (u.split + 1) / u.splits) - from;
        if (steps == 0) return;
        u32x4 rv[DIRECT ? 1 : RP::LOADS], lv[DIRECT ? 1 : LP::LOADS];
        // The step whose copies come next: its segment and number there, and where
        // it lies in the operands.
        int seg = from >= per, k = from - seg * per;
        const int whole = int(p.K / KS);  // steps of a segment that are whole
        uint64_t ra = rp.origin(seg, int64_t(k) * KS), la[2];
        la[0] = lp.origin(GATED ? 0 : seg, int64_t(k) * KS);
        la[1] = GATED ? lp.origin(1, int64_t(k) * KS) : 0;
        const uint64_t rstep = rp.advance(), lstep = lp.advance();
        const uint32_t mine =
            scalar(uint32_t(reinterpret_cast<uintptr_t>(lds)) + uint32_t(wave) * 64 * kChunk);
        constexpr int COPIES = RP::LOADS + LP::LOADS;
        constexpr bool SPREAD = !(RKC && LKC);
        auto copy = [&](int n, int at) {
            if (n < RP::LOADS) rp.copy(n, ra, mine + at);
            else if (n < COPIES)
                lp.copy(n - RP::LOADS, LP::upper(n - RP::LOADS) ? la[1] : la[0],
                        mine + at + RP::BYTES);
        };
        // Any step but a whole one straight to LDS: through registers.
        auto fetch = [&](int at) {
            const int64_t k0 = int64_t(k) * KS;
            if constexpr (DIRECT) {
                u32x4 a[RP::LOADS], b[LP::LOADS];
                rp.template fetch<true>(seg, k0, p.K, a);
                lp.template fetch<true>(seg, k0, p.K, b);
                RP::put(lds + at, a);
                LP::put(lds + at + RP::BYTES, b);
            } else {
                rp.template fetch<false>(seg, k0, p.K, rv);
                lp.template fetch<false>(seg, k0, p.K, lv);
            }
        };
        auto put = [&](int at) {
            if constexpr (!DIRECT) {
                RP::put(lds + at, rv);
                LP::put(lds + at + RP::BYTES, lv);
            }
        };
        auto next = [&]() {
            ra += rstep;
            la[0] += lstep;
            la[1] += lstep;
            if (++k == per) {
                k = 0;
                ++seg;
                ra = rp.origin(1, 0);
                if constexpr (!GATED) la[0] = lp.origin(1, 0);
            }
        };
        // Fragments in two sets: one is read while the other's products run.
        u32x4 rf_[2][SR], lf_[2][SC];
        auto read = [&](int at, int s, int set) {
            const AR_LDS char* const buf = lds + at;
#pragma unroll
            for (int j = 0; j < SC; ++j)
                lf_[set][j] = lf.read(buf + RP::BYTES, GATED ? j * (BC / 64) : j, s);
#pragma unroll
            for (int i = 0; i < SR; ++i) rf_[set][i] = rf.read(buf, i, s);
            // a phase's reads stay ahead of its products, and out of the next one's
            __builtin_amdgcn_sched_barrier(0);
        };
        // The products of a set; with `copies` some of the next step's copies among
        // them, so that the matrix unit does not wait for their issue.  The 8
        // wavefronts' copies of a step keep the address unit busy for as long as the
        // products of two quarters take, and are spread over as many; not where both
        // operands are K-contiguous, whose copies touch more lines and take longer
        // to arrive (8192 x 4096 x 16384: dx 1.73 -> 1.69 ms and the weight
        // gradients 1.78 -> 1.72 with spread copies, but the forward 1.95 -> 2.00).
        auto products = [&](int set, bool copies, int half, int at) {
            constexpr int H = SPREAD ? COPIES / 2 : COPIES, S = SR * SC;
            static_assert(COPIES % 2 == 0, "");
#pragma unroll
            for (int n = 0; n < S; ++n) {
                multiply<T>(lf_[set][n % SC], rf_[set][n / SC], acc[n / SC][n % SC]);
                if (DIRECT && copies) {
#pragma unroll
                    for (int c = n * H / S; c < (n + 1) * H / S; ++c) copy(half * H + c, at);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        for (int n = 0; n < 2; ++n) {  // the first two steps
            if (n == 1) {
                put(0);
                landed();
                __builtin_amdgcn_s_barrier();
                if (steps == 1) break;
                next();
            }
            if (DIRECT && k < whole) {
#pragma unroll
                for (int c = 0; c < COPIES; ++c) copy(c, n * HALF);
            } else {
                fetch(n * HALF);
            }
        }
        read(0, 0, 0);
        int at = 0;
        bool late = false;  // whether the next step's second half is still to come
        for (int t = 0; t < steps; ++t) {
            read(at, 1, 1);
            products(0, SPREAD && late, 1, HALF - at);
            read(at, 2, 0);
            products(1, false, 0, 0);
            read(at, 3, 1);
            products(0, false, 0, 0);
            // The step's last fragments are here, and the next step's panels: after
            // the barrier this buffer is free, and the other one whole.
            if (t + 1 < steps) put(HALF - at);
            landed();
            __builtin_amdgcn_s_barrier();
            late = t + 2 < steps;
            if (late) {
                next();
                if (!DIRECT || k >= whole) {
                    fetch(at);
                    late = false;
                }
            }
            if (t + 1 < steps) read(HALF - at, 0, 0);
            products(1, late, 0, at);
            at = HALF - at;
        }
    }
};

// Squares to memory: each wavefront passes a row of squares at a time through
// its own part of LDS, as fp32, and stores whole runs of the output's rows.
// `f(i, j, e)` is element e of the accumulators' layout.
template <int SC>
struct Store {
    static constexpr int PITCH = SC * 32 + 4;              // floats a row
    static constexpr int BYTES = 32 * PITCH * 4;           // a wavefront's part
    template <class F>
    static __device__ __forceinline__ void fill(AR_LDS float* part, F&& f) {
        const int lane = int(threadIdx.x) & 63;
#pragma unroll
        for (int j = 0; j < SC; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                typedef float f4 __attribute__((ext_vector_type(4)));
                const f4 v = {f(j, 4 * q), f(j, 4 * q + 1), f(j, 4 * q + 2), f(j, 4 * q + 3)};
                *(AR_LDS f4*)(part + (lane & 31) * PITCH + j * 32 + 8 * q + 4 * (lane >> 5)) = v;
            }
    }
    // rows r0 .. of `out`, columns c0 .. of the SC * 32; the last columns of an
    // incomplete chunk of `shift` fewer lie so much further on
    template <class T>
    static __device__ __forceinline__ void store(const AR_LDS float* part, T* out, int64_t stride,
                                                 int64_t r0, int64_t rows, int64_t c0, int64_t cols,
                                                 bool accumulate, int chunk, int shift) {
        constexpr int VEC = Num<T>::VEC, PER = SC * 32 / VEC, ROWS = 64 / PER;
        const int lane = int(threadIdx.x) & 63;
#pragma unroll
        for (int b = 0; b < 32; b += ROWS) {
            const int r = b + lane / PER, c = lane % PER * VEC;
            const int64_t left = cols - c0 - c;
            if (r0 + r >= rows || left <= 0) continue;
            T* const at = out + (r0 + r) * stride + c0 + c;
            const AR_LDS float* const row = part + r * PITCH;
            float v[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                v[e] = row[c + e + (shift && left - e <= chunk - shift ? shift : 0)];
            const int n = int(left < VEC ? left : VEC);
            if (accumulate) {
                float old[VEC];
                Num<T>::unpack(n == VEC ? load_vec(at) : load_part(at, n), old);
#pragma unroll
                for (int e = 0; e < VEC; ++e) v[e] += old[e];
            }
            if (n == VEC) store_vec(at, Num<T>::pack(v));
            else store_part(at, Num<T>::pack(v), n);
        }
    }
};

}  // namespace arp
