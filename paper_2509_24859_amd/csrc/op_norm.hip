// Norm after a block, gate, residual scale, residual sum and the norm before the next block, forward and backward,
// and their C entry points.
//
// A row's channels lie in the registers of one workgroup, eight to a thread, so that every tensor is read once and
// written once: the pass is bound by memory.  A workgroup takes rows in turn and keeps what belongs to its channels
// (weights, biases, scale, and in the backward pass the sums over rows) in registers throughout.  In the backward pass a
// workgroup works on several rows at a time where they are short, each by a team of its threads, and adds the teams' sums up
// in LDS: as many waits are hidden as by so many workgroups, with one's partial sums.
//
// Measured, bfloat16, RMS norms on both sides, one gate, a scale: forward of 4,096 x 8,192 63 us, 4.2 TB/s, backward 97 us, 4.1
// TB/s (a copy reaches 4.9); one row 4.5 us in the kernel.  Backward of 11,366 x 1,176: 54 us, 3.0 TB/s, in float32 95, 3.4.  A
// workgroup of 1,024 threads has a compute unit to itself: between its sums over the row it waits, and half of the registers
// that would let a second one in hold the next row and the vectors.
#include <math.h>

#include <type_traits>

#include "harp_ctx.h"
#include "ops_common.h"

using namespace harp;
using namespace harp::ops;

namespace {

constexpr int kPer = 8;                               // channels a thread holds
constexpr int kMaxThreads = HARP_NORM_MAX_COLS / kPer;
constexpr int kMaxWaves = kMaxThreads / kWave;
constexpr int kFewThreads = 512, kTeamThreads = 768;    // a thread has 256, 168 and, with kMaxThreads, 128 registers

// Everything but the data, as the kernels see it.
struct Form {
    int64_t rows, rows_per_gate, ldgate;
    int32_t cols, after, before, gate_act;
    float eps_after, eps_before;
    const float *w_after, *b_after, *w_before, *b_before, *scale;
    const void *gate;
    bool past;                                        // results are stored past the caches
};

// The channels of a thread: 8 t .. 8 t + 7.
__device__ __forceinline__ int channel(int j) { return int(threadIdx.x) * kPer + j; }

// A thread's channels of a row as they are stored: what is asked for ahead of its use takes half the registers in 16 bits.
// Pieces of 16 bytes; WIDE: every row begins at a multiple of 16 bytes and holds whole pieces.  Without, the pieces are read
// where they lie (memory takes any alignment of elements: the backward pass of 2,313 rows of 1,155 floats 38 us element by
// element, 33 so), and the last one of a row element by element.
template <typename T, bool WIDE> struct Raw {
    static constexpr int kHold = 16 / int(sizeof(T)), kPieces = kPer / kHold;
    typedef T Piece __attribute__((ext_vector_type(kHold)));
    typedef Piece Loose __attribute__((aligned(sizeof(T))));
    typedef typename std::conditional<WIDE, Piece, Loose>::type Stored;
    Piece piece[kPieces];

    // In the row's last piece the elements that are there, the last one in the place of those that are not (no load waits
    // for another to be chosen from); get() puts zeros there.
    __device__ __forceinline__ void load(const T *row, int cols) {
        if (WIDE || channel(kPer) <= cols) {
#pragma unroll
            for (int k = 0; k < kPieces; ++k) piece[k] = Piece(T(0.0f));
            if (channel(kPer) <= cols)
#pragma unroll
                for (int k = 0; k < kPieces; ++k) piece[k] = *reinterpret_cast<const Stored *>(row + channel(k * kHold));
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) piece[j / kHold][j % kHold] = row[channel(j) < cols ? channel(j) : cols - 1];
        }
    }
    __device__ __forceinline__ void get(float (&v)[kPer], int cols) const {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            v[j] = to_f32(T(piece[j / kHold][j % kHold]));
            if (!WIDE && channel(j) >= cols) v[j] = 0;
        }
    }
    // past: not kept in the caches
    __device__ __forceinline__ void store(T *row, int cols, const float (&v)[kPer], bool past) {
        row += channel(0);
#pragma unroll
        for (int j = 0; j < kPer; ++j) piece[j / kHold][j % kHold] = T(v[j]);
        if (channel(kPer) <= cols) {
#pragma unroll
            for (int k = 0; k < kPieces; ++k) store_as<WIDE ? 16 : int(sizeof(T))>(row + k * kHold, piece[k], past);
        } else if (!WIDE) {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                if (channel(j) < cols) row[j] = T(v[j]);
        }
    }
};

// A vector over the channels, `other` where there is none; several are asked for before the first is taken.
struct Vector {
    Raw<float, false> raw;
    const float *p;
    __device__ __forceinline__ Vector(const float *at, int cols) : p(at) {
        if (p) raw.load(p, cols);
    }
    __device__ __forceinline__ void get(float (&v)[kPer], int cols, float other) const {
        if (p) {
            raw.get(v, cols);
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = other;
        }
    }
};

// N sums over a row's threads (threadIdx.x), the same in every thread.  `turn` alternates between two buffers, so that one barrier a
// round is enough: a buffer is written again only after everybody has passed the next round's barrier.
struct Exchange {
    f32x4 (*buf)[kMaxWaves];
    int turn;
};
template <int N> __device__ __forceinline__ void block_sum(float (&v)[N], Exchange &x) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const float s = sum16(v[k]);
        v[k] = (lane_of(s, 0) + lane_of(s, 16)) + (lane_of(s, 32) + lane_of(s, 48));
    }
    const int waves = blockDim.x / kWave;
    if (waves == 1) return;
    f32x4 *b = x.buf[x.turn] + threadIdx.y * waves;
    x.turn ^= 1;
    if (threadIdx.x % kWave == 0) {
        f32x4 q = {0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < N; ++k) q[k] = v[k];
        b[threadIdx.x / kWave] = q;
    }
    __syncthreads();
    const int w = threadIdx.x % 16;
    const f32x4 q = w < waves ? b[w] : f32x4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = sum16(q[k]);
}

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + __expf(-x)); }
__device__ __forceinline__ float rstd_of(float squares, float inv_cols, float eps) { return 1.0f / sqrtf(squares * inv_cols + eps); }

__device__ __forceinline__ void subtract(float (&v)[kPer], float mean, int cols) {
#pragma unroll
    for (int j = 0; j < kPer; ++j)
        if (channel(j) < cols) v[j] -= mean;           // channels beyond cols stay 0
}

// v - mean (LAYER), and 1 / sqrt(mean of squares + eps) of what is left.
__device__ __forceinline__ float center(float (&v)[kPer], int kind, int cols, float eps, Exchange &x) {
    const float inv_cols = 1.0f / float(cols);
    if (kind == HARP_NORM_LAYER) {
        float s[1] = {0};
#pragma unroll
        for (int j = 0; j < kPer; ++j) s[0] += v[j];
        block_sum(s, x);
        subtract(v, s[0] * inv_cols, cols);
    }
    float s[1] = {0};
#pragma unroll
    for (int j = 0; j < kPer; ++j) s[0] += v[j] * v[j];
    block_sum(s, x);
    return rstd_of(s[0], inv_cols, eps);
}

// BIAS: there is a b_after or b_before.  A thread has the 128 registers that workgroups of 1,024 threads leave it and needs 71 to
// 128 of them, whatever the type and alignment: short rows are no reason for a variant of fewer threads.
template <typename T, bool WIDE, bool BIAS>
__global__ __launch_bounds__(kMaxThreads) void norm_forward(Form f, const T *x, int64_t ldx, const T *y, int64_t ldy, T *h,
                                                            int64_t ldh, T *z, int64_t ldz) {
    __shared__ f32x4 buf[2][kMaxWaves];
    Exchange ex = {buf, 0};
    const int cols = f.cols;
    Raw<T, WIDE> next_x, next_y;
    auto ask = [&](int64_t r) {
        if (y) next_y.load(y + r * ldy, cols);
        if (x) next_x.load(x + r * ldx, cols);
    };
    ask(blockIdx.x);                                     // there are no more workgroups than rows
    float wa[kPer], ba[kPer], wb[kPer], bb[kPer], sc[kPer];
    {
        const Vector vs(f.scale, cols), va(f.w_after, cols), vb(f.w_before, cols), vab(BIAS ? f.b_after : nullptr, cols),
            vbb(BIAS ? f.b_before : nullptr, cols);
        vs.get(sc, cols, 1.0f);
        va.get(wa, cols, 1.0f);
        vb.get(wb, cols, 1.0f);
        vab.get(ba, cols, 0.0f);
        vbb.get(bb, cols, 0.0f);
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        wa[j] *= sc[j];
        ba[j] *= sc[j];
    }
    for (int64_t r = blockIdx.x; r < f.rows; r += gridDim.x) {
        float v[kPer];
        Raw<T, WIDE> here_x = next_x, gate;
        if (f.gate && y) gate.load(static_cast<const T *>(f.gate) + r / f.rows_per_gate * f.ldgate, cols);
        if (y) next_y.get(v, cols);
        else next_x.get(v, cols);
        if (r + gridDim.x < f.rows) ask(r + gridDim.x);
        if (y) {
            float rstd = 1.0f;
            if (f.after != HARP_NORM_NONE) rstd = center(v, f.after, cols, f.eps_after, ex);
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = BIAS ? v[j] * rstd * wa[j] + ba[j] : v[j] * rstd * wa[j];
            if (f.gate) {
                float g[kPer];
                gate.get(g, cols);
#pragma unroll
                for (int j = 0; j < kPer; ++j) v[j] *= f.gate_act == HARP_GATE_SIGMOID ? sigmoid(g[j]) : g[j];
            }
            if (x) {
                float a[kPer];
                here_x.get(a, cols);
#pragma unroll
                for (int j = 0; j < kPer; ++j) v[j] += a[j];
            }
            if (h) here_x.store(h + r * ldh, cols, v, f.past);
        }
        if (f.before != HARP_NORM_NONE) {
            const float rstd = center(v, f.before, cols, f.eps_before, ex);
#pragma unroll
            for (int j = 0; j < kPer; ++j) v[j] = BIAS ? v[j] * rstd * wb[j] + bb[j] : v[j] * rstd * wb[j];
            here_x.store(z + r * ldz, cols, v, f.past);
        }
    }
}

// How rows are dealt to workgroups in the backward pass: slabs of rows of which none reaches into a gate's group
// without holding it whole or lying inside it, so that a group's sum is either a workgroup's own or a sum of
// workgroups' partial sums.
struct Slabs {
    int64_t rows;             // rows of a slab
    int64_t per_group;        // slabs of a gate's group (without a gate: of all rows), 0: a slab holds whole groups
    int64_t rows_per_group;
    int64_t count;
};
__device__ __forceinline__ void slab_rows(const Slabs &s, int64_t all, int64_t i, int64_t &begin, int64_t &end) {
    if (s.per_group == 0) {
        begin = i * s.rows;
        end = begin + s.rows < all ? begin + s.rows : all;
    } else {
        const int64_t group = i / s.per_group, stop = (group + 1) * s.rows_per_group;
        begin = group * s.rows_per_group + i % s.per_group * s.rows;
        end = begin + s.rows < stop ? begin + s.rows : stop;
        end = end < all ? end : all;
    }
}

// d through the norm: (d - mean(d) - a rstd^2 mean(d a)) rstd, the first mean for LAYER only.  c0 = sum d, c1 = sum d a.
__device__ __forceinline__ float through(float d, float a, float rstd, float c0, float c1, int kind, float inv_cols) {
    if (kind == HARP_NORM_NONE) return d;
    const float m = kind == HARP_NORM_LAYER ? c0 * inv_cols : 0.0f;
    return (d - m - a * (rstd * rstd) * (c1 * inv_cols)) * rstd;
}

// With D the gradient of h, n = the normalised y, f the gate's factor, the sums over rows are all made of four:
//   A1 = sum D f n, A0 = sum D f:   dw_after = scale A1, db_after = scale A0, dscale = w_after A1 + b_after A0
//   B1 = sum dz n(h), B0 = sum dz:  dw_before, db_before
// and a gate's f is the same for all rows of its group: with G1 = sum D n, G0 = sum D over them A1 = f G1, A0 = f G0 and
// dgate = f' scale (w_after G1 + b_after G0).  A slab inside one group (GROUPS false) adds up G alone.
// BIAS: there is a b_after, or db_after or db_before is wanted; without, A0, B0 and G0 are not needed.
// The statistics of both norms are summed in one round, what the second gradient needs in another; the next row and its gate are
// asked for before the current one is worked on, the first before the vectors.
// A team is the threads of one threadIdx.y; teams take a slab's rows, with GROUPS its groups, in turn.
enum { kA1, kB1, kA0, kB0 };
template <typename T, bool WIDE, bool BIAS, bool GROUPS, int MOST>
__global__ __launch_bounds__(MOST) void norm_backward(Form f, Slabs slabs, const T *dh, int64_t lddh, const T *dz, int64_t lddz,
                                                             const T *h, int64_t ldh, const T *y, int64_t ldy, T *dx, int64_t lddx,
                                                             T *dy, int64_t lddy, T *dgate, int64_t lddgate, float *partial,
                                                             float *gate_partial) {
    __shared__ f32x4 buf[2][kMaxWaves], pool[2][MOST == kMaxThreads ? 1 : MOST];
    Exchange ex = {buf, 0};
    const int cols = f.cols, teams = MOST == kMaxThreads ? 1 : int(blockDim.y);
    const int team = MOST == kMaxThreads ? 0 : __builtin_amdgcn_readfirstlane(int(threadIdx.y));
    const float inv_cols = 1.0f / float(cols);
    int64_t begin, end;
    slab_rows(slabs, f.rows, blockIdx.x, begin, end);

    float wb[kPer], c[kPer], cb[kPer];                   // c: scale w_after, times the gate's factor where that is one vector; cb: scale b_after
    float B1[kPer] = {}, B0[kPer] = {}, A1[kPer] = {}, A0[kPer] = {}, G1[kPer] = {}, G0[kPer] = {};
    Raw<T, WIDE> gate, next_gate;
    auto load_gate = [&](int64_t r, Raw<T, WIDE> &to) { to.load(static_cast<const T *>(f.gate) + r / f.rows_per_gate * f.ldgate, cols); };
    auto factors = [&](float (&factor)[kPer], float (&slope)[kPer]) {
        gate.get(factor, cols);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            slope[j] = 1.0f;
            if (f.gate_act == HARP_GATE_SIGMOID) {
                factor[j] = sigmoid(factor[j]);
                slope[j] = factor[j] * (1.0f - factor[j]);
            }
        }
    };
    Raw<T, WIDE> next_h, next_dz, next_y, next_dh;
    auto ask = [&](int64_t r) {
        if (dz) {
            next_h.load(h + r * ldh, cols);
            next_dz.load(dz + r * lddz, cols);
        }
        if (y) next_y.load(y + r * ldy, cols);
        if (dh) next_dh.load(dh + r * lddh, cols);
        if (GROUPS) load_gate(r, next_gate);
    };
    const int64_t unit = GROUPS ? f.rows_per_gate : 1;
    int64_t r = begin + team * unit, left = unit, following;
    if (r < end) ask(r);
    {
        const bool gated = !GROUPS && f.gate && begin < end;
        if (gated) load_gate(begin, gate);
        const Vector vb(f.w_before, cols), vs(f.scale, cols), va(f.w_after, cols), vab(BIAS && GROUPS ? f.b_after : nullptr, cols);
        vb.get(wb, cols, 1.0f);
        vs.get(cb, cols, 1.0f);
        va.get(c, cols, 1.0f);
        float ba[kPer], factor[kPer], slope[kPer];
        vab.get(ba, cols, 0.0f);
        if (gated) factors(factor, slope);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            c[j] *= cb[j];
            cb[j] *= ba[j];
            if (gated) c[j] *= factor[j];
        }
    }
    // Every team makes as many turns, so that all meet at the barriers; one whose rows are done adds nothing.
    for (int64_t first = begin; first < end; r = following) {
        const bool live = r < end;
        following = r + 1;
        if (--left == 0) {
            following += (teams - 1) * unit;
            first += teams * unit;
            left = unit;
        }
        float a[kPer] = {}, e[kPer] = {}, b[kPer] = {}, d[kPer] = {};
        if (live) {
            if (dz) {
                next_h.get(a, cols);
                next_dz.get(e, cols);
            }
            if (y) next_y.get(b, cols);
            if (dh) next_dh.get(d, cols);
            if (GROUPS) gate = next_gate;
            if (following < end) ask(following);
        }
        if (f.before == HARP_NORM_LAYER || f.after == HARP_NORM_LAYER) {
            float m[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                m[0] += a[j];
                m[1] += b[j];
            }
            block_sum(m, ex);
            if (f.before == HARP_NORM_LAYER) subtract(a, m[0] * inv_cols, cols);
            if (f.after == HARP_NORM_LAYER) subtract(b, m[1] * inv_cols, cols);
        }
        float s[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const float g = e[j] * wb[j];
            s[0] += a[j] * a[j];
            s[1] += g * a[j];
            s[2] += g;
            s[3] += b[j] * b[j];
        }
        block_sum(s, ex);
        const float rstd_h = rstd_of(s[0], inv_cols, f.eps_before);
        const float rstd_y = f.after != HARP_NORM_NONE ? rstd_of(s[3], inv_cols, f.eps_after) : 1.0f;
        if (dz && live) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                B1[j] += e[j] * (a[j] * rstd_h);
                if (BIAS) B0[j] += e[j];
                d[j] += through(e[j] * wb[j], a[j], rstd_h, s[2], s[1], f.before, inv_cols);
            }
        }
        Raw<T, WIDE> out;
        if (dx && live) out.store(dx + r * lddx, cols, d, f.past);
        if (!y) continue;
        float k[2] = {0, 0};
        if (live) {
            float factor[kPer], slope[kPer];
            if (GROUPS) factors(factor, slope);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                if (channel(j) >= cols) d[j] = 0;
                G1[j] += d[j] * (b[j] * rstd_y);
                if (BIAS) G0[j] += d[j];
                d[j] *= GROUPS ? c[j] * factor[j] : c[j];
                k[0] += d[j];
                k[1] += d[j] * b[j];
            }
        }
        if (f.after != HARP_NORM_NONE) {
            block_sum(k, ex);
#pragma unroll
            for (int j = 0; j < kPer; ++j) d[j] = through(d[j], b[j], rstd_y, k[0], k[1], f.after, inv_cols);
        }
        if (!live) continue;
        if (dy) out.store(dy + r * lddy, cols, d, f.past);
        if (GROUPS && (left == unit || r + 1 == f.rows)) {       // a gate's last row: its gradient, and its share of the sums
            float factor[kPer], slope[kPer];
            factors(factor, slope);
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                A1[j] += factor[j] * G1[j];
                slope[j] *= BIAS ? c[j] * G1[j] + cb[j] * G0[j] : c[j] * G1[j];
                if (BIAS) A0[j] += factor[j] * G0[j];
                G1[j] = G0[j] = 0;
            }
            if (dgate) out.store(dgate + r / f.rows_per_gate * lddgate, cols, slope, f.past);
        }
    }
    // The teams' sums, in the teams' order, to the first.
    auto gather = [&](float (&v)[kPer]) {
        const int at = int(threadIdx.x), step = int(blockDim.x);
        if (team) {
            pool[0][at + (team - 1) * step] = f32x4{v[0], v[1], v[2], v[3]};
            pool[1][at + (team - 1) * step] = f32x4{v[4], v[5], v[6], v[7]};
        }
        __syncthreads();
        if (!team)
            for (int i = 0; i < teams - 1; ++i)
#pragma unroll
                for (int j = 0; j < kPer; ++j) v[j] += pool[j / 4][at + i * step][j % 4];
        __syncthreads();
    };
    if (teams > 1) {
        gather(GROUPS ? A1 : G1);
        gather(B1);
        if (BIAS) {
            gather(GROUPS ? A0 : G0);
            gather(B0);
        }
        if (team) return;
    }
    auto put = [&](float *to, const float (&v)[kPer]) {
        Raw<float, false> raw;
        raw.store(to, cols, v, false);
    };
    if (!GROUPS) {
        float factor[kPer], slope[kPer];
#pragma unroll
        for (int j = 0; j < kPer; ++j) factor[j] = 1.0f;
        const bool gated = f.gate && y && begin < end;
        if (gated) {
            load_gate(begin, gate);
            const Vector vs(gate_partial ? f.scale : nullptr, cols), va(gate_partial ? f.w_after : nullptr, cols),
                vab(BIAS && gate_partial ? f.b_after : nullptr, cols);
            factors(factor, slope);
            float wa[kPer], ba[kPer], sc[kPer];
            vs.get(sc, cols, 1.0f);
            va.get(wa, cols, 1.0f);
            vab.get(ba, cols, 0.0f);
#pragma unroll
            for (int j = 0; j < kPer; ++j) slope[j] *= sc[j] * (BIAS ? wa[j] * G1[j] + ba[j] * G0[j] : wa[j] * G1[j]);
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j) slope[j] = 0;
        }
        if (gate_partial) put(gate_partial + int64_t(blockIdx.x) * cols, slope);
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            A1[j] = factor[j] * G1[j];
            A0[j] = factor[j] * G0[j];
        }
    }
    if (!partial) return;
    constexpr int kSums = BIAS ? 4 : 2;
    float *p = partial + int64_t(blockIdx.x) * kSums * cols;
    put(p + kA1 * int64_t(cols), A1);
    put(p + kB1 * int64_t(cols), B1);
    if (BIAS) {
        put(p + kA0 * int64_t(cols), A0);
        put(p + kB0 * int64_t(cols), B0);
    }
}

// Sums of the slabs' partial sums: 32 channels a workgroup, 32 threads to a channel, each a run of slabs in order, then
// the runs in order.
constexpr int kJoinCols = 32, kJoinRuns = 32;
template <int N> __device__ __forceinline__ void join_runs(const float *partial, int block, int64_t count, int64_t stride, int64_t pitch, int cols, float (&v)[N]) {
    __shared__ float runs[N][kJoinRuns][kJoinCols + 1];
    const int c = block * kJoinCols + threadIdx.x % kJoinCols, run = threadIdx.x / kJoinCols;
    const int64_t each = (count + kJoinRuns - 1) / kJoinRuns, first = run * each, last = first + each < count ? first + each : count;
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0;
    if (c < cols)
#pragma unroll 4
        for (int64_t i = first; i < last; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += partial[i * stride + k * pitch + c];
#pragma unroll
    for (int k = 0; k < N; ++k) runs[k][run][threadIdx.x % kJoinCols] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] = 0;
        if (run == 0)
            for (int i = 0; i < kJoinRuns; ++i) v[k] += runs[k][i][threadIdx.x % kJoinCols];
    }
}
struct Sums { float *dw_after, *db_after, *dscale, *dw_before, *db_before; };
// What gates' groups of several slabs have of their gates' gradients, [group][per_group][cols].
struct Gates {
    const float *partial;
    void *dgate;
    int64_t per_group, ld;
};
// Few slabs are added up by a thread for each channel: by runs, 226 gates of one slab each and 1,883 channels cost 23 us.
constexpr int kJoinSlabs = 32, kJoinThreads = kJoinCols * kJoinRuns;
__host__ __device__ inline int gate_blocks(int64_t per_group, int cols) {
    const int at_once = per_group > kJoinSlabs ? kJoinCols : kJoinThreads;
    return (cols + at_once - 1) / at_once;
}
// Workgroups: first those of the sums, if there is `partial`, then gate_blocks() for each group.
template <typename T, bool BIAS>
__global__ __launch_bounds__(kJoinThreads) void norm_sums(Form f, const float *partial, int64_t count, Sums out, int accumulate, Gates gates) {
    constexpr int N = BIAS ? 4 : 2;
    const uint32_t mine = partial ? uint32_t(f.cols + kJoinCols - 1) / kJoinCols : 0;
    if (blockIdx.x >= mine) {
        const uint32_t blocks = uint32_t(gate_blocks(gates.per_group, f.cols));
        const int64_t group = (blockIdx.x - mine) / blocks;
        const int block = int((blockIdx.x - mine) % blocks);
        const float *p = gates.partial + group * gates.per_group * f.cols;
        T *to = static_cast<T *>(gates.dgate) + group * gates.ld;
        if (gates.per_group > kJoinSlabs) {
            float v[1];
            join_runs<1>(p, block, gates.per_group, f.cols, 0, f.cols, v);
            const int c = block * kJoinCols + threadIdx.x;
            if (threadIdx.x < kJoinCols && c < f.cols) to[c] = T(v[0]);
        } else {
            const int c = block * kJoinThreads + threadIdx.x;
            if (c >= f.cols) return;
            float v = 0;
#pragma unroll 8
            for (int i = 0; i < int(gates.per_group); ++i) v += p[int64_t(i) * f.cols + c];
            to[c] = T(v);
        }
        return;
    }
    float v[N];
    join_runs<N>(partial, blockIdx.x, count, int64_t(N) * f.cols, f.cols, f.cols, v);
    const int c = blockIdx.x * kJoinCols + threadIdx.x;
    if (threadIdx.x >= kJoinCols || c >= f.cols) return;
    const float w = f.w_after ? f.w_after[c] : 1.0f, s = f.scale ? f.scale[c] : 1.0f;
    auto put = [&](float *p, float x) {
        if (p) p[c] = accumulate ? p[c] + x : x;
    };
    const float a0 = BIAS ? v[N > 2 ? kA0 : 0] : 0.0f, b0 = BIAS ? v[N > 2 ? kB0 : 0] : 0.0f;
    put(out.dw_after, s * v[kA1]);
    put(out.db_after, s * a0);
    put(out.dscale, BIAS && f.b_after ? w * v[kA1] + f.b_after[c] * a0 : w * v[kA1]);
    put(out.dw_before, v[kB1]);
    put(out.db_before, b0);
}
int threads_for(int cols) { return int(round_up(size_t((cols + kPer - 1) / kPer), kWave)); }

int teams_for(int cols, int threads) {
    const int t = threads_for(cols);
    return t <= threads ? threads / t : 1;
}
// Rows of a gate's group that there are: the kernels make a turn for each.
int64_t group_rows(const harp_norm *n) { return n->gate && n->rows_per_gate < n->rows ? n->rows_per_gate : n->rows; }

// A workgroup a compute unit (places), with as many teams as it holds; a second one would bring more partial sums than it
// hides of the first's waits (2,313 rows of 1,155 floats, a gate for 257: one 33, two 50, three 59 us).  Gates' groups are
// split into as many slabs as there are places for them, or whole ones are put together, a team for each, whichever makes fewer
// turns of the busiest place; a slab costs four turns more, for its vectors and its partial sums.  The layout does not depend
// on which gradients are wanted: the caller's workspace is sized before that is known.
Slabs slabs_for(const harp_ctx *ctx, const harp_norm *n) {
    if (n->rows == 0) return Slabs{0, 0, 0, 0};
    const int64_t places = ctx->n_cu, teams = teams_for(n->cols, kTeamThreads), turns = 4;
    const int64_t per = group_rows(n), groups = (n->rows + per - 1) / per;
    const int64_t most = (per + teams - 1) / teams;
    int64_t parts = places / groups < most ? places / groups : most;
    if (parts < 1) parts = 1;
    const int64_t rows = (per + parts - 1) / parts, whole = (groups + places - 1) / places;
    parts = (per + rows - 1) / rows;                     // those that hold rows
    const int64_t split = (groups * parts + places - 1) / places * ((rows + teams - 1) / teams + turns);
    const int64_t together = (whole + teams - 1) / teams * per + turns;
    if (split < together) return Slabs{rows, parts, per, groups * parts};
    return Slabs{whole * per, 0, 0, (n->rows + whole * per - 1) / (whole * per)};
}

int check_norm(harp_ctx *ctx, const harp_norm *n) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!n) return fail(ctx, HARP_ERR_INVALID_ARG, "null norm");
    if (n->rows < 0 || n->rows >= int64_t(1) << 31) return fail(ctx, HARP_ERR_SHAPE, "rows must be in 0 .. 2^31 - 1");
    if (n->cols < 1 || n->cols > HARP_NORM_MAX_COLS) return fail(ctx, HARP_ERR_SHAPE, "cols must be in 1 .. %d", HARP_NORM_MAX_COLS);
    if (!type_bytes(n->type)) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown type");
    if (n->after < HARP_NORM_NONE || n->after > HARP_NORM_LAYER || n->before < HARP_NORM_NONE || n->before > HARP_NORM_LAYER)
        return fail(ctx, HARP_ERR_INVALID_ARG, "unknown norm");
    if (!(n->eps_after >= 0) || !(n->eps_before >= 0)) return fail(ctx, HARP_ERR_INVALID_ARG, "eps must be >= 0");
    if (!aligned(n->w_after, 4) || !aligned(n->b_after, 4) || !aligned(n->w_before, 4) || !aligned(n->b_before, 4) || !aligned(n->scale, 4))
        return fail(ctx, HARP_ERR_INVALID_ARG, "a vector is not aligned to its elements");
    if (n->gate) {
        if (n->rows_per_gate < 1) return fail(ctx, HARP_ERR_SHAPE, "rows_per_gate must be >= 1");
        if (n->ldgate < n->cols) return fail(ctx, HARP_ERR_SHAPE, "ldgate is below cols");
        if (n->gate_act != HARP_GATE_LINEAR && n->gate_act != HARP_GATE_SIGMOID) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown gate_act");
    }
    return HARP_OK;
}

struct Operand { const void *p; int64_t ld; const char *name; };
// Leading dimensions and element alignment of what is there; whether all of it can be read in pieces of 16 bytes.
int check_operands(harp_ctx *ctx, const harp_norm *n, const Operand *o, int count, bool &wide) {
    const size_t e = size_t(type_bytes(n->type));
    wide = n->cols % kPer == 0;
    for (int i = 0; i < count; ++i) {
        if (!o[i].p) continue;
        if (o[i].ld < n->cols) return fail(ctx, HARP_ERR_SHAPE, "%s: leading dimension below cols", o[i].name);
        if (!aligned(o[i].p, e)) return fail(ctx, HARP_ERR_INVALID_ARG, "%s is not aligned to its elements", o[i].name);
        wide = wide && aligned(o[i].p, 16) && o[i].ld * int64_t(e) % 16 == 0;
    }
    return HARP_OK;
}

Form form_of(const harp_norm *n) {
    return Form{n->rows, n->gate ? group_rows(n) : 1, n->ldgate, n->cols, n->after, n->before, n->gate_act, n->eps_after, n->eps_before,
                n->w_after, n->b_after, n->w_before, n->b_before, n->scale, n->gate,
                // results larger than the L2 caches: forward of 4,096 x 8,192 65.3 us through them, 63.8 past them
                size_t(n->rows) * size_t(n->cols) * size_t(type_bytes(n->type)) >= size_t(32) << 20};
}

template <typename T, bool WIDE>
void run_forward(const harp_ctx *ctx, const harp_norm *n, const void *x, int64_t ldx, const void *y, int64_t ldy, void *h, int64_t ldh,
                 void *z, int64_t ldz, hipStream_t st) {
    const int threads = threads_for(n->cols);
    const int64_t most = int64_t(ctx->n_cu) * (2048 / threads < 16 ? 2048 / threads : 16);
    const dim3 grid(uint32_t(n->rows < most ? n->rows : most)), block(threads);
#define RUN(BIAS) norm_forward<T, WIDE, BIAS><<<grid, block, 0, st>>>(form_of(n), static_cast<const T *>(x), ldx, static_cast<const T *>(y), ldy, static_cast<T *>(h), ldh, static_cast<T *>(z), ldz)
    if (n->b_after || n->b_before) RUN(true);
    else RUN(false);
#undef RUN
}

constexpr int kMostSums = 4;

template <typename T, bool WIDE>
void run_backward(const harp_norm *n, const harp_norm_grads *g, const Slabs &s, float *workspace, hipStream_t st) {
    const int threads = threads_for(n->cols);
    const bool bias = n->b_after || g->db_after || g->db_before;
    const bool sums = g->dw_after || g->db_after || g->dscale || g->dw_before || g->db_before;
    float *partial = sums ? workspace : nullptr;
    float *gate_partial = s.per_group && g->dgate ? workspace + s.count * kMostSums * n->cols : nullptr;
#define RUN(BIAS, GROUPS, MOST)                                                                                                     \
    norm_backward<T, WIDE, BIAS, GROUPS, MOST><<<dim3(uint32_t(s.count)), dim3(threads, teams), 0, st>>>(                                        \
        form_of(n), s, static_cast<const T *>(g->dh), g->lddh, static_cast<const T *>(g->dz), g->lddz, static_cast<const T *>(g->h), \
        g->ldh, static_cast<const T *>(g->y), g->ldy, static_cast<T *>(g->dx), g->lddx, static_cast<T *>(g->dy), g->lddy,            \
        static_cast<T *>(g->dgate), g->lddgate, partial, gate_partial)
    if (s.count > 0) {
        const bool groups = n->gate && s.per_group == 0;
        const int64_t units = groups ? s.rows / group_rows(n) : s.rows;
        // With 168 registers this one form keeps 50 values of a thread in memory (11,366 rows of 1,173, a gate a row: 237 us, 169 so).
        const bool fewer = sizeof(T) == 4 && bias && groups;
        int teams = teams_for(n->cols, fewer ? kFewThreads : kTeamThreads);
        if (teams > units) teams = int(units);
        const int all = threads * teams;
#define PICK(MOST)                           \
    if (bias && groups) RUN(true, true, MOST);   \
    else if (bias) RUN(true, false, MOST);       \
    else if (groups) RUN(false, true, MOST);     \
    else RUN(false, false, MOST)
        if (all <= kFewThreads) {
            PICK(kFewThreads);
        } else if (all <= kTeamThreads) {
            PICK(kTeamThreads);
        } else {
            PICK(kMaxThreads);
        }
#undef PICK
    }
#undef RUN
    const uint32_t across = uint32_t((n->cols + kJoinCols - 1) / kJoinCols);
    const Sums out = {g->dw_after, g->db_after, g->dscale, g->dw_before, g->db_before};
    // (slabs_for() splits so few groups that the grid is within its limits)
    const int64_t blocks = (sums ? across : 0) + (gate_partial ? s.count / s.per_group * gate_blocks(s.per_group, n->cols) : 0);
    if (blocks == 0) return;
    const Gates gates = {gate_partial, g->dgate, s.per_group, g->lddgate};
    const dim3 grid(static_cast<uint32_t>(blocks)), block(kJoinThreads);
    if (bias) norm_sums<T, true><<<grid, block, 0, st>>>(form_of(n), partial, s.count, out, g->accumulate, gates);
    else norm_sums<T, false><<<grid, block, 0, st>>>(form_of(n), partial, s.count, out, g->accumulate, gates);
}

size_t workspace_for(const harp_ctx *ctx, const harp_norm *n) {
    const Slabs s = slabs_for(ctx, n);
    return round_up(size_t(s.count) * (kMostSums + (n->gate && s.per_group ? 1 : 0)) * size_t(n->cols) * 4, 256) + 256;
}

}  // namespace

extern "C" {

int harp_norm_forward(harp_ctx *ctx, const harp_norm *n, const void *x, int64_t ldx, const void *y, int64_t ldy, void *h,
                      int64_t ldh, void *z, int64_t ldz, void *hip_stream) {
    int rc = check_norm(ctx, n);
    if (rc != HARP_OK) return rc;
    if (n->rows == 0) return HARP_OK;
    if (!x && !y) return fail(ctx, HARP_ERR_INVALID_ARG, "x and y are both null");
    if (n->before != HARP_NORM_NONE && !z) return fail(ctx, HARP_ERR_INVALID_ARG, "null z");
    if (n->before == HARP_NORM_NONE && (!y || !h)) return fail(ctx, HARP_ERR_INVALID_ARG, "without a norm before, y and h are needed");
    const Operand ops[] = {{x, ldx, "x"}, {y, ldy, "y"}, {y ? h : nullptr, ldh, "h"}, {n->before ? z : nullptr, ldz, "z"},
                           {y ? n->gate : nullptr, n->ldgate, "gate"}};
    bool wide;
    rc = check_operands(ctx, n, ops, 5, wide);
    if (rc != HARP_OK) return rc;
    hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
#define RUN(T) (wide ? run_forward<T, true>(ctx, n, x, ldx, y, ldy, h, ldh, z, ldz, st) : run_forward<T, false>(ctx, n, x, ldx, y, ldy, h, ldh, z, ldz, st))
    if (n->type == HARP_F32) RUN(float);
    else if (n->type == HARP_BF16) RUN(__bf16);
    else RUN(_Float16);
#undef RUN
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(ctx, e, "launching the norm kernel");
    return HARP_OK;
}

size_t harp_norm_workspace_bytes(harp_ctx *ctx, const harp_norm *n) {
    return check_norm(ctx, n) == HARP_OK ? workspace_for(ctx, n) : 0;
}

int harp_norm_backward(harp_ctx *ctx, const harp_norm *n, const harp_norm_grads *g, void *workspace, size_t workspace_bytes,
                       void *hip_stream) {
    int rc = check_norm(ctx, n);
    if (rc != HARP_OK) return rc;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null grads");
    if (n->rows > 0) {
        if (!g->dh && !g->dz) return fail(ctx, HARP_ERR_INVALID_ARG, "dh and dz are both null");
        if (g->dz && (!g->h || n->before == HARP_NORM_NONE)) return fail(ctx, HARP_ERR_INVALID_ARG, "dz needs h and a norm before");
    }
    if (!g->y && n->rows > 0 && (g->dy || g->dgate || g->dw_after || g->db_after || g->dscale))
        return fail(ctx, HARP_ERR_INVALID_ARG, "these gradients need y");
    if (g->dgate && !n->gate) return fail(ctx, HARP_ERR_INVALID_ARG, "dgate without a gate");
    const Operand ops[] = {{g->dh, g->lddh, "dh"}, {g->dz, g->lddz, "dz"}, {g->dz ? g->h : nullptr, g->ldh, "h"}, {g->y, g->ldy, "y"},
                           {g->dx, g->lddx, "dx"}, {g->dy, g->lddy, "dy"}, {g->dgate, g->lddgate, "dgate"},
                           {g->y ? n->gate : nullptr, n->ldgate, "gate"}};
    bool wide;
    rc = check_operands(ctx, n, ops, 8, wide);
    if (rc != HARP_OK) return rc;
    if (!aligned(g->dw_after, 4) || !aligned(g->db_after, 4) || !aligned(g->dw_before, 4) || !aligned(g->db_before, 4) || !aligned(g->dscale, 4))
        return fail(ctx, HARP_ERR_INVALID_ARG, "a sum is not aligned to its elements");
    const size_t need = workspace_for(ctx, n);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
        return fail(ctx, HARP_ERR_WORKSPACE, "the workspace needs %zu bytes, aligned to 256", need);
    hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    const Slabs s = slabs_for(ctx, n);
    float *p = static_cast<float *>(workspace);
#define RUN(T) (wide ? run_backward<T, true>(n, g, s, p, st) : run_backward<T, false>(n, g, s, p, st))
    if (n->type == HARP_F32) RUN(float);
    else if (n->type == HARP_BF16) RUN(__bf16);
    else RUN(_Float16);
#undef RUN
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(ctx, e, "launching the norm's backward kernels");
    return HARP_OK;
}

}  // extern "C"
