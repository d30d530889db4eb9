// The tiled matrix product that harp_linear and harp_gated share: its tiles, its main loop, its epilogues, and the form for few tokens.
#pragma once

#include <math.h>

#include <type_traits>

#include "harp_ctx.h"
#include "ops_common.h"

namespace {

using namespace harp;
using namespace harp::ops;

template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
    typedef bf16x8 Frag;
    static __device__ __forceinline__ f32x4 run(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<_Float16> {
    typedef f16x8 Frag;
    static __device__ __forceinline__ f32x4 run(Frag a, Frag b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// x / (1 + exp(-x)) and the like by way of the logistic function: a quotient of hardware reciprocal and exponential.
// Every form keeps its relative accuracy where the result is small: (1 + erf(u)) / 2 is taken as erfc(-u) / 2, whose two parts
// do not cancel below zero (1 + erff(u) is 4% off at z = -5 and 0 at z = -6).  What is left is the rounding of the
// exponential's and erfc's arguments, up to z^2 units of 2^-24 of the result and a few more for the tanh form's cube:
// under 2^-14 of it down to z = -8, where results of 16 bits are rounded to 2^-8 or 2^-11.
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
constexpr float kTanhA = 1.5957691216057308f;             // 2 sqrt(2 / pi): (1 + tanh(u)) / 2 = logistic(2 u)
constexpr float kTanhB = 0.044715f;

__device__ __forceinline__ float activate(float z, int act) {
    switch (act) {
        case HARP_ACT_RELU: return z > 0 ? z : z != z ? z : 0.0f;
        case HARP_ACT_GELU: return 0.5f * z * erfcf(z * -0.70710678f);
        case HARP_ACT_GELU_TANH: return z * logistic(kTanhA * z * (1.0f + kTanhB * z * z));
        case HARP_ACT_SILU: return z * logistic(z);
        default: return z;
    }
}
__device__ __forceinline__ float slope(float z, int act) {
    switch (act) {
        case HARP_ACT_RELU: return z > 0 ? 1.0f : 0.0f;
        case HARP_ACT_GELU: return 0.5f * erfcf(z * -0.70710678f) + z * 0.39894228f * __expf(-0.5f * z * z);
        case HARP_ACT_GELU_TANH: {
            // beyond 16 it is 1 or 0 in 32 bits; a z z without end would make NaN of the zero s (1 - s)
            const float square = fminf(z * z, 256.0f), s = logistic(kTanhA * z * (1.0f + kTanhB * square));
            return s + z * s * (1.0f - s) * kTanhA * (1.0f + 3.0f * kTanhB * square);
        }
        case HARP_ACT_SILU: {
            const float s = logistic(z);
            return s * (1.0f + z * (1.0f - s));
        }
        default: return 1.0f;
    }
}

// What becomes of D[p][q].
enum { kForward, kInput, kWeight };
struct Epilogue {
    int kind, act, accumulate, out_f32;
    int past;                        // results are stored past the caches
    void *out;
    const void *bias, *residual;     // residual: [p][q]
    const void *slope_at;            // kInput: Z
    void *keep;                      // kForward: Z
    int64_t ldo, ldr, ldz;
};
template <typename T> __device__ __forceinline__ void finish(const Epilogue &e, int64_t p, int64_t q, float d) {
    if (e.kind == kForward) {
        if (e.bias) d += to_f32(static_cast<const T *>(e.bias)[q]);
        if (e.keep) static_cast<T *>(e.keep)[p * e.ldz + q] = T(d);
        d = activate(d, e.act);
    } else if (e.kind == kInput && e.act != HARP_ACT_NONE) {
        d *= slope(to_f32(static_cast<const T *>(e.slope_at)[p * e.ldz + q]), e.act);
    }
    if (e.residual) d += to_f32(static_cast<const T *>(e.residual)[p * e.ldr + q]);
    if (e.out_f32) {
        float *o = static_cast<float *>(e.out) + p * e.ldo + q;
        *o = e.accumulate ? *o + d : d;
    } else {
        T *o = static_cast<T *>(e.out) + p * e.ldo + q;
        *o = T(e.accumulate ? to_f32(*o) + d : d);
    }
}

// The same for q .. q + 3.
template <typename T> __device__ __forceinline__ void finish4(const Epilogue &e, int64_t p, int64_t q, int64_t Q, f32x4 d) {
    if (q + 4 > Q) {
#pragma unroll 1
        for (int k = 0; k < 4 && q < Q; ++k, ++q) {
            finish<T>(e, p, q, d.x);
            d = f32x4{d.y, d.z, d.w, 0};
        }
        return;
    }
    if (e.kind == kForward) {
        if (e.bias) d += load4(static_cast<const T *>(e.bias) + q);
        if (e.keep) store4(static_cast<T *>(e.keep) + p * e.ldz + q, d, e.past);
        for (int k = 0; k < 4; ++k) d[k] = activate(d[k], e.act);
    } else if (e.kind == kInput && e.act != HARP_ACT_NONE) {
        const f32x4 z = load4(static_cast<const T *>(e.slope_at) + p * e.ldz + q);
        for (int k = 0; k < 4; ++k) d[k] *= slope(z[k], e.act);
    }
    if (e.residual) d += load4(static_cast<const T *>(e.residual) + p * e.ldr + q);
    if (e.out_f32) {
        float *o = static_cast<float *>(e.out) + p * e.ldo + q;
        store4(o, e.accumulate ? d + load4(o) : d, e.past);
    } else {
        T *o = static_cast<T *>(e.out) + p * e.ldo + q;
        store4(o, e.accumulate ? d + load4(o) : d, e.past);
    }
}

// What becomes of the gated block's products.  Forward: of gate and up, the two halves of Z, both in one workgroup's tile.  Back:
// of D = dH.  Either way for columns q .. q + 3 of F.
enum { kLinear, kGatedForward, kGatedBack };       // the form of a product
struct Gated {
    int act, past;
    int64_t F, ldh, ldz, lddz;
    const void *bias;
    void *h;                         // H, may be absent on the way back
    void *z;                         // forward: receives Z, or absent; back: Z
    void *dz;
};
template <typename T> __device__ __forceinline__ void gated1(const Gated &e, int64_t p, int64_t q, float gate, float up) {
    if (e.bias) gate += to_f32(static_cast<const T *>(e.bias)[q]), up += to_f32(static_cast<const T *>(e.bias)[e.F + q]);
    if (e.z) {
        T *z = static_cast<T *>(e.z) + p * e.ldz + q;
        z[0] = T(gate);
        z[e.F] = T(up);
    }
    static_cast<T *>(e.h)[p * e.ldh + q] = T(activate(gate, e.act) * up);
}
template <typename T> __device__ __forceinline__ void gated_back1(const Gated &e, int64_t p, int64_t q, float d) {
    const T *z = static_cast<const T *>(e.z) + p * e.ldz + q;
    const float gate = to_f32(z[0]), up = to_f32(z[e.F]), a = activate(gate, e.act);
    T *dz = static_cast<T *>(e.dz) + p * e.lddz + q;
    dz[0] = T(d * up * slope(gate, e.act));
    dz[e.F] = T(d * a);
    if (e.h) static_cast<T *>(e.h)[p * e.ldh + q] = T(a * up);
}
template <typename T> __device__ __forceinline__ void gated4(const Gated &e, int64_t p, int64_t q, f32x4 gate, f32x4 up, int act) {
    if (q + 4 > e.F) {
#pragma unroll 1
        for (; q < e.F; ++q) {
            gated1<T>(e, p, q, gate.x, up.x);
            gate = f32x4{gate.y, gate.z, gate.w, 0};
            up = f32x4{up.y, up.z, up.w, 0};
        }
        return;
    }
    if (e.bias) gate += load4(static_cast<const T *>(e.bias) + q), up += load4(static_cast<const T *>(e.bias) + e.F + q);
    if (e.z) {
        T *z = static_cast<T *>(e.z) + p * e.ldz + q;
        store4(z, gate, e.past);
        store4(z + e.F, up, e.past);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) gate[k] = activate(gate[k], act) * up[k];
    store4(static_cast<T *>(e.h) + p * e.ldh + q, gate, e.past);
}
// With Z's columns as they have been read.
template <typename T> __device__ __forceinline__ void gated_back4(const Gated &e, int64_t p, int64_t q, f32x4 d, f32x4 gate, f32x4 up, int act) {
    f32x4 dgate, dup, h;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float a = activate(gate[k], act);
        dgate[k] = d[k] * up[k] * slope(gate[k], act);
        dup[k] = d[k] * a;
        h[k] = a * up[k];
    }
    T *dz = static_cast<T *>(e.dz) + p * e.lddz + q;
    store4(dz, dgate, e.past);
    store4(dz + e.F, dup, e.past);
    if (e.h) store4(static_cast<T *>(e.h) + p * e.ldh + q, h, e.past);
}
template <typename T> __device__ __forceinline__ void gated_back(const Gated &e, int64_t p, int64_t q, f32x4 d, int act) {
    if (q + 4 <= e.F) {
        const T *z = static_cast<const T *>(e.z) + p * e.ldz + q;
        gated_back4<T>(e, p, q, d, load4(z), load4(z + e.F), act);
        return;
    }
#pragma unroll 1
    for (; q < e.F; ++q) {
        gated_back1<T>(e, p, q, d.x);
        d = f32x4{d.y, d.z, d.w, 0};
    }
}

// Shares of r that several workgroups summed up apart, in their order, and the epilogue.
template <typename T>
__global__ __launch_bounds__(256) void join(const float *partial, int shares, int64_t P, int64_t Q, Epilogue e) {
    const int64_t across = (Q + 3) / 4;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < P * across; i += int64_t(gridDim.x) * 256) {
        const int64_t p = i / across, q = i % across * 4;
        f32x4 d = {0, 0, 0, 0};
        if (q + 4 <= Q) {
#pragma unroll 4
            for (int s = 0; s < shares; ++s) d += load4(partial + (s * P + p) * Q + q);
        } else {
            for (int s = 0; s < shares; ++s)
                for (int k = 0; k < 4; ++k)
                    if (q + k < Q) d[k] += partial[(s * P + p) * Q + q + k];
        }
        finish4<T>(e, p, q, Q, d);
    }
}

// Rows of `cols` elements anywhere, to rows of a multiple of 8 that begin at multiples of 16 bytes and end with zeros.
template <typename T>
__global__ __launch_bounds__(256) void pack(const T *from, int64_t ld, int64_t rows, int64_t cols, T *to, int64_t ldto) {
    const int64_t across = ldto / 8;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < rows * across; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / across, c = i % across * 8;
        typedef typename Mfma<T>::Frag Loose __attribute__((aligned(sizeof(T))));
        typename Mfma<T>::Frag v = {};
        if (c + 8 <= cols) {
            v = *reinterpret_cast<const Loose *>(from + row * ld + c);
        } else {
            for (int k = 0; k < 8; ++k)
                if (c + k < cols) v[k] = from[row * ld + c + k];
        }
        *reinterpret_cast<typename Mfma<T>::Frag *>(to + row * ldto + c) = v;
    }
}

// ---------------------------------------------------------------------------------------------- tiles
// A workgroup makes a tile of BP x BQ of D, 32 of r at a time.  Both operands go from memory straight into LDS, three or four
// steps before they are multiplied (five buffers, all of LDS for tiles of 256 x 256).  Two steps are sent for at once: where r
// is contiguous they are the two halves of lines of 128 bytes.
//
// LDS holds pieces of 16 bytes.  Where r is contiguous in memory a row of the tile is 4 pieces of 8 r, piece c of row
// `row` at place c ^ (row / 2 & 3): the 8 rows that a wavefront reads at once then lie in 8 different places of 128 bytes.
// Where p or q is contiguous a row is one r with B / 8 pieces of 8 p, moved by swap(r); four rows of 16 p are transposed
// by the read.
constexpr int kDeep = 32;

__device__ __forceinline__ int swap_of(int r) { return (r & 3) << 1 | (r >> 3 & 1) << 3; }

// 16 bytes a lane, from base + off to LDS, lane after lane from `to` on (the same for the wavefront).  Written out, because
// the compiler waits for every such load before any read of LDS that it cannot tell from the load's target; here the waits
// are the kernel's own (vmcnt counts these loads).  There is no result register, and addresses are taken at issue.  m0 is
// named as written so that the compiler keeps no value of its own there across the statement; that it hands m0 out to nobody
// is what its warning, turned off here, is about.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(off), "s"(base) : "memory", "m0");
}
#pragma clang diagnostic pop
template <typename T> __device__ __forceinline__ uint32_t lds_address(const T *p) {
    return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void *)p));
}

// One operand of a workgroup of THREADS threads: ACROSS: p is contiguous, else r.
template <typename T, bool ACROSS, int B, int THREADS> struct Side {
    static constexpr int kLoads = B * kDeep * 2 / 16 / THREADS;      // pieces a thread brings
    static constexpr int kRow = ACROSS ? B / 8 : kDeep / 8;          // pieces in a row of LDS
    const char *base;                                                // the tile's r0, the same for all threads
    int64_t step;
    uint32_t off[kLoads];                                            // bytes; a tile spans less than 2^31 (kMostCols)

    // LDS address of the first of the pieces that this wavefront brings with its load i
    __device__ __forceinline__ static uint32_t target(const T *lds, int i) {
        return lds_address(lds) + uint32_t(i * THREADS + __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave) * kWave) * 16;
    }
    __device__ __forceinline__ static int place(int i) { return i * THREADS + int(threadIdx.x); }
    // r (relative to the tile) of piece i of this thread
    __device__ __forceinline__ static int depth(int i) {
        const int id = place(i);
        return ACROSS ? id / kRow : ((id % kRow) ^ (id / kRow / 2 & 3)) * 8;
    }
    // HALF: the tile's rows are runs of HALF rows of one matrix and HALF of another by turns, `a` being that of this wavefront's.
    template <int HALF = 0> __device__ __forceinline__ void begin(const T *a, int64_t ld, int64_t p0, int64_t P, int64_t r0) {
        static_assert(HALF == 0 || (!ACROSS && HALF % (kWave / kRow) == 0), "a wavefront's pieces have to be of one matrix");
        step = (ACROSS ? kDeep * ld : kDeep) * int64_t(sizeof(T));
        base = reinterpret_cast<const char *>(ACROSS ? a + r0 * ld + p0 : a + p0 * ld + r0);
        // beyond the edge: anything that is there
        const int last = int(ACROSS ? (P + 7) / 8 * 8 - 8 - p0 : P - 1 - p0);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int id = place(i), row = id / kRow;
            const int p = ACROSS ? ((id % kRow) ^ swap_of(row)) * 8 : HALF ? row / (2 * (HALF ? HALF : 1)) * HALF + row % (HALF ? HALF : 1) : row;
            const int at = p < last ? p : last;
            off[i] = uint32_t(ACROSS ? depth(i) * ld + at : at * ld + depth(i)) * uint32_t(sizeof(T));
        }
    }
    // The next step, or the next two: one after the other, each piece's two halves of a line together.
    __device__ __forceinline__ void load(T *lds) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) load_to_lds(base, off[i], target(lds, i));
        base += step;
    }
    __device__ __forceinline__ void load_two(T *lds, T *after) {
        const char *next = base + step;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            load_to_lds(base, off[i], target(lds, i));
            load_to_lds(next, off[i], target(after, i));
        }
        base = next + step;
    }
    // The last, partial step of `left` r: what is beyond is read from the last r there are, and made zeros by clear() when
    // it has arrived.  Rows of r that are not a multiple of 8 long have zeros up to there.
    __device__ __forceinline__ int beyond(int i, int left) const { return depth(i) - (ACROSS ? left - 1 : (left + 7) / 8 * 8 - 8); }
    __device__ __forceinline__ void load_partial(T *lds, int left) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int n = beyond(i, left);
            const uint32_t back = n > 0 ? uint32_t(ACROSS ? n * (step / kDeep) : n * int64_t(sizeof(T))) : 0;
            load_to_lds(base, off[i] - back, target(lds, i));
        }
    }
    __device__ __forceinline__ void clear(T *lds, int left) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            if (beyond(i, left) > 0) *reinterpret_cast<u32x4 *>(lds + place(i) * 8) = u32x4{0, 0, 0, 0};
    }
};

// Fragments of 16 p by 32 r of a tile in LDS: lane l has p = l % 16 and r = 8 (l / 16) .. + 7 of the 32.
template <typename T, bool ACROSS, int B, int COUNT> struct Fragments {
    typedef typename Mfma<T>::Frag Frag;
    int at[ACROSS ? COUNT : 1];
    __device__ __forceinline__ void begin(int p0) {
        const int lane = threadIdx.x % kWave, i = lane % 16, g = lane / 16;
        if constexpr (ACROSS) {
            const int r = 8 * g + i / 4;
#pragma unroll
            for (int j = 0; j < COUNT; ++j) at[j] = r * B + (((p0 / 8 + 2 * j) ^ swap_of(r)) | (i % 4 / 2)) * 8 + i % 2 * 4;
        } else {
            at[0] = (p0 + i) * kDeep + (g ^ (i / 2 & 3)) * 8;
        }
    }
    __device__ __forceinline__ Frag read(const T *lds, int j) const {
        if constexpr (ACROSS) {
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            typedef short s16x8 __attribute__((ext_vector_type(8)));
            typedef __attribute__((address_space(3))) s16x4 *Lds;
            const T *a = lds + at[j];
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)a);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(a + 4 * B));
            const s16x8 v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(Frag, v);
        } else {
            return *reinterpret_cast<const Frag *>(lds + at[0] + 16 * j * kDeep);
        }
    }
};

// Which tile a workgroup takes.  Workgroups go to the 8 dies in turn, each with an L2 of its own: a die takes tiles that
// are neighbours, in columns of kGroup tiles, so that what they share is read into one L2.
constexpr int kDies = 8, kGroup = 8;
__device__ __forceinline__ void tile_of(int id, int tiles_p, int tiles_q, int &tp, int &tq) {
    const int n = tiles_p * tiles_q, die = id % kDies, each = n / kDies, more = n % kDies;
    id = id / kDies + die * each + (die < more ? die : more);
    const int wide = kGroup * tiles_q, first = id / wide * kGroup;
    const int high = tiles_p - first < kGroup ? tiles_p - first : kGroup;
    tp = first + id % wide % high;
    tq = id % wide / high;
}

// Measured: X [4096][4096], W [16384][4096], bfloat16, bias, tanh GELU, Z kept: 478 us, 1,150 TFLOP/s (a plain library product
// of these sizes reaches 1,517); the gradients of X [4096][16384], W [4096][16384] through GELU, weights' added to 32 bits:
// 1,021 us with the bias's, 1,080.  Matrix units are busy 51 to 61% of the cycles.  What bounds it: bringing the operands into
// LDS (20%: with the loads taken out of the loop the probe ran 376 us of 472) and the epilogue, in which every compute unit
// stores and reads at once while none multiplies (11%; its code, some 50 KB straight for one activation, is part of that, how
// much has not been told apart).  Tiles of 256 x 256 read each operand least; two workgroups a compute
// unit with 256 x 128, which would cover each other's epilogues, need half as much again from L2 and took 632 us of 433; four
// wavefronts of 128 x 128 each, which would read LDS a third less, 544: one to a SIMD, they wait at every barrier.
// WP x WQ wavefronts, each a part of BP / WP x BQ / WQ of the tile.  With `partial` the sums of blockIdx.y's share of r go
// there, [share][P][Q], instead of through the epilogue.
//
// FORM kGatedForward: half of each wavefront's columns are the gate's, rows q of b, half the same of what it is multiplied with,
// rows F + q, so that a lane has both of an element; Q is F, and a tile BQ / 2 of it.
template <typename T, bool A_ACROSS, bool B_ACROSS, int BP, int BQ, int WP, int WQ, int FORM = kLinear, typename E = Epilogue>
__global__ __launch_bounds__(WP * WQ * kWave) void product(const T *a, int64_t lda, const T *b, int64_t ldb, int64_t P, int64_t Q, int64_t R,
                                                           int tiles_p, int tiles_q, int64_t share, float *partial, E e) {
    constexpr int kThreads = WP * WQ * kWave, kP = BP / WP / 16, kQ = BQ / WQ / 16;
    constexpr bool kPairs = !(A_ACROSS && B_ACROSS);
    constexpr int kBuffers = kPairs ? 5 : 4;
    __shared__ __align__(16) T la[kBuffers][BP * kDeep];
    __shared__ __align__(16) T lb[kBuffers][BQ * kDeep];
    int tp, tq;
    tile_of(blockIdx.x, tiles_p, tiles_q, tp, tq);
    constexpr int kHalf = FORM == kGatedForward ? BQ / WQ / 2 : 0;
    const int64_t p0 = int64_t(tp) * BP, q0 = int64_t(tq) * (kHalf ? BQ / 2 : BQ);
    const int64_t r0 = int64_t(blockIdx.y) * share, r1 = r0 + share < R ? r0 + share : R;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int wp = wave / WQ * (BP / WP), wq = wave % WQ * (BQ / WQ);
    Side<T, A_ACROSS, BP, kThreads> sa;
    Side<T, B_ACROSS, BQ, kThreads> sb;
    sa.begin(a, lda, p0, P, r0);
    if constexpr (kHalf != 0) {
        const int first = __builtin_amdgcn_readfirstlane(int(threadIdx.x)) / decltype(sb)::kRow;       // row of the tile
        static_assert(kThreads / decltype(sb)::kRow % (2 * kHalf) == 0, "the same matrix with every load");
        sb.template begin<kHalf>(first / kHalf % 2 ? b + Q * ldb : b, ldb, q0, Q, r0);
    } else {
        sb.begin(b, ldb, q0, Q, r0);
    }
    Fragments<T, A_ACROSS, BP, kP> fa;
    Fragments<T, B_ACROSS, BQ, kQ> fb;
    fa.begin(wp);
    fb.begin(wq);
    f32x4 acc[kP][kQ] = {};
    typedef typename Mfma<T>::Frag Frag;
    const int steps = int((r1 - r0 + kDeep - 1) / kDeep), odd = int((r1 - r0) % kDeep);     // odd: r of a partial last step
    // An operand of a step, whole or not; of two steps where r is contiguous and they share lines.
    auto bring = [&](auto &side, auto *lds, int i) {
        if (i >= steps) return;
        if (i + 1 < steps || odd == 0) side.load(lds[i % kBuffers]);
        else side.load_partial(lds[i % kBuffers], odd);
    };
    auto bring_two = [&](auto &side, auto *lds, int i) {
        if (i + 2 < steps || (i + 2 == steps && odd == 0)) {
            side.load_two(lds[i % kBuffers], lds[(i + 1) % kBuffers]);
        } else {
            bring(side, lds, i);
            bring(side, lds, i + 1);
        }
    };
    auto barrier = [] {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // Step i is in LDS for everybody, and nobody reads the buffer of step i - 1 any more.  Loads into LDS are counted by
    // vmcnt, which a barrier alone does not wait for; they arrive in order, so what was sent for after step i may be out
    // still: of an operand that comes in pairs the next pair of steps, of the other kBuffers - 2 steps.  At the end there is
    // less, and the wait is for more than has to be.
    constexpr int kA = decltype(sa)::kLoads, kB = decltype(sb)::kLoads;
    constexpr int kOut = (kPairs && !A_ACROSS ? 2 : kBuffers - 2) * kA + (kPairs && !B_ACROSS ? 2 : kBuffers - 2) * kB;
    auto arrived = [&](int i) {
        if (i + kBuffers - 2 < steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kOut) : "memory");
        else if (i + 2 < steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kA + kB) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        if (i + 1 == steps && odd) {
            sa.clear(la[i % kBuffers], odd);
            sb.clear(lb[i % kBuffers], odd);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier();
    };
    auto read = [&](int buffer, Frag (&x)[kP], Frag (&y)[kQ]) {
#pragma unroll
        for (int j = 0; j < kQ; ++j) y[j] = fb.read(lb[buffer], j);
#pragma unroll
        for (int i = 0; i < kP; ++i) x[i] = fa.read(la[buffer], i);
    };
    // A step's products from registers.  The q operand first: a lane then holds four neighbouring q of one p.
    auto multiply = [&](const Frag (&x)[kP], const Frag (&y)[kQ]) {
#pragma unroll
        for (int i = 0; i < kP; ++i)
#pragma unroll
            for (int j = 0; j < kQ; ++j) acc[i][j] = Mfma<T>::run(y[j], x[i], acc[i][j]);
    };
    // ... while the reads of the next step's operands go on among the instructions.
    auto interleave = [] {
        constexpr int kReads = kP * (A_ACROSS ? 2 : 1) + kQ * (B_ACROSS ? 2 : 1), kEach = kP * kQ / kReads;
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);       // matrix instructions
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);           // LDS read
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kP * kQ - kReads * kEach, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    Frag x[2][kP], y[2][kQ];
    if (steps > 0) {
        // First what steps 0 and 1 need, then the rest that the buffers hold, in an order in which no step's loads lie among
        // the last kOut when it is waited for.
        static_assert(!A_ACROSS || B_ACROSS, "only the second operand comes in pairs: the order would have to be another");
        if (kPairs && !A_ACROSS) bring_two(sa, la, 0);
        else { bring(sa, la, 0); bring(sa, la, 1); }
        if (kPairs && !B_ACROSS) bring_two(sb, lb, 0);
        else { bring(sb, lb, 0); bring(sb, lb, 1); }
        if (kPairs) bring_two(sa, la, 2);
        if (kPairs && !B_ACROSS) bring_two(sb, lb, 2);
        for (int i = 2; i < kBuffers; ++i) {
            if (!kPairs) bring(sa, la, i);
            if (!kPairs || B_ACROSS) bring(sb, lb, i);
        }
        if (steps >= kBuffers + 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kOut) : "memory");
        else arrived(steps - 1);                         // few steps: all of them
        barrier();
        read(0, x[0], y[0]);
        // Step i has its operands in registers.  Behind its barrier step i + 1 has arrived, and the buffers of step i and of
        // the one before are free: for step i + kBuffers, and for pairs every other time, for steps i + 4 and i + 5.  A round
        // of steps at a time while all that they bring is whole: buffers are known then.
        constexpr int kRound = kBuffers % 2 ? 2 * kBuffers : kBuffers;
        int i = 0;
        for (; i + kRound + kBuffers < steps; i += kRound) {
#pragma unroll
            for (int k = 0; k < kRound; ++k) {
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kOut) : "memory");
                barrier();
                if (!(kPairs && !A_ACROSS)) sa.load(la[k % kBuffers]);
                else if (k % 2 == 0) sa.load_two(la[(k + 4) % kBuffers], la[k % kBuffers]);
                if (!(kPairs && !B_ACROSS)) sb.load(lb[k % kBuffers]);
                else if (k % 2 == 0) sb.load_two(lb[(k + 4) % kBuffers], lb[k % kBuffers]);
                __builtin_amdgcn_sched_barrier(0);
                read((k + 1) % kBuffers, x[(k + 1) % 2], y[(k + 1) % 2]);
                multiply(x[k % 2], y[k % 2]);
                interleave();
            }
        }
        for (; i + 1 < steps; ++i) {
            arrived(i + 1);
            if (!(kPairs && !A_ACROSS)) bring(sa, la, i + kBuffers);
            else if (i % 2 == 0) bring_two(sa, la, i + 4);
            if (!(kPairs && !B_ACROSS)) bring(sb, lb, i + kBuffers);
            else if (i % 2 == 0) bring_two(sb, lb, i + 4);
            read((i + 1) % kBuffers, x[1], y[1]);
            multiply(x[0], y[0]);
#pragma unroll
            for (int k = 0; k < kP; ++k) x[0][k] = x[1][k];
#pragma unroll
            for (int k = 0; k < kQ; ++k) y[0][k] = y[1][k];
        }
        multiply(x[0], y[0]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        barrier();                                       // all have read all: LDS is free
    }
    // 16 p at a time through LDS (the tiles are done with): a lane then holds four q of a row whose other q its neighbours
    // hold, and rows are stored in whole lines.  What the epilogue reads of the next 16 p is asked for before the current
    // ones are worked on (4,096 x 16,384 x 4,096 forward with bias, tanh GELU and Z kept 515 us without, 497 so); not of a
    // weight gradient to add to, where reads and writes of 32 bits contend for memory (508 us without, 540 so).
    if constexpr (FORM == kLinear)
        if (partial) e = Epilogue{kWeight, HARP_ACT_NONE, 0, 1, 0, partial + int64_t(blockIdx.y) * P * Q, nullptr, nullptr, nullptr, nullptr, Q, 0, 0};
    constexpr int kCols = BQ / WQ, kPitch = kCols + 4, kLanes = (kHalf ? kHalf : kCols) / 4, kRows = kWave / kLanes, kParts = 16 / kRows;
    static_assert(WP * WQ * 16 * kPitch * 4 <= kBuffers * BP * kDeep * 2, "the wavefronts' rows have to fit into the first operand's LDS");
    float *rows = reinterpret_cast<float *>(&la[0][0]) + wave * 16 * kPitch;
    const int64_t q = q0 + (kHalf ? wq / 2 : wq) + lane % kLanes * 4;
    auto row_of = [&](int i, int k) { return p0 + wp + 16 * i + k * kRows + lane / kLanes; };
    auto through_lds = [&](int i) {
#pragma unroll
        for (int j = 0; j < kQ; ++j) *reinterpret_cast<f32x4 *>(rows + lane % 16 * kPitch + 16 * j + lane / 16 * 4) = acc[i][j];
        __builtin_amdgcn_wave_barrier();
    };
    auto from_lds = [&](int k, int col = 0) {
        return *reinterpret_cast<const f32x4 *>(rows + (k * kRows + lane / kLanes) * kPitch + lane % kLanes * 4 + col);
    };
    auto for_act = [&](auto call) {                      // an activation known when compiled
        if (e.act == HARP_ACT_NONE) call(std::integral_constant<int, HARP_ACT_NONE>());
        else if (e.act == HARP_ACT_RELU) call(std::integral_constant<int, HARP_ACT_RELU>());
        else if (e.act == HARP_ACT_GELU) call(std::integral_constant<int, HARP_ACT_GELU>());
        else if (e.act == HARP_ACT_GELU_TANH) call(std::integral_constant<int, HARP_ACT_GELU_TANH>());
        else call(std::integral_constant<int, HARP_ACT_SILU>());
    };
    if constexpr (FORM == kGatedForward) {
        const bool ragged = q0 + BQ / 2 > Q && Q % 4 != 0;
        auto rows_of = [&](auto act) {
#pragma unroll
            for (int i = 0; i < kP; ++i) {
                through_lds(i);
#pragma unroll
                for (int k = 0; k < kParts; ++k)
                    if (row_of(i, k) < P && q + 4 <= Q) gated4<T>(e, row_of(i, k), q, from_lds(k), from_lds(k, kHalf), act);
                __builtin_amdgcn_wave_barrier();
            }
        };
        if (!ragged) {
            for_act(rows_of);
        } else {
#pragma unroll
            for (int i = 0; i < kP; ++i) {
                through_lds(i);
#pragma unroll 1
                for (int k = 0; k < kParts; ++k)
                    if (row_of(i, k) < P && q < Q) gated4<T>(e, row_of(i, k), q, from_lds(k), from_lds(k, kHalf), e.act);
                __builtin_amdgcn_wave_barrier();
            }
        }
    } else if constexpr (FORM == kGatedBack) {
        auto rows_of = [&](auto act) {
            f32x4 gate[2][kParts], up[2][kParts];
            auto ask = [&](int i) {
#pragma unroll
                for (int k = 0; k < kParts; ++k) {
                    if (row_of(i, k) >= P || q >= Q) continue;
                    const T *z = static_cast<const T *>(e.z) + row_of(i, k) * e.ldz + q;
                    gate[i % 2][k] = load4(z);
                    up[i % 2][k] = load4(z + e.F);
                }
            };
            ask(0);
#pragma unroll
            for (int i = 0; i < kP; ++i) {
                if (i + 1 < kP) ask(i + 1);
                through_lds(i);
#pragma unroll
                for (int k = 0; k < kParts; ++k)
                    if (row_of(i, k) < P && q < Q) gated_back4<T>(e, row_of(i, k), q, from_lds(k), gate[i % 2][k], up[i % 2][k], act);
                __builtin_amdgcn_wave_barrier();
            }
        };
        if (q0 + BQ <= Q || Q % 4 == 0) {
            for_act(rows_of);
        } else {
#pragma unroll
            for (int i = 0; i < kP; ++i) {
                through_lds(i);
#pragma unroll 1
                for (int k = 0; k < kParts; ++k)
                    if (row_of(i, k) < P && q < Q) gated_back<T>(e, row_of(i, k), q, from_lds(k), e.act);
                __builtin_amdgcn_wave_barrier();
            }
        }
    } else {
    auto wide_rows_of = [&](auto act) {
        f32x4 bias = {0, 0, 0, 0}, z[2][kParts], more[2][kParts];
        if (e.bias && q < Q) bias = load4(static_cast<const T *>(e.bias) + q);
        auto ask = [&](int i) {
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
                const int64_t p = row_of(i, k);
                if (p >= P || q >= Q) continue;
                if (act != HARP_ACT_NONE && e.kind == kInput) z[i % 2][k] = load4(static_cast<const T *>(e.slope_at) + p * e.ldz + q);
                if (e.residual) more[i % 2][k] = load4(static_cast<const T *>(e.residual) + p * e.ldr + q);
            }
        };
        ask(0);
#pragma unroll
        for (int i = 0; i < kP; ++i) {
            if (i + 1 < kP) ask(i + 1);
            through_lds(i);
#pragma unroll
            for (int k = 0; k < kParts; ++k) {
                const int64_t p = row_of(i, k);
                if (p >= P || q >= Q) continue;
                f32x4 d = from_lds(k) + bias;
                if (e.kind == kForward) {
                    if (e.keep) store4(static_cast<T *>(e.keep) + p * e.ldz + q, d, e.past);
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] = activate(d[j], act);
                } else if (act != HARP_ACT_NONE) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) d[j] *= slope(z[i % 2][k][j], act);
                }
                if (e.residual) d += more[i % 2][k];
                if (e.out_f32) store4(static_cast<float *>(e.out) + p * e.ldo + q, d, e.past);
                else store4(static_cast<T *>(e.out) + p * e.ldo + q, d, e.past);
            }
            __builtin_amdgcn_wave_barrier();
        }
    };
    if (A_ACROSS || (q0 + BQ > Q && Q % 4 != 0)) {       // some lane's four q are not all there
#pragma unroll
        for (int i = 0; i < kP; ++i) {
            through_lds(i);
#pragma unroll 1
            for (int k = 0; k < kParts; ++k)
                if (row_of(i, k) < P && q < Q) finish4<T>(e, row_of(i, k), q, Q, from_lds(k));
            __builtin_amdgcn_wave_barrier();
        }
    } else if (e.act == HARP_ACT_NONE) {
        wide_rows_of(std::integral_constant<int, HARP_ACT_NONE>());
    } else if (e.act == HARP_ACT_RELU) {
        wide_rows_of(std::integral_constant<int, HARP_ACT_RELU>());
    } else if (e.act == HARP_ACT_GELU) {
        wide_rows_of(std::integral_constant<int, HARP_ACT_GELU>());
    } else if (e.act == HARP_ACT_GELU_TANH) {
        wide_rows_of(std::integral_constant<int, HARP_ACT_GELU_TANH>());
    } else {
        wide_rows_of(std::integral_constant<int, HARP_ACT_SILU>());
    }
    }
}

// ---------------------------------------------------------------------------------------------- few tokens
// Y of at most 16 TILES tokens: the weights are read once, straight into registers, and bound it.  A workgroup makes 16
// outputs of all tokens; its four wavefronts take 64 of r in turn and are joined at the end.  In a piece of 64 r lane l
// has row l % 16 and the 16 r from 16 (l / 16) on, 32 bytes of a row, so that four lanes read whole lines; the same r of
// the tokens meet them, whatever their order.  One token through W [16384][4096] with bias and GELU: 29.7 us, 4.5 TB/s (a copy
// reaches 4.9).
constexpr int kFewWaves = 4;
template <typename T, bool WIDE> __device__ __forceinline__ typename Mfma<T>::Frag eight(const T *row, int64_t r, int64_t R) {
    typename Mfma<T>::Frag v = {};
    if (WIDE) {
        if (r < R) v = *reinterpret_cast<const typename Mfma<T>::Frag *>(row + r);
    } else if (r + 8 <= R) {
        typedef typename Mfma<T>::Frag Loose __attribute__((aligned(sizeof(T))));       // where it lies
        v = *reinterpret_cast<const Loose *>(row + r);
    } else {
        for (int k = 0; k < 8; ++k)
            if (r + k < R) v[k] = row[r + k];
    }
    return v;
}
// FORM kGatedForward: of 16 outputs both the gate's rows and those F further on, half as many pieces of each on their way.
template <typename T, bool WIDE, int TILES, int FORM = kLinear, typename E = Epilogue>
__global__ __launch_bounds__(kFewWaves * kWave) void few_tokens(const T *x, int64_t ldx, const T *w, int64_t ldw, int64_t M, int64_t N, int64_t R,
                                                                int64_t share, float *partial, E e) {
    constexpr int kSides = FORM == kGatedForward ? 2 : 1;
    __shared__ float sums[kSides][kFewWaves][TILES * 16][17];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, i = lane % 16, g = lane / 16;
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    const int64_t r0 = int64_t(blockIdx.y) * share, r1 = r0 + share < R ? r0 + share : R;
    const T *wr[kSides];
#pragma unroll
    for (int d = 0; d < kSides; ++d) wr[d] = w + ((n0 + i < N ? n0 + i : N - 1) + d * N) * ldw;
    const T *xr[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) xr[t] = x + (16 * t + i < M ? 16 * t + i : M - 1) * ldx;
    f32x4 acc[kSides][TILES] = {};
    // several pieces are asked for before the first is used: a compute unit then has 128 KB of weights on their way
    constexpr int kAhead = (TILES == 1 ? 4 : 2) / kSides;
    for (int64_t r = r0 + wave * 64 + 16 * g; r - 16 * g < r1; r += kAhead * kFewWaves * 64) {
        typename Mfma<T>::Frag a[kSides][kAhead][2], b[TILES][kAhead][2];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int d = 0; d < kSides; ++d)
#pragma unroll
                for (int h = 0; h < 2; ++h) a[d][k][h] = eight<T, WIDE>(wr[d], r + k * kFewWaves * 64 + 8 * h, r1);
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int h = 0; h < 2; ++h) b[t][k][h] = eight<T, WIDE>(xr[t], r + k * kFewWaves * 64 + 8 * h, r1);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int t = 0; t < TILES; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int d = 0; d < kSides; ++d) acc[d][t] = Mfma<T>::run(a[d][k][h], b[t][k][h], acc[d][t]);
    }
#pragma unroll
    for (int d = 0; d < kSides; ++d)
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int k = 0; k < 4; ++k) sums[d][wave][16 * t + i][4 * g + k] = acc[d][t][k];
    __syncthreads();
    for (int at = threadIdx.x; at < TILES * 256; at += kFewWaves * kWave) {
        const int m = at / 16, n = at % 16;
        float d[kSides] = {};
#pragma unroll
        for (int side = 0; side < kSides; ++side)
            for (int v = 0; v < kFewWaves; ++v) d[side] += sums[side][v][m][n];
        if (m >= M || n0 + n >= N) continue;
        if constexpr (FORM == kGatedForward) {
            if (partial) {                     // as the product of 2 N columns would be
                float *to = partial + (int64_t(blockIdx.y) * M + m) * 2 * N + n0 + n;
                to[0] = d[0];
                to[N] = d[1];
            } else {
                gated1<T>(e, m, n0 + n, d[0], d[1]);
            }
        } else {
            if (partial) partial[(int64_t(blockIdx.y) * M + m) * N + n0 + n] = d[0];
            else finish<T>(e, m, n0 + n, d[0]);
        }
    }
}

// ---------------------------------------------------------------------------------------------- on the host
// Columns at most (a tile of 256 rows then spans less than 2^31 bytes); rows further apart than that are packed.
constexpr int64_t kMostCols = int64_t(1) << 22;
bool sizes_fit(int64_t M, int64_t N, int64_t K) {
    return M >= 0 && M < int64_t(1) << 31 && N >= 1 && K >= 1 && N < kMostCols && K < kMostCols;
}

// How a product is launched.
struct Plan {
    bool few, big;               // few tokens; tiles of 256 x 256, else of 128 x 128
    int shares;                  // of r, joined by a second launch
    int64_t share;               // r of one, a multiple of kPiece
};
constexpr int kFewTokens = 64, kPiece = 64;

int64_t tiles(int64_t P, int64_t Q, int side) { return (P + side - 1) / side * ((Q + side - 1) / side); }

Plan split(Plan p, int64_t R, int64_t shares) {
    const int64_t steps = (R + kPiece - 1) / kPiece;
    shares = shares < steps ? shares : steps;
    shares = shares < 1 ? 1 : shares;
    const int64_t each = (steps + shares - 1) / shares;
    p.share = (each < 1 ? 1 : each) * kPiece;
    p.shares = int(steps ? (steps + each - 1) / each : 1);
    return p;
}

Plan plan_for(const harp_ctx *ctx, int kind, int64_t P, int64_t Q, int64_t R) {
    Plan p = {};
    const int64_t cu = ctx->n_cu;
    if (kind == kForward && P <= kFewTokens) {
        p.few = true;
        const int64_t groups = (Q + 15) / 16;
        // 4 workgroups a compute unit, of at least four pieces a wavefront (8 of them: a second launch that costs 4 us)
        int64_t shares = 4 * cu / (groups > 0 ? groups : 1);
        const int64_t most = R / (16 * kPiece);
        shares = shares < most ? shares : most;
        return split(p, R, shares < 16 ? shares : 16);
    }
    // Microseconds by what was measured (4,096 x 16,384 x 4,096 and 1,537 x 1,224 x 4,904): a round of workgroups takes 0.74 for
    // 32 of r and 13 around them with tiles of 256 x 256, one to a compute unit; 0.5 and 8 with tiles of 128 x 128, two to a
    // compute unit.  Shares of r cost a launch, and their sums' way through memory.
    double best = 1e300;
    for (int big = 0; big < 2; ++big) {
        const int64_t n = tiles(P, Q, big ? 256 : 128), slots = big ? cu : 2 * cu;
        for (int64_t shares = 1; shares <= 16; ++shares) {
            if (shares > 1 && (n * shares > slots || R < shares * 4 * kPiece)) break;
            Plan t = {};
            t.big = big;
            t = split(t, R, shares);
            double us = double((n * t.shares + slots - 1) / slots) * (double(t.share < R ? t.share : R) / 32 * (big ? 0.74 : 0.5) + (big ? 13 : 8));
            if (t.shares > 1) us += 4 + double(t.shares) * double(P) * double(Q) * 8 / 4e6;
            if (us < best) {
                best = us;
                p = t;
            }
        }
    }
    return p;
}

size_t packed_bytes(int64_t rows, int64_t cols) { return round_up(size_t(rows) * round_up(size_t(cols), 8) * 2, 256); }
size_t partial_bytes(const harp_ctx *ctx, int kind, int64_t P, int64_t Q, int64_t R) {
    const Plan p = plan_for(ctx, kind, P, Q, R);
    return p.shares > 1 ? round_up(size_t(p.shares) * size_t(P) * size_t(Q) * 4, 256) : 0;
}

// One operand as it is called with: A(p, r), rows of `cols` elements ld apart.
struct Given { const void *a; int64_t ld, rows, cols; };

bool wide_rows(const Given &g) { return g.cols % 8 == 0 && g.ld % 8 == 0 && g.ld < kMostCols && aligned(g.a, 16); }

uint32_t blocks_for(int64_t threads) {
    const int64_t n = (threads + 255) / 256;
    return uint32_t(n < 16384 ? n : 16384);
}

template <typename T> Given packed(Given g, unsigned char *&ws, hipStream_t st) {
    if (wide_rows(g) || g.rows == 0) return g;
    const int64_t ld = int64_t(round_up(size_t(g.cols), 8));
    T *to = reinterpret_cast<T *>(ws);
    ws += packed_bytes(g.rows, g.cols);
    pack<T><<<dim3(blocks_for(g.rows * (ld / 8))), dim3(256), 0, st>>>(static_cast<const T *>(g.a), g.ld, g.rows, g.cols, to, ld);
    return Given{to, ld, g.rows, g.cols};
}

template <typename T, bool A_ACROSS, bool B_ACROSS>
void launch_tiles(const Plan &plan, const Given &a, const Given &b, int64_t P, int64_t Q, int64_t R, float *partial, const Epilogue &e,
                  hipStream_t st) {
    const int side = plan.big ? 256 : 128;
    const int tp = int((P + side - 1) / side), tq = int((Q + side - 1) / side);
    const dim3 grid(uint32_t(tp) * uint32_t(tq), uint32_t(plan.shares));
    const T *pa = static_cast<const T *>(a.a), *pb = static_cast<const T *>(b.a);
    if (plan.big) product<T, A_ACROSS, B_ACROSS, 256, 256, 2, 4><<<grid, dim3(512), 0, st>>>(pa, a.ld, pb, b.ld, P, Q, R, tp, tq, plan.share, partial, e);
    else product<T, A_ACROSS, B_ACROSS, 128, 128, 2, 2><<<grid, dim3(256), 0, st>>>(pa, a.ld, pb, b.ld, P, Q, R, tp, tq, plan.share, partial, e);
}

struct Matrix { const char *name; const void *p; int64_t ld, cols; size_t element; bool needed; };

int check_operands(harp_ctx *ctx, int type, int act, const Matrix *m, int count) {
    if (type != HARP_BF16 && type != HARP_F16) return fail(ctx, HARP_ERR_INVALID_ARG, "type must be HARP_BF16 or HARP_F16");
    if (act < HARP_ACT_NONE || act > HARP_ACT_SILU) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown activation");
    for (int i = 0; i < count; ++i) {
        if (!m[i].p && m[i].needed) return fail(ctx, HARP_ERR_INVALID_ARG, "null %s", m[i].name);
        if (!m[i].p) continue;
        if (m[i].ld < m[i].cols) return fail(ctx, HARP_ERR_SHAPE, "%s: leading dimension below its columns", m[i].name);
        if (!aligned(m[i].p, m[i].element)) return fail(ctx, HARP_ERR_INVALID_ARG, "%s is not aligned to its elements", m[i].name);
    }
    return HARP_OK;
}

// Compute units finish their tiles together; what they then store at once has to leave the L2 caches of 32 MiB at the
// fabric's pace.  Past the caches the gradients of 4,096 tokens take 1,010 us where they took 1,033; the
// products that read such results next pay some of it back (an MLP of 4,096 channels and tokens forward 960 us for 966).
bool passes_the_caches(int64_t P, int64_t Q, int element) { return size_t(P) * size_t(Q) * size_t(element) >= size_t(32) << 20; }

}  // namespace
