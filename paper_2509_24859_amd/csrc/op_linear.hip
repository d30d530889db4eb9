// Matrix product with bias, activation and residual in its epilogue, its gradients, and their C entry points.
//
// The three products are one form, D[p][q] = sum over r of A(p, r) B(q, r):
//   forward          p = token,  q = output,  r = input     A = X, B = W, both with r contiguous
//   input gradient   p = token,  q = input,   r = output    A = dY, r contiguous; B = W, q contiguous
//   weight gradient  p = output, q = input,   r = token     A = dY, B = X, p and q contiguous
#include <math.h>

#include <type_traits>

#include "harp_ctx.h"
#include "ops_common.h"

using namespace harp;
using namespace harp::ops;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

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
    __device__ __forceinline__ void begin(const T *a, int64_t ld, int64_t p0, int64_t P, int64_t r0) {
        step = (ACROSS ? kDeep * ld : kDeep) * int64_t(sizeof(T));
        base = reinterpret_cast<const char *>(ACROSS ? a + r0 * ld + p0 : a + p0 * ld + r0);
        // beyond the edge: anything that is there
        const int last = int(ACROSS ? (P + 7) / 8 * 8 - 8 - p0 : P - 1 - p0);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int id = place(i), p = ACROSS ? ((id % kRow) ^ swap_of(id / kRow)) * 8 : id / kRow, at = p < last ? p : last;
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
template <typename T, bool A_ACROSS, bool B_ACROSS, int BP, int BQ, int WP, int WQ>
__global__ __launch_bounds__(WP * WQ * kWave) void product(const T *a, int64_t lda, const T *b, int64_t ldb, int64_t P, int64_t Q, int64_t R,
                                                           int tiles_p, int tiles_q, int64_t share, float *partial, Epilogue e) {
    constexpr int kThreads = WP * WQ * kWave, kP = BP / WP / 16, kQ = BQ / WQ / 16;
    constexpr bool kPairs = !(A_ACROSS && B_ACROSS);
    constexpr int kBuffers = kPairs ? 5 : 4;
    __shared__ __align__(16) T la[kBuffers][BP * kDeep];
    __shared__ __align__(16) T lb[kBuffers][BQ * kDeep];
    int tp, tq;
    tile_of(blockIdx.x, tiles_p, tiles_q, tp, tq);
    const int64_t p0 = int64_t(tp) * BP, q0 = int64_t(tq) * BQ;
    const int64_t r0 = int64_t(blockIdx.y) * share, r1 = r0 + share < R ? r0 + share : R;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int wp = wave / WQ * (BP / WP), wq = wave % WQ * (BQ / WQ);
    Side<T, A_ACROSS, BP, kThreads> sa;
    Side<T, B_ACROSS, BQ, kThreads> sb;
    sa.begin(a, lda, p0, P, r0);
    sb.begin(b, ldb, q0, Q, r0);
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
    if (partial) e = Epilogue{kWeight, HARP_ACT_NONE, 0, 1, 0, partial + int64_t(blockIdx.y) * P * Q, nullptr, nullptr, nullptr, nullptr, Q, 0, 0};
    constexpr int kCols = BQ / WQ, kPitch = kCols + 4, kLanes = kCols / 4, kRows = kWave / kLanes, kParts = 16 / kRows;
    static_assert(WP * WQ * 16 * kPitch * 4 <= kBuffers * BP * kDeep * 2, "the wavefronts' rows have to fit into the first operand's LDS");
    float *rows = reinterpret_cast<float *>(&la[0][0]) + wave * 16 * kPitch;
    const int64_t q = q0 + wq + lane % kLanes * 4;
    auto row_of = [&](int i, int k) { return p0 + wp + 16 * i + k * kRows + lane / kLanes; };
    auto through_lds = [&](int i) {
#pragma unroll
        for (int j = 0; j < kQ; ++j) *reinterpret_cast<f32x4 *>(rows + lane % 16 * kPitch + 16 * j + lane / 16 * 4) = acc[i][j];
        __builtin_amdgcn_wave_barrier();
    };
    auto from_lds = [&](int k) { return *reinterpret_cast<const f32x4 *>(rows + (k * kRows + lane / kLanes) * kPitch + lane % kLanes * 4); };
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
template <typename T, bool WIDE, int TILES>
__global__ __launch_bounds__(kFewWaves * kWave) void few_tokens(const T *x, int64_t ldx, const T *w, int64_t ldw, int64_t M, int64_t N, int64_t R,
                                                                int64_t share, float *partial, Epilogue e) {
    __shared__ float sums[kFewWaves][TILES * 16][17];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, i = lane % 16, g = lane / 16;
    const int64_t n0 = int64_t(blockIdx.x) * 16;
    const int64_t r0 = int64_t(blockIdx.y) * share, r1 = r0 + share < R ? r0 + share : R;
    const T *wr = w + (n0 + i < N ? n0 + i : N - 1) * ldw;
    const T *xr[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) xr[t] = x + (16 * t + i < M ? 16 * t + i : M - 1) * ldx;
    f32x4 acc[TILES] = {};
    // several pieces are asked for before the first is used: a compute unit then has 128 KB of weights on their way
    constexpr int kAhead = TILES == 1 ? 4 : 2;
    for (int64_t r = r0 + wave * 64 + 16 * g; r - 16 * g < r1; r += kAhead * kFewWaves * 64) {
        typename Mfma<T>::Frag a[kAhead][2], b[TILES][kAhead][2];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) a[k][h] = eight<T, WIDE>(wr, r + k * kFewWaves * 64 + 8 * h, r1);
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
                for (int h = 0; h < 2; ++h) acc[t] = Mfma<T>::run(a[k][h], b[t][k][h], acc[t]);
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
        for (int k = 0; k < 4; ++k) sums[wave][16 * t + i][4 * g + k] = acc[t][k];
    __syncthreads();
    for (int at = threadIdx.x; at < TILES * 256; at += kFewWaves * kWave) {
        const int m = at / 16, n = at % 16;
        float d = 0;
        for (int v = 0; v < kFewWaves; ++v) d += sums[v][m][n];
        if (m >= M || n0 + n >= N) continue;
        if (partial) partial[(int64_t(blockIdx.y) * M + m) * N + n0 + n] = d;
        else finish<T>(e, m, n0 + n, d);
    }
}

// Column sums of dY.  A workgroup takes 256 columns, 8 to a thread, and kSumRows rows, every eighth to a thread: pieces of 16
// bytes wherever they lie, several rows asked for at a time; bound by reading dY.  The second launch adds the slabs up.
// 4,096 x 4,096 in 61 us with a column and 256 rows to a thread.
constexpr int kSumRows = 64, kSumCols = 256;
template <typename T>
__global__ __launch_bounds__(256) void column_sums(const T *dy, int64_t ld, int64_t M, int64_t N, float *partial) {
    typedef typename Mfma<T>::Frag Piece;
    typedef Piece Loose __attribute__((aligned(sizeof(T))));
    __shared__ float runs[8][kSumCols + 1];
    const int part = threadIdx.x % 32, run = threadIdx.x / 32;
    const int64_t n = int64_t(blockIdx.x) * kSumCols + part * 8, m0 = int64_t(blockIdx.y) * kSumRows;
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (n + 8 <= N) {
        Piece v[kSumRows / 8] = {};
#pragma unroll
        for (int i = 0; i < kSumRows / 8; ++i)
            if (m0 + run + 8 * i < M) v[i] = *reinterpret_cast<const Loose *>(dy + (m0 + run + 8 * i) * ld + n);
#pragma unroll
        for (int i = 0; i < kSumRows / 8; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] += to_f32(T(v[i][k]));
    } else {
        for (int64_t m = m0 + run; m < m0 + kSumRows && m < M; m += 8)
            for (int k = 0; k < 8; ++k)
                if (n + k < N) s[k] += to_f32(dy[m * ld + n + k]);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) runs[run][part * 8 + k] = s[k];
    __syncthreads();
    const int64_t at = int64_t(blockIdx.x) * kSumCols + threadIdx.x;
    float d = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) d += runs[i][threadIdx.x];
    if (at < N) partial[int64_t(blockIdx.y) * N + at] = d;
}
// 16 columns a workgroup, 16 threads to a column, each a run of slabs in order, then the runs in order.
__global__ __launch_bounds__(256) void column_join(const float *partial, int64_t count, int64_t N, float *out, int accumulate) {
    __shared__ float runs[16][17];
    const int c = threadIdx.x % 16, run = threadIdx.x / 16;
    const int64_t n = int64_t(blockIdx.x) * 16 + c, each = (count + 15) / 16;
    const int64_t last = (run + 1) * each < count ? (run + 1) * each : count;
    float s = 0;
    if (n < N)
#pragma unroll 4
        for (int64_t i = run * each; i < last; ++i) s += partial[i * N + n];
    runs[run][c] = s;
    __syncthreads();
    if (run != 0 || n >= N) return;
    s = 0;
    for (int i = 0; i < 16; ++i) s += runs[i][c];
    out[n] = accumulate ? out[n] + s : s;
}

template <typename T>
__global__ __launch_bounds__(256) void act_grad(int64_t M, int64_t N, int act, const T *dy, int64_t lddy, const T *z, int64_t ldz, T *dz,
                                                int64_t lddz) {
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= N) return;
    for (int64_t m = blockIdx.y; m < M; m += gridDim.y)
        dz[m * lddz + n] = T(to_f32(dy[m * lddy + n]) * slope(to_f32(z[m * ldz + n]), act));
}

int64_t slabs_of(int64_t M) { return (M + kSumRows - 1) / kSumRows; }

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
size_t most(size_t a, size_t b) { return a > b ? a : b; }

// Both operands packed, and shares of r or column sums.
size_t workspace_for(const harp_ctx *ctx, int64_t M, int64_t N, int64_t K) {
    const size_t x = packed_bytes(M, K), w = packed_bytes(N, K), dy = packed_bytes(M, N);
    const size_t forward = x + w + partial_bytes(ctx, kForward, M, N, K);
    const size_t input = dy + w + partial_bytes(ctx, kInput, M, K, N);
    const size_t weight = dy + x + most(partial_bytes(ctx, kWeight, N, K, M), round_up(size_t(slabs_of(M)) * size_t(N) * 4, 256));
    return most(most(forward, input), weight) + 256;
}

struct Matrix { const char *name; const void *p; int64_t ld, cols; size_t element; bool needed; };

int check(harp_ctx *ctx, int64_t M, int64_t N, int64_t K, int type, int act, const Matrix *m, int count, const void *workspace,
          size_t workspace_bytes) {
    if (!sizes_fit(M, N, K)) return fail(ctx, HARP_ERR_SHAPE, "0 <= M < 2^31 and 1 <= N, K < 2^22 are wanted");
    if (type != HARP_BF16 && type != HARP_F16) return fail(ctx, HARP_ERR_INVALID_ARG, "type must be HARP_BF16 or HARP_F16");
    if (act < HARP_ACT_NONE || act > HARP_ACT_SILU) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown activation");
    for (int i = 0; i < count; ++i) {
        if (!m[i].p && m[i].needed) return fail(ctx, HARP_ERR_INVALID_ARG, "null %s", m[i].name);
        if (!m[i].p) continue;
        if (m[i].ld < m[i].cols) return fail(ctx, HARP_ERR_SHAPE, "%s: leading dimension below its columns", m[i].name);
        if (!aligned(m[i].p, m[i].element)) return fail(ctx, HARP_ERR_INVALID_ARG, "%s is not aligned to its elements", m[i].name);
    }
    const size_t need = workspace_for(ctx, M, N, K);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
        return fail(ctx, HARP_ERR_WORKSPACE, "the workspace needs %zu bytes, aligned to 256", need);
    const hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    return HARP_OK;
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

template <typename T, bool WIDE>
void launch_few(const Plan &plan, const Given &x, const Given &w, int64_t M, int64_t N, int64_t R, float *partial, const Epilogue &e,
                hipStream_t st) {
    const dim3 grid(uint32_t((N + 15) / 16), uint32_t(plan.shares)), block(kFewWaves * kWave);
    const T *px = static_cast<const T *>(x.a), *pw = static_cast<const T *>(w.a);
    if (M <= 16) few_tokens<T, WIDE, 1><<<grid, block, 0, st>>>(px, x.ld, pw, w.ld, M, N, R, plan.share, partial, e);
    else if (M <= 32) few_tokens<T, WIDE, 2><<<grid, block, 0, st>>>(px, x.ld, pw, w.ld, M, N, R, plan.share, partial, e);
    else few_tokens<T, WIDE, 4><<<grid, block, 0, st>>>(px, x.ld, pw, w.ld, M, N, R, plan.share, partial, e);
}

template <typename T>
void launch_product(const harp_ctx *ctx, Given a, Given b, int64_t P, int64_t Q, int64_t R, Epilogue e, void *workspace, hipStream_t st) {
    const Plan plan = plan_for(ctx, e.kind, P, Q, R);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    // Compute units finish their tiles together; what they then store at once has to leave the L2 caches of 32 MiB at the
    // fabric's pace.  Past the caches the gradients of 4,096 tokens take 1,010 us where they took 1,033; the
    // products that read such results next pay some of it back (an MLP of 4,096 channels and tokens forward 960 us for 966).
    e.past = size_t(P) * size_t(Q) * (e.out_f32 ? 4 : 2) >= size_t(32) << 20;
    if (!plan.few) {
        a = packed<T>(a, ws, st);
        b = packed<T>(b, ws, st);
    }
    float *partial = plan.shares > 1 ? reinterpret_cast<float *>(ws) : nullptr;
    if (plan.few) {
        if (wide_rows(a) && wide_rows(b)) launch_few<T, true>(plan, a, b, P, Q, R, partial, e, st);
        else launch_few<T, false>(plan, a, b, P, Q, R, partial, e, st);
    } else if (e.kind == kForward) {
        launch_tiles<T, false, false>(plan, a, b, P, Q, R, partial, e, st);
    } else if (e.kind == kInput) {
        launch_tiles<T, false, true>(plan, a, b, P, Q, R, partial, e, st);
    } else {
        launch_tiles<T, true, true>(plan, a, b, P, Q, R, partial, e, st);
    }
    if (partial) join<T><<<dim3(blocks_for(P * ((Q + 3) / 4))), dim3(256), 0, st>>>(partial, plan.shares, P, Q, e);
}

template <typename T> void launch_sums(const harp_linear_weight *g, uint32_t across, int64_t slabs, float *partial, hipStream_t st) {
    for (int64_t first = 0; first < slabs; first += 65535) {      // a launch has 65,535 rows of workgroups at most
        const int64_t row = first * kSumRows;
        column_sums<T><<<dim3(across, uint32_t(slabs - first < 65535 ? slabs - first : 65535)), dim3(256), 0, st>>>(
            static_cast<const T *>(g->dY) + row * g->lddy, g->lddy, g->M - row, g->N, partial + first * g->N);
    }
}

int launched(harp_ctx *ctx) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HARP_OK : hip_fail(ctx, e, "launching the product's kernels");
}

}  // namespace

extern "C" {

size_t harp_linear_workspace_bytes(harp_ctx *ctx, int64_t M, int64_t N, int64_t K) {
    return ctx && sizes_fit(M, N, K) ? workspace_for(ctx, M, N, K) : 0;
}

int harp_linear_forward(harp_ctx *ctx, const harp_linear *g, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    const bool some = g->M > 0;
    const Matrix m[] = {{"X", g->X, g->ldx, g->K, 2, some}, {"W", g->W, g->ldw, g->K, 2, true}, {"bias", g->bias, g->N, g->N, 2, false},
                        {"residual", g->residual, g->ldr, g->N, 2, false}, {"Y", g->Y, g->ldy, g->N, 2, some}, {"Z", g->Z, g->ldz, g->N, 2, false}};
    const int rc = check(ctx, g->M, g->N, g->K, g->type, g->act, m, 6, workspace, workspace_bytes);
    if (rc != HARP_OK || !some) return rc;
    const Epilogue e = {kForward, g->act, 0, 0, 0, g->Y, g->bias, g->residual, nullptr, g->Z, g->ldy, g->ldr, g->ldz};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) launch_product<__bf16>(ctx, {g->X, g->ldx, g->M, g->K}, {g->W, g->ldw, g->N, g->K}, g->M, g->N, g->K, e, workspace, st);
    else launch_product<_Float16>(ctx, {g->X, g->ldx, g->M, g->K}, {g->W, g->ldw, g->N, g->K}, g->M, g->N, g->K, e, workspace, st);
    return launched(ctx);
}

int harp_linear_grad_input(harp_ctx *ctx, const harp_linear_input *g, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    const bool some = g->M > 0;
    const Matrix m[] = {{"dY", g->dY, g->lddy, g->N, 2, some}, {"W", g->W, g->ldw, g->K, 2, true},
                        {"Z", g->act != HARP_ACT_NONE ? g->Z : nullptr, g->ldz, g->K, 2, some && g->act != HARP_ACT_NONE},
                        {"residual", g->residual, g->ldr, g->K, 2, false}, {"dX", g->dX, g->lddx, g->K, 2, some}};
    const int rc = check(ctx, g->M, g->N, g->K, g->type, g->act, m, 5, workspace, workspace_bytes);
    if (rc != HARP_OK || !some) return rc;
    const Epilogue e = {kInput, g->act, 0, 0, 0, g->dX, nullptr, g->residual, g->act != HARP_ACT_NONE ? g->Z : nullptr, nullptr, g->lddx, g->ldr, g->ldz};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) launch_product<__bf16>(ctx, {g->dY, g->lddy, g->M, g->N}, {g->W, g->ldw, g->N, g->K}, g->M, g->K, g->N, e, workspace, st);
    else launch_product<_Float16>(ctx, {g->dY, g->lddy, g->M, g->N}, {g->W, g->ldw, g->N, g->K}, g->M, g->K, g->N, e, workspace, st);
    return launched(ctx);
}

int harp_linear_grad_weight(harp_ctx *ctx, const harp_linear_weight *g, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    if (g->dw_type != g->type && g->dw_type != HARP_F32) return fail(ctx, HARP_ERR_INVALID_ARG, "dw_type must be type or HARP_F32");
    const bool some = g->M > 0;
    const Matrix m[] = {{"dY", g->dY, g->lddy, g->N, 2, some}, {"X", g->X, g->ldx, g->K, 2, some},
                        {"dW", g->dW, g->lddw, g->K, size_t(type_bytes(g->dw_type)), true}, {"dbias", g->dbias, g->N, g->N, 4, false}};
    const int rc = check(ctx, g->M, g->N, g->K, g->type, HARP_ACT_NONE, m, 4, workspace, workspace_bytes);
    if (rc != HARP_OK) return rc;
    if (!some && g->accumulate) return HARP_OK;
    const Epilogue e = {kWeight, HARP_ACT_NONE, g->accumulate, g->dw_type == HARP_F32, 0, g->dW, nullptr, nullptr, nullptr, nullptr, g->lddw, 0, 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) launch_product<__bf16>(ctx, {g->dY, g->lddy, g->M, g->N}, {g->X, g->ldx, g->M, g->K}, g->N, g->K, g->M, e, workspace, st);
    else launch_product<_Float16>(ctx, {g->dY, g->lddy, g->M, g->N}, {g->X, g->ldx, g->M, g->K}, g->N, g->K, g->M, e, workspace, st);
    if (g->dbias) {
        float *partial = static_cast<float *>(workspace);
        const int64_t slabs = slabs_of(g->M);
        const uint32_t across = uint32_t((g->N + kSumCols - 1) / kSumCols);
        if (some && g->type == HARP_BF16) launch_sums<__bf16>(g, across, slabs, partial, st);
        else if (some) launch_sums<_Float16>(g, across, slabs, partial, st);
        column_join<<<dim3(uint32_t((g->N + 15) / 16)), dim3(256), 0, st>>>(partial, slabs, g->N, g->dbias, g->accumulate);
    }
    return launched(ctx);
}

int harp_act_grad(harp_ctx *ctx, int64_t M, int64_t N, int32_t type, int32_t act, const void *dY, int64_t lddy, const void *Z,
                  int64_t ldz, void *dZ, int64_t lddz, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (M < 0 || N < 0 || M >= int64_t(1) << 31 || N >= int64_t(1) << 31) return fail(ctx, HARP_ERR_SHAPE, "M and N must be in 0 .. 2^31 - 1");
    const size_t element = size_t(type_bytes(type));
    if (!element) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown type");
    if (act < HARP_ACT_NONE || act > HARP_ACT_SILU) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown activation");
    if (M == 0 || N == 0) return HARP_OK;
    if (!dY || !Z || !dZ) return fail(ctx, HARP_ERR_INVALID_ARG, "null dY, Z or dZ");
    if (lddy < N || ldz < N || lddz < N) return fail(ctx, HARP_ERR_SHAPE, "a leading dimension is below N");
    if (!aligned(dY, element) || !aligned(Z, element) || !aligned(dZ, element))
        return fail(ctx, HARP_ERR_INVALID_ARG, "a pointer is not aligned to its elements");
    hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    const dim3 grid(uint32_t((N + 255) / 256), uint32_t(M < 65535 ? M : 65535));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
#define RUN(T) act_grad<T><<<grid, dim3(256), 0, st>>>(M, N, act, static_cast<const T *>(dY), lddy, static_cast<const T *>(Z), ldz, static_cast<T *>(dZ), lddz)
    if (type == HARP_F32) RUN(float);
    else if (type == HARP_BF16) RUN(__bf16);
    else RUN(_Float16);
#undef RUN
    return launched(ctx);
}

}  // extern "C"
