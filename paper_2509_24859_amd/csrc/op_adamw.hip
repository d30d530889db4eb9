// One AdamW step over many tensors, with moments in 32 bits or in 8, and its C entry points.
//
// Nothing is reused and nothing is summed over the tensors, so the step is bound by what it streams: 28 bytes a
// parameter with moments in 32 bits (gradient 2, master, m and v 4 + 4 each, copy 2), 16 with moments in 8.
//
// Measured, bfloat16 gradients and copies: 201 million parameters of 10 tensors 1,065 us, 5.3 TB/s (a copy reaches 4.9); 50 million with
// moments in 8 bits 218 us, 3.7 TB/s: decoding, two hashes and encoding are some 400 vector instructions for four elements;
// 400 tensors of 1,400 elements on average 9 us.
#include <math.h>
#include <string.h>

#include <new>

#include "harp_ctx.h"
#include "ops_common.h"

using namespace harp;
using namespace harp::ops;

namespace {

constexpr int kBlock = 256;               // elements that share an exponent: one wavefront, four elements a lane
constexpr int kThreads = 256;
constexpr int kChunk = 4096;              // elements a workgroup works on
constexpr int kAhead = 2;
constexpr int kTopM = 15, kTopV = 31;     // largest exponent fields of the two codes

struct Tensor {                           // a tensor as the kernels see it
    int64_t n;
    float *p;
    const void *grad;
    void *copy, *m, *v;
    uint8_t *m_exp, *v_exp;
    __bf16 *m_seen, *v_seen;
    double weight_decay;
    uint64_t first_block;                 // place of its first block of 256 among all tensors' (for the rounding's hash)
    int32_t state, grad_type, copy_type;
    int32_t wide;                         // four elements can be read and written at once
};
struct Chunk { uint32_t tensor, index; };  // workgroup -> elements index * kChunk .. of the tensor

struct Step {
    float beta1, beta2, one_minus_beta1, one_minus_beta2, eps, step_size, inv_sqrt_c2;
    double lr;
    uint64_t seed;
    const float *grad_scale;
    const int32_t *skip;
};

// Elements i .. i + 3 of a tensor of n; `wide`: all are there and aligned.  What is not there is 0.
template <typename T> __device__ __forceinline__ f32x4 four_of(const void *p, int64_t i, int64_t n, bool wide) {
    const T *a = static_cast<const T *>(p) + i;
    if (wide) return load4(a);
    f32x4 v;
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = i + j < n ? to_f32(a[j]) : 0.0f;
    return v;
}
__device__ __forceinline__ f32x4 gradient(const void *p, int type, int64_t i, int64_t n, bool wide) {
    return type == HARP_F32 ? four_of<float>(p, i, n, wide) : type == HARP_BF16 ? four_of<__bf16>(p, i, n, wide) : four_of<_Float16>(p, i, n, wide);
}
template <typename T> __device__ __forceinline__ void put_four(void *p, int64_t i, int64_t n, bool wide, f32x4 v) {
    T *a = static_cast<T *>(p) + i;
    if (wide) {
        store4(a, v);
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) a[j] = T(v[j]);
}
__device__ __forceinline__ void put_copy(void *p, int type, int64_t i, int64_t n, bool wide, f32x4 v) {
    if (type == HARP_BF16) put_four<__bf16>(p, i, n, wide, v);
    else put_four<_Float16>(p, i, n, wide, v);
}
// Four codes, the first in the lowest byte.
__device__ __forceinline__ uint32_t codes_of(const uint8_t *a, int64_t i, int64_t n, bool wide) {
    if (wide) return *reinterpret_cast<const uint32_t *>(a + i);
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) c |= i + j < n ? uint32_t(a[i + j]) << (8 * j) : 0;
    return c;
}
__device__ __forceinline__ void put_codes(uint8_t *a, int64_t i, int64_t n, bool wide, uint32_t c) {
    if (wide) {
        *reinterpret_cast<uint32_t *>(a + i) = c;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i + j < n) a[i + j] = uint8_t(c >> (8 * j));
}

// Square root within a unit of the last place, also of numbers so small that the instruction alone is not.
__device__ __forceinline__ float root(float v) {
    const bool small = v < 0x1p-96f;
    return __builtin_amdgcn_sqrtf(small ? v * 0x1p32f : v) * (small ? 0x1p-16f : 1.0f);
}

// The new moments and the new weight.  Every product and sum is rounded by itself (no fused multiply-add): the
// moments in 8 bits are then the same whoever computes them from the formula in 32 bits.  What is taken off the weight
// is summed up first, decay included: 1 - lr weight_decay as a factor would cost the weight two more roundings.
__device__ __forceinline__ void update(const Step &s, float g, float decay, float &p, float &m, float &v) {
#pragma clang fp contract(off)
    m = m * s.beta1 + g * s.one_minus_beta1;
    v = v * s.beta2 + (g * g) * s.one_minus_beta2;
    p = p - (p * decay + s.step_size * m * __builtin_amdgcn_rcpf(root(v) * s.inv_sqrt_c2 + s.eps));
}

// 64 random bits for elements 2 k and 2 k + 1 of all tensors' blocks, from z = k kGamma + seed (splitmix64: Steele, Lea,
// Flood 2014).  Of the lower 32 the lower 16 round m of the even element and the upper its v, of the upper 32 those of
// the odd one.
constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;
__device__ __forceinline__ uint64_t hash(uint64_t z) {
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

// The value of a magnitude code (5 or 4 bits of exponent, 3 of fraction): a whole number below 2^34 times the
// block's unit, a power of two that a float holds for every exponent byte in 64..254.
__device__ __forceinline__ float block_unit(uint32_t exponent, int top) {
    if (exponent == 255) return __uint_as_float(0x7FC00000u);
    return __uint_as_float(((exponent > 64 ? exponent : 64) - top - 2) << 23);   // a cleared byte is the smallest one
}
__device__ __forceinline__ float decode(uint32_t mag, float unit) {
    const uint32_t e = mag >> 3, f = mag & 7;
    const float scale = __uint_as_float((127 + (e > 0 ? e - 1 : 0)) << 23);
    return float(e > 0 ? 8 + f : f) * scale * unit;
}

// Exponent byte of a block whose largest magnitude has these bits: its exponent after rounding up to 3 bits of
// fraction, so that the largest code is never passed.
__device__ __forceinline__ uint32_t block_exponent(uint32_t largest) {
    if (largest >= 0x7F800000u) return 255;
    const uint32_t e = (largest + 0xFFFFFu) >> 23;
    return e < 64 ? 64 : e > 254 ? 254 : e;
}
// Code of a magnitude, `rnd` of 16 bits: the 20 bits below the code are cut off after rnd / 2^16 of one is added.  A v that is
// not zero gets the smallest code at least: v begins at a thousandth of a square where the block's largest is a whole one, so
// that an element's first v can lie below the codes while its m does not; with v zero its next step, unless a gradient as large
// came again, would be m / eps, hundreds of lr.  The smallest code is 2^-16.5 of the block's largest gradient, the smallest of
// m 2^-17: that step is under lr.
__device__ __forceinline__ uint32_t encode(uint32_t bits, uint32_t exponent, int top, uint32_t rnd) {
    const uint32_t mag = bits & 0x7FFFFFFFu, field = mag >> 23;
    const uint32_t whole = (mag & 0x7FFFFFu) | (field ? 0x800000u : 0u);
    const int rel = int(field ? field : 1) - int(exponent) + top;
    const int down = 1 - rel < 31 ? 1 - rel : 31;
    const uint32_t fixed = rel >= 1 ? (uint32_t(rel - 1) << 23) + whole : whole >> down;
    const uint32_t most = top == kTopM ? 127 : 255, least = top == kTopM ? 0 : mag < 1 ? mag : 1;
    const uint32_t code = larger((fixed + (rnd << 4)) >> 20, least);
    return exponent == 255 ? 0 : code < most ? code : most;
}

__global__ __launch_bounds__(kThreads) void adamw_step(const Tensor *tensors, const Chunk *chunks, Step s) {
    if (s.skip && *s.skip) return;
    const Chunk c = chunks[blockIdx.x];
    const Tensor &t = tensors[c.tensor];
    const float scale = s.grad_scale ? *s.grad_scale : 1.0f;
    const float decay = float(s.lr * t.weight_decay);
    const int64_t begin = int64_t(c.index) * kChunk, n = t.n;
    const int64_t end = begin + kChunk < n ? begin + kChunk : n;
    if (t.state == HARP_STATE_F32) {
        // kAhead pieces of four are read before the first is worked on
        auto piece = [&](int64_t at, bool wide) {
            f32x4 g[kAhead], p[kAhead], m[kAhead], v[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t i = at + k * 4 * kThreads;
                g[k] = gradient(t.grad, t.grad_type, i, n, wide);
                p[k] = four_of<float>(t.p, i, n, wide);
                m[k] = four_of<float>(t.m, i, n, wide);
                v[k] = four_of<float>(t.v, i, n, wide);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t i = at + k * 4 * kThreads;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float pj = p[k][j], mj = m[k][j], vj = v[k][j];
                    update(s, g[k][j] * scale, decay, pj, mj, vj);
                    p[k][j] = pj;
                    m[k][j] = mj;
                    v[k][j] = vj;
                }
                put_four<float>(t.p, i, n, wide, p[k]);
                put_four<float>(t.m, i, n, wide, m[k]);
                put_four<float>(t.v, i, n, wide, v[k]);
                if (t.copy) put_copy(t.copy, t.copy_type, i, n, wide, p[k]);
            }
        };
        if (t.wide && begin + kChunk <= n)
            for (int64_t i = begin + 4 * threadIdx.x; i < end; i += kAhead * 4 * kThreads) piece(i, true);
        else
            for (int64_t i = begin + 4 * threadIdx.x; i < end; i += kAhead * 4 * kThreads) piece(i, false);
        return;
    }
    uint8_t *tm = static_cast<uint8_t *>(t.m), *tv = static_cast<uint8_t *>(t.v);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    constexpr int kStep = kThreads / kWave * kBlock;       // to a wavefront's next block
    const uint64_t lane_part = uint64_t(2 * lane) * kGamma;
    auto blocks = [&](int64_t first, bool wide) {
        uint32_t cm[kAhead], cv[kAhead], em[kAhead], ev[kAhead];
        f32x4 g[kAhead], p[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t at = first + k * kStep, i = at + 4 * lane, b = (at < end ? at : first) / kBlock;
            cm[k] = codes_of(tm, i, n, wide);
            cv[k] = codes_of(tv, i, n, wide);
            g[k] = gradient(t.grad, t.grad_type, i, n, wide);
            p[k] = four_of<float>(t.p, i, n, wide);
            em[k] = t.m_exp[b];
            ev[k] = t.v_exp[b];
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int64_t at = first + k * kStep, i = at + 4 * lane, b = at / kBlock;
            if (at >= end) break;
            const float um = block_unit(em[k], kTopM), uv = block_unit(ev[k], kTopV);
            float m[4], v[4];
            uint32_t most_m = 0, most_v = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = cm[k] >> (8 * j) & 255;
                m[j] = decode(a & 127, um);
                m[j] = a & 128 ? -m[j] : m[j];
                v[j] = decode(cv[k] >> (8 * j) & 255, uv);
                float pj = p[k][j];
                update(s, g[k][j] * scale, decay, pj, m[j], v[j]);
                p[k][j] = pj;
                if (wide || i + j < n) {                   // what is not there has no say in the block's exponent
                    most_m = larger(most_m, __float_as_uint(m[j]) & 0x7FFFFFFFu);
                    most_v = larger(most_v, __float_as_uint(v[j]) & 0x7FFFFFFFu);
                }
            }
            const uint32_t nm = block_exponent(wave_max(most_m)), nv = block_exponent(wave_max(most_v));
            // k = (element's place) / 2: the block's part is the same for the wavefront
            const uint64_t z = (t.first_block + b) * (kBlock / 2) * kGamma + s.seed + lane_part;
            uint32_t out_m = 0, out_v = 0;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint64_t bits = hash(z + h * kGamma);
#pragma unroll
                for (int j = 2 * h; j < 2 * h + 2; ++j) {
                    const uint32_t r = uint32_t(bits >> (32 * (j & 1))), bm = __float_as_uint(m[j]);
                    out_m |= (encode(bm, nm, kTopM, r & 0xFFFF) | (bm >> 24 & 128)) << (8 * j);
                    out_v |= encode(__float_as_uint(v[j]), nv, kTopV, r >> 16) << (8 * j);
                }
            }
            put_four<float>(t.p, i, n, wide, p[k]);
            if (t.copy) put_copy(t.copy, t.copy_type, i, n, wide, p[k]);
            put_codes(tm, i, n, wide, out_m);
            put_codes(tv, i, n, wide, out_v);
            if (lane == 0) {
                t.m_exp[b] = uint8_t(nm);
                t.v_exp[b] = uint8_t(nv);
            }
        }
    };
    if (t.wide && begin + kChunk <= n)
        for (int64_t at = begin + wave * kBlock; at < end; at += kAhead * kStep) blocks(at, true);
    else
        for (int64_t at = begin + wave * kBlock; at < end; at += kAhead * kStep) blocks(at, false);
}

__global__ __launch_bounds__(kThreads) void adamw_read(const Tensor *tensors, const Chunk *chunks) {
    const Chunk c = chunks[blockIdx.x];
    const Tensor &t = tensors[c.tensor];
    if (t.state != HARP_STATE_8BIT) return;
    const int64_t begin = int64_t(c.index) * kChunk, n = t.n;
    const int64_t end = begin + kChunk < n ? begin + kChunk : n;
    const uint8_t *tm = static_cast<const uint8_t *>(t.m), *tv = static_cast<const uint8_t *>(t.v);
    auto pieces = [&](int64_t first, bool wide) {
        uint32_t cm[2 * kAhead], cv[2 * kAhead], em[2 * kAhead], ev[2 * kAhead];
#pragma unroll
        for (int k = 0; k < 2 * kAhead; ++k) {
            const int64_t i = first + k * 4 * kThreads, b = (i < end ? i : first) / kBlock;
            cm[k] = codes_of(tm, i, n, wide);
            cv[k] = codes_of(tv, i, n, wide);
            em[k] = t.m_exp[b];
            ev[k] = t.v_exp[b];
        }
#pragma unroll
        for (int k = 0; k < 2 * kAhead; ++k) {
            const int64_t i = first + k * 4 * kThreads;
            const float um = block_unit(em[k], kTopM), uv = block_unit(ev[k], kTopV);
            f32x4 m, v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = cm[k] >> (8 * j) & 255;
                m[j] = decode(a & 127, um);
                m[j] = a & 128 ? -m[j] : m[j];
                v[j] = decode(cv[k] >> (8 * j) & 255, uv);
            }
            if (t.m_seen) put_four<__bf16>(t.m_seen, i, n, wide, m);
            if (t.v_seen) put_four<__bf16>(t.v_seen, i, n, wide, v);
        }
    };
    static_assert(kChunk == 2 * kAhead * 4 * kThreads, "one round of a workgroup is a chunk");
    if (begin + 4 * int(threadIdx.x) >= end) return;
    if (t.wide && begin + kChunk <= n) pieces(begin + 4 * threadIdx.x, true);
    else pieces(begin + 4 * threadIdx.x, false);
}

const char *tensor_fault(const harp_adamw_tensor &t) {
    if (t.n < 0 || t.n >= int64_t(1) << 40) return "n must be in 0 .. 2^40 - 1";
    if (t.state != HARP_STATE_F32 && t.state != HARP_STATE_8BIT) return "state must be HARP_STATE_F32 or HARP_STATE_8BIT";
    if (!type_bytes(t.grad_type)) return "unknown grad_type";
    if (t.copy && t.copy_type != HARP_BF16 && t.copy_type != HARP_F16) return "copy_type must be HARP_BF16 or HARP_F16";
    if (t.flags) return "flags must be 0";
    if (!(t.weight_decay >= 0) || isinf(t.weight_decay)) return "weight_decay must be a finite number >= 0";
    if (t.n == 0) return nullptr;
    if (!t.p || !t.grad || !t.m || !t.v) return "null p, grad, m or v";
    if (t.state == HARP_STATE_8BIT && (!t.m_exp || !t.v_exp)) return "8-bit states need m_exp and v_exp";
    if (!aligned(t.p, 4) || !aligned(t.grad, size_t(type_bytes(t.grad_type))) || !aligned(t.copy, 2) ||
        !aligned(t.m_seen, 2) || !aligned(t.v_seen, 2) ||
        (t.state == HARP_STATE_F32 && (!aligned(t.m, 4) || !aligned(t.v, 4))))
        return "a pointer is not aligned to its elements";
    return nullptr;
}

struct PlanLayout {
    size_t chunks_at, bytes;
    int64_t n_chunks;
};
// false: malformed (`why` says what is wrong)
bool plan_layout(const harp_adamw_tensor *tensors, int32_t n, PlanLayout &y, const char *&why, int &which) {
    why = "null tensors or a negative count";
    which = 0;
    if (n < 0 || (n > 0 && !tensors)) return false;
    y.n_chunks = 0;
    for (int32_t i = 0; i < n; ++i) {
        which = i;
        if ((why = tensor_fault(tensors[i]))) return false;
        y.n_chunks += (tensors[i].n + kChunk - 1) / kChunk;
    }
    why = "more than 2^24 - 1 pieces of 4,096 elements (a launch has at most 2^32 - 1 threads)";
    if (y.n_chunks >= 1 << 24) return false;
    y.chunks_at = round_up(size_t(n) * sizeof(Tensor), 256);
    y.bytes = y.chunks_at + round_up(size_t(y.n_chunks) * sizeof(Chunk), 256) + 256;
    return true;
}

}  // namespace

struct harp_adamw {
    const Tensor *tensors;
    const Chunk *chunks;
    int64_t n_chunks;
    int device;
};

extern "C" {

size_t harp_adamw_plan_bytes(const harp_adamw_tensor *tensors, int32_t n_tensors) {
    PlanLayout y;
    const char *why;
    int which;
    return plan_layout(tensors, n_tensors, y, why, which) ? y.bytes : 0;
}

int harp_adamw_plan(harp_ctx *ctx, const harp_adamw_tensor *tensors, int32_t n_tensors, void *plan_buf,
                    size_t plan_bytes, harp_adamw **out, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!out) return fail(ctx, HARP_ERR_INVALID_ARG, "null out");
    *out = nullptr;
    PlanLayout y;
    const char *why;
    int which;
    if (!plan_layout(tensors, n_tensors, y, why, which)) return fail(ctx, HARP_ERR_INVALID_ARG, "tensor %d: %s", which, why);
    if (!plan_buf || !aligned(plan_buf, 256) || plan_bytes < y.bytes)
        return fail(ctx, HARP_ERR_WORKSPACE, "the plan needs %zu bytes, aligned to 256", y.bytes);
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    hipStreamCaptureStatus capture = hipStreamCaptureStatusNone;
    e = hipStreamIsCapturing(st, &capture);
    if (e != hipSuccess) return hip_fail(ctx, e, "asking whether the stream is being captured");
    if (capture != hipStreamCaptureStatusNone)
        return fail(ctx, HARP_ERR_INVALID_ARG, "a plan cannot be made while the stream is being captured: it is waited for");
    harp_adamw *view = new (std::nothrow) harp_adamw;
    unsigned char *host = new (std::nothrow) unsigned char[y.bytes];
    if (!view || !host) {
        delete view;
        delete[] host;
        return fail(ctx, HARP_ERR_INVALID_ARG, "out of host memory");
    }
    memset(host, 0, y.bytes);
    Tensor *t = reinterpret_cast<Tensor *>(host);
    Chunk *c = reinterpret_cast<Chunk *>(host + y.chunks_at);
    uint64_t block = 0;
    for (int32_t i = 0; i < n_tensors; ++i) {
        const harp_adamw_tensor &a = tensors[i];
        Tensor d = {};
        d.n = a.n;
        d.p = a.p;
        d.grad = a.grad;
        d.copy = a.copy;
        d.m = a.m;
        d.v = a.v;
        d.m_exp = a.m_exp;
        d.v_exp = a.v_exp;
        d.m_seen = static_cast<__bf16 *>(a.m_seen);
        d.v_seen = static_cast<__bf16 *>(a.v_seen);
        d.weight_decay = a.weight_decay;
        d.first_block = block;
        d.state = a.state;
        d.grad_type = a.grad_type;
        d.copy_type = a.copy_type;
        d.wide = aligned(a.p, 16) && aligned(a.grad, 4 * size_t(type_bytes(a.grad_type))) && aligned(a.copy, 8) && aligned(a.m_seen, 8) &&
                 aligned(a.v_seen, 8) && aligned(a.m, a.state == HARP_STATE_F32 ? 16 : 4) && aligned(a.v, a.state == HARP_STATE_F32 ? 16 : 4);
        t[i] = d;
        block += uint64_t(a.n + kBlock - 1) / kBlock;
        for (int64_t k = 0; k * kChunk < a.n; ++k) *c++ = Chunk{uint32_t(i), uint32_t(k)};
    }
    e = hipMemcpyAsync(plan_buf, host, y.bytes, hipMemcpyHostToDevice, st);
    if (e == hipSuccess) e = hipStreamSynchronize(st);
    delete[] host;
    if (e != hipSuccess) {
        delete view;
        return hip_fail(ctx, e, "writing the plan");
    }
    view->tensors = static_cast<const Tensor *>(plan_buf);
    view->chunks = reinterpret_cast<const Chunk *>(static_cast<unsigned char *>(plan_buf) + y.chunks_at);
    view->n_chunks = y.n_chunks;
    view->device = ctx->device;
    *out = view;
    return HARP_OK;
}

int harp_adamw_step(harp_ctx *ctx, const harp_adamw *plan, const harp_adamw_hyper *h, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!plan || !h) return fail(ctx, HARP_ERR_INVALID_ARG, "null plan or hyper");
    if (plan->device != ctx->device) return fail(ctx, HARP_ERR_INVALID_ARG, "the plan belongs to another device");
    if (!(h->lr >= 0) || isinf(h->lr) || !(h->beta1 >= 0 && h->beta1 < 1) || !(h->beta2 >= 0 && h->beta2 < 1) ||
        !(h->eps >= 0) || isinf(h->eps))
        return fail(ctx, HARP_ERR_INVALID_ARG, "lr and eps must be finite and >= 0, beta1 and beta2 in [0, 1)");
    if (h->step < 1) return fail(ctx, HARP_ERR_INVALID_ARG, "step must be >= 1");
    if (plan->n_chunks == 0) return HARP_OK;
    Step s;
    s.beta1 = float(h->beta1);
    s.beta2 = float(h->beta2);
    s.one_minus_beta1 = float(1.0 - h->beta1);
    s.one_minus_beta2 = float(1.0 - h->beta2);
    s.eps = float(h->eps);
    s.step_size = float(h->lr / (1.0 - pow(h->beta1, double(h->step))));
    s.inv_sqrt_c2 = float(1.0 / sqrt(1.0 - pow(h->beta2, double(h->step))));
    s.lr = h->lr;
    s.seed = h->seed;
    s.grad_scale = h->grad_scale;
    s.skip = h->skip;
    hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    hipLaunchKernelGGL(adamw_step, dim3(uint32_t(plan->n_chunks)), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream),
                       plan->tensors, plan->chunks, s);
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(ctx, e, "launching the AdamW kernel");
    return HARP_OK;
}

int harp_adamw_read_state(harp_ctx *ctx, const harp_adamw *plan, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!plan) return fail(ctx, HARP_ERR_INVALID_ARG, "null plan");
    if (plan->device != ctx->device) return fail(ctx, HARP_ERR_INVALID_ARG, "the plan belongs to another device");
    if (plan->n_chunks == 0) return HARP_OK;
    hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    hipLaunchKernelGGL(adamw_read, dim3(uint32_t(plan->n_chunks)), dim3(kThreads), 0, static_cast<hipStream_t>(hip_stream),
                       plan->tensors, plan->chunks);
    e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(ctx, e, "launching the state reader");
    return HARP_OK;
}

void harp_adamw_release(harp_adamw *plan) { delete plan; }

}  // extern "C"
