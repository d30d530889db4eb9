// One AdamW step over many tensors, with moments in 32 bits or in 8, and its C entry points.
//
// Nothing is reused and nothing is summed over the tensors, so the step is bound by what it streams: 28 bytes a
// parameter with moments in 32 bits (gradient 2, master, m and v 4 + 4 each, copy 2), 16 with moments in 8.
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
    int32_t wide;                         // pointers allow loads of four elements
};
struct Chunk { uint32_t tensor, index; };  // workgroup -> elements index * kChunk .. of the tensor

struct Step {
    float beta1, beta2, one_minus_beta1, one_minus_beta2, eps, step_size, inv_sqrt_c2;
    double lr;
    uint64_t seed;
    const float *grad_scale;
    const int32_t *skip;
};

__device__ __forceinline__ float element(const void *p, int type, int64_t i) {
    return type == HARP_F32 ? static_cast<const float *>(p)[i]
           : type == HARP_BF16 ? to_f32(static_cast<const __bf16 *>(p)[i])
                               : to_f32(static_cast<const _Float16 *>(p)[i]);
}
__device__ __forceinline__ void put_copy(void *p, int type, int64_t i, float v) {
    if (type == HARP_BF16) static_cast<__bf16 *>(p)[i] = __bf16(v);
    else static_cast<_Float16 *>(p)[i] = _Float16(v);
}

// The new moments and the new weight.  Every product and sum is rounded by itself (no fused multiply-add): the
// moments in 8 bits are then the same whoever computes them from the formula in 32 bits.  What is taken off the weight
// is summed up first, decay included: 1 - lr weight_decay as a factor would cost the weight two more roundings.
__device__ __forceinline__ void update(const Step &s, float g, float decay, float &p, float &m, float &v) {
#pragma clang fp contract(off)
    m = m * s.beta1 + g * s.one_minus_beta1;
    v = v * s.beta2 + (g * g) * s.one_minus_beta2;
    p = p - (p * decay + s.step_size * m / (sqrtf(v) * s.inv_sqrt_c2 + s.eps));
}

// 64 random bits for elements 2 k and 2 k + 1 of all tensors' blocks (splitmix64: Steele, Lea, Flood 2014).  Of the
// lower 32 the lower 16 round m of the even element and the upper its v, of the upper 32 those of the odd one.
__device__ __forceinline__ uint64_t hash_pair(uint64_t seed, uint64_t k) {
    uint64_t z = k * 0x9E3779B97F4A7C15ull + seed;
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
// Code of a magnitude, `rnd` of 16 bits: the 20 bits below the code are cut off after rnd / 2^16 of one is added.
__device__ __forceinline__ uint32_t encode(uint32_t bits, uint32_t exponent, int top, uint32_t rnd) {
    const uint32_t mag = bits & 0x7FFFFFFFu, field = mag >> 23;
    const uint32_t whole = (mag & 0x7FFFFFu) | (field ? 0x800000u : 0u);
    const int rel = int(field ? field : 1) - int(exponent) + top;
    const int down = 1 - rel < 31 ? 1 - rel : 31;
    const uint32_t fixed = rel >= 1 ? (uint32_t(rel - 1) << 23) + whole : whole >> down;
    const uint32_t code = (fixed + (rnd << 4)) >> 20, most = top == kTopM ? 127 : 255;
    return exponent == 255 ? 0 : code < most ? code : most;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    for (int d = 32; d; d >>= 1) {
        const uint32_t y = __shfl_xor(x, d);
        x = x > y ? x : y;
    }
    return x;
}

__global__ __launch_bounds__(kThreads) void adamw_step(const Tensor *tensors, const Chunk *chunks, Step s) {
    if (s.skip && *s.skip) return;
    const Chunk c = chunks[blockIdx.x];
    const Tensor &t = tensors[c.tensor];
    const float scale = s.grad_scale ? *s.grad_scale : 1.0f;
    const float decay = float(s.lr * t.weight_decay);
    const int64_t begin = int64_t(c.index) * kChunk;
    const int64_t end = begin + kChunk < t.n ? begin + kChunk : t.n;
    if (t.state == HARP_STATE_F32) {
        float *m = static_cast<float *>(t.m), *v = static_cast<float *>(t.v);
        for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) {
            float p = t.p[i], mi = m[i], vi = v[i];
            update(s, element(t.grad, t.grad_type, i) * scale, decay, p, mi, vi);
            t.p[i] = p;
            m[i] = mi;
            v[i] = vi;
            if (t.copy) put_copy(t.copy, t.copy_type, i, p);
        }
        return;
    }
    uint8_t *m = static_cast<uint8_t *>(t.m), *v = static_cast<uint8_t *>(t.v);
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    for (int64_t at = begin + wave * kBlock; at < end; at += kThreads / kWave * kBlock) {
        const int64_t b = at / kBlock;
        const uint32_t em = t.m_exp[b], ev = t.v_exp[b];
        const float um = block_unit(em, kTopM), uv = block_unit(ev, kTopV);
        float mi[4] = {0, 0, 0, 0}, vi[4] = {0, 0, 0, 0};
        uint32_t most_m = 0, most_v = 0;
        for (int j = 0; j < 4; ++j) {
            const int64_t i = at + 4 * lane + j;
            if (i >= t.n) continue;
            const uint32_t cm = m[i], cv = v[i];
            mi[j] = decode(cm & 127, um);
            if (cm & 128) mi[j] = -mi[j];
            vi[j] = decode(cv, uv);
            float p = t.p[i];
            update(s, element(t.grad, t.grad_type, i) * scale, decay, p, mi[j], vi[j]);
            t.p[i] = p;
            if (t.copy) put_copy(t.copy, t.copy_type, i, p);
            const uint32_t am = __float_as_uint(mi[j]) & 0x7FFFFFFFu, av = __float_as_uint(vi[j]) & 0x7FFFFFFFu;
            most_m = most_m > am ? most_m : am;
            most_v = most_v > av ? most_v : av;
        }
        const uint32_t nm = block_exponent(wave_max(most_m)), nv = block_exponent(wave_max(most_v));
        const uint64_t pair = ((t.first_block + b) * kBlock + 4 * lane) / 2;
        const uint64_t h[2] = {hash_pair(s.seed, pair), hash_pair(s.seed, pair + 1)};
        for (int j = 0; j < 4; ++j) {
            const int64_t i = at + 4 * lane + j;
            if (i >= t.n) continue;
            const uint32_t r = uint32_t(h[j >> 1] >> (32 * (j & 1)));
            const uint32_t bm = __float_as_uint(mi[j]);
            m[i] = uint8_t(encode(bm, nm, kTopM, r & 0xFFFF) | (bm >> 24 & 128));
            v[i] = uint8_t(encode(__float_as_uint(vi[j]), nv, kTopV, r >> 16));
        }
        if (lane == 0) {
            t.m_exp[b] = uint8_t(nm);
            t.v_exp[b] = uint8_t(nv);
        }
    }
}

__global__ __launch_bounds__(kThreads) void adamw_read(const Tensor *tensors, const Chunk *chunks) {
    const Chunk c = chunks[blockIdx.x];
    const Tensor &t = tensors[c.tensor];
    if (t.state != HARP_STATE_8BIT) return;
    const int64_t begin = int64_t(c.index) * kChunk;
    const int64_t end = begin + kChunk < t.n ? begin + kChunk : t.n;
    const uint8_t *m = static_cast<const uint8_t *>(t.m), *v = static_cast<const uint8_t *>(t.v);
    for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) {
        if (t.m_seen) {
            const float x = decode(m[i] & 127, block_unit(t.m_exp[i / kBlock], kTopM));
            t.m_seen[i] = __bf16(m[i] & 128 ? -x : x);
        }
        if (t.v_seen) t.v_seen[i] = __bf16(decode(v[i], block_unit(t.v_exp[i / kBlock], kTopV)));
    }
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
        t[i] = d;
        block += uint64_t(a.n + kBlock - 1) / kBlock;
        for (int64_t k = 0; k * kChunk < a.n; ++k) *c++ = Chunk{uint32_t(i), uint32_t(k)};
    }
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    hipError_t e = hipSetDevice(ctx->device);
    if (e == hipSuccess) e = hipMemcpyAsync(plan_buf, host, y.bytes, hipMemcpyHostToDevice, st);
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
