// Rotary positions: pairs of a head's channels turned by an angle that grows with the token's position, and the frequencies
// of contexts longer than those trained on.
#include <math.h>

#include "harp_ctx.h"
#include "ops_common.h"

using namespace harp;
using namespace harp::ops;

namespace {

struct Rotary {
    int64_t tokens, x_token, x_step, y_token, y_step, first, period;
    int heads, head, turned, inverse;
    float magnitude;
    const double *frequency;
    const int64_t *positions;
};

// Elements of a piece: 16 bytes where the memory takes them in one go.
template <typename T> constexpr int kPiece = int(16 / sizeof(T));
template <typename T> struct Piece { T v[kPiece<T>]; };

// `count` elements from p on, wherever they lie; the rest of the piece is left as it was.
template <typename T> __device__ __forceinline__ void take(Piece<T> &to, const T *p, int count) {
    typedef T Vec __attribute__((ext_vector_type(kPiece<T>)));
    typedef Vec Loose __attribute__((aligned(sizeof(T))));
    if (count >= kPiece<T>) {
        const Vec v = *reinterpret_cast<const Loose *>(p);
#pragma unroll
        for (int k = 0; k < kPiece<T>; ++k) to.v[k] = v[k];
    } else {
        for (int k = 0; k < kPiece<T>; ++k)
            if (k < count) to.v[k] = p[k];
    }
}
template <typename T> __device__ __forceinline__ void put(T *p, const Piece<T> &from, int count) {
    typedef T Vec __attribute__((ext_vector_type(kPiece<T>)));
    typedef Vec Loose __attribute__((aligned(sizeof(T))));
    if (count >= kPiece<T>) {
        Vec v;
#pragma unroll
        for (int k = 0; k < kPiece<T>; ++k) v[k] = from.v[k];
        *reinterpret_cast<Loose *>(p) = v;
    } else {
        for (int k = 0; k < kPiece<T>; ++k)
            if (k < count) p[k] = from.v[k];
    }
}

// A thread takes one piece of pairs of a token (16 bytes of a and of b) through `each` heads, so that an angle is taken once
// for them; threads behind a token's pairs copy its other channels, two pieces each.  Bound by memory: 40 heads of 128 of 4,096
// tokens, 16 bits, read and written in 17.3 us, 4.8 TB/s; one token of 72 heads 4 us, of which most is the angles' functions and
// the launch.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void turn(Rotary r, const T *x, T *y, int pieces, int lanes, int each, int64_t items) {
    constexpr int N = kPiece<T>;
    for (int64_t id = int64_t(blockIdx.x) * 256 + threadIdx.x; id < items; id += int64_t(gridDim.x) * 256) {
        const int64_t group = id / lanes, chunks = (r.heads + each - 1) / each, t = group / chunks;
        const int lane = int(id - group * lanes), h0 = int(group - t * chunks) * each;
        const int h1 = h0 + each < r.heads ? h0 + each : r.heads;
        const T *from = x + t * r.x_token + h0 * r.x_step;
        T *to = y + t * r.y_token + h0 * r.y_step;
        // two pieces of a head: channels at[0] .. and at[1] .., `count` elements of the pair of pieces each
        const bool turning = lane < pieces;
        const int half = r.turned / 2, p0 = lane * N;
        int at[2], count[2];
        if (!turning) {
            at[0] = r.turned + (lane - pieces) * 2 * N;
            at[1] = at[0] + N;
            count[0] = r.head - at[0];
            count[1] = r.head - at[1];
        } else if (INTERLEAVED) {
            at[0] = 2 * p0;
            at[1] = at[0] + N;
            count[0] = r.turned - at[0];
            count[1] = r.turned - at[1];
        } else {
            at[0] = p0;
            at[1] = half + p0;
            count[0] = count[1] = half - p0;
        }
        float c[N], s[N];
        if (turning) {
            const int64_t p = r.positions ? r.positions[t] : r.first + (r.period > 0 ? t % r.period : t);
            const double where = double(p) * 0.15915494309189533577;          // 1 / (2 pi): in turns
#pragma unroll
            for (int k = 0; k < N; ++k) {
                // whole turns are taken off in 64 bits: at 10^6 turns 2^-33 of one is left, under the rounding to 32 bits
                double turns = p0 + k < half ? where * r.frequency[p0 + k] : 0.0;
                turns -= rint(turns);
                sincospif(2.0f * float(turns), &s[k], &c[k]);
                c[k] *= r.magnitude;
                s[k] *= r.inverse ? -r.magnitude : r.magnitude;
            }
        }
        for (int h = h0; h < h1; ++h, from += r.x_step, to += r.y_step) {
            Piece<T> a, b;
            take(a, from + at[0], count[0]);
            take(b, from + at[1], count[1]);
            if (turning) {
                float u[2 * N], w[2 * N];
#pragma unroll
                for (int k = 0; k < N; ++k) u[k] = to_f32(a.v[k]), u[N + k] = to_f32(b.v[k]);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const int i = INTERLEAVED ? 2 * k : k, j = INTERLEAVED ? 2 * k + 1 : N + k;
                    w[i] = u[i] * c[k] - u[j] * s[k];
                    w[j] = u[j] * c[k] + u[i] * s[k];
                }
#pragma unroll
                for (int k = 0; k < N; ++k) a.v[k] = T(w[k]), b.v[k] = T(w[N + k]);
            }
            put(to + at[0], a, count[0]);
            put(to + at[1], b, count[1]);
        }
    }
}

template <typename T> void launch(const harp_ctx *ctx, const harp_rotary_args *g, hipStream_t st) {
    const bool copy = g->X != g->Y && g->turned < g->head;
    const Rotary r = {g->tokens, g->x_token, g->x_step, g->y_token, g->y_step, g->first, g->period, g->heads, g->head, g->turned,
                      g->inverse, g->magnitude, g->frequency, g->positions};
    constexpr int N = kPiece<T>;
    const int pieces = (g->turned / 2 + N - 1) / N, lanes = pieces + (copy ? (g->head - g->turned + 2 * N - 1) / (2 * N) : 0);
    const int64_t threads = g->tokens * lanes * g->heads, fill = int64_t(ctx->n_cu) * 1024;
    int64_t each = threads / fill;
    each = each < 1 ? 1 : each > 8 ? 8 : each;
    const int64_t items = g->tokens * lanes * ((g->heads + each - 1) / each), blocks = (items + 255) / 256;
    const dim3 grid(uint32_t(blocks < (1 << 20) ? blocks : 1 << 20));
    const T *x = static_cast<const T *>(g->X);
    T *y = static_cast<T *>(g->Y);
    if (g->layout == HARP_ROTARY_HALF) turn<T, false><<<grid, dim3(256), 0, st>>>(r, x, y, pieces, lanes, int(each), items);
    else turn<T, true><<<grid, dim3(256), 0, st>>>(r, x, y, pieces, lanes, int(each), items);
}

}  // namespace

extern "C" {

int harp_rotary_frequencies(int32_t turned, double base, int32_t scaling, double factor, double original, double low, double high,
                            double *frequency, float *magnitude) {
    if (turned < 2 || turned % 2 || turned >= 1 << 16) return HARP_ERR_SHAPE;
    if (!frequency || !(base > 0) || !isfinite(base) || scaling < HARP_SCALING_NONE || scaling > HARP_SCALING_BY_PARTS) return HARP_ERR_INVALID_ARG;
    if (scaling != HARP_SCALING_NONE && (!(factor >= 1) || !isfinite(factor))) return HARP_ERR_INVALID_ARG;
    if (scaling == HARP_SCALING_NTK && turned == 2) return HARP_ERR_SHAPE;      // its one pair does not know the base
    if (scaling == HARP_SCALING_BY_PARTS && (!(original > 0) || !(low < high) || !isfinite(original) || !isfinite(low) || !isfinite(high)))
        return HARP_ERR_INVALID_ARG;
    if (scaling == HARP_SCALING_NTK) base *= pow(factor, double(turned) / (turned - 2));
    for (int i = 0; i < turned / 2; ++i) {
        double f = pow(base, -2.0 * i / turned);
        if (scaling == HARP_SCALING_LINEAR) f /= factor;
        if (scaling == HARP_SCALING_BY_PARTS) {
            double g = (original * f / 6.283185307179586477 - low) / (high - low);
            g = g < 0 ? 0 : g > 1 ? 1 : g;
            f *= (1 - g) / factor + g;
        }
        frequency[i] = f;
    }
    if (magnitude) *magnitude = scaling == HARP_SCALING_BY_PARTS ? float(0.1 * log(factor) + 1) : 1.0f;
    return HARP_OK;
}

int harp_rotary(harp_ctx *ctx, const harp_rotary_args *g, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    if (g->tokens < 0 || g->tokens >= int64_t(1) << 31 || g->heads < 1 || g->heads >= 1 << 16 || g->head < 2 || g->head >= 1 << 16 ||
        g->turned < 2 || g->turned > g->head || g->turned % 2)
        return fail(ctx, HARP_ERR_SHAPE, "0 <= tokens < 2^31, 1 <= heads < 2^16 and an even 2 <= turned <= head < 2^16 are wanted");
    const size_t element = size_t(type_bytes(g->type));
    if (!element) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown type");
    if (g->layout != HARP_ROTARY_HALF && g->layout != HARP_ROTARY_INTERLEAVED) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown layout");
    if (!g->frequency) return fail(ctx, HARP_ERR_INVALID_ARG, "null frequency");
    if (!aligned(g->frequency, 8) || !aligned(g->positions, 8)) return fail(ctx, HARP_ERR_INVALID_ARG, "frequency or positions are not aligned to 8 bytes");
    if (g->period < 0) return fail(ctx, HARP_ERR_INVALID_ARG, "a period below 0");
    if (g->tokens == 0) return HARP_OK;
    if (!g->X || !g->Y) return fail(ctx, HARP_ERR_INVALID_ARG, "null X or Y");
    if (!aligned(g->X, element) || !aligned(g->Y, element)) return fail(ctx, HARP_ERR_INVALID_ARG, "X or Y is not aligned to its elements");
    const int64_t far = int64_t(1) << 40;
    if (g->x_token < 0 || g->x_step < 0 || g->y_token < 0 || g->y_step < 0 || g->x_token > far || g->x_step > far || g->y_token > far || g->y_step > far)
        return fail(ctx, HARP_ERR_SHAPE, "distances must be in 0 .. 2^40");
    if (!clear_of_each_other(g->tokens, g->heads, g->head, g->y_token, g->y_step)) return fail(ctx, HARP_ERR_SHAPE, "Y: elements lie over each other");
    if (g->X == g->Y && ((g->tokens > 1 && g->x_token != g->y_token) || (g->heads > 1 && g->x_step != g->y_step)))
        return fail(ctx, HARP_ERR_SHAPE, "Y is X with other distances");
    const hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_F32) launch<float>(ctx, g, st);
    else if (g->type == HARP_BF16) launch<__bf16>(ctx, g, st);
    else launch<_Float16>(ctx, g, st);
    const hipError_t launched = hipGetLastError();
    return launched == hipSuccess ? HARP_OK : hip_fail(ctx, launched, "launching the rotation");
}

}  // extern "C"
