// Norm after a block, gate, residual scale, residual sum and the norm before the next block, forward and backward,
// and their C entry points.
//
// A row's channels lie in the registers of one workgroup, eight to a thread, so that every tensor is read once and
// written once: the pass is bound by memory.  A workgroup takes rows in turn and keeps what belongs to its channels
// (weights, biases, scale, and in the backward pass the sums over rows) in registers throughout.
#include <math.h>

#include "harp_ctx.h"
#include "ops_common.h"

using namespace harp;
using namespace harp::ops;

namespace {

constexpr int kPer = 8;                               // channels a thread holds
constexpr int kMaxThreads = HARP_NORM_MAX_COLS / kPer;
constexpr int kMaxWaves = kMaxThreads / kWave;
constexpr int kSums = 5;                              // column sums in 32 bits: dw_after, db_after, dscale, dw_before, db_before

// Everything but the data, as the kernels see it.
struct Form {
    int64_t rows, rows_per_gate, ldgate;
    int32_t cols, after, before, gate_act;
    float eps_after, eps_before;
    const float *w_after, *b_after, *w_before, *b_before, *scale;
    const void *gate;
};

// The channels of thread t: 8 t .. 8 t + 7 where rows can be read in wide pieces, else t, t + blockDim, ...
template <bool WIDE> __device__ __forceinline__ int channel(int j) {
    return WIDE ? int(threadIdx.x) * kPer + j : int(threadIdx.x) + j * int(blockDim.x);
}

template <typename T, bool WIDE> __device__ __forceinline__ void load_row(const T *row, int cols, float (&v)[kPer]) {
    if (WIDE) {
        const bool in = int(threadIdx.x) * kPer < cols;
        for (int k = 0; k < kPer; k += 4) {
            const f32x4 q = in ? load4(row + channel<WIDE>(k)) : f32x4{0, 0, 0, 0};
            for (int j = 0; j < 4; ++j) v[k + j] = q[j];
        }
    } else {
        for (int j = 0; j < kPer; ++j) v[j] = channel<WIDE>(j) < cols ? to_f32(row[channel<WIDE>(j)]) : 0.0f;
    }
}
template <typename T, bool WIDE> __device__ __forceinline__ void store_row(T *row, int cols, const float (&v)[kPer]) {
    if (WIDE) {
        if (int(threadIdx.x) * kPer < cols)
            for (int k = 0; k < kPer; k += 4) store4(row + channel<WIDE>(k), f32x4{v[k], v[k + 1], v[k + 2], v[k + 3]});
    } else {
        for (int j = 0; j < kPer; ++j)
            if (channel<WIDE>(j) < cols) row[channel<WIDE>(j)] = T(v[j]);
    }
}
// A vector over the channels, `other` where there is none.
template <bool WIDE> __device__ __forceinline__ void load_vector(const float *p, int cols, float other, float (&v)[kPer]) {
    for (int j = 0; j < kPer; ++j) v[j] = p && channel<WIDE>(j) < cols ? p[channel<WIDE>(j)] : other;
}

// N sums over the workgroup, the same in every thread.  `turn` alternates between two buffers, so that one barrier a
// round is enough: a buffer is written again only after everybody has passed the next round's barrier.
template <int N> __device__ __forceinline__ void block_sum(float (&v)[N], float (*buf)[kMaxWaves][4], int &turn) {
    for (int k = 0; k < N; ++k)
        for (int d = 32; d; d >>= 1) v[k] += __shfl_xor(v[k], d);
    const int waves = blockDim.x / kWave;
    if (waves == 1) return;
    float(*b)[4] = buf[turn];
    turn ^= 1;
    if (threadIdx.x % kWave == 0)
        for (int k = 0; k < N; ++k) b[threadIdx.x / kWave][k] = v[k];
    __syncthreads();
    for (int k = 0; k < N; ++k) v[k] = 0;
    for (int w = 0; w < waves; ++w)
        for (int k = 0; k < N; ++k) v[k] += b[w][k];
}

__device__ __forceinline__ float sigmoid(float x) { return 1.0f / (1.0f + __expf(-x)); }

// v - mean (LAYER), and 1 / sqrt(mean of squares + eps) of what is left.  Channels beyond cols stay 0.
template <bool WIDE>
__device__ __forceinline__ float center(float (&v)[kPer], int kind, int cols, float eps, float (*buf)[kMaxWaves][4], int &turn) {
    if (kind == HARP_NORM_LAYER) {
        float s[1] = {0};
        for (int j = 0; j < kPer; ++j) s[0] += v[j];
        block_sum(s, buf, turn);
        const float mean = s[0] / float(cols);
        for (int j = 0; j < kPer; ++j)
            if (channel<WIDE>(j) < cols) v[j] -= mean;
    }
    float s[1] = {0};
    for (int j = 0; j < kPer; ++j) s[0] += v[j] * v[j];
    block_sum(s, buf, turn);
    return 1.0f / sqrtf(s[0] / float(cols) + eps);
}

template <typename T, bool WIDE>
__global__ __launch_bounds__(kMaxThreads) void norm_forward(Form f, const T *x, int64_t ldx, const T *y, int64_t ldy, T *h,
                                                            int64_t ldh, T *z, int64_t ldz) {
    __shared__ float buf[2][kMaxWaves][4];
    int turn = 0;
    const int cols = f.cols;
    float wa[kPer], ba[kPer], wb[kPer], bb[kPer], sc[kPer];
    load_vector<WIDE>(f.w_after, cols, 1.0f, wa);
    load_vector<WIDE>(f.b_after, cols, 0.0f, ba);
    load_vector<WIDE>(f.w_before, cols, 1.0f, wb);
    load_vector<WIDE>(f.b_before, cols, 0.0f, bb);
    load_vector<WIDE>(f.scale, cols, 1.0f, sc);
    for (int64_t r = blockIdx.x; r < f.rows; r += gridDim.x) {
        float a[kPer], v[kPer];
        if (y) {
            load_row<T, WIDE>(y + r * ldy, cols, v);
            if (x) load_row<T, WIDE>(x + r * ldx, cols, a);
            if (f.after != HARP_NORM_NONE) {
                const float rstd = center<WIDE>(v, f.after, cols, f.eps_after, buf, turn);
                for (int j = 0; j < kPer; ++j) v[j] = v[j] * rstd * wa[j] + ba[j];
            }
            if (f.gate) {
                float g[kPer];
                load_row<T, WIDE>(static_cast<const T *>(f.gate) + r / f.rows_per_gate * f.ldgate, cols, g);
                for (int j = 0; j < kPer; ++j) v[j] *= f.gate_act == HARP_GATE_SIGMOID ? sigmoid(g[j]) : g[j];
            }
            for (int j = 0; j < kPer; ++j) v[j] = channel<WIDE>(j) < cols ? v[j] * sc[j] : 0.0f;
            if (x)
                for (int j = 0; j < kPer; ++j) v[j] += a[j];
            if (h) store_row<T, WIDE>(h + r * ldh, cols, v);
        } else {
            load_row<T, WIDE>(x + r * ldx, cols, v);
        }
        if (f.before != HARP_NORM_NONE) {
            const float rstd = center<WIDE>(v, f.before, cols, f.eps_before, buf, turn);
            for (int j = 0; j < kPer; ++j) v[j] = v[j] * rstd * wb[j] + bb[j];
            store_row<T, WIDE>(z + r * ldz, cols, v);
        }
    }
}

// How rows are dealt to workgroups in the backward pass: slabs of rows of which none reaches into a gate's group
// without holding it whole or lying inside it, so that a group's sum is either a workgroup's own or a sum of
// workgroups' partial sums.
struct Slabs {
    int64_t rows;             // rows of a slab
    int64_t per_group;        // slabs of a gate's group, 0: a slab holds whole groups (or there is no gate)
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

template <typename T, bool WIDE>
__global__ __launch_bounds__(kMaxThreads) void norm_backward(Form f, Slabs slabs, const T *dh, int64_t lddh, const T *dz, int64_t lddz,
                                                             const T *h, int64_t ldh, const T *y, int64_t ldy, T *dx, int64_t lddx,
                                                             T *dy, int64_t lddy, T *dgate, int64_t lddgate, float *partial,
                                                             float *gate_partial) {
    __shared__ float buf[2][kMaxWaves][4];
    int turn = 0;
    const int cols = f.cols;
    const float inv_cols = 1.0f / float(cols);
    float wa[kPer], ba[kPer], wb[kPer], sc[kPer];
    load_vector<WIDE>(f.w_after, cols, 1.0f, wa);
    load_vector<WIDE>(f.b_after, cols, 0.0f, ba);
    load_vector<WIDE>(f.w_before, cols, 1.0f, wb);
    load_vector<WIDE>(f.scale, cols, 1.0f, sc);
    float sum[kSums][kPer] = {}, dg[kPer] = {};
    int64_t begin, end;
    slab_rows(slabs, f.rows, blockIdx.x, begin, end);
    for (int64_t r = begin; r < end; ++r) {
        float d[kPer];                                   // D, the gradient of h
        if (dh) load_row<T, WIDE>(dh + r * lddh, cols, d);
        else for (int j = 0; j < kPer; ++j) d[j] = 0;
        if (dz) {
            float a[kPer], e[kPer];
            load_row<T, WIDE>(h + r * ldh, cols, a);
            load_row<T, WIDE>(dz + r * lddz, cols, e);
            const float rstd = center<WIDE>(a, f.before, cols, f.eps_before, buf, turn);
            float c[2] = {0, 0};
            for (int j = 0; j < kPer; ++j) {
                sum[3][j] += e[j] * (a[j] * rstd);
                sum[4][j] += e[j];
                e[j] *= wb[j];
                c[0] += e[j];
                c[1] += e[j] * a[j];
            }
            block_sum(c, buf, turn);
            for (int j = 0; j < kPer; ++j) d[j] += through(e[j], a[j], rstd, c[0], c[1], f.before, inv_cols);
        }
        if (dx) store_row<T, WIDE>(dx + r * lddx, cols, d);
        if (!y) continue;
        float a[kPer], g[kPer];
        load_row<T, WIDE>(y + r * ldy, cols, a);
        float rstd = 1.0f;
        if (f.after != HARP_NORM_NONE) rstd = center<WIDE>(a, f.after, cols, f.eps_after, buf, turn);
        if (f.gate) load_row<T, WIDE>(static_cast<const T *>(f.gate) + r / f.rows_per_gate * f.ldgate, cols, g);
        float c[2] = {0, 0};
        for (int j = 0; j < kPer; ++j) {
            if (channel<WIDE>(j) >= cols) d[j] = 0;
            const float hat = a[j] * rstd, t = hat * wa[j] + ba[j];
            float factor = 1.0f, slope = 1.0f;
            if (f.gate) {
                factor = g[j];
                if (f.gate_act == HARP_GATE_SIGMOID) {
                    factor = sigmoid(g[j]);
                    slope = factor * (1.0f - factor);
                }
                dg[j] += d[j] * t * sc[j] * slope;
            }
            sum[2][j] += d[j] * t * factor;
            d[j] *= factor * sc[j];
            sum[0][j] += d[j] * hat;
            sum[1][j] += d[j];
            d[j] *= wa[j];
            c[0] += d[j];
            c[1] += d[j] * a[j];
        }
        if (f.after != HARP_NORM_NONE) {
            block_sum(c, buf, turn);
            for (int j = 0; j < kPer; ++j) d[j] = through(d[j], a[j], rstd, c[0], c[1], f.after, inv_cols);
        }
        if (dy) store_row<T, WIDE>(dy + r * lddy, cols, d);
        if (dgate && slabs.per_group == 0 && (r + 1 == f.rows || (r + 1) % f.rows_per_gate == 0)) {
            store_row<T, WIDE>(dgate + r / f.rows_per_gate * lddgate, cols, dg);
            for (int j = 0; j < kPer; ++j) dg[j] = 0;
        }
    }
    for (int j = 0; j < kPer; ++j) {
        const int c = channel<WIDE>(j);
        if (c >= cols) continue;
        for (int k = 0; k < kSums; ++k) partial[(int64_t(blockIdx.x) * kSums + k) * cols + c] = sum[k][j];
        if (gate_partial) gate_partial[int64_t(blockIdx.x) * cols + c] = dg[j];
    }
}

// The slabs' partial sums to one vector each, in the slabs' order; one thread a channel.
struct Sums { float *out[kSums]; };
__global__ __launch_bounds__(256) void norm_sums(const float *partial, int64_t count, int cols, Sums sums, int accumulate) {
    const int c = blockIdx.x * 256 + threadIdx.x, k = blockIdx.y;
    if (c >= cols || !sums.out[k]) return;
    float s = 0;
    for (int64_t i = 0; i < count; ++i) s += partial[(i * kSums + k) * cols + c];
    sums.out[k][c] = accumulate ? sums.out[k][c] + s : s;
}
template <typename T>
__global__ __launch_bounds__(256) void gate_sums(const float *partial, int64_t per_group, int cols, T *dgate, int64_t lddgate,
                                                 int64_t first_group) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    const int64_t group = first_group + blockIdx.y;
    if (c >= cols) return;
    float s = 0;
    for (int64_t i = 0; i < per_group; ++i) s += partial[(group * per_group + i) * cols + c];
    dgate[group * lddgate + c] = T(s);
}

int threads_for(int cols) { return int(round_up(size_t((cols + kPer - 1) / kPer), kWave)); }

// As many workgroups as are resident: 1,024 threads a compute unit in the backward pass (it takes about 128 registers).
Slabs slabs_for(const harp_ctx *ctx, const harp_norm *n) {
    Slabs s;
    const int64_t want = int64_t(ctx->n_cu) * (kMaxThreads / threads_for(n->cols) < 16 ? kMaxThreads / threads_for(n->cols) : 16);
    s.rows = (n->rows + want - 1) / want;
    if (s.rows < 1) s.rows = 1;
    s.per_group = 0;
    s.rows_per_group = n->gate ? n->rows_per_gate : n->rows;
    if (n->gate && n->rows > 0) {
        const int64_t per = n->rows_per_gate < n->rows ? n->rows_per_gate : n->rows;
        if (per <= s.rows) {
            s.rows = s.rows / per * per;
        } else {
            s.rows_per_group = per;
            s.per_group = (per + s.rows - 1) / s.rows;
            s.rows = (per + s.per_group - 1) / s.per_group;
            s.count = (n->rows + per - 1) / per * s.per_group;
            return s;
        }
    }
    s.count = (n->rows + s.rows - 1) / s.rows;
    return s;
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
    return Form{n->rows, n->gate ? n->rows_per_gate : 1, n->ldgate, n->cols, n->after, n->before, n->gate_act, n->eps_after, n->eps_before,
                n->w_after, n->b_after, n->w_before, n->b_before, n->scale, n->gate};
}

template <typename T, bool WIDE>
void run_forward(const harp_ctx *ctx, const harp_norm *n, const void *x, int64_t ldx, const void *y, int64_t ldy, void *h, int64_t ldh,
                 void *z, int64_t ldz, hipStream_t st) {
    const int threads = threads_for(n->cols);
    const int64_t most = int64_t(ctx->n_cu) * (2048 / threads < 16 ? 2048 / threads : 16);
    norm_forward<T, WIDE><<<dim3(uint32_t(n->rows < most ? n->rows : most)), dim3(threads), 0, st>>>(
        form_of(n), static_cast<const T *>(x), ldx, static_cast<const T *>(y), ldy, static_cast<T *>(h), ldh, static_cast<T *>(z), ldz);
}

template <typename T, bool WIDE>
void run_backward(const harp_norm *n, const harp_norm_grads *g, const Slabs &s, float *partial, hipStream_t st) {
    const int threads = threads_for(n->cols);
    float *gate_partial = s.per_group && g->dgate ? partial + s.count * kSums * n->cols : nullptr;
    if (s.count > 0)
        norm_backward<T, WIDE><<<dim3(uint32_t(s.count)), dim3(threads), 0, st>>>(
            form_of(n), s, static_cast<const T *>(g->dh), g->lddh, static_cast<const T *>(g->dz), g->lddz,
            static_cast<const T *>(g->h), g->ldh, static_cast<const T *>(g->y), g->ldy, static_cast<T *>(g->dx), g->lddx,
            static_cast<T *>(g->dy), g->lddy, static_cast<T *>(g->dgate), g->lddgate, partial, gate_partial);
    const uint32_t across = uint32_t((n->cols + 255) / 256);
    const Sums sums = {{g->dw_after, g->db_after, g->dscale, g->dw_before, g->db_before}};
    bool any = false;
    for (int k = 0; k < kSums; ++k) any = any || sums.out[k];
    if (any) norm_sums<<<dim3(across, kSums), dim3(256), 0, st>>>(partial, s.count, n->cols, sums, g->accumulate);
    if (gate_partial) {
        const int64_t groups = s.count / s.per_group;
        for (int64_t first = 0; first < groups; first += 65535)
            gate_sums<T><<<dim3(across, uint32_t(groups - first < 65535 ? groups - first : 65535)), dim3(256), 0, st>>>(
                gate_partial, s.per_group, n->cols, static_cast<T *>(g->dgate), g->lddgate, first);
    }
}

size_t workspace_for(const harp_ctx *ctx, const harp_norm *n) {
    const Slabs s = slabs_for(ctx, n);
    return round_up(size_t(s.count) * (kSums + (s.per_group ? 1 : 0)) * size_t(n->cols) * 4, 256) + 256;
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
