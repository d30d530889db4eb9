// Matrix product with bias, activation and residual in its epilogue, its gradients, and their C entry points.
//
// The three products are one form, D[p][q] = sum over r of A(p, r) B(q, r):
//   forward          p = token,  q = output,  r = input     A = X, B = W, both with r contiguous
//   input gradient   p = token,  q = input,   r = output    A = dY, r contiguous; B = W, q contiguous
//   weight gradient  p = output, q = input,   r = token     A = dY, B = X, p and q contiguous
#include <math.h>

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

// x / (1 + exp(-x)) and the like by way of the logistic function: a quotient of hardware reciprocal and exponential,
// within a few units of 2^-24, where results are rounded to 2^-8 or 2^-11.
__device__ __forceinline__ float logistic(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
constexpr float kTanhA = 1.5957691216057308f;             // 2 sqrt(2 / pi): (1 + tanh(u)) / 2 = logistic(2 u)
constexpr float kTanhB = 0.044715f;

__device__ __forceinline__ float activate(float z, int act) {
    switch (act) {
        case HARP_ACT_RELU: return z > 0 ? z : z != z ? z : 0.0f;
        case HARP_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678f));
        case HARP_ACT_GELU_TANH: return z * logistic(kTanhA * z * (1.0f + kTanhB * z * z));
        case HARP_ACT_SILU: return z * logistic(z);
        default: return z;
    }
}
__device__ __forceinline__ float slope(float z, int act) {
    switch (act) {
        case HARP_ACT_RELU: return z > 0 ? 1.0f : 0.0f;
        case HARP_ACT_GELU: return 0.5f * (1.0f + erff(z * 0.70710678f)) + z * 0.39894228f * __expf(-0.5f * z * z);
        case HARP_ACT_GELU_TANH: {
            const float s = logistic(kTanhA * z * (1.0f + kTanhB * z * z));
            return s + z * s * (1.0f - s) * kTanhA * (1.0f + 3.0f * kTanhB * z * z);
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

// A(p, r) = a[p * row + r * col].
template <typename T> struct Operand { const T *a; int64_t row, col; };

constexpr int kTile = 64, kDeep = 32, kPitch = kDeep + 8;

// Four wavefronts on a tile of 64 x 64, each 32 x 32; elements are staged one by one, so any stride and size will do.
template <typename T>
__global__ __launch_bounds__(256) void product(Operand<T> a, Operand<T> b, int64_t P, int64_t Q, int64_t R, Epilogue e) {
    __shared__ __align__(16) T la[kTile * kPitch], lb[kTile * kPitch];
    const int64_t p0 = int64_t(blockIdx.y) * kTile, q0 = int64_t(blockIdx.x) * kTile;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int wp = wave / 2 * 32, wq = wave % 2 * 32;
    f32x4 acc[2][2] = {};
    for (int64_t r0 = 0; r0 < R; r0 += kDeep) {
        for (int i = threadIdx.x; i < kTile * kDeep; i += 256) {
            const int pa = a.col == 1 ? i / kDeep : i % kTile, ra = a.col == 1 ? i % kDeep : i / kTile;
            la[pa * kPitch + ra] = p0 + pa < P && r0 + ra < R ? a.a[(p0 + pa) * a.row + (r0 + ra) * a.col] : T(0.0f);
            const int qb = b.col == 1 ? i / kDeep : i % kTile, rb = b.col == 1 ? i % kDeep : i / kTile;
            lb[qb * kPitch + rb] = q0 + qb < Q && r0 + rb < R ? b.a[(q0 + qb) * b.row + (r0 + rb) * b.col] : T(0.0f);
        }
        __syncthreads();
        typename Mfma<T>::Frag fa[2], fb[2];
        for (int i = 0; i < 2; ++i) {
            fa[i] = *reinterpret_cast<const typename Mfma<T>::Frag *>(la + (wp + 16 * i + lane % 16) * kPitch + 8 * (lane / 16));
            fb[i] = *reinterpret_cast<const typename Mfma<T>::Frag *>(lb + (wq + 16 * i + lane % 16) * kPitch + 8 * (lane / 16));
        }
        // the q operand first: a lane then holds four neighbouring q of one p
        for (int i = 0; i < 2; ++i)
            for (int j = 0; j < 2; ++j) acc[i][j] = Mfma<T>::run(fb[j], fa[i], acc[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 2; ++i)
        for (int j = 0; j < 2; ++j)
            for (int k = 0; k < 4; ++k) {
                const int64_t p = p0 + wp + 16 * i + lane % 16, q = q0 + wq + 16 * j + 4 * (lane / 16) + k;
                if (p < P && q < Q) finish<T>(e, p, q, acc[i][j][k]);
            }
}

// Column sums of dY: partial sums of slabs of rows, then the slabs in order.
constexpr int kSumRows = 256;
template <typename T>
__global__ __launch_bounds__(256) void column_sums(const T *dy, int64_t ld, int64_t M, int64_t N, float *partial) {
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= N) return;
    const int64_t begin = int64_t(blockIdx.y) * kSumRows, end = begin + kSumRows < M ? begin + kSumRows : M;
    float s = 0;
    for (int64_t m = begin; m < end; ++m) s += to_f32(dy[m * ld + n]);
    partial[int64_t(blockIdx.y) * N + n] = s;
}
__global__ __launch_bounds__(256) void column_join(const float *partial, int64_t count, int64_t N, float *out, int accumulate) {
    const int64_t n = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (n >= N) return;
    float s = 0;
    for (int64_t i = 0; i < count; ++i) s += partial[i * N + n];
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

bool sizes_fit(int64_t M, int64_t N, int64_t K) {
    const int64_t most = int64_t(1) << 31;
    return M >= 0 && N >= 1 && K >= 1 && M < most && N < most && K < most;
}

size_t workspace_for(int64_t M, int64_t N, int64_t) { return round_up(size_t(slabs_of(M)) * size_t(N) * 4, 256) + 256; }

struct Matrix { const char *name; const void *p; int64_t ld, cols; size_t element; bool needed; };

int check(harp_ctx *ctx, int64_t M, int64_t N, int64_t K, int type, int act, const Matrix *m, int count, const void *workspace,
          size_t workspace_bytes) {
    if (!sizes_fit(M, N, K)) return fail(ctx, HARP_ERR_SHAPE, "M >= 0 and N, K >= 1 are wanted, each below 2^31");
    if (type != HARP_BF16 && type != HARP_F16) return fail(ctx, HARP_ERR_INVALID_ARG, "type must be HARP_BF16 or HARP_F16");
    if (act < HARP_ACT_NONE || act > HARP_ACT_SILU) return fail(ctx, HARP_ERR_INVALID_ARG, "unknown activation");
    for (int i = 0; i < count; ++i) {
        if (!m[i].p && m[i].needed) return fail(ctx, HARP_ERR_INVALID_ARG, "null %s", m[i].name);
        if (!m[i].p) continue;
        if (m[i].ld < m[i].cols) return fail(ctx, HARP_ERR_SHAPE, "%s: leading dimension below its columns", m[i].name);
        if (!aligned(m[i].p, m[i].element)) return fail(ctx, HARP_ERR_INVALID_ARG, "%s is not aligned to its elements", m[i].name);
    }
    const size_t need = workspace_for(M, N, K);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
        return fail(ctx, HARP_ERR_WORKSPACE, "the workspace needs %zu bytes, aligned to 256", need);
    const hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    return HARP_OK;
}

template <typename T>
void launch_product(const void *a, int64_t a_row, int64_t a_col, const void *b, int64_t b_row, int64_t b_col, int64_t P, int64_t Q,
                    int64_t R, const Epilogue &e, hipStream_t st) {
    const Operand<T> oa = {static_cast<const T *>(a), a_row, a_col}, ob = {static_cast<const T *>(b), b_row, b_col};
    product<T><<<dim3(uint32_t((Q + kTile - 1) / kTile), uint32_t((P + kTile - 1) / kTile)), dim3(256), 0, st>>>(oa, ob, P, Q, R, e);
}

int launched(harp_ctx *ctx) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HARP_OK : hip_fail(ctx, e, "launching the product's kernels");
}

}  // namespace

extern "C" {

size_t harp_linear_workspace_bytes(harp_ctx *ctx, int64_t M, int64_t N, int64_t K) {
    return ctx && sizes_fit(M, N, K) ? workspace_for(M, N, K) : 0;
}

int harp_linear_forward(harp_ctx *ctx, const harp_linear *g, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    const bool some = g->M > 0;
    const Matrix m[] = {{"X", g->X, g->ldx, g->K, 2, some}, {"W", g->W, g->ldw, g->K, 2, true}, {"bias", g->bias, g->N, g->N, 2, false},
                        {"residual", g->residual, g->ldr, g->N, 2, false}, {"Y", g->Y, g->ldy, g->N, 2, some}, {"Z", g->Z, g->ldz, g->N, 2, false}};
    const int rc = check(ctx, g->M, g->N, g->K, g->type, g->act, m, 6, workspace, workspace_bytes);
    if (rc != HARP_OK || !some) return rc;
    const Epilogue e = {kForward, g->act, 0, 0, g->Y, g->bias, g->residual, nullptr, g->Z, g->ldy, g->ldr, g->ldz};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) launch_product<__bf16>(g->X, g->ldx, 1, g->W, g->ldw, 1, g->M, g->N, g->K, e, st);
    else launch_product<_Float16>(g->X, g->ldx, 1, g->W, g->ldw, 1, g->M, g->N, g->K, e, st);
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
    const Epilogue e = {kInput, g->act, 0, 0, g->dX, nullptr, g->residual, g->Z, nullptr, g->lddx, g->ldr, g->ldz};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) launch_product<__bf16>(g->dY, g->lddy, 1, g->W, 1, g->ldw, g->M, g->K, g->N, e, st);
    else launch_product<_Float16>(g->dY, g->lddy, 1, g->W, 1, g->ldw, g->M, g->K, g->N, e, st);
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
    const Epilogue e = {kWeight, HARP_ACT_NONE, g->accumulate, g->dw_type == HARP_F32, g->dW, nullptr, nullptr, nullptr, nullptr, g->lddw, 0, 0};
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) launch_product<__bf16>(g->dY, 1, g->lddy, g->X, 1, g->ldx, g->N, g->K, g->M, e, st);
    else launch_product<_Float16>(g->dY, 1, g->lddy, g->X, 1, g->ldx, g->N, g->K, g->M, e, st);
    if (g->dbias) {
        float *partial = static_cast<float *>(workspace);
        const uint32_t across = uint32_t((g->N + 255) / 256);
        const int64_t slabs = slabs_of(g->M);
        if (some) {
            if (g->type == HARP_BF16) column_sums<__bf16><<<dim3(across, uint32_t(slabs)), dim3(256), 0, st>>>(static_cast<const __bf16 *>(g->dY), g->lddy, g->M, g->N, partial);
            else column_sums<_Float16><<<dim3(across, uint32_t(slabs)), dim3(256), 0, st>>>(static_cast<const _Float16 *>(g->dY), g->lddy, g->M, g->N, partial);
        }
        column_join<<<dim3(across), dim3(256), 0, st>>>(partial, slabs, g->N, g->dbias, g->accumulate);
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
