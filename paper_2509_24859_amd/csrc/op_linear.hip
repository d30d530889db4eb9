// Matrix product with bias, activation and residual in its epilogue, its gradients, and their C entry points.
//
// The three products are one form, D[p][q] = sum over r of A(p, r) B(q, r):
//   forward          p = token,  q = output,  r = input     A = X, B = W, both with r contiguous
//   input gradient   p = token,  q = input,   r = output    A = dY, r contiguous; B = W, q contiguous
//   weight gradient  p = output, q = input,   r = token     A = dY, B = X, p and q contiguous
#include "op_product.h"

namespace {

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

size_t most(size_t a, size_t b) { return a > b ? a : b; }
// Both operands packed, and shares of r or column sums.
size_t workspace_for(const harp_ctx *ctx, int64_t M, int64_t N, int64_t K) {
    const size_t x = packed_bytes(M, K), w = packed_bytes(N, K), dy = packed_bytes(M, N);
    const size_t forward = x + w + partial_bytes(ctx, kForward, M, N, K);
    const size_t input = dy + w + partial_bytes(ctx, kInput, M, K, N);
    const size_t weight = dy + x + most(partial_bytes(ctx, kWeight, N, K, M), round_up(size_t(slabs_of(M)) * size_t(N) * 4, 256));
    return most(most(forward, input), weight) + 256;
}

int check(harp_ctx *ctx, int64_t M, int64_t N, int64_t K, int type, int act, const Matrix *m, int count, const void *workspace,
          size_t workspace_bytes) {
    if (!sizes_fit(M, N, K)) return fail(ctx, HARP_ERR_SHAPE, "0 <= M < 2^31 and 1 <= N, K < 2^22 are wanted");
    const int rc = check_operands(ctx, type, act, m, count);
    if (rc != HARP_OK) return rc;
    const size_t need = workspace_for(ctx, M, N, K);
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
        return fail(ctx, HARP_ERR_WORKSPACE, "the workspace needs %zu bytes, aligned to 256", need);
    const hipError_t e = hipSetDevice(ctx->device);
    if (e != hipSuccess) return hip_fail(ctx, e, "hipSetDevice");
    return HARP_OK;
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
    e.past = passes_the_caches(P, Q, e.out_f32 ? 4 : 2);
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
