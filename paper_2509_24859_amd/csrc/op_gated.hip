// The first half of a gated MLP block, H = act(X Wg^T + bg) * (X Wu^T + bu), the way back through it, and their C entry points.
//
// Wg and Wu are the two halves of one matrix W [2 F][K], Z [M][2 F] = X W^T + bias likewise.  Forward a workgroup makes the
// same columns of both halves, so that neither half's sums leave the registers before they are multiplied; back, the product
// dH = dY W2 takes Z in its epilogue and stores both halves of dZ.  dX and dW are then plain products of dZ (harp_linear).
//
// 4,096 tokens, W [24576][4096], bfloat16, SiLU, Z kept: 656 to 680 us, 1,210 to 1,257 TFLOP/s (a library product of these sizes
// alone reaches 1,457); without the way through one kernel, Z would be written and read again, 600 MB, 120 us.  Back through W2
// [4096][12288] and the gate with H made again: 425 us, 970 TFLOP/s.  One token: 32 us in the kernel, 6.3 TB/s of weights, which the last cache
// partly holds (1 to 4 GiB of them: 5.3 to 5.7 TB/s).  What bounds
// the tiles is what bounds harp_linear's: bringing operands into LDS, and the epilogue's stores.
#include "op_product.h"

namespace {

// Shares of r that several workgroups summed up apart, in their order, and the epilogue.  FORM kGatedForward: of both halves.
template <typename T, int FORM>
__global__ __launch_bounds__(256) void gated_join(const float *partial, int shares, int64_t P, Gated e) {
    const int64_t across = (e.F + 3) / 4, Q = FORM == kGatedForward ? 2 * e.F : e.F;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < P * across; i += int64_t(gridDim.x) * 256) {
        const int64_t p = i / across, q = i % across * 4;
        auto sum = [&](const float *at) {
            f32x4 d = {0, 0, 0, 0};
            if (q + 4 <= e.F) {
#pragma unroll 4
                for (int s = 0; s < shares; ++s) d += load4(at + s * P * Q);
            } else {
                for (int s = 0; s < shares; ++s)
                    for (int k = 0; k < 4; ++k)
                        if (q + k < e.F) d[k] += at[s * P * Q + k];
            }
            return d;
        };
        const float *at = partial + p * Q + q;
        if (FORM == kGatedForward) gated4<T>(e, p, q, sum(at), sum(at + e.F), e.act);
        else gated_back<T>(e, p, q, sum(at), e.act);
    }
}

// dH as it is given, through the gate.  Four columns a thread.
template <typename T> __global__ __launch_bounds__(256) void gate_grad(const T *dh, int64_t ld, int64_t M, Gated e) {
    const int64_t across = (e.F + 3) / 4;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < M * across; i += int64_t(gridDim.x) * 256) {
        const int64_t p = i / across, q = i % across * 4;
        f32x4 d = {0, 0, 0, 0};
        if (q + 4 <= e.F) {
            d = load4(dh + p * ld + q);
        } else {
            for (int k = 0; k < 4; ++k)
                if (q + k < e.F) d[k] = to_f32(dh[p * ld + q + k]);
        }
        gated_back<T>(e, p, q, d, e.act);
    }
}

constexpr int64_t kMostWidth = int64_t(1) << 21;
bool gated_sizes_fit(int64_t M, int64_t F, int64_t K) { return F >= 1 && F < kMostWidth && K >= 1 && K < kMostWidth && sizes_fit(M, 2 * F, K); }

size_t gated_workspace_for(const harp_ctx *ctx, int64_t M, int64_t F, int64_t K) {
    const size_t forward = packed_bytes(M, K) + packed_bytes(2 * F, K) + partial_bytes(ctx, kForward, M, 2 * F, K);
    const size_t back = packed_bytes(M, K) + packed_bytes(K, F) + partial_bytes(ctx, kInput, M, F, K);
    return (forward > back ? forward : back) + 256;
}

int gated_check(harp_ctx *ctx, int64_t M, int64_t F, int64_t K, int type, int act, const Matrix *m, int count, bool lent, const void *workspace,
                size_t workspace_bytes) {
    if (!gated_sizes_fit(M, F, K)) return fail(ctx, HARP_ERR_SHAPE, "0 <= M < 2^31 and 1 <= F, K, N < 2^21 are wanted");
    const int rc = check_operands(ctx, type, act, m, count);
    if (rc != HARP_OK) return rc;
    const size_t need = lent ? gated_workspace_for(ctx, M, F, K) : 0;
    if (lent && (!workspace || !aligned(workspace, 256) || workspace_bytes < need))
        return fail(ctx, HARP_ERR_WORKSPACE, "the workspace needs %zu bytes, aligned to 256", need);
    const hipError_t e = hipSetDevice(ctx->device);
    return e == hipSuccess ? HARP_OK : hip_fail(ctx, e, "hipSetDevice");
}

template <typename T> void launch_forward(const harp_ctx *ctx, const harp_gated *g, void *workspace, hipStream_t st) {
    const int64_t M = g->M, F = g->F, K = g->K;
    const Plan plan = plan_for(ctx, kForward, M, 2 * F, K);
    Gated e = {g->act, 0, F, g->ldh, g->ldz, 0, g->bias, g->H, g->Z, nullptr};
    e.past = passes_the_caches(M, g->Z ? 3 * F : F, 2);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    Given x = {g->X, g->ldx, M, K}, w = {g->W, g->ldw, 2 * F, K};
    if (!plan.few) {
        x = packed<T>(x, ws, st);
        w = packed<T>(w, ws, st);
    }
    float *partial = plan.shares > 1 ? reinterpret_cast<float *>(ws) : nullptr;
    const T *px = static_cast<const T *>(x.a), *pw = static_cast<const T *>(w.a);
    if (plan.few) {
        const dim3 grid(uint32_t((F + 15) / 16), uint32_t(plan.shares)), block(kFewWaves * kWave);
        auto run = [&](auto wide) {
            constexpr bool W = decltype(wide)::value;
            if (M <= 16) few_tokens<T, W, 1, kGatedForward, Gated><<<grid, block, 0, st>>>(px, x.ld, pw, w.ld, M, F, K, plan.share, partial, e);
            else if (M <= 32) few_tokens<T, W, 2, kGatedForward, Gated><<<grid, block, 0, st>>>(px, x.ld, pw, w.ld, M, F, K, plan.share, partial, e);
            else few_tokens<T, W, 4, kGatedForward, Gated><<<grid, block, 0, st>>>(px, x.ld, pw, w.ld, M, F, K, plan.share, partial, e);
        };
        if (wide_rows(x) && wide_rows(w)) run(std::true_type());
        else run(std::false_type());
    } else if (partial) {
        launch_tiles<T, false, false>(plan, x, w, M, 2 * F, K, partial, Epilogue(), st);
    } else if (plan.big) {
        const int tp = int((M + 255) / 256), tq = int((F + 127) / 128);
        product<T, false, false, 256, 256, 4, 2, kGatedForward, Gated><<<dim3(uint32_t(tp) * uint32_t(tq)), dim3(512), 0, st>>>(
            px, x.ld, pw, w.ld, M, F, K, tp, tq, plan.share, nullptr, e);
    } else {
        const int tp = int((M + 127) / 128), tq = int((F + 63) / 64);
        product<T, false, false, 128, 128, 2, 2, kGatedForward, Gated><<<dim3(uint32_t(tp) * uint32_t(tq)), dim3(256), 0, st>>>(
            px, x.ld, pw, w.ld, M, F, K, tp, tq, plan.share, nullptr, e);
    }
    if (partial) gated_join<T, kGatedForward><<<dim3(blocks_for(M * ((F + 3) / 4))), dim3(256), 0, st>>>(partial, plan.shares, M, e);
}

template <typename T> void launch_back(const harp_ctx *ctx, const harp_gated_grads *g, void *workspace, hipStream_t st) {
    const int64_t M = g->M, F = g->F, N = g->N;
    Gated e = {g->act, 0, F, g->ldh, g->ldz, g->lddz, nullptr, g->H, const_cast<void *>(g->Z), g->dZ};
    e.past = passes_the_caches(M, g->H ? 3 * F : 2 * F, 2);
    if (!g->W) {
        gate_grad<T><<<dim3(blocks_for(M * ((F + 3) / 4))), dim3(256), 0, st>>>(static_cast<const T *>(g->dY), g->lddy, M, e);
        return;
    }
    const Plan plan = plan_for(ctx, kInput, M, F, N);
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    const Given dy = packed<T>({g->dY, g->lddy, M, N}, ws, st), w = packed<T>({g->W, g->ldw, N, F}, ws, st);
    float *partial = plan.shares > 1 ? reinterpret_cast<float *>(ws) : nullptr;
    const T *pd = static_cast<const T *>(dy.a), *pw = static_cast<const T *>(w.a);
    const int side = plan.big ? 256 : 128, tp = int((M + side - 1) / side), tq = int((F + side - 1) / side);
    const dim3 grid(uint32_t(tp) * uint32_t(tq));
    if (partial) launch_tiles<T, false, true>(plan, dy, w, M, F, N, partial, Epilogue(), st);
    else if (plan.big) product<T, false, true, 256, 256, 2, 4, kGatedBack, Gated><<<grid, dim3(512), 0, st>>>(pd, dy.ld, pw, w.ld, M, F, N, tp, tq, plan.share, nullptr, e);
    else product<T, false, true, 128, 128, 2, 2, kGatedBack, Gated><<<grid, dim3(256), 0, st>>>(pd, dy.ld, pw, w.ld, M, F, N, tp, tq, plan.share, nullptr, e);
    if (partial) gated_join<T, kGatedBack><<<dim3(blocks_for(M * ((F + 3) / 4))), dim3(256), 0, st>>>(partial, plan.shares, M, e);
}

int gated_launched(harp_ctx *ctx) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HARP_OK : hip_fail(ctx, e, "launching the gated block's kernels");
}

}  // namespace

extern "C" {

size_t harp_gated_workspace_bytes(harp_ctx *ctx, int64_t M, int64_t F, int64_t K) {
    return ctx && gated_sizes_fit(M, F, K) ? gated_workspace_for(ctx, M, F, K) : 0;
}

int harp_gated_forward(harp_ctx *ctx, const harp_gated *g, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    const bool some = g->M > 0;
    const Matrix m[] = {{"X", g->X, g->ldx, g->K, 2, some}, {"W", g->W, g->ldw, g->K, 2, true}, {"bias", g->bias, g->F, g->F, 2, false},
                        {"H", g->H, g->ldh, g->F, 2, some}, {"Z", g->Z, g->ldz, 2 * g->F, 2, false}};
    const int rc = gated_check(ctx, g->M, g->F, g->K, g->type, g->act, m, 5, true, workspace, workspace_bytes);
    if (rc != HARP_OK || !some) return rc;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) launch_forward<__bf16>(ctx, g, workspace, st);
    else launch_forward<_Float16>(ctx, g, workspace, st);
    return gated_launched(ctx);
}

int harp_gated_grad(harp_ctx *ctx, const harp_gated_grads *g, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    const bool some = g->M > 0;
    const int64_t N = g->W ? g->N : g->F;
    if (g->M > 1 && g->dZ && g->dZ == g->Z && g->lddz != g->ldz) return fail(ctx, HARP_ERR_SHAPE, "dZ is Z with another distance of rows");
    const Matrix m[] = {{"dY", g->dY, g->lddy, N, 2, some}, {"W", g->W, g->ldw, g->F, 2, false}, {"Z", g->Z, g->ldz, 2 * g->F, 2, some},
                        {"dZ", g->dZ, g->lddz, 2 * g->F, 2, some}, {"H", g->H, g->ldh, g->F, 2, false}};
    const int rc = gated_check(ctx, g->M, g->F, N, g->type, g->act, m, 5, g->W != nullptr, workspace, workspace_bytes);
    if (rc != HARP_OK || !some) return rc;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) launch_back<__bf16>(ctx, g, workspace, st);
    else launch_back<_Float16>(ctx, g, workspace, st);
    return gated_launched(ctx);
}

}  // extern "C"
