// Balance loss of a router, its per-expert counts and gradients (Background, "Mixture of Experts": what keeps a
// trained router from sending every token to the same few experts):
//   p_t = softmax(W_r u_t) over all E,   f_e = counts_e / (k Tv),   m_e = mean over the Tv valid tokens of p_te
//   loss = coef E sum_e f_e m_e          (coef when all experts get the same share)
//   dg_te = coef E / Tv p_te (f_e - sum_j f_j p_tj),   dW_r = sum_t dg_t u_t^T,   du_t = W_r^T dg_t
// The shares f are constants of the differentiation.  They lie near 1 / E, and the gradient depends only on how far
// they differ from it, so that difference is taken from the whole numbers before anything is rounded.
// The counts come first (from the active sets alone), so that one pass over u gives the loss and the gradients.
#include <algorithm>

#include "la.h"

namespace swimba {

namespace {

constexpr int BL_COUNT_BLOCKS = 64;
constexpr int BL_TOKENS = 4;        // tokens a warp works at a time

// Counts of this block's share of the entries; cnt[block][0 .. E) experts, cnt[block][E] valid tokens.
__global__ void __launch_bounds__(256)
balance_count_kernel(const int32_t *__restrict__ idx, const uint8_t *__restrict__ valid, int64_t T, int k, int E,
                     int *__restrict__ cnt, int *d_status, bool check)
{
    __shared__ int hist[SWIMBA_MAX_EXPERTS + 1];
    grid_dep_launch();
    grid_dep_wait();
    for (int i = threadIdx.x; i <= E; i += blockDim.x) hist[i] = 0;
    __syncthreads();
    for (int64_t t = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; t < T; t += (int64_t)gridDim.x * blockDim.x) {
        if (valid && !valid[t]) continue;
        atomicAdd(&hist[E], 1);
        for (int j = 0; j < k; ++j) {
            const int e = idx[t * k + j];
            if ((unsigned)e < (unsigned)E) atomicAdd(&hist[e], 1);
            else if (check) atomicCAS(d_status, 0, SWIMBA_ERR_DEVICE_BOUNDS);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i <= E; i += blockDim.x) cnt[blockIdx.x * (E + 1) + i] = hist[i];
}

// Sum of the count blocks into shared memory: total[0 .. E] (E: valid tokens).  All threads of the block.
__device__ __forceinline__ void total_counts(const int *cnt, int nblk, int E, int *total)
{
    for (int i = threadIdx.x; i <= E; i += blockDim.x) {
        int s = 0;
#pragma unroll 8
        for (int b = 0; b < nblk; ++b) s += cnt[b * (E + 1) + i];
        total[i] = s;
    }
    __syncthreads();
}
// f_e - 1 / E from the whole numbers.
__device__ __forceinline__ float share_difference(int count, int valid, int k, int E)
{
    if (valid <= 0) return 0.f;
    return (float)((double)((long long)count * E - (long long)k * valid) / ((double)k * valid * E));
}

// Any F % 8 == 0, E <= 64, both types: a warp per BL_TOKENS tokens; logits by FMA with the features across the
// lanes, softmax with the experts across the lanes, then dg (kept for dW when asked) and du.
template <typename T>
__global__ void __launch_bounds__(256)
balance_tokens_kernel(const T *__restrict__ u, const T *__restrict__ W, const uint8_t *__restrict__ valid, int64_t Tn,
                      int F, int E, int k, float coef, const int *__restrict__ cnt, int ncnt, float *__restrict__ dg,
                      T *__restrict__ du, float *__restrict__ mean_part)
{
    __shared__ int total[SWIMBA_MAX_EXPERTS + 1];
    __shared__ float lg[8][BL_TOKENS][SWIMBA_MAX_EXPERTS];
    __shared__ float psum[8][SWIMBA_MAX_EXPERTS];
    grid_dep_launch();
    grid_dep_wait();
    total_counts(cnt, ncnt, E, total);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int nv = total[E];
    const float d0 = lane < E ? share_difference(total[lane], nv, k, E) : 0.f;
    const float d1 = lane + 32 < E ? share_difference(total[lane + 32], nv, k, E) : 0.f;
    const float c = nv > 0 ? coef * E / nv : 0.f;
    float p0 = 0.f, p1 = 0.f;
    for (int64_t t0 = ((int64_t)blockIdx.x * 8 + warp) * BL_TOKENS; t0 < Tn; t0 += (int64_t)gridDim.x * 8 * BL_TOKENS) {
        const int n = (int)min((int64_t)BL_TOKENS, Tn - t0);
        for (int e0 = 0; e0 < E; e0 += 8) {
            float acc[BL_TOKENS][8];
#pragma unroll
            for (int i = 0; i < BL_TOKENS; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[i][e] = 0.f;
            for (int f = lane * 8; f < F; f += 256) {
                float uv[BL_TOKENS][8];
#pragma unroll
                for (int i = 0; i < BL_TOKENS; ++i) {
                    if (i < n) load8(u + (t0 + i) * F + f, uv[i]);
                    else
#pragma unroll
                        for (int x = 0; x < 8; ++x) uv[i][x] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (e0 + e >= E) break;
                    float wv[8];
                    load8(W + (int64_t)(e0 + e) * F + f, wv);
#pragma unroll
                    for (int i = 0; i < BL_TOKENS; ++i)
#pragma unroll
                        for (int x = 0; x < 8; ++x) acc[i][e] = fmaf(uv[i][x], wv[x], acc[i][e]);
                }
            }
#pragma unroll
            for (int i = 0; i < BL_TOKENS; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (e0 + e >= E) break;
                    const float s = warp_sum(acc[i][e]);
                    if (lane == e) lg[warp][i][e0 + e] = s;
                }
        }
        __syncwarp();
        for (int i = 0; i < n; ++i) {
            const bool ok = !valid || valid[t0 + i];
            const float g0 = lane < E ? lg[warp][i][lane] : -INFINITY, g1 = lane + 32 < E ? lg[warp][i][lane + 32] : -INFINITY;
            float m = fmaxf(g0, g1);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float x0 = lane < E ? expf(g0 - m) : 0.f, x1 = lane + 32 < E ? expf(g1 - m) : 0.f;
            const float s = warp_sum(x0 + x1);
            // (a padded token's features may hold anything: its probabilities are taken as zero, not multiplied by it)
            const float q0 = ok ? x0 / s : 0.f, q1 = ok ? x1 / s : 0.f;
            p0 += q0;
            p1 += q1;
            const float fb = warp_sum(q0 * d0 + q1 * d1);
            const float a0 = c * q0 * (d0 - fb), a1 = c * q1 * (d1 - fb);
            __syncwarp();
            if (lane < E) lg[warp][i][lane] = a0;
            if (lane + 32 < E) lg[warp][i][lane + 32] = a1;
            if (dg) {
                if (lane < E) dg[(t0 + i) * E + lane] = a0;
                if (lane + 32 < E) dg[(t0 + i) * E + lane + 32] = a1;
            }
        }
        __syncwarp();
        if (du) {
            for (int f = lane * 8; f < F; f += 256) {
                float acc[BL_TOKENS][8];
#pragma unroll
                for (int i = 0; i < BL_TOKENS; ++i)
#pragma unroll
                    for (int x = 0; x < 8; ++x) acc[i][x] = 0.f;
                for (int e = 0; e < E; ++e) {
                    float wv[8];
                    load8(W + (int64_t)e * F + f, wv);
#pragma unroll
                    for (int i = 0; i < BL_TOKENS; ++i) {
                        const float a = i < n ? lg[warp][i][e] : 0.f;
#pragma unroll
                        for (int x = 0; x < 8; ++x) acc[i][x] = fmaf(a, wv[x], acc[i][x]);
                    }
                }
#pragma unroll
                for (int i = 0; i < BL_TOKENS; ++i) {
                    if (i >= n) break;
                    T o[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) o[x] = from_f32<T>(acc[i][x]);
                    uint4 *dst = reinterpret_cast<uint4 *>(du + (t0 + i) * F + f);
                    dst[0] = reinterpret_cast<const uint4 *>(o)[0];
                    if (sizeof(T) == 4) dst[1] = reinterpret_cast<const uint4 *>(o)[1];
                }
            }
            __syncwarp();
        }
    }
    if (lane < E) psum[warp][lane] = p0;
    if (lane + 32 < E) psum[warp][lane + 32] = p1;
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        float s = 0.f;
        for (int w = 0; w < 8; ++w) s += psum[w][e];
        mean_part[(int64_t)blockIdx.x * E + e] = s;
    }
}

// part[split][e][f] = sum over the split's tokens of dg_te u_tf; a thread owns eight features and eight experts.
constexpr int BW_TOK = 64;
template <typename T>
__global__ void __launch_bounds__(128)
balance_dw_kernel(const T *__restrict__ u, const float *__restrict__ dg, const uint8_t *__restrict__ valid, int64_t Tn,
                  int F, int E, int64_t per, float *__restrict__ part)
{
    __shared__ float s[BW_TOK][8];
    __shared__ int live[BW_TOK];
    grid_dep_launch();
    grid_dep_wait();
    const int f = (blockIdx.x * 128 + threadIdx.x) * 8, e0 = blockIdx.z * 8;
    const int64_t a = blockIdx.y * per, b = min(Tn, a + per);
    float acc[8][8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int x = 0; x < 8; ++x) acc[e][x] = 0.f;
    for (int64_t t0 = a; t0 < b; t0 += BW_TOK) {
        const int n = (int)min((int64_t)BW_TOK, b - t0);
        __syncthreads();
        for (int i = threadIdx.x; i < n * 8; i += 128)
            s[i >> 3][i & 7] = e0 + (i & 7) < E ? dg[(t0 + (i >> 3)) * E + e0 + (i & 7)] : 0.f;
        for (int i = threadIdx.x; i < n; i += 128) live[i] = !valid || valid[t0 + i];
        __syncthreads();
        if (f < F) {
#pragma unroll 4
            for (int i = 0; i < n; ++i) {
                if (!live[i]) continue;
                float uv[8];
                load8(u + (t0 + i) * F + f, uv);
#pragma unroll
                for (int e = 0; e < 8; ++e)
#pragma unroll
                    for (int x = 0; x < 8; ++x) acc[e][x] = fmaf(s[i][e], uv[x], acc[e][x]);
            }
        }
    }
    if (f < F)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e0 + e >= E) break;
            float4 *p = reinterpret_cast<float4 *>(part + ((int64_t)blockIdx.y * E + e0 + e) * F + f);
            p[0] = make_float4(acc[e][0], acc[e][1], acc[e][2], acc[e][3]);
            p[1] = make_float4(acc[e][4], acc[e][5], acc[e][6], acc[e][7]);
        }
}

// dW (+)= sum of the splits, four entries a thread; the last block gives counts, mean probabilities and the loss.
__global__ void __launch_bounds__(256)
balance_sum_kernel(const float *__restrict__ part, int nsplit, int64_t EF, float *dW, bool add,
                   const int *__restrict__ cnt, int ncnt, const float *__restrict__ mean_part, int nmean, int E, int k,
                   float coef, float *__restrict__ loss, int32_t *__restrict__ counts, float *__restrict__ mean_prob)
{
    __shared__ int total[SWIMBA_MAX_EXPERTS + 1];
    __shared__ float mean[SWIMBA_MAX_EXPERTS], run[4][SWIMBA_MAX_EXPERTS];
    grid_dep_launch();
    grid_dep_wait();
    if (blockIdx.x + 1 < gridDim.x) {
        const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
        if (i >= EF) return;
        float4 s = add ? *reinterpret_cast<const float4 *>(dW + i) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
        for (int b = 0; b < nsplit; ++b) {
            const float4 v = *reinterpret_cast<const float4 *>(part + (int64_t)b * EF + i);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        *reinterpret_cast<float4 *>(dW + i) = s;
        return;
    }
    total_counts(cnt, ncnt, E, total);
    const int nv = total[E], e = threadIdx.x & 63, r = threadIdx.x >> 6;
    if (e < E) {
        float s = 0.f;
        for (int b = r; b < nmean; b += 4) s += mean_part[(int64_t)b * E + e];
        run[r][e] = s;
    }
    __syncthreads();
    if (threadIdx.x < E) {
        const float m = run[0][e] + run[1][e] + run[2][e] + run[3][e];
        mean[e] = nv > 0 ? m / nv : 0.f;
        if (counts) counts[e] = total[e];
        if (mean_prob) mean_prob[e] = mean[e];
    }
    __syncthreads();
    if (threadIdx.x == 0 && loss) {
        double s = 0.0;
        for (int i = 0; i < E; ++i) s += (double)total[i] * mean[i];
        *loss = nv > 0 ? (float)(coef * E * s / ((double)k * nv)) : 0.f;
    }
}

int bl_blocks(int64_t T, int sm_count) { return (int)std::min<int64_t>(ceil_div64(T, 8 * BL_TOKENS), 4 * sm_count); }
int bl_splits(int64_t T, int F, int E, int sm_count)
{
    const int64_t cols = (int64_t)ceil_div(F, 1024) * ceil_div(E, 8);
    return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div64(T, BW_TOK), 4 * sm_count / cols));
}

struct BalanceLayout {
    size_t cnt, mean, dg, part, total;
};
BalanceLayout bl_layout(int64_t T, int F, int E, int sm_count)
{
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    BalanceLayout l;
    size_t o = 0;
    l.cnt = o;  o += up(sizeof(int) * BL_COUNT_BLOCKS * (E + 1));
    l.mean = o; o += up(sizeof(float) * bl_blocks(T, sm_count) * E);
    l.dg = o;   o += up(sizeof(float) * T * E);
    l.part = o; o += up(sizeof(float) * bl_splits(T, F, E, sm_count) * E * F);
    l.total = o;
    return l;
}

template <typename T>
int run_balance(LaunchCtx &ctx, const void *u, const void *W, const int32_t *idx, const uint8_t *valid, int64_t Tn, int F,
                int E, int k, float coef, int sm_count, float *loss, int32_t *counts, float *mean_prob, float *dW,
                bool add, void *du, char *ws)
{
    const BalanceLayout l = bl_layout(Tn, F, E, sm_count);
    int *cnt = (int *)(ws + l.cnt);
    float *mean = (float *)(ws + l.mean), *dg = (float *)(ws + l.dg), *part = (float *)(ws + l.part);
    const int ncnt = (int)std::min<int64_t>(BL_COUNT_BLOCKS, ceil_div64(Tn, 256)), nblk = bl_blocks(Tn, sm_count);
    ctx.begin(STAGE_BALANCE_COUNT);
    launch_kernel(balance_count_kernel, dim3(ncnt), dim3(256), 0, ctx.stream, true, idx, valid, Tn, k, E, cnt,
                  ctx.d_status, ctx.check_indices);
    ctx.end();
    ctx.begin(STAGE_BALANCE_TOKENS);
    launch_kernel(balance_tokens_kernel<T>, dim3(nblk), dim3(256), 0, ctx.stream, true, (const T *)u, (const T *)W, valid,
                  Tn, F, E, k, coef, (const int *)cnt, ncnt, dW ? dg : (float *)nullptr, (T *)du, mean);
    ctx.end();
    const int splits = bl_splits(Tn, F, E, sm_count);
    const int64_t per = ceil_div64(ceil_div64(Tn, splits), BW_TOK) * BW_TOK, EF = (int64_t)E * F;
    const int used = (int)ceil_div64(Tn, per);
    if (dW) {
        ctx.begin(STAGE_BALANCE_DW);
        launch_kernel(balance_dw_kernel<T>, dim3(ceil_div(F, 1024), used, ceil_div(E, 8)), dim3(128), 0, ctx.stream, true,
                      (const T *)u, (const float *)dg, valid, Tn, F, E, per, part);
        ctx.end();
    }
    ctx.begin(STAGE_BALANCE_SUM);
    launch_kernel(balance_sum_kernel, dim3((unsigned)(dW ? ceil_div64(EF, 1024) : 0) + 1), dim3(256), 0, ctx.stream, true,
                  (const float *)part, used, EF, dW, add, (const int *)cnt, ncnt, (const float *)mean, nblk, E, k, coef,
                  loss, counts, mean_prob);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace

size_t balance_workspace_bytes(int dtype, int64_t T, int F, int E, int sm_count)
{
    (void)dtype;
    return bl_layout(T, F, E, sm_count).total;
}

int launch_balance(LaunchCtx &ctx, int dtype, const void *u, const void *W, const int32_t *idx, const uint8_t *valid,
                   int64_t T, int F, int E, int k, float coef, int sm_count, float *loss, int32_t *counts,
                   float *mean_prob, float *dW, bool add, void *du, void *workspace)
{
    if (dtype == SWIMBA_DTYPE_FP32)
        return run_balance<float>(ctx, u, W, idx, valid, T, F, E, k, coef, sm_count, loss, counts, mean_prob, dW, add, du,
                                  (char *)workspace);
    return run_balance<__nv_bfloat16>(ctx, u, W, idx, valid, T, F, E, k, coef, sm_count, loss, counts, mean_prob, dW, add,
                                      du, (char *)workspace);
}

}  // namespace swimba
