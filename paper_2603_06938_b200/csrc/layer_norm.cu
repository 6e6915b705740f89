// Layer norm over each of `groups` equal channel groups of a row, and its gradients (what follows linear
// attention, whose rows carry no denominator, with a group per head; with one group the norm in front of a layer):
//   mu, var over the group's entries, xh = (x - mu) rstd, rstd = 1 / sqrt(var + eps),  y = xh w + b
//   z = w dy:  dx = rstd (z - mean(z) - xh mean(z xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
// A row is read once: its entries stay in registers between the sums and the results, eight of them in each of
// NV places a thread; the statistics are fp32 and in two passes over the registers (mean, then squares around it).
#include <algorithm>

#include "la.h"

namespace swimba {

namespace {

constexpr int LN_THREADS = 256;

__device__ __forceinline__ void put8(float *p, const float (&v)[8])
{
    *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void put8(__nv_bfloat16 *p, const float (&v)[8])
{
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 q = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        o[i] = *reinterpret_cast<const uint32_t *>(&q);
    }
    *reinterpret_cast<uint4 *>(p) = make_uint4(o[0], o[1], o[2], o[3]);
}

// How a block of 256 threads lies over rows: `team` threads (a power of two) per group, gpb groups of a row and rpb rows
// at a time.  Groups beyond gpb go to other blocks (grid.y).
struct LnShape {
    int team, nv, gpb, rpb, ychunks;
};
inline LnShape ln_shape(int groups, int width)
{
    LnShape s;
    const int chunks = width / 8;
    s.nv = chunks <= 256 ? 1 : chunks <= 512 ? 2 : chunks <= 1024 ? 4 : 8;
    s.team = 1;
    while (s.team * s.nv < chunks) s.team *= 2;
    s.gpb = std::min(groups, LN_THREADS / s.team);
    s.ychunks = ceil_div(groups, s.gpb);
    s.gpb = ceil_div(groups, s.ychunks);
    s.rpb = LN_THREADS / (s.team * s.gpb);
    return s;
}

// Sum over the threads of a team; `red` has one float per warp and is used when a team is wider than a warp.
template <int K> __device__ __forceinline__ void team_sum(float (&v)[K], int team, float *red)
{
    const int width = min(team, 32);
    for (int o = width >> 1; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < K; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (team > 32) {
        const int warp = threadIdx.x >> 5, per = team >> 5, first = warp / per * per;
        __syncthreads();
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int i = 0; i < K; ++i) red[i * 8 + warp] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < K; ++i) {
            v[i] = 0.f;
            for (int w = 0; w < per; ++w) v[i] += red[i * 8 + first + w];
        }
    }
}

template <typename T, int NV>
__global__ void __launch_bounds__(LN_THREADS)
layer_norm_kernel(const T *__restrict__ x, int64_t ldx, const float *__restrict__ wt, const float *__restrict__ bias,
                  int64_t rows, int groups, int width, float eps, int team, int gpb, int rpb, T *__restrict__ y,
                  float *__restrict__ mean, float *__restrict__ rstd)
{
    __shared__ float red[8];
    grid_dep_launch();
    const int tid = threadIdx.x, t = tid % team, slot = tid / team;
    const int g = blockIdx.y * gpb + slot % gpb, rslot = slot / gpb;
    const bool mine = rslot < rpb && g < groups;
    float w[NV][8], b[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * team) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) { w[i][e] = 1.f; b[i][e] = 0.f; }
        (void)c;
    }
    grid_dep_wait();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * team) * 8;
        if (mine && c < width) {
            if (wt) load8(wt + (int64_t)g * width + c, w[i]);
            if (bias) load8(bias + (int64_t)g * width + c, b[i]);
        }
    }
    const int64_t D = (int64_t)groups * width;
    const float inv = 1.f / width;
    for (int64_t r0 = (int64_t)blockIdx.x * rpb; r0 < rows; r0 += (int64_t)gridDim.x * rpb) {
        const int64_t r = r0 + rslot;
        const bool live = mine && r < rows;
        float v[NV][8], s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * team) * 8;
            if (live && c < width) load8(x + r * ldx + (int64_t)g * width + c, v[i]);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += v[i][e];
        }
        team_sum(s, team, red);
        const float mu = s[0] * inv;
        s[0] = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * team) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[i][e] -= mu;
                if (c < width) s[0] = fmaf(v[i][e], v[i][e], s[0]);
            }
        }
        team_sum(s, team, red);
        const float rs = rsqrtf(s[0] * inv + eps);
        if (!live) continue;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * team) * 8;
            if (c >= width) continue;
            float o[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(v[i][e] * rs, w[i][e], b[i][e]);
            put8(y + r * D + (int64_t)g * width + c, o);
        }
        if (t == 0) {
            if (mean) mean[r * groups + g] = mu;
            if (rstd) rstd[r * groups + g] = rs;
        }
    }
}

// dx, and each block's sums of dy xh and dy over the rows that it met: partial[block][0 dw | 1 db][D].
template <typename T, int NV>
__global__ void __launch_bounds__(LN_THREADS)
layer_norm_backward_kernel(const T *__restrict__ dy, const T *__restrict__ x, int64_t ldx, const float *__restrict__ wt,
                           const float *__restrict__ mean, const float *__restrict__ rstd, int64_t rows, int groups,
                           int width, int team, int gpb, int rpb, T *__restrict__ dx, float *__restrict__ partial)
{
    __shared__ float red[16];
    __shared__ float sums[LN_THREADS * 8];
    grid_dep_launch();
    grid_dep_wait();
    const int tid = threadIdx.x, t = tid % team, slot = tid / team;
    const int g = blockIdx.y * gpb + slot % gpb, rslot = slot / gpb;
    const bool mine = rslot < rpb && g < groups;
    float w[NV][8], aw[NV][8], ab[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * team) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e) { w[i][e] = 1.f; aw[i][e] = 0.f; ab[i][e] = 0.f; }
        if (wt && mine && c < width) load8(wt + (int64_t)g * width + c, w[i]);
    }
    const int64_t D = (int64_t)groups * width;
    const float inv = 1.f / width;
    for (int64_t r0 = (int64_t)blockIdx.x * rpb; r0 < rows; r0 += (int64_t)gridDim.x * rpb) {
        const int64_t r = r0 + rslot;
        const bool live = mine && r < rows;
        typename Raw8<T>::type rx[NV], rd[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * team) * 8;
            if (live && c < width) {
                load_raw8(x + r * ldx + (int64_t)g * width + c, rx[i]);
                load_raw8(dy + r * D + (int64_t)g * width + c, rd[i]);
            }
        }
        const float mu = live ? mean[r * groups + g] : 0.f, rs = live ? rstd[r * groups + g] : 0.f;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * team) * 8;
            if (!(live && c < width)) continue;
            float xv[8], dv[8];
            unpack8(rx[i], xv);
            unpack8(rd[i], dv);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = (xv[e] - mu) * rs, z = dv[e] * w[i][e];
                s[0] += z;
                s[1] = fmaf(z, xh, s[1]);
                aw[i][e] = fmaf(dv[e], xh, aw[i][e]);
                ab[i][e] += dv[e];
            }
        }
        team_sum(s, team, red);
        if (!live) continue;
        const float m0 = s[0] * inv, m1 = s[1] * inv;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * team) * 8;
            if (c >= width) continue;
            float xv[8], dv[8], o[8];
            unpack8(rx[i], xv);
            unpack8(rd[i], dv);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = (xv[e] - mu) * rs;
                o[e] = rs * (dv[e] * w[i][e] - m0 - xh * m1);
            }
            put8(dx + r * D + (int64_t)g * width + c, o);
        }
    }
    if (!partial) return;
    // the rows of a block side by side: their sums meet in shared memory, in order
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * team) * 8;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[e * LN_THREADS + tid] = k == 0 ? aw[i][e] : ab[i][e];
            __syncthreads();
            if (rslot == 0 && mine && c < width) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    o[e] = 0.f;
                    for (int q = 0; q < rpb; ++q) o[e] += sums[e * LN_THREADS + tid + q * gpb * team];
                }
                put8(partial + ((int64_t)blockIdx.x * 2 + k) * D + (int64_t)g * width + c, o);
            }
        }
}

// dw, db [D] = the blocks' partial sums, added in a fixed order: 32 columns and 8 runs of blocks per thread block.
__global__ void __launch_bounds__(256)
layer_norm_sum_kernel(const float *__restrict__ partial, int nblk, int64_t D, float *__restrict__ dw,
                      float *__restrict__ db)
{
    __shared__ float s[8][33];
    grid_dep_launch();
    grid_dep_wait();
    const int lane = threadIdx.x & 31, run = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + lane;
    float v = 0.f;
    if (c < 2 * D)
#pragma unroll 8
        for (int i = run; i < nblk; i += 8) v += partial[(int64_t)i * 2 * D + c];
    s[run][lane] = v;
    __syncthreads();
    if (run == 0 && c < 2 * D) {
        float o = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) o += s[i][lane];
        if (c < D) {
            if (dw) dw[c] = o;
        } else if (db) {
            db[c - D] = o;
        }
    }
}

int ln_blocks(const LnShape &s, int64_t rows, int sm_count, int per_sm)
{
    const int64_t need = ceil_div64(rows, s.rpb);
    return (int)std::min<int64_t>(need, std::max(1, per_sm * sm_count / s.ychunks));
}

template <typename T, int NV>
int run_norm(LaunchCtx &ctx, const LnShape &s, const void *x, int64_t ldx, const float *w, const float *b, int64_t rows,
             int groups, int width, float eps, int sm_count, void *y, float *mean, float *rstd)
{
    ctx.begin(STAGE_LAYER_NORM);
    launch_kernel(layer_norm_kernel<T, NV>, dim3(ln_blocks(s, rows, sm_count, 8), s.ychunks), dim3(LN_THREADS), 0,
                  ctx.stream, true, (const T *)x, ldx, w, b, rows, groups, width, eps, s.team, s.gpb, s.rpb, (T *)y,
                  mean, rstd);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

template <typename T, int NV>
int run_backward(LaunchCtx &ctx, const LnShape &s, const void *dy, const void *x, int64_t ldx, const float *w,
                 const float *mean, const float *rstd, int64_t rows, int groups, int width, int sm_count, void *dx,
                 float *partial)
{
    ctx.begin(STAGE_LAYER_NORM_BACKWARD);
    launch_kernel(layer_norm_backward_kernel<T, NV>, dim3(ln_blocks(s, rows, sm_count, 2), s.ychunks), dim3(LN_THREADS),
                  0, ctx.stream, true, (const T *)dy, (const T *)x, ldx, w, mean, rstd, rows, groups, width, s.team,
                  s.gpb, s.rpb, (T *)dx, partial);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace

int launch_layer_norm(LaunchCtx &ctx, int dtype, const void *x, int64_t ldx, const float *w, const float *b, int64_t rows,
                      int groups, int width, float eps, int sm_count, void *y, float *mean, float *rstd)
{
    const LnShape s = ln_shape(groups, width);
#define LN_RUN(T, NV) run_norm<T, NV>(ctx, s, x, ldx, w, b, rows, groups, width, eps, sm_count, y, mean, rstd)
    if (dtype == SWIMBA_DTYPE_FP32)
        return s.nv == 1 ? LN_RUN(float, 1) : s.nv == 2 ? LN_RUN(float, 2) : s.nv == 4 ? LN_RUN(float, 4) : LN_RUN(float, 8);
    return s.nv == 1 ? LN_RUN(__nv_bfloat16, 1) : s.nv == 2 ? LN_RUN(__nv_bfloat16, 2)
           : s.nv == 4 ? LN_RUN(__nv_bfloat16, 4) : LN_RUN(__nv_bfloat16, 8);
#undef LN_RUN
}

size_t layer_norm_partial_bytes(int64_t rows, int groups, int width, int sm_count)
{
    const LnShape s = ln_shape(groups, width);
    return (size_t)ln_blocks(s, rows, sm_count, 2) * 2 * groups * width * sizeof(float);
}

int launch_layer_norm_backward(LaunchCtx &ctx, int dtype, const void *dy, const void *x, int64_t ldx, const float *w,
                               const float *mean, const float *rstd, int64_t rows, int groups, int width, int sm_count,
                               void *dx, float *dw, float *db, float *partial)
{
    const LnShape s = ln_shape(groups, width);
#define LN_RUN(T, NV) run_backward<T, NV>(ctx, s, dy, x, ldx, w, mean, rstd, rows, groups, width, sm_count, dx, partial)
    int rc;
    if (dtype == SWIMBA_DTYPE_FP32)
        rc = s.nv == 1 ? LN_RUN(float, 1) : s.nv == 2 ? LN_RUN(float, 2) : s.nv == 4 ? LN_RUN(float, 4) : LN_RUN(float, 8);
    else
        rc = s.nv == 1 ? LN_RUN(__nv_bfloat16, 1) : s.nv == 2 ? LN_RUN(__nv_bfloat16, 2)
             : s.nv == 4 ? LN_RUN(__nv_bfloat16, 4) : LN_RUN(__nv_bfloat16, 8);
#undef LN_RUN
    if (rc != SWIMBA_OK || !partial) return rc;
    const int64_t D = (int64_t)groups * width;
    ctx.begin(STAGE_LAYER_NORM_SUM);
    launch_kernel(layer_norm_sum_kernel, dim3((unsigned)ceil_div64(2 * D, 32)), dim3(256), 0, ctx.stream, true, partial,
                  ln_blocks(s, rows, sm_count, 2), D, dw, db);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace swimba
