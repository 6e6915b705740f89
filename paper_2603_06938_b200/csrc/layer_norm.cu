// Layer norm over each of `groups` equal channel groups of a row, and its gradients (what follows linear
// attention, whose rows carry no denominator, with a group per head; with one group the norm in front of a layer):
//   mu, var over the group's entries, xh = (x - mu) rstd, rstd = 1 / sqrt(var + eps),  y = xh w + b
//   z = w dy:  dx = rstd (z - mean(z) - xh mean(z xh)),  dw = sum over rows of dy xh,  db = sum over rows of dy
// A row is read once: its entries stay in registers between the sums and the results, eight of them in each of
// NV places a thread; the statistics are fp32 and in two passes over the registers (mean, then squares around it).
// Instruction issue bounds these kernels as soon as it can (2048 entries a row by 256 threads: 77 us forward, 154
// backward of 32768 rows): few threads a row, so that the sums across threads are shared by many entries, arithmetic on pairs,
// and places at distances known when compiling.  So that forward takes 47 us, 5.7 TB/s (a copy of the same bytes 45), with the
// weights in shared memory (from the L1 cache, whose wavefronts they half fill, 61).  Backward takes 111 us, 3.6 TB/s, with
// 45 % of the issue slots in use and two blocks an SM, whose warps wait for each other's sums and for shared memory.  In fp32
// 103 and 214 us (floors 82 and 123).
#include <algorithm>
#include <climits>

#include "la.h"
#include "tc05.cuh"

namespace swimba {

namespace {

constexpr int LN_THREADS = 256;

// Eight entries as four pairs.
__device__ __forceinline__ void pairs8(const Raw8h &r, uint64_t (&v)[4])
{
    const uint32_t w[4] = {r.a.x, r.a.y, r.a.z, r.a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = tc::f32x2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ void pairs8(const Raw8f &r, uint64_t (&v)[4])
{
    v[0] = tc::f32x2(r.a.x, r.a.y); v[1] = tc::f32x2(r.a.z, r.a.w);
    v[2] = tc::f32x2(r.b.x, r.b.y); v[3] = tc::f32x2(r.b.z, r.b.w);
}
template <typename T> __device__ __forceinline__ void load_pairs(const T *p, uint64_t (&v)[4])
{
    typename Raw8<T>::type r;
    load_raw8(p, r);
    pairs8(r, v);
}
__device__ __forceinline__ void put8(float *p, const uint64_t (&v)[4])
{
    const float2 a = tc::f32x2_get(v[0]), b = tc::f32x2_get(v[1]), c = tc::f32x2_get(v[2]), d = tc::f32x2_get(v[3]);
    *reinterpret_cast<float4 *>(p) = make_float4(a.x, a.y, b.x, b.y);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(c.x, c.y, d.x, d.y);
}
__device__ __forceinline__ void put8(__nv_bfloat16 *p, const uint64_t (&v)[4])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(tc::f32x2_bf16(v[0]), tc::f32x2_bf16(v[1]), tc::f32x2_bf16(v[2]), tc::f32x2_bf16(v[3]));
}
// Entries that are taken apart anew in every pass over them: as fp32 they would fill the registers of a second block.
__device__ __forceinline__ void anew(Raw8h &r) { asm volatile("" : "+r"(r.a.x), "+r"(r.a.y), "+r"(r.a.z), "+r"(r.a.w)); }
__device__ __forceinline__ void anew(Raw8f &) {}
__device__ __forceinline__ float both(uint64_t v)
{
    const float2 f = tc::f32x2_get(v);
    return f.x + f.y;
}

// s / width from 1 / width, with what is left of s put right (one Newton step): a row of equal entries has them as its mean, to
// the bit, where the product alone is off by 2^-24.  (A division takes registers enough to change how many blocks an SM
// holds: 32768 x 2048 forward 50 us instead of 46.)
__device__ __forceinline__ float ln_mean(float s, int width, float inv)
{
    const float m = s * inv;
    return fmaf(fmaf(-m, (float)width, s), inv, m);
}

// Weights in shared memory: of every eight the first four, then the second four of all, so that threads side by side read side
// by side (in place, 32 bytes a thread, half of every wavefront goes unused).
__device__ __forceinline__ void stage_weights(float *to, const float *from, float none, int n)
{
    for (int i = threadIdx.x; i < n; i += LN_THREADS) to[(i >> 2 & 1) * (n >> 1) + (i >> 3) * 4 + (i & 3)] = from ? from[i] : none;
}
__device__ __forceinline__ void staged_pairs(const float *w, int half, uint64_t (&v)[4])      // half: entries of all over 2
{
    const float4 a = *reinterpret_cast<const float4 *>(w), b = *reinterpret_cast<const float4 *>(w + half);
    v[0] = tc::f32x2(a.x, a.y); v[1] = tc::f32x2(a.z, a.w);
    v[2] = tc::f32x2(b.x, b.y); v[3] = tc::f32x2(b.z, b.w);
}

// How a block of 256 threads lies over rows: `team` threads (a power of two) per group, gpb groups of a row and rpb rows
// at a time.  Groups beyond gpb go to other blocks (grid.y).
struct LnShape {
    int team, nv, gpb, rpb, ychunks;
};
// most: places a thread at most while a warp or part of one has a row (wider rows take more warps first, then more places).
// room: entries of the groups that a block works at most, where a thread has more than two places (but one group always fits).
inline LnShape ln_shape(int groups, int width, int most, int room)
{
    LnShape s;
    const int chunks = width / 8;
    s.nv = 1;
    s.team = 1;
    while (s.team < 32 && s.team < chunks) s.team *= 2;
    while (s.nv < most && s.team * s.nv < chunks) s.nv *= 2;
    while (s.team < LN_THREADS && s.team * s.nv < chunks) s.team *= 2;
    while (s.team * s.nv < chunks) s.nv *= 2;
    s.gpb = std::min(groups, LN_THREADS / s.team);
    if (s.nv > 2) s.gpb = std::max(1, std::min(s.gpb, room / width));
    s.ychunks = ceil_div(groups, s.gpb);
    s.gpb = ceil_div(groups, s.ychunks);
    s.rpb = LN_THREADS / (s.team * s.gpb);
    return s;
}
constexpr int LN_FORWARD_PLACES = 8, LN_BACKWARD_PLACES = 4;
constexpr int LN_FORWARD_ROOM = 8192;     // (their weights, 64 KB, leave an SM three blocks)

// Sums over the threads of a team.  A team wider than a warp meets in `red` (8 floats per sum), of which there are two,
// taken in turn, so that one barrier of the team a call is enough; every thread of the team calls it.
template <int K> __device__ __forceinline__ void team_sum(float (&v)[K], int team, float *red, int &turn)
{
    if (team >= 32) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < K; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    } else {
        for (int o = team >> 1; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < K; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    }
    if (team > 32) {
        const int warp = threadIdx.x >> 5, per = team >> 5, first = warp / per * per;
        float *r = red + turn * K * 8;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int i = 0; i < K; ++i) r[i * 8 + warp] = v[i];
        tc::named_bar_sync(1 + threadIdx.x / team, team);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (per == 8) {
                const float4 x = *reinterpret_cast<const float4 *>(r + i * 8), y = *reinterpret_cast<const float4 *>(r + i * 8 + 4);
                v[i] = ((x.x + x.y) + (x.z + x.w)) + ((y.x + y.y) + (y.z + y.w));
            } else {
                v[i] = 0.f;
                for (int w = 0; w < per; ++w) v[i] += r[i * 8 + first + w];
            }
        }
    }
}

// Few entries a thread (NV 1 or 2 places), whose weights stay in registers.  R rows (or sets of rpb rows) at a time: their loads are in flight together and one barrier serves their sums.
template <typename T, int NV, int R>
__global__ void __launch_bounds__(LN_THREADS)
layer_norm_kernel(const T *__restrict__ x, int64_t ldx, const float *__restrict__ wt, const float *__restrict__ bias,
                  int64_t rows, int groups, int width, float eps, int team, int gpb, int rpb, T *__restrict__ y,
                  float *__restrict__ mean, float *__restrict__ rstd)
{
    __shared__ __align__(16) float red[2 * R * 8];
    grid_dep_launch();
    const int tid = threadIdx.x, t = tid % team, slot = tid / team;
    const int g = blockIdx.y * gpb + slot % gpb, rslot = slot / gpb;
    const bool mine = rslot < rpb && g < groups;
    grid_dep_wait();
    const int64_t D = (int64_t)groups * width, step = (int64_t)gridDim.x * rpb;
    const float inv = 1.f / width;
    const float *wg = wt + (int64_t)g * width, *bg = bias + (int64_t)g * width;
    uint64_t w[NV][4], b[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * team) * 8;
#pragma unroll
        for (int e = 0; e < 4; ++e) { w[i][e] = tc::f32x2(1.f, 1.f); b[i][e] = 0ull; }
        if (!mine || c >= width) continue;
        if (wt) load_pairs(wg + c, w[i]);
        if (bias) load_pairs(bg + c, b[i]);
    }
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * rpb; r0 < rows; r0 += R * step) {
        uint64_t v[R][NV][4];
        float s[R];
#pragma unroll
        for (int k = 0; k < R; ++k)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int64_t r = r0 + k * step + rslot;
                const int c = (t + i * team) * 8;
                typename Raw8<T>::type raw = {};
                if (mine && r < rows && c < width) load_raw8(x + r * ldx + (int64_t)g * width + c, raw);
                pairs8(raw, v[k][i]);
            }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            uint64_t a2[2] = {0ull, 0ull};
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) a2[e & 1] = tc::f32x2_add(a2[e & 1], v[k][i][e]);
            s[k] = both(tc::f32x2_add(a2[0], a2[1]));
        }
        team_sum(s, team, red, turn);
        float mu[R];
#pragma unroll
        for (int k = 0; k < R; ++k) {
            mu[k] = ln_mean(s[k], width, inv);
            const uint64_t m2 = tc::f32x2(-mu[k], -mu[k]);
            uint64_t a2[2] = {0ull, 0ull};
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if ((t + i * team) * 8 < width)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[k][i][e] = tc::f32x2_add(v[k][i][e], m2);
                        a2[e & 1] = tc::f32x2_fma(v[k][i][e], v[k][i][e], a2[e & 1]);
                    }
            s[k] = both(tc::f32x2_add(a2[0], a2[1]));
        }
        team_sum(s, team, red, turn);
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const int64_t r = r0 + k * step + rslot;
            const float rs = rsqrtf(s[k] * inv + eps);
            const uint64_t rs2 = tc::f32x2(rs, rs);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * team) * 8;
                uint64_t o[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = tc::f32x2_fma(tc::f32x2_mul(v[k][i][e], rs2), w[i][e], b[i][e]);
                if (mine && r < rows && c < width) put8(y + r * D + (int64_t)g * width + c, o);
            }
            if (mine && r < rows && t == 0) {
                if (mean) mean[r * groups + g] = mu[k];
                if (rstd) rstd[r * groups + g] = rs;
            }
        }
    }
}

// More entries a thread (NV 4 or 8 places) of one row at a time.  The weights come from shared memory with every row, the
// entries stay as they were loaded.  TEAM: the team, where it is a warp (0: any), so that a thread's places lie at distances
// known when compiling (with those and without the defaults of missing weights: half the instructions).
template <typename T, int NV, int TEAM>
__global__ void __launch_bounds__(LN_THREADS, sizeof(T) == 2 && !(NV == 8 && TEAM) ? 3 : 2)
layer_norm_wide_kernel(const T *__restrict__ x, int64_t ldx, const float *__restrict__ wt, const float *__restrict__ bias,
                       int64_t rows, int groups, int width, float eps, int any_team, int gpb, int rpb, T *__restrict__ y,
                       float *__restrict__ mean, float *__restrict__ rstd)
{
    extern __shared__ __align__(16) float staged[];
    __shared__ __align__(16) float red[2 * 8];
    grid_dep_launch();
    const int team = TEAM ? TEAM : any_team;
    const int tid = threadIdx.x, t = tid % team, slot = tid / team;
    const int g = blockIdx.y * gpb + slot % gpb, rslot = slot / gpb;
    const bool mine = rslot < rpb && g < groups;
    grid_dep_wait();
    const int64_t D = (int64_t)groups * width, step = (int64_t)gridDim.x * rpb;
    const float inv = 1.f / width;
    const int g0 = blockIdx.y * gpb, nw = min(gpb, groups - g0) * width;
    const float *sw = staged + (slot % gpb * width >> 1) + t * 4, *sb = sw + nw;
    stage_weights(staged, wt ? wt + (int64_t)g0 * width : nullptr, 1.f, nw);
    stage_weights(staged + nw, bias ? bias + (int64_t)g0 * width : nullptr, 0.f, nw);
    __syncthreads();
    int turn = 0;
    for (int64_t r0 = (int64_t)blockIdx.x * rpb; r0 < rows; r0 += step) {
        const int64_t r = r0 + rslot;
        const bool live = mine && r < rows;
        const T *px = x + r * ldx + (int64_t)g * width + t * 8;
        T *py = y + r * D + (int64_t)g * width + t * 8;
        typename Raw8<T>::type raw[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw[i] = {};
            if (live && (t + i * team) * 8 < width) load_raw8(px + i * team * 8, raw[i]);
        }
        uint64_t v[4], a2[2] = {0ull, 0ull};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            pairs8(raw[i], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) a2[e & 1] = tc::f32x2_add(a2[e & 1], v[e]);
        }
        float s[1] = {both(tc::f32x2_add(a2[0], a2[1]))};
        team_sum(s, team, red, turn);
        const float mu = ln_mean(s[0], width, inv);
        const uint64_t m2 = tc::f32x2(-mu, -mu);
        a2[0] = a2[1] = 0ull;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if ((t + i * team) * 8 >= width) continue;
            anew(raw[i]);
            pairs8(raw[i], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = tc::f32x2_add(v[e], m2);
                a2[e & 1] = tc::f32x2_fma(v[e], v[e], a2[e & 1]);
            }
        }
        s[0] = both(tc::f32x2_add(a2[0], a2[1]));
        team_sum(s, team, red, turn);
        const float rs = rsqrtf(s[0] * inv + eps);
        const uint64_t rs2 = tc::f32x2(rs, rs);
        if (live && t == 0) {
            if (mean) mean[r * groups + g] = mu;
            if (rstd) rstd[r * groups + g] = rs;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!live || (t + i * team) * 8 >= width) continue;
            uint64_t w[4], b[4], o[4];
            asm volatile("" ::: "memory");               // (not all weights at once: they would not fit the registers)
            staged_pairs(sw + i * team * 4, nw >> 1, w);
            staged_pairs(sb + i * team * 4, nw >> 1, b);
            anew(raw[i]);
            pairs8(raw[i], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = tc::f32x2_fma(tc::f32x2_mul(tc::f32x2_add(v[e], m2), rs2), w[e], b[e]);
            put8(py + i * team * 8, o);
        }
    }
}

// dx, and each block's sums of dy xh and dy over the rows that it met: partial[block][0 dw | 1 db][D].
// The rows come through a ring of stages in shared memory, rpb rows of x and dy each, filled by bulk copies ahead of their
// use, and are read from there twice (sums, then dx): what a thread keeps in registers is the sums over rows, and
// with rows and weights beside them no second block would fit an SM (154 us for 32768 x 2048 that way).
constexpr int LN_STAGES = 4;
struct LnRows {
    int64_t rows, ldx, D;
    int groups, width, team, gpb, rpb, sets, stages;     // sets: of rpb rows, in a stage
};
template <typename T, int NV>
__global__ void __launch_bounds__(LN_THREADS, NV <= 4 ? 2 : 1)
layer_norm_backward_kernel(const T *__restrict__ dy, const T *__restrict__ x, const float *__restrict__ wt,
                           const float *__restrict__ mean, const float *__restrict__ rstd, const LnRows a,
                           T *__restrict__ dx, float *__restrict__ partial, int *d_status)
{
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ __align__(16) float red[2 * 2 * 8];
    __shared__ uint64_t full[LN_STAGES], empty[LN_STAGES];
    __shared__ int abort_flag;
    const int tid = threadIdx.x, t = tid % a.team, slot = tid / a.team, lane = tid & 31;
    const int g0 = blockIdx.y * a.gpb, ng = min(a.gpb, a.groups - g0), gl = slot % a.gpb, rslot = slot / a.gpb;
    const bool mine = rslot < a.rpb && gl < ng;
    const int seg = ng * a.width;                   // entries of a row that this block works
    float *sw = reinterpret_cast<float *>(smem);    // the weights, then the stages: x rows, dy rows
    T *ring = reinterpret_cast<T *>(sw + a.gpb * a.width);
    const int per = a.rpb * a.sets;                 // rows of a stage
    const int64_t stage = (int64_t)2 * per * a.gpb * a.width;
    if (tid == 0) {
        for (int i = 0; i < LN_STAGES; ++i) {
            tc::mbar_init(&full[i], 1);
            tc::mbar_init(&empty[i], LN_THREADS / 32);
        }
        abort_flag = 0;
        tc::fence_mbar_init();
    }
    grid_dep_launch();
    grid_dep_wait();
    for (int i = tid; i < seg; i += LN_THREADS) sw[i] = wt ? wt[(int64_t)g0 * a.width + i] : 1.f;
    __syncthreads();
    const int64_t nchunks = (a.rows + per - 1) / per;
    // (warp 0) chunk number i of this block into its stage, if there is one
    auto fill = [&](int64_t i) {
        const int64_t ch = blockIdx.x + i * gridDim.x;
        if (ch >= nchunks) return;
        const int s = (int)(i % a.stages);
        const bool room = tc::mbar_wait(&empty[s], (uint32_t)((i / a.stages) & 1) ^ 1, &abort_flag, d_status);
        if (!__all_sync(0xffffffffu, room)) return;
        const int64_t r0 = ch * per;
        const int n = (int)min((int64_t)per, a.rows - r0);
        const uint32_t bytes = (uint32_t)(seg * sizeof(T));
        if (lane == 0) tc::mbar_arrive_expect_tx(&full[s], 2 * n * bytes);
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int64_t ld = k == 0 ? a.ldx : a.D;
            const T *src = (k == 0 ? x : dy) + r0 * ld + (int64_t)g0 * a.width;
            T *dst = ring + s * stage + (int64_t)k * per * seg;
            if (ld == seg) {                        // rows back to back
                if (lane == 0) tc::bulk_load(dst, src, n * bytes, &full[s]);
            } else {
                for (int r = lane; r < n; r += 32) tc::bulk_load(dst + (int64_t)r * seg, src + r * ld, bytes, &full[s]);
            }
        }
    };
    if (tid < 32)
        for (int i = 0; i < a.stages; ++i) fill(i);
    uint64_t aw[NV][4], ab[NV][4];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) aw[i][e] = ab[i][e] = 0ull;
    const float inv = 1.f / a.width;
    int turn = 0;
    int64_t it = 0;
    for (int64_t ch = blockIdx.x; ch < nchunks; ch += gridDim.x, ++it) {
        if (tid < 32 && it > 0) fill(it - 1 + a.stages);
        const int st = (int)(it % a.stages);
        const float *pw = sw + gl * a.width;
        tc::mbar_wait(&full[st], (uint32_t)((it / a.stages) & 1), &abort_flag, d_status);
#pragma unroll 2
        for (int q = 0; q < a.sets; ++q) {
            const int lr = q * a.rpb + rslot;
            const int64_t r = ch * per + lr;
            const bool live = mine && r < a.rows;
            // (x - mu, then times rstd: x rstd - mu rstd would leave a rounding of mu rstd where x is mu)
            const float rs = live ? rstd[r * a.groups + g0 + gl] : 0.f, mu = live ? mean[r * a.groups + g0 + gl] : 0.f;
            const T *px = ring + st * stage + (int64_t)lr * seg + gl * a.width, *pd = px + (int64_t)per * seg;
            const uint64_t rs2 = tc::f32x2(rs, rs), m2 = tc::f32x2(-mu, -mu);
            uint64_t s0 = 0ull, s1 = 0ull;
            if (live) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (t + i * a.team) * 8;
                    if (c >= a.width) continue;
                    uint64_t xv[4], dv[4], w[4];
                    load_pairs(px + c, xv);
                    load_pairs(pd + c, dv);
                    load_pairs(pw + c, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t xh = tc::f32x2_mul(tc::f32x2_add(xv[e], m2), rs2), z = tc::f32x2_mul(dv[e], w[e]);
                        s0 = tc::f32x2_add(s0, z);
                        s1 = tc::f32x2_fma(z, xh, s1);
                        aw[i][e] = tc::f32x2_fma(dv[e], xh, aw[i][e]);
                        ab[i][e] = tc::f32x2_add(ab[i][e], dv[e]);
                    }
                }
            }
            float s[2] = {both(s0), both(s1)};
            __syncwarp();
            team_sum(s, a.team, red, turn);
            // rs (z - m0 - xh m1)
            const float c0 = -rs * s[0] * inv, c1 = -rs * s[1] * inv;
            const uint64_t c02 = tc::f32x2(c0, c0), c12 = tc::f32x2(c1, c1);
            if (live) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int c = (t + i * a.team) * 8;
                    if (c >= a.width) continue;
                    uint64_t xv[4], dv[4], w[4], o[4];
                    load_pairs(px + c, xv);
                    load_pairs(pd + c, dv);
                    load_pairs(pw + c, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = tc::f32x2_fma(tc::f32x2_mul(dv[e], w[e]), rs2, tc::f32x2_fma(tc::f32x2_mul(tc::f32x2_add(xv[e], m2), rs2), c12, c02));
                    put8(dx + r * a.D + (int64_t)(g0 + gl) * a.width + c, o);
                }
            }
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&empty[st]);
    }
    tc::settle_copies(&abort_flag);
    if (!partial) return;
    // the rows of a block side by side: their sums meet in shared memory, in order (every stage that was filled has been
    // taken; what is left of the ring is room enough)
    float *sums = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * a.team) * 8;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 f = tc::f32x2_get(k == 0 ? aw[i][e] : ab[i][e]);
                sums[2 * e * LN_THREADS + tid] = f.x;
                sums[(2 * e + 1) * LN_THREADS + tid] = f.y;
            }
            __syncthreads();
            if (rslot == 0 && mine && c < a.width) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    o[e] = 0.f;
                    for (int q = 0; q < a.rpb; ++q) o[e] += sums[e * LN_THREADS + tid + q * a.gpb * a.team];
                }
                float4 *p = reinterpret_cast<float4 *>(partial + ((int64_t)blockIdx.x * 2 + k) * a.D + (int64_t)(g0 + gl) * a.width + c);
                p[0] = make_float4(o[0], o[1], o[2], o[3]);
                p[1] = make_float4(o[4], o[5], o[6], o[7]);
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

// Blocks over the rows: as many as are resident together (a block walks the rows from there on).
template <typename K> int ln_resident(K kern)
{
    int n = 0;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, LN_THREADS, 0) != cudaSuccess || n < 1) n = 1;
    return n;
}
int ln_blocks(const LnShape &s, int64_t rows, int sm_count, int per_sm)
{
    const int64_t need = ceil_div64(rows, s.rpb);
    return (int)std::min<int64_t>(need, std::max(1, per_sm * sm_count / s.ychunks));
}
constexpr size_t LN_ROOM = 220 * 1024;     // of shared memory on an SM
constexpr int LN_GRAD_BLOCKS = 2;          // per SM, resident together: each leaves D partial sums twice
constexpr size_t LN_GRAD_ROOM = 100 * 1024;  // of shared memory for one of them, where its rows are short enough

template <typename T, int NV, int R>
int run_norm(LaunchCtx &ctx, const LnShape &s, const void *x, int64_t ldx, const float *w, const float *b, int64_t rows,
             int groups, int width, float eps, int sm_count, void *y, float *mean, float *rstd)
{
    static const int resident = ln_resident(layer_norm_kernel<T, NV, R>);
    ctx.begin(STAGE_LAYER_NORM);
    launch_kernel(layer_norm_kernel<T, NV, R>, dim3(ln_blocks(s, rows, sm_count, resident), s.ychunks), dim3(LN_THREADS),
                  0, ctx.stream, true, (const T *)x, ldx, w, b, rows, groups, width, eps, s.team, s.gpb, s.rpb, (T *)y,
                  mean, rstd);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

template <typename T, int NV, int TEAM>
int run_norm_wide(LaunchCtx &ctx, const LnShape &s, const void *x, int64_t ldx, const float *w, const float *b, int64_t rows,
                  int groups, int width, float eps, int sm_count, void *y, float *mean, float *rstd)
{
    const auto kern = layer_norm_wide_kernel<T, NV, TEAM>;
    static const int fitting = ln_resident(kern);
    const size_t smem = (size_t)2 * s.gpb * width * sizeof(float);
    if (!ensure_dynamic_smem((const void *)kern, smem)) return SWIMBA_ERR_CUDA;
    const int resident = std::max(1, std::min<int>(fitting, (int)(LN_ROOM / smem)));
    ctx.begin(STAGE_LAYER_NORM);
    launch_kernel(kern, dim3(ln_blocks(s, rows, sm_count, resident), s.ychunks), dim3(LN_THREADS), smem, ctx.stream, true,
                  (const T *)x, ldx, w, b, rows, groups, width, eps, s.team, s.gpb, s.rpb, (T *)y, mean, rstd);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

// Sets of rows a stage of the gradient's ring holds: short rows come several at a time, so that one wait serves them.
int ln_sets(size_t es, const LnShape &s, int width)
{
    const size_t one = 2 * (size_t)s.rpb * s.gpb * width * es;
    return (int)std::max<size_t>(1, std::min<size_t>(4, 24 * 1024 / one));
}

template <typename T, int NV>
int run_backward(LaunchCtx &ctx, const LnShape &s, const void *dy, const void *x, int64_t ldx, const float *w,
                 const float *mean, const float *rstd, int64_t rows, int groups, int width, int sm_count, void *dx,
                 float *partial)
{
    auto kern = layer_norm_backward_kernel<T, NV>;
    const size_t weights = (size_t)s.gpb * width * sizeof(float);
    const int sets = ln_sets(sizeof(T), s, width);
    const size_t stage = (size_t)2 * sets * s.rpb * s.gpb * width * sizeof(T);
    const int stages = LN_GRAD_ROOM > weights ? (int)std::min<size_t>(LN_STAGES, (LN_GRAD_ROOM - weights) / stage) : 0;
    const LnRows a{rows, ldx, (int64_t)groups * width, groups, width, s.team, s.gpb, s.rpb, sets, std::max(1, stages)};
    const size_t smem = std::max<size_t>(weights + a.stages * stage, LN_THREADS * 8 * sizeof(float));
    if (!ensure_dynamic_smem((const void *)kern, smem)) return SWIMBA_ERR_CUDA;
    ctx.begin(STAGE_LAYER_NORM_BACKWARD);
    launch_kernel(kern, dim3(ln_blocks(s, rows, sm_count, LN_GRAD_BLOCKS), s.ychunks), dim3(LN_THREADS), smem, ctx.stream,
                  true, (const T *)dy, (const T *)x, w, mean, rstd, a, (T *)dx, partial, ctx.d_status);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace

// Rows (or sets of rpb rows) a thread of few places takes at a time: enough bytes in flight without spilling.
constexpr int ln_rows(int nv) { return nv == 1 ? 4 : 2; }

int launch_layer_norm(LaunchCtx &ctx, int dtype, const void *x, int64_t ldx, const float *w, const float *b, int64_t rows,
                      int groups, int width, float eps, int sm_count, void *y, float *mean, float *rstd)
{
    const LnShape s = ln_shape(groups, width, LN_FORWARD_PLACES, LN_FORWARD_ROOM);
#define LN_ARGS ctx, s, x, ldx, w, b, rows, groups, width, eps, sm_count, y, mean, rstd
#define LN_RUN(T) (s.nv == 1   ? run_norm<T, 1, ln_rows(1)>(LN_ARGS) : s.nv == 2 ? run_norm<T, 2, ln_rows(2)>(LN_ARGS) \
                   : s.nv == 4 ? s.team == 32 ? run_norm_wide<T, 4, 32>(LN_ARGS) : run_norm_wide<T, 4, 0>(LN_ARGS)     \
                   : s.team == 32 ? run_norm_wide<T, 8, 32>(LN_ARGS) : run_norm_wide<T, 8, 0>(LN_ARGS))
    return dtype == SWIMBA_DTYPE_FP32 ? LN_RUN(float) : LN_RUN(__nv_bfloat16);
#undef LN_ARGS
#undef LN_RUN
}

size_t layer_norm_partial_bytes(int64_t rows, int groups, int width, int sm_count)
{
    const LnShape s = ln_shape(groups, width, LN_BACKWARD_PLACES, INT_MAX);
    return (size_t)ln_blocks(s, rows, sm_count, LN_GRAD_BLOCKS) * 2 * groups * width * sizeof(float);
}

int launch_layer_norm_backward(LaunchCtx &ctx, int dtype, const void *dy, const void *x, int64_t ldx, const float *w,
                               const float *mean, const float *rstd, int64_t rows, int groups, int width, int sm_count,
                               void *dx, float *dw, float *db, float *partial)
{
    const LnShape s = ln_shape(groups, width, LN_BACKWARD_PLACES, INT_MAX);
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
                  ln_blocks(s, rows, sm_count, LN_GRAD_BLOCKS), D, dw, db);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace swimba
