// Linear attention with a decay for each head: the CUDA-core kernel (fp32, and bf16 head sizes that the
// tensor-core kernel does not take), the chain of segment states, the sum over shared heads and the
// single-token step.  What a job is: la.h.
#include <algorithm>

#include "la.h"

namespace swimba {

namespace {

constexpr int LA_TS = 16;        // tokens staged in shared memory at a time
constexpr int LA_COLS = 64;      // columns of v (and o) a block of 256 threads works

// One (job, sequence, head, segment) and LA_COLS columns of its v: the recurrence token by token with the
// state in registers.  Lane l of a half-warp holds the entries dk = l + 16 m (m < KR) of four columns;
// per token it adds k v, multiplies by the decay and contributes to o, which the sixteen lanes sum.
// STATE_ONLY: from a zero state, and only the end state is kept (in seg).
template <typename T, int KR, bool STATE_ONLY>
__global__ void __launch_bounds__(256, KR <= 8 ? 2 : 1)
la_steps_kernel(const __grid_constant__ LaArgs a)
{
    constexpr int DKP = KR * 16;
    __shared__ float sq[STATE_ONLY ? 1 : LA_TS * DKP], sk[LA_TS * DKP], sv[LA_TS * LA_COLS],
        so[STATE_ONLY ? 1 : LA_TS * LA_COLS];
    grid_dep_launch();
    grid_dep_wait();
    int64_t id = blockIdx.x;
    const int nrun = STATE_ONLY ? a.nseg - 1 : a.nseg;   // (the last segment's end state enters nothing)
    int seg = (int)(id % nrun);
    id /= nrun;
    const int h = (int)(id % a.H);
    id /= a.H;
    const int b = (int)(id % a.B);
    const LaJob &j = a.job[id / a.B];
    const int c0 = blockIdx.y * LA_COLS;
    if (c0 >= j.dv) return;
    const int tid = threadIdx.x, lane16 = tid & 15, col = (tid >> 4) * 4;   // four columns c0 + col ..
    const int dk = j.dk, dv = j.dv;
    const LaDecay lam = la_decay(a.log_decay[h]);
    // segments are numbered in the order of the walk; w counts its tokens
    const int place = j.reverse ? a.nseg - 1 - seg : seg, first = place * a.seg_len, last = min(a.L, first + a.seg_len);
    const int w0 = j.reverse ? a.L - last : first, w1 = w0 + (last - first);
    const T *q = (const T *)j.q + (int64_t)b * a.L * j.ldq + (int64_t)(h / j.rq) * dk;
    const T *k = (const T *)j.k + (int64_t)b * a.L * j.ldk + (int64_t)(h / j.rk) * dk;
    const T *v = (const T *)j.v + (int64_t)b * a.L * j.ldv + (int64_t)(h / j.rv) * dv;
    const int64_t bh = (int64_t)b * a.H + h, ssize = (int64_t)dk * dv;

    auto at = [&](int m, int c) {
        const int64_t d = lane16 + 16 * m, e = c0 + col + c;
        return j.transposed ? d * dv + e : e * dk + d;
    };
    auto inside = [&](int m, int c) { return lane16 + 16 * m < dk && c0 + col + c < dv; };
    float s[KR][4];
    const float *from = STATE_ONLY ? nullptr
                        : seg > 0  ? j.seg + (bh * a.nseg + seg) * ssize
                        : j.s_in   ? j.s_in + bh * ssize
                                   : nullptr;
#pragma unroll
    for (int m = 0; m < KR; ++m)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[m][c] = from && inside(m, c) ? from[at(m, c)] : 0.f;

    for (int w = w0; w < w1; w += LA_TS) {
        const int n = min(LA_TS, w1 - w);
        __syncthreads();
        for (int i = tid; i < n * DKP; i += 256) {
            const int r = i / DKP, d = i % DKP, t = j.reverse ? a.L - 1 - (w + r) : w + r;
            sk[i] = d < dk ? to_f32<T>(k[t * j.ldk + d]) : 0.f;
            if (!STATE_ONLY) sq[i] = d < dk ? to_f32<T>(q[t * j.ldq + d]) : 0.f;
        }
        for (int i = tid; i < n * LA_COLS; i += 256) {
            const int r = i / LA_COLS, e = c0 + i % LA_COLS, t = j.reverse ? a.L - 1 - (w + r) : w + r;
            sv[i] = e < dv ? to_f32<T>(v[t * j.ldv + e]) : 0.f;
        }
        __syncthreads();
        for (int r = 0; r < n; ++r) {
            const float4 v4 = *reinterpret_cast<const float4 *>(sv + r * LA_COLS + col);
            const float vv[4] = {v4.x, v4.y, v4.z, v4.w};
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < KR; ++m) {
                const float kk = sk[r * DKP + lane16 + 16 * m];
                const float qq = STATE_ONLY ? 0.f : sq[r * DKP + lane16 + 16 * m];
                const float ka = kk * j.scale_a;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    // the decay meets the state before the token (forward) or behind it (backward)
                    const float y = s[m][c];
                    const float x = j.reverse ? fmaf(ka, vv[c], y) : fmaf(lam.hi, y, fmaf(lam.lo, y, ka * vv[c]));
                    if (!STATE_ONLY) acc[c] = fmaf(x, qq, acc[c]);
                    s[m][c] = j.reverse ? fmaf(lam.hi, x, lam.lo * x) : x;
                }
            }
            if (!STATE_ONLY) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int o = 8; o > 0; o >>= 1) acc[c] += __shfl_xor_sync(0xffffffffu, acc[c], o);
                if (lane16 < 4) {
                    const float x = lane16 == 0 ? acc[0] : lane16 == 1 ? acc[1] : lane16 == 2 ? acc[2] : acc[3];
                    so[r * LA_COLS + col + lane16] = x * j.scale_c;
                }
            }
        }
        if (!STATE_ONLY) {
            __syncthreads();
            for (int i = tid; i < n * LA_COLS; i += 256) {
                const int r = i / LA_COLS, e = c0 + i % LA_COLS, t = j.reverse ? a.L - 1 - (w + r) : w + r;
                if (e >= dv) continue;
                const int64_t p = ((int64_t)b * a.L + t) * j.ldo + (int64_t)h * dv + e;
                if (j.o_f32) ((float *)j.o)[p] = so[i];
                else ((T *)j.o)[p] = from_f32<T>(so[i]);
            }
        }
    }
    float *to = STATE_ONLY ? j.seg + (bh * a.nseg + seg + 1) * ssize
                : seg == a.nseg - 1 && j.s_out ? j.s_out + bh * ssize : nullptr;
    if (to) {
#pragma unroll
        for (int m = 0; m < KR; ++m)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (inside(m, c)) to[at(m, c)] = s[m][c];
    }
}

}  // namespace

// seg[.., i] holds the end state of piece i - 1 from a zero entry (i >= 1); on exit the state that enters piece i.  One
// thread per four entries walks a sequence's pieces.
__global__ void __launch_bounds__(256)
la_chain_kernel(const __grid_constant__ LaArgs a)
{
    grid_dep_launch();
    grid_dep_wait();
    const LaJob &j = a.job[blockIdx.z];
    const int64_t ssize = (int64_t)j.dk * j.dv;
    const int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 4;
    if (i >= ssize) return;
    const int h = (int)(blockIdx.y % a.H);
    const double l2 = la_log2_decay(a.log_decay[h]);
    // every piece but the sequence's last, the first of a walk backward, is whole (and behind the last there may be empty ones)
    const int len = a.seg_len / a.per, all = a.nseg * a.per, last = (a.nseg - 1) * a.per;
    const float whole = (float)exp2(l2 * len);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (j.s_in) s = *reinterpret_cast<const float4 *>(j.s_in + blockIdx.y * ssize + i);
    float *p = j.seg + (int64_t)blockIdx.y * all * ssize + i;
#pragma unroll 4
    for (int g = 1; g <= last; ++g) {
        const float4 l = *reinterpret_cast<const float4 *>(p + g * ssize);
        const int tokens = j.reverse ? a.L - (all - g) * len : len;        // of the piece in front
        const float lam = tokens >= len ? whole : (float)exp2(l2 * max(0, tokens));
        s.x = fmaf(lam, s.x, l.x);
        s.y = fmaf(lam, s.y, l.y);
        s.z = fmaf(lam, s.z, l.z);
        s.w = fmaf(lam, s.w, l.w);
        *reinterpret_cast<float4 *>(p + g * ssize) = s;
    }
}

namespace {

int launch_chain(LaunchCtx &ctx, const LaArgs &a)
{
    int64_t most = 0;
    for (int i = 0; i < a.njobs; ++i) most = std::max<int64_t>(most, (int64_t)a.job[i].dk * a.job[i].dv);
    ctx.begin(STAGE_LA_CHAIN);
    launch_kernel(la_chain_kernel, dim3((unsigned)ceil_div64(most, 1024), (unsigned)(a.B * a.H), a.njobs), dim3(256), 0,
                  ctx.stream, true, a);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

template <typename T, int KR> int launch_steps_k(LaunchCtx &ctx, const LaArgs &a)
{
    int dv = 0;
    for (int i = 0; i < a.njobs; ++i) dv = std::max(dv, a.job[i].dv);
    const unsigned slices = ceil_div(dv, LA_COLS);
    const unsigned one = (unsigned)(a.njobs * a.B * a.H);
    if (a.nseg > 1) {
        ctx.begin(STAGE_LA_STATES);
        launch_kernel(la_steps_kernel<T, KR, true>, dim3(one * (a.nseg - 1), slices), dim3(256), 0, ctx.stream, true, a);
        ctx.end();
        const int rc = launch_chain(ctx, a);
        if (rc != SWIMBA_OK) return rc;
    }
    ctx.begin(STAGE_LA_STEPS);
    launch_kernel(la_steps_kernel<T, KR, false>, dim3(one * a.nseg, slices), dim3(256), 0, ctx.stream, true, a);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

template <typename T> int launch_steps(LaunchCtx &ctx, const LaArgs &a)
{
    int dk = 0;
    for (int i = 0; i < a.njobs; ++i) dk = std::max(dk, a.job[i].dk);
    if (dk <= 16) return launch_steps_k<T, 1>(ctx, a);
    if (dk <= 32) return launch_steps_k<T, 2>(ctx, a);
    if (dk <= 64) return launch_steps_k<T, 4>(ctx, a);
    if (dk <= 128) return launch_steps_k<T, 8>(ctx, a);
    return launch_steps_k<T, 16>(ctx, a);
}

// out[t, g, n] = sum_i part[t, g r + i, n], four entries a thread, heads in order.
template <typename T>
__global__ void __launch_bounds__(256)
la_head_sum_kernel(const float *__restrict__ part, int64_t nout, int r, int N, T *__restrict__ out)
{
    grid_dep_launch();
    grid_dep_wait();
    const int64_t i = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * 4;
    if (i >= nout) return;
    const float *p = part + (i / N) * r * N + i % N;
    float4 s = *reinterpret_cast<const float4 *>(p);
    for (int h = 1; h < r; ++h) {
        const float4 v = *reinterpret_cast<const float4 *>(p + (int64_t)h * N);
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float4 *>(out + i) = s;
    } else {
        const __nv_bfloat162 a = __floats2bfloat162_rn(s.x, s.y), b = __floats2bfloat162_rn(s.z, s.w);
        *reinterpret_cast<uint2 *>(out + i) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
}

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p)
{
    const uint2 r = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16),
                       __uint_as_float(r.y & 0xffff0000u));
}

// One token for each of B sequences: S <- lambda S + v k^T (fp32, from s_in to s_out), o = scale S q.
// A group of LR lanes owns ROWS rows of a head's state at a time, four entries of each row a lane, all of whose
// loads are in flight before the first is used.  Bound by the state's bytes, read and written once.
constexpr int ST_ROWS = 8;
template <typename T, int LR>
__global__ void __launch_bounds__(256)
la_step_kernel(const float *__restrict__ log_decay, const T *__restrict__ q, int64_t ldq, const T *__restrict__ k,
               int64_t ldk, const T *__restrict__ v, int64_t ldv, const float *s_in, int64_t nwork, int H, int G, int P,
               int N, float scale, T *__restrict__ o, float *s_out)
{
    grid_dep_launch();
    grid_dep_wait();
    const int sub = threadIdx.x % LR;
    const int64_t wk = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) / LR;
    const int pgroups = ceil_div(P, ST_ROWS);
    const bool live = wk < nwork;
    const int64_t bh = live ? wk / pgroups : 0;
    const int p0 = live ? (int)(wk % pgroups) * ST_ROWS : P;
    const int h = (int)(bh % H);
    const int64_t b = bh / H;
    const int g = h / (H / G);
    const LaDecay lam = la_decay(log_decay[h]);
    const int64_t base = (bh * P + p0) * N;
    float acc[ST_ROWS], vv[ST_ROWS];
#pragma unroll
    for (int r = 0; r < ST_ROWS; ++r) {
        acc[r] = 0.f;
        vv[r] = p0 + r < P ? to_f32<T>(v[b * ldv + (int64_t)h * P + p0 + r]) : 0.f;
    }
    for (int n = sub * 4; n < N; n += LR * 4) {
        float4 s[ST_ROWS];
#pragma unroll
        for (int r = 0; r < ST_ROWS; ++r)
            if (p0 + r < P) s[r] = __ldcs(reinterpret_cast<const float4 *>(s_in + base + (int64_t)r * N + n));
        const float4 kk = load4(k + b * ldk + (int64_t)g * N + n), qq = load4(q + b * ldq + (int64_t)g * N + n);
#pragma unroll
        for (int r = 0; r < ST_ROWS; ++r) {
            if (p0 + r >= P) continue;
            s[r].x = fmaf(lam.hi, s[r].x, fmaf(lam.lo, s[r].x, vv[r] * kk.x));
            s[r].y = fmaf(lam.hi, s[r].y, fmaf(lam.lo, s[r].y, vv[r] * kk.y));
            s[r].z = fmaf(lam.hi, s[r].z, fmaf(lam.lo, s[r].z, vv[r] * kk.z));
            s[r].w = fmaf(lam.hi, s[r].w, fmaf(lam.lo, s[r].w, vv[r] * kk.w));
            acc[r] = fmaf(s[r].x, qq.x, fmaf(s[r].y, qq.y, fmaf(s[r].z, qq.z, fmaf(s[r].w, qq.w, acc[r]))));
            __stcs(reinterpret_cast<float4 *>(s_out + base + (int64_t)r * N + n), s[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < ST_ROWS; ++r)
#pragma unroll
        for (int d = LR / 2; d > 0; d >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], d);
    if (sub == 0) {
#pragma unroll
        for (int r = 0; r < ST_ROWS; ++r)
            if (p0 + r < P) o[bh * P + p0 + r] = from_f32<T>(acc[r] * scale);
    }
}

template <typename T, int LR>
void run_step(LaunchCtx &ctx, const float *log_decay, const void *q, int64_t ldq, const void *k, int64_t ldk,
              const void *v, int64_t ldv, const float *s_in, int B, int H, int G, int P, int N, float scale, void *o,
              float *s_out)
{
    const int64_t nwork = (int64_t)B * H * ceil_div(P, ST_ROWS);
    const int threads = nwork * LR >= 148 * 256 ? 256 : 64;     // (few rows: spread over the SMs)
    launch_kernel(la_step_kernel<T, LR>, dim3((unsigned)ceil_div64(nwork * LR, threads)), dim3(threads), 0, ctx.stream,
                  true, log_decay, (const T *)q, ldq, (const T *)k, ldk, (const T *)v, ldv, s_in, nwork, H, G, P, N,
                  scale, (T *)o, s_out);
}

template <typename T>
void run_step_n(LaunchCtx &ctx, const float *log_decay, const void *q, int64_t ldq, const void *k, int64_t ldk,
                const void *v, int64_t ldv, const float *s_in, int B, int H, int G, int P, int N, float scale, void *o,
                float *s_out)
{
    // lanes per row: no more than the row has groups of four entries
    if (N >= 128) run_step<T, 32>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, o, s_out);
    else if (N >= 64) run_step<T, 16>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, o, s_out);
    else if (N >= 32) run_step<T, 8>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, o, s_out);
    else run_step<T, 4>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, o, s_out);
}

}  // namespace

namespace {
// What a segment's length is a multiple of: token-by-token segments have 64 tokens at least, tiles 128.
constexpr int LA_STEP_SEG = 64, LA_TILE_SEG = 128;
// The most segments a sequence is cut into: token by token, as many as give every SM two blocks; by tiles, as many
// as fill four waves (pieces included).
int la_most(bool tiles, int B, int H, int N, int P, int njobs, int sm_count)
{
    const int64_t blocks = (int64_t)njobs * B * H * (tiles ? 1 : ceil_div(std::max(N, P), LA_COLS));
    return (int)std::max<int64_t>(1, (tiles ? 4 : 2) * sm_count / blocks);
}
}  // namespace

void la_plan(int dtype, int B, int L, int H, int N, int P, int njobs, int sm_count, int *seg_len, int *nseg, int *per)
{
    *per = 1;
    const bool tiles = la_tiles_shape(dtype, N, P);
    const int most = la_most(tiles, B, H, N, P, njobs, sm_count);
    if (!tiles) {
        const int len = std::max(LA_STEP_SEG, ceil_div(ceil_div(L, most), 16) * 16);
        *seg_len = std::min(len, L);
        *nseg = ceil_div(L, *seg_len);
        return;
    }
    // Waves of CTAs times tiles per CTA, in tiles: the outputs, and, where sequences are cut, the pass for the states (about
    // 0.7 of a tile each, in pieces that fill the SMs), their chain (0.15 a piece) and two more launches (about 4).
    const int nt = ceil_div(L, LA_TILE_SEG);
    const int64_t items = (int64_t)njobs * B * H;
    const bool wide = P == 128 && (njobs == 1 || N == 128);
    double best = 1e30;
    for (int n = 1; n <= std::min(most, nt); ++n) {
        const int len = ceil_div(nt, n), ns = ceil_div(nt, len);
        double states = 0;
        int pieces = 1;
        if (ns > 1) {
            states = 1e30;
            for (int p = 1; p <= 4 && p * ns <= std::min(most, nt); ++p) {
                if (len % p != 0) continue;
                const double c = 0.7 * ceil_div64(items * (ns - 1) * p, sm_count) * (len / p) + 4 + 0.15 * ns * p;
                if (c < states) { states = c; pieces = p; }
            }
        }
        LaArgs cuts;
        const double cost = n == 1 && wide ? la_cuts(items, nt, sm_count, &cuts) : (double)ceil_div64(items * ns, sm_count) * len + states;
        if (cost < best) {
            best = cost;
            *seg_len = len * LA_TILE_SEG;
            *nseg = ns;
            *per = pieces;
        }
    }
}

size_t la_segment_bytes(int dtype, int B, int L, int H, int N, int P, int njobs, int sm_count)
{
    // the most pieces that a call of up to B sequences and L tokens is cut into; none where sequences stay whole
    const bool tiles = la_tiles_shape(dtype, N, P);
    int64_t most = 0;
    for (int b = 1; b <= B; ++b) {
        const int n = std::min(la_most(tiles, b, H, N, P, njobs, sm_count), ceil_div(L, tiles ? LA_TILE_SEG : LA_STEP_SEG));
        if (n == 1) break;
        most = std::max<int64_t>(most, (int64_t)b * n);
    }
    return (size_t)most * H * N * P * sizeof(float);
}

int launch_la(LaunchCtx &ctx, int dtype, const LaArgs &a, int sm_count)
{
    if (!la_tiles_shape(dtype, a.job[0].dk, a.job[0].dv) || !la_tiles_reach(a))
        return dtype == SWIMBA_DTYPE_FP32 ? launch_steps<float>(ctx, a) : launch_steps<__nv_bfloat16>(ctx, a);
    if (a.nseg > 1) {
        int rc = launch_la_tiles(ctx, a, true, sm_count);
        if (rc == SWIMBA_OK) rc = launch_chain(ctx, a);
        if (rc != SWIMBA_OK) return rc;
    }
    return launch_la_tiles(ctx, a, false, sm_count);
}

int launch_la_head_sum(LaunchCtx &ctx, int dtype, const float *part, int64_t T, int G, int r, int N, void *out)
{
    const int64_t nout = T * G * N;
    const dim3 grid((unsigned)ceil_div64(nout, 1024));
    ctx.begin(STAGE_LA_HEAD_SUM);
    if (dtype == SWIMBA_DTYPE_FP32)
        launch_kernel(la_head_sum_kernel<float>, grid, dim3(256), 0, ctx.stream, true, part, nout, r, N, (float *)out);
    else
        launch_kernel(la_head_sum_kernel<__nv_bfloat16>, grid, dim3(256), 0, ctx.stream, true, part, nout, r, N,
                      (__nv_bfloat16 *)out);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

int launch_la_step(LaunchCtx &ctx, int dtype, const float *log_decay, const void *q, int64_t ldq, const void *k,
                   int64_t ldk, const void *v, int64_t ldv, const float *s_in, int B, int H, int G, int P, int N,
                   float scale, int sm_count, void *o, float *s_out)
{
    (void)sm_count;
    ctx.begin(STAGE_LA_STEP);
    if (dtype == SWIMBA_DTYPE_FP32)
        run_step_n<float>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, o, s_out);
    else
        run_step_n<__nv_bfloat16>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, o, s_out);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace swimba
