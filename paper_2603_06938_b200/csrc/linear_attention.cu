// Linear attention with a decay for each head: the CUDA-core kernel (fp32, and bf16 heads of more than 128
// entries, which the tensor-core kernels do not take), the chain of segment states, the sum over shared heads and the
// single-token step.  What a job is: la.h.
#include <algorithm>
#include <type_traits>

#include "la.h"

namespace swimba {

namespace {

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p)
{
    const uint2 r = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16),
                       __uint_as_float(r.y & 0xffff0000u));
}

constexpr int LA_C = 32;         // tokens of a chunk
constexpr int LA_COLS = 64;      // columns of v (and o) a block of 256 threads works

// Shared memory of a block, for jobs of up to dk entries: the chunk in fp32 (rows of q and k padded by four, so that threads on
// neighbouring rows read different banks), the scores, the state, and the next chunk as it arrives.
struct ChunkSmem {
    int q, k, v, wv, p, s, stage, bytes;      // (offsets in floats; bytes in all)
};
__host__ __device__ constexpr ChunkSmem chunk_smem(int dk, int elt, bool state_only)
{
    ChunkSmem m{};
    int at = 0;
    m.q = at;     at += state_only ? 0 : LA_C * (dk + 4);
    m.k = at;     at += LA_C * (dk + 4);
    m.v = at;     at += state_only ? 0 : LA_C * LA_COLS;
    m.wv = at;    at += LA_C * LA_COLS;
    m.p = at;     at += state_only ? 0 : LA_C * (LA_C + 4);
    m.s = at;     at += dk * LA_COLS;
    m.stage = at;
    m.bytes = at * 4 + LA_C * ((state_only ? 1 : 2) * dk + LA_COLS) * elt;
    return m;
}

__device__ __forceinline__ void copy16(void *dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src) : "memory");
}

// R rows of o by two columns a thread: o_i = sum_{j <= i} P_ij v_j + w_i sum_d q_id S_d.  The rows i0 .. i0 + R - 1 lie in one
// group of four, whose scores behind the diagonal are never touched (what a later token holds must not matter, NaN or not).
template <int R>
__device__ __forceinline__ void chunk_carried(const float *sq, int ldq, const float *ss, int dk, float (&acc)[R][2])
{
#pragma unroll 2
    for (int d = 0; d < dk; d += 4) {
        float4 qq[R];
#pragma unroll
        for (int r = 0; r < R; ++r) qq[r] = *reinterpret_cast<const float4 *>(sq + r * ldq + d);
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            const float2 s = *reinterpret_cast<const float2 *>(ss + (d + z) * LA_COLS);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float x = z == 0 ? qq[r].x : z == 1 ? qq[r].y : z == 2 ? qq[r].z : qq[r].w;
                acc[r][0] = fmaf(x, s.x, acc[r][0]);
                acc[r][1] = fmaf(x, s.y, acc[r][1]);
            }
        }
    }
}
template <int R>
__device__ __forceinline__ void chunk_inside(const float *sp, const float *sv, int i0, float (&acc)[R][2])
{
    const int diag = i0 & ~3;
    for (int j = 0; j <= diag; j += 4) {
        float4 p[R];
#pragma unroll
        for (int r = 0; r < R; ++r) p[r] = *reinterpret_cast<const float4 *>(sp + r * (LA_C + 4) + j);
#pragma unroll
        for (int z = 0; z < 4; ++z) {
            const float2 s = *reinterpret_cast<const float2 *>(sv + (j + z) * LA_COLS);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float x = z == 0 ? p[r].x : z == 1 ? p[r].y : z == 2 ? p[r].z : p[r].w;
                if (j + z <= i0 + r) {
                    acc[r][0] = fmaf(x, s.x, acc[r][0]);
                    acc[r][1] = fmaf(x, s.y, acc[r][1]);
                }
            }
        }
    }
}

// S_d <- (hi + lo) S_d + sum_t k_td (w v)_t, R rows d by two columns at a time; group rg of `groups` takes every so many-th R.
// (Rows behind the last token are zeros.)
template <int R>
__device__ __forceinline__ void chunk_state(const float *sk, int ld, const float *swv, float *ss, int rg, int groups, int dk, int n,
                                            float hi, float lo)
{
    for (int d = rg * R; d < dk; d += groups * R) {
        float u[R][2];
#pragma unroll
        for (int r = 0; r < R; ++r) u[r][0] = u[r][1] = 0.f;
#pragma unroll 4
        for (int t = 0; t < (n + 3 & ~3); ++t) {
            const float2 x = *reinterpret_cast<const float2 *>(swv + t * LA_COLS);
#pragma unroll
            for (int r = 0; r < R; r += 4) {
                const float4 kk = *reinterpret_cast<const float4 *>(sk + t * ld + d + r);
                const float kr[4] = {kk.x, kk.y, kk.z, kk.w};
#pragma unroll
                for (int z = 0; z < 4; ++z) {
                    u[r + z][0] = fmaf(kr[z], x.x, u[r + z][0]);
                    u[r + z][1] = fmaf(kr[z], x.y, u[r + z][1]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float2 *at = reinterpret_cast<float2 *>(ss + (d + r) * LA_COLS);
            const float2 s = *at;
            *at = make_float2(fmaf(hi, s.x, fmaf(lo, s.x, u[r][0])), fmaf(hi, s.y, fmaf(lo, s.y, u[r][1])));
        }
    }
}

// One (job, sequence, head, segment) and LA_COLS columns of its v, by chunks of 32 tokens in fp32, with r the place of a token
// in the order of the walk and the state S in shared memory:
//   P_ij = scale_p lambda^(i - j) q_i k_j  (j <= i),   o_i = sum_j P_ij v_j + scale_c lambda^(i + first) S^T q_i
//   S <- lambda^n S + sum_j k_j (scale_a lambda^(n - j - first) v_j)^T
// (first = 1 walking forward, 0 backward).  A thread works a few rows by two columns of each product.  Chunks, because a
// recurrence token by token spends four operations on an entry of the state and as many shuffles as operations on its sums:
// gradients of 2 x 1000 tokens, 16 heads of 128 x 128, fp32: 556 us, by tokens 1139; 256 tokens of 8 heads of 16 x 64: 36 us,
// by tokens in segments 63.  Bound by reads of shared memory (a chunk of 128 keys takes 18000 cycles, a third of them in
// fused multiply-adds) and, with few heads, by the latency of a chunk's four phases (6000 cycles).
// STATE_ONLY: from a zero state, and only the end state is kept (in seg).
template <typename T, bool STATE_ONLY>
__global__ void __launch_bounds__(256)
la_chunks_kernel(const __grid_constant__ LaArgs a, int dk_most)
{
    extern __shared__ __align__(16) float smf[];
    __shared__ float pow_hi[LA_C + 1], pow_lo;           // lambda^m; the rest of lambda^LA_C, which multiplies up
    const ChunkSmem m = chunk_smem(dk_most, sizeof(T), STATE_ONLY);
    float *sq = smf + m.q, *sk = smf + m.k, *sv = smf + m.v, *swv = smf + m.wv, *sp = smf + m.p, *ss = smf + m.s;
    T *stage = reinterpret_cast<T *>(smf + m.stage);
    grid_dep_launch();
    grid_dep_wait();
    int64_t id = blockIdx.x;
    const int nrun = STATE_ONLY ? a.nseg - 1 : a.nseg;   // (the last segment's end state enters nothing)
    const int seg = (int)(id % nrun);
    id /= nrun;
    const int h = (int)(id % a.H);
    id /= a.H;
    const int b = (int)(id % a.B);
    const LaJob &j = a.job[id / a.B];
    const int c0 = blockIdx.y * LA_COLS, dk = j.dk, dv = j.dv;
    if (c0 >= dv) return;
    const int nc = min(LA_COLS, dv - c0), ld = dk + 4, tid = threadIdx.x;
    const bool rev = j.reverse != 0;
    const double l2 = la_log2_decay(a.log_decay[h]);
    if (tid <= LA_C) {
        const double l = exp2(l2 * tid);
        pow_hi[tid] = (float)l;
        if (tid == LA_C) pow_lo = (float)(l - (double)(float)l);
    }
    // segments are numbered in the order of the walk; w counts its tokens
    const int place = rev ? a.nseg - 1 - seg : seg, begin = place * a.seg_len, end = min(a.L, begin + a.seg_len);
    const int w0 = rev ? a.L - end : begin, w1 = w0 + (end - begin);
    const T *q = (const T *)j.q + (int64_t)b * a.L * j.ldq + (int64_t)(h / j.rq) * dk;
    const T *k = (const T *)j.k + (int64_t)b * a.L * j.ldk + (int64_t)(h / j.rk) * dk;
    const T *v = (const T *)j.v + (int64_t)b * a.L * j.ldv + (int64_t)(h / j.rv) * dv + c0;
    const int64_t bh = (int64_t)b * a.H + h, ssize = (int64_t)dk * dv;
    constexpr int EPC = 16 / sizeof(T);                  // entries of a copy (rows and widths are multiples of it)

    // the chunk at w: rows of k, then q, then v
    auto fetch = [&](int w) {
        const int n = min(LA_C, w1 - w);
        auto rows = [&](const T *src, int64_t lds, int width, T *dst) {
            const int per = width / EPC;
            const uint32_t inv = (1u << 20) / per + 1;       // (i / per for i per < 2^20)
            for (int i = tid; i < n * per; i += 256) {
                const int r = i * inv >> 20, c = (i - r * per) * EPC, t = rev ? a.L - 1 - (w + r) : w + r;
                copy16(dst + r * width + c, src + t * lds + c);
            }
        };
        rows(k, j.ldk, dk, stage);
        if (!STATE_ONLY) rows(q, j.ldq, dk, stage + LA_C * dk);
        rows(v, j.ldv, nc, stage + LA_C * dk * (STATE_ONLY ? 1 : 2));
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (w0 < w1) fetch(w0);

    // the state, zero behind the columns
    const float *from = STATE_ONLY ? nullptr
                        : seg > 0  ? j.seg + (bh * a.nseg + seg) * ssize
                        : j.s_in   ? j.s_in + bh * ssize
                                   : nullptr;
    // (four entries side by side in memory at a time: of a row d, or of a column)
    auto state_at = [&](int i, int &d, int &c) {
        if (j.transposed) { d = i >> 4; c = (i & 15) * 4; }
        else { d = ((i >> 7) * 2 + (i & 1)) * 4; c = i >> 1 & 63; }
        return j.transposed ? (int64_t)d * dv + c0 + c : (int64_t)(c0 + c) * dk + d;
    };
    for (int i = tid; i < dk * (LA_COLS / 4); i += 256) {
        int d, c;
        const int64_t at = state_at(i, d, c);
        const float4 x = from && c < nc ? *reinterpret_cast<const float4 *>(from + at) : make_float4(0.f, 0.f, 0.f, 0.f);
        float *to = ss + d * LA_COLS + c;
        if (j.transposed) *reinterpret_cast<float4 *>(to) = x;
        else { to[0] = x.x; to[LA_COLS] = x.y; to[2 * LA_COLS] = x.z; to[3 * LA_COLS] = x.w; }
    }
    // threads by column pairs and rows: 32, 16 or 8 pairs wide, as the columns need
    const int pairs = nc > 32 ? 32 : nc > 16 ? 16 : 8;
    const int cp = (tid % pairs) * 2, rg = tid / pairs;      // row group: 4, 2 or 1 rows
    const bool column = cp < nc;
    const int first = rev ? 0 : 1;

    for (int w = w0; w < w1; w += LA_C) {
        const int n = min(LA_C, w1 - w);
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();                                     // the chunk is there, and the one in front is done with
        auto unpack = [&](const T *src, int width, int lds, float *dst) {
            const int per = width / 4;
            const uint32_t inv = (1u << 20) / per + 1;
#pragma unroll 2
            for (int i = tid; i < LA_C * per; i += 256) {
                const int r = i * inv >> 20, c = (i - r * per) * 4;
                *reinterpret_cast<float4 *>(dst + r * lds + c) = r < n ? load4(src + r * width + c) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        };
        unpack(stage, dk, ld, sk);
        if (!STATE_ONLY) unpack(stage + LA_C * dk, dk, ld, sq);
        {
            const T *src = stage + LA_C * dk * (STATE_ONLY ? 1 : 2);
            for (int i = tid; i < LA_C * (LA_COLS / 4); i += 256) {
                const int r = i / (LA_COLS / 4), c = i % (LA_COLS / 4) * 4;
                const float4 x = r < n && c < nc ? load4(src + r * nc + c) : make_float4(0.f, 0.f, 0.f, 0.f);
                if (!STATE_ONLY) *reinterpret_cast<float4 *>(sv + r * LA_COLS + c) = x;
                const float e = r < n ? j.scale_a * pow_hi[n - r - first] : 0.f;
                *reinterpret_cast<float4 *>(swv + r * LA_COLS + c) = make_float4(e * x.x, e * x.y, e * x.z, e * x.w);
            }
        }
        __syncthreads();
        if (w + LA_C < w1) fetch(w + LA_C);
        auto outputs = [&](auto rows) {
            constexpr int R = decltype(rows)::value;
            const int i0 = rg * R;
            float acc[R][2];
#pragma unroll
            for (int r = 0; r < R; ++r) acc[r][0] = acc[r][1] = 0.f;
            if (column && i0 < n) {
                chunk_carried<R>(sq + i0 * ld, ld, ss + cp, dk, acc);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float e = i0 + r < n ? j.scale_c * pow_hi[i0 + r + first] : 0.f;
                    acc[r][0] *= e;
                    acc[r][1] *= e;
                }
            }
            __syncthreads();                                 // scores are there, and S has been read
            if (column && i0 < n) {
                chunk_inside<R>(sp + i0 * (LA_C + 4), sv + cp, i0, acc);
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    if (i0 + r >= n) continue;
                    const int t = rev ? a.L - 1 - (w + i0 + r) : w + i0 + r;
                    const int64_t at = ((int64_t)b * a.L + t) * j.ldo + (int64_t)h * dv + c0 + cp;
                    if (sizeof(T) == 4 || j.o_f32) *reinterpret_cast<float2 *>((float *)j.o + at) = make_float2(acc[r][0], acc[r][1]);
                    else *reinterpret_cast<__nv_bfloat162 *>((__nv_bfloat16 *)j.o + at) = __floats2bfloat162_rn(acc[r][0], acc[r][1]);
                }
            }
        };
        if (!STATE_ONLY) {
            // scores of rows i, i + 16 by columns j, j + 16
            const int i = tid >> 4, jj = tid & 15;
            float s00 = 0.f, s10 = 0.f, s11 = 0.f;           // (i, jj), (i + 16, jj), (i + 16, jj + 16); the fourth is behind
#pragma unroll 2
            for (int d = 0; d < dk; d += 4) {
                const float4 q0 = *reinterpret_cast<const float4 *>(sq + i * ld + d), q1 = *reinterpret_cast<const float4 *>(sq + (i + 16) * ld + d);
                const float4 k0 = *reinterpret_cast<const float4 *>(sk + jj * ld + d), k1 = *reinterpret_cast<const float4 *>(sk + (jj + 16) * ld + d);
                s00 = fmaf(q0.w, k0.w, fmaf(q0.z, k0.z, fmaf(q0.y, k0.y, fmaf(q0.x, k0.x, s00))));
                s10 = fmaf(q1.w, k0.w, fmaf(q1.z, k0.z, fmaf(q1.y, k0.y, fmaf(q1.x, k0.x, s10))));
                s11 = fmaf(q1.w, k1.w, fmaf(q1.z, k1.z, fmaf(q1.y, k1.y, fmaf(q1.x, k1.x, s11))));
            }
            sp[i * (LA_C + 4) + jj] = jj <= i ? j.scale_p * pow_hi[i - jj] * s00 : 0.f;
            sp[(i + 16) * (LA_C + 4) + jj] = j.scale_p * pow_hi[i + 16 - jj] * s10;
            sp[(i + 16) * (LA_C + 4) + jj + 16] = jj <= i ? j.scale_p * pow_hi[i - jj] * s11 : 0.f;
            if (pairs == 32) outputs(std::integral_constant<int, 4>{});
            else if (pairs == 16) outputs(std::integral_constant<int, 2>{});
            else outputs(std::integral_constant<int, 1>{});
        }
        if (column) {                                        // eight rows a thread where there are as many, else four
            if (dk * pairs >= 2048) chunk_state<8>(sk, ld, swv + cp, ss + cp, rg, 256 / pairs, dk, n, pow_hi[n], n == LA_C ? pow_lo : 0.f);
            else chunk_state<4>(sk, ld, swv + cp, ss + cp, rg, 256 / pairs, dk, n, pow_hi[n], n == LA_C ? pow_lo : 0.f);
        }
    }
    __syncthreads();
    float *to = STATE_ONLY ? j.seg + (bh * a.nseg + seg + 1) * ssize
                : seg == a.nseg - 1 && j.s_out ? j.s_out + bh * ssize : nullptr;
    if (to)
        for (int i = tid; i < dk * (LA_COLS / 4); i += 256) {
            int d, c;
            const int64_t at = state_at(i, d, c);
            if (c >= nc) continue;
            const float *x = ss + d * LA_COLS + c;
            *reinterpret_cast<float4 *>(to + at) = j.transposed ? *reinterpret_cast<const float4 *>(x)
                                                                : make_float4(x[0], x[LA_COLS], x[2 * LA_COLS], x[3 * LA_COLS]);
        }
}

}  // namespace

// seg[.., i] holds the end state of piece i - 1 from a zero entry (i >= 1); on exit the state that enters piece i.  One
// thread per four entries walks a sequence's pieces.  (7 us for 9 pieces of 16 heads of 64 x 64: a launch and nine latencies.)
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
    const float log_decay = a.log_decay[h];
    // every piece but the sequence's last, the first of a walk backward, is whole (and behind the last there may be empty ones)
    const int len = a.seg_len / a.per, all = a.nseg * a.per, last = (a.nseg - 1) * a.per;
    const LaDecay whole = la_decay(log_decay, len);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (j.s_in) s = *reinterpret_cast<const float4 *>(j.s_in + blockIdx.y * ssize + i);
    float *p = j.seg + (int64_t)blockIdx.y * all * ssize + i;
#pragma unroll 4
    for (int g = 1; g <= last; ++g) {
        const float4 l = *reinterpret_cast<const float4 *>(p + g * ssize);
        const int tokens = j.reverse ? a.L - (all - g) * len : len;        // of the piece in front
        const LaDecay lam = tokens >= len ? whole : la_decay(log_decay, max(0, tokens));
        s.x = fmaf(lam.hi, s.x, fmaf(lam.lo, s.x, l.x));
        s.y = fmaf(lam.hi, s.y, fmaf(lam.lo, s.y, l.y));
        s.z = fmaf(lam.hi, s.z, fmaf(lam.lo, s.z, l.z));
        s.w = fmaf(lam.hi, s.w, fmaf(lam.lo, s.w, l.w));
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

template <typename T> int launch_steps(LaunchCtx &ctx, const LaArgs &a)
{
    int dk = 0, dv = 0;
    for (int i = 0; i < a.njobs; ++i) {
        dk = std::max(dk, a.job[i].dk);
        dv = std::max(dv, a.job[i].dv);
    }
    const unsigned slices = ceil_div(dv, LA_COLS), one = (unsigned)(a.njobs * a.B * a.H);
    const size_t states = chunk_smem(dk, sizeof(T), true).bytes, outputs = chunk_smem(dk, sizeof(T), false).bytes;
    if (!ensure_dynamic_smem((const void *)la_chunks_kernel<T, true>, states) ||
        !ensure_dynamic_smem((const void *)la_chunks_kernel<T, false>, outputs))
        return SWIMBA_ERR_CUDA;
    if (a.nseg > 1) {
        ctx.begin(STAGE_LA_STATES);
        launch_kernel(la_chunks_kernel<T, true>, dim3(one * (a.nseg - 1), slices), dim3(256), states, ctx.stream, true, a, dk);
        ctx.end();
        const int rc = launch_chain(ctx, a);
        if (rc != SWIMBA_OK) return rc;
    }
    ctx.begin(STAGE_LA_CHUNKS);
    launch_kernel(la_chunks_kernel<T, false>, dim3(one * a.nseg, slices), dim3(256), outputs, ctx.stream, true, a, dk);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
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

// One token for each of B sequences: S <- lambda S + v k^T (fp32, from s_in to s_out), o = scale S q.
// A group of LR lanes owns ROWS rows of a head's state at a time, four entries of each row a lane, all of whose
// loads are in flight before the first is used.  Bound by the state's bytes, read and written once: 128 sequences of 16 heads
// of 128 x 128 take 52 us, 5.2 TB/s (a copy reaches 6.6).  Of one sequence a call takes 12 us, half of them the Python binding's
// checks of three strided tensors (the layer norm, one launch too, takes 6).
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
              const void *v, int64_t ldv, const float *s_in, int B, int H, int G, int P, int N, float scale,
              int sm_count, void *o, float *s_out)
{
    const int64_t nwork = (int64_t)B * H * ceil_div(P, ST_ROWS);
    const int threads = nwork * LR >= sm_count * 256 ? 256 : 64;     // (few rows: spread over the SMs)
    launch_kernel(la_step_kernel<T, LR>, dim3((unsigned)ceil_div64(nwork * LR, threads)), dim3(threads), 0, ctx.stream,
                  true, log_decay, (const T *)q, ldq, (const T *)k, ldk, (const T *)v, ldv, s_in, nwork, H, G, P, N,
                  scale, (T *)o, s_out);
}

template <typename T>
void run_step_n(LaunchCtx &ctx, const float *log_decay, const void *q, int64_t ldq, const void *k, int64_t ldk,
                const void *v, int64_t ldv, const float *s_in, int B, int H, int G, int P, int N, float scale,
                int sm_count, void *o, float *s_out)
{
    // lanes per row: no more than the row has groups of four entries
    if (N >= 128) run_step<T, 32>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, sm_count, o, s_out);
    else if (N >= 64) run_step<T, 16>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, sm_count, o, s_out);
    else if (N >= 32) run_step<T, 8>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, sm_count, o, s_out);
    else run_step<T, 4>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, sm_count, o, s_out);
}

}  // namespace

namespace {
// What a segment has at least, by chunks 64 tokens, and what its length is a multiple of by tiles.
constexpr int LA_STEP_SEG = 64, LA_TILE_SEG = 128;
// The most segments a sequence is cut into: by chunks, as many as give every SM two blocks; by tiles, as many
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
        // Waves of blocks times chunks, in chunks: the outputs, and, where sequences are cut, the pass for the states (half of
        // that) and two more launches (about 6).  Measured (us): 1024 tokens of 16 heads of 16 x 64, whole 92, two segments 75,
        // four 50, eight (chosen) 35; gradients of 2 x 1000 tokens of 16 heads of 128 x 128, whole (chosen) 557, two 522; of 256
        // tokens of 8 heads of 16 x 64, whole (chosen) 32, two 32, four 24.
        const int64_t blocks = (int64_t)njobs * B * H * ceil_div(std::max(N, P), LA_COLS);
        double best = 1e30;
        for (int n = 1; n <= std::min(most, ceil_div(L, LA_STEP_SEG)); ++n) {
            const int len = ceil_div(ceil_div(L, n), LA_C), ns = ceil_div(L, len * LA_C);
            const double cost = (double)ceil_div64(blocks * ns, sm_count) * len +
                                (ns > 1 ? 0.5 * ceil_div64(blocks * (ns - 1), sm_count) * len + 6 : 0);
            if (cost >= best) continue;
            best = cost;
            *seg_len = std::min(len * LA_C, L);
            *nseg = ns;
        }
        return;
    }
    // Waves of CTAs times tiles per CTA, in tiles: the outputs, and, where sequences are cut, the pass for the states (about
    // 0.7 of a tile each, in pieces that fill the SMs), their chain (0.15 a piece) and two more launches (about 9).
    // Measured (us), 16 heads of 64 x 64: 65536 tokens, whole 824, five segments 283, nine (chosen) 175, 18 204; 8192 tokens,
    // whole 119, four 50, eight 38, nine 37, 16 46 (chosen: within 2 of the best); 2048 tokens, whole 32, four 23, eight
    // (chosen) 20; 1024 tokens, whole (chosen) 19, two 20, four 19; 4 x 8192 tokens, whole 113, two (chosen) 90, four 110.
    // 16 heads of 128 x 128, 8192 tokens: whole 258, shared walks 173, four segments 123, nine (chosen) 98.
    const int nt = ceil_div(L, LA_TILE_SEG);
    const int64_t items = (int64_t)njobs * B * H;
    const bool wide = P > 64 && (njobs == 1 || N > 64);
    double best = 1e30;
    for (int n = 1; n <= std::min(most, nt); ++n) {
        const int len = ceil_div(nt, n), ns = ceil_div(nt, len);
        double states = 0;
        int pieces = 1;
        if (ns > 1) {
            states = 1e30;
            for (int p = 1; p <= 4 && p * ns <= std::min(most, nt); ++p) {
                if (len % p != 0) continue;
                const double c = 0.7 * ceil_div64(items * (ns - 1) * p, sm_count) * (len / p) + 9 + 0.15 * ns * p;
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
    if (!la_tiles_shape(dtype, a.job[0].dk, a.job[0].dv))
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
    ctx.begin(STAGE_LA_STEP);
    if (dtype == SWIMBA_DTYPE_FP32)
        run_step_n<float>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, sm_count, o, s_out);
    else
        run_step_n<__nv_bfloat16>(ctx, log_decay, q, ldq, k, ldk, v, ldv, s_in, B, H, G, P, N, scale, sm_count, o, s_out);
    ctx.end();
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace swimba
