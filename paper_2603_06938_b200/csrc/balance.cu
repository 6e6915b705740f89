// Balance loss of a router, its per-expert counts and gradients (Background, "Mixture of Experts": what keeps a
// trained router from sending every token to the same few experts):
//   p_t = softmax(W_r u_t) over all E,   f_e = counts_e / (k Tv),   m_e = mean over the Tv valid tokens of p_te
//   loss = coef E sum_e f_e m_e          (coef when all experts get the same share)
//   dg_te = coef E / Tv p_te (f_e - sum_j f_j p_tj),   dW_r = sum_t dg_t u_t^T,   du_t = W_r^T dg_t
// The shares f are constants of the differentiation.  They lie near 1 / E, and the gradient depends only on how far
// they differ from it, so that difference is taken from the whole numbers before anything is rounded.
// The counts come first (from the active sets alone), so that one pass over u gives the loss and the gradients.
#include <algorithm>
#include <cstddef>

#include "la.h"
#include "tc05.cuh"

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

// ------------------------------------------------------------------------------------------
// Up to 16 experts, bf16, F a multiple of 16 up to 2048: one pass over u for everything.  A block keeps 16 tokens of u in
// shared memory and its sixteen warps a share of the features each; all products are m16n8k16:
//   logits  u [16 tokens, features] x W^T, the warps' parts added in order; softmax and dg with an expert a lane
//   dW      dg^T [experts, 16 tokens] x u, in registers over all the block's tokens (one partial sum a block)
//   du      dg [16 tokens, experts] x W, staged where u stood and copied out from there
// dg enters the products as bf16 parts: three for dW, an fp32 result (2^-24 of it), two for du, which is bf16 itself.  With
// up to eight experts the first two parts lie side by side, as the rows (dW) or the depth (du) of one product.
// The work between two barriers is short and its latency counts: eight warps that also made the copies took 88 us for 32768
// tokens, F = 2048, E = 8 (FMA kernels with u read twice: 284 us for the call).  Now the call takes 81 us (floor 41), counts
// and sums included (E = 16: 108): 268 MB in the main pass, whose warps wait at its barriers more than for memory.
// ------------------------------------------------------------------------------------------
constexpr int BF_TOK = 16, BF_WARPS = 16, BF_NT = 16;      // tokens of a tile, warps, most n-tiles of 8 features a warp has
constexpr int BF_MATH = BF_WARPS * 32, BF_THREADS = BF_MATH + 32;        // and one warp for the copies
constexpr int BF_COUNT_HERE = 8192;                         // entries that every block counts by itself

__device__ __forceinline__ void bf_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
        "{%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void bf_ldmatrix(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void bf_ldmatrix_trans(uint32_t addr, uint32_t (&r)[4])
{
    tc::ldmatrix_x4_trans(addr, r[0], r[1], r[2], r[3]);
}

template <int EP> struct BfSmall {
    uint64_t full[2], done[2];
    int abort_flag;
    uint32_t ok;                                            // tokens of the tile that count
    int total[SWIMBA_MAX_EXPERTS + 1];
    alignas(16) float part[BF_WARPS][BF_TOK][EP];
    alignas(16) __nv_bfloat16 dg[3][BF_TOK][24];           // parts of dg (rows of 48 bytes); EP = 8: [0] the first two side by side
    float psum[BF_TOK][EP];
};
static_assert(offsetof(BfSmall<8>, part) % 16 == 0 && offsetof(BfSmall<8>, dg) % 16 == 0 && offsetof(BfSmall<16>, dg) % 16 == 0, "read in pairs and rows of 16 bytes");

template <int EP>
__global__ void __launch_bounds__(BF_THREADS, 1)
balance_fused_kernel(const __nv_bfloat16 *__restrict__ u, const __nv_bfloat16 *__restrict__ W,
                     const int32_t *__restrict__ idx, const uint8_t *__restrict__ valid, int64_t Tn, int F, int E, int k,
                     float coef, int *__restrict__ cnt, int ncnt, bool count_here, bool check, __nv_bfloat16 *__restrict__ du,
                     float *__restrict__ part, float *__restrict__ mean_part, int *d_status)
{
    extern __shared__ __align__(16) uint8_t smem[];
    const int pitch = F * 2 + 16;                           // (rows 16 bytes apart in the banks)
    BfSmall<EP> &sm = *reinterpret_cast<BfSmall<EP> *>(smem);
    uint8_t *sW = smem + (sizeof(BfSmall<EP>) + 15) / 16 * 16, *sU = sW + EP * pitch;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int64_t ntiles = (Tn + BF_TOK - 1) / BF_TOK;
    if (tid == 0) {
        tc::mbar_init(&sm.full[0], 1);
        tc::mbar_init(&sm.full[1], 1);
        tc::mbar_init(&sm.done[0], BF_WARPS);
        tc::mbar_init(&sm.done[1], BF_WARPS);
        sm.abort_flag = 0;
        tc::fence_mbar_init();
    }
    for (int i = tid; i < 3 * BF_TOK * 24; i += BF_THREADS) (&sm.dg[0][0][0])[i] = __float2bfloat16_rn(0.f);
    __syncthreads();
    grid_dep_launch();
    grid_dep_wait();
    if (warp == BF_WARPS) {
        // ---- copies: a row a lane; a tile's du goes out before the tile after next comes in
        auto load = [&](int64_t t, int s) {
            if (t >= ntiles) return;
            const int n = (int)min((int64_t)BF_TOK, Tn - t * BF_TOK);
            if (lane == 0) tc::mbar_arrive_expect_tx(&sm.full[s], (uint32_t)(n * F * 2));
            __syncwarp();
            if (lane < n) tc::bulk_load(sU + (s * BF_TOK + lane) * pitch, u + (t * BF_TOK + lane) * F, (uint32_t)(F * 2), &sm.full[s]);
        };
        load(blockIdx.x, 0);
        load((int64_t)blockIdx.x + gridDim.x, 1);
        int64_t it = 0;
        for (int64_t t = blockIdx.x; t < ntiles; t += gridDim.x, ++it) {
            const int s = (int)(it & 1);
            const bool done = tc::mbar_wait(&sm.done[s], (uint32_t)((it >> 1) & 1), &sm.abort_flag, d_status);
            if (!__all_sync(0xffffffffu, done)) break;
            if (du && lane < BF_TOK && t * BF_TOK + lane < Tn) {
                tc::bulk_store(du + (t * BF_TOK + lane) * F, sU + (s * BF_TOK + lane) * pitch, (uint32_t)(F * 2));
                tc::bulk_commit_group();
                tc::bulk_wait_read_all();
            }
            __syncwarp();
            load(t + 2 * (int64_t)gridDim.x, s);
        }
        tc::settle_copies(&sm.abort_flag);
        return;
    }
    // (from here on the warps that calculate)
    auto meet = [] { tc::named_bar_sync(1, BF_MATH); };
    for (int i = tid; i < EP * (F / 8); i += BF_MATH) {
        const int e = i / (F / 8), c = i % (F / 8);
        *reinterpret_cast<uint4 *>(sW + e * pitch + c * 16) =
            e < E ? *reinterpret_cast<const uint4 *>(W + (int64_t)e * F + c * 8) : make_uint4(0, 0, 0, 0);
    }
    if (count_here) {
        for (int i = tid; i <= E; i += BF_MATH) sm.total[i] = 0;
        meet();
        for (int64_t i = tid; i < Tn * k; i += BF_MATH) {
            const int64_t t = i / k;
            if (valid && !valid[t]) continue;
            if (i % k == 0) atomicAdd(&sm.total[E], 1);
            const int e = idx[i];
            if ((unsigned)e < (unsigned)E) atomicAdd(&sm.total[e], 1);
            else if (check) atomicCAS(d_status, 0, SWIMBA_ERR_DEVICE_BOUNDS);
        }
        meet();
        if (blockIdx.x == 0)
            for (int i = tid; i <= E; i += BF_MATH) cnt[i] = sm.total[i];
    } else {
        for (int i = tid; i <= E; i += BF_MATH) {
            int v = 0;
#pragma unroll 8
            for (int b = 0; b < ncnt; ++b) v += cnt[b * (E + 1) + i];
            sm.total[i] = v;
        }
        meet();
    }
    const int nv = sm.total[E];
    const int te = tid % EP, tt = tid / EP;                 // softmax: expert and token of this thread (tt < 16)
    const float dev = te < E ? share_difference(sm.total[te], nv, k, E) : 0.f;
    const float c = nv > 0 ? coef * E / nv : 0.f;
    const int steps = F / 16, fw = (steps + BF_WARPS - 1) / BF_WARPS;
    const int k0 = min(warp * fw, steps), k1 = min(k0 + fw, steps);      // this warp's features: 16 k0 .. 16 k1 - 1
    const uint32_t bW = tc::smem_u32(sW), bU = tc::smem_u32(sU), bD = tc::smem_u32(&sm.dg[0][0][0]);
    // addresses of a lane's row in the blocks that ldmatrix takes: rows first, then columns (A), columns first (B)
    const int ra = (lane & 7) + ((lane >> 3) & 1) * 8, ca = (lane >> 4) * 8, rb = (lane & 7) + (lane >> 4) * 8, cb = ((lane >> 3) & 1) * 8;
    float acc[BF_NT][4];
#pragma unroll
    for (int i = 0; i < BF_NT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
    float psum = 0.f;
    int64_t it = 0;
    uint8_t ok_next = 0;
    if (tid < BF_TOK) {
        const int64_t t = (int64_t)blockIdx.x * BF_TOK + tid;
        ok_next = t < Tn && (!valid || valid[t]);
    }
    for (int64_t t = blockIdx.x; t < ntiles; t += gridDim.x, ++it) {
        const int s = (int)(it & 1);
        uint8_t *tile = sU + s * BF_TOK * pitch;
        const uint32_t bT = bU + s * BF_TOK * pitch;
        if (warp == 0) {
            const uint32_t m = __ballot_sync(0xffffffffu, ok_next) & 0xffffu;
            if (lane == 0) sm.ok = m;
            const int64_t nt = (t + gridDim.x) * BF_TOK + tid;
            ok_next = tid < BF_TOK && nt < Tn && (!valid || valid[nt]);
        }
        tc::mbar_wait(&sm.full[s], (uint32_t)((it >> 1) & 1), &sm.abort_flag, d_status);
        meet();
        const uint32_t ok = sm.ok;
        if (ok != 0xffffu) {                                // padding may hold anything, and rows behind the last token do
            for (int i = tid; i < BF_TOK * (F / 8); i += BF_MATH)
                if (!(ok >> (i / (F / 8)) & 1u)) *reinterpret_cast<uint4 *>(tile + i / (F / 8) * pitch + i % (F / 8) * 16) = make_uint4(0, 0, 0, 0);
            meet();
        }
        // ---- logits
        float lg[EP / 8][4];
#pragma unroll
        for (int n = 0; n < EP / 8; ++n) lg[n][0] = lg[n][1] = lg[n][2] = lg[n][3] = 0.f;
#pragma unroll 4
        for (int ks = k0; ks < k1; ++ks) {
            uint32_t a[4], b[4];
            bf_ldmatrix(bT + ra * pitch + (ks * 16 + ca) * 2, a);
            // rows of W: experts 0..7 (depth 0..7 and 8..15), then 8..15
            bf_ldmatrix(bW + (EP == 16 ? rb : (lane & 7)) * pitch + (ks * 16 + cb) * 2, b);
            bf_mma(lg[0], a, b[0], b[1]);
            if constexpr (EP == 16) bf_mma(lg[1], a, b[2], b[3]);
        }
        {
            const int g = lane >> 2, q = (lane & 3) * 2;
#pragma unroll
            for (int n = 0; n < EP / 8; ++n) {
                *reinterpret_cast<float2 *>(&sm.part[warp][g][n * 8 + q]) = make_float2(lg[n][0], lg[n][1]);
                *reinterpret_cast<float2 *>(&sm.part[warp][g + 8][n * 8 + q]) = make_float2(lg[n][2], lg[n][3]);
            }
        }
        meet();
        // ---- softmax over the experts, dg
        if (tt < BF_TOK) {
            float g = 0.f;
#pragma unroll
            for (int w = 0; w < BF_WARPS; ++w) g += sm.part[w][tt][te];
            if (te >= E) g = -INFINITY;
            float m = g;
#pragma unroll
            for (int o = EP / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float x = te < E ? expf(g - m) : 0.f;
            float sum = x;
#pragma unroll
            for (int o = EP / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            const float p = (ok >> tt & 1u) ? x / sum : 0.f;
            psum += p;
            float fb = p * dev;
#pragma unroll
            for (int o = EP / 2; o > 0; o >>= 1) fb += __shfl_xor_sync(0xffffffffu, fb, o);
            const float dg = c * p * (dev - fb);
            const __nv_bfloat16 p0 = __float2bfloat16_rn(dg);
            const float r1 = dg - __bfloat162float(p0);
            const __nv_bfloat16 p1 = __float2bfloat16_rn(r1), p2 = __float2bfloat16_rn(r1 - __bfloat162float(p1));
            sm.dg[0][tt][te] = p0;
            if (EP == 8) {
                sm.dg[0][tt][8 + te] = p1;
                sm.dg[2][tt][te] = p2;
            } else {
                sm.dg[1][tt][te] = p1;
                sm.dg[2][tt][te] = p2;
            }
        }
        meet();
        // ---- dW and du, 16 features at a time
        uint32_t at[3][4], ad[2][4];                        // dg^T (rows: experts), dg (rows: tokens)
#pragma unroll
        for (int q = 0; q < 3; ++q)
            if (q != 1 || EP == 16) bf_ldmatrix_trans(bD + (q * BF_TOK + rb) * 48 + cb * 2, at[q]);
#pragma unroll
        for (int q = 0; q < EP / 8; ++q) bf_ldmatrix(bD + (q * BF_TOK + ra) * 48 + ca * 2, ad[q]);
#pragma unroll
        for (int i = 0; i < BF_NT / 2; ++i) {
            const int ks = k0 + i;
            if (ks >= k1) break;
            if (part) {
                uint32_t b[4];                              // tokens 0..7, 8..15 of features 0..7, then of 8..15
                bf_ldmatrix_trans(bT + ra * pitch + (ks * 16 + ca) * 2, b);
#pragma unroll
                for (int q = 0; q < 3; ++q)
                    if (q != 1 || EP == 16) {
                        bf_mma(acc[2 * i], at[q], b[0], b[1]);
                        bf_mma(acc[2 * i + 1], at[q], b[2], b[3]);
                    }
            }
            if (du) {
                float d0[4] = {0.f, 0.f, 0.f, 0.f}, d1[4] = {0.f, 0.f, 0.f, 0.f};
                uint32_t b[4];                              // experts 0..7 (and 8..15) of features 0..7, then of 8..15
                if (EP == 16) {
                    bf_ldmatrix_trans(bW + ra * pitch + (ks * 16 + ca) * 2, b);
#pragma unroll
                    for (int q = 0; q < EP / 8; ++q) {
                        bf_mma(d0, ad[q], b[0], b[1]);
                        bf_mma(d1, ad[q], b[2], b[3]);
                    }
                } else {                                    // the two parts meet the same eight experts
                    bf_ldmatrix_trans(bW + (lane & 7) * pitch + (ks * 16 + ca) * 2, b);
                    bf_mma(d0, ad[0], b[0], b[0]);
                    bf_mma(d1, ad[0], b[2], b[2]);
                }
                __syncwarp();                               // (this warp's products have read these features of u)
                const int g = lane >> 2, f = ks * 16 + (lane & 3) * 2;
                uint8_t *r0 = tile + g * pitch + f * 2, *r1 = tile + (g + 8) * pitch + f * 2;
                *reinterpret_cast<uint32_t *>(r0) = tc::pack_bf16x2(d0[0], d0[1]);
                *reinterpret_cast<uint32_t *>(r1) = tc::pack_bf16x2(d0[2], d0[3]);
                *reinterpret_cast<uint32_t *>(r0 + 16) = tc::pack_bf16x2(d1[0], d1[1]);
                *reinterpret_cast<uint32_t *>(r1 + 16) = tc::pack_bf16x2(d1[2], d1[3]);
            }
        }
        // du, or zeros in the place of padding, were written by ordinary stores where bulk copies read and write next.  (For
        // every tile: to know here whether there was padding costs a register too many, 84 us instead of 81.)
        tc::fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&sm.done[s]);
    }
    if (tt < BF_TOK) sm.psum[tt][te] = psum;
    meet();
    if (tid < E) {
        float v = 0.f;
        for (int i = 0; i < BF_TOK; ++i) v += sm.psum[i][tid];
        mean_part[(int64_t)blockIdx.x * E + tid] = v;
    }
    if (part) {
        const int g = lane >> 2, q = (lane & 3) * 2;
#pragma unroll
        for (int i = 0; i < BF_NT; ++i) {
            const int f = (k0 * 2 + i) * 8 + q;
            if (k0 * 2 + i >= k1 * 2) break;
            float *p = part + ((int64_t)blockIdx.x * E + g) * F + f;
            if (EP == 8) {
                if (g < E) *reinterpret_cast<float2 *>(p) = make_float2(acc[i][0] + acc[i][2], acc[i][1] + acc[i][3]);
            } else {
                if (g < E) *reinterpret_cast<float2 *>(p) = make_float2(acc[i][0], acc[i][1]);
                if (g + 8 < E) *reinterpret_cast<float2 *>(p + 8 * (int64_t)F) = make_float2(acc[i][2], acc[i][3]);
            }
        }
    }
}

// Any F % 8 == 0, E <= 64, both types: a warp per BL_TOKENS tokens; logits by FMA with the features across the
// lanes, softmax with the experts across the lanes, then dg (kept for dW when asked) and du.  Bound by those FMAs and a second
// read of u: the call, 32768 tokens, takes 459 us for bf16, F = 4096, E = 8 (floor 82), 839 for F = 2048, E = 32 (floor 41),
// and 360 in fp32 for F = 2048, E = 8 (floor 82).
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

// dW (+)= sum of the partial sums in a fixed order: 128 entries and eight runs of partial sums a block; the last block
// gives counts, mean probabilities and the loss.
__global__ void __launch_bounds__(256)
balance_sum_kernel(const float *__restrict__ part, int nsplit, int64_t EF, float *dW, bool add,
                   const int *__restrict__ cnt, int ncnt, const float *__restrict__ mean_part, int nmean, int E, int k,
                   float coef, float *__restrict__ loss, int32_t *__restrict__ counts, float *__restrict__ mean_prob)
{
    __shared__ int total[SWIMBA_MAX_EXPERTS + 1];
    __shared__ float mean[SWIMBA_MAX_EXPERTS], run[4][SWIMBA_MAX_EXPERTS];
    __shared__ float4 sums[8][32];
    grid_dep_launch();
    grid_dep_wait();
    if (blockIdx.x + 1 < gridDim.x) {
        const int lane = threadIdx.x & 31, row = threadIdx.x >> 5;
        const int64_t i = ((int64_t)blockIdx.x * 32 + lane) * 4;
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < EF)
#pragma unroll 8
            for (int b = row; b < nsplit; b += 8) {
                const float4 v = *reinterpret_cast<const float4 *>(part + (int64_t)b * EF + i);
                s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
            }
        sums[row][lane] = s;
        __syncthreads();
        if (row > 0 || i >= EF) return;
        s = add ? *reinterpret_cast<const float4 *>(dW + i) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const float4 v = sums[b][lane];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        *reinterpret_cast<float4 *>(dW + i) = s;
        return;
    }
    total_counts(cnt, ncnt, E, total);
    const int nv = total[E], e = threadIdx.x & 63, r = threadIdx.x >> 6;
    if (e < E) {
        float s = 0.f;
#pragma unroll 8
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

bool bl_fused(int dtype, int F, int E) { return dtype == SWIMBA_DTYPE_BF16 && E <= 16 && F % 16 == 0 && F <= 2048; }
size_t bl_fused_smem(int F, int E)
{
    const size_t small = E <= 8 ? sizeof(BfSmall<8>) : sizeof(BfSmall<16>);
    return (small + 15) / 16 * 16 + ((E <= 8 ? 8 : 16) + 2 * BF_TOK) * (size_t)(F * 2 + 16);
}
int bl_fused_blocks(int64_t T, int sm_count) { return (int)std::min<int64_t>(ceil_div64(T, BF_TOK), sm_count); }

struct BalanceLayout {
    size_t cnt, mean, dg, part, total;
};
BalanceLayout bl_layout(int dtype, int64_t T, int F, int E, int sm_count)
{
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    const bool fused = bl_fused(dtype, F, E);
    BalanceLayout l;
    size_t o = 0;
    l.cnt = o;  o += up(sizeof(int) * BL_COUNT_BLOCKS * (E + 1));
    l.mean = o; o += up(sizeof(float) * (fused ? bl_fused_blocks(T, sm_count) : bl_blocks(T, sm_count)) * E);
    l.dg = o;   o += fused ? 0 : up(sizeof(float) * T * E);
    l.part = o; o += up(sizeof(float) * (fused ? bl_fused_blocks(T, sm_count) : bl_splits(T, F, E, sm_count)) * E * F);
    l.total = o;
    return l;
}
void launch_sum(LaunchCtx &ctx, const float *part, int nsplit, int64_t EF, float *dW, bool add, const int *cnt, int ncnt,
                const float *mean, int nmean, int E, int k, float coef, float *loss, int32_t *counts, float *mean_prob)
{
    ctx.begin(STAGE_BALANCE_SUM);
    launch_kernel(balance_sum_kernel, dim3((unsigned)(dW ? ceil_div64(EF, 128) : 0) + 1), dim3(256), 0, ctx.stream, true,
                  part, nsplit, EF, dW, add, cnt, ncnt, mean, nmean, E, k, coef, loss, counts, mean_prob);
    ctx.end();
}
int launch_count(LaunchCtx &ctx, const int32_t *idx, const uint8_t *valid, int64_t Tn, int k, int E, int *cnt)
{
    const int ncnt = (int)std::min<int64_t>(BL_COUNT_BLOCKS, ceil_div64(Tn, 256));
    ctx.begin(STAGE_BALANCE_COUNT);
    launch_kernel(balance_count_kernel, dim3(ncnt), dim3(256), 0, ctx.stream, true, idx, valid, Tn, k, E, cnt,
                  ctx.d_status, ctx.check_indices);
    ctx.end();
    return ncnt;
}

template <int EP>
int run_fused(LaunchCtx &ctx, const void *u, const void *W, const int32_t *idx, const uint8_t *valid, int64_t Tn, int F,
              int E, int k, float coef, int sm_count, float *loss, int32_t *counts, float *mean_prob, float *dW, bool add,
              void *du, char *ws)
{
    const BalanceLayout l = bl_layout(SWIMBA_DTYPE_BF16, Tn, F, E, sm_count);
    int *cnt = (int *)(ws + l.cnt);
    float *mean = (float *)(ws + l.mean), *part = (float *)(ws + l.part);
    const bool here = Tn * k <= BF_COUNT_HERE;
    const int ncnt = here ? 1 : launch_count(ctx, idx, valid, Tn, k, E, cnt), nblk = bl_fused_blocks(Tn, sm_count);
    auto kern = balance_fused_kernel<EP>;
    const size_t smem = bl_fused_smem(F, E);
    if (!ensure_dynamic_smem((const void *)kern, smem)) return SWIMBA_ERR_CUDA;
    ctx.begin(STAGE_BALANCE_TOKENS);
    launch_kernel(kern, dim3(nblk), dim3(BF_THREADS), smem, ctx.stream, true, (const __nv_bfloat16 *)u, (const __nv_bfloat16 *)W,
                  idx, valid, Tn, F, E, k, coef, cnt, ncnt, here, ctx.check_indices, (__nv_bfloat16 *)du,
                  dW ? part : (float *)nullptr, mean, ctx.d_status);
    ctx.end();
    launch_sum(ctx, part, nblk, (int64_t)E * F, dW, add, cnt, ncnt, mean, nblk, E, k, coef, loss, counts, mean_prob);
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

template <typename T>
int run_balance(LaunchCtx &ctx, const void *u, const void *W, const int32_t *idx, const uint8_t *valid, int64_t Tn, int F,
                int E, int k, float coef, int sm_count, float *loss, int32_t *counts, float *mean_prob, float *dW,
                bool add, void *du, char *ws)
{
    const BalanceLayout l = bl_layout(sizeof(T) == 4 ? SWIMBA_DTYPE_FP32 : SWIMBA_DTYPE_BF16, Tn, F, E, sm_count);
    int *cnt = (int *)(ws + l.cnt);
    float *mean = (float *)(ws + l.mean), *dg = (float *)(ws + l.dg), *part = (float *)(ws + l.part);
    const int ncnt = launch_count(ctx, idx, valid, Tn, k, E, cnt), nblk = bl_blocks(Tn, sm_count);
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
    launch_sum(ctx, part, used, EF, dW, add, cnt, ncnt, mean, nblk, E, k, coef, loss, counts, mean_prob);
    return cudaGetLastError() == cudaSuccess ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace

size_t balance_workspace_bytes(int dtype, int64_t T, int F, int E, int sm_count)
{
    return bl_layout(dtype, T, F, E, sm_count).total;
}

int launch_balance(LaunchCtx &ctx, int dtype, const void *u, const void *W, const int32_t *idx, const uint8_t *valid,
                   int64_t T, int F, int E, int k, float coef, int sm_count, float *loss, int32_t *counts,
                   float *mean_prob, float *dW, bool add, void *du, void *workspace)
{
    if (dtype == SWIMBA_DTYPE_FP32)
        return run_balance<float>(ctx, u, W, idx, valid, T, F, E, k, coef, sm_count, loss, counts, mean_prob, dW, add, du,
                                  (char *)workspace);
    if (bl_fused(dtype, F, E)) {
        auto run = E <= 8 ? run_fused<8> : run_fused<16>;
        return run(ctx, u, W, idx, valid, T, F, E, k, coef, sm_count, loss, counts, mean_prob, dW, add, du, (char *)workspace);
    }
    return run_balance<__nv_bfloat16>(ctx, u, W, idx, valid, T, F, E, k, coef, sm_count, loss, counts, mean_prob, dW, add,
                                      du, (char *)workspace);
}

}  // namespace swimba
