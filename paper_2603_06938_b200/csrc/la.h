// Linear attention with a decay for each head: the jobs its kernels work.
//
// One job is the map  (q, k, v, entry state) -> (o, exit state)  of
//   forward in time   S_t = lambda S_{t-1} + a k_t v_t^T,          o_t = p-part + c-part = S_t^T q_t
//   backward in time  R_t = lambda R_{t+1} + a k_t v_t^T,  with the entry state already at the last token
//                     (R_L = E + a k_L v_L^T) and the exit state lambda R_1 in front of the first
// with DK = entries of q and k, DV = entries of v and o, both of which a gradient call sets as it needs:
//   forward    q, k, v -> o                    scores and carried part times scale, a = 1
//   d query    q := do, k := v, v := k         the same with the state transposed
//   d key      q := v, k := do, v := q         backward in time, entered by the final state's gradient,
//   d value    q := k, k := q,  v := do        whose products do q^T carry the scale (a = scale), not the read
#pragma once
#include "internal.h"
#include "tc05.cuh"

namespace swimba {

struct LaJob {
    const void *q, *k, *v;       // rows of token t of sequence b start at ((b L + t) ld)
    int64_t ldq, ldk, ldv;       // elements from token to token
    int rq, rk, rv;              // head h reads stream h / r
    int dk, dv;
    int reverse;                 // 1: backward in time
    int transposed;              // states lie as [DK][DV] (0: as [DV][DK])
    const float *s_in;           // [B, H, DV, DK] (or transposed); NULL: zeros
    float *s_out;                // may be NULL
    void *o;                     // [B, L, H, DV], rows ldo apart
    int64_t ldo;
    int o_f32;                   // o is float whatever the dtype
    float scale_p, scale_c, scale_a;   // of the scores inside a tile, of the carried state's part, of what the state adds
    float *seg;                  // [B, H, nseg per] states in the layout of s_in, when sequences are cut
};

constexpr int LA_MAX_JOBS = 3;
struct LaArgs {
    LaJob job[LA_MAX_JOBS];
    int njobs;
    const float *log_decay;      // [H]
    int B, L, H;
    int seg_len, nseg;           // tokens per segment (the last in the sequence may be shorter), segments per sequence
    int per;                     // pieces per segment, of seg_len / per tokens, that the pass for the states works
    // CTAs of the kernel for more than 64 values: the first `whole` (job, segment, head, sequence)s have one each; the tiles of the others
    // are shared by ncut, of which number c gives the outputs of tiles cut[c] .. cut[c + 1] - 1 of the walk and carries only
    // the state through those in front
    int whole, ncut, cut[5];
};

// log2 of the decay.  Held above -1e4, where one step underflows to nothing already, so that the zeroth
// power of a decay of exp(-infinity) is 1 and not a NaN.
__device__ __forceinline__ float la_log2_decay(float g)
{
    const float g2 = g * 1.4426950408889634f;
    return g2 < -1.0e4f ? -1.0e4f : g2;
}

// The decay over m tokens as a sum of two floats: multiplied up over the memory of a slow head, the rounding of one would be
// the largest error there is (256 tokens one by one: 3e-6; 128 tiles of a head that forgets 2.3e-5 a token: 1.4e-6).
struct LaDecay {
    float hi, lo;
};
__device__ __forceinline__ LaDecay la_decay(float g, int m = 1)
{
    const double l = exp2((double)la_log2_decay(g) * m);
    return LaDecay{(float)l, (float)(l - (double)(float)l)};
}

// w v in bf16 parts:
//   three parts  in fp32, each part what is left of the product behind those in front (2^-24 of it)
//   two parts    with the weight in two bf16 parts of its own (wh, wm): wh v; and its remainder, which is itself a bf16
//                number and so comes exactly from a fused multiply-add, with wm v in one (2^-17)
// The two parts of the weights of two values:
__device__ __forceinline__ void la_split(float w0, float w1, uint32_t (&p)[2])
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        p[i] = tc::pack_bf16x2(w0, w1);
        w0 -= __uint_as_float(p[i] << 16);
        w1 -= __uint_as_float(p[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ __nv_bfloat162 la_pair(uint32_t v) { return *reinterpret_cast<const __nv_bfloat162 *>(&v); }
__device__ __forceinline__ uint32_t la_bits(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t *>(&v); }
// How the CTAs of the kernel for 128 values share `items` walks of nt tiles; returns the time, in tiles.
double la_cuts(int64_t items, int nt, int sm_count, LaArgs *a);
// Segments the kernels cut every sequence of a call into, and the bytes they keep for that.
void la_plan(int dtype, int B, int L, int H, int N, int P, int njobs, int sm_count, int *seg_len, int *nseg, int *per);
// (bytes of one job's segment states; grows with B and with L)
size_t la_segment_bytes(int dtype, int B, int L, int H, int N, int P, int njobs, int sm_count);
// Tensor map of [B, L, streams, D], rows ld apart, for boxes of 128 tokens of 64 entries of one stream.  Rows behind
// the sequence read as zeros and are not written.
bool la_stream_map(TmapCache *cache, CUtensorMap *m, const void *p, int D, int streams, int L, int B, int64_t ld);
// The tensor-core kernels (la_tiles.cu): the head sizes they take, their launches (states: the pass that leaves every
// segment's end state).
bool la_tiles_shape(int dtype, int N, int P);
int launch_la_tiles(LaunchCtx &ctx, const LaArgs &a, bool states, int sm_count);
int launch_la_wide(LaunchCtx &ctx, const LaArgs &a, bool states, int sm_count);      // those of more than 64 values (la_wide.cu)
// Runs the jobs: per-segment states, their chain, outputs; or outputs alone when nseg == 1.
int launch_la(LaunchCtx &ctx, int dtype, const LaArgs &a, int sm_count);
// out[t, g, :] = sum over the r heads of group g of part[t, g r + i, :], in that order.
int launch_la_head_sum(LaunchCtx &ctx, int dtype, const float *part, int64_t T, int G, int r, int N, void *out);
int launch_la_step(LaunchCtx &ctx, int dtype, const float *log_decay, const void *q, int64_t ldq, const void *k,
                   int64_t ldk, const void *v, int64_t ldv, const float *s_in, int B, int H, int G, int P, int N,
                   float scale, int sm_count, void *o, float *s_out);

// Layer norm over each of `groups` equal channel groups of a row (every group: width entries).
int launch_layer_norm(LaunchCtx &ctx, int dtype, const void *x, int64_t ldx, const float *w, const float *b, int64_t rows,
                      int groups, int width, float eps, int sm_count, void *y, float *mean, float *rstd);
size_t layer_norm_partial_bytes(int64_t rows, int groups, int width, int sm_count);
int launch_layer_norm_backward(LaunchCtx &ctx, int dtype, const void *dy, const void *x, int64_t ldx, const float *w,
                               const float *mean, const float *rstd, int64_t rows, int groups, int width, int sm_count,
                               void *dx, float *dw, float *db, float *partial);

// Balance loss of a router (see swimba_balance_loss).
size_t balance_workspace_bytes(int dtype, int64_t T, int F, int E, int sm_count);
int launch_balance(LaunchCtx &ctx, int dtype, const void *u, const void *W, const int32_t *idx, const uint8_t *valid,
                   int64_t T, int F, int E, int k, float coef, int sm_count, float *loss, int32_t *counts,
                   float *mean_prob, float *dW, bool add, void *du, void *workspace);

}  // namespace swimba
