// Linear attention with a decay for each head on the tensor cores (bf16; heads of up to 128 entries of keys and 64 of values,
// made up to 64 or 128 by the zeros that copies read behind a head): tiles of 128 tokens, the carried state on chip.  What a
// job is: la.h.  Per tile, with n tokens, r the place of a token in the order of the walk, and the state S [DK, DV] entering it:
//   QK   A = Q K^T                                            scores
//        P_ij = scale_p lambda^|i-j| A_ij  for tokens j that i sees, else 0
//   PV   O1 = P V,   QS  O2 = Q S,   o_i = O1_i + scale_c lambda^(r_i + first) O2_i
//   KV   D = K^T (w V),  w_j = scale_a lambda^(n - r_j - first),   S <- lambda^n S + D
// (first = 1 walking forward, 0 backward, where the decay follows the read of a token).
//
// Precision.  Sums are fp32 in tensor memory, the state stays fp32 in registers.  P and the state's copy for QS are
// rounded to bf16 (a term of o, which is bf16 itself, passes one of the two).  w V is not: it goes into the state and is
// taken as the sum of bf16 parts, one product each: three where the state is a result (2^-24 of it), else two (2^-17).
//
// Measured, 65536 tokens of 16 heads of 64 x 64 (floor 82 us): cut into segments, the states alone 65 us (238 MB read, 3.7
// TB/s; their loads alone take 50, the rest is shared memory, 176 KB of reads and writes a tile against 128 bytes a cycle),
// their chain 7, the outputs 112 (537 MB, 4.8 TB/s; the loads and stores without the making of w V 97).
//
// A token's bits reach nobody in front of it: scores are masked by selection, and entries of V that are infinite or NaN,
// which a zero of P would turn into NaN, are zeros in PV; the epilogue adds them to the rows that see them.
#include <algorithm>
#include <cstddef>

#include "la.h"
#include "tc05.cuh"

namespace swimba {

namespace {

constexpr int LT = 128;                      // tokens per tile
constexpr int LDV = 64;                      // columns of v
constexpr int MARKS = 4;                     // places of the marks of tiles whose V is not all finite
constexpr int PARTS = 3;                     // bf16 parts of w V at most
constexpr uint32_t SLAB = LT * 128;          // 128 rows of 64 bf16
// warps: copies, products, tensor memory, spare; 8 for the masks, 8 for w V, 8 for the state, 4 for o.  Every role's loops
// are kept short: the four schedulers' instruction caches hold about 700 instructions each, and unrolled roles that did not
// fit waited for instructions most of the time (9000 cycles a tile; now about 3200, 4200 with 128 keys).
constexpr int THREADS = 1024;
constexpr int WARP_TMA = 0, WARP_MMA = 1, WARP_ALLOC = 2, WARP_MASK = 4, WARP_W = 12, WARP_STATE = 20, WARP_O = 28;
// tensor memory columns: scores, P (bf16), Q S, P V, a D for each part of w V
constexpr uint32_t TM_QK = 0, TM_P = 128, TM_QS = 192, TM_PV = 256, TM_KV = 320, TM_COLS = 512;

template <int DK> struct Sm {
    static constexpr int NS = DK == 64 ? 3 : 2;           // stages of Q, K and V
    static constexpr uint32_t QB = DK / 64 * SLAB;        // bytes of a Q or K tile
    static constexpr uint32_t Q = 0, K = Q + NS * QB, V = K + NS * QB, VW = V + NS * SLAB, S = VW + PARTS * SLAB,
                              SMALL = S + DK * 128;
};
struct Small {
    uint64_t full_q[3], full_k[3], full_v[3], free_q[3], free_k[3], free_v[3];
    uint64_t qk_full, qk_read, p_full, qs_done, pv_done, vw_full[4], kv_done[4], kv_read, s_full, o_free;
    uint64_t d_free[2];                      // (states alone) D has been read
    uint32_t tmem;
    int abort_flag;
    // 1 + the tile whose V is not all finite, in place t % 4: with three stages of V the warps of w V mark tile t + 2 while
    // the epilogue may still look for the mark of t and the masks for that of t - 1
    int odd_tile[MARKS];
    alignas(16) float pow_col[32];           // factors of a score block's columns
    float pow_diag[64];                      // scale_p lambda^|m - 31|: the block on the diagonal
    float pow[LT + 1];                       // lambda^m
    LaDecay whole[8];                        // lambda^LT (where the state is a result, in two floats), for each warp of the state
};

static_assert(offsetof(Small, pow_col) % 16 == 0 && Sm<64>::SMALL % 16 == 0 && Sm<128>::SMALL % 16 == 0, "read in fours");

struct Maps {
    CUtensorMap q[LA_MAX_JOBS], k[LA_MAX_JOBS], v[LA_MAX_JOBS], o[LA_MAX_JOBS];
};

__device__ __forceinline__ uint64_t pair_of(uint32_t a, uint32_t b) { return tc::f32x2(__uint_as_float(a), __uint_as_float(b)); }

// STATE_ONLY: from a zero state, and only the end state is kept (in seg).
template <int DK, bool STATE_ONLY>
__global__ void __launch_bounds__(THREADS, 1)
la_tiles_kernel(const __grid_constant__ Maps maps, const __grid_constant__ LaArgs a, int *d_status)
{
    typedef Sm<DK> L;
    constexpr int NS = L::NS;
    extern __shared__ __align__(1024) uint8_t smem[];
    Small *sm = (Small *)(smem + L::SMALL);
    int *abort_flag = &sm->abort_flag;
    if ((tc::smem_u32(smem) & 1023u) != 0) {       // the swizzled tiles need a 1024-byte aligned base
        if (threadIdx.x == 0) atomicCAS(d_status, 0, SWIMBA_ERR_DEVICE_BOUNDS);
        return;
    }
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;

    // the jobs on one head side by side: they read the same rows at about the same time
    int64_t id = blockIdx.x;
    const int ji = (int)(id % a.njobs);
    id /= a.njobs;
    // segments, or pieces of them for the states alone, in the order of the walk (the last segment's end state enters nothing)
    const int nall = STATE_ONLY ? a.nseg * a.per : a.nseg, nrun = STATE_ONLY ? nall - a.per : nall;
    const int seg = (int)(id % nrun), len = STATE_ONLY ? a.seg_len / a.per : a.seg_len;
    id /= nrun;
    const int h = (int)(id % a.H), b = (int)(id / a.H);
    const LaJob &j = a.job[ji];
    const bool rev = j.reverse != 0;
    // three parts where the state is a result; two (2^-17) where only the read of it is, whose copy is rounded to bf16
    const int parts = j.s_out && (STATE_ONLY || seg == nall - 1) ? 3 : 2;
    const int place = rev ? nall - 1 - seg : seg;
    const int t_begin = min(a.L, place * len), t_end = min(a.L, t_begin + len);
    const int ntiles = (t_end - t_begin + LT - 1) / LT;
    auto tile_at = [&](int t) { return t_begin + (rev ? ntiles - 1 - t : t) * LT; };       // first token of tile t
    auto tile_n = [&](int t) { return min(LT, t_end - tile_at(t)); };

    // w V of the halves of a tile; for the states alone two tiles, the second where Q would be
    static_assert(NS * L::QB >= PARTS * SLAB, "w V over Q");
    auto vw_slot = [](int t, int hf) { return STATE_ONLY ? (t & 1) * 2 + hf : hf; };
    auto vw_phase = [](int t) { return STATE_ONLY ? t >> 1 : t; };
    // D; for the states alone those of two tiles in turn, the second where scores would be
    auto d_of = [](int t) { return STATE_ONLY && (t & 1) ? TM_QK : TM_KV; };

    if (tid == 0) {
        for (int s = 0; s < NS; ++s) {
            tc::mbar_init(&sm->full_q[s], 1);
            tc::mbar_init(&sm->full_k[s], 1);
            tc::mbar_init(&sm->full_v[s], 1);
            tc::mbar_init(&sm->free_q[s], 1);
            tc::mbar_init(&sm->free_k[s], 1);
            tc::mbar_init(&sm->free_v[s], STATE_ONLY ? 16 : j.o_f32 ? 4 : 1);
        }
        for (int s = 0; s < 4; ++s) {
            tc::mbar_init(&sm->vw_full[s], 8);
            tc::mbar_init(&sm->kv_done[s], 1);
        }
        for (int i = 0; i < MARKS; ++i) sm->odd_tile[i] = 0;
        tc::mbar_init(&sm->qk_full, 1);
        tc::mbar_init(&sm->qk_read, 8);
        tc::mbar_init(&sm->p_full, 8);
        tc::mbar_init(&sm->qs_done, 1);
        tc::mbar_init(&sm->pv_done, 1);
        tc::mbar_init(&sm->kv_read, 8);
        tc::mbar_init(&sm->s_full, 8);
        tc::mbar_init(&sm->o_free, 4);
        tc::mbar_init(&sm->d_free[0], 8);
        tc::mbar_init(&sm->d_free[1], 8);
        *abort_flag = 0;
        tc::fence_mbar_init();
    }
    if (warp == WARP_ALLOC) {
        tc::tmem_alloc(&sm->tmem, TM_COLS);
        tc::tmem_relinquish();
    }
    if (warp == WARP_TMA && lane == 0) {
        if (!STATE_ONLY) tc::prefetch_tmap(&maps.q[ji]);
        tc::prefetch_tmap(&maps.k[ji]);
        tc::prefetch_tmap(&maps.v[ji]);
    }
    grid_dep_launch();
    grid_dep_wait();
    const float g2 = la_log2_decay(a.log_decay[h]);
    if (tid <= LT) sm->pow[tid] = exp2f(tid * g2);
    else if (tid >= 256 && tid < 288) sm->pow_col[tid - 256] = exp2f((rev ? tid - 256 : 287 - tid) * g2);
    else if (tid >= 320 && tid < 383) sm->pow_diag[tid - 320] = j.scale_p * exp2f(abs(tid - 351) * g2);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = sm->tmem;

    if (warp == WARP_TMA) {
        // ------------------------------------------------------------------ loads, in the order in which room comes free
        const bool leader = tc::elect_one();
        for (int t = 0; t < ntiles; ++t) {
            const int s = t % NS, at = tile_at(t);
            const uint32_t ph = ((t / NS) & 1) ^ 1;
            auto load = [&](uint64_t *full, uint64_t *room, uint32_t dst, uint32_t bytes, const CUtensorMap *m, int col, int stream) {
                tc::mbar_wait(room, ph, abort_flag, d_status);
                if (leader && !*(volatile int *)abort_flag) {
                    tc::mbar_arrive_expect_tx(full, bytes);
                    for (uint32_t o = 0; o < bytes; o += SLAB)
                        tc::tma_load_4d(smem + dst + o, m, full, col + (int)(o / SLAB) * 64, stream, at, b);
                }
                __syncwarp();
            };
            load(&sm->full_k[s], &sm->free_k[s], L::K + s * L::QB, L::QB, &maps.k[ji], 0, h / j.rk);
            if (!STATE_ONLY) load(&sm->full_q[s], &sm->free_q[s], L::Q + s * L::QB, L::QB, &maps.q[ji], 0, h / j.rq);
            load(&sm->full_v[s], &sm->free_v[s], L::V + s * SLAB, SLAB, &maps.v[ji], 0, h / j.rv);
        }
        // No copy may be in flight when the CTA leaves: after an abort nobody else has waited for the last ones (those
        // that were not issued any more never arrive, and these waits run out soon).
        auto settle = [&](uint64_t *full, uint32_t ph) {
            int quiet = 0;
            if (*(volatile int *)abort_flag) tc::mbar_wait(full, ph, &quiet, d_status, 10000000ll);
            else tc::mbar_wait(full, ph, abort_flag, d_status);
        };
        for (int t = max(0, ntiles - NS); t < ntiles; ++t) {
            settle(&sm->full_k[t % NS], (t / NS) & 1);
            if (!STATE_ONLY) settle(&sm->full_q[t % NS], (t / NS) & 1);
            settle(&sm->full_v[t % NS], (t / NS) & 1);
        }
    } else if (warp == WARP_MMA) {
        // ------------------------------------------------------------------ products
        const bool leader = tc::elect_one();
        constexpr uint32_t id_qk = tc::idesc_bf16(128, 128, 0, 0);      // Q (K-major) x K (K-major)
        constexpr uint32_t id_qs = tc::idesc_bf16(128, LDV, 0, 1);      // Q (K-major) x S (MN-major); P (TMEM) x V (MN-major)
        // K (MN-major) x the parts of wV side by side (MN-major): K is read once for all of them
        const uint32_t id_kv = tc::idesc_bf16(128, parts * LDV, 1, 1);
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint32_t base = tc::smem_u32(smem);
        const uint64_t dQ = tc::smem_desc_sw128(base + L::Q, 16, 1024), dK = tc::smem_desc_sw128(base + L::K, 16, 1024);
        // (64 keys: both halves of the 128 rows of D are the same 64 keys)
        const uint64_t dKt = tc::smem_desc_sw128(base + L::K, DK == 128 ? SLAB : 0, 1024);
        const uint64_t dV = tc::smem_desc_sw128(base + L::V, SLAB, 1024), dW = tc::smem_desc_sw128(base + L::VW, SLAB, 1024),
                       dW2 = tc::smem_desc_sw128(base + L::Q, SLAB, 1024);
        const uint64_t dS = tc::smem_desc_sw128(base + L::S, SLAB, 1024);
        auto scores = [&](int t) {
            const int s = t % NS;
            const uint32_t ph = (t / NS) & 1;
            tc::mbar_wait(&sm->full_k[s], ph, abort_flag, d_status);
            tc::mbar_wait(&sm->full_q[s], ph, abort_flag, d_status);
            if (t > 0) tc::mbar_wait(&sm->qk_read, (t - 1) & 1, abort_flag, d_status);
            tc::tc_fence_after();
            if (leader) {
                const uint64_t q = tc::smem_desc_fresh(tc::smem_desc_advance(dQ, s * L::QB));
                const uint64_t k = tc::smem_desc_fresh(tc::smem_desc_advance(dK, s * L::QB));
#pragma unroll
                for (int kk = 0; kk < DK / 16; ++kk) {
                    const uint32_t o = (kk >> 2) * SLAB + (kk & 3) * 32;
                    tc::mma_ss(tm + TM_QK, tc::smem_desc_advance(q, o), tc::smem_desc_advance(k, o), id_qk, kk > 0);
                }
                tc::mma_commit(&sm->qk_full);
            }
            __syncwarp();
        };
        if (!STATE_ONLY && ntiles > 0) scores(0);
        for (int t = 0; t < ntiles; ++t) {
            const int s = t % NS;
            const uint32_t ph = (t / NS) & 1;
            // KV, by halves of the tile: w V of one is made while the other is multiplied.  It does not wait for the state.
            if (STATE_ONLY) {
                tc::mbar_wait(&sm->full_k[s], ph, abort_flag, d_status);
                if (t > 1) tc::mbar_wait(&sm->d_free[t & 1], ((t >> 1) - 1) & 1, abort_flag, d_status);
            } else if (t > 0) tc::mbar_wait(&sm->kv_read, (t - 1) & 1, abort_flag, d_status);
#pragma unroll 1
            for (int hf = 0; hf < 2; ++hf) {
                const int u = vw_slot(t, hf);
                tc::mbar_wait(&sm->vw_full[u], vw_phase(t) & 1, abort_flag, d_status);
                tc::tc_fence_after();
                if (leader) {
                    const uint64_t k = tc::smem_desc_fresh(tc::smem_desc_advance(dKt, s * L::QB + hf * 8192));
                    const uint64_t w = tc::smem_desc_fresh(tc::smem_desc_advance(u < 2 ? dW : dW2, hf * 8192));
#pragma unroll
                    for (int kk = 0; kk < LT / 32; ++kk)
                        tc::mma_ss(tm + d_of(t), tc::smem_desc_advance(k, kk * 2048), tc::smem_desc_advance(w, kk * 2048), id_kv,
                                   hf + kk > 0);
                    tc::mma_commit(&sm->kv_done[u]);
                    if (hf == 1) tc::mma_commit(&sm->free_k[s]);
                }
                __syncwarp();
            }
            if (STATE_ONLY) continue;
            // QS: the carried part, once the state is there and the epilogue has read the tile in front
            tc::mbar_wait(&sm->s_full, t & 1, abort_flag, d_status);
            if (t > 0) tc::mbar_wait(&sm->o_free, (t - 1) & 1, abort_flag, d_status);
            tc::tc_fence_after();
            if (leader) {
                const uint64_t q = tc::smem_desc_fresh(tc::smem_desc_advance(dQ, s * L::QB));
                const uint64_t st = tc::smem_desc_fresh(dS);
#pragma unroll
                for (int kk = 0; kk < DK / 16; ++kk)
                    tc::mma_ss(tm + TM_QS, tc::smem_desc_advance(q, (kk >> 2) * SLAB + (kk & 3) * 32),
                               tc::smem_desc_advance(st, kk * 2048), id_qs, kk > 0);
                tc::mma_commit(&sm->qs_done);
                tc::mma_commit(&sm->free_q[s]);
            }
            __syncwarp();
            if (t + 1 < ntiles) scores(t + 1);
            // PV
            tc::mbar_wait(&sm->full_v[s], ph, abort_flag, d_status);
            tc::mbar_wait(&sm->p_full, t & 1, abort_flag, d_status);
            tc::tc_fence_after();
            if (leader) {
                const uint64_t v = tc::smem_desc_fresh(tc::smem_desc_advance(dV, s * SLAB));
#pragma unroll
                for (int kk = 0; kk < LT / 16; ++kk)
                    tc::mma_ts(tm + TM_PV, tm + TM_P + kk * 8, tc::smem_desc_advance(v, kk * 2048), id_qs, kk > 0);
                tc::mma_commit(&sm->pv_done);
            }
            __syncwarp();
        }
    } else if (!STATE_ONLY && warp >= WARP_MASK && warp < WARP_W) {
        // ------------------------------------------------------------------ masks: half a row of the scores per thread
        const int q4 = warp & 3, half = (warp - WARP_MASK) >> 2, i = q4 * 32 + lane;
        const uint32_t row = tmem + ((uint32_t)(q4 * 32) << 16), from = row + TM_QK + half * 64, to = row + TM_P + half * 32;
        const float scale_p = j.scale_p;
        const uint32_t keep = rev ? 0xffffffffu << lane : 0xffffffffu >> (31 - lane);
        for (int t = 0; t < (STATE_ONLY ? 0 : ntiles); ++t) {
            tc::mbar_wait(&sm->qk_full, t & 1, abort_flag, d_status);
            tc::tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < 2; ++k) {
                const int bl = half * 2 + k;
                const bool seen = rev ? bl >= q4 : bl <= q4;
                uint32_t x[32], o[16];
                if (seen) {
                    tc::tmem_ld32(from + k * 32, x);
                    tc::tmem_ld_wait();
                }
                if (k == 1) {
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&sm->qk_read);
                }
                if (!seen) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = 0u;
                } else {
                    if (bl == q4) {
                        const float *f = &sm->pow_diag[31 + lane];
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const float v = f[-e] * __uint_as_float(x[e]);
                            x[e] = keep >> e & 1u ? __float_as_uint(v) : 0u;
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = tc::pack_bf16x2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1]));
                    } else {                     // a factor for the row's place before the block, one for each column's in it
                        const float rho = scale_p * sm->pow[rev ? 32 * bl - i : i - 32 * bl - 31];
                        const uint64_t r2 = tc::f32x2(rho, rho);
#pragma unroll
                        for (int e = 0; e < 16; e += 2) {
                            const float4 c = *reinterpret_cast<const float4 *>(&sm->pow_col[2 * e]);
                            o[e] = tc::f32x2_bf16(tc::f32x2_mul(pair_of(x[2 * e], x[2 * e + 1]), tc::f32x2_mul(r2, tc::f32x2(c.x, c.y))));
                            o[e + 1] = tc::f32x2_bf16(tc::f32x2_mul(pair_of(x[2 * e + 2], x[2 * e + 3]), tc::f32x2_mul(r2, tc::f32x2(c.z, c.w))));
                        }
                    }
                }
                if (k == 0 && t > 0) {           // (P has been read, by the epilogue too where V was not all finite)
                    tc::mbar_wait(&sm->pv_done, (t - 1) & 1, abort_flag, d_status);
                    if (((volatile int *)sm->odd_tile)[(t - 1) % MARKS] == t) tc::mbar_wait(&sm->o_free, (t - 1) & 1, abort_flag, d_status);
                    tc::tc_fence_after();
                }
                tc::tmem_st16(to + k * 16, o);
            }
            tc::tmem_st_wait();
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm->p_full);
        }
    } else if (warp >= WARP_MASK && warp < WARP_STATE) {
        // ------------------------------------------------------------------ w V: eight entries of two rows at a time (for the
        // states alone the warps of the masks make the first half of a tile)
        const int ltid = (tid - WARP_MASK * 32) & 255, r0 = ltid >> 3;
        const int hf_begin = STATE_ONLY && warp >= WARP_W ? 1 : 0, hf_end = STATE_ONLY ? hf_begin + 1 : 2;
        const uint64_t neg = tc::f32x2(-1.f, -1.f);
        const float scale_a = j.scale_a;
        for (int t = 0; t < ntiles; ++t) {
            const int s = t % NS, n = tile_n(t);
            tc::mbar_wait(&sm->full_v[s], (t / NS) & 1, abort_flag, d_status);
            // (states alone: every tile's additions as they are at the end of the walk)
            const float tail = STATE_ONLY ? scale_a * exp2f((rev ? tile_at(t) - t_begin : t_end - tile_at(t) - n) * g2) : scale_a;
            const uint32_t off = tc::sw128_offset(r0, ltid & 7);           // (32 rows on: 4096 bytes, same swizzle)
            uint32_t odd = 0;
#pragma unroll 1
            for (int hf = hf_begin; hf < hf_end; ++hf) {
                const int i = hf * 2;
                uint4 v[2];
                float w[2];
                const int u = vw_slot(t, hf);
                if (vw_phase(t) > 0) tc::mbar_wait(&sm->kv_done[u], (vw_phase(t) - 1) & 1, abort_flag, d_status);
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const int rr = r0 + 32 * (i + z), e = rev ? rr + 1 : n - 1 - rr;      // n - r - first steps of decay
                    v[z] = *reinterpret_cast<const uint4 *>(smem + L::V + s * SLAB + off + (i + z) * 4096);
                    w[z] = rr < n ? tail * sm->pow[e] : 0.f;
                }
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const uint32_t in[4] = {v[z].x, v[z].y, v[z].z, v[z].w};
                    uint8_t *dst = smem + (u < 2 ? L::VW : L::Q) + off + (i + z) * 4096;
                    uint32_t p[PARTS][4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)      // (an exponent of all ones, infinity or NaN, carries into the sign's place)
                        odd |= (in[k] & 0x7f807f80u) + 0x00800080u;
                    if (parts == 2) {
                        uint32_t wp[2];
                        la_split(w[z], w[z], wp);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const __nv_bfloat162 x = la_pair(in[k]), wh = la_pair(wp[0]), p0 = __hmul2(wh, x);
                            p[0][k] = la_bits(p0);
                            p[1][k] = la_bits(__hfma2(la_pair(wp[1]), x, __hfma2(wh, x, __hneg2(p0))));
                        }
                    } else {
                        const uint64_t w2 = tc::f32x2(w[z], w[z]);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            uint64_t x = tc::f32x2_mul(w2, pair_of(in[k] << 16, in[k] & 0xffff0000u));
                            p[0][k] = tc::f32x2_bf16(x);
                            x = tc::f32x2_fma(neg, pair_of(p[0][k] << 16, p[0][k] & 0xffff0000u), x);
                            p[1][k] = tc::f32x2_bf16(x);
                            x = tc::f32x2_fma(neg, pair_of(p[1][k] << 16, p[1][k] & 0xffff0000u), x);
                            p[2][k] = tc::f32x2_bf16(x);
                        }
                        *reinterpret_cast<uint4 *>(dst + 2 * SLAB) = make_uint4(p[2][0], p[2][1], p[2][2], p[2][3]);
                    }
                    *reinterpret_cast<uint4 *>(dst) = make_uint4(p[0][0], p[0][1], p[0][2], p[0][3]);
                    *reinterpret_cast<uint4 *>(dst + SLAB) = make_uint4(p[1][0], p[1][1], p[1][2], p[1][3]);
                }
                if (!STATE_ONLY && (odd & 0x80008000u)) {
#pragma unroll 1
                    for (int z = 0; z < 8; ++z) {
                        uint32_t *at = reinterpret_cast<uint32_t *>(smem + L::V + s * SLAB + off + (i + (z >> 2)) * 4096) + (z & 3);
                        uint32_t in = *at;
                        if ((in & 0x7f80u) == 0x7f80u) in &= 0xffff0000u;
                        if ((in & 0x7f800000u) == 0x7f800000u) in &= 0xffffu;
                        *at = in;
                    }
                    ((volatile int *)sm->odd_tile)[t % MARKS] = t + 1;
                }
                tc::fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm->vw_full[u]);
            }
            if (STATE_ONLY && lane == 0) tc::mbar_arrive(&sm->free_v[s]);
        }
    } else if (warp >= WARP_STATE && warp < WARP_O) {
        // ------------------------------------------------------------------ the state: half a key's columns per thread (of
        // 64 keys a quarter: the rows of D come twice)
        constexpr int NC = DK == 128 ? 32 : 16;
        const int q4 = warp & 3, d = (q4 * 32 + lane) % DK;
        const int cc = (warp - WARP_STATE) / 4 * 32 + (DK == 128 ? 0 : (q4 >> 1) * 16);
        const uint32_t row = tmem + ((uint32_t)(q4 * 32) << 16) + cc;
        const int64_t bh = (int64_t)b * a.H + h, ssize = (int64_t)j.dk * j.dv;
        const int64_t step = j.transposed ? 1 : j.dk, at0 = j.transposed ? (int64_t)d * j.dv + cc : cc * step + d;
        const int nv = d < j.dk ? j.dv - cc : 0;             // columns of this thread's that the state has (in eights)
        const float *from = STATE_ONLY ? nullptr
                            : seg > 0  ? j.seg + (bh * a.nseg + seg) * a.per * ssize
                            : j.s_in   ? j.s_in + bh * ssize
                                       : nullptr;
        uint64_t st[NC / 2];
#pragma unroll
        for (int e = 0; e < NC / 2; ++e) st[e] = from && (2 * e & ~7) < nv ? tc::f32x2(from[at0 + 2 * e * step], from[at0 + (2 * e + 1) * step]) : 0ull;
        auto publish = [&]() {                   // the bf16 copy that QS reads: row d, columns side by side
#pragma unroll
            for (int e = 0; e < NC / 2; e += 4)
                *reinterpret_cast<uint4 *>(smem + L::S + tc::sw128_offset(d, (cc >> 3) + (e >> 2))) =
                    make_uint4(tc::f32x2_bf16(st[e]), tc::f32x2_bf16(st[e + 1]), tc::f32x2_bf16(st[e + 2]), tc::f32x2_bf16(st[e + 3]));
            tc::fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm->s_full);
        };
        // S <- dec S + D, the small parts of D first, so that S is rounded once a tile.  (The accumulators of the products cut
        // where this rounds: tiles that added up in D would lose 2^-24 of all they hold with each of eight products, always
        // towards zero: 1e-5 after 57 tiles of a head that forgets nothing.)
        constexpr int AT = DK == 128 ? 8 : 16;               // columns at a time (128 keys fill the registers with S)
        auto load = [](uint32_t from, uint32_t (&r)[AT]) {
            if constexpr (AT == 8) tc::tmem_ld8(from, r);
            else tc::tmem_ld16(from, r);
        };
        auto collect = [&](uint32_t from, LaDecay dec) {
            const uint64_t hi2 = tc::f32x2(dec.hi, dec.hi), lo2 = tc::f32x2(dec.lo, dec.lo);
#pragma unroll
            for (int k = 0; k < NC; k += AT) {
                uint32_t x[AT], y[AT];
                load(from + LDV + k, x);
                if (parts == 3) {
                    load(from + 2 * LDV + k, y);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < AT; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) + __uint_as_float(y[e]));
                }
                load(from + k, y);
                tc::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < AT / 2; ++e) {
                    uint64_t &s = st[k / 2 + e];
                    uint64_t d = tc::f32x2_add(pair_of(x[2 * e], x[2 * e + 1]), pair_of(y[2 * e], y[2 * e + 1]));
                    if (!STATE_ONLY && parts == 3) d = tc::f32x2_fma(lo2, s, d);
                    s = tc::f32x2_fma(hi2, s, d);
                }
            }
        };
        if (!STATE_ONLY) {
            if (lane == 0) sm->whole[warp - WARP_STATE] = parts == 3 ? la_decay(a.log_decay[h], LT) : LaDecay{sm->pow[LT], 0.f};
            __syncwarp();
        }
        for (int t = 0; t < (STATE_ONLY ? 0 : ntiles); ++t) {
            if (t > 0) tc::mbar_wait(&sm->qs_done, (t - 1) & 1, abort_flag, d_status);
            publish();
            const int n = tile_n(t);
            tc::mbar_wait(&sm->kv_done[1], t & 1, abort_flag, d_status);
            tc::tc_fence_after();
            collect(row + TM_KV, n == LT ? sm->whole[warp - WARP_STATE] : LaDecay{sm->pow[n], 0.f});
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm->kv_read);
        }
        for (int t = 0; t < (STATE_ONLY ? ntiles : 0); ++t) {
            tc::mbar_wait(&sm->kv_done[vw_slot(t, 1)], vw_phase(t) & 1, abort_flag, d_status);
            tc::tc_fence_after();
            collect(row + d_of(t), LaDecay{1.f, 0.f});
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm->d_free[t & 1]);
        }
        float *to = STATE_ONLY ? j.seg + (bh * nall + seg + 1) * ssize
                    : seg == a.nseg - 1 && j.s_out ? j.s_out + bh * ssize : nullptr;
        if (to) {
#pragma unroll
            for (int e = 0; e < NC / 2; ++e) {
                if ((2 * e & ~7) >= nv) continue;
                const float2 v = tc::f32x2_get(st[e]);
                to[at0 + 2 * e * step] = v.x;
                to[at0 + (2 * e + 1) * step] = v.y;
            }
        }
    } else if (warp >= WARP_O) {
        // ------------------------------------------------------------------ o: a row per thread, staged where V stood
        const int q4 = warp & 3, r = q4 * 32 + lane;
        const uint32_t row = tmem + ((uint32_t)(q4 * 32) << 16);
        for (int t = 0; t < (STATE_ONLY ? 0 : ntiles); ++t) {
            const int s = t % NS, n = tile_n(t), at = tile_at(t);
            const float w = r < n ? j.scale_c * sm->pow[rev ? n - 1 - r : r + 1] : 0.f;
            const uint64_t w2 = tc::f32x2(w, w);
            tc::mbar_wait(&sm->qs_done, t & 1, abort_flag, d_status);
            tc::mbar_wait(&sm->pv_done, t & 1, abort_flag, d_status);
            tc::tc_fence_after();
            const bool odd = ((volatile int *)sm->odd_tile)[t % MARKS] == t + 1;
            uint8_t *stage = smem + L::V + s * SLAB;
#pragma unroll 1
            for (int c = 0; c < 64; c += 16) {
                uint32_t x[16], y[16];
                tc::tmem_ld16(row + TM_QS + c, x);
                tc::tmem_ld16(row + TM_PV + c, y);
                tc::tmem_ld_wait();
                if (odd) {                       // what is not finite, for the rows that see it
                    const __nv_bfloat16 *v = (const __nv_bfloat16 *)j.v + ((int64_t)b * a.L + at) * j.ldv +
                                             (int64_t)(h / j.rv) * j.dv + c;
#pragma unroll 1
                    for (int jb = 0; jb < 8; ++jb) {
                        uint32_t p[8];
                        tc::tmem_ld8(row + TM_P + jb * 8, p);
                        tc::tmem_ld_wait();
#pragma unroll 1
                        for (int k = 0; k < 16; ++k) {
                            const int jj = jb * 16 + k;
                            uint32_t pw = 0;
#pragma unroll
                            for (int z = 0; z < 8; ++z) pw = z == (k >> 1) ? p[z] : pw;
                            const float pf = __uint_as_float(k & 1 ? pw & 0xffff0000u : pw << 16);
                            if (jj < n && (rev ? jj >= r : jj <= r)) {
#pragma unroll
                                for (int g = 0; g < 16; g += 8) {
                                    if (c + g >= j.dv) continue;
                                    const uint4 u4 = *reinterpret_cast<const uint4 *>(v + jj * j.ldv + g);
                                    const uint32_t in[4] = {u4.x, u4.y, u4.z, u4.w};
#pragma unroll
                                    for (int e = 0; e < 8; ++e) {
                                        const float u = __uint_as_float(e & 1 ? in[e >> 1] & 0xffff0000u : in[e >> 1] << 16);
                                        if (!isfinite(u)) y[g + e] = __float_as_uint(fmaf(pf, u, __uint_as_float(y[g + e])));
                                    }
                                }
                            }
                        }
                        __syncwarp();
                    }
                }
                if (c == 48) {                   // everything in tensor memory has been read
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&sm->o_free);
                }
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float2 u = tc::f32x2_get(tc::f32x2_fma(w2, pair_of(x[e], x[e + 1]), pair_of(y[e], y[e + 1])));
                    y[e] = __float_as_uint(u.x);
                    y[e + 1] = __float_as_uint(u.y);
                }
                if (j.o_f32) {
                    if (r < n) {
                        uint4 *p = reinterpret_cast<uint4 *>((float *)j.o + ((int64_t)b * a.L + at + r) * j.ldo + (int64_t)h * j.dv + c);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c + (4 * e & ~7) < j.dv) p[e] = make_uint4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
                    }
                    __syncwarp();
                } else {
#pragma unroll
                    for (int e = 0; e < 16; e += 8)
                        *reinterpret_cast<uint4 *>(stage + tc::sw128_offset(r, (c + e) >> 3)) =
                            make_uint4(tc::f32x2_bf16(pair_of(y[e], y[e + 1])), tc::f32x2_bf16(pair_of(y[e + 2], y[e + 3])),
                                       tc::f32x2_bf16(pair_of(y[e + 4], y[e + 5])), tc::f32x2_bf16(pair_of(y[e + 6], y[e + 7])));
                }
            }
            if (j.o_f32) {
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm->free_v[s]);
                continue;
            }
            tc::fence_proxy_async_smem();
            tc::named_bar_sync(1, 128);
            if (q4 == 0) {                       // (rows behind the sequence are clipped by the tensor map)
                if (tc::elect_one()) {
                    tc::tma_store_4d(&maps.o[ji], stage, 0, h, at, b);
                    tc::bulk_commit_group();
                    tc::bulk_wait_read_all();
                    tc::mbar_arrive(&sm->free_v[s]);
                }
                __syncwarp();
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == WARP_ALLOC) tc::tmem_dealloc(tmem, TM_COLS);
}

template <int DK, bool STATE_ONLY>
bool run_tiles(LaunchCtx &ctx, const Maps &maps, const LaArgs &a)
{
    const size_t smem = Sm<DK>::SMALL + sizeof(Small);
    if (!ensure_dynamic_smem((const void *)la_tiles_kernel<DK, STATE_ONLY>, smem)) return false;
    const int64_t n = (int64_t)a.njobs * a.B * a.H * (STATE_ONLY ? (a.nseg - 1) * a.per : a.nseg);
    ctx.begin(STATE_ONLY ? STAGE_LA_STATES : STAGE_LA_TILES);
    launch_kernel(la_tiles_kernel<DK, STATE_ONLY>, dim3((unsigned)n), dim3(THREADS), smem, ctx.stream, true, maps, a,
                  ctx.d_status);
    ctx.end();
    return cudaGetLastError() == cudaSuccess;
}

}  // namespace

bool la_stream_map(TmapCache *cache, CUtensorMap *m, const void *p, int D, int streams, int L, int B, int64_t ld)
{
    const uint64_t dims[4] = {(uint64_t)D, (uint64_t)streams, (uint64_t)L, (uint64_t)B};
    const uint64_t strides[3] = {(uint64_t)D * 2, (uint64_t)ld * 2, (uint64_t)ld * L * 2};
    const uint32_t box[4] = {64, 1, LT, 1};
    return encode_tmap_bf16_cached(cache, m, p, 4, dims, strides, box);
}

bool la_tiles_shape(int dtype, int N, int P)
{
    return dtype == SWIMBA_DTYPE_BF16 && N <= 128 && P <= 128;
}

int launch_la_tiles(LaunchCtx &ctx, const LaArgs &all, bool states, int sm_count)
{
    // jobs of one pair of head sizes, made up to 64 or 128 with zeros by the copies, go in one launch
    auto full = [](int n) { return n <= 64 ? 64 : 128; };
    for (int dk : {64, 128})
        for (int dv : {64, 128}) {
            LaArgs a = all;
            a.njobs = 0;
            for (int i = 0; i < all.njobs; ++i)
                if (full(all.job[i].dk) == dk && full(all.job[i].dv) == dv) a.job[a.njobs++] = all.job[i];
            if (a.njobs == 0) continue;
            if (dv == 128) {
                const int rc = launch_la_wide(ctx, a, states, sm_count);
                if (rc != SWIMBA_OK) return rc;
                continue;
            }
            Maps maps;
            for (int i = 0; i < a.njobs; ++i) {
                const LaJob &j = a.job[i];
                if (!la_stream_map(ctx.tmaps, &maps.q[i], j.q, j.dk, a.H / j.rq, a.L, a.B, j.ldq) ||
                    !la_stream_map(ctx.tmaps, &maps.k[i], j.k, j.dk, a.H / j.rk, a.L, a.B, j.ldk) ||
                    !la_stream_map(ctx.tmaps, &maps.v[i], j.v, j.dv, a.H / j.rv, a.L, a.B, j.ldv) ||
                    (!states && !j.o_f32 && !la_stream_map(ctx.tmaps, &maps.o[i], j.o, j.dv, a.H, a.L, a.B, j.ldo)))
                    return SWIMBA_ERR_CUDA;
            }
            const bool ok = dk == 64 ? (states ? run_tiles<64, true>(ctx, maps, a) : run_tiles<64, false>(ctx, maps, a))
                                     : (states ? run_tiles<128, true>(ctx, maps, a) : run_tiles<128, false>(ctx, maps, a));
            if (!ok) return SWIMBA_ERR_CUDA;
        }
    return SWIMBA_OK;
}

}  // namespace swimba
