// Linear attention with a decay for each head on the tensor cores, heads of 65 to 128 values (bf16; up to 128
// entries of keys; made up with zeros as there): the same five steps per tile of 128 tokens as in la_tiles.cu, with all values of a head in one CTA, so that scores and masks
// are made once.  What makes room for that in shared memory (two or three stages of Q, K and V, the bf16 state):
//   w V   is made transposed, [DV, tokens], straight into tensor memory, a quarter of a tile at a time and two of them in
//         turn, and is the A operand of KV:  D = (w V)^T K
//   S     lies in tensor memory in fp32, [DV, DK]; between two tiles it is read, rounded for QS and scaled by lambda^n,
//         and KV adds to it (where the state is a result, without what the copy for QS holds of it)
//   O     one region: Q S^T, scaled row by row in place, then P V on top
// Shared memory bounds such a tile first: 7860 cycles of reads and writes for two CTAs of 64 values each against 3900 here;
// the chain scores - masks - P V - o of a tile is not much shorter.  Measured, 4 sequences of 8192 tokens, 16 heads of
// 128 x 128: 190 us (floor 82), 3.7 us a tile and CTA, 64 walks on 128 SMs; without an exit state 152, 3.0 us a tile; their
// gradients, 192 walks, 428 us (floor 144).
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <type_traits>

#include "la.h"
#include "tc05.cuh"

namespace swimba {

namespace {

constexpr int LT = 128;                      // tokens per tile
constexpr int DV = 128;
constexpr int MARKS = 4;                     // places of the marks of tiles whose V is not all finite
constexpr uint32_t SLAB = LT * 128;          // 128 rows of 64 bf16
constexpr uint32_t VB = 2 * SLAB;            // bytes of a V tile
// warps: copies, products, tensor memory, spare; 8 for the masks and, while scores are made, the state, 8 for w V, 8 for o
constexpr int THREADS = 896;
constexpr int WARP_TMA = 0, WARP_MMA = 1, WARP_ALLOC = 2, WARP_MASK = 4, WARP_W = 12, WARP_O = 20;
// tensor memory columns: scores and over them P (bf16), O, S, w V of quarters of a tile: four of them in two parts, or two in three
constexpr uint32_t TM_QK = 0, TM_O = 128, TM_S = 256, TM_VW = 384, TM_COLS = 512;

template <int DK> struct Sm {
    // stages: a Q tile is free early in its step, a K tile half way, a V tile when o, staged in its place, is on its way
    static constexpr int NQ = DK == 64 ? 2 : 1, NK = DK == 64 ? 3 : 2, NV = 3;
    static constexpr uint32_t QB = DK / 64 * SLAB;        // bytes of a Q or K tile
    static constexpr uint32_t Q = 0, K = Q + NQ * QB, V = K + NK * QB, S = V + NV * VB, SMALL = S + QB;
};
struct Small {
    uint64_t full_q[2], full_k[3], full_v[3], free_q[2], free_k[3], free_v[3];
    uint64_t qk_full, p_full, qs_done, o_scaled, pv_done, o_free, s_full, s_scaled, kv_done, vw_full[4], vw_done[4];
    uint64_t d_full[2], d_free[2];           // the additions of a tile that only carries the state: made, added
    uint32_t tmem;
    int abort_flag;
    int odd_tile[MARKS];                     // 1 + the tile whose V is not all finite, in place t % 4 (as in la_tiles.cu)
    alignas(16) float pow_col[32];           // factors of a score block's columns
    float pow_diag[64];                      // scale_p lambda^|m - 31|: the block on the diagonal
    float pow[LT + 1];                       // lambda^m
    LaDecay whole[8];                        // lambda^LT in two floats, for each warp of the state
    alignas(16) float weight[LT];            // of a whole tile's tokens in w V
    alignas(16) uint32_t wsplit[LT / 2][2];  // their bf16 parts, two tokens at a time
};
static_assert(offsetof(Small, pow_col) % 16 == 0 && offsetof(Small, weight) % 16 == 0 && offsetof(Small, wsplit) % 16 == 0 && Sm<64>::SMALL % 16 == 0 && Sm<128>::SMALL % 16 == 0, "read in fours");

struct Maps {
    CUtensorMap q[LA_MAX_JOBS], k[LA_MAX_JOBS], v[LA_MAX_JOBS], o[LA_MAX_JOBS];
};

__device__ __forceinline__ float low_half(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high_half(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
__device__ __forceinline__ uint32_t bits2(uint32_t a, uint32_t b) { return tc::pack_bf16x2(__uint_as_float(a), __uint_as_float(b)); }

// STATE_ONLY: from a zero state, and only the end state is kept (in seg).
template <int DK, bool STATE_ONLY>
__global__ void __launch_bounds__(THREADS, 1)
la_wide_kernel(const __grid_constant__ Maps maps, const __grid_constant__ LaArgs a, int *d_status)
{
    typedef Sm<DK> L;
    constexpr int NQ = L::NQ, NK = L::NK, NV = L::NV;
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
    int part = 0, nparts = 1;
    if (!STATE_ONLY && id >= a.whole) {
        nparts = a.ncut;
        part = (int)((id - a.whole) % nparts);
        id = a.whole + (id - a.whole) / nparts;
    }
    const int ji = (int)(id % a.njobs);
    id /= a.njobs;
    // segments, or pieces of them for the states alone, in the order of the walk (the last segment's end state enters nothing)
    const int nall = STATE_ONLY ? a.nseg * a.per : a.nseg, nrun = STATE_ONLY ? nall - a.per : nall;
    const int seg = (int)(id % nrun), len = STATE_ONLY ? a.seg_len / a.per : a.seg_len;
    id /= nrun;
    const int h = (int)(id % a.H), b = (int)(id / a.H);
    const LaJob &j = a.job[ji];
    const bool rev = j.reverse != 0;
    // three parts where the state is a result; two where only the read of it is, whose copy is rounded to bf16
    const int parts = j.s_out && (STATE_ONLY || (seg == nall - 1 && part == nparts - 1)) ? 3 : 2, ring = 8 / parts;       // quarters of w V there is room for
    const int place = rev ? nall - 1 - seg : seg;
    const int t_begin = min(a.L, place * len), t_end = min(a.L, t_begin + len);
    const int nwalk = (t_end - t_begin + LT - 1) / LT;
    auto tile_at = [&](int t) { return t_begin + (rev ? nwalk - 1 - t : t) * LT; };        // first token of tile t
    auto tile_n = [&](int t) { return min(LT, t_end - tile_at(t)); };
    // this CTA's tiles: those in front of n_pre only carry the state; barriers that the others alone use count from there
    const int n_pre = STATE_ONLY ? nwalk : nparts > 1 ? a.cut[part] : 0;
    const int ntiles = STATE_ONLY || nparts == 1 ? nwalk : a.cut[part + 1];
    // where only the read of the state is (bf16) those tiles add up in S; else in D, of two tiles in turn where scores and o will be
    const bool apart = parts == 3;
    auto d_of = [](int t) { return t & 1 ? TM_O : TM_QK; };
    // tokens walked behind tile t in front of tile n_pre; tile -1: all of them
    auto tokens_left = [&](int t) {
        return rev ? (t < 0 ? t_end : tile_at(t)) - (n_pre > 0 ? tile_at(n_pre - 1) : t_end)
                   : min(t_end, t_begin + n_pre * LT) - (t < 0 ? t_begin : min(t_end, tile_at(t) + LT));
    };

    if (tid == 0) {
        for (int s = 0; s < NQ; ++s) {
            tc::mbar_init(&sm->full_q[s], 1);
            tc::mbar_init(&sm->free_q[s], 1);
        }
        for (int s = 0; s < NK; ++s) {
            tc::mbar_init(&sm->full_k[s], 1);
            tc::mbar_init(&sm->free_k[s], 1);
        }
        for (int s = 0; s < NV; ++s) {
            tc::mbar_init(&sm->full_v[s], 1);
            tc::mbar_init(&sm->free_v[s], 8);
        }
        for (int s = 0; s < 4; ++s) {
            tc::mbar_init(&sm->vw_full[s], 8);
            tc::mbar_init(&sm->vw_done[s], 1);
        }
        for (int i = 0; i < MARKS; ++i) sm->odd_tile[i] = 0;
        tc::mbar_init(&sm->qk_full, 1);
        tc::mbar_init(&sm->p_full, 8);
        tc::mbar_init(&sm->qs_done, 1);
        tc::mbar_init(&sm->o_scaled, 8);
        tc::mbar_init(&sm->pv_done, 1);
        tc::mbar_init(&sm->o_free, 8);
        tc::mbar_init(&sm->s_full, 8);
        tc::mbar_init(&sm->s_scaled, 8);
        tc::mbar_init(&sm->kv_done, 1);
        for (int s = 0; s < 2; ++s) {
            tc::mbar_init(&sm->d_full[s], 1);
            tc::mbar_init(&sm->d_free[s], STATE_ONLY ? 16 : 8);
        }
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
    else if (tid >= 512 && tid < 640) sm->weight[tid - 512] = j.scale_a * exp2f((rev ? tid - 511 : 639 - tid) * g2);
    else if (tid >= 640 && tid < 704) {
        const int q = 2 * (tid - 640);
        uint32_t p[2];
        la_split(j.scale_a * exp2f((rev ? q + 1 : 127 - q) * g2), j.scale_a * exp2f((rev ? q + 2 : 126 - q) * g2), p);
        *reinterpret_cast<uint2 *>(sm->wsplit[tid - 640]) = make_uint2(p[0], p[1]);
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = sm->tmem;

    if (warp == WARP_TMA) {
        // ------------------------------------------------------------------ loads, in the order in which room comes free
        const bool leader = tc::elect_one();
        auto load = [&](int t, int i, int ns, uint64_t *full, uint64_t *room, uint32_t dst, uint32_t bytes, const CUtensorMap *m, int stream) {
            if (i < 0 || t >= ntiles) return;
            const int st = i % ns;
            tc::mbar_wait(&room[st], ((i / ns) & 1) ^ 1, abort_flag, d_status);
            if (leader && !*(volatile int *)abort_flag) {
                tc::mbar_arrive_expect_tx(&full[st], bytes);
                for (uint32_t o = 0; o < bytes; o += SLAB)
                    tc::tma_load_4d(smem + dst + st * bytes + o, m, &full[st], (int)(o / SLAB) * 64, stream, tile_at(t), b);
            }
            __syncwarp();
        };
        auto load_q = [&](int t) { if (!STATE_ONLY) load(t, t - n_pre, NQ, sm->full_q, sm->free_q, L::Q, L::QB, &maps.q[ji], h / j.rq); };
        auto load_k = [&](int t) { load(t, t, NK, sm->full_k, sm->free_k, L::K, L::QB, &maps.k[ji], h / j.rk); };
        auto load_v = [&](int t) { load(t, t, NV, sm->full_v, sm->free_v, L::V, VB, &maps.v[ji], h / j.rv); };
        // with one Q tile at a time the next one's load is waited for: its rows are brought to L2 a step before
        auto ahead_q = [&](int t) {
            if (STATE_ONLY || NQ > 1 || t < n_pre || t >= ntiles) return;
#pragma unroll 1
            for (int r = tile_at(t) + lane; r < tile_at(t) + tile_n(t); r += 32) {
                const char *p = (const char *)((const __nv_bfloat16 *)j.q + ((int64_t)b * a.L + r) * j.ldq + (int64_t)(h / j.rq) * j.dk);
#pragma unroll
                for (int o = 0; o < DK * 2; o += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + o));
            }
            __syncwarp();
        };
        for (int t = -NV; t < ntiles; ++t) {
            load_q(t + NQ);
            ahead_q(t + NQ + 1);
            load_k(t + NK);
            load_v(t + NV);
        }
        // No copy may be in flight when the CTA leaves: after an abort nobody else has waited for the last ones (those
        // that were not issued any more never arrive, and these waits run out soon).
        auto settle = [&](uint64_t *full, uint32_t ph) {
            int quiet = 0;
            if (*(volatile int *)abort_flag) tc::mbar_wait(full, ph, &quiet, d_status, 10000000ll);
            else tc::mbar_wait(full, ph, abort_flag, d_status);
        };
        if (!STATE_ONLY)
            for (int t = max(0, ntiles - n_pre - NQ); t < ntiles - n_pre; ++t) settle(&sm->full_q[t % NQ], (t / NQ) & 1);
        for (int t = max(0, ntiles - NK); t < ntiles; ++t) settle(&sm->full_k[t % NK], (t / NK) & 1);
        for (int t = max(0, ntiles - NV); t < ntiles; ++t) settle(&sm->full_v[t % NV], (t / NV) & 1);
    } else if (warp == WARP_MMA) {
        // ------------------------------------------------------------------ products
        const bool leader = tc::elect_one();
        constexpr uint32_t id_qk = tc::idesc_bf16(128, 128, 0, 0);      // Q x K, Q x S (all K-major)
        constexpr uint32_t id_pv = tc::idesc_bf16(128, DV, 0, 1);       // P (TMEM) x V (MN-major)
        constexpr uint32_t id_kv = tc::idesc_bf16(128, DK, 0, 1);       // (w V)^T (TMEM) x K (MN-major)
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        const uint32_t base = tc::smem_u32(smem);
        const uint64_t dQ = tc::smem_desc_sw128(base + L::Q, 16, 1024), dK = tc::smem_desc_sw128(base + L::K, 16, 1024);
        const uint64_t dKt = tc::smem_desc_sw128(base + L::K, SLAB, 1024), dV = tc::smem_desc_sw128(base + L::V, SLAB, 1024);
        const uint64_t dS = tc::smem_desc_sw128(base + L::S, 16, 1024);
        auto scores = [&](int t) {
            const int f = t - n_pre;
            tc::mbar_wait(&sm->full_k[t % NK], (t / NK) & 1, abort_flag, d_status);
            tc::mbar_wait(&sm->full_q[f % NQ], (f / NQ) & 1, abort_flag, d_status);
            tc::tc_fence_after();
            if (leader) {
                const uint64_t q = tc::smem_desc_fresh(tc::smem_desc_advance(dQ, f % NQ * L::QB));
                const uint64_t k = tc::smem_desc_fresh(tc::smem_desc_advance(dK, t % NK * L::QB));
#pragma unroll
                for (int kk = 0; kk < DK / 16; ++kk) {
                    const uint32_t o = (kk >> 2) * SLAB + (kk & 3) * 32;
                    tc::mma_ss(tm + TM_QK, tc::smem_desc_advance(q, o), tc::smem_desc_advance(k, o), id_qk, kk > 0);
                }
                tc::mma_commit(&sm->qk_full);
            }
            __syncwarp();
        };
        // KV, by quarters of the tile, onto S or (fresh) into D; done: the barrier behind it
        auto add = [&](int t, auto fresh, uint32_t to, uint64_t *done) {
#pragma unroll 1
            for (int qd = 0; qd < 4; ++qd) {
                const int buf = qd & (ring - 1);
                tc::mbar_wait(&sm->vw_full[buf], parts == 3 ? qd >> 1 : t & 1, abort_flag, d_status);
                tc::tc_fence_after();
                if (leader) {
                    uint64_t k = tc::smem_desc_fresh(tc::smem_desc_advance(dKt, t % NK * L::QB + qd * 4096));
#pragma unroll 1
                    for (int p = 0; p < parts; ++p) {
                        tc::mma_ts(to, tm + TM_VW + (buf * parts + p) * 16, k, id_kv, !decltype(fresh)::value || qd + p > 0);
                        tc::mma_ts(to, tm + TM_VW + (buf * parts + p) * 16 + 8, tc::smem_desc_advance(k, 2048), id_kv, 1);
                    }
                    tc::mma_commit(&sm->vw_done[buf]);
                    if (qd == 3) {
                        if (done) tc::mma_commit(done);
                        tc::mma_commit(&sm->free_k[t % NK]);
                    }
                }
                __syncwarp();
            }
        };
#pragma unroll 1
        for (int t = 0; t < n_pre; ++t) {
            tc::mbar_wait(&sm->full_k[t % NK], (t / NK) & 1, abort_flag, d_status);
            if (apart) {                     // (what stood in D has been added)
                if (t > 1) tc::mbar_wait(&sm->d_free[t & 1], ((t >> 1) - 1) & 1, abort_flag, d_status);
                add(t, std::true_type{}, tm + d_of(t), &sm->d_full[t & 1]);
            } else {                         // (the state that enters is in S; of the states alone the first tile clears it)
                if (!STATE_ONLY && t == 0) tc::mbar_wait(&sm->d_free[0], 0, abort_flag, d_status);
                uint64_t *done = t == n_pre - 1 ? &sm->d_full[0] : nullptr;
                if (STATE_ONLY && t == 0) add(t, std::true_type{}, tm + TM_S, done);
                else add(t, std::false_type{}, tm + TM_S, done);
            }
        }
        if (ntiles > n_pre) {                // (scores and o come where D stood)
            for (int t = apart ? max(0, n_pre - 2) : n_pre; t < n_pre; ++t) tc::mbar_wait(&sm->d_free[t & 1], (t >> 1) & 1, abort_flag, d_status);
            scores(n_pre);
        }
#pragma unroll 1
        for (int t = n_pre; t < ntiles; ++t) {
            const int f = t - n_pre;
            // QS: the carried part, once the state is there and the epilogue has read the tile in front
            tc::mbar_wait(&sm->s_full, f & 1, abort_flag, d_status);
            if (f > 0) tc::mbar_wait(&sm->o_free, (f - 1) & 1, abort_flag, d_status);
            tc::tc_fence_after();
            if (leader) {
                const uint64_t q = tc::smem_desc_fresh(tc::smem_desc_advance(dQ, f % NQ * L::QB)), st = tc::smem_desc_fresh(dS);
#pragma unroll
                for (int kk = 0; kk < DK / 16; ++kk) {
                    const uint32_t o = (kk >> 2) * SLAB + (kk & 3) * 32;
                    tc::mma_ss(tm + TM_O, tc::smem_desc_advance(q, o), tc::smem_desc_advance(st, o), id_qk, kk > 0);
                }
                tc::mma_commit(&sm->qs_done);
                tc::mma_commit(&sm->free_q[f % NQ]);
            }
            __syncwarp();
            tc::mbar_wait(&sm->s_scaled, f & 1, abort_flag, d_status);
            add(t, std::false_type{}, tm + TM_S, &sm->kv_done);
            // PV, on top of the scaled carried part (and behind KV: by then w V has been made of all of V, where o is staged)
            tc::mbar_wait(&sm->full_v[t % NV], (t / NV) & 1, abort_flag, d_status);
            tc::mbar_wait(&sm->p_full, f & 1, abort_flag, d_status);
            tc::mbar_wait(&sm->o_scaled, f & 1, abort_flag, d_status);
            tc::tc_fence_after();
            if (leader) {
                const uint64_t v = tc::smem_desc_fresh(tc::smem_desc_advance(dV, t % NV * VB));
#pragma unroll
                for (int kk = 0; kk < LT / 16; ++kk)
                    tc::mma_ts(tm + TM_O, tm + TM_QK + (kk >> 2) * 64 + (kk & 3) * 8, tc::smem_desc_advance(v, kk * 2048), id_pv, 1);
                tc::mma_commit(&sm->pv_done);
            }
            __syncwarp();
            if (t + 1 < ntiles) {
                // the next scores go where P stands, which the epilogue reads too if V was not all finite
                tc::mbar_wait(&sm->pv_done, f & 1, abort_flag, d_status);
                if (((volatile int *)sm->odd_tile)[t % MARKS] == t + 1) tc::mbar_wait(&sm->o_free, f & 1, abort_flag, d_status);
                scores(t + 1);
            }
        }
    } else if (STATE_ONLY && ((warp >= WARP_MASK && warp < WARP_W) || warp >= WARP_O)) {
        // ------------------------------------------------------------------ the state alone, a quarter of a value's row per
        // thread: where it is a result, every tile's additions by themselves, and added up here, where sums are rounded, not cut
        constexpr int NC = DK / 4;
        const int q4 = warp & 3, i = q4 * 32 + lane, c0 = (warp < WARP_W ? (warp - WARP_MASK) >> 2 : 2 + ((warp - WARP_O) >> 2)) * NC;
        const uint32_t row = tmem + ((uint32_t)(q4 * 32) << 16) + c0;
        uint64_t st[NC / 2];
#pragma unroll
        for (int e = 0; e < NC / 2; ++e) st[e] = 0ull;
        for (int t = 0; t < (apart ? ntiles : min(ntiles, 1)); ++t) {
            tc::mbar_wait(&sm->d_full[t & 1], (t >> 1) & 1, abort_flag, d_status);
            tc::tc_fence_after();
#pragma unroll
            for (int c = 0; c < NC; c += 16) {
                uint32_t x[16];
                tc::tmem_ld16(row + (apart ? d_of(t) : TM_S) + c, x);
                tc::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    st[c / 2 + e] = tc::f32x2_add(st[c / 2 + e], tc::f32x2(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])));
            }
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm->d_free[t & 1]);
        }
        const int64_t ssize = (int64_t)j.dk * j.dv, step = j.transposed ? j.dv : 1;
        float *to = j.seg + (((int64_t)b * a.H + h) * nall + seg + 1) * ssize + (j.transposed ? c0 * step + i : (int64_t)i * j.dk + c0);
        const int nd = i < j.dv ? j.dk - c0 : 0;                 // entries of this thread's that the state has (in eights)
#pragma unroll
        for (int e = 0; e < NC; e += 2) {
            if ((e & ~7) >= nd) continue;
            const float2 v = tc::f32x2_get(st[e / 2]);
            to[e * step] = v.x;
            to[(e + 1) * step] = v.y;
        }
    } else if (!STATE_ONLY && warp >= WARP_MASK && warp < WARP_W) {
        // ------------------------------------------------------------------ masks: half a row of the scores per thread, its
        // result over the first half of what it was made from; and the state, half a value's row per thread: between two
        // tiles its bf16 copy for QS goes to shared memory and it is scaled where it stands.
        // The accumulators of the products cut where other sums round.  S, with 24 products a tile added to it, would lose up to
        // 2^-23 of all it holds with each, always towards zero (2.5e-5 of a state of 64 tiles).  Where the state is a result, what
        // the copy holds is therefore taken out of S until the tile's products are in: they add up beside what a tile forgets
        // of it and 2^-9 (5e-7, whatever the memory).  Heads that forget more than half of it in a tile have no use for that.
        const int q4 = warp & 3, half = (warp - WARP_MASK) >> 2, i = q4 * 32 + lane;
        const uint32_t quarter = tmem + ((uint32_t)(q4 * 32) << 16), row = quarter + TM_QK + half * 64;
        const float scale_p = j.scale_p;
        const uint32_t keep = rev ? 0xffffffffu << lane : 0xffffffffu >> (31 - lane);
        constexpr int NC = DK / 2;
        const uint32_t srow = quarter + TM_S + half * NC;
        const int64_t bh = (int64_t)b * a.H + h, ssize = (int64_t)j.dk * j.dv;
        const int64_t step = j.transposed ? j.dv : 1, at0 = j.transposed ? half * NC * step + i : (int64_t)i * j.dk + half * NC;
        const int nd = i < j.dv ? j.dk - half * NC : 0;          // entries of this thread's that the state has (in eights)
        if (n_pre < ntiles) {                    // the state that enters
            const float *from = seg > 0  ? j.seg + (bh * a.nseg + seg) * a.per * ssize
                                : j.s_in ? j.s_in + bh * ssize
                                         : nullptr;
            const float dec = n_pre > 0 ? exp2f(tokens_left(-1) * g2) : 1.f;
#pragma unroll 1
            for (int c = 0; c < NC; c += 16) {
                uint32_t x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = from && c + (e & 8) < nd ? __float_as_uint(dec * from[at0 + (c + e) * step]) : 0u;
                __syncwarp();
                tc::tmem_st16(srow + c, x);
            }
            tc::tmem_st_wait();
            // and what the tiles in front add to it, as it is in front of the first tile that this CTA gives outputs of
            if (!apart && n_pre > 0) {
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm->d_free[0]);
                tc::mbar_wait(&sm->d_full[0], 0, abort_flag, d_status);
                tc::tc_fence_after();
            }
            for (int t = 0; t < (apart ? n_pre : 0); ++t) {
                tc::mbar_wait(&sm->d_full[t & 1], (t >> 1) & 1, abort_flag, d_status);
                tc::tc_fence_after();
                const uint32_t d = quarter + d_of(t) + half * NC;
#pragma unroll 1
                for (int c = 0; c < NC; c += 16) {
                    uint32_t x[16], y[16];
                    tc::tmem_ld16(srow + c, x);
                    tc::tmem_ld16(d + c, y);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) + __uint_as_float(y[e]));
                    tc::tmem_st16(srow + c, x);
                }
                tc::tmem_st_wait();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm->d_free[t & 1]);
            }
        }
        const bool take = parts == 3 && sm->pow[LT] >= 0.5f;
        LaDecay &whole = sm->whole[warp - WARP_MASK];
        if (take && lane == 0) whole = la_decay(a.log_decay[h], LT);
        __syncwarp();
        uint8_t *copy = smem + L::S + i * 128 + (DK == 128 ? half * SLAB : 0);       // (its chunks of 16 bytes are swizzled by the row)
        auto copy_of = [&](int c) { return reinterpret_cast<uint4 *>(copy + ((((DK == 128 ? 0 : half * 4) + (c >> 3)) ^ (i & 7)) * 16)); };
        auto put_back = [](uint32_t *v, const uint4 &c) {            // eight entries and what their copy holds of them
            const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[2 * e] = __float_as_uint(__uint_as_float(v[2 * e]) + low_half(w[e]));
                v[2 * e + 1] = __float_as_uint(__uint_as_float(v[2 * e + 1]) + high_half(w[e]));
            }
        };
        // half a row of the state through f, 16 columns at a time; then the barrier of the pass, the copy's or the one for S
        auto pass_over = [&](auto &&f, bool copy_pass) {
            uint32_t x[2][16];
            tc::tmem_ld16(srow, x[0]);
#pragma unroll 1
            for (int c = 0; c < NC; c += 32) {
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                    const int cz = c + z * 16;
                    tc::tmem_ld_wait();
                    tc::tmem_ld16(srow + (cz + 16) % NC, x[z ^ 1]);    // (behind the last: the first once more, unused)
                    f(cz, x[z]);
                }
            }
            tc::tmem_ld_wait();
            tc::tmem_st_wait();
            if (copy_pass) tc::fence_proxy_async_smem();
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(copy_pass ? &sm->s_full : &sm->s_scaled);
        };
        auto put_copy = [&](int c, const uint32_t (&r)[16]) {
#pragma unroll
            for (int e = 0; e < 16; e += 8)
                *copy_of(c + e) = make_uint4(bits2(r[e], r[e + 1]), bits2(r[e + 2], r[e + 3]), bits2(r[e + 4], r[e + 5]), bits2(r[e + 6], r[e + 7]));
        };
        // the state that enters tile t; the copy first: QS runs while the state is scaled for KV to add to
        auto hand_over = [&](int t) {
            if (!take) {
                const float dec = sm->pow[tile_n(t)];
                pass_over([&](int c, uint32_t (&r)[16]) { put_copy(c, r); }, true);
                pass_over([&](int c, uint32_t (&r)[16]) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(dec * __uint_as_float(r[e]));
                    tc::tmem_st16(srow + c, r);
                }, false);
            } else {
                const LaDecay dec = tile_n(t) == LT ? whole : LaDecay{sm->pow[tile_n(t)], 0.f};
                pass_over([&](int c, uint32_t (&r)[16]) {
                    if (t > n_pre) {
                        put_back(r, *copy_of(c));
                        put_back(r + 8, *copy_of(c + 8));
                        tc::tmem_st16(srow + c, r);
                    }
                    put_copy(c, r);
                }, true);
                pass_over([&](int c, uint32_t (&r)[16]) {
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        const uint32_t c2 = bits2(r[e], r[e + 1]);
                        const float s0 = __uint_as_float(r[e]), s1 = __uint_as_float(r[e + 1]);
                        r[e] = __float_as_uint(fmaf(dec.lo, s0, fmaf(dec.hi, s0, -low_half(c2))));
                        r[e + 1] = __float_as_uint(fmaf(dec.lo, s1, fmaf(dec.hi, s1, -high_half(c2))));
                    }
                    tc::tmem_st16(srow + c, r);
                }, false);
            }
        };
        if (ntiles > n_pre) hand_over(n_pre);
        for (int t = n_pre; t < ntiles; ++t) {
            const int f = t - n_pre;
            tc::mbar_wait(&sm->qk_full, f & 1, abort_flag, d_status);
            tc::tc_fence_after();
#pragma unroll 1
            for (int k = 0; k < 2; ++k) {
                const int bl = half * 2 + k;
                uint32_t x[32], o[16];
                if (rev ? bl < q4 : bl > q4) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = 0u;
                } else {
                    tc::tmem_ld32(row + k * 32, x);
                    tc::tmem_ld_wait();
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
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 c = *reinterpret_cast<const float4 *>(&sm->pow_col[e]);
                            o[e / 2] = tc::pack_bf16x2(__uint_as_float(x[e]) * (rho * c.x), __uint_as_float(x[e + 1]) * (rho * c.y));
                            o[e / 2 + 1] = tc::pack_bf16x2(__uint_as_float(x[e + 2]) * (rho * c.z), __uint_as_float(x[e + 3]) * (rho * c.w));
                        }
                    }
                }
                tc::tmem_st16(row + k * 16, o);
            }
            tc::tmem_st_wait();
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm->p_full);
            if (t + 1 < ntiles) {
                tc::mbar_wait(&sm->kv_done, f & 1, abort_flag, d_status);
                tc::mbar_wait(&sm->qs_done, f & 1, abort_flag, d_status);
                tc::tc_fence_after();
                hand_over(t + 1);
            }
        }
        float *to = seg == a.nseg - 1 && part == nparts - 1 && j.s_out ? j.s_out + bh * ssize : nullptr;
        if (to) {                                // (what the copy holds of it is still there)
            tc::mbar_wait(&sm->kv_done, (ntiles - n_pre - 1) & 1, abort_flag, d_status);
            tc::tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < NC; c += 16) {
                uint32_t x[16];
                __syncwarp();
                tc::tmem_ld16(srow + c, x);
                tc::tmem_ld_wait();
                if (take) {
                    put_back(x, *copy_of(c));
                    put_back(x + 8, *copy_of(c + 8));
                }
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (c + (e & 8) < nd) to[at0 + (c + e) * step] = __uint_as_float(x[e]);
            }
        }
    } else if (warp >= WARP_W && warp < WARP_O) {
        // ------------------------------------------------------------------ (w V)^T: 16 values of a quarter of a tile, 32
        // tokens, transposed on the way from shared memory
        const int q4 = warp & 3, lg = (warp - WARP_W) >> 2;
        // this lane's row of the 8 x 8 blocks: (token octet, value octet) = (lane / 16, lane / 8 % 2), token lane % 8
        const uint32_t row0 = tc::sw128_offset((lane >> 4) * 8 + (lane & 7), (q4 & 1) * 4 + lg * 2 + ((lane >> 3) & 1));
        const uint32_t slab = L::V + (q4 >> 1) * SLAB, src0 = tc::smem_u32(smem) + slab + row0;
        const uint32_t to = tmem + TM_VW + ((uint32_t)(q4 * 32 + lg * 16) << 16);
        for (int t = 0; t < ntiles; ++t) {
            const int s = t % NV, n = tile_n(t), shift = rev ? 0 : LT - n;
            // (tiles that only carry the state: their additions as they are in front of the first that does not)
            const float tail = t < n_pre ? exp2f(tokens_left(t) * g2) : 1.f;
            tc::mbar_wait(&sm->full_v[s], (t / NV) & 1, abort_flag, d_status);
            __nv_bfloat162 odd = la_pair(0u);         // becomes NaN with the first entry that is not finite
#pragma unroll 1
            for (int qd = 0; qd < 4; ++qd) {
                uint32_t r[8], w[4][2];               // (weights of two tokens: three parts as floats, two in bf16 parts)
                const uint32_t at = src0 + s * VB + qd * 4096;
                tc::ldmatrix_x4_trans(at, r[0], r[1], r[2], r[3]);
                tc::ldmatrix_x4_trans(at + 2048, r[4], r[5], r[6], r[7]);      // (16 tokens on: same swizzle)
                const int j0 = qd * 32 + (lane & 3) * 2;
                if (t >= n_pre && n == LT) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const uint2 x = *reinterpret_cast<const uint2 *>(parts == 3 ? (const uint32_t *)&sm->weight[j0 + c * 8]
                                                                                    : sm->wsplit[(j0 >> 1) + c * 4]);
                        w[c][0] = x.x; w[c][1] = x.y;
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int jj = j0 + c * 8;
                        const float w0 = jj < n ? tail * sm->weight[jj + shift] : 0.f, w1 = jj + 1 < n ? tail * sm->weight[jj + 1 + shift] : 0.f;
                        if (parts == 3) { w[c][0] = __float_as_uint(w0); w[c][1] = __float_as_uint(w1); }
                        else la_split(w0, w1, w[c]);
                    }
                }
                const int buf = qd & (ring - 1);
                if (4 * t + qd >= ring) {             // (what stood in this place of the ring has been multiplied)
                    tc::mbar_wait(&sm->vw_done[buf], (parts == 3 ? qd >> 1 : t & 1) ^ 1, abort_flag, d_status);
                    tc::tc_fence_after();
                }
                if (!STATE_ONLY)
#pragma unroll
                    for (int e = 0; e < 8; ++e) odd = __hfma2(la_pair(r[e]), la_pair(0u), odd);
                const uint32_t dst = to + buf * parts * 16;
                uint32_t p[8];
                if (parts == 2) {                     // (the remainder of a bf16 product is a bf16 number: la.h)
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e] = la_bits(__hmul2(la_pair(w[e >> 1][0]), la_pair(r[e])));
                    tc::tmem_st_16x128b_x4(dst, p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const __nv_bfloat162 rest = __hfma2(la_pair(w[e >> 1][0]), la_pair(r[e]), __hneg2(la_pair(p[e])));
                        p[e] = la_bits(__hfma2(la_pair(w[e >> 1][1]), la_pair(r[e]), rest));
                    }
                    tc::tmem_st_16x128b_x4(dst + 16, p);
                } else {
                    uint32_t p1[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        p[e] = tc::pack_bf16x2(__uint_as_float(w[e >> 1][0]) * low_half(r[e]), __uint_as_float(w[e >> 1][1]) * high_half(r[e]));
                    tc::tmem_st_16x128b_x4(dst, p);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x0 = fmaf(__uint_as_float(w[e >> 1][0]), low_half(r[e]), -low_half(p[e]));
                        const float x1 = fmaf(__uint_as_float(w[e >> 1][1]), high_half(r[e]), -high_half(p[e]));
                        p1[e] = tc::pack_bf16x2(x0, x1);
                        p[e] = tc::pack_bf16x2(x0 - low_half(p1[e]), x1 - high_half(p1[e]));
                    }
                    tc::tmem_st_16x128b_x4(dst + 16, p1);
                    tc::tmem_st_16x128b_x4(dst + 32, p);
                }
                tc::tmem_st_wait();
                tc::tc_fence_before();
                __syncwarp();
                if (t >= n_pre && qd == 3 && __any_sync(0xffffffffu, __hisnan(odd.x) || __hisnan(odd.y))) {
                    // what is not finite gives way to zeros, now that all of it has been read; PV comes behind KV
                    ((volatile int *)sm->odd_tile)[t % MARKS] = t + 1;
                    const int col = lg * 16 + (lane & 15);
#pragma unroll 1
                    for (int i = lane >> 4; i < LT; i += 2) {
                        unsigned short *e = reinterpret_cast<unsigned short *>(
                            smem + slab + s * VB + tc::sw128_offset(i, (q4 & 1) * 4 + (col >> 3))) + (col & 7);
                        if ((*e & 0x7f80) == 0x7f80) *e = 0;
                    }
                    tc::fence_proxy_async_smem();
                    __syncwarp();
                }
                if (lane == 0) tc::mbar_arrive(&sm->vw_full[buf]);
            }
            if (t < n_pre && lane == 0) tc::mbar_arrive(&sm->free_v[s]);
        }
    } else if (warp >= WARP_O) {
        // ------------------------------------------------------------------ o: half a row per thread, staged where V stood
        const int q4 = warp & 3, half = (warp - WARP_O) >> 2, r = q4 * 32 + lane;
        const uint32_t row = tmem + ((uint32_t)(q4 * 32) << 16), mine = row + TM_O + half * 64;
        for (int t = n_pre; t < ntiles; ++t) {
            const int f = t - n_pre, s = t % NV, n = tile_n(t), at = tile_at(t);
            const float w = r < n ? j.scale_c * sm->pow[rev ? n - 1 - r : r + 1] : 0.f;
            tc::mbar_wait(&sm->qs_done, f & 1, abort_flag, d_status);
            tc::tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {   // the carried part, for PV to add to
                uint32_t x[32];
                tc::tmem_ld32(mine + c, x);
                tc::tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(w * __uint_as_float(x[e]));
                tc::tmem_st32(mine + c, x);
            }
            tc::tmem_st_wait();
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sm->o_scaled);
            tc::mbar_wait(&sm->pv_done, f & 1, abort_flag, d_status);
            tc::tc_fence_after();
            const bool odd = ((volatile int *)sm->odd_tile)[t % MARKS] == t + 1;
            uint8_t *stage = smem + L::V + s * VB + half * SLAB;
#pragma unroll 1
            for (int c = 0; c < 64; c += 32) {
                uint32_t y[32];
                __syncwarp();
                tc::tmem_ld32(mine + c, y);
                tc::tmem_ld_wait();
                if (odd) {                       // what is not finite, for the rows that see it
                    const __nv_bfloat16 *v = (const __nv_bfloat16 *)j.v + ((int64_t)b * a.L + at) * j.ldv +
                                             (int64_t)(h / j.rv) * j.dv + half * 64 + c;
#pragma unroll 1
                    for (int jj = 0; jj < n; ++jj) {
                        uint32_t p[8], pw = 0;   // (the eight columns that hold token jj)
                        __syncwarp();
                        tc::tmem_ld8(row + TM_QK + (jj >> 6) * 64 + (jj >> 4 & 3) * 8, p);
                        tc::tmem_ld_wait();
#pragma unroll
                        for (int z = 0; z < 8; ++z) pw = z == (jj >> 1 & 7) ? p[z] : pw;
                        const float pf = __uint_as_float(jj & 1 ? pw & 0xffff0000u : pw << 16);
                        if (rev ? jj >= r : jj <= r) {
#pragma unroll
                            for (int g = 0; g < 32; g += 8) {
                                if (half * 64 + c + g >= j.dv) continue;
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
                if (c == 32) {                   // everything in tensor memory has been read
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&sm->o_free);
                }
                if (j.o_f32) {
                    if (r < n) {
                        uint4 *p = reinterpret_cast<uint4 *>((float *)j.o + ((int64_t)b * a.L + at + r) * j.ldo + (int64_t)h * j.dv + half * 64 + c);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (half * 64 + c + (4 * e & ~7) < j.dv) p[e] = make_uint4(y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e += 8)
                        *reinterpret_cast<uint4 *>(stage + tc::sw128_offset(r, (c + e) >> 3)) =
                            make_uint4(bits2(y[e], y[e + 1]), bits2(y[e + 2], y[e + 3]), bits2(y[e + 4], y[e + 5]), bits2(y[e + 6], y[e + 7]));
                }
            }
            if (j.o_f32) {
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&sm->free_v[s]);
                continue;
            }
            tc::fence_proxy_async_smem();
            tc::named_bar_sync(1 + half, 128);
            if (q4 == 0) {                       // (rows behind the sequence are clipped by the tensor map)
                if (tc::elect_one()) {
                    tc::tma_store_4d(&maps.o[ji], stage, half * 64, h, at, b);
                    tc::bulk_commit_group();
                    tc::bulk_wait_read_all();
                    tc::mbar_arrive_n(&sm->free_v[s], 4);
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
bool run_wide(LaunchCtx &ctx, const Maps &maps, const LaArgs &a)
{
    const size_t smem = Sm<DK>::SMALL + sizeof(Small);
    if (!ensure_dynamic_smem((const void *)la_wide_kernel<DK, STATE_ONLY>, smem)) return false;
    const int64_t items = (int64_t)a.njobs * a.B * a.H * (STATE_ONLY ? (a.nseg - 1) * a.per : a.nseg);
    const int64_t n = STATE_ONLY ? items : a.whole + (items - a.whole) * a.ncut;
    ctx.begin(STATE_ONLY ? STAGE_LA_STATES : STAGE_LA_TILES);
    launch_kernel(la_wide_kernel<DK, STATE_ONLY>, dim3((unsigned)n), dim3(THREADS), smem, ctx.stream, true, maps, a,
                  ctx.d_status);
    ctx.end();
    return cudaGetLastError() == cudaSuccess;
}

}  // namespace

double la_cuts(int64_t items, int nt, int sm_count, LaArgs *a)
{
    // Whole waves of walks first, what is left shared so that its CTAs end together: a tile that only carries the state takes
    // three quarters of the time of the others where the state is a result (w V in three parts), so each part is a quarter as
    // long as the one in front (4 sequences of 8192, 16 heads: 195 us; 0.21 as long 214, 0.17 209; whole walks 279, two
    // segments 210, four 259).
    constexpr double RATIO = 0.25;
    const int64_t whole = items / sm_count * sm_count, rest = items - whole;
    double best = (double)ceil_div64(items, sm_count) * nt;
    a->whole = (int)items;
    a->ncut = 1;
    if (rest == 0) return best;
    for (int m = 2; m <= 4 && m <= nt; ++m) {
        const double first = nt * (1.0 - RATIO) / (1.0 - pow(RATIO, m));
        const double cost = (double)(whole / sm_count) * nt + (double)ceil_div64(rest * m, sm_count) * (first + 1.0);
        if (cost >= best) continue;
        best = cost;
        a->whole = (int)whole;
        a->ncut = m;
        double at = 0;
        for (int c = 0; c < m; ++c) {
            a->cut[c] = std::max(c, (int)(at + 0.5));
            at += first * pow(RATIO, c);
        }
        a->cut[m] = nt;
        for (int c = m - 1; c > 0; --c) a->cut[c] = std::min(a->cut[c], a->cut[c + 1] - 1);
    }
    return best;
}

int launch_la_wide(LaunchCtx &ctx, const LaArgs &all, bool states, int sm_count)
{
    LaArgs a = all;
    const int64_t items = (int64_t)a.njobs * a.B * a.H * a.nseg;
    a.whole = (int)items;
    a.ncut = 1;
    if (a.nseg == 1) la_cuts(items, ceil_div(a.L, LT), sm_count, &a);
    Maps maps;
    for (int i = 0; i < a.njobs; ++i) {
        const LaJob &j = a.job[i];
        if (!la_stream_map(ctx.tmaps, &maps.q[i], j.q, j.dk, a.H / j.rq, a.L, a.B, j.ldq) ||
            !la_stream_map(ctx.tmaps, &maps.k[i], j.k, j.dk, a.H / j.rk, a.L, a.B, j.ldk) ||
            !la_stream_map(ctx.tmaps, &maps.v[i], j.v, j.dv, a.H / j.rv, a.L, a.B, j.ldv) ||
            (!states && !j.o_f32 && !la_stream_map(ctx.tmaps, &maps.o[i], j.o, j.dv, a.H, a.L, a.B, j.ldo)))
            return SWIMBA_ERR_CUDA;
    }
    const bool ok = a.job[0].dk <= 64 ? (states ? run_wide<64, true>(ctx, maps, a) : run_wide<64, false>(ctx, maps, a))
                                      : (states ? run_wide<128, true>(ctx, maps, a) : run_wide<128, false>(ctx, maps, a));
    return ok ? SWIMBA_OK : SWIMBA_ERR_CUDA;
}

}  // namespace swimba
