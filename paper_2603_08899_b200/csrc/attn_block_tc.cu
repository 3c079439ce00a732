// Tensor-core tree attention over a block-scaled E4M3 cache: tcgen05.mma kind::f16, f16 operands, fp32 accumulators in tensor memory.
//
// The mathematics is attn_block.cu's (the V scale in the exponent's argument); the structure that of the two-M-tile bf16 kernel (attn_tc.cu:
// one persistent CTA per SM, a key tile in two halves of 64 keys, S and O in tensor memory, P over S, stream-K split of the ragged batch, merge of
// split pairs).  What differs:
//   - K and V come through registers: four warps load the codes (16 bytes a thread and row piece, a tile of K and one of V under way at any
//     time), turn them into f16, exactly, and write them where the tensor pipe reads them.  With products in 8 bits (kind::f8f6f4) q and the weights
//     would have to be E4M3 too, 3 bits where bf16 has 7; as f16 they keep 11.  The codes travel in half the bytes of a bf16 cache all the same.
//     Rows past the last slot, and pages outside the pool, are written as zeros.
//   - the scales of a tile go with its K, through shared memory, as {ks, log2 vs, 1 / vs} of every 32 keys: a thread's row has one factor
//     and one addend of the exponent's argument per 32 keys;
//   - q is turned into f16 by the softmax threads, a row each, scaled by the power of two that brings the row's largest magnitude into [1, 2).
//
// For whole trees (rows x heads of a kv head > 32): the products bind, 256 FLOP per byte of a bf16 cache and twice that here.
#include "e4m3.cuh"
#include "tc_walk.cuh"

namespace confu {

namespace tc {
namespace blktc {

constexpr int kThreads = 512;            // warps 0-3: softmax of M tile 0, 4-7: of M tile 1, 8-11: codes to f16, 12: MMA
template <int D> constexpr int kTile = kTileKeys * D * 2;             // a 128-key tile as f16
template <int D> constexpr int kStages = D == 128 ? 2 : 4;            // stage g = [V of the CTA's g-1st key tile | K of its g-th]
constexpr uint32_t kTmemCols = 512;                 // S0 | S1 | O0 | O1, 128 columns each; P_t overlays S_t
constexpr float kRescaleThreshold = 8.f;            // weights stay <= 2^8
constexpr float kLeastScale = 7.8886091e-31f;       // 2^-100
// Scales of a tile are read by the softmax threads until they have handed over its weights.  Tile g + 5 (g + 3 with two stages) is not
// converted before P V of tile g: a ring of eight is enough.
constexpr int kScaleRing = 8;
// f16 x f16 -> fp32 (formats 0), M = 128: N = 64 keys, B K-major; N = D, B MN-major
constexpr uint32_t kIdescS = (1u << 4) | ((64u >> 3) << 17) | ((128u >> 4) << 24);
template <int D> constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((128u >> 4) << 24);

struct BlockParams {
    const uint8_t *k, *v, *k_soft, *v_soft;
    const float *ks, *vs, *ks_soft, *vs_soft;
    const __nv_bfloat16* q;
    int64_t n_pages;
    int block;
};

template <int D>
struct SharedStorage {
    alignas(1024) uint8_t q[2 * kTile<D>];               // two M tiles
    alignas(1024) uint8_t kv[kStages<D>][2][kTile<D>];   // [stage][0: V tile, 1: K tile]
    alignas(16) float4 scales[kScaleRing][4];            // per 32 keys: ks, log2 vs, 1 / vs
    alignas(8) uint64_t q_full[2];
    uint64_t kv_full[kStages<D>], kv_empty[kStages<D>];
    uint64_t scales_full[kScaleRing];
    uint64_t s_full[2][2], p_full[2][2], o_done[2];      // [M tile][half of the key tile]
    uint64_t pv0_done[2];                 // P V of half 0 of a run's last tile has completed
    uint32_t tmem_base;
    int abort;
    alignas(16) float4 xpose[8][32 * 8];                 // per softmax warp: a 32 x 32 fp32 tile, as in attn_tc.cu
};

// ------------------------------------------------------------------------------------ roles
struct TileRef {
    int64_t row;                       // first slot in the pool (soft prompts: 0)
    int g, valid;                      // kv head; keys of the tile that exist
    int page;                          // -1: the soft prompts, -2: outside the pool
};

// The CTA's key tiles in walking order.
struct TileWalk {
    Walker w;
    Segment s;
    int t;
    bool run;
    __device__ void begin(const PlanView& pv, const Params& prm)
    {
        run = w.begin(pv, prm, blockIdx.x, kPlanCta, s);
        t = s.t0;
    }
    __device__ bool next(const Params& prm, const BlockParams& bp, TileRef& r)
    {
        if (!run) return false;
        r.g = s.g;
        if (t >= s.nkt) {
            r.page = -1;
            r.row = 0;
            r.valid = prm.d.S;
        } else {
            const int page = __ldg(prm.map.block_table + (size_t)s.b * prm.map.max_pages + t);
            const int64_t left = s.P + prm.d.T + prm.d.C - (int64_t)t * kTileKeys;
            r.valid = (int)min(left, (int64_t)kTileKeys);
            r.page = (uint32_t)page < (uint64_t)bp.n_pages ? page : -2;
            r.row = (int64_t)page * kTileKeys;
        }
        if (++t == s.t1) {
            run = w.next(s);
            t = s.t0;
        }
        return true;
    }
};

// 16 bytes of a row: thread t has piece t % (D / 16) of rows t / (D / 16), + 2048 / D, ...
template <int D>
struct Codes {
    static constexpr int kPieces = D / 16, kRows = 128 / kPieces, n = kTileKeys / kRows;
    uint4 w[n];
    __device__ __forceinline__ void load(const uint8_t* pool, const TileRef& r, int Hkv, int tid)
    {
        const size_t pitch = (size_t)Hkv * D;
        const uint8_t* p = pool + ((size_t)r.row * Hkv + r.g) * D + (tid / kPieces) * pitch + (tid % kPieces) * 16;
        const int valid = r.page == -2 ? 0 : r.valid - tid / kPieces;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            w[i] = make_uint4(0u, 0u, 0u, 0u);
            if (i * kRows < valid)
                asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                             : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w)
                             : "l"(p + (size_t)i * kRows * pitch));
        }
    }
    // into [D / 64 halves][128 rows][128 B], 128-byte swizzle.  Lanes of the second half write their two pieces the other way round: eight lanes
    // then meet eight different groups of banks.
    __device__ __forceinline__ void store(uint8_t* tile, int tid) const
    {
        const int piece = tid % kPieces, half = piece >> 2, c0 = 2 * (piece & 3), first = half;
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int row = tid / kPieces + i * kRows;
            uint4 lo, hi;
            e4m3_to_f16x4(w[i].x, lo.x, lo.y);
            e4m3_to_f16x4(w[i].y, lo.z, lo.w);
            e4m3_to_f16x4(w[i].z, hi.x, hi.y);
            e4m3_to_f16x4(w[i].w, hi.z, hi.w);
            uint8_t* to = tile + half * kHalfTile + row * 128;
            const uint4 a = first ? hi : lo, b = first ? lo : hi;
            *reinterpret_cast<uint4*>(to + (((c0 + first) ^ (row & 7)) << 4)) = a;
            *reinterpret_cast<uint4*>(to + (((c0 + 1 - first) ^ (row & 7)) << 4)) = b;
        }
    }
};

template <int D>
__device__ void convert_role(SharedStorage<D>& sh, const Params& prm, const BlockParams& bp, const PlanView& pv)
{
    const int tid = threadIdx.x & 127, Hkv = prm.d.Hkv, nb = kTileKeys / bp.block;
    TileWalk walk;
    walk.begin(pv, prm);
    TileRef cur, next;                               // tiles g and g + 1 of the walk
    if (!walk.next(prm, bp, cur)) return;
    bool have_next = walk.next(prm, bp, next);
    Codes<D> k, v;
    float ks = 1.f, vs = 1.f;                        // threads 0-3: of 32 keys of the tile whose K is under way
    auto load_k = [&](const TileRef& r) {
        k.load(r.page == -1 ? bp.k_soft : bp.k, r, Hkv, tid);
        ks = vs = 1.f;
        if (tid < 4 && tid * 32 < r.valid && r.page != -2) {
            const size_t at = ((size_t)(r.page == -1 ? 0 : r.page) * Hkv + r.g) * nb + tid * 32 / bp.block;
            ks = __ldg((r.page == -1 ? bp.ks_soft : bp.ks) + at);
            vs = __ldg((r.page == -1 ? bp.vs_soft : bp.vs) + at);
        }
    };
    auto load_v = [&](const TileRef& r) { v.load(r.page == -1 ? bp.v_soft : bp.v, r, Hkv, tid); };
    load_k(cur);
    load_v(cur);
    bool have_cur = true;
    for (uint32_t g = 0;; ++g) {                     // stage g: V of tile g - 1, K of tile g
        const uint32_t st = g % kStages<D>;
        if (!mbar_wait(&sh.kv_empty[st], ((g / kStages<D>) & 1) ^ 1, &sh.abort, prm.wait_ns)) return;
        if (g > 0) {
            v.store(sh.kv[st][0], tid);
            if (have_cur) load_v(cur);
        }
        if (have_cur) {
            k.store(sh.kv[st][1], tid);
            if (tid < 4) {
                const float least = fmaxf(vs, kLeastScale);
                sh.scales[g % kScaleRing][tid] = make_float4(ks, log2f(least), 1.f / least, 0.f);
                mbar_arrive(&sh.scales_full[g % kScaleRing]);
            }
            if (have_next) load_k(next);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(&sh.kv_full[st]);
        if (!have_cur) return;
        cur = next;
        have_cur = have_next;
        if (have_next) have_next = walk.next(prm, bp, next);
    }
}

// One warp drives the tensor pipe, one lane of it issues: as in attn_tc.cu, without the wait for repaired rows.
template <int D, bool kTwo>
__device__ void mma_role(SharedStorage<D>& sh, const Params& prm, const PlanView& pv, uint32_t tmem)
{
    constexpr int kMt = kTwo ? 2 : 1;
    Walker w;
    Segment s;
    uint32_t stage = 0, seg = 0;
    const bool issuer = elect_lane();
    const uint32_t q_lo = desc_lo(smem_u32(sh.q), 16);
    const uint32_t v_lo0 = desc_lo(smem_u32(sh.kv[0][0]), kHalfTile), k_lo0 = desc_lo(smem_u32(sh.kv[0][1]), 16);
    constexpr uint32_t kTileStep = kTile<D> >> 4, kStageStep = 2 * kTileStep;

    // half h of S_t = Q_t K_h^T: D / 16 steps of 16 head dims; step i sits in 64-column half i/4 at byte 32*(i%4) of the swizzled row
    auto issue_qk = [&](int t, int h, uint32_t kl) {
        if (!issuer) return;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            const uint32_t off = ((uint32_t)(i >> 2) * kHalfTile + (uint32_t)(i & 3) * 32u) >> 4;
            mma_ss(tmem + t * 128 + h * 64, q_lo + t * kTileStep + off, kl + h * (8192u >> 4) + off, kIdescS, i > 0 ? 1u : 0u);
        }
        tc_commit(&sh.s_full[t][h]);
    };
    // O_t += P_t V over half h: 4 steps of 16 keys (2048 B of the V tile and 8 columns of f16 pairs each)
    auto issue_pv = [&](int t, int h, uint32_t vl, bool first_of_run) {
        if (!issuer) return;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            mma_ts(tmem + 256 + t * 128, tmem + t * 128 + h * 64 + i * 8, vl + (4 * h + i) * (2048u >> 4), kIdescO<D>,
                   (first_of_run && h == 0 && i == 0) ? 0u : 1u);
    };
    bool have_prev = false, prev_first = false, prev_last = false;
    auto run_stage = [&](bool have_cur, bool cur_first, bool cur_last) -> bool {
        const uint32_t st = stage % kStages<D>;
        if (!mbar_wait(&sh.kv_full[st], (stage / kStages<D>) & 1, &sh.abort, prm.wait_ns)) return false;
        tc_fence_after();
        const uint32_t vl = v_lo0 + st * kStageStep, kl = k_lo0 + st * kStageStep;
        if (have_prev) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int t = 0; t < kMt; ++t) {
                    // (At the start of a run this P V overwrites the run before's O_t; the softmax threads hand P over only
                    // after they have read that O_t out.)
                    if (!mbar_wait(&sh.p_full[t][h], (stage - 1) & 1, &sh.abort, prm.wait_ns)) return false;
                    tc_fence_after();
                    issue_pv(t, h, vl, prev_first);
                    // before half 1 of a tile rescales O it waits for the P V of half 0: for the Q K^T behind it, or, at the end of
                    // a run, for a barrier of its own
                    if (prev_last) {
                        if (issuer) tc_commit(h == 0 ? &sh.pv0_done[t] : &sh.o_done[t]);
                    } else
                        issue_qk(t, h, kl);
                }
            }
        }
        if (have_cur && cur_first) {
#pragma unroll
            for (int t = 0; t < kMt; ++t) {
                if (!mbar_wait(&sh.q_full[t], seg & 1, &sh.abort, prm.wait_ns)) return false;
                tc_fence_after();
                issue_qk(t, 0, kl);
                issue_qk(t, 1, kl);
            }
        }
        if (issuer) tc_commit(&sh.kv_empty[st]);
        ++stage;
        have_prev = have_cur;
        prev_first = cur_first;
        prev_last = cur_last;
        return true;
    };
    for (bool run = w.begin(pv, prm, blockIdx.x, kPlanCta, s); run; run = w.next(s)) {
        const int n_tiles = s.t1 - s.t0;
        for (int j = 0; j < n_tiles; ++j)
            if (!run_stage(true, j == 0, j + 1 == n_tiles)) return;
        ++seg;
    }
    if (have_prev) run_stage(false, false, false);
}

__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// A row of q -> f16 in the M tile that the tensor pipe reads, divided by 2^e with 2^e <= largest magnitude < 2^(e + 1); returns 2^e.
template <int D>
__device__ __forceinline__ float put_q_row(const __nv_bfloat16* q, bool there, uint8_t* tile, int row)
{
    uint4 raw[D / 8];
    float amax = 0.f;
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
        raw[j] = there ? __ldg(reinterpret_cast<const uint4*>(q) + j) : make_uint4(0u, 0u, 0u, 0u);
        const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            amax = fmaxf(amax, fabsf(__uint_as_float(w[k] << 16)));
            amax = fmaxf(amax, fabsf(__uint_as_float(w[k] & 0xffff0000u)));
        }
    }
    const int e = min(max((int)(__float_as_uint(amax) >> 23) - 127, -125), 125);
    const float down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
    for (int j = 0; j < D / 8; ++j) {
        const uint32_t w[4] = {raw[j].x, raw[j].y, raw[j].z, raw[j].w};
        uint32_t o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = pack_f16(__uint_as_float(w[k] << 16) * down, __uint_as_float(w[k] & 0xffff0000u) * down);
        *reinterpret_cast<uint4*>(tile + (j >> 3) * kHalfTile + row * 128 + (((j & 7) ^ (row & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
    }
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// max of 32 floats held as raw bits, as four chains of three-input max
__device__ __forceinline__ float max32(const uint32_t* sv)
{
    float a[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        a[k] = fmaxf(__uint_as_float(sv[8 * k]), __uint_as_float(sv[8 * k + 1]));
#pragma unroll
        for (int j = 2; j < 8; j += 2)
            asm("max.f32 %0, %0, %1, %2;" : "+f"(a[k]) : "f"(__uint_as_float(sv[8 * k + j])), "f"(__uint_as_float(sv[8 * k + j + 1])));
    }
    return fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
}

// exp2(s * a + add) of 32 scores -> 16 packed f16 pairs; returns their fp32 sum
__device__ __forceinline__ float weights32(const uint32_t* sv, float a, float add, uint32_t* pk)
{
    uint64_t sum2 = f2_pack(0.f, 0.f);
    const uint64_t a2 = f2_pack(a, a), add2 = f2_pack(add, add);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        float x0, x1;
        f2_unpack(f2_fma(f2_pack(__uint_as_float(sv[2 * j]), __uint_as_float(sv[2 * j + 1])), a2, add2), x0, x1);
        x0 = ex2(x0);
        x1 = ex2(x1);
        sum2 = f2_add(sum2, f2_pack(x0, x1));
        pk[j] = pack_f16(x0, x1);
    }
    float s0, s1;
    f2_unpack(sum2, s0, s1);
    return s0 + s1;
}

template <int D>
__device__ void softmax_role(SharedStorage<D>& sh, const Params& prm, const BlockParams& bp, const PlanView& pv, uint32_t tmem, int t /*M tile*/)
{
    const int lane_row = threadIdx.x & 127;                 // row of the M tile = TMEM lane
    const int warp_in_wg = (threadIdx.x >> 5) & 3;
    const uint32_t lane_base = (uint32_t)(warp_in_wg * 32) << 16;
    const uint32_t s_addr = tmem + lane_base + t * 128;
    const uint32_t o_addr = tmem + lane_base + 256 + t * 128;
    const int G = prm.G, T = prm.d.T, R = prm.d.T + prm.d.C, S = prm.d.S, Hq = prm.d.Hq;
    const int hl = lane_row % G;

    Walker w;
    Segment s;
    uint32_t seg = 0, g = 0;                                // runs, tiles: s_full[t][half] completes once a tile
    for (bool run = w.begin(pv, prm, blockIdx.x, kPlanCta, s); run; run = w.next(s)) {
        const int r = prm.rpt * (2 * s.rg + t) + lane_row / G;            // query row of this thread in this pair
        const bool row_valid = lane_row < prm.rpt * G && r < R;
        const uint64_t mask = row_valid ? pv.mask[(size_t)s.b * kMaxRows + r] : 0ull;
        // (every Q K^T of the run before has completed: this thread has seen its last scores)
        const float q_scale = put_q_row<D>(bp.q + (((size_t)s.b * R + (row_valid ? r : 0)) * Hq + s.g * G + hl) * D, row_valid, sh.q + t * kTile<D>, lane_row);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(&sh.q_full[t]);
        const float c = prm.c * q_scale;
        float m_ref = -INFINITY, l = 0.f;
        for (int tile = s.t0; tile < s.t1; ++tile, ++g) {
            if (!mbar_wait(&sh.scales_full[g % kScaleRing], (g / kScaleRing) & 1, &sh.abort, prm.wait_ns)) return;
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                uint32_t sv[64];
                if (!mbar_wait(&sh.s_full[t][h], g & 1, &sh.abort, prm.wait_ns)) return;
                tc_fence_after();
                tmem_ld32(s_addr + h * 64, *reinterpret_cast<uint32_t(*)[32]>(&sv[0]));
                tmem_ld32(s_addr + h * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&sv[32]));
                tc_wait_ld();
                if (tile >= s.masked) {
                    uint64_t lo, hi;
                    visible_bits(s, tile, R, T, S, r, row_valid, mask, lo, hi);
                    const uint64_t vis = h ? hi : lo;
#pragma unroll
                    for (int j = 0; j < 64; ++j)
                        if (!((vis >> j) & 1ull)) sv[j] = 0xff800000u;           // -inf
                }
                const float4 sc0 = sh.scales[g % kScaleRing][2 * h], sc1 = sh.scales[g % kScaleRing][2 * h + 1];
                // (a factor of 0 would turn the -infinity of masked keys into NaN)
                const float a0 = fmaxf(c * sc0.x, 1.1754944e-38f), a1 = fmaxf(c * sc1.x, 1.1754944e-38f);
                // the reference maximum follows the running maximum; O is brought along when it moves.  P V of the half before
                // has completed when the other half's next completion of s_full is there, or, in half 1 of the run's last
                // tile, that of pv0_done (see the issuing warp).
                const float m_new = fmaxf(m_ref, fmaxf(fmaf(max32(sv), a0, sc0.y), fmaf(max32(sv + 32), a1, sc1.y)));
                if (tile == s.t0 && h == 0) {
                    m_ref = m_new;
                } else {
                    const bool move = m_new - m_ref > kRescaleThreshold;         // false when both are -inf (NaN)
                    if (__any_sync(0xffffffffu, move)) {
                        const bool last = h == 1 && tile + 1 == s.t1;
                        if (!mbar_wait(last ? &sh.pv0_done[t] : &sh.s_full[t][h ^ 1], (last ? seg : g + h) & 1, &sh.abort, prm.wait_ns)) return;
                        tc_fence_after();
                        const float alpha = move ? ex2(m_ref - m_new) : 1.f;
                        if (move) { m_ref = m_new; l *= alpha; }
#pragma unroll 1
                        for (int q4 = 0; q4 < D / 16; ++q4) {
                            uint32_t ov[16];
                            tmem_ld16(o_addr + q4 * 16, ov);
                            tc_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) ov[j] = __float_as_uint(__uint_as_float(ov[j]) * alpha);
                            tmem_st16(o_addr + q4 * 16, ov);
                        }
                    }
                }
                // P over the columns of the half (whose scores sit in registers by now); masked scores get weight exactly 0
                const float neg_m = (m_ref == -INFINITY) ? 0.f : -m_ref;
                uint32_t pk[32];
                l = fmaf(weights32(sv, a0, sc0.y + neg_m, pk), sc0.z, l);
                l = fmaf(weights32(sv + 32, a1, sc1.y + neg_m, pk + 16), sc1.z, l);
                tmem_st32(s_addr + h * 64, pk);
                tc_wait_st();
                tc_fence_before();
                mbar_arrive(&sh.p_full[t][h]);
            }
        }
        // ---- epilogue of this pair / range: as in attn_tc.cu ----
        if (!mbar_wait(&sh.o_done[t], seg & 1, &sh.abort, prm.wait_ns)) return;
        tc_fence_after();
        const int h = s.g * G + hl;
        const int lane = threadIdx.x & 31;
        float4* xp = sh.xpose[threadIdx.x >> 5];
        const bool whole = s.part_slot < 0;
        const float inv_l = whole ? 1.f / l : 1.f;
        __nv_bfloat16* o_ptr[4];
        float* p_ptr = nullptr;
        if (whole) {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                const int lr = warp_in_wg * 32 + 8 * kk + (lane >> 2);
                const int rk = prm.rpt * (2 * s.rg + t) + lr / G;
                o_ptr[kk] = (lr < prm.rpt * G && rk < R)
                                ? prm.out + (((size_t)s.b * R + rk) * Hq + s.g * G + lr % G) * D + 8 * (lane & 3)
                                : nullptr;
            }
        } else {
            p_ptr = prm.partials + (size_t)s.part_slot * (partial_slot_bytes() / sizeof(float)) +
                    (size_t)(t * 128 + warp_in_wg * 32 + (lane >> 3)) * kPartD + 4 * (lane & 7);
        }
#pragma unroll 1
        for (int q4 = 0; q4 < D / 32; ++q4) {
            uint32_t ov[32];
            tmem_ld32(o_addr + q4 * 32, ov);
            tc_wait_ld();
#pragma unroll
            for (int q = 0; q < 8; ++q)
                xp[lane * 8 + (q ^ (lane & 7))] =
                    make_float4(__uint_as_float(ov[4 * q]) * inv_l, __uint_as_float(ov[4 * q + 1]) * inv_l,
                                __uint_as_float(ov[4 * q + 2]) * inv_l, __uint_as_float(ov[4 * q + 3]) * inv_l);
            __syncwarp();
            if (whole) {
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) {
                    const int k = 8 * kk + (lane >> 2), q = 2 * (lane & 3);
                    const float4 a = xp[k * 8 + (q ^ (k & 7))], b2 = xp[k * 8 + ((q + 1) ^ (k & 7))];
                    if (o_ptr[kk])
                        *reinterpret_cast<uint4*>(o_ptr[kk] + q4 * 32) =
                            make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b2.x, b2.y), pack_bf16(b2.z, b2.w));
                }
            } else {
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const int k = 4 * kk + (lane >> 3);
                    *reinterpret_cast<float4*>(p_ptr + (size_t)(4 * kk) * kPartD + q4 * 32) = xp[k * 8 + ((lane & 7) ^ (k & 7))];
                }
            }
            __syncwarp();
        }
        if (whole) {
            if (row_valid && prm.lse) prm.lse[((size_t)s.b * R + r) * Hq + h] = natural_lse(m_ref, l);
        } else {
            float* ml = prm.partials + (size_t)s.part_slot * (partial_slot_bytes() / sizeof(float)) + (size_t)kPartRows * kPartD;
            ml[t * 128 + lane_row] = m_ref;
            ml[kPartRows + t * 128 + lane_row] = l;
        }
        // the P of the next run's first tile is only handed over after this point, which is what keeps the tensor pipe from overwriting
        // O_t before it has been read
        tc_fence_before();
        ++seg;
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) attention_block_tc_kernel(const Params prm, const BlockParams bp)
{
    extern __shared__ uint8_t smem_raw[];
    SharedStorage<D>& sh = *reinterpret_cast<SharedStorage<D>*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = threadIdx.x >> 5;

    if (threadIdx.x == 0) {
        // a stage is full when every converting thread has written its pieces, free again when its MMAs have completed
        for (int i = 0; i < kStages<D>; ++i) { mbar_init(&sh.kv_full[i], 128); mbar_init(&sh.kv_empty[i], 1); }
        for (int i = 0; i < kScaleRing; ++i) mbar_init(&sh.scales_full[i], 4);
        for (int t = 0; t < 2; ++t) {
            mbar_init(&sh.q_full[t], 128);
            for (int h = 0; h < 2; ++h) {
                mbar_init(&sh.s_full[t][h], 1);
                mbar_init(&sh.p_full[t][h], 128);
            }
            mbar_init(&sh.o_done[t], 1);
            mbar_init(&sh.pv0_done[t], 1);
        }
        sh.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem_base)),
                     "r"(kTmemCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    const PlanView pv = plan_view(const_cast<void*>(prm.plan), prm.d.B, prm.d.Hkv);
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // 512 threads x 128 registers = 256 x 176 + 128 x 104 + 128 x 56
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 176;");
        const int t = warp >> 2;
        if (t < prm.n_mt) softmax_role<D>(sh, prm, bp, pv, tmem, t);
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        convert_role<D>(sh, prm, bp, pv);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 12) {
            if (prm.n_mt > 1) mma_role<D, true>(sh, prm, pv, tmem);
            else mma_role<D, false>(sh, prm, pv, tmem);
        }
        __syncwarp();
    }
    // ---- teardown ----
    tc_fence_before();
    __syncthreads();
    if (sh.abort) {
        if (threadIdx.x == 0 && prm.status)
            for (int b = 0; b < prm.d.B; ++b) prm.status[b] = CONFU_ST_TIMEOUT;
        __syncthreads();
    }
    if (warp == 12) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

template <int D>
cudaError_t launch(const Params& prm, const BlockParams& bp, int units, cudaStream_t st)
{
    const size_t smem = sizeof(SharedStorage<D>) + 1024;
    static OncePerDevice attr_done;
    cudaError_t e = attr_done.run([&] { return cudaFuncSetAttribute(attention_block_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem); });
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute pdl[1];
    pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    pdl[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)units);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = pdl;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attention_block_tc_kernel<D>, prm, bp);
}

}  // namespace blktc
}  // namespace tc

cudaError_t launch_attention_block_tc(const Ctx* ctx, const confu_dims& d, const void* q, const void* k_cache, const void* v_cache,
                                      int64_t n_slots, const SlotMap& map, const int32_t* prefix_len, const void* k_soft, const void* v_soft,
                                      const void* plan, void* partials, void* out, float* lse, int32_t* status, cudaStream_t st)
{
    using namespace tc;
    Params prm;
    prm.d = d;
    prm.map = map;
    prm.prefix_len = prefix_len;
    prm.plan = plan;
    prm.prefetch = 0;
    prm.partials = (float*)partials;
    prm.out = (__nv_bfloat16*)out;
    prm.lse = lse;
    prm.status = status;
    set_rows(prm, d, kPlanCta);
    prm.c = (d.sm_scale != 0.f ? d.sm_scale : 1.f / sqrtf((float)d.D)) * 1.4426950408889634f;
    prm.wait_ns = ctx->wait_ns;
    prm.k_scale = prm.v_scale = nullptr;
    blktc::BlockParams bp;
    bp.k = (const uint8_t*)k_cache;
    bp.v = (const uint8_t*)v_cache;
    bp.k_soft = (const uint8_t*)k_soft;
    bp.v_soft = (const uint8_t*)v_soft;
    bp.ks = ctx->k_block_scale;
    bp.vs = ctx->v_block_scale;
    bp.ks_soft = ctx->k_soft_scale;
    bp.vs_soft = ctx->v_soft_scale;
    bp.q = (const __nv_bfloat16*)q;
    bp.n_pages = n_slots / kTileKeys;
    bp.block = ctx->block;
    const cudaError_t e = d.D == 64 ? blktc::launch<64>(prm, bp, ctx->sm_count, st) : blktc::launch<128>(prm, bp, ctx->sm_count, st);
    if (e != cudaSuccess) return e;
    return launch_combine(prm, ctx->sm_count, st);
}

}  // namespace confu
