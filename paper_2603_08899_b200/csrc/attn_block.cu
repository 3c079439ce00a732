// Tree attention over a block-scaled E4M3 cache, keys and values kept in registers (mma.sync, f16 operands, fp32 sums).
//
// An entry stands for code * scale, one scale per block of 32, 64 or 128 slots and kv head, for K (ks) and V (vs) each.  With
//     s' = c ks (q . k_code) + log2 vs,   m' = max s',   p' = 2^(s' - m')
//     O = sum p' v_code,   l = sum p' / vs,   out = O / l
// the V scale is part of the exponent's argument (it costs nothing per key), and weights are largest where weight times V scale is: what
// rounding them to f16 loses is 2^-11 of the largest contribution.  lse = ln 2 (m' + log2 l) is the softmax's own.  Every E4M3 code is
// an f16 number, and q, times the power of two that brings a row's largest magnitude into [1, 2), is one but for what is smaller than
// 2^-17 of it: nothing else is rounded.
//
// For few query rows (decoding, short chains) the kernel is bound by reading the cache, 2 D bytes a key, and what counts is
// how many bytes are on their way.  So there is no shared-memory stage: a warp takes 32 keys at a time and loads K and V straight into the
// registers that the products read, the next 32 keys' K as soon as this one's is used up, V likewise: 8 KB a warp under way at D = 128.
//   S = Q K^T    a lane's fragment of K^T is 16 contiguous bytes of a key (the head dims of a product's 16 steps are whatever
//                bytes the lane has; Q's fragments are laid out in shared memory to match)
//   O += P V     keys in pairs: a lane has the same 16 columns of two neighbouring keys, byte permutes pair them up
// Warps of a CTA that work on the same rows take different keys and meet at the end of a run in shared memory.  The plan, its shares and
// the merge of split pairs are those of the two-M-tile kernel (attn_tc.cu).
//
// Keys past the sequence's last slot are masked and their V bytes read as 0; page ids outside the pool are not followed and read as zeros.
#include "e4m3.cuh"
#include "tc_walk.cuh"

namespace confu {
namespace tc {
namespace blk {

constexpr int kChunk = 32;                           // keys a warp works on at a time
constexpr float kRescaleThreshold = 8.f;             // the reference maximum follows past 2^8: weights stay far below f16's 65504
constexpr float kLeastScale = 7.8886091e-31f;        // 2^-100: no block has less

struct BlockParams {
    const uint8_t *k, *v, *k_soft, *v_soft;
    const float *ks, *vs, *ks_soft, *vs_soft;
    const __nv_bfloat16* q;
    int64_t n_pages;
    int block;
    int wr;                                          // groups of warps that share rows: each has kMt M tiles of 16 rows
};

// kMt M tiles of 16 rows a warp, kWarps warps
template <int D, int kMt, int kWarps>
struct Shape {
    static constexpr int kThreads = kWarps * 32;
    // a row of partial sums: a lane's 32 (16) columns apart by 4 floats, rows by 16 banks, so that a warp's 16-byte stores meet no bank twice
    static constexpr int kSeg = D / 4 + 4, kPitch = 4 * kSeg;
    static constexpr int kQBytes = kMt * (D / 16) * 32 * 16;              // of a row group
    static constexpr int kOBytes = kWarps * kMt * 16 * kPitch * 4;
    static constexpr int kStatBytes = kWarps * kMt * 16 * 8;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint4& a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint4 ldg16(const uint8_t* p)
{
    uint4 v;
    asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ uint2 ldg8(const uint8_t* p)
{
    uint2 v;
    asm volatile("ld.global.nc.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "l"(p));
    return v;
}

// K of a chunk: lane (n = lane / 4, x = lane % 4) has, of keys n, n + 8, n + 16, n + 24, the bytes 16 x .. 16 x + 15 and, at D = 128, those 64 further on
template <int D>
struct KRegs {
    uint4 w[4][D / 64];
    __device__ __forceinline__ void load(const uint8_t* p, size_t pitch, int lane)
    {
        p += (lane >> 2) * pitch + (lane & 3) * 16;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int h = 0; h < D / 64; ++h) w[t][h] = ldg16(p + 8 * t * pitch + 64 * h);
    }
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int h = 0; h < D / 64; ++h) w[t][h] = make_uint4(0u, 0u, 0u, 0u);
    }
    // four bytes of key tile t for the product's step j
    __device__ __forceinline__ uint32_t word(int t, int j) const
    {
        const uint4& v = w[t][j / 4];
        return j % 4 == 0 ? v.x : j % 4 == 1 ? v.y : j % 4 == 2 ? v.z : v.w;
    }
};

// V of a chunk: the lane has, of keys 8 t + 2 x and 8 t + 2 x + 1, the D / 8 bytes from n * D / 8 on
template <int D>
struct VRegs {
    uint32_t w[4][2][D / 32];
    __device__ __forceinline__ void load(const uint8_t* p, size_t pitch, int lane)
    {
        p += 2 * (lane & 3) * pitch + (lane >> 2) * (D / 8);
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const uint8_t* at = p + (8 * t + o) * pitch;
                if constexpr (D == 128) {
                    const uint4 v = ldg16(at);
                    w[t][o][0] = v.x; w[t][o][1] = v.y; w[t][o][2] = v.z; w[t][o][3] = v.w;
                } else {
                    const uint2 v = ldg8(at);
                    w[t][o][0] = v.x; w[t][o][1] = v.y;
                }
            }
    }
    // keys from `valid` on read as 0
    __device__ __forceinline__ void cut(int valid, int lane)
    {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int o = 0; o < 2; ++o)
                if (8 * t + 2 * (lane & 3) + o >= valid)
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) w[t][o][i] = 0u;
    }
};

// Where a chunk's keys are, and their scales.
struct Chunk {
    const uint8_t *k, *v;
    float ks, vs;
    int tile, sub;                                   // key tile, which 32 keys of it
    int valid;                                       // keys of it that exist (0: nothing to do)
    bool inside;                                     // its page lies in the pool
};

template <int D, int kMt, int kWarps>
__global__ void __launch_bounds__(kWarps * 32, 1) attention_block_kernel(const Params prm, const BlockParams bp)
{
    using Sh = Shape<D, kMt, kWarps>;
    extern __shared__ __align__(16) uint8_t smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int G = prm.G, T = prm.d.T, R = prm.d.T + prm.d.C, S = prm.d.S, Hq = prm.d.Hq, Hkv = prm.d.Hkv;
    const int wr = bp.wr, wk = kWarps / wr, row_group = warp % wr, key_group = warp / wr;
    uint4* q_frag = reinterpret_cast<uint4*>(smem);                                              // [M tile][step][lane]
    float* o_part = reinterpret_cast<float*>(smem + wr * Sh::kQBytes);                            // [warp][row][pitch]
    float2* stat = reinterpret_cast<float2*>(smem + wr * Sh::kQBytes + Sh::kOBytes);              // [warp][row]: m, l
    const PlanView pv = plan_view(const_cast<void*>(prm.plan), prm.d.B, Hkv);
    const size_t pitch = (size_t)Hkv * D;
    const int nb = kTileKeys / bp.block;
    asm volatile("griddepcontrol.wait;" ::: "memory");

    Walker w;
    Segment s;
    for (bool run = w.begin(pv, prm, blockIdx.x, kPlanCta, s); run; run = w.next(s)) {
        // ---- Q: rows of this group, head by head; row m of it is query row r0 + m / G, head m % G of the kv head's ----
        const int r0 = prm.rpt * prm.tpg * s.rg, n_rows = min(R - r0, prm.rpt * prm.tpg) * G;
        float q_scale[kMt][2];                       // of the lane's rows n and n + 8 of an M tile
        int row_r[kMt][2];                           // their query rows, -1: none
        uint64_t mask[kMt][2];
#pragma unroll
        for (int mt = 0; mt < kMt; ++mt) {
            uint32_t raw[2][D / 16][2];              // the lane's bf16 of both rows: steps of four
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                const int m = (row_group * kMt + mt) * 16 + (lane >> 2) + 8 * o;
                const bool there = m < n_rows;
                const int r = there ? r0 + m / G : 0;
                row_r[mt][o] = there ? r : -1;
                mask[mt][o] = there ? pv.mask[(size_t)s.b * kMaxRows + r] : 0ull;
                const __nv_bfloat16* q = bp.q + (((size_t)s.b * R + r) * Hq + s.g * G + (there ? m % G : 0)) * D;
                float amax = 0.f;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) {
                    const uint2 x = there ? __ldg(reinterpret_cast<const uint2*>(q + (j / 4) * 64 + (lane & 3) * 16 + (j % 4) * 4)) : make_uint2(0u, 0u);
                    raw[o][j][0] = x.x;
                    raw[o][j][1] = x.y;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        amax = fmaxf(amax, fabsf(__uint_as_float(raw[o][j][i] << 16)));
                        amax = fmaxf(amax, fabsf(__uint_as_float(raw[o][j][i] & 0xffff0000u)));
                    }
                }
                amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
                amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
                // 2^e <= amax < 2^(e + 1); both it and its reciprocal are normal numbers
                const int e = min(max((int)(__float_as_uint(amax) >> 23) - 127, -125), 125);
                q_scale[mt][o] = __uint_as_float((uint32_t)(e + 127) << 23);
                const float down = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        raw[o][j][i] = pack_f16(__uint_as_float(raw[o][j][i] << 16) * down, __uint_as_float(raw[o][j][i] & 0xffff0000u) * down);
            }
            if (key_group == 0)
#pragma unroll
                for (int j = 0; j < D / 16; ++j)
                    q_frag[((row_group * kMt + mt) * (D / 16) + j) * 32 + lane] = make_uint4(raw[0][j][0], raw[1][j][0], raw[0][j][1], raw[1][j][1]);
        }
        __syncthreads();
        const uint4* my_q = q_frag + (size_t)row_group * kMt * (D / 16) * 32 + lane;

        float m_ref[kMt][2], l[kMt][2], o_acc[kMt][D / 8][4];
#pragma unroll
        for (int mt = 0; mt < kMt; ++mt) {
            m_ref[mt][0] = m_ref[mt][1] = -INFINITY;
            l[mt][0] = l[mt][1] = 0.f;
#pragma unroll
            for (int u = 0; u < D / 8; ++u) o_acc[mt][u][0] = o_acc[mt][u][1] = o_acc[mt][u][2] = o_acc[mt][u][3] = 0.f;
        }

        // ---- the keys: chunk c is 32 keys of tile t0 + c / 4; this warp's are key_group, key_group + wk, ... ----
        const int n_chunks = 4 * (s.t1 - s.t0);
        const int32_t* table = prm.map.block_table + (size_t)s.b * prm.map.max_pages;
        int page_base = -1, pages = 0;               // a lane's page of 32 tiles
        auto locate = [&](int c) -> Chunk {
            Chunk x;
            x.tile = s.t0 + (c >> 2);
            x.sub = c & 3;
            x.valid = 0;
            x.inside = false;
            x.k = x.v = nullptr;
            x.ks = x.vs = 1.f;
            if (c >= n_chunks) return x;
            const int rel = c >> 2;
            if (page_base < 0 || rel >= page_base + 32) {
                page_base = rel & ~31;
                const int t = s.t0 + page_base + lane;
                pages = t < min(s.t1, s.nkt) ? __ldg(table + t) : -1;
            }
            const int page = __shfl_sync(0xffffffffu, pages, rel - page_base);
            const int at = x.sub * kChunk / bp.block;
            if (x.tile >= s.nkt) {                   // the soft prompts
                x.valid = min(max(S - x.sub * kChunk, 0), kChunk);
                x.inside = true;
                x.k = bp.k_soft + ((size_t)(x.sub * kChunk) * Hkv + s.g) * D;
                x.v = bp.v_soft + ((size_t)(x.sub * kChunk) * Hkv + s.g) * D;
                if (x.valid > 0) {
                    x.ks = __ldg(bp.ks_soft + s.g * nb + at);
                    x.vs = __ldg(bp.vs_soft + s.g * nb + at);
                }
                return x;
            }
            const int64_t left = s.P + R - ((int64_t)x.tile * kTileKeys + x.sub * kChunk);
            x.valid = (int)min(max(left, (int64_t)0), (int64_t)kChunk);
            x.inside = (uint32_t)page < (uint64_t)bp.n_pages;
            if (x.valid > 0 && x.inside) {
                const size_t slot = (size_t)page * kTileKeys + x.sub * kChunk;
                x.k = bp.k + (slot * Hkv + s.g) * D;
                x.v = bp.v + (slot * Hkv + s.g) * D;
                const size_t sc = ((size_t)page * Hkv + s.g) * nb + at;
                x.ks = __ldg(bp.ks + sc);
                x.vs = __ldg(bp.vs + sc);
            }
            return x;
        };
        KRegs<D> kr;
        VRegs<D> vr;
        auto load_k = [&](const Chunk& x) {
            // (soft prompts: rows past the last one are not there to be read)
            if (x.valid <= 0) return;
            if (!x.inside) kr.clear();
            else if (x.tile < s.nkt || x.valid == kChunk) kr.load(x.k, pitch, lane);
            else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int h = 0; h < D / 64; ++h)
                        kr.w[t][h] = 8 * t + (lane >> 2) < x.valid ? ldg16(x.k + (8 * t + (lane >> 2)) * pitch + (lane & 3) * 16 + 64 * h) : make_uint4(0u, 0u, 0u, 0u);
            }
        };
        auto load_v = [&](const Chunk& x) {
            if (x.valid <= 0) return;
            if (!x.inside) vr.cut(0, lane);
            else if (x.tile < s.nkt || x.valid == kChunk) vr.load(x.v, pitch, lane);
            else {
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int o = 0; o < 2; ++o)
#pragma unroll
                        for (int i = 0; i < D / 32; ++i) {
                            const int key = 8 * t + 2 * (lane & 3) + o;
                            vr.w[t][o][i] = key < x.valid ? __ldg(reinterpret_cast<const uint32_t*>(x.v + key * pitch + (lane >> 2) * (D / 8)) + i) : 0u;
                        }
            }
        };
        Chunk cur = locate(key_group);
        load_k(cur);
        load_v(cur);
#pragma unroll 1
        for (int c = key_group; c < n_chunks; c += wk) {
            const Chunk next = locate(c + wk);
            if (cur.valid <= 0) {                    // past the last slot, or the last soft prompt
                load_k(next);
                load_v(next);
                cur = next;
                continue;
            }
            // ---- scores ----
            float sc[kMt][4][4];
#pragma unroll
            for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
                for (int t = 0; t < 4; ++t) sc[mt][t][0] = sc[mt][t][1] = sc[mt][t][2] = sc[mt][t][3] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                uint4 a[kMt];
#pragma unroll
                for (int mt = 0; mt < kMt; ++mt) a[mt] = my_q[(mt * (D / 16) + j) * 32];
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    uint32_t b0, b1;
                    e4m3_to_f16x4(kr.word(t, j), b0, b1);
#pragma unroll
                    for (int mt = 0; mt < kMt; ++mt) mma_f16(sc[mt][t], a[mt], b0, b1);
                }
            }
            load_k(next);
            // ---- weights ----
            const float vs = fmaxf(cur.vs, kLeastScale), off = log2f(vs), inv_vs = 1.f / vs;
            const float ck = prm.c * cur.ks;
            uint32_t p[kMt][4][2];                   // f16 pairs: key tile, row n or n + 8
#pragma unroll
            for (int mt = 0; mt < kMt; ++mt) {
                if (cur.tile >= s.masked) {
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        uint64_t lo, hi;
                        visible_bits(s, cur.tile, R, T, S, row_r[mt][o], row_r[mt][o] >= 0, mask[mt][o], lo, hi);
                        const uint32_t vis = (uint32_t)((cur.sub & 2 ? hi : lo) >> (32 * (cur.sub & 1)));
#pragma unroll
                        for (int t = 0; t < 4; ++t)
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                if (!((vis >> (8 * t + 2 * (lane & 3) + i)) & 1u)) sc[mt][t][2 * o + i] = -INFINITY;
                    }
                    if (row_r[mt][0] < 0)            // (rows that do not exist see every key: none but those that are there)
#pragma unroll
                        for (int t = 0; t < 4; ++t) sc[mt][t][0] = sc[mt][t][1] = 0.f;
                    if (row_r[mt][1] < 0)
#pragma unroll
                        for (int t = 0; t < 4; ++t) sc[mt][t][2] = sc[mt][t][3] = 0.f;
                }
                float alpha[2], a_row[2], add[2];
                bool move = false;
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    float top = fmaxf(fmaxf(fmaxf(sc[mt][0][2 * o], sc[mt][0][2 * o + 1]), fmaxf(sc[mt][1][2 * o], sc[mt][1][2 * o + 1])),
                                      fmaxf(fmaxf(sc[mt][2][2 * o], sc[mt][2][2 * o + 1]), fmaxf(sc[mt][3][2 * o], sc[mt][3][2 * o + 1])));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
                    // (a factor of 0 would turn the -infinity of masked keys into NaN)
                    a_row[o] = fmaxf(ck * q_scale[mt][o], 1.1754944e-38f);
                    const float m_new = fmaxf(m_ref[mt][o], fmaf(top, a_row[o], off));
                    const bool mv = m_new - m_ref[mt][o] > kRescaleThreshold;        // false when both are -inf (NaN)
                    alpha[o] = mv ? ex2(m_ref[mt][o] - m_new) : 1.f;
                    if (mv) m_ref[mt][o] = m_new;
                    move = move || mv;
                    add[o] = off - (m_ref[mt][o] == -INFINITY ? 0.f : m_ref[mt][o]);
                }
                if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                    for (int u = 0; u < D / 8; ++u) {
                        o_acc[mt][u][0] *= alpha[0];
                        o_acc[mt][u][1] *= alpha[0];
                        o_acc[mt][u][2] *= alpha[1];
                        o_acc[mt][u][3] *= alpha[1];
                    }
                    l[mt][0] *= alpha[0];
                    l[mt][1] *= alpha[1];
                }
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    float sum = 0.f;
#pragma unroll
                    for (int t = 0; t < 4; ++t) {
                        const float x0 = ex2(fmaf(sc[mt][t][2 * o], a_row[o], add[o])), x1 = ex2(fmaf(sc[mt][t][2 * o + 1], a_row[o], add[o]));
                        sum += x0 + x1;
                        p[mt][t][o] = pack_f16(x0, x1);
                    }
                    l[mt][o] = fmaf(sum, inv_vs, l[mt][o]);
                }
            }
            // ---- O += P V ----
            if (cur.valid < kChunk) vr.cut(cur.valid, lane);
#pragma unroll
            for (int h = 0; h < 2; ++h) {            // 16 keys: key tiles 2 h and 2 h + 1
                uint4 a[kMt];
#pragma unroll
                for (int mt = 0; mt < kMt; ++mt) a[mt] = make_uint4(p[mt][2 * h][0], p[mt][2 * h][1], p[mt][2 * h + 1][0], p[mt][2 * h + 1][1]);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {   // four columns of a lane
                    uint32_t b0[4], b1[4];
                    const uint32_t e0 = vr.w[2 * h][0][i], d0 = vr.w[2 * h][1][i], e1 = vr.w[2 * h + 1][0][i], d1 = vr.w[2 * h + 1][1][i];
                    e4m3_to_f16x4(__byte_perm(e0, d0, 0x5140), b0[0], b0[1]);
                    e4m3_to_f16x4(__byte_perm(e0, d0, 0x7362), b0[2], b0[3]);
                    e4m3_to_f16x4(__byte_perm(e1, d1, 0x5140), b1[0], b1[1]);
                    e4m3_to_f16x4(__byte_perm(e1, d1, 0x7362), b1[2], b1[3]);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int mt = 0; mt < kMt; ++mt) mma_f16(o_acc[mt][4 * i + k], a[mt], b0[k], b1[k]);
                }
            }
            load_v(next);
            cur = next;
        }

        // ---- the end of a run: the warps of a row group meet ----
        const int my_rows = warp * kMt * 16;
#pragma unroll
        for (int mt = 0; mt < kMt; ++mt)
#pragma unroll
            for (int o = 0; o < 2; ++o) {
                l[mt][o] += __shfl_xor_sync(0xffffffffu, l[mt][o], 1);
                l[mt][o] += __shfl_xor_sync(0xffffffffu, l[mt][o], 2);
                const int row = mt * 16 + (lane >> 2) + 8 * o;
                if ((lane & 3) == 0) stat[my_rows + row] = make_float2(m_ref[mt][o], l[mt][o]);
                // columns n' of a product's tile u: head dim n' * D / 8 + u; the lane's two columns are 2 x and 2 x + 1: D / 4 contiguous head dims
                float* to = o_part + (size_t)(my_rows + row) * Sh::kPitch + (lane & 3) * Sh::kSeg;
#pragma unroll
                for (int u = 0; u < D / 4; u += 4) {
                    const int c = u < D / 8 ? 2 * o : 2 * o + 1;
                    const int v = u % (D / 8);
                    *reinterpret_cast<float4*>(to + u) = make_float4(o_acc[mt][v][c], o_acc[mt][v + 1][c], o_acc[mt][v + 2][c], o_acc[mt][v + 3][c]);
                }
            }
        __syncthreads();
        constexpr int kVec = D / 4;                  // float4s of a row
        const bool whole = s.part_slot < 0;
        for (int i = threadIdx.x; i < n_rows * kVec; i += Sh::kThreads) {
            const int m = i / kVec, x = i % kVec;
            const int rg = m / (kMt * 16), row = m % (kMt * 16);
            float M = -INFINITY;
            for (int k = 0; k < wk; ++k) M = fmaxf(M, stat[(k * wr + rg) * kMt * 16 + row].x);
            float L = 0.f;
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int k = 0; k < wk; ++k) {
                const int at = (k * wr + rg) * kMt * 16 + row;
                const float2 ml = stat[at];
                const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - M);
                const float4 v = *reinterpret_cast<const float4*>(o_part + (size_t)at * Sh::kPitch + (x / (kVec / 4)) * Sh::kSeg + (x % (kVec / 4)) * 4);
                L = fmaf(f, ml.y, L);
                acc.x = fmaf(f, v.x, acc.x);
                acc.y = fmaf(f, v.y, acc.y);
                acc.z = fmaf(f, v.z, acc.z);
                acc.w = fmaf(f, v.w, acc.w);
            }
            const int r = r0 + m / G;
            if (whole) {
                const size_t row_out = ((size_t)s.b * R + r) * Hq + s.g * G + m % G;
                const float inv = 1.f / L;
                reinterpret_cast<uint2*>(prm.out + row_out * D)[x] = make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
                if (prm.lse && x == 0) prm.lse[row_out] = natural_lse(M, L);
            } else {
                float* part = prm.partials + (size_t)s.part_slot * (partial_slot_bytes() / sizeof(float));
                const int t = (r - r0) / prm.rpt, at = t * 128 + (r - r0 - t * prm.rpt) * G + m % G;
                reinterpret_cast<float4*>(part + (size_t)at * kPartD)[x] = acc;
                if (x == 0) {
                    part[(size_t)kPartRows * kPartD + at] = M;
                    part[(size_t)kPartRows * kPartD + kPartRows + at] = L;
                }
            }
        }
        __syncthreads();                             // shared memory is the next run's
    }
}

template <int D, int kMt, int kWarps>
cudaError_t launch(const Params& prm, const BlockParams& bp, int units, cudaStream_t st)
{
    using Sh = Shape<D, kMt, kWarps>;
    static OncePerDevice attr_done;
    cudaError_t e = attr_done.run([&] {
        return cudaFuncSetAttribute(attention_block_kernel<D, kMt, kWarps>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                    (kMt == 2 ? 8 : 1) * Sh::kQBytes + Sh::kOBytes + Sh::kStatBytes);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute pdl[1];
    pdl[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    pdl[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)units);
    cfg.blockDim = dim3(Sh::kThreads);
    cfg.dynamicSmemBytes = bp.wr * Sh::kQBytes + Sh::kOBytes + Sh::kStatBytes;
    cfg.stream = st;
    cfg.attrs = pdl;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attention_block_kernel<D, kMt, kWarps>, prm, bp);
}

}  // namespace blk
}  // namespace tc

cudaError_t launch_attention_block(const Ctx* ctx, const confu_dims& d, const void* q, const void* k_cache, const void* v_cache,
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
    blk::BlockParams bp;
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
    // M tiles of 16 rows of a row group: one, two, or two for each of 2, 4, 8 groups of warps
    const int rows = (d.T + d.C < prm.rpt * prm.tpg ? d.T + d.C : prm.rpt * prm.tpg) * prm.G, tiles = (rows + 15) / 16;
    bp.wr = 1;
    while (2 * bp.wr < tiles) bp.wr *= 2;
    const int units = ctx->sm_count;
    cudaError_t e;
    if (tiles == 1) e = d.D == 64 ? blk::launch<64, 1, 12>(prm, bp, units, st) : blk::launch<128, 1, 12>(prm, bp, units, st);
    else e = d.D == 64 ? blk::launch<64, 2, 8>(prm, bp, units, st) : blk::launch<128, 2, 8>(prm, bp, units, st);
    if (e != cudaSuccess) return e;
    return launch_combine(prm, ctx->sm_count, st);
}

}  // namespace confu
