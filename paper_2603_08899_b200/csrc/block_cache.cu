// Writing into a block-scaled E4M3 cache: a step's own rows behind the prefixes, and the accepted path's entries to where
// they stay.  A block (32, 64 or 128 slots of a page) of a kv head has one scale, a power of two that whoever writes finds:
//   need  = smallest 2^e with  amax(new entries of the block and head) <= 448 * 2^e
//   scale = need where the block holds nothing yet, else max(scale, need); where it grows, the entries that stay are
//           encoded again: code' = e4m3(code * old / new)
// Both are bound by latency (a launch, two dependent loads, a barrier): a layer's attention waits for the append.  A block of slots
// and head belongs to one CTA, so that its maximum is a reduction within it and nobody else reads or writes its scale.
#include "e4m3.cuh"

namespace confu {

namespace {

constexpr int kThreads = 256;

// largest finite magnitude of eight bf16 numbers
__device__ __forceinline__ float amax8(const uint4& v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float a = fabsf(__uint_as_float(w[i] << 16)), b = fabsf(__uint_as_float(w[i] & 0xffff0000u));
        m = fmaxf(m, a < INFINITY ? a : 0.f);        // (false for NaN)
        m = fmaxf(m, b < INFINITY ? b : 0.f);
    }
    return m;
}

// largest over the CTA of values >= 0, for every thread; `slots`: a word per warp.  Two barriers: what a thread has read before the
// call may be overwritten after it.
__device__ __forceinline__ float cta_max(float v, float* slots)
{
    v = warp_max(v);
    if ((threadIdx.x & 31) == 0) slots[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < blockDim.x / 32 ? slots[threadIdx.x & 31] : 0.f;
    v = warp_max(v);
    __syncthreads();
    return v;
}

__device__ __forceinline__ uint2 encode8(const uint4& v, float s)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16) / s;
        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u) / s;
    }
    return make_uint2(e4m3_pack4(x[0], x[1], x[2], x[3]), e4m3_pack4(x[4], x[5], x[6], x[7]));
}

// four codes of a block with scale `was` -> codes for scale `now`
__device__ __forceinline__ uint32_t recode4(uint32_t codes, float was, float now)
{
    float x[4];
    e4m3_to_f32x4(codes, x);
    return e4m3_pack4(x[0] * was / now, x[1] * was / now, x[2] * was / now, x[3] * was / now);
}
__device__ __forceinline__ uint4 recode16(const uint4& v, float was, float now)
{
    return make_uint4(recode4(v.x, was, now), recode4(v.y, was, now), recode4(v.z, was, now), recode4(v.w, was, now));
}

// Where block `jb` of sequence b lies: its first slot in the pool and its place in the scales.  A negative page id has none.
struct BlockAt {
    int64_t slot, scale;
    bool ok;
};
__device__ __forceinline__ BlockAt block_at(const SlotMap& map, int b, int64_t jb, int block, int Hkv, int g)
{
    const int64_t s = jb * block;
    const int page = map.block_table[(size_t)b * map.max_pages + (s >> 7)];
    const int sub = (int)(s & (kTileKeys - 1)) / block, nb = kTileKeys / block;
    return {(int64_t)page * kTileKeys + (s & (kTileKeys - 1)), ((int64_t)page * Hkv + g) * nb + sub, page >= 0};
}

// CTA (sequence, kv head, K or V; block of slots): its rows' maximum, the scale, the codes.
template <int D>
__global__ void __launch_bounds__(kThreads) append_block_kernel(int R, int Hkv, int block, const __nv_bfloat16* __restrict__ k_rows,
                                                                const __nv_bfloat16* __restrict__ v_rows, uint8_t* k_cache, uint8_t* v_cache,
                                                                float* k_scale, float* v_scale, const SlotMap map,
                                                                const int32_t* __restrict__ prefix_len)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int kPerRow = D / 8, kRows = kThreads / kPerRow, kMost = kTileKeys / kRows;       // units of eight entries
    __shared__ float slots[kThreads / 32];
    const int kv = blockIdx.x & 1, g = (blockIdx.x >> 1) % Hkv, b = (blockIdx.x >> 1) / Hkv;
    const int64_t P = prefix_len[b], jb = P / block + blockIdx.y;
    const int64_t first = max(P, jb * block), end = min(P + R, (jb + 1) * block);
    if (first >= end) return;
    const BlockAt at = block_at(map, b, jb, block, Hkv, g);
    if (!at.ok) return;
    float* scale = (kv ? v_scale : k_scale) + at.scale;
    uint8_t* codes = (kv ? v_cache : k_cache) + (at.slot * Hkv + g) * D;       // of the block's first slot; a slot is Hkv * D further on
    const __nv_bfloat16* rows = (kv ? v_rows : k_rows) + (((size_t)b * R + (size_t)(first - P)) * Hkv + g) * D;
    const int n = (int)(end - first), kept = (int)(first - jb * block);
    const int row0 = threadIdx.x / kPerRow, col = threadIdx.x % kPerRow;
    const size_t pitch = (size_t)Hkv * D;
    uint4 v[kMost];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int r = row0 + i * kRows;
        v[i] = r < n ? *reinterpret_cast<const uint4*>(rows + r * pitch + col * 8) : make_uint4(0u, 0u, 0u, 0u);
    }
    const float was = kept > 0 ? *scale : 0.f;
#pragma unroll
    for (int i = 0; i < kMost; ++i) m = fmaxf(m, amax8(v[i]));
    const float now = fmaxf(was, e4m3_block_scale(cta_max(m, slots)));
    if (threadIdx.x == 0) *scale = now;
    if (kept > 0 && now > was)
        for (int u = threadIdx.x; u < kept * (D / 16); u += kThreads) {
            uint4* p = reinterpret_cast<uint4*>(codes + (u / (D / 16)) * pitch + (u % (D / 16)) * 16);
            *p = recode16(*p, was, now);
        }
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int r = row0 + i * kRows;
        if (r < n) *reinterpret_cast<uint2*>(codes + (kept + r) * pitch + col * 8) = encode8(v[i], now);
    }
}

// CTA (sequence, kv head, K or V; layer): every entry that moves is in registers before the first is written (the sources
// of a block may lie in the blocks behind it, whose scales change too).
constexpr int kCompactThreads = 128;
template <int D>
__global__ void __launch_bounds__(kCompactThreads) compact_block_kernel(int T, int Hkv, int block, void* const* __restrict__ k_layers,
                                                                        void* const* __restrict__ v_layers, float* const* __restrict__ k_scales,
                                                                        float* const* __restrict__ v_scales, const SlotMap map,
                                                                        const int32_t* __restrict__ prefix_len, const int32_t* __restrict__ accept_len,
                                                                        const int32_t* __restrict__ path, int32_t* __restrict__ new_prefix_len,
                                                                        int32_t* __restrict__ status)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    constexpr int kPerRow = D / 16, kRows = kCompactThreads / kPerRow, kMost = (CONFU_MAX_DEPTH + kRows - 1) / kRows;
    constexpr int kBlocks = 3;                       // 63 slots lie in three blocks of 32 at most
    __shared__ int32_t nodes[kPathLen];
    __shared__ uint32_t amax[kBlocks];               // bits of floats >= 0: they order like them
    const int kv = blockIdx.x & 1, g = (blockIdx.x >> 1) % Hkv, b = (blockIdx.x >> 1) / Hkv, layer = blockIdx.y;
    const int tid = threadIdx.x;
    int a = accept_len[b];
    bool ok = a >= 0 && a <= CONFU_MAX_DEPTH;
    if (tid < kPathLen) {
        const int node = path[(size_t)b * kPathLen + tid];
        nodes[tid] = node;
        if (tid == 0) ok = ok && node == 0;
        else if (ok && tid <= a) ok = node > path[(size_t)b * kPathLen + tid - 1] && node < T;
    }
    if (tid < kBlocks) amax[tid] = 0u;
    ok = __syncthreads_and(ok);
    if (!ok) a = 0;
    const int64_t P = prefix_len[b];
    if (g == 0 && kv == 0 && layer == 0 && tid == 0) {
        if (new_prefix_len) new_prefix_len[b] = (int32_t)P + a + 1;
        if (!ok && status) status[b] = CONFU_ST_BAD_PATH;
    }
    if (a == 0) return;
    uint8_t* pool = static_cast<uint8_t*>(kv ? v_layers[layer] : k_layers[layer]);
    float* scales = kv ? v_scales[layer] : k_scales[layer];
    const size_t pitch = (size_t)Hkv * D;
    const int64_t jb0 = (P + 1) / block;             // first destination block
    const int row0 = tid / kPerRow, col = tid % kPerRow;
    uint4 v[kMost];
    float from[kMost];                               // scale of the block that an entry comes from
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int k = 1 + row0 + i * kRows;
        from[i] = 0.f;
        if (k <= a) {
            const int64_t s = P + nodes[k];
            const BlockAt at = block_at(map, b, s / block, block, Hkv, g);
            if (at.ok) {
                from[i] = scales[at.scale];
                v[i] = *reinterpret_cast<const uint4*>(pool + ((at.slot + s % block) * Hkv + g) * D + col * 16);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int k = 1 + row0 + i * kRows;
        if (from[i] > 0.f) {
            // magnitudes of codes order like their values; 0x7f is NaN
            uint32_t m = 0u;
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const uint32_t mag = w[q] & 0x7f7f7f7fu;
                m = __vmaxu4(m, mag & ~__vcmpeq4(mag, 0x7f7f7f7fu));
            }
            m = max(max(m & 0xffu, (m >> 8) & 0xffu), max((m >> 16) & 0xffu, m >> 24));
            float x[4];
            e4m3_to_f32x4(m, x);
            atomicMax(&amax[(P + k) / block - jb0], __float_as_uint(x[0] * from[i]));
        }
    }
    float was[kBlocks];
    BlockAt to[kBlocks];
    const int n_blocks = (int)((P + a) / block - jb0) + 1;
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) {
        to[j] = {0, 0, false};
        was[j] = 1.f;
        if (j < n_blocks) {
            to[j] = block_at(map, b, jb0 + j, block, Hkv, g);
            if (to[j].ok) was[j] = scales[to[j].scale];
        }
    }
    __syncthreads();                                 // everything that moves, and every scale, has been read
    float now[kBlocks];
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) {
        now[j] = fmaxf(was[j], e4m3_block_scale(__uint_as_float(amax[j])));
        if (to[j].ok && tid == 0 && now[j] > was[j]) scales[to[j].scale] = now[j];
    }
    // what stays in the block that the root is in
    const int kept = (int)(P + 1 - jb0 * block);
    if (kept > 0 && to[0].ok && now[0] > was[0])
        for (int u = tid; u < kept * kPerRow; u += kCompactThreads) {
            uint4* p = reinterpret_cast<uint4*>(pool + ((to[0].slot + u / kPerRow) * Hkv + g) * D + (u % kPerRow) * 16);
            *p = recode16(*p, was[0], now[0]);
        }
#pragma unroll
    for (int i = 0; i < kMost; ++i) {
        const int k = 1 + row0 + i * kRows;
        if (from[i] > 0.f) {
            const int64_t s = P + k;
            const int j = (int)(s / block - jb0);
            const float s_to = j == 0 ? now[0] : j == 1 ? now[1] : now[2];
            const int64_t slot = j == 0 ? to[0].slot : j == 1 ? to[1].slot : to[2].slot;
            if (j == 0 ? to[0].ok : j == 1 ? to[1].ok : to[2].ok)
                *reinterpret_cast<uint4*>(pool + ((slot + s % block) * Hkv + g) * D + col * 16) =
                    from[i] == s_to ? v[i] : recode16(v[i], from[i], s_to);
        }
    }
    (void)pitch;
}

}  // namespace

cudaError_t launch_append_block(const Ctx* ctx, const confu_dims& d, const void* k_rows, const void* v_rows, void* k_cache,
                                void* v_cache, const SlotMap& map, const int32_t* prefix_len, cudaStream_t st)
{
    const int R = d.T + d.C;
    // (as many blocks as R slots can touch, wherever the first of them lies)
    const dim3 grid((unsigned)(2 * d.B * d.Hkv), (unsigned)((R + ctx->block - 2) / ctx->block + 1));
    auto kernel = d.D == 64 ? append_block_kernel<64> : append_block_kernel<128>;
    return launch_pdl(kernel, grid, dim3(kThreads), st, R, (int)d.Hkv, ctx->block, (const __nv_bfloat16*)k_rows, (const __nv_bfloat16*)v_rows,
                      (uint8_t*)k_cache, (uint8_t*)v_cache, ctx->k_block_scale, ctx->v_block_scale, map, prefix_len);
}

cudaError_t launch_compact_block(const Ctx* ctx, const confu_dims& d, int n_layers, void* const* k_layers, void* const* v_layers,
                                 const SlotMap& map, const int32_t* prefix_len, const int32_t* accept_len, const int32_t* path,
                                 int32_t* new_prefix_len, int32_t* status, cudaStream_t st)
{
    const dim3 grid((unsigned)(2 * d.B * d.Hkv), (unsigned)n_layers);
    auto kernel = d.D == 64 ? compact_block_kernel<64> : compact_block_kernel<128>;
    return launch_pdl(kernel, grid, dim3(kCompactThreads), st, (int)d.T, (int)d.Hkv, ctx->layer_block, k_layers, v_layers, ctx->k_block_layers,
                      ctx->v_block_layers, map, prefix_len, accept_len, path, new_prefix_len, status);
}

}  // namespace confu
