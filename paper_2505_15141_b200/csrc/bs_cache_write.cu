// bs_cache_append: new keys and values into the e4m3 cache.  bs_cache_keep_path: the accepted path of a tree of
// drafts to the front of its tree.
//
// Both work on (block, head) pairs, the unit that shares a scale.  The scale of a block is the smallest power of
// two that holds its largest value, and it never shrinks while the block has older tokens: if a new token needs a
// larger one, the older codes are brought to it (a shift of their exponents, see bs_cache_common.cuh).
#include "bs_cache_common.cuh"

namespace bs {

// ---- append ------------------------------------------------------------------------------------

struct CacheAppendParams {
    const void* x[2];                 // keys, values [T, Hkv, d], d contiguous
    long long stride_t[2], stride_h[2];   // in elements
    uint8_t* cache[2];
    float* scale[2];
    const int32_t* slot_map;          // [T]
    int T, Hkv, bt, bt_log2, n_blocks;
    int unit_log2;                    // tokens whose runs one group of warps writes
    int warps_log2;                   // warps in a group
};

constexpr int kApThreads = 256;
constexpr int kApSteps = 8;           // 16-byte pieces of a run a lane holds

// Eight values as they were loaded.
template <typename T> struct Raw8;
template <> struct Raw8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = ld_stream(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void unpack(float (&f)[8]) const { Elem<__nv_bfloat16>::unpack(v, f); }
};
template <> struct Raw8<float> {
    uint4 v, w;
    __device__ __forceinline__ void load(const float* p) {
        v = ld_stream(reinterpret_cast<const uint4*>(p));
        w = ld_stream(reinterpret_cast<const uint4*>(p) + 1);
    }
    __device__ __forceinline__ void unpack(float (&f)[8]) const {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
        f[4] = __uint_as_float(w.x); f[5] = __uint_as_float(w.y); f[6] = __uint_as_float(w.z); f[7] = __uint_as_float(w.w);
    }
};

// A run is a maximal stretch of tokens whose slots are consecutive within one block.  A group of warps owns the
// runs that begin among `unit` consecutive tokens, for one head of the keys or of the values.  A run is held in
// registers whole (eight tokens' 16-byte pieces per lane: 16 tokens of 128 values per warp, as many warps as the
// block needs), so the input is read once: maximum, scale, codes.  Bound by HBM on prompts, by latency on a round.  The
// loads of a run are unconditional (tokens behind it repeat its last one) so that all of them are in flight at once.
// Prompts of 28576 tokens, 8 heads of 128, bf16: 176 MB in 43 us (4.1 TB/s); one token 2.9 us in a graph.
template <typename T, int D>
__global__ void __launch_bounds__(kApThreads, sizeof(T) == 2 ? 3 : 2) cache_append_kernel(const CacheAppendParams p) {
    constexpr int kLanes = D / 8;                             // lanes that hold a token
    constexpr int kPer = 32 / kLanes;                         // tokens per warp and step
    __shared__ float s_max[2][kApThreads / 32];
    pdl_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int nw = 1 << p.warps_log2;
    const int group = warp >> p.warps_log2, w = warp & (nw - 1);
    const unsigned unit = blockIdx.x * (unsigned)(kApThreads / 32 >> p.warps_log2) + group;
    const unsigned heads = 2u * p.Hkv, chunk = unit / heads;
    const int hk = (int)(unit - chunk * heads);
    const long long first = (long long)chunk << p.unit_log2;
    if (first >= p.T) return;                                 // whole groups leave: group barriers stay matched
    const int kv = hk >= p.Hkv, h = hk - kv * p.Hkv;
    const T* x = static_cast<const T*>(kv ? p.x[1] : p.x[0]) + (long long)h * (kv ? p.stride_h[1] : p.stride_h[0]);
    const long long st = kv ? p.stride_t[1] : p.stride_t[0];
    uint8_t* cache = kv ? p.cache[1] : p.cache[0];
    float* scales = kv ? p.scale[1] : p.scale[0];
    const int last = (int)min((long long)p.T, first + (1ll << p.unit_log2));
    const int mask = p.bt - 1;
    const long long nslots = (long long)p.n_blocks << p.bt_log2;
    const int sub = lane / kLanes, piece = (lane % kLanes) * 8;
    int phase = 0;

    for (int i0 = (int)first; i0 < last; i0 += 32) {
        const int ti = i0 + lane;
        const int slot = ti < last ? __ldg(p.slot_map + ti) : -1;
        const int before = ti < last && ti > 0 ? __ldg(p.slot_map + ti - 1) : -2;
        const bool ok = slot >= 0 && slot < nslots;
        unsigned leaders = __ballot_sync(0xffffffffu, ok && (before + 1 != slot || (slot & mask) == 0));
        while (leaders) {
            const int src = __ffs(leaders) - 1;
            leaders &= leaders - 1;
            const int i = i0 + src;
            const int slot0 = __shfl_sync(0xffffffffu, slot, src);
            const int blk = slot0 >> p.bt_log2, off0 = slot0 & mask;
            // length of the run: up to 128 slots, all loads at once
            int n = 0;
            {
                int z[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int j = q * 32 + lane;
                    z[q] = j < p.bt - off0 && i + j < p.T ? __ldg(p.slot_map + i + j) : -1;
                }
                bool whole = true;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const unsigned m = __ballot_sync(0xffffffffu, z[q] == slot0 + q * 32 + lane);
                    if (whole) n += m == 0xffffffffu ? 32 : __ffs(~m) - 1;
                    whole = whole && m == 0xffffffffu;
                }
            }
            float* sc = scales + (size_t)blk * p.Hkv + h;
            uint8_t* block = cache + (((size_t)blk * p.Hkv + h) << p.bt_log2) * D;
            const float old = off0 ? __ldcg(sc) : 0.f;
            Raw8<T> v[kApSteps];
            const T* row0 = x + (long long)i * st + piece;
#pragma unroll
            for (int s = 0; s < kApSteps; ++s) {
                const int j = ((((s << p.warps_log2) + w) * kPer) + sub) - off0;
                v[s].load(row0 + (long long)min(max(j, 0), n - 1) * st);
            }
            float mx = 0.f;
#pragma unroll
            for (int s = 0; s < kApSteps; ++s) {              // the repeated tokens do not change the maximum
                float f[8];
                v[s].unpack(f);
#pragma unroll
                for (int e = 0; e < 8; ++e) {                 // infinities and NaN do not set the scale
                    const float a = fabsf(f[e]);
                    mx = fmaxf(mx, a <= 3.402823466e38f ? a : 0.f);
                }
            }
            mx = warp_max(mx);
            if (nw > 1) {
                if (lane == 0) s_max[phase][warp] = mx;
                asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(nw * 32) : "memory");
                for (int q = 0; q < nw; ++q) mx = fmaxf(mx, s_max[phase][group * nw + q]);
                phase ^= 1;
            }
            const float fresh = pow2_scale(mx);
            const float now = off0 ? fmaxf(old, fresh) : fresh;
            const float inv = 1.f / now;                      // exact: a power of two
            const bool grow = off0 && fresh > old;
#pragma unroll
            for (int s = 0; s < kApSteps; ++s) {
                const int off = (((s << p.warps_log2) + w) * kPer) + sub;
                if (off >= off0 && off < off0 + n) {
                    float f[8];
                    v[s].unpack(f);
                    *reinterpret_cast<uint2*>(block + off * D + piece) =
                        make_uint2(e4m3x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
                                   e4m3x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv));
                }
            }
            if (grow) {                                       // older tokens of the block follow its scale
                const float again = old * inv;
                for (int s = 0; s < kApSteps; ++s) {
                    const int off = (((s << p.warps_log2) + w) * kPer) + sub;
                    if (off < off0) {
                        uint2* q = reinterpret_cast<uint2*>(block + off * D + piece);
                        const uint2 c = __ldcg(q);
                        *q = make_uint2(rescale_codes(c.x, again), rescale_codes(c.y, again));
                    }
                }
            }
            if (w == 0 && lane == 0 && (grow || !off0)) *sc = now;
        }
    }
}

// ---- keep path -----------------------------------------------------------------------------------

struct CacheKeepParams {
    const int32_t* out_nodes;         // [B, Nmax]
    const int32_t* accept_len;        // [B]
    const int32_t* seq_len;           // [B] position of the tree's root
    const int32_t* block_table;       // [B, W]
    uint8_t* cache[2];
    float* scale[2];
    int32_t* status;                  // [B] or NULL
    int B, Nmax, W, Hkv, bt, bt_log2, n_blocks;
};

constexpr int kKeepWarps = 4;

// A warp per (sequence, head, keys or values): token j of the path moves from seq_len + node_j to
// seq_len + 1 + j, never to the right, so the destination blocks are written in ascending order and no block is
// read after it was written.  Latency only: a path has at most 31 tokens; 256 trees take 2.9 us in a graph.
template <int D>
__global__ void __launch_bounds__(kKeepWarps * 32) cache_keep_kernel(const CacheKeepParams p) {
    constexpr int kLanes = D / 16, kPer = 32 / kLanes;        // lanes per token, tokens per step
    constexpr int kSteps = (BS_MAX_GAMMA + kPer - 1) / kPer;
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const long long unit = (long long)blockIdx.x * kKeepWarps + (threadIdx.x >> 5);
    const int hk = (int)(unit % (2 * p.Hkv));
    const long long bl = unit / (2 * p.Hkv);
    if (bl >= p.B) return;
    const int b = (int)bl;
    const int kv = hk >= p.Hkv, h = hk - kv * p.Hkv;
    uint8_t* cache = kv ? p.cache[1] : p.cache[0];
    float* scales = kv ? p.scale[1] : p.scale[0];
    const int tau = p.accept_len[b];
    const long long base = p.seq_len[b];
    const int st = p.status ? __ldcg(p.status + b) : 0;
    // the plan gave the sequence no slots: its path was never written
    if (st & (BS_DEV_BAD_LENGTH | BS_DEV_NO_BLOCKS | BS_DEV_NO_ROOM)) return;
    if (tau == 0 && base >= 0) return;
    // lane j holds token j of the path
    const bool mine = lane < tau && tau <= p.Nmax;
    const int node = mine ? p.out_nodes[(size_t)b * p.Nmax + lane] : 0;
    const int prev = __shfl_up_sync(0xffffffffu, node, 1);
    const int nmax_node = __shfl_sync(0xffffffffu, node, (tau - 1) & 31);
    const long long end = base + 1 + nmax_node;               // tokens up to the deepest source
    int bits = 0;
    if (tau < 0 || tau > p.Nmax || base < 0) bits = BS_DEV_BAD_LENGTH;
    else if (mine && (node < lane + 1 || node > p.Nmax || (lane && node <= prev))) bits = BS_DEV_BAD_TREE;
    bits = __reduce_or_sync(0xffffffffu, (unsigned)bits);
    if (!bits && end > (long long)p.W << p.bt_log2) bits = BS_DEV_BAD_LENGTH;
    int sblk = -1, soff = 0;
    if (!bits) {
        const long long src = base + node;
        sblk = mine ? p.block_table[(size_t)b * p.W + (src >> p.bt_log2)] : -1;
        soff = (int)(src & (p.bt - 1));
        const int dblk = mine ? p.block_table[(size_t)b * p.W + ((base + 1 + lane) >> p.bt_log2)] : -1;
        const bool bad = mine && (sblk < 0 || sblk >= p.n_blocks || dblk < 0 || dblk >= p.n_blocks);
        if (__any_sync(0xffffffffu, bad)) bits = BS_DEV_BAD_BLOCK;
    }
    if (bits) {
        if (p.status && hk == 0 && lane == 0) atomicOr(p.status + b, bits);
        return;
    }
    const float sscale = mine ? __ldcg(scales + (size_t)sblk * p.Hkv + h) : 0.f;
    const int sub = lane / kLanes, piece = (lane % kLanes) * 16;

    for (int j0 = 0; j0 < tau;) {                             // one destination block at a time
        const long long dst0 = base + 1 + j0;
        const int lead = (int)(dst0 & (p.bt - 1));
        const int m = min(tau - j0, p.bt - lead);             // path tokens that end up in it
        const int blk = p.block_table[(size_t)b * p.W + (dst0 >> p.bt_log2)];
        float* sc = scales + (size_t)blk * p.Hkv + h;
        uint8_t* block = cache + (((size_t)blk * p.Hkv + h) << p.bt_log2) * D;
        const float old = __ldcg(sc);
        const bool here = lane >= j0 && lane < j0 + m;
        const float now = fmaxf(old, warp_max(here ? sscale : 0.f));
        uint4 v[kSteps];
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int j = s * kPer + sub;
            const int from = (j0 + j) & 31;
            const int jb = __shfl_sync(0xffffffffu, sblk, from), jo = __shfl_sync(0xffffffffu, soff, from);
            if (j < m)
                v[s] = __ldcg(reinterpret_cast<const uint4*>(cache + ((((size_t)jb * p.Hkv + h) << p.bt_log2) + jo) * D + piece));
        }
        __syncwarp();                                         // every source of this block has been read
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const int j = s * kPer + sub;
            const float js = __shfl_sync(0xffffffffu, sscale, (j0 + j) & 31);
            if (j < m) {
                const float f = js / now;
                if (js != now)
                    v[s] = make_uint4(rescale_codes(v[s].x, f), rescale_codes(v[s].y, f), rescale_codes(v[s].z, f),
                                      rescale_codes(v[s].w, f));
                *reinterpret_cast<uint4*>(block + (lead + j) * D + piece) = v[s];
            }
        }
        if (now > old) {                                      // older tokens of the block follow its scale
            const float f = old / now;
            for (int o = sub; o < lead; o += kPer) {
                uint4* q = reinterpret_cast<uint4*>(block + o * D + piece);
                const uint4 c = *q;
                *q = make_uint4(rescale_codes(c.x, f), rescale_codes(c.y, f), rescale_codes(c.z, f), rescale_codes(c.w, f));
            }
            if (lane == 0) *sc = now;
        }
        j0 += m;
    }
}

}  // namespace bs

using namespace bs;

static int log2_of(int x) {
    int l = 0;
    while ((1 << l) < x) ++l;
    return l;
}

extern "C" bs_status bs_cache_append(const void* k, const void* v, bs_dtype dtype, long long k_stride_t,
                                     long long k_stride_h, long long v_stride_t, long long v_stride_h,
                                     const int32_t* slot_map, int T, int Hkv, int d, void* k_cache, float* k_scale,
                                     void* v_cache, float* v_scale, int n_blocks, int block_tokens, void* stream) {
    if (T < 1 || Hkv < 1 || d < 1 || n_blocks < 1 || block_tokens < 1) return BS_ERR_INVALID_ARG;
    if (dtype != BS_F32 && dtype != BS_BF16) return BS_ERR_INVALID_ARG;
    if (!k || !v || !slot_map || !k_cache || !k_scale || !v_cache || !v_scale) return BS_ERR_INVALID_ARG;
    if (!cache_geometry_ok(Hkv, d, n_blocks, block_tokens)) return BS_ERR_UNSUPPORTED;
    // 16-byte loads of the inputs, 8-byte stores of the codes
    const long long vec = dtype == BS_F32 ? 4 : 8;
    if ((k_stride_t % vec) || (k_stride_h % vec) || (v_stride_t % vec) || (v_stride_h % vec)) return BS_ERR_UNSUPPORTED;
    const uintptr_t al = reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) |
                         reinterpret_cast<uintptr_t>(k_cache) | reinterpret_cast<uintptr_t>(v_cache);
    if (al & 15) return BS_ERR_INVALID_ARG;
    CacheAppendParams p;
    p.x[0] = k; p.x[1] = v;
    p.stride_t[0] = k_stride_t; p.stride_t[1] = v_stride_t;
    p.stride_h[0] = k_stride_h; p.stride_h[1] = v_stride_h;
    p.cache[0] = static_cast<uint8_t*>(k_cache); p.cache[1] = static_cast<uint8_t*>(v_cache);
    p.scale[0] = k_scale; p.scale[1] = v_scale;
    p.slot_map = slot_map;
    p.T = T; p.Hkv = Hkv; p.bt = block_tokens; p.bt_log2 = log2_of(block_tokens); p.n_blocks = n_blocks;
    const int run = kApSteps * (32 / (d / 8));                // tokens a warp holds
    p.warps_log2 = block_tokens > run ? log2_of(block_tokens / run) : 0;
    // A round has a run every few tokens, and a group of warps takes its runs one after another: few tokens, so that
    // none waits for another's run.  With many tokens most groups would find no run, and launching them is the cost.
    // 8 heads of 128; units of 1, 4, 8 tokens, of a block: 64 sequences with 4 tokens each, blocks of 64 tokens, 14.4, 12.3,
    // 13.4, 41.0 us; 256 with 4, 35, 27, 28, 43; 256 with 8, 48, 31, 29, 35; 512 with 8, 88, 53, 45, 53; 1024 with 9, 179, 99, 86, 82; prompts of 2048
    // tokens, one 39, 18, 14, 12, two 68, 29, 21, 14, four 129, 47, 33, 21.  Blocks of 16 and 128 order them alike.
    const long long rows = (long long)T * Hkv * 2;
    p.unit_log2 = rows <= 24576 ? 2 : rows <= 65536 ? 3 : p.bt_log2;
    const long long units = (((long long)T + (1ll << p.unit_log2) - 1) >> p.unit_log2) * 2 * Hkv;
    const int per = kApThreads / 32 >> p.warps_log2;
    const long long grid = (units + per - 1) / per;
    if (units > 0x7fffffffLL) return BS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == BS_F32)
        return cuda_status(d == 64 ? launch_pdl(cache_append_kernel<float, 64>, (unsigned)grid, kApThreads, 0, st, p)
                                   : launch_pdl(cache_append_kernel<float, 128>, (unsigned)grid, kApThreads, 0, st, p));
    return cuda_status(d == 64 ? launch_pdl(cache_append_kernel<__nv_bfloat16, 64>, (unsigned)grid, kApThreads, 0, st, p)
                               : launch_pdl(cache_append_kernel<__nv_bfloat16, 128>, (unsigned)grid, kApThreads, 0, st, p));
}

extern "C" bs_status bs_cache_keep_path(const int32_t* out_nodes, const int32_t* accept_len, const int32_t* seq_len, int B,
                                        int Nmax, const int32_t* block_table, int max_blocks, int Hkv, int d, void* k_cache,
                                        float* k_scale, void* v_cache, float* v_scale, int n_blocks, int block_tokens,
                                        int32_t* status, void* stream) {
    if (B < 1 || Nmax < 1 || max_blocks < 1 || Hkv < 1 || d < 1 || n_blocks < 1 || block_tokens < 1) return BS_ERR_INVALID_ARG;
    if (!out_nodes || !accept_len || !seq_len || !block_table || !k_cache || !k_scale || !v_cache || !v_scale)
        return BS_ERR_INVALID_ARG;
    if (B > BS_MAX_BATCH || Nmax > BS_MAX_GAMMA || max_blocks > BS_MAX_SEQ_BLOCKS ||
        !cache_geometry_ok(Hkv, d, n_blocks, block_tokens))
        return BS_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(k_cache) | reinterpret_cast<uintptr_t>(v_cache)) & 15) return BS_ERR_INVALID_ARG;
    CacheKeepParams p;
    p.out_nodes = out_nodes; p.accept_len = accept_len; p.seq_len = seq_len; p.block_table = block_table;
    p.cache[0] = static_cast<uint8_t*>(k_cache); p.cache[1] = static_cast<uint8_t*>(v_cache);
    p.scale[0] = k_scale; p.scale[1] = v_scale; p.status = status;
    p.B = B; p.Nmax = Nmax; p.W = max_blocks; p.Hkv = Hkv; p.bt = block_tokens; p.bt_log2 = log2_of(block_tokens);
    p.n_blocks = n_blocks;
    const long long grid = ((long long)B * 2 * Hkv + kKeepWarps - 1) / kKeepWarps;
    if (grid > 0x7fffffffLL) return BS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cuda_status(d == 64 ? launch_pdl(cache_keep_kernel<64>, (unsigned)grid, kKeepWarps * 32, 0, st, p)
                               : launch_pdl(cache_keep_kernel<128>, (unsigned)grid, kKeepWarps * 32, 0, st, p));
}
