// bs_cache_attention: attention of the new tokens of a round (a chain or a tree of drafts, or a piece of a prompt)
// over the e4m3 cache.
//
//   out_i = sum_j 2^(t_ij) v_j / sum_j 2^(t_ij),   t_ij = log2(e) softmax_scale q_i . k_j
//
// A CTA works on 128 cached tokens at a time, for the rows (new token, query head of the group) of one key head.
// Both products run on the tensor cores with the cache's codes as they are:
//
//   S^T [128 tokens, N rows] = K [128, d] Q^T     K K-major, as the TMA copy leaves it (swizzled)
//   O^T [d, N rows]          = V^T P^T            V^T is the same tile read M-major; P^T from shared memory, N-major
//
// i.e. the tokens (and then d) are the 128 lanes of the MMA and the rows its N: a few rows cost no more than their
// share, and no code is ever converted.  The other operand has to be e4m3 as well (kind::f8f6f4): a bf16 query, scaled by a
// power of two so that its row's largest element lies in [128, 256), is the sum of two e4m3 numbers exactly (four
// significant bits, a signed remainder of four more; elements below 2^-9 of the largest lose bits under 2^-17
// of it), and a probability is split the same way (relative error 2^-8 as in bf16), so each product is two MMAs
// into one accumulator.  Their accumulation was measured against 64 bits: error 2^-20 of the largest product.
//
// Scales.  Keys: t_ij = S_ij * (scale of j's block * c_i).  Values: the scale of a token's block joins the exponent:
//   P''_ij = 2^(t_ij + log2 s_j + 8 - m_i),  m_i = max_j (t_ij + log2 s_j) over the tile,
// which uses the e4m3 range up to 256 whatever the scales are; the sum of the probabilities takes P'' / s_j in fp32.
// O^T of every tile is taken from tensor memory and joined in fp32 registers with the tile's own factor 2^(m_i - m),
// so a token far below the row's running maximum keeps its bits relative to its own tile.
//
// Roles of the 12 warps: 0 TMA producer, 1 MMA issuer, 2-3 queries (split into e4m3 one work item ahead), 4-7 and 8-11
// two softmax groups that take the tiles in turn, each with its own maximum, sum and accumulator (joined at the end of an
// item); a thread is a token in the softmax and an element of d in the accumulator.
//
// Work.  Item = (sequence, key head, N rows).  All tiles of all items, in order, are cut into equal contiguous shares,
// one per CTA, from the lengths on the device; an item that spans several CTAs is joined by the one that finishes
// last, in the order of the shares (the result does not depend on who that is).
#include "bs_cache_common.cuh"
#include "bs_pipeline.cuh"
#include "bs_tensor.cuh"

#include <atomic>

namespace bs {

constexpr int kCaThreads = 384;
constexpr int kCaTile = 128;                   // tokens of a tile = MMA lanes
constexpr int kCaSmem = 230400;                // of 232448 bytes a CTA may use
constexpr int kCaScaleRing = 8;                // tiles whose scales are kept; more than the tiles in flight
constexpr int kCaMaxPages = 8;                 // blocks of 16 tokens in a tile

struct CacheAttnParams {
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    long long q_st, q_sh, o_st, o_sh;          // strides of a token and a head, elements
    const int32_t* cu_new;
    const int32_t* kv_len;
    const int32_t* block_table;
    const int32_t* node_parent;                // NULL: chains
    const float* k_scale;
    const float* v_scale;
    int32_t* status;
    float* partial;                            // [grid, 2] pieces
    uint32_t* ticket;                          // [grid] arrivals at an item, kept by its first CTA; zero between calls
    float scale_log2;                          // softmax_scale * log2(e)
    int B, T, W, Nmax, Hq, Hkv, G, TQ;         // TQ: new tokens of an item, N / G
    int bt_log2, n_blocks;
};

// The piece of the work a role is at.
struct CaCursor {
    int b, h, rt, nrt;                         // item
    int n, base, q0;                           // its sequence: new tokens, position of the first, its row
    int t, ntiles;                             // next tile, tiles of the item
    long long x, end;                          // the same counted over all work; end of this CTA's share
};

__device__ __forceinline__ int ca_limit(const CacheAttnParams& p, int base, int n, int rt) {   // tokens an item may see
    return base + (p.node_parent ? n : min(n, (rt + 1) * p.TQ));
}
__device__ __forceinline__ int ca_tiles(int limit) { return max(1, (limit + kCaTile - 1) / kCaTile); }

// Lengths of sequence b; false (and no work) if they make no sense.
__device__ __forceinline__ bool ca_seq(const CacheAttnParams& p, int b, int& n, int& base, int& q0) {
    const int c0 = __ldg(p.cu_new + b), c1 = __ldg(p.cu_new + b + 1), kv = __ldg(p.kv_len + b);
    const bool ok = c0 >= 0 && c1 >= c0 && c1 <= p.T && kv >= 0 && kv <= (long long)p.W << p.bt_log2 &&
                    (!p.node_parent || c1 - c0 <= p.Nmax + 1);
    n = ok ? c1 - c0 : 0;
    base = kv - n;
    q0 = c0;
    return ok;
}
__device__ __forceinline__ long long ca_head_work(const CacheAttnParams& p, int n, int base) {
    long long w = 0;
    for (int rt = 0; rt * p.TQ < n; ++rt) w += ca_tiles(ca_limit(p, base, n, rt));
    return w;
}
__device__ __forceinline__ void ca_item(const CacheAttnParams& p, CaCursor& c) {
    c.ntiles = ca_tiles(ca_limit(p, c.base, c.n, c.rt));
}
// To the next item (c.t = 0).
__device__ __forceinline__ void ca_next(const CacheAttnParams& p, CaCursor& c) {
    c.t = 0;
    if (++c.rt == c.nrt) {
        c.rt = 0;
        if (++c.h == p.Hkv) {
            c.h = 0;
            do {
                ++c.b;
            } while (c.b < p.B && (!ca_seq(p, c.b, c.n, c.base, c.q0) || c.n == 0));
            if (c.b >= p.B) return;
            c.nrt = (c.n + p.TQ - 1) / p.TQ;
        }
    }
    ca_item(p, c);
}

__device__ __forceinline__ uint64_t ca_desc(uint32_t addr, uint32_t lbo, uint32_t sbo, uint32_t swizzle) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | ((uint64_t)(lbo >> 4) << 16) | ((uint64_t)(sbo >> 4) << 32) |
           (1ull << 46) | ((uint64_t)swizzle << 61);
}
__device__ __forceinline__ void ca_mma(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void ca_tma(uint32_t dst, const CUtensorMap* tm, int block_head, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
        ::"r"(dst), "l"(tm), "r"(0), "r"(0), "r"(block_head), "r"(bar) : "memory");
}
__device__ __forceinline__ void ca_ld16(uint32_t taddr, float (&v)[16]) {
    uint32_t u[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
          "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
        : "r"(taddr) : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ float ca_warp_max(float v) {        // NaN only if every lane has one
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}
// Barrier of `threads` threads that also tells whether any of them brought a true predicate.
__device__ __forceinline__ bool ca_bar_any(int id, int threads, bool pred) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %3, 0;\n\t"
        "barrier.cta.red.or.pred q, %1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r) : "r"(id), "r"(threads), "r"((uint32_t)pred) : "memory");
    return r != 0;
}
__device__ __forceinline__ uint32_t ca_half2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t ca_half2_to_e4m3x2(uint32_t h) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f16x2 %0, %1;" : "=h"(r) : "r"(h));
    return r;
}
// Two values as hi + lo, each a pair of e4m3.  They pass through fp16 (2^-12), where hi and the remainder are exact.
__device__ __forceinline__ void ca_split2(float a, float b, uint32_t& hi, uint32_t& lo) {
    const uint32_t h = ca_half2(a, b);
    hi = ca_half2_to_e4m3x2(h);
    const uint32_t back = e4m3x2_to_half2(hi);
    const __half2 rem = __hsub2(*reinterpret_cast<const __half2*>(&h), *reinterpret_cast<const __half2*>(&back));
    lo = ca_half2_to_e4m3x2(*reinterpret_cast<const uint32_t*>(&rem));
}
// Four words, each four e4m3 of hi (or of lo), from 16 values.
__device__ __forceinline__ void ca_split16(const float (&v)[16], uint32_t (&hi)[4], uint32_t (&lo)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h0, l0, h1, l1;
        ca_split2(v[4 * i], v[4 * i + 1], h0, l0);
        ca_split2(v[4 * i + 2], v[4 * i + 3], h1, l1);
        hi[i] = h0 | (h1 << 16);
        lo[i] = l0 | (l1 << 16);
    }
}

template <int N, int D> struct CaLayout {
    static constexpr int kTileBytes = kCaTile * D;            // K or V of a tile
    static constexpr int kQBytes = N * D;                     // one term of the queries
    static constexpr int kPBytes = N * kCaTile;               // one term of the probabilities
    static constexpr int kMergeBytes = N * D * 4;
    static constexpr int kFixed = 4 * kQBytes + 4 * kPBytes + kMergeBytes;
    // shared memory besides the ring: the static arrays of the kernel take up to 14 KB
    static constexpr int kSlotsFit = (kCaSmem - 14336 - 1024 - kFixed) / kTileBytes;
    static constexpr int kSlots = kSlotsFit > 12 ? 12 : kSlotsFit;
    static constexpr int kDynamic = kSlots * kTileBytes + kFixed + 1024;
    static constexpr int kTmemCols = 4 * N <= 64 ? 64 : 4 * N <= 128 ? 128 : 256;
    static constexpr int kPiece = N * D + 2 * N;              // floats of a partial result
    static_assert(kSlots >= 4 && kSlots / 2 + 2 <= kCaScaleRing, "ring");
    static_assert(N % 16 == 0 && N <= 64, "rows");
};

template <int N, int D>
__global__ void __launch_bounds__(kCaThreads, 1)
cache_attention_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                       const CacheAttnParams p) {
    using L = CaLayout<N, D>;
    constexpr int SLOTS = L::kSlots;
    constexpr uint32_t kSw = D == 128 ? 2 : 4;                // 128-byte or 64-byte swizzle: a token's row
    extern __shared__ unsigned char ca_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(ca_smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_q = smem + SLOTS * L::kTileBytes;        // [2 buffers][2 terms]
    unsigned char* s_p = s_q + 4 * L::kQBytes;                // [2 groups][2 terms]
    float* s_merge = reinterpret_cast<float*>(s_p + 4 * L::kPBytes);   // [N][D]
    __shared__ __align__(8) unsigned long long b_full[SLOTS], b_empty[SLOTS], b_qfull[2], b_qempty[2], b_s[2], b_p[2], b_o[2],
        b_mfull, b_mempty, b_drain;
    __shared__ __align__(16) float s_red[2][4][N];            // maxima of the warps of a group
    __shared__ __align__(16) float s_m[8][N];                 // per warp: the tile's maximum
    __shared__ __align__(16) float2 s_ab[8][N];               // per warp: factors of the accumulator and of the tile
    __shared__ __align__(16) float s_c[2][N];                 // per query buffer: softmax scale of the row
    __shared__ uint32_t s_anc[2][32];                         // per query buffer: ancestors of the tree's nodes
    __shared__ float s_scale[kCaScaleRing][kCaMaxPages][2];
    __shared__ float2 s_mml[N];                               // merge: maximum and sum of the other group
    __shared__ uint32_t s_nan[2][N][D / 32];                  // per group: results a masked-tile NaN of V belongs to
    __shared__ long long s_w[kCaThreads / 32];
    __shared__ long long s_start_off;
    __shared__ int s_start_b;
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    __shared__ int s_last[2];

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (int s = 0; s < SLOTS; ++s) {
            mbar_init(smem_u32(&b_full[s]), 1);
            mbar_init(smem_u32(&b_empty[s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(smem_u32(&b_qfull[a]), 2);              // the two query warps
            mbar_init(smem_u32(&b_qempty[a]), 9);             // the MMAs and the eight softmax warps
            mbar_init(smem_u32(&b_s[a]), 1);
            mbar_init(smem_u32(&b_p[a]), 4);                  // the four warps of a softmax group
            mbar_init(smem_u32(&b_o[a]), 1);
        }
        mbar_init(smem_u32(&b_mfull), 4);
        mbar_init(smem_u32(&b_mempty), 4);
        mbar_init(smem_u32(&b_drain), 1);
        s_abort = 0;
        s_start_b = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tc_alloc(smem_u32(&s_tmem), L::kTmemCols);
    if (warp == 0 && lane < 2) {
        const CUtensorMap* tm = lane ? &tm_v : &tm_k;
        asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory");
    }
    pdl_enter();

    // ---- this CTA's share of the work ----
    const int per = (p.B + kCaThreads - 1) / kCaThreads;
    long long mine = 0;
    for (int b = tid * per; b < min(p.B, (tid + 1) * per); ++b) {
        int n, base, q0;
        if (!ca_seq(p, b, n, base, q0) && p.status && blockIdx.x == 0) atomicOr(p.status + b, BS_DEV_BAD_LENGTH);
        mine += p.Hkv * ca_head_work(p, n, base);
    }
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) s_w[warp] = incl;
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    long long work = 0, before = 0;
#pragma unroll
    for (int w = 0; w < kCaThreads / 32; ++w) {
        if (w < warp) before += s_w[w];
        work += s_w[w];
    }
    const long long grid = work < (long long)gridDim.x ? work : gridDim.x;
    const long long x_lo = grid ? blockIdx.x * work / grid : 0, x_hi = grid && blockIdx.x < grid ? (blockIdx.x + 1) * work / grid : 0;
    const long long from = before + incl - mine;
    if (x_lo < x_hi && x_lo >= from && x_lo < from + mine) {
        long long off = x_lo - from;
        for (int b = tid * per; b < min(p.B, (tid + 1) * per); ++b) {
            int n, base, q0;
            ca_seq(p, b, n, base, q0);
            const long long w = p.Hkv * ca_head_work(p, n, base);
            if (off < w) {
                s_start_b = b;
                s_start_off = off;
                break;
            }
            off -= w;
        }
    }
    __syncthreads();
    const uint32_t tmem = s_tmem;
    CaCursor cur;
    cur.x = x_lo;
    cur.end = x_lo < x_hi ? x_hi : x_lo;
    cur.b = s_start_b;
    if (cur.x < cur.end) {
        ca_seq(p, cur.b, cur.n, cur.base, cur.q0);
        cur.nrt = (cur.n + p.TQ - 1) / p.TQ;
        const long long hw = ca_head_work(p, cur.n, cur.base);
        cur.h = (int)(s_start_off / hw);
        long long off = s_start_off - cur.h * hw;
        cur.rt = 0;
        ca_item(p, cur);
        while (off >= cur.ntiles) {
            off -= cur.ntiles;
            ++cur.rt;
            ca_item(p, cur);
        }
        cur.t = (int)off;
    }

    if (warp == 0) {
        // ================================ TMA producer ================================
        // ring of slots: K of a tile, then V of it, K of the next, ...
        int slot = 0, tile = 0;
        uint32_t ph = 0;
        long long filled = 0;
        bool ok = true;
        const uint32_t page_bytes = (uint32_t)D << p.bt_log2;
        while (cur.x < cur.end && ok) {
            const int limit = ca_limit(p, cur.base, cur.n, cur.rt);
            const int te = (int)min((long long)cur.ntiles, cur.t + (cur.end - cur.x));
            for (int t = cur.t; t < te && ok; ++t, ++tile) {
                const int valid = min(kCaTile, limit - t * kCaTile);
                const int pages = valid > 0 ? (valid + (1 << p.bt_log2) - 1) >> p.bt_log2 : 0;
                int blk = 0;
                float ks = 0.f, vs = 0.f;
                if (lane < pages) {
                    blk = __ldg(p.block_table + (size_t)cur.b * p.W + ((t * kCaTile) >> p.bt_log2) + lane);
                    if (blk < 0 || blk >= p.n_blocks) {
                        if (p.status) atomicOr(p.status + cur.b, BS_DEV_BAD_BLOCK);
                        blk = 0;
                    }
                    ks = __ldg(p.k_scale + (size_t)blk * p.Hkv + cur.h);
                    vs = __ldg(p.v_scale + (size_t)blk * p.Hkv + cur.h);
                }
                for (int kv = 0; kv < 2 && ok; ++kv) {
                    if (!mbar_wait_warp(smem_u32(&b_empty[slot]), ph ^ 1u) || __any_sync(0xffffffffu, s_abort)) { ok = false; break; }
                    // the ring of scales is deeper than the tiles in flight: its entry is free when a slot is
                    if (kv == 0 && lane < pages) {
                        s_scale[tile % kCaScaleRing][lane][0] = ks;
                        s_scale[tile % kCaScaleRing][lane][1] = vs;
                    }
                    __syncwarp();
                    const uint32_t bar = smem_u32(&b_full[slot]);
                    if (lane == 0) {
                        if (pages) mbar_arrive_expect_tx(bar, pages * page_bytes);
                        else mbar_arrive(bar);
                    }
                    __syncwarp();
                    if (lane < pages)
                        ca_tma(smem_u32(smem + slot * L::kTileBytes) + lane * page_bytes, kv ? &tm_v : &tm_k, blk * p.Hkv + cur.h, bar);
                    ++filled;
                    if (++slot == SLOTS) { slot = 0; ph ^= 1u; }
                }
            }
            cur.x += te - cur.t;
            cur.t = te;
            if (cur.t == cur.ntiles && cur.x < cur.end) ca_next(p, cur);
        }
        if (!ok) {                                            // leave no copy in flight behind
            if (lane == 0) {
                s_abort = 1;
                if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
                const int k = (int)min((long long)SLOTS, filled);
                for (int i = 1; i <= k; ++i) {
                    const long long f = filled - i;
                    mbar_wait(smem_u32(&b_full[f % SLOTS]), (uint32_t)((f / SLOTS) & 1));
                }
            }
            __syncwarp();
        }
    } else if (warp == 1) {
        // ================================= MMA issuer =================================
        if (lane == 0) {
            constexpr uint32_t id_s = (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(kCaTile >> 4) << 24);
            constexpr uint32_t id_o = (1u << 4) | (1u << 15) | (1u << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(D >> 4) << 24);
            bool ok = true;
            uint32_t g = 0;                                   // tiles issued
            int item = 0;
            // O^T of tile k: V^T P^T, both terms of P
            auto pv = [&](uint32_t k) {
                const uint32_t w = k & 1;
                const uint32_t slot = (2 * k + 1) % SLOTS;
                if (!mbar_wait(smem_u32(&b_p[w]), (k >> 1) & 1) || s_abort) return false;
                if (!mbar_wait(smem_u32(&b_full[slot]), ((2 * k + 1) / SLOTS) & 1)) return false;
                tc_fence_after();
                const uint32_t sv = smem_u32(smem + slot * L::kTileBytes);
                const uint32_t sp = smem_u32(s_p + w * 2 * L::kPBytes);
#pragma unroll
                for (int term = 0; term < 2; ++term)
#pragma unroll
                    for (int s = 0; s < kCaTile / 32; ++s)
                        ca_mma(tmem + 2 * N + w * N, ca_desc(sv + s * 32 * D, 0, 8 * D, kSw),
                               ca_desc(sp + term * L::kPBytes + s * 512, 128, 2048, 0), id_o, (term | s) ? 1u : 0u);
                tc_commit(smem_u32(&b_empty[slot]));
                tc_commit(smem_u32(&b_o[w]));
                return true;
            };
            while (cur.x < cur.end && ok) {
                const int te = (int)min((long long)cur.ntiles, cur.t + (cur.end - cur.x));
                if (!mbar_wait(smem_u32(&b_qfull[item & 1]), (uint32_t)((item >> 1) & 1)) || s_abort) { ok = false; break; }
                const uint32_t sq = smem_u32(s_q + (item & 1) * 2 * L::kQBytes);
                for (int t = cur.t; t < te && ok; ++t, ++g) {
                    const uint32_t w = g & 1;
                    const uint32_t slot = (2 * g) % SLOTS;
                    if (!mbar_wait(smem_u32(&b_full[slot]), ((2 * g) / SLOTS) & 1) || s_abort) { ok = false; break; }
                    // S of tile g - 2 has been read: P of it was waited for when its O was issued
                    tc_fence_after();
                    const uint32_t sk = smem_u32(smem + slot * L::kTileBytes);
#pragma unroll
                    for (int term = 0; term < 2; ++term)
#pragma unroll
                        for (int s = 0; s < D / 32; ++s)
                            ca_mma(tmem + w * N, ca_desc(sk + s * 32, 16, 8 * D, kSw),
                                   ca_desc(sq + term * L::kQBytes + s * 256, 128, 8 * D, 0), id_s, (term | s) ? 1u : 0u);
                    tc_commit(smem_u32(&b_empty[slot]));
                    tc_commit(smem_u32(&b_s[w]));
                    if (t + 1 == te) tc_commit(smem_u32(&b_qempty[item & 1]));
                    if (g > 0) ok = pv(g - 1);
                }
                ++item;
                cur.x += te - cur.t;
                cur.t = te;
                if (cur.t == cur.ntiles && cur.x < cur.end) ca_next(p, cur);
            }
            if (ok && g > 0) ok = pv(g - 1);
            if (!ok) {
                s_abort = 1;
                if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
                tc_commit(smem_u32(&b_drain));                // leave no MMA in flight behind
                mbar_wait(smem_u32(&b_drain), 0);
            }
        }
        __syncwarp();
    } else if (warp < 4) {
        // ================================== queries ==================================
        constexpr int kLanes = D / 8;                         // lanes of a row
        constexpr int kRows = 64 / kLanes;                    // rows per pass of the two warps
        const int qt = tid - 64, sub = qt / kLanes, piece = (qt % kLanes) * 8;
        int item = 0;
        bool ok = true;
        while (cur.x < cur.end && ok) {
            const int buf = item & 1;
            const int te = (int)min((long long)cur.ntiles, cur.t + (cur.end - cur.x));
            if (item >= 2) ok = mbar_wait_warp(smem_u32(&b_qempty[buf]), (uint32_t)(((item >> 1) - 1) & 1)) && !__any_sync(0xffffffffu, s_abort);
            if (!ok) break;
            const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
            unsigned char* q_hi = s_q + buf * 2 * L::kQBytes;
#pragma unroll 4
            for (int r0 = 0; r0 < N; r0 += kRows) {
                const int r = r0 + sub;
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = 0.f;
                if (r < rows)
                    Elem<__nv_bfloat16>::unpack(__ldg(reinterpret_cast<const uint4*>(
                        p.q + (long long)(cur.q0 + i0 + r / p.G) * p.q_st + (long long)(cur.h * p.G + r % p.G) * p.q_sh + piece)), f);
                float mx = 0.f;
                bool fin = true;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    mx = fmaxf(mx, fabsf(f[e]));
                    fin = fin && fabsf(f[e]) <= 3.402823466e38f;
                }
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) {
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
                    fin = __shfl_xor_sync(0xffffffffu, (int)fin, o) && fin;
                }
                // 2^x brings the row's largest element into [128, 256)
                int x = mx > 0.f && fin ? 7 - ((int)(__float_as_uint(mx) >> 23) - 127) : 0;
                x = min(x, 120);
                const float up = __uint_as_float((uint32_t)(x + 127) << 23);
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) ca_split2(f[2 * e] * up, f[2 * e + 1] * up, hi[e], lo[e]);
                unsigned char* at = q_hi + (r >> 3) * (8 * D) + (piece >> 4) * 128 + (r & 7) * 16 + (piece & 15);
                *reinterpret_cast<uint2*>(at) = make_uint2(hi[0] | (hi[1] << 16), hi[2] | (hi[3] << 16));
                *reinterpret_cast<uint2*>(at + L::kQBytes) = make_uint2(lo[0] | (lo[1] << 16), lo[2] | (lo[3] << 16));
                // a row with an infinity or a NaN has no softmax: its scale makes every result NaN
                if (piece == 0) s_c[buf][r] = r >= rows ? 0.f : fin ? p.scale_log2 * __uint_as_float((uint32_t)(127 - x) << 23) : __int_as_float(0x7fc00000);
            }
            if (p.node_parent && warp == 2) {                 // ancestors-or-self of node `lane`
                int par = 0;
                if (lane >= 1 && lane < cur.n) {
                    par = __ldg(p.node_parent + (size_t)cur.b * p.Nmax + lane - 1);
                    if (par < 0 || par >= lane) {
                        if (p.status) atomicOr(p.status + cur.b, BS_DEV_BAD_TREE);
                        par = 0;
                    }
                }
                uint32_t anc = 1u << lane;
                if (lane) anc |= 1u;
                for (int k = 1; k < cur.n; ++k) {
                    const int kp = __shfl_sync(0xffffffffu, par, k);
                    const uint32_t pa = __shfl_sync(0xffffffffu, anc, kp);
                    if (lane == k) anc |= pa;
                }
                s_anc[buf][lane] = anc;
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_qfull[buf]));
            ++item;
            cur.x += te - cur.t;
            cur.t = te;
            if (cur.t == cur.ntiles && cur.x < cur.end) ca_next(p, cur);
        }
        if (!ok && lane == 0) {
            s_abort = 1;
            if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
        }
    } else {
        // ================================== softmax ==================================
        const int g = (warp >> 2) - 1;                        // group 0: warps 4-7, group 1: warps 8-11
        const int wq = warp & 3;                              // lane quarter of tensor memory
        const int tok = wq * 32 + lane;                       // this thread's token of a tile
        const int dim = D == 128 ? tok : wq * 16 + lane;      // its element of d (64: lanes 0-15)
        const bool has_dim = D == 128 || lane < 16;
        const int w8 = warp - 4;
        const uint32_t t_lane = tmem + ((uint32_t)(wq * 32) << 16);
        uint32_t g0 = 0;                                      // tiles of this CTA before the current item
        int item = 0, merges = 0;
        bool ok = true;
        for (int i = tok; i < N * (D / 32); i += 128) (&s_nan[g][0][0])[i] = 0u;   // its group's barriers order this
        // A wait that gave up leaves `ok` false in its warp only; the warps of a group leave together, at a barrier.
        while (cur.x < cur.end) {
            const int buf = item & 1;
            const int te = (int)min((long long)cur.ntiles, cur.t + (cur.end - cur.x));
            const int nt = te - cur.t;
            const int limit = ca_limit(p, cur.base, cur.n, cur.rt);
            const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
            // positions up to here are seen by every row of the item
            const int seen = p.node_parent ? cur.base : cur.base + i0 + 1;
            float acc[N], lsum[N];
#pragma unroll
            for (int r = 0; r < N; ++r) acc[r] = lsum[r] = 0.f;
            float m_run[(N + 31) / 32];                       // running maxima of rows lane, lane + 32
#pragma unroll
            for (int i = 0; i < (N + 31) / 32; ++i) m_run[i] = -INFINITY;
            bool nan_seen = false;

            for (int t = cur.t + (int)((g - g0) & 1u); t < te; t += 2) {
                const uint32_t k = g0 + (uint32_t)(t - cur.t);   // running tile number
                const uint32_t par = (k >> 1) & 1;
                const uint32_t vslot = (2 * k + 1) % SLOTS;
                if (ok) ok = mbar_wait_warp(smem_u32(&b_s[g]), par) &&
                             mbar_wait_warp(smem_u32(&b_full[vslot]), ((2 * k + 1) / SLOTS) & 1) &&
                             !__any_sync(0xffffffffu, s_abort);
                if (ok && t < cur.t + 2)         // constants of the item, written by the query warps
                    ok = mbar_wait_warp(smem_u32(&b_qfull[buf]), (uint32_t)((item >> 1) & 1));
                const int pos = t * kCaTile + tok;
                const bool masked = (t + 1) * kCaTile > seen;
                unsigned long long vis = ~0ull;               // rows that see this thread's token
                float ks = 0.f, lsv = 0.f, isv = 0.f;
                if (ok) {
                    tc_fence_after();
                    if (masked) {
                        if (pos >= limit) vis = 0ull;
                        else if (!p.node_parent) {
                            const long long r0 = (long long)(pos - cur.base - i0) * p.G;
                            vis = r0 <= 0 ? ~0ull : r0 < 64 ? ~0ull << r0 : 0ull;
                        } else if (pos >= cur.base) {
                            vis = 0ull;
                            for (int i = 0; i * p.G < rows; ++i)
                                if ((s_anc[buf][i0 + i] >> (pos - cur.base)) & 1u) vis |= (~0ull >> (64 - p.G)) << (i * p.G);
                        }
                    }
                    if (vis) {
                        const float* sc = s_scale[k % kCaScaleRing][tok >> p.bt_log2];
                        const float sv = fmaxf(sc[1], 5.421010862e-20f);    // 2^-64
                        ks = sc[0];
                        lsv = __log2f(sv);
                        isv = 1.f / sv;
                    }
                    // pass 1: maxima over the tile's tokens
#pragma unroll
                    for (int c = 0; c < N; c += 16) {
                        float v[16];
                        ca_ld16(t_lane + g * N + c, v);
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float4 cc = *reinterpret_cast<const float4*>(&s_c[buf][c + i]);
                            float a[4] = {fmaf(v[i] * ks, cc.x, lsv), fmaf(v[i + 1] * ks, cc.y, lsv),
                                          fmaf(v[i + 2] * ks, cc.z, lsv), fmaf(v[i + 3] * ks, cc.w, lsv)};
                            if (masked)
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    if (!((vis >> (c + i + e)) & 1ull)) a[e] = -INFINITY;
                            const float4 mx = make_float4(ca_warp_max(a[0]), ca_warp_max(a[1]), ca_warp_max(a[2]), ca_warp_max(a[3]));
                            if (lane == 0) *reinterpret_cast<float4*>(&s_red[g][wq][c + i]) = mx;
                        }
                    }
                    // a masked tile: codes of V that a row must not see may be anything, and 0 * NaN is NaN
                    if (masked && vis != ~0ull) {
                        const unsigned long long all = rows >= 64 ? ~0ull : (1ull << rows) - 1ull;
                        if ((vis & all) != all) {
                            unsigned char* vt = smem + vslot * L::kTileBytes;
#pragma unroll
                            for (int c = 0; c < D / 16; ++c) {
                                uint4* q = reinterpret_cast<uint4*>(vt + (D == 128 ? tok * 128 + ((c ^ (tok & 7)) << 4)
                                                                                   : tok * 64 + ((c ^ ((tok >> 1) & 3)) << 4)));
                                uint32_t w[4] = {q->x, q->y, q->z, q->w};
                                bool touched = false;
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const uint32_t bad = (vis & all) ? __vcmpeq4(w[e] & 0x7f7f7f7fu, 0x7f7f7f7fu) : 0xffffffffu;
                                    if (bad) {
                                        touched = true;
                                        w[e] &= ~bad;
                                        if (vis & all) {      // the rows that do see it get their NaN at the end
                                            nan_seen = true;
                                            for (int r = 0; r < rows; ++r)
                                                if ((vis >> r) & 1ull)
                                                    for (int y = 0; y < 4; ++y)
                                                        if ((bad >> (8 * y)) & 1u) {
                                                            const int dd = c * 16 + e * 4 + y;
                                                            atomicOr(&s_nan[g][r][dd >> 5], 1u << (dd & 31));
                                                        }
                                        }
                                    }
                                }
                                if (touched) *q = make_uint4(w[0], w[1], w[2], w[3]);
                            }
                        }
                    }
                }
                if (ca_bar_any(1 + g, 128, !ok)) { ok = false; break; }
                // maxima of the four warps; factors of this tile, for this warp's rows
#pragma unroll
                for (int i = 0; i < (N + 31) / 32; ++i) {
                    const int r = i * 32 + lane;
                    if (r < N) {
                        const float mt = fmaxf(fmaxf(s_red[g][0][r], s_red[g][1][r]), fmaxf(s_red[g][2][r], s_red[g][3][r]));
                        const float mn = fmaxf(m_run[i], mt);
                        s_m[w8][r] = mt == -INFINITY ? 0.f : mt;
                        s_ab[w8][r] = mn == -INFINITY ? make_float2(1.f, 0.f)
                                                      : make_float2(ex2(m_run[i] - mn), ex2(mt - mn) * 0.00390625f);
                        m_run[i] = mn;
                    }
                }
                __syncwarp();
                // pass 2: probabilities, their sums, and the two e4m3 terms
                unsigned char* sp = s_p + g * 2 * L::kPBytes + (tok >> 3) * 128 + (tok & 7) * 16;
                const float lsv8 = lsv + 8.f;
#pragma unroll
                for (int c = 0; c < N; c += 16) {
                    float v[16];
                    ca_ld16(t_lane + g * N + c, v);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const float4 cc = *reinterpret_cast<const float4*>(&s_c[buf][c + i]);
                        const float4 mm = *reinterpret_cast<const float4*>(&s_m[w8][c + i]);
                        const float4 ab0 = *reinterpret_cast<const float4*>(&s_ab[w8][c + i]);
                        const float4 ab1 = *reinterpret_cast<const float4*>(&s_ab[w8][c + i + 2]);
                        float a[4] = {fmaf(v[i] * ks, cc.x, lsv8 - mm.x), fmaf(v[i + 1] * ks, cc.y, lsv8 - mm.y),
                                      fmaf(v[i + 2] * ks, cc.z, lsv8 - mm.z), fmaf(v[i + 3] * ks, cc.w, lsv8 - mm.w)};
                        if (masked)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (!((vis >> (c + i + e)) & 1ull)) a[e] = -INFINITY;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[i + e] = ex2(a[e]);
                        lsum[c + i] = fmaf(v[i] * isv, ab0.y, lsum[c + i] * ab0.x);
                        lsum[c + i + 1] = fmaf(v[i + 1] * isv, ab0.w, lsum[c + i + 1] * ab0.z);
                        lsum[c + i + 2] = fmaf(v[i + 2] * isv, ab1.y, lsum[c + i + 2] * ab1.x);
                        lsum[c + i + 3] = fmaf(v[i + 3] * isv, ab1.w, lsum[c + i + 3] * ab1.z);
                    }
                    uint32_t hi[4], lo[4];
                    ca_split16(v, hi, lo);
                    *reinterpret_cast<uint4*>(sp + (c >> 4) * 2048) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *reinterpret_cast<uint4*>(sp + (c >> 4) * 2048 + L::kPBytes) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_p[g]));
                // this tile's O^T joins the accumulator
                ok = mbar_wait_warp(smem_u32(&b_o[g]), par);
                if (ok) {
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < N; c += 16) {
                        float v[16];
                        ca_ld16(t_lane + 2 * N + g * N + c, v);
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            const float4 ab = *reinterpret_cast<const float4*>(&s_ab[w8][c + i]);
                            acc[c + i] = fmaf(v[i], ab.y, acc[c + i] * ab.x);
                            acc[c + i + 1] = fmaf(v[i + 1], ab.w, acc[c + i + 1] * ab.z);
                        }
                    }
                    tc_fence_before();
                }
                __syncwarp();
            }

            // ---- end of the item (or of this CTA's part of it) ----
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_qempty[buf]));   // its constants have been read
            const int lead = (int)(g0 & 1);                   // the group of its first tile writes the result
            const bool takes_part = g == lead || nt > 1;
            if (takes_part) {
                // sums over the tokens: over the lanes, then over the warps
#pragma unroll
                for (int r = 0; r < N; ++r) {
                    const float s = warp_sum(lsum[r]);
                    if (lane == 0) s_red[g][wq][r] = s;
                }
                if (ca_bar_any(1 + g, 128, !ok)) { ok = false; break; }
                float l_run[(N + 31) / 32];
#pragma unroll
                for (int i = 0; i < (N + 31) / 32; ++i) {
                    const int r = i * 32 + lane;
                    l_run[i] = r < N ? (s_red[g][0][r] + s_red[g][1][r]) + (s_red[g][2][r] + s_red[g][3][r]) : 0.f;
                }
                if (ca_bar_any(1 + g, 128, nan_seen)) {
                    if (has_dim)
#pragma unroll
                        for (int r = 0; r < N; ++r)
                            if ((s_nan[g][r][dim >> 5] >> (dim & 31)) & 1u) acc[r] = __int_as_float(0x7fc00000);
                    ca_bar_any(1 + g, 128, false);
                    for (int i = tok; i < N * (D / 32); i += 128) (&s_nan[g][0][0])[i] = 0u;
                    ca_bar_any(1 + g, 128, false);
                }
                if (g != lead) {
                    ok = merges == 0 || mbar_wait_warp(smem_u32(&b_mempty), (uint32_t)((merges - 1) & 1));
                    if (ok) {
                        if (has_dim)
#pragma unroll
                            for (int r = 0; r < N; ++r) s_merge[r * D + dim] = acc[r];
                        if (wq == 0)
#pragma unroll
                            for (int i = 0; i < (N + 31) / 32; ++i)
                                if (i * 32 + lane < N) s_mml[i * 32 + lane] = make_float2(m_run[i], l_run[i]);
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&b_mfull));
                    }
                } else {
                    if (nt > 1) {
                        ok = mbar_wait_warp(smem_u32(&b_mfull), (uint32_t)(merges & 1));
                        if (ok) {
#pragma unroll
                            for (int i = 0; i < (N + 31) / 32; ++i) {
                                const int r = i * 32 + lane;
                                if (r < N) {
                                    const float2 o = s_mml[r];
                                    const float mn = fmaxf(m_run[i], o.x);
                                    const float fa = m_run[i] == -INFINITY ? 0.f : ex2(m_run[i] - mn);
                                    const float fb = o.x == -INFINITY ? 0.f : ex2(o.x - mn);
                                    s_ab[w8][r] = make_float2(fa, fb);
                                    l_run[i] = l_run[i] * fa + o.y * fb;
                                    m_run[i] = mn;
                                }
                            }
                            __syncwarp();
                            if (has_dim)
#pragma unroll
                                for (int r = 0; r < N; ++r) {
                                    const float2 ab = s_ab[w8][r];
                                    acc[r] = acc[r] * ab.x + s_merge[r * D + dim] * ab.y;
                                }
                            __syncwarp();
                            if (lane == 0) mbar_arrive(smem_u32(&b_mempty));
                        }
                    }
                    bool write = ok;
                    if (nt < cur.ntiles) {
                        // part of an item: leave it in the workspace; the CTA that completes the item joins the parts
                        const long long xi = cur.x - cur.t;    // the item's first tile over all work
                        const int c_first = (int)(((xi + 1) * grid - 1) / work);
                        const int c_last = (int)(((xi + cur.ntiles) * grid - 1) / work);
                        float* part = p.partial + ((size_t)blockIdx.x * 2 + (cur.t == 0 ? 1 : 0)) * L::kPiece;
                        if (has_dim)
#pragma unroll
                            for (int r = 0; r < N; ++r)
                                if (r < rows) part[r * D + dim] = acc[r];
                        if (wq == 0)
#pragma unroll
                            for (int i = 0; i < (N + 31) / 32; ++i)
                                if (i * 32 + lane < N) {
                                    part[N * D + i * 32 + lane] = m_run[i];
                                    part[N * D + N + i * 32 + lane] = l_run[i];
                                }
                        __threadfence();
                        if (ca_bar_any(1 + g, 128, !ok)) { ok = false; break; }
                        if (tid == 128 + g * 128) {
                            const uint32_t old = atomicAdd(p.ticket + c_first, 1u);
                            const bool last = old == (uint32_t)(c_last - c_first);
                            if (last) p.ticket[c_first] = 0u;
                            s_last[g] = last;
                        }
                        ca_bar_any(1 + g, 128, false);
                        write = s_last[g] != 0;               // written again only after further barriers of the group
                        if (write) {
                            __threadfence();
                            // maxima and sums over the parts, for rows lane, lane + 32
#pragma unroll
                            for (int i = 0; i < (N + 31) / 32; ++i) {
                                const int r = i * 32 + lane;
                                float mm = -INFINITY, ll = 0.f;
                                if (r < N)
                                    for (int c = c_first; c <= c_last; ++c) {
                                        const float* q = p.partial + ((size_t)c * 2 + (c == c_first ? 1 : 0)) * L::kPiece + N * D;
                                        const float mc = __ldcg(q + r), lc = __ldcg(q + N + r);
                                        const float mn = fmaxf(mm, mc);
                                        ll = (mm == -INFINITY ? ll * 0.f : ll * ex2(mm - mn)) + (mc == -INFINITY ? lc * 0.f : lc * ex2(mc - mn));
                                        mm = mn;
                                    }
                                m_run[i] = mm;
                                l_run[i] = ll;
                            }
#pragma unroll
                            for (int r = 0; r < N; ++r) acc[r] = 0.f;
                            for (int c = c_first; c <= c_last; ++c) {
                                const float* q = p.partial + ((size_t)c * 2 + (c == c_first ? 1 : 0)) * L::kPiece;
                                __syncwarp();
#pragma unroll
                                for (int i = 0; i < (N + 31) / 32; ++i) {
                                    const int r = i * 32 + lane;
                                    if (r < N) {
                                        const float mc = __ldcg(q + N * D + r);
                                        s_m[w8][r] = mc == -INFINITY ? 0.f : ex2(mc - m_run[i]);
                                    }
                                }
                                __syncwarp();
                                if (has_dim)
#pragma unroll
                                    for (int r = 0; r < N; ++r)
                                        if (r < rows) acc[r] = fmaf(__ldcg(q + r * D + dim), s_m[w8][r], acc[r]);
                            }
                        }
                    }
                    if (write) {
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < (N + 31) / 32; ++i) {
                            const int r = i * 32 + lane;
                            if (r < N) s_m[w8][r] = l_run[i] == 0.f ? 0.f : 1.f / l_run[i];   // nothing seen: zeros
                        }
                        __syncwarp();
                        if (has_dim) {
                            __nv_bfloat16* o = p.out + (long long)(cur.q0 + i0) * p.o_st + (long long)cur.h * p.G * p.o_sh + dim;
                            int hh = 0;
#pragma unroll
                            for (int r = 0; r < N; ++r)
                                if (r < rows) {
                                    o[hh * p.o_sh] = __float2bfloat16_rn(acc[r] * s_m[w8][r]);
                                    if (++hh == p.G) { hh = 0; o += p.o_st; }
                                }
                        }
                        __syncwarp();
                    }
                }
            }
            if (nt > 1) ++merges;
            ++item;
            g0 += nt;
            cur.x += nt;
            cur.t = te;
            if (cur.t == cur.ntiles && cur.x < cur.end) ca_next(p, cur);
        }
        if (!ok && lane == 0) {
            s_abort = 1;
            if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
        }
    }

    // ---- all roles meet; tensor memory goes back ----
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tc_free(tmem, L::kTmemCols);
    }
}

static std::atomic<bool> g_ca_attr[8][64];

// Codes [n_blocks * Hkv, bt, d] as a tensor of bytes; a box is one block of one head, swizzled by its row length.
static bool ca_map(CUtensorMap* tm, const void* base, int n_blocks, int Hkv, int bt, int d) {
    EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)bt, (cuuint64_t)n_blocks * Hkv};
    const cuuint64_t strides[2] = {(cuuint64_t)d, (cuuint64_t)d * bt};
    const cuuint32_t box[3] = {(cuuint32_t)d, (cuuint32_t)bt, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<void*>(base), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, d == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int N, int D>
static bs_status launch_ca(const CUtensorMap* tm, const CacheAttnParams& p, cudaStream_t st) {
    using L = CaLayout<N, D>;
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) dev = 0;
    auto kern = cache_attention_kernel<N, D>;
    constexpr int variant = (N / 16 - 1) * 2 + (D == 128);
    if (!g_ca_attr[variant][dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynamic) != cudaSuccess)
            return cuda_status(cudaGetLastError());
        g_ca_attr[variant][dev] = true;
    }
    return cuda_status(launch_pdl(kern, sm_count(), kCaThreads, L::kDynamic, st, tm[0], tm[1], p));
}

static size_t ca_ticket_bytes() { return align_up(sizeof(uint32_t) * (size_t)sm_count(), 256); }

}  // namespace bs

using namespace bs;

extern "C" size_t bs_cache_workspace_bytes(int Hq, int Hkv, int d) {
    if (Hkv < 1 || Hq < Hkv || Hq % Hkv || Hq / Hkv > 64 || (d != 64 && d != 128)) return 0;
    return ca_ticket_bytes() + align_up(sizeof(float) * 2 * (size_t)sm_count() * (64 * d + 2 * 64), 256);
}

extern "C" bs_status bs_cache_attention(const void* q, long long q_stride_t, long long q_stride_h, const int32_t* cu_new,
                                        const int32_t* kv_len, const int32_t* block_table, int max_blocks,
                                        const int32_t* node_parent, int Nmax, const void* k_cache, const float* k_scale,
                                        const void* v_cache, const float* v_scale, int n_blocks, int block_tokens, int B,
                                        int T, int Hq, int Hkv, int d, int max_new, float softmax_scale, void* out,
                                        long long out_stride_t, long long out_stride_h, int32_t* status, void* workspace,
                                        size_t workspace_bytes, void* stream) {
    if (B < 1 || T < 1 || Hq < 1 || Hkv < 1 || d < 1 || max_blocks < 1 || n_blocks < 1 || block_tokens < 1 || max_new < 1 ||
        Nmax < 0 || !isfinite(softmax_scale))
        return BS_ERR_INVALID_ARG;
    if (!q || !cu_new || !kv_len || !block_table || !k_cache || !k_scale || !v_cache || !v_scale || !out || !workspace)
        return BS_ERR_INVALID_ARG;
    if (Hq % Hkv) return BS_ERR_INVALID_ARG;
    if (B > BS_MAX_BATCH || max_blocks > BS_MAX_SEQ_BLOCKS || Hq / Hkv > 64 || (node_parent && Nmax > BS_MAX_GAMMA) ||
        !cache_geometry_ok(Hkv, d, n_blocks, block_tokens))
        return BS_ERR_UNSUPPORTED;
    if ((q_stride_t % 8) || (q_stride_h % 8) || (out_stride_t % 8) || (out_stride_h % 8)) return BS_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(k_cache) |
         reinterpret_cast<uintptr_t>(v_cache)) & 15)
        return BS_ERR_INVALID_ARG;
    if (workspace_bytes < bs_cache_workspace_bytes(Hq, Hkv, d) || (reinterpret_cast<uintptr_t>(workspace) & 255))
        return BS_ERR_WORKSPACE;
    CacheAttnParams p;
    p.q = static_cast<const __nv_bfloat16*>(q); p.out = static_cast<__nv_bfloat16*>(out);
    p.q_st = q_stride_t; p.q_sh = q_stride_h; p.o_st = out_stride_t; p.o_sh = out_stride_h;
    p.cu_new = cu_new; p.kv_len = kv_len; p.block_table = block_table; p.node_parent = node_parent;
    p.k_scale = k_scale; p.v_scale = v_scale; p.status = status;
    p.ticket = static_cast<uint32_t*>(workspace);
    p.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + ca_ticket_bytes());
    p.scale_log2 = softmax_scale * kLog2e;
    p.B = B; p.T = T; p.W = max_blocks; p.Nmax = Nmax; p.Hq = Hq; p.Hkv = Hkv; p.G = Hq / Hkv;
    p.n_blocks = n_blocks;
    p.bt_log2 = 4;
    while ((1 << p.bt_log2) < block_tokens) ++p.bt_log2;
    CUtensorMap tm[2];
    if (!ca_map(&tm[0], k_cache, n_blocks, Hkv, block_tokens, d) || !ca_map(&tm[1], v_cache, n_blocks, Hkv, block_tokens, d))
        return BS_ERR_CUDA;
    // the narrowest tile that takes all rows of a sequence's key head at once, so that its cache is read once
    const long long rows = (long long)max_new * p.G;
    const int N = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 48 ? 48 : 64;
    p.TQ = N / p.G;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (d == 128)
        return N == 16 ? launch_ca<16, 128>(tm, p, st) : N == 32 ? launch_ca<32, 128>(tm, p, st)
             : N == 48 ? launch_ca<48, 128>(tm, p, st) : launch_ca<64, 128>(tm, p, st);
    return N == 16 ? launch_ca<16, 64>(tm, p, st) : N == 32 ? launch_ca<32, 64>(tm, p, st)
         : N == 48 ? launch_ca<48, 64>(tm, p, st) : launch_ca<64, 64>(tm, p, st);
}
