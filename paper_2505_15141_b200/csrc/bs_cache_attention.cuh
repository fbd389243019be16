// Shared parts of the two attention kernels over the e4m3 cache (bs_cache_attention.cu, bs_cache_attention_rows.cu): the
// work list, the copies, the queries, tensor-core and tensor-memory instructions.
#pragma once

#include "bs_cache_common.cuh"
#include "bs_pipeline.cuh"
#include "bs_tensor.cuh"

#include <atomic>

namespace bs {

constexpr int kCaTile = 128;                   // tokens of a tile
constexpr int kCaSmem = 230400;                // of 232448 bytes a CTA may use
constexpr int kCaScaleRing = 8;                // tiles whose scales are kept; more than the tiles in flight
constexpr int kCaMaxPages = 8;                 // blocks of 16 tokens in a tile
constexpr int kCaMaxRows = 128;                // rows of an item, at most
constexpr float kCaMinScaleV = 5.421010862e-20f;   // 2^-64, the smallest scale of V that the header allows
// What an item costs besides its tiles (queries, joining, results), in tiles, when the work is cut into shares.  Measured with
// 1, 2, 4 and 6: prompt pieces of 1 to 36 tiles 186, 152, 141, 139 us, trees on 1 to 33 tiles 177, 161, 153, 149 us, long
// items the same.
constexpr int kCaItemCost = 4;

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
    volatile uint32_t* abort;                  // [1] set when a wait gave up, cleared with the workspace
    float scale_log2;                          // softmax_scale * log2(e)
    int B, T, W, Nmax, Hkv, G, TQ;             // TQ: new tokens of an item, N / G
    int bt_log2, n_blocks;
};

// The piece of the work a role is at.
struct CaCursor {
    int b, h, rt, nrt;                         // item
    int n, base, q0;                           // its sequence: new tokens, position of the first, its row
    int t, ntiles;                             // next tile, tiles of the item
    // The work is a line: every item takes kCaItemCost places and then one for each tile.
    long long x, end;                          // place of the next tile; end of this CTA's share
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
#pragma unroll 1
    for (int rt = 0; rt * p.TQ < n; ++rt) w += kCaItemCost + ca_tiles(ca_limit(p, base, n, rt));
    return w;
}
__device__ __forceinline__ void ca_item(const CacheAttnParams& p, CaCursor& c) {
    c.ntiles = ca_tiles(ca_limit(p, c.base, c.n, c.rt));
}
// To the next item (c.t = 0).
__device__ __forceinline__ void ca_next(const CacheAttnParams& p, CaCursor& c) {
    c.t = 0;
    c.x += kCaItemCost;
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
// MMA and commit are executed by the whole converged warp under the predicate of one elected thread: issued from a branch
// that a single thread took they cost 46 cycles each and 260 for the first result, this way 39 to 48 (N = 16 to 64) and 150.
__device__ __forceinline__ uint32_t ca_elect() {
    uint32_t r;
    asm volatile("{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\tselp.u32 %0, 1, 0, e;\n\t}" : "=r"(r));
    return r;
}
__device__ __forceinline__ void ca_mma(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t elected) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 e, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(elected) : "memory");
}
__device__ __forceinline__ void ca_commit(uint32_t bar, uint32_t elected) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %1, 0;\n\t"
        "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
        ::"r"(bar), "r"(elected) : "memory");
}
__device__ __forceinline__ void ca_tma(uint32_t dst, const CUtensorMap* tm, int block_head, uint32_t bar, uint32_t elected) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %6, 0;\n\t"
        "@e cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}"
        ::"r"(dst), "l"(tm), "r"(0), "r"(0), "r"(block_head), "r"(bar), "r"(elected) : "memory");
}
// 16 columns of tensor memory, thread = lane; the values may be used after ca_ld16_wait.
__device__ __forceinline__ void ca_ld16(uint32_t taddr, float (&u)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=f"(u[0]), "=f"(u[1]), "=f"(u[2]), "=f"(u[3]), "=f"(u[4]), "=f"(u[5]), "=f"(u[6]), "=f"(u[7]),
          "=f"(u[8]), "=f"(u[9]), "=f"(u[10]), "=f"(u[11]), "=f"(u[12]), "=f"(u[13]), "=f"(u[14]), "=f"(u[15])
        : "r"(taddr));
}
__device__ __forceinline__ void ca_ld16_wait(float (&u)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(u[0]), "+f"(u[1]), "+f"(u[2]), "+f"(u[3]), "+f"(u[4]), "+f"(u[5]), "+f"(u[6]), "+f"(u[7]),
                   "+f"(u[8]), "+f"(u[9]), "+f"(u[10]), "+f"(u[11]), "+f"(u[12]), "+f"(u[13]), "+f"(u[14]), "+f"(u[15]));
}
__device__ __forceinline__ float4 lds4(const float* p) {
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(smem_u32(p)));
    return v;
}
__device__ __forceinline__ float ca_warp_max(float v) {        // NaN only if every lane has one
    float r;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
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
// Four values as hi + lo, each four e4m3.  They pass through fp16 (2^-12), where hi and the remainder are exact.
__device__ __forceinline__ void ca_split4(float a, float b, float c, float d, uint32_t& hi, uint32_t& lo) {
    asm("{\n\t.reg .b16 p, q;\n\t.reg .b32 x, y, u, v;\n\t"
        "cvt.rn.f16x2.f32 x, %3, %2;\n\t"
        "cvt.rn.f16x2.f32 y, %5, %4;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 p, x;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 q, y;\n\t"
        "mov.b32 %0, {p, q};\n\t"
        "cvt.rn.f16x2.e4m3x2 u, p;\n\t"
        "cvt.rn.f16x2.e4m3x2 v, q;\n\t"
        "sub.rn.f16x2 x, x, u;\n\t"
        "sub.rn.f16x2 y, y, v;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 p, x;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 q, y;\n\t"
        "mov.b32 %1, {p, q};\n\t}"
        : "=r"(hi), "=r"(lo) : "f"(a), "f"(b), "f"(c), "f"(d));
}

__device__ __forceinline__ void ca_st16(uint32_t taddr, const float (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
          "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "r"(taddr));
}
__device__ __forceinline__ void ca_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 16 columns of an MMA result whose two terms stand `n` columns apart.
__device__ __forceinline__ void ca_result16(uint32_t taddr, int n, float (&x)[16]) {
    float w[16];
    ca_ld16(taddr, x);
    ca_ld16(taddr + n, w);
    ca_ld16_wait(x);
    ca_ld16_wait(w);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] += w[i];
}
// Bounded wait of a converged warp.  The loop is out of line: the kernel waits in many places, and its instructions have to
// stay in the instruction cache.
// A try may suspend the warp for a millisecond: polling would take issue slots from the warps that work.
static __device__ __noinline__ bool ca_wait_loop(uint32_t bar, uint32_t parity) {
    const long long t0 = clock64();
    for (;;) {
        uint32_t ok;
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000000u) : "memory");
        if (ok) return true;
        if (clock64() - t0 > kWaitCycles) return false;
    }
}
__device__ __forceinline__ bool ca_wait(uint32_t bar, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) || __all_sync(0xffffffffu, ca_wait_loop(bar, parity));
}


// Token `tok` of a tile of V that some rows must not see: its codes may be anything, and 0 * NaN is NaN.  A token nobody
// sees becomes zero.  In one that some see, NaN codes become zero and the results they belong to are marked; true if
// there were any.  Row r sees it if r >= first_row (chains), or if bit `bit` of its node's ancestors is set (trees).
// Once per item at most, so kept out of the way of the loop's instructions.
struct CaWho {
    const uint32_t* anc;                       // ancestors of the item's first node, NULL: chain
    int bit, first_row, rows, G;
    bool any;
};
template <int D>
__device__ __noinline__ bool ca_clean_v(unsigned char* tile, int tok, const CaWho who, uint32_t* marks) {
    bool found = false;
#pragma unroll 1
    for (int c = 0; c < D / 16; ++c) {
        uint4* q = reinterpret_cast<uint4*>(tile + (D == 128 ? tok * 128 + ((c ^ (tok & 7)) << 4) : tok * 64 + ((c ^ ((tok >> 1) & 3)) << 4)));
        if (!who.any) {
            *q = make_uint4(0u, 0u, 0u, 0u);
            continue;
        }
        const uint4 v = *q;
        const uint32_t bx = __vcmpeq4(v.x & 0x7f7f7f7fu, 0x7f7f7f7fu), by = __vcmpeq4(v.y & 0x7f7f7f7fu, 0x7f7f7f7fu);
        const uint32_t bz = __vcmpeq4(v.z & 0x7f7f7f7fu, 0x7f7f7f7fu), bw = __vcmpeq4(v.w & 0x7f7f7f7fu, 0x7f7f7f7fu);
        if (bx | by | bz | bw) {
            found = true;
            *q = make_uint4(v.x & ~bx, v.y & ~by, v.z & ~bz, v.w & ~bw);
            uint32_t bits = 0u;                               // of 16 elements
#pragma unroll 1
            for (int y = 0; y < 16; ++y) {
                const uint32_t w = y < 4 ? bx : y < 8 ? by : y < 12 ? bz : bw;
                bits |= ((w >> (8 * (y & 3))) & 1u) << y;
            }
            bits <<= (c & 1) * 16;
#pragma unroll 1
            for (int r = 0; r < who.rows; ++r)
                if (who.anc ? (who.anc[r / who.G] >> who.bit) & 1u : r >= who.first_row) atomicOr(marks + r * (D / 32) + (c >> 1), bits);
        }
    }
    return found;
}

// ---- this CTA's share of the work ----
struct CaShare {                               // shared memory
    long long w[32];
    int items[32];
    long long off;
    int b;
};
struct CaPart {
    long long work, grid;                      // length of the line of work, CTAs that have a share of it
};
// All threads of the CTA, after the grid dependency; ends with a barrier of all of them.
template <int THREADS>
__device__ __forceinline__ CaPart ca_share(const CacheAttnParams& p, CaShare& sh, CaCursor& cur) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) sh.b = -1;
    const int per = (p.B + THREADS - 1) / THREADS;
    long long mine = 0;
    int items = 0;
#pragma unroll 1
    for (int b = tid * per; b < min(p.B, (tid + 1) * per); ++b) {
        int n, base, q0;
        if (!ca_seq(p, b, n, base, q0) && p.status && blockIdx.x == 0) atomicOr(p.status + b, BS_DEV_BAD_LENGTH);
        mine += p.Hkv * ca_head_work(p, n, base);
        items += p.Hkv * ((n + p.TQ - 1) / p.TQ);
    }
    items = __reduce_add_sync(0xffffffffu, items);
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
    }
    if (lane == 31) {
        sh.w[warp] = incl;
        sh.items[warp] = items;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    long long work = 0, before = 0, all = 0;
#pragma unroll 1
    for (int w = 0; w < THREADS / 32; ++w) {
        if (w < warp) before += sh.w[w];
        work += sh.w[w];
        all += sh.items[w];
    }
    // Little work: where items are short, shares of a whole one of two tiles (they are worked on side by side).  Long ones
    // are cut; a part takes about 0.3 of a tile's time to join, so least + 0.3 tiles / least is what a CTA waits for.  (One
    // figure for all tiles, from two long contexts with 20 rows and from one key head over 20000 tokens; parts of 128 rows are four
    // times as large.)
    const float tiles = all ? (float)(work - kCaItemCost * all) / (float)all : 0.f;   // of an item
    const int least = tiles <= 8.f ? kCaItemCost + 2 : max(2, (int)sqrtf(0.3f * tiles));
    const long long grid = min((work + least - 1) / least, (long long)gridDim.x);
    const long long x_lo = grid ? blockIdx.x * work / grid : 0, x_hi = grid && blockIdx.x < grid ? (blockIdx.x + 1) * work / grid : 0;
    const long long from = before + incl - mine;
    if (x_lo < x_hi && x_lo >= from && x_lo < from + mine) {
        long long off = x_lo - from;
#pragma unroll 1
        for (int b = tid * per; b < min(p.B, (tid + 1) * per); ++b) {
            int n, base, q0;
            ca_seq(p, b, n, base, q0);
            const long long w = p.Hkv * ca_head_work(p, n, base);
            if (off < w) {
                sh.b = b;
                sh.off = off;
                break;
            }
            off -= w;
        }
    }
    __syncthreads();
    cur.x = x_lo;
    cur.end = x_lo < x_hi ? x_hi : x_lo;
    cur.b = sh.b;
    if (cur.x < cur.end) {
        ca_seq(p, cur.b, cur.n, cur.base, cur.q0);
        cur.nrt = (cur.n + p.TQ - 1) / p.TQ;
        const long long hw = ca_head_work(p, cur.n, cur.base);
        cur.h = (int)(sh.off / hw);
        long long off = sh.off - cur.h * hw;
        cur.rt = 0;
        ca_item(p, cur);
        while (off >= kCaItemCost + cur.ntiles) {
            off -= kCaItemCost + cur.ntiles;
            ++cur.rt;
            ca_item(p, cur);
        }
        cur.t = (int)max(0ll, off - kCaItemCost);
        cur.x += kCaItemCost + cur.t - off;                   // behind the item's own places
    }
    return CaPart{work, grid};
}
// The tiles of a cursor's item that are in this CTA's share.
__device__ __forceinline__ int ca_tiles_here(const CaCursor& c) { return (int)min((long long)(c.ntiles - c.t), c.end - c.x); }
__device__ __forceinline__ void ca_advance(const CacheAttnParams& p, CaCursor& c, int tiles) {
    c.x += tiles;
    c.t += tiles;
    if (c.t == c.ntiles && c.x < c.end) ca_next(p, c);
}
__device__ __forceinline__ void ca_give_up(const CacheAttnParams& p, volatile int* s_abort) {   // one thread
    *s_abort = 1;
    *p.abort = 1u;
    if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
}

// ---- TMA producer: one warp for the tiles of K (kv = 0), one for those of V ----
// One warp could not issue the copies of 16-token blocks fast enough (106 to 133 cycles each: 4.3 TB/s measured for one
// warp, 6.5 TB/s for two).  The block numbers of up to 32 blocks are fetched one group ahead, across items, and the scales
// of a tile come with cp.async and a barrier of their own (the producer of K): nothing here waits for memory.
template <int D, uint32_t RING>
__device__ __forceinline__ void ca_produce(const CacheAttnParams& p, CaCursor cur, int kv, const CUtensorMap* tm, unsigned char* ring,
                                           unsigned long long* b_full, unsigned long long* b_empty, unsigned long long* b_scale,
                                           float (*s_scale)[kCaMaxPages][2], uint32_t* s_tiles, volatile int* s_abort) {
    const int lane = threadIdx.x & 31;
    const uint32_t elected = ca_elect();
    uint32_t slot = 0, ph = 0, tile = 0;
    bool ok = true;
    const uint32_t page_bytes = (uint32_t)D << p.bt_log2;
    const int ppt_log2 = 7 - p.bt_log2;                       // blocks of a tile
    auto group_tiles = [&](const CaCursor& c) { return min(32 >> ppt_log2, ca_tiles_here(c)); };
    auto fetch = [&](const CaCursor& c, int tiles) {          // this lane's block of the group
        const int limit = ca_limit(p, c.base, c.n, c.rt);
        const int pages = limit > 0 ? (limit + (1 << p.bt_log2) - 1) >> p.bt_log2 : 0;
        const int page = (c.t << ppt_log2) + lane;
        return lane < tiles << ppt_log2 && page < pages ? __ldg(p.block_table + (size_t)c.b * p.W + page) : 0;
    };
    int n_tiles = cur.x < cur.end ? group_tiles(cur) : 0;
    int ids = cur.x < cur.end ? fetch(cur, n_tiles) : 0;
#pragma unroll 1
    while (cur.x < cur.end && ok) {
        CaCursor nxt = cur;
        ca_advance(p, nxt, n_tiles);
        const int next_tiles = nxt.x < nxt.end ? group_tiles(nxt) : 0;
        const int next_ids = nxt.x < nxt.end ? fetch(nxt, next_tiles) : 0;
        if (ids < 0 || ids >= p.n_blocks) {
            if (p.status) atomicOr(p.status + cur.b, BS_DEV_BAD_BLOCK);
            ids = 0;
        }
        const int limit = ca_limit(p, cur.base, cur.n, cur.rt);
#pragma unroll 1
        for (int j = 0; j < n_tiles && ok; ++j, ++tile) {
            const int valid = min(kCaTile, limit - (cur.t + j) * kCaTile);
            const int pages = valid > 0 ? (valid + (1 << p.bt_log2) - 1) >> p.bt_log2 : 0;
            if (!ca_wait(smem_u32(b_empty + slot), ph ^ 1u) || __any_sync(0xffffffffu, *s_abort)) { ok = false; break; }
            const uint32_t bar = smem_u32(b_full + slot);
            if (lane == 0) mbar_arrive_expect_tx(bar, pages * page_bytes);
            __syncwarp();
            uint32_t dst = smem_u32(ring + slot * (kCaTile * D));
#pragma unroll 1
            for (int i = 0; i < pages; ++i, dst += page_bytes)
                ca_tma(dst, tm, __shfl_sync(0xffffffffu, ids, (j << ppt_log2) + i) * p.Hkv + cur.h, bar, elected);
            if (!kv) {
                const int blk = __shfl_sync(0xffffffffu, ids, ((j << ppt_log2) + lane) & 31);
                if (lane < pages) {
                    // S of two tiles at most is ahead of the softmax, so the entry of tile - 8 has been read
                    const uint32_t at = smem_u32(s_scale[tile % kCaScaleRing][lane]);
                    const size_t e = (size_t)blk * p.Hkv + cur.h;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at), "l"(p.k_scale + e) : "memory");
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at + 4), "l"(p.v_scale + e) : "memory");
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(b_scale + tile % kCaScaleRing)) : "memory");
            }
            if (++slot == RING) { slot = 0; ph ^= 1u; }
        }
        cur = nxt;
        n_tiles = next_tiles;
        ids = next_ids;
    }
    if (lane == 0) {
        s_tiles[kv] = tile;
        if (!ok) ca_give_up(p, s_abort);
    }
    __syncwarp();
}
// After a wait that gave up, behind the barrier at which all roles meet: nothing is issued any more, and nothing may be left
// in flight that writes this CTA's shared or tensor memory, whichever role it was that gave up.  Every wait is bounded.
template <uint32_t RING>
__device__ __noinline__ void ca_drain(int warp, unsigned long long (*b_full)[RING], const uint32_t* s_tiles, unsigned long long* b_drain) {
    if (warp < 2) {
        const uint32_t tiles = s_tiles[warp];
#pragma unroll 1
        for (uint32_t f = tiles > RING ? tiles - RING : 0u; f < tiles; ++f) ca_wait(smem_u32(&b_full[warp][f % RING]), (f / RING) & 1);
        asm volatile("cp.async.wait_all;" ::: "memory");      // scales
    } else if (warp == 2) {
        ca_commit(smem_u32(b_drain), ca_elect());
        ca_wait(smem_u32(b_drain), 0);
    }
    __syncwarp();
}
template <uint32_t RING>
__device__ __forceinline__ void ca_init_rings(unsigned long long (*b_full)[RING], unsigned long long (*b_empty)[RING],
                                              unsigned long long* b_scale) {
    for (uint32_t s = 0; s < RING; ++s)
        for (int kv = 0; kv < 2; ++kv) {
            mbar_init(smem_u32(&b_full[kv][s]), 1);
            mbar_init(smem_u32(&b_empty[kv][s]), 1);
        }
    for (int s = 0; s < kCaScaleRing; ++s) mbar_init(smem_u32(b_scale + s), 32);   // the producer's lanes
}

// ---- queries, split into e4m3 an item ahead ----
// Buffer i of shared memory: hi, then lo, ROWS x D bytes each, in 8 x 16-byte core matrices.  qt: 0 to THREADS - 1.
// THREADS = 32: a warp of its own, for few rows.  128: the accumulator warps, before the item's first tile; for 64 rows a
// warp of its own took 9 us, which every CTA waited for at its start and at short items.
template <int ROWS, int D, int THREADS>
__device__ __forceinline__ void ca_queries(const CacheAttnParams& p, const CaCursor& cur, int buf, int qt, unsigned char* s_q,
                                           float (*s_c)[ROWS], uint32_t (*s_anc)[32]) {
    constexpr int kLanes = D / 8;                             // lanes of a row
    constexpr int kRows = THREADS / kLanes;                   // rows per pass
    const int lane = qt & 31, sub = qt / kLanes, piece = (qt % kLanes) * 8;
    const int inv_g = (65536 + p.G - 1) / p.G;                // exact for r < 128, G <= 64
    {
        const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
        unsigned char* q_hi = s_q + buf * 2 * (ROWS * D);
        // the loads of a batch of rows first: one by one, each would wait for memory (1400 cycles a pass, measured)
        constexpr int kBatch = ROWS <= kRows ? 1 : ROWS / kRows < 8 ? ROWS / kRows : 8;
#pragma unroll 1
        for (int rb = 0; rb < ROWS; rb += kBatch * kRows) {
            uint4 raw[kBatch];
#pragma unroll
            for (int z = 0; z < kBatch; ++z) {
                const int r = min(rb + z * kRows + sub, rows - 1), i = r * inv_g >> 16;   // r / G
                raw[z] = __ldg(reinterpret_cast<const uint4*>(p.q + (long long)(cur.q0 + i0 + i) * p.q_st +
                                                              (long long)(cur.h * p.G + r - i * p.G) * p.q_sh + piece));
            }
#pragma unroll
            for (int z = 0; z < kBatch; ++z) {
                const int r = rb + z * kRows + sub;
                // the row's largest magnitude, two bf16 at a time: their bits order as whole numbers do
                uint32_t m2 = __vmaxu2(__vmaxu2(raw[z].x & 0x7fff7fffu, raw[z].y & 0x7fff7fffu),
                                       __vmaxu2(raw[z].z & 0x7fff7fffu, raw[z].w & 0x7fff7fffu));
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) m2 = __vmaxu2(m2, __shfl_xor_sync(0xffffffffu, m2, o));
                const uint32_t mx = max(m2 >> 16, m2 & 0xffffu);
                const bool fin = mx < 0x7f80u;                // no infinity, no NaN
                // 2^x brings the row's largest element into [128, 256)
                const int x = mx && fin ? min(7 - ((int)(mx >> 7) - 127), 120) : 0;
                const float up = __uint_as_float((uint32_t)(x + 127) << 23);
                float f[8];
                Elem<__nv_bfloat16>::unpack(raw[z], f);
                uint2 hi, lo;
                ca_split4(f[0] * up, f[1] * up, f[2] * up, f[3] * up, hi.x, lo.x);
                ca_split4(f[4] * up, f[5] * up, f[6] * up, f[7] * up, hi.y, lo.y);
                unsigned char* at = q_hi + (r >> 3) * (8 * D) + (piece >> 4) * 128 + (r & 7) * 16 + (piece & 15);
                *reinterpret_cast<uint2*>(at) = hi;
                *reinterpret_cast<uint2*>(at + ROWS * D) = lo;
                // a row with an infinity or a NaN has no softmax: its scale makes every result NaN.  (Rows behind the item's
                // last repeat it; nobody reads their results.)
                if (piece == 0)
                    s_c[buf][r] = r >= rows ? 0.f : fin ? p.scale_log2 * __uint_as_float((uint32_t)(127 - x) << 23) : __int_as_float(0x7fc00000);
            }
        }
        if (p.node_parent && qt < 32) {            // ancestors-or-self of node `lane`
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
#pragma unroll 1
            for (int k = 1; k < cur.n; ++k) {
                const int kp = __shfl_sync(0xffffffffu, par, k);
                const uint32_t pa = __shfl_sync(0xffffffffu, anc, kp);
                if (lane == k) anc |= pa;
            }
            s_anc[buf][lane] = anc;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
    }
}

// Many rows (bs_cache_attention_rows.cu); tm: K and V; TQ and G are set.
bs_status launch_cache_attention_rows(const CUtensorMap* tm, const CacheAttnParams& p, int rows, int d, cudaStream_t st);

}  // namespace bs
