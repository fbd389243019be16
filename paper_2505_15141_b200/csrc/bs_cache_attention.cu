// bs_cache_attention: attention of the new tokens of a round (a chain or a tree of drafts, or a piece of a prompt)
// over the e4m3 cache.
//
//   out_i = sum_j 2^(t_ij) v_j / sum_j 2^(t_ij),   t_ij = log2(e) softmax_scale q_i . k_j
//
// This file: the entry point, and the kernel for up to 32 rows (new token, query head of the group) of a key head;
// bs_cache_attention_rows.cu has the one for more.  A CTA works on tiles of 128 cached tokens.  Both products run on
// the tensor cores with the cache's codes as they are:
//
//   S^T [128 tokens, N rows] = K [128, d] Q^T     K K-major, as the TMA copy leaves it (swizzled)
//   O^T [d, N rows]          = V^T P^T            V^T is the same tile read M-major; P^T from shared memory, N-major
//
// i.e. the tokens (and then d) are the 128 lanes of the MMA and the rows its N = 16 or 32: a few rows cost no more than
// their share, and no code is ever converted.  The other operand has to be e4m3 as well (kind::f8f6f4): a bf16 query,
// scaled by a power of two so that its row's largest element lies in [128, 256), is the sum of two e4m3 numbers exactly
// (four significant bits, a signed remainder of four more; elements below 2^-9 of the largest lose bits under 2^-17
// of it), and a probability is split the same way (relative error 2^-8 as in bf16).  Their accumulation was measured
// against 64 bits: error 2^-20 of the largest product.  On 200 to 4096 tokens of normal data the splits add 1.0e-4 to 1.6e-4 to a
// result (norm, relative to 64 bits) whose rounding to bf16 adds 1.6e-3.
//
// Scales.  Keys: t_ij = S_ij * (scale of j's block * c_i).  Values: the scale of a token's block joins the exponent:
//   P''_ij = 2^(t_ij + log2 s_j + 8 - m_i),  m_i = max_j (t_ij + log2 s_j) over the tile,
// which uses the e4m3 range up to 256 whatever the scales are; the sum of the probabilities takes P'' / s_j in fp32.
// O^T of every tile is taken from tensor memory and joined in fp32 with the tile's own factor 2^(m_i - m),
// so a token far below the row's running maximum keeps its bits relative to its own tile.
//
// Roles of the 16 warps: 0 and 1 TMA producers of K and V (one producer of both: 4.3 TB/s of 16-byte-row boxes of
// 16-token blocks, two: 6.5), 2 MMA issuer, 3 queries (split into e4m3 one work item ahead), 4-7 accumulator (a thread
// is an element of d), 8-11 and 12-15 two softmax groups that take the tiles in turn, each with its own maximum and
// sum (a thread is a token).  Sums and accumulator stand in tensor memory, and the loops over rows are rolled: the
// roles run side by side and share one instruction cache, and every larger form of them (unrolled rows, a third
// softmax group, accumulators in registers) was slower.
//
// Work.  Item = (sequence, key head, N rows).  All items, in order, a few places and one for each tile, are cut into equal
// contiguous shares, one per CTA, from the lengths on the device; an item that spans several CTAs is joined by the one that
// finishes last, in the order of the shares (the result does not depend on who that is).
//
// Bound by the instructions of the softmax on 16 rows (47 % of issue slots, DRAM 50 % busy: both softmax groups
// and the accumulator are chained within a tile), close to HBM's rate when a row count of 4 leaves little to do.
// 32 query / 8 key heads of 128, caches larger than L2, a call alone on the GPU: 256 sequences of 4096 tokens, 4 rows, 2.15 GB
// in 0.45 ms (4.8 TB/s); 64 sequences, 16 rows, 0.138 ms (3.9 TB/s); 32 rows 0.178 ms; two sequences of 100003 and 131072
// tokens, 20 rows, 0.147 ms (3.2 TB/s); one token on 200 cached ones 9.3 us in a graph.
#include "bs_cache_attention.cuh"

namespace bs {

// Sums of 16 per-lane values over the lanes of a warp: lanes 2j and 2j + 1 end with that of row j.  Every step halves the
// values and the lanes that hold them: 16 shuffles rather than 80.
__device__ __forceinline__ float ca_row_sums16(float (&x)[16], int lane) {
#pragma unroll
    for (int h = 8; h > 0; h >>= 1) {
        const bool up = lane & (2 * h);
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float keep = up ? x[i + h] : x[i], give = up ? x[i] : x[i + h];
            x[i] = keep + __shfl_xor_sync(0xffffffffu, give, 2 * h);
        }
    }
    return x[0] + __shfl_xor_sync(0xffffffffu, x[0], 1);
}

template <int N, int D> struct CaLayout {
    static constexpr int kGroups = 2;                         // softmax groups = tiles in flight
    static constexpr int kWarps = 8 + 4 * kGroups;            // 2 producers, MMA issuer, queries, 4 accumulator, softmax
    static constexpr int kThreads = 32 * kWarps;
    // An MMA costs the same for 16 to 64 rows: the two terms of the split operand are one operand of twice the rows
    // (results in columns of their own, added when they are read), half the instructions.
    static constexpr int kCols = 2 * N;                       // tensor-memory columns of S or O of a group
    static constexpr int kColO = kGroups * kCols, kColL = 2 * kGroups * kCols, kColA = kColL + kGroups * N;
    static constexpr int kColsUsed = kColA + N;
    static constexpr int kTmemCols = kColsUsed <= 64 ? 64 : kColsUsed <= 128 ? 128 : kColsUsed <= 256 ? 256 : 512;
    static constexpr int kTileBytes = kCaTile * D;            // K or V of a tile
    static constexpr int kQBytes = N * D;                     // one term of the queries
    static constexpr int kPBytes = N * kCaTile;               // one term of the probabilities
    static constexpr int kFixed = 4 * kQBytes + 2 * kGroups * kPBytes;
    // shared memory besides the rings: the kernel's static arrays, in the order of their declaration; then barriers and words
    static constexpr int kStatic = 4 * N * (4 * kGroups + 4 * kGroups + 4 * kGroups + 2 * (4 * kGroups + 4) + 2 * kGroups) +
                                   8 * 2 * kGroups * N + 4 * 2 * N + 4 * 2 * 32 + 8 * kCaScaleRing * kCaMaxPages +
                                   4 * 2 * N * (D / 32) + (int)sizeof(CaShare) + 512;
    static constexpr int kSlotsFit = (kCaSmem - 20480 - 1024 - kFixed) / kTileBytes;   // 20480: rings of 5 or 6 tiles
    static constexpr int kRing = kSlotsFit / 2 > 6 ? 6 : kSlotsFit / 2;   // tiles in the ring of K, and in that of V
    static constexpr int kDynamic = 2 * kRing * kTileBytes + kFixed + 1024;
    static constexpr int kPiece = N * D + 2 * N;              // floats of a partial result
    static_assert(kRing >= 3 && kRing + 2 <= kCaScaleRing, "ring");
    static_assert(kStatic + kDynamic <= kCaSmem, "shared memory");
    static_assert(kColsUsed <= 512, "tensor memory");
    static_assert(N % 16 == 0 && N <= 32, "rows");
};

template <int N, int D>
__global__ void __launch_bounds__(CaLayout<N, D>::kThreads, 1)
cache_attention_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                       const CacheAttnParams p) {
    using L = CaLayout<N, D>;
    constexpr uint32_t RING = L::kRing;
    constexpr int kCaThreads = L::kThreads;
    constexpr uint32_t NG = L::kGroups;
    constexpr uint32_t kSw = D == 128 ? 2 : 4;                // 128-byte or 64-byte swizzle: a token's row
    extern __shared__ unsigned char ca_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(ca_smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_q = smem + 2 * RING * L::kTileBytes;        // [2 buffers][2 terms]
    unsigned char* s_p = s_q + 4 * L::kQBytes;                // [2 groups][2 terms]
    __shared__ __align__(8) unsigned long long b_full[2][RING], b_empty[2][RING], b_scale[kCaScaleRing], b_qfull[2], b_qempty[2], b_s[NG], b_p[NG],
        b_o[NG], b_ofree[NG], b_mt[NG][2], b_l[2], b_lfree[2], b_drain;
    __shared__ __align__(16) float s_red[NG][4][N];           // maxima of the warps of a softmax group
    __shared__ __align__(16) float s_lred[NG][4][N];          // sums of the warps of a softmax group
    __shared__ __align__(16) float s_m[4 * NG][N];            // per softmax warp: 8 - the tile's maximum
    __shared__ __align__(16) float s_a[4 * NG + 4][N], s_b[4 * NG + 4][N];   // per softmax and accumulator warp: factors of what there is and of the tile
    __shared__ float s_mt[NG][2][N];                          // maxima of a group's tiles, for the accumulator
    __shared__ float2 s_ml[2][NG][N];                         // per item parity and group: running maximum and sum
    __shared__ __align__(16) float s_c[2][N];                 // per query buffer: softmax scale of the row
    __shared__ uint32_t s_anc[2][32];                         // per query buffer: ancestors of the tree's nodes
    __shared__ __align__(8) float s_scale[kCaScaleRing][kCaMaxPages][2];
    __shared__ uint32_t s_nan[2][N][D / 32];                  // per item parity: results a NaN of a masked tile of V belongs to
    __shared__ volatile int s_nan_any[2];
    __shared__ CaShare s_share;
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    __shared__ int s_last;
    __shared__ uint32_t s_tiles[2];                           // tiles whose copies the producers have issued

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        ca_init_rings<RING>(b_full, b_empty, b_scale);
        for (int a = 0; a < 2; ++a) {
            mbar_init(smem_u32(&b_qfull[a]), 1);
            mbar_init(smem_u32(&b_qempty[a]), 1 + 4 * NG);    // the MMAs and the softmax warps
            mbar_init(smem_u32(&b_l[a]), 4 * NG);
            mbar_init(smem_u32(&b_lfree[a]), 4);
            s_nan_any[a] = 0;
        }
        for (int g = 0; g < NG; ++g) {
            mbar_init(smem_u32(&b_s[g]), 1);
            mbar_init(smem_u32(&b_p[g]), 4);                  // the four warps of a softmax group
            mbar_init(smem_u32(&b_o[g]), 1);
            mbar_init(smem_u32(&b_ofree[g]), 4);              // the four accumulator warps
            mbar_init(smem_u32(&b_mt[g][0]), 1);
            mbar_init(smem_u32(&b_mt[g][1]), 1);
        }
        mbar_init(smem_u32(&b_drain), 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < 2 * N * (D / 32); i += kCaThreads) (&s_nan[0][0][0])[i] = 0u;
    if (warp == 2) tc_alloc(smem_u32(&s_tmem), L::kTmemCols);
    if (warp == 0 && lane < 2) {
        const CUtensorMap* tm = lane ? &tm_v : &tm_k;
        asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory");
    }
    pdl_enter();

    CaCursor cur;
    const CaPart share = ca_share<L::kThreads>(p, s_share, cur);
    const uint32_t tmem = s_tmem;

    if (warp < 2) {
        // K: warp 0, V: warp 1
        ca_produce<D, RING>(p, cur, warp, warp ? &tm_v : &tm_k, smem + warp * RING * L::kTileBytes, b_full[warp], b_empty[warp], b_scale, s_scale, s_tiles, &s_abort);
    } else if (warp == 2) {
        // ================================= MMA issuer =================================
        // S of tiles 0 and 1, then, whenever the probabilities of a tile are there: S of the tile two further on, whose
        // place in tensor memory they have left, and O of the tile itself.
        constexpr uint32_t id_s = (1u << 4) | ((uint32_t)(L::kCols >> 3) << 17) | ((uint32_t)(kCaTile >> 4) << 24);
        constexpr uint32_t id_o = (1u << 4) | (1u << 15) | (1u << 16) | ((uint32_t)(L::kCols >> 3) << 17) | ((uint32_t)(D >> 4) << 24);
        const uint32_t elected = ca_elect();
        uint32_t total = cur.x < cur.end ? 0xffff0000u : 0u;  // tiles of this CTA, known when its last item is through
        uint32_t ks = 0, kph = 0, vs = 0, vph = 0;            // places in the rings of K and V
        int item = -1, left = 0;                              // tiles of the item whose S is still to be issued
        bool ok = true;
#pragma unroll 1
        for (uint32_t j = 0; j < total + 2 && ok; ++j) {      // S of tile j, O of tile j - 2
            const uint32_t u = j & 1;
            if (j >= 2) ok = ca_wait(smem_u32(&b_p[u]), ((j >> 1) - 1) & 1);
            if (ok && j < total) {
                if (left == 0) {
                    if (item >= 0) ca_advance(p, cur, ca_tiles_here(cur));
                    if (cur.x >= cur.end) {
                        total = j;
                    } else {
                        ++item;
                        left = ca_tiles_here(cur);
                        ok = ca_wait(smem_u32(&b_qfull[item & 1]), (uint32_t)((item >> 1) & 1));
                    }
                }
            }
            if (ok && j < total) {
                ok = ca_wait(smem_u32(&b_full[0][ks]), kph) && !__any_sync(0xffffffffu, s_abort);
                if (!ok) break;
                tc_fence_after();
                const uint64_t dk = ca_desc(smem_u32(smem + ks * L::kTileBytes), 16, 8 * D, kSw);
                const uint64_t dq = ca_desc(smem_u32(s_q + (item & 1) * 2 * L::kQBytes), 128, 8 * D, 0);
#pragma unroll
                for (int s = 0; s < D / 32; ++s)
                    ca_mma(tmem + u * L::kCols, dk + ((s * 32) >> 4), dq + ((s * 256) >> 4), id_s, s ? 1u : 0u, elected);
                ca_commit(smem_u32(&b_s[u]), elected);
                ca_commit(smem_u32(&b_empty[0][ks]), elected);
                if (--left == 0) ca_commit(smem_u32(&b_qempty[item & 1]), elected);
                if (++ks == RING) { ks = 0; kph ^= 1u; }
            }
            if (ok && j >= 2) {
                const uint32_t k = j - 2;
                if (!ca_wait(smem_u32(&b_full[1][vs]), vph) || (k >= 2 && !ca_wait(smem_u32(&b_ofree[u]), ((k >> 1) - 1) & 1)) ||
                    __any_sync(0xffffffffu, s_abort)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint64_t dv = ca_desc(smem_u32(smem + (RING + vs) * L::kTileBytes), 0, 8 * D, kSw);
                const uint64_t dp = ca_desc(smem_u32(s_p + u * 2 * L::kPBytes), 128, 2048, 0);
#pragma unroll
                for (int s = 0; s < kCaTile / 32; ++s)
                    ca_mma(tmem + L::kColO + u * L::kCols, dv + ((s * 32 * D) >> 4), dp + ((s * 512) >> 4), id_o, s ? 1u : 0u, elected);
                ca_commit(smem_u32(&b_o[u]), elected);
                ca_commit(smem_u32(&b_empty[1][vs]), elected);
                if (++vs == RING) { vs = 0; vph ^= 1u; }
            }
        }
        if (!ok && lane == 0) ca_give_up(p, &s_abort);
        __syncwarp();
    } else if (warp == 3) {
        // ================================== queries ==================================
        int item = 0;
        bool ok = true;
#pragma unroll 1
        while (cur.x < cur.end && ok) {
            const int buf = item & 1;
            if (item >= 2) ok = ca_wait(smem_u32(&b_qempty[buf]), (uint32_t)(((item >> 1) - 1) & 1)) && !__any_sync(0xffffffffu, s_abort);
            if (!ok) break;
            ca_queries<N, D, 32>(p, cur, buf, lane, s_q, s_c, s_anc);
            if (lane == 0) mbar_arrive(smem_u32(&b_qfull[buf]));
            ++item;
            ca_advance(p, cur, ca_tiles_here(cur));
        }
        if (!ok && lane == 0) ca_give_up(p, &s_abort);
    } else if (warp < 8) {
        // ================================ accumulator ================================
        // O^T of every tile into fp32 (tensor memory, 16 rows at a time in one short loop: code that does not fit the
        // instruction cache nearest to the warps costs more than the arithmetic); at the end of an item the sums join and
        // the result leaves
        const int wq = warp & 3;                              // lane quarter of tensor memory
        const int dim = D == 128 ? wq * 32 + lane : wq * 16 + lane;   // this thread's element of d (64: lanes 0-15)
        const bool has_dim = D == 128 || lane < 16;
        float* f_a = s_a[4 * NG + wq];
        float* f_b = s_b[4 * NG + wq];
        const uint32_t t_lane = tmem + ((uint32_t)(wq * 32) << 16), t_acc = t_lane + L::kColA;
        uint32_t k = 0;                                       // running tile number
        int item = 0;
        bool ok = true;
#pragma unroll 1
        while (cur.x < cur.end) {
            const int buf = item & 1;
            const int nt = ca_tiles_here(cur);
            const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
            float m_run = -INFINITY, l_run = 0.f;             // row `lane`
#pragma unroll 1
            for (int t = 0; t < nt; ++t, ++k) {
                const uint32_t g = k % NG, kk = k / NG;
                if (ok) ok = ca_wait(smem_u32(&b_mt[g][kk & 1]), (kk >> 1) & 1) && !__any_sync(0xffffffffu, s_abort);
                if (!ok) continue;
                if (lane < N) {
                    const float mt = s_mt[g][kk & 1][lane], mn = fmaxf(m_run, mt);
                    f_a[lane] = mn == -INFINITY ? 1.f : ex2(m_run - mn);
                    f_b[lane] = mn == -INFINITY ? 0.f : ex2(mt - mn) * 0.00390625f;
                    m_run = mn;
                }
                __syncwarp();
                ok = ca_wait(smem_u32(&b_o[g]), kk & 1);
                if (!ok) continue;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < N; c += 16) {
                    float x[16], old[16];
                    if (t) ca_ld16(t_acc + c, old);
                    ca_result16(t_lane + L::kColO + g * L::kCols + c, N, x);
                    if (t) ca_ld16_wait(old);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const float4 fb = lds4(f_b + c + i);
                        x[i] *= fb.x; x[i + 1] *= fb.y; x[i + 2] *= fb.z; x[i + 3] *= fb.w;
                    }
                    if (t) {
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float4 fa = lds4(f_a + c + i);
                            x[i] = fmaf(old[i], fa.x, x[i]);
                            x[i + 1] = fmaf(old[i + 1], fa.y, x[i + 1]);
                            x[i + 2] = fmaf(old[i + 2], fa.z, x[i + 2]);
                            x[i + 3] = fmaf(old[i + 3], fa.w, x[i + 3]);
                        }
                    }
                    ca_st16(t_acc + c, x);
                }
                ca_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_ofree[g]));
            }
            // ---- end of the item, or of this CTA's part of it: the sums of the groups ----
            if (ok) ok = ca_wait(smem_u32(&b_l[buf]), (uint32_t)((item >> 1) & 1)) && !__any_sync(0xffffffffu, s_abort);
            // A wait that gave up leaves `ok` false in its warp only; the four leave together, here.  Behind it all of them have
            // seen b_l, so what they read below is the same for each and they meet at the barriers that depend on it.
            if (ca_bar_any(1 + NG, 128, !ok)) { ok = false; break; }
            if (lane < N)
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const float2 x = s_ml[buf][g][lane];
                    l_run += x.y * (x.x == -INFINITY ? 0.f : ex2(x.x - m_run));
                }
            // 16 rows of the accumulator; results that a NaN of a masked tile belongs to
            const bool nans = s_nan_any[buf] != 0;
            auto acc16 = [&](int c, float (&y)[16]) {
                ca_ld16(t_acc + c, y);
                ca_ld16_wait(y);
                if (nans && has_dim)
#pragma unroll 1
                    for (int r = 0; r < 16; ++r)
                        if ((s_nan[buf][c + r][dim >> 5] >> (dim & 31)) & 1u)
#pragma unroll
                            for (int i = 0; i < 16; ++i) y[i] = i == r ? __int_as_float(0x7fc00000) : y[i];
            };
            bool write = true, joined = false;
            long long c_first = 0, c_last = 0;
            if (nt < cur.ntiles) {
                // part of an item: leave it in the workspace; the CTA that completes the item joins the parts
                const long long xi = cur.x - cur.t;           // the item's first tile over all work
                c_first = ((xi + 1) * share.grid - 1) / share.work;
                c_last = ((xi + cur.ntiles) * share.grid - 1) / share.work;
                float* part = p.partial + ((size_t)blockIdx.x * 2 + (cur.t == 0 ? 1 : 0)) * L::kPiece;
#pragma unroll 1
                for (int c = 0; c < rows; c += 16) {
                    float y[16];
                    acc16(c, y);
                    if (has_dim)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (c + r < rows) part[(c + r) * D + dim] = y[r];
                }
                if (wq == 0 && lane < N) {
                    part[N * D + lane] = m_run;
                    part[N * D + N + lane] = l_run;
                }
                __threadfence();
                ca_bar_any(1 + NG, 128, false);
                if (wq == 0 && lane == 0) {
                    const uint32_t old = atomicAdd(p.ticket + c_first, 1u);
                    const bool last = old == (uint32_t)(c_last - c_first);
                    if (last) p.ticket[c_first] = 0u;
                    s_last = last;
                }
                ca_bar_any(1 + NG, 128, false);
                write = joined = s_last != 0;                 // written again only after a further barrier of the group
                if (joined) {
                    __threadfence();
                    // maximum and sum of the row over the parts
                    float mm = -INFINITY, ll = 0.f;
                    if (lane < N)
#pragma unroll 4
                        for (int c = (int)c_first; c <= (int)c_last; ++c) {
                            const float* q = p.partial + ((size_t)c * 2 + (c == c_first ? 1 : 0)) * L::kPiece + N * D;
                            const float mc = __ldcg(q + lane), lc = __ldcg(q + N + lane);
                            const float mn = fmaxf(mm, mc);
                            ll = (mm == -INFINITY ? ll * 0.f : ll * ex2(mm - mn)) + (mc == -INFINITY ? lc * 0.f : lc * ex2(mc - mn));
                            mm = mn;
                        }
                    m_run = mm;
                    l_run = ll;
                }
            }
            if (write) {
                __syncwarp();
                if (lane < N) {
                    f_a[lane] = l_run == 0.f ? 0.f : 1.f / l_run;   // nothing seen: zeros
                    f_b[lane] = m_run;
                }
                __syncwarp();
                __nv_bfloat16* o = p.out + (long long)(cur.q0 + i0) * p.o_st + (long long)cur.h * p.G * p.o_sh + dim;
                int hh = 0;
#pragma unroll 1
                for (int c = 0; c < rows; c += 16) {
                    float y[16];
                    if (!joined) {
                        acc16(c, y);
                    } else {
#pragma unroll
                        for (int r = 0; r < 16; ++r) y[r] = 0.f;
#pragma unroll 1
                        for (int z = (int)c_first; z <= (int)c_last; ++z) {
                            const float* q = p.partial + ((size_t)z * 2 + (z == c_first ? 1 : 0)) * L::kPiece;
                            float v[16];
                            float4 mc[4];
#pragma unroll
                            for (int r = 0; r < 16; ++r) v[r] = c + r < rows && has_dim ? __ldcg(q + (c + r) * D + dim) : 0.f;
#pragma unroll
                            for (int i = 0; i < 4; ++i) mc[i] = __ldcg(reinterpret_cast<const float4*>(q + N * D + c) + i);
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float4 mm = lds4(f_b + c + 4 * i);
                                y[4 * i] = fmaf(v[4 * i], mc[i].x == -INFINITY ? 0.f : ex2(mc[i].x - mm.x), y[4 * i]);
                                y[4 * i + 1] = fmaf(v[4 * i + 1], mc[i].y == -INFINITY ? 0.f : ex2(mc[i].y - mm.y), y[4 * i + 1]);
                                y[4 * i + 2] = fmaf(v[4 * i + 2], mc[i].z == -INFINITY ? 0.f : ex2(mc[i].z - mm.z), y[4 * i + 2]);
                                y[4 * i + 3] = fmaf(v[4 * i + 3], mc[i].w == -INFINITY ? 0.f : ex2(mc[i].w - mm.w), y[4 * i + 3]);
                            }
                        }
                    }
                    if (has_dim)
#pragma unroll
                        for (int r = 0; r < 16; ++r)
                            if (c + r < rows) {
                                o[hh * p.o_sh] = __float2bfloat16_rn(y[r] * f_a[c + r]);
                                if (++hh == p.G) { hh = 0; o += p.o_st; }
                            }
                }
                __syncwarp();
            }
            if (nans) {                                       // uniform: the marks have been read by all
                ca_bar_any(1 + NG, 128, false);
                for (int i = wq * 32 + lane; i < N * (D / 32); i += 128) (&s_nan[buf][0][0])[i] = 0u;
                if (wq == 0 && lane == 0) s_nan_any[buf] = 0;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_lfree[buf]));
            ++item;
            ca_advance(p, cur, nt);
        }
        if (!ok && lane == 0) ca_give_up(p, &s_abort);
    } else {
        // ================================== softmax ==================================
        const uint32_t g = (uint32_t)(warp >> 2) - 2u;        // group 0: warps 8-11, group 1: warps 12-15
        const int wq = warp & 3;                              // lane quarter of tensor memory
        const int tok = wq * 32 + lane;                       // this thread's token of a tile
        const int w8 = warp - 8;
        const uint32_t t_s = tmem + ((uint32_t)(wq * 32) << 16) + g * L::kCols;
        const uint32_t t_l = tmem + ((uint32_t)(wq * 32) << 16) + L::kColL + g * N;
        uint32_t g0 = 0;                                      // tiles of this CTA before the current item
        int item = 0;
        bool ok = true;
        // A wait that gave up leaves `ok` false in its warp only; the warps of a group leave together, at a barrier.
#pragma unroll 1
        while (cur.x < cur.end) {
            const int buf = item & 1;
            const int nt = ca_tiles_here(cur), te = cur.t + nt;
            const int limit = ca_limit(p, cur.base, cur.n, cur.rt);
            const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
            // positions below this are seen by every row of the item
            const int seen = p.node_parent ? cur.base : cur.base + i0 + 1;
            // the accumulator is through with the item two before this one, which used the same sums and marks
            if (ok && item >= 2) ok = ca_wait(smem_u32(&b_lfree[buf]), (uint32_t)(((item >> 1) - 1) & 1));
            float m_run = -INFINITY;                          // running maximum of row `lane`
            const int t_first = cur.t + (int)((g + NG - g0 % NG) % NG);

#pragma unroll 1
            for (int t = t_first; t < te; t += NG) {
                const uint32_t k = g0 + (uint32_t)(t - cur.t);   // running tile number
                const uint32_t kk = k / NG;
                const uint32_t vslot = k % RING;
                const bool first = t == t_first;
                if (ok) ok = ca_wait(smem_u32(&b_scale[k % kCaScaleRing]), (k / kCaScaleRing) & 1) &&
                             (!first || ca_wait(smem_u32(&b_qfull[buf]), (uint32_t)((item >> 1) & 1))) &&   // its constants
                             !__any_sync(0xffffffffu, s_abort);
                const int pos = t * kCaTile + tok;
                const bool masked = (t + 1) * kCaTile > seen;
                if (ok && masked) ok = ca_wait(smem_u32(&b_full[1][vslot]), (k / RING) & 1);   // V is looked at
                uint32_t vis = ~0u;                           // rows that see this thread's token
                float ks = 0.f, lsv = 0.f, isv = 0.f;
                if (ok) {
                    if (masked) {
                        if (pos >= limit) vis = 0u;
                        else if (!p.node_parent) {
                            const long long r0 = (long long)(pos - cur.base - i0) * p.G;
                            vis = r0 <= 0 ? ~0u : r0 < 32 ? ~0u << r0 : 0u;
                        } else if (pos >= cur.base) {
                            vis = 0u;
#pragma unroll 1
                            for (int i = 0; i * p.G < rows; ++i)
                                if ((s_anc[buf][i0 + i] >> (pos - cur.base)) & 1u) vis |= (~0u >> (32 - p.G)) << (i * p.G);
                        }
                        const uint32_t all = rows >= 32 ? ~0u : (1u << rows) - 1u;
                        if ((vis & all) != all) {
                            const CaWho who{p.node_parent ? &s_anc[buf][i0] : nullptr, (pos - cur.base) & 31, __ffs(vis) - 1, rows, p.G, (vis & all) != 0u};
                            if (ca_clean_v<D>(smem + (RING + vslot) * L::kTileBytes, tok, who, &s_nan[buf][0][0])) s_nan_any[buf] = 1;
                        }
                    }
                    if (vis) {
                        const float* sc = s_scale[k % kCaScaleRing][tok >> p.bt_log2];
                        const float sv = fmaxf(sc[1], kCaMinScaleV);
                        ks = sc[0];
                        lsv = __log2f(sv);
                        isv = __fdividef(1.f, sv);
                    }
                    ok = ca_wait(smem_u32(&b_s[g]), kk & 1);
                }
                // Exponents t = S * ks * c + lsv (+ m) of this thread's token, 16 rows at a time.
                auto exponents = [&](int c, float (&x)[16], const float* m) {
                    ca_result16(t_s + c, N, x);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const float4 cc = lds4(&s_c[buf][c + i]);
                        float4 z = make_float4(lsv, lsv, lsv, lsv);
                        if (m) {
                            const float4 mm = lds4(m + c + i);
                            z = make_float4(lsv + mm.x, lsv + mm.y, lsv + mm.z, lsv + mm.w);
                        }
                        x[i] = fmaf(x[i] * ks, cc.x, z.x);
                        x[i + 1] = fmaf(x[i + 1] * ks, cc.y, z.y);
                        x[i + 2] = fmaf(x[i + 2] * ks, cc.z, z.z);
                        x[i + 3] = fmaf(x[i + 3] * ks, cc.w, z.w);
                    }
                    if (masked) {
                        uint32_t v = vis >> c;
                        asm volatile("" : "+r"(v));           // keeps this a branch: most tiles have no mask
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (!((v >> i) & 1u)) x[i] = -INFINITY;
                    }
                };
                if (ok) {
                    tc_fence_after();
                    // pass 1: maxima over the warp's 32 tokens
#pragma unroll 1
                    for (int c = 0; c < N; c += 16) {
                        float x[16];
                        exponents(c, x, nullptr);
#pragma unroll
                        for (int i = 0; i < 16; i += 4)       // the same from every lane: cheaper than a branch
                            *reinterpret_cast<float4*>(&s_red[g][wq][c + i]) =
                                make_float4(ca_warp_max(x[i]), ca_warp_max(x[i + 1]), ca_warp_max(x[i + 2]), ca_warp_max(x[i + 3]));
                    }
                }
                // The product of this group's last tile is done: its P may be overwritten.  It was issued after the accumulator
                // had taken the tile before it, so the maxima of that one may be overwritten, too.
                if (ok && k >= NG) ok = ca_wait(smem_u32(&b_o[g]), (kk - 1) & 1);
                if (ca_bar_any(1 + g, 128, !ok)) { ok = false; break; }
                // the tile's maxima over the four warps; factors of the sums, for this warp's own use
                if (lane < N) {
                    const float mt = fmaxf(fmaxf(s_red[g][0][lane], s_red[g][1][lane]), fmaxf(s_red[g][2][lane], s_red[g][3][lane]));
                    const float mn = fmaxf(m_run, mt);
                    s_m[w8][lane] = mt == -INFINITY ? 0.f : 8.f - mt;
                    s_a[w8][lane] = mn == -INFINITY ? 1.f : ex2(m_run - mn);
                    s_b[w8][lane] = mn == -INFINITY ? 0.f : ex2(mt - mn) * 0.00390625f;
                    if (wq == 0) s_mt[g][kk & 1][lane] = mt;
                    m_run = mn;
                }
                __syncwarp();
                if (wq == 0 && lane == 0) mbar_arrive(smem_u32(&b_mt[g][kk & 1]));
                // pass 2: probabilities P'' (scaled by 2^8), their sums, their two e4m3 terms
                unsigned char* sp = s_p + g * 2 * L::kPBytes + (tok >> 3) * 128 + (tok & 7) * 16;
#pragma unroll 1
                for (int c = 0; c < N; c += 16) {
                    float x[16], old[16];
                    if (!first) ca_ld16(t_l + c, old);
                    exponents(c, x, s_m[w8]);
                    if (!first) ca_ld16_wait(old);
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = ex2(x[i]);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) ca_split4(x[i], x[i + 1], x[i + 2], x[i + 3], hi[i / 4], lo[i / 4]);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {         // the sums
                        const float4 fb = lds4(&s_b[w8][c + i]);
                        x[i] *= isv * fb.x; x[i + 1] *= isv * fb.y; x[i + 2] *= isv * fb.z; x[i + 3] *= isv * fb.w;
                    }
                    if (!first) {
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float4 fa = lds4(&s_a[w8][c + i]);
                            x[i] = fmaf(old[i], fa.x, x[i]);
                            x[i + 1] = fmaf(old[i + 1], fa.y, x[i + 1]);
                            x[i + 2] = fmaf(old[i + 2], fa.z, x[i + 2]);
                            x[i + 3] = fmaf(old[i + 3], fa.w, x[i + 3]);
                        }
                    }
                    ca_st16(t_l + c, x);
                    *reinterpret_cast<uint4*>(sp + (c >> 4) * 2048) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *reinterpret_cast<uint4*>(sp + (c >> 4) * 2048 + L::kPBytes) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                ca_st_wait();
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_p[g]));   // S of this tile has been read, too
            }

            // ---- end of the item: this group's running maxima and sums ----
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_qempty[buf]));   // its constants have been read
            float l_run = 0.f;
            if (t_first < te) {                               // over the lanes, then over the warps
#pragma unroll 1
                for (int c = 0; c < N; c += 16) {
                    float y[16];
                    ca_ld16(t_l + c, y);
                    ca_ld16_wait(y);
                    s_lred[g][wq][c + (lane >> 1)] = ca_row_sums16(y, lane);
                }
                if (ca_bar_any(1 + g, 128, !ok)) { ok = false; break; }
                if (lane < N) l_run = (s_lred[g][0][lane] + s_lred[g][1][lane]) + (s_lred[g][2][lane] + s_lred[g][3][lane]);
            }
            if (wq == 0 && lane < N) s_ml[buf][g][lane] = make_float2(m_run, l_run);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_l[buf]));
            ++item;
            g0 += nt;
            ca_advance(p, cur, nt);
        }
        if (!ok && lane == 0) ca_give_up(p, &s_abort);
    }

    // ---- all roles meet; tensor memory goes back ----
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (s_abort) ca_drain<RING>(warp, b_full, s_tiles, &b_drain);
    if (warp == 2) {
        tc_fence_after();
        tc_free(tmem, L::kTmemCols);
    }
}

static std::atomic<bool> g_ca_attr[4][64];

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
    return cuda_status(launch_pdl(kern, sm_count(), L::kThreads, L::kDynamic, st, tm[0], tm[1], p));
}

// Workspace: an arrival counter per CTA and behind them the abort word, then the parts of items.
static size_t ca_ticket_bytes() { return align_up(sizeof(uint32_t) * ((size_t)sm_count() + 1), 256); }

}  // namespace bs

using namespace bs;

extern "C" size_t bs_cache_workspace_bytes(int Hq, int Hkv, int d) {
    if (Hkv < 1 || Hq < Hkv || Hq % Hkv || Hq / Hkv > 64 || (d != 64 && d != 128)) return 0;
    return ca_ticket_bytes() + align_up(sizeof(float) * 2 * (size_t)sm_count() * kCaMaxRows * (d + 2), 256);
}

extern "C" bs_status bs_cache_get_device_status(const void* workspace, size_t workspace_bytes, void* stream) {
    if (!workspace) return BS_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < ca_ticket_bytes()) return BS_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint32_t aborted = 0;
    cudaError_t e = cudaMemcpyAsync(&aborted, static_cast<const uint32_t*>(workspace) + sm_count(), sizeof(aborted),
                                    cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) return cuda_status(e);
    return aborted ? BS_ERR_TIMEOUT : BS_OK;
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
    p.abort = p.ticket + sm_count();
    p.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + ca_ticket_bytes());
    p.scale_log2 = softmax_scale * kLog2e;
    p.B = B; p.T = T; p.W = max_blocks; p.Nmax = Nmax; p.Hkv = Hkv; p.G = Hq / Hkv;
    p.n_blocks = n_blocks;
    p.bt_log2 = 4;
    while ((1 << p.bt_log2) < block_tokens) ++p.bt_log2;
    CUtensorMap tm[2];
    if (!ca_map(&tm[0], k_cache, n_blocks, Hkv, block_tokens, d) || !ca_map(&tm[1], v_cache, n_blocks, Hkv, block_tokens, d))
        return BS_ERR_CUDA;
    // The fewest rows that take a sequence's key head at once, so that its cache is read once.  Tokens as lanes cost
    // in proportion to the rows, rows as lanes the same for any number up to 64 and more for the few: 64 sequences of 4096
    // tokens, 8 key heads of 128, with 8 rows 137 us for tiles of 16, 172 for 32, 215 for 64, 262 for 128; with 32 rows 178 for
    // 32, 217 for 64; with 48 rows 315 (two items) and 220, with 64 rows 319 and 223, and 268 for 128.  Prompts take 128 at
    // once: the copies and the scales serve twice the rows.
    const long long rows = (long long)max_new * p.G;
    const int N = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : kCaMaxRows;
    p.TQ = N / p.G;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (N > 32) return launch_cache_attention_rows(tm, p, N, d, st);
    if (d == 128) return N == 16 ? launch_ca<16, 128>(tm, p, st) : launch_ca<32, 128>(tm, p, st);
    return N == 16 ? launch_ca<16, 64>(tm, p, st) : launch_ca<32, 64>(tm, p, st);
}
