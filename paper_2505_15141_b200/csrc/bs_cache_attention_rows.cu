// The attention of bs_cache_attention for many rows (new tokens x query heads of a key head): 33 to 64 of them, or 128 at a
// time.  The work list, copies, scales and arithmetic are those of bs_cache_attention.cu; the products lie the other way:
//
//   S [128 lanes, 128 tokens] = Q K^T          O [128 lanes, d] = P V^T^T   (P from shared memory, V read N-major)
//
// A lane of tensor memory is a row, so a thread has its row's exponents in a line: maximum, sum and factors are scalars
// of the thread, nothing crosses lanes, and the scales of K and V are the same for 16 tokens at least.  A thread's
// work on an exponent is about a third of what it is with tokens as lanes, at the price of MMAs that always cost
// 128 rows (1024 cycles a tile of 128 values a head; the copy of the tile takes 1360 at HBM's rate).
//
// R = 64: the rows of a tile stand in lanes 0-63 or 64-127, by turns (the MMA reads its 128 rows of Q from 64 rows further
// ahead; what it finds there ends in lanes nobody reads), so both halves of the warps work, on a tile each, with a
// maximum, sum and accumulator each, joined at the end of an item.  R = 128: two teams of four warps take the tiles in turn.
//
// Tensor memory: S of two tiles, O of one, the fp32 accumulator (O * 2^(m_tile - m) is added after every tile, as there).
//
// Bound by the four dependent stages of a tile (S, softmax, O, join) with two tiles in flight and, with 64 rows, one softmax warp
// for each sub-partition of the SM: issue slots 33 %, tensor
// pipe 29 %, DRAM 27 % of their peaks at 63 rows.  32 query / 8 key heads of 128, 64 sequences of 4096 tokens, 64 rows:
// 0.22 ms for 0.54 GB; pieces of 512 and 333 new tokens behind up to 4096 (47 GFLOP): 0.142 ms with 128 rows at a time (calls
// alone on the GPU; 0.135 among others).
//
// Warps: 0, 1 producers, 2 MMA issuer, 4-7 queries and accumulator, then the softmax teams.
#include "bs_cache_attention.cuh"

namespace bs {

// Pairs of fp32 in one instruction.
__device__ __forceinline__ uint64_t pk(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void upk(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

template <int R, int D> struct CrLayout {
    static constexpr int kTeamWarps = R / 32;                 // warps of a team = of a tile
    static constexpr int kTeams = 2;                          // tiles in flight
    static constexpr int kHalves = 128 / R;                   // places a tile's rows can stand in
    static constexpr int kSoft = kTeams * kTeamWarps;
    static constexpr int kWarps = 8 + kSoft;
    static constexpr int kThreads = 32 * kWarps;
    static constexpr int kColO = 256, kColA = 256 + D;        // S: 0-127, 128-255
    static constexpr int kTmemCols = 512;
    static constexpr int kTileBytes = kCaTile * D;
    static constexpr int kQBytes = R * D;                     // one term of the queries
    static constexpr int kPBytes = 128 * kCaTile;             // one term of the probabilities of 128 lanes
    static constexpr int kPBufs = kHalves == 1 ? 2 : 1;       // the halves share one
    static constexpr int kMerge = kHalves == 1 ? 0 : R * D * 4;
    static constexpr int kFixed = 4 * kQBytes + 2 * kPBufs * kPBytes + kMerge;
    // shared memory besides the rings: the kernel's static arrays, in the order of their declaration; then barriers and words
    static constexpr int kStatic = 4 * 2 * R + 4 * 2 * 32 + 4 * 4 * R + 8 * 4 * R + 16 * 8 * kSoft + 8 * (kHalves > 1 ? R : 1) +
                                   8 * kCaScaleRing * kCaMaxPages + 4 * 2 * R * (D / 32) + (int)sizeof(CaShare) + 512;
    static constexpr int kSlotsFit = (kCaSmem - kStatic - 1024 - kFixed) / kTileBytes;
    static constexpr int kRing = kSlotsFit / 2 > 6 ? 6 : kSlotsFit / 2;
    static constexpr int kDynamic = 2 * kRing * kTileBytes + kFixed + 1024;
    static constexpr int kPiece = R * D + 2 * R;              // floats of a partial result
    static_assert(kRing >= 2 && kRing + 2 <= kCaScaleRing, "ring");
    static_assert(kStatic + kDynamic <= kCaSmem, "shared memory");
    // Q is read from R rows before its buffer and up to R rows behind it: rings in front, P behind
    static_assert(2 * kRing * kTileBytes >= R * D && 2 * kPBufs * kPBytes >= R * D, "rows next to Q");
};

template <int R, int D>
__global__ void __launch_bounds__(CrLayout<R, D>::kThreads, 1)
cache_attention_rows_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                            const CacheAttnParams p) {
    using L = CrLayout<R, D>;
    constexpr uint32_t RING = L::kRing;
    constexpr int TW = L::kTeamWarps;
    constexpr uint32_t kSw = D == 128 ? 2 : 4;
    extern __shared__ unsigned char cr_smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(cr_smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_q = smem + 2 * RING * L::kTileBytes;     // [2 buffers][2 terms]
    unsigned char* s_p = s_q + 4 * L::kQBytes;                // [buffers][2 terms]
    float* s_merge = reinterpret_cast<float*>(s_p + 2 * L::kPBufs * L::kPBytes);   // [D][R]
    __shared__ __align__(8) unsigned long long b_full[2][RING], b_empty[2][RING], b_scale[kCaScaleRing], b_qfull[2], b_qempty[2], b_s[2], b_p[2], b_o[2],
        b_ofree[2], b_mt[2][2], b_l[2], b_lfree[2], b_drain;
    __shared__ float s_c[2][R];                               // per query buffer: softmax scale of the row
    __shared__ uint32_t s_anc[2][32];                         // per query buffer: ancestors of the tree's nodes
    __shared__ float s_mt[2][2][R];                           // maxima of a team's tiles, for the accumulator
    __shared__ float2 s_ml[2][2][R];                          // per item parity and team: running maximum and sum
    __shared__ __align__(16) float4 s_tab[L::kSoft][8];       // per softmax warp: scale of K, log2 and inverse of that of V, by 16 tokens
    __shared__ float2 s_hl[L::kHalves > 1 ? R : 1];           // merge: maximum and sum of the second half
    __shared__ __align__(8) float s_scale[kCaScaleRing][kCaMaxPages][2];
    __shared__ uint32_t s_nan[2][R][D / 32];                  // per item parity: results a NaN of a masked tile of V belongs to
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
            mbar_init(smem_u32(&b_qfull[a]), 4);              // the accumulator warps
            mbar_init(smem_u32(&b_qempty[a]), 1 + L::kSoft);  // the MMAs and the softmax warps
            mbar_init(smem_u32(&b_s[a]), 1);
            mbar_init(smem_u32(&b_p[a]), TW);
            mbar_init(smem_u32(&b_o[a]), 1);
            mbar_init(smem_u32(&b_ofree[a]), TW);
            mbar_init(smem_u32(&b_mt[a][0]), TW);
            mbar_init(smem_u32(&b_mt[a][1]), TW);
            mbar_init(smem_u32(&b_l[a]), L::kSoft);
            mbar_init(smem_u32(&b_lfree[a]), 4);
            s_nan_any[a] = 0;
        }
        mbar_init(smem_u32(&b_drain), 1);
        s_abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < 2 * R * (D / 32); i += L::kThreads) (&s_nan[0][0][0])[i] = 0u;
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
        // place in tensor memory they have left, and O of the tile itself.  O goes first where S begins an item: the
        // queries of that item are split when the accumulator has finished the item two before it, maybe with this very O.
        constexpr uint32_t id_s = (1u << 4) | ((uint32_t)(kCaTile >> 3) << 17) | (8u << 24);
        constexpr uint32_t id_o = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | (8u << 24);
        const uint32_t elected = ca_elect();
        uint32_t total = cur.x < cur.end ? 0xffff0000u : 0u;  // tiles of this CTA, known when its last item is through
        uint32_t ks = 0, kph = 0, vs = 0, vph = 0;            // places in the rings of K and V
        int item = -1, left = 0;                              // tiles of the item whose S is still to be issued
        bool ok = true;
#pragma unroll 1
        for (uint32_t j = 0; j < total + 2 && ok; ++j) {      // S of tile j, O of tile j - 2
            const uint32_t u = j & 1;
            if (j >= 2) ok = ca_wait(smem_u32(&b_p[u]), ((j >> 1) - 1) & 1);
            const bool s_first = left > 0;
#pragma unroll 1
            for (int turn = 0; turn < 2 && ok; ++turn) {
                if ((turn == 0) == s_first) {
                    if (j >= total) continue;
                    if (left == 0) {
                        if (item >= 0) ca_advance(p, cur, ca_tiles_here(cur));
                        if (cur.x >= cur.end) {
                            total = j;
                            continue;
                        }
                        ++item;
                        left = ca_tiles_here(cur);
                        ok = ca_wait(smem_u32(&b_qfull[item & 1]), (uint32_t)((item >> 1) & 1));
                    }
                    ok = ok && ca_wait(smem_u32(&b_full[0][ks]), kph) && !__any_sync(0xffffffffu, s_abort);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t dk = ca_desc(smem_u32(smem + ks * L::kTileBytes), 16, 8 * D, kSw);
                    const uint64_t dq = ca_desc(smem_u32(s_q + (item & 1) * 2 * L::kQBytes) - (L::kHalves > 1 && u ? R * D : 0), 128, 8 * D, 0);
#pragma unroll
                    for (int term = 0; term < 2; ++term)
#pragma unroll
                        for (int s = 0; s < D / 32; ++s)
                            ca_mma(tmem + u * 128, dq + ((term * L::kQBytes + s * 256) >> 4), dk + ((s * 32) >> 4), id_s, (term | s) ? 1u : 0u, elected);
                    ca_commit(smem_u32(&b_s[u]), elected);
                    ca_commit(smem_u32(&b_empty[0][ks]), elected);
                    if (--left == 0) ca_commit(smem_u32(&b_qempty[item & 1]), elected);
                    if (++ks == RING) { ks = 0; kph ^= 1u; }
                } else {
                    if (j < 2) continue;
                    const uint32_t k = j - 2;
                    if (!ca_wait(smem_u32(&b_full[1][vs]), vph) || (k >= 1 && !ca_wait(smem_u32(&b_ofree[u ^ 1]), ((k - 1) >> 1) & 1)) ||
                        __any_sync(0xffffffffu, s_abort)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint64_t dv = ca_desc(smem_u32(smem + (RING + vs) * L::kTileBytes), 0, 8 * D, kSw);
                    const uint64_t dp = ca_desc(smem_u32(s_p + (L::kPBufs > 1 ? u * 2 * L::kPBytes : 0)), 128, 1024, 0);
#pragma unroll
                    for (int term = 0; term < 2; ++term)
#pragma unroll
                        for (int s = 0; s < kCaTile / 32; ++s)
                            ca_mma(tmem + L::kColO, dp + ((term * L::kPBytes + s * 256) >> 4), dv + ((s * 32 * D) >> 4), id_o, (term | s) ? 1u : 0u, elected);
                    ca_commit(smem_u32(&b_o[u]), elected);
                    ca_commit(smem_u32(&b_empty[1][vs]), elected);
                    if (++vs == RING) { vs = 0; vph ^= 1u; }
                }
            }
        }
        if (!ok && lane == 0) ca_give_up(p, &s_abort);
        __syncwarp();
    } else if (warp == 3) {
        // nothing: warps 4-7 have to be the four quarters of tensor memory
    } else if (warp < 8) {
        // ================================ accumulator ================================
        const int wq = warp & 3;                              // lane quarter of tensor memory
        const int half = L::kHalves > 1 ? wq / TW : 0;        // where its tiles' rows stand
        const int row = (wq * 32 + lane) & (R - 1);
        const uint32_t t_lane = tmem + ((uint32_t)(wq * 32) << 16), t_acc = t_lane + L::kColA;
        uint32_t k = 0;                                       // running tile number
        int item = 0;
        bool ok = true;
        CaCursor qc = cur;                                    // the queries are an item ahead
        int q_item = 0;
        auto queries = [&]() {
            if (qc.x >= qc.end || !ok) return;
            const int qb = q_item & 1;
            // the products and the constants of the item that had this buffer are done with: its tiles have been joined here
            if (q_item >= 2) ok = ca_wait(smem_u32(&b_qempty[qb]), (uint32_t)(((q_item >> 1) - 1) & 1)) && !__any_sync(0xffffffffu, s_abort);
            if (!ok) return;
            ca_queries<R, D, 128>(p, qc, qb, wq * 32 + lane, s_q, s_c, s_anc);
            if (lane == 0) mbar_arrive(smem_u32(&b_qfull[qb]));
            ++q_item;
            ca_advance(p, qc, ca_tiles_here(qc));
        };
        queries();
#pragma unroll 1
        while (cur.x < cur.end) {
            const int buf = item & 1;
            const int nt = ca_tiles_here(cur);
            const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
            queries();
            float m_run = -INFINITY;
            bool have = false;                                // the accumulator holds something
#pragma unroll 1
            for (int t = 0; t < nt; ++t, ++k) {
                const uint32_t u = k & 1, kk = k >> 1;
                if (L::kHalves > 1 && (int)u != half) continue;
                if (ok) ok = ca_wait(smem_u32(&b_mt[u][kk & 1]), (kk >> 1) & 1) && !__any_sync(0xffffffffu, s_abort);
                if (!ok) continue;
                const float mt = s_mt[u][kk & 1][row], mn = fmaxf(m_run, mt);
                const float fa = mn == -INFINITY ? 1.f : ex2(m_run - mn), fb = mn == -INFINITY ? 0.f : ex2(mt - mn) * 0.00390625f;
                m_run = mn;
                ok = ca_wait(smem_u32(&b_o[u]), kk & 1);
                if (!ok) continue;
                tc_fence_after();
                float xa[16], oa[16], xb[16], ob[16];
                auto join = [&](int c, float (&x)[16], const float (&old)[16]) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[i] = have ? fmaf(old[i], fa, x[i] * fb) : x[i] * fb;
                    ca_st16(t_acc + c, x);
                };
                ca_ld16(t_lane + L::kColO, xa);
                ca_ld16(t_acc, oa);                           // not used before there is something
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    ca_ld16_wait(xa);
                    ca_ld16_wait(oa);
                    ca_ld16(t_lane + L::kColO + c + 16, xb);
                    ca_ld16(t_acc + c + 16, ob);
                    join(c, xa, oa);
                    ca_ld16_wait(xb);
                    ca_ld16_wait(ob);
                    if (c + 32 < D) {
                        ca_ld16(t_lane + L::kColO + c + 32, xa);
                        ca_ld16(t_acc + c + 32, oa);
                    }
                    join(c + 16, xb, ob);
                }
                have = true;
                ca_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_ofree[u]));
            }
            // ---- end of the item, or of this CTA's part of it: the sums of the teams ----
            if (ok) ok = ca_wait(smem_u32(&b_l[buf]), (uint32_t)((item >> 1) & 1)) && !__any_sync(0xffffffffu, s_abort);
            // A wait that gave up leaves `ok` false in its warp only; the four leave together, here.  Behind it all of them have
            // seen b_l, so what they read below is the same for each and they meet at the barriers that depend on it; and the
            // item before has been read out of the merge buffer.
            if (ca_bar_any(1, 128, !ok)) { ok = false; break; }
            float l_run = 0.f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (L::kHalves == 1 || u == half) {
                    const float2 x = s_ml[buf][u][row];
                    l_run += x.y * (x.x == -INFINITY ? 0.f : ex2(x.x - m_run));
                }
            const bool nans = s_nan_any[buf] != 0;
            const uint32_t* marks = s_nan[buf][row];
            // 16 elements of this half's accumulator
            auto mine16 = [&](int c, float (&y)[16]) {
                if (have) {
                    ca_ld16(t_acc + c, y);
                    ca_ld16_wait(y);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = 0.f;
                }
            };
            float f0 = 1.f, f1 = 0.f;                         // factors of the halves
            if (L::kHalves > 1) {
                if (half) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        float y[16];
                        mine16(c, y);
#pragma unroll
                        for (int i = 0; i < 16; ++i) s_merge[(c + i) * R + row] = y[i];
                    }
                    s_hl[row] = make_float2(m_run, l_run);
                }
                ca_bar_any(1, 128, false);
                if (!half) {
                    const float2 x = s_hl[row];
                    const float mn = fmaxf(m_run, x.x);
                    f0 = m_run == -INFINITY ? 0.f : ex2(m_run - mn);
                    f1 = x.x == -INFINITY ? 0.f : ex2(x.x - mn);
                    l_run = l_run * f0 + x.y * f1;
                    m_run = mn;
                }
            }
            auto acc16 = [&](int c, float (&y)[16]) {         // of both halves
                mine16(c, y);
                if (L::kHalves > 1)
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = fmaf(s_merge[(c + i) * R + row], f1, y[i] * f0);
                if (nans) {
                    const uint32_t b = marks[c >> 5] >> (c & 31);
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if ((b >> i) & 1u) y[i] = __int_as_float(0x7fc00000);
                }
            };
            const bool leads = half == 0;                     // these warps write the result
            bool write = true, joined = false;
            int c_first = 0, c_last = 0;
            if (nt < cur.ntiles) {
                // part of an item: leave it in the workspace; the CTA that completes the item joins the parts
                const long long xi = cur.x - cur.t;           // the item's first tile over all work
                c_first = (int)(((xi + 1) * share.grid - 1) / share.work);
                c_last = (int)(((xi + cur.ntiles) * share.grid - 1) / share.work);
                float* part = p.partial + ((size_t)blockIdx.x * 2 + (cur.t == 0 ? 1 : 0)) * L::kPiece;
                if (leads) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        float y[16];
                        acc16(c, y);
                        if (row < rows)
#pragma unroll
                            for (int i = 0; i < 16; i += 4)
                                *reinterpret_cast<float4*>(part + row * D + c + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
                    }
                    part[R * D + row] = m_run;
                    part[R * D + R + row] = l_run;
                }
                __threadfence();
                ca_bar_any(1, 128, false);
                if (wq == 0 && lane == 0) {
                    const uint32_t old = atomicAdd(p.ticket + c_first, 1u);
                    const bool last = old == (uint32_t)(c_last - c_first);
                    if (last) p.ticket[c_first] = 0u;
                    s_last = last;
                }
                ca_bar_any(1, 128, false);
                write = joined = s_last != 0;                 // written again only after a further barrier of the group
                if (joined) {
                    __threadfence();
                    float mm = -INFINITY, ll = 0.f;
#pragma unroll 4
                    for (int z = c_first; z <= c_last; ++z) {
                        const float* q = p.partial + ((size_t)z * 2 + (z == c_first ? 1 : 0)) * L::kPiece + R * D;
                        const float mc = __ldcg(q + row), lc = __ldcg(q + R + row);
                        const float mn = fmaxf(mm, mc);
                        ll = (mm == -INFINITY ? ll * 0.f : ll * ex2(mm - mn)) + (mc == -INFINITY ? lc * 0.f : lc * ex2(mc - mn));
                        mm = mn;
                    }
                    m_run = mm;
                    l_run = ll;
                }
            }
            if (write && (joined || leads)) {
                const float inv = l_run == 0.f ? 0.f : 1.f / l_run;   // nothing seen: zeros
                __nv_bfloat16* o = p.out + (long long)(cur.q0 + i0 + row / p.G) * p.o_st + (long long)(cur.h * p.G + row % p.G) * p.o_sh;
                auto put16 = [&](int c, const float (&y)[16]) {
                    if (row < rows) {
                        uint32_t w[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const __nv_bfloat162 b = __floats2bfloat162_rn(y[2 * i] * inv, y[2 * i + 1] * inv);
                            w[i] = *reinterpret_cast<const uint32_t*>(&b);
                        }
                        *reinterpret_cast<uint4*>(o + c) = make_uint4(w[0], w[1], w[2], w[3]);
                        *reinterpret_cast<uint4*>(o + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                    }
                };
                if (!joined) {
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        float y[16];
                        acc16(c, y);
                        put16(c, y);
                    }
                } else {                                      // each half of the warps takes its half of the elements
                    constexpr int kPart = D / L::kHalves;
#pragma unroll 1
                    for (int c = half * kPart; c < (half + 1) * kPart; c += 16) {
                        float y[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = 0.f;
                        if (row < rows)
#pragma unroll 4
                            for (int z = c_first; z <= c_last; ++z) {
                                const float* q = p.partial + ((size_t)z * 2 + (z == c_first ? 1 : 0)) * L::kPiece;
                                const float mc = __ldcg(q + R * D + row);
                                float4 v[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) v[i] = __ldcg(reinterpret_cast<const float4*>(q + row * D + c) + i);
                                const float f = mc == -INFINITY ? 0.f : ex2(mc - m_run);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    y[4 * i] = fmaf(v[i].x, f, y[4 * i]);
                                    y[4 * i + 1] = fmaf(v[i].y, f, y[4 * i + 1]);
                                    y[4 * i + 2] = fmaf(v[i].z, f, y[4 * i + 2]);
                                    y[4 * i + 3] = fmaf(v[i].w, f, y[4 * i + 3]);
                                }
                            }
                        put16(c, y);
                    }
                }
            }
            if (nans) {                                       // uniform: the marks have been read by all
                ca_bar_any(1, 128, false);
                for (int i = wq * 32 + lane; i < R * (D / 32); i += 128) (&s_nan[buf][0][0])[i] = 0u;
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
        const uint32_t u = (uint32_t)(warp - 8) / TW;         // team
        const int tw = (warp - 8) % TW;
        const int row = tw * 32 + lane;
        // lanes of tensor memory: a half of its own, or all of them
        const uint32_t t_s = tmem + ((uint32_t)((warp & 3) * 32) << 16) + u * 128;
        // a row's probabilities: 16-byte pieces of 16 tokens, 128 apart
        const int prow = (L::kHalves > 1 ? (int)u * R : 0) + row;
        unsigned char* sp = s_p + (L::kPBufs > 1 ? u * 2 * L::kPBytes : 0) + (prow >> 3) * 1024 + (prow & 7) * 16;
        uint32_t g0 = 0;                                      // tiles of this CTA before the current item
        int item = 0;
        bool ok = true;
        // A wait that gave up leaves `ok` false in its warp; the warps of a team wait for one another only through
        // bounded waits.
#pragma unroll 1
        while (cur.x < cur.end && ok) {
            const int buf = item & 1;
            const int nt = ca_tiles_here(cur);
            const int limit = ca_limit(p, cur.base, cur.n, cur.rt);
            const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
            const int seen = p.node_parent ? cur.base : cur.base + i0 + 1;   // positions below this are seen by every row
            // the accumulator is through with the item two before this one, which used the same sums and marks
            if (item >= 2) ok = ca_wait(smem_u32(&b_lfree[buf]), (uint32_t)(((item >> 1) - 1) & 1));
            float m_run = -INFINITY, l_run = 0.f, cr = 0.f;
            int sees = 0;                                     // chains: positions below this are seen by the row
            uint32_t anc = 0u;                                // trees: its node's ancestors
            const int t_first = cur.t + (int)((u ^ g0) & 1u);
#pragma unroll 1
            for (int t = t_first; t < cur.t + nt && ok; t += 2) {
                const uint32_t k = g0 + (uint32_t)(t - cur.t), kk = k >> 1;   // running tile number
                const uint32_t vslot = k % RING;
                const bool masked = (t + 1) * kCaTile > seen;
                ok = ca_wait(smem_u32(&b_scale[k % kCaScaleRing]), (k / kCaScaleRing) & 1) &&
                     (!masked || ca_wait(smem_u32(&b_full[1][vslot]), (k / RING) & 1)) &&   // V is looked at
                     (t != t_first || ca_wait(smem_u32(&b_qfull[buf]), (uint32_t)((item >> 1) & 1))) && !__any_sync(0xffffffffu, s_abort);
                if (!ok) break;
                if (t == t_first) {
                    cr = s_c[buf][row];
                    const int i = min(i0 + row / p.G, cur.n - 1);
                    sees = min(limit, cur.base + i + 1);
                    anc = p.node_parent ? s_anc[buf][i] : 0u;
                }
                const int pos0 = t * kCaTile;
                if (masked) {
#pragma unroll 1
                    for (int j = tw * 32 + lane; j < kCaTile; j += TW * 32) {
                        const int pos = pos0 + j;
                        const int first = p.node_parent ? 0 : (int)max(0ll, min((long long)kCaMaxRows, (long long)(pos - cur.base - i0) * p.G));
                        const bool new_tok = p.node_parent && pos >= cur.base;
                        CaWho who{new_tok ? &s_anc[buf][i0] : nullptr, (pos - cur.base) & 31, first, rows, p.G, pos < limit && first < rows};
                        if (new_tok && pos < limit) {
                            who.any = false;
#pragma unroll 1
                            for (int i = 0; i * p.G < rows; ++i) who.any = who.any || ((s_anc[buf][i0 + i] >> who.bit) & 1u);
                        }
                        if ((!who.any || who.anc || who.first_row > 0) && ca_clean_v<D>(smem + (RING + vslot) * L::kTileBytes, j, who, &s_nan[buf][0][0]))
                            s_nan_any[buf] = 1;
                    }
                }
                if (lane < 8) {
                    const float* z = s_scale[k % kCaScaleRing][(lane * 16) >> p.bt_log2];
                    const float sv = fmaxf(z[1], kCaMinScaleV);
                    s_tab[warp - 8][lane] = make_float4(z[0], __log2f(sv), __fdividef(1.f, sv), 0.f);
                }
                __syncwarp();
                const float4* tab = s_tab[warp - 8];
                ok = ca_wait(smem_u32(&b_s[u]), kk & 1);
                if (!ok) break;
                tc_fence_after();
                // which of 16 tokens the row sees
                auto seen16 = [&](int c) {
                    const int q = pos0 + c;
                    const int old = max(0, min(16, (p.node_parent ? cur.base : sees) - q));
                    uint32_t v = (1u << old) - 1u;
                    if (p.node_parent) {
                        const int d = q - cur.base;           // of the first of them
                        const uint32_t a = d >= 32 || d <= -32 ? 0u : d >= 0 ? anc >> d : anc << -d;
                        const int in = max(0, min(16, limit - q));
                        v |= a & ((1u << in) - 1u);
                    }
                    return v;
                };
                // pass 1: the row's maximum of t + log2(scale of V).  Tiles without a mask, nearly all of them, have short
                // loops of their own; their tensor-memory loads run 16 tokens ahead.
                float mx = -INFINITY;
                auto max16 = [&](const float4 z, const float (&x)[16]) {
                    const uint64_t kx2 = pk(z.x * cr, z.x * cr), vx2 = pk(z.y, z.y);
                    float a[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float q0, q1, q2, q3;
                        upk(fma2(pk(x[4 * i], x[4 * i + 1]), kx2, vx2), q0, q1);
                        upk(fma2(pk(x[4 * i + 2], x[4 * i + 3]), kx2, vx2), q2, q3);
                        a[i] = fmaxf(fmaxf(q0, q1), fmaxf(q2, q3));
                    }
                    mx = fmaxf(mx, fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3])));
                };
                float x[16], y[16];
                if (masked) {
#pragma unroll 1
                    for (int c = 0; c < kCaTile; c += 16) {
                        const uint32_t sx = seen16(c);
                        const float kx = tab[c >> 4].x * cr, vx = tab[c >> 4].y;
                        ca_ld16(t_s + c, x);
                        ca_ld16_wait(x);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if ((sx >> i) & 1u) mx = fmaxf(mx, fmaf(x[i], kx, vx));
                    }
                } else {
                    ca_ld16(t_s, x);
#pragma unroll 1
                    for (int c = 0; c < kCaTile; c += 32) {
                        const float4 z0 = tab[c >> 4], z1 = tab[(c >> 4) + 1];
                        ca_ld16_wait(x);
                        ca_ld16(t_s + c + 16, y);
                        max16(z0, x);
                        ca_ld16_wait(y);
                        ca_ld16(t_s + ((c + 32) & (kCaTile - 1)), x);   // in the end: the first tokens, for pass 2
                        max16(z1, y);
                    }
                }
                // The product of this team's last tile is done: its P may be overwritten, and the accumulator has taken the
                // maxima of the tile before it.
                if (k >= 2) {
                    ok = ca_wait(smem_u32(&b_o[u]), (kk - 1) & 1);
                    if (!ok) break;
                }
                s_mt[u][kk & 1][row] = mx;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_mt[u][kk & 1]));
                const float mn = fmaxf(m_run, mx);
                const float fa = mn == -INFINITY ? 1.f : ex2(m_run - mn), fb = mn == -INFINITY ? 0.f : ex2(mx - mn) * 0.00390625f;
                m_run = mn;
                const float m8 = mx == -INFINITY ? 0.f : 8.f - mx;
                // pass 2: probabilities (scaled by 2^8), their sum, their two e4m3 terms
                float sum = 0.f;
                auto split16 = [&](int c, const float (&x)[16]) {   // x: probabilities
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) ca_split4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3], hi[i], lo[i]);
                    *reinterpret_cast<uint4*>(sp + (c >> 4) * 128) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *reinterpret_cast<uint4*>(sp + (c >> 4) * 128 + L::kPBytes) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                };
                auto prob16 = [&](int c, const float4 z, float (&x)[16]) {
                    const uint64_t kx2 = pk(z.x * cr, z.x * cr), vx2 = pk(z.y + m8, z.y + m8);
                    uint64_t sa = 0ull, sb = 0ull;
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        upk(fma2(pk(x[i], x[i + 1]), kx2, vx2), x[i], x[i + 1]);
                        upk(fma2(pk(x[i + 2], x[i + 3]), kx2, vx2), x[i + 2], x[i + 3]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[i + e] = ex2(x[i + e]);
                        sa = add2(sa, pk(x[i], x[i + 1]));
                        sb = add2(sb, pk(x[i + 2], x[i + 3]));
                    }
                    float s0, s1;
                    upk(add2(sa, sb), s0, s1);
                    sum = fmaf(s0 + s1, z.z, sum);
                    split16(c, x);
                };
                if (masked) {
#pragma unroll 1
                    for (int c = 0; c < kCaTile; c += 16) {
                        float s0 = 0.f;
                        const uint32_t sx = seen16(c);
                        const float kx = tab[c >> 4].x * cr, vx = tab[c >> 4].y + m8;
                        ca_ld16(t_s + c, x);
                        ca_ld16_wait(x);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            x[i] = (sx >> i) & 1u ? ex2(fmaf(x[i], kx, vx)) : 0.f;
                            s0 += x[i];
                        }
                        if (sx) sum = fmaf(s0, tab[c >> 4].z, sum);   // blocks behind the sequence have no scale
                        split16(c, x);
                    }
                } else {
#pragma unroll 1
                    for (int c = 0; c < kCaTile; c += 32) {
                        const float4 z0 = tab[c >> 4], z1 = tab[(c >> 4) + 1];
                        ca_ld16_wait(x);
                        ca_ld16(t_s + c + 16, y);
                        prob16(c, z0, x);
                        ca_ld16_wait(y);
                        ca_ld16(t_s + ((c + 32) & (kCaTile - 1)), x);
                        prob16(c + 16, z1, y);
                    }
                    ca_ld16_wait(x);
                }
                l_run = fmaf(l_run, fa, sum * fb);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_p[u]));   // S of this tile has been read, too
            }
            // ---- end of the item: this team's running maximum and sum ----
            s_ml[buf][u][row] = make_float2(m_run, l_run);
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_u32(&b_qempty[buf]));        // its constants have been read
                mbar_arrive(smem_u32(&b_l[buf]));
            }
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

static std::atomic<bool> g_cr_attr[4][64];

template <int R, int D>
static bs_status launch_cr(const CUtensorMap* tm, const CacheAttnParams& p, cudaStream_t st) {
    using L = CrLayout<R, D>;
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) dev = 0;
    auto kern = cache_attention_rows_kernel<R, D>;
    constexpr int variant = (R == 128) * 2 + (D == 128);
    if (!g_cr_attr[variant][dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynamic) != cudaSuccess)
            return cuda_status(cudaGetLastError());
        g_cr_attr[variant][dev] = true;
    }
    return cuda_status(launch_pdl(kern, sm_count(), L::kThreads, L::kDynamic, st, tm[0], tm[1], p));
}

bs_status launch_cache_attention_rows(const CUtensorMap* tm, const CacheAttnParams& p, int rows, int d, cudaStream_t st) {
    if (d == 128) return rows <= 64 ? launch_cr<64, 128>(tm, p, st) : launch_cr<128, 128>(tm, p, st);
    return rows <= 64 ? launch_cr<64, 64>(tm, p, st) : launch_cr<128, 64>(tm, p, st);
}

}  // namespace bs
