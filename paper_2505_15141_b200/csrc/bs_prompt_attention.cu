// bs_prompt_attention: causal attention of whole prompts to themselves, packed sequences, grouped heads, bf16.
//
//   out_i = sum_{j <= i} p_ij v_j / sum_{j <= i} p_ij,   p_ij = 2^(c q_i . k_j - m_i),   c = softmax_scale * log2(e)
//
// One pass over the keys with a reference m_i of the row: the products S = Q K^T and O += P V run on the tensor cores with their
// accumulators in tensor memory; P is written there, too, as bf16, and is the A operand of the second product.  The
// reference is the row's maximum when it was last looked at: only where a later score exceeds it by more than 8 (2^8 times; fp32
// and bf16 hold that with the same relative precision) is it moved and the accumulator rescaled, which is rare after
// the first tiles.  P is rounded to bf16 (2^-8 relative at most); its sum is taken before that, in fp32.
//
// An item is a pair of row tiles of one key head; a tile holds 128 / G new tokens x G query heads (G = Hq / Hkv), so that the heads of a
// group share the copies of K and V and short prompts fill the tiles.  Two tiles are in flight: while the softmax of one
// runs, the tensor cores work on the other.  The last tile of keys is only as wide as it is seen.
//
// Warps: 0-3 and 4-7 softmax of the two tiles, a row a thread; 8 MMA issuer; 9 copies (TMA); 10 scheduler; 11 looks through the tiles
// of V that are seen in part.  The grid has a CTA for every item, the longest first; a running CTA takes over the item of one that
// has not begun (cluster launch control), so that copies and products of the next item begin under the end of the one before.
//
// Heads of 128 fill tensor memory with S and O of two tiles, and P takes the place of S; the chain of a tile is then S, softmax, P V, S of
// the next keys.  Heads of 64 leave room for P beside S, which takes the products out of that chain (4 prompts of 1000 to
// 4095, 16 heads: 160 -> 122 us at that step; 126 now).
//
// Measured, 32 query and 8 key heads of 128: one prompt of 16384, 2.0 ms, 1.1 PFLOP/s at the 1.45 to 1.5 GHz that the power limit leaves;
// 16 prompts of 1 to 4096, 0.50 ms, 0.91 PFLOP/s.  No unit is full: tensor pipe 54 %, special-function unit 55 %, issue slots 30 % (one prompt of
// 4096).  The products alone set four fifths of the time: without any softmax they and the copies take 1.63 (1.35 PFLOP/s; the library's
// sustained rate is 1.42) and 0.41 ms; the rest is softmax that they do not cover, and ends of items.  What made no difference, or a loss: two threads a row (+8 %),
// a part of the exponentials as polynomials on the FMA units (+-1 %; heads of 64, where the softmax is the longer part, +2 to
// 8 %: it is the warps' instructions one after the other that take the time, not the special-function units, busy for half of it), no look
// at the maxima but at the sums (+8 %), a warpgroup of its own for the results (+-1 %), four streams of 64 keys (+8 to 11 %), an
// issuer for each row tile (+12 to 18 %: in one order of issue the tiles stay half a step apart), turns at the exponentials (+5 and, heads
// of 64, +33 %), for heads of 64 the next scores fetched under the exponentials (+14 %).  Two CTAs as a pair on products of 256 rows, each with half of K
// and V: copies and products alone take as long as here (1.66 and 0.41 ms), so that neither shared memory nor the copies set
// the pace, and with the softmax, whose P then waits for eight warps of two SMs, it is 24 % slower (2.47 and 0.60 ms).
#include "bs_cache_attention.cuh"
#include "bs_overlap.cuh"
#include "bs_prompt_items.cuh"

namespace bs {

constexpr int kPaItems = 2;                    // items known to a CTA: the current and the next
constexpr int kPaThreads = 384;
constexpr float kPaSlack = 8.f;                // a score may exceed the reference by this much (log2)

struct PromptAttnParams {
    __nv_bfloat16* out;
    long long o_st, o_sh;
    const int32_t* cu;
    int32_t* status;
    float c;                                   // softmax_scale * log2(e)
    long long limit;                           // cycles of a wait
    int B, T, Hkv, G, TQ;                      // TQ: tokens of a row tile, 128 / G
};

template <int D> struct PaLayout {
    static constexpr int kTileBytes = kPaKeys * D * 2;        // of Q, K or V
    static constexpr int kChunk = 128 * 128;                  // 128 rows of 64 elements
    static constexpr int kChunks = D / 64;
    static constexpr int kRing = D == 128 ? 4 : 8;            // half of the places are for V
    static constexpr int kOut = 32 * 128;                     // 32 rows of 64 results, for each softmax warp
    static constexpr int kDynamic = (2 + kRing) * kTileBytes + 8 * kOut + 1024;
    // Tensor memory: the scores of row tile i at i * kColS, its probabilities kColP further, its accumulator at kColO + i * D.  Heads of 64
    // leave room for P beside S.
    static constexpr bool kApart = D == 64;
    static constexpr int kColS = kApart ? 192 : 128, kColP = kApart ? 128 : 0, kColO = 2 * kColS;
    static_assert(kColO + 2 * D <= 512, "tensor memory");
    static constexpr uint32_t kTmemCols = 512;
};

__device__ __forceinline__ void pa_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t elected) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 e, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(elected) : "memory");
}
__device__ __forceinline__ void pa_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc, uint32_t elected) {
    asm volatile(
        "{\n\t.reg .pred p, e;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 e, %5, 0;\n\t"
        "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(elected) : "memory");
}
__device__ __forceinline__ void pa_tma(uint32_t dst, const CUtensorMap* tm, int x, int head, int row, uint32_t bar, uint32_t elected) {
    asm volatile(
        "{\n\t.reg .pred e;\n\t"
        "setp.ne.b32 e, %6, 0;\n\t"
        "@e cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n\t}"
        ::"r"(dst), "l"(tm), "r"(x), "r"(head), "r"(row), "r"(bar), "r"(elected) : "memory");
}
__device__ __forceinline__ void pa_ld32(uint32_t taddr, float* u) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=f"(u[0]), "=f"(u[1]), "=f"(u[2]), "=f"(u[3]), "=f"(u[4]), "=f"(u[5]), "=f"(u[6]), "=f"(u[7]),
          "=f"(u[8]), "=f"(u[9]), "=f"(u[10]), "=f"(u[11]), "=f"(u[12]), "=f"(u[13]), "=f"(u[14]), "=f"(u[15]),
          "=f"(u[16]), "=f"(u[17]), "=f"(u[18]), "=f"(u[19]), "=f"(u[20]), "=f"(u[21]), "=f"(u[22]), "=f"(u[23]),
          "=f"(u[24]), "=f"(u[25]), "=f"(u[26]), "=f"(u[27]), "=f"(u[28]), "=f"(u[29]), "=f"(u[30]), "=f"(u[31])
        : "r"(taddr));
}
// The loaded values may be used behind this.
__device__ __forceinline__ void pa_ld32_wait(float* u) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+f"(u[0]), "+f"(u[1]), "+f"(u[2]), "+f"(u[3]), "+f"(u[4]), "+f"(u[5]), "+f"(u[6]), "+f"(u[7]),
          "+f"(u[8]), "+f"(u[9]), "+f"(u[10]), "+f"(u[11]), "+f"(u[12]), "+f"(u[13]), "+f"(u[14]), "+f"(u[15]),
          "+f"(u[16]), "+f"(u[17]), "+f"(u[18]), "+f"(u[19]), "+f"(u[20]), "+f"(u[21]), "+f"(u[22]), "+f"(u[23]),
          "+f"(u[24]), "+f"(u[25]), "+f"(u[26]), "+f"(u[27]), "+f"(u[28]), "+f"(u[29]), "+f"(u[30]), "+f"(u[31]));
}
__device__ __forceinline__ void pa_st16(uint32_t taddr, const uint32_t (&v)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
        ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]),
          "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ uint64_t pa_pk(float lo, float hi) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void pa_upk(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t pa_fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t pa_add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float pa_max3(float a, float b, float c) {   // NaN if one is
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
__device__ __forceinline__ uint32_t pa_bf16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ void pa_few_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 80;"); }

// Bounded wait of a converged warp; false if it gave up or another role has.  In line: with a call anywhere in the kernel its
// registers cannot be split unevenly.  What has arrived already, the usual case, costs one try and one vote; looking at the other
// roles' word there as well made it 150 cycles, on the path from product to product.  Some waits last as long as an item (for an
// item's place, for the first tile of V that is seen in part, of the warps whose row tile an item lacks), so the limit is the longest
// item's.  Time counted from the last tile copied took 0.5 to 3 % longer in all calls, and 15 % with the steps told by the issuer.
// ALONE: when everything ends, whoever gave up.
template <bool ALONE = false>
__device__ __forceinline__ bool pa_wait(const void* barrier, uint32_t parity, long long limit, const volatile int* gave_up) {
    const uint32_t bar = smem_u32(barrier);
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
    const long long t0 = clock64();
    uint32_t ok;
    do {                                                      // a try may suspend the warp: polling would take issue slots
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000000u) : "memory");
    } while (!ok && (ALONE || !*gave_up) && clock64() - t0 <= limit);
    return __all_sync(0xffffffffu, ok != 0);
}

// A tile of V that some rows see only in part: 0 * NaN is NaN, so what a row must not see may not be there.  Tokens behind the
// sequence become zero.  Elements that are not finite become zero, too, and first[element] the first token that has one there:
// rows from that token on see it, and get NaN.  One warp; where everything is finite it only reads: x * 0 is added up, which is NaN
// once x is not finite.
template <int D>
__device__ __forceinline__ void pa_clean_v(unsigned char* tile, int pos0, int n, int* first, volatile int* marked) {
    const int lane = threadIdx.x & 31;
    constexpr int kBatch = 8;                                 // pieces of 16 bytes in flight
    const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
    __nv_bfloat162 strange = zero;
    auto look = [&](uint32_t w) { strange = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w), zero, strange); };
#pragma unroll 1
    for (int i0 = lane; i0 < kPaKeys * D / 8; i0 += 32 * kBatch) {
        uint4 v[kBatch];
#pragma unroll
        for (int z = 0; z < kBatch; ++z) {
            uint4* at = reinterpret_cast<uint4*>(tile + (i0 + 32 * z) * 16);
            if (pos0 + (((i0 + 32 * z) >> 3) & (kPaKeys - 1)) < n) {
                v[z] = *at;
            } else {
                v[z] = make_uint4(0u, 0u, 0u, 0u);
                *at = v[z];
            }
        }
#pragma unroll
        for (int z = 0; z < kBatch; ++z) { look(v[z].x); look(v[z].y); look(v[z].z); look(v[z].w); }
    }
    if (!__any_sync(0xffffffffu, !(__low2float(strange) == 0.f && __high2float(strange) == 0.f))) return;
    *marked = 1;
#pragma unroll 1
    for (int i = lane; i < kPaKeys * D / 8; i += 32) {
        const int tok = (i >> 3) & (kPaKeys - 1), e0 = (i >> 10) * 64 + ((i & 7) ^ (tok & 7)) * 8;   // the copy's swizzle
        uint16_t* at = reinterpret_cast<uint16_t*>(tile + i * 16);
#pragma unroll 1
        for (int e = 0; e < 8; ++e)
            if ((at[e] & 0x7f80u) == 0x7f80u) {
                at[e] = 0;
                atomicMin(first + e0 + e, pos0 + tok);
            }
    }
}
// Keys of tile j that a row tile beginning at token i0 sees any of, as many as the products take.
__device__ __forceinline__ int pa_keys(const PromptAttnParams& p, int n, int i0, int j) {
    return min(kPaKeys, (min(n, i0 + p.TQ) - j * kPaKeys + 15) & ~15);
}
// Whether some row of the tile of rows that begins at token i0 does not see all of tile j of the keys.
__device__ __forceinline__ bool pa_masked(int i0, int j) { return (j + 1) * kPaKeys > i0 + 1; }
__device__ __forceinline__ int pa_first_masked(int i0) { return (i0 + 1) / kPaKeys; }

// Set where a wait gave up, for calls without a status array, too; there is no workspace that could hold it.
__device__ uint32_t g_pa_gave_up;

template <int D>
__global__ void __launch_bounds__(kPaThreads, 1)
prompt_attention_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                        const __grid_constant__ CUtensorMap tm_v, const PromptAttnParams p) {
    using L = PaLayout<D>;
    constexpr uint32_t RING = L::kRing;
    extern __shared__ unsigned char pa_smem_raw[];
    unsigned char* s_q = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(pa_smem_raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* s_kv = s_q + 2 * L::kTileBytes;            // K and V of a tile of keys follow one another in the ring
    unsigned char* s_out = s_kv + RING * L::kTileBytes;
    __shared__ __align__(8) unsigned long long b_full[RING], b_empty[RING], b_part[RING / 2], b_qfull[2], b_qempty[2], b_s[2], b_sfree[2], b_p[2][2], b_o[2],
        b_item[kPaItems], b_done[kPaItems], b_next, b_drain;
    __shared__ PaItem s_item[kPaItems];
    __shared__ int s_first[kPaItems][D];                      // see pa_clean_v
    __shared__ volatile int s_marked[kPaItems];               // some element of it is
    __shared__ __align__(16) uint4 s_next;                    // answer of the launch control
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    __shared__ uint32_t s_copies, s_parts, s_last, s_qcopies[2];   // copies issued; of the last 32, those by way of warp 11

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (uint32_t s = 0; s < RING; ++s) {
            mbar_init(smem_u32(&b_full[s]), 1);
            mbar_init(smem_u32(&b_empty[s]), 1);
            if (s < RING / 2) mbar_init(smem_u32(&b_part[s]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&b_qfull[i]), 1);
            mbar_init(smem_u32(&b_qempty[i]), 1);
            mbar_init(smem_u32(&b_s[i]), 1);
            mbar_init(smem_u32(&b_sfree[i]), 4);
            mbar_init(smem_u32(&b_p[i][0]), 4);               // the first half of the keys, the second
            mbar_init(smem_u32(&b_p[i][1]), 4);
            mbar_init(smem_u32(&b_o[i]), 1);
        }
        for (int s = 0; s < kPaItems; ++s) {
            mbar_init(smem_u32(&b_item[s]), 1);
            mbar_init(smem_u32(&b_done[s]), 11);              // copies, MMAs, V, eight softmax warps
        }
        mbar_init(smem_u32(&b_next), 1);
        mbar_init(smem_u32(&b_drain), 1);
        s_abort = 0;
        s_copies = s_parts = s_last = s_qcopies[0] = s_qcopies[1] = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 8) tc_alloc(smem_u32(&s_tmem), L::kTmemCols);
    if (warp == 9 && lane < 3) {
        const CUtensorMap* tm = lane == 0 ? &tm_q : lane == 1 ? &tm_k : &tm_v;
        asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    pdl_enter();

    // Registers: 208 for the softmax warps, 80 for the others; 256 * 208 + 128 * 80 of the 384 * 168 that the launch gives.
    bool ok = true;
    auto wait = [&](const unsigned long long* bar, uint32_t parity) { return pa_wait(bar, parity, p.limit, &s_abort); };

    if (warp == 10) {
        // ================================= scheduler =================================
        pa_few_registers();
        const uint32_t elected = ca_elect();
        PaWalk w = {};
        pa_walk_load(p, w);
        long long item = blockIdx.x;
        bool more = true, looked = false;
        uint32_t asked = 0, answered = 0;
        auto next = [&]() {                                   // the item of a CTA that has not begun, if there is one
            if (lane == 0) mbar_arrive_expect_tx(smem_u32(&b_next), 16);
            __syncwarp();
            asm volatile(
                "{\n\t.reg .pred e;\n\t"
                "setp.ne.b32 e, %2, 0;\n\t"
                "@e clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];\n\t}"
                ::"r"(smem_u32(&s_next)), "r"(smem_u32(&b_next)), "r"(elected) : "memory");
            ++asked;
            ok = wait(&b_next, answered & 1);
            if (!ok) return;
            ++answered;
            uint32_t canceled, x;
            asm volatile(
                "{\n\t.reg .pred c;\n\t.reg .b128 h;\n\t.reg .b32 y, z, u;\n\t"
                "ld.shared.b128 h, [%2];\n\t"
                "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 c, h;\n\t"
                "selp.u32 %0, 1, 0, c;\n\t"
                "mov.u32 %1, 0;\n\t"
                "@c clusterlaunchcontrol.query_cancel.get_first_ctaid.v4.b32.b128 {%1, y, z, u}, h;\n\t}"
                : "=r"(canceled), "=r"(x) : "r"(smem_u32(&s_next)) : "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // it is read before the next answer comes
            __syncwarp();
            more = canceled != 0;
            item = x;
        };
#pragma unroll 1
        for (uint32_t k = 0; ok; ++k) {                       // the k-th item of this CTA
            const uint32_t slot = k % kPaItems;
            PaItem it = {0, 0, 0, 0, 0, 0};
            const bool there = pa_take(p, w, item, more, ok, looked, it, next);
            if (ok && k >= kPaItems) ok = wait(&b_done[slot], (k / kPaItems - 1) & 1);
            if (!ok) break;
            for (int i = lane; i < D; i += 32) s_first[slot][i] = 0x7fffffff;
            if (lane == 0) {
                s_item[slot] = it;
                s_marked[slot] = 0;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_item[slot]));
            if (!there) break;
        }
        if (!ok && lane == 0) s_abort = 1;
        if (asked != answered) pa_wait<true>(&b_next, answered & 1, p.limit, &s_abort);   // whoever gave up: an answer on its way is waited for
        __syncwarp();
    } else if (warp == 9) {
        // ================================== copies ==================================
        pa_few_registers();
        const uint32_t elected = ca_elect();
        uint32_t at = 0, ph = 0, count = 0, parts = 0, last = 0, uses[2] = {0u, 0u};
        const uint32_t q_bytes = (uint32_t)(p.TQ * p.G * D * 2);
        // A tile of V that is seen in part goes by way of warp 11, which tells b_full when it has looked through it.  It has done so
        // long before its barrier is needed again: RING / 2 tiles of V further on, where the tile's place is, too.
        auto tile = [&](const CUtensorMap* tm, const PaItem& it, int j, bool part) {
            ok = wait(&b_empty[at], ph ^ 1u);
            if (!ok) return;
            const uint32_t bar = smem_u32(part ? &b_part[parts % (RING / 2)] : &b_full[at]), dst = smem_u32(s_kv + at * L::kTileBytes);
            parts += part;
            last = last << 1 | (part ? 1u : 0u);
            if (lane == 0) mbar_arrive_expect_tx(bar, L::kTileBytes);
            __syncwarp();
#pragma unroll
            for (int c = 0; c < L::kChunks; ++c) pa_tma(dst + c * L::kChunk, tm, c * 64, it.h, it.row0 + j * kPaKeys, bar, elected);
            ++count;
            if (++at == RING) { at = 0; ph ^= 1u; }
        };
#pragma unroll 1
        for (uint32_t k = 0; ok; ++k) {
            const uint32_t slot = k % kPaItems;
            ok = wait(&b_item[slot], (k / kPaItems) & 1);
            if (!ok) break;
            const PaItem it = s_item[slot];
            const int nt = max(it.nt0, it.nt1);
            if (nt == 0) break;
#pragma unroll 1
            for (int j = 0; j < nt && ok; ++j) {
                tile(&tm_k, it, j, false);
                if (j == 0)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (!ok || (i ? it.nt1 : it.nt0) == 0) continue;
                        if (uses[i]) ok = wait(&b_qempty[i], (uses[i] - 1) & 1);
                        if (!ok) continue;
                        const uint32_t bar = smem_u32(&b_qfull[i]), dst = smem_u32(s_q + i * L::kTileBytes);
                        if (lane == 0) mbar_arrive_expect_tx(bar, q_bytes);
                        __syncwarp();
#pragma unroll
                        for (int c = 0; c < L::kChunks; ++c)
                            pa_tma(dst + c * L::kChunk, &tm_q, c * 64, it.h * p.G, it.row0 + it.i0 + i * p.TQ, bar, elected);
                        ++uses[i];
                    }
                if (ok) tile(&tm_v, it, j, pa_masked(it.i0, j));
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_done[slot]));
        }
        if (lane == 0) {
            s_copies = count;
            s_parts = parts;
            s_last = last;
            s_qcopies[0] = uses[0];
            s_qcopies[1] = uses[1];
            if (!ok) s_abort = 1;
        }
    } else if (warp == 8) {
        // ================================= MMA issuer =================================
        pa_few_registers();
        // Step g is a tile of keys of an item.  In the order of issue: P V of step g - 1 and Q K^T of step g for row tile 0, then for row
        // tile 1; MMAs are carried out in this order, so S may overwrite the P that the product before it has read.  Where P has
        // a place of its own, Q K^T goes first, as soon as the scores of step g - 1 are in registers.
        constexpr uint32_t id_rows = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);   // S: N is the keys that are seen
        constexpr uint32_t id_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | (8u << 24);
        const uint32_t elected = ca_elect();
        uint32_t at = 0, ph = 0;                              // place in the ring: K of step g, or V of step g - 1 behind it
        uint32_t items = 0, steps[2] = {0u, 0u}, q_steps[2] = {0u, 0u}, q_uses[2] = {0u, 0u};
        PaItem cur = {0, 0, 0, 0, 0, 0}, prev = cur;
        int j = 0, jp = 0, nt = 0;                            // step of the current item; that of the step before
        uint32_t prev_slot = 0, v_at = 0, v_ph = 0;
        bool have_p = false, have_q = true;
#pragma unroll 1
        while (ok) {
            // step g: the next tile of keys, of the next item if the current one has no more
            if (have_q && j == nt) {
                ok = wait(&b_item[items % kPaItems], (items / kPaItems) & 1);
                if (!ok) break;
                cur = s_item[items % kPaItems];
                nt = max(cur.nt0, cur.nt1);
                j = 0;
                have_q = nt > 0;
                ++items;
            }
            if (!have_q && !have_p) break;
            const uint32_t k_at = at, k_ph = ph;
            if (have_q) {
                if (++at == RING) { at = 0; ph ^= 1u; }
            }
            const uint32_t nv_at = at, nv_ph = ph;            // V of step g
            if (have_q) {
                if (++at == RING) { at = 0; ph ^= 1u; }
            }
            // what has arrived long since is waited for before what has not: the probabilities
            if (have_p) ok = wait(&b_full[v_at], v_ph);
            if (have_q) ok = ok && wait(&b_full[k_at], k_ph);
            if (!ok) break;
            auto pv = [&](int i) {
                if (!have_p || jp >= (i ? prev.nt1 : prev.nt0)) return;
                const uint64_t dv = ca_desc(smem_u32(s_kv + v_at * L::kTileBytes), L::kChunk, 1024, 2);
                const int keys = pa_keys(p, prev.n, prev.i0 + i * p.TQ, jp);
#pragma unroll
                for (int s = 0; s < kPaKeys / 16; ++s) {
                    if (s % (kPaKeys / 32) == 0) {            // half of P is there
                        ok = ok && wait(&b_p[i][s / (kPaKeys / 32)], steps[i] & 1);
                        if (!ok) return;
                        tc_fence_after();
                    }
                    if (s * 16 < keys) pa_mma_ts(tmem + L::kColO + i * D, tmem + i * L::kColS + L::kColP + s * 8, dv + ((s * 2048) >> 4), id_o, (jp | s) ? 1u : 0u, elected);
                }
                ++steps[i];
                ca_commit(smem_u32(&b_o[i]), elected);
            };
            auto qk = [&](int i) {
                if (!ok || !have_q || j >= (i ? cur.nt1 : cur.nt0)) return;
                if (j == 0) ok = wait(&b_qfull[i], q_uses[i] & 1);
                if (L::kApart && q_steps[i]) ok = ok && wait(&b_sfree[i], (q_steps[i] - 1) & 1);
                if (!ok) return;
                ++q_steps[i];
                tc_fence_after();
                const uint64_t dq = ca_desc(smem_u32(s_q + i * L::kTileBytes), 16, 1024, 2);
                const uint64_t dk = ca_desc(smem_u32(s_kv + k_at * L::kTileBytes), 16, 1024, 2);
                const uint32_t id_s = id_rows | ((uint32_t)(pa_keys(p, cur.n, cur.i0 + i * p.TQ, j) >> 3) << 17);
#pragma unroll
                for (int s = 0; s < D / 16; ++s) {
                    const uint32_t off = ((s >> 2) * L::kChunk + (s & 3) * 32) >> 4;
                    pa_mma_ss(tmem + i * L::kColS, dq + off, dk + off, id_s, s ? 1u : 0u, elected);
                }
                ca_commit(smem_u32(&b_s[i]), elected);
                if (j == (i ? cur.nt1 : cur.nt0) - 1) {
                    ca_commit(smem_u32(&b_qempty[i]), elected);
                    ++q_uses[i];
                }
            };
            if (L::kApart) {
                qk(0); pv(0); qk(1);
                if (ok && have_q) ca_commit(smem_u32(&b_empty[k_at]), elected);
                pv(1);
                if (ok && have_p) ca_commit(smem_u32(&b_empty[v_at]), elected);
            } else {
                pv(0); qk(0); pv(1);
                if (ok && have_p) ca_commit(smem_u32(&b_empty[v_at]), elected);
                qk(1);
                if (ok && have_q) ca_commit(smem_u32(&b_empty[k_at]), elected);
            }
            if (!ok) break;
            if (have_p && jp == max(prev.nt0, prev.nt1) - 1 && lane == 0) mbar_arrive(smem_u32(&b_done[prev_slot]));
            __syncwarp();
            have_p = have_q;
            prev = cur;
            prev_slot = (items - 1) % kPaItems;
            jp = j;
            v_at = nv_at;
            v_ph = nv_ph;
            if (have_q) ++j;
        }
        // every product is through before this CTA's memory goes
        ca_commit(smem_u32(&b_drain), elected);
        if (!pa_wait<true>(&b_drain, 0, p.limit, &s_abort)) ok = false;   // whoever gave up: this one is waited for
        if (!ok && lane == 0) s_abort = 1;
        __syncwarp();
    } else if (warp < 8) {
        // ================================== softmax ==================================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
        const int i = warp >> 2;                              // row tile
        const int row = (warp & 3) * 32 + lane;
        const uint32_t t_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + i * L::kColS, t_p = t_s + L::kColP, t_o = t_lane + L::kColO + i * D;
        const int tok = row / p.G, head = row - tok * p.G;
        uint32_t steps = 0;                                   // tiles of keys so far, over all items
        uint32_t ring = 0;                                    // K and V tiles of the items so far
#pragma unroll 1
        for (uint32_t k = 0; ok; ++k) {
            const uint32_t slot = k % kPaItems;
            ok = wait(&b_item[slot], (k / kPaItems) & 1);
            if (!ok) break;
            const PaItem it = s_item[slot];
            if (it.nt0 == 0) break;
            const int nt = (i ? it.nt1 : it.nt0), i0 = it.i0 + i * p.TQ, pos = i0 + tok;
            const bool valid = tok < p.TQ && pos < it.n;
            float m = -INFINITY, l = 0.f;
#pragma unroll 1
            for (int j = 0; j < nt; ++j, ++steps) {
                const int pos0 = j * kPaKeys;
                const bool masked = pa_masked(i0, j);
                ok = wait(&b_s[i], steps & 1);
                if (!ok) break;
                tc_fence_after();
                // the scores, 64 at a time: the largest of the first are found while the others are on their way
                float s[128], top[2];
                pa_ld32(t_s, s);
                pa_ld32(t_s + 32, s + 32);
                const int sees = pos - pos0;                  // columns up to this one
                const int all = i0 + (warp & 3) * 32 / p.G - pos0;   // columns that the warp's first row sees, and so every one
#pragma unroll
                for (int c0 = 0; c0 < 128; c0 += 64) {
                    pa_ld32_wait(s + c0);
                    pa_ld32_wait(s + c0 + 32);
                    if (c0 == 0) {
                        pa_ld32(t_s + 64, s + 64);
                        pa_ld32(t_s + 96, s + 96);
                    } else if (L::kApart) {                   // S may be written again
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&b_sfree[i]));
                    }
                    if (masked)
#pragma unroll
                        for (int c = c0; c < c0 + 64; c += 16)
                            if (c + 15 > all)
#pragma unroll
                                for (int e = c; e < c + 16; ++e)
                                    if (e > sees) s[e] = -INFINITY;
                    float a[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[e] = pa_max3(s[c0 + e], s[c0 + e + 4], s[c0 + e + 8]);
#pragma unroll
                    for (int c = c0 + 12; c < c0 + 60; c += 8)
#pragma unroll
                        for (int e = 0; e < 4; ++e) a[e] = pa_max3(a[e], s[c + e], s[c + e + 4]);
                    top[c0 / 64] = pa_max3(pa_max3(a[0], a[1], a[2]), pa_max3(a[3], s[c0 + 60], s[c0 + 61]), pa_max3(s[c0 + 62], s[c0 + 63], s[c0 + 63]));
                }
                float mx = pa_max3(top[0], top[1], top[1]) * p.c;
                if (!(mx < INFINITY)) mx = __int_as_float(0x7fc00000);   // a row that sees a NaN or an infinite score: all NaN
                const bool moves = valid && !(mx <= m + kPaSlack);
                if (j == 0) {
                    m = mx;
                } else if (__any_sync(0xffffffffu, moves)) {
                    // the products so far
                    ok = wait(&b_o[i], (steps - 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
                    // a row's own scores alone decide when its reference moves: its result does not depend on the others
                    const float mn = moves ? mx : m, f = moves ? ex2(m - mn) : 1.f;
                    m = mn;
                    l *= f;
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        float o[16];
                        ca_ld16(t_o + c, o);
                        ca_ld16_wait(o);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] *= f;
                        ca_st16(t_o + c, o);
                    }
                    ca_st_wait();
                }
                if (L::kApart && j > 0) {                     // the product before has read its P
                    ok = wait(&b_o[i], (steps - 1) & 1);
                    if (!ok) break;
                    tc_fence_after();
                }
                const float nm = m == -INFINITY ? 0.f : -m;
                const int keys = pa_keys(p, it.n, i0, j);
                const uint64_t c2 = pa_pk(p.c, p.c), nm2 = pa_pk(nm, nm);
                uint64_t sum[2] = {0ull, 0ull};
#pragma unroll
                for (int c = 0; c < 128; c += 32) {
                    if (c < 64 || keys > 64) {                // else the product does not read it
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            float x, y;
                            pa_upk(pa_fma2(pa_pk(s[c + 2 * e], s[c + 2 * e + 1]), c2, nm2), x, y);
                            x = ex2(x);
                            y = ex2(y);
                            sum[e & 1] = pa_add2(sum[e & 1], pa_pk(x, y));
                            w[e] = pa_bf16x2(x, y);
                        }
                        pa_st16(t_p + (c >> 1), w);
                    }
                    if (c == 96 && masked) {                  // what was marked in V is seen behind this
                        const uint32_t r = ring + 2 * j + 1;
                        ok = wait(&b_full[r % RING], (r / RING) & 1);
                        if (!ok) break;
                    }
                    if (c & 32) {                             // half of P: the product may begin
                        ca_st_wait();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&b_p[i][c >> 6]));
                    }
                }
                float s0, s1;
                pa_upk(pa_add2(sum[0], sum[1]), s0, s1);
                l += s0 + s1;
                if (!ok) break;
            }
            if (!ok) break;
            if (nt > 0) {
                ok = wait(&b_o[i], (steps - 1) & 1);
                if (!ok) break;
                tc_fence_after();
                const float inv = 1.f / l;
                // Results leave through shared memory, so that eight lanes store the 128 bytes of a row side by side: a lane storing
                // its own row touches 32 lines per instruction, 2000 cycles a tile.
                __nv_bfloat16* mine = valid ? p.out + (long long)(it.row0 + pos) * p.o_st + (long long)(it.h * p.G + head) * p.o_sh : nullptr;
                unsigned char* stage = s_out + warp * L::kOut;
                const int* first = s_first[slot];
                const bool marked = s_marked[slot] != 0;
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += 64) {
#pragma unroll 1
                    for (int c = c0; c < c0 + 64; c += 32) {
                        float y[32];
                        pa_ld32(t_o + c, y);
                        pa_ld32_wait(y);
#pragma unroll
                        for (int e = 0; e < 32; ++e) y[e] *= inv;
                        if (marked)
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (first[c + e] <= pos) y[e] = __int_as_float(0x7fc00000);
#pragma unroll
                        for (int e = 0; e < 32; e += 8)
                            *reinterpret_cast<uint4*>(stage + lane * 128 + ((((c - c0 + e) >> 3) ^ (lane & 7)) << 4)) =
                                make_uint4(pa_bf16x2(y[e], y[e + 1]), pa_bf16x2(y[e + 2], y[e + 3]), pa_bf16x2(y[e + 4], y[e + 5]), pa_bf16x2(y[e + 6], y[e + 7]));
                    }
                    __syncwarp();
#pragma unroll
                    for (int r0 = 0; r0 < 32; r0 += 4) {
                        const int r = r0 + (lane >> 3), piece = lane & 7;
                        __nv_bfloat16* o = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), r));
                        const uint4 v = *reinterpret_cast<const uint4*>(stage + r * 128 + ((piece ^ (r & 7)) << 4));
                        if (o) *reinterpret_cast<uint4*>(o + c0 + piece * 8) = v;
                    }
                    __syncwarp();
                }
                tc_fence_before();
            }
            ring += 2 * max(it.nt0, it.nt1);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_done[slot]));
        }
        if (!ok && lane == 0) s_abort = 1;
    } else {
        // ============================ V, seen in part =============================
        pa_few_registers();
        uint32_t ring = 0, parts = 0;                         // copies of K and V of the items so far; tiles looked through
#pragma unroll 1
        for (uint32_t k = 0; ok; ++k) {
            const uint32_t slot = k % kPaItems;
            ok = wait(&b_item[slot], (k / kPaItems) & 1);
            if (!ok) break;
            const PaItem it = s_item[slot];
            const int nt = max(it.nt0, it.nt1);
            if (nt == 0) break;
#pragma unroll 1
            for (int j = pa_first_masked(it.i0); j < nt; ++j, ++parts) {
                const uint32_t at = (ring + 2 * j + 1) % RING;
                ok = wait(&b_part[parts % (RING / 2)], (parts / (RING / 2)) & 1);
                if (!ok) break;
                pa_clean_v<D>(s_kv + at * L::kTileBytes, j * kPaKeys, it.n, s_first[slot], &s_marked[slot]);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_full[at]));
            }
            ring += 2 * nt;
            __syncwarp();
            if (ok && lane == 0) mbar_arrive(smem_u32(&b_done[slot]));
        }
        if (!ok && lane == 0) s_abort = 1;
    }

    // ---- all roles meet; tensor memory goes back ----
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (s_abort) {
        // a wait gave up: nothing is issued any more, and no copy may be in flight when the memory goes (the products have been
        // waited for)
        if (warp == 9) {
            const uint32_t n = s_copies, m = s_parts;
            for (uint32_t f = n > RING ? n - RING : 0u; f < n; ++f)
                if (!((s_last >> (n - 1 - f)) & 1u)) pa_wait<true>(&b_full[f % RING], (f / RING) & 1, p.limit, &s_abort);
            for (uint32_t f = m > RING / 2 ? m - RING / 2 : 0u; f < m; ++f) pa_wait<true>(&b_part[f % (RING / 2)], (f / (RING / 2)) & 1, p.limit, &s_abort);
            for (int i = 0; i < 2; ++i)
                if (s_qcopies[i]) pa_wait<true>(&b_qfull[i], (s_qcopies[i] - 1) & 1, p.limit, &s_abort);
        }
        if (tid == 0) {
            g_pa_gave_up = 1u;
            if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
        }
        __syncthreads();
    }
    if (warp == 8) {
        tc_fence_after();
        tc_free(tmem, L::kTmemCols);
    }
}

static std::atomic<bool> g_pa_attr[2][64];

// [T, H, d] bf16; a box is 64 elements of `heads` heads of `rows` tokens, rows of 128 bytes, swizzled.
static bool pa_map(CUtensorMap* tm, const void* base, int T, int H, int d, long long st, long long sh, int heads, int rows) {
    EncodeTiledFn enc = encode_tiled_fn();
    const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)H, (cuuint64_t)T};
    const cuuint64_t strides[2] = {(cuuint64_t)sh * 2, (cuuint64_t)st * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)rows};
    const cuuint32_t estr[3] = {1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
static bs_status launch_pa(const CUtensorMap* tm, const PromptAttnParams& p, long long grid, cudaStream_t st) {
    using L = PaLayout<D>;
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) dev = 0;
    auto kern = prompt_attention_kernel<D>;
    if (!g_pa_attr[D == 128][dev]) {
        if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynamic) != cudaSuccess)
            return cuda_status(cudaGetLastError());
        g_pa_attr[D == 128][dev] = true;
    }
    return cuda_status(launch_pdl(kern, (unsigned)grid, kPaThreads, L::kDynamic, st, tm[0], tm[1], tm[2], p));
}

}  // namespace bs

using namespace bs;

extern "C" bs_status bs_prompt_get_device_status(void* stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    void* at = nullptr;
    uint32_t gave_up = 0;
    cudaError_t e = cudaGetSymbolAddress(&at, g_pa_gave_up);
    if (e == cudaSuccess) e = cudaMemcpyAsync(&gave_up, at, sizeof(gave_up), cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess && gave_up) {
        e = cudaMemsetAsync(at, 0, sizeof(gave_up), st);
        if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    }
    if (e != cudaSuccess) return cuda_status(e);
    return gave_up ? BS_ERR_TIMEOUT : BS_OK;
}

extern "C" bs_status bs_prompt_attention(const void* q, long long q_stride_t, long long q_stride_h, const void* k, long long k_stride_t,
                                         long long k_stride_h, const void* v, long long v_stride_t, long long v_stride_h,
                                         const int32_t* cu_seqlens, int B, int T, int Hq, int Hkv, int d, float softmax_scale, void* out,
                                         long long out_stride_t, long long out_stride_h, int32_t* status, void* stream) {
    if (B < 1 || T < 0 || Hq < 1 || Hkv < 1 || d < 1 || !(softmax_scale > 0.f) || !isfinite(softmax_scale * kLog2e) || !cu_seqlens)
        return BS_ERR_INVALID_ARG;
    if (Hq % Hkv || (T > 0 && (!q || !k || !v || !out))) return BS_ERR_INVALID_ARG;
    if (B > BS_MAX_BATCH || Hq / Hkv > 64 || (d != 64 && d != 128)) return BS_ERR_UNSUPPORTED;
    if ((q_stride_t | q_stride_h | k_stride_t | k_stride_h | v_stride_t | v_stride_h | out_stride_t | out_stride_h) & 7)
        return BS_ERR_UNSUPPORTED;
    if (q_stride_t < 0 || q_stride_h < 0 || k_stride_t < 0 || k_stride_h < 0 || v_stride_t < 0 || v_stride_h < 0) return BS_ERR_UNSUPPORTED;
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v) | reinterpret_cast<uintptr_t>(out)) & 15)
        return BS_ERR_INVALID_ARG;
    if (T == 0) return BS_OK;
    PromptAttnParams p;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.o_st = out_stride_t; p.o_sh = out_stride_h;
    p.cu = cu_seqlens; p.status = status;
    p.c = softmax_scale * kLog2e;
    p.limit = pa_wait_limit(T);
    p.B = B; p.T = T; p.Hkv = Hkv; p.G = Hq / Hkv; p.TQ = 128 / p.G;
    // pairs of row tiles: each sequence rounds up once
    const long long grid = ((long long)T / (2 * p.TQ) + B) * Hkv;
    // tokens are counted in 32 bits, up to a few tiles behind the last
    if (T > (1 << 30) || grid > 0x7fffffffLL) return BS_ERR_UNSUPPORTED;
    // CTAs write results while others still read
    const Rows to = rows_of(out, out_stride_t, out_stride_h, T, Hq, d, 2);
    if (rows_overlap(to, rows_of(q, q_stride_t, q_stride_h, T, Hq, d, 2)) || rows_overlap(to, rows_of(k, k_stride_t, k_stride_h, T, Hkv, d, 2)) ||
        rows_overlap(to, rows_of(v, v_stride_t, v_stride_h, T, Hkv, d, 2)))
        return BS_ERR_INVALID_ARG;
    if (!encode_tiled_fn()) return BS_ERR_CUDA;
    CUtensorMap tm[3];
    if (!pa_map(&tm[0], q, T, Hq, d, q_stride_t, q_stride_h, p.G, p.TQ) || !pa_map(&tm[1], k, T, Hkv, d, k_stride_t, k_stride_h, 1, kPaKeys) ||
        !pa_map(&tm[2], v, T, Hkv, d, v_stride_t, v_stride_h, 1, kPaKeys))
        return BS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return d == 128 ? launch_pa<128>(tm, p, grid, st) : launch_pa<64>(tm, p, grid, st);
}
