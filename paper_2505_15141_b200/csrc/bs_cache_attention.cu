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
// Roles of the 16 warps: 0 and 1 TMA producers of K and V, 2 MMA issuer, 3 queries (split into e4m3 one work item ahead),
// 4-7 accumulator (a thread is an element of d), 8-11 and 12-15 two softmax groups that take the tiles in turn, each with
// its own maximum and sum (a thread is a token).
//
// Work.  Item = (sequence, key head, N rows).  All tiles of all items, in order, are cut into equal contiguous shares,
// one per CTA, from the lengths on the device; an item that spans several CTAs is joined by the one that finishes
// last, in the order of the shares (the result does not depend on who that is).
#include "bs_cache_common.cuh"
#include "bs_pipeline.cuh"
#include "bs_tensor.cuh"

#include <atomic>

namespace bs {

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
#pragma unroll 1
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
__device__ __forceinline__ void ca_ld16(uint32_t taddr, uint32_t (&u)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]),
          "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15])
        : "r"(taddr));
}
__device__ __forceinline__ void ca_ld16_wait(uint32_t (&u)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]),
                   "+r"(u[8]), "+r"(u[9]), "+r"(u[10]), "+r"(u[11]), "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15]));
}
// Pairs of fp32 (rows 2i, 2i + 1) in one instruction.
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
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ void lds_2x2(const float* p, uint64_t& a, uint64_t& b) {   // four floats of shared memory
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(smem_u32(p)));
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
// 16 rows of an MMA result as pairs; WIDE: the two terms stand `n` columns apart and are added.
template <bool WIDE>
__device__ __forceinline__ void ca_result16(uint32_t taddr, int n, uint64_t (&x)[8]) {
    uint32_t u[16], w[16];
    ca_ld16(taddr, u);
    if (WIDE) ca_ld16(taddr + n, w);
    ca_ld16_wait(u);
    if (WIDE) ca_ld16_wait(w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        x[i] = pk(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
        if (WIDE) x[i] = add2(x[i], pk(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1])));
    }
}
// Sums of 16 per-lane values over the lanes of a warp: lanes 2j and 2j + 1 end with that of row ca_sum_row(lane).  Every
// step halves the values and the lanes that hold them: 16 shuffles rather than 80.
__device__ __forceinline__ int ca_sum_row(int lane) { return (lane >> 1 & 8) | (lane >> 1 & 4) | (lane >> 1 & 2) | (lane >> 1 & 1); }
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

// Bounded wait of a converged warp.  The loop is out of line: the kernel waits in many places, and its instructions have to
// stay in the instruction cache.
__device__ __noinline__ bool ca_wait_loop(uint32_t bar, uint32_t parity) { return mbar_wait(bar, parity); }
__device__ __forceinline__ bool ca_wait(uint32_t bar, uint32_t parity) {
    return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) || __all_sync(0xffffffffu, ca_wait_loop(bar, parity));
}

template <int N, int D> struct CaLayout {
    static constexpr int kGroups = 2;                         // softmax groups
    static constexpr int kWarps = 8 + 4 * kGroups + 2;        // 2 producers, 2 MMA issuers, 4 accumulator, softmax, 2 query warps
    static constexpr int kThreads = 32 * kWarps;
    static constexpr bool kOne = N == 16;                     // one group of 16 rows: sums and accumulator in registers
    // For few rows an MMA costs the same up to N = 64: the two terms of the split operand are one operand of twice the rows
    // (results in columns of their own, added when they are read), half the instructions.
    static constexpr bool kWide = N <= 32;
    static constexpr int kCols = kWide ? 2 * N : N;           // tensor-memory columns of S or O of a group
    static constexpr int kColO = kGroups * kCols, kColL = 2 * kGroups * kCols, kColA = kColL + kGroups * N;
    static constexpr int kColsUsed = kColA + N;
    static constexpr int kTmemCols = kColsUsed <= 64 ? 64 : kColsUsed <= 128 ? 128 : kColsUsed <= 256 ? 256 : 512;
    static constexpr int kTileBytes = kCaTile * D;            // K or V of a tile
    static constexpr int kQBytes = N * D;                     // one term of the queries
    static constexpr int kPBytes = N * kCaTile;               // one term of the probabilities
    static constexpr int kFixed = 4 * kQBytes + 2 * kGroups * kPBytes;
    // shared memory besides the rings: the static arrays of the kernel take up to 20 KB
    static constexpr int kSlotsFit = (kCaSmem - 20480 - 1024 - kFixed) / kTileBytes;
    static constexpr int kRing = kSlotsFit / 2 > 6 ? 6 : kSlotsFit / 2;   // tiles in the ring of K, and in that of V
    static constexpr int kDynamic = 2 * kRing * kTileBytes + kFixed + 1024;
    static constexpr int kPiece = N * D + 2 * N;              // floats of a partial result
    static_assert(kRing >= 3 && kRing < kCaScaleRing, "ring");
    static_assert(kColsUsed <= 512, "tensor memory");
    static_assert(N % 16 == 0 && N <= 64, "rows");
};

// Token `tok` of a tile of V that some rows must not see (`vis`: those that do): its codes may be anything, and 0 * NaN is
// NaN.  A token nobody sees becomes zero.  In one that some see, NaN codes become zero and the results they belong
// to are marked; true if there were any.  Once per item at most, so kept out of the way of the loop's instructions.
template <int D>
__device__ __noinline__ bool ca_clean_v(unsigned char* tile, int tok, unsigned long long vis, uint32_t* marks) {
    bool found = false;
#pragma unroll 1
    for (int c = 0; c < D / 16; ++c) {
        uint4* q = reinterpret_cast<uint4*>(tile + (D == 128 ? tok * 128 + ((c ^ (tok & 7)) << 4) : tok * 64 + ((c ^ ((tok >> 1) & 3)) << 4)));
        if (!vis) {
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
            for (unsigned long long rest = vis; rest; rest &= rest - 1ull)
                atomicOr(marks + (__ffsll((long long)rest) - 1) * (D / 32) + (c >> 1), bits);
        }
    }
    return found;
}

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
    __shared__ __align__(8) unsigned long long b_full[2][RING], b_empty[2][RING], b_qfull[2], b_qempty[2], b_s[NG], b_free[NG],
        b_p[NG], b_o[NG], b_ofree[NG], b_mt[NG][2], b_l[2], b_lfree[2], b_drain[2];
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
    __shared__ long long s_w[kCaThreads / 32];
    __shared__ long long s_start_off;
    __shared__ int s_start_b;
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_abort;
    __shared__ int s_last;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        for (uint32_t s = 0; s < RING; ++s) {
            mbar_init(smem_u32(&b_full[0][s]), 1);
            mbar_init(smem_u32(&b_full[1][s]), 33);           // the producer's expect and its lanes' scales
            mbar_init(smem_u32(&b_empty[0][s]), 1);
            mbar_init(smem_u32(&b_empty[1][s]), 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(smem_u32(&b_qfull[a]), 2);              // the two query warps
            mbar_init(smem_u32(&b_qempty[a]), 1 + 4 * NG);    // the MMAs and the softmax warps
            mbar_init(smem_u32(&b_l[a]), 4 * NG);
            mbar_init(smem_u32(&b_lfree[a]), 4);
            mbar_init(smem_u32(&b_drain[a]), 1);
            s_nan_any[a] = 0;
        }
        for (int g = 0; g < NG; ++g) {
            mbar_init(smem_u32(&b_s[g]), 1);
            mbar_init(smem_u32(&b_free[g]), 4);               // the four warps of a softmax group
            mbar_init(smem_u32(&b_p[g]), 4);
            mbar_init(smem_u32(&b_o[g]), 1);
            mbar_init(smem_u32(&b_ofree[g]), 4);              // the four accumulator warps
            mbar_init(smem_u32(&b_mt[g][0]), 1);
            mbar_init(smem_u32(&b_mt[g][1]), 1);
        }
        s_abort = 0;
        s_start_b = -1;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    for (int i = tid; i < 2 * N * (D / 32); i += kCaThreads) (&s_nan[0][0][0])[i] = 0u;
    if (warp == 2) tc_alloc(smem_u32(&s_tmem), L::kTmemCols);
    if (warp == 0 && lane < 2) {
        const CUtensorMap* tm = lane ? &tm_v : &tm_k;
        asm volatile("prefetch.tensormap [%0];" ::"l"(tm) : "memory");
    }
    pdl_enter();

    // ---- this CTA's share of the work ----
    const int per = (p.B + kCaThreads - 1) / kCaThreads;
    long long mine = 0;
#pragma unroll 1
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
#pragma unroll 1
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

    if (warp < 2) {
        // ========================= TMA producers: K (warp 0), V (warp 1) =========================
        // One warp could not issue the copies of 16-token blocks fast enough (106 to 133 cycles each, 4.3 TB/s measured
        // for one warp, 6.5 TB/s for two).  The block numbers of up to 32 blocks are fetched one group ahead, across items,
        // and the scales travel with cp.async on V's barrier: nothing here waits for memory.
        const int kv = warp;
        const uint32_t elected = ca_elect();
        uint32_t slot = 0, ph = 0, tile = 0;
        bool ok = true;
        const uint32_t page_bytes = (uint32_t)D << p.bt_log2;
        const int ppt_log2 = 7 - p.bt_log2;                   // blocks of a tile
        const CUtensorMap* tm = kv ? &tm_v : &tm_k;
        unsigned char* ring = smem + kv * RING * L::kTileBytes;
        auto group_tiles = [&](const CaCursor& c) {
            return (int)min(min((long long)(32 >> ppt_log2), c.end - c.x), (long long)(c.ntiles - c.t));
        };
        auto fetch = [&](const CaCursor& c, int tiles) {      // this lane's block of the group
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
            nxt.x += n_tiles;
            nxt.t += n_tiles;
            if (nxt.t == nxt.ntiles && nxt.x < nxt.end) ca_next(p, nxt);
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
                if (!ca_wait(smem_u32(&b_empty[kv][slot]), ph ^ 1u) || __any_sync(0xffffffffu, s_abort)) { ok = false; break; }
                const uint32_t bar = smem_u32(&b_full[kv][slot]);
                if (lane == 0) mbar_arrive_expect_tx(bar, pages * page_bytes);
                __syncwarp();
                uint32_t dst = smem_u32(ring + slot * L::kTileBytes);
#pragma unroll 1
                for (int i = 0; i < pages; ++i, dst += page_bytes)
                    ca_tma(dst, tm, __shfl_sync(0xffffffffu, ids, (j << ppt_log2) + i) * p.Hkv + cur.h, bar, elected);
                if (kv) {
                    const int blk = __shfl_sync(0xffffffffu, ids, ((j << ppt_log2) + lane) & 31);
                    if (lane < pages) {
                        // the ring of scales is deeper than that of V: its entry is free when the slot is
                        const uint32_t at = smem_u32(s_scale[tile % kCaScaleRing][lane]);
                        const size_t e = (size_t)blk * p.Hkv + cur.h;
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at), "l"(p.k_scale + e) : "memory");
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at + 4), "l"(p.v_scale + e) : "memory");
                    }
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
                }
                if (++slot == RING) { slot = 0; ph ^= 1u; }
            }
            cur = nxt;
            n_tiles = next_tiles;
            ids = next_ids;
        }
        if (!ok) {                                            // leave no copy in flight behind
            if (lane == 0) {
                s_abort = 1;
                if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
#pragma unroll 1
                for (uint32_t f = tile > RING ? tile - RING : 0u; f < tile; ++f)
                    mbar_wait(smem_u32(&b_full[kv][f % RING]), (f / RING) & 1);
            }
            __syncwarp();
        }
    } else if (warp == 2) {
        // ============================ MMA issuer of S^T = K Q^T ============================
        // runs NG tiles ahead: S of tile j is issued when that of tile j - NG has been taken out of tensor memory
        constexpr int kN = L::kCols;
        constexpr uint32_t idesc = (1u << 4) | ((uint32_t)(kN >> 3) << 17) | ((uint32_t)(kCaTile >> 4) << 24);
        const uint32_t elected = ca_elect();
        uint32_t j = 0, slot = 0, ph = 0;
        int item = 0;
        bool ok = true;
#pragma unroll 1
        while (cur.x < cur.end && ok) {
            const int nt = (int)min((long long)(cur.ntiles - cur.t), cur.end - cur.x);
            ok = ca_wait(smem_u32(&b_qfull[item & 1]), (uint32_t)((item >> 1) & 1));
            const uint64_t dq = ca_desc(smem_u32(s_q + (item & 1) * 2 * L::kQBytes), 128, 8 * D, 0);
#pragma unroll 1
            for (int t = 0; t < nt && ok; ++t, ++j) {
                const uint32_t g = j % NG;
                if ((j >= NG && !ca_wait(smem_u32(&b_free[g]), (j / NG - 1) & 1)) || !ca_wait(smem_u32(&b_full[0][slot]), ph) ||
                    __any_sync(0xffffffffu, s_abort)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint64_t dk = ca_desc(smem_u32(smem + slot * L::kTileBytes), 16, 8 * D, kSw);
#pragma unroll
                for (int term = 0; term < (L::kWide ? 1 : 2); ++term)
#pragma unroll
                    for (int s = 0; s < D / 32; ++s)
                        ca_mma(tmem + g * L::kCols, dk + ((s * 32) >> 4), dq + ((term * L::kQBytes + s * 256) >> 4), idesc,
                               (term | s) ? 1u : 0u, elected);
                ca_commit(smem_u32(&b_s[g]), elected);
                ca_commit(smem_u32(&b_empty[0][slot]), elected);
                if (++slot == RING) { slot = 0; ph ^= 1u; }
            }
            if (ok) ca_commit(smem_u32(&b_qempty[item & 1]), elected);
            ++item;
            cur.x += nt;
            cur.t += nt;
            if (cur.t == cur.ntiles && cur.x < cur.end) ca_next(p, cur);
        }
        if (!ok) {
            if (lane == 0) {
                s_abort = 1;
                if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
            }
            __syncwarp();
            ca_commit(smem_u32(&b_drain[0]), elected);        // leave no MMA in flight behind
            ca_wait(smem_u32(&b_drain[0]), 0);
        }
        __syncwarp();
    } else if (warp == 3) {
        // =========================== MMA issuer of O^T = V^T P^T ===========================
        constexpr int kN = L::kCols;
        constexpr uint32_t idesc = (1u << 4) | (1u << 15) | (1u << 16) | ((uint32_t)(kN >> 3) << 17) | ((uint32_t)(D >> 4) << 24);
        const uint32_t elected = ca_elect();
        const uint32_t total = (uint32_t)(cur.end - cur.x);
        uint32_t slot = 0, ph = 0;
        bool ok = true;
#pragma unroll 1
        for (uint32_t k = 0; k < total && ok; ++k) {
            const uint32_t g = k % NG;
            if (!ca_wait(smem_u32(&b_p[g]), (k / NG) & 1) || !ca_wait(smem_u32(&b_full[1][slot]), ph) ||
                (k >= NG && !ca_wait(smem_u32(&b_ofree[g]), (k / NG - 1) & 1)) || __any_sync(0xffffffffu, s_abort)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint64_t dv = ca_desc(smem_u32(smem + (RING + slot) * L::kTileBytes), 0, 8 * D, kSw);
            const uint64_t dp = ca_desc(smem_u32(s_p + g * 2 * L::kPBytes), 128, 2048, 0);
#pragma unroll
            for (int term = 0; term < (L::kWide ? 1 : 2); ++term)
#pragma unroll
                for (int s = 0; s < kCaTile / 32; ++s)
                    ca_mma(tmem + L::kColO + g * L::kCols, dv + ((s * 32 * D) >> 4), dp + ((term * L::kPBytes + s * 512) >> 4),
                           idesc, (term | s) ? 1u : 0u, elected);
            ca_commit(smem_u32(&b_o[g]), elected);
            ca_commit(smem_u32(&b_empty[1][slot]), elected);
            if (++slot == RING) { slot = 0; ph ^= 1u; }
        }
        if (!ok) {
            if (lane == 0) {
                s_abort = 1;
                if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
            }
            __syncwarp();
            ca_commit(smem_u32(&b_drain[1]), elected);
            ca_wait(smem_u32(&b_drain[1]), 0);
        }
        __syncwarp();
    } else if (warp >= 8 + 4 * NG) {
        // ================================== queries ==================================
        constexpr int kLanes = D / 8;                         // lanes of a row
        constexpr int kRows = 64 / kLanes;                    // rows per pass of the two warps
        const int qt = tid - 32 * (8 + 4 * NG), sub = qt / kLanes, piece = (qt % kLanes) * 8;
        int item = 0;
        bool ok = true;
#pragma unroll 1
        while (cur.x < cur.end && ok) {
            const int buf = item & 1;
            const int te = (int)min((long long)cur.ntiles, cur.t + (cur.end - cur.x));
            if (item >= 2) ok = ca_wait(smem_u32(&b_qempty[buf]), (uint32_t)(((item >> 1) - 1) & 1)) && !__any_sync(0xffffffffu, s_abort);
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
                uint2 hi, lo;
                ca_split4(f[0] * up, f[1] * up, f[2] * up, f[3] * up, hi.x, lo.x);
                ca_split4(f[4] * up, f[5] * up, f[6] * up, f[7] * up, hi.y, lo.y);
                unsigned char* at = q_hi + (r >> 3) * (8 * D) + (piece >> 4) * 128 + (r & 7) * 16 + (piece & 15);
                *reinterpret_cast<uint2*>(at) = hi;
                *reinterpret_cast<uint2*>(at + L::kQBytes) = lo;
                // a row with an infinity or a NaN has no softmax: its scale makes every result NaN
                if (piece == 0) s_c[buf][r] = r >= rows ? 0.f : fin ? p.scale_log2 * __uint_as_float((uint32_t)(127 - x) << 23) : __int_as_float(0x7fc00000);
            }
            if (p.node_parent && qt < 32) {                   // ancestors-or-self of node `lane`
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
        uint64_t racc[8];                                     // the accumulator where there is one group of rows
#pragma unroll 1
        while (cur.x < cur.end) {
            const int buf = item & 1;
            const int te = (int)min((long long)cur.ntiles, cur.t + (cur.end - cur.x));
            const int nt = te - cur.t;
            const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
            float m_run[(N + 31) / 32], l_run[(N + 31) / 32]; // rows lane, lane + 32
#pragma unroll
            for (int i = 0; i < (N + 31) / 32; ++i) { m_run[i] = -INFINITY; l_run[i] = 0.f; }
#pragma unroll 1
            for (int t = 0; t < nt; ++t, ++k) {
                const uint32_t g = k % NG, kk = k / NG;
                if (ok) ok = ca_wait(smem_u32(&b_mt[g][kk & 1]), (kk >> 1) & 1) && !__any_sync(0xffffffffu, s_abort);
                if (!ok) continue;
#pragma unroll
                for (int i = 0; i < (N + 31) / 32; ++i) {
                    const int r = i * 32 + lane;
                    if (r < N) {
                        const float mt = s_mt[g][kk & 1][r], mn = fmaxf(m_run[i], mt);
                        f_a[r] = mn == -INFINITY ? 1.f : ex2(m_run[i] - mn);
                        f_b[r] = mn == -INFINITY ? 0.f : ex2(mt - mn) * 0.00390625f;
                        m_run[i] = mn;
                    }
                }
                __syncwarp();
                ok = ca_wait(smem_u32(&b_o[g]), kk & 1);
                if (!ok) continue;
                tc_fence_after();
#pragma unroll 1
                for (int c = 0; c < N; c += 16) {
                    uint64_t x[8];
                    uint32_t old[16];
                    if (!L::kOne && t) ca_ld16(t_acc + c, old);
                    ca_result16<L::kWide>(t_lane + L::kColO + g * L::kCols + c, N, x);
                    if (!L::kOne && t) ca_ld16_wait(old);
                    float y[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        uint64_t a0, a1, b0, b1;
                        lds_2x2(f_b + c + i, b0, b1);
                        uint64_t y0 = mul2(x[i / 2], b0), y1 = mul2(x[i / 2 + 1], b1);
                        if (t) {
                            lds_2x2(f_a + c + i, a0, a1);
                            if (L::kOne) {
                                y0 = fma2(racc[i / 2], a0, y0);
                                y1 = fma2(racc[i / 2 + 1], a1, y1);
                            } else {
                                y0 = fma2(pk(__uint_as_float(old[i]), __uint_as_float(old[i + 1])), a0, y0);
                                y1 = fma2(pk(__uint_as_float(old[i + 2]), __uint_as_float(old[i + 3])), a1, y1);
                            }
                        }
                        if (L::kOne) {
                            racc[i / 2] = y0;
                            racc[i / 2 + 1] = y1;
                        } else {
                            upk(y0, y[i], y[i + 1]);
                            upk(y1, y[i + 2], y[i + 3]);
                        }
                    }
                    if (!L::kOne) ca_st16(t_acc + c, y);
                }
                if (!L::kOne) ca_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&b_ofree[g]));
            }
            // ---- end of the item, or of this CTA's part of it: the sums of the groups ----
            if (ok) ok = ca_wait(smem_u32(&b_l[buf]), (uint32_t)((item >> 1) & 1)) && !__any_sync(0xffffffffu, s_abort);
#pragma unroll
            for (int i = 0; i < (N + 31) / 32; ++i) {
                const int r = i * 32 + lane;
                if (r < N)
#pragma unroll
                    for (int g = 0; g < NG; ++g) {
                        const float2 x = s_ml[buf][g][r];
                        l_run[i] += x.y * (x.x == -INFINITY ? 0.f : ex2(x.x - m_run[i]));
                    }
            }
            // 16 rows of the accumulator; results that a NaN of a masked tile belongs to
            const bool nans = s_nan_any[buf] != 0;
            auto acc16 = [&](int c, float (&y)[16]) {
                if (L::kOne) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) upk(racc[i], y[2 * i], y[2 * i + 1]);
                } else {
                    uint32_t u[16];
                    ca_ld16(t_acc + c, u);
                    ca_ld16_wait(u);
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = __uint_as_float(u[i]);
                }
                if (nans && has_dim)
#pragma unroll 1
                    for (int r = 0; r < 16; ++r)
                        if ((s_nan[buf][c + r][dim >> 5] >> (dim & 31)) & 1u)
#pragma unroll
                            for (int i = 0; i < 16; ++i) y[i] = i == r ? __int_as_float(0x7fc00000) : y[i];
            };
            bool write = ok, joined = false;
            long long c_first = 0, c_last = 0;
            if (nt < cur.ntiles) {
                // part of an item: leave it in the workspace; the CTA that completes the item joins the parts
                const long long xi = cur.x - cur.t;           // the item's first tile over all work
                c_first = ((xi + 1) * grid - 1) / work;
                c_last = ((xi + cur.ntiles) * grid - 1) / work;
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
                if (wq == 0)
#pragma unroll
                    for (int i = 0; i < (N + 31) / 32; ++i)
                        if (i * 32 + lane < N) {
                            part[N * D + i * 32 + lane] = m_run[i];
                            part[N * D + N + i * 32 + lane] = l_run[i];
                        }
                __threadfence();
                if (ca_bar_any(1 + NG, 128, !ok)) { ok = false; break; }
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
                    // maxima and sums over the parts, for rows lane, lane + 32
#pragma unroll
                    for (int i = 0; i < (N + 31) / 32; ++i) {
                        const int r = i * 32 + lane;
                        float mm = -INFINITY, ll = 0.f;
                        if (r < N)
#pragma unroll 4
                            for (int c = (int)c_first; c <= (int)c_last; ++c) {
                                const float* q = p.partial + ((size_t)c * 2 + (c == c_first ? 1 : 0)) * L::kPiece + N * D;
                                const float mc = __ldcg(q + r), lc = __ldcg(q + N + r);
                                const float mn = fmaxf(mm, mc);
                                ll = (mm == -INFINITY ? ll * 0.f : ll * ex2(mm - mn)) + (mc == -INFINITY ? lc * 0.f : lc * ex2(mc - mn));
                                mm = mn;
                            }
                        m_run[i] = mm;
                        l_run[i] = ll;
                    }
                }
            }
            if (write) {
                __syncwarp();
#pragma unroll
                for (int i = 0; i < (N + 31) / 32; ++i) {
                    const int r = i * 32 + lane;
                    if (r < N) {
                        f_a[r] = l_run[i] == 0.f ? 0.f : 1.f / l_run[i];   // nothing seen: zeros
                        f_b[r] = m_run[i];
                    }
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
                            float v[16], mc[16];
#pragma unroll
                            for (int r = 0; r < 16; ++r) {
                                v[r] = c + r < rows && has_dim ? __ldcg(q + (c + r) * D + dim) : 0.f;
                                mc[r] = __ldcg(q + N * D + c + r);
                            }
#pragma unroll
                            for (int r = 0; r < 16; ++r)
                                y[r] = fmaf(v[r], mc[r] == -INFINITY ? 0.f : ex2(mc[r] - f_b[c + r]), y[r]);
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
            cur.x += nt;
            cur.t = te;
            if (cur.t == cur.ntiles && cur.x < cur.end) ca_next(p, cur);
        }
        if (!ok && lane == 0) {
            s_abort = 1;
            if (p.status) atomicOr(p.status, BS_DEV_TIMEOUT);
        }
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
        uint64_t rsum[8], rt[8];                              // where there is one group of rows: sums and exponents
        // A wait that gave up leaves `ok` false in its warp only; the warps of a group leave together, at a barrier.
#pragma unroll 1
        while (cur.x < cur.end) {
            const int buf = item & 1;
            const int te = (int)min((long long)cur.ntiles, cur.t + (cur.end - cur.x));
            const int nt = te - cur.t;
            const int limit = ca_limit(p, cur.base, cur.n, cur.rt);
            const int i0 = cur.rt * p.TQ, rows = min(p.TQ, cur.n - i0) * p.G;
            // positions below this are seen by every row of the item
            const int seen = p.node_parent ? cur.base : cur.base + i0 + 1;
            // the accumulator is through with the item two before this one, which used the same sums and marks
            if (ok && item >= 2) ok = ca_wait(smem_u32(&b_lfree[buf]), (uint32_t)(((item >> 1) - 1) & 1));
            float m_run[(N + 31) / 32];                       // running maxima of rows lane, lane + 32
#pragma unroll
            for (int i = 0; i < (N + 31) / 32; ++i) m_run[i] = -INFINITY;
            const int t_first = cur.t + (int)((g + NG - g0 % NG) % NG);

#pragma unroll 1
            for (int t = t_first; t < te; t += NG) {
                const uint32_t k = g0 + (uint32_t)(t - cur.t);   // running tile number
                const uint32_t kk = k / NG;
                const uint32_t vslot = k % RING;
                const bool first = t == t_first;
                if (ok) ok = ca_wait(smem_u32(&b_full[1][vslot]), (k / RING) & 1) &&
                             (!first || ca_wait(smem_u32(&b_qfull[buf]), (uint32_t)((item >> 1) & 1))) &&   // its constants
                             !__any_sync(0xffffffffu, s_abort);
                const int pos = t * kCaTile + tok;
                const bool masked = (t + 1) * kCaTile > seen;
                unsigned long long vis = ~0ull;               // rows that see this thread's token
                float ks = 0.f, lsv = 0.f, isv = 0.f;
                if (ok) {
                    if (masked) {
                        if (pos >= limit) vis = 0ull;
                        else if (!p.node_parent) {
                            const long long r0 = (long long)(pos - cur.base - i0) * p.G;
                            vis = r0 <= 0 ? ~0ull : r0 < 64 ? ~0ull << r0 : 0ull;
                        } else if (pos >= cur.base) {
                            vis = 0ull;
#pragma unroll 1
                            for (int i = 0; i * p.G < rows; ++i)
                                if ((s_anc[buf][i0 + i] >> (pos - cur.base)) & 1u) vis |= (~0ull >> (64 - p.G)) << (i * p.G);
                        }
                        const unsigned long long all = rows >= 64 ? ~0ull : (1ull << rows) - 1ull;
                        if ((vis & all) != all && ca_clean_v<D>(smem + (RING + vslot) * L::kTileBytes, tok, vis & all, &s_nan[buf][0][0]))
                            s_nan_any[buf] = 1;
                    }
                    if (vis) {
                        const float* sc = s_scale[k % kCaScaleRing][tok >> p.bt_log2];
                        const float sv = fmaxf(sc[1], 5.421010862e-20f);    // 2^-64
                        ks = sc[0];
                        lsv = __log2f(sv);
                        isv = __fdividef(1.f, sv);
                    }
                    ok = ca_wait(smem_u32(&b_s[g]), kk & 1);
                }
                const uint64_t ks2 = pk(ks, ks), lsv2 = pk(lsv, lsv), isv2 = pk(isv, isv);
                // Exponents t = S * ks * c + lsv of this thread's token, 16 rows at a time.
                auto exponents = [&](int c, uint64_t (&x)[8]) {
                    ca_result16<L::kWide>(t_s + c, N, x);
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        uint64_t c0, c1;
                        lds_2x2(&s_c[buf][c + 2 * i], c0, c1);
                        x[i] = fma2(mul2(x[i], ks2), c0, lsv2);
                        x[i + 1] = fma2(mul2(x[i + 1], ks2), c1, lsv2);
                    }
                    if (masked) {
                        const uint32_t v = (uint32_t)(vis >> c);
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            float a, b;
                            upk(x[i], a, b);
                            x[i] = pk((v >> (2 * i)) & 1u ? a : -INFINITY, (v >> (2 * i + 1)) & 1u ? b : -INFINITY);
                        }
                    }
                };
                if (ok) {
                    tc_fence_after();
                    // pass 1: maxima over the warp's 32 tokens
#pragma unroll 1
                    for (int c = 0; c < N; c += 16) {
                        uint64_t x[8];
                        exponents(c, x);
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            float e[4];
                            upk(x[i], e[0], e[1]);
                            upk(x[i + 1], e[2], e[3]);
                            // the same from every lane: cheaper than a branch
                            *reinterpret_cast<float4*>(&s_red[g][wq][c + 2 * i]) =
                                make_float4(ca_warp_max(e[0]), ca_warp_max(e[1]), ca_warp_max(e[2]), ca_warp_max(e[3]));
                            if (L::kOne) {
                                rt[i] = x[i];
                                rt[i + 1] = x[i + 1];
                            }
                        }
                    }
                    if (L::kOne) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&b_free[g]));
                    }
                }
                // The product of this group's last tile is done: its P may be overwritten.  It was issued after the accumulator
                // had taken the tile before it, so the maxima of that one may be overwritten, too.
                if (ok && k >= NG) ok = ca_wait(smem_u32(&b_o[g]), (kk - 1) & 1);
                if (ca_bar_any(1 + g, 128, !ok)) { ok = false; break; }
                // the tile's maxima over the four warps; factors of the sums, for this warp's own use
#pragma unroll
                for (int i = 0; i < (N + 31) / 32; ++i) {
                    const int r = i * 32 + lane;
                    if (r < N) {
                        const float mt = fmaxf(fmaxf(s_red[g][0][r], s_red[g][1][r]), fmaxf(s_red[g][2][r], s_red[g][3][r]));
                        const float mn = fmaxf(m_run[i], mt);
                        s_m[w8][r] = mt == -INFINITY ? 0.f : 8.f - mt;
                        s_a[w8][r] = mn == -INFINITY ? 1.f : ex2(m_run[i] - mn);
                        s_b[w8][r] = mn == -INFINITY ? 0.f : ex2(mt - mn) * 0.00390625f;
                        if (wq == 0) s_mt[g][kk & 1][r] = mt;
                        m_run[i] = mn;
                    }
                }
                __syncwarp();
                if (wq == 0 && lane == 0) mbar_arrive(smem_u32(&b_mt[g][kk & 1]));
                // pass 2: probabilities P'' (scaled by 2^8), their sums, their two e4m3 terms
                unsigned char* sp = s_p + g * 2 * L::kPBytes + (tok >> 3) * 128 + (tok & 7) * 16;
#pragma unroll 1
                for (int c = 0; c < N; c += 16) {
                    uint64_t x[8];
                    uint32_t old[16];
                    if (!L::kOne && !first) ca_ld16(t_l + c, old);
                    if (L::kOne) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) x[i] = rt[i];
                    } else {
                        exponents(c, x);
                        if (!first) ca_ld16_wait(old);
                    }
                    uint32_t hi[4], lo[4];
                    float y[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        uint64_t m0, m1, a0, a1, b0, b1;
                        lds_2x2(&s_m[w8][c + i], m0, m1);
                        lds_2x2(&s_b[w8][c + i], b0, b1);
                        float e[4];
                        upk(add2(x[i / 2], m0), e[0], e[1]);
                        upk(add2(x[i / 2 + 1], m1), e[2], e[3]);
#pragma unroll
                        for (int z = 0; z < 4; ++z) e[z] = ex2(e[z]);
                        uint64_t l0 = mul2(mul2(pk(e[0], e[1]), isv2), b0), l1 = mul2(mul2(pk(e[2], e[3]), isv2), b1);
                        if (!first) {
                            lds_2x2(&s_a[w8][c + i], a0, a1);
                            if (L::kOne) {
                                l0 = fma2(rsum[i / 2], a0, l0);
                                l1 = fma2(rsum[i / 2 + 1], a1, l1);
                            } else {
                                l0 = fma2(pk(__uint_as_float(old[i]), __uint_as_float(old[i + 1])), a0, l0);
                                l1 = fma2(pk(__uint_as_float(old[i + 2]), __uint_as_float(old[i + 3])), a1, l1);
                            }
                        }
                        if (L::kOne) {
                            rsum[i / 2] = l0;
                            rsum[i / 2 + 1] = l1;
                        } else {
                            upk(l0, y[i], y[i + 1]);
                            upk(l1, y[i + 2], y[i + 3]);
                        }
                        ca_split4(e[0], e[1], e[2], e[3], hi[i / 4], lo[i / 4]);
                    }
                    if (!L::kOne) ca_st16(t_l + c, y);
                    *reinterpret_cast<uint4*>(sp + (c >> 4) * 2048) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    *reinterpret_cast<uint4*>(sp + (c >> 4) * 2048 + L::kPBytes) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                if (!L::kOne) ca_st_wait();
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&b_p[g]));
                    if (!L::kOne) mbar_arrive(smem_u32(&b_free[g]));
                }
            }

            // ---- end of the item: this group's running maxima and sums ----
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_qempty[buf]));   // its constants have been read
            float l_run[(N + 31) / 32];
#pragma unroll
            for (int i = 0; i < (N + 31) / 32; ++i) l_run[i] = 0.f;
            if (t_first < te) {                               // over the lanes, then over the warps
#pragma unroll 1
                for (int c = 0; c < N; c += 16) {
                    float y[16];
                    if (L::kOne) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) upk(rsum[i], y[2 * i], y[2 * i + 1]);
                    } else {
                        uint32_t u[16];
                        ca_ld16(t_l + c, u);
                        ca_ld16_wait(u);
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = __uint_as_float(u[i]);
                    }
                    s_lred[g][wq][c + ca_sum_row(lane)] = ca_row_sums16(y, lane);
                }
                if (ca_bar_any(1 + g, 128, !ok)) { ok = false; break; }
#pragma unroll
                for (int i = 0; i < (N + 31) / 32; ++i) {
                    const int r = i * 32 + lane;
                    if (r < N) l_run[i] = (s_lred[g][0][r] + s_lred[g][1][r]) + (s_lred[g][2][r] + s_lred[g][3][r]);
                }
            }
            if (wq == 0)
#pragma unroll
                for (int i = 0; i < (N + 31) / 32; ++i)
                    if (i * 32 + lane < N) s_ml[buf][g][i * 32 + lane] = make_float2(m_run[i], l_run[i]);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&b_l[buf]));
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
    if (warp == 2) {
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
    return cuda_status(launch_pdl(kern, sm_count(), L::kThreads, L::kDynamic, st, tm[0], tm[1], p));
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
