// bs_cache_plan: block tables and slot maps of a round, built on the device from lengths that are on the
// device (accepted lengths, speculation lengths chosen by the bandit), so that a round needs no trip to the host.
//
// Free blocks are a stack.  For every sequence L = seq_len + kept tokens stay and n new ones come; it should
// hold ceil((L + n) / bt) blocks.  Surplus blocks go back first, in such an order that the j-th of them
// (counted over the sequences, ascending within one) becomes the (j + 1)-th from the top; then the j-th missing
// block is the (j + 1)-th from the top.  A round that is planned and given back whole leaves the stack as it was.
// Leading blocks that a sequence shares with others (n_shared) count as needed for ever: they are never returned.
//
// Everything is prefix sums over the batch, which is small (B <= 4096): one CTA.  It also writes the slots of an ordinary
// round; a large slot map (prompts) is written by a second launch over many CTAs from the finished tables.  Bound by
// latency: a handful of dependent loads and block-wide scans.  64 sequences take 6.4 us in a graph.
#include "bs_common.cuh"

#include <atomic>

namespace bs {

struct CachePlanParams {
    int32_t* seq_len;          // [B] in / out
    const int32_t* kept;       // [B] or NULL
    const int32_t* last_cu;    // [B + 1] or NULL: cu_new of the plan whose tokens `kept` counts; may be cu_new
    const int32_t* n_shared;   // [B] or NULL: leading blocks that are not the plan's to return
    const int32_t* n_new;      // [B]
    const uint8_t* active;     // [B] or NULL
    int32_t* block_table;      // [B, W] in / out
    int32_t* n_held;           // [B] in / out
    int32_t* free_blocks;      // [n_blocks] in / out
    int32_t* n_free;           // [1] in / out
    int32_t* kv_len;           // [B]
    int32_t* cu_new;           // [B + 1]
    int32_t* slot_map;         // [T]
    int32_t* positions;        // [T] or NULL
    int32_t* status;           // [B] or NULL
    int extra, bt_log2, B, W, n_blocks, T;
    int inline_slots;          // slot_map and positions are written here
};

constexpr int kPlanThreads = 1024;
constexpr int kSlotThreads = 256;
// Slots that the planning CTA writes itself; larger maps take a launch of their own.  64 sequences, planned and given
// back, one launch against two: 512 slots 18.4 and 26.6 us, 4096 20.5 and 24.6, 8192 22.5 and 22.5, 16384 28.7 and 22.5,
// 65536 61 and 25.
constexpr int kPlanSlotsInline = 8192;

// Inclusive prefix sum over the CTA's threads of a pair of counts; `total` is the sum over all of them.
__device__ __forceinline__ longlong2 plan_scan(longlong2 v, longlong2* s_w, longlong2& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
        if (lane >= o) { v.x += x; v.y += y; }
    }
    __syncthreads();                                   // s_w of the scan before this one has been read
    if (lane == 31) s_w[warp] = v;
    __syncthreads();
    longlong2 w = s_w[lane];                           // kPlanThreads / 32 = 32 warps
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, w.x, o), y = __shfl_up_sync(0xffffffffu, w.y, o);
        if (lane >= o) { w.x += x; w.y += y; }
    }
    total.x = __shfl_sync(0xffffffffu, w.x, 31);
    total.y = __shfl_sync(0xffffffffu, w.y, 31);
    const long long bx = __shfl_sync(0xffffffffu, w.x, (warp + 31) & 31), by = __shfl_sync(0xffffffffu, w.y, (warp + 31) & 31);
    if (warp) { v.x += bx; v.y += by; }
    return v;
}

__global__ void __launch_bounds__(kPlanThreads) cache_plan_kernel(const CachePlanParams p) {
    extern __shared__ int32_t plan_smem[];
    __shared__ longlong2 s_w[kPlanThreads / 32];
    int32_t* s_cu = plan_smem;                         // [B + 1] first new token of each sequence
    int32_t* s_len = s_cu + p.B + 1;                   // [B] L
    int32_t* s_held = s_len + p.B;                     // [B] blocks held before
    int32_t* s_rank = s_held + p.B;                    // [B] rank of the first block returned or taken
    int32_t* s_delta = s_rank + p.B;                   // [B] blocks taken (> 0) or returned (< 0)
    int32_t* s_new = s_delta + p.B;                    // [B] new tokens granted
    int32_t* s_bits = s_new + p.B;                     // [B] status bits
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bt = 1 << p.bt_log2;
    pdl_enter();

    // ---- lengths; what does not fit the slot map is refused ----
    const int n_free = min(max(__ldcg(p.n_free), 0), p.n_blocks);
    longlong2 total, carry = make_longlong2(0, 0);
    long long returned = 0;
    for (int b0 = 0; b0 < p.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        long long L = 0, n = 0;
        int held = 0, shared = 0, bits = 0;
        if (b < p.B) {
            const bool act = !p.active || p.active[b];
            const int len = __ldcg(p.seq_len + b);
            int keep = act && p.kept ? p.kept[b] : 0;
            if (keep > 0 && p.last_cu) {                       // of no new tokens none stay, whatever was verified
                const int got = p.last_cu[b + 1] - p.last_cu[b];
                keep = got <= 0 ? 0 : keep > got ? -1 : keep;
            }
            held = __ldcg(p.n_held + b);
            L = (long long)len + keep;
            n = act ? (long long)p.n_new[b] + p.extra : 0;
            shared = p.n_shared ? p.n_shared[b] : 0;
            if (len < 0 || keep < 0 || n < 0 || held < 0 || held > p.W || L > (long long)held * bt ||
                L + n > (long long)p.W * bt || shared < 0 || shared > held ||
                (n > 0 && L < (long long)shared * bt)) {       // its tokens would be written into shared blocks
                bits = BS_DEV_BAD_LENGTH;
                n = 0;
            }
        }
        const longlong2 inc = plan_scan(make_longlong2(n, 0), s_w, total);
        if (n > 0 && carry.x + inc.x > p.T) bits |= BS_DEV_NO_ROOM;
        carry.x += total.x;
        const int delta = bits || b >= p.B ? 0 : max((int)((L + n + bt - 1) >> p.bt_log2), shared) - held;
        if (b < p.B) {
            s_len[b] = (int)((bits & BS_DEV_BAD_LENGTH) ? 0 : L);
            s_held[b] = held;
            s_delta[b] = delta;
            s_new[b] = bits ? 0 : (int)n;
            s_bits[b] = bits;
        }
        plan_scan(make_longlong2(delta < 0 ? -delta : 0, 0), s_w, total);
        returned += total.x;
    }
    // ---- blocks: who takes, who gives, at which rank ----
    const long long avail = (long long)n_free + returned;
    carry = make_longlong2(0, 0);
    long long taken = 0;
    int new_carry = 0;
    for (int b0 = 0; b0 < p.B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        const int delta = b < p.B ? s_delta[b] : 0;
        const longlong2 mine = make_longlong2(delta > 0 ? delta : 0, delta < 0 ? -delta : 0);
        const longlong2 inc = plan_scan(mine, s_w, total);
        const bool refused = delta > 0 && carry.x + inc.x > avail;
        // takes are refused from some sequence on, so the ranks of those before it are their plain prefix sums
        if (b < p.B) {
            s_rank[b] = (int)(delta > 0 ? carry.x + inc.x - mine.x : carry.y + inc.y - mine.y);
            if (refused) { s_delta[b] = 0; s_new[b] = 0; s_bits[b] |= BS_DEV_NO_BLOCKS; }
        }
        carry.x += total.x;
        carry.y += total.y;
        const longlong2 cu = plan_scan(make_longlong2(b < p.B ? s_new[b] : 0, delta > 0 && !refused ? delta : 0), s_w, total);
        if (b < p.B) s_cu[b + 1] = new_carry + (int)cu.x;
        new_carry += (int)total.x;
        taken += total.y;
    }
    if (tid == 0) s_cu[0] = 0;
    __syncthreads();

    // ---- per-sequence results; surplus blocks go back ----
    for (int b = tid; b < p.B; b += kPlanThreads) {
        const int bits = s_bits[b];
        if (!(bits & BS_DEV_BAD_LENGTH)) p.seq_len[b] = s_len[b];
        p.n_held[b] = s_held[b] + s_delta[b];
        p.kv_len[b] = s_len[b] + s_new[b];
        p.cu_new[b + 1] = s_cu[b + 1];
        if (p.status) p.status[b] = bits;
    }
    if (tid == 0) {
        p.cu_new[0] = 0;
        *p.n_free = (int)(avail - taken);
    }
    const int top = (int)avail;
    if (returned) {
        for (int b = warp; b < p.B; b += kPlanThreads / 32) {
            const int give = -s_delta[b];
            for (int j = lane; j < give; j += 32) {
                int32_t* e = p.block_table + (size_t)b * p.W + (s_held[b] - give + j);
                const int at = top - 1 - (s_rank[b] + j);
                if (at >= 0 && at < p.n_blocks) p.free_blocks[at] = *e;
                *e = -1;
            }
        }
        __syncthreads();
    }
    // ---- missing blocks are taken ----
    if (taken) {
        for (int b = warp; b < p.B; b += kPlanThreads / 32) {
            const int take = s_delta[b];
            for (int j = lane; j < take; j += 32) {
                const int at = top - 1 - (s_rank[b] + j);
                p.block_table[(size_t)b * p.W + s_held[b] + j] = at < p.n_blocks ? __ldcg(p.free_blocks + at) : -1;
            }
        }
    }
    // ---- slots: a token's block is in the table from before, or the one taken above (read from the stack, where
    //      nobody writes any more) ----
    if (!p.inline_slots) return;
    const int T_new = s_cu[p.B];
    int b = 0;
    for (int i = tid; i < p.T; i += kPlanThreads) {
        int slot = -1, pos = -1;
        if (i < T_new) {
            int lo = b, hi = p.B;                      // the last sequence with s_cu[b] <= i; i only grows
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s_cu[mid] <= i) lo = mid; else hi = mid;
            }
            b = lo;
            pos = s_len[b] + (i - s_cu[b]);
            const int pg = pos >> p.bt_log2, held = s_held[b];
            int blk;
            if (pg < held) {
                blk = __ldcg(p.block_table + (size_t)b * p.W + pg);
            } else {
                const int at = top - 1 - (s_rank[b] + pg - held);
                blk = at < p.n_blocks ? __ldcg(p.free_blocks + at) : -1;
            }
            if (blk >= 0 && blk < p.n_blocks) slot = (blk << p.bt_log2) + (pos & (bt - 1));
        }
        p.slot_map[i] = slot;
        if (p.positions) p.positions[i] = pos;
    }
}

// The slots of a large map, from what cache_plan_kernel wrote: a warp takes 128 tokens, whose sequences lie close together.
__global__ void __launch_bounds__(kSlotThreads) cache_slots_kernel(const CachePlanParams p) {
    pdl_enter();
    const int T_new = __ldcg(p.cu_new + p.B);
    const int lane = threadIdx.x & 31;
    const int first = (blockIdx.x * (kSlotThreads / 32) + (threadIdx.x >> 5)) * 128;
    int b = 0, from = 0, to = 0;                       // tokens of the sequence looked up last
#pragma unroll 1
    for (int q = 0; q < 4; ++q) {
        const int i = first + q * 32 + lane;
        if (i >= p.T) break;
        int slot = -1, pos = -1;
        if (i < T_new) {
            if (i >= to) {
                int lo = b, hi = p.B;                  // the last sequence with cu_new[b] <= i
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (__ldcg(p.cu_new + mid) <= i) lo = mid; else hi = mid;
                }
                b = lo;
                from = __ldcg(p.cu_new + b);
                to = __ldcg(p.cu_new + b + 1);
            }
            pos = __ldcg(p.seq_len + b) + i - from;
            const int blk = __ldcg(p.block_table + (size_t)b * p.W + (pos >> p.bt_log2));
            if (blk >= 0 && blk < p.n_blocks) slot = (blk << p.bt_log2) + (pos & ((1 << p.bt_log2) - 1));
        }
        p.slot_map[i] = slot;
        if (p.positions) p.positions[i] = pos;
    }
}

static std::atomic<bool> g_plan_attr[64];

}  // namespace bs

using namespace bs;

extern "C" bs_status bs_cache_plan_next(int32_t* seq_len, const int32_t* kept, const int32_t* last_cu,
                                        const int32_t* n_shared, const int32_t* n_new, int extra, const uint8_t* active, int B,
                                        int block_tokens, int32_t* block_table, int max_blocks, int32_t* n_held,
                                        int32_t* free_blocks, int n_blocks, int32_t* n_free, int32_t* kv_len, int32_t* cu_new,
                                        int32_t* slot_map, int32_t* positions, int T, int32_t* status, void* stream) {
    if (B < 1 || max_blocks < 1 || n_blocks < 1 || T < 1 || extra < 0) return BS_ERR_INVALID_ARG;
    if (!seq_len || !n_new || !block_table || !n_held || !free_blocks || !n_free || !kv_len || !cu_new || !slot_map)
        return BS_ERR_INVALID_ARG;
    int lg = 4;
    while (lg < 7 && (1 << lg) != block_tokens) ++lg;
    if ((1 << lg) != block_tokens) return BS_ERR_UNSUPPORTED;
    // slots and ranks are 32 bits wide
    if (B > BS_MAX_BATCH || max_blocks > BS_MAX_SEQ_BLOCKS || extra > (1 << 20) ||
        ((long long)n_blocks << lg) > 0x7fffffffLL)
        return BS_ERR_UNSUPPORTED;
    CachePlanParams p;
    p.seq_len = seq_len; p.kept = kept; p.last_cu = last_cu; p.n_shared = n_shared; p.n_new = n_new; p.active = active;
    p.block_table = block_table; p.n_held = n_held; p.free_blocks = free_blocks; p.n_free = n_free; p.kv_len = kv_len; p.cu_new = cu_new;
    p.slot_map = slot_map; p.positions = positions; p.status = status;
    p.extra = extra; p.bt_log2 = lg; p.B = B; p.W = max_blocks; p.n_blocks = n_blocks; p.T = T;
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64) dev = 0;
    const size_t smem = sizeof(int32_t) * (7 * (size_t)B + 1);
    if (!g_plan_attr[dev]) {
        if (cudaFuncSetAttribute(cache_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)(sizeof(int32_t) * (7 * BS_MAX_BATCH + 1))) != cudaSuccess)
            return cuda_status(cudaGetLastError());
        g_plan_attr[dev] = true;
    }
    p.inline_slots = T <= kPlanSlotsInline;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = launch_pdl(cache_plan_kernel, 1, kPlanThreads, smem, st, p);
    if (e != cudaSuccess || p.inline_slots) return cuda_status(e);
    return cuda_status(launch_pdl(cache_slots_kernel, (unsigned)(((long long)T + 1023) / 1024), kSlotThreads, 0, st, p));
}

extern "C" bs_status bs_cache_plan(int32_t* seq_len, const int32_t* kept, const int32_t* n_new, int extra,
                                   const uint8_t* active, int B, int block_tokens, int32_t* block_table, int max_blocks,
                                   int32_t* n_held, int32_t* free_blocks, int n_blocks, int32_t* n_free, int32_t* kv_len,
                                   int32_t* cu_new, int32_t* slot_map, int32_t* positions, int T, int32_t* status,
                                   void* stream) {
    return bs_cache_plan_next(seq_len, kept, nullptr, nullptr, n_new, extra, active, B, block_tokens, block_table, max_blocks,
                              n_held, free_blocks, n_blocks, n_free, kv_len, cu_new, slot_map, positions, T, status, stream);
}
