// bs_logits_adjust and bs_history_update: what is done to the logits of a round before they are verified, and the token
// history that it reads.
//
//   x = logit;  seen (in the prompt, emitted, or drafted on the way to this row): x = x > 0 ? x / r : x r
//   x -= f c + p [c > 0],  c = times emitted or drafted on the way;   x += bias;   forbidden by the row's grammar mask: -inf
//
// adjust: bound by HBM, the rows are read and written once, the history once for all rows of a sequence.  A warp takes 256 tokens of
// the vocabulary of one sequence, eight a lane.  Few of them change by more than the mask (700 tokens of a history in 152064 are one in
// a warp), so the rows are copied as they are, masked in the type's own bits, and the elements that change are mended behind it,
// each in each row by a lane.  With the arithmetic in the rows for all elements the kernel was bound by instructions (73 us instead of
// 56 for 64 sequences of 3 to 9 bf16 rows of 152064: 0.25 GB, 4.6 TB/s; rows with masks alone 6.2).  Where many change
// (frequent tokens, long histories on small vocabularies) the rows are worked on whole.  Two rows of bf16 in flight and 48 warps an SM
// were faster than four rows and 32 warps.  Biases are added in the order of the list, so that sums do not depend on timing.
// In place, only what is forbidden and those elements are written, nothing else is read.
//
// history: entries of 16 bits, 2 x (times emitted, up to 16383) + (in the prompt).  A history that begins anew is built in
// shared memory piece by piece and written once; what a round adds goes to its few entries by compare-and-swap.  Only whole
// numbers are added: the order does not show.
#include "bs_common.cuh"
#include "bs_overlap.cuh"

namespace bs {

// Ancestors of node `lane` in a tree, itself included (bit n: node n; the root is bit 0): lane n holds the parent of node n.
__device__ __forceinline__ uint32_t tree_ancestors(int parent, int nodes) {
    const int lane = threadIdx.x & 31;
    uint32_t anc = 1u << lane;
    for (int n = 1; n <= nodes; ++n) {                        // parents come before their children
        const int up = __shfl_sync(0xffffffffu, parent, n);
        const uint32_t of_up = __shfl_sync(0xffffffffu, anc, up);
        if (lane == n) anc |= of_up;
    }
    return anc | 1u;
}

struct AdjustParams {
    const void* x;
    void* y;
    const int32_t* gamma;
    const int32_t* draft_tokens;
    const int32_t* node_parent;
    const int16_t* history;
    const float *repetition, *presence, *frequency;
    const int32_t *bias_begin, *bias_tokens;
    const float* bias_values;
    const uint32_t* masks;
    const int32_t* mask_row;
    int32_t* status;
    int extra, row_begin, row_end, B, R, N, V, n_masks, n_bias, in_place;
};

constexpr int kAdWarps = 4;
constexpr int kAdLane = 8;                     // tokens of a lane
constexpr int kAdWarp = 32 * kAdLane;          // of a warp
constexpr int kAdFew = 32;                     // elements of a warp that are mended one by one: up to about 40 it is less work than in the rows

// Eight elements of a lane.  VEC: neighbours, two or one 16-byte accesses of all of them; else 32 apart, one by one, for rows that
// begin anywhere.  `need`: a bit for each element.
template <typename T, bool VEC> struct AdIo;
template <typename T> struct AdIo<T, true> {
    static constexpr int kWords = (int)sizeof(T) * 2;
    __device__ static __forceinline__ void load(const T* p, uint32_t need, uint32_t (&w)[kWords]) {
        if (!need) return;
#pragma unroll
        for (int i = 0; i < kWords; i += 4) {
            const uint4 v = __ldcg(reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) + 4 * i));
            w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
        }
    }
    __device__ static __forceinline__ void store(T* p, uint32_t need, const uint32_t (&w)[kWords]) {
        if (!need) return;
#pragma unroll
        for (int i = 0; i < kWords; i += 4)
            __stcg(reinterpret_cast<uint4*>(reinterpret_cast<char*>(p) + 4 * i), make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]));
    }
};
template <> struct AdIo<float, false> {
    static constexpr int kWords = 8;
    __device__ static __forceinline__ void load(const float* p, uint32_t need, uint32_t (&w)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((need >> e) & 1u) w[e] = __float_as_uint(p[32 * e]);
    }
    __device__ static __forceinline__ void store(float* p, uint32_t need, const uint32_t (&w)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((need >> e) & 1u) p[32 * e] = __uint_as_float(w[e]);
    }
};
template <> struct AdIo<__nv_bfloat16, false> {
    static constexpr int kWords = 4;
    __device__ static __forceinline__ void load(const __nv_bfloat16* p, uint32_t need, uint32_t (&w)[4]) {
        const unsigned short* u = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((need >> e) & 1u) w[e >> 1] |= (uint32_t)u[32 * e] << (16 * (e & 1));
    }
    __device__ static __forceinline__ void store(__nv_bfloat16* p, uint32_t need, const uint32_t (&w)[4]) {
        unsigned short* u = reinterpret_cast<unsigned short*>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((need >> e) & 1u) u[32 * e] = (unsigned short)(w[e >> 1] >> (16 * (e & 1)));
    }
};
__device__ __forceinline__ void ad_unpack(const uint32_t (&w)[8], float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(w[e]);
}
__device__ __forceinline__ void ad_unpack(const uint32_t (&w)[4], float (&f)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        f[2 * e] = __uint_as_float(w[e] << 16);
        f[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
}
__device__ __forceinline__ void ad_pack(const float (&f)[8], uint32_t (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = __float_as_uint(f[e]);
}
__device__ __forceinline__ void ad_pack(const float (&f)[8], uint32_t (&w)[4]) {   // the one rounding
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
        w[e] = *reinterpret_cast<const uint32_t*>(&b);
    }
}
// One element; in place it may just have been written by another lane.
__device__ __forceinline__ float ad_one(const float* p) { return __ldcg(p); }
__device__ __forceinline__ float ad_one(const __nv_bfloat16* p) {
    return __uint_as_float((uint32_t)__ldcg(reinterpret_cast<const unsigned short*>(p)) << 16);
}
// What is not allowed becomes -inf, in the type's own bits.
__device__ __forceinline__ void ad_forbid(uint32_t allowed, uint32_t (&w)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (!((allowed >> e) & 1u)) w[e] = 0xff800000u;
}
__device__ __forceinline__ void ad_forbid(uint32_t allowed, uint32_t (&w)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t keep = ((allowed >> (2 * e)) & 1u ? 0x0000ffffu : 0u) | ((allowed >> (2 * e + 1)) & 1u ? 0xffff0000u : 0u);
        w[e] = (w[e] & keep) | (0xff80ff80u & ~keep);
    }
}

// The biases of this warp's 256 tokens, summed into s_sum in the order of the list; true if there are any.  Every warp looks
// through the list by itself, 128 entries at a time.
__device__ __forceinline__ bool ad_biases(const AdjustParams& p, int lo, int hi, int v0, int& bits, float* s_sum) {
    const int lane = threadIdx.x & 31;
    bool found = false;
#pragma unroll 1
    for (uint32_t i = lo + lane; i - lane < (uint32_t)hi; i += 128) {   // behind the last entry 31 bits do not hold it
        int t[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = i + 32 * k < (uint32_t)hi ? __ldg(p.bias_tokens + i + 32 * k) : p.V;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (i + 32 * k < (uint32_t)hi && (t[k] < 0 || t[k] >= p.V)) bits |= BS_DEV_BAD_TOKEN;
            const int off = t[k] - v0;
            const bool hit = off >= 0 && off < kAdWarp && t[k] < p.V;
            if (!__any_sync(0xffffffffu, hit)) continue;
            if (!found) {
#pragma unroll
                for (int e = 0; e < 8; ++e) s_sum[32 * e + lane] = 0.f;
                found = true;
            }
            const float v = hit ? __ldg(p.bias_values + i + 32 * k) : 0.f;
            // entries of the same token one after the other, the others at once
            const uint32_t same = __match_any_sync(0xffffffffu, hit ? off : -1);
            int turn = __popc(same & ((1u << lane) - 1u));
            const int turns = __reduce_max_sync(0xffffffffu, hit ? turn + 1 : 0);
            for (int z = 0; z < turns; ++z) {
                __syncwarp();
                if (hit && turn == z) s_sum[off] += v;
            }
        }
    }
    __syncwarp();
    return found;
}

template <typename T, bool VEC>
__global__ void __launch_bounds__(kAdWarps * 32, 12) logits_adjust_kernel(const AdjustParams p) {
    using Io = AdIo<T, VEC>;
    __shared__ float s_sum[kAdWarps][kAdWarp];                // biases
    __shared__ float2 s_list[kAdWarps][kAdFew];               // elements that change
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = blockIdx.x;
    const int v0 = ((int)blockIdx.y * kAdWarps + warp) * kAdWarp;
    pdl_enter();
    const int first = VEC ? v0 + lane * kAdLane : v0 + lane;  // token of element 0
    // elements of this lane that are there (VEC: V is a multiple of 8)
    const uint32_t there = VEC ? (first < p.V ? 0xffu : 0u)
                               : (first < p.V ? 0xffu >> (7 - min(7, (p.V - 1 - first) >> 5)) : 0u);
    const bool pen = p.repetition || p.presence || p.frequency;
    uint32_t h[4] = {0u, 0u, 0u, 0u};
    if (pen && p.history)
        AdIo<__nv_bfloat16, VEC>::load(reinterpret_cast<const __nv_bfloat16*>(p.history) + (size_t)b * p.V + first, there, h);
    const float rep = p.repetition ? __ldg(p.repetition + b) : 1.f, pres = p.presence ? __ldg(p.presence + b) : 0.f,
                freq = p.frequency ? __ldg(p.frequency + b) : 0.f;
    int mask = p.mask_row && lane < p.R ? __ldg(p.mask_row + (size_t)b * p.R + lane) : -1;   // of row `lane`
    int tok = -1, parent = 0;                                 // drafted token `lane`; parent of node `lane`
    if (pen && p.draft_tokens) {
        if (lane < p.N) tok = __ldg(p.draft_tokens + (size_t)b * p.N + lane);
        if (p.node_parent && lane >= 1 && lane <= p.N) parent = __ldg(p.node_parent + (size_t)b * p.N + lane - 1);
    }
    int bits = 0, rows = p.row_end;
    if (p.gamma) {
        int g = __ldg(p.gamma + b);
        if (g < 0 || g > p.R - p.extra) { g = 0; bits |= BS_DEV_BAD_GAMMA; }   // no sum: it could pass 32 bits
        rows = min(rows, g + p.extra);
    }
    if (rows <= p.row_begin && !(p.status && blockIdx.y == 0)) return;   // the whole CTA
    uint32_t any = 0u;                                        // elements with a bias, then those that are seen, too
    bool biased = false;
    if (p.bias_begin) {
        const int lo = __ldg(p.bias_begin + b), hi = __ldg(p.bias_begin + b + 1);
        if (lo < 0 || hi > p.n_bias || lo > hi) {
            bits |= BS_DEV_BAD_LENGTH;
        } else if (ad_biases(p, lo, hi, v0, bits, s_sum[warp])) {
            biased = true;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (s_sum[warp][VEC ? lane * 8 + e : 32 * e + lane] != 0.f) any |= 1u << e;
        }
    }
    if (mask < -1 || mask >= p.n_masks) {
        mask = -1;
        if (lane >= p.row_begin && lane < rows) bits |= BS_DEV_BAD_MASK;
    }
    // the rows of this sequence (a bit each) that stand behind drafted token `lane`
    uint32_t behind = 0u;
    if (pen && p.draft_tokens) {
        if (p.node_parent) {
            if (parent < 0 || (lane > 0 && parent >= lane)) {
                if (lane < rows) bits |= BS_DEV_BAD_TREE;
                parent = 0;
            }
            const uint32_t anc = tree_ancestors(parent, min(p.N, rows - 1));
#pragma unroll 1
            for (int r = 1; r < rows; ++r) {                  // node lane + 1 among the ancestors of node r
                const uint32_t of_row = __shfl_sync(0xffffffffu, anc, r);
                if (lane < 31 && (of_row >> (lane + 1)) & 1u) behind |= 1u << r;
            }
        } else {
            behind = lane < rows - 1 ? ~0u >> (32 - rows) & ~1u << lane : 0u;
        }
        if (lane < p.N && (tok < 0 || tok >= p.V) && lane < rows - 1) bits |= BS_DEV_BAD_TOKEN;
    }
    if (p.status && blockIdx.y == 0) {
        if (bits) atomicOr(p.status + b, bits);
        if (rows <= p.row_begin) return;
    }
    const uint32_t drafted = __ballot_sync(0xffffffffu, behind && tok >= v0 && tok < min(v0 + kAdWarp, p.V));

    auto past = [&](int e) { return (h[e >> 1] >> (16 * (e & 1))) & 0xffffu; };   // of an element
    // What is added to an element in every row.  Both ways of working below do x g + addend in one rounding and then subtract for the
    // drafted tokens one after the other: a row's bits do not show which of them it was.  -0 leaves every x as it is.
    auto bias_of = [&](int off) {
        const float a = biased ? s_sum[warp][off] : 0.f;
        return a == 0.f ? -0.f : a;
    };
    auto addend = [&](float bias, uint32_t times) { return times ? bias - fmaf(freq, (float)times, pres) : bias; };
    if (h[0] | h[1] | h[2] | h[3]) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (past(e)) any |= 1u << e;
    }
    any &= there;
    const float inv = 1.f / rep;
    const T* x = reinterpret_cast<const T*>(p.x) + (size_t)b * p.R * p.V + first;
    T* y = reinterpret_cast<T*>(p.y) + (size_t)b * p.R * p.V + first;
    const size_t mask_words = (size_t)((p.V + 31) >> 5);
    // what of a lane's elements the drafted tokens before a row fall on
    auto drafted_on = [&](int row, auto&& found) {
        uint32_t d = drafted;
#pragma unroll 1
        while (d) {
            const int l = __ffs(d) - 1;
            d &= d - 1;
            const int t = __shfl_sync(0xffffffffu, tok, l) - v0;
            const uint32_t rr = __shfl_sync(0xffffffffu, behind, l);
            if ((VEC ? t >> 3 : t & 31) == lane && ((rr >> (row & 31)) & 1u)) found(VEC ? t & 7 : t >> 5);
        }
    };

    // ---- few elements of this warp change by more than the mask, the usual case: rows are copied, those elements mended behind it ----
    uint32_t mine = any;                                      // drafted tokens among them, whatever the row
    for (uint32_t d = drafted; d; d &= d - 1) {
        const int t = __shfl_sync(0xffffffffu, tok, __ffs(d) - 1) - v0;
        if ((VEC ? t >> 3 : t & 31) == lane) mine |= 1u << (VEC ? t & 7 : t >> 5);
    }
    const int count = __reduce_add_sync(0xffffffffu, __popc(mine));
    if (count <= kAdFew) {
        if (p.in_place) {                                     // only what is forbidden is written, nothing read
            const uint32_t bit = 1u << lane;
            T* at = reinterpret_cast<T*>(p.y) + ((size_t)b * p.R + p.row_begin) * p.V + v0 + lane;
            auto word_of = [&](int r) {                       // lane e < 8: tokens v0 + 32 e ..
                const int m = __shfl_sync(0xffffffffu, mask, r & 31);
                return m >= 0 && r < rows && lane < 8 && v0 + 32 * lane < p.V ? __ldg(p.masks + (size_t)m * mask_words + (v0 >> 5) + lane) : ~0u;
            };
            uint32_t next = word_of(p.row_begin);
#pragma unroll 1
            for (int r = p.row_begin; r < rows; ++r, at += p.V) {
                const uint32_t word = next;
                next = word_of(r + 1);
                if (!__any_sync(0xffffffffu, word != ~0u)) continue;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t word_e = __shfl_sync(0xffffffffu, word, e);
                    if (!(word_e & bit) && v0 + lane + 32 * e < p.V) at[32 * e] = static_cast<T>(-INFINITY);
                }
            }
        } else {
            constexpr int kRows = 4 / sizeof(T);              // in flight: 32 bytes a lane
#pragma unroll 1
            for (int r0 = p.row_begin; r0 < rows; r0 += kRows) {
                uint32_t w[kRows][Io::kWords], allowed[kRows];
#pragma unroll
                for (int k = 0; k < kRows; ++k) {
                    const int m = __shfl_sync(0xffffffffu, mask, (r0 + k) & 31);
                    allowed[k] = there;
                    if (m >= 0 && r0 + k < rows) {
                        const uint32_t* words = p.masks + (size_t)m * mask_words + (v0 >> 5);
                        if (VEC) {
                            if (there) allowed[k] = __ldg(reinterpret_cast<const unsigned char*>(words) + lane);
                        } else {
                            const uint32_t word = lane < 8 && v0 + 32 * lane < p.V ? __ldg(words + lane) : 0u;
                            uint32_t a = 0u;
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if ((__shfl_sync(0xffffffffu, word, e) >> lane) & 1u) a |= 1u << e;
                            allowed[k] = a & there;
                        }
                    }
                }
#pragma unroll
                for (int k = 0; k < kRows; ++k) {
#pragma unroll
                    for (int i = 0; i < Io::kWords; ++i) w[k][i] = 0u;
                    if (r0 + k < rows) Io::load(x + (size_t)(r0 + k) * p.V, allowed[k], w[k]);
                }
#pragma unroll
                for (int k = 0; k < kRows; ++k)
                    if (r0 + k < rows) {
                        if (allowed[k] != there) ad_forbid(allowed[k], w[k]);
                        Io::store(y + (size_t)(r0 + k) * p.V, there, w[k]);
                    }
            }
        }
        if (!count) return;
        // the elements, one behind the other: place in the warp's tokens and history, bias
        float2* list = s_list[warp];
        int at = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t who = __ballot_sync(0xffffffffu, (mine >> e) & 1u);
            if (!who) continue;
            const int off = VEC ? lane * 8 + e : 32 * e + lane;
            if ((mine >> e) & 1u)
                list[at + __popc(who & ((1u << lane) - 1u))] = make_float2(__int_as_float(off | past(e) << 16), bias_of(off));
            at += __popc(who);
        }
        __syncwarp();                                         // behind it, too: what the other lanes have stored of the rows
        const int tasks = count * (rows - p.row_begin);       // an element in a row: a lane each
        const uint32_t per = 65536u / (uint32_t)count + 1u;   // t / count for t < 1024, count <= 32
#pragma unroll 1
        for (int t0 = 0; t0 < tasks; t0 += 32) {
            const int t = min(t0 + lane, tasks - 1), r = p.row_begin + (int)(((uint32_t)t * per) >> 16), l = t - (r - p.row_begin) * count;
            const float2 entry = list[l];
            const uint32_t info = __float_as_uint(entry.x), times = info >> 17;
            const int off = (int)(info & 0xffffu);
            const size_t place = ((size_t)b * p.R + r) * p.V + v0 + off;
            float f = ad_one(reinterpret_cast<const T*>(p.x) + place);
            const int m = __shfl_sync(0xffffffffu, mask, r);
            const uint32_t word = m >= 0 ? __ldg(p.masks + (size_t)m * mask_words + ((v0 + off) >> 5)) : ~0u;
            int hits = 0;                                     // drafted tokens before the row: they count like emitted ones
            for (uint32_t d = drafted; d; d &= d - 1) {
                const int j = __ffs(d) - 1;
                const int at_j = __shfl_sync(0xffffffffu, tok, j) - v0;
                const uint32_t rr = __shfl_sync(0xffffffffu, behind, j);
                hits += at_j == off && ((rr >> r) & 1u);
            }
            f = fmaf(f, (info >> 16) != 0u || hits ? (f > 0.f ? inv : rep) : 1.f, addend(entry.y, times));
            for (int z = 0; z < hits; ++z) f -= z || times ? freq : freq + pres;
            if (!((word >> ((v0 + off) & 31)) & 1u)) f = -INFINITY;
            if (t0 + lane < tasks) reinterpret_cast<T*>(p.y)[place] = static_cast<T>(f);
        }
        return;
    }

    // ---- many: worked on in the rows, the next one on its way while one is ----
    float add[8];
    uint32_t seen = 0u, counted = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t v = past(e);
        add[e] = addend(bias_of(VEC ? lane * 8 + e : 32 * e + lane), v >> 1);
        if (v) seen |= 1u << e;
        if (v >> 1) counted |= 1u << e;
    }
    struct Row { uint32_t w[Io::kWords], allowed, own; };
    auto load = [&](int r, Row& row) {
        row.own = 0u;
        row.allowed = there;
#pragma unroll
        for (int i = 0; i < Io::kWords; ++i) row.w[i] = 0u;
        const int m = __shfl_sync(0xffffffffu, mask, r & 31);
        if (r >= rows) return;
        if (m >= 0) {
            const uint32_t* words = p.masks + (size_t)m * mask_words + (v0 >> 5);
            if (VEC) {
                if (there) row.allowed = __ldg(reinterpret_cast<const unsigned char*>(words) + lane);
            } else {
                const uint32_t word = lane < 8 && v0 + 32 * lane < p.V ? __ldg(words + lane) : 0u;
                uint32_t a = 0u;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((__shfl_sync(0xffffffffu, word, e) >> lane) & 1u) a |= 1u << e;
                row.allowed = a & there;
            }
        }
        if (drafted) drafted_on(r, [&](int e) { row.own |= 1u << e; });
        // in place only what changes is needed (VEC: all eight, unless none changes or all are forbidden)
        uint32_t need = row.allowed;
        if (p.in_place && (!VEC || row.allowed == there)) need &= any | row.own;
        Io::load(x + (size_t)r * p.V, need, row.w);
    };
    Row next;
    load(p.row_begin, next);
#pragma unroll 1
    for (int r = p.row_begin; r < rows; ++r) {
        Row row = next;
        load(r + 1, next);
        float f[8];
        ad_unpack(row.w, f);
        const uint32_t penalised = seen | row.own;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float g = f[e] > 0.f ? inv : rep;
            f[e] = fmaf(f[e], (penalised >> e) & 1u ? g : 1.f, add[e]);
        }
        if (drafted) {                                    // they count like emitted ones
            uint32_t known = counted;
            drafted_on(r, [&](int hit) {
                const float less = (known >> hit) & 1u ? freq : freq + pres;
                known |= 1u << hit;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e == hit) f[e] -= less;
            });
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!((row.allowed >> e) & 1u)) f[e] = -INFINITY;
        ad_pack(f, row.w);
        Io::store(y + (size_t)r * p.V, p.in_place ? there & (any | row.own | ~row.allowed) : there, row.w);
    }
}

// ---- the token history --------------------------------------------------------------------------------------

constexpr int kHiThreads = 256;
constexpr int kHiPiece = 8192;                 // entries of a CTA of a history that begins anew: 16 KB of shared memory
constexpr int kHiMost = 16383;

struct HistoryParams {
    int16_t* history;
    const uint8_t* fresh;
    const int32_t *cu_prompt, *prompt, *out_tokens, *out_len;
    int32_t* status;
    int V, Tp, W;
};

// One more of token `tok`: emitted (2, no further than the largest count) or in the prompt (1).
__device__ __forceinline__ void history_add(int16_t* row, int tok, bool prompt) {
    unsigned short* at = reinterpret_cast<unsigned short*>(row) + tok;
    unsigned short old = *at;
    for (;;) {
        const unsigned short to = prompt ? old | 1u : (old >> 1) >= kHiMost ? old : (unsigned short)(old + 2u);
        if (to == old) return;
        const unsigned short was = atomicCAS(at, old, to);
        if (was == old) return;
        old = was;
    }
}
// Its tokens: false, and none, if the lengths make no sense.
__device__ __forceinline__ bool history_lengths(const HistoryParams& p, int b, int& c0, int& n, int& m) {
    c0 = n = m = 0;
    if (p.cu_prompt) {
        c0 = __ldg(p.cu_prompt + b);
        n = __ldg(p.cu_prompt + b + 1) - c0;
    }
    if (p.out_len) m = __ldg(p.out_len + b);
    const bool ok = c0 >= 0 && n >= 0 && c0 <= p.Tp - n && m >= 0 && m <= p.W;
    if (!ok) n = m = 0;
    return ok;
}

// A round, or pieces of prompts: a CTA (a warp where there are no prompts) for every sequence.
template <int THREADS>
__device__ __forceinline__ void history_scatter(const HistoryParams& p, int b, int t, int c0, int n, int m, bool ok) {
    int16_t* row = p.history + (size_t)b * p.V;
    bool bad = false;
    for (uint32_t i = t; i < (uint32_t)n; i += THREADS) {     // behind the last token 31 bits do not hold it
        const int tok = __ldg(p.prompt + c0 + i);
        if (tok < 0 || tok >= p.V) bad = true;
        else history_add(row, tok, true);
    }
    for (int i = t; i < m; i += THREADS) {
        const int tok = __ldg(p.out_tokens + (size_t)b * p.W + i);
        if (tok < 0 || tok >= p.V) bad = true;
        else history_add(row, tok, false);
    }
    if (p.status && bad) atomicOr(p.status + b, BS_DEV_BAD_TOKEN);
    if (p.status && !ok && t == 0) atomicOr(p.status + b, BS_DEV_BAD_LENGTH);
}
__global__ void __launch_bounds__(kHiThreads) history_round_kernel(const HistoryParams p, int B) {
    pdl_enter();
    const int b = blockIdx.x * (kHiThreads / 32) + (threadIdx.x >> 5);
    if (b >= B) return;
    int c0, n, m;
    const bool ok = history_lengths(p, b, c0, n, m);
    history_scatter<32>(p, b, threadIdx.x & 31, c0, n, m, ok);
}

// blockIdx.y: sequence, blockIdx.x: piece of its vocabulary
__global__ void __launch_bounds__(kHiThreads) history_prompts_kernel(const HistoryParams p) {
    __shared__ __align__(16) uint32_t s_words[kHiPiece / 2 + 4];
    const int b = blockIdx.y, tid = threadIdx.x;
    pdl_enter();
    int c0, n, m;
    const bool ok = history_lengths(p, b, c0, n, m);
    if (!p.fresh || !__ldg(p.fresh + b)) {
        if (blockIdx.x == 0) history_scatter<kHiThreads>(p, b, tid, c0, n, m, ok);
        return;
    }
    // entry v lies at place v - v0 + shift, so that 16-byte pieces are the same here and in the history
    const int v0 = blockIdx.x * kHiPiece, nv = min(kHiPiece, p.V - v0);
    int16_t* row = p.history + (size_t)b * p.V + v0;
    const int shift = (int)((reinterpret_cast<uintptr_t>(row) >> 1) & 7);
    for (int i = tid; i < kHiPiece / 2 + 4; i += kHiThreads) s_words[i] = 0u;
    __syncthreads();
    bool bad = false;
    for (uint32_t i = tid; i < (uint32_t)n; i += kHiThreads) {
        const int t = __ldg(p.prompt + c0 + i), at = t - v0 + shift;
        if (t < 0 || t >= p.V) bad = true;
        else if (t >= v0 && t < v0 + nv) atomicOr(s_words + (at >> 1), 1u << (16 * (at & 1)));
    }
    for (int i = tid; i < m; i += kHiThreads) {               // W <= 32: no count overflows
        const int t = __ldg(p.out_tokens + (size_t)b * p.W + i), at = t - v0 + shift;
        if (t < 0 || t >= p.V) bad = true;
        else if (t >= v0 && t < v0 + nv) atomicAdd(s_words + (at >> 1), 2u << (16 * (at & 1)));
    }
    if (p.status && blockIdx.x == 0) {
        if (bad) atomicOr(p.status + b, BS_DEV_BAD_TOKEN);
        if (!ok && tid == 0) atomicOr(p.status + b, BS_DEV_BAD_LENGTH);
    }
    __syncthreads();
    int16_t* base = row - shift;                              // on a 16-byte boundary
    const int16_t* s_entry = reinterpret_cast<const int16_t*>(s_words);
    for (int i = tid; i * 8 < nv + shift; i += kHiThreads) {
        const int lo = max(i * 8, shift), hi = min(i * 8 + 8, nv + shift);
        if (hi - lo == 8) {
            *reinterpret_cast<uint4*>(base + i * 8) = *reinterpret_cast<const uint4*>(s_words + i * 4);
        } else {
            for (int j = lo; j < hi; ++j) base[j] = s_entry[j];
        }
    }
}

template <typename T>
static cudaError_t launch_adjust(const AdjustParams& p, bool vec, cudaStream_t st) {
    // the low tokens of all sequences first: they are the frequent ones, of which there is more to change
    const dim3 grid(p.B, div_up(div_up(p.V, kAdWarp), kAdWarps));
    return vec ? launch_pdl(logits_adjust_kernel<T, true>, grid, kAdWarps * 32, 0, st, p)
               : launch_pdl(logits_adjust_kernel<T, false>, grid, kAdWarps * 32, 0, st, p);
}

}  // namespace bs

using namespace bs;

extern "C" bs_status bs_history_update(int16_t* history, int B, int V, const uint8_t* fresh, const int32_t* cu_prompt,
                                       const int32_t* prompt_tokens, int Tp, const int32_t* out_tokens, const int32_t* out_len, int W,
                                       int32_t* status, void* stream) {
    if (!history || B < 1 || V < 1 || Tp < 0 || W < 0 || (cu_prompt && Tp > 0 && !prompt_tokens) || (out_len && W > 0 && !out_tokens))
        return BS_ERR_INVALID_ARG;
    if (B > BS_MAX_BATCH || V > BS_MAX_VOCAB || W > BS_MAX_GAMMA + 1) return BS_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(history) & 1) return BS_ERR_INVALID_ARG;
    HistoryParams p = {history, fresh, cu_prompt, prompt_tokens, out_tokens, out_len, status, V, cu_prompt ? Tp : 0, W};
    const cudaStream_t st = (cudaStream_t)stream;
    if (!fresh && !cu_prompt) {
        if (!out_len) return BS_OK;
        return cuda_status(launch_pdl(history_round_kernel, div_up(B, kHiThreads / 32), kHiThreads, 0, st, p, B));
    }
    const dim3 grid(fresh ? div_up(V, kHiPiece) : 1, B);
    return cuda_status(launch_pdl(history_prompts_kernel, grid, kHiThreads, 0, st, p));
}

extern "C" bs_status bs_logits_adjust(const void* logits, void* out, bs_dtype dtype, const int32_t* gamma, int extra, int row_begin,
                                      int row_end, const int32_t* draft_tokens, const int32_t* node_parent, int Nmax,
                                      const int16_t* history, const float* repetition, const float* presence, const float* frequency,
                                      const int32_t* bias_begin, const int32_t* bias_tokens, const float* bias_values, int n_bias,
                                      const uint32_t* masks, int n_masks, const int32_t* mask_row, int B, int R, int V, int32_t* status,
                                      void* stream) {
    if (B < 1 || R < 1 || V < 1 || !logits || !out || Nmax < 0 || n_bias < 0 || n_masks < 0) return BS_ERR_INVALID_ARG;
    if (dtype != BS_F32 && dtype != BS_BF16) return BS_ERR_INVALID_ARG;
    if (extra < 0 || extra > 1 || row_begin < 0 || row_end < row_begin || row_end > R) return BS_ERR_INVALID_ARG;
    if (B > BS_MAX_BATCH || R > BS_MAX_GAMMA + 1 || V > BS_MAX_VOCAB || Nmax > BS_MAX_GAMMA) return BS_ERR_UNSUPPORTED;
    if (draft_tokens && Nmax < R - 1) return BS_ERR_INVALID_ARG;
    if (node_parent && !draft_tokens) return BS_ERR_INVALID_ARG;
    if ((repetition || presence || frequency) && !history && !draft_tokens) return BS_ERR_INVALID_ARG;
    if (bias_begin && n_bias > 0 && (!bias_tokens || !bias_values)) return BS_ERR_INVALID_ARG;
    if (mask_row && n_masks > 0 && !masks) return BS_ERR_INVALID_ARG;
    const long long es = dtype == BS_F32 ? 4 : 2;
    if ((reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out)) % es || (reinterpret_cast<uintptr_t>(history) & 1))
        return BS_ERR_INVALID_ARG;
    if (logits != out && rows_overlap(rows_of(logits, 0, V, 1, (long long)B * R, V, es), rows_of(out, 0, V, 1, (long long)B * R, V, es)))
        return BS_ERR_INVALID_ARG;
    AdjustParams p = {logits, out, gamma, draft_tokens, node_parent, history, repetition, presence, frequency, bias_begin,
                      bias_tokens, bias_values, masks, mask_row, status, extra, row_begin, row_end, B, R, Nmax, V, n_masks, n_bias,
                      logits == out};
    // Eight neighbours a lane where every row starts on 16 bytes and ends with a lane; else elements 32 apart.
    const uintptr_t at = reinterpret_cast<uintptr_t>(logits) | reinterpret_cast<uintptr_t>(out) | (history ? reinterpret_cast<uintptr_t>(history) : 0);
    const bool vec = V % kAdLane == 0 && at % 16 == 0;
    return cuda_status(dtype == BS_F32 ? launch_adjust<float>(p, vec, (cudaStream_t)stream)
                                       : launch_adjust<__nv_bfloat16>(p, vec, (cudaStream_t)stream));
}
