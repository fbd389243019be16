// The items of bs_prompt_attention, how a CTA takes them and how long its warps wait.  Nothing here is of the GPU but the operations of a warp: a test that
// stands in for these runs it on the host, with numbers in orders that a GPU does not give on demand.
#pragma once

#include "banditspec.h"

namespace bs {

constexpr int kPaKeys = 128;                   // keys of a tile

struct PaItem {
    int row0, n, i0, h;                        // sequence: first row, length; first token of the item, key head
    int nt0, nt1;                              // tiles of keys that each row tile sees; both 0: no more items
};

// Items in the order of their numbers: 32 sequences at a time, and of these the items with the most keys first, whichever sequence
// they are of, so that none of the long ones begins last (sequence after sequence: 4 prompts of 1000 to 4095, 157 us
// against 122 when both were measured); the key heads of the same rows together.
struct PaWalk {
    int b0;                                    // 32 sequences, one a lane
    long long before, items;                   // items of the sequences before them; their own
    int end;                                   // where the sequences up to the last of them end, at most
    int row0, n, pairs;                        // this lane's
};
template <class P>
__device__ __forceinline__ void pa_walk_load(const P& p, PaWalk& w) {
    const int lane = threadIdx.x & 31, b = w.b0 + lane;
    int c0 = 0, c1 = 0;
    if (b < p.B) { c0 = __ldg(p.cu + b); c1 = __ldg(p.cu + b + 1); }
    bool ok = c0 >= 0 && c1 >= c0 && c1 <= p.T;
    int end = max(w.end, ok ? c1 : 0);                        // of the sequences up to this lane's: a row is one sequence's only
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) end = max(end, __shfl_up_sync(0xffffffffu, end, o));
    const int earlier = __shfl_up_sync(0xffffffffu, end, 1);
    ok = ok && c0 >= (lane ? earlier : w.end);
    if (!ok && b < p.B && p.status) atomicOr(p.status + b, BS_DEV_BAD_LENGTH);
    w.row0 = c0;
    w.n = ok ? c1 - c0 : 0;
    w.pairs = (w.n + 2 * p.TQ - 1) / (2 * p.TQ);
    w.end = __shfl_sync(0xffffffffu, end, 31);
    w.items = (long long)__reduce_add_sync(0xffffffffu, (unsigned)w.pairs) * p.Hkv;
}
template <class P>
__device__ __forceinline__ bool pa_walk_to(const P& p, PaWalk& w, long long item, PaItem& it) {
    if (item < w.before) {
        w.b0 = 0; w.before = 0; w.end = 0;
        pa_walk_load(p, w);
    }
    while (item >= w.before + w.items) {
        if (w.b0 + 32 >= p.B) return false;
        w.before += w.items;
        w.b0 += 32;
        pa_walk_load(p, w);
    }
    // pairs from the `level`-th on come first: the largest level at which there are enough of them
    const long long t = item - w.before;
    auto from = [&](int level) { return (long long)__reduce_add_sync(0xffffffffu, (unsigned)max(0, w.pairs - level)) * p.Hkv; };
    int lo = 0, hi = (int)__reduce_max_sync(0xffffffffu, (unsigned)w.pairs);   // from(lo) > t >= from(hi)
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (from(mid) > t) lo = mid;
        else hi = mid;
    }
    const int rank = (int)(t - from(hi));                     // among the items of this level
    uint32_t who = __ballot_sync(0xffffffffu, w.pairs > lo);
    for (int skip = rank / p.Hkv; skip > 0; --skip) who &= who - 1;
    const int l = __ffs(who) - 1;
    it.h = rank % p.Hkv;
    it.i0 = lo * 2 * p.TQ;
    it.row0 = __shfl_sync(0xffffffffu, w.row0, l);
    it.n = __shfl_sync(0xffffffffu, w.n, l);
    it.nt0 = (min(it.n, it.i0 + p.TQ) + kPaKeys - 1) / kPaKeys;
    it.nt1 = it.i0 + p.TQ < it.n ? (min(it.n, it.i0 + 2 * p.TQ) + kPaKeys - 1) / kPaKeys : 0;
    return true;
}

// Cycles after which a wait gives up, in a call of T tokens: about a second, and 20000 for every tile of keys of the longest item there can
// be, six times what a tile takes (3150 for a pair of row tiles, heads of 128).
inline long long pa_wait_limit(int T) { return 2000000000LL + 20000LL * ((T + kPaKeys - 1) / kPaKeys); }

// The next item of a CTA.  `item` is the number of a CTA that has just begun or will not run (`looked`: it was looked at), `next` asks the
// launch control for another and clears `more` if there is none, `ok` if it gave up.  The grid has a few more CTAs than there are
// items, and nothing promises that their numbers come in order: a number behind the last item says nothing of the others.
template <class P, class Next>
__device__ __forceinline__ bool pa_take(const P& p, PaWalk& w, const long long& item, const bool& more, const bool& ok, bool& looked, PaItem& it, Next&& next) {
    while (ok && more) {
        if (!looked) {
            looked = true;
            if (pa_walk_to(p, w, item, it)) return true;
        }
        next();
        looked = false;
    }
    return false;
}

}  // namespace bs
