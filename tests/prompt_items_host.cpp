// Runs bs_prompt_items.cuh on the host: the warps that take items of bs_prompt_attention, with the operations of a warp stood in for and CTA
// numbers handed out in any order.  A lane is a fiber; all lanes of a warp stop at each operation of the warp.
//
// stdin:  T Hkv TQ B cu[0..B] running n number[0..n-1]   -- the first `running` numbers begin as CTAs, the others are asked for
// With an argument: the limit of a wait in a call of so many tokens.
// stdout: "item cta row0 n i0 h nt0 nt1" in the order of taking, "status b bits"
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <algorithm>
#include <memory>
#include <vector>

#define __device__
#define __forceinline__ inline
using std::max;
using std::min;

struct Warp {
    ucontext_t main, lane[32];
    std::vector<char> stack[32];
    int at[32] = {};                           // operations of a lane so far
    uint64_t brought[2][32];
    bool done[32] = {}, asks = false, more = true;
    long long item = 0;
    int cta = 0;
};
static Warp* g_warp;
static int g_lane;
struct { int x; } threadIdx;

static void stop() {
    Warp* w = g_warp;
    const int l = g_lane;
    swapcontext(&w->lane[l], &w->main);
    threadIdx.x = l;
}
// What every lane brings to an operation: a lane is never more than one operation ahead of another.
static const uint64_t* bring(uint64_t v) {
    Warp* w = g_warp;
    const int l = g_lane, half = w->at[l]++ & 1;
    w->brought[half][l] = v;
    stop();
    return w->brought[half];
}
template <class T> T __ldg(const T* p) { return *p; }
template <class T> T __shfl_sync(unsigned, T v, int from) { return (T)bring((uint64_t)v)[from & 31]; }
template <class T> T __shfl_up_sync(unsigned, T v, int by) {
    const int l = g_lane;
    const uint64_t* a = bring((uint64_t)v);
    return (T)a[l >= by ? l - by : l];
}
static unsigned __reduce_add_sync(unsigned, unsigned v) {
    const uint64_t* a = bring(v);
    unsigned s = 0;
    for (int l = 0; l < 32; ++l) s += (unsigned)a[l];
    return s;
}
static unsigned __reduce_max_sync(unsigned, unsigned v) {
    const uint64_t* a = bring(v);
    return (unsigned)*std::max_element(a, a + 32);
}
static int __reduce_max_sync(unsigned, int v) {
    const uint64_t* a = bring((uint64_t)(int64_t)v);
    int s = (int)(int64_t)a[0];
    for (int l = 1; l < 32; ++l) s = max(s, (int)(int64_t)a[l]);
    return s;
}
static unsigned __ballot_sync(unsigned, bool v) {
    const uint64_t* a = bring(v);
    unsigned s = 0;
    for (int l = 0; l < 32; ++l) s |= (unsigned)a[l] << l;
    return s;
}
static int __ffs(unsigned v) { return __builtin_ffs((int)v); }
static int atomicOr(int* p, int v) { const int old = *p; *p |= v; return old; }

#include "bs_prompt_items.cuh"

struct Params { const int32_t* cu; int32_t* status; int B, T, Hkv, TQ; };
static Params g_p;

static void lane_main() {
    Warp* w = g_warp;
    const int l = g_lane;
    threadIdx.x = l;
    bs::PaWalk walk = {};
    bs::pa_walk_load(g_p, walk);
    long long item = w->item;
    bool more = true, ok = true, looked = false;
    auto next = [&]() {
        w->asks = true;
        stop();
        more = w->more;
        item = w->item;
    };
    for (;;) {
        bs::PaItem it = {};
        if (!bs::pa_take(g_p, walk, item, more, ok, looked, it, next)) break;
        if (l == 0) printf("item %d %d %d %d %d %d %d\n", w->cta, it.row0, it.n, it.i0, it.h, it.nt0, it.nt1);
    }
    w->done[l] = true;
    swapcontext(&w->lane[l], &w->main);
}

int main(int argc, char** argv) {
    if (argc > 1) {
        printf("%lld\n", bs::pa_wait_limit(atoi(argv[1])));
        return 0;
    }
    int running = 0, n = 0;
    if (scanf("%d %d %d %d", &g_p.T, &g_p.Hkv, &g_p.TQ, &g_p.B) != 4) return 2;
    std::vector<int32_t> cu(g_p.B + 1), status(g_p.B);
    for (auto& c : cu) if (scanf("%d", &c) != 1) return 2;
    if (scanf("%d %d", &running, &n) != 2) return 2;
    std::vector<long long> number(n);
    for (auto& x : number) if (scanf("%lld", &x) != 1) return 2;
    g_p.cu = cu.data();
    g_p.status = status.data();
    std::vector<std::unique_ptr<Warp>> warps;
    for (int c = 0; c < running && c < n; ++c) {
        warps.emplace_back(new Warp);
        Warp* w = warps.back().get();
        w->cta = c;
        w->item = number[c];
        for (int l = 0; l < 32; ++l) {
            w->stack[l].resize(32768);
            getcontext(&w->lane[l]);
            w->lane[l].uc_stack.ss_sp = w->stack[l].data();
            w->lane[l].uc_stack.ss_size = w->stack[l].size();
            w->lane[l].uc_link = nullptr;
            makecontext(&w->lane[l], lane_main, 0);
        }
    }
    int given = running;
    srand(1);
    while (!warps.empty()) {                                  // one CTA's piece after the other, in any order
        const size_t c = (size_t)rand() % warps.size();
        Warp* w = warps[c].get();
        if (w->asks) {
            w->asks = false;
            w->more = given < n;
            w->item = w->more ? number[given++] : 0;
        }
        while (!w->asks && !w->done[31]) {
            for (int l = 0; l < 32; ++l) {
                g_warp = w;
                g_lane = l;
                swapcontext(&w->main, &w->lane[l]);
            }
        }
        if (w->done[31]) warps.erase(warps.begin() + c);
    }
    for (int b = 0; b < g_p.B; ++b) printf("status %d %d\n", b, status[b]);
    return 0;
}
