// bs_rotary, bs_rotary_frequencies: rotary positions of queries and keys.
//
//   (a, b) -> (a cos w - b sin w, b cos w + a sin w),   w = position * frequency of the pair
//
// A frequency is held in turns as a 64-bit binary fraction, off by two steps of it at most, so the angle modulo one turn is the low
// half of an integer product and off by 2^-31 turns at the farthest position, where the product in fp32 is off by 0.01 radians at
// position 100000.  Its fp32 value, at most half a turn, is rounded by 2^-26 turns at most.
//
// Bound by HBM: every element is read and written once.  A warp takes a token, or a part of its heads where there are few tokens: it
// computes the token's sines and cosines (a lane those of every 32nd pair) into shared memory and sweeps over heads x chunks of
// pairs, so that they are computed once for many heads.  Warps do not wait for one another; the first chunks are on their way
// while a warp looks for the position (trees: a search for the sequence, a walk to the root).
#include "bs_common.cuh"
#include "bs_overlap.cuh"

namespace bs {

constexpr int kRoWarps = 4;
constexpr int kRoMaxRot = 256;
constexpr int kRoBatch = 1;                    // chunks of a lane in flight
constexpr int kRoTarget = 24;                  // warps for each SM: below that, a token's heads are divided

// Division by a number that the host knows.
struct RoDiv {
    uint32_t m;
    int shift;
    __device__ __forceinline__ int div(int n) const { return (int)(((uint64_t)(uint32_t)n * m) >> shift); }
};

struct RotaryParams {
    const void *q, *k;
    void *q_out, *k_out;
    long long q_st, q_sh, k_st, k_sh, qo_st, qo_sh, ko_st, ko_sh;
    const int32_t* positions;
    const uint64_t* freq;                      // [rot / 2] turns x 2^64
    const int32_t* cu_new;
    const int32_t* node_parent;                // NULL: chains
    float amplitude;
    int rot, T, Hq, H, d, B, Nmax;             // H: heads of q and k
    int chunks;                                // of a head, those that are only copied among them
    int parts, part_items;                     // of a token; chunks of a part
    RoDiv by_chunk;
};

template <typename T, int P> struct alignas(sizeof(T) * P) RoVec { T v[P]; };

// Elements pass through once: around L1, where every line would take a place (24000 tokens of 40 heads: 89 us through it, 82 around it).
template <typename V> __device__ __forceinline__ V ro_ld(const V* p) {
    if constexpr (sizeof(V) == 16) {
        const uint4 v = __ldcg(reinterpret_cast<const uint4*>(p));
        return *reinterpret_cast<const V*>(&v);
    } else if constexpr (sizeof(V) == 8) {
        const uint2 v = __ldcg(reinterpret_cast<const uint2*>(p));
        return *reinterpret_cast<const V*>(&v);
    } else {
        return *p;
    }
}
template <typename V> __device__ __forceinline__ void ro_st(V* p, const V& v) {
    if constexpr (sizeof(V) == 16) __stcg(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(&v));
    else if constexpr (sizeof(V) == 8) __stcg(reinterpret_cast<uint2*>(p), *reinterpret_cast<const uint2*>(&v));
    else *p = v;
}
__device__ __forceinline__ float ro_float(float x) { return x; }
__device__ __forceinline__ float ro_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void ro_set(float& y, float x) { y = x; }
__device__ __forceinline__ void ro_set(__nv_bfloat16& y, float x) { y = __float2bfloat16_rn(x); }

// Position of token t (a converged warp asks); < 0: the row is left alone.  A tree's node n stands depth(n) behind its root.
__device__ __forceinline__ int ro_position(const RotaryParams& p, int t) {
    const int lane = threadIdx.x & 31;
    const int pos = __ldg(p.positions + t);
    if (!p.node_parent || pos < 0) return pos;
    // the sequence: the last b with cu_new[b] <= t, 32 candidates at a time
    int lo = 0, n = p.B;
    while (n > 1) {
        const int step = (n + 31) / 32;
        const int at = lane * step;
        const unsigned le = __ballot_sync(0xffffffffu, at < n && __ldg(p.cu_new + lo + at) <= t);
        if (!le) return -1;
        const int last = 31 - __clz(le);
        lo += last * step;
        n = min(step, n - last * step);
    }
    const int c0 = __ldg(p.cu_new + lo), c1 = __ldg(p.cu_new + lo + 1), row = t - c0;
    if (row < 0 || t >= c1 || row > p.Nmax) return -1;
    int parent = 0;
    if (lane < p.Nmax) {
        parent = __ldg(p.node_parent + (size_t)lo * p.Nmax + lane);
        if (parent < 0 || parent > lane) parent = 0;           // not an earlier node: hangs under the root
    }
    int depth = 0;
    for (int node = row; node > 0; ++depth) node = __shfl_sync(0xffffffffu, parent, node - 1);
    return pos - row + depth;
}

// P pairs are loaded as two vectors of P elements: the halves' (HALF), or 2P neighbours' (two by two).
template <typename T, int P, bool HALF>
__global__ void __launch_bounds__(kRoWarps * 32) rotary_kernel(const RotaryParams p) {
    using Vec = RoVec<T, P>;
    __shared__ float s_cos[kRoWarps][kRoMaxRot / 2], s_sin[kRoWarps][kRoMaxRot / 2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long task = (long long)blockIdx.x * kRoWarps + warp;
    if (task >= (long long)p.T * p.parts) return;
    const int t = p.parts == 1 ? (int)task : (int)(task / p.parts), part = (int)(task - (long long)t * p.parts);
    const int half = p.rot / 2, n_rot = half / P;
    const int end = min(p.H * p.chunks, (part + 1) * p.part_items);
    pdl_enter();
    struct Item { int c, at_a, at_b; const T* x; T* y; };
    auto item = [&](int i) {
        Item r;
        const int head = p.by_chunk.div(i);
        r.c = i - head * p.chunks;
        if (head < p.Hq) {
            r.x = (const T*)p.q + t * p.q_st + (long long)head * p.q_sh;
            r.y = (T*)p.q_out + t * p.qo_st + (long long)head * p.qo_sh;
        } else {
            r.x = (const T*)p.k + t * p.k_st + (long long)(head - p.Hq) * p.k_sh;
            r.y = (T*)p.k_out + t * p.ko_st + (long long)(head - p.Hq) * p.ko_sh;
        }
        const bool halves = HALF && r.c < n_rot;              // behind the rotated part: rot = 2 P n_rot
        r.at_a = halves ? r.c * P : r.c * 2 * P;
        r.at_b = halves ? half + r.c * P : r.at_a + P;
        return r;
    };
    Vec a[kRoBatch], b[kRoBatch];
    auto load = [&](int base) {
#pragma unroll
        for (int u = 0; u < kRoBatch; ++u)
            if (base + 32 * u < end) {
                const Item r = item(base + 32 * u);
                a[u] = ro_ld(reinterpret_cast<const Vec*>(r.x + r.at_a));
                b[u] = ro_ld(reinterpret_cast<const Vec*>(r.x + r.at_b));
            }
    };
    int base = part * p.part_items + lane;
    load(base);
    const int pos = ro_position(p, t);
    if (pos < 0) return;
    float *cos_of = s_cos[warp], *sin_of = s_sin[warp];
    for (int j = lane; j < half; j += 32) {
        const int64_t turns = (int64_t)((uint64_t)(uint32_t)pos * __ldg(p.freq + j));   // of a turn, in [-1/2, 1/2) x 2^64
        float s, c;
        sincospif((float)turns * 1.0842021724855044e-19f, &s, &c);                      // 2^-63: half turns; rounded to 2^-24 of the angle
        const int at = (j % P) * n_rot + j / P;               // the chunks of a warp's lanes lie side by side
        cos_of[at] = c * p.amplitude;
        sin_of[at] = s * p.amplitude;
    }
    __syncwarp();
#pragma unroll 1
    for (;;) {
#pragma unroll
        for (int u = 0; u < kRoBatch; ++u)
            if (base + 32 * u < end) {
                const Item r = item(base + 32 * u);
                if (r.c < n_rot) {
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        T& ra = HALF ? a[u].v[e] : (2 * e < P ? a[u].v[(2 * e) % P] : b[u].v[(2 * e) % P]);
                        T& rb = HALF ? b[u].v[e] : (2 * e + 1 < P ? a[u].v[(2 * e + 1) % P] : b[u].v[(2 * e + 1) % P]);
                        const float fa = ro_float(ra), fb = ro_float(rb), co = cos_of[e * n_rot + r.c], si = sin_of[e * n_rot + r.c];
                        ro_set(ra, fmaf(fa, co, -fb * si));   // the one rounding to T
                        ro_set(rb, fmaf(fb, co, fa * si));
                    }
                }
                ro_st(reinterpret_cast<Vec*>(r.y + r.at_a), a[u]);
                ro_st(reinterpret_cast<Vec*>(r.y + r.at_b), b[u]);
            }
        base += 32 * kRoBatch;
        if (base - lane >= end) break;
        load(base);
    }
}

static RoDiv ro_div(uint32_t d) {
    RoDiv r;
    int log = 0;
    while ((1u << log) < d) ++log;
    r.shift = 31 + log;                                       // m = ceil(2^shift / d) < 2^32, error n (m d - 2^shift) < 2^shift for n < 2^31
    r.m = (uint32_t)(((1ull << r.shift) + d - 1) / d);
    return r;
}

template <typename T, int P>
static cudaError_t launch_rotary(RotaryParams p, bool copies, bool half, cudaStream_t st) {
    p.chunks = (copies ? p.d : p.rot) / (2 * P);
    p.by_chunk = ro_div((uint32_t)p.chunks);
    // Few tokens: their heads are divided among warps, down to one chunk a lane.
    const int per_token = p.H * p.chunks, most = div_up(per_token, 32);
    const long long want = ((long long)kRoTarget * sm_count() + p.T - 1) / p.T;
    p.parts = want < most ? (int)want : most;
    p.part_items = div_up(most, p.parts) * 32;
    p.parts = div_up(per_token, p.part_items);
    const long long grid = ((long long)p.T * p.parts + kRoWarps - 1) / kRoWarps;
    if (grid > 0x7fffffffLL) return cudaErrorInvalidConfiguration;
    return half ? launch_pdl(rotary_kernel<T, P, true>, (unsigned)grid, kRoWarps * 32, 0, st, p)
                : launch_pdl(rotary_kernel<T, P, false>, (unsigned)grid, kRoWarps * 32, 0, st, p);
}

}  // namespace bs

using namespace bs;

extern "C" bs_status bs_rotary_frequencies(bs_rotary_scaling scaling, int rot, double base, double factor, double low, double high,
                                           double original, uint64_t* freq_host, float* amplitude_host) {
    if (!freq_host || !amplitude_host) return BS_ERR_INVALID_ARG;
    if (rot < 2 || rot > kRoMaxRot || (rot & 1)) return BS_ERR_UNSUPPORTED;
    if (scaling < BS_ROTARY_PLAIN || scaling > BS_ROTARY_YARN || !(base > 1.0) || !isfinite(base)) return BS_ERR_INVALID_ARG;
    if (scaling != BS_ROTARY_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) return BS_ERR_INVALID_ARG;
    if (scaling >= BS_ROTARY_BANDS && (!(original >= 1.0) || !(low > 0.0) || !(high > low) || !isfinite(high) || !isfinite(original)))
        return BS_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    double first = 0, last = 0;
    if (scaling == BS_ROTARY_YARN) {
        // the pairs that turn `high` and `low` times within the original length
        first = fmax(floor(rot * log(original / (high * two_pi)) / (2 * log(base))), 0.0);
        last = fmin(ceil(rot * log(original / (low * two_pi)) / (2 * log(base))), rot - 1.0);
    }
    // 64 bits of mantissa: a frequency's error is multiplied by the position, 2^31 at most.
    typedef long double wide;
    const wide turn = 8 * atanl((wide)1);
    for (int i = 0; i < rot / 2; ++i) {
        wide f = powl((wide)base, (wide)(-2 * i) / rot);
        if (scaling == BS_ROTARY_LINEAR) f /= factor;
        if (scaling == BS_ROTARY_BANDS) {
            const wide keep = fminl(fmaxl((original * f / turn - low) / ((wide)high - low), (wide)0), (wide)1);
            f *= keep + (1 - keep) / factor;
        }
        if (scaling == BS_ROTARY_YARN) {
            const wide ramp = fminl(fmaxl((i - first) / fmaxl(last - first, (wide)1 / 1000), (wide)0), (wide)1);
            f *= 1 - ramp + ramp / factor;
        }
        freq_host[i] = (uint64_t)(ldexpl(f / turn, 64) + (wide)1 / 2);           // f <= 1
    }
    *amplitude_host = scaling == BS_ROTARY_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.0f;
    return BS_OK;
}

extern "C" bs_status bs_rotary(const void* q, long long q_stride_t, long long q_stride_h, const void* k, long long k_stride_t,
                               long long k_stride_h, bs_dtype dtype, const int32_t* positions, const uint64_t* freq,
                               float amplitude, int rot, int interleaved, const int32_t* cu_new, const int32_t* node_parent, int B,
                               int Nmax, int T, int Hq, int Hkv, int d, void* q_out, long long qo_stride_t, long long qo_stride_h,
                               void* k_out, long long ko_stride_t, long long ko_stride_h, void* stream) {
    if (T < 0 || Hq < 0 || Hkv < 0 || Hq + Hkv < 1 || d < 2 || !freq || (T > 0 && !positions)) return BS_ERR_INVALID_ARG;
    if (dtype != BS_F32 && dtype != BS_BF16) return BS_ERR_INVALID_ARG;
    if (T > 0 && ((Hq && (!q || !q_out)) || (Hkv && (!k || !k_out)))) return BS_ERR_INVALID_ARG;
    if (node_parent && (!cu_new || B < 1 || Nmax < 0)) return BS_ERR_INVALID_ARG;
    if (node_parent && (Nmax > BS_MAX_GAMMA || B > BS_MAX_BATCH)) return BS_ERR_UNSUPPORTED;
    if (rot < 2 || rot > d || (rot & 1) || (d & 1) || rot > kRoMaxRot || Hq > 4096 || Hkv > 4096 || d > 4096) return BS_ERR_UNSUPPORTED;
    if (!isfinite(amplitude)) return BS_ERR_INVALID_ARG;
    if (T == 0) return BS_OK;
    const int es = dtype == BS_F32 ? 4 : 2;
    if (((Hq ? reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(q_out) : 0) |
         (Hkv ? reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(k_out) : 0)) % es)
        return BS_ERR_INVALID_ARG;
    // in place, or apart
    const Rows from[2] = {rows_of(q, q_stride_t, q_stride_h, T, Hq, d, es), rows_of(k, k_stride_t, k_stride_h, T, Hkv, d, es)};
    const Rows to[2] = {rows_of(q_out, qo_stride_t, qo_stride_h, T, Hq, d, es), rows_of(k_out, ko_stride_t, ko_stride_h, T, Hkv, d, es)};
    for (int i = 0; i < 2; ++i)
        if ((!same_rows(from[i], to[i]) && rows_overlap(from[i], to[i])) || rows_overlap(from[i], to[1 - i])) return BS_ERR_INVALID_ARG;
    if (rows_overlap(to[0], to[1])) return BS_ERR_INVALID_ARG;
    RotaryParams p = {};
    p.q = q; p.k = k; p.q_out = q_out; p.k_out = k_out;
    p.q_st = q_stride_t; p.q_sh = q_stride_h; p.k_st = k_stride_t; p.k_sh = k_stride_h;
    p.qo_st = qo_stride_t; p.qo_sh = qo_stride_h; p.ko_st = ko_stride_t; p.ko_sh = ko_stride_h;
    p.positions = positions; p.freq = freq; p.cu_new = cu_new; p.node_parent = node_parent;
    p.amplitude = amplitude;
    p.rot = rot; p.T = T; p.Hq = Hq; p.H = Hq + Hkv; p.d = d; p.B = B; p.Nmax = Nmax;
    const bool copies = rot < d && ((Hq && !same_rows(from[0], to[0])) || (Hkv && !same_rows(from[1], to[1])));
    // the widest vector that divides both parts of a head and that every row starts on
    auto fits = [&](int P) {
        auto ok = [&](const void* x, long long st, long long sh) {
            return reinterpret_cast<uintptr_t>(x) % (uintptr_t)(P * es) == 0 && st % P == 0 && sh % P == 0;
        };
        return (rot / 2) % P == 0 && (d - rot) % (2 * P) == 0 &&
               (!Hq || (ok(q, q_stride_t, q_stride_h) && ok(q_out, qo_stride_t, qo_stride_h))) &&
               (!Hkv || (ok(k, k_stride_t, k_stride_h) && ok(k_out, ko_stride_t, ko_stride_h)));
    };
    const cudaStream_t st = (cudaStream_t)stream;
    const bool half = !interleaved;
    if (dtype == BS_F32)
        return cuda_status(fits(4) ? launch_rotary<float, 4>(p, copies, half, st) : fits(2) ? launch_rotary<float, 2>(p, copies, half, st)
                                                                                    : launch_rotary<float, 1>(p, copies, half, st));
    return cuda_status(fits(8)   ? launch_rotary<__nv_bfloat16, 8>(p, copies, half, st)
                       : fits(4) ? launch_rotary<__nv_bfloat16, 4>(p, copies, half, st)
                       : fits(2) ? launch_rotary<__nv_bfloat16, 2>(p, copies, half, st)
                                 : launch_rotary<__nv_bfloat16, 1>(p, copies, half, st));
}
