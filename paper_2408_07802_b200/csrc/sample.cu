// One token of every row of logits, drawn with a given random number.
//
// With x in descending order (equal ones by ascending index) and w_i = e^((x_i - x_0) / T), the tokens kept are a prefix of that
// order: the first top_k, of these the ones with w_i >= min_p, of these the ones before which less than top_p of what is left
// lies.  M being the sum of the kept weights, the token is the first one up to which (it included) more than u M lies.
//
// Three passes over a row, of which the first comes from HBM and the others from L2 (or L1): 4 or 2 bytes a logit.
//   1  the maximum
//   2  how many logits lie in each of 4096 ranges of (x_0 - x) / T.  From these counts alone follow the range where the first
//      top_k end, and, by the mean weight of a range, small windows of ranges that hold the ends of the mass that is looked for
//   3  the logits in the windows are put aside, the weights of the others between them summed in 64 bits
// What was put aside is sorted, its weights are summed in order, and every border is then known as if the row had been sorted.
// A sum of weights in 32 bits is off by 10^-7, and of 50 thousand alike each has 2 10^-5 of the mass: the token would be another
// one in a row of every hundred.  So sums and weights next to a border are 64 bits.
// Where a border does not lie in its window (the mean weights were too far off), or more logits lie in the windows than there is
// room for (many equal ones), descend() finds the borders digit by digit of the logits' order, with sums of integers.
//
// Few rows: up to 8 CTAs of a cluster share a row.
#include <float.h>
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace kr {

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_CLUSTER = 8;
constexpr int RANGES = 4096, PER = RANGES / THREADS;
constexpr int FINE = 3072;             // ranges of 1 / 256, then of 1 / 32: up to 44, where a weight is 10^-19
constexpr int ROOM = 4096, ROOM_PER = ROOM / THREADS;

struct SampleParams {
    const void *logits;
    long long row_stride;
    const float *uniforms, *temperature, *top_p, *min_p;
    const int *top_k;
    float temperature_all, top_p_all, min_p_all;
    int top_k_all;
    int *ids;
    float *logprob;
    int rows, vocab;
};

// The order of logits as unsigned numbers; -0 and +0 are equal
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o); }

// Range of a logit: the same roundings for every logit, so a larger logit is never in a later range
struct Ranges {
    float top, per_nat;   // x_0; 256 / T
    __device__ __forceinline__ int of(float x) const {
        const float t = (top - x) * per_nat;
        return static_cast<int>(fminf(fminf(t, fmaf(t, 0.125f, FINE * 0.875f)), RANGES - 1.f));
    }
    static __device__ __forceinline__ float begin(int r) { return (r <= FINE ? r : FINE + (r - FINE) * 8) / 256.f; }
};

struct Smem {
    uint32_t count[RANGES];          // of this CTA's part of the row
    union {
        struct {
            uint32_t before[RANGES + 1];   // logits of the row in earlier ranges
            float mass[RANGES + 1];        // what they weigh, about
            float spread[RANGES + 1];      // and how far that may be off
        };
        struct {
            u64 mass256[256];
            uint32_t count256[256];
        };
    };
    u64 aside[ROOM];                 // order << 32 | ~index
    uint8_t kind[RANGES];            // of a range: 0 .. 2 summed (before the windows of the token, of top_p, of the limits), ASIDE, LATER
    float top[MAX_CLUSTER];
    double all[MAX_CLUSTER], gaps[MAX_CLUSTER][3];
    double warp_d[WARPS];
    float warp_f[WARPS];
    uint32_t warp_u[WARPS];
    u64 warp_l[WARPS];
    uint32_t n_aside;
    int odd[MAX_CLUSTER], first[MAX_CLUSTER];
    int k_range;
    u64 found, found_above;
};
enum Kind { ASIDE = 3, LATER = 4 };

template <bool H16>
struct Row {
    static constexpr int VEC = H16 ? 8 : 4, BATCH = 4;
    const uint8_t *p;
    int n, head, vecs;   // head: logits before the first 16-byte boundary
    __device__ __forceinline__ Row(const void *base, long long at, int vocab) {
        p = static_cast<const uint8_t *>(base) + at * (H16 ? 2 : 4);
        n = vocab;
        head = min(n, static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(p) & 15)) & 15) / (H16 ? 2 : 4)));
        vecs = (n - head) / VEC;
    }
    __device__ __forceinline__ float at(int i) const {
        return H16 ? from_h16(reinterpret_cast<const uint16_t *>(p)[i]) : reinterpret_cast<const float *>(p)[i];
    }
    // f(index, logit) for every logit of part `part` of `parts`, in any order
    template <typename F>
    __device__ __forceinline__ void visit(int part, int parts, F f) const {
        const int per = (vecs + parts - 1) / parts, lo = min(vecs, part * per), hi = min(vecs, lo + per);
        const uint4 *v = reinterpret_cast<const uint4 *>(p + head * (H16 ? 2 : 4));
        for (int i0 = lo + threadIdx.x; i0 < hi; i0 += THREADS * BATCH) {
            uint4 raw[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
                if (i0 + b * THREADS < hi) raw[b] = v[i0 + b * THREADS];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (i0 + b * THREADS >= hi) break;
                const int e = head + (i0 + b * THREADS) * VEC;
                const uint32_t w[4] = {raw[b].x, raw[b].y, raw[b].z, raw[b].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (H16) {
                        f(e + 2 * j, h16_lo(w[j]));
                        f(e + 2 * j + 1, h16_hi(w[j]));
                    } else {
                        f(e + j, __uint_as_float(w[j]));
                    }
                }
            }
        }
        if (part == 0) {
            const int rest = n - vecs * VEC;   // before the first vector and behind the last
            if (threadIdx.x < rest) {
                const int i = threadIdx.x < head ? threadIdx.x : vecs * VEC + threadIdx.x;
                f(i, at(i));
            }
        }
    }
};

__device__ __forceinline__ double weight_of(float top, float x, double inv_t) { return exp((static_cast<double>(x) - static_cast<double>(top)) * inv_t); }

// Sum over the CTA in a fixed order, for every thread
__device__ __forceinline__ double block_sum(Smem &sm, double v) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm.warp_d[threadIdx.x >> 5] = v;
    __syncthreads();
    double s = 0.;
    for (int w = 0; w < WARPS; ++w) s += sm.warp_d[w];
    return s;
}

// Sums of what the threads before hold
template <typename T>
__device__ __forceinline__ T block_before(T (&warp)[WARPS], T v, T &total) {
    const int lane = threadIdx.x & 31;
    T upto = v;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const T x = __shfl_up_sync(0xFFFFFFFFu, upto, o);
        if (lane >= o) upto += x;
    }
    __syncthreads();
    if (lane == 31) warp[threadIdx.x >> 5] = upto;
    __syncthreads();
    T before = 0;
    total = 0;
    for (int w = 0; w < WARPS; ++w) {
        if (w < threadIdx.x >> 5) before += warp[w];
        total += warp[w];
    }
    return before + (upto - v);
}

// What a row asks for
struct Ask {
    float top;       // its largest logit
    double inv_t;
    int k;           // 0: no limit
    double p, m, u;  // p >= 1, m <= 0: no limit
};

__device__ __forceinline__ void give(const SampleParams &s, int r, int id, float logprob) {
    if (threadIdx.x == 0) {
        s.ids[r] = id;
        if (s.logprob) s.logprob[r] = logprob;
    }
}

// ---------------------------------------------------------------- any row, digit by digit

// The first token, in the order, up to which the weights (counts: 1 each) make `want` or more: the order of its logit, and what the
// larger logits make.  `want` is first made from the sum of all.  Tokens of the order `k_key` count k_ties times, whatever their
// number, and those below it not at all.  All threads of the CTA; weights are integers, so the order of the additions is of no
// importance.
template <bool H16, bool COUNTS, typename W, typename F>
__device__ __forceinline__ uint32_t descend(Smem &sm, const Row<H16> &row, uint32_t k_key, u64 k_ties, W weight, F want_of, u64 &want, u64 &above,
                                            u64 &total) {
    uint32_t key = 0;
    above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        if (threadIdx.x < 256) sm.mass256[threadIdx.x] = 0;
        __syncthreads();
        auto add = [&](uint32_t o, u64 w) { atomicAdd(&sm.mass256[(o >> shift) & 255], w); };
        row.visit(0, 1, [&](int, float x) {
            const uint32_t o = order_of(x);
            if (o > k_key && (shift == 24 || (o ^ key) >> (shift + 8) == 0)) {
                const uint32_t active = __activemask();
                int same;
                __match_all_sync(active, o, &same);   // many equal ones: one addition for all
                if (!same) add(o, COUNTS ? 1 : weight(x));
                else if (__ffs(active) - 1 == (threadIdx.x & 31)) add(o, (COUNTS ? 1 : weight(x)) * __popc(active));
            }
        });
        __syncthreads();
        if (threadIdx.x == 0) {
            if (k_ties && (shift == 24 || (k_key ^ key) >> (shift + 8) == 0)) add(k_key, (COUNTS ? 1 : weight(value_of(k_key))) * k_ties);
            if (shift == 24) {
                u64 all = 0;
                for (int i = 0; i < 256; ++i) all += sm.mass256[i];
                sm.found_above = all;
            }
        }
        __syncthreads();
        if (shift == 24) {
            total = sm.found_above;
            want = want_of(total);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            u64 a = above;
            int digit = 255, last = 0;
            for (; digit >= 0; --digit) {
                if (sm.mass256[digit]) last = digit;
                if (a + sm.mass256[digit] >= want) break;
                a += sm.mass256[digit];
            }
            if (digit < 0) {   // (there is not so much)
                digit = last;
                a -= sm.mass256[last];
            }
            sm.found = digit;
            sm.found_above = a;
        }
        __syncthreads();
        key |= static_cast<uint32_t>(sm.found) << shift;
        above = sm.found_above;
    }
    __syncthreads();
    return key;
}

template <bool H16>
__device__ __noinline__ void sample_any(const SampleParams &s, Smem &sm, int r, const Ask a) {
    const Row<H16> row(s.logits, r * s.row_stride, s.vocab);
    const int bits = 62 - (32 - __clz(s.vocab));   // the sum of all weights stays below 2^62
    const double one = static_cast<double>(1ull << bits);
    uint32_t k_key = 0;
    u64 k_ties = 0, want, above, total;
    if (a.k > 0 && a.k < s.vocab) {
        k_key = descend<H16, true>(sm, row, 0u, 0, [](float) { return 1ull; }, [&](u64) { return static_cast<u64>(a.k); }, want, above, total);
        k_ties = a.k - above;
    }
    auto weight = [&](float x) -> u64 {
        const double w = weight_of(a.top, x, a.inv_t);
        return w >= a.m ? static_cast<u64>(__double2ll_rn(w * one)) : 0ull;
    };
    auto upto = [&](u64 want, u64 above, uint32_t key) {   // with the token that reaches `want`
        const u64 w = max(1ull, weight(value_of(key))), ties = want > above ? (want - above + w - 1) / w : 1;
        return above + ties * w;
    };
    uint32_t key = descend<H16, false>(sm, row, k_key, k_ties, weight, [&](u64 all) {
        const double p = ceil(a.p * static_cast<double>(all));
        return a.p >= 1. ? all : (p >= 1. ? static_cast<u64>(p) : 1ull);
    }, want, above, total);
    const u64 mass = a.p >= 1. ? total : min(total, upto(want, above, key));
    key = descend<H16, false>(sm, row, k_key, k_ties, weight, [&](u64) {
        return min(mass, static_cast<u64>(a.u * static_cast<double>(mass)) + 1);
    }, want, above, total);
    const u64 w = max(1ull, weight(value_of(key)));
    uint32_t ties = want > above ? static_cast<uint32_t>((want - above + w - 1) / w) : 1u;   // the so-many-th of its equals
    const int per = (s.vocab + THREADS - 1) / THREADS, lo = min(s.vocab, (int)threadIdx.x * per), hi = min(s.vocab, lo + per);
    uint32_t mine = 0, all;
    for (int i = lo; i < hi; ++i) mine += order_of(row.at(i)) == key;
    const uint32_t before = block_before(sm.warp_u, mine, all);
    ties = min(ties, all);
    if (before < ties && ties <= before + mine) {
        uint32_t seen = before;
        for (int i = lo; i < hi; ++i) {
            seen += order_of(row.at(i)) == key;
            if (seen == ties) {
                sm.found = i;
                break;
            }
        }
    }
    __syncthreads();
    const double y = (static_cast<double>(a.top) - static_cast<double>(value_of(key))) * a.inv_t;
    give(s, r, static_cast<int>(sm.found), static_cast<float>(-y - log(static_cast<double>(mass) / one)));
}

// ---------------------------------------------------------------- the three passes

// First range up to which, it included, `mass` holds `want` or more (MORE: more than `want`).  A whole warp.
template <bool MORE>
__device__ __forceinline__ int range_of_mass(const Smem &sm, float want) {
    const int lane = threadIdx.x & 31;
    int at = 0;
#pragma unroll
    for (int step = RANGES / 32; step > 0; step /= 32) {   // 128, 4
        const float m = sm.mass[at + (lane + 1) * step];
        const uint32_t reached = __ballot_sync(0xFFFFFFFFu, MORE ? m > want : m >= want);
        if (!reached) return RANGES - 1;
        at += (__ffs(reached) - 1) * step;
    }
    const float m = sm.mass[at + (lane & 3) + 1];
    const uint32_t reached = __ballot_sync(0xFFFFFFFFu, (MORE ? m > want : m >= want) && lane < 4);
    return reached ? at + __ffs(reached) - 1 : RANGES - 1;
}

__device__ __forceinline__ uint32_t n_cluster_ctas() {
    uint32_t n;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
}

template <typename T>
__device__ __forceinline__ T *in_cta(T *p, uint32_t rank) {   // the same place in another CTA of the cluster
    T *q;
    asm volatile("mapa.u64 %0, %1, %2;" : "=l"(q) : "l"(p), "r"(rank));
    return q;
}

template <bool H16>
__global__ void __launch_bounds__(THREADS, 2) sample_kernel(const SampleParams s) {
    extern __shared__ uint8_t smem_raw[];
    Smem &sm = *reinterpret_cast<Smem *>(smem_raw);
    const int parts = n_cluster_ctas(), part = cluster_ctarank();
    const int r = blockIdx.x / parts, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    for (int i = tid; i < RANGES; i += THREADS) sm.count[i] = 0;
    if (tid == 0) sm.n_aside = 0;
    pdl_wait();
    const Row<H16> row(s.logits, r * s.row_stride, s.vocab);
    const float t = s.temperature ? s.temperature[r] : s.temperature_all, u = s.uniforms[r];
    Ask a;
    a.k = s.top_k ? s.top_k[r] : s.top_k_all;
    a.k = a.k <= 0 || a.k >= s.vocab ? 0 : a.k;
    const float p = s.top_p ? s.top_p[r] : s.top_p_all, m = s.min_p ? s.min_p[r] : s.min_p_all;
    a.p = fmaxf(p, 0.f);
    a.m = fminf(m, 1.f);
    a.u = u;
    a.inv_t = 1. / static_cast<double>(t);

    // 1: the maximum
    {
        float top = -INFINITY;
        bool odd = !(t >= 0.f && t < INFINITY && u >= 0.f && u < 1.f) || p != p || m != m;
        row.visit(part, parts, [&](int, float x) {
            top = fmaxf(top, x);
            odd |= !(x < INFINITY);
        });
        const uint32_t any = __ballot_sync(0xFFFFFFFFu, odd);
#pragma unroll
        for (int o = 16; o > 0; o /= 2) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (lane == 0) {
            sm.warp_f[warp] = top;
            sm.warp_u[warp] = any;
        }
        __syncthreads();
        if (tid < parts) {   // to every CTA of the cluster
            float all = -INFINITY;
            uint32_t bad = 0;
            for (int w = 0; w < WARPS; ++w) {
                all = fmaxf(all, sm.warp_f[w]);
                bad |= sm.warp_u[w];
            }
            *in_cta(&sm.top[part], tid) = all;
            *in_cta(&sm.odd[part], tid) = bad != 0;
        }
        cluster_sync_all();
        a.top = -INFINITY;
        odd = false;
        for (int i = 0; i < parts; ++i) {
            a.top = fmaxf(a.top, sm.top[i]);
            odd |= sm.odd[i] != 0;
        }
        if (odd || a.top == -INFINITY) {   // no distribution
            if (part == 0) give(s, r, -1, NAN);
            return;
        }
    }
    if (t == 0.f || a.k == 1) {   // the likeliest token, of several the first
        int first = INT_MAX;
        row.visit(part, parts, [&](int i, float x) {
            if (x == a.top) first = min(first, i);
        });
        first = __reduce_min_sync(0xFFFFFFFFu, first);
        __syncthreads();
        if (lane == 0) sm.warp_u[warp] = first;
        __syncthreads();
        if (tid == 0) {
            for (int w = 0; w < WARPS; ++w) first = min(first, static_cast<int>(sm.warp_u[w]));
            *in_cta(&sm.first[part], 0u) = first;
        }
        cluster_sync_all();
        if (part == 0) {
            for (int i = 0; i < parts; ++i) first = min(first, sm.first[i]);
            give(s, r, first, 0.f);
        }
        return;
    }

    // 2: how many logits in each range
    Ranges ranges;
    ranges.top = a.top;
    ranges.per_nat = fminf(256.f / t, 1e30f);
    const float per_bit = fminf(1.4426950408889634f / t, 1e30f);
    float sum = 0.f;
    row.visit(part, parts, [&](int, float x) {
        atomicAdd(&sm.count[ranges.of(x)], 1u);
        sum += ex2_approx((x - a.top) * per_bit);
    });
    {
        const double all = block_sum(sm, sum);
        if (tid < parts) *in_cta(&sm.all[part], tid) = all;
    }
    cluster_sync_all();
    // A logit of a range weighs as much as one in its middle, give or take width / sqrt(12).  By how much the sum of all weights differs
    // from the ranges' is known, and the ranges before a place have a part of that in proportion to their variance; what is then
    // left of the variance is that of a bridge, small behind the few largest logits, which have most of it.
    float mass_all = 0.f;
    {
        for (int c = 0; c < parts; ++c) mass_all += static_cast<float>(sm.all[c]);
        uint32_t n[PER], mine = 0, all;
        float mass = 0.f, total, var = 0.f, var_all;
        const int r0 = tid * PER;
#pragma unroll
        for (int i = 0; i < PER; ++i) n[i] = 0;
        for (int c = 0; c < parts; ++c) {
            const uint4 *from = reinterpret_cast<const uint4 *>(in_cta(&sm.count[r0], c));
#pragma unroll
            for (int i = 0; i < PER / 4; ++i) {
                const uint4 x = from[i];
                n[4 * i] += x.x;
                n[4 * i + 1] += x.y;
                n[4 * i + 2] += x.z;
                n[4 * i + 3] += x.w;
            }
        }
        auto weigh = [&](int i, float &w, float &v) {
            const float y0 = Ranges::begin(r0 + i), width = Ranges::begin(r0 + i + 1) - y0, mid = __expf(-y0 - width / 2);
            w = n[i] * mid;
            v = w * mid * width * width * (1.f / 12.f);
        };
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            float w, v;
            weigh(i, w, v);
            mine += n[i];
            mass += w;
            var += v;
        }
        uint32_t at = block_before(sm.warp_u, mine, all);
        float up = block_before(sm.warp_f, mass, total), v_up = block_before(sm.warp_f, var, var_all);
        if (tid == 0) {
            sm.k_range = RANGES;
            sm.before[0] = 0;
            sm.mass[0] = sm.spread[0] = 0.f;
        }
        __syncthreads();
        const float share = var_all > 0.f ? (mass_all - total) / var_all : 0.f, inv_var = var_all > 0.f ? 1.f / var_all : 0.f;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            float w, v;
            weigh(i, w, v);
            if (a.k > 0 && at < a.k && at + n[i] >= a.k) sm.k_range = r0 + i;
            at += n[i];
            up += w;
            v_up += v;
            sm.before[r0 + i + 1] = at;
            sm.mass[r0 + i + 1] = up + share * v_up;
            // five standard deviations, and the roundings of the sums
            sm.spread[r0 + i + 1] = 5.f * sqrtf(fmaxf(0.f, v_up * (var_all - v_up) * inv_var)) + 4e-6f * mass_all;
        }
        __syncthreads();
    }
    // windows: of the limits (top_k, min_p), of the end of top_p, of the token
    int e0 = sm.k_range, e1 = e0, p0, p1, s0, s1;
    if (a.m > 0.) {
        const float y = -logf(static_cast<float>(a.m));
        Ranges at = ranges;
        at.top = 0.f;
        at.per_nat = 256.f;
        const int m0 = at.of(-fmaxf(0.f, y - 1e-4f * (1.f + y))), m1 = at.of(-(y + 1e-4f * (1.f + y)));
        if (e0 > m1) {
            e0 = m0;
            e1 = m1;
        } else if (e0 >= m0) {
            e0 = m0;
            e1 = m1;
        }
    }
    // (a border may be as far off as at the end of the range that it seems to be in, or at its beginning)
    auto off = [&](int range) { return fmaxf(sm.spread[min(range, RANGES)], sm.spread[min(range + 1, RANGES)]); };
    const float z_lo = sm.mass[min(e0, RANGES)] - (e0 < RANGES ? off(e0) : 0.f);
    const float z_hi = sm.mass[min(e1 + 1, RANGES)] + (e1 < RANGES ? off(e1) : 0.f);
    float mass_lo = z_lo, mass_hi = z_hi;
    if (a.p < 1.) {
        const float pf = static_cast<float>(a.p), lo = pf * z_lo, hi = pf * z_hi;
        mass_lo = lo - off(range_of_mass<false>(sm, lo));
        mass_hi = hi + off(range_of_mass<false>(sm, hi));
        p0 = min(range_of_mass<false>(sm, mass_lo), e1);
        p1 = min(range_of_mass<false>(sm, mass_hi), e1);
        mass_hi = fminf(mass_hi + __expf(-Ranges::begin(p0)), sm.mass[min(p1 + 1, RANGES)] + off(p1));
    } else {
        p0 = e0;
        p1 = e1;
    }
    s0 = min(range_of_mass<true>(sm, u * mass_lo - off(range_of_mass<true>(sm, u * mass_lo))), p1);
    s1 = min(range_of_mass<true>(sm, u * mass_hi + off(range_of_mass<true>(sm, u * mass_hi))), p1);
    // counts of what is summed and of what is put aside
    const uint32_t n_s = sm.before[min(s1 + 1, RANGES)], n_gap0 = sm.before[min(s0, RANGES)];
    const uint32_t n_gap1 = p0 > s1 ? sm.before[min(p0, RANGES)] - n_s : 0;
    const int after_p = min(max(p1, s1) + 1, RANGES);
    const uint32_t n_gap2 = e0 >= after_p ? sm.before[min(e0, RANGES)] - sm.before[after_p] : 0;
    const uint32_t n_aside = sm.before[min(e1 + 1, RANGES)] - n_gap0 - n_gap1 - n_gap2;
    if (n_aside > ROOM) {   // (the same for every CTA)
        cluster_sync_all();   // (all have read the others' counts)
        if (part == 0) sample_any<H16>(s, sm, r, a);
        return;
    }
    for (int i = tid; i < RANGES; i += THREADS) {
        const bool aside = (i >= s0 && i <= s1) || (i >= p0 && i <= p1) || (i >= e0 && i <= e1);
        sm.kind[i] = aside ? ASIDE : (i > e1 ? LATER : (i > s1) + (i > p1));
    }
    __syncthreads();

    // 3: sums and windows
    {
        double sum0 = 0., sum1 = 0., sum2 = 0.;
        u64 *list = in_cta(&sm.aside[0], 0u);
        uint32_t *n = in_cta(&sm.n_aside, 0u);
        row.visit(part, parts, [&](int i, float x) {
            const int kind = sm.kind[ranges.of(x)];
            if (kind == ASIDE) {
                list[atomicAdd(n, 1u)] = static_cast<u64>(order_of(x)) << 32 | static_cast<uint32_t>(~i);
            } else if (kind != LATER) {
                const double w = weight_of(a.top, x, a.inv_t);
                sum0 += kind == 0 ? w : 0.;
                sum1 += kind == 1 ? w : 0.;
                sum2 += kind == 2 ? w : 0.;
            }
        });
        sum0 = block_sum(sm, sum0);
        sum1 = block_sum(sm, sum1);
        sum2 = block_sum(sm, sum2);
        if (tid == 0) {
            double *to = in_cta(&sm.gaps[part][0], 0u);
            to[0] = sum0;
            to[1] = sum1;
            to[2] = sum2;
        }
        cluster_sync_all();
        if (part != 0) return;
    }
    double gap0 = 0., gap1 = 0., gap2 = 0.;
    for (int c = 0; c < parts; ++c) {
        gap0 += sm.gaps[c][0];
        gap1 += sm.gaps[c][1];
        gap2 += sm.gaps[c][2];
    }
    // in descending order
    int size = 32;
    while (size < (int)n_aside) size *= 2;
    for (int i = n_aside + tid; i < size; i += THREADS) sm.aside[i] = 0;
    for (int k = 2; k <= size; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            __syncthreads();
            for (int i = tid; i < size / 2; i += THREADS) {
                const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
                const u64 x = sm.aside[lo], y = sm.aside[hi];
                if ((x < y) == ((lo & k) == 0)) {
                    sm.aside[lo] = y;
                    sm.aside[hi] = x;
                }
            }
        }
    __syncthreads();
    // thread i has the places ROOM_PER i .. of the order
    const int at = tid * ROOM_PER;
    double w[ROOM_PER], mine = 0., all;
    int range[ROOM_PER];
#pragma unroll
    for (int i = 0; i < ROOM_PER; ++i) {
        w[i] = 0.;
        range[i] = RANGES;
        if (at + i < (int)n_aside) {
            const float x = value_of(static_cast<uint32_t>(sm.aside[at + i] >> 32));
            w[i] = weight_of(a.top, x, a.inv_t);
            range[i] = ranges.of(x);
        }
        mine += w[i];
    }
    const double before = block_before(sm.warp_d, mine, all);
    auto gaps_before = [&](int range) { return gap0 + (range > s1 ? gap1 : 0.) + (range > p1 ? gap2 : 0.); };
    double z = 0., up = before, in_s = 0., in_p = 0.;   // allowed by the limits; weights in the window of the token, up to the end of that of top_p
    bool allowed[ROOM_PER];
#pragma unroll
    for (int i = 0; i < ROOM_PER; ++i) {
        const uint32_t rank = at + i + n_gap0 + (range[i] > s1 ? n_gap1 : 0) + (range[i] > p1 ? n_gap2 : 0);
        allowed[i] = at + i < (int)n_aside && (a.k == 0 || rank < a.k) && (w[i] >= a.m || rank == 0);
        z += allowed[i] ? w[i] : 0.;
        in_s += range[i] <= s1 ? w[i] : 0.;
        in_p += range[i] <= p1 ? w[i] : 0.;
    }
    z = block_sum(sm, z) + gap0 + gap1 + gap2;
    in_s = block_sum(sm, in_s);
    bool fits = true;
    double mass = z;
    if (a.p < 1.) {
        in_p = block_sum(sm, in_p);
        double before_p = 0.;   // weights put aside in front of the window of top_p
        mass = 0.;
        const double want = a.p * z;
#pragma unroll
        for (int i = 0; i < ROOM_PER; ++i) {
            const uint32_t rank = at + i + n_gap0 + (range[i] > s1 ? n_gap1 : 0) + (range[i] > p1 ? n_gap2 : 0);
            allowed[i] = allowed[i] && (up + gaps_before(range[i]) < want || rank == 0);
            up += w[i];
            mass += allowed[i] ? w[i] : 0.;
            before_p += range[i] < p0 ? w[i] : 0.;
        }
        mass = block_sum(sm, mass) + gap0 + gap1;
        before_p = block_sum(sm, before_p) + gap0 + gap1;
        fits = (before_p <= want || (p0 == 0 && s0 == 0)) && want <= gap0 + gap1 + in_p;
    }
    const double want = a.u * mass;
    fits = fits && gap0 <= want && want < gap0 + in_s;
    if (!fits) {
        __syncthreads();
        sample_any<H16>(s, sm, r, a);
        return;
    }
    if (tid == 0) sm.found = ~0ull;
    __syncthreads();
    up = before;
    int token = ROOM;
#pragma unroll
    for (int i = 0; i < ROOM_PER; ++i) {
        up += w[i];
        if (token == ROOM && allowed[i] && range[i] <= s1 && gap0 + up > want) token = at + i;
    }
    token = __reduce_min_sync(0xFFFFFFFFu, token);
    if (lane == 0 && token < ROOM) atomicMin(&sm.found, static_cast<u64>(token));
    __syncthreads();
    // (the sum up to the last one, rounded otherwise than `mass`, may fall short of it)
    if (sm.found == ~0ull) {
        token = -1;
#pragma unroll
        for (int i = 0; i < ROOM_PER; ++i)
            if (allowed[i] && range[i] <= s1) token = at + i;
        token = __reduce_max_sync(0xFFFFFFFFu, token);
        if (lane == 0) sm.warp_u[warp] = token + 1;
        __syncthreads();
        token = 0;
        for (int i = 0; i < WARPS; ++i) token = max(token, static_cast<int>(sm.warp_u[i]));
        if (token == 0) {
            sample_any<H16>(s, sm, r, a);
            return;
        }
        --token;
    } else {
        token = static_cast<int>(sm.found);
    }
    if (tid == 0) {
        const u64 e = sm.aside[token];
        const double y = (static_cast<double>(a.top) - static_cast<double>(value_of(static_cast<uint32_t>(e >> 32)))) * a.inv_t;
        s.ids[r] = static_cast<int>(~static_cast<uint32_t>(e));
        if (s.logprob) s.logprob[r] = static_cast<float>(-y - log(mass));
    }
}

template <bool H16>
int launch(const SampleParams &p, cudaStream_t st) {
    static DeviceOnce configured;
    if (!configured.done()) {
        int rc = cuda_check(cudaFuncSetAttribute(sample_kernel<H16>, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(Smem)),
                            "sample tokens: shared memory opt-in");
        if (rc) return rc;
        configured.set();
    }
    const int sms = sm_count();
    if (sms <= 0) return KRAKEN_ECUDA;
    // CTAs that share a row: as many as leave all of them running at once, with at least four vectors a thread
    int cluster = 1;
    while (cluster < MAX_CLUSTER && (long long)p.rows * 2 * cluster <= 2LL * sms && p.vocab / (2 * cluster) >= THREADS * (H16 ? 8 : 4) * 2) cluster *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(p.rows * cluster);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = sizeof(Smem);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cuda_check(cudaLaunchKernelEx(&cfg, sample_kernel<H16>, p), "sample tokens: launch");
}

}  // namespace

}  // namespace kr

extern "C" int kraken_op_sample_tokens(const kraken_sample_args *a, void *stream) {
    using namespace kr;
    if (!a) return KRAKEN_EINVAL;
    if (a->rows == 0) return KRAKEN_OK;
    const size_t size = a->dtype ? 2 : 4;
    if (a->rows < 0 || a->vocab < 1 || !a->logits || !a->uniforms || !a->ids || (a->dtype != 0 && a->dtype != 1) || a->row_stride < 0 ||
        (reinterpret_cast<uintptr_t>(a->logits) % size) != 0)
        return KRAKEN_EINVAL;
    if ((!a->temperature && !(a->temperature_all >= 0.f && isfinite(a->temperature_all))) || (!a->top_p && isnan(a->top_p_all)) ||
        (!a->min_p && isnan(a->min_p_all)))
        return KRAKEN_EINVAL;
    if (a->vocab > KRAKEN_SAMPLE_MAX_VOCAB || a->rows >= 1 << 27) return KRAKEN_EUNSUPPORTED;
    SampleParams p;
    p.logits = a->logits;
    p.row_stride = a->row_stride;
    p.uniforms = a->uniforms;
    p.temperature = a->temperature;
    p.top_p = a->top_p;
    p.min_p = a->min_p;
    p.top_k = a->top_k;
    p.temperature_all = a->temperature_all;
    p.top_p_all = a->top_p_all;
    p.min_p_all = a->min_p_all;
    p.top_k_all = a->top_k_all;
    p.ids = a->ids;
    p.logprob = a->logprob;
    p.rows = a->rows;
    p.vocab = a->vocab;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return a->dtype ? launch<true>(p, st) : launch<false>(p, st);
}
