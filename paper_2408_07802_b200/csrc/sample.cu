// One token of every row of logits, drawn with a given random number.
//
// With x in descending order (equal ones by ascending index) and w_i = e^((x_i - x_0) / T), the tokens kept are a prefix of that
// order: the first top_k, of these the ones with w_i >= min_p, of these the ones before which less than top_p of what is left
// lies.  M being the sum of the kept weights, the token is the first one up to which (it included) more than u M lies.
//
// Three passes over a row, of which the first comes from HBM and the others from L2 (or L1): 4 or 2 bytes a logit.
//   1  the maximum
//   2  how many logits lie in each of 8192 ranges of (x_0 - x) / T, and the sum of all weights in 32 bits.  From these counts follow
//      the range where the first top_k end, and, by the mean weight of a range, small windows of ranges that hold the ends of the
//      mass that is looked for
//   3  the logits in the windows are put aside, the weights of the others between them summed in 64 bits
// What was put aside (some hundred logits) is sorted, its weights are summed in order, and every border is then known as if the
// row had been sorted.  A sum of weights in 32 bits is off by 10^-7, and of 50 thousand alike each has 2 10^-5 of the mass: the
// token would be another one in a row of every hundred.  So sums and weights next to a border are 64 bits.
// Where a border does not lie in its window (the mean weights were too far off), more logits lie in the windows than there is
// room for (many equal ones), or the temperature is beyond 10^-29 .. 10^29, sample_any() finds the borders digit by digit of the logits'
// order, with sums of integers: 0.3 to 0.6 ms for a row of 50257 fp32 logits (1.1 with every weight added by itself in 64 bits), 1.0 to
// 1.7 for 16-bit ones of 105 to 132 thousand.
//
// Few rows: up to 8 CTAs of a cluster share a row.
//
// What bounds it, on a B200 (a graph of calls).  512 rows of 50257 fp32 logits: 109 us where reading them takes 16 (103 MB come from
// HBM, once); issue slots are busy 55 % of the time, a row's CTA being at its barriers (maximum, counts, windows, ranks) for the
// rest of it, and two CTAs an SM is what registers and the table of counts leave.  64 mixed rows: 28.6 us; one row: 17 us; these are
// the steps one after the other.  Weights in 64 bits throughout took 156 us for the 512 rows: in pass 2 they are 32 bits, in pass 3 logits
// are compared with the windows' borders in steps of the exponent and weights are the table's times a 32-bit rest.
#include <float.h>
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace kr {

namespace {

typedef unsigned long long u64;

constexpr int THREADS = 512, WARPS = THREADS / 32;
constexpr int MAX_CLUSTER = 8;
constexpr int RANGES = 8192, PER = RANGES / THREADS;
// ranges of 1 / 512 in the exponent of 2 (2 steps) up to an exponent of 12, then of 1 / 16: up to 140, where a weight is 10^-42
constexpr int FINE = 6144, FINEST = 2;
constexpr int ROOM = 4096;
// What sums of weights in 32 bits may be off by, of the sum of all (found: below 2 10^-7).  The window of a uniform within twice this of
// 1 reaches to the row's end, which may be more than there is room for: with 4 10^-6 one in 75 calls of 512 rows of 50257 was 0.5 ms late
// for a single row; now one in 600.
constexpr float ROUNDINGS = 5e-7f;
constexpr double LOG2E = 1.4426950408889634074;
constexpr int STEPS = 1024;            // of the table of powers of two

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

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
    float c;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(c) : "f"(a), "f"(b));
    return c;
}

// The order of logits as unsigned numbers; -0 and +0 are equal
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) { return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o); }

// How far a logit lies below the largest, as an exponent of two (t = (x_0 - x) log2(e) / T in 32 bits, at most 2000) and in whole
// steps of 1 / 1024; its range.  The same roundings for every logit, so a larger logit is never in a later range.
struct Below {
    float d, t, shifted;
    int k;
    __device__ __forceinline__ Below(float x, float top, float per) {
        d = top - x;
        t = fminf(d * per, 2000.f);
        shifted = fmaf(t, 1024.f, 12582912.f);   // 1.5 2^23: the nearest integer in the low bits
        k = __float_as_int(shifted) & 0x3FFFFF;
    }
    __device__ __forceinline__ int range() const {
        const int r = k / FINEST;
        return min(min(r, (r >> 5) + (FINE - FINE / 32)), RANGES - 1);
    }
};

// Ranges: FINEST steps each up to FINE, then 32 times as many
struct Ranges {
    static __device__ __forceinline__ int first(int r) {   // step; none behind the last range
        return r >= RANGES ? INT_MAX : (r <= FINE ? r : FINE + (r - FINE) * 32) * FINEST;
    }
    static __device__ __forceinline__ float begin(int r) { return (first(r) - 0.5f) * (1.f / 1024.f); }
    // what a logit in the middle of a range weighs, and the variance of the weight of one anywhere in it
    static __device__ __forceinline__ void weigh(int r, float &w, float &v) {
        const float steps = FINEST * (r < FINE ? 1.f : 32.f), width = steps * (0.693147181f / 1024.f);
        w = ex2_approx(-(begin(r) + 0.5f / 1024.f * steps));
        v = w * w * (width * width * (1.f / 12.f));
    }
};

struct Smem {
    union {
        uint32_t count[RANGES];      // of this CTA's part of the row
        double weight[ROOM];         // of what is put aside
        u64 mass256[256];
    };
    u64 aside[ROOM];                 // order << 32 | ~index
    // of the whole row, before the ranges of thread i: logits, what they weigh, the variance of that
    uint32_t before[THREADS + 1];
    float mass[THREADS + 1], var[THREADS + 1];
    double power[STEPS];             // 2^(-i / 1024)
    float top[MAX_CLUSTER];
    double all[MAX_CLUSTER], gaps[MAX_CLUSTER][3];
    double warp_d[WARPS][3];
    float warp_f[WARPS], warp_v[WARPS];
    uint32_t warp_u[WARPS];
    uint32_t n_aside;
    int first[MAX_CLUSTER];
    struct {
        int s0, s1, p0, p1, e0, e1;
        uint32_t n_gap0, n_gap1, n_gap2, n_aside;
    } windows;
    int token;
    u64 found, found_above;
    alignas(16) uint32_t row_count[];   // [RANGES] of the whole row, where CTAs share it
};

template <bool H16>
struct Row {
    static constexpr int VEC = H16 ? 8 : 4;
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
    // f(index, logit) for every logit of part `part` of `parts`, in any order.  BATCH: vectors that a thread requests at a time; ROLLED:
    // for a long f, whose copies would have to be fetched: the 32-bit words of a vector one after the other.
    template <int BATCH, bool ROLLED, typename F>
    __device__ __forceinline__ void visit(int part, int parts, F f) const {
        const int per = (vecs + parts - 1) / parts, lo = min(vecs, part * per), hi = min(vecs, lo + per);
        const uint4 *v = reinterpret_cast<const uint4 *>(p + head * (H16 ? 2 : 4));
        auto word = [&](int e, uint32_t w) {
            if (H16) {
                f(e, h16_lo(w));
                f(e + 1, h16_hi(w));
            } else {
                f(e, __uint_as_float(w));
            }
        };
        constexpr int STEP = H16 ? 2 : 1;
        uint4 next[BATCH];   // requested while the ones before are worked on
        auto request = [&](int i0) {
#pragma unroll
            for (int b = 0; b < BATCH; ++b)
                if (i0 + b * THREADS < hi) next[b] = v[i0 + b * THREADS];
        };
        request(lo + threadIdx.x);
#pragma unroll 1
        for (int i0 = lo + threadIdx.x; i0 < hi; i0 += THREADS * BATCH) {
            uint4 raw[BATCH];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) raw[b] = next[b];
            request(i0 + THREADS * BATCH);
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (i0 + b * THREADS >= hi) break;
                const int e = head + (i0 + b * THREADS) * VEC;
                if (ROLLED) {
#pragma unroll 1
                    for (int j = 0; j < 4; ++j) word(e + j * STEP, j == 0 ? raw[b].x : (j == 1 ? raw[b].y : (j == 2 ? raw[b].z : raw[b].w)));
                } else {
                    word(e, raw[b].x);
                    word(e + STEP, raw[b].y);
                    word(e + 2 * STEP, raw[b].z);
                    word(e + 3 * STEP, raw[b].w);
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

// e^((x - top) / T) by a table of 2^(-i / 1024) and a short polynomial for what is left of the exponent (Tang's table method).
struct Weights {
    const double *power;
    double top, per_nat;         // x_0; log2(e) / T
    float per_hi, per_lo;        // the same in two pieces
    // of one logit, in 64 bits, to some 10^-15 of it
    __device__ __forceinline__ double of(float x) const {
        const double t = (top - static_cast<double>(x)) * per_nat;
        if (!(t < 1000.)) return 0.;
        const double shifted = fma(t, 1024., 6755399441055744.);   // 1.5 2^52: the nearest integer in the low bits
        const int k = __double2loint(shifted);
        const double r = fma(shifted - 6755399441055744., 1. / 1024., -t);
        double q = fma(r, 9.6181291076284772e-3, 5.5504108664821580e-2);   // (ln 2)^i / i!, i = 4 .. 1
        q = fma(r, q, 2.4022650695910071e-1);
        q = fma(r, q, 6.9314718055994531e-1);
        const double b = power[k & (STEPS - 1)], w = fma(b * r, q, b);
        return __hiloint2double(__double2hiint(w) - (k >> 10) * (1 << 20), __double2loint(w));
    }
    // The same with 32-bit instructions for most of it: b (1 + g), b the power of two from the table and g, 3 10^-4 at most, what the
    // rest of the exponent adds, rounded once; off by up to 1.5 10^-11 of it, and to be summed in 64 bits: a border, with a part q of
    // the mass before it, is off by at most q (1 - q) twice that.  (g b formed and summed in 32 bits: 512 rows of 50257 in 106 us in place
    // of 109, but weights off by 10^-10, and half a million equal ones a CTA by 4 10^-9.)
    __device__ __forceinline__ double fast(float x, const Below &y) const {
        // top - x = d + d_lo (Knuth's exact difference)
        const float topf = static_cast<float>(top), xx = y.d - topf, d_lo = (topf - (y.d - xx)) - (x + xx);
        const float t_lo = fmaf(y.d, per_hi, -y.t) + fmaf(y.d, per_lo, d_lo * per_hi);   // t + t_lo: the exponent
        const float r = fmaf(y.shifted - 12582912.f, 1.f / 1024.f, -y.t), e = r - t_lo;   // (r is exact)
        // 2^e - 1; ln 2 in two pieces
        const float g = fmaf(r, 0.69314718f, fmaf(e * e, fmaf(e, 5.5504109e-2f, 2.4022651e-1f), fmaf(r, -1.9046543e-9f, -6.9314718e-1f * t_lo)));
        const double p = power[y.k & (STEPS - 1)], b = __hiloint2double(__double2hiint(p) - (y.k >> 10) * (1 << 20), __double2loint(p));
        return fma(b, static_cast<double>(g), b);
    }
};

// Sums over the CTA (alone: over the warp) in a fixed order, for every thread
template <int N>
__device__ __forceinline__ void block_sums(Smem &sm, double (&v)[N], bool alone = false) {
#pragma unroll
    for (int o = 16; o > 0; o /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
    if (alone) return;
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) sm.warp_d[threadIdx.x >> 5][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (threadIdx.x & 31) < WARPS ? sm.warp_d[threadIdx.x & 31][i] : 0.;
#pragma unroll
    for (int o = 8; o > 0; o /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xFFFFFFFFu, v[i], o);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __shfl_sync(0xFFFFFFFFu, v[i], 0);
}

// Inclusive sums over a warp
template <typename T>
__device__ __forceinline__ T warp_upto(T v) {
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
        const T x = __shfl_up_sync(0xFFFFFFFFu, v, o);
        if ((threadIdx.x & 31) >= o) v += x;
    }
    return v;
}

// What a row asks for
struct Ask {
    float top;       // its largest logit
    Weights weights;
    int k;           // 0: no limit
    double p, m, u;  // p >= 1, m <= 0: no limit
};

// (formed anew by sample_any(): an argument of that size would lie in local memory, which the logits on their way push out of L1)
__device__ __forceinline__ Ask ask_of(const SampleParams &s, const double *power, int r, float top) {
    Ask a;
    const float t = s.temperature ? s.temperature[r] : s.temperature_all, p = s.top_p ? s.top_p[r] : s.top_p_all;
    a.k = s.top_k ? s.top_k[r] : s.top_k_all;
    a.k = a.k <= 0 || a.k >= s.vocab ? 0 : a.k;
    a.p = fmaxf(p, 0.f);
    a.m = fminf(s.min_p ? s.min_p[r] : s.min_p_all, 1.f);
    a.u = s.uniforms[r];
    a.top = top;
    a.weights.power = power;
    a.weights.top = top;
    a.weights.per_nat = LOG2E / static_cast<double>(t);
    a.weights.per_hi = static_cast<float>(fmin(a.weights.per_nat, 1e30));
    a.weights.per_lo = static_cast<float>(fmin(a.weights.per_nat, 1e30) - static_cast<double>(a.weights.per_hi));
    return a;
}

__device__ __forceinline__ void give(const SampleParams &s, int r, int id, float logprob) {
    if (threadIdx.x == 0) {
        s.ids[r] = id;
        if (s.logprob) s.logprob[r] = logprob;
    }
}

__device__ __forceinline__ float logprob_of(const Ask &a, float x, double mass) {
    return static_cast<float>((static_cast<double>(x) - a.weights.top) * a.weights.per_nat * (1. / LOG2E) - log(mass));
}

__device__ __forceinline__ uint32_t n_cluster_ctas() {
    uint32_t n;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return n;
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
        auto add = [&](uint32_t o, u64 w) {   // (two native additions of 32 bits with the carry: one of 64 would be tried until it succeeds)
            uint32_t *at = reinterpret_cast<uint32_t *>(&sm.mass256[(o >> shift) & 255]);
            const uint32_t low = static_cast<uint32_t>(w), old = atomicAdd(at, low);
            atomicAdd(at + 1, static_cast<uint32_t>(w >> 32) + (old + low < old));
        };
        row.template visit<1, true>(0, 1, [&](int, float x) {
            const uint32_t o = order_of(x);
            if (o > k_key && (shift == 24 || (o ^ key) >> (shift + 8) == 0)) {
                // of the lanes' digits the first few are added up in the warp: at first most logits have one of very few
                const u64 w = COUNTS ? 1ull : weight(x);
                const uint32_t digit = (o >> shift) & 255;
                uint32_t active = __activemask();
                bool done = false;
#pragma unroll 1
                for (int round = 0; round < 4 && active; ++round) {
                    const int leader = __ffs(active) - 1;
                    const uint32_t theirs = __shfl_sync(active, digit, leader);
                    const uint32_t group = __ballot_sync(active, digit == theirs);
                    if (digit == theirs) {
                        // sums of up to 32 numbers of 27 bits (w < 2^62)
                        const uint32_t a = __reduce_add_sync(group, static_cast<uint32_t>(w) & 0x7FFFFFFu);
                        const uint32_t b = COUNTS ? 0u : __reduce_add_sync(group, static_cast<uint32_t>(w >> 27) & 0x7FFFFFFu);
                        const uint32_t c = COUNTS ? 0u : __reduce_add_sync(group, static_cast<uint32_t>(w >> 54));
                        if ((threadIdx.x & 31) == leader) add(o, (static_cast<u64>(c) << 54) + (static_cast<u64>(b) << 27) + a);
                        done = true;
                        break;
                    }
                    active &= ~group;
                }
                if (!done) add(o, w);
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
__device__ __noinline__ void sample_any(const SampleParams &s, Smem &sm, int r, float top, bool summed) {
    const Ask a = ask_of(s, sm.power, r, top);
    const Row<H16> row(s.logits, r * s.row_stride, s.vocab);
    // the unit of the integers: the sum of all weights (in 32 bits, from pass 2, where that was) lies between 2^60 and 2^61, so what vocab
    // roundings do to a sum is below vocab 2^-61 of all
    double about = 0.;
    if (summed) {
        for (int c = 0; c < static_cast<int>(n_cluster_ctas()); ++c) about += sm.all[c];
    } else {
        double all[1] = {0.};
        row.template visit<1, true>(0, 1, [&](int, float x) { all[0] += a.weights.of(x); });
        block_sums(sm, all);
        about = all[0];
    }
    const double one = static_cast<double>(1ull << (60 - ilogb(about)));
    uint32_t k_key = 0;
    u64 k_ties = 0, want, above, total;
    if (a.k > 0 && a.k < s.vocab) {
        k_key = descend<H16, true>(sm, row, 0u, 0, [](float) { return 1ull; }, [&](u64) { return static_cast<u64>(a.k); }, want, above, total);
        k_ties = a.k - above;
    }
    auto weight = [&](float x) -> u64 {
        const double w = a.weights.of(x);
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
    uint32_t mine = 0;
    for (int i = lo; i < hi; ++i) mine += order_of(row.at(i)) == key;
    const uint32_t upto_mine = warp_upto(mine);
    if ((threadIdx.x & 31) == 31) sm.warp_u[threadIdx.x >> 5] = upto_mine;
    __syncthreads();
    uint32_t before = upto_mine - mine, all = 0;
    for (int w = 0; w < WARPS; ++w) {
        if (w < threadIdx.x >> 5) before += sm.warp_u[w];
        all += sm.warp_u[w];
    }
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
    give(s, r, static_cast<int>(sm.found), logprob_of(a, value_of(key), static_cast<double>(mass) / one));
}

// ---------------------------------------------------------------- the three passes

template <typename T>
__device__ __forceinline__ T *in_cta(T *p, uint32_t rank) {   // the same place in another CTA of the cluster
    T *q;
    asm volatile("mapa.u64 %0, %1, %2;" : "=l"(q) : "l"(p), "r"(rank));
    return q;
}

// The counts of the row, range by range, as its distribution.  A logit of a range weighs as much as one in its middle, give or
// take width / sqrt(12).  By how much the sum of all weights differs from the ranges' is known, and the ranges before a place have
// a part of that in proportion to their variance (share = difference / variance of all); what is then left of the variance is that
// of a bridge, small behind the few largest logits, which have most of it.
struct Distribution {
    const uint32_t *count;
    float share, var_all, inv_var, mass_all;
};

// A range, and what lies before it and up to its end: logits, about what they weigh, and how far that may be off
struct Place {
    int range;
    uint32_t n0, n1;
    float mass0, mass1, off;
};

// The first range up to whose end the row has `want` of the mass (OF_MASS) or logits (OF_COUNT), or range number `want`, or the last
// one.  A whole warp; each half of it looks for its own `want`.
enum By { OF_MASS, OF_COUNT, OF_RANGE };
__device__ __forceinline__ Place find(const Smem &sm, const Distribution &d, By by, float want_mass, uint32_t want) {
    static_assert(THREADS == 512 && PER == 16, "three steps of 16, 16 and 2, then 16 ranges, one a lane of a half");
    const int lane = threadIdx.x & 31, l = lane & 15, half = lane & 16;
    auto first = [&](bool reached, int none) {   // of the lanes of the half
        const uint32_t some = __ballot_sync(0xFFFFFFFFu, reached) >> half & 0xFFFFu;
        return some ? __ffs(some) - 1 : none;
    };
    auto reached = [&](int i) { return by == OF_MASS ? sm.mass[i] + d.share * sm.var[i] >= want_mass : sm.before[i] >= want; };
    int block = 32 * first(reached(32 * (l + 1)), 15);
    block += 2 * first(reached(block + 2 * (l + 1)), 15);
    block += first(l < 2 && reached(block + (l & 1) + 1), 1);
    if (by == OF_RANGE) block = want / PER;
    const int r = block * PER + l;
    const uint32_t n = d.count[r];
    float w, v;
    Ranges::weigh(r, w, v);
    uint32_t n_up = n;
    float up = n * w, v_up = n * v;
#pragma unroll
    for (int o = 1; o < 16; o *= 2) {
        const uint32_t x = __shfl_up_sync(0xFFFFFFFFu, n_up, o, 16);
        const float y = __shfl_up_sync(0xFFFFFFFFu, up, o, 16), z = __shfl_up_sync(0xFFFFFFFFu, v_up, o, 16);
        if (l >= o) {
            n_up += x;
            up += y;
            v_up += z;
        }
    }
    n_up += sm.before[block];
    v_up += sm.var[block];
    const float mass = up + sm.mass[block] + d.share * v_up;
    const int at = first(by == OF_MASS ? mass >= want_mass : (by == OF_COUNT ? n_up >= want : r == want), 15);
    Place p;
    p.range = block * PER + at;
    p.n1 = __shfl_sync(0xFFFFFFFFu, n_up, at, 16);
    p.n0 = p.n1 - __shfl_sync(0xFFFFFFFFu, n, at, 16);
    p.mass1 = __shfl_sync(0xFFFFFFFFu, mass, at, 16);
    const float before = __shfl_sync(0xFFFFFFFFu, mass, max(at - 1, 0), 16), v0 = __shfl_sync(0xFFFFFFFFu, v_up, max(at - 1, 0), 16);
    const float v1 = __shfl_sync(0xFFFFFFFFu, v_up, at, 16), v_begin = at ? v0 : sm.var[block];
    p.mass0 = at ? before : sm.mass[block] + d.share * v_begin;
    // (five standard deviations, at whichever end is more, and the roundings of the sums)
    const float g = fmaxf(fmaxf(v_begin * (d.var_all - v_begin), v1 * (d.var_all - v1)) * d.inv_var, 0.f);
    p.off = g * rsqrtf(fmaxf(g, 1e-37f)) * 5.f + ROUNDINGS * d.mass_all;
    return p;
}

template <bool H16>
__global__ void __launch_bounds__(THREADS, 2) sample_kernel(const __grid_constant__ SampleParams s) {
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Smem &sm = *reinterpret_cast<Smem *>(smem_raw);
    const int parts = n_cluster_ctas(), part = cluster_ctarank();
    const int r = blockIdx.x / parts, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    cluster_arrive();   // (waited for before the first store into another CTA's shared memory: by then all of them run)
    for (int i = tid; i < RANGES / 4; i += THREADS) reinterpret_cast<uint4 *>(sm.count)[i] = make_uint4(0u, 0u, 0u, 0u);
    for (int i = tid; i < STEPS; i += THREADS) sm.power[i] = exp2(i * (-1. / STEPS));
    if (tid == 0) sm.n_aside = 0;
    pdl_wait();
    pdl_trigger();
    const Row<H16> row(s.logits, r * s.row_stride, s.vocab);
    const float t = s.temperature ? s.temperature[r] : s.temperature_all, u = s.uniforms[r];
    const float p = s.top_p ? s.top_p[r] : s.top_p_all, m = s.min_p ? s.min_p[r] : s.min_p_all;

    // 1: the maximum
    float top = -INFINITY;
    {
        row.template visit<4, false>(part, parts, [&](int, float x) { top = max_nan(top, x); });
#pragma unroll
        for (int o = 16; o > 0; o /= 2) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
        if (lane == 0) sm.warp_f[warp] = top;
        __syncthreads();
        cluster_wait();
        if (warp == 0) {   // to every CTA of the cluster
            top = lane < WARPS ? sm.warp_f[lane] : -INFINITY;
#pragma unroll
            for (int o = 8; o > 0; o /= 2) top = max_nan(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            top = __shfl_sync(0xFFFFFFFFu, top, 0);
            if (lane < parts) *in_cta(&sm.top[part], lane) = top;
        }
        cluster_sync_all();
        top = -INFINITY;
        for (int i = 0; i < parts; ++i) top = max_nan(top, sm.top[i]);
        // (one of the row's logits is NaN or the largest infinite; parameters out of range)
        if (!(fabsf(top) < INFINITY) || !(t >= 0.f && t < INFINITY && u >= 0.f && u < 1.f) || p != p || m != m) {
            if (part == 0) give(s, r, -1, NAN);
            return;
        }
    }
    const Ask a = ask_of(s, sm.power, r, top);
    if (t == 0.f || a.k == 1) {   // the likeliest token, of several the first
        int first = INT_MAX;
        row.template visit<2, false>(part, parts, [&](int i, float x) {
            if (x == a.top) first = min(first, i);
        });
        first = __reduce_min_sync(0xFFFFFFFFu, first);
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
    // The passes below take log2(e) / T in two pieces of 32 bits, and differences of logits in 32: beyond these temperatures a piece is no
    // normal number, and logits that count may be further apart than fp32 holds.
    if (!(t > 1e-29f && t < 1e29f)) {
        if (part == 0) sample_any<H16>(s, sm, r, top, false);
        return;
    }
    // 2: how many logits in each range
    const float per = a.weights.per_hi;
    auto range_of = [&](float x) { return Below(x, top, per).range(); };
    {
        float sum = 0.f;
        row.template visit<2, false>(part, parts, [&](int, float x) {
            const Below y(x, top, per);
            atomicAdd(&sm.count[y.range()], 1u);
            sum += ex2_approx(-y.t);
        });
        double all[1] = {sum};
        block_sums(sm, all);
        if (tid < parts) *in_cta(&sm.all[part], tid) = all[0];
    }
    cluster_sync_all();
    Distribution d;
    d.count = sm.count;
    if (parts > 1) {   // every CTA adds up its share of the ranges, for all
        const int some = RANGES / parts;
#pragma unroll 1
        for (int i = part * some + 2 * tid; i < (part + 1) * some; i += 2 * THREADS) {
            uint2 x[MAX_CLUSTER], sum = make_uint2(0u, 0u);
#pragma unroll
            for (int c = 0; c < MAX_CLUSTER; ++c)
                if (c < parts) x[c] = *reinterpret_cast<const uint2 *>(in_cta(&sm.count[i], c));
#pragma unroll
            for (int c = 0; c < MAX_CLUSTER; ++c)
                if (c < parts) {
                    sum.x += x[c].x;
                    sum.y += x[c].y;
                }
#pragma unroll
            for (int c = 0; c < MAX_CLUSTER; ++c)
                if (c < parts) *reinterpret_cast<uint2 *>(in_cta(&sm.row_count[i], c)) = sum;
        }
        d.count = sm.row_count;
        cluster_sync_all();
    }
    {
        d.mass_all = 0.f;
        for (int c = 0; c < parts; ++c) d.mass_all += static_cast<float>(sm.all[c]);
        uint32_t n_mine = 0;
        float mass = 0.f, var = 0.f;
#pragma unroll 1
        for (int i = 0; i < PER; i += 4) {
            const uint4 x = *reinterpret_cast<const uint4 *>(&d.count[tid * PER + i]);
            const uint32_t n[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float w, v;
                Ranges::weigh(tid * PER + i + j, w, v);
                n_mine += n[j];
                mass += n[j] * w;
                var += n[j] * v;
            }
        }
        uint32_t n_up = warp_upto(n_mine);
        float up = warp_upto(mass), v_up = warp_upto(var);
        if (lane == 31) {
            sm.warp_u[warp] = n_up;
            sm.warp_f[warp] = up;
            sm.warp_v[warp] = v_up;
        }
        __syncthreads();
        const uint32_t n_w = warp_upto(lane < WARPS ? sm.warp_u[lane] : 0u);
        const float m_w = warp_upto(lane < WARPS ? sm.warp_f[lane] : 0.f), v_w = warp_upto(lane < WARPS ? sm.warp_v[lane] : 0.f);
        const uint32_t n_0 = __shfl_sync(0xFFFFFFFFu, n_w, max(warp - 1, 0));
        const float m_0 = __shfl_sync(0xFFFFFFFFu, m_w, max(warp - 1, 0)), v_0 = __shfl_sync(0xFFFFFFFFu, v_w, max(warp - 1, 0));
        sm.before[tid + 1] = n_up + (warp ? n_0 : 0u);
        sm.mass[tid + 1] = up + (warp ? m_0 : 0.f);
        sm.var[tid + 1] = v_up + (warp ? v_0 : 0.f);
        if (tid == 0) {
            sm.before[0] = 0;
            sm.mass[0] = sm.var[0] = 0.f;
        }
        const float total = __shfl_sync(0xFFFFFFFFu, m_w, 31);
        d.var_all = __shfl_sync(0xFFFFFFFFu, v_w, 31);
        d.inv_var = d.var_all > 0.f ? 1.f / d.var_all : 0.f;
        d.share = (d.mass_all - total) * d.inv_var;
        __syncthreads();
    }
    // Windows of ranges: of the limits (top_k, min_p), of the end of top_p, of the token.  (One warp of every CTA; they find the same.)
    if (warp == 0) {
        // (no limits, or none that is reached before the last range: all but that range, where the weights of 2^24 tokens together are less
        // than 10^-34 of the largest.  With the range in the window, 20 allowed tokens of 50257 and a top_k of 50 took 310 us a row in place of 14.)
        const uint32_t n_all = s.vocab - d.count[RANGES - 1];
        int e0 = RANGES - 1, e1 = RANGES - 2, p0 = e0, p1 = e1, s0 = e0, s1 = e1;
        uint32_t e_n0 = n_all, e_n1 = n_all, p_n0 = 0, p_n1 = 0, s_n0 = 0, s_n1 = 0;
        float mass_lo = d.mass_all * (1.f - ROUNDINGS), mass_hi = d.mass_all * (1.f + ROUNDINGS);   // of what is left, so far
        const bool hi = lane >= 16;   // the lower half looks for the lower end of a window
        auto of = [&](auto v, int end) { return __shfl_sync(0xFFFFFFFFu, v, end * 16); };
        int m0 = 0, m1 = 0;
        if (a.m > 0.) {
            const float y = -__log2f(static_cast<float>(a.m)), slack = 1e-5f * (1.f + y);
            m0 = Below(0.f, fmaxf(0.f, y - slack), 1.f).range();
            m1 = Below(0.f, y + slack, 1.f).range();
        }
        float wanted = 0.f;   // by this half
#pragma unroll 1
        for (int step = 0; step < 6; ++step) {   // (one copy of the search: code that runs a few times a row takes its time to be fetched)
            // 0: the end of the first top_k   1: the range of min_p   2: the end of top_p   4: the token   3, 5: 2 and 4 with what may be off
            if (step == 0 ? a.k == 0 : (step == 1 ? !(a.m > 0.) || e0 < m0 : (step <= 3 && a.p >= 1.))) continue;
            if (step == 2 || step == 4) wanted = (step == 2 ? static_cast<float>(a.p) : u) * (hi ? mass_hi : mass_lo);
            const Place f = find(sm, d, step == 0 ? OF_COUNT : (step == 1 ? OF_RANGE : OF_MASS), wanted, step == 0 ? a.k : (hi ? m1 : m0));
            if (step == 2 || step == 4) {
                wanted += hi ? f.off : -f.off;
                if (__any_sync(0xFFFFFFFFu, hi ? wanted > f.mass1 : wanted < f.mass0)) continue;   // not in the same range
                ++step;
            }
            const int from = of(f.range, 0), to = of(f.range, 1);
            const uint32_t n0 = of(f.n0, 0), n1 = of(f.n1, 1);
            if (step <= 1) {
                if (from == RANGES - 1) continue;   // (no limit either: what it cuts off or leaves is in the last range)
                e0 = from;
                e1 = to;
                e_n0 = n0;
                e_n1 = n1;
                mass_lo = of(f.mass0 - f.off, 0);
                mass_hi = of(f.mass1 + f.off, 1);
            } else if (step == 3) {
                p0 = from < e0 ? from : e0;
                p_n0 = from < e0 ? n0 : e_n0;
                p1 = to < e1 ? to : e1;
                p_n1 = to < e1 ? n1 : e_n1;
                mass_lo = of(wanted, 0);
                // (up to the end of a token)
                mass_hi = fminf(of(wanted, 1) + ex2_approx(-Ranges::begin(from)), of(f.mass1 + f.off, 1));
            } else {
                s0 = from;
                s_n0 = n0;
                s1 = to;
                s_n1 = n1;
            }
        }
        if (a.p >= 1.) {
            p0 = e0;
            p1 = e1;
            p_n0 = e_n0;
            p_n1 = e_n1;
        }
        if (s0 > p0) {
            s0 = p0;
            s_n0 = p_n0;
        }
        if (s1 > p1) {
            s1 = p1;
            s_n1 = p_n1;
        }
        // logits between the windows
        const uint32_t n_gap0 = s_n0, n_gap1 = p0 > s1 ? p_n0 - s_n1 : 0, n_gap2 = e0 > p1 ? e_n0 - p_n1 : 0;
        const uint32_t n_aside = e_n1 - n_gap0 - n_gap1 - n_gap2;
        if (lane == 0) sm.windows = {s0, s1, p0, p1, e0, e1, n_gap0, n_gap1, n_gap2, n_aside};
    }
    __syncthreads();
    const int s0 = sm.windows.s0, s1 = sm.windows.s1, p0 = sm.windows.p0, p1 = sm.windows.p1, e0 = sm.windows.e0, e1 = sm.windows.e1;
    const uint32_t n_gap0 = sm.windows.n_gap0, n_gap1 = sm.windows.n_gap1, n_gap2 = sm.windows.n_gap2, n_aside = sm.windows.n_aside;
    if (n_aside > ROOM) {   // (the same for every CTA)
        cluster_sync_all();   // (all have read the others' counts)
        if (part == 0) sample_any<H16>(s, sm, r, top, true);
        return;
    }

    // 3: sums and windows
    {
        double sums[3] = {0., 0., 0.};
        u64 *list = in_cta(&sm.aside[0], 0u);
        uint32_t *n = in_cta(&sm.n_aside, 0u);
        // where the windows begin and end, in steps
        const int at_s = Ranges::first(s0), after_s = Ranges::first(s1 + 1), at_p = Ranges::first(p0), after_p = Ranges::first(p1 + 1);
        const int at_e = Ranges::first(e0), after_e = Ranges::first(e1 + 1);
        row.template visit<1, H16>(part, parts, [&](int i, float x) {
            const Below y(x, top, per);
            if (y.k >= after_e) return;
            if (y.k >= (y.k >= after_p ? at_e : (y.k >= after_s ? at_p : at_s))) {
                list[atomicAdd(n, 1u)] = static_cast<u64>(order_of(x)) << 32 | static_cast<uint32_t>(~i);
                return;
            }
            const double w = a.weights.fast(x, y);
            if (y.k >= after_p) sums[2] += w;
            else if (y.k >= after_s) sums[1] += w;
            else sums[0] += w;
        });
        block_sums(sm, sums);
        if (tid == 0) {
            double *to = in_cta(&sm.gaps[part][0], 0u);
            to[0] = sums[0];
            to[1] = sums[1];
            to[2] = sums[2];
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
    // in descending order: by counting how many are larger, some threads a key, where there are few; else a bitonic sort
    int size = 32;
    while (size < (int)n_aside) size *= 2;
    if (size <= THREADS) {
        const int each = THREADS / size, i = tid / each;   // threads of a key (at most 16)
        const u64 key = i < (int)n_aside ? sm.aside[i] : 0;
        int rank = 0;
#pragma unroll 8
        for (int j = tid & (each - 1); j < (int)n_aside; j += each) rank += sm.aside[j] > key;
#pragma unroll 1
        for (int o = each / 2; o > 0; o /= 2) rank += __shfl_xor_sync(0xFFFFFFFFu, rank, o);
        __syncthreads();
        if (i < (int)n_aside && (tid & (each - 1)) == 0) sm.aside[rank] = key;
    } else {
        for (int i = n_aside + tid; i < size; i += THREADS) sm.aside[i] = 0;
#pragma unroll 1
        for (int k = 2; k <= size; k *= 2)
#pragma unroll 1
            for (int j = k / 2; j > 0; j /= 2) {
                __syncthreads();
#pragma unroll 1
                for (int i = tid; i < size / 2; i += THREADS) {
                    const int lo = 2 * i - (i & (j - 1)), hi = lo + j;
                    const u64 x = sm.aside[lo], y = sm.aside[hi];
                    if ((x < y) == ((lo & k) == 0)) {
                        sm.aside[lo] = y;
                        sm.aside[hi] = x;
                    }
                }
            }
    }
    __syncthreads();
    // The borders among them.  Few: one warp, and the others wait for what it finds.
    const bool alone = n_aside <= 256;
    const int threads = alone ? 32 : THREADS;
    double mass = 0.;
    if (!alone || warp == 0) {
        // thread i has `per` places of the order from per i on
        const int per = (n_aside + threads - 1) / threads, lo = min((int)n_aside, tid * per), hi = min((int)n_aside, lo + per);
        auto value = [&](int i) { return value_of(static_cast<uint32_t>(sm.aside[i] >> 32)); };
        double mine = 0.;
#pragma unroll 1
        for (int i = lo; i < hi; ++i) {
            const double w = a.weights.of(value(i));
            sm.weight[i] = w;
            mine += w;
        }
        const double upto = warp_upto(mine);
        double before = upto - mine;
        if (!alone) {
            if (lane == 31) sm.warp_d[warp][0] = upto;
            __syncthreads();
            for (int w = 0; w < warp; ++w) before += sm.warp_d[w][0];
        }
        // what is left by the limits; the weights in the window of the token, and up to the end of that of top_p; those put aside before it
        double sums[3] = {0., 0., 0.}, before_p = 0.;
        auto left = [&](int i, int range) {
            const uint32_t rank = i + n_gap0 + (range > s1 ? n_gap1 : 0) + (range > p1 ? n_gap2 : 0);
            return rank == 0 || ((a.k == 0 || rank < a.k) && sm.weight[i] >= a.m);
        };
#pragma unroll 1
        for (int i = lo; i < hi; ++i) {
            const int range = range_of(value(i));
            const double w = sm.weight[i];
            if (left(i, range)) sums[0] += w;
            if (range <= s1) sums[1] += w;
            if (range <= p1) sums[2] += w;
            if (range < p0) before_p += w;
        }
        block_sums(sm, sums, alone);
        const double z = sums[0] + gap0 + gap1 + gap2, in_s = sums[1], in_p = sums[2], want_p = a.p * z;
        mass = z;
        bool fits = true;
        auto kept = [&](int i, int range, double up) {   // `up`: the weights put aside before it
            if (!left(i, range)) return false;
            if (a.p >= 1. || i + n_gap0 == 0) return true;
            return up + gap0 + (range > s1 ? gap1 : 0.) + (range > p1 ? gap2 : 0.) < want_p;
        };
        if (a.p < 1.) {
            double more[2] = {0., before_p}, up = before;
#pragma unroll 1
            for (int i = lo; i < hi; ++i) {
                const double w = sm.weight[i];
                if (kept(i, range_of(value(i)), up)) more[0] += w;
                up += w;
            }
            block_sums(sm, more, alone);
            mass = more[0] + gap0 + gap1;
            fits = (more[1] + gap0 + gap1 <= want_p || (p0 == 0 && s0 == 0)) && want_p <= gap0 + gap1 + in_p;
        }
        const double want = a.u * mass;
        fits = fits && gap0 <= want && want < gap0 + in_s;
        // the first one kept up to which there is more than `want`; where the sums, rounded otherwise than `mass`, fall short of it, the last
        int token = INT_MAX, last = -1;
        {
            double up = before;
#pragma unroll 1
            for (int i = lo; i < hi; ++i) {
                const int range = range_of(value(i));
                const bool is = kept(i, range, up) && range <= s1;
                up += sm.weight[i];
                if (is) last = i;
                if (is && token == INT_MAX && gap0 + up > want) token = i;
            }
        }
        token = __reduce_min_sync(0xFFFFFFFFu, token);
        last = __reduce_max_sync(0xFFFFFFFFu, last);
        if (!alone) {
            if (lane == 0) {
                sm.warp_u[warp] = token;
                reinterpret_cast<int *>(sm.warp_f)[warp] = last;
            }
            __syncthreads();
            token = __reduce_min_sync(0xFFFFFFFFu, lane < WARPS ? static_cast<int>(sm.warp_u[lane]) : INT_MAX);
            last = __reduce_max_sync(0xFFFFFFFFu, lane < WARPS ? reinterpret_cast<int *>(sm.warp_f)[lane] : -1);
        }
        if (token == INT_MAX) token = last;
        if (tid == 0) sm.token = fits ? token : -1;
    }
    __syncthreads();
    if (sm.token < 0) {
        sample_any<H16>(s, sm, r, top, true);
        return;
    }
    if (tid == 0) {
        const u64 e = sm.aside[sm.token];
        s.ids[r] = static_cast<int>(~static_cast<uint32_t>(e));
        if (s.logprob) s.logprob[r] = logprob_of(a, value_of(static_cast<uint32_t>(e >> 32)), mass);
    }
}

constexpr int SHARED_SMEM = sizeof(Smem) + RANGES * sizeof(uint32_t);

template <bool H16>
int launch(const SampleParams &p, cudaStream_t st) {
    static DeviceOnce configured;
    if (!configured.done()) {
        int rc = cuda_check(cudaFuncSetAttribute(sample_kernel<H16>, cudaFuncAttributeMaxDynamicSharedMemorySize, SHARED_SMEM),
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
    cfg.dynamicSmemBytes = cluster > 1 ? SHARED_SMEM : sizeof(Smem);
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
