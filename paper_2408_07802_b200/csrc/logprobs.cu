// Log probability of a given token, entropy and the largest logits of every row, in one pass over the logits.
//
//   x = scale * logit, m = max x, S = sum e^(x - m):  lse = m + log S,  logprob = x_t - lse,
//   entropy = log S + sum (m - x) e^(x - m) / S       (every term of the sum is positive: nothing cancels)
//
// 4 (or 2) bytes a logit against 13 instructions (2048 x 50257, k = 5): 148 SMs can issue those of 2.9e12 logits a second, so fp32
// is bound by HBM and 16-bit logits by issue.  Every thread keeps a maximum and the two sums of its own logits, brought to a larger
// maximum 16 logits at a time; the threads of a row meet at the end.
//
// The alternatives are found in the same pass.  After chunks 1, 3, 9, 27 ... the largest logits so far of groups of 4 threads are
// looked at: the k-th largest of them is a bound that k logits reach.  A thread compares the maximum of its 16 logits, which
// it has anyway, with the bound and where it is reached notes its place and that maximum: some 100 of a row for k = 20.  At the
// end the bound is taken once more, the places whose maximum reaches it are read again and the logits that do, not many more
// than k, are ranked by counting, by keys of a logit and its index whose order is that of the list.  Where more places or
// logits reach the bound than there is room for (a vocabulary in rising order, or of few different values) the row is gone
// through again by exact_top(), which works with the distinct keys and cuts down what it has put aside.
// Measured on 2048 x 50257 fp32: 72.3 us with k = 5 (5.7 TB/s), 62.6 without alternatives (6.6 TB/s, the copy bandwidth); bf16 57.0
// and 43.4 us.  Spills: 4 loads and 18 stores a warp and row, none in the loop over the chunks.  Logits
// put aside at once (a warp then goes through the 16 of a thread some hundred times a row): 98 us with k = 20 against 80; looks
// without barriers at 32 groups: 144 with k = 32; a ring of bulk copies filled by a warp of its own: 88 with k = 5.
//
// Few rows: up to 8 CTAs of a cluster share a row and join through each other's shared memory.
#include <float.h>
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace kr {

namespace {

constexpr int LP_MAX_TOP = KRAKEN_LOGPROBS_MAX_TOP;
constexpr int PER_THREAD = 16;                       // logits of a thread in a chunk
constexpr int GROUP = 4;
constexpr int MAX_CLUSTER = 8;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.69314718055994531f;
typedef unsigned long long Key;

// Threads of a CTA and CTAs of an SM.  Smaller CTAs keep more rows going side by side, one's end beside another's middle, but
// take longer over a single row, and their bounds from fewer groups (2048 x 50257 with 128 threads against 256, fp32: k = 5 72.5
// against 76 us, k = 20 80 against 84; bf16: 57 against 67, 63 against 70; 592 rows, fp32, k = 5: 29 against 26).
template <int T>
struct Shape {
    static constexpr int WARPS = T / 32, CTAS = 1024 / T, GROUPS = T / GROUP;
    static constexpr int TOP = T == 128 ? 20 : LP_MAX_TOP;                       // alternatives at most
    static constexpr int CHUNK_ADDS = (TOP - 1) * GROUP * PER_THREAD + 1;       // see exact_top
    // room for keys put aside and for places noted.  (Shared memory is taken from L1, which the loads on their way go through:
    // 27 KB for each of 8 CTAs made the sums alone of 2048 x 50257 take 87 us instead of 63.)
    static constexpr int ASIDE = T == 128 ? 1280 : 2048, PLACES = T == 128 ? 512 : 896;
    static_assert(GROUPS >= TOP, "the bound is the k-th of the groups");
    static_assert(ASIDE > CHUNK_ADDS + TOP, "after a cut a chunk has to fit");
};

struct LogprobParams {
    const void *logits;
    long long row_stride;
    const int *targets;
    float *logprob, *entropy, *lse;
    int *top_ids;
    float *top_logprobs;
    int rows, vocab, top;
    float scale;
    uint32_t *status;
};

// Larger logit first, of equal ones the lower index; NaN as -inf; -0 and +0 are equal.  Every key is above 0.
__device__ __forceinline__ Key order_key(float x, int i) {
    if (!(x > -INFINITY)) x = -INFINITY;
    const uint32_t u = __float_as_uint(x + 0.f);
    const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return (static_cast<Key>(o) << 32) | static_cast<uint32_t>(~i);
}

__device__ __forceinline__ float key_value(Key k) {
    const uint32_t o = static_cast<uint32_t>(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}

// Sum of 2^u and of u 2^u, u = (x - base) k, over some logits; base = their maximum m, or 0 for -inf
struct Sums {
    float m, s, d;
    __device__ __forceinline__ float base() const { return m == -INFINITY ? 0.f : m; }
    __device__ __forceinline__ void rise_to(float mx, float k) {
        if (mx == m) return;
        if (m > -INFINITY) {
            const float step = fminf((mx - m) * k, 1000.f), c = ex2_approx(-step);   // (2^-1000: 0)
            d = (d - s * step) * c;
            s *= c;
        }
        m = mx;
    }
    __device__ __forceinline__ void join(Sums o, float k) {
        const float mx = fmaxf(m, o.m);
        rise_to(mx, k);
        o.rise_to(mx, k);
        s += o.s;
        d += o.d;
    }
};

template <int T>
struct Smem {
    Key aside[Shape<T>::ASIDE];
    Key group[Shape<T>::GROUPS];
    float high[Shape<T>::GROUPS];
    Key list[MAX_CLUSTER * LP_MAX_TOP];   // of every CTA of the cluster, in order; 0: none
    Key tau;
    float bound;
    float2 places[Shape<T>::PLACES];    // largest logit of the 16, and (as bits) chunk * T + thread
    int noted;
    int count;                // keys put aside
    int sum;
    Sums warp[Shape<T>::WARPS], cta[MAX_CLUSTER];
};

template <bool H16>
struct Chunk {   // 16 logits of a thread, in vectors of 16 bytes
    static constexpr int VEC = H16 ? 8 : 4, VECS = PER_THREAD / VEC;
    uint4 raw[VECS];
    __device__ __forceinline__ float at(int i) const {   // i known when compiled
        const uint4 &v = raw[i / VEC];
        const int e = i % VEC;
        if (H16) {
            const uint32_t w = e / 2 == 0 ? v.x : (e / 2 == 1 ? v.y : (e / 2 == 2 ? v.z : v.w));
            return (e & 1) ? h16_hi(w) : h16_lo(w);
        }
        return __uint_as_float(e == 0 ? v.x : (e == 1 ? v.y : (e == 2 ? v.z : v.w)));
    }
};

// The k-th largest of the groups' largest logits.  All threads; two barriers.
template <int T>
__device__ __forceinline__ float kth_of_groups(Smem<T> &sm, float high, int k) {
    static_assert(GROUP == 4, "the threads of a group rank its logit");
#pragma unroll
    for (int off = 1; off < GROUP; off <<= 1) high = fmaxf(high, __shfl_xor_sync(0xFFFFFFFFu, high, off));
    if (threadIdx.x % GROUP == 0) sm.high[threadIdx.x / GROUP] = high;
    __syncthreads();
    int ranks = 0;   // logits above, and in the upper half those equal
#pragma unroll
    for (int i = 0; i < Shape<T>::GROUPS; i += GROUP) {
        const float x = sm.high[i + threadIdx.x % GROUP];
        ranks += (x > high ? 1 : 0) + (x == high ? 1 << 16 : 0);
    }
    ranks += __shfl_xor_sync(0xFFFFFFFFu, ranks, 1);
    ranks += __shfl_xor_sync(0xFFFFFFFFu, ranks, 2);
    const int above = ranks & 0xFFFF, equal = ranks >> 16;
    if (above < k && above + equal >= k) sm.bound = high;   // (one value, from one or more threads)
    __syncthreads();
    return sm.bound;
}

// The same with every thread a group of its own, for parts too short to fill k groups (or forbidden but for a few logits), found
// bit by bit: the largest value that the logits of k threads reach.  All threads; 32 barriers, half as long as counting.
template <int T>
__device__ __noinline__ float kth_of_threads(float high, int k) {
    const uint32_t mine = static_cast<uint32_t>(order_key(high, 0) >> 32);
    uint32_t reached = 0;
    for (uint32_t bit = 0x80000000u; bit != 0; bit >>= 1)
        if (__syncthreads_count(mine >= (reached | bit)) >= k) reached |= bit;
    return key_value(static_cast<Key>(reached) << 32);
}

// f(rank, key) for those of n keys whose rank is below k, four threads a key.  All threads.
template <int T, typename F>
__device__ __forceinline__ void ranked(const Key *keys, int n, int k, F f) {
    for (int i0 = 0; i0 < n; i0 += T / 4) {
        const int at = i0 + threadIdx.x / 4;
        const Key mine = at < n ? keys[at] : 0;
        int above = 0;
#pragma unroll 4
        for (int i = threadIdx.x % 4; i < n; i += 4) above += keys[i] > mine;
        above += __shfl_xor_sync(0xFFFFFFFFu, above, 1);
        above += __shfl_xor_sync(0xFFFFFFFFu, above, 2);
        if (mine != 0 && above < k && threadIdx.x % 4 == 0) f(above, mine);
    }
}

// The same of the groups' largest keys; 0 when there are fewer than k.
template <int T>
__device__ __forceinline__ Key kth_of_groups(Smem<T> &sm, Key best, int k) {
#pragma unroll
    for (int off = 1; off < GROUP; off <<= 1) {
        const Key o = __shfl_xor_sync(0xFFFFFFFFu, best, off);
        best = o > best ? o : best;
    }
    if (threadIdx.x % GROUP == 0) sm.group[threadIdx.x / GROUP] = best;
    if (threadIdx.x == 0) sm.tau = 0;
    __syncthreads();
    if (threadIdx.x < Shape<T>::GROUPS) {
        const Key mine = sm.group[threadIdx.x];
        int above = 0;
#pragma unroll 16
        for (int i = 0; i < Shape<T>::GROUPS; ++i) above += sm.group[i] > mine;
        if (above == k - 1 && mine != 0) sm.tau = mine;
    }
    __syncthreads();
    return sm.tau;
}

// Cuts the n keys put aside down to the k largest and returns the smallest of these, found bit by bit.  All threads.
template <int T>
__device__ __noinline__ Key cut(Smem<T> &sm, int n, int k) {
    constexpr int MOST = (Shape<T>::ASIDE + T - 1) / T;
    Key mine[MOST];
#pragma unroll
    for (int i = 0; i < MOST; ++i) {
        const int at = threadIdx.x + i * T;
        mine[i] = at < n ? sm.aside[at] : 0;
    }
    Key tau = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const Key t = tau | (1ull << bit);
        int c = 0;
#pragma unroll
        for (int i = 0; i < MOST; ++i) c += mine[i] >= t;
        c = __reduce_add_sync(0xFFFFFFFFu, c);
        __syncthreads();
        if (threadIdx.x == 0) sm.sum = 0;
        __syncthreads();
        if ((threadIdx.x & 31) == 0 && c) atomicAdd(&sm.sum, c);
        __syncthreads();
        if (sm.sum >= k) tau = t;
    }
    if (threadIdx.x == 0) sm.count = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < MOST; ++i)
        if (mine[i] != 0 && mine[i] >= tau) sm.aside[atomicAdd(&sm.count, 1)] = mine[i];
    __syncthreads();
    return tau;
}

// The part of a row that a CTA reads, in vectors of 16 bytes that start on 16 bytes: `before` elements of the row's first
// vector lie in front of the row, and are not read any more than those behind its end.
template <bool H16, int T>
struct Span {
    using C = Chunk<H16>;
    static constexpr int VEC = C::VEC, VECS = C::VECS, SIZE = H16 ? 2 : 4, CHUNK = VECS * T;   // CHUNK: vectors
    static constexpr uint32_t NONE = H16 ? (KRAKEN_F16 ? 0xFC00FC00u : 0xFF80FF80u) : 0xFF800000u;      // -inf
    const uint8_t *row;
    const uint4 *vectors;
    int vocab, before, lo, hi;         // vectors lo .. hi - 1
    int clean_lo, clean_hi;            // of these, the ones that lie in the row whole
    int chunks;
    __device__ __forceinline__ Span(const uint8_t *r, int v, int rank, int cluster) : row(r), vocab(v) {
        before = static_cast<int>((reinterpret_cast<uintptr_t>(row) & 15) / SIZE);
        vectors = reinterpret_cast<const uint4 *>(row - before * SIZE);
        const int n = (before + vocab + VEC - 1) / VEC, per = (n + cluster - 1) / cluster;
        lo = min(n, rank * per);
        hi = min(n, lo + per);
        clean_lo = max(lo, before > 0 ? 1 : 0);
        clean_hi = min(hi, (before + vocab) / VEC);
        chunks = (hi - lo + CHUNK - 1) / CHUNK;
    }
    __device__ __forceinline__ int index(int chunk, int i) const {   // of logit i of this thread's chunk; maybe outside the part
        return (lo + (chunk * VECS + i / VEC) * T + (int)threadIdx.x) * VEC + i % VEC - before;
    }
    __device__ __forceinline__ bool has(int index) const {
        return index >= max(0, lo * VEC - before) && index < min(vocab, hi * VEC - before);
    }
    __device__ __forceinline__ void load(C &c, int chunk) const {   // -inf outside the part
        const int v0 = lo + chunk * CHUNK;
        if (v0 >= clean_lo && v0 + CHUNK <= clean_hi) {
#pragma unroll
            for (int i = 0; i < VECS; ++i) c.raw[i] = __ldcs(vectors + v0 + i * T + threadIdx.x);
            return;
        }
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int v = v0 + i * T + threadIdx.x;
            c.raw[i] = make_uint4(NONE, NONE, NONE, NONE);
            if (v >= clean_lo && v < clean_hi) {
                c.raw[i] = __ldcs(vectors + v);
            } else if (v < hi) {   // the row's first or last vector: element by element
                uint32_t w[4] = {NONE, NONE, NONE, NONE};
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const int at = v * VEC - before + e;
                    if (at < 0 || at >= vocab) continue;
                    if (H16) {
                        const uint32_t h = reinterpret_cast<const uint16_t *>(row)[at];
                        w[e / 2] = (e & 1) ? (w[e / 2] & 0xFFFFu) | (h << 16) : (w[e / 2] & 0xFFFF0000u) | h;
                    } else {
                        w[e] = reinterpret_cast<const uint32_t *>(row)[at];
                    }
                }
                c.raw[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
    __device__ __forceinline__ int first() const { return max(0, lo * VEC - before); }    // logits first .. first + count - 1
    __device__ __forceinline__ int count() const { return max(0, min(vocab, hi * VEC - before) - first()); }
    __device__ __forceinline__ float value(int at) const {
        return H16 ? from_h16(reinterpret_cast<const uint16_t *>(row)[at]) : reinterpret_cast<const float *>(row)[at];
    }
    // f(logit, index) for the logits of vector i of a thread's chunk
    template <typename F>
    __device__ __forceinline__ void each(int chunk, int thread, int i, F f) const {
        const int v = lo + (chunk * VECS + i) * T + thread;
        if (v >= clean_lo && v < clean_hi) {
            C c;
            c.raw[0] = vectors[v];
#pragma unroll
            for (int e = 0; e < VEC; ++e) f(c.at(e), v * VEC - before + e);
        } else if (v < hi) {
            for (int e = 0; e < VEC; ++e) {
                const int at = v * VEC - before + e;
                if (at < 0 || at >= vocab) continue;
                f(value(at), at);
            }
        }
    }
};

// The k largest keys of the part, and maybe some more, into sm.aside; any order, any ties.  A bound is raised from a chunk as
// long as many threads exceed it, after which a chunk adds at most (k - 1) * GROUP * PER_THREAD + 1 keys; where these might not
// fit, the keys put aside are cut down to k first.
template <bool H16, int T>
__device__ __noinline__ void exact_top(Smem<T> &sm, const Span<H16, T> &span, int k) {
    __syncthreads();
    if (threadIdx.x == 0) sm.count = 0;
    Key tau = 0;
    for (int chunk = 0; chunk < span.chunks; ++chunk) {
        Chunk<H16> c;
        span.load(c, chunk);
        Key best = 0;
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            const int at = span.index(chunk, i);
            if (!span.has(at)) continue;
            const Key key = order_key(c.at(i), at);
            best = key > best ? key : best;
        }
        const int over = __syncthreads_count(best >= tau && best != 0);
        if (over == 0) continue;
        if (chunk == 0 || over > Shape<T>::GROUPS) {
            const Key bound = kth_of_groups<T>(sm, best, k);
            tau = bound > tau ? bound : tau;
        }
        const int n = sm.count;
        if (n + Shape<T>::CHUNK_ADDS > Shape<T>::ASIDE) {
            const Key bound = cut<T>(sm, n, k);
            tau = bound > tau ? bound : tau;
        } else {
            __syncthreads();   // everyone has read the count
        }
        if (best < tau || best == 0) continue;
#pragma unroll
        for (int i = 0; i < PER_THREAD; ++i) {
            const int at = span.index(chunk, i);
            if (!span.has(at)) continue;
            const Key key = order_key(c.at(i), at);
            if (key >= tau) sm.aside[atomicAdd(&sm.count, 1)] = key;
        }
    }
    __syncthreads();
}

template <bool H16, bool TOP, int T>
__global__ void __launch_bounds__(T, Shape<T>::CTAS) logprobs_kernel(const LogprobParams p, int cluster) {
    using C = Chunk<H16>;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    Smem<T> &sm = *reinterpret_cast<Smem<T> *>(smem_raw);
    const int rank = blockIdx.x % cluster, tid = threadIdx.x;
    if (cluster > 1) {
        // the CTAs of a cluster write into the first one's shared memory at the end: by then it has to run, and to be ready
        if (TOP && rank == 0)
            for (int i = tid; i < MAX_CLUSTER * LP_MAX_TOP; i += T) sm.list[i] = 0;
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }
    pdl_wait();
    const float k2 = p.scale * LOG2E;
    const int step = gridDim.x / cluster;   // rows side by side; with clusters every row has its own
    auto row_at = [&](long long r) { return static_cast<const uint8_t *>(p.logits) + r * p.row_stride * Span<H16, T>::SIZE; };
    C cur, next;
    Span<H16, T>(row_at(blockIdx.x / cluster), p.vocab, rank, cluster).load(cur, 0);
    for (long long r = blockIdx.x / cluster; r < p.rows; r += step) {
        const uint8_t *row = row_at(r);
        float x_t = 0.f;
        int target = -1;
        if (p.logprob && rank == 0 && tid == 0) {
            target = p.targets[r];
            if (target >= 0 && target < p.vocab)
                x_t = H16 ? from_h16(reinterpret_cast<const uint16_t *>(row)[target]) : reinterpret_cast<const float *>(row)[target];
        }
        const Span<H16, T> span(row, p.vocab, rank, cluster);
        Sums run = {-INFINITY, 0.f, 0.f};
        float bound = -INFINITY;
        if (TOP && tid == 0) sm.count = sm.noted = 0;
        int look = 0;   // the chunk after which the bound is taken next
        for (int chunk = 0; chunk < span.chunks; ++chunk) {
            // with the last chunk the next row's first one is requested: the end of a row takes longer than the way to memory
            if (chunk + 1 < span.chunks) span.load(next, chunk + 1);
            else if (r + step < p.rows) Span<H16, T>(row_at(r + step), p.vocab, rank, cluster).load(next, 0);
            float high = -INFINITY;   // (a NaN is passed over)
#pragma unroll
            for (int i = 0; i < PER_THREAD; ++i) high = fmaxf(high, cur.at(i));
            run.rise_to(fmaxf(run.m, high), k2);
            const uint64_t minus_base = splat2(-run.base()), scale = splat2(k2);
            uint64_t s = splat2(0.f), d = splat2(0.f);
#pragma unroll
            for (int i = 0; i < PER_THREAD; i += 2) {
                const uint64_t u = mul2(add2(pk2(cur.at(i), cur.at(i + 1)), minus_base), scale);
                float u0, u1;
                upk2(u, u0, u1);
                const uint64_t e = pk2(ex2_approx(u0), ex2_approx(u1));
                s = add2(s, e);
                d = fma2(pk2(fmaxf(u0, -1000.f), fmaxf(u1, -1000.f)), e, d);   // (u = -inf: 0; a NaN stays one in e)
            }
            float s0, s1, d0, d1;
            upk2(s, s0, s1);
            upk2(d, d0, d1);
            run.s += s0 + s1;
            run.d += d0 + d1;
            if (TOP) {
                if (chunk == look) {
                    bound = fmaxf(bound, kth_of_groups<T>(sm, run.m, p.top));
                    if (bound == -INFINITY) bound = kth_of_threads<T>(run.m, p.top);
                    bound = fmaxf(bound, -FLT_MAX);   // no bound: every logit that is not forbidden
                    look = 3 * look + 2;
                }
                if (high >= bound) {
                    const int at = atomicAdd(&sm.noted, 1);
                    if (at < Shape<T>::PLACES) sm.places[at] = make_float2(high, __int_as_float(chunk * T + tid));
                }
            }
            cur = next;
        }

        // the logits that reach the bound of the whole part
        bool all_found = false;
        if (TOP) {
            if (look > 2) bound = fmaxf(bound, kth_of_groups<T>(sm, run.m, p.top));
            else __syncthreads();
            const int noted = sm.noted;
            all_found = noted <= Shape<T>::PLACES;
            if (all_found) {
                for (int i = tid; i < noted; i += T) {
                    if (!(sm.places[i].x >= bound)) continue;
                    const int place = __float_as_int(sm.places[i].y);
#pragma unroll
                    for (int v = 0; v < C::VECS; ++v)
                        span.each(place / T, place % T, v, [&](float x, int at) {
                            if (x >= bound) {
                                const int n = atomicAdd(&sm.count, 1);
                                if (n < Shape<T>::ASIDE) sm.aside[n] = order_key(x, at);
                            }
                        });
                }
            }
        }
        // the threads' sums
        auto over_lanes = [&](int lanes) {
            float m = run.m;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1)
                if (off < lanes) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, off));
            run.rise_to(m, k2);
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) {
                if (off >= lanes) continue;
                run.s += __shfl_xor_sync(0xFFFFFFFFu, run.s, off);
                run.d += __shfl_xor_sync(0xFFFFFFFFu, run.d, off);
            }
        };
        over_lanes(32);
        if (tid % 32 == 0) sm.warp[tid / 32] = run;
        __syncthreads();
        run = sm.warp[tid % Shape<T>::WARPS];
        over_lanes(Shape<T>::WARPS);
        const Key *keys = sm.aside;
        int n = 0;
        if (TOP) {
            n = sm.count;
            // (fewer than asked for: forbidden ones and NaN are among them)
            all_found = all_found && n <= Shape<T>::ASIDE && n >= min(p.top, span.count());
            if (!all_found && span.count() <= T) {
                // a part of a few logits: all of them
                n = span.count();
                if (tid < n) sm.aside[tid] = order_key(span.value(span.first() + tid), span.first() + tid);
                __syncthreads();
            } else if (!all_found) {
                exact_top<H16, T>(sm, span, p.top);
                n = sm.count;
            }
            if (n > 3 * T) {   // (ranking 768 keys takes half as long as cutting them down)
                __syncthreads();
                cut<T>(sm, n, p.top);
                n = sm.count;
            }
        }
        if (cluster > 1) {
            asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            if (tid == 0) {
                const uint32_t at = map_to_cta(smem_u32(&sm.cta[rank]), 0);
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at), "f"(run.m) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 4), "f"(run.s) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(at + 8), "f"(run.d) : "memory");
            }
            if (TOP) {
                const uint32_t list = map_to_cta(smem_u32(&sm.list[rank * p.top]), 0);
                ranked<T>(sm.aside, n, p.top, [&](int place, Key key) {
                    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(list + 8 * place), "l"(key) : "memory");
                });
            }
            cluster_sync_all();
            if (rank != 0) return;
            run = tid % MAX_CLUSTER < cluster ? sm.cta[tid % MAX_CLUSTER] : Sums{-INFINITY, 0.f, 0.f};
            over_lanes(MAX_CLUSTER);
            keys = sm.list;
            n = cluster * p.top;
        }
        const float m = run.base(), log_s = log2f(run.s) * LN2;
        if (TOP)
            ranked<T>(keys, n, p.top, [&](int place, Key key) {
                if (p.top_ids) p.top_ids[r * p.top + place] = static_cast<int>(~static_cast<uint32_t>(key));
                if (p.top_logprobs) p.top_logprobs[r * p.top + place] = (key_value(key) - m) * p.scale - log_s;
            });
        if (tid == 0) {
            if (p.lse) p.lse[r] = m * p.scale + log_s;
            if (p.entropy) p.entropy[r] = log_s - run.d / run.s * LN2;
            if (p.logprob) {
                float v = 0.f;
                if (target >= p.vocab) {
                    v = NAN;
                    if (p.status) atomicOr(p.status, STATUS_BAD_TOKEN);
                } else if (target >= 0) {
                    v = (x_t - m) * p.scale - log_s;
                }
                p.logprob[r] = v;
            }
        }
        __syncthreads();   // shared memory is the next row's
    }
}

// CTAs of a row: more while they do not fill half the SMs, none with less than a chunk.  (48 x 51200 bf16, k = 20: 11.4 us with one
// a row, 9.8 with 2, 10.0 with 4, 11.7 with 8; one row of 50257 fp32: 12.1 with one, 10.0 with 2, 9.0 with 4, 8.9 with 8.)
int cluster_of(int rows, int vocab) {
    const int sms = sm_count() > 0 ? sm_count() : 148;
    int c = 1;
    while (c < MAX_CLUSTER && (long long)rows * c * 2 < sms && vocab / (2 * c) >= 256 * PER_THREAD) c *= 2;
    return c;
}

template <bool H16, bool TOP, int T>
int launch(const LogprobParams &p, int cluster, cudaStream_t st) {
    static DeviceOnce configured;
    constexpr int SMEM = sizeof(Smem<T>);
    if (!configured.done()) {
        int rc = cuda_check(cudaFuncSetAttribute(logprobs_kernel<H16, TOP, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM),
                            "token logprobs: shared memory opt-in");
        if (rc) return rc;
        configured.set();
    }
    cudaLaunchConfig_t cfg = {};
    // one row after the other in each CTA of all that run at once
    const int side = Shape<T>::CTAS * (sm_count() > 0 ? sm_count() : 148);
    cfg.gridDim = dim3(cluster > 1 || p.rows < side ? p.rows * cluster : side);
    cfg.blockDim = dim3(T);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cuda_check(cudaLaunchKernelEx(&cfg, logprobs_kernel<H16, TOP, T>, p, cluster), "token logprobs: launch");
}

template <bool H16, bool TOP>
int launch_rows(const LogprobParams &p, cudaStream_t st) {
    const int cluster = cluster_of(p.rows, p.vocab), sms = sm_count() > 0 ? sm_count() : 148;
    // many rows: see Shape
    return p.rows >= 8 * sms && p.top <= Shape<128>::TOP ? launch<H16, TOP, 128>(p, cluster, st) : launch<H16, TOP, 256>(p, cluster, st);
}

}  // namespace

}  // namespace kr

extern "C" int kraken_op_token_logprobs(const kraken_logprobs_args *a, uint32_t *d_status, void *stream) {
    using namespace kr;
    if (!a || a->rows < 0) return KRAKEN_EINVAL;
    if (a->rows == 0) return KRAKEN_OK;
    if (!a->logits || a->vocab < 1 || a->row_stride < 0 || a->dtype < 0 || a->dtype > 1 || a->top < 0 || a->top > a->vocab ||
        !(a->scale > 0.f) || !isfinite(a->scale * LOG2E) || (a->logprob && !a->targets) || (a->top > 0 && !a->top_ids && !a->top_logprobs))
        return KRAKEN_EINVAL;
    if (a->top > LP_MAX_TOP || a->vocab > 1 << 30) return KRAKEN_EUNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(a->logits) & (a->dtype ? 1 : 3)) return KRAKEN_EUNSUPPORTED;
    LogprobParams p;
    p.logits = a->logits;
    p.row_stride = a->row_stride;
    p.targets = a->targets;
    p.logprob = a->logprob;
    p.entropy = a->entropy;
    p.lse = a->lse;
    p.top_ids = a->top_ids;
    p.top_logprobs = a->top_logprobs;
    p.rows = a->rows;
    p.vocab = a->vocab;
    p.top = a->top;
    p.scale = a->scale;
    p.status = d_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (a->dtype) return a->top ? launch_rows<true, true>(p, st) : launch_rows<true, false>(p, st);
    return a->top ? launch_rows<false, true>(p, st) : launch_rows<false, false>(p, st);
}
