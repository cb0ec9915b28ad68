// Attention of chunks of new tokens over a key/value cache in pages, on the sm_100a tensor cores (tcgen05 + TMEM).
//
//   x_ij = scale q_i.k_j  [cap tanh(x/cap)]  [+ slope (j - p_i)]  for  p_i - window < j <= p_i,   p_i = n_keys - tokens + i
//   out_i = sum_j softmax(x_i)_j v_j,   lse_i = log sum_j e^x_ij
//
// A work unit is two tiles of query rows of one (chunk, key/value head) against the keys that any of them sees.  A tile has up to
// 128 rows: 128 / rep consecutive tokens times the rep = n_head / n_kv_head query heads that share the keys, so a few tokens of
// grouped heads fill it as well as many tokens of single ones, and keys and values are fetched once for all of them.
//
//   warp 0      cuts the work, hands the units out (a ring of two in shared memory), looks pages up and starts the copies:
//               both Q tiles, then per step a stage of V_j and K_{j+1} (two stages)
//   warp 1      issues the products, per key tile j and query tile w:  S_w = Q_w K_j^T,  O_w (+)= P_w V_j
//               (P from tensor memory, where it takes the place of S for head dims above 64)
//   warps 2-3   see to the values of masked tiles; copy what the copy engine cannot (LANES)
//   warps 4-11  softmax: one thread per query row, warps 4-7 tile 0, warps 8-11 tile 1
//
// The maximum in use is only raised when a row's maximum gets past it by more than 8 in the exponent of 2 (numerator and
// denominator carry the same factor).  P is rounded to 16 bits for the second product, like the output it is summed to; the sum
// of the weights is fp32 of the unrounded ones.
//
// Hidden keys have weight 0, and 0 times a NaN or an infinity is one: in tiles that some row does not see all of ("masked", at
// both ends of a unit's keys only), values that no row sees are zeroed in shared memory before the product, and values that are
// not finite are zeroed and noted; rows that do see them get NaN in these elements at the end.
//
// The tiles of a call are one line that is cut into equal parts, one for each CTA (one per SM).  A unit cut apart leaves its parts
// (maximum, sum, output) in the workspace and a second kernel joins them.
//
// What bounds it.  Products at the tensor cores' rate would be 2 x 512 cycles a query tile and key tile with head dims of 128;
// a row's 128 exponentials take as long in the special-function units.  A key tile takes 3.7 to 4.2 thousand cycles with both query
// tiles at work, each of which goes through scores, weights and product one after the other while the other one does the same; with
// a cap or slopes (GENERAL) 7 to 8 thousand, as every score goes back to tensor memory on the way.  A
// unit costs some 9 thousand cycles besides (its first keys and scores, its last product, the way out), a call 12 thousand (the
// lengths read and the work cut, the first copies) and the second kernel.  Measured on a B200, a graph of calls:
//   2048 tokens after 32768, 32 on 8 heads of 128:   1140 us, 1.0 PFLOP/s (floor at 1.66: 682); 1320 us, 0.86 PFLOP/s, on a hot card
//   four prompts of 1129 to 2048, 16 heads of 128:   104 us (34; tensor cores busy 27 % of the time, issue slots as much)
//   24 sequences, three in four with a single token, up to 4000 keys, 16 on 4 heads of 64, capped:   148 us (17); 205 with scores five
//   times as large, where one in 400 is beyond half of the cap and nearly every warp has one
//   five tokens after 1500, 32 on 8 heads of 128:    19 us (1), the start and two kernels; the decode step with a row for each: 15
// With copies by lanes (pages of 100 slots) the same take 2010, 161, 181 and 26 us: 64 threads copy what a few requests do otherwise.
// The size of the code counts: with a tile's 128 scores in registers, everything written out for them, instructions came from
// beyond the first cache all the time.  So the scores are read from tensor memory twice, 32 at a time (four prompts 111 -> 104),
// masks are bits, and there is one form of a step (one for tiles that every row sees whole and one for the others: 137).
#include <float.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "paged.cuh"

namespace kr {

namespace {

constexpr int TQ = 128;         // rows of a query tile
constexpr int TK = 128;         // keys of a tile
constexpr int THREADS = 384, AUX = 64;
constexpr int SIDE = 3;         // masked tiles at either end of a unit's keys: its tokens' limits span at most 255 keys
// What beginning and finishing a unit costs, in tiles (1: the mixed batch 150 us in place of 146; 3: four prompts 102 in place of 104,
// but windows with slopes 55 in place of 50), and a CTA's places at least (3: five drafted tokens 20.4 us in place of 19.3)
constexpr int BEGIN = 2, MIN_PART = 2;
// Where the sums of a head's places end: more than the places of chunks that lie behind one another can be (the host sees to that), and
// two of them still fit 32 bits.  Chunks may lie on one another as often as q_start goes back, and a sum that wrapped round would send
// the search for a CTA's share out of the list of chunks.
constexpr uint32_t MOST_PLACES = 0x7FFFFFFFu;
// A weight is 2^(score - m); the first tile's largest is 2^HEADROOM, and m is raised when one gets past 2^(HEADROOM + RAISE).  Half numbers end at 2^16 and 2^-24: with 7, 10^5 weights of 2^-25 of the largest still count.
constexpr float HEADROOM = KRAKEN_F16 ? 7.f : 0.f;
constexpr float RAISE = 8.f;

// m: the score that has the weight 2^HEADROOM; l: the sum of the weights
__device__ __forceinline__ float lse_of_weights(float m, float l) { return l == 0.f ? -INFINITY : m + (log2f(l) - HEADROOM) * LN2; }

// s -> cap tanh(scale s / cap) by way of u = 2 log2(e) scale s / cap, which is of the size of the result's exponent whatever the two
// factors are.  Up to `border` an odd polynomial in u, fitted to tanh up to 1/2 (to 1.4e-8 of it, 1.2e-7 with the roundings); beyond,
// cap (1 - 2 / (1 + 2^u)), off by up to 2e-7 cap.  (With coefficients for s itself, powers of scale / cap had to fit 32 bits.)
struct Cap {
    float by, border, cap, c[5];
    Cap() = default;
    Cap(double scale, double cap_) : cap(static_cast<float>(cap_)) {
        constexpr double FIT[5] = {1., -0.33333069, 0.13324779, -0.052986074, 0.017135004}, TO_T = 0.5 * 0.693147180559945309417;
        const double ideal = scale / cap_ / TO_T;
        // A factor so small that 32 bits hold it with less than 22 of their own: another one, that leaves u below the ideal's border for
        // every s there is
        const bool tiny = fabs(ideal) < 0.25 * FLT_MIN;
        by = static_cast<float>(tiny ? copysign(FLT_MIN, ideal) : ideal);
        border = tiny ? FLT_MAX : LOG2E;
        const double t = tiny ? fabs(ideal) / FLT_MIN * TO_T : TO_T;   // of 1 in u
        for (int i = 0; i < 5; ++i) c[i] = static_cast<float>(FIT[i] * (tiny ? fabs(scale) / FLT_MIN : cap_ * TO_T) * pow(t, 2 * i));
    }
};

struct ChunkParams {
    PagedView c;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    const int *chunk_seq, *q_start, *n_keys;
    const float *slopes;
    long long q_row, q_head, out_row, out_head, lse_row;
    float scale, cap;
    Cap capped;   // where there is a cap
    int chunks, rows, n_head, rep, window, head_dim;
    int heads;        // query heads of a tile
    int head_tiles;   // tiles that the heads of a key/value head make
    int tokens;       // tokens of a tile
    uint32_t *status;
    uint8_t *workspace;
    Divisor by_page, by_heads;
    int box;          // keys of a copy
};

// Scores that are more than the product times a positive factor (the instances of the kernel with GENERAL)
__host__ __device__ inline bool is_general(const ChunkParams &p) { return p.cap > 0.f || p.slopes || !(p.scale > 0.f); }

// The n lowest bits (none for n <= 0, all for n >= 32)
__device__ __forceinline__ uint32_t below(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u); }

// Whether a 16-bit number, or one of a pair, is infinite or NaN
constexpr uint32_t EXPONENT = KRAKEN_F16 ? 0x7C00u : 0x7F80u;
__device__ __forceinline__ bool odd_h16(uint32_t pair) {
    return (pair & EXPONENT) == EXPONENT || (pair & (EXPONENT << 16)) == EXPONENT << 16;
}

__device__ __forceinline__ uint64_t tanh_poly(uint64_t u, const Cap &k) {
    const uint64_t y = mul2(u, u);
    return mul2(u, fma2(y, fma2(y, fma2(y, fma2(y, splat2(k.c[4]), splat2(k.c[3])), splat2(k.c[2])), splat2(k.c[1])), splat2(k.c[0])));
}
__device__ __forceinline__ void tanh_near(float (&s)[32], const Cap &k) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) upk2(tanh_poly(mul2(pk2(s[i], s[i + 1]), splat2(k.by)), k), s[i], s[i + 1]);
}
// The same where some may be beyond the border (to the last bit as above for one that is not)
__device__ __forceinline__ void tanh_any(float (&s)[32], const Cap &k) {
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        const uint64_t u = mul2(pk2(s[i], s[i + 1]), splat2(k.by));
        float u0, u1;
        upk2(u, u0, u1);
        upk2(tanh_poly(u, k), s[i], s[i + 1]);
        const float far0 = fmaf(-2.f, rcp_approx(1.f + ex2_approx(u0)) * k.cap, k.cap), far1 = fmaf(-2.f, rcp_approx(1.f + ex2_approx(u1)) * k.cap, k.cap);
        s[i] = fabsf(u0) <= k.border ? s[i] : far0;
        s[i + 1] = fabsf(u1) <= k.border ? s[i + 1] : far1;
    }
}

// What a chunk brings
struct Chunk {
    int row0, tokens, seq, pos0;   // first row; tokens (0: nothing to do); position of the first token (negative: it sees nothing)
};

__device__ __forceinline__ Chunk chunk_of(const ChunkParams &p, int c, bool &bad) {
    Chunk k;
    k.row0 = p.q_start[c];
    const int end = p.q_start[c + 1], n = p.n_keys[c];
    k.seq = p.chunk_seq ? p.chunk_seq[c] : c;
    k.tokens = 0;
    k.pos0 = 0;
    if (k.seq < 0 || (k.row0 == end && end >= 0 && end <= p.rows)) return k;
    if (k.row0 < 0 || end < k.row0 || end > p.rows || k.seq >= p.c.n_seqs || n < 0 || n > (long long)p.c.max_pages * p.c.page_size) {
        bad = true;
        return k;
    }
    k.tokens = end - k.row0;
    k.pos0 = n - k.tokens;
    return k;
}

// First key that a query at position `pos` sees (pos may be negative, and then sees none)
__device__ __forceinline__ int first_seen(const ChunkParams &p, int pos) {
    return p.window > 0 && pos >= p.window ? pos - p.window + 1 : 0;
}

// Keys that tokens [t0, t1) of a chunk see: [lo, hi), key tiles [j0, j1)
struct Span {
    int lo, hi, j0, j1;
};

__device__ __forceinline__ Span span_of(const ChunkParams &p, const Chunk &k, int t0, int t1) {
    Span s;
    s.hi = max(0, k.pos0 + t1);
    s.lo = first_seen(p, k.pos0 + t0);
    if (s.hi <= s.lo) s.hi = s.lo = 0;
    s.j0 = s.lo / TK;
    s.j1 = (s.hi + TK - 1) / TK;
    return s;
}

// sum over i < n of floor((a i + b) / 128), a <= 256, n < 2^22: the lattice points under a line, by Euclid's steps
__device__ __forceinline__ long long floors(unsigned n, unsigned a, unsigned b) {
    unsigned m = TK;
    long long sum = 0;
    while (n > 0) {
        sum += (long long)(n - 1) * n / 2 * (a / m);
        a %= m;
        sum += (long long)n * (b / m);
        b %= m;
        const unsigned y = a * n + b;
        if (y < m) break;
        n = y / m;
        b = y % m;
        const unsigned t = m;
        m = a;
        a = t;
    }
    return sum;
}

// Places of all pairs of query tiles of a chunk (of one head): ceil(hi / 128) - floor(lo / 128) + BEGIN summed, of which all but the
// last hi and all lo lie on lines
__device__ __forceinline__ int chunk_places(const ChunkParams &p, const Chunk &k) {
    const int S = 2 * p.tokens, n = (k.tokens + S - 1) / S;
    if (n <= 2) {
        int sum = 0;
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const Span s = span_of(p, k, i * S, min(k.tokens, (i + 1) * S));
            sum += s.j1 - s.j0 + BEGIN;
        }
        return sum;
    }
    long long sum = (long long)n * BEGIN;
    // pairs i < n - 1 end at pos0 + (i + 1) S; from i0 on that is above 0
    const int i0 = k.pos0 >= 0 ? 0 : min(n - 1, -k.pos0 / S);
    int from[2] = {i0, n};
    unsigned at[2] = {(unsigned)(k.pos0 + (i0 + 1) * S + TK - 1), 0u};
    if (p.window > 0) {
        // pairs begin at pos0 + i S + 1 - window; from i1 on that is at least 0
        const long long first = (long long)k.pos0 + 1 - p.window, i1 = first >= 0 ? 0 : (S - 1 - first) / S;
        from[1] = (int)min((long long)n, i1);
        at[1] = (unsigned)(first + i1 * S);
    }
#pragma unroll 1
    for (int e = 0; e < 2; ++e) {
        const int many = (e ? n : n - 1) - (e ? from[1] : from[0]);
        const long long part = many > 0 ? floors(many, S, e ? at[1] : at[0]) : 0;
        sum += e ? -part : part;
    }
    return static_cast<int>(sum + (max(0, k.pos0 + k.tokens) + TK - 1) / TK);   // (all chunks' together are below 2^31)
}

struct Item {
    int row0, tokens, pos0, seq, kvh, h0, heads;
    int t0;              // first token of the pair of query tiles
    int lo, hi;          // keys that some row of the unit sees
    int lo_max, hi_min;  // a tile within [lo_max, hi_min) is seen whole by every row
    int j0, j1;          // key tiles of this CTA's part
    int a0[2], a1[2];    // of these, those of query tile w
    int u0;              // first key tile of the unit
    int r0;              // first masked tile at the far end
    int part;            // -1: the whole unit; 1: its beginning; 0: what follows
    int tile0;           // key tiles of this CTA before
    int last;            // no more items
    __device__ __forceinline__ bool masked(int j) const { return j * TK < lo_max || (j + 1) * TK > hi_min; }
    __device__ __forceinline__ int place(int j) const { return (j + 1) * TK > hi_min ? SIDE + j - r0 : j - u0; }
};

// A unit in parts: who has them and what it is
struct Joint {
    int last_cta;   // -1: nothing to join
    int row0, tokens, t0, h0, heads;
    int pad[2];
};

// A place between two tiles on the line of all tiles
struct Cut {
    int u, c, pair, t;   // unit head (all: the end), chunk, pair of query tiles, tiles of the unit before it
};

template <int HD>
struct Cfg {
    static constexpr int HALVES = HD / 64;
    static constexpr int TILE_BYTES = TK * 128;            // 128 rows x 64 elements
    static constexpr int Q_BYTES = HALVES * TILE_BYTES, KV_BYTES = HALVES * TILE_BYTES;
    static constexpr bool SEPARATE_P = HD <= 64;           // tensor memory has room for P beside S
    static constexpr int P_COL0 = SEPARATE_P ? 256 : 0, P_STRIDE = SEPARATE_P ? TK / 2 : TK;
    static constexpr int O_COL0 = SEPARATE_P ? 384 : 256, O_STRIDE = SEPARATE_P ? HD : TK;
    static constexpr int TMEM_COLS = 512;
    static constexpr int WORDS = HD / 32;
    static constexpr int PART_FLOATS = 2 * TQ * (HD + 2);  // [w][HD / 4][128 rows][4] output, [w][m, l][128 rows]
};

template <int HD>
struct Smem {
    uint8_t q[2][Cfg<HD>::Q_BYTES];
    struct {
        uint8_t v[Cfg<HD>::KV_BYTES], k[Cfg<HD>::KV_BYTES];
    } ring[2];
    uint32_t odd[2][2 * SIDE][TK][Cfg<HD>::WORDS];   // bits of the elements that are not finite, of the item's masked tiles
    long long at[4][TK];                             // LANES: where a key's row of its page begins, -1: nowhere
    Item items[2];
    uint32_t odd_tiles[2][2];                        // which of them have any: [item slot][aux warp]
    uint32_t visible[4][4], missing[4][2];           // of a tile's keys, those whose page exists; whether any does not
    uint64_t q_full, q_empty, b_full[2], b_empty[2], s_full[2], p_ready[2], pv_done[2], s_free[2], p_free[2], v_full[2], v_ready[2], item_full[2],
        item_empty[2], at_ready;
    uint32_t upto[THREADS], sum[THREADS / 32];
    Chunk cut_chunk[2];
    Cut cut[2];
    int end_last;
    uint32_t tmem, gave_up;
};

// The products with operand descriptors as a low and a high word: a step along the operand adds to the low one only
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a_lo, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool add) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        ".reg .b64 a, b;\n"
        "setp.ne.b32 p, %5, 0;\n"
        "mov.b64 a, {%1, %3};\n"
        "mov.b64 b, {%2, %3};\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %4, p;\n"
        "}\n" ::"r"(d), "r"(a_lo), "r"(b_lo), "r"(hi), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b_lo, uint32_t hi, uint32_t idesc, bool add) {
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        ".reg .b64 b;\n"
        "setp.ne.b32 p, %5, 0;\n"
        "mov.b64 b, {%2, %3};\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %4, p;\n"
        "}\n" ::"r"(d), "r"(a), "r"(b_lo), "r"(hi), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}

template <int HD, bool GENERAL, bool LANES>
__global__ void __launch_bounds__(THREADS, 1)
paged_chunk_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
                   const ChunkParams p) {
    using C = Cfg<HD>;
    extern __shared__ uint8_t smem_raw[];
    Smem<HD> &sm = *reinterpret_cast<Smem<HD> *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    volatile uint32_t *gave_up = &sm.gave_up;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(&sm.q_full, LANES ? AUX : 1);
        mbar_init(&sm.q_empty, 1);
        mbar_init(&sm.at_ready, 2);
        for (int s = 0; s < 2; ++s) {
            mbar_init(&sm.b_full[s], LANES ? AUX : 1);
            mbar_init(&sm.b_empty[s], 1);
            mbar_init(&sm.s_full[s], 1);
            mbar_init(&sm.p_ready[s], 4);
            mbar_init(&sm.pv_done[s], 1);
            mbar_init(&sm.s_free[s], 4);
            mbar_init(&sm.p_free[s], 1);
            mbar_init(&sm.v_full[s], 1);
            mbar_init(&sm.v_ready[s], 2);
            mbar_init(&sm.item_full[s], 1);
            mbar_init(&sm.item_empty[s], 11);   // the issuer, two aux warps, eight softmax warps
        }
        sm.gave_up = 0;
        fence_barrier_init();
        if (!LANES) {
            prefetch_tensormap(&tm_q);
            prefetch_tensormap(&tm_k);
            prefetch_tensormap(&tm_v);
        }
    }
    if (warp == 1) {
        tmem_alloc(&sm.tmem, C::TMEM_COLS);
        tmem_relinquish();
    }
    pdl_wait();
    const int units = p.c.n_kv_head * p.head_tiles, S = 2 * p.tokens;
    Joint *joints = reinterpret_cast<Joint *>(p.workspace);
    float *slots = reinterpret_cast<float *>(p.workspace + sizeof(Joint) * gridDim.x);
    if (threadIdx.x == 0) joints[blockIdx.x].last_cta = -1;

    // The line: head by head, of each the chunks in order, of each its pairs of query tiles, of each BEGIN places and then one for every
    // key tile.  CTA i of n has the places from x_i = floor(total / n) i + min(i, total mod n) on.
    bool bad = false;
    uint32_t per_head;
    const int run = (p.chunks + THREADS - 1) / THREADS;   // chunks that a thread adds up
    {
        const int c_lo = min(p.chunks, (int)threadIdx.x * run), c_hi = min(p.chunks, c_lo + run);
        uint32_t upto = 0;
#pragma unroll 1
        for (int c = c_lo; c < c_hi; ++c) {
            const Chunk k = chunk_of(p, c, bad);
            if (k.tokens > 0) upto = min(upto + chunk_places(p, k), MOST_PLACES);
        }
        if (bad && blockIdx.x == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, off);
            if (lane >= off) upto = min(upto + v, MOST_PLACES);
        }
        if (lane == 31) sm.sum[warp] = upto;
        sm.upto[threadIdx.x] = upto;   // of the warp
        __syncthreads();
    }
    if (warp < 2) {   // where this CTA's share begins (warp 0) and ends (warp 1)
        uint32_t warps = lane < THREADS / 32 ? sm.sum[lane] : 0u;
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, warps, off);
            if (lane >= off) warps = min(warps + v, MOST_PLACES);
        }
        per_head = __shfl_sync(0xFFFFFFFFu, warps, THREADS / 32 - 1);
        if (per_head == MOST_PLACES) {   // (only where chunks lie on one another: nothing is done)
            per_head = 0;
            if (blockIdx.x == 0 && threadIdx.x == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
        }
        const unsigned long long total = (unsigned long long)per_head * units;
        const int n_cta = static_cast<int>(max(1ull, min((unsigned long long)gridDim.x, total / MIN_PART)));
        const unsigned long long share = total >> 32 ? total / n_cta : (uint32_t)total / (uint32_t)n_cta, rest = total - share * n_cta;
        auto place = [&](int cta) { return share * cta + min((unsigned long long)cta, rest); };
        // a cut so near to a unit's end goes there: joining costs more than being late
        const int snap = 2 + static_cast<int>(min(share, 1ull << 20)) / 16;
        auto snapped = [&](int t, int tiles) { return t < snap ? 0 : (tiles - t < snap ? tiles : t); };
        Cut cut = {units, 0, 0, 0};
        int end_last = -1;   // the last CTA that has a part of the unit at the second cut
        const int cta = blockIdx.x + warp;
        if (cta < n_cta && per_head > 0) {
            const unsigned long long x = place(cta);
            cut.u = x >> 32 ? static_cast<int>(x / per_head) : static_cast<int>((uint32_t)x / per_head);
            uint32_t left = static_cast<uint32_t>(x - (unsigned long long)cut.u * per_head);
            // the warp, the thread and the chunk
            const int w = __ffs(__ballot_sync(0xFFFFFFFFu, warps > left)) - 1;
            left -= w ? __shfl_sync(0xFFFFFFFFu, warps, w - 1) : 0u;
            const uint32_t upto = sm.upto[w * 32 + lane];
            const int t = __ffs(__ballot_sync(0xFFFFFFFFu, upto > left)) - 1;
            left -= t ? __shfl_sync(0xFFFFFFFFu, upto, t - 1) : 0u;
            Chunk k;
#pragma unroll 1
            for (cut.c = (w * 32 + t) * run;; ++cut.c) {
                k = chunk_of(p, cut.c, bad);
                if (run == 1) break;
                const uint32_t here = k.tokens > 0 ? chunk_places(p, k) : 0;
                if (left < here) break;
                left -= here;
            }
#pragma unroll 1
            for (int i0 = 0;; i0 += 32) {   // 32 pairs at a time
                const int i = i0 + lane;
                int tiles = 0;
                uint32_t up = 0;
                if (i * S < k.tokens) {
                    const Span s = span_of(p, k, i * S, min(k.tokens, (i + 1) * S));
                    tiles = s.j1 - s.j0;
                    up = tiles + BEGIN;
                }
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, up, off);
                    if (lane >= off) up += v;
                }
                const uint32_t found = __ballot_sync(0xFFFFFFFFu, left < up);
                if (found) {
                    const int l = __ffs(found) - 1;
                    tiles = __shfl_sync(0xFFFFFFFFu, tiles, l);
                    const int o = left - (__shfl_sync(0xFFFFFFFFu, up, l) - tiles - BEGIN);
                    cut.pair = i0 + l;
                    cut.t = snapped(max(0, o - BEGIN), tiles);
                    if (warp == 1 && cut.t > 0 && cut.t < tiles) {
                        // of the cuts after this one, those that lie in the same unit and stay there
                        const unsigned long long x0 = x - o;
#pragma unroll 1
                        for (int c0 = cta; c0 < n_cta; c0 += 32) {
                            const unsigned long long at = place(c0 + lane) - x0;
                            const int t = at < tiles + BEGIN ? snapped(max(0, static_cast<int>(at) - BEGIN), tiles) : tiles;
                            const uint32_t in = __ballot_sync(0xFFFFFFFFu, c0 + lane < n_cta && t < tiles);
                            if (in) end_last = c0 + 31 - __clz(in);
                            if (in != 0xFFFFFFFFu) break;
                        }
                    }
                    break;
                }
                left -= __shfl_sync(0xFFFFFFFFu, up, 31);
                if ((i0 + 32) * S >= k.tokens) break;   // (the lengths changed under the kernel)
            }
            if (lane == 0) sm.cut_chunk[warp] = k;
        }
        if (lane == 0) {
            sm.cut[warp] = cut;
            if (warp == 1) sm.end_last = end_last;
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    pdl_trigger();
    const uint32_t tmem_base = sm.tmem;

    if (warp < 4) {
        if (warp == 0) {
            // ------------------------------------------------------------------ units and copies
            bool ok = true;
            uint32_t n_items = 0, loads = 0, bundles = 0;
            int tile0 = 0;
            bool bad_page = false;
            auto publish = [&](const Item &it) {
                const int slot = n_items & 1;
                ok = mbar_wait(&sm.item_empty[slot], ((n_items >> 1) & 1u) ^ 1u, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) return;
                if (lane == 0) {
                    sm.items[slot] = it;
                    sm.odd_tiles[slot][0] = sm.odd_tiles[slot][1] = 0;
                    mbar_arrive(&sm.item_full[slot]);
                }
                ++n_items;
            };
            Item it;
            memset(&it, 0, sizeof(it));
            Cut at = sm.cut[0];
            const Cut end = sm.cut[1];
            Chunk k = sm.cut_chunk[0];
            const int nbox = TK / p.box;
            while (ok && at.u < units) {
                const bool at_end = at.u == end.u && at.c == end.c && at.pair == end.pair;
                if (at_end && end.t == 0) break;
                const int pair = at.pair, t = at.t, u = at.u;
                const int t0 = pair * S, t1 = min(k.tokens, t0 + S);
                const Span all = span_of(p, k, t0, t1);
                const int tiles = all.j1 - all.j0, te = at_end ? end.t : tiles;
                if (te > t || tiles == 0) {
                    it.row0 = k.row0;
                    it.tokens = k.tokens;
                    it.pos0 = k.pos0;
                    it.seq = k.seq;
                    it.kvh = u / p.head_tiles;
                    const int first = u % p.head_tiles * p.heads;
                    it.h0 = it.kvh * p.rep + first;
                    it.heads = min(p.heads, p.rep - first);
                    it.t0 = t0;
                    it.lo = all.lo;
                    it.hi = all.hi;
                    it.lo_max = first_seen(p, k.pos0 + t1 - 1);
                    it.hi_min = max(0, k.pos0 + t0 + 1);
                    it.u0 = all.j0;
                    it.r0 = it.hi_min / TK;
                    it.j0 = all.j0 + t;
                    it.j1 = all.j0 + te;
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int b = min(t1, t0 + w * p.tokens), e = min(t1, b + p.tokens);
                        it.a0[w] = it.a1[w] = it.j0;
                        if (e > b) {
                            const Span s = span_of(p, k, b, e);
                            it.a0[w] = max(it.j0, s.j0);
                            it.a1[w] = max(it.a0[w], min(it.j1, s.j1));
                        }
                    }
                    it.part = te - t == tiles ? -1 : (t == 0 ? 1 : 0);
                    it.tile0 = tile0;
                    if (it.part == 1 && lane == 0) {
                        Joint j;
                        j.last_cta = sm.end_last;
                        j.row0 = k.row0;
                        j.tokens = k.tokens;
                        j.t0 = t0;
                        j.h0 = it.h0;
                        j.heads = it.heads;
                        j.pad[0] = j.pad[1] = 0;
                        joints[blockIdx.x] = j;
                    }
                    publish(it);
                    if (!LANES && ok && it.j0 < it.j1) {
                        // lane i looks up box i of a tile, one step before its copies
                        const int *table = p.c.table + it.seq * p.c.table_stride;
                        int page = 0, slot = 0;
                        auto look_up = [&](int j) {
                            const int key = j * TK + lane * p.box, n = p.by_page.quotient(key);
                            slot = key - n * p.c.page_size;
                            page = p.c.n_pages;   // (nothing there: zeros)
                            if (lane < nbox && j < it.j1 && key < it.hi && key + p.box > it.lo) page = table[n];
                        };
                        auto check = [&](int j) {   // pages that do not exist: their keys are not visible
                            const bool missing = page < 0 || page > p.c.n_pages || (page == p.c.n_pages && lane < nbox && j < it.j1 &&
                                                                                   j * TK + lane * p.box < it.hi && j * TK + (lane + 1) * p.box > it.lo);
                            if (missing) page = p.c.n_pages;
                            const uint32_t boxes = __ballot_sync(0xFFFFFFFFu, missing);
                            const int mark = (tile0 + j - it.j0) & 3;
                            if (boxes) {
                                bad_page = true;
                                if (lane < 4) {
                                    uint32_t bits = 0;
                                    for (int i = 0; i < 32; ++i)
                                        if (!(boxes >> ((lane * 32 + i) / p.box) & 1)) bits |= 1u << i;
                                    sm.visible[mark][lane] = bits;
                                }
                            }
                            if (lane == 0) {
                                sm.missing[mark][0] = boxes != 0;
                                sm.missing[mark][1] = 0;
                            }
                            __syncwarp();
                        };
                        look_up(it.j0);
                        ok = mbar_wait(&sm.q_empty, (loads & 1u) ^ 1u, gave_up);
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (!ok) break;
                        ++loads;
                        if (lane == 0) {
                            const bool use[2] = {it.a0[0] < it.a1[0], it.a0[1] < it.a1[1]};
                            mbar_expect_tx(&sm.q_full, (use[0] + use[1]) * C::HALVES * 128 * p.heads * p.tokens);
#pragma unroll
                            for (int w = 0; w < 2; ++w)
                                if (use[w])
#pragma unroll
                                    for (int hf = 0; hf < C::HALVES; ++hf)
                                        tma_load_4d(sm.q[w] + hf * C::TILE_BYTES, &tm_q, &sm.q_full, hf * 64, it.h0,
                                                    k.row0 + t0 + w * p.tokens, 0);
                        }
                        int v_page = p.c.n_pages, v_slot = 0;
                        for (int j = it.j0 - 1; j < it.j1; ++j, ++bundles) {
                            const bool has_v = j >= it.j0, has_k = j + 1 < it.j1;
                            if (has_k) check(j + 1);
                            const int k_page = page, k_slot = slot;
                            look_up(j + 2);
                            const int st = bundles & 1;
                            ok = mbar_wait(&sm.b_empty[st], ((bundles >> 1) & 1u) ^ 1u, gave_up);
                            ok = __all_sync(0xFFFFFFFFu, ok);
                            if (!ok) break;
                            // (values of a masked tile go by way of the aux warps)
                            const bool mend_v = has_v && it.masked(j);
                            uint64_t *v_bar = mend_v ? &sm.v_full[st] : &sm.b_full[st];
                            if (lane == 0) {
                                mbar_expect_tx(&sm.b_full[st], ((has_v && !mend_v) + has_k) * C::KV_BYTES);
                                if (mend_v) mbar_expect_tx(&sm.v_full[st], C::KV_BYTES);
                            }
                            __syncwarp();
                            if (lane < nbox) {
#pragma unroll
                                for (int hf = 0; hf < C::HALVES; ++hf) {
                                    const int to = hf * C::TILE_BYTES + lane * p.box * 128;
                                    if (has_k) tma_load_4d(sm.ring[st].k + to, &tm_k, &sm.b_full[st], hf * 64, k_slot, it.kvh, k_page);
                                    if (has_v) tma_load_4d(sm.ring[st].v + to, &tm_v, v_bar, hf * 64, v_slot, it.kvh, v_page);
                                }
                            }
                            __syncwarp();
                            v_page = k_page;
                            v_slot = k_slot;
                        }
                    }
                    tile0 += it.j1 - it.j0;
                }
                if (at_end) break;
                at.t = 0;
                if (++at.pair * S >= k.tokens) {   // the next chunk with tokens, or the first of the next head
                    at.pair = 0;
                    k.tokens = 0;
#pragma unroll 1
                    for (int c0 = at.c + 1; k.tokens == 0; c0 += 32) {
                        if (c0 >= p.chunks) {
                            if (++at.u == units) break;
                            c0 = 0;
                        }
                        Chunk mine;
                        mine.row0 = mine.tokens = mine.seq = mine.pos0 = 0;
                        if (c0 + lane < p.chunks) mine = chunk_of(p, c0 + lane, bad);
                        const uint32_t any = __ballot_sync(0xFFFFFFFFu, mine.tokens > 0);
                        const int l = any ? __ffs(any) - 1 : 0;
                        if (any) at.c = c0 + l;
                        k.row0 = __shfl_sync(0xFFFFFFFFu, mine.row0, l);
                        k.tokens = __shfl_sync(0xFFFFFFFFu, mine.tokens, l);
                        k.seq = __shfl_sync(0xFFFFFFFFu, mine.seq, l);
                        k.pos0 = __shfl_sync(0xFFFFFFFFu, mine.pos0, l);
                    }
                }
            }
            if (ok) {
                it.last = 1;
                publish(it);
            }
            if (bad_page && lane == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
        } else if (warp == 1) {
            // ------------------------------------------------------------------ products
            if (lane == 0) {
                // head dims below HD: K is zero beyond head_dim
                const int qk_steps = (p.head_dim + 15) / 16;
                constexpr uint32_t idesc_qk = umma_idesc_h16(TQ, TK);
                const uint32_t idesc_pv = umma_idesc_h16(TQ, qk_steps * 16) | (1u << 16);   // V is MN-major
                auto issue_qk = [&](int w, int st) {
                    const uint64_t qd = umma_desc_sw128_kmajor(smem_u32(sm.q[w])), kd = umma_desc_sw128_kmajor(smem_u32(sm.ring[st].k));
                    const uint32_t q_lo = static_cast<uint32_t>(qd), k_lo = static_cast<uint32_t>(kd), hi = static_cast<uint32_t>(kd >> 32);
#pragma unroll
                    for (int ks = 0; ks < HD / 16; ++ks) {
                        if (ks >= qk_steps) break;
                        const uint32_t off = ((ks >> 2) * C::TILE_BYTES + (ks & 3) * 32) >> 4;
                        mma_ss(tmem_base + w * TK, q_lo + off, k_lo + off, hi, idesc_qk, ks != 0);
                    }
                    umma_commit(&sm.s_full[w]);
                };
                auto issue_pv = [&](int w, int st, bool first, bool last) {
                    const uint64_t vd = umma_desc_sw128_mnmajor(smem_u32(sm.ring[st].v), C::TILE_BYTES);
                    const uint32_t v_lo = static_cast<uint32_t>(vd), hi = static_cast<uint32_t>(vd >> 32);
                    const uint32_t p_tmem = tmem_base + C::P_COL0 + w * C::P_STRIDE, o_tmem = tmem_base + C::O_COL0 + w * C::O_STRIDE;
#pragma unroll
                    for (int ks = 0; ks < TK / 16; ++ks) mma_ts(o_tmem, p_tmem + ks * 8, v_lo + (ks * 2048 >> 4), hi, idesc_pv, !first || ks > 0);
                    if (last) umma_commit(&sm.pv_done[w]);
                    else if (C::SEPARATE_P) umma_commit(&sm.p_free[w]);
                };
                bool ok = true;
                uint32_t n_items = 0, loads = 0, bundles = 0, tile_cnt[2] = {0, 0}, fixes[2] = {0, 0};
                while (ok) {
                    const int slot = n_items & 1;
                    if (!(ok = mbar_wait(&sm.item_full[slot], (n_items >> 1) & 1u, gave_up))) break;
                    ++n_items;
                    const Item it = sm.items[slot];
                    mbar_arrive(&sm.item_empty[slot]);
                    if (it.last) break;
                    if (it.j0 >= it.j1) continue;
                    if (!(ok = mbar_wait(&sm.q_full, loads & 1u, gave_up))) break;
                    ++loads;
                    for (int j = it.j0 - 1; ok && j < it.j1; ++j, ++bundles) {
                        const int st = bundles & 1;
                        if (!(ok = mbar_wait(&sm.b_full[st], (bundles >> 1) & 1u, gave_up))) break;
                        if (!LANES && j >= it.j0 && it.masked(j)) {
                            if (!(ok = mbar_wait(&sm.v_ready[st], fixes[st] & 1u, gave_up))) break;
                            ++fixes[st];
                        }
                        tc_fence_after_sync();
                        if (C::SEPARATE_P) {
#pragma unroll
                            for (int w = 0; w < 2; ++w) {
                                if (j + 1 >= it.a0[w] && j + 1 < it.a1[w]) {
                                    // the scores before are in the softmax warps' registers
                                    if (j >= it.a0[w] && !(ok = mbar_wait(&sm.s_free[w], tile_cnt[w] & 1u, gave_up))) break;
                                    tc_fence_after_sync();
                                    issue_qk(w, st);
                                }
                            }
                            if (!ok) break;
                        }
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            if (j >= it.a0[w] && j < it.a1[w]) {
                                if (!(ok = mbar_wait(&sm.p_ready[w], tile_cnt[w] & 1u, gave_up))) break;
                                ++tile_cnt[w];
                                tc_fence_after_sync();
                                issue_pv(w, st, j == it.a0[w], j + 1 == it.a1[w]);
                            }
                            if (!C::SEPARATE_P && j + 1 >= it.a0[w] && j + 1 < it.a1[w]) issue_qk(w, st);
                        }
                        if (!ok) break;
                        umma_commit(&sm.b_empty[st]);
                        if (j + 2 == it.j1) umma_commit(&sm.q_empty);   // the item's last scores are issued
                    }
                }
            }
            __syncwarp();
        } else if (warp < 4) {
            // ------------------------------------------------------------------ values of masked tiles; copies by lanes
            const int aux = warp - 2, tid = aux * 32 + lane;
            bool ok = true, bad_page = false;
            uint32_t n_items = 0, loads = 0, bundles = 0, look_ups = 0, fixes[2] = {0, 0};
            while (ok) {
                const int slot = n_items & 1;
                ok = mbar_wait(&sm.item_full[slot], (n_items >> 1) & 1u, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                ++n_items;
                const Item it = sm.items[slot];
                if (it.last) break;
                // V_j: rows that nobody sees are zeroed, elements that are not finite zeroed and noted.  Warp `aux` has keys 64 aux ..
                // + 63; eight lanes have a row's pieces.
                auto mend = [&](int j, uint8_t *v) {
                    const int key0 = j * TK + aux * 64, sub = lane >> 3, piece = lane & 7;
                    bool any = false;
#pragma unroll 4
                    for (int i = 0; i < 16 * C::HALVES; ++i) {
                        const int hf = i >> 4, row = aux * 64 + (i & 15) * 4 + sub, key = key0 + (i & 15) * 4 + sub;
                        uint4 *at = reinterpret_cast<uint4 *>(v + hf * C::TILE_BYTES + row * 128 + ((piece ^ (row & 7)) * 16));
                        if (key < it.lo || key >= it.hi) {
                            *at = make_uint4(0u, 0u, 0u, 0u);
                        } else {
                            const uint4 x = *at;
                            any |= odd_h16(x.x) | odd_h16(x.y) | odd_h16(x.z) | odd_h16(x.w);
                        }
                    }
                    if (__any_sync(0xFFFFFFFFu, any)) {
                        const int place = it.place(j);
                        for (int i = lane; i < 64 * C::WORDS; i += 32) {   // a word: 32 elements of a key, four pieces
                            const int row = aux * 64 + i / C::WORDS, word = i % C::WORDS;
                            uint32_t bits = 0;
                            for (int q = 0; q < 4; ++q) {
                                const int piece = (word & 1) * 4 + q;
                                uint16_t *at = reinterpret_cast<uint16_t *>(v + (word >> 1) * C::TILE_BYTES + row * 128 + ((piece ^ (row & 7)) * 16));
                                for (int e = 0; e < 8; ++e)
                                    if ((at[e] & EXPONENT) == EXPONENT) {
                                        bits |= 1u << (q * 8 + e);
                                        at[e] = 0;
                                    }
                            }
                            sm.odd[slot][place][row][word] = bits;
                        }
                        if (lane == 0) sm.odd_tiles[slot][aux] |= 1u << place;
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                };
                if (!LANES) {
                    for (int j = it.j0; ok && j < it.j1; ++j) {
                        if (!it.masked(j)) continue;
                        const int st = (bundles + 1 + j - it.j0) & 1;
                        ok = mbar_wait(&sm.v_full[st], fixes[st] & 1u, gave_up);
                        ++fixes[st];
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (!ok) break;
                        mend(j, sm.ring[st].v);
                        if (lane == 0) mbar_arrive(&sm.v_ready[st]);
                    }
                    if (it.j0 < it.j1) bundles += it.j1 - it.j0 + 1;
                } else if (it.j0 < it.j1) {
                    ok = mbar_wait(&sm.q_empty, (loads & 1u) ^ 1u, gave_up);
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    ++loads;
                    const int pieces = p.head_dim / 8;
                    for (int i = tid; i < 2 * TQ * C::HALVES * 8; i += AUX) {
                        const int piece = i % (C::HALVES * 8), row = i / (C::HALVES * 8) % TQ, w = i / (C::HALVES * 8 * TQ);
                        const int token = p.by_heads.quotient(row), g = row - token * p.heads, tk = it.t0 + w * p.tokens + token;
                        const bool live = token < p.tokens && tk < it.tokens && g < it.heads && piece < pieces;
                        const uint16_t *src = p.q + (live ? (long long)(it.row0 + tk) * p.q_row + (it.h0 + g) * p.q_head + piece * 8 : 0);
                        copy16(smem_u32(sm.q[w] + (piece >> 3) * C::TILE_BYTES + row * 128 + (((piece & 7) ^ (row & 7)) * 16)), src, live);
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    fence_proxy_async_smem();
                    mbar_arrive(&sm.q_full);
                    const int *table = p.c.table + it.seq * p.c.table_stride;
                    for (int j = it.j0 - 1; j < it.j1; ++j, ++bundles) {
                        const bool has_v = j >= it.j0, has_k = j + 1 < it.j1;
                        const int mark = (it.tile0 + j + 1 - it.j0) & 3;   // of K's tile; V's is the one before
                        if (has_k) {
                            // thread t has keys t and t + 64; a warp of 32 keys makes a word
                            uint32_t words[2];
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const int local = tid + i * 64, key = (j + 1) * TK + local, n = p.by_page.quotient(key);
                                long long at = -1;
                                bool missing = false;
                                if (key >= it.lo && key < it.hi) {
                                    const int page = table[n];
                                    missing = page < 0 || page >= p.c.n_pages;
                                    if (!missing) at = page * p.c.page_stride + (key - n * p.c.page_size) * p.c.slot_stride + it.kvh * p.c.head_stride;
                                }
                                sm.at[mark][local] = at;
                                words[i] = __ballot_sync(0xFFFFFFFFu, missing);
                            }
                            if (lane == 0) {
                                sm.visible[mark][aux] = ~words[0];
                                sm.visible[mark][2 + aux] = ~words[1];
                                sm.missing[mark][aux] = (words[0] | words[1]) != 0;
                            }
                            bad_page |= (words[0] | words[1]) != 0;
                        }
                        // the other warp's places too (a wait with a limit, like all here: the other warp may have given up)
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&sm.at_ready);
                        ok = mbar_wait(&sm.at_ready, look_ups++ & 1u, gave_up);
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (!ok) break;
                        const int st = bundles & 1;
                        ok = mbar_wait(&sm.b_empty[st], ((bundles >> 1) & 1u) ^ 1u, gave_up);
                        ok = __all_sync(0xFFFFFFFFu, ok);
                        if (!ok) break;
                        // a warp has its half of the rows, so that it mends what it copied itself
#pragma unroll 1
                        for (int kv = 0; kv < 2; ++kv) {
                            if (kv ? !has_v : !has_k) continue;
                            const uint16_t *base = kv ? p.c.v : p.c.k;
                            uint8_t *to = kv ? sm.ring[st].v : sm.ring[st].k;
                            const long long *at = sm.at[kv ? (mark + 3) & 3 : mark];
#pragma unroll 8
                            for (int i = lane; i < 64 * C::HALVES * 8; i += 32) {
                                const int piece = i % (C::HALVES * 8), row = aux * 64 + i / (C::HALVES * 8);
                                const long long a = at[row];
                                const bool live = a >= 0 && piece < pieces;
                                copy16(smem_u32(to + (piece >> 3) * C::TILE_BYTES + row * 128 + (((piece & 7) ^ (row & 7)) * 16)),
                                       base + (live ? a + piece * 8 : 0), live);
                            }
                        }
                        asm volatile("cp.async.wait_all;" ::: "memory");
                        __syncwarp();
                        if (has_v && it.masked(j)) mend(j, sm.ring[st].v);
                        fence_proxy_async_smem();
                        mbar_arrive(&sm.b_full[st]);
                    }
                }
                if (!ok) break;
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.item_empty[slot]);
            }
            if (bad_page && lane == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
        }
    } else {
        // ------------------------------------------------------------------ softmax
        const int w = (warp - 4) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lane_addr = tmem_base + (static_cast<uint32_t>(quarter * 32) << 16);
        const uint32_t s_addr = lane_addr + w * TK, p_addr = lane_addr + C::P_COL0 + w * C::P_STRIDE, o_addr = lane_addr + C::O_COL0 + w * C::O_STRIDE;
        const int token = p.by_heads.quotient(row), g = row - token * p.heads;
        // s holds scores (GENERAL), or products that one factor makes scores
        const float to_log2 = GENERAL ? LOG2E : p.scale * LOG2E, to_score = GENERAL ? 1.f : p.scale;
        bool ok = true;
        uint32_t n_items = 0, tile_cnt = 0, done_cnt = 0, pf_cnt = 0;
        while (ok) {
            const int slot = n_items & 1;
            ok = mbar_wait(&sm.item_full[slot], (n_items >> 1) & 1u, gave_up);
            ok = __all_sync(0xFFFFFFFFu, ok);
            if (!ok) break;
            ++n_items;
            const Item &it = sm.items[slot];
            if (it.last) break;
            const int tk = it.t0 + w * p.tokens + token, pos = it.pos0 + tk;
            const bool live = token < p.tokens && tk < it.tokens && g < it.heads;
            const int hi = live ? max(0, pos + 1) : 0, lo = first_seen(p, pos);
            const float slope = GENERAL && p.slopes && live ? p.slopes[it.h0 + g] : 0.f;
            const int a0 = it.a0[w], a1 = it.a1[w], lo_max = it.lo_max, hi_min = it.hi_min, tile0 = it.tile0 - it.j0;
            float m = -INFINITY, l = 0.f;
            for (int j = a0; j < a1; ++j, ++tile_cnt) {
                ok = mbar_wait(&sm.s_full[w], tile_cnt & 1u, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                tc_fence_after_sync();
                const int mark = (tile0 + j) & 3;
                const bool missing = (sm.missing[mark][0] | sm.missing[mark][1]) != 0;
                const bool masked = j * TK < lo_max || (j + 1) * TK > hi_min || missing;
                // the tile in four steps, twice: the scores and their maximum; the weights.  (GENERAL: one copy of a step with both ways to
                // tanh; two of them take 160 us in place of 148 for the mixed batch, 215 in place of 205 with five times its scores.)
                float mx = -INFINITY;
#pragma unroll(GENERAL ? 1 : 2)
                for (int c = 0; c < TK / 32; ++c) {
                    float s[32];
                    tmem_ld_32x32(s_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s));
                    tmem_ld_wait();
                    if (GENERAL) {
                        if (p.cap > 0.f) {
                            float high[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int i = 0; i < 32; i += 2) high[(i >> 1) & 3] = max3f(high[(i >> 1) & 3], fabsf(s[i]), fabsf(s[i + 1]));
                            const float most = fmaxf(fmaxf(high[0], high[1]), fmaxf(high[2], high[3])) * fabsf(p.capped.by);
                            // (each score goes its own way, whatever others a warp holds: where all of them are near, that is known beforehand)
                            if (__all_sync(0xFFFFFFFFu, !live || most <= p.capped.border)) {
                                tanh_near(s, p.capped);
                            } else {
                                tanh_any(s, p.capped);
                            }
                        } else if (!p.slopes) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) s[i] *= p.scale;
                        }
                        if (p.slopes) {
                            // a place's distance bias: the first of each 16 places anew, the others by steps
                            const uint64_t step = splat2(2.f * slope), factor = splat2(p.cap > 0.f ? 1.f : p.scale);
#pragma unroll
                            for (int i = 0; i < 32; i += 16) {
                                const float first = static_cast<float>(j * TK + c * 32 + i - pos) * slope;
                                uint64_t bias = pk2(first, first + slope);
#pragma unroll
                                for (int e = 0; e < 16; e += 2) {
                                    upk2(fma2(pk2(s[i + e], s[i + e + 1]), factor, bias), s[i + e], s[i + e + 1]);
                                    bias = add2(bias, step);
                                }
                            }
                        }
                    }
                    if (masked) {
                        uint32_t bits = below(hi - j * TK - c * 32) & ~below(lo - j * TK - c * 32);
                        if (missing) bits &= sm.visible[mark][c];
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (!(bits >> i & 1)) s[i] = -INFINITY;
                    }
                    float mc[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        mc[q] = max3f(s[q * 8], s[q * 8 + 1], s[q * 8 + 2]);
#pragma unroll
                        for (int i = 3; i + 1 < 8; i += 2) mc[q] = max3f(mc[q], s[q * 8 + i], s[q * 8 + i + 1]);
                        mc[q] = fmaxf(mc[q], s[q * 8 + 7]);
                    }
                    mx = max3f(mx, fmaxf(mc[0], mc[1]), fmaxf(mc[2], mc[3]));
                    if (GENERAL || masked) tmem_st_32x32(s_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s));
                }
                if (GENERAL || masked) tmem_st_wait();
                bool raise = false;
                float f = 1.f;
                if (j == a0) {
                    m = mx;
                } else if ((mx - m) * to_log2 > RAISE) {   // (also from -inf; not from -inf to -inf)
                    raise = true;
                    f = ex2_approx((m - mx) * to_log2);
                    m = mx;
                }
                float neg = m == -INFINITY ? 0.f : HEADROOM - m * to_log2;
                // scores whose product with log2(e) may be infinite, or further from the rounded one than weights last: m is taken off first
                float off = 0.f;
                if (fabsf(neg) > 65536.f) {
                    neg = HEADROOM;
                    off = m;
                }
                const bool far = __any_sync(0xFFFFFFFFu, live && off != 0.f);   // (a row that takes off 0 stays as it is)
                if (C::SEPARATE_P && j > a0) {
                    ok = mbar_wait(&sm.p_free[w], pf_cnt & 1u, gave_up);
                    ++pf_cnt;
                    ok = __all_sync(0xFFFFFFFFu, ok);
                    if (!ok) break;
                    tc_fence_after_sync();
                }
                float sum0 = 0.f, sum1 = 0.f, sum2 = 0.f, sum3 = 0.f;
#pragma unroll 2
                for (int c = 0; c < TK / 32; ++c) {
                    float s[32];
                    tmem_ld_32x32(s_addr + c * 32, *reinterpret_cast<uint32_t(*)[32]>(&s));
                    tmem_ld_wait();
                    if (far) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) s[i] -= off;
                    }
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        float x0 = s[2 * i], x1 = s[2 * i + 1], x2 = s[2 * i + 2], x3 = s[2 * i + 3];
                        fma2(x0, x1, to_log2, neg);
                        fma2(x2, x3, to_log2, neg);
                        x0 = ex2_approx(x0);
                        x1 = ex2_approx(x1);
                        x2 = ex2_approx(x2);
                        x3 = ex2_approx(x3);
                        sum0 += x0;
                        sum1 += x1;
                        sum2 += x2;
                        sum3 += x3;
                        pk[i] = pack_h16x2(x0, x1);
                        pk[i + 1] = pack_h16x2(x2, x3);
                    }
                    tmem_st_32x16(p_addr + c * 16, pk);
                }
                if (C::SEPARATE_P) {
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm.s_free[w]);
                }
                l = l * f + ((sum0 + sum1) + (sum2 + sum3));
                if (__any_sync(0xFFFFFFFFu, raise)) {
                    // (rare) O_w holds every product issued so far: these scores were committed after the last one, and the next
                    // one waits for this warp
#pragma unroll 1
                    for (int c = 0; c < HD / 32; ++c) {
                        uint32_t r[32];
                        tmem_ld_32x32(o_addr + c * 32, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * f);
                        tmem_st_32x32(o_addr + c * 32, r);
                    }
                }
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.p_ready[w]);
            }
            if (!ok) break;
            if (a0 < a1) {
                ok = mbar_wait(&sm.pv_done[w], done_cnt & 1u, gave_up);
                ok = __all_sync(0xFFFFFFFFu, ok);
                if (!ok) break;
                ++done_cnt;
                tc_fence_after_sync();
            }
            const uint32_t odd0 = sm.odd_tiles[slot][0], odd1 = sm.odd_tiles[slot][1];
            if ((odd0 | odd1) && a0 < a1) {   // (rare) elements that a value which is not finite goes into
#pragma unroll 1
                for (int c = 0; c < C::WORDS; ++c) {
                    uint32_t odd = 0;
#pragma unroll 1
                    for (int j = a0; j < a1; ++j) {
                        if (!it.masked(j)) continue;
                        const int place = it.place(j);
#pragma unroll 1
                        for (int i = 0; i < TK; ++i)
                            if (((i < 64 ? odd0 : odd1) >> place & 1) && j * TK + i >= lo && j * TK + i < hi) odd |= sm.odd[slot][place][i][c];
                    }
                    __syncwarp();
                    uint32_t r[32];
                    tmem_ld_32x32(o_addr + c * 32, r);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (odd >> i & 1) r[i] = 0x7FFFFFFFu;
                    tmem_st_32x32(o_addr + c * 32, r);
                    tmem_st_wait();
                }
            }
            const float inv = l == 0.f ? 0.f : 1.f / l;
            const bool empty = l == 0.f, whole = it.part < 0;   // (empty: O may hold anything)
            uint16_t *dst = p.out + (long long)(it.row0 + tk) * p.out_row + (it.h0 + g) * p.out_head;
            uint4 *slot_o = reinterpret_cast<uint4 *>(slots + ((long long)blockIdx.x * 2 + (it.part & 1)) * C::PART_FLOATS + w * TQ * HD) + row;
#pragma unroll 1
            for (int c = 0; c < HD / 32; ++c) {
                uint32_t r[32];
                if (a0 < a1) {
                    tmem_ld_32x32(o_addr + c * 32, r);
                    tmem_ld_wait();
                }
                if (whole) {
                    if (live) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (c * 32 + 8 * i >= p.head_dim) break;
                            uint4 u;
                            u.x = pack_h16x2(__uint_as_float(r[8 * i + 0]) * inv, __uint_as_float(r[8 * i + 1]) * inv);
                            u.y = pack_h16x2(__uint_as_float(r[8 * i + 2]) * inv, __uint_as_float(r[8 * i + 3]) * inv);
                            u.z = pack_h16x2(__uint_as_float(r[8 * i + 4]) * inv, __uint_as_float(r[8 * i + 5]) * inv);
                            u.w = pack_h16x2(__uint_as_float(r[8 * i + 6]) * inv, __uint_as_float(r[8 * i + 7]) * inv);
                            if (empty) u = make_uint4(0u, 0u, 0u, 0u);
                            reinterpret_cast<uint4 *>(dst + c * 32)[i] = u;
                        }
                    }
                } else if (live && !empty) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) slot_o[(c * 8 + i) * TQ] = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
                }
            }
            if (live) {
                if (!whole) {
                    float *ml = slots + ((long long)blockIdx.x * 2 + (it.part & 1)) * C::PART_FLOATS + 2 * TQ * HD + w * 2 * TQ;
                    ml[row] = m;
                    ml[TQ + row] = l;
                } else if (p.lse) {
                    p.lse[(long long)(it.row0 + tk) * p.lse_row + it.h0 + g] = lse_of_weights(m * to_score, l);
                }
            }
            // O_w may be overwritten once this warp group has released its next P, which comes later in program order
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.item_empty[slot]);
        }
    }

    __syncwarp();
    if (*gave_up) {
        for (int i = 0; i < 64; ++i) __nanosleep(10000);
        if (threadIdx.x == 0 && p.status) atomicOr(p.status, STATUS_WAIT_LIMIT);
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == 1) tmem_dealloc(tmem_base, C::TMEM_COLS);
}

// Joins the parts of the units that were cut: out = sum_i o_i 2^(m_i - m) / sum_i l_i 2^(m_i - m).  CTA (i, y) has columns
// y HD / JOIN_Y .. of the unit that begins in CTA i of the kernel above, if one does; a thread has a row.
constexpr int JOIN_Y = 8;

template <int HD>
__global__ void __launch_bounds__(2 * TQ) paged_chunk_join_kernel(const ChunkParams p, int n_cta) {
    using C = Cfg<HD>;
    constexpr int Q4 = HD / JOIN_Y / 4;   // groups of four columns
    pdl_wait();
    const int begin = blockIdx.x;
    const Joint u = reinterpret_cast<const Joint *>(p.workspace)[begin];
    if (u.last_cta < 0) return;
    const float *slots = reinterpret_cast<const float *>(p.workspace + sizeof(Joint) * n_cta);
    const int w = threadIdx.x / TQ, row = threadIdx.x % TQ;
    const int token = p.by_heads.quotient(row), g = row - token * p.heads, tk = u.t0 + w * p.tokens + token;
    const int e0 = blockIdx.y * (HD / JOIN_Y);
    if (token >= p.tokens || tk >= u.tokens || g >= u.heads || e0 >= p.head_dim) return;
    const bool general = is_general(p);
    const float to_log2 = general ? LOG2E : p.scale * LOG2E, to_score = general ? 1.f : p.scale;
    auto slot = [&](int i) { return slots + ((long long)i * 2 + (i == begin ? 1 : 0)) * C::PART_FLOATS; };
    float m = -INFINITY;
    for (int i = begin; i <= u.last_cta; ++i) {
        const float *ml = slot(i) + 2 * TQ * HD + w * 2 * TQ;
        if (ml[TQ + row] != 0.f) m = fmaxf(m, ml[row]);
    }
    float l = 0.f, o[Q4 * 4];
#pragma unroll
    for (int e = 0; e < Q4 * 4; ++e) o[e] = 0.f;
#pragma unroll 2
    for (int i = begin; i <= u.last_cta; ++i) {
        const float *s = slot(i), *ml = s + 2 * TQ * HD + w * 2 * TQ;
        const float li = ml[TQ + row];
        if (li == 0.f) continue;   // (nothing seen: its output was not written)
        const float f = ex2_approx((ml[row] - m) * to_log2);
        l += li * f;
#pragma unroll
        for (int q = 0; q < Q4; ++q) {
            const float4 x = reinterpret_cast<const float4 *>(s + w * TQ * HD)[(e0 / 4 + q) * TQ + row];
            o[4 * q] += x.x * f;
            o[4 * q + 1] += x.y * f;
            o[4 * q + 2] += x.z * f;
            o[4 * q + 3] += x.w * f;
        }
    }
    const long long r = u.row0 + tk;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    uint16_t *dst = p.out + r * p.out_row + (u.h0 + g) * p.out_head + e0;
#pragma unroll
    for (int q = 0; q < Q4; q += 2) {
        if (e0 + 4 * q >= p.head_dim) break;
        *reinterpret_cast<uint4 *>(dst + 4 * q) =
            make_uint4(pack_h16x2(o[4 * q] * inv, o[4 * q + 1] * inv), pack_h16x2(o[4 * q + 2] * inv, o[4 * q + 3] * inv),
                       pack_h16x2(o[4 * q + 4] * inv, o[4 * q + 5] * inv), pack_h16x2(o[4 * q + 6] * inv, o[4 * q + 7] * inv));
    }
    if (p.lse && blockIdx.y == 0) p.lse[r * p.lse_row + u.h0 + g] = lse_of_weights(m * to_score, l);
}

template <int HD>
size_t workspace_bytes() {
    const int sms = sm_count() > 0 ? sm_count() : 148;
    return (size_t)sms * (sizeof(Joint) + 2 * Cfg<HD>::PART_FLOATS * sizeof(float));
}

template <int HD, bool GENERAL, bool LANES>
int launch_form(const ChunkParams &p, const CUtensorMap &tm_q, const CUtensorMap &tm_k, const CUtensorMap &tm_v, cudaStream_t st) {
    static DeviceOnce configured;
    constexpr int SMEM = sizeof(Smem<HD>) + 1024;
    static_assert(SMEM <= 227 * 1024, "shared memory of a CTA");
    if (!configured.done()) {
        int rc = cuda_check(cudaFuncSetAttribute(paged_chunk_kernel<HD, GENERAL, LANES>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM),
                            "paged chunk attention: shared memory opt-in");
        if (rc) return rc;
        configured.set();
    }
    const int sms = sm_count();
    if (sms <= 0) return KRAKEN_ECUDA;
    // at most so many places: every pair of query tiles against all the keys that the page table has room for
    const long long pairs = (p.rows + 2 * p.tokens - 1) / (2 * p.tokens) + p.chunks;
    const long long tiles = ((long long)p.c.max_pages * p.c.page_size + TK - 1) / TK + BEGIN;
    const int grid = static_cast<int>(std::max(1LL, std::min<long long>(sms, pairs * p.c.n_kv_head * p.head_tiles * tiles / MIN_PART)));
    int rc = cuda_check(launch_pdl(paged_chunk_kernel<HD, GENERAL, LANES>, dim3(grid), dim3(THREADS), SMEM, st, tm_q, tm_k, tm_v, p),
                        "paged chunk attention: launch");
    if (rc || grid == 1) return rc;
    return cuda_check(launch_pdl(paged_chunk_join_kernel<HD>, dim3(grid, JOIN_Y), dim3(2 * TQ), 0, st, p, grid), "paged chunk attention join: launch");
}

template <int HD>
int launch(const ChunkParams &p, cudaStream_t st) {
    const bool general = is_general(p);
    CUtensorMap tm_q, tm_k, tm_v;
    // Strides of 0 and what else a tensor map cannot hold: the lanes copy.  A dimension of one may have any stride.
    const long long hd = p.head_dim;
    const long long slot = p.c.page_size > 1 ? p.c.slot_stride : hd, head = p.c.n_kv_head > 1 ? p.c.head_stride : hd,
                    page = p.c.n_pages > 1 ? p.c.page_stride : hd, q_row = p.rows > 1 ? p.q_row : hd, q_head = p.n_head > 1 ? p.q_head : hd;
    if (p.c.page_size % 8 == 0 && slot > 0 && head > 0 && page > 0 && q_row > 0 && q_head > 0) {
        const uint64_t dims[4] = {(uint64_t)hd, (uint64_t)p.c.page_size, (uint64_t)p.c.n_kv_head, (uint64_t)p.c.n_pages};
        const uint64_t strides[3] = {(uint64_t)slot, (uint64_t)head, (uint64_t)page};
        const uint32_t box[4] = {64, (uint32_t)p.box, 1, 1};
        const uint64_t q_dims[4] = {(uint64_t)hd, (uint64_t)p.n_head, (uint64_t)p.rows, 1};
        const uint64_t q_strides[3] = {(uint64_t)q_head, (uint64_t)q_row, (uint64_t)hd};
        const uint32_t q_box[4] = {64, (uint32_t)p.heads, (uint32_t)p.tokens, 1};
        if (encode_tma_4d_bf16(&tm_k, p.c.k, dims, strides, box) == KRAKEN_OK && encode_tma_4d_bf16(&tm_v, p.c.v, dims, strides, box) == KRAKEN_OK &&
            encode_tma_4d_bf16(&tm_q, p.q, q_dims, q_strides, q_box) == KRAKEN_OK)
            return general ? launch_form<HD, true, false>(p, tm_q, tm_k, tm_v, st) : launch_form<HD, false, false>(p, tm_q, tm_k, tm_v, st);
    }
    memset(&tm_q, 0, sizeof(tm_q));
    return general ? launch_form<HD, true, true>(p, tm_q, tm_q, tm_q, st) : launch_form<HD, false, true>(p, tm_q, tm_q, tm_q, st);
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

}  // namespace kr

extern "C" int kraken_paged_chunk_attention_workspace(int32_t head_dim, size_t *bytes) {
    using namespace kr;
    if (!bytes) return KRAKEN_EINVAL;
    if (!decode_head_dim_ok(head_dim)) return KRAKEN_EUNSUPPORTED;
    *bytes = head_dim <= 64 ? workspace_bytes<64>() : workspace_bytes<128>();
    return KRAKEN_OK;
}

extern "C" int kraken_op_paged_chunk_attention(const kraken_paged_cache *cache, const kraken_paged_chunk_args *a, uint32_t *d_status,
                                               void *stream) {
    using namespace kr;
    ChunkParams p = {};
    if (!a) return KRAKEN_EINVAL;
    int rc = paged_view(cache, &p.c);
    if (rc) return rc;
    if (a->rows == 0 || a->chunks == 0) return KRAKEN_OK;
    if (a->rows < 0 || a->chunks < 0 || !a->q || !a->out || !a->q_start || !a->n_keys || a->n_head < 1 || a->n_head % cache->n_kv_head != 0 ||
        a->window < 0 || !isfinite(a->score_cap) || a->score_cap < 0.f)
        return KRAKEN_EINVAL;
    // (factors in the kernel: a score of 0 times an infinite one would be a NaN)
    if (a->score_cap > 0.f) p.capped = Cap(a->scale, a->score_cap);
    if (!isfinite(a->scale * LOG2E) || (a->score_cap > 0.f && (!isfinite(1.f / a->score_cap) || !isfinite(p.capped.by))))
        return KRAKEN_EINVAL;
    if (!a->chunk_seq && a->chunks > cache->n_seqs) return KRAKEN_EINVAL;
    if ((a->rows > 1 && a->out_row_stride == 0) || (a->n_head > 1 && a->out_head_stride == 0) || (a->lse && a->rows > 1 && a->lse_row_stride == 0))
        return KRAKEN_EINVAL;
    if (!aligned16(a->q) || !aligned16(a->out) || ((a->q_row_stride | a->q_head_stride | a->out_row_stride | a->out_head_stride) & 7))
        return KRAKEN_EUNSUPPORTED;
    if (!a->workspace || a->workspace_bytes < (cache->head_dim <= 64 ? workspace_bytes<64>() : workspace_bytes<128>())) return KRAKEN_ECAPACITY;
    if (!aligned16(a->workspace)) return KRAKEN_EINVAL;
    p.workspace = static_cast<uint8_t *>(a->workspace);
    p.q = static_cast<const uint16_t *>(a->q);
    p.out = static_cast<uint16_t *>(a->out);
    p.lse = a->lse;
    p.chunk_seq = a->chunk_seq;
    p.q_start = a->q_start;
    p.n_keys = a->n_keys;
    p.slopes = a->slopes;
    p.q_row = a->q_row_stride;
    p.q_head = a->q_head_stride;
    p.out_row = a->out_row_stride;
    p.out_head = a->out_head_stride;
    p.lse_row = a->lse_row_stride;
    p.scale = a->scale;
    p.cap = a->score_cap;
    p.chunks = a->chunks;
    p.rows = a->rows;
    p.n_head = a->n_head;
    p.rep = a->n_head / cache->n_kv_head;
    p.window = a->window;
    p.head_dim = cache->head_dim;
    p.head_tiles = (p.rep + TQ - 1) / TQ;
    p.heads = (p.rep + p.head_tiles - 1) / p.head_tiles;
    p.tokens = TQ / p.heads;
    // (the places of a head are added up in 32 bits)
    const long long pairs = (long long)a->rows / (2 * p.tokens) + a->chunks;
    if (a->rows >= 1 << 22 || a->chunks >= 1 << 22 || pairs * ((long long)cache->max_pages * cache->page_size / TK + 2 + BEGIN) >= 1LL << 31)
        return KRAKEN_EUNSUPPORTED;
    p.status = d_status;
    p.by_page = Divisor(cache->page_size);
    p.by_heads = Divisor(p.heads);
    p.box = 8;
    while (p.box < TK && cache->page_size % (2 * p.box) == 0) p.box *= 2;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    return cache->head_dim <= 64 ? launch<64>(p, st) : launch<128>(p, st);
}
