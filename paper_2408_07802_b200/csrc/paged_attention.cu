// Decode-step attention over a key/value cache in pages: one query per head and row against the cached keys of the
// row's sequence, which the page table leads to.
//
//   x_j = scale q.k_j  [cap tanh(x/cap)]  [+ slope (j - (n - 1))],  out = sum_j softmax(x)_j v_j,  lse = log sum_j e^x_j
//
// A row reads every key and value once for up to 16 of the n_head / n_kv_head query heads that share it (for more heads once for
// each 16 of them): 4 bytes a key element against 4 FLOP per query head, at most 16 FLOP a byte or 100 TFLOP/s at the copy
// bandwidth.  So this is bound by HBM, and the products run on the warp-level tensor instructions, which take both operands from
// registers.  Rows of the same sequence read its keys each for itself.
//
// The products of 16 keys with the 8 or 16 query heads of a tile (m16n8k16):
//   S[head, key] = Q K^T        the heads are the rows (rows 8..15 are empty up to 8 heads); a lane reads 16 bytes (8
//                               consecutive elements) of one key and feeds them to two products; Q is held with the same
//                               order of elements in the k slots, which is all a dot product needs
//   O^T[e, head] += V^T P^T     P comes straight from the score accumulators (their layout is that of the second operand); a
//                               lane reads 16 bytes of four keys and pairs neighbouring keys by byte permutes; rows g and
//                               g + 8 of product j stand for elements 8 g + 2 j and 8 g + 2 j + 1
// P goes into the product as the sum of two 16-bit numbers (its rounding and the rounding of the rest), so its rounding,
// which would be as large as that of the output, does not count.  Maximum and sum are kept in fp32, and the maximum in use
// is only raised when a score exceeds it by more than 8 in the exponent of 2 (numerator and denominator carry the same
// factor), so most blocks need one vote of the warp where a running maximum would take shuffles and a rescaling.
//
// Measured, 32 query heads on 8 of 128: one sequence of 131072 keys 86 us = 6.2 TB/s; 64 sequences of 8192 322 us = 6.7 TB/s.
// On the way there (the one sequence): a CTA per row and head 3955 us; the keys shared out 133; blocks copied ahead by the lanes
// into shared memory 120, whatever the number of instructions (541, then 350 a block) and of stages: 16-byte copies of 64-byte
// pieces; by the copy engine 90.  Below that, 5 us pass before the first key is there and 3 in the joining kernel.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "paged.cuh"

namespace kr {

namespace {

constexpr int PA_WARPS = 4;
constexpr int STAGES = 2;                // steps of a warp in shared memory: one being used, one on its way
// What beginning and finishing a unit costs, in tiles: without it a CTA whose share is a run of short sequences took 17 us
// longer than the others (64 ragged sequences).
constexpr int BEGIN = 1;
// Units of up to so many tiles are not split where there is a CTA for each: working off the tiles one after the other then takes
// no longer than joining parts (24 sequences of 500 keys, 16 heads of 64: 11.4 against 16.4 us; one sequence: 8.3 against 8.1;
// with 8 tiles, one sequence of 1000 keys: 12.4 against 8.3).
constexpr int WHOLE_TILES = 4;
// A weight is 2^(score - m) with m so chosen that the largest of a block is 2^HEADROOM when m is set, and m is raised when a
// score would get past 2^(HEADROOM + 8).  HEADROOM = 7 in the half image: half numbers end at 2^16 and 2^-24, and weights that
// round to nothing against the largest one, 10^5 of them, would be missing from the output and not from the sum.
constexpr float HEADROOM = KRAKEN_F16 ? 7.f : 0.f;
constexpr float RAISE = HEADROOM + 8.f;

struct PagedAttnParams {
    PagedView c;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    const int *row_seq, *n_keys;
    const float *slopes;
    long long q_row, q_head, out_row, out_head, lse_row;
    float scale, cap;
    int rows, n_head, window;
    uint32_t *status;
    uint8_t *workspace;
    Divisor by_page;
    int box;   // keys of a copy: 16 or 8
    bool whole;   // CTA i works on unit i, all of it: known from the size of the page table
};

__device__ __forceinline__ void mma_keys(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32." KRAKEN_MMA_T "." KRAKEN_MMA_T ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// One step of a warp: SUBS blocks of 16 keys of one (sequence, key/value head).  A block lies in shared memory as tiles of
// 16 rows x 128 bytes (64 elements), the halves of K and then those of V, with the 128-byte swizzle: the 16-byte piece c of
// row r is at r * 128 + (c ^ (r & 7)) * 16.  Of a block a lane reads (g = lane / 4, t = lane % 4)
//   keys g and g + 8 of K: of every half the pieces 2t and 2t + 1;      keys 2t, 2t + 1, 2t + 8, 2t + 9 of V: piece g
// which in this layout are free of bank conflicts.
template <int HD>
struct Step {
    static constexpr int HF = (HD + 63) / 64;       // 64-element halves of a head
    static constexpr int HALF = 16 * 128;           // bytes of a tile
    static constexpr int BLOCK = 2 * HF * HALF;
    static constexpr int SUBS = HD <= 64 ? 2 : 1;
    static constexpr int BYTES = SUBS * BLOCK;
    static constexpr int KEYS = SUBS * 16;          // of a warp
    static constexpr int TILE = KEYS * PA_WARPS;    // of the CTA
};

template <int HD, int NT>
struct Running {   // online softmax of 8 NT heads over the keys of one warp
    static constexpr int HF = Step<HD>::HF;
    float m[NT], base[NT], l[NT];   // head 8 nt + g: exponent in use (log2 domain; base: 0 for -inf), this lane's part of the sum
    float o[NT][HF * 4][4];         // heads 8 nt + 2t + {0, 1}
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt] = -INFINITY;
            base[nt] = l[nt] = 0.f;
#pragma unroll
            for (int j = 0; j < HF * 4; ++j) o[nt][j][0] = o[nt][j][1] = o[nt][j][2] = o[nt][j][3] = 0.f;
        }
    }
};

__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : (i == 1 ? v.y : (i == 2 ? v.z : v.w)); }

// Score options that the caller asked for, uniform over the launch
struct ScoreForm {
    float scale, cap, inv_cap;
    bool plain;      // neither cap nor slopes: one product takes the scale and log2(e)
    float scale2;    // scale * log2(e)
};

// `mask`: which keys of the step are visible; `back`: position of its first key minus that of the query
template <int HD, int NT>
__device__ __forceinline__ void take_step(Running<HD, NT> &run, const uint8_t *step, const uint4 (&q)[NT][2 * Step<HD>::HF],
                                          uint32_t mask, int back, const ScoreForm &f, const float (&slope)[NT], int lane) {
    constexpr int HF = Step<HD>::HF, SUBS = Step<HD>::SUBS, BLOCK = Step<HD>::BLOCK, HALF = Step<HD>::HALF;
    constexpr uint32_t ALL = SUBS == 2 ? 0xFFFFFFFFu : 0xFFFFu;
    const int g = lane >> 2, t = lane & 3;
    float s[2 * SUBS][4];   // [8 keys]: head g, keys 2t and 2t + 1; head g + 8, the same keys
#pragma unroll
    for (int kt = 0; kt < 2 * SUBS; ++kt) {
        float z[4] = {0.f, 0.f, 0.f, 0.f};   // two chains of products: a chain of all of them would take twice as long
        s[kt][0] = s[kt][1] = s[kt][2] = s[kt][3] = 0.f;
#pragma unroll
        for (int c = 0; c < 2 * HF; ++c) {
            const uint4 k = *reinterpret_cast<const uint4 *>(step + (kt >> 1) * BLOCK + (c >> 1) * HALF + (kt & 1) * 1024 + g * 128 +
                                                             ((2 * t + (c & 1)) ^ g) * 16);
            const uint4 a = q[0][c], b = NT == 2 ? q[NT - 1][c] : make_uint4(0u, 0u, 0u, 0u);
            mma_keys(s[kt], a.x, b.x, a.y, b.y, k.x, k.y);
            mma_keys(z, a.z, b.z, a.w, b.w, k.z, k.w);
        }
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) s[kt][i] += z[i];
    }
    bool over = false;
#pragma unroll
    for (int kt = 0; kt < 2 * SUBS; ++kt)
#pragma unroll
        for (int i = 0; i < 2 * NT; ++i) {
            float x = s[kt][i];
            if (f.plain) {
                x *= f.scale2;
            } else {
                x *= f.scale;
                if (f.cap > 0.f) x = f.cap * tanhf(x * f.inv_cap);
                x = (x + slope[i >> 1] * static_cast<float>(back + kt * 8 + 2 * t + (i & 1))) * LOG2E;
            }
            s[kt][i] = x;
        }
    if (mask != ALL) {
#pragma unroll
        for (int kt = 0; kt < 2 * SUBS; ++kt)
#pragma unroll
            for (int i = 0; i < 2 * NT; ++i)
                if (!(mask >> (kt * 8 + 2 * t + (i & 1)) & 1)) s[kt][i] = -INFINITY;
    }
    float top[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        top[nt] = fmaxf(s[0][2 * nt], s[0][2 * nt + 1]);
#pragma unroll
        for (int kt = 1; kt < 2 * SUBS; ++kt) top[nt] = fmaxf(top[nt], fmaxf(s[kt][2 * nt], s[kt][2 * nt + 1]));
        over |= top[nt] > run.m[nt] + RAISE;
    }
    if (__any_sync(0xFFFFFFFFu, over)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float mx = fmaxf(top[nt], __shfl_xor_sync(0xFFFFFFFFu, top[nt], 1));
            mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 2));
            mx = fmaxf(mx - HEADROOM, run.m[nt]);
            run.base[nt] = mx == -INFINITY ? 0.f : mx;   // nothing visible yet: every weight is 2^-inf = 0
            const float corr = ex2_approx(run.m[nt] - run.base[nt]);
            run.m[nt] = mx;
            run.l[nt] *= corr;
            const float c0 = __shfl_sync(0xFFFFFFFFu, corr, t * 8), c1 = __shfl_sync(0xFFFFFFFFu, corr, t * 8 + 4);
#pragma unroll
            for (int j = 0; j < HF * 4; ++j) {
                run.o[nt][j][0] *= c0;
                run.o[nt][j][1] *= c1;
                run.o[nt][j][2] *= c0;
                run.o[nt][j][3] *= c1;
            }
        }
    }
    uint32_t hi[NT][2 * SUBS], lo[NT][2 * SUBS];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int kt = 0; kt < 2 * SUBS; ++kt) {
            const float p0 = ex2_approx(s[kt][2 * nt] - run.base[nt]), p1 = ex2_approx(s[kt][2 * nt + 1] - run.base[nt]);
            run.l[nt] += p0 + p1;
            hi[nt][kt] = pack_h16x2(p0, p1);
            lo[nt][kt] = pack_h16x2(p0 - h16_lo(hi[nt][kt]), p1 - h16_hi(hi[nt][kt]));
        }
#pragma unroll
    for (int sb = 0; sb < SUBS; ++sb)
#pragma unroll
        for (int hf = 0; hf < HF; ++hf) {
            uint4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = *reinterpret_cast<const uint4 *>(step + sb * BLOCK + (HF + hf) * HALF + (i >> 1) * 1024 + (2 * t + (i & 1)) * 128 +
                                                        (g ^ (2 * t + (i & 1))) * 16);
            if (mask != ALL) {   // what lies behind the visible keys may be anything, and 0 times a NaN is one
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(mask >> (sb * 16 + (i >> 1) * 8 + 2 * t + (i & 1)) & 1)) v[i] = make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a0 = __byte_perm(word(v[0], j), word(v[1], j), 0x5410), a1 = __byte_perm(word(v[0], j), word(v[1], j), 0x7632);
                const uint32_t a2 = __byte_perm(word(v[2], j), word(v[3], j), 0x5410), a3 = __byte_perm(word(v[2], j), word(v[3], j), 0x7632);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma_keys(run.o[nt][hf * 4 + j], a0, a1, a2, a3, hi[nt][2 * sb], hi[nt][2 * sb + 1]);
                    mma_keys(run.o[nt][hf * 4 + j], a0, a1, a2, a3, lo[nt][2 * sb], lo[nt][2 * sb + 1]);
                }
            }
        }
}

// What row r asks for: its visible keys lo .. n - 1 of sequence seq.  False: padding, or (bad) no such sequence or length.
struct RowKeys {
    int seq, lo, n, tiles;   // tiles from lo rounded down to a multiple of 16; at least one (a row without keys writes zeros)
    __device__ __forceinline__ int start() const { return lo & ~15; }
};

template <int TILE>
__device__ __forceinline__ bool row_keys(const PagedAttnParams &p, int r, RowKeys &k, bool &bad) {
    k.seq = p.row_seq ? p.row_seq[r] : r;
    k.n = p.n_keys[r];
    k.tiles = 0;
    if (k.seq < 0) return false;
    if (k.seq >= p.c.n_seqs || k.n < 0 || k.n > (long long)p.c.max_pages * p.c.page_size) {
        bad = true;
        return false;
    }
    k.lo = p.window > 0 && k.n > p.window ? k.n - p.window : 0;
    k.tiles = max(1, (k.n - k.start() + TILE - 1) / TILE);
    return true;
}

// The work of a call is a line: rows in order, of each row its (key/value head, head tile) units in order, of each unit `begin`
// places for its beginning and end and then one for every key tile (begin: BEGIN, or 0 where there are no more tiles than
// CTAs; a unit is one place where none is to be split).  CTA i of G takes the places [total i / G, total (i + 1) / G), the same
// number for every CTA whatever the lengths, and works on the tiles among them; G is at most total / (begin + 1), so that
// there are some.  A unit that lies in one CTA is finished there; of one that does not, every CTA leaves its part in the
// workspace (slot 1 where the unit begins, slot 0 elsewhere: a CTA has at most one of each) and the CTA with the beginning
// notes who has the rest, for the joining kernel.
struct Part {
    int row, unit, last_cta;   // row = -1: nothing to join
    int pad;
};

// A part in the workspace, as the accumulators lie in a warp: [NT][HF * 4 products][32 lanes][4] o, then [2][HEADS] m and l.
template <int HD, int NT>
struct PartShape {
    static constexpr int HEADS = 8 * NT, PRODUCTS = Step<HD>::HF * 4;
    static constexpr int O_FLOATS = NT * PRODUCTS * 128;
    static constexpr int FLOATS = O_FLOATS + 2 * HEADS;
};

// Accumulator of product j, head tile nt: elements e and e + 1 of heads 8 nt + 2t and 8 nt + 2t + 1 are (x, z) and (y, w).
template <int HD>
__device__ __forceinline__ void store_pair(const PagedAttnParams &p, int row, int h0, int heads, int nt, int j, int lane, float4 o,
                                           const float (&l)[2]) {
    const int h = nt * 8 + 2 * (lane & 3), e = (j >> 2) * 64 + (lane >> 2) * 8 + 2 * (j & 3);
    if (e >= HD) return;
    uint16_t *out = p.out + row * p.out_row + (h0 + h) * p.out_head + e;
    const float i0 = l[0] == 0.f ? 0.f : 1.f / l[0], i1 = l[1] == 0.f ? 0.f : 1.f / l[1];
    if (h < heads) *reinterpret_cast<uint32_t *>(out) = pack_h16x2(o.x * i0, o.z * i0);
    if (h + 1 < heads) *reinterpret_cast<uint32_t *>(out + p.out_head) = pack_h16x2(o.y * i1, o.w * i1);
}

// The tiles of a call are added up in the lower bits of a 64-bit number, and the rows that have some above them; a call that might
// not fit is refused.  (Two numbers would take twice the shuffles before the first key is asked for.)
constexpr int ROWS_AT = 40;

// A place on the line of tiles
struct Place {
    int r, unit, tile;
    RowKeys k;
};

template <int HD, int NT>
struct Smem {
    uint8_t ring[PA_WARPS][STAGES][Step<HD>::BYTES];
    float4 o[PA_WARPS][4][32];   // four products of every warp, to be joined
    float m[PA_WARPS][8 * NT], l[PA_WARPS][8 * NT];
    uint64_t full[PA_WARPS][STAGES];
    long long sum[PA_WARPS], before;
    int most[PA_WARPS];
    RowKeys keys;
    int row;
    uint32_t gave_up;
};

// Spills: up to 24 bytes a thread, 44 in the instance for 64-wide heads (128 registers), where they are one store and less than one
// load a step and warp, 0.3 % of its instructions.
//
// BOXES: pages of a multiple of 16 (or 8) keys, which the copy engine brings in as boxes of 16 (8) keys, one 64-element half at
// a time, by tensor maps over (element, slot, head, page); with other page sizes the lanes copy, each the pieces that it will
// read itself.
template <int HD, int NT, bool BOXES>
__global__ void __launch_bounds__(PA_WARPS * 32) paged_attn_kernel(const __grid_constant__ CUtensorMap tm_k,
                                                                   const __grid_constant__ CUtensorMap tm_v, const PagedAttnParams p) {
    constexpr int HF = Step<HD>::HF, SUBS = Step<HD>::SUBS, BLOCK = Step<HD>::BLOCK, HALF = Step<HD>::HALF, KEYS = Step<HD>::KEYS;
    constexpr int TILE = Step<HD>::TILE, HEADS = 8 * NT;
    using Shape = PartShape<HD, NT>;
    extern __shared__ uint8_t smem_raw[];
    Smem<HD, NT> &sm = *reinterpret_cast<Smem<HD, NT> *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    if (threadIdx.x == 0) {
        sm.row = -1;
        sm.gave_up = 0;
        if (BOXES) {
            for (int i = 0; i < PA_WARPS * STAGES; ++i) mbar_init(&sm.full[0][0] + i, 1);
            fence_barrier_init();
            prefetch_tensormap(&tm_k);
            prefetch_tensormap(&tm_v);
        }
    }
    pdl_wait();
    const int rep = p.n_head / p.c.n_kv_head;
    const int head_tiles = (rep + HEADS - 1) / HEADS;
    const int units = p.c.n_kv_head * head_tiles;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    Part *parts = reinterpret_cast<Part *>(p.workspace);
    float *slots = reinterpret_cast<float *>(p.workspace + sizeof(Part) * gridDim.x);

    // `at`: the tile being worked on; `ahead`: the tile whose copy is issued next, up to STAGES - 1 further on
    Place at;
    bool bad = false;
    int begin = 0;
    long long all = 0, n_cta = 0, row_c0 = 0;   // places, CTAs that share them, first place of row at.r
    // places left to the copies and to the work: they go on by one place a tile, and by `begin` where a unit begins
    long long to_issue;
    if (p.whole) {
        at.r = blockIdx.x / units;
        at.unit = blockIdx.x % units;
        at.tile = 0;
        row_keys<TILE>(p, at.r, at.k, bad);
        if (bad && at.unit == 0 && threadIdx.x == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
        to_issue = at.k.tiles;
        pdl_trigger();
        if (to_issue == 0) return;
        __syncthreads();
    } else {
        if (threadIdx.x == 0) parts[blockIdx.x].row = -1;
        // where this CTA's share begins: every thread adds up the tiles of a run of rows
        const int per = (p.rows + PA_WARPS * 32 - 1) / (PA_WARPS * 32);
        const int row_lo = min(p.rows, (int)threadIdx.x * per), row_hi = min(p.rows, row_lo + per);
        long long mine = 0;
        int most = 0;
        for (int r = row_lo; r < row_hi; ++r) {
            RowKeys k;
            row_keys<TILE>(p, r, k, bad);
            if (k.tiles > 0) mine += (1LL << ROWS_AT) + k.tiles;
            most = max(most, k.tiles);
        }
        most = __reduce_max_sync(0xFFFFFFFFu, most);
        long long upto = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long v = __shfl_up_sync(0xFFFFFFFFu, upto, off);
            if (lane >= off) upto += v;
        }
        if (lane == 31) {
            sm.sum[warp] = upto;
            sm.most[warp] = most;
        }
        __syncthreads();
        long long total = 0;
#pragma unroll
        for (int w = 0; w < PA_WARPS; ++w) {
            if (w < warp) upto += sm.sum[w];
            total += sm.sum[w];
            most = max(most, sm.most[w]);
        }
        // a unit is one place: units of few tiles, and more of them than half the CTAs
        const long long n_units = (total >> ROWS_AT) * units;
        const bool whole = most <= WHOLE_TILES && n_units <= gridDim.x && 2 * n_units >= gridDim.x;
        begin = (total & ((1LL << ROWS_AT) - 1)) * units <= gridDim.x ? 0 : BEGIN;
        auto places = [&](long long sum) {
            const long long rows = sum >> ROWS_AT, tiles = sum & ((1LL << ROWS_AT) - 1);
            return (whole ? rows : tiles + rows * begin) * units;
        };
        all = places(total);
        n_cta = whole ? all : min((long long)gridDim.x, all / (begin + 1));
        const long long c0 = blockIdx.x < n_cta ? all * blockIdx.x / n_cta : all;
        const long long c1 = blockIdx.x < n_cta ? all * (blockIdx.x + 1) / n_cta : all;
        {
            long long before = places(upto - mine);
            if (c0 < c1 && c0 >= before && c0 < places(upto)) {
                for (int r = row_lo; r < row_hi; ++r) {
                    RowKeys k;
                    row_keys<TILE>(p, r, k, bad);
                    const long long here = k.tiles > 0 ? (whole ? 1LL : k.tiles + begin) * units : 0;
                    if (c0 < before + here) {
                        sm.row = r;
                        sm.keys = k;
                        sm.before = before;
                        break;
                    }
                    before += here;
                }
            }
        }
        if (bad && blockIdx.x == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
        pdl_trigger();
        if (c0 >= c1) return;
        __syncthreads();
        at.r = sm.row;
        at.k = sm.keys;
        if (at.r < 0) return;   // (no such row, here and below: the lengths changed under the kernel)
        row_c0 = sm.before;
        const int weight = whole ? 1 : at.k.tiles + begin, skipped = static_cast<int>((c0 - row_c0) % weight);
        at.unit = static_cast<int>((c0 - row_c0) / weight);
        at.tile = max(0, skipped - begin);
        to_issue = whole ? at.k.tiles : c1 - c0 - max(0, begin - skipped);
    }
    Place ahead = at;
    long long left = to_issue;
    bool bad_page = false;
    auto step_row = [&](Place &w) {   // to the next row with tiles; false when there is none
        do {
            if (++w.r == p.rows) return false;
            row_keys<TILE>(p, w.r, w.k, bad);
        } while (w.k.tiles == 0);
        return true;
    };
    // Lane i looks up the page of box i of a step (BOXES), or of key i; -1: not visible.  A step is looked up one step before its
    // copies need it.
    const int box = BOXES ? p.box : 1;   // keys
    int page, slot, head = 0;
    auto look_up = [&] {
        const int key = ahead.k.start() + ahead.tile * TILE + warp * KEYS + (BOXES ? min(lane * box, KEYS) : lane & (KEYS - 1));
        const int n = p.by_page.quotient(key);
        slot = key - n * p.c.page_size;
        page = key < ahead.k.n && (BOXES ? lane * box < KEYS : key >= ahead.k.lo) ? p.c.table[ahead.k.seq * p.c.table_stride + n] : -1;
    };
    int fill = 0;
    uint32_t seen[STAGES - 1];   // keys visible in the steps under way, oldest first
    auto issue = [&]() -> uint32_t {
        uint32_t mask = 0;
        if (to_issue > 0) {
            const int key0 = ahead.k.start() + ahead.tile * TILE + warp * KEYS;
            if (key0 < ahead.k.n) {
                uint8_t *to = sm.ring[warp][fill];
                if constexpr (BOXES) {
                    const int key = key0 + lane * box;
                    const bool mine = lane * box < KEYS && key < ahead.k.n && key + box > ahead.k.lo;
                    const bool there = mine && page >= 0 && page < p.c.n_pages;
                    bad_page |= mine && !there;
                    const uint32_t boxes = __ballot_sync(0xFFFFFFFFu, there);   // (every lane has read what this stage held before)
#pragma unroll
                    for (int i = 0; i < KEYS / 8; ++i)
                        if (boxes >> i & 1) mask |= ((1u << box) - 1u) << ((i * box) & 31);
                    // of these the keys lo .. n - 1
                    const int to_n = ahead.k.n - key0, to_lo = ahead.k.lo - key0;
                    if (to_n < 32) mask &= (1u << to_n) - 1u;
                    if (to_lo > 0) mask = to_lo >= 32 ? 0u : mask >> to_lo << to_lo;
                    if (boxes) {
                        uint64_t *full = &sm.full[warp][fill];
                        if (lane == 0) mbar_expect_tx(full, __popc(boxes) * box * (2 * HF * 128));
                        __syncwarp();
                        if (there) {
                            uint8_t *row = to + (lane * box / 16) * BLOCK + (lane * box % 16) * 128;
#pragma unroll
                            for (int hf = 0; hf < HF; ++hf) {
                                tma_load_4d(row + hf * HALF, &tm_k, full, hf * 64, slot, head, page);
                                tma_load_4d(row + (HF + hf) * HALF, &tm_v, full, hf * 64, slot, head, page);
                            }
                        }
                    }
                } else {
                    const int key = key0 + (lane & (KEYS - 1));
                    // (a step begins up to 15 keys in front of a window: their pages may have been given back)
                    const bool mine = key < ahead.k.n && key >= ahead.k.lo;
                    if (page < 0 || page >= p.c.n_pages) {
                        bad_page |= mine;
                        page = -1;
                    }
                    mask = __ballot_sync(0xFFFFFFFFu, mine && page >= 0);
                    if (SUBS == 1) mask &= 0xFFFFu;
                    const long long off = max(page, 0) * p.c.page_stride + slot * p.c.slot_stride + head * p.c.head_stride;
                    const uint32_t at = smem_u32(to);
#pragma unroll
                    for (int sb = 0; sb < SUBS; ++sb) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int who = sb * 16 + g + 8 * i;
                            const uint16_t *row = p.c.k + __shfl_sync(0xFFFFFFFFu, off, who);
#pragma unroll
                            for (int c = 0; c < 2 * HF; ++c) {
                                const int e = (c >> 1) * 64 + (2 * t + (c & 1)) * 8;
                                const bool in = (mask >> who & 1) && e < HD;
                                copy16(at + sb * BLOCK + (c >> 1) * HALF + i * 1024 + g * 128 + ((2 * t + (c & 1)) ^ g) * 16,
                                       in ? row + e : p.c.k, in);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int who = sb * 16 + 2 * t + (i & 1) + (i >> 1) * 8;
                            const uint16_t *row = p.c.v + __shfl_sync(0xFFFFFFFFu, off, who);
#pragma unroll
                            for (int hf = 0; hf < HF; ++hf) {
                                const int e = hf * 64 + g * 8;
                                const bool in = (mask >> who & 1) && e < HD;
                                copy16(at + sb * BLOCK + (HF + hf) * HALF + (i >> 1) * 1024 + (2 * t + (i & 1)) * 128 +
                                           (g ^ (2 * t + (i & 1))) * 16, in ? row + e : p.c.v, in);
                            }
                        }
                    }
                }
            }
            if (--to_issue > 0) {
                if (++ahead.tile == ahead.k.tiles) {
                    ahead.tile = 0;
                    to_issue -= begin;
                    if (++ahead.unit == units) {
                        ahead.unit = 0;
                        if (to_issue > 0 && !step_row(ahead)) to_issue = 0;
                    }
                    head = ahead.unit / head_tiles;
                }
                if (to_issue > 0) look_up();
            }
        }
        if (!BOXES) asm volatile("cp.async.commit_group;" ::: "memory");
        if (++fill == STAGES) fill = 0;
        return mask;
    };
    // the oldest step under way has arrived
    uint32_t phases = 0;
    auto arrived = [&](int stage, uint32_t mask) {
        if constexpr (BOXES) {
            if (!mask) return;
            mbar_wait(&sm.full[warp][stage], phases >> stage & 1, &sm.gave_up);
            phases ^= 1u << stage;
            __syncwarp();
        } else {
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
        }
    };
    head = ahead.unit / head_tiles;
    look_up();
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) seen[i] = issue();

    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    const ScoreForm form = {p.scale, p.cap, p.cap > 0.f ? 1.f / p.cap : 0.f, p.cap <= 0.f && !p.slopes, p.scale * LOG2E};
    int use = 0;
    uint4 q[NT][2 * HF];
    float slope[NT];
    auto load_q = [&] {
        const int first = at.unit % head_tiles * HEADS, heads = min(HEADS, rep - first), h0 = at.unit / head_tiles * rep + first;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int h = nt * 8 + g;
#pragma unroll
            for (int c = 0; c < 2 * HF; ++c) {
                const int e = (c >> 1) * 64 + (2 * t + (c & 1)) * 8;
                q[nt][c] = h < heads && e < HD ? *reinterpret_cast<const uint4 *>(p.q + at.r * p.q_row + (h0 + h) * p.q_head + e) : zero;
            }
            slope[nt] = p.slopes && h < heads ? p.slopes[h0 + h] : 0.f;
        }
    };
    load_q();
    while (left > 0) {
        const int seg = static_cast<int>(min(left, (long long)(at.k.tiles - at.tile)));
        const int first = at.unit % head_tiles * HEADS, heads = min(HEADS, rep - first), h0 = at.unit / head_tiles * rep + first;
        const int row = at.r;
        Running<HD, NT> run;
        run.clear();
        for (int i = 0; i < seg; ++i) {
            const uint32_t mask = seen[0];
            arrived(use, mask);
#pragma unroll
            for (int j = 0; j + 1 < STAGES - 1; ++j) seen[j] = seen[j + 1];
            // the step used before has been read: its place takes the next copies
            seen[STAGES - 2] = issue();
            if (mask)
                take_step<HD, NT>(run, sm.ring[warp][use], q, mask,
                                  at.k.start() + (at.tile + i) * TILE + warp * KEYS - (at.k.n - 1), form, slope, lane);
            if (++use == STAGES) use = 0;
        }

        const bool begins = at.tile == 0, whole = begins && seg == at.k.tiles;
        float *slot = slots + ((long long)blockIdx.x * 2 + (begins ? 1 : 0)) * Shape::FLOATS;
        if (begins && !whole && threadIdx.x == 0) {
            // the CTA with the unit's last place x: the largest i with all i / n_cta (rounded down) <= x
            const long long x = row_c0 + (long long)(at.unit + 1) * (at.k.tiles + begin) - 1;
            parts[blockIdx.x] = {row, at.unit, static_cast<int>(((x + 1) * n_cta - 1) / all), 0};
        }
        // the next unit's queries are requested before this one is finished
        left -= seg;
        if (left > begin) {
            left -= begin;
            at.tile = 0;
            if (++at.unit == units) {
                at.unit = 0;
                row_c0 += (long long)units * (at.k.tiles + begin);
                if (!step_row(at)) left = 0;
            }
            if (left > 0) load_q();
        } else {
            left = 0;
        }

        // the warps' results of the unit meet in shared memory, four products at a time: warp w joins product w
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float l_sum = run.l[nt];
            l_sum += __shfl_xor_sync(0xFFFFFFFFu, l_sum, 1);
            l_sum += __shfl_xor_sync(0xFFFFFFFFu, l_sum, 2);
            float c[PA_WARPS][2], m[2], l[2] = {0.f, 0.f};
#pragma unroll
            for (int hf = 0; hf < HF; ++hf) {
                __syncthreads();
                if (hf == 0 && t == 0) {
                    sm.m[warp][nt * 8 + g] = run.m[nt];
                    sm.l[warp][nt * 8 + g] = l_sum;
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float(&o)[4] = run.o[nt][hf * 4 + j];
                    sm.o[warp][j][lane] = make_float4(o[0], o[1], o[2], o[3]);
                }
                __syncthreads();
                if (hf == 0) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int h = nt * 8 + 2 * t + e;
                        m[e] = -INFINITY;
#pragma unroll
                        for (int w = 0; w < PA_WARPS; ++w) m[e] = fmaxf(m[e], sm.m[w][h]);
                        const float base = m[e] == -INFINITY ? 0.f : m[e];
#pragma unroll
                        for (int w = 0; w < PA_WARPS; ++w) {
                            c[w][e] = ex2_approx(sm.m[w][h] - base);
                            l[e] += sm.l[w][h] * c[w][e];
                        }
                    }
                }
                float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < PA_WARPS; ++w) {
                    const float4 x = sm.o[w][warp][lane];
                    o.x += x.x * c[w][0];
                    o.y += x.y * c[w][1];
                    o.z += x.z * c[w][0];
                    o.w += x.w * c[w][1];
                }
                const int j = hf * 4 + warp;
                if (whole) store_pair<HD>(p, row, h0, heads, nt, j, lane, o, l);
                else *reinterpret_cast<float4 *>(slot + ((nt * HF * 4 + j) * 32 + lane) * 4) = o;
            }
            if (warp == 0 && g == 0) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int h = nt * 8 + 2 * t + e;
                    if (!whole) {
                        slot[Shape::O_FLOATS + h] = m[e];
                        slot[Shape::O_FLOATS + HEADS + h] = l[e];
                    } else if (p.lse && h < heads) {
                        p.lse[row * p.lse_row + h0 + h] = lse_of(m[e], l[e]);
                    }
                }
            }
        }
    }
    // (nothing is under way here unless the lengths changed under the kernel)
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) {
        arrived(use, seen[i]);
        if (++use == STAGES) use = 0;
    }
    if (!BOXES) asm volatile("cp.async.wait_all;" ::: "memory");
    if (BOXES && *static_cast<volatile uint32_t *>(&sm.gave_up)) {
        for (int i = 0; i < 64; ++i) __nanosleep(10000);
        if (lane == 0 && p.status) atomicOr(p.status, STATUS_WAIT_LIMIT);
    }
    if (bad_page && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
}

// Joins the parts of the units that were split: out = sum_i o_i 2^(m_i - m) / sum_i l_i 2^(m_i - m).  A warp has one product
// (128 floats of every part) and takes BATCH parts at a time: what this kernel waits for is the way to L2 and back.
//   FEW = false  many units, of few parts each: CTA i joins the unit that begins in CTA i of the kernel above (if one does),
//                a warp per product;
//   FEW = true   few units, of many parts each: CTA (i, j) joins product j of unit i, whose beginning it looks for among the
//                parts; its warps share the parts.  (One sequence of 131072 keys, 55 parts a unit: 8 us with one CTA a unit.)
constexpr int JOIN_BATCH = 8, FEW_WARPS = 16;

template <int HD, int NT, bool FEW>
__global__ void __launch_bounds__(FEW ? FEW_WARPS * 32 : NT *PartShape<HD, NT>::PRODUCTS * 32)
paged_attn_join_kernel(const PagedAttnParams p, int n_cta) {
    constexpr int HEADS = 8 * NT, GROUPS = FEW ? FEW_WARPS : 1, BATCH = FEW ? JOIN_BATCH / 2 : JOIN_BATCH;
    using Shape = PartShape<HD, NT>;
    __shared__ float2 sm_m[GROUPS][32], sm_l[GROUPS][32];
    __shared__ float4 sm_o[GROUPS][32];
    __shared__ int sm_begin;
    pdl_wait();
    const Part *parts = reinterpret_cast<const Part *>(p.workspace);
    const int rep = p.n_head / p.c.n_kv_head, head_tiles = (rep + HEADS - 1) / HEADS, units = p.c.n_kv_head * head_tiles;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, group = FEW ? warp : 0, product = FEW ? blockIdx.y : warp;
    int begin = blockIdx.x;
    if (FEW) {
        if (threadIdx.x == 0) sm_begin = -1;
        __syncthreads();
        for (int i = threadIdx.x; i < n_cta; i += FEW_WARPS * 32)
            if (parts[i].row >= 0 && (long long)parts[i].row * units + parts[i].unit == blockIdx.x) sm_begin = i;
        __syncthreads();
        begin = sm_begin;
        if (begin < 0) return;
    }
    const Part part = parts[begin];
    if (part.row < 0) return;
    const int first = part.unit % head_tiles * HEADS, heads = min(HEADS, rep - first), h0 = part.unit / head_tiles * rep + first;
    const int nt = product / Shape::PRODUCTS, j = product % Shape::PRODUCTS, h = nt * 8 + 2 * (lane & 3);
    const float *slots = reinterpret_cast<const float *>(p.workspace + sizeof(Part) * n_cta);
    float2 m = make_float2(-INFINITY, -INFINITY), l = make_float2(0.f, 0.f);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    auto scale_to = [&](float mx, float my, float2 &base) {   // the sums so far go over to a larger maximum
        base = make_float2(mx == -INFINITY ? 0.f : mx, my == -INFINITY ? 0.f : my);
        const float ax = ex2_approx(m.x - base.x), ay = ex2_approx(m.y - base.y);
        m = make_float2(mx, my);
        l.x *= ax;
        l.y *= ay;
        o.x *= ax;
        o.y *= ay;
        o.z *= ax;
        o.w *= ay;
    };
    auto add = [&](const float2 base, const float2 mi, const float2 li, const float4 oi) {
        const float cx = ex2_approx(mi.x - base.x), cy = ex2_approx(mi.y - base.y);
        l.x += li.x * cx;
        l.y += li.y * cy;
        o.x += oi.x * cx;
        o.y += oi.y * cy;
        o.z += oi.z * cx;
        o.w += oi.w * cy;
    };
    for (int i0 = begin + group; i0 <= part.last_cta; i0 += GROUPS * BATCH) {
        float2 mi[BATCH], li[BATCH];
        float4 oi[BATCH];
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            const int i = i0 + b * GROUPS;
            mi[b] = make_float2(-INFINITY, -INFINITY);
            li[b] = make_float2(0.f, 0.f);
            oi[b] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i <= part.last_cta) {
                const float *slot = slots + ((long long)i * 2 + (i == begin ? 1 : 0)) * Shape::FLOATS;
                mi[b] = *reinterpret_cast<const float2 *>(slot + Shape::O_FLOATS + h);
                li[b] = *reinterpret_cast<const float2 *>(slot + Shape::O_FLOATS + HEADS + h);
                oi[b] = *reinterpret_cast<const float4 *>(slot + (product * 32 + lane) * 4);
            }
        }
        float mx = m.x, my = m.y;
#pragma unroll
        for (int b = 0; b < BATCH; ++b) {
            mx = fmaxf(mx, mi[b].x);
            my = fmaxf(my, mi[b].y);
        }
        float2 base;
        scale_to(mx, my, base);
#pragma unroll
        for (int b = 0; b < BATCH; ++b) add(base, mi[b], li[b], oi[b]);
    }
    if (GROUPS > 1) {
        sm_m[group][lane] = m;
        sm_l[group][lane] = l;
        sm_o[group][lane] = o;
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int w = 1; w < GROUPS; ++w) {
            const float2 mw = sm_m[w][lane];
            float2 base;
            scale_to(fmaxf(m.x, mw.x), fmaxf(m.y, mw.y), base);
            add(base, mw, sm_l[w][lane], sm_o[w][lane]);
        }
    }
    const float ls[2] = {l.x, l.y};
    store_pair<HD>(p, part.row, h0, heads, nt, j, lane, o, ls);
    if (p.lse && j == 0 && lane < 4) {
        if (h < heads) p.lse[part.row * p.lse_row + h0 + h] = lse_of(m.x, l.x);
        if (h + 1 < heads) p.lse[part.row * p.lse_row + h0 + h + 1] = lse_of(m.y, l.y);
    }
}

// CTAs of the grid: all that run at once, and no more than there can be tiles.
constexpr int MAX_CTAS_PER_SM = 4;

size_t workspace_bytes(int rep, int head_dim) {
    const int sms = sm_count() > 0 ? sm_count() : 148;
    const size_t heads = rep <= 8 ? 8 : 16;
    return (size_t)sms * MAX_CTAS_PER_SM * (sizeof(Part) + 2 * heads * ((head_dim + 63) / 64 * 64 + 2) * sizeof(float));
}

template <int HD, int NT, bool BOXES>
int launch_nt(const PagedAttnParams &p, const CUtensorMap &tm_k, const CUtensorMap &tm_v, cudaStream_t st) {
    static std::atomic<int> resident[MAX_DEVICES];   // CTAs of this instance that an SM of the device holds
    const int dev = device_slot(), sms = sm_count();
    if (dev < 0 || sms <= 0) return KRAKEN_ECUDA;
    int n = resident[dev].load(std::memory_order_relaxed);
    constexpr int SMEM = sizeof(Smem<HD, NT>) + 1024;
    if (n <= 0) {
        int rc = cuda_check(cudaFuncSetAttribute(paged_attn_kernel<HD, NT, BOXES>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM),
                            "paged attention: shared memory opt-in");
        if (!rc) rc = cuda_check(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, paged_attn_kernel<HD, NT, BOXES>, PA_WARPS * 32, SMEM),
                                 "paged attention: occupancy");
        if (rc) return rc;
        n = n < 1 ? 1 : (n > MAX_CTAS_PER_SM ? MAX_CTAS_PER_SM : n);
        resident[dev].store(n, std::memory_order_relaxed);
    }
    const int rep = p.n_head / p.c.n_kv_head;
    const long long units = (long long)p.c.n_kv_head * ((rep + 8 * NT - 1) / (8 * NT)) * p.rows;
    const long long keys = (long long)p.c.max_pages * p.c.page_size;
    const long long seen = p.window > 0 && p.window < keys ? p.window : keys;
    // (a window that begins inside a 16-key block touches up to 15 keys more)
    const long long tiles = std::min((keys + Step<HD>::TILE - 1) / Step<HD>::TILE, (seen + 15 + Step<HD>::TILE - 1) / Step<HD>::TILE);
    PagedAttnParams q = p;
    // nothing is split, and nothing joined, where the host knows that already (the kernel above sees to it where only the lengths say so)
    q.whole = tiles <= WHOLE_TILES && units <= (long long)sms * n;
    const long long grid = q.whole ? units : std::min<long long>((long long)sms * n, units * tiles);
    int rc = cuda_check(launch_pdl(paged_attn_kernel<HD, NT, BOXES>, dim3((unsigned)grid), dim3(PA_WARPS * 32), SMEM, st, tm_k, tm_v, q),
                        "paged attention: launch");
    if (rc || q.whole || tiles == 1) return rc;
    // fewer units than an eighth of the CTAs: over 8 parts each where the lengths are alike
    constexpr int PRODUCTS = NT * PartShape<HD, NT>::PRODUCTS;
    const bool few = units * JOIN_BATCH < grid;
    return cuda_check(few ? launch_pdl(paged_attn_join_kernel<HD, NT, true>, dim3((unsigned)units, PRODUCTS), dim3(FEW_WARPS * 32), 0, st, p,
                                       (int)grid)
                          : launch_pdl(paged_attn_join_kernel<HD, NT, false>, dim3((unsigned)grid), dim3(PRODUCTS * 32), 0, st, p, (int)grid),
                      "paged attention join: launch");
}

template <int HD>
int launch(const PagedAttnParams &p, cudaStream_t st) {
    const bool narrow = p.n_head / p.c.n_kv_head <= 8;
    CUtensorMap tm_k, tm_v;
    // Places of the cache that lie on one another (one head's keys for all, as an expanded tensor) are not a tensor map's: the lanes
    // copy.  A dimension of one may have any stride.
    const long long slot = p.c.page_size > 1 ? p.c.slot_stride : HD, head = p.c.n_kv_head > 1 ? p.c.head_stride : HD,
                    page = p.c.n_pages > 1 ? p.c.page_stride : HD;
    if (p.c.page_size % 8 == 0 && slot > 0 && head > 0 && page > 0) {
        const uint64_t dims[4] = {(uint64_t)HD, (uint64_t)p.c.page_size, (uint64_t)p.c.n_kv_head, (uint64_t)p.c.n_pages};
        const uint64_t strides[3] = {(uint64_t)slot, (uint64_t)head, (uint64_t)page};
        const uint32_t box[4] = {64, (uint32_t)p.box, 1, 1};
        // (strides that a tensor map cannot hold: the lanes copy)
        if (encode_tma_4d_bf16(&tm_k, p.c.k, dims, strides, box) == KRAKEN_OK &&
            encode_tma_4d_bf16(&tm_v, p.c.v, dims, strides, box) == KRAKEN_OK)
            return narrow ? launch_nt<HD, 1, true>(p, tm_k, tm_v, st) : launch_nt<HD, 2, true>(p, tm_k, tm_v, st);
    }
    memset(&tm_k, 0, sizeof(tm_k));
    return narrow ? launch_nt<HD, 1, false>(p, tm_k, tm_k, st) : launch_nt<HD, 2, false>(p, tm_k, tm_k, st);
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

}  // namespace kr

extern "C" int kraken_paged_attention_workspace(int32_t n_head, int32_t n_kv_head, int32_t head_dim, size_t *bytes) {
    using namespace kr;
    if (!bytes || n_head < 1 || n_kv_head < 1 || n_head % n_kv_head != 0) return KRAKEN_EINVAL;
    if (!decode_head_dim_ok(head_dim)) return KRAKEN_EUNSUPPORTED;
    *bytes = workspace_bytes(n_head / n_kv_head, head_dim);
    return KRAKEN_OK;
}

extern "C" int kraken_op_paged_attention(const kraken_paged_cache *cache, const kraken_paged_attention_args *a,
                                         uint32_t *d_status, void *stream) {
    using namespace kr;
    PagedAttnParams p;
    if (!a) return KRAKEN_EINVAL;
    int rc = paged_view(cache, &p.c);
    if (rc) return rc;
    if (a->rows == 0) return KRAKEN_OK;
    if (a->rows < 0 || !a->q || !a->out || !a->n_keys || a->n_head < 1 || a->n_head % cache->n_kv_head != 0 || a->window < 0 ||
        !isfinite(a->score_cap) || a->score_cap < 0.f)
        return KRAKEN_EINVAL;
    // (these two are factors in the kernel: a score of 0 times an infinite one would be a NaN)
    if (!isfinite(a->scale * LOG2E) || (a->score_cap > 0.f && !isfinite(1.f / a->score_cap))) return KRAKEN_EINVAL;
    if (!a->row_seq && a->rows > cache->n_seqs) return KRAKEN_EINVAL;
    // (no two rows or heads of the output in one place)
    if ((a->rows > 1 && a->out_row_stride == 0) || (a->n_head > 1 && a->out_head_stride == 0) ||
        (a->lse && a->rows > 1 && a->lse_row_stride == 0))
        return KRAKEN_EINVAL;
    if (!aligned16(a->q) || !aligned16(a->out) ||
        ((a->q_row_stride | a->q_head_stride | a->out_row_stride | a->out_head_stride) & 7))
        return KRAKEN_EUNSUPPORTED;
    // (the smallest tile has 64 keys)
    const long long capacity = (long long)cache->max_pages * cache->page_size;
    if (a->rows >= 1 << (63 - ROWS_AT) || a->rows * (capacity / 64 + 2) >= 1LL << ROWS_AT) return KRAKEN_EUNSUPPORTED;
    if (!a->workspace || a->workspace_bytes < workspace_bytes(a->n_head / cache->n_kv_head, cache->head_dim)) return KRAKEN_ECAPACITY;
    if (!aligned16(a->workspace)) return KRAKEN_EINVAL;
    p.workspace = static_cast<uint8_t *>(a->workspace);
    p.q = static_cast<const uint16_t *>(a->q);
    p.out = static_cast<uint16_t *>(a->out);
    p.lse = a->lse;
    p.row_seq = a->row_seq;
    p.n_keys = a->n_keys;
    p.slopes = a->slopes;
    p.q_row = a->q_row_stride;
    p.q_head = a->q_head_stride;
    p.out_row = a->out_row_stride;
    p.out_head = a->out_head_stride;
    p.lse_row = a->lse_row_stride;
    p.scale = a->scale;
    p.cap = a->score_cap;
    p.rows = a->rows;
    p.n_head = a->n_head;
    p.window = a->window;
    p.status = d_status;
    p.by_page = Divisor(cache->page_size);
    p.box = cache->page_size % 16 == 0 ? 16 : 8;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (cache->head_dim) {
        case 64: return launch<64>(p, st);
        case 72: return launch<72>(p, st);
        case 96: return launch<96>(p, st);
        case 104: return launch<104>(p, st);
        default: return launch<128>(p, st);
    }
}
