// Decode-step attention over a key/value cache in pages: one query per head and row against the cached keys of the
// row's sequence, which the page table leads to.
//
//   x_j = scale q.k_j  [cap tanh(x/cap)]  [+ slope (j - (n - 1))],  out = sum_j softmax(x)_j v_j,  lse = log sum_j e^x_j
//
// Every key and value is used by the n_head / n_kv_head query heads that share it and read once: 4 bytes a key element
// against 4 FLOP per query head, so up to 16 heads a group this is bound by HBM (16 FLOP a byte: 100 TFLOP/s at the copy
// bandwidth) and the products run on the warp-level tensor instructions, which take both operands from registers.
//
// The products of a 16-key block, with the keys as rows and the query heads as the 8 columns (m16n8k16):
//   S^T[key, head] = K Q^T    a lane reads 16 bytes (8 consecutive elements) of a key and feeds them to two products; Q is
//                             held with the same order of elements in the k slots, which is all a dot product needs
//   O^T[e, head] += V^T P^T   a lane reads 16 bytes of four keys and pairs neighbouring keys by byte permutes; rows g and
//                             g + 8 of product j stand for elements 8 g + 2 j and 8 g + 2 j + 1, so a lane ends with
//                             8 consecutive elements of two heads.  P^T gets from the accumulator layout to the operand
//                             layout by a transposing 8 x 8 move inside the warp.
// P goes into the product as the sum of two 16-bit numbers (its rounding and the rounding of the rest), so its rounding,
// which would be as large as that of the output, does not count; a running maximum and sum are kept in fp32.
#include <math.h>

#include <algorithm>

#include "paged.cuh"

namespace kr {

namespace {

constexpr int PA_WARPS = 4;
constexpr int TILE = PA_WARPS * 16;   // keys of a tile: 16 for every warp
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.69314718055994531f;

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
};

__device__ __forceinline__ void mma_keys(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32." KRAKEN_MMA_T "." KRAKEN_MMA_T ".f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// The 16-key block at key0 of one (sequence, key/value head) as a lane holds it: keys g and g + 8 of K, keys 2t, 2t + 1,
// 2t + 8, 2t + 9 of V (g = lane / 4, t = lane % 4).
template <int HD>
struct KeyBlock {
    static constexpr int CH = (HD + 31) / 32;   // 32-element chunks of a key, 8 elements of each per lane
    static constexpr int HF = (HD + 63) / 64;   // 64-element halves of a value, 8 elements of each per lane
    uint4 k[2][CH], v[4][HF];
};

template <int HD, int NT>
struct Running {   // online softmax of 8 NT heads over the keys of one warp; heads 8 nt + 2t + {0, 1} per lane
    static constexpr int HF = KeyBlock<HD>::HF;
    float m[NT][2], l[NT][2];       // maximum in use (log2 domain), this lane's part of the sum
    float o[NT][HF * 4][4];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = 0.f;
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

// `live[i]`: whether key g + 8 i of the block is visible; `back`: position of key g minus that of the query
template <int HD, int NT>
__device__ __forceinline__ void take_block(Running<HD, NT> &run, const KeyBlock<HD> &b, const uint4 (&q)[NT][KeyBlock<HD>::CH],
                                           const bool (&live)[2], int back, const ScoreForm &f, const float (&slope)[NT][2]) {
    constexpr int CH = KeyBlock<HD>::CH, HF = KeyBlock<HD>::HF;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            mma_keys(s, b.k[0][c].x, b.k[1][c].x, b.k[0][c].y, b.k[1][c].y, q[nt][c].x, q[nt][c].y);
            mma_keys(s, b.k[0][c].z, b.k[1][c].z, b.k[0][c].w, b.k[1][c].w, q[nt][c].z, q[nt][c].w);
        }
        // s[2 i + e]: key g + 8 i, head 2t + e
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float x = s[i];
            if (f.plain) {
                x *= f.scale2;
            } else {
                x *= f.scale;
                if (f.cap > 0.f) x = f.cap * tanhf(x * f.inv_cap);
                x = (x + slope[nt][i & 1] * static_cast<float>(back + (i >> 1) * 8)) * LOG2E;
            }
            s[i] = live[i >> 1] ? x : -INFINITY;
        }
        float p[4];
        bool moved = false;
        float corr[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            float mx = fmaxf(s[e], s[2 + e]);
            mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
            mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
            mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
            mx = fmaxf(mx, run.m[nt][e]);
            const float base = mx == -INFINITY ? 0.f : mx;   // nothing visible yet: every weight is 2^-inf = 0
            corr[e] = ex2_approx(run.m[nt][e] - base);
            moved |= mx != run.m[nt][e];
            run.m[nt][e] = mx;
            p[e] = ex2_approx(s[e] - base);
            p[2 + e] = ex2_approx(s[2 + e] - base);
            run.l[nt][e] = run.l[nt][e] * corr[e] + (p[e] + p[2 + e]);
        }
        if (__any_sync(0xFFFFFFFFu, moved)) {
#pragma unroll
            for (int j = 0; j < HF * 4; ++j) {
                run.o[nt][j][0] *= corr[0];
                run.o[nt][j][1] *= corr[1];
                run.o[nt][j][2] *= corr[0];
                run.o[nt][j][3] *= corr[1];
            }
        }
        uint32_t hi[2], lo[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t w = pack_h16x2(p[2 * i], p[2 * i + 1]);
            hi[i] = transpose_8x8(w);
            lo[i] = transpose_8x8(pack_h16x2(p[2 * i] - h16_lo(w), p[2 * i + 1] - h16_hi(w)));
        }
#pragma unroll
        for (int hf = 0; hf < HF; ++hf)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t v0 = word(b.v[0][hf], j), v1 = word(b.v[1][hf], j), v2 = word(b.v[2][hf], j), v3 = word(b.v[3][hf], j);
                const uint32_t a0 = __byte_perm(v0, v1, 0x5410), a1 = __byte_perm(v0, v1, 0x7632);
                const uint32_t a2 = __byte_perm(v2, v3, 0x5410), a3 = __byte_perm(v2, v3, 0x7632);
                mma_keys(run.o[nt][hf * 4 + j], a0, a1, a2, a3, hi[0], hi[1]);
                mma_keys(run.o[nt][hf * 4 + j], a0, a1, a2, a3, lo[0], lo[1]);
            }
    }
}

// What row r asks for: its visible keys lo .. n - 1 of sequence seq.  False: padding, or (bad) no such sequence or length.
struct RowKeys {
    int seq, lo, n, tiles;   // tiles of TILE keys, at least one (a row without keys writes zeros)
};

__device__ __forceinline__ bool row_keys(const PagedAttnParams &p, int r, RowKeys &k, bool &bad) {
    k.seq = p.row_seq ? p.row_seq[r] : r;
    k.tiles = 0;
    if (k.seq < 0) return false;
    k.n = p.n_keys[r];
    if (k.seq >= p.c.n_seqs || k.n < 0 || k.n > (long long)p.c.max_pages * p.c.page_size) {
        bad = true;
        return false;
    }
    k.lo = p.window > 0 && k.n > p.window ? k.n - p.window : 0;
    k.tiles = max(1, (k.n - k.lo + TILE - 1) / TILE);
    return true;
}

// The work of a call is a line of tiles: rows in order, of each row its (key/value head, head tile) units in order, of each
// unit its key tiles.  CTA i of G (at most one per tile) takes tiles [total i / G, total (i + 1) / G): the same number for every CTA, whatever the
// lengths.  A unit that lies in one CTA is finished there; of one that does not, every CTA leaves its part in the
// workspace (slot 1 where the unit begins, slot 0 elsewhere: a CTA has at most one of each) and the CTA with the
// beginning notes who has the rest, for the joining kernel.
struct Part {
    int row, unit, last_cta;   // row = -1: nothing to join
    int pad;
};

template <int HD, int NT>
struct PartShape {
    static constexpr int HEADS = 8 * NT;
    static constexpr int FLOATS = HEADS * (HD + 2);   // [HEADS] m, [HEADS] l, [HEADS][HD] o
};

template <int HD, int NT>
__global__ void __launch_bounds__(PA_WARPS * 32) paged_attn_kernel(const PagedAttnParams p) {
    constexpr int CH = KeyBlock<HD>::CH, HF = KeyBlock<HD>::HF, HEADS = 8 * NT;
    __shared__ float sm_m[PA_WARPS][HEADS], sm_l[PA_WARPS][HEADS];
    __shared__ float sm_o[PA_WARPS][HEADS][HF * 64];
    __shared__ long long sm_sum[PA_WARPS];
    __shared__ int sm_row;
    __shared__ long long sm_before;
    pdl_wait();
    const int rep = p.n_head / p.c.n_kv_head;
    const int head_tiles = (rep + HEADS - 1) / HEADS;
    const int units = p.c.n_kv_head * head_tiles;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    Part *parts = reinterpret_cast<Part *>(p.workspace);
    float *slots = reinterpret_cast<float *>(p.workspace + sizeof(Part) * gridDim.x);
    if (threadIdx.x == 0) {
        parts[blockIdx.x].row = -1;
        sm_row = -1;
    }

    // where this CTA's share begins: every thread adds up the tiles of a run of rows
    const int per = (p.rows + PA_WARPS * 32 - 1) / (PA_WARPS * 32);
    const int row_lo = min(p.rows, (int)threadIdx.x * per), row_hi = min(p.rows, row_lo + per);
    long long mine = 0;
    bool bad = false;
    for (int r = row_lo; r < row_hi; ++r) {
        RowKeys k;
        row_keys(p, r, k, bad);
        mine += k.tiles;
    }
    long long upto = mine;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long v = __shfl_up_sync(0xFFFFFFFFu, upto, off);
        if (lane >= off) upto += v;
    }
    if (lane == 31) sm_sum[warp] = upto;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < PA_WARPS; ++w) {
        if (w < warp) upto += sm_sum[w];
        total += sm_sum[w];
    }
    const long long all = total * units;
    const long long n_cta = min((long long)gridDim.x, all);   // no CTA between the two ends of a unit is without a tile
    const long long c0 = blockIdx.x < n_cta ? all * blockIdx.x / n_cta : all;
    const long long c1 = blockIdx.x < n_cta ? all * (blockIdx.x + 1) / n_cta : all;
    {
        long long before = upto - mine;
        if (c0 < c1 && c0 >= before * units && c0 < upto * units) {
            for (int r = row_lo; r < row_hi; ++r) {
                RowKeys k;
                row_keys(p, r, k, bad);
                if (c0 < (before + k.tiles) * units) {
                    sm_row = r;
                    sm_before = before;
                    break;
                }
                before += k.tiles;
            }
        }
    }
    if (bad && blockIdx.x == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
    if (c0 >= c1) return;
    __syncthreads();

    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
    const ScoreForm form = {p.scale, p.cap, p.cap > 0.f ? 1.f / p.cap : 0.f, p.cap <= 0.f && !p.slopes, p.scale * LOG2E};
    int r = sm_row;
    RowKeys k;
    // (no such row, here and below: the lengths changed under the kernel)
    if (r < 0 || !row_keys(p, r, k, bad)) return;
    long long row_c0 = sm_before * units;          // first tile of row r
    int unit = static_cast<int>((c0 - row_c0) / k.tiles);
    int tile = static_cast<int>((c0 - row_c0) % k.tiles);
    long long left = c1 - c0;
    bool bad_page = false;
    while (left > 0) {
        const int seg = static_cast<int>(min(left, (long long)(k.tiles - tile)));
        const int hk = unit / head_tiles, first = unit % head_tiles * HEADS;
        const int heads = min(HEADS, rep - first), h0 = hk * rep + first;
        const int *table = p.c.table + k.seq * p.c.table_stride;
        uint4 q[NT][CH];
        float slope[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int h = nt * 8 + g, e = c * 32 + t * 8;
                q[nt][c] = h < heads && e < HD ? *reinterpret_cast<const uint4 *>(p.q + r * p.q_row + (h0 + h) * p.q_head + e) : zero;
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int h = nt * 8 + 2 * t + e;
                slope[nt][e] = p.slopes && h < heads ? p.slopes[h0 + h] : 0.f;
            }
        }
        Running<HD, NT> run;
        run.clear();
        const int end = min((long long)k.n, k.lo + (long long)(tile + seg) * TILE);
        for (int key0 = k.lo + tile * TILE + warp * 16; key0 < end; key0 += TILE) {
            // lanes 0..15 look up the page of one key each; -1: not visible
            const int key = key0 + (lane & 15);
            int page = -1;
            if (key < end) {
                page = table[key / p.c.page_size];
                if (page < 0 || page >= p.c.n_pages) {
                    page = -1;
                    bad_page = true;
                }
            }
            const int slot = key % p.c.page_size;
            KeyBlock<HD> b;
            bool live[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int pg = __shfl_sync(0xFFFFFFFFu, page, g + 8 * i), sl = __shfl_sync(0xFFFFFFFFu, slot, g + 8 * i);
                live[i] = pg >= 0;
                const uint16_t *row = p.c.k + pg * p.c.page_stride + sl * p.c.slot_stride + hk * p.c.head_stride;
#pragma unroll
                for (int c = 0; c < CH; ++c)
                    b.k[i][c] = live[i] && c * 32 + t * 8 < HD ? __ldcs(reinterpret_cast<const uint4 *>(row + c * 32 + t * 8)) : zero;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int who = 2 * t + (i & 1) + (i >> 1) * 8;
                const int pg = __shfl_sync(0xFFFFFFFFu, page, who), sl = __shfl_sync(0xFFFFFFFFu, slot, who);
                const uint16_t *row = p.c.v + pg * p.c.page_stride + sl * p.c.slot_stride + hk * p.c.head_stride;
#pragma unroll
                for (int hf = 0; hf < HF; ++hf)
                    b.v[i][hf] = pg >= 0 && hf * 64 + g * 8 < HD ? __ldcs(reinterpret_cast<const uint4 *>(row + hf * 64 + g * 8)) : zero;
            }
            take_block<HD, NT>(run, b, q, live, key0 + g - (k.n - 1), form, slope);
        }

        // sums over the lanes that hold the same heads; then the warps through shared memory
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float l = run.l[nt][e];
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 4);
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 8);
                l += __shfl_xor_sync(0xFFFFFFFFu, l, 16);
                const int h = nt * 8 + 2 * t + e;
                if (g == 0) {
                    sm_m[warp][h] = run.m[nt][e];
                    sm_l[warp][h] = l;
                }
#pragma unroll
                for (int hf = 0; hf < HF; ++hf)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        sm_o[warp][h][hf * 64 + g * 8 + 2 * j] = run.o[nt][hf * 4 + j][e];
                        sm_o[warp][h][hf * 64 + g * 8 + 2 * j + 1] = run.o[nt][hf * 4 + j][2 + e];
                    }
            }
        __syncthreads();
        const bool whole = tile == 0 && seg == k.tiles;
        float *slot = slots + ((long long)blockIdx.x * 2 + (tile == 0 ? 1 : 0)) * PartShape<HD, NT>::FLOATS;
        for (int i = threadIdx.x; i < heads * HD; i += PA_WARPS * 32) {
            const int h = i / HD, e = i % HD;
            float m = -INFINITY;
#pragma unroll
            for (int w = 0; w < PA_WARPS; ++w) m = fmaxf(m, sm_m[w][h]);
            const float base = m == -INFINITY ? 0.f : m;
            float l = 0.f, o = 0.f;
#pragma unroll
            for (int w = 0; w < PA_WARPS; ++w) {
                const float c = ex2_approx(sm_m[w][h] - base);
                l += sm_l[w][h] * c;
                o += sm_o[w][h][e] * c;
            }
            if (whole) {
                p.out[r * p.out_row + (h0 + h) * p.out_head + e] = to_h16(l == 0.f ? 0.f : o / l);
                if (p.lse && e == 0) p.lse[r * p.lse_row + h0 + h] = l == 0.f ? -INFINITY : (m + log2f(l)) * LN2;
            } else {
                slot[2 * HEADS + i] = o;
                if (e == 0) {
                    slot[h] = m;
                    slot[HEADS + h] = l;
                }
            }
        }
        if (tile == 0 && !whole && threadIdx.x == 0) {
            // the CTA with the unit's last tile x: the largest i with all i / n_cta (rounded down) <= x
            const long long x = row_c0 + (long long)(unit + 1) * k.tiles - 1;
            parts[blockIdx.x] = {r, unit, static_cast<int>(((x + 1) * n_cta - 1) / all), 0};
        }
        left -= seg;
        tile = 0;
        if (++unit == units && left > 0) {
            unit = 0;
            row_c0 += (long long)units * k.tiles;
            do {
                if (++r == p.rows) {
                    left = 0;
                    break;
                }
                row_keys(p, r, k, bad);
            } while (k.tiles == 0);
        }
        __syncthreads();
    }
    if (bad_page && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
}

// Joins the parts of the unit that begins in CTA blockIdx.x of the kernel above, head blockIdx.y of it:
// out = sum_i o_i 2^(m_i - m) / sum_i l_i 2^(m_i - m).  A warp takes every 8th part, a lane 4 elements of the head.
constexpr int JOIN_WARPS = 8;

template <int HD, int NT>
__global__ void __launch_bounds__(JOIN_WARPS * 32) paged_attn_join_kernel(const PagedAttnParams p, int n_cta) {
    constexpr int HEADS = 8 * NT;
    __shared__ float sm_m[JOIN_WARPS], sm_l[JOIN_WARPS];
    __shared__ float4 sm_o[JOIN_WARPS][32];
    pdl_wait();
    const Part part = reinterpret_cast<const Part *>(p.workspace)[blockIdx.x];
    if (part.row < 0) return;
    const int rep = p.n_head / p.c.n_kv_head, head_tiles = (rep + HEADS - 1) / HEADS;
    const int hk = part.unit / head_tiles, first = part.unit % head_tiles * HEADS, h = blockIdx.y;
    if (first + h >= rep) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float *slots = reinterpret_cast<const float *>(p.workspace + sizeof(Part) * n_cta);
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i = blockIdx.x + warp; i <= part.last_cta; i += JOIN_WARPS) {
        const float *slot = slots + ((long long)i * 2 + (i == (int)blockIdx.x ? 1 : 0)) * PartShape<HD, NT>::FLOATS;
        const float mi = slot[h], li = slot[HEADS + h];
        const float4 oi = lane * 4 < HD ? *reinterpret_cast<const float4 *>(slot + 2 * HEADS + h * HD + lane * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
        const float mx = fmaxf(m, mi), base = mx == -INFINITY ? 0.f : mx;
        const float a = ex2_approx(m - base), b = ex2_approx(mi - base);
        m = mx;
        l = l * a + li * b;
        o.x = o.x * a + oi.x * b;
        o.y = o.y * a + oi.y * b;
        o.z = o.z * a + oi.z * b;
        o.w = o.w * a + oi.w * b;
    }
    if (lane == 0) {
        sm_m[warp] = m;
        sm_l[warp] = l;
    }
    sm_o[warp][lane] = o;
    __syncthreads();
    if (warp != 0) return;
    float mx = -INFINITY;
#pragma unroll
    for (int w = 0; w < JOIN_WARPS; ++w) mx = fmaxf(mx, sm_m[w]);
    const float base = mx == -INFINITY ? 0.f : mx;
    l = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < JOIN_WARPS; ++w) {
        const float c = ex2_approx(sm_m[w] - base);
        const float4 ow = sm_o[w][lane];
        l += sm_l[w] * c;
        o.x += ow.x * c;
        o.y += ow.y * c;
        o.z += ow.z * c;
        o.w += ow.w * c;
    }
    const int head = hk * rep + first + h;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (lane * 4 < HD) {
        uint2 u;
        u.x = pack_h16x2(o.x * inv, o.y * inv);
        u.y = pack_h16x2(o.z * inv, o.w * inv);
        *reinterpret_cast<uint2 *>(p.out + part.row * p.out_row + head * p.out_head + lane * 4) = u;
    }
    if (p.lse && lane == 0) p.lse[part.row * p.lse_row + head] = l == 0.f ? -INFINITY : (mx + log2f(l)) * LN2;
}

// CTAs of the grid: all that run at once, and no more than there can be tiles.
constexpr int MAX_CTAS_PER_SM = 4;

size_t workspace_bytes(int rep, int head_dim) {
    const int sms = sm_count() > 0 ? sm_count() : 148;
    const size_t heads = rep <= 8 ? 8 : 16;
    return (size_t)sms * MAX_CTAS_PER_SM * (sizeof(Part) + 2 * heads * (head_dim + 2) * sizeof(float));
}

template <int HD, int NT>
int launch_nt(const PagedAttnParams &p, cudaStream_t st) {
    static std::atomic<int> resident[MAX_DEVICES];   // CTAs of this instance that an SM of the device holds
    const int dev = device_slot(), sms = sm_count();
    if (dev < 0 || sms <= 0) return KRAKEN_ECUDA;
    int n = resident[dev].load(std::memory_order_relaxed);
    if (n <= 0) {
        int rc = cuda_check(cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, paged_attn_kernel<HD, NT>, PA_WARPS * 32, 0),
                            "paged attention: occupancy");
        if (rc) return rc;
        n = n < 1 ? 1 : (n > MAX_CTAS_PER_SM ? MAX_CTAS_PER_SM : n);
        resident[dev].store(n, std::memory_order_relaxed);
    }
    const int rep = p.n_head / p.c.n_kv_head;
    const long long units = (long long)p.c.n_kv_head * ((rep + 8 * NT - 1) / (8 * NT)) * p.rows;
    const long long keys = (long long)p.c.max_pages * p.c.page_size;
    const long long seen = p.window > 0 && p.window < keys ? p.window : keys;
    const long long tiles = (seen + TILE - 1) / TILE;
    const long long grid = std::min<long long>((long long)sms * n, units * tiles);
    int rc = cuda_check(launch_pdl(paged_attn_kernel<HD, NT>, dim3((unsigned)grid), dim3(PA_WARPS * 32), 0, st, p),
                        "paged attention: launch");
    // with one tile a unit nothing is ever split
    if (rc || tiles == 1) return rc;
    return cuda_check(launch_pdl(paged_attn_join_kernel<HD, NT>, dim3((unsigned)grid, std::min(rep, 8 * NT)), dim3(JOIN_WARPS * 32), 0,
                                 st, p, (int)grid), "paged attention join: launch");
}

template <int HD>
int launch(const PagedAttnParams &p, cudaStream_t st) {
    return p.n_head / p.c.n_kv_head <= 8 ? launch_nt<HD, 1>(p, st) : launch_nt<HD, 2>(p, st);
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
        !isfinite(a->scale) || !isfinite(a->score_cap) || a->score_cap < 0.f)
        return KRAKEN_EINVAL;
    if (!a->row_seq && a->rows > cache->n_seqs) return KRAKEN_EINVAL;
    if (!aligned16(a->q) || !aligned16(a->out) ||
        ((a->q_row_stride | a->q_head_stride | a->out_row_stride | a->out_head_stride) & 7))
        return KRAKEN_EUNSUPPORTED;
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
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (cache->head_dim) {
        case 64: return launch<64>(p, st);
        case 72: return launch<72>(p, st);
        case 96: return launch<96>(p, st);
        case 104: return launch<104>(p, st);
        default: return launch<128>(p, st);
    }
}
