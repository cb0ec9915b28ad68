// Append of new tokens' keys and values to a cache in pages, with the rotation by position on the way.
//
//   K[page, h, slot] = R(p) k[r, h]     V[page, h, slot] = v[r, h]     q_out[r, h] = R(p) q[r, h]
//   R(p): the pair (a, b) number i of the first rot_dim elements -> (a cos t - b sin t, b cos t + a sin t), t = p f_i
//
// One pass: every value is read once and written once, so the floor is 4 bytes a value at the copy bandwidth.
#include "paged.cuh"

namespace kr {

namespace {

constexpr int MAX_HALF = 64;   // rot_dim <= head_dim <= 128

struct AppendParams {
    PagedView c;
    const uint16_t *k, *v, *q;
    uint16_t *q_out;
    long long k_row, k_head, v_row, v_head, q_row, q_head, qo_row, qo_head;
    const int *row_seq, *row_pos;
    const float *inv_freq;
    int rows, n_head, rot_dim, head_dim;
    uint32_t *status;
};

enum AppendForm { PAIRS_FAR_8, PAIRS_FAR_4, PAIRS_NEAR };   // (i, i + half) in pieces of 8 or 4 elements; (2i, 2i + 1)

// (cos, sin) of p * f.  The product has up to 55 significant bits and is formed and reduced in 64 bits, by whole turns
// subtracted in two pieces of 2 pi (Cody and Waite): an fp32 angle at position 10^6 would be off by 0.03.  What remains,
// at most pi, is rounded to fp32 (1.2e-7).
__device__ __forceinline__ float2 turn_of(int p, float f) {
    const double a = static_cast<double>(p) * static_cast<double>(f);
    const double n = rint(a * 0.15915494309189533577);              // 1 / (2 pi)
    double r = fma(n, -6.283185307179586477, a);
    r = fma(n, -2.4492935982947064e-16, r);                          // 2 pi minus its 64-bit rounding
    float2 cs;
    sincospif(static_cast<float>(r * 0.31830988618379067154), &cs.y, &cs.x);   // (in half turns: no far arguments to allow for)
    return cs;
}

// (a, b) -> (a cos - b sin, b cos + a sin) for two neighbouring pairs
__device__ __forceinline__ void turn_pairs(uint32_t &a, uint32_t &b, uint64_t c, uint64_t s, uint64_t minus_s) {
    const uint64_t x = pk2(h16_lo(a), h16_hi(a)), y = pk2(h16_lo(b), h16_hi(b));
    float lo, hi;
    upk2(fma2(x, c, mul2(y, minus_s)), lo, hi);
    a = pack_h16x2(lo, hi);
    upk2(fma2(y, c, mul2(x, s)), lo, hi);
    b = pack_h16x2(lo, hi);
}

// One CTA per row.  A thread has the same piece i of every head that it works on, so the piece's cosines and sines are in its
// registers and nothing is divided per piece, and the first AHEAD pieces of queries and keys, and again of values, are
// requested before the row's page is looked up and its angles are formed: what is read does not depend on where it goes.
//   64 threads, 4 pieces ahead    many rows: more rows side by side (four prompts, 6010 rows of 16 + 2 x 16 heads of 128: 25.8
//                                 against 26.1 us, an elementwise kernel over as many bytes 23.7)
//   128 threads, 2 pieces ahead   few rows: a row takes less time (one row of 32 + 2 x 8 heads: 2.2 against 2.7 us; 64 rows of
//                                 16 + 2 x 16 heads of 64: 1.8 against 2.1)
// (In a graph, on rotating inputs larger than L2 together; on one input over and over the prompts take 23.1 us.)  The 128-thread
// kernel for far pairs spills 20 bytes a thread: 3 of a warp's 550 instructions read them back.
// Tried: 256 threads that work each piece's head and place out (232 instructions a warp and piece: 31 us, bound by issue);
// CTAs that stay and request a row ahead (31 us: the registers of two rows halve the rows side by side).
template <AppendForm FORM, int THREADS, int AHEAD>
__global__ void __launch_bounds__(THREADS, THREADS == 64 ? 10 : 7) paged_append_kernel(const AppendParams p) {
    constexpr int W = FORM == PAIRS_FAR_4 ? 4 : 8;        // elements of a rotated piece (of each of the two with PAIRS_FAR)
    constexpr int PAIRS = FORM == PAIRS_FAR_8 ? 8 : 4;    // pairs that a thread turns
    __shared__ __align__(16) float cosines[MAX_HALF], sines[MAX_HALF];
    pdl_wait();
    const int tid = threadIdx.x, half = p.rot_dim / 2;
    const long long r = blockIdx.x;
    const int seq = p.row_seq ? p.row_seq[r] : static_cast<int>(r), pos = p.row_pos[r];
    const float freq = tid < half ? p.inv_freq[tid] : 0.f;

    // queries and keys: pieces that are rotated, then pieces that are copied; values: copied
    const int turned = FORM == PAIRS_NEAR ? p.rot_dim / 8 : half / W;
    const int units = turned + (p.head_dim - p.rot_dim) / 8, whole = p.head_dim / 8;
    const int n_q = p.q ? p.n_head : 0, n_kv = p.c.n_kv_head, n_qk = n_q + n_kv;
    const int step_qk = THREADS / units, step_v = THREADS / whole;    // heads that the CTA works on side by side
    const int i_qk = tid % units, h_qk = tid < step_qk * units ? tid / units : n_qk;
    const int i_v = tid % whole, h_v = tid < step_v * whole ? tid / whole : n_kv;
    const bool turns = i_qk < turned;
    const int e_qk = turns ? i_qk * W : p.rot_dim + (i_qk - turned) * 8;      // first element of the piece

    struct Piece {
        uint4 a, b;   // the two halves of the pairs (8 bytes of each with W = 4), or the piece and nothing
    };
    auto load_qk = [&](Piece &x, int h) {
        const uint16_t *src = (h < n_q ? p.q + r * p.q_row + h * p.q_head : p.k + r * p.k_row + (h - n_q) * p.k_head) + e_qk;
        if (FORM == PAIRS_FAR_4 && turns) {
            const uint2 a = __ldcs(reinterpret_cast<const uint2 *>(src)), b = __ldcs(reinterpret_cast<const uint2 *>(src + half));
            x.a = make_uint4(a.x, a.y, 0u, 0u);
            x.b = make_uint4(b.x, b.y, 0u, 0u);
        } else {
            x.a = __ldcs(reinterpret_cast<const uint4 *>(src));
            if (FORM == PAIRS_FAR_8 && turns) x.b = __ldcs(reinterpret_cast<const uint4 *>(src + half));
        }
    };
    auto load_v = [&](uint4 &x, int h) {
        x = __ldcs(reinterpret_cast<const uint4 *>(p.v + r * p.v_row + h * p.v_head + i_v * 8));
    };
    Piece qk[AHEAD];
    uint4 v[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        if (h_qk + j * step_qk < n_qk) load_qk(qk[j], h_qk + j * step_qk);
        if (h_v + j * step_v < n_kv) load_v(v[j], h_v + j * step_v);
    }
    if (seq < 0) return;
    int page = -1, slot = 0;
    if (seq < p.c.n_seqs && pos >= 0) {
        const int n = pos / p.c.page_size;
        slot = pos - n * p.c.page_size;
        if (n < p.c.max_pages) page = p.c.table[seq * p.c.table_stride + n];
    }
    if (tid < half) {
        const float2 t = turn_of(pos, freq);
        cosines[tid] = t.x;
        sines[tid] = t.y;
    }
    __syncthreads();
    if (page < 0 || page >= p.c.n_pages) {
        if (tid == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
        return;
    }
    const long long at = page * p.c.page_stride + slot * p.c.slot_stride;
    float c[PAIRS], s[PAIRS];
    if (turns) {
#pragma unroll
        for (int j = 0; j < PAIRS; j += 4) {
            *reinterpret_cast<float4 *>(c + j) = *reinterpret_cast<const float4 *>(&cosines[i_qk * PAIRS + j]);
            *reinterpret_cast<float4 *>(s + j) = *reinterpret_cast<const float4 *>(&sines[i_qk * PAIRS + j]);
        }
    }
    auto store_qk = [&](Piece y, int h) {
        uint16_t *dst = (h < n_q ? p.q_out + r * p.qo_row + h * p.qo_head : p.c.k + at + (h - n_q) * p.c.head_stride) + e_qk;
        uint32_t a[4] = {y.a.x, y.a.y, y.a.z, y.a.w}, b[4] = {y.b.x, y.b.y, y.b.z, y.b.w};
        if (!turns) {
            *reinterpret_cast<uint4 *>(dst) = y.a;
        } else if (FORM == PAIRS_NEAR) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float lo = h16_lo(a[j]), hi = h16_hi(a[j]);
                a[j] = pack_h16x2(lo * c[j] - hi * s[j], hi * c[j] + lo * s[j]);
            }
            *reinterpret_cast<uint4 *>(dst) = make_uint4(a[0], a[1], a[2], a[3]);
        } else {
#pragma unroll
            for (int j = 0; j < W / 2; ++j)
                turn_pairs(a[j], b[j], pk2(c[2 * j], c[2 * j + 1]), pk2(s[2 * j], s[2 * j + 1]), pk2(-s[2 * j], -s[2 * j + 1]));
            if (W == 8) {
                *reinterpret_cast<uint4 *>(dst) = make_uint4(a[0], a[1], a[2], a[3]);
                *reinterpret_cast<uint4 *>(dst + half) = make_uint4(b[0], b[1], b[2], b[3]);
            } else {
                *reinterpret_cast<uint2 *>(dst) = make_uint2(a[0], a[1]);
                *reinterpret_cast<uint2 *>(dst + half) = make_uint2(b[0], b[1]);
            }
        }
    };
    auto store_v = [&](const uint4 &y, int h) {
        *reinterpret_cast<uint4 *>(p.c.v + at + h * p.c.head_stride + i_v * 8) = y;
    };
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        if (h_qk + j * step_qk < n_qk) store_qk(qk[j], h_qk + j * step_qk);
        if (h_v + j * step_v < n_kv) store_v(v[j], h_v + j * step_v);
    }
    for (int h = h_qk + AHEAD * step_qk; h < n_qk; h += step_qk) {
        Piece y;
        load_qk(y, h);
        store_qk(y, h);
    }
    for (int h = h_v + AHEAD * step_v; h < n_kv; h += step_v) {
        uint4 y;
        load_v(y, h);
        store_v(y, h);
    }
}

template <AppendForm FORM>
cudaError_t launch(const AppendParams &p, cudaStream_t st) {
    const int sms = sm_count() > 0 ? sm_count() : 148;
    return p.rows >= 4 * sms ? launch_pdl(paged_append_kernel<FORM, 64, 4>, dim3(p.rows), dim3(64), 0, st, p)
                             : launch_pdl(paged_append_kernel<FORM, 128, 2>, dim3(p.rows), dim3(128), 0, st, p);
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace

}  // namespace kr

extern "C" int kraken_op_paged_append(const kraken_paged_cache *cache, const kraken_paged_append_args *a,
                                      uint32_t *d_status, void *stream) {
    using namespace kr;
    AppendParams p;
    if (!a) return KRAKEN_EINVAL;
    int rc = paged_view(cache, &p.c);
    if (rc) return rc;
    if (a->rows == 0) return KRAKEN_OK;
    if (a->rows < 0 || !a->k || !a->v || !a->row_pos || a->rot_dim < 0 || (a->rot_dim > 0 && !a->inv_freq) ||
        (a->q && (!a->q_out || a->n_head < 1)))
        return KRAKEN_EINVAL;
    if (!a->row_seq && a->rows > cache->n_seqs) return KRAKEN_EINVAL;
    // (no two places of the cache, rows or heads of q_out in one place)
    if ((cache->n_pages > 1 && cache->page_stride == 0) || (cache->n_kv_head > 1 && cache->head_stride == 0) ||
        (cache->page_size > 1 && cache->slot_stride == 0) ||
        (a->q && ((a->rows > 1 && a->q_out_row_stride == 0) || (a->n_head > 1 && a->q_out_head_stride == 0))))
        return KRAKEN_EINVAL;
    if (a->rot_dim % 8 != 0 || a->rot_dim > cache->head_dim) return KRAKEN_EUNSUPPORTED;
    if (!aligned16(a->k) || !aligned16(a->v) || ((a->k_row_stride | a->k_head_stride | a->v_row_stride | a->v_head_stride) & 7))
        return KRAKEN_EUNSUPPORTED;
    if (a->q && (!aligned16(a->q) || !aligned16(a->q_out) ||
                 ((a->q_row_stride | a->q_head_stride | a->q_out_row_stride | a->q_out_head_stride) & 7)))
        return KRAKEN_EUNSUPPORTED;
    p.k = static_cast<const uint16_t *>(a->k);
    p.v = static_cast<const uint16_t *>(a->v);
    p.q = static_cast<const uint16_t *>(a->q);
    p.q_out = static_cast<uint16_t *>(a->q_out);
    p.k_row = a->k_row_stride;
    p.k_head = a->k_head_stride;
    p.v_row = a->v_row_stride;
    p.v_head = a->v_head_stride;
    p.q_row = a->q_row_stride;
    p.q_head = a->q_head_stride;
    p.qo_row = a->q_out_row_stride;
    p.qo_head = a->q_out_head_stride;
    p.row_seq = a->row_seq;
    p.row_pos = a->row_pos;
    p.inv_freq = a->inv_freq;
    p.rows = a->rows;
    p.n_head = a->n_head;
    p.rot_dim = a->rot_dim;
    p.head_dim = cache->head_dim;
    p.status = d_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (a->interleaved || a->rot_dim == 0) e = launch<PAIRS_NEAR>(p, st);
    else if (a->rot_dim % 16 == 0) e = launch<PAIRS_FAR_8>(p, st);
    else e = launch<PAIRS_FAR_4>(p, st);
    return cuda_check(e, "paged append: launch");
}
