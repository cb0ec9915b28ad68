// Append of new tokens' keys and values to a cache in pages, with the rotation by position on the way.
//
//   K[page, h, slot] = R(p) k[r, h]     V[page, h, slot] = v[r, h]     q_out[r, h] = R(p) q[r, h]
//   R(p): the pair (a, b) number i of the first rot_dim elements -> (a cos t - b sin t, b cos t + a sin t), t = p f_i
//
// One pass: every value is read once and written once, so the floor is 4 bytes a value at the copy bandwidth.
#include "paged.cuh"

namespace kr {

namespace {

constexpr int APP_THREADS = 256;
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
    sincosf(static_cast<float>(r), &cs.y, &cs.x);
    return cs;
}

__device__ __forceinline__ void turn_pair(uint32_t &a, uint32_t &b, const float2 lo, const float2 hi) {
    const float a0 = h16_lo(a), a1 = h16_hi(a), b0 = h16_lo(b), b1 = h16_hi(b);
    a = pack_h16x2(a0 * lo.x - b0 * lo.y, a1 * hi.x - b1 * hi.y);
    b = pack_h16x2(b0 * lo.x + a0 * lo.y, b1 * hi.x + a1 * hi.y);
}

// One CTA per row.
template <AppendForm FORM>
__global__ void __launch_bounds__(APP_THREADS) paged_append_kernel(const AppendParams p) {
    __shared__ float2 cs[MAX_HALF];
    pdl_wait();
    const int r = blockIdx.x;
    const int seq = p.row_seq ? p.row_seq[r] : r;
    if (seq < 0) return;
    const int pos = p.row_pos[r];
    int page = -1;
    if (seq < p.c.n_seqs && pos >= 0 && pos / p.c.page_size < p.c.max_pages)
        page = p.c.table[seq * p.c.table_stride + pos / p.c.page_size];
    if (page < 0 || page >= p.c.n_pages) {
        if (threadIdx.x == 0 && p.status) atomicOr(p.status, STATUS_BAD_PAGE);
        return;
    }
    const int half = p.rot_dim / 2;
    for (int i = threadIdx.x; i < half; i += APP_THREADS) cs[i] = turn_of(pos, p.inv_freq[i]);
    __syncthreads();
    const long long at = page * p.c.page_stride + (pos % p.c.page_size) * p.c.slot_stride;

    // units of a head: pieces of 16 bytes, or pairs of pieces that are rotated together
    constexpr int W = FORM == PAIRS_FAR_4 ? 4 : 8;
    const int turned = FORM == PAIRS_NEAR ? p.rot_dim / 8 : half / W;
    const int whole = p.head_dim / 8;
    const int units = turned + (p.head_dim - p.rot_dim) / 8;
    const int n_q = p.q ? p.n_head : 0, n_kv = p.c.n_kv_head;
    const int total = (n_q + n_kv) * units + n_kv * whole;
    for (int u = threadIdx.x; u < total; u += APP_THREADS) {
        const uint16_t *src;
        uint16_t *dst;
        int i;
        if (u < (n_q + n_kv) * units) {
            int h = u / units;
            i = u % units;
            if (h < n_q) {
                src = p.q + r * p.q_row + h * p.q_head;
                dst = p.q_out + r * p.qo_row + h * p.qo_head;
            } else {
                h -= n_q;
                src = p.k + r * p.k_row + h * p.k_head;
                dst = p.c.k + at + h * p.c.head_stride;
            }
        } else {
            const int w = u - (n_q + n_kv) * units;
            const int h = w / whole;
            i = turned + w % whole;   // copied pieces only
            src = p.v + r * p.v_row + h * p.v_head - p.rot_dim;
            dst = p.c.v + at + h * p.c.head_stride - p.rot_dim;
        }
        if (i >= turned) {
            const int e = p.rot_dim + (i - turned) * 8;
            *reinterpret_cast<uint4 *>(dst + e) = *reinterpret_cast<const uint4 *>(src + e);
        } else if (FORM == PAIRS_NEAR) {
            uint4 x = *reinterpret_cast<const uint4 *>(src + i * 8);
            uint32_t *w = reinterpret_cast<uint32_t *>(&x);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float2 t = cs[i * 4 + j];
                const float a = h16_lo(w[j]), b = h16_hi(w[j]);
                w[j] = pack_h16x2(a * t.x - b * t.y, b * t.x + a * t.y);
            }
            *reinterpret_cast<uint4 *>(dst + i * 8) = x;
        } else {
            uint32_t a[W / 2], b[W / 2];
            if (W == 8) {
                *reinterpret_cast<uint4 *>(a) = *reinterpret_cast<const uint4 *>(src + i * W);
                *reinterpret_cast<uint4 *>(b) = *reinterpret_cast<const uint4 *>(src + half + i * W);
            } else {
                *reinterpret_cast<uint2 *>(a) = *reinterpret_cast<const uint2 *>(src + i * W);
                *reinterpret_cast<uint2 *>(b) = *reinterpret_cast<const uint2 *>(src + half + i * W);
            }
#pragma unroll
            for (int j = 0; j < W / 2; ++j) turn_pair(a[j], b[j], cs[i * W + 2 * j], cs[i * W + 2 * j + 1]);
            if (W == 8) {
                *reinterpret_cast<uint4 *>(dst + i * W) = *reinterpret_cast<uint4 *>(a);
                *reinterpret_cast<uint4 *>(dst + half + i * W) = *reinterpret_cast<uint4 *>(b);
            } else {
                *reinterpret_cast<uint2 *>(dst + i * W) = *reinterpret_cast<uint2 *>(a);
                *reinterpret_cast<uint2 *>(dst + half + i * W) = *reinterpret_cast<uint2 *>(b);
            }
        }
    }
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
    const dim3 grid(a->rows), block(APP_THREADS);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (a->interleaved || a->rot_dim == 0) e = launch_pdl(paged_append_kernel<PAIRS_NEAR>, grid, block, 0, st, p);
    else if (a->rot_dim % 16 == 0) e = launch_pdl(paged_append_kernel<PAIRS_FAR_8>, grid, block, 0, st, p);
    else e = launch_pdl(paged_append_kernel<PAIRS_FAR_4>, grid, block, 0, st, p);
    return cuda_check(e, "paged append: launch");
}
