// Log probability of a given token, entropy and the largest logits of every row.
//
//   x = scale * logit, m = max x, S = sum e^(x - m):  lse = m + log S,  logprob = x_t - lse,
//   entropy = log S + sum (m - x) e^(x - m) / S       (every term of the sum is positive: nothing cancels)
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace kr {

namespace {

constexpr int LP_THREADS = 512;
constexpr int LP_MAX_TOP = 32;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.69314718055994531f;

struct LogprobParams {
    const void *logits;
    long long row_stride;
    const int *targets;
    float *logprob, *entropy, *lse;
    int *top_ids;
    float *top_logprobs;
    int vocab, top;
    float scale;
    uint32_t *status;
};

template <bool H16>
__device__ __forceinline__ float logit_at(const void *row, int i) {
    return H16 ? from_h16(static_cast<const uint16_t *>(row)[i]) : static_cast<const float *>(row)[i];
}

// Orders logits as the alternatives are listed: larger value first, of equal ones the lower index; NaN as -inf.
// -0 and +0 are equal.
__device__ __forceinline__ unsigned long long order_key(float x, int i) {
    if (!(x > -INFINITY)) x = -INFINITY;
    const uint32_t u = __float_as_uint(x + 0.f);
    const uint32_t o = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return (static_cast<unsigned long long>(o) << 32) | static_cast<uint32_t>(~i);
}

__device__ __forceinline__ float key_value(unsigned long long k) {
    const uint32_t o = static_cast<uint32_t>(k >> 32);
    return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}

template <typename T, typename F>
__device__ __forceinline__ T block_reduce(T v, F f, T *sm) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v = f(v, __shfl_xor_sync(0xFFFFFFFFu, v, off));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) sm[threadIdx.x >> 5] = v;
    __syncthreads();
    T r = sm[0];
    for (int w = 1; w < LP_THREADS / 32; ++w) r = f(r, sm[w]);
    return r;
}

// One CTA per row: a pass for the maximum, one for the sums, one for every alternative.
template <bool H16>
__global__ void __launch_bounds__(LP_THREADS) logprobs_kernel(const LogprobParams p) {
    __shared__ unsigned long long sm_k[LP_THREADS / 32];
    __shared__ float sm_f[LP_THREADS / 32];
    pdl_wait();
    const long long r = blockIdx.x;
    const void *row = static_cast<const uint8_t *>(p.logits) + r * p.row_stride * (H16 ? 2 : 4);
    float m = -INFINITY;
    for (int i = threadIdx.x; i < p.vocab; i += LP_THREADS) m = fmaxf(m, logit_at<H16>(row, i));
    m = block_reduce(m, [](float a, float b) { return fmaxf(a, b); }, sm_f);
    if (m == -INFINITY) m = 0.f;   // nothing but -inf: S = 0, log S = -inf, no NaN on the way
    float s = 0.f, d = 0.f;
    for (int i = threadIdx.x; i < p.vocab; i += LP_THREADS) {
        const float x = logit_at<H16>(row, i);
        const float y = (x - m) * p.scale;
        const float e = ex2_approx(y * LOG2E);
        s += e;
        if (x > -INFINITY) d -= y * e;
    }
    s = block_reduce(s, [](float a, float b) { return a + b; }, sm_f);
    d = block_reduce(d, [](float a, float b) { return a + b; }, sm_f);
    const float log_s = log2f(s) * LN2;
    const float lse = m * p.scale + log_s;
    if (threadIdx.x == 0) {
        if (p.lse) p.lse[r] = lse;
        if (p.entropy) p.entropy[r] = log_s + d / s;
        if (p.logprob) {
            const int t = p.targets[r];
            float v = 0.f;
            if (t >= p.vocab) {
                v = NAN;
                if (p.status) atomicOr(p.status, STATUS_BAD_TOKEN);
            } else if (t >= 0) {
                v = (logit_at<H16>(row, t) - m) * p.scale - log_s;
            }
            p.logprob[r] = v;
        }
    }
    unsigned long long last = ~0ull;
    for (int k = 0; k < p.top; ++k) {
        unsigned long long best = 0;
        for (int i = threadIdx.x; i < p.vocab; i += LP_THREADS) {
            const unsigned long long key = order_key(logit_at<H16>(row, i), i);
            if (key < last && key > best) best = key;
        }
        best = block_reduce(best, [](unsigned long long a, unsigned long long b) { return a > b ? a : b; }, sm_k);
        last = best;
        if (threadIdx.x == 0) {
            if (p.top_ids) p.top_ids[r * p.top + k] = static_cast<int>(~static_cast<uint32_t>(best));
            if (p.top_logprobs) p.top_logprobs[r * p.top + k] = (key_value(best) - m) * p.scale - log_s;
        }
    }
}

}  // namespace

}  // namespace kr

extern "C" int kraken_op_token_logprobs(const kraken_logprobs_args *a, uint32_t *d_status, void *stream) {
    using namespace kr;
    if (!a || a->rows < 0) return KRAKEN_EINVAL;
    if (a->rows == 0) return KRAKEN_OK;
    if (!a->logits || a->vocab < 1 || a->row_stride < 0 || a->dtype < 0 || a->dtype > 1 || a->top < 0 ||
        a->top > a->vocab || !(a->scale > 0.f) || !isfinite(a->scale) || (a->logprob && !a->targets) ||
        (a->top > 0 && !a->top_ids && !a->top_logprobs))
        return KRAKEN_EINVAL;
    if (a->top > LP_MAX_TOP) return KRAKEN_EUNSUPPORTED;
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
    p.vocab = a->vocab;
    p.top = a->top;
    p.scale = a->scale;
    p.status = d_status;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = a->dtype ? launch_pdl(logprobs_kernel<true>, dim3(a->rows), dim3(LP_THREADS), 0, st, p)
                                   : launch_pdl(logprobs_kernel<false>, dim3(a->rows), dim3(LP_THREADS), 0, st, p);
    return cuda_check(e, "token logprobs: launch");
}
