// Verification of drafted tokens against the target's probabilities.
//
// One block per sequence, everything in 64 bits: row by row the probability of the next draft under both models, up to the first draft that does
// not stand; then one token from what is left of that row.
#include "spd_device.h"

using namespace spdd;

namespace {

constexpr int NTV = 1024, NWV = NTV / WAVE;

// A logit as it counts.
__device__ __forceinline__ float logit(float x) { return x != x ? -INFINITY : fminf(x, 3.402823466e38f); }

__device__ __forceinline__ double block_reduce(double v, double *red, bool maximum) {
    for (int o = 1; o < WAVE; o <<= 1) {
        const double w = __shfl_xor(v, o, WAVE);
        v = maximum ? fmax(v, w) : v + w;
    }
    __syncthreads();
    if (threadIdx.x % WAVE == 0) red[threadIdx.x / WAVE] = v;
    __syncthreads();
    v = red[0];
    for (int i = 1; i < NWV; ++i) v = maximum ? fmax(v, red[i]) : v + red[i];
    return v;
}

template <typename T> struct Row {
    const void *base;
    size_t at;
    double by_tau, top, inv;      // inv: 1 / sum of exp, 0 where no logit is finite
    __device__ double z(int v) const { return (double)logit(Store<T>::load1(base, at + v)) * by_tau; }
    __device__ double p(int v) const { return inv == 0.0 ? 0.0 : exp(z(v) - top) * inv; }
    __device__ void measure(int vocab, double *red) {
        top = -INFINITY;
        for (int v = threadIdx.x; v < vocab; v += NTV) top = fmax(top, z(v));
        top = block_reduce(top, red, true);
        double sum = 0.0;
        if (top > -INFINITY)
            for (int v = threadIdx.x; v < vocab; v += NTV) sum += exp(z(v) - top);
        sum = block_reduce(sum, red, false);
        inv = top > -INFINITY ? 1.0 / sum : 0.0;
    }
};

template <typename T>
__global__ __launch_bounds__(NTV) void verify_kernel(const VerifyArgs a) {
    __shared__ double red[NWV], part[NTV + 1];
    __shared__ int chosen;
    const int s = blockIdx.x, tid = threadIdx.x;
    const int lo = as_global(a.first)[s], hi = as_global(a.first)[s + 1];
    int descends = 0;
    for (int i = tid; i < a.n_seq; i += NTV) descends |= as_global(a.first)[i + 1] < as_global(a.first)[i];
    const bool fits = !__syncthreads_or(descends) && lo >= 0 && hi <= a.n_tokens;
    if (!fits || lo == hi) {
        if (tid == 0) {
            as_global(a.out_accepted)[s] = 0;
            if (!fits && a.err) *as_global(a.err) = 1;
        }
        return;
    }
    const bool drawn = a.draft_logits != nullptr;
    int t = lo;
    bool refused = false;
    int x = 0;
    Row<T> p{a.logits, 0, a.by_tau, 0.0, 0.0}, q{a.draft_logits, 0, a.by_draft_tau, 0.0, 0.0};
    for (;; ++t) {
        p.at = (size_t)t * a.row_stride;
        p.measure(a.vocab, red);
        if (t == hi - 1) break;
        q.at = (size_t)t * a.draft_stride;
        if (drawn) q.measure(a.vocab, red);
        x = as_global(a.tokens)[t + 1];
        const bool known = (unsigned)x < (unsigned)a.vocab;
        if (!known && tid == 0 && a.err) *as_global(a.err) = 1;
        refused = !known || !((double)as_global(a.u)[t] * (drawn ? q.p(x) : 1.0) < p.p(x));
        if (refused) break;
        if (tid == 0) {
            as_global(a.out_tokens)[t] = x;
            as_global(a.out_logprobs)[t] = (float)log(p.p(x));
        }
    }
    // one token of row t
    const int each = (a.vocab + NTV - 1) / NTV, v0 = min(a.vocab, tid * each), v1 = min(a.vocab, v0 + each);
    bool rest = refused;
    const auto weight = [&](int v) { return !rest ? p.p(v) : drawn ? fmax(p.p(v) - q.p(v), 0.0) : v == x ? 0.0 : p.p(v); };
    for (;;) {
        double sum = 0.0;
        for (int v = v0; v < v1; ++v) sum += weight(v);
        __syncthreads();
        part[tid + 1] = sum;
        __syncthreads();
        if (tid == 0) {
            part[0] = 0.0;
            for (int i = 0; i < NTV; ++i) part[i + 1] += part[i];
            chosen = -1;
        }
        __syncthreads();
        if (part[NTV] > 0.0 || !rest) break;
        rest = false;
    }
    const double bound = (double)as_global(a.u)[hi - 1] * part[NTV];
    int mine = -1;                               // the first token past the bound; the last with a weight where none is
    double sum = part[tid];
    for (int v = v0; v < v1; ++v) {
        const double w = weight(v);
        sum += w;
        if (w > 0.0 && sum > bound && mine < 0) mine = v;
    }
    int last = -1;
    for (int v = v0; v < v1; ++v) last = weight(v) > 0.0 ? v : last;
    const double found = -block_reduce(mine >= 0 ? -(double)mine : -INFINITY, red, true), end = block_reduce((double)last, red, true);
    if (tid == 0) {
        const int v = found < INFINITY ? (int)found : end >= 0.0 ? (int)end : 0;
        as_global(a.out_tokens)[t] = v;
        as_global(a.out_logprobs)[t] = p.inv == 0.0 ? -INFINITY : (float)(p.z(v) - p.top + log(p.inv));
        as_global(a.out_accepted)[s] = t - lo;
        if (p.inv == 0.0 && a.err) *as_global(a.err) = 1;
    }
    for (int i = t + 1 + tid; i < hi; i += NTV) {
        as_global(a.out_tokens)[i] = -1;
        as_global(a.out_logprobs)[i] = 0.f;
    }
}

template <typename T> hipError_t launch(hipStream_t s, const VerifyArgs &a) {
    hipLaunchKernelGGL(verify_kernel<T>, dim3((unsigned)a.n_seq), dim3(NTV), 0, s, a);
    return hipGetLastError();
}

}  // namespace

extern "C" size_t spd_op_verify_drafts_scratch_bytes(int32_t n_seq, int32_t n_tokens, int32_t vocab) {
    (void)n_seq; (void)n_tokens; (void)vocab;
    return 0;
}

extern "C" int spd_op_verify_drafts(int32_t dtype, const void *logits, int64_t row_stride, const void *draft_logits, int64_t draft_stride, const int32_t *tokens, const int32_t *first,
                                    const float *u, int32_t n_seq, int32_t n_tokens, int32_t vocab, float tau, float draft_tau, int32_t *out_tokens, float *out_logprobs,
                                    int32_t *out_accepted, void *scratch, size_t scratch_bytes, int32_t *err, void *hip_stream) {
    if (dtype != SPD_DTYPE_FP32 && dtype != SPD_DTYPE_BF16 && dtype != SPD_DTYPE_FP16) return SPD_EINVAL;
    const int el = dtype == SPD_DTYPE_FP32 ? 4 : 2;
    if (n_seq < 0 || n_tokens < 0 || vocab < 1 || vocab > (1 << 24) || !(tau > 0.f) || !(tau < INFINITY) || (draft_logits && (!(draft_tau > 0.f) || !(draft_tau < INFINITY)))) return SPD_EINVAL;
    if (n_seq == 0) return SPD_OK;
    if (!first || !out_accepted || (n_tokens > 0 && (!logits || !tokens || !u || !out_tokens || !out_logprobs)) || n_seq > (1 << 20) || n_tokens > (1 << 20)) return SPD_EINVAL;
    if (row_stride < vocab || (draft_logits && draft_stride < vocab) || ((uintptr_t)logits | (uintptr_t)draft_logits) % el) return SPD_EINVAL;
    const size_t need = spd_op_verify_drafts_scratch_bytes(n_seq, n_tokens, vocab);
    if (need && (!scratch || (uintptr_t)scratch % 256)) return SPD_EINVAL;
    if (scratch_bytes < need) return SPD_EWORKSPACE;
    const auto rows = [&](int64_t stride) { return n_tokens ? ((size_t)(n_tokens - 1) * stride + vocab) * el : 0; };
    const size_t ids = (size_t)n_tokens * 4;
    const spdk::Span sz{logits, rows(row_stride)}, sd{draft_logits, rows(draft_stride)}, st{tokens, ids}, sf{first, (size_t)(n_seq + 1) * 4}, su{u, ids}, ot{out_tokens, ids}, ol{out_logprobs, ids},
        oa{out_accepted, (size_t)n_seq * 4}, se{err, 4}, sw{scratch, need};
    if (spdk::over_any(ot, {sz, sd, st, sf, su, ol, oa, se, sw}) || spdk::over_any(ol, {sz, sd, st, sf, su, oa, se, sw}) || spdk::over_any(oa, {sz, sd, st, sf, su, se, sw}) ||
        spdk::over_any(sw, {sz, sd, st, sf, su, se})) return SPD_EINVAL;
    VerifyArgs a{logits, draft_logits, row_stride, draft_stride, tokens, first, u, n_seq, n_tokens, vocab, 1.0 / tau, draft_logits ? 1.0 / draft_tau : 1.0, out_tokens, out_logprobs, out_accepted, err};
    hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch<float>(s, a) : dtype == SPD_DTYPE_FP16 ? launch<half_t>(s, a) : launch<bf16_t>(s, a);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}
