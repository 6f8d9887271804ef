// Verification of drafted tokens against the target's probabilities, and the draw of the token behind those that stand.
//
// Bound: every row of logits is read once, whatever stands (which rows count hangs on the rows before them), and the one row that a sequence's last token
// is drawn from once or twice more.  Three launches:
//   * slices of all rows: largest logit and sum of exponentials;
//   * a block per slice and sequence puts its sequence's rows together, finds the first draft that does not stand, and sums its slice of what that leaves, max(p - q, 0);
//   * a block per sequence finds the slice where the draw falls, and the token in it.
// Exponentials and sums are in 64 bits: of a hundred thousand borders between tokens, one in a thousand draws meets one that sums of fp32 exponentials have moved.
#include "spd_attention.h"

#include <algorithm>

using namespace spdd;
using namespace spda;

namespace {

constexpr int NTV = 256, NWV = NTV / WAVE;

// A logit as it counts: no number is -inf, +inf the largest finite number.
__device__ __forceinline__ float logit(float x) { return fminf(fmaxf(x, -INFINITY), 3.402823466e38f); }

// 2^x for x <= 0: x to the nearest whole number and a rest of at most 1/2, whose exponential is ten terms of its series; the next one is 2e-13.
__device__ __forceinline__ double exp2_64(double x) {
    x = fmax(x, -2000.0);
    const double k = rint(x), f = x - k;
    constexpr double L = 0.69314718055994530942;
    double y = 1.0;
#pragma unroll
    for (int n = 10; n >= 1; --n) y = fma(y, f * (L / n), 1.0);
    return ldexp(y, (int)k);
}

// Sums over the block, the same in all threads.
__device__ __forceinline__ double wave_add(double v) {
#pragma unroll
    for (int o = 1; o < WAVE; o <<= 1) v += __shfl_xor(v, o, WAVE);
    return v;
}
__device__ __forceinline__ double block_add(double v, double *red) {
    v = wave_add(v);
    __syncthreads();
    if (threadIdx.x % WAVE == 0) red[threadIdx.x / WAVE] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

typedef u32x4 __attribute__((aligned(2))) u32x4_any;      // on no grid but that of the elements

// N logits from v0 on (fewer behind the vocabulary's end: -inf).  Rows may lie anywhere: 16 bytes at a time, aligned or not.
template <typename T, int N> __device__ __forceinline__ void load_logits(const void *row, int v0, int vocab, float (&z)[N]) {
    constexpr int VEC = 16 / (int)sizeof(T);
    static_assert(N == VEC, "one load");
    if (v0 + VEC <= vocab) {
        const u32x4_any x = *(const u32x4_any __attribute__((address_space(1))) *)((const T *)row + v0);
        Store<T>::unpack(x, z);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) z[e] = v0 + e < vocab ? Store<T>::load1(row, v0 + e) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) z[e] = logit(z[e]);
}

template <typename T> __device__ __forceinline__ const void *row_of(const void *base, int64_t stride, int t) { return (const T *)base + (int64_t)t * stride; }

// Rows 0 .. n_tokens - 1: the target's; behind them the drafter's.
template <typename T, int E>
__global__ __launch_bounds__(NTV) void verify_sums_kernel(const VerifyArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T), PIECES = E / VEC;
    __shared__ float tops[NWV];
    __shared__ double red[NWV];
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), r = blockIdx.x / a.slices, slice = blockIdx.x - r * a.slices;
    const bool draft = r >= a.n_tokens;
    const int t = draft ? r - a.n_tokens : r;
    // rows that nothing asks about: no sequence's, and the drafter's at a sequence's last token
    bool last = false, inside = false;
    for (int i = lane; i <= a.n_seq; i += WAVE) {
        const int f = as_global(a.first)[i];
        last = last || f == t + 1;
        inside = inside || (i == 0 && f <= t) ;
    }
    if (!__any(inside) || t >= as_global(a.first)[a.n_seq] || (draft && __any(last))) return;
    const void *row = draft ? row_of<T>(a.draft_logits, a.draft_stride, t) : row_of<T>(a.logits, a.row_stride, t);
    const double c = draft ? a.by_draft_tau : a.by_tau;
    float z[PIECES][VEC], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) load_logits<T, VEC>(row, (slice * PIECES + i) * NTV * VEC + tid * VEC, a.vocab, z[i]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = fmaxf(top, z[i][e]);
    top = wave_max(top);
    if (lane == 0) tops[tid / WAVE] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    double sum = 0.0;
    if (top > -INFINITY)
#pragma unroll
        for (int i = 0; i < PIECES; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum += exp2_64(((double)z[i][e] - (double)top) * c);
    sum = block_add(sum, red);
    if (tid == 0) {
        as_global(a.top)[blockIdx.x] = top;
        as_global(a.sum)[blockIdx.x] = sum;
    }
}

// A row's largest logit and the inverse of its sum, by a wave.
__device__ __forceinline__ void whole_row(const VerifyArgs &a, int r, double c, int lane, float &top, double &inv) {
    const size_t at = (size_t)r * a.slices;
    top = -INFINITY;
    for (int i = lane; i < a.slices; i += WAVE) top = fmaxf(top, as_global(a.top)[at + i]);
    top = wave_max(top);
    double sum = 0.0;
    for (int i = lane; i < a.slices; i += WAVE) {
        const float m = as_global(a.top)[at + i];
        if (m > -INFINITY) sum += as_global(a.sum)[at + i] * exp2_64(((double)m - (double)top) * c);
    }
    sum = wave_add(sum);
    inv = top > -INFINITY ? 1.0 / sum : 0.0;
}
template <typename T> __device__ __forceinline__ double exponent(const void *row, int v, float top, double c) { return ((double)logit(Store<T>::load1(row, v)) - (double)top) * c; }

// What a row leaves of VEC tokens from v0 on.
template <typename T, int VEC>
__device__ __forceinline__ void weights(const VerifyArgs &a, const VerifyPick &k, bool rest, int v0, double (&w)[VEC]) {
    float z[VEC];
    load_logits<T, VEC>(row_of<T>(a.logits, a.row_stride, k.row), v0, a.vocab, z);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = k.inv == 0.0 ? 0.0 : exp2_64(((double)z[e] - (double)k.top) * a.by_tau) * k.inv;
    if (!rest) return;
    if (a.draft_logits) {
        load_logits<T, VEC>(row_of<T>(a.draft_logits, a.draft_stride, k.row), v0, a.vocab, z);
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = fmax(w[e] - (k.draft_inv == 0.0 ? 0.0 : exp2_64(((double)z[e] - (double)k.draft_top) * a.by_draft_tau) * k.draft_inv), 0.0);
    } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = v0 + e == k.token ? 0.0 : w[e];
    }
}

template <typename T, int E>
__global__ __launch_bounds__(NTV) void verify_drafts_kernel(const VerifyArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T), PIECES = E / VEC;
    __shared__ int stop;
    __shared__ double red[NWV];
    __shared__ VerifyPick pick;
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), wv = tid / WAVE, s = blockIdx.x / a.slices, slice = blockIdx.x - s * a.slices;
    int descends = 0;
    for (int i = tid; i < a.n_seq; i += NTV) descends |= as_global(a.first)[i + 1] < as_global(a.first)[i];
    if (tid == 0) stop = INT32_MAX;
    const bool sorted = !__syncthreads_or(descends);
    const int lo = as_global(a.first)[s], hi = as_global(a.first)[s + 1];
    const bool fits = sorted && lo >= 0 && hi <= a.n_tokens;
    if (!fits || lo == hi) {
        if (tid == 0 && slice == 0) {
            as_global(a.out_accepted)[s] = 0;
            a.pick[s].row = -1;
            if (!fits && a.err) *as_global(a.err) = 1;
        }
        return;
    }
    // a wave per row: does its draft stand?  (Those behind the first that does not are looked at in vain.)
    const bool drawn = a.draft_logits != nullptr;
    for (int t = lo + wv; t < hi - 1; t += NWV) {
        const int x = as_global(a.tokens)[t + 1];
        const bool known = (unsigned)x < (unsigned)a.vocab;
        float top;
        double inv, p = 0.0, q = 1.0, e = 0.0;
        whole_row(a, t, a.by_tau, lane, top, inv);
        if (known && inv != 0.0) {
            e = exponent<T>(row_of<T>(a.logits, a.row_stride, t), x, top, a.by_tau);
            p = exp2_64(e) * inv;
        }
        const double log2_p = e + log2(inv);
        if (drawn) {
            whole_row(a, a.n_tokens + t, a.by_draft_tau, lane, top, inv);
            q = known && inv != 0.0 ? exp2_64(exponent<T>(row_of<T>(a.draft_logits, a.draft_stride, t), x, top, a.by_draft_tau)) * inv : 0.0;
        }
        const bool stands = (double)as_global(a.u)[t] * q < p;
        if (lane == 0) {
            if (!stands) atomicMin(&stop, t);
            else if (slice == 0) {
                as_global(a.out_tokens)[t] = x;
                as_global(a.out_logprobs)[t] = (float)(log2_p * 0.69314718055994530942);
            }
        }
    }
    __syncthreads();
    const bool refused = stop < hi - 1;
    const int row = refused ? stop : hi - 1;
    if (wv == 0) {
        VerifyPick k{};
        k.row = row;
        k.refused = refused;
        k.token = refused ? as_global(a.tokens)[row + 1] : -1;
        whole_row(a, row, a.by_tau, lane, k.top, k.inv);
        if (refused && drawn) whole_row(a, a.n_tokens + row, a.by_draft_tau, lane, k.draft_top, k.draft_inv);
        if (lane == 0) {
            pick = k;
            if (slice == 0) {
                a.pick[s] = k;
                as_global(a.out_accepted)[s] = row - lo;
                if (a.err && (k.inv == 0.0 || (refused && (unsigned)k.token >= (unsigned)a.vocab))) *as_global(a.err) = 1;
            }
        }
    }
    if (slice == 0)
        for (int i = row + 1 + tid; i < hi; i += NTV) {
            as_global(a.out_tokens)[i] = -1;
            as_global(a.out_logprobs)[i] = 0.f;
        }
    if (!refused) return;                        // (the slices' sums are there)
    __syncthreads();
    const VerifyPick k = pick;
    double sum = 0.0;
#pragma unroll 1
    for (int i = 0; i < PIECES; ++i) {
        double w[VEC];
        weights<T, VEC>(a, k, true, (slice * PIECES + i) * NTV * VEC + tid * VEC, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += w[e];
    }
    sum = block_add(sum, red);
    if (tid == 0) a.rest[(size_t)s * a.slices + slice] = sum;
}

template <typename T, int E>
__global__ __launch_bounds__(NTV) void verify_pick_kernel(const VerifyArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T), PIECES = E / VEC;
    __shared__ double red[NWV], before_slice;
    __shared__ int found, last, in_slice;
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), wv = tid / WAVE, s = blockIdx.x;
    const VerifyPick k = a.pick[s];
    if (k.row < 0) return;
    const double u = (double)as_global(a.u)[as_global(a.first)[s + 1] - 1];
    if (tid == 0) { found = INT32_MAX; last = -1; in_slice = -1; }
    // a slice's sum: what is left, or (all stand, or nothing is left) p itself
    bool rest = k.refused;
    const auto slice_sum = [&](int i) {
        if (rest) return a.rest[(size_t)s * a.slices + i];
        const size_t at = (size_t)k.row * a.slices + i;
        const float m = as_global(a.top)[at];
        return m > -INFINITY ? as_global(a.sum)[at] * exp2_64(((double)m - (double)k.top) * a.by_tau) * k.inv : 0.0;
    };
    double total;
    for (;;) {
        double sum = 0.0;
        for (int i = tid; i < a.slices; i += NTV) sum += slice_sum(i);
        total = block_add(sum, red);
        if (total > 0.0 || !rest) break;
        rest = false;
    }
    const double bound = u * total;
    if (wv == 0) {                               // the slice where the sums pass it; the last with a weight where none does
        double before = 0.0;
        int pick = -1;
        double pick_before = 0.0;
        for (int i0 = 0; i0 < a.slices; i0 += WAVE) {
            const double mine = i0 + lane < a.slices ? slice_sum(i0 + lane) : 0.0;
            double upto = mine;
#pragma unroll
            for (int o = 1; o < WAVE; o <<= 1) {
                const double x = __shfl_up(upto, o, WAVE);
                if (lane >= o) upto += x;
            }
            const u64 some = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && before + upto > bound);
            if (past) {
                pick = i0 + __builtin_ctzll(past);
                pick_before = before + (__shfl(upto, pick - i0, WAVE) - __shfl(mine, pick - i0, WAVE));
                break;
            }
            if (some) {
                pick = i0 + 63 - __builtin_clzll(some);
                pick_before = before + (__shfl(upto, pick - i0, WAVE) - __shfl(mine, pick - i0, WAVE));
            }
            before += __shfl(upto, WAVE - 1, WAVE);
        }
        if (lane == 0) { in_slice = pick; before_slice = pick_before; }
    }
    __syncthreads();
    double before = before_slice;
    if (in_slice >= 0)
#pragma unroll 1
        for (int i = 0; i < PIECES; ++i) {
            const int v0 = (in_slice * PIECES + i) * NTV * VEC + tid * VEC;
            double w[VEC], mine = 0.0;
            weights<T, VEC>(a, k, rest, v0, w);
#pragma unroll
            for (int e = 0; e < VEC; ++e) mine += w[e];
            double upto = mine;
#pragma unroll
            for (int o = 1; o < WAVE; o <<= 1) {
                const double x = __shfl_up(upto, o, WAVE);
                if (lane >= o) upto += x;
            }
            __syncthreads();
            if (lane == WAVE - 1) red[wv] = upto;
            __syncthreads();
            double at = before + (upto - mine);
            for (int j = 0; j < wv; ++j) at += red[j];
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                at += w[e];
                if (w[e] > 0.0) {
                    atomicMax(&last, v0 + e);
                    if (at > bound) { atomicMin(&found, v0 + e); break; }
                }
            }
            before += (red[0] + red[1]) + (red[2] + red[3]);
            __syncthreads();
            if (found != INT32_MAX) break;
        }
    __syncthreads();
    if (tid == 0) {
        const int v = found != INT32_MAX ? found : last >= 0 ? last : 0;
        as_global(a.out_tokens)[k.row] = v;
        const double e = k.inv == 0.0 ? 0.0 : exponent<T>(row_of<T>(a.logits, a.row_stride, k.row), v, k.top, a.by_tau);
        as_global(a.out_logprobs)[k.row] = k.inv == 0.0 ? -INFINITY : (float)((e + log2(k.inv)) * 0.69314718055994530942);
    }
}

// Logits per thread of a slice: 32, or 8 where that leaves too few blocks to fill the GPU.
int each_for(int n_tokens, int vocab) { return (long long)n_tokens * 2 * ((vocab + 32 * NTV - 1) / (32 * NTV)) < 512 ? 8 : 32; }
int slices_for(int n_tokens, int vocab) {
    const int n = NTV * each_for(n_tokens, vocab);
    return (vocab + n - 1) / n;
}

template <typename T, int E> hipError_t launch_each(hipStream_t s, const VerifyArgs &a) {
    hipLaunchKernelGGL((verify_sums_kernel<T, E>), dim3((unsigned)(a.n_tokens * (a.draft_logits ? 2 : 1) * a.slices)), dim3(NTV), 0, s, a);
    hipLaunchKernelGGL((verify_drafts_kernel<T, E>), dim3((unsigned)(a.n_seq * a.slices)), dim3(NTV), 0, s, a);
    hipLaunchKernelGGL((verify_pick_kernel<T, E>), dim3((unsigned)a.n_seq), dim3(NTV), 0, s, a);
    return hipGetLastError();
}
template <typename T> hipError_t launch(hipStream_t s, const VerifyArgs &a) { return each_for(a.n_tokens, a.vocab) == 8 ? launch_each<T, 8>(s, a) : launch_each<T, 32>(s, a); }

}  // namespace

extern "C" size_t spd_op_verify_drafts_scratch_bytes(int32_t n_seq, int32_t n_tokens, int32_t vocab) {
    if (n_seq <= 0 || n_tokens < 0 || vocab <= 0) return 0;
    const size_t slices = (size_t)slices_for(n_tokens, vocab), rows = 2 * (size_t)n_tokens * slices;
    return up256(rows * 8) + up256(rows * 4) + up256(n_seq * slices * 8) + up256(n_seq * sizeof(VerifyPick));
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
    const int slices = slices_for(n_tokens, vocab);
    if ((long long)std::max(2 * n_tokens, n_seq) * slices > INT32_MAX) return SPD_EINVAL;
    const double log2e = 1.4426950408889634074;
    char *w = (char *)scratch;
    VerifyArgs a{logits, draft_logits, row_stride, draft_stride, tokens, first, u, n_seq, n_tokens, vocab, log2e / tau, draft_logits ? log2e / draft_tau : 1.0, out_tokens, out_logprobs, out_accepted, err, slices};
    const size_t row_sums = 2 * (size_t)n_tokens * slices;
    a.sum = (double *)w; w += up256(row_sums * 8);
    a.top = (float *)w; w += up256(row_sums * 4);
    a.rest = (double *)w; w += up256((size_t)n_seq * slices * 8);
    a.pick = (VerifyPick *)w;
    hipStream_t s = (hipStream_t)hip_stream;
    if (n_tokens == 0) {                         // (sequences without tokens: a = 0 each)
        hipLaunchKernelGGL((verify_drafts_kernel<float, 8>), dim3((unsigned)(n_seq * slices)), dim3(NTV), 0, s, a);
        return hipGetLastError() == hipSuccess ? SPD_OK : SPD_EHIP;
    }
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch<float>(s, a) : dtype == SPD_DTYPE_FP16 ? launch<half_t>(s, a) : launch<bf16_t>(s, a);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}
