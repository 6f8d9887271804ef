// Beam search's selection: the best continuations of a group's beams over the vocabulary.
//
// Within a row the order of continuations is that of its logits; the log-sum-exp and the beam's
// score move all of them alike.  So one pass over the logits leaves, per slice of a row, the
// n_out best (sort keys, exact) with the slice's maximum and sum of exponentials, and a second,
// small kernel puts a group's slices together and ranks what is left, at most n_in * n_out
// continuations, by score in 64 bits.
// Selection within a wave: with E entries per lane the n_out-th largest of the 64 lanes' best
// bounds the n_out-th largest entry from below, and is found in 32 ballots whatever n_out is;
// about n_out entries lie above it.
#include "spd_device.h"

using namespace spdd;

namespace {

typedef unsigned long long u64;

constexpr int NTB = 256, NWB = NTB / WAVE;       // slices: threads and waves per block
constexpr int E = 16;                            // entries per thread
constexpr int SLICE = NTB * E;
constexpr int NTM = 1024;                        // merge: a wave per row
constexpr int EM = 4;                            // keys per lane and turn there

// Larger is better: higher logit, then lower id.  0: no entry (an excluded one, -inf, is none either).
__device__ __forceinline__ u64 sort_key(float z, int id) {
    const uint32_t u = __float_as_uint(z);
    const uint32_t hi = (u & 0x80000000u) ? ~u : u | 0x80000000u;
    return z == -INFINITY ? 0ull : ((u64)hi << 32) | (0xFFFFFFFFu - (uint32_t)id);
}
__device__ __forceinline__ float key_logit(u64 k) {
    const uint32_t hi = (uint32_t)(k >> 32);
    return __uint_as_float((hi & 0x80000000u) ? hi & 0x7FFFFFFFu : ~hi);
}
__device__ __forceinline__ int key_id(u64 k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

// A logit as it counts: what is no number is excluded, +inf is the largest number, -0 is 0.
__device__ __forceinline__ float clean(float z) {
    if (z != z) return -INFINITY;
    return fminf(z, 3.402823466e38f) + 0.f;
}

// The n best of a wave's keys (N per lane), best first, into best[0 .. n) (LDS, this wave's); 0 where there are fewer.
// `list`: LDS, WAVE keys of this wave's.
template <int N>
__device__ __forceinline__ void wave_best(const u64 (&key)[N], int n, u64 *list, u64 *best) {
    const int lane = threadIdx.x & (WAVE - 1);
    u64 top = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) top = key[e] > top ? key[e] : top;
    const uint32_t top_hi = (uint32_t)(top >> 32);
    uint32_t bound = 0;                          // the n-th largest of the lanes' best logits; 0 where fewer have one
#pragma unroll
    for (int b = 31; b >= 0; --b) {
        const uint32_t t = bound | (1u << b);
        if (__popcll(__ballot(top_hi >= t)) >= n) bound = t;
    }
    int count = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) count += __popcll(__ballot(key[e] != 0 && (uint32_t)(key[e] >> 32) >= bound));
    u64 least = (u64)bound << 32;
    if (count > WAVE) {
        // many equal logits: the n-th largest key itself (keys differ in their ids)
        least = 0;
        for (int b = 63; b >= 0; --b) {
            const u64 t = least | (1ull << b);
            int c = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) c += __popcll(__ballot(key[e] >= t));
            if (c >= n) least = t;
        }
    }
    int at = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const bool in = key[e] != 0 && key[e] >= least;
        const u64 m = __ballot(in);
        if (in) list[at + __popcll(m & ((1ull << lane) - 1ull))] = key[e];
        at += __popcll(m);
    }
    if (lane < n) best[lane] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const u64 mine = lane < at ? list[lane] : 0;
    int rank = 0;
    for (int i = 0; i < at; ++i) rank += list[i] > mine;
    if (mine && rank < n) best[rank] = mine;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

template <typename LT> __device__ __forceinline__ float logit_at(const void *p, size_t i) { return Store<LT>::load1(p, i); }

__device__ __forceinline__ bool row_runs(const SelectArgs &a, int row) {
    const float score = as_global(a.scores)[row];
    return score > -INFINITY && !(a.ended && as_global(a.ended)[row] != 0);       // (a score that is no number: no beam)
}

// One block per (row, slice).
template <typename LT, bool ALIGNED>
__global__ __launch_bounds__(NTB) void beam_slice_kernel(const SelectArgs a) {
    constexpr int VEC = Store<LT>::VEC;
    __shared__ u64 list[NWB][WAVE], best[NWB][SPD_K_MAX];
    __shared__ float red[NWB];
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), w = tid / WAVE;
    const int row = blockIdx.x / a.slices, slice = blockIdx.x % a.slices;
    if (!row_runs(a, row)) return;
    const char *z_row = (const char *)a.logits + (size_t)row * a.row_stride * sizeof(LT);
    const int lo = slice * SLICE;
    float z[E];
#pragma unroll
    for (int i = 0; i < E; ++i) z[i] = -INFINITY;
    if (ALIGNED) {
#pragma unroll
        for (int j = 0; j < E / VEC; ++j) {
            const int at = lo + (j * NTB + tid) * VEC;
            if (at + VEC <= a.vocab) {
                float f[VEC];
                Store<LT>::unpack(global_load16(z_row + (size_t)at * sizeof(LT)), f);
#pragma unroll
                for (int v = 0; v < VEC; ++v) z[j * VEC + v] = f[v];
            } else {
#pragma unroll
                for (int v = 0; v < VEC; ++v)
                    if (at + v < a.vocab) z[j * VEC + v] = logit_at<LT>(z_row, at + v);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int at = lo + (i / VEC * NTB + tid) * VEC + i % VEC;
            if (at < a.vocab) z[i] = logit_at<LT>(z_row, at);
        }
    }
    float m = -INFINITY;
    u64 key[E];
#pragma unroll
    for (int i = 0; i < E; ++i) {
        z[i] = clean(z[i]);
        m = fmaxf(m, z[i]);
        key[i] = sort_key(z[i], lo + (i / VEC * NTB + tid) * VEC + i % VEC);
    }
    m = block_max<NTB>(m, red);
    const float c = 1.4426950408889634f / a.tau, ref = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) sum += exp2f((z[i] - ref) * c);
    sum = block_sum<NTB>(sum, red);
    wave_best<E>(key, a.n_out, list[w], best[w]);
    __syncthreads();
    const size_t part = (size_t)row * a.slices + slice;
    if (w == 0) {
        u64 k[1] = {lane < NWB * a.n_out ? best[lane / a.n_out][lane % a.n_out] : 0};
        __builtin_amdgcn_wave_barrier();
        int rank = 0;
        for (int i = 0; i < NWB * a.n_out; ++i) {
            const u64 other = best[i / a.n_out][i % a.n_out];
            rank += other > k[0] || (other == k[0] && i < lane);
        }
        if (lane < NWB * a.n_out && rank < a.n_out) ((global_ptr<u64>)a.best)[part * a.n_out + rank] = k[0];
    }
    if (tid == NTB - 1) { as_global(a.top)[part] = m; as_global(a.sum)[part] = sum; }
}

// One block per group, a wave per row; then the group's continuations are ranked.
__global__ __launch_bounds__(NTM) void beam_merge_kernel(const SelectArgs a) {
    __shared__ u64 list[SPD_K_MAX][WAVE], best[SPD_K_MAX][SPD_K_MAX];
    __shared__ double score[SPD_K_MAX * SPD_K_MAX];
    __shared__ int token[SPD_K_MAX * SPD_K_MAX];
    __shared__ int s_ended[SPD_K_MAX];
    __shared__ int present;
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), b = tid / WAVE, g = blockIdx.x, row = g * a.n_in + b;
    if (tid == 0) present = 0;
    if (b < a.n_in) {
        const float s = as_global(a.scores)[row];
        const bool ended = a.ended && as_global(a.ended)[row] != 0;
        if (row_runs(a, row)) {
            const size_t part = (size_t)row * a.slices;
            float M = -INFINITY;
            for (int i = lane; i < a.slices; i += WAVE) M = fmaxf(M, as_global(a.top)[part + i]);
            M = wave_max(M);
            const float c = 1.4426950408889634f / a.tau;
            float sum = 0.f;
            for (int i = lane; i < a.slices; i += WAVE) {
                const float t = as_global(a.top)[part + i];
                if (t > -INFINITY) sum += as_global(a.sum)[part + i] * exp2f((t - M) * c);
            }
            sum = wave_sum(sum);
            const u64 *keys = a.best + part * a.n_out;
            const int n = a.slices * a.n_out;
            u64 kept = 0;                                         // lane i: the i-th best so far
            for (int i0 = 0; i0 < n; i0 += EM * WAVE) {
                u64 key[EM + 1];
#pragma unroll
                for (int e = 0; e < EM; ++e) {
                    const int i = i0 + e * WAVE + lane;
                    key[e] = i < n ? ((global_ptr<const u64>)keys)[i] : 0;
                }
                key[EM] = kept;
                wave_best<EM + 1>(key, a.n_out, list[b], best[b]);
                kept = lane < a.n_out ? best[b][lane] : 0;
            }
            if (lane < a.n_out) {
                const double lse = (double)M / a.tau + log((double)sum);
                score[b * a.n_out + lane] = kept ? (double)s + ((double)key_logit(kept) / a.tau - lse) : -INFINITY;
                token[b * a.n_out + lane] = key_id(kept);
            }
        } else if (lane < a.n_out) {                              // an ended beam goes on as it is; an absent one has no continuation
            score[b * a.n_out + lane] = ended && lane == 0 && s > -INFINITY ? (double)s : -INFINITY;
            token[b * a.n_out + lane] = a.end_token;
        }
        if (lane == 0) s_ended[b] = ended;
    }
    __syncthreads();
    const int n = a.n_in * a.n_out;
    if (tid < n) {
        const double mine = score[tid];
        const int tok = token[tid], beam = tid / a.n_out;
        const bool there = mine > -INFINITY;
        int rank = 0;
        for (int i = 0; i < n; ++i) {
            const double other = score[i];
            const int ob = i / a.n_out;
            rank += other > mine || (other == mine && (ob < beam || (ob == beam && token[i] < tok)));
        }
        if (there) atomicAdd(&present, 1);
        if (there && rank < a.n_out) {
            const int at = g * a.n_out + rank;
            as_global(a.out_scores)[at] = (float)mine;
            as_global(a.out_tokens)[at] = tok;
            as_global(a.out_parents)[at] = beam;
            if (a.out_ended) as_global(a.out_ended)[at] = s_ended[beam] || tok == a.end_token;
        }
    }
    __syncthreads();
    if (tid < a.n_out && tid >= present) {                        // fewer continuations than asked for
        const int at = g * a.n_out + tid;
        as_global(a.out_scores)[at] = -INFINITY;
        as_global(a.out_tokens)[at] = 0;
        as_global(a.out_parents)[at] = tid < a.n_in ? tid : 0;
        if (a.out_ended) as_global(a.out_ended)[at] = 0;
    }
}

template <typename LT>
hipError_t launch_select(hipStream_t s, const SelectArgs &a) {
    const unsigned blocks = (unsigned)((long long)a.n_groups * a.n_in * a.slices);
    const bool aligned = (uintptr_t)a.logits % 16 == 0 && a.row_stride * (int64_t)sizeof(LT) % 16 == 0;
    if (aligned) hipLaunchKernelGGL((beam_slice_kernel<LT, true>), dim3(blocks), dim3(NTB), 0, s, a);
    else hipLaunchKernelGGL((beam_slice_kernel<LT, false>), dim3(blocks), dim3(NTB), 0, s, a);
    hipLaunchKernelGGL(beam_merge_kernel, dim3(a.n_groups), dim3(NTM), 0, s, a);
    return hipGetLastError();
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

extern "C" size_t spd_op_beam_select_scratch_bytes(int32_t n_groups, int32_t n_in, int32_t n_out, int32_t vocab) {
    if (n_groups <= 0 || n_in <= 0 || n_out <= 0 || vocab <= 0) return 0;
    const size_t parts = (size_t)n_groups * n_in * (((size_t)vocab + SLICE - 1) / SLICE);
    return up256(parts * n_out * 8) + 2 * up256(parts * 4);
}

extern "C" int spd_op_beam_select(int32_t dtype, const void *logits, int64_t row_stride, int32_t n_groups, int32_t n_in, int32_t n_out, int32_t vocab,
                                  const float *scores, const int32_t *ended, int32_t end_token, float tau, float *out_scores, int32_t *out_tokens,
                                  int32_t *out_parents, int32_t *out_ended, void *scratch, size_t scratch_bytes, void *hip_stream) {
    if (dtype != SPD_DTYPE_FP32 && dtype != SPD_DTYPE_BF16 && dtype != SPD_DTYPE_FP16) return SPD_EINVAL;
    if (n_groups < 0 || n_in < 1 || n_in > SPD_K_MAX || n_out < 1 || n_out > SPD_K_MAX || vocab < 1 || vocab > (1 << 30)) return SPD_EINVAL;
    if (!(tau > 0.f) || !(tau < INFINITY) || !(1.4426950408889634f / tau < INFINITY) || row_stride < vocab) return SPD_EINVAL;
    if (ended && (end_token < 0 || end_token >= vocab)) return SPD_EINVAL;
    if (n_groups == 0) return SPD_OK;
    if (!logits || !scores || !out_scores || !out_tokens || !out_parents || (uintptr_t)logits % (dtype == SPD_DTYPE_FP32 ? 4 : 2)) return SPD_EINVAL;
    if (!scratch || (uintptr_t)scratch % 256) return SPD_EINVAL;
    if (scratch_bytes < spd_op_beam_select_scratch_bytes(n_groups, n_in, n_out, vocab)) return SPD_EWORKSPACE;
    SelectArgs a{logits, row_stride, n_groups, n_in, n_out, vocab, scores, ended, end_token, tau, out_scores, out_tokens, out_parents, out_ended,
                 (vocab + SLICE - 1) / SLICE, nullptr, nullptr, nullptr};
    const long long parts = (long long)n_groups * n_in * a.slices;
    if (parts > INT32_MAX) return SPD_EINVAL;
    a.best = (u64 *)scratch;
    a.top = (float *)((char *)scratch + up256((size_t)parts * n_out * 8));
    a.sum = (float *)((char *)a.top + up256((size_t)parts * 4));
    hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch_select<float>(s, a) : dtype == SPD_DTYPE_FP16 ? launch_select<half_t>(s, a) : launch_select<bf16_t>(s, a);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}
