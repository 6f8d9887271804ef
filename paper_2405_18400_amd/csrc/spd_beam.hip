// Beam search's selection: the best continuations of a group's beams over the vocabulary.
//
// Within a row the order of continuations is that of its logits; the log-sum-exp and the beam's
// score move all of them alike.  So one pass over the logits leaves, per slice of a row, the
// n_out best (sort keys, exact) with the slice's maximum and sum of exponentials, and a second,
// small kernel puts a row's slices together and ranks what is left of a group, at most n_in * n_out
// continuations.  Scores are put together and compared in 64 bits, but a row's sum of exponentials is an fp32 sum of
// the hardware's exponentials (2^-23 of each) and its logarithm fp32 (2^-24): some 1e-7 in a score, a fifth of the rounding of its
// result at a score of ten.  Within a row it changes nothing; equal rows have equal sums; continuations of different rows that are nearer to each other may
// change places.  Exponentials in 64 bits would cost several times the eight instructions that a logit takes now.
// A wave has a slice to itself, all of it in registers, NE entries per lane: no barrier anywhere, and the selection is paid once per
// wave.  128 rows of 50258 (22.5 MB read of 112 of them, 3.6 us at a large read's rate): 18.7 us with 64-bit keys for every
// entry, 9.2 with keys for those alone that can be among the best; 64 rows of 131072 in bf16 22.8 -> 9.9.  The second kernel, a chain of
// dependent steps in one block per group: 15.5 -> 6.6 and 34 -> 9.8 us.
#include "spd_device.h"

using namespace spdd;

namespace {

typedef unsigned long long u64;

constexpr int NTB = 256, NWB = NTB / WAVE;       // slices: threads and waves per block
constexpr int NTM = 1024;                        // merge: a wave per row
constexpr int EM = 8;                            // keys per lane and turn there
// Waves of the first kernel that the GPU holds at once, for each number of entries per lane: 256 compute units of four SIMDs, by the registers.
constexpr int CUS = 256;
constexpr int waves_per_simd(int ne) { return ne <= 16 ? 8 : ne == 32 ? 3 : 2; }

// Order of fp32 numbers as unsigned ones.
__device__ __forceinline__ uint32_t ordered(float z) {
    const uint32_t u = __float_as_uint(z);
    return (int32_t)u < 0 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float((int32_t)o < 0 ? o & 0x7FFFFFFFu : ~o); }

// Larger is better: higher logit (-0 is 0), then lower id.  0: no entry.
__device__ __forceinline__ u64 sort_key(float z, int id) { return ((u64)ordered(z + 0.f) << 32) | (0xFFFFFFFFu - (uint32_t)id); }
__device__ __forceinline__ float key_logit(u64 k) { return from_ordered((uint32_t)(k >> 32)); }
__device__ __forceinline__ int key_id(u64 k) { return (int)(0xFFFFFFFFu - (uint32_t)k); }

// A logit as it counts: what is no number (a signalling NaN too, which a maximum or median would hand on) is excluded, +inf is the largest number.
__device__ __forceinline__ float clean(float z) { return z >= -3.402823466e38f ? fminf(z, 3.402823466e38f) : -INFINITY; }

__device__ __forceinline__ int lanes_below(u64 mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }
// Over the wave, by the vector unit's own lane-crossing moves: a third of the time of six trips through the LDS crossbar.
__device__ __forceinline__ float all_max(float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_max_last(v)), WAVE - 1)); }
__device__ __forceinline__ float all_sum(float v) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_sum_last(v)), WAVE - 1)); }
// log x for x > 0: of the mantissa, at most 1, in fp32 (2^-24 off), of the power of two in 64 bits.
__device__ __forceinline__ double log_of(float x) {
    return 0.69314718055994531 * ((double)__builtin_amdgcn_frexp_expf(x) + (double)__builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(x)));
}
__device__ __forceinline__ void lds_written() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The n-th largest of the lanes' 16-bit numbers.
__device__ __forceinline__ uint32_t nth_upper(uint32_t x, int n) {
    uint32_t bound = 0;
#pragma unroll
    for (int b = 15; b >= 0; --b) {
        const uint32_t t = bound | (1u << b);
        if (__popcll(__ballot(x >= t)) >= n) bound = t;
    }
    return bound;
}

// Numbers of a wave's list that may be among its n largest values v (N per lane; -inf: none there), at most WAVE: put(place, e) stores what
// stands for entry e.  Returns their number; more than WAVE: there are too many.  Of equal values those with the lower index (j, lane, x),
// e = j * VEC + x, come first.
//   * The n-th largest of the lanes' maxima, cut to its upper 16 bits, bounds the n-th largest value from below: 16 ballots.  About n
//     entries are not below it.
//   * Many equal values (masks of a finite number, ties): strictly above the bound there are few, and of the equal ones the first are taken.
//   * Otherwise (few lanes hold all large values) the n-th largest value itself is found bit by bit.
template <int N, int VEC, typename F>
__device__ __forceinline__ int wave_candidates(const float (&v)[N], float top, int n, F &&put) {   // top: this lane's largest
    const uint32_t bound = nth_upper(ordered(top) >> 16, n);
    const auto above = [&](float t) {            // (t is -inf at least: what is excluded is never above it)
        int at = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const u64 m = __ballot(v[e] > t);
            if (m) {
                const int place = at + lanes_below(m);
                if (v[e] > t && place < WAVE) put(place, e);
                at += __popcll(m);
            }
        }
        return at;
    };
    constexpr uint32_t LEAST = 0x007Fu;          // the upper bits of -inf's order
    // the number in front of the bound; in front of 0 that is not -0, which equals it
    const float below = bound <= LEAST ? -INFINITY : from_ordered((bound << 16) - (bound == 0x8000u ? 2u : 1u));
    int at = above(below);
    if (at <= WAVE) return at;
    float t = bound <= LEAST ? -INFINITY : from_ordered(bound << 16);
    at = above(t);
    if (at > WAVE) {
        uint32_t o = 0;
        for (int b = 31; b >= 0; --b) {
            const uint32_t c = o | (1u << b);
            int count = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) count += __popcll(__ballot(ordered(v[e] + 0.f) >= c));
            if (count >= n) o = c;
        }
        t = from_ordered(o);
        at = above(t);
    }
    if (at >= n || t == -INFINITY) return at;
#pragma unroll
    for (int j = 0; j < N / VEC; ++j) {          // the first n - at of those equal to t
        if (at < n) {
            u64 m[VEC];
            int place = at, all = 0;
#pragma unroll
            for (int x = 0; x < VEC; ++x) {
                m[x] = __ballot(v[j * VEC + x] == t);
                place += lanes_below(m[x]);
                all += __popcll(m[x]);
            }
#pragma unroll
            for (int x = 0; x < VEC; ++x)
                if (v[j * VEC + x] == t) {
                    if (place < n) put(place, j * VEC + x);
                    ++place;
                }
            at = min(at + all, n);
        }
    }
    return at;
}

// The n best of the first `count` keys of a list (LDS, this wave's), best first; lane i returns the i-th, 0 past the last.  `best`: n keys of this wave's.
__device__ __forceinline__ u64 ranked(u64 *list, int count, int n, u64 *best) {
    const int lane = threadIdx.x & (WAVE - 1);
    if (lane < n) best[lane] = 0;
    if (lane >= count && lane < ((count + 3) & ~3)) list[lane] = 0;
    lds_written();
    const u64 mine = lane < count ? list[lane] : 0;
    int rank = 0;
    for (int i = 0; i < count; i += 4) {         // (four at a time: one wait for their way from LDS)
        const u64 a = list[i], b = list[i + 1], c = list[i + 2], d = list[i + 3];
        rank += (a > mine) + (b > mine) + (c > mine) + (d > mine);
    }
    if (mine && rank < n) best[rank] = mine;
    lds_written();
    const u64 k = lane < n ? best[lane] : 0;
    lds_written();
    return k;
}

// A wave's entries: their largest, that of this lane, and this lane's sum of exp2((z - largest) c).  A NaN or +inf among them leaves no number in
// the sum; only then are they looked at one by one and replaced (clean(): three of the twelve instructions an entry would cost).
template <int N>
__device__ __forceinline__ void statistics(float (&z)[N], float c, float &top, float &largest, float &sum) {
    const auto all = [&]() {
        top = z[0];
#pragma unroll
        for (int e = 1; e < N; ++e) top = fmaxf(top, z[e]);
        largest = all_max(top);
        const float ref = largest == -INFINITY ? 0.f : largest;
        float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < N; ++e) part[e % 4] += __builtin_amdgcn_exp2f((z[e] - ref) * c);
        sum = (part[0] + part[1]) + (part[2] + part[3]);
    };
    all();
    if (__any(sum != sum)) {
#pragma unroll
        for (int e = 0; e < N; ++e) z[e] = clean(z[e]);
        all();
    }
}

__device__ __forceinline__ bool row_runs(const SelectArgs &a, int row) {
    const float score = as_global(a.scores)[row];
    return score > -INFINITY && !(a.ended && as_global(a.ended)[row] != 0);       // (a score that is no number: no beam)
}

// VEC logits of a lane, which lie side by side.
template <typename LT, int VEC> __device__ __forceinline__ void load_logits(const char *p, float *f) {
    if constexpr (VEC == Store<LT>::VEC) Store<LT>::unpack(global_load16(p), f);
    else if constexpr (sizeof(LT) == 4) {
        const u32x2 v = *(const u32x2 __attribute__((address_space(1))) *)p;
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y);
    } else {
        float g[8];
        const uint32_t v = *(const uint32_t __attribute__((address_space(1))) *)p;
        Store<LT>::unpack(u32x4{v, 0, 0, 0}, g);
        f[0] = g[0]; f[1] = g[1];
    }
}

// A wave per slice of 64 NE entries; lane l's vector j holds entries VEC (64 j + l) ...
template <typename LT, int NE, int VEC>
__global__ __launch_bounds__(NTB, waves_per_simd(NE)) void beam_slice_kernel(const SelectArgs a) {
    __shared__ u64 list[NWB][WAVE], best[NWB][SPD_K_MAX];
    const int lane = threadIdx.x & (WAVE - 1), w = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
    const int part = blockIdx.x * NWB + w, row = part / a.slices, slice = part - row * a.slices;
    if (row >= a.n_groups * a.n_in) return;
    const char *z_row = (const char *)a.logits + (size_t)row * a.row_stride * sizeof(LT);
    const int lo = slice * WAVE * NE + lane * VEC;
    const auto id = [&](int e) { return lo + (e / VEC) * WAVE * VEC + e % VEC; };
    float z[NE];
    if (slice * WAVE * NE + WAVE * NE <= a.vocab) {
#pragma unroll
        for (int j = 0; j < NE / VEC; ++j) {
            if constexpr (VEC == 1) z[j] = Store<LT>::load1(z_row, id(j));
            else load_logits<LT, VEC>(z_row + (size_t)id(j * VEC) * sizeof(LT), &z[j * VEC]);
        }
    } else {
#pragma unroll
        for (int e = 0; e < NE; ++e) z[e] = id(e) < a.vocab ? Store<LT>::load1(z_row, id(e)) : -INFINITY;
    }
    if (!row_runs(a, row)) return;               // (looked at while the logits are under way: a trip to memory less)
    float top, m, sum;
    statistics(z, a.log2_by_tau, top, m, sum);
    sum = all_sum(sum);
    const int count = wave_candidates<NE, VEC>(z, top, a.n_out, [&](int place, int e) { list[w][place] = sort_key(z[e], id(e)); });
    const u64 k = ranked(list[w], count, a.n_out, best[w]);
    if (lane < a.n_out) ((global_ptr<u64>)a.best)[(size_t)part * a.n_out + lane] = k;
    if (lane == 0) { as_global(a.top)[part] = m; as_global(a.sum)[part] = sum; }
}

// What a group's block keeps of its rows: up to n_out continuations of each, best first, by place beam * n_out + rank.
constexpr int MOST = SPD_K_MAX * SPD_K_MAX;
struct Group {
    u64 list[SPD_K_MAX][WAVE], best[SPD_K_MAX][SPD_K_MAX];
    double score[MOST], c_score[MOST];
    int token[MOST], chosen[MOST], ended[SPD_K_MAX], count;
};

// This wave's row: its best keys (lane i: the i-th, 0 where there is none), largest logit and sum of exponentials -> its continuations' scores.
__device__ __forceinline__ void put_row(const SelectArgs &a, Group &s, int b, float row_score, u64 kept, float M, float sum) {
    const int lane = threadIdx.x & (WAVE - 1);
    if (lane >= a.n_out) return;
    const double lse = (double)M * a.by_tau + (sum > 0.f ? log_of(sum) : 0.0);
    s.score[b * a.n_out + lane] = kept ? (double)row_score + ((double)key_logit(kept) * a.by_tau - lse) : -INFINITY;
    s.token[b * a.n_out + lane] = key_id(kept);
}
// An ended beam goes on as it is; an absent one has no continuation.
__device__ __forceinline__ void put_no_row(const SelectArgs &a, Group &s, int b, float row_score, bool ended) {
    const int lane = threadIdx.x & (WAVE - 1);
    if (lane >= a.n_out) return;
    s.score[b * a.n_out + lane] = ended && lane == 0 && row_score > -INFINITY ? (double)row_score : -INFINITY;
    s.token[b * a.n_out + lane] = a.end_token;
}

// The group's continuations in order, by all threads of its block (any number of waves).
__device__ __forceinline__ void rank_group(const SelectArgs &a, Group &s, int g) {
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), n = a.n_in * a.n_out;
    __syncthreads();
    // those that can be among the best by their scores in fp32 (rounding keeps the order)
    int present = 0;
    if (tid < WAVE) {
        float v[MOST / WAVE], top = -INFINITY;
#pragma unroll
        for (int e = 0; e < MOST / WAVE; ++e) {
            const int at = lane * (MOST / WAVE) + e;
            const double x = at < n ? s.score[at] : -INFINITY;
            present += __popcll(__ballot(x > -INFINITY));
            v[e] = x > -INFINITY ? fmaxf((float)x, -3.402823466e38f) : -INFINITY;
            top = fmaxf(top, v[e]);
        }
        const int count = wave_candidates<MOST / WAVE, MOST / WAVE>(v, top, a.n_out, [&](int place, int e) { s.chosen[place] = lane * (MOST / WAVE) + e; });
        // equal ones in fp32 may differ in 64 bits: where some were left out for being equal, all are looked at
        int reach = 0;
        float least = INFINITY;
        lds_written();
        if (lane < min(count, WAVE)) least = fmaxf((float)s.score[s.chosen[lane]], -3.402823466e38f);
        least = -all_max(-least);
#pragma unroll
        for (int e = 0; e < MOST / WAVE; ++e) reach += __popcll(__ballot(v[e] >= least && v[e] > -INFINITY));
        const bool few = count <= WAVE && reach == count;
        if (few && lane < count) s.c_score[lane] = s.score[s.chosen[lane]];
        if (few && lane >= count && lane < ((count + 3) & ~3)) { s.c_score[lane] = -INFINITY; s.chosen[lane] = MOST; }
        if (lane == 0) s.count = few ? count : -1;
    }
    __syncthreads();
    const int few = s.count;
    if (few < 0) {
        for (int i = tid; i < MOST; i += blockDim.x) {
            s.chosen[i] = i;
            s.c_score[i] = i < n ? s.score[i] : -INFINITY;
        }
        __syncthreads();
    }
    const int of = few < 0 ? n : few;
    for (int q = tid; q < of; q += blockDim.x) {
        const int at = s.chosen[q];
        const double mine = s.c_score[q];
        int rank = 0;
        for (int i = 0; i < of; i += 4) {
            const double o0 = s.c_score[i], o1 = s.c_score[i + 1], o2 = s.c_score[i + 2], o3 = s.c_score[i + 3];
            // (continuations lie by beam, those of a beam by logit and id: among equals the lower place goes first)
            const int p0 = s.chosen[i], p1 = s.chosen[i + 1], p2 = s.chosen[i + 2], p3 = s.chosen[i + 3];
            rank += (o0 > mine || (o0 == mine && p0 < at)) + (o1 > mine || (o1 == mine && p1 < at));
            rank += (o2 > mine || (o2 == mine && p2 < at)) + (o3 > mine || (o3 == mine && p3 < at));
        }
        if (mine > -INFINITY && rank < a.n_out) {
            const int to = g * a.n_out + rank, tok = s.token[at], beam = at / a.n_out;
            as_global(a.out_scores)[to] = (float)mine;
            as_global(a.out_tokens)[to] = tok;
            as_global(a.out_parents)[to] = beam;
            if (a.out_ended) as_global(a.out_ended)[to] = s.ended[beam] || tok == a.end_token;
        }
    }
    if (tid < a.n_out && tid >= present) {                        // fewer continuations than asked for
        const int to = g * a.n_out + tid;
        as_global(a.out_scores)[to] = -INFINITY;
        as_global(a.out_tokens)[to] = 0;
        as_global(a.out_parents)[to] = tid < a.n_in ? tid : 0;
        if (a.out_ended) as_global(a.out_ended)[to] = 0;
    }
}

// One block per group, a wave per row, over the slices' results.
__global__ __launch_bounds__(NTM) void beam_merge_kernel(const SelectArgs a) {
    __shared__ Group s;
    const int lane = threadIdx.x & (WAVE - 1), b = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), g = blockIdx.x, row = g * a.n_in + b;
    // asked for at once (a row that does not run has nothing there: what comes is not looked at)
    const size_t part = (size_t)row * a.slices;
    const u64 *keys = a.best + part * a.n_out;
    const int n = a.slices * a.n_out;
    u64 key[EM], kept = 0;                                        // kept, lane i: the i-th best so far
    const auto fetch = [&](int i0) {
#pragma unroll
        for (int e = 0; e < EM; ++e) {
            const int i = i0 + EM * lane + e;                     // (a lane's keys are a stretch of a sorted list: its first is a good bound)
            key[e] = i < n ? ((global_ptr<const u64>)keys)[i] : 0;
        }
    };
    fetch(0);
    const float first_top = lane < a.slices ? as_global(a.top)[part + lane] : -INFINITY, first_sum = lane < a.slices ? as_global(a.sum)[part + lane] : 0.f;
    const float row_score = as_global(a.scores)[row];
    const bool ended = a.ended && as_global(a.ended)[row] != 0;
    if (lane == 0) s.ended[b] = ended;
    if (row_score > -INFINITY && !ended) {                        // (a score that is no number: no beam)
        const float c = a.log2_by_tau;
        float M = -INFINITY, sum = 0.f;
        for (int i = lane; i < a.slices; i += WAVE) {
            const float t = i < WAVE ? first_top : as_global(a.top)[part + i], x = i < WAVE ? first_sum : as_global(a.sum)[part + i];
            if (t == -INFINITY) continue;
            const float up = fmaxf(M, t);
            sum = sum * (M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((M - up) * c)) + x * __builtin_amdgcn_exp2f((t - up) * c);
            M = up;
        }
        const float mine = M;
        M = all_max(M);
        sum = all_sum(mine == -INFINITY ? 0.f : sum * __builtin_amdgcn_exp2f((mine - M) * c));
        for (int i0 = 0; i0 < n; i0 += EM * WAVE) {
            if (i0) fetch(i0);
            u64 top = kept;
#pragma unroll
            for (int e = 0; e < EM; ++e) top = key[e] > top ? key[e] : top;
            const uint32_t bound = nth_upper((uint32_t)(top >> 48), a.n_out);
            const auto from = [&](u64 least) {                    // the keys not below `least`
                int at = 0;
#pragma unroll
                for (int e = 0; e <= EM; ++e) {
                    const u64 k = e ? key[e - 1] : kept;
                    const bool in = k >= least;
                    const u64 m = __ballot(in);
                    if (m) {
                        const int place = at + lanes_below(m);
                        if (in && place < WAVE) s.list[b][place] = k;
                        at += __popcll(m);
                    }
                }
                return at;
            };
            int count = from(bound ? (u64)bound << 48 : 1);
            if (count > WAVE) {                                   // many equal logits: the n-th largest key itself
                u64 least = 0;
                for (int q = 63; q >= 0; --q) {
                    const u64 t = least | (1ull << q);
                    int c = __popcll(__ballot(kept >= t));
#pragma unroll
                    for (int e = 0; e < EM; ++e) c += __popcll(__ballot(key[e] >= t));
                    if (c >= a.n_out) least = t;
                }
                count = from(least);
            }
            kept = ranked(s.list[b], count, a.n_out, s.best[b]);
        }
        put_row(a, s, b, row_score, kept, M, sum);
    } else {
        put_no_row(a, s, b, row_score, ended);
    }
    rank_group(a, s, g);
}

// Small vocabularies, all in one launch: a block per group, a wave per row, 64 * 32 entries at a time in registers.
constexpr int SMALL_NE = 32, SMALL = 4096;
template <typename LT>
__global__ __launch_bounds__(NTM) void beam_small_kernel(const SelectArgs a) {
    __shared__ Group s;
    const int lane = threadIdx.x & (WAVE - 1), b = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE), g = blockIdx.x, row = g * a.n_in + b;
    const char *z_row = (const char *)a.logits + (size_t)row * a.row_stride * sizeof(LT);
    float z[SMALL_NE];
    const auto fetch = [&](int lo) {
#pragma unroll
        for (int e = 0; e < SMALL_NE; ++e) {
            const int i = lo + e * WAVE + lane;
            z[e] = i < a.vocab ? Store<LT>::load1(z_row, i) : -INFINITY;
        }
    };
    fetch(0);
    const float row_score = as_global(a.scores)[row];
    const bool ended = a.ended && as_global(a.ended)[row] != 0;
    if (lane == 0) s.ended[b] = ended;
    if (row_score > -INFINITY && !ended) {
        const float c = a.log2_by_tau;
        float M = -INFINITY, sum = 0.f;
        u64 kept = 0;
        for (int lo = 0; lo < a.vocab; lo += SMALL_NE * WAVE) {
            if (lo) fetch(lo);
            float top, m, more;
            statistics(z, c, top, m, more);
            const float up = fmaxf(M, m), ref = up == -INFINITY ? 0.f : up;
            sum = sum * __builtin_amdgcn_exp2f((M - ref) * c) + more * __builtin_amdgcn_exp2f((m - ref) * c);    // (of nothing: 0 times 0)
            M = up;
            const int count = wave_candidates<SMALL_NE, 1>(z, top, a.n_out, [&](int place, int e) { s.list[b][place] = sort_key(z[e], lo + e * WAVE + lane); });
            const u64 before = kept;
            kept = ranked(s.list[b], count, a.n_out, s.best[b]);
            if (lo) {                                             // with those of the entries before
                if (lane < a.n_out) { s.list[b][lane] = before; s.list[b][a.n_out + lane] = kept; }
                kept = ranked(s.list[b], 2 * a.n_out, a.n_out, s.best[b]);
            }
        }
        put_row(a, s, b, row_score, kept, M, all_sum(sum));
    } else {
        put_no_row(a, s, b, row_score, ended);
    }
    rank_group(a, s, g);
}

// Entries per lane of a slice.  The first kernel takes a round for as many waves as the GPU holds, some 1.5 us and 0.05 per entry; the second a turn for every EM * 64 keys
// that a row's slices leave, 2 us and, where many of them are kept, more, and 10 us more where more than a wave's worth of keys come from so few slices that a
// lane holds half a slice's and the first halves alone are fewer than n_out.  So, counted in entries, rounds * (32 + entries) + 96 * turns + 200 there, and the least of it.
// Measured over 160 calls of 1 to 512 rows of 5000 to 256000, fp32 and bf16, n_out 4 to 16: on (geometric) average 1.3% over each call's best, 12% under a
// bound on the waves alone (of single calls 35% less to 14% more); 16 or 64 in place of 32, 32 or 64 in place of 96, 100 or 300 in place of 200 are within half a percent.
// us at 8 / 16 / 32 / 64 entries: 128 rows of 32000 in fp32 14.0 / 13.3 / 13.5 / 14.5, 16 of 131072 17.5 / 13.5 / 11.5 / 12.3, 512 of 16000 in bf16
// 17.9 / 15.4 / 19.4 / 21.7; 64 of 5000, 16 of each kept, 26 / 27 / 14.5 / 15.8.
int entries_per_lane(long long rows, int vocab, int n_out) {
    int best = 0;
    long long least = 0;
    for (int ne = 8; ne <= 64; ne *= 2) {
        const long long slices = ((long long)vocab + WAVE * ne - 1) / (WAVE * ne), places = CUS * 4 * waves_per_simd(ne), keys = slices * n_out;
        const bool halves = n_out > EM && keys > WAVE && slices <= n_out;
        const long long cost = (rows * slices + places - 1) / places * (32 + ne) + (keys + EM * WAVE - 1) / (EM * WAVE) * 96 + (halves ? 200 : 0);
        if (best == 0 || cost < least) { best = ne; least = cost; }
    }
    return best;
}

template <typename LT, int VEC>
void launch_slices(hipStream_t s, const SelectArgs &a, int ne, unsigned blocks) {
    if (ne == 8) hipLaunchKernelGGL((beam_slice_kernel<LT, 8, VEC>), dim3(blocks), dim3(NTB), 0, s, a);
    else if (ne == 16) hipLaunchKernelGGL((beam_slice_kernel<LT, 16, VEC>), dim3(blocks), dim3(NTB), 0, s, a);
    else if (ne == 32) hipLaunchKernelGGL((beam_slice_kernel<LT, 32, VEC>), dim3(blocks), dim3(NTB), 0, s, a);
    else hipLaunchKernelGGL((beam_slice_kernel<LT, 64, VEC>), dim3(blocks), dim3(NTB), 0, s, a);
}

template <typename LT>
hipError_t launch_select(hipStream_t s, const SelectArgs &a, int ne) {
    if (a.vocab <= SMALL) {
        hipLaunchKernelGGL(beam_small_kernel<LT>, dim3(a.n_groups), dim3(a.n_in * WAVE), 0, s, a);
        return hipGetLastError();
    }
    const unsigned blocks = (unsigned)(((long long)a.n_groups * a.n_in * a.slices + NWB - 1) / NWB);
    // as many logits per load as the rows' addresses allow
    const auto on = [&](int bytes) { return (uintptr_t)a.logits % bytes == 0 && (a.n_groups * a.n_in == 1 || a.row_stride * (int64_t)sizeof(LT) % bytes == 0); };
    if (on(16)) launch_slices<LT, Store<LT>::VEC>(s, a, ne, blocks);
    else if (on(2 * sizeof(LT))) launch_slices<LT, 2>(s, a, ne, blocks);
    else launch_slices<LT, 1>(s, a, ne, blocks);
    hipLaunchKernelGGL(beam_merge_kernel, dim3(a.n_groups), dim3(a.n_in * WAVE), 0, s, a);
    return hipGetLastError();
}

size_t up256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

extern "C" size_t spd_op_beam_select_scratch_bytes(int32_t n_groups, int32_t n_in, int32_t n_out, int32_t vocab) {
    if (n_groups <= 0 || n_in <= 0 || n_out <= 0 || vocab <= SMALL) return 0;
    const long long rows = (long long)n_groups * n_in;
    const int slice = WAVE * entries_per_lane(rows, vocab, n_out);
    const size_t parts = (size_t)rows * (((size_t)vocab + slice - 1) / slice);
    return up256(parts * n_out * 8) + 2 * up256(parts * 4);
}

extern "C" int spd_test_beam_select_cut(int32_t n_groups, int32_t n_in, int32_t n_out, int32_t vocab, int32_t *out) {
    if (!out || n_groups <= 0 || n_in <= 0 || n_out <= 0 || vocab <= 0) return SPD_EINVAL;
    out[0] = vocab <= SMALL ? 0 : entries_per_lane((long long)n_groups * n_in, vocab, n_out);
    out[1] = vocab <= SMALL ? 1 : (vocab + WAVE * out[0] - 1) / (WAVE * out[0]);
    return SPD_OK;
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
    const size_t need = spd_op_beam_select_scratch_bytes(n_groups, n_in, n_out, vocab);
    if (need && (!scratch || (uintptr_t)scratch % 256)) return SPD_EINVAL;
    if (scratch_bytes < need) return SPD_EWORKSPACE;
    // a group's outputs may take the place of its own scores or ended, and lie apart from everything else that is read or written
    const size_t in_bytes = (size_t)n_groups * n_in * 4, out_bytes = (size_t)n_groups * n_out * 4;
    const spdk::Span sz{logits, ((size_t)(n_groups * (size_t)n_in - 1) * row_stride + vocab) * (dtype == SPD_DTYPE_FP32 ? 4 : 2)}, sw{scratch, need}, ss{scores, in_bytes}, sd{ended, in_bytes},
        outs[4] = {{out_scores, out_bytes}, {out_tokens, out_bytes}, {out_parents, out_bytes}, {out_ended, out_bytes}};
    const auto unless_same = [&](const spdk::Span &in, const spdk::Span &out) { return in.p == out.p && n_in == n_out ? spdk::Span{} : in; };
    for (int i = 0; i < 4; ++i) {
        if (spdk::over_any(outs[i], {sz, sw, unless_same(ss, outs[i]), unless_same(sd, outs[i])})) return SPD_EINVAL;
        for (int j = i + 1; j < 4; ++j)
            if (spdk::over_any(outs[i], {outs[j]})) return SPD_EINVAL;
    }
    if (spdk::over_any(sw, {sz, ss, sd})) return SPD_EINVAL;
    const int ne = entries_per_lane((long long)n_groups * n_in, vocab, n_out), slice = WAVE * ne;
    SelectArgs a{logits, row_stride, n_groups, n_in, n_out, vocab, scores, ended, end_token, 1.4426950408889634f / tau, 1.0 / (double)tau, out_scores, out_tokens, out_parents, out_ended,
                 (vocab + slice - 1) / slice, nullptr, nullptr, nullptr};
    const long long parts = (long long)n_groups * n_in * a.slices;
    if (parts > INT32_MAX - NWB) return SPD_EINVAL;
    a.best = (u64 *)scratch;
    a.top = (float *)((char *)scratch + up256((size_t)parts * n_out * 8));
    a.sum = (float *)((char *)a.top + up256((size_t)parts * 4));
    hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch_select<float>(s, a, ne) : dtype == SPD_DTYPE_FP16 ? launch_select<half_t>(s, a, ne) : launch_select<bf16_t>(s, a, ne);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}
