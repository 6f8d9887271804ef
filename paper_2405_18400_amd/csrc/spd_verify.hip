// Verification of drafted tokens against the target's probabilities, and the draw of the token behind those that stand.
//
// Bound: every row of logits is read once, whatever stands (which rows count hangs on the rows before them), and the one row that a sequence's last token
// is drawn from three times more.  Four launches:
//   * slices of all rows: largest logit and sum of exponentials, in fp32;
//   * a block per slice and sequence puts its sequence's rows together, finds the first draft that does not stand (with sums of 64 bits where those of 32 might be wrong), and sums its slice of that row again, in 64 bits;
//   * the same blocks sum what that row leaves, max(p - q, 0);
//   * a block per sequence finds the slice where the draw falls, and the token in it.
// Whether a draft stands is one comparison, which sums of fp32 exponentials hardly ever turn: those that they might (their error is bounded) are made again with sums of 64 bits.  The draw falls between as many
// borders as there are tokens: of a hundred thousand, one in a thousand draws meets one that such sums have moved.  So that row is in 64 bits always; all rows in 64 bits took 61 us where fp32 takes what reading takes.
// Measured, the four in turn: 32 sequences with 190 tokens, 131072 logits in bf16, 100 MB in all: 24.9 us (3.7 TB/s; vector unit 70% busy), 21.6 and 14.6 (vector unit 50% busy, exponentials in 64 bits), 11.2 (a
// block's chain of trips and sums); one sequence of five tokens, 32000 logits in fp32: 3.7, 9.9, 5.2 and 8.4, chains all of them.
#include "spd_attention.h"

#include <algorithm>

using namespace spdd;
using namespace spda;

namespace {

constexpr int NTV = 256, NWV = NTV / WAVE;

// A logit as it counts: no number is -inf, +inf the largest finite number.
__device__ __forceinline__ float logit(float x) { return fminf(fmaxf(x, -INFINITY), 3.402823466e38f); }

// 2^(d c), d c < 1000, in 64 bits: to the nearest power of two by adding 1.5 2^52, which leaves the whole number in the low bits, and a rest of at most 1/2, whose
// exponential is ten terms of its series; the next one is 2e-13.  (As conversions and ldexp these steps take the time of twice as many products.)  What is below 2^-1021 is 0.
__device__ __forceinline__ double exp2_64(double d, double c) {
    constexpr double MAGIC = 6755399441055744.0, L = 0.69314718055994530942;
    constexpr double C[11] = {1.0, L, L * L / 2, L * L * L / 6, L * L * L * L / 24, L * L * L * L * L / 120, L * L * L * L * L * L / 720, L * L * L * L * L * L * L / 5040,
                              L * L * L * L * L * L * L * L / 40320, L * L * L * L * L * L * L * L * L / 362880, L * L * L * L * L * L * L * L * L * L / 3628800};
    const double t = fma(d, c, MAGIC), f = fma(d, c, -(t - MAGIC));
    double y = C[10];
#pragma unroll
    for (int n = 9; n >= 0; --n) y = fma(y, f, C[n]);
    const u64 bits = __builtin_bit_cast(u64, y) + ((u64)(uint32_t)__builtin_bit_cast(u64, t) << 52);       // (the exponent's place: modulo 2^12)
    return d * c >= -1021.0 ? __builtin_bit_cast(double, bits) : 0.0;             // (0 for -inf too)
}

// exp((z - top) / tau), c = log2(e) / tau, z <= top.
__device__ __forceinline__ double exp_64(float z, float top, double c) { return exp2_64((double)z - (double)top, c); }

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

// N numbers' sums over the block, each by one thread to `out`.
template <int N> __device__ __forceinline__ void block_adds(const double (&v)[N], double (*red)[NWV], double *out) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const double x = wave_add(v[i]);
        if (threadIdx.x % WAVE == 0) red[i][threadIdx.x / WAVE] = x;
    }
    __syncthreads();
    if (threadIdx.x < N) out[threadIdx.x] = (red[threadIdx.x][0] + red[threadIdx.x][1]) + (red[threadIdx.x][2] + red[threadIdx.x][3]);
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
    __shared__ float tops[NWV], red[NWV];
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), wv = tid / WAVE, r = blockIdx.x / a.slices, slice = blockIdx.x - r * a.slices;
    const bool draft = r >= a.n_tokens;
    const int t = draft ? r - a.n_tokens : r;
    // rows that nothing asks about: no sequence's, and the drafter's at a sequence's last token
    bool last = false, inside = false;
    for (int i = lane; i <= a.n_seq; i += WAVE) {
        const int f = as_global(a.first)[i];
        last = last || f == t + 1;
        inside = inside || (i == 0 && f <= t);
    }
    if (!__any(inside) || t >= as_global(a.first)[a.n_seq] || (draft && __any(last))) return;
    const void *row = draft ? row_of<T>(a.draft_logits, a.draft_stride, t) : row_of<T>(a.logits, a.row_stride, t);
    const float c = (float)(draft ? a.by_draft_tau : a.by_tau);
    float z[PIECES][VEC], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) load_logits<T, VEC>(row, (slice * PIECES + i) * NTV * VEC + tid * VEC, a.vocab, z[i]);
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) top = fmaxf(top, z[i][e]);
    top = wave_max(top);
    if (lane == 0) tops[wv] = top;
    __syncthreads();
    top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
    const float from = top == -INFINITY ? 0.f : top;
    float sum = 0.f, all = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float x = __builtin_amdgcn_exp2f((z[i][e] - from) * c);
            all += x;
            sum += __builtin_amdgcn_fractf(x);
        }
    // One of the largest stays out: next to its 1 a likely token's log p, the logarithm of 1 and what the others add up to, would be lost.  So a thread adds up what is less than 1, and counts the ones.
    float ones = rintf(all - sum);
    if (const u64 with = __ballot(ones > 0.f)) {
        bool first = lane == __builtin_ctzll(with) && tops[wv] == top;
        for (int w = 0; w < wv; ++w) first = first && tops[w] != top;
        ones -= first ? 1.f : 0.f;
    }
    sum = wave_sum(sum + ones);
    if (lane == 0) red[tid / WAVE] = sum;
    __syncthreads();
    if (tid == 0) {
        as_global(a.top)[blockIdx.x] = top;
        as_global(a.sum)[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
    }
}

// A row's largest logit, and its sum of exponentials, by 16 lanes.  How far it may be off, in steps of 2^-24 of itself: an exponent x is off by three steps of itself, and the mean of -x, every term counting as
// much as it weighs, is at most log2 of their number, so all terms together by 3 ln 2 log2(vocab), and again as much where slices are put together; the exponential by two; the sums of a slice (E terms and nine
// joins) by one each; and two for every time that a lane's slices so far are brought down.
constexpr int ROWL = 16;
double sum_off(int each, int vocab, int slices) { return 0x1p-24 * (4.2 * log2((double)vocab) + (each + 9) + 2.0 * ((slices + ROWL - 1) / ROWL + 3)); }
__device__ __forceinline__ void whole_row(const VerifyArgs &a, int r, double c, int lane, float &top, double &sum) {
    const size_t at = (size_t)r * a.slices;
    float m = -INFINITY;                         // the lane's slices so far
    double s = 0.0;
    for (int i = lane; i < a.slices; i += ROWL) {
        const float x = as_global(a.top)[at + i], y = as_global(a.sum)[at + i], up = fmaxf(m, x);
        if (up == -INFINITY) continue;
        s = s * (double)__builtin_amdgcn_exp2f((m - up) * (float)c) + (1.0 + (double)y) * (double)__builtin_amdgcn_exp2f((x - up) * (float)c);
        m = up;
    }
    top = m;
#pragma unroll
    for (int o = 1; o < ROWL; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, WAVE));
    s = m == -INFINITY ? 0.0 : s * (double)__builtin_amdgcn_exp2f((m - top) * (float)c);
#pragma unroll
    for (int o = 1; o < ROWL; o <<= 1) s += __shfl_xor(s, o, WAVE);
    sum = s;
}

// Whether all of `first` ascends (every thread of the block looks at some of it).
__device__ __forceinline__ bool ascends(const VerifyArgs &a) {
    int descends = 0;
    for (int i = threadIdx.x; i < a.n_seq; i += NTV) descends |= as_global(a.first)[i + 1] < as_global(a.first)[i];
    return !__syncthreads_or(descends);
}

// p(x) / q(x) for the draft x behind token t, of the rows' largest logits and sums, by the difference of the two logarithms: they may lie below anything that 64 bits hold.  (Its two products without their
// roundings: they may be large and near to each other.)  0 where p(x) is, some 2^900 where q(x) is 0 or far below p(x).  below_top: how far x's logit lies below the largest, where there is one.
template <typename T>
__device__ __forceinline__ double quotient(const VerifyArgs &a, int t, int x, float top, double sum, float draft_top, double draft_sum, double &below_top) {
    if ((unsigned)x >= (unsigned)a.vocab) return 0.0;
    const float z = logit(Store<T>::load1(row_of<T>(a.logits, a.row_stride, t), x));
    float y = -INFINITY;
    if (a.draft_logits) y = logit(Store<T>::load1(row_of<T>(a.draft_logits, a.draft_stride, t), x));
    if (z == -INFINITY) return 0.0;
    below_top = (double)z - (double)top;
    if (!a.draft_logits) return exp2_64(below_top, a.by_tau) / sum;
    if (y == -INFINITY) return 0x1p900;
    const double dq = (double)y - (double)draft_top, lq = dq * a.by_draft_tau;
    return exp2_64(fmin(fma(below_top, a.by_tau, -lq) - fma(dq, a.by_draft_tau, -lq), 900.0), 1.0) * (draft_sum / sum);
}

// A row's sum of exponentials in 64 bits, by the block.
template <typename T> __device__ double exact_row(const VerifyArgs &a, const void *row, float top, double c, double *red) {
    constexpr int VEC = 16 / (int)sizeof(T);
    double sum = 0.0;
    for (int v0 = threadIdx.x * VEC; v0 < a.vocab; v0 += NTV * VEC) {
        float z[VEC];
        load_logits<T, VEC>(row, v0, a.vocab, z);
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum += exp_64(z[e], top, c);
    }
    return block_add(sum, red);
}

template <typename T, int E>
__global__ __launch_bounds__(NTV) void verify_drafts_kernel(const VerifyArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T), PIECES = E / VEC;
    __shared__ int stop, unsure;
    __shared__ double red[PIECES][NWV];
    __shared__ float last_top[2];
    const int tid = threadIdx.x, s = blockIdx.x / a.slices, slice = blockIdx.x - s * a.slices, lane = tid % ROWL;
    const bool sorted = ascends(a);
    const int lo = as_global(a.first)[s], hi = as_global(a.first)[s + 1];
    const bool fits = sorted && lo >= 0 && hi <= a.n_tokens, drawn = a.draft_logits != nullptr;
    if (!fits || lo == hi) {
        if (tid == 0 && slice == 0) {
            as_global(a.out_accepted)[s] = 0;
            a.pick[s].row = -1;
            if (!fits && a.err) *as_global(a.err) = 1;
        }
        return;
    }
    // 16 lanes per row: does its draft stand?  (Those behind the first that does not are looked at in vain.)  Where u is nearer to p / q than fp32 sums may be off, which is seldom, the block sums that draft's
    // rows in 64 bits, and goes on behind it if it stands.
    for (int from = lo;;) {
        if (tid == 0) stop = unsure = INT32_MAX;
        __syncthreads();
        for (int t0 = from; t0 < hi - 1; t0 += NTV / ROWL) {
            const int t = t0 + tid / ROWL, row = min(t, hi - 2);           // (all lanes take part in the exchange)
            float top, draft_top = -INFINITY;
            double sum, draft_sum = 0.0, below_top = 0.0;
            whole_row(a, row, a.by_tau, lane, top, sum);
            if (drawn) whole_row(a, a.n_tokens + row, a.by_draft_tau, lane, draft_top, draft_sum);
            if (lane != 0 || t >= hi - 1) continue;
            const int x = as_global(a.tokens)[t + 1];
            const double r = quotient<T>(a, t, x, top, sum, draft_top, draft_sum, below_top), u = (double)as_global(a.u)[t];
            const bool near = r > 0.0 && fabs(u - r) <= a.unsure * r;
            if (near) atomicMin(&unsure, t);
            else if (!(u < r)) atomicMin(&stop, t);
            if (slice == 0 && (near || u < r)) {
                as_global(a.out_tokens)[t] = x;
                as_global(a.out_logprobs)[t] = (float)((below_top * a.by_tau - log2(sum)) * 0.69314718055994530942);
            }
        }
        __syncthreads();
        const int t = unsure;
        if (t >= stop) break;
        float top, draft_top = -INFINITY;
        double sum, draft_sum = 0.0, below_top;
        whole_row(a, t, a.by_tau, lane, top, sum);
        sum = exact_row<T>(a, row_of<T>(a.logits, a.row_stride, t), top, a.by_tau, red[0]);
        if (drawn) {
            whole_row(a, a.n_tokens + t, a.by_draft_tau, lane, draft_top, draft_sum);
            if (draft_top > -INFINITY) draft_sum = exact_row<T>(a, row_of<T>(a.draft_logits, a.draft_stride, t), draft_top, a.by_draft_tau, red[0]);
        }
        const bool stands = (double)as_global(a.u)[t] < quotient<T>(a, t, as_global(a.tokens)[t + 1], top, sum, draft_top, draft_sum, below_top);
        __syncthreads();                         // (everyone has read the marks)
        if (!stands) {
            if (tid == 0) stop = t;
            break;
        }
        from = t + 1;
    }
    __syncthreads();
    const bool refused = stop < hi - 1;
    const int row = refused ? stop : hi - 1;
    if (tid < 2 * ROWL) {                        // the largest logits of the last row, the target's and the drafter's
        const bool draft = tid >= ROWL;
        float top;
        double sum;
        whole_row(a, draft && refused && drawn ? a.n_tokens + row : row, draft ? a.by_draft_tau : a.by_tau, lane, top, sum);
        if (lane == 0) last_top[draft] = top;
    }
    if (slice == 0)
        for (int i = row + 1 + tid; i < hi; i += NTV) {
            as_global(a.out_tokens)[i] = -1;
            as_global(a.out_logprobs)[i] = 0.f;
        }
    __syncthreads();
    if (slice == 0 && tid == 0) {
        const int x = refused ? as_global(a.tokens)[row + 1] : -1;
        a.pick[s] = VerifyPick{last_top[0], last_top[1], row, x, refused};
        as_global(a.out_accepted)[s] = row - lo;
        if (a.err && (last_top[0] == -INFINITY || (refused && (unsigned)x >= (unsigned)a.vocab))) *as_global(a.err) = 1;
    }
    // that row's sums, in 64 bits
#pragma unroll
    for (int d = 0; d < 2; ++d) {
        if (d && !(refused && drawn)) break;
        const void *z_row = d ? row_of<T>(a.draft_logits, a.draft_stride, row) : row_of<T>(a.logits, a.row_stride, row);
        const double c = d ? a.by_draft_tau : a.by_tau;
        const float top = last_top[d];
        double sum[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            float z[VEC];
            load_logits<T, VEC>(z_row, (slice * PIECES + i) * NTV * VEC + tid * VEC, a.vocab, z);
            sum[i] = 0.0;
#pragma unroll
            for (int e = 0; e < VEC; ++e) sum[i] += top == -INFINITY ? 0.0 : exp_64(z[e], top, c);
        }
        block_adds<PIECES>(sum, red, a.exact + ((size_t)d * a.n_seq + s) * a.pieces + slice * PIECES);
    }
}

// The inverses of a sequence's last row's sums (0 where no logit is finite), by the block: the target's, the drafter's.
__device__ __forceinline__ void inverses(const VerifyArgs &a, const VerifyPick &k, int s, double *red, double &inv, double &draft_inv) {
    double sum = 0.0, draft = 0.0;
    for (int i = threadIdx.x; i < a.pieces; i += NTV) {
        sum += a.exact[(size_t)s * a.pieces + i];
        if (k.refused && a.draft_logits) draft += a.exact[((size_t)a.n_seq + s) * a.pieces + i];
    }
    sum = block_add(sum, red);
    draft = block_add(draft, red);
    inv = sum > 0.0 ? 1.0 / sum : 0.0;
    draft_inv = draft > 0.0 ? 1.0 / draft : 0.0;
}

// What a sequence's last row leaves of VEC tokens from v0 on.
template <typename T, int VEC>
__device__ __forceinline__ void weights(const VerifyArgs &a, const VerifyPick &k, double inv, double draft_inv, bool rest, int v0, double (&w)[VEC]) {
    float z[VEC], y[VEC];
    load_logits<T, VEC>(row_of<T>(a.logits, a.row_stride, k.row), v0, a.vocab, z);
    const bool drawn = rest && a.draft_logits;
    if (drawn) load_logits<T, VEC>(row_of<T>(a.draft_logits, a.draft_stride, k.row), v0, a.vocab, y);
#pragma unroll
    for (int e = 0; e < VEC; ++e) w[e] = inv == 0.0 ? 0.0 : exp_64(z[e], k.top, a.by_tau) * inv;
    if (drawn && draft_inv != 0.0) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = fmax(w[e] - exp_64(y[e], k.draft_top, a.by_draft_tau) * draft_inv, 0.0);
    }
    if (rest && !drawn) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) w[e] = v0 + e == k.token ? 0.0 : w[e];
    }
}

template <typename T, int E>
__global__ __launch_bounds__(NTV) void verify_rest_kernel(const VerifyArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T), PIECES = E / VEC;
    __shared__ double red[NWV], reds[PIECES][NWV];
    const int s = blockIdx.x / a.slices, slice = blockIdx.x - s * a.slices;
    const VerifyPick k = a.pick[s];
    if (k.row < 0 || !k.refused) return;         // (p itself: its sums are there)
    double inv, draft_inv, sum[PIECES];
    inverses(a, k, s, red, inv, draft_inv);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        double w[VEC];
        weights<T, VEC>(a, k, inv, draft_inv, true, (slice * PIECES + i) * NTV * VEC + threadIdx.x * VEC, w);
        sum[i] = 0.0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) sum[i] += w[e];
    }
    block_adds<PIECES>(sum, reds, a.rest + (size_t)s * a.pieces + slice * PIECES);
}

template <typename T>
__global__ __launch_bounds__(NTV) void verify_pick_kernel(const VerifyArgs a) {
    constexpr int VEC = 16 / (int)sizeof(T);
    __shared__ double red[NWV], part[NWV], before_piece;
    __shared__ int found, last, in_piece;
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), wv = tid / WAVE, s = blockIdx.x;
    const VerifyPick k = a.pick[s];
    if (k.row < 0) return;
    const double u = (double)as_global(a.u)[as_global(a.first)[s + 1] - 1];
    if (tid == 0) { found = INT32_MAX; last = -1; in_piece = -1; }
    double inv, draft_inv;
    inverses(a, k, s, red, inv, draft_inv);
    // a piece's sum: what is left, or (all stand, or nothing is left) p itself
    bool rest = k.refused;
    const auto piece_sum = [&](int i) { return rest ? a.rest[(size_t)s * a.pieces + i] : a.exact[(size_t)s * a.pieces + i] * inv; };
    double total;
    for (;;) {
        double sum = 0.0;
        for (int i = tid; i < a.pieces; i += NTV) sum += piece_sum(i);
        total = block_add(sum, red);
        if (total > 0.0 || !rest) break;
        rest = false;
    }
    const double bound = u * total;
    const auto running = [&](double v) {         // sums up to and with each lane's
#pragma unroll
        for (int o = 1; o < WAVE; o <<= 1) {
            const double x = __shfl_up(v, o, WAVE);
            if (lane >= o) v += x;
        }
        return v;
    };
    if (wv == 0) {                               // the piece where the sums pass it; the last with a weight where none does
        double before = 0.0, pick_before = 0.0;
        int pick = -1;
        for (int i0 = 0; i0 < a.pieces; i0 += WAVE) {
            const double mine = i0 + lane < a.pieces ? piece_sum(i0 + lane) : 0.0, upto = running(mine);
            const u64 some = __ballot(mine > 0.0), past = __ballot(mine > 0.0 && before + upto > bound);
            const int at = past ? __builtin_ctzll(past) : some ? 63 - __builtin_clzll(some) : -1;
            if (at >= 0) {
                pick = i0 + at;
                pick_before = before + (__shfl(upto, at, WAVE) - __shfl(mine, at, WAVE));
            }
            if (past) break;
            before += __shfl(upto, WAVE - 1, WAVE);
        }
        if (lane == 0) { in_piece = pick; before_piece = pick_before; }
    }
    __syncthreads();
    if (in_piece >= 0) {                         // its tokens lie in the order of threads
        const int v0 = in_piece * NTV * VEC + tid * VEC;
        double w[VEC], mine = 0.0;
        weights<T, VEC>(a, k, inv, draft_inv, rest, v0, w);
#pragma unroll
        for (int e = 0; e < VEC; ++e) mine += w[e];
        const double upto = running(mine);
        if (lane == WAVE - 1) part[wv] = upto;
        __syncthreads();
        double at = before_piece + (upto - mine);
        for (int j = 0; j < wv; ++j) at += part[j];
        int first_past = INT32_MAX, last_some = -1;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            at += w[e];
            if (w[e] > 0.0) {
                last_some = v0 + e;
                if (at > bound) first_past = min(first_past, v0 + e);
            }
        }
        if (first_past != INT32_MAX) atomicMin(&found, first_past);
        if (last_some >= 0) atomicMax(&last, last_some);
    }
    __syncthreads();
    if (tid == 0) {
        const int v = found != INT32_MAX ? found : last >= 0 ? last : 0;
        as_global(a.out_tokens)[k.row] = v;
        float logp = -INFINITY;
        if (inv != 0.0) logp = (float)((((double)logit(Store<T>::load1(row_of<T>(a.logits, a.row_stride, k.row), v)) - (double)k.top) * a.by_tau + log2(inv)) * 0.69314718055994530942);
        as_global(a.out_logprobs)[k.row] = logp;
    }
}

constexpr int SEQS_MAX = 1 << 16;                // (every block looks through the sequences)
constexpr double TAU_MIN = 0x1p-100;             // (and 1 / tau: what fp32 exponents hold)

// Logits per thread of a slice: 32, or 8 where that leaves the GPU with fewer blocks than it is busy with (eight of a kind per compute unit, twice), or where 8 hold a row.  Measured, us with 32 / 8 logits, by blocks of 32:
//   bf16, 131072 logits:  256: 36.3 / 27.7 | 1024: 45.0 / 34.3 | 2048: 50.2 / 41.0 | 4096: 58.7 / 57.8 | 6080: 68.3 / 83.2        bf16, 32000: 3200: 57.2 / 51.5 | 4800: 62.8 / 60.1 | 7200: 78.7 / 91.3
//   fp32, 32000 logits:   40: 45.7 / 28.5 | 1520: 56.8 / 39.9 | 4800: 75.4 / 70.6 | 7200: 95.4 / 101.6                            fp32, 1000:  6000: 202 / 173 | 12000: 212 / 173
int each_for(int n_seq, int n_tokens, int vocab) {
    return vocab <= 8 * NTV || std::max(2LL * n_tokens, (long long)n_seq) * ((vocab + 32 * NTV - 1) / (32 * NTV)) < 4096 ? 8 : 32;
}
int slices_for(int n_seq, int n_tokens, int vocab) {
    const int n = NTV * each_for(n_seq, n_tokens, vocab);
    return (vocab + n - 1) / n;
}

template <typename T, int E> hipError_t launch_each(hipStream_t s, const VerifyArgs &a) {
    hipLaunchKernelGGL((verify_sums_kernel<T, E>), dim3((unsigned)(a.n_tokens * (a.draft_logits ? 2 : 1) * a.slices)), dim3(NTV), 0, s, a);
    hipLaunchKernelGGL((verify_drafts_kernel<T, E>), dim3((unsigned)(a.n_seq * a.slices)), dim3(NTV), 0, s, a);
    hipLaunchKernelGGL((verify_rest_kernel<T, E>), dim3((unsigned)(a.n_seq * a.slices)), dim3(NTV), 0, s, a);
    hipLaunchKernelGGL((verify_pick_kernel<T>), dim3((unsigned)a.n_seq), dim3(NTV), 0, s, a);
    return hipGetLastError();
}
template <typename T> hipError_t launch(hipStream_t s, const VerifyArgs &a) { return each_for(a.n_seq, a.n_tokens, a.vocab) == 8 ? launch_each<T, 8>(s, a) : launch_each<T, 32>(s, a); }

}  // namespace

extern "C" size_t spd_op_verify_drafts_scratch_bytes(int32_t n_seq, int32_t n_tokens, int32_t vocab) {
    if (n_seq <= 0 || n_tokens < 0 || vocab <= 0) return 0;
    const size_t slices = (size_t)slices_for(n_seq, n_tokens, vocab), rows = 2 * (size_t)n_tokens * slices;
    const size_t pieces = slices * (each_for(n_seq, n_tokens, vocab) / 4);            // (of fp32 logits: the most)
    return 2 * up256(rows * 4) + up256(2 * n_seq * pieces * 8) + up256(n_seq * pieces * 8) + up256(n_seq * sizeof(VerifyPick));
}

extern "C" int spd_op_verify_drafts(int32_t dtype, const void *logits, int64_t row_stride, const void *draft_logits, int64_t draft_stride, const int32_t *tokens, const int32_t *first,
                                    const float *u, int32_t n_seq, int32_t n_tokens, int32_t vocab, double tau, double draft_tau, int32_t *out_tokens, float *out_logprobs,
                                    int32_t *out_accepted, void *scratch, size_t scratch_bytes, int32_t *err, void *hip_stream) {
    if (dtype != SPD_DTYPE_FP32 && dtype != SPD_DTYPE_BF16 && dtype != SPD_DTYPE_FP16) return SPD_EINVAL;
    const int el = dtype == SPD_DTYPE_FP32 ? 4 : 2;
    if (n_seq < 0 || n_tokens < 0 || vocab < 1 || vocab > (1 << 24) || !(tau >= TAU_MIN) || !(tau <= 1.0 / TAU_MIN) || (draft_logits && (!(draft_tau >= TAU_MIN) || !(draft_tau <= 1.0 / TAU_MIN)))) return SPD_EINVAL;
    if (n_seq == 0) return SPD_OK;
    if (!first || !out_accepted || (n_tokens > 0 && (!logits || !tokens || !u || !out_tokens || !out_logprobs)) || n_seq > SEQS_MAX || n_tokens > (1 << 20)) return SPD_EINVAL;
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
    const int slices = slices_for(n_seq, n_tokens, vocab);
    if ((long long)std::max(2 * n_tokens, n_seq) * slices > UINT32_MAX / NTV) return SPD_EINVAL;      // (threads of a grid are counted in 32 bits)
    const double log2e = 1.4426950408889634074;
    char *w = (char *)scratch;
    VerifyArgs a{logits, draft_logits, row_stride, draft_stride, tokens, first, u, n_seq, n_tokens, vocab, log2e / tau, draft_logits ? log2e / draft_tau : 1.0, out_tokens, out_logprobs, out_accepted, err, slices};
    const size_t row_sums = 2 * (size_t)n_tokens * slices;
    a.top = (float *)w; w += up256(row_sums * 4);
    a.sum = (float *)w; w += up256(row_sums * 4);
    a.pieces = slices * (each_for(n_seq, n_tokens, vocab) / (16 / el));
    a.unsure = 2.1 * sum_off(each_for(n_seq, n_tokens, vocab), vocab, slices);          // (two rows)
    a.exact = (double *)w; w += up256(2 * (size_t)n_seq * a.pieces * 8);
    a.rest = (double *)w; w += up256((size_t)n_seq * a.pieces * 8);
    a.pick = (VerifyPick *)w;
    hipStream_t s = (hipStream_t)hip_stream;
    if (n_tokens == 0) {                         // (sequences without tokens: a = 0 each)
        hipLaunchKernelGGL((verify_drafts_kernel<float, 8>), dim3((unsigned)(n_seq * slices)), dim3(NTV), 0, s, a);
        return hipGetLastError() == hipSuccess ? SPD_OK : SPD_EHIP;
    }
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch<float>(s, a) : dtype == SPD_DTYPE_FP16 ? launch<half_t>(s, a) : launch<bf16_t>(s, a);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}
