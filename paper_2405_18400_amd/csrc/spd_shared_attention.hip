// Attention of one query per sequence and head over a paged cache, for groups of sequences that
// share their first positions.
//
// Bound: the cached keys and values stream through once -- a group's shared ones once for all its
// sequences, which is what the operator is for -- so the work is cut by KEYS, and all query rows
// that need a key meet it in one place:
//   * a "shared" block owns (group, key/value head, chunk of shared positions, tile of query rows); its rows are the
//     query heads of that key/value head in all sequences of the group;
//   * an "own" block owns (sequence, key/value head, chunk of its own positions); its rows are that sequence's query heads;
//   * each leaves (maximum, sum, O) per row and a second kernel puts a row's chunks together in chunk order.
// Both products run on the matrix cores, S^T [key, row] = K Q^T and O^T [feature, row] = V^T P^T, operands straight from
// memory into registers:
//   * 16 keys x 32 features of K are one operand as they lie (a lane holds eight features of one key);
//   * S^T's accumulator holds keys 16 u + 4 kk + r (kk: the lane's group of 16) of one row, which is P^T's operand layout
//     when the eight k indices of a lane stand for those keys, so probabilities never leave their registers;
//   * a lane fetches DH / 16 features of each of those eight keys of V, 16 lanes a whole row, and turns them round in registers.
// K and V of a 16-bit cache are exact in their type; queries and probabilities go in as two fp16 numbers (24 bits, scaled by
// powers of two into fp16's range) or three bf16 numbers (24 bits): the error against 64 bits is that of fp32 arithmetic.
// An fp32 cache takes the fp32 products.  Four waves share a block's keys, 32 each in turn, with a running maximum and sum of their own.
// Measured, heads of 128: four sequences of 74 positions, 32 heads in fp16, 6.5 us (latency: lengths, page numbers, keys, result); five of 1027
// shared and about 20 own, 40 heads in fp32 (45 MB), 16.1 us and 3.9 for the join.
#include "spd_attention.h"

#include <algorithm>

using namespace spdd;
using namespace spda;

namespace {

constexpr int NTS = 256, NWS = NTS / WAVE;
constexpr int KEYS = 32;                         // keys of a wave's turn
constexpr int ROWS = 16;                         // query rows of a tile
constexpr int CHUNK_MAX = 4096;                  // positions of a chunk at most (its page numbers lie in LDS)
constexpr int PAGE_MIN = 4;                      // the smallest page: four keys of a lane lie on one

// Scores of rows whose reference m is far from zero.  Where an fp32 number's step is one or more, the product in fma(score, scale, -reference) is not the one
// that the reference was rounded from, and a probability passes every bound.  Formed from the rounded product, the largest exponent is the
// reference's own and the difference is exact.  Leaves exponents, over scale, so that the reference is zero from there on.
template <typename KT, int NU>
__device__ __forceinline__ void far_scores(f32x4v (&s)[NU], float scale, float m) {
    const float inv = __builtin_amdgcn_rcpf(scale), from = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) s[u][r] = fabsf(m) > FAR ? ((s[u][r] * scale - from) + Type<KT>::P_BITS) * inv : s[u][r];
}

// One turn's scores of a lane's row against its reference m: what the exponents are taken from.  Where a probability would pass 2^SLACK in any row (or a reference is far from
// zero) the references are raised, and sums and results so far follow.
template <typename KT, int NU, int FV>
__device__ __forceinline__ float raised(f32x4v (&s)[NU], f32x4v (&o)[FV], float scale, float &m, float &l) {
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[u][r]);
    mx *= scale;
    if (__any((mx > m + SLACK) | (fabsf(m) > FAR))) {
        mx = fmaxf(mx, __shfl_xor(mx, 16, WAVE));            // the lane groups hold different keys of the same rows
        mx = fmaxf(mx, __shfl_xor(mx, 32, WAVE));
        mx = fmaxf(mx, m);
        const float corr = exp2_below(m, mx);
        m = mx;
        l *= corr;
#pragma unroll
        for (int e = 0; e < FV; ++e) o[e] *= corr;
        if (__any((fabsf(mx) > FAR) & (mx != -INFINITY))) far_scores<KT>(s, scale, mx);
    }
    return fabsf(m) > FAR ? 0.f : m - Type<KT>::P_BITS;      // (-inf: nothing seen yet, no score)
}

// Two features of eight keys (word i of each), turned round: eight keys of each feature.
template <int VW>
__device__ __forceinline__ void turned(const uint32_t (&v)[2][4][VW], int i, u32x4 &even, u32x4 &odd) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t x = v[k / 2][2 * (k % 2)][i], y = v[k / 2][2 * (k % 2) + 1][i];
        even[k] = __builtin_amdgcn_perm(y, x, 0x05040100u);
        odd[k] = __builtin_amdgcn_perm(y, x, 0x07060302u);
    }
}

template <typename KT> __device__ __forceinline__ f32x4v mfma16(u32x4 a, u32x4 b, f32x4v c);
template <> __device__ __forceinline__ f32x4v mfma16<half_t>(u32x4 a, u32x4 b, f32x4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4v mfma16<bf16_t>(u32x4 a, u32x4 b, f32x4v c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// B bytes of one lane, in words.
template <int B> __device__ __forceinline__ void load_words(const char *p, uint32_t (&w)[B / 4]) {
    if constexpr (B == 4) w[0] = *(const uint32_t __attribute__((address_space(1))) *)p;
    else if constexpr (B == 8) { const u32x2 v = *(const u32x2 __attribute__((address_space(1))) *)p; w[0] = v.x; w[1] = v.y; }
    else {
#pragma unroll
        for (int i = 0; i < B / 16; ++i) {
            const u32x4 v = global_load16(p + 16 * i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    }
}

// The bits that any thread of the block has set (N of them), by one barrier, which also says that the pages' places have been written.
template <int N>
__device__ __forceinline__ int block_any(int bits, int *flags) {
    int all = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) all |= __any((bits >> i) & 1) ? 1 << i : 0;
    if ((threadIdx.x & (WAVE - 1)) == 0) flags[threadIdx.x / WAVE] = all;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int v = 0; v < NWS; ++v) all |= flags[v];
    return all;
}

// A stretch of positions read through one row of the table.
struct Stretch { int row, lo, hi; };

// What a block does: rows r0 .. r0 + n_rows - 1 of the sequences from `seq` on (row r: sequence seq + r / group, query head
// kvh * group + r % group), over one or two stretches; its results go to `slot`, or to the output where there is one slot.
// `shared`: positions that a row's sequence must have to take part (those that end before have a block of their own), or -1.
struct Unit { int seq, kvh, r0, n_rows, slot, shared; Stretch a, b; };

// Whether a sequence's lengths are in bounds.
__device__ __forceinline__ bool seq_fits(const SharedAttnArgs &p, int shared, int len) {
    return shared >= 0 && len >= 0 && shared <= p.max_shared && (len <= shared || len - shared <= p.max_own) && (long long)len <= (long long)p.c.table_stride << p.c.page_shift;
}

template <typename KT, int DH, int RT>
struct Lds {
    static constexpr int PARTS = Type<KT>::PARTS;
    static constexpr int Q_WORDS = RT * ROWS * DH * (sizeof(KT) == 4 ? 1 : 0) + RT * ROWS * DH * PARTS / 2 * (sizeof(KT) == 2 ? 1 : 0);
    static constexpr int HALF = DH > 128 ? 128 : DH, STRIDE = HALF + 4;      // the waves' results meet 128 features at a time
    static constexpr int O_WORDS = NWS * ROWS * STRIDE;
    static constexpr int WORDS = Q_WORDS > O_WORDS ? Q_WORDS : O_WORDS;
};

constexpr int PAGES = CHUNK_MAX / PAGE_MIN + 4;

// `resolve` reads the lengths and sets the stretches; false: there are none.  Queries are asked for before that, page numbers before
// the queries are put in place: each of these is a trip to memory.
template <typename KT, int DH, int RT, typename F>
__device__ __forceinline__ bool attend(const SharedAttnArgs &p, Unit &un, F &&resolve, uint32_t *lds, u64 *pages, int *flags, float (*lds_m)[ROWS], float (*lds_l)[ROWS], float *row_scale) {
    constexpr bool F32 = sizeof(KT) == 4;
    constexpr int PARTS = Type<KT>::PARTS;
    constexpr int NJ = F32 ? DH / 16 : DH / 32;                              // 16-byte pieces of a key per lane
    constexpr int FV = DH / 16, VB = FV * (int)sizeof(KT), VW = VB / 4;      // features, bytes, words of a value row per lane
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), w = __builtin_amdgcn_readfirstlane(tid / WAVE), col = lane % ROWS, kk = lane / ROWS;
    const int d = p.c.d_head, shift = p.c.page_shift, page_size = 1 << shift, group = p.group;
    const int tiles = (min(un.n_rows, RT * ROWS) + ROWS - 1) / ROWS;

    constexpr int TPR = NTS / (RT * ROWS), N8 = DH / 8, PP = (N8 + TPR - 1) / TPR;       // threads per row; pieces of eight features
    const int q_row = tid / TPR, q_t = tid % TPR;
    float x[PP][8];
    {
        const int r = un.r0 + min(q_row, un.n_rows - 1), rs = over(r, p.by_group), s = un.seq + rs, hq = un.kvh * group + r - rs * group;   // (rows past the last repeat it)
        const float *q = p.q + ((size_t)s * p.n_heads + hq) * d;
#pragma unroll
        for (int i = 0; i < PP; ++i)
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const int at = 8 * (q_t + i * TPR) + e;
                const float4 v = at < d ? global_load_float4(q + at) : make_float4(0.f, 0.f, 0.f, 0.f);
                x[i][e] = v.x; x[i][e + 1] = v.y; x[i][e + 2] = v.z; x[i][e + 3] = v.w;
            }
    }
    if (!resolve(un)) return false;
    auto entry_page = [&](int lo_a, int n_a, int lo_b, int i) {
        const int row = i < n_a ? un.a.row : un.b.row, entry = i < n_a ? (lo_a >> shift) + i : (lo_b >> shift) + i - n_a;
        return as_global(p.c.table)[(size_t)row * p.c.table_stride + entry];
    };
    auto pages_of = [&](int lo, int hi) { return hi > lo ? ((hi - 1) >> shift) - (lo >> shift) + 1 : 0; };
    const int first_n_a = pages_of(un.a.lo, min(un.a.hi, (un.a.lo & ~3) + CHUNK_MAX)), first_n = first_n_a + pages_of(un.b.lo, un.b.hi);
    int early_page = 0;
    if (tid < first_n) early_page = entry_page(un.a.lo, first_n_a, un.b.lo, tid);
    // queries, as the products take them: piece (step j, part) of a tile holds a lane's eight (fp32: four) features
    {
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < PP; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[i][e]));
        float up = 1.f, down = 1.f;
        if constexpr (sizeof(KT) == 2 && PARTS == 2) {
#pragma unroll
            for (int o = 1; o < TPR; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, WAVE));
            scaling(top, up, down);
        }
        if (q_t == 0) row_scale[q_row] = down * (1.4426950408889634f / sqrtf((float)d));     // to logarithms of base 2
#pragma unroll
        for (int i = 0; i < PP; ++i) {
            const int piece = q_t + i * TPR;
            if (piece >= N8) break;
            u32x4 *to = (u32x4 *)lds;
            if constexpr (F32) {
#pragma unroll
                for (int e = 0; e < 8; e += 4) { // feature 16 j + 4 kk + c of piece j: word c
                    const int f = 8 * piece + e;
                    to[((q_row / ROWS) * NJ + f / 16) * WAVE + ((f / 4) % 4) * ROWS + q_row % ROWS] =
                        u32x4{__float_as_uint(x[i][e]), __float_as_uint(x[i][e + 1]), __float_as_uint(x[i][e + 2]), __float_as_uint(x[i][e + 3])};
                }
            } else {
                uint32_t part[4][PARTS];
#pragma unroll
                for (int e = 0; e < 8; e += 2) query_parts<KT>(x[i][e] * up, x[i][e + 1] * up, part[e / 2]);
#pragma unroll
                for (int q = 0; q < PARTS; ++q)
                    to[(((q_row / ROWS) * NJ + piece / 4) * PARTS + q) * WAVE + (piece % 4) * ROWS + q_row % ROWS] = u32x4{part[0][q], part[1][q], part[2][q], part[3][q]};
            }
        }
    }
    const u32x4 *Q = (const u32x4 *)lds;
    f32x4v o[RT][FV];
    float m[RT], l[RT], scale[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int e = 0; e < FV; ++e) o[rt][e] = f32x4v{0.f, 0.f, 0.f, 0.f};
        m[rt] = -INFINITY; l[rt] = 0.f;
    }

    const int row_bytes = d * (int)sizeof(KT);
    const u64 head_bytes = (u64)row_bytes << shift, page_bytes = head_bytes * p.c.n_kv_heads;
    const char *Kh = (const char *)p.c.K + (size_t)un.kvh * head_bytes, *Vh = (const char *)p.c.V + (size_t)un.kvh * head_bytes;
    u32x4 kf[2][NJ];
    uint32_t vf[2][4][VW];
    const int k_at = 16 * kk, v_at = col * VB;               // this lane's bytes of a row (a head narrower than DH: only those inside)
    // A stretch longer than a chunk (a long sequence that ends inside the shared positions) goes panel by panel; one panel
    // takes both stretches where there are two.
    for (int panel = un.a.lo;;) {
    const int lo_a = panel, hi_a = min(un.a.hi, (panel & ~3) + CHUNK_MAX);
    // where the pages of both stretches begin
    const int first_a = lo_a >> shift, n_a = pages_of(lo_a, hi_a), first_b = un.b.lo >> shift, n_b = pages_of(un.b.lo, un.b.hi);
    bool bad = false;
    for (int i = tid; i < n_a + n_b; i += NTS) {
        const int page = i == tid && panel == un.a.lo ? early_page : entry_page(lo_a, n_a, un.b.lo, i);
        const bool ok = (unsigned)page < (unsigned)p.c.n_pages;
        pages[i] = ok ? (u64)page * page_bytes : 0;          // (a page that is none: its keys are masked)
        bad = bad || !ok;
    }
    const bool any_bad = block_any<1>(bad, flags) != 0;
    if (any_bad && tid == 0 && p.err) *as_global(p.err) = 1;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) scale[rt] = row_scale[rt * ROWS + col];
    // turns of 32 keys, from a multiple of four on
    const int base_a = lo_a & ~3, base_b = un.b.lo & ~3;
    const int turns_a = n_a ? (hi_a - base_a + KEYS - 1) / KEYS : 0, turns_b = n_b ? (un.b.hi - base_b + KEYS - 1) / KEYS : 0, turns = turns_a + turns_b;
    auto stretch = [&](int t, int &tb, int &lo, int &hi, int &index0) {
        const bool in_a = t < turns_a;
        tb = in_a ? base_a + KEYS * t : base_b + KEYS * (t - turns_a);
        lo = in_a ? lo_a : un.b.lo;
        hi = in_a ? hi_a : un.b.hi;
        index0 = in_a ? -first_a : n_a - first_b;
    };
    auto fetch_k = [&](int t) {
        int tb, lo, hi, index0;
        stretch(t, tb, lo, hi, index0);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int pos = min(max(tb + 16 * u + col, lo), hi - 1);
            const char *row = Kh + (pages[(pos >> shift) + index0] + (uint32_t)((pos & (page_size - 1)) * row_bytes + k_at));
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (DH > 32 || 64 * j + k_at < (int)row_bytes) kf[u][j] = global_load16(row + 64 * j);
                else kf[u][j] = u32x4{0, 0, 0, 0};
            }
        }
    };
    auto fetch_v = [&](int t) {
        int tb, lo, hi, index0;
        stretch(t, tb, lo, hi, index0);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int pos = min(max(tb + 16 * u + 4 * kk, lo & ~3), (hi - 1) & ~3);
            const char *row = Vh + (pages[(pos >> shift) + index0] + (uint32_t)((pos & (page_size - 1)) * row_bytes + v_at));
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (DH > 32 || v_at < (int)row_bytes) load_words<VB>(row + r * row_bytes, vf[u][r]);
                else {
#pragma unroll
                    for (int i = 0; i < VW; ++i) vf[u][r][i] = 0;
                }
            }
        }
    };
    int t = w;
    if (t < turns) { fetch_k(t); fetch_v(t); }
    for (; t < turns; t += NWS) {
        int tb, lo, hi, index0;
        stretch(t, tb, lo, hi, index0);
        f32x4v st[RT][2];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (rt >= tiles) break;
#pragma unroll
            for (int u = 0; u < 2; ++u) st[rt][u] = f32x4v{0.f, 0.f, 0.f, 0.f};
            if constexpr (F32) {
                f32x4v part[2][4];               // four sums per tile: one chain of d_head / 4 products would double the error
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int c = 0; c < 4; ++c) part[u][c] = f32x4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const u32x4 q = Q[(rt * NJ + j) * WAVE + lane];
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int u = 0; u < 2; ++u) part[u][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[u][j][c]), __uint_as_float(q[c]), part[u][c], 0, 0, 0);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) st[rt][u] = (part[u][0] + part[u][1]) + (part[u][2] + part[u][3]);
            } else {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int q = PARTS - 1; q >= 0; --q) {
                        const u32x4 b = Q[((rt * NJ + j) * PARTS + q) * WAVE + lane];
#pragma unroll
                        for (int u = 0; u < 2; ++u) st[rt][u] = mfma16<KT>(kf[u][j], b, st[rt][u]);
                    }
            }
        }
        if (t + NWS < turns) fetch_k(t + NWS);
        // keys outside the stretch, or on no page: no score, and no value that could be a NaN
        if (tb < lo || tb + KEYS > hi || any_bad) {
            asm volatile("");                   // (a branch: seldom taken)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int pos = min(max(tb + 16 * u + 4 * kk, lo & ~3), (hi - 1) & ~3);
                const bool page_ok = !any_bad || (unsigned)entry_page(lo_a, n_a, un.b.lo, (pos >> shift) + index0) < (unsigned)p.c.n_pages;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = tb + 16 * u + 4 * kk + r;
                    const bool in = at >= lo && at < hi && page_ok;
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) st[rt][u][r] = in ? st[rt][u][r] : -INFINITY;
#pragma unroll
                    for (int i = 0; i < VW; ++i) vf[u][r][i] = in ? vf[u][r][i] : 0;
                }
            }
        }
        uint32_t pt[RT][PARTS][4];               // 16-bit caches: eight probabilities per lane and part
        float pf[RT][8];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            if (rt >= tiles) break;
            const float ref = raised<KT>(st[rt], o[rt], scale[rt], m[rt], l[rt]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                pf[rt][i] = __builtin_amdgcn_exp2f(fmaf(st[rt][i / 4][i % 4], scale[rt], -ref)) * Type<KT>::P_SCALE;
                l[rt] += pf[rt][i];
            }
            if constexpr (!F32) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    uint32_t part[PARTS];
                    parts_of<KT>(pf[rt][i], pf[rt][i + 1], part);
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) pt[rt][q][i / 2] = part[q];
                }
            }
        }
        if constexpr (F32) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if (rt >= tiles) break;
#pragma unroll
                for (int i = 0; i < 8; ++i)
#pragma unroll
                    for (int e = 0; e < FV; ++e)
                        o[rt][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[i / 4][i % 4][e]), pf[rt][i], o[rt][e], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                u32x4 even, odd;
                turned(vf, i, even, odd);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    if (rt >= tiles) break;
#pragma unroll
                    for (int q = PARTS - 1; q >= 0; --q) {
                        const u32x4 b = u32x4{pt[rt][q][0], pt[rt][q][1], pt[rt][q][2], pt[rt][q][3]};
                        o[rt][2 * i] = mfma16<KT>(even, b, o[rt][2 * i]);
                        o[rt][2 * i + 1] = mfma16<KT>(odd, b, o[rt][2 * i + 1]);
                    }
                }
            }
        }
        if (t + NWS < turns) fetch_v(t + NWS);
    }
    panel = hi_a;
    if (panel >= un.a.hi) break;
    __syncthreads();                             // the page numbers have been read
    }

    // the four waves' results, a tile of rows and 128 features at a time, in wave order
    constexpr int HALF = Lds<KT, DH, RT>::HALF, STRIDE = Lds<KT, DH, RT>::STRIDE, NH = DH / HALF, FH = FV / NH;
    float *O = (float *)lds;
    for (int rt = 0; rt < tiles; ++rt) {
        float mt = m[0], lt = l[0];
#pragma unroll
        for (int i = 1; i < RT; ++i) { mt = i == rt ? m[i] : mt; lt = i == rt ? l[i] : lt; }
        lt += __shfl_xor(lt, 16, WAVE);
        lt += __shfl_xor(lt, 32, WAVE);
        for (int h = 0; h < NH; ++h) {
            __syncthreads();                     // Q, or the tile before, has been read
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int hh = 0; hh < NH; ++hh)
                    if (i == rt && hh == h) {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int e = 0; e < FH; ++e) O[(w * ROWS + col) * STRIDE + FH * (4 * kk + r) + e] = o[i][hh * FH + e][r];
                    }
            if (kk == 0) { lds_m[w][col] = mt; lds_l[w][col] = lt; }
            __syncthreads();
            for (int i = tid; i < ROWS * HALF / 4; i += NTS) {
                const int row = i / (HALF / 4), c = 4 * (i % (HALF / 4)), r = un.r0 + rt * ROWS + row;
                if (rt * ROWS + row >= un.n_rows) continue;
                float M = lds_m[0][row], L = 0.f;
#pragma unroll
                for (int v = 1; v < NWS; ++v) M = fmaxf(M, lds_m[v][row]);
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int v = 0; v < NWS; ++v) {
                    const float f = exp2_below(lds_m[v][row], M);
                    L += f * lds_l[v][row];
                    const float4 z = *(const float4 *)&O[(v * ROWS + row) * STRIDE + c];
                    y.x += f * z.x; y.y += f * z.y; y.z += f * z.z; y.w += f * z.w;
                }
                const int feature = NH * FH * (c / FH) + h * FH + c % FH, rs = over(r, p.by_group), s = un.seq + rs, hq = un.kvh * group + r - rs * group;
                if (feature >= d) continue;
                const size_t at = (size_t)s * p.n_heads + hq;
                float *to = p.out + at * d + feature;
                if (p.slots > 1) {
                    to = p.part + (at * p.slots + un.slot) * d + feature;
                    if (feature == 0) {
                        const int len = un.shared < 0 ? 0 : as_global(p.len)[s];
                        const bool on = un.shared < 0 || (len >= un.shared && seq_fits(p, un.shared, len));
                        as_global(p.part_ml)[2 * (at * p.slots + un.slot)] = on ? M : -INFINITY;
                        as_global(p.part_ml)[2 * (at * p.slots + un.slot) + 1] = on ? L : 0.f;
                    }
                } else {
                    const float inv = L == 0.f ? 0.f : 1.f / L;               // (nothing seen: zeros)
                    y.x *= inv; y.y *= inv; y.z *= inv; y.w *= inv;
                }
                if constexpr (FH >= 4) *(f32x4 __attribute__((address_space(1))) *)to = f32x4{y.x, y.y, y.z, y.w};
                else {                            // two features of a lane lie side by side
                    as_global(to)[0] = y.x; as_global(to)[1] = y.y;
                    as_global(to)[2] = y.z; as_global(to)[3] = y.w;
                }
            }
        }
    }
    return true;
}

// Many rows: the block's four waves share out ROWS instead of keys, so nothing has to be put together at the end.  Keys and values
// come through LDS, 16 bytes per lane straight from memory, ST stages of SK keys deep; pieces of a row are permuted by the row number,
// so that neither the operand reads (16 rows side by side) nor the row reads meet in a bank.  One barrier per stage says both "this
// stage has arrived" and "the one before has been read".
// Measured, 64 heads of 128 on 8 in fp16: eight sequences over 8191 positions (37 MB) 15.3 us, bound by a block's chain; sixteen over
// 65537 (271 MB; 69 GFLOP with the two parts of queries and probabilities) 80 .. 97 us, 3.4 TB/s and 0.85 PFLOP/s at best, the matrix cores busy for 34% of it and the
// vector unit for 39%, in turn.  Eight groups of eight over 2001, 32 heads on 8 in bf16 (127 MB), 34.5 us, 3.7 TB/s (17% and 25%).
template <int DH, int RT> struct Stage {
    static constexpr int SK = DH == 64 || (DH == 128 && RT == 1) ? 64 : 32;             // keys
    static constexpr int NU = RT == 1 && SK == 64 ? 4 : 2;                              // tiles of 16 keys that go through the products together
    static constexpr int ROWB = DH * 2, PIECES = ROWB / 16;                             // bytes and 16-byte pieces of a row
    static constexpr int HALF = SK * ROWB, BYTES = 2 * HALF;                            // K, then V
    static constexpr int LOADS = HALF / 16 / NTS;                                       // pieces per thread, of K as of V
    static constexpr int ST = BYTES >= 32 * 1024 ? (DH == 256 ? 3 : 2) : 4;
};
template <int PIECES> __device__ __forceinline__ int permuted(int row, int piece) {
    return PIECES >= 16 ? piece ^ (row & 15) : piece ^ ((row & 7) ^ ((row >> 3) & 1));
}
// False: none of the chunk's positions is there, or no row needs them.
template <typename KT, int DH, int RT>
__device__ __forceinline__ bool attend_many(const SharedAttnArgs &p, const Unit &un, char *lds, u64 *pages, int *flags) {
    constexpr int PARTS = Type<KT>::PARTS, NJ = DH / 32, FV = DH / 16, VW = FV / 2;
    typedef Stage<DH, RT> S;
    constexpr int SK = S::SK, NU = S::NU, ROWB = S::ROWB, PIECES = S::PIECES, HALF = S::HALF, BYTES = S::BYTES, LOADS = S::LOADS, ST = S::ST;
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), w = __builtin_amdgcn_readfirstlane(tid / WAVE), col = lane % ROWS, kk = lane / ROWS;
    const int shift = p.c.page_shift, page_size = 1 << shift, group = p.group;
    const int row0 = w * RT * ROWS;                          // this wave's rows of the unit
    const u64 head_bytes = (u64)ROWB << shift, page_bytes = head_bytes * p.c.n_kv_heads;
    // asked for at once: the queries, the group's shared length and the page numbers of the whole chunk
    float x[RT][NJ][8];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int rr = un.r0 + min(row0 + rt * ROWS + col, un.n_rows - 1), rs = over(rr, p.by_group), s = un.seq + rs, hq = un.kvh * group + rr - rs * group;   // (rows past the last repeat it)
        const float *q = p.q + ((size_t)s * p.n_heads + hq) * DH + 8 * kk;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const float4 v = global_load_float4(q + 32 * j + e);
                x[rt][j][e] = v.x; x[rt][j][e + 1] = v.y; x[rt][j][e + 2] = v.z; x[rt][j][e + 3] = v.w;
            }
    }
    int len[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) len[rt] = as_global(p.len)[un.seq + over(un.r0 + min(row0 + rt * ROWS + col, un.n_rows - 1), p.by_group)];
    const int lo = un.a.lo, first = lo >> shift;
    const int last = min((un.a.hi - 1) >> shift, p.c.table_stride - 1);
    int page = 0;
    const int32_t *entries = p.c.table + (size_t)un.a.row * p.c.table_stride + first;
    if (tid <= last - first) page = as_global(entries)[tid];
    const int to = as_global(p.shared)[over(un.seq, p.by_width)], hi = min(un.a.hi, to);
    if ((to < 0 || to > p.max_shared) && p.err && tid == 0) *as_global(p.err) = 1;
    if (hi <= lo || to > p.max_shared) return false;
    const int n_pages = ((hi - 1) >> shift) - first + 1;     // (at most the row's entries: max_shared is)
    bool bad = false, on = false;                // (on: a sequence of these rows reaches behind the shared positions, and so needs all of them)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) on = on || (len[rt] >= to && seq_fits(p, to, len[rt]));
    for (int i = tid; i < n_pages; i += NTS) {
        if (i != tid) page = as_global(entries)[i];
        const bool ok = (unsigned)page < (unsigned)p.c.n_pages;
        pages[i] = ok ? (u64)page * page_bytes : 0;          // (a page that is none: its keys are masked)
        bad = bad || !ok;
    }
    const int found = block_any<2>((int)bad | (int)on << 1, flags);
    if (!(found & 2)) return false;
    const bool any_bad = found & 1;
    if (any_bad && tid == 0 && p.err) *as_global(p.err) = 1;

    const int base = lo & ~3, stages = (hi - base + SK - 1) / SK;
    const char *Kh = (const char *)p.c.K + (size_t)un.kvh * head_bytes, *Vh = (const char *)p.c.V + (size_t)un.kvh * head_bytes;
    // Blocks go through their chunks in step, and pages are a power of two apart: started at the same place of a page they would all
    // ask the same memory channels at once.  So each starts at a place of its own.
    const int turn = (int)(blockIdx.x * 5u % (unsigned)stages);
    const auto place_of = [&](int t) { return t + turn < stages ? t + turn : t + turn - stages; };
    auto fetch = [&](int t) {
        char *to = lds + (t % ST) * BYTES + w * (WAVE * 16);
        const int at0 = base + place_of(t) * SK;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int at = tid + i * NTS, key = at / PIECES, pos = min(max(at0 + key, lo), hi - 1);
            const u64 from = pages[(pos >> shift) - first] + (uint32_t)((pos & (page_size - 1)) * ROWB + 16 * permuted<PIECES>(key, at % PIECES));
            to_lds16(Kh + from, to + i * (NTS * 16));
            to_lds16(Vh + from, to + HALF + i * (NTS * 16));
        }
    };
#pragma unroll
    for (int t = 0; t < ST - 1; ++t)
        if (t < stages) fetch(t);

    // this lane's queries: row col of each tile, features 32 j + 8 kk .. + 7
    u32x4 Q[RT][NJ][PARTS];
    float scale[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        float top = 0.f;
        float up = 1.f, down = 1.f;
        if constexpr (PARTS == 2) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[rt][j][e]));
            top = fmaxf(top, __shfl_xor(top, 16, WAVE));
            top = fmaxf(top, __shfl_xor(top, 32, WAVE));
            scaling(top, up, down);
        }
        scale[rt] = down * (1.4426950408889634f / sqrtf((float)DH));
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                uint32_t part[PARTS];
                query_parts<KT>(x[rt][j][e] * up, x[rt][j][e + 1] * up, part);
#pragma unroll
                for (int q2 = 0; q2 < PARTS; ++q2) Q[rt][j][q2][e / 2] = part[q2];
            }
    }
    f32x4v o[RT][FV];
    float m[RT], l[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int e = 0; e < FV; ++e) o[rt][e] = f32x4v{0.f, 0.f, 0.f, 0.f};
        m[rt] = -INFINITY; l[rt] = 0.f;
    }
    for (int t = 0; t < stages; ++t) {
        // the oldest stage under way has arrived (of this wave's loads: at most the ST - 2 younger ones are out)
        const int younger = min(stages - 1 - t, ST - 2);
        if (ST > 3 && younger >= 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * 2 * LOADS) : "memory");
        else if (ST > 2 && younger >= 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (t + ST - 1 < stages) fetch(t + ST - 1);
        const char *k_tile = lds + (t % ST) * BYTES, *v_tile = k_tile + HALF;
#pragma unroll
        for (int sub = 0; sub < SK / (16 * NU); ++sub) {
            const int key0 = sub * 16 * NU, tb = base + place_of(t) * SK + key0;
            f32x4v st[RT][NU];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int u = 0; u < NU; ++u) st[rt][u] = f32x4v{0.f, 0.f, 0.f, 0.f};
            u32x4 k[NJ][NU];
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const int key = key0 + 16 * u + col;
                    k[j][u] = *(const u32x4 *)(k_tile + key * ROWB + 16 * permuted<PIECES>(key, 4 * j + kk));
                }
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = PARTS - 1; q >= 0; --q)
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) st[rt][u] = mfma16<KT>(k[j][u], Q[rt][j][q], st[rt][u]);
            // values of 32 keys at a time, a half ahead of their products
            uint32_t vf[NU / 2][2][4][VW];
            const auto read_v = [&](int h) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int key = key0 + 32 * h + 16 * u + 4 * kk + r;
#pragma unroll
                        for (int i = 0; i < VW; i += (VW < 4 ? VW : 4)) {
                            const int byte = 2 * FV * col + 4 * i;
                            const char *from = v_tile + key * ROWB + 16 * permuted<PIECES>(key, byte / 16) + byte % 16;
                            if constexpr (VW == 2) {
                                const u32x2 v = *(const u32x2 *)from;
                                vf[h][u][r][0] = v.x; vf[h][u][r][1] = v.y;
                            } else {
                                const u32x4 v = *(const u32x4 *)from;
                                vf[h][u][r][i] = v.x; vf[h][u][r][i + 1] = v.y; vf[h][u][r][i + 2] = v.z; vf[h][u][r][i + 3] = v.w;
                            }
                        }
                    }
            };
            read_v(0);
            const bool cut = tb < lo || tb + 16 * NU > hi || any_bad;
            uint32_t there = 0;                              // bit 4 u + r: this lane's key 16 u + 4 kk + r counts
            if (cut) {                                       // keys that do not count: no score (and, below, no value that could be a NaN)
                asm volatile("");                           // (a branch: seldom taken)
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    const int pos = min(max(tb + 16 * u + 4 * kk, lo & ~3), (hi - 1) & ~3);
                    const bool page_ok = !any_bad || (unsigned)as_global(entries)[(pos >> shift) - first] < (unsigned)p.c.n_pages;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int at = tb + 16 * u + 4 * kk + r;
                        const bool in = at >= lo && at < hi && page_ok;
                        there |= (uint32_t)in << (4 * u + r);
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) st[rt][u][r] = in ? st[rt][u][r] : -INFINITY;
                    }
                }
            }
            u32x4 pt[RT][NU / 2][PARTS];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                const float ref = raised<KT>(st[rt], o[rt], scale[rt], m[rt], l[rt]);
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        const float p0 = __builtin_amdgcn_exp2f(fmaf(st[rt][u][r], scale[rt], -ref)) * Type<KT>::P_SCALE;
                        const float p1 = __builtin_amdgcn_exp2f(fmaf(st[rt][u][r + 1], scale[rt], -ref)) * Type<KT>::P_SCALE;
                        l[rt] += p0 + p1;
                        uint32_t part[PARTS];
                        parts_of<KT>(p0, p1, part);
#pragma unroll
                        for (int q = 0; q < PARTS; ++q) pt[rt][u / 2][q][2 * (u % 2) + r / 2] = part[q];
                    }
            }
#pragma unroll
            for (int h = 0; h < NU / 2; ++h) {               // 32 keys at a time
                if (h + 1 < NU / 2) read_v(h + 1);
                if (cut) {
                    asm volatile("");
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int i = 0; i < VW; ++i) vf[h][u][r][i] = (there >> (4 * (2 * h + u) + r)) & 1 ? vf[h][u][r][i] : 0;
                }
#pragma unroll
                for (int i = 0; i < VW; ++i) {
                    u32x4 even, odd;
                    turned(vf[h], i, even, odd);
#pragma unroll
                    for (int q = PARTS - 1; q >= 0; --q)
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) {
                            o[rt][2 * i] = mfma16<KT>(even, pt[rt][h][q], o[rt][2 * i]);
                            o[rt][2 * i + 1] = mfma16<KT>(odd, pt[rt][h][q], o[rt][2 * i + 1]);
                        }
                }
            }
        }
    }
    // O by rows, through LDS (a lane's features of a row are FV here and FV there): whole lines
    constexpr int STRIDE = DH + 4;
    float *O = (float *)lds + w * ROWS * STRIDE;
    __syncthreads();                                         // the stages have been read
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        l[rt] += __shfl_xor(l[rt], 16, WAVE);
        l[rt] += __shfl_xor(l[rt], 32, WAVE);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < FV; e += 4) *(f32x4v *)&O[col * STRIDE + FV * (4 * kk + i) + e] = f32x4v{o[rt][e][i], o[rt][e + 1][i], o[rt][e + 2][i], o[rt][e + 3][i]};
        auto place = [&](int r) {
            const int rs = over(un.r0 + r, p.by_group);
            return ((size_t)(un.seq + rs) * p.n_heads + un.kvh * group + un.r0 + r - rs * group) * p.slots + un.slot;
        };
        const int r = row0 + rt * ROWS + col;
        if (kk == 0 && r < un.n_rows) {
            const bool on = len[rt] >= to && seq_fits(p, to, len[rt]);
            as_global(p.part_ml)[2 * place(r)] = on ? m[rt] : -INFINITY;
            as_global(p.part_ml)[2 * place(r) + 1] = on ? l[rt] : 0.f;
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < ROWS * DH / 4 / WAVE; ++i) {
            const int at = lane + i * WAVE, row = at / (DH / 4), c = 4 * (at % (DH / 4));
            const f32x4v y = *(const f32x4v *)&O[row * STRIDE + c];
            if (row0 + rt * ROWS + row < un.n_rows)
                *(f32x4 __attribute__((address_space(1))) *)(p.part + place(row0 + rt * ROWS + row) * DH + c) = f32x4{y[0], y[1], y[2], y[3]};
        }
        __builtin_amdgcn_wave_barrier();
    }
    return true;
}

// A unit without positions, or rows that take no part in it: no sum.
__device__ __forceinline__ void nothing(const SharedAttnArgs &p, const Unit &un, int row) {
    const int group = p.n_heads / p.c.n_kv_heads, r = un.r0 + row, rs = over(r, p.by_group), s = un.seq + rs, hq = un.kvh * group + r - rs * group;
    const size_t at = (size_t)s * p.n_heads + hq;
    if (p.slots > 1) {
        as_global(p.part_ml)[2 * (at * p.slots + un.slot)] = -INFINITY;
        as_global(p.part_ml)[2 * (at * p.slots + un.slot) + 1] = 0.f;
    } else {
        for (int c = 0; c < p.c.d_head; ++c) as_global(p.out)[at * p.c.d_head + c] = 0.f;
    }
}

// TILE: query rows of a shared block; MANY: its waves share out rows, not keys.
template <typename KT, int DH, int TILE, bool MANY>
__global__ __launch_bounds__(NTS, (MANY && DH <= 128) || (sizeof(KT) * DH <= 512 && TILE == ROWS) ? 2 : 1) void shared_attn_kernel(const SharedAttnArgs p) {
    constexpr int RT = MANY ? 1 : TILE / ROWS;
    extern __shared__ __align__(1024) uint32_t lds[];        // lds_bytes()
    __shared__ u64 pages[PAGES];
    __shared__ int flags[NWS];
    __shared__ float lds_m[NWS][ROWS], lds_l[NWS][ROWS], row_scale[RT * ROWS];
    const int group = p.group;
    int b = blockIdx.x;
    Unit un;
    un.b = Stretch{0, 0, 0};
    un.shared = -1;
    if (b < p.shared_blocks) {
        // row tiles of a chunk on one XCD (blocks go to the eight in turn), so that its keys come through that L2
        const int of8 = over(b / 8, p.by_row_tiles), chunk8 = 8 * of8 + b % 8, tile = b / 8 - of8 * p.row_tiles;
        if (chunk8 >= p.shared_blocks_per_tile) return;
        const int gh = over(chunk8, p.by_shared_chunks), c = chunk8 - gh * p.shared_chunks, g = over(gh, p.by_kv_heads);
        un.kvh = gh - g * p.c.n_kv_heads;
        un.seq = g * p.width;
        un.r0 = tile * TILE;
        un.n_rows = min(p.width * group - un.r0, TILE);
        un.slot = c;
        if constexpr (MANY) {
            un.a = Stretch{un.seq, c * p.shared_chunk, (c + 1) * p.shared_chunk};
            if (!attend_many<KT, DH, TILE / (NWS * ROWS)>(p, un, (char *)lds, pages, flags))
                for (int r = threadIdx.x; r < un.n_rows; r += NTS) nothing(p, un, r);
        } else {
            const auto resolve = [&](Unit &u) {
                int to = as_global(p.shared)[g];
                bool on = true;                  // a sequence of these rows reaches behind the shared positions: others have blocks of their own
                if (p.width == 1) {              // nothing is shared: the whole sequence
                    const int len = as_global(p.len)[g];
                    to = seq_fits(p, to, len) ? len : -1;
                } else {
                    if (to > p.max_shared) to = -1;
                    u.shared = to;
                    const int row = min((int)(threadIdx.x & (WAVE - 1)), u.n_rows - 1), len = as_global(p.len)[u.seq + over(u.r0 + row, p.by_group)];
                    on = __any(len >= to && seq_fits(p, to, len));       // (every wave looks at all rows)
                }
                if (to < 0 && p.err && threadIdx.x == 0) *as_global(p.err) = 1;
                u.a = Stretch{u.seq, c * p.shared_chunk, min((c + 1) * p.shared_chunk, to)};
                return on && u.a.hi > u.a.lo;
            };
            if (!attend<KT, DH, RT>(p, un, resolve, lds, pages, flags, lds_m, lds_l, row_scale))
                for (int r = threadIdx.x; r < un.n_rows; r += NTS) nothing(p, un, r);
        }
        return;
    }
    b -= p.shared_blocks;
    const int sc = over(b, p.by_own_tiles), tile = b - sc * p.own_tiles, sh = over(sc, p.by_own_chunks), c = sc - sh * p.own_chunks;
    un.seq = over(sh, p.by_kv_heads);
    un.kvh = sh - un.seq * p.c.n_kv_heads;
    un.r0 = tile * ROWS;
    un.n_rows = min(group - un.r0, ROWS);
    un.slot = p.shared_chunks + c;
    const auto resolve = [&](Unit &u) {
        const int gi = over(u.seq, p.by_width), lead = gi * p.width;
        int shared = as_global(p.shared)[gi], len = as_global(p.len)[u.seq];
        if (!seq_fits(p, shared, len)) {
            shared = len = 0;
            if (p.err && threadIdx.x == 0) *as_global(p.err) = 1;
        }
        if (p.shared_chunks == 0) {              // one block for all of it
            u.a = Stretch{lead, 0, min(shared, len)};
            u.b = Stretch{u.seq, shared, max(shared, len)};
        } else {
            const bool within = len < shared;
            const int lo = within ? 0 : shared, each = ((within ? len : len - shared) + p.own_chunks - 1) / p.own_chunks;
            u.a = Stretch{within ? lead : u.seq, min(lo + c * each, len), min(lo + (c + 1) * each, len)};
        }
        return u.a.hi > u.a.lo || u.b.hi > u.b.lo;
    };
    if (!attend<KT, DH, 1>(p, un, resolve, lds, pages, flags, lds_m, lds_l, row_scale))
        for (int r = threadIdx.x; r < un.n_rows; r += NTS) nothing(p, un, r);
}

// A block per (sequence, query head).  A thread's first chunks are asked for together with all maxima and sums: one trip to
// memory for up to UM * groups chunks.  Every wave forms the row's maximum and sum for itself, so the block meets once.  Sums in a fixed order.
// Measured, 512 rows of 128: 33 chunks each 4.0 us (a launch and three trips to memory); 1024 rows of 64: 8.0 us.
constexpr int UM = 8;
__global__ __launch_bounds__(NTS) void shared_merge_kernel(const SharedAttnArgs p) {
    __shared__ float4 acc[NTS];
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), d = p.c.d_head, per = d / 4, groups = NTS / per, gi = tid / per, ci = tid % per;
    const size_t row = blockIdx.x;
    const float *ml = p.part_ml + 2 * row * p.slots, *part = p.part + row * p.slots * d + 4 * ci;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const auto pair = [&](int i) { return ((global_ptr<const f32x2>)ml)[i]; };       // a chunk's maximum and sum
    float4 x[UM];
    f32x2 xml[UM];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int u = 0; u < UM; ++u) {
            const int i = i0 + u * groups;
            xml[u] = f32x2{-INFINITY, 0.f};
            if (i < p.slots) {
                xml[u] = pair(i);
                x[u] = global_load_float4(part + (size_t)i * d);
            }
        }
    };
    fetch(gi);
    const f32x2 first = lane < p.slots ? pair(lane) : f32x2{-INFINITY, 0.f};
    float M = first[0];
    for (int i = lane + WAVE; i < p.slots; i += WAVE) M = fmaxf(M, pair(i)[0]);
    M = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_max_last(M)), WAVE - 1));
    float L = first[1] == 0.f ? 0.f : first[1] * exp2_below(first[0], M);
    for (int i = lane + WAVE; i < p.slots; i += WAVE) {
        const f32x2 v = pair(i);
        if (v[1] != 0.f) L += v[1] * exp2_below(v[0], M);
    }
    L = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_sum_last(L)), WAVE - 1));
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = gi; i0 < p.slots; i0 += UM * groups) {
        if (i0 != gi) fetch(i0);
#pragma unroll
        for (int u = 0; u < UM; ++u) {
            if (xml[u][1] == 0.f) continue;      // nothing there: its O was not written
            const float f = exp2_below(xml[u][0], M);
            y.x += f * x[u].x; y.y += f * x[u].y; y.z += f * x[u].z; y.w += f * x[u].w;
        }
    }
    acc[tid] = y;
    __syncthreads();
    if (tid >= per) return;
    y = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int g = 0; g < groups; ++g) {
        const float4 z = acc[g * per + tid];
        y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
    }
    const float inv = L == 0.f ? 0.f : 1.f / L;
    *(f32x4 __attribute__((address_space(1))) *)(p.out + row * d + 4 * tid) = f32x4{y.x * inv, y.y * inv, y.z * inv, y.w * inv};
}

// How a call is cut: chunks of shared and of own positions per unit, and the positions of a shared chunk.
// A block costs 5 us whatever its chunk (three trips to memory before its first product, its results' way back), and each chunk
// a partial result per row, so a call takes one block per compute unit; where that leaves a block more than LONG positions, two run
// beside each other and fill each other's waits.  Measured both ways over 299 calls (seven head layouts, the three types, 2 to 64 sequences over 1024 to 65536 shared positions):
// at 192 to 832 positions of a block two take 13% longer on average, at 1024 5% (from 20% longer to 7% shorter), at 2048 they are even (from 14% shorter, mostly
// tiles of 128 rows, to 12% longer, mostly where a compute unit holds one block anyway: d_head 256, fp32).  us, one / two: 64 rows x 16384 positions x 8 heads x 128 in fp16
// 23.8 / 27.7; eight groups of 32 rows x 4096 x 8 37.1 / 44.4, x 8192 66.1 / 68.8; 128 rows x 32768 x 8 56.2 / 55.8, x 65536 98.7 / 86.3.
struct Cut { int shared_chunks, shared_chunk, own_chunks; };
constexpr int WHOLE = 512;                       // positions up to which a sequence's block takes shared and own ones in one go
constexpr int CUS = 256, LONG = 1536;
// Rows of a shared block; from 4 * ROWS on its waves share out rows, not keys.  (A sequence on its own may have a single chunk, whose block writes the output:
// the kernel whose waves share out keys.)
int tile_rows(int dtype, int d_head, int width, int group) {
    const int rows = width * group;
    const bool many = dtype != SPD_DTYPE_FP32 && d_head >= 64;
    if (rows <= ROWS || (dtype == SPD_DTYPE_FP32 && d_head > 128) || (many && width == 1)) return ROWS;
    if (!many) return 2 * ROWS;
    return rows > 4 * ROWS && d_head <= 128 && dtype == SPD_DTYPE_FP16 ? 8 * ROWS : 4 * ROWS;
}
Cut cut_for(int dtype, int n_seq, int width, int n_heads, int n_kv_heads, int d_head, int max_shared, int max_own) {
    const int groups = n_seq / width, group = n_heads / n_kv_heads;
    if (width > 1 && (long long)max_shared + max_own <= WHOLE) return Cut{0, 0, 1};
    const long long shared = std::max<long long>(1, width == 1 ? (long long)max_shared + max_own : max_shared);
    const long long units = (long long)groups * n_kv_heads * ((width * group - 1) / tile_rows(dtype, d_head, width, group) + 1), own_units = (long long)n_seq * n_kv_heads;
    const auto cut = [&](long long positions, long long of, long long blocks) {
        const long long n = std::max<long long>(1, std::min(blocks / of, (positions + NWS * KEYS - 1) / (NWS * KEYS)));
        const long long chunk = ((positions + n - 1) / n + KEYS - 1) / KEYS * KEYS;
        return std::min<long long>(chunk, CHUNK_MAX);
    };
    long long chunk = cut(shared, units, CUS);
    if (chunk > LONG || width == 1) chunk = cut(shared, units, 2 * CUS);
    const long long own_chunk = cut(std::max(1, max_own), own_units, 2 * CUS);
    return Cut{(int)((shared + chunk - 1) / chunk), (int)chunk, width == 1 ? 0 : (int)((std::max(1, max_own) + own_chunk - 1) / own_chunk)};
}

template <typename KT, int DH, int TILE, bool MANY>
constexpr int lds_bytes() {
    int b = 4 * Lds<KT, DH, MANY ? 1 : TILE / ROWS>::WORDS;
    if constexpr (MANY) b = std::max(b, Stage<DH, TILE / (NWS * ROWS)>::ST * Stage<DH, TILE / (NWS * ROWS)>::BYTES);
    return b;
}

template <typename KT, int DH, int TILE, bool MANY>
hipError_t launch_tiles(hipStream_t s, SharedAttnArgs a) {
    const int group = a.n_heads / a.c.n_kv_heads, groups = a.c.n_seq / a.width;
    a.group = group;
    a.row_tiles = (a.width * group + TILE - 1) / TILE;
    a.own_tiles = (group + ROWS - 1) / ROWS;
    const long long per_tile = (long long)groups * a.c.n_kv_heads * a.shared_chunks, shared_blocks = (per_tile + 7) / 8 * 8 * a.row_tiles;
    const long long blocks = shared_blocks + (long long)a.c.n_seq * a.c.n_kv_heads * a.own_chunks * a.own_tiles;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    a.shared_blocks = (int)shared_blocks;
    a.shared_blocks_per_tile = (int)per_tile;
    a.by_group = divisor(group); a.by_kv_heads = divisor(a.c.n_kv_heads); a.by_width = divisor(a.width); a.by_row_tiles = divisor(a.row_tiles);
    a.by_own_tiles = divisor(a.own_tiles); a.by_shared_chunks = divisor(std::max(1, a.shared_chunks)); a.by_own_chunks = divisor(std::max(1, a.own_chunks));
    constexpr int lds = lds_bytes<KT, DH, TILE, MANY>();
    if (lds > 60 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)shared_attn_kernel<KT, DH, TILE, MANY>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((shared_attn_kernel<KT, DH, TILE, MANY>), dim3((unsigned)blocks), dim3(NTS), lds, s, a);
    if (a.slots > 1) hipLaunchKernelGGL(shared_merge_kernel, dim3((unsigned)(a.c.n_seq * a.n_heads)), dim3(NTS), 0, s, a);
    return hipGetLastError();
}

template <typename KT, int DH>
hipError_t launch_rows(hipStream_t s, const SharedAttnArgs &a, int dtype) {
    const int tile = a.shared_chunks ? tile_rows(dtype, a.c.d_head, a.width, a.n_heads / a.c.n_kv_heads) : ROWS;
    if (tile == ROWS) return launch_tiles<KT, DH, ROWS, false>(s, a);
    if constexpr (sizeof(KT) == 2 && DH >= 64) {
        if constexpr (DH <= 128 && Type<KT>::PARTS == 2)
            if (tile == 8 * ROWS) return launch_tiles<KT, DH, 8 * ROWS, true>(s, a);
        return launch_tiles<KT, DH, 4 * ROWS, true>(s, a);
    } else if constexpr (sizeof(KT) == 4 && DH > 128) {
        return hipErrorInvalidValue;             // (tiles of 16 rows alone)
    } else {
        return launch_tiles<KT, DH, 2 * ROWS, false>(s, a);
    }
}

template <typename KT>
hipError_t launch_width(hipStream_t s, const SharedAttnArgs &a, int dtype) {
    if (a.c.d_head <= 32) return launch_rows<KT, 32>(s, a, dtype);
    if (a.c.d_head == 64) return launch_rows<KT, 64>(s, a, dtype);
    if (a.c.d_head == 128) return launch_rows<KT, 128>(s, a, dtype);
    return launch_rows<KT, 256>(s, a, dtype);
}

}  // namespace

extern "C" size_t spd_op_attention_shared_scratch_bytes(int32_t n_seq, int32_t width, int32_t n_heads, int32_t n_kv_heads, int32_t d_head, int32_t max_shared,
                                                        int32_t max_own) {
    if (n_seq <= 0 || width <= 0 || n_seq % width || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || d_head <= 0 || max_shared < 0 || max_own < 0) return 0;
    int slots = 0;                               // (the most of the three types)
    for (int dtype : {SPD_DTYPE_FP32, SPD_DTYPE_BF16, SPD_DTYPE_FP16}) {
        const Cut c = cut_for(dtype, n_seq, width, n_heads, n_kv_heads, d_head, max_shared, max_own);
        slots = std::max(slots, c.shared_chunks + c.own_chunks);
    }
    const size_t parts = (size_t)n_seq * n_heads * slots;
    return slots > 1 ? up256(parts * 8) + up256(parts * d_head * 4) : 0;
}

extern "C" int spd_test_attention_shared_cut(int32_t dtype, int32_t n_seq, int32_t width, int32_t n_heads, int32_t n_kv_heads, int32_t d_head, int32_t max_shared, int32_t max_own,
                                             int32_t *out) {
    if (!out || n_seq <= 0 || width <= 0 || n_seq % width || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || max_shared < 0 || max_own < 0) return SPD_EINVAL;
    const Cut c = cut_for(dtype, n_seq, width, n_heads, n_kv_heads, d_head, max_shared, max_own);
    const int group = n_heads / n_kv_heads, tile = c.shared_chunks ? tile_rows(dtype, d_head, width, group) : ROWS;
    out[0] = c.shared_chunks; out[1] = c.shared_chunk; out[2] = c.own_chunks; out[3] = tile;
    out[4] = c.shared_chunks * (n_seq / width) * n_kv_heads * ((width * group + tile - 1) / tile);
    out[5] = out[6] = 0;
    if (tile >= 4 * ROWS) {
        const bool two = tile == 8 * ROWS;
        out[5] = d_head == 64 ? (two ? Stage<64, 2>::SK : Stage<64, 1>::SK) : d_head == 128 ? (two ? Stage<128, 2>::SK : Stage<128, 1>::SK) : Stage<256, 1>::SK;
        out[6] = d_head == 64 ? (two ? Stage<64, 2>::ST : Stage<64, 1>::ST) : d_head == 128 ? (two ? Stage<128, 2>::ST : Stage<128, 1>::ST) : Stage<256, 1>::ST;
    }
    return SPD_OK;
}

extern "C" int spd_op_attention_shared(int32_t dtype, const float *q, const void *K, const void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads,
                                       int32_t page_size, int32_t d_head, int32_t n_seq, int32_t table_stride, const int32_t *shared, const int32_t *len,
                                       int32_t width, int32_t n_heads, int32_t max_shared, int32_t max_own, float *out, void *scratch, size_t scratch_bytes,
                                       int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache((void *)K, (void *)V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    const int rc = spdk::paged_cache_status(dtype, c, page_size);
    if (rc != SPD_OK) return rc;
    if (width < 1 || n_seq % width || n_heads < 1 || n_heads % n_kv_heads || max_shared < 0 || max_own < 0) return SPD_EINVAL;
    const long long room = (long long)table_stride * page_size;      // (the longest shared and the longest own part may be different sequences')
    if (max_shared > room || max_own > room || (long long)max_shared + max_own > INT32_MAX / 2) return SPD_EINVAL;
    if (n_seq == 0) return SPD_OK;
    if ((long long)n_seq * n_heads > (1 << 24)) return SPD_EINVAL;
    if (!q || !shared || !len || !out || ((uintptr_t)q | (uintptr_t)out) % 16) return SPD_EINVAL;
    const size_t need = spd_op_attention_shared_scratch_bytes(n_seq, width, n_heads, n_kv_heads, d_head, max_shared, max_own);
    if (need && (!scratch || (uintptr_t)scratch % 256)) return SPD_EINVAL;
    if (scratch_bytes < need) return SPD_EWORKSPACE;
    // what is written lies apart from what other blocks read (several share a head's queries)
    const size_t rows = (size_t)n_seq * n_heads * d_head * 4, pool = spdk::pool_bytes(dtype, c);
    const spdk::Span sq{q, rows}, so{out, rows}, sK{K, pool}, sV{V, pool}, st{table, (size_t)n_seq * table_stride * 4}, ss{shared, (size_t)(n_seq / width) * 4}, sl{len, (size_t)n_seq * 4},
        se{err, 4}, sw{scratch, need};
    if (spdk::over_any(so, {sq, sK, sV, st, ss, sl, se, sw}) || spdk::over_any(sw, {sq, sK, sV, st, ss, sl, se})) return SPD_EINVAL;
    const Cut cut = cut_for(dtype, n_seq, width, n_heads, n_kv_heads, d_head, max_shared, max_own);
    SharedAttnArgs a{};
    a.c = c; a.q = q; a.out = out; a.shared = shared; a.len = len; a.err = err;
    a.width = width; a.n_heads = n_heads; a.max_shared = max_shared; a.max_own = max_own;
    a.shared_chunks = cut.shared_chunks; a.shared_chunk = cut.shared_chunk; a.own_chunks = cut.own_chunks; a.slots = cut.shared_chunks + cut.own_chunks;
    a.part_ml = (float *)scratch;
    a.part = (float *)((char *)scratch + up256((size_t)n_seq * n_heads * a.slots * 8));
    hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch_width<float>(s, a, dtype) : dtype == SPD_DTYPE_FP16 ? launch_width<half_t>(s, a, dtype) : launch_width<bf16_t>(s, a, dtype);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}
