// Causal attention of every sequence's new tokens over a paged cache.
//
// Rows of a key/value head: its query heads of all new tokens of a sequence, token by token.  A block owns (64 or 128 rows of a
// sequence, key/value head, chunk of positions); rows share every key that they meet, so the tile's rows are what a cached byte is used for.  Both
// products run on the matrix cores, S^T [key, row] = K Q^T and O^T [feature, row] = V^T P^T, in tiles of 32 keys or features by 32 rows:
//   * S^T's accumulator holds, of one row, keys 8 i + 4 h + r (h: the lane's half, r < 4, i < 4), which is P^T's operand layout when a lane's eight k indices
//     stand for keys 4 h .. 4 h + 3 and 8 + 4 h .. 8 + 4 h + 3: probabilities never leave their registers;
//   * V^T's operand for those keys is two reads of four keys each that LDS turns round on the way (16-bit types; fp32 values go in one by one).
// Keys and values come through LDS in stages of 64 positions, two deep, 16 bytes per lane straight from memory; codes of 8 bits come through registers and
// lie in LDS as fp16 numbers, which they are exactly: a key's scale multiplies its scores, a value's its probability
// (held by the power of two of the largest scale so far, or, where scales lie far apart, row by row by the largest product of both).  Pieces of a row are permuted by the row's
// number, so that the operand reads meet in no bank.  One barrier per stage.
// Bound: the matrix cores where there are many rows (and with all 24 bits of them two or three products for each), else the vector unit, which forms some 500 instructions per wave and stage
// (masks, exponentials, parts of them, codes to numbers) in between: a wave's products and its exponentials follow one another, and two blocks per compute unit are what registers allow.
// Measured (kernel alone; then what the bytes or products alone would take): 512 tokens of 64 heads on 8 behind 32257 positions in fp16, 24 bits, 0.94 ms = 1.16 PFLOP/s in two products each, the rate of a large
// fp16 product; 2999 tokens of 32 heads in bf16 from their beginnings 52 us (23); 40 tokens of eight sequences over 4001 positions of 8 bits 31 us (9); four tokens behind 73 positions 9 us.
// The four waves of a block of 128 rows share out rows; of 64, rows and the stage's halves.  Where there are few tiles the positions are cut into chunks, and a second
// kernel puts a row's chunks together in order.
#include "spd_attention.h"

#include <algorithm>

using namespace spdd;
using namespace spda;

namespace {

constexpr int NT = 256, NW = NT / WAVE;
constexpr int TR = 32;                           // rows (and keys, features) of a matrix product
// 8 bits: scales of values that lie no further than 2^NARROW apart are held by the largest.  The largest product of a row's is 2^12 2^-13 at least then, and what 16 bits lose, 2^-25, is 2^-24 of it.
// LIFT_MAX: a row may be up to that power of two larger: its sums, of up to 2^30 keys, stay below 2^(15 + 7 + 30 + 64), inside of fp32's range.
constexpr int NARROW = 12, LIFT_MAX = 64;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct q8_t { int8_t b; };                       // codes: fp16 numbers in the products
template <typename KT> struct InLds { typedef KT type; };
template <> struct InLds<q8_t> { typedef half_t type; };

// Queries and probabilities are PARTS numbers of the cache's type each: all 24 bits where rows are fp32, one number where they are of 16 bits.
// P: exp2(score - reference + P_BITS) P_SCALE, as for Type.
template <typename KT, typename IO> struct Kind {
    typedef typename InLds<KT>::type LT;
    static constexpr bool F32 = sizeof(KT) == 4, Q8 = sizeof(KT) == 1;
    static constexpr int PARTS = sizeof(IO) == 4 ? Type<LT>::PARTS : 1;
    // (one number of 16 bits: an exponent that is off by 2^-20 does not show, and the factor would be an instruction per key)
    static constexpr bool IN_EXPONENT = PARTS == 1 && !F32;
    static constexpr float P_SCALE = IN_EXPONENT ? 1.f : Type<LT>::P_SCALE, P_BITS = Type<LT>::PARTS == 2 ? Type<LT>::P_BITS : IN_EXPONENT ? -24.f : 0.f;
};

template <typename KT, typename IO, int DH, int RW> struct Shape {
    typedef Kind<KT, IO> T;
    static constexpr int KW = NW / RW, ROWS = RW * TR;                                  // waves that share out keys; rows of a block
    static constexpr int ROWB = DH * (T::F32 ? 4 : 2), PIECES = ROWB / 16;              // bytes and 16-byte pieces of a row in LDS
    static constexpr int SK = (DH == 256 || T::F32) && KW == 1 ? 32 : 64, NU = SK / (TR * KW);       // keys of a stage; tiles of keys of a wave
    static constexpr int HALF = SK * ROWB, BYTES = 2 * HALF, LOADS = HALF / 16 / NT;    // K, then V; pieces per thread, of K as of V
    // Heads of 256 with 24 bits over bf16 or fp32: queries and results together are more than a wave's registers, so a block takes half of the features of the values (its scores are formed
    // twice).
    static constexpr int FS = DH == 256 && (T::F32 || T::PARTS == 3) ? 2 : 1;
    static constexpr int ST = 2, LDS = ST * BYTES;
    static constexpr int PER_CU = LDS <= 80 * 1024 && DH <= 128 && T::PARTS < 3 ? 2 : 1;   // blocks side by side: 256 or 512 registers
};

// Where piece `piece` of row `key` lies.  K: 16 rows side by side are read at one piece.  V: four rows by four pieces (fp32: two rows, four apart, by eight).
template <int PIECES> __device__ __forceinline__ int k_place(int key, int piece) {
    return PIECES >= 16 ? piece ^ (key & 15) : PIECES == 8 ? piece ^ ((key >> 1) & 7) : piece ^ ((key >> 2) & 3);
}
template <int PIECES, bool F32> __device__ __forceinline__ int v_place(int key, int piece) {
    if (F32) return PIECES >= 16 ? piece ^ (((key >> 2) & 1) << 3) : piece;
    return PIECES >= 16 ? piece ^ ((key & 3) << 2) : PIECES == 8 ? piece ^ (((key >> 1) & 1) << 2) : piece;
}

template <typename LT> __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c);
template <> __device__ __forceinline__ f32x16 mfma32<half_t>(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x16 mfma32<bf16_t>(u32x4 a, u32x4 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// 16 bytes per lane straight into LDS, `to` + 16 lane on.  Written out, because the compiler, which knows the instruction, lets every turned read wait for all of them; they are
// waited for once per stage.  (No vector register is written; M0 is set right before its use, and named as lost.)
__device__ __forceinline__ void stage16(const char *from, uint32_t off, const char *to) {     // (from + off, off per lane)
#if defined(__HIP_DEVICE_COMPILE__)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"((uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)to), "v"(off), "s"(from) : "memory", "m0");
#endif
}

// The same for N pieces in a row (at most four), 1024 bytes apart in memory as in LDS: the offset of the instruction counts for both.
template <int N> __device__ __forceinline__ void stage16_each(const char *from, const uint32_t (&off)[N], const char *to) {
#if defined(__HIP_DEVICE_COMPILE__)
    const uint32_t m = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) char *)to;
    if constexpr (N == 1) stage16(from, off[0], to);
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %3\n\tglobal_load_lds_dwordx4 %2, %3 offset:1024" ::"s"(m), "v"(off[0]), "v"(off[1]), "s"(from) : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %5\n\tglobal_load_lds_dwordx4 %2, %5 offset:1024\n\tglobal_load_lds_dwordx4 %3, %5 offset:2048\n\t"
                     "global_load_lds_dwordx4 %4, %5 offset:0xc00" ::"s"(m), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(from) : "memory", "m0");
#endif
}

// All loads have arrived, in registers (the compiler knows) and in LDS.
__device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0)
    asm volatile("" ::: "memory");
}

// Four rows of four 16-bit numbers per lane, turned round among 16 lanes: lane i gets four rows of column i.
__device__ __forceinline__ u32x2 turned_read(const char *p) {
    u32x2 v{0, 0};
#if defined(__HIP_DEVICE_COMPILE__)
    v = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)p));
#endif
    return v;
}

// Four codes as four fp16 numbers: 1024 + 128 + code, less 1152.
__device__ __forceinline__ void codes_to_half(uint32_t codes, uint32_t &lo, uint32_t &hi) {
    const uint32_t x = codes ^ 0x80808080u;
    const f16x2 off{(_Float16)-1152.f, (_Float16)-1152.f};
    lo = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u)) + off);
    hi = __builtin_bit_cast(uint32_t, __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u)) + off);
}

// Two fp32 numbers as pairs of LT, PARTS of them; one: rounded to nearest.
template <typename LT, int PARTS> __device__ __forceinline__ void probability_parts(float x, float y, uint32_t (&out)[PARTS]) {
    if constexpr (PARTS > 1) parts_of<LT>(x, y, out);
    else if constexpr (sizeof(LT) == 2) {
        typedef _Float16 hpair __attribute__((ext_vector_type(2)));
        typedef __bf16 bpair __attribute__((ext_vector_type(2)));
        if constexpr (Type<LT>::PARTS == 2) out[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v{x, y}), hpair));
        else out[0] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2v{x, y}), bpair));
    }
}

// Adds the two numbers of a pair.
template <typename LT> __device__ __forceinline__ float pair_sum(uint32_t pair, float sum) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __bf16 bpair __attribute__((ext_vector_type(2)));
    if constexpr (Type<LT>::PARTS == 2) return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, pair), f16x2{(_Float16)1.f, (_Float16)1.f}, sum, false);
    else return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bpair, pair), __builtin_bit_cast(bpair, 0x3F803F80u), sum, false);
#else
    return sum;
#endif
}

// Whether any of the 16 bytes' numbers is infinite or none.
template <int BYTES> __device__ __forceinline__ bool not_finite(u32x4 v, bool bf) {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (BYTES == 4) bad |= (v[i] & 0x7F800000u) == 0x7F800000u;
        else {
            const uint32_t e = bf ? 0x7F80u : 0x7C00u;
            bad |= ((v[i] & e) == e) | (((v[i] >> 16) & e) == e);
        }
    }
    return bad;
}

// The tile of rows that is the block's: of the launch's x-th, the tiles farthest behind their sequence's beginning first (they see the most keys; a call whose last blocks are its
// longest ones waits for them: prompts of 2999 tokens in the order of their rows 54 us, so 50 at the time).  Up to 64 sequences are looked at by one wave at once, one trip to memory: sequences with more than T tiles each have one at
// every height below T, so x is found by going down from the tallest.  More sequences: tiles in the order of rows, sequence s's from over(first[s]) + s on (over: whole tiles in front), which
// needs no sum over sequences; late ones first.  False: none, or first descends somewhere (then there is no telling whose rows are whose).  The launch's first block looks for sequences whose numbers do not fit
// (others see their own only, and a sequence outside of all rows is nobody's).
struct Whose { int seq, a, b, len, tile; };
__device__ __forceinline__ bool fits(const PagedAttnArgs &p, int a, int b, int len) {
    return a >= 0 && b <= p.n_tokens && len >= b - a && len <= p.max_len && (long long)len <= (long long)p.c.table_stride << p.c.page_shift;
}
__device__ __forceinline__ bool whose(const PagedAttnArgs &p, int x, int log2_rows, int lane, Whose &w, bool &descends) {
    const bool look = blockIdx.x == 0 && p.err;
    if (p.c.n_seq <= WAVE) {
        const int i = min(lane, p.c.n_seq - 1), a = as_global(p.first)[i], b = as_global(p.first)[i + 1], len = as_global(p.len)[i];
        descends = __any(b < a);
        if (descends) return false;
        if (look && !fits(p, a, b, len)) *as_global(p.err) = 1;
        const int tokens = max(min(b, p.n_tokens) - max(a, 0), 0);
        const int tiles = lane < p.c.n_seq ? (tokens * p.group + (1 << log2_rows) - 1) >> log2_rows : 0;
        const auto tallest = [&](int below) { return (int)__int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_max_last(tiles < below ? (float)tiles : 0.f)), WAVE - 1)); };
        for (int top = tallest(INT32_MAX); top > 0;) {
            const u64 with = __ballot(tiles >= top);
            const int next = tallest(top), n = __popcll(with), of = n * (top - next);
            if (x >= of) {
                x -= of;
                top = next;
                continue;
            }
            int down = 0;
            if (n > 1)
                while (x >= n) { x -= n; ++down; }
            else {
                down = x;
                x = 0;
            }
            u64 left = with;
            for (; x > 0; --x) left &= left - 1;
            const int s = __builtin_ctzll(left);
            w.seq = s;
            w.a = __builtin_amdgcn_readlane(a, s);
            w.b = __builtin_amdgcn_readlane(b, s);
            w.len = __builtin_amdgcn_readlane(len, s);
            w.tile = top - 1 - down;
            return true;
        }
        return false;
    }
    const int tile = p.n_tiles - 1 - x;
    int s = 0;
    bool bad = false;
    const auto start = [&](int i, int f) { return (int)(((unsigned)min(max(f, 0), p.n_tokens) * (unsigned)p.group) >> log2_rows) + i; };
    for (int i0 = 0; i0 < p.c.n_seq; i0 += WAVE) {
        const int i = min(i0 + lane, p.c.n_seq - 1), a = as_global(p.first)[i], b = as_global(p.first)[i + 1];
        bad = bad || b < a;
        if (look && !fits(p, a, b, as_global(p.len)[i])) *as_global(p.err) = 1;
        s += __popcll(__ballot(i0 + lane < p.c.n_seq && start(i + 1, b) <= tile));
    }
    descends = __any(bad);
    if (descends || s >= p.c.n_seq) return false;
    w.seq = s;
    w.a = __builtin_amdgcn_readfirstlane(as_global(p.first)[s]);
    w.b = __builtin_amdgcn_readfirstlane(as_global(p.first)[s + 1]);
    w.len = __builtin_amdgcn_readfirstlane(as_global(p.len)[s]);
    w.tile = tile - start(s, w.a);
    return true;
}

template <typename IO> __device__ __forceinline__ void store_rows(void *p, size_t i, float4 v) {
    if constexpr (sizeof(IO) == 4) *(f32x4 __attribute__((address_space(1))) *)((float *)p + i) = f32x4{v.x, v.y, v.z, v.w};
    else {
        uint32_t lo[1], hi[1];
        probability_parts<IO, 1>(v.x, v.y, lo);
        probability_parts<IO, 1>(v.z, v.w, hi);
        *(u32x2 __attribute__((address_space(1))) *)((uint16_t *)p + i) = u32x2{lo[0], hi[0]};
    }
}

template <typename KT, typename IO, int DH, int RW>
__global__ __launch_bounds__(NT, (Shape<KT, IO, DH, RW>::PER_CU)) void paged_attn_kernel(const PagedAttnArgs p) {
    typedef Kind<KT, IO> T;
    typedef Shape<KT, IO, DH, RW> S;
    typedef typename T::LT LT;
    constexpr bool F32 = T::F32, Q8 = T::Q8;
    constexpr int PARTS = T::PARTS, KW = S::KW, ROWS = S::ROWS, ROWB = S::ROWB, PIECES = S::PIECES, SK = S::SK, NU = S::NU, HALF = S::HALF, BYTES = S::BYTES, LOADS = S::LOADS;
    constexpr bool LEAN = DH == 256 || Q8 || (F32 && DH == 128);                   // registers are scarce
    constexpr int FS = S::FS, NJ = F32 ? DH / 8 : DH / 16, NF = DH / TR / FS, PIECE_EL = F32 ? 4 : 8, LOG2_ROWS = RW == 4 ? 7 : 6;
    extern __shared__ __align__(1024) char lds[];
    __shared__ int bad_stage[2], odd_stage[2];               // the stage, + 1, that has a key on no page, a value that is no finite number
    __shared__ __align__(16) float k_sc[2][SK], v_sc[2][SK];
    __shared__ int v_exp[2];
    __shared__ u64 odd_keys[2];
    __shared__ float join_m[RW][WAVE], join_l[RW][WAVE];
    __shared__ int join_e[Q8 && KW > 1 ? RW : 1][WAVE];
    const int tid = threadIdx.x, lane = tid & (WAVE - 1), wv = __builtin_amdgcn_readfirstlane(tid / WAVE), col = lane & (TR - 1), h = lane / TR, rw = wv % RW, kw = wv / RW;
    const int d = p.c.d_head, shift = p.c.page_shift, in_page = (1 << shift) - 1, group = p.group;
    // which rows, which positions
    const int block = blockIdx.x / FS, share = blockIdx.x % FS, rest = over(block, p.by_kv_heads), kvh = block - rest * p.c.n_kv_heads, tile_r = over(rest, p.by_splits), split = rest - tile_r * p.splits;
    Whose own;
    bool descends;
    const bool found = whose(p, tile_r, LOG2_ROWS, lane, own, descends);
    if (descends && blockIdx.x == 0 && tid == 0 && p.err) *as_global(p.err) = 1;
    if (!found) return;
    const int r0 = own.tile * ROWS, n = own.b - own.a, from = max(own.a, 0), n_rows = min(((min(own.b, p.n_tokens) - from) * group) - r0, ROWS);
    if (n_rows <= 0) return;
    const int len = own.len;
    if (!fits(p, own.a, own.b, len)) {
        if (split == 0 && share == 0)
            for (int i = tid; i < n_rows * d / 4; i += NT) {
                const int r = r0 + i / (d / 4), tok = over(r, p.by_group);
                store_rows<IO>(p.out, ((size_t)(from + tok) * p.n_heads + kvh * group + r - tok * group) * d + 4 * (i % (d / 4)), make_float4(0.f, 0.f, 0.f, 0.f));
            }
        return;
    }
    const int pos0 = len - n, pos_min = pos0 + over(r0, p.by_group), pos_max = pos0 + over(r0 + n_rows - 1, p.by_group);
    const int lo = split * p.chunk, hi = min(pos_max + 1, lo + p.chunk);
    if (lo >= hi) return;
    const int stages = (hi - lo + SK - 1) / SK;
    const int r = r0 + min(rw * TR + col, n_rows - 1), tok = over(r, p.by_group), pos = pos0 + tok;       // (rows past the last repeat it)
    const bool active = rw * TR < n_rows;
    const int wave_lo = __builtin_amdgcn_readfirstlane(pos), wave_hi = __builtin_amdgcn_readlane(pos, TR - 1);
    const size_t row_at = (size_t)(own.a + tok) * p.n_heads + kvh * group + r - tok * group;

    const int row_bytes = d * (int)sizeof(KT), row_shift = 31 - __builtin_clz((unsigned)row_bytes), head_shift = row_shift + shift;
    const char *K = (const char *)p.c.K, *V = (const char *)p.c.V;
    const int32_t *entries = p.c.table + (size_t)own.seq * p.c.table_stride;
    if (tid < 2) bad_stage[tid] = odd_stage[tid] = 0;
    if constexpr (DH == 32) {                                // heads narrower than the tile: nothing is ever put behind their ends
        for (int i = tid; i < S::LDS / 16; i += NT) ((u32x4 *)lds)[i] = u32x4{0, 0, 0, 0};
        __syncthreads();
    }
    const auto of_share = [&]() { return FS == 1 || lane % PIECES / (PIECES / 2) == share; };      // (places are permuted within halves of a row)
    // A wave's part of a stage is LOADS pieces of KEYS keys each, side by side.  Where they lie on one page, page number (asked for a stage ahead) and address are formed once, by the wave; a lane's part of
    // the address stays the same, but for the permutation.  Shorter pages: piece by piece, or, where a piece lies on several, page by page.
    // Measured, 2999 tokens of prompts over pages of 16: a piece's address each and page numbers as vector loads 51.1 us, so 48.8.
    constexpr int KEYS = WAVE / PIECES, OWN = KEYS * LOADS;
    const bool one = DH > 32 && OWN <= 1 << shift, whole = KEYS <= 4 || KEYS <= 1 << shift;
    const auto place = [&](int i) { return ((wv * LOADS + i) * WAVE + lane) * 16; };          // of this thread's piece i in LDS
    int page[LOADS], scale_page = 0;
    const auto entry = [&](int pos) { return ((const __attribute__((address_space(4))) int32_t *)entries)[pos >> shift]; };      // (of the wave: a scalar load)
    const auto ask = [&](int t) {
        if (one) page[0] = entry(min(lo + t * SK + wv * OWN, (hi - 1) & ~(OWN - 1)));
        else if (whole) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) page[i] = entry(min(lo + t * SK + wv * OWN + i * KEYS, (hi - 1) & ~(KEYS - 1)));
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) page[i] = as_global(entries)[min(lo + t * SK + wv * OWN + i * KEYS + lane / PIECES, hi - 1) >> shift];
        }
    };
    u32x2 kc[LOADS], vc[LOADS];                              // Q8: a stage's codes and scales on their way
    float scale_in = 0.f;
    float v_low = 200.f;                                     // (of the scales that have been this lane's)
    int drop = 0, drop_next = 0, v_top = -200;               // (drop: bit i: this thread's piece i of the stage is of a key that does not count)
    const auto fetch = [&](int t) {
        char *to = lds + (t % 2) * BYTES + wv * (LOADS * WAVE * 16);
        const bool end = lo + (t + 1) * SK > hi;
        int lane = tid & (WAVE - 1);
        if constexpr (LEAN) asm volatile("" : "+v"(lane));
        drop_next = 0;
        bool bad = false;
        if constexpr (Q8) {                                  // scales, and page numbers for the next stage's: in front of the codes (behind them they wait for room on the way to memory, 700 cycles)
            if (wv < 2) {
                const int at = lo + t * SK + lane % SK;
                const bool ok = (unsigned)scale_page < (unsigned)p.c.n_pages;
                scale_in = 0.f;
                if (ok && at < hi) scale_in = as_global(wv == 0 ? p.k_scale : p.v_scale)[((size_t)(uint32_t)(scale_page * p.c.n_kv_heads + kvh) << shift) + (at & in_page)];
                if (t + 1 < stages) scale_page = as_global(entries)[min(lo + (t + 1) * SK + lane % SK, hi - 1) >> shift];
            }
        }
        if (one) {
            constexpr int UNIT = Q8 ? 8 : 16;
            const int pg = __builtin_amdgcn_readfirstlane(page[0]), pos0 = min(lo + t * SK + wv * OWN, (hi - 1) & ~(OWN - 1)), key = wv * OWN + lane / PIECES, slot = lane % PIECES;
            bad = (unsigned)pg >= (unsigned)p.c.n_pages;
            const u64 row = ((u64)(uint32_t)((bad ? 0 : pg) * p.c.n_kv_heads + kvh) << head_shift) + ((u64)(uint32_t)(pos0 & in_page) << row_shift);
            const char *k_row = K + row, *v_row = V + row;
            // a key's bits go into its row's places by exclusive or: piece i's by a constant
            const uint32_t in_row = (uint32_t)(lane / PIECES) * (PIECES * UNIT), k_off = in_row + UNIT * k_place<PIECES>(key, slot), v_off = in_row + UNIT * v_place<PIECES, F32>(key, slot);
            if constexpr (Q8) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) kc[i] = *(const u32x2 __attribute__((address_space(1))) *)(k_row + i * (WAVE * UNIT) + (k_off ^ UNIT * k_place<PIECES>(KEYS * i, 0)));
#pragma unroll
                for (int i = 0; i < LOADS; ++i) vc[i] = *(const u32x2 __attribute__((address_space(1))) *)(v_row + i * (WAVE * UNIT) + (v_off ^ UNIT * v_place<PIECES, F32>(KEYS * i, 0)));
            } else {
                constexpr int EACH = LOADS < 4 ? LOADS : 4;
#pragma unroll
                for (int i = 0; i < LOADS; i += EACH) {
                    uint32_t off[EACH];
#pragma unroll
                    for (int e = 0; e < EACH; ++e) off[e] = k_off ^ UNIT * k_place<PIECES>(KEYS * (i + e), 0);
                    stage16_each<EACH>(k_row + i * (WAVE * 16), off, to + i * (WAVE * 16));
                }
                if (of_share())
#pragma unroll
                    for (int i = 0; i < LOADS; i += EACH) {
                        uint32_t off[EACH];
#pragma unroll
                        for (int e = 0; e < EACH; ++e) off[e] = v_off ^ UNIT * v_place<PIECES, F32>(KEYS * (i + e), 0);
                        stage16_each<EACH>(v_row + i * (WAVE * 16), off, to + HALF + i * (WAVE * 16));
                    }
            }
            if (end || bad)
#pragma unroll
                for (int i = 0; i < LOADS; ++i) drop_next |= (int)(bad || lo + t * SK + key + KEYS * i >= hi) << i;
        } else
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int key0 = wv * OWN + i * KEYS, key = key0 + lane / PIECES, slot = lane % PIECES, at = lo + t * SK + key;
            const int kp = k_place<PIECES>(key, slot), vp = v_place<PIECES, F32>(key, slot);
            const auto issue = [&](const char *k_row, const char *v_row, uint32_t off) {
                if constexpr (Q8) {
                    if (DH > 32 || 8 * kp < d) kc[i] = *(const u32x2 __attribute__((address_space(1))) *)(k_row + (off + 8 * kp));
                    if (DH > 32 || 8 * vp < d) vc[i] = *(const u32x2 __attribute__((address_space(1))) *)(v_row + (off + 8 * vp));
                } else {
                    if (DH > 32 || PIECE_EL * kp < d) stage16(k_row, off + 16 * kp, to + i * (WAVE * 16));
                    if ((DH > 32 || PIECE_EL * vp < d) && of_share()) stage16(v_row, off + 16 * vp, to + HALF + i * (WAVE * 16));
                }
            };
            bool ok;
            if (whole) {                                     // the wave's first row, and the lane's behind it
                const int pg = __builtin_amdgcn_readfirstlane(page[i]), pos0 = min(lo + t * SK + key0, (hi - 1) & ~(KEYS - 1));
                ok = (unsigned)pg < (unsigned)p.c.n_pages;
                const u64 row = ((u64)(uint32_t)((ok ? pg : 0) * p.c.n_kv_heads + kvh) << head_shift) + ((u64)(uint32_t)(pos0 & in_page) << row_shift);
                issue(K + row, V + row, (uint32_t)(lane / PIECES) << row_shift);
            } else {                                         // short pages: page by page, each for its own lanes
                ok = (unsigned)page[i] < (unsigned)p.c.n_pages;
                const int pos0 = min(at, hi - 1);
                u64 left = __ballot(true);
                while (left) {
                    const int first = __builtin_ctzll(left), pg = __builtin_amdgcn_readlane(page[i], first), pos1 = __builtin_amdgcn_readlane(pos0, first) & ~in_page;
                    const bool mine = (pos0 & ~in_page) == pos1;
                    left &= ~__ballot(mine);
                    const u64 row = (u64)(uint32_t)(((unsigned)pg < (unsigned)p.c.n_pages ? pg : 0) * p.c.n_kv_heads + kvh) << head_shift;
                    if (mine) issue(K + row, V + row, (uint32_t)(pos0 & in_page) << row_shift);
                }
            }
            bad = bad || !ok;
            if (end || !ok) drop_next |= (int)(!ok || at >= hi) << i;
        }
        if (bad) {
            bad_stage[t % 2] = t + 1;
            if (p.err) *as_global(p.err) = 1;
        }
    };
    const auto put = [&](int t) {                            // Q8: codes and scales to LDS
        char *to = lds + (t % 2) * BYTES;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int slot = lane % PIECES, key = wv * OWN + i * KEYS + lane / PIECES;
            u32x4 x;
            uint32_t a, b;
            codes_to_half(kc[i].x, a, b); x.x = a; x.y = b;
            codes_to_half(kc[i].y, a, b); x.z = a; x.w = b;
            if (DH > 32 || 8 * k_place<PIECES>(key, slot) < d) *(u32x4 *)(to + place(i)) = x;
            codes_to_half(vc[i].x, a, b); x.x = a; x.y = b;
            codes_to_half(vc[i].y, a, b); x.z = a; x.w = b;
            if (DH > 32 || 8 * v_place<PIECES, F32>(key, slot) < d) *(u32x4 *)(to + HALF + place(i)) = x;
        }
        if (wv == 0 && lane < SK) k_sc[t % 2][lane] = scale_in;
        if (wv == 1) {                                       // the values' scales by the power of two of the largest so far, and whether some have been far smaller
            const float size = fabsf(scale_in);
            const float ex = size > 0.f && size < INFINITY ? (float)__builtin_amdgcn_frexp_expf(size) : -200.f;
            v_top = max(v_top, (int)__int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_max_last(ex)), WAVE - 1)));
            v_low = ex > -200.f ? fminf(v_low, ex) : v_low;
            const bool odd = !(size < INFINITY);             // counts as zero; rows that see it get no number
            if (lane < SK) v_sc[t % 2][lane] = odd ? 0.f : ldexpf(scale_in, -v_top);
            const u64 keys = __ballot(odd && lane < SK);
            if (keys && lane == 0) { odd_stage[t % 2] = t + 1; odd_keys[t % 2] = keys; }
            const bool apart = __ballot(v_low < (float)(v_top - NARROW));
            if (lane == 0) v_exp[t % 2] = 2 * v_top + apart;
        }
    };

    ask(0);
    if constexpr (Q8)
        if (wv < 2) scale_page = as_global(entries)[min(lo + lane % SK, hi - 1) >> shift];
    // this lane's query: its row's features 16 j + 8 h .. + 7 (fp32: 8 j + 4 h .. + 3)
    u32x4 Q[NJ][PARTS];
    float scale = 1.4426950408889634f / sqrtf((float)d);     // to logarithms of base 2
    {
        const size_t q_at = (size_t)(own.a + tok) * p.q_stride + (size_t)(kvh * group + r - tok * group) * d;
        if constexpr (F32) {
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int f = 8 * j + 4 * h;
                const float4 x = DH > 32 || f < d ? global_load_float4((const float *)p.q + q_at + f) : make_float4(0.f, 0.f, 0.f, 0.f);
                Q[j][0] = u32x4{__float_as_uint(x.x), __float_as_uint(x.y), __float_as_uint(x.z), __float_as_uint(x.w)};
            }
        } else {
            float x[NJ][8];
            float top = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int f = 16 * j + 8 * h;
                const bool in = DH > 32 || f < d;
                if constexpr (sizeof(IO) == 4) {
                    const float4 a = in ? global_load_float4((const float *)p.q + q_at + f) : make_float4(0.f, 0.f, 0.f, 0.f), b = in ? global_load_float4((const float *)p.q + q_at + f + 4) : make_float4(0.f, 0.f, 0.f, 0.f);
                    x[j][0] = a.x; x[j][1] = a.y; x[j][2] = a.z; x[j][3] = a.w; x[j][4] = b.x; x[j][5] = b.y; x[j][6] = b.z; x[j][7] = b.w;
                } else {
                    Q[j][0] = in ? global_load16((const uint16_t *)p.q + q_at + f) : u32x4{0, 0, 0, 0};
                    Store<IO>::unpack(Q[j][0], x[j]);
                }
            }
            if constexpr (!(sizeof(IO) == 2 && Type<IO>::PARTS == Type<LT>::PARTS)) {        // (rows of the products' own type go in as they are)
                float up = 1.f, down = 1.f;
                if constexpr (Type<LT>::PARTS == 2) {
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
#pragma unroll
                        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(x[j][e]));
                    top = fmaxf(top, __shfl_xor(top, TR, WAVE));
                    scaling(top, up, down);
                }
                scale *= down;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        uint32_t part[PARTS];
                        if constexpr (PARTS > 1) query_parts<LT>(x[j][e] * up, x[j][e + 1] * up, part);
                        else probability_parts<LT, 1>(x[j][e] * up, x[j][e + 1] * up, part);
#pragma unroll
                        for (int q = 0; q < PARTS; ++q) Q[j][q][e / 2] = part[q];
                    }
            }
        }
    }
    wait_loads();                                            // (queries are waited for here: else the products of every stage would wait for whatever has been asked for since)
    f32x16 o[NF];
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[f][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    int o_exp = -200, scales_now = -400;                     // Q8: the power of two that the row's O is held by; what it went by
    __syncthreads();                                         // (the stages' marks)
    fetch(0);
    drop = drop_next;
    if (stages > 1) ask(1);
    if constexpr (Q8) put(0);

    for (int t = 0; t < stages; ++t) {
        const int stage0 = lo + t * SK;
        char *const k_tile = lds + (t % 2) * BYTES, *const v_tile = k_tile + HALF;
        if constexpr (!Q8) {
            wait_loads();
            // Values that do not count are zero; one that some rows see and others do not must not be what zero times it is not zero.
            if (drop) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    if ((drop >> i) & 1) *(u32x4 *)(v_tile + place(i)) = u32x4{0, 0, 0, 0};
            }
            if (stage0 + SK - 1 > pos_min) {
                bool odd = false;
#pragma unroll
                for (int i = 0; i < LOADS; ++i) odd = odd || (of_share() && not_finite<sizeof(LT)>(*(const u32x4 *)(v_tile + place(i)), Type<LT>::PARTS == 3));
                if (odd) odd_stage[t % 2] = t + 1;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (t + 1 < stages) {
            fetch(t + 1);
            if (t + 2 < stages) ask(t + 2);
        }
        const bool any_bad = bad_stage[t % 2] == t + 1;
        const int tb = stage0 + kw * (TR * NU), key_base = kw * (TR * NU);
        if (!Q8 && odd_stage[t % 2] == t + 1) {              // seldom: rows that see such a value get no number at its feature, and it counts as zero from here on
            if (active)
                for (int key = key_base; key < key_base + TR * NU; ++key) {
                    const bool seen = stage0 + key <= pos;
                    int half = h;
                    asm volatile("" : "+v"(half));           // (or all these places would be formed ahead of the stages, and kept)
#pragma unroll
                    for (int f = 0; f < NF; ++f)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int feature = share * (DH / 2) + TR * f + 8 * (i / 4) + 4 * half + i % 4;
                            const char *at = v_tile + key * ROWB + 16 * v_place<PIECES, F32>(key, feature / PIECE_EL) + feature % PIECE_EL * (int)sizeof(LT);
                            bool odd;
                            if constexpr (F32) odd = (*(const uint32_t *)at & 0x7F800000u) == 0x7F800000u;
                            else {
                                const uint32_t e = Type<LT>::PARTS == 3 ? 0x7F80u : 0x7C00u;
                                odd = (*(const uint16_t *)at & e) == e;
                            }
                            if (odd && seen) o[f][i] = NAN;
                        }
                }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                u32x4 *at = (u32x4 *)(v_tile + place(i));
                u32x4 x = *at;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (F32) x[e] = (x[e] & 0x7F800000u) == 0x7F800000u ? 0 : x[e];
                    else {
                        const uint32_t ex = Type<LT>::PARTS == 3 ? 0x7F80u : 0x7C00u;
                        if ((x[e] & ex) == ex) x[e] &= 0xFFFF0000u;
                        if (((x[e] >> 16) & ex) == ex) x[e] &= 0xFFFFu;
                    }
                }
                *at = x;
            }
            __syncthreads();
        }
        if (Q8 && odd_stage[t % 2] == t + 1) {
            bool seen = false;
            for (u64 left = odd_keys[t % 2]; left; left &= left - 1) seen = seen || stage0 + __builtin_ctzll(left) <= pos;
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[f][i] = seen ? NAN : o[f][i];
        }
        if (active && tb <= wave_hi) {
            f32x16 st[NU];
            // pieces of keys are asked for KD ahead of their products
            constexpr int KD = NJ < 4 ? NJ : Q8 && PARTS == 2 && RW == 4 ? 1 : DH == 256 && (F32 || PARTS == 3) ? 2 : LEAN ? 4 : NJ < 8 ? NJ : 8, STEPS = NU * NJ;
            int k_off = 16 * k_place<PIECES>(key_base + col, h);             // (piece 2 j + h lies where piece h does, but for the bits of 2 j)
            if constexpr (LEAN) asm volatile("" : "+v"(k_off));              // (formed from here on in every stage: kept, the places of all pieces are a register each)
            const char *k_row = k_tile + (key_base + col) * ROWB;
            const auto key_piece = [&](int i) { return *(const u32x4 *)(k_row + TR * (i / NJ) * ROWB + (k_off ^ 32 * (i % NJ))); };
            u32x4 k[KD];
#pragma unroll
            for (int i = 0; i < KD; ++i) k[i] = key_piece(i);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int u = i / NJ, j = i % NJ;
                if (j == 0)
#pragma unroll
                    for (int e = 0; e < 16; ++e) st[u][e] = 0.f;
                if constexpr (F32) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) st[u] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(k[i % KD][c]), __uint_as_float(Q[j][0][c]), st[u], 0, 0, 0);
                } else {
#pragma unroll
                    for (int q = PARTS - 1; q >= 0; --q) st[u] = mfma32<LT>(k[i % KD], Q[j][q], st[u]);
                }
                if (i + KD < STEPS) k[i % KD] = key_piece(i + KD);
            }
            if constexpr (DH >= 64) {                        // in this order: reads from LDS (0x100), products (0x8)
                constexpr int EACH = F32 ? 4 : PARTS;
                __builtin_amdgcn_sched_group_barrier(0x100, KD, 0);
#pragma unroll
                for (int i = 0; i < STEPS - KD; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x8, EACH, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x8, KD * EACH, 0);
            }
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                if constexpr (Q8) {
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const float4 s = *(const float4 *)&k_sc[t % 2][key_base + TR * u + 2 * i + 4 * h];
                        st[u][i] *= s.x; st[u][i + 1] *= s.y; st[u][i + 2] *= s.z; st[u][i + 3] *= s.w;
                    }
                }
            }
            const bool masked = tb + TR * NU - 1 > wave_lo || any_bad;
            if (masked) {                                    // keys behind a row's own position, or on no page: no score
#pragma unroll
                for (int u = 0; u < NU; ++u)
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const int at = tb + TR * u + 2 * i + 4 * h;          // (four keys lie on one page)
                        const bool ok = !any_bad || (unsigned)as_global(entries)[min(at, hi - 1) >> shift] < (unsigned)p.c.n_pages;
#pragma unroll
                        for (int e = 0; e < 4; ++e) st[u][i + e] = ok && at + e <= pos ? st[u][i + e] : -INFINITY;
                    }
            }
            // The reference is raised where a probability would pass 2^SLACK; only that row's, so that a row's result hangs on nothing but itself.
            float mx = -INFINITY;
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) mx = fmaxf(mx, st[u][i]);
            mx *= scale;
            if (__any((mx > m + SLACK) | (fabsf(m) > FAR))) {
                mx = fmaxf(mx, __shfl_xor(mx, TR, WAVE));    // the lane's halves hold different keys of the same rows
                mx = mx > m + SLACK ? mx : m;
                const float corr = exp2_below(m, mx);
                m = mx;
                l *= corr;
#pragma unroll
                for (int f = 0; f < NF; ++f)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[f][i] *= corr;
                if (__any((fabsf(m) > FAR) & (m != -INFINITY))) {        // far from zero, an exponent is formed from the rounded score
                    const float inv = __builtin_amdgcn_rcpf(scale);
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int i = 0; i < 16; ++i) st[u][i] = fabsf(m) > FAR && m != -INFINITY ? ((st[u][i] * scale - m) + T::P_BITS) * inv : st[u][i];
                }
            }
            float ref = fabsf(m) > FAR ? 0.f : m - T::P_BITS;            // (-inf, nothing seen yet: no score either)
            const int scales = Q8 ? __builtin_amdgcn_readfirstlane(v_exp[t % 2]) : 0;
            int lift = 0;                                    // Q8: probabilities are 2^lift times what they are elsewhere
            if (Q8 && (scales != scales_now || (scales & 1))) {
                const int ex = scales >> 1;
                scales_now = scales;
                if (scales & 1) {
                    // Next to the largest scale, which the row may not see, or hardly weigh, those that count for it may leave nothing of a probability in 16 bits: rows go by the largest product of both in the stage.
                    float most = -INFINITY;
#pragma unroll
                    for (int u = 0; u < NU; ++u)
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float4 s = *(const float4 *)&v_sc[t % 2][key_base + TR * u + 2 * i + 4 * h];
#pragma unroll
                            for (int e = 0; e < 4; ++e) most = fmaxf(most, fmaf(st[u][i + e], scale, -ref) + __builtin_amdgcn_logf(fabsf(e == 0 ? s.x : e == 1 ? s.y : e == 2 ? s.z : s.w)));
                        }
                    most = fmaxf(most, __shfl_xor(most, TR, WAVE));
                    lift = most > -INFINITY ? 14 - (int)ceilf(fminf(fmaxf(most, -100.f), 100.f)) : ex - o_exp;     // (nothing: as it was)
                    lift = min(max(lift, 0), LIFT_MAX);
                    ref -= (float)lift;
                    l = ldexpf(l, lift);
                }
                if (__any(ex - lift != o_exp)) {
                    const float f0 = ldexpf(1.f, o_exp - (ex - lift));
                    o_exp = ex - lift;
#pragma unroll
                    for (int f = 0; f < NF; ++f)
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[f][i] *= f0;
                }
            }
            // pieces of values are asked for VD ahead of their products
            constexpr int VD = NF < 4 ? NF : Q8 && PARTS == 2 && RW == 4 ? 2 : 4, VALUES = NU * 2 * NF;
            int at4 = lane % 16;
            if constexpr (LEAN) asm volatile("" : "+v"(at4));
            const int t4 = at4 / 4, fg = (lane / 16) % 2;
            const auto value_piece = [&](int i) {            // 16 keys, i / NF, by 32 features, i % NF
                const int f = i % NF, key = key_base + 16 * (i / NF) + 4 * h + t4;
                const char *at = v_tile + key * ROWB + 16 * v_place<PIECES, F32>(t4, 4 * f + 2 * fg + (lane % 4) / 2) + 8 * (lane % 2) + share * (ROWB / 2);     // (a place hangs on key % 4 alone)
                const u32x2 x = turned_read(at), y = turned_read(at + 8 * ROWB);
                return u32x4{x.x, x.y, y.x, y.y};
            };
            u32x4 v[VD];
            if constexpr (!F32) {
#pragma unroll
                for (int i = 0; i < VD; ++i) v[i] = value_piece(i);
            }
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                if constexpr (F32) {
                    float pf[16];
                    int half = h;
                    if constexpr (LEAN) asm volatile("" : "+v"(half));
                    const char *v_row = v_tile + (key_base + 4 * half) * ROWB;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        pf[i] = __builtin_amdgcn_exp2f(fmaf(st[u][i], scale, -ref)) * T::P_SCALE;
                        l += pf[i];
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
#pragma unroll
                        for (int f = 0; f < NF; ++f) {
                            const float v = *(const float *)(v_row + (TR * u + 8 * (i / 4) + i % 4) * ROWB + 16 * v_place<PIECES, F32>(4 * half, 8 * f) + 4 * col + share * (ROWB / 2));
                            o[f] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, pf[i], o[f], 0, 0, 0);
                        }
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < 2; ++g) {            // 16 keys at a time
                        u32x4 pt[PARTS];
#pragma unroll
                        for (int i = 8 * g; i < 8 * g + 8; i += 4) {
                            float pf[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                pf[e] = __builtin_amdgcn_exp2f(fmaf(st[u][i + e], scale, -ref));
                                if (T::P_SCALE != 1.f) pf[e] *= T::P_SCALE;
                            }
                            if constexpr (PARTS > 1 || Q8) l += (pf[0] + pf[1]) + (pf[2] + pf[3]);
                            if constexpr (Q8) {
                                const float4 s = *(const float4 *)&v_sc[t % 2][key_base + TR * u + 2 * i + 4 * h];
                                pf[0] *= s.x; pf[1] *= s.y; pf[2] *= s.z; pf[3] *= s.w;
                            }
#pragma unroll
                            for (int e = 0; e < 4; e += 2) {
                                uint32_t part[PARTS];
                                probability_parts<LT, PARTS>(pf[e], pf[e + 1], part);
                                if constexpr (PARTS == 1 && !Q8) l = pair_sum<LT>(part[0], l);       // (of what they weigh, one instruction for two)
#pragma unroll
                                for (int q = 0; q < PARTS; ++q) pt[q][(i % 8) / 2 + e / 2] = part[q];
                            }
                        }
#pragma unroll
                        for (int f = 0; f < NF; ++f) {
                            const int i = (2 * u + g) * NF + f;
#pragma unroll
                            for (int q = PARTS - 1; q >= 0; --q) o[f] = mfma32<LT>(v[i % VD], pt[q], o[f]);
                            if (i + VD < VALUES) v[i % VD] = value_piece(i + VD);
                        }
                    }
                }
            }
            if constexpr (!F32 && DH >= 64) {                // (as above; Q8: and two reads of scales for every 16 keys)
                constexpr int SCALES = Q8 ? 2 : 0;
                __builtin_amdgcn_sched_group_barrier(0x100, 2 * VD + SCALES, 0);
#pragma unroll
                for (int i = 0; i < VALUES; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x8, PARTS, 0);
                    if (i % NF == 0 && i + NF < VALUES) __builtin_amdgcn_sched_group_barrier(0x100, 2 + SCALES, 0);
                    else if (i + VD < VALUES) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
                }
            }
            if (Q8 && (scales & 1)) l = ldexpf(l, -lift);
        }
        if constexpr (Q8)
            if (t + 1 < stages) put(t + 1);
        drop = drop_next;
    }
    l += __shfl_xor(l, TR, WAVE);
    if constexpr (KW > 1) {                                  // two waves have shared out the keys of the same rows
        __syncthreads();
        float *O = (float *)lds + rw * (NF * 16) * WAVE + lane;
        if (kw == 1) {
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int i = 0; i < 16; ++i) O[(f * 16 + i) * WAVE] = o[f][i];
            join_m[rw][lane] = m;
            join_l[rw][lane] = l;
            if (Q8) join_e[rw][lane] = o_exp;
        }
        __syncthreads();
        if (kw == 1) return;
        const float m1 = join_m[rw][lane], M = fmaxf(m, m1);
        float f0 = exp2_below(m, M), f1 = exp2_below(m1, M);
        l = l * f0 + join_l[rw][lane] * f1;
        if constexpr (Q8) {                                  // (a wave with no key to see in the last stages has not followed their scales)
            const int ex1 = join_e[rw][lane], ex = max(o_exp, ex1);
            f0 = ldexpf(f0, o_exp - ex);
            f1 = ldexpf(f1, ex1 - ex);
            o_exp = ex;
        }
        m = M;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[f][i] = o[f][i] * f0 + O[(f * 16 + i) * WAVE] * f1;
    }
    if (!active || rw * TR + col >= n_rows) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;              // (nothing seen: zeros)
    const size_t at = p.splits > 1 ? row_at * p.splits + split : row_at;
    if (p.splits > 1 && h == 0 && share == 0) {
        as_global(p.part_ml)[2 * at] = m;
        as_global(p.part_ml)[2 * at + 1] = l;
    }
#pragma unroll
    for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int feature = share * (DH / 2) + TR * f + 2 * i + 4 * h;
            if (DH == 32 && feature >= d) continue;
            float4 y = make_float4(o[f][i] * inv, o[f][i + 1] * inv, o[f][i + 2] * inv, o[f][i + 3] * inv);
            if constexpr (Q8) y = make_float4(ldexpf(y.x, o_exp), ldexpf(y.y, o_exp), ldexpf(y.z, o_exp), ldexpf(y.w, o_exp));
            if (p.splits > 1) store_rows<float>(p.part, at * d + feature, y);
            else store_rows<IO>(p.out, at * d + feature, y);
        }
}

// A wave puts MR rows' chunks together: d_head / 4 lanes a chunk, chunks side by side, sums in a fixed order.  What it needs of the lengths, references and sums and its first chunks is one
// trip to memory (chunks that a row does not reach hold anything, and are not looked at).
// Measured, rows of 128: 22656 with two chunks each 9.3 us with two rows per wave (with one row, and a trip for each of the three, 11.0); 2560 with eight 4.6 with one.
constexpr int SPLITS_MAX = WAVE;
template <typename IO, int MR>
__global__ __launch_bounds__(NT) void paged_merge_kernel(const PagedAttnArgs p) {
    const int lane = threadIdx.x & (WAVE - 1), d = p.c.d_head, per = d / 4, side = WAVE / per, mine = lane / per, rows = p.n_tokens * p.n_heads;
    const int row0 = (blockIdx.x * NW + threadIdx.x / WAVE) * MR;
    if (row0 >= rows) return;
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 ml[MR];
    float4 x[MR];
#pragma unroll
    for (int r = 0; r < MR; ++r) {
        const size_t at = (size_t)min(row0 + r, rows - 1) * p.splits;
        ml[r] = ((global_ptr<const f32x2>)p.part_ml)[at + min(lane, p.splits - 1)];
        x[r] = global_load_float4(p.part + (at + min(mine, p.splits - 1)) * d + 4 * (lane % per));
    }
    int t[MR], s[MR];
#pragma unroll
    for (int r = 0; r < MR; ++r) { t[r] = over(min(row0 + r, rows - 1), p.by_heads); s[r] = 0; }
    bool bad = false;
    for (int i0 = 0; i0 < p.c.n_seq; i0 += WAVE) {
        const int i = min(i0 + lane, p.c.n_seq - 1), a = as_global(p.first)[i], b = as_global(p.first)[i + 1];
        bad = bad || b < a;
#pragma unroll
        for (int r = 0; r < MR; ++r) s[r] += __popcll(__ballot(i0 + lane < p.c.n_seq && b <= t[r]));
    }
    if (__any(bad)) return;
#pragma unroll
    for (int r = 0; r < MR; ++r) {
        if (row0 + r >= rows || s[r] >= p.c.n_seq) continue;
        const int a = as_global(p.first)[s[r]], b = as_global(p.first)[s[r] + 1], len = as_global(p.len)[s[r]], n = b - a;
        if (t[r] < a || !fits(p, a, b, len)) continue;           // (not theirs, or zeros already)
        const int chunks = over(len - n + t[r] - a, p.by_chunk) + 1;
        const float m = lane < chunks ? ml[r][0] : -INFINITY;
        const float M = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_max_last(m)), WAVE - 1));
        float l = lane < chunks ? ml[r][1] * exp2_below(m, M) : 0.f;
        const float L = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wave_sum_last(l)), WAVE - 1));
        l = L == 0.f ? 0.f : l / L;              // a chunk's share
        const size_t at = (size_t)(row0 + r) * p.splits;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int c0 = 0; c0 < chunks; c0 += side) {
            const int c = c0 + mine;
            const float f = __shfl(l, min(c, WAVE - 1), WAVE);
            if (c >= chunks) continue;           // (one that weighs nothing counts: what is no number in it stays none)
            const float4 z = c0 ? global_load_float4(p.part + (at + c) * d + 4 * (lane % per)) : x[r];
            y.x += f * z.x; y.y += f * z.y; y.z += f * z.z; y.w += f * z.w;
        }
        for (int o = per; o < WAVE; o <<= 1) {
            y.x += __shfl_xor(y.x, o, WAVE); y.y += __shfl_xor(y.y, o, WAVE); y.z += __shfl_xor(y.z, o, WAVE); y.w += __shfl_xor(y.w, o, WAVE);
        }
        if (lane < per) store_rows<IO>(p.out, (size_t)(row0 + r) * d + 4 * lane, y);
    }
}

// How a call is cut.  Tiles of 128 rows use a key twice as often as those of 64, whose waves halve the keys of a stage instead: that pays where the rows of a sequence fill no more than one.  Chunks
// of positions where there are fewer tiles than places for blocks, as many as fill these (two per compute unit where the second gains more than it costs), none of under 256 positions.  Measured before the last steps, which left the order as it is, us (rows of a tile, chunks; the rule's own first):
//   2999 tokens of prompts, bf16:                 128: 51.4 | 64: 67.3
//   708 tokens behind 2003 positions, 8 bits:     128, 2: 76.6 | 1: 96.0 | 3: 85.4 | 64, 1: 77.0
//   40 tokens behind 4001 positions, 8 bits:      64, 8: 35.7 | 4: 46.0 | 6: 42.6 | 11: 42.0 | 16: 43.6 | 128, 8: 42.0
//   261 tokens behind 500 positions, fp32:        128, 2: 61 | 1: 98 | 3: 84 | 4: 69 | 64, 1: 65.7
//   four tokens behind 73 positions, fp16:        64, 1: 10.4 | 2: 14.2
struct Cut { int rows, splits, chunk; };
constexpr int CUS = 256, CHUNK_MIN = 256, SEQS_MAX = 1 << 16;        // (every block looks through the sequences)
Cut cut_for(int dtype, int io_dtype, int n_seq, int n_tokens, int n_heads, int n_kv_heads, int d_head, int max_new, int max_len) {
    const long long group = n_heads / n_kv_heads;
    Cut c;
    c.rows = std::max(1, max_new) * group <= 64 && !(dtype == SPD_DTYPE_FP32 && d_head == 256) ? 64 : 128;
    const long long blocks = std::max<long long>(n_seq, (n_tokens * group + c.rows - 1) / c.rows) * n_kv_heads;
    const int positions = std::max(1, max_len);
    const bool two = d_head <= 128 && dtype != SPD_DTYPE_FP32 && !(dtype == SPD_DTYPE_BF16 && io_dtype == SPD_DTYPE_FP32);     // blocks that share a compute unit gain by it
    long long n = std::min<long long>(std::max<long long>(1, (two ? 2 : 1) * CUS / blocks), (positions + CHUNK_MIN - 1) / CHUNK_MIN);
    n = std::min<long long>(n, SPLITS_MAX);
    c.chunk = (int)(((positions + n - 1) / n + 63) / 64 * 64);
    c.splits = (positions + c.chunk - 1) / c.chunk;
    return c;
}

template <typename KT, typename IO, int DH, int RW>
hipError_t launch_rows(hipStream_t s, PagedAttnArgs a) {
    typedef Shape<KT, IO, DH, RW> S;
    a.n_tiles = (int)((long long)a.n_tokens * a.group / S::ROWS + a.c.n_seq);
    const long long blocks = (long long)a.n_tiles * a.c.n_kv_heads * a.splits * S::FS;
    if (S::LDS > 60 * 1024) {
        const hipError_t e = hipFuncSetAttribute((const void *)paged_attn_kernel<KT, IO, DH, RW>, hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((paged_attn_kernel<KT, IO, DH, RW>), dim3((unsigned)blocks), dim3(NT), S::LDS, s, a);
    const int all_rows = a.n_tokens * a.n_heads;
    if (a.splits > 1 && all_rows <= 8192) hipLaunchKernelGGL((paged_merge_kernel<IO, 1>), dim3((unsigned)((all_rows + NW - 1) / NW)), dim3(NT), 0, s, a);      // (fewer than the GPU holds)
    else if (a.splits > 1) hipLaunchKernelGGL((paged_merge_kernel<IO, 2>), dim3((unsigned)((all_rows + 2 * NW - 1) / (2 * NW))), dim3(NT), 0, s, a);
    return hipGetLastError();
}

template <typename KT, typename IO>
hipError_t launch(hipStream_t s, const PagedAttnArgs &a, int rows) {
    const int d = a.c.d_head;
    if (rows == 64) {
        if (d <= 32) return launch_rows<KT, IO, 32, 2>(s, a);
        if (d == 64) return launch_rows<KT, IO, 64, 2>(s, a);
        if (d == 128) return launch_rows<KT, IO, 128, 2>(s, a);
        if constexpr (sizeof(KT) != 4) return launch_rows<KT, IO, 256, 2>(s, a);
    }
    if (d <= 32) return launch_rows<KT, IO, 32, 4>(s, a);
    if (d == 64) return launch_rows<KT, IO, 64, 4>(s, a);
    if (d == 128) return launch_rows<KT, IO, 128, 4>(s, a);
    return launch_rows<KT, IO, 256, 4>(s, a);
}

bool io_fits(int dtype, int io) {
    if (io == SPD_DTYPE_FP32) return dtype >= SPD_DTYPE_FP32 && dtype <= SPD_DTYPE_INT8;
    return dtype == SPD_DTYPE_INT8 ? io == SPD_DTYPE_FP16 || io == SPD_DTYPE_BF16 : dtype == io && io != SPD_DTYPE_INT8;
}

}  // namespace

extern "C" size_t spd_op_attention_paged_scratch_bytes(int32_t dtype, int32_t io_dtype, int32_t n_seq, int32_t n_tokens, int32_t n_heads, int32_t n_kv_heads, int32_t d_head,
                                                       int32_t max_new, int32_t max_len) {
    if (!io_fits(dtype, io_dtype) || n_seq <= 0 || n_tokens <= 0 || n_heads <= 0 || n_kv_heads <= 0 || n_heads % n_kv_heads || d_head <= 0 || max_new < 0 || max_len < 0) return 0;
    const Cut c = cut_for(dtype, io_dtype, n_seq, n_tokens, n_heads, n_kv_heads, d_head, max_new, max_len);
    const size_t parts = (size_t)n_tokens * n_heads * c.splits;
    return c.splits > 1 ? up256(parts * 8) + up256(parts * d_head * 4) : 0;
}

extern "C" int spd_op_attention_paged(int32_t dtype, int32_t io_dtype, const void *q, int64_t q_stride, const void *K, const void *V, const float *K_scale, const float *V_scale,
                                      const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size, int32_t d_head, int32_t n_seq, int32_t table_stride, const int32_t *first,
                                      const int32_t *len, int32_t n_tokens, int32_t n_heads, int32_t max_new, int32_t max_len, void *out, void *scratch, size_t scratch_bytes,
                                      int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache((void *)K, (void *)V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    const int rc = spdk::paged_cache_status(dtype, c, page_size, K_scale, V_scale);
    if (rc != SPD_OK) return rc;
    if (!io_fits(dtype, io_dtype) || n_tokens < 0 || n_heads < 1 || n_heads % n_kv_heads || max_new < 0 || max_len < 0 || max_len > (long long)table_stride * page_size || max_len > INT32_MAX / 2 ||
        (long long)n_pages * n_kv_heads > INT32_MAX) return SPD_EINVAL;
    if (n_tokens == 0 || n_seq == 0) return SPD_OK;
    if ((long long)n_tokens * n_heads > (1 << 24) || n_seq > SEQS_MAX) return SPD_EINVAL;
    const int io_bytes = io_dtype == SPD_DTYPE_FP32 ? 4 : 2;
    if (!q || !first || !len || !out || ((uintptr_t)q | (uintptr_t)out) % 16 || q_stride < (int64_t)n_heads * d_head || q_stride % 8) return SPD_EINVAL;
    const size_t need = spd_op_attention_paged_scratch_bytes(dtype, io_dtype, n_seq, n_tokens, n_heads, n_kv_heads, d_head, max_new, max_len);
    if (need && (!scratch || (uintptr_t)scratch % 256)) return SPD_EINVAL;
    if (scratch_bytes < need) return SPD_EWORKSPACE;
    const size_t rows = (size_t)n_tokens * n_heads * d_head * io_bytes, q_bytes = ((size_t)(n_tokens - 1) * q_stride + (size_t)n_heads * d_head) * io_bytes, pool = spdk::pool_bytes(dtype, c),
                 scales = spdk::scale_bytes(c);
    const spdk::Span sq{q, q_bytes}, so{out, rows}, sK{K, pool}, sV{V, pool}, sk{K_scale, scales}, sv{V_scale, scales}, st{table, (size_t)n_seq * table_stride * 4},
        sf{first, (size_t)(n_seq + 1) * 4}, sl{len, (size_t)n_seq * 4}, se{err, 4}, sw{scratch, need};
    if (spdk::over_any(so, {sq, sK, sV, sk, sv, st, sf, sl, se, sw}) || spdk::over_any(sw, {sq, sK, sV, sk, sv, st, sf, sl, se})) return SPD_EINVAL;
    const Cut cut = cut_for(dtype, io_dtype, n_seq, n_tokens, n_heads, n_kv_heads, d_head, max_new, max_len);
    const int group = n_heads / n_kv_heads;
    if (((long long)n_tokens * group / cut.rows + n_seq) * n_kv_heads * cut.splits * 2 > UINT32_MAX / NT) return SPD_EINVAL;       // (threads of a grid are counted in 32 bits)
    PagedAttnArgs a{c, K_scale, V_scale, q, q_stride, out, first, len, err, n_tokens, n_heads, group, max_len, 0, cut.splits, cut.chunk, divisor(group), divisor(n_kv_heads), divisor(cut.splits), divisor(n_heads), divisor(cut.chunk),
                    (float *)scratch, (float *)((char *)scratch + up256((size_t)n_tokens * n_heads * cut.splits * 8))};
    hipStream_t s = (hipStream_t)hip_stream;
    hipError_t e;
    if (dtype == SPD_DTYPE_FP32) e = launch<float, float>(s, a, cut.rows);
    else if (dtype == SPD_DTYPE_FP16) e = io_dtype == SPD_DTYPE_FP32 ? launch<half_t, float>(s, a, cut.rows) : launch<half_t, half_t>(s, a, cut.rows);
    else if (dtype == SPD_DTYPE_BF16) e = io_dtype == SPD_DTYPE_FP32 ? launch<bf16_t, float>(s, a, cut.rows) : launch<bf16_t, bf16_t>(s, a, cut.rows);
    else e = io_dtype == SPD_DTYPE_FP32 ? launch<q8_t, float>(s, a, cut.rows) : io_dtype == SPD_DTYPE_FP16 ? launch<q8_t, half_t>(s, a, cut.rows) : launch<q8_t, bf16_t>(s, a, cut.rows);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}
