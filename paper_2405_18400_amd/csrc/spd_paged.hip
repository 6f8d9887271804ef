// The paged key/value cache of a batch of sequences: appending new tokens (with the rotary
// positions applied on the way) and following a selection of beams.
//
// Both are bound by memory traffic where there is much to move and by latency where there is
// little.  What they need besides the data itself -- page numbers, angles, which row a beam goes
// on in -- is formed again by every block that uses it: it is a few dozen instructions, and a
// kernel of its own would cost a launch.
#include "spd_attention.h"

#include <algorithm>

using namespace spdd;
using namespace spda;

namespace {

constexpr int NTP = 256;             // threads per block
constexpr int COPIES = 8;            // 16-byte pieces under way per thread when pages are copied

__device__ __forceinline__ bool page_ok(const PagedCache &c, int page) { return (unsigned)page < (unsigned)c.n_pages; }
__device__ __forceinline__ void flag(int32_t *err) { if (err) *as_global(err) = 1; }

// Four elements, as the cache stores them.
template <typename KT> __device__ __forceinline__ void store_four(void *p, size_t i, const float4 v);
template <> __device__ __forceinline__ void store_four<float>(void *p, size_t i, const float4 v) {
    *(f32x4 __attribute__((address_space(1))) *)((float *)p + i) = f32x4{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ void store_words(void *p, size_t i, uint32_t a, uint32_t b) {
    *(u32x2 __attribute__((address_space(1))) *)((uint16_t *)p + i) = u32x2{a, b};
}
template <> __device__ __forceinline__ void store_four<half_t>(void *p, size_t i, const float4 v) {
    store_words(p, i, Store<half_t>::bits(v.x) | (uint32_t)Store<half_t>::bits(v.y) << 16, Store<half_t>::bits(v.z) | (uint32_t)Store<half_t>::bits(v.w) << 16);
}
// Round to nearest even; a NaN stays one (its payload could otherwise round up to an infinity).
__device__ __forceinline__ uint32_t bf16_of(float v) {
    const uint32_t u = __float_as_uint(v);
    return v != v ? (u >> 16) | 0x40u : (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}
template <> __device__ __forceinline__ void store_four<bf16_t>(void *p, size_t i, const float4 v) {
    store_words(p, i, bf16_of(v.x) | bf16_of(v.y) << 16, bf16_of(v.z) | bf16_of(v.w) << 16);
}

template <typename OT> __device__ __forceinline__ uint32_t two_words(float x, float y) {
    if constexpr (sizeof(OT) == 2 && Type<OT>::PARTS == 2) return Store<half_t>::bits(x) | (uint32_t)Store<half_t>::bits(y) << 16;
    else return bf16_of(x) | bf16_of(y) << 16;
}

// cos and sin of pos * theta^(-2i / d_head).  The angle is formed and reduced to a quarter turn in 64 bits (at position
// 100000 fp32 leaves 0.004 of it), the functions of what remains are fp32: off by 2^-24.
__device__ __forceinline__ float2 rotation(int pos, int i, double log2_theta, int d_head) {
    const double angle = (double)pos * exp2(-2.0 * i / d_head * log2_theta);
    const double quarters = rint(angle * 0.63661977236758134308);                    // 2 / pi
    double r = fma(-quarters, 1.57079632679489655800, angle);                        // pi / 2 in two parts
    r = fma(-quarters, 6.12323399573676603587e-17, r);
    float s, c;
    sincosf((float)r, &s, &c);
    const int q = (int)((long long)quarters & 3);
    const float cs = (q & 1) ? s : c, sn = (q & 1) ? c : s;
    return make_float2(q == 1 || q == 2 ? -cs : cs, q >= 2 ? -sn : sn);
}

// Measured: four tokens of 32 + 2 x 32 heads of 128 3.3 us (latency); 4099 tokens of 64 + 2 x 8 heads, 319 MB in all, 61 us, 5.2 TB/s
// (a large copy: 4.8).
// One block: part `part` of one token's pieces of four elements, q heads first, then k, then v.  U pieces per thread are
// asked for before the position, the page and the angles are known.
template <typename KT, int U>
__global__ __launch_bounds__(NTP) void append_paged_kernel(const AppendArgs a) {
    __shared__ float2 turn[128];
    const int tid = threadIdx.x, t = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int d = a.c.d_head, per_head = d / 4;
    const int q_end = a.n_heads * per_head, k_end = q_end + a.c.n_kv_heads * per_head, end = k_end + a.c.n_kv_heads * per_head;
    const int seq = as_global(a.seq)[t], pos = as_global(a.pos)[t];
    if (seq < 0) return;                                                              // padding
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int p = (part * U + u) * NTP + tid;
        if (p < q_end) x[u] = global_load_float4(a.q + (size_t)t * a.q_stride + 4 * p);
        else if (p < k_end) x[u] = global_load_float4(a.k + (size_t)t * a.kv_stride + 4 * (p - q_end));
        else if (p < end) x[u] = global_load_float4(a.v + (size_t)t * a.kv_stride + 4 * (p - k_end));
    }
    if (seq >= a.c.n_seq || pos < 0 || (pos >> a.c.page_shift) >= a.c.table_stride) {
        if (tid == 0) flag(a.err);
        return;
    }
    const int page = as_global(a.c.table)[(size_t)seq * a.c.table_stride + (pos >> a.c.page_shift)];
    if (tid < d / 2) turn[tid] = rotation(pos, tid, a.log2_theta, d);
    __syncthreads();
    if (!page_ok(a.c, page)) {
        if (tid == 0) flag(a.err);
        return;
    }
    const int page_size = 1 << a.c.page_shift, row = pos & (page_size - 1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int p = (part * U + u) * NTP + tid;
        if (p >= end) break;
        float4 y = x[u];
        if (p < k_end) {
            const float2 c0 = turn[2 * (p % per_head)], c1 = turn[2 * (p % per_head) + 1];
            y.x = x[u].x * c0.x - x[u].y * c0.y;
            y.y = x[u].x * c0.y + x[u].y * c0.x;
            y.z = x[u].z * c1.x - x[u].w * c1.y;
            y.w = x[u].z * c1.y + x[u].w * c1.x;
        }
        if (p < q_end) {
            store_four<float>(a.q_out, (size_t)t * q_end * 4 + 4 * p, y);
        } else {
            const int at = p < k_end ? p - q_end : p - k_end, head = at / per_head;
            store_four<KT>(p < k_end ? a.c.K : a.c.V, (((size_t)page * a.c.n_kv_heads + head) * page_size + row) * d + 4 * (at % per_head), y);
        }
    }
}

// few tokens: one piece per thread, so that many blocks share the way to memory; many: four, so that angles and page
// numbers are formed for more of them
long long append_blocks(AppendArgs &a, bool &few) {
    const long long pieces = (long long)(a.n_heads + 2 * a.c.n_kv_heads) * (a.c.d_head / 4);
    few = pieces * a.n_tokens < 4LL * NTP * 1024;
    const int u = few ? 1 : 4;
    a.parts = (int)((pieces + u * NTP - 1) / (u * NTP));
    return (long long)a.n_tokens * a.parts;
}

template <typename KT>
hipError_t launch_append(hipStream_t s, AppendArgs a) {
    bool few;
    const long long blocks = append_blocks(a, few);
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    if (few) hipLaunchKernelGGL((append_paged_kernel<KT, 1>), dim3((unsigned)blocks), dim3(NTP), 0, s, a);
    else hipLaunchKernelGGL((append_paged_kernel<KT, 4>), dim3((unsigned)blocks), dim3(NTP), 0, s, a);
    return hipGetLastError();
}

// ---- eight bits per value ----

struct q8_t { int8_t b; };

// cos and sin of pos * theta^(-2i / d_head) in 64 bits: a key's place between two codes hangs on them.  2i / d_head is exact, so the logarithm's two parts times it
// are off by 2^-106 of it, and the frequency by the last place of exp2.  The angle is reduced to a quarter turn as in rotation(); the rest of at most
// pi / 4 goes through the Taylor series, whose first terms left out are below 2^-57.
__device__ __forceinline__ double2 rotation64(int pos, int i, double log2_theta, double log2_theta_low, int d_head) {
    const double part = -2.0 * i / d_head, y = part * log2_theta, low = fma(part, log2_theta, -y) + part * log2_theta_low;
    const double f = exp2(y), angle = (double)pos * fma(f, 0.69314718055994530942 * low, f);
    const double quarters = rint(angle * 0.63661977236758134308);                    // 2 / pi
    double r = fma(-quarters, 1.57079632679489655800, angle);                        // pi / 2 in two parts
    r = fma(-quarters, 6.12323399573676603587e-17, r);
    const double z = r * r;
    double s = 1.0, c = 1.0;
#pragma unroll
    for (int k = 8; k >= 1; --k) {                                                   // x - x^3/3! + .. + x^17/17!, 1 - x^2/2! + .. + x^16/16!
        s = fma(s, -z * (1.0 / (2.0 * k * (2.0 * k + 1.0))), 1.0);
        c = fma(c, -z * (1.0 / (2.0 * k * (2.0 * k - 1.0))), 1.0);
    }
    s *= r;
    const int q = (int)((long long)quarters & 3);
    const double cs = (q & 1) ? s : c, sn = (q & 1) ? c : s;
    return make_double2(q == 1 || q == 2 ? -cs : cs, q >= 2 ? -sn : sn);
}

__device__ __forceinline__ float finite(float x) { return x != x ? 0.f : fminf(fmaxf(x, -3.402823466e38f), 3.402823466e38f); }

// The code of x: x / scale, whose rounding to 64 bits is the nearest (a product with the inverse and one correction), to the nearest whole number.
__device__ __forceinline__ int code_of(double x, double scale, double inv) {
    double n = x * inv;
    n = fma(fma(-n, scale, x), inv, n);
    return min(max((int)rint(n), -127), 127);
}

// append_paged_kernel into codes and scales.  A row's d_head / 4 threads lie in one wave, next to each other, and find its largest value by exchanging theirs.
// Bound by memory, though half of the arithmetic is in 64 bits (vector unit 72% busy).  Measured: three tokens of 32 + 2 x 32 heads of 128 4.0 us (latency); 4099 tokens of 64 + 2 x 8
// heads, 168 MB read and 145 written, 63 us, 5.0 TB/s, a large copy's rate.
template <int U>
__global__ __launch_bounds__(NTP) void append_q8_kernel(const AppendQ8Args p) {
    const AppendArgs &a = p.a;
    __shared__ double2 turn[128];
    const int tid = threadIdx.x, t = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
    const int d = a.c.d_head, per_head = d / 4;
    const int q_end = a.n_heads * per_head, k_end = q_end + a.c.n_kv_heads * per_head, end = k_end + a.c.n_kv_heads * per_head;
    const int seq = as_global(a.seq)[t], pos = as_global(a.pos)[t];
    if (seq < 0) return;                                                              // padding
    float4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int at = (part * U + u) * NTP + tid;
        x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at < q_end) x[u] = global_load_float4(a.q + (size_t)t * a.q_stride + 4 * at);
        else if (at < k_end) x[u] = global_load_float4(a.k + (size_t)t * a.kv_stride + 4 * (at - q_end));
        else if (at < end) x[u] = global_load_float4(a.v + (size_t)t * a.kv_stride + 4 * (at - k_end));
    }
    if (seq >= a.c.n_seq || pos < 0 || (pos >> a.c.page_shift) >= a.c.table_stride) {
        if (tid == 0) flag(a.err);
        return;
    }
    const int page = as_global(a.c.table)[(size_t)seq * a.c.table_stride + (pos >> a.c.page_shift)];
    if (tid < d / 2) turn[tid] = rotation64(pos, tid, a.log2_theta, p.log2_theta_low, d);
    __syncthreads();
    if (!page_ok(a.c, page)) {
        if (tid == 0) flag(a.err);
        return;
    }
    const int page_size = 1 << a.c.page_shift, row = pos & (page_size - 1);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int at = (part * U + u) * NTP + tid;               // (threads past the end stay for the exchange)
        const bool is_q = at < q_end, turned = at < k_end;
        double y[4];
        const float in[4] = {is_q ? x[u].x : finite(x[u].x), is_q ? x[u].y : finite(x[u].y), is_q ? x[u].z : finite(x[u].z), is_q ? x[u].w : finite(x[u].w)};
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            const double2 c = turn[2 * (at % per_head) + e / 2];
            y[e] = turned ? fma((double)in[e], c.x, -((double)in[e + 1] * c.y)) : (double)in[e];
            y[e + 1] = turned ? fma((double)in[e], c.y, (double)in[e + 1] * c.x) : (double)in[e + 1];
        }
        if (is_q) store_four<float>(a.q_out, (size_t)t * q_end * 4 + 4 * at, make_float4((float)y[0], (float)y[1], (float)y[2], (float)y[3]));
        double top = fmax(fmax(fabs(y[0]), fabs(y[1])), fmax(fabs(y[2]), fabs(y[3])));
        for (int o = 1; o < per_head; o <<= 1) top = fmax(top, __shfl_xor(top, o, WAVE));
        if (is_q || at >= end) continue;
        const float scale = (float)(top / 127.0);
        const double inv = scale > 0.f ? 1.0 / (double)scale : 0.0;
        const int of = turned ? at - q_end : at - k_end, head = of / per_head;
        const size_t place = ((size_t)page * a.c.n_kv_heads + head) * page_size + row;
        uint32_t codes = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) codes |= (uint32_t)(code_of(y[e], (double)scale, inv) & 0xFF) << (8 * e);
        *(uint32_t __attribute__((address_space(1))) *)((int8_t *)(turned ? a.c.K : a.c.V) + place * d + 4 * (of % per_head)) = codes;
        if (of % per_head == 0) as_global(turned ? p.k_scale : p.v_scale)[place] = scale;
    }
}

hipError_t launch_append_q8(hipStream_t s, AppendQ8Args p) {
    bool few;
    const long long blocks = append_blocks(p.a, few);
    if (few) hipLaunchKernelGGL((append_q8_kernel<1>), dim3((unsigned)blocks), dim3(NTP), 0, s, p);
    else hipLaunchKernelGGL((append_q8_kernel<4>), dim3((unsigned)blocks), dim3(NTP), 0, s, p);
    return hipGetLastError();
}

// Eight elements of a row, as fp32 numbers.
template <typename KT> __device__ __forceinline__ void load_eight(const void *p, size_t i, float (&x)[8]) {
    const u32x4 v = global_load16((const KT *)p + i);
    Store<KT>::unpack(v, x);
}
template <> __device__ __forceinline__ void load_eight<float>(const void *p, size_t i, float (&x)[8]) {
    const float4 a = global_load_float4((const float *)p + i), b = global_load_float4((const float *)p + i + 4);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <> __device__ __forceinline__ void load_eight<q8_t>(const void *p, size_t i, float (&x)[8]) {
    const u32x2 v = *(const u32x2 __attribute__((address_space(1))) *)((const int8_t *)p + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)(int8_t)((e < 4 ? v.x : v.y) >> (8 * (e % 4)));
}

// A thread: U pieces of eight elements of a row, a block's width apart; a token's keys in front, then its values.  Places, page numbers and rows are three trips to memory, each of them
// asked for all pieces at once.  Measured: 60001 tokens of 2 x 8 heads of 128 from 8 to 16 bits, 404 MB in all, 88 us, 4.6 TB/s (a large copy: 5.0; one piece after the other, 1.4 times as long);
// twenty tokens of 2 x 32 heads 3.0 us (latency).
template <typename KT, typename OT, int U>
__global__ __launch_bounds__(NTP) void read_paged_kernel(const ReadArgs a) {
    const int d = a.c.d_head, row_pieces = a.c.n_kv_heads * d / 8, page_size = 1 << a.c.page_shift, pieces = a.n_tokens * 2 * row_pieces, i0 = blockIdx.x * (NTP * U) + threadIdx.x;
    int token[U], seq[U], pos[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        token[u] = over(min(i0 + u * NTP, pieces - 1), a.by_token);
        seq[u] = as_global(a.seq)[token[u]];
        pos[u] = as_global(a.pos)[token[u]];
    }
    int page[U];
    bool ok[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        ok[u] = (unsigned)seq[u] < (unsigned)a.c.n_seq && pos[u] >= 0 && (pos[u] >> a.c.page_shift) < a.c.table_stride;
        page[u] = ok[u] ? as_global(a.c.table)[(size_t)seq[u] * a.c.table_stride + (pos[u] >> a.c.page_shift)] : -1;
    }
    float x[U][8], scale[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        ok[u] = page_ok(a.c, page[u]);
        if (!ok[u]) {
            if (seq[u] >= 0) flag(a.err);        // (negative: padding)
            continue;
        }
        const int in_token = min(i0 + u * NTP, pieces - 1) - token[u] * 2 * row_pieces, at = 8 * (in_token >= row_pieces ? in_token - row_pieces : in_token);
        const bool is_v = in_token >= row_pieces;
        const size_t place = ((size_t)page[u] * a.c.n_kv_heads + at / d) * page_size + (pos[u] & (page_size - 1));
        load_eight<KT>(is_v ? a.c.V : a.c.K, place * d + at % d, x[u]);
        if constexpr (sizeof(KT) == 1) scale[u] = as_global(is_v ? a.v_scale : a.k_scale)[place];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (!ok[u] || i0 + u * NTP >= pieces) continue;
        if constexpr (sizeof(KT) == 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[u][e] *= scale[u];
                asm("" : "+v"(x[u][e]));         // (an fp32 number: a value is the same whatever type it is read in.  Product and conversion as one instruction round once)
            }
        }
        const int in_token = i0 + u * NTP - token[u] * 2 * row_pieces, at = 8 * (in_token >= row_pieces ? in_token - row_pieces : in_token);
        void *out = in_token >= row_pieces ? a.v_out : a.k_out;
        const size_t to = (size_t)token[u] * a.c.n_kv_heads * d + at;
        if constexpr (sizeof(OT) == 2) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = two_words<OT>(x[u][2 * e], x[u][2 * e + 1]);
            *(u32x4 __attribute__((address_space(1))) *)((uint16_t *)out + to) = w;
        } else {
            store_four<OT>(out, to, make_float4(x[u][0], x[u][1], x[u][2], x[u][3]));
            store_four<OT>(out, to + 4, make_float4(x[u][4], x[u][5], x[u][6], x[u][7]));
        }
    }
}

template <typename KT, typename OT>
hipError_t launch_read_as(hipStream_t s, ReadArgs a) {
    const int per_token = 2 * (a.c.n_kv_heads * a.c.d_head / 8), most = std::max(1, (1 << 30) / per_token), n = a.n_tokens;      // (pieces are counted in 31 bits)
    const size_t token_bytes = (size_t)a.c.n_kv_heads * a.c.d_head * sizeof(OT);
    a.by_token = divisor(per_token);
    for (int t = 0; t < n; t += most) {
        ReadArgs b = a;
        b.n_tokens = std::min(most, n - t);
        b.seq += t; b.pos += t;
        b.k_out = (char *)a.k_out + (size_t)t * token_bytes; b.v_out = (char *)a.v_out + (size_t)t * token_bytes;
        const long long pieces = (long long)b.n_tokens * per_token;
        // few pieces: one per thread, so that many blocks share the way to memory
        if (pieces < 4LL * NTP * 1024) hipLaunchKernelGGL((read_paged_kernel<KT, OT, 1>), dim3((unsigned)((pieces + NTP - 1) / NTP)), dim3(NTP), 0, s, b);
        else hipLaunchKernelGGL((read_paged_kernel<KT, OT, 4>), dim3((unsigned)((pieces + 4 * NTP - 1) / (4 * NTP))), dim3(NTP), 0, s, b);
    }
    return hipGetLastError();
}

template <typename KT>
hipError_t launch_read(hipStream_t s, const ReadArgs &a, int out_dtype) {
    return out_dtype == SPD_DTYPE_FP32 ? launch_read_as<KT, float>(s, a) : out_dtype == SPD_DTYPE_FP16 ? launch_read_as<KT, half_t>(s, a) : launch_read_as<KT, bf16_t>(s, a);
}

// What the beams of a group go on in, one lane per beam.  A row's first child keeps it; further children take the rows that
// got no child, in order (there are as many of them), so that every beam has a row -- and with it a page to write into
// next -- of its own, and no page has to be found or given back.
struct BeamRows {
    bool ok;              // the group's arguments hold
    int parent, row;      // per lane
    uint32_t further;     // beams that need their parent's unfinished page copied
};
__device__ __forceinline__ int nth_set_bit(uint32_t mask, int n) {
    for (; n > 0; --n) mask &= mask - 1;
    return __ffs((int)mask) - 1;
}
__device__ __forceinline__ BeamRows beam_rows(const ReorderArgs &a, int g, int lane) {
    const bool in = lane < a.width;
    BeamRows r;
    r.parent = in ? as_global(a.parents)[g * a.width + lane] : 0;
    const int len = in ? as_global(a.len)[g * a.width + lane] : as_global(a.len)[g * a.width];
    const int len0 = __builtin_amdgcn_readfirstlane(len);
    r.ok = !__any(len != len0 || (unsigned)r.parent >= (unsigned)a.width) && len0 >= 0 && (long long)len0 <= (long long)a.c.table_stride << a.c.page_shift;
    uint32_t living = 0;
    bool first = true;
    for (int i = 0; i < a.width; ++i) {
        const int p = __shfl(r.parent, i, WAVE);
        if (i < lane && p == r.parent) first = false;
        living |= 1u << (p & 31);
    }
    r.further = (uint32_t)__ballot(in && !first);
    const uint32_t spare = ~living & ((1u << a.width) - 1u);
    r.row = !in || first ? r.parent : nth_set_bit(spare, __popc(r.further & ((1u << lane) - 1u)));
    return r;
}

// Measured: two further children of 32 layers x 32 heads x 10 rows x 128 in fp16, 10.5 MB read and as much written, 6.9 us (parents and
// lengths, then page numbers, are two trips to memory before the copy's own); eight groups of five further children, 16 layers x 8 heads x some 40 rows x 128 in bf16,
// 109 MB each way, 44 us (4.9 TB/s, a large copy's rate).
// Blocks 0 .. groups - 1: a group's tables.  The others: (group, further child, layer, share of the key/value heads); where shared positions are
// given, one child more stands for the rows of a page on which they end, which the group's first sequence has to have.  Those rows are written on the page of
// its parent, the rows behind them are read from there and written elsewhere, and no page's rows in front are copied to: no block waits for another.
template <bool SHARED>
__global__ __launch_bounds__(NTP) void beam_reorder_kernel(const ReorderArgs a) {
    const int lane = threadIdx.x & (WAVE - 1), w = threadIdx.x / WAVE;
    const bool tables = (int)blockIdx.x < a.n_groups;
    int rest = blockIdx.x - a.n_groups;
    const int share = rest % a.shares;
    rest /= a.shares;
    const int layer = rest % a.n_layers;
    rest /= a.n_layers;
    const int child = tables ? 0 : rest % a.children, g = tables ? blockIdx.x : rest / a.children;
    const int page_size = 1 << a.c.page_shift;
    BeamRows r = beam_rows(a, g, lane);
    const int len = as_global(a.len)[g * a.width];
    const int entry = len >> a.c.page_shift, filled = len & (page_size - 1);
    const int32_t *table = a.c.table + (size_t)g * a.width * a.c.table_stride;
    // the pages being filled: each beam's own, or copying would spoil another's
    int page = lane;
    if (r.ok && filled && r.further) {
        if (lane < a.width) page = as_global(table)[(size_t)lane * a.c.table_stride + entry];
        bool good = lane >= a.width || page_ok(a.c, page);
        for (int i = 0; i < a.width; ++i) {
            const int p = __shfl(page, i, WAVE);
            if (lane < a.width && i != lane && p == page) good = false;
        }
        r.ok = !__any(!good);
    }
    // shared positions: whole pages of them, and rows on the page where they end, which pages `have` and `want` hold for the first sequence so far and from now on
    int whole = 0, tail = 0, have = 0, want = 0;
    if constexpr (SHARED) {
        const int shared = as_global(a.shared)[g], first = __shfl(r.parent, 0, WAVE);
        if (shared < 0 || (long long)shared > (long long)a.c.table_stride << a.c.page_shift) r.ok = false;
        if (r.ok) {
            whole = min(shared, len) >> a.c.page_shift;
            tail = min(shared, len) & (page_size - 1);
            if (tail && first) {
                have = as_global(table)[whole];
                want = as_global(table)[(size_t)first * a.c.table_stride + whole];
                r.ok = page_ok(a.c, have) && page_ok(a.c, want);
            }
        }
    }
    if (tables) {
        if (!r.ok && threadIdx.x == 0) flag(a.err);
        int32_t *out = a.table_out + (size_t)g * a.width * a.c.table_stride;
        for (int j = w; j < a.width; j += NTP / WAVE) {
            const int parent = r.ok ? __shfl(r.parent, j, WAVE) : j, row = r.ok ? __shfl(r.row, j, WAVE) : j;
            for (int e = lane; e < a.c.table_stride; e += WAVE)
                as_global(out)[(size_t)j * a.c.table_stride + e] = as_global(table)[(size_t)(SHARED && r.ok && e < whole ? 0 : e < entry ? parent : row) * a.c.table_stride + e];
        }
        return;
    }
    if (!r.ok) return;
    size_t from, to;
    int row0 = 0, row1 = filled;                             // rows of the page that are copied
    if (SHARED && child == a.width - 1) {
        if (have == want) return;
        from = (size_t)have; to = (size_t)want;
        row1 = tail;
    } else {
        if (!filled || child >= __popc(r.further)) return;
        const int j = nth_set_bit(r.further, child);
        from = (size_t)__shfl(page, __shfl(r.parent, j, WAVE), WAVE); to = (size_t)__shfl(page, __shfl(r.row, j, WAVE), WAVE);
        if (SHARED && whole == entry) row0 = tail;
        if (SHARED && row0 >= row1) return;
    }
    // 16-byte pieces: the rows of this share's heads, keys then values
    const size_t head_bytes = (size_t)page_size * a.row_bytes, page_bytes = head_bytes * a.c.n_kv_heads;
    const int per_head = (row1 - row0) * (a.row_bytes / 16), h0 = share * a.heads_per_share, h1 = min(a.c.n_kv_heads, h0 + a.heads_per_share);
    const int pieces = (h1 - h0) * per_head;
    const float by_head = 1.0f / (float)per_head;            // (at most 2^16 pieces: (p + 1/2) / per_head is never near a whole number)
    for (int i0 = threadIdx.x; i0 < 2 * pieces; i0 += COPIES * NTP) {
        u32x4 v[COPIES];
        char *to_at[COPIES];
#pragma unroll
        for (int u = 0; u < COPIES; ++u) {                   // asked for together: one trip to memory
            const int i = i0 + u * NTP;
            if (i >= 2 * pieces) break;
            const int p = i < pieces ? i : i - pieces, head = (int)(((float)p + 0.5f) * by_head);
            char *pool = (char *)(i < pieces ? a.c.K : a.c.V) + (size_t)layer * a.layer_bytes;
            const size_t at = (size_t)(h0 + head) * head_bytes + (size_t)row0 * a.row_bytes + 16 * (size_t)(p - head * per_head);
            v[u] = global_load16(pool + from * page_bytes + at);
            to_at[u] = pool + to * page_bytes + at;
        }
#pragma unroll
        for (int u = 0; u < COPIES; ++u)
            if (i0 + u * NTP < 2 * pieces) *(u32x4 __attribute__((address_space(1))) *)to_at[u] = v[u];
    }
}

}  // namespace

namespace spdk {

int paged_cache_status(int dtype, const PagedCache &c, int page_size) {
    if (dtype != SPD_DTYPE_FP32 && dtype != SPD_DTYPE_BF16 && dtype != SPD_DTYPE_FP16) return SPD_EINVAL;
    if (!c.K || !c.V || (!c.table && c.n_seq > 0) || ((uintptr_t)c.K | (uintptr_t)c.V) % 16 || (uintptr_t)c.table % 4) return SPD_EINVAL;
    if (c.n_pages <= 0 || c.n_kv_heads <= 0 || c.n_seq < 0 || c.table_stride <= 0) return SPD_EINVAL;
    if (page_size < 4 || page_size > 1024 || (page_size & (page_size - 1))) return SPD_EINVAL;
    if (c.d_head < 8 || c.d_head > 256 || (c.d_head & (c.d_head - 1))) return SPD_EINVAL;
    return SPD_OK;
}

int paged_cache_status(int dtype, const PagedCache &c, int page_size, const float *k_scale, const float *v_scale) {
    const bool q8 = dtype == SPD_DTYPE_INT8;
    if ((k_scale != nullptr) != q8 || (v_scale != nullptr) != q8 || ((uintptr_t)k_scale | (uintptr_t)v_scale) % 16) return SPD_EINVAL;
    return paged_cache_status(q8 ? SPD_DTYPE_FP32 : dtype, c, page_size);
}

PagedCache paged_cache(void *K, void *V, const int32_t *table, int n_pages, int n_kv_heads, int page_size, int d_head, int n_seq, int table_stride) {
    return PagedCache{K, V, table, n_pages, n_kv_heads, page_size > 0 ? __builtin_ctz((unsigned)page_size) : 0, d_head, n_seq, table_stride};
}

}  // namespace spdk

// What the two append operators look at: the arguments, and that what is written lies apart from what other blocks read.  (n_tokens 0: SPD_OK too, nothing to do.)
static int append_status(const AppendArgs &a, size_t pool, spdk::Span k_scale, spdk::Span v_scale, float rope_theta) {
    const PagedCache &c = a.c;
    const int64_t heads = (int64_t)a.n_heads * c.d_head, kv_heads = (int64_t)c.n_kv_heads * c.d_head;
    if (a.n_tokens < 0 || !(rope_theta > 0.f) || !(rope_theta < INFINITY) || a.n_heads < 0 || heads > (1 << 24) || kv_heads > (1 << 24)) return SPD_EINVAL;
    if (a.n_tokens == 0) return SPD_OK;
    if (!a.k || !a.v || !a.seq || !a.pos || a.kv_stride < kv_heads || a.kv_stride % 4 || ((uintptr_t)a.k | (uintptr_t)a.v) % 16) return SPD_EINVAL;
    if ((a.q == nullptr) != (a.q_out == nullptr) || (a.q == nullptr) != (a.n_heads == 0)) return SPD_EINVAL;
    if (a.q && (a.q_stride < heads || a.q_stride % 4 || ((uintptr_t)a.q | (uintptr_t)a.q_out) % 16)) return SPD_EINVAL;
    if (a.q == a.q_out && a.q && a.q_stride != heads) return SPD_EINVAL;
    const size_t out_bytes = (size_t)a.n_tokens * heads * 4, kv_bytes = ((size_t)(a.n_tokens - 1) * a.kv_stride + (size_t)kv_heads) * 4,
                 q_bytes = a.q ? ((size_t)(a.n_tokens - 1) * a.q_stride + (size_t)heads) * 4 : 0, ids = (size_t)a.n_tokens * 4;
    const spdk::Span sk{a.k, kv_bytes}, sv{a.v, kv_bytes}, sq{a.q, q_bytes}, st{c.table, (size_t)c.n_seq * c.table_stride * 4}, ss{a.seq, ids}, sp{a.pos, ids}, sK{c.K, pool}, sV{c.V, pool}, se{a.err, 4};
    if (spdk::over_any(spdk::Span{a.q_out, out_bytes}, {sk, sv, a.q == a.q_out ? spdk::Span{} : sq, st, ss, sp, sK, sV, k_scale, v_scale, se})) return SPD_EINVAL;
    if (spdk::over_any(sK, {sV, k_scale, v_scale, sk, sv, sq, st, ss, sp, se}) || spdk::over_any(sV, {k_scale, v_scale, sk, sv, sq, st, ss, sp, se})) return SPD_EINVAL;
    if (spdk::over_any(k_scale, {v_scale, sk, sv, sq, st, ss, sp, se}) || spdk::over_any(v_scale, {sk, sv, sq, st, ss, sp, se})) return SPD_EINVAL;
    return SPD_OK;
}

extern "C" int spd_op_append_paged(int32_t dtype, void *K, void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                                   int32_t d_head, int32_t n_seq, int32_t table_stride, const float *q, int64_t q_stride, const float *k, const float *v,
                                   int64_t kv_stride, const int32_t *seq, const int32_t *pos, int32_t n_tokens, int32_t n_heads, float rope_theta,
                                   float *q_out, int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache(K, V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    int rc = spdk::paged_cache_status(dtype, c, page_size);
    if (rc != SPD_OK) return rc;
    const AppendArgs a{c, q, k, v, q_stride, kv_stride, seq, pos, n_tokens, n_heads, 0, log2((double)rope_theta), q_out, err};
    rc = append_status(a, spdk::pool_bytes(dtype, c), {}, {}, rope_theta);
    if (rc != SPD_OK || n_tokens == 0) return rc;
    hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch_append<float>(s, a) : dtype == SPD_DTYPE_FP16 ? launch_append<half_t>(s, a) : launch_append<bf16_t>(s, a);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}

extern "C" int spd_op_append_paged_q8(int8_t *K, int8_t *V, float *K_scale, float *V_scale, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                                      int32_t d_head, int32_t n_seq, int32_t table_stride, const float *q, int64_t q_stride, const float *k, const float *v, int64_t kv_stride,
                                      const int32_t *seq, const int32_t *pos, int32_t n_tokens, int32_t n_heads, float rope_theta, float *q_out, int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache(K, V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    int rc = spdk::paged_cache_status(SPD_DTYPE_INT8, c, page_size, K_scale, V_scale);
    if (rc != SPD_OK) return rc;
    const double log2_theta = log2((double)rope_theta);
    AppendQ8Args p{{c, q, k, v, q_stride, kv_stride, seq, pos, n_tokens, n_heads, 0, log2_theta, q_out, err}, K_scale, V_scale, (double)(log2l((long double)rope_theta) - (long double)log2_theta)};
    const size_t scales = spdk::scale_bytes(c);
    rc = append_status(p.a, spdk::pool_bytes(SPD_DTYPE_INT8, c), {K_scale, scales}, {V_scale, scales}, rope_theta);
    if (rc != SPD_OK || n_tokens == 0) return rc;
    bool few;
    if (append_blocks(p.a, few) > UINT32_MAX / NTP) return SPD_EINVAL;           // (threads of a grid are counted in 32 bits)
    return launch_append_q8((hipStream_t)hip_stream, p) == hipSuccess ? SPD_OK : SPD_EHIP;
}

extern "C" int spd_op_read_paged(int32_t dtype, const void *K, const void *V, const float *K_scale, const float *V_scale, const int32_t *table, int32_t n_pages, int32_t n_kv_heads,
                                 int32_t page_size, int32_t d_head, int32_t n_seq, int32_t table_stride, const int32_t *seq, const int32_t *pos, int32_t n_tokens, int32_t out_dtype,
                                 void *k_out, void *v_out, int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache((void *)K, (void *)V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    const int rc = spdk::paged_cache_status(dtype, c, page_size, K_scale, V_scale);
    if (rc != SPD_OK) return rc;
    if (n_tokens < 0 || (out_dtype != SPD_DTYPE_FP32 && out_dtype != SPD_DTYPE_FP16 && out_dtype != SPD_DTYPE_BF16) || (int64_t)n_kv_heads * d_head > (1 << 24)) return SPD_EINVAL;
    if (n_tokens == 0) return SPD_OK;
    if (!seq || !pos || !k_out || !v_out || ((uintptr_t)k_out | (uintptr_t)v_out) % 16) return SPD_EINVAL;
    const size_t pool = spdk::pool_bytes(dtype, c), scales = spdk::scale_bytes(c), out = (size_t)n_tokens * n_kv_heads * d_head * (out_dtype == SPD_DTYPE_FP32 ? 4 : 2), ids = (size_t)n_tokens * 4;
    const spdk::Span so{k_out, out}, sw{v_out, out}, sK{K, pool}, sV{V, pool}, sk{K_scale, scales}, sv{V_scale, scales}, st{table, (size_t)n_seq * table_stride * 4}, ss{seq, ids}, sp{pos, ids}, se{err, 4};
    if (spdk::over_any(so, {sw, sK, sV, sk, sv, st, ss, sp, se}) || spdk::over_any(sw, {sK, sV, sk, sv, st, ss, sp, se})) return SPD_EINVAL;
    const ReadArgs a{c, K_scale, V_scale, seq, pos, n_tokens, k_out, v_out, err};
    hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch_read<float>(s, a, out_dtype) : dtype == SPD_DTYPE_FP16 ? launch_read<half_t>(s, a, out_dtype)
                         : dtype == SPD_DTYPE_BF16 ? launch_read<bf16_t>(s, a, out_dtype) : launch_read<q8_t>(s, a, out_dtype);
    return e == hipSuccess ? SPD_OK : SPD_EHIP;
}

// Whether any layer of a pool (pool bytes each, `apart` from one to the next) lies over o: the first layer that ends behind its beginning does, or none.
static bool over_layers(const void *base, size_t pool, size_t apart, int n_layers, const spdk::Span &o) {
    const uintptr_t b = (uintptr_t)base, at = (uintptr_t)o.p;
    const size_t l = at < b + pool ? 0 : (at - b - pool) / apart + 1;
    return l < (size_t)n_layers && spdk::overlap((const void *)(b + l * apart), pool, o.p, o.bytes);
}

static int reorder(int32_t dtype, void *K, void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                   int32_t d_head, int32_t n_seq, int32_t table_stride, int32_t n_layers, int64_t layer_stride, int32_t width,
                   const int32_t *parents, const int32_t *len, const int32_t *shared, int32_t *table_out, int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache(K, V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    const int rc = spdk::paged_cache_status(dtype, c, page_size);
    if (rc != SPD_OK) return rc;
    if (width < 1 || width > SPD_K_MAX || n_seq % width || n_layers < 1) return SPD_EINVAL;
    const int elem = dtype == SPD_DTYPE_FP32 ? 4 : 2;
    const int64_t layer_elems = (int64_t)n_pages * n_kv_heads * page_size * d_head;
    if (n_layers > 1 && (layer_stride < layer_elems || layer_stride % (16 / elem))) return SPD_EINVAL;
    if (n_seq == 0) return SPD_OK;
    if (!parents || !len || !table_out) return SPD_EINVAL;
    // what is written lies apart from what other blocks read (layers may lie in turn: a layer's keys, its values, the next layer's keys, other things between them)
    const size_t table_bytes = (size_t)n_seq * table_stride * 4, ids = (size_t)n_seq * 4, pool = spdk::pool_bytes(dtype, c), apart = n_layers > 1 ? (size_t)layer_stride * elem : pool;
    const spdk::Span st{table, table_bytes}, sp{parents, ids}, sl{len, ids}, sh{shared, (size_t)(n_seq / width) * 4}, so{table_out, table_bytes}, se{err, 4};
    if (spdk::over_any(so, {st, sp, sl, sh, se})) return SPD_EINVAL;
    for (const void *p : {(const void *)K, (const void *)V})
        for (const spdk::Span &o : {st, sp, sl, sh, so, se})
            if (o.p && over_layers(p, pool, apart, n_layers, o)) return SPD_EINVAL;
    const uintptr_t kp = (uintptr_t)K, vp = (uintptr_t)V;
    if (over_layers((const void *)std::min(kp, vp), pool, apart, n_layers, spdk::Span{(const void *)std::max(kp, vp), pool})) return SPD_EINVAL;      // (the others of its layers lie alike)
    ReorderArgs a{c, parents, len, shared, table_out, err, n_layers, width, n_seq / width, width == 1 ? 0 : width - 1 + (shared != nullptr), d_head * elem, 0, 0, (size_t)layer_stride * elem};
    // about 32 KB of keys and values per block
    a.heads_per_share = std::max(1, 16384 / (page_size * a.row_bytes));
    a.shares = (n_kv_heads + a.heads_per_share - 1) / a.heads_per_share;
    const long long blocks = a.n_groups + (long long)a.n_groups * a.children * n_layers * a.shares;
    if (blocks > INT32_MAX) return SPD_EINVAL;
    if (shared) hipLaunchKernelGGL(beam_reorder_kernel<true>, dim3((unsigned)blocks), dim3(NTP), 0, (hipStream_t)hip_stream, a);
    else hipLaunchKernelGGL(beam_reorder_kernel<false>, dim3((unsigned)blocks), dim3(NTP), 0, (hipStream_t)hip_stream, a);
    return hipGetLastError() == hipSuccess ? SPD_OK : SPD_EHIP;
}

extern "C" int spd_op_beam_reorder(int32_t dtype, void *K, void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                                   int32_t d_head, int32_t n_seq, int32_t table_stride, int32_t n_layers, int64_t layer_stride, int32_t width,
                                   const int32_t *parents, const int32_t *len, int32_t *table_out, int32_t *err, void *hip_stream) {
    return reorder(dtype, K, V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride, n_layers, layer_stride, width, parents, len, nullptr, table_out, err, hip_stream);
}

extern "C" int spd_op_beam_reorder_shared(int32_t dtype, void *K, void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                                          int32_t d_head, int32_t n_seq, int32_t table_stride, int32_t n_layers, int64_t layer_stride, int32_t width,
                                          const int32_t *parents, const int32_t *len, const int32_t *shared, int32_t *table_out, int32_t *err, void *hip_stream) {
    if (!shared && n_seq > 0) return SPD_EINVAL;
    return reorder(dtype, K, V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride, n_layers, layer_stride, width, parents, len, shared, table_out, err, hip_stream);
}
