// The paged key/value cache of a batch of sequences: appending new tokens (with the rotary
// positions applied on the way) and following a selection of beams.
//
// Both are bound by memory traffic where there is much to move and by latency where there is
// little.  What they need besides the data itself -- page numbers, angles, which row a beam goes
// on in -- is formed again by every block that uses it: it is a few dozen instructions, and a
// kernel of its own would cost a launch.
#include "spd_device.h"

#include <algorithm>

using namespace spdd;

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

template <typename KT>
hipError_t launch_append(hipStream_t s, AppendArgs a) {
    const long long pieces = (long long)(a.n_heads + 2 * a.c.n_kv_heads) * (a.c.d_head / 4);
    // few tokens: one piece per thread, so that many blocks share the way to memory; many: four, so that angles and page
    // numbers are formed for more of them
    const bool few = pieces * a.n_tokens < 4LL * NTP * 1024;
    const int u = few ? 1 : 4;
    a.parts = (int)((pieces + u * NTP - 1) / (u * NTP));
    const long long blocks = (long long)a.n_tokens * a.parts;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    if (few) hipLaunchKernelGGL((append_paged_kernel<KT, 1>), dim3((unsigned)blocks), dim3(NTP), 0, s, a);
    else hipLaunchKernelGGL((append_paged_kernel<KT, 4>), dim3((unsigned)blocks), dim3(NTP), 0, s, a);
    return hipGetLastError();
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

PagedCache paged_cache(void *K, void *V, const int32_t *table, int n_pages, int n_kv_heads, int page_size, int d_head, int n_seq, int table_stride) {
    return PagedCache{K, V, table, n_pages, n_kv_heads, page_size > 0 ? __builtin_ctz((unsigned)page_size) : 0, d_head, n_seq, table_stride};
}

}  // namespace spdk

extern "C" int spd_op_append_paged(int32_t dtype, void *K, void *V, const int32_t *table, int32_t n_pages, int32_t n_kv_heads, int32_t page_size,
                                   int32_t d_head, int32_t n_seq, int32_t table_stride, const float *q, int64_t q_stride, const float *k, const float *v,
                                   int64_t kv_stride, const int32_t *seq, const int32_t *pos, int32_t n_tokens, int32_t n_heads, float rope_theta,
                                   float *q_out, int32_t *err, void *hip_stream) {
    const PagedCache c = spdk::paged_cache(K, V, table, n_pages, n_kv_heads, page_size, d_head, n_seq, table_stride);
    const int rc = spdk::paged_cache_status(dtype, c, page_size);
    if (rc != SPD_OK) return rc;
    if (n_tokens < 0 || !(rope_theta > 0.f) || !(rope_theta < INFINITY) || n_heads < 0 || (long long)n_heads * d_head > (1 << 24) || (long long)n_kv_heads * d_head > (1 << 24)) return SPD_EINVAL;
    if (n_tokens == 0) return SPD_OK;
    if (!k || !v || !seq || !pos || kv_stride < (int64_t)n_kv_heads * d_head || kv_stride % 4 || ((uintptr_t)k | (uintptr_t)v) % 16) return SPD_EINVAL;
    if ((q == nullptr) != (q_out == nullptr) || (q == nullptr) != (n_heads == 0)) return SPD_EINVAL;
    if (q && (q_stride < (int64_t)n_heads * d_head || q_stride % 4 || ((uintptr_t)q | (uintptr_t)q_out) % 16)) return SPD_EINVAL;
    if (q == q_out && q && q_stride != (int64_t)n_heads * d_head) return SPD_EINVAL;
    // what is written lies apart from what other blocks read
    const size_t out_bytes = (size_t)n_tokens * n_heads * d_head * 4, kv_bytes = ((size_t)(n_tokens - 1) * kv_stride + (size_t)n_kv_heads * d_head) * 4,
                 q_bytes = q ? ((size_t)(n_tokens - 1) * q_stride + (size_t)n_heads * d_head) * 4 : 0, pool = spdk::pool_bytes(dtype, c), ids = (size_t)n_tokens * 4;
    const spdk::Span sk{k, kv_bytes}, sv{v, kv_bytes}, sq{q, q_bytes}, st{table, (size_t)n_seq * table_stride * 4}, ss{seq, ids}, sp{pos, ids}, sK{K, pool}, sV{V, pool}, se{err, 4};
    if (spdk::over_any(spdk::Span{q_out, out_bytes}, {sk, sv, q == q_out ? spdk::Span{} : sq, st, ss, sp, sK, sV, se}) || spdk::over_any(sK, {sV, sk, sv, sq, st, ss, sp, se}) ||
        spdk::over_any(sV, {sk, sv, sq, st, ss, sp, se})) return SPD_EINVAL;
    AppendArgs a{c, q, k, v, q_stride, kv_stride, seq, pos, n_tokens, n_heads, 0, log2((double)rope_theta), q_out, err};
    hipStream_t s = (hipStream_t)hip_stream;
    const hipError_t e = dtype == SPD_DTYPE_FP32 ? launch_append<float>(s, a) : dtype == SPD_DTYPE_FP16 ? launch_append<half_t>(s, a) : launch_append<bf16_t>(s, a);
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
